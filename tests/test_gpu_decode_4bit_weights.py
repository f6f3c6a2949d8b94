"""4-bit decode: the softmax weights lose nothing to bf16 on their way into the value product."""
import numpy as np
import pytest
import torch

from rows_helpers import f64
from test_gpu_decode_4bit import DEV, HALF, U24, decode, make


@pytest.fixture(scope="module")
def st():
    import paper_2510_17238_amd as st
    return st


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d,q_len", [(2, 2, 128, 1), (4, 1, 64, 1), (8, 1, 128, 1), (7, 1, 64, 1), (8, 2, 128, 4), (9, 1, 64, 1), (16, 1, 128, 1), (8, 2, 128, 8), (17, 1, 64, 1)])
@pytest.mark.parametrize("n_src,n_rsn", [(40, 70), (400, 500), (1500, 2100), (3, 5000)])
def test_weights_in_full(st, hq, hkv, d, q_len, n_src, n_rsn):
    """A weight goes in as two bf16 numbers, the second what the first left: half a step of half a step, 2^-16 of it, is lost.  The other terms: a score in 32
    bits (d + 4 roundings of its terms, 4 of itself, two steps of the function), the sums of weights and products in 32 bits (64 + N / 16 a lane), the result rounded
    once.  Values of either sign: the result is small beside them, and weights of one bf16 number are outside."""
    dual, rows = make(st, 90 + hq, 1, hkv, d, n_src, n_rsn, [n_src], [n_rsn])
    q = torch.randn((1, q_len, hq, d), generator=torch.Generator(device=DEV).manual_seed(91), device=DEV).to(torch.bfloat16)
    out, _ = decode(st, q, dual, [n_src], [n_rsn])
    out, q, scale = f64(out), f64(q), d ** -0.5
    worst = 0.0
    for t in range(q_len):
        seen = n_rsn - q_len + t + 1
        k, v = (np.concatenate([rows[0][i][0], rows[1][i][0, :seen]]) for i in (0, 1))
        for h in range(hq):
            kk, vv, x = k[:, h // (hq // hkv)], v[:, h // (hq // hkv)], q[0, t, h]
            s = kk @ x * scale
            delta = ((d + 4) * (np.abs(kk) @ np.abs(x)) * scale + 4 * np.abs(s) + 4).max() * U24
            p = np.exp(s - s.max())
            ref, mag = p @ vv / p.sum(), p @ np.abs(vv) / p.sum()
            bound = HALF * np.abs(ref) * (1 + HALF) + (2.0 ** -16 + 2 * delta + 2 * (64 + len(kk) / 16) * U24) * mag * (1 + HALF)
            worst = max(worst, float((np.abs(out[0, t, h] - ref) / bound).max()))
    assert worst <= 1.0, worst


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d,q_len", [(2, 2, 128, 1), (4, 1, 64, 1), (8, 2, 128, 4), (16, 1, 128, 1), (8, 2, 128, 8), (17, 1, 64, 1)])
@pytest.mark.parametrize("n_src,n_rsn", [(512, 256), (512, 2048)])
def test_large_values_under_rising_scores(st, hq, hkv, d, q_len, n_src, n_rsn):
    """Values of 2^115 and -2^115, scores that rise by 7.5 powers of two once a wave has seen its first 64 tokens.  Relative to the largest score, all 2,560 of them add up to
    less than 2^127; relative to the first, 64 of them to more than 2^128.  The result is the value itself: what is lost of weights and sums, below 2^-14, rounds to it or to
    the next bf16 number below, half a step."""
    dual, _ = make(st, 5, 1, hkv, d, n_src, n_rsn, [0], [0])
    sign = torch.where(torch.arange(d, device=DEV) % 3 == 0, -1.0, 1.0)
    for which, n, first in ((st.ST_SOURCE, n_src, 0), (st.ST_REASONING, n_rsn, 256)):
        k = torch.zeros((1, n, hkv, d), dtype=torch.bfloat16, device=DEV)
        k[:, :, :, 0] = (2.0 * (torch.arange(n, device=DEV) % 512 >= first)).to(torch.bfloat16)[None, :, None]
        v = (sign * 2.0 ** 115).to(torch.bfloat16).expand(1, n, hkv, d).contiguous()
        st.st_kv_append(dual, which, k, v)
    q = torch.zeros((1, q_len, hq, d), dtype=torch.bfloat16, device=DEV)
    q[..., 0] = 7.5 / 2 * np.log(2.0) * d ** 0.5
    out, _ = decode(st, q, dual, [n_src], [n_rsn], unit_tokens=512)
    assert float((out.double() / (sign.double() * 2.0 ** 115) - 1.0).abs().max()) <= HALF
