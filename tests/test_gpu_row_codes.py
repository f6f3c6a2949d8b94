"""Codes and scales of keys that lie next to a line between two scales, or that 32 bits do not hold: those of the row in 64 bits, whatever lies beside it."""
import numpy as np
import pytest
import torch

from oracle import layer_ops as L
from oracle import streaming_attention as O
from rows_helpers import f64, spec_of
from test_gpu_cache_rows import DEV, cache_of, gen, pair, read, stored

EPS = 1.0e-6


@pytest.fixture(scope="module")
def st():
    import paper_2510_17238_amd as st
    return st


# Rows m, -m, na times a, nb times b, then zeros (weight 1): normalised, m is within 4 * 2^-24 of itself under a line between two scales -- the last
# value that rounds to 1.5 (4 bits) or 1.75 (8 bits) times a power of two.
TIES = {("mxfp4", 64): [(1.6640625, 0.158203125, 20, 0.58203125, 40), (1.25, 0.80859375, 52, 0.94140625, 8), (1.265625, 0.2734375, 33, 0.49609375, 23)],
        ("mxfp4", 128): [(1.8671875, 0.205078125, 111, 0.23046875, 13), (1.9375, 1.90625, 56, 0.150390625, 64), (1.6015625, 0.392578125, 66, 0.6015625, 58)],
        ("fp8", 64): [(1.9140625, 1.15625, 51, 0.28125, 9), (1.6875, 0.1591796875, 2, 0.40234375, 56), (1.484375, 0.365234375, 38, 0.33203125, 18)],
        ("fp8", 128): [(1.2265625, 0.9609375, 64, 0.1533203125, 21), (1.15625, 0.2421875, 75, 0.455078125, 33), (1.5625, 0.2470703125, 17, 0.1259765625, 27)]}


def tie(d, m, a, na, b, nb):
    x = np.zeros(d)
    x[0], x[1], x[2:2 + na], x[2 + na:2 + na + nb] = m, -m, a, b
    return x


def scales(store, x):
    """2^k of every row (8 bits) or block (4 bits)."""
    if store == "fp8":
        return 2.0 ** O.quantize_rows_e4m3(x)[1]
    return 2.0 ** L.block_exponent(np.abs(x.reshape(*x.shape[:-1], -1, 32)).max(-1), 6.0)


def stored_scales(store, c, b, n):
    """The same, as the cache holds them for the first n keys of sequence b: [n, heads] or [n, heads, blocks]."""
    page = c.page_table[b].long()
    if store == "fp8":
        return f64(c.k_scale[page].permute(0, 2, 1).reshape(-1, c.n_kv_heads))[:n]
    blocks = c.head_dim // 32
    x = c.k_scale[page][..., :c.head_dim // 2].reshape(-1, c.n_kv_heads, blocks, 16).permute(0, 3, 1, 2).reshape(-1, c.n_kv_heads, blocks)
    return 2.0 ** (x[:n].cpu().numpy().astype(np.float64) - 127)


@pytest.mark.gpu
@pytest.mark.parametrize("store,d", list(TIES))
@pytest.mark.parametrize("n", [1, 7, 35])
@pytest.mark.parametrize("beside", ["zeros", "others"])
def test_largest_values_of_both_signs_next_to_a_line(st, store, d, n, beside):
    """Without rotation anywhere, and rotated by position 0."""
    batch, hkv = 3, 2
    for turned in (False, True):
        x = np.zeros((batch, n, hkv, d))
        if beside == "others":
            x = f64(torch.randn((batch, n, hkv, d), generator=gen(31), device=DEV).to(torch.bfloat16))
        for i, t in enumerate((0,) if turned else range(0, n, 3)):
            for b in range(batch):
                x[b, t, (i + b) % hkv] = tie(d, *TIES[store, d][(i + b) % 3]) * (-1.0) ** i
        k = torch.from_numpy(x).to(torch.bfloat16).to(DEV)
        assert np.array_equal(f64(k), x)
        spec, rope = spec_of(st, dim=d)
        c, _ = cache_of(st, np.random.default_rng(31), store, batch, -(-n // 16), hkv, d)
        w = torch.ones(d, dtype=torch.bfloat16, device=DEV)
        st.st_kv_append_norm_rope(pair(st, c), st.ST_SOURCE, k, k, w, spec if turned else None, eps=EPS)
        got, _ = read(st, pair(st, c), st.ST_SOURCE, batch, n)
        for b in range(batch):
            y = L.normalise(x[b], np.ones(d), EPS)
            y = L.bf16(L.rotate(y, np.arange(n), *rope) if turned else y)
            assert np.array_equal(f64(got[b]), stored(store, y)), (turned, b)
            assert np.array_equal(stored_scales(store, c, b, n), scales(store, y)), (turned, b)


@pytest.mark.gpu
@pytest.mark.parametrize("store", ["bf16", "fp8", "mxfp4"])
@pytest.mark.parametrize("d,n", [(64, 1), (128, 21)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_huge_keys_without_a_weight(st, store, d, n, layout):
    """Keys whose products pass 2^128 on the way and whose rotation, times an attention factor of a half, does not."""
    spec, rope = spec_of(st, dim=d, layout=layout, attention=0.5, rotary=32)
    x = torch.randn((2, n, 2, d), generator=gen(32), device=DEV).to(torch.bfloat16)
    lo, hi = L._pairs(32, layout)
    for i, (p, q) in enumerate(((1.0, 1.0), (1.5, -1.0), (-1.25, 1.5), (1.0, 0.0))):
        x[0, i * 5 % n, i % 2, int(lo[3 * i])], x[0, i * 5 % n, i % 2, int(hi[3 * i])] = p * 2.0 ** 127, q * 2.0 ** 127
    c, _ = cache_of(st, np.random.default_rng(32), store, 2, 2, 2, d)
    st.st_kv_append_norm_rope(pair(st, c), st.ST_SOURCE, x, x, None, spec)
    got, _ = read(st, pair(st, c), st.ST_SOURCE, 2, n)
    y = np.stack([L.bf16(L.rotate(f64(x)[b], np.arange(n), *rope)) for b in range(2)])
    assert np.abs(y).max() < 2.0 ** 127
    assert np.array_equal(f64(got), stored(store, y))
