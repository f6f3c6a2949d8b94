"""Gradients of the norm's weights against a bound that follows the order of the sums, tight enough that a lost token would show."""
import numpy as np
import pytest
import torch

from oracle import layer_ops as L
from rows_helpers import f64, spec_of
from test_gpu_norm_rope import FWD_UNITS, U24, inputs, spread


@pytest.fixture(scope="module")
def st():
    import paper_2510_17238_amd as st
    return st


def additions(n, heads, all_heads, d):
    """Sums in 32 bits that a row goes through: a lane's rows one after the other (a step's rows are dealt out to the 256 / (d / 8) lane groups, a
    workgroup of at most 1,024 walks several steps); the lane groups are added up in 64 bits and rounded once."""
    groups = 256 // (d // 8)
    tokens = 1
    while tokens < 32 and tokens * all_heads < 4 * groups and n >= 2 * tokens * 1024:
        tokens *= 2
    steps = -(-n // tokens)
    lane = -(-steps // min(steps, 1024)) * -(-tokens * heads // groups)
    return lane + 1


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,n,hq,hkv,d,fused", [("f32", 1, 5, 1, 128, False), ("f32", 1801, 16, 8, 128, True), ("bf16", 5003, 16, 8, 128, True), ("f32", 4100, 4, 2, 64, True),
                                                    ("f32", 17003, 3, 1, 64, False), ("bf16", 33001, 1, 1, 64, True), ("bf16", 9001, 3, 1, 128, True)])
def test_every_token_counts(st, dtype, n, hq, hkv, d, fused):
    q, k, wq, wk, pos = inputs(dtype, n, hq, hkv, d, fused, 51)
    sp, (freq, a, layout) = spec_of(st, dim=d, rotary=32)
    gq, gk = (torch.randn(x.shape, device=x.device).to(x.dtype) for x in (q, k))
    _, _, dwq, dwk = st.st_norm_rope_bwd_qk(gq, gk, q, k, wq, wk, pos, sp, eps=1.0e-5)
    for dw, g, x, w in ((dwq, gq, q, wq), (dwk, gk, k, wk)):
        g64, x64 = f64(g), f64(x)
        turned, r = L.rotate(g64, f64(pos), freq, a, layout, back=True), 1.0 / np.sqrt((x64 * x64).mean(-1, keepdims=True) + np.float32(1.0e-5))
        term, size = turned * x64 * r, a * spread(g64, freq, layout) * np.abs(x64) * r
        # a term: the rotated gradient and r, whose roundings are the forward's, and two products; then the sums; then the rounding from 64 bits
        bound = (FWD_UNITS + 4 + additions(n, x.shape[1], hq + hkv, d) + 1) * U24 * size.sum((0, 1))
        ref = term.sum((0, 1))
        assert (np.abs(f64(dw) - ref) <= bound).all(), float((np.abs(f64(dw) - ref) / bound).max())
        # without its first or its last token, or the last row of that, the same sum is outside
        for lost in (term[0].sum(0), term[-1].sum(0), term[-1, -1]):
            assert (np.abs(lost) > 2 * bound).any()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,heads", [(128, 16), (64, 32)])
def test_small_rows_between_large_ones(st, dtype, d, heads):
    """One token whose heads are one row for each lane group: gradients 1 and -1 in the first and the last row, 2^-26 between them, x of size 1.  All terms are exact (but
    for r, one factor of them all), and so is their sum in 64 bits; in 32 a row beside a large one is lost."""
    t = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    sp, _ = spec_of(st, dim=d)
    sign = torch.where(torch.arange(d, device="cuda") % 3 == 0, -1.0, 1.0)
    x = sign.expand(1, heads, d).to(t).contiguous()
    g = torch.full((1, heads, d), 2.0 ** -26, device="cuda")
    g[0, 0], g[0, -1] = 1.0, -1.0
    w, pos = torch.ones(d, device="cuda", dtype=t), torch.zeros(1, dtype=torch.int32, device="cuda")
    _, _, dwq, dwk = st.st_norm_rope_bwd_qk(g.to(t), g.to(t), x, x, w, w, pos, sp, eps=0.0)
    ref = (heads - 2) * 2.0 ** -26 * f64(sign)
    for dw in (dwq, dwk):
        assert (np.abs(f64(dw) - ref) <= 4 * U24 * np.abs(ref)).all(), f64(dw) / ref
