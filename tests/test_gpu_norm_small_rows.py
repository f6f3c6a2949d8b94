"""Rows whose squares 32 bits do not hold, with little or no eps to hide it: norm + rotation and its gradients as for any other row."""
import numpy as np
import pytest
import torch

from oracle import layer_ops as L
from rows_helpers import f64, spec_of
from test_gpu_norm_rope import DEV, DT, FWD_UNITS, HALF_STEP, U24, check_bwd, check_fwd, inputs

# sizes of the rows: squares below the least fp32 number, just above it, past the largest, and ordinary ones among them
SIZES = [2.0 ** -80, 1.0, 2.0 ** -73, 2.0 ** 100, 2.0 ** -62, 2.0 ** 62, 2.0 ** -100]


@pytest.fixture(scope="module")
def st():
    import paper_2510_17238_amd as st
    return st


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,n,hq,hkv,d", [("bf16", 1, 7, 2, 128), ("bf16", 50, 4, 2, 64), ("f32", 31, 3, 1, 128), ("f32", 2100, 2, 2, 64)])
@pytest.mark.parametrize("eps", [0.0, 1.0e-48, 1.0e-60])
def test_rows_of_any_size(st, dtype, n, hq, hkv, d, eps):
    q, k, wq, wk, pos = inputs(dtype, n, hq, hkv, d, False, 41)
    for x in (q, k):
        x *= torch.tensor(np.resize(SIZES, x.shape[0] * x.shape[1]), device=DEV).view(x.shape[0], x.shape[1], 1).to(DT[dtype])
    sp, rope = spec_of(st, dim=d, rotary=32)
    q_out, k_out = st.st_norm_rope_apply_qk(q, k, wq, wk, pos, sp, eps=eps)
    check_fwd(q_out, q, wq, pos, eps, rope, dtype)
    check_fwd(k_out, k, wk, pos, eps, rope, dtype)
    gq, gk = torch.randn_like(q_out), torch.randn_like(k_out)
    dq, dk, dwq, dwk = st.st_norm_rope_bwd_qk(gq, gk, q, k, wq, wk, pos, sp, eps=eps)
    check_bwd(dq, dwq, gq, q, wq, pos, eps, rope, dtype)
    check_bwd(dk, dwk, gk, k, wk, pos, eps, rope, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_the_least_numbers(st, dtype):
    """Subnormal rows, whose inverse root is past the largest fp32 number."""
    d = 128
    q, _, wq, _, pos = inputs(dtype, 9, 2, 1, d, False, 42)
    q = (torch.sign(q.float()) * 2.0 ** -131).to(DT[dtype])
    sp, rope = spec_of(st)
    out, _ = st.st_norm_rope_apply_qk(q, None, wq, None, pos, sp, eps=0.0)
    check_fwd(out, q, wq, pos, 0.0, rope, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_zero_rows(st, dtype):
    """Zero rows stay zero under an eps that 32 bits do not hold, with gradients g w / sqrt(eps); without eps they are undefined, as 0 / 0 is."""
    q, _, wq, _, pos = inputs(dtype, 5, 4, 1, 64, False, 43)
    q[:, 1] = 0.0
    sp, rope = spec_of(st, dim=64)
    out, _ = st.st_norm_rope_apply_qk(q, None, wq, None, pos, sp, eps=1.0e-50)
    assert bool((out[:, 1] == 0.0).all())
    check_fwd(out, q, wq, pos, 1.0e-50, rope, dtype)
    g = torch.randn_like(out)
    dq, _, dw, _ = st.st_norm_rope_bwd_qk(g, None, q, None, wq, None, pos, sp, eps=1.0e-50)
    check_bwd(dq, dw, g, q, wq, pos, 1.0e-50, rope, dtype)
    out, _ = st.st_norm_rope_apply_qk(q, None, wq, None, pos, sp, eps=0.0)
    assert bool(torch.isnan(out[:, 1]).all()) and bool(torch.isfinite(out[:, [0, 2, 3]].float()).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_eps_past_32_bits(st, dtype):
    """An eps that 32 bits do not hold from above: rows of its size."""
    q, _, wq, _, pos = inputs(dtype, 6, 2, 1, 128, False, 44)
    q *= 2.0 ** 70
    sp, rope = spec_of(st)
    for eps in (1.0e42, 1.0e39):
        out, _ = st.st_norm_rope_apply_qk(q, None, wq, None, pos, sp, eps=eps)
        check_fwd(out, q, wq, pos, eps, rope, dtype)
