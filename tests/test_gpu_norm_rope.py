"""Heads normalised and rotated in one pass, and the gradients of that pass, against the formulas in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import layer_ops as L
from rows_helpers import f64, spec_of

DEV = "cuda"
U24 = 2.0 ** -24
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def st():
    import paper_2510_17238_amd as st
    return st


def inputs(dtype, n, hq, hkv, d, fused, seed, most=5000):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rand = lambda *shape: torch.randn(shape, generator=g, device=DEV)
    if fused:
        x = (rand(n, hq + 2 * hkv, d) * 1.7).to(DT[dtype])
        q, k = x[:, :hq], x[:, hq:hq + hkv]
    else:
        q, k = (rand(n, hq, d) * 1.7).to(DT[dtype]), (rand(n, hkv, d) * 0.4).to(DT[dtype])
    wq, wk = ((1.0 + 0.3 * rand(d)).to(DT[dtype]) for _ in range(2))
    pos = torch.randint(0, most, (n,), generator=g, device=DEV, dtype=torch.int32)
    return q, k, wq, wk, pos


def spread(y, freq, layout):
    """|y| of every dim plus |y| of its rotation partner: what an fp32 rotation's error is relative to."""
    lo, hi = L._pairs(2 * len(freq), layout)
    out = np.abs(y)
    both = out[..., lo] + out[..., hi]
    out[..., lo] = both
    out[..., hi] = both
    return out


# fp32 arithmetic of a result, in units of 2^-24 of its terms: a sum of 8 products and 3 or 4 more sums, halved by the root (6), the root (2), two
# products (2), cos and sin (an angle of up to pi rounded to 24 bits, 4; two steps of the function, 4; the factor, 1), the rotation (3)
FWD_UNITS = 22


def check_fwd(out, x, w, pos, eps, rope, dtype):
    n = L.normalise(f64(x), f64(w), eps)
    ref = L.rotate(n, f64(pos), *rope)
    bound = HALF_STEP[dtype] * np.abs(ref) + FWD_UNITS * U24 * rope[1] * spread(n, rope[0], rope[2])
    err = np.abs(f64(out) - ref)
    assert (err <= bound * (1 + HALF_STEP[dtype])).all(), float((err / np.maximum(bound, 1e-300)).max())


def check_bwd(dx, dw, g, x, w, pos, eps, rope, dtype):
    g64, x64, w64 = f64(g), f64(x), f64(w)
    ref, ref_w = L.norm_rope_bwd(g64, x64, w64, f64(pos), eps, *rope)
    h = L.rotate(g64, f64(pos), rope[0], rope[1], rope[2], back=True)
    around = rope[1] * spread(g64, rope[0], rope[2])
    if w is None:
        bound = HALF_STEP[dtype] * np.abs(ref) + 16 * U24 * around
    else:
        r = 1.0 / np.sqrt((x64 * x64).mean(-1, keepdims=True) + eps)
        terms = r * around * np.abs(w64) + np.abs(x64) * r ** 3 * (around * np.abs(w64 * x64)).mean(-1, keepdims=True)
        # the forward's units, the sum over the row (12) and r squared (8), the products that join them (5)
        bound = HALF_STEP[dtype] * np.abs(ref) + (FWD_UNITS + 25) * U24 * terms
        # rows a lane adds up one after the other, of which there are at most all; then 64 lane groups and 1,024 workgroups pairwise or 16 deep
        rows = x64.shape[0] * x64.shape[1]
        bound_w = (FWD_UNITS + 4 + min(rows, 2 + rows // 16) + 40) * U24 * (around * np.abs(x64) * r).sum((0, 1))
        if dw is not None:
            assert (np.abs(f64(dw) - ref_w) <= bound_w).all(), float((np.abs(f64(dw) - ref_w) / bound_w).max())
    err = np.abs(f64(dx) - ref)
    assert (err <= bound * (1 + HALF_STEP[dtype])).all(), float((err / np.maximum(bound, 1e-300)).max())


CASES = [
    # dtype, tokens, q heads, kv heads, dim, fused, spec
    ("bf16", 1, 32, 8, 128, True, {}),
    ("f32", 1, 1, 1, 64, False, {}),
    ("bf16", 2, 16, 2, 64, True, dict(layout="interleaved")),
    ("bf16", 33, 5, 1, 128, False, dict(rotary=96)),
    ("f32", 67, 16, 8, 128, True, dict(rotary=32, scaling="linear", factor=2.5)),
    ("f32", 129, 8, 4, 64, False, dict(rotary=16, layout="interleaved", scaling="ntk", factor=4.0)),
    ("bf16", 700, 7, 7, 64, False, dict(rotary=48, scaling="yarn", factor=8.0, original=4096)),
    ("f32", 301, 3, 1, 128, True, dict(scaling="yarn", factor=4.0, original=32768, layout="interleaved")),
    ("bf16", 5003, 16, 8, 128, True, dict(rotary=64, scaling="yarn", factor=4.0, original=32768, attention=0.75)),
    ("f32", 4100, 4, 2, 64, True, dict(rotary=32)),
    ("bf16", 2500, 1, 1, 64, False, dict(theta=1.0e4)),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,n,hq,hkv,d,fused,spec", CASES)
def test_forward_and_gradients(st, dtype, n, hq, hkv, d, fused, spec):
    q, k, wq, wk, pos = inputs(dtype, n, hq, hkv, d, fused, 7 * n + d)
    sp, rope = spec_of(st, dim=d, **spec)
    eps = 1.0e-5
    q_out, k_out = st.st_norm_rope_apply_qk(q, k, wq, wk, pos, sp, eps=eps)
    check_fwd(q_out, q, wq, pos, np.float32(eps), rope, dtype)
    check_fwd(k_out, k, wk, pos, np.float32(eps), rope, dtype)
    gq, gk = torch.randn_like(q_out), torch.randn_like(k_out)
    dq, dk, dwq, dwk = st.st_norm_rope_bwd_qk(gq, gk, q, k, wq, wk, pos, sp, eps=eps)
    check_bwd(dq, dwq, gq, q, wq, pos, np.float32(eps), rope, dtype)
    check_bwd(dk, dwk, gk, k, wk, pos, np.float32(eps), rope, dtype)
    again = st.st_norm_rope_bwd_qk(gq, gk, q, k, wq, wk, pos, sp, eps=eps)
    assert all(torch.equal(a, b) for a, b in zip((dq, dk, dwq, dwk), again))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,n,hq,hkv,d,fused,spec", [
    ("bf16", 33001, 1, 1, 64, True, dict(rotary=32)),               # 32 tokens a step of the backward pass, the last one short
    ("f32", 17003, 3, 1, 64, False, dict(layout="interleaved")),    # 16
    ("bf16", 9001, 3, 1, 128, True, dict(rotary=112)),              # 8
])
def test_few_heads_of_many_tokens(st, dtype, n, hq, hkv, d, fused, spec):
    test_forward_and_gradients(st, dtype, n, hq, hkv, d, fused, spec)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d,norm_q,norm_k", [("bf16", 128, False, True), ("f32", 64, True, False), ("bf16", 64, False, False)])
def test_without_weights(st, dtype, d, norm_q, norm_k):
    q, k, wq, wk, pos = inputs(dtype, 85, 6, 3, d, False, 11)
    wq, wk = wq if norm_q else None, wk if norm_k else None
    sp, rope = spec_of(st, dim=d, rotary=32)
    q_out, k_out = st.st_norm_rope_apply_qk(q, k, wq, wk, pos, sp)
    check_fwd(q_out, q, wq, pos, np.float32(1e-6), rope, dtype)
    check_fwd(k_out, k, wk, pos, np.float32(1e-6), rope, dtype)
    gq, gk = torch.randn_like(q_out), torch.randn_like(k_out)
    dq, dk, dwq, dwk = st.st_norm_rope_bwd_qk(gq, gk, q if norm_q else None, k if norm_k else None, wq, wk, pos, sp)
    assert (dwq is not None, dwk is not None) == (norm_q, norm_k)
    check_bwd(dq, dwq, gq, q, wq, pos, np.float32(1e-6), rope, dtype)
    check_bwd(dk, dwk, gk, k, wk, pos, np.float32(1e-6), rope, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_queries_alone_in_place_and_slices(st, dtype):
    n, hq, hkv, d = 77, 8, 2, 128
    q, k, wq, wk, pos = inputs(dtype, n, hq, hkv, d, True, 3)
    sp, rope = spec_of(st)
    q_out, k_out = st.st_norm_rope_apply_qk(q, k, wq, wk, pos, sp)
    alone, none = st.st_norm_rope_apply_qk(q, None, wq, None, pos, sp)
    assert none is None and torch.equal(alone, q_out)
    qd, kd = q.contiguous(), k.contiguous()
    st.st_norm_rope_apply_qk(qd, kd, wq, wk, pos, sp, q_out=qd, k_out=kd)
    assert torch.equal(qd, q_out) and torch.equal(kd, k_out)
    # gradients written into slices of one projection's gradient, over the results' gradients and over the inputs
    gq, gk = torch.randn_like(q_out), torch.randn_like(k_out)
    dq, dk, dwq, dwk = st.st_norm_rope_bwd_qk(gq, gk, q, k, wq, wk, pos, sp)
    flat = torch.full((n, hq + 2 * hkv, d), 7.0, dtype=q.dtype, device=DEV)
    st.st_norm_rope_bwd_qk(gq, gk, q, k, wq, wk, pos, sp, dq=flat[:, :hq], dk=flat[:, hq:hq + hkv])
    assert torch.equal(flat[:, :hq], dq) and torch.equal(flat[:, hq:hq + hkv], dk) and bool((flat[:, hq + hkv:] == 7.0).all())
    g2q, g2k = gq.clone(), gk.clone()
    st.st_norm_rope_bwd_qk(g2q, g2k, q, k, wq, wk, pos, sp, dq=g2q, dk=g2k, weight_grads=False)
    assert torch.equal(g2q, dq) and torch.equal(g2k, dk)
    x = torch.cat((q, k, k), 1)
    got = st.st_norm_rope_bwd_qk(gq, gk, x[:, :hq], x[:, hq:hq + hkv], wq, wk, pos, sp, dq=x[:, :hq], dk=x[:, hq:hq + hkv])
    assert torch.equal(x[:, :hq], dq) and torch.equal(x[:, hq:hq + hkv], dk) and torch.equal(x[:, hq + hkv:], k) and torch.equal(got[2], dwq)
    only = st.st_norm_rope_bwd_qk(gq, None, q, None, wq, None, pos, sp)
    assert torch.equal(only[0], dq) and torch.equal(only[2], dwq) and only[1] is None and only[3] is None


@pytest.mark.gpu
def test_no_tokens(st):
    sp, _ = spec_of(st)
    q, k = torch.empty((0, 4, 128), device=DEV), torch.empty((0, 2, 128), device=DEV)
    w, pos = torch.ones(128, device=DEV), torch.empty(0, dtype=torch.int32, device=DEV)
    q_out, k_out = st.st_norm_rope_apply_qk(q, k, w, w, pos, sp)
    assert q_out.shape == q.shape and k_out.shape == k.shape
    dq, dk, dwq, dwk = st.st_norm_rope_bwd_qk(q, k, q, k, w, w, pos, sp)
    assert bool((dwq == 0).all()) and bool((dwk == 0).all())


@pytest.mark.gpu
def test_zero_and_non_finite_rows_stay_with_themselves(st):
    n, h, d = 40, 4, 128
    q, k, wq, wk, pos = inputs("f32", n, h, h, d, False, 5)
    sp, rope = spec_of(st)
    clean, _ = st.st_norm_rope_apply_qk(q, k, wq, wk, pos, sp)
    q[3, 1] = 0.0
    q[7, 2, 5] = float("nan")
    q[9, 0, 100] = float("inf")
    out, _ = st.st_norm_rope_apply_qk(q, k, wq, wk, pos, sp)
    assert bool((out[3, 1] == 0).all()) and bool(torch.isnan(out[7, 2]).all()) and bool(torch.isnan(out[9, 0]).any())
    touched = torch.zeros(n, h, dtype=torch.bool, device=DEV)
    for t, hh in ((3, 1), (7, 2), (9, 0)):
        touched[t, hh] = True
    assert torch.equal(out[~touched], clean[~touched])


@pytest.mark.gpu
def test_far_positions(st):
    n, d = 64, 64
    q, k, wq, wk, _ = inputs("f32", n, 2, 1, d, False, 9)
    pos = torch.linspace(2 ** 31 - 1 - 64, 2 ** 31 - 1, n, dtype=torch.float64).long().clamp(max=2 ** 31 - 1).to(torch.int32).to(DEV)
    sp, rope = spec_of(st, dim=d)
    out, _ = st.st_norm_rope_apply_qk(q, k, wq, wk, pos, sp)
    n64 = L.normalise(f64(q), f64(wq), np.float32(1e-6))
    ref = L.rotate(n64, f64(pos), *rope)
    # angles of 2^31 in 64 bits: each of the frequency, the product and the reduction is off by 2^-53 of it, here and in the oracle
    bound = (HALF_STEP["f32"] * np.abs(ref) + (FWD_UNITS * U24 + 6 * 2.0 ** (31 - 53)) * spread(n64, rope[0], rope[2]))
    assert (np.abs(f64(out) - ref) <= bound).all()


@pytest.mark.gpu
def test_rows_past_32_bit_offsets(st):
    """Rows whose element offsets pass 2^31: a strided slice over a long buffer."""
    n, hq, hkv, d = 3, 2, 1, 64
    stride = 2 ** 30 + 64
    buf = torch.zeros(2 * stride + (hq + hkv) * d, dtype=torch.bfloat16, device=DEV)
    x = buf.as_strided((n, hq + hkv, d), (stride, d, 1))
    q, k, wq, wk, pos = inputs("bf16", n, hq, hkv, d, False, 21)
    x[:, :hq] = q
    x[:, hq:] = k
    sp, rope = spec_of(st, dim=d)
    a = st.st_norm_rope_apply_qk(x[:, :hq], x[:, hq:], wq, wk, pos, sp)
    b = st.st_norm_rope_apply_qk(q, k, wq, wk, pos, sp)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    gq, gk = torch.randn_like(b[0]), torch.randn_like(b[1])
    ref = st.st_norm_rope_bwd_qk(gq, gk, q, k, wq, wk, pos, sp)
    st.st_norm_rope_bwd_qk(gq, gk, x[:, :hq], x[:, hq:], wq, wk, pos, sp, dq=x[:, :hq], dk=x[:, hq:])
    assert torch.equal(x[:, :hq], ref[0]) and torch.equal(x[:, hq:], ref[1])


@pytest.mark.gpu
def test_other_stream_and_graph_replays(st):
    n, hq, hkv, d = 300, 16, 8, 128
    q, k, wq, wk, pos = inputs("bf16", n, hq, hkv, d, True, 13)
    sp, _ = spec_of(st)
    gq, gk = torch.randn((n, hq, d), device=DEV).bfloat16(), torch.randn((n, hkv, d), device=DEV).bfloat16()
    ref = st.st_norm_rope_apply_qk(q, k, wq, wk, pos, sp), st.st_norm_rope_bwd_qk(gq, gk, q, k, wq, wk, pos, sp)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = st.st_norm_rope_apply_qk(q, k, wq, wk, pos, sp), st.st_norm_rope_bwd_qk(gq, gk, q, k, wq, wk, pos, sp)
    side.synchronize()
    flat = lambda r: [*r[0], *r[1]]
    assert all(torch.equal(a, b) for a, b in zip(flat(ref), flat(got)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = st.st_norm_rope_apply_qk(q, k, wq, wk, pos, sp), st.st_norm_rope_bwd_qk(gq, gk, q, k, wq, wk, pos, sp)
    for turn in range(4):
        q.copy_(torch.randn_like(q))
        gk.copy_(torch.randn_like(gk))
        want = st.st_norm_rope_apply_qk(q, k, wq, wk, pos, sp), st.st_norm_rope_bwd_qk(gq, gk, q, k, wq, wk, pos, sp)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(flat(out), flat(want))), turn


@pytest.mark.gpu
def test_results_are_of_the_stream_of_the_call(st):
    """stream=: memory that the current stream has just let go, with work on it still under way, is not where the results go."""
    n, hq, hkv, d = 4096, 16, 8, 128
    q, k, wq, wk, pos = inputs("bf16", n, hq, hkv, d, True, 14)
    sp, _ = spec_of(st)
    gq, gk = torch.randn((n, hq, d), device=DEV).bfloat16(), torch.randn((n, hkv, d), device=DEV).bfloat16()
    both = lambda **kw: [*st.st_norm_rope_apply_qk(q, k, wq, wk, pos, sp, **kw), *st.st_norm_rope_bwd_qk(gq, gk, q, k, wq, wk, pos, sp, **kw)]
    ref = both()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    slow = torch.randn((4096, 4096), device=DEV)
    for shape, dtype in [(x.shape, x.dtype) for x in ref]:
        y = torch.empty(shape, dtype=dtype, device=DEV)
        for _ in range(4):
            slow @ slow
        y.fill_(7.0)
        del y
    got = both(stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ref, got))


@pytest.mark.gpu
def test_rotation_alone_is_the_plain_rotation(st):
    """Without weights and with the plain spec: st_rope_apply_qk within a step of the result's type."""
    q, k, _, _, pos = inputs("bf16", 200, 8, 4, 128, False, 2)
    sp, rope = spec_of(st)
    a = st.st_norm_rope_apply_qk(q, k, None, None, pos, sp)
    b = st.st_rope_apply_qk(q, k, pos, 1.0e6, q_out=torch.empty_like(q), k_out=torch.empty_like(k))
    for x, y, src in zip(a, b, (q, k)):
        gap = np.abs(f64(x) - f64(y))
        assert (gap <= 2 * HALF_STEP["bf16"] * np.abs(f64(y)) + 2 * FWD_UNITS * U24 * spread(f64(src), rope[0], rope[2])).all()
