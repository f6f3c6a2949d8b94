"""4-bit decode with the work units of 1,024, 2,048 and 4,096 tokens that large launches take: many sequences over the pages of a few, so that the launch
is large and the caches are small, against 64 bits; and the rule that chooses the unit, by the number of workgroups that a launch stamps."""
import numpy as np
import pytest
import torch

from oracle import layer_ops as L
from rows_helpers import f64
from test_gpu_decode_4bit import DEV, HALF, U24, check, make
from test_gpu_decode_long_units import _stamped_workgroups


@pytest.fixture(scope="module")
def st():
    import paper_2510_17238_amd as st
    return st


def many_over_few(st, dual, copies, bound):
    """The sequences of `dual`, `copies` times over, with page tables for `bound` tokens."""
    wide = []
    for c in (dual.source, dual.reasoning):
        table = torch.zeros((c.batch, bound // 16), dtype=torch.int32, device=DEV)
        own = min(c.max_pages_per_seq, bound // 16)
        table[:, :own] = c.page_table[:, :own]
        w = st.KVCache(1, copies * c.batch, bound // 16, c.n_kv_heads, c.head_dim, table.repeat(copies, 1).contiguous(), mxfp4=True)
        w.n_pages, w.k_pool, w.v_pool, w.k_scale = c.n_pages, c.k_pool, c.v_pool, c.k_scale
        wide.append(w)
    return st.DualCache(*wide)


def lengths(unit, bound):
    """One short of, at and one past a unit, a ragged tail, the whole bound, one token, none."""
    return [unit - 1, unit + 1, bound, 0, 1], [unit, bound - 37, 33, unit + 1, 0]


# (copies of the five sequences, so many that the rule takes the unit: 1,024 tokens from 512 units on, 2,048 and 4,096 from thousands)
@pytest.mark.gpu
@pytest.mark.parametrize("unit,bound,copies", [(1024, 4096, 7), (2048, 4096, 105), (4096, 8192, 53)])
@pytest.mark.parametrize("hq,d,q_len,rope", [(4, 128, 1, None), (4, 64, 4, 1.0e6), (8, 128, 3, None), (8, 64, 4, None), (8, 128, 8, 1.0e6), (10, 64, 5, None)])
def test_long_units(st, unit, bound, copies, hq, d, q_len, rope):
    hkv = 2
    rows_a_head = q_len * hq // hkv
    if unit == 2048 and rows_a_head > 8:
        copies = 53                                                     # (from half as many units on, and as many of 4,096 take those)
    src, rsn = lengths(unit, bound)
    dual, rows = make(st, 70 + q_len, 5, hkv, d, max(src), max(rsn), src, rsn)
    wide = many_over_few(st, dual, copies, bound)
    q = torch.randn((5, q_len, hq, d), generator=torch.Generator(device=DEV).manual_seed(71), device=DEV).to(torch.bfloat16)
    tq = q.repeat(copies, 1, 1, 1)
    ts, tr = (torch.tensor(x * copies, dtype=torch.int32, device=DEV) for x in (src, rsn))
    lse = torch.empty((5 * copies, q_len, hq), device=DEV)
    out, workgroups = _stamped_workgroups(st, lambda: st.st_attn_decode_dual(tq, wide, ts, tr, bound, bound, lse=lse, rope_theta=rope))
    taken = min(unit, 2048) if rows_a_head <= 8 else unit               # (few rows: none of 4,096)
    assert workgroups == 5 * copies * hkv * 2 * (bound // taken)
    assert torch.equal(out.view(copies, -1), out[:5].reshape(1, -1).expand(copies, -1))
    assert torch.equal(lse.view(copies, -1), lse[:5].reshape(1, -1).expand(copies, -1))
    turned, slack = f64(q), None
    if rope is not None:
        freq, a = L.frequencies(d, rope)
        turned, slack = np.zeros(q.shape), np.zeros(q.shape)
        for b in range(5):
            exact = L.rotate(f64(q[b]), np.maximum(rsn[b] - q_len + np.arange(q_len), 0), freq, a, "half")
            turned[b] = L.bf16(exact)
            slack[b] = 2 * HALF * np.abs(exact) + 16 * U24 * (np.abs(f64(q[b])) + np.abs(np.roll(f64(q[b]), d // 2, -1)))
    check(f64(out[:5]), f64(lse[:5]), turned, rows, src, rsn, d ** -0.5, q_slack=slack)


@pytest.mark.gpu
@pytest.mark.parametrize("hq,d,q_len", [(4, 128, 1), (8, 64, 3), (8, 128, 8)])
def test_a_unit_of_the_callers_choice(st, hq, d, q_len):
    """unit_tokens = 1,024: four steps a wave."""
    src, rsn = lengths(1024, 2048)
    dual, rows = make(st, 80, 5, 2, d, max(src), max(rsn), src, rsn)
    q = torch.randn((5, q_len, hq, d), generator=torch.Generator(device=DEV).manual_seed(81), device=DEV).to(torch.bfloat16)
    ts, tr = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (src, rsn))
    lse = torch.empty((5, q_len, hq), device=DEV)
    out = st.st_attn_decode_dual(q, dual, ts, tr, max(src), max(rsn), lse=lse, unit_tokens=1024)
    check(f64(out), f64(lse), f64(q), rows, src, rsn, d ** -0.5)
