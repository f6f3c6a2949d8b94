"""4-bit decode, several tokens a step: a token that a row does not see does not reach it, whatever its values are."""
import pytest
import torch

from test_gpu_decode_4bit import DEV, decode, make


@pytest.fixture(scope="module")
def st():
    import paper_2510_17238_amd as st
    return st


# 4, 8, 16 and 32 rows a KV head; caches for one launch and for two; the last tokens in a step of their own, or across two pages
@pytest.mark.gpu
@pytest.mark.parametrize("q_len,hq,hkv,d", [(4, 2, 2, 128), (4, 4, 2, 64), (8, 4, 2, 128), (8, 8, 2, 128), (5, 10, 2, 64), (6, 1, 1, 64)])
@pytest.mark.parametrize("n_src,n_rsn", [(33, 100), (0, 67), (700, 1500), (1300, 5), (40, 1030)])
@pytest.mark.parametrize("unit", [0, 128])
def test_tokens_that_a_row_does_not_see(st, q_len, hq, hkv, d, n_src, n_rsn, unit):
    dual, _ = make(st, 61, 2, hkv, d, n_src, n_rsn, [n_src] * 2, [n_rsn] * 2)
    q = torch.randn((2, q_len, hq, d), device=DEV).to(torch.bfloat16)
    clean, clean_l = decode(st, q, dual, [n_src] * 2, [n_rsn] * 2, unit_tokens=unit)
    group = hq // hkv
    for back, bad in ((1, float("nan")), (1, 2.0 ** 127 * 1.9921875), (min(3, q_len - 1), float("-inf"))):
        first = n_rsn - back                                              # the last `back` tokens, seen by the last `back` rows (the first of them by all those)
        at = torch.tensor([first] * 2, dtype=torch.int32, device=DEV)
        old_k, old_v = (torch.zeros((2, back, hkv, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        st.st_kv_read(dual, st.ST_REASONING, old_k, old_v, first=at)
        for what in ("value", "key", "both"):
            k, v = old_k.clone(), old_v.clone()
            if what != "value":
                k[0, 0, hkv - 1, 5] = bad
            if what != "key":
                v[0, 0, hkv - 1, 3], v[0, 0, hkv - 1, d - 1] = bad, bad
            st.st_kv_append_norm_rope(dual, st.ST_REASONING, k, v, None, None, start_len=at)
            out, lse = decode(st, q, dual, [n_src] * 2, [n_rsn] * 2, unit_tokens=unit)
            blind = q_len - back
            assert torch.equal(out[:, :blind], clean[:, :blind]) and torch.equal(lse[:, :blind], clean_l[:, :blind]), (back, bad, what)
            assert torch.equal(out[1], clean[1]) and torch.equal(out[0, :, :(hkv - 1) * group], clean[0, :, :(hkv - 1) * group])
            seen = out[0, blind:, (hkv - 1) * group:]
            if what != "key" and abs(bad) < float("inf"):
                # (a value that reads as infinite: its dims alone)
                assert bool((~torch.isfinite(seen[..., [3, d - 1]])).all())
            elif what != "key":
                assert bool(torch.isnan(seen[..., :32]).all()) and bool(torch.isnan(seen[..., d - 32:]).all())
            if what == "value":
                assert bool(torch.isfinite(seen[..., 32:d - 32]).all())
                assert torch.equal(lse[0], clean_l[0])
            elif bad != bad or abs(bad) == float("inf"):
                assert bool(torch.isnan(seen).all())
        st.st_kv_append_norm_rope(dual, st.ST_REASONING, old_k, old_v, None, None, start_len=at)
        again, again_l = decode(st, q, dual, [n_src] * 2, [n_rsn] * 2, unit_tokens=unit)
        assert torch.equal(again, clean) and torch.equal(again_l, clean_l)


@pytest.mark.gpu
@pytest.mark.parametrize("q_len,hq,hkv,d", [(2, 1, 1, 128), (4, 2, 1, 64), (8, 4, 2, 128), (8, 8, 2, 128)])
@pytest.mark.parametrize("n_src,n_rsn", [(33, 100), (700, 1500)])
def test_no_bit_of_a_row_depends_on_later_tokens(st, q_len, hq, hkv, d, n_src, n_rsn):
    """The last token's key replaced by ones that score higher and higher for the last row: the other rows stay as they are, bit by bit."""
    g = torch.Generator(device=DEV).manual_seed(62)
    dual, _ = make(st, 62, 2, hkv, d, n_src, n_rsn, [n_src] * 2, [n_rsn] * 2)
    q = torch.randn((2, q_len, hq, d), generator=g, device=DEV).to(torch.bfloat16)
    at = torch.tensor([n_rsn - 1] * 2, dtype=torch.int32, device=DEV)
    ref = None
    for size in (0.25, 4.0, 16.0, 64.0, 1024.0):
        k = (size * torch.randn((2, 1, hkv, d), generator=g, device=DEV)).to(torch.bfloat16)
        st.st_kv_append_norm_rope(dual, st.ST_REASONING, k, k, None, None, start_len=at)
        out, lse = decode(st, q, dual, [n_src] * 2, [n_rsn] * 2)
        if ref is not None:
            assert torch.equal(out[:, :-1], ref[0][:, :-1]) and torch.equal(lse[:, :-1], ref[1][:, :-1]), size
            assert not torch.equal(out[:, -1], ref[0][:, -1])
        ref = out, lse


@pytest.mark.gpu
@pytest.mark.parametrize("q_len,hq,hkv,d", [(4, 2, 2, 64), (8, 4, 2, 128), (8, 8, 2, 128)])
@pytest.mark.parametrize("n_src,n_rsn", [(33, 100), (700, 1500)])
def test_with_rotated_queries(st, q_len, hq, hkv, d, n_src, n_rsn):
    """The rotation in the kernel: the angles are still there when a step is gone through limit by limit."""
    dual, _ = make(st, 63, 2, hkv, d, n_src, n_rsn, [n_src] * 2, [n_rsn] * 2)
    q = torch.randn((2, q_len, hq, d), generator=torch.Generator(device=DEV).manual_seed(63), device=DEV).to(torch.bfloat16)
    clean, clean_l = decode(st, q, dual, [n_src] * 2, [n_rsn] * 2, theta_base=1.0e4)
    at = torch.tensor([n_rsn - 1] * 2, dtype=torch.int32, device=DEV)
    k, v = (torch.zeros((2, 1, hkv, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    st.st_kv_read(dual, st.ST_REASONING, k, v, first=at)
    v[1, 0, 0, 40] = float("nan")
    st.st_kv_append_norm_rope(dual, st.ST_REASONING, k, v, None, None, start_len=at)
    out, lse = decode(st, q, dual, [n_src] * 2, [n_rsn] * 2, theta_base=1.0e4)
    group = hq // hkv
    assert torch.equal(out[:, :-1], clean[:, :-1]) and torch.equal(lse, clean_l) and torch.equal(out[0], clean[0])
    last = out[1, -1, :group]
    assert bool(torch.isnan(last[:, 32:64]).all()) and torch.equal(last[:, :32], clean[1, -1, :group, :32]) and torch.equal(last[:, 64:], clean[1, -1, :group, 64:])
