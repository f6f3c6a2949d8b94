"""Decode over caches held in 4 bits against a softmax in 64 bits over the values that the codes stand for."""
import numpy as np
import pytest
import torch

from oracle import layer_ops as L
from rows_helpers import f64, spec_of

DEV = "cuda"
U24, HALF = 2.0 ** -24, 2.0 ** -8


@pytest.fixture(scope="module")
def st():
    import paper_2510_17238_amd as st
    return st


def make(st, seed, batch, hkv, d, src_cap, rsn_cap, n_src, n_rsn, magnitude=1.0):
    """Two caches of scale bytes 255 and codes 0xff, filled with n_src, n_rsn tokens; and the rows as stored (read back)."""
    rng, g = np.random.default_rng(seed), torch.Generator(device=DEV).manual_seed(seed)
    caches, rows = [], []
    for cap in (src_cap, rsn_cap):
        pages = max(1, -(-cap // 16))
        table = rng.permutation(batch * pages + 2)[:batch * pages].astype(np.int32).reshape(batch, pages)
        caches.append(st.KVCache(batch * pages + 2, batch, pages, hkv, d, torch.from_numpy(table).to(DEV), fill=0xff, mxfp4=True))
    dual = st.DualCache(*caches)
    for which, lens in ((st.ST_SOURCE, n_src), (st.ST_REASONING, n_rsn)):
        most = max(1, max(lens))
        k = (magnitude * torch.randn((batch, most, hkv, d), generator=g, device=DEV)).to(torch.bfloat16)
        v = (torch.randn((batch, most, hkv, d), generator=g, device=DEV) * torch.exp2(torch.randint(-3, 4, (batch, most, 1, 1), generator=g, device=DEV).float())).to(torch.bfloat16)
        st.st_kv_append(dual, which, k, v, n_new=torch.tensor(lens, dtype=torch.int32, device=DEV))
        k_out, v_out = torch.zeros_like(k), torch.zeros_like(v)
        st.st_kv_read(dual, which, k_out, v_out, n=torch.tensor(lens, dtype=torch.int32, device=DEV))
        rows.append((f64(k_out), f64(v_out)))
    return dual, rows


def check(out, lse, q, rows, vis, rsn, scale, q_slack=None):
    """out, lse against 64 bits.  Terms of the bound: a score's product of D terms in fp32 (D + 2 roundings), times the scale (2 more) and
    the function (2 steps): a weight is off by that part of itself; weights are rounded to bf16 (half a step) for the product, which sums
    in fp32; sums of up to 64 + N / 16 weights a lane; the result is rounded once.  Weights are relative to the largest of their unit and units to the largest of the row, both by the fp32
    function, which gives 0 below 2^-126: of N weights at most N 2^-126 is lost at either place, times the values.  q_slack: |q| that the
    rotation may have moved."""
    batch, q_len, hq, d = q.shape
    hkv = rows[0][0].shape[2]
    for b in range(batch):
        for t in range(q_len):
            ns, nr = vis[b], max(0, rsn[b] - q_len + t + 1)
            k = np.concatenate([rows[0][0][b, :ns], rows[1][0][b, :nr]])
            v = np.concatenate([rows[0][1][b, :ns], rows[1][1][b, :nr]])
            for h in range(hq):
                kk, vv, x = k[:, h // (hq // hkv)], v[:, h // (hq // hkv)], q[b, t, h]
                got, got_l = out[b, t, h], lse[b, t, h]
                if len(kk) == 0:
                    assert (got == 0).all() and got_l == -np.inf
                    continue
                s = kk @ x * scale
                size = np.abs(kk) @ np.abs(x) * scale
                delta = ((d + 4) * size + 4 * np.abs(s) + 4).max() * U24
                if q_slack is not None:
                    delta += (np.abs(kk) @ q_slack[b, t, h] * scale).max()
                p = np.exp(s - s.max())
                ref, mag = p @ vv / p.sum(), p @ np.abs(vv) / p.sum()
                sums = (64 + len(kk) / 16) * U24
                bound = HALF * np.abs(ref) * (1 + HALF) + (HALF + 2 * delta + 2 * sums) * mag * (1 + HALF) + 2 * len(kk) * 2.0 ** -126 * np.abs(vv).max()
                assert (np.abs(got - ref) <= bound).all(), (b, t, h, float((np.abs(got - ref) / np.maximum(bound, 1e-300)).max()))
                ref_l = s.max() + np.log(p.sum())
                assert abs(got_l - ref_l) <= delta + sums + 4 * U24 * (np.abs(ref_l) + np.abs(s).max() + 1), (b, t, h, got_l - ref_l)


def decode(st, q, dual, vis, rsn, src_bound=None, rsn_bound=None, **kw):
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    lse = torch.full(q.shape[:3], 5.0, device=DEV)
    call = st.st_attn_decode_dual if "theta_base" not in kw else st.st_attn_decode_dual_rope
    out = call(q, dual, dev(vis), dev(rsn), max(vis) if src_bound is None else src_bound, max(rsn) if rsn_bound is None else rsn_bound, lse=lse, **kw)
    return out, lse


CASES = [
    # q heads, kv heads, dim, q_len, source, reasoning tokens
    (4, 1, 128, 1, [96], [300]),
    (2, 2, 64, 1, [0, 1, 17], [1, 0, 0]),
    (32, 8, 128, 1, [64, 63, 65, 640], [64, 129, 1, 300]),
    (16, 1, 64, 1, [1000, 5], [31, 900]),
    (16, 8, 128, 1, [2048, 1500], [4097, 33]),
    (8, 8, 64, 1, [3000, 4096, 0], [1025, 2047, 5000]),
    (5, 1, 128, 3, [100, 1200], [3, 777]),
    (5, 1, 64, 6, [0, 1100], [6, 777]),
    (8, 2, 128, 8, [2000, 15, 16], [8, 2500, 200]),
    (4, 4, 128, 17, [700], [1300]),
    (32, 1, 64, 1, [40], [20]),
    (8, 2, 64, 5, [300, 4], [2, 0]),              # fewer reasoning tokens than queries: rows that see the source alone, or nothing
]


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d,q_len,src,rsn", CASES)
@pytest.mark.parametrize("unit", [0, 128, 512])
def test_against_64_bits(st, hq, hkv, d, q_len, src, rsn, unit):
    dual, rows = make(st, hq * d + q_len, len(src), hkv, d, max(src) + 40, max(rsn) + 40, src, rsn)
    q = torch.randn((len(src), q_len, hq, d), device=DEV).to(torch.bfloat16)
    vis = [max(0, s - i) for i, s in enumerate(src)]            # (a slice of the source cache, as earlier sentences leave it)
    out, lse = decode(st, q, dual, vis, rsn, unit_tokens=unit)
    check(f64(out), f64(lse), f64(q), rows, vis, rsn, d ** -0.5)
    again, lse2 = decode(st, q, dual, vis, rsn, unit_tokens=unit)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    # bounds beyond the lengths, a scale of the caller's
    wide, lse3 = decode(st, q, dual, vis, rsn, src_bound=max(src) + 33, rsn_bound=max(rsn) + 40, scale=0.05)
    check(f64(wide), f64(lse3), f64(q), rows, vis, rsn, np.float64(np.float32(0.05)))


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d,q_len,src,rsn", [(4, 1, 128, 1, [96, 7], [300, 1]), (8, 2, 64, 2, [1500, 3], [20, 900]), (8, 2, 128, 8, [600], [700])])
def test_rotated_queries(st, hq, hkv, d, q_len, src, rsn):
    """The query rotation in the kernel: the rotated query is rounded to bf16, half a step of it and the rotation's own error."""
    dual, rows = make(st, 5, len(src), hkv, d, max(src), max(rsn), src, rsn)
    q = torch.randn((len(src), q_len, hq, d), device=DEV).to(torch.bfloat16)
    out, lse = decode(st, q, dual, src, rsn, theta_base=1.0e4)
    freq, a = L.frequencies(d, 1.0e4)
    turned, slack = np.zeros(q.shape), np.zeros(q.shape)
    for b in range(len(src)):
        pos = np.maximum(rsn[b] - q_len + np.arange(q_len), 0)
        exact = L.rotate(f64(q[b]), pos, freq, a, "half")
        turned[b] = L.bf16(exact)
        slack[b] = 2 * HALF * np.abs(exact) + 16 * U24 * (np.abs(f64(q[b])) + np.abs(np.roll(f64(q[b]), d // 2, -1)))
    check(f64(out), f64(lse), turned, rows, src, rsn, d ** -0.5, q_slack=slack)


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d,q_len,src,rsn", [(4, 1, 128, 1, [200], [300]), (4, 1, 64, 1, [1500], [300]), (8, 2, 128, 8, [200], [300])])
def test_large_scores_and_values(st, hq, hkv, d, q_len, src, rsn):
    dual, rows = make(st, 6, 1, hkv, d, src[0], rsn[0], src, rsn, magnitude=2.0 ** 5)
    q = (4.0 * torch.randn((1, q_len, hq, d), device=DEV)).to(torch.bfloat16)
    out, lse = decode(st, q, dual, src, rsn)
    check(f64(out), f64(lse), f64(q), rows, src, rsn, d ** -0.5)


@pytest.mark.gpu
@pytest.mark.parametrize("n_src,n_rsn,q_len,hq", [(33, 100, 1, 4), (33, 1500, 1, 4), (700, 1500, 5, 8)])
@pytest.mark.parametrize("d", [64, 128])
def test_visible_nan_reaches_its_rows_and_no_others(st, n_src, n_rsn, q_len, hq, d):
    for what in ("key", "value"):
        dual, _ = make(st, 7, 2, 2, d, n_src, n_rsn, [n_src, n_src], [n_rsn, n_rsn])
        q = torch.randn((2, q_len, hq, d), device=DEV).to(torch.bfloat16)
        clean, _ = decode(st, q, dual, [n_src] * 2, [n_rsn] * 2)
        bad = torch.randn((2, 1, 2, d), device=DEV).to(torch.bfloat16)
        k, v = bad.clone(), bad.clone()
        (k if what == "key" else v)[0, 0, 1, 3] = float("nan")
        at = torch.tensor([7, 7], dtype=torch.int32, device=DEV)
        st.st_kv_append_norm_rope(dual, st.ST_SOURCE, k, v, None, None, start_len=at)
        out, _ = decode(st, q, dual, [n_src] * 2, [n_rsn] * 2)
        heads = hq // 2
        poisoned = out[0, :, heads:]
        assert bool(torch.isnan(poisoned).all() if what == "key" else torch.isnan(poisoned[..., :32]).all())
        assert bool(torch.isfinite(out[0, :, :heads]).all()) and bool(torch.isfinite(out[1]).all())
        # not visible: nothing of it
        st.st_kv_append_norm_rope(dual, st.ST_SOURCE, k, v, None, None, start_len=torch.tensor([n_src - 1] * 2, dtype=torch.int32, device=DEV))
        st.st_kv_append_norm_rope(dual, st.ST_SOURCE, bad, bad, None, None, start_len=at)
        out, _ = decode(st, q, dual, [n_src - 1] * 2, [n_rsn] * 2)
        assert bool(torch.isfinite(out).all())


@pytest.mark.gpu
def test_static_scratch_streams_and_graph(st):
    src, rsn = [300, 1500, 0], [2000, 40, 7]
    dual, rows = make(st, 8, 3, 8, 128, 1600, 2100, src, rsn)
    q = torch.randn((3, 1, 32, 128), device=DEV).to(torch.bfloat16)
    ref, ref_l = decode(st, q, dual, src, rsn)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    vis, n = dev(src), dev(rsn)
    out = torch.empty_like(q)
    st.st_attn_decode_dual_static(q, dual, vis, n, 1500, 2000, out)
    assert torch.equal(out, ref)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for s in streams:
        with torch.cuda.stream(s):
            outs.append(st.st_attn_decode_dual(q, dual, vis, n, 1500, 2000))
    torch.cuda.synchronize()
    assert all(torch.equal(o, ref) for o in outs)
    ws = torch.empty(st.st_decode_workspace_bytes(3, 32, 8, 128, 1, 1500, 2000), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        st.st_attn_decode_dual(q, dual, vis, n, 1500, 2000, out=out, workspace=ws)
    for turn in range(4):
        q.copy_(torch.randn_like(q))
        vis.copy_(dev([300 - turn, 1500 - 100 * turn, 0]))
        want, _ = decode(st, q, dual, vis.tolist(), rsn, src_bound=1500)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), turn


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d,q_len", [(32, 8, 128, 1), (16, 4, 128, 4), (8, 2, 64, 8), (8, 2, 128, 8)])
def test_a_captured_step_of_growing_caches(st, hq, hkv, d, q_len):
    """Rows from the projections into the cache and the decode that sees them, captured once, replayed for step after step: what the same calls
    give one by one, in caches that end as theirs do.  4, 16 (one launch, more than the default LDS) and 32 rows."""
    n_src, n_rsn, steps = [40, 130], [9, 64], 5
    twins = [make(st, 11, 2, hkv, d, 160, 64 + 16 * 5, n_src, n_rsn)[0] for _ in range(2)]
    g = torch.Generator(device=DEV).manual_seed(12)
    new = torch.zeros((2, q_len, hq + 2 * hkv, d), dtype=torch.bfloat16, device=DEV)          # a projection's output: queries, keys, values
    w = (1.0 + 0.2 * torch.randn(d, generator=g, device=DEV)).to(torch.bfloat16)
    spec, _ = spec_of(st)
    vis = torch.tensor(n_src, dtype=torch.int32, device=DEV)
    most = 64 + q_len * steps
    lens = [torch.tensor(n_rsn, dtype=torch.int32, device=DEV) for _ in range(2)]
    bufs = [(torch.empty((2 * q_len, hq, d), dtype=torch.bfloat16, device=DEV), torch.empty((2, q_len, hq, d), dtype=torch.bfloat16, device=DEV)) for _ in range(2)]
    flat = new.view(2 * q_len, hq + 2 * hkv, d)

    def step(i):
        q, out = bufs[i]
        before = lens[i]
        pos = (before[:, None] + torch.arange(q_len, dtype=torch.int32, device=DEV)).reshape(-1)
        st.st_norm_rope_apply_qk(flat[:, :hq], None, w, None, pos, spec, q_out=q)
        st.st_kv_append_norm_rope(twins[i], st.ST_REASONING, new[:, :, hq:hq + hkv], new[:, :, hq + hkv:], w, spec, start_len=before)
        before += q_len
        st.st_attn_decode_dual(q.view(2, q_len, hq, d), twins[i], vis, before, 130, most, out=out, workspace=ws)

    ws = torch.empty(st.st_decode_workspace_bytes(2, hq, hkv, d, q_len, 130, most), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(0)
    for turn in range(steps):
        new.copy_(torch.randn(new.shape, generator=g, device=DEV))
        step(1)
        want = bufs[1][1].clone()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(bufs[0][1], want) and bool(torch.isfinite(want).all()), turn
    a, b = twins[0].reasoning, twins[1].reasoning
    assert torch.equal(a.k_pool, b.k_pool) and torch.equal(a.v_pool, b.v_pool) and torch.equal(a.k_scale, b.k_scale)
    assert a.appended_len.tolist() == b.appended_len.tolist() == [n + q_len * steps for n in n_rsn]


@pytest.mark.gpu
@pytest.mark.parametrize("vis", [1500, 1501, 1519])
def test_tokens_stored_beside_a_decode_that_does_not_see_them(st, vis):
    """On another stream, into the page that the visible tokens end in: no byte is shared with them."""
    dual, _ = make(st, 15, 4, 8, 128, 1600, 600, [vis] * 4, [600] * 4)
    q = torch.randn((4, 1, 32, 128), device=DEV).to(torch.bfloat16)
    ref, _ = decode(st, q, dual, [vis] * 4, [600] * 4)
    dev = lambda x: torch.tensor([x] * 4, dtype=torch.int32, device=DEV)
    seen, n, start, n_new = dev(vis), dev(600), dev(vis), torch.tensor([1, 7, 20, 37], dtype=torch.int32, device=DEV)
    k, v = (torch.randn((4, 37, 8, 128), device=DEV).to(torch.bfloat16) for _ in range(2))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    outs = []
    for i in range(40):
        st.st_kv_append_norm_rope(dual, st.ST_SOURCE, k, v, None, None, n_new=n_new, start_len=start, stream=side)
        outs.append(st.st_attn_decode_dual(q, dual, seen, n, vis, 600))
    torch.cuda.synchronize()
    assert all(torch.equal(o, ref) for o in outs)


@pytest.mark.gpu
def test_pools_past_4_gib(st):
    hkv, d = 8, 128
    n_pages = 2 ** 32 // (d // 2 * hkv * 16) + 9
    tab = [[n_pages - 1 - i for i in range(4)]]
    big, small = [], []
    for x in range(2):
        big.append(st.KVCache(n_pages, 1, 4, hkv, d, torch.tensor(tab, dtype=torch.int32, device=DEV), mxfp4=True))
        small.append(st.KVCache(4, 1, 4, hkv, d, torch.arange(4, dtype=torch.int32, device=DEV).reshape(1, 4), mxfp4=True))
    k, v = (torch.randn((1, 60, hkv, d), device=DEV).to(torch.bfloat16) for _ in range(2))
    q = torch.randn((1, 1, 32, d), device=DEV).to(torch.bfloat16)
    outs = []
    for c in (big, small):
        dual = st.DualCache(*c)
        for which in (st.ST_SOURCE, st.ST_REASONING):
            st.st_kv_append(dual, which, k, v)
        outs += [decode(st, q, dual, [60], [60])[0], decode(st, q, dual, [60], [60], src_bound=64, rsn_bound=64, unit_tokens=128)[0]]
    assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[3])


@pytest.mark.gpu
@pytest.mark.parametrize("store", ["bf16", "fp8", "mxfp4"])
def test_a_layers_steps_together(st, store):
    """A sentence taken in, then tokens decoded: projections' slices -> norm + rotation of the queries, keys and values into the caches, attention;
    every step against 64 bits over the rows that the caches hold."""
    hq, hkv, d, batch, eps = 16, 8, 128, 3, 1.0e-6
    spec, rope = spec_of(st, scaling="yarn", factor=2.0, original=4096)
    g = torch.Generator(device=DEV).manual_seed(4)
    wq, wk = ((1 + 0.2 * torch.randn(d, generator=g, device=DEV)).to(torch.bfloat16) for _ in range(2))
    caches = []
    for cap in (64, 32):
        table = torch.randperm(batch * cap // 16, generator=torch.Generator().manual_seed(cap)).to(torch.int32).reshape(batch, cap // 16).to(DEV)
        caches.append(st.KVCache(batch * cap // 16, batch, cap // 16, hkv, d, table, fp8=store == "fp8", mxfp4=store == "mxfp4"))
    dual = st.DualCache(*caches)

    def projected(tokens):
        return (1.5 * torch.randn((batch, tokens, hq + 2 * hkv, d), generator=g, device=DEV)).to(torch.bfloat16)

    n_src = [50, 1, 33]
    x = projected(50)
    st.st_kv_append_norm_rope(dual, st.ST_SOURCE, x[:, :, hq:hq + hkv], x[:, :, hq + hkv:], wk, spec, eps=eps,
                              n_new=torch.tensor(n_src, dtype=torch.int32, device=DEV))
    vis = torch.tensor(n_src, dtype=torch.int32, device=DEV)
    for step in range(20):
        x = projected(1)
        pos = torch.full((batch,), step, dtype=torch.int32, device=DEV)
        q, _ = st.st_norm_rope_apply_qk(x[:, 0, :hq], None, wq, None, pos, spec, eps=eps)
        st.st_kv_append_norm_rope(dual, st.ST_REASONING, x[:, :, hq:hq + hkv], x[:, :, hq + hkv:], wk, spec, eps=eps, start_len=pos)
        rsn = pos + 1
        lse = torch.empty((batch, 1, hq), device=DEV)
        out = st.st_attn_decode_dual(q[:, None], dual, vis, rsn, 64, 32, lse=lse)
        if step % 6 == 1:
            rows = []
            for which, cap in ((st.ST_SOURCE, 64), (st.ST_REASONING, 32)):
                k, v = (torch.zeros((batch, cap, hkv, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
                st.st_kv_read(dual, which, k, v)
                rows.append((f64(k), f64(v)))
            # the queries themselves: half a step of bf16 from the definition
            n = L.normalise(f64(x[:, 0, :hq]), f64(wq), eps)
            ref = L.rotate(n, f64(pos), *rope)
            assert (np.abs(f64(q) - ref) <= HALF * np.abs(ref) + 1e-5).all()
            if store == "mxfp4":
                check(f64(out), f64(lse), f64(q[:, None]), rows, n_src, [step + 1] * batch, d ** -0.5)
            else:
                for b in range(batch):
                    for h in range(hq):
                        k = np.concatenate([rows[0][0][b, :n_src[b], h // 2], rows[1][0][b, :step + 1, h // 2]])
                        v = np.concatenate([rows[0][1][b, :n_src[b], h // 2], rows[1][1][b, :step + 1, h // 2]])
                        s = k @ f64(q[b, h]) * d ** -0.5
                        p = np.exp(s - s.max())
                        mag = p @ np.abs(v) / p.sum()
                        assert (np.abs(f64(out[b, 0, h]) - p @ v / p.sum()) <= 3 * HALF * mag + 1e-3 * mag).all()
    assert caches[0].appended_len.tolist() == n_src and caches[1].appended_len.tolist() == [20] * batch
