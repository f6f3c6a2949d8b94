"""New tokens' rows into paged caches of every storage format -- normalised, rotated, coded -- and rows read back."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import layer_ops as L
from oracle import streaming_attention as O
from rows_helpers import f64, spec_of

DEV = "cuda"
FORMATS = ["bf16", "fp8", "mxfp4"]


@pytest.fixture(scope="module")
def st():
    import paper_2510_17238_amd as st
    return st


def cache_of(st, rng, store, batch, pages, hkv, d, extra=3, fill=0xab):
    """A cache with a shuffled page table over a pool with pages to spare, pre-set to a pattern."""
    n = batch * pages + extra
    table = rng.permutation(n)[:batch * pages].astype(np.int32).reshape(batch, pages)
    c = st.KVCache(n, batch, pages, hkv, d, torch.from_numpy(table).to(DEV), fill=fill, fp8=store == "fp8", mxfp4=store == "mxfp4")
    return c, table


def pair(st, cache):
    return st.DualCache(cache, cache)


def stored(store, x):
    """What a cache holds for bf16 rows (fp64 array [..., D])."""
    if store == "bf16":
        return x
    if store == "mxfp4":
        return L.mxfp4(x)
    return O.dequantize_rows_e4m3(*O.quantize_rows_e4m3(x))


def rand_rows(g, *shape, spread=True):
    x = torch.randn(shape, generator=g, device=DEV)
    if spread:
        x = x * torch.exp2(torch.randint(-6, 7, (*shape[:-1], 1), generator=g, device=DEV).float())
    return x.to(torch.bfloat16)


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def read(st, caches, which, batch, most, first=None, n=None):
    c = caches.source if which == st.ST_SOURCE else caches.reasoning
    k = torch.full((batch, most, c.n_kv_heads, c.head_dim), 9.0, dtype=torch.bfloat16, device=DEV)
    v = torch.full_like(k, -9.0)
    dev = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device=DEV)
    return st.st_kv_read(caches, which, k, v, first=dev(first), n=dev(n))


def same(a, b):
    """Equal values, NaN where NaN."""
    a, b = np.asarray(a, np.float64), np.asarray(b, np.float64)
    return np.array_equal(np.isnan(a), np.isnan(b)) and np.array_equal(a[~np.isnan(a)], b[~np.isnan(b)])


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_codes_of_every_significand(st, d):
    """Every bf16 significand in every position against a block's largest value, signs and exponents mixed, ties among them."""
    rng = np.random.default_rng(d)
    blocks = []
    for shift in range(-3, 8):
        m = (1.0 + np.arange(128) / 128.0) * 2.0 ** -shift
        for lead in (4.0, 5.0, 6.0, 6.03125, 7.96875):
            blocks += [np.append(np.resize(m[i:i + 31], 31), lead) for i in range(0, 128, 31)]
    x = np.array(blocks) * rng.choice((-1.0, 1.0), (len(blocks), 32)) * 2.0 ** rng.integers(-90, 90, (len(blocks), 1))
    x = np.concatenate([x, np.zeros((3, 32)), np.full((1, 32), 2.0 ** -133), np.full((1, 32), 2.0 ** -101), np.full((1, 32), 1.5 * 2.0 ** 126)])
    rows = -(-len(x) // (d // 32))
    x = np.resize(x, (rows * (d // 32), 32)).reshape(1, rows, 1, d)
    t = torch.from_numpy(x).to(torch.bfloat16).to(DEV)
    assert np.array_equal(f64(t), x)                       # (bf16 holds them)
    c, _ = cache_of(st, rng, "mxfp4", 1, -(-rows // 16), 1, d)
    st.st_kv_append(pair(st, c), st.ST_SOURCE, t, t)
    k, v = read(st, pair(st, c), st.ST_SOURCE, 1, rows)
    want = L.mxfp4(x)
    assert np.array_equal(f64(k), want) and np.array_equal(f64(v), want)
    assert np.array_equal(np.signbit(f64(k)), np.signbit(want))


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_blocks_with_non_finite_elements(st, d):
    x = torch.randn((1, 20, 2, d), device=DEV).to(torch.bfloat16)
    x[0, 3, 0, 5], x[0, 17, 1, d - 1], x[0, 18, 0, 33] = float("inf"), float("nan"), float("-inf")
    c, _ = cache_of(st, np.random.default_rng(0), "mxfp4", 1, 2, 2, d)
    st.st_kv_append(pair(st, c), st.ST_SOURCE, x, x)
    k, v = read(st, pair(st, c), st.ST_SOURCE, 1, 20)
    want = L.mxfp4(f64(x))
    assert np.isnan(want).sum() == 3 * 32 and same(f64(k), want) and same(f64(v), want)


@pytest.mark.gpu
@pytest.mark.parametrize("store", FORMATS)
@pytest.mark.parametrize("hkv,d,batch,chunks", [(8, 128, 3, (1, 40, 16, 7)), (1, 64, 2, (17, 1, 1, 30)), (3, 64, 1, (33, 15)), (5, 128, 33, (2, 50))])
def test_plain_rows_as_by_the_plain_append(st, store, hkv, d, batch, chunks):
    """Without weight and spec: bit for bit what st_kv_append stores, pools, scales and lengths, chunk after chunk with ragged counts."""
    rng, g = np.random.default_rng(hkv * d), gen(hkv + d)
    pages = -(-sum(chunks) // 16) + 1
    a, table = cache_of(st, rng, store, batch, pages, hkv, d)
    b = st.KVCache(a.n_pages, batch, pages, hkv, d, a.page_table, fill=0xab, fp8=store == "fp8", mxfp4=store == "mxfp4")
    ca, cb = pair(st, a), pair(st, b)
    rows = []
    for i, most in enumerate(chunks):
        k, v = rand_rows(g, batch, most, hkv, d), rand_rows(g, batch, most, hkv, d)
        n = rng.integers(0, most + 1, batch).astype(np.int32) if i else np.full(batch, most, np.int32)
        n_dev = None if i == 0 else torch.from_numpy(n).to(DEV)
        st.st_kv_append(ca, st.ST_SOURCE, k, v, n_new=n_dev)
        start = b.appended_len.clone() if i % 2 else None
        st.st_kv_append_norm_rope(cb, st.ST_SOURCE, k, v, None, None, start_len=start, n_new=n_dev)
        assert torch.equal(a.appended_len, b.appended_len)
        rows.append((k, v, n))
    for x, y in ((a.k_pool, b.k_pool), (a.v_pool, b.v_pool), (a.k_scale, b.k_scale), (a.v_scale, b.v_scale)):
        if x is not None:
            bits = lambda t: t.view(torch.uint8) if t.dtype != torch.bfloat16 else t.view(torch.int16)
            assert torch.equal(bits(x), bits(y))
    # and read back: what the format holds for the rows
    lens = a.appended_len.cpu().numpy()
    k_all, v_all = read(st, ca, st.ST_SOURCE, batch, int(lens.max()), n=lens.tolist())
    for i in range(batch):
        for got, which in ((k_all, 0), (v_all, 1)):
            x = np.concatenate([f64(r[which][i, :r[2][i]]) for r in rows])
            want = stored(store, x)
            assert np.array_equal(f64(got[i, :lens[i]]), want), (i, which)
        assert bool((k_all[i, lens[i]:] == 9.0).all()) and bool((v_all[i, lens[i]:] == -9.0).all())


@pytest.mark.gpu
def test_undefined_elements_of_8_bit_rows(st):
    """An undefined element of an 8-bit row leaves the others as they are: what st_kv_append stores."""
    rng, g = np.random.default_rng(6), gen(6)
    a, _ = cache_of(st, rng, "fp8", 2, 2, 3, 128)
    b = st.KVCache(a.n_pages, 2, 2, 3, 128, a.page_table, fill=0xab, fp8=True)
    k, v = rand_rows(g, 2, 21, 3, 128), rand_rows(g, 2, 21, 3, 128)
    k[0, 2, 1, 77], k[1, 20, 0, 0], v[1, 3, 2, 127] = float("nan"), float("nan"), float("nan")
    st.st_kv_append(pair(st, a), st.ST_SOURCE, k, v)
    st.st_kv_append_norm_rope(pair(st, b), st.ST_SOURCE, k, v, None, None)
    for x, y in ((a.k_pool, b.k_pool), (a.v_pool, b.v_pool), (a.k_scale.view(torch.int32), b.k_scale.view(torch.int32)), (a.v_scale.view(torch.int32), b.v_scale.view(torch.int32))):
        assert torch.equal(x, y)
    got, _ = read(st, pair(st, b), st.ST_SOURCE, 2, 21)
    assert int(torch.isnan(got).sum()) == 2
    # rotated as well: the element's pair
    spec, _ = spec_of(st)
    st.st_kv_append_norm_rope(pair(st, b), st.ST_SOURCE, k, v, None, spec, start_len=torch.zeros(2, dtype=torch.int32, device=DEV))
    got, _ = read(st, pair(st, b), st.ST_SOURCE, 2, 21)
    assert int(torch.isnan(got).sum()) == 4 and bool(torch.isnan(got[0, 2, 1, 13])) and bool(torch.isnan(got[0, 2, 1, 77]))


@pytest.mark.gpu
@pytest.mark.parametrize("store", FORMATS)
def test_undefined_and_huge_keys_through_the_norm(st, store):
    """Rows that 32 bits do not hold are formed in 64: elements of 2^70, of 2^-70 without eps, an undefined element (its whole row)."""
    d, n = 128, 24
    g = gen(7)
    c, _ = cache_of(st, np.random.default_rng(7), store, 1, 2, 1, d)
    x = torch.randn((1, n, 1, d), generator=g, device=DEV)
    x[0, 1::3] *= 2.0 ** 70
    x[0, 2::3] *= 2.0 ** -70
    x = x.to(torch.bfloat16)
    x[0, 5, 0, 9] = float("nan")
    w = (1.0 + 0.3 * torch.randn(d, generator=g, device=DEV)).to(torch.bfloat16)
    spec, rope = spec_of(st)
    st.st_kv_append_norm_rope(pair(st, c), st.ST_SOURCE, x, x, w, spec, eps=0.0)
    k, _ = read(st, pair(st, c), st.ST_SOURCE, 1, n)
    rows = [i for i in range(n) if i != 5]
    want = stored(store, L.bf16(L.norm_rope(f64(x)[0][rows], f64(w), np.array(rows), 0.0, *rope)))
    assert np.array_equal(f64(k)[0][rows], want) and bool(torch.isnan(k[0, 5]).all())


@pytest.mark.gpu
def test_unusual_weights(st):
    """Weights up to 2^100 on elements that the row's norm has made as small: products that 32 bits lose on the way."""
    d, n = 128, 16
    g = gen(8)
    x = torch.randn((1, n, 1, d), generator=g, device=DEV)
    x[..., 1::2] *= 2.0 ** -128                                  # bf16 values of few bits, below the smallest normal number
    w = 1.0 + 0.3 * torch.randn(d, generator=g, device=DEV)
    w[1::2] *= 2.0 ** 125
    x, w = x.to(torch.bfloat16), w.to(torch.bfloat16)
    spec, rope = spec_of(st)
    for store in FORMATS:
        c, _ = cache_of(st, np.random.default_rng(8), store, 1, 2, 1, d)
        st.st_kv_append_norm_rope(pair(st, c), st.ST_SOURCE, x, x, w, spec, eps=1e-6)
        k, _ = read(st, pair(st, c), st.ST_SOURCE, 1, n)
        assert np.array_equal(f64(k)[0], stored(store, L.bf16(L.norm_rope(f64(x)[0], f64(w), np.arange(n), 1e-6, *rope))))


@pytest.mark.gpu
@pytest.mark.parametrize("attention", [2.0 ** 25, 2.0 ** -25, 0.75])
@pytest.mark.parametrize("layout,rotary", [("half", 96), ("interleaved", 32), ("half", 128)])
def test_unusual_attention_factors(st, attention, layout, rotary):
    """Rotated dims of another size than the others, with a norm and without, in part of a page and in whole ones."""
    d, n = 128, 39
    g = gen(12)
    x = torch.randn((2, n, 3, d), generator=g, device=DEV).to(torch.bfloat16)
    w = (1.0 + 0.3 * torch.randn(d, generator=g, device=DEV)).to(torch.bfloat16)
    spec, rope = spec_of(st, rotary=rotary, layout=layout, attention=attention)
    for store in FORMATS:
        for weight in (w, None):
            c, _ = cache_of(st, np.random.default_rng(12), store, 2, 4, 3, d)
            start = torch.tensor([0, 9], dtype=torch.int32, device=DEV)
            st.st_kv_append_norm_rope(pair(st, c), st.ST_SOURCE, x, x, weight, spec, eps=1e-6, start_len=start)
            k = torch.zeros((2, n, 3, d), dtype=torch.bfloat16, device=DEV)
            st.st_kv_read(pair(st, c), st.ST_SOURCE, k, torch.zeros_like(k), first=start)
            for b, first in ((0, 0), (1, 9)):
                want = L.norm_rope(f64(x)[b], f64(weight) if weight is not None else None, np.arange(first, first + n), 1e-6, *rope)
                assert np.array_equal(f64(k)[b], stored(store, L.bf16(want))), (store, b)


@pytest.mark.gpu
@pytest.mark.parametrize("store", FORMATS)
def test_rows_for_more_tokens_than_there_are_pages(st, store):
    """max_new and max_n are strides and bounds: up to the largest number, whatever the page table holds."""
    B = st.binding
    d, most = 64, 2 ** 31 - 1
    c, _ = cache_of(st, np.random.default_rng(9), store, 1, 2, 2, d)
    dual, lib, p = pair(st, c), B.load_library(), lambda t: t.data_ptr()
    k, v = rand_rows(gen(9), 1, 21, 2, d), rand_rows(gen(10), 1, 21, 2, d)
    n = torch.tensor([21], dtype=torch.int32, device=DEV)
    stream = torch.cuda.current_stream().cuda_stream
    assert lib.st_kv_append_norm_rope(C.byref(dual.struct()), st.ST_SOURCE, p(k), 2 * d, p(v), 2 * d, None, p(n), most, 1, 32, None, 0.0, None, stream) == 0
    assert int(c.appended_len[0]) == 21
    out = [torch.full((1, 22, 2, d), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    assert lib.st_kv_read(C.byref(dual.struct()), st.ST_SOURCE, p(out[0]), p(out[1]), None, p(n), most, 1, stream) == 0
    for got, want in zip(out, (k, v)):
        assert np.array_equal(f64(got)[0, :21], stored(store, f64(want)[0])) and bool((got[0, 21] == 7.0).all())


@pytest.mark.gpu
def test_binding_refuses_what_the_kernels_cannot_take(st):
    c, table = cache_of(st, np.random.default_rng(3), "mxfp4", 2, 2, 2, 64)
    k = torch.zeros((2, 5, 2, 64), dtype=torch.bfloat16, device=DEV)
    i = torch.zeros(2, dtype=torch.int32, device=DEV)
    away = st.KVCache(c.n_pages, 2, 2, 2, 64, c.page_table, device="cpu", mxfp4=True)          # pools in host memory
    append = lambda cache=c, k=k, v=k, w=None, **kw: st.st_kv_append_norm_rope(pair(st, cache), st.ST_SOURCE, k, v, w, None, **kw)
    read = lambda cache=c, k=k, v=k.clone(), **kw: st.st_kv_read(pair(st, cache), st.ST_SOURCE, k, v, **kw)
    for call in (append, read):
        for bad in (dict(cache=away), dict(k=k.cpu()), dict(v=k.float()), dict(v=k[:, :4]), dict(k=k[:1])):
            with pytest.raises(TypeError):
                call(**bad)
    for bad in (dict(w=torch.ones(64, device=DEV)), dict(w=torch.ones(32, dtype=torch.bfloat16, device=DEV)), dict(start_len=i.long()), dict(n_new=i[:1]),
                dict(start_len=i.cpu()), dict(k=k.transpose(2, 3).contiguous().transpose(2, 3))):
        with pytest.raises(TypeError):
            append(**bad)
    for bad in (dict(first=i.long()), dict(n=i[:1]), dict(k=k.repeat(1, 2, 1, 1)[:, ::2])):
        with pytest.raises(TypeError):
            read(**bad)
    assert int(c.appended_len.abs().sum()) == 0


SPECS = [dict(), dict(layout="interleaved"), dict(rotary=32, scaling="linear", factor=3.0), dict(rotary=48, scaling="ntk", factor=2.0),
         dict(scaling="yarn", factor=4.0, original=4096), dict(layout="interleaved", rotary=16, scaling="yarn", factor=8.0, original=4096, attention=0.9)]


@pytest.mark.gpu
@pytest.mark.parametrize("store", FORMATS)
@pytest.mark.parametrize("i", range(len(SPECS)))
@pytest.mark.parametrize("norm", [True, False])
def test_normalised_and_rotated_keys(st, store, i, norm):
    """Keys in 64 bits, rounded to bf16 once, coded: value for value what the definition gives."""
    d, hkv, batch, most = (64, 128)[i % 2], (2, 8, 1)[i % 3], 2, (50, 1, 19)[i % 3]
    rng, g = np.random.default_rng(i), gen(100 + i)
    spec, rope = spec_of(st, dim=d, **SPECS[i])
    start, n = rng.integers(0, 3000, batch).astype(np.int32), np.array([most, rng.integers(0, most + 1)], np.int32)
    c, _ = cache_of(st, rng, store, batch, -(-(3000 + most) // 16), hkv, d)
    qkv = (torch.randn((batch, most, 2 * hkv, d), generator=g, device=DEV) * 2.0).to(torch.bfloat16)
    k_new, v_new = qkv[:, :, :hkv], qkv[:, :, hkv:]
    w = (1.0 + 0.3 * torch.randn(d, generator=g, device=DEV)).to(torch.bfloat16) if norm else None
    st.st_kv_append_norm_rope(pair(st, c), st.ST_SOURCE, k_new, v_new, w, spec, eps=1e-5, start_len=torch.from_numpy(start).to(DEV),
                              n_new=torch.from_numpy(n).to(DEV))
    assert np.array_equal(c.appended_len.cpu().numpy(), start + n)
    k, v = read(st, pair(st, c), st.ST_SOURCE, batch, most, first=start.tolist(), n=n.tolist())
    for b in range(batch):
        x = f64(k_new[b, :n[b]])
        want = L.bf16(L.norm_rope(x, f64(w), start[b] + np.arange(n[b]), 1e-5, *rope))
        want_k, want_v = stored(store, want), stored(store, f64(v_new[b, :n[b]]))
        assert np.array_equal(f64(k[b, :n[b]]), want_k) and np.array_equal(f64(v[b, :n[b]]), want_v)
        assert bool((k[b, n[b]:] == 9.0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("store", FORMATS)
def test_only_the_new_tokens_slots_are_written(st, store):
    """Slots before and behind the new tokens keep their bytes; tokens past the page table and on page ids outside the pool are dropped."""
    rng, g = np.random.default_rng(8), gen(8)
    batch, pages, hkv, d = 3, 3, 2, 64
    c, table = cache_of(st, rng, store, batch, pages, hkv, d)
    c.page_table[1, 1] = c.n_pages + 5
    c.page_table[1, 2] = -1
    ca = pair(st, c)
    first_k, first_v = rand_rows(g, batch, 48, hkv, d), rand_rows(g, batch, 48, hkv, d)
    st.st_kv_append_norm_rope(ca, st.ST_SOURCE, first_k, first_v, None, None)
    before = read(st, ca, st.ST_SOURCE, batch, 48)
    k, v = rand_rows(g, batch, 21, hkv, d), rand_rows(g, batch, 21, hkv, d)
    start = [13, 5, 40]
    st.st_kv_append_norm_rope(ca, st.ST_SOURCE, k, v, None, None, start_len=torch.tensor(start, dtype=torch.int32, device=DEV))
    assert c.appended_len.tolist() == [34, 26, 48]
    after = read(st, ca, st.ST_SOURCE, batch, 48)
    for b in range(batch):
        lo, hi = start[b], min(start[b] + 21, 48)
        for x, y in zip(before, after):
            assert torch.equal(x[b, :lo], y[b, :lo]) and torch.equal(x[b, hi:], y[b, hi:])
    for b in (0, 2):
        assert not torch.equal(before[0][b, start[b]:start[b] + 8], after[0][b, start[b]:start[b] + 8])
    # sequence 1: its second and third page are not in the pool, its rows there neither written nor read
    assert bool((after[0][1, 16:] == 9.0).all()) and bool((after[1][1, 16:] == -9.0).all())
    # pages of nobody
    used = set(table.reshape(-1).tolist()) - {int(table[1, 1]), int(table[1, 2])}
    spare = [p for p in range(c.n_pages) if p not in used]
    raw = c.k_pool[spare]
    assert bool((raw == (171.0 if store == "bf16" else 0xab)).all())


@pytest.mark.gpu
@pytest.mark.parametrize("store", FORMATS)
def test_lengths_and_empty_calls(st, store):
    rng = np.random.default_rng(1)
    c, _ = cache_of(st, rng, store, 4, 2, 2, 128)
    ca = pair(st, c)
    x = torch.randn((4, 5, 2, 128), device=DEV).to(torch.bfloat16)
    dev = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
    st.st_kv_append_norm_rope(ca, st.ST_SOURCE, x, x, None, None, n_new=dev([0, 5, -3, 99]))
    assert c.appended_len.tolist() == [0, 5, 0, 5]
    st.st_kv_append_norm_rope(ca, st.ST_SOURCE, x, x, None, None, start_len=dev([-4, 3, 30, 77]), n_new=dev([1, 0, 5, 5]))
    assert c.appended_len.tolist() == [1, 3, 32, 32]
    st.st_kv_append_norm_rope(ca, st.ST_SOURCE, x[:, :0], x[:, :0], None, None, start_len=dev([7, 0, 2, 9]))
    assert c.appended_len.tolist() == [7, 0, 2, 9]
    one = x[:, :1].contiguous()
    st.st_kv_append_norm_rope(ca, st.ST_SOURCE, one, one, None, None)
    assert c.appended_len.tolist() == [8, 1, 3, 10]
    # the cache's own lengths as start_len: the same as none given
    st.st_kv_append_norm_rope(ca, st.ST_SOURCE, x, x, None, None, start_len=c.appended_len)
    assert c.appended_len.tolist() == [13, 6, 8, 15]
    k, v = read(st, ca, st.ST_SOURCE, 4, 40, first=[-1, 31, 40, 2], n=[3, 9, 4, -1])
    assert bool((k[0, 3:] == 9.0).all()) and bool((k[1, 1:] == 9.0).all()) and bool((k[2:] == 9.0).all())
    st.st_kv_read(ca, st.ST_SOURCE, k[:, :0].contiguous(), v[:, :0].contiguous())


@pytest.mark.gpu
@pytest.mark.parametrize("store,hkv,d", [("mxfp4", 8, 128), ("fp8", 8, 128), ("bf16", 8, 64)])
def test_pools_past_4_gib(st, store, hkv, d):
    rng, g = np.random.default_rng(2), gen(2)
    per = {"mxfp4": d // 2, "fp8": d, "bf16": 2 * d}[store] * hkv * 16
    n_pages = 2 ** 32 // per + 40
    table = torch.tensor([[n_pages - 1, 3], [n_pages - 2, n_pages - 40]], dtype=torch.int32, device=DEV)
    c = st.KVCache(n_pages, 2, 2, hkv, d, table, fp8=store == "fp8", mxfp4=store == "mxfp4")
    small = st.KVCache(4, 2, 2, hkv, d, torch.tensor([[0, 1], [2, 3]], dtype=torch.int32, device=DEV), fp8=store == "fp8", mxfp4=store == "mxfp4")
    k, v = rand_rows(g, 2, 27, hkv, d), rand_rows(g, 2, 27, hkv, d)
    spec, _ = spec_of(st, dim=d)
    got = []
    for x in (c, small):
        st.st_kv_append_norm_rope(pair(st, x), st.ST_SOURCE, k, v, None, spec)
        got.append(read(st, pair(st, x), st.ST_SOURCE, 2, 27))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


@pytest.mark.gpu
def test_rope_append_of_4_bits(st):
    """st_kv_append_rope into a 4-bit cache: the plain spec."""
    rng, g = np.random.default_rng(3), gen(3)
    c, _ = cache_of(st, rng, "mxfp4", 2, 4, 4, 128)
    e = st.KVCache(c.n_pages, 2, 4, 4, 128, c.page_table, fill=0xab, mxfp4=True)
    for most in (20, 1, 9):
        k, v = rand_rows(g, 2, most, 4, 128), rand_rows(g, 2, most, 4, 128)
        st.st_kv_append_rope(pair(st, c), st.ST_SOURCE, k, v, 1.0e4)
        st.st_kv_append_norm_rope(pair(st, e), st.ST_SOURCE, k, v, None, st.RopeSpec(theta_base=1.0e4))
    assert torch.equal(c.k_pool, e.k_pool) and torch.equal(c.v_pool, e.v_pool) and torch.equal(c.k_scale, e.k_scale)


@pytest.mark.gpu
@pytest.mark.parametrize("store", FORMATS)
def test_graph_replays_and_other_streams(st, store):
    rng, g = np.random.default_rng(4), gen(4)
    c, _ = cache_of(st, rng, store, 3, 5, 2, 128)
    e = st.KVCache(c.n_pages, 3, 5, 2, 128, c.page_table, fill=0xab, fp8=store == "fp8", mxfp4=store == "mxfp4")
    k, v = rand_rows(g, 3, 19, 2, 128), rand_rows(g, 3, 19, 2, 128)
    w = torch.ones(128, dtype=torch.bfloat16, device=DEV)
    spec, _ = spec_of(st)
    start = torch.tensor([0, 16, 30], dtype=torch.int32, device=DEV)
    outs = [torch.zeros_like(k), torch.zeros_like(v)]

    def call(cache, outs):
        ca = pair(st, cache)
        st.st_kv_append_norm_rope(ca, st.ST_SOURCE, k, v, w, spec, start_len=start)
        st.st_kv_read(ca, st.ST_SOURCE, *outs, first=start)

    call(c, outs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(c, outs)
    for turn in range(4):
        k.copy_(torch.randn_like(k))
        start.copy_(torch.tensor([turn, 16 + 3 * turn, 30 + turn], dtype=torch.int32))
        ref = [torch.zeros_like(k), torch.zeros_like(v)]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call(e, ref)
        torch.cuda.current_stream().wait_stream(side)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], ref[0]) and torch.equal(outs[1], ref[1]) and torch.equal(c.appended_len, e.appended_len), turn
