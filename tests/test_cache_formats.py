"""What the calls on 4-bit caches, the append of rows from the projections and the read refuse (host checks, no GPU)."""
import ctypes as C
import os

import pytest

FAKE, OFF, OTHER = 0x10000, 0x10008, 0x20000          # never dereferenced: the checks come first


@pytest.fixture(scope="module")
def lib():
    import paper_2510_17238_amd as st
    if not os.path.exists(st.library_path()):
        import __graft_entry__
        __graft_entry__.build()
    return st.load_library()


def cache(B, **kw):
    a = dict(k_pool=FAKE, v_pool=FAKE, page_table=FAKE, appended_len=FAKE, max_pages_per_seq=4, n_pages=8, page_size=16, n_kv_heads=2, head_dim=128,
             dtype=B.ST_MXFP4, k_scale=FAKE, v_scale=None)
    a.update(kw)
    return B._KVCacheStruct(*[a[n] for n, _ in B._KVCacheStruct._fields_])


def dual(B, src=None, rsn=None):
    return B._DualCacheStruct(cache(B, **(src or {})), cache(B, **(rsn or {})))


def append(lib, B, caches=None, **kw):
    a = dict(which=B.ST_SOURCE, k=FAKE, ks=256, v=FAKE, vs=256, start=None, n=None, max_new=8, batch=1, bound=64, w=FAKE, eps=1e-6, spec=B.RopeSpec())
    a.update(kw)
    c = caches if caches is not None else dual(B)
    return lib.st_kv_append_norm_rope(C.byref(c), a["which"], a["k"], a["ks"], a["v"], a["vs"], a["start"], a["n"], a["max_new"], a["batch"], a["bound"],
                                      a["w"], a["eps"], None if a["spec"] is None else C.byref(a["spec"]), None)


def test_append_refusals(lib):
    import paper_2510_17238_amd.binding as B
    for code, kw in [(1, dict(k=None)), (1, dict(v=None)), (1, dict(k=OFF)), (1, dict(v=OFF)), (1, dict(which=2)), (1, dict(batch=0)), (1, dict(max_new=-1)),
                     (2, dict(ks=248)), (2, dict(vs=0)), (1, dict(ks=260)), (1, dict(vs=257)), (4, dict(bound=65)), (4, dict(bound=-1)), (1, dict(w=OFF)),
                     (1, dict(eps=-1.0)), (1, dict(eps=float("nan"))), (1, dict(spec=B.RopeSpec(theta_base=-1.0))), (5, dict(spec=B.RopeSpec(rotary_dim=8))),
                     (2, dict(batch=1 << 30, max_new=1 << 20))]:
        assert append(lib, B, **kw) == code, (kw, lib.st_last_error())
        assert b"st_kv_append_norm_rope" in lib.st_last_error()
    for code, kw in [(1, dict(k_pool=None)), (1, dict(k_pool=OFF)), (1, dict(k_scale=None)), (1, dict(k_scale=OFF)), (1, dict(page_table=None)),
                     (1, dict(appended_len=None)), (5, dict(page_size=32)), (5, dict(head_dim=96)), (5, dict(dtype=9)), (5, dict(dtype=B.ST_F32)), (1, dict(n_pages=0)),
                     (1, dict(dtype=B.ST_FP8_E4M3))]:
        assert append(lib, B, caches=dual(B, src=kw)) == code, (kw, lib.st_last_error())
    assert append(lib, B, max_new=0, k=None, v=None) == 0                                  # nothing to do
    assert lib.st_kv_append_norm_rope(None, 0, FAKE, 256, FAKE, 256, None, None, 8, 1, 64, None, 0.0, None, None) == 1


def test_append_refuses_lengths_that_it_writes(lib):
    import paper_2510_17238_amd.binding as B
    c = dual(B)
    own = c.source.appended_len
    call = lambda start, n: lib.st_kv_append_norm_rope(C.byref(c), B.ST_SOURCE, FAKE, 256, FAKE, 256, start, n, 8, 1, 65, None, 0.0, None, None)
    assert call(0x7000, own) == 1 and b"appended_len" in lib.st_last_error()
    assert call(None, own) == 4 and call(own, own) == 4                     # read before they are written: on to the next check
    assert append(lib, B, eps=float("inf")) == 1


def test_read_refusals(lib):
    import paper_2510_17238_amd.binding as B

    def read(src=None, **kw):
        a = dict(which=B.ST_SOURCE, k=FAKE, v=FAKE, first=None, n=None, max_n=8, batch=1)
        a.update(kw)
        c = dual(B, src=src)
        return lib.st_kv_read(C.byref(c), a["which"], a["k"], a["v"], a["first"], a["n"], a["max_n"], a["batch"], None)

    for code, kw in [(1, dict(k=None)), (1, dict(v=OFF)), (1, dict(which=-1)), (1, dict(batch=0)), (1, dict(max_n=-1)), (2, dict(batch=1 << 30, max_n=1 << 20))]:
        assert read(**kw) == code, (kw, lib.st_last_error())
        assert b"st_kv_read" in lib.st_last_error()
    assert read(src=dict(dtype=5)) == 5 and read(src=dict(k_scale=None)) == 1
    assert read(max_n=0, k=None, v=None) == 0


def test_calls_on_4_bit_caches(lib):
    """Which calls take them, and that the others say so."""
    import paper_2510_17238_amd.binding as B
    c = dual(B)
    ref = C.byref(c)
    assert lib.st_kv_append(ref, B.ST_SOURCE, FAKE, FAKE, None, 8, 1, 65, None) == 4         # passes the dtype check
    assert lib.st_kv_append_rope(ref, B.ST_SOURCE, FAKE, FAKE, None, 8, 1, 64, 0.0, None) == 1
    assert lib.st_kv_append_rope(ref, B.ST_SOURCE, FAKE, FAKE, None, 8, 1, 65, 1e6, None) == 4
    lens = B._DualLensStruct(FAKE, FAKE, 1, 64, 64, 0)
    assert lib.st_attn_decode_dual(FAKE, None, FAKE, ref, C.byref(lens), 1, 4, 0.0, None, 0, None) == 1       # no workspace
    assert lib.st_attn_decode_dual(FAKE, None, FAKE, ref, C.byref(lens), 1, 4, 0.0, FAKE, 256, None) == 4
    assert b"workspace" in lib.st_last_error()
    many = B._DualLensStruct(FAKE, FAKE, 17, 64, 64, 0)
    assert lib.st_attn_decode_dual(FAKE, None, FAKE, ref, C.byref(many), 1, 4, 0.0, FAKE, 1 << 30, None) == 5  # 34 rows
    mixed = dual(B, rsn=dict(dtype=B.ST_BF16))
    assert lib.st_attn_decode_dual(FAKE, None, FAKE, C.byref(mixed), C.byref(lens), 1, 4, 0.0, FAKE, 1 << 30, None) == 5
    assert lib.st_attn_decode_dual_append(FAKE, None, FAKE, FAKE, FAKE, ref, C.byref(lens), 1, 4, 0.0, 1e6, FAKE, 1 << 30, None) == 5
    assert lib.st_attn_source_chunk(FAKE, None, FAKE, ref, FAKE, None, 8, 64, 1, 4, 0.0, FAKE, 1 << 30, None) == 5
    assert b"4-bit" in lib.st_last_error()
