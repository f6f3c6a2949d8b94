"""Heads normalised and rotated: the oracle against differences and known values, and what the library refuses (no GPU)."""
import ctypes as C

import numpy as np
import pytest

from oracle import layer_ops as L


@pytest.fixture(scope="module")
def lib():
    import os
    import paper_2510_17238_amd as st
    if not os.path.exists(st.library_path()):
        import __graft_entry__
        __graft_entry__.build()
    return st.load_library()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rotary,scaling,factor", [(64, "plain", 1.0), (32, "yarn", 4.0), (48, "ntk", 2.0), (16, "linear", 3.0)])
def test_oracle_gradients_are_differences(layout, rotary, scaling, factor):
    rng = np.random.default_rng(rotary)
    freq, a = L.frequencies(rotary, scaling=scaling, factor=factor, original_positions=4096)
    x, w, g = rng.standard_normal((3, 2, 64)), 1 + 0.3 * rng.standard_normal(64), rng.standard_normal((3, 2, 64))
    pos = np.array([0, 5, 4000])
    loss = lambda x, w: (L.norm_rope(x, w, pos, 1e-3, freq, a, layout) * g).sum()
    dx, dw = L.norm_rope_bwd(g, x, w, pos, 1e-3, freq, a, layout)
    step = 1e-5
    for _ in range(40):
        i = tuple(rng.integers(0, s) for s in x.shape)
        e = np.zeros_like(x)
        e[i] = step
        assert abs((loss(x + e, w) - loss(x - e, w)) / (2 * step) - dx[i]) < 1e-7
        e = np.zeros_like(w)
        e[i[2]] = step
        assert abs((loss(x, w + e) - loss(x, w - e)) / (2 * step) - dw[i[2]]) < 1e-7


def test_oracle_rotation_is_relative():
    """Rotated rows' products depend on the difference of their positions alone."""
    rng = np.random.default_rng(0)
    freq, a = L.frequencies(64)
    x, y = rng.standard_normal((1, 1, 64)), rng.standard_normal((1, 1, 64))
    dot = lambda i, j: (L.rotate(x, np.array([i]), freq, a, "half") * L.rotate(y, np.array([j]), freq, a, "half")).sum()
    assert abs(dot(10, 3) - dot(1007, 1000)) < 1e-9 and abs(dot(10, 3) - dot(10, 4)) > 1e-3


def test_oracle_frequencies():
    plain, one = L.frequencies(128)
    assert one == 1.0 and plain[0] == 1.0 and abs(plain[64 - 1] - 1e6 ** (-126 / 128)) < 1e-18
    yarn, a = L.frequencies(128, scaling="yarn", factor=4.0, original_positions=32768)
    # pairs that turn often keep their frequency, pairs that turn less than once over the trained length are slowed by the factor
    turns = plain * 32768 / (2 * np.pi)
    assert np.array_equal(yarn[turns > 64], plain[turns > 64]) and np.allclose(yarn[turns < 0.5], plain[turns < 0.5] / 4.0, rtol=1e-15)
    assert abs(a - (0.1 * np.log(4.0) + 1.0)) < 1e-15 and (np.diff(yarn) < 0).all()
    ntk, _ = L.frequencies(128, scaling="ntk", factor=4.0)
    assert ntk[0] == 1.0 and abs(ntk[-1] / plain[-1] - 0.25) < 1e-12


def test_oracle_codes():
    x = np.zeros(32)
    x[:12] = [6.0, 5.0, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, -5.0, 0.2500001, 4.9999, -0.2]
    assert np.array_equal(L.mxfp4(x)[:12], [6.0, 4.0, 4.0, 2.0, 2.0, 1.0, 1.0, 0.0, -4.0, 0.5, 4.0, 0.0])
    assert np.array_equal(L.mxfp4(np.full(32, 6.5)), np.full(32, 6.0)) and np.array_equal(L.mxfp4(np.full(32, -7.5)), np.full(32, -8.0))
    assert np.array_equal(L.mxfp4(np.zeros(64)), np.zeros(64))
    y = np.concatenate([np.full(32, np.inf), np.ones(32)])
    assert np.isnan(L.mxfp4(y)[:32]).all() and np.array_equal(L.mxfp4(y)[32:], np.ones(32))


FAKE, OFF = 0x1000, 0x1008          # never dereferenced: the checks come first


def _fwd(lib, B, **kw):
    spec = kw.pop("spec", B.RopeSpec())
    a = dict(q_out=FAKE, q=FAKE, qs=512, hq=4, wq=FAKE, k_out=FAKE, k=FAKE, ks=256, hkv=2, wk=FAKE, pos=FAKE, n=5, d=128, eps=1e-6, dt=B.ST_BF16)
    a.update(kw)
    return lib.st_norm_rope_apply_qk(a["q_out"], a["q"], a["qs"], a["hq"], a["wq"], a["k_out"], a["k"], a["ks"], a["hkv"], a["wk"], a["pos"], a["n"],
                                     a["d"], a["eps"], C.byref(spec) if spec is not None else None, a["dt"], None)


def test_forward_refusals(lib):
    import paper_2510_17238_amd.binding as B
    S = B.RopeSpec
    bad = [
        (1, dict(q=None)), (1, dict(q_out=None)), (1, dict(k=None)), (1, dict(k_out=None)), (1, dict(pos=None)), (1, dict(spec=None)),
        (1, dict(q=OFF)), (1, dict(k_out=OFF)), (1, dict(wq=OFF)), (1, dict(hq=0)), (1, dict(hkv=-1)), (1, dict(n=-1)), (1, dict(eps=-1.0)),
        (1, dict(eps=float("nan"))), (2, dict(qs=504)), (2, dict(ks=128)), (1, dict(qs=516)), (1, dict(qs=520)), (5, dict(d=96)), (5, dict(dt=B.ST_FP8_E4M3)),
        (1, dict(spec=S(theta_base=0.0))), (1, dict(spec=S(theta_base=float("nan")))), (1, dict(spec=S(layout=2))), (5, dict(spec=S(rotary_dim=24))),
        (2, dict(spec=S(rotary_dim=144))), (2, dict(spec=S(rotary_dim=-16))), (1, dict(spec=S(scaling=4))), (1, dict(spec=S(scaling=1, factor=0.5))),
        (1, dict(spec=S(scaling=3, factor=2.0))), (1, dict(spec=S(scaling=3, factor=2.0, original_positions=4096, beta_fast=1.0, beta_slow=2.0))),
        (1, dict(spec=S(attention_factor=-1.0))), (1, dict(spec=S(scaling=2, factor=float("inf")))), (1, dict(spec=S(scaling=3, factor=2.0, original_positions=64, theta_base=1.0))),
    ]
    for code, kw in bad:
        assert _fwd(lib, B, **kw) == code, (kw, lib.st_last_error())
        assert b"st_norm_rope_apply_qk" in lib.st_last_error()
    assert _fwd(lib, B, n=0) == 0 and _fwd(lib, B, n=0, q=None, q_out=None, pos=None) == 0


def test_gradient_refusals(lib):
    import paper_2510_17238_amd.binding as B

    def bwd(**kw):
        spec = B.RopeSpec()
        a = dict(dq=0x2000, dqs=512, dwq=FAKE, gq=FAKE, q=FAKE, qs=512, hq=4, wq=FAKE, dk=0x2000, dks=256, dwk=FAKE, gk=FAKE, k=FAKE, ks=256, hkv=2, wk=FAKE,
                 pos=FAKE, n=5, d=128, eps=1e-6, dt=B.ST_BF16, ws=FAKE, wb=1 << 20)
        a.update(kw)
        return lib.st_norm_rope_bwd_qk(a["dq"], a["dqs"], a["dwq"], a["gq"], a["q"], a["qs"], a["hq"], a["wq"], a["dk"], a["dks"], a["dwk"], a["gk"], a["k"],
                                       a["ks"], a["hkv"], a["wk"], a["pos"], a["n"], a["d"], a["eps"], C.byref(spec), a["dt"], a["ws"], a["wb"], None)

    need = lib.st_norm_rope_bwd_workspace_bytes(5, 4, 2, 128)
    assert need == 5 * 2 * 128 * 4 and lib.st_norm_rope_bwd_workspace_bytes(1 << 20, 4, 2, 128) == 1024 * 2 * 128 * 4
    assert lib.st_norm_rope_bwd_workspace_bytes(-1, 4, 2, 128) == 0
    for code, kw in [(1, dict(dq=None)), (1, dict(gq=None)), (1, dict(q=None)), (1, dict(ws=None)), (1, dict(ws=OFF)), (4, dict(wb=need - 1)), (1, dict(wq=None)),
                     (1, dict(dwk=0x1002)), (2, dict(dks=248)), (1, dict(dqs=516)), (1, dict(q=0x2000, qs=1024)), (1, dict(gq=0x2000, dqs=1024)), (5, dict(dt=7)),
                     (1, dict(hkv=0)), (1, dict(pos=None)), (5, dict(d=32)), (1, dict(eps=-1e-3)), (1, dict(gk=OFF))]:
        assert bwd(**kw) == code, (kw, lib.st_last_error())
        assert b"st_norm_rope_bwd_qk" in lib.st_last_error()


def test_refusals_of_sizes_and_shared_results(lib):
    import paper_2510_17238_amd.binding as B
    for code, kw in [(2, dict(hq=65537, qs=65537 * 128)), (2, dict(hkv=65537, ks=65537 * 128)), (2, dict(n=2 ** 40 + 1)), (1, dict(eps=float("inf")))]:
        assert _fwd(lib, B, **kw) == code, (kw, lib.st_last_error())
    spec = B.RopeSpec()

    def bwd(dwq, dwk, hkv=2, eps=1e-6):
        return lib.st_norm_rope_bwd_qk(0x2000, 512, dwq, FAKE, FAKE, 512, 4, FAKE, 0x4000, 256, dwk, FAKE, FAKE, 256, hkv, FAKE, FAKE, 5, 128, eps, C.byref(spec),
                                       B.ST_BF16, FAKE, 1 << 20, None)
    assert bwd(0x8000, 0x8000) == 1 and b"one array" in lib.st_last_error()
    assert bwd(0x8000, 0x9000, hkv=65537) == 2 and bwd(0x8000, 0x9000, eps=float("inf")) == 1


def test_binding_refusals():
    import torch
    import paper_2510_17238_amd as st
    x = torch.zeros((3, 2, 128), dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        st.st_norm_rope_apply_qk(x, None, None, None, torch.zeros(3, dtype=torch.int32), st.RopeSpec())       # host tensors
