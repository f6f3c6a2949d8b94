"""Codes and scales of keys that 32 bits do not hold: those of the row in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import layer_ops as L
from rows_helpers import f64, spec_of
from test_gpu_cache_rows import DEV, cache_of, gen, pair, read, stored


@pytest.fixture(scope="module")
def st():
    import paper_2510_17238_amd as st
    return st


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
