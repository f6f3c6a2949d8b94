"""Plumbing of the tests of normalised, rotated and coded rows."""
import torch

from oracle import layer_ops as L


def spec_of(st, layout="half", rotary=0, scaling="plain", factor=1.0, original=0, theta=1.0e6, attention=0.0, dim=128):
    """(the library's spec, the oracle's (frequencies, factor, layout))."""
    kinds = {"plain": st.ST_ROPE_PLAIN, "linear": st.ST_ROPE_LINEAR, "ntk": st.ST_ROPE_NTK, "yarn": st.ST_ROPE_YARN}
    spec = st.RopeSpec(theta_base=theta, layout=st.ST_ROPE_HALF if layout == "half" else st.ST_ROPE_INTERLEAVED, rotary_dim=rotary,
                       scaling=kinds[scaling], factor=factor, original_positions=original, attention_factor=attention)
    freq, a = L.frequencies(rotary or dim, theta, scaling, factor, original)
    return spec, (freq, attention or a, layout)


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()
