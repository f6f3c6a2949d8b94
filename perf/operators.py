"""What lies between a layer's projections and its attention, as cases that can be timed.

Four parts of an attention layer whose heads are normalised (the Qwen3 shapes of the benchmark): queries and keys
normalised per head and rotated in one pass, the gradients of that pass, new keys and values on their way into a paged
cache (and rows read back out of it), and decoding over a pair of caches held in 4 bits.  The structures (cache lengths, new
tokens per stream) follow from the case alone, the values from the seed.

Every part has a plain form in elementary torch operations.  `own` selects the library's calls instead.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
EPS = 1.0e-6
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------ the cases
def _rows(name, op, dtype, tokens, heads, dim, fused, layout, rotary, scaling, factor, original, positions):
    """`tokens` tokens of heads[0] query and heads[1] KV heads at stream positions below `positions`; fused: queries and keys are
    slices of one projection's output; rotary: leading dims that are rotated."""
    return {"name": name, "op": op, "dtype": dtype, "tokens": tokens, "q_heads": heads[0], "kv_heads": heads[1], "head_dim": dim,
            "fused": fused, "layout": layout, "rotary": rotary, "scaling": scaling, "factor": factor, "original": original,
            "positions": positions}


def _append(name, store, batch, new, cached, kv_heads, dim, layout, rotary, scaling, factor, original, lens):
    """new[0] .. new[1] tokens for each of `batch` streams that hold up to `cached` already; store: what the cache holds."""
    return {"name": name, "op": "append", "store": store, "batch": batch, "new_lo": new[0], "new_hi": new[1], "cached": cached,
            "kv_heads": kv_heads, "head_dim": dim, "layout": layout, "rotary": rotary, "scaling": scaling, "factor": factor,
            "original": original, "lens": lens}


def _decode(name, batch, src, rsn, new, heads, dim, lens):
    """`new` reasoning tokens of each stream over src[0] .. src[1] source and rsn[0] .. rsn[1] reasoning tokens in 4 bits."""
    return {"name": name, "op": "decode", "batch": batch, "src_lo": src[0], "src_hi": src[1], "rsn_lo": rsn[0], "rsn_hi": rsn[1],
            "new": new, "q_heads": heads[0], "kv_heads": heads[1], "head_dim": dim, "lens": lens}


def listed():
    return [
        # the smallest: one token of one listener on its way to the attention, bound by latency
        _rows("norm_rope_token", "norm_rope", "bf16", 1, (32, 8), 128, True, "half", 128, "plain", 1.0, 0, 4096),
        # prefill of eight long documents, 16K tokens each, straight out of the fused projection
        _rows("norm_rope_8x16k", "norm_rope", "bf16", 131072, (32, 8), 128, True, "half", 128, "plain", 1.0, 0, 16384),
        # a numerics study in full precision: half of each head rotated, neighbouring dims paired, positions past the trained length
        _rows("norm_rope_f32_yarn", "norm_rope", "f32", 4099, (16, 2), 64, False, "interleaved", 32, "yarn", 4.0, 32768, 131072),
        # fine-tuning step of a small model's layer: four sequences of about 4K tokens
        _rows("norm_rope_bwd_4x4k", "norm_rope_bwd", "bf16", 16001, (16, 8), 128, True, "half", 128, "plain", 1.0, 0, 4200),
        # gradients of a short ragged batch in full precision, three quarters of each head rotated
        _rows("norm_rope_bwd_f32", "norm_rope_bwd", "f32", 1801, (16, 8), 128, False, "half", 96, "ntk", 2.0, 0, 8192),
        # serving: one decoded token of each of 64 streams stored in 4 bits
        _append("append_token_64", "mxfp4", 64, (1, 1), 16384, 8, 128, "half", 128, "plain", 1.0, 0, 1),
        # an arriving sentence for each of 64 streams, in 4 bits
        _append("append_sentence_64", "mxfp4", 64, (7, 190), 8192, 8, 128, "half", 128, "plain", 1.0, 0, 2),
        # documents taken in whole: sixteen of up to 4K tokens, in 4 bits
        _append("append_document_16", "mxfp4", 16, (1500, 4096), 0, 8, 128, "half", 128, "yarn", 4.0, 32768, 3),
        # one listener: a token over a hundred source and a few hundred reasoning tokens, bound by latency
        _decode("decode_listener", 1, (96, 96), (300, 300), 1, (32, 8), 128, 4),
        # serving: 32 streams, 2K source and 1K to 6K reasoning tokens
        _decode("decode_32", 32, (2048, 2048), (1024, 6144), 1, (16, 8), 128, 5),
        # 64 long streams, the largest cache
        _decode("decode_64_long", 64, (1024, 8192), (2048, 24576), 1, (32, 8), 128, 6),
        # the same kind of streams, eight drafted tokens verified in one call
        _decode("decode_64_of_8", 64, (1024, 8192), (2048, 16384), 8, (32, 8), 128, 7),
    ]


def _log(rng, lo, hi):
    """An integer of [lo, hi], spread over the logarithm."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def _draw_rotation(rng, dim):
    scaling = rng.choice(("plain", "plain", "linear", "ntk", "yarn"))
    original = rng.choice((4096, 32768)) if scaling == "yarn" else 0
    return (rng.choice(("half", "half", "interleaved")), rng.choice([r for r in (16, 32, 64, 96, 128) if r <= dim] + [dim, dim]), scaling,
            1.0 if scaling == "plain" else rng.choice((1.5, 2.0, 4.0, 8.0)), original)


def draw(rng):
    op = rng.choice(("norm_rope", "norm_rope", "norm_rope_bwd", "norm_rope_bwd", "append", "append", "append", "decode", "decode", "decode"))
    dim = rng.choice((64, 128, 128))
    heads = rng.choice(((16, 8), (32, 8), (16, 2), (8, 4), (5, 1)))
    if op in ("norm_rope", "norm_rope_bwd"):
        dtype = rng.choice(("bf16", "bf16", "f32"))
        most = {"norm_rope": 100000, "norm_rope_bwd": 16000}[op] // (2 if dtype == "f32" else 1)
        case = _rows("", op, dtype, _log(rng, 1, most), heads, dim, rng.random() < 0.5, *_draw_rotation(rng, dim), _log(rng, 64, 131072))
    elif op == "append":
        batch = _log(rng, 1, 64)
        top = _log(rng, 1, 32768 // batch)
        case = _append("", rng.choice(("mxfp4", "mxfp4", "fp8", "bf16")), batch, (rng.choice((0, top // 3, top)), top), _log(rng, 1, 16384),
                       heads[1], dim, *_draw_rotation(rng, dim), rng.randrange(1 << 20))
    else:
        batch = _log(rng, 1, 64)
        new = rng.choice((1, 1, 2, 4, 32 * heads[1] // heads[0]))
        new = max(1, min(new, 32 * heads[1] // heads[0]))
        src, rsn = _log(rng, 16, 8192), max(new, _log(rng, 16, 16384))
        lo = rng.choice((0.0, 0.3, 1.0))
        case = _decode("", batch, (int(src * lo), src), (max(new, int(rsn * lo)), rsn), new, heads, dim, rng.randrange(1 << 20))
    del case["name"]
    return case


# ------------------------------------------------------------------ structures: from the case alone
def _new_tokens(case):
    """(tokens cached, tokens arriving) of every stream."""
    rng = np.random.default_rng([case["lens"], 1])
    start = rng.integers(0, case["cached"] + 1, case["batch"])
    return start.astype(np.int32), rng.integers(case["new_lo"], case["new_hi"] + 1, case["batch"]).astype(np.int32)


def _cache_lengths(case):
    """(source tokens, reasoning tokens with the new ones) of every stream; the longest of either has the full length."""
    rng = np.random.default_rng([case["lens"], 2])
    src = rng.integers(case["src_lo"], case["src_hi"] + 1, case["batch"]).astype(np.int32)
    rsn = rng.integers(case["rsn_lo"], case["rsn_hi"] + 1, case["batch"]).astype(np.int32)
    src[rng.integers(case["batch"])] = case["src_hi"]
    rsn[rng.integers(case["batch"])] = case["rsn_hi"]
    return src, rsn


def _pages(rng, batch, tokens):
    """Pages per stream for `tokens` tokens, and a shuffled table of them."""
    per = max(1, -(-tokens // PAGE))
    return per, rng.permutation(batch * per).astype(np.int32).reshape(batch, per)


def _row_bytes(store, dim):
    """Bytes that a cache holds for one row: codes and scales."""
    return {"bf16": 2 * dim, "fp8": dim + 4, "mxfp4": dim // 2 + dim // 32}[store]


def work(case):
    d, hkv = case["head_dim"], case["kv_heads"]
    if case["op"] in ("norm_rope", "norm_rope_bwd"):
        rows = case["tokens"] * (case["q_heads"] + hkv)
        size = 2 if case["dtype"] == "bf16" else 4
        if case["op"] == "norm_rope":               # x in, y out; sums, scale, weight, rotation
            return {"bytes": rows * d * size * 2 + case["tokens"] * 4, "flops": rows * d * 8}
        return {"bytes": rows * d * size * 3 + case["tokens"] * 4 + 16 * d, "flops": rows * d * 20}
    if case["op"] == "append":
        rows = int(_new_tokens(case)[1].sum()) * hkv * 2
        # rows in, codes out; codes in, rows out
        return {"bytes": rows * (4 * d + 2 * _row_bytes(case["store"], d)), "flops": rows * d * 8}
    src, rsn = _cache_lengths(case)
    tokens = int(src.sum()) + int(rsn.sum())
    rows = case["batch"] * case["new"] * case["q_heads"]
    pairs = case["new"] * tokens - case["batch"] * case["new"] * (case["new"] - 1) // 2
    return {"bytes": tokens * hkv * 2 * _row_bytes("mxfp4", d) + rows * d * 4, "flops": 4 * d * case["q_heads"] * pairs}


# ------------------------------------------------------------------ inputs
def _spec(case):
    import paper_2510_17238_amd as st
    return st.RopeSpec(theta_base=1.0e6, layout={"half": st.ST_ROPE_HALF, "interleaved": st.ST_ROPE_INTERLEAVED}[case["layout"]],
                       rotary_dim=case["rotary"], factor=case["factor"], original_positions=case["original"],
                       scaling={"plain": st.ST_ROPE_PLAIN, "linear": st.ST_ROPE_LINEAR, "ntk": st.ST_ROPE_NTK,
                                "yarn": st.ST_ROPE_YARN}[case["scaling"]])


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _projected(g, shape, dtype):
    """What a projection leaves: some dims carry several times what the others do."""
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    return (x * (0.6 + 2.4 * torch.rand(shape[-1:], generator=g, device="cuda") ** 3)).to(dtype)


def _weight(g, dim, dtype):
    return (1.0 + 0.3 * torch.randn(dim, generator=g, device="cuda")).to(dtype)


def prepare(case, seed):
    g = _gen(seed)
    state = {"case": case}
    return {"norm_rope": _prepare_rows, "norm_rope_bwd": _prepare_rows, "append": _prepare_append, "decode": _prepare_decode}[case["op"]](case, g, seed, state)


def _prepare_rows(case, g, seed, state):
    n, hq, hkv, d, dtype = case["tokens"], case["q_heads"], case["kv_heads"], case["head_dim"], DTYPES[case["dtype"]]
    if case["fused"]:
        qkv = _projected(g, (n, hq + 2 * hkv, d), dtype)
        state["q"], state["k"] = qkv[:, :hq], qkv[:, hq:hq + hkv]
    else:
        state["q"], state["k"] = _projected(g, (n, hq, d), dtype), _projected(g, (n, hkv, d), dtype)
    state["q_weight"], state["k_weight"] = _weight(g, d, dtype), _weight(g, d, dtype)
    state["pos"] = ((torch.arange(n, device="cuda") + int(seed) * 977) % case["positions"]).to(torch.int32)
    if case["op"] == "norm_rope_bwd":
        state["d_q"] = torch.randn((n, hq, d), generator=g, device="cuda").to(dtype)
        state["d_k"] = torch.randn((n, hkv, d), generator=g, device="cuda").to(dtype)
    if own:
        import paper_2510_17238_amd as st
        state["spec"] = _spec(case)
        state["q_out"], state["k_out"] = (torch.empty(x.shape, dtype=dtype, device="cuda") for x in (state["q"], state["k"]))
        if case["op"] == "norm_rope_bwd":
            state["ws"] = torch.empty(max(256, st.st_norm_rope_bwd_workspace_bytes(n, hq, hkv, d)), dtype=torch.uint8, device="cuda")
    return state


def _append_inputs(case, g):
    b, most, hkv, d = case["batch"], max(1, case["new_hi"]), case["kv_heads"], case["head_dim"]
    return (_projected(g, (b, most, hkv, d), torch.bfloat16), torch.randn((b, most, hkv, d), generator=g, device="cuda").to(torch.bfloat16),
            _weight(g, d, torch.bfloat16))


def _prepare_append(case, g, seed, state):
    b, hkv, d = case["batch"], case["kv_heads"], case["head_dim"]
    state["k_new"], state["v_new"], state["k_weight"] = _append_inputs(case, g)
    start, n = _new_tokens(case)
    state["start"], state["n"] = torch.from_numpy(start).to("cuda"), torch.from_numpy(n).to("cuda")
    # (rows past a stream's tokens are left as they are)
    state["k_out"], state["v_out"] = torch.zeros_like(state["k_new"]), torch.zeros_like(state["v_new"])
    if own:
        import paper_2510_17238_amd as st
        state["spec"] = _spec(case)
        rng = np.random.default_rng([int(seed), 3])
        caches = []
        for tokens in (PAGE, int((start + n).max())):
            per, table = _pages(rng, b, tokens)
            caches.append(st.KVCache(b * per, b, per, hkv, d, torch.from_numpy(table).to("cuda"), fp8=case["store"] == "fp8", mxfp4=case["store"] == "mxfp4"))
        state["caches"] = st.DualCache(*caches)
        state["bound"] = int((start + n).max())
    return state


def _two_to(k):
    """2^k in 32 bits for whole k from -126 on, exactly."""
    return ((k.to(torch.int32) + 127) << 23).view(torch.float32)


def _code_rows(x):
    """bf16 rows -> (4-bit codes as bytes, scale exponents) per block of 32: the E2M1 value nearest to x / 2^k, ties to the even code, k the
    smallest integer from -100 on with max |x| <= 6 * 2^k (0 where all are zero)."""
    f = x.float().reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    top = f.abs().amax(-1)
    k = torch.zeros_like(top, dtype=torch.int32)
    m, e = torch.frexp(torch.where(top > 0, top, torch.ones_like(top)))
    k = torch.where(top > 0, torch.clamp(e - 3 + (m > 0.75).to(torch.int32), min=-100), k)      # 6 = 0.75 * 2^3
    y = (f * _two_to(-k)[..., None]).abs()
    lines = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=x.device)
    code = torch.zeros_like(y, dtype=torch.uint8)
    for i in range(7):                          # past the line between codes i and i + 1; on it, the even one of the two
        code += (y > lines[i]) if i % 2 == 0 else (y >= lines[i])
    code += torch.where(torch.signbit(f), 8, 0).to(torch.uint8)
    return code.reshape(x.shape), k


def _prepare_decode(case, g, seed, state):
    b, hkv, hq, d, new = case["batch"], case["kv_heads"], case["q_heads"], case["head_dim"], case["new"]
    src, rsn = _cache_lengths(case)
    state["src"], state["rsn"] = src, rsn
    q = _projected(g, (b, new, hq, d), torch.float32)
    state["q"] = (q * torch.rsqrt((q * q).mean(-1, keepdim=True))).to(torch.bfloat16)
    rng = np.random.default_rng([int(seed), 4])
    if own:
        import paper_2510_17238_amd as st
        caches = []
    for which, lens, most in (("s", src, case["src_hi"]), ("r", rsn, case["rsn_hi"])):
        if own:
            per, table = _pages(rng, b, most)
            caches.append(st.KVCache(b * per, b, per, hkv, d, torch.from_numpy(table).to("cuda"), mxfp4=True))
        rows = max(1, most)
        k = _projected(g, (b, rows, hkv, d), torch.bfloat16)
        v = torch.randn((b, rows, hkv, d), generator=g, device="cuda").to(torch.bfloat16)
        if own:
            state[which + "_new"] = (k, v)
        else:
            for name, x in (("k", k), ("v", v)):
                code, exponent = _code_rows(x)
                state[which + name] = (code[..., 0::2] | (code[..., 1::2] << 4), (exponent + 127).to(torch.uint8))
                del code, exponent
        del k, v
    if own:
        state["caches"] = st.DualCache(*caches)
        for which, kind, lens in (("s", st.ST_SOURCE, src), ("r", st.ST_REASONING, rsn)):
            k, v = state.pop(which + "_new")
            st.st_kv_append(state["caches"], kind, k, v, n_new=torch.from_numpy(lens).to("cuda"))
        state["src_d"], state["rsn_d"] = torch.from_numpy(src).to("cuda"), torch.from_numpy(rsn).to("cuda")
        state["out"] = torch.empty_like(state["q"])
        state["lse"] = torch.empty((b, new, hq), dtype=torch.float32, device="cuda")
        state["ws"] = torch.empty(max(256, st.st_decode_workspace_bytes(b, hq, hkv, d, new, case["src_hi"], case["rsn_hi"])),
                                  dtype=torch.uint8, device="cuda")
    return state


# ------------------------------------------------------------------ one pass
def run(state):
    case = state["case"]
    if own:
        return {"norm_rope": _own_rows, "norm_rope_bwd": _own_rows_bwd, "append": _own_append, "decode": _own_decode}[case["op"]](case, state)
    return {"norm_rope": _plain_rows, "norm_rope_bwd": _plain_rows_bwd, "append": _plain_append, "decode": _plain_decode}[case["op"]](case, state)


def _own_rows(case, s):
    import paper_2510_17238_amd as st
    return st.st_norm_rope_apply_qk(s["q"], s["k"], s["q_weight"], s["k_weight"], s["pos"], s["spec"], eps=EPS, q_out=s["q_out"], k_out=s["k_out"])


def _own_rows_bwd(case, s):
    import paper_2510_17238_amd as st
    return st.st_norm_rope_bwd_qk(s["d_q"], s["d_k"], s["q"], s["k"], s["q_weight"], s["k_weight"], s["pos"], s["spec"], eps=EPS,
                                  dq=s["q_out"], dk=s["k_out"], workspace=s["ws"])


def _own_append(case, s):
    import paper_2510_17238_amd as st
    st.st_kv_append_norm_rope(s["caches"], st.ST_REASONING, s["k_new"], s["v_new"], s["k_weight"], s["spec"], eps=EPS, start_len=s["start"],
                              n_new=s["n"], host_len_upper_bound=s["bound"])
    st.st_kv_read(s["caches"], st.ST_REASONING, s["k_out"], s["v_out"], first=s["start"], n=s["n"])
    return s["k_out"], s["v_out"], s["caches"].reasoning.appended_len


def _own_decode(case, s):
    import paper_2510_17238_amd as st
    st.st_attn_decode_dual(s["q"], s["caches"], s["src_d"], s["rsn_d"], case["src_hi"], case["rsn_hi"], out=s["out"], lse=s["lse"], workspace=s["ws"])
    return s["out"], s["lse"]


# the plain forms ---------------------------------------------------------
def _frequencies(case):
    """Angle per position of every rotated pair, in 64 bits, and the factor on the rotated dims."""
    r, s, theta = case["rotary"], case["factor"], 1.0e6
    i = torch.arange(r // 2, dtype=torch.float64, device="cuda")
    if case["scaling"] == "ntk":
        theta = theta * s ** (r / (r - 2))
    f = theta ** (-2.0 * i / r)
    if case["scaling"] == "linear":
        f = f / s
    if case["scaling"] != "yarn":
        return f, 1.0

    def pair(turns):                            # the pair that turns so often over the trained length
        return r * math.log(case["original"] / (turns * 2.0 * math.pi)) / (2.0 * math.log(theta))

    lo, hi = max(math.floor(pair(32.0)), 0), min(math.ceil(pair(1.0)), r - 1)
    ramp = ((i - lo) / max(hi - lo, 1e-3)).clamp(0.0, 1.0)
    return f * (1.0 - ramp) + f / s * ramp, 0.1 * math.log(s) + 1.0 if s > 1.0 else 1.0


def _cos_sin(case, pos, dtype):
    f, a = _frequencies(case)
    angle = pos.double()[..., None] * f
    return (torch.cos(angle) * a).to(dtype), (torch.sin(angle) * a).to(dtype)


def _turn(case, x, cos, sin):
    """Pairs of the leading rotary dims of x[..., heads, D] turned by [..., 1, rotary / 2] angles."""
    r = case["rotary"]
    if case["layout"] == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        return torch.cat((a * cos - b * sin, b * cos + a * sin, x[..., r:]), -1)
    a, b = x[..., 0:r:2], x[..., 1:r:2]
    return torch.cat((torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2), x[..., r:]), -1)


def _plain_rows(case, s):
    cos, sin = _cos_sin(case, s["pos"], torch.float32)
    outs = []
    for x, w in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])):
        x = x.float()
        n = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
        outs.append(_turn(case, n, cos[:, None], sin[:, None]).to(w.dtype))
    return tuple(outs)


def _plain_rows_bwd(case, s):
    cos, sin = _cos_sin(case, s["pos"], torch.float32)
    grads, weights = [], []
    for g, x, w in ((s["d_q"], s["q"], s["q_weight"]), (s["d_k"], s["k"], s["k_weight"])):
        x, g, d = x.float(), _turn(case, g.float(), cos[:, None], -sin[:, None]), case["head_dim"]
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        h = g * w.float()
        grads.append((r * h - x * (r ** 3 / d) * (h * x).sum(-1, keepdim=True)).to(w.dtype))
        weights.append((g * x * r).double().sum((0, 1)).float())
    return (*grads, *weights)


_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0)


def _stored(case, x):
    """What a cache gives back for bf16 rows, as bf16."""
    if case["store"] == "bf16":
        return x
    if case["store"] == "mxfp4":
        code, k = _code_rows(x)
        values = torch.tensor(_E2M1, device=x.device)[code.int()]
        return (values.reshape(*k.shape, 32) * _two_to(k)[..., None]).reshape(x.shape).to(torch.bfloat16)
    f = x.float()
    top = f.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(torch.where(top > 0, top, torch.ones_like(top)))
    k = torch.where(top > 0, torch.clamp(e - 9 + (m > 0.875).to(torch.int32), min=-100), torch.zeros_like(e))      # 448 = 0.875 * 2^9
    return ((f * _two_to(-k)).to(torch.float8_e4m3fn).float() * _two_to(k)).to(torch.bfloat16)


def _round_once(x):
    """64 bits to bf16 in one rounding: 32 bits in between that fall on the middle of two bf16 values are moved to the side they came from."""
    f = x.float()
    bits = f.view(torch.int32)
    off = torch.sign((x - f.double()) * torch.sign(x)).to(torch.int32)
    return torch.where((bits & 0xffff) == 0x8000, bits + off, bits).view(torch.float32).to(torch.bfloat16)


def _plain_append(case, s):
    # keys in 64 bits: a value next to the line between two codes has to fall on its own side
    most = s["k_new"].shape[1]
    pos = s["start"][:, None] + torch.arange(most, device="cuda")
    cos, sin = _cos_sin(case, pos, torch.float64)
    x = s["k_new"].double()
    n = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * s["k_weight"].double()
    k = _round_once(_turn(case, n, cos[:, :, None], sin[:, :, None]))
    here = (torch.arange(most, device="cuda") < s["n"][:, None])[:, :, None, None]
    return torch.where(here, _stored(case, k), s["k_out"]), torch.where(here, _stored(case, s["v_new"]), s["v_out"]), s["start"] + s["n"]


def _decoded(pair, b, n):
    """The first n rows of stream b, [heads, n, D] in fp32."""
    code, scale = pair[0][b, :n], pair[1][b, :n]
    lut = torch.tensor(_E2M1, device="cuda")
    x = torch.stack((lut[(code & 15).int()], lut[(code >> 4).int()]), -1).reshape(*scale.shape, 32)
    return (x * _two_to(scale.int() - 127)[..., None]).reshape(*code.shape[:2], -1).transpose(0, 1)


def _plain_decode(case, s):
    new, hq, hkv, d = case["new"], case["q_heads"], case["kv_heads"], case["head_dim"]
    out = torch.empty_like(s["q"])
    lse = torch.empty((case["batch"], new, hq), dtype=torch.float32, device="cuda")
    for b in range(case["batch"]):
        ns, nr = int(s["src"][b]), int(s["rsn"][b])
        k = torch.cat((_decoded(s["sk"], b, ns), _decoded(s["rk"], b, nr)), 1)
        v = torch.cat((_decoded(s["sv"], b, ns), _decoded(s["rv"], b, nr)), 1)
        q = s["q"][b].float().reshape(new, hkv, hq // hkv, d).permute(1, 0, 2, 3).reshape(hkv, -1, d) / math.sqrt(d)
        score = torch.matmul(q, k.transpose(1, 2).contiguous()).reshape(hkv, new, hq // hkv, -1)
        if new > 1:
            col = torch.arange(ns + nr, device="cuda")
            hidden = col[None] > (ns + nr - new + torch.arange(new, device="cuda"))[:, None]
            score = score.masked_fill(hidden[None, :, None], float("-inf"))
        top = score.amax(-1, keepdim=True)
        p = torch.exp(score - top)
        total = p.sum(-1, keepdim=True)
        o = torch.matmul(p.reshape(hkv, -1, ns + nr), v.contiguous()).reshape(hkv, new, hq // hkv, d) / total
        out[b] = o.permute(1, 0, 2, 3).reshape(new, hq, d).to(torch.bfloat16)
        lse[b] = (top + torch.log(total))[..., 0].permute(1, 0, 2).reshape(new, hq)
    return out, lse


# ------------------------------------------------------------------ the definitions in 64 bits
def _phases(case, pos):
    """exp(i angle) of every pair, times the attention factor; the frequencies pair by pair."""
    r, s, base = case["rotary"], case["factor"], 1.0e6
    f, a = [], 1.0
    for i in range(r // 2):
        plain = math.exp(-2.0 * i / r * math.log(base))
        if case["scaling"] == "linear":
            plain = plain / s
        elif case["scaling"] == "ntk":
            plain = math.exp(-2.0 * i / r * (math.log(base) + r / (r - 2.0) * math.log(s)))
        elif case["scaling"] == "yarn":
            edge = [r / 2.0 * (math.log(case["original"]) - math.log(2.0 * math.pi * turns)) / math.log(base) for turns in (32.0, 1.0)]
            lo, hi = max(0, math.floor(edge[0])), min(r - 1, math.ceil(edge[1]))
            share = min(1.0, max(0.0, (i - lo) / (hi - lo if hi > lo else 1e-3)))
            plain = share * plain / s + (1.0 - share) * plain
            a = 1.0 + 0.1 * math.log(s)
        f.append(plain)
    angle = pos.double()[..., None] * torch.tensor(f, dtype=torch.float64, device="cuda")
    return torch.polar(torch.full_like(angle, a), angle)


def _definition(case, x, w, phase):
    """Rows [..., heads, D] in 64 bits, normalised, weighted and turned (phase: [..., rotary / 2])."""
    r = case["rotary"]
    n = x / torch.sqrt(x.square().sum(-1, keepdim=True) / case["head_dim"] + EPS) * w
    lead = n[..., :r]
    z = torch.complex(*lead.unflatten(-1, (2, r // 2)).unbind(-2)) if case["layout"] == "half" else torch.complex(*lead.unflatten(-1, (r // 2, 2)).unbind(-1))
    z = z * phase[..., None, :]
    turned = torch.cat((z.real, z.imag), -1) if case["layout"] == "half" else torch.view_as_real(z).flatten(-2)
    return torch.cat((turned, n[..., r:]), -1)


def _power(k):
    """2^k in 64 bits, from its exponent's bits."""
    return ((k.long() + 1023) << 52).view(torch.float64)


def _value_of(store, x):
    """What a cache in `store` holds for 64-bit rows that bf16 holds exactly: the nearest of the format's values."""
    if store == "bf16":
        return x
    block, largest, bits, lowest = (32, 6.0, 1, 0) if store == "mxfp4" else (x.shape[-1], 448.0, 3, -6)
    y = x.unflatten(-1, (-1, block))
    top = y.abs().amax(-1, keepdim=True)
    k = torch.where(top > 0, torch.ceil(torch.log2(torch.where(top > 0, top, torch.full_like(top, largest)) / largest)).clamp(min=-100.0), torch.zeros_like(top))
    k = torch.where(largest * _power(k - 1) >= top, (k - 1).clamp(min=-100.0), k)       # (where the logarithm fell on the wrong side)
    k = torch.where(top > largest * _power(k), k + 1, k)
    k = torch.where(top > 0, k, torch.zeros_like(k))
    z = y * _power(-k)
    step = _power(torch.floor(torch.log2(z.abs().clamp(min=2.0 ** lowest))) - bits)
    return (torch.round(z / step) * step * _power(k)).flatten(-2)                       # (torch.round: ties to even)


def _to_bf16(x):
    """64-bit values rounded once to 8 bits of significand, ties to even."""
    m, e = torch.frexp(x)
    return torch.round(m * 256.0) * _power(e - 8)


def exact(case, seed):
    was = globals()["own"]
    globals()["own"] = False
    try:
        s = prepare(case, seed)
    finally:
        globals()["own"] = was
    return {"norm_rope": _exact_rows, "norm_rope_bwd": _exact_rows_bwd, "append": _exact_append, "decode": _exact_decode}[case["op"]](case, s)


def _exact_rows(case, s):
    phase = _phases(case, s["pos"])
    return tuple(_definition(case, s[x].double(), s[w].double(), phase) for x, w in (("q", "q_weight"), ("k", "k_weight")))


def _exact_rows_bwd(case, s):
    phase = _phases(case, s["pos"])
    grads, weights = [], []
    for g, x, w in (("d_q", "q", "q_weight"), ("d_k", "k", "k_weight")):
        x64, w64 = s[x].double().requires_grad_(True), s[w].double().requires_grad_(True)
        with torch.enable_grad():
            dx, dw = torch.autograd.grad(_definition(case, x64, w64, phase), (x64, w64), s[g].double())
        grads.append(dx)
        weights.append(dw)
    return (*grads, *weights)


def _exact_append(case, s):
    phase = _phases(case, s["start"][:, None] + torch.arange(s["k_new"].shape[1], device="cuda"))
    k = _value_of(case["store"], _to_bf16(_definition(case, s["k_new"].double(), s["k_weight"].double(), phase)))
    v = _value_of(case["store"], s["v_new"].double())
    for b in range(case["batch"]):
        k[b, int(s["n"][b]):] = 0.0
        v[b, int(s["n"][b]):] = 0.0
    return k, v, s["start"] + s["n"]


def _exact_decode(case, s):
    new, hq, hkv, d = case["new"], case["q_heads"], case["kv_heads"], case["head_dim"]
    # the codes' values: sign, two bits of exponent, one bit of significand
    values = torch.tensor([(-1.0) ** (c >> 3) * ((c & 1) * 0.5 if (c >> 1) & 3 == 0 else (1.0 + (c & 1) * 0.5) * 2.0 ** (((c >> 1) & 3) - 1)) for c in range(16)],
                          dtype=torch.float64, device="cuda")
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty((case["batch"], new, hq), dtype=torch.float64, device="cuda")

    def rows(pair, b, n):
        code, scale = pair[0][b, :n].long(), pair[1][b, :n].double()
        x = torch.empty((*code.shape[:2], d), dtype=torch.float64, device="cuda")
        x[..., 0::2] = values[code % 16]
        x[..., 1::2] = values[code // 16]
        return x * _power(scale - 127).repeat_interleave(32, -1)

    for b in range(case["batch"]):
        ns, nr = int(s["src"][b]), int(s["rsn"][b])
        k, v = (torch.cat((rows(s["s" + x], b, ns), rows(s["r" + x], b, nr))) for x in "kv")
        for h in range(hkv):
            heads = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
            score = s["q"][b, :, heads].double() @ k[:, h].T.contiguous() * d ** -0.5         # [new, group, tokens]
            for t in range(new - 1):
                score[t, :, ns + nr - new + t + 1:] = -math.inf
            lse[b, :, heads] = torch.logsumexp(score, -1)
            out[b, :, heads] = torch.softmax(score, -1) @ v[:, h].contiguous()
    return out, lse
