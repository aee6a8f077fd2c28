"""The low-bit operators and what they are measured on: the layer's two big streams, cache and weights, held in 8 and 4 bits.

append    `kvra_append_kv_q8`: rotary embedding of a chunk's K and Q, K and V into a cache of e4m3 values with one power-of-two
          scale (e8m0) for each block of 64 tokens and head.
attn      `kvra_chunk_attn_q8`: causal attention of a chunk's queries over that cache.
linear    `kvra_linear_w4`: a linear layer whose weights are e2m1 values with one power-of-two scale for each 32 along a row;
          plain, with residual, or as the gate and up projections of a SwiGLU MLP.
pack      `kvra_pack_w4` and `kvra_unpack_w4`: bf16 weights into that format and back.

Activations and unquantised weights are bf16.  What a cache holds is returned as e4m3 values and their scales.
"""
import math

import torch

own = False

BLOCK = 64                   # tokens of a cache block
GROUP = 32                   # weights of a row that share a scale
E_MIN, E_MAX = -100, 120     # exponents a scale may have
ROPE_BASE = 10000.0
WORKSPACE = 128 << 20        # what a program that attends keeps: enough for every shape

LAYOUTS = [(32, 32, 128), (32, 8, 128), (32, 1, 128), (71, 1, 64), (2, 2, 64), (8, 2, 128), (16, 16, 64), (5, 5, 128)]


def _append(name, H, Hkv, d, prefix, c):
    case = {"op": "append", "H": H, "Hkv": Hkv, "d": d, "prefix": prefix, "c": c}
    return dict(case, name=name) if name else case


def _attn(name, H, Hkv, d, prefix, c):
    case = {"op": "attn", "H": H, "Hkv": Hkv, "d": d, "prefix": prefix, "c": c}
    return dict(case, name=name) if name else case


def _linear(name, form, m, n, k):
    case = {"op": "linear", "form": form, "m": m, "n": n, "k": k}
    return dict(case, name=name) if name else case


def _pack(name, n, k):
    case = {"op": "pack", "n": n, "k": k}
    return dict(case, name=name) if name else case


def listed():
    return [
        # one new token into a block that holds tokens already, Llama-7B heads: latency
        _append("append_one_15001", 32, 32, 128, 15001, 1),
        # the first chunk of the balanced 16k prompt
        _append("append_prompt_5824", 32, 32, 128, 0, 5824),
        # the smallest prompt's second chunk: launch and latency
        _attn("attn_tiny_96", 2, 2, 64, 160, 96),
        # a token behind a 16k prompt: the step of the extension phase, the whole cache of a layer is read
        _attn("attn_one_16k", 32, 32, 128, 16383, 1),
        # a follow-up turn: few tokens behind a prompt, grouped queries, odd lengths
        _attn("attn_turn_gqa8_5901", 32, 8, 128, 5824, 77),
        # the last chunk of the Falcon-7B prompt: multi-query, head_dim 64
        _attn("attn_falcon7b_8k", 71, 1, 64, 7104, 1088),
        # the last chunk of the balanced 16k prompt: a matrix-bound launch
        _attn("attn_chunk_16k", 32, 32, 128, 15296, 1088),
        # a token through Llama-7B's q/k/v projection: the weights are read once
        _linear("linear_one_qkv", "plain", 1, 12288, 4096),
        # a handful of tokens through its gate and up projections
        _linear("linear_few_swiglu", "swiglu", 13, 11008, 4096),
        # a prompt's chunk through the down projection, with the residual
        _linear("linear_chunk_down", "residual", 777, 4096, 11008),
        # weights of a small layer, rows that end inside a kilobyte
        _pack("pack_small", 704, 1088),
        # the down projection of Llama-7B
        _pack("pack_down", 4096, 11008),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attn", "attn", "linear", "linear", "pack"])
    if op == "append":
        H, Hkv, d = rng.choice(LAYOUTS)
        return _append(None, H, Hkv, d, rng.choice([0, _log(rng, 1, 16000)]), _log(rng, 1, 5824))
    if op == "attn":
        H, Hkv, d = rng.choice(LAYOUTS)
        c = _log(rng, 1, 4096)
        most = 32 * 128 * 1088 * 16384 // (H * d * c) - c     # at most the largest listed case's work
        while most < 0:
            c = _log(rng, 1, 4096)
            most = 32 * 128 * 1088 * 16384 // (H * d * c) - c
        return _attn(None, H, Hkv, d, rng.choice([0, _log(rng, 1, max(1, min(most, 32000)))]) if most > 0 else 0, c)
    if op == "linear":
        n, k = 32 * _log(rng, 8, 384), 64 * _log(rng, 4, 172)
        return _linear(None, rng.choice(["plain", "residual", "swiglu"]), _log(rng, 1, min(2048, 777 * 4096 * 11008 // (2 * n * k))), n, k)
    return _pack(None, 32 * _log(rng, 8, 384), 64 * _log(rng, 4, 172))


# ---- inputs ----------------------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, *shape, std=1.0):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).mul_(std).to(torch.bfloat16)


def _exponent(amax, high):
    """The smallest e with amax <= high * 2^e (high = 448 = 0.875 * 2^9 or 6 = 0.75 * 2^3), clamped."""
    mant, ex = torch.frexp(amax)
    hm, he = math.frexp(high)
    e = ex - he + (mant > hm).to(ex.dtype)
    return torch.where(amax > 0, e, torch.full_like(e, E_MIN)).clamp(E_MIN, E_MAX)


def _quantised_cache(g, rows, capacity, Hkv, d):
    """A cache whose first `rows` rows hold N(0, 1) values that came in at once: codes (uint8) and scales (uint8)."""
    blocks = (capacity + BLOCK - 1) // BLOCK
    x = torch.zeros(blocks * BLOCK, Hkv, d, device="cuda")
    x[:rows] = torch.randn(rows, Hkv, d, generator=g, device="cuda").to(torch.bfloat16).float()
    b = x.view(blocks, BLOCK, Hkv, d)
    e = _exponent(b.abs().amax(dim=(1, 3)), 448.0)
    codes = torch.ldexp(b, -e[:, None, :, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    return codes.view(blocks * BLOCK, Hkv, d)[:capacity].contiguous(), (e + 127).to(torch.uint8)


def _quantised_weights(g, n, k):
    """N(0, 0.02^2) weights as packed e2m1 codes [n, k/2] and scales [n, k/32]."""
    w = torch.randn(n, k, generator=g, device="cuda").mul_(0.02).to(torch.bfloat16).float()
    code, e = _codes4(w)
    code = code.view(n, k // 2, 2)
    return (code[..., 0] | code[..., 1] << 4).to(torch.uint8), (e + 127).to(torch.uint8)


def _codes4(w):
    """e2m1 codes (sign, two exponent bits, one mantissa bit) of w [n, k] in 32 bits, and the groups' exponents; ties to even."""
    n, k = w.shape
    grouped = w.view(n, k // GROUP, GROUP)
    e = _exponent(grouped.abs().amax(dim=2), 6.0)
    a = torch.ldexp(grouped, -e[..., None]).view(n, k)
    m = a.abs()
    # borders between 0, .5, 1, 1.5, 2, 3, 4, 6: a value on one goes to the even code
    code = ((m > 0.25).int() + (m >= 0.75).int() + (m > 1.25).int() + (m >= 1.75).int() + (m > 2.5).int() + (m >= 3.5).int()
            + (m > 5.0).int())
    return code | (torch.signbit(a).int() << 3), e


def prepare(case, seed):
    g = _gen(seed)
    op = case["op"]
    s = dict(case)
    if op in ("append", "attn"):
        H, Hkv, d, p, c = (case[x] for x in ("H", "Hkv", "d", "prefix", "c"))
        cap = p + c
        s["kc"], s["ks"] = _quantised_cache(g, p if op == "append" else cap, cap, Hkv, d)
        s["vc"], s["vs"] = _quantised_cache(g, p if op == "append" else cap, cap, Hkv, d)
        s["q"] = _normal(g, c, H, d)
        s["out"] = torch.empty_like(s["q"])
        if op == "append":
            s["k"], s["v"] = _normal(g, c, Hkv, d), _normal(g, c, Hkv, d)
        else:
            s["workspace"] = torch.zeros(WORKSPACE, dtype=torch.uint8, device="cuda")
    elif op == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        s["x"] = _normal(g, m, k)
        s["w"], s["ws"] = _quantised_weights(g, n, k)
        s["w2"], s["ws2"] = _quantised_weights(g, n, k) if case["form"] == "swiglu" else (None, None)
        s["residual"] = _normal(g, m, n) if case["form"] == "residual" else None
        s["out"] = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    else:
        n, k = case["n"], case["k"]
        s["w"] = _normal(g, n, k, std=0.02)
        s["codes"] = torch.empty(n, k // 2, dtype=torch.uint8, device="cuda")
        s["scales"] = torch.empty(n, k // GROUP, dtype=torch.uint8, device="cuda")
        s["out"] = torch.empty(n, k, dtype=torch.bfloat16, device="cuda")
    return s


# ---- the plain forms -------------------------------------------------------------------------------------------------
def _rotate(x, p, to):
    """Half-split rotary embedding of rows [c, heads, d] at positions p, p + 1, ..., in 64 bits."""
    c, _, d = x.shape
    i = torch.arange(d // 2, dtype=torch.float64, device=x.device)
    pos = torch.arange(p, p + c, dtype=torch.float64, device=x.device)
    phi = (pos[:, None] * torch.pow(torch.tensor(ROPE_BASE, dtype=torch.float64, device=x.device), -2.0 * i / d))[:, None, :]
    cos, sin = phi.cos(), phi.sin()
    lo, hi = x[..., :d // 2].double(), x[..., d // 2:].double()
    return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], dim=-1).to(to)


def _append_plain(cache, scale, new, p):
    """Rows p .. of a cache and of its scales take the rows `new` [c, Hkv, d] (64 bits)."""
    c, Hkv, d = new.shape
    b0, b1 = p // BLOCK, (p + c + BLOCK - 1) // BLOCK
    held = p - b0 * BLOCK                                # rows the first block holds already
    old_e = scale[b0].int() - 127
    old = torch.ldexp(cache[b0 * BLOCK:p].view(torch.float8_e4m3fn).double(), old_e[None, :, None])
    pad = (b1 - b0) * BLOCK - held - c
    x = torch.nn.functional.pad(torch.cat([old, new]), (0, 0, 0, 0, 0, pad)).view(b1 - b0, BLOCK, Hkv, d)
    y = x.abs()
    if held:
        y = y.clone()
        y[0, :held] = 0
    e = _exponent(y.amax(dim=(1, 3)), 448.0)
    if held:
        e[0] = torch.maximum(e[0], old_e)
    codes = torch.ldexp(x, -e[:, None, :, None]).float().to(torch.float8_e4m3fn).view(torch.uint8)
    cache[b0 * BLOCK:p + c] = codes.view(-1, Hkv, d)[:held + c]
    scale[b0:b1] = (e + 127).to(torch.uint8)


def _values8(codes, scale, rows, to):
    e = (scale.int() - 127).repeat_interleave(BLOCK, dim=0)[:rows]
    return torch.ldexp(codes[:rows].view(torch.float8_e4m3fn).to(to), e[..., None])


def _values4(codes, scale, to):
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=to, device=codes.device)
    table = torch.cat([table, -table])
    c = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(1)
    v = table[c.long()]
    return torch.ldexp(v.view(v.shape[0], -1, GROUP), (scale.int() - 127)[..., None]).view(v.shape)


def _attend(q, K, V, p, scale):
    """q [c, H, d], K and V [p + c, Hkv, d], all of one type: softmax(scale q K^T) V, key j visible to row r iff j <= p + r."""
    c, H, d = q.shape
    n, Hkv, _ = K.shape
    G = H // Hkv
    qg = q.view(c, Hkv, G, d).permute(1, 0, 2, 3).reshape(Hkv, c * G, d)
    s = torch.matmul(qg, K.permute(1, 2, 0).contiguous()).mul_(scale)
    hidden = torch.arange(n, device=q.device)[None, :] > torch.arange(p, p + c, device=q.device).repeat_interleave(G)[:, None]
    s.masked_fill_(hidden[None], -math.inf)
    s.sub_(s.amax(dim=-1, keepdim=True)).exp_()
    o = torch.matmul(s, V.permute(1, 0, 2).contiguous()) / s.sum(dim=-1, keepdim=True)
    return o.view(Hkv, c, G, d).permute(1, 0, 2, 3).reshape(c, H, d)


def _cache_out(s):
    e4m3, e8m0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
    return {"q": s["out"], "k": s["kc"].view(e4m3), "v": s["vc"].view(e4m3), "k_scale": s["ks"].view(e8m0), "v_scale": s["vs"].view(e8m0)}


def run(s):
    op = s["op"]
    if own:
        from paper_2405_05329_amd import kvra
        stream = torch.cuda.current_stream()
        if op == "append":
            kvra.kvra_append_kv_q8(s["k"], s["v"], s["q"], s["out"], s["kc"], s["vc"], s["ks"], s["vs"], s["prefix"], s["c"],
                                   s["prefix"] + s["c"], s["H"], s["Hkv"], s["d"], ROPE_BASE, stream)
            return _cache_out(s)
        if op == "attn":
            kvra.kvra_chunk_attn_q8(s["q"], s["kc"], s["vc"], s["ks"], s["vs"], s["prefix"], s["c"], s["H"], s["Hkv"], s["d"],
                                    1.0 / math.sqrt(s["d"]), s["out"], s["workspace"], WORKSPACE, stream)
        elif op == "linear":
            kvra.kvra_linear_w4(s["x"], s["w"], s["ws"], s["w2"], s["ws2"], s["residual"], s["out"], s["m"], s["n"], s["k"], stream)
        else:
            kvra.kvra_pack_w4(s["w"], s["codes"], s["scales"], s["n"], s["k"], stream)
            kvra.kvra_unpack_w4(s["codes"], s["scales"], s["out"], s["n"], s["k"], stream)
        return s["out"]
    if op == "append":
        s["out"] = _rotate(s["q"], s["prefix"], torch.bfloat16)
        _append_plain(s["kc"], s["ks"], _rotate(s["k"], s["prefix"], torch.float64), s["prefix"])
        _append_plain(s["vc"], s["vs"], s["v"].double(), s["prefix"])
        return _cache_out(s)
    if op == "attn":
        n = s["prefix"] + s["c"]
        K, V = _values8(s["kc"], s["ks"], n, torch.float32), _values8(s["vc"], s["vs"], n, torch.float32)
        return _attend(s["q"].float(), K, V, s["prefix"], 1.0 / math.sqrt(s["d"])).to(torch.bfloat16)
    if op == "linear":
        x = s["x"].float()
        y = torch.matmul(x, _values4(s["w"], s["ws"], torch.float32).T)
        if s["w2"] is not None:
            y = y / (1.0 + torch.exp(-y)) * torch.matmul(x, _values4(s["w2"], s["ws2"], torch.float32).T)
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return y.to(torch.bfloat16)
    code, e = _codes4(s["w"].float())
    code = code.view(s["n"], s["k"] // 2, 2)
    return _values4((code[..., 0] | code[..., 1] << 4).to(torch.uint8), (e + 127).to(torch.uint8), torch.float32).to(torch.bfloat16)


def work(case):
    op = case["op"]
    if op in ("append", "attn"):
        H, Hkv, d, p, c = (case[x] for x in ("H", "Hkv", "d", "prefix", "c"))
        if op == "append":
            blocks = (p + c + BLOCK - 1) // BLOCK - p // BLOCK
            return {"bytes": c * d * (2 * 2 * Hkv + 2 * Hkv + 4 * H) + 2 * blocks * Hkv, "flops": 3 * c * d * (H + Hkv)}
        n = p + c
        return {"bytes": 2 * n * Hkv * d + 2 * ((n + BLOCK - 1) // BLOCK) * Hkv + 4 * c * H * d, "flops": 4 * d * H * (c * p + c * (c + 1) // 2)}
    n, k = case["n"], case["k"]
    packed = n * k // 2 + n * k // GROUP
    if op == "linear":
        m, mats = case["m"], 2 if case["form"] == "swiglu" else 1
        return {"bytes": mats * packed + 2 * m * k + 2 * m * n * (2 if case["form"] == "residual" else 1), "flops": 2 * mats * m * n * k}
    return {"bytes": 2 * (2 * n * k + packed), "flops": n * k}


# ---- the definition in 64 bits, by other routes ----------------------------------------------------------------------
_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _nearest(x, values):
    """The index of the nearest of rising `values` for each of x >= 0; ties to the even index."""
    v = torch.tensor(values, dtype=torch.float64, device=x.device)
    hi = torch.searchsorted(v, x.contiguous()).clamp(1, len(values) - 1)
    below, above = x - v[hi - 1], v[hi] - x
    return torch.where((below < above) | ((below == above) & (hi % 2 == 1)), hi - 1, hi)


def _scale64(amax, high):
    e = torch.ceil(torch.log2(amax.clamp_min(1e-300) / high))
    e = torch.where(amax > high * torch.pow(2.0, e), e + 1, torch.where(amax <= high * torch.pow(2.0, e - 1), e - 1, e))
    return e.clamp(E_MIN, E_MAX)


def _e4m3_table():
    return [(m / 8.0) * 2.0 ** -6 if e == 0 else (1 + m / 8.0) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127]


def _append64(cache, scale, new, p):
    table = torch.tensor(_e4m3_table(), dtype=torch.float64, device=new.device)
    first, c = p - p % BLOCK, new.shape[0]
    held = p - first
    code = cache[first:p].long()
    value = table[(code & 127).clamp_max(126)] * torch.where(code > 127, -1.0, 1.0).double()
    if held:
        value = value * torch.pow(2.0, scale[first // BLOCK].double() - 127)[None, :, None]
    out, out_scale = cache.view(torch.float8_e4m3fn).double(), torch.pow(2.0, scale.double() - 127)
    block = torch.arange(first, p + c, device=new.device) // BLOCK - first // BLOCK
    peak = torch.zeros(int(block[-1]) + 1, new.shape[1], dtype=torch.float64, device=new.device)
    peak.index_reduce_(0, block[held:], new.abs().amax(dim=2), "amax")
    e = _scale64(peak, 448.0)
    if held:
        e[0] = torch.maximum(e[0], scale[first // BLOCK].double() - 127)
    x = torch.cat([value, new]) / torch.pow(2.0, e)[block][..., None]
    out[first:p + c] = table[_nearest(x.abs(), _e4m3_table())] * torch.sign(x)
    out_scale[first // BLOCK:first // BLOCK + e.shape[0]] = torch.pow(2.0, e)
    return out, out_scale


def _turn64(x, p):
    c, heads, d = x.shape
    z = torch.complex(x[..., :d // 2].double(), x[..., d // 2:].double())
    freq = torch.exp(torch.arange(d // 2, device=x.device, dtype=torch.float64) * (-2.0 * math.log(ROPE_BASE) / d))
    phi = torch.outer(torch.arange(p, p + c, device=x.device, dtype=torch.float64), freq)
    z = z * torch.polar(torch.ones_like(phi), phi)[:, None, :]
    return torch.cat([z.real, z.imag], dim=2)


def _weights64(codes, scale):
    v = torch.empty(codes.shape[0], codes.shape[1] * 2, dtype=torch.float64, device=codes.device)
    table = torch.tensor(_E2M1 + [-x for x in _E2M1], dtype=torch.float64, device=codes.device)
    v[:, 0::2], v[:, 1::2] = table[(codes % 16).long()], table[(codes // 16).long()]
    return v * torch.pow(2.0, scale.double() - 127).repeat_interleave(GROUP, dim=1)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "append":
        p = s["prefix"]
        k, ks = _append64(s["kc"], s["ks"], _turn64(s["k"], p), p)
        v, vs = _append64(s["vc"], s["vs"], s["v"].double(), p)
        return {"q": _turn64(s["q"], p), "k": k, "v": v, "k_scale": ks, "v_scale": vs}
    if op == "attn":
        H, Hkv, p, c = s["H"], s["Hkv"], s["prefix"], s["c"]
        table = torch.tensor(_e4m3_table(), dtype=torch.float64, device="cuda")

        def values(codes, scale):
            x = codes.long()
            v = table[(x & 127).clamp_max(126)] * torch.where(x > 127, -1.0, 1.0).double()
            rows = torch.arange(codes.shape[0], device="cuda") // BLOCK
            return (v * torch.pow(2.0, scale.double() - 127)[rows][..., None]).transpose(0, 1)

        K, V = values(s["kc"], s["ks"]), values(s["vc"], s["vs"])
        q = s["q"].double().view(c, Hkv, H // Hkv, -1).permute(1, 2, 0, 3)      # [Hkv, G, c, d]
        o = torch.empty(q.shape, dtype=torch.float64, device="cuda")
        row = torch.arange(c, device="cuda")[:, None] + p
        key = torch.arange(p + c, device="cuda")[None, :]
        for g in range(Hkv):
            for h in range(H // Hkv):
                w = torch.softmax(torch.where(key <= row, q[g, h] @ K[g].T / math.sqrt(s["d"]), -math.inf), dim=1)
                o[g, h] = w @ V[g]
        return o.permute(2, 0, 1, 3).reshape(c, H, -1)
    if op == "linear":
        x = s["x"].double()
        y = x @ _weights64(s["w"], s["ws"]).T
        if s["w2"] is not None:
            y = torch.nn.functional.silu(y) * (x @ _weights64(s["w2"], s["ws2"]).T)
        return y if s["residual"] is None else y + s["residual"].double()
    w = s["w"].double().view(s["n"], -1, GROUP)
    unit = torch.pow(2.0, _scale64(w.abs().amax(dim=2), 6.0))[..., None]
    v = torch.tensor(_E2M1, dtype=torch.float64, device="cuda")[_nearest((w / unit).abs(), _E2M1)]
    return (v * torch.sign(w) * unit).view(s["n"], s["k"])
