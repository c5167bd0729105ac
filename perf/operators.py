"""What is timed of the microscaled operators: one call each, as a decoder layer with 4-bit weights, 8-bit activations and an
8-bit cache makes it.

A case is one call (`kind`):

  norm       h = resid + x, RMSNorm of h with a gain, the result in E4M3 with a power-of-two scale per 32 values
  swiglu     SiLU(gate) * up of a gate/up product's rows, in the same form
  weights    a weight matrix into E2M1 with a scale per 32 values, in the order that the product streams
  product    C = A W^T: rows of activations in 8 (E4M3) or 4 bits (E2M1) on such weights
  append     the keys and values of a window into the 8-bit cache: one scale per 32 positions, head and K or V
  attention  the window's queries over that cache: causal, grouped heads, a length per sequence, sliding window and sinks

Formats.  Along a row, every 32 values share the scale 2^(byte - 127): the smallest power of two with which the largest finite
magnitude does not exceed the format's (448 or 6).  Rows are padded with zeros to a multiple of 128 values.  The weights' and the
cache's byte orders are those of include/sjd.h; `_pack_*` and `_unpack_*` are that description in torch.

Sizes are those of the repository's own decoders (widths 1536 and 4096, FFN 4096 and 11008, heads of 64 and 128, caches up to
4224 positions) or generic ones around them.
"""
from __future__ import annotations

import math

import torch

own = False

HEADS = {64: 24, 128: 32}                  # the two decoders' heads by their size


def listed():
    return [
        # one token between two layers of the 4096-wide decoder: nothing but latency
        dict(name="norm_token", kind="norm", rows=1, d=4096, dtype="fp32"),
        # a long prompt's rows through the same norm
        dict(name="norm_prompt", kind="norm", rows=2048, d=4096, dtype="bf16"),
        # the FFN hidden of 128 rows (eight images of 16 drafts), from the gate/up product's rows
        dict(name="swiglu_batch", kind="swiglu", rows=128, F=11008, dtype="fp32"),
        # laying out the gate/up weights of one layer when a model is loaded
        dict(name="weights_gate_up", kind="weights", N=22016, K=4096, dtype="bf16"),
        # the auto-regressive step: one row on the gate/up weights
        dict(name="product_token", kind="product", M=1, N=22016, K=4096, bits=8, dtype="fp32"),
        # the narrow decoder's gate/up on an odd number of rows, activations in 4 bits
        dict(name="product_4bit", kind="product", M=101, N=8192, K=1536, bits=4, dtype="bf16"),
        # a long prompt on the gate/up weights: the matrix cores are what is left
        dict(name="product_prompt", kind="product", M=2048, N=22016, K=4096, bits=8, dtype="bf16"),
        # the window of one decoding step of eight images into their caches
        dict(name="append_window", kind="append", B=8, L=16, kv=32, hd=128, n=583, dtype="fp32"),
        # a prompt of 1000 tokens for two sequences at once
        dict(name="append_prompt", kind="append", B=2, L=1000, kv=32, hd=128, n=0, dtype="bf16"),
        # one token late in a 64 x 64 image, every query head its own keys
        dict(name="attention_token", kind="attention", B=1, L=1, H=32, kv=32, hd=128, n=4095, window=0, sinks=0, dtype="fp32"),
        # windows of 16 drafts of eight images of different lengths
        dict(name="attention_batch", kind="attention", B=8, L=16, H=32, kv=32, hd=128, n=1239, window=0, sinks=0, dtype="fp32"),
        # grouped heads over a very long cache, of which a sliding window and the prompt's tokens stay visible
        dict(name="attention_sinks", kind="attention", B=2, L=32, H=32, kv=8, hd=128, n=65501, window=16384, sinks=64, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def _drawn(rng):
    kind = rng.choice(["norm", "swiglu", "weights", "product", "product", "product", "append", "attention", "attention", "attention"])
    dtype = rng.choice(["fp32", "bf16"])
    if kind == "norm":
        return dict(kind=kind, rows=_log_int(rng, 1, 2048), d=rng.choice([1536, 4096, _log_int(rng, 64, 8192)]), dtype=dtype)
    if kind == "swiglu":
        return dict(kind=kind, rows=_log_int(rng, 1, 2048), F=rng.choice([4096, 11008, _log_int(rng, 64, 11008)]), dtype=dtype)
    if kind == "weights":
        return dict(kind=kind, N=_log_int(rng, 16, 22016), K=rng.choice([1536, 4096, 11008, _log_int(rng, 64, 8192)]), dtype=dtype)
    if kind == "product":
        N, K = rng.choice([(4608, 1536), (1536, 1536), (8192, 1536), (1536, 4096), (12288, 4096), (4096, 4096), (22016, 4096), (4096, 11008),
                           (_log_int(rng, 64, 22016), _log_int(rng, 64, 8192))])
        return dict(kind=kind, M=_log_int(rng, 1, 2048), N=N, K=K, bits=rng.choice([8, 8, 4]), dtype=dtype)
    hd = rng.choice([64, 128])
    B = rng.choice([1, 1, 2, 3, 4, 8, 11])
    if kind == "append":
        return dict(kind=kind, B=B, L=_log_int(rng, 1, 1024), kv=rng.choice([1, 2, 8, HEADS[hd]]), hd=hd, n=rng.choice([0, rng.randint(1, 4096)]), dtype=dtype)
    kv = rng.choice([1, 4, 8, HEADS[hd]])
    H = HEADS[hd] if kv == HEADS[hd] else kv * rng.choice([1, 3, 4, 7, 8])
    n = _log_int(rng, 1, 65536 // B)
    near = rng.random() < 0.4
    return dict(kind=kind, B=B, L=_log_int(rng, 1, 128), H=H, kv=kv, hd=hd, n=n, window=_log_int(rng, 1, max(2, n)) if near else 0,
                sinks=rng.choice([0, 4, 64, 121]) if near else 0, dtype=dtype)


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        c = _drawn(rng)
        held = c.get("B", 1) * c.get("kv", 0) * (c.get("n", 0) + c.get("L", 0)) * c.get("hd", 0)
        scores = c.get("B", 1) * c.get("H", 0) * c.get("L", 0) * (c.get("n", 0) + c.get("L", 0))
        if _cost(c) <= most and held <= 1 << 28 and scores <= 1 << 28:      # (the plain form holds all of them in 32 bits)
            return c


# ---- the formats --------------------------------------------------------------------------------------------------
def _up(n, m):
    return -(-n // m) * m


def _scale_bytes(amax, bits):
    """byte of the smallest 2^(byte - 127) with amax <= 448 (E4M3) or 6 (E2M1) times it; amax finite, fp32"""
    b = amax.view(torch.int32)
    top, half = (8, 0x600000) if bits == 8 else (2, 0x400000)      # 448 = 1.75 * 2^8, 6 = 1.5 * 2^2
    return ((b >> 23) - top + ((b & 0x7FFFFF) > half).to(torch.int32)).clamp_(0, 254)


def _pow2(byte, sign=1):
    """2^(sign * (byte - 127)) in fp32; sign -1: for bytes up to 253"""
    e = byte.to(torch.int32) if sign > 0 else 254 - byte.to(torch.int32)
    return torch.where(e > 0, e << 23, torch.full_like(e, 1 << 22)).view(torch.float32)


def _e2m1(y):
    """codes 0 .. 15 of |y| <= 6, ties to the even code"""
    a = y.abs()
    c = (a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5)
    return c + torch.signbit(y).to(torch.uint8) * 8


def _quantise(x, bits):
    """rows of fp32 -> codes [rows, Kp] (one byte per value: E4M3, or E2M1 in its low half), scale bytes [rows, Kp / 32]"""
    rows, K = x.shape
    Kp = _up(K, 128)
    x = torch.nn.functional.pad(x, (0, Kp - K)).view(rows, Kp // 32, 32)
    scale = _scale_bytes(x.abs().amax(-1), bits)
    y = x * _pow2(scale, -1)[..., None]
    codes = y.to(torch.float8_e4m3fn).view(torch.uint8) if bits == 8 else _e2m1(y)
    return codes.view(rows, Kp), scale.to(torch.uint8)


def _pair(codes):
    """two 4-bit codes to a byte, the first in the low half"""
    return codes[..., 0::2] | codes[..., 1::2] << 4


def _unpair(b):
    return torch.stack((b & 15, b >> 4), -1).flatten(-2)


def _value(codes, bits):
    if bits == 8:
        return codes.view(torch.float8_e4m3fn).to(torch.float32)
    m = (codes & 7).to(torch.float32)
    v = torch.where(m < 4, m * 0.5, torch.where(m < 6, m - 2, 2 * m - 8))
    return torch.where(codes > 7, -v, v)


def _dequantise(codes, scales, bits):
    return (_value(codes, bits).view(*scales.shape, 32) * _pow2(scales)[..., None]).view(codes.shape)


REC = 4352      # bytes of a record of packed weights: 16 features x 512 values of E2M1 and their scales


def _pack_weights(codes, scales):
    """codes [N, Kp] one a byte, scales [N, Kp / 32] -> packed [ceil(N / 16), ceil(K / 512), REC]"""
    N, Kp = codes.shape
    nt, kg = -(-N // 16), -(-Kp // 512)
    c = torch.nn.functional.pad(codes, (0, kg * 512 - Kp, 0, nt * 16 - N))
    s = torch.nn.functional.pad(scales, (0, kg * 16 - Kp // 32, 0, nt * 16 - N))
    c = _pair(c).view(nt, 16, kg, 4, 4, 16).permute(0, 2, 3, 4, 1, 5).reshape(nt, kg, 4096)       # step, quarter, feature, byte
    s = s.view(nt, 16, kg, 4, 4).permute(0, 2, 4, 1, 3).reshape(nt, kg, 256)                      # quarter, feature, step
    return torch.cat((c, s), -1).contiguous()


def _unpack_weights(w, N, K):
    nt, kg, _ = w.shape
    c = _unpair(w[..., :4096].reshape(nt, kg, 4, 4, 16, 16).permute(0, 4, 1, 2, 3, 5).reshape(nt * 16, kg * 256))
    s = w[..., 4096:].reshape(nt, kg, 4, 16, 4).permute(0, 3, 1, 4, 2).reshape(nt * 16, kg * 16)
    return c[:N, :_up(K, 128)], s[:N, :_up(K, 128) // 32]


def _pack_cache(k, v):
    """codes [..., 32, hd] of a block's keys and values -> its record [..., 64 * hd]"""
    lead, hd = k.shape[:-2], k.shape[-1]
    k = k.reshape(-1, 2, 16, hd // 32, 4, 8).permute(0, 1, 3, 4, 2, 5).reshape(-1, hd // 32, 2, 64, 8)
    v = v.reshape(-1, 2, 4, 4, hd // 16, 16).permute(0, 4, 2, 5, 1, 3).reshape(-1, hd // 32, 2, 64, 8)
    return torch.stack((k, v), 1).permute(0, 1, 2, 4, 3, 5).reshape(*lead, 64 * hd)


def _unpack_cache(rec, hd):
    lead = rec.shape[:-1]
    x = rec.reshape(-1, 2, hd // 32, 64, 2, 8).permute(1, 0, 2, 4, 3, 5)
    k = x[0].reshape(-1, 2, hd // 32, 4, 16, 8).permute(0, 1, 4, 2, 3, 5).reshape(*lead, 32, hd)
    v = x[1].reshape(-1, hd // 16, 4, 16, 2, 4).permute(0, 4, 2, 5, 1, 3).reshape(*lead, 32, hd)
    return k, v


def _block_scale(x):
    """scale bytes of blocks [..., 32, hd] of fp32"""
    return _scale_bytes(x.abs().amax((-1, -2)), 8)


# ---- inputs -------------------------------------------------------------------------------------------------------
def _type(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 17)


def _normal(g, *shape):
    return torch.randn(*shape, device="cuda", generator=g)


def _activations(g, rows, K):
    """rows with a few channels that are far larger than the others, as a decoder's residual stream has them"""
    x = _normal(g, rows, K)
    x[:, torch.randint(0, K, (max(1, K // 512),), device="cuda", generator=g)] *= 20
    return x


def _lengths(case, g):
    """cached positions per sequence: n for the first, shorter ones behind it"""
    n = torch.full((case["B"],), case["n"], dtype=torch.int32, device="cuda")
    if case["B"] > 1 and case["n"]:
        n[1:] -= (torch.rand(case["B"] - 1, device="cuda", generator=g) * 0.5 * case["n"]).to(torch.int32)
    return n


def prepare(case, seed):
    g, t, kind = _gen(seed), _type(case), case["kind"]
    s = dict(case=dict(case))
    if kind == "norm":
        s["x"], s["resid"] = _normal(g, case["rows"], case["d"]).to(t), _activations(g, case["rows"], case["d"])
        s["gain"] = 1 + 0.1 * _normal(g, case["d"])
    elif kind == "swiglu":
        s["h"] = _normal(g, case["rows"], 2 * case["F"]).to(t)              # a gate/up product's rows: gates, then ups
    elif kind == "weights":
        s["w"] = (0.02 * _normal(g, case["N"], case["K"])).to(t)
    elif kind == "product":
        s["a"], s["a_scales"] = _quantise(_activations(g, case["M"], case["K"]), case["bits"])
        if case["bits"] == 4:
            s["a"] = _pair(s["a"]).contiguous()
        s["w"] = _pack_weights(*_quantise(0.02 * _normal(g, case["N"], case["K"]), 4))
    else:
        B, L, kv, hd = case["B"], case["L"], case["kv"], case["hd"]
        cap = _up(case["n"] + L, 32)
        s["len"], s["cap"] = _lengths(case, g), cap
        k, v = (_normal(g, B, kv, cap // 32, 32, hd) for _ in range(2))
        if kind == "append":                                        # nothing behind the cached positions yet
            held = (torch.arange(cap, device="cuda") < s["len"][:, None]).view(B, 1, cap // 32, 32, 1)
            k, v = k * held, v * held
        scales = torch.stack((_block_scale(k), _block_scale(v)), -1)
        k, v = (x.mul_(_pow2(scales[..., i], -1)[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8) for i, x in enumerate((k, v)))
        s["cache"], s["scales"] = _pack_cache(k, v), scales.to(torch.uint8)
        if kind == "append":
            qkv = _normal(g, B * L, 3 * kv * hd).to(t)              # a QKV product's rows: queries, keys, values
            s["k"], s["v"] = qkv[:, kv * hd:2 * kv * hd], qkv[:, 2 * kv * hd:]
        else:
            s["q"] = _normal(g, B * L, case["H"] * hd).to(t)
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------
def run(s):
    return (_own if own else _plain)[s["case"]["kind"]](s)


def _plain_norm(s):
    h = s["resid"].add_(s["x"])             # (in place, as from layer to layer)
    y = h * torch.rsqrt(h.square().mean(-1, keepdim=True) + 1e-5) * s["gain"]
    codes, scales = _quantise(y, 8)
    return codes.view(torch.float8_e4m3fn), scales.view(torch.float8_e8m0fnu), h


def _plain_swiglu(s):
    F = s["case"]["F"]
    gate, up = s["h"][:, :F].to(torch.float32), s["h"][:, F:].to(torch.float32)
    codes, scales = _quantise(gate / (1 + torch.exp(-gate)) * up, 8)
    return codes.view(torch.float8_e4m3fn), scales.view(torch.float8_e8m0fnu)


def _plain_weights(s):
    return _pack_weights(*_quantise(s["w"].to(torch.float32), 4))          # (exact, so the bytes have to be equal)


def _plain_product(s):
    c = s["case"]
    a = _unpair(s["a"]) if c["bits"] == 4 else s["a"]
    a = _dequantise(a, s["a_scales"], c["bits"])
    w = _dequantise(*_unpack_weights(s["w"], c["N"], c["K"]), 4)
    return (a @ w.t()).to(_type(c))


def _plain_append(s):
    c = s["case"]
    B, L, kv, hd, cap = c["B"], c["L"], c["kv"], c["hd"], s["cap"]
    at = torch.arange(cap, device="cuda") - s["len"][:, None]                                   # place in the window, < 0: cached
    new, held = ((at >= 0) & (at < L)).view(B, 1, -1, 32, 1), (at < 0).view(B, 1, -1, 32, 1)
    touched = new.any(-2).squeeze(-1)                                                           # [B, 1, blocks]
    row = (at.clamp(0, L - 1) + L * torch.arange(B, device="cuda")[:, None]).view(-1)
    codes, scales = [], []
    for i, (x, old) in enumerate(zip((s["k"], s["v"]), _unpack_cache(s["cache"], hd))):
        x = x[row].to(torch.float32).view(B, cap // 32, 32, kv, hd).permute(0, 3, 1, 2, 4)
        was = old.view(torch.float8_e4m3fn).to(torch.float32) * _pow2(s["scales"][..., i])[..., None, None]
        x = torch.where(new, x, torch.where(held, was, torch.zeros_like(was)))
        sc = _block_scale(x.contiguous())
        x = (x * _pow2(sc, -1)[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        codes.append(torch.where(touched[..., None, None], x, old))
        scales.append(torch.where(touched, sc.to(torch.uint8), s["scales"][..., i]))
    s["cache"].copy_(_pack_cache(*codes))
    s["scales"].copy_(torch.stack(scales, -1))
    return s["cache"].view(torch.float8_e4m3fn), s["scales"].view(torch.float8_e8m0fnu)


def _plain_attention(s):
    c = s["case"]
    B, L, H, kv, hd, cap = c["B"], c["L"], c["H"], c["kv"], c["hd"], s["cap"]
    k, v = (x.view(torch.float8_e4m3fn).to(torch.float32) * _pow2(s["scales"][..., i])[..., None, None]
            for i, x in enumerate(_unpack_cache(s["cache"], hd)))
    k, v = k.reshape(B * kv, cap, hd), v.reshape(B * kv, cap, hd)
    g = H // kv
    q = s["q"].to(torch.float32).view(B, L, kv, g, hd).permute(0, 2, 1, 3, 4).reshape(B * kv, L * g, hd)
    p = torch.bmm(q, k.transpose(1, 2).contiguous()).mul_(1 / math.sqrt(hd)).view(B, kv, L, g, cap)
    p.masked_fill_(~_visible(s).view(B, 1, L, 1, cap), -math.inf)
    p = p.sub_(p.amax(-1, keepdim=True)).exp_()
    den = p.sum(-1, keepdim=True)
    o = torch.bmm(p.view(B * kv, L * g, cap), v).view(B, kv, L, g, hd) / den
    return o.permute(0, 2, 1, 3, 4).reshape(B * L, H * hd).to(_type(c))


def _visible(s):
    """[B, L, cap]: which cached positions a query sees"""
    c = s["case"]
    pos = s["len"].view(-1, 1, 1) + torch.arange(c["L"], device="cuda").view(1, -1, 1)
    key = torch.arange(s["cap"], device="cuda").view(1, 1, -1)
    see = key <= pos
    return see & ((key > pos - c["window"]) | (key < c["sinks"])) if c["window"] else see


_plain = dict(norm=_plain_norm, swiglu=_plain_swiglu, weights=_plain_weights, product=_plain_product, append=_plain_append, attention=_plain_attention)


# The framework's calls.  Outputs and workspaces are buffers that a program keeps from step to step; the first call on a state makes them.
def _kept(s, name, make):
    if name not in s:
        s[name] = make()
    return s[name]


def _bytes(*shape):
    return torch.empty(*shape, dtype=torch.uint8, device="cuda")


def _own_norm(s):
    from paper_2410_01699_amd import binding as B
    rows, Kp = s["case"]["rows"], _up(s["case"]["d"], 128)
    codes, scales = _kept(s, "codes", lambda: _bytes(rows, Kp)), _kept(s, "code_scales", lambda: _bytes(rows, Kp // 32))
    B.sjd_mx_rmsnorm(B.SJD_MX8, s["x"], s["resid"], s["gain"], 1e-5, codes, scales, stream=torch.cuda.current_stream())
    return codes.view(torch.float8_e4m3fn), scales.view(torch.float8_e8m0fnu), s["resid"]


def _own_swiglu(s):
    from paper_2410_01699_amd import binding as B
    rows, F = s["case"]["rows"], s["case"]["F"]
    codes, scales = _kept(s, "codes", lambda: _bytes(rows, _up(F, 128))), _kept(s, "code_scales", lambda: _bytes(rows, _up(F, 128) // 32))
    B.sjd_mx_quantize(B.SJD_MX8, s["h"][:, :F], codes, scales, up=s["h"][:, F:], stream=torch.cuda.current_stream())
    return codes.view(torch.float8_e4m3fn), scales.view(torch.float8_e8m0fnu)


def _own_weights(s):
    from paper_2410_01699_amd import binding as B
    N, K = s["case"]["N"], s["case"]["K"]
    w = _kept(s, "packed", lambda: _bytes(B.sjd_mx_weights_bytes(N, K)).view(-(-N // 16), -(-K // 512), REC))
    B.sjd_mx_weights(s["w"], w, stream=torch.cuda.current_stream())
    return w


def _own_product(s):
    from paper_2410_01699_amd import binding as B
    c = s["case"]
    out = _kept(s, "out", lambda: torch.empty(c["M"], c["N"], dtype=_type(c), device="cuda"))
    ws = _kept(s, "ws", lambda: _bytes(B.sjd_mx_product_workspace(c["M"], c["N"], c["K"])))
    B.sjd_mx_product(B.SJD_MX8 if c["bits"] == 8 else B.SJD_MX4, s["a"], s["a_scales"], s["w"], c["K"], out, ws, stream=torch.cuda.current_stream())
    return out


def _own_append(s):
    from paper_2410_01699_amd import binding as B
    c = s["case"]
    B.sjd_kv8_append(s["k"], s["v"], s["len"], c["L"], c["kv"], c["hd"], s["cap"], s["cache"], s["scales"], stream=torch.cuda.current_stream())
    return s["cache"].view(torch.float8_e4m3fn), s["scales"].view(torch.float8_e8m0fnu)


def _own_attention(s):
    from paper_2410_01699_amd import binding as B
    c = s["case"]
    out = _kept(s, "out", lambda: torch.empty_like(s["q"]))
    ws = _kept(s, "ws", lambda: _bytes(B.sjd_kv8_attention_workspace(c["B"], c["L"], c["H"], c["kv"], c["hd"], s["cap"])))
    B.sjd_kv8_attention(s["q"], s["cache"], s["scales"], s["len"], c["L"], c["H"], c["kv"], c["hd"], s["cap"], c["window"], c["sinks"], out, ws,
                        stream=torch.cuda.current_stream())
    return out


_own = dict(norm=_own_norm, swiglu=_own_swiglu, weights=_own_weights, product=_own_product, append=_own_append, attention=_own_attention)


# ---- what a pass cannot do without --------------------------------------------------------------------------------
def work(case):
    e, kind = 4 if case["dtype"] == "fp32" else 2, case["kind"]
    if kind == "norm":          # x and the residual in, the residual and 33 / 32 bytes a value out
        n = case["rows"] * case["d"]
        return dict(bytes=n * (e + 8 + 33 / 32) + 4 * case["d"], flops=7 * n)
    if kind == "swiglu":
        n = case["rows"] * case["F"]
        return dict(bytes=n * (2 * e + 33 / 32), flops=7 * n)
    if kind == "weights":
        n = case["N"] * case["K"]
        return dict(bytes=n * (e + 17 / 32), flops=4 * n)
    if kind == "product":
        M, N, K = case["M"], case["N"], case["K"]
        return dict(bytes=M * K * (case["bits"] / 8 + 1 / 32) + N * K * 17 / 32 + M * N * e, flops=2 * M * N * K)
    B, L, kv, hd, n = case["B"], case["L"], case["kv"], case["hd"], case["n"]
    mean = n if B == 1 else n * (1 + 0.75 * (B - 1)) / B            # the lengths that prepare() draws, on average
    if kind == "append":        # the window in and out, and what its first block holds already in, half a block on average
        return dict(bytes=2 * B * kv * hd * (L * (e + 1) + (16 if n else 0)), flops=8 * B * L * kv * hd)
    seen = mean + (L + 1) / 2 if not case["window"] else min(mean + (L + 1) / 2, case["window"] + case["sinks"])
    read = mean + L if not case["window"] else min(mean + L, case["window"] + L + case["sinks"])
    return dict(bytes=2 * B * kv * hd * read + 2 * B * L * case["H"] * hd * e, flops=4 * B * L * case["H"] * hd * seen)


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------
def _table(bits):
    """the values of a format's codes, from its definition"""
    v = []
    for code in range(256 if bits == 8 else 16):
        mant, ebits, bias = (3, 4, 7) if bits == 8 else (1, 2, 1)
        e, m = code >> mant & (1 << ebits) - 1, code & (1 << mant) - 1
        a = math.ldexp(1 + m / (1 << mant), e - bias) if e else math.ldexp(m / (1 << mant), 1 - bias)
        a = math.nan if bits == 8 and code & 127 == 127 else a
        v.append(-a if code >> (mant + ebits) else a)
    return torch.tensor(v, dtype=torch.float64, device="cuda")


def _codes64(y, bits):
    """y over its block's scale, before it is rounded, and the scales: [rows, Kp], [rows, Kp / 32] in 64 bits"""
    rows, K = y.shape
    z = torch.zeros(rows, _up(K, 128), dtype=torch.float64, device="cuda")
    z[:, :K] = y
    z = z.view(rows, -1, 32)
    a = z.abs().amax(-1)
    e = torch.ceil(torch.log2(a.clamp_min(1e-300) / (448 if bits == 8 else 6)))
    e = torch.where(a * 2.0 ** -(e - 1) <= (448 if bits == 8 else 6), e - 1, e).clamp(-127, 127)
    return (z * 2.0 ** -e[..., None]).view(rows, -1), 2.0 ** e


def exact(case, seed):
    kind, s = case["kind"], prepare(case, seed)
    if kind == "weights":
        return None                                     # (bytes, which have to be equal)
    if kind == "norm":
        h = s["resid"].double() + s["x"].double()
        y = h / torch.sqrt((h * h).sum(-1, keepdim=True) / case["d"] + 1e-5) * s["gain"].double()
        return (*_codes64(y, 8), h)
    if kind == "swiglu":
        h = s["h"].double()
        return _codes64(h[:, :case["F"]] * torch.sigmoid(h[:, :case["F"]]) * h[:, case["F"]:], 8)
    if kind == "product":
        M, N, K, bits = case["M"], case["N"], case["K"], case["bits"]
        k = torch.arange(K, device="cuda")
        a = s["a"].long()
        a = a[:, k] if bits == 8 else a[:, k // 2] >> 4 * (k % 2) & 15
        a = _table(bits)[a] * 2.0 ** (s["a_scales"][:, k // 32].double() - 127)
        return a @ _weights64(s["w"], N, K).t()
    B, L, kv, hd = case["B"], case["L"], case["kv"], case["hd"]
    if kind == "append":
        return None if B * kv * s["cap"] * hd > 1 << 26 else _append64(s)
    o = torch.empty(B, L, case["H"], hd, dtype=torch.float64, device="cuda")
    see, at = _visible(s), _cache_at(hd)
    for b in range(B):
        for j in range(kv):
            x = _table(8)[s["cache"][b, j].int()][:, at] * 2.0 ** (s["scales"][b, j].double() - 127)[:, :, None, None]     # [blocks, 2, 32, hd]
            k, v = x[:, 0].reshape(-1, hd), x[:, 1].reshape(-1, hd)
            heads = slice(j * (case["H"] // kv), (j + 1) * (case["H"] // kv))
            q = s["q"].double().view(B, L, case["H"], hd)[b, :, heads].reshape(-1, hd)
            w = (q @ k.t() / math.sqrt(hd)).view(L, -1, k.shape[0])
            w = torch.softmax(torch.where(see[b][:, None], w, -math.inf), -1)
            o[b, :, heads] = (w.reshape(-1, k.shape[0]) @ v).view(L, -1, hd)
    return o.view(B * L, -1)


def _weights64(w, N, K):
    """the packed weights' values, each from its place: [N, K]"""
    out = torch.empty(N, K, dtype=torch.float64, device="cuda")
    k = torch.arange(K, device="cuda")
    step, quarter = k % 512 // 128, k % 128 // 32
    table = _table(4)
    for f in range(16):
        rec = w[:(N - f + 15) // 16]                    # the tiles that hold a feature n with n % 16 = f
        code = rec[:, k // 512, step * 1024 + (quarter * 16 + f) * 16 + k % 32 // 2].int() >> 4 * (k % 2).int() & 15
        scale = rec[:, k // 512, 4096 + (quarter * 16 + f) * 4 + step].double()
        out[f::16] = table[code] * 2.0 ** (scale - 127)
    return out


def _cache_at(hd):
    """[2, 32, hd]: the byte of position p, dimension d of K and V in a block's record"""
    p, d = torch.arange(32, device="cuda")[:, None], torch.arange(hd, device="cuda")[None]
    ok, lk, ek = p // 16 * (hd // 32) + d // 32, d % 32 // 8 * 16 + p % 16, d % 8
    ov, lv, ev = d // 16 + 0 * p, p % 16 // 4 * 16 + d % 16, p // 16 * 4 + p % 4
    return torch.stack([o // 2 * 1024 + lane * 16 + o % 2 * 8 + e + i * 32 * hd for i, (o, lane, e) in enumerate(((ok, lk, ek), (ov, lv, ev)))])


def _append64(s):
    """the codes before they are rounded, and the scales"""
    c = s["case"]
    L, kv, hd, at = c["L"], c["kv"], c["hd"], _cache_at(c["hd"])
    codes, scales = _table(8)[s["cache"].int()], 2.0 ** (s["scales"].double() - 127)
    for b, n in enumerate(s["len"].tolist()):
        for blk in range(n // 32, (n + L + 31) // 32):
            for i, x in enumerate((s["k"], s["v"])):
                old = codes[b, :, blk][:, at[i]] * scales[b, :, blk, i, None, None]         # [kv, 32, hd]
                lo, hi = max(n, 32 * blk), min(n + L, 32 * blk + 32)
                old[:, lo - 32 * blk:] = 0
                old[:, lo - 32 * blk:hi - 32 * blk] = x[b * L + lo - n:b * L + hi - n].double().view(-1, kv, hd).transpose(0, 1)
                y, e = _block64(old.reshape(kv, -1))
                codes[b, :, blk][:, at[i].reshape(-1)] = y
                scales[b, :, blk, i] = e
    return codes, scales


def _block64(z):
    a = z.abs().amax(-1)
    e = torch.ceil(torch.log2(a.clamp_min(1e-300) / 448))
    e = torch.where(a * 2.0 ** -(e - 1) <= 448, e - 1, e).clamp(-127, 127)
    return z * 2.0 ** -e[:, None], 2.0 ** e
