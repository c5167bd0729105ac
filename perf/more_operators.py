"""What is timed of the operators around a decoder layer's products when its keys and values lie in pages: one call each.

A case is one call (`kind`):

  rope       heads of rows (queries and keys of a QKV product) turned by their positions: half or interleaved pairs, all of a head or its
             first dimensions, frequencies plain or scaled for contexts longer than the trained one
  append     the keys and values of every sequence's new tokens into the pages of its cache, the keys (and the queries, into rows of their
             own) turned on the way
  attention  the new tokens' queries over the paged cache: causal, grouped heads, any number of tokens a sequence, sliding window and sinks;
             sequences that begin with the same pages (one prompt, several images) have that prefix computed once for all
  norm       h = resid + scale * gate * RMSNorm(x), kept; RMSNorm(h): the norm behind one block, its gate and residual scale, the norm before the next

The cache.  A pool of pages of `page` positions, [n_pages][kv heads][page / 32] records of 64 * hd values; position p of a sequence is in the
page that entry p / page of its table row names.  A record holds the keys, then the values of 32 positions, in units of 16 bytes (E = 8
bf16 or 4 fp32):
  K[p][d] at E (32 (d / E) + p) + d % E
  V[p][d] at 32 hd + E (32 E' (d / 32) + 32 u + d % 32) + e, E' = 32 / E, where bf16: p = 16 t + 8 j + 4 h + i, u = 2 t + h, e = 4 j + i;
                                                                               fp32: u = p / 4, e = p % 4
Frequencies are whole numbers of 2^-64 turns a position, so that a position's angle is a product of whole numbers.

Sizes are those of the repository's own decoders (widths 1536 and 4096, heads of 64 and 128, windows of 16 drafts, 8 images) or generic ones around
them.
"""
from __future__ import annotations

import math

import torch

own = False

HEADS = {64: 24, 128: 32}                  # the two decoders' heads by their size


def listed():
    return [
        # queries and keys of one token of the 4096-wide decoder: nothing but latency
        dict(name="rope_token", kind="rope", rows=1, heads=64, hd=128, rot=128, pairs="half", scaling="plain", at=1087, dtype="fp32"),
        # a long document's rows behind 100 k positions, grouped heads, half of each head turned, a context stretched 16 times
        dict(name="rope_prompt", kind="rope", rows=4001, heads=40, hd=128, rot=64, pairs="interleaved", scaling="parts", at=100000, dtype="bf16"),
        # one decoding step of eight images: windows of 16 drafts behind caches of different lengths
        dict(name="append_window", kind="append", B=8, L=16, ragged=False, H=32, kv=32, hd=128, rot=128, pairs="half", scaling="plain", n=583, page=32, dtype="fp32"),
        # six prompts of up to 1000 tokens of a batch, grouped heads
        dict(name="append_prompt", kind="append", B=6, L=1000, ragged=True, H=32, kv=8, hd=128, rot=128, pairs="interleaved", scaling="linear", n=0, page=64, dtype="bf16"),
        # one token late in a 64 x 64 image, every query head its own keys
        dict(name="attention_token", kind="attention", B=1, L=1, ragged=False, H=32, kv=32, hd=128, n=4095, prefix=0, window=0, sinks=0, page=32, dtype="fp32"),
        # windows of 16 drafts of eight images of different lengths
        dict(name="attention_window", kind="attention", B=8, L=16, ragged=False, H=32, kv=32, hd=128, n=1239, prefix=0, window=0, sinks=0, page=64, dtype="fp32"),
        # eight images of the narrow decoder, windows of 16 drafts, behind one long prompt
        dict(name="attention_drafts", kind="attention", B=8, L=16, ragged=False, H=24, kv=24, hd=64, n=1650, prefix=1121, window=0, sinks=0, page=32, dtype="bf16"),
        # sixteen conversations, one token each, behind one long document: grouped heads
        dict(name="attention_prefix", kind="attention", B=16, L=1, ragged=False, H=32, kv=8, hd=128, n=14600, prefix=14001, window=0, sinks=0, page=128, dtype="bf16"),
        # few tokens on a very long cache of which a sliding window and the prompt's first tokens stay visible
        dict(name="attention_sinks", kind="attention", B=3, L=5, ragged=True, H=32, kv=4, hd=128, n=50001, prefix=0, window=16384, sinks=64, page=256, dtype="bf16"),
        # two prompts of about 2000 tokens: the matrix cores are what is left
        dict(name="attention_prompt", kind="attention", B=2, L=2040, ragged=True, H=32, kv=8, hd=128, n=0, prefix=0, window=0, sinks=0, page=64, dtype="bf16"),
        # one token between two blocks of the 4096-wide decoder
        dict(name="norm_token", kind="norm", rows=1, d=4096, gate="vector", dtype="fp32"),
        # a long prompt's rows through the same norms, each row with a gate of its own
        dict(name="norm_prompt", kind="norm", rows=2048, d=4096, gate="rows", dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def _drawn_turn(rng, hd):
    rot = rng.choice([hd, hd, hd // 2, 2 * rng.randint(1, hd // 2)])
    return dict(rot=rot, pairs=rng.choice(["half", "interleaved"]), scaling=rng.choice(["plain", "linear", "parts"]))


def _drawn(rng):
    kind = rng.choice(["rope", "append", "append", "attention", "attention", "attention", "attention", "norm"])
    dtype = rng.choice(["fp32", "bf16"])
    if kind == "norm":
        return dict(kind=kind, rows=_log_int(rng, 1, 4096), d=rng.choice([1536, 4096, _log_int(rng, 64, 8192)]), gate=rng.choice(["none", "vector", "rows"]), dtype=dtype)
    hd = rng.choice([64, 128, 128, 96])
    kv = rng.choice([1, 4, 8, HEADS.get(hd, 16)])
    H = kv * rng.choice([1, 1, 4, 7, 8]) if kv <= 8 else kv
    if kind == "rope":
        return dict(kind=kind, rows=_log_int(rng, 1, 4096), heads=H + kv, hd=hd, **_drawn_turn(rng, hd), at=_log_int(rng, 1, 1000000), dtype=dtype)
    B, page = rng.choice([1, 1, 2, 3, 5, 8, 16, 33]), rng.choice([32, 64, 128, 256])
    if kind == "append":
        return dict(kind=kind, B=B, L=_log_int(rng, 1, 1024), ragged=rng.random() < 0.5, H=H, kv=kv, hd=hd, **_drawn_turn(rng, hd), n=rng.choice([0, rng.randint(1, 4096)]), page=page, dtype=dtype)
    n = _log_int(rng, 1, 65536 // B) if rng.random() < 0.8 else 0
    near, shared = rng.random() < 0.25, B > 1 and n and rng.random() < 0.6
    return dict(kind=kind, B=B, L=_log_int(rng, 1, 2048), ragged=rng.random() < 0.5, H=H, kv=kv, hd=hd, n=n, prefix=rng.randint(1, n) if shared else 0,
                window=_log_int(rng, 1, max(2, n)) if near else 0, sinks=rng.choice([0, 4, 64, 121]) if near else 0, page=page, dtype=dtype)


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        c = _drawn(rng)
        cap = c.get("n", 0) + c.get("L", 0) + c.get("page", 0)
        held, scores = c.get("B", 0) * c.get("kv", 0) * cap * c.get("hd", 0), c.get("B", 0) * c.get("H", 0) * c.get("L", 0) * cap
        if _cost(c) <= most and held <= 1 << 28 and (scores <= 1 << 28 or c["kind"] == "append"):      # (the plain form holds all of them in 32 bits)
            return c


# ---- what a case means --------------------------------------------------------------------------------------------
def _type(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def _tokens(case):
    """new tokens per sequence: L for the first, where they are ragged shorter ones behind it"""
    L = case["L"]
    return [L - (b * 37 * (L // 7 + 1)) % (L // 2 + 1) if case["ragged"] else L for b in range(case["B"])]


def _cached(case):
    """cached positions per sequence: n for the first, shorter ones behind it, never less than the shared prefix"""
    n, least = case["n"], max(case.get("prefix", 0), case["n"] // 2)
    return [n - int((b * 0.618034 % 1.0) * (n - least)) for b in range(case["B"])]


def _frequencies(case):
    """radians a position of every pair"""
    f = 10000.0 ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64) / case["rot"])
    if case["scaling"] == "linear":
        return f / 4
    if case["scaling"] == "parts":              # pairs that turn less than once in the trained 4096 positions 16 times slower, 32 times or more as they are
        keep = ((4096 * f / (2 * math.pi) - 1) / 31).clamp(0, 1)
        return f * keep + f / 16 * (1 - keep)
    return f


def _magnitude(case):
    return 0.1 * math.log(16) + 1 if case["scaling"] == "parts" else 1.0


def _turns(f):
    """the same in 2^-64 turns, as 64-bit whole numbers"""
    whole = [round(x / (2 * math.pi) * 2.0 ** 64) % 2 ** 64 for x in f.tolist()]
    return torch.tensor([x - 2 ** 64 if x >= 2 ** 63 else x for x in whole], dtype=torch.int64)


def _units(case):
    return 8 if case["dtype"] == "bf16" else 4


# ---- inputs -------------------------------------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 29)


def _normal(g, *shape):
    return torch.randn(*shape, device="cuda", generator=g)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g, t, kind = _gen(seed), _type(case), case["kind"]
    s = dict(case=dict(case))
    if kind == "norm":
        rows, d = case["rows"], case["d"]
        s["x"], s["resid"] = _normal(g, rows, d).to(t), _normal(g, rows, d)
        s["resid"][:, torch.randint(0, d, (max(1, d // 512),), device="cuda", generator=g)] *= 20      # (a residual stream has a few large channels)
        s["post"], s["pre"] = 1 + 0.1 * _normal(g, d), 1 + 0.1 * _normal(g, d)
        s["gate"] = None if case["gate"] == "none" else _normal(g, 1 if case["gate"] == "vector" else rows, d).to(t)
        return s
    if "rot" in case:
        f = _frequencies(case)
        s["frequencies"], s["turns"] = f.cuda(), _turns(f).cuda()
    hd = case["hd"]
    if kind == "rope":
        rows, heads = case["rows"], case["heads"]
        s["x"] = _normal(g, rows, heads * hd + 4 * hd).to(t)[:, :heads * hd]              # (values stand behind the heads that turn)
        s["pos"] = torch.arange(case["at"], case["at"] + rows, dtype=torch.int32, device="cuda")
        s["pos"] = s["pos"][torch.randperm(rows, device="cuda", generator=g)].contiguous()
        return s
    B, H, kv, page = case["B"], case["H"], case["kv"], case["page"]
    tokens, cached = _tokens(case), _cached(case)
    s["start"], s["len"] = _ints([sum(tokens[:b]) for b in range(B + 1)]), _ints(cached)
    width = max(-(-(n + m) // page) for n, m in zip(cached, tokens))
    shared = case.get("prefix", 0) // page                                              # whole pages that all tables begin with
    s["pages"] = B * (width - shared) + shared + 3
    ids = torch.randperm(s["pages"], device="cuda", generator=g).to(torch.int32)
    s["table"] = torch.cat((ids[:shared].expand(B, shared), ids[shared:shared + B * (width - shared)].view(B, -1)), 1).contiguous()
    s["cache"] = _normal(g, s["pages"], kv, page // 32, 64 * hd).to(t)
    rows = sum(tokens)
    if kind == "append":
        qkv = _normal(g, rows, (H + 2 * kv) * hd).to(t)                                 # a QKV product's rows
        s["q"], s["k"], s["v"] = qkv[:, :H * hd], qkv[:, H * hd:(H + kv) * hd], qkv[:, (H + kv) * hd:]
    else:
        s["q"] = _normal(g, rows, H * hd).to(t)
        if case["prefix"]:
            s["groups"], s["prefix"] = _ints([0, B]), _ints([case["prefix"]])
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------
def run(s):
    return (_own if own else _plain)[s["case"]["kind"]](s)


def _turned(s, x, pos):
    """heads [rows, n, hd] turned by their rows' positions, in 32 bits"""
    c, x = s["case"], x.to(torch.float32)
    rot = c["rot"]
    angle = pos.to(torch.float64)[:, None] * s["frequencies"]
    cos, sin = ((f * _magnitude(c)).to(torch.float32)[:, None] for f in (torch.cos(angle), torch.sin(angle)))
    if c["pairs"] == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    return torch.cat((y, x[..., rot:]), -1)


def _plain_rope(s):
    c = s["case"]
    return _turned(s, s["x"].reshape(c["rows"], -1, c["hd"]), s["pos"]).to(_type(c)).view(c["rows"], -1)


def _rows(s):
    """sequence and position of every row"""
    row = torch.arange(s["q"].shape[0], device="cuda")
    seq = (row[:, None] >= s["start"][None, 1:]).sum(-1)
    return seq, row - s["start"][seq] + s["len"][seq]


def _pack(k, v, E):
    """values [..., 32, hd] of a record's keys and values -> [..., 64 * hd]"""
    lead, hd = k.shape[:-2], k.shape[-1]
    k = k.reshape(-1, 32, hd // E, E).transpose(1, 2).reshape(-1, 32 * hd)
    if E == 8:
        v = v.reshape(-1, 2, 2, 2, 4, hd // 32, 32).permute(0, 5, 1, 3, 6, 2, 4).reshape(-1, 32 * hd)       # t, j, h, i -> (t, h), (j, i)
    else:
        v = v.reshape(-1, 8, 4, hd // 32, 32).permute(0, 3, 1, 4, 2).reshape(-1, 32 * hd)
    return torch.cat((k, v), -1).view(*lead, 64 * hd)


def _unpack(rec, hd, E):
    lead = rec.shape[:-1]
    k, v = rec.reshape(-1, 2, 32 * hd).unbind(1)
    k = k.reshape(-1, hd // E, 32, E).transpose(1, 2).reshape(*lead, 32, hd)
    if E == 8:
        v = v.reshape(-1, hd // 32, 2, 2, 32, 2, 4).permute(0, 2, 5, 3, 6, 1, 4).reshape(*lead, 32, hd)
    else:
        v = v.reshape(-1, hd // 32, 8, 32, 4).permute(0, 2, 4, 1, 3).reshape(*lead, 32, hd)
    return k, v


def _plain_append(s):
    c = s["case"]
    kv, hd, page, t = c["kv"], c["hd"], c["page"], _type(c)
    seq, pos = _rows(s)
    q = _turned(s, s["q"].reshape(len(seq), -1, hd), pos).to(t).view(len(seq), -1)
    k = _turned(s, s["k"].reshape(len(seq), kv, hd), pos).to(t)
    where = s["table"][seq, pos // page].long() * (page // 32) + pos % page // 32                  # record of every row, heads apart
    at, of = torch.unique(where, return_inverse=True)                                             # records that are touched
    pool = s["cache"].view(s["pages"], kv, page // 32, 64 * hd)
    page_of, part = at // (page // 32), at % (page // 32)
    old_k, old_v = _unpack(pool[page_of, :, part], hd, _units(c))                                 # [touched, kv, 32, hd]
    old_k[of, :, pos % 32], old_v[of, :, pos % 32] = k, s["v"].reshape(len(seq), kv, hd)
    pool[page_of, :, part] = _pack(old_k, old_v, _units(c))
    return s["cache"], q


def _visible(s, pos, cap):
    """which of the positions 0 .. cap - 1 a query at `pos` sees"""
    c, pos, key = s["case"], pos[..., None], torch.arange(cap, device="cuda")
    see = key <= pos
    return see & ((key > pos - c["window"]) | (key < c["sinks"])) if c["window"] else see


def _plain_attention(s):
    c = s["case"]
    B, L, H, kv, hd = c["B"], c["L"], c["H"], c["kv"], c["hd"]
    cap, g = s["table"].shape[1] * c["page"], H // kv
    k, v = (x.permute(0, 2, 1, 3, 4, 5).reshape(B * kv, cap, hd).to(torch.float32) for x in _unpack(s["cache"][s["table"].long()], hd, _units(c)))
    row = s["start"][:-1, None] + torch.arange(L, device="cuda")                                  # [B, L], rows behind a sequence's last are another's
    q = s["q"][row.clamp_max(s["q"].shape[0] - 1)].to(torch.float32).view(B, L, kv, g, hd).permute(0, 2, 1, 3, 4).reshape(B * kv, L * g, hd)
    p = torch.bmm(q, k.transpose(1, 2).contiguous()).mul_(1 / math.sqrt(hd)).view(B, kv, L, g, cap)
    pos = s["len"][:, None] + torch.arange(L, device="cuda")
    p.masked_fill_(~_visible(s, pos, cap).view(B, 1, L, 1, cap), -math.inf)
    p = p.sub_(p.amax(-1, keepdim=True)).exp_()
    den = p.sum(-1, keepdim=True)
    o = torch.bmm(p.view(B * kv, L * g, cap), v).view(B, kv, L, g, hd) / den
    o = o.permute(0, 2, 1, 3, 4).reshape(B, L, H * hd)
    return o[row < s["start"][1:, None]].to(_type(c))


def _plain_norm(s):
    x = s["x"].to(torch.float32)
    y = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-5) * s["post"]
    h = s["resid"].add_(0.5 * (y if s["gate"] is None else s["gate"].to(torch.float32) * y))      # (in place, as from layer to layer)
    return (h * torch.rsqrt(h.square().mean(-1, keepdim=True) + 1e-5) * s["pre"]).to(_type(s["case"])), h


_plain = dict(rope=_plain_rope, append=_plain_append, attention=_plain_attention, norm=_plain_norm)


# The framework's calls.  Outputs and workspaces are buffers that a program keeps from step to step; the first call on a state makes them.
def _kept(s, name, make):
    if name not in s:
        s[name] = make()
    return s[name]


def _pool(s, B):
    c = s["case"]
    return _kept(s, "pool", lambda: B.sjd_pages(0 if c["dtype"] == "fp32" else 1, c["kv"], c["hd"], c["page"], s["pages"]))


def _own_rope(s):
    from paper_2410_01699_amd import binding as B
    c = s["case"]
    out = _kept(s, "out", lambda: torch.empty(s["x"].shape, dtype=s["x"].dtype, device="cuda"))
    B.sjd_rope(s["x"], out, s["pos"], c["hd"], s["turns"], interleaved=c["pairs"] == "interleaved", magnitude=_magnitude(c), stream=torch.cuda.current_stream())
    return out


def _own_append(s):
    from paper_2410_01699_amd import binding as B
    c = s["case"]
    out = _kept(s, "out", lambda: torch.empty(s["q"].shape, dtype=s["q"].dtype, device="cuda"))
    B.sjd_page_append(_pool(s, B), s["k"], s["v"], s["start"], s["len"], s["table"], s["cache"], turns=s["turns"], interleaved=c["pairs"] == "interleaved",
                      magnitude=_magnitude(c), q=s["q"], q_out=out, stream=torch.cuda.current_stream())
    return s["cache"], out


def _own_attention(s):
    from paper_2410_01699_amd import binding as B
    c = s["case"]
    rows, width = s["q"].shape[0], s["table"].shape[1]
    out = _kept(s, "out", lambda: torch.empty_like(s["q"]))
    ws = _kept(s, "ws", lambda: torch.empty(B.sjd_page_attention_workspace(_pool(s, B), rows, c["B"], 1 if c["prefix"] else 0, c["H"], width), dtype=torch.uint8, device="cuda"))
    B.sjd_page_attention(_pool(s, B), s["q"], s["start"], s["len"], s["table"], s["cache"], out, ws, scale=1 / math.sqrt(c["hd"]), window=c["window"], sinks=c["sinks"],
                         groups=s.get("groups"), prefix=s.get("prefix"), stream=torch.cuda.current_stream())
    return out


def _own_norm(s):
    from paper_2410_01699_amd import binding as B
    out = _kept(s, "out", lambda: torch.empty_like(s["x"]))
    B.sjd_block_norm(s["x"], s["resid"], 1e-5, out, post=s["post"], gate=s["gate"], scale=0.5, pre=s["pre"], stream=torch.cuda.current_stream())
    return out, s["resid"]


_own = dict(rope=_own_rope, append=_own_append, attention=_own_attention, norm=_own_norm)


# ---- what a pass cannot do without --------------------------------------------------------------------------------
def work(case):
    e, kind = 4 if case["dtype"] == "fp32" else 2, case["kind"]
    if kind == "norm":          # x, the residual (and a gate) in; the residual and the normed rows out
        n = case["rows"] * case["d"]
        gate = n if case["gate"] == "rows" else case["d"] if case["gate"] == "vector" else 0
        return dict(bytes=n * (2 * e + 8) + gate * e + 8 * case["d"], flops=10 * n)
    if kind == "rope":
        n = case["rows"] * case["heads"] * case["hd"]
        return dict(bytes=2 * n * e + 4 * case["rows"], flops=3 * case["rows"] * case["heads"] * case["rot"])
    kv, hd, tokens, cached = case["kv"], case["hd"], _tokens(case), _cached(case)
    if kind == "append":
        n = sum(tokens) * (case["H"] + 2 * kv) * hd
        return dict(bytes=2 * n * e, flops=3 * sum(tokens) * (case["H"] + kv) * case["rot"])
    w, sinks = case["window"] or 1 << 30, case["sinks"]
    read, seen = 0, 0
    for n, m in zip(cached, tokens):
        first = max(0, n + 1 - w)                                                   # of the first query's window
        read += n + m - first + min(sinks, first)
        seen += sum(min(p + 1, w) + min(sinks, max(0, p + 1 - w)) for p in range(n, n + m)) if m < 64 else \
            m * min((2 * n + m + 1) / 2, w + sinks)
    if case["prefix"]:                                                              # read once for all
        first = max(0, min(cached) + 1 - w)
        read -= (case["B"] - 1) * max(0, case["prefix"] - first + min(sinks, first, case["prefix"]))
    return dict(bytes=2 * kv * hd * max(read, 1) * e + 2 * sum(tokens) * case["H"] * hd * e, flops=4 * case["H"] * hd * seen)


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------
def _turned64(case, x, pos):
    """heads [rows, n, hd] in 64 bits as complex numbers times e^(i angle)"""
    x, rot = x.double(), case["rot"]
    one, two = (slice(0, rot // 2), slice(rot // 2, rot)) if case["pairs"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    angle = pos.double()[:, None, None] * _frequencies(case).cuda()
    z = torch.complex(x[..., one], x[..., two]) * torch.polar(torch.full_like(angle, _magnitude(case)), angle)
    x = x.clone()
    x[..., one], x[..., two] = z.real, z.imag
    return x


def _record_at(hd, E):
    """[2, 32, hd]: the place of position p, dimension d of K and V in a record"""
    p, d = torch.arange(32, device="cuda")[:, None], torch.arange(hd, device="cuda")[None]
    k = E * (32 * (d // E) + p) + d % E
    u, e = (p // 16 * 2 + p // 4 % 2, p // 8 % 2 * 4 + p % 4) if E == 8 else (p // 4, p % 4)
    return torch.stack((k, 32 * hd + E * (32 * (32 // E) * (d // 32) + 32 * u + d % 32) + e))


def exact(case, seed):
    kind, s = case["kind"], prepare(case, seed)
    if kind == "norm":
        x, h = s["x"].double(), s["resid"].double()
        y = x / torch.sqrt((x * x).sum(-1, keepdim=True) / case["d"] + 1e-5) * s["post"].double() * 0.5
        h = h + (y if s["gate"] is None else y * s["gate"].double())
        return h / torch.sqrt((h * h).sum(-1, keepdim=True) / case["d"] + 1e-5) * s["pre"].double(), h
    hd = case["hd"]
    if kind == "rope":
        return _turned64(case, s["x"].reshape(case["rows"], -1, hd), s["pos"]).view(case["rows"], -1)
    B, H, kv, page, at = case["B"], case["H"], case["kv"], case["page"], _record_at(hd, _units(case))
    start, table = s["start"].tolist(), s["table"].long()
    if kind == "append":
        if s["cache"].numel() > 1 << 28:
            return None
        cache, q = s["cache"].double(), torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
        for b, n in enumerate(s["len"].tolist()):
            rows = slice(start[b], start[b + 1])
            pos = torch.arange(n, n + start[b + 1] - start[b], device="cuda")
            q[rows] = _turned64(case, s["q"][rows].reshape(len(pos), H, hd), pos).view(len(pos), -1)
            k = _turned64(case, s["k"][rows].reshape(len(pos), kv, hd), pos)
            for x, a in ((k, at[0]), (s["v"][rows].reshape(len(pos), kv, hd).double(), at[1])):
                cache[table[b, pos // page][:, None, None], torch.arange(kv, device="cuda")[:, None], (pos % page // 32)[:, None, None], a[pos % 32][:, None]] = x
        return cache, q
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    for b, n in enumerate(s["len"].tolist()):
        m = start[b + 1] - start[b]
        see = _visible(s, torch.arange(n, n + m, device="cuda"), table.shape[1] * page)
        for j in range(kv):
            x = s["cache"][table[b], j][..., at].double()                             # [pages, page / 32, 2, 32, hd]
            k, v = x[:, :, 0].reshape(-1, hd), x[:, :, 1].reshape(-1, hd)
            cols = slice(j * (H // kv) * hd, (j + 1) * (H // kv) * hd)
            q = s["q"][start[b]:start[b + 1], cols].double().reshape(-1, hd)
            w = (q @ k.t() / math.sqrt(hd)).view(m, -1, k.shape[0])
            w = torch.softmax(torch.where(see[:, None], w, -math.inf), -1)
            out[start[b]:start[b + 1], cols] = (w.reshape(-1, k.shape[0]) @ v).view(m, -1)
    return out
