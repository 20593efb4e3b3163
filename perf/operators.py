"""Timing cases of the operators next to the cascading cache: per-head norms of queries and keys with the position rotation
(`norm`), appending to a paged cache held in 4 bits with the rotation on the way (`append`) and attention over that cache
(`attend`: one token, a few, chunks, ragged batches).

Page format (the same bytes on both sides).  A page holds `page_size` consecutive tokens of one sequence; per KV head it is a row of
groups of 32 tokens.  Token r of a group, channel c of d, in a group of GROUP bytes (a multiple of 128):
  K codes at 0:            byte (c / 32) * 512 + r * 16 + c % 32 / 2, low four bits for even c
  V codes at 16 d:         byte (c / 64) * 1024 + (r / 4 % 4) * 256 + c % 16 * 16 + c / 32 % 2 * 8 + r / 16 * 4 + r % 4, low four bits where c / 16 is even
  K exponents at 32 d:     byte (c / 32) * 32 + r % 16 * 2 + r / 16, scale 2^(byte - 127)
  V scales at 32 d + d:    bf16 number (r / 4 % 4) * 8 + r / 16 * 4 + r % 4
A code is a sign bit and three bits that stand for 0, 0.5, 1, 1.5, 2, 3, 4, 6.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
ROPE_POSITIONS = 1 << 18

BASE = dict(op="attend", dtype="bf16", hq=32, hkv=8, d=128, page=64, seqs=1, new=1, context=4096, ragged=False, rope=True, norm=True, window=0,
            base=500000.0, fused=True)


def listed():
    def case(name, **over):
        return dict(BASE, name=name, **over)

    return [
        # the norms of one generated token: latency of a launch
        case("norm_1", op="norm", context=70000),
        # a chunk of a prompt, q and k as views of a fused projection
        case("norm_4096", op="norm", new=4096, context=65536),
        # fp32, norms alone (the cascading cache rotates by itself), odd number of tokens
        case("norm_f32_1000_d64", op="norm", dtype="f32", hq=16, hkv=2, d=64, new=1000, rope=False, fused=False),
        # one token for each of 32 sequences, its queries rotated in the same call
        case("append_b32", op="append", seqs=32, context=16384, ragged=True),
        # a chunk of a long prompt, from a position inside a page
        case("append_4096", op="append", new=4096, context=40009),
        # fp32, a ragged batch with odd lengths, small pages
        case("append_f32_ragged_d64", op="append", dtype="f32", hq=16, hkv=2, d=64, page=32, seqs=5, new=301, context=777, ragged=True, base=10000.0),
        # interactive generation on one long conversation
        case("decode_b1_128k", context=131071),
        # a serving batch of 32 sequences of different lengths
        case("decode_b32_16k", seqs=32, context=16384, ragged=True),
        # fp32, short caches: latency
        case("decode_f32_b4_1k_d64", dtype="f32", hq=16, hkv=2, d=64, page=32, seqs=4, context=1000, ragged=True),
        # a whole new prompt
        case("chunk_4096_fresh", new=4096, context=0),
        # a chunk late in a long prompt
        case("chunk_2048_on_64k", new=2048, context=63500, page=128),
        # requests in all states in one call (single tokens, a sequence without any, chunks), sliding window
        case("mixed_b8_window", d=64, hq=16, hkv=4, seqs=8, new=400, context=3000, ragged=True, window=1024),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = [work(c) for c in listed()]
    most = {k: max(w[k] for w in most) for k in ("bytes", "flops")}
    while True:
        c = dict(BASE)
        c["op"] = rng.choices(["norm", "append", "attend"], [2, 3, 6])[0]
        c["dtype"] = rng.choices(["bf16", "f32"], [3, 1])[0]
        c["d"] = rng.choice([64, 128, 128])
        c["hkv"] = rng.choice([1, 2, 4, 8, 8])
        c["hq"] = c["hkv"] * rng.choice([1, 2, 4, 4, 5, 8])
        c["page"] = rng.choice([32, 64, 64, 96, 128, 256])
        c["seqs"] = _log_int(rng, 1, 48)
        c["context"] = _log_int(rng, 1, 131072) if rng.random() < 0.9 else 0
        c["new"] = 1 if rng.random() < 0.4 else _log_int(rng, 2, 4096)
        c["ragged"] = c["seqs"] > 1 and rng.random() < 0.7
        c["base"] = rng.choice([10000.0, 500000.0])
        c["rope"] = rng.random() < 0.8
        c["norm"] = c["op"] != "norm" or not c["rope"] or rng.random() < 0.8
        c["fused"] = rng.random() < 0.5
        c["window"] = _log_int(rng, 1, 8192) if c["op"] == "attend" and rng.random() < 0.2 else 0
        if c["op"] == "norm":
            c["seqs"], c["ragged"] = 1, False
        if c["dtype"] == "f32" and c["new"] * c["seqs"] > 4096:
            continue
        w = work(c)
        # what the plain form holds at once: the logits of all queries, padded to the longest sequence, and the keys in 32 bits
        keys = c["seqs"] * (c["context"] + c["new"])
        if c["op"] == "attend" and (c["hq"] * c["new"] * keys > 5e9 or c["hkv"] * c["d"] * keys > 7e8):
            continue
        if w["bytes"] <= most["bytes"] and w["flops"] <= most["flops"]:
            return c


def _torch_dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _lengths(c):
    """Tokens cached and new tokens of every sequence: those of the case, or for a ragged batch numbers below (a single token and
    none among the new ones where there are several)."""
    n = c["seqs"]
    if not c["ragged"]:
        return [c["context"]] * n, [c["new"]] * n
    have = [c["context"] * (1 + (37 * i + 11) % 64) // 64 for i in range(n)]
    new = [c["new"] if i == 0 or c["new"] == 1 else 0 if i == 2 else 1 if i % 3 == 1 else 1 + (c["new"] - 1) * ((29 * i) % 64) // 64 for i in range(n)]
    return have, new


def _group_bytes(d):
    return -(-(33 * d + 64) // 128) * 128


def work(case):
    c = dict(BASE, **case)
    e, d = 2 if c["dtype"] == "bf16" else 4, c["d"]
    have, new = _lengths(c)
    t = sum(new)
    row = d + d // 32 + 2      # a cached key and value
    if c["op"] == "norm":
        n = c["new"] * (c["hq"] + c["hkv"]) * d
        return {"bytes": 2.0 * n * e + 2 * d * e + 4 * c["new"], "flops": 10.0 * n}
    if c["op"] == "append":      # keys and values in, codes out and back as values; queries in and out
        nbytes = t * c["hkv"] * (2 * d * e + 2 * row + 2 * d * e) + (2.0 * t * c["hq"] * d * e if c["rope"] else 0)
        return {"bytes": float(nbytes), "flops": 20.0 * t * c["hkv"] * d}
    keys = pairs = 0
    for h, n in zip(have, new):
        w = c["window"] or h + n
        keys += min(h + n, w + n - 1) if n else 0
        full = max(0, min(n, w - h))      # rows that see all keys before them
        pairs += full * h + full * (full + 1) // 2 + (n - full) * w
    return {"bytes": float(keys * c["hkv"] * row + 2 * t * c["hq"] * d * e), "flops": 4.0 * d * c["hq"] * pairs}


# ---------------------------------------------------------------- the plain form

VALUES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _rotated(x, positions, base):
    """x [tokens, heads, d] turned to its positions, in 64 bits: what is next to a border between two codes has to fall on its side."""
    d = x.shape[-1]
    theta = base ** (torch.arange(d // 2, device=x.device, dtype=torch.float64) * (-2.0 / d))
    angle = positions.double()[:, None, None] * theta
    lo, hi = x.double().chunk(2, -1)
    return torch.cat([lo * angle.cos() - hi * angle.sin(), hi * angle.cos() + lo * angle.sin()], -1)


def _codes(y):
    """The nearest codes of y, ties to the even code."""
    a = y.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)).to(torch.uint8)
    return code | ((y < 0).to(torch.uint8) << 3)


def _quantised(k, v):
    """K codes, K exponents (biased), V codes and V scales of rows [tokens, heads, d]."""
    blocks = k.unflatten(-1, (-1, 32))
    frac, exp = torch.frexp(blocks.abs().amax(-1))      # amax = frac * 2^exp, 1/2 <= frac < 1; 7 * 2^e >= amax
    exp = torch.where(frac > 0, (exp - 3 + (frac > 0.875)).clamp(-126, 127), torch.full_like(exp, -127))
    k_codes = _codes(torch.ldexp(blocks, -exp[..., None])).flatten(-2)
    scale = (v.float().abs().amax(-1) / 6.0).bfloat16()
    v_codes = _codes(v.double() / torch.where(scale > 0, scale, torch.ones_like(scale)).double()[..., None])
    return k_codes, (exp + 127).to(torch.uint8), v_codes, scale


def _places(c, batch):
    """For every new token: its sequence, its number in it and its position."""
    t = torch.arange(batch["n_tokens"], device=DEVICE)
    seq = torch.searchsorted(batch["new_offsets"].long(), t, right=True) - 1
    i = t - batch["new_offsets"].long()[seq]
    return seq, i, batch["lengths"].long()[seq] + i


def _byte_places(c, batch, seq, pos):
    """Where in the pages' bytes the new tokens' K codes, V codes, K exponents and V scales sit."""
    d, heads = c["d"], torch.arange(c["hkv"], device=DEVICE)
    page = batch["page_table"].long()[seq, pos // c["page"]]
    at = page[:, None] * c["hkv"] + heads
    at = (at * (c["page"] // 32) + (pos % c["page"] // 32)[:, None]) * _group_bytes(d)
    r = (pos % 32)[:, None, None]
    ch = torch.arange(0, d, 2, device=DEVICE)
    k = at[..., None] + ch // 32 * 512 + r * 16 + ch % 32 // 2
    pair = torch.arange(d // 2, device=DEVICE)      # channels 32 (pair / 16) + pair % 16 and + 16
    v = at[..., None] + 16 * d + pair // 32 * 1024 + r // 4 % 4 * 256 + pair % 16 * 16 + pair // 16 % 2 * 8 + r // 16 * 4 + r % 4
    ke = at[..., None] + 32 * d + torch.arange(d // 32, device=DEVICE) * 32 + r % 16 * 2 + r // 16
    vs = at[..., None] + 33 * d + (r // 4 % 4 * 8 + r // 16 * 4 + r % 4) * 2 + torch.arange(2, device=DEVICE)
    return k, v, ke, vs


def _value(values, code):
    return values[code.int()]


def _write(c, batch, pages, k, v):
    seq, _, pos = _places(c, batch)
    flat = pages.view(-1)
    at_k, at_v, at_ke, at_vs = _byte_places(c, batch, seq, pos)
    k_codes, exp, v_codes, scale = _quantised(k, v)
    flat[at_k] = k_codes[..., 0::2] | k_codes[..., 1::2] << 4
    v_codes = v_codes.unflatten(-1, (-1, 2, 16))
    flat[at_v] = (v_codes[..., 0, :] | v_codes[..., 1, :] << 4).flatten(-2)
    flat[at_ke] = exp
    flat[at_vs] = scale.contiguous().view(torch.uint8).unflatten(-1, (-1, 2))


def _read(c, batch, pages, values):
    seq, _, pos = _places(c, batch)
    flat = pages.view(-1)
    at_k, at_v, at_ke, at_vs = _byte_places(c, batch, seq, pos)
    codes = flat[at_k]
    k = _value(values, torch.stack([codes & 15, codes >> 4], -1).flatten(-2))
    k = torch.ldexp(k.unflatten(-1, (-1, 32)), flat[at_ke][..., None].int() - 127).flatten(-2)
    codes = flat[at_v].unflatten(-1, (-1, 16))
    v = _value(values, torch.stack([codes & 15, codes >> 4], -2).flatten(-3)) * flat[at_vs].view(torch.bfloat16).float()
    return k.to(_torch_dtype(c)), v.to(_torch_dtype(c))


def _cached(c, batch, pages, values):
    """All rows that the page table lists, in 32 bits: K and V [sequences, heads, rows, d]."""
    d = c["d"]
    n = -(-batch["max_length"] // c["page"])
    g = pages.view(-1, c["hkv"], c["page"] // 32, _group_bytes(d))[batch["page_table"][:, :n].long()]      # [seqs, pages, heads, groups, bytes]
    g = g.transpose(1, 2).flatten(2, 3)      # [seqs, heads, groups, bytes]
    both = lambda x: _value(values, torch.stack([x & 15, x >> 4], -1))  # noqa: E731
    k = both(g[..., :16 * d].unflatten(-1, (d // 32, 32, 16))).flatten(-2)      # [.., block, key, 32]
    exp = g[..., 32 * d:33 * d].unflatten(-1, (d // 32, 16, 2)).transpose(-1, -2).flatten(-2)      # [.., block, key]
    k = torch.ldexp(k, exp[..., None].int() - 127).transpose(-2, -3).flatten(-2).flatten(2, 3)
    v = both(g[..., 16 * d:32 * d].unflatten(-1, (d // 64, 4, 16, 2, 2, 4)))      # [.., c/64, r/4%4, c%16, c/32%2, r/16, r%4, c/16%2]
    lead = v.dim() - 7
    v = v.permute(*range(lead), *(lead + x for x in (4, 1, 5, 0, 3, 6, 2))).flatten(-4).flatten(-4, -2)      # [.., r, c]
    s = g[..., 33 * d:33 * d + 64].contiguous().view(torch.bfloat16).float().unflatten(-1, (4, 2, 4)).transpose(-2, -3).flatten(-3)
    return k, (v * s[..., None]).flatten(2, 3)


def _plain(state):
    c, x = state["case"], state
    out = _torch_dtype(c)
    if c["op"] == "norm":
        def each(y, weight):
            y = y.float()
            if c["norm"]:
                y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6) * weight.float()
            return (_rotated(y, x["positions"], c["base"]) if c["rope"] else y).to(out)
        return [each(x["q"], x["q_weight"]), each(x["k"], x["k_weight"])]
    batch = x["batch"]
    if c["op"] == "append":
        _, _, pos = _places(c, batch)
        _write(c, batch, x["pages"], _rotated(x["k"], pos, c["base"]) if c["rope"] else x["k"].double(), x["v"])
        got = list(_read(c, batch, x["pages"], x["values"]))
        return got + [_rotated(x["q"], pos, c["base"]).to(out)] if c["rope"] else got
    seq, i, _ = _places(c, batch)
    k, v = _cached(c, batch, x["pages"], x["values"])
    n, g = batch["max_new"], c["hq"] // c["hkv"]
    q = torch.zeros((c["seqs"], n, c["hq"], c["d"]), device=DEVICE)
    q[seq, i] = x["q"].float()
    q = q.view(c["seqs"], n, c["hkv"], g, c["d"]).transpose(1, 2).reshape(c["seqs"], c["hkv"], n * g, c["d"])
    s = torch.matmul(q, k.transpose(-1, -2)).mul_(1.0 / math.sqrt(c["d"])).view(c["seqs"], c["hkv"], n, g, -1)
    j = torch.arange(k.shape[2], device=DEVICE)
    pos = (batch["lengths"].long()[:, None] + torch.arange(n, device=DEVICE))[..., None]      # [seqs, n, 1]
    hidden = j > pos if not c["window"] else (j > pos) | (j <= pos - c["window"])
    s.masked_fill_(hidden[:, None, :, None], -math.inf)
    s -= s.amax(-1, keepdim=True)
    s.exp_()
    s /= s.sum(-1, keepdim=True)
    o = torch.matmul(s.view(c["seqs"], c["hkv"], n * g, -1), v).view(c["seqs"], c["hkv"], n, g, c["d"])
    return o.transpose(1, 2)[seq, i].flatten(1, 2).to(out)


# ---------------------------------------------------------------- inputs

def prepare(case, seed):
    c = dict(BASE, **case)
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32)

    def tokens(n):
        """Queries, keys and values of n tokens: views of one projection's output, or arrays of their own.  Some key channels are large."""
        hq, hkv, d = c["hq"], c["hkv"], c["d"]
        x = normal(n, hq + 2 * hkv, d)
        x[:, hq:hq + hkv] *= (0.5 * normal(hkv, d)).exp()
        x = x.to(_torch_dtype(c))
        q, k, v = x.split([hq, hkv, hkv], 1)
        return (q, k, v) if c["fused"] else (q.contiguous(), k.contiguous(), v.contiguous())

    state = {"case": c}
    if c["op"] == "norm":
        state["q"], state["k"], _ = tokens(c["new"])
        state["q_weight"], state["k_weight"] = (1.0 + 0.2 * normal(2, c["d"])).to(_torch_dtype(c))
        state["positions"] = torch.arange(c["context"], c["context"] + c["new"], device=DEVICE, dtype=torch.int32)
        if own:
            from paper_2406_17808_amd import paged
            state["rope_table"] = paged.RopeTable(ROPE_POSITIONS, c["d"], c["base"], DEVICE) if c["rope"] else None
        return state

    have, new = _lengths(c)
    total = [h + n for h, n in zip(have, new)]
    pages = [-(-x // c["page"]) for x in total]
    # pages of the sequences in the order in which a pool hands them out after a while: any
    order = torch.randperm(sum(pages) + 3, generator=gen, device=DEVICE)
    table = torch.zeros((c["seqs"], max(pages)), device=DEVICE, dtype=torch.int32)
    first = 0
    for s, n in enumerate(pages):
        table[s, :n] = order[first:first + n]
        first += n
    i32 = lambda x: torch.tensor(x, device=DEVICE, dtype=torch.int32)  # noqa: E731
    offsets = [0]
    for n in new:
        offsets.append(offsets[-1] + n)
    batch = {"lengths": i32(have), "new_offsets": i32(offsets), "page_table": table, "n_tokens": offsets[-1], "max_new": max(new),
             "max_length": max(total)}
    state["batch"] = batch
    state["pages"] = torch.zeros((sum(pages) + 3, c["hkv"] * (c["page"] // 32) * _group_bytes(c["d"])), device=DEVICE, dtype=torch.uint8)
    state["values"] = torch.tensor(VALUES + [-x for x in VALUES], device=DEVICE)
    state["q"], state["k"], state["v"] = tokens(offsets[-1])
    if c["op"] == "attend":      # the cache as appending left it, sequence by sequence
        for s in range(c["seqs"]):
            for a in range(0, total[s], 16384):
                n = min(16384, total[s] - a)
                one = {"lengths": i32([a]), "new_offsets": i32([0, n]), "page_table": table[s:s + 1], "n_tokens": n}
                _, k, v = tokens(n)
                _write(c, one, state["pages"], k.float(), v.float())
    if own:      # the handles that a program keeps from step to step
        from paper_2406_17808_amd import binding as B
        from paper_2406_17808_amd import paged
        cfg = B.make_paged_config(n_q_heads=c["hq"], n_kv_heads=c["hkv"], head_dim=c["d"],
                                  dtype=B.CASCADE_BF16 if c["dtype"] == "bf16" else B.CASCADE_F32, page_size=c["page"],
                                  n_pages=state["pages"].shape[0], max_seqs=c["seqs"], window=c["window"])
        rope = paged.RopeTable(ROPE_POSITIONS, c["d"], c["base"], DEVICE) if c["rope"] and c["op"] == "append" else None
        state["cache"] = paged.PagedKVCache(cfg, DEVICE, pages=state["pages"], rope=rope)
        state["paged_batch"] = paged.PagedBatch(**batch)
    return state


def run(state):
    if not own:
        return _plain(state)
    c = state["case"]
    if c["op"] == "norm":
        from paper_2406_17808_amd import paged
        return list(paged.qk_norm_rope(state["q"], state["k"], state["q_weight"] if c["norm"] else None, state["k_weight"] if c["norm"] else None,
                                       eps=1e-6, norm=c["norm"], positions=state["positions"] if c["rope"] else None, rope=state["rope_table"]))
    cache, batch = state["cache"], state["paged_batch"]
    if c["op"] == "append":
        q = cache.append(batch, state["k"], state["v"], q=state["q"] if c["rope"] else None)
        got = list(cache.read(batch))
        return got + [q] if c["rope"] else got
    return cache.attend(batch, state["q"])


# ---------------------------------------------------------------- the definition in 64 bits

def _turn(x, positions, base):
    """Pairs as complex numbers times exp(i angle)."""
    half = x.shape[-1] // 2
    freq = torch.tensor([math.pow(base, -i / half) for i in range(half)], device=x.device, dtype=torch.float64)
    z = torch.complex(x[..., :half].double(), x[..., half:].double())
    turned = z * torch.polar(torch.ones((), device=x.device, dtype=torch.float64), positions.double()[:, None, None] * freq)
    return torch.cat([turned.real, turned.imag], -1)


def _nearest(y):
    """y rounded to the eight magnitudes: spacing 1/2 up to 2, 1 up to 4, 2 up to 6; torch.round takes ties to even multiples, which are
    the even codes."""
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0)).double()
    return torch.sign(y) * (torch.round(a / step) * step).clamp(max=6.0)


def exact(case, seed):
    c = dict(BASE, **case)
    x = prepare(dict(case), seed)
    if c["op"] == "norm":
        got = []
        for y, w in ((x["q"], x["q_weight"]), (x["k"], x["k_weight"])):
            y = y.double()
            if c["norm"]:
                y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / c["d"] + 1e-6) * w.double()
            got.append(_turn(y, x["positions"], c["base"]) if c["rope"] else y)
        return got
    batch = x["batch"]
    have, offsets = batch["lengths"].tolist(), batch["new_offsets"].tolist()
    if c["op"] == "append":
        pos = torch.cat([torch.arange(h, h + b - a) for h, a, b in zip(have, offsets, offsets[1:])]).to(DEVICE)
        k = (_turn(x["k"], pos, c["base"]) if c["rope"] else x["k"].double()).unflatten(-1, (-1, 32))
        top = k.abs().amax(-1, keepdim=True)
        scale = torch.exp2(torch.ceil(torch.log2(top / 7.0)))
        scale = torch.where(top > 7.0 * scale, 2 * scale, torch.where(top <= 3.5 * scale, scale / 2, scale))      # log2 near a whole number
        scale = torch.where(top > 0, scale, torch.ones_like(scale))
        v = x["v"].double()
        step = (x["v"].float().abs().amax(-1, keepdim=True) / 6.0).bfloat16().double()
        got = [(_nearest(k / scale) * scale).flatten(-2), _nearest(v / torch.where(step > 0, step, torch.ones_like(step))) * step]
        return got + [_turn(x["q"], pos, c["base"])] if c["rope"] else got
    d, g, page, size = c["d"], c["hq"] // c["hkv"], c["page"], _group_bytes(c["d"])
    raw = x["pages"].view(-1, c["hkv"], page // 32, size)
    values = torch.tensor(VALUES + [-y for y in VALUES], device=DEVICE, dtype=torch.float64)
    r, ch = torch.arange(32, device=DEVICE)[:, None], torch.arange(d, device=DEVICE)[None]
    k_byte = torch.div(ch, 32, rounding_mode="floor") * 512 + r * 16 + torch.div(ch % 32, 2, rounding_mode="floor")
    v_byte = 16 * d + ch // 64 * 1024 + (r // 4) % 4 * 256 + ch % 16 * 16 + (ch // 32) % 2 * 8 + r // 16 * 4 + r % 4
    e_byte = 32 * d + ch // 32 * 32 + r % 16 * 2 + r // 16
    s_byte = 33 * d + 2 * ((r // 4) % 4 * 8 + r // 16 * 4 + r % 4)
    out = torch.empty(x["q"].shape, device=DEVICE, dtype=torch.float64)
    for s in range(c["seqs"]):
        a, b = offsets[s], offsets[s + 1]
        n = have[s] + b - a
        if a == b:
            continue
        pages = x["batch"]["page_table"][s, :-(-n // page)].long()
        see = torch.arange(have[s], n, device=DEVICE)[:, None] - torch.arange(n, device=DEVICE)[None]      # how far back a key lies
        hidden = (see < 0) | (see >= c["window"]) if c["window"] else see < 0
        for h in range(c["hkv"]):
            one = raw[pages, h].reshape(-1, size)      # [groups, bytes]
            k = values[((one[:, k_byte] >> (4 * (ch % 2))) & 15).long()] * torch.exp2(one[:, e_byte].double() - 127)
            v = values[((one[:, v_byte] >> (4 * ((ch // 16) % 2))) & 15).long()]
            v = v * (((one[:, s_byte + 1].int() << 24) | (one[:, s_byte].int() << 16)).view(torch.float32).double())
            k, v = k.reshape(-1, d)[:n], v.reshape(-1, d)[:n]
            for i in range(g):
                p = (x["q"][a:b, h * g + i].double() @ k.T) / math.sqrt(d)
                out[a:b, h * g + i] = torch.softmax(p.masked_fill_(hidden, -math.inf), -1) @ v
    return out
