"""The attention half of a decode step, as cases that can be timed and checked: what stands between the
query/key/value product of a decoder layer and its output product.

  rope    rotary positions: every token's query and key heads are turned by angles that grow with its position
  store   a key/value cache of 16, 8 or 4 bits a value: keys and values are quantised as they are written, then read back
  attend  attention of a few new tokens of each sequence over that cache: one token (plain decode), or a tree of
          drafted ones, each of which sees the whole past and its own ancestors

A case is one pass through one of them.  With `own` false it is computed in its plain form, from the quantised
values as they are numbered by (page, position, head, channel); with `own` true by the library's calls, from the
same values in the library's cache layout.
"""
import math

import torch

own = False

UNIT = 32              # positions of a block of the cache layout, channels of a unit


def listed():
    return [
        # the smallest call: one token's heads, 64 of queries and 64 of keys, all latency
        _rope("rope_one", 1, 128, 128),
        # a long prompt far into a context that the model was not trained for; queries share key heads
        _rope("rope_prompt", 4096, 72, 128, scaling="parts", start=100000, gap=8 * 128),
        # half of every head, neighbours paired, gradients in fp32, a token count that nothing divides
        _rope("rope_partial_f32", 509, 40, 128, rot=64, pairs="neighbours", transpose=True, f32=True),
        # one new token of each of sixteen sequences
        _store("store_step_8", 8, 64, 128, 0, seqs=16, tokens=1, past=1500),
        # a prompt into an empty cache, small groups
        _store("store_prompt_4", 4, 64, 128, 32, seqs=1, tokens=4096, past=0),
        # chunks of several sequences that begin and end inside blocks and pages, heads of 96 channels
        _store("store_ragged_8", 8, 10, 96, 96, seqs=5, tokens=173, past=333, ragged=True, page=96),
        # one sequence, a short past, nothing quantised: launch and latency
        _attend("attend_short_16", 16, 40, 40, 128, 0, seqs=1, tokens=1, past=300),
        # sixteen sequences of different lengths, a key head for every query head: the cache's bytes
        _attend("attend_step_8", 8, 64, 64, 128, 0, seqs=16, tokens=1, past=4000, ragged=True),
        # one long sequence, eight query heads to a key head, four bits
        _attend("attend_long_4", 4, 64, 8, 128, 64, seqs=1, tokens=1, past=131071),
        # a tree of as many drafted tokens as a product takes vectors
        _attend("attend_tree_8", 8, 96, 96, 128, 0, seqs=1, tokens=32, past=2048),
        # trees of 64 tokens and shared key heads: 512 rows to a head, matrix work
        _attend("attend_tree_shared_8", 8, 64, 8, 128, 128, seqs=4, tokens=64, past=8192),
        # small trees of uneven size, seven query heads to a key head, empty rows, empty sequences
        _attend("attend_ragged_4", 4, 28, 4, 96, 32, seqs=6, tokens=11, past=700, ragged=True, page=96, empty=True),
    ]


def _rope(name, tokens, heads, dim, rot=0, pairs="halves", scaling="none", start=0, gap=0, transpose=False, f32=False):
    """heads of `dim` channels, the first `rot` of them (0: all) turned; rows of heads * dim + gap values."""
    c = {"name": name} if name else {}
    c.update(op="rope", tokens=tokens, heads=heads, dim=dim, rot=rot or dim, pairs=pairs, scaling=scaling, start=start,
             gap=gap, transpose=transpose, f32=f32)
    return c


def _store(name, bits, heads, dim, group, seqs, tokens, past, ragged=False, page=64):
    """`tokens` new ones of each of `seqs` sequences after about `past` positions; group 0: one scale a head."""
    c = {"name": name} if name else {}
    c.update(op="store", bits=bits, heads=heads, dim=dim, group=group or dim, seqs=seqs, tokens=tokens, past=past,
             ragged=ragged, page=page)
    return c


def _attend(name, bits, q_heads, heads, dim, group, seqs, tokens, past, ragged=False, page=64, empty=False):
    c = _store(name, bits, heads, dim, group, seqs, tokens, past, ragged, page)
    c.update(op="attend", q_heads=q_heads, empty=empty)
    return c


# ---- drawn cases -----------------------------------------------------------------------------------

def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choices(["rope", "store", "attend"], [3, 3, 6])[0]
        dim = rng.choices([128, 64, 96, 192, 256], [8, 3, 2, 1, 1])[0]
        if op == "rope":
            rot = rng.choice([dim, dim, dim // 2, dim // 4])
            c = _rope(None, _log_uniform(rng, 1, 4096), rng.randint(1, 144), dim, rot, rng.choice(["halves", "halves", "neighbours"]),
                      rng.choice(["none", "linear", "base", "parts"]), rng.choice([0, 17, 5000, 900000]), rng.choice([0, 0, 1024, 8, 2]),
                      rng.random() < 0.25, rng.random() < 0.3)
            if c["tokens"] * c["heads"] * dim * (2 if c["f32"] else 1) > 4096 * 72 * 128:
                continue
        else:
            bits = rng.choices([8, 4, 16], [4, 4, 2])[0]
            group = rng.choice([g for g in (32, 64, 96, 128, dim) if dim % g == 0])
            seqs, heads, page = _log_uniform(rng, 1, 32), _log_uniform(rng, 1, 96), rng.choice([64, 32, 96, 128, 256])
            ragged = rng.random() < 0.6
            if op == "store":
                c = _store(None, bits, heads, dim, group, seqs, _log_uniform(rng, 1, 4096), rng.choice([0, 1, 63, 500, 2047]), ragged, page)
                if seqs * c["tokens"] * heads * dim > 4096 * 64 * 128 or seqs * heads * (c["past"] + c["tokens"]) * dim > 1 << 27:
                    continue
            else:
                shared = rng.choice([1, 1, 2, 4, 5, 7, 8, 16])
                tokens = 1 if rng.random() < 0.4 else _log_uniform(rng, 2, 64)
                c = _attend(None, bits, heads * shared, heads, dim, group, seqs, tokens, _log_uniform(rng, 16, 131072), ragged, page,
                            rng.random() < 0.2)
                if heads * shared > 256 or seqs * tokens > 256:
                    continue
                if seqs * heads * (c["past"] + tokens) * dim > 16 * 64 * 4096 * 128 or work(c)["flops"] > 7e10:
                    continue
        if 24 * 128 not in c.values():     # (a size that this repository does not measure)
            return c


# ---- inputs ----------------------------------------------------------------------------------------

def _generator(seed, k):
    gen = torch.Generator(device="cuda")
    gen.manual_seed((seed * 1000003 + 7919 * k + 29) % (1 << 62))
    return gen


def _lengths(case):
    """Per sequence: new tokens, positions before them.  The same for every seed, as they are sizes."""
    gen = torch.Generator()
    gen.manual_seed(case["past"] * 4099 + case["tokens"] * 64 + case["seqs"])
    count, past = [], []
    for s in range(case["seqs"]):
        u, v = torch.rand(2, generator=gen).tolist()
        if not case["ragged"]:
            u, v = 0.0, 0.0
        count.append(case["tokens"] if s == 0 else max(1, round(case["tokens"] * (1 - u))))
        past.append(case["past"] if s == 0 else round(case["past"] * (1 - 0.9 * v)))
        if case.get("empty") and s % 3 == 1:
            past[s] = 0                     # a sequence that begins with this step
        if case.get("empty") and s % 4 == 2:
            count[s] = 0                    # one that takes no part in it
    return count, past


def _channels(case, gen):
    """Values as keys and values have them: N(0, 1), and a few channels of every head several times louder."""
    loud = torch.randint(0, case["dim"], (2,), device="cuda", generator=gen)
    gain = torch.ones(case["dim"], device="cuda")
    gain[loud] = 3 + 4 * torch.rand(2, device="cuda", generator=gen)
    return gain


def _toward_zero(x):
    """Non-negative x to fp16, rounded towards zero."""
    h = x.half()
    return torch.where(h.to(x.dtype) > x, (h.view(torch.int16) - 1).view(torch.float16), h)


def _number(v):
    """A divisor as a tensor (torch multiplies by the rounded reciprocal of a plain number)."""
    return torch.full((), float(v), device="cuda")


def _quantise(x, bits, group):
    """x fp16 [..., dim] -> codes (uint8, or x itself), scales and offsets fp16 [..., dim / group]."""
    if bits == 16:
        return x, None, None
    g = x.float().unflatten(-1, (-1, group))
    if bits == 8:
        scale, offset = _toward_zero(g.abs().amax(-1) / _number(127)), None
        s = scale.float()[..., None]
        code = torch.where(s > 0, torch.round(g / s), torch.zeros_like(g)).clamp(-127, 127) + 128
    else:
        offset = g.amin(-1).half()
        scale = _toward_zero((g.amax(-1) - g.amin(-1)) / _number(15))
        s = scale.float()[..., None]
        code = torch.where(s > 0, torch.round((g - offset.float()[..., None]) / s), torch.zeros_like(g)).clamp(0, 15)
    return code.to(torch.uint8).flatten(-2), scale, offset


def _values(code, scale, offset, bits, group):
    """What the codes stand for, fp16 (one rounding of scale * code + offset)."""
    if bits == 16:
        return code
    u = code.unflatten(-1, (-1, group)).float()
    v = scale.float()[..., None] * (u - 128) if bits == 8 else scale.float()[..., None] * u + offset.float()[..., None]
    return v.half().flatten(-2)


def _cache_sizes(case):
    unit = UNIT * case["dim"] * case["bits"] // 8
    scales = 0 if case["bits"] == 16 else case["dim"] // case["group"] * UNIT * (2 if case["bits"] == 8 else 4)
    return unit, scales


def _pack(k, v, bits):
    """Codes, scales and offsets (or fp16 values) [pages][page][heads][...] -> the library's cache layout:
    bytes [pages][heads][page / 32][keys | their scales | values | their scales]."""
    parts = []
    for which, (code, scale, offset) in (("k", k), ("v", v)):
        pages, page, heads, dim = code.shape
        blocks = page // UNIT
        t = code.view(pages, blocks, UNIT, heads, dim).permute(0, 3, 1, 2, 4)             # [pages][heads][blocks][32][dim]
        if which == "k":      # position 8a + 4j + b, channel 32c + 8g + e
            t = t.reshape(pages, heads, blocks, 4, 2, 4, dim // 32, 4, 8).permute(0, 1, 2, 6, 7, 3, 5, 4, 8)   # c g a b j e
        else:                 # position 8g + e, channel 32c + 16u + r
            t = t.reshape(pages, heads, blocks, 4, 8, dim // 32, 2, 16).permute(0, 1, 2, 5, 3, 7, 6, 4)        # c g r u e
        t = t.reshape(pages, heads, blocks, dim // 32, 64, 2, 8)
        if bits == 16:
            t = t.permute(0, 1, 2, 3, 5, 4, 6).contiguous().view(torch.uint8)
        elif bits == 4 and which == "k":      # channel e in nibble e / 2 + 4 (e % 2)
            n = t[..., [0, 2, 4, 6, 1, 3, 5, 7]]
            t = n[..., 0::2] | (n[..., 1::2] << 4)
        elif bits == 4:                       # a byte holds channels r and 16 + r; positions 0 2 1 3 of each four
            n = t[..., [0, 2, 1, 3, 4, 6, 5, 7]]
            t = n[..., 0, :] | (n[..., 1, :] << 4)
        parts.append(t.reshape(pages, heads, blocks, -1))
        if scale is not None:
            groups = scale.shape[-1]
            both = torch.stack([scale] if offset is None else [scale, offset], -1)        # [pages][page][heads][groups][1 or 2]
            if which == "k":                  # [group][4a + b][j][scale, offset]
                both = both.view(pages, blocks, 4, 2, 4, heads, groups, -1).permute(0, 5, 1, 6, 2, 4, 3, 7)
            else:                             # [group][scale, offset][position]
                both = both.view(pages, blocks, UNIT, heads, groups, -1).permute(0, 3, 1, 4, 5, 2)
            parts.append(both.reshape(pages, heads, blocks, -1).contiguous().view(torch.uint8))
    return torch.cat(parts, -1)


def _tables(case, seed):
    """Every sequence's pages, drawn from the pool in any order; entries beyond its length repeat its first page."""
    count, past = _lengths(case)
    need = [max(1, -(-(c + p) // case["page"])) for c, p in zip(count, past)]
    order = torch.randperm(sum(need), device="cuda", generator=_generator(seed, 1)).to(torch.int32)
    width, at, rows = max(need), 0, []
    for n in need:
        rows.append(torch.cat([order[at:at + n], order[at:at + 1].expand(width - n)]))
        at += n
    return count, past, sum(need), torch.stack(rows).contiguous()


def _tree(case, count, seed):
    """A tree of drafted tokens for each sequence: bit j of a token's word says that it sees token j of its sequence."""
    gen = torch.Generator()
    gen.manual_seed((seed * 31 + 11) % (1 << 62))
    words = []
    for n in count:
        mine = []
        for t in range(n):
            parent = int(torch.randint(max(0, t - 4), t + 1, (1,), generator=gen)) - 1 if t else -1
            mine.append((mine[parent] if parent >= 0 else 0) | 1 << t)
        if case["empty"]:
            mine = [0 if t % 5 == 3 else w for t, w in enumerate(mine)]
        words += mine
    return torch.tensor([w - (1 << 64) if w >> 63 else w for w in words], dtype=torch.int64, device="cuda")


def _frequencies(case):
    """Radians a position of every pair, fp64, on the host."""
    n, base, factor, trained = case["rot"] // 2, 10000.0, 8.0, 8192
    if case["scaling"] == "base" and case["rot"] > 2:
        base *= factor ** (case["rot"] / (case["rot"] - 2))
    f = [base ** (-2.0 * i / case["rot"]) for i in range(n)]
    if case["scaling"] == "linear":
        f = [x / factor for x in f]
    if case["scaling"] == "parts":        # pairs that turn often in the trained length stay, slow ones are stretched
        keep = [min(1.0, max(0.0, (trained * x / (2 * math.pi) - 1.0) / (32.0 - 1.0))) for x in f]
        f = [x * k + x / factor * (1 - k) for x, k in zip(f, keep)]
    return f


def _amplitude(case):
    return 1.2079441541679836 if case["scaling"] == "parts" else 1.0      # 0.1 ln 8 + 1


def prepare(case, seed):
    if case["op"] == "rope":
        gen = _generator(seed, 0)
        row = case["heads"] * case["dim"]
        x = torch.randn((case["tokens"], row + case["gap"]), device="cuda", generator=gen)
        x = x if case["f32"] else x.half()
        turns = [round(f / (2 * math.pi) * 2.0 ** 64) for f in _frequencies(case)]
        step = torch.randint(0, 2, (case["tokens"],), device="cuda", generator=gen)
        return {"case": case, "x": x, "y": torch.empty((case["tokens"], row), dtype=x.dtype, device="cuda"),
                "positions": (case["start"] + step.cumsum(0)).to(torch.int32),
                "turns": torch.tensor(turns, dtype=torch.int64, device="cuda")}   # 2^-64 of a turn a position
    count, past, pages, table = _tables(case, seed)
    heads, dim, page, bits, group = (case[k] for k in ("heads", "dim", "page", "bits", "group"))
    first = [0]
    for c in count:
        first.append(first[-1] + c)
    s = {"case": case, "pages": pages, "table": table, "tokens": first[-1], "most_tokens": max(count),
         "most_positions": max(c + p for c, p in zip(count, past)),
         "first": torch.tensor(first, dtype=torch.int32, device="cuda"), "past": torch.tensor(past, dtype=torch.int32, device="cuda")}
    gen = _generator(seed, 2)
    if case["op"] == "store":             # keys and values in the rows of one product, behind the queries
        s["qkv"] = torch.randn((first[-1], 3 * heads * dim), device="cuda", generator=gen).view(-1, 3 * heads, dim) \
            .mul_(_channels(case, gen)).half().flatten(1)
        s["k"], s["v"] = s["qkv"][:, heads * dim:2 * heads * dim], s["qkv"][:, 2 * heads * dim:]
        s["pool"] = torch.full((pages * heads * (page // UNIT) * 2 * sum(_cache_sizes(case)),), 255, dtype=torch.uint8, device="cuda")
        s["cache"] = [_quantise(torch.zeros((pages, page, heads, dim), dtype=torch.float16, device="cuda"), bits, group) for _ in range(2)]
        s["out"] = [torch.empty((first[-1], heads * dim), dtype=torch.float16, device="cuda") for _ in range(2)]
    else:
        s["cache"], packed = [], []
        for _ in range(2):
            gain, parts = _channels(case, gen), []
            step = max(1, (1 << 26) // (page * heads * dim))
            for a in range(0, pages, step):
                x = torch.randn((min(step, pages - a), page, heads, dim), device="cuda", generator=gen).mul_(gain).half()
                parts.append(_quantise(x, bits, group))
            s["cache"].append([None if p[0] is None else torch.cat(p) for p in zip(*parts)])
        # beyond a sequence's last position its pages hold what was there before: here nothing that is a number
        dead = torch.ones((pages, page), dtype=torch.bool, device="cuda")
        for i, (c, p) in enumerate(zip(count, past)):
            at = torch.arange(c + p, device="cuda")
            dead[table[i, at // page].long(), at % page] = False
        step = max(1, (1 << 27) // (page * heads * dim))
        for a in range(0, pages, step):
            kv = []
            for code, scale, offset in s["cache"]:
                marked = code[a:a + step] if scale is None else scale[a:a + step]
                marked = torch.where(dead[a:a + step, :, None, None], float("nan"), marked).half()
                kv.append((marked, None, None) if scale is None else
                          (code[a:a + step], marked, None if offset is None else offset[a:a + step]))
            packed.append(_pack(*kv, bits).view(-1))
        s["pool"] = torch.cat(packed)
        s["q"] = torch.randn((first[-1], case["q_heads"] * dim), device="cuda", generator=gen).mul_(1.5).half()
        s["mask"] = _tree(case, count, seed)
        s["y"] = torch.empty((first[-1], case["q_heads"] * dim), dtype=torch.float16, device="cuda")
    if own:      # the handles and the workspace that a program keeps beside these buffers
        import paper_2206_09557_amd as L
        s["kv"] = L.lutgemm_kv_cache(s["pool"], pages, page, heads, dim, bits, group)
        s["step"] = L.lutgemm_kv_step(s["first"], s["past"], table, len(count), table.shape[1], first[-1], s["most_tokens"])
        if case["op"] == "attend":
            s["ws_bytes"] = L.lutgemm_attention_workspace_bytes(s["kv"], s["step"], case["q_heads"], s["most_positions"])
            s["ws"] = torch.empty(s["ws_bytes"], dtype=torch.uint8, device="cuda")
            L.lutgemm_workspace_init(s["ws"], s["ws_bytes"], torch.cuda.current_stream().cuda_stream)
    return s


# ---- one pass --------------------------------------------------------------------------------------

def run(s):
    c = s["case"]
    if not own:
        return {"rope": _plain_rope, "store": _plain_store, "attend": _plain_attend}[c["op"]](s)
    import paper_2206_09557_amd as L
    stream = torch.cuda.current_stream().cuda_stream
    if c["op"] == "rope":
        flags = (L.LUTGEMM_Y_F32 if c["f32"] else L.LUTGEMM_Y_F16) | (L.LUTGEMM_ROPE_NEIGHBOURS if c["pairs"] == "neighbours" else 0) | \
                (L.LUTGEMM_ROPE_TRANSPOSE if c["transpose"] else 0)
        row = c["heads"] * c["dim"]
        L.lutgemm_rope(s["x"], s["y"], s["positions"], s["turns"], c["tokens"], c["heads"], c["dim"], c["rot"], row + c["gap"], row,
                       _amplitude(c), flags, stream)
        return s["y"]
    row = c["heads"] * c["dim"]
    if c["op"] == "store":
        L.lutgemm_kv_write(s["k"], s["v"], None, s["kv"], s["step"], 3 * row, 3 * row, stream)
        L.lutgemm_kv_read(s["kv"], s["step"], s["out"][0], s["out"][1], row, row, stream)
        return s["out"]
    row = c["q_heads"] * c["dim"]
    L.lutgemm_attention(s["q"], s["mask"], s["kv"], s["step"], s["y"], c["q_heads"], row, row, c["dim"] ** -0.5, s["most_positions"],
                        s["ws"], s["ws_bytes"], stream)
    return s["y"]


def _plain_rope(s):
    c = s["case"]
    x = s["x"][:, :c["heads"] * c["dim"]].view(c["tokens"], c["heads"], c["dim"]).float()
    # the angle in turns, modulo one, in 64-bit integers: a product in fp32 would lose it at long positions
    turn = (s["positions"].long()[:, None] * s["turns"] >> 32).float() * (2 * math.pi * 2.0 ** -32)
    cos, sin = (_amplitude(c) * f(turn)[:, None] for f in (torch.cos, torch.sin))
    sin = -sin if c["transpose"] else sin
    a, b = _pairs(x, c)
    return _unpair(a * cos - b * sin, a * sin + b * cos, x, c).to(s["x"].dtype).flatten(1)


def _pairs(x, c):
    r = c["rot"]
    return (x[..., 0:r:2], x[..., 1:r:2]) if c["pairs"] == "neighbours" else (x[..., :r // 2], x[..., r // 2:r])


def _unpair(a, b, x, c):
    turned = torch.stack([a, b], -1).flatten(-2) if c["pairs"] == "neighbours" else torch.cat([a, b], -1)
    return torch.cat([turned, x[..., c["rot"]:]], -1)


def _plain_store(s):
    c = s["case"]
    first = s["first"].long()
    count = first[1:] - first[:-1]
    seq = torch.repeat_interleave(count, output_size=s["tokens"])                              # the sequence of every token
    at = s["past"].long()[seq] + torch.arange(s["tokens"], device="cuda") - first[seq]          # its position
    where = (s["table"].long()[seq, at // c["page"]], at % c["page"])
    for x, cache in zip((s["k"], s["v"]), s["cache"]):
        for held, new in zip(cache, _quantise(x.unflatten(-1, (c["heads"], c["dim"])), c["bits"], c["group"])):
            if held is not None:
                held[where] = new
    return [_values(*[None if p is None else p[where] for p in cache], c["bits"], c["group"]).flatten(1) for cache in s["cache"]]


def _plain_attend(s):
    c = s["case"]
    heads, dim, shared = c["heads"], c["dim"], c["q_heads"] // c["heads"]
    first, past, table = s["first"].long(), s["past"].long(), s["table"].long()
    count = first[1:] - first[:-1]
    t = torch.arange(s["most_tokens"], device="cuda")
    row = (first[:-1, None] + t).clamp(max=s["tokens"] - 1)                                    # [seqs][most tokens]
    q = s["q"].view(-1, heads, shared, dim)[row].permute(0, 2, 1, 3, 4).flatten(2, 3).float()  # [seqs][heads][tokens * shared][dim]
    k, v = (_values(*[None if p is None else p[table].flatten(1, 2) for p in kv], c["bits"], c["group"]).permute(0, 2, 1, 3).float().contiguous()
            for kv in s["cache"])                                                              # [seqs][heads][positions][dim]
    at = torch.arange(k.shape[2], device="cuda")
    drafted = at - past[:, None]                                                               # [seqs][positions]
    sees = (s["mask"][row][:, :, None] >> drafted.clamp(0, 63)[:, None]) & 1 == 1
    live = (drafted < 0)[:, None] | ((drafted < count[:, None])[:, None] & sees)               # [seqs][tokens][positions]
    live = live[:, None, :, None].expand(-1, heads, -1, shared, -1).flatten(2, 3)
    score = torch.matmul(q, k.transpose(-1, -2).contiguous()) * dim ** -0.5
    score = torch.where(live, score, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top > -math.inf, top, 0.0))
    total = p.sum(-1, keepdim=True)
    y = torch.matmul(p, v) / torch.where(total > 0, total, 1.0)
    y = y.unflatten(2, (-1, shared)).permute(0, 2, 1, 3, 4).flatten(2)                         # [seqs][tokens][q_heads * dim]
    return y[t < count[:, None]].half()


# ---- what a pass cannot do without, and its result in 64 bits --------------------------------------

def work(case):
    if case["op"] == "rope":
        n = case["tokens"] * case["heads"] * case["dim"]
        return {"bytes": 2 * n * (4 if case["f32"] else 2) + 4 * case["tokens"] + 4 * case["rot"],
                "flops": 3 * case["tokens"] * case["heads"] * case["rot"]}
    count, past = _lengths(case)
    held = 2 * case["heads"] * sum(_cache_sizes(case)) / UNIT      # bytes of one position
    n = sum(count)
    if case["op"] == "store":            # read and write keys and values, write and read the cache
        values = 2 * n * case["heads"] * case["dim"]
        return {"bytes": 2 * (2 * values + n * held), "flops": 6 * values}
    seen = [(c, p + c) for c, p in zip(count, past)]
    return {"bytes": sum(l for c, l in seen if c) * held + n * (4 * case["q_heads"] * case["dim"] + 8),
            "flops": 4 * case["q_heads"] * case["dim"] * sum(c * l for c, l in seen)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        h, d, r = case["heads"], case["dim"], case["rot"]
        x = s["x"].double()[:, :h * d].reshape(-1, h, d)
        y = x.clone()
        angle = s["positions"].double()[:, None] * torch.tensor(_frequencies(case), dtype=torch.float64, device="cuda")
        turn = torch.polar(torch.full_like(angle, _amplitude(case)), -angle if case["transpose"] else angle)[:, None]
        i = torch.arange(r // 2, device="cuda")
        i, j = (2 * i, 2 * i + 1) if case["pairs"] == "neighbours" else (i, i + r // 2)
        z = torch.complex(x[..., i], x[..., j]) * turn
        y[..., i], y[..., j] = z.real, z.imag
        return y.reshape(-1, h * d)
    bits, group, heads, dim = (case[k] for k in ("bits", "group", "heads", "dim"))
    if case["op"] == "store":
        out = []
        for x in (s["k"], s["v"]):
            g = x.double().reshape(-1, heads * dim // group, group)
            if bits == 8:
                scale = _toward_zero(g.abs().amax(2, keepdim=True) / _number(127)).double()
                g = scale * torch.round(g / scale.clamp(min=2.0 ** -24)).clamp(-127, 127)
            elif bits == 4:
                low = g.amin(2, keepdim=True)
                scale = _toward_zero((g.amax(2, keepdim=True) - low) / _number(15)).double()
                g = low + scale * torch.round((g - low) / scale.clamp(min=2.0 ** -24)).clamp(0, 15)
            out.append(g.reshape(-1, heads * dim).half().double())
        return out
    count, past = _lengths(case)
    shared, page = case["q_heads"] // heads, case["page"]
    y = torch.zeros((s["tokens"], heads, shared, dim), dtype=torch.float64, device="cuda")
    q, at = s["q"].double().view(-1, heads, shared, dim), 0
    for i, (n, p) in enumerate(zip(count, past)):
        if n == 0:
            continue
        where = torch.arange(n + p, device="cuda")
        where = (s["table"][i].long()[where // page], where % page)
        see = torch.ones((n, n + p), dtype=torch.bool, device="cuda")
        see[:, p:] = (s["mask"][at:at + n, None] >> torch.arange(n, device="cuda")) & 1 == 1
        for h in range(heads):
            kv = []
            for code, scale, offset in s["cache"]:
                x = code[where[0], where[1], h].double().view(n + p, -1, group if bits < 16 else dim)
                if bits < 16:
                    x = scale[where[0], where[1], h].double()[..., None] * (x - 128 if bits == 8 else x)
                    x = (x if offset is None else x + offset[where[0], where[1], h].double()[..., None]).half().double()
                kv.append(x.reshape(n + p, dim))
            score = (q[at:at + n, h].reshape(n * shared, dim) @ kv[0].t().contiguous() / math.sqrt(dim)).view(n, shared, -1)
            score = score.masked_fill(~see[:, None], -math.inf)
            weight = torch.nan_to_num(torch.softmax(score, -1), nan=0.0)
            y[at:at + n, h] = (weight.flatten(0, 1) @ kv[1]).view(n, shared, dim)
        at += n
    return y.reshape(-1, case["q_heads"] * dim)
