"""What surrounds the products and attention of a serving step, as cases that can be timed and checked.

  norm    the residual's addition and a root-mean-square norm, which give a product its input, in fp16 or in 8 bits with scales
  adapt   low-rank adapters of many requests at once, beside a product whose weights they share
  place   where a step's tokens stand: rows, positions and pages of every sequence from its lengths, pages taken from
          the free ones and given back

A case is one pass through one of them.  With `own` false it is computed in its plain form; with `own` true by the
library's calls.
"""
import math

import torch

own = False

EPS = 1e-5


def listed():
    return [
        # one token of a decode step: a row of the largest layer here, all latency
        _norm("norm_one", 1, 12288),
        # a prompt through that layer
        _norm("norm_prompt", 4096, 12288),
        # 8 bits, a scale for every 128 channels, a residual stream in fp32, a token count that nothing divides
        _norm("norm_8_f32", 509, 8192, stream_f32=True, group=128),
        # an odd number of channels in rows apart from one another, a product's fp32 outputs
        _norm("norm_odd", 77, 5003, x_f32=True, stream_f32=True, gap=21),
        # one token, one adapter beside a query/key/value product
        _adapt("adapt_one", 1, 15360, 5120, 4, 16),
        # a full batch of tokens, every one with an adapter of its own, beside the widest product but one
        _adapt("adapt_step", 32, 36864, 12288, 64, 16, spread="each"),
        # a step of several sequences with drafted tokens, some without adapter, ranks of all kinds, fp32 results
        _adapt("adapt_mixed", 21, 22016, 8192, 6, 64, spread="some", mixed=True, seqs=7, f32=True),
        # prompts of three requests at once
        _adapt("adapt_prompt", 4096, 12288, 5120, 3, 64, spread="some", mixed=True, seqs=3),
        # one new token of each of sixteen sequences
        _place("place_step", 16, 1, 1500, 64),
        # drafted trees of many sequences, some of them idle, small pages
        _place("place_trees", 1000, 8, 700, 32, idle=True),
        # prompts of uneven length, more of them than there are pages for
        _place("place_short", 300, 500, 0, 64, ragged=True, room=0.6),
        # long prompts behind long pasts
        _place("place_prompts", 96, 8192, 5000, 64, ragged=True),
    ]


def _norm(name, tokens, n, x_f32=False, stream_f32=False, group=0, gap=0):
    """group 0: fp16 out; else 8 bits with a scale for every `group` channels; rows of n + gap values."""
    c = {"name": name} if name else {}
    c.update(op="norm", tokens=tokens, n=n, x_f32=x_f32, stream_f32=stream_f32, group=group, gap=gap)
    return c


def _adapt(name, tokens, m, n, count, rank, spread="one", mixed=False, seqs=0, f32=False):
    """`count` adapters of up to `rank` beside an m x n product; seqs: tokens belong to so many sequences, which have adapters."""
    c = {"name": name} if name else {}
    c.update(op="adapt", tokens=tokens, m=m, n=n, count=count, rank=rank, spread=spread, mixed=mixed, seqs=seqs, f32=f32)
    return c


def _place(name, seqs, fresh, past, page, ragged=False, idle=False, room=1.5):
    """`fresh` new tokens of each of `seqs` sequences behind about `past`; room: free pages over those needed."""
    c = {"name": name} if name else {}
    c.update(op="place", seqs=seqs, fresh=fresh, past=past, page=page, ragged=ragged, idle=idle, room=room)
    return c


# ---- drawn cases -----------------------------------------------------------------------------------

def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choices(["norm", "adapt", "place"], [3, 4, 3])[0]
        if op == "norm":
            n = _log_uniform(rng, 64, 16384)
            group = rng.choice([0, 0, 32, 64, 128, 256, -1])
            if group:
                n = max(n // 256, 1) * 256
            elif rng.random() < 0.6:
                n = (n + 7) // 8 * 8
            c = _norm(None, _log_uniform(rng, 1, 4096), n, rng.random() < 0.3, rng.random() < 0.4, n if group < 0 else group,
                      rng.choice([0, 0, 8, 1024, 3]))
            most = work(_norm(None, 4096, 12288))
        elif op == "adapt":
            rank = rng.choice([8, 16, 16, 24, 32, 64, 64, 128])
            tokens = _log_uniform(rng, 1, 4096)
            c = _adapt(None, tokens, _log_uniform(rng, 256, 49152), _log_uniform(rng, 32, 6144) * 8,
                       _log_uniform(rng, 1, 64), rank, rng.choice(["one", "some", "each"]), rng.random() < 0.5,
                       rng.choice([0, 0, rng.randint(1, tokens)]), rng.random() < 0.3)
            if c["count"] * rank * (c["m"] + c["n"]) > 64 * 16 * (36864 + 12288):
                continue
            most = work(_adapt(None, 4096, 12288, 5120, 3, 64, seqs=3))
        else:
            c = _place(None, _log_uniform(rng, 1, 4096), _log_uniform(rng, 1, 8192), rng.choice([0, 1, 63, 700, 5000]),
                       rng.choice([64, 32, 96, 128, 256]), rng.random() < 0.6, rng.random() < 0.3, rng.choice([1.5, 1.1, 0.6]))
            if c["seqs"] * (c["past"] + c["fresh"]) > 1 << 24:
                continue
            most = work(_place(None, 96, 8192, 5000, 64))
        if all(work(c)[k] <= most[k] for k in most):
            return c


# ---- inputs ----------------------------------------------------------------------------------------

def _generator(seed, k):
    gen = torch.Generator(device="cuda")
    gen.manual_seed((seed * 1000003 + 7919 * k + 31) % (1 << 62))
    return gen


def _type(f32):
    return torch.float32 if f32 else torch.float16


def prepare(case, seed):
    return {"norm": _prepare_norm, "adapt": _prepare_adapt, "place": _prepare_place}[case["op"]](case, _generator(seed, 0))


def _prepare_norm(case, gen):
    tokens, n, row = case["tokens"], case["n"], case["n"] + case["gap"]
    # a residual stream has a few channels many times louder than the others
    loud = torch.ones(row, device="cuda")
    loud[torch.randint(0, n, (3,), device="cuda", generator=gen)] = 20.0
    stream = torch.randn((tokens, row), device="cuda", generator=gen).mul_(2 * loud).to(_type(case["stream_f32"]))
    x = torch.randn((tokens, row), device="cuda", generator=gen).to(_type(case["x_f32"]))
    weight = (1 + 0.2 * torch.randn(n, device="cuda", generator=gen)).half()
    s = {"case": case, "x": x, "residual": stream, "weight": weight, "sum": torch.empty((tokens, row), dtype=stream.dtype, device="cuda")}
    if case["group"]:
        s["codes"] = torch.empty((tokens, n // case["group"], case["group"]), dtype=torch.int8, device="cuda")
        s["scales"] = torch.empty((tokens, n // case["group"]), device="cuda")
        s["values"] = torch.empty((tokens, n // case["group"], case["group"]), dtype=torch.float16, device="cuda")
    else:
        s["y"] = torch.empty((tokens, n), dtype=torch.float16, device="cuda")
    return s


def _prepare_adapt(case, gen):
    tokens, m, n, count, rank = (case[k] for k in ("tokens", "m", "n", "count", "rank"))
    down = (torch.randn((count, rank, n), device="cuda", generator=gen) / math.sqrt(n)).half()
    up = (torch.randn((count, m, rank), device="cuda", generator=gen) * (0.5 / math.sqrt(rank))).half()
    ranks = torch.randint(1, rank + 1, (count,), device="cuda", generator=gen, dtype=torch.int32) if case["mixed"] else \
        torch.full((count,), rank, dtype=torch.int32, device="cuda")
    # beyond an adapter's rank its store holds whatever was there before
    beyond = torch.arange(rank, device="cuda") >= ranks[:, None]
    down.masked_fill_(beyond[:, :, None], float("nan"))
    up.masked_fill_(beyond[:, None, :], float("nan"))
    seqs = case["seqs"] or tokens
    of = torch.randint(0, count, (seqs,), device="cuda", generator=gen, dtype=torch.int32)
    if case["spread"] == "one":
        of = of[:1].expand(seqs).contiguous()
    elif case["spread"] == "each":
        of = torch.randperm(count, device="cuda", generator=gen).to(torch.int32).repeat(-(-seqs // count))[:seqs].contiguous()
    else:
        of = torch.where(torch.rand(seqs, device="cuda", generator=gen) < 0.25, -1, of).to(torch.int32)
        of[:1].clamp_(min=0)
    owner = None
    if case["seqs"]:      # every sequence's tokens follow one another
        cut = torch.rand((seqs,), device="cuda", generator=gen).add_(0.2).cumsum(0)
        owner = torch.searchsorted(cut / cut[-1], torch.arange(tokens, device="cuda") / tokens, right=True).clamp_(max=seqs - 1).to(torch.int32)
    s = {"case": case, "down": down, "up": up, "ranks": ranks, "of": of, "owner": owner,
         "scales": 0.5 + torch.rand(count, device="cuda", generator=gen),
         "x": torch.randn((tokens, n), device="cuda", generator=gen).half(),
         "base": torch.randn((tokens, m), device="cuda", generator=gen).to(_type(case["f32"])),
         "y": torch.empty((tokens, m), dtype=_type(case["f32"]), device="cuda")}
    if own:      # the handle and the workspace that a program keeps beside these buffers
        import paper_2206_09557_amd as L
        s["adapters"] = L.lutgemm_adapters(down, up, ranks, s["scales"], m, n, count, rank)
        s["ws_bytes"] = L.lutgemm_adapt_workspace_bytes(s["adapters"], tokens)
        s["ws"] = torch.empty(s["ws_bytes"], dtype=torch.uint8, device="cuda")
        L.lutgemm_workspace_init(s["ws"], s["ws_bytes"], torch.cuda.current_stream().cuda_stream)
    return s


def _width(case):
    """Pages of a sequence's row of the table."""
    return -(-(case["past"] + case["fresh"]) // case["page"])


def _prepare_place(case, gen):
    seqs, page, width = case["seqs"], case["page"], _width(case)

    def lengths(most):
        if not case["ragged"]:
            return torch.full((seqs,), most, dtype=torch.int64, device="cuda")
        return torch.ceil(most * (1 - 0.95 * torch.rand(seqs, device="cuda", generator=gen))).long()

    past, fresh = lengths(case["past"]), lengths(case["fresh"])
    if case["idle"]:
        fresh[torch.rand(seqs, device="cuda", generator=gen) < 0.3] = 0
    if not case["ragged"] and case["past"]:      # the same length, but not all at the same place of a page
        past -= torch.randint(0, min(case["past"], page), (seqs,), device="cuda", generator=gen)
    owned = (past + page - 1) // page
    needed = int(((past + fresh + page - 1) // page).sum())
    taken = int(owned.sum())
    pages = seqs * width + 1                     # of the pool; some belong to sequences that take no part in the step
    free = min(pages - taken, int(case["room"] * (needed - taken)) + 1)
    order = torch.randperm(pages, device="cuda", generator=gen).to(torch.int32)
    table = torch.full((seqs, width), -1, dtype=torch.int32, device="cuda")
    table[torch.arange(width, device="cuda") < owned[:, None]] = order[:taken]
    stack = torch.full((pages,), -1, dtype=torch.int32, device="cuda")
    stack[:free] = order[taken:taken + free]
    tokens = seqs * case["fresh"]
    whole = {"dtype": torch.int32, "device": "cuda"}
    s = {"case": case, "past": past.to(torch.int32), "fresh": fresh.to(torch.int32), "owned": owned.to(torch.int32), "table": table,
         "free": stack, "count": torch.full((1,), free, **whole), "pages": pages, "tokens": tokens,
         "first": torch.empty(seqs + 1, **whole), "positions": torch.empty(tokens, **whole), "owner": torch.empty(tokens, **whole),
         "slots": torch.empty(tokens, dtype=torch.int64, device="cuda")}
    if own:
        import paper_2206_09557_amd as L
        s["handle"] = L.lutgemm_kv_pages(s["free"], s["count"], s["owned"], table, s["pages"], page, seqs, width)
    return s


# ---- one pass --------------------------------------------------------------------------------------

def run(s):
    c = s["case"]
    if not own:
        return {"norm": _plain_norm, "adapt": _plain_adapt, "place": _plain_place}[c["op"]](s)
    import paper_2206_09557_amd as L
    stream = torch.cuda.current_stream().cuda_stream
    if c["op"] == "norm":
        row = c["n"] + c["gap"]
        flags = (L.LUTGEMM_Y_F32 if c["x_f32"] else L.LUTGEMM_Y_F16) | (L.LUTGEMM_NORM_STREAM_F32 if c["stream_f32"] else 0)
        out, scales = (s["codes"], s["scales"]) if c["group"] else (s["y"], None)
        L.lutgemm_rms_norm(s["x"], s["residual"], s["weight"], s["sum"], out, scales, c["tokens"], c["n"], c["group"], row, row, c["n"], EPS,
                           flags, stream)
        if c["group"]:      # (what the codes stand for)
            out = torch.mul(s["codes"], s["scales"][:, :, None], out=s["values"]).flatten(1)
        return [s["sum"][:, :c["n"]], out]
    if c["op"] == "adapt":
        L.lutgemm_adapt(s["x"], s["base"], s["adapters"], s["of"], s["owner"], s["y"], c["tokens"], c["seqs"], c["n"], c["m"], c["m"],
                        L.LUTGEMM_Y_F32 if c["f32"] else L.LUTGEMM_Y_F16, s["ws"], s["ws_bytes"], stream)
        return s["y"]
    # a step placed and, as where all of it is refused, its pages given back: the next pass finds what this one found
    L.lutgemm_kv_place(s["handle"], s["past"], s["fresh"], s["tokens"], c["fresh"], s["first"], s["positions"], s["owner"], s["slots"], stream)
    L.lutgemm_kv_trim(s["handle"], s["past"], stream)
    return [s[k] for k in _PLACED]


_PLACED = ("first", "positions", "owner", "slots", "owned", "table", "free", "count")


def _plain_norm(s):
    c, n = s["case"], s["case"]["n"]
    v = s["x"][:, :n].float() + s["residual"][:, :n].float()
    s["sum"][:, :n] = v
    y = v * torch.rsqrt(v.square().mean(-1, keepdim=True) + EPS) * s["weight"].float()
    if c["group"]:
        y = y.unflatten(-1, (-1, c["group"]))
        scale = y.abs().amax(-1, keepdim=True) / torch.full((), 127.0, device="cuda")     # (by a plain number torch would multiply)
        y = (torch.round(y / scale) * scale).flatten(1)
    return [s["sum"][:, :n], y.half()]


def _plain_adapt(s):
    c = s["case"]
    count, rank = c["count"], c["rank"]
    of = s["of"] if s["owner"] is None else s["of"][s["owner"].long()]
    live = torch.arange(rank, device="cuda") < s["ranks"][:, None]
    down = torch.where(live[:, :, None], s["down"], 0).float().flatten(0, 1)
    up = torch.where(live[:, None, :], s["up"], 0).float().transpose(1, 2).reshape(count * rank, c["m"])
    h = torch.matmul(s["x"].float(), down.t().contiguous()).view(-1, count, rank) * s["scales"][:, None]
    h = torch.where((torch.arange(count, device="cuda") == of[:, None])[:, :, None], h, 0)
    return (s["base"].float() + torch.matmul(h.flatten(1), up)).to(s["base"].dtype)


def _plain_place(s):
    c = s["case"]
    page, seqs, width, dummy = c["page"], c["seqs"], s["table"].shape[1], s["table"].shape[0]
    past, fresh, owned, free = (s[k].long() for k in ("past", "fresh", "owned", "count"))
    fits = (fresh > 0) & (fresh <= c["fresh"]) & (past + fresh <= width * page)
    want = torch.where(fits, fresh, 0)
    need = torch.where(fits, ((past + want + page - 1) // page - owned).clamp(min=0), 0)
    served = (want.cumsum(0) <= s["tokens"]) & (need.cumsum(0) <= free)       # (sums do not fall: nobody behind the first who waits)
    want, need = want * served, need * served
    ends, page_ends = want.cumsum(0), need.cumsum(0)
    s["first"][0] = 0
    s["first"][1:] = ends
    # pages, the free ones from the top of the stack down
    k = torch.arange(s["pages"], device="cuda")
    seq = torch.searchsorted(page_ends, k, right=True)
    taken = seq < seqs
    at = seq.clamp(max=seqs - 1)
    table = torch.cat([s["table"], torch.empty_like(s["table"][:1])])
    col = torch.where(taken, owned[at] + k - (page_ends - need)[at], 0)
    table[torch.where(taken, at, dummy), col] = s["free"][(free - 1 - k).clamp(min=0)]
    # rows
    t = torch.arange(s["tokens"], device="cuda")
    seq = torch.searchsorted(ends, t, right=True)
    live = seq < seqs
    at = seq.clamp(max=seqs - 1)
    position = past[at] + t - (ends - want)[at]
    s["positions"].copy_(torch.where(live, position, 0))
    s["owner"].copy_(torch.where(live, at, -1))
    col = torch.where(live, position // page, 0)
    s["slots"].copy_(torch.where(live, table[at, col] * page + position % page, -1))
    owned, free = owned + need, free - page_ends[-1]
    # and back
    keep = (past + page - 1) // page
    back = (owned - keep).clamp(min=0)
    page_ends = back.cumsum(0)
    k = torch.arange(s["pages"], device="cuda")
    seq = torch.searchsorted(page_ends, k, right=True)
    taken = seq < seqs
    at = seq.clamp(max=seqs - 1)
    col = torch.where(taken, keep[at] + k - (page_ends - back)[at], 0)
    number = table[torch.where(taken, at, dummy), col]
    stack = torch.cat([s["free"], torch.empty_like(s["free"][:1])])
    stack[torch.where(taken, free + page_ends[-1] - 1 - k, s["pages"])] = number
    table[torch.where(taken, at, dummy), col] = -1
    s["table"].copy_(table[:-1])
    s["free"].copy_(stack[:-1])
    s["count"].copy_(free + page_ends[-1])
    s["owned"].copy_(owned - back)
    return [s[k] for k in _PLACED]


# ---- what a pass cannot do without, and its result in 64 bits --------------------------------------

def work(case):
    if case["op"] == "norm":
        n = case["tokens"] * case["n"]
        scales = 4 * n // case["group"] if case["group"] else 0
        size = (4 if case["x_f32"] else 2) + 2 * (4 if case["stream_f32"] else 2) + (1 if case["group"] else 2)
        return {"bytes": n * size + scales + 2 * case["n"], "flops": 5 * n}
    if case["op"] == "adapt":
        t, m, n, rank = (case[k] for k in ("tokens", "m", "n", "rank"))
        used = 1 if case["spread"] == "one" else min(case["seqs"] or t, case["count"])
        rank = (rank + 1) / 2 if case["mixed"] else rank
        share = 0.75 if case["spread"] == "some" else 1.0
        return {"bytes": int(2 * used * rank * (m + n) + t * (2 * n * share + 2 * m * (4 if case["f32"] else 2))),
                "flops": int(2 * t * share * rank * (m + n))}
    tokens = case["seqs"] * case["fresh"]
    pages = case["seqs"] * (-(-case["fresh"] // case["page"]))
    return {"bytes": 24 * case["seqs"] + 16 * tokens + 24 * pages, "flops": 8 * (case["seqs"] + tokens + pages)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "place":
        return None      # whole numbers
    if case["op"] == "norm":
        n, g = case["n"], case["group"]
        v = s["x"][:, :n].double() + s["residual"][:, :n].double()
        y = v / ((v * v).sum(1, keepdim=True) / n + EPS).sqrt() * s["weight"].double()
        if g:
            y = y.reshape(-1, n // g, g)
            step = y.abs().max(2, keepdim=True)[0] / 127
            y = ((y / step).round() * step).reshape(-1, n)
        return [v, y]
    y = s["base"].double()
    of = s["of"].tolist()
    of = [of[k] for k in (range(case["tokens"]) if s["owner"] is None else s["owner"].tolist())]
    for a in sorted(set(of)):
        if 0 <= a < case["count"]:
            rows = torch.tensor([t for t, b in enumerate(of) if a == b], device="cuda")
            r = int(s["ranks"][a])
            h = s["x"][rows].double() @ s["down"][a, :r].double().t().contiguous()
            y[rows] += float(s["scales"][a]) * (h @ s["up"][a, :, :r].double().t().contiguous())
    return y
