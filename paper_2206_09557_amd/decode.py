"""The attention half of a decoder layer over a quantised cache: norm, query/key/value product, rotary positions, cache, attention,
output product, low-rank adapters beside both products, all calls of this library.

    python -m paper_2206_09557_amd.decode [--seqs 4 --prompt 200 --steps 64 --kv-bits 8 --adapters 3 --rank 16]

fills the cache with prompts, decodes from a captured graph whose tokens are placed and whose pages are taken on the device, then has a
tree of drafted tokens looked at in one step and its accepted branch kept, and prints what a step takes and how far a token decoded by
itself is from the same token in a chunk of its prompt.
"""
from __future__ import annotations

import argparse
import math
import sys

import numpy as np

from . import lutgemm as L

MOST_ROWS = 32      # vectors of one product


class AttentionHalf:
    """One layer: packed weights (bits, alpha, z on the device), its cache, buffers for steps of up to 32 tokens.

    Rotary positions: `turns` (lutgemm_rope_frequencies of rot_dim), on the first rot_dim channels of a head (0: all), neighbours or halves
    paired, times `amplitude` (the one that goes with stretched frequencies).

    norm: fp16 weights [hidden] of a root-mean-square norm in front of the first product, which `run` then takes after adding its
    x to a residual stream.  adapters: lutgemm_adapters beside the first and the second product (either may be None);
    `adapter_of` (int32 [seqs] on the device, -1: none) says whose sequences they are.  pages: of a pool that the sequences share, who take
    them as they grow; 0: each has its own for `longest` positions.

    `place` says where the next step's tokens stand, `run` launches the step (and may be captured), `keep` advances the
    lengths by all of the step's tokens, or by those of a drafted tree that were accepted.  `advance` is a step of one token of every
    sequence with all of that on the device, for a graph to replay (not between a step's `place` and `keep`); `advanced` tells the host
    afterwards what the lengths are, which `place`, `keep` and `end` have to know."""

    def __init__(self, qkv, out, hidden, heads, kv_heads, head_dim, seqs, longest, q=3, g=128, kv_bits=8, kv_group=0, page=64,
                 turns=None, rot_dim=0, neighbours=False, amplitude=1.0, norm=None, eps=1e-5, adapters=(None, None), pages=0):
        import torch
        self.torch, self.weights, self.hidden, self.heads, self.kv_heads, self.dim = torch, (qkv, out), hidden, heads, kv_heads, head_dim
        self.q, self.g, self.seqs = q, g, seqs
        self.row = (heads + 2 * kv_heads) * head_dim
        width = -(-(longest + MOST_ROWS + bool(pages)) // page)        # (one more: `advance`)
        held = pages or seqs * width
        self.pool = torch.empty(L.lutgemm_kv_pool_bytes(held, page, kv_heads, head_dim, kv_bits, kv_group), dtype=torch.uint8,
                                device="cuda")
        self.cache = L.lutgemm_kv_cache(self.pool, held, page, kv_heads, head_dim, kv_bits, kv_group)
        self.page, self.shared = page, bool(pages)
        if self.shared:
            self.table = torch.empty(seqs, width, dtype=torch.int32, device="cuda")
            self.free, self.free_count, self.owned = (torch.empty(n, dtype=torch.int32, device="cuda") for n in (pages, 1, seqs))
            self.pages = L.lutgemm_kv_pages(self.free, self.free_count, self.owned, self.table, pages, page, seqs, width)
            L.lutgemm_kv_pages_init(self.pages, self._stream())
            self.taken, self.left = [0] * seqs, pages          # the host's count of them
            self.fresh = torch.zeros(seqs, dtype=torch.int32, device="cuda")
            # of `advance`: which sequences have as many positions as they may, and what the others and they ask for (nothing where they rest)
            self.full = torch.zeros(seqs, dtype=torch.bool, device="cuda")
            self.asked = torch.zeros(2, seqs, dtype=torch.int32, device="cuda")
            self.resting = [False] * seqs
            self._ask()
        else:
            self.table = torch.arange(seqs * width, dtype=torch.int32, device="cuda").view(seqs, width)
        self.longest = longest
        self.norm, self.eps, self.adapters = norm, float(eps), tuple(adapters)
        for a, (m, n) in zip(self.adapters, self.shapes()):
            if a is not None and (a.m, a.n) != (m, n):
                raise ValueError(f"adapters beside a {m} x {n} product are not {a.m} x {a.n}")
        if norm is not None and (norm.shape != (hidden,) or norm.dtype != torch.float16 or not norm.is_contiguous()):
            raise ValueError(f"a norm has {hidden} fp16 weights")
        self.owner = torch.zeros(MOST_ROWS, dtype=torch.int32, device="cuda")
        self.adapter_of = torch.zeros(seqs, dtype=torch.int32, device="cuda") - 1
        self.normed = torch.empty(MOST_ROWS, hidden, dtype=torch.float16, device="cuda")
        self.rot_dim, self.amplitude = rot_dim or head_dim, float(amplitude)
        self.rope_flags = L.LUTGEMM_Y_F16 | (L.LUTGEMM_ROPE_NEIGHBOURS if neighbours else 0)
        turns = L.lutgemm_rope_frequencies(self.rot_dim) if turns is None else turns
        if len(turns) * 2 != self.rot_dim:
            raise ValueError(f"{self.rot_dim} channels are turned by {self.rot_dim // 2} frequencies, not {len(turns)}")
        self.turns = torch.from_numpy(turns.view(np.int64)).cuda()
        self.lengths = [0] * seqs
        # a step that `keep` has not ended; whether the host knows the lengths; whether there may be a graph that advances them unseen
        self.placed, self.known, self.captured = False, True, False
        self.past = torch.zeros(seqs, dtype=torch.int32, device="cuda")
        self.first = torch.zeros(seqs + 1, dtype=torch.int32, device="cuda")
        self.positions = torch.zeros(MOST_ROWS, dtype=torch.int32, device="cuda")
        self.mask = torch.zeros(MOST_ROWS, dtype=torch.int64, device="cuda")
        self.rows = torch.zeros(MOST_ROWS, dtype=torch.int32, device="cuda")
        self.qkv = torch.empty(MOST_ROWS, self.row, dtype=torch.float16, device="cuda")
        self.mixed = torch.empty(MOST_ROWS, heads * head_dim, dtype=torch.float16, device="cuda")
        self.step = L.lutgemm_kv_step(self.first, self.past, self.table, seqs, width, MOST_ROWS, MOST_ROWS)
        # one workspace for all of it: for every number of tokens, as attention's need does not grow with them (where more rows make another
        # plan there may be fewer splits)
        self.ws_bytes = max([L.lutgemm_workspace_bytes(m, n, q, g, 8, b) for m, n in self.shapes() for b in range(1, MOST_ROWS + 1)] +
                            [L.lutgemm_attention_workspace_bytes(self.cache, self._step(t, t), heads, longest) for t in range(1, MOST_ROWS + 1)] +
                            [L.lutgemm_adapt_workspace_bytes(a, t) for a in self.adapters if a is not None for t in range(1, MOST_ROWS + 1)])
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device="cuda")
        L.lutgemm_workspace_init(self.ws, self.ws_bytes, self._stream())

    def shapes(self):
        return (self.row, self.hidden), (self.hidden, self.heads * self.dim)

    def _stream(self):
        return self.torch.cuda.current_stream().cuda_stream

    def _step(self, tokens, most):
        return L.lutgemm_kv_step(self.first, self.past, self.table, self.seqs, self.table.shape[1], tokens, most)

    def _set(self, tensor, values, kind):
        tensor[:len(values)].copy_(self.torch.from_numpy(np.asarray(values, dtype=kind)))

    def place(self, counts, depths=None, mask=None):
        """counts[s] tokens of sequence s come next; depths: of a tree's tokens below their sequence's last (0 at its roots), mask:
        which of their sequence's new tokens each sees, as bits.  Without them the tokens follow one another."""
        if len(counts) != self.seqs or min(counts) < 0 or sum(counts) < 1 or sum(counts) > MOST_ROWS:
            raise ValueError(f"a step has counts of {self.seqs} sequences and 1 to {MOST_ROWS} tokens")
        if any(n + c > self.longest for n, c in zip(self.lengths, counts)):
            raise ValueError(f"a sequence would be longer than {self.longest}")
        if depths is not None and [len(d) for d in depths] != list(counts):
            raise ValueError("a step has a depth for every token, by sequences")
        if mask is not None and len(mask) != sum(counts):
            raise ValueError("a step has a mask word for every token")
        self._check_known()
        needed = [0] * self.seqs
        if self.shared:
            needed = [max(0, -(-(n + c) // self.page) - t) if c else 0 for n, c, t in zip(self.lengths, counts, self.taken)]
            if sum(needed) > self.left:
                raise ValueError(f"a step needs {sum(needed)} pages more, of {self.left} that are free")
        self.counts, self.placed = list(counts), True
        if not self.shared:                         # (else the device writes it)
            self._set(self.first, np.concatenate([[0], np.cumsum(counts)]), np.int32)
        self._set(self.past, self.lengths, np.int32)
        below = [np.arange(c) for c in counts] if depths is None else [np.asarray(d) for d in depths]
        self._set(self.positions, np.concatenate([n + b for n, b in zip(self.lengths, below)]), np.int32)
        self.masked = mask is not None
        if self.masked:
            self._set(self.mask, np.array(mask, dtype=np.uint64).view(np.int64), np.int64)
        if self.adapters != (None, None):
            self._set(self.owner, np.repeat(np.arange(self.seqs), counts), np.int32)
        self.step = self._step(sum(counts), max(counts))
        if self.shared:
            self._set(self.fresh, counts, np.int32)
            if any(c and r for c, r in zip(counts, self.resting)):
                self.resting = [r and not c for c, r in zip(counts, self.resting)]
                self._ask()
            L.lutgemm_kv_place(self.pages, self.past, self.fresh, sum(counts), max(counts), self.first, None, None, None, self._stream())
            self.taken = [t + n for t, n in zip(self.taken, needed)]
            self.left -= sum(needed)

    def _check_known(self):
        """Nothing of this class runs when a graph is replayed: once there may be one, the device's lengths are looked at, and waited for."""
        if not self.known or self.captured and self.past.tolist() != self.lengths:
            raise ValueError("the lengths have advanced on the device: `advanced` tells them")

    def _product(self, weights, x, y, m, n, batch):
        bits, alpha, z = weights
        if batch == 1:
            L.lutgemm_gemv(x, bits, alpha, z, y, self.q, self.g, 8, m, n, L.LUTGEMM_Y_F16, self.ws, self.ws_bytes, self._stream())
        else:
            L.lutgemm_gemm(x, bits, alpha, z, y, self.q, self.g, 8, m, n, batch, L.LUTGEMM_Y_F16, self.ws, self.ws_bytes, self._stream())

    def _adapt(self, adapters, x, y, tokens):
        if adapters is not None:
            L.lutgemm_adapt(x, y, adapters, self.adapter_of, self.owner, y, tokens, self.seqs, adapters.n, adapters.m, adapters.m, L.LUTGEMM_Y_F16, self.ws,
                            self.ws_bytes, self._stream())

    def run(self, x, y, residual=None):
        """x, y: fp16 [tokens][hidden], contiguous.  residual (with a norm): the stream's rows, fp16 or fp32, to which x is added before its
        norm.  Five to eight calls on the current stream; nothing is allocated."""
        tokens, stream = self.step.tokens, self._stream()
        for rows in (x, y):
            if rows.shape != (tokens, self.hidden) or rows.dtype != self.torch.float16 or not rows.is_contiguous():
                raise ValueError(f"a step of {tokens} tokens takes and gives contiguous fp16 rows [{tokens}][{self.hidden}]")
        if residual is not None and (self.norm is None or residual.shape != (tokens, self.hidden) or not residual.is_contiguous() or
                                     residual.dtype not in (self.torch.float16, self.torch.float32)):
            raise ValueError(f"a residual stream of {tokens} tokens is contiguous fp16 or fp32 rows [{tokens}][{self.hidden}], and a norm's")
        (m, n), (hidden, mixed) = self.shapes()
        queries = self.heads * self.dim
        if self.norm is not None:
            wide = residual is not None and residual.dtype == self.torch.float32
            L.lutgemm_rms_norm(x, residual, self.norm, residual, self.normed, None, tokens, hidden, 0, hidden, hidden, hidden, self.eps,
                               L.LUTGEMM_Y_F16 | (L.LUTGEMM_NORM_STREAM_F32 if wide else 0), stream)
            x = self.normed
        self._product(self.weights[0], x, self.qkv, m, n, tokens)
        self._adapt(self.adapters[0], x, self.qkv, tokens)
        L.lutgemm_rope(self.qkv, self.qkv, self.positions, self.turns, tokens, self.heads + self.kv_heads, self.dim, self.rot_dim,
                       self.row, self.row, self.amplitude, self.rope_flags, stream)
        keys, values = self.qkv[:, queries:], self.qkv[:, queries + self.kv_heads * self.dim:]
        L.lutgemm_kv_write(keys, values, None, self.cache, self.step, self.row, self.row, stream)
        L.lutgemm_attention(self.qkv, self.mask if self.masked else None, self.cache, self.step, self.mixed, self.heads, self.row, mixed,
                            1.0 / math.sqrt(self.dim), self.longest, self.ws, self.ws_bytes, stream)
        self._product(self.weights[1], self.mixed, y, hidden, mixed, tokens)
        self._adapt(self.adapters[1], self.mixed, y, tokens)

    def advance(self, x, y, residual=None):
        """One token of every sequence that does not rest, x [seqs][hidden], their rows one after the other: placed, run, and their lengths
        advanced, all on the device, so that a captured call can be replayed (`rest`, `end` and `place` say whose rows the next replay
        takes).  A sequence that finds no page, or is `longest` positions long, waits, and those behind it (till it rests or ends): their
        rows of y and residual mean nothing, their lengths stay.  The host learns of it by `advanced`."""
        if not self.shared:
            raise ValueError("sequences that advance on the device share their pages")
        if self.seqs > MOST_ROWS or any(n >= self.longest and not r for n, r in zip(self.lengths, self.resting)):
            raise ValueError(f"up to {MOST_ROWS} sequences advance, up to a length of {self.longest}")
        self.masked, self.placed, self.known = False, False, False
        self.captured = self.captured or self.torch.cuda.is_current_stream_capturing()
        self.step = self._step(self.seqs, 1)
        # One of `longest` positions asks for more rows than there are: it waits (a sequence whose table holds no more would be passed over, and
        # those behind it would have one another's rows of x).
        self.torch.ge(self.past, self.longest, out=self.full)
        self.torch.where(self.full, self.asked[1], self.asked[0], out=self.fresh)
        L.lutgemm_kv_place(self.pages, self.past, self.fresh, self.seqs, self.seqs + 1, self.first, self.positions, self.owner, None, self._stream())
        self.run(x, y, residual)
        self.past.add_(self.first[1:] - self.first[:-1])

    def advanced(self):
        """What the device has made of the lengths since the last `place` or `advanced`; waits for it."""
        if not self.shared:
            raise ValueError("sequences that advance on the device share their pages")
        lengths = self.past.tolist()
        if lengths != self.lengths:                 # (a step that was placed before is not what it was)
            self.lengths, self.placed = lengths, False
        self.taken = self.owned.tolist()
        self.left, self.known = int(self.free_count), True
        return self.lengths

    def keep(self, accepted=None):
        """The step's tokens become the past; accepted: of each sequence which of its tokens (ascending) do, next to each other."""
        if not self.placed:
            raise ValueError("a step that `place` has placed is kept, once")
        self._check_known()
        if accepted is None:
            kept = self.counts
        else:
            accepted = [[int(t) for t in a] for a in accepted]
            if len(accepted) != self.seqs or any(a != sorted(set(a) & set(range(c))) for a, c in zip(accepted, self.counts)):
                raise ValueError("of each sequence some of the step's tokens are kept, in ascending order")
            kept = [len(a) for a in accepted]
            if any(a != list(range(len(a))) for a in accepted):
                # the accepted tokens' keys and values, still in the product's rows, over the first of the drafted ones
                begins = np.concatenate([[0], np.cumsum(self.counts)])
                rows = np.concatenate([np.asarray(a, dtype=np.int64) + b for a, b in zip(accepted, begins)])
                self._set(self.rows, rows, np.int32)
                self._set(self.first, np.concatenate([[0], np.cumsum(kept)]), np.int32)
                queries = self.heads * self.dim
                keys, values = self.qkv[:, queries:], self.qkv[:, queries + self.kv_heads * self.dim:]
                L.lutgemm_kv_write(keys, values, self.rows, self.cache, self._step(sum(kept), max(kept)), self.row, self.row, self._stream())
        self.lengths = [n + k for n, k in zip(self.lengths, kept)]
        self.placed = False
        if self.shared:
            self._set(self.past, self.lengths, np.int32)
            self._trim(self.lengths)

    def _trim(self, lengths):
        L.lutgemm_kv_trim(self.pages, self.past, self._stream())
        back = [max(0, t - -(-n // self.page)) for t, n in zip(self.taken, lengths)]
        self.taken = [t - b for t, b in zip(self.taken, back)]
        self.left += sum(back)

    def end(self, seq):
        """Sequence `seq` is over, between two steps: its pages are free, and the next tokens that are placed are a new one's first, which rests
        till then."""
        if self.placed:
            raise ValueError("a sequence ends after `keep`, or after `advanced`")
        self._check_known()
        self.lengths[seq] = 0
        if self.shared:
            self._set(self.past, self.lengths, np.int32)
            self._trim(self.lengths)
            self.rest(seq)

    def rest(self, seq, resting=True):
        """Sequence `seq` has no part in `advance`, captured or not, until `place` brings tokens of it or `resting` is false."""
        if not self.shared:
            raise ValueError("sequences that advance on the device share their pages")
        self.resting[seq] = bool(resting)
        self._ask()

    def _ask(self):
        self.asked.copy_(self.torch.from_numpy(np.array([[0 if r else n for r in self.resting] for n in (1, self.seqs + 1)], dtype=np.int32)))

    def fill(self, x, y):
        """A prompt of every sequence, x [seqs][length][hidden], in chunks; y: their outputs."""
        length = x.shape[1]
        for s in range(self.seqs):
            for at in range(0, length, MOST_ROWS):
                n = min(MOST_ROWS, length - at)
                self.place([n if k == s else 0 for k in range(self.seqs)])
                self.run(x[s, at:at + n], y[s, at:at + n])
                self.keep()


def random_layer(hidden, heads, kv_heads, head_dim, q=3, g=128, seed=0):
    """Packed weights of a layer that keeps activations of N(0, 1) near N(0, 1)."""
    import torch
    rng = np.random.default_rng(seed)
    packed = []
    for m, n in (((heads + 2 * kv_heads) * head_dim, hidden), (hidden, heads * head_dim)):
        w = (rng.standard_normal((m, n), dtype=np.float32) / math.sqrt(n)).astype(np.float16)
        bits, alpha, z = L.lutgemm_pack_bcq(w, q, g)
        packed.append((torch.from_numpy(bits).cuda(), torch.from_numpy(alpha.view(np.int16)).cuda(),
                       None if z is None else torch.from_numpy(z.view(np.int16)).cuda()))
    return packed


def random_adapters(m, n, count, rank, seed=0):
    """Low-rank adapters beside an m x n product, of about a tenth of its outputs."""
    import torch
    rng = np.random.default_rng(seed)
    down = torch.from_numpy((rng.standard_normal((count, rank, n)) / math.sqrt(n)).astype(np.float16)).cuda()
    up = torch.from_numpy((0.1 * rng.standard_normal((count, m, rank)) / math.sqrt(rank)).astype(np.float16)).cuda()
    return L.lutgemm_adapters(down, up, None, None, m, n, count, rank)


def main(argv=None):
    ap = argparse.ArgumentParser(description="decode with one layer's attention half")
    ap.add_argument("--hidden", type=int, default=5120)
    ap.add_argument("--heads", type=int, default=40)
    ap.add_argument("--kv-heads", type=int, default=40)
    ap.add_argument("--head-dim", type=int, default=128)
    ap.add_argument("--seqs", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=200)
    ap.add_argument("--steps", type=int, default=64)
    ap.add_argument("--kv-bits", type=int, choices=[4, 8, 16], default=8)
    ap.add_argument("--kv-group", type=int, default=0)
    ap.add_argument("--adapters", type=int, default=3, help="low-rank adapters that the sequences have in turn; 0: none")
    ap.add_argument("--rank", type=int, default=16, help="their rank, a multiple of 8")
    args = ap.parse_args(argv)

    import torch

    if not torch.cuda.is_available():
        print("decode: no GPU visible", file=sys.stderr)
        return 2
    if args.seqs < 1 or args.seqs > MOST_ROWS or args.prompt < 1 or args.steps < 1:
        print(f"decode: 1 to {MOST_ROWS} sequences, a prompt and steps", file=sys.stderr)
        return 2
    qkv, out = random_layer(args.hidden, args.heads, args.kv_heads, args.head_dim)
    longest, page = args.prompt + args.steps + MOST_ROWS + 8, 64
    norm = (1 + 0.1 * torch.randn(args.hidden, device="cuda")).half()
    shapes = ((args.heads + 2 * args.kv_heads) * args.head_dim, args.hidden), (args.hidden, args.heads * args.head_dim)
    adapters = [random_adapters(m, n, args.adapters, args.rank, seed=k) if args.adapters else None for k, (m, n) in enumerate(shapes)]
    # (pages for every sequence's prompt and steps, and for one's drafted tree)
    pages = args.seqs * -(-(args.prompt + args.steps) // page) + -(-MOST_ROWS // page)
    half = AttentionHalf(qkv, out, args.hidden, args.heads, args.kv_heads, args.head_dim, args.seqs, longest, kv_bits=args.kv_bits, kv_group=args.kv_group,
                         page=page, norm=norm, adapters=adapters, pages=pages)
    if args.adapters:
        half.adapter_of.copy_(torch.arange(args.seqs) % args.adapters)
    x = torch.randn(args.seqs, args.prompt, args.hidden, device="cuda").half()
    y = torch.empty_like(x)
    half.fill(x, y)

    # The prompt's last token once more, by itself.
    alone = torch.empty(args.seqs, args.hidden, dtype=torch.float16, device="cuda")
    half.lengths = [args.prompt - 1] * args.seqs
    half.place([1] * args.seqs)
    half.run(x[:, -1].contiguous(), alone)
    half.keep()
    apart = ((alone - y[:, -1]).float().norm() / y[:, -1].float().norm()).item()
    print(f"{args.seqs} prompts of {args.prompt}: the last token by itself and in its chunk differ by {apart:.1e} of their norm")

    # Decode: one step captured; its tokens are placed, its pages taken and its lengths advanced within it.
    token, result = torch.randn(args.seqs, args.hidden, device="cuda").half(), torch.empty(args.seqs, args.hidden, dtype=torch.float16, device="cuda")
    stream = torch.zeros(args.seqs, args.hidden, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        half.advance(token, result, stream)
    half._set(half.past, half.lengths, np.int32)
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    for _ in range(args.steps):
        graph.replay()
    end.record()
    torch.cuda.synchronize()
    half.advanced()
    print(f"{args.steps} decode steps of {args.seqs} tokens: {begin.elapsed_time(end) * 1e3 / args.steps:.1f} us a step, {half.left} of {pages} pages left")

    # A drafted tree for the first sequence: two roots, the second with two children; the branch 1, 3 is accepted.
    depths, seen, branch = [0, 0, 1, 1], [0b0001, 0b0010, 0b0110, 0b1010], [1, 3]
    none = [[] for _ in range(args.seqs - 1)]
    half.place([4] + [0] * (args.seqs - 1), [depths] + none, seen)
    drafted = torch.randn(4, args.hidden, device="cuda").half()
    looked = torch.empty_like(drafted)
    half.run(drafted, looked)
    half.keep([branch] + none)
    torch.cuda.synchronize()
    print(f"a tree of 4 drafted tokens: {len(branch)} kept, lengths now {half.lengths}, outputs finite: {bool(torch.isfinite(looked).all())}")
    return 0


if __name__ == "__main__":
    sys.exit(main())
