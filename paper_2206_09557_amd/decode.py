"""The attention half of a decoder layer over a quantised cache: query/key/value product, rotary positions, cache, attention,
output product, all calls of this library.

    python -m paper_2206_09557_amd.decode [--seqs 4 --prompt 200 --steps 64 --kv-bits 8]

fills the cache with prompts, decodes from a captured graph whose lengths advance on the device, then has a tree of drafted
tokens looked at in one step and its accepted branch kept, and prints what a step takes and how far a token decoded by
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

    `place` says where the next step's tokens stand, `run` launches the step (and may be captured), `keep` advances the
    lengths by all of the step's tokens, or by those of a drafted tree that were accepted."""

    def __init__(self, qkv, out, hidden, heads, kv_heads, head_dim, seqs, longest, q=3, g=128, kv_bits=8, kv_group=0, page=64,
                 turns=None, rot_dim=0, neighbours=False, amplitude=1.0):
        import torch
        self.torch, self.weights, self.hidden, self.heads, self.kv_heads, self.dim = torch, (qkv, out), hidden, heads, kv_heads, head_dim
        self.q, self.g, self.seqs = q, g, seqs
        self.row = (heads + 2 * kv_heads) * head_dim
        pages = -(-(longest + MOST_ROWS) // page)
        self.pool = torch.empty(L.lutgemm_kv_pool_bytes(seqs * pages, page, kv_heads, head_dim, kv_bits, kv_group), dtype=torch.uint8,
                                device="cuda")
        self.cache = L.lutgemm_kv_cache(self.pool, seqs * pages, page, kv_heads, head_dim, kv_bits, kv_group)
        self.table = torch.arange(seqs * pages, dtype=torch.int32, device="cuda").view(seqs, pages)
        self.longest = longest
        self.rot_dim, self.amplitude = rot_dim or head_dim, float(amplitude)
        self.rope_flags = L.LUTGEMM_Y_F16 | (L.LUTGEMM_ROPE_NEIGHBOURS if neighbours else 0)
        turns = L.lutgemm_rope_frequencies(self.rot_dim) if turns is None else turns
        if len(turns) * 2 != self.rot_dim:
            raise ValueError(f"{self.rot_dim} channels are turned by {self.rot_dim // 2} frequencies, not {len(turns)}")
        self.turns = torch.from_numpy(turns.view(np.int64)).cuda()
        self.lengths = [0] * seqs
        self.past = torch.zeros(seqs, dtype=torch.int32, device="cuda")
        self.first = torch.zeros(seqs + 1, dtype=torch.int32, device="cuda")
        self.positions = torch.zeros(MOST_ROWS, dtype=torch.int32, device="cuda")
        self.mask = torch.zeros(MOST_ROWS, dtype=torch.int64, device="cuda")
        self.rows = torch.zeros(MOST_ROWS, dtype=torch.int32, device="cuda")
        self.qkv = torch.empty(MOST_ROWS, self.row, dtype=torch.float16, device="cuda")
        self.mixed = torch.empty(MOST_ROWS, heads * head_dim, dtype=torch.float16, device="cuda")
        self.step = L.lutgemm_kv_step(self.first, self.past, self.table, seqs, pages, MOST_ROWS, MOST_ROWS)
        # one workspace for all of it: for every number of tokens, as attention's need does not grow with them (where more rows make another
        # plan there may be fewer splits)
        self.ws_bytes = max([L.lutgemm_workspace_bytes(m, n, q, g, 8, b) for m, n in self.shapes() for b in range(1, MOST_ROWS + 1)] +
                            [L.lutgemm_attention_workspace_bytes(self.cache, self._step(t, t), heads, longest) for t in range(1, MOST_ROWS + 1)])
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
        self.counts = list(counts)
        self._set(self.first, np.concatenate([[0], np.cumsum(counts)]), np.int32)
        self._set(self.past, self.lengths, np.int32)
        below = [np.arange(c) for c in counts] if depths is None else [np.asarray(d) for d in depths]
        self._set(self.positions, np.concatenate([n + b for n, b in zip(self.lengths, below)]), np.int32)
        self.masked = mask is not None
        if self.masked:
            self._set(self.mask, np.array(mask, dtype=np.uint64).view(np.int64), np.int64)
        self.step = self._step(sum(counts), max(counts))

    def _product(self, weights, x, y, m, n, batch):
        bits, alpha, z = weights
        if batch == 1:
            L.lutgemm_gemv(x, bits, alpha, z, y, self.q, self.g, 8, m, n, L.LUTGEMM_Y_F16, self.ws, self.ws_bytes, self._stream())
        else:
            L.lutgemm_gemm(x, bits, alpha, z, y, self.q, self.g, 8, m, n, batch, L.LUTGEMM_Y_F16, self.ws, self.ws_bytes, self._stream())

    def run(self, x, y):
        """x, y: fp16 [tokens][hidden], contiguous.  Five calls on the current stream; nothing is allocated."""
        tokens, stream = self.step.tokens, self._stream()
        for rows in (x, y):
            if rows.shape != (tokens, self.hidden) or rows.dtype != self.torch.float16 or not rows.is_contiguous():
                raise ValueError(f"a step of {tokens} tokens takes and gives contiguous fp16 rows [{tokens}][{self.hidden}]")
        (m, n), (hidden, mixed) = self.shapes()
        queries = self.heads * self.dim
        self._product(self.weights[0], x, self.qkv, m, n, tokens)
        L.lutgemm_rope(self.qkv, self.qkv, self.positions, self.turns, tokens, self.heads + self.kv_heads, self.dim, self.rot_dim,
                       self.row, self.row, self.amplitude, self.rope_flags, stream)
        keys, values = self.qkv[:, queries:], self.qkv[:, queries + self.kv_heads * self.dim:]
        L.lutgemm_kv_write(keys, values, None, self.cache, self.step, self.row, self.row, stream)
        L.lutgemm_attention(self.qkv, self.mask if self.masked else None, self.cache, self.step, self.mixed, self.heads, self.row, mixed,
                            1.0 / math.sqrt(self.dim), self.longest, self.ws, self.ws_bytes, stream)
        self._product(self.weights[1], self.mixed, y, hidden, mixed, tokens)

    def keep(self, accepted=None):
        """The step's tokens become the past; accepted: of each sequence which of its tokens (ascending) do, next to each other."""
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
    args = ap.parse_args(argv)

    import torch

    if not torch.cuda.is_available():
        print("decode: no GPU visible", file=sys.stderr)
        return 2
    if args.seqs < 1 or args.seqs > MOST_ROWS or args.prompt < 1 or args.steps < 1:
        print(f"decode: 1 to {MOST_ROWS} sequences, a prompt and steps", file=sys.stderr)
        return 2
    qkv, out = random_layer(args.hidden, args.heads, args.kv_heads, args.head_dim)
    longest = args.prompt + args.steps + MOST_ROWS + 8

    def layer():
        return AttentionHalf(qkv, out, args.hidden, args.heads, args.kv_heads, args.head_dim, args.seqs, longest, kv_bits=args.kv_bits,
                             kv_group=args.kv_group)

    half = layer()
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

    # Decode: one step captured, lengths and positions advanced within it.
    token, result = torch.randn(args.seqs, args.hidden, device="cuda").half(), torch.empty(args.seqs, args.hidden, dtype=torch.float16, device="cuda")
    half.place([1] * args.seqs)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        half.run(token, result)
        half.past.add_(1)
        half.positions[:args.seqs].add_(1)
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    for _ in range(args.steps):
        graph.replay()
    end.record()
    torch.cuda.synchronize()
    half.lengths = [n + args.steps for n in half.lengths]
    print(f"{args.steps} decode steps of {args.seqs} tokens: {begin.elapsed_time(end) * 1e3 / args.steps:.1f} us a step")

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
