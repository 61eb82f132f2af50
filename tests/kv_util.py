"""Helpers of the cache and attention tests: caches in the oracle's layout, steps, uploads."""
import numpy as np

import paper_2206_09557_amd as L
from oracle import kv_oracle as K

from gpu_util import torch_cuda


class Cache:
    """A pool on the device, a page table that deals its pages out in a shuffled order, lengths per sequence."""

    def __init__(self, seqs, table_pages, page, heads, dim, bits, group, seed=0, spare=2):
        torch = torch_cuda()
        self.page, self.heads, self.dim, self.bits, self.group = page, heads, dim, bits, group or dim
        self.pages = seqs * table_pages + spare
        rng = np.random.default_rng(seed)
        self.table = rng.permutation(self.pages)[:seqs * table_pages].reshape(seqs, table_pages).astype(np.int32)
        n = L.lutgemm_kv_pool_bytes(self.pages, page, heads, dim, bits, group)
        assert n == K.pool_bytes(self.pages, page, heads, dim, bits, self.group)
        self.fill = rng.integers(0, 256, n, dtype=np.uint8)       # what the memory held before
        self.d_pool = torch.from_numpy(self.fill.copy()).cuda()
        self.c = L.lutgemm_kv_cache(self.d_pool, self.pages, page, heads, dim, bits, group)

    def step(self, counts, past, table=None, most=None):
        torch = torch_cuda()
        first = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        table = self.table if table is None else table
        t = [torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda() for a in (first, past, table)]
        return L.lutgemm_kv_step(*t, len(counts), table.shape[1], int(first[-1]), max(counts) if most is None else most)

    def pool(self):
        return self.d_pool.cpu().numpy()

    def put(self, pool, seq, position, head, key, x):
        page = int(self.table[seq, position // self.page])
        K.put(pool, (page, position % self.page, head, self.page, self.heads), key, x, self.bits, self.group)

    def rounded(self, x):
        """What the cache makes of x [..., dim]."""
        return K.values(*K.quantise(x, self.bits, self.group), self.bits, self.group)


def up(x):
    torch = torch_cuda()
    x = np.ascontiguousarray(x)
    return torch.from_numpy(x.view(np.int16) if x.dtype == np.float16 else x.view(np.int64) if x.dtype == np.uint64 else x).cuda()


def stream():
    return torch_cuda().cuda.current_stream().cuda_stream


def keys_and_values(rng, shape):
    """N(0, 1) with two loud channels, fp16."""
    x = rng.standard_normal(shape)
    x[..., rng.integers(0, shape[-1], 2)] *= 8
    return x.astype(np.float16)
