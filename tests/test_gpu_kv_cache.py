"""GPU parity of lutgemm_kv_write and lutgemm_kv_read: every byte of the pool against the oracle's, which places each value by
itself from the layout's text; what is read back bit for bit; edges of blocks, pages and tables."""
import numpy as np
import pytest

import paper_2206_09557_amd as L

from gpu_util import torch_cuda
from kv_util import Cache, keys_and_values, stream, up

pytestmark = pytest.mark.gpu


def _write(cache, step, k, v, rows=None, heads_row=None):
    row = k.shape[1] if k is not None else v.shape[1]
    L.lutgemm_kv_write(None if k is None else up(k), None if v is None else up(v), None if rows is None else up(np.asarray(rows, np.int32)),
                       cache.c, step, row, row, stream())


def _read(cache, step, tokens):
    torch = torch_cuda()
    row = cache.heads * cache.dim + 8
    out = [torch.full((tokens, row), 77.0, dtype=torch.float16, device="cuda") for _ in range(2)]
    L.lutgemm_kv_read(cache.c, step, out[0], out[1], row, row, stream())
    got = [o.cpu().numpy() for o in out]
    assert all((g[:, cache.heads * cache.dim:] == 77).all() for g in got)
    return [g[:, :cache.heads * cache.dim].reshape(tokens, cache.heads, cache.dim) for g in got]


CASES = [(bits, dim, group) for bits in (4, 8) for dim, group in ((64, 32), (64, 0), (96, 96), (128, 32), (128, 64), (192, 96), (256, 128))] + \
        [(16, dim, 0) for dim in (64, 96, 128, 192, 256)]


@pytest.mark.parametrize("bits,dim,group", CASES)
def test_bytes_and_values(bits, dim, group):
    counts, past, page = [1, 0, 37, 5], [0, 9, 30, 91], 96
    cache = Cache(4, 2, page, 2, dim, bits, group, seed=dim + bits)
    rng = np.random.default_rng(bits * 1000 + dim + group)
    n = sum(counts)
    rows = [np.concatenate([keys_and_values(rng, (n, 2, dim)).reshape(n, -1), np.full((n, 8), np.nan, np.float16)], 1) for _ in range(2)]
    rows[0][3, :dim] = 1.5            # a constant group: s = 0 with an offset, the largest code without
    rows[1][4, :dim] = 0
    rows[0][5, :dim] = np.float16(2.0 ** -24) * (np.arange(dim) % 3)       # scales below fp16's smallest
    rows[1][6, :32] = np.where(np.arange(32) % 2, 65504.0, -65504.0)       # the whole range of the type
    step = cache.step(counts, past)
    print("case write", bits, dim, group, flush=True)
    _write(cache, step, *rows)
    pool = cache.pool()
    want = cache.fill.copy()
    at = 0
    kv = [r[:, :2 * dim].reshape(n, 2, dim) for r in rows]
    for s, c in enumerate(counts):
        for j in range(c):
            for h in range(2):
                for key in (True, False):
                    cache.put(want, s, past[s] + j, h, key, kv[0 if key else 1][at, h])
            at += 1
    np.testing.assert_array_equal(pool, want)       # every byte that is not a new position's is as it was
    got = _read(cache, step, n)
    for g, x in zip(got, kv):
        np.testing.assert_array_equal(g.view(np.uint16) & 0x7fff, cache.rounded(x).view(np.uint16) & 0x7fff)
        same = g != 0
        np.testing.assert_array_equal(g[same], cache.rounded(x)[same])
        if bits < 16:       # no further than half a step, plus what rounding the scale down leaves at the end
            size = np.abs(x.astype(np.float64)).reshape(n, 2, -1, cache.group)
            step_size = (2 * size.max(-1) / (15 if bits == 4 else 254)).repeat(cache.group, -1).reshape(x.shape)
            assert (np.abs(g.astype(np.float64) - x) <= 0.65 * step_size + 2.0 ** -10 * np.abs(x.astype(np.float64)) + 2e-6).all()


@pytest.mark.parametrize("bits", [4, 8])
def test_not_finite(bits):
    cache = Cache(1, 1, 32, 1, 64, bits, 32)
    x = np.ones((3, 64), np.float16) * np.arange(64, dtype=np.float16)
    x[0, 3], x[1, 40], x[2, 63] = np.inf, np.nan, -np.inf
    step = cache.step([3], [0])
    _write(cache, step, x, x)
    for g in _read(cache, step, 3):
        bad = np.array([[True, False], [False, True], [False, True]])
        assert (np.isnan(g.reshape(3, 2, 32)) == bad[..., None]).all()
    cache16 = Cache(1, 1, 32, 1, 64, 16, 0)
    step = cache16.step([3], [0])
    _write(cache16, step, x, x)
    np.testing.assert_array_equal(_read(cache16, step, 3)[0][:, 0].view(np.uint16), x.view(np.uint16))


@pytest.mark.parametrize("bits", [4, 8, 16])
def test_token_by_token_is_the_prompt_at_once(bits):
    rng = np.random.default_rng(3)
    k, v = (keys_and_values(rng, (70, 3, 128)).reshape(70, -1) for _ in range(2))
    whole, single = (Cache(1, 3, 32, 3, 128, bits, 64, seed=1) for _ in range(2))
    _write(whole, whole.step([70], [5]), k, v)
    for t in range(70):
        _write(single, single.step([1], [5 + t]), k[t:t + 1], v[t:t + 1])
    np.testing.assert_array_equal(whole.pool(), single.pool())


@pytest.mark.parametrize("bits", [4, 8, 16])
def test_rows_taken_by_number_and_one_side_alone(bits):
    """The accepted tokens of a drafted tree are written next to each other; a negative row is left out."""
    rng = np.random.default_rng(4)
    k, v = (keys_and_values(rng, (9, 2, 64)).reshape(9, -1) for _ in range(2))
    a, b = (Cache(2, 2, 32, 2, 64, bits, 32, seed=2) for _ in range(2))
    _write(a, a.step([3, 2], [30, 4]), k, v, rows=[7, 0, 2, 8, 8])
    take = [7, 0, 2, 8, 8]
    _write(b, b.step([3, 2], [30, 4]), k[take], None)
    _write(b, b.step([3, 2], [30, 4]), None, v[take])
    np.testing.assert_array_equal(a.pool(), b.pool())
    before = a.pool()
    _write(a, a.step([3], [30]), k, v, rows=[1, -1, 3])
    got = _read(a, a.step([3], [30]), 3)
    np.testing.assert_array_equal(got[0][[0, 2]], a.rounded(k[[1, 3]].reshape(2, 2, 64)))
    np.testing.assert_array_equal(got[1][1], a.rounded(v[0].reshape(2, 64)))
    _write(a, a.step([3], [30]), k, v, rows=[7, 0, 2])
    np.testing.assert_array_equal(a.pool(), before)


@pytest.mark.parametrize("bits", [4, 8, 16])
def test_what_the_device_arrays_say_is_checked(bits):
    """Pages outside the pool, positions beyond the table, rows beyond the tokens: left out, the rest as it should be."""
    cache = Cache(3, 2, 32, 1, 64, bits, 0, seed=5)
    rng = np.random.default_rng(6)
    k = keys_and_values(rng, (40, 64))
    table = cache.table.copy()
    table[0, 1], table[1, 0] = cache.pages, -1
    step = cache.step([10, 8, 20], [28, 30, 55], table)
    want = cache.fill.copy()
    _write(cache, step, k[:38], k[:38])
    for s, j, row in [(0, j, j) for j in range(4)] + [(1, 2 + j, 12 + j) for j in range(6)] + [(2, j, 18 + j) for j in range(9)]:
        for key in (True, False):
            cache.put(want, s, (28, 30, 55)[s] + j, 0, key, k[row])
    np.testing.assert_array_equal(cache.pool(), want)
    got = _read(cache, step, 38)[0][:, 0]
    live = np.zeros(38, bool)
    live[[*range(4), *range(12, 18), *range(18, 27)]] = True
    np.testing.assert_array_equal(got[live], cache.rounded(k[:38][live]))
    assert (got[~live] == 0).all()


def test_offsets_beyond_32_bits():
    """The last page of a pool of more than 4 GiB."""
    torch = torch_cuda()
    heads, dim, page = 8, 128, 256
    pages = (1 << 32) // (2 * 2 * heads * dim * page) + 40
    pool = torch.empty(L.lutgemm_kv_pool_bytes(pages, page, heads, dim, 16), dtype=torch.uint8, device="cuda")
    assert pool.numel() > 1 << 32
    c = L.lutgemm_kv_cache(pool, pages, page, heads, dim, 16)
    t = [torch.tensor(a, dtype=torch.int32, device="cuda") for a in ([0, 5], [3], [pages - 1])]
    step = L.lutgemm_kv_step(*t, 1, 1, 5, 5)
    x = torch.randn(5, heads * dim, device="cuda").half()
    y = torch.zeros_like(x)
    z = torch.zeros_like(x)
    L.lutgemm_kv_write(x, -x, None, c, step, heads * dim, heads * dim, stream())
    L.lutgemm_kv_read(c, step, y, z, heads * dim, heads * dim, stream())
    torch.cuda.synchronize()
    assert (x == y).all() and (z == -x).all()
