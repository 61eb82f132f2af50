"""Every kernel of the attention half, by the plan that takes it: attention's for each width, head size, group and number of rows, with
tokens that see nothing, a page that is not there and what is not finite where nobody looks; the stores that go past the
caches against the ones that do not."""
import numpy as np
import pytest

import paper_2206_09557_amd as L
from oracle import kv_oracle as K

from gpu_util import make_workspace, torch_cuda
from kv_util import Cache, keys_and_values, stream, up
import test_gpu_kv_cache
from test_gpu_attention import _check, _fill, _run, _tree

pytestmark = pytest.mark.gpu

GROUPS = {64: (32, 64), 96: (32, 96), 128: (32, 64, 128), 192: (32, 64, 96, 192), 256: (32, 64, 128, 256)}
CASES = [(bits, dim, group) for dim in GROUPS for bits in (16, 8, 4) for group in (GROUPS[dim] if bits != 16 else (0,))]
# tokens and query heads of a key head, whether the plan is told of a context that is worth all wavefronts of a compute unit
ROWS = [(3, 5, False), (3, 5, True), (5, 5, False), (13, 3, False), (25, 4, False), (50, 4, False)]


def _tiles(rows, dim):
    if rows <= 16:
        return 1
    if rows <= 32 and dim <= 128:
        return 2
    tiles = 8 if dim == 256 else 4
    while tiles < (16 if dim <= 128 else 8) and 16 * tiles < rows:
        tiles *= 2
    return tiles


@pytest.mark.parametrize("bits,dim,group", CASES)
def test_every_kernel(bits, dim, group):
    torch = torch_cuda()
    rng = np.random.default_rng(bits * 1000 + dim + group)
    page, past, columns = 64, 333, 24576
    for tokens, shared, long in ROWS:
        cache = Cache(1, -(-(past + tokens) // page) + 1, page, 1, dim, bits, group, seed=dim)
        cache.d_pool.fill_(255)                # what is not written is NaN
        k, v = _fill(cache, rng, [past], [tokens])[0]
        held = cache.table.shape[1]
        cache.table = np.concatenate([cache.table, np.full((1, columns - held), -1, cache.table.dtype)], 1)
        cache.table[0, 2] = -1                 # positions 128 .. 191 are not there
        seen = np.r_[0:128, 192:past + tokens]
        mask = _tree(rng, [tokens], True)
        step = cache.step([tokens], [past])
        hint = columns * page if long else past + tokens
        q = (1.5 * rng.standard_normal((tokens, shared, dim))).astype(np.float16)
        plan = L.lutgemm_plan_attention(cache.c, step, shared, hint)
        if long:
            assert plan[0] == 1 and plan[4] in (4, 8, 12, 16)
        else:
            assert plan[0] == _tiles(tokens * shared, dim)
        print("case kernel", bits, dim, group, tokens, shared, hint, plan, flush=True)
        nbytes = L.lutgemm_attention_workspace_bytes(cache.c, step, shared, hint)
        ws = make_workspace(nbytes)
        y = torch.empty(tokens, shared * dim, dtype=torch.float16, device="cuda")
        L.lutgemm_attention(up(q.reshape(tokens, -1)), up(mask), cache.c, step, y, shared, shared * dim, shared * dim, dim ** -0.5, hint, ws,
                            nbytes, stream())
        _check(y.cpu().numpy().reshape(tokens, shared, dim), *K.attention(q, k[seen], v[seen], past - 64, mask, dim ** -0.5), dim)


@pytest.mark.parametrize("bits,dim,group,waves", [(16, 64, 0, 12), (4, 64, 64, 16), (8, 128, 128, 8), (4, 128, 32, 8), (8, 192, 64, 8),
                                                  (16, 256, 0, 4)])
def test_all_wavefronts_and_splits(bits, dim, group, waves):
    """A few of 128 splits, of all the wavefronts of a compute unit each."""
    rng = np.random.default_rng(dim)
    page, past, columns = 256, 26001, 6144
    cache = Cache(1, -(-(past + 2) // page), page, 1, dim, bits, group)
    k, v = _fill(cache, rng, [past], [2])[0]
    cache.table = np.concatenate([cache.table, np.full((1, columns - cache.table.shape[1]), -1, cache.table.dtype)], 1)
    step = cache.step([2], [past])
    plan = L.lutgemm_plan_attention(cache.c, step, 5, columns * page)
    assert plan[2] == 128 and plan[3] * 2 < past and plan[4] == waves
    print("case splits", bits, dim, group, plan, flush=True)
    q = (1.5 * rng.standard_normal((2, 5, dim))).astype(np.float16)
    y = _run(cache, step, q, None, 5, dim ** -0.5, columns * page)
    _check(y, *K.attention(q, k, v, past, None, dim ** -0.5), dim)


@pytest.mark.parametrize("dim", sorted(GROUPS))
@pytest.mark.parametrize("tokens,shared,past", [(20, 1, 6001), (25, 4, 1100), (25, 4, 6001), (64, 3, 2500)])
def test_splits_of_many_rows(dim, tokens, shared, past):
    """They are joined by a kernel of their own, several sets of lanes to a row from five splits on."""
    rng = np.random.default_rng(dim + tokens)
    cache = Cache(1, -(-(past + tokens) // 64), 64, 1, dim, 8, 0)
    k, v = _fill(cache, rng, [past], [tokens])[0]
    step, mask = cache.step([tokens], [past]), _tree(rng, [tokens], True)
    plan = L.lutgemm_plan_attention(cache.c, step, shared, past + tokens)
    assert plan[0] > 1 and plan[2] > 1
    print("case joined", dim, tokens, shared, past, plan, flush=True)
    q = (1.5 * rng.standard_normal((tokens, shared, dim))).astype(np.float16)
    y = _run(cache, step, q, mask, shared, dim ** -0.5, past + tokens)
    _check(y, *K.attention(q, k, v, past, mask, dim ** -0.5), dim)


def test_all_wavefronts_of_a_compute_unit():
    """Plans with more than four wavefronts a workgroup are made, with and without splits."""
    found = set()
    cache = L.lutgemm_kv_cache
    for bits, dim, group in CASES:
        for seqs, positions in ((256, 1 << 14), (64, 1 << 16), (1, 1 << 20)):
            c = cache(16, 1, 64, 1, dim, bits, group)
            s = L.lutgemm_kv_step(16, 16, 16, seqs, 1 << 15, seqs, 1)
            plan = L.lutgemm_plan_attention(c, s, 1, positions)
            found.add((plan[4], plan[2] > 1))
    assert {(8, False), (8, True), (12, False), (12, True)} <= found, found


@pytest.mark.parametrize("bits,dim,group", [c for c in CASES if c not in test_gpu_kv_cache.CASES and c[0] != 16])
def test_every_group_is_written_and_read(bits, dim, group):
    test_gpu_kv_cache.test_bytes_and_values(bits, dim, group)


def test_a_long_read_past_the_caches():
    """36 MB of rows at once, and in two parts of less."""
    torch = torch_cuda()
    rng = np.random.default_rng(1)
    tokens, heads, dim = 1100, 64, 128
    row = heads * dim
    cache = Cache(1, 18, 64, heads, dim, 4, 32)
    k, v = (up(keys_and_values(rng, (tokens, row))) for _ in range(2))
    L.lutgemm_kv_write(k, v, None, cache.c, cache.step([tokens], [0]), row, row, stream())
    out = [[torch.full((tokens, row), 7.0, dtype=torch.float16, device="cuda") for _ in range(2)] for _ in range(2)]
    L.lutgemm_kv_read(cache.c, cache.step([tokens], [0]), *out[0], row, row, stream())
    for at, n in ((0, 600), (600, 500)):
        L.lutgemm_kv_read(cache.c, cache.step([n], [at]), out[1][0][at:], out[1][1][at:], row, row, stream())
    for a, b in zip(*out):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("f32", [False, True])
def test_many_rows_turned_past_the_caches(neighbours, f32):
    torch = torch_cuda()
    dt, tokens, heads, dim = (torch.float32, 1100, 60, 128) if f32 else (torch.float16, 2200, 60, 128)
    flags = (L.LUTGEMM_Y_F32 if f32 else L.LUTGEMM_Y_F16) | (L.LUTGEMM_ROPE_NEIGHBOURS if neighbours else 0)
    row = heads * dim
    x = torch.randn(tokens, row, device="cuda", generator=torch.Generator("cuda").manual_seed(2)).to(dt)
    positions = torch.arange(5000, 5000 + tokens, dtype=torch.int32, device="cuda")
    turns = up(L.lutgemm_rope_frequencies(dim))
    whole, parts = torch.empty_like(x), torch.empty_like(x)
    L.lutgemm_rope(x, whole, positions, turns, tokens, heads, dim, dim, row, row, 1.0, flags, stream())
    for at in range(0, tokens, 300):
        n = min(300, tokens - at)
        L.lutgemm_rope(x[at:], parts[at:], positions[at:], turns, n, heads, dim, dim, row, row, 1.0, flags, stream())
    assert torch.equal(whole, parts)
    half = x.clone()                          # in place
    L.lutgemm_rope(half, half, positions, turns, tokens, heads, dim, dim, row, row, 1.0, flags, stream())
    assert torch.equal(whole, half)
