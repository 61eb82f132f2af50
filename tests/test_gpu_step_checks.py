"""GPU checks of what the kernels make of a step whose device arrays hold nonsense: left out, and nothing else disturbed."""
import numpy as np
import pytest

import paper_2206_09557_amd as L
from oracle import kv_oracle as K

from gpu_util import torch_cuda
from kv_util import Cache, keys_and_values, stream, up
from test_gpu_attention import _check, _fill, _run

pytestmark = pytest.mark.gpu

LEAST = -(1 << 31)


def _with_first(step, first):
    """The step with other first rows."""
    d_first = up(np.asarray(first, np.int32))
    return L.lutgemm_kv_step(d_first, step._held[1], step._held[2], step.seqs, step.table_pages, step.tokens, step.most_tokens)


@pytest.mark.parametrize("end", [LEAST, LEAST + 2, -1, 2])
@pytest.mark.parametrize("bits", [4, 8, 16])
def test_rows_that_end_before_they_begin_are_not_moved(bits, end):
    """Sequence 0's rows are 3 up to `end`: none, however far below.  Sequence 1's begin where those end, cut to 0."""
    torch = torch_cuda()
    rng = np.random.default_rng(bits)
    cache = Cache(2, 2, 32, 2, 64, bits, 0, seed=3)
    k, v = (keys_and_values(rng, (6, 2, 64)) for _ in range(2))
    past = [20, 25]
    step = _with_first(cache.step([3, 3], past, most=6), [3, end, 6])
    print("case rows", bits, end, flush=True)
    L.lutgemm_kv_write(up(k.reshape(6, -1)), up(v.reshape(6, -1)), None, cache.c, step, 128, 128, stream())
    want, begin = cache.fill.copy(), max(end, 0)
    for row in range(begin, 6):
        for h in range(2):
            for key, x in ((True, k), (False, v)):
                cache.put(want, 1, past[1] + row - begin, h, key, x[row, h])
    np.testing.assert_array_equal(cache.pool(), want)
    out = [torch.full((6, 128), 77.0, dtype=torch.float16, device="cuda") for _ in range(2)]
    L.lutgemm_kv_read(cache.c, step, *out, 128, 128, stream())
    for got, x in zip(out, (k, v)):
        got = got.cpu().numpy().reshape(6, 2, 64)
        np.testing.assert_array_equal(got[begin:], cache.rounded(x)[begin:])
        assert (got[:begin] == 77).all()


@pytest.mark.parametrize("shared,tiles", [(1, 1), (4, 2), (16, 8)])
@pytest.mark.parametrize("end", [LEAST, LEAST + 2, -1])
def test_rows_that_end_before_they_begin_see_nothing(shared, tiles, end):
    torch = torch_cuda()
    rng = np.random.default_rng(shared)
    cache = Cache(2, 20, 32, 1, 64, 8, 0, seed=4)
    past = [20, 25]
    held = _fill(cache, rng, past, [0, 6])
    q = rng.standard_normal((6, shared, 64)).astype(np.float16)
    step = _with_first(cache.step([3, 3], past, most=6), [3, end, 6])
    plan = L.lutgemm_plan_attention(cache.c, step, shared)
    assert plan[0] == tiles
    print("case rows seen", shared, end, plan, flush=True)
    y = _run(cache, step, q, None, shared, 0.125, 0)
    _check(y, *K.attention(q, *held[1], past[1], None, 0.125), 64)
    # sequence 0 alone: no row is written
    alone = L.lutgemm_kv_step(up(np.array([3, end], np.int32)), step._held[1], step._held[2], 1, 20, 6, 6)
    y = _run(cache, alone, q, None, shared, 0.125, 0, d_y=torch.full((6, shared * 64 + 8), 77.0, dtype=torch.float16, device="cuda"))
    assert (y == 77).all()


@pytest.mark.parametrize("past", [(1 << 30) + 5, (1 << 31) - 7])
@pytest.mark.parametrize("shared,tiles", [(1, 1), (4, 2), (16, 8), (43, 16)])
@pytest.mark.parametrize("bits", [16, 4])
def test_a_missing_page_of_a_sequence_longer_than_its_table(bits, shared, tiles, past):
    """A length that no table holds: the rows see all that the table has, and nothing where it names no page."""
    rng = np.random.default_rng(shared + bits)
    cache = Cache(1, 20, 32, 1, 64, bits, 0, seed=5)
    k, v = _fill(cache, rng, [634], [6])[0]
    table = cache.table.copy()
    seen = np.ones(640, bool)
    for page in (0, 7, 8, 19):
        table[0, page] = -1
        seen[32 * page:32 * page + 32] = False
    q = rng.standard_normal((6, shared, 64)).astype(np.float16)
    step = cache.step([6], [past], table)
    plan = L.lutgemm_plan_attention(cache.c, step, shared)
    assert plan[0] == tiles
    print("case missing page", bits, shared, past, plan, flush=True)
    y = _run(cache, step, q, None, shared, 0.125, 0)
    none = np.zeros((6, 1, 64), np.float16)
    _check(y, *K.attention(q, np.concatenate([k[seen], none]), np.concatenate([v[seen], none]), int(seen.sum()), [0] * 6, 0.125), 64)
