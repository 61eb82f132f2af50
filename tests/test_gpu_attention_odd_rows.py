"""GPU parity of attention for odd numbers of rows whose splits' partial results meet in memory."""
import numpy as np
import pytest

import paper_2206_09557_amd as L
from oracle import kv_oracle as K

from kv_util import Cache
from test_gpu_attention import _check, _fill, _run, _tree

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("tokens,shared", [(1, 1), (3, 5), (17, 1), (13, 3), (43, 5)])
def test_odd_rows_in_several_splits(dim, tokens, shared):
    rng = np.random.default_rng(dim + tokens)
    past = 3000
    cache = Cache(1, 49, 64, 2, dim, 8, 0)
    k, v = _fill(cache, rng, [past], [tokens])[0]
    q = (1.5 * rng.standard_normal((tokens, 2 * shared, dim))).astype(np.float16)
    step, mask = cache.step([tokens], [past]), _tree(rng, [tokens], tokens > 1)
    plan = L.lutgemm_plan_attention(cache.c, step, 2 * shared, past + tokens)
    assert plan[2] > 1
    print("case odd rows", dim, tokens, shared, plan, flush=True)
    y = _run(cache, step, q, mask, 2 * shared, dim ** -0.5, past + tokens)
    _check(y, *K.attention(q, k, v, past, mask, dim ** -0.5), dim)
