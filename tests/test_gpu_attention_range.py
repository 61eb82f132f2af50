"""GPU checks of attention where scores or weights leave the ordinary range: scores too large for their differences to be
told, one score far above a long tail, infinite ones."""
import numpy as np
import pytest

import paper_2206_09557_amd as L
from oracle import kv_oracle as K

from kv_util import Cache, keys_and_values, stream, up
from test_gpu_attention import _check, _run

pytestmark = pytest.mark.gpu

DIM = 64


def _write(cache, k, v):
    n = len(k)
    L.lutgemm_kv_write(up(k.reshape(n, -1)), up(v.reshape(n, -1)), None, cache.c, cache.step([n], [0]), DIM, DIM, stream())


def _scores(rng, scores):
    """Keys whose first channel is `scores`, the rest zero; values as usual."""
    k = np.zeros((len(scores), 1, DIM), np.float16)
    k[:, 0, 0] = scores
    return k, keys_and_values(rng, (len(scores), 1, DIM))


@pytest.mark.parametrize("tokens,shared,tiles", [(2, 5, 1), (4, 5, 2), (10, 5, 4), (40, 5, 16)])
@pytest.mark.parametrize("order", ["rising", "falling", "shuffled"])
def test_scores_that_differ_by_more_than_any_weight(tokens, shared, tiles, order):
    """Up to 5e9, where fp32 counts in hundreds: the largest takes all, and its value comes out as it is."""
    rng = np.random.default_rng(tokens)
    n = 700 + tokens
    at = np.linspace(-60000, 60000, n)
    k, v = _scores(rng, {"rising": at, "falling": at[::-1], "shuffled": rng.permutation(at)}[order])
    cache = Cache(1, 30, 64, 1, DIM, 16, 0)
    _write(cache, k, v)
    q = np.zeros((tokens, shared, DIM), np.float16)
    q[..., 0] = np.linspace(30000, 60000, tokens * shared).reshape(tokens, shared)
    q[0, 0, 0] = -60000
    step = cache.step([tokens], [700])
    plan = L.lutgemm_plan_attention(cache.c, step, shared)
    assert plan[0] == tiles
    print("case large", tokens, shared, order, plan, flush=True)
    y = _run(cache, step, q, None, shared, 1.0, 0).reshape(tokens * shared, DIM)
    for r in range(tokens * shared):
        seen = k[:701 + r // shared, 0, 0].astype(np.float64) * float(q[r // shared, r % shared, 0])
        np.testing.assert_array_equal(y[r], v[int(seen.argmax()), 0])


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("tokens,shared,past,hint", [(1, 1, 4000, 32), (1, 4, 30000, 0), (3, 8, 9000, 0), (20, 5, 5000, 0), (20, 5, 300, 0)])
def test_one_high_score_over_a_long_tail(bits, tokens, shared, past, hint):
    """The first position's score stands above all others by up to 2^30; its value is zero, so that the result is the tail's share alone.
    A weight is rounded to fp16, by 2^-32 of its row's largest at most, beside what every weight may be off."""
    rng = np.random.default_rng(past)
    n = past + tokens
    k, v = _scores(rng, rng.uniform(-1, 0, n))
    k[0, 0, 0] = 20
    v[0] = 0
    v[1:] = np.abs(v[1:])
    cache = Cache(1, -(-n // 64), 64, 1, DIM, bits, 0)
    _write(cache, k, v)
    k, v = cache.rounded(k), cache.rounded(v)
    q = np.zeros((tokens, shared, DIM), np.float16)
    q[..., 0] = np.linspace(1.0, 0.55, tokens * shared).reshape(tokens, shared)
    step = cache.step([tokens], [past])
    print("case tail", bits, tokens, shared, past, L.lutgemm_plan_attention(cache.c, step, shared, hint), flush=True)
    y = _run(cache, step, q, None, shared, 1.0, hint).astype(np.float64)
    ref, mass, reach = K.attention(q, k, v, past, None, 1.0)
    score = (DIM + 8) * 2.0 ** -24 * reach * 2 + 2.0 ** -20          # as in the other tests of attention
    bound = 2.0 ** -11 * np.abs(ref) + (2.0 ** -10 + 2 * score) * mass + 2.0 ** -24 + 2.0 ** -32 * np.abs(v.astype(np.float64)).sum(0)
    err = np.abs(y - ref)
    worst = (err / bound).max()
    assert worst <= 1


@pytest.mark.parametrize("tokens,shared,tiles", [(2, 5, 1), (4, 5, 2), (10, 5, 4), (40, 5, 16)])
@pytest.mark.parametrize("pages,first,last", [(8, 0, 256), (8, 64, 100), (60, 0, 350)])
def test_keys_that_are_infinitely_far(tokens, shared, tiles, pages, first, last):
    """Scores of -inf count for nothing, whole blocks of them before any other score included; with none but those a row is zero.  One
    of +inf or NaN makes a row NaN."""
    rng = np.random.default_rng(last)
    past = 350
    cache = Cache(1, pages, 64, 1, DIM, 16, 0)
    k, v = (keys_and_values(rng, (past + tokens, 1, DIM)) for _ in range(2))
    k[first:last, 0, 0] = -np.inf
    _write(cache, k, v)
    q = rng.standard_normal((tokens, shared, DIM)).astype(np.float16)
    q[..., 0] = np.abs(q[..., 0]) + np.float16(0.5)
    q[-1, 0, 0], q[-1, 1, 0] = -1.0, 0.0
    step = cache.step([tokens], [past])
    plan = L.lutgemm_plan_attention(cache.c, step, shared)
    assert plan[0] == tiles
    print("case infinite", tokens, shared, pages, first, last, plan, flush=True)
    y = _run(cache, step, q, None, shared, DIM ** -0.5, 0)
    seen = np.r_[0:first, last:past + tokens]
    odd = np.zeros((tokens, shared), bool)
    odd[-1, :2] = True
    np.testing.assert_array_equal(np.isnan(y), np.repeat(odd[..., None], DIM, 2))
    ref, mass, reach = K.attention(q, k[seen], v[seen], past - (last - first), None, DIM ** -0.5)
    _check(y[~odd], ref[~odd], mass[~odd], reach, DIM)
    # none but those
    mask = np.zeros(tokens, np.uint64)
    k[:past, 0, 0] = -np.inf
    _write(cache, k[:past], v[:past])
    y = _run(cache, step, q, mask, shared, DIM ** -0.5, 0)
    assert (y[~odd] == 0).all() and np.isnan(y[odd]).all()
