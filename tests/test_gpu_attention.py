"""GPU parity of lutgemm_attention with the 64-bit oracle, on what the cache holds: types, head layouts, lengths, masks."""
import numpy as np
import pytest

import paper_2206_09557_amd as L
from oracle import kv_oracle as K

from gpu_util import make_workspace, torch_cuda
from kv_util import Cache, keys_and_values, stream, up

pytestmark = pytest.mark.gpu


def _tree(rng, counts, empty=False):
    words = []
    for n in counts:
        mine = []
        for t in range(n):
            parent = int(rng.integers(-1, t)) if t else -1
            mine.append((mine[parent] if parent >= 0 else 0) | 1 << t)
        if empty:
            mine = [0 if t % 3 == 1 else w | 1 << 63 >> (t % 7) for t, w in enumerate(mine)]      # bits beyond the tokens too
        words += mine
    return np.array(words, dtype=np.uint64)


def _run(cache, step, q, mask, q_heads, scale, most_positions, d_y=None, ws=None):
    torch = torch_cuda()
    tokens, row = q.shape[0], q_heads * cache.dim
    padded = np.concatenate([q.reshape(tokens, row), np.full((tokens, 16), np.nan, np.float16)], 1)
    d_y = torch.full((tokens, row + 8), 77.0, dtype=torch.float16, device="cuda") if d_y is None else d_y
    nbytes = L.lutgemm_attention_workspace_bytes(cache.c, step, q_heads, most_positions)
    ws = make_workspace(nbytes) if ws is None else ws
    L.lutgemm_attention(up(padded), None if mask is None else up(mask), cache.c, step, d_y, q_heads, row + 16, row + 8, scale,
                        most_positions, ws, nbytes, stream())
    y = d_y.cpu().numpy()
    assert (y[:, row:] == 77).all()
    assert int(ws[:32768].sum()) == 0        # the counters are as they were
    return y[:, :row].reshape(tokens, q_heads, cache.dim)


def _check(y, ref, mass, reach, dim):
    """y fp16 against the oracle.  Its own rounding (half an ulp); a weight's rounding to fp16 and that of their sum's share, 2^-11
    each, against the mass that the weights carry; the scores' rounding in fp32 (dim products, log2 e, exp2), on
    both sides of the quotient."""
    score = (dim + 8) * 2.0 ** -24 * reach * 2 + 2.0 ** -20
    bound = 2.0 ** -11 * np.abs(ref) + (2.0 ** -10 + 2 * score) * mass + 2.0 ** -24
    err = np.abs(y.astype(np.float64) - ref)
    assert (err <= bound).all(), (err / bound).max()


def _fill(cache, rng, past, counts):
    """Random keys and values for every sequence's positions; what the cache makes of them, per sequence."""
    held = []
    for s, (p, c) in enumerate(zip(past, counts)):
        k, v = (keys_and_values(rng, (p + c, cache.heads, cache.dim)) for _ in range(2))
        if p + c:
            step = cache.step([p + c], [0], cache.table[s:s + 1])
            row = cache.heads * cache.dim
            L.lutgemm_kv_write(up(k.reshape(p + c, row)), up(v.reshape(p + c, row)), None, cache.c, step, row, row, stream())
        held.append((cache.rounded(k), cache.rounded(v)))
    return held


@pytest.mark.parametrize("bits,dim,group,heads,shared,page,counts,past,masked", [
    (16, 128, 0, 2, 1, 32, [1], [0], None),                                  # one token that sees itself
    (16, 64, 0, 3, 1, 64, [1, 1, 1], [31, 32, 33], None),
    (8, 128, 0, 2, 1, 64, [1, 1], [500, 129], "tree"),
    (4, 128, 32, 1, 8, 64, [1], [1000], None),
    (4, 128, 64, 2, 4, 32, [5, 3, 0, 1], [95, 0, 40, 7], "tree"),
    (8, 96, 96, 2, 7, 96, [11, 2], [300, 5], "empty"),
    (4, 96, 32, 1, 7, 96, [11, 1, 4], [0, 64, 0], "empty"),
    (16, 96, 0, 1, 3, 32, [64], [17], "tree"),
    (8, 64, 32, 1, 16, 64, [33, 64], [70, 0], "tree"),
    (8, 192, 64, 2, 2, 64, [9], [200], "tree"),
    (4, 192, 96, 1, 3, 64, [21], [45], None),
    (8, 256, 128, 1, 5, 128, [13], [333], "tree"),
    (4, 256, 0, 1, 2, 32, [2], [64], None),
    (16, 256, 0, 1, 1, 64, [64], [100], "empty"),
    (16, 192, 0, 1, 1, 32, [17], [31], None),
    (8, 128, 128, 1, 5, 32, [40], [1], "tree"),
    (4, 256, 64, 1, 1, 64, [3], [90], None),
    (8, 192, 32, 1, 1, 64, [3], [90], None),
    (4, 192, 192, 1, 2, 64, [3], [90], None),
    (4, 256, 32, 1, 33, 64, [2], [90], "tree"),
    (4, 64, 64, 4, 1, 64, [32], [63], "tree")])
def test_against_oracle(bits, dim, group, heads, shared, page, counts, past, masked):
    rng = np.random.default_rng(bits * 7 + dim + sum(past))
    most = max(p + c for p, c in zip(past, counts))
    cache = Cache(len(counts), -(-most // page) + 1, page, heads, dim, bits, group, seed=dim)
    cache.d_pool.fill_(255)                   # what is not written is NaN
    held = _fill(cache, rng, past, counts)
    q = (1.5 * rng.standard_normal((sum(counts), heads * shared, dim))).astype(np.float16)
    mask = None if masked is None else _tree(rng, counts, masked == "empty")
    step = cache.step(counts, past)
    for hint in (most, 0, 32 * 60):           # the split, from one workgroup to many; the result is right for any hint
        plan = L.lutgemm_plan_attention(cache.c, step, heads * shared, hint)
        print("case attention", bits, dim, group, heads, shared, page, counts, past, masked, hint, plan, flush=True)
        y = _run(cache, step, q, mask, heads * shared, dim ** -0.5, hint)
        at = 0
        for s, n in enumerate(counts):
            ref, mass, reach = K.attention(q[at:at + n], *held[s], past[s], None if mask is None else mask[at:at + n], dim ** -0.5)
            _check(y[at:at + n], ref, mass, reach, dim)
            if masked == "empty" and past[s] == 0:
                none = [t for t in range(n) if int(mask[at + t]) & ((1 << n) - 1) == 0]
                assert (y[[at + t for t in none]] == 0).all()
            at += n


@pytest.mark.parametrize("bits,heads,shared,tokens,past", [(8, 1, 1, 1, 9000), (4, 2, 8, 1, 5003), (16, 1, 4, 16, 4100), (8, 1, 2, 64, 3500),
                                                            (4, 1, 1, 32, 6007)])
def test_split_positions(bits, heads, shared, tokens, past):
    rng = np.random.default_rng(past)
    cache = Cache(1, -(-(past + tokens) // 64), 64, heads, 128, bits, 64, seed=1)
    held = _fill(cache, rng, [past], [tokens])
    q = (1.5 * rng.standard_normal((tokens, heads * shared, 128))).astype(np.float16)
    mask, step = _tree(rng, [tokens]), cache.step([tokens], [past])
    plan = L.lutgemm_plan_attention(cache.c, step, heads * shared, past + tokens)
    assert plan[2] > 1
    print("case split", bits, heads, shared, tokens, past, plan, flush=True)
    y = _run(cache, step, q, mask, heads * shared, 128 ** -0.5, past + tokens)
    _check(y, *K.attention(q, *held[0], past, mask, 128 ** -0.5), 128)
    # a hint that is far too small: fewer and longer splits, the same result to the same bound
    short = _run(cache, step, q, mask, heads * shared, 128 ** -0.5, 40)
    _check(short, *K.attention(q, *held[0], past, mask, 128 ** -0.5), 128)
    nbytes = L.lutgemm_attention_workspace_bytes(cache.c, step, heads * shared, past + tokens)
    ws = make_workspace(nbytes)
    for _ in range(20):                       # bit for bit from run to run, whoever arrives last
        np.testing.assert_array_equal(_run(cache, step, q, mask, heads * shared, 128 ** -0.5, past + tokens, ws=ws), y)


@pytest.mark.parametrize("spread", [0.0, 30.0, 300.0])
def test_scores_of_any_size(spread):
    """All alike, far apart, rising from position to position (the kept maximum is raised again and again)."""
    rng = np.random.default_rng(1)
    past, dim = 700, 64
    cache = Cache(1, 12, 64, 1, dim, 16, 0)
    k, v = (keys_and_values(rng, (past + 2, 1, dim)) for _ in range(2))
    q = np.zeros((2, 2, dim), np.float16)
    q[..., 0] = 1.0
    k[..., 0] = (spread * np.linspace(-1, 1, past + 2)[:, None]).astype(np.float16)
    k[..., 1:] = 0
    L.lutgemm_kv_write(up(k.reshape(-1, dim)), up(v.reshape(-1, dim)), None, cache.c, cache.step([past + 2], [0]), dim, dim, stream())
    y = _run(cache, cache.step([2], [past]), q, None, 2, 1.0, past + 2)
    _check(y, *K.attention(q, k, v, past, None, 1.0), dim)


@pytest.mark.parametrize("bits", [16, 8])
def test_not_finite_where_it_is_not_seen(bits):
    """Infinities and NaNs in keys and values of new tokens reach the rows that see them and no others."""
    rng = np.random.default_rng(2)
    past, n, dim, heads, shared = 40, 6, 64, 2, 3
    cache = Cache(1, 2, 32, heads, dim, bits, 32)
    k, v = (keys_and_values(rng, (past + n, heads, dim)) for _ in range(2))
    v[past + 1, 0, 5], v[past + 1, 0, 40] = np.inf, -np.inf
    v[past + 2, 0, 5] = -np.inf
    v[past + 3, 1, 9] = np.nan
    k[past + 4, 1, 0] = np.nan
    row = heads * dim
    L.lutgemm_kv_write(up(k.reshape(-1, row)), up(v.reshape(-1, row)), None, cache.c, cache.step([past + n], [0]), row, row, stream())
    mask = np.array([1, 2, 6, 8, 16, 33], dtype=np.uint64)     # tokens 0 and 5 see nothing odd
    q = rng.standard_normal((n, heads * shared, dim)).astype(np.float16)
    y = _run(cache, cache.step([n], [past]), q, mask, heads * shared, dim ** -0.5, past + n)
    kk, vv = cache.rounded(k), cache.rounded(v)
    with np.errstate(invalid="ignore"):
        ref, mass, reach = K.attention(q, kk, vv, past, mask, dim ** -0.5)
    fine = np.isfinite(ref)
    assert fine[[0, 5]].all() and not fine.all()
    np.testing.assert_array_equal(np.isnan(y), np.isnan(ref))
    np.testing.assert_array_equal(y[np.isinf(ref)], ref[np.isinf(ref)])
    _check(y[fine], ref[fine], mass[fine], reach, dim)


def test_what_the_device_arrays_say_is_checked():
    """Pages outside the pool hold nothing; rows beyond the host's count are not written."""
    torch = torch_cuda()
    rng = np.random.default_rng(7)
    cache = Cache(2, 3, 32, 1, 64, 8, 0)
    past, counts = [70, 20], [4, 4]
    held = _fill(cache, rng, past, counts)
    q = rng.standard_normal((8, 2, 64)).astype(np.float16)
    table = cache.table.copy()
    table[0, 1] = cache.pages + 7
    y = _run(cache, cache.step(counts, past, table), q, None, 2, 0.125, 0)
    keep = np.r_[0:32, 64:74]
    ref = K.attention(q[:4], held[0][0][keep], held[0][1][keep], 38, None, 0.125)
    _check(y[:4], *ref, 64)
    d_y = torch.full((8, 2 * 64 + 8), 77.0, dtype=torch.float16, device="cuda")
    step = cache.step(counts, past, most=2)       # the second half of each sequence's rows is not announced
    y = _run(cache, step, q, None, 2, 0.125, 0, d_y=d_y)
    assert (y[2:4] == 77).all() and (y[6:] == 77).all() and (y[:2] != 77).any()


def test_workspace_of_a_product_and_a_graph():
    """Captured once, replayed with other lengths; the workspace is one that a product uses too."""
    torch = torch_cuda()
    rng = np.random.default_rng(8)
    cache = Cache(2, 40, 64, 2, 128, 8, 0)
    held = _fill(cache, rng, [2000, 1500], [1, 1])
    q = rng.standard_normal((2, 4, 128)).astype(np.float16)
    first, past = up(np.array([0, 1, 2], np.int32)), up(np.array([0, 0], np.int32))
    table = up(cache.table)
    step = L.lutgemm_kv_step(first, past, table, 2, 40, 2, 1)
    nbytes = max(L.lutgemm_attention_workspace_bytes(cache.c, step, 4, 0), L.lutgemm_workspace_bytes(512, 2048, 3, 128))
    ws = make_workspace(nbytes)
    d_q, d_y = up(q.reshape(2, -1)), torch.zeros((2, 512), dtype=torch.float16, device="cuda")
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        L.lutgemm_attention(d_q, None, cache.c, step, d_y, 4, 512, 512, 128 ** -0.5, 0, ws, nbytes, side.cuda_stream)
    for lengths in ([2000, 1500], [0, 1], [33, 700], [2000, 1500]):
        past.copy_(torch.tensor(lengths, dtype=torch.int32))
        d_y.fill_(77)
        graph.replay()
        torch.cuda.synchronize()
        for s, p in enumerate(lengths):
            ref = K.attention(q[s:s + 1], held[s][0][:p + 1], held[s][1][:p + 1], p, None, 128 ** -0.5)
            _check(d_y[s:s + 1].cpu().numpy().reshape(1, 4, 128), *ref, 128)
