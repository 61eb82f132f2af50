"""CPU checks that what is asked about sizes and the calls themselves agree, at the limits and beyond (no call gets as far as the GPU)."""
import random

import pytest

import paper_2206_09557_amd as L

A = 1 << 20      # an aligned address that nothing reads


def _code(call, *args):
    with pytest.raises(L.LutGemmError) as e:
        call(*args)
    return e.value.code


def _asked_and_called(pages=4, page=64, heads=2, dim=128, bits=8, group=0, seqs=1, table_pages=4, tokens=1, most=1, q_heads=4, positions=0):
    """What the plan says (None: it is made), the workspace's bytes, the call's code with no workspace at all."""
    c = L.lutgemm_kv_cache(A, pages, page, heads, dim, bits, group)
    s = L.lutgemm_kv_step(A, A, A, seqs, table_pages, tokens, most)
    row = max(q_heads, 1) * dim
    called = _code(L.lutgemm_attention, A, None, c, s, A, q_heads, row, row, 1.0, positions, A, 0)
    try:
        plan = L.lutgemm_plan_attention(c, s, q_heads, positions)
        return None, plan, L.lutgemm_attention_workspace_bytes(c, s, q_heads, positions), called
    except L.LutGemmError as e:
        return e.code, None, L.lutgemm_attention_workspace_bytes(c, s, q_heads, positions), called


@pytest.mark.parametrize("sizes,code", [
    (dict(), None), (dict(page=1 << 20, table_pages=1 << 10), None), (dict(page=1 << 20, table_pages=(1 << 10) + 1), L.LUTGEMM_EUNSUPPORTED),
    (dict(page=64, table_pages=1 << 25), L.LUTGEMM_EUNSUPPORTED), (dict(heads=4, q_heads=1 << 14, most=64, tokens=64), None),
    (dict(q_heads=(1 << 14) + 2), L.LUTGEMM_EUNSUPPORTED), (dict(most=65, tokens=65), L.LUTGEMM_EUNSUPPORTED), (dict(seqs=65535), None),
    (dict(seqs=65536), L.LUTGEMM_EUNSUPPORTED), (dict(tokens=-1), L.LUTGEMM_EINVAL), (dict(most=-1), L.LUTGEMM_EINVAL),
    (dict(q_heads=3), L.LUTGEMM_EINVAL), (dict(q_heads=0), L.LUTGEMM_EINVAL), (dict(positions=-1), L.LUTGEMM_EINVAL),
    (dict(heads=4097, q_heads=4097), L.LUTGEMM_EUNSUPPORTED), (dict(page=48), L.LUTGEMM_EINVAL)])
def test_what_is_asked_is_what_is_called(sizes, code):
    asked, _, nbytes, called = _asked_and_called(**sizes)
    assert asked == code and (nbytes > 0) == (code is None)
    assert called == (L.LUTGEMM_EWORKSPACE if code is None else code)


def test_any_sizes():
    rng = random.Random(5)
    for _ in range(3000):
        heads = rng.choice([1, 2, 3, 8, 30, 96, 4096])
        sizes = dict(page=rng.choice([32, 64, 96, 1 << 20]), heads=heads, dim=rng.choice([64, 96, 128, 192, 256]), bits=rng.choice([4, 8, 16]),
                     seqs=rng.choice([1, 5, 300, 65535]), table_pages=rng.choice([1, 7, 1000, 1 << 14, 1 << 25]), most=rng.randint(1, 64), tokens=64,
                     q_heads=heads * rng.choice([1, 2, 5, 16, 128, 4096]), positions=rng.choice([0, 1, 5000, 1 << 40]))
        asked, plan, nbytes, called = _asked_and_called(**sizes)
        assert called == (L.LUTGEMM_EWORKSPACE if asked is None else asked), sizes
        if plan:
            assert heads * plan[1] <= 65535 and plan[2] <= 128 and nbytes >= 32768, (sizes, plan)      # sides of a grid


@pytest.mark.parametrize("most,shared,dim,rows", [(1, 1, 64, 1), (1, 3, 96, 3), (3, 5, 128, 15), (17, 1, 128, 17), (13, 3, 64, 39), (31, 1, 256, 31), (5, 5, 192, 25)])
def test_partial_results_begin_on_16_bytes(most, shared, dim, rows):
    """Of every split: `rows` sums of `dim` floats, which are moved 16 bytes at a time, and two floats a row."""
    c = L.lutgemm_kv_cache(A, 4, 64, 2, dim, 8, 0)
    s = L.lutgemm_kv_step(A, A, A, 1, 1 << 11, most, most)
    plan = L.lutgemm_plan_attention(c, s, 2 * shared)
    assert plan[1] == 1 and plan[2] > 1
    nbytes = L.lutgemm_attention_workspace_bytes(c, s, 2 * shared) - 32768
    each = nbytes // (2 * plan[2])
    assert nbytes == each * 2 * plan[2] and each % 16 == 0 and 0 <= each - 4 * rows * (dim + 2) < 16


def test_pools_beyond_any_offset():
    """2^73 bytes: the product of the sizes leaves 64 bits, and none of its low bits is a size."""
    for pages, page, heads, dim, bits in [((1 << 31) - 1, 1 << 20, 1 << 12, 256, 16), (1 << 22, 1 << 20, 1 << 12, 128, 16), ((1 << 31) - 1, 1 << 20, 4000, 192, 4)]:
        assert L.lutgemm_kv_pool_bytes(pages, page, heads, dim, bits) == 0
        c, s = L.lutgemm_kv_cache(A, pages, page, heads, dim, bits), L.lutgemm_kv_step(A, A, A, 1, 1, 1, 1)
        row = heads * dim
        assert _code(L.lutgemm_kv_write, A, A, None, c, s, row, row) == L.LUTGEMM_EUNSUPPORTED
        assert _code(L.lutgemm_kv_read, c, s, A, A, row, row) == L.LUTGEMM_EUNSUPPORTED
        assert _code(L.lutgemm_attention, A, None, c, s, A, heads, row, row, 1.0, 0, A, 1 << 40) == L.LUTGEMM_EUNSUPPORTED
    assert L.lutgemm_kv_pool_bytes(1 << 20, 1 << 20, 1 << 12, 256, 16) == 1 << 62
