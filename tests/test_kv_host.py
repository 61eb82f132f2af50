"""CPU checks of the attention half: sizes, frequencies, plans, and what the entry points refuse (all before any GPU call)."""
import numpy as np
import pytest

import paper_2206_09557_amd as L
from oracle import kv_oracle as K

A = 1 << 20      # an aligned address that nothing reads: every call below is refused


def _cache(pool=A, pages=4, page=64, heads=2, dim=128, bits=8, group=0):
    return L.lutgemm_kv_cache(pool, pages, page, heads, dim, bits, group)


def _step(first=A, past=A, table=A, seqs=1, table_pages=4, tokens=1, most=1):
    return L.lutgemm_kv_step(first, past, table, seqs, table_pages, tokens, most)


@pytest.mark.parametrize("scaling", range(4))
def test_frequencies(scaling):
    for rot in (2, 24, 128):
        t = L.lutgemm_rope_frequencies(rot, 10000.0, scaling, 4.0, 1.0, 32.0, 4096.0)
        f = K.frequencies(rot, 10000.0, scaling, 4.0, 1.0, 32.0, 4096.0)
        # both in double, some operations apart: 2^-48 of a value
        assert np.abs(t.astype(np.float64) / 2.0 ** 64 * 2 * np.pi - f).max() <= 2.0 ** -48


def test_frequency_refusals():
    for args in [(0,), (3,), (65538,), (8, 1.0), (8, float("nan")), (8, 1e4, 1, 0.5), (8, 1e4, 3, 2.0, 5.0, 5.0, 100.0), (8, 1e4, 3, 2.0, 1.0, 4.0, 0.0),
                 (8, 1e300, 2, 1e300)]:
        with pytest.raises(L.LutGemmError) as e:
            L.lutgemm_rope_frequencies(*args)
        assert e.value.code == L.LUTGEMM_EINVAL
    with pytest.raises(L.LutGemmError) as e:
        L.lutgemm_rope_frequencies(8, 1e4, 4)
    assert e.value.code == L.LUTGEMM_EUNSUPPORTED


def test_pool_sizes():
    for bits in (4, 8, 16):
        for dim in (64, 96, 128, 192, 256):
            for group in (0, 32, dim):
                assert L.lutgemm_kv_pool_bytes(3, 96, 5, dim, bits, group) == K.pool_bytes(3, 96, 5, dim, bits, group or dim)
    assert L.lutgemm_kv_pool_bytes(1 << 20, 64, 8, 128, 16) == 2 * 2 * (1 << 20) * 64 * 8 * 128
    for bad in [(0, 64, 1, 64, 8), (1, 48, 1, 64, 8), (1, 0, 1, 64, 8), (1, 64, 0, 64, 8), (1, 64, 1, 80, 8), (1, 64, 1, 64, 5), (1, 64, 1, 96, 8, 64),
                (1, 64, 1, 64, 8, 16), (1, 64, 1, 64, 8, -32)]:
        assert L.lutgemm_kv_pool_bytes(*bad) == 0


def test_rope_refusals():
    good = dict(x=A, y=A + 4096, p=A, t=A, tokens=1, heads=2, dim=64, rot=64, xs=128, ys=128, flags=0)

    def code(**change):
        g = {**good, **change}
        with pytest.raises(L.LutGemmError) as e:
            L.lutgemm_rope(g["x"], g["y"], g["p"], g["t"], g["tokens"], g["heads"], g["dim"], g["rot"], g["xs"], g["ys"], 1.0, g["flags"])
        return e.value.code

    for change in [dict(x=0), dict(y=None), dict(p=0), dict(t=0), dict(tokens=-1), dict(heads=0), dict(rot=0), dict(rot=3), dict(rot=66), dict(dim=65, rot=64),
                   dict(xs=127), dict(ys=127), dict(x=A + 1), dict(y=A + 4097), dict(p=A + 2), dict(t=A + 4), dict(x=A + 2, flags=L.LUTGEMM_Y_F32),
                   dict(y=A, ys=256)]:
        assert code(**change) == L.LUTGEMM_EINVAL, change
    for change in [dict(flags=2), dict(flags=32), dict(dim=514, rot=64, xs=2048, ys=2048)]:
        assert code(**change) == L.LUTGEMM_EUNSUPPORTED, change


def _bad_caches():
    E, U = L.LUTGEMM_EINVAL, L.LUTGEMM_EUNSUPPORTED
    return [(None, E), (_cache(pool=0), E), (_cache(pool=A + 8), E), (_cache(pages=0), E), (_cache(page=33), E), (_cache(heads=0), E), (_cache(dim=0), E),
            (_cache(dim=112), U), (_cache(bits=3), U), (_cache(group=96), E), (_cache(group=16), U), (_cache(group=-1), E), (_cache(pages=1 << 40), U)]


def _bad_steps():
    E, U = L.LUTGEMM_EINVAL, L.LUTGEMM_EUNSUPPORTED
    return [(None, E), (_step(first=0), E), (_step(past=0), E), (_step(table=0), E), (_step(first=A + 2), E), (_step(seqs=0), E), (_step(table_pages=0), E),
            (_step(tokens=-1), E), (_step(most=-1), E), (_step(seqs=70000), U)]


def test_cache_refusals():
    def code(call, *args):
        with pytest.raises(L.LutGemmError) as e:
            call(*args)
        return e.value.code

    for c, want in _bad_caches():
        assert code(L.lutgemm_kv_write, A, A, None, c, _step(), 256, 256) == want
        assert code(L.lutgemm_kv_read, c, _step(), A, A, 256, 256) == want
    for s, want in _bad_steps():
        assert code(L.lutgemm_kv_write, A, A, None, _cache(), s, 256, 256) == want
        assert code(L.lutgemm_kv_read, _cache(), s, A, A, 256, 256) == want
    E = L.LUTGEMM_EINVAL
    for k, v, rows, ks, vs in [(None, None, None, 256, 256), (A + 2, A, None, 256, 256), (A, A + 8, None, 256, 256), (A, A, A + 1, 256, 256),
                               (A, A, None, 248, 256), (A, A, None, 256, 255), (A, A, None, 260, 256)]:
        assert code(L.lutgemm_kv_write, k, v, rows, _cache(), _step(), ks, vs) == E
        if rows is None:
            assert code(L.lutgemm_kv_read, _cache(), _step(), k, v, ks, vs) == E


def test_attention_refusals_and_plans():
    def code(c=None, s=None, q=A, mask=None, y=A + 8192, q_heads=4, qs=512, ys=512, most=0, ws=A, nbytes=1 << 40):
        with pytest.raises(L.LutGemmError) as e:
            L.lutgemm_attention(q, mask, _cache() if c is None else c, _step() if s is None else s, y, q_heads, qs, ys, 1.0, most, ws, nbytes)
        return e.value.code

    for c, want in _bad_caches()[1:]:
        assert code(c=c) == want
        if c.pool and c.pool % 16 == 0:
            assert L.lutgemm_attention_workspace_bytes(c, _step(), 4) == 0
    for s, want in _bad_steps()[1:]:
        assert code(s=s) == want
    for change in [dict(q=0), dict(y=0), dict(ws=0), dict(q=A + 2), dict(y=A + 8), dict(ws=A + 4), dict(mask=A + 4), dict(q_heads=0), dict(q_heads=3), dict(qs=511),
                   dict(qs=508), dict(ys=256), dict(most=-1)]:
        assert code(**change) == L.LUTGEMM_EINVAL, change
    assert code(s=_step(most=65, tokens=65)) == L.LUTGEMM_EUNSUPPORTED
    need = L.lutgemm_attention_workspace_bytes(_cache(), _step(), 4)
    assert need >= 32768 and code(nbytes=need - 1) == L.LUTGEMM_EWORKSPACE
    # what a plan covers: all rows, all positions; no split that has nothing to do
    for seqs, heads, shared, tokens, positions, dim in [(1, 1, 1, 1, 1, 64), (1, 40, 1, 1, 300, 128), (16, 64, 1, 1, 4000, 128), (1, 8, 8, 1, 131072, 128),
                                                        (4, 8, 8, 64, 8256, 128), (1, 96, 1, 32, 2080, 256), (300, 96, 2, 7, 5000, 96)]:
        c = _cache(heads=heads, dim=dim, pages=1 << 20)
        s = _step(seqs=seqs, tokens=seqs * tokens, most=tokens, table_pages=1 << 12)
        row_tiles, row_blocks, splits, chunk, waves = L.lutgemm_plan_attention(c, s, heads * shared, positions)
        assert 16 * row_tiles * row_blocks >= tokens * shared > 16 * row_tiles * (row_blocks - 1)
        assert chunk % 32 == 0 and chunk * splits >= positions > chunk * (splits - 1)
        rows = min(16 * row_tiles, tokens * shared)
        floats = 0 if splits == 1 else seqs * heads * row_blocks * splits * rows * (dim + 2)
        assert L.lutgemm_attention_workspace_bytes(c, s, heads * shared, positions) == 32768 + 4 * floats
