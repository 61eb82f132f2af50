"""CPU checks of placing, norm and adapters: what the entry points refuse (all before any GPU call), workspace and plan of adapters."""
import pytest

import paper_2206_09557_amd as L

A = 1 << 20      # an aligned address that nothing reads: every call below is refused
E, U, W = L.LUTGEMM_EINVAL, L.LUTGEMM_EUNSUPPORTED, L.LUTGEMM_EWORKSPACE


def _refused(call, *args):
    with pytest.raises(L.LutGemmError) as e:
        call(*args)
    return e.value.code


def _pages(free=A, count=A, owned=A, table=A, pages=8, page_tokens=64, seqs=2, table_pages=4):
    return L.lutgemm_kv_pages(free, count, owned, table, pages, page_tokens, seqs, table_pages)


BAD_PAGES = [(dict(free=0), E), (dict(count=0), E), (dict(owned=0), E), (dict(table=0), E), (dict(free=A + 2), E), (dict(table=A + 1), E), (dict(pages=0), E),
             (dict(page_tokens=48), E), (dict(page_tokens=0), E), (dict(seqs=0), E), (dict(table_pages=0), E), (dict(pages=1 << 31), U), (dict(seqs=65536), U),
             (dict(page_tokens=1 << 21), U), (dict(table_pages=(1 << 24) + 1), U), (dict(pages=(1 << 30) + 1), U), (dict(seqs=65535, table_pages=1 << 15), U)]


@pytest.mark.parametrize("change,want", BAD_PAGES, ids=lambda v: str(v))
def test_pages_are_checked(change, want):
    g = _pages(**change)
    assert _refused(L.lutgemm_kv_pages_init, g) == want
    assert _refused(L.lutgemm_kv_place, g, A, A, 4, 2, A, A, A, A) == want
    assert _refused(L.lutgemm_kv_trim, g, A) == want


def test_place_and_trim_refusals():
    good = dict(pages=_pages(), past=A, fresh=A, tokens=4, most=2, first=A, positions=A, owner=A, slots=A)
    for change in [dict(pages=None), dict(past=0), dict(fresh=None), dict(first=0), dict(tokens=-1), dict(most=-1), dict(past=A + 2), dict(fresh=A + 1), dict(first=A + 2),
                   dict(positions=A + 2), dict(owner=A + 3), dict(slots=A + 4)]:
        assert _refused(L.lutgemm_kv_place, *{**good, **change}.values()) == E, change
    assert _refused(L.lutgemm_kv_place, *{**good, "tokens": (1 << 30) + 1}.values()) == U
    assert _refused(L.lutgemm_kv_trim, None, A) == E and _refused(L.lutgemm_kv_trim, _pages(), 0) == E and _refused(L.lutgemm_kv_trim, _pages(), A + 2) == E


def _norm(**change):
    g = dict(x=A, residual=A + (1 << 16), weight=A, sum=A + (2 << 16), y=A + (3 << 16), scales=None, tokens=3, n=64, group=0, xs=64, ss=64, ys=64, eps=1e-5, flags=0)
    return _refused(L.lutgemm_rms_norm, *{**g, **change}.values())


def test_norm_refusals():
    for change in [dict(x=0), dict(y=None), dict(tokens=-1), dict(n=0), dict(xs=63), dict(ss=63), dict(ys=63), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("inf")),
                   dict(eps=float("nan")), dict(x=A + 1), dict(residual=A + 1), dict(sum=A + 1), dict(y=A + 1), dict(weight=A + 1), dict(x=A + 2, flags=L.LUTGEMM_Y_F32),
                   dict(sum=A + 2, flags=L.LUTGEMM_NORM_STREAM_F32), dict(scales=A + 2), dict(group=32), dict(group=-32, scales=A), dict(group=96, scales=A)]:
        assert _norm(**change) == E, change
    for change in [dict(flags=2), dict(flags=16), dict(n=32769, xs=40000, ss=40000, ys=40000), dict(tokens=(1 << 21) + 1), dict(group=16, scales=A), dict(xs=(1 << 28) + 1),
                   dict(ss=1 << 29), dict(ys=1 << 29)]:
        assert _norm(**change) == U, change


def test_norm_overlaps_are_refused():
    for change in [dict(y=A + 2), dict(y=A + 2 * 64 * 2 + 126),            # into a row of x; into its last one
                   dict(sum=A + (1 << 16) + 2), dict(sum=A + (3 << 16)), dict(sum=A + (3 << 16) + 64),   # residual, y
                   dict(y=A, ys=128), dict(sum=A, ss=128),                 # the same place, other strides
                   dict(y=A, scales=A, group=32), dict(sum=A, flags=L.LUTGEMM_NORM_STREAM_F32), dict(y=A, flags=L.LUTGEMM_Y_F32),   # other types
                   dict(xs=128, ys=128, y=A + 64), dict(xs=128, ys=128, y=A + 254), dict(xs=128, ys=128, y=A - 64),      # side by side, but not far enough
                   dict(xs=128, ys=100, y=A + 128)]:
        assert _norm(**change) == E, change


def _adapters(down=A, up=A, ranks=A, scales=A, m=96, n=64, count=3, rank=16):
    return L.lutgemm_adapters(down, up, ranks, scales, m, n, count, rank)


BAD_ADAPTERS = [(dict(m=0), E), (dict(n=0), E), (dict(n=12), E), (dict(count=0), E), (dict(rank=0), E), (dict(rank=12), E), (dict(count=1025), U), (dict(rank=264), U),
                (dict(m=(1 << 20) + 1), U), (dict(n=(1 << 20) + 8), U)]


@pytest.mark.parametrize("change,want", BAD_ADAPTERS, ids=lambda v: str(v))
def test_adapters_are_checked(change, want):
    a = _adapters(**change)
    assert _refused(L.lutgemm_adapt, A, A, a, A, None, A, 3, 0, 64, 96, 96, 0, A, 1 << 40) == want
    assert _refused(L.lutgemm_plan_adapt, a, 3) == want
    assert L.lutgemm_adapt_workspace_bytes(a, 3) == 0


def test_adapt_refusals():
    good = dict(x=A, base=A, adapters=_adapters(), of=A, owner=A, y=A, tokens=3, seqs=2, xs=64, bs=96, ys=96, flags=0, ws=A, nbytes=1 << 40)
    for change in [dict(adapters=None), dict(x=0), dict(base=0), dict(of=0), dict(y=0), dict(ws=0), dict(tokens=-1), dict(seqs=0), dict(x=A + 8), dict(ws=A + 4), dict(of=A + 2),
                   dict(owner=A + 2), dict(base=A + 1), dict(y=A + 1), dict(base=A + 2, flags=L.LUTGEMM_Y_F32), dict(xs=56), dict(xs=68), dict(bs=95), dict(ys=95),
                   dict(bs=104), dict(adapters=_adapters(down=0)), dict(adapters=_adapters(up=0)), dict(adapters=_adapters(down=A + 2)),
                   dict(adapters=_adapters(up=A + 8)), dict(adapters=_adapters(ranks=A + 2)), dict(adapters=_adapters(scales=A + 1))]:
        assert _refused(L.lutgemm_adapt, *{**good, **change}.values()) == E, change
    for change in [dict(flags=2), dict(flags=8), dict(tokens=65537)]:
        assert _refused(L.lutgemm_adapt, *{**good, **change}.values()) == U, change
    need = L.lutgemm_adapt_workspace_bytes(_adapters(), 3)
    assert need > 32768 and _refused(L.lutgemm_adapt, *{**good, "nbytes": need - 1}.values()) == W


@pytest.mark.parametrize("tokens", [1, 3, 32, 64, 65, 256, 257, 300, 4096, 65536])
@pytest.mark.parametrize("count,rank,m,n", [(1, 8, 1, 8), (3, 16, 5000, 5120), (64, 64, 12288, 12288), (1024, 256, 49152, 1 << 20)])
def test_a_plan_covers_everything(tokens, count, rank, m, n):
    a = _adapters(m=m, n=n, count=count, rank=rank)
    tile, tiles, parts, part, rows = L.lutgemm_plan_adapt(a, tokens)
    assert tile in (16, 32, 64) and rows % 256 == 0
    assert part % 256 == 0 and part * parts >= n > part * (parts - 1)
    # the most tiles that an assignment of tokens to adapters (or to none) can need: every group ends in a tile of one token
    groups = min(count + 1, tokens)
    assert tiles == groups + (tokens - groups) // tile
    floats = parts * tiles * tile * rank
    table = 0 if tokens <= 256 else 4 + (4 + tile) * tiles
    pad = next(r for r in (32, 64, 128, 256) if r >= rank)
    joined = tiles * tile * (pad + 1) if tokens > 256 or (tokens > 64 and tile == 64) else 0
    assert L.lutgemm_adapt_workspace_bytes(a, tokens) == 32768 + 4 * (table + floats + joined)
    assert tiles <= 65535 and 32768 + 4 * floats < 1 << 40
