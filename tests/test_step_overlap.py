"""CPU checks of outputs over inputs, which lutgemm_adapt and lutgemm_rms_norm refuse before any GPU call."""
import pytest

import paper_2206_09557_amd as L

A = 1 << 20      # an aligned address that nothing reads: every call below is refused
FAR = A + (1 << 16)
E, U = L.LUTGEMM_EINVAL, L.LUTGEMM_EUNSUPPORTED


def _refused(call, *args):
    with pytest.raises(L.LutGemmError) as e:
        call(*args)
    return e.value.code


def _adapt(**change):
    """Three tokens of 64 values beside a product of 96: rows of 128, 192 and 192 bytes (384 in fp32)."""
    adapters = L.lutgemm_adapters(2 * A, 3 * A, None, None, 96, 64, 3, 16)
    g = dict(x=A, base=FAR, adapters=adapters, of=4 * A, owner=None, y=FAR, tokens=3, seqs=0, xs=64, bs=96, ys=96, flags=0, ws=5 * A, nbytes=1 << 20)
    return _refused(L.lutgemm_adapt, *{**g, **change}.values())


@pytest.mark.parametrize("change", [
    dict(y=FAR + 2), dict(y=FAR - 190), dict(y=FAR + 3 * 192 - 2), dict(y=FAR + 96, bs=128, ys=128),          # into base: rows, its last one, a gap too small
    dict(y=FAR + 192, bs=192, ys=128), dict(y=FAR + 576, bs=384, ys=100), dict(y=FAR + 384, bs=96, ys=1 << 20),     # rows of other strides that meet
    dict(y=FAR + 2 * 384 + 380, bs=192, ys=96, flags=L.LUTGEMM_Y_F32),
    dict(y=A), dict(y=A, base=A), dict(y=A + 2 * 128 + 126), dict(y=A - 2), dict(y=A + 128, xs=128, ys=128),                      # into x
    dict(x=FAR + 192), dict(y=A + 64, ys=1 << 30)], ids=str)
def test_adapters_results_over_inputs(change):
    assert _adapt(**change) == E


@pytest.mark.parametrize("change", [dict(xs=1 << 41), dict(bs=(1 << 40) + 1, ys=(1 << 40) + 1), dict(ys=1 << 62, y=2 * FAR), dict(bs=(1 << 63) - 1, y=2 * FAR)], ids=str)
def test_strides_beyond_what_offsets_hold(change):
    assert _adapt(**change) == U
