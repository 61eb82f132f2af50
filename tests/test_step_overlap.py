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


def _norm(**change):
    """Three rows of 64 values in 128 bytes, and in 64 with two scales each."""
    g = dict(x=A, residual=2 * A, weight=3 * A, sum=4 * A, y=5 * A, scales=6 * A, tokens=3, n=64, group=32, xs=64, ss=64, ys=64, eps=1e-5, flags=0)
    return _refused(L.lutgemm_rms_norm, *{**g, **change}.values())


@pytest.mark.parametrize("change", [
    dict(scales=A), dict(scales=A + 3 * 128 - 4), dict(scales=A - 20), dict(scales=2 * A + 256), dict(scales=3 * A), dict(scales=3 * A + 124),
    dict(scales=4 * A + 380), dict(scales=5 * A), dict(scales=5 * A + 188), dict(scales=5 * A - 20), dict(scales=5 * A + 60, ys=1 << 20), dict(scales=5 * A + 64, ys=80),
    dict(scales=2 * A + 128, ss=74), dict(weight=5 * A), dict(weight=5 * A + 190), dict(weight=5 * A - 126), dict(weight=4 * A), dict(weight=4 * A + 200),
    dict(weight=4 * A + 128, ss=100), dict(weight=5 * A + 382, scales=None, group=0), dict(weight=4 * A + 764, flags=L.LUTGEMM_NORM_STREAM_F32)], ids=str)
def test_norms_outputs_over_scales_and_weights(change):
    assert _norm(**change) == E
