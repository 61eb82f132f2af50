"""GPU parity of lutgemm_rms_norm with the 64-bit oracle: types, strides, alignments, outputs in place, 8 bits with scales."""
import numpy as np
import pytest

import paper_2206_09557_amd as L
from oracle import step_oracle as S

from gpu_util import torch_cuda

pytestmark = pytest.mark.gpu

EPS = 1e-5
MARK = 77


def _dtype(f32):
    return np.float32 if f32 else np.float16


def _rows(rng, tokens, n, stride, f32, loud=1.0):
    x = (rng.standard_normal((tokens, stride)) * loud).astype(_dtype(f32))
    x[:, rng.integers(0, n, 2)] *= 20
    return x


def _up(x, offset=0):
    """On the device, `offset` elements behind a place of 256 bytes' alignment, as one flat buffer with as many behind it."""
    torch = torch_cuda()
    flat = np.full(x.size + 2 * offset, MARK, x.dtype)
    flat[offset:offset + x.size] = x.reshape(-1)
    return torch.from_numpy(flat).cuda()[offset:]


def _down(t, like, stride):
    return t.cpu().numpy()[:like * stride].reshape(like, stride)


def _call(x, r, w, sum_, y, scales, tokens, n, group, xs, ss, ys, flags, eps=EPS):
    torch = torch_cuda()
    L.lutgemm_rms_norm(x, r, w, sum_, y, scales, tokens, n, group, xs, ss, ys, eps, flags, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()


def _check_y(y, ref):
    # s, the root, its product with s and with the weight: five roundings of fp32 at most, and one to fp16 (of a number so close to
    # the exact one that it may fall on the other side of a middle)
    bound = (2.0 ** -11 + 6 * 2.0 ** -24) * np.abs(ref) + 2.0 ** -25
    err = np.abs(y.astype(np.float64) - ref)
    assert (err <= bound).all(), (err - bound).max()


def _check_sum(got, s, f32):
    bound = 2.0 ** -24 * np.abs(s) * (1.0 if f32 else 1.01) + (2.0 ** -149 if f32 else 2.0 ** -11 * np.abs(s) + 2.0 ** -25)
    assert (np.abs(got.astype(np.float64) - s) <= bound).all()


@pytest.mark.parametrize("tokens,n,x_f32,stream_f32,gaps,offset,parts", [
    (1, 1, False, False, (0, 0, 0), 0, "rws"), (1, 8, False, False, (0, 0, 0), 0, "rws"), (3, 7, True, False, (1, 2, 3), 1, "rws"),
    (2, 63, False, True, (0, 0, 0), 0, "rw"), (5, 64, False, False, (8, 8, 8), 0, "rws"), (1, 512, True, True, (0, 0, 0), 0, "ws"),
    (4, 520, False, False, (0, 0, 0), 0, ""), (7, 2048, True, False, (8, 16, 24), 0, "rs"), (3, 2049, False, True, (0, 0, 0), 0, "rws"),
    (2, 2056, False, False, (0, 0, 0), 4, "rws"), (9, 4096, False, True, (0, 8, 0), 0, "rws"), (2, 5003, True, True, (21, 21, 0), 0, "rws"),
    (1, 5120, False, False, (0, 0, 0), 0, "w"), (3, 8192, True, True, (0, 0, 0), 0, "rws"), (2, 8200, False, False, (0, 0, 0), 0, "rws"),
    (1, 12288, False, False, (0, 0, 0), 0, "rws"), (2, 12289, False, False, (0, 0, 0), 0, "rws"), (2, 16384, True, False, (0, 0, 0), 0, "rws"),
    (2, 16392, False, True, (0, 0, 0), 0, "rws"), (1, 32768, False, False, (0, 0, 0), 0, "rws"), (2, 32767, True, True, (1, 0, 3), 0, "rws"),
    (700, 1032, False, False, (0, 0, 8), 0, "rws")])
def test_against_oracle(tokens, n, x_f32, stream_f32, gaps, offset, parts):
    print("case norm", tokens, n, x_f32, stream_f32, gaps, offset, parts, flush=True)
    rng = np.random.default_rng(tokens * 7 + n)
    xs, ss, ys = (n + g for g in gaps)
    x, r = _rows(rng, tokens, n, xs, x_f32), _rows(rng, tokens, n, ss, stream_f32, 3.0) if "r" in parts else None
    w = (1 + 0.2 * rng.standard_normal(n)).astype(np.float16) if "w" in parts else None
    s, ref = S.rms_norm(x[:, :n], None if r is None else r[:, :n], w, EPS)
    d_sum = _up(np.full((tokens, ss), MARK, _dtype(stream_f32)), offset) if "s" in parts else None
    d_y = _up(np.full((tokens, ys), MARK, np.float16), offset)
    flags = (L.LUTGEMM_Y_F32 if x_f32 else 0) | (L.LUTGEMM_NORM_STREAM_F32 if stream_f32 else 0)
    args = (_up(x, offset), None if r is None else _up(r, offset), None if w is None else _up(w, offset))
    _call(*args, d_sum, d_y, None, tokens, n, 0, xs, ss, ys, flags)
    y = _down(d_y, tokens, ys)
    _check_y(y[:, :n], ref)
    assert (y[:, n:] == MARK).all() and (d_y.cpu().numpy()[tokens * ys:] == MARK).all()
    if d_sum is not None:
        got = _down(d_sum, tokens, ss)
        _check_sum(got[:, :n], s, stream_f32)
        assert (got[:, n:] == MARK).all() and (d_sum.cpu().numpy()[tokens * ss:] == MARK).all()
    again = _up(np.full((tokens, ys), MARK, np.float16), offset)
    _call(*args, d_sum, again, None, tokens, n, 0, xs, ss, ys, flags)
    np.testing.assert_array_equal(again.cpu().numpy(), d_y.cpu().numpy())


@pytest.mark.parametrize("x_f32,stream_f32", [(False, False), (True, False), (False, True), (True, True)])
def test_every_width(x_f32, stream_f32):
    """Rows of every number of runs and threads, whole 16 bytes and not, few and many of them, to fp16 and to 8 bits."""
    torch = torch_cuda()
    rng = np.random.default_rng(6 + x_f32 + 2 * stream_f32)
    flags = (L.LUTGEMM_Y_F32 if x_f32 else 0) | (L.LUTGEMM_NORM_STREAM_F32 if stream_f32 else 0)
    for n in (504, 512, 520, 1024, 1056, 2048, 4096, 4104, 6144, 6176, 8192, 8224, 12320, 16384, 16416, 24576, 24608, 32768):
        for tokens, gap in ((3, 0), (3, 1), (1030, 0)):
            if tokens * n > 1 << 24:
                continue
            print("case width", n, tokens, gap, x_f32, stream_f32, flush=True)
            stride = n + gap
            x, r = _rows(rng, tokens, n, stride, x_f32), _rows(rng, tokens, n, stride, stream_f32, 3.0)
            d_x, d_r, d_y = _up(x), _up(r), _up(np.full((tokens, stride), MARK, np.float16))
            few = np.unique([0, tokens // 2, tokens - 1])
            s, ref = S.rms_norm(x[few, :n], r[few, :n], None, EPS)
            _call(d_x, d_r, None, d_r, d_y, None, tokens, n, 0, stride, stride, stride, flags)
            y = _down(d_y, tokens, stride)
            _check_y(y[few, :n], ref)
            assert (y[:, n:] == MARK).all()
            _check_sum(_down(d_r, tokens, stride)[few, :n], s, stream_f32)
            if n % 32:
                continue
            codes, scales = _up(np.full((tokens, stride), MARK, np.int8)), torch.empty(tokens, n // 32, device="cuda")
            _call(d_x, _up(r), None, None, codes, scales, tokens, n, 32, stride, stride, stride, flags)
            steps = scales.cpu().numpy()[few].repeat(32, 1).astype(np.float64)
            y = _down(codes, tokens, stride)
            assert (np.abs(y[few, :n] * steps - ref) <= steps * (0.5 + 127 * 8 * 2.0 ** -24)).all() and (y[:, n:] == MARK).all()


@pytest.mark.parametrize("tokens,n,group,x_f32,stream_f32,gap,offset", [
    (1, 32, 32, False, False, 0, 0), (3, 96, 32, False, False, 0, 0), (2, 1, 0, False, False, 0, 0), (5, 77, 0, True, True, 3, 1), (4, 2048, 64, False, True, 0, 0),
    (509, 1024, 128, False, True, 0, 0), (2, 8192, 128, False, True, 8, 0), (3, 5120, 0, False, False, 0, 0), (2, 12288, 96, True, False, 0, 0),
    (1, 32768, 32, False, False, 0, 0), (2, 1536, 512, False, False, 4, 3), (2, 20000, 0, False, False, 0, 0), (1, 32736, 1056, True, True, 0, 0)])
def test_eight_bits(tokens, n, group, x_f32, stream_f32, gap, offset):
    print("case norm8", tokens, n, group, x_f32, stream_f32, gap, offset, flush=True)
    torch = torch_cuda()
    rng = np.random.default_rng(tokens + n)
    stride, g = n + gap, group or n
    x, r = _rows(rng, tokens, n, stride, x_f32), _rows(rng, tokens, n, stride, stream_f32, 3.0)
    w = (1 + 0.2 * rng.standard_normal(n)).astype(np.float16)
    if n // g > 1:
        w[:g] = 0                              # a group of zeros
    _, ref = S.rms_norm(x[:, :n], r[:, :n], w, EPS)
    d_y = _up(np.full((tokens, stride), MARK, np.int8), offset)
    d_scales = torch.full((tokens * (n // g) + 2,), float(MARK), device="cuda")
    flags = (L.LUTGEMM_Y_F32 if x_f32 else 0) | (L.LUTGEMM_NORM_STREAM_F32 if stream_f32 else 0)
    _call(_up(x, offset), _up(r, offset), _up(w), None, d_y, d_scales, tokens, n, group, stride, stride, stride, flags)
    y, scales = _down(d_y, tokens, stride), d_scales.cpu().numpy()
    assert (y[:, n:] == MARK).all() and (scales[-2:] == MARK).all() and np.abs(y[:, :n].astype(int)).max() <= 127
    scales = scales[:-2].reshape(tokens, n // g).astype(np.float64)
    ref = ref.reshape(tokens, n // g, g)
    exact = np.abs(ref).max(-1) / 127
    assert (np.abs(scales - exact) <= 7 * 2.0 ** -24 * exact).all()          # the five roundings of y, the division's
    # half a step, and what the roundings move a quotient of up to 127: five of y, one of 1 / scale's, one of the product
    bound = scales[..., None] * (0.5 + 127 * 8 * 2.0 ** -24)
    assert (np.abs(y[:, :n].reshape(ref.shape) * scales[..., None] - ref) <= bound).all()
    if n // g > 1:
        assert (scales[:, 0] == 0).all() and (y[:, :g] == 0).all()


@pytest.mark.parametrize("x_f32,stream_f32", [(False, False), (True, False), (False, True), (True, True)])
def test_ends_of_rows(x_f32, stream_f32):
    """Rows that end anywhere in a run of eight, shorter ones too, that begin on any value's bytes: in place, and to 8 bits; what is behind a row stays."""
    torch = torch_cuda()
    rng = np.random.default_rng(60 + x_f32 + 2 * stream_f32)
    flags = (L.LUTGEMM_Y_F32 if x_f32 else 0) | (L.LUTGEMM_NORM_STREAM_F32 if stream_f32 else 0)
    for k, n in enumerate((1, 2, 5, 7, 8, 9, 11, 14, 15, 511, 513, 516, 519, 2047, 2050, 4101, 8191, 8193, 16387, 24577, 32761)):
        tokens, stride = 1030 if 500 < n < 3000 else 3, n + k % 4
        print("case ends", n, tokens, stride, x_f32, stream_f32, flush=True)
        x, r = _rows(rng, tokens, n, stride, x_f32), _rows(rng, tokens, n, stride, stream_f32, 3.0)
        w = (1 + 0.1 * rng.standard_normal(n)).astype(np.float16)
        d_x, d_r, d_y = _up(x), _up(r), _up(np.full((tokens, stride), MARK, np.float16))
        s, ref = S.rms_norm(x[:, :n], r[:, :n], w, EPS)
        _call(d_x, d_r, _up(w), d_r, d_y, None, tokens, n, 0, stride, stride, stride, flags)
        y = _down(d_y, tokens, stride)
        _check_y(y[:, :n], ref)
        assert (y[:, n:] == MARK).all()
        after = _down(d_r, tokens, stride)
        _check_sum(after[:, :n], s, stream_f32)
        np.testing.assert_array_equal(after[:, n:], r[:, n:])
        codes, scales = _up(np.full((tokens, stride), MARK, np.int8)), torch.empty(tokens, 1, device="cuda")
        _call(d_x, _up(r), _up(w), None, codes, scales, tokens, n, 0, stride, stride, stride, flags)
        steps = scales.cpu().numpy().astype(np.float64)
        y = _down(codes, tokens, stride)
        assert (np.abs(y[:, :n] * steps - ref) <= steps * (0.5 + 127 * 8 * 2.0 ** -24)).all() and (y[:, n:] == MARK).all()


def test_in_place():
    """sum over residual, y over x; sum over x where y goes elsewhere; y over the residual; rows side by side in one buffer."""
    torch = torch_cuda()
    rng = np.random.default_rng(5)
    tokens, n = 37, 1160
    for x_f32, stream_f32, where in [(False, False, "sum=r y=x"), (True, True, "sum=x"), (False, True, "sum=r"), (False, False, "y=r"), (False, False, "side")]:
        x, r = _rows(rng, tokens, n, n, x_f32), _rows(rng, tokens, n, n, stream_f32, 3.0)
        s, ref = S.rms_norm(x, r, None, EPS)
        flags = (L.LUTGEMM_Y_F32 if x_f32 else 0) | (L.LUTGEMM_NORM_STREAM_F32 if stream_f32 else 0)
        d_x, d_r = _up(x), _up(r)
        d_sum = d_r if "sum=r" in where else d_x if "sum=x" in where else None
        d_y = d_x if "y=x" in where else d_r if "y=r" in where else torch.empty(tokens, n, dtype=torch.float16, device="cuda")
        stride = n
        if where == "side":                # x, y, residual and sum are columns of one matrix
            both = torch.full((tokens, 4 * n), float(MARK), dtype=torch.float16, device="cuda")
            both[:, :n], both[:, 2 * n:3 * n] = d_x.view(tokens, n), d_r.view(tokens, n)
            d_x, d_y, d_r, d_sum, stride = both, both[:, n:], both[:, 2 * n:], both[:, 3 * n:], 4 * n
        _call(d_x, d_r, None, d_sum, d_y, None, tokens, n, 0, stride, stride, stride, flags)
        if where == "side":
            got = both.cpu().numpy()
            np.testing.assert_array_equal(got[:, :n], x)
            np.testing.assert_array_equal(got[:, 2 * n:3 * n], r)
            _check_y(got[:, n:2 * n], ref)
            _check_sum(got[:, 3 * n:], s, False)
            continue
        _check_y(d_y.cpu().numpy().reshape(tokens, n), ref)
        if d_sum is not None:
            _check_sum(d_sum.cpu().numpy().reshape(tokens, n), s, stream_f32)


def test_values_at_the_ends():
    """fp32 rows whose squares leave 32 bits, rows of zeros, the smallest numbers; infinities and NaNs stay in their rows."""
    torch = torch_cuda()
    rng = np.random.default_rng(8)
    n = 256
    x = rng.standard_normal((8, n)).astype(np.float32)
    x[0] *= np.float32(1e30)
    x[1] = 0
    x[2] *= np.float32(1e-30)
    x[3, 7] = np.inf
    x[4, 200] = np.nan
    x[5, 40] = -np.inf
    x[6] *= np.float32(1e-3)
    with np.errstate(invalid="ignore"):
        _, ref = S.rms_norm(x, None, None, EPS)
    d_y = torch.full((8, n), float(MARK), dtype=torch.float16, device="cuda")
    _call(_up(x), None, None, None, d_y, None, 8, n, 0, n, 0, n, L.LUTGEMM_Y_F32)
    y = d_y.cpu().numpy()
    for t in (0, 1, 2, 6, 7):
        _check_y(y[t], ref[t])
    for t, c in ((3, 7), (5, 40)):                     # an infinity over an infinite root is no number; the others vanish
        assert np.isnan(y[t, c]) and (np.delete(y[t], c) == 0).all()
    assert np.isnan(y[4]).all()
    codes, scales = torch.full((8, n), 1, dtype=torch.int8, device="cuda"), torch.empty(8, n // 32, device="cuda")
    _call(_up(x), None, None, None, codes, scales, 8, n, 32, n, 0, n, L.LUTGEMM_Y_F32)
    codes, scales = codes.cpu().numpy(), scales.cpu().numpy()
    for t, c in ((3, 7), (5, 40)):
        assert (np.isnan(scales[t]) == (np.arange(n // 32) == c // 32)).all() and (np.delete(scales[t], c // 32) == 0).all() and (codes[t] == 0).all()
    assert np.isnan(scales[4]).all() and (codes[4] == 0).all()
    assert (scales[1] == 0).all() and (codes[1] == 0).all()
    for t in (0, 6, 7):
        steps = scales[t].repeat(32).astype(np.float64)
        assert (np.abs(codes[t] * steps - ref[t]) <= steps * (0.5 + 127 * 8 * 2.0 ** -24)).all()
    assert (scales[2] == 0).all() == bool((np.abs(ref[2]).reshape(-1, 32).max(1) < 2.0 ** -100).all())


def test_many_rows_and_far_ones():
    """More rows than a grid's second side has; rows 2^28 elements apart, 2^32 bytes and more in all; large outputs in place."""
    torch = torch_cuda()
    x = torch.randn(70001, 16, device="cuda").half()
    y = torch.empty_like(x)
    _call(x, None, None, None, y, None, 70001, 16, 0, 16, 0, 16, 0)
    _check_y(y.cpu().numpy(), S.rms_norm(x.cpu().numpy(), None, None, EPS)[1])
    rng = np.random.default_rng(3)
    n, stride = 136, 1 << 28
    rows = rng.standard_normal((9, n)).astype(np.float16)
    far = torch.empty(8 * stride + n, dtype=torch.float16, device="cuda")
    for t in range(9):
        far[t * stride:t * stride + n] = torch.from_numpy(rows[t]).cuda()
    _call(far, None, None, None, far, None, 9, n, 0, stride, 0, stride, 0)
    got = np.stack([far[t * stride:t * stride + n].cpu().numpy() for t in range(9)])
    _check_y(got, S.rms_norm(rows, None, None, EPS)[1])
    del far
    x = rng.standard_normal((3000, 5120)).astype(np.float16)
    r = rng.standard_normal((3000, 5120)).astype(np.float32)
    d_x, d_r = _up(x), _up(r)
    _call(d_x, d_r, None, d_r, d_x, None, 3000, 5120, 0, 5120, 5120, 5120, L.LUTGEMM_NORM_STREAM_F32)
    few = [0, 1, 1499, 2999]
    s, ref = S.rms_norm(x[few], r[few], None, EPS)
    _check_y(d_x.cpu().numpy().reshape(3000, 5120)[few], ref)
    _check_sum(d_r.cpu().numpy().reshape(3000, 5120)[few], s, True)


def test_a_captured_norm_is_replayed():
    torch = torch_cuda()
    n = 1000
    x, r = torch.randn(5, n, device="cuda").half(), torch.zeros(5, n, device="cuda")
    codes, scales = torch.empty(5, n, dtype=torch.int8, device="cuda"), torch.empty(5, 1, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        L.lutgemm_rms_norm(x, r, None, r, codes, scales, 5, n, 0, n, n, n, EPS, L.LUTGEMM_NORM_STREAM_F32, torch.cuda.current_stream().cuda_stream)
    total = np.zeros((5, n))
    for _ in range(4):
        x.normal_()
        graph.replay()
        torch.cuda.synchronize()
        s, ref = S.rms_norm(x.cpu().numpy(), total.astype(np.float32), None, EPS)
        _check_sum(r.cpu().numpy(), s, True)
        steps = scales.cpu().numpy().astype(np.float64)
        assert (np.abs(codes.cpu().numpy() * steps - ref) <= steps * (0.5 + 127 * 8 * 2.0 ** -24)).all()
        total = r.cpu().numpy().astype(np.float64)


def test_nothing_to_do_and_another_stream():
    torch = torch_cuda()
    n = 640
    x = torch.randn(6, n, device="cuda").half()
    y = torch.full((6, n), float(MARK), dtype=torch.float16, device="cuda")
    L.lutgemm_rms_norm(x, None, None, None, y, None, 0, n, 0, n, 0, n, EPS, 0, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert (y == MARK).all()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    L.lutgemm_rms_norm(x, None, None, None, y, None, 6, n, 0, n, 0, n, EPS, 0, side.cuda_stream)
    side.synchronize()
    _check_y(y.cpu().numpy(), S.rms_norm(x.cpu().numpy(), None, None, EPS)[1])
