"""GPU parity of lutgemm_rope with the 64-bit oracle, its gradient, and its refusals."""
import numpy as np
import pytest

import paper_2206_09557_amd as L
from oracle import kv_oracle as K

from gpu_util import torch_cuda

pytestmark = pytest.mark.gpu


def _call(x, positions, turns, heads, dim, rot, x_stride, y_stride, flags, amplitude=1.0, in_place=False, offset=0):
    """x [tokens][x_stride] numpy; returns y [tokens][y_stride], pre-filled with a mark."""
    torch = torch_cuda()
    tokens = x.shape[0]
    flat = np.concatenate([np.zeros(offset, x.dtype), x.reshape(-1)])
    d_x = torch.from_numpy(flat).cuda()[offset:]
    d_y = d_x if in_place else torch.full((tokens * y_stride + offset,), 77.0, dtype=d_x.dtype, device="cuda")[offset:]
    d_p = torch.from_numpy(np.asarray(positions, np.int32)).cuda()
    d_t = torch.from_numpy(turns.view(np.int64)).cuda()
    L.lutgemm_rope(d_x, d_y, d_p, d_t, tokens, heads, dim, rot, x_stride, y_stride, amplitude, flags,
                   torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    return d_y.cpu().numpy().reshape(tokens, y_stride)


def _check(y, ref, f32, amplitude):
    # sin and cos: series 3e-8, angle 2^-32 of a turn and its fp32 form 2^-25 of an eighth, 1e-7 in all; two products and a sum of
    # fp32.  A result is at most amplitude * sqrt(2) * |pair|; 4e-7 of that, plus the rounding of the type.
    size = amplitude * 2 * np.abs(ref).max()
    bound = 4e-7 * size + (0 if f32 else 2.0 ** -11 * np.abs(ref) + 2.0 ** -25)
    err = np.abs(y.astype(np.float64) - ref)
    assert (err <= bound).all(), (err - bound).max()


@pytest.mark.parametrize("tokens,heads,dim,rot,neighbours,transpose,f32,gap,start,amplitude", [
    (1, 1, 2, 2, False, False, False, 0, 1, 1.0),
    (1, 128, 128, 128, False, False, False, 0, 4095, 1.0),
    (3, 5, 128, 64, True, False, False, 8, -7, 1.0),
    (67, 9, 96, 24, False, False, False, 0, 1 << 20, 1.25),        # halves of 12: single pairs
    (2, 40, 128, 128, False, True, True, 4, 999983, 1.0),
    (5, 3, 64, 64, True, True, True, 3, 2147483000, 0.5),          # rows that begin anywhere
    (4, 2, 192, 48, True, False, False, 2, 77, 1.0),
    (1, 7, 512, 512, False, False, True, 1, 12, 1.0),
    (300, 72, 128, 128, False, False, False, 1024, 100000, 1.0),
    (9, 2, 66, 22, False, False, False, 0, 5, 1.0)])
def test_against_oracle(tokens, heads, dim, rot, neighbours, transpose, f32, gap, start, amplitude):
    rng = np.random.default_rng(tokens * 131 + dim)
    dt = np.float32 if f32 else np.float16
    x = rng.standard_normal((tokens, heads * dim + gap)).astype(dt)
    positions = (start + np.arange(tokens) * 3) % (1 << 31)
    turns = L.lutgemm_rope_frequencies(rot, scaling=L.LUTGEMM_ROPE_PARTS, factor=8.0, trained=8192.0)
    flags = (L.LUTGEMM_Y_F32 if f32 else 0) | (L.LUTGEMM_ROPE_NEIGHBOURS if neighbours else 0) | (L.LUTGEMM_ROPE_TRANSPOSE if transpose else 0)
    few = np.unique([0, tokens // 2, tokens - 1])
    ref = K.rope(x[few, :heads * dim].reshape(-1, heads, dim), positions[few], turns, rot, neighbours, transpose, amplitude)
    for in_place in (False, True):
        y_stride = x.shape[1] if in_place else heads * dim + 2 * (gap % 8)
        for offset in ((0, 1) if tokens < 10 else (0,)):
            print("case rope", tokens, heads, dim, rot, neighbours, transpose, f32, gap, in_place, offset, flush=True)
            y = _call(x, positions, turns, heads, dim, rot, x.shape[1], y_stride, flags, amplitude, in_place, offset)
            _check(y[few, :heads * dim].reshape(ref.shape), ref, f32, amplitude)
            # what is not turned is copied bit for bit; what is between rows stays
            same = y[:, :heads * dim].reshape(tokens, heads, dim)[..., rot:]
            assert (same == x[:, :heads * dim].reshape(tokens, heads, dim)[..., rot:]).all()
            rest = y[:, heads * dim:]
            assert (rest == (x[:, heads * dim:] if in_place else 77)).all()


def test_gradient_is_the_transpose_and_the_differences():
    tokens, heads, dim, rot, amplitude = 3, 2, 64, 32, 1.5
    rng = np.random.default_rng(5)
    x = rng.standard_normal((tokens, heads * dim)).astype(np.float32)
    w = rng.standard_normal((tokens, heads * dim)).astype(np.float32)     # loss = sum(w * rope(x))
    positions, turns = [3, 1000, 70000], L.lutgemm_rope_frequencies(rot)

    def f(v, flags):
        return _call(v, positions, turns, heads, dim, rot, heads * dim, heads * dim, L.LUTGEMM_Y_F32 | flags, amplitude).astype(np.float64)

    for flags in (0, L.LUTGEMM_ROPE_NEIGHBOURS):
        grad = f(w, flags | L.LUTGEMM_ROPE_TRANSPOSE)
        for t, i in [(0, 0), (1, 15), (1, 16), (2, 31), (2, 32), (0, 64 + 7), (1, 127)]:
            up, down = x.copy(), x.copy()
            up[t, i] += 0.5
            down[t, i] -= 0.5
            step = float(up[t, i]) - float(down[t, i])
            diff = ((f(up, flags) - f(down, flags)) * w).sum() / step
            # linear: the quotient is off by the roundings of the two results alone, two values near 4 of 24 bits each
            assert abs(diff - grad[t, i]) <= 4e-6
    # amplitude 1: turning back undoes it
    y = _call(x, positions, turns, heads, dim, rot, heads * dim, heads * dim, L.LUTGEMM_Y_F32)
    back = _call(y, positions, turns, heads, dim, rot, heads * dim, heads * dim, L.LUTGEMM_Y_F32 | L.LUTGEMM_ROPE_TRANSPOSE)
    assert np.abs(back - x).max() <= 4e-6


def test_nothing_to_do():
    torch = torch_cuda()
    d = torch.full((64,), 3.0, dtype=torch.float16, device="cuda")
    t = torch.zeros(32, dtype=torch.int64, device="cuda")
    L.lutgemm_rope(d, d, t, t, 0, 1, 64, 64, 64, 64, 1.0, 0, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert (d == 3).all()
