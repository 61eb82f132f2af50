"""GPU checks of where outputs of lutgemm_adapt and lutgemm_rms_norm may stand: next to inputs, between their rows, and refused on any byte of them."""
import numpy as np
import pytest

import paper_2206_09557_amd as L
from oracle import step_oracle as S

from gpu_util import make_workspace, torch_cuda
import test_gpu_adapt as A

pytestmark = pytest.mark.gpu

ROOM = 4096      # bytes that everything stands in


def _bytes(at, rows, stride, n, size):
    """The bytes of a matrix whose first value is `at` values behind the beginning."""
    return {b for t in range(rows) for b in range((at + t * stride) * size, (at + t * stride + n) * size)}


def _draw(rng, rows, n, size, eights=False):
    """(at, stride) of rows that end within the room."""
    step = 8 if eights else 1
    stride = n + step * int(rng.integers(0, 12)) if rng.random() < 0.7 else 24 * int(rng.integers(1, 4))
    return step * int(rng.integers(0, (ROOM // size - rows * stride) // step)), stride


def test_adapters_results_next_to_what_they_read():
    """x, base and y anywhere in one buffer: refused if and only if y has a byte of x or base, else right, with everything else as it was."""
    torch = torch_cuda()
    rng = np.random.default_rng(5)
    m, n, rank = 20, 16, 8
    a = A.Set(rng, m, n, 2, rank)
    ws = make_workspace(L.lutgemm_adapt_workspace_bytes(a.handle, 5))
    taken = {True: 0, False: 0}
    for k in range(500):
        tokens, f32 = int(rng.integers(1, 6)), bool(rng.integers(2))
        size, dt = (4, np.float32) if f32 else (2, np.float16)
        (x_at, xs), (b_at, bs), (y_at, ys) = _draw(rng, tokens, n, 2, True), _draw(rng, tokens, m, size), _draw(rng, tokens, m, size)
        if k % 3 == 0:                             # side by side, or nearly
            bs = ys = 2 * m + int(rng.integers(0, 3))
            b_at = int(rng.integers(0, ROOM // size - (tokens + 1) * bs))
            y_at = b_at + m + int(rng.integers(-1, 3))
        xb, bb, yb = _bytes(x_at, tokens, xs, n, 2), _bytes(b_at, tokens, bs, m, size), _bytes(y_at, tokens, ys, m, size)
        if xb & bb or (b_at, size) == (y_at, size):
            continue
        held = np.full(ROOM + 64, 0x3c, np.uint8)
        x, base = rng.standard_normal((tokens, n)).astype(np.float16), rng.standard_normal((tokens, m)).astype(dt)
        for t in range(tokens):
            held[:ROOM].view(np.float16)[x_at + t * xs:x_at + t * xs + n] = x[t]
            held[:ROOM].view(dt)[b_at + t * bs:b_at + t * bs + m] = base[t]
        room = torch.from_numpy(held).cuda()
        of = torch.arange(tokens, dtype=torch.int32, device="cuda") % 3 - 1
        address = room.data_ptr()
        args = (address + 2 * x_at, address + size * b_at, a.handle, of, None, address + size * y_at, tokens, 0, xs, bs, ys, L.LUTGEMM_Y_F32 if f32 else 0, ws, ws.numel(),
                torch.cuda.current_stream().cuda_stream)
        fine = not yb & (xb | bb)
        taken[fine] += 1
        if fine:
            L.lutgemm_adapt(*args)
        else:
            with pytest.raises(L.LutGemmError) as e:
                L.lutgemm_adapt(*args)
            assert e.value.code == L.LUTGEMM_EINVAL
        torch.cuda.synchronize()
        after = room.cpu().numpy()
        others = np.ones(ROOM + 64, bool)
        if fine:
            y = np.stack([after[:ROOM].view(dt)[y_at + t * ys:y_at + t * ys + m] for t in range(tokens)])
            A._check(y, *S.adapt(x, base, a.down, a.up, None, a.scales, of.tolist()), f32, n, rank)
            others[list(yb)] = False
        np.testing.assert_array_equal(after[others], held[others])
    assert min(taken.values()) > 100, taken
