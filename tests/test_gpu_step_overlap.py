"""GPU checks of where outputs of lutgemm_adapt and lutgemm_rms_norm may stand: next to inputs, between their rows, and refused on any byte of them."""
import numpy as np
import pytest

import paper_2206_09557_amd as L
from oracle import step_oracle as S

from gpu_util import make_workspace, torch_cuda
import test_gpu_adapt as A
import test_gpu_rms_norm as N

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


def test_norms_outputs_next_to_what_they_read():
    """x, residual, weight, sum, y and scales anywhere in one buffer: refused if and only if an output has a byte that it may not have, else right."""
    torch = torch_cuda()
    rng = np.random.default_rng(6)
    eps, n = 1e-5, 32
    taken = {True: 0, False: 0}
    for k in range(900):
        tokens, bits8 = int(rng.integers(1, 5)), bool(rng.integers(2))
        x_f32, s_f32 = bool(rng.integers(2)), bool(rng.integers(2))
        sizes = {"x": 4 if x_f32 else 2, "residual": 4 if s_f32 else 2, "sum": 4 if s_f32 else 2, "y": 1 if bits8 else 2, "weight": 2, "scales": 4}
        at, stride = {}, {}
        for name in ("x", "residual", "y"):
            at[name], stride[name] = _draw(rng, tokens, n, sizes[name])
        stride["sum"] = stride["residual"]
        at["sum"] = at["residual"] if k % 4 == 0 else int(rng.integers(0, ROOM // sizes["sum"] - tokens * stride["sum"]))
        if k % 4 == 1 and sizes["y"] == sizes["x"]:
            at["y"], stride["y"] = at["x"], stride["x"]
        at["weight"], at["scales"] = int(rng.integers(0, ROOM // 2 - n)), int(rng.integers(0, ROOM // 4 - tokens))
        used = [name for name in at if bits8 or name != "scales"]
        mine = {name: _bytes(at[name], 1, 0, {"weight": n, "scales": tokens}[name], sizes[name]) if name in ("weight", "scales") else
                _bytes(at[name], tokens, stride[name], n, sizes[name]) for name in used}
        if mine["x"] & mine["residual"] or mine["weight"] & (mine["x"] | mine["residual"]):
            continue

        def same(a, b):
            return at[a] == at[b] and sizes[a] == sizes[b] and (stride[a] == stride[b] or tokens == 1)

        fine = min(stride.values()) >= n and all(      # (rows do not overlap those of their own matrix either)
            not mine[i] & mine[o] or (o in ("sum", "y") and i in ("x", "residual") and same(i, o))
            for o in used if o in ("sum", "y", "scales") for i in ("x", "residual", "weight"))
        outs = [o for o in used if o in ("sum", "y", "scales")]
        fine = fine and all(not mine[a] & mine[b] for a in outs for b in outs if a < b)
        held = np.full(ROOM + 64, 0x3c, np.uint8)
        kinds = {1: np.int8, 2: np.float16, 4: np.float32}
        x, r = rng.standard_normal((tokens, n)).astype(kinds[sizes["x"]]), rng.standard_normal((tokens, n)).astype(kinds[sizes["residual"]])
        w = (1 + 0.1 * rng.standard_normal(n)).astype(np.float16)

        def rows(buffer, name):
            v = buffer[:ROOM].view(kinds[sizes[name]])
            return [v[at[name] + t * stride[name]:][:n] for t in range(tokens)]

        for t in range(tokens):
            rows(held, "x")[t][:], rows(held, "residual")[t][:] = x[t], r[t]
        held[:ROOM].view(np.float16)[at["weight"]:][:n] = w
        room = torch.from_numpy(held).cuda()
        p = {name: room.data_ptr() + at[name] * sizes[name] for name in at}
        args = (p["x"], p["residual"], p["weight"], p["sum"], p["y"], p["scales"] if bits8 else None, tokens, n, 0, stride["x"], stride["sum"], stride["y"], eps,
                (L.LUTGEMM_Y_F32 if x_f32 else 0) | (L.LUTGEMM_NORM_STREAM_F32 if s_f32 else 0), torch.cuda.current_stream().cuda_stream)
        taken[fine] += 1
        if fine:
            L.lutgemm_rms_norm(*args)
        else:
            with pytest.raises(L.LutGemmError) as e:
                L.lutgemm_rms_norm(*args)
            assert e.value.code == L.LUTGEMM_EINVAL
        torch.cuda.synchronize()
        after = room.cpu().numpy()
        others = np.ones(ROOM + 64, bool)
        if fine:
            s, ref = S.rms_norm(x, r, w, eps)
            N._check_sum(np.stack(rows(after, "sum")), s, s_f32)
            y = np.stack(rows(after, "y"))
            if bits8:
                steps = after[:ROOM].view(np.float32)[at["scales"]:][:tokens, None].astype(np.float64)
                assert (np.abs(y * steps - ref) <= steps * (0.5 + 127 * 8 * 2.0 ** -24)).all()
            else:
                N._check_y(y, ref)
            for o in outs:
                others[list(mine[o])] = False
        np.testing.assert_array_equal(after[others], held[others])
    assert min(taken.values()) > 100, taken
