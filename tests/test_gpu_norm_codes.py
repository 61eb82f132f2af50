"""GPU checks of lutgemm_rms_norm's 8 bits at the ends of what the header promises: the quotient's bound, and scales next to 2^-100."""
import numpy as np
import pytest

import paper_2206_09557_amd as L

from gpu_util import torch_cuda

pytestmark = pytest.mark.gpu


def _codes(x, weight, group, eps):
    """Codes [tokens][n], scales [tokens][groups] of fp32 rows."""
    torch = torch_cuda()
    tokens, n = x.shape
    codes, scales = torch.full((tokens, n), 99, dtype=torch.int8, device="cuda"), torch.empty(tokens, n // (group or n), device="cuda")
    L.lutgemm_rms_norm(torch.from_numpy(x).cuda(), None, None if weight is None else torch.from_numpy(weight).cuda(), None, codes, scales, tokens, n, group, n, 0, n, eps,
                       L.LUTGEMM_Y_F32, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    return codes.cpu().numpy(), scales.cpu().numpy()


@pytest.mark.parametrize("n,group", [(1024, 32), (4096, 128), (2048, 0), (2050, 0)])
def test_the_quotients_bound(n, group):
    """Rows whose mean square is a half, eps the other half: the root is 1, so that y is x and a code is that of a quotient known exactly."""
    rng = np.random.default_rng(n)
    x = rng.standard_normal((1000, n))
    x = (x / np.sqrt(2 * (x * x).mean(1, keepdims=True))).astype(np.float32)
    # 1 / sqrt(1 + d) rounds to 1 while |d| / 2 is under half a step below it, 2^-25
    assert np.abs((x.astype(np.float64) ** 2).mean(1) - 0.5).max() < 2.0 ** -25
    codes, scales = _codes(x, None, group, 0.5)
    g = group or n
    top = np.abs(x).reshape(len(x), -1, g).max(2).astype(np.float64)
    assert (np.abs(scales - top / 127) <= 2.0 ** -24 * top / 127).all()
    quotient = x.astype(np.float64) / scales.astype(np.float64).repeat(g, 1)
    # three roundings: of the scale, of its inverse, of the product; of three together a little over the sum
    assert (np.abs(codes - quotient) <= 0.5 + 3.001 * 2.0 ** -24 * np.abs(quotient)).all()
    assert np.abs(codes.astype(int)).max() == 127


@pytest.mark.parametrize("group,n", [(32, 128), (0, 100)])
def test_scales_next_to_the_least(group, n):
    """Groups whose largest is just below 2^-100 have a scale of zero and codes of zero, from 2^-100 on they have both; eps of 1 makes the root 1."""
    least, rng = np.float32(2.0 ** -100), np.random.default_rng(n)
    tops = np.array([least, np.nextafter(least, np.float32(0)), np.nextafter(least, np.float32(1)), least / 2, least * 3, 2.0 ** -126, 2.0 ** -149, 0, 2.0 ** -90], np.float32)
    g = group or n
    top = rng.permutation(np.tile(tops, 4 * n // g)).reshape(-1, n // g)
    x = (rng.uniform(-1, 1, (*top.shape, g)) * top[..., None]).astype(np.float32)
    x[..., 5] = -top                                # (products with less than one, rounded, are no larger)
    codes, scales = _codes(x.reshape(len(top), n), None, group, 1.0)
    live = top >= least
    np.testing.assert_array_equal(scales == 0, ~live)
    assert (np.abs(scales[live] - top[live].astype(np.float64) / 127) <= 2.0 ** -24 * top[live].astype(np.float64) / 127).all()
    codes = codes.reshape(x.shape)
    assert (codes[~live] == 0).all() and (codes[live][:, 5] == -127).all()
    quotient = x[live].astype(np.float64) / scales[live].astype(np.float64)[:, None]
    assert (np.abs(codes[live] - quotient) <= 0.5 + 3.001 * 2.0 ** -24 * np.abs(quotient)).all()


@pytest.mark.parametrize("weight", [False, True])
def test_small_rows_under_the_usual_eps(weight):
    """Values near 1e-30, whose y are a few hundred times that: above 2^-100, so they have codes."""
    rng = np.random.default_rng(9)
    n, eps = 256, float(np.float32(1e-5))
    x = (rng.standard_normal((6, n)) * 1e-30).astype(np.float32)
    w = (1 + 0.1 * rng.standard_normal(n)).astype(np.float16) if weight else None
    ref = x.astype(np.float64) / np.sqrt((x.astype(np.float64) ** 2).mean(1, keepdims=True) + eps) * (1.0 if w is None else w.astype(np.float64))
    assert np.abs(ref).reshape(6, -1, 32).max(2).min() > 2.0 ** -100
    codes, scales = _codes(x, w, 32, eps)
    steps = scales.astype(np.float64).repeat(32, 1)
    # half a step, and what the roundings move a quotient of up to 127: five of y, three of the quotient
    assert (scales > 0).all() and (np.abs(codes * steps - ref) <= steps * (0.5 + 127 * 8 * 2.0 ** -24)).all()
    assert (np.abs(codes.astype(int)).reshape(6, -1, 32).max(2) == 127).all()
