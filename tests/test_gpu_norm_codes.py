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
