"""GPU checks of decode.AttentionHalf over steps of every size and its options, against the plain computation in 64 bits."""
import numpy as np
import pytest

import paper_2206_09557_amd as L

from gpu_util import torch_cuda
import test_gpu_decode as D

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("counts", [[16, 1], [1, 11], [12, 12], [32, 0]])
def test_steps_between_the_smallest_and_the_largest(monkeypatch, counts):
    """Where a context may grow long, more rows can mean fewer splits: a step of 11 to 16 tokens needs the largest workspace."""
    torch = torch_cuda()
    monkeypatch.setattr(D, "KV", 4)
    half, (qkv, out), turns = D._layer(2, 32768)
    x = D._tokens(torch, sum(counts), D.HIDDEN, seed=9)
    half.place(counts)
    y = torch.full((sum(counts), D.HIDDEN), float("nan"), dtype=torch.float16, device="cuda")
    print("case step", counts, half.ws_bytes, flush=True)
    half.run(D._up(torch, x), y)
    at = 0
    for n in counts:
        if n:
            D._close(y[at:at + n].cpu().numpy(), D._reference(x[at:at + n], qkv, out, turns))
        at += n
