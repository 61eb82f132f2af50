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


@pytest.mark.parametrize("rot_dim,neighbours,amplitude", [(0, False, 1.2), (32, True, 1.0), (16, False, 0.75), (64, True, 1.2)])
def test_positions_as_the_kernels_offer_them(monkeypatch, rot_dim, neighbours, amplitude):
    """Stretched frequencies with their amplitude, part of a head, neighbours paired: a prompt in chunks and a token after it."""
    torch = torch_cuda()
    rot = rot_dim or D.DIM
    qkv, out = D.decode.random_layer(D.HIDDEN, D.HEADS, D.KV, D.DIM, D.Q, D.G, seed=3)
    turns = L.lutgemm_rope_frequencies(rot, scaling=L.LUTGEMM_ROPE_PARTS, factor=8.0, trained=64.0)
    half = D.decode.AttentionHalf(qkv, out, D.HIDDEN, D.HEADS, D.KV, D.DIM, 1, 80, D.Q, D.G, 16, turns=turns, rot_dim=rot_dim,
                                  neighbours=neighbours, amplitude=amplitude)
    dense = D._weights(qkv, (D.HEADS + 2 * D.KV) * D.DIM, D.HIDDEN), D._weights(out, D.HIDDEN, D.HEADS * D.DIM)
    x = D._tokens(torch, 1, 42, D.HIDDEN, seed=8)
    y = torch.empty(1, 41, D.HIDDEN, dtype=torch.float16, device="cuda")
    half.fill(D._up(torch, x[:, :41].copy()), y)
    last = torch.empty(1, D.HIDDEN, dtype=torch.float16, device="cuda")
    half.place([1])
    half.run(D._up(torch, x[0, 41:].copy()), last)
    whole_rope = D.K.rope
    monkeypatch.setattr(D.K, "rope", lambda v, positions, t, dim: whole_rope(v, positions, t, rot, neighbours, False, amplitude))
    ref = D._reference(x[0], *dense, turns)
    D._close(np.concatenate([y[0].cpu().numpy(), last.cpu().numpy()]), ref)
