"""GPU checks of the attention half as a whole: a prompt in chunks, decoding by itself and from a graph, a drafted tree whose
accepted branch is kept, against a plain computation in 64 bits."""
import numpy as np
import pytest

import paper_2206_09557_amd as L
from oracle import bcq_oracle as O
from oracle import kv_oracle as K
from paper_2206_09557_amd import decode

from gpu_util import torch_cuda

pytestmark = pytest.mark.gpu

HIDDEN, HEADS, KV, DIM, Q, G = 512, 8, 2, 64, 3, 128


def _weights(packed, m, n):
    bits, alpha, z = packed
    planes = L.lutgemm_unpack_bcq(bits.cpu().numpy(), m, n, Q)
    return O.dequant(planes, O.decode_alpha(alpha.cpu().numpy(), m, n // G, Q), None, G)


def _reference(x, qkv, out, turns):
    """The outputs of one sequence's tokens x [tokens][hidden], each seeing those before it.  The stages' results are kept in 64 bits."""
    y = x.astype(np.float64) @ qkv.T
    tokens = len(x)
    heads = y[:, :(HEADS + KV) * DIM].reshape(tokens, HEADS + KV, DIM)
    turned = K.rope(heads, np.arange(tokens), turns, DIM)
    q, k, v = turned[:, :HEADS], turned[:, HEADS:], y[:, (HEADS + KV) * DIM:].reshape(tokens, KV, DIM)
    mixed = np.empty((tokens, HEADS, DIM))
    for t in range(tokens):
        for h in range(HEADS):
            s = k[:t + 1, h // (HEADS // KV)] @ q[t, h] * DIM ** -0.5
            w = np.exp(s - s.max())
            mixed[t, h] = w / w.sum() @ v[:t + 1, h // (HEADS // KV)]
    return mixed.reshape(tokens, -1) @ out.T


def _layer(seqs, longest, kv_bits=16):
    qkv, out = decode.random_layer(HIDDEN, HEADS, KV, DIM, Q, G, seed=3)
    half = decode.AttentionHalf(qkv, out, HIDDEN, HEADS, KV, DIM, seqs, longest, Q, G, kv_bits)
    dense = _weights(qkv, (HEADS + 2 * KV) * DIM, HIDDEN), _weights(out, HIDDEN, HEADS * DIM)
    return half, dense, L.lutgemm_rope_frequencies(DIM)


def _close(y, ref):
    """Relative to the norm.  Products are within 1e-3 (their own tests); rounding to fp16 after the product, the turn, the attention and
    the last product adds 2^-12 (rms half an ulp) each; what the queries' and keys' errors of 2 x 1.3e-3 do to a score of the
    order of one, twice that to the weights' ratio.  Together under 1e-3 + 1e-3 + 4 * 2^-12 + 4 * 1.3e-3 = 8.2e-3."""
    ref = np.asarray(ref)
    assert np.linalg.norm(y.astype(np.float64) - ref) <= 1e-2 * np.linalg.norm(ref)


def _tokens(torch, *shape, seed):
    return np.random.default_rng(seed).standard_normal(shape).astype(np.float16)


def _up(torch, x):
    return torch.from_numpy(x).cuda()


def test_chunks_and_single_tokens():
    torch = torch_cuda()
    half, (qkv, out), turns = _layer(2, 80)
    x = _tokens(torch, 2, 45, HIDDEN, seed=1)
    d_x = _up(torch, x)
    d_y = torch.full((2, 45, HIDDEN), float("nan"), dtype=torch.float16, device="cuda")
    half.fill(d_x[:, :41].contiguous(), chunk := torch.empty(2, 41, HIDDEN, dtype=torch.float16, device="cuda"))
    d_y[:, :41] = chunk
    for t in range(41, 45):
        half.place([1, 1])
        one = torch.empty(2, HIDDEN, dtype=torch.float16, device="cuda")
        half.run(d_x[:, t].contiguous(), one)
        half.keep()
        d_y[:, t] = one
    assert half.lengths == [45, 45]
    y = d_y.cpu().numpy()
    for s in range(2):
        _close(y[s], _reference(x[s], qkv, out, turns))


@pytest.mark.parametrize("kv_bits", [16, 8, 4])
def test_a_captured_step_advances(kv_bits):
    """Replays against the same steps launched one by one: the same bits."""
    torch = torch_cuda()
    x = _up(torch, _tokens(torch, 3, 33, HIDDEN, seed=2))
    token = _up(torch, _tokens(torch, 3, HIDDEN, seed=4))
    results = []
    for captured in (False, True):
        half, _, _ = _layer(3, 96, kv_bits)
        half.fill(x, torch.empty_like(x))
        half.place([1, 1, 1])
        y = torch.empty(3, HIDDEN, dtype=torch.float16, device="cuda")
        seen = []

        def step():
            half.run(token, y)
            half.past.add_(1)
            half.positions[:3].add_(1)

        if captured:
            graph = torch.cuda.CUDAGraph()
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.graph(graph, stream=side):
                step()
        for _ in range(5):
            graph.replay() if captured else step()
            seen.append(y.cpu().numpy())
            torch.cuda.synchronize()
        results.append(seen)
    for a, b in zip(*results):
        assert np.isfinite(a.astype(np.float64)).all()
        np.testing.assert_array_equal(a, b)


def test_an_accepted_branch_is_as_if_decoded():
    torch = torch_cuda()
    half, (qkv, out), turns = _layer(2, 96)
    x = _tokens(torch, 2, 40, HIDDEN, seed=5)
    half.fill(_up(torch, x), torch.empty(2, 40, HIDDEN, dtype=torch.float16, device="cuda"))
    # sequence 0: tokens 0 and 1 are roots, 2 and 3 children of 1, 4 of 3; sequence 1: a chain of two
    draft = _tokens(torch, 7, HIDDEN, seed=6)
    half.place([5, 2], [[0, 0, 1, 1, 2], [0, 1]], [0b00001, 0b00010, 0b00110, 0b01010, 0b11010, 0b01, 0b11])
    looked = torch.empty(7, HIDDEN, dtype=torch.float16, device="cuda")
    half.run(_up(torch, draft), looked)
    half.keep([[1, 3, 4], [0]])
    assert half.lengths == [43, 41]
    after = _tokens(torch, 2, HIDDEN, seed=7)
    y = torch.empty(2, HIDDEN, dtype=torch.float16, device="cuda")
    half.place([1, 1])
    half.run(_up(torch, after), y)
    y, looked = y.cpu().numpy(), looked.cpu().numpy()
    ref0 = _reference(np.concatenate([x[0], draft[[1, 3, 4]], after[:1]]), qkv, out, turns)
    ref1 = _reference(np.concatenate([x[1], draft[[5]], after[1:]]), qkv, out, turns)
    _close(looked[[1, 3, 4]], ref0[40:43])
    _close(looked[5:6], ref1[40:41])
    _close(y, np.stack([ref0[43], ref1[41]]))
    _close(looked[2:3], _reference(np.concatenate([x[0], draft[[1, 2]]]), qkv, out, turns)[41:])
    _close(looked[6:7], _reference(np.concatenate([x[1], draft[[5, 6]]]), qkv, out, turns)[41:])


def test_refuses_what_does_not_fit():
    half, _, _ = _layer(2, 40)
    for counts in ([1], [0, 0], [20, 13], [41, 0]):
        with pytest.raises(ValueError):
            half.place(counts)


def test_the_command_runs(capsys):
    assert decode.main(["--hidden", "512", "--heads", "8", "--kv-heads", "2", "--head-dim", "64", "--seqs", "2", "--prompt", "40",
                        "--steps", "3"]) == 0
    printed = capsys.readouterr().out
    assert "outputs finite: True" in printed and "lengths now [45, 43]" in printed
