"""GPU checks of decode.AttentionHalf with what surrounds it: norm and residual stream, low-rank adapters by sequence, pages that sequences share,
steps placed on the device, against the plain computation in 64 bits."""
import numpy as np
import pytest

import paper_2206_09557_amd as L
from oracle import step_oracle as S
from paper_2206_09557_amd import decode

from gpu_util import torch_cuda
import test_gpu_decode as D

pytestmark = pytest.mark.gpu

COUNT, RANK, EPS = 3, 16, 1e-5
SHAPES = ((D.HEADS + 2 * D.KV) * D.DIM, D.HIDDEN), (D.HIDDEN, D.HEADS * D.DIM)


class Serving:
    """A layer with norm, adapters and shared pages, and what it is made of in 64 bits."""

    def __init__(self, seqs, longest, pages, page=32, kv_bits=16):
        torch = torch_cuda()
        qkv, out = decode.random_layer(D.HIDDEN, D.HEADS, D.KV, D.DIM, D.Q, D.G, seed=3)
        self.dense = [D._weights(w, m, n) for w, (m, n) in zip((qkv, out), SHAPES)]
        self.weight = (1 + 0.2 * np.random.default_rng(4).standard_normal(D.HIDDEN)).astype(np.float16)
        self.adapters = [decode.random_adapters(m, n, COUNT, RANK, seed=k) for k, (m, n) in enumerate(SHAPES)]
        self.held = [tuple(t.cpu().numpy().astype(np.float64) for t in a._held[:2]) for a in self.adapters]
        self.half = decode.AttentionHalf(qkv, out, D.HIDDEN, D.HEADS, D.KV, D.DIM, seqs, longest, D.Q, D.G, kv_bits, page=page,
                                         norm=torch.from_numpy(self.weight).cuda(), eps=EPS, adapters=self.adapters, pages=pages)
        self.of = [s % (COUNT + 1) - 1 for s in range(seqs)]          # the first has none
        self.half.adapter_of.copy_(torch.tensor(self.of, dtype=torch.int32))

    def merged(self, seq):
        """Both products' weights with the sequence's adapter in them."""
        a = self.of[seq]
        return [w if a < 0 else w + up[a] @ down[a] for w, (down, up) in zip(self.dense, self.held)]

    def reference(self, seq, x):
        """Outputs of a sequence's tokens; x [tokens][hidden] in 64 bits is what the norm is of."""
        s = np.asarray(x, np.float64)
        normed = s / np.sqrt((s * s).mean(1, keepdims=True) + EPS) * self.weight.astype(np.float64)
        return D._reference(normed, *self.merged(seq), L.lutgemm_rope_frequencies(D.DIM))


def test_prompts_and_single_tokens():
    """Three sequences, one without adapter, from one pool; the single tokens' x is added to a residual stream before the norm."""
    torch = torch_cuda()
    sv = Serving(3, 80, pages=7)
    half, seqs = sv.half, 3
    x = D._tokens(torch, seqs, 41, D.HIDDEN, seed=1)
    y = torch.empty(seqs, 41, D.HIDDEN, dtype=torch.float16, device="cuda")
    half.fill(D._up(torch, x), y)
    seen, outputs = [x[s].astype(np.float64) for s in range(seqs)], [y[s].cpu().numpy() for s in range(seqs)]
    for k in range(3):
        more = D._tokens(torch, seqs, D.HIDDEN, seed=20 + k)
        stream = np.random.default_rng(30 + k).standard_normal((seqs, D.HIDDEN)).astype(np.float32)
        d_stream, one = D._up(torch, stream), torch.empty(seqs, D.HIDDEN, dtype=torch.float16, device="cuda")
        half.place([1] * seqs)
        half.run(D._up(torch, more), one, d_stream)
        half.keep()
        total = stream.astype(np.float64) + more
        assert np.abs(d_stream.cpu().numpy() - total).max() <= 2.0 ** -24 * np.abs(total).max()
        for s in range(seqs):
            seen[s] = np.concatenate([seen[s], total[s:s + 1]])
            outputs[s] = np.concatenate([outputs[s], one[s:s + 1].cpu().numpy()])
    assert half.lengths == [44] * 3 and half.left == 1 == int(half.free_count) and half.taken == [2] * 3
    for s in range(seqs):
        D._close(outputs[s], sv.reference(s, seen[s]))
    # the adapter matters to those that have one: by far more than what is allowed above
    sv.of = [-1] * 3
    for s in range(1, seqs):
        ref = sv.reference(s, seen[s])
        assert np.linalg.norm(outputs[s] - ref) > 3e-2 * np.linalg.norm(ref)


@pytest.mark.parametrize("kv_bits", [16, 4])
def test_a_captured_step_advances_on_the_device(kv_bits):
    """Replays that place their tokens and take their pages, across pages' ends, against steps placed by the host: the same bits."""
    torch = torch_cuda()
    x = D._up(torch, D._tokens(torch, 4, 29, D.HIDDEN, seed=2))
    token = D._up(torch, D._tokens(torch, 4, D.HIDDEN, seed=4))
    results = []
    for captured in (False, True):
        half = Serving(4, 120, pages=12, kv_bits=kv_bits).half
        half.fill(x, torch.empty_like(x))
        y, stream = torch.empty(4, D.HIDDEN, dtype=torch.float16, device="cuda"), torch.zeros(4, D.HIDDEN, device="cuda")
        if captured:
            graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.graph(graph, stream=side):
                half.advance(token, y, stream)
        seen = []
        for _ in range(40):
            if captured:
                graph.replay()
            else:
                half.place([1] * 4)
                half.run(token, y, stream)
                half.keep()
            torch.cuda.synchronize()
            seen.append((y.cpu().numpy(), stream.cpu().numpy()))
        if captured:
            half.advanced()
        assert half.lengths == [69] * 4 and half.taken == [3] * 4 and half.left == 0 == int(half.free_count)
        results.append(seen)
    for (a, s), (b, t) in zip(*results):
        assert np.isfinite(a.astype(np.float64)).all()
        np.testing.assert_array_equal(a, b)
        np.testing.assert_array_equal(s, t)


def test_pages_that_run_out():
    """The host refuses a step that lacks pages; on the device the last sequences wait, and go on when another one has ended."""
    torch = torch_cuda()
    sv = Serving(3, 90, pages=4)
    half = sv.half
    x = D._tokens(torch, 3, 32, D.HIDDEN, seed=5)
    y = torch.empty(3, 32, D.HIDDEN, dtype=torch.float16, device="cuda")
    half.fill(D._up(torch, x), y)                  # a page each, one is left
    with pytest.raises(ValueError):
        half.place([1, 1, 0])
    assert half.left == 1 and half.lengths == [32] * 3
    one = torch.empty(3, D.HIDDEN, dtype=torch.float16, device="cuda")
    token = D._tokens(torch, 3, D.HIDDEN, seed=6)
    half.advance(D._up(torch, token), one)
    for call in (lambda: half.place([1, 0, 0]), lambda: half.end(0)):       # the host does not know the lengths yet
        with pytest.raises(ValueError):
            call()
    assert half.advanced() == [33, 32, 32] and half.left == 0
    D._close(one[:1].cpu().numpy(), sv.reference(0, np.concatenate([x[0], token[:1]]))[32:])
    half.end(1)
    assert half.left == 1 and half.lengths == [33, 0, 32] and int(half.free_count) == 1
    half.place([1, 0, 1])
    with pytest.raises(ValueError):
        half.end(2)                                # its new token is not kept yet
    last = torch.empty(2, D.HIDDEN, dtype=torch.float16, device="cuda")
    more = D._tokens(torch, 2, D.HIDDEN, seed=7)
    half.run(D._up(torch, more), last)
    half.keep()
    assert half.lengths == [34, 0, 33] and half.left == 0
    D._close(last[:1].cpu().numpy(), sv.reference(0, np.concatenate([x[0], token[:1], more[:1]]))[33:])
    D._close(last[1:].cpu().numpy(), sv.reference(2, np.concatenate([x[2], more[1:]]))[32:])
    with pytest.raises(ValueError):
        half.place([0, 1, 0])


def test_an_accepted_branch_gives_pages_back():
    torch = torch_cuda()
    sv = Serving(2, 96, pages=6)
    half = sv.half
    x = D._tokens(torch, 2, 30, D.HIDDEN, seed=8)
    half.fill(D._up(torch, x), torch.empty(2, 30, D.HIDDEN, dtype=torch.float16, device="cuda"))
    draft = D._tokens(torch, 7, D.HIDDEN, seed=9)
    half.place([5, 2], [[0, 0, 1, 1, 2], [0, 1]], [0b00001, 0b00010, 0b00110, 0b01010, 0b11010, 0b01, 0b11])
    assert half.left == 3 == int(half.free_count)  # the first sequence's tree reaches into its second page
    looked = torch.empty(7, D.HIDDEN, dtype=torch.float16, device="cuda")
    half.run(D._up(torch, draft), looked)
    half.keep([[1, 3], [0]])
    assert half.lengths == [32, 31] and half.left == 4 == int(half.free_count)
    y, after = torch.empty(2, D.HIDDEN, dtype=torch.float16, device="cuda"), D._tokens(torch, 2, D.HIDDEN, seed=10)
    half.place([1, 1])
    half.run(D._up(torch, after), y)
    y, looked = y.cpu().numpy(), looked.cpu().numpy()
    ref0 = sv.reference(0, np.concatenate([x[0], draft[[1, 3]], after[:1]]))
    ref1 = sv.reference(1, np.concatenate([x[1], draft[[5]], after[1:]]))
    D._close(looked[[1, 3]], ref0[30:32])
    D._close(looked[5:6], ref1[30:31])
    D._close(y, np.stack([ref0[32], ref1[31]]))


def test_what_a_layer_refuses():
    torch = torch_cuda()
    qkv, out = decode.random_layer(D.HIDDEN, D.HEADS, D.KV, D.DIM, D.Q, D.G, seed=3)
    wrong = decode.random_adapters(D.HIDDEN, D.HIDDEN, 1, 8)

    def layer(**more):
        return decode.AttentionHalf(qkv, out, D.HIDDEN, D.HEADS, D.KV, D.DIM, 1, 64, D.Q, D.G, 16, **more)

    for more in (dict(adapters=(wrong, None)), dict(norm=torch.ones(D.HIDDEN, device="cuda")), dict(norm=torch.ones(8, device="cuda").half())):
        with pytest.raises(ValueError):
            layer(**more)
    half = layer()
    half.place([1])
    x = torch.zeros(1, D.HIDDEN, dtype=torch.float16, device="cuda")
    for call in (lambda: half.run(x, x.clone(), x.clone()), lambda: half.advance(x, x.clone())):      # no norm, no shared pages
        with pytest.raises(ValueError):
            call()
    half = layer(norm=torch.ones(D.HIDDEN, device="cuda").half(), pages=3)
    half.place([1])
    with pytest.raises(ValueError):
        half.run(x, x.clone(), torch.zeros(1, D.HIDDEN, device="cuda").double())
    half.advance(x, x.clone())
    with pytest.raises(ValueError):
        half.keep()                                # it was not placed by the host
