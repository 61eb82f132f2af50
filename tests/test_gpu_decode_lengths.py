"""GPU checks of decode.AttentionHalf where a captured step and steps placed by the host take turns."""
import numpy as np
import pytest

from gpu_util import torch_cuda
import test_gpu_decode as D
from test_gpu_decode_serving import Serving

pytestmark = pytest.mark.gpu


def _captured(torch, half, x, y, *residual):
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        half.advance(x, y, *residual)
    return graph


def test_replays_and_placed_steps_in_turn():
    """A graph is replayed again after `advanced`: the host's calls are refused till it has asked, and go on from there."""
    torch = torch_cuda()
    sv = Serving(2, 90, pages=6)
    half = sv.half
    x = D._tokens(torch, 2, 30, D.HIDDEN, seed=1)
    half.fill(D._up(torch, x), torch.empty(2, 30, D.HIDDEN, dtype=torch.float16, device="cuda"))
    token, y = torch.empty(2, D.HIDDEN, dtype=torch.float16, device="cuda"), torch.empty(2, D.HIDDEN, dtype=torch.float16, device="cuda")
    graph = _captured(torch, half, token, y)
    assert half.advanced() == [30, 30]
    seen, results = [x[s] for s in range(2)], [[], []]
    for turn in range(3):
        for _ in range(2):
            more = D._tokens(torch, 2, D.HIDDEN, seed=10 * turn + len(results[0]))
            token.copy_(D._up(torch, more))
            graph.replay()
            torch.cuda.synchronize()
            for s in range(2):
                seen[s] = np.concatenate([seen[s], more[s:s + 1]])
                results[s].append(y[s].cpu().numpy())
        for call in (lambda: half.place([1, 1]), lambda: half.end(0), half.keep):
            with pytest.raises(ValueError):
                call()
        assert half.advanced() == [len(t) for t in seen] == half.past.tolist()
        more = D._tokens(torch, 2, D.HIDDEN, seed=90 + turn)
        one = torch.empty(2, D.HIDDEN, dtype=torch.float16, device="cuda")
        half.place([1, 1])
        half.run(D._up(torch, more), one)
        half.keep()
        for s in range(2):
            seen[s] = np.concatenate([seen[s], more[s:s + 1]])
            results[s].append(one[s].cpu().numpy())
    assert half.lengths == [39, 39] == half.past.tolist() and half.taken == [2, 2] == half.owned.tolist()
    for s in range(2):
        D._close(np.stack(results[s]), sv.reference(s, seen[s])[30:])


def test_replays_beyond_the_longest():
    """Sequences that may not grow wait, and those behind them; what they then get is what they would have had."""
    torch = torch_cuda()
    longest, begin = 40, (30, 38, 31)
    sv = Serving(3, longest, pages=9)
    half = sv.half
    x = D._tokens(torch, 3, 38, D.HIDDEN, seed=2)
    y, seen, results = torch.empty(38, D.HIDDEN, dtype=torch.float16, device="cuda"), [], [[], [], []]
    for s, n in enumerate(begin):
        for at, count in ((0, 30), (30, n - 30)):
            if count:
                half.place([count if k == s else 0 for k in range(3)])
                half.run(D._up(torch, x[s, at:at + count]), y[:count])
                half.keep()
        seen.append(x[s, :n])
    token, y = torch.empty(3, D.HIDDEN, dtype=torch.float16, device="cuda"), torch.empty(3, D.HIDDEN, dtype=torch.float16, device="cuda")
    graph = _captured(torch, half, token, y)
    half.advanced()
    for k in range(13):
        more = D._tokens(torch, 3, D.HIDDEN, seed=30 + k)
        token.copy_(D._up(torch, more))
        graph.replay()
        torch.cuda.synchronize()
        for s in range(3 if k < 2 else 1 if k < 10 else 0):
            seen[s] = np.concatenate([seen[s], more[s:s + 1]])
            results[s].append(y[s].cpu().numpy())
    assert half.advanced() == [40, 40, 33] == [len(t) for t in seen] and half.left == 3
    for s in (0, 1):
        half.end(s)
    more = D._tokens(torch, 1, D.HIDDEN, seed=60)
    half.place([0, 0, 1])
    half.run(D._up(torch, more), y[:1])
    half.keep()
    seen[2] = np.concatenate([seen[2], more])
    results[2].append(y[0].cpu().numpy())
    for s in range(3):
        D._close(np.stack(results[s]), sv.reference(s, seen[s])[begin[s]:])


def test_sequences_that_are_over_sit_replays_out():
    """The others' rows follow one another; a new sequence takes part from its first placed tokens on."""
    torch = torch_cuda()
    sv = Serving(4, 90, pages=6)
    half = sv.half
    x = D._tokens(torch, 4, 30, D.HIDDEN, seed=3)
    half.fill(D._up(torch, x), torch.empty(4, 30, D.HIDDEN, dtype=torch.float16, device="cuda"))
    token, y = torch.empty(4, D.HIDDEN, dtype=torch.float16, device="cuda"), torch.empty(4, D.HIDDEN, dtype=torch.float16, device="cuda")
    stream = torch.empty(4, D.HIDDEN, device="cuda")
    graph = _captured(torch, half, token, y, stream)
    half.advanced()
    seen, results, at = [x[s] for s in range(4)], [[] for _ in range(4)], [30] * 4

    def replay(takers):
        more = D._tokens(torch, 4, D.HIDDEN, seed=100 + sum(map(len, results)))
        token.copy_(D._up(torch, more))
        stream.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert half.owner[:4].tolist() == takers + [-1] * (4 - len(takers))
        for row, s in enumerate(takers):
            seen[s] = np.concatenate([seen[s], more[row:row + 1]])
            results[s].append(y[row].cpu().numpy())

    replay([0, 1, 2, 3])
    half.advanced()
    half.end(1)
    half.rest(2)
    for _ in range(3):
        replay([0, 3])
    assert half.advanced() == [34, 0, 31, 34] and half.left == 1 and half.taken == [2, 0, 1, 2]
    first = results[1]
    D._close(np.stack(first), sv.reference(1, seen[1])[30:])
    seen[1], results[1], at[1] = D._tokens(torch, 5, D.HIDDEN, seed=4), [], 5
    half.place([0, 5, 0, 0])
    half.run(D._up(torch, seen[1]), torch.empty(5, D.HIDDEN, dtype=torch.float16, device="cuda"))
    half.keep()
    replay([0, 1, 3])
    half.rest(2, False)
    replay([0, 1, 2, 3])
    assert half.advanced() == [36, 7, 32, 36] == [len(t) for t in seen] and half.left == 0
    for s in range(4):
        D._close(np.stack(results[s]), sv.reference(s, seen[s])[at[s]:])
