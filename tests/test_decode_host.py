"""CPU checks of decode.AttentionHalf: what it holds and refuses, on host memory, with no call that would reach a GPU."""
import pytest

import paper_2206_09557_amd as L
from paper_2206_09557_amd import decode


class _Stream:
    cuda_stream = 0


@pytest.fixture
def on_host(monkeypatch):
    """Tensors of the device are host tensors, and the workspace is not prepared."""
    import torch

    def host(make):
        return lambda *args, **kw: make(*args, **{k: v for k, v in kw.items() if k != "device"})

    for name in ("empty", "zeros", "arange"):
        monkeypatch.setattr(torch, name, host(getattr(torch, name)))
    monkeypatch.setattr(torch.Tensor, "cuda", lambda self: self)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: _Stream)
    monkeypatch.setattr(L.lutgemm, "lutgemm_workspace_init", lambda *args: None)


def _half(hidden, heads, kv_heads, dim, seqs, longest, kv_bits, **more):
    return decode.AttentionHalf(None, None, hidden, heads, kv_heads, dim, seqs, longest, kv_bits=kv_bits, **more)


@pytest.mark.parametrize("hidden,heads,kv_heads,dim,seqs,longest,kv_bits", [
    (512, 8, 4, 64, 2, 32768, 4), (1024, 16, 8, 64, 1, 32768, 4), (1024, 16, 8, 64, 30, 2072, 16), (2048, 32, 16, 64, 1, 32768, 4),
    (512, 8, 2, 64, 2, 80, 16), (640, 10, 2, 128, 3, 5000, 8), (5120, 40, 40, 128, 4, 312, 8)])
def test_no_step_needs_more_workspace_than_there_is(on_host, hidden, heads, kv_heads, dim, seqs, longest, kv_bits):
    half = _half(hidden, heads, kv_heads, dim, seqs, longest, kv_bits)
    for tokens in range(1, decode.MOST_ROWS + 1):
        for m, n in half.shapes():
            assert L.lutgemm_workspace_bytes(m, n, half.q, half.g, 8, tokens) <= half.ws_bytes
        for most in range(1, tokens + 1):
            step = half._step(tokens, most)
            assert 0 < L.lutgemm_attention_workspace_bytes(half.cache, step, heads, longest) <= half.ws_bytes, (tokens, most)


@pytest.mark.parametrize("counts,depths,mask", [
    ([1], None, None), ([2, -1], None, None), ([0, 0], None, None), ([20, 13], None, None), ([80, 1], None, None),
    ([2, 1], [[0, 1]], None), ([2, 1], [[0, 1], [0, 1]], None), ([2, 1], [[0], [0, 1]], None), ([2, 1], None, [1, 3]), ([2, 1], None, [1, 3, 1, 1])])
def test_steps_that_are_refused(on_host, counts, depths, mask):
    half = _half(512, 8, 2, 64, 2, 80, 16)
    with pytest.raises(ValueError):
        half.place(counts, depths, mask)
    half.place([2, 1], [[0, 0], [0]], [1, 2, 1])
    assert half.step.tokens == 3 and half.mask[:3].tolist() == [1, 2, 1] and half.positions[:3].tolist() == [0, 0, 0]


@pytest.mark.parametrize("accepted", [[[0]], [[0], [0], []], [[3], [0]], [[0], [2]], [[-1], []], [[1, 0], []], [[1, 1], []], [[0, 40], []]])
def test_tokens_that_cannot_be_kept(on_host, monkeypatch, accepted):
    """Rows that the step does not have are not read, another sequence's are not taken."""
    written = []
    monkeypatch.setattr(L.lutgemm, "lutgemm_kv_write", lambda *args: written.append(args))
    half = _half(512, 8, 2, 64, 2, 80, 16)
    half.place([3, 2])
    with pytest.raises(ValueError):
        half.keep(accepted)
    assert half.lengths == [0, 0] and not written
    half.keep([[1, 2], [0]])
    assert half.lengths == [2, 1] and len(written) == 1 and half.rows[:3].tolist() == [1, 2, 3] and half.first.tolist() == [0, 2, 3]


@pytest.mark.parametrize("turned,rot_dim", [(64, 32), (32, 0), (32, 64)])
def test_frequencies_of_other_channels_are_refused(on_host, turned, rot_dim):
    with pytest.raises(ValueError):
        _half(512, 8, 2, 64, 2, 80, 16, turns=L.lutgemm_rope_frequencies(turned), rot_dim=rot_dim)
    half = _half(512, 8, 2, 64, 2, 80, 16, turns=L.lutgemm_rope_frequencies(turned), rot_dim=turned)
    assert len(half.turns) == turned // 2


def test_kept_tokens_in_any_container(on_host, monkeypatch):
    import numpy as np
    import torch
    monkeypatch.setattr(L.lutgemm, "lutgemm_kv_write", lambda *args: None)
    for accepted in ([np.array([1, 2]), np.array([0])], (torch.tensor([1, 2]), torch.tensor([0])), ((1, 2), range(1))):
        half = _half(512, 8, 2, 64, 2, 80, 16)
        half.place(np.array([3, 2]))
        half.keep(accepted)
        assert half.lengths == [2, 1] and half.rows[:3].tolist() == [1, 2, 3]


def test_rows_that_a_step_cannot_take(on_host, monkeypatch):
    """Too few, too many, of another type, not one after the other: refused before anything is launched."""
    import torch
    half = _half(512, 8, 2, 64, 2, 80, 16)
    monkeypatch.setattr(half, "_product", lambda *args: pytest.fail("launched"))
    half.place([2, 1])
    good = torch.empty(3, 512, dtype=torch.float16)
    for bad in (good[:2], good[:, :256], good.float(), torch.empty(512, 3, dtype=torch.float16).t(), torch.empty(3, 1024, dtype=torch.float16)[:, ::2],
                torch.empty(1, 3, 512, dtype=torch.float16)):
        for x, y in ((bad, good), (good, bad)):
            with pytest.raises(ValueError):
                half.run(x, y)
