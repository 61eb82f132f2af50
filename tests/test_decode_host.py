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
