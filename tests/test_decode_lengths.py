"""CPU checks of what decode.AttentionHalf knows of its sequences' lengths and pages, on host memory: the calls that place and trim are the oracle's."""
import pytest

import paper_2206_09557_amd as L
from oracle import step_oracle as S
from paper_2206_09557_amd import decode

from test_decode_host import _half, on_host  # noqa: F401 (a fixture)


class Device:
    """Placing and trimming of host tensors; what is copied into them by name."""

    def __init__(self, monkeypatch):
        self.pages = self.handle = None
        for name in ("pages_init", "place", "trim"):
            monkeypatch.setattr(L.lutgemm, "lutgemm_kv_" + name, getattr(self, name))
        monkeypatch.setattr(L.lutgemm, "lutgemm_kv_write", lambda *args: None)

    def _kept(self):
        import torch
        free, count, owned, table = self.handle._held
        for t, a in zip((free, owned, table), self.pages.arrays()):
            t.view(-1)[:a.size].copy_(torch.from_numpy(a.reshape(-1)))
        count.fill_(len(self.pages.free))

    def pages_init(self, handle, stream):
        self.handle, self.pages = handle, S.Pages(handle.pages, handle.page_tokens, handle.seqs, handle.table_pages)
        self._kept()

    def place(self, handle, past, fresh, tokens, most, first, positions, owner, slots, stream):
        import torch
        for t, a in zip((first, positions, owner, slots), self.pages.place(past.tolist(), fresh.tolist(), tokens, most)):
            if t is not None:
                t[:len(a)].copy_(torch.from_numpy(a))
        self._kept()

    def trim(self, handle, lengths, stream):
        self.pages.trim(lengths.tolist())
        self._kept()


@pytest.fixture
def device(on_host, monkeypatch):  # noqa: F811
    return Device(monkeypatch)


@pytest.mark.parametrize("pages", [0, 9])
def test_a_step_is_kept_once(device, pages):
    """What a second `keep` would add is positions that nobody wrote."""
    half = _half(512, 8, 2, 64, 2, 80, 16, page=32, pages=pages)
    with pytest.raises(ValueError):
        half.keep()
    half.place([3, 2])
    half.keep()
    for again in (None, [[0], [0]]):
        with pytest.raises(ValueError):
            half.keep(again)
    assert half.lengths == [3, 2]
    half.end(1)
    with pytest.raises(ValueError):
        half.keep()
    assert half.lengths == [3, 0] and half.past.tolist() == ([3, 0] if pages else [0, 0])
    half.place([1, 1])
    half.keep([[0], []])
    assert half.lengths == [4, 0]


def test_only_shared_pages_are_advanced(device):
    """The device keeps no lengths of sequences with pages of their own; the host's stay."""
    half = _half(512, 8, 2, 64, 2, 80, 16)
    half.place([3, 2])
    half.keep()
    with pytest.raises(ValueError):
        half.advanced()
    assert half.lengths == [3, 2] and half.known
    half.place([1, 1])
    half.keep()
    assert half.lengths == [4, 3]
