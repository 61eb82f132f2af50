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
    import torch
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
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


class Decoding:
    """A layer whose `advance` is captured and replayed, on the host: a replay does what it did to the tensors, and runs none of the class."""

    def __init__(self, monkeypatch, *args, **more):
        self.half = _half(*args, **more)
        monkeypatch.setattr(self.half, "run", lambda *rows: None)

    def capture(self, monkeypatch, device):
        """Nothing is executed."""
        import copy
        import torch
        kept = {name: t.clone() for name, t in vars(self.half).items() if torch.is_tensor(t)}
        pages = copy.deepcopy(device.pages)
        with monkeypatch.context() as m:
            m.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
            self.half.advance(None, None)
        for name, t in kept.items():
            vars(self.half)[name].copy_(t)
        device.pages = pages

    def replay(self):
        state = dict(vars(self.half))
        self.half.advance(None, None)
        vars(self.half).update(state)


def test_replays_that_the_host_has_not_asked_about(device, monkeypatch):
    """A graph is replayed again after `advanced`: no step is placed or kept, and no sequence ends, by lengths that are no longer so."""
    d = Decoding(monkeypatch, 512, 8, 2, 64, 2, 80, 16, page=32, pages=6)
    half = d.half
    half.place([30, 1])
    half.keep()
    d.capture(monkeypatch, device)
    assert half.advanced() == [30, 1]
    for k in range(3):
        d.replay()
    assert half.past.tolist() == [33, 4] and half.owned.tolist() == [2, 1]
    for call in (lambda: half.place([1, 1]), lambda: half.end(0), half.keep):
        with pytest.raises(ValueError):
            call()
    assert half.past.tolist() == [33, 4] and half.lengths == [30, 1]
    assert half.advanced() == [33, 4] and half.taken == [2, 1] and half.left == 3
    half.place([1, 0])
    half.keep()
    half.end(1)
    assert half.lengths == [34, 0] == half.past.tolist() and half.left == 4
    # one between a step's place and its keep: the step is not what it was
    half.place([2, 2])
    d.replay()
    with pytest.raises(ValueError):
        half.keep()
    assert half.advanced() == [35, 1]
    with pytest.raises(ValueError):
        half.keep()
    half.place([2, 2])
    half.keep([[0], [0, 1]])
    assert half.lengths == [36, 3] == half.past.tolist()


@pytest.mark.parametrize("seqs,page", [(3, 32), (32, 32)])
def test_replays_beyond_the_longest(device, monkeypatch, seqs, page):
    """A sequence of `longest` positions waits, and those behind it: nobody has another's row, and none is longer."""
    longest = 64                                   # (with 32 tokens more the table's pages end there)
    d = Decoding(monkeypatch, 512, 8, 2, 64, seqs, longest, 16, page=page, pages=200)
    half = d.half
    lengths = [5, longest - 2] + [9] * (seqs - 2)
    for s, n in enumerate(lengths):
        for at in range(0, n, 32):
            half.place([min(32, n - at) if k == s else 0 for k in range(seqs)])
            half.keep()
    d.capture(monkeypatch, device)
    assert half.advanced() == lengths
    for k in range(5):
        d.replay()
        served = seqs if k < 2 else 1
        assert half.first.tolist() == [min(s, served) for s in range(seqs + 1)]
        assert half.owner[:seqs].tolist() == list(range(served)) + [-1] * (seqs - served)
        assert half.positions[:served].tolist() == [5 + k, longest - 2 + k, *[9 + k] * (seqs - 2)][:served]
    assert half.advanced() == [10, longest] + [11] * (seqs - 2)
    with pytest.raises(ValueError):
        half.place([0, 1] + [0] * (seqs - 2))
    half.place([1, 0] + [1] * (seqs - 2))
    half.keep()
    assert half.lengths == [11, longest] + [12] * (seqs - 2) == half.past.tolist()
    half.end(1)
    assert half.owned.tolist() == half.taken == [1, 0] + [1] * (seqs - 2)


def test_sequences_that_are_over_or_idle_sit_replays_out(device, monkeypatch):
    """They get no token and no page; the others' rows follow one another."""
    d = Decoding(monkeypatch, 512, 8, 2, 64, 3, 64, 16, page=32, pages=4)
    half = d.half
    half.place([10, 7, 15])
    half.keep()
    half.place([21, 0, 0])
    half.keep()
    half.end(1)
    d.capture(monkeypatch, device)
    assert half.advanced() == [31, 0, 15]
    for k in range(2):
        d.replay()
        assert half.first.tolist() == [0, 1, 1, 2] and half.owner[:3].tolist() == [0, 2, -1] and half.positions[:3].tolist() == [31 + k, 15 + k, 0]
    assert half.advanced() == [33, 0, 17] and half.taken == [2, 0, 1] and half.left == 1
    half.rest(0)                                   # nobody else is told of a token of its
    half.rest(1, False)
    d.replay()
    assert half.first.tolist() == [0, 0, 1, 2] and half.advanced() == [33, 1, 18] and half.left == 0
    # tokens that are placed, or to be told otherwise, end it
    half.end(2)
    half.place([1, 0, 3])
    half.keep()
    half.rest(1)
    d.replay()
    assert half.first.tolist() == [0, 1, 1, 2] and half.advanced() == [35, 1, 4]
    for s in range(3):
        half.rest(s)
    d.replay()
    assert half.first.tolist() == [0, 0, 0, 0] and half.past.tolist() == [35, 1, 4]
    half.rest(1, False)
    half.place([29, 0, 0])
    half.keep()
    half.rest(0)
    half.advance(None, None)                       # (one of 64 positions may rest)
    assert half.advanced() == [64, 2, 4] and half.owner[:3].tolist() == [1, -1, -1]


def test_sequences_with_pages_of_their_own_do_not_rest(device):
    half = _half(512, 8, 2, 64, 2, 80, 16)
    with pytest.raises(ValueError):
        half.rest(0)
    half.place([1, 1])
    half.keep()
    half.end(0)
    half.place([1, 1])
    half.keep()
    assert half.lengths == [1, 2]


@pytest.mark.parametrize("pages,adapters", [(0, False), (0, True), (9, False), (9, True)])
def test_what_a_step_copies(device, monkeypatch, pages, adapters):
    """Whose the tokens are matters to adapters alone; with shared pages the device writes where the sequences' rows begin."""
    half = _half(512, 8, 2, 64, 2, 80, 16, page=32, pages=pages)
    if adapters:
        half.adapters = (None, L.lutgemm_adapters(16, 16, None, None, 512, 512, 1, 8))
    copied, put = [], half._set
    names = {id(t): name for name, t in vars(half).items()}

    def spy(tensor, values, kind):
        copied.append(names[id(tensor)])
        put(tensor, values, kind)

    monkeypatch.setattr(half, "_set", spy)
    half.place([3, 2])
    assert sorted(copied) == sorted(["past", "positions"] + ["owner"] * adapters + (["fresh"] if pages else ["first"]))
    assert half.first.tolist() == [0, 3, 5] and half.positions[:5].tolist() == [0, 1, 2, 0, 1]
    if adapters:
        assert half.owner[:5].tolist() == [0, 0, 0, 1, 1]


@pytest.mark.parametrize("count,rank", [(3, 16), (24, 256), (40, 128), (64, 64)])
def test_a_layer_has_workspace_for_adapters_of_any_step(on_host, count, rank):  # noqa: F811
    """Fewer tokens may need more than more of them do: a call that has too little is refused."""
    hidden, heads, dim = 5120, 40, 128
    shapes = (3 * heads * dim, hidden), (hidden, heads * dim)
    adapters = [L.lutgemm_adapters(16, 16, None, None, m, n, count, rank) for m, n in shapes]
    half = _half(hidden, heads, heads, dim, 4, 100, 16, adapters=adapters)
    for a, (m, n) in zip(adapters, shapes):
        need = [L.lutgemm_adapt_workspace_bytes(a, t) for t in range(1, decode.MOST_ROWS + 1)]
        assert max(need) <= half.ws_bytes
        fewer = [t for t in range(1, decode.MOST_ROWS) if need[t - 1] > need[t]]
        assert bool(fewer) == (count > 3)
        for t in fewer:
            with pytest.raises(L.LutGemmError) as e:
                L.lutgemm_adapt(16, 16, a, 16, None, 16, t, 0, n, m, m, 0, 16, need[t])
            assert e.value.code == L.LUTGEMM_EWORKSPACE
