"""GPU checks of lutgemm_kv_place and lutgemm_kv_trim: whole numbers, equal to those of an oracle that goes sequence by sequence."""
import numpy as np
import pytest

import paper_2206_09557_amd as L
from oracle import step_oracle as S

from gpu_util import torch_cuda

pytestmark = pytest.mark.gpu

MARK = 123456


class Placer:
    """The calls on a set of pages, beside the oracle's."""

    def __init__(self, pages, page_tokens, seqs, table_pages):
        torch = torch_cuda()
        self.torch, self.pages, self.seqs, self.width = torch, pages, seqs, table_pages
        whole = dict(dtype=torch.int32, device="cuda")
        self.free, self.count = torch.full((pages + 1,), MARK, **whole), torch.full((2,), MARK, **whole)
        self.owned, self.table = torch.full((seqs + 1,), MARK, **whole), torch.full((seqs * table_pages + 1,), MARK, **whole)
        self.handle = L.lutgemm_kv_pages(self.free, self.count, self.owned, self.table, pages, page_tokens, seqs, table_pages)
        self.oracle = S.Pages(pages, page_tokens, seqs, table_pages)
        L.lutgemm_kv_pages_init(self.handle, self.stream())
        self.check()

    def stream(self):
        return self.torch.cuda.current_stream().cuda_stream

    def up(self, a):
        return self.torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()

    def check(self):
        self.torch.cuda.synchronize()
        free, owned, table = self.oracle.arrays()
        assert int(self.count[0]) == len(free) and int(self.count[1]) == MARK
        np.testing.assert_array_equal(self.free.cpu().numpy()[:len(free)], free)
        np.testing.assert_array_equal(self.owned.cpu().numpy()[:-1], owned)
        np.testing.assert_array_equal(self.table.cpu().numpy()[:-1].reshape(self.seqs, self.width), table)
        assert int(self.free[-1]) == int(self.owned[-1]) == int(self.table[-1]) == MARK

    def place(self, past, fresh, tokens, most, outputs=(True, True, True)):
        torch = self.torch
        first = torch.full((self.seqs + 2,), MARK, dtype=torch.int32, device="cuda")
        out = [torch.full((tokens + 1,), MARK, dtype=t, device="cuda") if wanted else None
               for t, wanted in zip((torch.int32, torch.int32, torch.int64), outputs)]
        L.lutgemm_kv_place(self.handle, self.up(past), self.up(fresh), tokens, most, first, *out, self.stream())
        want = self.oracle.place(past, fresh, tokens, most)
        self.check()
        assert int(first[-1]) == MARK
        np.testing.assert_array_equal(first.cpu().numpy()[:-1], want[0])
        for got, w in zip(out, want[1:]):
            if got is not None:
                assert int(got[-1]) == MARK
                np.testing.assert_array_equal(got.cpu().numpy()[:-1], w)
        return want[0]

    def trim(self, lengths):
        L.lutgemm_kv_trim(self.handle, self.up(lengths), self.stream())
        self.oracle.trim(lengths)
        self.check()


def test_one_sequence_token_by_token():
    p = Placer(4, 32, 1, 3)
    for past in range(0, 96, 7):
        p.place([past], [min(7, 96 - past)], 8, 8)
    p.place([90], [7], 8, 8)                       # more than the table holds
    p.trim([33])
    p.trim([0])
    p.trim([0])


@pytest.mark.parametrize("seqs,page,width,pages,most,tokens", [
    (5, 64, 4, 20, 9, 30), (63, 32, 3, 60, 70, 1000), (64, 96, 2, 100, 33, 700), (300, 32, 5, 700, 40, 5000),
    (1025, 32, 2, 1500, 8, 4000), (4097, 64, 2, 5000, 5, 9000), (9000, 32, 3, 20000, 60, 150000), (65535, 32, 1, 60000, 2, 70000),
    (40, 64, 600, 30000, 38400, 400000)])
def test_steps_of_every_kind(seqs, page, width, pages, most, tokens):
    """Steps in a row: idle sequences, lengths that do not fit, more than most, pages and rows that run out, drafts refused."""
    print("case place", seqs, page, width, pages, most, tokens, flush=True)
    rng = np.random.default_rng(seqs)
    p = Placer(pages, page, seqs, width)
    past = np.zeros(seqs, np.int64)
    for k in range(4):
        fresh = rng.integers(0, most + 2, seqs)
        fresh[rng.random(seqs) < 0.2] = 0
        fresh[rng.random(seqs) < 0.02] = -3
        asked = past.copy()
        asked[rng.random(seqs) < 0.02] = -1
        first = p.place(asked, fresh, tokens, most, outputs=[(True, True, True), (False, True, False), (True, False, True), (False, False, False)][k])
        past += np.diff(first)
        # some drafts are refused, some sequences end, some are left as they are
        past = np.where(rng.random(seqs) < 0.3, np.maximum(past - 20, 0), past)
        past[rng.random(seqs) < 0.2] = 0
        lengths = past.copy()
        kept = rng.random(seqs) < 0.1
        lengths[kept] = -1
        p.trim(lengths)


def test_the_rows_run_out_at_the_first_of_them():
    p = Placer(64, 32, 6, 8)
    p.place([0] * 6, [5, 6, 0, 7, 1, 1], 11, 8)    # 5 + 6 rows: the one with 7 waits, and the ones behind it
    p.place([5, 6, 0, 0, 0, 0], [0, 0, 0, 7, 1, 1], 9, 8)
    p.place([5, 6, 0, 7, 1, 1], [1] * 6, 0, 8)     # no rows at all
    p.place([5, 6, 0, 7, 1, 1], [0] * 6, 4, 8)     # nobody


def test_the_pages_run_out_at_the_first_of_them():
    p = Placer(5, 32, 4, 4)
    p.place([0] * 4, [32, 65, 33, 1], 200, 100)    # 1 + 3 pages; the third needs two of the one that is left
    p.place([32, 65, 0, 0], [0, 0, 1, 1], 10, 2)   # one each: the last one waits
    p.place([32, 65, 1, 0], [1, 31, 31, 1], 100, 50)   # the first needs a page that is not there: all wait
    p.place([31, 65, 1, 0], [1, 31, 31, 1], 100, 50)   # within its page: served, up to the last
    p.trim([0, -1, 0, 0])
    p.place([0, 65, 0, 0], [64, 31, 1, 0], 100, 64)


def test_a_trim_undoes_a_place():
    torch = torch_cuda()
    for seqs, width, page in ((30, 9, 32), (5000, 4, 64)):
        p = Placer(seqs * width, page, seqs, width)
        rng = np.random.default_rng(3)
        past = rng.integers(0, width * page // 2, seqs)
        p.place(np.zeros(seqs, int), past, int(past.sum()), int(past.max()))
        free, table = p.free.clone(), p.table.clone()
        fresh = rng.integers(1, width * page // 2, seqs)
        p.place(past, fresh, int(fresh.sum()), int(fresh.max()))
        p.trim(past)
        assert torch.equal(p.table, table) and torch.equal(p.free[:int(p.count[0])], free[:int(p.count[0])])


def test_nonsense_in_device_memory_stays_there():
    """Counts and ownership out of range are taken as the nearest ones in range; page numbers are passed on, slots of bad ones are -1."""
    torch = torch_cuda()
    seqs, page, width, pages = 3, 32, 2, 4
    whole = dict(dtype=torch.int32, device="cuda")
    free = torch.tensor([9, -7, 2, 3, MARK], **whole)
    count, owned = torch.tensor([99, MARK], **whole), torch.tensor([-5, 77, 1, MARK], **whole)
    table = torch.tensor([-1, -1, 50, 1, 0, -1, MARK], **whole)
    handle = L.lutgemm_kv_pages(free, count, owned, table, pages, page, seqs, width)
    first, slots = torch.full((seqs + 2,), MARK, **whole), torch.full((101,), MARK, dtype=torch.int64, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    L.lutgemm_kv_place(handle, torch.tensor([31, 31, 31], **whole), torch.tensor([33, 2, 33], **whole), 100, 40, first, None, None, slots, stream)
    torch.cuda.synchronize()
    assert first.tolist() == [0, 33, 35, 68, MARK] and count.tolist() == [1, MARK] and owned.tolist() == [2, 77, 2, MARK]
    assert table.tolist() == [3, 2, 50, 1, 0, -7, MARK]
    want = [3 * 32 + 31] + [2 * 32 + k for k in range(32)] + [-1, 32] + [31] + [-1] * 32 + [-1] * 32 + [MARK]
    assert slots.tolist() == want
    L.lutgemm_kv_trim(handle, torch.tensor([-1, 0, 40000], **whole), stream)
    torch.cuda.synchronize()
    assert owned.tolist() == [2, 0, 2, MARK] and count.tolist() == [3, MARK] and free.tolist()[:3] == [9, 1, 50] and free.tolist()[-1] == MARK
    assert table.tolist() == [3, 2, -1, -1, 0, -7, MARK]
    owned[0], count[0] = 2, 4                       # more pages come back than the stack has room for
    L.lutgemm_kv_trim(handle, torch.zeros(seqs, **whole), stream)
    torch.cuda.synchronize()
    assert count.tolist() == [4, MARK] and free.tolist()[-1] == MARK and owned.tolist() == [0, 0, 0, MARK]


def test_a_captured_place_is_replayed():
    torch = torch_cuda()
    p = Placer(200, 32, 12, 10)
    whole = dict(dtype=torch.int32, device="cuda")
    past, fresh = torch.zeros(12, **whole), torch.ones(12, **whole)
    first, positions, owner = torch.empty(13, **whole), torch.empty(16, **whole), torch.empty(16, **whole)
    slots = torch.empty(16, dtype=torch.int64, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        s = torch.cuda.current_stream().cuda_stream
        L.lutgemm_kv_place(p.handle, past, fresh, 16, 4, first, positions, owner, slots, s)
        past.add_(fresh)
        L.lutgemm_kv_trim(p.handle, past, s)
    for k in range(70):
        held = past.tolist()
        graph.replay()
        want = p.oracle.place(held, [1] * 12, 16, 4)
        p.oracle.trim([h + 1 for h in held])
        p.check()
        for got, w in zip((first, positions, owner, slots), want):
            np.testing.assert_array_equal(got.cpu().numpy(), w)
    torch.cuda.synchronize()
