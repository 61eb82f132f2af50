"""GPU parity of lutgemm_adapt with the 64-bit oracle: every number of tokens and adapter, ranks, types, strides, tokens without an adapter."""
import numpy as np
import pytest

import paper_2206_09557_amd as L
from oracle import step_oracle as S

from gpu_util import make_workspace, torch_cuda

pytestmark = pytest.mark.gpu

MARK = 77


class Set:
    """Adapters in stores that hold NaN beyond every adapter's rank."""

    def __init__(self, rng, m, n, count, rank, ranks=None, scales=True):
        torch = torch_cuda()
        self.m, self.n, self.count, self.rank = m, n, count, rank
        self.down = (rng.standard_normal((count, rank, n)) / np.sqrt(n)).astype(np.float16)
        self.up = (rng.standard_normal((count, m, rank)) / np.sqrt(rank)).astype(np.float16)
        self.ranks = None if ranks is None else np.asarray(ranks, np.int32)
        self.scales = (0.5 + rng.random(count)).astype(np.float32) if scales else None
        if ranks is not None:
            for a, r in enumerate(ranks):
                self.down[a, r:], self.up[a, :, r:] = np.nan, np.nan
        self.d = [None if a is None else torch.from_numpy(a).cuda() for a in (self.down, self.up, self.ranks, self.scales)]
        self.handle = L.lutgemm_adapters(*self.d, m, n, count, rank)


def _run(a, x, base, of, owner=None, seqs=0, f32=False, x_stride=0, base_stride=0, y_stride=0, in_place=False, offset=0, ws=None, stream=None):
    """y [tokens][y_stride or m]; checks what is behind rows and in gaps."""
    torch = torch_cuda()
    tokens = len(x)
    xs, bs, ys = x_stride or a.n, base_stride or a.m, y_stride or a.m
    ys = bs if in_place else ys
    dt = np.float32 if f32 else np.float16
    wide = np.full((tokens, xs), np.nan, np.float16)
    wide[:, :a.n] = x
    d_x = torch.from_numpy(wide).cuda()
    flat = np.full(tokens * bs + 2 * offset, MARK, dt)
    rows = np.full((tokens, bs), MARK, dt)
    rows[:, :a.m] = base
    flat[offset:offset + tokens * bs] = rows.reshape(-1)
    d_base = torch.from_numpy(flat).cuda()[offset:]
    d_y = d_base if in_place else torch.full((tokens * ys + 2 * offset,), float(MARK), dtype=d_base.dtype, device="cuda")[offset:]
    d_of = torch.from_numpy(np.asarray(of, np.int32)).cuda()
    d_owner = None if owner is None else torch.from_numpy(np.asarray(owner, np.int32)).cuda()
    nbytes = L.lutgemm_adapt_workspace_bytes(a.handle, tokens)
    ws = make_workspace(nbytes) if ws is None else ws
    stream = stream or torch.cuda.current_stream()
    torch.cuda.synchronize()
    L.lutgemm_adapt(d_x, d_base, a.handle, d_of, d_owner, d_y, tokens, seqs, xs, bs, ys, L.LUTGEMM_Y_F32 if f32 else 0, ws, ws.numel(), stream.cuda_stream)
    torch.cuda.synchronize()
    assert (ws[:32768] == 0).all(), "a product's counters"
    y = d_y.cpu().numpy()
    assert (y[tokens * ys:] == MARK).all()
    y = y[:tokens * ys].reshape(tokens, ys)
    assert (y[:, a.m:] == MARK).all()
    return y[:, :a.m]


def _check(y, ref, reach, mass, f32, n, rank):
    # The first product: a chain of n / 32 (at most; parts and wavefronts make shorter ones) sums of exact products of 22 bits, each step
    # of the matrix unit 2^-24 of what it holds, and up to 2^-23 of a step's own sum of 32: 2^-24 (n / 32 + 40) of the sum of
    # magnitudes is more than any of it.  h in two parts of fp16: 2^-22 of its largest, scale and powers of two included.  The second product the same
    # with its rank.  Then one addition, and the rounding of the type.
    bound = 2.0 ** -24 * (n / 32 + 40) * reach + 2.0 ** -22 * mass + 2.0 ** -24 * (rank / 16 + 40) * reach + 2.0 ** -24 * np.abs(ref)
    if not f32:
        bound = bound * 1.001 + 2.0 ** -11 * np.abs(ref) + 2.0 ** -25
    err = np.abs(y.astype(np.float64) - ref)
    assert np.isfinite(ref).all() and (err <= bound).all(), (err - bound).max()
    # and as a whole: a rounding is half a step at most, errors of products grow with the root of their number
    size = np.linalg.norm(ref)
    assert np.linalg.norm(err) <= (2.0 ** -11 if not f32 else 0.0) * size + 2.0 ** -24 * (2 + (n / 32) ** 0.5) * np.linalg.norm(reach + np.abs(ref)) + 2.0 ** -22 * np.linalg.norm(mass)


def _case(tokens, m, n, count, rank, of, ranks=None, scales=True, f32=False, owner=None, seqs=0, seed=0, **more):
    rng = np.random.default_rng(seed + tokens * 31 + m + n)
    a = Set(rng, m, n, count, rank, ranks, scales)
    x = rng.standard_normal((tokens, n)).astype(np.float16)
    base = rng.standard_normal((tokens, m)).astype(np.float32 if f32 else np.float16)
    mine = of if owner is None else [of[s] if 0 <= s < seqs else -1 for s in owner]
    y = _run(a, x, base, of, owner, seqs, f32, **more)
    ref, reach, mass = S.adapt(x, base, a.down, a.up, a.ranks, a.scales, mine)
    _check(y, ref, reach, mass, f32, n, rank)
    none = [t for t, k in enumerate(mine) if not 0 <= k < count]
    np.testing.assert_array_equal(y[none], base[none])
    return a, x, base, mine, y


@pytest.mark.parametrize("tokens,m,n,count,rank,f32", [
    (1, 1, 8, 1, 8, False), (1, 16, 32, 1, 16, True), (2, 17, 40, 2, 8, False), (3, 100, 264, 3, 24, True), (16, 64, 512, 1, 16, False), (17, 80, 520, 1, 32, False),
    (33, 255, 1032, 2, 40, True), (5, 257, 4104, 4, 64, False), (64, 130, 136, 5, 16, False), (65, 130, 136, 5, 16, False), (31, 300, 96, 40, 72, True),
    (100, 70, 600, 7, 128, False), (128, 64, 72, 33, 16, True), (129, 68, 72, 3, 24, False), (256, 36, 40, 70, 8, True), (256, 36, 40, 256, 8, False), (257, 36, 40, 31, 8, True), (9, 1000, 2048, 3, 256, True), (300, 333, 264, 3, 64, False), (1000, 90, 72, 1, 8, False), (130, 515, 1288, 100, 16, False),
    (2100, 40, 64, 1024, 8, True), (1, 5120, 12288, 2, 16, False), (24, 900, 8192, 24, 16, False)])
def test_against_oracle(tokens, m, n, count, rank, f32):
    rng = np.random.default_rng(tokens)
    for spread in ("any", "each", "one"):
        of = rng.integers(-1, count + 1, tokens) if spread == "any" else np.arange(tokens) % count if spread == "each" else np.full(tokens, count - 1)
        print("case adapt", tokens, m, n, count, rank, f32, spread, flush=True)
        _case(tokens, m, n, count, rank, of, f32=f32)


@pytest.mark.parametrize("rank", [8, 16, 24, 32, 48, 64, 72, 128, 136, 256])
@pytest.mark.parametrize("tokens,count", [(64, 1), (60, 2), (70, 1), (200, 2), (141, 3)])
def test_tiles_of_every_size(tokens, count, rank):
    """16, 32 and 64 tokens to a tile, full, of up to four and of up to sixteen; rows of four elements and of any; results over base and beside it."""
    for m, f32, in_place in ((340, False, False), (340, True, True), (1028, True, False), (341, False, True)):
        tile = L.lutgemm_plan_adapt(L.lutgemm_adapters(16, 16, None, None, m, 264, count, rank), tokens)[0]
        assert tile == (16 if rank > 128 else 64 if tokens // count >= 48 else 32)
        for of in (np.arange(tokens) % count, np.where(np.arange(tokens) < 3, 0, -1), np.where(np.arange(tokens) < tile + 9, count - 1, -1)):
            print("case tiles", tokens, count, rank, m, f32, in_place, flush=True)
            _case(tokens, m, 264, count, rank, of, f32=f32, in_place=in_place)


@pytest.mark.parametrize("tokens,count,rank", [(7, 5, 16), (40, 6, 64), (200, 9, 80), (90, 4, 256)])
def test_ranks_of_every_kind(tokens, count, rank):
    """What the stores hold beyond a rank is NaN; an adapter of rank 0 adds nothing."""
    rng = np.random.default_rng(rank)
    ranks = rng.integers(1, rank + 1, count)
    ranks[0], ranks[1], ranks[2] = 0, 1, rank
    print("case ranks", tokens, count, rank, flush=True)
    for scales in (True, False):
        _case(tokens, 200, 328, count, rank, np.arange(tokens) % count, ranks, scales)


@pytest.mark.parametrize("tokens,seqs", [(1, 1), (20, 3), (64, 64), (64, 7), (500, 13)])
def test_tokens_of_sequences(tokens, seqs):
    """owner says whose a token is: rows behind the last sequence, and owners out of range, have no adapter."""
    rng = np.random.default_rng(tokens)
    owner = np.sort(rng.integers(0, seqs, tokens))
    if tokens > 10:
        owner[-5:] = -1
        owner[3], owner[4] = seqs, -(1 << 31)
    of = rng.integers(0, 4, seqs)
    of[seqs // 2] = -1
    print("case owner", tokens, seqs, flush=True)
    _case(tokens, 96, 256, 4, 16, of, owner=owner, seqs=seqs)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("tokens", [3, 90])
def test_strides_alignments_and_in_place(tokens, f32):
    of = np.arange(tokens) % 4 - 1
    for more in [dict(in_place=True), dict(x_stride=264 + 72, base_stride=160, y_stride=168), dict(base_stride=131, y_stride=137, offset=1), dict(base_stride=136, offset=3, in_place=True),
                 dict(base_stride=136, y_stride=129)]:
        print("case strides", tokens, f32, more, flush=True)
        _case(tokens, 129, 264, 3, 24, of, f32=f32, **more)


@pytest.mark.parametrize("rank", [16, 40, 128])
@pytest.mark.parametrize("tokens,count", [(2, 1), (30, 2), (70, 1), (96, 3), (300, 2)])
def test_ends_of_rows(tokens, count, rank):
    """Rows that end anywhere in a run of four, shorter ones too, that begin on any value's bytes; tokens without an adapter among them."""
    for k, m in enumerate((1, 2, 3, 4, 5, 6, 7, 62, 63, 65, 127, 129, 130, 255, 513, 514, 515, 517)):
        f32, in_place = k % 2 == 1, k % 3 == 0
        print("case ends", tokens, count, rank, m, f32, in_place, flush=True)
        for more in (dict(), dict(base_stride=m + 1 + k % 4, offset=k % 4)):
            _case(tokens, m, 72, count, rank, np.arange(tokens) % (count + 1), f32=f32 != bool(more), in_place=in_place, **more)


@pytest.mark.parametrize("tokens", [12, 80])
def test_large_and_special_values(tokens):
    """A_a x beyond fp16's range, far below it, infinities and NaNs in one token and one adapter, which the others do not see."""
    torch = torch_cuda()
    rng = np.random.default_rng(tokens)
    m, n, count, rank = 70, 520, 3, 16
    a = Set(rng, m, n, count, rank, scales=False)
    a.down[0] = (rng.standard_normal((rank, n)) * 30).astype(np.float16)
    a.up[0] = (rng.standard_normal((m, rank)) * 2.0 ** -14).astype(np.float16)
    a.down[1] = (rng.standard_normal((rank, n)) * 2.0 ** -20).astype(np.float16)
    a.up[1] = (rng.standard_normal((m, rank)) * 1000).astype(np.float16)
    a.down[2, 3, 5] = np.inf
    for d, h in zip(a.d, (a.down, a.up)):
        d.copy_(torch.from_numpy(h))
    x = rng.standard_normal((tokens, n)).astype(np.float16)
    x[::3] *= 300                                  # adapter 0's tokens: products of some 10^5
    x[1, 7], x[4, 9] = np.nan, -np.inf             # two tokens of adapter 1
    base = rng.standard_normal((tokens, m)).astype(np.float32)
    of = np.arange(tokens) % 3
    y = _run(a, x, base, of, f32=True)
    fine = [t for t in range(tokens) if of[t] != 2 and t not in (1, 4)]
    ref, reach, mass = S.adapt(x[fine], base[fine], a.down, a.up, None, None, of[fine])
    _check(y[fine], ref, reach, mass, True, n, rank)
    assert not np.isfinite(y[[1, 4]]).any() and not np.isfinite(y[of == 2]).any()


@pytest.mark.parametrize("tokens,count,spread", [(8192, 3, "any"), (9000, 5, "any"), (9000, 1, "one"), (20000, 40, "each")])
def test_many_tokens(tokens, count, spread):
    """More than the sorting keeps in registers, and as many: small products, in numpy."""
    rng = np.random.default_rng(tokens + count)
    m, n, rank = 24, 16, 8
    of = rng.integers(-1, count + 1, tokens) if spread == "any" else np.arange(tokens) % count if spread == "each" else np.zeros(tokens, int)
    print("case many", tokens, count, spread, flush=True)
    a = Set(rng, m, n, count, rank)
    x, base = rng.standard_normal((tokens, n)).astype(np.float16), rng.standard_normal((tokens, m)).astype(np.float32)
    y = _run(a, x, base, of, f32=True)
    live = (of >= 0) & (of < count)
    pick = np.where(live, of, 0)
    h = np.einsum("trn,tn->tr", a.down.astype(np.float64)[pick], x.astype(np.float64))
    c = np.where(live, a.scales.astype(np.float64)[pick], 0.0)[:, None]
    ref = base + c * np.einsum("tmr,tr->tm", a.up.astype(np.float64)[pick], h)
    reach = c * np.einsum("tmr,trn,tn->tm", np.abs(a.up.astype(np.float64))[pick], np.abs(a.down.astype(np.float64))[pick], np.abs(x.astype(np.float64)))
    mass = c * np.abs(a.up.astype(np.float64))[pick].sum(2) * np.abs(h).max(1)[:, None]
    _check(y, ref, reach, mass, True, n, rank)
    np.testing.assert_array_equal(y[~live], base[~live])


def test_an_infinite_weight_stays_in_its_row():
    """One row of B: its own results are no numbers, those of the others what they are without it (also of ranks that share an instruction)."""
    torch = torch_cuda()
    for rank in (8, 16, 32, 64, 128):
        rng = np.random.default_rng(rank)
        a = Set(rng, 200, 64, 1, rank, scales=False)
        x, base = rng.standard_normal((5, 64)).astype(np.float16), rng.standard_normal((5, 200)).astype(np.float32)
        before = _run(a, x, base, [0] * 5, f32=True)
        a.d[1][0, 70, 1] = float("inf")
        y = _run(a, x, base, [0] * 5, f32=True)
        assert not np.isfinite(y[:, 70]).any()
        np.testing.assert_array_equal(np.delete(y, 70, 1), np.delete(before, 70, 1))


def test_the_same_from_run_to_run_and_beside_others():
    """Bitwise: again, on another stream, and for a token whose neighbours have other values."""
    torch = torch_cuda()
    a, x, base, of, y = _case(50, 400, 1544, 5, 32, np.arange(50) % 5)
    side = torch.cuda.Stream()
    np.testing.assert_array_equal(_run(a, x, base, of, stream=side), y)
    other = x.copy()
    other[1:] = np.float16(3)
    np.testing.assert_array_equal(_run(a, other, base, of)[0], y[0])


@pytest.mark.parametrize("tokens", [6, 100])
def test_a_captured_call_is_replayed_with_other_adapters(tokens):
    torch = torch_cuda()
    rng = np.random.default_rng(1)
    m, n, count, rank = 300, 640, 6, 16
    a = Set(rng, m, n, count, rank)
    x = torch.from_numpy(rng.standard_normal((tokens, n)).astype(np.float16)).cuda()
    base = torch.from_numpy(rng.standard_normal((tokens, m)).astype(np.float16)).cuda()
    of, y = torch.zeros(tokens, dtype=torch.int32, device="cuda"), torch.empty_like(base)
    nbytes = L.lutgemm_adapt_workspace_bytes(a.handle, tokens)
    ws = make_workspace(nbytes)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        L.lutgemm_adapt(x, base, a.handle, of, None, y, tokens, 0, n, m, m, 0, ws, nbytes, torch.cuda.current_stream().cuda_stream)
    for k in range(5):
        mine = rng.integers(-1, count, tokens).astype(np.int32)
        of.copy_(torch.from_numpy(mine))
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        L.lutgemm_adapt(x, base, a.handle, of, None, y, tokens, 0, n, m, m, 0, ws, nbytes, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert torch.equal(got, y)
        ref, reach, mass = S.adapt(x.cpu().numpy(), base.cpu().numpy(), a.down, a.up, None, a.scales, mine)
        _check(got.cpu().numpy(), ref, reach, mass, False, n, rank)


def test_offsets_beyond_32_bits():
    """Rows of base and y 2^31 bytes apart; an adapter that begins 2^32 bytes and more into the store of B."""
    torch = torch_cuda()
    rng = np.random.default_rng(2)
    m, n, rank = 260, 64, 16
    a = Set(rng, m, n, 2, rank)
    x = rng.standard_normal((4, n)).astype(np.float16)
    base = rng.standard_normal((4, m)).astype(np.float16)
    stride = (1 << 30) + 8
    d_base, d_y = (torch.empty(3 * stride + m, dtype=torch.float16, device="cuda") for _ in range(2))
    for t in range(4):
        d_base[t * stride:t * stride + m] = torch.from_numpy(base[t]).cuda()
    of = torch.tensor([0, 1, -1, 1], dtype=torch.int32, device="cuda")
    ws = make_workspace(L.lutgemm_adapt_workspace_bytes(a.handle, 4))
    stream = torch.cuda.current_stream().cuda_stream
    L.lutgemm_adapt(torch.from_numpy(x).cuda(), d_base, a.handle, of, None, d_y, 4, 0, n, stride, stride, 0, ws, ws.numel(), stream)
    torch.cuda.synchronize()
    y = np.stack([d_y[t * stride:t * stride + m].cpu().numpy() for t in range(4)])
    _check(y, *S.adapt(x, base, a.down, a.up, None, a.scales, of.tolist()), False, n, rank)
    del d_base, d_y
    m, rank, count = 1 << 20, 256, 9               # 2^29 bytes an adapter
    down = torch.zeros(count, rank, 8, dtype=torch.float16, device="cuda")
    up = torch.empty(count, m, rank, dtype=torch.float16, device="cuda")
    down[8] = torch.randn(rank, 8, device="cuda").half()
    up[8] = torch.randn(m, rank, device="cuda", dtype=torch.float16)
    handle = L.lutgemm_adapters(down, up, None, None, m, 8, count, rank)
    x, zero, y = torch.randn(1, 8, device="cuda").half(), torch.zeros(1, m, device="cuda"), torch.empty(1, m, device="cuda")
    ws = make_workspace(L.lutgemm_adapt_workspace_bytes(handle, 1))
    L.lutgemm_adapt(x, zero, handle, torch.tensor([8], dtype=torch.int32, device="cuda"), None, y, 1, 0, 8, m, m, L.LUTGEMM_Y_F32, ws, ws.numel(), stream)
    torch.cuda.synchronize()
    some = np.r_[0:100, m // 2:m // 2 + 100, m - 100:m]
    h_up = up[8][torch.from_numpy(some).cuda()].cpu().numpy()[None]
    ref, reach, mass = S.adapt(x.cpu().numpy(), np.zeros((1, len(some)), np.float32), down[8:].cpu().numpy(), h_up, None, None, [0])
    _check(y[:, torch.from_numpy(some).cuda()].cpu().numpy(), ref, reach, mass, True, 8, rank)


def test_graphs_that_share_a_workspace():
    """Two captured calls of different sizes and a product, in turn on one workspace, with the program's own calls between the replays."""
    torch = torch_cuda()
    rng = np.random.default_rng(12)
    m, n = 512, 640
    a = Set(rng, m, n, 4, 16)
    W = (rng.standard_normal((m, n)) * 0.05).astype(np.float16)
    bits, alpha, _ = L.lutgemm_pack_bcq(W, 3, 128)
    d_bits, d_alpha = torch.from_numpy(bits).cuda(), torch.from_numpy(alpha.view(np.int16)).cuda()
    nbytes = max(L.lutgemm_adapt_workspace_bytes(a.handle, 130), L.lutgemm_workspace_bytes(m, n, 3, 128, 8, 6))
    ws = make_workspace(nbytes)
    sets = []
    for tokens in (6, 130):
        x = torch.from_numpy(rng.standard_normal((tokens, n)).astype(np.float16)).cuda()
        of = torch.from_numpy((np.arange(tokens) % 5 - 1).astype(np.int32)).cuda()
        sets.append((tokens, x, torch.zeros(tokens, m, dtype=torch.float16, device="cuda"), of))

    def call(k):
        tokens, x, y, of = sets[k]
        s = torch.cuda.current_stream().cuda_stream
        if k == 0:
            L.lutgemm_gemm(x, d_bits, d_alpha, None, y, 3, 128, 8, m, n, tokens, 0, ws, nbytes, s)
        else:
            y.zero_()
        L.lutgemm_adapt(x, y, a.handle, of, None, y, tokens, 0, n, m, m, 0, ws, nbytes, s)

    want = []
    for k in range(2):
        call(k)
        torch.cuda.synchronize()
        want.append(sets[k][2].clone())
    graphs = []
    for k in range(2):
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=side):
            call(k)
        graphs.append(graph)
    for turn in range(6):
        for k in (0, 1, 1, 0):
            sets[k][2].fill_(float("nan"))
            graphs[k].replay()
            if turn % 2:
                torch.cuda.synchronize()
            assert torch.equal(sets[k][2], want[k])
            call(1 - k)
            assert torch.equal(sets[1 - k][2], want[1 - k])


def test_no_tokens():
    torch = torch_cuda()
    a = Set(np.random.default_rng(0), 32, 64, 2, 8)
    y = torch.full((4, 32), float(MARK), dtype=torch.float16, device="cuda")
    ws = make_workspace(L.lutgemm_adapt_workspace_bytes(a.handle, 0))
    L.lutgemm_adapt(y, y, a.handle, torch.zeros(4, dtype=torch.int32, device="cuda"), None, y, 0, 0, 64, 32, 32, 0, ws, ws.numel(),
                    torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert (y == MARK).all()
