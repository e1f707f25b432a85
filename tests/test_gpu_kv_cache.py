"""The paged 8-bit cache on the GPU against 64 bits: appending with the rotation on the way, and reading
back. Scales and codes have to be those of the reference, bit for bit."""
import math

import pytest
import torch

import kv_ref as R
from gpu_util import say
from paper_2510_03425_amd import device as D

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


class Setup:
    """A pool with random contents on the GPU and as the reference has it, and a batch."""

    def __init__(self, gpu, heads, dim, page, past, new, seed=0, spare=2, max_new=None, max_len=None, tail=0):
        g = self.gen = torch.Generator().manual_seed(seed + 17 * dim + page)
        self.gpu, self.heads, self.dim = gpu, heads, dim
        self.past, self.new = past, new
        cols = max(1, max(-(-(a + b) // page) for a, b in zip(past, new)))
        n = len(past) * cols + spare
        shape = (n, heads, page // 16, 2)
        pages = torch.randint(-127, 128, (*shape, 16 * dim), generator=g, dtype=torch.int8)
        scales = torch.exp(torch.randn(shape, generator=g) * 0.5) * 0.02
        self.table = torch.randperm(n, generator=g)[:len(past) * cols].view(len(past), cols).to(torch.int32)
        self.ref = R.Cache(pages, scales)
        self.cache = D.KvCache(pages.to(gpu), scales.to(gpu))
        self.start = [0]
        for x in new:
            self.start.append(self.start[-1] + x)
        self.rows = self.start[-1] + tail
        self.max_new, self.max_len = max_new or max(1, *new), max_len or max(1, *(a + b for a, b in zip(past, new)))
        self.batch = self.make_batch(self.start, past)

    def make_batch(self, start, past, max_new=None):
        def i32(v):
            return torch.tensor(v, dtype=torch.int32, device=self.gpu)

        return D.KvBatch(i32(start), i32(past), self.table.to(self.gpu), max_new or self.max_new, self.max_len)

    def heads_of(self, h, dtype, std=1.0, n=None):
        return (torch.randn(self.rows if n is None else n, h, self.dim, generator=self.gen) * std).to(dtype)

    def append_ref(self, k, v, tab=None, inter=False):
        for s, (past, new) in enumerate(zip(self.past, self.new)):
            rows = slice(self.start[s], self.start[s] + min(new, self.max_new))
            kk = k[rows].double()
            if tab is not None:
                kk = R.turn(kk, tab, torch.arange(past, past + kk.shape[0]), inter)
            self.ref.append(self.table[s], past, kk, v[rows].double())

    def same(self):
        s = self.cache.scales.cpu()
        assert torch.equal(s.isnan(), self.ref.scales.isnan()) and torch.equal(s.nan_to_num(7), self.ref.scales.nan_to_num(7)), "scales"
        # codes of tokens that sequences have; those behind a sequence's end are nobody's
        for i, (past, new) in enumerate(zip(self.past, self.new)):
            for t in range(past + min(new, self.max_new)):
                at = self.ref.where(self.table[i], t)
                if at is None:
                    continue
                mine = R.Cache.codes(self.gpu_codes, *at)
                for a, b, what in zip(mine, self.ref.codes(*at), "kv"):
                    assert torch.equal(a[:, t % 16], b[:, t % 16]), (what, i, t)

    @property
    def gpu_codes(self):
        c = R.Cache.__new__(R.Cache)
        c.pages, c.heads, c.dim = self.cache.pages.cpu(), self.heads, self.dim
        return c


BATCHES = [  # past, new
    ([0], [1]), ([0], [16]), ([0], [17]), ([15], [1]), ([16], [1]), ([5], [3]), ([31, 0, 7, 100], [1, 1, 1, 1]), ([0, 3, 64, 50], [40, 0, 1, 33]),
    ([12], [70]), ([1000, 1], [2, 129]),
]


@pytest.mark.parametrize("past,new", BATCHES)
@pytest.mark.parametrize("heads,dim,page,dtype,rot,inter", [
    (2, 64, 16, F16, 64, False), (1, 256, 64, BF16, 256, False), (2, 128, 32, F32, 96, False), (3, 64, 128, BF16, 26, True),
    (1, 128, 16, F16, 128, True), (2, 256, 256, F32, 60, False),
])
def test_append(built_lib, gpu, past, new, heads, dim, page, dtype, rot, inter):
    say("append", past, new, heads, dim, page, dtype, rot, inter)
    t = Setup(gpu, heads, dim, page, past, new, seed=sum(past))
    tab = R.table(t.max_len + 3, rot, 1e4).float()
    rope = D.Rope(tab.to(gpu), dim, inter)
    k, v, q = t.heads_of(heads, dtype, 2.0), t.heads_of(heads, dtype, 0.3), t.heads_of(5, dtype)
    q_out = D.kv_append(t.cache, t.batch, k.to(gpu), v.to(gpu), rope, q.to(gpu))
    t.append_ref(k, v, tab, inter)
    t.same()
    pos = torch.cat([torch.arange(a, a + b) for a, b in zip(past, new)])
    R.check(q_out, R.turn(q, tab, pos, inter), R.turn_bound(q, tab, pos, inter, dtype), "q")
    # what it stands for, read back from every sequence's beginning
    rows = [0]
    for a, b in zip(past, new):
        rows.append(rows[-1] + a + b)
    back = t.make_batch(rows, [0] * len(past), max(1, max(a + b for a, b in zip(past, new))))
    for out in (F32, dtype):
        ko, vo = (torch.full((rows[-1] + 2, heads, dim), 9.0, dtype=out, device=gpu) for _ in range(2))
        D.kv_read(t.cache, back, ko, vo)
        for s in range(len(past)):
            kr, vr = t.ref.read(t.table[s], 0, rows[s + 1] - rows[s])
            for got, ref in ((ko, kr), (vo, vr)):
                R.check(got[rows[s]:rows[s + 1]], ref, ref.abs() * (R.EPS + R.HALF_STEP[out] * (1 + R.EPS)) + 2.0 ** -25, "read")
        assert bool((ko[rows[-1]:] == 9.0).all()) and bool((vo[rows[-1]:] == 9.0).all())
        alone = torch.empty_like(vo)
        D.kv_read(t.cache, back, None, alone)
        assert torch.equal(alone[:rows[-1]], vo[:rows[-1]])


@pytest.mark.parametrize("dim,dtype", [(64, F16), (128, BF16), (256, F32)])
def test_token_by_token(built_lib, gpu, dim, dtype):
    """Blocks that grow: earlier codes are rounded again as the scale rises, and pages follow one another."""
    t = Setup(gpu, 2, dim, 16, [3], [0], max_new=1, max_len=64)
    t.table = torch.tensor([[1, 0, 2, 3]], dtype=torch.int32)
    t.ref = R.Cache(torch.randint(-127, 128, (4, 2, 1, 2, 16 * dim), generator=t.gen, dtype=torch.int8), torch.rand(4, 2, 1, 2, generator=t.gen))
    t.cache = D.KvCache(t.ref.pages.to(gpu), t.ref.scales.to(gpu))
    tab = R.table(64, dim, 1e4).float()
    rope = D.Rope(tab.to(gpu), dim)
    t.start, t.rows = [0, 1], 1
    b = t.make_batch([0, 1], [3])
    for i in range(3, 40):
        t.past, t.new = [i], [1]
        k, v = t.heads_of(2, dtype, 1.0 + i % 7), t.heads_of(2, dtype, 0.1 * (1 + i % 5))
        D.kv_append(t.cache, b, k.to(gpu), v.to(gpu), rope)
        b.past += 1
        t.append_ref(k, v, tab)
        t.same()


def test_strided_operands_and_rows_behind(built_lib, gpu):
    t = Setup(gpu, 2, 64, 32, [9, 40], [5, 20], tail=6)
    tab = R.table(70, 64, 1e4).float()
    rope = D.Rope(tab.to(gpu), 64)
    for gap in (0, 1):  # rows of one matrix q | k | v, at 16-byte addresses or not
        whole = torch.randn(t.rows, 8 * 64 + gap, generator=t.gen).half()
        d = whole.to(gpu)
        q, k, v = (d[:, a * 64:b * 64].view(t.rows, b - a, 64) for a, b in ((0, 4), (4, 6), (6, 8)))
        D.kv_append(t.cache, t.batch, k, v, rope, q, q)
        host = [whole[:, a * 64:b * 64].reshape(t.rows, b - a, 64) for a, b in ((0, 4), (4, 6), (6, 8))]
        t.append_ref(host[1], host[2], tab)
        t.same()
        pos = torch.cat([torch.arange(9, 14), torch.arange(40, 60)])
        R.check(q[:25], R.turn(host[0][:25], tab, pos), R.turn_bound(host[0][:25], tab, pos, False, F16), "q in place")
        # rows of no sequence, and the keys and values themselves, are as they were
        assert torch.equal(q[25:].cpu(), host[0][25:]) and torch.equal(d[:, 256:].cpu(), whole[:, 256:])


def test_values_at_their_ends(built_lib, gpu):
    """Zeros, subnormal and huge numbers, ties of the rounding, NaN and infinities: in blocks of their own."""
    t = Setup(gpu, 2, 64, 16, [0], [16 * 9])
    k, v = t.heads_of(2, F32), t.heads_of(2, F32)
    for x in (k, v):
        x[0:16] = 0
        x[16:32] *= 1e-44
        x[32:48] *= 1e-38
        x[48:64] = x[48:64].clamp(-3, 3) * 1e38
        x[64:80] = torch.randint(-127, 128, (16, 2, 64), generator=t.gen) + 0.5  # of a block's scale 1:
        x[64:80, :, 0] = 127.0
        x[64:80] = x[64:80].clamp(-127, 127)
        x[80, 0, 5], x[97, 1, 6], x[113, 0, 7] = math.nan, math.inf, -math.inf
        x[128:144, 0] = 5.0
    D.kv_append(t.cache, t.batch, k.to(gpu), v.to(gpu))
    t.append_ref(k, v)
    t.same()
    assert int(t.ref.scales.isnan().sum()) == 6


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_values_beside_the_borders_of_codes(built_lib, gpu, dim):
    """Quotients on the border of two codes, and one and a few steps of fp32 to either side of it."""
    n = 16 * 40
    t = Setup(gpu, 2, dim, 16, [0], [n])
    both = []
    for _ in range(2):
        most = torch.exp(8 * torch.randn(n // 16, 1, 2, 1, generator=t.gen, dtype=torch.float64)).float()
        scale = (most.double() / 127).float().double()
        x = ((torch.randint(-127, 127, (n // 16, 16, 2, dim), generator=t.gen) + 0.5) * scale).float()
        step = torch.randint(-3, 4, x.shape, generator=t.gen, dtype=torch.int32)
        x = (x.view(torch.int32) + step).view(torch.float32)
        x = torch.minimum(torch.maximum(x, -most), most)
        x[:, 3, :, 7] = most[:, 0, :, 0]
        both.append(x.reshape(n, 2, dim))
    D.kv_append(t.cache, t.batch, both[0].to(gpu), both[1].to(gpu))
    t.append_ref(*both)
    t.same()


def test_two_graphs_of_one_cache(built_lib, gpu):
    """Steps of different widths, each a graph, in turn: each continues what the other wrote."""
    t = Setup(gpu, 2, 128, 32, [0, 0], [0, 0], max_new=5, max_len=128)
    tab = R.table(128, 128, 1e4).float()
    rope = D.Rope(tab.to(gpu), 128)
    steps = []
    for new in ([3, 5], [1, 1]):
        rows = sum(new)
        k, v = (torch.zeros(rows, 2, 128, dtype=F16, device=gpu) for _ in range(2))
        b = t.make_batch([0, new[0], rows], [0, 0])
        steps.append([new, k, v, b, None])
    for st in steps:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            D.kv_append(t.cache, st[3], st[1], st[2], rope)
        st[4] = graph
    past = [0, 0]
    for i in range(12):
        new, k, v, b, graph = steps[i % 2]
        kh, vh = (torch.randn(*k.shape, generator=t.gen).mul_(1 + i % 4).half() for _ in range(2))
        k.copy_(kh), v.copy_(vh), b.past.copy_(torch.tensor(past, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        t.past, t.new, t.start = list(past), new, [0, new[0], sum(new)]
        t.append_ref(kh, vh, tab)
        t.same()
        past = [a + c for a, c in zip(past, new)]


def test_scale_that_was_nan_or_zero(built_lib, gpu):
    t = Setup(gpu, 1, 64, 16, [4, 4, 0], [2, 2, 2])
    for s, x in ((0, math.nan), (1, 0.0), (2, math.nan)):  # (of the last the block's first token is new)
        p = int(t.table[s][0])
        t.ref.scales[p] = x
        t.cache.scales[p] = x
    k, v = t.heads_of(1, F16), t.heads_of(1, F16)
    D.kv_append(t.cache, t.batch, k.to(gpu), v.to(gpu))
    t.append_ref(k, v)
    t.same()


def test_pages_that_are_not_there(built_lib, gpu):
    """Ids outside the pool and columns beyond the table: nothing is stored, and reads are NaN."""
    t = Setup(gpu, 2, 64, 16, [0, 10, 0], [40, 30, 5])
    t.table[0, 1], t.table[1, 0], t.table[2, 0] = -1, t.ref.n, 2 ** 31 - 1
    t.batch = t.make_batch(t.start, t.past)
    before = t.cache.pages.clone()
    k, v = t.heads_of(2, F16), t.heads_of(2, F16)
    D.kv_append(t.cache, t.batch, k.to(gpu), v.to(gpu))
    t.append_ref(k, v)
    t.same()
    used = {int(p) for row, n in zip(t.table, (3, 3, 1)) for p in row[:n]}
    for p in range(t.ref.n):
        if p not in used:
            assert torch.equal(t.cache.pages[p], before[p])
    # a sequence longer than its table
    long = t.make_batch([0, 60, 60, 60], [0, 0, 0], 64)
    ko, vo = (torch.zeros(60, 2, 64, device=gpu) for _ in range(2))
    D.kv_read(t.cache, long, ko, vo)
    kr, vr = t.ref.read(t.table[0], 0, 40)  # (what lies behind it in its last block is nobody's)
    assert kr[16:32].isnan().all()
    R.check(ko[:40], kr, kr.abs() * R.EPS, "k")
    R.check(vo[:40], vr, vr.abs() * R.EPS, "v")
    assert ko[48:].isnan().all() and vo[48:].isnan().all()


def test_odd_batches(built_lib, gpu):
    """More new tokens than max_new, starts and lengths out of their range: what is there is done, and
    nothing outside of it is touched."""
    t = Setup(gpu, 1, 64, 16, [0, 0], [40, 8], max_new=33)
    k, v = t.heads_of(1, F16), t.heads_of(1, F16)
    D.kv_append(t.cache, t.batch, k.to(gpu), v.to(gpu))
    t.append_ref(k, v)
    t.same()
    before = [t.cache.pages.clone(), t.cache.scales.clone()]
    for start, past in (([0, -5, -9], [0, 0]), ([60, 70, 80], [0, 0]), ([9, 3, 3], [0, 0]), ([0, 5, 5], [2 ** 31 - 1, 0])):
        D.kv_append(t.cache, t.make_batch(start, past), k.to(gpu), v.to(gpu))
    torch.cuda.synchronize()
    assert torch.equal(t.cache.pages, before[0]) and torch.equal(t.cache.scales, before[1])


def test_positions_beyond_the_table(built_lib, gpu):
    t = Setup(gpu, 1, 64, 16, [14], [4])
    tab = R.table(16, 64, 1e4).float()
    k, v, q = (t.heads_of(1, F16) for _ in range(3))
    got = D.kv_append(t.cache, t.batch, k.to(gpu), v.to(gpu), D.Rope(tab.to(gpu), 64), q.to(gpu))
    t.append_ref(k, v, tab)
    t.same()
    assert got[:2].isfinite().all() and got[2:].isnan().all()
    assert bool(t.cache.scales[int(t.table[0, 1]), 0, 0, 0].isnan()) and not bool(t.cache.scales[int(t.table[0, 1]), 0, 0, 1].isnan())


def test_pool_beyond_32_bits(built_lib, gpu):
    """Pages whose bytes lie beyond 2^31 and 2^32."""
    n = 70000
    cache = D.KvCache.empty(n, 64, 2, 256, gpu)  # 65536 bytes a page: 4.6 GB
    table = torch.tensor([[n - 1, 3], [40000, 65537]], dtype=torch.int32, device=gpu)

    def i32(*v):
        return torch.tensor(v, dtype=torch.int32, device=gpu)

    b = D.KvBatch(i32(0, 70, 165), i32(0, 3), table, 95, 128)
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn(165, 2, 256, generator=g).half() for _ in range(2))
    D.kv_append(cache, b, k.to(gpu), v.to(gpu))
    ko, vo = (torch.zeros(165, 2, 256, device=gpu) for _ in range(2))
    D.kv_read(cache, b, ko, vo)
    for x, y in ((k, ko), (v, vo)):
        # half a code of the largest magnitude (of two roundings for none: blocks are written once)
        assert float((x.double() - y.double().cpu()).abs().max()) <= float(x.abs().max()) / 254 * (1 + 2.0 ** -20)


def test_graph_and_streams(built_lib, gpu):
    """A captured decoding step: lengths move on the device between replays; eager work goes on beside it."""
    t = Setup(gpu, 2, 128, 32, [5, 30], [1, 1], max_new=1, max_len=64)
    t.table = torch.tensor([[0, 1], [2, 3]], dtype=torch.int32)
    b = t.make_batch([0, 1, 2], [5, 30])
    tab = R.table(64, 128, 1e4).float()
    rope = D.Rope(tab.to(gpu), 128)
    k, v = (torch.zeros(2, 2, 128, dtype=BF16, device=gpu) for _ in range(2))
    q, qo = (torch.zeros(2, 6, 128, dtype=BF16, device=gpu) for _ in range(2))
    D.kv_append(t.cache, b, k, v, rope, q, qo)  # (rows of zeros raise nothing that the next ones do not)
    t.append_ref(k.cpu(), v.cpu(), tab)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        D.kv_append(t.cache, b, k, v, rope, q, qo)
        b.past += 1
    for i in range(6):
        t.past = [5 + i, 30 + i]
        kk, vv, qq = t.heads_of(2, BF16), t.heads_of(2, BF16), t.heads_of(6, BF16)
        for dst, src in ((k, kk), (v, vv), (q, qq)):
            dst.copy_(src)
        graph.replay()
        torch.cuda.synchronize()
        t.append_ref(kk, vv, tab)
        t.same()
        pos = torch.tensor(t.past)
        R.check(qo, R.turn(qq, tab, pos), R.turn_bound(qq, tab, pos, False, BF16), "q")
