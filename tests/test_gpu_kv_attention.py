"""Attention over the paged 8-bit cache on the GPU against 64 bits."""
import math

import pytest
import torch

import kv_ref as R
from gpu_util import say
from paper_2510_03425_amd import _lib as L
from paper_2510_03425_amd import device as D
from test_gpu_kv_cache import Setup

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


def _run(t, q, window=0, scale=None, rows=None, batch=None, ws=None):
    n, hq, d = q.shape
    out = torch.full((n, hq, d), 3.0, dtype=q.dtype, device=t.gpu)
    lse = torch.full((n, hq), 3.0, device=t.gpu)
    D.kv_attention(t.cache, batch or t.batch, q.to(t.gpu), out, lse, scale, window, ws)
    return out, lse


def _check(t, q, out, lse, window=0, scale=None):
    scale = t.dim ** -0.5 if scale is None else scale
    for s, (past, new) in enumerate(zip(t.past, t.new)):
        rows = slice(t.start[s], t.start[s] + min(new, t.max_new))
        n = rows.stop - rows.start
        if not n:
            continue
        k, v = t.ref.read(t.table[s], 0, past + n)
        o, e, ob, eb = R.attention(q[rows], k, v, past, scale, window)
        R.check(lse[rows], e, eb, f"lse of sequence {s}")
        R.check(out[rows], o, ob * (1 + R.HALF_STEP[q.dtype]) + o.abs().nan_to_num(0) * R.HALF_STEP[q.dtype] + 2.0 ** -25, f"out of sequence {s}")
    assert bool((out[t.start[-1]:] == 3.0).all()) and bool((lse[t.start[-1]:] == 3.0).all())


# single tokens, a few, chunks and prompts; lengths of one, around blocks, tiles and pages
BATCHES = [
    ([0], [1]), ([15, 16, 17], [1, 1, 1]), ([62, 63, 64, 0], [1, 1, 1, 1]), ([300, 5, 1000], [1, 1, 1]), ([0], [70]), ([40, 0, 200], [3, 9, 1]),
    ([0, 130], [64, 33]), ([3000], [1]), ([777], [130]),
]
SHAPES = [  # kv heads, query heads, dim, page, dtype
    (2, 4, 64, 16, F16), (2, 14, 64, 64, BF16), (2, 12, 128, 32, F16), (1, 4, 256, 64, BF16), (4, 8, 256, 16, F16), (1, 1, 128, 256, BF16),
    (1, 33, 64, 32, F16),
]


@pytest.mark.parametrize("past,new", BATCHES)
@pytest.mark.parametrize("hkv,hq,dim,page,dtype", SHAPES)
def test_attention(built_lib, gpu, past, new, hkv, hq, dim, page, dtype):
    say("attention", past, new, hkv, hq, dim, page, dtype)
    t = Setup(gpu, hkv, dim, page, past, new, seed=sum(past) + hq, tail=3)
    q = t.heads_of(hq, dtype)
    out, lse = _run(t, q)
    _check(t, q, out, lse)
    again, e2 = _run(t, q)
    assert torch.equal(out, again) and torch.equal(lse, e2)


@pytest.mark.parametrize("past,new", BATCHES)
@pytest.mark.parametrize("hkv,hq,dim,page,dtype", SHAPES)
def test_attention_laid_out_for_long_sequences(built_lib, gpu, past, new, hkv, hq, dim, page, dtype):
    """The same with room for 2^20 tokens, which has many rows by large tiles and several sequences in shares."""
    say("long", past, new, hkv, hq, dim, page, dtype)
    t = Setup(gpu, hkv, dim, page, past, new, seed=sum(past) + hq, tail=3, max_len=1 << 20)
    q = t.heads_of(hq, dtype)
    for window in (0, 70):
        out, lse = _run(t, q, window)
        _check(t, q, out, lse, window)


@pytest.mark.parametrize("hkv,hq,dim,new", [(1, 24, 128, 400), (1, 25, 256, 390), (16, 48, 64, 260), (3, 33, 128, 300)])
def test_windows_of_many_rows(built_lib, gpu, hkv, hq, dim, new):
    """Enough rows for large tiles, their windows in parts; the first of them at the sequence's beginning, or far behind it."""
    for past in (0, 1500):
        t = Setup(gpu, hkv, dim, 64, [past], [new], seed=hq)
        q = t.heads_of(hq, F16)
        for window in (450, 513, 700):
            out, lse = _run(t, q, window)
            _check(t, q, out, lse, window)


@pytest.mark.parametrize("window", [1, 5, 16, 64, 65, 100, 1000])
@pytest.mark.parametrize("hkv,hq,dim,page,dtype", SHAPES[1:5])
def test_window(built_lib, gpu, window, hkv, hq, dim, page, dtype):
    say("window", window, hkv, hq, dim, page)
    t = Setup(gpu, hkv, dim, page, [0, 70, 500, 63], [90, 1, 40, 2], seed=window)
    q = t.heads_of(hq, dtype)
    out, lse = _run(t, q, window)
    _check(t, q, out, lse, window)
    t = Setup(gpu, hkv, dim, page, [0, 70, 500, 63], [1, 1, 1, 1], seed=window)
    q = t.heads_of(hq, dtype)
    out, lse = _run(t, q, window)
    _check(t, q, out, lse, window)


@pytest.mark.parametrize("dim,hq,new", [(64, 4, 1), (128, 2, 40), (256, 2, 1), (256, 2, 200)])
def test_many_parts(built_lib, gpu, dim, hq, new):
    """Long sequences, split over the chip and joined; one of them short."""
    t = Setup(gpu, 1, dim, 64, [9000, 3, 4500], [new, 1, new], seed=dim)
    assert L.mebp_kv_attention_workspace_bytes(3, new, t.max_len, hq, 1, dim) > 256 or new > 100
    q = t.heads_of(hq, BF16)
    out, lse = _run(t, q)
    _check(t, q, out, lse)


def test_sure_and_flat_rows(built_lib, gpu):
    """One key far above the others, early, late and in a block's middle; all alike; scores far apart."""
    for scale in (1.0, 20.0, 1e-4, -1.0):
        for dim, new in ((64, 1), (128, 35), (256, 150)):
            t = Setup(gpu, 1, dim, 32, [400], [new], seed=int(scale * 10))
            q = t.heads_of(2, F16)
            out, lse = _run(t, q, scale=scale)
            _check(t, q, out, lse, scale=scale)


@pytest.mark.parametrize("new", [1, 150])
def test_queries_at_their_ends(built_lib, gpu, new):
    """Rows of zeros, subnormal and huge numbers, and NaN and infinities: rows of their own."""
    t = Setup(gpu, 1, 64, 32, [100], [max(new, 8)] if new > 1 else [8], seed=3, max_new=max(new, 8))
    for dtype, tiny, huge in ((F16, 2.0 ** -22, 6e4), (BF16, 2.0 ** -130, 1e30)):
        q = t.heads_of(3, dtype)
        q[0, 0] = 0
        q[1, 1] = (q[1, 1].float() * tiny).to(dtype)
        q[2, 2] = (q[2, 2].float().clamp(-1, 1) * huge).to(dtype)
        q[3, 0, 5], q[4, 1, 6], q[5, 2, 7] = math.nan, math.inf, -math.inf
        out, lse = _run(t, q)
        bad = torch.zeros(q.shape[0], 3, dtype=torch.bool)
        bad[3, 0] = bad[4, 1] = bad[5, 2] = True
        assert torch.equal(out.isnan().all(2).cpu(), bad) and torch.equal(out.isnan().any(2).cpu(), bad) and torch.equal(lse.isnan().cpu(), bad)
        q[bad] = 0
        big = torch.zeros_like(bad)
        big[2, 2] = True
        o, e = out.clone(), lse.clone()
        # (a row of scores far beyond what its differences can be resolved to in fp32 is all on one key)
        if dtype is F16:
            q[2, 2] = 0
        keep = ~(bad | big)
        k, v = t.ref.read(t.table[0], 0, 100 + t.new[0])
        ro, re, rob, reb = R.attention(q, k, v, 100, 0.125, 0)
        m = keep[..., None].expand_as(ro)
        R.check(e.cpu()[keep], re[keep], reb[keep], "lse")
        R.check(o.cpu()[m], ro[m], (rob + ro.abs() * R.HALF_STEP[dtype])[m] + 2.0 ** -25, "out")
        assert out[2, 2].isfinite().all() and lse[2, 2].isfinite()


@pytest.mark.parametrize("new", [1, 200])
def test_scales_far_apart(built_lib, gpu, new):
    """Blocks whose values are many orders of magnitude apart, the small ones where the weight is and the
    other way round, and blocks of nothing."""
    for case in range(4):
        t = Setup(gpu, 1, 128, 32, [300], [new], seed=case)
        b = torch.arange(t.ref.scales.numel() // 2).view(t.ref.scales.shape[:3])
        size = [torch.where(b % 2 == 0, 1e-6, 1e3), torch.where(b < 8, 1e10, 1e-10), torch.where(b < 8, 1e-10, 1e10), torch.where(b % 3 == 0, 0.0, 1.0)][case]
        t.ref.scales[..., 1] = size * t.ref.scales[..., 1]
        if case == 3:
            t.ref.scales[..., 0] = size * t.ref.scales[..., 0]
        t.cache.scales.copy_(t.ref.scales)
        q = t.heads_of(2, BF16, 0.2)
        out, lse = _run(t, q)
        _check(t, q, out, lse)


@pytest.mark.parametrize("new", [1, 90])
@pytest.mark.parametrize("hkv,hq,dim,page,dtype", SHAPES[:4])
def test_nan_blocks_and_pages_that_are_not_there(built_lib, gpu, new, hkv, hq, dim, page, dtype):
    """A row that sees a block of NaN, or whose page is not there, is NaN; one that does not is what it was."""
    t = Setup(gpu, hkv, dim, page, [250, 300, 280, 260], [new] * 4, seed=11)
    for s, tok, w, x in ((0, 290 if new > 1 else 249, 0, math.nan), (1, 100, 1, math.nan), (2, 330 if new > 1 else 20, 1, math.nan)):
        p, b = t.ref.where(t.table[s], tok)
        t.ref.scales[p, 0, b, w] = x
    t.table[3, 0] = -1  # a window leaves the page behind
    t.cache.scales.copy_(t.ref.scales)
    t.batch = t.make_batch(t.start, t.past)
    q = t.heads_of(hq, dtype)
    for window in (0, 60):
        out, lse = _run(t, q, window)
        _check(t, q, out, lse, window)
        if window:  # what is NaN or not there lies behind three of the sequences' first rows
            assert out[[new, 2 * new, 3 * new]].isfinite().all()


def test_lengths_that_are_not_right(built_lib, gpu):
    """Longer than the table, than max_len, more tokens than max_new, starts out of range."""
    t = Setup(gpu, 1, 64, 16, [30], [4], max_len=32)
    q = t.heads_of(2, F16)
    out, lse = _run(t, q)
    assert out[2:].isnan().all() and lse[2:].isnan().all()
    k, v = t.ref.read(t.table[0], 0, 32)
    o, e, ob, eb = R.attention(q[:2], k, v, 30, 0.125, 0)
    R.check(lse[:2], e, eb, "lse")
    R.check(out[:2], o, ob + o.abs() * 2.0 ** -11 + 2.0 ** -25, "out")
    # nothing of these rows is a sequence's, or within its table
    for start, past, want in (([5, 9], [0], 3.0), ([3, 1], [0], 3.0), ([-4, 0], [0], 3.0), ([0, 4], [2 ** 31 - 1], math.nan)):
        b = t.make_batch(start, past)
        out, lse = _run(t, q, batch=b)
        assert bool((out == want).all()) if want == want else bool(out.isnan().all())
    t = Setup(gpu, 1, 64, 16, [30], [40], max_new=33)
    q = t.heads_of(2, F16)
    out, lse = _run(t, q)
    assert bool((out[33:] == 3.0).all()) and bool((lse[33:] == 3.0).all())
    k, v = t.ref.read(t.table[0], 0, 70)
    o, e, ob, eb = R.attention(q[:33], k, v, 30, 0.125, 0)
    R.check(out[:33], o, ob + o.abs() * 2.0 ** -11 + 2.0 ** -25, "out")


def test_strided_operands(built_lib, gpu):
    t = Setup(gpu, 2, 64, 32, [100, 3], [20, 1])
    for gap in (8, 1):
        whole = torch.randn(t.rows, 4 * 64 + gap, generator=t.gen).half()
        o = torch.full((4, t.rows, 64 + gap), 3.0, dtype=F16, device=gpu)
        out = o[:, :, :64].transpose(0, 1)
        D.kv_attention(t.cache, t.batch, whole.to(gpu)[:, :256].view(t.rows, 4, 64), out)
        plain, lse = _run(t, whole[:, :256].reshape(t.rows, 4, 64))
        assert torch.equal(out, plain) and bool((o[:, :, 64:] == 3.0).all())
        _check(t, whole[:, :256].reshape(t.rows, 4, 64), plain, lse)


def test_shared_pages(built_lib, gpu):
    """Sequences that share the pages of a prefix see what one that has them alone sees."""
    t = Setup(gpu, 2, 128, 32, [70, 70], [1, 1])
    t.table[1, :2] = t.table[0, :2]
    t.batch = t.make_batch(t.start, t.past)
    q = t.heads_of(4, BF16)
    out, lse = _run(t, q)
    _check(t, q, out, lse)


@pytest.mark.parametrize("new", [1, 300])
def test_graph_stream_and_guards(built_lib, gpu, new):
    t = Setup(gpu, 1, 64, 64, [1500], [new], max_len=3000)
    t.table = torch.arange(t.table.shape[1], dtype=torch.int32)[None]
    t.batch = t.make_batch(t.start, t.past)
    q = t.heads_of(4, F16)
    want = _run(t, q)
    qd = q.to(gpu)
    out, lse = torch.zeros_like(want[0]), torch.zeros_like(want[1])
    ws = torch.empty(max(256, L.mebp_kv_attention_workspace_bytes(1, new, 3000, 4, 1, 64)), dtype=torch.uint8, device=gpu)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        D.kv_attention(t.cache, t.batch, qd, out, lse, ws=ws)
    side.synchronize()
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        D.kv_attention(t.cache, t.batch, qd, out, lse, ws=ws)
    for past in (1500, 0, 63, 1000):
        t.batch.past.fill_(past)
        t.past = [past]
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        eager = _run(t, q)
        assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1])
        _check(t, q, out, lse)
    was = L.mebp_set_workspace_guards(True)
    try:
        guarded = _run(t, q)
    finally:
        L.mebp_set_workspace_guards(was)
    assert torch.equal(guarded[0], out) and torch.equal(guarded[1], lse)


def test_nothing_to_do(built_lib, gpu):
    t = Setup(gpu, 1, 64, 16, [0, 5], [0, 0], tail=2)
    q = t.heads_of(2, F16)
    out, lse = _run(t, q)
    assert bool((out == 3.0).all())
    empty = torch.zeros(0, 2, 64, dtype=F16, device=gpu)
    assert D.kv_attention(t.cache, t.batch, empty).shape == (0, 2, 64)


@pytest.mark.parametrize("seqs,longest,most", [(300, 400, 1), (260, 200, 3), (2, 20000, 1), (33, 2000, 2)])
@pytest.mark.parametrize("hkv,hq,dim,page,dtype", [(1, 7, 64, 32, F16), (2, 14, 64, 64, BF16), (1, 5, 128, 16, F16), (1, 8, 256, 64, BF16)])
def test_ragged_batches_in_equal_shares(built_lib, gpu, seqs, longest, most, hkv, hq, dim, page, dtype):
    """Many sequences of all lengths, some without a new token: each workgroup's share begins and ends inside them."""
    say("shares", seqs, longest, most, hkv, hq, dim)
    gen = torch.Generator().manual_seed(seqs + dim)
    new = torch.randint(0, most + 1, (seqs,), generator=gen).tolist() if seqs > 2 else [1, 1]
    past = torch.randint(0, longest, (seqs,), generator=gen).tolist()
    new[0], past[0], past[-1] = most, longest, 0
    t = Setup(gpu, hkv, dim, page, past, new, seed=dim, tail=2)
    q = t.heads_of(hq, dtype)
    for window in (0, 300):
        for room in (t.max_len, 1 << 16):  # (with room for long sequences several are dealt out in shares)
            t.max_len = room
            t.batch = t.make_batch(t.start, t.past)
            out, lse = _run(t, q, window)
            again, e2 = _run(t, q, window)
            assert torch.equal(out, again) and torch.equal(lse, e2)
            _check(t, q, out, lse, window)


@pytest.mark.parametrize("hq,new", [(1, 70), (1, 200), (3, 50), (3, 130), (5, 97), (12, 40), (100, 3), (200, 1)])
def test_window_of_many_rows_in_parts(built_lib, gpu, hq, new):
    """The tiles that a row tile sees, by windows of all sizes: no part of them is left out, whatever the heads in a group."""
    t = Setup(gpu, 1, 64, 64, [2000], [new], seed=hq, max_len=2300)
    q = t.heads_of(hq, F16)
    for window in (1, 2, 63, 64, 65, 127, 128, 129, 191, 257, 700):
        out, lse = _run(t, q, window)
        _check(t, q, out, lse, window)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("past,new", [(0, 33), (0, 100), (5000, 40), (5000, 1), (200, 64)])
def test_outputs_at_odd_addresses(built_lib, gpu, dim, past, new):
    """Rows whose elements no vector reaches, out of one workgroup and joined, are what they are elsewhere."""
    t = Setup(gpu, 1, dim, 64, [past], [new], seed=dim)
    q = t.heads_of(4, BF16)
    want = _run(t, q)
    whole = torch.full((new, 4 * dim + 3), 3.0, dtype=BF16, device=gpu)
    out = whole[:, 1:1 + 4 * dim].view(new, 4, dim)
    lse = torch.zeros(new, 4, device=gpu)
    D.kv_attention(t.cache, t.batch, q.to(gpu), out, lse)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    assert bool((whole[:, 0] == 3.0).all()) and bool((whole[:, 1 + 4 * dim:] == 3.0).all())


def test_two_graphs_and_one_workspace(built_lib, gpu):
    """Graphs of different calls that were given the same scratch, replayed in turn on one stream."""
    cases = []
    ws = torch.empty(64 << 20, dtype=torch.uint8, device=gpu)
    for new, past, window in ((1, 9000, 0), (200, 700, 256), (1, 3000, 100)):
        t = Setup(gpu, 1, 128, 64, [past, 100], [new, 1], seed=new)
        q = t.heads_of(4, F16)
        want = _run(t, q, window)
        qd, out, lse = q.to(gpu), torch.zeros_like(want[0]), torch.zeros_like(want[1])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            D.kv_attention(t.cache, t.batch, qd, out, lse, None, window, ws)
        cases.append((t, graph, want, out, lse, qd))
    for _ in range(3):
        for t, graph, want, out, lse, _ in cases:
            out.zero_()
            graph.replay()
        torch.cuda.synchronize()
        for t, graph, want, out, lse, _ in cases:
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


@pytest.mark.parametrize("seqs", [3, 40])
def test_lengths_beyond_max_len_in_a_batch(built_lib, gpu, seqs):
    """Whatever a sequence's past says, the others are what they are, and its rows from max_len on are NaN."""
    past = [2 ** 31 - 1 if s % 3 == 1 else 4000 + 10 * s for s in range(seqs)]
    t = Setup(gpu, 1, 64, 64, [min(p, 5000) for p in past], [2] * seqs, max_len=4399)
    t.batch = t.make_batch(t.start, past)
    q = t.heads_of(4, F16)
    for window in (0, 100):
        out, lse = _run(t, q, window)
        for s, p in enumerate(past):
            for i in range(2):
                r = 2 * s + i
                if p + i >= 4399:
                    assert out[r].isnan().all() and lse[r].isnan().all()
                    continue
                k, v = t.ref.read(t.table[s], 0, p + i + 1)
                o, e, ob, eb = R.attention(q[r:r + 1], k, v, p + i, 0.125, window)
                R.check(lse[r:r + 1], e, eb, "lse")
                R.check(out[r:r + 1], o, ob + o.abs() * 2.0 ** -11 + 2.0 ** -25, "out")


@pytest.mark.parametrize("room", [0, 1 << 20])
@pytest.mark.parametrize("dim,new", [(64, 1), (64, 90), (128, 1), (128, 90), (256, 1), (256, 90)])
def test_scales_at_both_ends(built_lib, gpu, room, dim, new):
    """Values 10^50 and 10^70 apart, the large ones first or last, or one block in the middle: no sum overflows."""
    for case in range(5):
        t = Setup(gpu, 1, dim, 32, [900], [new], seed=case, max_len=room or None)
        b = torch.arange(t.ref.scales.numel() // 2).view(t.ref.scales.shape[:3])
        order = torch.empty_like(b)
        for i, p in enumerate(t.table[0]):
            order[int(p)] = 2 * i + torch.arange(2)
        size = [torch.where(order < 20, 1e25, 1e-25), torch.where(order < 20, 1e-25, 1e25), 10.0 ** (30 - 2 * order.clamp(0, 33).double()),
                torch.where(order == 30, 1e33, 1e-37), torch.where(order == 1, 1e33, 1e-37)][case]
        t.ref.scales[..., 1] = size.float() * t.ref.scales[..., 1]
        t.cache.scales.copy_(t.ref.scales)
        q = t.heads_of(4, BF16)
        out, lse = _run(t, q)
        assert out.isfinite().all()
        _check(t, q, out, lse)


@pytest.mark.parametrize("room", [0, 1 << 20])
@pytest.mark.parametrize("hkv,hq,dim,new", [(1, 2, 64, 1), (2, 14, 64, 3), (1, 4, 128, 1), (1, 4, 256, 1), (1, 4, 64, 90), (1, 4, 128, 90), (1, 2, 256, 90)])
def test_infinite_and_smallest_scales(built_lib, gpu, room, hkv, hq, dim, new):
    """An infinite scale is as one of NaN, for the rows that see it; the smallest ones are numbers like others."""
    say("infinite scales", room, hkv, hq, dim, new)
    for case in range(4):
        t = Setup(gpu, hkv, dim, 32, [250, 300, 140], [new] * 3, seed=case, max_len=room or None)
        q = t.heads_of(hq, BF16)
        if case < 3:
            for s, tok, w in ((0, 100, 1), (1, 303 if new > 1 else 280, 0), (2, 10, 1)):
                p, b = t.ref.where(t.table[s], tok)
                t.ref.scales[p, 0, b, w] = math.nan
            gives = (math.inf, -math.inf, math.nan)[case]
            t.cache.scales.copy_(torch.where(t.ref.scales.isnan(), torch.full_like(t.ref.scales, gives), t.ref.scales))
        else:
            t.ref.scales[..., 1] = 2.0 ** -149 * torch.randint(1, 40, t.ref.scales.shape[:-1], generator=t.gen)
            t.ref.scales[:, :, ::2, 1] *= 2.0 ** 3
            t.cache.scales.copy_(t.ref.scales)
        for window in (0, 60):
            out, lse = _run(t, q, window)
            _check(t, q, out, lse, window)
