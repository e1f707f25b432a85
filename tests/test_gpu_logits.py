"""The operators on logits on the GPU against 64 bits: log probabilities with entropy and top
alternatives, their gradient, and distillation from a teacher's top logits."""
import math

import pytest
import torch

import logits_ref as R
from gpu_util import say
from paper_2510_03425_amd import _lib as L
from paper_2510_03425_amd import device as D

pytestmark = pytest.mark.gpu
INF, NAN = math.inf, math.nan
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
EPS = 2.0 ** -24


def _logits(rows, vocab, dtype, seed, std=3.0, pad=0, gpu="cuda"):
    """The logits on the CPU, and the same on the GPU in rows `pad` elements further apart, with
    7 behind each row's end."""
    g = torch.Generator().manual_seed(seed)
    z = (torch.randn((rows, vocab), generator=g) * std).to(dtype)
    return z, _upload(z, pad, gpu)


def _upload(z, pad=0, gpu="cuda"):
    buf = torch.full((z.shape[0], z.shape[1] + pad), 7.0, dtype=z.dtype, device=gpu)
    buf[:, :z.shape[1]] = z.to(gpu)
    return buf[:, :z.shape[1]]


def _padding_untouched(view):
    base = view._base if view._base is not None else view
    assert torch.equal(base[:, view.shape[1]:], torch.full_like(base[:, view.shape[1]:], 7.0))


def _check_scores(z, got, targets, top_k, tau):
    ref = R.scores(z, targets, top_k, tau)
    E, Dr = R.softmax_bound(z, tau)
    mx = z.double().abs()
    mx = float(mx[torch.isfinite(mx)].max()) / tau if torch.isfinite(mx).any() else 0.0
    R.close(got["lse"], ref["lse"], E + 4 * EPS * (mx + 20), "lse")
    # H = ln s - (sum e (z - m)) / s / tau: the weighted sum's terms are off by E of D each
    R.close(got["entropy"], ref["entropy"], E * (1 + 2 * Dr) + 4 * EPS * (Dr + 20), "entropy")
    if targets is not None:
        R.close(got["logp"], ref["logp"], E + 4 * EPS * (Dr + 20) + 4 * EPS * ref["logp"].abs().nan_to_num(0, 0, 0), "logp")
    if top_k:
        assert torch.equal(got["top_ids"].cpu(), ref["top_ids"]), "top_ids"
        R.close(got["top_logp"], ref["top_logp"],
                E + 4 * EPS * (Dr + 20) + 4 * EPS * ref["top_logp"].abs().nan_to_num(0, 0, 0), "top_logp")


SHAPES = [  # rows, vocab, top_k: one column to more than one part of a row
    (1, 1, 1), (1, 2, 5), (3, 7, 64), (2, 63, 3), (5, 255, 64), (4, 1000, 20), (3, 2049, 1), (2, 4096, 8), (2, 4099, 33),
    (1, 50257, 20), (7, 12289, 64), (1025, 1030, 4), (2, 151936, 64), (3, 65536, 7), (1, 70001, 64), (159, 65537, 2), (160, 65537, 2), (256, 17000, 33),
]


@pytest.mark.parametrize("rows,vocab,top_k", SHAPES)
@pytest.mark.parametrize("dtype,pad,tau", [(F32, 0, 1.0), (F16, 3, 0.7), (BF16, 1, 2.5)])
def test_scores(built_lib, gpu, rows, vocab, top_k, dtype, pad, tau):
    say("scores", rows, vocab, top_k, dtype)
    z, zd = _logits(rows, vocab, dtype, 1 + rows + vocab, pad=pad)
    t = torch.randint(0, vocab, (rows,), generator=torch.Generator().manual_seed(5), dtype=torch.int32)
    got = D.token_logprobs(zd, t.to(gpu), top_k, tau)
    torch.cuda.synchronize()
    _check_scores(z, got, t, top_k, tau)
    _padding_untouched(zd)


def _special_rows(vocab, dtype):
    """Rows where a softmax or an order of logits goes wrong most easily."""
    lowest = torch.finfo(dtype).min
    g = torch.Generator().manual_seed(3)
    base = (torch.randn(vocab, generator=g) * 3).to(dtype)
    rows = {"ordinary": base.clone(), "equal": torch.full((vocab,), 1.5), "zero": torch.zeros(vocab),
            "signed zeros": torch.where(torch.arange(vocab) % 3 == 0, 0.0, -0.0), "masked": torch.full((vocab,), -INF),
            "lowest": torch.full((vocab,), lowest), "rising": torch.arange(vocab).float() / vocab * 20,
            "falling": -torch.arange(vocab).float() / vocab * 20, "steps": (torch.arange(vocab) // 100 % 5).float()}
    one = torch.full((vocab,), -INF)
    one[vocab // 2] = -3.0
    rows["one left"] = one
    few = torch.full((vocab,), -INF)
    few[vocab // 3:vocab // 3 + 3] = torch.tensor([1.0, 2.0, 1.0])
    rows["few left"] = few
    low = base.clone().float()
    low[: vocab // 2] = lowest
    rows["half lowest"] = low
    peak = base.clone().float()
    peak[vocab - 1] = 60.0
    rows["sure of the last"] = peak
    for name, v in (("nan", NAN), ("inf", INF)):
        r = base.clone().float()
        r[vocab // 5] = v
        rows[name] = r
    return list(rows), torch.stack([r.to(dtype) for r in rows.values()])


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("vocab,top_k", [(1003, 20), (20001, 64), (70001, 64), (150001, 9)])
def test_scores_of_special_rows(built_lib, gpu, dtype, vocab, top_k):
    names, z = _special_rows(vocab, dtype)
    t = torch.arange(len(names), dtype=torch.int32) * 37 % vocab
    t[names.index("sure of the last")] = vocab - 1
    zd = _upload(z)
    got = D.token_logprobs(zd, t.to(gpu), top_k)
    torch.cuda.synchronize()
    for i, n in enumerate(names):
        say("special row", n, dtype, vocab)
        _check_scores(z[i:i + 1], {k: v[i:i + 1] for k, v in got.items()}, t[i:i + 1], top_k, 1.0)


def test_targets_out_of_range_and_absent_outputs(built_lib, gpu):
    z, zd = _logits(6, 5000, F32, 9)
    t = torch.tensor([-1, 4999, 5000, -7, 0, 2 ** 31 - 1], dtype=torch.int32)
    got = D.token_logprobs(zd, t.to(gpu), 0)
    _check_scores(z, got, t, 0, 1.0)
    # any subset of the outputs gives the same bits
    whole = D.token_logprobs(zd, t.to(gpu), 9)
    for names in (["logp"], ["entropy"], ["lse", "top_ids"], ["top_logp"]):
        out = {k: torch.empty_like(whole[k]) for k in names}
        D.token_logprobs(zd, t.to(gpu), 9, out=out)
        for k in names:
            assert torch.equal(out[k].nan_to_num(7.0), whole[k].nan_to_num(7.0)), k


# ------------------------------------------------------------------ gradient of the scores
GRADS = [(F32, F32), (F32, BF16), (F16, F16), (F16, F32), (BF16, BF16), (BF16, F16)]


@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 7), (2, 1000), (5, 4099), (1, 50257), (1030, 515)])
@pytest.mark.parametrize("dtype,gtype", GRADS)
def test_scores_grad(built_lib, gpu, rows, vocab, dtype, gtype):
    say("scores grad", rows, vocab, dtype, gtype)
    tau = 0.8
    z, zd = _logits(rows, vocab, dtype, rows + vocab, pad=2)
    g = torch.Generator().manual_seed(1)
    t = torch.randint(-1, vocab, (rows,), generator=g, dtype=torch.int32)
    dl, de = torch.randn(rows, generator=g), torch.randn(rows, generator=g)
    s = D.token_logprobs(zd, t.to(gpu), 0, tau)
    E, Dr = R.softmax_bound(z, tau)
    for a, b in ((dl, de), (dl, None), (None, de)):
        dz = _upload(torch.zeros(rows, vocab, dtype=gtype), pad=5)
        D.token_logprobs_backward(zd, t.to(gpu), s["lse"], s["entropy"], None if a is None else a.to(gpu),
                                  None if b is None else b.to(gpu), dz, tau)
        torch.cuda.synchronize()
        ref, mag = R.scores_grad(z, t, tau, a, b)
        # q from the fp32 lse (E, and 2^-24 of both terms of the exponent), the entropy's own error
        rel = 3 * E + 6 * EPS * (Dr + 40)
        extra = 0.0 if b is None else b.abs()[:, None] / tau * (E * (1 + 2 * Dr) + 8 * EPS * (Dr + 20))
        R.close(dz, ref, rel * mag + extra + R.HALF_STEP[gtype] * 1.001 * ref.abs() + R.TINY[gtype], "dz")
        _padding_untouched(dz)


def test_scores_grad_of_special_rows(built_lib, gpu):
    for dtype in (F32, BF16):
        names, z = _special_rows(5003, dtype)
        keep = [i for i, n in enumerate(names) if n not in ("nan", "inf")]
        z = z[keep]
        n = len(keep)
        t = torch.arange(n, dtype=torch.int32) * 37
        t[0] = 5003  # beyond the vocabulary: its row is NaN
        zd = _upload(z)
        dl, de = torch.linspace(-1, 1, n), torch.linspace(1, 2, n)
        s = D.token_logprobs(zd, t.to(gpu))
        dz = D.token_logprobs_backward(zd, t.to(gpu), s["lse"], s["entropy"], dl.to(gpu), de.to(gpu),
                                       torch.empty_like(zd, dtype=F32))
        ref, mag = R.scores_grad(z, t, 1.0, dl, de)
        for i in range(n):
            E, Dr = R.softmax_bound(z[i:i + 1], 1.0)
            lse = float(s["lse"][i]) if math.isfinite(float(s["lse"][i])) else 0.0
            # an lse of the size of the type's lowest value is itself rounded by 2^-24 of it
            wide = 2 * EPS * abs(lse)
            if wide > 1:
                assert not torch.isnan(dz[i]).any()
                continue
            extra = float(de[i]) * (E * (1 + 2 * Dr) + 8 * EPS * (Dr + 20))
            say("special row", names[keep[i]])
            R.close(dz[i:i + 1], ref[i:i + 1], (3 * E + 6 * EPS * (Dr + 40) + wide) * mag[i:i + 1] + extra
                    + EPS * ref[i:i + 1].abs() + 1e-37, names[keep[i]])


# ------------------------------------------------------------------ distillation
def _teacher(rows, k, vocab, seed):
    g = torch.Generator().manual_seed(seed)
    ids = torch.stack([torch.randperm(vocab, generator=g)[:k] if vocab >= k else torch.randint(0, vocab, (k,), generator=g)
                       for _ in range(rows)]).to(torch.int32)
    return ids, torch.randn((rows, k), generator=g) * 2 + 5, torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32)


def _check_distill(z, ids, tl, t, w, tau, alpha, loss, dz, what=""):
    ref, lmag, g, gmag = R.distill(z, ids, tl, t, w, tau, alpha)
    E, Dr = R.softmax_bound(z, tau)
    E1, D1 = R.softmax_bound(z, 1.0)
    E, Dr = max(E, E1), max(Dr, D1)
    wt = torch.ones(len(ref)) if w is None else w.abs()
    # the teacher's probabilities and logarithms (range up to 40), the student's logs: absolute E each
    tol = 4 * E * lmag + wt * (alpha * tau * tau + 1) * (2 * E + 8 * EPS * (Dr + 60))
    R.close(loss, ref, tol, what + " loss")
    if dz is not None:
        rel = 4 * E + 8 * EPS * 60
        R.close(dz, g, rel * gmag + R.HALF_STEP[dz.dtype] * 1.001 * g.abs() + R.TINY[dz.dtype], what + " dz")


MODES = [(1.0, 1.0), (2.0, 0.7), (1.0, 0.4), (0.5, 1.0), (3.0, 0.0)]  # tau, alpha


@pytest.mark.parametrize("rows,vocab,k", [(1, 1, 1), (2, 5, 8), (3, 1000, 64), (4, 4099, 16), (1, 50257, 32), (1030, 700, 3), (2, 70001, 64)])
@pytest.mark.parametrize("dtype,gtype", [(F32, F32), (F32, BF16), (F16, F16), (BF16, BF16), (BF16, F32)])
def test_distill(built_lib, gpu, rows, vocab, k, dtype, gtype):
    z, zd = _logits(rows, vocab, dtype, rows + vocab, pad=3)
    ids, tl, t = _teacher(rows, k, vocab, rows)
    w = torch.rand(rows, generator=torch.Generator().manual_seed(2)) + 0.5
    for tau, alpha in MODES:
        say("distill", rows, vocab, k, dtype, gtype, tau, alpha)
        dz = _upload(torch.zeros(rows, vocab, dtype=gtype), pad=1)
        loss = D.distill_topk(zd, ids.to(gpu), tl.to(gpu), None, dz, tau, alpha, t.to(gpu), w.to(gpu))
        only = D.distill_topk(zd, ids.to(gpu), tl.to(gpu), None, None, tau, alpha, t.to(gpu), w.to(gpu))
        torch.cuda.synchronize()
        _check_distill(z, ids, tl, t, w, tau, alpha, loss, dz)
        _check_distill(z, ids, tl, t, w, tau, alpha, only, None)
        _padding_untouched(dz)
        _padding_untouched(zd)


@pytest.mark.parametrize("vocab", [900, 20001, 70001])
@pytest.mark.parametrize("tau,alpha", [(1.0, 1.0), (2.0, 0.6), (1.0, 0.5)])
def test_distill_of_special_entries(built_lib, gpu, vocab, tau, alpha):
    """Absent, repeated and out-of-range entries and targets, a target among the entries, rows of
    weight 0 with NaN logits, masked student rows."""
    n, k = 15, 6
    z, _ = _logits(n, vocab, F32, 4)
    ids, tl, t = _teacher(n, k, vocab, 8)
    w = torch.rand(n, generator=torch.Generator().manual_seed(2)) + 0.5
    ids[0, 2:] = -1
    ids[1] = -1                      # no entry at all
    ids[2, 3] = ids[2, 0]            # twice the same, next to each other and not
    ids[2, 4] = ids[2, 5]
    ids[3, 1] = vocab                # beyond the vocabulary
    t[4] = ids[4, 3]                 # the label among the entries
    t[5], t[6] = -1, vocab
    tl[7, :3] = -INF
    tl[8] = -INF
    z[9] = NAN
    w[9] = 0.0
    z[10] = -INF                     # nothing left of the student's row
    z[11, ids[11, 2].long()] = -INF  # the student has masked a token of the teacher's
    ids[12] = ids[12, 0].clone()     # one token, k times
    t[12] = ids[12, 0]
    tl[13] = torch.tensor([300.0, 0.0, -300.0, 1.0, 299.0, -1e30])
    z[14], ids[14], t[14] = NAN, -1, -1  # nothing to learn from
    zd = _upload(z)
    dz = torch.empty_like(zd)
    loss = D.distill_topk(zd, ids.to(gpu), tl.to(gpu), None, dz, tau, alpha, t.to(gpu), w.to(gpu))
    torch.cuda.synchronize()
    for i in range(n):
        s = slice(i, i + 1)
        _check_distill(z[s], ids[s], tl[s], t[s], w[s], tau, alpha, loss[s], dz[s], f"row {i}")


@pytest.mark.parametrize("rows,vocab,dtype,gtype", [
    # rows of which a workgroup holds all in registers, some in LDS too, and some not at all
    (97, 50257, F32, BF16), (96, 120001, F32, F32), (96, 131071, BF16, BF16), (98, 245763, F16, F16),
])
@pytest.mark.parametrize("tau,alpha", [(1.0, 1.0), (2.0, 0.7), (1.5, 0.7)])
def test_distill_of_long_rows(built_lib, gpu, rows, vocab, dtype, gtype, tau, alpha):
    say("distill rows", rows, vocab, dtype, gtype, tau, alpha)
    z, zd = _logits(rows, vocab, dtype, rows + vocab, pad=1)
    ids, tl, t = _teacher(rows, 8, vocab, rows)
    w = torch.rand(rows, generator=torch.Generator().manual_seed(2)) + 0.5
    w[3] = 0.0
    dz = _upload(torch.zeros(rows, vocab, dtype=gtype), pad=3)
    loss = D.distill_topk(zd, ids.to(gpu), tl.to(gpu), None, dz, tau, alpha, t.to(gpu), w.to(gpu))
    torch.cuda.synchronize()
    some = torch.tensor([0, 1, 3, 17, rows - 1])
    _check_distill(z[some], ids[some], tl[some], t[some], w[some], tau, alpha, loss[some.to(gpu)], dz[some.to(gpu)])
    _padding_untouched(dz)
    # every row against 64 bits on the GPU, as a whole
    u, q = zd.double(), torch.empty((rows, vocab), dtype=torch.float64, device=gpu)
    p = torch.softmax(tl.to(gpu).double() / tau, 1)
    q.copy_(alpha * tau * torch.softmax(u / tau, 1))
    q.scatter_add_(1, ids.to(gpu).long(), -alpha * tau * p)
    if alpha < 1:
        q += (1 - alpha) * torch.softmax(u, 1)
        q.scatter_add_(1, t.to(gpu).long()[:, None], torch.full((rows, 1), alpha - 1, dtype=torch.float64, device=gpu))
    q *= w.to(gpu).double()[:, None]
    err = (dz.double() - q).norm(dim=1) / q.norm(dim=1).clamp_min(1e-300)
    assert bool((err <= 1e-5 + R.HALF_STEP[gtype] * 1.01).all()), err.max()


@pytest.mark.parametrize("vocab,copies", [(1003, 1), (40003, 1), (70001, 1), (40003, 7)])  # (70001: by parts)
@pytest.mark.parametrize("tau,alpha", [(1.0, 1.0), (2.0, 0.6), (1.5, 0.5)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_distill_of_special_students(built_lib, gpu, vocab, copies, tau, alpha, dtype):
    names, z = _special_rows(vocab, dtype)
    late = z[0].clone()
    late[: vocab // 2] = -INF  # the first columns are masked off
    names, z = names + ["first half masked"], torch.cat([z, late[None]])
    n = len(names)
    ids, tl, t = _teacher(n, 5, vocab, 3)
    at = names.index("one left")
    ids[at] = vocab // 2  # (other tokens are masked: an infinite loss)
    t[at] = vocab // 2
    rep = lambda x: x.repeat(copies, *[1] * (x.dim() - 1)).to(gpu)
    zd = _upload(z.repeat(copies, 1))
    dz = torch.empty_like(zd, dtype=F32)
    loss = D.distill_topk(zd, rep(ids), rep(tl), None, dz, tau, alpha, rep(t), None)
    only = D.distill_topk(zd, rep(ids), rep(tl), None, None, tau, alpha, rep(t), None)
    torch.cuda.synchronize()
    for i, name in enumerate(names):
        say("special student", name, dtype, vocab, tau, alpha)
        s, d = slice(i, i + 1), slice((copies - 1) * n + i, (copies - 1) * n + i + 1)
        if name in ("lowest", "half lowest"):
            # the loss of a token at the type's lowest value is of its size, or beyond the type
            assert not torch.isnan(dz[d]).any()
            _check_distill(z[s], ids[s], tl[s], t[s], None, tau, alpha, R.distill(z[s], ids[s], tl[s], t[s], None, tau, alpha)[0],
                           dz[d], name)
            continue
        _check_distill(z[s], ids[s], tl[s], t[s], None, tau, alpha, loss[d], dz[d], name)
        _check_distill(z[s], ids[s], tl[s], t[s], None, tau, alpha, only[d], None, name)


# ------------------------------------------------------------------ how they are called
def _all_calls(z, t, ids, tl, w, ws, dz, dz2):
    s = D.token_logprobs(z, t, 17, 1.3, ws=ws)
    D.token_logprobs_backward(z, t, s["lse"], s["entropy"], w, w, dz2, 1.3)
    loss = D.distill_topk(z, ids, tl, None, dz, 2.0, 0.6, t, w, ws)
    return [s[k] for k in sorted(s)] + [dz2, loss, dz]


@pytest.mark.parametrize("rows,vocab", [(3, 30011), (3, 70011), (1040, 3001)])
def test_streams_graphs_and_repeats_give_the_same_bits(built_lib, gpu, rows, vocab):
    def inputs(seed):
        z, zd = _logits(rows, vocab, BF16, seed)
        ids, tl, t = _teacher(rows, 16, vocab, seed)
        return [zd, t.to(gpu), ids.to(gpu), tl.to(gpu), torch.linspace(0.5, 1.5, rows, device=gpu)]

    nb = L.mebp_logits_workspace_bytes(rows, vocab, 17)
    a, b = inputs(1), inputs(2)
    ws = [torch.randint(0, 255, (nb,), dtype=torch.uint8, device=gpu) for _ in range(2)]
    dz = [[torch.empty_like(a[0]) for _ in range(2)] for _ in range(2)]
    first = [x.clone() for x in _all_calls(*a, ws[0], *dz[0])]
    other = [x.clone() for x in _all_calls(*b, ws[1], *dz[1])]
    torch.cuda.synchronize()
    # two streams at once, each with its own workspace
    st = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for i, x in enumerate((a, b)):
        st[i].wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st[i]):
            got.append(_all_calls(*x, ws[i], *dz[i]))
    torch.cuda.synchronize()
    for want, have in zip((first, other), got):
        assert all(torch.equal(x, y) for x, y in zip(want, have))
    # two captured graphs that share a workspace, replayed in turn with eager calls between
    graphs, outs = [], []
    for i, x in enumerate((a, b)):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            outs.append(_all_calls(*x, ws[0], *dz[i]))
        graphs.append(gr)
    for rep in range(3):
        for i, want in enumerate((first, other)):
            for o in outs[i]:
                o.fill_(-5)
            graphs[i].replay()
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(want, outs[i])), (rep, i)
            _all_calls(*b, ws[1], *dz[1])


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("rows,vocab", [(2, 20001), (2, 70001), (1040, 1001)])
def test_gradients_in_place(built_lib, gpu, dtype, rows, vocab):
    z, zd = _logits(rows, vocab, dtype, 6, pad=3)
    ids, tl, t = (x.to(gpu) for x in _teacher(rows, 9, vocab, 6))
    w = torch.linspace(0.5, 1.5, rows, device=gpu)
    w[1] = 0.0
    s = D.token_logprobs(zd, t)
    want = D.token_logprobs_backward(zd, t, s["lse"], s["entropy"], w, w)
    here = _upload(z, 3)
    D.token_logprobs_backward(here, t, s["lse"], s["entropy"], w, w, here)
    assert torch.equal(want, here)
    _padding_untouched(here)
    for tau, alpha in MODES:
        want = torch.empty_like(zd)
        lw = D.distill_topk(zd, ids, tl, None, want, tau, alpha, t, w)
        here = _upload(z, 3)
        lh = D.distill_topk(here, ids, tl, None, here, tau, alpha, t, w)
        assert torch.equal(want, here) and torch.equal(lw, lh)
        _padding_untouched(here)


def test_gradients_against_differences(built_lib, gpu):
    """The losses' own differences along random directions, in fp32: a step of h = 2^-5 leaves the
    third derivative's h^2 / 6 (at most about 1/6 of a row's weight and direction cubed) and the
    fp32 loss's rounding over h."""
    rows, vocab, h = 8, 300, 2.0 ** -5
    z, zd = _logits(rows, vocab, F32, 12)
    ids, tl, t = (x.to(gpu) for x in _teacher(rows, 12, vocab, 12))
    v = torch.randn((rows, vocab), generator=torch.Generator().manual_seed(1)).to(gpu)
    v = v / v.abs().amax(1, keepdim=True)
    for tau, alpha in MODES:
        f = lambda x: D.distill_topk(x, ids, tl, None, None, tau, alpha, t).double()
        dz = torch.empty_like(zd)
        D.distill_topk(zd, ids, tl, None, dz, tau, alpha, t)
        diff = (f(zd + h * v) - f(zd - h * v)) / (2 * h)
        bound = h * h / 6 * (alpha / tau + 1 - alpha) + 2 ** -22 * (20 * (tau * tau + 1)) / h
        R.close((dz.double() * v).sum(1), diff, bound, f"distill {tau} {alpha}")
    s = D.token_logprobs(zd, t)
    one = torch.ones(rows, device=gpu)
    for name, dl, de in (("logp", one, None), ("entropy", None, one)):
        f = lambda x: D.token_logprobs(x, t)[name].double()
        dz = D.token_logprobs_backward(zd, t, s["lse"], s["entropy"], dl, de)
        diff = (f(zd + h * v) - f(zd - h * v)) / (2 * h)
        R.close((dz.double() * v).sum(1), diff, h * h / 6 * (1 if de is None else 20) + 2 ** -22 * 40 / h, name)


def test_rows_beyond_32_bit_offsets(built_lib, gpu):
    """Three rows 2^31 + 64 elements apart."""
    vocab, ld = 3001, 2 ** 31 + 64
    buf = torch.empty(2 * ld + vocab, dtype=BF16, device=gpu)
    z, _ = _logits(3, vocab, BF16, 2)
    far = buf.as_strided((3, vocab), (ld, 1))
    far.copy_(z)
    near = _upload(z)
    ids, tl, t = (x.to(gpu) for x in _teacher(3, 8, vocab, 1))
    w = torch.ones(3, device=gpu)
    a, b = D.token_logprobs(near, t, 8), D.token_logprobs(far, t, 8)
    assert all(torch.equal(a[k], b[k]) for k in a)
    want = torch.empty_like(near)
    lw = D.distill_topk(near, ids, tl, None, want, 2.0, 0.5, t, w)
    want2 = D.token_logprobs_backward(near, t, a["lse"], a["entropy"], w, w)
    D.token_logprobs_backward(far, t, a["lse"], a["entropy"], w, w, far)
    assert torch.equal(far, want2)
    far.copy_(z)
    lh = D.distill_topk(far, ids, tl, None, far, 2.0, 0.5, t, w)
    assert torch.equal(far, want) and torch.equal(lw, lh)


def test_no_rows(built_lib, gpu):
    z = torch.empty((0, 100), device=gpu)
    e = lambda *s, dt=F32: torch.empty(s, dtype=dt, device=gpu)
    i32 = torch.int32
    assert D.token_logprobs(z, e(0, dt=i32), 5)["top_ids"].shape == (0, 5)
    assert D.token_logprobs_backward(z, e(0, dt=i32), e(0), e(0), e(0)).shape == (0, 100)
    assert D.distill_topk(z, e(0, 4, dt=i32), e(0, 4), dz=torch.empty_like(z)).shape == (0,)


def test_guarded_workspaces(built_lib, gpu):
    prev = L.mebp_set_workspace_guards(True)
    try:
        for rows, vocab in ((2, 30011), (2, 70011), (1030, 501)):
            z, zd = _logits(rows, vocab, F32, 3)
            ids, tl, t = (x.to(gpu) for x in _teacher(rows, 64, vocab, 1))
            D.token_logprobs(zd, t, 64)
            D.distill_topk(zd, ids, tl, None, torch.empty_like(zd), 2.0, 0.5, t)
            D.distill_topk(zd, ids, tl, None, None, 2.0, 0.5, t)
    finally:
        L.mebp_set_workspace_guards(prev)
