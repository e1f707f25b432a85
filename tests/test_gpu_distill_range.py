"""Distillation from a teacher's top logits on the GPU over the temperatures and values that it
accepts, against 64 bits."""
import math

import pytest
import torch

import logits_ref as R
from gpu_util import say
from mebp_inputs import MINI, make_inputs
from paper_2510_03425_amd import device as D

pytestmark = pytest.mark.gpu
INF = math.inf
F32, BF16 = torch.float32, torch.bfloat16
EPS = 2.0 ** -24


def _close(z, ids, tl, t, tau, alpha, loss, dz, what):
    """Of rows with an entry each; logits less their row's largest, which changes no softmax."""
    x, v = z.double() - z.double().amax(1, keepdim=True), tl.double() - tl.double().amax(1, keepdim=True)
    ref, lmag, g, gmag = R.distill(x, ids, v, t, None, tau, alpha)
    fin = torch.where(torch.isfinite(x), x, x.new_zeros(()))
    both = min(tau, 1.0) if alpha < 1 else tau
    dr = min(float((-fin).amax()) / both, 104.0)
    # weights and their sums as in any softmax; the teacher's probabilities too, of logits that
    # are at most 104 temperatures apart, and their logarithms
    e = (3 * dr + 3 * 104 + 4 + z.shape[1] / 1024 + 8 + 20 + 64) * EPS
    R.close(loss, ref, 4 * e * (lmag + alpha * tau * tau + 1), what + " loss")
    R.close(dz, g, 4 * e * gmag + R.HALF_STEP[dz.dtype] * 1.001 * g.abs() + R.TINY[dz.dtype], what + " dz")


def _teacher(rows, k, vocab, seed):
    g = torch.Generator().manual_seed(seed)
    ids = torch.stack([torch.randperm(vocab, generator=g)[:k] for _ in range(rows)]).to(torch.int32)
    return ids, torch.randn((rows, k), generator=g) * 2 + 5, torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,vocab", [(6, 1003), (6, 70001), (97, 40003)])
@pytest.mark.parametrize("tau,alpha", [(1e-6, 1.0), (1e-3, 1.0), (0.05, 0.5), (20.0, 0.5), (1e4, 1.0), (1e4, 0.5), (0.05, 0.0), (1e-6, 0.0)])
def test_distill_at_any_temperature(built_lib, gpu, dtype, rows, vocab, tau, alpha):
    say("distill temperature", rows, vocab, dtype, tau, alpha)
    tau = float(torch.tensor(tau, dtype=F32))
    z = (torch.randn((rows, vocab), generator=torch.Generator().manual_seed(rows)) * 3).to(dtype)
    z[1] = z[1] + 2000
    z[2, : vocab // 2] = z[2, : vocab // 2] - 60
    ids, tl, t = _teacher(rows, 9, vocab, 5)
    tl[3] += 1000  # (a teacher's raw logits)
    zd, dz = z.to(gpu), torch.empty((rows, vocab), device=gpu)
    loss = D.distill_topk(zd, ids.to(gpu), tl.to(gpu), None, dz, tau, alpha, t.to(gpu))
    only = D.distill_topk(zd, ids.to(gpu), tl.to(gpu), None, None, tau, alpha, t.to(gpu))
    torch.cuda.synchronize()
    some = slice(0, 6)
    for got in (loss, only):
        _close(z[some], ids[some], tl[some], t[some], tau, alpha, got[some], dz[some], f"{tau} {alpha}")


@pytest.mark.parametrize("tau", [0.5, 1.0, 0.05])
def test_teachers_logits_at_the_ends_of_the_type(built_lib, gpu, tau):
    """A teacher's logits are finite entries up to fp32's ends at any temperature: a row of nothing but the
    lowest value is uniform, one far above the rest has all."""
    tau = float(torch.tensor(tau, dtype=F32))
    top = torch.finfo(F32).max
    z = torch.randn((4, 900), generator=torch.Generator().manual_seed(1))
    ids, tl, t = _teacher(4, 5, 900, 2)
    tl[0], tl[1] = -top, top
    tl[2, 0] = top
    tl[3, :4] = -top
    zd, dz = z.to(gpu), torch.empty((4, 900), device=gpu)
    loss = D.distill_topk(zd, ids.to(gpu), tl.to(gpu), None, dz, tau, 1.0)
    torch.cuda.synchronize()
    _close(z, ids, tl, t, tau, 1.0, loss, dz, f"ends {tau}")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("copies,vocab", [(1, 1003), (1, 40003), (1, 70001), (60, 40003)])
@pytest.mark.parametrize("tau,alpha", [(1.0, 1.0), (2.0, 0.6), (1.5, 0.5)])
def test_students_at_the_lowest_value(built_lib, gpu, dtype, copies, vocab, tau, alpha):
    """Rows of nothing but the type's lowest value (all alike: uniform), rows with half of it, entries and
    labels where they have a weight, and -1e9 in the place of -inf."""
    low = torch.finfo(dtype).min
    g = torch.Generator().manual_seed(3)
    z = torch.stack([torch.full((vocab,), low), torch.randn(vocab, generator=g) * 3, torch.full((vocab,), -1e9),
                     torch.randn(vocab, generator=g)])
    z[1, : vocab // 2] = low
    z[3, ::2] = -1e9
    z = z.to(dtype)
    ids, tl, t = _teacher(4, 6, vocab // 2 - 2, 3)
    ids, t = ids + vocab // 2, t + vocab // 2  # the second halves
    ids[3], t[3] = ids[3] // 2 * 2 + 1, t[3] // 2 * 2 + 1
    rep = lambda x: x.repeat(copies, *[1] * (x.dim() - 1)).to(gpu)
    zd = rep(z)
    dz = torch.empty_like(zd, dtype=F32)
    loss = D.distill_topk(zd, rep(ids), rep(tl), None, dz, tau, alpha, rep(t))
    only = D.distill_topk(zd, rep(ids), rep(tl), None, None, tau, alpha, rep(t))
    torch.cuda.synchronize()
    last = slice(4 * copies - 4, 4 * copies)
    for i in range(4):
        s = slice(i, i + 1)
        for got in (loss, only):
            _close(z[s], ids[s], tl[s], t[s], tau, alpha, got[last][s], dz[last][s], f"row {i}")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,vocab", [(3, 1003), (3, 70001), (97, 40003), (97, 151936)])
def test_hard_labels_alone_know_no_temperature(built_lib, gpu, dtype, rows, vocab):
    """At alpha 0 no softmax at tau is part of the loss: every temperature gives the same bits."""
    say("hard labels alone", rows, vocab, dtype)
    z = (torch.randn((rows, vocab), generator=torch.Generator().manual_seed(rows)) * 3).to(dtype)
    z[1, : vocab // 2] = -INF
    ids, tl, t = (x.to(gpu) for x in _teacher(rows, 3, vocab, 5))
    t[1] = vocab - 1
    zd, got = z.to(gpu), []
    for tau in (1.0, 1e-6, 0.3, 2.0, 1e6):
        dz = torch.empty_like(zd)
        loss = D.distill_topk(zd, ids, tl, None, dz, tau, 0.0, t)
        only = D.distill_topk(zd, ids, tl, None, None, tau, 0.0, t)
        got.append((loss, only, dz))
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))
    want = torch.logsumexp(zd.double(), 1) - zd.double().gather(1, t.long()[:, None])[:, 0]
    assert float((got[0][0].double() - want).abs().max()) <= 1e-4


def test_hard_labels_alone_need_no_entries(built_lib, gpu):
    z = torch.randn((5, 3001), generator=torch.Generator().manual_seed(1)).to(gpu)
    ids, tl, t = (x.to(gpu) for x in _teacher(5, 4, 3001, 2))
    a, b = torch.empty_like(z), torch.empty_like(z)
    want = D.distill_topk(z, ids, tl, None, a, 1.0, 0.0, t)
    assert torch.equal(D.distill_topk(z, None, None, None, b, 1.0, 0.0, t), want) and torch.equal(a, b)
    # on the head, in more than one block of rows
    cfg = MINI.with_(name="entries", n_layers=1, hidden=128, n_heads=1, n_kv_heads=1, head_dim=128, ffn=192, vocab=50304,
                     batch=1, seq=64)
    dm = D.DeviceModel(make_inputs(cfg, seed=3, norm="random"), device=str(gpu))
    rows = 1700
    x = torch.randn((rows, 128), generator=torch.Generator().manual_seed(4)).to(gpu)
    ids, tl, t = (v.to(gpu) for v in _teacher(rows, 4, cfg.vocab, 5))
    a, b = torch.empty_like(x), torch.empty_like(x)
    dm.lm_head_distill(x, a, ids, tl, 1.0, 0.0, t)
    loss = dm.loss.clone()
    dm.lm_head_distill(x, b, None, None, 1.0, 0.0, t)
    assert torch.equal(loss, dm.loss) and torch.equal(a, b)


@pytest.mark.parametrize("tau", [0.02, 0.5, 1.0, 1.7])
@pytest.mark.parametrize("vocab", [1003, 70001])
def test_an_unlikely_entry_at_a_students_lowest_value(built_lib, gpu, tau, vocab):
    """Its term is alpha tau p times the distance, a number of fp32 where the distance in temperatures is none."""
    tau = float(torch.tensor(tau, dtype=F32))
    z = torch.randn((3, vocab), generator=torch.Generator().manual_seed(1))
    ids, tl, t = _teacher(3, 4, vocab, 2)
    z[torch.arange(3), ids[:, 0].long()] = torch.finfo(F32).min
    tl[:, 0] = tl[:, 1:].amin(1) - torch.tensor([5.0, 20.0, 60.0]) * tau
    zd, dz = z.to(gpu), torch.empty((3, vocab), device=gpu)
    loss = D.distill_topk(zd, ids.to(gpu), tl.to(gpu), None, dz, tau, 1.0)
    only = D.distill_topk(zd, ids.to(gpu), tl.to(gpu), None, None, tau, 1.0)
    torch.cuda.synchronize()
    assert bool(torch.isfinite(loss).all())
    for got in (loss, only):
        _close(z, ids, tl, t, tau, 1.0, got, dz, f"{tau}")
