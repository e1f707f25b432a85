"""Rows whose largest logit comes late and stands far above the first ones, on the GPU against 64
bits: log probabilities that are not above 0, entropies that are not below it, and both to the
bits that a sum relative to the row's largest logit has."""
import pytest
import torch

import logits_ref as R
from gpu_util import say
from paper_2510_03425_amd import device as D

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
EPS = 2.0 ** -24


def _weight_error(z, tau):
    """Relative error of a sum of weights: an exponent of at most 104 (further down they are 0) is off by
    three roundings of it, the hardware's exp2 by 2^-22; a lane's additions (of 256 lanes, 4 logits
    a vector), a vector's, and those of the joins."""
    x = z.double()
    x = torch.where(torch.isfinite(x), x, x.new_zeros(()))
    dr = min(float((x.amax(1) - x.amin(1)).max()) / tau, 104.0)
    return (3 * dr + 4 + z.shape[1] / 1024 + 8 + 20) * EPS


def _check(z, t, k, tau, got):
    ref = R.scores(z, t, k, tau)
    e = _weight_error(z, tau)
    q = torch.softmax(z.double() / tau, 1)
    rest = 1 - q.amax(1)  # what the largest logit's own weight, 1, leaves
    lq = torch.log_softmax(z.double() / tau, 1)
    spread = torch.where(q > 0, q * lq, torch.zeros_like(q)).abs().sum(1)
    assert bool((got["logp"] <= 0).all()) and bool((got["entropy"] >= 0).all())
    # (logp: the logarithm's own rounding, that of its argument, and of the difference beside it)
    own = e * rest + 8 * EPS
    R.close(got["logp"], ref["logp"], own + 4 * EPS * ref["logp"].abs(), "logp")
    R.close(got["entropy"], ref["entropy"], 2 * e * (spread + rest) + 8 * EPS * (1 + ref["entropy"]), "entropy")
    R.close(got["lse"], ref["lse"], own + 4 * EPS * (z.double().abs().amax(1) / tau + ref["lse"].abs()), "lse")
    if k:
        assert bool((got["top_logp"] <= 0).all())
        assert torch.equal(got["top_ids"].cpu(), ref["top_ids"])
        R.close(got["top_logp"], ref["top_logp"], own[:, None] + 4 * EPS * ref["top_logp"].abs(), "top_logp")


def _rows(n, vocab, dtype, late=True):
    """n rows of standard normal logits and one 8 .. 48 above, behind the first three quarters or not."""
    g = torch.Generator().manual_seed(vocab + n)
    z = torch.randn((n, vocab), generator=g)
    at = torch.randint(vocab * 3 // 4 if late else 0, vocab, (n,), generator=g)
    z[torch.arange(n), at] = torch.linspace(8, 48, n)
    return z.to(dtype), at.to(torch.int32)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("rows,vocab,k", [(41, 50257, 0), (41, 50257, 9), (41, 70001, 0), (41, 70001, 64), (165, 66001, 3), (41, 3001, 5)])
def test_scores_of_sure_rows(built_lib, gpu, dtype, rows, vocab, k):
    say("sure rows", rows, vocab, k, dtype)
    z, t = _rows(rows, vocab, dtype)
    for tau in (1.0, 0.7):
        tau = float(torch.tensor(tau, dtype=F32))
        _check(z, t, k, tau, D.token_logprobs(z.to(gpu), t.to(gpu), k, tau))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tau", [1e-6, 1e-3, 0.05, 0.2, 20.0, 1e4, 1e6])
@pytest.mark.parametrize("vocab", [5003, 70001])
def test_scores_at_any_temperature(built_lib, gpu, dtype, tau, vocab):
    tau = float(torch.tensor(tau, dtype=F32))
    say("temperature", tau, vocab, dtype)
    z = (torch.randn((9, vocab), generator=torch.Generator().manual_seed(6)) * 4).to(dtype)
    z[2, : vocab // 2] = -float("inf")  # the first columns masked
    z[3] = z[3] + 300
    z[4] = z[4] - 7e4
    z[5] = torch.linspace(-20, 20, vocab)  # (each group's largest above the last one's)
    t = torch.randint(vocab // 2, vocab, (9,), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    _check(z, t, 6, tau, D.token_logprobs(z.to(gpu), t.to(gpu), 6, tau))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,vocab", [(13, 3001), (13, 70001), (97, 40003), (97, 151936)])
@pytest.mark.parametrize("tau", [1.0, 2.0, 3.0, 0.2])
def test_hard_label_of_sure_students(built_lib, gpu, dtype, rows, vocab, tau):
    """The cross-entropy of a label that the student is sure of, beside a distillation term of weight
    2^-20: the sum at temperature 1 of a call at 3 stands up to 2^69 above that at the first logits."""
    say("sure students", rows, vocab, tau, dtype)
    z, t = _rows(rows, vocab, dtype)
    tau, alpha = float(torch.tensor(tau, dtype=F32)), 2.0 ** -20
    ids = t[:, None].clone()
    tl = torch.zeros((rows, 1))
    zd, args = z.to(gpu), (ids.to(gpu), tl.to(gpu))
    dz = torch.empty_like(zd, dtype=F32)
    loss = D.distill_topk(zd, *args, None, dz, tau, alpha, t.to(gpu))
    only = D.distill_topk(zd, *args, None, None, tau, alpha, t.to(gpu))
    torch.cuda.synchronize()
    some = slice(0, rows, 1 if vocab < 10000 else 6)
    ref, lmag, g, gmag = R.distill(z[some], ids[some], tl[some], t[some], None, tau, alpha)
    e = max(_weight_error(z, tau), _weight_error(z, 1.0))
    rest = 1 - torch.softmax(z[some].double(), 1).amax(1)
    for got in (loss[some], only[some]):
        assert bool((got >= 0).all())
        R.close(got, ref, e * rest + 16 * EPS + 4 * e * alpha * (tau * tau * 40 + 1) + 8 * EPS * lmag, "loss")
    R.close(dz[some], g, (4 * e + 16 * EPS) * gmag + R.TINY[F32], "dz")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,vocab,k", [(3, 5003, 64), (3, 70001, 20), (170, 66001, 64), (3, 40003, 1)])
def test_alternatives_beside_long_runs_of_nan(built_lib, gpu, dtype, rows, vocab, k):
    """Lanes, waves and parts that see nothing but NaN rank nothing and leave the others' order alone."""
    z = torch.randn((rows, vocab), generator=torch.Generator().manual_seed(9)).to(dtype)
    z[0, : vocab * 2 // 3] = float("nan")
    z[1, (torch.arange(vocab) // 8) % 2 == 0] = float("nan")  # whole vectors of lanes
    z[2, 100:] = float("nan")
    got = D.token_logprobs(z.to(gpu), torch.zeros(rows, dtype=torch.int32, device=gpu), k)
    x = torch.where(torch.isnan(z), torch.full_like(z, -float("inf")), z)[:3]
    val, ids = torch.sort(x.double(), dim=1, descending=True, stable=True)
    want = torch.where(val[:, :k] > -float("inf"), ids[:, :k], -torch.ones_like(ids[:, :k])).to(torch.int32)
    assert torch.equal(got["top_ids"][:3].cpu(), want)
    assert bool(torch.isnan(got["lse"][:3]).all()) and bool(torch.isnan(got["entropy"][:3]).all())
