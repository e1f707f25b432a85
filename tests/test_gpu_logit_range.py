"""The operators on logits on the GPU at the ends of what they accept: large gradients of the
entropy beside masked columns, rows whose log-sum-exp has no room for the number of their columns."""
import math

import pytest
import torch

import logits_ref as R
from gpu_util import say
from paper_2510_03425_amd import device as D

pytestmark = pytest.mark.gpu
INF = math.inf
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
EPS = 2.0 ** -24


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("tau,d_entropy", [(1e-6, 1000.0), (1e-3, 5e5), (1.0, 1e20), (1.0, -1e30)])
def test_masked_columns_have_no_gradient_whatever_the_entropys_is(built_lib, gpu, dtype, tau, d_entropy):
    """d_entropy / tau beyond 3.4e8: its product with a weight's logarithm is no number of fp32 where
    the logarithm is far below any weight's. Columns whose weight is 0 (masked by -inf, by the type's
    lowest value or by -3e4 of fp16) have gradient 0 at any such factor."""
    say("masked columns", dtype, tau, d_entropy)
    z = (torch.randn((4, 3001), generator=torch.Generator().manual_seed(1)) * 0.5).to(dtype)
    z[0, 2000:] = -INF
    z[1, :700] = torch.finfo(dtype).min
    z[2, ::2] = -3e4
    zd = z.to(gpu)
    t = torch.tensor([5, 800, 1, 7], dtype=torch.int32, device=gpu)
    s = D.token_logprobs(zd, t, 0, tau)
    one, de = torch.ones(4, device=gpu), torch.full((4,), d_entropy, device=gpu)
    for dl in (one, None):
        dz = D.token_logprobs_backward(zd, t, s["lse"], s["entropy"], dl, de, torch.empty_like(zd, dtype=F32), tau)
        assert not torch.isnan(dz).any()
        assert bool((dz[0, 2000:] == 0).all()) and bool((dz[1, :700] == 0).all()) and bool((dz[2, ::2] == 0).all())


def _grad_ref(z, t, tau, d_logp, d_entropy):
    """The gradient in 64 bits, of logits less their row's largest (no row is empty), and the sum of its
    terms' magnitudes."""
    u = (z.double() - z.double().amax(1, keepdim=True)) / tau
    lq = u - torch.log(torch.exp(u).sum(1, keepdim=True))
    q = torch.exp(lq)
    qlq = torch.where(q > 0, q * lq, torch.zeros_like(q))
    h = -qlq.sum(1, keepdim=True)
    one = torch.zeros_like(q).scatter_(1, t.long()[:, None], 1.0)
    A, B = d_logp.double()[:, None], d_entropy.double()[:, None]
    return ((A * (one - q) - B * (qlq + q * h)) / tau, (A.abs() * (one + q) + B.abs() * (qlq.abs() + q * h)) / tau,
            B.abs() * q / tau)


def _wide_rows(vocab, dtype):
    """Rows whose log-sum-exp is large beside the differences of their logits."""
    low, f = torch.finfo(dtype).min, 6e4 if dtype is F16 else 1e9
    g = torch.Generator().manual_seed(2)
    rows = {"all masked by a finite value": torch.full((vocab,), -f), "all lowest": torch.full((vocab,), low),
            "all large": torch.full((vocab,), f), "one above the rest": torch.full((vocab,), -f),
            "shifted": torch.randn(vocab, generator=g) + 4096, "shifted down": torch.randn(vocab, generator=g) * 3 - 3e4,
            "ordinary": torch.randn(vocab, generator=g) * 5}
    rows["one above the rest"][vocab // 3] = 0.0
    return list(rows), torch.stack(list(rows.values())).to(dtype)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("vocab", [1003, 40003])
@pytest.mark.parametrize("tau", [1.0, 0.05, 1e-3, 1e-6, 20.0, 1e4])
@pytest.mark.parametrize("in_place", [False, True])
def test_gradient_of_rows_with_a_large_log_sum_exp(built_lib, gpu, dtype, vocab, tau, in_place):
    """An fp32 log-sum-exp of 1e9 has no room for the logarithm of the number of columns: all weights of
    a row of equal logits would be 1. Up to 128 it is off by 2^-18 at most, and weights by as much."""
    names, z = _wide_rows(vocab, dtype)
    tau = float(torch.tensor(tau, dtype=F32))
    n = len(names)
    # (a quotient beyond fp32 is no logit: the row's log-sum-exp is -inf, its gradient 0 by definition)
    keep = [i for i in range(n) if float(z[i].double().abs().max()) / tau < 3.4029e38]
    names, z = [names[i] for i in keep], z[keep]
    t = (torch.arange(len(keep), dtype=torch.int32) * 131 + 7) % vocab
    dl, de = torch.linspace(1, 2, len(keep)) * tau, torch.linspace(0.5, -1, len(keep)) * tau
    zd = z.to(gpu)
    s = D.token_logprobs(zd, t.to(gpu), 0, tau)
    dz = zd if in_place else torch.empty_like(zd, dtype=F32)
    D.token_logprobs_backward(zd, t.to(gpu), s["lse"], s["entropy"], dl.to(gpu), de.to(gpu), dz, tau)
    torch.cuda.synchronize()
    ref, mag, per_h = _grad_ref(z, t, tau, dl, de)
    for i, name in enumerate(names):
        say("wide row", name, dtype, vocab, tau)
        # a weight: its exponent, at most 104 of it, times 1 / tau and log2(e) (2^-24 each); the sum of them:
        # additions of a lane's columns, of a vector's and of the joins; the log-sum-exp as above; the
        # hardware's exp2 and log2
        x = z[i].double()
        dr = min(float((x.max() - x.min()) / tau), 104.0)
        rel = (5 * dr + vocab / 1024 + 60) * EPS + 2 ** -17
        # the entropy's own error: its terms as above, times their logarithms. A weight below 2^-126 is 0:
        # that is 2^-126 times (|d_logp| + |d_entropy| (|ln q| + H)) / tau <= 2 + 1 * (88 + 11) at most
        tol = rel * mag[i] + (rel * (12 + dr) + 20 * EPS) * per_h[i] + 128 * 2.0 ** -126
        tol = tol + R.HALF_STEP[dz.dtype] * 1.001 * ref[i].abs() + R.TINY[dz.dtype]
        R.close(dz[i], ref[i], tol, name)


def test_wide_rows_by_parts_and_beside_ordinary_ones(built_lib, gpu):
    """The whole of such a row, and nothing of its neighbours, is written by one of its parts."""
    vocab = 30011
    z = torch.randn((5, vocab), generator=torch.Generator().manual_seed(4)) * 2
    z[1], z[3] = -1e9, z[3] + 5e4
    t = torch.tensor([3, vocab - 1, 7, 20000, 0], dtype=torch.int32)
    zd, buf = z.to(gpu), torch.full((5, vocab + 5), 7.0, device=gpu)
    one = torch.ones(5, device=gpu)
    s = D.token_logprobs(zd, t.to(gpu))
    for dz in (buf[:, :vocab], zd):
        D.token_logprobs_backward(zd, t.to(gpu), s["lse"], s["entropy"], one, None, dz)
        got = dz.double().cpu()
        want = torch.nn.functional.one_hot(t.long(), vocab) - torch.softmax(z.double(), 1)
        assert float((got - want).abs().max()) <= 2 ** -14  # (q of at most 1, 40 logits apart)
        assert bool((got.sum(1).abs() <= 2 ** -13).all())
    assert bool((buf[:, vocab:] == 7.0).all())


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("vocab", [1003, 40003])
@pytest.mark.parametrize("in_place", [False, True])
def test_gradient_of_rows_without_a_softmax(built_lib, gpu, dtype, vocab, in_place):
    """A NaN or +inf logit makes its row NaN, masked columns and all; a row of nothing but -inf is 0; the rows
    beside them are their own."""
    z = torch.randn((6, vocab), generator=torch.Generator().manual_seed(8)).to(dtype)
    z[1, vocab - 1], z[2, 5], z[3], z[4, 7] = float("nan"), INF, -INF, -INF
    z[1, 3:9] = -INF
    t = torch.tensor([1, 2, 5, 0, 7, -1], dtype=torch.int32)
    zd = z.to(gpu)
    s = D.token_logprobs(zd, t.to(gpu))
    one = torch.ones(6, device=gpu)
    dz = zd if in_place else torch.empty_like(zd)
    D.token_logprobs_backward(zd, t.to(gpu), s["lse"], s["entropy"], one, one, dz)
    got = dz.double().cpu()
    assert bool(torch.isnan(got[1:3]).all()) and bool((got[3] == 0).all())
    # the label on a masked column: 1 there, as the header has it
    for r, hot in ((0, 1.0), (4, 1.0), (5, 0.0)):
        lq = torch.log_softmax(z[r].double(), 0)
        q = lq.exp()
        h = torch.special.entr(q)
        want = torch.zeros(vocab, dtype=torch.float64)
        if hot:
            want[t[r]] = 1.0
        want = want - hot * q + h - q * h.sum()
        # (a lane's additions as above; fp32 numbers of the row)
        R.close(got[r], want, (vocab / 1024 + 200) * EPS * (q * (2 + (-lq).clamp_max(104) + h.sum())) + 2 ** -18 * q
                + R.HALF_STEP[dtype] * 1.001 * want.abs() + 2.0 ** -126 * 128 + R.TINY[dtype], f"row {r}")
