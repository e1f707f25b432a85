"""The operators on logits in 64 bits, and the error bounds that their tests use (no test
functions here)."""
import math

import torch

INF, NAN = math.inf, math.nan
HALF_STEP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -126}


def softmax_bound(z, tau):
    """Relative error of a softmax weight or of the sum of them that fp32 may have.

    A weight exp2((z - m) c): the difference, c, and the product are rounded (2^-24 each, of an
    exponent whose natural logarithm is at most D), the hardware's exp2 is off by at most 2^-22 (and
    a reference that lags behind scales all alike). A sum: at most vocab / 256 additions per lane of
    a 256-lane workgroup, one vector of 8, and 6 + 4 + 6 levels above, 2^-24 each."""
    f = z.double()
    f = torch.where(torch.isfinite(f), f, torch.zeros_like(f))
    D = float((f.amax(1) - f.amin(1)).max()) / tau if f.numel() else 0.0
    D = min(D, 104.0)  # (weights further below the largest are 0 in fp32)
    return (3 * D + 4 + z.shape[1] / 256 + 8 + 16) * 2.0 ** -24, D


def scores(z, targets, top_k, tau):
    u = z.double() / tau
    n, v = u.shape
    m = u.amax(1, keepdim=True)
    bad = torch.isnan(u).any(1) | (m[:, 0] == INF)
    empty = (m[:, 0] == -INF) & ~bad
    m = torch.where(torch.isfinite(m), m, torch.zeros_like(m))
    e = torch.exp(u - m)
    s = e.sum(1, keepdim=True)
    lse = (m + torch.log(s))[:, 0]
    q = e / s
    # (not u - lse, which loses ln s beside logits of a type's lowest value)
    lq = (u - m) - torch.log(s)
    ent = -(torch.where(q > 0, q * lq, torch.zeros_like(q))).sum(1)
    ent[empty], lse[empty] = 0.0, -INF
    ent[bad], lse[bad] = NAN, NAN
    out = {"lse": lse, "entropy": ent}
    if targets is not None:
        t = targets.long()
        ok = (t >= 0) & (t < v)
        lp = lq.gather(1, t.clamp(0, v - 1)[:, None])[:, 0]
        lp[empty] = -INF
        lp[bad] = NAN
        lp[t >= v] = NAN
        lp[t < 0] = 0.0
        out["logp"] = lp
    if top_k:
        ids = torch.full((n, top_k), -1, dtype=torch.int32)
        tl = torch.full((n, top_k), -INF, dtype=torch.float64)
        for r in range(n):
            x = z[r].double()
            x = torch.where(torch.isnan(x), torch.full_like(x, -INF), x)
            val, order = torch.sort(x, descending=True, stable=True)
            c = min(top_k, int((val > -INF).sum()))
            ids[r, :c] = order[:c].to(torch.int32)
            tl[r, :c] = lq[r][order[:c]]
            if bad[r]:
                tl[r, :c] = NAN
        out["top_ids"], out["top_logp"] = ids, tl
    return out


def scores_grad(z, targets, tau, d_logp, d_entropy):
    """The gradient, and the sum of its terms' magnitudes (for the bound)."""
    s = scores(z, None, 0, tau)
    n, v = z.shape
    lse, ent = s["lse"][:, None], s["entropy"][:, None]
    lq = z.double() / tau - lse
    q = torch.exp(lq)
    A = torch.zeros(n, 1, dtype=torch.float64) if d_logp is None else d_logp.double()[:, None].clone()
    one = torch.zeros_like(q)
    if d_logp is not None:
        t = targets.long()
        A[t < 0] = 0.0
        A[t >= v] = NAN
        ok = (t >= 0) & (t < v)
        one[ok.nonzero()[:, 0], t[ok]] = 1.0
    B = torch.zeros(n, 1, dtype=torch.float64) if d_entropy is None else d_entropy.double()[:, None]
    qlq = torch.where(q > 0, q * lq, torch.zeros_like(q))
    g = (A * (one - q) - B * (qlq + q * ent)) / tau
    mag = (A.abs() * (one + q) + B.abs() * (qlq.abs() + q * ent.abs())) / tau
    empty = torch.isneginf(lse[:, 0])
    g[empty], mag[empty] = 0.0, 0.0
    return g, mag


def distill(z, ids, teacher, targets, weight, tau, alpha):
    """Row losses, the gradient, and the sums of their terms' magnitudes."""
    n, v = z.shape
    k = ids.shape[1]
    w = torch.ones(n, dtype=torch.float64) if weight is None else weight.double()
    loss, lmag = torch.zeros(n, dtype=torch.float64), torch.zeros(n, dtype=torch.float64)
    dz, gmag = torch.zeros(n, v, dtype=torch.float64), torch.zeros(n, v, dtype=torch.float64)
    for r in range(n):
        if w[r] == 0:
            continue
        x = z[r].double()
        t = -1 if alpha == 1 else int(targets[r])
        use = (ids[r] >= 0) & (teacher[r] != -INF) if alpha > 0 else torch.zeros(k, dtype=torch.bool)
        i, tl = ids[r][use].long(), teacher[r][use].double() / tau
        if bool((x == -INF).all()):
            loss[r] = INF if (len(i) or t >= 0) else 0.0
            if bool((i >= v).any()) or t >= v:
                loss[r] = NAN
            loss[r] *= w[r]
            continue
        if bool(torch.isnan(x).any()) or bool((x == INF).any()):
            if len(i) or t >= 0:
                loss[r], dz[r] = NAN, NAN
            continue
        q, q1 = torch.softmax(x / tau, 0), torch.softmax(x, 0)
        L = torch.zeros((), dtype=torch.float64)
        if len(i):
            if bool((i >= v).any()):
                loss[r], dz[r] = NAN, NAN
                continue
            p = torch.softmax(tl, 0)
            lq = x / tau - torch.logsumexp(x / tau, 0)
            seen = p > 1e-45
            term = torch.where(seen, p * (torch.log(p) - lq[i]), torch.zeros_like(p))
            L += alpha * tau * tau * term.sum()
            lmag[r] += alpha * tau * tau * torch.where(seen, p * (torch.log(p).abs() + lq[i].abs()), torch.zeros_like(p)).sum()
            dz[r] += alpha * tau * q
            gmag[r] += alpha * tau * q
            dz[r].index_add_(0, i, -alpha * tau * p)
            gmag[r].index_add_(0, i, alpha * tau * p)
        if t >= v:
            loss[r], dz[r] = NAN, NAN
            continue
        if t >= 0:
            ce = torch.logsumexp(x, 0) - x[t]
            L += (1 - alpha) * ce
            lmag[r] += (1 - alpha) * ce.abs()
            dz[r] += (1 - alpha) * q1
            gmag[r] += (1 - alpha) * q1
            dz[r, t] -= 1 - alpha
            gmag[r, t] += 1 - alpha
        loss[r] = w[r] * L
        dz[r] *= w[r]
        gmag[r] *= w[r].abs()
        lmag[r] *= w[r].abs()
    return loss, lmag, dz, gmag


def close(got, ref, tol, what):
    """Equal where the reference is not finite (NaN as NaN), within tol elsewhere."""
    got, ref = got.double().cpu(), ref.double().cpu()
    fine = torch.isfinite(ref)
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), f"{what}: NaN in other places"
    inf = torch.isinf(ref)
    assert torch.equal(got[inf], ref[inf]), f"{what}: infinities"
    tol = tol.double().cpu().expand_as(ref) if isinstance(tol, torch.Tensor) else torch.full_like(ref, tol)
    d = (got - ref).abs()[fine]
    bad = ~(d <= tol[fine])
    if bad.any():
        worst = int((d / tol[fine].clamp_min(1e-300)).argmax())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} beyond the bound, worst {float(d[worst]):.3e} "
                             f"where {float(tol[fine][worst]):.3e} is allowed")
