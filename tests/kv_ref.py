"""Rotary positions, the paged 8-bit cache and attention over it in 64 bits on the CPU, and the error
bounds that their tests use (no test functions here)."""
import math

import torch

from logits_ref import HALF_STEP

INF, NAN = math.inf, math.nan
F64 = torch.float64
EPS = 2.0 ** -24
BLOCK = 16


def frequencies(rot, theta, factor=1.0, original=0, low=1.0, high=32.0):
    f = theta ** (-torch.arange(0, rot, 2, dtype=F64) / rot)
    if not original:
        return f / factor
    g = ((original * f / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
    return f * (g + (1 - g) / factor)


def table(n_pos, rot, theta, gain=1.0, **kw):
    a = torch.arange(n_pos, dtype=F64)[:, None] * frequencies(rot, theta, **kw)
    return gain * torch.stack([torch.cos(a), torch.sin(a)], 2)


def pair_index(rot, interleaved):
    j = torch.arange(rot // 2)
    return (2 * j, 2 * j + 1) if interleaved else (j, j + rot // 2)


def turn(x, tab, pos, interleaved=False, backward=False):
    """x [tokens][heads][dim] in 64 bits turned by tab [n_pos][rot / 2][2] at pos."""
    y = x.double().clone()
    ok = (pos >= 0) & (pos < tab.shape[0])
    t = tab.double()[pos.clamp(0, tab.shape[0] - 1).long()]
    t = torch.where(ok[:, None, None], t, torch.full_like(t, NAN))[:, None]
    a, b = pair_index(2 * tab.shape[1], interleaved)
    c, s = t[..., 0], t[..., 1] * (-1 if backward else 1)
    xa, xb = x.double()[..., a], x.double()[..., b]
    y[..., a] = xa * c - xb * s
    y[..., b] = xb * c + xa * s
    return y


def turn_bound(x, tab, pos, interleaved, dtype):
    """Two products and a sum in fp32, one of the products possibly exact inside a fused step, and one
    rounding to the type: 3 half steps of |x_a c| + |x_b s| and one of the result. A half step relative to the
    result is for normal numbers: below 2^-14 those of fp16 are all 2^-24 apart, and a rounding is off by up to half of
    that, 2^-25, whatever the result."""
    m = turn(x.double().abs(), tab.abs() * torch.tensor([1.0, -1.0]), pos, interleaved).abs()
    m = torch.maximum(m, turn(x.double().abs(), tab.abs(), pos, interleaved).abs())
    return m * (3 * EPS + HALF_STEP[dtype] * (1 + 2 * EPS)) + (2.0 ** -25 if dtype is torch.float16 else 0.0)


class Cache:
    """Codes and scales as the library lays them out, on the CPU."""

    def __init__(self, pages, scales):
        self.pages, self.scales = pages.clone(), scales.clone()
        self.n, self.heads, self.blocks = pages.shape[:3]
        self.dim = pages.shape[4] // BLOCK
        self.page = self.blocks * BLOCK

    def where(self, row, tok):
        """(page, block) of a token of the sequence with the table row, or None."""
        c = tok // self.page
        if c >= len(row) or not 0 <= int(row[c]) < self.n:
            return None
        return int(row[c]), tok % self.page // BLOCK

    def codes(self, page, b):
        k = self.pages[page, :, b, 0].view(self.heads, BLOCK, self.dim)
        v = self.pages[page, :, b, 1].view(self.heads, self.dim, BLOCK).transpose(1, 2)
        return k, v

    def append(self, row, past, k, v):
        """New keys (turned already) and values [n][heads][dim] in 64 bits."""
        n, tok = k.shape[0], past
        while tok < past + n:
            end = min((tok // BLOCK + 1) * BLOCK, past + n)
            at = self.where(row, tok)
            if at is not None:
                for x, c, w in zip((k, v), self.codes(*at), (0, 1)):
                    new = x[tok - past:end - past].transpose(0, 1)
                    amax = new.abs().amax((1, 2))
                    want = torch.where(torch.isfinite(amax), amax / 127.0, torch.full_like(amax, NAN)).float()
                    old = self.scales[at[0], :, at[1], w].clone() if tok % BLOCK else torch.zeros_like(want)
                    scale = torch.maximum(old, want)
                    self.scales[at[0], :, at[1], w] = scale
                    sc = torch.where(scale > 0, scale, torch.ones_like(scale)).double()[:, None, None]
                    # (under a scale of NaN codes are 0)
                    r = torch.where(scale.isnan()[:, None, None], torch.zeros_like(new), torch.round(new / sc).clamp(-127, 127))
                    c[:, tok % BLOCK:tok % BLOCK + end - tok] = torch.where(torch.isfinite(r), r, torch.zeros_like(r)).to(torch.int8)
                    if tok % BLOCK:
                        rise = torch.where(scale > 0, old.double() / sc[:, 0, 0], torch.zeros_like(sc[:, 0, 0]))[:, None, None]
                        c[:, :tok % BLOCK] = torch.round(c[:, :tok % BLOCK].double() * rise).nan_to_num(0).to(torch.int8)
            tok = end

    def read(self, row, first, n):
        """Keys and values [n][heads][dim] in 64 bits."""
        k = torch.full((n, self.heads, self.dim), NAN, dtype=F64)
        v = k.clone()
        for i in range(n):
            at = self.where(row, first + i)
            if at is None:
                continue
            t = (first + i) % BLOCK
            for o, c, w in zip((k, v), self.codes(*at), (0, 1)):
                o[i] = c[:, t].double() * self.scales[at[0], :, at[1], w].double()[:, None]
        return k, v


def attention(q, k, v, past, scale, window=0):
    """q [n][heads][dim] of tokens past .., over k, v [length][kv heads][dim]: out, lse, and the bounds of
    their errors but for the rounding of out."""
    n, hq, d = q.shape
    length, hkv = k.shape[:2]
    k, v = (x.repeat_interleave(hq // hkv, 1) for x in (k, v))
    i = torch.arange(past, past + n)[:, None]
    j = torch.arange(length)[None, :]
    hide = (j > i) | ((j <= i - window) if window else torch.zeros_like(j > i))
    qd = q.double()
    # (float products on the CPU, heads first)
    dot = torch.matmul(qd.permute(1, 0, 2), k.permute(1, 2, 0))
    x = (dot * scale).masked_fill(hide, -INF)
    size = (torch.matmul(qd.abs().permute(1, 0, 2), k.abs().permute(1, 2, 0)) * abs(scale)).masked_fill(hide, 0.0)
    lse = torch.logsumexp(x, 2)
    w = torch.exp(x - lse[..., None])
    w = torch.where(torch.isnan(x), torch.full_like(w, NAN), w).masked_fill(hide, 0.0)
    vv = v.permute(1, 0, 2)
    # (a value that is NaN where nothing sees it is no term)
    out = torch.einsum("hnj,hjd->hnd", w, vv.nan_to_num(0))
    bad = torch.isnan(w).any(2) | ((w > 0) & torch.isnan(vv).any(2)[:, None]).any(2)
    seen = ~hide[None].expand(hq, -1, -1)
    bad |= (seen & torch.isnan(vv).any(2)[:, None]).any(2) | (seen & torch.isnan(x)).any(2)
    out[bad] = NAN
    lse[(seen & torch.isnan(x)).any(2)] = NAN
    # a score: products exact, d fp32 additions, the row's and the block's factor and the difference of
    # the running maximum (whose own size is that of a score): (d + 6) half steps of sum |q k|; a weight
    # besides: exp2's 2^-22; for the output one rounding to fp16 (2^-11), or 2^-25 of a weight 2^5
    delta = (d + 6) * EPS * size.nan_to_num(0).amax(2, keepdim=True)
    terms = torch.einsum("hnj,hjd->hnd", w.nan_to_num(0), vv.abs().nan_to_num(0))
    vmax = vv.abs().nan_to_num(0).amax()
    add = (64 + length / 64) * EPS
    bound = terms * (2.0 ** -11 + 2 * (2 * delta + 2.0 ** -22 + add)) + length * 2.0 ** -29 * vmax
    lse_bound = delta[..., 0] + 2.0 ** -22 + add + 6 * EPS * (lse.nan_to_num(0, 0, 0).abs() + 8)
    return out.permute(1, 0, 2), lse.t(), bound.permute(1, 0, 2), lse_bound.t()


def check(got, ref, bound, what):
    g, r = got.double().cpu(), ref.double()
    fine = torch.isfinite(r)
    assert torch.equal(torch.isnan(g), torch.isnan(r)), f"{what}: NaN in other places"
    assert torch.equal(g[~fine & ~torch.isnan(r)], r[~fine & ~torch.isnan(r)]), f"{what}: infinities differ"
    d = (g - r).abs()[fine]
    b = (bound if torch.is_tensor(bound) else torch.full_like(r, bound)).expand_as(r)[fine]
    over = d > b
    assert not bool(over.any()), f"{what}: off by {float((d - b).max())} beyond its bound, at {int(over.sum())} of {d.numel()}"
