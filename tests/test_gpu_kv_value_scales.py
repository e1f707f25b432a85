"""Attention over the paged 8-bit cache where the values' scales of a sequence's blocks are far apart. Every row
is held to what it sees by itself: its own keys, of its own kv head."""
import math

import pytest
import torch

import kv_ref as R
from gpu_util import say
from paper_2510_03425_amd import device as D
from test_gpu_kv_cache import Setup

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


def _value_scales(t, size):
    """The scales of the values of block b of every sequence times size(b) (a tensor of block numbers in, one of
    factors out)."""
    per = t.cache.struct.page_tokens // 16
    for row in t.table:
        for i, p in enumerate(row.tolist()):
            t.ref.scales[p, :, :, 1] *= size(i * per + torch.arange(per)).float()
    t.cache.scales.copy_(t.ref.scales)


def _check_rows(t, q, out, window):
    group = q.shape[1] // t.heads
    for s, (past, new) in enumerate(zip(t.past, t.new)):
        k, v = t.ref.read(t.table[s], 0, past + new)
        for i in range(new):
            r, pos = t.start[s] + i, past + i
            lo = max(0, pos - window + 1) if window else 0
            for h in range(t.heads):
                g = slice(h * group, (h + 1) * group)
                o, _, b, _ = R.attention(q[r:r + 1, g], k[lo:pos + 1, h:h + 1], v[lo:pos + 1, h:h + 1], pos - lo, t.dim ** -0.5)
                R.check(out[r:r + 1, g], o, b * (1 + R.HALF_STEP[q.dtype]) + o.abs() * R.HALF_STEP[q.dtype] + 2.0 ** -25,
                        f"sequence {s}, position {pos}, kv head {h}")


def _run(t, q, window):
    return D.kv_attention(t.cache, t.batch, q.to(t.gpu), window=window)


@pytest.mark.parametrize("room", [0, 1 << 20])  # (with room for long sequences many rows go by large tiles)
@pytest.mark.parametrize("hkv,hq,dim,past,new", [
    (1, 4, 64, 0, 40), (2, 6, 64, 3, 90), (1, 4, 128, 0, 40), (1, 6, 128, 0, 100), (2, 4, 256, 0, 21), (1, 4, 256, 0, 130), (1, 3, 128, 60, 7),
])
def test_rows_do_not_depend_on_blocks_that_they_do_not_see(built_lib, gpu, room, hkv, hq, dim, past, new):
    """Blocks whose values are 2^24 and 2^40 times those of the blocks before them, which rows in front of them do not
    see; and the other way round, blocks that windows have left behind."""
    say("unseen blocks", room, hkv, hq, dim, past, new)
    for dtype, low, high in ((BF16, 1.0, 2.0 ** 24), (BF16, 1.0, 2.0 ** 40), (F16, 2.0 ** -14, 2.0 ** 10)):
        for window, size in ((0, lambda b: torch.where(b % 2 == 1, high, low)), (0, lambda b: torch.where(b >= 1, high, low)),
                             (0, lambda b: torch.where(b == 3, high, low)), (17, lambda b: torch.where(b % 4 == 0, high, low)),
                             (40, lambda b: torch.where(b < 2, high, low)), (5, lambda b: torch.where(b % 3 == 1, high, low))):
            t = Setup(gpu, hkv, dim, 32, [past], [new], seed=new, max_len=room or None)
            _value_scales(t, size)
            q = t.heads_of(hq, dtype, 0.5)
            _check_rows(t, q, _run(t, q, window), window)


def _check_to_rounding(t, q, out, window=0):
    """Every output within the roundings of fp32 and its type's, relative to its own terms sum w |v| alone: of a weight
    2^-17 (two bf16) and 2^-22 (its exponential), of its score and its row's sum of weights the same again, (dim + 6)
    half steps of sum |q k|, and half a step for each addition (a wave adds a quarter of the keys at least)."""
    (past,), (new,) = t.past, t.new
    k, v = (x.repeat_interleave(q.shape[1] // t.heads, 1).permute(1, 0, 2) for x in t.ref.read(t.table[0], 0, past + new))
    qd, length, scale = q.double().permute(1, 0, 2), past + new, t.dim ** -0.5
    i, j = torch.arange(past, length)[:, None], torch.arange(length)[None, :]
    hide = (j > i) | ((j <= i - window) if window else torch.zeros_like(j > i))
    w = torch.softmax((qd @ k.transpose(1, 2) * scale).masked_fill(hide, -math.inf), 2)
    o, terms = w @ v, w @ v.abs()
    size = (qd.abs() @ k.abs().transpose(1, 2) * scale).masked_fill(hide, 0).amax(2, keepdim=True)
    delta = (t.dim + 6) * R.EPS * size
    bound = terms * (2.0 ** -17 + 2 * (2 * delta + 2.0 ** -22 + (64 + length / 4) * R.EPS))
    half, least = R.HALF_STEP[q.dtype], 2.0 ** -25 if q.dtype is F16 else 2.0 ** -134
    R.check(out.permute(1, 0, 2), o, bound * (1 + half) + o.abs() * half + least, "out")


@pytest.mark.parametrize("dim,hq,past,new,room", [
    (64, 4, 3000, 1, 0), (64, 8, 2000, 4, 0), (64, 2, 2000, 70, 1 << 20), (128, 4, 3000, 1, 0), (128, 2, 2000, 100, 1 << 20), (256, 4, 3000, 1, 0),
    (256, 2, 2000, 70, 1 << 20),
])
def test_many_small_weights_beside_a_sure_key(built_lib, gpu, dim, hq, past, new, room):
    """One key takes all but a small part of the softmax, in a block of large scale whose values are 0 where the others'
    many small ones are looked for."""
    say("sure key", dim, hq, past, new, room)
    for at in (3, past // 2 + 5, past):
        for dtype, low, ratio in ((F16, 60.0, 255.0), (F16, 60.0, 500.0), (BF16, 1.0, 255.0), (BF16, 1.0, 2.0 ** 30), (BF16, 2.0 ** -60, 2.0 ** 90),
                                  (BF16, 2.0 ** -110, 2.0 ** 30)):
            t = Setup(gpu, 1, dim, 64, [past], [new], seed=at, max_len=room or None)
            keys = t.ref.pages[:, :, :, 0].view(*t.ref.pages.shape[:3], 16, dim)
            keys.zero_()
            keys[..., 0] = torch.randint(0, 26, keys.shape[:-1], generator=t.gen, dtype=torch.int8)
            t.ref.scales[..., 0] = 1 / 127
            t.ref.scales[..., 1] *= low / 0.02
            p, b = t.ref.where(t.table[0], at)
            t.ref.scales[p, :, b, 1] = low * ratio
            k, v = t.ref.codes(p, b)
            k[:, at % 16, 0] = 127
            v[..., : dim if dtype is F16 else dim // 2] = 0
            t.cache.pages.copy_(t.ref.pages)
            t.cache.scales.copy_(t.ref.scales)
            q = torch.zeros(new, hq, dim, dtype=dtype)
            q[..., 0] = dim ** 0.5 * torch.linspace(12, 22, hq).to(dtype)
            _check_to_rounding(t, q, _run(t, q, 0))


@pytest.mark.parametrize("dim,hq,past,new,room", [
    (64, 4, 700, 1, 0), (64, 8, 300, 4, 0), (64, 2, 300, 70, 1 << 20), (128, 4, 700, 1, 0), (128, 2, 300, 100, 1 << 20), (256, 4, 700, 1, 0),
    (256, 2, 300, 70, 1 << 20),
])
def test_scales_below_zero(built_lib, gpu, dim, hq, past, new, room):
    """Appending writes none, but a number is its code times its block's scale whatever that is."""
    say("scales below zero", dim, hq, past, new, room)
    for dtype, size in ((F16, 1.0), (F16, 100.0), (BF16, 1e9), (BF16, 1e30), (BF16, 1e-30)):
        for every in (1, 2):
            t = Setup(gpu, 1, dim, 64, [past], [new], seed=every, max_len=room or None)
            flat = t.ref.scales.view(-1, 2)
            flat[::every, 1] *= -size
            flat[::every, 0] *= -1
            t.cache.scales.copy_(t.ref.scales)
            q = t.heads_of(hq, dtype, 0.5)
            _check_to_rounding(t, q, _run(t, q, 0))


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("before", [0.5, -0.5, -1e-3, -40.0])
def test_appending_to_a_block_of_a_scale_below_zero(built_lib, gpu, dim, before):
    """Its scale is at least that large, and its earlier tokens stay what they were to half a code."""
    t = Setup(gpu, 2, dim, 16, [5], [4], seed=1)
    p = int(t.table[0, 0])
    t.cache.scales[p] = t.ref.scales[p] = before
    old_k, old_v = t.ref.read(t.table[0], 0, 5)
    k, v = t.heads_of(2, BF16), t.heads_of(2, BF16)
    D.kv_append(t.cache, t.batch, k.to(gpu), v.to(gpu))
    ko, vo = (torch.zeros(9, 2, dim, device=gpu) for _ in range(2))
    D.kv_read(t.cache, t.make_batch([0, 9], [0], 9), ko, vo)
    scales = t.cache.scales[p].cpu()[:, 0]
    for got, old, new, s in ((ko, old_k, k, scales[:, 0]), (vo, old_v, v, scales[:, 1])):
        want = torch.maximum((new.double().abs().amax((0, 2)) / 127).float(), torch.full((2,), abs(before)))
        assert torch.equal(s, want)
        x = torch.cat([old, new.double()])
        assert bool(((got.cpu().double() - x).abs() <= s.double()[None, :, None] / 2 * (1 + 2.0 ** -20) + x.abs() * R.EPS).all())


@pytest.mark.parametrize("dim,hq,past,new,room", [
    (64, 4, 700, 1, 0), (64, 8, 300, 4, 0), (64, 2, 300, 70, 1 << 20), (128, 4, 700, 1, 0), (128, 2, 300, 100, 1 << 20), (256, 4, 700, 1, 0),
    (256, 2, 300, 70, 1 << 20),
])
def test_one_element_of_a_query_far_above_the_others(built_lib, gpu, dim, hq, past, new, room):
    """Where keys have nothing for it the others make the scores."""
    say("large element", dim, hq, past, new, room)
    for dtype, large in ((F16, 60000.0), (BF16, 2.0 ** 30), (BF16, 2.0 ** 60), (BF16, 2.0 ** 120)):
        t = Setup(gpu, 1, dim, 64, [past], [new], seed=5, max_len=room or None)
        t.ref.pages[:, :, :, 0].view(*t.ref.pages.shape[:3], 16, dim)[..., 7] = 0
        t.cache.pages.copy_(t.ref.pages)
        q = t.heads_of(hq, dtype, 0.5)
        q[..., 7] = large
        _check_to_rounding(t, q, _run(t, q, 0))


@pytest.mark.parametrize("dim,hq,past,new,room", [
    (64, 4, 700, 1, 0), (64, 8, 300, 4, 0), (64, 2, 300, 70, 1 << 20), (128, 4, 700, 1, 0), (128, 2, 300, 100, 1 << 20), (256, 4, 700, 1, 0),
    (256, 2, 300, 70, 1 << 20),
])
def test_queries_and_scales_of_keys_at_opposite_ends(built_lib, gpu, dim, hq, past, new, room):
    """Scores of ordinary size from queries at bf16's lower end and keys' scales at fp32's upper one, and the other way round."""
    say("opposite ends", dim, hq, past, new, room)
    for by in (125, 100, -60, -120):
        t = Setup(gpu, 1, dim, 64, [past], [new], seed=9, max_len=room or None)
        t.ref.scales[..., 0] *= 2.0 ** by
        t.cache.scales.copy_(t.ref.scales)
        q = (t.heads_of(hq, torch.float32) * 2.0 ** -by).to(BF16)
        _check_to_rounding(t, q, _run(t, q, 0))
