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
