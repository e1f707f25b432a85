"""Rotary positions on the GPU against 64 bits: tables, the rotation and its gradient."""
import math

import pytest
import torch

import kv_ref as R
from gpu_util import say
from paper_2510_03425_amd import _lib as L
from paper_2510_03425_amd import device as D

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.mark.parametrize("n_pos,rot,kw", [
    (1, 2, {}), (3, 64, dict(theta=1e6)), (1000, 256, dict(factor=8.0)), (131072, 64, dict(factor=8.0, original=8192)),
    (5000, 34, dict(theta=1e6, factor=4.0, original=1000, low=0.5, high=3.0, gain=1.2)), (65, 1024, {}),
])
def test_positions(built_lib, gpu, n_pos, rot, kw):
    say("rope positions", n_pos, rot, kw)
    got = D.Rope.make(n_pos, rot, device=gpu, **kw).table
    # parameters as the call takes them, in fp32
    kw = {k: (v if k == "original" else float(torch.tensor(v, dtype=F32))) for k, v in dict(dict(theta=1e4), **kw).items()}
    ref = R.table(n_pos, rot, **kw)
    # the frequency's and the angle's own rounding in 64 bits, 4 half steps of the angle, and one to fp32
    bound = ref.abs() * R.EPS + torch.arange(n_pos, dtype=R.F64)[:, None, None] * 4 * 2.0 ** -53 * 1.2 + 2.0 ** -149
    R.check(got, ref, bound, "table")


CASES = [  # tokens, heads, dim, rot
    (1, 14, 64, 64), (1, 1, 2, 2), (7, 3, 64, 32), (33, 5, 128, 128), (5, 2, 256, 256), (130, 12, 128, 96), (3, 4, 80, 80), (9, 7, 72, 48),
    (4, 2, 40, 16), (17, 3, 50, 26), (2, 9, 64, 6), (257, 1, 96, 96), (11, 2, 1024, 1024),
    (2051, 13, 256, 256), (9001, 5, 128, 64),  # (several heads a thread; in fp32 and 16 bits on either side of the L2s' size)
    (30001, 5, 128, 64),
]


def _heads(n, h, d, dtype, gap, gen, gpu):
    """[n][h][d] in rows `gap` elements longer than the heads, which hold 7."""
    x = torch.randn(n, h, d, generator=gen).to(dtype)
    buf = torch.full((n, h * d + gap), 7.0, dtype=dtype, device=gpu)
    buf[:, :h * d] = x.reshape(n, -1).to(gpu)
    return x, buf, buf[:, :h * d].view(n, h, d)


@pytest.mark.parametrize("n,h,d,rot", CASES)
@pytest.mark.parametrize("dtype,gap,inter,back", [(F32, 0, False, False), (F16, 8, True, False), (BF16, 0, False, True), (F32, 3, True, True),
                                                  (BF16, 1, False, False)])
def test_apply(built_lib, gpu, n, h, d, rot, dtype, gap, inter, back):
    say("rope apply", n, h, d, rot, dtype, gap, inter, back)
    g = torch.Generator().manual_seed(n * 7 + d)
    tab = R.table(300, rot, 1e4, 1.1).float()
    rope = D.Rope(tab.to(gpu), d, inter)
    x, buf, xd = _heads(n, h, d, dtype, gap, g, gpu)
    pos = torch.randint(0, 300, (n,), generator=g, dtype=torch.int32)
    ref, bound = R.turn(x, tab, pos, inter, back), R.turn_bound(x, tab, pos, inter, dtype)
    out = torch.full((n, h * d + gap), 5.0, dtype=dtype, device=gpu)
    view = out[:, :h * d].view(n, h, d)
    got = D.rope_apply(rope, xd, pos.to(gpu), view, backward=back)
    assert got is view
    R.check(got, ref, bound, "out of place")
    assert bool((out[:, h * d:] == 5.0).all())
    assert torch.equal(got[..., rot:], xd[..., rot:])
    again = D.rope_apply(rope, xd, pos.to(gpu), backward=back)
    assert torch.equal(again, got)
    D.rope_apply(rope, xd, pos.to(gpu), xd, backward=back)
    assert torch.equal(xd, got) and bool((buf[:, h * d:] == 7.0).all())


def test_heads_outside_tokens(built_lib, gpu):
    """[heads][tokens][dim] in memory, and a tensor that is the same for every token."""
    g = torch.Generator().manual_seed(4)
    tab = R.table(64, 64, 1e4).float()
    rope = D.Rope(tab.to(gpu), 64)
    x = torch.randn(5, 19, 64, generator=g)
    pos = torch.arange(19, dtype=torch.int32)
    out = torch.empty(5, 19, 64, device=gpu).transpose(0, 1)
    D.rope_apply(rope, x.to(gpu).transpose(0, 1), pos.to(gpu), out)
    R.check(out, R.turn(x.transpose(0, 1), tab, pos), R.turn_bound(x.transpose(0, 1), tab, pos, False, F32), "transposed")
    same = x[:, :1].transpose(0, 1).expand(19, 5, 64)
    got = D.rope_apply(rope, same.to(gpu)[:1].expand(19, 5, 64), pos.to(gpu))
    R.check(got, R.turn(same, tab, pos), R.turn_bound(same, tab, pos, False, F32), "broadcast")


def test_special_values_and_positions(built_lib, gpu):
    tab = R.table(10, 64, 1e4).float()
    rope = D.Rope(tab.to(gpu), 96)
    x = torch.randn(6, 2, 96, generator=torch.Generator().manual_seed(2))
    x[0, 0, 3], x[1, 1, 90], x[2, 0, 40] = math.nan, math.inf, -math.inf
    pos = torch.tensor([1, 2, 3, 10, -1, 2 ** 31 - 1], dtype=torch.int32)
    got = D.rope_apply(rope, x.to(gpu), pos.to(gpu)).cpu()
    assert torch.equal(got[1:, :, 64:], x[1:, :, 64:])  # copied elements whatever the position
    assert got[3:, :, :64].isnan().all() and not got[3:, :, 64:].isnan().any()
    bad = got[0, 0].isnan().nonzero()[:, 0].tolist()
    assert bad == [3, 35]
    assert not got[2, 0, [8, 40]].isfinite().any() and got[2, 0, :8].isfinite().all()


def test_gradient_by_differences(built_lib, gpu):
    g = torch.Generator().manual_seed(8)
    rope = D.Rope.make(100, 48, theta=1e4, interleaved=True, gain=1.3, device=gpu)
    x, c, e = (torch.randn(4, 3, 64, generator=g).to(gpu) for _ in range(3))
    pos = torch.tensor([0, 5, 99, 41], dtype=torch.int32, device=gpu)
    # the map is linear: <c, f(e)> = <f^T(c), e> to rounding (768 products of numbers of about 1)
    left = (c.double() * D.rope_apply(rope, e, pos).double()).sum()
    right = (D.rope_apply(rope, c, pos, backward=True).double() * e.double()).sum()
    assert abs(float(left - right)) < 768 * 8 * R.EPS * 4


def test_stream_and_graph(built_lib, gpu):
    g = torch.Generator().manual_seed(9)
    rope = D.Rope.make(4096, 128, device=gpu)
    x = torch.randn(100, 6, 128, generator=g).to(gpu).half()
    pos = torch.arange(100, dtype=torch.int32, device=gpu)
    out = torch.zeros_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        D.rope_apply(rope, x, pos, out)
    side.synchronize()
    want = D.rope_apply(rope, x, pos)
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        D.rope_apply(rope, x, pos, out)
    for shift in (0, 7, 3000):
        pos.copy_(torch.arange(100, dtype=torch.int32, device=gpu) + shift)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, D.rope_apply(rope, x, pos))


def test_empty_and_refused(built_lib, gpu):
    rope = D.Rope.make(8, 64, device=gpu)
    x = torch.zeros(0, 2, 64, device=gpu)
    assert D.rope_apply(rope, x, torch.zeros(0, dtype=torch.int32, device=gpu)).shape == (0, 2, 64)
    x = torch.zeros(3, 2, 64, device=gpu)
    pos = torch.zeros(3, dtype=torch.int32, device=gpu)
    for bad in (pos.long(), pos[:2], pos.cpu()):
        with pytest.raises(ValueError):
            D.rope_apply(rope, x, bad)
    with pytest.raises(L.MebpError):
        D.rope_apply(rope, x, pos, x[:, :, :].flip(0)[:2])
    with pytest.raises(L.MebpError):
        D.rope_apply(rope, torch.zeros(3, 2, 32, device=gpu), pos)
    with pytest.raises(ValueError):
        D.rope_apply(rope, torch.zeros(3, 64, 2, device=gpu).transpose(1, 2), pos)
