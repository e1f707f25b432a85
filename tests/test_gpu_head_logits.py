"""The LM head's logits and the operators on them on the GPU, against the oracle's blocks and 64-bit
losses: logits and their gradient, scores, distillation, and whole distillation steps from a
teacher's recorded alternatives."""
import numpy as np
import pytest
import torch

import logits_ref as R
import oracle as O
from gpu_util import TOL, max_row_rel_l2, rel_l2, say, ROW_TOL
from mebp_inputs import MINI, PROJ, make_inputs
from paper_2510_03425_amd import _lib as L
from paper_2510_03425_amd import device as D
from paper_2510_03425_amd.device import DeviceModel

pytestmark = pytest.mark.gpu


def _inputs(cfg, seed=6):
    inp = make_inputs(cfg, seed=seed, norm="random")
    # logits with a standard deviation of about 4: confident rows beside flat ones
    inp.norm_final = (np.asarray(inp.norm_final) * (4 / (0.02 * cfg.hidden**0.5))).astype(np.float32)
    return inp


class _Ref:
    """z = rmsnorm(x) E^T in float64, with autograd."""

    def __init__(self, inp, device="cpu"):
        cfg = inp.cfg
        self.E = torch.from_numpy(O.dequant(*inp.emb, cfg.hidden, 32).astype(np.float64)).to(device)
        self.w = torch.from_numpy(np.asarray(inp.norm_final, np.float64)).to(device)
        self.eps = cfg.rms_eps

    def hf(self, x):
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + self.eps) * self.w

    def logits(self, x):
        return self.hf(x) @ self.E.t()


def _teacher(rows, k, vocab, seed):
    g = torch.Generator().manual_seed(seed)
    ids = torch.stack([torch.randperm(vocab, generator=g)[:k] for _ in range(rows)]).to(torch.int32)
    return ids, torch.randn((rows, k), generator=g) * 2 + 5, torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32)


def _distill_loss(z, ids, tl, t, w, tau, alpha):
    """Sum of the rows' losses of double logits (every entry present)."""
    p = torch.softmax(tl.to(z) / tau, 1)
    kl = (p * (torch.log(p) - torch.log_softmax(z / tau, 1).gather(1, ids.long()))).sum(1)
    ce = -torch.log_softmax(z, 1).gather(1, t.long()[:, None])[:, 0]
    return (w.to(z) * (alpha * tau * tau * kl + (1 - alpha) * ce)).sum()


@pytest.mark.parametrize("rows", [1, 3, 64, 257])
def test_logits_and_their_gradient(built_lib, gpu, rows):
    inp = _inputs(MINI)
    dm, ref = DeviceModel(inp, device=str(gpu)), _Ref(inp)
    V, d = MINI.vocab, MINI.hidden
    x = torch.randn((rows, d), generator=torch.Generator().manual_seed(rows))
    say("head logits", rows)
    xr = x.double().requires_grad_()
    zr = ref.logits(xr)
    # both operands in fp16 (half a step each, and their product's), the sum in fp32
    mag = ref.hf(x.double()).abs() @ ref.E.abs().t()
    bound = (2 * 2.0 ** -11 + 2.0 ** -22 + (d + 8) * 2.0 ** -24) * mag
    for dtype in (torch.float32, torch.float16):
        z = dm.lm_head_logits(x.to(gpu), dtype)
        R.close(z, zr.detach(), bound + R.HALF_STEP[dtype] * (zr.detach().abs() + bound) + R.TINY[dtype], "logits")
    dz = (torch.randn((rows, V), generator=torch.Generator().manual_seed(1)) / rows).bfloat16()
    dx = dm.lm_head_logits_backward(x.to(gpu), dz.to(gpu))
    want = torch.autograd.grad(zr, xr, dz.double())[0]
    assert rel_l2(dx.cpu(), want) <= TOL and max_row_rel_l2(dx.cpu(), want) <= ROW_TOL


def test_logits_with_a_pitch_leave_the_columns_behind(built_lib, gpu):
    inp = _inputs(MINI)
    dm = DeviceModel(inp, device=str(gpu))
    x = torch.randn((70, MINI.hidden), generator=torch.Generator().manual_seed(3)).to(gpu)
    want = dm.lm_head_logits(x)
    buf = torch.full((70, MINI.vocab + 24), 7.0, device=gpu)
    ws, nb = dm._head_ws(70)
    L.mebp_lm_head_logits(dm.ccfg, dm.emb, D.ptr(dm.norm_final), D.ptr(x), 70, D.logits_struct(buf[:, :MINI.vocab]),
                          D.ptr(ws), nb, D.stream_handle())
    assert torch.equal(buf[:, :MINI.vocab], want) and bool((buf[:, MINI.vocab:] == 7.0).all())


def test_scores_of_the_head_are_those_of_its_logits(built_lib, gpu):
    inp = _inputs(MINI)
    dm = DeviceModel(inp, device=str(gpu))
    for rows, k, tau in ((1, 64, 1.0), (33, 5, 0.7), (300, 20, 1.0)):
        x = torch.randn((rows, MINI.hidden), generator=torch.Generator().manual_seed(rows)).to(gpu)
        t = torch.randint(-1, MINI.vocab, (rows,), generator=torch.Generator().manual_seed(2), dtype=torch.int32).to(gpu)
        want = D.token_logprobs(dm.lm_head_logits(x), t, k, tau)
        got = dm.lm_head_logprobs(x, t, k, tau)
        for name in want:
            assert torch.equal(got[name], want[name]), name


@pytest.mark.parametrize("tau,alpha", [(1.0, 1.0), (2.0, 0.7), (1.5, 0.4), (1.0, 0.0)])
def test_distillation_of_the_head(built_lib, gpu, tau, alpha):
    inp = _inputs(MINI)
    dm, ref = DeviceModel(inp, device=str(gpu)), _Ref(inp)
    rows = 321
    x = torch.randn((rows, MINI.hidden), generator=torch.Generator().manual_seed(4))
    ids, tl, t = _teacher(rows, 12, MINI.vocab, 5)
    w = (torch.rand(rows, generator=torch.Generator().manual_seed(2)) + 0.5) / rows
    w[::7] = 0.0
    dx, rl = torch.full_like(x, float("nan"), device=gpu), torch.empty(rows, device=gpu)
    say("head distillation", tau, alpha)
    dm.lm_head_distill(x.to(gpu), dx, ids.to(gpu), tl.to(gpu), tau, alpha, t.to(gpu), w.to(gpu), rl)
    xr = x.double().requires_grad_()
    loss = _distill_loss(ref.logits(xr), ids, tl, t, w, tau, alpha)
    want = torch.autograd.grad(loss, xr)[0]
    say("loss", dm.loss.item(), loss.item(), "dx", rel_l2(dx.cpu(), want))
    assert abs(dm.loss.item() - loss.item()) <= 1e-3 * abs(loss.item())
    assert abs(rl.double().sum().item() - dm.loss.item()) <= 1e-5 * abs(dm.loss.item())
    assert rel_l2(dx.cpu(), want) <= TOL and max_row_rel_l2(dx.cpu(), want) <= ROW_TOL
    assert bool((dx[::7] == 0).all()) and bool((rl[::7] == 0).all())


def test_hard_labels_alone_are_the_next_token_loss(built_lib, gpu):
    inp = _inputs(MINI)
    dm = DeviceModel(inp, device=str(gpu))
    B, T, N = MINI.batch, MINI.seq, MINI.n_tokens
    x = torch.randn((N, MINI.hidden), generator=torch.Generator().manual_seed(8)).to(gpu)
    dx0, dx1 = torch.empty_like(x), torch.empty_like(x)
    dm.lm_head(x, dx0)
    loss0 = dm.loss.item()
    ids = torch.from_numpy(np.asarray(inp.ids)).view(B, T)
    t = torch.full((B, T), -1, dtype=torch.int32)
    t[:, :-1] = ids[:, 1:]
    none = torch.full((N, 1), -1, dtype=torch.int32)
    dm.lm_head_distill(x, dx1, none.to(gpu), torch.zeros((N, 1), device=gpu), 1.0, 0.0, t.view(-1).to(gpu),
                       torch.full((N,), 1.0 / (B * (T - 1)), device=gpu))
    assert abs(dm.loss.item() - loss0) <= 2e-3 * abs(loss0)
    assert rel_l2(dx1.cpu(), dx0.cpu()) <= 2 * TOL


@pytest.mark.parametrize("vocab,rows,block", [(50304, 1700, 1536), (70016, 1100, 1024)])
def test_more_rows_than_a_block_holds(built_lib, gpu, vocab, rows, block):
    """A block of `block` rows and the last one of some (of the larger vocabulary: by parts of
    rows), on guarded workspaces."""
    hidden = 128
    cfg = MINI.with_(name="blocks", n_layers=1, hidden=hidden, n_heads=1, n_kv_heads=1, head_dim=128, ffn=192, vocab=vocab,
                     batch=1, seq=64)
    inp = _inputs(cfg)
    prev = L.mebp_set_workspace_guards(True)
    try:
        dm, ref = DeviceModel(inp, device=str(gpu)), _Ref(inp, gpu)
        x = torch.randn((rows, hidden), generator=torch.Generator().manual_seed(4)).to(gpu)
        ids, tl, t = (a.to(gpu) for a in _teacher(rows, 16, vocab, 5))
        w = torch.full((rows,), 1.0 / rows, device=gpu)
        say("head blocks", rows, vocab)
        dx = torch.full_like(x, float("nan"))
        dm.lm_head_distill(x, dx, ids, tl, 2.0, 0.6, t, w)
        s = dm.lm_head_logprobs(x, t, 8)
        z = dm.lm_head_logits(x)
        back = dm.lm_head_logits_backward(x, z.bfloat16())
    finally:
        L.mebp_set_workspace_guards(prev)
    loss, want = 0.0, torch.empty_like(x, dtype=torch.float64)
    for r in range(0, rows, 170):
        q = slice(r, r + 170)
        xr = x[q].double().requires_grad_()
        zr = ref.logits(xr)
        part = _distill_loss(zr, ids[q], tl[q], t[q], w[q], 2.0, 0.6)
        want[q] = torch.autograd.grad(part, xr)[0]
        loss += part.item()
        lp = torch.log_softmax(z[q].double(), 1)  # (of the head's own logits: their fp16 operands left out)
        assert torch.allclose(s["logp"][q].double(), lp.gather(1, t[q].long()[:, None])[:, 0], rtol=0, atol=1e-4)
        assert torch.equal(s["top_ids"][q].long(), torch.topk(z[q], 8, dim=1)[1])
    assert abs(dm.loss.item() - loss) <= 1e-3 * abs(loss)
    assert rel_l2(dx.cpu(), want.cpu()) <= TOL
    # z^T z x: each block with its own rows
    for q in (slice(0, 40), slice(block - 6, block + 9), slice(rows - 40, rows)):
        xr = x[q].double().requires_grad_()
        g = torch.autograd.grad(ref.logits(xr), xr, z[q].bfloat16().double())[0]
        assert rel_l2(back[q].cpu(), g.cpu()) <= TOL


def _teacher_pass(cfg, gpu, k):
    """A teacher's hidden states of the batch and its top k alternatives at each position."""
    inp = _inputs(cfg, seed=31)
    tm = DeviceModel(inp, device=str(gpu))
    tm.ids.copy_(torch.from_numpy(np.asarray(make_inputs(cfg, seed=6).ids)))
    x = torch.empty((tm.N, cfg.hidden), device=gpu)
    y = torch.empty_like(x)
    tm.embed(x)
    for l in range(tm.L):
        tm.layer_forward(l, x, y)
        x, y = y, x
    s = tm.lm_head_logprobs(x, None, k)
    return s["top_ids"], s["top_logp"]


@pytest.mark.parametrize("cfg,tau,alpha", [
    (MINI, 2.0, 0.7), (MINI.with_(name="mini_arch", qkv_bias=True, qk_norm=True, sandwich_norm=True, embed_scale=True), 1.0, 1.0),
    (MINI.with_(name="one_token", seq=1, batch=3), 1.0, 1.0)])
def test_distillation_step_from_a_recorded_teacher(built_lib, gpu, cfg, tau, alpha):
    ids, tl = _teacher_pass(cfg, gpu, 8)
    inp = _inputs(cfg)
    dm = DeviceModel(inp, device=str(gpu))
    N = dm.N
    t = torch.zeros((cfg.batch, cfg.seq), dtype=torch.int32)
    t[:, :-1] = torch.from_numpy(np.asarray(inp.ids)).view(cfg.batch, cfg.seq)[:, 1:]
    t = t.view(-1)
    w = torch.full((N,), 1.0 / N)
    dx0, rl = torch.empty((N, cfg.hidden), device=gpu), torch.empty(N, device=gpu)
    say("distillation step", cfg.name)
    w_gpu, tg = w.to(gpu), t.to(gpu)
    step = lambda: dm.train_step_distill(ids, tl, tau, alpha, tg, w_gpu, rl, dx0)  # noqa: E731
    step()
    torch.cuda.synchronize()
    # the oracle's layers around the 64-bit loss
    E = O.decompress_embedding(cfg, inp)
    ck = [O.embed(E, inp.ids, O.embed_scale(cfg))]
    for l in range(cfg.n_layers):
        ck.append(O.layer_forward(cfg, l, O.decompress_layer(cfg, inp, l), ck[l]))
    xr = torch.from_numpy(ck[-1]).requires_grad_()
    loss = _distill_loss(_Ref(inp).logits(xr), ids.cpu(), tl.cpu(), t, w, tau, alpha)
    g = torch.autograd.grad(loss, xr)[0].numpy()
    errs = {}
    for l in reversed(range(cfg.n_layers)):
        g, grads = O.layer_backward(cfg, l, O.decompress_layer(cfg, inp, l), ck[l], g)
        for p, (dA, dB) in grads.items():
            if np.linalg.norm(dA) > 0:
                errs[f"dA{l}{p}"] = rel_l2(dm.dA[l][p].cpu(), dA)
            if np.linalg.norm(dB) > 0:
                errs[f"dB{l}{p}"] = rel_l2(dm.dB[l][p].cpu(), dB)
    errs["dx0"] = rel_l2(dx0.cpu(), g)
    say("loss", dm.loss.item(), loss.item(), "worst", max(errs.values()))
    assert abs(dm.loss.item() - loss.item()) <= 2e-3 * abs(loss.item())
    for k, e in errs.items():
        if cfg.seq == 1 and k[-1] in "qk":
            continue  # one key: the softmax is 1 and q and k have no gradient but rounding
        assert e <= TOL, (k, e)
    # the same bits again, guarded, and from a captured graph
    first = [x.clone() for x in (dm.loss, dx0, rl, dm.grad_probe())]
    prev = L.mebp_set_workspace_guards(True)
    try:
        dm.distill_ws = None
        step()
    finally:
        L.mebp_set_workspace_guards(prev)
    assert all(torch.equal(a, b) for a, b in zip(first, (dm.loss, dx0, rl, dm.grad_probe())))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for rep in range(3):
        dx0.zero_()
        dm.loss.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, (dm.loss, dx0, rl, dm.grad_probe()))), rep
        dm.lm_head_logprobs(dm.ckpt[-1], tg, 3)  # eager work in between


def test_adapters_gradient_by_differences(built_lib, gpu):
    """The step's loss along one adapter's gradient: a central difference of h = 2^-6 along the
    normalised direction against its norm. The loss is fp32 with fp16 operands (2^-11 relative, mostly
    alike on both sides) and h^2 times a third derivative of order one: 5 %."""
    cfg = MINI
    ids, tl = _teacher_pass(cfg, gpu, 8)
    dm = DeviceModel(_inputs(cfg), device=str(gpu))
    w = torch.full((dm.N,), 1.0 / dm.N, device=gpu)
    step = lambda: dm.train_step_distill(ids, tl, 2.0, 1.0, None, w)  # noqa: E731
    step()
    i = PROJ.index("down")
    g = dm.dB[1]["down"].clone()
    B = next(t for t in dm.keep if t.data_ptr() == dm.lora[1].B[i])
    n = float(g.norm())
    at = {}
    for sign in (1, -1):
        B += sign * 2.0 ** -6 / n * g
        step()
        at[sign] = float(dm.loss)
        B -= sign * 2.0 ** -6 / n * g
    diff = (at[1] - at[-1]) / 2 ** -5
    say("directional derivative", diff, "gradient's norm", n)
    assert abs(diff - n) <= 0.05 * n


def test_no_rows(built_lib, gpu):
    dm = DeviceModel(_inputs(MINI), device=str(gpu))
    x = torch.empty((0, MINI.hidden), device=gpu)
    assert dm.lm_head_logits(x).shape == (0, MINI.vocab)
    assert dm.lm_head_logprobs(x, None, 3)["top_ids"].shape == (0, 3)
