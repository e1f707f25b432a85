"""Distillation steps whose head lies in the step's own workspace, where the cross-entropy has its
logits or its copy of the weights, or behind it: the same loss and gradients as the single calls."""
import numpy as np
import pytest
import torch

from gpu_util import rel_l2, say
from mebp_inputs import MINI, make_inputs
from paper_2510_03425_amd import _lib as L
from paper_2510_03425_amd.device import DeviceModel

pytestmark = pytest.mark.gpu

SHAPES = {  # placement: hidden, B, T
    "logits": (128, 4, 1250), "weights": (1024, 1, 256), "behind": (128, 1, 100),
}


def _model(where, gpu):
    hidden, B, T = SHAPES[where]
    cfg = MINI.with_(name=where, n_layers=3, hidden=hidden, ffn=352, vocab=50304, batch=B, seq=T)
    inp = make_inputs(cfg, seed=7, norm="random")
    inp.norm_final = (np.asarray(inp.norm_final) * (3 / (0.02 * hidden**0.5))).astype(np.float32)
    dm = DeviceModel(inp, device=str(gpu))
    g = torch.Generator().manual_seed(5)
    n = dm.N
    ids = torch.randint(0, cfg.vocab, (n, 4), generator=g, dtype=torch.int32).to(gpu)
    tl = (torch.randn((n, 4), generator=g) * 2).to(gpu)
    t = torch.randint(0, cfg.vocab, (n,), generator=g, dtype=torch.int32).to(gpu)
    return dm, (ids, tl, 2.0, 0.6, t, torch.full((n,), 1.0 / n, device=gpu))


@pytest.mark.parametrize("where", list(SHAPES))
def test_step_is_its_single_calls(built_lib, gpu, where):
    dm, args = _model(where, gpu)
    need = L.mebp_distill_step_workspace_bytes(dm.ccfg, dm.B, dm.T)
    say("placement", where, need, dm.ws_bytes)
    assert (need == dm.ws_bytes) == (where != "behind")
    rl, dx0 = torch.empty(dm.N, device=gpu), torch.empty((dm.N, dm.cfg.hidden), device=gpu)
    step = lambda: dm.train_step_distill(*args, rl, dx0)  # noqa: E731
    step()
    assert (dm.distill_ws is None) == (where != "behind")
    first = [x.clone() for x in (dm.loss, rl, dx0, dm.grad_probe())]
    # the single calls, each with a workspace of its own
    x = [torch.empty_like(dx0) for _ in range(dm.L + 1)]
    dm.embed(x[0])
    for l in range(dm.L):
        dm.layer_forward(l, x[l], x[l + 1])
    g, h, one = torch.empty_like(dx0), torch.empty_like(dx0), torch.empty(dm.N, device=gpu)
    dm.lm_head_distill(x[-1], g, *args, one)
    assert torch.allclose(first[0], dm.loss, rtol=1e-4, atol=0) and rel_l2(first[1].cpu(), one.cpu()) <= 1e-4
    for l in reversed(range(dm.L)):
        dm.layer_backward(l, x[l], g, h)
        g, h = h, g
    # (16-bit intermediates, which sums in another order may round the other way)
    assert rel_l2(first[2].cpu(), g.cpu()) <= 5e-3 and rel_l2(first[3].cpu(), dm.grad_probe().cpu()) <= 5e-3
    # next-token steps in the same workspace before and after, guards around the head's slots, a captured step
    dm.train_step(dx0)
    step()
    assert all(torch.equal(a, b) for a, b in zip(first, (dm.loss, rl, dx0, dm.grad_probe())))
    prev = L.mebp_set_workspace_guards(True)
    try:
        step()
    finally:
        L.mebp_set_workspace_guards(prev)
    assert all(torch.equal(a, b) for a, b in zip(first, (dm.loss, rl, dx0, dm.grad_probe())))
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        step()
    for rep in range(3):
        dm.train_step(dx0)
        dm.loss.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, (dm.loss, rl, dx0, dm.grad_probe()))), rep
