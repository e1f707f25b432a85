"""A model's forward pass over a cache on the GPU: layers against the oracle on the cache's numbers,
whole models in prompts, chunks and single tokens, and the run that a user makes with them."""
import numpy as np
import pytest
import torch

import kv_ref as R
import oracle as O
from gpu_util import ROW_TOL, TOL, max_row_rel_l2, rel_l2, say, to_np
from mebp_inputs import CONFIGS, MINI, make_inputs
from paper_2510_03425_amd import _lib as L
from paper_2510_03425_amd import device as D

pytestmark = pytest.mark.gpu


def _quantised(monkeypatch, chunks):
    """The oracle's attention on what a cache that was appended to in these chunks holds."""
    from oracle import mebp_oracle as M
    plain = M.attention

    def attention(q, k, v, window):
        kq, vq = k.copy(), v.copy()
        for b in range(k.shape[0]):
            h, d = k.shape[2:]
            n = -(-k.shape[1] // 16)
            c = R.Cache(torch.zeros(n, h, 1, 2, 16 * d, dtype=torch.int8), torch.zeros(n, h, 1, 2))
            row, at = torch.arange(n), 0
            for m in chunks:
                c.append(row, at, torch.from_numpy(k[b, at:at + m]), torch.from_numpy(v[b, at:at + m]))
                at += m
            kq[b], vq[b] = (x.numpy() for x in c.read(row, 0, at))
        return plain(q, kq, vq, window)

    monkeypatch.setattr(M, "attention", attention)


def _hidden(cfg, inp):
    """Every layer's output by the oracle, [layers + 1][B T][d]."""
    x = [O.embed(O.decompress_embedding(cfg, inp), inp.ids, O.embed_scale(cfg)).reshape(cfg.n_tokens, -1)]
    for l in range(cfg.n_layers):
        x.append(O.layer_forward(cfg, l, O.decompress_layer(cfg, inp, l), x[-1]))
    return x


def _i32(gpu, v):
    return torch.tensor(v, dtype=torch.int32, device=gpu)


@pytest.mark.parametrize("chunks", [[160], [100, 1, 1, 7, 51], [1] * 20 + [140]])
@pytest.mark.parametrize("arch", [{}, dict(qkv_bias=True), dict(qk_norm=True, sandwich_norm=True, embed_scale=True)])
def test_model_in_chunks(built_lib, gpu, monkeypatch, chunks, arch):
    """Two sequences of 160 tokens through a local and a global layer, in the same chunks each."""
    say("cached model", chunks[:5], arch)
    cfg = MINI.with_(**arch)
    inp = make_inputs(cfg, seed=5, norm="random")
    _quantised(monkeypatch, chunks)
    ref = _hidden(cfg, inp)[-1].reshape(2, 160, -1)
    dm = D.DeviceModel(inp, device=str(gpu))
    caches, ropes = dm.kv_caches(12, 32), dm.ropes(160)
    table = torch.randperm(12, generator=torch.Generator().manual_seed(2))[:10].view(2, 5).to(torch.int32).to(gpu)
    past = _i32(gpu, [0, 0])
    got, at = torch.empty(2, 160, cfg.hidden, device=gpu), 0
    for m in chunks:
        batch = D.KvBatch(_i32(gpu, [0, m, 2 * m]), past, table, m, 160)
        y = dm.forward_cached(dm.ids[:, at:at + m].reshape(-1).contiguous(), caches, batch, ropes)
        got[:, at:at + m] = y.view(2, m, -1)
        past += m
        at += m
    g = to_np(got)
    assert rel_l2(g, ref) <= TOL
    assert max_row_rel_l2(g.reshape(320, -1), ref.reshape(320, -1)) <= ROW_TOL


def test_layer_is_the_training_layer_but_for_8_bits(built_lib, gpu):
    """A whole prompt against mebp_layer_forward_ckpt: a key or value is off by half a code, 1/254 of its
    block's largest (about 3 of its deviations), an output of attention by less, as it averages values."""
    cfg = CONFIGS["qwen2.5-0.5b"].with_(n_layers=1, vocab=0, batch=2, seq=150)
    inp = make_inputs(cfg, seed=3, n_layers=1)
    dm = D.DeviceModel(inp, device=str(gpu))
    x = torch.randn(300, cfg.hidden, generator=torch.Generator().manual_seed(1)).to(gpu)
    y, z = torch.empty_like(x), torch.empty_like(x)
    dm.layer_forward(0, x, y)
    batch = D.KvBatch(_i32(gpu, [0, 150, 300]), _i32(gpu, [0, 0]), _i32(gpu, [[0, 1, 2], [3, 4, 5]]), 150, 192)
    ws = dm.cached_ws(300, batch)
    dm.layer_forward_cached(0, x, z, dm.kv_caches(6)[0], batch, D.Rope.make(150, 64, cfg.layer_theta(0), device=gpu), ws)
    assert rel_l2(to_np(z - x), to_np(y - x)) <= 0.03


def test_rows_of_no_sequence(built_lib, gpu):
    """They go through the layer with an attention output of 0, whatever the workspace held, and change
    nothing for the others."""
    cfg = MINI.with_(vocab=0)
    inp = make_inputs(cfg, seed=6)
    dm = D.DeviceModel(inp, device=str(gpu))
    x = torch.randn(40, cfg.hidden, generator=torch.Generator().manual_seed(1)).to(gpu)
    rope = D.Rope.make(64, 64, cfg.layer_theta(1), device=gpu)
    outs = []
    for fill, rows in ((0xFF, 40), (0, 40), (0x7B, 30)):
        cache = dm.kv_caches(2, 64)[0]
        batch = D.KvBatch(_i32(gpu, [0, 10, 30]), _i32(gpu, [0, 3]), _i32(gpu, [[0], [1]]), 20, 64)
        ws = dm.cached_ws(rows, batch)
        ws.fill_(fill)
        cache.pages.fill_(1)
        cache.scales.fill_(0.1)
        y = torch.empty_like(x[:rows])
        dm.layer_forward_cached(1, x[:rows].contiguous(), y, cache, batch, rope, ws)
        outs.append(y)
    assert torch.equal(outs[0], outs[1]) and outs[0].isfinite().all()
    assert rel_l2(to_np(outs[2]), to_np(outs[0][:30])) <= 1e-3


def test_rows_around_sequences(built_lib, gpu):
    """Rows before the first sequence and those behind a sequence's max_new have no attention either."""
    cfg = MINI.with_(vocab=0)
    dm = D.DeviceModel(make_inputs(cfg, seed=6), device=str(gpu))
    x = torch.randn(40, cfg.hidden, generator=torch.Generator().manual_seed(2)).to(gpu)
    rope = D.Rope.make(64, 64, cfg.layer_theta(1), device=gpu)
    outs = []
    # the same tokens of two sequences: with rows around them, and those rows behind all
    for fill, start, new in ((0xFF, [3, 17, 40], 9), (0, [3, 17, 40], 9), (0x7B, [0, 9, 18], 9)):
        cache = dm.kv_caches(2, 64)[0]
        batch = D.KvBatch(_i32(gpu, start), _i32(gpu, [0, 3]), _i32(gpu, [[0], [1]]), new, 64)
        order = list(range(40)) if start[0] else [*range(3, 12), *range(17, 26), *range(0, 3), *range(12, 17), *range(26, 40)]
        rows = torch.tensor(order, device=gpu)
        ws = dm.cached_ws(40, batch)
        ws.fill_(fill)
        cache.pages.fill_(1)
        cache.scales.fill_(0.1)
        y = torch.empty_like(x)
        dm.layer_forward_cached(1, x[rows].contiguous(), y, cache, batch, rope, ws)
        back = torch.empty_like(y)
        back[rows] = y
        outs.append(back)
    assert torch.equal(outs[0], outs[1]) and outs[0].isfinite().all()
    assert rel_l2(to_np(outs[2]), to_np(outs[0])) <= 1e-3


def test_guarded_and_captured_steps(built_lib, gpu):
    cfg = MINI
    inp = make_inputs(cfg, seed=7)
    dm = D.DeviceModel(inp, device=str(gpu))
    caches, ropes = dm.kv_caches(4, 64), dm.ropes(128)
    table, past = _i32(gpu, [[2, 0], [1, 3]]), _i32(gpu, [0, 0])
    prompt = D.KvBatch(_i32(gpu, [0, 50, 53]), past, table, 50, 128)
    ids = dm.ids.reshape(-1)[:53].contiguous()
    want = dm.forward_cached(ids, caches, prompt, ropes)
    was = L.mebp_set_workspace_guards(True)
    try:
        assert torch.equal(dm.forward_cached(ids, caches, prompt, ropes), want)
    finally:
        L.mebp_set_workspace_guards(was)
    past.copy_(_i32(gpu, [50, 3]))
    step = D.KvBatch(_i32(gpu, [0, 1, 2]), past, table, 1, 128)
    tok = ids[:2].clone()
    ws = dm.cached_ws(2, step)
    out = torch.empty(2, cfg.hidden, device=gpu)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        dm.forward_cached(tok, caches, step, ropes, ws)
    torch.cuda.current_stream().wait_stream(side)
    twin = [D.KvCache(c.pages.clone(), c.scales.clone()) for c in caches]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out.copy_(dm.forward_cached(tok, caches, step, ropes, ws))
        past += 1
    eager_past = past.clone()
    eager = D.KvBatch(_i32(gpu, [0, 1, 2]), eager_past, table, 1, 128)
    for i in range(5):
        tok.copy_(ids[10 + 2 * i:12 + 2 * i])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dm.forward_cached(tok.clone(), twin, eager, ropes), out)
        eager_past += 1


def test_train_then_answer(built_lib, gpu):
    """Steps on a text, then its continuation token by token from the cache, and a policy-gradient step on
    what was sampled: the run that these operators are for."""
    cfg = MINI.with_(batch=1, seq=64)
    inp = make_inputs(cfg, seed=8)
    dm = D.DeviceModel(inp, device=str(gpu))
    dm.train_step()
    caches, ropes = dm.kv_caches(3, 64), dm.ropes(192)
    table, past = _i32(gpu, [[2, 0, 1]]), _i32(gpu, [0])
    x = dm.forward_cached(dm.ids.reshape(-1), caches, D.KvBatch(_i32(gpu, [0, 64]), past, table, 64, 192), ropes)
    # the prompt's scores from the cache are those of the training forward pass, but for 8 bits
    targets = torch.roll(dm.ids.reshape(-1), -1).contiguous()
    a, b = dm.lm_head_logprobs(x, targets), dm.lm_head_logprobs(dm.ckpt[-1], targets)
    assert rel_l2(to_np(a["logp"]), to_np(b["logp"])) <= TOL
    past += 64
    step = D.KvBatch(_i32(gpu, [0, 1]), past, table, 1, 192)
    tokens, last = [], x[-1:].contiguous()
    for _ in range(20):
        top = dm.lm_head_logprobs(last, top_k=4)
        tokens.append(top["top_ids"][:, 0].clone())
        last = dm.forward_cached(tokens[-1], caches, step, ropes)
        past += 1
    # the same tokens at once behind the prompt, into pages of their own
    again = dm.kv_caches(3, 64)
    zero = _i32(gpu, [0])
    whole = torch.cat([dm.ids.reshape(-1)] + tokens)
    y = dm.forward_cached(whole, again, D.KvBatch(_i32(gpu, [0, 84]), zero, table, 84, 192), ropes)
    assert rel_l2(to_np(y[-1:]), to_np(last)) <= TOL
    z = dm.lm_head_logits(y[63:83].contiguous())
    t = torch.cat(tokens)
    s = D.token_logprobs(z, t)
    d = D.token_logprobs_backward(z, t, s["lse"], s["entropy"], torch.full((20,), 0.05, device=gpu))
    assert d.isfinite().all()
    dx = dm.lm_head_logits_backward(y[63:83].contiguous(), d.to(torch.bfloat16))
    assert dx.isfinite().all() and float(dx.abs().max()) > 0
