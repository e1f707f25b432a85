"""Host-only checks of the operators on logits: what they refuse before touching the GPU, and the
64-bit reference of their tests against differences."""
import ctypes as C
import math

import pytest
import torch

import logits_ref as R
from mebp_inputs import CONFIGS, MINI
from paper_2510_03425_amd import _lib as L
from paper_2510_03425_amd import device as D
from paper_2510_03425_amd.device import make_config

Z, T, OUT, DZ, WS = 0x1000000, 0x2000000, 0x3000000, 0x8000000, 0x10000000
BIG = 1 << 40


def _z(**kw):
    a = dict(data=Z, ld=1000, rows=4, vocab=1000, dtype=L.MEBP_F32)
    a.update(kw)
    return L.MebpLogits(**a)


def _scores(z=None, targets=T, tau=1.0, top_k=5, ws=WS, nb=BIG, **out):
    o = dict(logp=OUT, lse=OUT + 0x100, entropy=OUT + 0x200, top_ids=OUT + 0x300, top_logp=OUT + 0x400)
    o.update(out)
    return L.mebp_token_logprobs(z or _z(), targets, tau, top_k, L.MebpTokenScores(**o), ws, nb, 0, check=False)


def _grad(z=None, dz=None, targets=T, tau=1.0, lse=OUT, entropy=OUT, d_logp=OUT, d_entropy=OUT):
    return L.mebp_token_logprobs_backward(z or _z(), targets, tau, lse, entropy, d_logp, d_entropy,
                                          dz or _z(data=DZ), 0, check=False)


def _distill(z=None, dz=None, loss=OUT, ws=WS, nb=BIG, **kw):
    d = dict(ids=T, logits=T, targets=T, row_weight=T, k=8, temperature=2.0, alpha=0.5)
    d.update(kw)
    return L.mebp_distill_topk(z or _z(), L.MebpDistill(**d), loss, dz, ws, nb, 0, check=False)


@pytest.mark.parametrize("call", [_scores, _grad, _distill])
@pytest.mark.parametrize("bad,code", [
    (dict(data=0), L.MEBP_EINVAL), (dict(data=Z + 2), L.MEBP_EINVAL), (dict(ld=999), L.MEBP_EINVAL),
    (dict(rows=-1), L.MEBP_EINVAL), (dict(vocab=0), L.MEBP_EINVAL), (dict(dtype=3), L.MEBP_EINVAL),
    (dict(dtype=-1), L.MEBP_EINVAL), (dict(rows=(1 << 22) + 1), L.MEBP_EUNSUPPORTED),
    (dict(vocab=(1 << 30) + 1, ld=1 << 31), L.MEBP_EUNSUPPORTED), (dict(ld=(1 << 32) + 1), L.MEBP_EUNSUPPORTED),
])
def test_logits_refused(built_lib, call, bad, code):
    assert call(z=_z(**bad)) == code and L.mebp_last_error()


@pytest.mark.parametrize("call", [_scores, _grad, _distill])
@pytest.mark.parametrize("tau", [0.0, -1.0, math.nan, math.inf, 1e-7, 1e7])
def test_temperature_refused(built_lib, call, tau):
    r = call(temperature=tau) if call is _distill else call(tau=tau)
    assert r == L.MEBP_EINVAL and "temperature" in L.mebp_last_error()


def test_scores_refused(built_lib):
    assert _scores(top_k=65) == L.MEBP_EUNSUPPORTED and _scores(top_k=-1) == L.MEBP_EUNSUPPORTED
    assert _scores(targets=0) == L.MEBP_EINVAL  # logp without targets
    assert _scores(top_k=0) == L.MEBP_EINVAL    # alternatives' outputs without any
    assert _scores(targets=T + 1) == L.MEBP_EINVAL and _scores(lse=OUT + 2) == L.MEBP_EINVAL
    assert _scores(logp=0, lse=0, entropy=0, top_ids=0, top_logp=0) == L.MEBP_EINVAL
    assert _scores(ws=0) == L.MEBP_EINVAL and _scores(ws=WS + 16) == L.MEBP_EINVAL
    need = L.mebp_logits_workspace_bytes(4, 100000, 64)
    assert _scores(z=_z(vocab=100000, ld=100000), top_k=64, nb=need - 1) == L.MEBP_EWORKSPACE
    assert L.mebp_token_logprobs(_z(), T, 1.0, 0, None, WS, BIG, 0, check=False) == L.MEBP_EINVAL
    assert L.mebp_token_logprobs(None, T, 1.0, 0, L.MebpTokenScores(lse=OUT), WS, BIG, 0, check=False) == L.MEBP_EINVAL


def test_grad_refused(built_lib):
    assert _grad(lse=0) == L.MEBP_EINVAL and _grad(d_logp=0, d_entropy=0) == L.MEBP_EINVAL
    assert _grad(targets=0) == L.MEBP_EINVAL and _grad(entropy=0) == L.MEBP_EINVAL
    assert _grad(d_entropy=OUT + 1) == L.MEBP_EINVAL
    assert _grad(dz=_z(data=DZ, rows=3)) == L.MEBP_EINVAL and _grad(dz=_z(data=DZ, vocab=999)) == L.MEBP_EINVAL
    assert _grad(dz=_z(data=DZ, ld=900)) == L.MEBP_EINVAL


@pytest.mark.parametrize("dz", [dict(data=Z + 4), dict(data=Z, ld=1004), dict(data=Z, dtype=L.MEBP_BF16),
                                dict(data=Z + 15996), dict(data=Z - 15996)])
def test_overlapping_gradients_refused(built_lib, dz):
    for r in (_grad(dz=_z(**dz)), _distill(dz=_z(**dz))):
        assert r == L.MEBP_EINVAL and "overlap" in L.mebp_last_error()


def test_distill_refused(built_lib):
    assert _distill(k=0) == L.MEBP_EUNSUPPORTED and _distill(k=65) == L.MEBP_EUNSUPPORTED
    assert _distill(alpha=-0.1) == L.MEBP_EINVAL and _distill(alpha=1.1) == L.MEBP_EINVAL
    assert _distill(alpha=math.nan) == L.MEBP_EINVAL
    assert _distill(ids=0) == L.MEBP_EINVAL and _distill(logits=0) == L.MEBP_EINVAL
    assert _distill(targets=0) == L.MEBP_EINVAL  # alpha < 1
    assert _distill(loss=0) == L.MEBP_EINVAL and _distill(row_weight=T + 2) == L.MEBP_EINVAL
    assert _distill(ws=WS + 1) == L.MEBP_EINVAL and _distill(nb=0) == L.MEBP_EWORKSPACE
    assert L.mebp_distill_topk(_z(), None, OUT, None, WS, BIG, 0, check=False) == L.MEBP_EINVAL


def test_no_rows_enqueue_nothing(built_lib):
    z = _z(rows=0, data=0)
    out = L.MebpTokenScores()
    assert L.mebp_token_logprobs(z, 0, 1.0, 5, out, WS, BIG, 0, check=False) == L.MEBP_OK
    assert _grad(z=z, dz=z, targets=0, lse=0, entropy=0, d_logp=0, d_entropy=0) == L.MEBP_OK
    assert _distill(z=z, dz=z, ids=0, logits=0, targets=0, row_weight=0, loss=0) == L.MEBP_OK


def test_workspace_sizes(built_lib):
    f = L.mebp_logits_workspace_bytes
    assert f(-1, 10) == 0 and f(1, 0) == 0 and f(1, 10, 65) == 0 and f((1 << 22) + 1, 10) == 0
    for rows in (1, 3, 100, 255, 1000, 1 << 22):
        for vocab in (1, 1000, 151936, 262144):
            assert 256 <= f(rows, vocab, 0) <= f(rows, vocab, 64) <= 4 << 20, (rows, vocab)
    prev = L.mebp_set_workspace_guards(True)
    try:
        assert f(1, 1000, 5) >= 3 * 256
        guarded = f(1, 262144, 64)
    finally:
        L.mebp_set_workspace_guards(prev)
    assert guarded > f(1, 262144, 64)


def test_struct_sizes(built_lib):
    assert C.sizeof(L.MebpLogits) == 32 and C.sizeof(L.MebpTokenScores) == 40 and C.sizeof(L.MebpDistill) == 48


def test_tensors_refused():
    z = torch.zeros(4, 10)
    with pytest.raises(ValueError, match="GPU"):
        D.token_logprobs(z)
    for bad in (torch.zeros(4, 10, dtype=torch.float64), torch.zeros(10), torch.zeros(10, 4).t()):
        with pytest.raises(ValueError, match="matrix"):
            D.logits_struct(bad)
    like = torch.zeros(1)
    for bad in (torch.zeros(4, dtype=torch.int64), torch.zeros(5, dtype=torch.int32), torch.zeros(8, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError, match="targets"):
            D._operand(bad, torch.int32, (4,), like, "targets")


def test_reference_gradients_against_differences():
    """Central differences in 64 bits of the reference's own losses."""
    g = torch.Generator().manual_seed(0)
    z = torch.randn((5, 23), generator=g, dtype=torch.float64) * 2
    z[1, 5:] = -math.inf
    ids = torch.randint(0, 5, (5, 4), generator=g, dtype=torch.int32)
    tl = torch.randn((5, 4), generator=g)
    t = torch.tensor([1, 4, -1, 3, 0], dtype=torch.int32)
    w = torch.rand(5, generator=g)
    v = torch.randn(z.shape, generator=g, dtype=torch.float64)
    h = 1e-5
    for tau, alpha in ((1.0, 1.0), (2.0, 0.6), (0.7, 0.0)):
        f = lambda x: R.distill(x, ids, tl, t, w, tau, alpha)[0]
        d = R.distill(z, ids, tl, t, w, tau, alpha)[2]
        assert torch.allclose((f(z + h * v) - f(z - h * v)) / (2 * h), (d * v).sum(1), rtol=1e-7, atol=1e-8)
    for tau in (1.0, 0.6):
        s = lambda x: R.scores(x, t, 0, tau)
        for name, a, b in (("logp", torch.ones(5), None), ("entropy", None, torch.ones(5))):
            d, _ = R.scores_grad(z, t, tau, a, b)
            want = (s(z + h * v)[name] - s(z - h * v)[name]) / (2 * h)
            assert torch.allclose(want, (d * v).sum(1), rtol=1e-7, atol=1e-8), name


# ------------------------------------------------------------------ the head's logits
EMB = L.MebpQ4(q4=0x1000, scale=0x2000)


def _head(f, *args, cfg=None, emb=EMB, norm=0x300000, x=0x400000, rows=8, ws=WS, nb=BIG):
    return f(cfg or make_config(MINI), emb, norm, x, rows, *args, ws, nb, 0, check=False)


def _hz(**kw):
    a = dict(data=Z, ld=MINI.vocab, rows=8, vocab=MINI.vocab, dtype=L.MEBP_F32)
    a.update(kw)
    return L.MebpLogits(**a)


HEAD_CALLS = {
    "logits": lambda **kw: _head(L.mebp_lm_head_logits, _hz(rows=kw.get("rows", 8)), **kw),
    "backward": lambda **kw: _head(L.mebp_lm_head_logits_backward, _hz(rows=kw.get("rows", 8), dtype=L.MEBP_BF16), DZ, **kw),
    "logprobs": lambda **kw: _head(L.mebp_lm_head_logprobs, T, 1.0, 5, L.MebpTokenScores(lse=OUT), **kw),
    "distill": lambda **kw: _head(L.mebp_lm_head_distill_backward, L.MebpDistill(T, T, T, T, 8, 1.0, 0.5), OUT, OUT, DZ, **kw),
}


@pytest.mark.parametrize("name", list(HEAD_CALLS))
def test_head_refused(built_lib, name):
    call = HEAD_CALLS[name]
    assert call(x=0) == L.MEBP_EINVAL and call(x=0x400004) == L.MEBP_EINVAL
    assert call(norm=0) == L.MEBP_EINVAL and call(emb=None) == L.MEBP_EINVAL
    assert call(rows=-1) == L.MEBP_EINVAL and call(ws=0) == L.MEBP_EINVAL and call(ws=WS + 64) == L.MEBP_EINVAL
    c = make_config(MINI)
    need = L.mebp_head_workspace_bytes(c, 8, 5 if name == "logprobs" else 0)
    assert call(nb=need - 1) == L.MEBP_EWORKSPACE
    c.vocab = 0
    assert call(cfg=c) == L.MEBP_EINVAL and "vocab" in L.mebp_last_error()
    assert call(rows=0, x=0) == L.MEBP_OK


def test_head_logits_refused(built_lib):
    f = lambda z: _head(L.mebp_lm_head_logits, z)
    assert f(None) == L.MEBP_EINVAL and f(_hz(rows=7)) == L.MEBP_EINVAL and f(_hz(vocab=32)) == L.MEBP_EINVAL
    assert f(_hz(dtype=L.MEBP_BF16)) == L.MEBP_EUNSUPPORTED and f(_hz(ld=MINI.vocab + 4)) == L.MEBP_EUNSUPPORTED
    assert f(_hz(ld=1 << 20)) == L.MEBP_EUNSUPPORTED and f(_hz(data=Z + 8)) == L.MEBP_EINVAL
    far = _head(L.mebp_lm_head_logits, _hz(rows=4096, ld=(1 << 20) - 8), rows=4096)
    assert far == L.MEBP_EUNSUPPORTED and "blocks" in L.mebp_last_error()
    b = lambda z, dx=DZ: _head(L.mebp_lm_head_logits_backward, z, dx)
    ok = _hz(dtype=L.MEBP_BF16)
    assert b(_hz()) == L.MEBP_EUNSUPPORTED and b(ok, 0) == L.MEBP_EINVAL and b(ok, DZ + 4) == L.MEBP_EINVAL
    assert b(ok, 0x400000) == L.MEBP_EINVAL and "dx" in L.mebp_last_error()
    size = 8 * MINI.hidden * 4  # of x, and of dx
    for at in (0x400000 + size - 16, 0x400000 - size + 16):
        assert b(ok, at) == L.MEBP_EINVAL and "dx" in L.mebp_last_error()


def test_head_operators_refused(built_lib):
    s = lambda t, tau, k, out: _head(L.mebp_lm_head_logprobs, t, tau, k, out)
    assert s(T, 0.0, 5, L.MebpTokenScores(lse=OUT)) == L.MEBP_EINVAL
    assert s(T, 1.0, 65, L.MebpTokenScores(lse=OUT)) == L.MEBP_EUNSUPPORTED
    assert s(0, 1.0, 5, L.MebpTokenScores(logp=OUT)) == L.MEBP_EINVAL
    assert s(T, 1.0, 0, L.MebpTokenScores(top_ids=OUT)) == L.MEBP_EINVAL
    d = lambda loss=OUT, rl=0, **kw: _head(L.mebp_lm_head_distill_backward, L.MebpDistill(
        **dict(dict(ids=T, logits=T, targets=T, row_weight=0, k=8, temperature=1.0, alpha=0.5), **kw)), loss, rl, DZ)
    assert d(k=0) == L.MEBP_EUNSUPPORTED and d(alpha=2.0) == L.MEBP_EINVAL and d(ids=0) == L.MEBP_EINVAL
    assert d(targets=0) == L.MEBP_EINVAL and d(loss=0) == L.MEBP_EINVAL and d(rl=OUT + 1) == L.MEBP_EINVAL


def test_head_workspace_sizes(built_lib):
    c = make_config(MINI)
    assert L.mebp_head_workspace_bytes(c, -1) == 0 and L.mebp_head_workspace_bytes(c, 8, 65) == 0
    assert 0 < L.mebp_head_workspace_bytes(c, 8) <= L.mebp_head_workspace_bytes(c, 8, 64) < L.mebp_head_workspace_bytes(c, 900, 64)
    # many rows go in blocks: their logits and gradients stay within the budget of 512 MiB
    big = make_config(CONFIGS["gemma3-4b"])
    a, b = L.mebp_head_workspace_bytes(big, 4096), L.mebp_head_workspace_bytes(big, 16384)
    assert b - a == (16384 - 4096) * 4 and a < 900 << 20
    step = L.mebp_distill_step_workspace_bytes(c, 2, 160)
    assert step == L.mebp_workspace_bytes(c, 2, 160) + L.mebp_head_workspace_bytes(c, 320)
    assert L.mebp_distill_step_workspace_bytes(c, 0, 160) == 0


def test_distillation_step_refused(built_lib):
    c = make_config(MINI)
    d = L.MebpDistill(T, T, T, T, 8, 1.0, 0.5)
    need = L.mebp_distill_step_workspace_bytes(c, 2, 160)
    n = c.n_layers
    base, lora, grads = (L.MebpLayerBase * n)(), (L.MebpLayerLora * n)(), (L.MebpLayerLoraGrad * n)()
    for l in range(n):
        for i in range(7):
            base[l].w[i].q4, base[l].w[i].scale = 0x1000, 0x2000
            lora[l].A[i] = lora[l].B[i] = grads[l].dA[i] = grads[l].dB[i] = 0x3000
        base[l].norm_attn = base[l].norm_mlp = 0x4000
    f = lambda distill=d, nb=need, ckpt=0x5000, loss=OUT, rl=0: L.mebp_train_step_distill(
        c, EMB, base, 0x300000, lora, T, 2, 160, distill, ckpt, loss, rl, grads, 0, WS, nb, 0, check=False)
    assert f(nb=need - 1) == L.MEBP_EWORKSPACE
    assert f(nb=L.mebp_workspace_bytes(c, 2, 160)) == L.MEBP_EWORKSPACE
    assert f(distill=None) == L.MEBP_EINVAL and f(ckpt=0) == L.MEBP_EINVAL and f(loss=0) == L.MEBP_EINVAL
    assert f(rl=OUT + 2) == L.MEBP_EINVAL
    assert f(distill=L.MebpDistill(T, T, T, T, 99, 1.0, 0.5)) == L.MEBP_EUNSUPPORTED
