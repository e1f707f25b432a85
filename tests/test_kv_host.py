"""Host-only checks of the operators of a forward pass over a cache: what they refuse before touching the
GPU, their workspaces, and the 64-bit reference of their tests."""
import ctypes as C
import math

import pytest
import torch

import kv_ref as R
from mebp_inputs import CONFIGS, MINI
from paper_2510_03425_amd import _lib as L
from paper_2510_03425_amd import device as D
from paper_2510_03425_amd.device import make_config

K, V, Q, OUT, WS, PG, SC, TAB, ST, PA, TB, LSE = (i << 36 for i in range(1, 13))
BIG = 1 << 34


def _heads(at, **kw):
    a = dict(data=at, ld=512, head_ld=64, tokens=4, heads=2, dim=64, dtype=L.MEBP_F16)
    a.update(kw)
    return L.MebpHeads(**a)


def _rope(**kw):
    a = dict(table=TAB, rot=64, n_pos=100, interleaved=0)
    a.update(kw)
    return L.MebpRope(**a)


def _cache(**kw):
    a = dict(pages=PG, scales=SC, n_pages=9, page_tokens=64, heads=2, dim=64)
    a.update(kw)
    return L.MebpKvCache(**a)


def _batch(**kw):
    a = dict(start=ST, past=PA, table=TB, table_ld=3, max_pages=3, seqs=2, max_new=4, max_len=190)
    a.update(kw)
    return L.MebpKvBatch(**a)


def _apply(rope=None, x=None, y=None, pos=ST, backward=0):
    return L.mebp_rope_apply(rope or _rope(), x or _heads(Q), pos, y or _heads(OUT), backward, check=False)


def _append(cache=None, batch=None, rope=0, k=None, v=None, q=None, q_out=None):
    return L.mebp_kv_append(cache or _cache(), batch or _batch(), _rope() if rope == 0 else rope, k or _heads(K), v or _heads(V),
                            q, q_out, check=False)


def _read(cache=None, batch=None, k=None, v=None):
    return L.mebp_kv_read(cache or _cache(), batch or _batch(), k, v, check=False)


def _attend(cache=None, batch=None, q=None, out=None, lse=LSE, scale=0.125, window=0, ws=WS, nb=BIG):
    return L.mebp_kv_attention(cache or _cache(), batch or _batch(), q or _heads(Q, heads=4), out or _heads(OUT, heads=4), lse, scale,
                               window, ws, nb, check=False)


@pytest.mark.parametrize("bad,code", [
    (dict(data=0), L.MEBP_EINVAL), (dict(data=Q + 1), L.MEBP_EINVAL), (dict(tokens=-1), L.MEBP_EINVAL), (dict(heads=0), L.MEBP_EINVAL),
    (dict(dim=0), L.MEBP_EINVAL), (dict(dtype=3), L.MEBP_EINVAL), (dict(dtype=-1), L.MEBP_EINVAL), (dict(ld=-1), L.MEBP_EINVAL),
    (dict(head_ld=-1), L.MEBP_EINVAL), (dict(tokens=(1 << 24) + 1), L.MEBP_EUNSUPPORTED), (dict(heads=1025), L.MEBP_EUNSUPPORTED),
    (dict(dim=1025), L.MEBP_EUNSUPPORTED), (dict(ld=(1 << 32) + 1), L.MEBP_EUNSUPPORTED),
])
def test_heads_refused(built_lib, bad, code):
    assert _apply(x=_heads(Q, **bad)) == code and L.mebp_last_error()
    assert _append(k=_heads(K, **bad)) == code and _attend(q=_heads(Q, **bad)) == code
    assert _read(k=_heads(K, **bad)) == code


def test_outputs_that_overlap_themselves_refused(built_lib):
    assert _apply(y=_heads(OUT, head_ld=63)) == L.MEBP_EINVAL and "overlap" in L.mebp_last_error()
    assert _apply(y=_heads(OUT, ld=127)) == L.MEBP_EINVAL
    assert _apply(y=_heads(OUT, ld=0)) == L.MEBP_EINVAL
    assert _read(k=_heads(K, ld=100)) == L.MEBP_EINVAL
    # tokens within heads are as good
    assert _apply(rope=_rope(n_pos=0), y=_heads(OUT, ld=64, head_ld=256)) == L.MEBP_EINVAL and "rope" in L.mebp_last_error()


@pytest.mark.parametrize("bad", [dict(table=0), dict(table=TAB + 4), dict(rot=0), dict(rot=63), dict(rot=66), dict(n_pos=0),
                                 dict(interleaved=2)])
def test_rope_refused(built_lib, bad):
    assert _apply(rope=_rope(**bad)) == L.MEBP_EINVAL and "rope" in L.mebp_last_error()
    assert _append(rope=_rope(**bad)) == L.MEBP_EINVAL


def test_rope_positions_refused(built_lib):
    def call(rope=None, **kw):
        a = dict(theta=1e4, factor=2.0, original=0, low=1.0, high=32.0, gain=1.0)
        a.update(kw)
        return L.mebp_rope_positions(rope or _rope(), L.MebpRopeScaling(**a), check=False)

    for bad in (dict(theta=0.0), dict(theta=math.nan), dict(theta=math.inf), dict(factor=0.5), dict(factor=math.inf), dict(gain=math.nan),
                dict(original=-1), dict(original=100, low=-1.0), dict(original=100, high=1.0), dict(original=100, high=math.inf)):
        assert call(**bad) == L.MEBP_EINVAL and L.mebp_last_error(), bad
    assert L.mebp_rope_positions(_rope(), None, check=False) == L.MEBP_EINVAL
    assert call(rope=_rope(table=0)) == L.MEBP_EINVAL
    assert L.mebp_rope_positions(None, L.MebpRopeScaling(1e4, 1, 0, 1, 32, 1), check=False) == L.MEBP_EINVAL


def test_rope_apply_refused(built_lib):
    assert _apply(pos=0) == L.MEBP_EINVAL and _apply(pos=ST + 2) == L.MEBP_EINVAL
    for bad in (dict(tokens=3), dict(heads=3, ld=1024), dict(dim=32), dict(dtype=L.MEBP_BF16)):
        assert _apply(y=_heads(OUT, **bad)) == L.MEBP_EINVAL
    # in part over x, over the positions, over the table
    assert _apply(y=_heads(Q + 128)) == L.MEBP_EINVAL and "overlap" in L.mebp_last_error()
    assert _apply(y=_heads(Q, ld=1024)) == L.MEBP_EINVAL
    assert _apply(y=_heads(ST)) == L.MEBP_EINVAL and _apply(y=_heads(TAB)) == L.MEBP_EINVAL
    assert _apply(x=_heads(Q, tokens=1 << 24, heads=1024), y=_heads(OUT, tokens=1 << 24, heads=1024, ld=1 << 16)) == L.MEBP_EUNSUPPORTED
    assert _apply(x=_heads(0, tokens=0), y=_heads(0, tokens=0), pos=0) == L.MEBP_OK


def test_rows_of_one_matrix_side_by_side(built_lib):
    """Outputs in the columns beside what is read are apart; one column into it they are not. (There are no
    sequences, so that nothing is launched.)"""
    none = _batch(seqs=0)
    for at, ok in ((Q + 2 * 256, True), (Q + 2 * 255, False), (Q - 2 * 128, True), (Q - 2 * 127, False), (Q + 2 * 384, True),
                   (Q + 2 * 385, False), (Q + 2 * (512 + 256), True), (Q + 2 * (2 * 512 + 384), True)):
        got = _append(batch=none, q=_heads(Q, heads=4), q_out=_heads(Q, heads=4), k=_heads(at), v=_heads(V))
        assert got == (L.MEBP_OK if ok else L.MEBP_EINVAL), (at - Q, got)
    # other distances of the tokens
    assert _append(batch=none, q=_heads(Q, heads=4), q_out=_heads(Q, heads=4), k=_heads(Q + 512, ld=400), v=_heads(V)) == L.MEBP_EINVAL


@pytest.mark.parametrize("bad,code", [
    (dict(pages=0), L.MEBP_EINVAL), (dict(pages=PG + 8), L.MEBP_EINVAL), (dict(scales=0), L.MEBP_EINVAL), (dict(scales=SC + 4), L.MEBP_EINVAL),
    (dict(n_pages=0), L.MEBP_EINVAL), (dict(heads=0), L.MEBP_EINVAL), (dict(page_tokens=0), L.MEBP_EINVAL),
    (dict(page_tokens=8), L.MEBP_EUNSUPPORTED), (dict(page_tokens=48), L.MEBP_EUNSUPPORTED), (dict(page_tokens=1 << 17), L.MEBP_EUNSUPPORTED),
    (dict(dim=96), L.MEBP_EUNSUPPORTED), (dict(heads=1025), L.MEBP_EUNSUPPORTED),
])
def test_cache_refused(built_lib, bad, code):
    assert _append(cache=_cache(**bad)) == code and _read(cache=_cache(**bad), k=_heads(K)) == code
    assert _attend(cache=_cache(**bad)) == code and "cache" in L.mebp_last_error()


@pytest.mark.parametrize("bad,code", [
    (dict(start=0), L.MEBP_EINVAL), (dict(past=0), L.MEBP_EINVAL), (dict(table=0), L.MEBP_EINVAL), (dict(start=ST + 2), L.MEBP_EINVAL),
    (dict(table_ld=2), L.MEBP_EINVAL), (dict(max_pages=0), L.MEBP_EINVAL), (dict(seqs=-1), L.MEBP_EINVAL), (dict(max_new=0), L.MEBP_EINVAL),
    (dict(max_len=0), L.MEBP_EINVAL), (dict(seqs=65536), L.MEBP_EUNSUPPORTED), (dict(max_new=(1 << 24) + 1), L.MEBP_EUNSUPPORTED),
    (dict(max_len=(1 << 30) + 1), L.MEBP_EUNSUPPORTED),
])
def test_batch_refused(built_lib, bad, code):
    assert _append(batch=_batch(**bad)) == code and _read(batch=_batch(**bad), v=_heads(V)) == code
    assert _attend(batch=_batch(**bad)) == code and "batch" in L.mebp_last_error()


def test_append_refused(built_lib):
    for bad in (dict(tokens=3), dict(heads=1), dict(dim=32), dict(dtype=L.MEBP_F32)):
        assert _append(v=_heads(V, **bad)) == L.MEBP_EINVAL
    assert _append(k=_heads(K, heads=3), v=_heads(V, heads=3)) == L.MEBP_EINVAL
    q, qo = _heads(Q, heads=4), _heads(OUT, heads=4)
    assert _append(q=q) == L.MEBP_EINVAL and _append(q_out=qo) == L.MEBP_EINVAL
    assert _append(q=q, q_out=qo, rope=None) == L.MEBP_EINVAL and "together" in L.mebp_last_error()
    assert _append(q=q, q_out=_heads(OUT, heads=5)) == L.MEBP_EINVAL
    assert _append(q=q, q_out=_heads(Q + 64, heads=4)) == L.MEBP_EINVAL and "overlap" in L.mebp_last_error()
    for at in (K, V, PG, SC, TAB, ST, PA, TB):
        assert _append(q=q, q_out=_heads(at, heads=4)) == L.MEBP_EINVAL and "overlap" in L.mebp_last_error(), hex(at)
    for at in (K, V, ST, PA, TB, TAB):
        assert _append(cache=_cache(pages=at)) == L.MEBP_EINVAL and "overlap" in L.mebp_last_error()
        assert _append(cache=_cache(scales=at)) == L.MEBP_EINVAL
    assert _append(cache=_cache(scales=PG + 64)) == L.MEBP_EINVAL
    assert _append(batch=_batch(max_new=1 << 24), cache=_cache(heads=1024), k=_heads(K, heads=1024, ld=1 << 17),
                   v=_heads(V, heads=1024, ld=1 << 17)) == L.MEBP_EUNSUPPORTED
    nothing = dict(k=_heads(0, tokens=0), v=_heads(0, tokens=0))
    assert _append(**nothing) == L.MEBP_OK
    assert _append(batch=_batch(seqs=0, start=0, past=0, table=0)) == L.MEBP_OK


def test_read_refused(built_lib):
    assert _read() == L.MEBP_EINVAL and "neither" in L.mebp_last_error()
    assert _read(k=_heads(K), v=_heads(V, tokens=5)) == L.MEBP_EINVAL
    assert _read(k=_heads(K), v=_heads(K + 64)) == L.MEBP_EINVAL and "overlap" in L.mebp_last_error()
    assert _read(k=_heads(PG)) == L.MEBP_EINVAL and _read(v=_heads(ST)) == L.MEBP_EINVAL
    assert _read(k=_heads(K, heads=1)) == L.MEBP_EINVAL


def test_attention_refused(built_lib):
    assert _attend(q=_heads(Q, heads=3), out=_heads(OUT, heads=3)) == L.MEBP_EINVAL and "multiple" in L.mebp_last_error()
    f32 = dict(heads=4, dtype=L.MEBP_F32)
    assert _attend(q=_heads(Q, **f32), out=_heads(OUT, **f32)) == L.MEBP_EUNSUPPORTED
    assert _attend(out=_heads(OUT, heads=4, dtype=L.MEBP_BF16)) == L.MEBP_EINVAL and _attend(out=_heads(OUT, heads=4, tokens=5)) == L.MEBP_EINVAL
    assert _attend(scale=math.nan) == L.MEBP_EINVAL and _attend(scale=math.inf) == L.MEBP_EINVAL
    assert _attend(scale=3e38) == L.MEBP_EINVAL and _attend(scale=-3e38) == L.MEBP_EINVAL  # (times log2 e)
    assert _attend(window=-1) == L.MEBP_EINVAL and _attend(lse=LSE + 2) == L.MEBP_EINVAL
    assert _attend(ws=0) == L.MEBP_EINVAL and _attend(ws=WS + 16) == L.MEBP_EINVAL
    need = L.mebp_kv_attention_workspace_bytes(2, 4, 5000, 4, 2, 64)
    assert _attend(batch=_batch(max_len=5000), nb=need - 1) == L.MEBP_EWORKSPACE
    for at in (Q, PG, SC, ST, PA, TB, LSE, WS):
        assert _attend(out=_heads(at, heads=4)) == L.MEBP_EINVAL and "overlap" in L.mebp_last_error(), hex(at)
    for at in (Q, PG, SC, ST, PA, TB, WS):
        assert _attend(lse=at) == L.MEBP_EINVAL and "overlap" in L.mebp_last_error(), hex(at)
    assert _attend(ws=PG) == L.MEBP_EINVAL
    assert _attend(q=_heads(0, heads=4, tokens=0), out=_heads(0, heads=4, tokens=0)) == L.MEBP_OK


def test_workspaces(built_lib):
    f = L.mebp_kv_attention_workspace_bytes
    assert f(0, 1, 1, 1, 1, 64) == 256 and f(1, 1, 64, 8, 4, 256) == 256
    for bad in ((-1, 1, 1, 4, 2, 64), (1, 0, 1, 4, 2, 64), (1, 1, 0, 4, 2, 64), (1, 1, 1, 3, 2, 64), (1, 1, 1, 4, 2, 96), (1, 1, 1, 4, 2, 64, -1)):
        assert f(*bad) == 0, bad
    # one long sequence is split over the chip; a window keeps it short
    assert f(1, 1, 131072, 12, 2, 128) > 64 * f(1, 1, 131072, 12, 2, 128, 64)
    assert L.mebp_kv_page_bytes(64, 4, 256) == 64 * 4 * 256 * 2 and L.mebp_kv_page_bytes(60, 4, 256) == 0
    for cfg in CONFIGS.values():
        c = make_config(cfg)
        small, large = (L.mebp_cached_workspace_bytes(c, n, 4, n, 4096) for n in (1, 512))
        assert 0 < small < large
        assert L.mebp_cached_workspace_bytes(c, 0, 1, 1, 1) == 0 == L.mebp_cached_workspace_bytes(c, 1, 1, 1, 0)


def test_cached_layer_refused(built_lib):
    from test_abi_host import _fake_layer
    c = make_config(MINI)
    base, lora = _fake_layer()
    need = L.mebp_cached_workspace_bytes(c, 4, 2, 4, 190)

    def call(layer=0, x=Q, y=OUT, rows=4, cache=None, batch=None, rope=0, ws=WS, nb=need, base=base):
        return L.mebp_layer_forward_cached(c, layer, base, lora, x, y, rows, cache or _cache(), batch or _batch(),
                                           _rope() if rope == 0 else rope, ws, nb, check=False)

    assert call(layer=2) == L.MEBP_EINVAL and call(x=0) == L.MEBP_EINVAL and call(y=0) == L.MEBP_EINVAL
    assert call(rows=0) == L.MEBP_EINVAL and call(base=None) == L.MEBP_EINVAL
    assert call(y=Q) == L.MEBP_EINVAL and "overlap" in L.mebp_last_error()
    assert call(y=PG) == L.MEBP_EINVAL and call(ws=PG) == L.MEBP_EINVAL and call(ws=Q & ~255) == L.MEBP_EINVAL
    assert call(cache=_cache(heads=1)) == L.MEBP_EINVAL and call(cache=_cache(dim=128)) == L.MEBP_EINVAL
    assert call(rope=None) == L.MEBP_EINVAL and call(rope=_rope(rot=66)) == L.MEBP_EINVAL
    assert call(batch=_batch(seqs=0)) == L.MEBP_EINVAL and call(batch=_batch(past=0)) == L.MEBP_EINVAL
    assert call(nb=need - 1) == L.MEBP_EWORKSPACE and call(ws=0) == L.MEBP_EINVAL and call(ws=WS + 64) == L.MEBP_EINVAL


def test_wrappers_refuse_what_is_not_on_the_gpu():
    x = torch.zeros(2, 2, 64)
    with pytest.raises(ValueError):
        D.Rope(torch.zeros(4, 32, 2))
    with pytest.raises(ValueError):
        D.KvCache(torch.zeros(1, 2, 4, 2, 1024, dtype=torch.int8), torch.zeros(1, 2, 4, 2))
    with pytest.raises(ValueError):
        D.KvBatch(torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros(1, 1, dtype=torch.int32), 1, 64)
    with pytest.raises(ValueError):
        D.heads_struct(x)


# ------------------------------------------------------------------------------- the reference
def test_reference_rotation():
    tab = R.table(50, 32, 1e4)
    g = torch.Generator().manual_seed(0)
    x = torch.randn(50, 3, 40, generator=g, dtype=R.F64)
    pos = torch.arange(50)
    for inter in (False, True):
        y = R.turn(x, tab, pos, inter)
        assert torch.allclose(y[0], x[0]) and torch.equal(y[..., 32:], x[..., 32:])
        assert torch.allclose(y.norm(dim=2), x.norm(dim=2)) and torch.allclose(R.turn(y, tab, pos, inter, True), x)
        # products of two rotated heads depend on the distance of their positions alone
        same = torch.ones(50, 1, 40, dtype=R.F64)
        u, w = R.turn(same, tab, pos, inter)[:, 0], R.turn(same * 2, tab, pos, inter)[:, 0]
        assert torch.allclose((u[5:] * w[:-5]).sum(1), (u[5] * w[0]).sum().expand(45))
        # the backward is the gradient: central differences of a random weighting of y
        c = torch.randn(50, 3, 40, generator=g, dtype=R.F64)
        e = torch.zeros_like(x)
        e[7, 1, 3] = 1e-6
        d = ((R.turn(x + e, tab, pos, inter) - R.turn(x - e, tab, pos, inter)) * c).sum() / 2e-6
        assert abs(float(d - R.turn(c, tab, pos, inter, True)[7, 1, 3])) < 1e-6


def test_reference_scaling():
    f = R.frequencies(64, 1e4)
    assert torch.allclose(R.frequencies(64, 1e4, factor=8.0), f / 8)
    g = R.frequencies(64, 1e4, factor=8.0, original=4096)
    turns = 4096 * f / (2 * math.pi)
    assert torch.equal(g[turns > 32], f[turns > 32]) and torch.allclose(g[turns < 1], f[turns < 1] / 8)
    assert (g[:-1] > g[1:]).all()


def test_reference_cache_and_attention():
    g = torch.Generator().manual_seed(1)
    c = R.Cache(torch.randint(-127, 128, (5, 2, 2, 2, 16 * 64), generator=g, dtype=torch.int8), torch.rand(5, 2, 2, 2, generator=g))
    k, v = (torch.randn(40, 2, 64, generator=g, dtype=R.F64) for _ in range(2))
    row = torch.tensor([3, 0])
    c.append(row, 0, k[:21], v[:21])
    for i in range(21, 40):
        c.append(row, i, k[i:i + 1], v[i:i + 1])
    kr, vr = c.read(row, 0, 40)
    for x, y in ((k, kr), (v, vr)):
        # one rounding each, and one more each time that a later token raised the block's scale (8 at most here)
        assert float((x - y).abs().max()) <= 5 * float(x.abs().max()) / 127
    q = torch.randn(3, 4, 64, generator=g, dtype=R.F64)
    out, lse, _, _ = R.attention(q, kr, vr, 37, 0.125, 9)
    for n in range(3):
        for h in range(4):
            lo, hi = 37 + n - 8, 37 + n + 1
            x = (kr[lo:hi, h // 2] @ q[n, h]) * 0.125
            assert abs(float(torch.logsumexp(x, 0) - lse[n, h])) < 1e-12
            assert torch.allclose(torch.softmax(x, 0) @ vr[lo:hi, h // 2], out[n, h])
