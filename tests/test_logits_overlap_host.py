"""Host-only: outputs of the operators on logits that overlap what a call reads."""
import pytest

from mebp_inputs import MINI
from paper_2510_03425_amd import _lib as L
from paper_2510_03425_amd.device import make_config

Z, DZ, T, A, B, OUT, WS = (0x1000000 * i for i in range(1, 8))
ROWS, V, K = 4, 1000, 5
SIZE = ROWS * V * 4  # of the logits, fp32


def _z(data=Z):
    return L.MebpLogits(data, V, ROWS, V, L.MEBP_F32)


def _scores(targets=T, **out):
    o = dict(logp=OUT, lse=OUT + 0x100, entropy=OUT + 0x200, top_ids=OUT + 0x300, top_logp=OUT + 0x400)
    o.update(out)
    return L.mebp_token_logprobs(_z(), targets, 1.0, K, L.MebpTokenScores(**o), WS, 0, 0, check=False)


def _grad(dz=DZ, **kw):
    a = dict(targets=T, lse=A, entropy=A, d_logp=B, d_entropy=B)
    a.update(kw)
    return L.mebp_token_logprobs_backward(_z(), a["targets"], 0.0, a["lse"], a["entropy"], a["d_logp"], a["d_entropy"], _z(dz), 0,
                                          check=False)


def _distill(loss=OUT, dz=DZ, head=False, **kw):
    d = L.MebpDistill(**dict(dict(ids=T, logits=A, targets=B, row_weight=B + 0x100, k=K, temperature=1.0, alpha=0.5), **kw))
    if head:
        return L.mebp_lm_head_distill_backward(make_config(MINI), L.MebpQ4(q4=0x1000, scale=0x2000), 0x300000, 0x400000, ROWS, d,
                                               0x9000000, loss, DZ, WS, 0, 0, check=False)
    return L.mebp_distill_topk(_z(), d, loss, _z(dz) if dz else None, WS, 0, 0, check=False)


def test_calls_that_lie_apart_are_taken(built_lib):
    """As far as the workspace, which is too small here (the gradient has none: its temperature)."""
    assert _scores() == L.MEBP_EWORKSPACE and _distill() == L.MEBP_EWORKSPACE and _distill(head=True) == L.MEBP_EWORKSPACE
    assert _grad() == L.MEBP_EINVAL and "temperature" in L.mebp_last_error()
    # right behind one another, the same operand read twice, operands that the call does not read
    assert _scores(logp=T + 4 * ROWS, lse=T + 8 * ROWS) == L.MEBP_EWORKSPACE
    assert _distill(targets=T, row_weight=T, logits=T) == L.MEBP_EWORKSPACE
    assert _distill(loss=T, alpha=0.0) == L.MEBP_EWORKSPACE and _distill(loss=B, alpha=1.0) == L.MEBP_EWORKSPACE
    assert _distill(loss=T - 8, alpha=0.0) == L.MEBP_EWORKSPACE and _distill(loss=B - 8, alpha=1.0) == L.MEBP_EWORKSPACE
    assert _scores(logp=0, lse=T) == L.MEBP_EWORKSPACE and _scores(logp=0, lse=T - 8) == L.MEBP_EWORKSPACE
    assert _distill(dz=Z) == L.MEBP_EWORKSPACE  # in place


@pytest.mark.parametrize("out", [dict(lse=T), dict(logp=T + 4),
                                 dict(top_logp=Z + SIZE - 4), dict(entropy=Z - 4 * ROWS + 4)])
def test_scores(built_lib, out):
    assert _scores(**out) == L.MEBP_EINVAL and "overlap" in L.mebp_last_error()


@pytest.mark.parametrize("kw", [dict(targets=DZ), dict(lse=DZ + SIZE - 4), dict(entropy=DZ - 4 * ROWS + 4), dict(d_logp=DZ + 64), dict(d_entropy=DZ)])
def test_gradient_of_the_scores(built_lib, kw):
    assert L.mebp_token_logprobs_backward(_z(), *[dict(dict(targets=T, lse=A, entropy=A, d_logp=B, d_entropy=B), **kw)[n] if n else 1.0
                                                  for n in ("targets", "", "lse", "entropy", "d_logp", "d_entropy")],
                                          _z(DZ), 0, check=False) == L.MEBP_EINVAL
    assert "overlap" in L.mebp_last_error()


@pytest.mark.parametrize("kw", [dict(loss=T), dict(loss=A + 4 * ROWS * K - 4), dict(loss=B), dict(loss=B + 0x100), dict(loss=Z + 400),
                                dict(loss=DZ), dict(loss=Z, dz=0), dict(ids=DZ), dict(logits=DZ + SIZE - 4), dict(row_weight=DZ + 4)])
def test_distillation(built_lib, kw):
    assert _distill(**kw) == L.MEBP_EINVAL and "overlap" in L.mebp_last_error()


@pytest.mark.parametrize("kw", [dict(loss=T), dict(loss=A + 4), dict(loss=B), dict(loss=B + 0x100), dict(loss=0x400000), dict(loss=DZ),
                                dict(ids=DZ), dict(targets=DZ + 16)])
def test_distillation_of_the_head(built_lib, kw):
    assert _distill(head=True, **kw) == L.MEBP_EINVAL and "overlap" in L.mebp_last_error()
