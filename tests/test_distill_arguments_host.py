"""Host-only: which operands of a distillation its weight alpha leaves unread."""
import pytest

from mebp_inputs import MINI
from paper_2510_03425_amd import _lib as L
from paper_2510_03425_amd.device import make_config

Z, T, OUT, WS = 0x1000000, 0x2000000, 0x3000000, 0x10000000


def _calls(**kw):
    """Both entry points with a workspace too small, the last thing that they check."""
    d = L.MebpDistill(**dict(dict(ids=T, logits=T, targets=T, row_weight=0, k=8, temperature=2.0, alpha=0.5), **kw))
    z = L.MebpLogits(data=Z, ld=1000, rows=4, vocab=1000, dtype=L.MEBP_F32)
    yield L.mebp_distill_topk(z, d, OUT, None, WS, 0, 0, check=False)
    yield L.mebp_lm_head_distill_backward(make_config(MINI), L.MebpQ4(q4=0x1000, scale=0x2000), 0x300000, 0x400000, 8, d, OUT,
                                          0, 0x8000000, WS, 0, 0, check=False)


@pytest.mark.parametrize("unread", [dict(ids=0, logits=0), dict(ids=0), dict(logits=0), dict(ids=T + 1, logits=T + 2)])
def test_entries_are_not_read_at_alpha_0(built_lib, unread):
    assert list(_calls(alpha=0.0, **unread)) == [L.MEBP_EWORKSPACE] * 2
    assert list(_calls(alpha=1e-6, **unread)) == [L.MEBP_EINVAL] * 2
    assert list(_calls(alpha=0.0, targets=0, **unread)) == [L.MEBP_EINVAL] * 2


def test_labels_are_not_read_at_alpha_1(built_lib):
    assert list(_calls(alpha=1.0, targets=0)) == [L.MEBP_EWORKSPACE] * 2
    assert list(_calls(alpha=0.0, k=0)) == [L.MEBP_EUNSUPPORTED] * 2
