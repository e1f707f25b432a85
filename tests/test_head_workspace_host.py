"""Host-only: what the workspaces of the LM head's calls hold at once."""
import pytest

from mebp_inputs import CONFIGS
from paper_2510_03425_amd import _lib as L
from paper_2510_03425_amd.device import make_config

SMALL = 2 << 20  # statistics, alternatives, picked logits and row losses of a block


@pytest.mark.parametrize("name", ["qwen2.5-0.5b", "gemma3-1b", "qwen2.5-1.5b", "gemma3-4b"])
@pytest.mark.parametrize("rows", [1, 64, 256, 16384])
def test_a_block_of_logits_and_gradients_is_all_that_the_head_holds(built_lib, name, rows):
    """The final norm is read before the gradient is written where it lay, the products' planes
    and sums lie where the logits were."""
    c = make_config(CONFIGS[name])
    need = L.mebp_head_workspace_bytes(c, rows, 64)
    block = max(1, min(rows, (512 << 20) // (6 * c.vocab) // 256 * 256))
    assert 6 * block * c.vocab <= need <= 6 * block * c.vocab + 4 * rows + SMALL


@pytest.mark.parametrize("name,B,T", [("gemma3-4b", 8, 2048), ("gemma3-4b", 4, 1024), ("gemma3-4b", 1, 256), ("qwen2.5-1.5b", 4, 1024),
                                      ("qwen2.5-0.5b", 8, 2048), ("qwen2.5-0.5b", 1, 256)])
def test_a_distillation_step_takes_no_more_than_a_step(built_lib, name, B, T):
    """The head's logits lie where the cross-entropy has its own, or its copy of the weights."""
    c = make_config(CONFIGS[name])
    assert L.mebp_distill_step_workspace_bytes(c, B, T) == L.mebp_workspace_bytes(c, B, T)


def test_a_distillation_step_takes_a_head_more_where_it_fits_nowhere(built_lib):
    for name, cfg in CONFIGS.items():
        if not cfg.vocab:
            continue
        c = make_config(cfg)
        for B, T in ((1, 1), (1, 3), (2, 100), (1, 256), (3, 333), (4, 1024)):
            step, head = L.mebp_workspace_bytes(c, B, T), L.mebp_head_workspace_bytes(c, B * T)
            assert L.mebp_distill_step_workspace_bytes(c, B, T) in (step, step + head), (name, B, T)
