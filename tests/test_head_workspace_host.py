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
