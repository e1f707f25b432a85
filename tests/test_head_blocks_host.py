"""Host-only: the blocks of rows that the LM head's calls run in, for any budget of theirs."""
import os
import subprocess
import sys

import pytest

from mebp_inputs import CONFIGS
from paper_2510_03425_amd import _lib as L
from paper_2510_03425_amd.device import make_config

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CALLS = """
from mebp_inputs import CONFIGS
from paper_2510_03425_amd import _lib as L
from paper_2510_03425_amd.device import make_config
c = make_config(CONFIGS["gemma3-4b"])
emb, out = L.MebpQ4(q4=0x1000, scale=0x2000), []
for rows in (64, 4096, 1 << 16):
    for ld in (c.vocab, c.vocab + 64):
        for f, dtype in ((L.mebp_lm_head_logits, L.MEBP_F32), (L.mebp_lm_head_logits, L.MEBP_F16)):
            z = L.MebpLogits(0x1000000, ld, rows, c.vocab, dtype)
            out.append(f(c, emb, 0x300000, 0x400000, rows, z, 0x10000000, 0, 0, check=False))
        z = L.MebpLogits(0x1000000, ld, rows, c.vocab, L.MEBP_BF16)
        out.append(L.mebp_lm_head_logits_backward(c, emb, 0x300000, 0x100000000000, rows, z, 0x400000, 0x10000000, 0, 0, check=False))
print(sorted(set(out)), L.mebp_head_workspace_bytes(c, 1 << 16) - 4 * (1 << 16))
"""


@pytest.mark.parametrize("mb", [1, 512, 4096, 65536])
def test_contiguous_logits_fit_a_block_at_any_budget(built_lib, mb):
    """Refused for the workspace alone, which is too small here; a block stays below 2^30 logits."""
    r = subprocess.run([sys.executable, "-c", CALLS], cwd=ROOT, env=dict(os.environ, MEBP_LM_CHUNK_MB=str(mb)),
                       capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr
    codes, block = r.stdout.strip().rsplit(" ", 1)
    assert codes == str([L.MEBP_EWORKSPACE]), codes
    assert int(block) <= 6 * 2 ** 30 + (2 << 20)


def test_a_vocabulary_beyond_the_products_is_refused(built_lib):
    """The rows of a tile are addressed with 32 bits, in a block of the head's as in the caller's matrix."""
    c = make_config(CONFIGS["qwen2.5-0.5b"])
    emb, x, ws = L.MebpQ4(q4=0x1000, scale=0x2000), 0x400000, 0x10000000
    for vocab, ok in ((151936, True), (1 << 20, False), (1 << 22, False)):
        c.vocab = vocab
        s = L.mebp_lm_head_logprobs(c, emb, 0x300000, x, 4, 0, 1.0, 0, L.MebpTokenScores(lse=0x1000000), ws, 0, 0, check=False)
        d = L.mebp_lm_head_distill_backward(c, emb, 0x300000, x, 4, L.MebpDistill(0x1000, 0x1000, 0, 0, 4, 1.0, 1.0), 0x1000000,
                                            0, 0x8000000, ws, 0, 0, check=False)
        assert (s, d) == ((L.MEBP_EWORKSPACE,) * 2 if ok else (L.MEBP_EUNSUPPORTED,) * 2), vocab
        assert (L.mebp_head_workspace_bytes(c, 4) > 0) == ok and (L.mebp_distill_step_workspace_bytes(c, 1, 4) > 0) == ok
