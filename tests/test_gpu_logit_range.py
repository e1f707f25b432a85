"""The operators on logits on the GPU at the ends of what they accept: large gradients of the
entropy beside masked columns."""
import math

import pytest
import torch

from gpu_util import say
from paper_2510_03425_amd import device as D

pytestmark = pytest.mark.gpu
INF = math.inf
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("tau,d_entropy", [(1e-6, 1000.0), (1e-3, 5e5), (1.0, 1e20), (1.0, -1e30)])
def test_masked_columns_have_no_gradient_whatever_the_entropys_is(built_lib, gpu, dtype, tau, d_entropy):
    """d_entropy / tau beyond 3.4e8: its product with a weight's logarithm is no number of fp32 where
    the logarithm is far below any weight's. Columns whose weight is 0 (masked by -inf, by the type's
    lowest value or by -3e4 of fp16) have gradient 0 at any such factor."""
    say("masked columns", dtype, tau, d_entropy)
    z = (torch.randn((4, 3001), generator=torch.Generator().manual_seed(1)) * 0.5).to(dtype)
    z[0, 2000:] = -INF
    z[1, :700] = torch.finfo(dtype).min
    z[2, ::2] = -3e4
    zd = z.to(gpu)
    t = torch.tensor([5, 800, 1, 7], dtype=torch.int32, device=gpu)
    s = D.token_logprobs(zd, t, 0, tau)
    one, de = torch.ones(4, device=gpu), torch.full((4,), d_entropy, device=gpu)
    for dl in (one, None):
        dz = D.token_logprobs_backward(zd, t, s["lse"], s["entropy"], dl, de, torch.empty_like(zd, dtype=F32), tau)
        assert not torch.isnan(dz).any()
        assert bool((dz[0, 2000:] == 0).all()) and bool((dz[1, :700] == 0).all()) and bool((dz[2, ::2] == 0).all())
