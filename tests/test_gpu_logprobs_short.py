"""Short rows on both sides of the choice between a warp and a block per row."""
import pytest
import torch

import paper_2504_09135_b200 as disc
from test_gpu_logprobs import _check, _logits

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,V,ld,offset,top", [
    (800, 1000, 1003, 5, 16), (800, 1024, 1024, 0, 1), (800, 301, 302, 1, 7), (800, 256, 256, 0, 64), (1000, 1000, 1000, 0, 0),      # warps
    (800, 1000, 1000, 0, 17), (600, 1000, 1003, 5, 16), (600, 100, 100, 0, 13), (30, 255, 255, 3, 64), (30, 1024, 1024, 0, 0)])        # blocks
def test_short_rows(dtype, n, V, ld, offset, top):
    z = _logits(n, V, dtype, n + V, ld, offset)
    z[3] = 0.0
    z[5] = -3.0
    z[5, V // 2] = 2.0
    t = torch.randint(-1, V, (n,), dtype=torch.int32, device=DEV)
    _check(z, t, top, 0.7, disc.disc_logprobs(z, t, top=top, inv_temperature=0.7))
