"""Clipping by factors that fp32 does not hold in full: the largest norms to the smallest
limits."""
import math

import pytest
import torch

import ops_ref as R
from paper_2506_20686_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


# the norm is about 71 std: factors of 1e-36 (24 bits of fp32), 1e-39 and 1e-42 (fewer), 1e-59
# (none) and 1e-33
@pytest.mark.parametrize("std,limit", [(1e20, 1e-14), (1e30, 1e-7), (1e33, 1e-7), (1e30, 1e-27),
                                       (1e34, 1e3)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_small_factors(std, limit, dtype):
    g = torch.Generator().manual_seed(3)
    t = [(torch.randn(n, generator=g) * std).to(dtype).to(DEV) for n in (5000, 13, 2)]
    ref = math.sqrt(sum((x.cpu().double() ** 2).sum().item() for x in t))
    norm = B.grad_norm(t)
    out = [torch.full_like(x, 5.0) for x in t]
    B.grad_clip(t, norm, limit, out)
    limit = torch.tensor(limit, dtype=torch.float32).double().item()
    for x, o in zip(t, out):
        # roundings of the norm, of the factor and of the product, and the result's own
        want = x.cpu().double() * (limit / ref)
        R.check("clipped", o, want, (R.HALF[dtype] + 3.1 * R.U) * want.abs())
    B.grad_clip(t, norm, limit)
    for x, o in zip(t, out):
        assert torch.equal(x, o)
