"""Layer norm at the widths where one lane adds the most values, against bounds
with the longest chain of additions that the kernel makes there."""
import pytest
import torch

import ops_ref as R
from paper_2506_20686_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F4 = torch.bfloat16, torch.float32


def chain(c, dtype):
    """Additions one after the other in a row's sum: a lane's elements (its 16-byte chunks of a
    row's, over 1, 4, 16, 64 or 256 lanes), then a step per halving of the lanes."""
    per = 16 // torch.empty(0, dtype=dtype).element_size()
    chunks = -(-c // per)
    lanes = 1 if chunks <= 4 else 4 if chunks <= 8 else 16 if chunks <= 64 else \
        64 if chunks <= 256 else 256
    return -(-chunks // lanes) * per + lanes.bit_length() - 1


@pytest.mark.parametrize("spread", [1.0, 0.01])
@pytest.mark.parametrize("dtype", [BF, F4])
@pytest.mark.parametrize("c", [16, 25, 32, 64, 200, 256, 449, 512, 1024, 1500, 2048, 4096, 6000, 8192])
def test_widths_of_long_chains(c, dtype, spread, monkeypatch):
    # values of one sign, whose partial sums grow at every addition
    g = torch.Generator().manual_seed(c)
    m = 67
    x = (3 + spread * torch.rand(m, c, generator=g)).to(dtype)
    gamma = (torch.rand(c, generator=g) + 0.5).to(dtype)
    beta = (torch.rand(c, generator=g)).to(dtype)
    dout = (torch.rand(m, c, generator=g) + 0.5).to(dtype)
    monkeypatch.setattr(R, "_chain", lambda width: chain(width, dtype))
    got = B.layer_norm_fwd(x.to(DEV), gamma.to(DEV), beta.to(DEV))
    for name, a, b, e in zip(("out", "mean", "rstd"), got, *R.ln_fwd(x, gamma, beta, 1e-5)):
        R.check(name, a, b, e)
    grads = B.layer_norm_bwd(x.to(DEV), gamma.to(DEV), got[1], got[2], dout.to(DEV))
    ref, bound = R.ln_bwd(x, gamma, got[1].cpu(), got[2].cpu(), dout)
    for name, a, b, e in zip(("dx", "dgamma", "dbeta"), grads, ref, bound):
        R.check(name, a, b, e)
