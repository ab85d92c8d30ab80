"""How many bits the linear projection keeps where its bf16 outputs or random
inputs would hide a loss (plain 64-bit forms in ops_ref.py)."""
import pytest
import torch

import ops_ref as R
from paper_2506_20686_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16
NAMES = {B.ACT_GELU: "gelu", B.ACT_SILU: "silu"}


# the one-pass kernel of narrow projections, whole and ragged; dz formed in the staging
# (k up to 128) in tiles of 64 and of 128; dz made beforehand, the same, whole and ragged
@pytest.mark.parametrize("m,k,n", [(4096, 8, 8), (4096, 3, 2), (2000, 128, 136), (33000, 128, 136),
                                   (1024, 136, 8), (1024, 137, 6), (16500, 136, 8),
                                   (16500, 137, 130)])
@pytest.mark.parametrize("act", [B.ACT_GELU, B.ACT_SILU], ids=NAMES.get)
def test_dx_takes_dz_in_24_bits(m, k, n, act):
    # every dx is the difference of two dz of one dout at neighbouring z, so small that its own
    # rounding hides nothing of their low bits
    g = torch.Generator().manual_seed(m + k + n)
    h = (n + 1) // 2
    z = torch.exp2(-9 + 3 * torch.rand(m, h, generator=g))
    z = (z * torch.where(torch.rand(m, h, generator=g) < 0.5, -1.0, 1.0)).to(BF)
    near = (z.view(torch.int16) ^ 1).view(BF)
    z = torch.stack([z, near], 2).view(m, 2 * h)[:, :n].contiguous()
    dout = (1 + torch.rand(m, h, generator=g)).to(BF).repeat_interleave(2, 1)[:, :n].contiguous()
    pair = torch.arange(k) % (n // 2)
    w = torch.zeros(k, n, dtype=BF)
    w[torch.arange(k), 2 * pair], w[torch.arange(k), 2 * pair + 1] = 1, -1
    x = torch.zeros(m, k, dtype=BF)
    dx = B.linear_bwd(*(t.to(DEV) for t in (x, w, dout, z)), act)[0]
    dy = dout.to(R.F8)
    dz = dy * R.act_grad(z.to(R.F8), act)
    # at z this small act' is 0.5 and a little: its value is off by at most 8 roundings of 1,
    # and dz by that times dout.  The other terms of a sum are zeros, which add nothing; of a
    # dz's three parts only the first is of its size, so three partial sums are, each rounded
    # twice at most.  (In 16 bits a dz is off by up to 2^-18, 64 roundings.)
    a = 2 * pair
    ref = dz[:, a] - dz[:, a + 1]
    e = 2 * 8 * R.U * dy[:, a] + 6 * R.U * torch.maximum(dz[:, a], dz[:, a + 1])
    R.check("dx", dx, ref, R.HALF[BF] * ref.abs() + 1.01 * e)
