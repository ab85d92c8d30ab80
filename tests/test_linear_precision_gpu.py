"""How many bits the linear projection keeps where its bf16 outputs or random
inputs would hide a loss: dz in the products of dx, the activations and their
derivatives in the tails (plain 64-bit forms in ops_ref.py)."""
import pytest
import torch

import ops_ref as R
from paper_2506_20686_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F4 = torch.bfloat16, torch.float32
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


def tail_points(limit):
    """z over both tails, dense around zero, in fp32."""
    g = torch.Generator().manual_seed(7)
    return torch.cat([torch.linspace(-limit, limit, 20001), torch.randn(9000, generator=g),
                      torch.randn(2000, generator=g) * 1e-3, torch.tensor([0.0, -0.0])])[:, None]


# e^(-z^2/2) and e^z stay above 2^-126 up to here, the least normal fp32
LIMIT = {B.ACT_GELU: 13.0, B.ACT_SILU: 87.0}


@pytest.mark.parametrize("act", [B.ACT_GELU, B.ACT_SILU], ids=NAMES.get)
def test_activation_values_in_the_tails_fp32(act):
    # one weight of 1: the product gives z itself.  Of the value: the exponential is good to
    # 4 roundings, the reciprocal to 2, the polynomial to 4, and there are 4 more products
    # and sums
    z = tail_points(LIMIT[act])
    out, back = B.linear_fwd(z.to(DEV), torch.ones(1, 1, device=DEV), act=act, save_z=True)
    assert torch.equal(back.cpu(), z)
    ref = R.act(z.to(R.F8), act)
    R.check("out", out, ref, 14 * R.U * ref.abs())


# dz formed in the staging, and made beforehand (k above 128)
@pytest.mark.parametrize("k", [1, 130])
@pytest.mark.parametrize("act", [B.ACT_GELU, B.ACT_SILU], ids=NAMES.get)
def test_activation_derivatives_in_the_tails_fp32(act, k):
    # one column of ones: dx is dz, and with dout = 1 act'(z), in whose two terms the value's
    # 14 roundings and those of a product and a sum enter (they cancel near its zero)
    z = tail_points(LIMIT[act])
    x = torch.zeros(z.shape[0], k)
    dx, _, db = B.linear_bwd(x.to(DEV), torch.ones(k, 1, device=DEV),
                             torch.ones(z.shape, device=DEV), z.to(DEV), act)
    zd = z.to(R.F8)
    ref = R.act_grad(zd, act)
    if act == B.ACT_GELU:
        parts = 0.5 * torch.erfc(-zd * R.SQRT_HALF) + (ref - 0.5 * torch.erfc(-zd * R.SQRT_HALF)).abs()
    else:
        parts = torch.sigmoid(zd) * (1 + zd.abs() * torch.sigmoid(-zd))
    bound = 17 * R.U * parts
    R.check("dx", dx, ref.expand(-1, k), bound.expand(-1, k))
    # and the sum over the rows, in any order
    R.check("dbias", db, ref.sum(0), bound.sum(0) + z.shape[0] * R.U * ref.abs().sum(0))


@pytest.mark.parametrize("m,k,n", [(300, 40, 24), (77, 33, 45)])
def test_least_magnitudes_fp32(m, k, n):
    # a value enters the products in three parts of 8 bits, the last of them no finer than
    # bf16's least subnormal, 2^-133: to 24 bits, or to 2^-134 where that is more (below
    # 2^-110); the other operand is scaled up, so that no result is itself that small
    g = torch.Generator().manual_seed(m)
    small = (torch.randn(m, k, generator=g) * torch.exp2(-95 - 35 * torch.rand(m, 1, generator=g)))
    big = torch.randn(k, n, generator=g) * 2.0 ** 60
    out, _ = B.linear_fwd(small.to(DEV), big.to(DEV))
    (ref, _), (e, _) = R.lin_fwd(small, big, None, None, 0)
    R.check("out", out, ref, e + 2.0 ** -134 * big.to(R.F8).abs().sum(0))
    # dx = dz W^T of small dz; dW = x^T dz of small x
    dx = B.linear_bwd(torch.zeros(m, n).to(DEV), big.t().contiguous().to(DEV), small.to(DEV))[0]
    (ref, _, _), (e, _, _) = R.lin_bwd(torch.zeros(m, n), big.t().contiguous(), small, None, 0)
    R.check("dx", dx, ref, e + 2.0 ** -134 * big.to(R.F8).abs().sum(0))
    dz = torch.randn(m, n, generator=g) * 2.0 ** 60
    dw = B.linear_bwd(small.to(DEV), torch.zeros(k, n).to(DEV), dz.to(DEV))[1]
    (_, ref, _), (_, e, _) = R.lin_bwd(small, torch.zeros(k, n), dz, None, 0)
    R.check("dw", dw, ref, e + 2.0 ** -134 * dz.to(R.F8).abs().sum(0))
