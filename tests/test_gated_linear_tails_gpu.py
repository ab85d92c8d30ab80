"""Gated linear projection: derivatives of the sigmoid and of silu where one side of the
sigmoid is next to 1, through the gradient of the bias.

x is 1 in one channel, so that z is a bf16 of W exactly; b and dout are 1; and one row's
dbias is dz itself.  The 32-bit roundings, U each: exp(-|z|) is an exponential in base 2 (one
step, 2 U) of a product by log2(e), rounded twice (2 |z| U); 1 + e; a reciprocal (2 U); the
product that makes the small side; the derivative's own; two factors of 1 and the planes of dz.
Both sides of the sigmoid stay within (2 |z| + 8) U of themselves, its derivative within (2 |z| +
20) U; silu's, p (1 + z q), within (4 |z| + 24) U of p (1 + |z| q)."""
import pytest
import torch

import ops_ref as R
from paper_2506_20686_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F4 = torch.bfloat16, torch.float32


# rows of 128 + 128 channels; whole words; ragged; enough tiles for the 128-wide ones
@pytest.mark.parametrize("m,k,f", [(1, 8, 128), (1, 8, 64), (1, 16, 200), (1, 7, 133), (1, 8, 3),
                                   (33000, 136, 128)])
@pytest.mark.parametrize("dtype", [BF, F4])
@pytest.mark.parametrize("act", [B.ACT_SIGMOID, B.ACT_SILU])
def test_derivatives_far_out(m, k, f, act, dtype):
    z = torch.linspace(-30, 30, f).to(BF)  # bf16 values in either type
    x = torch.zeros(m, k, dtype=dtype)
    x[0, 0] = 1
    w = torch.zeros(k, 2 * f, dtype=dtype)
    w[0, :f] = z.to(dtype)
    w[0, f:] = 1
    dy = torch.zeros(m, f, dtype=dtype)
    dy[0] = 1
    _, _, db = B.gated_linear_bwd(x.to(DEV), w.to(DEV), dy.to(DEV), None, act)
    z = z.double()
    p, q = torch.sigmoid(z), torch.sigmoid(-z)
    if act == B.ACT_SIGMOID:
        slope, value = p * q, p
        bound = (2 * z.abs() + 20) * R.U * slope
    else:
        slope, value = p * (1 + z * q), z * p
        bound = (4 * z.abs() + 24) * R.U * p * (1 + z.abs() * q)
    R.check("da", db[:f], slope, bound)
    R.check("db", db[f:], value, (2 * z.abs() + 20) * R.U * value.abs())
