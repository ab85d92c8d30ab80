"""Layer norm through the C ABI against its plain 64-bit form (bounds in ops_ref.py)."""
import pytest
import torch

import ops_ref as R
from paper_2506_20686_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F4 = torch.bfloat16, torch.float32


def inputs(m, c, dtype, seed, affine=True, shift=0.3):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(m, c, generator=g) * 1.5 + shift).to(dtype)
    gamma = (torch.randn(c, generator=g) * 0.2 + 1).to(dtype) if affine else None
    beta = (torch.randn(c, generator=g) * 0.2).to(dtype) if affine else None
    dout = torch.randn(m, c, generator=g).to(dtype)
    return x, gamma, beta, dout


def dev(t):
    return None if t is None else t.to(DEV)


def both(m, c, dtype, seed=0, eps=1e-5, **kw):
    x, gamma, beta, dout = inputs(m, c, dtype, seed, **kw)
    got = B.layer_norm_fwd(dev(x), dev(gamma), dev(beta), eps)
    for name, a, b, e in zip(("out", "mean", "rstd"), got, *R.ln_fwd(x, gamma, beta, eps)):
        R.check(name, a, b, e)
    mean, rstd = got[1], got[2]
    grads = B.layer_norm_bwd(dev(x), dev(gamma), mean, rstd, dev(dout))
    ref, bound = R.ln_bwd(x, gamma, mean.cpu(), rstd.cpu(), dout)
    for name, a, b, e in zip(("dx", "dgamma", "dbeta"), grads, ref, bound):
        R.check(name, a, b, e)


# one row and one column, whole and ragged multiples of every vector and lane count,
# odd widths, the widest rows, many short rows (several rounds of the grid)
SIZES = [(1, 1), (1, 8192), (3, 7), (5, 8), (64, 128), (65, 129), (1000, 384), (517, 833),
         (33, 1024), (20, 1025), (9, 2049), (6, 2056), (5, 4096), (4, 8191), (2999, 128),
         (40007, 16), (70, 3), (300, 640), (31, 250), (4099, 56)]


@pytest.mark.parametrize("dtype", [BF, F4])
@pytest.mark.parametrize("m,c", SIZES)
def test_forward_and_backward(m, c, dtype):
    both(m, c, dtype, seed=m + c)


@pytest.mark.parametrize("dtype", [BF, F4])
def test_without_weights(dtype):
    both(77, 384, dtype, affine=False)
    both(50, 33, dtype, affine=False)


def test_one_weight_of_the_two():
    x, gamma, beta, _ = inputs(40, 128, F4, 3)
    for g, b in ((gamma, None), (None, beta)):
        got = B.layer_norm_fwd(dev(x), dev(g), dev(b))
        for a, r, e in zip(got, *R.ln_fwd(x, g, b, 1e-5)):
            R.check("one weight", a, r, e)


def test_rows_far_from_zero():
    # a mean 1000 times the deviation: the deviations are taken from the mean, not
    # from a difference of squares
    both(64, 200, F4, shift=1500.0)


def test_constant_and_zero_rows():
    x = torch.zeros(8, 128)
    x[1::2] = 3.0
    out, mean, rstd = B.layer_norm_fwd(dev(x))
    assert torch.equal(out.cpu(), torch.zeros(8, 128))
    assert torch.equal(mean.cpu(), x[:, 0])
    assert torch.allclose(rstd.cpu(), torch.full((8,), 1e-5).rsqrt(), rtol=4 * R.U)


@pytest.mark.parametrize("dtype", [BF, F4])
@pytest.mark.parametrize("c", [128, 833, 4096])
def test_nothing_outside_the_outputs_is_written(dtype, c):
    m, pad = 37, 64
    x, gamma, beta, dout = (dev(t) for t in inputs(m, c, dtype, 5))
    ref, rb = B.layer_norm_fwd(x, gamma, beta), None
    rb = B.layer_norm_bwd(x, gamma, ref[1], ref[2], dout)
    big = [torch.full((n + 2 * pad,), 7.0, dtype=t, device=DEV)
           for n, t in ((m * c, dtype), (m, F4), (m, F4), (m * c, dtype), (c, F4), (c, F4))]
    at = [t.data_ptr() + pad * t.element_size() for t in big]
    code = B.BF16 if dtype == BF else B.F32
    need = B.tri_layer_norm_bwd_workspace_bytes(code, m, c)
    ws = torch.full((need + 256,), 9, dtype=torch.uint8, device=DEV)
    s = torch.cuda.current_stream().cuda_stream
    assert B.tri_layer_norm_fwd(code, m, c, 1e-5, x.data_ptr(), gamma.data_ptr(), beta.data_ptr(),
                                at[0], at[1], at[2], s) == B.OK
    assert B.tri_layer_norm_bwd(code, m, c, x.data_ptr(), gamma.data_ptr(), at[1], at[2],
                                dout.data_ptr(), at[3], at[4], at[5], ws.data_ptr(), need,
                                s) == B.OK
    for t, r in zip(big, (*ref, *rb)):
        assert torch.equal(t[pad:-pad], r.reshape(-1))
        assert bool((t[:pad] == 7).all()) and bool((t[-pad:] == 7).all())
    assert bool((ws[need:] == 9).all())


@pytest.mark.parametrize("c", [128, 833])
def test_in_place_and_without_weight_gradients(c):
    m = 100
    x, gamma, beta, dout = (dev(t) for t in inputs(m, c, BF, 6))
    out, mean, rstd = B.layer_norm_fwd(x, gamma, beta)
    dx, dg, db = B.layer_norm_bwd(x, gamma, mean, rstd, dout)
    s = torch.cuda.current_stream().cuda_stream
    y, d = x.clone(), dout.clone()
    assert B.tri_layer_norm_fwd(B.BF16, m, c, 1e-5, y.data_ptr(), gamma.data_ptr(),
                                beta.data_ptr(), y.data_ptr(), mean.data_ptr(), rstd.data_ptr(),
                                s) == B.OK
    assert torch.equal(y, out)
    # no weight gradients: no workspace; dx over dout
    assert B.tri_layer_norm_bwd(B.BF16, m, c, x.data_ptr(), gamma.data_ptr(), mean.data_ptr(),
                                rstd.data_ptr(), d.data_ptr(), d.data_ptr(), None, None, None, 0,
                                s) == B.OK
    assert torch.equal(d, dx)
    # one of the two, dx over dout again
    d, only = dout.clone(), torch.zeros(c, device=DEV)
    ws = torch.empty(B.tri_layer_norm_bwd_workspace_bytes(B.BF16, m, c), dtype=torch.uint8,
                     device=DEV)
    assert B.tri_layer_norm_bwd(B.BF16, m, c, x.data_ptr(), gamma.data_ptr(), mean.data_ptr(),
                                rstd.data_ptr(), d.data_ptr(), d.data_ptr(), None,
                                only.data_ptr(), ws.data_ptr(), ws.numel(), s) == B.OK
    assert torch.equal(d, dx) and torch.equal(only, db)
    only.zero_()
    assert B.tri_layer_norm_bwd(B.BF16, m, c, x.data_ptr(), gamma.data_ptr(), mean.data_ptr(),
                                rstd.data_ptr(), dout.data_ptr(), d.data_ptr(), only.data_ptr(),
                                None, ws.data_ptr(), ws.numel(), s) == B.OK
    assert torch.equal(only, dg)


@pytest.mark.parametrize("dtype,c", [(BF, 128), (F4, 129), (BF, 5000)])
def test_bitwise_reproducible(dtype, c):
    x, gamma, beta, dout = (dev(t) for t in inputs(3001, c, dtype, 8))
    _, mean, rstd = B.layer_norm_fwd(x, gamma, beta)
    a, b = (B.layer_norm_bwd(x, gamma, mean, rstd, dout) for _ in range(2))
    for s, t in zip(a, b):
        assert torch.equal(s, t)


def test_gradient_against_differences():
    # L = sum(dout out) in fp32 against central differences of the 64-bit form
    x, gamma, beta, dout = inputs(3, 9, F4, 11)
    _, mean, rstd = B.layer_norm_fwd(dev(x), dev(gamma), dev(beta))
    dx, dg, db = (t.cpu().double() for t in B.layer_norm_bwd(dev(x), dev(gamma), mean, rstd,
                                                            dev(dout)))

    def loss(x, g, b):
        xd = x - x.mean(1, keepdim=True)
        out = xd / torch.sqrt((xd * xd).mean(1, keepdim=True) + 1e-5) * g + b
        return (out * dout.double()).sum()

    args, h = [x.double(), gamma.double(), beta.double()], 1e-5
    for i, grad in enumerate((dx, dg, db)):
        for at in range(args[i].numel()):
            v = []
            for sign in (1, -1):
                p = [t.clone() for t in args]
                p[i].view(-1)[at] += sign * h
                v.append(loss(*p))
            # differences: third derivative times h^2 and 64-bit rounding over h
            assert abs((v[0] - v[1]).item() / (2 * h) - grad.reshape(-1)[at].item()) < 1e-5


def test_offsets_past_32_bits():
    m, c = (1 << 24) + 5, 129  # 2.16e9 elements, odd width
    g = torch.Generator(DEV).manual_seed(1)
    x = torch.empty(m, c, dtype=BF, device=DEV)
    for a in range(0, m, 1 << 21):
        x[a:a + (1 << 21)].normal_(generator=g)
    out, mean, rstd = B.layer_norm_fwd(x)
    rows = torch.tensor([0, 1, (1 << 24) - 1, m - 2, m - 1], device=DEV)
    (ro, rm, rr), (eo, em, er) = R.ln_fwd(x[rows].cpu(), None, None, 1e-5)
    R.check("out", out[rows], ro, eo)
    R.check("mean", mean[rows], rm, em)
    # backward with dout nonzero in the last rows only: the sums over rows are theirs
    dout = torch.zeros_like(x)
    dout[-3:] = 1.0
    dx, dg, db = B.layer_norm_bwd(x, None, mean, rstd, dout)
    t = slice(m - 3, m)
    ref, bound = R.ln_bwd(x[t].cpu(), None, mean[t].cpu(), rstd[t].cpu(), dout[t].cpu())
    R.check("dx", dx[t], ref[0], bound[0])
    R.check("dgamma", dg, ref[1], bound[1])
    R.check("dbeta", db, ref[2], bound[2])
    assert not bool(dx[:5].any()) and not bool(dx[(1 << 24) - 9:m - 3].any())
