"""The linear projection with bias, activation and residual, and its backward,
through the C ABI against the plain 64-bit form (bounds in ops_ref.py)."""
import pytest
import torch

import ops_ref as R
from paper_2506_20686_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F4 = torch.bfloat16, torch.float32
ACTS = [B.ACT_NONE, B.ACT_RELU, B.ACT_GELU, B.ACT_SILU]


def inputs(m, k, n, dtype, seed):
    g = torch.Generator().manual_seed(seed)

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=g) * std).to(dtype)

    return {"x": normal(m, k), "w": normal(k, n, std=k ** -0.5), "bias": normal(n, std=0.3),
            "residual": normal(m, n, std=1.5), "z": normal(m, n, std=1.2), "dout": normal(m, n)}


def dev(t):
    return None if t is None else t.to(DEV)


def forward(t, act, bias=True, residual=True, save_z=True):
    b, r = (t["bias"] if bias else None), (t["residual"] if residual else None)
    out, z = B.linear_fwd(dev(t["x"]), dev(t["w"]), dev(b), dev(r), act, save_z)
    (ro, rz), (eo, ez) = R.lin_fwd(t["x"], t["w"], b, r, act)
    R.check("out", out, ro, eo)
    if save_z:
        R.check("z", z, rz, ez)
    else:
        assert z is None


def backward(t, act):
    z = t["z"] if act else None
    got = B.linear_bwd(dev(t["x"]), dev(t["w"]), dev(t["dout"]), dev(z), act)
    for name, a, r, e in zip(("dx", "dw", "dbias"), got,
                             *R.lin_bwd(t["x"], t["w"], t["dout"], z, act)):
        R.check(name, a, r, e)


# single rows and columns, every tile's whole and ragged multiples, odd sizes in each
# direction, long sums, few rows with wide outputs, many rows with narrow ones
SIZES = [(1, 1, 1), (1, 384, 1536), (2, 7, 3), (5, 128, 128), (16, 2048, 24), (17, 33, 65),
         (64, 64, 64), (100, 128, 128), (128, 256, 384), (129, 136, 72), (300, 449, 131),
         (257, 40, 200), (1000, 8, 8), (1500, 384, 520), (4001, 128, 128), (70, 1001, 16),
         (33, 16, 1000), (513, 130, 257), (8, 8192, 32), (8, 24, 8192), (2500, 1, 5),
         (90, 132, 68), (70, 20, 12), (301, 129, 128), (140, 128, 129), (260, 4, 300)]


@pytest.mark.parametrize("dtype", [BF, F4])
@pytest.mark.parametrize("m,k,n", SIZES)
def test_forward(m, k, n, dtype):
    t = inputs(m, k, n, dtype, m + k + n)
    forward(t, ACTS[(m + k + n) % 4])
    forward(t, B.ACT_NONE, bias=False, residual=False, save_z=False)


@pytest.mark.parametrize("dtype", [BF, F4])
@pytest.mark.parametrize("m,k,n", SIZES)
def test_backward(m, k, n, dtype):
    t = inputs(m, k, n, dtype, 7 * (m + k + n))
    backward(t, B.ACT_NONE)
    backward(t, ACTS[1 + (m + k + n) % 3])


@pytest.mark.parametrize("dtype", [BF, F4])
@pytest.mark.parametrize("m,k,n", [(1, 7, 130), (7, 1, 131), (130, 1, 7), (1, 130, 1), (2, 3, 129),
                                   (3, 2, 1), (5, 1, 300), (1, 1, 1001), (6, 1, 2), (2, 2, 3)])
def test_matrices_below_one_chunk(m, k, n, dtype):
    # a matrix of 1 to 7 elements, on each side, beside short and wide ones
    t = inputs(m, k, n, dtype, m + 3 * k + n)
    forward(t, B.ACT_SILU)
    backward(t, B.ACT_RELU)
    backward(t, B.ACT_GELU)


@pytest.mark.parametrize("dtype", [BF, F4])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("bias,residual,save_z", [(True, False, False), (False, True, True),
                                                  (True, True, False)])
def test_epilogues(act, bias, residual, save_z, dtype):
    forward(inputs(150, 96, 80, dtype, act), act, bias, residual, save_z)


@pytest.mark.parametrize("dtype", [BF, F4])
@pytest.mark.parametrize("act", ACTS)
def test_activation_gradients(act, dtype):
    t = inputs(333, 72, 88, dtype, 20 + act)
    # far out on both sides, at zero, and around the steepest places
    t["z"].view(-1)[:12] = torch.tensor([0.0, -0.0, 90.0, -90.0, 1e4, -1e4, 30.0, -30.0, 1.414,
                                         -1.414, 1e-20, -1e-20]).to(dtype)
    backward(t, act)


def test_activation_values_far_out():
    # x W alone gives z: 1 x 1 weights
    z = torch.tensor([[0.0], [100.0], [-100.0], [1e4], [-1e4], [12.0], [-12.0], [-6.0], [1e-20],
                      [-1e-20]])
    for dtype in (BF, F4):
        for act in ACTS:
            t = {"x": z.to(dtype), "w": torch.ones(1, 1, dtype=dtype)}
            out, _ = B.linear_fwd(dev(t["x"]), dev(t["w"]), act=act)
            (ro, _), (eo, _) = R.lin_fwd(t["x"], t["w"], None, None, act)
            # gelu's lower tail cancels: 1 + erf is good to U, times |z| / 2
            R.check("out", out, ro, eo + R.U * t["x"].to(R.F8).abs())


def test_small_and_large_magnitudes_fp32():
    # the fp32 products keep 24 bits over the whole range of exponents
    t = inputs(60, 50, 40, F4, 3)
    t["x"] *= torch.logspace(-18, 18, 60)[:, None]
    t["w"] *= torch.logspace(-9, 9, 40)[None, :]
    t["dout"] *= torch.logspace(9, -9, 40)[None, :] * torch.logspace(9, -9, 60)[:, None]
    forward(t, B.ACT_NONE, bias=False, residual=False)
    backward(t, B.ACT_NONE)


@pytest.mark.parametrize("dtype", [BF, F4])
@pytest.mark.parametrize("m,k,n", [(130, 128, 136), (37, 45, 51), (130, 128, 64), (77, 129, 140)])
def test_nothing_outside_the_outputs_is_written(m, k, n, dtype):
    t = {a: dev(b) for a, b in inputs(m, k, n, dtype, 5).items()}
    ref = (*B.linear_fwd(t["x"], t["w"], t["bias"], t["residual"], B.ACT_GELU, True),
           *B.linear_bwd(t["x"], t["w"], t["dout"], t["z"], B.ACT_GELU))
    pad = 64
    big = [torch.full((e + 2 * pad,), 7.0, dtype=d, device=DEV)
           for e, d in ((m * n, dtype), (m * n, dtype), (m * k, dtype), (k * n, F4), (n, F4))]
    at = [b.data_ptr() + pad * b.element_size() for b in big]
    code = B.BF16 if dtype == BF else B.F32
    need = B.tri_linear_bwd_workspace_bytes(code, m, k, n, B.ACT_GELU)
    ws = torch.full((need + 256,), 9, dtype=torch.uint8, device=DEV)
    s = torch.cuda.current_stream().cuda_stream
    p = {a: b.data_ptr() for a, b in t.items()}
    assert B.tri_linear_fwd(code, m, k, n, B.ACT_GELU, p["x"], p["w"], p["bias"], p["residual"],
                            at[0], at[1], s) == B.OK
    assert B.tri_linear_bwd(code, m, k, n, B.ACT_GELU, p["x"], p["w"], p["z"], p["dout"], at[2],
                            at[3], at[4], ws.data_ptr(), need, s) == B.OK
    for b, r in zip(big, ref):
        assert torch.equal(b[pad:-pad], r.reshape(-1))
        assert bool((b[:pad] == 7).all()) and bool((b[-pad:] == 7).all())
    assert bool((ws[need:] == 9).all())
    # each gradient by itself, and the output over the residual
    for keep in range(3):
        for b in big[2:]:
            b.fill_(7.0)
        args = [at[2 + i] if i == keep else None for i in range(3)]
        assert B.tri_linear_bwd(code, m, k, n, B.ACT_GELU, p["x"], p["w"], p["z"], p["dout"],
                                *args, ws.data_ptr(), need, s) == B.OK
        for i, b in enumerate(big[2:]):
            want = ref[2 + i].reshape(-1) if i == keep else torch.full_like(b[pad:-pad], 7.0)
            assert torch.equal(b[pad:-pad], want), (keep, i)
    r = t["residual"].clone()
    assert B.tri_linear_fwd(code, m, k, n, B.ACT_GELU, p["x"], p["w"], p["bias"], r.data_ptr(),
                            r.data_ptr(), None, s) == B.OK
    assert torch.equal(r, ref[0])


@pytest.mark.parametrize("dtype,act", [(BF, B.ACT_NONE), (BF, B.ACT_SILU), (F4, B.ACT_NONE)])
def test_bitwise_reproducible(dtype, act):
    t = {a: dev(b) for a, b in inputs(5000, 128, 132, dtype, 9).items()}
    z = t["z"] if act else None
    a, b = ((*B.linear_fwd(t["x"], t["w"], t["bias"], t["residual"], act, True),
             *B.linear_bwd(t["x"], t["w"], t["dout"], z, act)) for _ in range(2))
    for s, r in zip(a, b):
        assert torch.equal(s, r)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("m,k,n", [(40003, 128, 96), (33333, 77, 128), (70001, 5, 3),
                                   (20000, 40, 200), (9000, 300, 33)])
def test_many_rows(m, k, n, act):
    # several rounds of every workgroup: sampled rows of the row-wise results, and the sums
    # over rows by a dout that is zero elsewhere
    t = inputs(m, k, n, BF, 3 * m + act)
    rows = torch.unique(torch.cat([torch.arange(40), torch.arange(m - 40, m),
                                   torch.linspace(40, m - 41, 300).long()]))
    keep = torch.zeros(m, 1, dtype=BF)
    keep[rows] = 1
    t["dout"] = t["dout"] * keep
    z = t["z"] if act else None
    got = B.linear_bwd(dev(t["x"]), dev(t["w"]), dev(t["dout"]), dev(z), act)
    ref, bound = R.lin_bwd(t["x"][rows], t["w"], t["dout"][rows], z[rows] if act else None, act)
    R.check("dx", got[0][rows.to(DEV)], ref[0], bound[0])
    R.check("dw", got[1], ref[1], bound[1])
    R.check("dbias", got[2], ref[2], bound[2])
    assert int(torch.count_nonzero(got[0])) == int(torch.count_nonzero(got[0][rows.to(DEV)]))


def test_long_sum_over_rows():
    # 300,000 rows: dw and dbias stay fp32-accurate (random roundings of partial sums
    # grow as sqrt(m) U relative to the sum: 3.3e-5 / 100 in pieces of 30 rows and up)
    m, k, n = 300000, 32, 24
    t = inputs(m, k, n, BF, 31)
    got = B.linear_bwd(dev(t["x"]), dev(t["w"]), dev(t["dout"]))
    x, dy = t["x"].to(R.F8), t["dout"].to(R.F8)
    R.fro("dw", got[1], x.t() @ dy, 1e-5)
    R.fro("dbias", got[2], dy.sum(0), 1e-5)


def test_gradient_against_differences():
    t = inputs(4, 6, 5, F4, 13)
    for act in ACTS:
        z = B.linear_fwd(dev(t["x"]), dev(t["w"]), dev(t["bias"]), None, act, True)[1]
        got = [g.cpu().double() for g in B.linear_bwd(dev(t["x"]), dev(t["w"]), dev(t["dout"]),
                                                      z if act else None, act)]
        args, h = [t["x"].double(), t["w"].double(), t["bias"].double()], 1e-5

        def loss(x, w, b):
            return (R.act(x @ w + b, act) * t["dout"].double()).sum()

        for i, grad in enumerate(got):
            for at in range(args[i].numel()):
                v = []
                for sign in (1, -1):
                    p = [a.clone() for a in args]
                    p[i].view(-1)[at] += sign * h
                    v.append(loss(*p).item())
                assert abs((v[0] - v[1]) / (2 * h) - grad.reshape(-1)[at].item()) < 2e-5


def test_offsets_past_32_bits():
    m, k, n = (1 << 24) + 5, 8, 129  # 2.16e9 outputs, odd width
    g = torch.Generator(DEV).manual_seed(1)
    x = torch.randn(m, k, generator=g, device=DEV).to(BF)
    w = (torch.randn(k, n, generator=g, device=DEV) * 0.3).to(BF)
    out, _ = B.linear_fwd(x, w)
    rows = torch.tensor([0, 1, (1 << 24) - 1, m - 2, m - 1], device=DEV)
    (ro, _), (eo, _) = R.lin_fwd(x[rows].cpu(), w.cpu(), None, None, 0)
    R.check("out", out[rows], ro, eo)
    out.zero_()
    out[-3:] = 1.0  # dout nonzero in the last rows only: the sums over rows are theirs
    dx, dw, db = B.linear_bwd(x, w, out)
    t = slice(m - 3, m)
    ref, bound = R.lin_bwd(x[t].cpu(), w.cpu(), out[t].cpu(), None, 0)
    R.check("dx", dx[t], ref[0], bound[0])
    R.check("dw", dw, ref[1], bound[1])
    R.check("dbias", db, ref[2], bound[2])
    assert not bool(dx[:m - 3].any())
