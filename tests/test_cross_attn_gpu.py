"""Cross attention through the C ABI against its plain 64-bit form (bounds in
cross_ref.py)."""
import math

import pytest
import torch

import cross_ref as C
import ops_ref as R
from paper_2506_20686_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F4 = torch.bfloat16, torch.float32


def dev(t):
    return None if t is None else t.to(DEV)


def inputs(b, nq, nk, h, hk, d, dtype, bias="none", mask=False, seed=0):
    g = torch.Generator().manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g).to(dtype)

    q, k, v, dout = normal(b, nq, h, d), normal(b, nk, hk, d), normal(b, nk, hk, d), \
        normal(b, nq, h, d)
    x = {"none": None, "shared": normal(nq, nk, h), "each": normal(b, nq, nk, h)}[bias]
    m = None
    if mask:  # holes anywhere, one key at least
        m = (torch.rand(b, nk, generator=g) < 0.6).to(torch.uint8)
        m[torch.arange(b), torch.randint(nk, (b,), generator=g)] = 1
    return q, k, v, x, m, dout


def both(q, k, v, bias, mask, dout, scale=None):
    q_, k_, v_, x, m, y = (dev(t) for t in (q, k, v, bias, mask, dout))
    out, stat = B.cross_attn_fwd(q_, k_, v_, x, m, scale)
    for name, a, r, e in zip(("out", "stat"), (out, stat), *C.attn_fwd(q, k, v, bias, mask, scale)):
        R.check(name, a, r, e)
    grads = B.cross_attn_bwd(q_, k_, v_, out, stat, y, x, m, scale)
    ref, bound = C.attn_bwd(q, k, v, dout, bias, mask, scale)
    for name, a, r, e in zip(("dq", "dk", "dv", "dbias"), grads, ref, bound):
        if r is None:
            assert a is None
        else:
            R.check(name, a, r, e)
    return (out, stat, *grads)


# one query and one key; around the 32-row and the 32- and 64-key tiles; every padded
# width of the channels and odd eights; shared key heads; few queries to many keys and the
# other way (loops that are split)
SIZES = [(1, 1, 1, 1, 1, 8), (1, 1, 1, 2, 1, 16), (2, 7, 33, 4, 4, 32), (1, 33, 31, 3, 3, 24),
         (2, 130, 65, 4, 2, 48), (1, 64, 64, 2, 2, 64), (3, 1, 700, 8, 2, 64),
         (1, 5, 2100, 8, 1, 16), (2, 300, 20, 4, 4, 40), (1, 129, 257, 2, 1, 128),
         (1, 40, 100, 2, 2, 96), (1, 700, 90, 1, 1, 72), (5, 32, 128, 4, 4, 32),
         (2, 11, 32, 6, 2, 8), (1, 1500, 3, 2, 2, 32), (1, 3, 1500, 1, 1, 128),
         (2, 1, 130, 7, 1, 56), (1, 97, 640, 5, 5, 24), (1, 45, 70, 16, 16, 24),
         (3, 50, 40, 8, 8, 64), (1, 1, 1, 4, 4, 8), (1, 300, 420, 4, 4, 32),
         (2, 70, 500, 4, 4, 56), (1, 290, 33, 4, 4, 128), (1, 20, 9000, 2, 2, 32)]


@pytest.mark.parametrize("dtype", [BF, F4])
@pytest.mark.parametrize("bias,mask", [("none", False), ("shared", True), ("each", False)])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_forward_and_backward(size, bias, mask, dtype):
    both(*inputs(*size, dtype, bias, mask, seed=sum(size)))


@pytest.mark.parametrize("dtype", [BF, F4])
def test_mask_without_bias_and_scale(dtype):
    both(*inputs(2, 70, 150, 4, 2, 32, dtype, "none", True, seed=5), scale=1.3)


@pytest.mark.parametrize("dtype", [BF, F4])
@pytest.mark.parametrize("bias,hk", [("none", 2), ("each", 2), ("each", 4), ("shared", 4)])
def test_nothing_masked_has_an_effect(dtype, bias, hk):
    q, k, v, x, m, y = inputs(2, 70, 100, 4, hk, 32, dtype, bias, True, seed=7)
    if bias == "shared":
        m[1] = m[0]
    want = both(q, k, v, x, m, y)
    off = (m == 0)
    for value in (math.nan, math.inf, -math.inf):
        k2, v2 = k.clone(), v.clone()
        k2[off], v2[off] = value, value
        x2 = None if x is None else x.clone()
        if x2 is not None:
            if bias == "shared":
                x2.permute(1, 0, 2)[off[0]] = value
            else:
                x2.permute(0, 2, 1, 3)[off] = value
        out, stat = B.cross_attn_fwd(dev(q), dev(k2), dev(v2), dev(x2), dev(m))
        got = (out, stat, *B.cross_attn_bwd(dev(q), dev(k2), dev(v2), out, stat, dev(y), dev(x2),
                                            dev(m)))
        for a, b in zip(got, want):
            assert (a is None and b is None) or torch.equal(a, b)
    assert not bool(want[3].cpu()[off].any()) and not bool(want[4].cpu()[off].any())


@pytest.mark.parametrize("dtype", [BF, F4])
@pytest.mark.parametrize("nk", [5, 40, 700])
def test_rows_without_a_key(dtype, nk):
    # the first sample has no valid key; in the second a bias of -inf leaves queries 1
    # and 4 none, and takes single keys from the others
    q, k, v, x, m, y = inputs(2, 37, nk, 4, 4, 32, dtype, "each", True, seed=nk)
    m[0] = 0
    x[1, 1], x[1, 4] = -math.inf, -math.inf
    x[1, :, 2, 1] = -math.inf
    m[1, 0] = 1
    args = [dev(t) for t in (q, k, v)]
    out, stat = B.cross_attn_fwd(*args, dev(x), dev(m))
    (ro, rs), (eo, es) = C.attn_fwd(q, k, v, x, m)
    R.check("out", out, ro, eo)
    empty = rs[..., 0] == -math.inf
    assert bool(empty[0].all()) and bool(empty[1, 1].all()) and bool(empty[1, 4].all())
    got = stat.cpu()
    assert bool((got[..., 0][empty] == -math.inf).all()) and not bool(got[..., 1][empty].any())
    R.check("stat", got[~empty], rs[~empty], es[~empty])
    grads = B.cross_attn_bwd(*args, out, stat, dev(y), dev(x), dev(m))
    for a, r, e in zip(grads, *C.attn_bwd(q, k, v, y, x, m)):
        R.check("gradient", a, r, torch.where(e.isfinite(), e, torch.zeros_like(e)))
    assert not bool(grads[0].cpu()[empty].any()) and not bool(grads[1][0].any())


@pytest.mark.parametrize("dtype", [BF, F4])
@pytest.mark.parametrize("nk", [6, 100, 900])
def test_bias_of_the_types_lowest_value(dtype, nk):
    # query 0: every key at the lowest value, which takes the logits whole, so that all
    # weigh alike; query 1: half of the keys
    q, k, v, _, _, y = inputs(1, 3, nk, 2, 2, 32, dtype, seed=nk)
    x = torch.zeros(3, nk, 2, dtype=dtype)
    x[0] = torch.finfo(dtype).min
    x[1, ::2] = torch.finfo(dtype).min
    out, stat = B.cross_attn_fwd(dev(q), dev(k), dev(v), dev(x))
    lowest = torch.finfo(dtype).min
    assert bool((stat[0, 0, :, 0].cpu().double() == lowest).all())
    n = torch.log(torch.tensor(float(nk), dtype=R.F8))
    assert torch.allclose(stat[0, 0, :, 1].cpu().double(), n, rtol=(nk + 8) * R.U)
    half = R.HALF[dtype]
    mean = v[0].double().mean(0)
    # P is 1 (exact in any type), the sums those of nk terms
    bound = half * mean.abs() + (2 * nk + 20) * R.U * v[0].double().abs().mean(0)
    R.check("out", out[0, 0], mean, bound)
    m = torch.ones(1, nk, dtype=torch.uint8)
    m[0, ::2] = 0
    r, e = C.attn_fwd(q[:, 1:2], k, v, None, m)
    R.check("out", out[:, 1:2], r[0], e[0])
    dq, dk, dv, db = B.cross_attn_bwd(dev(q), dev(k), dev(v), out, stat, dev(y), dev(x))
    p = 1.0 / nk
    dp = torch.einsum("hc,khc->hk", y[0, 0].double(), v[0].double())
    ds = p * (dp - dp.mean(1, keepdim=True))
    mag = torch.einsum("hc,khc->hk", y[0, 0].double().abs(), v[0].double().abs())
    scale = 1 / math.sqrt(32)
    R.check("dbias", db[0], ds.t(), half * ds.t().abs() + (
        (2 * 36 + 4 * nk + 60) * R.U * p * (mag + mag.mean(1, keepdim=True))).t())
    want = scale * torch.einsum("hk,khc->hc", ds, k[0].double())
    # dS' (shifted by the rounding of out) and P = 1 / nk rounded for the products
    shift = 2 * half * (y[0, 0].double().abs() * v[0].double().abs().mean(0)).sum(1)
    size = ds.abs() + p * shift[:, None] + (4 * nk + 200) * R.U * p * mag
    hp = half if dtype == BF else 2 * (nk + 16) * R.U
    R.check("dq", dq[0, 0], want, half * want.abs() + 2.1 * scale * torch.einsum(
        "hk,khc->hc", hp * size + (4 * nk + 200) * R.U * p * mag, k[0].double().abs()))


@pytest.mark.parametrize("dtype", [BF, F4])
def test_one_valid_key_has_no_gradient_of_the_logits(dtype):
    for nk, at in ((1, 0), (90, 77)):
        q, k, v, x, _, y = inputs(2, 50, nk, 4, 2, 32, dtype, "shared", seed=nk)
        m = torch.zeros(2, nk, dtype=torch.uint8)
        m[:, at] = 1
        out, stat = B.cross_attn_fwd(dev(q), dev(k), dev(v), dev(x), dev(m))
        want = v[:, at].repeat_interleave(2, dim=1)[:, None].expand(-1, 50, -1, -1)
        assert torch.equal(out.cpu(), want)
        dq, dk, dv, db = B.cross_attn_bwd(dev(q), dev(k), dev(v), out, stat, dev(y), dev(x), dev(m))
        assert not bool(dq.any()) and not bool(dk.any()) and not bool(db.any())
        both(q, k, v, x, m, y)


def test_sharp_weights():
    # logits far apart: one key takes nearly all of a row
    q, k, v, x, m, y = inputs(1, 70, 200, 4, 4, 64, BF, "each", True, seed=3)
    both((q * 6).to(BF), k, v, x, m, y)
    both((q * 6).to(BF), k, v, None, None, y)


@pytest.mark.parametrize("dtype", [BF, F4])
@pytest.mark.parametrize("size", [(2, 37, 70, 4, 2, 24), (1, 3, 900, 4, 1, 64), (1, 900, 5, 2, 2, 8),
                                  (2, 37, 70, 8, 8, 24), (1, 300, 420, 4, 4, 32)],
                         ids=str)
def test_nothing_outside_the_outputs_is_written(size, dtype):
    b, nq, nk, h, hk, d = size
    q, k, v, x, m, y = (dev(t) for t in inputs(*size, dtype, "each", True, seed=1))
    ref = B.cross_attn_fwd(q, k, v, x, m)
    ref += B.cross_attn_bwd(q, k, v, *ref, y, x, m)
    pad, code = 64, B.BF16 if dtype == BF else B.F32
    big = [torch.full((t.numel() + 2 * pad,), 7.0, dtype=t.dtype, device=DEV) for t in ref]
    at = [t.data_ptr() + pad * t.element_size() for t in big]
    sizes = (code, b, nq, nk, h, hk, d, b)
    s, scale = torch.cuda.current_stream().cuda_stream, 1 / math.sqrt(d)
    L, ws = B.lib(), []
    for name in ("fwd", "bwd"):
        need = B._sized(f"tri_cross_attn_{name}_workspace_bytes", *sizes)
        ws.append((torch.full((need + 256,), 9, dtype=torch.uint8, device=DEV), need))
    ins = [t.data_ptr() for t in (q, k, v, x, m)]
    assert L.tri_cross_attn_fwd(*sizes, scale, *ins, at[0], at[1], ws[0][0].data_ptr(), ws[0][1],
                                s) == B.OK
    assert L.tri_cross_attn_bwd(*sizes, scale, *ins, at[0], at[1], y.data_ptr(), *at[2:],
                                ws[1][0].data_ptr(), ws[1][1], s) == B.OK
    for t, r in zip(big, ref):
        assert torch.equal(t[pad:-pad], r.reshape(-1))
        assert bool((t[:pad] == 7).all()) and bool((t[-pad:] == 7).all())
    for w, need in ws:
        assert bool((w[need:] == 9).all())
    # without dbias: the others are the same
    for t in big[2:]:
        t.fill_(7.0)
    assert L.tri_cross_attn_bwd(*sizes, scale, *ins, at[0], at[1], y.data_ptr(), *at[2:5], None,
                                ws[1][0].data_ptr(), ws[1][1], s) == B.OK
    for t, r in zip(big[2:5], ref[2:5]):
        assert torch.equal(t[pad:-pad], r.reshape(-1))
    assert bool((big[5] == 7).all())


def test_unbatched_and_bitwise_reproducible():
    for size in ((1, 300, 500, 4, 2, 32), (1, 2, 3000, 4, 4, 64)):
        q, k, v, x, m, y = (dev(t) for t in inputs(*size, BF, "shared", True, seed=2))
        one = B.cross_attn_fwd(q, k, v, x, m)
        one += B.cross_attn_bwd(q, k, v, *one, y, x, m)
        two = B.cross_attn_fwd(q[0], k[0], v[0], x, m[0])
        two += B.cross_attn_bwd(q[0], k[0], v[0], *two, y[0], x, m[0])
        for a, c in zip(one, two):
            assert torch.equal(a.reshape(-1), c.reshape(-1))


def test_gradients_against_differences():
    # L = sum(dout out) in fp32 against central differences of the 64-bit form
    q, k, v, x, m, y = inputs(1, 3, 4, 2, 1, 8, F4, "shared", True, seed=11)
    out, stat = B.cross_attn_fwd(dev(q), dev(k), dev(v), dev(x), dev(m))
    grads = B.cross_attn_bwd(dev(q), dev(k), dev(v), out, stat, dev(y), dev(x), dev(m))
    args, h = [t.double() for t in (q, k, v, x)], 1e-5

    def loss(a):
        s = torch.einsum("qhc,kc->hqk", a[0][0], a[1][0, :, 0]) / math.sqrt(8)
        s = s + a[3].permute(2, 0, 1)
        s = s.masked_fill(m[0] == 0, -math.inf)
        return (torch.einsum("hqk,kc->qhc", torch.softmax(s, 2), a[2][0, :, 0]) * y[0].double()).sum()

    for i, grad in enumerate(grads):
        for at in range(args[i].numel()):
            pair = []
            for sign in (1, -1):
                p = [t.clone() for t in args]
                p[i].view(-1)[at] += sign * h
                pair.append(loss(p).item())
            # differences: third derivative times h^2 and 64-bit rounding over h; fp32
            assert abs((pair[0] - pair[1]) / (2 * h) - grad.reshape(-1)[at].item()) < 2e-5


def test_offsets_past_32_bits():
    b, nq, nk, h, d = 9, 3, 131072, 16, 128  # 2.4e9 elements of k
    g = torch.Generator(DEV).manual_seed(1)
    k, v = (torch.empty(b, nk, h, d, dtype=BF, device=DEV) for _ in range(2))
    for t in (k, v):
        for i in range(b):
            t[i].normal_(generator=g)
    q, y = (torch.randn(b, nq, h, d, generator=g, device=DEV).to(BF) for _ in range(2))
    mask = torch.zeros(b, nk, dtype=torch.uint8, device=DEV)
    mask[:, -70:] = 1
    out, stat = B.cross_attn_fwd(q, k, v, None, mask)
    dq, dk, dv, _ = B.cross_attn_bwd(q, k, v, out, stat, y, None, mask)
    last = [t[-1:].cpu() for t in (q, y)] + [t[-1:, -70:].cpu() for t in (k, v)]
    (ro, rs), (eo, es) = C.attn_fwd(last[0], last[2], last[3])
    R.check("out", out[-1:], ro, eo)
    R.check("stat", stat[-1:], rs, es)
    ref, bound = C.attn_bwd(last[0], last[2], last[3], last[1])
    for a, r, e in zip((dq[-1:], dk[-1:, -70:], dv[-1:, -70:]), ref, bound):
        R.check("gradient", a, r, e)
    assert not bool(dk[-1, :-70].any()) and not bool(dv[0, :-70].any())
