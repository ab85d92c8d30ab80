"""Cross attention through the C ABI: one valid key in loops that are split; many samples with
a bias map each, or one for all (bounds in cross_ref.py)."""
import pytest
import torch

import cross_ref as C
import ops_ref as R
from paper_2506_20686_amd import binding as B
from test_cross_attn_gpu import DEV, BF, F4, both, dev, inputs

pytestmark = pytest.mark.gpu


# (queries, keys, heads, key heads): loops of 2 to 8 splits; tiles shared by four waves, a
# wave's own in groups of four, and four heads side by side in groups of two
@pytest.mark.parametrize("dtype", [BF, F4])
@pytest.mark.parametrize("bias", ["none", "shared", "each"])
@pytest.mark.parametrize("nq,nk,h,hk", [(50, 900, 4, 2), (50, 2100, 4, 2), (50, 2100, 4, 4),
                                        (5, 2100, 4, 2), (3, 1500, 1, 1)])
def test_one_valid_key_of_split_loops(nq, nk, h, hk, bias, dtype):
    # samples of one valid key in the first, a middle and the last split; of two keys in
    # different splits, which have gradients; of none
    q, k, v, x, _, y = inputs(5, nq, nk, h, hk, 32, dtype, bias, seed=nk + nq)
    one = (3, nk // 2 + 1, nk - 1)
    m = torch.zeros(5, nk, dtype=torch.uint8)
    for b, at in enumerate(one):
        m[b, at] = 1
    m[3, 1] = m[3, nk - 2] = 1
    out, stat = B.cross_attn_fwd(dev(q), dev(k), dev(v), dev(x), dev(m))
    # P is exp2 of the rounding of s c alone, 1 up to that, and out = (v P) (1 / P): the product
    # by matrix instructions (2 U), the reciprocal and the product (U each), out's own rounding
    for b, at in enumerate(one):
        want = v[b, at].repeat_interleave(h // hk, dim=0)[None].expand(nq, -1, -1).double()
        R.check("out", out[b], want, (R.HALF[dtype] + 4.1 * R.U) * want.abs())
    dq, dk, dv, db = B.cross_attn_bwd(dev(q), dev(k), dev(v), out, stat, dev(y), dev(x), dev(m))
    for b in (0, 1, 2, 4):
        assert not bool(dq[b].any()) and not bool(dk[b].any())
        if bias == "each":
            assert not bool(db[b].any())
    assert bool(dq[3].any()) and bool(dk[3].any()) and not bool(dv[4].any())
    if bias == "shared":  # of the sample with two keys alone
        keys = torch.arange(nk)
        assert not bool(db[:, (keys != 1) & (keys != nk - 2)].any())
    keep = slice(0, 4)  # the plain form has no row without a key
    both(q[keep], k[keep], v[keep], x[keep] if bias == "each" else x, m[keep], y[keep])


def test_many_samples_with_a_map_each():
    # 512 maps of 768 x 768 x 4 heads (2.4 GB), taken as they lie: the first and the last sample
    b, n, h, d = 512, 768, 4, 8
    g = torch.Generator(DEV).manual_seed(1)

    def normal(*shape):
        return torch.empty(shape, dtype=BF, device=DEV).normal_(generator=g)

    q, k, v, y, x = *(normal(b, n, h, d) for _ in range(4)), normal(b, n, n, h)
    m = (torch.rand(b, n, generator=g, device=DEV) < 0.7).to(torch.uint8)
    m[:, 5] = 1
    out, stat = B.cross_attn_fwd(q, k, v, x, m)
    grads = B.cross_attn_bwd(q, k, v, out, stat, y, x, m)
    for i in (0, b - 1):
        at = slice(i, i + 1)
        q1, k1, v1, y1, x1, m1 = (t[at].cpu() for t in (q, k, v, y, x, m))
        for a, r, e in zip((out, stat), *C.attn_fwd(q1, k1, v1, x1, m1)):
            R.check("forward", a[at], r, e)
        for name, a, r, e in zip(("dq", "dk", "dv", "dbias"), grads,
                                 *C.attn_bwd(q1, k1, v1, y1, x1, m1)):
            R.check(name, a[at], r, e)


# one map of many samples: sums of dS over them, by slabs of samples from 16 of them on (fewer
# samples than slices, as many and more, and more than twice), of four heads side by side and
# of planes (shared key heads, heads not in fours); and past 2^20 columns, four a thread
@pytest.mark.parametrize("dtype", [BF, F4])
@pytest.mark.parametrize("b,nq,nk,h,hk,d", [
    (16, 9, 33, 4, 4, 16), (17, 31, 13, 8, 8, 24), (64, 5, 40, 4, 4, 8), (150, 7, 11, 4, 4, 8),
    (16, 9, 33, 4, 2, 16), (17, 31, 13, 3, 3, 24), (70, 6, 65, 5, 5, 8), (150, 3, 11, 6, 2, 8),
    (15, 20, 70, 4, 4, 32), (15, 20, 70, 2, 2, 32), (16, 1, 1, 4, 4, 8), (40, 1, 1, 1, 1, 8),
    (16, 100, 660, 16, 16, 8), (16, 90, 650, 18, 18, 8)])
def test_a_map_that_many_samples_share(b, nq, nk, h, hk, d, dtype):
    q, k, v, x, m, y = inputs(b, nq, nk, h, hk, d, dtype, "shared", True, seed=b + nk)
    got = both(q, k, v, x, m, y)
    again = B.cross_attn_bwd(dev(q), dev(k), dev(v), *got[:2], dev(y), dev(x), dev(m))
    for a, c in zip(again, got[2:]):  # in a fixed order
        assert torch.equal(a, c)
