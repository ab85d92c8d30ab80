"""The linear projection in its 128-wide tiles, which take the large calls:
forward, dx and dW, whole and ragged rows, both types, every source of dz
(plain 64-bit forms and bounds in ops_ref.py)."""
import math

import pytest
import torch

import ops_ref as R
from paper_2506_20686_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F4 = torch.bfloat16, torch.float32
NONE, RELU, GELU, SILU = B.ACT_NONE, B.ACT_RELU, B.ACT_GELU, B.ACT_SILU


def tiles(rows, cols):
    return -(-rows // 128) * -(-cols // 128)


def wide(dtype, m, width, terms):
    """A result [m][width] of sums of `terms` goes in 128-wide tiles: there are enough of
    them for the 256 CUs, and for fp32 the sums are long."""
    return width > 64 and tiles(m, width) >= 256 and (dtype == BF or terms >= 256)


def wide_w(m, k, n):
    """dW does: 256 workgroups of at least 512 rows."""
    return k > 64 and n > 64 and tiles(k, n) * -(-m // 512) >= 256


def inputs(m, k, n, dtype, seed):
    g = torch.Generator().manual_seed(seed)

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=g) * std).to(dtype)

    return {"x": normal(m, k), "w": normal(k, n, std=k ** -0.5), "bias": normal(n, std=0.3),
            "residual": normal(m, n, std=1.5), "z": normal(m, n, std=1.2), "dout": normal(m, n)}


def dev(t):
    return None if t is None else t.to(DEV)


@pytest.mark.parametrize("dtype,m,k,n,act", [
    (BF, 33000, 128, 128, NONE), (BF, 16390, 72, 200, GELU), (BF, 33001, 77, 129, SILU),
    (BF, 33000, 130, 127, RELU), (F4, 33000, 256, 128, GELU), (F4, 16500, 260, 132, SILU)])
def test_forward(dtype, m, k, n, act):
    assert wide(dtype, m, n, k) and (dtype == BF or k % 4 == n % 4 == 0)
    t = inputs(m, k, n, dtype, m + k + n)
    # all of the epilogue, each part missing, and the plain product
    for bias, residual, save_z, a in ((True, True, True, act), (False, True, False, NONE),
                                      (True, False, True, act), (False, False, False, NONE)):
        b, r = (t["bias"] if bias else None), (t["residual"] if residual else None)
        out, z = B.linear_fwd(dev(t["x"]), dev(t["w"]), dev(b), dev(r), a, save_z)
        (ro, rz), (eo, ez) = R.lin_fwd(t["x"], t["w"], b, r, a)
        R.check("out", out, ro, eo)
        if save_z:
            R.check("z", z, rz, ez)


# (dtype, m, k, n, act, whether dx and dW go in 128-wide tiles)
BACKWARD = [
    (BF, 16500, 256, 136, NONE, 1, 0), (BF, 16500, 256, 136, GELU, 1, 0),
    (BF, 16500, 255, 131, RELU, 1, 0), (BF, 16500, 255, 131, SILU, 1, 0),
    (BF, 33000, 128, 136, SILU, 1, 0), (BF, 33001, 127, 130, GELU, 1, 0),
    (F4, 16500, 256, 260, NONE, 1, 0), (F4, 16500, 255, 261, SILU, 1, 0),
    (BF, 33000, 256, 136, RELU, 1, 1), (BF, 33000, 256, 136, SILU, 1, 1),
    (BF, 33001, 257, 131, NONE, 1, 1), (BF, 33001, 257, 131, GELU, 1, 1),
    (BF, 33000, 128, 512, GELU, 1, 1), (F4, 33000, 256, 260, RELU, 1, 1),
    (F4, 33000, 128, 512, SILU, 1, 1), (F4, 33001, 257, 261, NONE, 1, 1),
    (F4, 33001, 257, 261, GELU, 1, 1),
    (BF, 1600, 1024, 1024, NONE, 0, 1), (BF, 1600, 1024, 1024, SILU, 0, 1),
    (BF, 1600, 1023, 1025, RELU, 0, 1), (BF, 1600, 1023, 1025, GELU, 0, 1),
    (BF, 16300, 128, 1024, GELU, 0, 1), (BF, 16300, 127, 1023, SILU, 0, 1),
    (F4, 1600, 1024, 1024, GELU, 0, 1), (F4, 1600, 1023, 1025, NONE, 0, 1),
    (F4, 33000, 256, 136, RELU, 0, 1), (F4, 16300, 127, 1023, GELU, 0, 1),
]


@pytest.mark.parametrize("dtype,m,k,n,act,wx,ww", BACKWARD)
def test_backward(dtype, m, k, n, act, wx, ww):
    assert wide(dtype, m, k, n) == wx and wide_w(m, k, n) == ww
    t = inputs(m, k, n, dtype, m + 3 * k + n)
    z = t["z"] if act else None
    args = (dev(t["x"]), dev(t["w"]), dev(t["dout"]), dev(z), act)
    got = B.linear_bwd(*args)
    ref, bound = R.lin_bwd(t["x"], t["w"], t["dout"], z, act)
    for name, a, r, e in zip(("dx", "dw", "dbias"), got, ref, bound):
        R.check(name, a, r, e)
    # the worst case of a sum over m rows hides a row that is missing from it; the random
    # roundings of dw and dbias do not: each is a step of the partial sum, which grows as
    # the root of its terms, and dz itself is good to 16
    for name, a, r in zip(("dw", "dbias"), got[1:], ref[1:]):
        R.fro(name, a, r, (2 * math.sqrt(m) + 16) * R.U)
    # dx by itself and dW by itself are launches of their own, with the same results
    code = B.BF16 if dtype == BF else B.F32
    need = B.tri_linear_bwd_workspace_bytes(code, m, k, n, act)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    s = torch.cuda.current_stream().cuda_stream
    x, w, dout, zz, _ = args
    for keep in ((1, 0, 0), (0, 1, 1), (0, 0, 1)):
        alone = [torch.empty_like(a) if f else None for f, a in zip(keep, got)]
        assert B.tri_linear_bwd(code, m, k, n, act, x.data_ptr(), w.data_ptr(),
                                zz.data_ptr() if act else None, dout.data_ptr(),
                                *(None if a is None else a.data_ptr() for a in alone),
                                ws.data_ptr(), need, s) == B.OK
        for a, b in zip(alone, got):
            assert a is None or torch.equal(a, b)


@pytest.mark.parametrize("dtype,m,k,n", [(BF, 33000, 128, 128), (BF, 33001, 77, 129),
                                         (F4, 16500, 260, 132)])
def test_output_over_the_residual(dtype, m, k, n):
    assert wide(dtype, m, n, k)
    t = {a: b.to(DEV) for a, b in inputs(m, k, n, dtype, 4).items()}
    want, _ = B.linear_fwd(t["x"], t["w"], t["bias"], t["residual"], SILU)
    r = t["residual"].data_ptr()
    code = B.BF16 if dtype == BF else B.F32
    assert B.tri_linear_fwd(code, m, k, n, SILU, t["x"].data_ptr(), t["w"].data_ptr(),
                            t["bias"].data_ptr(), r, r, None,
                            torch.cuda.current_stream().cuda_stream) == B.OK
    assert torch.equal(t["residual"], want)


def test_gelu_backward_in_a_graph():
    # dz made beforehand, both products and the splits' sums, replayed on other inputs with
    # eager work between; the workspace full of other values before each replay
    m, k, n = 1700, 512, 512
    assert wide_w(m, k, n) is False
    sets = [{a: b.to(DEV) for a, b in inputs(m, k, n, BF, s).items()} for s in (1, 2)]
    t = {a: b.clone() for a, b in sets[0].items()}
    ws = torch.empty(B.tri_linear_bwd_workspace_bytes(B.BF16, m, k, n, GELU), dtype=torch.uint8,
                     device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = B.linear_bwd(t["x"], t["w"], t["dout"], t["z"], GELU, ws)
    for s in (1, 0, 1):
        want = B.linear_bwd(*(sets[s][a] for a in ("x", "w", "dout", "z")), GELU)
        for a in t:
            t[a].copy_(sets[s][a])
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
