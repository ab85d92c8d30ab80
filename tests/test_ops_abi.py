"""Refusals of the layer norm, the linear projection and the relative position
bias (CPU): every call here is invalid or only sizes a workspace, and the
library returns before any HIP call.  The wrappers' own checks likewise."""
import ctypes
import os
import re

import pytest
import torch

from paper_2506_20686_amd import binding as B

P = 0x10000  # fake, 16-byte aligned, never touched
INV, UNS, WS = B.ERR_INVALID_ARG, B.ERR_UNSUPPORTED, B.ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2506_20686_amd import build
        build.build()
    return B.lib()


def test_exports_every_declared_symbol(lib):
    header = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include",
                          "triattn.h")
    text = re.sub(r"/\*.*?\*/", "", open(header).read(), flags=re.S)
    names = set(re.findall(r"\b(tri_(?:layer_norm|linear|rel_bias)_\w+)\s*\(", text))
    assert len(names) == 9
    for name in names:
        assert hasattr(lib, name), name


def call(fn, order, base, over):
    a = dict(base, **over)
    assert set(over) <= set(base), over
    return fn(*(a[k] for k in order.split()))


PTR = {"stream": None, "ws": P, "wsb": 1 << 40}
LN = dict(PTR, dtype=B.BF16, m=100, c=130, eps=1e-5, x=P, gamma=P, beta=P, out=P, mean=P, rstd=P,
          dout=P, dx=P, dgamma=P, dbeta=P)
LN_SIZES = [(dict(dtype=-1), INV), (dict(dtype=2), INV), (dict(m=0), INV), (dict(m=-3), INV),
            (dict(m=(1 << 31) + 1), INV), (dict(c=0), INV), (dict(c=8193), UNS)]
LN_FWD = "dtype m c eps x gamma beta out mean rstd stream"
LN_BWD = "dtype m c x gamma mean rstd dout dx dgamma dbeta ws wsb stream"


@pytest.mark.parametrize("over,code", LN_SIZES + [
    (dict(eps=-1.0), INV), (dict(eps=float("nan")), INV), (dict(eps=float("inf")), INV)] + [
    (dict([(k, v)]), INV) for k in ("x", "out", "mean", "rstd") for v in (None, P + 8)] + [
    (dict(gamma=P + 2), INV), (dict(beta=P + 4), INV)])
def test_layer_norm_fwd_refuses(lib, over, code):
    assert call(lib.tri_layer_norm_fwd, LN_FWD, LN, over) == code


@pytest.mark.parametrize("over,code", LN_SIZES + [
    (dict([(k, v)]), INV) for k in ("x", "mean", "rstd", "dout", "dx") for v in (None, P + 8)] + [
    (dict(gamma=P + 2), INV), (dict(dgamma=P + 4), INV), (dict(dbeta=P + 4), INV),
    (dict(ws=None), WS), (dict(ws=P + 8), WS), (dict(wsb=0), WS),
    (dict(wsb=0, dgamma=None), WS), (dict(wsb=0, dbeta=None), WS)])
def test_layer_norm_bwd_refuses(lib, over, code):
    assert call(lib.tri_layer_norm_bwd, LN_BWD, LN, over) == code


LIN = dict(PTR, dtype=B.BF16, m=100, k=33, n=65, act=B.ACT_GELU, x=P, w=P, bias=P, residual=P,
           out=P, z=P, dout=P, dx=P, dw=P, dbias=P)
LIN_SIZES = [(dict(dtype=-1), INV), (dict(dtype=2), INV), (dict(m=0), INV), (dict(k=0), INV),
             (dict(n=0), INV), (dict(m=(1 << 31) + 1), INV), (dict(k=8193), UNS),
             (dict(n=8193), UNS), (dict(act=-1), INV), (dict(act=4), INV),
             (dict(m=1 << 30, k=64, n=64), UNS), (dict(m=1 << 29, k=1, n=129), UNS)]
LIN_FWD = "dtype m k n act x w bias residual out z stream"
LIN_BWD = "dtype m k n act x w z dout dx dw dbias ws wsb stream"


@pytest.mark.parametrize("over,code", LIN_SIZES + [
    (dict([(k, v)]), INV) for k in ("x", "w", "out") for v in (None, P + 8)] + [
    (dict([(k, P + 8)]), INV) for k in ("bias", "residual", "z")])
def test_linear_fwd_refuses(lib, over, code):
    assert call(lib.tri_linear_fwd, LIN_FWD, LIN, over) == code


@pytest.mark.parametrize("over,code", LIN_SIZES + [
    (dict([(k, v)]), INV) for k in ("x", "w", "dout") for v in (None, P + 8)] + [
    (dict([(k, P + 8)]), INV) for k in ("dx", "dw", "dbias", "z")] + [
    (dict(z=None), INV), (dict(dx=None, dw=None, dbias=None), INV), (dict(ws=None), WS),
    (dict(ws=P + 8), WS), (dict(wsb=0), WS), (dict(wsb=0, dx=None, dw=None), WS)])
def test_linear_bwd_refuses(lib, over, code):
    assert call(lib.tri_linear_bwd, LIN_BWD, LIN, over) == code


def edges(*values):
    return (ctypes.c_int32 * max(len(values), 1))(*values)


REL = dict(PTR, dtype=B.BF16, batch=2, n=50, h=4, ne=3, edges=edges(-1, 0, 7), pos=P, chain=P,
           table=P, base=P, out=P, dout=P, dtable=P)
REL_SIZES = [(dict(dtype=-1), INV), (dict(batch=0), INV), (dict(batch=(1 << 20) + 1), INV),
             (dict(n=0), INV), (dict(n=8193), INV), (dict(h=0), INV), (dict(h=257), UNS),
             (dict(batch=1 << 20, n=8192, h=256), UNS), (dict(batch=128, n=8192, h=64), UNS),
             (dict(ne=0), INV), (dict(ne=256), UNS), (dict(edges=None), INV),
             (dict(edges=edges(0, 0, 1)), INV), (dict(edges=edges(3, 2, 5)), INV),
             (dict(edges=edges(3, 4, -5)), INV), (dict(pos=None), INV), (dict(pos=P + 2), INV),
             (dict(chain=P + 2), INV)]
REL_FWD = "dtype batch n h ne edges pos chain table base out stream"
REL_BWD = "dtype batch n h ne edges pos chain dout dtable ws wsb stream"


@pytest.mark.parametrize("over,code", REL_SIZES + [
    (dict([(k, v)]), INV) for k in ("table", "out") for v in (None, P + 8)] + [
    (dict(base=P + 8), INV)])
def test_rel_bias_fwd_refuses(lib, over, code):
    assert call(lib.tri_rel_bias_fwd, REL_FWD, REL, over) == code


@pytest.mark.parametrize("over,code", REL_SIZES + [
    (dict([(k, v)]), INV) for k in ("dout", "dtable") for v in (None, P + 8)] + [
    (dict(ws=None), WS), (dict(ws=P + 8), WS), (dict(wsb=0), WS)])
def test_rel_bias_bwd_refuses(lib, over, code):
    assert call(lib.tri_rel_bias_bwd, REL_BWD, REL, over) == code


def test_workspace_sizes(lib):
    """Sizes are what a call accepts and one byte less is refused; they stay small beside
    the tensors of large calls and do not overflow at the limits."""
    for dtype in (B.F32, B.BF16):
        for m, c in ((1, 1), (48, 384), (768 * 768, 128), (1 << 31, 8192)):
            need = B.tri_layer_norm_bwd_workspace_bytes(dtype, m, c)
            assert 0 < need and need % 256 == 0 and need <= 64 * c * 1024 + 256
            assert call(lib.tri_layer_norm_bwd, LN_BWD, LN,
                        dict(dtype=dtype, m=m, c=c, wsb=need - 1)) == WS
        for m, k, n in ((1, 1, 1), (1500, 384, 1536), (768 * 768, 128, 128), (1 << 14, 8192, 8192)):
            need = B.tri_linear_bwd_workspace_bytes(dtype, m, k, n, B.ACT_NONE)
            assert 0 < need and need % 256 == 0
            assert call(lib.tri_linear_bwd, LIN_BWD, LIN,
                        dict(dtype=dtype, m=m, k=k, n=n, wsb=need - 1)) == WS
        for b, n, h, ne in ((1, 1, 1, 1), (1, 768, 4, 64), (64, 8192, 64, 255), (1 << 20, 300, 5, 64)):
            need = B.tri_rel_bias_bwd_workspace_bytes(dtype, b, n, h, ne)
            assert 0 < need and need % 256 == 0
            e = edges(*range(ne))
            assert call(lib.tri_rel_bias_bwd, REL_BWD, REL, dict(
                dtype=dtype, batch=b, n=n, h=h, ne=ne, edges=e, wsb=need - 1)) == WS


def test_workspace_size_errors(lib):
    z = ctypes.c_size_t(0)
    r = ctypes.byref(z)
    assert lib.tri_layer_norm_bwd_workspace_bytes(B.BF16, 4, 4, None) == INV
    assert lib.tri_layer_norm_bwd_workspace_bytes(B.BF16, 0, 4, r) == INV
    assert lib.tri_layer_norm_bwd_workspace_bytes(B.BF16, 4, 9000, r) == UNS
    assert lib.tri_linear_bwd_workspace_bytes(B.BF16, 4, 4, 4, 0, None) == INV
    assert lib.tri_linear_bwd_workspace_bytes(B.BF16, 4, 4, 4, 9, r) == INV
    assert lib.tri_linear_bwd_workspace_bytes(B.BF16, 4, 9000, 4, 0, r) == UNS
    assert lib.tri_rel_bias_bwd_workspace_bytes(B.BF16, 1, 4, 4, 3, None) == INV
    assert lib.tri_rel_bias_bwd_workspace_bytes(B.BF16, 1, 4, 4, 0, r) == INV
    assert lib.tri_rel_bias_bwd_workspace_bytes(B.BF16, 1, 4, 300, 3, r) == UNS


def test_wrappers_refuse_what_is_not_theirs():
    x = torch.zeros(4, 8)  # a CPU tensor: no call may take it
    i = torch.zeros(4, dtype=torch.int32)
    for fn in (lambda: B.layer_norm_fwd(x), lambda: B.layer_norm_bwd(x, None, x, x, x),
               lambda: B.linear_fwd(x, x.t().contiguous()),
               lambda: B.linear_bwd(x, x.t().contiguous(), x),
               lambda: B.rel_bias_fwd(i, [0], torch.zeros(2, 4)),
               lambda: B.rel_bias_bwd(i, [0], torch.zeros(4, 4, 4))):
        with pytest.raises(ValueError):
            fn()
    with pytest.raises(TypeError):
        B.layer_norm_fwd([1.0])
    with pytest.raises(ValueError):
        B.layer_norm_fwd(torch.zeros(4))
    with pytest.raises(ValueError):
        B.linear_fwd(x.double(), x.double())
    for bad in ([0.5, "a"], None):
        with pytest.raises(TypeError):
            B._edges_arr(bad)
    with pytest.raises(ValueError):
        B._edges_arr([0, 1 << 31])


def test_edges():
    assert B.rel_bias_edges(2) == [-1, 0, 1, 2]
    # differences -2 .. 2 clipped give buckets 0 .. 4
    for d, want in ((-9, 0), (-2, 0), (-1, 1), (0, 2), (1, 3), (2, 4), (9, 4)):
        assert sum(e <= d for e in B.rel_bias_edges(2)) == want
    far = B.rel_bias_edges(16, 512, 16)
    assert far == sorted(set(far)) and far[-1] == 512 and far[0] == -511 and len(far) == 64
    for bad in ((0,), (4, 4, 2), (4, 0, -1)):
        with pytest.raises(ValueError):
            B.rel_bias_edges(*bad)
