"""Refusals of the cross attention, the gated linear projection and the clipping of
gradients (CPU): every call here is invalid or only sizes a workspace, and the library
returns before any HIP call.  The wrappers' own checks likewise."""
import ctypes
import os
import re

import pytest
import torch

from paper_2506_20686_amd import binding as B

P = 0x10000  # fake, 16-byte aligned, never touched
INV, UNS, WS = B.ERR_INVALID_ARG, B.ERR_UNSUPPORTED, B.ERR_WORKSPACE
NAN, INF = float("nan"), float("inf")


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
    names = set(re.findall(r"\b(tri_(?:cross_attn|gated_linear|grad)_\w+)\s*\(", text))
    assert len(names) == 10
    for name in names:
        assert hasattr(lib, name), name


def call(fn, order, base, over):
    a = dict(base, **over)
    assert set(over) <= set(base), over
    return fn(*(a[k] for k in order.split()))


PTR = {"stream": None, "ws": P, "wsb": 1 << 60}
XAT = dict(PTR, dtype=B.BF16, b=2, nq=50, nk=70, h=8, hk=2, d=24, bb=2, scale=0.2, q=P, k=P, v=P,
           bias=P, mask=P + 1, out=P, stat=P, dout=P, dq=P, dk=P, dv=P, dbias=P)
SIZED = "dtype b nq nk h hk d bb"
XAT_FWD = SIZED + " scale q k v bias mask out stat ws wsb stream"
XAT_BWD = SIZED + " scale q k v bias mask out stat dout dq dk dv dbias ws wsb stream"
XAT_SIZES = [(dict(dtype=-1), INV), (dict(dtype=2), INV), (dict(b=0), INV),
             (dict(b=(1 << 20) + 1), INV), (dict(nq=0), INV), (dict(nk=0), INV), (dict(nk=-5), INV),
             (dict(nq=(1 << 22) + 1), INV), (dict(nk=(1 << 22) + 1), INV), (dict(h=0), INV),
             (dict(hk=0), INV), (dict(hk=3), INV), (dict(h=2, hk=8), INV), (dict(d=0), INV),
             (dict(bb=3), INV), (dict(bb=-1), INV), (dict(h=264, hk=264), UNS), (dict(d=136), UNS),
             (dict(d=20), UNS), (dict(d=4), UNS), (dict(nq=1 << 22, h=64, hk=1), UNS),
             (dict(b=1 << 20, nq=1 << 10, h=16, hk=16, d=128, bb=1), UNS),
             (dict(b=1 << 20, nk=1 << 13, nq=1, h=1, hk=1, d=8, bb=1), UNS),
             (dict(nq=1 << 21, nk=65, bb=1), UNS),
             (dict(nq=1 << 13, nk=(1 << 13) - 63, h=256, hk=256, d=8, bb=1), UNS)]
XAT_ARGS = [(dict(scale=s), INV) for s in (0.0, -1.0, NAN, INF)] + [
    (dict([(k, v)]), INV) for k in ("q", "k", "v", "out", "stat") for v in (None, P + 8)] + [
    (dict(bias=None), INV), (dict(bias=P + 8), INV), (dict(bb=0), INV), (dict(ws=None), WS),
    (dict(ws=P + 8), WS), (dict(wsb=0), WS)]


@pytest.mark.parametrize("over,code", XAT_SIZES + XAT_ARGS)
def test_cross_attn_fwd_refuses(lib, over, code):
    assert call(lib.tri_cross_attn_fwd, XAT_FWD, XAT, over) == code


@pytest.mark.parametrize("over,code", XAT_SIZES + XAT_ARGS + [
    (dict([(k, v)]), INV) for k in ("dout", "dq", "dk", "dv") for v in (None, P + 8)] + [
    (dict(dbias=P + 8), INV), (dict(bb=0, bias=None), INV)])
def test_cross_attn_bwd_refuses(lib, over, code):
    assert call(lib.tri_cross_attn_bwd, XAT_BWD, XAT, over) == code


GLU = dict(PTR, dtype=B.BF16, m=100, k=33, f=65, act=B.ACT_GELU, x=P, w=P, bias=P, out=P, dout=P,
           dx=P, dw=P, dbias=P)
GLU_FWD = "dtype m k f act x w bias out stream"
GLU_BWD = "dtype m k f act x w bias dout dx dw dbias ws wsb stream"
GLU_SIZES = [(dict(dtype=-1), INV), (dict(dtype=2), INV), (dict(m=0), INV), (dict(k=0), INV),
             (dict(f=0), INV), (dict(m=(1 << 31) + 1), INV), (dict(k=8193), UNS),
             (dict(f=4097), UNS), (dict(act=-1), INV), (dict(act=5), INV),
             (dict(m=1 << 30, f=33), UNS)]


@pytest.mark.parametrize("over,code", GLU_SIZES + [
    (dict([(k, v)]), INV) for k in ("x", "w", "out") for v in (None, P + 8)] + [
    (dict(bias=P + 8), INV)])
def test_gated_linear_fwd_refuses(lib, over, code):
    assert call(lib.tri_gated_linear_fwd, GLU_FWD, GLU, over) == code


@pytest.mark.parametrize("over,code", GLU_SIZES + [(dict(m=1 << 30, k=65, f=1), UNS)] + [
    (dict([(k, v)]), INV) for k in ("x", "w", "dout") for v in (None, P + 8)] + [
    (dict([(k, P + 8)]), INV) for k in ("bias", "dx", "dw", "dbias")] + [
    (dict(dx=None, dw=None, dbias=None), INV), (dict(ws=None), WS), (dict(ws=P + 8), WS),
    (dict(wsb=0), WS), (dict(wsb=0, dx=None, dw=None), WS)])
def test_gated_linear_bwd_refuses(lib, over, code):
    assert call(lib.tri_gated_linear_bwd, GLU_BWD, GLU, over) == code


def test_the_linear_projection_still_refuses_sigmoid(lib):
    assert lib.tri_linear_fwd(B.BF16, 4, 4, 4, B.ACT_SIGMOID, P, P, None, None, P, None,
                              None) == INV


def ints(*v):
    return (ctypes.c_int64 * max(len(v), 1))(*v)


def kinds(*v):
    return (ctypes.c_int32 * max(len(v), 1))(*v)


def ptrs(*v):
    return (ctypes.c_void_p * max(len(v), 1))(*v)


GRAD = dict(PTR, n=3, kinds=kinds(0, 1, 0), sizes=ints(5, 0, 70000), grads=ptrs(P, None, P),
            outs=ptrs(P, None, P), norm=P + 4, limit=1.0)
GRAD_NORM, GRAD_CLIP = "n kinds sizes grads norm ws wsb stream", "n kinds sizes grads norm limit outs stream"
GRAD_BAD = [(dict(n=0), INV), (dict(n=(1 << 20) + 1), INV), (dict(sizes=None), INV),
            (dict(kinds=None), INV), (dict(grads=None), INV), (dict(sizes=ints(5, -1, 3)), INV),
            (dict(kinds=kinds(0, 2, 0)), INV), (dict(kinds=kinds(-1, 1, 0)), INV),
            (dict(grads=ptrs(None, None, P)), INV), (dict(grads=ptrs(P, None, P + 8)), INV),
            (dict(sizes=ints(5, 0, 1 << 39)), UNS), (dict(sizes=ints(1 << 38, 0, 1 << 38)), UNS),
            (dict(sizes=ints((1 << 63) - 1, 0, (1 << 63) - 1)), UNS), (dict(norm=None), INV),
            (dict(norm=P + 2), INV)]


@pytest.mark.parametrize("over,code", GRAD_BAD + [(dict(ws=None), WS), (dict(ws=P + 8), WS),
                                                  (dict(wsb=0), WS)])
def test_grad_norm_refuses(lib, over, code):
    assert call(lib.tri_grad_norm, GRAD_NORM, GRAD, over) == code


@pytest.mark.parametrize("over,code", GRAD_BAD + [
    (dict(outs=None), INV), (dict(outs=ptrs(P, None, None)), INV),
    (dict(outs=ptrs(P + 4, None, P)), INV)] + [
    (dict(limit=v), INV) for v in (0.0, -1.0, NAN, INF)])
def test_grad_clip_refuses(lib, over, code):
    assert call(lib.tri_grad_clip, GRAD_CLIP, GRAD, over) == code


def test_workspace_sizes(lib):
    """Sizes are what a call accepts and one byte less is refused."""
    for dtype in (B.F32, B.BF16):
        for b, nq, nk, h, hk, d, bb in ((1, 1, 1, 1, 1, 8, 0), (2, 768, 768, 16, 16, 24, 1),
                                        (700, 32, 128, 4, 4, 32, 700), (3, 1, 30011, 16, 4, 64, 0),
                                        (1, 1 << 22, 5, 8, 8, 128, 0)):
            s = (dtype, b, nq, nk, h, hk, d, bb)
            over = dict(zip(SIZED.split(), s), bias=P if bb else None, dbias=None)
            for name, order in (("fwd", XAT_FWD), ("bwd", XAT_BWD)):
                need = B._sized(f"tri_cross_attn_{name}_workspace_bytes", *s)
                assert 0 < need and need % 256 == 0
                assert call(getattr(lib, f"tri_cross_attn_{name}"), order, XAT,
                            dict(over, wsb=need - 1)) == WS
        for m, k, f in ((1, 1, 1), (1500, 384, 1000), (768 * 768, 128, 128)):
            need = B._sized("tri_gated_linear_bwd_workspace_bytes", dtype, m, k, f)
            assert need >= 0 and need % 256 == 0
            assert call(lib.tri_gated_linear_bwd, GLU_BWD, GLU,
                        dict(dtype=dtype, m=m, k=k, f=f, wsb=need - 1)) == WS
    z = ctypes.c_size_t(0)
    assert lib.tri_grad_norm_workspace_bytes(3, GRAD["sizes"], ctypes.byref(z)) == B.OK
    need = z.value
    assert need % 256 == 0 and call(lib.tri_grad_norm, GRAD_NORM, GRAD, dict(wsb=need - 1)) == WS


def test_workspace_size_errors(lib):
    r = ctypes.byref(ctypes.c_size_t(0))
    for name in ("fwd", "bwd"):
        f = getattr(lib, f"tri_cross_attn_{name}_workspace_bytes")
        assert f(B.BF16, 1, 4, 4, 2, 2, 8, 0, None) == INV
        assert f(B.BF16, 1, 0, 4, 2, 2, 8, 0, r) == INV
        assert f(B.BF16, 1, 4, 4, 2, 2, 9, 0, r) == UNS
    f = lib.tri_gated_linear_bwd_workspace_bytes
    assert f(B.BF16, 4, 4, 4, None) == INV and f(B.BF16, 0, 4, 4, r) == INV
    assert f(B.BF16, 4, 4, 5000, r) == UNS
    f = lib.tri_grad_norm_workspace_bytes
    assert f(1, ints(4), None) == INV and f(0, ints(4), r) == INV


def test_wrappers_refuse_what_is_not_theirs():
    x, q = torch.zeros(4, 8), torch.zeros(4, 2, 8)  # CPU tensors: no call may take them
    for fn in (lambda: B.cross_attn_fwd(q, q, q), lambda: B.cross_attn_bwd(q, q, q, q, q, q),
               lambda: B.gated_linear_fwd(x, x.t().contiguous()),
               lambda: B.gated_linear_bwd(x, x.t().contiguous(), x), lambda: B.grad_norm([x]),
               lambda: B.GradList([]), lambda: B.grad_clip([x], x, 1.0),
               lambda: B.cross_attn_fwd(x, x, x), lambda: B.cross_attn_fwd(q.double(), q, q),
               lambda: B.grad_norm([x.double()])):
        with pytest.raises(ValueError):
            fn()
    for fn in (lambda: B.cross_attn_fwd([1.0], q, q), lambda: B.gated_linear_fwd(None, x),
               lambda: B.grad_norm([3.0]), lambda: B.grad_norm([x, None])):
        with pytest.raises((TypeError, ValueError)):
            fn()


def test_names_of_the_timed_kernels():
    for i, name in enumerate(["xat_planes", "xat_fwd", "xat_join", "xat_dq", "xat_dkv", "xat_dbias",
                              "glu_fwd", "glu_dz", "grad_norm", "grad_clip"]):
        assert B.tri_attn_timing_read(34 + i)[0] == name
