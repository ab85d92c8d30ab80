"""Gated linear projection through the C ABI against its plain 64-bit form (bounds in
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
ACTS = [B.ACT_NONE, B.ACT_RELU, B.ACT_GELU, B.ACT_SILU, B.ACT_SIGMOID]


def dev(t):
    return None if t is None else t.to(DEV)


def inputs(m, k, f, dtype, seed=0, bias=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(m, k, generator=g).to(dtype)
    w = (torch.randn(k, 2 * f, generator=g) / math.sqrt(k)).to(dtype)
    b = torch.randn(2 * f, generator=g).to(dtype) if bias else None
    return x, w, b, torch.randn(m, f, generator=g).to(dtype)


def both(m, k, f, act, dtype, seed=0, bias=True):
    x, w, b, dy = inputs(m, k, f, dtype, seed, bias)
    out = B.gated_linear_fwd(dev(x), dev(w), dev(b), act)
    ref, bound = C.gated_fwd(x, w, b, act)
    R.check("out", out, ref, bound)
    grads = B.gated_linear_bwd(dev(x), dev(w), dev(dy), dev(b), act)
    for name, a, r, e in zip(("dx", "dw", "dbias"), grads, *C.gated_bwd(x, w, b, dy, act)):
        R.check(name, a, r, e)


# one of everything; whole and ragged multiples of the tiles (64 x 32 and 128 x 64
# outputs), halves that are no whole 16-byte words of rows that are; few and many rows
SIZES = [(1, 1, 1), (1, 384, 1024), (3, 7, 5), (64, 64, 32), (65, 33, 33), (130, 128, 128),
         (777, 129, 211), (100, 40, 4), (100, 40, 12), (50, 300, 1), (37, 8, 500), (4100, 96, 64),
         (2000, 24, 150), (20000, 16, 8), (9, 1000, 65), (33000, 128, 64), (256, 256, 20),
         (1000, 128, 128), (33, 8, 8), (70001, 64, 24), (31, 120, 104), (40, 16, 128),
         (200, 136, 28), (90, 20, 36), (600, 200, 4)]


@pytest.mark.parametrize("dtype", [BF, F4])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_forward_and_backward(size, dtype):
    both(*size, ACTS[sum(size) % 5], dtype, seed=sum(size))


@pytest.mark.parametrize("dtype", [BF, F4])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("size", [(300, 64, 96), (131, 50, 45)], ids=str)
def test_activations(size, act, dtype):
    both(*size, act, dtype, seed=act)
    both(*size, act, dtype, seed=act, bias=False)


@pytest.mark.parametrize("dtype", [BF, F4])
@pytest.mark.parametrize("size", [(70, 64, 40), (129, 33, 37), (5000, 128, 64), (9000, 128, 128),
                                  (300, 136, 72)], ids=str)
def test_nothing_outside_the_outputs_is_written(size, dtype):
    m, k, f = size
    x, w, b, dy = (dev(t) for t in inputs(m, k, f, dtype, 1))
    ref = (B.gated_linear_fwd(x, w, b), *B.gated_linear_bwd(x, w, dy, b))
    pad, code, act = 64, B.BF16 if dtype == BF else B.F32, B.ACT_SILU
    big = [torch.full((t.numel() + 2 * pad,), 7.0, dtype=t.dtype, device=DEV) for t in ref]
    at = [t.data_ptr() + pad * t.element_size() for t in big]
    need = B._sized("tri_gated_linear_bwd_workspace_bytes", code, m, k, f)
    ws = torch.full((need + 256,), 9, dtype=torch.uint8, device=DEV)
    s, L = torch.cuda.current_stream().cuda_stream, B.lib()
    ins = [t.data_ptr() for t in (x, w, b)]
    assert L.tri_gated_linear_fwd(code, m, k, f, act, *ins, at[0], s) == B.OK
    assert L.tri_gated_linear_bwd(code, m, k, f, act, *ins, dy.data_ptr(), *at[1:], ws.data_ptr(),
                                  need, s) == B.OK
    for t, r in zip(big, ref):
        assert torch.equal(t[pad:-pad], r.reshape(-1))
        assert bool((t[:pad] == 7).all()) and bool((t[-pad:] == 7).all())
    assert bool((ws[need:] == 9).all())
    # each result alone
    for i in range(3):
        big[1 + i].fill_(7.0)
        only = [at[1 + i] if j == i else None for j in range(3)]
        assert L.tri_gated_linear_bwd(code, m, k, f, act, *ins, dy.data_ptr(), *only, ws.data_ptr(),
                                      need, s) == B.OK
        assert torch.equal(big[1 + i][pad:-pad], ref[1 + i].reshape(-1))


@pytest.mark.parametrize("size,dtype", [((3001, 128, 128), BF), ((2000, 65, 33), F4)], ids=str)
def test_bitwise_reproducible(size, dtype):
    x, w, b, dy = (dev(t) for t in inputs(*size, dtype, 8))
    one, two = (B.gated_linear_bwd(x, w, dy, b, B.ACT_GELU) for _ in range(2))
    for s, t in zip(one, two):
        assert torch.equal(s, t)


def test_gradients_against_differences():
    x, w, b, dy = inputs(3, 4, 3, F4, 11)
    for act in (B.ACT_GELU, B.ACT_SILU, B.ACT_SIGMOID):
        grads = B.gated_linear_bwd(dev(x), dev(w), dev(dy), dev(b), act)
        args, h = [t.double() for t in (x, w, b)], 1e-5

        def loss(a):
            z = a[0] @ a[1] + a[2]
            return (C.act(z[:, :3], act) * z[:, 3:] * dy.double()).sum().item()

        for i, grad in enumerate(grads):
            for at in range(args[i].numel()):
                pair = []
                for sign in (1, -1):
                    p = [t.clone() for t in args]
                    p[i].view(-1)[at] += sign * h
                    pair.append(loss(p))
                assert abs((pair[0] - pair[1]) / (2 * h) - grad.reshape(-1)[at].item()) < 2e-5


def test_offsets_past_32_bits():
    m, k, f = (1 << 22) + 5, 24, 261  # 2.2e9 elements of dz
    g = torch.Generator(DEV).manual_seed(1)
    x = torch.randn(m, k, generator=g, device=DEV).to(BF)
    w = (torch.randn(k, 2 * f, generator=g, device=DEV) / 5).to(BF)
    dy = torch.zeros(m, f, dtype=BF, device=DEV)
    dy[-3:] = torch.randn(3, f, generator=g, device=DEV).to(BF)
    out = B.gated_linear_fwd(x, w)
    rows = torch.tensor([0, 1, 1 << 22, m - 2, m - 1], device=DEV)
    ref, bound = C.gated_fwd(x[rows].cpu(), w.cpu(), None, B.ACT_SILU)
    R.check("out", out[rows], ref, bound)
    dx, dw, db = B.gated_linear_bwd(x, w, dy)
    ref, bound = C.gated_bwd(x[-3:].cpu(), w.cpu(), None, dy[-3:].cpu(), B.ACT_SILU)
    for name, a, r, e in zip(("dx", "dw", "dbias"), (dx[-3:], dw, db), ref, bound):
        R.check(name, a, r, e)
    assert not bool(dx[:-3].any())
