"""Plain 64-bit forms of the layer norm, the linear projection and the relative
position bias (torch, on the CPU), with bounds on how far a kernel may be from
them.

Every bound is worked out from the roundings of the method, U = 2^-24 being
the fp32 half step and HALF[dtype] that of the output's type: an output is off
by its own rounding, HALF |value|, and by the error of the fp32 value that is
rounded.  A sum of L terms that are added one after the other is off by at
most L U times the sum of the terms' magnitudes; a matrix instruction may round
its partial sums twice, hence 2 L U there."""
import math

import torch

U = 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
F8 = torch.float64


def check(name, got, ref, bound):
    """got within `bound` (elementwise, of ref's shape) of ref."""
    got = got.detach().cpu().to(F8)
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    assert bool(torch.isfinite(got).all()), f"{name}: non-finite"
    worst = ((got - ref).abs() / (bound + 1e-37)).max().item() if ref.numel() else 0.0
    assert worst <= 1.0, f"{name}: error {worst:.3g} times the bound"


def fro(name, got, ref, bound):
    """The 2-norm of the error at most `bound` times that of ref."""
    norm = ref.norm().item()
    err = (got.detach().cpu().to(F8) - ref).norm().item()
    assert err <= bound * norm + 1e-30, f"{name}: relative error {err / max(norm, 1e-300):.3g}"


# ---- layer norm ------------------------------------------------------------------------
# A lane adds at most c / 64 values (c / 256 where a workgroup shares a row), then the
# lanes' sums meet in at most 8 more steps.

def _chain(c):
    return c / 64 + 10


def ln_fwd(x, gamma, beta, eps):
    """(out, mean, rstd) and their bounds."""
    half, c = HALF[x.dtype], x.shape[1]
    x = x.to(F8)
    g = torch.ones(c, dtype=F8) if gamma is None else gamma.to(F8)
    b = torch.zeros(c, dtype=F8) if beta is None else beta.to(F8)
    mean = x.mean(1)
    d = x - mean[:, None]
    var = (d * d).mean(1)
    rstd = 1.0 / torch.sqrt(var + eps)
    xhat = d * rstd[:, None]
    out = xhat * g + b
    n = _chain(c)
    e_mean = (n + 1) * U * x.abs().mean(1)
    # the variance is off by n + 3 roundings and, to second order, by the mean's error
    # squared; the root halves that, the root and the division add 2 each
    rel = (n / 2 + 6) * U + e_mean ** 2 * rstd ** 2
    e_xhat = rstd[:, None] * (e_mean[:, None] + 2 * U * d.abs()) + rel[:, None] * xhat.abs()
    e_out = half * out.abs() + 1.01 * (g.abs() * e_xhat + 3 * U * ((xhat * g).abs() + b.abs()))
    return (out, mean, rstd), (e_out, e_mean, 1.01 * rel * rstd)


def ln_bwd(x, gamma, mean, rstd, dout):
    """(dx, dgamma, dbeta) from the statistics given, and their bounds."""
    half, (m, c) = HALF[x.dtype], x.shape
    x, dy, mean, rstd = (t.to(F8) for t in (x, dout, mean, rstd))
    g = torch.ones(c, dtype=F8) if gamma is None else gamma.to(F8)
    xhat = (x - mean[:, None]) * rstd[:, None]
    w = dy * g
    c1, c2 = (w * xhat).mean(1, keepdim=True), w.mean(1, keepdim=True)
    dx = rstd[:, None] * (w - c1 * xhat - c2)
    n = _chain(c)
    e_c1 = (n + 6) * U * (w * xhat).abs().mean(1, keepdim=True)
    e_c2 = (n + 3) * U * w.abs().mean(1, keepdim=True)
    inner = xhat.abs() * e_c1 + e_c2 + 5 * U * (w.abs() + (c1 * xhat).abs() + c2.abs())
    e_dx = half * dx.abs() + 1.01 * (rstd[:, None] * inner + U * dx.abs())
    terms = dy * xhat
    dg, db = terms.sum(0), dy.sum(0)
    return (dx, dg, db), (e_dx, (m + 4) * U * terms.abs().sum(0), (m + 1) * U * dy.abs().sum(0))


# ---- linear projection ------------------------------------------------------------------

SQRT_HALF = math.sqrt(0.5)


def act(z, a):
    if a == 1:
        return torch.clamp(z, min=0)
    if a == 2:
        return 0.5 * z * torch.erfc(-z * SQRT_HALF)
    return z * torch.sigmoid(z) if a == 3 else z


def act_grad(z, a):
    if a == 1:
        return (z > 0).to(z.dtype)
    if a == 2:
        return 0.5 * torch.erfc(-z * SQRT_HALF) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if a == 3:
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def lin_fwd(x, w, bias, residual, a):
    """(out, z) and their bounds: no activation is steeper than 1.13, and its own
    evaluation is good to 16 roundings of its argument's size."""
    half, k = HALF[x.dtype], x.shape[1]
    x, w = x.to(F8), w.to(F8)
    z = x @ w
    mag = x.abs() @ w.abs()
    if bias is not None:
        z = z + bias.to(F8)
        mag = mag + bias.to(F8).abs()
    e_z = 2 * (k + 2) * U * mag
    out = act(z, a)
    e = 1.13 * e_z + (16 * U * z.abs() if a else 0)
    if residual is not None:
        out = out + residual.to(F8)
        e = e + U * out.abs()
    return (out, z), (half * out.abs() + 1.01 * e, half * z.abs() + 1.01 * e_z)


def lin_bwd(x, w, dout, z, a):
    """(dx, dw, dbias) from the z given, and their bounds: act' is good to 16 roundings
    of 1 + |z|; dz enters the products in 24 bits, bf16 dx of an activation in 16."""
    dt, (m, k), n = x.dtype, x.shape, w.shape[1]
    x, w, dy = x.to(F8), w.to(F8), dout.to(F8)
    dz, e_dz = dy, torch.zeros_like(dy)
    if a:
        dz = dy * act_grad(z.to(F8), a)
        e_dz = 16 * U * dy.abs() * (1 + z.to(F8).abs()) if a > 1 else e_dz
    cut = 2.0 ** -16 if a > 1 and dt == torch.bfloat16 else 0.0
    dx, dw, db = dz @ w.t(), x.t() @ dz, dz.sum(0)
    e_dx = HALF[dt] * dx.abs() + 1.01 * (
        (2 * (n + 2) * U + cut) * (dz.abs() @ w.abs().t()) + e_dz @ w.abs().t())
    e_dw = 2 * (m + 2) * U * (x.abs().t() @ dz.abs()) + x.abs().t() @ e_dz
    e_db = (m + 2) * U * dz.abs().sum(0) + e_dz.sum(0)
    return (dx, dw, db), (e_dx, e_dw, e_db)


# ---- relative position bias ----------------------------------------------------------------

def buckets(pos, edges, chain):
    """[b, n, n] for pos [b, n]."""
    d = pos.long()[:, :, None] - pos.long()[:, None, :]
    b = torch.zeros_like(d)
    for e in edges:
        b += d >= e
    if chain is not None:
        b[chain[:, :, None] != chain[:, None, :]] = len(edges) + 1
    return b


def rel_fwd(pos, edges, table, chain, base):
    """Exactly what the kernel gives: one sum, rounded once to the table's type (the
    fp32 sum of two bf16 values is rounded once more on the way)."""
    out = table[buckets(pos, edges, chain)]
    return out if base is None else (out.float() + base.float()).to(table.dtype)


def rel_bwd(pos, edges, dout, chain):
    """dtable and its bound."""
    b, rows = buckets(pos, edges, chain).reshape(-1), len(edges) + 1 + (chain is not None)
    flat = dout.reshape(-1, dout.shape[-1]).to(F8)
    ref = torch.zeros((rows, flat.shape[1]), dtype=F8).index_add_(0, b, flat)
    mag = torch.zeros_like(ref).index_add_(0, b, flat.abs())
    count = torch.bincount(b, minlength=rows).to(F8)[:, None]
    return ref, (count + 1) * U * mag
