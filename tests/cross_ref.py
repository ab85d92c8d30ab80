"""Plain 64-bit forms of the cross attention and of the gated linear projection
(torch, on the CPU), with bounds on how far a kernel may be from them.

The bounds count roundings, as those of ops_ref.py do: U = 2^-24 is the fp32 half
step, HALF[dtype] that of the output's type; matrix instructions may round a
partial sum twice.  With bf16 tensors the weights P and the dS of a product are
rounded to bf16, HALF of each."""
import math

import torch

import ops_ref as R

U, HALF, F8 = R.U, R.HALF, R.F8


def heads_first(t, group=1):
    """[b, n, h, d] -> [b, h * group, n, d] in 64 bits, each head `group` times."""
    return t.to(F8).permute(0, 2, 1, 3).repeat_interleave(group, dim=1).contiguous()


def back(t):
    return t.permute(0, 2, 1, 3).contiguous()


def softmax_parts(q, k, bias, mask, scale):
    """Logits (-inf where masked), their maximum, weights, log-sum beside the maximum, and
    the bound on the relative error of a weight."""
    b, nq, h, d = q.shape
    g = h // k.shape[2]
    Q, K = heads_first(q), heads_first(k, g)
    if mask is not None:  # what is masked may hold anything
        K = torch.where((mask != 0)[:, None, :, None], K, torch.zeros_like(K))
    s = Q @ K.mT * scale
    e_s = 2 * (d + 4) * U * (Q.abs() @ K.abs().mT) * scale
    if bias is not None:
        x = bias.to(F8)
        x = (x if x.dim() == 4 else x[None]).permute(0, 3, 1, 2)
        s = s + x
        e_s = e_s + 2 * U * torch.where(x.isfinite(), s.abs(), torch.zeros_like(s))
    if mask is not None:
        s = s.masked_fill((mask == 0)[:, None, None, :], -math.inf)
    on = s.isfinite()
    m = s.amax(dim=3, keepdim=True)
    base = torch.where(m.isfinite(), m, torch.zeros_like(m))
    w = torch.exp(s - base)
    total = w.sum(dim=3, keepdim=True)
    p = torch.where(total > 0, w / total.clamp_min(1e-300), torch.zeros_like(w))
    e_s = torch.where(on, e_s, torch.zeros_like(e_s)).amax(dim=3, keepdim=True)
    size = torch.where(on, s.abs(), torch.zeros_like(s)).amax(dim=3, keepdim=True)
    # exponent: the logits' error twice (itself, the maximum), a product and a sum in the
    # logit's size; the exponential itself; the sum of nk weights and its reciprocal
    delta = 2 * e_s + (8 * size + 8 + s.shape[3]) * U
    return s, m, p, torch.log(total.clamp_min(1.0)), e_s, delta


def attn_fwd(q, k, v, bias=None, mask=None, scale=None):
    """(out, stat) and their bounds."""
    scale = 1 / math.sqrt(q.shape[3]) if scale is None else scale
    half = HALF[q.dtype]
    hp = half if q.dtype == torch.bfloat16 else 0.0
    _, m, p, ls, e_s, delta = softmax_parts(q, k, bias, mask, scale)
    V = heads_first(v, q.shape[2] // k.shape[2])
    if mask is not None:
        V = torch.where((mask != 0)[:, None, :, None], V, torch.zeros_like(V))
    out = p @ V
    nk = k.shape[1]
    e = half * out.abs() + 1.01 * (hp + 2 * delta + 2 * (nk + 16) * U) * (p @ V.abs())
    stat = torch.cat([m, ls], dim=3)
    e_stat = torch.cat([e_s + 2 * U * torch.where(m.isfinite(), m.abs(), torch.zeros_like(m)),
                        delta + 4 * U * ls.abs()], dim=3)
    return (back(out), back(stat)), (back(e), back(e_stat))


def attn_bwd(q, k, v, dout, bias=None, mask=None, scale=None):
    """(dq, dk, dv, dbias) and their bounds."""
    b, nq, h, d = q.shape
    nk, hk = k.shape[1:3]
    g = h // hk
    scale = 1 / math.sqrt(d) if scale is None else scale
    half = HALF[q.dtype]
    hp = half if q.dtype == torch.bfloat16 else 0.0
    _, _, p, _, e_s, delta = softmax_parts(q, k, bias, mask, scale)
    dP = 3 * delta  # the weights are formed again from rounded statistics
    Q, K, V, Y = heads_first(q), heads_first(k, g), heads_first(v, g), heads_first(dout)
    if mask is not None:
        keep = (mask != 0)[:, None, :, None]
        K, V = torch.where(keep, K, torch.zeros_like(K)), torch.where(keep, V, torch.zeros_like(V))
    dp = Y @ V.mT
    e_dp = 2 * (d + 4) * U * (Y.abs() @ V.abs().mT)
    D = (p * dp).sum(3, keepdim=True)
    out = p @ V
    # the shift dO . out is off D by the rounding of out (and the weights' in it)
    shift = (2 * half + 2 * hp + 4 * delta + (d + nk) * U) * (Y.abs() * (p @ V.abs())).sum(
        3, keepdim=True)
    e_D = (p * (e_dp + (dP + (nk + 8) * U) * (dp.abs() + D.abs() + shift))).sum(3, keepdim=True) \
        + 4 * U * (D.abs() + shift)
    ds = p * (dp - D)
    e_ds = p * (e_dp + e_D + (dP + 4 * U) * ((dp - D).abs() + shift))
    # dq: the shifted dS and P rounded for their products, e P K taken off again
    moved = ds.abs() + p * shift
    n2 = 2 * (nk + 16) * U
    e_dq = scale * (((hp + n2) * moved + e_ds) @ K.abs()
                    + (shift * (hp + dP + n2) + e_D) * (p @ K.abs()))
    dq = scale * (ds @ K)
    rows = 2 * (nq * g + 16) * U

    def keys(t):  # sum over the heads of a key head
        return t.reshape(b, hk, g, nk, d).sum(2)

    dk = keys(scale * (ds.mT @ Q))
    e_dk = keys(scale * ((((hp + rows) * ds.abs() + e_ds).mT) @ Q.abs()))
    dv = keys(p.mT @ Y)
    e_dv = keys(((hp + dP + rows) * p).mT @ Y.abs())
    res, bound = [back(dq), back(dk), back(dv)], [
        half * back(dq).abs() + 1.01 * back(e_dq), half * back(dk).abs() + 1.01 * back(e_dk),
        half * back(dv).abs() + 1.01 * back(e_dv)]
    db = e_db = None
    if bias is not None:
        db, e_db = ds.permute(0, 2, 3, 1), e_ds.permute(0, 2, 3, 1) + b * U * ds.abs().permute(
            0, 2, 3, 1)
        if bias.dim() == 3:
            db, e_db = db.sum(0), e_db.sum(0)
        e_db = half * db.abs() + 1.01 * e_db
    return res + [db], bound + [e_db]


# ---- gated linear projection -------------------------------------------------------------

def act(z, a):
    return torch.sigmoid(z) if a == 4 else R.act(z, a)


def act_grad(z, a):
    if a == 4:
        return torch.sigmoid(z) * torch.sigmoid(-z)
    return R.act_grad(z, a)


def gated(x, w, bias):
    """a, b and the bounds of their fp32 values."""
    x, w = x.to(F8), w.to(F8)
    z, mag = x @ w, x.abs() @ w.abs()
    if bias is not None:
        z, mag = z + bias.to(F8), mag + bias.to(F8).abs()
    e = 2 * (x.shape[1] + 2) * U * mag
    f = w.shape[1] // 2
    return z[:, :f], z[:, f:], e[:, :f], e[:, f:]


def gated_fwd(x, w, bias, a):
    za, zb, ea, eb = gated(x, w, bias)
    v = act(za, a)
    out = v * zb
    # no activation is steeper than 1.13; its evaluation is good to 16 roundings of 1 + |z|
    ev = 1.13 * ea + (16 * U * (1 + za.abs()) if a else 0)
    return out, HALF[x.dtype] * out.abs() + 1.01 * (ev * zb.abs() + (v.abs() + ev) * eb
                                                    + 2 * U * out.abs())


def gated_bwd(x, w, bias, dout, a):
    """(dx, dw, dbias) and their bounds; no activation's second derivative passes 1.13."""
    dt, (m, k) = x.dtype, x.shape
    za, zb, ea, eb = gated(x, w, bias)
    x, w, dy = x.to(F8), w.to(F8), dout.to(F8)
    v, s = act(za, a), act_grad(za, a)
    tail = 16 * U * (1 + za.abs()) if a else torch.zeros_like(za)
    ev, es = 1.13 * ea + tail, (0 if a < 2 else 1.13) * ea + tail
    dz = torch.cat([dy * zb * s, dy * v], dim=1)
    e_dz = dy.abs().repeat(1, 2) * torch.cat(
        [(zb.abs() + eb) * es + eb * s.abs() + 3 * U * (zb * s).abs(), ev + U * v.abs()], dim=1)
    n = w.shape[1]
    dx, dw, db = dz @ w.t(), x.t() @ dz, dz.sum(0)
    return (dx, dw, db), (
        HALF[dt] * dx.abs() + 1.01 * ((2 * (n + 2) * U * dz.abs() + e_dz) @ w.abs().t()),
        x.abs().t() @ (2 * (m + 2) * U * dz.abs() + 1.01 * e_dz),
        ((m + 2) * U * dz.abs() + 1.01 * e_dz).sum(0))
