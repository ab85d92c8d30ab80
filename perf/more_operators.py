"""Cross attention, the gated linear projection and the clipping of gradients by their
global norm, as measurable cases.

A case is a dict of plain values.  "op" names the operator:

  att   attention of queries to keys and values of another length, with a pair bias
        and a key mask or without (binding.cross_attn_fwd / _bwd)
  glu   out = act(x Wa + ba) * (x Wb + bb) and its gradients
        (binding.gated_linear_fwd / _bwd)
  clip  the norm of a list of gradients, and the list scaled so that it does not pass
        a limit (binding.grad_norm, binding.grad_clip)

and "mode" is what the caller does with it: "fwd" (a forward), "bwd" (a backward, given
what the forward saved), "train" (both, one after the other), "norm" or "clip" (the norm
and the scaling).  Where `own` is false a pass computes the operator in its plain form.
"""
import math
import random

import torch

own = False


def _att(name, b, q, k, h, d, mode, hk=0, bias="none", mask=False, dtype="bf16"):
    return {"name": name, "op": "att", "mode": mode, "dtype": dtype, "b": b, "q": q, "k": k, "h": h,
            "hk": hk or h, "d": d, "bias": bias, "mask": mask}


def _glu(name, m, k, f, mode, act="silu", dtype="bf16", bias=True):
    return {"name": name, "op": "glu", "mode": mode, "dtype": dtype, "m": m, "k": k, "f": f,
            "act": act, "bias": bias}


def _clip(name, count, total, mode, dtype="f32", ratio=0.5):
    return {"name": name, "op": "clip", "mode": mode, "dtype": dtype, "count": count, "total": total,
            "ratio": ratio}


def listed():
    return [
        # a ligand's few atoms reading a short peptide, fp32: nothing but latency
        _att("att_f32_q7_k33_h4_d32_fwd", 1, 7, 33, 4, 32, "fwd", dtype="f32"),
        # the single representation of a 768-token crop attending to itself with the
        # pair representation's bias (384 channels in 16 heads), training
        _att("att_n768_h16_d24_bias_train", 1, 768, 768, 16, 24, "train", bias="shared"),
        # atoms in windows: 32 queries to the 128 keys around them, a bias of each
        # window, keys missing at the ends of chains, training
        _att("att_b737_q32_k128_h4_d32_train", 737, 32, 128, 4, 32, "train", bias="each", mask=True),
        # a decoder's tokens to an encoder's states of another, ragged length, training:
        # the largest call
        _att("att_b2_q2048_k4099_h16_d64_train", 2, 2048, 4099, 16, 64, "train", mask=True),
        # one new token a sequence reading long encoder states, four query heads to a
        # key head: inference
        _att("att_b3_q1_k30011_h16_hk4_fwd", 3, 1, 30011, 16, 64, "fwd", hk=4, mask=True),
        # one row: the feed-forward block of a single token, inference
        _glu("glu_m1_k384_f1024_silu_fwd", 1, 384, 1024, "fwd"),
        # the gated projections into a triangle update, 128 pair channels of a 768-token
        # crop, training
        _glu("glu_n768_k128_f128_sigmoid_train", 768 * 768, 128, 128, "train", act="sigmoid"),
        # the feed-forward block of a batch of single representations, training
        _glu("glu_m6001_k512_f2048_silu_train", 6001, 512, 2048, "train"),
        # fp32, odd sizes in every direction, backward
        _glu("glu_f32_m777_k129_f211_gelu_bwd", 777, 129, 211, "bwd", act="gelu", dtype="f32"),
        # the gradients of one block's norms and projections
        _clip("clip_14_tensors_f32", 14, 130000, "clip"),
        # the gradients of several blocks, matrices in bf16 and vectors and sums in fp32
        _clip("clip_60_tensors_mixed", 60, 64_000_000, "clip", dtype="mixed"),
        # one GPU's shard of flattened gradients: its norm alone
        _clip("norm_2_tensors_bf16", 2, 150_000_001, "norm", dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    if case["op"] == "att":  # the plain form's logits, too
        return max(w["bytes"], w["flops"] / 50, 14 * case["b"] * case["h"] * case["q"] * case["k"])
    return max(w["bytes"], w["flops"] / 50)


# a drawn call costs no more than the largest listed one
MAX_COST = {"att": 3.4e9, "glu": 1.5e9, "clip": 6e8}


def draw(rng):
    op = rng.choice(["att", "att", "att", "glu", "glu", "clip"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if op == "att":
        hk = rng.choice([1, 2, 4, 8, 16, rng.randint(1, 12)])
        h = hk * rng.choice([1, 1, 1, 2, 4, rng.randint(1, 8)])
        case = _att("", rng.choice([1, 2, _log_int(rng, 1, 800)]), _log_int(rng, 1, 4096),
                    _log_int(rng, 1, 32000), h, rng.choice([8, 16, 24, 32, 32, 48, 64, 64, 96, 128]),
                    rng.choice(["fwd", "train"]), hk, rng.choice(["none", "none", "shared", "each"]),
                    rng.choice([True, False]), dtype)
        shrink = ["b", "q", "k"]
    elif op == "glu":
        k, f = (rng.choice([_log_int(rng, 1, 2048), 8 * _log_int(rng, 1, 256), 128])
                for _ in range(2))
        case = _glu("", _log_int(rng, 1, 600000), k, f, rng.choice(["fwd", "bwd", "train"]),
                    rng.choice(["sigmoid", "silu", "gelu", "relu"]), dtype, rng.choice([True, False]))
        shrink = ["m"]
    else:
        count = _log_int(rng, 1, 60)
        case = _clip("", count, _log_int(rng, 400, 160_000_000), rng.choice(["norm", "clip", "clip"]),
                     rng.choice(["f32", "bf16", "mixed"]), rng.choice([0.01, 0.5, 3.0]))
        shrink = ["total"]
    while _cost(case) > MAX_COST[op]:
        at = max(shrink, key=lambda s: case[s])
        case[at] = max(1, case[at] * 7 // 8)
    del case["name"]
    return case


# ---- inputs ------------------------------------------------------------------------

def _normal(gen, shape, std=1.0, mean=0.0, dtype=torch.bfloat16):
    t = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)
    return t.mul_(std).add_(mean).to(dtype)


def _sizes(case):
    """Elements of each gradient: a few large matrices hold most, vectors the rest."""
    rng = random.Random(case["count"] * 1_000_003 + case["total"])
    weight = [math.exp(rng.uniform(0.0, math.log(2000.0))) for _ in range(case["count"])]
    each = [max(1, int(case["total"] * w / sum(weight))) for w in weight]
    each[0] += max(0, case["total"] - sum(each))
    return each


def _grad_dtype(case, i, size):
    if case["dtype"] == "mixed":
        small = size < 0.2 * case["total"] / case["count"]
        return torch.float32 if small or i % 5 == 0 else torch.bfloat16
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _inputs(case, seed):
    gen = torch.Generator("cuda").manual_seed(int(seed))
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    s = {"case": dict(case)}
    if case["op"] == "att":
        b, q, k, h, hk, d = (case[x] for x in ("b", "q", "k", "h", "hk", "d"))
        s["q"] = _normal(gen, (b, q, h, d), dtype=dt)
        s["k"] = _normal(gen, (b, k, hk, d), dtype=dt)
        s["v"] = _normal(gen, (b, k, hk, d), dtype=dt)
        lead = {"none": None, "shared": (), "each": (b,)}[case["bias"]]
        s["bias"] = None if lead is None else _normal(gen, lead + (q, k, h), dtype=dt)
        s["mask"] = None
        if case["mask"]:  # states past a sequence's length
            length = torch.randint((k + 1) // 2, k + 1, (b, 1), generator=gen, device="cuda")
            s["mask"] = (torch.arange(k, device="cuda")[None, :] < length).to(torch.uint8)
        s["dout"] = _normal(gen, (b, q, h, d), dtype=dt) if case["mode"] == "train" else None
    elif case["op"] == "glu":
        m, k, f = case["m"], case["k"], case["f"]
        s["x"] = _normal(gen, (m, k), dtype=dt)
        s["w"] = _normal(gen, (k, 2 * f), 1.0 / math.sqrt(k), dtype=dt)
        s["bias"] = _normal(gen, (2 * f,), 0.2, dtype=dt) if case["bias"] else None
        s["dout"] = _normal(gen, (m, f), dtype=dt) if case["mode"] != "fwd" else None
    else:
        each = _sizes(case)
        flat = _normal(gen, (sum(each),), 0.01, dtype=torch.float32)
        s["grads"] = [t.to(_grad_dtype(case, i, t.numel()), copy=True)
                      for i, t in enumerate(torch.split(flat, each))]
        s["clipped"] = [torch.empty_like(t) for t in s["grads"]] if case["mode"] == "clip" else None
        s["limit"] = case["ratio"] * 0.01 * math.sqrt(sum(each))
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own and case["op"] == "clip":
        # a training program keeps its gradients' lists from step to step
        from paper_2506_20686_amd import binding as B
        s["grads_list"] = B.GradList(s["grads"])
        s["clipped_list"] = B.GradList(s["clipped"]) if s["clipped"] else None
    return s


# ---- one pass: the framework's calls -------------------------------------------------

def _own_att(B, s, case):
    out, stat = B.cross_attn_fwd(s["q"], s["k"], s["v"], s["bias"], s["mask"])
    if case["mode"] == "fwd":
        return out, stat
    return (out, stat, *B.cross_attn_bwd(s["q"], s["k"], s["v"], out, stat, s["dout"], s["bias"],
                                         s["mask"]))


def _own_glu(B, s, case):
    act = {"relu": B.ACT_RELU, "gelu": B.ACT_GELU, "silu": B.ACT_SILU,
           "sigmoid": B.ACT_SIGMOID}[case["act"]]
    got = ()
    if case["mode"] != "bwd":
        got = (B.gated_linear_fwd(s["x"], s["w"], s["bias"], act),)
    if case["mode"] != "fwd":
        got += tuple(B.gated_linear_bwd(s["x"], s["w"], s["dout"], s["bias"], act))
    return got


def _own_clip(B, s, case):
    norm = B.grad_norm(s["grads_list"])
    if case["mode"] == "norm":
        return norm
    B.grad_clip(s["grads_list"], norm, s["limit"], s["clipped_list"])
    return norm, s["clipped"]


# ---- one pass: the plain forms --------------------------------------------------------

def _plain_att(s, case):
    b, nq, nk, h, hk, d = (case[x] for x in ("b", "q", "k", "h", "hk", "d"))
    g, dt, scale = h // hk, s["q"].dtype, 1.0 / math.sqrt(d)
    # heads first; the g query heads of a key head one after the other
    q = s["q"].float().view(b, nq, hk, g, d).permute(0, 2, 3, 1, 4).reshape(b, hk, g * nq, d)
    k = s["k"].float().permute(0, 2, 1, 3).contiguous()
    v = s["v"].float().permute(0, 2, 1, 3).contiguous()
    x = torch.matmul(q, k.transpose(2, 3).contiguous()).view(b, h, nq, nk) * scale
    if s["bias"] is not None:
        x = x + (s["bias"].float().permute(2, 0, 1)[None] if case["bias"] == "shared"
                 else s["bias"].float().permute(0, 3, 1, 2))
    if s["mask"] is not None:
        x = x.masked_fill(s["mask"][:, None, None, :] == 0, -math.inf)
    top = x.amax(dim=3, keepdim=True)
    p = torch.exp(x - top)
    total = p.sum(dim=3, keepdim=True)
    p = p / total
    stat = torch.cat([top, torch.log(total)], dim=3).permute(0, 2, 1, 3).contiguous()
    out = torch.matmul(p.view(b, hk, g * nq, nk), v).view(b, h, nq, d).permute(0, 2, 1, 3)
    out = out.to(dt).contiguous()
    if case["mode"] == "fwd":
        return out, stat
    do = s["dout"].float().view(b, nq, hk, g, d).permute(0, 2, 3, 1, 4).reshape(b, hk, g * nq, d)
    dp = torch.matmul(do, v.transpose(2, 3).contiguous()).view(b, h, nq, nk)
    ds = p * (dp - (p * dp).sum(dim=3, keepdim=True))
    flat = ds.view(b, hk, g * nq, nk)
    dq = (torch.matmul(flat, k) * scale).view(b, h, nq, d).permute(0, 2, 1, 3).to(dt).contiguous()
    turned = flat.transpose(2, 3).contiguous()
    dk = (torch.matmul(turned, q) * scale).permute(0, 2, 1, 3).to(dt).contiguous()
    turned = p.view(b, hk, g * nq, nk).transpose(2, 3).contiguous()
    dv = torch.matmul(turned, do).permute(0, 2, 1, 3).to(dt).contiguous()
    dbias = None
    if case["bias"] == "shared":
        dbias = ds.sum(dim=0).permute(1, 2, 0).to(dt).contiguous()
    elif case["bias"] == "each":
        dbias = ds.permute(0, 2, 3, 1).to(dt).contiguous()
    return out, stat, dq, dk, dv, dbias


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    sig = 1.0 / (1.0 + torch.exp(-z))
    return z * sig if act == "silu" else sig


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        cdf = 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
        return cdf + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    sig = 1.0 / (1.0 + torch.exp(-z))
    return sig * (1.0 + z * (1.0 - sig)) if act == "silu" else sig * (1.0 - sig)


def _plain_glu(s, case):
    x, w, dt, f, got = s["x"].float(), s["w"].float(), s["x"].dtype, case["f"], ()
    z = torch.matmul(x, w)
    if s["bias"] is not None:
        z = z + s["bias"].float()
    a, b = z[:, :f], z[:, f:]
    if case["mode"] != "bwd":
        got = ((_act(a, case["act"]) * b).to(dt),)
    if case["mode"] != "fwd":
        dy = s["dout"].float()
        dz = torch.cat([dy * b * _act_grad(a, case["act"]), dy * _act(a, case["act"])], dim=1)
        got += (torch.matmul(dz, w.t()).to(dt), torch.matmul(x.t(), dz), dz.sum(dim=0))
    return got


def _plain_clip(s, case):
    square = [(g.float() * g.float()).sum(dtype=torch.float64) for g in s["grads"]]
    norm = torch.sqrt(torch.stack(square).sum()).float()
    if case["mode"] == "norm":
        return norm
    factor = torch.where(norm > s["limit"], s["limit"] / norm, torch.ones_like(norm))
    return norm, [(g.float() * factor).to(g.dtype) for g in s["grads"]]


def run(state):
    s, case = state, state["case"]
    if own:
        from paper_2506_20686_amd import binding as B
        return {"att": _own_att, "glu": _own_glu, "clip": _own_clip}[case["op"]](B, s, case)
    return {"att": _plain_att, "glu": _plain_glu, "clip": _plain_clip}[case["op"]](s, case)


# ---- what a pass cannot do without ---------------------------------------------------

def work(case):
    """Bytes: every input read once, every output written once.  Flops: products and sums
    (attention: two products forward, five backward; the gated projection's backward three,
    one of them the forward's again)."""
    e, mode = 4 if case["dtype"] == "f32" else 2, case["mode"]
    if case["op"] == "att":
        b, q, k, h, hk, d = (case[x] for x in ("b", "q", "k", "h", "hk", "d"))
        maps = {"none": 0, "shared": q * k * h, "each": b * q * k * h}[case["bias"]]
        nbytes = (2 * b * q * h * d + 2 * b * k * hk * d + maps) * e + 8 * b * q * h
        nbytes += b * k if case["mask"] else 0
        if mode == "train":
            nbytes += (2 * b * q * h * d + 2 * b * k * hk * d + maps) * e
        return {"bytes": nbytes, "flops": 2 * b * h * q * k * d * (7 if mode == "train" else 2)}
    if case["op"] == "glu":
        m, k, f = case["m"], case["k"], case["f"]
        nbytes = (m * k + 2 * k * f) * e + 2 * f * e * case["bias"]
        nbytes += m * f * e * ((mode != "bwd") + (mode != "fwd"))
        if mode != "fwd":
            nbytes += m * k * e + 4 * (2 * k * f + 2 * f)
        return {"bytes": nbytes, "flops": 4 * m * k * f * {"fwd": 1, "bwd": 3, "train": 4}[mode]}
    nbytes, elements = 4, 0
    for i, n in enumerate(_sizes(case)):
        nbytes += n * _grad_dtype(case, i, n).itemsize * (2 if mode == "clip" else 1)
        elements += n
    return {"bytes": nbytes, "flops": elements * (3 if mode == "clip" else 2)}


# ---- the same in 64 bits, from the definitions -----------------------------------------

def _exact_att(case, s):
    f8, b, nq, h, hk, d = torch.float64, case["b"], case["q"], case["h"], case["hk"], case["d"]
    train, g = case["mode"] == "train", case["h"] // case["hk"]
    new = lambda t: torch.zeros(t.shape, dtype=f8, device="cuda")  # noqa: E731
    out, stat = new(s["q"]), torch.zeros((b, nq, h, 2), dtype=f8, device="cuda")
    dq, dk, dv = (new(s[x]) for x in "qkv") if train else (None, None, None)
    db = new(s["bias"]) if train and s["bias"] is not None else None
    # one head of as many samples at a time as leave room
    step = max(1, (1 << 26) // (nq * case["k"]))
    for b0 in range(0, b, step):
        at = slice(b0, min(b, b0 + step))
        for i in range(h):
            qi, ki, vi = (s[x][at, :, j].to(f8).contiguous() for x, j in
                          (("q", i), ("k", i // g), ("v", i // g)))
            logit = torch.bmm(qi, ki.mT.contiguous()) / math.sqrt(d)
            if s["bias"] is not None:
                logit += (s["bias"][None, :, :, i] if case["bias"] == "shared"
                          else s["bias"][at, :, :, i]).to(f8)
            if s["mask"] is not None:
                logit = torch.where(s["mask"][at, None, :] > 0, logit, torch.full_like(logit, -math.inf))
            lse = torch.logsumexp(logit, dim=2, keepdim=True)
            most = torch.max(logit, dim=2, keepdim=True).values
            p = torch.exp(logit - lse)
            out[at, :, i] = torch.bmm(p, vi)
            stat[at, :, i] = torch.cat([most, lse - most], dim=2)
            if train:
                do = s["dout"][at, :, i].to(f8).contiguous()
                dv[at, :, i // g] += torch.bmm(p.mT.contiguous(), do)
                # the softmax's Jacobian, with sum P dP as the output's product with dout
                ds = torch.bmm(do, vi.mT.contiguous()) - (do * out[at, :, i]).sum(2, keepdim=True)
                ds *= p
                dq[at, :, i] = torch.bmm(ds, ki) / math.sqrt(d)
                dk[at, :, i // g] += torch.bmm(ds.mT.contiguous(), qi) / math.sqrt(d)
                if case["bias"] == "shared":
                    db[:, :, i] += ds.sum(dim=0)
                elif db is not None:
                    db[at, :, :, i] = ds
    return [out, stat] + ([dq, dk, dv, db] if train else [])


def _exact_act(z, act):
    """(value, derivative) of the activation."""
    if act == "relu":
        on = torch.gt(z, 0).to(z.dtype)
        return z * on, on
    if act == "gelu":
        phi = torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
        cdf = torch.erfc(-z / math.sqrt(2)) / 2
        return z * cdf, cdf + z * phi
    sig, other = torch.sigmoid(z), torch.sigmoid(-z)
    return (z * sig, sig + z * sig * other) if act == "silu" else (sig, sig * other)


def _exact_glu(case, s):
    f8, m, k, f, mode = torch.float64, case["m"], case["k"], case["f"], case["mode"]
    wa, wb = s["w"][:, :f].to(f8).contiguous(), s["w"][:, f:].to(f8).contiguous()
    wat, wbt = wa.t().contiguous(), wb.t().contiguous()
    zero = torch.zeros(2 * f, dtype=f8, device="cuda")
    ba, bb = torch.split(zero if s["bias"] is None else s["bias"].to(f8), f)
    dw, db = torch.zeros((k, 2 * f), dtype=f8, device="cuda"), torch.zeros_like(zero)
    outs, dxs = [], []
    step = max(1, (1 << 23) // max(k, 2 * f))
    for r in range(0, m, step):
        x = s["x"][r:r + step].to(f8)
        a, b = torch.addmm(ba, x, wa), torch.addmm(bb, x, wb)
        value, slope = _exact_act(a, case["act"])
        if mode != "bwd":
            outs.append(value * b)
        if mode != "fwd":
            dy = s["dout"][r:r + step].to(f8)
            da, dbv = dy * b * slope, dy * value
            dxs.append(da @ wat + dbv @ wbt)
            xt = x.t().contiguous()
            dw[:, :f] += xt @ da
            dw[:, f:] += xt @ dbv
            db[:f] += da.sum(dim=0)
            db[f:] += dbv.sum(dim=0)
    res = [torch.cat(outs)] if mode != "bwd" else []
    return res + [torch.cat(dxs), dw, db] if mode != "fwd" else res


def _exact_clip(case, s):
    each = [torch.linalg.vector_norm(g.to(torch.float64)) for g in s["grads"]]
    norm = torch.linalg.vector_norm(torch.stack(each))
    if case["mode"] == "norm":
        return norm
    factor = min(1.0, s["limit"] / float(norm))
    return norm, [g.to(torch.float64) * factor for g in s["grads"]]


def exact(case, seed):
    return {"att": _exact_att, "glu": _exact_glu, "clip": _exact_clip}[case["op"]](
        case, _inputs(case, seed))
