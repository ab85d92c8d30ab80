"""Layer norm, the linear projection with its epilogue and the relative position
bias, as measurable cases.

A case is a dict of plain values.  "op" names the operator:

  ln   layer norm over rows of any width (binding.layer_norm_fwd / _bwd)
  lin  out = act(x W + bias) + residual and its gradients
       (binding.linear_fwd / _bwd)
  rel  a learned bias of h channels per pair of tokens, by buckets of the
       difference of their positions (binding.rel_bias_fwd / _bwd)

and "mode" is what the caller does with it: "fwd" (a forward), "bwd" (a
backward, given what the forward saved) or "train" (both, one after the
other).  Where `own` is false a pass computes the operator in its plain form.
"""
import math

import torch

own = False

EPS = 1e-5


def _ln(name, m, c, mode, dtype="bf16", affine=True):
    return {"name": name, "op": "ln", "mode": mode, "dtype": dtype, "m": m, "c": c,
            "affine": affine}


def _lin(name, m, k, n, mode, act="none", dtype="bf16", bias=True, residual=False, save_z=False):
    return {"name": name, "op": "lin", "mode": mode, "dtype": dtype, "m": m, "k": k, "n": n,
            "act": act, "bias": bias, "residual": residual, "save_z": save_z}


def _rel(name, n, h, mode, dtype="bf16", batch=1, exact=32, far=0, steps=0, chains=1, base=False):
    return {"name": name, "op": "rel", "mode": mode, "dtype": dtype, "batch": batch, "n": n, "h": h,
            "exact": exact, "far": far, "steps": steps, "chains": chains, "base": base}


def listed():
    return [
        # the single representation of a short peptide, fp32: nothing but latency
        _ln("ln_f32_m48_c384_fwd", 48, 384, "fwd", dtype="f32"),
        # the pair representation of a 768-token crop, training
        _ln("ln_n768_c128_train", 768 * 768, 128, "train"),
        # rows of an odd width (concatenated features), a ragged number of them, training
        _ln("ln_m9001_c833_train", 9001, 833, "train"),
        # the projection from the attention's output back to the pair channels, with
        # the residual stream added, at 768 tokens: inference
        _lin("lin_n768_k128_n128_res_fwd", 768 * 768, 128, 128, "fwd", residual=True),
        # the same, training: the largest call
        _lin("lin_n768_k128_n128_res_train", 768 * 768, 128, 128, "train", residual=True),
        # one row, inference: the hidden layer of a single token
        _lin("lin_m1_k384_n1536_silu_fwd", 1, 384, 1536, "fwd", act="silu"),
        # the hidden layer of the single representation of a long complex, backward
        _lin("lin_m1500_k384_n1536_gelu_bwd", 1500, 384, 1536, "bwd", act="gelu"),
        # fp32, odd sizes in every direction, backward
        _lin("lin_f32_m2777_k449_n131_relu_bwd", 2777, 449, 131, "bwd", act="relu", dtype="f32"),
        # the bias of a short peptide's attention, fp32: nothing but latency
        _rel("rel_f32_n40_h4_fwd", 40, 4, "fwd", dtype="f32"),
        # the attention's bias at 768 tokens (a complex of four chains), added to the
        # projected pair bias, with the table's gradient: training
        _rel("rel_n768_h4_base_train", 768, 4, "train", chains=4, base=True),
        # a long complex, 16 heads, buckets that widen with the distance: backward
        _rel("rel_n1536_h16_far_bwd", 1536, 16, "bwd", exact=16, far=512, steps=16, chains=2),
        # the position term of the pair representation (128 channels), a batch of
        # ragged maps: training
        _rel("rel_b2_n333_h128_train", 333, 128, "train", batch=2, chains=3),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


# a drawn call costs no more than the largest listed one
MAX_COST = 1.1e9


def draw(rng):
    op = rng.choice(["ln", "lin", "lin", "rel"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if op == "ln":
        c = rng.choice([_log_int(rng, 1, 4096), 8 * _log_int(rng, 1, 512), 128])
        case = _ln("", _log_int(rng, 1, 600000), c, rng.choice(["fwd", "train"]), dtype,
                   rng.choice([True, True, True, False]))
        shrink = "m"
    elif op == "lin":
        k, n = (rng.choice([_log_int(rng, 1, 2048), 8 * _log_int(rng, 1, 256), 128])
                for _ in range(2))
        act = rng.choice(["none", "none", "relu", "gelu", "silu"])
        mode = rng.choice(["fwd", "bwd", "train"] if act == "none" else ["fwd", "bwd"])
        case = _lin("", _log_int(rng, 1, 600000), k, n, mode, act, dtype,
                    rng.choice([True, True, False]), rng.choice([True, False]),
                    mode == "fwd" and rng.choice([True, False]))
        shrink = "m"
    else:
        exact = rng.choice([32, 32, rng.randint(1, 100)])
        steps = rng.choice([0, 0, rng.randint(1, 24)])
        case = _rel("", _log_int(rng, 1, 2048), rng.choice([4, 4, 8, 16, 128, rng.randint(1, 64)]),
                    rng.choice(["fwd", "bwd", "train"]), dtype, rng.choice([1, 1, 1, 2, 3]), exact,
                    exact * rng.randint(4, 40) if steps else 0, steps, rng.choice([1, 2, 5]),
                    rng.choice([True, False]))
        shrink = "n"
    while _cost(case) > (MAX_COST if op != "rel" else 2e8):
        case[shrink] = case[shrink] * 7 // 8
    del case["name"]
    return case


# ---- inputs ------------------------------------------------------------------------

def _normal(gen, shape, std=1.0, mean=0.0, dtype=torch.bfloat16):
    t = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)
    return t.mul_(std).add_(mean).to(dtype)


def _edges(case):
    """Upper borders of the buckets: differences up to `exact` apart have a bucket of
    their own, up to `far` in `steps` geometric steps, further ones share the last."""
    top = [float(case["exact"])]
    for i in range(case["steps"]):
        top.append(case["exact"] * (case["far"] / case["exact"]) ** ((i + 1) / case["steps"]))
    far = sorted({int(math.ceil(t)) for t in top[1:]})
    up = list(range(1, case["exact"] + 1)) + far
    return [1 - e for e in reversed(up)] + up


def _rows(case):
    return len(_edges(case)) + 1 + (1 if case["chains"] > 1 else 0)


def _tokens(gen, case):
    """Residue numbers and chains of a complex: each chain counts from 1; about one
    token in twenty repeats the number before it, as an atom of the same residue."""
    b, n = case["batch"], case["n"]
    cuts = torch.sort(torch.randint(1, max(n, 2), (b, case["chains"] - 1), generator=gen,
                                    device="cuda"), dim=1).values
    at = torch.arange(n, device="cuda")
    chain = (at[None, :, None] >= cuts[:, None, :]).sum(dim=2)
    step = (torch.rand((b, n), generator=gen, device="cuda") >= 0.05).to(torch.int64)
    count = torch.cumsum(step, dim=1)
    first = torch.cat([torch.zeros((b, 1), dtype=torch.int64, device="cuda"), cuts], dim=1)
    start = torch.gather(count, 1, torch.clamp(torch.gather(first, 1, chain), max=n - 1))
    return (count - start + 1).to(torch.int32), chain.to(torch.int32)


def _inputs(case, seed):
    gen = torch.Generator("cuda").manual_seed(int(seed))
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    s = {"case": dict(case)}
    if case["op"] == "ln":
        m, c = case["m"], case["c"]
        s["x"] = _normal(gen, (m, c), 1.5, 0.3, dt)
        s["gamma"] = _normal(gen, (c,), 0.2, 1.0, dt) if case["affine"] else None
        s["beta"] = _normal(gen, (c,), 0.2, 0.0, dt) if case["affine"] else None
        s["dout"] = _normal(gen, (m, c), dtype=dt) if case["mode"] == "train" else None
    elif case["op"] == "lin":
        m, k, n, mode = case["m"], case["k"], case["n"], case["mode"]
        s["x"] = _normal(gen, (m, k), dtype=dt)
        s["w"] = _normal(gen, (k, n), 1.0 / math.sqrt(k), dtype=dt)
        fwd = mode != "bwd"
        s["bias"] = _normal(gen, (n,), 0.2, dtype=dt) if case["bias"] and fwd else None
        s["residual"] = _normal(gen, (m, n), 1.5, dtype=dt) if case["residual"] and fwd else None
        s["z"] = _normal(gen, (m, n), dtype=dt) if not fwd and case["act"] != "none" else None
        s["dout"] = _normal(gen, (m, n), dtype=dt) if mode != "fwd" else None
    else:
        b, n, h, mode = case["batch"], case["n"], case["h"], case["mode"]
        s["pos"], chain = _tokens(gen, case)
        s["chain"] = chain if case["chains"] > 1 else None
        s["edges"] = _edges(case)
        s["borders"] = torch.tensor(s["edges"], dtype=torch.int64, device="cuda")
        s["table"] = _normal(gen, (_rows(case), h), dtype=dt)
        fwd = mode != "bwd"
        s["base"] = _normal(gen, (b, n, n, h), dtype=dt) if case["base"] and fwd else None
        s["dbias"] = _normal(gen, (b, n, n, h), dtype=dt) if mode != "fwd" else None
    return s


def prepare(case, seed):
    return _inputs(case, seed)


# ---- one pass: the framework's calls -------------------------------------------------

def _own_ln(B, s, train):
    out, mean, rstd = B.layer_norm_fwd(s["x"], s["gamma"], s["beta"], EPS)
    if not train:
        return out, mean, rstd
    return (out, mean, rstd, *B.layer_norm_bwd(s["x"], s["gamma"], mean, rstd, s["dout"]))


def _own_lin(B, s, case):
    act = {"none": B.ACT_NONE, "relu": B.ACT_RELU, "gelu": B.ACT_GELU, "silu": B.ACT_SILU}
    act, got = act[case["act"]], ()
    if case["mode"] != "bwd":
        got = B.linear_fwd(s["x"], s["w"], s["bias"], s["residual"], act, case["save_z"])
    if case["mode"] != "fwd":
        got += B.linear_bwd(s["x"], s["w"], s["dout"], s["z"], act)
    return got


def _own_rel(B, s, case):
    got = ()
    if case["mode"] != "bwd":
        got = (B.rel_bias_fwd(s["pos"], s["edges"], s["table"], s["chain"], s["base"]),)
    if case["mode"] != "fwd":
        got += (B.rel_bias_bwd(s["pos"], s["edges"], s["dbias"], s["chain"]),)
    return got


# ---- one pass: the plain forms --------------------------------------------------------

def _plain_ln(s, train):
    x = s["x"].float()
    mean = x.mean(dim=1)
    d = x - mean[:, None]
    rstd = torch.rsqrt((d * d).mean(dim=1) + EPS)
    xhat = d * rstd[:, None]
    o = xhat
    if s["gamma"] is not None:
        o = xhat * s["gamma"].float() + s["beta"].float()
    out = o.to(s["x"].dtype)
    if not train:
        return out, mean, rstd
    dy = s["dout"].float()
    w = dy * s["gamma"].float() if s["gamma"] is not None else dy
    c1, c2 = (w * xhat).mean(dim=1, keepdim=True), w.mean(dim=1, keepdim=True)
    dx = ((w - c1 * xhat - c2) * rstd[:, None]).to(s["x"].dtype)
    return out, mean, rstd, dx, (dy * xhat).sum(dim=0), dy.sum(dim=0)


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        cdf = 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
        return cdf + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    sig = 1.0 / (1.0 + torch.exp(-z))
    return sig * (1.0 + z * (1.0 - sig))


def _plain_lin(s, case):
    x, w, dt, got = s["x"].float(), s["w"].float(), s["x"].dtype, ()
    if case["mode"] != "bwd":
        z = torch.matmul(x, w)
        if s["bias"] is not None:
            z = z + s["bias"].float()
        out = _act(z, case["act"])
        if s["residual"] is not None:
            out = out + s["residual"].float()
        got = (out.to(dt), z.to(dt) if case["save_z"] else None)
    if case["mode"] != "fwd":
        dz = s["dout"].float()
        if case["act"] != "none":
            dz = dz * _act_grad(s["z"].float(), case["act"])
        dx = torch.matmul(dz, w.t()).to(dt)
        got += (dx, torch.matmul(x.t(), dz), dz.sum(dim=0))
    return got


def _buckets(s):
    d = s["pos"].long()[:, :, None] - s["pos"].long()[:, None, :]
    b = torch.bucketize(d, s["borders"], right=True)
    if s["chain"] is not None:
        b = torch.where(s["chain"][:, :, None] == s["chain"][:, None, :], b,
                        torch.full_like(b, len(s["edges"]) + 1))
    return b


def _plain_rel(s, case):
    got = ()
    b = _buckets(s)
    if case["mode"] != "bwd":
        out = s["table"].float()[b]
        if s["base"] is not None:
            out = out + s["base"].float()
        got = (out.to(s["table"].dtype),)
    if case["mode"] != "fwd":
        # per query the sums of a bucket's keys as a product with zeros and ones, then
        # the long sum over the queries in 64 bits
        rows = torch.arange(_rows(case), device="cuda")
        member = (b[:, :, None, :] == rows[None, None, :, None]).float()
        part = torch.matmul(member, s["dbias"].float())
        got += (part.sum(dim=(0, 1), dtype=torch.float64).float(),)
    return got


def run(state):
    s, case = state, state["case"]
    if own:
        from paper_2506_20686_amd import binding as B
        if case["op"] == "ln":
            return _own_ln(B, s, case["mode"] == "train")
        return _own_lin(B, s, case) if case["op"] == "lin" else _own_rel(B, s, case)
    if case["op"] == "ln":
        return _plain_ln(s, case["mode"] == "train")
    return _plain_lin(s, case) if case["op"] == "lin" else _plain_rel(s, case)


# ---- what a pass cannot do without ---------------------------------------------------

def work(case):
    """Bytes: every input read once, every output written once.  Flops: products and
    sums (layer norm: 8 an element forward, 14 backward)."""
    e, mode = 4 if case["dtype"] == "f32" else 2, case["mode"]
    if case["op"] == "ln":
        m, c = case["m"], case["c"]
        nbytes = 2 * m * c * e + 8 * m + (2 * c * e if case["affine"] else 0)
        if mode == "train":
            nbytes += 2 * m * c * e + 8 * c
        return {"bytes": nbytes, "flops": (22 if mode == "train" else 8) * m * c}
    if case["op"] == "lin":
        m, k, n = case["m"], case["k"], case["n"]
        nbytes = (m * k + k * n) * e
        if mode != "bwd":
            nbytes += m * n * e * (1 + case["residual"] + case["save_z"]) + n * e * case["bias"]
        if mode != "fwd":
            nbytes += (m * n * (1 + (case["act"] != "none")) + m * k) * e + 4 * (k * n + n)
        return {"bytes": nbytes, "flops": 2 * m * k * n * {"fwd": 1, "bwd": 2, "train": 3}[mode]}
    b, n, h, r = case["batch"], case["n"], case["h"], _rows(case)
    nbytes, pairs = 4 * b * n * (1 + (case["chains"] > 1)), b * n * n
    if mode != "bwd":
        nbytes += pairs * h * e * (1 + case["base"]) + r * h * e
    if mode != "fwd":
        nbytes += pairs * h * e + 4 * r * h
    flops = pairs * h * ((mode != "bwd") * case["base"] + (mode != "fwd")) + pairs
    return {"bytes": nbytes, "flops": flops}


# ---- the same in 64 bits, from the definitions -----------------------------------------

def _exact_ln(case, s):
    f8, m, c = torch.float64, case["m"], case["c"]
    g = s["gamma"].to(f8) if case["affine"] else torch.ones(c, dtype=f8, device="cuda")
    sh = s["beta"].to(f8) if case["affine"] else torch.zeros(c, dtype=f8, device="cuda")
    rows, dg, db = [], torch.zeros_like(g), torch.zeros_like(g)
    step = max(1, (1 << 23) // c)
    for a in range(0, m, step):
        x = s["x"][a:a + step].to(f8)
        var, mean = torch.var_mean(x, dim=1, unbiased=False)
        sd = torch.sqrt(var + EPS)
        xh = (x - mean[:, None]) / sd[:, None]
        got = [torch.addcmul(sh, xh, g), mean, 1.0 / sd]
        if case["mode"] == "train":
            dy = s["dout"][a:a + step].to(f8)
            dxh = dy * g
            # the normalisation's Jacobian: (I - 11^T / c - xh xh^T / c) / sd
            along = (dxh * xh).sum(dim=1, keepdim=True) / c
            got.append((dxh - dxh.sum(dim=1, keepdim=True) / c - xh * along) / sd[:, None])
            dg += (dy * xh).sum(dim=0)
            db += dy.sum(dim=0)
        rows.append(got)
    res = [torch.cat(t) for t in zip(*rows)]
    return res + [dg, db] if case["mode"] == "train" else res


def _exact_act(z, act):
    """(value, derivative) of the activation."""
    if act == "relu":
        on = torch.gt(z, 0).to(z.dtype)
        return z * on, on
    if act == "gelu":
        phi = torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
        cdf = torch.erfc(-z / math.sqrt(2)) / 2
        return z * cdf, cdf + z * phi
    if act == "silu":
        sig = torch.sigmoid(z)
        return z * sig, sig + z * sig * torch.sigmoid(-z)
    return z, torch.ones_like(z)


def _exact_lin(case, s):
    f8, m, k, n, mode = torch.float64, case["m"], case["k"], case["n"], case["mode"]
    w = s["w"].to(f8)
    wt = w.t().contiguous()
    dw = torch.zeros((k, n), dtype=f8, device="cuda")
    db = torch.zeros(n, dtype=f8, device="cuda")
    outs, zs, dxs = [], [], []
    step = max(1, (1 << 23) // max(k, n))
    for a in range(0, m, step):
        x = s["x"][a:a + step].to(f8)
        if mode != "bwd":
            z = x @ w
            if s["bias"] is not None:
                z += s["bias"].to(f8)
            o = _exact_act(z, case["act"])[0]
            if s["residual"] is not None:
                o = o + s["residual"][a:a + step].to(f8)
            outs.append(o)
            zs.append(z if case["save_z"] else None)
        if mode != "fwd":
            dz = s["dout"][a:a + step].to(f8)
            if case["act"] != "none":
                dz = dz * _exact_act(s["z"][a:a + step].to(f8), case["act"])[1]
            dxs.append(dz @ wt)
            dw += x.t().contiguous() @ dz
            db += dz.sum(dim=0)
    res = []
    if mode != "bwd":
        res += [torch.cat(outs), torch.cat(zs) if case["save_z"] else None]
    return res + [torch.cat(dxs), dw, db] if mode != "fwd" else res


def _exact_rel(case, s):
    f8, mode, res = torch.float64, case["mode"], []
    d = s["pos"].long()[:, :, None] - s["pos"].long()[:, None, :]
    bucket = torch.zeros_like(d)
    for e in s["edges"]:
        bucket += d >= e
    if s["chain"] is not None:
        bucket[s["chain"][:, :, None] != s["chain"][:, None, :]] = len(s["edges"]) + 1
    if mode != "bwd":
        out = torch.index_select(s["table"].to(f8), 0, bucket.reshape(-1))
        out = out.reshape(case["batch"], case["n"], case["n"], case["h"])
        res.append(out + s["base"].to(f8) if s["base"] is not None else out)
    if mode != "fwd":
        flat, which = s["dbias"].reshape(-1, case["h"]), bucket.reshape(-1)
        res.append(torch.stack([flat[which == r].to(f8).sum(dim=0) for r in range(_rows(case))]))
    return res


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "ln":
        return _exact_ln(case, s)
    return _exact_lin(case, s) if case["op"] == "lin" else _exact_rel(case, s)
