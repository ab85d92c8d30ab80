"""The cross attention, the gated linear projection and the clipping of gradients as they
are used together: a block that reads states of another length, forward, backward
and clipped, against torch's 64-bit autograd; the same captured into a graph; two
streams; what the wrappers refuse on the GPU."""
import math

import pytest
import torch

import cross_ref as C
import ops_ref as R
from paper_2506_20686_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F8 = torch.bfloat16, torch.float64
H, D, W, F = 4, 24, 96, 80
EPS, LIMIT = 1e-5, 5.0
WEIGHTS = ("wq", "wk", "wv", "pair", "wo", "g", "b", "wg", "bg", "wd")


def inputs(b, nq, nk, seed):
    g = torch.Generator().manual_seed(seed)

    def normal(*shape, std=1.0, mean=0.0):
        return (torch.randn(*shape, generator=g) * std + mean).to(BF)

    mask = torch.ones(b, nk, dtype=torch.uint8)
    mask[0, nk - nk // 3:] = 0
    return {"x": normal(b * nq, W), "e": normal(b * nk, 40), "wq": normal(W, W, std=W ** -0.5),
            "wk": normal(40, W, std=40 ** -0.5), "wv": normal(40, W, std=40 ** -0.5),
            "pair": normal(nq, nk, H), "mask": mask, "wo": normal(W, W, std=W ** -0.5),
            "g": normal(W, std=0.2, mean=1.0), "b": normal(W, std=0.2),
            "wg": normal(W, 2 * F, std=W ** -0.5), "bg": normal(2 * F, std=0.2),
            "wd": normal(F, W, std=F ** -0.5), "dy": normal(b * nq, W)}


def block(t, b, nq, nk):
    """Outputs and gradients with the framework's calls, the weights' ones clipped."""
    q = B.linear_fwd(t["x"], t["wq"])[0].view(b, nq, H, D)
    k = B.linear_fwd(t["e"], t["wk"])[0].view(b, nk, H, D)
    v = B.linear_fwd(t["e"], t["wv"])[0].view(b, nk, H, D)
    o, stat = B.cross_attn_fwd(q, k, v, t["pair"], t["mask"])
    x2, _ = B.linear_fwd(o.view(b * nq, W), t["wo"], None, t["x"])
    y, mean, rstd = B.layer_norm_fwd(x2, t["g"], t["b"], EPS)
    u = B.gated_linear_fwd(y, t["wg"], t["bg"], B.ACT_SILU)
    out, _ = B.linear_fwd(u, t["wd"], None, x2)
    # backward
    du, dwd, _ = B.linear_bwd(u, t["wd"], t["dy"])
    dyn, dwg, dbg = B.gated_linear_bwd(y, t["wg"], du, t["bg"], B.ACT_SILU)
    dx2, dg, db = B.layer_norm_bwd(x2, t["g"], mean, rstd, dyn)
    dx2 = (dx2.float() + t["dy"].float()).to(BF)
    do, dwo, _ = B.linear_bwd(o.view(b * nq, W), t["wo"], dx2)
    dq, dk, dv, dpair = B.cross_attn_bwd(q, k, v, o, stat, do.view(b, nq, H, D), t["pair"],
                                         t["mask"])
    dx, dwq, _ = B.linear_bwd(t["x"], t["wq"], dq.view(b * nq, W))
    de, dwk, _ = B.linear_bwd(t["e"], t["wk"], dk.view(b * nk, W))
    de2, dwv, _ = B.linear_bwd(t["e"], t["wv"], dv.view(b * nk, W))
    grads = [dwq, dwk, dwv, dpair, dwo, dg, db, dwg, dbg, dwd]
    norm = B.grad_norm(grads)
    clipped = B.grad_clip(grads, norm, LIMIT, [torch.empty_like(a) for a in grads])
    return dict(zip(WEIGHTS, clipped), out=out, norm=norm, dx=dx.float() + dx2.float(),
                de=de.float() + de2.float())


def plain(t, b, nq, nk):
    p = {k: v.to(F8).requires_grad_(True) for k, v in t.items() if v.dtype == BF and k != "dy"}
    q = (p["x"] @ p["wq"]).view(b, nq, H, D)
    k, v = ((p["e"] @ p[w]).view(b, nk, H, D) for w in ("wk", "wv"))
    s = torch.einsum("bqhd,bkhd->bhqk", q, k) / math.sqrt(D) + p["pair"].permute(2, 0, 1)
    s = s.masked_fill((t["mask"] == 0)[:, None, None], -math.inf)
    o = torch.einsum("bhqk,bkhd->bqhd", torch.softmax(s, 3), v)
    x2 = o.reshape(b * nq, W) @ p["wo"] + p["x"]
    d = x2 - x2.mean(1, keepdim=True)
    y = d / torch.sqrt((d * d).mean(1, keepdim=True) + EPS) * p["g"] + p["b"]
    z = y @ p["wg"] + p["bg"]
    out = (C.act(z[:, :F], B.ACT_SILU) * z[:, F:]) @ p["wd"] + x2
    (out * t["dy"].to(F8)).sum().backward()
    norm = torch.sqrt(sum((p[w].grad ** 2).sum() for w in WEIGHTS))
    f = min(1.0, LIMIT / norm.item())
    assert f < 1
    got = {w: p[w].grad * f for w in WEIGHTS}
    return dict(got, out=out.detach(), norm=norm, dx=p["x"].grad, de=p["e"].grad)


@pytest.mark.parametrize("size", [(1, 7, 5), (2, 40, 70), (3, 33, 150)], ids=str)
def test_block(size):
    # some eight bf16 stages, each good to 2^-8 / sqrt(3) or, for the attention's gradients,
    # 3.5e-3 of an output's norm; their errors add in squares to under 1e-2
    t = inputs(*size, sum(size))
    got = block({k: v.to(DEV) for k, v in t.items()}, *size)
    ref = plain(t, *size)
    for k in ref:
        R.fro(k, got[k], ref[k], 2e-2)


def test_block_in_a_graph():
    # captured once, replayed on other inputs with the program's own work between
    size = (2, 40, 300)
    t = {k: v.to(DEV) for k, v in inputs(*size, 1).items()}
    other = {k: v.to(DEV) for k, v in inputs(*size, 2).items()}
    first = {k: v.clone() for k, v in t.items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block(t, *size)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = block(t, *size)
    for src in (other, first, other):
        want = block(src, *size)  # eager work between the replays
        for k in t:
            t[k].copy_(src[k])
        graph.replay()
        torch.cuda.synchronize()
        for k in out:
            assert torch.equal(out[k], want[k]), k


def test_two_graphs_with_one_workspace():
    g = torch.Generator(DEV).manual_seed(4)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV).to(BF)

    # loops that are split, a bias in planes and one summed over the samples: all of a workspace
    q, y, k, v = normal(3, 5, 4, 40), normal(3, 5, 4, 40), normal(3, 2000, 2, 40), \
        normal(3, 2000, 2, 40)
    bias, x, w, du = normal(5, 2000, 4), normal(300, 200), normal(200, 96), normal(300, 48)
    out, stat = B.cross_attn_fwd(q, k, v, bias)
    sizes = (B.BF16, 3, 5, 2000, 4, 2, 40, 1)
    need = max(B._sized("tri_cross_attn_fwd_workspace_bytes", *sizes),
               B._sized("tri_cross_attn_bwd_workspace_bytes", *sizes),
               B._sized("tri_gated_linear_bwd_workspace_bytes", B.BF16, 300, 200, 48))
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    calls = [lambda s: B.cross_attn_fwd(q, k, v, bias, workspace=s),
             lambda s: B.cross_attn_bwd(q, k, v, out, stat, y, bias, workspace=s),
             lambda s: B.gated_linear_bwd(x, w, du, workspace=s),
             lambda s: (B.grad_norm([x, w], s),)]
    graphs, got = [], []
    for call in calls:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got.append(call(ws))
        graphs.append(graph)
    want = [call(None) for call in calls]
    for _ in range(3):
        ws.fill_(255)
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            for s, t in zip(a, b):
                assert torch.equal(s, t)


def test_two_streams_at_once():
    size = (2, 40, 70)
    t = [{k: v.to(DEV) for k, v in inputs(*size, s).items()} for s in (5, 6)]
    want = [block(a, *size) for a in t]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in t], []
    for a, s in zip(t, streams):
        with torch.cuda.stream(s):
            got.append(block(a, *size))
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        for k in w:
            assert torch.equal(g[k], w[k]), k


def test_a_call_repeated_while_an_earlier_backward_waits():
    # two forwards' states alive at once, their backwards in the other order
    size = (2, 33, 64)
    sets = [{k: v.to(DEV) for k, v in inputs(*size, s).items()} for s in (7, 8)]

    saved = []
    for t in sets:
        b, nq, nk = size
        q = t["x"].view(b, nq, H, D)
        k = B.linear_fwd(t["e"], t["wk"])[0].view(b, nk, H, D)
        saved.append((q, k, k, *B.cross_attn_fwd(q, k, k, t["pair"], t["mask"])))
    grads = [B.cross_attn_bwd(*s, t["dy"].view_as(s[0]), t["pair"], t["mask"])
             for s, t in reversed(list(zip(saved, sets)))]
    for (s, t), g in zip(reversed(list(zip(saved, sets))), grads):
        ref, bound = C.attn_bwd(*(a.cpu() for a in s[:3]), t["dy"].view_as(s[0]).cpu(),
                                t["pair"].cpu(), t["mask"].cpu())
        for name, a, r, e in zip(("dq", "dk", "dv", "dbias"), g, ref, bound):
            R.check(name, a, r, e)


def test_wrappers_refuse_what_the_library_cannot_take():
    q = torch.randn(2, 6, 4, 16, device=DEV).to(BF)
    k = torch.randn(2, 9, 2, 16, device=DEV).to(BF)
    bias = torch.zeros(6, 9, 4, device=DEV, dtype=BF)
    mask = torch.ones(2, 9, device=DEV, dtype=torch.uint8)
    out, stat = B.cross_attn_fwd(q, k, k, bias, mask)
    x, w = torch.randn(6, 16, device=DEV).to(BF), torch.randn(16, 8, device=DEV).to(BF)
    for call in (lambda: B.cross_attn_fwd(q, k, k[:, :8]), lambda: B.cross_attn_fwd(q, k.float(), k),
                 lambda: B.cross_attn_fwd(q, k, k, bias[:, :8]),
                 lambda: B.cross_attn_fwd(q, k, k, bias[None]),
                 lambda: B.cross_attn_fwd(q, k, k, bias, mask.bool()),
                 lambda: B.cross_attn_fwd(q, k, k, bias, mask[0]),
                 lambda: B.cross_attn_fwd(q.transpose(1, 2), k, k),
                 lambda: B.cross_attn_fwd(q.half(), k.half(), k.half()),
                 lambda: B.cross_attn_fwd(q[0, 0], k[0, 0], k[0, 0]),
                 lambda: B.cross_attn_bwd(q, k, k, out, stat[..., 0], q),
                 lambda: B.cross_attn_bwd(q, k, k, out, stat, q[:1]),
                 lambda: B.gated_linear_fwd(x, w[:, :7].contiguous()),
                 lambda: B.gated_linear_fwd(x, w.t()), lambda: B.gated_linear_fwd(x, w, w[0, :4]),
                 lambda: B.gated_linear_bwd(x, w, x), lambda: B.gated_linear_fwd(x.cpu(), w.cpu()),
                 lambda: B.grad_norm([x, w.cpu()]), lambda: B.grad_norm([x.t()]),
                 lambda: B.grad_clip([x], B.grad_norm([x]), 1.0, [w]),
                 lambda: B.grad_clip([x], stat, 1.0), lambda: B.grad_norm([x, w, x]),
                 lambda: B.grad_clip([x], B.grad_norm([x]).double(), 1.0)):
        with pytest.raises(ValueError):
            call()
    for call, code in ((lambda: B.cross_attn_fwd(q[:, :0], k, k), B.ERR_INVALID_ARG),
                       (lambda: B.cross_attn_fwd(q, k[:, :0], k[:, :0]), B.ERR_INVALID_ARG),
                       (lambda: B.cross_attn_fwd(q, torch.cat([k, k[:, :, :1]], 2),
                                                 torch.cat([k, k[:, :, :1]], 2)),
                        B.ERR_INVALID_ARG),  # three key heads for four
                       (lambda: B.cross_attn_fwd(q, k, k, scale=0.0), B.ERR_INVALID_ARG),
                       (lambda: B.cross_attn_fwd(q[..., :12].contiguous(), k[..., :12].contiguous(),
                                                 k[..., :12].contiguous()), B.ERR_UNSUPPORTED),
                       (lambda: B.gated_linear_fwd(x, w, act=9), B.ERR_INVALID_ARG),
                       (lambda: B.gated_linear_fwd(x[:0], w), B.ERR_INVALID_ARG),
                       (lambda: B.grad_clip([x], B.grad_norm([x]), 0.0), B.ERR_INVALID_ARG),
                       (lambda: B.grad_norm([torch.zeros(9, device=DEV)[1:]]),
                        B.ERR_INVALID_ARG)):  # 4 bytes in
        with pytest.raises(B.TriAttnError) as e:
            call()
        assert e.value.status == code
