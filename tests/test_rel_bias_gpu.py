"""The relative position bias and its table's gradient through the C ABI
against the plain 64-bit form (bounds in ops_ref.py)."""
import pytest
import torch

import ops_ref as R
from paper_2506_20686_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F4 = torch.bfloat16, torch.float32


def inputs(batch, n, h, edges, chains, dtype, seed, spread=None):
    g = torch.Generator().manual_seed(seed)
    if spread is None:  # residue numbers that restart with each chain, some repeated
        pos = torch.cumsum((torch.rand(batch, n, generator=g) > 0.1).int(), 1)
        chain = torch.sort(torch.randint(0, chains, (batch, n), generator=g), 1).values
        first = torch.stack([(chain == c).int().argmax(1) for c in range(chains)], 1)
        pos = pos - torch.gather(pos, 1, torch.gather(first, 1, chain))
    else:
        pos = torch.randint(-spread, spread + 1, (batch, n), generator=g)
        chain = torch.randint(0, chains, (batch, n), generator=g)
    rows = len(edges) + 1 + (chains > 1)
    return {"pos": pos.to(torch.int32), "chain": chain.to(torch.int32) if chains > 1 else None,
            "table": torch.randn(rows, h, generator=g).to(dtype),
            "base": torch.randn(batch, n, n, h, generator=g).to(dtype),
            "dout": torch.randn(batch, n, n, h, generator=g).to(dtype)}


def dev(t):
    return None if t is None else t.to(DEV)


def both(t, edges):
    pos, chain, table = dev(t["pos"]), dev(t["chain"]), dev(t["table"])
    for base in (None, t["base"]):
        got = B.rel_bias_fwd(pos, edges, table, chain, dev(base)).cpu()
        assert torch.equal(got, R.rel_fwd(t["pos"], edges, t["table"], t["chain"], base))
    got = B.rel_bias_bwd(pos, edges, dev(t["dout"]), chain)
    R.check("dtable", got, *R.rel_bwd(t["pos"], edges, t["dout"], t["chain"]))


CLIP = B.rel_bias_edges(32)
FAR = B.rel_bias_edges(16, 512, 16)
LONG = B.rel_bias_edges(80, 1760, 24)  # a table too long for the arguments
WIDE = [-(1 << 31), -70000, -500, 0, 1, 3, 900, 12345, (1 << 31) - 1]


# one token, heads that do and do not fill a vector, odd lengths, batches, one to 255
# edges (a table of up to 257 rows), edges far apart
@pytest.mark.parametrize("dtype", [BF, F4])
@pytest.mark.parametrize("batch,n,h,edges,chains", [
    (1, 1, 1, [0], 1), (1, 1, 4, CLIP, 2), (1, 2, 3, [0], 1), (1, 40, 4, CLIP, 1),
    (1, 129, 4, CLIP, 3), (2, 33, 16, FAR, 2), (3, 17, 5, CLIP, 1), (1, 50, 128, CLIP, 2),
    (1, 31, 64, FAR, 1), (1, 12, 256, list(range(-127, 128)), 2), (2, 9, 255, WIDE, 1),
    (1, 200, 1, CLIP, 2), (1, 257, 2, FAR, 1), (1, 77, 24, list(range(-127, 128)), 2),
    (1, 300, 8, CLIP, 1), (4, 64, 12, [-5, 9], 2), (1, 90, 16, LONG, 2), (1, 70, 4, LONG, 1),
    (2, 40, 65, LONG, 1), (1, 37, 64, WIDE, 2), (1, 60, 16, WIDE, 1), (300, 5, 4, CLIP, 2),
    (1, 130, 32, CLIP, 1), (1, 66, 200, FAR, 1)])
def test_forward_and_backward(batch, n, h, edges, chains, dtype):
    both(inputs(batch, n, h, edges, chains, dtype, n + h), edges)


@pytest.mark.parametrize("dtype", [BF, F4])
@pytest.mark.parametrize("spread", [3, 100, 2000, 100000, (1 << 31) - 1])
def test_positions_in_any_order(spread, dtype):
    # the difference of two int32 does not fit one
    edges = WIDE if spread > 9000 else LONG if spread > 1000 else CLIP
    t = inputs(2, 70, 4, edges, 3, dtype, spread % 97, spread)
    t["pos"][0, 0], t["pos"][0, 1] = -(1 << 31), (1 << 31) - 1
    both(t, edges)


def test_unbatched_is_the_batch_of_one():
    t = inputs(1, 21, 4, CLIP, 2, BF, 1)
    a = {k: dev(v) for k, v in t.items()}
    one = B.rel_bias_fwd(a["pos"][0], CLIP, a["table"], a["chain"][0], a["base"][0])
    assert torch.equal(one, B.rel_bias_fwd(a["pos"], CLIP, a["table"], a["chain"], a["base"])[0])
    assert torch.equal(B.rel_bias_bwd(a["pos"][0], CLIP, a["dout"][0], a["chain"][0]),
                       B.rel_bias_bwd(a["pos"], CLIP, a["dout"], a["chain"]))


def test_clipped_difference():
    pos = torch.arange(0, 100, dtype=torch.int32)
    table = torch.arange(0, 65, dtype=torch.float32)[:, None]
    out = B.rel_bias_fwd(dev(pos), CLIP, dev(table))[:, :, 0].cpu()
    d = (pos[:, None] - pos[None, :]).clamp(-32, 32) + 32
    assert torch.equal(out, d.float())


def test_minus_infinity_in_base_stays():
    t = inputs(1, 19, 4, CLIP, 1, BF, 2)
    t["base"][0, 3, 5] = float("-inf")
    got = B.rel_bias_fwd(dev(t["pos"]), CLIP, dev(t["table"]), None, dev(t["base"])).cpu()
    assert bool((got[0, 3, 5] == float("-inf")).all())
    assert torch.equal(got, R.rel_fwd(t["pos"], CLIP, t["table"], None, t["base"]))


@pytest.mark.parametrize("dtype", [BF, F4])
@pytest.mark.parametrize("n,h", [(37, 4), (20, 7), (16, 128)])
def test_nothing_outside_the_outputs_is_written(n, h, dtype):
    t = {k: dev(v) for k, v in inputs(2, n, h, CLIP, 2, dtype, 3).items()}
    ref = (B.rel_bias_fwd(t["pos"], CLIP, t["table"], t["chain"], t["base"]),
           B.rel_bias_bwd(t["pos"], CLIP, t["dout"], t["chain"]))
    pad, rows, code = 64, len(CLIP) + 2, B.BF16 if dtype == BF else B.F32
    big = [torch.full((e + 2 * pad,), 7.0, dtype=d, device=DEV)
           for e, d in ((2 * n * n * h, dtype), (rows * h, F4))]
    at = [b.data_ptr() + pad * b.element_size() for b in big]
    need = B.tri_rel_bias_bwd_workspace_bytes(code, 2, n, h, len(CLIP))
    ws = torch.full((need + 256,), 9, dtype=torch.uint8, device=DEV)
    s = torch.cuda.current_stream().cuda_stream
    p = {k: v.data_ptr() for k, v in t.items()}
    assert B.tri_rel_bias_fwd(code, 2, n, h, CLIP, p["pos"], p["chain"], p["table"], p["base"],
                              at[0], s) == B.OK
    assert B.tri_rel_bias_bwd(code, 2, n, h, CLIP, p["pos"], p["chain"], p["dout"], at[1],
                              ws.data_ptr(), need, s) == B.OK
    for b, r in zip(big, ref):
        assert torch.equal(b[pad:-pad], r.reshape(-1))
        assert bool((b[:pad] == 7).all()) and bool((b[-pad:] == 7).all())
    assert bool((ws[need:] == 9).all())
    # the output over the base
    base = t["base"].clone()
    assert B.tri_rel_bias_fwd(code, 2, n, h, CLIP, p["pos"], p["chain"], p["table"],
                              base.data_ptr(), base.data_ptr(), s) == B.OK
    assert torch.equal(base, ref[0])


@pytest.mark.parametrize("dtype,h", [(BF, 4), (F4, 16), (BF, 128)])
def test_bitwise_reproducible(dtype, h):
    t = {k: dev(v) for k, v in inputs(1, 300, h, FAR, 2, dtype, 4).items()}
    a, b = (B.rel_bias_bwd(t["pos"], FAR, t["dout"], t["chain"]) for _ in range(2))
    assert torch.equal(a, b)


def test_long_sums_keep_their_digits():
    # 1024^2 pairs of one chain in 3 buckets, all positive: 24 bits of the sums
    n, edges = 1024, [0, 1]
    g = torch.Generator().manual_seed(6)
    pos = torch.arange(n, dtype=torch.int32)
    dout = torch.rand(n, n, 4, generator=g)
    got = B.rel_bias_bwd(dev(pos), edges, dev(dout)).cpu()
    ref, _ = R.rel_bwd(pos[None], edges, dout[None], None)
    # about 500,000 terms a sum, in partial sums of at most some thousands: random
    # roundings of partial sums of size S / parts give well under 32 U
    assert float(((got.double() - ref) / ref).abs().max()) <= 32 * R.U


def test_offsets_past_32_bits():
    n, h = 8192, 33  # 2.2e9 elements
    pos = torch.arange(n, dtype=torch.int32, device=DEV) * 3
    table = torch.randn(len(CLIP) + 1, h, device=DEV).to(BF)
    out = B.rel_bias_fwd(pos, CLIP, table)
    for q in (0, 1, 4000, n - 1):
        d = torch.clamp(pos[q] - pos, -32, 32).long() + 32
        assert torch.equal(out[q], table[d]), q
    out.zero_()
    out[-1] = 1.0  # the last query row alone
    got = B.rel_bias_bwd(pos, CLIP, out)
    d = torch.clamp(pos[-1] - pos, -32, 32).long() + 32
    want = torch.bincount(d, minlength=len(CLIP) + 1).float()
    assert torch.equal(got, want[:, None].expand(-1, h))
