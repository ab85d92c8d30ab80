"""The names under which the linear projection's launches are timed."""
import pytest
import torch

from paper_2506_20686_amd import binding as B

DEV = "cuda:0"
BF = torch.bfloat16
# numbered after the older kernels, whose indices callers hold
LATER = ["ln_fwd", "ln_bwd", "ln_reduce", "lin_fwd", "lin_bwd_dx", "lin_bwd_w", "lin_reduce",
         "lin_dz", "lin_narrow", "rel_fwd", "rel_bwd", "rel_reduce", "lin_bwd_both"]


def test_indices_and_names():
    for i, name in enumerate(LATER):
        assert B.tri_attn_timing_read(21 + i)[0] == name


# dx and dW in one launch where dx does not fill the GPU, each in its own where it does,
# one pass over narrow bf16 rows; dz of gelu beforehand; the splits' sums
@pytest.mark.gpu
@pytest.mark.parametrize("m,k,n,act,launched", [
    (1500, 384, 256, B.ACT_NONE, {"lin_bwd_both", "lin_reduce"}),
    (1500, 384, 256, B.ACT_GELU, {"lin_dz", "lin_bwd_both", "lin_reduce"}),
    (16500, 256, 136, B.ACT_RELU, {"lin_bwd_dx", "lin_bwd_w", "lin_reduce"}),
    (5000, 128, 96, B.ACT_SILU, {"lin_narrow", "lin_reduce"}),
    (40, 200, 40, B.ACT_NONE, {"lin_bwd_both"})])
def test_launches_of_the_backward(m, k, n, act, launched):
    x, w, dy, z = (torch.randn(*s, device=DEV).to(BF) for s in ((m, k), (k, n), (m, n), (m, n)))
    B.tri_attn_timing_enable(True)
    try:
        B.tri_attn_timing_reset()
        B.linear_bwd(x, w, dy, z if act else None, act)
        got = {name: count for name, (_, count) in B.kernel_times().items() if count}
    finally:
        B.tri_attn_timing_enable(False)
        B.tri_attn_timing_reset()
    assert got == dict.fromkeys(launched, 1)
