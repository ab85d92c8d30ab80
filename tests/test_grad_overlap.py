"""tri_grad_clip refuses results that overlap each other or another tensor's gradient (CPU:
every call here is refused before any HIP call)."""
import pytest

from paper_2506_20686_amd import binding as B
from test_more_abi import GRAD, GRAD_CLIP, INV, call, ints, kinds, lib, ptrs  # noqa: F401

A = 0x100000  # fake, 16-byte aligned, never touched


def clip(lib, dtypes, sizes, grads, outs):
    return call(lib.tri_grad_clip, GRAD_CLIP, GRAD, dict(
        n=len(sizes), kinds=kinds(*dtypes), sizes=ints(*sizes), grads=ptrs(*grads),
        outs=ptrs(*outs)))


# 64 fp32 are 256 bytes, 64 bf16 are 128
@pytest.mark.parametrize("dtypes,sizes,grads,outs", [
    # the gradients in another order
    ((0, 0), (64, 64), (A, A + 256), (A + 256, A)),
    ((1, 1, 1), (64, 64, 64), (A, A + 128, A + 256), (A + 128, A + 256, A)),
    # in place, one tensor twice, or the second within the first
    ((0, 0), (64, 64), (A, A), (A, A)),
    ((0, 1), (64, 8), (A, A + 240), (A, A + 240)),
    # a gradient's own result shifted within it, either way
    ((0,), (64,), (A,), (A + 16,)),
    ((0,), (64,), (A + 16,), (A,)),
    # results that share one word
    ((0, 0), (64, 64), (A, A + 256), (A + 0x1000, A + 0x1000 + 240)),
    ((1, 0), (65, 64), (A, A + 256), (A + 0x1000, A + 0x1000 + 128)),
    # a result over another tensor's gradient, which is clipped in place
    ((0, 0, 0), (64, 4, 64), (A, 2 * A, A + 256), (A, A + 256, A + 256)),
    # two gradients that are one tensor, with results apart but one in its place
    ((0, 0), (64, 64), (A, A), (A, 2 * A)),
])
def test_overlaps_are_refused(lib, dtypes, sizes, grads, outs):  # noqa: F811
    assert clip(lib, dtypes, sizes, grads, outs) == INV


def test_overlap_in_a_long_list_is_refused(lib):  # noqa: F811
    n = 5000
    at = [A + 256 * ((i * 1117) % n) for i in range(n)]  # every place once, in no order
    assert len(set(at)) == n
    place = list(at)
    place[n - 1] = at[3]
    assert clip(lib, [0] * n, [64] * n, place, place) == INV
    assert clip(lib, [0] * n, [64] * n, at, at[1:] + at[:1]) == INV
