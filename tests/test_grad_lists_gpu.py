"""Lists of gradients that are kept from step to step, on a GPU: refusals before any launch,
and what is taken as it was."""
import pytest
import torch

from paper_2506_20686_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F4 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("was,now", [(F4, BF), (BF, F4)])
def test_a_changed_dtype_is_refused(was, now):
    t = [torch.ones(n, dtype=was, device=DEV) for n in (5, 60)]
    g = B.GradList(t)
    norm = B.grad_norm(g)
    kept = t[1].data
    t[1].data = torch.ones(60, dtype=now, device=DEV)
    with pytest.raises(ValueError):
        B.grad_norm(g)
    with pytest.raises(ValueError):
        B.grad_clip(g, norm, 1.0)
    t[1].data = kept
    assert torch.equal(B.grad_norm(g), norm)


def test_a_changed_device_is_refused():
    t = [torch.ones(n, device=DEV) for n in (5, 60)]
    g = B.GradList(t)
    norm = B.grad_norm(g)
    g.tensors[1] = torch.ones(60)
    with pytest.raises(ValueError):
        B.grad_norm(g)
    with pytest.raises(ValueError):
        B.grad_clip(g, norm, 1.0)


def test_tensors_that_come_to_share_storage_are_refused():
    t = [torch.ones(64, device=DEV), torch.ones(64, device=DEV)]
    g = B.GradList(t)
    norm = B.grad_norm(g)
    t[1].data = t[0].data
    with pytest.raises(ValueError):
        B.grad_norm(g)
    with pytest.raises(ValueError):
        B.grad_clip(g, norm, 1.0)
    assert bool((t[0] == 1).all())


def test_overlapping_results_are_refused_and_neighbours_are_not():
    flat = torch.randn(3 * 64, device=DEV)
    t = [flat[:64], flat[64:128], flat[128:]]
    norm = B.grad_norm(t)
    was = flat.clone()
    for out in ([t[1], t[2], t[0]], [t[0], flat[96:160], t[2]], [flat[:64], flat[32:96], t[2]]):
        with pytest.raises(B.TriAttnError) as e:
            B.grad_clip(t, norm, 1.0, out)
        assert e.value.status == B.ERR_INVALID_ARG
    assert torch.equal(flat, was)
    other = torch.empty_like(flat)
    B.grad_clip(t, norm, 1.0, [other[:64], other[64:128], other[128:]])
    B.grad_clip(t, norm, 1.0)  # one after the other in memory
    assert torch.equal(flat, other) and not torch.equal(flat, was)
    # one tensor in its place, one to memory of its own
    B.grad_clip([t[0], t[1]], norm, 1.0, [t[0], other[64:128]])


def test_a_long_list_is_clipped():
    n = 300
    flat = torch.randn(n * 16, device=DEV)
    t = [flat[16 * ((i * 7) % n):][:16] for i in range(n)]
    norm = B.grad_norm(t)
    want = flat * (1.0 / norm)
    B.grad_clip(t, norm, 1.0)
    assert torch.equal(flat, want)
