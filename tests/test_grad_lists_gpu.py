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
