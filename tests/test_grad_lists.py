"""Lists of gradients that are kept from step to step (CPU): what has changed since a list
was made is refused before any address reaches the library."""
import pytest
import torch

from paper_2506_20686_amd import binding as B

BF, F4 = torch.bfloat16, torch.float32


@pytest.fixture
def kept(monkeypatch):
    """GradList as it would be of tensors on a GPU."""
    monkeypatch.setattr(B, "_check", lambda *a: None)
    return lambda *t: B.GradList(t)


def test_addresses_of_what_was_checked(kept):
    t = [torch.zeros(4, 3), torch.zeros(0), torch.zeros(7, dtype=BF)]
    g = kept(*t)
    assert list(g.addresses()) == [x.data_ptr() for x in t]
    t[0].data = torch.ones(3, 4)  # another place, another shape of as many elements
    assert list(g.addresses()) == [x.data_ptr() for x in t]


@pytest.mark.parametrize("was,now", [(F4, BF), (BF, F4), (F4, torch.float64), (F4, torch.int32)])
def test_a_changed_dtype_is_refused(kept, was, now):
    # as many elements, fewer or more bytes: what a module's change of dtype does to its gradients
    t = [torch.zeros(5, dtype=was), torch.zeros(60, dtype=was)]
    g = kept(*t)
    t[1].data = torch.zeros(60, dtype=now)
    with pytest.raises(ValueError):
        g.addresses()


@pytest.mark.parametrize("change", [lambda l: l.append(torch.zeros(3)), lambda l: l.pop(),
                                    lambda l: l.clear(), lambda l: l.insert(0, torch.zeros(5))])
def test_a_changed_number_of_tensors_is_refused(kept, change):
    # the list is the one that grad_clip returns
    g = kept(torch.zeros(5), torch.zeros(5))
    change(g.tensors)
    with pytest.raises(ValueError):
        g.addresses()


def test_tensors_that_come_to_share_storage_are_refused(kept):
    t = [torch.zeros(8), torch.zeros(0), torch.zeros(8), torch.zeros(0)]
    g = kept(*t)
    g.addresses()  # tensors of no elements share nothing
    t[2].data = t[0].data
    with pytest.raises(ValueError):
        g.addresses()
    t[2].data = torch.zeros(8)
    g.addresses()
