"""What an optimizer handle keeps of the tensors that it was made of (CPU only)."""
import gc
import weakref

import pytest
import torch


@pytest.fixture(scope="module")
def ad():
    from paper_2608_12703_amd import ad as mod
    return mod


def _lists(n=3):
    make = lambda: [torch.zeros(200 + i) for i in range(n)]  # noqa: E731
    return dict(params=make(), grads=make(), m=make(), v=make(), copies=[torch.zeros(200 + i, dtype=torch.bfloat16) for i in range(n)])


@pytest.mark.parametrize("name", ["params", "grads", "m", "v", "copies"])
def test_the_handle_keeps_its_tensors(ad, name):
    """The kernels write to their addresses: a caller who puts other tensors into the lists must not free them."""
    lists = _lists()
    opt = ad.OptTensors(**lists)
    kept = weakref.ref(lists[name][1])
    at = lists[name][1].data_ptr()
    lists[name][1] = None
    lists[name].clear()
    gc.collect()
    assert kept() is not None and opt.tensors[name][1].data_ptr() == at
