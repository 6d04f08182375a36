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


def _views(flat, *cuts):
    return [flat[a:b] for a, b in cuts]


def test_tensors_that_a_step_would_write_twice_are_refused(ad):
    """Two workgroups would write the same element: what comes out hangs on their order."""
    half = torch.bfloat16
    for name in ("params", "m", "v", "copies"):
        lists = _lists()
        lists[name] = [lists[name][0], lists[name][1], lists[name][0]]
        for other, x in lists.items():                # (equal sizes)
            if other != name:
                x[2] = torch.zeros(200, dtype=x[2].dtype)
        with pytest.raises(ValueError, match="overlap"):
            ad.OptTensors(**lists)
    flat = torch.zeros(1000)
    apart, shared = [(0, 200), (200, 401), (401, 603)], [(0, 200), (199, 400), (401, 603)]
    for name in ("params", "m", "v"):
        assert ad.OptTensors(**dict(_lists(), **{name: _views(flat, *apart)})).steps
        with pytest.raises(ValueError, match="overlap"):
            ad.OptTensors(**dict(_lists(), **{name: _views(flat, *shared)}))
    # one buffer for two kinds of tensor, and a gradient that a step would write
    lists = _lists()
    with pytest.raises(ValueError, match="overlap"):
        ad.OptTensors(**dict(lists, m=lists["v"]))
    with pytest.raises(ValueError, match="overlap"):
        ad.OptTensors(**dict(lists, grads=lists["params"]))
    with pytest.raises(ValueError, match="overlap"):
        ad.OptTensors(**dict(lists, params=[x.to(half) for x in lists["params"]], grads=_views(lists["m"][0].view(half), (0, 200), (0, 201), (0, 202)),
                             copies=None))
    eight = dict(m=[torch.zeros(200 + i, dtype=torch.int8) for i in range(3)], v=[torch.zeros(200 + i, dtype=torch.uint8) for i in range(3)])
    scales = torch.zeros(20)
    good = dict(m_scale=_views(scales, (0, 2), (2, 4), (4, 6)), v_scale=_views(scales, (6, 8), (8, 10), (10, 12)))
    assert ad.OptTensors(**dict(_lists(), **eight, **good)).steps
    with pytest.raises(ValueError, match="overlap"):
        ad.OptTensors(**dict(_lists(), **eight, **dict(good, v_scale=_views(scales, (5, 7), (8, 10), (10, 12)))))


def test_tensors_that_are_only_read_may_be_the_same(ad):
    x = torch.zeros(200)
    assert ad.OptTensors(grads=[x, x]).count == 2                       # the norm counts it twice
    assert ad.OptTensors(m=[x, x], v=[x, x]).count == 2                 # a look at the states
    lists = _lists(2)
    for y in lists.values():
        y[1] = torch.zeros(200, dtype=y[1].dtype)
    assert ad.OptTensors(**dict(lists, grads=[x, x])).steps             # one gradient for two parameters
    empty = torch.zeros(0)
    assert ad.OptTensors(params=[empty, empty], grads=[empty, empty], m=[empty, empty], v=[empty, empty]).steps
