"""Step and learning rate on the device that ad_adamw refuses as numbers: nothing is written, as with a grad_scale that
is not finite."""
import math

import pytest
import torch

from paper_2608_12703_amd import ad

pytestmark = pytest.mark.gpu


def _made(state):
    """Three tensors, one of them longer than a workgroup's elements, everything that a step writes in `all`."""
    g = torch.Generator().manual_seed(3)
    sizes = [5, 9000, 300]
    rand = lambda n, scale: (torch.randn(n, generator=g) * scale).cuda()  # noqa: E731
    t = dict(params=[rand(n, 0.02) for n in sizes], copies=[torch.zeros(n, dtype=torch.bfloat16).cuda() for n in sizes])
    if state == "f32":
        t.update(m=[rand(n, 1e-3) for n in sizes], v=[rand(n, 1e-3).square() for n in sizes])
    else:
        t.update(m=[torch.full((n,), 9, dtype=torch.int8).cuda() for n in sizes],
                 v=[torch.full((n,), 90, dtype=torch.uint8).cuda() for n in sizes])
        t.update({k: [rand(-(-n // 128), 1e-6).abs() for n in sizes] for k in ("m_scale", "v_scale")})
    return ad.OptTensors(grads=[rand(n, 1e-2) for n in sizes], weight_decay=0.1, **t), [x for y in t.values() for x in y]


@pytest.mark.parametrize("scale", [False, True])
@pytest.mark.parametrize("state", ["f32", "8bit"])
@pytest.mark.parametrize("lr,step", [(1e-3, 0), (1e-3, -7), (1e-3, -2 ** 31), (math.nan, 3), (math.inf, 3), (-math.inf, 3), (-1e-3, 3)])
def test_scalars_out_of_range(lr, step, state, scale):
    opt, written = _made(state)
    before = [x.clone() for x in written]
    rate, count = torch.tensor([lr]).cuda(), torch.tensor([step], dtype=torch.int32).cuda()
    more = dict(grad_scale=torch.tensor([0.5]).cuda()) if scale else {}
    ad.adamw(opt, rate, count, **more)
    assert all(torch.equal(a, b) for a, b in zip(before, written))
    if step >= 1:                     # the rate alone on the device
        ad.adamw(opt, rate, step, **more)
    else:                             # the step alone
        ad.adamw(opt, lr, count, **more)
    assert all(torch.equal(a, b) for a, b in zip(before, written))
    rate.fill_(1e-3)
    count.fill_(2)
    ad.adamw(opt, rate, count, **more)
    assert all(bool(torch.isfinite(x.float()).all()) for x in written)
    assert not any(torch.equal(a, b) for a, b in zip(before[:3], written[:3]))


def test_the_first_step_after_one_that_was_left_out():
    """A norm that is not finite counts no step: the step that follows sees a count of 0 and a scale of NaN."""
    opt, written = _made("f32")
    before = [x.clone() for x in written]
    out, count, rate = torch.empty(2).cuda(), torch.zeros(1, dtype=torch.int32).cuda(), torch.tensor([1e-3]).cuda()
    ws = torch.empty(ad.grad_norm_workspace_size(opt), dtype=torch.uint8, device="cuda")
    opt.tensors["grads"][1][7] = math.inf
    ad.grad_norm(opt, 1.0, out, ws, step=count)
    ad.adamw(opt, rate, count, grad_scale=out[1:])
    assert int(count) == 0 and all(torch.equal(a, b) for a, b in zip(before, written))
