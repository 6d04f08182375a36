"""A training run that stops, is saved and goes on in another process's place: the bits of one that did not stop."""
import io

import pytest
import torch

from paper_2608_12703_amd.train import AdamW

pytestmark = pytest.mark.gpu

SHAPES = [(64, 200), (3000,), (129, 65), (7,)]


def _made(state, seed=0):
    g = torch.Generator().manual_seed(seed)
    types = (torch.bfloat16, torch.bfloat16, torch.float32, torch.bfloat16)
    params = [(torch.randn(s, generator=g) * 0.02).to(dt).cuda() for s, dt in zip(SHAPES, types)]
    grads = [torch.zeros(s, device="cuda") for s in SHAPES]
    return params, grads, AdamW(params, grads, lr=1e-3 * (1 + seed), state=state, seed=9 + seed)


def _steps(opt, grads, first, last, run=None):
    for k in range(first, last):
        g = torch.Generator().manual_seed(100 + k)
        for x in grads:
            x.copy_(torch.randn(x.shape, generator=g) * 1e-2)
        (run or opt.step)()


def _equal(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("state", ["f32", "8bit"])
def test_a_run_goes_on(state, captured):
    params, grads, opt = _made(state)
    _steps(opt, grads, 0, 3)
    opt.set_lr(4e-4)
    file = io.BytesIO()
    torch.save(opt.state_dict(), file)
    _steps(opt, grads, 3, 6)
    file.seek(0)
    params2, grads2, opt2 = _made(state, seed=1)
    run = None
    if captured:                                   # captured before its state is loaded; the seed is the graph's own
        opt2.seed = opt.seed
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            opt2.step()
        run = graph.replay
    opt2.load_state_dict(torch.load(file, weights_only=True))
    _steps(opt2, grads2, 3, 6, run)
    torch.cuda.synchronize()
    assert _equal(params, params2) and _equal(opt.master, opt2.master) and int(opt2.steps) == 6
    assert all(_equal(a, b) for a, b in zip(opt.states(), opt2.states()))


def test_new_parameters_are_stepped_from():
    params, grads, opt = _made("f32")
    _steps(opt, grads, 0, 2)
    g = torch.Generator().manual_seed(7)
    new = [(torch.randn(s, generator=g) + 3).to(p.dtype) for s, p in zip(SHAPES, params)]
    for p, n in zip(params, new):
        p.copy_(n)
    opt.read_params()
    _steps(opt, grads, 2, 3)
    # (a step moves by a few times the rate of 1e-3, the new values are 3 away from the old ones; half a step of bf16 at 8 is 2^-6)
    assert all(float((p.cpu().double() - n.double()).abs().max()) < 0.05 for p, n in zip(params, new))
