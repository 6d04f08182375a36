"""A training run that goes on from a saved optimizer: everything that the next step hangs on comes back (CPU: the class's
own bookkeeping, no step runs)."""
import io

import pytest
import torch

from paper_2608_12703_amd.train import AdamW

BF16 = torch.bfloat16


def _made(state, seed=0, fill=True):
    g = torch.Generator().manual_seed(seed)
    shapes = [(7, 40), (300,), (129, 3), (5,)]
    params = [torch.randn(s, generator=g).to(dt) for s, dt in zip(shapes, (BF16, BF16, torch.float32, torch.float32))]
    opt = AdamW(params, [torch.zeros(s) for s in shapes], lr=10.0 ** -(3 + seed), state=state, seed=seed + 5)
    if fill:
        for name, x in opt._states().items():
            for t in x:
                t.copy_(torch.randint(0, 90, t.shape, generator=g) if name != "master" else torch.randn(t.shape, generator=g))
        opt.steps.fill_(17 + seed)
    return params, opt


def _all(opt):
    return [t.clone() for x in opt._states().values() for t in x] + [opt.steps.clone(), opt.lr.clone()]


@pytest.mark.parametrize("state", ["f32", "8bit"])
def test_a_saved_optimizer_comes_back(state):
    params, opt = _made(state)
    file = io.BytesIO()
    torch.save(opt.state_dict(), file)
    file.seek(0)
    want, kept = _all(opt), opt.state_dict()
    other, back = _made(state, seed=1)
    at = [t.data_ptr() for x in back._states().values() for t in x] + [back.steps.data_ptr(), back.lr.data_ptr()]
    back.load_state_dict(torch.load(file, weights_only=True))
    assert all(torch.equal(a, b) for a, b in zip(want, _all(back))) and back.seed == opt.seed
    # in place: a captured step goes on with them
    assert at == [t.data_ptr() for x in back._states().values() for t in x] + [back.steps.data_ptr(), back.lr.data_ptr()]
    # the parameters are the float32 ones', rounded
    for p, m in zip(other, back.master):
        assert torch.equal(p, m.to(p.dtype))
    # what was saved does not change with the optimizer
    opt.steps.fill_(0)
    for x in opt._states().values():
        for t in x:
            t.zero_()
    back.load_state_dict(kept)
    assert all(torch.equal(a, b) for a, b in zip(want, _all(back)))


def test_parameters_that_are_loaded_anew_stay():
    """The float32 parameters behind bf16 ones are made once: after new values came into the parameters they are
    theirs again, and the states stay."""
    params, opt = _made("8bit")
    states = [t.clone() for name, x in opt._states().items() if name != "master" for t in x]
    new = [torch.randn(p.shape).to(p.dtype) for p in params]
    for p, n in zip(params, new):
        p.copy_(n)
    opt.read_params()
    for p, m, n in zip(params, opt.master, new):
        assert torch.equal(p, n) and torch.equal(m, n.float())
    assert all(torch.equal(a, b) for a, b in zip(states, [t for name, x in opt._states().items() if name != "master" for t in x]))


@pytest.mark.parametrize("bad", ["state", "count", "shape", "dtype", "missing", "steps"])
def test_what_does_not_fit_is_refused_whole(bad):
    _, opt = _made("f32")
    _, eight = _made("8bit")
    d = opt.state_dict()
    if bad == "state":
        d = eight.state_dict()
    elif bad == "count":
        d["m"] = d["m"][:3]
    elif bad == "shape":
        d["v"][3] = torch.zeros(6)
    elif bad == "dtype":
        d["v"][3] = d["v"][3].double()
    elif bad == "missing":
        del d["master"]
    else:
        d["steps"] = torch.zeros(2, dtype=torch.int32)
    params, other = _made("f32", seed=2)
    before, values = _all(other), [p.clone() for p in params]
    with pytest.raises((ValueError, KeyError)):
        other.load_state_dict(d)
    assert all(torch.equal(a, b) for a, b in zip(before, _all(other))) and all(torch.equal(a, b) for a, b in zip(values, params))
    assert other.seed == 7
