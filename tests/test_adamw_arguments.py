"""What train.AdamW refuses when it is made: found at the first step, it would have counted that step, and a list whose
tensors differ would have been stepped in part (CPU only)."""
import math

import pytest
import torch

from paper_2608_12703_amd.train import AdamW


def _lists():
    shapes = [(7, 40), (300,), (129, 3)]
    return [torch.zeros(s).to(dt) for s, dt in zip(shapes, (torch.bfloat16, torch.bfloat16, torch.float32))], [torch.zeros(s) for s in shapes]


@pytest.mark.parametrize("bad", [
    dict(lr=-1e-3), dict(lr=math.nan), dict(lr=math.inf), dict(lr=1e39), dict(betas=(1.0, 0.9)), dict(betas=(-0.1, 0.9)), dict(betas=(0.9, 1.0)),
    dict(betas=(0.9, math.nan)), dict(betas=(0.9,)), dict(eps=-1e-8), dict(eps=math.nan), dict(eps=math.inf), dict(weight_decay=-0.01),
    dict(weight_decay=math.nan), dict(weight_decay=math.inf), dict(max_norm=-1.0), dict(max_norm=math.nan), dict(max_norm=math.inf)])
def test_refused_when_it_is_made(bad):
    params, grads = _lists()
    with pytest.raises(ValueError):
        AdamW(params, grads, **bad)


def test_taken():
    params, grads = _lists()
    for good in (dict(), dict(lr=0.0), dict(betas=(0.0, 0.0)), dict(eps=0.0), dict(weight_decay=0.0), dict(max_norm=0.0)):
        AdamW(params, grads, **good)


@pytest.mark.parametrize("lr", [-1e-3, math.nan, math.inf, 1e39])
def test_a_rate_that_no_step_takes(lr):
    opt = AdamW(*_lists(), lr=1e-3)
    with pytest.raises(ValueError):
        opt.set_lr(lr)
    assert float(opt.lr) == pytest.approx(1e-3)
    opt.set_lr(2e-3)
    assert float(opt.lr) == pytest.approx(2e-3)
