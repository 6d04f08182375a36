"""The feed-forward sublayer's buffers: what a refused pass leaves behind."""
import pytest
import torch

from paper_2608_12703_amd import ad
from paper_2608_12703_amd.train import FeedForward
from test_gpu_train_ops import _sublayer

pytestmark = pytest.mark.gpu


def _made(rows=40, d=128, f=320, seed=51):
    params, x, dout = _sublayer(seed, d, f, rows)
    return [p.cuda() for p in params], x.cuda(), dout.cuda()


def test_a_refused_forward_pass_leaves_nothing_to_go_back_from():
    """The kept rows may be the refused pass's by then: backward does not mix the two."""
    params, x, dout = _made()
    ff = FeedForward(params, 40)
    out, dx = torch.empty_like(x), torch.empty_like(x)
    for bad in (dict(out=out[:, :64]), dict(out=out[:20]), dict(out=out.half()), dict(out=out[:1].expand(40, 128)),
                dict(out=out.cpu()), dict(x=x.double()), dict(x=x[:, :64])):
        ff.forward(x, out)
        a = dict(x=x * 2, out=out) | bad
        with pytest.raises((ValueError, ad.ADError)):
            ff.forward(a["x"], a["out"])
        with pytest.raises(ValueError, match="last forward"):
            ff.backward(dout, dx)
    assert not any(bool(g.any()) for g in ff.grads)
    ff.forward(x, out)
    ff.backward(dout, dx)


def test_a_refused_backward_pass_adds_nothing():
    params, x, dout = _made()
    ff, other = FeedForward(params, 40), FeedForward(params, 40)
    out, dx, want = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    ff.forward(x, out)
    other.forward(x, out)
    other.backward(dout, want)
    for bad in (dict(dx=dx[:, :64]), dict(dx=dx[:20]), dict(dx=dx.half()), dict(dx=dx[:1].expand(40, 128)), dict(dx=dx.cpu()),
                dict(dx=torch.empty(128, 40, device="cuda").t()), dict(copy=dx), dict(copy=dx[:20].bfloat16()),
                dict(dout=dout.double()), dict(dout=dout[:1].expand(40, 128)), dict(dout=dout[:, :64])):
        a = dict(dout=dout, dx=dx, copy=None) | bad
        with pytest.raises((ValueError, ad.ADError)):
            ff.backward(a["dout"], a["dx"], a["copy"])
        assert not any(bool(g.any()) for g in ff.grads), list(bad)
    ff.backward(dout, dx)                       # the forward pass still stands
    assert torch.equal(dx, want) and all(torch.equal(a, b) for a, b in zip(ff.grads, other.grads))
