"""The feed-forward sublayer's buffers: what a refused pass leaves behind, and what sublayers share."""
import pytest
import torch

from paper_2608_12703_amd import ad
from paper_2608_12703_amd.train import FeedForward, Scratch
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


def test_sublayers_share_their_scratch():
    """Forward through three, backward through them in the other order, as a stack of blocks has it: the
    results of sublayers with buffers of their own, captured and replayed too."""
    sizes, d, f = (70, 33, 70), 128, 320
    made = [_made(rows, d, f, 60 + i) for i, rows in enumerate(sizes)]
    alone = [FeedForward(p, 70) for p, _, _ in made]
    shared = Scratch(d, f, 80)
    stack = [FeedForward(p, rows, shared) for (p, _, _), rows in zip(made, sizes)]

    def run(ffs, outs, dxs):
        for ff, (_, x, _), out in zip(ffs, made, outs):
            ff.zero_grads()
            ff.forward(x, out)
        for ff, (_, _, dout), dx in reversed(list(zip(ffs, made, dxs))):
            ff.backward(dout, dx)

    results = []
    for ffs in (alone, stack):
        outs, dxs = ([torch.empty_like(x) for _, x, _ in made] for _ in range(2))
        run(ffs, outs, dxs)
        results.append([*outs, *dxs, *(g for ff in ffs for g in ff.grads)])
    assert all(torch.equal(a, b) for a, b in zip(*results))
    want = [t.clone() for t in results[1]]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(stack, results[1][:3], results[1][3:6])
    for rep in range(3):
        for t in results[1][:6]:
            t.fill_(-77.0)
        for t in (shared.narrow, shared.wide, shared.wide2):
            t.fill_(float(rep))
        shared.workspace.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results[1], want)), rep


def test_memory_of_a_sublayer_that_shares():
    """1.03 (d + f) bytes a row and 4, and its gradients: nothing that only a running pass needs.  (An
    allocation is rounded up to 512 bytes.)"""
    rows, d, f = 4096, 256, 640
    params, _, _ = _made(1, d, f)
    shared = Scratch(d, f, rows)
    before = torch.cuda.memory_allocated()
    ff = FeedForward(params, rows, shared)
    held = torch.cuda.memory_allocated() - before
    grads = sum(4 * p.numel() for p in params)
    assert held <= rows * ((d + f) * 33 // 32 + 4) + grads + 16 * 512
    assert ff.workspace is shared.workspace


def test_refused_scratch():
    params, _, _ = _made()
    for bad in (Scratch(64, 320, 40), Scratch(128, 384, 40), Scratch(128, 320, 39)):
        with pytest.raises(ValueError, match="scratch"):
            FeedForward(params, 40, bad)
