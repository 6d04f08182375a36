"""Attention over matrices and its gradients against their definition in float64 (bounds: attention_common)."""
import pytest
import torch

from attention_common import BF16, GUARD, Batch, Out, Ref, backward, forward, near, put, space
from paper_2608_12703_amd import ad

pytestmark = pytest.mark.gpu

BATCHES = {
    "one": dict(ql=[1], kl=[1], heads=1, kv=1),
    "token": dict(ql=[1], kl=[1500], heads=3, kv=3),
    "tokens": dict(ql=[1, 1, 2, 1], kl=[37, 0, 1, 300], heads=2, kv=1),
    "self": dict(ql=[5, 0, 33, 128, 129, 1], kl=[5, 0, 33, 128, 129, 1], causal=True),
    "self_full": dict(ql=[64, 31, 100], kl=[64, 31, 100], heads=6, kv=2),
    "self_padded": dict(ql=[40, 0, 77, 1], kl=[40, 0, 77, 1], causal=True, padded=True, heads=3, kv=3),
    "shorter": dict(ql=[130, 7, 64], kl=[67, 200, 65], causal=True, heads=4, kv=1),
    "cross": dict(ql=[17, 65, 3], kl=[1500, 217, 64], heads=2, kv=2),
    "cross_padded": dict(ql=[17, 65, 3], kl=[300, 217, 64], heads=2, kv=1, padded=True, lead=3),
    "windows": dict(ql=[70, 33, 150], kl=[300, 129, 64], window="random", heads=2, kv=2),
    "windows_causal": dict(ql=[70, 33, 150], kl=[70, 33, 150], window="random", causal=True, heads=4, kv=2, lead=5),
    "sharp": dict(ql=[96], kl=[200], spread=12.0),
    "long": dict(ql=[700], kl=[700], causal=True, heads=1, kv=1),
}


def _batch(name, **more):
    return Batch(seed=len(name) * 131 + sum(map(ord, name)), **BATCHES[name], **more)


@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 0), (3, 1)])
@pytest.mark.parametrize("name", BATCHES)
def test_forward(name, pad, shift):
    bt = _batch(name)
    ref = Ref(bt)
    at, o, rest, lse = forward(bt, pad, shift)
    got, low = o.get(), rest.get()
    near(got, ref.o, ref.tol_o, "o")
    near(lse.double().cpu(), ref.lse, ref.tol_lse, "lse")
    # what o's rounding took away: at most half of its step, and 0 where o is 0
    inside = ref.o != GUARD
    assert bool((low.abs() <= got.abs() * 2.0 ** -8)[inside].all()) and bool((low == GUARD)[~inside].all())
    # without lse and o_rest, o is the same
    again = Out(bt.q_rows, 64 * bt.heads)
    ad.attention(at, put(bt.q), put(bt.k), put(bt.v), again.t, workspace=space(ad.attention_workspace_size, at, bt))
    assert torch.equal(again.get(), got) and int(at.err_flag) == 0


@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 0), (3, 1)])
@pytest.mark.parametrize("name", BATCHES)
def test_backward(name, pad, shift):
    bt = _batch(name)
    ref = Ref(bt)
    dq, dk, dv = backward(bt, ref, pad, shift)
    near(dq, ref.dq, ref.tol_dq, "dq")
    near(dk, ref.dk, ref.tol_dk, "dk")
    near(dv, ref.dv, ref.tol_dv, "dv")


@pytest.mark.parametrize("dtype", [torch.float32, BF16])
@pytest.mark.parametrize("name", ["self_padded", "cross", "windows_causal"])
def test_backward_adds_the_other_gradient_of_the_queries(name, dtype):
    bt = _batch(name)
    res = torch.randn(bt.q_rows, 64 * bt.heads, generator=torch.Generator().manual_seed(1)).to(dtype)
    ref = Ref(bt, res)
    dq, dk, dv = backward(bt, ref, res=res)
    near(dq, ref.dq, ref.tol_dq + 2.0 ** -23 * res.double().abs(), "dq")
    near(dk, ref.dk, ref.tol_dk, "dk")


def test_a_row_of_one_key_has_no_gradient_for_its_query():
    """delta = dP there: with o_rest what is left is float32's, without it o's rounding shows."""
    bt = Batch([40], [40], causal=True, seed=3)
    ref = Ref(bt)
    dq, _, _ = backward(bt, ref)
    scale = float((bt.dout.double().abs() * ref.o.abs()).sum(1).max() * bt.k.double().abs().max()) / 8
    assert float(dq[0].abs().max()) <= scale * 2.0 ** -15
    without, _, _ = backward(bt, ref, rest=False)
    near(without, ref.dq, ref.tol_dq + scale * 2.0 ** -8, "dq without o_rest")
