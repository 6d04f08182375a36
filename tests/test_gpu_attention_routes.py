"""Every way through the forward pass, and the gradients of the same batches (bounds: attention_common; which way a batch
takes: test_attention_routes)."""
import functools

import pytest

from attention_common import GUARD, Batch, Ref, backward, forward, near
from attention_routes import ROUTES

pytestmark = pytest.mark.gpu


@functools.lru_cache(maxsize=2)
def _batch(name):
    bt = Batch(seed=sum(map(ord, name)), **ROUTES[name][1])
    return bt, Ref(bt)


@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 1)])
@pytest.mark.parametrize("name", ROUTES)
def test_ways_through_attention(name, pad, shift):
    bt, ref = _batch(name)
    at, o, rest, lse = forward(bt, pad, shift)
    got, low = o.get(), rest.get()
    near(got, ref.o, ref.tol_o, "o")
    near(lse.double().cpu(), ref.lse, ref.tol_lse, "lse")
    inside = ref.o != GUARD
    assert bool((low.abs() <= got.abs() * 2.0 ** -8)[inside].all()) and bool((low == GUARD)[~inside].all()) and int(at.err_flag) == 0
    dq, dk, dv = backward(bt, ref, pad, shift)
    near(dq, ref.dq, ref.tol_dq, "dq")
    near(dk, ref.dk, ref.tol_dk, "dk")
    near(dv, ref.dv, ref.tol_dv, "dv")
