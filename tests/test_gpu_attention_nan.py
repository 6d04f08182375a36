"""NaN and infinities in visible places: they come out where the definition has them, and a pass that is full of them (a
training step that diverged) takes a few times as long as any other."""
import math

import pytest
import torch

from attention_common import BF16, Batch, Ref, backward, forward, near
from paper_2608_12703_amd import ad

pytestmark = pytest.mark.gpu

SHAPES = {
    "few": dict(ql=[40, 9, 33], kl=[150, 70, 41], heads=4, kv=2),
    "parts": dict(ql=[3, 1], kl=[2600, 130], heads=1, kv=1),
    "wide": dict(ql=[140, 97] * 8, kl=[150, 64] * 8, heads=4, kv=4),
    "wide_many": dict(ql=[140, 35] * 20, kl=[150, 40] * 20, heads=6, kv=6),
}


@pytest.mark.parametrize("place", ["q", "k", "v", "dout"])
@pytest.mark.parametrize("what", ["element", "row", "rows"])
@pytest.mark.parametrize("name", SHAPES)
def test_what_is_nan_comes_out(name, what, place):
    """Every query sees every key of its sequence here.  The first sequence holds the NaN, the others are as without."""
    bt = Batch(seed=40, **SHAPES[name])
    rows = {"q": bt.q, "k": bt.k, "v": bt.v, "dout": bt.dout}[place]
    n = bt.kl[0] if place in "kv" else bt.ql[0]
    if what == "element":
        rows[n // 2, 70 % rows.shape[1]] = math.nan
    elif what == "row":
        rows[n - 1] = math.nan
    else:
        rows[:n] = math.nan
    ref = Ref(bt)
    if place != "dout":
        _, o, _, lse = forward(bt)
        near(o.get(), ref.o, ref.tol_o, "o")
        near(lse.double().cpu(), ref.lse, ref.tol_lse, "lse")
    dq, dk, dv = backward(bt, ref)
    near(dq, ref.dq, ref.tol_dq, "dq")
    near(dk, ref.dk, ref.tol_dk, "dk")
    near(dv, ref.dv, ref.tol_dv, "dv")


def _time(f):
    f()
    torch.cuda.synchronize()
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    a.record()
    f()
    b.record()
    b.synchronize()
    return a.elapsed_time(b)


@pytest.mark.parametrize("place", ["q", "kv", "dout", "all", "last"])
@pytest.mark.parametrize("causal", [False, True])
def test_a_pass_of_nan_ends_soon(causal, place):
    """32 sequences of 448 rows, 20 heads: 0.05 to 0.6 ms with finite rows.  Each wave computes its 32 rows again, of which
    one key (or query) is enough: 64 more round trips to memory of 1 to 2 us each, 0.2 ms, for each of up to 15 rounds
    of workgroups.  Walks to the end would be 448 to 1500 times as many."""
    nq, nk, heads, batch = 448, 448 if causal else 1500, 20, 32
    g = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda rows: torch.randn(rows, 64 * heads, generator=g, device="cuda").to(BF16)  # noqa: E731
    q, do, k, v = rand(batch * nq), rand(batch * nq), rand(batch * nk), rand(batch * nk)
    last = q.view(batch, nq, -1)[:, -1]           # one row of each sequence, which sees every key
    for t in {"q": (q,), "kv": (k, v), "dout": (do,), "all": (q, k, v, do), "last": (last,)}[place]:
        t.fill_(math.nan)
    ints = lambda n: torch.arange(batch + 1, dtype=torch.int32, device="cuda") * n  # noqa: E731
    at = ad.Attention(heads, heads, ints(nq), ints(nk), nq, nk, causal=causal)
    o, rest, dq, dk, dv = (torch.empty_like(t) for t in (q, q, q, k, v))
    lse = torch.empty(heads, batch * nq, device="cuda")
    buf = lambda size: torch.empty(max(size(at, batch * nq, batch * nk), 1), dtype=torch.uint8, device="cuda")  # noqa: E731
    fwd, bwd = buf(ad.attention_workspace_size), buf(ad.attention_backward_workspace_size)
    assert _time(lambda: ad.attention(at, q, k, v, o, lse, rest, fwd)) < 10.0
    assert _time(lambda: ad.attention_backward(at, q, k, v, o, rest, lse, do, None, dq, dk, dv, bwd)) < 10.0
    rows = slice(None) if place != "last" else slice(nq - 1, None, nq)
    assert bool(torch.isnan(dq[rows]).all()) and bool(torch.isnan(dk).all()) and bool(torch.isnan(dv).all())
    assert place == "dout" or bool(torch.isnan(o[rows]).all())
    assert place != "last" or int(torch.isnan(o).sum()) == int(torch.isnan(dq).sum()) == batch * 64 * heads
