"""Attention over matrices and its gradients against their definition in float64 (bounds: attention_common)."""
import functools

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
    # keys in parts, which a second launch joins
    "parts": dict(ql=[17, 65, 3], kl=[2600, 217, 64], heads=2, kv=1),
    "parts_causal": dict(ql=[40, 1, 3], kl=[1900, 2100, 0], heads=3, kv=3, causal=True, lead=3),
    "parts_windows": dict(ql=[33, 20, 2], kl=[2000, 129, 1], window="random", padded=True),
    # enough workgroups for four waves of 32 rows each (128, or 1024 with windows); with more than 512 of
    # them both gradients have a launch of their own (wide_many)
    "wide": dict(ql=[140, 97] * 8, kl=[150, 64] * 8, heads=4, kv=4),
    "wide_causal": dict(ql=[131, 140, 1, 129] * 4, kl=[131, 140, 1, 129] * 4, heads=4, kv=4, causal=True),
    "wide_longer": dict(ql=[131, 40, 140, 129] * 4, kl=[200, 300, 64, 1] * 4, heads=4, kv=4, causal=True, lead=1),
    "wide_shared": dict(ql=[70] * 20, kl=[90] * 20, heads=8, kv=4),
    "wide_cross": dict(ql=[33, 70, 128, 40] * 8, kl=[300, 1, 0, 129] * 8, heads=4, kv=4, padded=True),
    "wide_many": dict(ql=[140, 35] * 20, kl=[150, 40] * 20, heads=6, kv=6, causal=True),
    "wide_windows": dict(ql=[40, 128] * 32, kl=[150, 60] * 32, heads=16, kv=16, window="random"),
}


@functools.lru_cache(maxsize=None)
def _batch(name):
    bt = Batch(seed=len(name) * 131 + sum(map(ord, name)), **BATCHES[name])
    return bt, Ref(bt)


def test_both_kinds_of_kernel_run():
    """More than 32 rows, and workgroups of 128 rows enough: the rule that attention_rows.h has."""
    wide = {name for name, a in BATCHES.items() if max(a["ql"]) > 32 and
            -(-max(a["ql"]) // 128) * a.get("heads", 2) * len(a["ql"]) >= (1024 if "window" in a else 128)}
    assert wide == {name for name in BATCHES if name.startswith("wide")}


@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 0), (3, 1)])
@pytest.mark.parametrize("name", BATCHES)
def test_forward(name, pad, shift):
    bt, ref = _batch(name)
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
    bt, ref = _batch(name)
    dq, dk, dv = backward(bt, ref, pad, shift)
    near(dq, ref.dq, ref.tol_dq, "dq")
    near(dk, ref.dk, ref.tol_dk, "dk")
    near(dv, ref.dv, ref.tol_dv, "dv")


@pytest.mark.parametrize("dtype", [torch.float32, BF16])
@pytest.mark.parametrize("name", ["self_padded", "cross", "windows_causal", "wide_causal"])
def test_backward_adds_the_other_gradient_of_the_queries(name, dtype):
    bt, _ = _batch(name)
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


# ------------------------------------------------------------------- what is not visible, tables, streams

SIZES = {
    # few rows a workgroup, and four waves of 32 rows each (chosen by the number of workgroups)
    "few": dict(ql=[40, 9], kl=[150, 70], heads=2, kv=2),
    "parts": dict(ql=[3, 1], kl=[2600, 130], heads=1, kv=1),
    "few_split": dict(ql=[3, 1], kl=[700, 130], heads=1, kv=1),
    "wide": dict(ql=[140] * 16, kl=[150] * 16, heads=4, kv=4),
    "wide_shared": dict(ql=[70] * 20, kl=[90] * 20, heads=8, kv=4),
    "wide_many": dict(ql=[140, 35] * 20, kl=[150, 40] * 20, heads=6, kv=6),
    "wide_windows": dict(ql=[40] * 64, kl=[150] * 64, heads=16, kv=16),
}


def _poison(bt, keep_q, keep_k, value):
    """Copies of the batch's rows with `value` in those that nothing may read (keep: [rows] bool)."""
    out = []
    for x, keep in ((bt.q, keep_q), (bt.k, keep_k), (bt.v, keep_k), (bt.dout, keep_q)):
        y = x.clone()
        y[~keep] = value
        out.append(y)
    return out


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf"), torch.finfo(BF16).min])
@pytest.mark.parametrize("name", SIZES)
def test_hidden_places_have_no_influence(name, value):
    """Rows of no sequence, padding, keys that no window reaches, and queries that see nothing hold `value`."""
    kw = SIZES[name]
    bt = Batch(seed=5, padded=True, lead=2, **kw)
    g = torch.Generator().manual_seed(6)
    # windows that leave out the keys from 3/5 to 4/5 of the sequence, and rows without any
    win = torch.zeros(bt.q_rows, 2, dtype=torch.int32)
    keep_q, keep_k = torch.zeros(bt.q_rows, dtype=torch.bool), torch.zeros(bt.k_rows, dtype=torch.bool)
    for b, (nq, nk) in enumerate(zip(bt.ql, bt.kl)):
        a, z = 3 * nk // 5, 4 * nk // 5
        for i in range(nq):
            if i % 5 == 4:
                continue
            low = i % 2 == 0
            lo = int(torch.randint(-3, max(a - 1, 1), (1,), generator=g)) if low else z + int(torch.randint(0, max(nk - z - 1, 1), (1,), generator=g))
            hi = min(lo + int(torch.randint(1, 60, (1,), generator=g)), a) if low else lo + int(torch.randint(1, 60, (1,), generator=g))
            win[bt.cu_q[b] + i] = torch.tensor([lo, hi])
            keep_q[bt.cu_q[b] + i] = True
        k0 = bt.cu_k[b]
        keep_k[k0:k0 + a] = True
        keep_k[k0 + z:k0 + nk] = True
    bt.window = win
    clean = [bt.q, bt.k, bt.v, bt.dout]
    bt.q, bt.k, bt.v, bt.dout = [torch.where(k[:, None], x, torch.zeros((), dtype=BF16)) for x, k in
                                 zip(clean, (keep_q, keep_k, keep_k, keep_q))]
    ref = Ref(bt)
    bt.q, bt.k, bt.v, bt.dout = _poison(bt, keep_q, keep_k, value)
    _, o, rest, lse = forward(bt)
    near(o.get(), ref.o, ref.tol_o, "o")
    near(lse.double().cpu(), ref.lse, ref.tol_lse, "lse")
    assert not bool(torch.isnan(rest.get()).any())
    dq, dk, dv = backward(bt, ref)
    near(dq, ref.dq, ref.tol_dq, "dq")
    near(dk, ref.dk, ref.tol_dk, "dk")
    near(dv, ref.dv, ref.tol_dv, "dv")


@pytest.mark.parametrize("name", ["few", "wide", "wide_many"])
def test_gradient_in_place_of_the_other_one_with_hidden_infinities(name):
    """dq written over dq_res, where the rows' first result is not finite: the other gradient is added once."""
    kw = dict(SIZES[name], kl=SIZES[name]["ql"])
    bt = Batch(seed=12, causal=True, **kw)
    res = torch.randn(bt.q_rows, 64 * bt.heads, generator=torch.Generator().manual_seed(2)).to(BF16)
    ref = Ref(bt, res)
    last = torch.tensor([c - 1 for c in bt.cu_q[1:]])
    bt.k[last] = float("inf")
    at = bt.handle()
    dq = put(res)
    dk, dv = torch.empty_like(bt.k, device="cuda"), torch.empty_like(bt.v, device="cuda")
    o = ref.o.to(BF16)
    ad.attention_backward(at, put(bt.q), put(bt.k), put(bt.v), put(o), put((ref.o - o.double()).to(BF16)), ref.lse.float().cuda(),
                          put(bt.dout), dq, dq, dk, dv, space(ad.attention_backward_workspace_size, at, bt))
    before = torch.ones(bt.q_rows, dtype=torch.bool)
    before[last] = False
    near(dq.double().cpu()[before], ref.dq[before], (ref.tol_dq + 2.0 ** -23 * res.double().abs())[before], "dq")


@pytest.mark.parametrize("heads", [4, 12])
def test_many_rows_without_keys_and_keys_without_rows(heads):
    """Four waves that meet at no tile still keep out of each other's places (4 heads: both gradients in one launch)."""
    for ql, kl in (([140] * 16, [0, 150] * 8), ([0, 140] * 8, [150] * 16)):
        bt = Batch(ql, kl, heads=heads, kv=heads, seed=heads)
        ref = Ref(bt)
        at, o, _, lse = forward(bt)
        near(o.get(), ref.o, ref.tol_o, "o")
        near(lse.double().cpu(), ref.lse, ref.tol_lse, "lse")
        dq, dk, dv = backward(bt, ref)
        near(dq, ref.dq, ref.tol_dq, "dq")
        near(dk, ref.dk, ref.tol_dk, "dk")
        near(dv, ref.dv, ref.tol_dv, "dv")


@pytest.mark.parametrize("name", ["few", "wide"])
def test_causal_rows_do_not_see_what_comes(name):
    """The last key and value hold NaN: the rows before are as without them; the last row is NaN."""
    kw = dict(SIZES[name], kl=SIZES[name]["ql"])
    bt = Batch(seed=8, causal=True, **kw)
    ref = Ref(bt)
    last = torch.tensor([c - 1 for c in bt.cu_q[1:]])
    bt.k[last], bt.v[last] = float("nan"), float("inf")
    _, o, _, lse = forward(bt)
    got, z = o.get(), lse.double().cpu()
    before = torch.ones(bt.q_rows, dtype=torch.bool)
    before[last] = False
    near(got[before], ref.o[before], ref.tol_o[before], "o")
    near(z[:, before], ref.lse[:, before], ref.tol_lse[:, before], "lse")
    assert bool(torch.isnan(got[last]).all()) and bool(torch.isnan(z[:, last]).all())
    dq, _, _ = backward(bt, ref)
    near(dq[before], ref.dq[before], ref.tol_dq[before], "dq")


def test_scores_without_a_finite_value():
    """A row whose scores are all -infinity gives 0, as one that sees nothing; a +infinity gives NaN."""
    bt = Batch([4], [70], heads=1, kv=1, seed=9)
    bt.q[:] = 0
    bt.q[:, 0] = torch.tensor([1.0, -1.0, 1.0, 0.5], dtype=BF16)
    bt.k[:, 0] = -float("inf")
    _, o, _, lse = forward(bt)
    got, z = o.get(), lse.cpu()[0]
    assert not bool(got[0].any()) and z[0] == -float("inf") and bool(torch.isnan(got[1]).all())


@pytest.mark.parametrize("name", ["few", "parts", "few_split", "wide"])
@pytest.mark.parametrize("what", ["past", "negative", "back", "long", "length"])
def test_tables_out_of_range(name, what):
    """The kernels' own checks: the sequence is left out and AD_ERR_LENGTH set, the others are right."""
    bt = Batch(seed=10, padded=True, **SIZES[name])
    n, ref = bt.batch, Ref(bt)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    cq, ql, q_max = list(bt.cu_q), list(bt.ql), max(bt.ql)
    if what == "past":
        cq[n] += 1000000
    elif what == "negative":
        cq[0] = -5
    elif what == "back":
        cq[n] = cq[n - 1] - 3
    elif what == "length":
        ql[n - 1] = q_max + 1
    elif what == "long":
        cq[n] += 1                       # inside the matrix, but more than q_max rows
    out_of = 0 if what == "negative" else n - 1
    extra = 4
    grow = lambda x: torch.cat([x, torch.zeros(extra, x.shape[1], dtype=BF16)])  # noqa: E731
    rows, w, wk = bt.q_rows + extra, 64 * bt.heads, 64 * bt.kv
    at = ad.Attention(bt.heads, bt.kv, ints(cq), ints(bt.cu_k), q_max, max(bt.kl), q_len=ints(ql), k_len=ints(bt.kl))
    o, lse = Out(rows, w), torch.full((bt.heads, rows), GUARD, device="cuda")
    q, do = put(grow(bt.q)), put(grow(bt.dout))
    k, v = put(bt.k), put(bt.v)
    buf = lambda size: torch.empty(size(at, rows, bt.k_rows), dtype=torch.uint8, device="cuda")  # noqa: E731
    ad.attention(at, q, k, v, o.t, lse, None, buf(ad.attention_workspace_size))
    assert int(at.err_flag) == ad.AD_ERR_LENGTH
    got = o.get()
    skip = torch.zeros(rows, dtype=torch.bool)
    skip[bt.cu_q[out_of]:bt.cu_q[out_of + 1]] = True
    skip[bt.q_rows:] = True
    assert bool((got[skip] == GUARD).all())
    near(got[:bt.q_rows][~skip[:bt.q_rows]], ref.o[~skip[:bt.q_rows]], ref.tol_o[~skip[:bt.q_rows]], "o")
    at.err_flag.zero_()
    dq, dk, dv = Out(rows, w), Out(bt.k_rows, wk), Out(bt.k_rows, wk)
    o32 = grow(ref.o.to(BF16))
    z = torch.zeros(bt.heads, rows, device="cuda")
    z[:, :bt.q_rows] = ref.lse.float().cuda()
    low = put(grow((ref.o - ref.o.to(BF16).double()).to(BF16)))
    ad.attention_backward(at, q, k, v, put(o32), low, z, do, None, dq.t, dk.t, dv.t, buf(ad.attention_backward_workspace_size))
    assert int(at.err_flag) == ad.AD_ERR_LENGTH
    got = dq.get()
    assert bool((got[skip] == GUARD).all())
    near(got[:bt.q_rows][~skip[:bt.q_rows]], ref.dq[~skip[:bt.q_rows]], ref.tol_dq[~skip[:bt.q_rows]], "dq")
    gone = torch.zeros(bt.k_rows, dtype=torch.bool)
    gone[bt.cu_k[out_of]:bt.cu_k[out_of + 1]] = True
    for x, want, tol in ((dk.get(), ref.dk, ref.tol_dk), (dv.get(), ref.dv, ref.tol_dv)):
        assert bool((x[gone] == GUARD).all())
        near(x[~gone], want[~gone], tol[~gone], "dk, dv")


def test_empty_batches():
    for ql, kl in (([0, 0], [0, 0]), ([0, 3], [5, 0]), ([4, 0], [0, 6])):
        bt = Batch(ql, kl, seed=11, lead=1)
        ref = Ref(bt)
        _, o, _, lse = forward(bt)
        assert torch.equal(o.get(), ref.o) and torch.equal(lse.double().cpu(), ref.lse)
        dq, dk, dv = backward(bt, ref)
        assert torch.equal(dq, ref.dq) and torch.equal(dk, ref.dk) and torch.equal(dv, ref.dv)
    e = torch.empty(0, 64, dtype=BF16, device="cuda")
    at = ad.Attention(1, 1, torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), 0, 0)
    ad.attention(at, e, e, e, e, torch.empty(1, 0, device="cuda"))
    ad.attention_backward(at, e, e, e, e, None, torch.empty(1, 0, device="cuda"), e, None, e, e, e, torch.empty(0, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("name", SIZES)
def test_other_streams_and_graph_replays(name):
    """Two calls at once on streams of their own, and a captured forward and backward pass replayed on new inputs with
    eager work between: the bits of the eager calls."""
    bts = [Batch(seed=20 + i, **SIZES[name]) for i in range(2)]

    class Call:
        def __init__(self, bt):
            self.at = bt.handle()
            self.i = [x.cuda() for x in (bt.q, bt.k, bt.v, bt.dout)]
            q, k = self.i[:2]
            self.o, self.rest, self.dq = torch.empty_like(q), torch.empty_like(q), torch.empty_like(q)
            self.dk, self.dv = torch.empty_like(k), torch.empty_like(k)
            self.lse = torch.empty(bt.heads, bt.q_rows, device="cuda")
            size = max(ad.attention_workspace_size(self.at, bt.q_rows, bt.k_rows),
                       ad.attention_backward_workspace_size(self.at, bt.q_rows, bt.k_rows))
            self.ws = torch.empty(size, dtype=torch.uint8, device="cuda")

        def __call__(self):
            q, k, v, do = self.i
            ad.attention(self.at, q, k, v, self.o, self.lse, self.rest, self.ws)
            ad.attention_backward(self.at, q, k, v, self.o, self.rest, self.lse, do, None, self.dq, self.dk, self.dv, self.ws)

        def outputs(self):
            return [t.clone() for t in (self.o, self.rest, self.lse, self.dq, self.dk, self.dv)]

    calls = [Call(bt) for bt in bts]
    want = []
    for c in calls:
        c()
        want.append(c.outputs())
    for c in calls:
        for t in (c.o, c.dq, c.dk, c.dv):
            t.fill_(1.0)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(4):
        for c, st in zip(calls, streams):
            with torch.cuda.stream(st):
                c()
    torch.cuda.synchronize()
    for c, w in zip(calls, want):
        assert all(torch.equal(a, b) for a, b in zip(c.outputs(), w))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls[0]()
    for k in range(3):
        for a, b in zip(calls[0].i, calls[k % 2].i if k else calls[0].i):
            a.copy_(b)
        graph.replay()
        torch.randn(5000, device="cuda").sum()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(calls[0].outputs(), want[k % 2])), k
        if k == 1:
            for a, b in zip(calls[0].i, [x.cuda() for x in (bts[0].q, bts[0].k, bts[0].v, bts[0].dout)]):
                a.copy_(b)


def test_the_same_call_gives_the_same_bits():
    bt = Batch(seed=30, **SIZES["wide_shared"])
    ref = Ref(bt)
    one = [x.get() for x in forward(bt)[1:3]] + list(backward(bt, ref))
    for _ in range(3):
        again = [x.get() for x in forward(bt)[1:3]] + list(backward(bt, ref))
        assert all(torch.equal(a, b) for a, b in zip(one, again))


@pytest.mark.parametrize("ql,kl", [([200], [600]), ([520] * 13, [600] * 13)])
def test_offsets_past_31_bits(ql, kl):
    """Rows 2^22 elements apart: the last rows lie past 2^31 elements (and 2^32 bytes)."""
    ld, heads = 1 << 22, 2
    bt = Batch(ql[:1], kl[:1], heads=heads, kv=heads, causal=True, seed=31)
    # the batch's sequences share their rows' values; only the first one and the last one are looked at
    n = len(ql)
    rows_q, rows_k = sum(ql), sum(kl)
    if n > 1:       # (enough workgroups for the other kernels; rows closer together)
        ld = 1 << 19
    flat = torch.empty(rows_k * ld, dtype=BF16, device="cuda")
    kv = flat.view(rows_k, ld)
    k, v = kv[:, 8:8 + 64 * heads], kv[:, ld - 64 * heads:]
    k.copy_(bt.k.cuda().repeat(n, 1))
    v.copy_(bt.v.cuda().repeat(n, 1))
    q, do = bt.q.cuda().repeat(n, 1), bt.dout.cuda().repeat(n, 1)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    at = ad.Attention(heads, heads, ints([i * ql[0] for i in range(n + 1)]), ints([i * kl[0] for i in range(n + 1)]), ql[0], kl[0],
                      causal=True)
    ref = Ref(bt)
    o, lse = torch.empty_like(q), torch.empty(heads, rows_q, device="cuda")
    buf = lambda size: torch.empty(size(at, rows_q, rows_k), dtype=torch.uint8, device="cuda")  # noqa: E731
    ad.attention(at, q, k, v, o, lse, None, buf(ad.attention_workspace_size))
    near(o[-ql[0]:].double().cpu(), ref.o, ref.tol_o, "o")
    dk, dv = kv[:, 256:256 + 64 * heads], kv[:, 1024:1024 + 64 * heads]
    o16 = ref.o.to(BF16)
    rest = (ref.o - o16.double()).to(BF16).cuda().repeat(n, 1)
    dq = torch.empty_like(q)
    ad.attention_backward(at, q, k, v, o16.cuda().repeat(n, 1), rest, ref.lse.float().cuda().repeat(1, n), do, None, dq, dk, dv,
                          buf(ad.attention_backward_workspace_size))
    near(dq[-ql[0]:].double().cpu(), ref.dq, ref.tol_dq, "dq")
    near(dk[-kl[0]:].double().cpu(), ref.dk, ref.tol_dk, "dk")
    near(dv[-kl[0]:].double().cpu(), ref.dv, ref.tol_dv, "dv")
