"""Every kernel that a product can be given, and every way of cutting one, against float64.

tests/linear_kernels.py lists sizes by the kernel that they reach.  Tolerances are those of
tests/test_gpu_train_ops.py: K products exact in float32 sum to within 2 K 2^-24 sum |a b|, and a rounding to
bf16 is 2^-8 of the value.  The references are float64 products on the GPU."""
import pytest
import torch

import linear_kernels as sizes
from paper_2608_12703_amd import ad
from test_gpu_train_ops import BF16, F32, GUARD, U, Out, _gelu, _put, _slope, _space, _two

pytestmark = pytest.mark.gpu


def _draws(*seed):
    g = torch.Generator(device="cuda").manual_seed(sum((i + 1) * s for i, s in enumerate(seed)))
    return lambda *s, scale=1.0, dtype=BF16: (torch.randn(*s, generator=g, device="cuda") * scale).to(dtype)


def _get(out: Out):
    """An output's values in float64, on the GPU; nothing around them was written."""
    v = out.t.double()
    out.t.fill_(GUARD)
    assert bool((out.flat == GUARD).all()), "wrote outside the output"
    return v


def _near(got, want, tol, what):
    bad = ~((got - want).abs() <= tol)
    assert not bool(bad.any()), (what, float((got - want).abs()[bad].max()), bad.nonzero()[:3].tolist(), tuple(want.shape))


def _check_ckpt(k, v, tol):
    """A checkpoint of values known to within tol: its scales, its padding, and the values to half a step."""
    rows, cols = v.shape
    wide, slack = (torch.zeros(k.q.shape, dtype=torch.float64, device="cuda") for _ in range(2))
    wide[:, :cols], slack[:, :cols] = v, tol
    assert not bool(k.q[:, cols:].any())
    step = torch.exp2(k.scale.double() - 127.0)
    top, give = wide.abs().view(rows, -1, 32).amax(-1), slack.view(rows, -1, 32).amax(-1)
    assert bool((127 * step >= top - give).all()), "scale too small"
    assert bool(((127 * step / 2 <= top + give) | (k.scale == 1)).all()), "scale too large"
    off = (k.q.double().view(rows, -1, 32) * step[:, :, None]).view(rows, -1) - wide
    assert bool((off.abs() <= step.repeat_interleave(32, dim=1) / 2 + slack).all()), "further than half a step"


def _products(a, b):
    """a @ b and |a| @ |b| in float64 (contiguous operands)."""
    a, b = a.double().contiguous(), b.double().contiguous()
    return a @ b, a.abs() @ b.abs()


def _forward(rows, n, k, pad, shift, act, rt, yt, keep, parts=None):
    rnd = _draws(rows, n, k)
    x, w, bias = rnd(rows, k), rnd(n, k, scale=k ** -0.5), rnd(n)
    res = None if rt is None else rnd(rows, n, dtype=rt)
    y = Out(rows, n, yt, pad, shift)
    pre = Out(rows, n, BF16, pad, shift) if keep == "bf16" else None
    kept = ad.Ckpt.empty(rows, n) if keep == "ckpt" else None
    space = ad.linear_workspace_size(rows, n, k)
    assert parts is None or (space > 0) == parts
    ad.linear(_put(x, pad, shift), _put(w, pad, shift), bias, act, None if res is None else _put(res, pad, shift), y.t,
              None if pre is None else pre.t, kept, _space(space))
    h, mag = _products(x, w.t())
    h += bias.double()
    th = 2 * k * U * mag + 2 * U * (h.abs() + bias.double().abs())
    out, tol = (_gelu(h), 1.13 * th + h.abs() * (1e-7 + 8 * U)) if act == ad.ACT_GELU else (h, th)
    if res is not None:
        out = out + res.double()
        tol = tol + 2 * U * (out.abs() + res.double().abs())
    _near(_get(y), out, tol * 1.01 + out.abs() * _two(yt), "y")
    if pre is not None:
        _near(_get(pre), h, th * 1.01 + h.abs() * 2.0 ** -8, "pre")
    if kept is not None:
        _check_ckpt(kept, h, th)


def _dgrad(rows, n, k, pad, shift, src, ot, again):
    rnd = _draws(7, rows, n, k)
    dy, w, h16 = rnd(rows, n), rnd(n, k, scale=n ** -0.5), rnd(rows, k, scale=2.0)
    kept, h = None, h16.double()
    if src == "ckpt":
        kept, v = ad.Ckpt.empty(rows, k), torch.empty(rows, k, device="cuda")
        ad.ckpt_pack(h16, kept)
        ad.ckpt_unpack(kept, v)
        h = v.double()
    dx = Out(rows, k, ot, pad, shift)
    act_out = Out(rows, k, BF16, pad, shift) if again else None
    ad.linear_dgrad(_put(dy, pad, shift), _put(w, pad, shift), ad.ACT_NONE if src == "none" else ad.ACT_GELU,
                    _put(h16, pad, shift) if src == "bf16" else None, kept, dx.t, act_out.t if again else None,
                    _space(ad.linear_dgrad_workspace_size(rows, n, k)))
    want, mag = _products(dy, w)
    tol = 2 * n * U * mag
    if src != "none":
        s = _slope(h)
        tol = tol * 1.13 + want.abs() * (1e-7 + 16 * U) + 2 * U * (want * s).abs()
        want = want * s
    _near(_get(dx), want, tol * 1.01 + want.abs() * _two(ot), "dx")
    if again:
        _near(_get(act_out), _gelu(h), h.abs() * 1e-7 + _gelu(h).abs() * (8 * U + 2.0 ** -8) + 1e-37, "act_out")


def _wgrad(rows, n, k, pad, shift, src, parts=None):
    rnd = _draws(13, rows, n, k)
    dy, x16, kept, gain, shift_v = rnd(rows, n), rnd(rows, k), None, None, None
    x = mag = x16.double()
    if src != "bf16":
        kept, v = ad.Ckpt.empty(rows, k), torch.empty(rows, k, device="cuda")
        ad.ckpt_pack(x16, kept)
        ad.ckpt_unpack(kept, v)
        x = mag = v.double()
    if src == "affine":
        gain, shift_v = 1 + rnd(k, scale=0.1), rnd(k)
        x, mag = x * gain.double() + shift_v.double(), x.abs() * gain.double().abs() + shift_v.double().abs()
    dw, dbias = Out(n, k, F32, pad, shift), torch.empty(n, device="cuda")
    space = ad.linear_wgrad_workspace_size(rows, n, k)
    assert parts is None or (space > 0) == parts
    ws = _space(space)
    args = (_put(dy, pad, shift), _put(x16, pad, shift) if kept is None else None, kept, gain, shift_v)
    ad.linear_wgrad(*args, dw.t, dbias, ws)
    d = dy.double().t().contiguous()
    one, bias_one = dw.t.clone(), dbias.clone()
    _near(one.double(), d @ x, 2 * (rows + 4) * U * (d.abs() @ mag.abs()), "dw")
    _near(bias_one.double(), d.sum(1), 2 * (rows + 4) * U * d.abs().sum(1), "dbias")
    ad.linear_wgrad(*args, dw.t, dbias, ws, accumulate=True)
    assert torch.equal(dbias, bias_one + bias_one)
    assert torch.equal(_get(dw), (one + one).double())


FORWARD = [(ad.ACT_GELU, None, BF16, "ckpt"), (ad.ACT_NONE, F32, F32, None), (ad.ACT_GELU, BF16, F32, "bf16")]
DGRAD = [("none", BF16, False), ("bf16", F32, True), ("ckpt", BF16, True)]
LARGE = sizes.TILES_256 + sizes.TILES_128


@pytest.mark.parametrize("act,rt,yt,keep", FORWARD)
@pytest.mark.parametrize("P,Q,K,pad,shift,kernel", LARGE)
def test_forward_tiles(P, Q, K, pad, shift, kernel, act, rt, yt, keep):
    _forward(Q, P, K, pad, shift, act, rt, yt, keep)


@pytest.mark.parametrize("src,ot,again", DGRAD)
@pytest.mark.parametrize("P,Q,K,pad,shift,kernel", LARGE)
def test_input_gradient_tiles(P, Q, K, pad, shift, kernel, src, ot, again):
    _dgrad(Q, K, P, pad, shift, src, ot, again)


@pytest.mark.parametrize("P,Q,K,pad,shift,kernel,src",
                         [(*t, src) for t in sizes.WGRAD_256 for src in ("bf16", "ckpt", "affine")]
                         + [(*t, "bf16") for t in sizes.WGRAD_256_BF16]
                         + [(*t, src) for t in sizes.WGRAD_256_CKPT for src in ("ckpt", "affine")])
def test_weight_gradient_tiles_of_256(P, Q, K, pad, shift, kernel, src):
    _wgrad(K, Q, P, pad, shift, src)


@pytest.mark.parametrize("act,rt,yt,keep", [(ad.ACT_GELU, None, BF16, None), (ad.ACT_NONE, F32, F32, None),
                                            (ad.ACT_GELU, BF16, F32, "bf16"), (ad.ACT_NONE, BF16, BF16, "bf16")])
@pytest.mark.parametrize("rows,n,k,pad,kernel", sizes.FEW)
def test_few_rows(rows, n, k, pad, kernel, act, rt, yt, keep):
    _forward(rows, n, k, pad, pad, act, rt, yt, keep)


def test_few_rows_over_their_residual():
    """y may be the residual; a row of NaN stays a row of NaN."""
    for rows, n, k in ((1, 5120, 1280), (17, 384, 1280), (32, 4104, 200), (5, 200, 64)):
        rnd = _draws(rows, n, k)
        x, w, res, y = rnd(rows, k), rnd(n, k), rnd(rows, n, dtype=F32), torch.empty(rows, n, device="cuda")
        ws = _space(ad.linear_workspace_size(rows, n, k))
        ad.linear(x, w, None, ad.ACT_NONE, res, y, None, None, ws)
        over = res.clone()
        ad.linear(x, w, None, ad.ACT_NONE, over, over, None, None, ws)
        assert torch.equal(over, y)
        x[rows - 1, k - 1] = float("nan")
        ad.linear(x, w, None, ad.ACT_NONE, res, over, None, None, ws)
        assert bool(torch.isnan(over[rows - 1]).all()) and torch.equal(over[:rows - 1], y[:rows - 1])


@pytest.mark.parametrize("act,rt,yt,keep", FORWARD)
@pytest.mark.parametrize("rows,n,k,pad,shift,kernel", sizes.ANY_FWD)
def test_forward_any_alignment_in_parts(rows, n, k, pad, shift, kernel, act, rt, yt, keep):
    _forward(rows, n, k, pad, shift, act, rt, yt, keep, parts=True)


@pytest.mark.parametrize("src,ot,again", DGRAD)
@pytest.mark.parametrize("rows,n,k,pad,shift,kernel", sizes.ANY_DGRAD)
def test_input_gradient_any_alignment_in_parts(rows, n, k, pad, shift, kernel, src, ot, again):
    assert ad.linear_dgrad_workspace_size(rows, n, k) > 0
    _dgrad(rows, n, k, pad, shift, src, ot, again)


@pytest.mark.parametrize("rows,n,k,pad,shift,kernel,src", [(*t, "bf16") for t in sizes.ANY_WGRAD]
                         + [(*t, src) for t in sizes.ANY_WGRAD_CKPT for src in ("ckpt", "affine")])
def test_weight_gradient_any_alignment_in_parts(rows, n, k, pad, shift, kernel, src):
    _wgrad(rows, n, k, pad, shift, src, parts=True)


@pytest.mark.parametrize("pad", [0, 1])         # whole vectors, and none
def test_every_number_of_steps(pad):
    for K in sizes.STEPS:
        _forward(40, 136, K, pad, 0, ad.ACT_GELU, None, F32, "ckpt")
        _dgrad(40, K, 136, pad, 0, "bf16", F32, True)
        for src in ("bf16", "affine"):
            _wgrad(K, 40, 136, pad, 0, src)


@pytest.mark.parametrize("odd", ["x", "w", "residual", "y", "pre", "bias"])
def test_one_matrix_without_vectors(odd):
    """Any one argument may lie anywhere; the others' padding stays as it was."""
    rows, n, k = 140, 264, 584
    rnd = _draws(rows, n, k)
    x, w, bias, res = rnd(rows, k), rnd(n, k, scale=k ** -0.5), rnd(n + 1), rnd(rows, n, dtype=F32)
    at = lambda name, t: _put(t, 3, 1) if name == odd else _put(t)  # noqa: E731
    y, pre = (Out(rows, n, t, 3 if name == odd else 0, 1 if name == odd else 0) for name, t in (("y", F32), ("pre", BF16)))
    bias = bias[1:] if odd == "bias" else bias[:n]
    ad.linear(at("x", x), at("w", w), bias, ad.ACT_GELU, at("residual", res), y.t, pre.t, None,
              _space(ad.linear_workspace_size(rows, n, k)))
    h, mag = _products(x, w.t())
    h += bias.double()
    th = 2 * k * U * mag + 2 * U * (h.abs() + bias.double().abs())
    out = _gelu(h) + res.double()
    tol = 1.13 * th + h.abs() * (1e-7 + 8 * U) + 2 * U * (out.abs() + res.double().abs())
    _near(_get(y), out, tol * 1.01 + out.abs() * U, "y")
    _near(_get(pre), h, th * 1.01 + h.abs() * 2.0 ** -8, "pre")
