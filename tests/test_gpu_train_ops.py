"""The training operators (LayerNorm, projections and their gradients, 8-bit checkpoints)
against their definitions in float64.

Tolerances.  u = 2^-24 is half a float32 step, 2^-8 half a bf16 step (relative).  bf16 operands'
products are exact in float32, so a sum of K of them is off by at most K u sum |a b| in any
order; twice that is allowed (the matrix instruction adds several products at once).  A value
that is rounded to bf16 on top is off by 2^-8 of itself.  LayerNorm's row sums are trees of depth
at most 8 J + 8 <= 40 over a row of up to 2048 columns (J pieces of 8 in a lane), as deep for
wider rows: u * 48 of the sum of magnitudes bounds them.  A checkpoint holds a value to half of its
group's step.  GELU: erf is allowed 2e-7 absolute (an approximation good to 1.5e-7, and its
roundings), so h Phi(h) is off by |h| 1e-7 and a few roundings.
"""
import math

import numpy as np
import pytest
import torch

from paper_2608_12703_amd import ad
from paper_2608_12703_amd.train import FeedForward

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32
GUARD = -77.0


def _rand(g, *shape, scale=1.0, dtype=F32):
    return (torch.randn(*shape, generator=g) * scale).to(dtype)


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _put(t, pad=0, shift=0):
    """t on the GPU, rows `pad` elements apart, the first one `shift` elements into its buffer."""
    rows, cols = t.shape
    flat = torch.full((rows * (cols + pad) + shift + 8,), GUARD, dtype=t.dtype, device="cuda")
    view = flat[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(t)
    return view


class Out:
    """A [rows][cols] output inside a guarded buffer."""

    def __init__(self, rows, cols, dtype, pad=0, shift=0):
        n = rows * (cols + pad)
        self.flat = torch.full((shift + n + 64,), GUARD, dtype=dtype, device="cuda")
        self.t = self.flat[shift:shift + n].view(rows, cols + pad)[:, :cols]

    def get(self):
        """The values in float64; nothing around them was written."""
        v = self.t.double().cpu()
        self.t.fill_(GUARD)
        assert bool((self.flat == GUARD).all()), "wrote outside the output"
        return v


def _two(dtype):
    return 2.0 ** -8 if dtype == BF16 else U


def _near(got, want, tol, what):
    bad = ~((got - want).abs() <= tol)
    assert not bool(bad.any()), (what, float((got - want).abs()[bad].max()), int(bad.sum()), tuple(want.shape))


# ------------------------------------------------------------------- 8-bit checkpoints

def _pack_ref(v):
    """(q, s) of float32 rows v from the definition, in float64."""
    v = np.asarray(v, dtype=np.float64)
    rows, cols = v.shape
    ld = ad.LIB.ad_ckpt_ld(cols)
    wide = np.zeros((rows, ld))
    wide[:, :cols] = v
    q, s = np.zeros((rows, ld), np.int8), np.ones((rows, ld // 32), np.uint8)
    for r in range(rows):
        for j in range(ld // 32):
            x = wide[r, 32 * j:32 * j + 32]
            if not np.isfinite(x).all():
                s[r, j] = 255
                continue
            top, e = np.abs(x).max(), 1
            if top > 0:
                e = max(1, math.ceil(math.log2(top / 127.0)) + 127 - 2)
                while top > 127.0 * 2.0 ** (e - 127):
                    e += 1
            s[r, j] = e
            q[r, 32 * j:32 * j + 32] = np.rint(x / 2.0 ** (e - 127))      # exact quotient, ties to even
    return q, s


def _value_ref(q, s, cols):
    two = np.where(s == 255, np.nan, 2.0 ** (s.astype(np.float64) - 127))
    return torch.from_numpy((q.astype(np.float64).reshape(*s.shape, 32) * two[:, :, None]).reshape(q.shape)[:, :cols])


def _special(rows, cols, seed):
    v = np.random.default_rng(seed).standard_normal((rows, cols)).astype(np.float32)
    v *= 2.0 ** np.random.default_rng(seed + 1).integers(-8, 8, (rows, 1))
    if rows > 6 and cols >= 33:
        v[0] = 0.0
        v[1, :32] = 127.0 / 64.0 * 0.25          # the largest magnitude exactly 127 steps
        v[2, 5] = np.nextafter(np.float32(127.0 / 64.0), np.float32(4.0))
        v[3, :4] = [63.5, 0.5, 1.5, -2.5]        # ties at step 0.5 .. 1
        v[3, 4:32] = 0.25
        v[4, :32] *= np.float32(1e-42)           # below the normal range
        v[5, 7] = np.inf
        v[6, 32] = np.nan
    return v


@pytest.mark.parametrize("rows,cols,dtype,pad,shift", [
    (7, 384, F32, 0, 0), (9, 384, BF16, 0, 0), (1, 1, F32, 0, 0), (3, 31, BF16, 1, 1), (8, 33, F32, 0, 1),
    (64, 1280, BF16, 8, 0), (11, 1000, F32, 5, 0), (10, 1001, BF16, 0, 3), (2, 5120, F32, 0, 0), (0, 64, F32, 0, 0)])
def test_checkpoint_is_the_definition(rows, cols, dtype, pad, shift):
    x = torch.from_numpy(_special(rows, cols, rows + cols)).to(dtype)
    q, s = _pack_ref(x.float().numpy())
    k = ad.Ckpt.empty(rows, cols)
    k.q.fill_(-128)
    k.scale.fill_(77)
    ad.ckpt_pack(_put(x, pad, shift), k)
    np.testing.assert_array_equal(k.scale.cpu().numpy(), s)
    np.testing.assert_array_equal(k.q.cpu().numpy(), q)
    want = _value_ref(q, s, cols)
    for out_dtype in (F32, BF16):
        out = Out(rows, cols, out_dtype, pad, shift)
        ad.ckpt_unpack(k, out.t)
        np.testing.assert_array_equal(out.get().numpy(), want.numpy())     # exact in both
        gelu = Out(rows, cols, out_dtype, pad, shift)
        ad.ckpt_unpack(k, gelu.t, act=ad.ACT_GELU)
        g = 0.5 * want * (1 + torch.erf(want * math.sqrt(0.5)))
        got = gelu.get()
        assert bool((torch.isnan(got) == torch.isnan(g)).all())
        _near(torch.nan_to_num(got), torch.nan_to_num(g),
              torch.nan_to_num(want.abs() * 1e-7 + g.abs() * (8 * U + _two(out_dtype)) + 1e-37), "gelu")


def _check_ckpt(k, v, tol, what):
    """A checkpoint of values v known to within tol: its scales, and the values to half a step."""
    rows, cols = v.shape
    q, s = k.q.cpu().numpy(), k.scale.cpu().numpy().astype(np.int64)
    ld = q.shape[1]
    wide, slack = np.zeros((rows, ld)), np.zeros((rows, ld))
    wide[:, :cols], slack[:, :cols] = v.numpy(), tol.numpy()
    assert not q[:, cols:].any(), f"{what}: padding"
    top = np.abs(wide).reshape(rows, -1, 32).max(-1)
    give = slack.reshape(rows, -1, 32).max(-1)
    step = 2.0 ** (s - 127.0)
    assert (127 * step >= top - give).all(), f"{what}: scale too small"
    assert ((127 * step / 2 <= top + give) | (s == 1)).all(), f"{what}: scale too large"
    off = np.abs((q.reshape(rows, -1, 32) * step[:, :, None]).reshape(rows, ld) - wide)
    assert (off <= np.repeat(step, 32, axis=1) / 2 + slack).all(), f"{what}: further than half a step"


# ---------------------------------------------------------------------------- LayerNorm

LN_SHAPES = [(1, 1), (1, 64), (5, 7), (7, 384), (33, 511), (130, 768), (9, 1000), (6, 1280), (3, 1537), (4, 2048),
             (3, 2049), (5, 4096), (2, 5000), (3, 8192)]


@pytest.mark.parametrize("rows,cols", LN_SHAPES)
@pytest.mark.parametrize("xt,yt,pt,pad,shift,keep", [
    (F32, BF16, BF16, 0, 0, True), (F32, F32, F32, 0, 0, False), (BF16, BF16, BF16, 3, 1, True), (BF16, F32, F32, 8, 0, True)])
def test_layer_norm(rows, cols, xt, yt, pt, pad, shift, keep):
    g = _gen(rows * 10007 + cols)
    x = _rand(g, rows, cols)
    x = (x * 3 + 20 * _rand(g, rows, 1)).to(xt)       # row means far larger than the spread
    gain, bias = (1 + _rand(g, cols, scale=0.1)).to(pt), _rand(g, cols, scale=0.1, dtype=pt)
    y = Out(rows, cols, yt, pad, shift)
    mean, rstd = torch.full((rows,), GUARD, device="cuda"), torch.full((rows,), GUARD, device="cuda")
    k = ad.Ckpt.empty(rows, cols) if keep else None
    ad.layer_norm(_put(x, pad, shift), gain.cuda(), bias.cuda(), y.t, mean, rstd, k)
    X, G, B = x.double(), gain.double(), bias.double()
    mu = X.mean(1, keepdim=True)
    r = 1 / torch.sqrt((X - mu).square().mean(1, keepdim=True) + 1e-5)
    xh = (X - mu) * r
    dmu = 48 * U * X.abs().mean(1, keepdim=True)
    # the deviations are taken from the float32 mean: off by dmu each, which shifts the variance by dmu^2
    drel = 48 * U + 0.5 * (dmu * r).square()
    _near(mean.double().cpu()[:, None], mu, dmu, "mean")
    _near(rstd.double().cpu()[:, None], r, r * drel, "rstd")
    tol = dmu * r + xh.abs() * (drel + 4 * U)
    out = xh * G + B
    _near(y.get(), out, (tol * G.abs() + 3 * U * ((xh * G).abs() + B.abs())) * (1 + _two(yt)) + out.abs() * _two(yt), "y")
    if keep:
        _check_ckpt(k, xh, tol, "xhat")


def test_layer_norm_in_place_and_empty():
    g = _gen(3)
    x, gain, bias = _rand(g, 40, 320), 1 + _rand(g, 320, scale=0.1), _rand(g, 320)
    a, b = x.cuda(), torch.empty(40, 320, device="cuda")
    ad.layer_norm(a, gain.cuda(), bias.cuda(), b)
    ad.layer_norm(a, gain.cuda(), bias.cuda(), a)
    assert torch.equal(a, b)
    e = torch.empty(0, 320, device="cuda")
    ad.layer_norm(e, gain.cuda(), bias.cuda(), e, e.new_empty(0), e.new_empty(0), ad.Ckpt.empty(0, 320))


def test_layer_norm_row_of_equal_values_and_nan_row():
    x = torch.zeros(4, 256)
    x[1] = 3.0
    x[2, 9] = float("nan")
    x[3, 8] = float("inf")
    y, k = torch.empty(4, 256, device="cuda"), ad.Ckpt.empty(4, 256)
    one, zero = torch.ones(256, device="cuda"), torch.zeros(256, device="cuda")
    ad.layer_norm(x.cuda(), one, zero, y, xhat=k)
    y = y.cpu()
    assert not y[:2].any() and bool(torch.isnan(y[2]).all()) and bool(torch.isnan(y[3]).any())
    v = torch.empty(4, 256, device="cuda")
    ad.ckpt_unpack(k, v)
    assert not v[:2].cpu().any() and bool(torch.isnan(v[2]).all())


def _ln_bwd_ref(dy, xh, r, gain, dres):
    n = dy.shape[1]
    d = dy * gain
    a, b = d.sum(1, keepdim=True) / n, (d * xh).sum(1, keepdim=True) / n
    dx = r * (d - a - xh * b) + (0 if dres is None else dres)
    tol = 64 * U * r * (d.abs() + d.abs().mean(1, keepdim=True) + xh.abs() * (d * xh).abs().mean(1, keepdim=True)) \
        + 2 * U * dx.abs() + (0 if dres is None else 2 * U * dres.abs())
    return dx, tol


@pytest.mark.parametrize("rows,cols", LN_SHAPES + [(2100, 192)])
@pytest.mark.parametrize("src,dt,rt,ot,pt,pad,shift", [
    ("ckpt", BF16, F32, F32, BF16, 0, 0), ("x", F32, None, F32, F32, 0, 0), ("x16", BF16, BF16, BF16, BF16, 3, 1),
    ("ckpt", F32, F32, BF16, F32, 8, 0)])
def test_layer_norm_backward(rows, cols, src, dt, rt, ot, pt, pad, shift):
    g = _gen(rows * 101 + cols)
    x = (_rand(g, rows, cols) * 2 + _rand(g, rows, 1)).to(BF16 if src == "x16" else F32)
    dy, gain = _rand(g, rows, cols, dtype=dt), (1 + _rand(g, cols, scale=0.1)).to(pt)
    dres = None if rt is None else _rand(g, rows, cols, dtype=rt)
    mean = x.double().mean(1).float()
    rstd = (1 / torch.sqrt(x.double().var(1, unbiased=False) + 1e-5)).float()
    r = rstd.double()[:, None]
    k = None
    if src == "ckpt":
        k = ad.Ckpt.empty(rows, cols)
        ad.ckpt_pack(((x.double() - mean.double()[:, None]) * r).float().cuda(), k)
        xh = _value_ref(k.q.cpu().numpy(), k.scale.cpu().numpy(), cols)
    else:
        xh = (x.double() - mean.double()[:, None]) * r
    # x - mean in float32 is off by half a step of itself, so xhat by 2 u of itself: within the bounds
    dx, copy = Out(rows, cols, ot, pad, shift), Out(rows, cols, BF16, pad, shift)
    dgain, dbias = torch.full((cols,), 5.0, device="cuda"), torch.full((cols,), -3.0, device="cuda")
    ws = torch.empty(ad.layer_norm_backward_workspace_size(rows, cols), dtype=torch.uint8, device="cuda")
    args = (_put(dy, pad, shift), None if k else _put(x, pad, shift), None if k else mean.cuda(), rstd.cuda(), k,
            gain.cuda(), None if dres is None else _put(dres, pad, shift))
    ad.layer_norm_backward(*args, dx.t, copy.t, dgain, dbias, ws)
    first = dgain.clone(), dbias.clone()
    ad.layer_norm_backward(*args, dx.t, copy.t, dgain, dbias, ws, accumulate=True)
    D, R = dy.double(), None if dres is None else dres.double()
    want, tol = _ln_bwd_ref(D, xh, r, gain.double(), R)
    _near(dx.get(), want, tol * (1 + _two(ot)) + want.abs() * _two(ot), "dx")
    _near(copy.get(), want, tol * 1.01 + want.abs() * 2.0 ** -8, "dx_copy")
    n = rows + 40
    for name, got, ref, mag in (("dgain", 0, (D * xh).sum(0), (D * xh).abs().sum(0)), ("dbias", 1, D.sum(0), D.abs().sum(0))):
        _near(first[got].double().cpu(), ref, n * U * mag, name)
        both = (dgain, dbias)[got]
        assert torch.equal(both, first[got] + first[got]), f"{name}: accumulate"


def test_layer_norm_backward_aliases_no_params_and_empty():
    g = _gen(8)
    rows, cols = 50, 640
    dy, dres, gain = (_rand(g, rows, cols).cuda(), _rand(g, rows, cols).cuda(), _rand(g, cols).cuda())
    k, rstd = ad.Ckpt.empty(rows, cols), torch.rand(rows, generator=g).cuda()
    ad.ckpt_pack(_rand(g, rows, cols).cuda(), k)
    want = torch.empty_like(dy)
    ad.layer_norm_backward(dy, None, None, rstd, k, gain, dres, want, None, None, None, None)
    for alias in ("dres", "dy"):
        t = dict(dy=dy.clone(), dres=dres.clone())
        ad.layer_norm_backward(t["dy"], None, None, rstd, k, gain, t["dres"], t[alias], None, None, None, None)
        assert torch.equal(t[alias], want), alias
    e = torch.empty(0, cols, device="cuda")
    dg, db = torch.ones(cols, device="cuda"), torch.ones(cols, device="cuda")
    ad.layer_norm_backward(e, None, None, e.new_empty(0), ad.Ckpt.empty(0, cols), gain, None, e, None, dg, db, None,
                           accumulate=True)
    assert bool((dg == 1).all() and (db == 1).all())
    ad.layer_norm_backward(e, None, None, e.new_empty(0), ad.Ckpt.empty(0, cols), gain, None, e, None, dg, db, None)
    assert not dg.any() and not db.any()


# ---------------------------------------------------------------------------- products

# rows, n, k, padding, first element's offset: single rows and columns, tiles with one row or
# column over, splits of the reduction, sizes that no vector load divides
SHAPES = [(1, 1, 1, 0, 0), (1, 64, 64, 0, 0), (1, 1280, 5120, 0, 0), (2, 8, 8, 0, 0), (7, 384, 1536, 0, 0),
          (16, 130, 200, 6, 0), (17, 129, 65, 0, 1), (33, 1001, 77, 3, 0), (128, 128, 64, 0, 0), (129, 136, 1000, 8, 0),
          (200, 72, 4096, 0, 0), (257, 264, 264, 0, 0), (300, 1280, 320, 0, 0), (515, 640, 136, 8, 0), (1000, 24, 40, 0, 0),
          (640, 2056, 72, 0, 0), (64, 5120, 128, 0, 8)]


def _gelu(h):
    return 0.5 * h * (1 + torch.erf(h * math.sqrt(0.5)))


def _slope(h):
    return 0.5 * (1 + torch.erf(h * math.sqrt(0.5))) + h * torch.exp(-0.5 * h * h) / math.sqrt(2 * math.pi)


def _space(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda") if n else None


@pytest.mark.parametrize("rows,n,k,pad,shift", SHAPES)
@pytest.mark.parametrize("act,rt,yt,keep,bt", [
    (ad.ACT_GELU, None, BF16, "ckpt", BF16), (ad.ACT_NONE, F32, F32, None, BF16), (ad.ACT_GELU, BF16, F32, "bf16", F32),
    (ad.ACT_NONE, None, BF16, "ckpt", None)])
def test_linear(rows, n, k, pad, shift, act, rt, yt, keep, bt):
    g = _gen(rows + 31 * n + 977 * k)
    x, w = _rand(g, rows, k, dtype=BF16), _rand(g, n, k, scale=k ** -0.5, dtype=BF16)
    bias = None if bt is None else _rand(g, n, dtype=bt)
    res = None if rt is None else _rand(g, rows, n, dtype=rt)
    y = Out(rows, n, yt, pad, shift)
    pre = Out(rows, n, BF16, pad, shift) if keep == "bf16" else None
    kept = ad.Ckpt.empty(rows, n) if keep == "ckpt" else None
    ws = _space(ad.linear_workspace_size(rows, n, k))
    ad.linear(_put(x, pad, shift), _put(w, pad, shift), None if bias is None else bias.cuda(), act,
              None if res is None else _put(res, pad, shift), y.t, None if pre is None else pre.t, kept, ws)
    X, W = x.double(), w.double()
    B = torch.zeros(n, dtype=torch.float64) if bias is None else bias.double()
    h = X @ W.T + B
    th = 2 * k * U * (X.abs() @ W.abs().T) + 2 * U * (h.abs() + B.abs())
    out, tol = (_gelu(h), 1.13 * th + h.abs() * (1e-7 + 8 * U)) if act == ad.ACT_GELU else (h, th)
    if res is not None:
        out = out + res.double()
        tol = tol + 2 * U * (out.abs() + res.double().abs())
    _near(y.get(), out, tol * 1.01 + out.abs() * _two(yt), "y")
    if pre is not None:
        _near(pre.get(), h, th * 1.01 + h.abs() * 2.0 ** -8, "pre")
    if kept is not None:
        _check_ckpt(kept, h, th, "pre")


@pytest.mark.parametrize("rows,n,k,pad,shift", SHAPES)
@pytest.mark.parametrize("src,ot,again", [("none", BF16, False), ("bf16", F32, True), ("ckpt", BF16, True), ("ckpt", F32, False)])
def test_linear_dgrad(rows, n, k, pad, shift, src, ot, again):
    g = _gen(7 * rows + 31 * n + 977 * k)
    dy, w = _rand(g, rows, n, dtype=BF16), _rand(g, n, k, scale=n ** -0.5, dtype=BF16)
    h16 = (2 * _rand(g, rows, k)).to(BF16)
    kept = None
    if src == "ckpt":
        kept = ad.Ckpt.empty(rows, k)
        ad.ckpt_pack(h16.cuda(), kept)
        h = _value_ref(kept.q.cpu().numpy(), kept.scale.cpu().numpy(), k)
    else:
        h = h16.double()
    dx = Out(rows, k, ot, pad, shift)
    act_out = Out(rows, k, BF16, pad, shift) if again else None
    ad.linear_dgrad(_put(dy, pad, shift), _put(w, pad, shift), ad.ACT_NONE if src == "none" else ad.ACT_GELU,
                    _put(h16, pad, shift) if src == "bf16" else None, kept, dx.t, act_out.t if again else None,
                    _space(ad.linear_dgrad_workspace_size(rows, n, k)))
    D, W = dy.double(), w.double()
    want, tol = D @ W, 2 * n * U * (D.abs() @ W.abs())
    if src != "none":
        s = _slope(h)
        # the slope: erf to 2e-7 / 2, phi to a few roundings of |h phi|
        tol = tol * 1.13 + want.abs() * (1e-7 + 16 * U) + 2 * U * (want * s).abs()
        want = want * s
    _near(dx.get(), want, tol * 1.01 + want.abs() * _two(ot), "dx")
    if again:
        _near(act_out.get(), _gelu(h), h.abs() * 1e-7 + _gelu(h).abs() * (8 * U + 2.0 ** -8) + 1e-37, "act_out")


@pytest.mark.parametrize("rows,n,k,pad,shift", SHAPES + [(0, 40, 72, 0, 0), (3000, 64, 48, 0, 0)])
@pytest.mark.parametrize("src", ["bf16", "ckpt", "affine"])
def test_linear_wgrad(rows, n, k, pad, shift, src):
    g = _gen(13 * rows + 31 * n + 977 * k)
    dy, x16 = _rand(g, rows, n, dtype=BF16), _rand(g, rows, k, dtype=BF16)
    kept = gain = shift_v = None
    x, G, S = x16.double(), torch.ones(k, dtype=torch.float64), torch.zeros(k, dtype=torch.float64)
    if src != "bf16":
        kept = ad.Ckpt.empty(rows, k)
        ad.ckpt_pack(x16.cuda(), kept)
        x = _value_ref(kept.q.cpu().numpy(), kept.scale.cpu().numpy(), k)
    if src == "affine":
        pt = BF16 if rows % 2 else F32
        gain, shift_v = (1 + _rand(g, k, scale=0.1)).to(pt), _rand(g, k, dtype=pt)
        G, S = gain.double(), shift_v.double()
    dw, dbias = Out(n, k, F32, pad, shift), torch.full((n,), 9.0, device="cuda")
    ws = _space(ad.linear_wgrad_workspace_size(rows, n, k))
    args = (_put(dy, pad, shift), _put(x16, pad, shift) if kept is None else None, kept,
            None if gain is None else gain.cuda(), None if shift_v is None else shift_v.cuda())
    ad.linear_wgrad(*args, dw.t, dbias, ws)
    one, bias_one = dw.t.clone(), dbias.clone()
    D = dy.double()
    want = D.T @ (x * G + S)
    mag = D.abs().T @ (x.abs() * G.abs() + S.abs())
    _near(one.double().cpu(), want, 2 * (rows + 4) * U * mag, "dw")
    _near(bias_one.double().cpu(), D.sum(0), 2 * (rows + 4) * U * D.abs().sum(0), "dbias")
    dw.t.copy_(one)
    ad.linear_wgrad(*args, dw.t, dbias, ws, accumulate=True)
    assert torch.equal(dbias, bias_one + bias_one)
    again = dw.get()
    assert torch.equal(again, (one + one).double().cpu()), "accumulate"
    ad.linear_wgrad(*args, dw.t, None, ws)                      # without a bias
    assert torch.equal(dw.get(), one.double().cpu()), "the same call gives the same bits"


# Products of several rounds of 128 x 128 tiles, tiles past the last row and column, a reduction that ends
# inside a stage (tests/linear_kernels.py has those of 256 x 256); the references are float64 products
# on the GPU.
LARGE = [(4104, 4200, 200, 0, 0), (4500, 1032, 4104, 8, 8), (1000, 4104, 4360, 0, 0)]


@pytest.mark.parametrize("rows,n,k,pad,shift", LARGE)
@pytest.mark.parametrize("act,rt,yt,keep", [(ad.ACT_GELU, None, BF16, "ckpt"), (ad.ACT_NONE, F32, F32, None),
                                            (ad.ACT_GELU, BF16, F32, "bf16")])
def test_linear_large(rows, n, k, pad, shift, act, rt, yt, keep):
    g = torch.Generator(device="cuda").manual_seed(rows + n + k)
    rnd = lambda *s, scale=1.0, dtype=BF16: (torch.randn(*s, generator=g, device="cuda") * scale).to(dtype)  # noqa: E731
    x, w, bias = rnd(rows, k), rnd(n, k, scale=k ** -0.5), rnd(n)
    res = None if rt is None else rnd(rows, n, dtype=rt)
    y = Out(rows, n, yt, pad, shift)
    pre = Out(rows, n, BF16, pad, shift) if keep == "bf16" else None
    kept = ad.Ckpt.empty(rows, n) if keep == "ckpt" else None
    ad.linear(_put(x, pad, shift), _put(w, pad, shift), bias, act, None if res is None else _put(res, pad, shift), y.t,
              None if pre is None else pre.t, kept, _space(ad.linear_workspace_size(rows, n, k)))
    h = x.double() @ w.double().t().contiguous() + bias.double()
    th = 2 * k * U * (x.double().abs() @ w.double().abs().t().contiguous()) + 2 * U * (h.abs() + bias.double().abs())
    out, tol = (_gelu(h), 1.13 * th + h.abs() * (1e-7 + 8 * U)) if act == ad.ACT_GELU else (h, th)
    if res is not None:
        out = out + res.double()
        tol = tol + 2 * U * (out.abs() + res.double().abs())
    _near(y.get(), out.cpu(), (tol * 1.01 + out.abs() * _two(yt)).cpu(), "y")
    if pre is not None:
        _near(pre.get(), h.cpu(), (th * 1.01 + h.abs() * 2.0 ** -8).cpu(), "pre")
    if kept is not None:
        _check_ckpt(kept, h.cpu(), th.cpu(), "pre")


@pytest.mark.parametrize("rows,n,k,pad,shift", LARGE)
@pytest.mark.parametrize("src,ot,again", [("none", BF16, False), ("bf16", F32, True), ("ckpt", BF16, True)])
def test_linear_dgrad_large(rows, n, k, pad, shift, src, ot, again):
    g = torch.Generator(device="cuda").manual_seed(rows + n + k)
    rnd = lambda *s, scale=1.0, dtype=BF16: (torch.randn(*s, generator=g, device="cuda") * scale).to(dtype)  # noqa: E731
    n, k = k, n                    # the wide side is dx's
    dy, w, h16 = rnd(rows, n), rnd(n, k, scale=n ** -0.5), rnd(rows, k, scale=2.0)
    kept = None
    h = h16.double()
    if src == "ckpt":
        kept, v = ad.Ckpt.empty(rows, k), torch.empty(rows, k, device="cuda")
        ad.ckpt_pack(h16, kept)
        ad.ckpt_unpack(kept, v)    # (exact, tested by itself)
        h = v.double()
    dx = Out(rows, k, ot, pad, shift)
    act_out = Out(rows, k, BF16, pad, shift) if again else None
    ad.linear_dgrad(_put(dy, pad, shift), _put(w, pad, shift), ad.ACT_NONE if src == "none" else ad.ACT_GELU,
                    _put(h16, pad, shift) if src == "bf16" else None, kept, dx.t, act_out.t if again else None,
                    _space(ad.linear_dgrad_workspace_size(rows, n, k)))
    want, tol = dy.double() @ w.double(), 2 * n * U * (dy.double().abs() @ w.double().abs())
    if src != "none":
        s = _slope(h)
        tol = tol * 1.13 + want.abs() * (1e-7 + 16 * U) + 2 * U * (want * s).abs()
        want = want * s
    _near(dx.get(), want.cpu(), (tol * 1.01 + want.abs() * _two(ot)).cpu(), "dx")
    if again:
        _near(act_out.get(), _gelu(h).cpu(), (h.abs() * 1e-7 + _gelu(h).abs() * (8 * U + 2.0 ** -8) + 1e-37).cpu(), "act_out")


@pytest.mark.parametrize("rows,n,k,pad,shift", [(200, 4200, 4104, 0, 0), (4104, 1032, 4360, 8, 8), (9000, 1288, 1544, 0, 0)])
@pytest.mark.parametrize("src", ["bf16", "ckpt", "affine"])
def test_linear_wgrad_large(rows, n, k, pad, shift, src):
    g = torch.Generator(device="cuda").manual_seed(rows + n + k)
    rnd = lambda *s, scale=1.0, dtype=BF16: (torch.randn(*s, generator=g, device="cuda") * scale).to(dtype)  # noqa: E731
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
    ws = _space(ad.linear_wgrad_workspace_size(rows, n, k))
    args = (_put(dy, pad, shift), _put(x16, pad, shift) if kept is None else None, kept, gain, shift_v)
    ad.linear_wgrad(*args, dw.t, dbias, ws)
    d = dy.double().t().contiguous()
    one = dw.t.clone()
    _near(one.double().cpu(), (d @ x).cpu(), (2 * (rows + 4) * U * (d.abs() @ mag.abs())).cpu(), "dw")
    _near(dbias.double().cpu(), d.sum(1).cpu(), (2 * (rows + 4) * U * d.abs().sum(1)).cpu(), "dbias")
    ad.linear_wgrad(*args, dw.t, None, ws, accumulate=True)
    assert torch.equal(dw.get(), (one + one).double().cpu())


def test_rows_past_32_bit_offsets():
    """Rows whose elements lie past 2^31 of their matrix (and 2^32 bytes)."""
    rows, ld, n, k = 40000, 1 << 16, 72, 64
    g = _gen(5)
    big = torch.empty(rows, ld, dtype=BF16, device="cuda")
    x = _rand(g, rows, k, dtype=BF16)
    w = _rand(g, n, k, scale=0.1, dtype=BF16)
    xv = big[:, ld - k:]
    xv.copy_(x)
    y = torch.empty(rows, n, device="cuda")
    ad.linear(xv, w.cuda(), None, ad.ACT_NONE, None, y, None, None, None)
    X, W = x.double(), w.double()
    _near(y.double().cpu(), X @ W.T, 2 * k * U * (X.abs() @ W.abs().T), "linear")
    dw, dy = torch.empty(n, k, device="cuda"), _rand(g, rows, n, dtype=BF16)
    ws = _space(ad.linear_wgrad_workspace_size(rows, n, k))
    ad.linear_wgrad(dy.cuda(), xv, None, None, None, dw, None, ws)
    _near(dw.double().cpu(), dy.double().T @ X, 2 * rows * U * (dy.double().abs().T @ X.abs()), "wgrad")
    ones, zeros = torch.ones(k, device="cuda"), torch.zeros(k, device="cuda")
    out = torch.empty(rows, k, device="cuda")
    ad.layer_norm(xv, ones, zeros, out)
    xh = (X - X.mean(1, keepdim=True)) / torch.sqrt(X.var(1, unbiased=False, keepdim=True) + 1e-5)
    _near(out.double().cpu(), xh, 100 * U * (xh.abs() + 1), "layer_norm")
    kept = ad.Ckpt.empty(rows, k)
    ad.ckpt_pack(xv, kept)
    q, s = _pack_ref(x[-50:].float().numpy())
    np.testing.assert_array_equal(kept.q[-50:].cpu().numpy(), q)


def test_nan_stays_in_its_row():
    """A NaN row of x reaches its own row of y only; residual and y may be the same tensor."""
    g = _gen(4)
    x, w, res = _rand(g, 200, 256, dtype=BF16), _rand(g, 136, 256, dtype=BF16), _rand(g, 200, 136)
    clean = torch.empty(200, 136, device="cuda")
    ws = _space(ad.linear_workspace_size(200, 136, 256))
    ad.linear(x.cuda(), w.cuda(), None, ad.ACT_NONE, res.cuda(), clean, None, None, ws)
    x[17, 3] = float("nan")
    y = res.cuda()
    ad.linear(x.cuda(), w.cuda(), None, ad.ACT_NONE, y, y, None, None, ws)
    rows = torch.isnan(y).any(1).cpu()
    assert rows[17] and int(rows.sum()) == 1 and bool(torch.isnan(y[17]).all())
    keep = torch.arange(200) != 17
    assert torch.equal(y.cpu()[keep], clean.cpu()[keep])


def test_linear_rows_do_not_depend_on_the_weight_past_their_end():
    """Elements between the row's end and ld, and rows past the last one, are not read."""
    g = _gen(6)
    for rows, n, k, pad in ((70, 200, 72, 8), (70, 200, 75, 5)):
        x, w = _rand(g, rows, k, dtype=BF16), _rand(g, n, k, dtype=BF16)
        got = []
        for fill in (0.0, float("nan")):
            xb = torch.full((rows + 3, k + pad), fill, dtype=BF16, device="cuda")
            wb = torch.full((n + 3, k + pad), fill, dtype=BF16, device="cuda")
            xb[:rows, :k], wb[:n, :k] = x.cuda(), w.cuda()
            y = torch.empty(rows, n, device="cuda")
            ad.linear(xb[:rows, :k], wb[:n, :k], None, ad.ACT_NONE, None, y, None, None,
                      _space(ad.linear_workspace_size(rows, n, k)))
            got.append(y)
        assert torch.equal(*got)


# ------------------------------------------------------------------- streams, graphs, a sublayer

def _sublayer(seed, d, f, rows):
    g = _gen(seed)
    params = [(1 + _rand(g, d, scale=0.1)).to(BF16), _rand(g, d, scale=0.1, dtype=BF16),
              _rand(g, f, d, scale=d ** -0.5, dtype=BF16), _rand(g, f, scale=0.1, dtype=BF16),
              _rand(g, d, f, scale=f ** -0.5, dtype=BF16), _rand(g, d, scale=0.1, dtype=BF16)]
    return params, _rand(g, rows, d), _rand(g, rows, d)


@pytest.mark.parametrize("rows,d,f", [(1, 128, 256), (37, 384, 768), (300, 320, 640)])
def test_feed_forward_sublayer(rows, d, f):
    """Forward and backward of the sublayer against float64 autograd of the same function.
    The forward pass rounds LN(x) and GELU to bf16 (2^-8 relative each, averaging out over the
    products: 2 * 2^-8 of the rms bounds the difference in norm).  The backward pass reads xhat and
    the pre-activation from 8 bits, each within amax / 127 / 2 <= 2% of its rms, and rounds
    dout, dpre, act and the LayerNorm's dy to bf16: in norm, 4% of each gradient bounds it."""
    params, x, dout = _sublayer(rows, d, f, rows)
    ff = FeedForward([p.cuda() for p in params], rows + 5)
    X = x.cuda()
    out, dx, copy = torch.empty_like(X), torch.empty_like(X), torch.empty(rows, d, dtype=BF16, device="cuda")
    ff.forward(X, out)
    ff.backward(dout.cuda(), dx, copy)
    ps = [p.double().requires_grad_() for p in params]
    xd = x.double().requires_grad_()
    y = torch.nn.functional.layer_norm(xd, (d,), ps[0], ps[1])
    ref = xd + _gelu(y @ ps[2].T + ps[3]) @ ps[4].T + ps[5]
    ref.backward(dout.double())
    rel = lambda a, b: float((a.double().cpu() - b).norm() / b.norm())  # noqa: E731
    assert rel(out - X, (ref - xd).detach()) < 2 * 2.0 ** -8
    assert rel(dx - dout.cuda(), xd.grad - dout.double()) < 0.04
    assert torch.equal(copy, dx.to(BF16))
    for got, p in zip(ff.grads, ps):
        assert rel(got, p.grad) < 0.04
    once = [t.clone() for t in ff.grads]
    ff.forward(X, out)
    alias = dout.cuda()
    ff.backward(alias, alias)                      # dx over dout, gradients added
    assert torch.equal(alias, dx)
    for a, b in zip(ff.grads, once):
        assert torch.equal(a, b + b)


def test_feed_forward_gradient_against_differences():
    """dx along a direction against a central difference of the forward pass itself, whose output is
    float32 but whose operands are bf16: the step 2^-3 is large against their rounding, the third
    derivative enters with step^2 / 6; 5% of the difference is allowed."""
    rows, d, f = 64, 256, 512
    params, x, dout = _sublayer(11, d, f, rows)
    ff = FeedForward([p.cuda() for p in params], rows)
    v = _rand(_gen(12), rows, d)
    h = 2.0 ** -3
    outs = []
    for s in (h, -h):
        o = torch.empty(rows, d, device="cuda")
        ff.forward((x + s * v).cuda(), o)
        outs.append(o.double().cpu())
    want = float(((outs[0] - outs[1]) / (2 * h) * dout.double()).sum())
    o, dx = torch.empty(rows, d, device="cuda"), torch.empty(rows, d, device="cuda")
    ff.forward(x.cuda(), o)
    ff.backward(dout.cuda(), dx)
    got = float((dx.double().cpu() * v.double()).sum())
    scale = float((((outs[0] - outs[1]) / (2 * h)).norm() * dout.double().norm())) / math.sqrt(rows * d)
    assert abs(got - want) < 0.05 * max(abs(want), scale)


def test_feed_forward_in_place_any_number_of_rows_and_refusals():
    """out may be x; passes of every size share the buffers and the workspace, which stays where it is."""
    d, f, most = 128, 320, 700
    params, x, dout = _sublayer(31, d, f, most)
    dev = [p.cuda() for p in params]
    ff = FeedForward(dev, most)
    space = ff.workspace.data_ptr()
    for rows in (700, 1, 0, 65, 129, 512):
        X, D = x[:rows].cuda(), dout[:rows].cuda()
        alone = FeedForward(dev, max(rows, 1))
        want, dwant = torch.empty_like(X), torch.empty_like(X)
        alone.forward(X, want)
        alone.backward(D, dwant)
        ff.zero_grads()
        got, dgot = X.clone(), torch.empty_like(X)
        ff.forward(got, got)
        ff.backward(D, dgot)
        assert torch.equal(got, want) and torch.equal(dgot, dwant)
        assert all(torch.equal(a, b) for a, b in zip(ff.grads, alone.grads))
    assert ff.workspace.data_ptr() == space
    with pytest.raises(ValueError, match="rows"):
        ff.forward(torch.zeros(701, d, device="cuda"), torch.zeros(701, d, device="cuda"))
    with pytest.raises(ValueError, match="last forward"):
        ff.backward(torch.zeros(3, d, device="cuda"), torch.zeros(3, d, device="cuda"))


def test_two_streams_at_once():
    """Passes of two objects on two streams, each with its own workspace, at the same time."""
    shapes = ((300, 256, 512), (170, 128, 384))
    made = [(_sublayer(s[0], s[1], s[2], s[0]), s) for s in shapes]
    objs, ins, outs, want = [], [], [], []
    for (params, x, dout), s in made:
        ff = FeedForward([p.cuda() for p in params], s[0])
        X, D = x.cuda(), dout.cuda()
        o, g = torch.empty_like(X), torch.empty_like(X)
        ff.forward(X, o)
        ff.backward(D, g)
        objs.append(ff)
        ins.append((X, D))
        outs.append((o, g))
        want.append([t.clone() for t in (o, g, *ff.grads)])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in objs]
    for _ in range(5):
        for ff, (X, D), (o, g), st in zip(objs, ins, outs, streams):
            with torch.cuda.stream(st):
                ff.zero_grads()
                ff.forward(X, o)
                ff.backward(D, g)
    torch.cuda.synchronize()
    for ff, (o, g), w in zip(objs, outs, want):
        assert all(torch.equal(a, b) for a, b in zip((o, g, *ff.grads), w))


def test_binding_refuses_what_the_tensors_show():
    x, w = torch.zeros(8, 64, dtype=BF16, device="cuda"), torch.zeros(32, 64, dtype=BF16, device="cuda")
    y = torch.zeros(8, 32, device="cuda")
    ok = lambda **o: ad.linear(o.get("x", x), o.get("w", w), o.get("bias"), 0, o.get("res"), o.get("y", y), None,  # noqa: E731
                               o.get("keep"), _space(ad.linear_workspace_size(8, 32, 64)))
    ok()
    for bad in (dict(w=w[:, :32]), dict(y=y[:4]), dict(res=torch.zeros(8, 31, device="cuda")), dict(y=y.t()[:8]),
                dict(y=torch.zeros(32, 8, device="cuda").t()), dict(y=y.half()), dict(bias=torch.zeros(31, device="cuda")),
                dict(bias=torch.zeros(64, device="cuda")[::2]), dict(keep=ad.Ckpt.empty(8, 33)), dict(w=w.cpu())):
        with pytest.raises(ValueError):
            ok(**bad)
    with pytest.raises(ad.ADError, match="AD_EUNSUPPORTED"):
        ok(x=x.float())
    with pytest.raises(ad.ADError, match="AD_EINVAL"):
        ok(x=x[:1].expand(8, 64))                       # every row the same memory: ld 0
    with pytest.raises(ad.ADError, match="AD_ENOSPACE|AD_EINVAL"):
        ad.linear_wgrad(torch.zeros(4096, 128, dtype=BF16, device="cuda"), torch.zeros(4096, 64, dtype=BF16, device="cuda"),
                        None, None, None, torch.zeros(128, 64, device="cuda"), None, None)
    with pytest.raises(ValueError, match="same dtype"):
        ad.layer_norm(y, torch.ones(32, device="cuda"), torch.ones(32, dtype=BF16, device="cuda"), y)
    k = ad.Ckpt.empty(8, 64)
    with pytest.raises(ad.ADError, match="AD_EINVAL"):
        ad.ckpt_unpack(k, torch.zeros(8, 64, device="cuda"), act=7)


def test_checkpoint_of_nan_and_infinity_through_the_products():
    """A group of the pre-activation that holds a NaN or an infinity reads as NaN, and only it does."""
    g = _gen(17)
    rows, n, k = 40, 256, 64
    x, w = _rand(g, rows, k, dtype=BF16), _rand(g, n, k, dtype=BF16)
    w[70, 5] = float("inf")
    bias = torch.zeros(n, dtype=BF16)
    bias[200] = float("nan")
    y, kept, v = torch.empty(rows, n, device="cuda"), ad.Ckpt.empty(rows, n), torch.empty(rows, n, device="cuda")
    ad.linear(x.cuda(), w.cuda(), bias.cuda(), ad.ACT_NONE, None, y, None, kept, _space(ad.linear_workspace_size(rows, n, k)))
    ad.ckpt_unpack(kept, v)
    bad = torch.isnan(v).all(0).cpu()
    want = torch.zeros(n, dtype=torch.bool)
    want[64:96] = want[192:224] = True
    assert torch.equal(bad, want) and torch.equal(torch.isnan(v).any(0).cpu(), want)
    assert bool(torch.isnan(y[:, 200]).all()) and not bool(torch.isfinite(y[:, 70]).any())
    dx = torch.empty(rows, n, device="cuda")
    dy, w2 = _rand(g, rows, k, dtype=BF16), _rand(g, k, n, dtype=BF16)
    ad.linear_dgrad(dy.cuda(), w2.cuda(), ad.ACT_GELU, None, kept, dx, None, _space(ad.linear_dgrad_workspace_size(rows, k, n)))
    assert torch.equal(torch.isnan(dx).any(0).cpu(), want)
    dw = torch.empty(k, n, device="cuda")
    ad.linear_wgrad(dy.cuda(), None, kept, None, None, dw, None, _space(ad.linear_wgrad_workspace_size(rows, k, n)))
    assert torch.equal(torch.isnan(dw).any(0).cpu(), want)


@pytest.mark.parametrize("k", [64, 61])
def test_gelu_of_infinities_and_large_values(k):
    """GELU is 0 at -infinity, its slope 0 there and 1 at infinity; neither is NaN for any number."""
    h = torch.tensor([float("inf"), -float("inf"), 3e38, -3e38, 1e20, -1e20, 50.0, -50.0], dtype=BF16)
    pre = h.repeat(3, 8)[:, :k].contiguous()
    up = (pre > 0).double()
    dy = torch.ones(3, 16, dtype=BF16)
    w = torch.full((16, k), 0.125, dtype=BF16)
    dx, again = torch.empty(3, k, device="cuda"), torch.empty(3, k, dtype=BF16, device="cuda")
    ad.linear_dgrad(dy.cuda(), w.cuda(), ad.ACT_GELU, pre.cuda(), None, dx, again, _space(ad.linear_dgrad_workspace_size(3, 16, k)))
    assert torch.equal(dx.double().cpu(), 2 * up)
    want = torch.where(pre > 0, pre, torch.zeros_like(pre))
    assert torch.equal(again.cpu().float().abs(), want.float())
    # the forward product: zeros times a weight, and the values as its bias
    y = torch.empty(3, k, dtype=BF16, device="cuda")
    ad.linear(torch.zeros(3, 16, dtype=BF16, device="cuda"), w.t().contiguous().cuda(), pre[0].cuda(), ad.ACT_GELU, None, y, None,
              None, _space(ad.linear_workspace_size(3, k, 16)))
    assert torch.equal(y.cpu().float().abs(), want.float())


def test_other_stream_and_graph_replays():
    rows, d, f = 130, 256, 512
    params, x, dout = _sublayer(21, d, f, rows)
    dev = [p.cuda() for p in params]

    def run(ff, X, D, out, dx):
        ff.forward(X, out)
        ff.backward(D, dx)

    ff = FeedForward(dev, rows)
    X, D = x.cuda(), dout.cuda()
    out, dx = torch.empty_like(X), torch.empty_like(X)
    run(ff, X, D, out, dx)
    want = [t.clone() for t in (out, dx, *ff.grads)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ff.zero_grads()
        out.fill_(GUARD)
        run(ff, X, D, out, dx)
    side.synchronize()
    for a, b in zip((out, dx, *ff.grads), want):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        ff.zero_grads()
        run(ff, X, D, out, dx)
    other = torch.randn(1 << 20, device="cuda")
    for rep in range(4):
        out.fill_(GUARD)
        dx.fill_(GUARD)
        ff.workspace.fill_(255)
        other.mul_(1.001).add_(rep)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((out, dx, *ff.grads), want):
            assert torch.equal(a, b), rep
    # new inputs through the same graph
    X.copy_(x * 0.5)
    graph.replay()
    torch.cuda.synchronize()
    fresh = FeedForward(dev, rows)
    o2, d2 = torch.empty_like(X), torch.empty_like(X)
    run(fresh, X, D, o2, d2)
    for a, b in zip((out, dx, *ff.grads), (o2, d2, *fresh.grads)):
        assert torch.equal(a, b)
