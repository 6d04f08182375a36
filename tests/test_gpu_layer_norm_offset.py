"""LayerNorm of rows whose mean is far larger than their spread, and of rows of one value.

Tolerances.  u = 2^-24; row sums are trees that 48 u of the magnitudes' sum bounds.  The mean from one
sum is off by e0 <= 48 u mean |x|.  Its deviations x - m are off by u of themselves, their mean, taken
again, by e1 = 48 u (mean |x - mu| + e0); what is taken from the rows in the end is off by that and 3 u
of itself.  The variance is a difference of two means of squares of at most var + e0^2, off by
110 u of that, relative to var + eps."""
import pytest
import torch

from paper_2608_12703_amd import ad
from test_gpu_train_ops import BF16, F32, U, Out, _check_ckpt, _gen, _near, _put, _rand, _two

pytestmark = pytest.mark.gpu

COLS = [7, 33, 384, 511, 768, 1000, 1280, 2048, 2600, 5000, 8192]


def _check(x, yt, keep, pad=0, shift=0):
    rows, cols = x.shape
    g = _gen(cols)
    gain, bias = 1 + _rand(g, cols, scale=0.1), _rand(g, cols, scale=0.1)
    y = Out(rows, cols, yt, pad, shift)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    k = ad.Ckpt.empty(rows, cols) if keep else None
    ad.layer_norm(_put(x, pad, shift), gain.cuda(), bias.cuda(), y.t, mean, rstd, k)
    X, G, B = x.double(), gain.double(), bias.double()
    mu = X.mean(1, keepdim=True)
    d = X - mu
    var = d.square().mean(1, keepdim=True)
    r = 1 / torch.sqrt(var + 1e-5)
    e0 = 48 * U * X.abs().mean(1, keepdim=True)
    e1 = 48 * U * (d.abs().mean(1, keepdim=True) + e0)
    drel = 55 * U * (var + e0.square()) / (var + 1e-5) + 4 * U
    tol = r * (e1 + 3 * U * d.abs()) + (d * r).abs() * (drel + 2 * U)
    _near(mean.double().cpu()[:, None], mu, e1 + 2 * U * mu.abs(), "mean")
    _near(rstd.double().cpu()[:, None], r, r * drel, "rstd")
    out = d * r * G + B
    _near(y.get(), out, (tol * G.abs() + 3 * U * ((d * r * G).abs() + B.abs())) * (1 + _two(yt)) + out.abs() * _two(yt), "y")
    if keep:
        _check_ckpt(k, d * r, tol, "xhat")


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("dtype,yt,keep,pad,shift", [(F32, F32, False, 0, 0), (F32, BF16, True, 0, 0), (BF16, F32, True, 3, 1)])
def test_rows_of_one_value(cols, dtype, yt, keep, pad, shift):
    v = torch.tensor([0.1, -10.1, 1000.1, -100000.1, 3e6, 3.0, 0.0]).to(dtype)
    _check(v[:, None].repeat(1, cols), yt, keep, pad, shift)


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("yt,keep,pad,shift", [(F32, True, 0, 0), (F32, False, 3, 1)])
def test_means_far_larger_than_the_spread(cols, yt, keep, pad, shift):
    g = _gen(cols + 1)
    x = _rand(g, 8, cols)
    x *= torch.tensor([1.0, 1.0, 0.01, 1.0, 0.1, 30.0, 1e-3, 0.0])[:, None]
    x += torch.tensor([1e4, -1e4, 1e3, 100.0, -1e5, 1e6, 5.0, 7.1])[:, None]
    _check(x, yt, keep, pad, shift)


def test_a_nan_or_an_infinity_keeps_its_row_only():
    x = torch.full((5, 300), 1000.1)
    x[1, 7], x[2, 299], x[3, 0] = float("nan"), float("inf"), -float("inf")
    y, k = torch.empty(5, 300, device="cuda"), ad.Ckpt.empty(5, 300)
    mean, rstd = torch.empty(5, device="cuda"), torch.empty(5, device="cuda")
    ad.layer_norm(x.cuda(), torch.ones(300, device="cuda"), torch.zeros(300, device="cuda"), y, mean, rstd, k)
    bad = torch.tensor([False, True, True, True, False])
    assert torch.equal(torch.isnan(y).all(1).cpu(), bad) and torch.equal(torch.isnan(y).any(1).cpu(), bad)
    assert torch.equal(torch.isnan(rstd).cpu(), bad) and torch.equal(torch.isfinite(mean).cpu(), ~bad)
    assert not y[0].any() and not y[4].any()
    assert not k.q[:, 300:].any() and bool((k.scale[:, 10:] == 1).all())
