"""8-bit checkpoints of values up to the end of float32's range, through everything that reads them.

A value is q 2^(s - 127); float32 and bf16 hold it exactly up to q 2^(s - 127) = 2^128, which reads as
an infinity (a group whose largest magnitude is within half a step, 2^121, of 2^128 has such a
value).  The other values of that group, zeros among them, are ordinary numbers."""
import numpy as np
import pytest
import torch

from paper_2608_12703_amd import ad
from test_gpu_train_ops import BF16, F32, U, Out, _gen, _gelu, _ln_bwd_ref, _near, _pack_ref, _put, _rand, _space, _two, _value_ref

pytestmark = pytest.mark.gpu

F32_MAX, BF16_MAX = float(np.finfo(np.float32).max), float(torch.finfo(BF16).max)
# the largest magnitudes: below and above 127 * 2^120, where the scale byte passes 247
FINITE = [1.6e38, 127.0 * 2.0 ** 120, 1.7e38, 3e38]
TOPS = [s * v for v in FINITE + [BF16_MAX, F32_MAX] for s in (1, -1)]


def _groups(cols, tops, rows=None):
    """Row i: one group with tops[i] in it, beside zeros, ordinary and halved values of both signs."""
    rows = len(tops) if rows is None else rows
    v = np.random.default_rng(cols).standard_normal((rows, cols)).astype(np.float32)
    for i, top in enumerate(tops):
        at = 32 * (i % (cols // 32))
        v[i, at:at + 32] = 0.0
        v[i, at + 3] = top
        v[i, at + 8:at + 16] = np.float32(top) * np.float32([0.5, -0.5, 0.25, -0.25, 0.01, -0.01, 0.004, 0.003])
        v[i, at + 20:at + 22] = [1.0, -1.0]
    return torch.from_numpy(v)


def _packed(x):
    k = ad.Ckpt.empty(*x.shape)
    ad.ckpt_pack(x.cuda(), k)
    return k, _value_ref(k.q.cpu().numpy(), k.scale.cpu().numpy(), x.shape[1])


def _single(v):
    return v.float().double()       # 2^128 becomes an infinity


@pytest.mark.parametrize("cols", [200, 256, 1280])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_pack_and_unpack(cols, dtype):
    x = _groups(cols, TOPS).clamp(-float(torch.finfo(dtype).max), float(torch.finfo(dtype).max)).to(dtype)
    q, s = _pack_ref(x.float().numpy())
    k, want = _packed(x)
    np.testing.assert_array_equal(k.scale.cpu().numpy(), s)
    np.testing.assert_array_equal(k.q.cpu().numpy(), q)
    want = _single(want)
    assert int(torch.isinf(want).sum()) == int((x.float().abs() >= 127.5 * 2.0 ** 121).sum()) > 0
    for out_dtype in (F32, BF16):
        out, gelu = Out(len(TOPS), cols, out_dtype), Out(len(TOPS), cols, out_dtype)
        ad.ckpt_unpack(k, out.t)
        np.testing.assert_array_equal(out.get().numpy(), want.numpy())
        ad.ckpt_unpack(k, gelu.t, act=ad.ACT_GELU)
        got, big = gelu.get(), want.abs() > 1e30
        assert torch.equal(got[big].abs(), want[big].clamp(min=0))
        g = _gelu(want)
        _near(got[~big], g[~big], want[~big].abs() * 1e-7 + g[~big].abs() * (8 * U + _two(out_dtype)) + 1e-37, "gelu")


@pytest.mark.parametrize("k", [256, 251])       # whole vectors, and a width that has none
def test_slope_of_the_input_gradient(k):
    """Slope 1 at large positive values, 0 at large negative ones, 1/2 at the zeros beside them: off by
    erf's 1e-7 and a few roundings (the product itself, 16 / 8 = 2, is exact)."""
    rows = len(TOPS)
    kept, v = _packed(_groups(k, TOPS))
    v = _single(v)
    dy, w = torch.ones(rows, 16, dtype=BF16), torch.full((16, k), 0.125, dtype=BF16)
    dx, again = torch.empty(rows, k, device="cuda"), torch.empty(rows, k, dtype=BF16, device="cuda")
    ad.linear_dgrad(dy.cuda(), w.cuda(), ad.ACT_GELU, None, kept, dx, again, _space(ad.linear_dgrad_workspace_size(rows, 16, k)))
    c = v.clamp(-40.0, 40.0)                      # (the same slope in float64)
    slope = 0.5 * (1 + torch.erf(c * 0.5 ** 0.5)) + c * torch.exp(-0.5 * c * c) / (2 * np.pi) ** 0.5
    _near(dx.double().cpu(), 2 * slope, torch.full_like(v, 2 * (1e-7 + 20 * U)), "dx")
    big = v.abs() > 1e30
    assert torch.equal(again.double().cpu()[big].abs(), v[big].clamp(min=0))
    assert bool(torch.isfinite(again.double().cpu()[~big]).all())


@pytest.mark.parametrize("n,k,pad", [(64, 256, 0), (136, 200, 0), (37, 256, 1), (61, 201, 3)])
@pytest.mark.parametrize("affine", [False, True])
def test_weight_gradient(n, k, pad, affine):
    """Columns without an infinity against float64; gradients of 2^-100 keep the sums in range."""
    rows = len(TOPS)
    g = _gen(n + k)
    kept, x = _packed(_groups(k, TOPS))
    x = _single(x)
    dy = _rand(g, rows, n, scale=2.0 ** -100, dtype=BF16)
    gain, shift = (1 + _rand(g, k, scale=0.1), _rand(g, k)) if affine else (None, None)
    dw, dbias = Out(n, k, F32, pad), torch.empty(n, device="cuda")
    ad.linear_wgrad(_put(dy, pad), None, kept, None if gain is None else gain.cuda(), None if shift is None else shift.cuda(),
                    dw.t, dbias, _space(ad.linear_wgrad_workspace_size(rows, n, k)))
    D, ok = dy.double(), torch.isfinite(x).all(0)
    assert 0 < int((~ok).sum()) < 8
    G, S = (gain.double(), shift.double()) if affine else (torch.ones(k).double(), torch.zeros(k).double())
    x, G, S = x[:, ok], G[ok], S[ok]
    _near(dw.get()[:, ok], D.T @ (x * G + S), 2 * (rows + 4) * U * (D.abs().T @ (x.abs() * G.abs() + S.abs())), "dw")
    _near(dbias.double().cpu(), D.sum(0), 2 * (rows + 4) * U * D.abs().sum(0), "dbias")


@pytest.mark.parametrize("cols", [1280, 1283, 2600])
def test_layer_norm_backward(cols):
    """One large normalised value a row; gradients of 2^-120 keep every sum and product in range."""
    tops = [s * v for v in FINITE for s in (1, -1)]
    rows = len(tops)
    g = _gen(cols)
    x = _rand(g, rows, cols)
    for i, top in enumerate(tops):
        x[i, 64 + 32 * i:96 + 32 * i] = 0.0
        x[i, 70 + 32 * i] = top
    k, xh = _packed(x)
    dy, gain = _rand(g, rows, cols, scale=2.0 ** -120), 1 + _rand(g, cols, scale=0.1)
    r = torch.full((rows, 1), 2.0 ** -10, dtype=torch.float64)
    dx = Out(rows, cols, F32)
    dgain, dbias = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    ws = _space(ad.layer_norm_backward_workspace_size(rows, cols))
    ad.layer_norm_backward(dy.cuda(), None, None, r[:, 0].float().cuda(), k, gain.cuda(), None, dx.t, None, dgain, dbias, ws)
    D = dy.double()
    want, tol = _ln_bwd_ref(D, xh, r, gain.double(), None)
    assert float((want / r).abs().max()) < 1e38
    _near(dx.get(), want, tol, "dx")
    n = rows + 40
    _near(dgain.double().cpu(), (D * xh).sum(0), n * U * (D * xh).abs().sum(0), "dgain")
    _near(dbias.double().cpu(), D.sum(0), n * U * D.abs().sum(0), "dbias")
