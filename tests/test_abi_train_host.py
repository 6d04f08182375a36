"""The training operators' argument checks (CPU only: every call is refused before anything is
enqueued), and their workspace sizes."""
import ctypes

import pytest

EINVAL, ERANGE, ENOSPACE, EUNSUPPORTED = -1, -2, -3, -5
P = 0x100000            # an address that is never dereferenced


@pytest.fixture(scope="module")
def ad():
    from paper_2608_12703_amd import ad as mod
    return mod


def _mat(ad, ld, dtype=None, data=P):
    return ctypes.byref(ad.Mat(data, ld, ad.AD_BF16 if dtype is None else dtype))


def _ck(ad, q=P, scale=P):
    return ctypes.byref(ad.CkptView(q, scale))


def test_ckpt_ld(ad):
    assert [ad.LIB.ad_ckpt_ld(c) for c in (1, 128, 129, 1280, 5120)] == [128, 128, 256, 1280, 5120]
    assert ad.LIB.ad_ckpt_ld(0) == 0 and ad.LIB.ad_ckpt_ld((1 << 20) + 1) == 0


def test_ckpt_refusals(ad):
    pack = lambda rows=4, cols=100, x=None, k=None: ad.LIB.ad_ckpt_pack(  # noqa: E731
        rows, cols, _mat(ad, 100) if x is None else x, _ck(ad) if k is None else k, None)
    assert pack(rows=-1) == ERANGE and pack(rows=(1 << 24) + 1) == ERANGE
    assert pack(cols=0) == ERANGE and pack(cols=(1 << 20) + 1) == ERANGE
    assert pack(x=_mat(ad, 99)) == EINVAL                       # rows overlap
    assert pack(x=_mat(ad, (1 << 22) + 1)) == ERANGE
    assert pack(x=_mat(ad, 100, data=None)) == EINVAL
    assert pack(x=_mat(ad, 100, dtype=9)) == EINVAL
    assert pack(x=_mat(ad, 100, data=P + 1)) == EINVAL          # not aligned to its element
    assert pack(x=_mat(ad, 100, dtype=ad.AD_F32, data=P + 2)) == EINVAL
    assert pack(k=_ck(ad, q=None)) == EINVAL and pack(k=_ck(ad, scale=None)) == EINVAL
    assert pack(k=_ck(ad, q=P + 8)) == EINVAL and pack(k=_ck(ad, scale=P + 2)) == EINVAL
    assert b"ckpt" in ad.LIB.ad_last_error()
    assert pack(rows=1 << 24, cols=1 << 20, x=_mat(ad, 1 << 20)) == ERANGE
    assert ad.LIB.ad_ckpt_pack(4, 100, None, _ck(ad), None) == EINVAL
    assert ad.LIB.ad_ckpt_pack(4, 100, _mat(ad, 100), None, None) == EINVAL
    assert ad.LIB.ad_ckpt_unpack(4, 100, _ck(ad), 5, _mat(ad, 100), None) == EINVAL
    assert ad.LIB.ad_ckpt_unpack(4, 100, _ck(ad), 0, None, None) == EINVAL


def test_layer_norm_refusals(ad):
    def run(rows=4, cols=256, x="m", gain=P, bias=P, dt=1, y="m", mean=None, k=None):
        m = lambda v: _mat(ad, 8192) if v == "m" else v  # noqa: E731
        return ad.LIB.ad_layer_norm(rows, cols, m(x), gain, bias, dt, m(y), mean, None, k, None)

    assert run(x=None) == EINVAL and run(y=None) == EINVAL and run(gain=None) == EINVAL and run(bias=None) == EINVAL
    assert run(dt=2) == EINVAL and run(dt=0, gain=P + 2) == EINVAL and run(mean=P + 1) == EINVAL
    assert run(cols=8193, x=_mat(ad, 8193), y=_mat(ad, 8193)) == EUNSUPPORTED
    assert run(k=_ck(ad, q=P + 4)) == EINVAL
    n = ctypes.c_size_t()
    assert ad.LIB.ad_layer_norm_backward_workspace_size(100, 320, None) == EINVAL
    assert ad.LIB.ad_layer_norm_backward_workspace_size(-1, 320, ctypes.byref(n)) == ERANGE
    assert ad.LIB.ad_layer_norm_backward_workspace_size(4, 8193, ctypes.byref(n)) == EUNSUPPORTED
    assert ad.LIB.ad_layer_norm_backward_workspace_size(0, 320, ctypes.byref(n)) == 0 and n.value == 0
    assert ad.LIB.ad_layer_norm_backward_workspace_size(100, 320, ctypes.byref(n)) == 0 and n.value > 0
    need = n.value

    def back(dy="m", x=None, mean=None, rstd=P, k="k", gain=P, dt=1, dres=None, dx="m", copy=None, dg=P, db=P, ws=P,
             size=need, rows=100):
        m = lambda v: _mat(ad, 320) if v == "m" else v  # noqa: E731
        return ad.LIB.ad_layer_norm_backward(rows, 320, m(dy), m(x), mean, rstd, _ck(ad) if k == "k" else k, gain, dt,
                                             m(dres), m(dx), copy, dg, db, 0, ws, size, None)

    assert back(dy=None) == EINVAL and back(dx=None) == EINVAL and back(rstd=None) == EINVAL
    assert back(x="m", mean=P) == EINVAL                        # x and the checkpoint
    assert back(k=None) == EINVAL                               # neither
    assert back(k=None, x="m") == EINVAL                        # x without mean
    assert back(dg=None) == EINVAL and back(db=None) == EINVAL  # one of the pair
    assert back(copy=_mat(ad, 320, dtype=ad.AD_F32)) == EUNSUPPORTED
    assert back(dres=_mat(ad, 319)) == EINVAL
    assert back(size=need - 1) == ENOSPACE and b"workspace" in ad.LIB.ad_last_error()
    assert back(ws=None) == EINVAL and back(ws=P + 16) == EINVAL
    assert back(rows=-3) == ERANGE


def test_linear_refusals(ad):
    n = ctypes.c_size_t()
    for name in ("ad_linear_workspace_size", "ad_linear_dgrad_workspace_size", "ad_linear_wgrad_workspace_size"):
        f = getattr(ad.LIB, name)
        assert f(4, 8, 8, None) == EINVAL and f(-1, 8, 8, ctypes.byref(n)) == ERANGE
        assert f(4, 0, 8, ctypes.byref(n)) == ERANGE and f(4, 8, 1 << 21, ctypes.byref(n)) == ERANGE
        assert f(0, 8, 8, ctypes.byref(n)) == 0 and n.value == 0
    assert ad.LIB.ad_linear_dgrad_workspace_size(64, 2560, 1280, ctypes.byref(n)) == 0 and n.value > 0
    need = n.value
    f32 = _mat(ad, 4096, dtype=ad.AD_F32)
    m = lambda v: _mat(ad, 4096) if v == "m" else v  # noqa: E731

    def fwd(x="m", w="m", bias=P, bt=1, act=0, res=None, y="m", pre=None, k=None, rows=4, ws=P, size=1 << 40):
        return ad.LIB.ad_linear(rows, 1280, 2560, m(x), m(w), bias, bt, act, m(res), m(y), m(pre), k, ws, size, None)

    assert fwd(x=None) == EINVAL and fwd(w=None) == EINVAL and fwd(y=None) == EINVAL
    assert fwd(x=f32) == EUNSUPPORTED and fwd(w=f32) == EUNSUPPORTED and fwd(pre=f32) == EUNSUPPORTED
    assert fwd(bt=3) == EINVAL and fwd(act=2) == EINVAL and fwd(pre="m", k=_ck(ad)) == EINVAL
    assert fwd(x=_mat(ad, 2559)) == EINVAL and fwd(w=_mat(ad, 2559)) == EINVAL and fwd(y=_mat(ad, 1279)) == EINVAL
    assert fwd(res=_mat(ad, 1279)) == EINVAL and fwd(ws=P + 8) == EINVAL

    def dgrad(dy="m", w="m", act=1, pre="m", k=None, dx="m", again=None, size=1 << 40, ws=P):
        return ad.LIB.ad_linear_dgrad(64, 2560, 1280, m(dy), m(w), act, m(pre), k, m(dx), m(again), ws, size, None)

    assert dgrad(dy=f32) == EUNSUPPORTED and dgrad(w=f32) == EUNSUPPORTED and dgrad(pre=f32) == EUNSUPPORTED
    assert dgrad(pre=None) == EINVAL and dgrad(k=_ck(ad)) == EINVAL
    assert dgrad(act=0) == EINVAL and dgrad(act=0, pre=None, again="m") == EINVAL and dgrad(act=7) == EINVAL
    assert dgrad(size=need - 1) == ENOSPACE and dgrad(ws=None) == EINVAL

    def wgrad(dy="m", x="m", k=None, gain=None, shift=None, dt=1, dw=f32, db=P, size=1 << 40):
        return ad.LIB.ad_linear_wgrad(64, 2560, 1280, m(dy), m(x), k, gain, shift, dt, m(dw), db, 0, P, size, None)

    assert wgrad(dy=f32) == EUNSUPPORTED and wgrad(x=f32) == EUNSUPPORTED and wgrad(dw="m") == EUNSUPPORTED
    assert wgrad(x=None) == EINVAL and wgrad(k=_ck(ad)) == EINVAL
    assert wgrad(gain=P, shift=P) == EINVAL                     # an affine input needs the checkpoint
    assert wgrad(x=None, k=_ck(ad), gain=P) == EINVAL
    assert wgrad(x=None, k=_ck(ad), gain=P, shift=P, dt=4) == EINVAL
    assert wgrad(db=P + 2) == EINVAL and wgrad(dw=None) == EINVAL


def test_binding_refusals(ad):
    import torch
    x = torch.zeros(4, 64)
    with pytest.raises(ValueError, match="not on the current GPU"):
        ad.layer_norm(x, x[0], x[0], x)
    with pytest.raises(ValueError, match="checkpoint"):
        ad.Ckpt(torch.zeros(4, 64, dtype=torch.int8), torch.zeros(4, 4, dtype=torch.uint8), 64)
    k = ad.Ckpt.empty(4, 64, device="cpu")
    assert tuple(k.q.shape) == (4, 128) and tuple(k.scale.shape) == (4, 4)
    with pytest.raises(ValueError, match="not on the current GPU"):
        ad.ckpt_pack(x, k)
