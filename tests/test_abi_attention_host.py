"""Argument checks of attention and the optimizer (CPU only: every call is refused before anything is enqueued),
and their workspace sizes."""
import ctypes
import math

import pytest

EINVAL, ERANGE, ENOSPACE, EUNSUPPORTED = -1, -2, -3, -5
P = 0x100000            # an address that is never dereferenced


@pytest.fixture(scope="module")
def ad():
    from paper_2608_12703_amd import ad as mod
    return mod


def _attn(ad, **kw):
    a = dict(batch=2, q_heads=4, kv_heads=2, q_rows=100, k_rows=300, q_max=60, k_max=200, causal=0, cu_q=P, cu_k=P,
             q_len=None, k_len=None, window=None, err_flag=P)
    a.update(kw)
    return ctypes.byref(ad.AttnView(*a.values()))


def _mat(ad, ld, dtype=None, data=P):
    return ctypes.byref(ad.Mat(data, ld, ad.AD_BF16 if dtype is None else dtype))


BAD = [(dict(batch=-1), ERANGE), (dict(batch=65536), ERANGE), (dict(q_heads=0), ERANGE), (dict(kv_heads=0), ERANGE),
       (dict(q_heads=(1 << 14) + 1), ERANGE), (dict(kv_heads=3), EINVAL), (dict(kv_heads=8), EINVAL),
       (dict(q_rows=-1), ERANGE), (dict(k_rows=(1 << 24) + 1), ERANGE), (dict(q_max=-1), ERANGE),
       (dict(k_max=(1 << 24) + 1), ERANGE), (dict(batch=131071, q_heads=4), ERANGE), (dict(batch=60000, q_heads=10), ERANGE)]


@pytest.mark.parametrize("change,status", BAD)
def test_attention_sizes(ad, change, status):
    n = ctypes.c_size_t()
    for f in (ad.LIB.ad_attention_workspace_size, ad.LIB.ad_attention_backward_workspace_size):
        assert f(_attn(ad, **change), ctypes.byref(n)) == status
        assert f(_attn(ad), None) == EINVAL and f(None, ctypes.byref(n)) == EINVAL
        assert f(_attn(ad), ctypes.byref(n)) == 0 and n.value % 256 == 0
        assert f(_attn(ad, batch=0, q_rows=0, q_max=0), ctypes.byref(n)) == 0


def test_attention_refusals(ad):
    m = lambda v: _mat(ad, 256) if v == "m" else v  # noqa: E731
    f32 = _mat(ad, 256, dtype=ad.AD_F32)

    def fwd(a=None, q="m", k="m", v="m", o="m", rest=None, lse=P, ws=P, size=1 << 40):
        return ad.LIB.ad_attention(_attn(ad) if a is None else a, m(q), m(k), m(v), m(o), m(rest), lse, ws, size, None)

    for change, status in BAD:
        assert fwd(a=_attn(ad, **change)) == status
    for name in ("cu_q", "cu_k", "err_flag"):
        assert fwd(a=_attn(ad, **{name: None})) == EINVAL
    for name in ("cu_q", "cu_k", "err_flag", "q_len", "k_len", "window"):
        assert fwd(a=_attn(ad, **{name: P + 2})) == EINVAL
    for name in ("q", "k", "v", "o"):
        assert fwd(**{name: None}) == EINVAL and fwd(**{name: f32}) == EUNSUPPORTED
        assert fwd(**{name: _mat(ad, 127)}) == EINVAL and fwd(**{name: _mat(ad, (1 << 22) + 1)}) == ERANGE
        assert fwd(**{name: _mat(ad, 256, data=P + 1)}) == EINVAL and fwd(**{name: _mat(ad, 256, data=None)}) == EINVAL
    assert fwd(rest=f32) == EUNSUPPORTED and fwd(lse=P + 2) == EINVAL and fwd(ws=P + 8) == EINVAL
    n = ctypes.c_size_t()
    assert ad.LIB.ad_attention_backward_workspace_size(_attn(ad), ctypes.byref(n)) == 0 and n.value > 0

    def bwd(a=None, q="m", k="m", v="m", o="m", rest=None, lse=P, dout="m", res=None, dq="m", dk="m", dv="m", ws=P,
            size=1 << 40):
        return ad.LIB.ad_attention_backward(_attn(ad) if a is None else a, m(q), m(k), m(v), m(o), m(rest), lse, m(dout),
                                            m(res), m(dq), m(dk), m(dv), ws, size, None)

    for change, status in BAD:
        assert bwd(a=_attn(ad, **change)) == status
    for name in ("q", "k", "v", "o", "dout", "dq", "dk", "dv"):
        assert bwd(**{name: None}) == EINVAL and bwd(**{name: f32}) == EUNSUPPORTED
        assert bwd(**{name: _mat(ad, 127)}) == EINVAL
    assert bwd(rest=f32) == EUNSUPPORTED and bwd(lse=None) == EINVAL and bwd(lse=P + 1) == EINVAL
    assert bwd(res=_mat(ad, 255)) == EINVAL and bwd(res=_mat(ad, 256, dtype=5)) == EINVAL
    assert bwd(size=n.value - 1) == ENOSPACE and bwd(ws=None) == EINVAL and bwd(ws=P + 64) == EINVAL


def _tensor(ad, **kw):
    a = dict(n=100, param=P, copy=None, grad=P, m=P, v=P, m_scale=None, v_scale=None, weight_decay=0.01, param_dtype=0,
             grad_dtype=0, state=0)
    a.update(kw)
    return ad.OptTensor(*a.values())


def test_adamw_refusals(ad):
    def run(t=None, count=1, args=None, **kw):
        a = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, seed=0, lr_at=None, step_at=None, grad_scale=None)
        a.update(kw)
        t = _tensor(ad) if t is None else t
        return ad.LIB.ad_adamw((ad.OptTensor * 1)(t), count, ctypes.byref(ad.AdamwArgs(*a.values())), None)

    assert run(count=-1) == ERANGE
    assert ad.LIB.ad_adamw(None, 1, ctypes.byref(ad.AdamwArgs()), None) == EINVAL
    assert ad.LIB.ad_adamw((ad.OptTensor * 1)(_tensor(ad)), 1, None, None) == EINVAL
    for name, bad in (("lr", -1e-3), ("lr", math.nan), ("lr", math.inf), ("beta1", 1.0), ("beta1", -0.1), ("beta2", 1.0),
                      ("beta2", math.nan), ("eps", -1e-8), ("eps", math.nan), ("step", 0), ("step", -3)):
        assert run(**{name: bad}) == ERANGE, name
    for name in ("lr_at", "step_at", "grad_scale"):
        assert run(**{name: P + 2}) == EINVAL
    for bad, status in ((dict(n=-1), ERANGE), (dict(n=(1 << 40) + 1), ERANGE), (dict(param=None), EINVAL),
                        (dict(grad=None), EINVAL), (dict(m=None), EINVAL), (dict(v=None), EINVAL),
                        (dict(param=P + 2), EINVAL), (dict(grad=P + 1, grad_dtype=1), EINVAL), (dict(m=P + 2), EINVAL),
                        (dict(param_dtype=2), EINVAL), (dict(grad_dtype=-1), EINVAL), (dict(state=2), EINVAL),
                        (dict(state=1), EINVAL), (dict(state=1, m_scale=P), EINVAL),
                        (dict(state=1, m_scale=P, v_scale=P + 2), EINVAL), (dict(copy=P, param_dtype=1), EINVAL),
                        (dict(copy=P + 1), EINVAL), (dict(weight_decay=-0.1), ERANGE),
                        (dict(weight_decay=math.nan), ERANGE)):
        assert run(_tensor(ad, **bad)) == status, bad


def test_norm_and_state_refusals(ad):
    n = ctypes.c_size_t()
    one = (ad.OptTensor * 1)(_tensor(ad, n=100000))
    size = ad.LIB.ad_grad_norm_workspace_size
    assert size(one, 1, None) == EINVAL and size(None, 1, ctypes.byref(n)) == EINVAL and size(one, -1, ctypes.byref(n)) == ERANGE
    assert size(one, 0, ctypes.byref(n)) == 0 and n.value == 0
    assert size(one, 1, ctypes.byref(n)) == 0 and n.value > 0

    def norm(t=one, count=1, most=1.0, out=P, step=None, ws=P, have=n.value):
        return ad.LIB.ad_grad_norm(t, count, most, out, step, ws, have, None)

    assert norm(most=-1.0) == ERANGE and norm(most=math.nan) == ERANGE and norm(most=math.inf) == ERANGE
    assert norm(out=None) == EINVAL and norm(out=P + 2) == EINVAL and norm(step=P + 2) == EINVAL
    assert norm(have=n.value - 1) == ENOSPACE and norm(ws=None) == EINVAL and norm(ws=P + 8) == EINVAL
    assert norm(t=(ad.OptTensor * 1)(_tensor(ad, grad=None))) == EINVAL
    assert norm(t=(ad.OptTensor * 1)(_tensor(ad, grad_dtype=7))) == EINVAL
    assert ad.LIB.ad_opt_state(one, 1, P + 2, P, None) == EINVAL and ad.LIB.ad_opt_state(one, -1, P, P, None) == ERANGE
    assert ad.LIB.ad_opt_state((ad.OptTensor * 1)(_tensor(ad, m=None)), 1, P, P, None) == EINVAL
    assert ad.LIB.ad_opt_state((ad.OptTensor * 1)(_tensor(ad, state=1)), 1, P, P, None) == EINVAL


def test_binding_refusals(ad):
    import torch
    i32 = dict(dtype=torch.int32)
    cu = torch.tensor([0, 4], **i32)
    with pytest.raises(ValueError, match="int32"):
        ad.Attention(1, 1, cu.long(), cu, 4, 4)
    with pytest.raises(ValueError, match="cu_k"):
        ad.Attention(1, 1, cu, torch.zeros(3, **i32), 4, 4)
    with pytest.raises(ValueError, match="window"):
        ad.Attention(1, 1, cu, cu, 4, 4, window=torch.zeros(4, 3, **i32))
    at = ad.Attention(2, 1, cu, cu, 4, 4, window=torch.zeros(4, 2, **i32))
    with pytest.raises(ValueError, match="window has 4 rows"):
        ad.attention_workspace_size(at, 5, 4)
    x = torch.zeros(4, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="not on the current GPU"):
        ad.attention(at, x, x[:, :64], x[:, :64], x)
    f = [torch.zeros(10)]
    for kw in (dict(params=f, grads=[torch.zeros(9)]), dict(params=f, grads=[f[0].half()]), dict(params=f, grads=f * 2),
               dict(grads=f, m=[torch.zeros(10, dtype=torch.int8)]), dict(), dict(grads=f, weight_decay=[0.1, 0.2]),
               dict(params=f, copies=[torch.zeros(10)]), dict(params=[torch.zeros(10, 2)[:, 0]])):
        with pytest.raises(ValueError):
            ad.OptTensors(**kw)
