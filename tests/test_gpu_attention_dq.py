"""dq where its terms cancel: keys that share a large component, which sum_j dS_ij = 0 takes out of dq but which dS's
rounding errors are multiplied with.

Bound.  A value that lies anywhere between its neighbours is off by spacing / sqrt(12) in root mean square when it is rounded,
and bf16's spacing is at most 2^-7 of the value: 2^-7 / sqrt(12) of dq's own root mean square, with 5% for the chance of some
thousand values.  Besides that dq is off by what float32 and two bf16 parts lose (attention_common: scores, p, dP and delta as
there, and h^2 for dS in two parts of which each is rounded once): taken in full.  dS in one part is off by about 2^-7 /
sqrt(12) of itself times the shared component: over the bound, which the first test shows in float64.
"""
import math

import pytest
import torch

from attention_common import BF16, H, U, Batch, Ref, backward

SHARED = 8.0            # the component, where the keys differ by 1
SHAPES = {
    "few": dict(ql=[40, 9], kl=[40, 60], heads=2, kv=1),
    "few_causal": dict(ql=[100], kl=[100], heads=2, kv=2, causal=True),
    "few_windows": dict(ql=[40, 33], kl=[150, 129], heads=2, kv=2, window="random"),
    "both": dict(ql=[60] * 16, kl=[60] * 16, heads=8, kv=4),
    "wide": dict(ql=[60] * 40, kl=[60] * 40, heads=16, kv=16),
    "wide_windows": dict(ql=[40, 33] * 32, kl=[100, 60] * 32, heads=16, kv=16, window="random"),
}


def _batch(name):
    bt = Batch(seed=sum(map(ord, name)), spread=0.1, **SHAPES[name])
    bt.k = (bt.k.float() + SHARED).to(BF16)
    return bt


def _lost(bt, once=False):
    """What dq may lose besides its own rounding, [rows][columns]; once: what it loses with dS rounded once."""
    n = bt.heads // bt.kv
    wide = lambda x, m: x.double().view(-1, m, 64).transpose(0, 1)  # noqa: E731
    q, k, v, do = wide(bt.q, bt.heads), wide(bt.k, bt.kv), wide(bt.v, bt.kv), wide(bt.dout, bt.heads)
    lost = torch.zeros_like(q)
    for b in range(bt.batch):
        a, e, nq, nk = bt.cu_q[b], bt.cu_k[b], bt.ql[b], bt.kl[b]
        seen = bt.seen(b)
        for h in range(bt.heads):
            Q, K, V, D = q[h, a:a + nq], k[h // n, e:e + nk], v[h // n, e:e + nk], do[h, a:a + nq]
            x = (Q @ K.T / 8).masked_fill(~seen, -math.inf)
            lse = torch.logsumexp(x, 1, keepdim=True)
            lse = lse.masked_fill(lse == -math.inf, 0.0)
            p = torch.exp(x - lse)
            mag = (Q.abs() @ K.abs().T / 8).masked_fill(~seen, 0.0)
            el = 72 * U * mag + 2 * U * x.masked_fill(~seen, 0.0).abs() + 4 * U * lse.abs() + 4 * U
            o = p @ V
            ed = 64 * U * (D.abs() @ V.abs().T) + (64 * U + 2 * H * H) * (D * o).abs().sum(1, keepdim=True)
            ds = p * (D @ V.T - (D * o).sum(1, keepdim=True))
            if once:
                lost[h, a:a + nq] = (ds.to(BF16).double() - ds) @ K / 8
            else:
                lost[h, a:a + nq] = (ds.abs() * (H * H + el + nk * U) + p * ed * (1 + H)) @ K.abs() / 8
    return lost.transpose(0, 1).flatten(1)


def _rms(x):
    return float(x.square().mean().sqrt())


def _bound(bt, ref):
    return 1.05 * 2.0 ** -7 / math.sqrt(12) * _rms(ref.dq) + _rms(_lost(bt))


@pytest.mark.parametrize("name", ["few", "few_causal", "few_windows", "both"])
def test_one_part_would_be_over_the_bound(name):
    bt = _batch(name)
    assert _rms(_lost(bt, once=True)) > 1.2 * _bound(bt, Ref(bt))


@pytest.mark.gpu
@pytest.mark.parametrize("name", SHAPES)
def test_dq_where_its_terms_cancel(name):
    bt = _batch(name)
    ref = Ref(bt)
    dq, _, _ = backward(bt, ref)
    assert _rms(dq - ref.dq) <= _bound(bt, ref), (_rms(dq - ref.dq) / _rms(ref.dq), _bound(bt, ref) / _rms(ref.dq))
