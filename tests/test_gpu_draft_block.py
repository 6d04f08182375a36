"""The draft block's attention sublayers, the whole block and its optimizer: gradients against float64 autograd of the
definition and against differences, captured steps, refusals.

Tolerances.  h = 2^-8.  Every tensor that passes from one operator to the next is rounded to bf16 or to 8 bits: relative
errors of h a value, independent from value to value.  A gradient is a sum of many of their products, so in norm it is off by
at most h times the square root of the number of roundings on its way (under 12 forward and 12 backward, and an 8-bit checkpoint
is 1 / 254 of its group's largest, under 4 h of a typical value): 4 h sqrt(24) < 20 h of the gradient's norm bounds it with
everything counted as the worst of them.
"""
import math

import pytest
import torch

from paper_2608_12703_amd import ad
from paper_2608_12703_amd.train import AdamW, AttentionScratch, CrossAttention, DraftBlock, SelfAttention

pytestmark = pytest.mark.gpu

H = 2.0 ** -8
BF16, F32 = torch.bfloat16, torch.float32


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _params(d, f, seed):
    """A layer's 20 tensors (bf16), keys without bias."""
    g = _gen(seed)
    r = lambda *s, scale=0.02: (torch.randn(*s, generator=g) * scale).to(BF16)  # noqa: E731
    ln = lambda: [(1 + torch.randn(d, generator=g) * 0.1).to(BF16), r(d)]  # noqa: E731
    w = d ** -0.5
    b_qkv, b_xkv = r(3 * d), r(2 * d)
    b_qkv[d:2 * d] = 0
    b_xkv[:d] = 0
    return [*ln(), r(3 * d, d, scale=w), b_qkv, r(d, d, scale=w), r(d), *ln(), r(d, d, scale=w), r(d),
            r(2 * d, d, scale=w), b_xkv, r(d, d, scale=w), r(d), *ln(), r(f, d, scale=w), r(f), r(d, f, scale=f ** -0.5), r(d)]


class Data:
    """Ragged utterances, padded positions and packed audio, windows on some positions."""

    def __init__(self, d, seed=0, ql=(13, 40, 7), kl=(150, 64, 33), stride=40, window=False):
        g = _gen(seed)
        self.ql, self.kl, self.stride, self.heads = ql, kl, stride, d // 64
        self.rows, self.keys = stride * len(ql), sum(kl)
        self.x = torch.randn(self.rows, d, generator=g)
        self.enc = torch.randn(self.keys, d, generator=g).to(BF16)
        live = torch.zeros(self.rows, 1)
        for b, n in enumerate(ql):
            live[b * stride:b * stride + n] = 1
        self.live = live.bool()[:, 0]
        self.dout = torch.randn(self.rows, d, generator=g) * live * 0.1       # padding has no part in the loss
        self.dxq = torch.randn(self.rows, d, generator=g) * live * 0.1
        self.window = None
        if window:
            lo = torch.randint(0, 30, (self.rows,), generator=g)
            self.window = torch.stack([lo, lo + torch.randint(0, 60, (self.rows,), generator=g)], 1).to(torch.int32)
        ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        cu = [b * stride for b in range(len(ql) + 1)]
        ck = [0]
        for n in kl:
            ck.append(ck[-1] + n)
        self.cu_k = ck
        h = self.heads
        self.self_batch = ad.Attention(h, h, ints(cu), ints(cu), stride, stride, q_len=ints(ql), k_len=ints(ql),
                                       causal=True, covers=True)
        self.cross_batch = ad.Attention(h, h, ints(cu), ints(ck), stride, max(kl), q_len=ints(ql),
                                        window=None if self.window is None else self.window.cuda(), covers=True)


def _attend(q, k, v, heads, seen):
    s = lambda t: t.view(t.shape[0], heads, 64).transpose(0, 1)  # noqa: E731
    x = (s(q) @ s(k).transpose(1, 2) / 8).masked_fill(~seen, -math.inf)
    dead = ~seen.any(1)
    x = x.masked_fill(dead[:, None], 0.0)
    p = torch.softmax(x, -1).masked_fill(dead[:, None], 0.0)
    return (p @ s(v)).transpose(0, 1).flatten(1)


def _norm(x, g, b):
    return torch.nn.functional.layer_norm(x, (x.shape[1],), g, b, 1e-5)


def _self(p, x, t):
    qkv = _norm(x, p[0], p[1]) @ p[2].T + p[3]
    d = x.shape[1]
    o = torch.zeros_like(x)
    for b, n in enumerate(t.ql):
        r = slice(b * t.stride, b * t.stride + n)
        seen = torch.ones(n, n, dtype=torch.bool).tril()
        o = o.index_put((torch.arange(r.start, r.stop),), _attend(qkv[r, :d], qkv[r, d:2 * d], qkv[r, 2 * d:], t.heads, seen))
    return x + o @ p[4].T + p[5]


def _cross(p, x, t):
    q = _norm(x, p[0], p[1]) @ p[2].T + p[3]
    kv = t.enc.double() @ p[4].T + p[5]
    d = x.shape[1]
    o = torch.zeros_like(x)
    for b, (n, m) in enumerate(zip(t.ql, t.kl)):
        r, c = slice(b * t.stride, b * t.stride + n), slice(t.cu_k[b], t.cu_k[b + 1])
        seen = torch.ones(n, m, dtype=torch.bool)
        if t.window is not None:
            w, j = t.window[r].long(), torch.arange(m)
            seen = (j >= w[:, :1]) & (j < w[:, 1:])
        o = o.index_put((torch.arange(r.start, r.stop),), _attend(q[r], kv[c, :d], kv[c, d:], t.heads, seen))
    return x + o @ p[6].T + p[7], q


def _block(p, x, t):
    y, q = _cross(p[6:14], _self(p[:6], x, t), t)
    h = _norm(y, p[14], p[15]) @ p[16].T + p[17]
    return y + torch.nn.functional.gelu(h) @ p[18].T + p[19], q


def _leaves(params):
    return [q.double().requires_grad_() for q in params]


def _off(got, want):
    return float((got.double().cpu() - want).norm() / want.norm().clamp(min=1e-30))


def _close(got, want, what, tol=20 * H):
    assert _off(got, want) <= tol, (what, _off(got, want))


@pytest.mark.parametrize("d", [64, 192])
def test_self_attention_sublayer(d):
    t, params = Data(d, seed=d), _params(d, 2 * d, d)[:6]
    layer = SelfAttention([p.cuda() for p in params], t.rows, AttentionScratch(d, t.rows, 8, 3))
    x, out, dx = t.x.cuda(), torch.empty(t.rows, d, device="cuda"), torch.empty(t.rows, d, device="cuda")
    layer.forward(x, t.self_batch, out)
    layer.backward(t.dout.cuda(), dx)
    leaves, X = _leaves(params), t.x.double().requires_grad_()
    want = _self(leaves, X, t)
    (want * t.dout.double()).sum().backward()
    _close(out.cpu()[t.live] - t.x[t.live], (want - X).detach()[t.live], "out")
    _close(dx, X.grad, "dx")
    for i, (g, p) in enumerate(zip(layer.grads, leaves)):
        if i == 3:
            assert not bool(g[d:2 * d].any())
            _close(torch.cat([g[:d], g[2 * d:]]), torch.cat([p.grad[:d], p.grad[2 * d:]]), "b_qkv")
        else:
            _close(g, p.grad, i)
    first = [g.clone() for g in layer.grads]
    layer.backward(t.dout.cuda(), dx)                              # gradients are added to
    assert all(torch.allclose(g, 2 * f, rtol=1e-6, atol=0) for g, f in zip(layer.grads, first))
    assert int(t.self_batch.err_flag) == 0


@pytest.mark.parametrize("window,dxq", [(False, False), (True, True)])
def test_cross_attention_sublayer(window, dxq):
    d = 128
    t, params = Data(d, seed=5, window=window), _params(d, 2 * d, 6)[6:14]
    layer = CrossAttention([p.cuda() for p in params], t.rows, t.keys, AttentionScratch(d, t.rows, t.keys, 3))
    x, out, dx = t.x.cuda(), torch.empty(t.rows, d, device="cuda"), torch.empty(t.rows, d, device="cuda")
    xq = torch.empty(t.rows, d, device="cuda") if dxq else None
    layer.forward(x, t.enc.cuda(), t.cross_batch, out, xq)
    layer.backward(t.dout.cuda(), dx, dxq=t.dxq.cuda() if dxq else None)
    leaves, X = _leaves(params), t.x.double().requires_grad_()
    want, q = _cross(leaves, X, t)
    loss = (want * t.dout.double()).sum()
    if dxq:
        loss = loss + (q * t.dxq.double()).sum()
        _close(xq.cpu()[t.live], q.detach()[t.live], "xq")
    loss.backward()
    _close(out.cpu()[t.live] - t.x[t.live], (want - X).detach()[t.live], "out")
    _close(dx, X.grad, "dx")
    for i, (g, p) in enumerate(zip(layer.grads, leaves)):
        if i == 5:
            assert not bool(g[:d].any())
            _close(g[d:], p.grad[d:], "b_xkv")
        else:
            _close(g, p.grad, i)


def _made(d=128, f=192, seed=3):
    t = Data(d, seed=seed)
    params = [p.cuda() for p in _params(d, f, seed + 1)]
    return t, params, DraftBlock(params, t.rows, t.keys, 3)


def test_block_gradients():
    t, params, block = _made()
    x, out, dx = t.x.cuda(), torch.empty_like(t.x, device="cuda"), torch.empty_like(t.x, device="cuda")
    xq = torch.empty_like(x)
    block.forward(x, t.enc.cuda(), t.self_batch, t.cross_batch, out, xq)
    block.backward(t.dout.cuda(), dx, t.dxq.cuda())
    leaves, X = _leaves([p.cpu() for p in params]), t.x.double().requires_grad_()
    want, q = _block(leaves, X, t)
    ((want * t.dout.double()).sum() + (q * t.dxq.double()).sum()).backward()
    _close(out.cpu()[t.live] - t.x[t.live], (want - X).detach()[t.live], "out")
    _close(dx, X.grad, "dx")
    d = block.d
    for i, (g, p) in enumerate(zip(block.grads, leaves)):
        keep = torch.ones(len(p), dtype=torch.bool)
        if i in (3, 11):                                            # the keys' bias has a gradient of 0
            keep[d:2 * d] = i == 11
            keep[:d] = i == 3
        _close(g.cpu()[keep], p.grad[keep], i)


def test_block_gradient_against_differences():
    """Along the gradient itself: L(x + e g) - L(x - e g) = 2 e |g|^2 (1 + O(e^2)) + the passes' roundings, which do
    not depend on e.  e makes the difference far larger than those: the outputs' roundings are 20 h of the change of the
    sublayers' outputs at most, and e |g| is a tenth of |x|."""
    t, params, block = _made(seed=11)
    out, dx = torch.empty_like(t.x, device="cuda"), torch.empty_like(t.x, device="cuda")
    enc, dout = t.enc.cuda(), t.dout.cuda()

    def loss(x):
        block.forward(x, enc, t.self_batch, t.cross_batch, out)
        return float((out.double() * dout.double()).sum())

    x = t.x.cuda()
    loss(x)
    block.backward(dout, dx)
    g = dx.double()
    e = 0.1 * float(x.double().norm() / g.norm()) * 0.3
    diff = (loss((x.double() + e * g).float()) - loss((x.double() - e * g).float())) / (2 * e)
    assert diff == pytest.approx(float(g.square().sum()), rel=20 * H)


@pytest.mark.parametrize("state", ["f32", "8bit"])
def test_training_steps_and_their_graph(state):
    """Forward, backward and the step, eager and captured: the same bits every time, also after replays with other
    eager work between them."""
    def run(captured):
        t, params, block = _made(seed=21)
        opt = AdamW(block.params, block.grads, lr=1e-3, state=state, seed=9)
        x, out, dx = t.x.cuda(), torch.empty_like(t.x, device="cuda"), torch.empty_like(t.x, device="cuda")
        enc, dout = t.enc.cuda(), t.dout.cuda()

        def step():
            block.zero_grads()
            block.forward(x, enc, t.self_batch, t.cross_batch, out)
            block.backward(dout, dx)
            opt.step()

        if captured:
            side = torch.cuda.Stream()
            graph = torch.cuda.CUDAGraph()
            torch.cuda.synchronize()
            with torch.cuda.graph(graph, stream=side):
                step()
            step_ = graph.replay
        else:
            step_ = step
        for k in range(4):
            if k == 2:
                opt.set_lr(5e-4)
            step_()
            if captured:
                torch.randn(1000, device="cuda").sum()
                torch.cuda.synchronize()
        return params, opt, out.clone()

    p0, o0, y0 = run(False)
    p1, o1, y1 = run(True)
    assert torch.equal(y0, y1) and all(torch.equal(a, b) for a, b in zip(p0, p1))
    assert int(o0.steps) == int(o1.steps) == 4
    for a, b in zip(o0.states(), o1.states()):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    for p, m in zip(p1, o1.master):
        assert torch.equal(p, m.to(BF16)) and not torch.equal(p.cpu(), _params(128, 192, 22)[0][:0])
    d = 128
    assert not bool(p1[3][d:2 * d].any()) and not bool(p1[11][:d].any())       # keys keep no bias


def test_a_norm_that_is_not_finite_leaves_the_block():
    t, params, block = _made(seed=31)
    opt = AdamW(block.params, block.grads)
    before = [p.clone() for p in params]
    block.grads[2][5, 7] = math.inf
    opt.step()
    assert all(torch.equal(a, b) for a, b in zip(before, params)) and int(opt.steps) == 0
    block.zero_grads()
    block.grads[2].fill_(1.0)
    opt.step()
    assert int(opt.steps) == 1 and not torch.equal(before[2], params[2])
    n = math.sqrt(block.grads[2].numel())
    assert float(opt.norm[0]) == pytest.approx(n, rel=1e-6) and float(opt.norm[1]) == pytest.approx(1 / n, rel=1e-6)


def test_rows_of_no_sequence_have_no_part():
    """Without `covers`, rows outside the sequences are as if they were not there (their gradient is 0)."""
    d = 64
    t, params = Data(d, seed=41), _params(d, 2 * d, 42)
    dev = [p.cuda() for p in params]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    rows = t.rows + 30
    x = torch.cat([torch.full((10, d), 3.0), t.x, torch.full((20, d), -5.0)]).cuda()
    dout = torch.cat([torch.zeros(10, d), t.dout, torch.zeros(20, d)]).cuda()
    cu = ints([10 + b * t.stride for b in range(4)])
    batch = ad.Attention(1, 1, cu, cu, t.stride, t.stride, q_len=ints(t.ql), k_len=ints(t.ql), causal=True)
    scratch = AttentionScratch(d, rows, 8, 3)
    for buf in (scratch.wide, scratch.keys, scratch.narrow):
        buf.fill_(float("nan"))
    a, b = SelfAttention(dev[:6], rows, scratch), SelfAttention(dev[:6], t.rows, AttentionScratch(d, t.rows, 8, 3))
    a.o.fill_(float("nan"))
    out, dx = torch.empty_like(x), torch.empty_like(x)
    a.forward(x, batch, out)
    a.backward(dout, dx)
    y, dy = torch.empty(t.rows, d, device="cuda"), torch.empty(t.rows, d, device="cuda")
    b.forward(t.x.cuda(), t.self_batch, y)
    b.backward(t.dout.cuda(), dy)
    assert torch.equal(out[10:10 + t.rows], y) and torch.equal(dx[10:10 + t.rows], dy)
    for g, h in zip(a.grads, b.grads):
        assert bool(torch.isfinite(g).all()) and _off(g, h.double().cpu()) <= 1e-4


def test_refusals():
    t, params, block = _made(seed=51)
    x, enc = t.x.cuda(), t.enc.cuda()
    out, dx, dout = torch.empty_like(x), torch.empty_like(x), t.dout.cuda()
    with pytest.raises(ValueError, match="last forward"):
        block.self_attention.backward(dout, dx)
    block.forward(x, enc, t.self_batch, t.cross_batch, out)
    wrong = ad.Attention(1, 1, t.self_batch._tables[0], t.self_batch._tables[0], 40, 40)
    for bad in (lambda: block.self_attention.forward(x, wrong, out),
                lambda: block.self_attention.forward(x.double(), t.self_batch, out),
                lambda: block.self_attention.forward(torch.cat([x, x]), t.self_batch, out),
                lambda: block.cross_attention.forward(x, torch.cat([enc, enc]), t.cross_batch, out),
                lambda: block.cross_attention.forward(x, enc.float(), t.cross_batch, out),
                lambda: block.cross_attention.forward(x, enc, t.cross_batch, out, out[:, :64]),
                lambda: block.self_attention.backward(dout[:5], dx), lambda: block.self_attention.backward(dout, dx[:, :64]),
                lambda: block.cross_attention.backward(dout, dx, dxq=dout.half()),
                lambda: block.self_attention.backward(dout.half(), dx)):
        with pytest.raises((ValueError, ad.ADError)):
            bad()
        assert not any(bool(g.any()) for g in block.grads)
    with pytest.raises(ValueError, match="20"):
        DraftBlock(params[:19], 8, 8, 1)
    with pytest.raises(ValueError, match="scratch"):
        SelfAttention(params[:6], 1000, AttentionScratch(128, 10, 8, 3))
    with pytest.raises(ValueError, match="state"):
        AdamW(params, block.grads, state="4bit")
    with pytest.raises(ValueError):
        AdamW(params, block.grads[:3])


def test_a_training_step_of_the_objective():
    """What a training loop runs: the block, its final LayerNorm and the target's head, the objective, back through all of
    them, and the step, which the draft model reads its new weights from.  Gradients against autograd of L_tok + lambda
    L_anchor in float64 (the alignment term's gradient goes through the queries; tolerance above, with the head's logits,
    whose gradient is rounded to bf16, as two operators more)."""
    from paper_2608_12703_amd import synth
    from paper_2608_12703_amd.configs import Config
    from paper_2608_12703_amd.harness import Session
    cfg = Config(name="unit_step", n_layers=2, d_model=128, n_heads=2, d_ffn=256, vocab=1000, dtype="bf16", batch=3, k=4,
                 k_min=0, frames=150, frames_min=40, kv_max=0, geo_p=0.3, seed=13)
    dcfg = synth.draft_config(cfg)
    target, own = synth.make_params(cfg), synth.make_draft_params(cfg)
    named = {n: own[n] for n, _ in synth.param_specs(dcfg) if n not in ("tok_emb", "pos_emb")}
    named["tok_emb"], named["pos_emb"] = target["tok_emb"], target["pos_emb"]
    B, R, Ts, d, V, sigma, lam = 3, 24, [150, 90, 41], cfg.d_model, cfg.vocab, 5.0, 0.1
    sess = Session(dcfg, named, B, R - 1, Ts, want_logits=True)
    g = _gen(71)
    encs = [synth.make_encoder(cfg, b, T) for b, T in enumerate(Ts)]
    layer = sess.model.params[4:24]                        # the tensors that the draft model reads
    head, gain, bias = sess.model.params[0], sess.model.params[2], sess.model.params[3]
    f = layer[16].shape[0]
    ql, rows = [24, 17, 9], B * R
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    cu, off = [b * R for b in range(B + 1)], sess.enc_off.tolist() + [sess.frames_cap]
    self_batch = ad.Attention(2, 2, ints(cu), ints(cu), R, R, q_len=ints(ql), k_len=ints(ql), causal=True, covers=True)
    cross_batch = ad.Attention(2, 2, ints(cu), ints(off), R, max(b - a for a, b in zip(off, off[1:])), q_len=ints(ql),
                               k_len=ints(Ts), covers=True)
    x = torch.randn(rows, d, generator=g)
    live = torch.cat([torch.arange(R) < n for n in ql])
    targets = torch.where(live, torch.randint(0, V, (rows,), generator=g), -1)
    center = torch.where(live & (torch.rand(rows, generator=g) < 0.7), torch.randint(0, 41, (rows,), generator=g), -1)

    block = DraftBlock(layer, rows, sess.frames_cap, B)
    opt = AdamW(block.params, block.grads, state="8bit", seed=3)
    e = lambda *s, dt=F32: torch.empty(*s, dtype=dt, device="cuda")  # noqa: E731
    X, enc, err = x.cuda(), sess.upload_encoder(encs), torch.zeros(1, dtype=torch.int32, device="cuda")
    out, xq, h, mean, rstd, logits = e(rows, d), e(rows, d), e(rows, d, dt=BF16), e(rows), e(rows), e(rows, V)
    terms, row, dxq, dlogits, dh, dx = e(4), e(rows), e(rows, d), e(rows, V), e(rows, d), e(rows, d)
    need = max(ad.anchordraft_loss_workspace_size(sess.model, B, R), ad.linear_workspace_size(rows, V, d),
               ad.linear_dgrad_workspace_size(rows, V, d), ad.layer_norm_backward_workspace_size(rows, d))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    T32, C32 = targets.to(torch.int32).cuda(), center.to(torch.int32).cuda()

    def pass_():
        sess.prefill_encoder(encs)
        block.zero_grads()
        block.forward(X, enc, self_batch, cross_batch, out, xq)
        ad.layer_norm(out, gain, bias, h, mean, rstd)
        ad.linear(h, head, None, ad.ACT_NONE, None, logits, None, None, ws)
        ad.anchordraft_loss(sess.model, sess.cross_struct(), 0, B, R, xq, C32, sigma, lam, logits, T32, None, None, terms,
                            row, dxq, dlogits, None, err, ws)
        ad.linear_dgrad(dlogits.to(BF16), head, ad.ACT_NONE, None, None, dh, None, ws)
        ad.layer_norm_backward(dh, out, mean, rstd, None, gain, None, dx, None, None, None, None)
        block.backward(dx, dx, dxq)

    def reference(params):
        leaves, x64 = _leaves(params), x.double().requires_grad_()
        t = Data(d, ql=tuple(ql), kl=tuple(Ts), stride=R)
        t.enc = torch.cat([torch.from_numpy(v).float() for v in encs]).to(BF16)
        y, q = _block(leaves, x64, t)
        z = _norm(y, gain.cpu().double(), bias.cpu().double()) @ head.cpu().double().T
        loss = torch.nn.functional.cross_entropy(z, targets, ignore_index=-1)
        kv = (t.enc.double() @ leaves[10].T + leaves[11]).detach()
        n = int((center >= 0).sum())
        for r in torch.nonzero(center >= 0)[:, 0].tolist():
            b = r // R
            k = kv[t.cu_k[b]:t.cu_k[b + 1], :d].view(-1, 2, 64)
            a = torch.softmax(torch.einsum("hd,jhd->hj", q[r].view(2, 64), k) / 8, 1).mean(0)
            w = torch.exp(-(torch.arange(Ts[b]).double() - float(center[r])).square() / (2 * sigma ** 2))
            loss = loss - lam / n * (w / w.sum() * a.log()).sum()
        loss.backward()
        return loss, leaves, x64

    for step in range(2):               # the second pass sees the step's weights, in the block and in the draft model
        before = [p.cpu() for p in layer]
        pass_()
        assert int(err) == 0 and int(self_batch.err_flag) == 0 and int(cross_batch.err_flag) == 0
        loss, leaves, x64 = reference(before)
        assert float(terms[0]) == pytest.approx(float(loss.detach()), rel=4 * H)
        _close(dx, x64.grad, "dx", 22 * H)
        for i, (got, p) in enumerate(zip(block.grads, leaves)):
            keep = torch.ones(len(p), dtype=torch.bool)
            if i in (3, 11):
                keep[d:2 * d] = i == 11
                keep[:d] = i == 3
            _close(got.cpu()[keep], p.grad[keep], (step, i), 22 * H)
        opt.step()
        # (a step of 1e-3 is under half of bf16's step next to a LayerNorm's gain of 1: those move in float32 first)
        assert all(not torch.equal(a, b.cpu()) for a, b in zip(before, layer) if a.dim() > 1)
    assert int(opt.steps) == 2 and f == 256
