"""Batches for the attention tests, their definition in float64, and bounds on what float32 and bf16 lose.

Bounds.  u = 2^-24 and h = 2^-8 are half a step of float32 and of bf16, relative.
  scores     64 exact products added in float32, scaled, the largest one taken off: at most 72 u of the sum of
             magnitudes, and u of the value twice.
  p          its exponent's error and 4 u (exponential, quotient, the sum of n terms at n u); rounded to bf16, h more.
  lse        the scores' largest error, (n + 4) u, and 2 u of itself.
  o          sum p |v| (h + p's error) + n u, rounded once: h of itself.
  backward   p from lse (float32: u of itself more); dP 64 products of bf16; delta from o as two bf16 values (2 h^2
             of sum |dout o|, and 64 additions); dS rounded to bf16; sums of n or n rows in float32; outputs rounded once.
"""
import math

import torch

from paper_2608_12703_amd import ad

U, H = 2.0 ** -24, 2.0 ** -8
BF16 = torch.bfloat16
GUARD = -77.0


class Batch:
    """Sequences of ql query and kl key rows; padded: rows apart by the longest; lead: rows before the first
    sequence and after the last; window: None or a list of (lo, hi) for every row."""

    def __init__(self, ql, kl, heads=2, kv=2, causal=False, window=None, padded=False, seed=0, lead=0, spread=1.0):
        g = torch.Generator().manual_seed(seed)
        self.ql, self.kl, self.heads, self.kv, self.causal = ql, kl, heads, kv, causal
        self.batch = len(ql)

        def place(lens):
            own = [max(lens)] * len(lens) if padded else lens
            cu = [lead]
            for n in own:
                cu.append(cu[-1] + n)
            return cu, cu[-1] + lead

        self.padded = padded
        self.cu_q, self.q_rows = place(ql)
        self.cu_k, self.k_rows = place(kl)
        rand = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
        self.q = (rand(self.q_rows, 64 * heads) * spread).to(BF16)
        self.k = rand(self.k_rows, 64 * kv).to(BF16)
        self.v = rand(self.k_rows, 64 * kv).to(BF16)
        self.dout = rand(self.q_rows, 64 * heads).to(BF16)
        if window == "random":
            lo = torch.randint(-5, max(kl) + 3, (self.q_rows,), generator=g)
            self.window = torch.stack([lo, lo + torch.randint(-3, 70, (self.q_rows,), generator=g)], 1).to(torch.int32)
        else:
            self.window = window

    def seen(self, b):
        """[ql][kl] visible."""
        nq, nk = self.ql[b], self.kl[b]
        i, j = torch.arange(nq)[:, None], torch.arange(nk)[None]
        s = torch.ones(nq, nk, dtype=torch.bool)
        if self.causal:
            s &= j <= i + nk - nq
        if self.window is not None:
            w = self.window[self.cu_q[b]:self.cu_q[b] + nq].long()
            s &= (j >= w[:, :1]) & (j < w[:, 1:])
        return s

    def handle(self, err=None, **more):
        ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        a = dict(q_len=ints(self.ql), k_len=ints(self.kl)) if self.padded else {}
        return ad.Attention(self.heads, self.kv, ints(self.cu_q), ints(self.cu_k), max(self.ql), max(self.kl), **a,
                            causal=self.causal, window=None if self.window is None else self.window.cuda(), err_flag=err)


class Ref:
    """The definition on rows q, k, v, dout of the batch, and bounds (o, lse, dq, dk, dv and tol_*), all float64;
    rows of no sequence hold GUARD."""

    def __init__(self, bt, res=None):
        n = bt.heads // bt.kv
        wide = lambda x, m: x.double().view(-1, m, 64).transpose(0, 1)  # noqa: E731
        q, k, v, do = wide(bt.q, bt.heads), wide(bt.k, bt.kv), wide(bt.v, bt.kv), wide(bt.dout, bt.heads)
        full = lambda x: torch.full_like(x, GUARD)  # noqa: E731
        self.o, self.dq, self.dk, self.dv = full(q), full(q), full(k), full(v)
        self.tol_o, self.tol_dq, self.tol_dk, self.tol_dv = (torch.zeros_like(x) for x in (q, q, k, v))
        self.lse = torch.full(q.shape[:2], GUARD, dtype=torch.float64)
        self.tol_lse = torch.zeros_like(self.lse)
        for b in range(bt.batch):
            a, e, nq, nk = bt.cu_q[b], bt.cu_k[b], bt.ql[b], bt.kl[b]
            a1, e1 = bt.cu_q[b + 1], bt.cu_k[b + 1]
            for x in (self.o, self.dq):
                x[:, a:a1] = 0.0
            for x in (self.dk, self.dv):
                x[:, e:e1] = 0.0
            self.lse[:, a:a1] = -math.inf
            if res is not None:
                self.dq[:, a:a + nq] = wide(res, bt.heads)[:, a:a + nq]
            if not nq or not nk:
                continue
            seen = bt.seen(b)
            for hq in range(bt.heads):
                g = hq // n
                Q, K, V, D = q[hq, a:a + nq], k[g, e:e + nk], v[g, e:e + nk], do[hq, a:a + nq]
                x = (Q @ K.T / 8).masked_fill(~seen, -math.inf)
                mag = (Q.abs() @ K.abs().T / 8).masked_fill(~seen, 0.0)
                lse = torch.logsumexp(x, 1)
                p = torch.exp(x - lse.masked_fill(lse == -math.inf, 0.0)[:, None])
                ex = 72 * U * mag + 2 * U * x.masked_fill(~seen, 0.0).abs()      # a score's error
                top = ex.amax(1, keepdim=True)
                rows = (nk + 8) * U
                ep = ex + top + rows
                o = p @ V
                self.o[hq, a:a + nq] = o
                self.tol_o[hq, a:a + nq] = (p * (H + ep)) @ V.abs() + H * o.abs() + 1e-30
                self.lse[hq, a:a + nq] = lse
                self.tol_lse[hq, a:a + nq] = top[:, 0] + rows + 2 * U * lse.masked_fill(lse == -math.inf, 0.0).abs()
                # backward, from o and lse as given: o in two bf16 values, lse in float32
                el = ex + 4 * U * lse.masked_fill(lse == -math.inf, 0.0).abs()[:, None] + 4 * U
                dp = D @ V.T
                delta = (D * o).sum(1, keepdim=True)
                ed = 64 * U * (D.abs() @ V.abs().T) + (64 * U + 2 * H * H) * (D * o).abs().sum(1, keepdim=True)
                ds = p * (dp - delta)
                eds = ds.abs() * (H + el) + p * ed * (1 + H)
                self.dq[hq, a:a + nq] += ds @ K / 8
                self.tol_dq[hq, a:a + nq] = (eds + nk * U * ds.abs()) @ K.abs() / 8
                self.dk[g, e:e + nk] += ds.T @ Q / 8
                self.tol_dk[g, e:e + nk] += (eds + n * nq * U * ds.abs()).T @ Q.abs() / 8
                self.dv[g, e:e + nk] += p.T @ D
                self.tol_dv[g, e:e + nk] += (p * (H + el + n * nq * U)).T @ D.abs()
        flat = lambda x: x.transpose(0, 1).flatten(1)  # noqa: E731
        for name in ("dq", "dk", "dv"):
            t = getattr(self, "tol_" + name)
            t += H * getattr(self, name).abs() * (1 + H) + 1e-30
        for name in ("o", "dq", "dk", "dv", "tol_o", "tol_dq", "tol_dk", "tol_dv"):
            setattr(self, name, flat(getattr(self, name)))


def put(t, pad=0, shift=0):
    """t on the GPU, rows `pad` elements apart, the first one `shift` elements into its buffer."""
    rows, cols = t.shape
    flat = torch.full((rows * (cols + pad) + shift + 8,), GUARD, dtype=t.dtype, device="cuda")
    view = flat[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(t)
    return view


class Out:
    """A [rows][cols] output inside a guarded buffer."""

    def __init__(self, rows, cols, dtype=BF16, pad=0, shift=0):
        n = rows * (cols + pad)
        self.flat = torch.full((shift + n + 64,), GUARD, dtype=dtype, device="cuda")
        self.t = self.flat[shift:shift + n].view(rows, cols + pad)[:, :cols]

    def get(self):
        """The values in float64; nothing around them was written."""
        v = self.t.double().cpu()
        self.t.fill_(GUARD)
        assert bool((self.flat == GUARD).all()), "wrote outside the output"
        return v


def near(got, want, tol, what):
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    bad = ~(same | ((got - want).abs() <= tol))
    assert not bool(bad.any()), (what, float((got - want).abs()[bad].max()), int(bad.sum()), tuple(want.shape),
                                 bad.nonzero()[:4].tolist())


def space(size, at, bt):
    return torch.empty(size(at, bt.q_rows, bt.k_rows), dtype=torch.uint8, device="cuda")


def forward(bt, pad=0, shift=0, rest=True, err=None):
    """(o, o_rest, lse) of the kernels, on the GPU, and the handle."""
    at = bt.handle(err)
    w = 64 * bt.heads
    o, r = Out(bt.q_rows, w, pad=pad, shift=shift), Out(bt.q_rows, w, pad=pad, shift=shift) if rest else None
    lse = torch.full((bt.heads, bt.q_rows), GUARD, device="cuda")
    ad.attention(at, put(bt.q, pad, shift), put(bt.k, pad, shift), put(bt.v, pad, shift), o.t, lse,
                 None if r is None else r.t, space(ad.attention_workspace_size, at, bt))
    return at, o, r, lse


def backward(bt, ref, pad=0, shift=0, res=None, rest=True):
    """(dq, dk, dv) of the kernels from the reference's o and lse."""
    at = bt.handle()
    w, wk = 64 * bt.heads, 64 * bt.kv
    o = ref.o.to(BF16)
    low = (ref.o - o.double()).to(BF16)
    dq, dk, dv = Out(bt.q_rows, w, pad=pad, shift=shift), Out(bt.k_rows, wk, pad=pad, shift=shift), Out(bt.k_rows, wk, pad=pad, shift=shift)
    p = lambda x: put(x, pad, shift)  # noqa: E731
    ad.attention_backward(at, p(bt.q), p(bt.k), p(bt.v), p(o), p(low) if rest else None, ref.lse.float().cuda(), p(bt.dout),
                          None if res is None else p(res), dq.t, dk.t, dv.t,
                          space(ad.attention_backward_workspace_size, at, bt))
    assert int(at.err_flag) == 0
    return dq.get(), dk.get(), dv.get()
