"""The draft block's sublayers, forward and backward, and their optimizer, through the C-ABI.

    SelfAttention    out = x + Wo Attn(Wqkv LN(x) + bqkv) + bo         causal inside a sequence
    CrossAttention   out = x + Wxo Attn(Wxq LN(x) + bxq, Wxkv enc + bxkv) + bxo
    FeedForward      out = x + W2 GELU(W1 LN(x) + b1) + b2
    DraftBlock       the three in a row; their parameters are a model layer's, in ad_model_create's order
    AdamW            a step over all of them, clipped by the gradients' norm

From the forward to the backward pass the feed-forward sublayer keeps the normalised rows and the
pre-activation in 8 bits: 1.03 (d + f) bytes a row and 4 for LayerNorm's factor, where the LayerNorm
output, the pre-activation and GELU's output in bf16 would be 2 d + 4 f.  An attention sublayer keeps the normalised
rows in 8 bits, queries, keys, values, and its output in two bf16 values a number.  A running pass also needs
rows and a workspace (Scratch, AttentionScratch), which sublayers can share.  Like Session they own
their buffers and only call libad entry points.
"""
from __future__ import annotations

import torch

from . import ad


class Scratch:
    """What passes over up to max_rows rows need only while they run: rows of width d and f in bf16, and one
    workspace for every call, large enough for any number of rows up to max_rows (a captured pass
    keeps its address).  Sublayers whose passes follow one another, on one stream or as graphs that are
    replayed in turn, can share one; passes that may overlap need one each."""

    def __init__(self, d: int, f: int, max_rows: int, device="cuda"):
        empty = lambda *shape, dt=torch.bfloat16: torch.empty(*shape, dtype=dt, device=device)  # noqa: E731
        self.d, self.f, self.max_rows = d, f, max_rows
        self.narrow, self.wide, self.wide2 = empty(max_rows, d), empty(max_rows, f), empty(max_rows, f)
        # What a call needs changes with its rows at multiples of 64 only, and the LayerNorm's grows with them.
        need = ad.layer_norm_backward_workspace_size(max_rows, d)
        for rows in range(64, max_rows + 64, 64):
            need = max(need, *(size(rows, *shape) for shape in ((d, f), (f, d)) for size in
                               (ad.linear_workspace_size, ad.linear_dgrad_workspace_size,
                                ad.linear_wgrad_workspace_size)))
        self.workspace = empty(max(need, 1), dt=torch.uint8)


class FeedForward:
    """Buffers for up to max_rows rows.  params: (ln_gain [d], ln_bias [d], w1 [f][d], b1 [f],
    w2 [d][f], b2 [d]) on the GPU, w1 and w2 in bf16.  scratch: shared with other sublayers, or None
    for one of its own.  Gradients are float32 tensors of the parameters' shapes in `grads`, in the same
    order; backward adds to them (zero_grads clears them)."""

    def __init__(self, params, max_rows: int, scratch: Scratch | None = None):
        self.gain, self.bias, self.w1, self.b1, self.w2, self.b2 = params
        self.f, self.d = self.w1.shape
        d, f, dev = self.d, self.f, self.w1.device
        self.max_rows = max_rows
        self.scratch = Scratch(d, f, max_rows, dev) if scratch is None else scratch
        s = self.scratch
        if (s.d, s.f) != (d, f) or s.max_rows < max_rows or s.workspace.device != dev:
            raise ValueError(f"scratch of {(s.d, s.f)} for {s.max_rows} rows on {s.workspace.device}, "
                             f"expected {(d, f)} for {max_rows} on {dev}")
        self.rstd = torch.empty(max_rows, dtype=torch.float32, device=dev)
        self.xhat = ad.Ckpt.empty(max_rows, d, dev)
        self.pre = ad.Ckpt.empty(max_rows, f, dev)
        self.grads = [torch.zeros(p.shape, dtype=torch.float32, device=dev) for p in params]
        self.rows = None

    @property
    def workspace(self):
        return self.scratch.workspace

    def zero_grads(self):
        for g in self.grads:
            g.zero_()

    def _kept(self, rows: int):
        cut = lambda k: ad.Ckpt(k.q[:rows], k.scale[:rows], k.cols)  # noqa: E731
        return cut(self.xhat), cut(self.pre)

    def _rows(self, name: str, t, rows: int, *dtypes):
        """Refuses what a later call of the pass would refuse, before the first one has written."""
        if not t.is_cuda or t.get_device() != torch.cuda.current_device():
            raise ValueError(f"{name} is on {t.device}, not on the current GPU")
        if t.shape != (rows, self.d) or t.dtype not in dtypes:
            raise ValueError(f"{name} is {tuple(t.shape)} of {t.dtype}, expected {(rows, self.d)} of {dtypes}")
        ld, step = t.stride()
        if (self.d > 1 and step != 1) or (rows > 1 and not self.d <= ld <= 1 << 22):
            raise ValueError(f"{name}: the columns of a row must be adjacent, and rows apart by at most 2^22")

    def forward(self, x, out):
        """out <- x + W2 GELU(W1 LN(x) + b1) + b2 for float32 rows x [rows][d]; out may be x."""
        rows = x.shape[0]
        if rows > self.max_rows:
            raise ValueError(f"{rows} rows: the buffers hold {self.max_rows}")
        self.rows = None      # (a pass that is refused halfway leaves nothing to go back from)
        ws = self.workspace
        xhat, pre = self._kept(rows)
        narrow, wide = self.scratch.narrow[:rows], self.scratch.wide[:rows]
        ad.layer_norm(x, self.gain, self.bias, narrow, None, self.rstd[:rows], xhat)
        ad.linear(narrow, self.w1, self.b1, ad.ACT_GELU, None, wide, None, pre, ws)
        ad.linear(wide, self.w2, self.b2, ad.ACT_NONE, x, out, None, None, ws)
        self.rows = rows

    def backward(self, dout, dx, dx_copy=None):
        """dx <- dL/dx from dout = dL/dout (float32 [rows][d]), for the rows of the last forward
        pass, and the parameters' gradients added to `grads`.  dx may be dout; dx_copy is a bf16 copy of
        dx.  A refused pass adds nothing."""
        rows = dout.shape[0]
        if rows != self.rows:
            raise ValueError(f"{rows} rows, but the last forward pass had {self.rows}")
        self._rows("dout", dout, rows, torch.float32, torch.bfloat16)
        self._rows("dx", dx, rows, torch.float32, torch.bfloat16)
        if dx_copy is not None:
            self._rows("dx_copy", dx_copy, rows, torch.bfloat16)
        ws = self.workspace
        xhat, pre = self._kept(rows)
        ggain, gbias, gw1, gb1, gw2, gb2 = self.grads
        narrow, act, dpre = (t[:rows] for t in (self.scratch.narrow, self.scratch.wide, self.scratch.wide2))
        narrow.copy_(dout)    # the products' operand in bf16
        ad.linear_dgrad(narrow, self.w2, ad.ACT_GELU, None, pre, dpre, act, ws)
        ad.linear_wgrad(narrow, act, None, None, None, gw2, gb2, ws, accumulate=True)
        ad.linear_wgrad(dpre, None, xhat, self.gain, self.bias, gw1, gb1, ws, accumulate=True)
        ad.linear_dgrad(dpre, self.w1, ad.ACT_NONE, None, None, narrow, None, ws)     # dL/dLN(x)
        ad.layer_norm_backward(narrow, None, None, self.rstd[:rows], xhat, self.gain, dout, dx,
                               dx_copy, ggain, gbias, ws, accumulate=True)


class AttentionScratch:
    """What passes of attention sublayers over up to max_rows rows, max_keys key rows and max_batch sequences need
    only while they run: rows of width d and 3 d in bf16, and one workspace for every call.  Shared like Scratch."""

    def __init__(self, d: int, max_rows: int, max_keys: int, max_batch: int, device="cuda"):
        if d % 64:
            raise ValueError(f"width {d} is not a multiple of the heads' 64")
        empty = lambda *shape, dt=torch.bfloat16: torch.empty(*shape, dtype=dt, device=device)  # noqa: E731
        self.d, self.max_rows, self.max_keys, self.max_batch = d, max_rows, max_keys, max_batch
        self.narrow, self.narrow2 = empty(max_rows, d), empty(max_rows, d)
        self.wide, self.keys = empty(max_rows, 3 * d), empty(max_keys, 2 * d)
        need = ad.layer_norm_backward_workspace_size(max_rows, d)
        sizes = (ad.linear_workspace_size, ad.linear_dgrad_workspace_size, ad.linear_wgrad_workspace_size)
        for most, shapes in ((max_rows, ((3 * d, d), (d, d))), (max_keys, ((2 * d, d),))):
            for rows in range(64, most + 64, 64):
                need = max(need, *(size(rows, *shape) for shape in shapes for size in sizes))
        # attention's: a float for each row and head and 16 bytes for each 32 rows of a sequence; the keys'
        # parts of at most 512 workgroups of 32 rows (a call checks what it needs)
        need = max(need, 4 * (d // 64) * max_rows + 512 + 16 * max_batch * (max_rows // 32 + 1), 512 * 32 * 66 * 4)
        self.workspace = empty(need, dt=torch.uint8)


class _AttentionSublayer:
    """What self- and cross-attention share: LayerNorm before, the output projection with the residual behind."""

    def __init__(self, norm, w_o, b_o, max_rows: int, scratch: AttentionScratch):
        self.gain, self.bias = norm
        self.w_o, self.b_o = w_o, b_o
        self.d = d = w_o.shape[0]
        self.heads, self.max_rows, self.scratch, dev = d // 64, max_rows, scratch, w_o.device
        if scratch.d != d or scratch.max_rows < max_rows or scratch.workspace.device != dev:
            raise ValueError(f"scratch of width {scratch.d} for {scratch.max_rows} rows on {scratch.workspace.device}, "
                             f"expected {d} for {max_rows} on {dev}")
        empty = lambda *shape, dt=torch.bfloat16: torch.empty(*shape, dtype=dt, device=dev)  # noqa: E731
        self.rstd, self.xhat = empty(max_rows, dt=torch.float32), ad.Ckpt.empty(max_rows, d, dev)
        self.o, self.o_rest = empty(max_rows, d), empty(max_rows, d)
        self.lse = empty(self.heads * max_rows, dt=torch.float32)
        self.rows = None

    def zero_grads(self):
        for g in self.grads:
            g.zero_()

    def _kept(self, rows: int):
        return (ad.Ckpt(self.xhat.q[:rows], self.xhat.scale[:rows], self.d), self.rstd[:rows], self.o[:rows],
                self.o_rest[:rows], self.lse[:self.heads * rows].view(self.heads, rows))

    def _check(self, name: str, t, rows: int, *dtypes):
        """Refuses what a later call of the pass would refuse, before the first one has written."""
        if not t.is_cuda or t.get_device() != torch.cuda.current_device():
            raise ValueError(f"{name} is on {t.device}, not on the current GPU")
        if t.shape != (rows, self.d) or t.dtype not in dtypes:
            raise ValueError(f"{name} is {tuple(t.shape)} of {t.dtype}, expected {(rows, self.d)} of {dtypes}")
        ld, step = t.stride()
        if step != 1 or (rows > 1 and not self.d <= ld <= 1 << 22):
            raise ValueError(f"{name}: the columns of a row must be adjacent, and rows apart by at most 2^22")

    def _begin(self, x, out, batch, keys: int):
        rows = x.shape[0]
        if rows > self.max_rows:
            raise ValueError(f"{rows} rows: the buffers hold {self.max_rows}")
        self._check("x", x, rows, torch.float32)
        self._check("out", out, rows, torch.float32)
        if (batch.q_heads, batch.kv_heads) != (self.heads, self.heads):
            raise ValueError(f"the batch has {batch.q_heads} and {batch.kv_heads} heads, expected {self.heads}")
        need = max(ad.attention_workspace_size(batch, rows, keys), ad.attention_backward_workspace_size(batch, rows, keys))
        if need > self.scratch.workspace.nbytes:
            raise ValueError(f"attention over {batch.batch} sequences needs a workspace of {need} bytes, the scratch has "
                             f"{self.scratch.workspace.nbytes}")
        self.rows = None      # (a pass that is refused halfway leaves nothing to go back from)
        xhat, rstd, *_ = self._kept(rows)
        narrow = self.scratch.narrow[:rows]
        ad.layer_norm(x, self.gain, self.bias, narrow, None, rstd, xhat)
        return rows, narrow

    def _end(self, batch, rows: int, q, k, v, x, out):
        ws = self.scratch.workspace
        _, _, o, rest, lse = self._kept(rows)
        if not batch.covers:
            o.zero_()
        ad.attention(batch, q, k, v, o, lse, rest, ws)
        ad.linear(o, self.w_o, self.b_o, ad.ACT_NONE, x, out, None, None, ws)
        self.rows, self.batch = rows, batch

    def _start_back(self, dout, dx, dx_copy, gw_o, gb_o):
        """dL/do in scratch.narrow2, the output projection's gradients added."""
        rows = dout.shape[0]
        if rows != self.rows:
            raise ValueError(f"{rows} rows, but the last forward pass had {self.rows}")
        self._check("dout", dout, rows, torch.float32, torch.bfloat16)
        self._check("dx", dx, rows, torch.float32, torch.bfloat16)
        if dx_copy is not None:
            self._check("dx_copy", dx_copy, rows, torch.bfloat16)
        ws, s = self.scratch.workspace, self.scratch
        _, _, o, _, _ = self._kept(rows)
        narrow, do = s.narrow[:rows], s.narrow2[:rows]
        narrow.copy_(dout)    # the products' operand in bf16
        ad.linear_wgrad(narrow, o, None, None, None, gw_o, gb_o, ws, accumulate=True)
        ad.linear_dgrad(narrow, self.w_o, ad.ACT_NONE, None, None, do, None, ws)
        return rows, do

    def _finish_back(self, rows: int, dq, w, gw, gb, dout, dx, dx_copy, ggain, gbias):
        """From dq, the gradient of the projection w of the normalised rows."""
        ws = self.scratch.workspace
        xhat, rstd, *_ = self._kept(rows)
        narrow = self.scratch.narrow[:rows]
        ad.linear_wgrad(dq, None, xhat, self.gain, self.bias, gw, gb, ws, accumulate=True)
        ad.linear_dgrad(dq, w, ad.ACT_NONE, None, None, narrow, None, ws)       # dL/dLN(x)
        ad.layer_norm_backward(narrow, None, None, rstd, xhat, self.gain, dout, dx, dx_copy, ggain, gbias, ws,
                               accumulate=True)


def _grads(params, dev):
    return [torch.zeros(p.shape, dtype=torch.float32, device=dev) for p in params]


class SelfAttention(_AttentionSublayer):
    """Buffers for up to max_rows rows.  params: (ln_gain [d], ln_bias [d], w_qkv [3d][d], b_qkv [3d], w_o [d][d],
    b_o [d]) on the GPU, matrices in bf16.  `grads` as in FeedForward.  Keys carry no bias (a constant added to
    every key changes no probability): its part of b_qkv's gradient is 0."""

    def __init__(self, params, max_rows: int, scratch: AttentionScratch):
        gain, bias, self.w_qkv, self.b_qkv, w_o, b_o = params
        super().__init__((gain, bias), w_o, b_o, max_rows, scratch)
        self.qkv = torch.empty(max_rows, 3 * self.d, dtype=torch.bfloat16, device=w_o.device)
        self.grads = _grads(params, w_o.device)

    def forward(self, x, batch: ad.Attention, out):
        """out <- x + the sublayer of float32 rows x [rows][d]; out may be x.  batch: the sequences' rows, the same
        for queries and keys."""
        rows, narrow = self._begin(x, out, batch, x.shape[0])
        qkv, d = self.qkv[:rows], self.d
        ad.linear(narrow, self.w_qkv, self.b_qkv, ad.ACT_NONE, None, qkv, None, None, self.scratch.workspace)
        self._end(batch, rows, qkv[:, :d], qkv[:, d:2 * d], qkv[:, 2 * d:], x, out)

    def backward(self, dout, dx, dx_copy=None):
        """dx <- dL/dx from dout = dL/dout for the rows of the last forward pass, and the parameters'
        gradients added to `grads`.  dx may be dout; dx_copy is a bf16 copy of dx."""
        ggain, gbias, gw, gb, gw_o, gb_o = self.grads
        rows, do = self._start_back(dout, dx, dx_copy, gw_o, gb_o)
        _, _, o, rest, lse = self._kept(rows)
        d, qkv, dqkv = self.d, self.qkv[:rows], self.scratch.wide[:rows]
        cut = lambda t: (t[:, :d], t[:, d:2 * d], t[:, 2 * d:])  # noqa: E731
        if not self.batch.covers:      # (rows of no sequence are not written, and have no part in sums over rows)
            dqkv.zero_()
        ad.attention_backward(self.batch, *cut(qkv), o, rest, lse, do, None, *cut(dqkv), self.scratch.workspace)
        self._finish_back(rows, dqkv, self.w_qkv, gw, gb, dout, dx, dx_copy, ggain, gbias)
        gb[d:2 * d].zero_()


class CrossAttention(_AttentionSublayer):
    """Buffers for up to max_rows rows and max_keys rows of encoder states.  params: (ln_gain [d], ln_bias [d],
    w_xq [d][d], b_xq [d], w_xkv [2d][d], b_xkv [2d], w_xo [d][d], b_xo [d]).  The encoder is frozen: its states get no
    gradient; the key part of b_xkv's gradient is 0."""

    def __init__(self, params, max_rows: int, max_keys: int, scratch: AttentionScratch):
        gain, bias, self.w_q, self.b_q, self.w_kv, self.b_kv, w_o, b_o = params
        super().__init__((gain, bias), w_o, b_o, max_rows, scratch)
        if scratch.max_keys < max_keys:
            raise ValueError(f"scratch for {scratch.max_keys} keys, expected {max_keys}")
        empty = lambda *shape: torch.empty(*shape, dtype=torch.bfloat16, device=w_o.device)  # noqa: E731
        self.max_keys = max_keys
        self.q, self.kv = empty(max_rows, self.d), empty(max_keys, 2 * self.d)
        self.grads = _grads(params, w_o.device)

    def forward(self, x, enc, batch: ad.Attention, out, xq=None):
        """out <- x + the sublayer of float32 rows x and bf16 encoder states enc [keys][d]; out may be x.  xq
        (float32 [rows][d], optional) receives the query rows, the alignment objective's input."""
        keys, d = enc.shape[0], self.d
        if keys > self.max_keys:
            raise ValueError(f"{keys} keys: the buffers hold {self.max_keys}")
        self._check("enc", enc, keys, torch.bfloat16)
        if xq is not None:
            self._check("xq", xq, x.shape[0], torch.float32)
        rows, narrow = self._begin(x, out, batch, keys)
        q, kv, ws = self.q[:rows], self.kv[:keys], self.scratch.workspace
        if xq is None:
            ad.linear(narrow, self.w_q, self.b_q, ad.ACT_NONE, None, q, None, None, ws)
        else:
            ad.linear(narrow, self.w_q, self.b_q, ad.ACT_NONE, None, xq, None, None, ws)
            q.copy_(xq)
        ad.linear(enc, self.w_kv, self.b_kv, ad.ACT_NONE, None, kv, None, None, ws)
        self._end(batch, rows, q, kv[:, :d], kv[:, d:], x, out)
        self.enc = enc

    def backward(self, dout, dx, dx_copy=None, dxq=None):
        """As SelfAttention.backward; dxq (float32 or bf16 [rows][d], optional) is the objective's gradient for the
        query rows, which is added to attention's.  enc must still hold the last forward pass's states."""
        ggain, gbias, gw_q, gb_q, gw_kv, gb_kv, gw_o, gb_o = self.grads
        if dxq is not None:
            self._check("dxq", dxq, dout.shape[0], torch.float32, torch.bfloat16)
        rows, do = self._start_back(dout, dx, dx_copy, gw_o, gb_o)
        _, _, o, rest, lse = self._kept(rows)
        d, keys, s = self.d, self.enc.shape[0], self.scratch
        q, kv, dq, dkv = self.q[:rows], self.kv[:keys], s.wide[:rows, :d], s.keys[:keys]
        if not self.batch.covers:      # (rows of no sequence are not written, and have no part in sums over rows)
            dq.zero_()
            dkv.zero_()
        ad.attention_backward(self.batch, q, kv[:, :d], kv[:, d:], o, rest, lse, do, dxq, dq, dkv[:, :d], dkv[:, d:],
                              s.workspace)
        ad.linear_wgrad(dkv, self.enc, None, None, None, gw_kv, gb_kv, s.workspace, accumulate=True)
        gb_kv[:d].zero_()
        self._finish_back(rows, dq, self.w_q, gw_q, gb_q, dout, dx, dx_copy, ggain, gbias)


class DraftBlock:
    """A decoder block of the draft: self-attention, cross-attention, feed-forward.  params: a model layer's 20 tensors
    in ad_model_create's order, matrices in bf16 (the tensors themselves are read, so that an optimizer may write
    them).  `grads` in the same order."""

    def __init__(self, params, max_rows: int, max_keys: int, max_batch: int):
        params = list(params)
        if len(params) != 20:
            raise ValueError(f"{len(params)} parameters, expected a layer's 20")
        f, d = params[16].shape
        dev = params[16].device
        self.params, self.d, self.max_rows = params, d, max_rows
        scratch = AttentionScratch(d, max_rows, max_keys, max_batch, dev)
        self.self_attention = SelfAttention(params[0:6], max_rows, scratch)
        self.cross_attention = CrossAttention(params[6:14], max_rows, max_keys, scratch)
        self.feed_forward = FeedForward(params[14:20], max_rows, Scratch(d, f, max_rows, dev))
        self._parts = (self.self_attention, self.cross_attention, self.feed_forward)
        self.grads = self.self_attention.grads + self.cross_attention.grads + self.feed_forward.grads

    def zero_grads(self):
        for g in self.grads:
            g.zero_()

    def forward(self, x, enc, self_batch: ad.Attention, cross_batch: ad.Attention, out, xq=None):
        """out <- the block of float32 rows x [rows][d] and encoder states enc (bf16 [keys][d]); out may be x.  After a
        refused pass there is nothing to go back from."""
        for part in self._parts:       # (one that is refused halfway has new rows in some and old ones in others)
            part.rows = None
        self.self_attention.forward(x, self_batch, out)
        self.cross_attention.forward(out, enc, cross_batch, out, xq)
        self.feed_forward.forward(out, out)

    def backward(self, dout, dx, dxq=None):
        """dx <- dL/dx (float32) from dout = dL/dout, and the parameters' gradients added; dx may be dout.  A refused pass
        adds nothing."""
        rows = dout.shape[0]
        for part in self._parts:
            if part.rows != rows:
                raise ValueError(f"{rows} rows, but the last forward pass had {part.rows}")
        self.feed_forward._rows("dout", dout, rows, torch.float32, torch.bfloat16)
        self.feed_forward._rows("dx", dx, rows, torch.float32, torch.bfloat16)
        if dxq is not None:
            self.cross_attention._check("dxq", dxq, rows, torch.float32, torch.bfloat16)
        self.feed_forward.backward(dout, dx)
        self.cross_attention.backward(dx, dx, dxq=dxq)
        self.self_attention.backward(dx, dx)


class AdamW:
    """AdamW over a model's parameters (the paper's recipe: learning rate 1e-3, weight decay 0.01 on matrices, gradients
    clipped to norm 1).  params: bf16 or float32 tensors on the GPU, which a step writes; grads: tensors of their
    shapes, float32 or bf16.  bf16 parameters have float32 ones here, of which they are the rounded copies.
    state: "f32" or "8bit".  Learning rate, step count and norm live on the GPU, so that a step can be captured
    into a graph with the pass that makes its gradients.  The float32 parameters are made once: a step overwrites values
    that were put into bf16 ones since, unless read_params() is called.  state_dict() and load_state_dict() carry a
    training run over."""

    def __init__(self, params, grads, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.01,
                 max_norm: float = 1.0, state: str = "f32", seed: int = 0):
        if state not in ("f32", "8bit"):
            raise ValueError(f"state {state!r}, expected 'f32' or '8bit'")
        if not params or len(params) != len(grads):
            raise ValueError(f"{len(params)} parameters and {len(grads)} gradients")
        # (what a call of the step would refuse: the norm has counted the step by then)
        beta1, beta2 = betas
        if not (0.0 <= beta1 < 1.0 and 0.0 <= beta2 < 1.0):
            raise ValueError(f"betas {betas}, expected two numbers in [0, 1)")
        for name, x in (("lr", lr), ("eps", eps), ("weight_decay", weight_decay), ("max_norm", max_norm)):
            self._number(name, x)
        dev = params[0].device
        make = lambda n, dt: torch.zeros(n, dtype=dt, device=dev)  # noqa: E731
        self.params, self.grads, self.betas, self.eps, self.max_norm, self.seed = params, grads, betas, eps, max_norm, seed
        self.master = [p if p.dtype is torch.float32 else p.float() for p in params]
        eight = state == "8bit"
        states = dict(m=[make(p.numel(), torch.int8 if eight else torch.float32) for p in params],
                      v=[make(p.numel(), torch.uint8 if eight else torch.float32) for p in params])
        if eight:
            for name in ("m_scale", "v_scale"):
                states[name] = [make(-(-p.numel() // 128), torch.float32) for p in params]
        self.state, self._kept = state, states
        decay = [weight_decay if p.dim() > 1 else 0.0 for p in params]
        # (copies: float32 parameters are their own)
        groups = ([i for i, p in enumerate(params) if p.dtype is torch.float32],
                  [i for i, p in enumerate(params) if p.dtype is not torch.float32])
        pick = lambda x, at: [x[i] for i in at]  # noqa: E731
        self._all = ad.OptTensors(grads=grads)
        self._parts = [ad.OptTensors(params=pick(self.master, at), grads=pick(grads, at), weight_decay=pick(decay, at),
                                     copies=pick(params, at) if k else None,
                                     **{name: pick(x, at) for name, x in states.items()})
                       for k, at in enumerate(groups) if at]
        self._groups = [at for at in groups if at]
        self._workspace = make(max(ad.grad_norm_workspace_size(self._all), 1), torch.uint8)
        self.lr = torch.full((1,), lr, dtype=torch.float32, device=dev)
        self.steps = make(1, torch.int32)          # steps taken
        self.norm = make(2, torch.float32)         # the last gradients' norm, and the factor they were clipped with

    @staticmethod
    def _number(name: str, x: float):
        if not 0.0 <= x <= torch.finfo(torch.float32).max:
            raise ValueError(f"{name} {x}, expected a finite number of float32 that is not negative")

    def set_lr(self, lr: float):
        self._number("lr", lr)
        self.lr.fill_(lr)

    def step(self):
        """One step.  Gradients whose norm is not finite leave everything as it is."""
        ad.grad_norm(self._all, self.max_norm, self.norm, self._workspace, step=self.steps)
        for k, part in enumerate(self._parts):
            ad.adamw(part, self.lr, self.steps, *self.betas, self.eps, self.seed + k, self.norm[1:])

    def _states(self):
        """What a step reads and writes besides the parameters' copies: lists of tensors by name."""
        return dict(master=self.master, **self._kept)

    @torch.no_grad()
    def read_params(self):
        """Takes the parameters as they are now, after new values were put into them; the states stay."""
        for p, master in zip(self.params, self.master):
            if master is not p:
                master.copy_(p)

    def state_dict(self):
        """Copies of everything that the next step hangs on: the float32 parameters, the states as they are held, step
        count, learning rate and seed."""
        return dict(state=self.state, seed=self.seed, steps=self.steps.clone(), lr=self.lr.clone(),
                    **{name: [t.clone() for t in x] for name, x in self._states().items()})

    @torch.no_grad()
    def load_state_dict(self, saved):
        """Goes on from state_dict() of an optimizer over parameters of the same shapes, and writes the parameters.  In
        place: a captured step goes on with them (and with the seed that it was captured with).  What does not fit is
        refused as a whole."""
        if saved["state"] != self.state:
            raise ValueError(f"states in {saved['state']!r}, expected {self.state!r}")
        pairs = [(name, t, u) for name, x in self._states().items() for t, u in zip(x, saved[name], strict=True)]
        for name, t, u in (*pairs, ("steps", self.steps, saved["steps"]), ("lr", self.lr, saved["lr"])):
            if t.shape != u.shape or t.dtype is not u.dtype:
                raise ValueError(f"{name}: {tuple(u.shape)} of {u.dtype}, expected {tuple(t.shape)} of {t.dtype}")
        seed = int(saved["seed"])
        for _, t, u in (*pairs, ("", self.steps, saved["steps"]), ("", self.lr, saved["lr"])):
            t.copy_(u)
        for p, master in zip(self.params, self.master):
            if master is not p:
                p.copy_(master)
        self.seed = seed

    def states(self):
        """(m, v) of every parameter as float32 tensors of its shape."""
        out = [None] * len(self.params)
        for part, at in zip(self._parts, self._groups):
            m, v = (torch.empty(part.numel, dtype=torch.float32, device=self.lr.device) for _ in range(2))
            ad.opt_state(part, m, v)
            sizes = [self.params[i].numel() for i in at]
            for i, a, b in zip(at, m.split(sizes), v.split(sizes)):
                out[i] = (a.view(self.params[i].shape), b.view(self.params[i].shape))
        return out
