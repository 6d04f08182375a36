"""The feed-forward sublayer of the draft block, forward and backward, through the C-ABI.

    out = x + W2 GELU(W1 LN(x) + b1) + b2

(the third sublayer of the decoder's blocks; its parameters are a model's ln3_g, ln3_b, w_1,
b_1, w_2 and b_2).  From the forward to the backward pass a sublayer keeps the normalised rows and the
pre-activation in 8 bits: 1.03 (d + f) bytes a row and 4 for LayerNorm's factor, where the LayerNorm
output, the pre-activation and GELU's output in bf16 would be 2 d + 4 f.  A running pass also needs
2 d + 4 f bytes a row and a workspace (Scratch), which sublayers can share.  Like Session they own
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
