"""The feed-forward sublayer of the draft block, forward and backward, through the C-ABI.

    out = x + W2 GELU(W1 LN(x) + b1) + b2

(the third sublayer of the decoder's blocks; its parameters are a model's ln3_g, ln3_b, w_1,
b_1, w_2 and b_2).  What the backward pass needs is kept in 8 bits: the normalised rows and the
pre-activation, 1.03 bytes a value in place of two LayerNorm outputs, a pre-activation and a
GELU output in bf16.  Like Session it owns its buffers and only calls libad entry points.
"""
from __future__ import annotations

import torch

from . import ad


class FeedForward:
    """Buffers for up to max_rows rows.  params: (ln_gain [d], ln_bias [d], w1 [f][d], b1 [f],
    w2 [d][f], b2 [d]) on the GPU, w1 and w2 in bf16.  Gradients are float32 tensors of the same
    shapes in `grads`, in the same order; backward adds to them (zero_grads clears them)."""

    def __init__(self, params, max_rows: int):
        self.gain, self.bias, self.w1, self.b1, self.w2, self.b2 = params
        self.f, self.d = self.w1.shape
        d, f, dev = self.d, self.f, self.w1.device
        empty = lambda *shape, dt=torch.float32: torch.empty(*shape, dtype=dt, device=dev)  # noqa: E731
        self.max_rows = max_rows
        self.mean, self.rstd = empty(max_rows), empty(max_rows)
        self.xhat = ad.Ckpt.empty(max_rows, d, dev)
        self.pre = ad.Ckpt.empty(max_rows, f, dev)
        self.narrow, self.wide = empty(max_rows, d, dt=torch.bfloat16), empty(max_rows, f, dt=torch.bfloat16)
        self.wide2 = empty(max_rows, f, dt=torch.bfloat16)
        self.dnarrow = empty(max_rows, d, dt=torch.bfloat16)
        self.grads = [torch.zeros(p.shape, dtype=torch.float32, device=dev) for p in params]
        self.rows = None
        # One workspace for every call, large enough for any number of rows up to max_rows (a captured
        # pass keeps its address).  What a call needs changes with its rows at multiples of 64 only,
        # and the LayerNorm's grows with them.
        need = ad.layer_norm_backward_workspace_size(max_rows, d)
        for rows in range(64, max_rows + 64, 64):
            need = max(need, *(size(rows, *shape) for shape in ((d, f), (f, d)) for size in
                               (ad.linear_workspace_size, ad.linear_dgrad_workspace_size,
                                ad.linear_wgrad_workspace_size)))
        self.workspace = empty(max(need, 1), dt=torch.uint8)

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
        ad.layer_norm(x, self.gain, self.bias, self.narrow[:rows], self.mean[:rows], self.rstd[:rows], xhat)
        ad.linear(self.narrow[:rows], self.w1, self.b1, ad.ACT_GELU, None, self.wide[:rows], None, pre, ws)
        ad.linear(self.wide[:rows], self.w2, self.b2, ad.ACT_NONE, x, out, None, None, ws)
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
        dlow, act, dpre = self.dnarrow[:rows], self.wide[:rows], self.wide2[:rows]
        dlow.copy_(dout)      # the products' operand in bf16
        ad.linear_dgrad(dlow, self.w2, ad.ACT_GELU, None, pre, dpre, act, ws)
        ad.linear_wgrad(dlow, act, None, None, None, gw2, gb2, ws, accumulate=True)
        ad.linear_wgrad(dpre, None, xhat, self.gain, self.bias, gw1, gb1, ws, accumulate=True)
        ad.linear_dgrad(dpre, self.w1, ad.ACT_NONE, None, None, self.narrow[:rows], None, ws)
        ad.layer_norm_backward(self.narrow[:rows], None, None, self.rstd[:rows], xhat, self.gain, dout, dx,
                               dx_copy, ggain, gbias, ws, accumulate=True)
