"""ctypes binding over libad.so (the C-ABI declared in include/ad.h).

Argument marshalling only: every computation of the verify step runs in the library's
HIP kernels.  torch supplies device memory and the current stream.  Importing this
module loads the library; a missing library is an error, never a fallback.
"""
from __future__ import annotations

import ctypes
import os

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libad.so")

AD_F32, AD_BF16 = 0, 1
AD_PADDED, AD_PACKED = 0, 1
AD_ERR_LENGTH, AD_ERR_PAGE, AD_ERR_TOKEN, AD_ERR_FRAMES, AD_ERR_NONFINITE = 1, 2, 4, 8, 16
AD_ERR_TREE = 32
STATUS = {0: "AD_OK", -1: "AD_EINVAL", -2: "AD_ERANGE", -3: "AD_ENOSPACE", -4: "AD_EHIP",
          -5: "AD_EUNSUPPORTED"}

ACT_NONE, ACT_GELU = 0, 1
STATE_F, STATE_8 = 0, 1

_i32 = ctypes.c_int32
_ptr = ctypes.c_void_p
_size = ctypes.c_size_t


class ModelDesc(ctypes.Structure):
    _fields_ = [("n_layers", _i32), ("d_model", _i32), ("n_heads", _i32), ("d_ffn", _i32),
                ("vocab", _i32), ("max_pos", _i32), ("max_frames", _i32), ("dtype", _i32)]


class KV(ctypes.Structure):
    _fields_ = [("pool", _ptr), ("num_pages", _i32), ("pages_per_seq", _i32),
                ("kv_len", _ptr), ("block_table", _ptr)]


class Cross(ctypes.Structure):
    _fields_ = [("data", _ptr), ("frames_cap", _i32), ("enc_len", _ptr), ("enc_off", _ptr)]


class Step(ctypes.Structure):
    _fields_ = [("batch", _i32), ("layout", _i32), ("k_max", _i32), ("rows", _i32),
                ("tokens", _ptr), ("k", _ptr), ("cu_rows", _ptr), ("kv", KV), ("cross", Cross),
                ("accept_len", _ptr), ("out_tokens", _ptr), ("out_greedy", _ptr),
                ("out_logits", _ptr), ("out_hidden", _ptr), ("out_margin", _ptr),
                ("err_flag", _ptr), ("workspace", _ptr), ("workspace_bytes", _size),
                ("anchor_layer", _i32), ("out_anchor", _ptr), ("out_anchor_peak", _ptr),
                ("in_rows", _ptr), ("cross_window", _ptr), ("tap_layers", _i32 * 3),
                ("out_taps", _ptr), ("parents", _ptr), ("out_path", _ptr),
                ("out_xq", _ptr)]


class Mat(ctypes.Structure):
    _fields_ = [("data", _ptr), ("ld", ctypes.c_int64), ("dtype", _i32)]


class CkptView(ctypes.Structure):
    _fields_ = [("q", _ptr), ("scale", _ptr)]


class AttnView(ctypes.Structure):
    _fields_ = [("batch", _i32), ("q_heads", _i32), ("kv_heads", _i32), ("q_rows", _i32), ("k_rows", _i32),
                ("q_max", _i32), ("k_max", _i32), ("causal", _i32), ("cu_q", _ptr), ("cu_k", _ptr),
                ("q_len", _ptr), ("k_len", _ptr), ("window", _ptr), ("err_flag", _ptr)]


class OptTensor(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int64), ("param", _ptr), ("copy", _ptr), ("grad", _ptr), ("m", _ptr), ("v", _ptr),
                ("m_scale", _ptr), ("v_scale", _ptr), ("weight_decay", ctypes.c_double), ("param_dtype", _i32),
                ("grad_dtype", _i32), ("state", _i32)]


class AdamwArgs(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("step", _i32), ("seed", ctypes.c_uint32), ("lr_at", _ptr),
                ("step_at", _ptr), ("grad_scale", _ptr)]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run paper_2608_12703_amd.build.build()")
    lib = ctypes.CDLL(LIB_PATH)
    _mat, _ckpt = ctypes.POINTER(Mat), ctypes.POINTER(CkptView)
    _attn, _opt = ctypes.POINTER(AttnView), ctypes.POINTER(OptTensor)
    sig = {
        "ad_last_error": (ctypes.c_char_p, []),
        "ad_model_param_count": (_i32, [ctypes.POINTER(ModelDesc)]),
        "ad_model_create": (_i32, [ctypes.POINTER(ModelDesc), ctypes.POINTER(_ptr), _i32,
                                   ctypes.POINTER(_ptr)]),
        "ad_model_destroy": (_i32, [_ptr]),
        "ad_model_pack_size": (_i32, [_ptr, ctypes.POINTER(_size)]),
        "ad_model_pack": (_i32, [_ptr, _ptr, _size, _ptr]),
        "ad_workspace_size": (_i32, [_ptr, _i32, _i32, _i32, ctypes.POINTER(_size)]),
        "ad_cross_kv_prefill": (_i32, [_ptr, _ptr, ctypes.POINTER(Cross), _ptr]),
        "ad_verify_step": (_i32, [_ptr, ctypes.POINTER(Step), _ptr]),
        "ad_verify_step_static": (_i32, [_ptr, ctypes.POINTER(Step), _ptr]),
        "ad_kv_commit": (_i32, [_ptr, _ptr, _i32, _ptr]),
        "ad_kv_commit_tree": (_i32, [_ptr, _ptr, _ptr, _ptr, _i32, _i32, _ptr]),
        "ad_anchordraft_loss_workspace_size": (_i32, [_ptr, _i32, _i32, ctypes.POINTER(_size)]),
        "ad_anchordraft_loss": (_i32, [_ptr, _ptr, _i32, _i32, _i32, _ptr, _ptr, ctypes.c_float,
                                       ctypes.c_float, _ptr, _ptr, _ptr, _ptr, _ptr, _ptr, _ptr,
                                       _ptr, _ptr, _ptr, _ptr, _size, _ptr]),
        "ad_draft_heads_workspace_size": (_i32, [_ptr, _i32, _i32, ctypes.POINTER(_size)]),
        "ad_draft_heads": (_i32, [_ptr, _ptr, _i32, _ptr, _i32, _i32, _ptr, _ptr, _ptr, _i32,
                                  _ptr, _ptr, _size, _ptr]),
        "ad_kv_import": (_i32, [_ptr, ctypes.POINTER(KV), _i32, _ptr, _i32, _ptr, _ptr]),
        "ad_draft_input_workspace_size": (_i32, [_ptr, _i32, ctypes.POINTER(_size)]),
        "ad_draft_input": (_i32, [_ptr, _ptr, _ptr, _ptr, _ptr, _i32, _ptr, _ptr, _i32, _i32, _ptr,
                                  _ptr, _i32, _ptr, _ptr, _i32, _ptr, _ptr, _ptr, _i32, _ptr, _ptr,
                                  _ptr, _size, _ptr]),
        "ad_kv_export": (_i32, [_ptr, ctypes.POINTER(KV), _i32, _ptr, _i32, _ptr, _ptr]),
        "ad_ckpt_ld": (_i32, [_i32]),
        "ad_ckpt_pack": (_i32, [_i32, _i32, _mat, _ckpt, _ptr]),
        "ad_ckpt_unpack": (_i32, [_i32, _i32, _ckpt, _i32, _mat, _ptr]),
        "ad_layer_norm": (_i32, [_i32, _i32, _mat, _ptr, _ptr, _i32, _mat, _ptr, _ptr, _ckpt, _ptr]),
        "ad_layer_norm_backward_workspace_size": (_i32, [_i32, _i32, ctypes.POINTER(_size)]),
        "ad_layer_norm_backward": (_i32, [_i32, _i32, _mat, _mat, _ptr, _ptr, _ckpt, _ptr, _i32, _mat, _mat,
                                          _mat, _ptr, _ptr, _i32, _ptr, _size, _ptr]),
        "ad_linear_workspace_size": (_i32, [_i32, _i32, _i32, ctypes.POINTER(_size)]),
        "ad_linear": (_i32, [_i32, _i32, _i32, _mat, _mat, _ptr, _i32, _i32, _mat, _mat, _mat, _ckpt, _ptr,
                             _size, _ptr]),
        "ad_linear_dgrad_workspace_size": (_i32, [_i32, _i32, _i32, ctypes.POINTER(_size)]),
        "ad_linear_dgrad": (_i32, [_i32, _i32, _i32, _mat, _mat, _i32, _mat, _ckpt, _mat, _mat, _ptr, _size,
                                   _ptr]),
        "ad_linear_wgrad_workspace_size": (_i32, [_i32, _i32, _i32, ctypes.POINTER(_size)]),
        "ad_linear_wgrad": (_i32, [_i32, _i32, _i32, _mat, _mat, _ckpt, _ptr, _ptr, _i32, _mat, _ptr, _i32,
                                   _ptr, _size, _ptr]),
        "ad_attention_workspace_size": (_i32, [_attn, ctypes.POINTER(_size)]),
        "ad_attention": (_i32, [_attn, _mat, _mat, _mat, _mat, _mat, _ptr, _ptr, _size, _ptr]),
        "ad_attention_backward_workspace_size": (_i32, [_attn, ctypes.POINTER(_size)]),
        "ad_attention_backward": (_i32, [_attn, _mat, _mat, _mat, _mat, _mat, _ptr, _mat, _mat, _mat, _mat, _mat,
                                         _ptr, _size, _ptr]),
        "ad_adamw": (_i32, [_opt, _i32, ctypes.POINTER(AdamwArgs), _ptr]),
        "ad_opt_state": (_i32, [_opt, _i32, _ptr, _ptr, _ptr]),
        "ad_grad_norm_workspace_size": (_i32, [_opt, _i32, ctypes.POINTER(_size)]),
        "ad_grad_norm": (_i32, [_opt, _i32, ctypes.c_double, _ptr, _ptr, _ptr, _size, _ptr]),
        "ad_profile_enable": (_i32, [_ptr, _i32, _i32]),
        "ad_profile_read": (_i32, [_ptr, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(_i32)]),
    }
    for name, (res, args) in sig.items():
        f = getattr(lib, name)
        f.restype, f.argtypes = res, args
    return lib


LIB = _load()
EXPORTS = ("ad_last_error", "ad_model_param_count", "ad_model_create", "ad_model_destroy",
           "ad_model_pack_size", "ad_model_pack",
           "ad_workspace_size", "ad_cross_kv_prefill", "ad_verify_step", "ad_verify_step_static",
           "ad_kv_commit", "ad_kv_commit_tree",
           "ad_draft_heads_workspace_size", "ad_draft_heads", "ad_kv_import", "ad_kv_export",
           "ad_draft_input_workspace_size", "ad_draft_input",
           "ad_anchordraft_loss_workspace_size", "ad_anchordraft_loss",
           "ad_ckpt_ld", "ad_ckpt_pack", "ad_ckpt_unpack", "ad_layer_norm",
           "ad_layer_norm_backward_workspace_size", "ad_layer_norm_backward",
           "ad_linear_workspace_size", "ad_linear", "ad_linear_dgrad_workspace_size", "ad_linear_dgrad",
           "ad_linear_wgrad_workspace_size", "ad_linear_wgrad",
           "ad_attention_workspace_size", "ad_attention", "ad_attention_backward_workspace_size",
           "ad_attention_backward", "ad_adamw", "ad_opt_state", "ad_grad_norm_workspace_size", "ad_grad_norm",
           "ad_profile_enable", "ad_profile_read")
PROF_CROSS_ATTN, PROF_SELF_ATTN, PROF_GEMM, PROF_LM_HEAD, PROF_XQ_CROSS, PROF_XQ, PROF_ANCHOR = 1, 2, 3, 4, 5, 6, 7


class ADError(RuntimeError):
    def __init__(self, what: str, status: int):
        self.status = status
        msg = LIB.ad_last_error().decode()
        super().__init__(f"{what}: {STATUS.get(status, status)}: {msg}")


def check(status: int, what: str):
    if status != 0:
        raise ADError(what, status)


def ptr(t) -> int | None:
    """Device address of a tensor (None for None)."""
    return None if t is None else t.data_ptr()


# the current stream's handle without a Stream object around it (3 us a call, as long as a launch)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def stream_handle(stream=None) -> int:
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None:
        return _raw_stream(torch.cuda.current_device())
    return torch.cuda.current_stream().cuda_stream


def model_desc(cfg, max_pos=448, max_frames=1500) -> ModelDesc:
    return ModelDesc(cfg.n_layers, cfg.d_model, cfg.n_heads, cfg.d_ffn, cfg.vocab, max_pos,
                     max_frames, AD_BF16 if cfg.dtype == "bf16" else AD_F32)


def param_count(cfg) -> int:
    return LIB.ad_model_param_count(ctypes.byref(model_desc(cfg)))


class Model:
    """A model handle over caller-owned device parameters (kept alive here)."""

    def __init__(self, cfg, params: list, max_frames: int = 1500):
        self.cfg = cfg
        self.params = params
        self.desc = model_desc(cfg, max_pos=cfg.max_pos, max_frames=max_frames)
        arr = (_ptr * len(params))(*[p.data_ptr() for p in params])
        h = _ptr()
        check(LIB.ad_model_create(ctypes.byref(self.desc), arr, len(params), ctypes.byref(h)),
              "ad_model_create")
        self.handle = h

    def workspace_size(self, rows: int, batch: int, k_max: int) -> int:
        n = _size()
        check(LIB.ad_workspace_size(self.handle, rows, batch, k_max, ctypes.byref(n)),
              "ad_workspace_size")
        return n.value

    def pack_size(self) -> int:
        n = _size()
        check(LIB.ad_model_pack_size(self.handle, ctypes.byref(n)), "ad_model_pack_size")
        return n.value

    def pack(self, buffer, stream=None):
        """Tile the weights into `buffer` (a device tensor of at least pack_size() bytes,
        kept alive here), or return to the row-major parameters with buffer=None."""
        check(LIB.ad_model_pack(self.handle, ptr(buffer), 0 if buffer is None else
                                buffer.numel() * buffer.element_size(), stream_handle(stream)),
              "ad_model_pack")
        self.packed = buffer

    def draft_heads_workspace_size(self, n_heads: int, batch: int) -> int:
        n = _size()
        check(LIB.ad_draft_heads_workspace_size(self.handle, n_heads, batch, ctypes.byref(n)),
              "ad_draft_heads_workspace_size")
        return n.value

    def close(self):
        if getattr(self, "handle", None):
            LIB.ad_model_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def cross_kv_prefill(model: Model, enc, cross: Cross, stream=None):
    check(LIB.ad_cross_kv_prefill(model.handle, ptr(enc), ctypes.byref(cross),
                                  stream_handle(stream)), "ad_cross_kv_prefill")


def verify_step(model: Model, step: Step, stream=None):
    check(LIB.ad_verify_step(model.handle, ctypes.byref(step), stream_handle(stream)),
          "ad_verify_step")


def verify_step_static(model: Model, step: Step, stream=None):
    """ad_verify_step in the library's static scratch (step.workspace is ignored)."""
    check(LIB.ad_verify_step_static(model.handle, ctypes.byref(step), stream_handle(stream)),
          "ad_verify_step_static")


def kv_commit(kv_len, accept_len, batch: int, stream=None):
    check(LIB.ad_kv_commit(ptr(kv_len), ptr(accept_len), batch, stream_handle(stream)),
          "ad_kv_commit")


def kv_commit_tree(model: Model, kv: KV, accept_len, path, path_stride: int, batch: int,
                   stream=None):
    check(LIB.ad_kv_commit_tree(model.handle, ctypes.byref(kv), ptr(accept_len), ptr(path),
                                path_stride, batch, stream_handle(stream)), "ad_kv_commit_tree")


def anchordraft_loss_workspace_size(model: Model, batch: int, rows_per_seq: int) -> int:
    n = _size()
    check(LIB.ad_anchordraft_loss_workspace_size(model.handle, batch, rows_per_seq, ctypes.byref(n)),
          "ad_anchordraft_loss_workspace_size")
    return n.value


def anchordraft_loss(model: Model, cross, layer: int, batch: int, rows_per_seq: int, xq, center,
                     sigma: float, lam: float, logits, targets, feat, feat_target, out_terms,
                     out_row, out_dxq, out_dlogits, out_dfeat, err_flag, workspace, stream=None):
    """The AnchorDraft objective (ad.h: ad_anchordraft_loss); cross is a Cross struct or
    None, array arguments are device tensors or None."""
    check(LIB.ad_anchordraft_loss(
        model.handle, None if cross is None else ctypes.byref(cross), layer, batch, rows_per_seq,
        ptr(xq), ptr(center), sigma, lam, ptr(logits), ptr(targets), ptr(feat), ptr(feat_target),
        ptr(out_terms), ptr(out_row), ptr(out_dxq), ptr(out_dlogits), ptr(out_dfeat), ptr(err_flag),
        ptr(workspace), 0 if workspace is None else workspace.numel() * workspace.element_size(),
        stream_handle(stream)), "ad_anchordraft_loss")


def draft_heads(model: Model, heads_w, n_heads: int, hidden, layout: int, k_max: int, cu_rows,
                accept_len, out_tokens, batch: int, next_tokens, workspace, stream=None):
    check(LIB.ad_draft_heads(model.handle, ptr(heads_w), n_heads, ptr(hidden), layout, k_max,
                             ptr(cu_rows), ptr(accept_len), ptr(out_tokens), batch,
                             ptr(next_tokens), ptr(workspace), workspace.numel(),
                             stream_handle(stream)), "ad_draft_heads")


def draft_input_workspace_size(model: Model, batch: int) -> int:
    n = _size()
    check(LIB.ad_draft_input_workspace_size(model.handle, batch, ctypes.byref(n)),
          "ad_draft_input_workspace_size")
    return n.value


def draft_input(model: Model, w_fuse, b_fuse, w_in, b_in, batch: int, taps, hidden, layout: int,
                k_max: int, cu_rows, accept_len, rows: int, feature, tokens, token_stride: int,
                token_index, anchor, enc_len, half_window: int, window, out, workspace, stream=None):
    check(LIB.ad_draft_input(model.handle, ptr(w_fuse), ptr(b_fuse), ptr(w_in), ptr(b_in), batch,
                             ptr(taps), ptr(hidden), layout, k_max, ptr(cu_rows), ptr(accept_len),
                             rows, ptr(feature), ptr(tokens), token_stride, ptr(token_index),
                             ptr(anchor), ptr(enc_len), half_window, ptr(window), ptr(out),
                             ptr(workspace), workspace.numel(), stream_handle(stream)),
          "ad_draft_input")


# ------------------------------------------------------------------ training operators
# Tensors carry their own shapes here, so the binding checks what the C-ABI cannot see: that
# they agree with each other, lie on the current device and have their columns side by side.

_DTYPE = {torch.float32: AD_F32, torch.bfloat16: AD_BF16}
_byref = ctypes.byref


# (a call with a tensor on the GPU needs no check that CUDA has started: 0.2 us of 7 each)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _device(name: str, t) -> int:
    """The current GPU, where the call's tensors have to be."""
    if not t.is_cuda:
        raise ValueError(f"{name} is on {t.device}, not on the current GPU")
    return _current_device()


def _stream(stream, dev: int) -> int:
    return _raw_stream(dev) if stream is None and _raw_stream is not None else stream_handle(stream)


def _elsewhere(name: str, t):
    return ValueError(f"{name} is on {t.device}, not on the current GPU")


def _mat(name: str, t, rows: int, cols: int, dev: int):
    """A [rows][cols] float32 or bf16 tensor with adjacent columns as an ad_mat (None for None)."""
    if t is None:
        return None
    if t.get_device() != dev:
        raise _elsewhere(name, t)
    if t.shape != (rows, cols):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {(rows, cols)}")
    dtype = _DTYPE.get(t.dtype)
    if dtype is None:
        raise ValueError(f"{name} is {t.dtype}, expected float32 or bfloat16")
    ld, step = t.stride()
    if step != 1 and cols > 1:
        raise ValueError(f"{name}: the columns of a row must be adjacent")
    return _byref(Mat(t.data_ptr(), ld if rows > 1 else cols, dtype))


def _vec(name: str, t, n: int, dev: int):
    """The address of a contiguous [n] float32 or bf16 tensor (None for None)."""
    if t is None:
        return None
    if t.get_device() != dev:
        raise _elsewhere(name, t)
    if t.shape != (n,) or t.dtype not in _DTYPE or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous [{n}] tensor of float32 or bfloat16")
    return t.data_ptr()


def _floats(name: str, t, n: int, dev: int):
    """The address of a contiguous [n] float32 tensor (None for None)."""
    if t is None:
        return None
    if t.get_device() != dev:
        raise _elsewhere(name, t)
    if t.shape != (n,) or t.dtype is not torch.float32 or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous [{n}] tensor of float32")
    return t.data_ptr()


def _params(a_name: str, a, b_name: str, b, n: int, dev: int):
    """Two parameter vectors of one dtype: their addresses and that dtype."""
    if a is not None and b is not None and a.dtype != b.dtype:
        raise ValueError(f"{a_name} and {b_name} must have the same dtype")
    return _vec(a_name, a, n, dev), _vec(b_name, b, n, dev), AD_F32 if a is None else _DTYPE[a.dtype]


def _space(workspace, dev: int):
    if workspace is None:
        return None, 0
    if workspace.get_device() != dev:
        raise _elsewhere("workspace", workspace)
    if not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    return workspace.data_ptr(), workspace.nbytes


class Ckpt:
    """An activation of `cols` columns kept in 8 bits (ad.h: ad_ckpt): q int8 [rows][ld] and
    scale uint8 [rows][ld / 32], ld = cols rounded up to 128."""

    def __init__(self, q, scale, cols: int):
        ld = LIB.ad_ckpt_ld(cols)
        rows = q.shape[0]
        if not ld or q.shape != (rows, ld) or q.dtype is not torch.int8 or not q.is_contiguous():
            raise ValueError(f"a checkpoint's q must be a contiguous [{rows}][{ld}] int8 tensor")
        if scale.shape != (rows, ld // 32) or scale.dtype is not torch.uint8 or not scale.is_contiguous():
            raise ValueError(f"a checkpoint's scale must be a contiguous [{rows}][{ld // 32}] uint8 tensor")
        self.q, self.scale, self.rows, self.cols = q, scale, rows, cols

    @classmethod
    def empty(cls, rows: int, cols: int, device="cuda"):
        ld = LIB.ad_ckpt_ld(cols)
        return cls(torch.empty(rows, ld, dtype=torch.int8, device=device),
                   torch.empty(rows, ld // 32, dtype=torch.uint8, device=device), cols)


def _ckpt(name: str, k, rows: int, cols: int, dev: int):
    if k is None:
        return None
    q, scale = k.q, k.scale
    if q.get_device() != dev or scale.get_device() != dev:
        raise _elsewhere(name, q)
    if k.rows != rows or k.cols != cols:
        raise ValueError(f"{name} holds {(k.rows, k.cols)}, expected {(rows, cols)}")
    return _byref(CkptView(q.data_ptr(), scale.data_ptr()))


def ckpt_pack(x, ckpt: Ckpt, stream=None):
    """ckpt <- the rows of x in 8 bits."""
    rows, cols, dev = ckpt.rows, ckpt.cols, _device("ckpt", ckpt.q)
    check(LIB.ad_ckpt_pack(rows, cols, _mat("x", x, rows, cols, dev), _ckpt("ckpt", ckpt, rows, cols, dev),
                           _stream(stream, dev)), "ad_ckpt_pack")


def ckpt_unpack(ckpt: Ckpt, out, act: int = ACT_NONE, stream=None):
    """out <- act(the values of ckpt)."""
    rows, cols, dev = ckpt.rows, ckpt.cols, _device("ckpt", ckpt.q)
    check(LIB.ad_ckpt_unpack(rows, cols, _ckpt("ckpt", ckpt, rows, cols, dev), act, _mat("out", out, rows, cols, dev),
                             _stream(stream, dev)), "ad_ckpt_unpack")


def layer_norm(x, gain, bias, y, mean=None, rstd=None, xhat: Ckpt | None = None, stream=None):
    """LayerNorm of the rows of x into y (ad.h: ad_layer_norm); mean, rstd and xhat (the
    normalised rows in 8 bits) are kept for the backward pass when given."""
    (rows, cols), dev = x.shape, _device("x", x)
    g, b, dt = _params("gain", gain, "bias", bias, cols, dev)
    check(LIB.ad_layer_norm(rows, cols, _mat("x", x, rows, cols, dev), g, b, dt, _mat("y", y, rows, cols, dev),
                            _floats("mean", mean, rows, dev), _floats("rstd", rstd, rows, dev),
                            _ckpt("xhat", xhat, rows, cols, dev), _stream(stream, dev)), "ad_layer_norm")


def _workspace_size(name: str, *sizes) -> int:
    n = _size()
    check(getattr(LIB, name)(*sizes, ctypes.byref(n)), name)
    return n.value


def layer_norm_backward_workspace_size(rows: int, cols: int) -> int:
    return _workspace_size("ad_layer_norm_backward_workspace_size", rows, cols)


def layer_norm_backward(dy, x, mean, rstd, xhat, gain, dres, dx, dx_copy, dgain, dbias, workspace,
                        accumulate: bool = False, stream=None):
    """LayerNorm's gradients (ad.h: ad_layer_norm_backward) from x and mean, or from the
    checkpoint xhat (x and mean None); dres, dx_copy and the pair dgain, dbias may be None."""
    (rows, cols), dev = dy.shape, _device("dy", dy)
    ws, ws_bytes = _space(workspace, dev)
    g, _, dt = _params("gain", gain, "gain", None, cols, dev)
    check(LIB.ad_layer_norm_backward(
        rows, cols, _mat("dy", dy, rows, cols, dev), _mat("x", x, rows, cols, dev),
        _floats("mean", mean, rows, dev), _floats("rstd", rstd, rows, dev), _ckpt("xhat", xhat, rows, cols, dev),
        g, dt, _mat("dres", dres, rows, cols, dev), _mat("dx", dx, rows, cols, dev),
        _mat("dx_copy", dx_copy, rows, cols, dev), _floats("dgain", dgain, cols, dev),
        _floats("dbias", dbias, cols, dev), int(accumulate), ws, ws_bytes, _stream(stream, dev)),
        "ad_layer_norm_backward")


def linear_workspace_size(rows: int, n: int, k: int) -> int:
    return _workspace_size("ad_linear_workspace_size", rows, n, k)


def linear(x, w, bias, act: int, residual, y, pre, pre_ckpt, workspace, stream=None):
    """y = act(x w^T + bias) + residual (ad.h: ad_linear); bias, residual and the kept
    pre-activation (pre in bf16, or pre_ckpt in 8 bits) may be None."""
    (rows, k), n, dev = x.shape, w.shape[0], _device("x", x)
    ws, ws_bytes = _space(workspace, dev)
    b, _, dt = _params("bias", bias, "bias", None, n, dev)
    check(LIB.ad_linear(rows, n, k, _mat("x", x, rows, k, dev), _mat("w", w, n, k, dev), b, dt, act,
                        _mat("residual", residual, rows, n, dev), _mat("y", y, rows, n, dev),
                        _mat("pre", pre, rows, n, dev), _ckpt("pre_ckpt", pre_ckpt, rows, n, dev), ws, ws_bytes,
                        _stream(stream, dev)), "ad_linear")


def linear_dgrad_workspace_size(rows: int, n: int, k: int) -> int:
    return _workspace_size("ad_linear_dgrad_workspace_size", rows, n, k)


def linear_dgrad(dy, w, act: int, pre, pre_ckpt, dx, act_out, workspace, stream=None):
    """dx = (dy w) act'(pre) (ad.h: ad_linear_dgrad); act_out, when given, receives act(pre)."""
    (rows, n), k, dev = dy.shape, w.shape[1], _device("dy", dy)
    ws, ws_bytes = _space(workspace, dev)
    check(LIB.ad_linear_dgrad(rows, n, k, _mat("dy", dy, rows, n, dev), _mat("w", w, n, k, dev), act,
                              _mat("pre", pre, rows, k, dev), _ckpt("pre_ckpt", pre_ckpt, rows, k, dev),
                              _mat("dx", dx, rows, k, dev), _mat("act_out", act_out, rows, k, dev), ws, ws_bytes,
                              _stream(stream, dev)), "ad_linear_dgrad")


def linear_wgrad_workspace_size(rows: int, n: int, k: int) -> int:
    return _workspace_size("ad_linear_wgrad_workspace_size", rows, n, k)


def linear_wgrad(dy, x, x_ckpt, gain, shift, dw, dbias, workspace, accumulate: bool = False, stream=None):
    """dw = dy^T x and dbias = the column sums of dy (ad.h: ad_linear_wgrad), x in bf16 or as the
    checkpoint x_ckpt, of which gain and shift make the input; dbias may be None."""
    (rows, n), k, dev = dy.shape, dw.shape[1], _device("dy", dy)
    ws, ws_bytes = _space(workspace, dev)
    g, s, dt = _params("gain", gain, "shift", shift, k, dev)
    check(LIB.ad_linear_wgrad(rows, n, k, _mat("dy", dy, rows, n, dev), _mat("x", x, rows, k, dev),
                              _ckpt("x_ckpt", x_ckpt, rows, k, dev), g, s, dt, _mat("dw", dw, n, k, dev),
                              _floats("dbias", dbias, n, dev), int(accumulate), ws, ws_bytes, _stream(stream, dev)),
          "ad_linear_wgrad")


def _ints(name: str, t, shape, dev: int):
    """The address of a contiguous int32 tensor of this shape (None for None)."""
    if t is None:
        return None
    if t.get_device() != dev:
        raise _elsewhere(name, t)
    if tuple(t.shape) != shape or t.dtype is not torch.int32 or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {list(shape)} tensor of int32")
    return t.data_ptr()


class Attention:
    """What an attention call knows of its batch (ad.h: ad_attn), kept from one call to the next: heads,
    the tables of the sequences' rows (int32 tensors, read when the kernels run) and which keys are visible.
    q_max and k_max bound the rows of a sequence.  err_flag (int32 [1]) collects AD_ERR_* bits; without
    one the object has its own, `err_flag`.  covers: the caller says that every row of the matrices belongs to
    a sequence (as its padding at least), which callers that sum over rows need to know."""

    def __init__(self, q_heads: int, kv_heads: int, cu_q, cu_k, q_max: int, k_max: int, q_len=None, k_len=None,
                 causal: bool = False, window=None, err_flag=None, covers: bool = False):
        self.covers = covers
        self.batch = cu_q.shape[0] - 1
        if self.batch < 0:
            raise ValueError("cu_q needs at least one entry")
        dev = cu_q.get_device()
        if err_flag is None:
            err_flag = torch.zeros(1, dtype=torch.int32, device=cu_q.device)
        self.q_heads, self.kv_heads, self.window, self.err_flag = q_heads, kv_heads, window, err_flag
        self._dev, self._tables = dev, (cu_q, cu_k, q_len, k_len)
        window_rows = 0 if window is None else window.shape[0]
        self._fields = (_ints("cu_q", cu_q, (self.batch + 1,), dev), _ints("cu_k", cu_k, (self.batch + 1,), dev),
                        _ints("q_len", q_len, (self.batch,), dev), _ints("k_len", k_len, (self.batch,), dev),
                        _ints("window", window, (window_rows, 2), dev), _ints("err_flag", err_flag, (1,), dev))
        self._sizes = (q_max, k_max, int(causal))
        self._view = None

    def view(self, q_rows: int, k_rows: int):
        """The ad_attn of matrices with these rows."""
        kept = self._view
        if kept is None or kept[0] != (q_rows, k_rows):
            if self.window is not None and self.window.shape[0] != q_rows:
                raise ValueError(f"window has {self.window.shape[0]} rows, expected {q_rows}")
            s = AttnView(self.batch, self.q_heads, self.kv_heads, q_rows, k_rows, *self._sizes, *self._fields)
            kept = self._view = ((q_rows, k_rows), _byref(s))
        return kept[1]

    def on(self, dev: int):
        if self._dev != dev:
            raise ValueError(f"the batch's tables are on GPU {self._dev}, not on the current one")
        return dev


def _attn_space(name: str, at: Attention, q_rows: int, k_rows: int) -> int:
    n = _size()
    check(getattr(LIB, name)(at.view(q_rows, k_rows), ctypes.byref(n)), name)
    return n.value


def attention_workspace_size(at: Attention, q_rows: int, k_rows: int) -> int:
    return _attn_space("ad_attention_workspace_size", at, q_rows, k_rows)


def attention(at: Attention, q, k, v, o, lse=None, o_rest=None, workspace=None, stream=None):
    """o = softmax(q k^T / 8) v over the visible keys (ad.h: ad_attention); lse [q_heads][rows] and o_rest are
    kept for the backward pass when given."""
    rows, k_rows, dev = q.shape[0], k.shape[0], at.on(_device("q", q))
    wq, wk = 64 * at.q_heads, 64 * at.kv_heads
    ws, ws_bytes = _space(workspace, dev)
    check(LIB.ad_attention(at.view(rows, k_rows), _mat("q", q, rows, wq, dev), _mat("k", k, k_rows, wk, dev),
                           _mat("v", v, k_rows, wk, dev), _mat("o", o, rows, wq, dev),
                           _mat("o_rest", o_rest, rows, wq, dev), _table("lse", lse, at.q_heads, rows, dev), ws, ws_bytes,
                           _stream(stream, dev)), "ad_attention")


def _table(name: str, t, a: int, b: int, dev: int):
    """The address of a contiguous [a][b] float32 tensor (None for None)."""
    if t is None:
        return None
    if t.get_device() != dev:
        raise _elsewhere(name, t)
    if t.shape != (a, b) or t.dtype is not torch.float32 or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous [{a}][{b}] tensor of float32")
    return t.data_ptr()


def attention_backward_workspace_size(at: Attention, q_rows: int, k_rows: int) -> int:
    return _attn_space("ad_attention_backward_workspace_size", at, q_rows, k_rows)


def attention_backward(at: Attention, q, k, v, o, o_rest, lse, dout, dq_res, dq, dk, dv, workspace, stream=None):
    """The gradients dq (+ dq_res), dk and dv (ad.h: ad_attention_backward) from the forward pass's inputs, o,
    o_rest (or None) and lse; dq_res may be None."""
    rows, k_rows, dev = q.shape[0], k.shape[0], at.on(_device("q", q))
    wq, wk = 64 * at.q_heads, 64 * at.kv_heads
    ws, ws_bytes = _space(workspace, dev)
    if lse is None:
        raise ValueError("lse of the forward pass is needed")
    check(LIB.ad_attention_backward(
        at.view(rows, k_rows), _mat("q", q, rows, wq, dev), _mat("k", k, k_rows, wk, dev),
        _mat("v", v, k_rows, wk, dev), _mat("o", o, rows, wq, dev), _mat("o_rest", o_rest, rows, wq, dev),
        _table("lse", lse, at.q_heads, rows, dev), _mat("dout", dout, rows, wq, dev),
        _mat("dq_res", dq_res, rows, wq, dev), _mat("dq", dq, rows, wq, dev), _mat("dk", dk, k_rows, wk, dev),
        _mat("dv", dv, k_rows, wk, dev), ws, ws_bytes, _stream(stream, dev)), "ad_attention_backward")


class OptTensors:
    """Parameters with their gradients and optimizer states (ad.h: ad_opt_tensor), kept from one step to the
    next: lists of contiguous tensors of equal sizes on one GPU, of which a step's may not overlap (gradients among
    themselves may).  m and v are float32, or int8 and uint8 with the
    scales m_scale and v_scale of every 128 elements; copies (bf16) and any list that a call does not use may
    be None; weight_decay is one number or a list."""

    def __init__(self, params=None, grads=None, m=None, v=None, m_scale=None, v_scale=None, copies=None,
                 weight_decay=0.0):
        # (tuples of its own: the tensors live as long as their addresses are used, whatever becomes of the caller's lists)
        lists = {name: None if x is None else tuple(x) for name, x in
                 dict(params=params, grads=grads, m=m, v=v, m_scale=m_scale, v_scale=v_scale, copies=copies).items()}
        params, grads, m, v, m_scale, v_scale, copies = lists.values()
        given = [x for x in (grads, params, m) if x is not None]
        if not given:
            raise ValueError("no tensors given")
        self.count = len(given[0])
        for name, x in lists.items():
            if x is not None and len(x) != self.count:
                raise ValueError(f"{name} has {len(x)} tensors, expected {self.count}")
        if not isinstance(weight_decay, (list, tuple)):
            weight_decay = [weight_decay] * self.count
        elif len(weight_decay) != self.count:
            raise ValueError(f"weight_decay has {len(weight_decay)} numbers, expected {self.count}")
        self.tensors = lists
        self.device = given[0][0].get_device() if self.count else None
        self.numel = sum(t.numel() for t in given[0])
        self.array = (OptTensor * self.count)()
        self.steps = (params is not None and grads is not None and m is not None and v is not None)
        pick = lambda x, i: None if x is None else x[i]  # noqa: E731
        for i in range(self.count):
            e, n = self.array[i], given[0][i].numel()
            e.n, e.weight_decay = n, weight_decay[i]
            e.param = self._at("param", pick(params, i), n, torch.float32, torch.bfloat16)
            e.grad = self._at("grad", pick(grads, i), n, torch.float32, torch.bfloat16)
            e.copy = self._at("copy", pick(copies, i), n, torch.bfloat16)
            e.param_dtype = AD_F32 if params is None else _DTYPE[params[i].dtype]
            e.grad_dtype = AD_F32 if grads is None else _DTYPE[grads[i].dtype]
            eight = m is not None and m[i].dtype is torch.int8
            e.state = STATE_8 if eight else STATE_F
            e.m = self._at("m", pick(m, i), n, torch.int8 if eight else torch.float32)
            e.v = self._at("v", pick(v, i), n, torch.uint8 if eight else torch.float32)
            if eight:
                groups = -(-n // 128)
                if m_scale is None or v_scale is None:
                    raise ValueError("8-bit states need m_scale and v_scale")
                e.m_scale = self._at("m_scale", m_scale[i], groups, torch.float32)
                e.v_scale = self._at("v_scale", v_scale[i], groups, torch.float32)
        if self.steps:
            self._apart()

    def _apart(self):
        """Refuses a step that would write an element twice, or as it reads it as a gradient."""
        spans = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size(), name != "grads", f"{name}[{i}]")
                       for name, x in self.tensors.items() if x is not None for i, t in enumerate(x) if t is not None and t.numel())
        most = {False: (0, ""), True: (0, "")}      # how far those before reach: all of them, those that are written
        for begin, end, written, name in spans:
            over, other = most[not written]
            if begin < over:
                raise ValueError(f"{name} and {other} overlap: a step would write one of them twice, or as it reads it")
            for kind in (False, True) if written else (False,):
                most[kind] = max(most[kind], (end, name))

    def _at(self, name: str, t, n: int, *dtypes):
        if t is None:
            return None
        if t.get_device() != self.device:
            raise ValueError(f"{name} is on {t.device}, not on the other tensors' GPU")
        if t.numel() != n or t.dtype not in dtypes or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous tensor of {n} elements of {' or '.join(map(str, dtypes))}")
        return t.data_ptr()

    def on(self):
        """The current GPU, where the tensors have to be."""
        dev = _current_device() if self.count else torch.cuda.current_device()
        if self.count and self.device != dev:
            raise ValueError(f"the tensors are on GPU {self.device}, not on the current one")
        return dev


def _scalar(name: str, t, dtype, dev: int):
    if t is None:
        return None
    if t.get_device() != dev:
        raise _elsewhere(name, t)
    if t.numel() != 1 or t.dtype is not dtype:
        raise ValueError(f"{name} must be one number of {dtype}")
    return t.data_ptr()


def adamw(opt: OptTensors, lr, step, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8, seed: int = 0,
          grad_scale=None, stream=None):
    """One AdamW step (ad.h: ad_adamw).  lr and step are numbers, or tensors on the GPU (float32 [1], int32
    [1]) for a captured step; grad_scale is a float32 [1] on the GPU, or None."""
    dev = opt.on()
    if not opt.steps:
        raise ValueError("a step needs params, grads, m and v")
    lr_at = _scalar("lr", lr, torch.float32, dev) if isinstance(lr, torch.Tensor) else None
    step_at = _scalar("step", step, torch.int32, dev) if isinstance(step, torch.Tensor) else None
    a = AdamwArgs(0.0 if lr_at else lr, beta1, beta2, eps, 0 if step_at else step, seed & 0xFFFFFFFF, lr_at, step_at,
                  _scalar("grad_scale", grad_scale, torch.float32, dev))
    check(LIB.ad_adamw(opt.array, opt.count, _byref(a), _stream(stream, dev)), "ad_adamw")


def opt_state(opt: OptTensors, m, v, stream=None):
    """The states' values in float32, one tensor after the other, into m and v [sum of sizes] (either may
    be None; ad.h: ad_opt_state)."""
    dev = opt.on()
    check(LIB.ad_opt_state(opt.array, opt.count, _floats("m", m, opt.numel, dev), _floats("v", v, opt.numel, dev),
                           _stream(stream, dev)), "ad_opt_state")


def grad_norm_workspace_size(opt: OptTensors) -> int:
    return _workspace_size("ad_grad_norm_workspace_size", opt.array, opt.count)


def grad_norm(opt: OptTensors, max_norm: float, out, workspace, step=None, stream=None):
    """out[0] = the norm of all gradients, out[1] = the factor that clips it to max_norm (0: none); step (int32
    [1]) counts the finite ones (ad.h: ad_grad_norm)."""
    dev = opt.on()
    ws, ws_bytes = _space(workspace, dev)
    check(LIB.ad_grad_norm(opt.array, opt.count, max_norm, _floats("out", out, 2, dev),
                           _scalar("step", step, torch.int32, dev), ws, ws_bytes, _stream(stream, dev)), "ad_grad_norm")


def kv_import(model: Model, kv: KV, b: int, src, n: int, err_flag, stream=None):
    check(LIB.ad_kv_import(model.handle, ctypes.byref(kv), b, ptr(src), n, ptr(err_flag),
                           stream_handle(stream)), "ad_kv_import")


def kv_export(model: Model, kv: KV, b: int, dst, n: int, err_flag, stream=None):
    check(LIB.ad_kv_export(model.handle, ctypes.byref(kv), b, ptr(dst), n, ptr(err_flag),
                           stream_handle(stream)), "ad_kv_export")


def profile_enable(model: Model, kernel: int, max_launches: int):
    check(LIB.ad_profile_enable(model.handle, kernel, max_launches), "ad_profile_enable")


def profile_read(model: Model):
    """(summed milliseconds, number of timed launches) since the last read."""
    t, n = ctypes.c_double(), _i32()
    check(LIB.ad_profile_read(model.handle, ctypes.byref(t), ctypes.byref(n)), "ad_profile_read")
    return t.value, n.value
