// C-ABI entry points of the draft block's training operators: argument validation and the
// description of the operands handed to the launchers.
#include <cmath>
#include <cstdint>
#include <string>

#include "../../include/ad.h"
#include "status.h"
#include "train.h"

namespace {

using ad::check_hip;
using ad::fail;

constexpr int32_t kMaxRows = 1 << 24, kMaxCols = 1 << 20;
constexpr int64_t kMaxLd = 1 << 22;

#define AD_TRY(x)                    \
  do {                               \
    const ad_status s_ = (x);        \
    if (s_ != AD_OK) return s_;      \
  } while (0)

ad_status bad(const std::string& what) { return fail(AD_EINVAL, what); }

ad_status sizes_ok(int32_t rows, int32_t a, int32_t b = 1) {
  if (rows < 0 || rows > kMaxRows) return fail(AD_ERANGE, "rows must be in [0, 2^24]");
  if (a < 1 || a > kMaxCols || b < 1 || b > kMaxCols) return fail(AD_ERANGE, "widths must be in [1, 2^20]");
  return AD_OK;
}

bool dtype_ok(int32_t t) { return t == AD_F32 || t == AD_BF16; }

// A required matrix of `rows` rows (which may be 0) and `cols` columns.
ad_status mat_ok(const char* name, const ad_mat* m, int32_t rows, int32_t cols, bool bf16_only = false) {
  if (!m) return bad(std::string("NULL argument: ") + name);
  if (!dtype_ok(m->dtype)) return bad(std::string("unknown dtype: ") + name);
  if (bf16_only && m->dtype != AD_BF16) return fail(AD_EUNSUPPORTED, std::string(name) + " must be bf16");
  if (m->ld > kMaxLd) return fail(AD_ERANGE, std::string(name) + ": ld must be at most 2^22");
  if (m->ld < cols) return bad(std::string(name) + ": ld is smaller than the row");
  if (rows > 0 && !m->data) return bad(std::string("NULL argument: ") + name);
  if ((uintptr_t)m->data % (m->dtype == AD_BF16 ? 2 : 4)) return bad(std::string("misaligned: ") + name);
  return AD_OK;
}

ad_status ckpt_ok(const char* name, const ad_ckpt* k, int32_t rows) {
  if (!k) return bad(std::string("NULL argument: ") + name);
  if (rows > 0 && (!k->q || !k->scale)) return bad(std::string("NULL argument: ") + name);
  if ((uintptr_t)k->q % 16 || (uintptr_t)k->scale % 4) return bad(std::string("misaligned: ") + name);
  return AD_OK;
}

ad_status vec_ok(const char* name, const void* p, int32_t dtype) {
  if (!p) return bad(std::string("NULL argument: ") + name);
  if (!dtype_ok(dtype)) return bad(std::string("unknown dtype: ") + name);
  if ((uintptr_t)p % (dtype == AD_BF16 ? 2 : 4)) return bad(std::string("misaligned: ") + name);
  return AD_OK;
}

ad_status floats_ok(const char* name, const float* p) {
  return (uintptr_t)p % 4 ? bad(std::string("misaligned: ") + name) : AD_OK;
}

ad_status space_ok(const void* ws, size_t have, size_t need) {
  if (need && !ws) return bad("NULL argument: workspace");
  if ((uintptr_t)ws % 256) return bad("workspace must be 256-byte aligned");
  if (have < need) return fail(AD_ENOSPACE, "workspace needs " + std::to_string(need) + " bytes");
  return AD_OK;
}

ad::DMat mat(const ad_mat* m, int32_t cols) {
  ad::DMat d{};
  if (!m) return d;
  d.p = m->data;
  d.ld = m->ld;
  d.bf16 = m->dtype == AD_BF16;
  const uintptr_t p = (uintptr_t)m->data;
  // (kernels of whole vectors address a tile's 256 rows in 31 bits)
  d.vec = p % 16 == 0 && m->ld % (d.bf16 ? 8 : 4) == 0 && cols % 8 == 0 && m->ld <= (1 << 20);
  return d;
}

ad::DVec vec(const void* p, int32_t dtype) { return ad::DVec{p, dtype == AD_BF16, (uintptr_t)p % 16 == 0}; }

ad::DCkpt ckpt(const ad_ckpt* k, int32_t cols) {
  return k ? ad::DCkpt{k->q, k->scale, ad::ckpt_ld(cols)} : ad::DCkpt{nullptr, nullptr, ad::ckpt_ld(cols)};
}

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

size_t ln_bwd_bytes(int32_t rows, int32_t cols) {
  return align256(8ull * ad::ln_bwd_groups(rows, cols) * cols);
}
size_t linear_bytes(int kind, int32_t rows, int32_t n, int32_t k) {
  const int P = kind == ad::LIN_FWD ? n : k, Q = kind == ad::LIN_WGRAD ? n : rows,
            K = kind == ad::LIN_FWD ? k : kind == ad::LIN_DGRAD ? n : rows;
  return Q > 0 ? align256(4 * ad::lin_part_floats(kind, P, Q, K)) : 0;
}
ad_status linear_space(int kind, int32_t rows, int32_t n, int32_t k, size_t* bytes) {
  if (!bytes) return bad("NULL argument");
  AD_TRY(sizes_ok(rows, n, k));
  *bytes = linear_bytes(kind, rows, n, k);
  return AD_OK;
}

ad::LinOp op(const ad_mat* m, int extent) { return ad::LinOp{(const uint16_t*)m->data, m->ld, {}, extent}; }

// ----------------------------------------------------------------- attention

constexpr int32_t kMaxHeads = 1 << 14;    // 64 kMaxHeads = kMaxCols

ad_status attn_ok(const ad_attn* a) {
  if (!a) return bad("NULL argument");
  if (a->batch < 0 || a->batch > 65535) return fail(AD_ERANGE, "batch must be in [0, 65535]");
  if (a->q_heads < 1 || a->q_heads > kMaxHeads || a->kv_heads < 1 || a->kv_heads > kMaxHeads)
    return fail(AD_ERANGE, "heads must be in [1, 2^14]");
  if (a->q_heads % a->kv_heads) return bad("kv_heads must divide q_heads");
  if ((int64_t)a->batch * a->q_heads > ad::kMaxPairs) return fail(AD_ERANGE, "batch * q_heads must be at most 524280");
  if (a->q_rows < 0 || a->q_rows > kMaxRows || a->k_rows < 0 || a->k_rows > kMaxRows)
    return fail(AD_ERANGE, "rows must be in [0, 2^24]");
  if (a->q_max < 0 || a->q_max > kMaxRows || a->k_max < 0 || a->k_max > kMaxRows)
    return fail(AD_ERANGE, "q_max and k_max must be in [0, 2^24]");
  return AD_OK;
}

ad::AttnBatch attn_batch(const ad_attn* a) {
  ad::AttnBatch b{};
  b.batch = a->batch; b.heads = a->q_heads; b.kv_heads = a->kv_heads;
  b.group = a->q_heads / a->kv_heads;
  b.per_head = ad::per(a->q_heads); b.per_kv_head = ad::per(a->kv_heads);
  b.q_rows = a->q_rows; b.k_rows = a->k_rows;
  // (no sequence can have more rows than there are)
  b.q_max = a->q_max < a->q_rows ? a->q_max : a->q_rows;
  b.k_max = a->k_max < a->k_rows ? a->k_max : a->k_rows;
  b.causal = a->causal != 0;
  b.cu_q = a->cu_q; b.cu_k = a->cu_k; b.q_len = a->q_len; b.k_len = a->k_len; b.window = a->window;
  b.err = a->err_flag;
  return b;
}

// The sizes and the tables.
ad_status attn_call_ok(const ad_attn* a) {
  AD_TRY(attn_ok(a));
  if (!a->cu_q || !a->cu_k || !a->err_flag) return bad("NULL argument: cu_q, cu_k or err_flag");
  const void* tables[] = {a->cu_q, a->cu_k, a->q_len, a->k_len, a->window, a->err_flag};
  for (const void* t : tables)
    if ((uintptr_t)t % 4) return bad("misaligned table");
  return AD_OK;
}

ad::HMat hmat(const ad_mat* m) {
  ad::HMat d{};
  if (!m) return d;
  d.p = (uint16_t*)m->data;
  d.ld = m->ld;
  return d;
}

// ----------------------------------------------------------------- optimizer

ad_status tensors_ok(const ad_opt_tensor* t, int32_t count) {
  if (count < 0) return fail(AD_ERANGE, "count must not be negative");
  if (count > 0 && !t) return bad("NULL argument: tensors");
  for (int32_t i = 0; i < count; ++i)
    if (t[i].n < 0 || t[i].n > ad::kOptMost) return fail(AD_ERANGE, "n must be in [0, 2^37 - 8192]");
  return AD_OK;
}
ad_status array_ok(const char* name, const void* p, int size) {
  if (!p) return bad(std::string("NULL argument: ") + name);
  return (uintptr_t)p % size ? bad(std::string("misaligned: ") + name) : AD_OK;
}
int width(int32_t dtype) { return dtype == AD_BF16 ? 2 : 4; }

ad_status grad_ok(const ad_opt_tensor& t) {
  if (!dtype_ok(t.grad_dtype)) return bad("unknown dtype: grad");
  return t.n ? array_ok("grad", t.grad, width(t.grad_dtype)) : AD_OK;
}
ad_status state_ok(const ad_opt_tensor& t) {
  if (t.state != AD_STATE_F && t.state != AD_STATE_8) return bad("unknown state");
  if (!t.n) return AD_OK;
  const int size = t.state == AD_STATE_8 ? 1 : 4;
  AD_TRY(array_ok("m", t.m, size));
  AD_TRY(array_ok("v", t.v, size));
  if (t.state == AD_STATE_8) {
    AD_TRY(array_ok("m_scale", t.m_scale, 4));
    AD_TRY(array_ok("v_scale", t.v_scale, 4));
  }
  return AD_OK;
}

// Hands the tensors that hold something to `go`, a launch's worth at a time: the list and the tensors' places.
template <class F>
void by_launch(const ad_opt_tensor* t, int32_t count, double lr, F&& go) {
  ad::OptList l;
  int at[ad::kOptTensors];
  for (int i = 0; i < count;) {
    i = ad::opt_launch([&](int k) { return t[k].n; }, count, i, at, l.count);
    if (!l.count) return;
    l.first[0] = 0;
    for (int k = 0; k < l.count; ++k) {
      const ad_opt_tensor& f = t[at[k]];
      ad::OptTensor& d = l.t[k];
      d.n = f.n;
      d.param = f.param; d.copy = f.copy; d.grad = f.grad;
      d.m = f.m; d.v = f.v; d.m_scale = f.m_scale; d.v_scale = f.v_scale;
      d.keep = (float)(1.0 - lr * f.weight_decay);
      d.decay = (float)f.weight_decay;
      d.key = (uint32_t)at[k];
      d.kinds = (f.param_dtype == AD_BF16 ? ad::OPT_PARAM16 : 0) | (f.grad_dtype == AD_BF16 ? ad::OPT_GRAD16 : 0) |
                (f.state == AD_STATE_8 ? ad::OPT_STATE8 : 0);
      l.first[k + 1] = l.first[k] + (int)ad::opt_groups(f.n);
    }
    go(l, at);
  }
}
int64_t norm_parts(const ad_opt_tensor* t, int32_t count) {
  int64_t parts = 0;
  for (int32_t i = 0; i < count; ++i) parts += ad::opt_groups(t[i].n);
  return parts;
}

}  // namespace

extern "C" {

int32_t ad_ckpt_ld(int32_t cols) { return cols < 1 || cols > kMaxCols ? 0 : ad::ckpt_ld(cols); }

ad_status ad_ckpt_pack(int32_t rows, int32_t cols, const ad_mat* x, const ad_ckpt* k, void* stream) {
  AD_TRY(sizes_ok(rows, cols));
  AD_TRY(mat_ok("x", x, rows, cols));
  AD_TRY(ckpt_ok("ckpt", k, rows));
  if ((int64_t)rows * ((cols + 511) / 512) >= INT32_MAX) return fail(AD_ERANGE, "rows * cols is too large");
  (void)hipGetLastError();
  ad::launch_ckpt_pack(rows, cols, mat(x, cols), ckpt(k, cols), (hipStream_t)stream);
  return check_hip("ad_ckpt_pack");
}

ad_status ad_ckpt_unpack(int32_t rows, int32_t cols, const ad_ckpt* k, int32_t act, const ad_mat* out,
                         void* stream) {
  AD_TRY(sizes_ok(rows, cols));
  AD_TRY(ckpt_ok("ckpt", k, rows));
  AD_TRY(mat_ok("out", out, rows, cols));
  if (act != AD_ACT_NONE && act != AD_ACT_GELU) return bad("unknown act");
  if ((int64_t)rows * ((cols + 511) / 512) >= INT32_MAX) return fail(AD_ERANGE, "rows * cols is too large");
  (void)hipGetLastError();
  ad::launch_ckpt_unpack(rows, cols, ckpt(k, cols), act == AD_ACT_GELU, mat(out, cols), (hipStream_t)stream);
  return check_hip("ad_ckpt_unpack");
}

ad_status ad_layer_norm(int32_t rows, int32_t cols, const ad_mat* x, const void* gain, const void* bias,
                        int32_t param_dtype, const ad_mat* y, float* mean, float* rstd, const ad_ckpt* xhat,
                        void* stream) {
  AD_TRY(sizes_ok(rows, cols));
  AD_TRY(mat_ok("x", x, rows, cols));
  AD_TRY(vec_ok("gain", gain, param_dtype));
  AD_TRY(vec_ok("bias", bias, param_dtype));
  AD_TRY(mat_ok("y", y, rows, cols));
  AD_TRY(floats_ok("mean", mean));
  AD_TRY(floats_ok("rstd", rstd));
  if (xhat) AD_TRY(ckpt_ok("xhat", xhat, rows));
  if (cols > ad::kLnMaxCols) return fail(AD_EUNSUPPORTED, "LayerNorm takes at most 8192 columns");
  ad::LnFwdArgs a{};
  a.rows = rows; a.cols = cols;
  a.x = mat(x, cols); a.y = mat(y, cols);
  a.gain = vec(gain, param_dtype); a.bias = vec(bias, param_dtype);
  a.mean = mean; a.rstd = rstd; a.xhat = ckpt(xhat, cols);
  (void)hipGetLastError();
  ad::launch_layer_norm(a, (hipStream_t)stream);
  return check_hip("ad_layer_norm");
}

ad_status ad_layer_norm_backward_workspace_size(int32_t rows, int32_t cols, size_t* bytes) {
  if (!bytes) return bad("NULL argument");
  AD_TRY(sizes_ok(rows, cols));
  if (cols > ad::kLnMaxCols) return fail(AD_EUNSUPPORTED, "LayerNorm takes at most 8192 columns");
  *bytes = ln_bwd_bytes(rows, cols);
  return AD_OK;
}

ad_status ad_layer_norm_backward(int32_t rows, int32_t cols, const ad_mat* dy, const ad_mat* x, const float* mean,
                                 const float* rstd, const ad_ckpt* xhat, const void* gain, int32_t param_dtype,
                                 const ad_mat* dres, const ad_mat* dx, const ad_mat* dx_copy, float* dgain,
                                 float* dbias, int32_t accumulate, void* workspace, size_t workspace_bytes,
                                 void* stream) {
  AD_TRY(sizes_ok(rows, cols));
  AD_TRY(mat_ok("dy", dy, rows, cols));
  if ((x != nullptr) == (xhat != nullptr)) return bad("xhat comes from x and mean, or from the checkpoint");
  if (x) {
    AD_TRY(mat_ok("x", x, rows, cols));
    if (rows > 0 && !mean) return bad("NULL argument: mean");
  } else {
    AD_TRY(ckpt_ok("xhat", xhat, rows));
  }
  if (rows > 0 && !rstd) return bad("NULL argument: rstd");
  AD_TRY(floats_ok("mean", mean));
  AD_TRY(floats_ok("rstd", rstd));
  AD_TRY(vec_ok("gain", gain, param_dtype));
  if (dres) AD_TRY(mat_ok("dres", dres, rows, cols));
  AD_TRY(mat_ok("dx", dx, rows, cols));
  if (dx_copy) AD_TRY(mat_ok("dx_copy", dx_copy, rows, cols, true));
  if ((dgain != nullptr) != (dbias != nullptr)) return bad("dgain and dbias: both or neither");
  AD_TRY(floats_ok("dgain", dgain));
  AD_TRY(floats_ok("dbias", dbias));
  if (cols > ad::kLnMaxCols) return fail(AD_EUNSUPPORTED, "LayerNorm takes at most 8192 columns");
  AD_TRY(space_ok(workspace, workspace_bytes, dgain ? ln_bwd_bytes(rows, cols) : 0));
  ad::LnBwdArgs a{};
  a.rows = rows; a.cols = cols;
  a.dy = mat(dy, cols); a.x = mat(x, cols); a.dres = mat(dres, cols); a.dx = mat(dx, cols);
  a.copy = mat(dx_copy, cols);
  a.gain = vec(gain, param_dtype);
  a.mean = mean; a.rstd = rstd; a.xhat = ckpt(xhat, cols);
  a.dgain = dgain; a.dbias = dbias; a.accumulate = accumulate != 0;
  a.part = (float*)workspace;
  (void)hipGetLastError();
  ad::launch_layer_norm_backward(a, (hipStream_t)stream);
  return check_hip("ad_layer_norm_backward");
}

ad_status ad_linear_workspace_size(int32_t rows, int32_t n, int32_t k, size_t* bytes) {
  return linear_space(ad::LIN_FWD, rows, n, k, bytes);
}
ad_status ad_linear_dgrad_workspace_size(int32_t rows, int32_t n, int32_t k, size_t* bytes) {
  return linear_space(ad::LIN_DGRAD, rows, n, k, bytes);
}
ad_status ad_linear_wgrad_workspace_size(int32_t rows, int32_t n, int32_t k, size_t* bytes) {
  return linear_space(ad::LIN_WGRAD, rows, n, k, bytes);
}

ad_status ad_linear(int32_t rows, int32_t n, int32_t k, const ad_mat* x, const ad_mat* w, const void* bias,
                    int32_t bias_dtype, int32_t act, const ad_mat* residual, const ad_mat* y, const ad_mat* pre,
                    const ad_ckpt* pre_ckpt, void* workspace, size_t workspace_bytes, void* stream) {
  AD_TRY(sizes_ok(rows, n, k));
  AD_TRY(mat_ok("x", x, rows, k, true));
  AD_TRY(mat_ok("w", w, n, k, true));
  if (bias) AD_TRY(vec_ok("bias", bias, bias_dtype));
  if (act != AD_ACT_NONE && act != AD_ACT_GELU) return bad("unknown act");
  if (residual) AD_TRY(mat_ok("residual", residual, rows, n));
  AD_TRY(mat_ok("y", y, rows, n));
  if (pre && pre_ckpt) return bad("pre or pre_ckpt, not both");
  if (pre) AD_TRY(mat_ok("pre", pre, rows, n, true));
  if (pre_ckpt) AD_TRY(ckpt_ok("pre_ckpt", pre_ckpt, rows));
  AD_TRY(space_ok(workspace, workspace_bytes, linear_bytes(ad::LIN_FWD, rows, n, k)));
  if (rows == 0) return AD_OK;
  ad::LinArgs a{};
  a.P = op(w, n); a.Q = op(x, rows); a.K = k;
  a.part = (float*)workspace;
  a.bias = vec(bias, bias_dtype);
  a.gelu = act == AD_ACT_GELU;
  a.res = mat(residual, n); a.out = mat(y, n); a.pre = mat(pre, n); a.ck = ckpt(pre_ckpt, n);
  (void)hipGetLastError();
  ad::launch_linear(ad::LIN_FWD, a, (hipStream_t)stream);
  return check_hip("ad_linear");
}

ad_status ad_linear_dgrad(int32_t rows, int32_t n, int32_t k, const ad_mat* dy, const ad_mat* w, int32_t act,
                          const ad_mat* pre, const ad_ckpt* pre_ckpt, const ad_mat* dx, const ad_mat* act_out,
                          void* workspace, size_t workspace_bytes, void* stream) {
  AD_TRY(sizes_ok(rows, n, k));
  AD_TRY(mat_ok("dy", dy, rows, n, true));
  AD_TRY(mat_ok("w", w, n, k, true));
  if (act == AD_ACT_GELU) {
    if ((pre != nullptr) == (pre_ckpt != nullptr)) return bad("GELU needs pre or pre_ckpt, one of them");
    if (pre) AD_TRY(mat_ok("pre", pre, rows, k, true));
    else AD_TRY(ckpt_ok("pre_ckpt", pre_ckpt, rows));
    if (act_out) AD_TRY(mat_ok("act_out", act_out, rows, k, true));
  } else if (act == AD_ACT_NONE) {
    if (pre || pre_ckpt || act_out) return bad("pre, pre_ckpt and act_out need an activation");
  } else {
    return bad("unknown act");
  }
  AD_TRY(mat_ok("dx", dx, rows, k));
  AD_TRY(space_ok(workspace, workspace_bytes, linear_bytes(ad::LIN_DGRAD, rows, n, k)));
  if (rows == 0) return AD_OK;
  ad::LinArgs a{};
  a.P = op(w, k); a.Q = op(dy, rows); a.K = n;
  a.part = (float*)workspace;
  a.gelu = act == AD_ACT_GELU;
  a.out = mat(dx, k); a.pre = mat(pre, k); a.act_out = mat(act_out, k); a.ck = ckpt(pre_ckpt, k);
  (void)hipGetLastError();
  ad::launch_linear(ad::LIN_DGRAD, a, (hipStream_t)stream);
  return check_hip("ad_linear_dgrad");
}

ad_status ad_linear_wgrad(int32_t rows, int32_t n, int32_t k, const ad_mat* dy, const ad_mat* x,
                          const ad_ckpt* x_ckpt, const void* gain, const void* shift, int32_t param_dtype,
                          const ad_mat* dw, float* dbias, int32_t accumulate, void* workspace,
                          size_t workspace_bytes, void* stream) {
  AD_TRY(sizes_ok(rows, n, k));
  AD_TRY(mat_ok("dy", dy, rows, n, true));
  if ((x != nullptr) == (x_ckpt != nullptr)) return bad("x or x_ckpt, one of them");
  if (x) AD_TRY(mat_ok("x", x, rows, k, true));
  else AD_TRY(ckpt_ok("x_ckpt", x_ckpt, rows));
  if ((gain != nullptr) != (shift != nullptr)) return bad("gain and shift: both or neither");
  if (gain) {
    if (x) return bad("gain and shift go with x_ckpt");
    AD_TRY(vec_ok("gain", gain, param_dtype));
    AD_TRY(vec_ok("shift", shift, param_dtype));
  }
  AD_TRY(mat_ok("dw", dw, n, k));
  if (dw->dtype != AD_F32) return fail(AD_EUNSUPPORTED, "dw must be float32");
  AD_TRY(floats_ok("dbias", dbias));
  AD_TRY(space_ok(workspace, workspace_bytes, linear_bytes(ad::LIN_WGRAD, rows, n, k)));
  ad::LinArgs a{};
  if (x) a.P = op(x, k);
  else a.P = ad::LinOp{nullptr, 0, ckpt(x_ckpt, k), k};
  a.Q = op(dy, n); a.K = rows;
  a.part = (float*)workspace;
  a.gain = vec(gain, param_dtype); a.shift = vec(shift, param_dtype);
  a.accumulate = accumulate != 0;
  a.out = mat(dw, k); a.dbias = dbias;
  (void)hipGetLastError();
  ad::launch_linear(ad::LIN_WGRAD, a, (hipStream_t)stream);
  return check_hip("ad_linear_wgrad");
}

ad_status ad_attention_workspace_size(const ad_attn* a, size_t* bytes) {
  if (!bytes) return bad("NULL argument");
  AD_TRY(attn_ok(a));
  *bytes = align256(ad::attn_fwd_bytes(attn_batch(a)));
  return AD_OK;
}

ad_status ad_attention(const ad_attn* a, const ad_mat* q, const ad_mat* k, const ad_mat* v, const ad_mat* o,
                       const ad_mat* o_rest, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  AD_TRY(attn_call_ok(a));
  const int32_t wq = 64 * a->q_heads, wk = 64 * a->kv_heads;
  AD_TRY(mat_ok("q", q, a->q_rows, wq, true));
  AD_TRY(mat_ok("k", k, a->k_rows, wk, true));
  AD_TRY(mat_ok("v", v, a->k_rows, wk, true));
  AD_TRY(mat_ok("o", o, a->q_rows, wq, true));
  if (o_rest) AD_TRY(mat_ok("o_rest", o_rest, a->q_rows, wq, true));
  AD_TRY(floats_ok("lse", lse));
  ad::AttnFwdArgs f{};
  f.b = attn_batch(a);
  AD_TRY(space_ok(workspace, workspace_bytes, align256(ad::attn_fwd_bytes(f.b))));
  f.q = hmat(q); f.k = hmat(k); f.v = hmat(v); f.o = hmat(o); f.rest = hmat(o_rest);
  f.lse = lse;
  f.part = (float*)workspace;
  (void)hipGetLastError();
  ad::launch_attention(f, (hipStream_t)stream);
  return check_hip("ad_attention");
}

ad_status ad_attention_backward_workspace_size(const ad_attn* a, size_t* bytes) {
  if (!bytes) return bad("NULL argument");
  AD_TRY(attn_ok(a));
  *bytes = align256(ad::attn_bwd_bytes(attn_batch(a)));
  return AD_OK;
}

ad_status ad_attention_backward(const ad_attn* a, const ad_mat* q, const ad_mat* k, const ad_mat* v, const ad_mat* o,
                                const ad_mat* o_rest, const float* lse, const ad_mat* dout, const ad_mat* dq_res,
                                const ad_mat* dq, const ad_mat* dk, const ad_mat* dv, void* workspace,
                                size_t workspace_bytes, void* stream) {
  AD_TRY(attn_call_ok(a));
  const int32_t wq = 64 * a->q_heads, wk = 64 * a->kv_heads;
  AD_TRY(mat_ok("q", q, a->q_rows, wq, true));
  AD_TRY(mat_ok("k", k, a->k_rows, wk, true));
  AD_TRY(mat_ok("v", v, a->k_rows, wk, true));
  AD_TRY(mat_ok("o", o, a->q_rows, wq, true));
  if (o_rest) AD_TRY(mat_ok("o_rest", o_rest, a->q_rows, wq, true));
  AD_TRY(mat_ok("dout", dout, a->q_rows, wq, true));
  if (dq_res) AD_TRY(mat_ok("dq_res", dq_res, a->q_rows, wq));
  AD_TRY(mat_ok("dq", dq, a->q_rows, wq, true));
  AD_TRY(mat_ok("dk", dk, a->k_rows, wk, true));
  AD_TRY(mat_ok("dv", dv, a->k_rows, wk, true));
  if (a->q_rows > 0 && !lse) return bad("NULL argument: lse");
  AD_TRY(floats_ok("lse", lse));
  ad::AttnBwdArgs f{};
  f.b = attn_batch(a);
  AD_TRY(space_ok(workspace, workspace_bytes, align256(ad::attn_bwd_bytes(f.b))));
  f.q = hmat(q); f.k = hmat(k); f.v = hmat(v); f.o = hmat(o); f.rest = hmat(o_rest); f.dout = hmat(dout);
  f.dq = hmat(dq); f.dk = hmat(dk); f.dv = hmat(dv);
  f.res = mat(dq_res, wq);
  f.lse = lse;
  f.delta = (float*)workspace;
  (void)hipGetLastError();
  ad::launch_attention_backward(f, (hipStream_t)stream);
  return check_hip("ad_attention_backward");
}

ad_status ad_adamw(const ad_opt_tensor* tensors, int32_t count, const ad_adamw_args* args, void* stream) {
  AD_TRY(tensors_ok(tensors, count));
  if (!args) return bad("NULL argument: args");
  const ad_adamw_args& h = *args;
  if (!h.step_at && h.step < 1) return fail(AD_ERANGE, "step must be at least 1");
  if (!h.lr_at && !(h.lr >= 0 && std::isfinite(h.lr))) return fail(AD_ERANGE, "lr must be finite and not negative");
  if (!(h.beta1 >= 0 && h.beta1 < 1 && h.beta2 >= 0 && h.beta2 < 1)) return fail(AD_ERANGE, "betas must be in [0, 1)");
  if (!(h.eps >= 0 && std::isfinite(h.eps))) return fail(AD_ERANGE, "eps must be finite and not negative");
  const void* scalars[] = {h.lr_at, h.step_at, h.grad_scale};
  for (const void* p : scalars)
    if ((uintptr_t)p % 4) return bad("misaligned: lr_at, step_at or grad_scale");
  for (int32_t i = 0; i < count; ++i) {
    const ad_opt_tensor& t = tensors[i];
    if (!dtype_ok(t.param_dtype)) return bad("unknown dtype: param");
    if (!(t.weight_decay >= 0 && std::isfinite(t.weight_decay)))
      return fail(AD_ERANGE, "weight_decay must be finite and not negative");
    AD_TRY(grad_ok(t));
    AD_TRY(state_ok(t));
    if (t.copy && t.param_dtype == AD_BF16) return bad("copy goes with a float32 param");
    if ((uintptr_t)t.copy % 2) return bad("misaligned: copy");
    if (t.n) AD_TRY(array_ok("param", t.param, width(t.param_dtype)));
  }
  ad::AdamwArgs a{};
  a.b1 = (float)h.beta1; a.ob1 = (float)(1.0 - h.beta1);
  a.b2 = (float)h.beta2; a.ob2 = (float)(1.0 - h.beta2);
  const int step = h.step_at ? 1 : h.step;       // (not used where it is on the device)
  a.root = (float)(1.0 / std::sqrt(1.0 - std::pow(h.beta2, step)));
  a.rate = (float)(h.lr / (1.0 - std::pow(h.beta1, step)));
  a.eps = (float)h.eps;
  a.beta1 = h.beta1; a.beta2 = h.beta2; a.lr = h.lr;
  a.step = step; a.seed = h.seed;
  a.lr_at = h.lr_at; a.step_at = h.step_at; a.scale = h.grad_scale;
  (void)hipGetLastError();
  by_launch(tensors, count, h.lr_at ? 0.0 : h.lr,
            [&](const ad::OptList& l, const int*) { ad::launch_adamw(l, a, (hipStream_t)stream); });
  return check_hip("ad_adamw");
}

ad_status ad_opt_state(const ad_opt_tensor* tensors, int32_t count, float* m, float* v, void* stream) {
  AD_TRY(tensors_ok(tensors, count));
  AD_TRY(floats_ok("m", m));
  AD_TRY(floats_ok("v", v));
  for (int32_t i = 0; i < count; ++i) AD_TRY(state_ok(tensors[i]));
  (void)hipGetLastError();
  int64_t at = 0;
  int32_t done = 0;
  by_launch(tensors, count, 0.0, [&](const ad::OptList& l, const int* places) {
    int64_t first[ad::kOptTensors];
    for (int i = 0; i < l.count; ++i) {
      for (; done < places[i]; ++done) at += tensors[done].n;
      first[i] = at;
    }
    ad::launch_opt_state(l, m, v, first, (hipStream_t)stream);
  });
  return check_hip("ad_opt_state");
}

ad_status ad_grad_norm_workspace_size(const ad_opt_tensor* tensors, int32_t count, size_t* bytes) {
  if (!bytes) return bad("NULL argument");
  AD_TRY(tensors_ok(tensors, count));
  *bytes = align256(8 * (size_t)norm_parts(tensors, count));
  return AD_OK;
}

ad_status ad_grad_norm(const ad_opt_tensor* tensors, int32_t count, double max_norm, float* out, int32_t* step,
                       void* workspace, size_t workspace_bytes, void* stream) {
  AD_TRY(tensors_ok(tensors, count));
  if (!(max_norm >= 0 && std::isfinite(max_norm))) return fail(AD_ERANGE, "max_norm must be finite and not negative");
  AD_TRY(array_ok("out", out, 4));
  if ((uintptr_t)step % 4) return bad("misaligned: step");
  for (int32_t i = 0; i < count; ++i) AD_TRY(grad_ok(tensors[i]));
  const int64_t parts = norm_parts(tensors, count);
  AD_TRY(space_ok(workspace, workspace_bytes, align256(8 * (size_t)parts)));
  (void)hipGetLastError();
  double* part = (double*)workspace;
  bool done = false;
  by_launch(tensors, count, 0.0, [&](const ad::OptList& l, const int*) {
    // (the only list)
    done = part == workspace && l.first[l.count] == parts && ad::norm_of_few(l);
    if (done) return ad::launch_grad_norm_few(l, max_norm, out, step, (hipStream_t)stream);
    ad::launch_grad_squares(l, part, (hipStream_t)stream);
    part += l.first[l.count];
  });
  if (!done) ad::launch_grad_norm((const double*)workspace, parts, max_norm, out, step, (hipStream_t)stream);
  return check_hip("ad_grad_norm");
}

}  // extern "C"
