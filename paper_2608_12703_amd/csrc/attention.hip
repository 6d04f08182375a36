// Attention over matrices and its gradients (the draft block's training), 64-wide heads.
#include <algorithm>

#include "train.h"

namespace ad {

namespace {

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.69314718055994531f;
constexpr float kScale = 0.125f;                       // 1 / sqrt(64)
constexpr float kScale2 = kScale * kLog2e;             // scores in powers of two

// One sequence's rows; ok = false where its table entries are out of range.
struct Span {
  int q0, nq, oq, k0, nk, ok_;   // first row, rows that hold something, rows it owns; keys; keys it owns
  bool ok;
};
__device__ __forceinline__ Span span_of(const AttnBatch& a, int b) {
  Span s;
  s.q0 = a.cu_q[b];
  s.k0 = a.cu_k[b];
  const int qe = a.cu_q[b + 1], ke = a.cu_k[b + 1];
  s.ok = s.q0 >= 0 && qe >= s.q0 && qe <= a.q_rows && s.k0 >= 0 && ke >= s.k0 && ke <= a.k_rows;
  s.oq = qe - s.q0;
  s.ok_ = ke - s.k0;
  s.nq = a.q_len ? a.q_len[b] : s.oq;
  s.nk = a.k_len ? a.k_len[b] : s.ok_;
  s.ok = s.ok && s.oq <= a.q_max && s.ok_ <= a.k_max && s.nq >= 0 && s.nq <= s.oq && s.nk >= 0 && s.nk <= s.ok_;
  return s;
}

// The keys [lo, hi) that query i of the sequence sees (lo >= hi: none).
struct Keys {
  int lo, hi;
};
__device__ __forceinline__ Keys keys_of(const AttnBatch& a, const Span& s, int i) {
  Keys r = {0, s.nk};
  if (a.causal) r.hi = min(r.hi, max(i + s.nk - s.nq + 1, 0));
  if (a.window) {
    const int2 w = *(const int2*)(a.window + 2 * (size_t)(s.q0 + i));
    r.lo = max(r.lo, w.x);
    r.hi = min(r.hi, w.y);
  }
  return r;
}

__device__ __forceinline__ float at(const HMat& m, size_t row, int col) {
  return m.p ? bf16_to_f32(m.p[row * m.ld + col]) : 0.f;
}

// A row at a time, a lane a dimension: what is right whatever the keys hold, since only visible
// ones are read.
__device__ void fwd_row(const AttnFwdArgs& a, const Span& s, int h, int i) {
  const int d = threadIdx.x % kWave, g = h / (a.b.heads / a.b.kv_heads);
  const size_t row = s.q0 + i;
  float m = -INFINITY, l = 0.f, o = 0.f;
  if (i < s.nq) {
    const float q = at(a.q, row, 64 * h + d) * kScale2;
    const Keys r = keys_of(a.b, s, i);
    for (int j = r.lo; j < r.hi; ++j) {
      const float x = wave_sum(q * at(a.k, s.k0 + j, 64 * g + d)), top = fmaxf(m, x);
      const float base = top == -INFINITY ? 0.f : top;
      const float old = __builtin_amdgcn_exp2f(m - base), p = __builtin_amdgcn_exp2f(x - base);
      l = l * old + p;
      o = o * old;
      if (p != 0.f) o = fmaf(p, at(a.v, s.k0 + j, 64 * g + d), o);
      m = top;
    }
  }
  o = l == 0.f ? 0.f : o / l;
  const uint16_t hi = f32_to_bf16(o);
  a.o.p[row * a.o.ld + 64 * h + d] = hi;
  if (a.rest.p) a.rest.p[row * a.rest.ld + 64 * h + d] = f32_to_bf16(o - bf16_to_f32(hi));
  if (a.lse && d == 0) a.lse[(size_t)h * a.b.q_rows + row] = l == 0.f ? -INFINITY : (m + __log2f(l)) * kLn2;
}

__device__ void dq_row(const AttnBwdArgs& a, const Span& s, int h, int i) {
  const int d = threadIdx.x % kWave, g = h / (a.b.heads / a.b.kv_heads);
  const size_t row = s.q0 + i;
  float acc = 0.f;
  if (i < s.nq) {
    const float q = at(a.q, row, 64 * h + d) * kScale2, go = at(a.dout, row, 64 * h + d);
    const float delta = wave_sum(go * (at(a.o, row, 64 * h + d) + at(a.rest, row, 64 * h + d)));
    const float lse = a.lse[(size_t)h * a.b.q_rows + row] * kLog2e;
    if (d == 0) a.delta[(size_t)h * a.b.q_rows + row] = delta;
    Keys r = keys_of(a.b, s, i);
    if (lse == -INFINITY) r.hi = r.lo;
    for (int j = r.lo; j < r.hi; ++j) {
      const float k = at(a.k, s.k0 + j, 64 * g + d);
      const float p = __builtin_amdgcn_exp2f(wave_sum(q * k) - lse);
      const float dp = wave_sum(go * at(a.v, s.k0 + j, 64 * g + d));
      acc = fmaf(p * (dp - delta), k, acc);
    }
    acc *= kScale;
    if (a.res.p) acc += a.res.bf16 ? bf16_to_f32(((const uint16_t*)a.res.p)[row * a.res.ld + 64 * h + d])
                                   : ((const float*)a.res.p)[row * a.res.ld + 64 * h + d];
  }
  a.dq.p[row * a.dq.ld + 64 * h + d] = f32_to_bf16(acc);
}

__device__ void dkv_row(const AttnBwdArgs& a, const Span& s, int g, int j) {
  const int d = threadIdx.x % kWave, n = a.b.heads / a.b.kv_heads;
  const size_t row = s.k0 + j;
  float dk = 0.f, dv = 0.f;
  if (j < s.nk) {
    const float k = at(a.k, row, 64 * g + d) * kScale2, v = at(a.v, row, 64 * g + d);
    for (int h = g * n; h < (g + 1) * n; ++h)
      for (int i = 0; i < s.nq; ++i) {
        const Keys r = keys_of(a.b, s, i);
        const size_t qr = s.q0 + i;
        const float lse = a.lse[(size_t)h * a.b.q_rows + qr] * kLog2e;
        if (j < r.lo || j >= r.hi || lse == -INFINITY) continue;
        const float q = at(a.q, qr, 64 * h + d), go = at(a.dout, qr, 64 * h + d);
        const float p = __builtin_amdgcn_exp2f(wave_sum(q * k) - lse);
        const float ds = p * (wave_sum(go * v) - a.delta[(size_t)h * a.b.q_rows + qr]);
        dk = fmaf(ds, q, dk);
        dv = fmaf(p, go, dv);
      }
  }
  a.dk.p[row * a.dk.ld + 64 * g + d] = f32_to_bf16(dk * kScale);
  a.dv.p[row * a.dv.ld + 64 * g + d] = f32_to_bf16(dv);
}

__global__ void __launch_bounds__(256) attn_fwd_rows_kernel(AttnFwdArgs a, int tiles) {
  const int tile = blockIdx.x % tiles, h = blockIdx.x / tiles % a.b.heads, b = blockIdx.x / tiles / a.b.heads;
  const Span s = span_of(a.b, b);
  if (!s.ok) {
    if (threadIdx.x == 0) atomicOr(a.b.err, AD_ERR_LENGTH);
    return;
  }
  const int i = tile * 4 + threadIdx.x / kWave;
  if (i < s.oq) fwd_row(a, s, h, i);
}
__global__ void __launch_bounds__(256) attn_dq_rows_kernel(AttnBwdArgs a, int tiles) {
  const int tile = blockIdx.x % tiles, h = blockIdx.x / tiles % a.b.heads, b = blockIdx.x / tiles / a.b.heads;
  const Span s = span_of(a.b, b);
  if (!s.ok) {
    if (threadIdx.x == 0) atomicOr(a.b.err, AD_ERR_LENGTH);
    return;
  }
  const int i = tile * 4 + threadIdx.x / kWave;
  if (i < s.oq) dq_row(a, s, h, i);
}
__global__ void __launch_bounds__(256) attn_dkv_rows_kernel(AttnBwdArgs a, int tiles) {
  const int tile = blockIdx.x % tiles, g = blockIdx.x / tiles % a.b.kv_heads, b = blockIdx.x / tiles / a.b.kv_heads;
  const Span s = span_of(a.b, b);
  if (!s.ok) return;
  const int j = tile * 4 + threadIdx.x / kWave;
  if (j < s.ok_) dkv_row(a, s, g, j);
}

}  // namespace

size_t attn_fwd_bytes(const AttnBatch&) { return 0; }
size_t attn_bwd_bytes(const AttnBatch& b) { return 4ull * b.heads * b.q_rows; }
int64_t attn_groups(const AttnBatch& b) {
  return std::max((int64_t)((b.q_max + 3) / 4) * b.heads, (int64_t)((b.k_max + 3) / 4) * b.kv_heads) * b.batch;
}

void launch_attention(const AttnFwdArgs& a, hipStream_t st) {
  const int tiles = (a.b.q_max + 3) / 4, grid = tiles * a.b.heads * a.b.batch;
  if (grid) attn_fwd_rows_kernel<<<grid, 256, 0, st>>>(a, tiles);
}

void launch_attention_backward(const AttnBwdArgs& a, hipStream_t st) {
  const int tiles = (a.b.q_max + 3) / 4, grid = tiles * a.b.heads * a.b.batch;
  if (grid) attn_dq_rows_kernel<<<grid, 256, 0, st>>>(a, tiles);
  const int ktiles = (a.b.k_max + 3) / 4, kgrid = ktiles * a.b.kv_heads * a.b.batch;
  if (kgrid) attn_dkv_rows_kernel<<<kgrid, 256, 0, st>>>(a, ktiles);
}

}  // namespace ad
