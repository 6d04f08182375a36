// Shared by the kernels of the draft block's training operators: typed strided matrices,
// 8-bit checkpoints, GELU and its derivative, launcher declarations.
#pragma once

#include "common.h"

namespace ad {

// A matrix of float32 or bf16 rows.  vec: 8 columns at a multiple of 8 are whole and 16-byte
// aligned.
struct DMat {
  void* p;
  int64_t ld;
  int bf16, vec;
};

// A vector of parameters (LayerNorm gain, bias): float32 or bf16.  vec: 16-byte aligned.
struct DVec {
  const void* p;
  int bf16, vec;
};

// 8-bit checkpoint rows: q [rows][ld], scale [rows][ld / 32], ld a multiple of 128.
struct DCkpt {
  int8_t* q;
  uint8_t* scale;
  int ld;
};
constexpr int kCkptGroup = 32;
inline int ckpt_ld(int cols) { return (cols + 127) / 128 * 128; }

// The widest row that a LayerNorm workgroup keeps in its registers.
constexpr int kLnMaxCols = 8192;

// ----------------------------------------------------------------- elements

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// eight bf16 of 16 bytes
__device__ __forceinline__ void widen8(u32x4 u, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(u[i] << 16);
    v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
  }
}

// Columns c .. c + 7 of a row (columns from `cols` on read as 0), in 16-byte accesses of whatever
// alignment where all eight are there.  VEC: the caller knows that m.vec.
template <bool VEC = false>
__device__ __forceinline__ void load8(const DMat& m, size_t row, int c, int cols, float (&v)[8]) {
  if (m.bf16) {
    const uint16_t* p = (const uint16_t*)m.p + row * m.ld + c;
    if (VEC || m.vec) {
      u32x4 u = {0, 0, 0, 0};
      if (c < cols) u = *(const u32x4*)p;
      widen8(u, v);
    } else if (c + 8 <= cols) {
      u32x4 u;
      __builtin_memcpy(&u, p, 16);
      widen8(u, v);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = c + i < cols ? bf16_to_f32(p[i]) : 0.f;
    }
  } else {
    const float* p = (const float*)m.p + row * m.ld + c;
    if (VEC || m.vec) {
      f32x4 a = {0.f, 0.f, 0.f, 0.f}, b = a;
      if (c < cols) {
        a = *(const f32x4*)p;
        b = *(const f32x4*)(p + 4);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
    } else if (c + 8 <= cols) {
      __builtin_memcpy(v, p, 32);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = c + i < cols ? p[i] : 0.f;
    }
  }
}

template <bool VEC = false>
__device__ __forceinline__ void store8(const DMat& m, size_t row, int c, int cols, const float (&v)[8]) {
  if (m.bf16) {
    uint16_t* p = (uint16_t*)m.p + row * m.ld + c;
    if (VEC || m.vec) {
      if (c < cols)
        *(u32x4*)p = u32x4{f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3]),
                           f32x2_to_bf16x2(v[4], v[5]), f32x2_to_bf16x2(v[6], v[7])};
    } else if (c + 8 <= cols) {
      const u32x4 u = {f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3]), f32x2_to_bf16x2(v[4], v[5]),
                       f32x2_to_bf16x2(v[6], v[7])};
      __builtin_memcpy(p, &u, 16);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (c + i < cols) p[i] = f32_to_bf16(v[i]);
    }
  } else {
    float* p = (float*)m.p + row * m.ld + c;
    if (VEC || m.vec) {
      if (c < cols) {
        *(f32x4*)p = f32x4{v[0], v[1], v[2], v[3]};
        *(f32x4*)(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
      }
    } else if (c + 8 <= cols) {
      __builtin_memcpy(p, v, 32);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (c + i < cols) p[i] = v[i];
    }
  }
}

// Elements c .. c + 7 of a parameter vector of n (0 from n on).  VEC: the caller knows that g.vec and
// n % 8 == 0.
template <bool VEC = false>
__device__ __forceinline__ void load_vec8(const DVec& g, int c, int n, float (&v)[8]) {
  if (VEC && c >= n) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
  } else if (VEC || (g.vec && c + 8 <= n)) {
    if (g.bf16) {
      widen8(*(const u32x4*)((const uint16_t*)g.p + c), v);
    } else {
      const f32x4 a = *(const f32x4*)((const float*)g.p + c), b = *(const f32x4*)((const float*)g.p + c + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      v[i] = c + i >= n ? 0.f : g.bf16 ? bf16_to_f32(((const uint16_t*)g.p)[c + i]) : ((const float*)g.p)[c + i];
  }
}

// ----------------------------------------------------------------- 8-bit checkpoints

// The scale byte of a group whose largest magnitude has these bits (sign cleared; NaN and
// infinity give 255).  amax = m 2^(E - 127), 1 <= m < 2: 127 * 2^(s - 127) >= amax first
// holds at s = E - 6 when m <= 127 / 64 (mantissa bits 0x7e0000), at E - 5 otherwise.
__device__ __forceinline__ uint32_t ckpt_scale(uint32_t amax) {
  const int s = (int)(amax >> 23) - 6 + ((amax & 0x7fffffu) > 0x7e0000u);
  return amax >= 0x7f800000u ? 255u : (uint32_t)max(s, 1);
}
// 2^(127 - s), and 0 for a group that reads as NaN
__device__ __forceinline__ float ckpt_inv(uint32_t s) { return s == 255u ? 0.f : __uint_as_float((254u - s) << 23); }
// The integer nearest to v inv (ties to even) in the low byte: |v inv| <= 127, so adding
// 1.5 * 2^23 in one rounding leaves it in the low mantissa bits.
__device__ __forceinline__ uint32_t ckpt_round(float v, float inv) {
  return __float_as_uint(fmaf(v, inv, 12582912.f));
}
// four low bytes in one word
__device__ __forceinline__ uint32_t pack_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  const uint32_t ab = __builtin_amdgcn_perm(b, a, 0x0c0c0400u), cd = __builtin_amdgcn_perm(d, c, 0x0c0c0400u);
  return __builtin_amdgcn_perm(cd, ab, 0x05040100u);
}
// (s = 255: infinity, and every q of the group is 0, so the product is NaN)
__device__ __forceinline__ float ckpt_two(uint32_t s) { return __uint_as_float(s << 23); }
// Four values q * two, exact up to float32's range (2^128 is an infinity).  A signed byte converts in one
// instruction; as (q + 128 - 128) two from unsigned ones the weight gradient of 14336 rows from a checkpoint
// took 240 us in place of 225.  (q + 128) two - 128 two has no place here: 128 two overflows from s = 248 on.
__device__ __forceinline__ void ckpt_value4(uint32_t w, float two, float (&v)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = (float)(int8_t)(w >> (8 * i)) * two;
}
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// Eight values as bytes, and their group's scale: four neighbouring lanes, all of them active, hold one
// group of 32.  Lanes with in = false hold padding.
__device__ __forceinline__ u32x2 ckpt_of8(bool in, const float (&v)[8], uint32_t& s) {
  uint32_t m = abs_bits(v[0]);
#pragma unroll
  for (int i = 1; i < 8; ++i) m = max(m, abs_bits(v[i]));
  m = in ? m : 0;
  m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xf, 0xf, false));   // lane ^ 1
  m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xf, 0xf, false));   // lane ^ 2
  s = ckpt_scale(m);
  const float inv = ckpt_inv(s);
  const u32x2 w = {pack_bytes(ckpt_round(v[0], inv), ckpt_round(v[1], inv), ckpt_round(v[2], inv), ckpt_round(v[3], inv)),
                   pack_bytes(ckpt_round(v[4], inv), ckpt_round(v[5], inv), ckpt_round(v[6], inv), ckpt_round(v[7], inv))};
  return in && s != 255u ? w : u32x2{0, 0};
}
// Columns c .. c + 7 (c a multiple of 8) into a checkpoint row; v is 0 from the last column on.
__device__ __forceinline__ void ckpt_store8(const DCkpt& k, size_t row, int c, const float (&v)[8]) {
  uint32_t s;
  const u32x2 w = ckpt_of8(true, v, s);
  if (c < k.ld) {
    *(u32x2*)(k.q + row * k.ld + c) = w;
    if (c % kCkptGroup == 0) k.scale[row * (size_t)(k.ld / kCkptGroup) + c / kCkptGroup] = (uint8_t)s;
  }
}
__device__ __forceinline__ void ckpt_value8(u32x2 w, uint32_t s, float (&v)[8]) {
  const float two = ckpt_two(s);
  float a[4], b[4];
  ckpt_value4(w[0], two, a);
  ckpt_value4(w[1], two, b);
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
}
// Columns c .. c + 7 of a checkpoint row (0 past the padded row).
__device__ __forceinline__ void ckpt_load8(const DCkpt& k, size_t row, int c, float (&v)[8]) {
  u32x2 w = {0, 0};
  uint32_t s = 1;
  if (c < k.ld) {
    w = *(const u32x2*)(k.q + row * k.ld + c);
    s = k.scale[row * (size_t)(k.ld / kCkptGroup) + c / kCkptGroup];
  }
  ckpt_value8(w, s, v);
}

// ----------------------------------------------------------------- GELU

// Phi(h) and e = exp(-h^2 / 2), from erf's rational approximation in Abramowitz and Stegun, Handbook of
// Mathematical Functions, 7.1.26 (absolute error 1.5e-7 in erf): for x = |h| / sqrt(2),
//   1 - erf(x) = (a1 t + a2 t^2 + a3 t^3 + a4 t^4 + a5 t^5) exp(-x^2),  t = 1 / (1 + p x).
// One exponential serves the value and the slope (gradients); erff() alone takes about three times as long,
// and the epilogues that call this are as long as a quarter of their product.
struct Normal {
  float tail, e;   // 1 - Phi(|h|)
};
__device__ __forceinline__ Normal normal(float h) {
  const float e = __builtin_amdgcn_exp2f(h * h * -0.72134752044448170f);          // -log2(e) / 2
  const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(h), 0.23164189f, 1.0f));        // p / sqrt(2)
  float q = fmaf(t, 0.5f * 1.061405429f, 0.5f * -1.453152027f);
  q = fmaf(q, t, 0.5f * 1.421413741f);
  q = fmaf(q, t, 0.5f * -0.284496736f);
  q = fmaf(q, t, 0.5f * 0.254829592f);
  return Normal{q * t * e, e};
}
// h Phi(h) = max(h, 0) - |h| (1 - Phi(|h|)); |h| is kept finite, for h = inf (NaN comes through the tail)
__device__ __forceinline__ float gelu_value(float h, Normal n) {
  return fmaf(-fminf(fabsf(h), 1e30f), n.tail, fmaxf(h, 0.f));
}
// The value alone: 1 - Phi(|h|) = 2^p(|h|), p a polynomial fitted to log2(1 - Phi) on [0, 6.2] by least
// squares with weights Phi's tail, reweighted to level the error (5e-8 in Phi, float32 steps
// included).  From there on p falls to -infinity and the tail is 0.  No reciprocal: five of 20
// instruction slots less than above.
__device__ __forceinline__ float gelu_value(float h) {
  const float x = fabsf(h);
  float p = fmaf(-2.7720503e-6f, x, 3.8620758e-5f);
  p = fmaf(p, x, -1.8254764e-4f);
  p = fmaf(p, x, -1.4587007e-4f);
  p = fmaf(p, x, 7.0754718e-3f);
  p = fmaf(p, x, -5.2505028e-2f);
  p = fmaf(p, x, -4.5920491e-1f);
  p = fmaf(p, x, -1.1511058f);
  p = fmaf(p, x, -1.0f);
  return fmaf(-fminf(x, 1e30f), __builtin_amdgcn_exp2f(p), fmaxf(h, 0.f));
}
// d/dh (h Phi(h)) = Phi(h) + h phi(h); h is kept finite likewise: 1 at infinity, 0 at -infinity
__device__ __forceinline__ float gelu_slope(float h, Normal n) {
  return fmaf(__builtin_amdgcn_fmed3f(h, -1e30f, 1e30f), 0.39894228040143268f * n.e, h >= 0.f ? 1.0f - n.tail : n.tail);
}

// ----------------------------------------------------------------- launchers

struct LnFwdArgs {
  int rows, cols;
  DMat x, y;
  DVec gain, bias;
  float *mean, *rstd;   // or NULL
  DCkpt xhat;           // q NULL: none
};
void launch_layer_norm(const LnFwdArgs& a, hipStream_t st);

struct LnBwdArgs {
  int rows, cols;
  DMat dy, x, dres, dx, copy;   // p NULL: absent
  DVec gain;
  const float *mean, *rstd;
  DCkpt xhat;
  float *dgain, *dbias;         // or NULL
  int accumulate;
  float* part;                  // [workgroups][2][cols]
};
int ln_bwd_groups(int rows, int cols);
void launch_layer_norm_backward(const LnBwdArgs& a, hipStream_t st);

void launch_ckpt_pack(int rows, int cols, const DMat& x, const DCkpt& k, hipStream_t st);
void launch_ckpt_unpack(int rows, int cols, const DCkpt& k, bool gelu, const DMat& out, hipStream_t st);

// One operand of a product, along its output dimension (`extent`) and the reduction.
struct LinOp {
  const uint16_t* p;     // bf16, or NULL: the checkpoint
  int64_t ld;
  DCkpt ck;
  int extent;
};
enum LinKind : int { LIN_FWD = 0, LIN_DGRAD = 1, LIN_WGRAD = 2 };
// out[q][p] = sum over K of Q(q, .) P(p, .) with the epilogue of the kind.
struct LinArgs {
  LinOp P, Q;
  int K;
  // set by the launcher: the tiles, how many of them are computed whole, and the parts of the
  // reduction (of `steps` 64-wide steps each) that the others are computed in
  int tiles_p, tiles_q, whole, S, steps;
  float* part;           // S > 1: partial tiles [S][tiles - whole], then (wgrad) their rows' sums of dy
  float* part_sum;
  // epilogue
  DVec bias, gain, shift;
  int gelu, accumulate;
  DMat res, out, pre, act_out;
  DCkpt ck;              // fwd: the pre-activation out; dgrad: in
  float* dbias;
};
// Floats of workspace of a product of this kind with these extents.
size_t lin_part_floats(int kind, int P, int Q, int K);
void launch_linear(int kind, LinArgs a, hipStream_t st);

}  // namespace ad
