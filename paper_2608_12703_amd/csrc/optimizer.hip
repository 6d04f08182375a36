// AdamW over many tensors in one launch, 8-bit states, and the gradients' norm.
//
// All of it streams each tensor once: the floor is HBM traffic.  A workgroup takes kChunk elements of
// one tensor (the tensors of a launch are kernel arguments, found by their first workgroup), a
// lane 4 consecutive elements at a time, so that a wave's float32 access is 1 KB side by side.
//
// Measured for a draft block of 29.5 million parameters (a large copy reaches 5.2 TB/s): float32 states with bf16 copies
// 156 us for 885 MB (5.7 TB/s; 159 a pass, 160 with step and rate on the device), 8-bit states 100 us for 535 MB, their values
// read back 44 us for 295 MB (6.6), bf16 parameters with float32 states 115 us for 708 MB (6.1; 8-bit states 95), the norm
// 19 + 4 us for 118 MB.  17 vectors of 8064 elements in all: 4.9 us a pass, 5.6 with step and rate on the device, whose 64-bit
// scalars a thread of each workgroup computes before its loads.
// Float32 goes past the caches (nontemporal): what a step reads it does not read again before the next one.  Through the
// caches the first took 187 us and the third 107 (stores alone past them: 183 and 50); 8 elements a lane 197 and 116.  Bytes
// go through the caches: past them a byte-aligned word became four accesses (86 us).
#include <algorithm>

#include "train.h"
#include "top2.h"

namespace ad {

namespace {

constexpr int kPass = 1024, kChunk = kOptChunk;   // elements that a workgroup has at once, and in all
static_assert(kChunk % kPass == 0, "whole passes");
constexpr int kGroup = 128;                       // elements that share a scale: 32 lanes

// ----------------------------------------------------------------- elements of any alignment

constexpr int kE = 4;                             // consecutive elements of a lane: 16 bytes of float32

typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
// (KEEP: through the caches, for what is read again soon)
template <bool KEEP = false>
__device__ __forceinline__ void get(const float* p, int n, float (&v)[kE]) {
  if (n >= kE) {
    const f4 u = KEEP ? *(const f4*)p : __builtin_nontemporal_load((const f4*)p);
#pragma unroll
    for (int i = 0; i < kE; ++i) v[i] = u[i];
  } else {
#pragma unroll
    for (int i = 0; i < kE; ++i) v[i] = i < n ? p[i] : 0.f;
  }
}
__device__ __forceinline__ void put(float* p, int n, const float (&v)[kE]) {
  if (n >= kE) {
    __builtin_nontemporal_store(f4{v[0], v[1], v[2], v[3]}, (f4*)p);
  } else {
#pragma unroll
    for (int i = 0; i < kE; ++i)
      if (i < n) p[i] = v[i];
  }
}
__device__ __forceinline__ void get(const uint16_t* p, int n, float (&v)[kE]) {
  if (n >= kE) {
    u32x2 u;
    __builtin_memcpy(&u, p, 8);
#pragma unroll
    for (int i = 0; i < kE; ++i) v[i] = __uint_as_float(i % 2 ? u[i / 2] & 0xffff0000u : u[i / 2] << 16);
  } else {
#pragma unroll
    for (int i = 0; i < kE; ++i) v[i] = i < n ? bf16_to_f32(p[i]) : 0.f;
  }
}
__device__ __forceinline__ void put(uint16_t* p, int n, u32x2 u) {
  if (n >= kE) {
    __builtin_memcpy(p, &u, 8);
  } else {
#pragma unroll
    for (int i = 0; i < kE; ++i)
      if (i < n) p[i] = (uint16_t)(u[i / 2] >> (16 * (i % 2)));
  }
}
__device__ __forceinline__ u32x2 narrow(const float (&v)[kE]) {
  return u32x2{f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3])};
}
__device__ __forceinline__ uint32_t get_bytes(const void* p, int n) {
  uint32_t u = 0;
  if (n >= kE) {
    __builtin_memcpy(&u, p, 4);
  } else {
#pragma unroll
    for (int i = 0; i < kE; ++i)
      if (i < n) u |= (uint32_t)((const uint8_t*)p)[i] << (8 * i);
  }
  return u;
}
__device__ __forceinline__ void put_bytes(void* p, int n, uint32_t u) {
  if (n >= kE) {
    __builtin_memcpy(p, &u, 4);
  } else {
#pragma unroll
    for (int i = 0; i < kE; ++i)
      if (i < n) ((uint8_t*)p)[i] = (uint8_t)(u >> (8 * i));
  }
}

// ----------------------------------------------------------------- 8-bit states

// 32 random bits of 32: exclusive-ors of shifts between products with odd constants (the fractions of
// the square roots of 2 and 3); elements are the golden ratio's fraction apart.
constexpr uint32_t kGolden = 0x9E3779B9u;
__host__ __device__ __forceinline__ uint32_t mix(uint32_t x) {
  x ^= x >> 16;
  x *= 0x6A09E667u;
  x ^= x >> 15;
  x *= 0xBB67AE85u;
  return x ^ (x >> 16);
}
// 16 bits as a threshold inside (0, 1); exact
__device__ __forceinline__ float threshold(uint32_t bits) { return ((float)bits + 0.5f) * (1.0f / 65536.0f); }

// Largest of 32 lanes, as the bits of magnitudes (a NaN is larger than an infinity).
__device__ __forceinline__ uint32_t group_max(uint32_t m) {
  m = max(m, (uint32_t)ror16<8>((int)m));
  m = max(m, (uint32_t)ror16<4>((int)m));
  m = max(m, (uint32_t)ror16<2>((int)m));
  m = max(m, (uint32_t)ror16<1>((int)m));
  const auto r = __builtin_amdgcn_permlane16_swap(m, m, false, false);
  return max(r[0], r[1]);
}
constexpr uint32_t kTiny = 0x0d800000u;           // 2^-100
constexpr uint32_t kInf = 0x7f800000u;

// scale = top / unit and its inverse, of a group whose largest magnitude has the bits `top`; a group under
// 2^-100 is all zeros (scale 0), one that is not finite reads as NaN.
__device__ __forceinline__ void scale_of(uint32_t top, float unit, float& scale, float& inv) {
  const bool none = top < kTiny, bad = top >= kInf;
  const float t = __uint_as_float(none || bad ? 0x3f800000u : top);
  scale = none ? 0.f : bad ? __uint_as_float(0x7fc00000u) : t / unit;
  inv = none || bad ? 0.f : unit / t;
}

__device__ __forceinline__ int code_m(float m, float inv, float r) {
#pragma clang fp contract(off)
  const float x = m * inv, low = floorf(x);
  const float q = low + (x - low > r ? 1.f : 0.f);
  return (int)__builtin_amdgcn_fmed3f(q, -127.f, 127.f);
}
// x = v inv in [0, 65025]: the root's whole part by an approximate root and one comparison each way
// (squares of whole numbers up to 256 are exact)
__device__ __forceinline__ int code_v(float v, float inv, float r) {
#pragma clang fp contract(off)
  const float x = v * inv;
  float low = floorf(__builtin_amdgcn_sqrtf(x));
  if (low * low > x) low -= 1.f;
  if ((low + 1.f) * (low + 1.f) <= x) low += 1.f;
  const float q = low + (x - low * low > r * (2.f * low + 1.f) ? 1.f : 0.f);
  return (int)__builtin_amdgcn_fmed3f(q, v > 0.f && inv > 0.f ? 1.f : 0.f, 255.f);
}
__device__ __forceinline__ void value_m(uint32_t q, float s, float (&v)[kE]) {
#pragma unroll
  for (int i = 0; i < kE; ++i) v[i] = (float)(int8_t)(q >> (8 * i)) * s;
}
__device__ __forceinline__ void value_v(uint32_t q, float s, float (&v)[kE]) {
#pragma clang fp contract(off)
#pragma unroll
  for (int i = 0; i < kE; ++i) {
    const float r = (float)(uint8_t)(q >> (8 * i));
    v[i] = r * r * s;
  }
}

// ----------------------------------------------------------------- the step

// The tensor that a workgroup works on, and its place in it.
__device__ __forceinline__ int find(const OptList& l, int block) {
  const int i = threadIdx.x % kWave;
  return __popcll(__ballot(i < l.count && l.first[min(i, kOptTensors)] <= block)) - 1;
}

struct Hyper {
  float root, rate;
  uint32_t key;
  float lr;
  int fine;       // step and lr are what the host takes
};

template <bool STATE8>
__device__ __forceinline__ void adamw_pass(const OptTensor& t, const AdamwArgs& a, const Hyper& y, float keep, float gs,
                                           uint32_t key, int64_t i) {
#pragma clang fp contract(off)
  const int n = (int)min(t.n - i, (int64_t)kE);          // may be <= 0: the lane only takes part in its group
  float p[kE] = {}, g[kE] = {}, m[kE] = {}, v[kE] = {};
  if (n > 0) {
    if (t.kinds & OPT_GRAD16) get((const uint16_t*)t.grad + i, n, g);
    else get((const float*)t.grad + i, n, g);
    if (STATE8) {
      value_m(get_bytes((const int8_t*)t.m + i, n), t.m_scale[i / kGroup], m);
      value_v(get_bytes((const uint8_t*)t.v + i, n), t.v_scale[i / kGroup], v);
    } else {
      get((const float*)t.m + i, n, m);
      get((const float*)t.v + i, n, v);
    }
    if (t.kinds & OPT_PARAM16) get((const uint16_t*)t.param + i, n, p);
    else get((const float*)t.param + i, n, p);
  }
  uint32_t bits[kE];
#pragma unroll
  for (int e = 0; e < kE; ++e) bits[e] = mix(key + (uint32_t)(i + e) * kGolden);
  uint32_t top_m = 0, top_v = 0;
#pragma unroll
  for (int e = 0; e < kE; ++e) {
    const float ge = g[e] * gs;
    m[e] = m[e] * a.b1 + ge * a.ob1;
    v[e] = v[e] * a.b2 + ge * ge * a.ob2;
    const float den = __builtin_amdgcn_sqrtf(v[e]) * y.root + a.eps;
    p[e] = p[e] * keep - m[e] * __builtin_amdgcn_rcpf(den) * y.rate;
    if (STATE8) {
      top_m = max(top_m, e < n ? abs_bits(m[e]) : 0u);
      top_v = max(top_v, e < n ? abs_bits(v[e]) : 0u);
    }
  }
  if (n > 0) {
    if (t.kinds & OPT_PARAM16) {
      u32x2 u = {0, 0};
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        const uint32_t b = __float_as_uint(p[e]);
        const uint32_t up = (b & kInf) == kInf ? (uint32_t)f32_to_bf16(p[e]) : (b + (mix(bits[e] + kGolden) & 0xffffu)) >> 16;
        u[e / 2] |= up << (16 * (e % 2));
      }
      put((uint16_t*)t.param + i, n, u);
    } else {
      put((float*)t.param + i, n, p);
      if (t.copy) put((uint16_t*)t.copy + i, n, narrow(p));
    }
    if (!STATE8) {
      put((float*)t.m + i, n, m);
      put((float*)t.v + i, n, v);
    }
  }
  if (STATE8) {
    float ms, mi, vs, vi;
    scale_of(group_max(top_m), 127.f, ms, mi);
    scale_of(group_max(top_v), 65025.f, vs, vi);
    if (n > 0) {
      uint32_t cm[kE], cv[kE];
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        cm[e] = (uint32_t)code_m(m[e], mi, threshold(bits[e] & 0xffffu));
        cv[e] = (uint32_t)code_v(v[e], vi, threshold(bits[e] >> 16));
      }
      const uint32_t qm = pack_bytes(cm[0], cm[1], cm[2], cm[3]), qv = pack_bytes(cv[0], cv[1], cv[2], cv[3]);
      put_bytes((int8_t*)t.m + i, n, qm);
      put_bytes((uint8_t*)t.v + i, n, qv);
      if (i % kGroup == 0) {
        t.m_scale[i / kGroup] = ms;
        t.v_scale[i / kGroup] = vs;
      }
    }
  }
}

__global__ void __launch_bounds__(256) adamw_kernel(OptList l, AdamwArgs a) {
  __shared__ Hyper shared;
  const OptTensor& t = l.t[find(l, blockIdx.x)];
  Hyper y = {a.root, a.rate, a.key, 0.f, 1};
  float keep = t.keep;
  if (a.lr_at || a.step_at) {
    if (threadIdx.x == 0) {
      const int step = a.step_at ? *a.step_at : a.step;
      const double lr = a.lr_at ? (double)*a.lr_at : a.lr;
      shared.root = (float)(1.0 / sqrt(-expm1(step * log(a.beta2))));
      shared.rate = (float)(lr / -expm1(step * log(a.beta1)));
      shared.key = mix(a.seed + kGolden * (uint32_t)step);
      shared.lr = (float)lr;
      shared.fine = step >= 1 && lr >= 0.0 && lr < INFINITY;
    }
    __syncthreads();
    y = shared;
    keep = (float)(1.0 - (double)y.lr * (double)t.decay);
  }
  const float gs = a.scale ? *a.scale : 1.f;
  if (!y.fine || !(fabsf(gs) < INFINITY)) return;
  const uint32_t key = mix(t.key + y.key);
  const int64_t base = (int64_t)(blockIdx.x - l.first[&t - l.t]) * kChunk;
  for (int c = 0; c < kChunk; c += kPass) {
    const int64_t i = base + c + kE * threadIdx.x;
    if (base + c >= t.n) break;
    if (t.kinds & OPT_STATE8) adamw_pass<true>(t, a, y, keep, gs, key, i);
    else adamw_pass<false>(t, a, y, keep, gs, key, i);
  }
}

struct StateAt {
  int64_t at[kOptTensors];     // where a tensor's values begin in m and v
};
__global__ void __launch_bounds__(256) opt_state_kernel(OptList l, StateAt s, float* m, float* v) {
  const int k = find(l, blockIdx.x);
  const OptTensor& t = l.t[k];
  const int64_t base = (int64_t)(blockIdx.x - l.first[k]) * kChunk;
  for (int c = 0; c < kChunk; c += kPass) {
    const int64_t i = base + c + kE * threadIdx.x;
    const int n = (int)min(t.n - i, (int64_t)kE);
    if (n <= 0) break;
    float x[kE];
    if (m) {
      if (t.kinds & OPT_STATE8) value_m(get_bytes((const int8_t*)t.m + i, n), t.m_scale[i / kGroup], x);
      else get((const float*)t.m + i, n, x);
      put(m + s.at[k] + i, n, x);
    }
    if (v) {
      if (t.kinds & OPT_STATE8) value_v(get_bytes((const uint8_t*)t.v + i, n), t.v_scale[i / kGroup], x);
      else get((const float*)t.v + i, n, x);
      put(v + s.at[k] + i, n, x);
    }
  }
}

// ----------------------------------------------------------------- the norm

__device__ __forceinline__ double block_total(double s, double* red) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) s += __shfl_xor(s, o, kWave);
  if (threadIdx.x % kWave == 0) red[threadIdx.x / kWave] = s;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

// Consecutive elements from i on, n of them there.
__device__ __forceinline__ void add_squares(const OptTensor& t, int64_t i, int n, double& s) {
  float g[kE];
  if (t.kinds & OPT_GRAD16) get((const uint16_t*)t.grad + i, n, g);
  else get<true>((const float*)t.grad + i, n, g);      // (the step reads them next)
#pragma unroll
  for (int e = 0; e < kE; ++e) s = fma((double)g[e], (double)g[e], s);
}

__global__ void __launch_bounds__(256) grad_squares_kernel(OptList l, double* part) {
  __shared__ double red[4];
  const int k = find(l, blockIdx.x);
  const OptTensor& t = l.t[k];
  const int64_t base = (int64_t)(blockIdx.x - l.first[k]) * kChunk;
  double s = 0.0;
  for (int c = 0; c < kChunk; c += kPass) {
    const int64_t i = base + c + kE * threadIdx.x;
    const int n = (int)min(t.n - i, (int64_t)kE);
    if (n <= 0) break;
    add_squares(t, i, n, s);
  }
  s = block_total(s, red);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// out and step from 16 waves' sums
__device__ __forceinline__ void norm_out(double s, double max_norm, float* out, int* step) {
  __shared__ double red[16];
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) s += __shfl_xor(s, o, kWave);
  if (threadIdx.x % kWave == 0) red[threadIdx.x / kWave] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = red[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) s += red[i];
    const double norm = sqrt(s);
    out[0] = (float)norm;
    const bool fine = (float)norm < INFINITY;           // (NaN is not)
    out[1] = !fine ? __uint_as_float(0x7fc00000u) : max_norm > 0.0 && norm > max_norm ? (float)(max_norm / norm) : 1.f;
    if (step && fine) *step += 1;
  }
}

__global__ void __launch_bounds__(1024) grad_norm_kernel(const double* part, int64_t parts, double max_norm, float* out,
                                                         int* step) {
  double s = 0.0;
#pragma unroll 4
  for (int64_t i = threadIdx.x; i < parts; i += 1024) s += part[i];
  norm_out(s, max_norm, out, step);
}

// Few elements: sixteen waves take pieces of kPiece of the tensors in turn (first: in pieces), and there is no second
// launch.
constexpr int kPiece = 1024;
__global__ void __launch_bounds__(1024) grad_norm_few_kernel(OptList l, double max_norm, float* out, int* step) {
  const int lane = threadIdx.x % kWave, w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  double s = 0.0;
  for (int g = w; g < l.first[l.count]; g += 16) {
    const int k = find(l, g);
    const OptTensor& t = l.t[k];
#pragma unroll
    for (int c = 0; c < kPiece; c += kE * kWave) {
      const int64_t i = (int64_t)(g - l.first[k]) * kPiece + c + kE * lane;
      const int n = (int)min(t.n - i, (int64_t)kE);
      if (n > 0) add_squares(t, i, n, s);
    }
  }
  norm_out(s, max_norm, out, step);
}

}  // namespace

void launch_adamw(const OptList& l, AdamwArgs a, hipStream_t st) {
  a.key = mix(a.seed + kGolden * (uint32_t)a.step);
  if (l.first[l.count]) adamw_kernel<<<l.first[l.count], 256, 0, st>>>(l, a);
}
void launch_opt_state(const OptList& l, float* m, float* v, const int64_t* at, hipStream_t st) {
  StateAt s{};
  for (int i = 0; i < l.count; ++i) s.at[i] = at[i];
  if (l.first[l.count]) opt_state_kernel<<<l.first[l.count], 256, 0, st>>>(l, s, m, v);
}
void launch_grad_squares(const OptList& l, double* part, hipStream_t st) {
  if (l.first[l.count]) grad_squares_kernel<<<l.first[l.count], 256, 0, st>>>(l, part);
}
// Three rounds of the sixteen waves: 17 vectors of 1000 elements 6.0 us instead of 8.2, 40 of them 6.9 and 8.3; at four
// rounds (one tensor of 65536) 8.0 and 8.1, at five 9.5 and 8.4.
bool norm_of_few(const OptList& l) {
  int64_t pieces = 0;
  for (int k = 0; k < l.count; ++k) pieces += (l.t[k].n + kPiece - 1) / kPiece;
  return pieces <= 48;
}
void launch_grad_norm_few(OptList l, double max_norm, float* out, int* step, hipStream_t st) {
  for (int k = 0; k < l.count; ++k) l.first[k + 1] = l.first[k] + (int)((l.t[k].n + kPiece - 1) / kPiece);
  grad_norm_few_kernel<<<1, 1024, 0, st>>>(l, max_norm, out, step);
}
void launch_grad_norm(const double* part, int64_t parts, double max_norm, float* out, int* step, hipStream_t st) {
  grad_norm_kernel<<<1, 1024, 0, st>>>(part, parts, max_norm, out, step);
}

}  // namespace ad
