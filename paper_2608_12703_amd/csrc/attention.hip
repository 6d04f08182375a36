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
      o = fmaf(p, at(a.v, s.k0 + j, 64 * g + d), o);
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

// ----------------------------------------------------------------- matrix-core pieces
// v_mfma_f32_32x32x16_bf16: lane l supplies row (A) or column (B) l % 32 and reduction elements
// 8 (l / 32) .. + 7, and receives of column l % 32 the rows 8 (i / 4) + 4 (l / 32) + i % 4, i = 0 .. 15.
//
// Everything is computed transposed, keys on the rows and queries on the columns (S^T = K Q^T), so a lane has
// scores of one query only, and its sixteen scores of 32 keys are two B operands of the product that follows
// (O^T = V^T P^T): element e of half h of 16 keys is key 8 (e / 4) + 4 h + e % 4, and the other operand is
// read in that order.

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// Tiles of 64-wide rows in LDS: 128 bytes a row, its 16-byte pieces c at c ^ (row % 8), so that eight rows'
// same piece lies in different banks.
constexpr int kRowBytes = 128;

// A lane's place in a tile, as the A operand whose rows are the tile's rows (`row`: piece 2 s + h of row
// l % 32), and as the one whose rows are the tile's columns (`col`: 16 lanes read 4 rows of 16 columns).
struct Lane {
  uint32_t row, col;
  int h, n;       // l / 32, l % 32
  __device__ __forceinline__ explicit Lane(int l) {
    h = l >> 5;
    n = l & 31;
    row = n * kRowBytes + ((h ^ (n & 7)) << 4);
    const int c16 = l & 15, r = 4 * h + (c16 >> 2), piece = 2 * ((l >> 4) & 1) + ((c16 & 3) >> 1);
    col = r * kRowBytes + ((piece ^ r) << 4) + (c16 & 1) * 8;
  }
};
// rows 32 b .. + 31, columns 16 s .. + 15 as the reduction
__device__ __forceinline__ bf16x8 read_rows(const char* tile, const Lane& l, int b, int s) {
  return as_bf16x8(*(const uint4*)(tile + b * 32 * kRowBytes + (l.row ^ (s * 32))));
}
// columns 32 b .. + 31, rows 16 c .. + 15 as the reduction (in the order above)
__device__ __forceinline__ bf16x8 read_cols(const char* tile, const Lane& l, int b, int c) {
  typedef __attribute__((address_space(3))) s16x4* lp;
  const char* p = tile + c * 16 * kRowBytes + (l.col ^ (b * 64));
  const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)p);
  const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(p + 8 * kRowBytes));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
}
// eight values of a lane's column as an operand
__device__ __forceinline__ bf16x8 narrow(const f32x16& v, int e) {
  return as_bf16x8(make_uint4(f32x2_to_bf16x2(v[e], v[e + 1]), f32x2_to_bf16x2(v[e + 2], v[e + 3]),
                              f32x2_to_bf16x2(v[e + 4], v[e + 5]), f32x2_to_bf16x2(v[e + 6], v[e + 7])));
}
// with the lane that has the same column's other rows
__device__ __forceinline__ float other_half(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(threadIdx.x & 32 ? r[0] : r[1]);
}
__device__ __forceinline__ f32x16 zeros() {
  f32x16 z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.f;
  return z;
}

// 16 bytes of a row, whatever their alignment
__device__ __forceinline__ uint4 load16(const uint16_t* p) {
  uint4 u;
  __builtin_memcpy(&u, p, 16);
  return u;
}

// A tile of TR rows on its way from memory to LDS: thread t of 256 takes 16-byte piece t % 8 of rows
// t / 8 + 32 j.  Rows from n on (counted from the first of the sequence) become zeros.
template <int TR>
struct Stage {
  static constexpr int N = TR / 32;
  uint4 reg[N];
  __device__ __forceinline__ void load(const HMat& m, int first, int n, int col, int r0) {
    const int t = threadIdx.x, r = r0 + t / 8;
    const uint16_t* p = m.p + (first + (int64_t)r) * m.ld + col + (t % 8) * 8;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      reg[j] = make_uint4(0, 0, 0, 0);
      if (r + 32 * j < n) reg[j] = load16(p + (int64_t)(32 * j) * m.ld);
    }
  }
  __device__ __forceinline__ void store(char* tile) const {
    const int t = threadIdx.x, r = t / 8;
#pragma unroll
    for (int j = 0; j < N; ++j) *(uint4*)(tile + (r + 32 * j) * kRowBytes + (((t % 8) ^ (r & 7)) << 4)) = reg[j];
  }
};

// The tiles of one (sequence, head) follow each other on one of the eight XCDs, whose L2 then has its
// keys: workgroup id i runs on XCD i % 8.
struct Place {
  int b, h, tile;
  bool in;
};
__device__ __forceinline__ Place place_of(int tiles, int heads, int batch, bool last_first) {
  const int slot = blockIdx.x / 8, pair = slot / tiles * 8 + blockIdx.x % 8, t = slot % tiles;
  Place r;
  r.b = pair / heads;
  r.h = pair % heads;
  r.tile = last_first ? tiles - 1 - t : t;
  r.in = pair < batch * heads;
  return r;
}
int64_t places(int64_t tiles, int64_t heads, int64_t batch) { return (heads * batch + 7) / 8 * 8 * tiles; }

__device__ __forceinline__ int wave_min(int v) {
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) v = min(v, __shfl_xor(v, o, kWave));
  return v;
}
__device__ __forceinline__ int wave_most(int v) {
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) v = max(v, __shfl_xor(v, o, kWave));
  return v;
}
// What 32 queries (one a column, both halves alike) see together.
struct Range {
  int lo, hi;          // some of them may see [lo, hi)
  int all_lo, all_hi;  // all of them see [all_lo, all_hi)
};
__device__ __forceinline__ Range range_of(const Keys& k, bool in) {
  const bool some = in && k.lo < k.hi;
  Range r;
  r.lo = wave_min(some ? k.lo : 0x7fffffff);
  r.hi = wave_most(some ? k.hi : 0);
  r.all_lo = wave_most(in ? k.lo : 0);
  r.all_hi = wave_min(in ? k.hi : 0x7fffffff);
  return r;
}

// ----------------------------------------------------------------- forward

// QW waves of 32 queries each share tiles of keys (QW = 4), or four waves share 32 queries and take a
// quarter of each tile (QW = 1), where there are few queries.  One pass over the keys with the running
// maximum m and sum l; the maximum that is taken off is only moved when a score exceeds it by 8 (in
// powers of two), which keeps p under 256.
constexpr float kLazy = 8.f;

template <int QW>
__global__ void __launch_bounds__(256) attn_fwd_kernel(AttnFwdArgs a, int tiles, int splits, int chunk) {
  constexpr int TK = QW == 4 ? 64 : 128, NB = QW == 4 ? 2 : 1, kTileBytes = TK * kRowBytes;
  __shared__ __attribute__((aligned(16))) char lds[4 * kTileBytes];   // two stages of keys and values
  __shared__ int ends[8];
  const int split = blockIdx.x % splits;
  const int slot = blockIdx.x / splits / 8, pair = slot / tiles * 8 + blockIdx.x / splits % 8;
  const int b = pair / a.b.heads, h = pair % a.b.heads;
  const int tile = a.b.causal ? tiles - 1 - slot % tiles : slot % tiles;
  if (pair >= a.b.batch * a.b.heads) return;
  const Span s = span_of(a.b, b);
  if (!s.ok) {
    if (threadIdx.x == 0) atomicOr(a.b.err, AD_ERR_LENGTH);
    return;
  }
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), g = h / (a.b.heads / a.b.kv_heads);
  const Lane l(threadIdx.x % kWave);
  const int q0 = tile * 32 * QW + (QW == 4 ? 32 * w : 0), i = q0 + l.n;
  if (tile * 32 * QW >= s.oq) return;
  const bool in = i < s.nq;
  Keys keys = {0, s.nk};
  if (in) keys = keys_of(a.b, s, i);
  if (splits > 1) {
    keys.lo = max(keys.lo, split * chunk);
    keys.hi = min(keys.hi, (split + 1) * chunk);
  }
  const Range r = range_of(keys, in);

  bf16x8 q[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    uint4 u = make_uint4(0, 0, 0, 0);
    if (in) u = load16(a.q.p + (s.q0 + (int64_t)i) * a.q.ld + 64 * h + 16 * k + 8 * l.h);
    q[k] = as_bf16x8(u);
  }

  int first = r.lo, last = r.hi;
  if (QW == 4) {
    if (threadIdx.x % kWave == 0) {
      ends[w] = r.lo;
      ends[4 + w] = r.hi;
    }
    __syncthreads();
    first = min(min(ends[0], ends[1]), min(ends[2], ends[3]));
    last = max(max(ends[4], ends[5]), max(ends[6], ends[7]));
  }
  first = first / TK * TK;

  float m = -INFINITY, sum = 0.f;
  f32x16 o[2] = {zeros(), zeros()};
  Stage<TK> ks, vs;
  if (first < last) {
    ks.load(a.k, s.k0, s.nk, 64 * g, first);
    vs.load(a.v, s.k0, s.nk, 64 * g, first);
    ks.store(lds);
    vs.store(lds + kTileBytes);
  }
  __syncthreads();
  for (int k0 = first, at = 0; k0 < last; k0 += TK, at ^= 2 * kTileBytes) {
    const bool more = k0 + TK < last;
    if (more) {
      ks.load(a.k, s.k0, s.nk, 64 * g, k0 + TK);
      vs.load(a.v, s.k0, s.nk, 64 * g, k0 + TK);
    }
    const int mine = QW == 4 ? k0 : k0 + 32 * w;            // this wave's first key
    if (mine < r.hi && mine + 32 * NB > r.lo) {
      const char* kt = lds + at + (QW == 4 ? 0 : w * 32 * kRowBytes);
      const char* vt = kt + kTileBytes;
      f32x16 x[NB];
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        x[n] = zeros();
#pragma unroll
        for (int k = 0; k < 4; ++k) x[n] = mfma32(read_rows(kt, l, n, k), q[k], x[n]);
      }
      if (mine < r.all_lo || mine + 32 * NB > r.all_hi) {
        const int lo = keys.lo - mine - 4 * l.h;
        const unsigned len = max(keys.hi - keys.lo, 0);
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            x[n][e] = (unsigned)(32 * n + 8 * (e / 4) + e % 4 - lo) < len ? x[n][e] : -INFINITY;
      }
      float top = x[0][0];
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, x[n][e]);
      top = fmaxf(top, other_half(top)) * kScale2;
      if (__any(top > m + kLazy)) {
        const float now = fmaxf(m, top), old = __builtin_amdgcn_exp2f(m - (now == -INFINITY ? 0.f : now));
        m = now;
        sum *= old;
#pragma unroll
        for (int d = 0; d < 2; ++d)
#pragma unroll
          for (int e = 0; e < 16; ++e) o[d][e] *= old;
      }
      const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          x[n][e] = __builtin_amdgcn_exp2f(fmaf(x[n][e], kScale2, -base));
          sum += x[n][e];
        }
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const bf16x8 p = narrow(x[n], 8 * c);
#pragma unroll
          for (int d = 0; d < 2; ++d) o[d] = mfma32(read_cols(vt, l, d, 2 * n + c), p, o[d]);
        }
    }
    if (more) {
      ks.store(lds + (at ^ (2 * kTileBytes)));
      vs.store(lds + (at ^ (2 * kTileBytes)) + kTileBytes);
    }
    __syncthreads();
  }
  sum += other_half(sum);

  if constexpr (QW == 4) {
    // out through LDS, a row's 64 columns side by side; rows 136 bytes apart: columns of 32 rows in
    // different banks
    const float inv = sum == 0.f || !in ? 0.f : 1.f / sum;
    bool bad = false;
#pragma unroll
    for (int d = 0; d < 2; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        o[d][e] = inv == 0.f && sum == 0.f ? 0.f : o[d][e] * inv;
        bad |= !(fabsf(o[d][e]) < INFINITY);
      }
    char* buf = lds + w * 32 * 136;
    const auto put = [&](const HMat& m, bool rest) {
#pragma unroll
      for (int d = 0; d < 2; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float v[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            v[c] = in ? o[d][4 * e + c] : 0.f;
            if (rest) v[c] -= bf16_to_f32(f32_to_bf16(v[c]));
          }
          *(uint2*)(buf + l.n * 136 + 64 * d + 16 * e + 8 * l.h) = make_uint2(f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3]));
        }
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int row = 8 * j + threadIdx.x % kWave / 8, c = threadIdx.x % 8;
        uint2 u[2] = {*(const uint2*)(buf + row * 136 + 16 * c), *(const uint2*)(buf + row * 136 + 16 * c + 8)};
        if (q0 + row < s.oq) __builtin_memcpy(m.p + (s.q0 + (int64_t)(q0 + row)) * m.ld + 64 * h + 8 * c, u, 16);
      }
      __builtin_amdgcn_wave_barrier();
    };
    put(a.o, false);
    if (a.rest.p) put(a.rest, true);
    if (a.lse && l.h == 0 && i < s.oq)
      a.lse[(size_t)h * a.b.q_rows + s.q0 + i] = sum == 0.f || !in ? -INFINITY : (m + __log2f(sum)) * kLn2;
    // what is not finite may come from keys that this row does not see
    uint64_t again = __ballot(bad && in);
    if (again) __threadfence_block();
    again = (again | again >> 32) & 0xffffffffu;
    for (; again; again &= again - 1) fwd_row(a, s, h, q0 + __builtin_ctzll(again));
  } else {
    // the four waves' sums joined: [wave][dimension][query], and every thread 8 dimensions of a query
    float* part = (float*)lds;
    __shared__ float stat[4][2][32];
    __shared__ int bad[32];
#pragma unroll
    for (int d = 0; d < 2; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) part[(w * 64 + 32 * d + 8 * (e / 4) + 4 * l.h + e % 4) * 32 + l.n] = o[d][e];
    if (l.h == 0) {
      stat[w][0][l.n] = m;
      stat[w][1][l.n] = sum;
    }
    if (threadIdx.x < 32) bad[threadIdx.x] = 0;
    __syncthreads();
    const int n = threadIdx.x % 32, d0 = threadIdx.x / 32 * 8, row = q0 + n;
    const float top = fmaxf(fmaxf(stat[0][0][n], stat[1][0][n]), fmaxf(stat[2][0][n], stat[3][0][n]));
    const float base = top == -INFINITY ? 0.f : top;
    float v[8] = {}, total = 0.f;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float f = __builtin_amdgcn_exp2f(stat[u][0][n] - base);
      total = fmaf(stat[u][1][n], f, total);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = fmaf(part[(u * 64 + d0 + e) * 32 + n], f, v[e]);
    }
    const bool live = row < s.oq, some = row < s.nq && total != 0.f;
    if (splits > 1) {
      if (!live) return;
      const size_t at = ((size_t)split * a.b.heads + h) * a.b.q_rows + s.q0 + row;
      const size_t rows = (size_t)splits * a.b.heads * a.b.q_rows;
      *(f32x4*)(a.part + at * 64 + d0) = f32x4{v[0], v[1], v[2], v[3]};
      *(f32x4*)(a.part + at * 64 + d0 + 4) = f32x4{v[4], v[5], v[6], v[7]};
      if (d0 == 0) {
        a.part[rows * 64 + at] = some ? top : -INFINITY;
        a.part[rows * 65 + at] = some ? total : 0.f;
      }
      return;
    }
    const float inv = some ? 1.f / total : 0.f;
    uint32_t hi[4], low[4];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = some ? v[e] * inv : 0.f;
      if (!(fabsf(v[e]) < INFINITY)) bad[n] = 1;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      hi[e] = f32x2_to_bf16x2(v[2 * e], v[2 * e + 1]);
      low[e] = f32x2_to_bf16x2(v[2 * e] - bf16_to_f32(hi[e] & 0xffff), v[2 * e + 1] - bf16_to_f32(hi[e] >> 16));
    }
    __syncthreads();
    const bool again = live && bad[n];
    if (live && !again) {
      const int64_t qr = s.q0 + (int64_t)row;
      __builtin_memcpy(a.o.p + qr * a.o.ld + 64 * h + d0, hi, 16);
      if (a.rest.p) __builtin_memcpy(a.rest.p + qr * a.rest.ld + 64 * h + d0, low, 16);
      if (a.lse && d0 == 0) a.lse[(size_t)h * a.b.q_rows + qr] = some ? (top + __log2f(total)) * kLn2 : -INFINITY;
    }
    // what is not finite may come from keys that the row does not see
    for (uint32_t rows = (uint32_t)__ballot(again); rows; rows &= rows - 1)
      if (__builtin_ctz(rows) % 4 == w) fwd_row(a, s, h, q0 + __builtin_ctz(rows));
  }
}

// The parts of a row's keys joined: a wave a row and head, a lane a dimension.
__global__ void __launch_bounds__(256) attn_join_kernel(AttnFwdArgs a, int tiles, int splits) {
  const int tile = blockIdx.x % tiles, h = blockIdx.x / tiles % a.b.heads, b = blockIdx.x / tiles / a.b.heads;
  const Span s = span_of(a.b, b);
  const int i = tile * 4 + threadIdx.x / kWave, d = threadIdx.x % kWave;
  if (!s.ok || i >= s.oq) return;
  const size_t stride = (size_t)a.b.heads * a.b.q_rows, rows = stride * splits;
  const size_t row = s.q0 + i, at = (size_t)h * a.b.q_rows + row;
  // (lane u holds part u's maximum; there are at most 64)
  const float mu = d < splits ? a.part[rows * 64 + at + d * stride] : -INFINITY;
  const float lu = d < splits ? a.part[rows * 65 + at + d * stride] : 0.f;
  const float top = wave_max(mu), base = top == -INFINITY ? 0.f : top;
  const float f = __builtin_amdgcn_exp2f(mu - base);
  const float total = wave_sum(lu * f);
  float o = 0.f;
  for (int u = 0; u < splits; ++u)
    o = fmaf(a.part[(at + u * stride) * 64 + d], __int_as_float(__builtin_amdgcn_readlane(__float_as_int(f), u)), o);
  o = total == 0.f ? 0.f : o / total;
  if (__any(!(fabsf(o) < INFINITY))) {
    fwd_row(a, s, h, i);
    return;
  }
  const uint16_t hi = f32_to_bf16(o);
  a.o.p[row * a.o.ld + 64 * h + d] = hi;
  if (a.rest.p) a.rest.p[row * a.rest.ld + 64 * h + d] = f32_to_bf16(o - bf16_to_f32(hi));
  if (a.lse && d == 0) a.lse[at] = total == 0.f ? -INFINITY : (top + __log2f(total)) * kLn2;
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

// How a forward pass is cut: four waves of 32 queries where that gives every CU two workgroups, else 32
// queries a workgroup, and where that leaves CUs without work the keys in `splits` parts of `chunk`.
struct FwdPlan {
  bool few;
  int tiles, splits, chunk;
};
FwdPlan fwd_plan(const AttnBatch& b) {
  FwdPlan p = {false, (b.q_max + 127) / 128, 1, 0};
  if (!p.tiles || !b.batch) return p;
  const int64_t pairs = (int64_t)b.heads * b.batch;
  if (pairs * p.tiles >= 512 && b.q_max > 32) return p;
  p.few = true;
  p.tiles = (b.q_max + 31) / 32;
  const int stages = std::max((b.k_max + 127) / 128, 1);
  const int64_t groups = pairs * p.tiles;
  const int want = (int)std::min<int64_t>(std::min(stages, 64), std::max<int64_t>(512 / groups, 1));
  const int each = (stages + want - 1) / want;
  p.splits = (stages + each - 1) / each;
  p.chunk = each * 128;
  return p;
}

size_t attn_fwd_bytes(const AttnBatch& b) {
  const FwdPlan p = fwd_plan(b);
  return p.splits > 1 ? 4ull * 66 * p.splits * b.heads * b.q_rows : 0;
}
size_t attn_bwd_bytes(const AttnBatch& b) { return 4ull * b.heads * b.q_rows; }
int64_t attn_groups(const AttnBatch& b) {
  return std::max((int64_t)((b.q_max + 3) / 4) * b.heads, (int64_t)((b.k_max + 3) / 4) * b.kv_heads) * b.batch;
}

void launch_attention(const AttnFwdArgs& a, hipStream_t st) {
  const FwdPlan p = fwd_plan(a.b);
  const int grid = (int)places(p.tiles, a.b.heads, a.b.batch) * p.splits;
  if (!grid) return;
  if (!p.few) attn_fwd_kernel<4><<<grid, 256, 0, st>>>(a, p.tiles, 1, 0);
  else attn_fwd_kernel<1><<<grid, 256, 0, st>>>(a, p.tiles, p.splits, p.chunk);
  if (p.splits > 1) {
    const int rows = (a.b.q_max + 3) / 4;
    attn_join_kernel<<<rows * a.b.heads * a.b.batch, 256, 0, st>>>(a, rows, p.splits);
  }
}

void launch_attention_backward(const AttnBwdArgs& a, hipStream_t st) {
  const int tiles = (a.b.q_max + 3) / 4, grid = tiles * a.b.heads * a.b.batch;
  if (grid) attn_dq_rows_kernel<<<grid, 256, 0, st>>>(a, tiles);
  const int ktiles = (a.b.k_max + 3) / 4, kgrid = ktiles * a.b.kv_heads * a.b.batch;
  if (kgrid) attn_dkv_rows_kernel<<<kgrid, 256, 0, st>>>(a, ktiles);
}

}  // namespace ad
