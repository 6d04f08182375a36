// Attention over matrices and its gradients (the draft block's training), 64-wide heads.
//
// Forward, a query at a time: s_j = q . k_j / 8 over the keys it sees, m the largest so far and l the sum of
// exp(s_j - m), o = sum_j exp(s_j - m) v_j / l, lse = m + log l: one pass over the keys, 4 x 64 operations a visible pair.
// Backward: p_j = exp(s_j - lse), delta = dout . o, dS_j = p_j (dout . v_j - delta), dq = sum dS_j k_j / 8, and over
// the queries dk_j = sum dS q / 8, dv_j = sum p dout: five products, 10 x 64 operations, of which dq's kernel and that of
// dk and dv each do S and dP (7 products, and one more for dS's second part), because sums over queries and over keys in
// one kernel would need atomics, whose order changes results.
//
// Scores, sums and statistics are float32, results are rounded once.  p, and dS for dk, are rounded to bf16 for the second
// products, whose operands are bf16.  For dq dS goes in as two bf16 parts: the terms of a row cancel (their sum over the
// keys is 0), and rounded once dq was off by 0.0025 to 0.0029 of itself (root mean square) where its own rounding is 0.0017.
// The second part costs dq's kernel a quarter on large shapes (32 x 448 x 1500 197 to 250 us).
// m, lse and scores are kept in powers of two inside the kernels.
//
// For 64 keys x 32 queries a wave issues vector instructions (scale, exponential, maximum, sum, rounding; the issue of the
// products counted) for 860 cycles beside 512 of products forward, 1230 beside 1024 in dq, 1310 beside 1024 in dk and dv.
// Forward that is the bound of a large shape: by the counters of 8 x 2048 rows, 20 heads, vector instructions have 72% of a
// SIMD's cycles and products 43%, with 3.2 waves on it (195 us, 880 TF/s; a large bf16 product reaches 1630).  The gradients
// fill neither: 32 x 448 x 1500 53 and 44% in dq (2.4 waves), 39 and 31% in dk and dv (1.8), LDS 18 and 28%; waves wait for
// 35 and 41% of their cycles, and registers leave no room for more of them.
// Prologue and epilogue make short ones slower: 32 x 448 x 1500 forward 150 us (730 TF/s), 157 with o's rest.
#include <algorithm>
#include <type_traits>

#include "train.h"

namespace ad {

namespace {

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.69314718055994531f;
constexpr float kScale = 0.125f;                       // 1 / sqrt(64)
constexpr float kScale2 = kScale * kLog2e;             // scores in powers of two

__device__ __forceinline__ int key_head(const AttnBatch& a, int h) { return a.group == 1 ? h : h / a.group; }

__device__ __forceinline__ float at(const HMat& m, size_t row, int col) {
  return m.p ? bf16_to_f32(m.p[row * m.ld + col]) : 0.f;
}

// A row at a time, a lane a dimension: what is right whatever the keys hold, since only visible ones are read.  A key
// takes a wave about 0.9 us, so a walk ends where nothing can change any more: a sum that is NaN stays NaN.  32 x 448 x
// 1500, 20 heads, all rows NaN: 0.23 ms forward and 1.6 back, where walks to the end take 104 and 360.  (What is not finite
// in some columns only is walked to the end: an infinity in one column of every value, 35 ms and 39.)
__device__ void fwd_row(const AttnFwdArgs& a, const Span& s, int h, int i) {
  const int d = threadIdx.x % kWave, g = key_head(a.b, h);
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
      if (__all(l != l)) break;        // (so is o, in every lane)
    }
  }
  o = l == 0.f ? 0.f : o / l;
  const uint16_t hi = f32_to_bf16(o);
  a.o.p[row * a.o.ld + 64 * h + d] = hi;
  if (a.rest.p) a.rest.p[row * a.rest.ld + 64 * h + d] = f32_to_bf16(o - bf16_to_f32(hi));
  if (a.lse && d == 0) a.lse[(size_t)h * a.b.q_rows + row] = l == 0.f ? -INFINITY : (m + __log2f(l)) * kLn2;
}

__device__ void dq_row(const AttnBwdArgs& a, const Span& s, int h, int i) {
  const int d = threadIdx.x % kWave, g = key_head(a.b, h);
  const size_t row = s.q0 + i;
  float acc = 0.f;
  if (i < s.nq) {
    const float q = at(a.q, row, 64 * h + d) * kScale2, go = at(a.dout, row, 64 * h + d);
    const float delta = wave_sum(go * (at(a.o, row, 64 * h + d) + at(a.rest, row, 64 * h + d)));
    const float lse = a.lse[(size_t)h * a.b.q_rows + row] * kLog2e;
    Keys r = keys_of(a.b, s, i);
    if (lse == -INFINITY) r.hi = r.lo;
    for (int j = r.lo; j < r.hi; ++j) {
      const float k = at(a.k, s.k0 + j, 64 * g + d);
      const float p = __builtin_amdgcn_exp2f(wave_sum(q * k) - lse);
      const float dp = wave_sum(go * at(a.v, s.k0 + j, 64 * g + d));
      acc = fmaf(p * (dp - delta), k, acc);
      if (__all(acc != acc)) break;
    }
    acc *= kScale;
    if (a.res.p) acc += a.res.bf16 ? bf16_to_f32(((const uint16_t*)a.res.p)[row * a.res.ld + 64 * h + d])
                                   : ((const float*)a.res.p)[row * a.res.ld + 64 * h + d];
  }
  a.dq.p[row * a.dq.ld + 64 * h + d] = f32_to_bf16(acc);
}

__device__ void dkv_row(const AttnBwdArgs& a, const Span& s, int g, int j) {
  const int d = threadIdx.x % kWave, n = a.b.group;
  const size_t row = s.k0 + j;
  float dk = 0.f, dv = 0.f;
  if (j < s.nk) {
    const float k = at(a.k, row, 64 * g + d) * kScale2, v = at(a.v, row, 64 * g + d);
    const int first = a.b.causal ? max(j - (s.nk - s.nq), 0) : 0, tiles = (s.nq - first + kWave - 1) / kWave;
    // lse in powers of two of 64 queries of a head, a lane each, -infinity where they do not see the key
    const auto seen = [&](int t) {
      const int i = first + t % tiles * kWave + d;
      if (i >= s.nq) return -INFINITY;
      const Keys r = keys_of(a.b, s, i);
      return j >= r.lo && j < r.hi ? a.lse[(size_t)(g * n + t / tiles) * a.b.q_rows + s.q0 + i] * kLog2e : -INFINITY;
    };
    // (a query whose scores are NaN: so are its p and dS, and there is nothing to add up)
    bool more = true;
    for (int t = 0; t < n * tiles && more; ++t) {
      const float each = seen(t);
      more = !__any(each != each);
    }
    if (!more) dk = dv = __uint_as_float(0x7fc00000u);
    for (int t = 0; t < n * tiles && more; ++t) {
      const int h = g * n + t / tiles, i0 = first + t % tiles * kWave;
      const float each = seen(t);
      for (uint64_t left = __ballot(each != -INFINITY); left && more; left &= left - 1) {
        const int i = __builtin_ctzll(left);
        const size_t qr = s.q0 + (size_t)(i0 + i);
        const float lse = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(each), i));
        const float q = at(a.q, qr, 64 * h + d), go = at(a.dout, qr, 64 * h + d);
        const float p = __builtin_amdgcn_exp2f(wave_sum(q * k) - lse);
        const float ds = p * wave_sum(go * (v - at(a.o, qr, 64 * h + d) - at(a.rest, qr, 64 * h + d)));   // dP - delta
        dk = fmaf(ds, q, dk);
        dv = fmaf(p, go, dv);
        more = !__all(dk != dk && dv != dv);
      }
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

// Tiles of 64-wide rows in LDS: 128 bytes a row, 16-byte piece c of row r at c ^ turn(r).  LDS has 64
// banks of 4 bytes: 16 rows' same piece (16 lanes of a 16-byte read) lie in different banks, and so do four
// rows' same 64 bytes (32 lanes of a transposing read).  With c ^ (r % 8) a third of LDS' cycles were conflicts.
constexpr int kRowBytes = 128;
__device__ __forceinline__ int turn(int r) { return (r << 1 & 4) | (r >> 1 & 2) | (r >> 3 & 1); }

// A lane's place in a tile, as the A operand whose rows are the tile's rows (`row`: piece 2 s + h of row
// l % 32), and as the one whose rows are the tile's columns (`col`: 16 lanes read 4 rows of 16 columns).
struct Lane {
  uint32_t row, col;
  int h, n;       // l / 32, l % 32
  __device__ __forceinline__ explicit Lane(int l) {
    h = l >> 5;
    n = l & 31;
    row = n * kRowBytes + ((h ^ turn(n)) << 4);
    const int c16 = l & 15, r = 4 * h + (c16 >> 2), piece = 2 * ((l >> 4) & 1) + ((c16 & 3) >> 1);
    col = r * kRowBytes + ((piece ^ turn(r)) << 4) + (c16 & 1) * 8;
  }
};
// rows 32 b .. + 31, columns 16 s .. + 15 as the reduction
__device__ __forceinline__ bf16x8 read_rows(const char* tile, const Lane& l, int b, int s) {
  return as_bf16x8(*(const uint4*)(tile + b * 32 * kRowBytes + (l.row ^ (s * 32))));
}
// columns 32 b .. + 31, rows 16 c .. + 15 as the reduction (in the order above); 8 rows on, turn() differs by 1
__device__ __forceinline__ bf16x8 read_cols(const char* tile, const Lane& l, int b, int c) {
  typedef __attribute__((address_space(3))) s16x4* lp;
  const char* p = tile + c * 16 * kRowBytes;
  const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(p + (l.col ^ (b * 64))));
  const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(p + 8 * kRowBytes + (l.col ^ (b * 64) ^ 16)));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
}
// eight values of a lane's column as an operand
__device__ __forceinline__ bf16x8 narrow(const f32x16& v, int e) {
  return as_bf16x8(make_uint4(f32x2_to_bf16x2(v[e], v[e + 1]), f32x2_to_bf16x2(v[e + 2], v[e + 3]),
                              f32x2_to_bf16x2(v[e + 4], v[e + 5]), f32x2_to_bf16x2(v[e + 6], v[e + 7])));
}
// The same in two parts, the second what rounding took from the first.
__device__ __forceinline__ bf16x8 narrow(const f32x16& v, int e, bf16x8& rest) {
  uint32_t hi[4], low[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float x = v[e + 2 * i], y = v[e + 2 * i + 1];
    hi[i] = f32x2_to_bf16x2(x, y);
    low[i] = f32x2_to_bf16x2(x - __uint_as_float(hi[i] << 16), y - __uint_as_float(hi[i] & 0xffff0000u));
  }
  rest = as_bf16x8(make_uint4(low[0], low[1], low[2], low[3]));
  return as_bf16x8(make_uint4(hi[0], hi[1], hi[2], hi[3]));
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
__device__ __forceinline__ uint4 load16(const void* p) {
  uint4 u;
  __builtin_memcpy(&u, p, 16);
  return u;
}
// Waits here for what was loaded into these registers, and not where a loop first uses them: there the wait
// would be for every load in flight, each time round.
__device__ __forceinline__ void settled(bf16x8 (&v)[4]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) asm volatile("" : "+v"(v[k]));
}

// 32 rows of a matrix that a wave has as an operand (columns l % 32): loaded in whole rows, eight lanes a row,
// and turned in 4 KB of LDS of the wave's own.  Loaded as the operand has them, 32 bytes of 32 rows at a time,
// each line came from L2 four times over.
struct Rows {
  uint4 reg[4];     // row 8 j + lane / 8, columns 8 (lane % 8) .. + 7
  static __device__ __forceinline__ int row(int j) { return 8 * j + threadIdx.x % kWave / 8; }
  __device__ __forceinline__ void load(const HMat& m, int64_t first, int rows, int col) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      reg[j] = make_uint4(0, 0, 0, 0);
      if (row(j) < rows) reg[j] = load16(m.p + (first + row(j)) * m.ld + col + 8 * (threadIdx.x % 8));
    }
  }
  // as a tile of the wave's own
  __device__ __forceinline__ void place(char* buf) const {
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int j = 0; j < 4; ++j) *(uint4*)(buf + row(j) * kRowBytes + (((threadIdx.x % 8) ^ turn(row(j))) << 4)) = reg[j];
    __builtin_amdgcn_wave_barrier();
  }
  __device__ __forceinline__ void operand(char* buf, const Lane& l, bf16x8 (&v)[4]) const {
    place(buf);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = read_rows(buf, l, 0, k);
    __builtin_amdgcn_wave_barrier();
  }
};

// A tile of TR rows on its way from memory to LDS: thread t of 256 takes 16-byte piece t % 8 of rows
// t / 8 + 32 j.  Rows past the sequence's last one become zeros.  A scalar base and a 32-bit offset a lane.
template <int TR>
struct Stage {
  static constexpr int N = TR / 32;
  uint4 reg[N];
  const char* base;   // the sequence's first row
  int64_t pitch;      // bytes between rows
  int n, from;        // the sequence's rows, and the tile's first one
  __device__ __forceinline__ void init(const HMat& m, int first, int rows, int col) {
    base = (const char*)(m.p + first * m.ld + col);
    pitch = 2 * m.ld;
    n = rows;
  }
  __device__ __forceinline__ void load(int r0) {
    const char* p = base + r0 * pitch;
    const uint32_t t = threadIdx.x, c = (t % 8) * 16;
    from = r0;
    if (r0 + TR <= n) {
#pragma unroll
      for (int j = 0; j < N; ++j) reg[j] = load16(p + (uint32_t)((t / 8 + 32 * j) * (uint32_t)pitch + c));
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j)
        reg[j] = load16(p + (uint32_t)(min((int)t / 8 + 32 * j, n - 1 - r0) * (uint32_t)pitch + c));
    }
  }
  __device__ __forceinline__ void store(char* tile) {
    const int t = threadIdx.x, r = t / 8;
    if (from + TR > n)
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (from + r + 32 * j >= n) reg[j] = make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int j = 0; j < N; ++j) *(uint4*)(tile + (r + 32 * j) * kRowBytes + (((t % 8) ^ turn(r)) << 4)) = reg[j];
  }
};

// A tile of 64 rows to LDS by four waves, the loads in flight while the tile before is worked on.  DIRECT:
// straight into LDS through a buffer descriptor, whose end makes zeros of the rows past the sequence's
// last one (rows 16-byte aligned); a lane's 16 bytes land at its place in the wave's kilobyte, so it
// loads the piece that belongs there.  Else through registers.
constexpr uint32_t kBufferFlags = 0x00020000;   // raw buffer of 32-bit elements
constexpr uint32_t kPastEnd = 0x80000000u;      // further than any offset in a tile: 64 * 2^23 bytes

template <bool DIRECT>
struct Loads {
  const char* base;   // the sequence's first row
  int64_t pitch;      // bytes between rows
  int n, from;        // the sequence's rows, and the first one of the tile in registers
  uint32_t off[2];
  uint4 reg[DIRECT ? 1 : 2];
  // thread t takes piece t % 8 of rows t / 8 + 8 (t / 64) + 8 j: those of its wave side by side
  static __device__ __forceinline__ int row(int j) { return (threadIdx.x >> 6) * 16 + j * 8 + (threadIdx.x & 63) / 8; }
  __device__ __forceinline__ void init(const HMat& m, int first, int rows, int col) {
    base = (const char*)(m.p + first * m.ld + col);
    pitch = 2 * m.ld;
    n = rows;
#pragma unroll
    for (int j = 0; j < 2; ++j) off[j] = row(j) * (uint32_t)pitch + (((threadIdx.x % 8) ^ turn(row(j))) << 4);
  }
  // (more: bytes further along the row)
  __device__ __forceinline__ void issue(int r0, uint4* tile, int more = 0) {
    const char* p = base + r0 * pitch + more;
    if constexpr (DIRECT) {
      const int64_t left = r0 < n ? (n - 1 - r0) * pitch + kRowBytes : 0;
      const auto d = __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, (uint32_t)min(left, (int64_t)kPastEnd), kBufferFlags);
      const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
#pragma unroll
      for (int j = 0; j < 2; ++j)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(d, (__attribute__((address_space(3))) void*)(tile + (2 * w + j) * 64), 16, off[j], 0, 0, 0);
    } else {
      from = r0;
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if (r0 < n) reg[j] = load16(p + off[j] - (uint32_t)max(r0 + row(j) - (n - 1), 0) * (uint32_t)pitch);
    }
  }
  // before the barrier after which the tile is read
  __device__ __forceinline__ void arrive(uint4* tile) {
    if constexpr (!DIRECT) {
      const int w = threadIdx.x / kWave;
#pragma unroll
      for (int j = 0; j < 2; ++j)
        tile[(2 * w + j) * 64 + threadIdx.x % kWave] = from + row(j) < n ? reg[j] : make_uint4(0, 0, 0, 0);
    }
  }
};
// Every load of the wave has landed, every LDS access is done; then all waves meet.
__device__ __forceinline__ void landed() {
  __builtin_amdgcn_s_waitcnt(0x0070);
  __builtin_amdgcn_s_barrier();
}
// A wave's transposed 64 x 32 result (columns l.n) as rows: out(row, c, v) with columns 8 c .. + 7 of row, eight lanes a
// row, so that memory is accessed in whole rows.  buf: 8 KB of the wave's own; a row's 16-byte pieces p are at p ^ (row % 16).
template <class F>
__device__ __forceinline__ void by_rows(char* buf, const Lane& l, const f32x16 (&v)[2], F&& out) {
#pragma unroll
  for (int d = 0; d < 2; ++d)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      *(f32x4*)(buf + l.n * 256 + (((8 * d + 2 * e + l.h) ^ (l.n & 15)) << 4)) =
          f32x4{v[d][4 * e], v[d][4 * e + 1], v[d][4 * e + 2], v[d][4 * e + 3]};
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int row = 8 * j + threadIdx.x % kWave / 8, c = threadIdx.x % 8;
    const f32x4 x = *(const f32x4*)(buf + row * 256 + (((2 * c) ^ (row & 15)) << 4));
    const f32x4 y = *(const f32x4*)(buf + row * 256 + (((2 * c + 1) ^ (row & 15)) << 4));
    const float r[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
    out(row, c, r);
  }
}
// The columns (rows of the result) of which some lane says so, as bits.
__device__ __forceinline__ uint32_t columns(bool bad) {
  const uint64_t m = __ballot(bad);
  return (uint32_t)(m | m >> 32);
}
__device__ __forceinline__ uint4 narrow8(const float (&v)[8]) {
  return make_uint4(f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3]), f32x2_to_bf16x2(v[4], v[5]),
                    f32x2_to_bf16x2(v[6], v[7]));
}
// columns 8 c .. + 7 of head h of a row
__device__ __forceinline__ void store_piece(const HMat& m, int64_t row, int h, int c, uint4 u) {
  __builtin_memcpy(m.p + row * m.ld + 64 * h + 8 * c, &u, 16);
}

// The tiles of one (sequence, head) run on one of the eight XCDs, whose L2 then has its keys: workgroups are dealt
// to them in turn, and a row of the grid holds 8 pairs times their tiles.
struct Place {
  int b, h, tile;
  bool in;
};
// (a quotient by a product: the prologue is as long as its instructions)
__device__ __forceinline__ Place place_of(int heads, uint64_t per_head, int batch) {
  const int pair = blockIdx.y * 8 + blockIdx.x % 8;
  Place r;
  r.b = (int)(((uint64_t)pair * per_head) >> kPerShift);
  r.h = pair - r.b * heads;
  r.tile = blockIdx.x / 8;
  r.in = r.b < batch;
  return r;
}

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
__device__ __forceinline__ Range range_of(const Keys& k, bool in) {
  const bool some = in && k.lo < k.hi;
  Range r;
  r.lo = wave_min(some ? k.lo : 0x7fffffff);
  r.hi = wave_most(some ? k.hi : 0);
  r.all_lo = wave_most(in ? k.lo : 0);
  r.all_hi = wave_min(in ? k.hi : 0x7fffffff);
  return r;
}

// The same of the queries q0 .. + 31, of which this lane has q0 + l.n with `keys`: without windows from the rules alone.
__device__ __forceinline__ Range range_at(const AttnBatch& a, const Span& s, int q0, const Keys& keys, bool in) {
  if (a.window) return range_of(keys, in);
  const int rows = min(32, s.nq - q0);
  if (rows <= 0) return Range{0x7fffffff, 0, 0, 0x7fffffff};
  if (!a.causal) return Range{0, s.nk, 0, s.nk};
  const int first = q0 + s.nk - s.nq + 1;
  return Range{0, min(s.nk, max(first + rows - 1, 0)), 0, min(s.nk, max(first, 0))};
}

// Without windows: the keys that the `rows` queries from q0 on see end here.
__device__ __forceinline__ int ends_at(const AttnBatch& a, const Span& s, int q0, int rows) {
  rows = min(rows, s.nq - q0);
  return rows <= 0 ? 0 : a.causal ? min(s.nk, max(q0 + rows + s.nk - s.nq, 0)) : s.nk;
}

// ----------------------------------------------------------------- forward

// The maximum that is taken off is only moved when a score exceeds it by 8 (in powers of two): p stays under 256 and
// what is added up before keeps its scale, which saves 32 products a lane on most tiles.
constexpr float kLazy = 8.f;

// 32 queries, the four waves a quarter of each tile of 128 keys and their sums joined at the end: where there are few
// workgroups of 128 queries.  A tile takes 0.87 us, its loads a round trip to L2 or HBM ahead through registers.
// With splits a workgroup has `chunk` of the keys and leaves its sums to attn_join_kernel (20 heads of one query over
// 4000 keys: 8 + 5 us; a launch is 5 us by itself).

__global__ void __launch_bounds__(256, 2) attn_fwd_few_kernel(AttnFwdArgs a, int tiles, int splits, int chunk) {
  constexpr int TK = 128, kTileBytes = TK * kRowBytes;
  __shared__ __attribute__((aligned(16))) char lds[4 * kTileBytes];   // two stages of keys and values
  const Place at = place_of(a.b.heads, a.b.per_head, a.b.batch);
  if (!at.in) return;
  const int split = splits > 1 ? at.tile % splits : 0, nth = splits > 1 ? at.tile / splits : at.tile;
  const int b = at.b, h = at.h, tile = a.b.causal ? tiles - 1 - nth : nth;
  const Span s = span_of(a.b, b);
  if (!s.ok) {
    if (threadIdx.x == 0) atomicOr(a.b.err, AD_ERR_LENGTH);
    return;
  }
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), g = key_head(a.b, h);
  const Lane l(threadIdx.x % kWave);
  const int q0 = tile * 32, i = q0 + l.n;
  if (q0 >= s.oq) return;
  Stage<TK> ks, vs;
  ks.init(a.k, s.k0, s.nk, 64 * g);
  vs.init(a.v, s.k0, s.nk, 64 * g);
  // (without windows the first tile is under way before anything else is asked for)
  const bool early = !a.b.window && split * chunk < ends_at(a.b, s, q0, 32);
  if (early) {
    ks.load(split * chunk);
    vs.load(split * chunk);
  }
  const bool in = i < s.nq;
  Keys keys = {0, s.nk};
  if (in) keys = keys_of(a.b, s, i);
  if (splits > 1) {
    keys.lo = max(keys.lo, split * chunk);
    keys.hi = min(keys.hi, (split + 1) * chunk);
  }
  Range r = range_at(a.b, s, q0, keys, in);
  if (splits > 1 && !a.b.window) {
    r.lo = max(r.lo, split * chunk);
    r.hi = min(r.hi, (split + 1) * chunk);
    r.all_lo = max(r.all_lo, split * chunk);
    r.all_hi = min(r.all_hi, (split + 1) * chunk);
  }

  bf16x8 q[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    uint4 u = make_uint4(0, 0, 0, 0);
    if (in) u = load16(a.q.p + (s.q0 + (int64_t)i) * a.q.ld + 64 * h + 16 * k + 8 * l.h);
    q[k] = as_bf16x8(u);
  }
  settled(q);

  const int first = r.lo / TK * TK, last = r.hi;
  float m = -INFINITY, sum = 0.f;
  f32x16 o[2] = {zeros(), zeros()};
  if (first < last) {
    if (!early) {
      ks.load(first);
      vs.load(first);
    }
    ks.store(lds);
    vs.store(lds + kTileBytes);
  }
  __syncthreads();
  for (int k0 = first, buf = 0; k0 < last; k0 += TK, buf ^= 2 * kTileBytes) {
    const bool more = k0 + TK < last;
    if (more) {
      ks.load(k0 + TK);
      vs.load(k0 + TK);
    }
    const int mine = k0 + 32 * w;            // this wave's first key
    if (mine < r.hi && mine + 32 > r.lo) {
      const char* kt = lds + buf + w * 32 * kRowBytes;
      const char* vt = kt + kTileBytes;
      f32x16 x = zeros();
#pragma unroll
      for (int k = 0; k < 4; ++k) x = mfma32(read_rows(kt, l, 0, k), q[k], x);
      if (mine < r.all_lo || mine + 32 > r.all_hi) {
        const Mask mask = mask_of(keys, mine + 4 * l.h);
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = shows(mask, 8 * (e / 4) + e % 4) ? x[e] : -INFINITY;
      }
      float top = x[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) top = fmaxf(top, x[e]);
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
      for (int e = 0; e < 16; ++e) {
        x[e] = __builtin_amdgcn_exp2f(fmaf(x[e], kScale2, -base));
        sum += x[e];
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const bf16x8 p = narrow(x, 8 * c);
#pragma unroll
        for (int d = 0; d < 2; ++d) o[d] = mfma32(read_cols(vt, l, d, c), p, o[d]);
      }
    }
    if (more) {
      ks.store(lds + (buf ^ (2 * kTileBytes)));
      vs.store(lds + (buf ^ (2 * kTileBytes)) + kTileBytes);
    }
    __syncthreads();
  }
  sum += other_half(sum);

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
    const size_t each = part_rows(a.b), rows = splits * each;
    const size_t to = split * each + part_row(a.b, b, h, row);
    *(f32x4*)(a.part + to * 64 + d0) = f32x4{v[0], v[1], v[2], v[3]};
    *(f32x4*)(a.part + to * 64 + d0 + 4) = f32x4{v[4], v[5], v[6], v[7]};
    if (d0 == 0) {
      a.part[rows * 64 + to] = some ? top : -INFINITY;
      a.part[rows * 65 + to] = some ? total : 0.f;
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

// 32 queries, eight waves that take 32 keys each in turn, loaded a step ahead into places of their own: nobody waits for
// anybody before the end, and a CU has its keys at about 40 bytes a cycle (twelve waves: no more).
constexpr int kKeyWaves = 8;
__global__ void __launch_bounds__(64 * kKeyWaves) attn_fwd_keys_kernel(AttnFwdArgs a) {
  constexpr int W = kKeyWaves, kPlace = 64 * kRowBytes;
  __shared__ __attribute__((aligned(16))) char lds[W * kPlace];   // a wave's keys and values, then its sums
  __shared__ float stat[W][2][32];
  __shared__ int bad[32];
  const Place at = place_of(a.b.heads, a.b.per_head, a.b.batch);
  if (!at.in) return;
  const int h = at.h;
  const Span s = span_of(a.b, at.b);
  if (!s.ok) {
    if (threadIdx.x == 0) atomicOr(a.b.err, AD_ERR_LENGTH);
    return;
  }
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), g = key_head(a.b, h);
  const Lane l(threadIdx.x % kWave);
  const int q0 = at.tile * 32, i = q0 + l.n;
  if (q0 >= s.oq) return;
  const bool in = i < s.nq;
  Rows ks, vs, qs;
  const auto load = [&](int k0) {
    ks.load(a.k, s.k0 + (int64_t)k0, s.nk - k0, 64 * g);
    vs.load(a.v, s.k0 + (int64_t)k0, s.nk - k0, 64 * g);
  };
  // (without windows the first keys are under way before anything else is asked for)
  if (!a.b.window && 32 * w < s.nk) load(32 * w);
  qs.load(a.q, s.q0 + (int64_t)q0, s.nq - q0, 64 * h);
  Keys keys = {0, s.nk};
  if (in) keys = keys_of(a.b, s, i);
  const Range r = range_at(a.b, s, q0, keys, in);
  const int mine = a.b.window ? first_piece(r.lo, r.hi, w) : 32 * w;
  char* const kt = lds + w * kPlace;
  char* const vt = kt + 32 * kRowBytes;
  bf16x8 q[4];
  if (a.b.window && mine < r.hi) load(mine);
  qs.operand(kt, l, q);
  settled(q);
  float m = -INFINITY, sum = 0.f;
  f32x16 o[2] = {zeros(), zeros()};
  for (int k0 = mine; k0 < r.hi; k0 += 32 * W) {
    ks.place(kt);
    vs.place(vt);
    if (k0 + 32 * W < r.hi) load(k0 + 32 * W);
    f32x16 x = zeros();
#pragma unroll
    for (int k = 0; k < 4; ++k) x = mfma32(read_rows(kt, l, 0, k), q[k], x);
    if (k0 < r.all_lo || k0 + 32 > r.all_hi) {
      const Mask mask = mask_of(keys, k0 + 4 * l.h);
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] = shows(mask, 8 * (e / 4) + e % 4) ? x[e] : -INFINITY;
    }
    float top = x[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) top = fmaxf(top, x[e]);
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
    for (int e = 0; e < 16; ++e) {
      x[e] = __builtin_amdgcn_exp2f(fmaf(x[e], kScale2, -base));
      sum += x[e];
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const bf16x8 p = narrow(x, 8 * c);
#pragma unroll
      for (int d = 0; d < 2; ++d) o[d] = mfma32(read_cols(vt, l, d, c), p, o[d]);
    }
    __builtin_amdgcn_wave_barrier();
  }
  sum += other_half(sum);

  // the waves' sums joined: [wave][dimension][query], and every thread 4 dimensions of a query
  float* part = (float*)lds;
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
  const int n = threadIdx.x % 32, d0 = threadIdx.x / 32 * 4, row = q0 + n;
  float top = stat[0][0][n];
#pragma unroll
  for (int u = 1; u < W; ++u) top = fmaxf(top, stat[u][0][n]);
  const float base = top == -INFINITY ? 0.f : top;
  float v[4] = {}, total = 0.f;
#pragma unroll 4
  for (int u = 0; u < W; ++u) {
    const float f = __builtin_amdgcn_exp2f(stat[u][0][n] - base);
    total = fmaf(stat[u][1][n], f, total);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = fmaf(part[(u * 64 + d0 + e) * 32 + n], f, v[e]);
  }
  const bool live = row < s.oq, some = row < s.nq && total != 0.f;
  const float inv = some ? 1.f / total : 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[e] = some ? v[e] * inv : 0.f;
    if (!(fabsf(v[e]) < INFINITY)) bad[n] = 1;
  }
  uint32_t hi[2], low[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    hi[e] = f32x2_to_bf16x2(v[2 * e], v[2 * e + 1]);
    low[e] = f32x2_to_bf16x2(v[2 * e] - bf16_to_f32(hi[e] & 0xffff), v[2 * e + 1] - bf16_to_f32(hi[e] >> 16));
  }
  __syncthreads();
  const bool again = live && bad[n];
  if (live && !again) {
    const int64_t qr = s.q0 + (int64_t)row;
    __builtin_memcpy(a.o.p + qr * a.o.ld + 64 * h + d0, hi, 8);
    if (a.rest.p) __builtin_memcpy(a.rest.p + qr * a.rest.ld + 64 * h + d0, low, 8);
    if (a.lse && d0 == 0) a.lse[(size_t)h * a.b.q_rows + qr] = some ? (top + __log2f(total)) * kLn2 : -INFINITY;
  }
  // what is not finite may come from keys that the row does not see
  for (uint32_t rows = (uint32_t)__ballot(again); rows; rows &= rows - 1)
    if (__builtin_ctz(rows) % W == w) fwd_row(a, s, h, q0 + __builtin_ctz(rows));
}

// Four waves of 32 queries share tiles of 64 keys: the next tile is on its way straight to LDS while one is worked on, and
// 33 KB of LDS and 120 registers leave room for four workgroups on a CU, whose vector instructions and products overlap.
// 32 x 448 causal, 20 heads: 47 us; tiles through registers, conflicts in a third of LDS' cycles: 83.  Products of one tile beside
// the exponentials of the one before in the same wave: 175 us where this takes 109 (registers).
template <bool DIRECT>
__global__ void __launch_bounds__(256, DIRECT ? 4 : 2) attn_fwd_wide_kernel(AttnFwdArgs a, int tiles) {
  constexpr int TK = 64;
  // (distinct objects, so that the compiler can tell a read of one tile from the loads that fill another)
  __shared__ uint4 key0[512], key1[512], val0[512], val1[512];
  __shared__ int ends[8];
  Place at = place_of(a.b.heads, a.b.per_head, a.b.batch);
  if (!at.in) return;
  if (a.b.causal) at.tile = tiles - 1 - at.tile;        // (the longest first)
  const int h = at.h;
  const Span s = span_of(a.b, at.b);
  if (!s.ok) {
    if (threadIdx.x == 0) atomicOr(a.b.err, AD_ERR_LENGTH);
    return;
  }
  if (at.tile * 128 >= s.oq) return;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), g = key_head(a.b, h);
  const Lane l(threadIdx.x % kWave);
  const int q0 = at.tile * 128 + 32 * w, i = q0 + l.n;
  const bool in = i < s.nq;
  Loads<DIRECT> ks, vs;
  ks.init(a.k, s.k0, s.nk, 64 * g);
  vs.init(a.v, s.k0, s.nk, 64 * g);
  // (without windows the first tile is under way before anything else is asked for)
  int first = 0, last = ends_at(a.b, s, at.tile * 128, 128);
  if (!a.b.window && last > 0) {
    ks.issue(0, key0);
    vs.issue(0, val0);
  }
  Rows rows;
  rows.load(a.q, s.q0 + (int64_t)q0, s.nq - q0, 64 * h);
  Keys keys = {0, s.nk};
  if (in) keys = keys_of(a.b, s, i);
  const Range r = range_at(a.b, s, q0, keys, in);
  if (a.b.window) {
    if (threadIdx.x % kWave == 0) {
      ends[w] = r.lo;
      ends[4 + w] = r.hi;
    }
    __syncthreads();
    first = __builtin_amdgcn_readfirstlane(min(min(ends[0], ends[1]), min(ends[2], ends[3])) / TK * TK);
    last = __builtin_amdgcn_readfirstlane(max(max(ends[4], ends[5]), max(ends[6], ends[7])));
    if (first < last) {
      ks.issue(first, key0);
      vs.issue(first, val0);
    }
  }

  bf16x8 q[4];
  rows.operand((char*)((w < 2 ? key1 : val1) + w % 2 * 256), l, q);
  float m = -INFINITY, sum = 0.f;
  f32x16 o[2] = {zeros(), zeros()};
  const auto step = [&](int k0, const uint4* kt, const uint4* vt, uint4* next_kt, uint4* next_vt) {
    const bool more = k0 + TK < last;
    if (more) {
      ks.issue(k0 + TK, next_kt);
      vs.issue(k0 + TK, next_vt);
    }
    if (k0 < r.hi && k0 + TK > r.lo) {
      f32x16 x[2];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        x[n] = zeros();
#pragma unroll
        for (int k = 0; k < 4; ++k) x[n] = mfma32(read_rows((const char*)kt, l, n, k), q[k], x[n]);
      }
      if (k0 < r.all_lo || k0 + TK > r.all_hi) {
        const Mask mask = mask_of(keys, k0 + 4 * l.h);
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int e = 0; e < 16; ++e) x[n][e] = shows(mask, 32 * n + 8 * (e / 4) + e % 4) ? x[n][e] : -INFINITY;
      }
      float top = x[0][0];
#pragma unroll
      for (int n = 0; n < 2; ++n)
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
      for (int c = 0; c < 4; ++c) {
        f32x16& p = x[c / 2];
#pragma unroll
        for (int e = 8 * (c % 2); e < 8 * (c % 2) + 8; ++e) {
          p[e] = __builtin_amdgcn_exp2f(fmaf(p[e], kScale2, -base));
          sum += p[e];
        }
        const bf16x8 b = narrow(p, 8 * (c % 2));
#pragma unroll
        for (int d = 0; d < 2; ++d) o[d] = mfma32(read_cols((const char*)vt, l, d, c), b, o[d]);
      }
    }
    if (more) {
      ks.arrive(next_kt);
      vs.arrive(next_vt);
    }
    landed();
  };

  if (first < last) {
    ks.arrive(key0);
    vs.arrive(val0);
    settled(q);
    landed();
    for (int k0 = first; k0 < last; k0 += 2 * TK) {
      step(k0, key0, val0, key1, val1);
      if (k0 + TK >= last) break;
      step(k0 + TK, key1, val1, key0, val0);
    }
  }
  sum += other_half(sum);

  const float inv = sum == 0.f || !in ? 0.f : 1.f / sum;
  bool bad = false;
#pragma unroll
  for (int d = 0; d < 2; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      o[d][e] = inv == 0.f && sum == 0.f ? 0.f : o[d][e] * inv;
      bad |= !(fabsf(o[d][e]) < INFINITY);
      o[d][e] = in ? o[d][e] : 0.f;
    }
  if (first >= last) __syncthreads();      // (another wave's rows may still be in the place that is written next)
  // what is not finite may come from keys that the row does not see: such rows are computed again below
  uint32_t again = columns(bad && in);
  by_rows((char*)(w == 0 ? key0 : w == 1 ? key1 : w == 2 ? val0 : val1), l, o, [&](int row, int c, const float(&v)[8]) {
    if (q0 + row >= s.oq || again >> row & 1) return;
    const uint4 u = narrow8(v);
    store_piece(a.o, s.q0 + (int64_t)(q0 + row), h, c, u);
    if (!a.rest.p) return;
    const uint32_t hi[4] = {u.x, u.y, u.z, u.w};
    float low[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) low[e] = v[e] - bf16_to_f32((uint16_t)(hi[e / 2] >> (16 * (e % 2))));
    store_piece(a.rest, s.q0 + (int64_t)(q0 + row), h, c, narrow8(low));
  });
  if (a.lse && l.h == 0 && i < s.oq && !(again >> l.n & 1))
    a.lse[(size_t)h * a.b.q_rows + s.q0 + i] = sum == 0.f || !in ? -INFINITY : (m + __log2f(sum)) * kLn2;
  for (; again; again &= again - 1) fwd_row(a, s, h, q0 + __builtin_ctz(again));
}

// The parts of a row's keys joined: a wave a row and head, a lane a dimension.  4.8 us for 20 rows of 12 parts, most of it
// the launch and three round trips to memory.
__global__ void __launch_bounds__(256) attn_join_kernel(AttnFwdArgs a, int splits) {
  const int tile = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  const Span s = span_of(a.b, b);
  const int i = tile * 4 + threadIdx.x / kWave, d = threadIdx.x % kWave;
  if (!s.ok || i >= s.oq) return;
  const size_t stride = part_rows(a.b), rows = stride * splits;
  const size_t row = s.q0 + i, at = part_row(a.b, b, h, i);
  // (lane u holds part u's maximum; there are at most 64)
  const float mu = d < splits ? a.part[rows * 64 + at + d * stride] : -INFINITY;
  const float lu = d < splits ? a.part[rows * 65 + at + d * stride] : 0.f;
  const float top = wave_max(mu), base = top == -INFINITY ? 0.f : top;
  const float f = __builtin_amdgcn_exp2f(mu - base);
  const float total = wave_sum(lu * f);
  // (eight loads at once)
  float o = 0.f;
  for (int u0 = 0; u0 < splits; u0 += 8) {
    float v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = a.part[(at + min(u0 + u, splits - 1) * stride) * 64 + d];
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (u0 + u < splits) o = fmaf(v[u], __int_as_float(__builtin_amdgcn_readlane(__float_as_int(f), u0 + u)), o);
  }
  o = total == 0.f ? 0.f : o / total;
  if (__any(!(fabsf(o) < INFINITY))) {
    fwd_row(a, s, h, i);
    return;
  }
  const uint16_t hi = f32_to_bf16(o);
  a.o.p[row * a.o.ld + 64 * h + d] = hi;
  if (a.rest.p) a.rest.p[row * a.rest.ld + 64 * h + d] = f32_to_bf16(o - bf16_to_f32(hi));
  if (a.lse && d == 0) a.lse[(size_t)h * a.b.q_rows + row] = total == 0.f ? -INFINITY : (top + __log2f(total)) * kLn2;
}

// ----------------------------------------------------------------- backward

// What a query's column of the products needs: its row of q and dout, delta = dout . o, lse in powers of two, and
// the keys it sees.
__device__ __forceinline__ void dq_operands(const AttnBwdArgs& a, const Span& s, int h, int i, const Lane& l, bf16x8 (&q)[4],
                                            bf16x8 (&go)[4], float& delta, float& lse, Keys& keys) {
  const bool in = i < s.nq;
  const int64_t row = s.q0 + (int64_t)i;
  delta = lse = 0.f;
  keys = {0, s.nk};
  if (in) {
    keys = keys_of(a.b, s, i);
    lse = a.lse[(size_t)h * a.b.q_rows + row] * kLog2e;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    uint4 uq = make_uint4(0, 0, 0, 0), ud = uq, uo = uq, ur = uq;
    if (in) {
      const int c = 64 * h + 16 * k + 8 * l.h;
      uq = load16(a.q.p + row * a.q.ld + c);
      ud = load16(a.dout.p + row * a.dout.ld + c);
      uo = load16(a.o.p + row * a.o.ld + c);
      if (a.rest.p) ur = load16(a.rest.p + row * a.rest.ld + c);
    }
    q[k] = as_bf16x8(uq);
    go[k] = as_bf16x8(ud);
    float d[8], o[8], r[8];
    widen8(__builtin_bit_cast(u32x4, ud), d);
    widen8(__builtin_bit_cast(u32x4, uo), o);
    widen8(__builtin_bit_cast(u32x4, ur), r);
#pragma unroll
    for (int e = 0; e < 8; ++e) delta = fmaf(d[e], o[e] + r[e], delta);
  }
  delta += other_half(delta);
  if (lse == -INFINITY) lse = INFINITY;     // sees nothing: p = exp2(s - inf) = 0
  settled(q);
  settled(go);
}
// Of 32 keys, the first of this lane's being k: those that the query does not see give p = 0 and dP = 0.
__device__ __forceinline__ void hide(const Keys& keys, int k, f32x16& x, f32x16& y) {
  const Mask mask = mask_of(keys, k);
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const bool seen = shows(mask, 8 * (e / 4) + e % 4);
    x[e] = seen ? x[e] : -INFINITY;
    y[e] = seen ? y[e] : 0.f;
  }
}
// The 32 rows from q0 on.
__device__ __forceinline__ void dq_out(const AttnBwdArgs& a, const Span& s, int h, int q0, bool in, const Lane& l, char* buf,
                                       f32x16 (&dq)[2]) {
  bool bad = false;
#pragma unroll
  for (int d = 0; d < 2; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      dq[d][e] = in ? dq[d][e] * kScale : 0.f;
      bad |= !(fabsf(dq[d][e]) < INFINITY);
    }
  // what is not finite may come from keys that the row does not see: such rows are computed again below (and are not
  // written before: dq may be res)
  uint32_t again = columns(bad);
  by_rows(buf, l, dq, [&](int n, int c, const float(&v)[8]) {
    if (q0 + n >= s.oq || again >> n & 1) return;
    const int64_t to = s.q0 + (int64_t)(q0 + n);
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = v[e];
    if (a.res.p && q0 + n < s.nq) {
      float more[8];
      load8(a.res, to, 64 * h + 8 * c, 64 * a.b.heads, more);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] += more[e];
    }
    store_piece(a.dq, to, h, c, narrow8(x));
  });
  for (; again; again &= again - 1) dq_row(a, s, h, q0 + __builtin_ctz(again));
}

// dq of 32 queries, the four waves a quarter of each tile of 128 keys (where there are few workgroups of 128).  It leaves
// delta and what 32 queries see together for the kernel of dk and dv.  With windows of 41 of 1500 keys a workgroup walks
// over the two or three tiles that its queries see: 12 x 131 rows, 20 heads: 33 us, its loads' latencies.
__global__ void __launch_bounds__(256, 2) attn_dq_few_kernel(AttnBwdArgs a, int tiles) {
  constexpr int TK = 128, kTileBytes = TK * kRowBytes;
  __shared__ __attribute__((aligned(16))) char lds[4 * kTileBytes];
  Place at = place_of(a.b.heads, a.b.per_head, a.b.batch);
  if (!at.in) return;
  if (a.b.causal) at.tile = tiles - 1 - at.tile;        // (the longest first)
  const int h = at.h;
  const Span s = span_of(a.b, at.b);
  if (!s.ok) {
    if (threadIdx.x == 0) atomicOr(a.b.err, AD_ERR_LENGTH);
    return;
  }
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), g = key_head(a.b, h);
  const Lane l(threadIdx.x % kWave);
  const int q0 = at.tile * 32, i = q0 + l.n;
  if (q0 >= s.oq) return;
  Stage<TK> ks, vs;
  ks.init(a.k, s.k0, s.nk, 64 * g);
  vs.init(a.v, s.k0, s.nk, 64 * g);
  // (without windows the first tile is under way before anything else is asked for)
  const bool early = !a.b.window && ends_at(a.b, s, q0, 32) > 0;
  if (early) {
    ks.load(0);
    vs.load(0);
  }
  const bool in = i < s.nq;
  bf16x8 q[4], go[4];
  float delta, lse;
  Keys keys;
  dq_operands(a, s, h, i, l, q, go, delta, lse, keys);
  const Range r = range_at(a.b, s, q0, keys, in);
  if (w == 0) {
    if (in && l.h == 0) a.delta[(size_t)h * a.b.q_rows + s.q0 + i] = delta;
    if (a.b.window && h == 0 && threadIdx.x == 0 && q0 < s.nq)
      a.ranges[(size_t)at.b * a.blocks + at.tile] = make_int4(r.lo, r.hi, r.all_lo, r.all_hi);
  }
  const int first = r.lo / TK * TK, last = r.hi;
  f32x16 dq[2] = {zeros(), zeros()};
  if (first < last) {
    if (!early) {
      ks.load(first);
      vs.load(first);
    }
    ks.store(lds);
    vs.store(lds + kTileBytes);
  }
  __syncthreads();
  for (int k0 = first, buf = 0; k0 < last; k0 += TK, buf ^= 2 * kTileBytes) {
    const bool more = k0 + TK < last;
    if (more) {
      ks.load(k0 + TK);
      vs.load(k0 + TK);
    }
    const int mine = k0 + 32 * w;
    if (mine < r.hi && mine + 32 > r.lo) {
      const char* kt = lds + buf + w * 32 * kRowBytes;
      const char* vt = kt + kTileBytes;
      f32x16 x = zeros(), y = zeros();
#pragma unroll
      for (int k = 0; k < 4; ++k) x = mfma32(read_rows(kt, l, 0, k), q[k], x);
#pragma unroll
      for (int k = 0; k < 4; ++k) y = mfma32(read_rows(vt, l, 0, k), go[k], y);
#pragma unroll
      for (int e = 0; e < 16; ++e) y[e] -= delta;
      if (mine < r.all_lo || mine + 32 > r.all_hi) hide(keys, mine + 4 * l.h, x, y);
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] = __builtin_amdgcn_exp2f(fmaf(x[e], kScale2, -lse)) * y[e];
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        bf16x8 rest;
        const bf16x8 ds = narrow(x, 8 * c, rest);
#pragma unroll
        for (int d = 0; d < 2; ++d) {
          const bf16x8 k = read_cols(kt, l, d, c);
          dq[d] = mfma32(k, ds, dq[d]);
          dq[d] = mfma32(k, rest, dq[d]);
        }
      }
    }
    if (more) {
      ks.store(lds + (buf ^ (2 * kTileBytes)));
      vs.store(lds + (buf ^ (2 * kTileBytes)) + kTileBytes);
    }
    __syncthreads();
  }
  // the other waves' sums to the first one, which goes on alone
  float* part = (float*)lds;
  if (w > 0)
#pragma unroll
    for (int d = 0; d < 2; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) part[((w - 1) * 32 + 16 * d + e) * 64 + threadIdx.x % kWave] = dq[d][e];
  __syncthreads();
  if (w > 0) return;
#pragma unroll
  for (int d = 0; d < 2; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e)
#pragma unroll
      for (int u = 0; u < 3; ++u) dq[d][e] += part[(u * 32 + 16 * d + e) * 64 + threadIdx.x];
  dq_out(a, s, h, q0, in, l, lds, dq);
}

// dq of four waves of 32 queries that share tiles of 64 keys: as the forward kernel, with p from lse and two
// products more, dP^T = V dO^T and, from dS, dQ^T = K^T dS^T.  dP's accumulator starts from -delta.  It leaves delta
// (unless both gradients are in one launch) and what 32 queries see together for the kernel of dk and dv.
// 32 x 448 x 1500, 20 heads: 271 us (the median of traced launches; least 243), twice the products of the forward pass.
template <bool DIRECT>
__device__ __forceinline__ void dq_wide(const AttnBwdArgs& a, int tiles) {
  constexpr int TK = 64;
  __shared__ uint4 key0[512], key1[512], val0[512], val1[512];
  __shared__ int ends[8];
  Place at = place_of(a.b.heads, a.b.per_head, a.b.batch);
  if (!at.in) return;
  if (a.b.causal) at.tile = tiles - 1 - at.tile;        // (the longest first)
  const int h = at.h;
  const Span s = span_of(a.b, at.b);
  if (!s.ok) {
    if (threadIdx.x == 0) atomicOr(a.b.err, AD_ERR_LENGTH);
    return;
  }
  if (at.tile * 128 >= s.oq) return;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), g = key_head(a.b, h);
  const Lane l(threadIdx.x % kWave);
  const int q0 = at.tile * 128 + 32 * w, i = q0 + l.n;
  const bool in = i < s.nq;
  const int64_t row = s.q0 + (int64_t)i;
  Loads<DIRECT> ks, vs;
  ks.init(a.k, s.k0, s.nk, 64 * g);
  vs.init(a.v, s.k0, s.nk, 64 * g);
  // (without windows the first tile is under way before anything else is asked for)
  int first = 0, last = ends_at(a.b, s, at.tile * 128, 128);
  if (!a.b.window && last > 0) {
    ks.issue(0, key0);
    vs.issue(0, val0);
  }
  Rows rq, rg, ro, rr;
  rq.load(a.q, s.q0 + (int64_t)q0, s.nq - q0, 64 * h);
  rg.load(a.dout, s.q0 + (int64_t)q0, s.nq - q0, 64 * h);
  ro.load(a.o, s.q0 + (int64_t)q0, s.nq - q0, 64 * h);
  rr.load(a.rest, s.q0 + (int64_t)q0, a.rest.p ? s.nq - q0 : 0, 64 * h);
  float lse = 0.f;
  Keys keys = {0, s.nk};
  if (in) {
    keys = keys_of(a.b, s, i);
    lse = a.lse[(size_t)h * a.b.q_rows + row] * kLog2e;
  }
  const Range r = range_at(a.b, s, q0, keys, in);
  if (a.b.window) {
    if (threadIdx.x % kWave == 0) {
      if (h == 0 && q0 < s.nq) a.ranges[(size_t)at.b * a.blocks + q0 / 32] = make_int4(r.lo, r.hi, r.all_lo, r.all_hi);
      ends[w] = r.lo;
      ends[4 + w] = r.hi;
    }
    __syncthreads();
    first = __builtin_amdgcn_readfirstlane(min(min(ends[0], ends[1]), min(ends[2], ends[3])) / TK * TK);
    last = __builtin_amdgcn_readfirstlane(max(max(ends[4], ends[5]), max(ends[6], ends[7])));
    if (first < last) {
      ks.issue(first, key0);
      vs.issue(first, val0);
    }
  }

  if (lse == -INFINITY) lse = INFINITY;     // sees nothing: p = exp2(s - inf) = 0
  char* buf = (char*)((w < 2 ? key1 : val1) + w % 2 * 256);
  bf16x8 q[4], go[4];
  rq.operand(buf, l, q);
  rg.operand(buf, l, go);
  // delta: a row's eight lanes add up, and hand it over in the operand's order
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float d[8], o[8], e[8], sum = 0.f;
    widen8(__builtin_bit_cast(u32x4, rg.reg[j]), d);
    widen8(__builtin_bit_cast(u32x4, ro.reg[j]), o);
    widen8(__builtin_bit_cast(u32x4, rr.reg[j]), e);
#pragma unroll
    for (int c = 0; c < 8; ++c) sum = fmaf(d[c], o[c] + e[c], sum);
    sum += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(sum), 0xB1, 0xf, 0xf, false));    // lane ^ 1
    sum += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(sum), 0x4E, 0xf, 0xf, false));    // lane ^ 2
    sum += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(sum), 0x141, 0xf, 0xf, false));   // 7 - lane
    if (threadIdx.x % 8 == 0) ((float*)buf)[Rows::row(j)] = sum;
  }
  __builtin_amdgcn_wave_barrier();
  const float delta = ((const float*)buf)[l.n];
  settled(q);
  settled(go);
  if (a.delta && in && l.h == 0) a.delta[(size_t)h * a.b.q_rows + row] = delta;
  f32x16 dq[2] = {zeros(), zeros()}, off;     // off: dP - delta starts from -delta
#pragma unroll
  for (int e = 0; e < 16; ++e) off[e] = -delta;
  const auto step = [&](int k0, const uint4* kt, const uint4* vt, uint4* next_kt, uint4* next_vt) {
    const bool more = k0 + TK < last;
    if (more) {
      ks.issue(k0 + TK, next_kt);
      vs.issue(k0 + TK, next_vt);
    }
    if (k0 < r.hi && k0 + TK > r.lo) {
      const bool cut = k0 < r.all_lo || k0 + TK > r.all_hi;
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        f32x16 x = zeros(), y = off;
#pragma unroll
        for (int k = 0; k < 4; ++k) x = mfma32(read_rows((const char*)kt, l, n, k), q[k], x);
#pragma unroll
        for (int k = 0; k < 4; ++k) y = mfma32(read_rows((const char*)vt, l, n, k), go[k], y);
        if (cut) hide(keys, k0 + 32 * n + 4 * l.h, x, y);
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = __builtin_amdgcn_exp2f(fmaf(x[e], kScale2, -lse)) * y[e];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          bf16x8 rest;
          const bf16x8 ds = narrow(x, 8 * c, rest);
#pragma unroll
          for (int d = 0; d < 2; ++d) {
            const bf16x8 k = read_cols((const char*)kt, l, d, 2 * n + c);
            dq[d] = mfma32(k, ds, dq[d]);
            dq[d] = mfma32(k, rest, dq[d]);
          }
        }
      }
    }
    if (more) {
      ks.arrive(next_kt);
      vs.arrive(next_vt);
    }
    landed();
  };
  if (first < last) {
    ks.arrive(key0);
    vs.arrive(val0);
    landed();
    for (int k0 = first; k0 < last; k0 += 2 * TK) {
      step(k0, key0, val0, key1, val1);
      if (k0 + TK >= last) break;
      step(k0 + TK, key1, val1, key0, val0);
    }
  }
  if (first >= last) __syncthreads();      // (another wave's rows may still be in the place that is written next)
  dq_out(a, s, h, q0, in, l, (char*)(w == 0 ? key0 : w == 1 ? key1 : w == 2 ? val0 : val1), dq);
}

template <bool DIRECT>
__global__ void __launch_bounds__(256, DIRECT ? 3 : 2) attn_dq_wide_kernel(AttnBwdArgs a, int tiles) {
  dq_wide<DIRECT>(a, tiles);
}

// dk and dv: the same with the queries on the rows (S = Q K^T), a wave 32 keys and all of the queries that
// see them, of every head that shares them.

// What the products need of a tile's TQ queries besides their rows, on its way to LDS: [TQ] each of lse in powers of
// two (+infinity where a row sees nothing: p = 0), -delta, and the keys [lo, hi) that the query sees.
// OWN (TQ = 64): delta is computed here, four threads a query.
template <int TQ, bool OWN = false>
struct StatLoads {
  float lse, delta;
  int lo, hi, i;
  uint4 row[OWN ? 6 : 1];
  // (nothing waits for what is loaded here)
  __device__ __forceinline__ void issue(const AttnBwdArgs& a, const Span& s, int h, int i0) {
    i = i0 + (int)(OWN ? threadIdx.x / 4 : threadIdx.x);
    lse = delta = 0.f;
    lo = 0;
    hi = s.nk;
    if constexpr (OWN) {
#pragma unroll
      for (int c = 0; c < 6; ++c) row[c] = make_uint4(0, 0, 0, 0);
      if (i < s.nq) {
        const int64_t r = s.q0 + (int64_t)i;
        const int col = 64 * h + 16 * (threadIdx.x % 4);
        lse = a.lse[(size_t)h * a.b.q_rows + r];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          row[c] = load16(a.dout.p + r * a.dout.ld + col + 8 * c);
          row[2 + c] = load16(a.o.p + r * a.o.ld + col + 8 * c);
          if (a.rest.p) row[4 + c] = load16(a.rest.p + r * a.rest.ld + col + 8 * c);
        }
      }
    } else if (threadIdx.x < TQ && i < s.nq) {
      const size_t at = (size_t)h * a.b.q_rows + s.q0 + i;
      lse = a.lse[at];
      delta = a.delta[at];
      if (a.b.window) {
        lo = a.b.window[2 * ((size_t)s.q0 + i)];
        hi = a.b.window[2 * ((size_t)s.q0 + i) + 1];
      }
    }
  }
  __device__ __forceinline__ void arrive(const AttnBwdArgs& a, const Span& s, float* to) {
    if constexpr (OWN) {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float d[8], o[8], r[8];
        widen8(__builtin_bit_cast(u32x4, row[c]), d);
        widen8(__builtin_bit_cast(u32x4, row[2 + c]), o);
        widen8(__builtin_bit_cast(u32x4, row[4 + c]), r);
#pragma unroll
        for (int e = 0; e < 8; ++e) delta = fmaf(d[e], o[e] + r[e], delta);
      }
      delta += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(delta), 0xB1, 0xf, 0xf, false));   // lane ^ 1
      delta += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(delta), 0x4E, 0xf, 0xf, false));   // lane ^ 2
    }
    const int n = OWN ? threadIdx.x / 4 : threadIdx.x;
    if (OWN ? threadIdx.x % 4 == 0 : threadIdx.x < TQ) {
      const bool none = lse == -INFINITY || i >= s.nq;     // sees nothing
      int end = min(hi, s.nk);
      if (a.b.causal) end = min(end, i + s.nk - s.nq + 1);
      to[n] = i >= s.nq ? 0.f : none ? INFINITY : lse * kLog2e;
      to[TQ + n] = -delta;
      ((int*)to)[2 * TQ + n] = lo;
      ((int*)to)[3 * TQ + n] = none ? lo : end;
    }
  }
};

// (the first kernel's table is constant here: scalar loads)
typedef const __attribute__((address_space(4))) int* Table;
__device__ __forceinline__ Table ranges_of(const AttnBwdArgs& a, int b) {
  return (Table)(uintptr_t)(a.ranges + (size_t)b * a.blocks);
}

__device__ __forceinline__ void keys_operands(const AttnBwdArgs& a, const Span& s, int g, int j, const Lane& l, bf16x8 (&k)[4],
                                              bf16x8 (&v)[4]) {
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    uint4 uk = make_uint4(0, 0, 0, 0), uv = uk;
    if (j < s.nk) {
      const int64_t row = s.k0 + (int64_t)j;
      uk = load16(a.k.p + row * a.k.ld + 64 * g + 16 * c + 8 * l.h);
      uv = load16(a.v.p + row * a.v.ld + 64 * g + 16 * c + 8 * l.h);
    }
    k[c] = as_bf16x8(uk);
    v[c] = as_bf16x8(uv);
  }
  settled(k);
  settled(v);
}
// 32 queries (tiles qt of q and gt of dout) and the wave's 32 keys, this lane's being key j.  stat: of the lane's first
// query; cut: some of the queries do not see some of the keys.
template <int TQ>
__device__ __forceinline__ void dkv_block(const char* qt, const char* gt, const float* stat, bool cut, int j, const Lane& l,
                                          const bf16x8 (&k)[4], const bf16x8 (&v)[4], f32x16 (&dk)[2], f32x16 (&dv)[2]) {
  f32x16 x = zeros(), y;       // dP - delta: the product starts from -delta
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const f32x4 d = *(const f32x4*)(stat + TQ + 8 * e);
#pragma unroll
    for (int c = 0; c < 4; ++c) y[4 * e + c] = d[c];
  }
#pragma unroll
  for (int c = 0; c < 4; ++c) x = mfma32(read_rows(qt, l, 0, c), k[c], x);
#pragma unroll
  for (int c = 0; c < 4; ++c) y = mfma32(read_rows(gt, l, 0, c), v[c], y);
  if (cut) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int4 lo = *(const int4*)(stat + 2 * TQ + 8 * e), hi = *(const int4*)(stat + 3 * TQ + 8 * e);
      const int los[4] = {lo.x, lo.y, lo.z, lo.w}, his[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const bool seen = j >= los[c] && j < his[c];
        x[4 * e + c] = seen ? x[4 * e + c] : -INFINITY;
        y[4 * e + c] = seen ? y[4 * e + c] : 0.f;
      }
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const f32x4 lse = *(const f32x4*)(stat + 8 * e);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      x[4 * e + c] = __builtin_amdgcn_exp2f(fmaf(x[4 * e + c], kScale2, -lse[c]));
      y[4 * e + c] *= x[4 * e + c];
    }
  }
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const bf16x8 p = narrow(x, 8 * c), ds = narrow(y, 8 * c);
#pragma unroll
    for (int d = 0; d < 2; ++d) {
      dv[d] = mfma32(read_cols(gt, l, d, c), p, dv[d]);
      dk[d] = mfma32(read_cols(qt, l, d, c), ds, dk[d]);
    }
  }
}
// The 32 keys from j0 on.
__device__ __forceinline__ void dkv_out(const AttnBwdArgs& a, const Span& s, int g, int j0, const Lane& l, char* buf,
                                        f32x16 (&dk)[2], f32x16 (&dv)[2]) {
  const bool in = j0 + l.n < s.nk;
  bool bad = false;
#pragma unroll
  for (int d = 0; d < 2; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      dk[d][e] = in ? dk[d][e] * kScale : 0.f;
      dv[d][e] = in ? dv[d][e] : 0.f;
      bad |= !(fabsf(dk[d][e]) < INFINITY) || !(fabsf(dv[d][e]) < INFINITY);
    }
  uint32_t again = columns(bad);
  by_rows(buf, l, dk, [&](int n, int c, const float(&x)[8]) {
    if (j0 + n < s.ow && !(again >> n & 1)) store_piece(a.dk, s.k0 + (int64_t)(j0 + n), g, c, narrow8(x));
  });
  __builtin_amdgcn_wave_barrier();
  by_rows(buf, l, dv, [&](int n, int c, const float(&x)[8]) {
    if (j0 + n < s.ow && !(again >> n & 1)) store_piece(a.dv, s.k0 + (int64_t)(j0 + n), g, c, narrow8(x));
  });
  for (; again; again &= again - 1) dkv_row(a, s, g, j0 + __builtin_ctz(again));
}

// Four waves of 32 keys share tiles of 64 queries: four products a pair of tiles (S, dP, dV, dK).  64 accumulators
// and 32 operands of its own leave 190 registers' worth of work: two workgroups a CU (three by force: 34 registers
// spilled, 15% slower).  32 x 448 x 1500, 20 heads: 363 us (the median of traced launches; least 327); one 5000-long causal
// sequence, 12 heads, has 480 workgroups, of which the longest alone takes as long as all: 175 us (dq: 154).
template <bool DIRECT, bool OWN>
__device__ __forceinline__ void dkv_wide(const AttnBwdArgs& a, int before) {
  constexpr int TQ = 64;
  __shared__ uint4 q0[512], q1[512], g0[512], g1[512];
  __shared__ __attribute__((aligned(16))) float stat0[4 * TQ], stat1[4 * TQ];
  Place at = place_of(a.b.kv_heads, a.b.per_kv_head, a.b.batch);
  at.tile -= before;
  if (!at.in) return;
  const int g = at.h;
  const Span s = span_of(a.b, at.b);
  if (!s.ok) {
    if (threadIdx.x == 0) atomicOr(a.b.err, AD_ERR_LENGTH);
    return;
  }
  if (at.tile * 128 >= s.ow) return;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const Lane l(threadIdx.x % kWave);
  const int j0 = at.tile * 128 + 32 * w, j = j0 + l.n;
  Walk<TQ, Table> walk(a.b, s, ranges_of(a, at.b), g, at.tile * 128, min(at.tile * 128 + 128, s.nk));
  Loads<DIRECT> qs, gs;
  StatLoads<TQ, OWN> ss;
  qs.init(a.q, s.q0, s.nq, 0);
  gs.init(a.dout, s.q0, s.nq, 0);
  f32x16 dk[2] = {zeros(), zeros()}, dv[2] = {zeros(), zeros()};
  const auto issue = [&](uint4* qt, uint4* gt) {
    qs.issue(walk.t * TQ, qt, 128 * walk.h);
    gs.issue(walk.t * TQ, gt, 128 * walk.h);
    ss.issue(a, s, walk.h, walk.t * TQ);
  };
  const auto arrive = [&](uint4* qt, uint4* gt, float* stat) {
    qs.arrive(qt);
    gs.arrive(gt);
    ss.arrive(a, s, stat);
  };
  bool some = walk.settle();
  if (some) issue(q0, g0);
  Rows rk, rv;
  rk.load(a.k, s.k0 + (int64_t)j0, s.nk - j0, 64 * g);
  rv.load(a.v, s.k0 + (int64_t)j0, s.nk - j0, 64 * g);
  bf16x8 k[4], v[4];
  char* buf = (char*)((w < 2 ? q1 : g1) + w % 2 * 256);
  rk.operand(buf, l, k);
  rv.operand(buf, l, v);
  settled(k);
  settled(v);
  const auto step = [&](const uint4* qt, const uint4* gt, const float* stat, uint4* next_qt, uint4* next_gt, float* next_stat) {
    const int now = walk.t;
    ++walk.t;
    some = walk.settle();
    if (some) issue(next_qt, next_gt);
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const int u = 2 * now + n;
      if (32 * u >= s.nq) continue;
      const Range r = walk.seen(u);
      if (r.lo >= j0 + 32 || r.hi <= j0) continue;
      dkv_block<TQ>((const char*)qt + n * 32 * kRowBytes, (const char*)gt + n * 32 * kRowBytes, stat + 32 * n + 4 * l.h,
                    j0 < r.all_lo || min(j0 + 32, s.nk) > r.all_hi, j, l, k, v, dk, dv);
    }
    if (some) arrive(next_qt, next_gt, next_stat);
    landed();
  };
  if (some) {
    arrive(q0, g0, stat0);
    landed();
    while (true) {
      step(q0, g0, stat0, q1, g1, stat1);
      if (!some) break;
      step(q1, g1, stat1, q0, g0, stat0);
      if (!some) break;
    }
  } else {
    __syncthreads();      // (another wave's rows may still be in the place that is written next)
  }
  dkv_out(a, s, g, j0, l, (char*)(w == 0 ? q0 : w == 1 ? q1 : w == 2 ? g0 : g1), dk, dv);
}

template <bool DIRECT>
__global__ void __launch_bounds__(256, 2) attn_dkv_wide_kernel(AttnBwdArgs a) {
  dkv_wide<DIRECT, false>(a, 0);
}
// Both of them in one launch, for batches so small that their workgroups are on the chip at once (512, two a CU): those
// of dk and dv then compute delta themselves from dout, o and its rest.  12 x 128 causal, 20 heads: 23 us in two
// launches, 17 in one.
template <bool DIRECT>
__global__ void __launch_bounds__(256, 2) attn_bwd_both_kernel(AttnBwdArgs a, int dq_tiles) {
  if ((int)blockIdx.x / 8 < dq_tiles) dq_wide<DIRECT>(a, dq_tiles);
  else dkv_wide<DIRECT, true>(a, dq_tiles);
}

// 32 keys, the four waves a quarter of each tile of 128 queries (where there are few workgroups of 128).
__global__ void __launch_bounds__(256, 2) attn_dkv_few_kernel(AttnBwdArgs a) {
  constexpr int TQ = 128, kTileBytes = TQ * kRowBytes, kStageBytes = 2 * kTileBytes + 16 * TQ;
  __shared__ __attribute__((aligned(16))) char lds[2 * kStageBytes];
  const Place at = place_of(a.b.kv_heads, a.b.per_kv_head, a.b.batch);
  if (!at.in) return;
  const int g = at.h;
  const Span s = span_of(a.b, at.b);
  if (!s.ok) {
    if (threadIdx.x == 0) atomicOr(a.b.err, AD_ERR_LENGTH);
    return;
  }
  const int j0 = at.tile * 32;
  if (j0 >= s.ow) return;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const Lane l(threadIdx.x % kWave);
  const int j = j0 + l.n;
  bf16x8 k[4], v[4];
  keys_operands(a, s, g, j, l, k, v);
  Walk<TQ, Table> walk(a.b, s, ranges_of(a, at.b), g, j0, min(j0 + 32, s.nk));
  Stage<TQ> qs, gs;
  StatLoads<TQ> ss;
  f32x16 dk[2] = {zeros(), zeros()}, dv[2] = {zeros(), zeros()};
  const auto load = [&] {
    qs.init(a.q, s.q0, s.nq, 64 * walk.h);
    gs.init(a.dout, s.q0, s.nq, 64 * walk.h);
    qs.load(walk.t * TQ);
    gs.load(walk.t * TQ);
    ss.issue(a, s, walk.h, walk.t * TQ);
  };
  const auto store = [&](char* to) {
    qs.store(to);
    gs.store(to + kTileBytes);
    ss.arrive(a, s, (float*)(to + 2 * kTileBytes));
  };
  bool some = walk.settle();
  if (some) {
    load();
    store(lds);
  }
  __syncthreads();
  for (int buf = 0; some; buf ^= kStageBytes) {
    const int u = walk.t * (TQ / 32) + w;
    ++walk.t;
    some = walk.settle();
    if (some) load();
    if (32 * u < s.nq) {
      const Range r = walk.seen(u);
      if (r.lo < j0 + 32 && r.hi > j0)
        dkv_block<TQ>(lds + buf + w * 32 * kRowBytes, lds + buf + kTileBytes + w * 32 * kRowBytes,
                      (const float*)(lds + buf + 2 * kTileBytes) + 32 * w + 4 * l.h,
                      j0 < r.all_lo || min(j0 + 32, s.nk) > r.all_hi, j, l, k, v, dk, dv);
    }
    if (some) store(lds + (buf ^ kStageBytes));
    __syncthreads();
  }
  // the other waves' sums (48 KB) to the first one, which goes on alone
  float* part = (float*)lds;
  if (w > 0)
#pragma unroll
    for (int d = 0; d < 2; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        part[((w - 1) * 64 + 16 * d + e) * 64 + threadIdx.x % kWave] = dk[d][e];
        part[((w - 1) * 64 + 32 + 16 * d + e) * 64 + threadIdx.x % kWave] = dv[d][e];
      }
  __syncthreads();
  if (w > 0) return;
#pragma unroll
  for (int d = 0; d < 2; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e)
#pragma unroll
      for (int u = 0; u < 3; ++u) {
        dk[d][e] += part[(u * 64 + 16 * d + e) * 64 + threadIdx.x];
        dv[d][e] += part[(u * 64 + 32 + 16 * d + e) * 64 + threadIdx.x];
      }
  dkv_out(a, s, g, j0, l, lds, dk, dv);
}

}  // namespace

// rows of 16-byte pieces
bool whole(const HMat& m) { return (uintptr_t)m.p % 16 == 0 && m.ld % 8 == 0; }

dim3 grid_of(int tiles, int heads, int batch) { return dim3(8 * tiles, (heads * batch + 7) / 8); }

void launch_attention(const AttnFwdArgs& a, hipStream_t st) {
  const FwdPlan p = fwd_plan(a.b);
  if (!p.tiles || !a.b.batch) return;
  if (p.keys) return attn_fwd_keys_kernel<<<grid_of(p.tiles, a.b.heads, a.b.batch), 64 * kKeyWaves, 0, st>>>(a);
  const dim3 grid = grid_of(p.tiles * p.splits, a.b.heads, a.b.batch);
  if (p.few) attn_fwd_few_kernel<<<grid, 256, 0, st>>>(a, p.tiles, p.splits, p.chunk);
  else if (whole(a.k) && whole(a.v)) attn_fwd_wide_kernel<true><<<grid, 256, 0, st>>>(a, p.tiles);
  else attn_fwd_wide_kernel<false><<<grid, 256, 0, st>>>(a, p.tiles);
  if (p.splits > 1) attn_join_kernel<<<dim3((a.b.q_max + 3) / 4, a.b.heads, a.b.batch), 256, 0, st>>>(a, p.splits);
}

void launch_attention_backward(const AttnBwdArgs& args, hipStream_t st) {
  AttnBwdArgs a = args;
  const AttnBatch& b = a.b;
  if (!b.batch) return;
  a.blocks = (b.q_max + 31) / 32;
  a.ranges = (int4*)((char*)a.delta + attn_bwd_delta_bytes(b));
  const bool wide_q = wide_rows(b, b.q_max, b.heads), wide_k = wide_rows(b, b.k_max, b.kv_heads, true);
  const bool direct_q = whole(a.k) && whole(a.v), direct_k = whole(a.q) && whole(a.dout);
  const int tiles_q = wide_q ? (b.q_max + 127) / 128 : a.blocks, tiles_k = wide_k ? (b.k_max + 127) / 128 : (b.k_max + 31) / 32;
  const dim3 grid_q = grid_of(tiles_q, b.heads, b.batch), grid_k = grid_of(tiles_k, b.kv_heads, b.batch);
  if (!b.window && wide_q && wide_k && (size_t)grid_q.x * grid_q.y + (size_t)grid_k.x * grid_k.y <= 512) {
    a.delta = nullptr;
    const dim3 grid(grid_q.x + grid_k.x, grid_q.y);
    if (direct_q && direct_k) attn_bwd_both_kernel<true><<<grid, 256, 0, st>>>(a, tiles_q);
    else attn_bwd_both_kernel<false><<<grid, 256, 0, st>>>(a, tiles_q);
    return;
  }
  if (tiles_q > 0) {
    if (!wide_q) attn_dq_few_kernel<<<grid_q, 256, 0, st>>>(a, tiles_q);
    else if (direct_q) attn_dq_wide_kernel<true><<<grid_q, 256, 0, st>>>(a, tiles_q);
    else attn_dq_wide_kernel<false><<<grid_q, 256, 0, st>>>(a, tiles_q);
  }
  if (tiles_k > 0) {
    if (!wide_k) attn_dkv_few_kernel<<<grid_k, 256, 0, st>>>(a);
    else if (direct_k) attn_dkv_wide_kernel<true><<<grid_k, 256, 0, st>>>(a);
    else attn_dkv_wide_kernel<false><<<grid_k, 256, 0, st>>>(a);
  }
}

}  // namespace ad
