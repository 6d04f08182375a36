// Products of the draft block's training on the gfx950 matrix cores: a projection with bias,
// activation and residual, its gradient for the input, and its gradients for weight and bias.
//
// All three are out[q][p] = sum_r Q(q, r) P(p, r), p running along the output's rows in memory:
//             q          p       r      Q stored      P stored
//   forward   row m      col n   k      [m][k]        [n][k]     both contiguous along r
//   dgrad     row m      col k   n      [m][n]        [n][k]     P contiguous along p
//   wgrad     row n      col k   m      [m][n]        [m][k]     both contiguous along the output
// An operand that is contiguous along r ("KC") sits in LDS as [row][64 of r], one that is
// contiguous along its own dimension ("KS") as [64 of r][columns], each as it comes from memory,
// so that 16-byte loads go straight from memory to LDS; KS fragments are transposed by the
// LDS read itself (ds_read_b64_tr_b16: 16 lanes read four r of 16 columns, lane c gets column c's
// four).  P is the matrix instruction's first operand: a lane's four accumulators are four
// consecutive columns of one output row.  The epilogue takes them through LDS once more, a row of tiles
// at a time, to have 8 columns a lane and whole rows side by side: 16-byte stores, and four
// lanes hold a checkpoint's group of 32.  (Stored straight from the accumulators, with every choice
// made for every value, the epilogue took as long as 20 stages of products.)
//
// What bounds it.  A tile of T x T needs T^2 products for 2 T loads, and a CU takes in 25 to 60 bytes a
// clock: 128 x 128 tiles, two workgroups a CU, are bound by that (860 of 1060 us for 8192 cubed
// without any product), 256 x 256 tiles, eight waves of 128 x 64, by the products (660 us without
// loads) and what keeps the two from overlapping whole (794 us, 1385 TFLOP/s; the library's
// product 1485).  Launches too small for 256 x 256 tiles on every CU are bound by the time a stage takes
// one workgroup: they have a ring of four stages of 128 x 128 and one workgroup a CU.  Then there are
// a round's first loads and its epilogue, which nothing overlaps with 256 x 256 tiles: 13 us of 45 for
// 20 stages.  plan() weighs these by what was measured.
//
// LDS bank conflicts.  KC rows are 128 bytes: the 16-byte piece c of row r sits at place
// c ^ (r / 2 % 8), so the 16 rows that are read together cover every bank.  KS rows are 256 or
// 512 bytes: 32-byte pair t of row r sits at place t ^ (r % 4 + 4 (r / 8 % 2)) (low three bits),
// so the eight rows that 32 lanes read together do.  The direct loads store 1 KB in lane order;
// the permutation is made by the lanes' source addresses.
#include <algorithm>
#include <type_traits>

#include "linear_plan.h"
#include "train.h"

namespace ad {

namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));

// Direct loads go through buffer descriptors: a scalar base per stage and one 32-bit offset per
// lane (64-bit lane addresses cost twice the registers), and what lies past the descriptor's end
// arrives as zeros, which ends the reduction without a branch.
constexpr uint32_t kBufferFlags = 0x00020000;   // raw buffer of 32-bit elements
constexpr uint32_t kPastEnd = 0x80000000u;      // further than any offset in a tile: 255 * 2^23 + 128 bytes

__device__ __forceinline__ __amdgpu_buffer_rsrc_t descriptor(const char* base, uint32_t size) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, size, kBufferFlags);
}
__device__ __forceinline__ void buffer16(const char* base, uint32_t size, uint32_t off, uint4* lds) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(descriptor(base, size), (__attribute__((address_space(3))) void*)lds, 16, off, 0, 0, 0);
}
__device__ __forceinline__ const char* uniform(const void* p) {
  const uint64_t v = (uint64_t)p;
  return (const char*)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)v) |
                       (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32);
}

enum Src : int { SRC_DIRECT = 0, SRC_ANY = 1, SRC_CKPT = 2 };

__device__ __forceinline__ int ks_swz(int r) { return (r & 3) | ((r >> 1) & 4); }

// Eight elements moved down by `move` (0 to 8) places, zeros behind them.
__device__ __forceinline__ uint4 move_down(uint4 x, int move) {
  uint64_t lo = (uint64_t)x.y << 32 | x.x, hi = (uint64_t)x.w << 32 | x.z;
  const int bits = 16 * (move & 3);
  if (move >= 4) { lo = hi; hi = 0; }
  if (move >= 8) lo = 0;
  lo = lo >> bits | (bits ? hi << (64 - bits) : 0);
  hi >>= bits;
  return uint4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}
// Elements i .. i + 7 of a row of n < 8 (0 from n on).
__device__ __forceinline__ uint4 short_row(const uint16_t* row, int i, int n) {
  uint32_t e[8];
#pragma unroll
  for (int u = 0; u < 8; ++u) e[u] = i + u < n ? row[i + u] : 0;
  return uint4{e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16};
}

// The part of one operand's stage that a wave moves: R rows (KC) or columns (KS) x 64 of r in
// pieces of 1 KB, NW waves.  Direct: memory to LDS; otherwise through registers (any
// alignment; or a checkpoint's 8-bit values, which become bf16 on the way, exactly).
template <int R, int NW, bool KS, int SRC>
struct Loader {
  static constexpr int N = R / 8 / NW;   // pieces a wave
  static constexpr int RB = R / 8;       // 16-byte pieces in a KS row
  LinOp o;
  int r0, K, k0, w, lane;
  const char* base;       // the stage's first element
  const char* sbase;      // checkpoint: its scale
  int64_t left, sleft;    // KS: bytes from there to the end of the reduction's last row
  uint32_t size;          // the descriptor's, for the stage being loaded
  uint32_t off[N];        // bytes (a checkpoint's scale: a 32nd of its q's)
  uint4 reg[N];
  uint32_t sc[N];

  // place of this lane's 16 bytes of piece j: (row, r) of its first element
  __device__ __forceinline__ void place(int j, int& row, int& r) const {
    const int pc = w * N + j;
    if constexpr (KS) {
      const int at = pc * 64 + lane;   // 16-byte piece within the stage
      r = at / RB;
      const int t = (at % RB) / 2, u = (t & ~7) | ((t & 7) ^ ks_swz(r));
      row = u * 16 + (at & 1) * 8;
    } else {
      row = pc * 8 + lane / 8;
      r = 8 * ((lane % 8) ^ ((row >> 1) & 7));
    }
  }
  // checkpoint: 16 columns (one pair) at a time
  __device__ __forceinline__ void place_ck(int j, int& row, int& r) const {
    const int at = (w * (N / 2) + j) * 64 + lane;
    r = at / (R / 16);
    row = (at % (R / 16)) * 16;
  }

  __device__ __forceinline__ void init(const LinOp& op, int first, int K_, int k0_, int w_, int lane_) {
    o = op; r0 = first; K = K_; k0 = k0_; w = w_; lane = lane_;
    if constexpr (SRC == SRC_DIRECT) {
      base = uniform(KS ? o.p + (size_t)k0 * o.ld + r0 : o.p + (size_t)r0 * o.ld + k0);
      left = 2 * ((int64_t)(K - 1 - k0) * o.ld + (o.extent - r0));
#pragma unroll
      for (int j = 0; j < N; ++j) {
        int row, r;
        place(j, row, r);
        // rows and columns past the matrix read its last ones (their results are not stored)
        off[j] = KS ? 2u * ((uint32_t)r * (uint32_t)o.ld + (uint32_t)min(row, o.extent - 8 - r0))
                    : 2u * ((uint32_t)min(row, o.extent - 1 - r0) * (uint32_t)o.ld + (uint32_t)r);
      }
    } else if constexpr (SRC == SRC_ANY) {
      base = uniform(KS ? o.p + (size_t)k0 * o.ld : o.p + (size_t)r0 * o.ld);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        int row, r;
        place(j, row, r);
        off[j] = KS ? 2u * ((uint32_t)r * (uint32_t)o.ld + (uint32_t)min(r0 + row, max(o.extent - 8, 0)))
                    : 2u * ((uint32_t)min(row, o.extent - 1 - r0) * (uint32_t)o.ld + (uint32_t)(k0 + r));
      }
    } else if constexpr (SRC == SRC_CKPT) {
      const int ld = o.ck.ld, sld = ld / kCkptGroup;
      base = uniform(o.ck.q + (size_t)k0 * ld + r0);
      sbase = uniform(o.ck.scale + (size_t)k0 * sld + r0 / kCkptGroup);
      left = (int64_t)(K - k0) * ld - r0;
      sleft = (int64_t)(K - k0) * sld - r0 / kCkptGroup;
#pragma unroll
      for (int j = 0; j < N / 2; ++j) {
        // (columns past the padded row read the next one's; their results are not stored)
        int row, r;
        place_ck(j, row, r);
        off[j] = (uint32_t)r * ld + row;
      }
    }
  }

  // The stage at k0 into `lds` (direct) or into registers, in four parts between begin() and end().
  // Past the end of the reduction a direct load moves nothing (its descriptor is empty), so that a
  // wave's count of loads in flight does not depend on the stage.
  __device__ __forceinline__ void begin() {
    if constexpr (SRC == SRC_DIRECT && KS) {
      size = (uint32_t)max(min(left, (int64_t)kPastEnd), (int64_t)0);
    } else if constexpr (SRC == SRC_DIRECT) {
      size = k0 < K ? kPastEnd : 0;
      if (k0 + kBK > K) {   // the reduction ends in this stage
#pragma unroll
        for (int j = 0; j < N; ++j) {
          int row, r;
          place(j, row, r);
          if (k0 + r >= K) off[j] = kPastEnd;
        }
      }
    } else if constexpr (SRC == SRC_ANY) {
      if (k0 < K && k0 + kBK > K && (KS || K >= 8)) {   // (KC: off counts from the row's start)
#pragma unroll
        for (int j = 0; j < N; ++j) {
          int row, r;
          place(j, row, r);
          if (KS) off[j] -= 2u * (uint32_t)max(k0 + r - (K - 1), 0) * (uint32_t)o.ld;
          else off[j] -= 2u * (uint32_t)max(k0 + r - (K - 8), 0);
        }
      }
    }
  }
  template <int PART>
  __device__ __forceinline__ void part(uint4* lds) {
    if constexpr (SRC == SRC_DIRECT) {
#pragma unroll
      for (int j = PART * N / 4; j < (PART + 1) * N / 4; ++j) buffer16(base, size, off[j], lds + (w * N + j) * 64);
    } else if constexpr (SRC == SRC_ANY && PART == 0) {
      if (k0 >= K) return;
      // 16-byte loads of whatever alignment; a piece that reaches past the end of its row is the row's
      // last whole one for now, and commit() moves it into place (rows past the last are the last)
      const int n = KS ? o.extent : K;   // elements of a row
      if (n >= 8) {
#pragma unroll
        for (int j = 0; j < N; ++j) __builtin_memcpy(&reg[j], base + off[j], 16);
      } else {
#pragma unroll
        for (int j = 0; j < N; ++j) {
          int row, r;
          place(j, row, r);
          reg[j] = short_row(o.p + (size_t)(KS ? min(k0 + r, K - 1) : min(r0 + row, o.extent - 1)) * o.ld,
                             KS ? r0 + row : k0 + r, n);
        }
      }
    } else if constexpr (SRC == SRC_CKPT && PART == 0) {
      // past the last row: q = 0, scale byte 0 (a scale of 0)
      const __amdgpu_buffer_rsrc_t rq = descriptor(base, (uint32_t)max(min(left, (int64_t)kPastEnd), (int64_t)0));
      const __amdgpu_buffer_rsrc_t rs = descriptor(sbase, (uint32_t)max(min(sleft, (int64_t)kPastEnd), (int64_t)0));
#pragma unroll
      for (int j = 0; j < N / 2; ++j) {
        reg[j] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(rq, off[j], 0, 0));
        sc[j] = __builtin_amdgcn_raw_buffer_load_b8(rs, off[j] / kCkptGroup, 0, 0);
      }
    }
  }
  __device__ __forceinline__ void end() {
    if constexpr (SRC == SRC_DIRECT) {
      base += KS ? 2 * kBK * o.ld : (int64_t)(2 * kBK);
      if (KS) left -= 2 * kBK * o.ld;
    } else if constexpr (SRC == SRC_ANY) {
      if (KS) base += 2 * kBK * o.ld;
      else
#pragma unroll
        for (int j = 0; j < N; ++j) off[j] += 2 * kBK;
    } else if constexpr (SRC == SRC_CKPT) {
      base += kBK * (int64_t)o.ck.ld;
      left -= kBK * (int64_t)o.ck.ld;
      sbase += kBK * (int64_t)(o.ck.ld / kCkptGroup);
      sleft -= kBK * (int64_t)(o.ck.ld / kCkptGroup);
    }
    k0 += kBK;
  }
  __device__ __forceinline__ void all(uint4* lds) {
    part<0>(lds);
    part<1>(lds);
    part<2>(lds);
    part<3>(lds);
  }
  __device__ __forceinline__ void issue(uint4* lds) {
    begin();
    all(lds);
    end();
  }

  // registers into LDS, one half of them
  template <int HALF>
  __device__ __forceinline__ void commit(uint4* lds) {
    static_assert(N % 4 == 0);
    if constexpr (SRC == SRC_ANY) {
#pragma unroll
      for (int j = HALF * N / 2; j < (HALF + 1) * N / 2; ++j) {
        int row, r;
        place(j, row, r);
        const int n = KS ? o.extent : K, first = k0 - kBK;   // (k0 is the next stage's by now)
        if (n >= 8 && (KS ? r0 + R > n : first + kBK > n)) {
          const int at = KS ? r0 + row : first + r;
          reg[j] = move_down(reg[j], min(max(at - (n - 8), 0), 8));
        }
        if (KS && first + kBK > K && first + r >= K) reg[j] = uint4{0, 0, 0, 0};
        lds[(w * N + j) * 64 + lane] = reg[j];
      }
    } else if constexpr (SRC == SRC_CKPT) {
#pragma unroll
      for (int j = HALF * N / 4; j < (HALF + 1) * N / 4; ++j) {
        int row, r;
        place_ck(j, row, r);
        const int t = row / 16, u = (t & ~7) | ((t & 7) ^ ks_swz(r));
        const float two = ckpt_two(sc[j]);
        const uint32_t q[4] = {reg[j].x, reg[j].y, reg[j].z, reg[j].w};
        uint32_t b[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float v[4];
          ckpt_value4(q[i], two, v);
          b[2 * i] = f32x2_to_bf16x2(v[0], v[1]);
          b[2 * i + 1] = f32x2_to_bf16x2(v[2], v[3]);
        }
        uint4* to = lds + r * RB + u * 2;
        to[0] = uint4{b[0], b[1], b[2], b[3]};
        to[1] = uint4{b[4], b[5], b[6], b[7]};
      }
    }
  }
};

// The matrix instruction's operands of a wave: 16-row (or column) tiles tile0 .. of a stage with R rows
// (or columns).  Both layouts' permutations are exclusive-ors of address bits, so one lane
// offset serves every tile and step.  x0: a KS tile t is tile0 + (t ^ x0).
template <int R, bool KS>
struct Reader {
  uint32_t off;   // bytes
  __device__ __forceinline__ void init(int tile0, int x0, int lane) {
    const int c16 = lane & 15, g = lane >> 4;
    if constexpr (KS) {
      const int i = c16 >> 2;
      off = (8 * g + i) * R * 2 + (tile0 >> 3) * 256 + (((tile0 & 7) ^ x0 ^ ks_swz(8 * g + i)) * 32) + (c16 & 3) * 8;
    } else {
      off = (tile0 * 16 + c16) * 128 + ((g ^ (c16 >> 1)) * 16);
    }
  }
  // (the offsets of the tiles are recomputed at each use: kept, they would take the registers
  // that hold the products)
  __device__ __forceinline__ uint32_t fresh() const {
    uint32_t o = off;
    asm volatile("" : "+v"(o));
    return o;
  }
  // tile t of at most 8 (KS: tile0 a multiple of the tiles read), 32-wide step s
  static __device__ __forceinline__ bf16x8 read(const uint4* lds, uint32_t o, int t, int s) {
    if constexpr (KS) {
      const char* p = (const char*)lds + (o ^ (t * 32)) + s * 64 * R;
      typedef __attribute__((address_space(3))) s16x4* lp;
      const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)p);
      const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(p + 8 * R));
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      return as_bf16x8(*(const uint4*)((const char*)lds + (o ^ (s * 64)) + t * 2048));
    }
  }
};

// The epilogue where not every matrix and parameter allows whole vectors, of the joined tiles, and of few
// rows.  Few rows ask for what it reads (the residual and the bias of 8 columns of a row) before
// their product, and have whole vectors.
struct Extra {
  u32x4 lo, hi;
  float bias[8];
};
__device__ __forceinline__ Extra request(const LinArgs& a, int q, int c) {
  Extra e{};
  if (q >= a.Q.extent || c >= a.P.extent) return e;
  if (a.res.p && a.res.bf16) {
    e.lo = *(const u32x4*)((const uint16_t*)a.res.p + (size_t)q * a.res.ld + c);
  } else if (a.res.p) {
    const float* p = (const float*)a.res.p + (size_t)q * a.res.ld + c;
    e.lo = *(const u32x4*)p;
    e.hi = *(const u32x4*)(p + 4);
  }
  if (a.bias.p) load_vec8<true>(a.bias, c, a.P.extent, e.bias);
  return e;
}

// Columns c .. c + 7 of output row q (four neighbouring lanes hold one checkpoint group of 32; every
// lane of the wave calls this).  qsum: wgrad's sum of dy for row q.  FEW: `e` is what request()
// asked for.
template <int KIND, bool FEW = false>
__device__ __forceinline__ void epilogue(const LinArgs& a, int q, int c, float (&h)[8], float qsum, const Extra& e = {}) {
  const int cols = a.P.extent;
  const bool row = q < a.Q.extent;
  if constexpr (KIND == LIN_FWD) {
    float b[8];
    if (a.bias.p) {
      if (!FEW) load_vec8(a.bias, c, cols, b);
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] += FEW ? e.bias[i] : b[i];
    }
    if (a.pre.p && row) store8<FEW>(a.pre, q, c, cols, h);
    if (!FEW && a.ck.q) {
      float z[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) z[i] = c + i < cols ? h[i] : 0.f;   // (padding is written as 0)
      ckpt_store8(a.ck, q, row ? c : a.ck.ld, z);
    }
    if (!row) return;
    if (a.gelu)
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] = gelu_value(h[i]);
    if (a.res.p) {
      if (!FEW) {
        load8(a.res, q, c, cols, b);
      } else if (a.res.bf16) {
        widen8(e.lo, b);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          b[i] = __uint_as_float(e.lo[i]);
          b[4 + i] = __uint_as_float(e.hi[i]);
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] += b[i];
    }
    store8<FEW>(a.out, q, c, cols, h);
  } else if constexpr (KIND == LIN_DGRAD) {
    if (!row) return;
    if (a.gelu) {
      float x[8];
      if (a.ck.q) {
        ckpt_load8(a.ck, q, c, x);
      } else {
        load8(a.pre, q, c, cols, x);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const Normal n = normal(x[i]);
        h[i] *= gelu_slope(x[i], n);
        x[i] = gelu_value(x[i], n);
      }
      if (a.act_out.p) store8(a.act_out, q, c, cols, x);
    }
    store8(a.out, q, c, cols, h);
  } else {
    if (!row) return;
    if (a.gain.p) {
      float g[8], b[8];
      load_vec8(a.gain, c, cols, g);
      load_vec8(a.shift, c, cols, b);
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] = fmaf(h[i], g[i], b[i] * qsum);
    }
    if (a.accumulate) {
      float o[8];
      load8(a.out, q, c, cols, o);
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] += o[i];
    }
    store8(a.out, q, c, cols, h);
    if (a.dbias && c == 0) a.dbias[q] = a.accumulate ? a.dbias[q] + qsum : qsum;
  }
}

// The same where every matrix and parameter allows whole vectors, for the rows of one tile from q0 on and
// this lane's columns c .. c + 7: memory is reached through buffer descriptors, which leave out rows
// and columns past the last (no branches, 32-bit offsets), and parameters are read once.
struct TileMat {
  const char* base;
  uint32_t size, row, lane;   // bytes: to the end of the last row, of a row, of this lane's columns
  __device__ __forceinline__ void init(const void* p, int64_t ld, int bytes, int width, int q0, int rows, int c, int cols) {
    base = uniform((const char*)p + (int64_t)q0 * ld * bytes);
    size = rows > q0 ? (uint32_t)min(((int64_t)(rows - 1 - q0) * ld + width) * bytes, (int64_t)kPastEnd) : 0;
    row = (uint32_t)ld * bytes;
    lane = c < cols ? (uint32_t)c * bytes : kPastEnd;
  }
  __device__ __forceinline__ uint32_t at(int r) const { return lane + (uint32_t)r * row; }
  __device__ __forceinline__ u32x4 get(uint32_t off) const {
    return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(descriptor(base, size), off, 0, 0));
  }
  __device__ __forceinline__ void put(u32x4 v, uint32_t off) const {
    __builtin_amdgcn_raw_buffer_store_b128(v, descriptor(base, size), off, 0, 0);
  }
};
struct TileRows {   // float32 or bf16 rows
  TileMat m;
  bool bf16;
  __device__ __forceinline__ void init(const DMat& d, int q0, int rows, int c, int cols) {
    bf16 = d.bf16;
    m.init(d.p, d.ld, bf16 ? 2 : 4, cols, q0, d.p ? rows : 0, c, cols);
  }
  template <int N>
  __device__ __forceinline__ void store(int r, int step, const float (&v)[N][8]) const {
    if (bf16) {
#pragma unroll
      for (int n = 0; n < N; ++n)
        m.put(u32x4{f32x2_to_bf16x2(v[n][0], v[n][1]), f32x2_to_bf16x2(v[n][2], v[n][3]),
                    f32x2_to_bf16x2(v[n][4], v[n][5]), f32x2_to_bf16x2(v[n][6], v[n][7])}, m.at(r + n * step));
    } else {
#pragma unroll
      for (int n = 0; n < N; ++n) {
        m.put(__builtin_bit_cast(u32x4, f32x4{v[n][0], v[n][1], v[n][2], v[n][3]}), m.at(r + n * step));
        m.put(__builtin_bit_cast(u32x4, f32x4{v[n][4], v[n][5], v[n][6], v[n][7]}), m.at(r + n * step) + 16);
      }
    }
  }
};
// What the input's gradient multiplies by: nothing, or the slope at a pre-activation of this kind.  (A choice
// inside the kernel would keep the waits for it from being exact.)
enum Slope : int { SLOPE_NONE = 0, SLOPE_BF16 = 1, SLOPE_CKPT = 2 };
template <int KIND, int SLOPE>
struct TileEpilogue {
  TileRows out, in, also;    // in: residual, pre-activation or old gradient; also: pre or act_out
  TileMat q, scale;          // the checkpoint
  float b[8], g[8];          // bias; wgrad: shift and gain
  int c;
  struct Ask {
    u32x4 lo, hi;
    uint32_t s;
  };
  __device__ __forceinline__ void init(const LinArgs& a, int q0, int c_) {
    c = c_;
    const int cols = a.P.extent, rows = a.Q.extent;
    out.init(a.out, q0, rows, c, cols);
    in.init(KIND == LIN_FWD ? a.res : KIND == LIN_DGRAD ? a.pre : a.out, q0, rows, c, cols);
    also.init(KIND == LIN_FWD ? a.pre : a.act_out, q0, rows, c, cols);
    if constexpr (KIND != LIN_WGRAD) {
      const int ld = a.ck.ld, n = a.ck.q ? rows : 0;
      q.init(a.ck.q, ld, 1, ld, q0, n, c, ld);
      // (one lane of a group's four holds its scale's place when storing)
      scale.init(a.ck.scale, ld / kCkptGroup, 1, ld / kCkptGroup, q0, n, c / kCkptGroup,
                 c < ld && (KIND == LIN_DGRAD || c % kCkptGroup == 0) ? ld : 0);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = g[i] = 0.f;
    if (KIND == LIN_FWD && a.bias.p) load_vec8<true>(a.bias, c, cols, b);
    if (KIND == LIN_WGRAD && a.gain.p) {
      load_vec8<true>(a.gain, c, cols, g);
      load_vec8<true>(a.shift, c, cols, b);
    }
  }
  // N rows, `step` apart from r on.  Every choice is made once for all of them: the compiler waits for
  // everything in flight where two ways meet.
  template <int N>
  __device__ __forceinline__ void ask(const LinArgs& a, int r, int step, Ask (&e)[N]) const {
    if constexpr (KIND == LIN_DGRAD) {
      if constexpr (SLOPE == SLOPE_CKPT) {
#pragma unroll
        for (int n = 0; n < N; ++n) {
          const auto w = __builtin_amdgcn_raw_buffer_load_b64(descriptor(q.base, q.size), q.at(r + n * step), 0, 0);
          e[n].lo[0] = w[0];
          e[n].lo[1] = w[1];
          e[n].s = __builtin_amdgcn_raw_buffer_load_b8(descriptor(scale.base, scale.size), scale.at(r + n * step), 0, 0);
        }
      }
      if (SLOPE != SLOPE_BF16) return;
    } else if (KIND == LIN_FWD ? !a.res.p : !a.accumulate) {
      return;
    }
#pragma unroll
    for (int n = 0; n < N; ++n) e[n].lo = in.m.get(in.m.at(r + n * step));
    if (KIND == LIN_DGRAD || in.bf16) return;   // (a kept pre-activation is bf16)
#pragma unroll
    for (int n = 0; n < N; ++n) e[n].hi = in.m.get(in.m.at(r + n * step) + 16);
  }
  // (items I0 .. I0 + N - 1 of those asked for)
  template <int I0, int N, int M>
  __device__ __forceinline__ void received(const Ask (&e)[M], float (&v)[N][8]) const {
    if (KIND == LIN_DGRAD || in.bf16) {
#pragma unroll
      for (int n = 0; n < N; ++n) widen8(e[I0 + n].lo, v[n]);
    } else {
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v[n][i] = __uint_as_float(e[I0 + n].lo[i]);
          v[n][4 + i] = __uint_as_float(e[I0 + n].hi[i]);
        }
    }
  }
  template <int I0, int N, int M>
  __device__ __forceinline__ void rows(const LinArgs& a, int r, int step, float (&h)[N][8], const float (&qsum)[N],
                                       const Ask (&e)[M]) const {
    float x[N][8];
    if constexpr (KIND == LIN_FWD) {
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int i = 0; i < 8; ++i) h[n][i] += b[i];
      if (a.pre.p) also.store(r, step, h);
      if (a.ck.q) {
#pragma unroll
        for (int n = 0; n < N; ++n) {
          uint32_t s;
          const u32x2 w = ckpt_of8(c < a.P.extent, h[n], s);
          __builtin_amdgcn_raw_buffer_store_b64(w, descriptor(q.base, q.size), q.at(r + n * step), 0, 0);
          __builtin_amdgcn_raw_buffer_store_b8((uint8_t)s, descriptor(scale.base, scale.size), scale.at(r + n * step), 0, 0);
        }
      }
      if (a.gelu)
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
          for (int i = 0; i < 8; ++i) h[n][i] = gelu_value(h[n][i]);
      if (a.res.p) {
        received<I0>(e, x);
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
          for (int i = 0; i < 8; ++i) h[n][i] += x[n][i];
      }
    } else if constexpr (KIND == LIN_DGRAD) {
      if constexpr (SLOPE != SLOPE_NONE) {
        if constexpr (SLOPE == SLOPE_CKPT) {
#pragma unroll
          for (int n = 0; n < N; ++n) ckpt_value8(u32x2{e[I0 + n].lo[0], e[I0 + n].lo[1]}, e[I0 + n].s, x[n]);
        } else {
          received<I0>(e, x);
        }
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const Normal z = normal(x[n][i]);
            h[n][i] *= gelu_slope(x[n][i], z);
            x[n][i] = gelu_value(x[n][i], z);
          }
        if (a.act_out.p) also.store(r, step, x);
      }
    } else {
      if (a.gain.p)
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
          for (int i = 0; i < 8; ++i) h[n][i] = fmaf(h[n][i], g[i], b[i] * qsum[n]);
      if (a.accumulate) {
        received<I0>(e, x);
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
          for (int i = 0; i < 8; ++i) h[n][i] += x[n][i];
      }
    }
    out.store(r, step, h);
  }
};

// Workgroups are dealt round-robin over the 8 XCDs: number id of n, so ordered that each XCD has a
// contiguous range.
__device__ __forceinline__ int xcd_order(int id, int n) {
  const int x = id % 8;
  return x * (n / 8) + min(x, n % 8) + id / 8;
}
// Place of tile t: bands of 4 row tiles, column by column inside a band, so that neighbours in the
// order (the workgroups of one XCD) share both operands through its L2 (8 or 16: up to 3% slower).
__device__ __forceinline__ void tile_of(int t, int tp, int tq, int& ip, int& iq) {
  const int band = t / (4 * tp), rest = t % (4 * tp), h = min(4, tq - band * 4);
  iq = band * 4 + rest % h;
  ip = rest / h;
}

// The order inside a phase: its LDS reads, and LOADS loads of a later stage, spread between its
// products (VALU: and that many conversions of a checkpoint after each product).
template <int READS, int PRODUCTS, int LOADS = 0, int VALU = 0, int I = 0>
__device__ __forceinline__ void interleave() {
  if constexpr (I < READS) {
    constexpr int kLoad = LOADS * (I + 1) / READS - LOADS * I / READS;
    constexpr int kProducts = PRODUCTS * (I + 1) / READS - PRODUCTS * I / READS;
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);                                 // an LDS read
    if constexpr (kLoad > 0) __builtin_amdgcn_sched_group_barrier(0x020, kLoad, 0);    // loads
    if constexpr (VALU == 0 && kProducts > 0) {
      __builtin_amdgcn_sched_group_barrier(0x008, kProducts, 0);                       // products
    } else if constexpr (VALU > 0) {
#pragma unroll
      for (int j = 0; j < kProducts; ++j) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, VALU, 0);
      }
    }
    interleave<READS, PRODUCTS, LOADS, VALU, I + 1>();
  }
}

// The s_waitcnt immediate for at most n vector-memory operations outstanding and every LDS read done.
constexpr int wait_for(int n) { return (n & 15) | ((n >> 4) << 14) | 0x0070; }

// WP x WQ waves of TP x TQ 16 x 16 tiles, a ring of ST LDS stages (2 or 4; 2 where an operand goes
// through registers).  A stage is two 32-wide steps of G phases each (a half or a quarter of the
// wave's P tiles).  While a wave multiplies in one phase it reads the next one's operands, so no
// product waits for LDS.  The barrier falls before the stage's last phase, when all
// of it is in registers and its LDS is free: the loads of the stage ST later start there.
// SLOPE: what the epilogue of direct operands reads (the other one sees for itself).
template <int KIND, int WP, int WQ, int TP, int TQ, int ST, bool PKS, int PSRC, bool QKS, int QSRC, int SLOPE = SLOPE_NONE>
__global__ void __launch_bounds__(WP* WQ* kWave, ST == 2 && !(PSRC == SRC_CKPT && QSRC == SRC_ANY) ? 2 : 1) linear_kernel(LinArgs a) {
  constexpr int NW = WP * WQ, RP = WP * TP * 16, RQ = WQ * TQ * 16, NS = TQ / WP;
  static_assert(TP % 2 == 0 && TQ % WP == 0);
  static_assert(ST == 2 || (ST == 4 && PSRC == SRC_DIRECT && QSRC == SRC_DIRECT));
  // distinct objects, so that the compiler can tell a read of one stage from the direct loads that
  // fill another
  constexpr int kMore = ST > 2 ? 1 : 0;
  __shared__ uint4 p0[RP * 8], p1[RP * 8], q0[RQ * 8], q1[RQ * 8];
  __shared__ uint4 p2[kMore * RP * 8 + 1 - kMore], p3[kMore * RP * 8 + 1 - kMore];
  __shared__ uint4 q2[kMore * RQ * 8 + 1 - kMore], q3[kMore * RQ * 8 + 1 - kMore];
  __shared__ float sums[KIND == LIN_WGRAD ? RQ : 1];
  const int lane = threadIdx.x % kWave, w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int wp = w % WP, wq = w / WP;
  // whole tiles first, then the last `rest` tiles in S parts of the reduction each
  const int id = blockIdx.x, rest = a.tiles_p * a.tiles_q - a.whole;
  const bool part = id >= a.whole;
  const int split = part ? (id - a.whole) / rest : 0, nth = part ? (id - a.whole) % rest : 0;
  int ip, iq;
  tile_of(part ? a.whole + xcd_order(nth, rest) : xcd_order(id, a.whole), a.tiles_p, a.tiles_q, ip, iq);
  const int kbeg = split * a.steps * kBK, kend = part ? min(a.K, kbeg + a.steps * kBK) : a.K;
  const int steps = kend > kbeg ? (kend - kbeg + kBK - 1) / kBK : 0;
  Loader<RP, NW, PKS, PSRC> lp;
  Loader<RQ, NW, QKS, QSRC> lq;
  lp.init(a.P, ip * RP, kend, kbeg, w, lane);
  lq.init(a.Q, iq * RQ, kend, kbeg, w, lane);

  f32x4 acc[TP][TQ], csum[NS];
#pragma unroll
  for (int i = 0; i < TP; ++i)
#pragma unroll
    for (int j = 0; j < TQ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < NS; ++j) csum[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const bf16x8 ones = as_bf16x8(uint4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u});
  // wgrad: the WP waves that share a row of tiles sum dy for NS of them each; a wave's slot j is
  // its tile j ^ (wp NS), so the slots it sums are the first
  static_assert(KIND != LIN_WGRAD || (WP == 2 && TQ == 2 * NS && (TQ & (TQ - 1)) == 0));
  const int x0 = KIND == LIN_WGRAD ? wp * NS : 0;
  auto slot = [&](int j) { return j ^ x0; };
  Reader<RP, PKS> rp;
  Reader<RQ, QKS> rq;
  rp.init(wp * TP, 0, lane);
  rq.init(wq * TQ, x0, lane);

  // P tiles of a phase: half of them, or a quarter where a half's operands do not fit the registers
  constexpr int G = KIND == LIN_WGRAD && PSRC == SRC_CKPT && TP == 8 ? 4 : 2, H = TP / G;
  auto read_p = [&](bf16x8 (&f)[H], const uint4* ps, int s, int group) {
    const uint32_t o = rp.fresh();
#pragma unroll
    for (int i = 0; i < H; ++i) f[i] = rp.read(ps, o, group * H + i, s);
  };
  auto read_q = [&](bf16x8 (&f)[TQ], const uint4* qs, int s) {
    const uint32_t o = rq.fresh();
#pragma unroll
    for (int j = 0; j < TQ; ++j) f[j] = rq.read(qs, o, j, s);
  };
  auto multiply = [&](const bf16x8 (&fp)[H], const bf16x8 (&fq)[TQ], auto group) {
#pragma unroll
    for (int i = 0; i < H; ++i)
#pragma unroll
      for (int j = 0; j < TQ; ++j) acc[group.value * H + i][j] = mfma_bf16(fp[i], fq[j], acc[group.value * H + i][j]);
    if constexpr (KIND == LIN_WGRAD && group.value == G - 1)
#pragma unroll
      for (int j = 0; j < NS; ++j) csum[j] = mfma_bf16(ones, fq[j], csum[j]);
  };
  constexpr int kConvert = PSRC == SRC_CKPT ? 3 : 0;
  constexpr std::integral_constant<int, 0> none{};
  constexpr int kReadsP = H * (PKS ? 2 : 1), kReadsQ = TQ * (QKS ? 2 : 1);
  // this wave's loads but the newest `stages` stages' have landed and its LDS reads are in
  // registers; then everyone's
  constexpr int kLoads = (RP + RQ) / 8 / NW;
  static_assert(kLoads * (ST - 1) < 64);
  auto sync = [](auto stages) {
    __builtin_amdgcn_s_waitcnt(wait_for(kLoads * stages.value));
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  constexpr std::integral_constant<int, ST - 2> ahead{};
  constexpr bool kDirect = PSRC == SRC_DIRECT && QSRC == SRC_DIRECT;
  // A wave's loads of a stage.  With four stages they are spread over the four phases after the barrier
  // that freed its LDS: issued together, they hold up the products behind them for as long as they
  // take to be accepted (0.3 us a stage with one wave a SIMD).  With two stages they all start right
  // after the barrier, to have the rest of a stage to arrive in: before the products of that
  // phase, or between them in the weight gradient, which fits into its registers that way (eight
  // waves of 256: 199 against 239 us for 14336 x 1280 x 5120).
  constexpr bool kSpread = ST == 4, kBetween = !kSpread && kDirect && KIND == LIN_WGRAD;
  constexpr int kPart = kSpread ? (RP + RQ) / 32 / NW : 0;

  if (steps > 0) {
    bf16x8 pb[2][H], qa[TQ], qb[TQ];   // P operands of this phase and the next; Q's of the two steps
    lp.issue(p0);
    lq.issue(q0);
    lp.template commit<0>(p0);
    lp.template commit<1>(p0);
    lq.template commit<0>(q0);
    lq.template commit<1>(q0);
    if constexpr (ST == 4) {
      lp.issue(p1);
      lq.issue(q1);
      lp.issue(p2);
      lq.issue(q2);
      lp.issue(p3);
      lq.issue(q3);
      sync(std::integral_constant<int, ST - 1>{});
    } else if constexpr (kDirect) {
      lp.issue(p1);
      lq.issue(q1);
      sync(std::integral_constant<int, 1>{});
    } else {
      sync(none);
      lp.issue(p1);
      lq.issue(q1);
    }
    read_q(qa, q0, 0);
    read_p(pb[0], p0, 0, 0);
    // All phases but the last of the stage in (pc, qc); the loads of a later one, whose first part has
    // been issued, go on into (pf, qf); the next stage fills (pn, qn) from registers in the last two.
    auto phases = [&](const uint4* pc, const uint4* qc, uint4* pn, uint4* qn, uint4* pf, uint4* qf, bool next, auto load) {
      auto phase = [&](auto number) {
        constexpr int I = number.value, S = (I + 1) / G;
        constexpr bool kTurn = (I + 1) % G == 0;   // the next phase is the second step's first
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (kTurn) read_q(qb, qc, S);
        read_p(pb[(I + 1) % 2], pc, S, (I + 1) % G);
        if constexpr (load.value && kSpread) {
          lp.template part<I + 1>(pf);
          lq.template part<I + 1>(qf);
        }
        multiply(pb[I % 2], I < G ? qa : qb, std::integral_constant<int, I % G>{});
        if constexpr (I >= 2 * G - 3)
          if (next) {
            lp.template commit<I - (2 * G - 3)>(pn);
            lq.template commit<I - (2 * G - 3)>(qn);
          }
        interleave<kReadsP + (kTurn ? kReadsQ : 0), H * TQ, load.value ? kPart : 0, I >= 2 * G - 3 ? kConvert : 0>();
      };
      phase(std::integral_constant<int, 0>{});
      phase(std::integral_constant<int, 1>{});
      phase(std::integral_constant<int, 2>{});
      if constexpr (G == 4) {
        phase(std::integral_constant<int, 3>{});
        phase(std::integral_constant<int, 4>{});
        phase(std::integral_constant<int, 5>{});
        phase(std::integral_constant<int, 6>{});
      }
      if constexpr (load.value && kSpread) {
        lp.end();
        lq.end();
      }
    };
    constexpr std::integral_constant<int, G - 1> last{};
    constexpr std::true_type loads{};
    constexpr std::false_type no_loads{};
    // Stage t, not the last one, from (pc, qc); (pf, qf): the stage before it, which the loads fill.
    int t = 0;
    auto stage = [&](uint4* pc, uint4* qc, uint4* pn, uint4* qn, uint4* pf, uint4* qf, auto load) {
      phases(pc, qc, pn, qn, pf, qf, true, load);
      sync(ahead);
      if constexpr (kSpread || kBetween) {
        lp.begin();
        lq.begin();
      } else {
        lp.issue(pc);
        lq.issue(qc);
      }
      __builtin_amdgcn_sched_barrier(0);
      read_q(qa, qn, 0);
      read_p(pb[0], pn, 0, 0);
      if constexpr (kSpread) {
        lp.template part<0>(pc);
        lq.template part<0>(qc);
      } else if constexpr (kBetween) {
        lp.all(pc);
        lq.all(qc);
        lp.end();
        lq.end();
      }
      multiply(pb[1], qb, last);
      interleave<kReadsP + kReadsQ, H * TQ, kBetween ? kLoads : kPart>();
      ++t;
    };
    const uint4 *pe = p0, *qe = q0;   // the last stage
    if (steps > 1) {
      // (the first stage has no loads to go on with)
      stage(p0, q0, p1, q1, nullptr, nullptr, no_loads);
      if constexpr (ST == 2) {
        while (t + 2 < steps) {
          stage(p1, q1, p0, q0, p0, q0, loads);
          stage(p0, q0, p1, q1, p1, q1, loads);
        }
        pe = p1;
        qe = q1;
        if (t + 1 < steps) {
          stage(p1, q1, p0, q0, p0, q0, loads);
          pe = p0;
          qe = q0;
        }
      } else {
        while (t + 4 < steps) {
          stage(p1, q1, p2, q2, p0, q0, loads);
          stage(p2, q2, p3, q3, p1, q1, loads);
          stage(p3, q3, p0, q0, p2, q2, loads);
          stage(p0, q0, p1, q1, p3, q3, loads);
        }
        pe = p1;
        qe = q1;
        if (t + 1 < steps) {
          stage(p1, q1, p2, q2, p0, q0, loads);
          pe = p2;
          qe = q2;
          if (t + 1 < steps) {
            stage(p2, q2, p3, q3, p1, q1, loads);
            pe = p3;
            qe = q3;
            if (t + 1 < steps) {
              stage(p3, q3, p0, q0, p2, q2, loads);
              pe = p0;
              qe = q0;
            }
          }
        }
      }
    }
    phases(pe, qe, nullptr, nullptr, nullptr, nullptr, false, no_loads);
    multiply(pb[1], qb, last);
  }
  sync(none);   // no direct load is on its way, and the stages' LDS is free
  // (what follows derives its places anew: kept through the loop, they would take its registers)
  int late = lane;
  asm volatile("" : "+v"(late));
  const int c16 = late & 15, g = late >> 4;

  if constexpr (KIND == LIN_WGRAD) {
    if (g == 0)
#pragma unroll
      for (int j = 0; j < NS; ++j) sums[(wq * TQ + slot(j)) * 16 + c16] = csum[j][0];
    __syncthreads();
  }
  // One row of tiles at a time goes through the wave's own piece of LDS, [16][16 TP] floats (16-byte
  // chunk ch of row r at place ch ^ r), to come back as 8 columns a lane, whole rows side by side.
  constexpr int CPR = 2 * TP, kPiece = 16 * TP * 4;   // 8-column chunks in a row; 16-byte chunks in a piece
  uint4* mine = w < NW / 2 ? p0 + w * kPiece : p1 + (w - NW / 2) * kPiece;
  static_assert(NW / 2 * kPiece <= RP * 8);
  constexpr bool VEC = PSRC != SRC_ANY && QSRC != SRC_ANY;
  constexpr int NI = 16 * CPR / kWave, kRows = kWave / CPR;   // items of a row of tiles, rows between them
  constexpr int NB = KIND == LIN_FWD ? NI : 2;                 // items at a time (as many as fit the registers)
  const int r0 = late / CPR, k = late % CPR, c = ip * RP + wp * TP * 16 + 8 * k;
  TileEpilogue<KIND, SLOPE> te;
  if (VEC) te.init(a, iq * RQ, c);
  // What a row of tiles reads is asked for before the row's accumulators are moved; a pre-activation, which
  // is small, while the row before it is worked on (6% less for 14336 rows of 1280 into 5120, slope
  // and activation, now 258 us).
  constexpr bool kAhead = SLOPE != SLOPE_NONE;
  auto row_of = [&](int j) { return (wq * TQ + slot(j)) * 16 + r0; };   // of the tile: this lane's first item's
  typename TileEpilogue<KIND, SLOPE>::Ask asked[kAhead ? 2 : 1][NI];
  if (kAhead && !part) te.ask(a, row_of(0), kRows, asked[0]);
#pragma unroll
  for (int j = 0; j < TQ; ++j) {
    const int r_tile = row_of(j);
    auto& ask = asked[kAhead ? j % 2 : 0];
    if (VEC && !kAhead && !part) te.ask(a, r_tile, kRows, ask);
#pragma unroll
    for (int i = 0; i < TP; ++i)
      mine[c16 * 4 * TP + ((4 * i + g) ^ c16)] = __builtin_bit_cast(uint4, acc[i][j]);
    if (kAhead && !part && j + 1 < TQ) te.ask(a, row_of(j + 1), kRows, asked[kAhead ? (j + 1) % 2 : 0]);
    auto piece = [&](int it, float (&h)[8]) {
      const int r = it * kRows + r0;
      const f32x4 lo = __builtin_bit_cast(f32x4, mine[r * 4 * TP + ((2 * k) ^ r)]);
      const f32x4 hi = __builtin_bit_cast(f32x4, mine[r * 4 * TP + ((2 * k + 1) ^ r)]);
#pragma unroll
      for (int i = 0; i < 4; ++i) { h[i] = lo[i]; h[4 + i] = hi[i]; }
      return KIND == LIN_WGRAD ? sums[r_tile + it * kRows] : 0.f;
    };
    if (part) {
      // tile [RQ][RP] of split, tile, then its rows' sums
      const size_t at = (size_t)split * rest + xcd_order(nth, rest);
#pragma unroll
      for (int it = 0; it < NI; ++it) {
        float h[8];
        const int rt = r_tile + it * kRows;
        const float qsum = piece(it, h);
        float* to = a.part + (at * RQ + rt) * RP + wp * TP * 16 + 8 * k;
        *(f32x4*)to = f32x4{h[0], h[1], h[2], h[3]};
        *(f32x4*)(to + 4) = f32x4{h[4], h[5], h[6], h[7]};
        if (KIND == LIN_WGRAD && wp == 0 && k == 0) a.part_sum[at * RQ + rt] = qsum;
      }
    } else if constexpr (VEC) {
      auto group = [&](auto first) {
        float h[NB][8], qsum[NB];
#pragma unroll
        for (int it = 0; it < NB; ++it) qsum[it] = piece(first.value + it, h[it]);
        te.template rows<first.value>(a, r_tile + first.value * kRows, kRows, h, qsum, ask);
      };
      group(std::integral_constant<int, 0>{});
      if constexpr (NI > NB) group(std::integral_constant<int, NB>{});
      if constexpr (NI > 2 * NB) group(std::integral_constant<int, 2 * NB>{});
      if constexpr (NI > 3 * NB) group(std::integral_constant<int, 3 * NB>{});
      static_assert(NI <= 4 * NB);
    } else {
#pragma unroll 1
      for (int it = 0; it < NI; ++it) {
        float h[8];
        const float qsum = piece(it, h);
        epilogue<KIND>(a, iq * RQ + r_tile + it * kRows, c, h, qsum);
      }
    }
  }
  if constexpr (VEC && KIND == LIN_WGRAD) {   // (the other epilogue writes it with the row)
    const int q = iq * RQ + threadIdx.x;
    if (!part && ip == 0 && a.dbias && threadIdx.x < RQ && q < a.Q.extent)
      a.dbias[q] = a.accumulate ? a.dbias[q] + sums[threadIdx.x] : sums[threadIdx.x];
  }
}

// The tiles that were computed in S parts: joined in order, then the epilogue.  A wave takes 512
// columns of the tile's rows (TILE of them to a row).
template <int KIND, int TILE>
__global__ void __launch_bounds__(256) linear_join_kernel(LinArgs a) {
  const int rest = a.tiles_p * a.tiles_q - a.whole;
  constexpr int kRows = 512 / TILE, kUnits = TILE / kRows;   // rows of a wave, waves of a tile
  const int u = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + threadIdx.x / kWave);
  const int t = u / kUnits, lane = threadIdx.x % kWave;
  if (t >= rest) return;
  const int r = (u % kUnits) * kRows + lane / (TILE / 8), k = lane % (TILE / 8) * 8;
  int ip, iq;
  tile_of(a.whole + t, a.tiles_p, a.tiles_q, ip, iq);
  const int q = iq * TILE + r, c = ip * TILE + k;
  float h[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  float qsum = 0.f;
#pragma unroll 4
  for (int s = 0; s < a.S; ++s) {
    const size_t at = ((size_t)s * rest + t) * TILE + r;
    const f32x4 lo = *(const f32x4*)(a.part + at * TILE + k), hi = *(const f32x4*)(a.part + at * TILE + k + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      h[i] += lo[i];
      h[4 + i] += hi[i];
    }
    if (KIND == LIN_WGRAD) qsum += a.part_sum[at];
  }
  epilogue<KIND>(a, q, c, h, qsum);
}

// Forward product of at most 16 RT rows (single tokens, a decoding batch): the weight is read once and
// that is the floor, so it goes from memory straight to registers, many loads at a time, with no LDS
// and no second launch.  A workgroup owns PC columns; its eight waves share the reduction and add up
// in LDS, in order (sixteen were no faster: 8.4 against 8.1 us for 1280 x 5120).
template <int RT, int PC>
__global__ void __launch_bounds__(kFewWaves* kWave) linear_few_kernel(LinArgs a) {
  constexpr int U = kFewSteps, NW = kFewWaves;
  __shared__ f32x4 part[NW][RT * 16][PC / 4];
  const int lane = threadIdx.x % kWave, w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int c16 = lane & 15, g = lane >> 4, p0 = blockIdx.x * PC;
  constexpr int kItems = RT * 16 * PC / 8;
  const int t = threadIdx.x, q = t / (PC / 8), c = p0 + t % (PC / 8) * 8;
  Extra e{};
  if (t < kItems) e = request(a, q, c);
  const int all = (a.K + 31) / 32, each = (all + NW - 1) / NW;
  const int beg = w * each, end = min(all, beg + each);
  const uint16_t* pw = a.P.p + (size_t)min(p0 + c16 % PC, a.P.extent - 1) * a.P.ld + 8 * g;
  const uint16_t* px[RT];
  f32x4 acc[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    px[r] = a.Q.p + (size_t)min(16 * r + c16, a.Q.extent - 1) * a.Q.ld + 8 * g;
    acc[r] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  for (int s = beg; s < end; s += U) {
    u32x4 fw[U], fx[RT][U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      fw[u] = u32x4{0, 0, 0, 0};
#pragma unroll
      for (int r = 0; r < RT; ++r) fx[r][u] = u32x4{0, 0, 0, 0};
      if (s + u < end && 32 * (s + u) + 8 * g < a.K) {
        fw[u] = *(const u32x4*)(pw + 32 * (s + u));
#pragma unroll
        for (int r = 0; r < RT; ++r) fx[r][u] = *(const u32x4*)(px[r] + 32 * (s + u));
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int r = 0; r < RT; ++r)
        acc[r] = mfma_bf16(__builtin_bit_cast(bf16x8, fw[u]), __builtin_bit_cast(bf16x8, fx[r][u]), acc[r]);
  }
  if (4 * g < PC)
#pragma unroll
    for (int r = 0; r < RT; ++r) part[w][16 * r + c16][g] = acc[r];
  __syncthreads();
  if (t < kItems) {
    float h[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < NW; ++v) {
      const f32x4 lo = part[v][q][t % (PC / 8) * 2], hi = part[v][q][t % (PC / 8) * 2 + 1];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        h[i] += lo[i];
        h[4 + i] += hi[i];
      }
    }
    epilogue<LIN_FWD, true>(a, q, c, h, 0.f, e);
  }
}

template <int KIND, bool PKS, int PSRC, bool QKS, int QSRC, int SLOPE = SLOPE_NONE>
void launch_one(const LinArgs& a, const Plan& r, hipStream_t st) {
  const unsigned rest = a.tiles_p * a.tiles_q - a.whole, grid = a.whole + rest * a.S;
  if (r.tile == 256) {
    if constexpr (PSRC != SRC_ANY && QSRC == SRC_DIRECT) {
      linear_kernel<KIND, 2, 4, 8, 4, 2, PKS, PSRC, QKS, QSRC, SLOPE><<<grid, 512, 0, st>>>(a);
      if (rest) linear_join_kernel<KIND, 256><<<rest * 32, 256, 0, st>>>(a);
    }
    return;
  }
  if constexpr (PSRC == SRC_DIRECT && QSRC == SRC_DIRECT) {
    if (r.deep) linear_kernel<KIND, 2, 2, 4, 4, 4, PKS, PSRC, QKS, QSRC, SLOPE><<<grid, 256, 0, st>>>(a);
    else linear_kernel<KIND, 2, 2, 4, 4, 2, PKS, PSRC, QKS, QSRC, SLOPE><<<grid, 256, 0, st>>>(a);
  } else {
    linear_kernel<KIND, 2, 2, 4, 4, 2, PKS, PSRC, QKS, QSRC, SLOPE><<<grid, 256, 0, st>>>(a);
  }
  if (rest) linear_join_kernel<KIND, 128><<<rest * 8, 256, 0, st>>>(a);
}

bool whole(const DMat& m) { return !m.p || m.vec; }
bool whole(const DVec& v, int cols) { return !v.p || (v.vec && cols % 8 == 0); }

// Direct loads move 8 elements at a time: along the reduction (KC) or the output (KS).
bool direct_ok(const LinOp& o, int contiguous) {
  return (uintptr_t)o.p % 16 == 0 && o.ld % 8 == 0 && contiguous % 8 == 0;
}

}  // namespace

template <int RT, int PC>
void launch_few(const LinArgs& a, const FewPlan& f, hipStream_t st) {
  linear_few_kernel<RT, PC><<<f.grid, kFewWaves * kWave, 0, st>>>(a);
}

size_t lin_part_floats(int kind, int P, int Q, int K) { return plan_floats(kind == LIN_WGRAD, P, Q, K); }

void launch_linear(int kind, LinArgs a, hipStream_t st) {
  const bool pk = kind == LIN_FWD, qk = kind != LIN_WGRAD;   // contiguous along the reduction
  const bool q_direct = direct_ok(a.Q, qk ? a.K : a.Q.extent);
  // (the kernels of direct operands move whole vectors in their epilogues too)
  const int cols = a.P.extent;
  const bool direct = q_direct && (!a.P.p || direct_ok(a.P, pk ? a.K : cols)) && whole(a.out) && whole(a.res) &&
                      whole(a.pre) && whole(a.act_out) && whole(a.bias, cols) && whole(a.gain, cols) && whole(a.shift, cols);
  const Plan r = plan(a.P.extent, a.Q.extent, a.K, direct, !a.P.p);
  a.tiles_p = r.tiles_p; a.tiles_q = r.tiles_q; a.whole = r.whole; a.S = r.S; a.steps = r.steps;
  a.part_sum = r.S > 1 ? a.part + (size_t)r.S * (r.tiles_p * r.tiles_q - r.whole) * r.tile * r.tile : nullptr;
  if (kind == LIN_FWD && direct && !a.ck.q && a.Q.extent <= kFewRows) {
    // (a checkpoint's groups of 32 columns do not fit the workgroups of few rows)
    const FewPlan f = few_plan(a.P.extent, a.Q.extent, a.K);
    if (few_wins(f, r, a.P.extent, a.K)) {
      if (a.Q.extent <= 16) f.narrow ? launch_few<1, 8>(a, f, st) : launch_few<1, 16>(a, f, st);
      else f.narrow ? launch_few<2, 8>(a, f, st) : launch_few<2, 16>(a, f, st);
      return;
    }
  }
  if (kind == LIN_FWD) {
    if (direct) launch_one<LIN_FWD, false, SRC_DIRECT, false, SRC_DIRECT>(a, r, st);
    else launch_one<LIN_FWD, false, SRC_ANY, false, SRC_ANY>(a, r, st);
  } else if (kind == LIN_DGRAD) {
    if (direct && a.gelu && a.ck.q) launch_one<LIN_DGRAD, true, SRC_DIRECT, false, SRC_DIRECT, SLOPE_CKPT>(a, r, st);
    else if (direct && a.gelu) launch_one<LIN_DGRAD, true, SRC_DIRECT, false, SRC_DIRECT, SLOPE_BF16>(a, r, st);
    else if (direct) launch_one<LIN_DGRAD, true, SRC_DIRECT, false, SRC_DIRECT>(a, r, st);
    else launch_one<LIN_DGRAD, true, SRC_ANY, false, SRC_ANY>(a, r, st);
  } else if (!a.P.p) {
    if (direct) launch_one<LIN_WGRAD, true, SRC_CKPT, true, SRC_DIRECT>(a, r, st);
    else launch_one<LIN_WGRAD, true, SRC_CKPT, true, SRC_ANY>(a, r, st);
  } else {
    if (direct) launch_one<LIN_WGRAD, true, SRC_DIRECT, true, SRC_DIRECT>(a, r, st);
    else launch_one<LIN_WGRAD, true, SRC_ANY, true, SRC_ANY>(a, r, st);
  }
}

}  // namespace ad
