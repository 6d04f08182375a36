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
// consecutive columns of one output row, so the epilogue moves 16 bytes of float32 at a time, and
// two neighbouring tiles hold a whole 8-bit checkpoint group of 32 columns.
//
// LDS bank conflicts.  KC rows are 128 bytes: the 16-byte piece c of row r sits at place
// c ^ (r / 2 % 8), so the 16 rows that are read together cover every bank.  KS rows are 256 or
// 512 bytes: 32-byte pair t of row r sits at place t ^ (r % 4 + 4 (r / 8 % 2)) (low three bits),
// so the eight rows that 32 lanes read together do.  The direct loads store 1 KB in lane order;
// the permutation is made by the lanes' source addresses.
#include <algorithm>

#include "train.h"

namespace ad {

namespace {

constexpr int kBK = 64;   // reduction elements of one LDS stage

// 16 bytes that pieces past the end of the reduction read
__device__ const uint4 g_zero16 = {0, 0, 0, 0};

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

enum Src : int { SRC_DIRECT = 0, SRC_ANY = 1, SRC_CKPT = 2 };

__device__ __forceinline__ int ks_swz(int r) { return (r & 3) | ((r >> 1) & 4); }

// The part of one operand's stage that a wave moves: R rows (KC) or columns (KS) x 64 of r in
// pieces of 1 KB, NW waves.  Direct: memory to LDS; otherwise through registers (any
// alignment, element by element; or a checkpoint's 8-bit values, dequantised on the way).
template <int R, int NW, bool KS, int SRC>
struct Loader {
  static constexpr int N = R / 8 / NW;   // pieces a wave
  static constexpr int RB = R / 8;       // 16-byte pieces in a KS row
  LinOp o;
  int r0, K, k0, w, lane;
  const uint16_t* base;   // of the stage's first element
  uint32_t off[N];        // bytes
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
      base = KS ? o.p + (size_t)k0 * o.ld + r0 : o.p + (size_t)r0 * o.ld + k0;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        int row, r;
        place(j, row, r);
        // rows and columns past the matrix read its last ones (their results are not stored)
        off[j] = KS ? 2u * ((uint32_t)r * (uint32_t)o.ld + (uint32_t)min(row, o.extent - 8 - r0))
                    : 2u * ((uint32_t)min(row, o.extent - 1 - r0) * (uint32_t)o.ld + (uint32_t)r);
      }
    }
  }

  // stage at k0: into `lds` (direct), or into registers
  __device__ __forceinline__ void issue(uint4* lds) {
    if constexpr (SRC == SRC_DIRECT) {
      if (k0 + kBK <= K) {
#pragma unroll
        for (int j = 0; j < N; ++j) dma16((const char*)base + off[j], lds + (w * N + j) * 64);
      } else {
#pragma unroll
        for (int j = 0; j < N; ++j) {
          int row, r;
          place(j, row, r);
          const void* src = k0 + r < K ? (const void*)((const char*)base + off[j]) : (const void*)&g_zero16;
          dma16(src, lds + (w * N + j) * 64);
        }
      }
      base += KS ? (size_t)kBK * o.ld : (size_t)kBK;
    } else if constexpr (SRC == SRC_ANY) {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        int row, r;
        place(j, row, r);
        uint32_t e[8];
        const int a = r0 + row, k = k0 + r;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if constexpr (KS) e[i] = k < K && a + i < o.extent ? o.p[(size_t)k * o.ld + a + i] : 0;
          else e[i] = a < o.extent && k + i < K ? o.p[(size_t)a * o.ld + k + i] : 0;
        }
        reg[j] = uint4{e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16};
      }
    } else {
#pragma unroll
      for (int j = 0; j < N / 2; ++j) {
        int row, r;
        place_ck(j, row, r);
        const int c = r0 + row, k = k0 + r;
        reg[j] = uint4{0, 0, 0, 0};
        sc[j] = 1;
        if (k < K && c < o.ck.ld) {
          reg[j] = *(const uint4*)(o.ck.q + (size_t)k * o.ck.ld + c);
          sc[j] = o.ck.scale[(size_t)k * (o.ck.ld / kCkptGroup) + c / kCkptGroup];
        }
      }
    }
    k0 += kBK;
  }

  // registers into LDS
  __device__ __forceinline__ void commit(uint4* lds) {
    if constexpr (SRC == SRC_ANY) {
#pragma unroll
      for (int j = 0; j < N; ++j) lds[(w * N + j) * 64 + lane] = reg[j];
    } else if constexpr (SRC == SRC_CKPT) {
#pragma unroll
      for (int j = 0; j < N / 2; ++j) {
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

// The matrix instruction's operand of 16-row (or column) tile t, 32-wide step s of a stage.
template <int R, bool KS>
__device__ __forceinline__ bf16x8 fragment(const uint4* lds, int t, int s, int lane) {
  const int c16 = lane & 15, g = lane >> 4;
  if constexpr (KS) {
    const int i = c16 >> 2, u = (t & ~7) | ((t & 7) ^ (i | ((g & 1) << 2)));
    const uint16_t* p = (const uint16_t*)lds + (32 * s + 8 * g + i) * R + u * 16 + (c16 & 3) * 4;
    typedef const __attribute__((address_space(3))) s16x4* lp;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(lp)p);
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(lp)(p + 4 * R));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
  } else {
    return as_bf16x8(lds[(t * 16 + c16) * 8 + ((4 * s + g) ^ (c16 >> 1))]);
  }
}

// Largest of a value over the four 16-lane rows of a wave, as bits.
__device__ __forceinline__ uint32_t rows4_max_bits(uint32_t v) {
  const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max((uint32_t)a[0], (uint32_t)a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return max((uint32_t)b[0], (uint32_t)b[1]);
}

__device__ __forceinline__ f32x4 vec_at(const DVec& v, int c, int cols) {
  f32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = c + i < cols ? ld_vec(v, c + i) : 0.f;
  return r;
}

// Output row q, columns p .. p + 3 (h[0]) and p + 16 .. p + 19 (h[1]), p = 32 * n + 4 * (lane
// / 16): the four lanes lane % 16 + 16 * {0 .. 3} hold one group of 32 columns.  Every lane of
// the wave calls this.  qsum: wgrad's sum of dy for row q.
template <int KIND>
__device__ __forceinline__ void epilogue(const LinArgs& a, int q, int p, f32x4 (&h)[2], float qsum) {
  const int Pn = a.P.extent;
  const bool row = q < a.Q.extent;
  if constexpr (KIND == LIN_FWD) {
    if (a.bias.p)
#pragma unroll
      for (int u = 0; u < 2; ++u) h[u] += vec_at(a.bias, p + 16 * u, Pn);
    if (a.pre.p && row)
#pragma unroll
      for (int u = 0; u < 2; ++u) store4(a.pre, q, p + 16 * u, Pn, h[u]);
    if (a.ck.q) {
      uint32_t m = 0;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (p + 16 * u + i >= Pn) h[u][i] = 0.f;   // (padding is written as 0)
          m = max(m, abs_bits(h[u][i]));
        }
      const uint32_t s = ckpt_scale(rows4_max_bits(m));
      const float inv = ckpt_inv(s);
      if (row && p < a.ck.ld) {
        int8_t* to = a.ck.q + (size_t)q * a.ck.ld + p;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const uint32_t b = pack_bytes(ckpt_round(h[u][0], inv), ckpt_round(h[u][1], inv),
                                        ckpt_round(h[u][2], inv), ckpt_round(h[u][3], inv));
          *(uint32_t*)(to + 16 * u) = s == 255u ? 0u : b;
        }
        if (p % kCkptGroup == 0) a.ck.scale[(size_t)q * (a.ck.ld / kCkptGroup) + p / kCkptGroup] = (uint8_t)s;
      }
    }
    if (!row) return;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      f32x4 y = h[u];
      if (a.gelu)
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = gelu_value(y[i]);
      if (a.res.p) y += load4(a.res, q, p + 16 * u, Pn);
      store4(a.out, q, p + 16 * u, Pn, y);
    }
  } else if constexpr (KIND == LIN_DGRAD) {
    if (!row) return;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int c = p + 16 * u;
      f32x4 v = h[u];
      if (a.gelu) {
        f32x4 x;
        if (a.ck.q) {
          uint32_t w = 0, s = 1;
          if (c < a.ck.ld) {
            w = *(const uint32_t*)(a.ck.q + (size_t)q * a.ck.ld + c);
            s = a.ck.scale[(size_t)q * (a.ck.ld / kCkptGroup) + c / kCkptGroup];
          }
          float t[4];
          ckpt_value4(w, ckpt_two(s), t);
          x = f32x4{t[0], t[1], t[2], t[3]};
        } else {
          x = load4(a.pre, q, c, Pn);
        }
        if (a.act_out.p) {
          f32x4 y;
#pragma unroll
          for (int i = 0; i < 4; ++i) y[i] = gelu_value(x[i]);
          store4(a.act_out, q, c, Pn, y);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] *= gelu_slope(x[i]);
      }
      store4(a.out, q, c, Pn, v);
    }
  } else {
    if (!row) return;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int c = p + 16 * u;
      f32x4 v = h[u];
      if (a.gain.p) v = v * vec_at(a.gain, c, Pn) + vec_at(a.shift, c, Pn) * qsum;
      if (a.accumulate) v += load4(a.out, q, c, Pn);
      store4(a.out, q, c, Pn, v);
    }
    if (a.dbias && p == 0) a.dbias[q] = a.accumulate ? a.dbias[q] + qsum : qsum;
  }
}

// Tile of workgroup id: workgroups are dealt round-robin over the 8 XCDs, so each XCD takes a
// contiguous range of tiles, ordered in bands of 8 row tiles (column by column inside a
// band), and its workgroups share both operands through its L2.
__device__ __forceinline__ void tile_of(int id, int tp, int tq, int& ip, int& iq) {
  const int T = tp * tq, x = id % 8, l = id / 8;
  const int t = x * (T / 8) + min(x, T % 8) + l;
  const int band = t / (8 * tp), rest = t % (8 * tp), h = min(8, tq - band * 8);
  iq = band * 8 + rest % h;
  ip = rest / h;
}

// WP x WQ waves of TP x TQ 16 x 16 tiles.  Two LDS stages: the next one fills while this one is
// multiplied; one barrier a stage.
template <int KIND, int WP, int WQ, int TP, int TQ, bool PKS, int PSRC, bool QKS, int QSRC>
__global__ void __launch_bounds__(WP* WQ* kWave) linear_kernel(LinArgs a) {
  constexpr int NW = WP * WQ, RP = WP * TP * 16, RQ = WQ * TQ * 16, NS = TQ / WP;
  static_assert(TP % 2 == 0 && TQ % WP == 0);
  __shared__ uint4 p0[RP * 8], p1[RP * 8], q0[RQ * 8], q1[RQ * 8];
  __shared__ float sums[KIND == LIN_WGRAD ? RQ : 1];
  const int lane = threadIdx.x % kWave, w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int wp = w % WP, wq = w / WP, c16 = lane & 15, g = lane >> 4;
  const int tiles = a.tiles_p * a.tiles_q, split = blockIdx.x / tiles;
  int ip, iq;
  tile_of(blockIdx.x % tiles, a.tiles_p, a.tiles_q, ip, iq);
  const int kbeg = split * a.steps * kBK, kend = min(a.K, kbeg + a.steps * kBK);
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
  // its tile (j + wp NS) % TQ, so the slots it sums are the first
  auto slot = [&](int j) { return KIND == LIN_WGRAD ? (j + wp * NS) % TQ : j; };

  auto step = [&](const uint4* ps, const uint4* qs, uint4* pn, uint4* qn, bool more) {
    // this wave's loads of the stage have landed, then everyone's; the other stage is free
    __builtin_amdgcn_s_waitcnt(0x0070);   // vmcnt 0, lgkmcnt 0
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (more) {
      lp.issue(pn);
      lq.issue(qn);
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      bf16x8 fp[TP], fq[TQ];
#pragma unroll
      for (int i = 0; i < TP; ++i) fp[i] = fragment<RP, PKS>(ps, wp * TP + i, s, lane);
#pragma unroll
      for (int j = 0; j < TQ; ++j) fq[j] = fragment<RQ, QKS>(qs, wq * TQ + slot(j), s, lane);
#pragma unroll
      for (int i = 0; i < TP; ++i)
#pragma unroll
        for (int j = 0; j < TQ; ++j) acc[i][j] = mfma_bf16(fp[i], fq[j], acc[i][j]);
      if constexpr (KIND == LIN_WGRAD)
#pragma unroll
        for (int j = 0; j < NS; ++j) csum[j] = mfma_bf16(ones, fq[j], csum[j]);
    }
    if (more) {
      lp.commit(pn);
      lq.commit(qn);
    }
  };

  if (steps > 0) {
    lp.issue(p0);
    lq.issue(q0);
    lp.commit(p0);
    lq.commit(q0);
    for (int t = 0; t < steps; t += 2) {
      step(p0, q0, p1, q1, t + 1 < steps);
      if (t + 1 < steps) step(p1, q1, p0, q0, t + 2 < steps);
    }
  }

  if constexpr (KIND == LIN_WGRAD) {
    if (g == 0)
#pragma unroll
      for (int j = 0; j < NS; ++j) sums[(wq * TQ + slot(j)) * 16 + c16] = csum[j][0];
    __syncthreads();
  }
  const int pw = ip * RP + wp * TP * 16 + 4 * g, qw = iq * RQ + wq * TQ * 16 + c16;
#pragma unroll
  for (int j = 0; j < TQ; ++j) {
    const int q = qw + slot(j) * 16;
    const float qsum = KIND == LIN_WGRAD ? sums[(wq * TQ + slot(j)) * 16 + c16] : 0.f;
    if (a.S > 1) {
      if (q < a.Q.extent) {
#pragma unroll
        for (int i = 0; i < TP; ++i)
          if (pw + 16 * i < a.ldp)
            *(f32x4*)(a.part + ((size_t)split * a.Q.extent + q) * a.ldp + pw + 16 * i) = acc[i][j];
        if (KIND == LIN_WGRAD && ip == 0 && wp == 0 && g == 0) a.part_sum[(size_t)split * a.Q.extent + q] = qsum;
      }
      continue;
    }
#pragma unroll
    for (int i = 0; i < TP; i += 2) {
      f32x4 h[2] = {acc[i][j], acc[i + 1][j]};
      epilogue<KIND>(a, q, pw + 16 * i, h, qsum);
    }
  }
}

// Columns that the epilogue writes: a checkpoint's padding too.
__host__ __device__ inline int join_cols(const LinArgs& a, int kind) {
  return kind == LIN_FWD && a.ck.q ? a.ck.ld : a.P.extent;
}

// The partial products of a split reduction, joined in split order, and the epilogue: a wave
// takes 16 rows x 32 columns in the lane order of the matrix instruction's output.
template <int KIND>
__global__ void __launch_bounds__(256) linear_join_kernel(LinArgs a) {
  const int lane = threadIdx.x % kWave, c16 = lane & 15, g = lane >> 4;
  const unsigned cols = (join_cols(a, KIND) + 31) / 32, rows = (a.Q.extent + 15) / 16;
  const unsigned u = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + threadIdx.x / kWave);
  if (u >= cols * rows) return;
  const int q = (int)(u / cols) * 16 + c16, p = (int)(u % cols) * 32 + 4 * g;
  f32x4 h[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
  float qsum = 0.f;
  if (q < a.Q.extent) {
    for (int s = 0; s < a.S; ++s) {
      const float* from = a.part + ((size_t)s * a.Q.extent + q) * a.ldp + p;
      if (p < a.ldp) h[0] += *(const f32x4*)from;
      if (p + 16 < a.ldp) h[1] += *(const f32x4*)(from + 16);
      if (KIND == LIN_WGRAD) qsum += a.part_sum[(size_t)s * a.Q.extent + q];
    }
  }
  epilogue<KIND>(a, q, p, h, qsum);
}

struct Plan {
  int S, steps, tiles_p, tiles_q;
};
constexpr int kCUs = 256;

// (sizes only: the workspace is asked for before the operands' alignment is known)
Plan plan(int P, int Q, int K) {
  Plan r;
  r.tiles_p = (P + 127) / 128;
  r.tiles_q = (Q + 127) / 128;
  const int64_t tiles = (int64_t)r.tiles_p * r.tiles_q;
  const int steps = (K + kBK - 1) / kBK;
  // few tiles: the reduction is split until about every CU has a workgroup, in ranges of at
  // least four steps
  r.S = tiles >= kCUs ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>(kCUs / tiles, steps / 4));
  r.steps = (steps + r.S - 1) / r.S;
  r.S = r.steps ? (steps + r.steps - 1) / r.steps : 1;
  return r;
}

template <int KIND, bool PKS, int PSRC, bool QKS, int QSRC>
void launch_one(const LinArgs& a, hipStream_t st) {
  linear_kernel<KIND, 2, 2, 4, 4, PKS, PSRC, QKS, QSRC><<<a.tiles_p * a.tiles_q * a.S, 256, 0, st>>>(a);
  if (a.S > 1) {
    const unsigned units = (unsigned)((join_cols(a, KIND) + 31) / 32) * (unsigned)((a.Q.extent + 15) / 16);
    linear_join_kernel<KIND><<<(units + 3) / 4, 256, 0, st>>>(a);
  }
}

// Direct loads move 8 elements at a time: along the reduction (KC) or the output (KS).
bool direct_ok(const LinOp& o, int contiguous) {
  return (uintptr_t)o.p % 16 == 0 && o.ld % 8 == 0 && contiguous % 8 == 0;
}

}  // namespace

size_t lin_part_floats(int kind, int P, int Q, int K) {
  const Plan r = plan(P, Q, K);
  if (r.S <= 1) return 0;
  const size_t ldp = (P + 3) / 4 * 4;
  return (size_t)r.S * Q * ldp + (kind == LIN_WGRAD ? (size_t)r.S * Q : 0);
}

void launch_linear(int kind, LinArgs a, hipStream_t st) {
  const Plan r = plan(a.P.extent, a.Q.extent, a.K);
  a.S = r.S; a.steps = r.steps; a.tiles_p = r.tiles_p; a.tiles_q = r.tiles_q;
  a.ldp = (a.P.extent + 3) / 4 * 4;
  a.part_sum = a.part ? a.part + (size_t)a.S * a.Q.extent * a.ldp : nullptr;
  if (kind == LIN_FWD) {
    if (direct_ok(a.P, a.K) && direct_ok(a.Q, a.K)) launch_one<LIN_FWD, false, SRC_DIRECT, false, SRC_DIRECT>(a, st);
    else launch_one<LIN_FWD, false, SRC_ANY, false, SRC_ANY>(a, st);
  } else if (kind == LIN_DGRAD) {
    if (direct_ok(a.P, a.P.extent) && direct_ok(a.Q, a.K)) launch_one<LIN_DGRAD, true, SRC_DIRECT, false, SRC_DIRECT>(a, st);
    else launch_one<LIN_DGRAD, true, SRC_ANY, false, SRC_ANY>(a, st);
  } else if (!a.P.p) {
    if (direct_ok(a.Q, a.Q.extent)) launch_one<LIN_WGRAD, true, SRC_CKPT, true, SRC_DIRECT>(a, st);
    else launch_one<LIN_WGRAD, true, SRC_CKPT, true, SRC_ANY>(a, st);
  } else {
    if (direct_ok(a.P, a.P.extent) && direct_ok(a.Q, a.Q.extent)) launch_one<LIN_WGRAD, true, SRC_DIRECT, true, SRC_DIRECT>(a, st);
    else launch_one<LIN_WGRAD, true, SRC_ANY, true, SRC_ANY>(a, st);
  }
}

}  // namespace ad
