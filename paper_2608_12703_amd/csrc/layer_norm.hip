// LayerNorm forward and backward, and 8-bit activation checkpoints.
//
// All of these stream rows once; the floor is HBM traffic.  A lane holds 8 consecutive columns
// at a time (16 bytes of bf16), a wave 512, so rows of up to 2048 columns live in one wave's
// registers (J = 1 .. 4 pieces a lane) and need no LDS for their sums; wider rows, up to 8192
// columns, are spread over the four waves of a workgroup.
//
// Measured against a large copy's 4.9 TB/s: LayerNorm of 14336 x 1280 float32 rows into bf16 and
// the checkpoint 35 us (3.7 TB/s), its backward pass over 13331 such rows kept whole 60 us (4.6),
// packing 14336 x 5120 bf16 49 us (4.5), reading them back 34 us (6.5: 76 MB that were written just
// before, most likely from the last-level cache).  Loads must be whole
// vectors in one block each: as selects of a load and a zero they became eight loads of 4 bytes
// with a branch each, and the same LayerNorm took 52 us.
#include <algorithm>

#include "train.h"
#include "top2.h"

namespace ad {

namespace {

constexpr float kEps = 1e-5f;

// Sum over the wave: rotations inside 16-lane rows, then the row swaps (no LDS round trip).
__device__ __forceinline__ float wave_total(float v) {
  v += __int_as_float(ror16<8>(__float_as_int(v)));
  v += __int_as_float(ror16<4>(__float_as_int(v)));
  v += __int_as_float(ror16<2>(__float_as_int(v)));
  v += __int_as_float(ror16<1>(__float_as_int(v)));
  return rows4_sum(v);
}

// Sums over the lanes that share a row: the wave, or the workgroup's four waves.
template <int W, int N>
__device__ __forceinline__ void row_totals(float (&v)[N], float (*red)[4]) {
#pragma unroll
  for (int n = 0; n < N; ++n) v[n] = wave_total(v[n]);
  if constexpr (W == 4) {
    __syncthreads();
    if (threadIdx.x % kWave == 0)
#pragma unroll
      for (int n = 0; n < N; ++n) red[n][threadIdx.x / kWave] = v[n];
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = (red[n][0] + red[n][1]) + (red[n][2] + red[n][3]);
  }
}
template <int W>
__device__ __forceinline__ float row_total(float v, float (*red)[4]) {
  float one[1] = {v};
  row_totals<W>(one, red);
  return one[0];
}

// W: waves per row (1 or 4), VEC: every matrix and parameter allows whole vectors.  The statistics
// are two passes over the registers: the mean m, then the sum of the deviations from it and that of
// their squares.  m is off by its roundings, which are large beside the deviations where the mean is
// (alone, it made a row of 1e5 come out as 1 instead of 0).  The deviations' own mean c is that error:
// mean = m + c, var = sum (x - m)^2 / n - c^2, with c^2 as small as the roundings.  Columns past the
// row's end hold 0 throughout: with whole vectors a lane's piece is all in or all out, so it deviates
// from 0 instead of the mean.  A row a wave: two at a time had more loads in flight but fewer waves,
// and took 6% longer for 14336 x 1280 float32 into bf16 (26.7 us; 25.9 without c).
// (The bounds keep J = 3 at five waves a SIMD, and its element paths at four: 38 in place of 42 us.)
template <int J, int W, bool VEC>
__global__ void __launch_bounds__(256, J == 3 ? (VEC ? 5 : 4) : 1) ln_fwd_kernel(LnFwdArgs a) {
  // (contracted, m = total * inv_n is rounded in some columns' deviations and not in others')
#pragma clang fp contract(off)
  __shared__ float red[2][4];
  const int t = W == 1 ? threadIdx.x % kWave : threadIdx.x;
  const int first = W == 1 ? blockIdx.x * 4 + threadIdx.x / kWave : blockIdx.x;
  const int stride = W == 1 ? gridDim.x * 4 : gridDim.x;
  constexpr int kStep = 8 * kWave * W;
  const float inv_n = 1.0f / (float)a.cols;
  // (with W == 4 every wave of the workgroup has the same rows, so the barriers are met by all)
  for (int row = first; row < a.rows; row += stride) {
    float x[J][8], s = 0.f;
#pragma unroll
    for (int j = 0; j < J; ++j) load8<VEC>(a.x, row, 8 * t + j * kStep, a.cols, x[j]);
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) s += x[j][i];
    const float m0 = row_total<W>(s, red) * inv_n;
    float d[2] = {0.f, 0.f};   // the deviations' sum, and their squares'
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const float m = 8 * t + j * kStep < a.cols ? m0 : 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[j][i] = VEC || 8 * t + j * kStep + i < a.cols ? x[j][i] - m : 0.f;
        d[0] += x[j][i];
        d[1] = fmaf(x[j][i], x[j][i], d[1]);
      }
    }
    row_totals<W>(d, red);
    const float c0 = d[0] * inv_n, mean = m0 + c0;
    const float var = fmaf(-c0, c0, d[1] * inv_n);
    const float rstd = 1.0f / sqrtf((var < 0.f ? 0.f : var) + kEps);   // (NaN stays NaN)
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int c = 8 * t + j * kStep;
      float g[8], b[8], y[8];
      load_vec8<VEC>(a.gain, c, a.cols, g);
      load_vec8<VEC>(a.bias, c, a.cols, b);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[j][i] = (x[j][i] - c0) * rstd;
        y[i] = fmaf(x[j][i], g[i], b[i]);
      }
      if (VEC ? c >= a.cols : c + 8 > a.cols)   // the checkpoint's padding is 0
#pragma unroll
        for (int i = 0; i < 8; ++i) x[j][i] = c + i < a.cols ? x[j][i] : 0.f;
      store8<VEC>(a.y, row, c, a.cols, y);
      if (a.xhat.q) ckpt_store8(a.xhat, row, c, x[j]);
    }
    if (t == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
  }
}

// A workgroup walks rows g, g + G, ... and keeps the sums for dgain and dbias of its columns
// in registers; they leave once, as one of G partial rows.  The order of the sums depends
// on the number of rows and columns only.
template <int J, int W, bool VEC>
__global__ void __launch_bounds__(256) ln_bwd_kernel(LnBwdArgs a) {
  __shared__ float red[1][4];
  constexpr int kStep = 8 * kWave * W;
  const int w = threadIdx.x / kWave, t = W == 1 ? threadIdx.x % kWave : threadIdx.x;
  const int first = W == 1 ? blockIdx.x * 4 + w : blockIdx.x, stride = W == 1 ? gridDim.x * 4 : gridDim.x;
  float g[J][8], dg[J][8], db[J][8];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    load_vec8<VEC>(a.gain, 8 * t + j * kStep, a.cols, g[j]);
#pragma unroll
    for (int i = 0; i < 8; ++i) dg[j][i] = db[j][i] = 0.f;
  }
  const float inv_n = 1.0f / (float)a.cols;
  for (int row = first; row < a.rows; row += stride) {
    float xh[J][8], dy[J][8];
#pragma unroll
    for (int j = 0; j < J; ++j) load8<VEC>(a.dy, row, 8 * t + j * kStep, a.cols, dy[j]);
    const float rstd = a.rstd[row];
    if (a.xhat.q) {
#pragma unroll
      for (int j = 0; j < J; ++j) ckpt_load8(a.xhat, row, 8 * t + j * kStep, xh[j]);
    } else {
#pragma unroll
      for (int j = 0; j < J; ++j) load8<VEC>(a.x, row, 8 * t + j * kStep, a.cols, xh[j]);
      const float mean = a.mean[row];
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) xh[j][i] = (xh[j][i] - mean) * rstd;
    }
    float s = 0.f, sx = 0.f;
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        // (past the last column dy and the gain are 0; xhat may be anything there)
        if (!VEC) xh[j][i] = 8 * t + j * kStep + i < a.cols ? xh[j][i] : 0.f;
        dg[j][i] = fmaf(dy[j][i], xh[j][i], dg[j][i]);
        db[j][i] += dy[j][i];
        dy[j][i] *= g[j][i];
        s += dy[j][i];
        sx = fmaf(dy[j][i], xh[j][i], sx);
      }
    const float m = row_total<W>(s, red) * inv_n, mx = row_total<W>(sx, red) * inv_n;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int c = 8 * t + j * kStep;
      float d[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) d[i] = rstd * (dy[j][i] - m - xh[j][i] * mx);
      if (a.dres.p) {
        float r[8];
        load8<VEC>(a.dres, row, c, a.cols, r);
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] += r[i];
      }
      store8<VEC>(a.dx, row, c, a.cols, d);
      if (a.copy.p) store8<VEC>(a.copy, row, c, a.cols, d);
    }
  }
  if (!a.dgain) return;
  float* part = a.part + (size_t)blockIdx.x * 2 * a.cols;
  if constexpr (W == 4) {
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int c = 8 * t + j * kStep + i;
        if (c < a.cols) { part[c] = dg[j][i]; part[a.cols + c] = db[j][i]; }
      }
  } else {
    // the four waves hold the same columns: they are added in order (one wave after the other through
    // one row of LDS, with a barrier each, 4000 x 1280 took 21.0 us with both launches; this takes 20.4)
    __shared__ f32x4 sum[4][2][J * kStep / 4];
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int c = (8 * t + j * kStep) / 4 + h;
        sum[w][0][c] = f32x4{dg[j][4 * h], dg[j][4 * h + 1], dg[j][4 * h + 2], dg[j][4 * h + 3]};
        sum[w][1][c] = f32x4{db[j][4 * h], db[j][4 * h + 1], db[j][4 * h + 2], db[j][4 * h + 3]};
      }
    __syncthreads();
    for (int c = threadIdx.x; c < a.cols; c += 256)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float v = ((const float*)sum[0][h])[c];
#pragma unroll
        for (int o = 1; o < 4; ++o) v += ((const float*)sum[o][h])[c];
        part[h * a.cols + c] = v;
      }
  }
}

// dgain | dbias: column c of [groups][2 cols] partial rows, 16 columns x 64 row slices a
// workgroup, the slices joined in order.
__global__ void __launch_bounds__(1024) ln_param_kernel(int groups, int cols, const float* part, float* dgain,
                                                        float* dbias, int accumulate) {
  __shared__ float red[64][17];
  const int x = threadIdx.x % 16, y = threadIdx.x / 16, c = blockIdx.x * 16 + x;
  float s = 0.f;
  if (c < 2 * cols)
#pragma unroll 8
    for (int r = y; r < groups; r += 64) s += part[(size_t)r * 2 * cols + c];
  red[y][x] = s;
  __syncthreads();
  if (y < 8) {
    s = red[8 * y][x];
#pragma unroll
    for (int r = 1; r < 8; ++r) s += red[8 * y + r][x];
  }
  __syncthreads();
  if (y < 8) red[y][x] = s;
  __syncthreads();
  if (y == 0 && c < 2 * cols) {
#pragma unroll
    for (int r = 1; r < 8; ++r) s += red[r][x];
    float* o = c < cols ? dgain + c : dbias + (c - cols);
    *o = accumulate ? *o + s : s;
  }
}

// A wave takes 512 columns of one row at a time (unit u: row u / segs, segment u % segs; the
// launcher's caller has checked rows * segs < 2^31).
__global__ void __launch_bounds__(256) ckpt_pack_kernel(unsigned units, unsigned segs, int cols, DMat x, DCkpt k) {
  for (unsigned u = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + threadIdx.x / kWave); u < units; u += gridDim.x * 4) {
    const int c = (int)(u % segs) * 512 + 8 * (threadIdx.x % kWave);
    float v[8];
    load8(x, u / segs, c, cols, v);
    ckpt_store8(k, u / segs, c, v);
  }
}

template <bool GELU>
__global__ void __launch_bounds__(256) ckpt_unpack_kernel(unsigned units, unsigned segs, int cols, DCkpt k, DMat out) {
  for (unsigned u = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + threadIdx.x / kWave); u < units; u += gridDim.x * 4) {
    const int c = (int)(u % segs) * 512 + 8 * (threadIdx.x % kWave);
    float v[8];
    ckpt_load8(k, u / segs, c, v);
    if (GELU)
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = gelu_value(v[i]);
    store8(out, u / segs, c, cols, v);
  }
}

constexpr int kMaxGrid = 1 << 22;   // workgroups of 256 threads that a launch may have
int grid_of(int64_t groups) { return (int)std::min<int64_t>(groups, kMaxGrid); }

// J pieces of 8 columns a lane, one wave a row up to 2048 columns, else four
template <template <int, int> class F, class... A>
void by_width(int cols, A&&... args) {
  if (cols <= 512) F<1, 1>::run(args...);
  else if (cols <= 1024) F<2, 1>::run(args...);
  else if (cols <= 1536) F<3, 1>::run(args...);
  else if (cols <= 2048) F<4, 1>::run(args...);
  else if (cols <= 4096) F<2, 4>::run(args...);
  else F<4, 4>::run(args...);
}

bool whole(const DMat& m) { return !m.p || m.vec; }
bool whole(const DVec& v, int cols) { return v.vec && cols % 8 == 0; }

template <int J, int W>
struct Fwd {
  static void run(const LnFwdArgs& a, hipStream_t st) {
    const bool vec = whole(a.x) && whole(a.y) && whole(a.gain, a.cols) && whole(a.bias, a.cols);
    const int grid = grid_of(W == 1 ? (a.rows + 3) / 4 : a.rows);
    if (vec) ln_fwd_kernel<J, W, true><<<grid, 256, 0, st>>>(a);
    else ln_fwd_kernel<J, W, false><<<grid, 256, 0, st>>>(a);
  }
};
template <int J, int W>
struct Bwd {
  static void run(const LnBwdArgs& a, int groups, hipStream_t st) {
    const bool vec = whole(a.dy) && whole(a.x) && whole(a.dres) && whole(a.dx) && whole(a.copy) && whole(a.gain, a.cols);
    if (vec) ln_bwd_kernel<J, W, true><<<groups, 256, 0, st>>>(a);
    else ln_bwd_kernel<J, W, false><<<groups, 256, 0, st>>>(a);
  }
};

}  // namespace

void launch_layer_norm(const LnFwdArgs& a, hipStream_t st) {
  if (a.rows > 0) by_width<Fwd>(a.cols, a, st);
}

int ln_bwd_groups(int rows, int cols) {
  const int per = cols <= 2048 ? 4 : 1;   // rows a workgroup holds at a time
  return std::min((rows + per - 1) / per, 512);
}

void launch_layer_norm_backward(const LnBwdArgs& a, hipStream_t st) {
  const int groups = ln_bwd_groups(a.rows, a.cols);
  if (groups > 0) by_width<Bwd>(a.cols, a, groups, st);
  if (a.dgain)
    ln_param_kernel<<<(2 * a.cols + 15) / 16, 1024, 0, st>>>(groups, a.cols, a.part, a.dgain, a.dbias, a.accumulate);
}

void launch_ckpt_pack(int rows, int cols, const DMat& x, const DCkpt& k, hipStream_t st) {
  const unsigned segs = (k.ld + 511) / 512, units = (unsigned)rows * segs;
  if (units) ckpt_pack_kernel<<<grid_of((units + 3ull) / 4), 256, 0, st>>>(units, segs, cols, x, k);
}

void launch_ckpt_unpack(int rows, int cols, const DCkpt& k, bool gelu, const DMat& out, hipStream_t st) {
  const unsigned segs = (k.ld + 511) / 512, units = (unsigned)rows * segs;
  if (!units) return;
  const int grid = grid_of((units + 3ull) / 4);
  if (gelu) ckpt_unpack_kernel<true><<<grid, 256, 0, st>>>(units, segs, cols, k, out);
  else ckpt_unpack_kernel<false><<<grid, 256, 0, st>>>(units, segs, cols, k, out);
}

}  // namespace ad
