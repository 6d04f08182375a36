// Which rows of a batch belong to what, and how attention is cut into workgroups: rules on the tables and on
// sizes, without the HIP headers.
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>

#ifdef __HIPCC__
#define AD_BOTH __host__ __device__ __forceinline__
#else
#define AD_BOTH inline
#endif

namespace ad {

// What both passes know of a batch (ad_attn).
struct AttnBatch {
  int batch, heads, kv_heads, group, q_rows, k_rows, q_max, k_max, causal;   // group = heads / kv_heads
  uint64_t per_head, per_kv_head;                                            // per() of heads and kv_heads
  const int *cu_q, *cu_k, *q_len, *k_len, *window;
  int* err;
};
// n / d = (n per(d)) >> kPerShift for n < 2^24, d <= 2^14: per(d) d - 2^40 < d, so the quotient is off by less than
// n d / 2^40 < 1 / d.
constexpr int kPerShift = 40;
inline uint64_t per(int d) { return ((uint64_t(1) << kPerShift) + d - 1) / d; }

AD_BOTH int smaller(int a, int b) { return a < b ? a : b; }
AD_BOTH int larger(int a, int b) { return a > b ? a : b; }

// One sequence's rows; ok = false where its table entries are out of range.
struct Span {
  int q0, nq, oq, k0, nk, ow;    // first row, rows that hold something, rows it owns; the same of the keys
  bool ok;
};
AD_BOTH Span span_of(const AttnBatch& a, int b) {
  Span s;
  s.q0 = a.cu_q[b];
  s.k0 = a.cu_k[b];
  const int qe = a.cu_q[b + 1], ke = a.cu_k[b + 1];
  s.ok = s.q0 >= 0 && qe >= s.q0 && qe <= a.q_rows && s.k0 >= 0 && ke >= s.k0 && ke <= a.k_rows;
  s.oq = qe - s.q0;
  s.ow = ke - s.k0;
  s.nq = a.q_len ? a.q_len[b] : s.oq;
  s.nk = a.k_len ? a.k_len[b] : s.ow;
  s.ok = s.ok && s.oq <= a.q_max && s.ow <= a.k_max && s.nq >= 0 && s.nq <= s.oq && s.nk >= 0 && s.nk <= s.ow;
  return s;
}

// The keys [lo, hi) that query i of the sequence sees (lo >= hi: none), both ends in [0, nk] whatever the window holds.
struct Keys {
  int lo, hi;
};
AD_BOTH Keys keys_of(const AttnBatch& a, const Span& s, int i) {
  Keys r = {0, s.nk};
  if (a.causal) r.hi = smaller(r.hi, larger(i + s.nk - s.nq + 1, 0));
  if (a.window) {
    const int* w = a.window + 2 * ((size_t)s.q0 + i);
    r.lo = smaller(larger(w[0], 0), s.nk);
    r.hi = smaller(r.hi, larger(w[1], 0));
  }
  return r;
}

// Of the places from key `first` on, place e (at most a tile's) is seen where shows() says so: the keys' ends lie in
// [0, nk], so no difference overflows.
struct Mask {
  int lo;
  unsigned len;
};
AD_BOTH Mask mask_of(const Keys& k, int first) { return Mask{k.lo - first, (unsigned)larger(k.hi - k.lo, 0)}; }
AD_BOTH bool shows(const Mask& m, int e) { return (unsigned)(e - m.lo) < m.len; }

// What 32 queries see together.
struct Range {
  int lo, hi;          // some of them may see [lo, hi)
  int all_lo, all_hi;  // all of them see [all_lo, all_hi)
};

// The steps of a workgroup's keys [k0, k1): tiles of TQ queries of one head after the other, those that some
// of the keys are seen by.  ranges: of every 32 queries of the sequence the four numbers of a Range (read with windows only).
template <int TQ, class Table>
struct Walk {
  Table ranges;
  bool window, causal;
  int nq, nk, k0, k1, start, tiles, t, h, heads_end;
  AD_BOTH Walk(const AttnBatch& a, const Span& s, Table ranges_, int g, int k0_, int k1_) {
    ranges = ranges_;
    window = a.window;
    causal = a.causal;
    nq = s.nq; nk = s.nk; k0 = k0_; k1 = k1_;
    tiles = (nq + TQ - 1) / TQ;
    // (causal: the queries before key - (nk - nq) do not see the key)
    start = causal ? smaller(larger(k0 - (nk - nq), 0) / TQ, tiles) : 0;
    t = start;
    h = g * a.group;
    heads_end = k1 > k0 ? h + a.group : h;      // (keys that are all padding: no steps)
  }
  // what the queries 32 u .. + 31 see together
  AD_BOTH Range seen(int u) const {
    Range r = {0, nk, 0, nk};
    if (window) {
      const Table p = ranges + 4 * u;
      r = Range{p[0], p[1], p[2], p[3]};
    } else if (causal) {
      r.all_hi = 32 * u + nk - nq + 1;
      r.hi = smaller(nk, r.all_hi + 31);
    }
    return r;
  }
  AD_BOTH bool wanted() const {
    if (!window) return true;
    for (int u = t * (TQ / 32); u < smaller((t + 1) * (TQ / 32), (nq + 31) / 32); ++u) {
      const Range r = seen(u);
      if (r.lo < k1 && r.hi > k0) return true;
    }
    return false;
  }
  // from (h, t) on to a step that is wanted; false: there is none
  AD_BOTH bool settle() {
    for (; h < heads_end; ++h, t = start)
      for (; t < tiles; ++t)
        if (wanted()) return true;
    return false;
  }
};

// Where wave w starts that takes 32 of the keys [lo, hi) in turn with others; where there are none (lo the largest
// integer, hi = 0) it is not before hi, so that nothing is read.
AD_BOTH int first_piece(int lo, int hi, int w) { return smaller(lo, hi) / 32 * 32 + 32 * w; }

// ----------------------------------------------------------------- workgroups

// Whether four waves take 32 rows each (of `rows` at most a sequence), or 32 rows together.  A wide workgroup has a tile
// of 64 done in 0.9 us alone on its CU and in 0.75 among others, one of few rows 128 in 1.25 and 0.87: the
// latter is worth it only while there are fewer than about 128 of the former (448 x 1500, 20 heads: 80
// of them take 28.5 us, 280 small ones 21; 12 x 128 causal, 240: 8.7 and 12.7).  With windows a wide workgroup walks
// over what 128 rows see, most of which each wave leaves out (12 x 131, windows of 41 in 1500: 35 and 25 us); a
// workgroup of keys walks over the few queries that see them (36 and 76).
inline bool wide_rows(const AttnBatch& b, int rows, int heads, bool keys = false) {
  return rows > 32 && (int64_t)((rows + 127) / 128) * heads * b.batch >= (b.window && !keys ? 1024 : 128);
}

// How a forward pass is cut.  Where even the small workgroups leave CUs without work, eight waves have keys of their own
// (`keys`, in rounds of 256), or the keys are in `splits` parts of `chunk` and a second launch joins them.  A round takes
// 0.7 us, a part 1 us for every 128 keys and the second launch 4: with 20 workgroups 448 keys 8.4 and 11.1 us, 1500
// 11.2 and 11.1, 4000 20.7 and 13.4; with 80 1500 11.7 and 13.7, 4000 21.1 and 21.4; with 240 17.6 and 22.3, 46 and 53.
struct FwdPlan {
  bool few, keys;
  int tiles, splits, chunk;
};
inline FwdPlan fwd_plan(const AttnBatch& b) {
  FwdPlan p = {false, false, (b.q_max + 127) / 128, 1, 0};
  if (!p.tiles || !b.batch) return p;
  const int64_t pairs = (int64_t)b.heads * b.batch;
  if (wide_rows(b, b.q_max, b.heads)) return p;
  p.few = true;
  p.tiles = (b.q_max + 31) / 32;
  const int stages = std::max((b.k_max + 127) / 128, 1);
  const int64_t groups = pairs * p.tiles;
  const int want = (int)std::min<int64_t>(std::min(stages, 64), std::max<int64_t>(512 / groups, 1));
  const int each = (stages + want - 1) / want;
  p.splits = (stages + each - 1) / each;
  p.keys = p.splits > 1 && (stages + 1) / 2 <= 4 + 2 * each;
  if (p.keys) p.splits = 1;
  p.chunk = each * 128;
  return p;
}

// A part's rows, and a query's place among them.  By sequence and not by the matrix's rows, which may be far more: so
// all parts have at most the rows of fwd_plan's 512 workgroups.
AD_BOTH size_t part_rows(const AttnBatch& b) { return (size_t)b.heads * b.batch * b.q_max; }
AD_BOTH size_t part_row(const AttnBatch& a, int b, int h, int i) { return ((size_t)h * a.batch + b) * a.q_max + i; }
inline size_t attn_fwd_bytes(const AttnBatch& b) {
  const FwdPlan p = fwd_plan(b);
  return p.splits > 1 ? 4ull * 66 * p.splits * part_rows(b) : 0;
}
// delta [heads][q_rows], then what 32 queries of a sequence see together [batch][blocks]
inline size_t attn_bwd_delta_bytes(const AttnBatch& b) { return (4ull * b.heads * b.q_rows + 255) / 256 * 256; }
inline size_t attn_bwd_bytes(const AttnBatch& b) {
  return attn_bwd_delta_bytes(b) + 16ull * b.batch * ((b.q_max + 31) / 32);
}
// A launch's grid has 8 workgroups a tile in x and a row for 8 (sequence, head) pairs in y.
constexpr int kMaxPairs = 65535 * 8;
inline bool attn_fits(const AttnBatch& b) { return (int64_t)b.batch * b.heads <= kMaxPairs; }

}  // namespace ad
