// Which tensors an optimizer launch takes: rules on sizes, without the HIP headers.
#pragma once

#include <cstdint>

namespace ad {

constexpr int kOptChunk = 8192;                            // elements of a workgroup
// Tensors of one launch: kernel arguments hold 4 KB.
constexpr int kOptTensors = 40;
// Workgroups of one launch: they have 256 threads, of which a launch takes under 2^32.
constexpr int64_t kOptGroups = (1 << 24) - 1;
constexpr int64_t kOptMost = kOptGroups * kOptChunk;       // elements of a tensor

inline int64_t opt_groups(int64_t n) { return (n + kOptChunk - 1) / kOptChunk; }

// The places of the tensors that hold something and that one launch takes, from tensor i on (places: kOptTensors of
// them at most); returns where the next launch goes on.  size(i): elements of tensor i, up to kOptMost.
template <class Size>
inline int opt_launch(Size&& size, int count, int i, int* places, int& n) {
  int64_t groups = 0;
  for (n = 0; i < count; ++i) {
    const int64_t more = opt_groups(size(i));
    if (!more) continue;
    if (n == kOptTensors || groups + more > kOptGroups) break;
    groups += more;
    places[n++] = i;
  }
  return i;
}

}  // namespace ad
