// Which keys a query sees and which queries see a key, for the windowed-attention kernels.
#pragma once
#include "device_utils.h"

namespace gpp {

constexpr float LOG2E = 1.4426950408889634f;

struct Quotient {
  int q, r;
};
__device__ __forceinline__ Quotient divide(int n, const FastDiv &by) {
  uint32_t q = __umulhi((uint32_t)n, by.m), r = (uint32_t)n - q * by.d;
  if (r >= by.d) {
    ++q;
    r -= by.d;
  }
  return {(int)q, (int)r};
}

// length of sample b from the kept copy
__device__ __forceinline__ int window_length(const WindowProb &p, int b) {
  return p.lengths ? min(max(p.lengths[b], 0), p.seq) : p.seq;
}
// the same where the lengths come from the caller: `report`, one thread per sample, keeps them and tells of one out of range
__device__ __forceinline__ int window_length_checked(const WindowProb &p, const ExtPtrs &ext, int b, bool report, StageFlags *flags) {
  const GPP_G int32_t *lengths = p.ext_len >= 0 ? (const GPP_G int32_t *)ext.p[p.ext_len] : p.lengths;
  if (!lengths) return p.seq;
  const int given = lengths[b], len = min(max(given, 0), p.seq);
  if (report) {
    if (p.lengths_keep) p.lengths_keep[b] = len;
    if (given != len) flags->index_error = 1;
  }
  return len;
}

// Keys that query i (inside the length) sees: [0, sink_end) and [first, end), which do not meet.  `count` of them.
struct WindowKeys {
  int sink_end, first, end, count;
};
__device__ __forceinline__ WindowKeys window_keys(const WindowProb &p, int i, int len) {
  const int last = p.causal ? i + 1 : len;                                     // one behind the last key that may be seen at all
  const int w = (int)min(p.window ? p.window : (int64_t)p.seq, (int64_t)p.seq);
  const int sinks = (int)min(p.sinks, (int64_t)last);
  WindowKeys k;
  k.first = max(0, i - w + 1);
  k.end = max((int)min((int64_t)last, (int64_t)i + w), sinks);
  k.sink_end = min(sinks, k.first);
  k.count = k.sink_end + k.end - k.first;
  return k;
}

// Queries that see key j (inside the length): [first, end)
struct WindowQueries {
  int first, end;
};
__device__ __forceinline__ WindowQueries window_queries(const WindowProb &p, int j, int len) {
  const int w = (int)min(p.window ? p.window : (int64_t)p.seq, (int64_t)p.seq);
  WindowQueries q;
  q.first = p.causal ? j : (j < p.sinks ? 0 : max(0, j - w + 1));
  q.end = j < p.sinks ? len : (int)min((int64_t)len, (int64_t)j + w);
  return q;
}

}  // namespace gpp
