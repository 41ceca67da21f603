// Rotary positions with one to four axes, forward and backward (the transposed rotation), grouped over all branches of a level.
//   pair i of axis a at position p turns by t = p * w_i:  y0 = x0 cos t - x1 sin t,  y1 = x0 sin t + x1 cos t
//   backward:                                             dx0 = dy0 cos t + dy1 sin t,  dx1 = dy1 cos t - dy0 sin t
// Bound by memory: every element is read once and written once (32768 rows of 32 + 8 + 8 heads of 128 in bf16, 805 MB each way: 159 -
// 169 us, 4.8 - 5.1 TB/s, the rate of a large copy; a few rows: a launch, 3 us).  The angles of a row are shared by its heads, so a workgroup
// forms those of its rows once, in LDS, and then streams whole rows; angles are products in 64 bits, reduced to a fraction of a
// quarter turn there (a position of 10^5 times a frequency of 1 has 5 digits left of 32 bits behind the point), sine and cosine of
// that fraction are 32 bits.
#include "device_utils.h"

namespace gpp {

constexpr int ROT_MAX_PAIRS = 512;   // of a head: 4 KB of LDS per row of a workgroup
constexpr int ROT_MAX_ROWS = 16;     // rows of a workgroup at the most
constexpr int ROT_LDS = 2048;        // (cos, sin) entries of a workgroup: 16 KB, eight workgroups per compute unit
static_assert(ROT_MAX_PAIRS <= ROT_LDS, "the angles of a row fit");

int rotary_max_pairs() { return ROT_MAX_PAIRS; }

// Elements that a lane moves at once: 16 bytes where a pair's two columns (halves), a head, a row and the address allow it, or 8
// or 4 where only that, single elements otherwise.
int rotary_vec(const RotaryProb &p) {
  const int whole = p.dtype == DT_BF16 ? 8 : 4;
  for (int v = whole; v > 1; v >>= 1) {
    const int64_t unit = p.neighbours ? 2 * p.pairs : p.pairs;      // columns whose partners lie beside them
    const bool aligned = (((uintptr_t)p.x | (uintptr_t)p.y) & (v * (p.dtype == DT_BF16 ? 2 : 4) - 1)) == 0;
    if (aligned && unit % v == 0 && p.dh % v == 0 && p.cols % v == 0 && p.ld_x % v == 0 && p.ld_y % v == 0) return v;
  }
  return 1;
}

// Rows of a workgroup: many where the launch still has some workgroups per compute unit, so that forming the angles, which a
// workgroup does before anything else, is spread over more of them
int rotary_rows_per_block(int64_t launch_rows, int pairs) {
  int r = 1;
  while (r < ROT_MAX_ROWS && launch_rows / (2 * r) >= 2048 && 2 * r * pairs <= ROT_LDS) r *= 2;
  return r;
}

// cos and sin of `turns` turns (a turn is 2 pi), any size
__device__ __forceinline__ float2 cos_sin_turns(double turns) {
  double q = 4.0 * turns;
  const double whole = rint(q);
  const float f = (float)(q - whole);                         // quarter turns, at most a half to either side
  const int quarter = (int)(int64_t)(whole - 4.0 * floor(0.25 * whole));
  float s, c;
  sincospif(0.5f * f, &s, &c);
  const float cs = (quarter & 1) ? s : c, sn = (quarter & 1) ? c : s;
  return make_float2((quarter == 1 || quarter == 2) ? -cs : cs, (quarter >= 2) ? -sn : sn);
}

template <int BYTES>
struct RotWord;
template <>
struct RotWord<16> {
  typedef uint32_t type __attribute__((ext_vector_type(4)));
};
template <>
struct RotWord<8> {
  typedef uint32_t type __attribute__((ext_vector_type(2)));
};
template <>
struct RotWord<4> {
  typedef uint32_t type;
};
template <>
struct RotWord<2> {
  typedef uint16_t type;
};

template <typename T, int V>
struct RotChunk {
  typedef typename RotWord<sizeof(T) * V>::type word;
  T e[V];
  __device__ __forceinline__ void load(const GPP_G T *p) {
    const word w = *(const GPP_G word *)p;
    __builtin_memcpy(e, &w, sizeof(w));
  }
  __device__ __forceinline__ void store(GPP_G T *p) const {
    word w;
    __builtin_memcpy(&w, e, sizeof(w));
    *(GPP_G word *)p = w;
  }
  __device__ __forceinline__ float get(int i) const { return to_f32<T>(e[i]); }
  __device__ __forceinline__ void set(int i, float v) {
    if constexpr (sizeof(T) == 2) e[i] = f32_to_bf16_bits(v);
    else e[i] = v;
  }
};

// A row is units of V columns: first `turning` units that hold pairs (halves: a unit is V pairs, two chunks P columns apart;
// neighbours: V columns), head by head, then the columns that are handed on.
template <typename T, int V>
__global__ __launch_bounds__(256) void k_rotary(const RotaryProb *__restrict__ probs, int n, ExtPtrs ext) {
  __shared__ float2 angle[ROT_LDS];
  const int pi = find_prob(probs, n, blockIdx.x);
  const RotaryProb p = probs[pi];
  const GPP_G T *x = (const GPP_G T *)(p.ext_x >= 0 ? ext.p[p.ext_x] : p.x);
  GPP_G T *y = (GPP_G T *)(p.ext_y >= 0 ? ext.p[p.ext_y] : p.y);
  const GPP_G int32_t *pos = p.ext_pos >= 0 ? (const GPP_G int32_t *)ext.p[p.ext_pos] : p.pos;
  const int r0 = (blockIdx.x - p.blk_begin) * p.rows_per_block, nr = min(p.rows_per_block, p.rows - r0);
  if (p.pos_keep)
    for (int i = threadIdx.x; i < nr * p.axes; i += 256) p.pos_keep[(int64_t)r0 * p.axes + i] = pos[(int64_t)r0 * p.axes + i];
  if (!y) return;
  for (int i = threadIdx.x; i < nr * p.pairs; i += 256) {
    const int r = i / p.pairs, k = i - r * p.pairs;
    const RotaryPair t = p.table[k];
    float2 cs = cos_sin_turns((double)pos[(int64_t)(r0 + r) * p.axes + t.axis] * t.turns);
    if (p.backward) cs.y = -cs.y;
    angle[i] = cs;
  }
  __syncthreads();
  const bool nb = p.neighbours != 0 && V > 1;                 // (single elements: a unit is a pair in either pairing)
  const int per_head = nb ? 2 * p.pairs / V : p.pairs / V;    // units of a head that turn
  const int tail = (p.dh - 2 * p.pairs) / V;                  // chunks of a head that do not
  const int turning = p.heads * per_head, still = p.in_place ? 0 : p.heads * tail + (p.cols - p.heads * p.dh) / V;
  const int units = turning + still;
  for (int u = threadIdx.x; u < nr * units; u += 256) {
    const int r = u / units, c = u - r * units;
    const GPP_G T *xr = x + (int64_t)(r0 + r) * p.ld_x;
    GPP_G T *yr = y + (int64_t)(r0 + r) * p.ld_y;
    if (c >= turning) {                                       // handed on
      const int s = c - turning, h = tail ? s / tail : 0;
      const int64_t col = tail && h < p.heads ? (int64_t)h * p.dh + 2 * p.pairs + (s - h * tail) * V
                                              : (int64_t)p.heads * p.dh + (int64_t)(s - p.heads * tail) * V;
      RotChunk<T, V> a;
      a.load(xr + col);
      a.store(yr + col);
      continue;
    }
    const int h = c / per_head, k = c - h * per_head;
    const float2 *cs = angle + r * p.pairs;
    if (nb) {
      const int64_t col = (int64_t)h * p.dh + k * V;
      RotChunk<T, V> a, b;
      a.load(xr + col);
#pragma unroll
      for (int e = 0; e < V / 2; ++e) {
        const float2 t = cs[k * (V / 2) + e];
        const float x0 = a.get(2 * e), x1 = a.get(2 * e + 1);
        b.set(2 * e, x0 * t.x - x1 * t.y);
        b.set(2 * e + 1, x0 * t.y + x1 * t.x);
      }
      b.store(yr + col);
    } else {
      const int64_t c0 = (int64_t)h * p.dh + (p.neighbours ? 2 * k : k * V), c1 = p.neighbours ? c0 + 1 : c0 + p.pairs;
      RotChunk<T, V> a, b, ya, yb;
      a.load(xr + c0);
      b.load(xr + c1);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float2 t = cs[k * V + e];
        const float x0 = a.get(e), x1 = b.get(e);
        ya.set(e, x0 * t.x - x1 * t.y);
        yb.set(e, x0 * t.y + x1 * t.x);
      }
      ya.store(yr + c0);
      yb.store(yr + c1);
    }
  }
}

void launch_rotary(const RotaryProb *probs, int n, int total_blocks, int dtype, int vec, const ExtPtrs &ext, hipStream_t s) {
  if (total_blocks <= 0) return;
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(total_blocks), dim3(256), 0, s, probs, n, ext); };
  if (dtype == DT_BF16) {
    if (vec == 8) go(k_rotary<uint16_t, 8>);
    else if (vec == 4) go(k_rotary<uint16_t, 4>);
    else if (vec == 2) go(k_rotary<uint16_t, 2>);
    else go(k_rotary<uint16_t, 1>);
  } else {
    if (vec == 4) go(k_rotary<float, 4>);
    else if (vec == 2) go(k_rotary<float, 2>);
    else go(k_rotary<float, 1>);
  }
}

}  // namespace gpp
