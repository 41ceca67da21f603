// Attention inside a window with first tokens that stay visible, shared key / value heads and a length per sample, forward and
// backward, grouped over all branches of a level: the row-parallel kernels for every head dimension and type.
//   visible(i, j) = (not causal or j <= i) and (|i - j| < window or j < sinks),  i, j < length of the sample
//   P = softmax over the visible j of scale q_i.k_j,  O = P V
//   dV = P^T dO, dP = dO V^T, dS = P * (dP - rowsum(dO * O)), dQ = scale dS K, dK = scale dS^T Q
// (dK and dV summed over the query heads that share the key / value head).  One wavefront per query row (forward, dQ) or per
// key row (dK, dV); the running maximum and sum of the softmax go over 64 keys at a time.  Deterministic: no atomics.
// For what the matrix-core kernels (attention_window_mfma.hip) do not take: head dimensions above 128 or off 16 bytes, operands of two
// storage types, an output in a merge at a column off 16 bytes.  Bound by the loads of a key's row per lane: 4 x 512, window 128, 16
// heads of 64 in bf16 take 5.1 ms a step here, 45 us there.
#include "device_utils.h"
#include "window_utils.h"

namespace gpp {

constexpr int WIN_MAX_DH = 256;
constexpr int WIN_DPL = WIN_MAX_DH / 64;    // columns of a head per lane

int window_max_head_dim() { return WIN_MAX_DH; }
int window_blocks(int64_t batch, int heads, int seq) { return (int)(batch * heads * ((seq + 3) / 4)); }

struct WindowRow {
  int b, h, row;
};
__device__ __forceinline__ WindowRow window_row(const WindowProb &p, int heads, int blk) {
  const int rb = (p.seq + 3) / 4, bh = blk / rb;
  WindowRow w;
  w.b = bh / heads;
  w.h = bh % heads;
  w.row = (blk % rb) * 4 + (threadIdx.x >> 6);
  return w;
}
// dot product of dh values in LDS with a row in memory
__device__ __forceinline__ float lds_dot(const float *v, const GPP_G void *base, int64_t off, int dh, int dtype) {
  float s = 0.0f;
  for (int c = 0; c < dh; ++c) s += v[c] * load_as_f32((const void *)base, dtype, off + c);
  return s;
}

__global__ __launch_bounds__(256) void k_window_fwd(const WindowProb *__restrict__ probs, int n, ExtPtrs ext, StageFlags *flags) {
  __shared__ float lds[4][WIN_MAX_DH];
  const int pi = find_prob(probs, n, blockIdx.x);
  const WindowProb p = probs[pi];
  const WindowRow w = window_row(p, p.heads, blockIdx.x - p.blk_begin);
  const int lane = threadIdx.x & 63;
  float *qv = lds[threadIdx.x >> 6];
  const int len = window_length_checked(p, ext, w.b, w.h == 0 && w.row == 0 && lane == 0, flags);
  if (w.row >= p.seq) return;
  const GPP_G void *qkv = p.ext_qkv >= 0 ? ext.p[p.ext_qkv] : p.qkv;
  GPP_G void *out2 = p.ext_out >= 0 ? ext.p[p.ext_out] : nullptr;
  const int kh = w.h / (p.heads / p.kv_heads);
  const int64_t base = (int64_t)w.b * p.seq, row = base + w.row;
  const int64_t kcol = (int64_t)(p.heads + kh) * p.dh, vcol = (int64_t)(p.heads + p.kv_heads + kh) * p.dh;
  if (p.qkv_keep) {        // its own query, and the first of the heads that share them its key and value
    const int blocks = w.h % (p.heads / p.kv_heads) == 0 ? 3 : 1;
    for (int k = 0; k < blocks; ++k)
      for (int c = lane; c < p.dh; c += 64) {
        const int64_t col = (k == 0 ? (int64_t)w.h * p.dh : k == 1 ? kcol : vcol) + c;
        if (p.dtype == DT_BF16) ((GPP_G uint16_t *)p.qkv_keep)[row * p.ld_keep + col] = ((const GPP_G uint16_t *)qkv)[row * p.ld_qkv + col];
        else ((GPP_G float *)p.qkv_keep)[row * p.ld_keep + col] = ((const GPP_G float *)qkv)[row * p.ld_qkv + col];
      }
  }
  float o[WIN_DPL] = {0.0f}, m = -INFINITY, l = 0.0f;
  const float scale2 = p.scale * LOG2E;
  if (w.row < len) {
    for (int c = lane; c < p.dh; c += 64) qv[c] = load_as_f32((const void *)qkv, p.dtype, row * p.ld_qkv + (int64_t)w.h * p.dh + c);
    __builtin_amdgcn_wave_barrier();
    const WindowKeys keys = window_keys(p, w.row, len);
    for (int part = 0; part < 2; ++part) {
      const int end = part ? keys.end : keys.sink_end;
      for (int j0 = part ? keys.first : 0; j0 < end; j0 += 64) {
        const int j = j0 + lane;
        const float s = j < end ? lds_dot(qv, qkv, (base + j) * p.ld_qkv + kcol, p.dh, p.dtype) * scale2 : -INFINITY;
        const float m_new = fmaxf(m, wave_max(s)), ref = m_new == -INFINITY ? 0.0f : m_new;
        const float e = __builtin_amdgcn_exp2f(s - ref), alpha = __builtin_amdgcn_exp2f(m - ref);
        l = l * alpha + wave_sum(e);
        m = m_new;
#pragma unroll
        for (int k = 0; k < WIN_DPL; ++k) o[k] *= alpha;
        for (int i = 0; i < min(64, end - j0); ++i) {
          const float pr = lane_f32(e, i);
#pragma unroll
          for (int k = 0; k < WIN_DPL; ++k)
            if (lane + 64 * k < p.dh) o[k] += pr * load_as_f32((const void *)qkv, p.dtype, (base + j0 + i) * p.ld_qkv + vcol + lane + 64 * k);
        }
      }
    }
  }
  const float inv = l > 0.0f ? 1.0f / l : (w.row < len ? NAN : 0.0f);      // (every row inside the length sees itself)
#pragma unroll
  for (int k = 0; k < WIN_DPL; ++k) {
    const int c = lane + 64 * k;
    if (c >= p.dh) continue;
    const float v = w.row < len ? o[k] * inv : 0.0f;
    if (p.out) store_from_f32((void *)p.out, p.out_dtype, row * p.ld_out + (int64_t)w.h * p.dh + c, v);
    if (out2) store_from_f32((void *)out2, p.out_dtype, row * p.ld_ext + (int64_t)w.h * p.dh + c, v);
    if (p.o_lo) store_from_f32((void *)p.o_lo, DT_BF16, row * p.ld_lo + (int64_t)w.h * p.dh + c, v - bf16_bits_to_f32(f32_to_bf16_bits(v)));
  }
  if (p.lse && lane == 0) p.lse[((int64_t)w.b * p.heads + w.h) * p.seq + w.row] = m + __builtin_amdgcn_logf(l);
}

// dQ of one query row per wave, and delta = rowsum(dO * O)
__global__ __launch_bounds__(256) void k_window_dq(const WindowProb *__restrict__ probs, int n, ExtPtrs ext) {
  __shared__ float lds[4][2 * WIN_MAX_DH];
  const int pi = find_prob(probs, n, blockIdx.x);
  const WindowProb p = probs[pi];
  const WindowRow w = window_row(p, p.heads, blockIdx.x - p.blk_begin);
  const int lane = threadIdx.x & 63;
  float *qv = lds[threadIdx.x >> 6], *gv = qv + WIN_MAX_DH;
  const int len = window_length(p, w.b);
  if (w.row >= p.seq) return;
  const GPP_G void *dout = p.ext_dout >= 0 ? ext.p[p.ext_dout] : p.dout;
  GPP_G void *dqkv = p.ext_out >= 0 ? ext.p[p.ext_out] : p.out;
  const int kh = w.h / (p.heads / p.kv_heads);
  const int64_t base = (int64_t)w.b * p.seq, row = base + w.row, stat = ((int64_t)w.b * p.heads + w.h) * p.seq + w.row;
  const int64_t kcol = (int64_t)(p.heads + kh) * p.dh, vcol = (int64_t)(p.heads + p.kv_heads + kh) * p.dh;
  float dq[WIN_DPL] = {0.0f};
  const float scale2 = p.scale * LOG2E;
  if (w.row < len) {
    float d = 0.0f;
    for (int c = lane; c < p.dh; c += 64) {
      qv[c] = load_as_f32((const void *)p.qkv, p.dtype, row * p.ld_qkv + (int64_t)w.h * p.dh + c);
      const float g = load_as_f32((const void *)dout, p.out_dtype, row * p.ld_dout + (int64_t)w.h * p.dh + c);
      gv[c] = g;
      const float low = p.o_lo ? load_as_f32((const void *)p.o_lo, DT_BF16, row * p.ld_lo + (int64_t)w.h * p.dh + c) : 0.0f;
      d += g * (load_as_f32((const void *)p.o, p.out_dtype, row * p.ld_o + (int64_t)w.h * p.dh + c) + low);
    }
    d = wave_sum(d);
    if (lane == 0) p.delta[stat] = d;
    const float lse = p.lse[stat];
    __builtin_amdgcn_wave_barrier();
    const WindowKeys keys = window_keys(p, w.row, len);
    for (int part = 0; part < 2 && keys.count > 1; ++part) {      // (a single key's probability is constant: no gradient)
      const int end = part ? keys.end : keys.sink_end;
      for (int j0 = part ? keys.first : 0; j0 < end; j0 += 64) {
        const int j = j0 + lane;
        float ds = 0.0f;
        if (j < end) {
          const float s = lds_dot(qv, p.qkv, (base + j) * p.ld_qkv + kcol, p.dh, p.dtype) * scale2;
          ds = __builtin_amdgcn_exp2f(s - lse) * (lds_dot(gv, p.qkv, (base + j) * p.ld_qkv + vcol, p.dh, p.dtype) - d);
        }
        for (int i = 0; i < min(64, end - j0); ++i) {
          const float di = lane_f32(ds, i);
#pragma unroll
          for (int k = 0; k < WIN_DPL; ++k)
            if (lane + 64 * k < p.dh) dq[k] += di * load_as_f32((const void *)p.qkv, p.dtype, (base + j0 + i) * p.ld_qkv + kcol + lane + 64 * k);
        }
      }
    }
  }
  if (!dqkv) return;
#pragma unroll
  for (int k = 0; k < WIN_DPL; ++k)
    if (lane + 64 * k < p.dh) store_from_f32((void *)dqkv, p.grad_dtype, row * p.ld_out + (int64_t)w.h * p.dh + lane + 64 * k, dq[k] * p.scale);
}

// dK and dV of one key row per wave, over the query heads that share it
__global__ __launch_bounds__(256) void k_window_dkv(const WindowProb *__restrict__ probs, int n, ExtPtrs ext) {
  __shared__ float lds[4][2 * WIN_MAX_DH];
  const int pi = find_prob(probs, n, blockIdx.x);
  const WindowProb p = probs[pi];
  const WindowRow w = window_row(p, p.kv_heads, blockIdx.x - p.blk_begin);
  const int lane = threadIdx.x & 63;
  float *kv = lds[threadIdx.x >> 6], *vv = kv + WIN_MAX_DH;
  const int len = window_length(p, w.b);
  const GPP_G void *dout = p.ext_dout >= 0 ? ext.p[p.ext_dout] : p.dout;
  GPP_G void *dqkv = p.ext_out >= 0 ? ext.p[p.ext_out] : p.out;
  if (w.row >= p.seq || !dqkv) return;
  const int64_t base = (int64_t)w.b * p.seq, row = base + w.row;
  const int64_t kcol = (int64_t)(p.heads + w.h) * p.dh, vcol = (int64_t)(p.heads + p.kv_heads + w.h) * p.dh;
  float dk[WIN_DPL] = {0.0f}, dv[WIN_DPL] = {0.0f};
  const float scale2 = p.scale * LOG2E;
  if (w.row < len) {
    for (int c = lane; c < p.dh; c += 64) {
      kv[c] = load_as_f32((const void *)p.qkv, p.dtype, row * p.ld_qkv + kcol + c);
      vv[c] = load_as_f32((const void *)p.qkv, p.dtype, row * p.ld_qkv + vcol + c);
    }
    __builtin_amdgcn_wave_barrier();
    const WindowQueries q = window_queries(p, w.row, len);
    const int group = p.heads / p.kv_heads;
    for (int h = w.h * group; h < (w.h + 1) * group; ++h) {
      const int64_t stat0 = ((int64_t)w.b * p.heads + h) * p.seq;
      for (int i0 = q.first; i0 < q.end; i0 += 64) {
        const int i = i0 + lane;
        float pr = 0.0f, ds = 0.0f;
        if (i < q.end) {
          const float s = lds_dot(kv, p.qkv, (base + i) * p.ld_qkv + (int64_t)h * p.dh, p.dh, p.dtype) * scale2;
          pr = __builtin_amdgcn_exp2f(s - p.lse[stat0 + i]);
          if (window_keys(p, i, len).count > 1)
            ds = pr * (lds_dot(vv, dout, (base + i) * p.ld_dout + (int64_t)h * p.dh, p.dh, p.out_dtype) - p.delta[stat0 + i]);
        }
        for (int t = 0; t < min(64, q.end - i0); ++t) {
          const float pt = lane_f32(pr, t), dt = lane_f32(ds, t);
#pragma unroll
          for (int k = 0; k < WIN_DPL; ++k) {
            const int c = lane + 64 * k;
            if (c >= p.dh) continue;
            dk[k] += dt * load_as_f32((const void *)p.qkv, p.dtype, (base + i0 + t) * p.ld_qkv + (int64_t)h * p.dh + c);
            dv[k] += pt * load_as_f32((const void *)dout, p.out_dtype, (base + i0 + t) * p.ld_dout + (int64_t)h * p.dh + c);
          }
        }
      }
    }
  }
#pragma unroll
  for (int k = 0; k < WIN_DPL; ++k) {
    const int c = lane + 64 * k;
    if (c >= p.dh) continue;
    store_from_f32((void *)dqkv, p.grad_dtype, row * p.ld_out + kcol + c, dk[k] * p.scale);
    store_from_f32((void *)dqkv, p.grad_dtype, row * p.ld_out + vcol + c, dv[k]);
  }
}

void launch_window_fwd(const WindowProb *probs, int n, int total_blocks, const ExtPtrs &ext, StageFlags *flags, hipStream_t s) {
  if (total_blocks > 0) hipLaunchKernelGGL(k_window_fwd, dim3(total_blocks), dim3(256), 0, s, probs, n, ext, flags);
}
void launch_window_dq(const WindowProb *probs, int n, int total_blocks, const ExtPtrs &ext, hipStream_t s) {
  if (total_blocks > 0) hipLaunchKernelGGL(k_window_dq, dim3(total_blocks), dim3(256), 0, s, probs, n, ext);
}
void launch_window_dkv(const WindowProb *probs, int n, int total_blocks, const ExtPtrs &ext, hipStream_t s) {
  if (total_blocks > 0) hipLaunchKernelGGL(k_window_dkv, dim3(total_blocks), dim3(256), 0, s, probs, n, ext);
}

}  // namespace gpp
