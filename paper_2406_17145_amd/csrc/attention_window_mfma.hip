// Windowed attention on the matrix cores, head dimensions up to 128 in bf16 or fp32 (see attention_window.hip for the mathematics).
//
// A workgroup of four waves owns 128 rows (queries: forward, dQ; keys: dK and dV), 32 per wave, whose operands stay in registers; the
// other side streams through LDS in tiles, copied from memory straight into LDS, two buffers: tile t + 1 arrives while tile t
// is multiplied.  Only tiles that hold a visible pair are streamed, only waves that have one in a tile multiply it, and only
// where the window's edge, the diagonal, the last first token or the end of the sample crosses a wave's 32 rows are
// elements masked.  Rows behind a sample's length read as zero.
//
// v_mfma_f32_32x32 leaves lane l with column l % 32 of the result and 16 of its rows.  Every score product is arranged so that what a
// lane holds of it is, without any exchange between lanes, an operand of the next product: the 8 contraction slots that a lane
// feeds into a step of 16 are accumulator registers 8c .. 8c + 7, score rows 16c + {0..3, 8..11} + 4 (l / 32), and the other operand
// is read from LDS at those rows.
//   forward      S^T = K Q^T              O^T  += V^T P^T
//   backward dQ  S^T = K Q^T, dP^T = V dO^T,  dQ^T += K^T dS^T
//   backward dKV S   = Q K^T, dP   = dO V^T,  dV += P^T dO,  dK += dS^T Q
// P and dS enter the second products in the storage type, as operands of the matrix cores; all sums are fp32.  In bf16 the output is
// then off by up to 0.0023 (l2-relative), the gradients by 0.0024 to 0.0025, where rounding nothing but the results costs 0.0017.  For
// rowsum(dO * O) O is read back as it was rounded; where queries see few keys, whose score gradients are small differences, with what the
// rounding took off (o_lo).  Peaked probabilities over many keys still show it: dQ and dK are off by 0.005 with scores spread by 8.
// No atomics: dQ has its own kernel, and sums over a long run of queries that are split over workgroups meet in a fixed order.
//
// What bounds it.  Long rows: matrix cores and vector unit (exponentials, masks, conversions) of a SIMD's two waves are busy half of the
// time each, and the clock falls under the load.  1 x 16384, window 4096, causal, 16 heads of 128 over 2, bf16: forward 572 us
// (0.84 PFLOP/s of visible pairs, matrix cores busy 52 %), dQ 731 - 744 (0.98, 59 %), dK and dV 1036 - 1104 (0.9, 55 %), joining 12.  Heads of
// 64: twice the vector work per product, and bank conflicts; 2 x 8192, window 1024, causal, 16 heads over 4: a step of 407 us, 0.71 PFLOP/s
// where heads of 128 reach 0.98, matrix cores busy 34 to 45 %.  Short rows: a wave's chain through a tile, some 2000 cycles, between a
// launch's first loads and last stores; 4 x 512, window 128, 16 heads of 64 over 4: forward 13 - 14 us, dK and dV 20, dQ and the joining 13.
#include <algorithm>

#include "gemm_direct.h"
#include "window_utils.h"

namespace gpp {

typedef __attribute__((ext_vector_type(8))) float f32x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;

constexpr int WIN_ROWS = 128;     // rows that a workgroup owns

// A tile row of DH elements takes RB bytes of LDS, half a bank line, a whole one or two, in chunks of 16 bytes; the 1 KB that a copy
// instruction of a wave fills (RPG rows) is followed by 16 bytes of padding.  Chunk c of row r lies at position c ^ win_swizzle(r)
// of its row.  Both reads are to find their banks free if the LDS serves 16 consecutive lanes together: along rows they read the same chunk
// of 16 consecutive rows (the swizzle spreads the rows of a group over the quarters of a line, the padding moves group after
// group on by a chunk); across rows, the transposing read takes 64 bytes of each of four consecutive rows (each row another
// quarter).  Measured, conflicts are 0 to 4 % of the LDS's active cycles with heads of 128 in bf16 and in fp32, 2 to 20 % with heads of 96,
// and with rows of 128 bytes (heads of 64: 4 x 512 and 2 x 8192 alike) 24 to 40 %: there it serves other lanes together.
// A swizzle alone would do, but one that touches more bits of c costs every read of a row an address of its own.
template <int RB>
__device__ __forceinline__ int win_swizzle(int row) {
  return RB == 128 ? (((row >> 1) & 1) << 2) | (((row >> 2) & 1) << 1) : (RB == 256 ? (row & 3) << 2 : (row & 1) << 3);
}

// (KG: waves that share 32 rows and take 32 rows of a tile each)
template <typename T, int DH, int KG = 1>
struct WinTile {
  static constexpr int ES = sizeof(T), RB = DH * ES <= 128 ? 128 : (DH * ES <= 256 ? 256 : 512), CPR = RB / 16, EPC = 16 / ES;
  static constexpr int KT = RB == 512 && KG == 1 ? 32 : 64;     // rows of a streamed tile (fp32 rows of 512 bytes: two buffers of two tiles are 65 KB)
  static constexpr int GROUP = 1040, RPG = 1024 / RB;
  static constexpr int SUB = KT / 32, BYTES = KT / RPG * GROUP;
  static constexpr int KS = DH / 16, DB = DH / 32;
  static __host__ __device__ constexpr int at(int row) { return row / RPG * GROUP + row % RPG * RB; }
};

// ---- operands ---------------------------------------------------------------------------------------------
template <typename T>
struct WinFrag;
template <>
struct WinFrag<uint16_t> {
  typedef bf16x8 type;
  static __device__ __forceinline__ f32x16 mma(const bf16x8 &a, const bf16x8 &b, const f32x16 &c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ bf16x8 pack(const f32x16 &v, int c) {
    bf16x8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = (bf16_t)v[8 * c + e];
    return r;
  }
  static __device__ __forceinline__ float dot(const bf16x8 &a, const bf16x8 &b, float c) {
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
#pragma unroll
    for (int e = 0; e < 8; e += 2) c = __builtin_amdgcn_fdot2_f32_bf16((bf16x2){a[e], a[e + 1]}, (bf16x2){b[e], b[e + 1]}, c, false);
    return c;
  }
};
template <>
struct WinFrag<float> {
  typedef f32x8 type;
  // (the order of a contraction does not matter: slot e of both lane halves is one step of two)
  static __device__ __forceinline__ f32x16 mma(const f32x8 &a, const f32x8 &b, f32x16 c) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
    return c;
  }
  static __device__ __forceinline__ f32x8 pack(const f32x16 &v, int c) {
    f32x8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = v[8 * c + e];
    return r;
  }
  static __device__ __forceinline__ float dot(const f32x8 &a, const f32x8 &b, float c) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c = fmaf(a[e], b[e], c);
    return c;
  }
};

// operand rows that a wave keeps: lane's row, columns 16 s + 8 (l / 32) .. of step s; columns beyond the head are zero
template <typename T, int DH>
struct WinRows {
  typename WinFrag<T>::type f[DH / 16];
};
template <typename T, int DH>
__device__ __forceinline__ WinRows<T, DH> win_rows(const GPP_G void *base, int64_t row, int64_t ld, int64_t col0, int dh) {
  const int h = (threadIdx.x & 63) >> 5;
  const GPP_G T *p = (const GPP_G T *)base + row * ld + col0;
  constexpr int EPC = 16 / sizeof(T);
  WinRows<T, DH> r;
#pragma unroll
  for (int s = 0; s < DH / 16; ++s) {
    u32x4 part[8 / EPC];
#pragma unroll
    for (int k = 0; k < 8 / EPC; ++k) {
      const int col = 16 * s + 8 * h + k * EPC;
      part[k] = *(const GPP_G u32x4 *)(p + (col < dh ? col : 0));
#pragma unroll
      for (int e = 0; e < 4; ++e) part[k][e] = col < dh ? part[k][e] : 0u;
    }
    __builtin_memcpy(&r.f[s], part, sizeof(part));
  }
  return r;
}
// A lane's addresses inside a tile: of its row's chunks (read along rows) and of its column blocks (read across rows), as far as
// the swizzle makes them differ; everything else about a read is a constant offset.
template <typename T, int DH>
struct WinLane {
  typedef WinTile<T, DH> C;
  static constexpr int NR = C::ES == 2 ? (C::RB == 128 ? C::KS : (C::KS + 1) / 2) : (C::RB == 512 ? 2 : C::KS);
  uint32_t row[NR], col[C::DB];
  // variant and constant offset of step s of a row
  static __device__ __forceinline__ constexpr int variant(int s) { return C::ES == 2 ? (C::RB == 128 ? s : s >> 1) : (C::RB == 512 ? (s >> 1) & 1 : s); }
  static __device__ __forceinline__ constexpr int offset(int s) {
    return C::ES == 2 ? (C::RB == 128 ? 0 : (s & 1) * 32) : (C::RB == 512 ? (s >> 2) * 256 + (s & 1) * 64 : 0);
  }
};
template <typename T, int DH>
__device__ __forceinline__ WinLane<T, DH> win_lane() {
  typedef WinTile<T, DH> C;
  typedef WinLane<T, DH> L;
  const int l = threadIdx.x & 63, row = l & 31;
  L r;
#pragma unroll
  for (int s = C::KS - 1; s >= 0; --s)      // (of the steps that share a variant the first one's address, without its offset)
    r.row[L::variant(s)] = C::at(row) + ((((16 * s + 8 * (l >> 5)) / C::EPC) ^ win_swizzle<C::RB>(row)) << 4) - L::offset(s);
  const int blk = l >> 4, q = l & 15, cr = 4 * (blk >> 1) + (q >> 2);
#pragma unroll
  for (int d = 0; d < C::DB; ++d) {
    const int col = 32 * d + 16 * (blk & 1) + 4 * (q & 3);
    r.col[d] = C::ES == 2 ? C::at(cr) + (((col >> 3) ^ win_swizzle<C::RB>(cr)) << 4) + (col & 7) * 2 : 0;
  }
#pragma unroll
  for (int k = 0; k < L::NR; ++k) asm("" : "+v"(r.row[k]));      // kept as they are: not formed again at every read
  if constexpr (C::ES == 2) {
#pragma unroll
    for (int d = 0; d < C::DB; ++d) asm("" : "+v"(r.col[d]));
  }
  return r;
}
// lane takes row row0 + l % 32, columns 16 s + 8 (l / 32) .. (row0: a multiple of 32)
template <typename T, int DH>
__device__ __forceinline__ typename WinFrag<T>::type win_row_frag(const WinLane<T, DH> &lane, const unsigned char *tile, int row0, int s) {
  typedef WinTile<T, DH> C;
  typedef WinLane<T, DH> L;
  const unsigned char *p = tile + lane.row[L::variant(s)] + (C::at(row0) + L::offset(s));
  u32x4 part[8 / C::EPC];
#pragma unroll
  for (int k = 0; k < 8 / C::EPC; ++k) part[k] = *(const u32x4 *)(p + 16 * k);
  typename WinFrag<T>::type r;
  __builtin_memcpy(&r, part, sizeof(part));
  return r;
}
// lane takes column 32 d + l % 32 of rows row0 + {0..3, 8..11} + 4 (l / 32) (row0: a multiple of 16)
template <typename T, int DH>
__device__ __forceinline__ typename WinFrag<T>::type win_col_frag(const WinLane<T, DH> &lane, const unsigned char *tile, int row0, int d) {
  typedef WinTile<T, DH> C;
  if constexpr (sizeof(T) == 2) {
    typedef __attribute__((address_space(3))) s16x4 lds_v4;
    const unsigned char *p = tile + lane.col[d] + C::at(row0);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4 *)p), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4 *)(p + C::at(8)));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  } else {
    const int l = threadIdx.x & 63, col = 32 * d + (l & 31);
    f32x8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int row = (e & 3) + 8 * (e >> 2) + 4 * (l >> 5);
      r[e] = *(const float *)(tile + C::at(row0) + C::at(row) + (((col >> 2) ^ win_swizzle<C::RB>(row)) << 4) + (col & 3) * 4);
    }
    return r;
  }
}
__device__ __forceinline__ f32x16 win_zero() {
  f32x16 z;
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = 0.0f;
  return z;
}
// row of a 32-row result that register r of this lane holds
__device__ __forceinline__ int win_acc_row(int r) { return 8 * (r >> 2) + 4 * ((threadIdx.x & 63) >> 5) + (r & 3); }

// maximum and sum of a lane and its partner 32 lanes on
__device__ __forceinline__ float win_half_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float win_half_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// ---- copies into LDS -----------------------------------------------------------------------------------------
// where this lane's pieces of a tile lie behind the tile's first row: copy q of wave w of NW fills the KB w * N + q of the tile
template <typename T, int DH, int NW, int KG = 1>
struct WinCopy {
  static constexpr int N = WinTile<T, DH, KG>::KT / WinTile<T, DH>::RPG / NW;
  uint32_t off[N];
};
template <typename T, int DH, int NW, int KG = 1>
__device__ __forceinline__ WinCopy<T, DH, NW, KG> win_copy_offsets(int wave, int64_t ld, int dh) {
  typedef WinTile<T, DH> C;
  const int l = threadIdx.x & 63;
  WinCopy<T, DH, NW, KG> r;
#pragma unroll
  for (int q = 0; q < r.N; ++q) {
    const int row = (wave * r.N + q) * C::RPG + l / C::CPR, c = (l % C::CPR) ^ win_swizzle<C::RB>(row);
    r.off[q] = c * C::EPC < dh ? (uint32_t)(row * ld * C::ES) + c * 16 : OOB_OFFSET;
  }
  return r;
}
__device__ __forceinline__ rsrc4 win_rsrc(const GPP_G void *base, uint32_t bytes) {
  const uint64_t a = (uint64_t)base;
  return (rsrc4){(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)a),
                 (uint32_t)__builtin_amdgcn_readfirstlane((int)((uint32_t)(a >> 32) & 0xffffu)),
                 (uint32_t)__builtin_amdgcn_readfirstlane((int)bytes), 0x00020000u};
}
template <typename T, int DH, int NW, int KG>
__device__ __forceinline__ void win_copy(rsrc4 rs, const WinCopy<T, DH, NW, KG> &o, uint32_t dst, int wave) {
#pragma unroll
  for (int q = 0; q < o.N; ++q) lds_copy16(rs, dst + (wave * o.N + q) * WinTile<T, DH>::GROUP, o.off[q]);
}
// 4 bytes per lane to consecutive LDS words (as lds_copy16)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void lds_copy4(rsrc4 rs, uint32_t dst, uint32_t off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(dst), "v"(off), "s"(rs) : "m0");
}
#pragma clang diagnostic pop
// bytes of a tile's valid rows: rows [first, len) of it, at most KT, dh columns of the last
__device__ __forceinline__ uint32_t win_tile_bytes(int rows, int64_t ld, int dh, int es) {
  return rows <= 0 ? 0u : (uint32_t)(((int64_t)(rows - 1) * ld + dh) * es);
}

// Consecutive workgroups go round the eight XCDs, each with an L2 of its own.  Work is numbered so that `by.d` neighbours share what
// they read (a sample's key / value head): each such run goes to one XCD, runs in turn, so that samples of unequal lengths are spread
// over all of them; runs that are left over are cut into eight contiguous pieces.
__device__ __forceinline__ int win_spread(int idx, int total, const FastDiv &by) {
  const int full = divide(total >> 3, by).q * 8 * (int)by.d;
  if (idx < full) {
    const Quotient run = divide(idx >> 3, by);
    return ((idx & 7) + 8 * run.q) * (int)by.d + run.r;
  }
  idx -= full;
  total -= full;
  const int xcd = idx & 7, per = total >> 3, rem = total & 7;
  return full + xcd * per + min(xcd, rem) + (idx >> 3);
}

// The fields of a record that every kernel needs, asked for in one go: read where they are used, behind branches, they come one
// memory round trip after the other (a third of a microsecond each)
__device__ __forceinline__ void win_fetch(const WindowProb &p) {
  asm volatile("" ::"s"(p.qkv), "s"(p.out), "s"(p.o), "s"(p.dout), "s"(p.lse), "s"(p.delta), "s"(p.lengths), "s"(p.ld_qkv), "s"(p.ld_out), "s"(p.window),
               "s"(p.sinks), "s"(p.heads), "s"(p.kv_heads), "s"(p.seq), "s"(p.dh), "s"(p.causal), "s"(p.scale), "s"(p.ext_out), "s"(p.query_units),
               "s"(p.units), "s"(p.whole), "s"(p.o_lo), "s"(p.ld_lo), "s"(p.by_group.m), "s"(p.by_kv_heads.m), "s"(p.by_key_blocks.m));
}

// Visible rows of a 32-row result as bits, shifted so that register r of the lane has bit 8 (r / 4) + r % 4; and a value kept where the
// bit is set (two instructions an element, where comparing every row with its bounds takes five)
__device__ __forceinline__ uint32_t win_low_bits(int n) { return (uint32_t)((1ull << min(max(n, 0), 32)) - 1); }
__device__ __forceinline__ uint32_t win_bits(int first, int end, int sinks) {
  return ((win_low_bits(end) & ~win_low_bits(first)) | win_low_bits(sinks)) >> (4 * ((threadIdx.x & 63) >> 5));
}
__device__ __forceinline__ float win_keep_bit(float v, uint32_t bits, int r, float hidden) {
  uint32_t t = (uint32_t)((int32_t)(bits << (31 - (8 * (r >> 2) + (r & 3)))) >> 31);
  asm("" : "+v"(t));      // (taken for a condition, it becomes a comparison and a choice: four instructions)
  return __uint_as_float((__float_as_uint(v) & t) | (__float_as_uint(hidden) & ~t));
}

// ---- which tiles of keys a block of queries streams -------------------------------------------------------------------
struct WinRange {
  int n, sinks, first;      // tiles: [0, sinks) and then [first, first + n - sinks)
  __device__ __forceinline__ int tile(int t) const { return t < sinks ? t : first + t - sinks; }
};
template <int KT>
__device__ __forceinline__ WinRange win_range(const WindowProb &p, int q0, int q1, int len) {
  WinRange r = {0, 0, 0};
  if (q0 >= len) return r;
  const WindowKeys a = window_keys(p, q0, len), b = window_keys(p, q1, len);
  r.first = a.first / KT;
  r.sinks = min((b.sink_end + KT - 1) / KT, r.first);
  r.n = r.sinks + (b.end - 1) / KT - r.first + 1;
  return r;
}
// The tiles of K and V of a block of queries one after the other, each pair to LDS byte `dst`
template <typename T, int DH, int KG>
struct WinKeyStream {
  typedef WinTile<T, DH, KG> C;
  const GPP_G T *k;             // the next tile of keys
  int64_t ld, step, v;          // row stride; elements from tile to tile, from K to V
  int sinks, rows;              // tiles until the jump to the window; rows of the sample from the next tile on
  int jump;                     // rows that the jump skips
  uint32_t whole, tail;         // bytes of a whole tile, of the sample's last one
  __device__ __forceinline__ WinKeyStream(const GPP_G T *kbase, int64_t to_v, int64_t ld_, int dh, const WinRange &r, int len) {
    ld = ld_;
    v = to_v;
    step = C::KT * ld;
    const int first = r.sinks > 0 ? 0 : r.first * C::KT;
    k = kbase + first * ld;
    rows = len - first;
    sinks = r.sinks > 0 ? r.sinks : -1;
    jump = (r.first - r.sinks) * C::KT;
    whole = win_tile_bytes(C::KT, ld, dh, C::ES);
    tail = win_tile_bytes((len - 1) % C::KT + 1, ld, dh, C::ES);
  }
  template <int NW>
  __device__ __forceinline__ void copy(const WinCopy<T, DH, NW, KG> &co, uint32_t dst, int wave) {
    const uint32_t bytes = rows >= C::KT ? whole : tail;
    rsrc4 rk = win_rsrc(k, bytes), rv = win_rsrc(k + v, bytes);
    settle(rk, rv);
    win_copy(rk, co, dst, wave);
    win_copy(rv, co, dst + C::BYTES, wave);
    k += step;
    rows -= C::KT;
    if (--sinks == 0) {
      k += jump * ld;
      rows -= jump;
    }
  }
};
// what of a tile of keys a wave's queries [q0, q1] see: nothing, all of it, or some
enum { WIN_NONE, WIN_ALL, WIN_SOME };
struct WinWave {
  int first0, first1, end0, end1, sink0, sink1;      // of the first and the last query
  bool active;
  __device__ __forceinline__ int sees(int k0, int kt) const {
    if (!active || !((k0 < end1 && k0 + kt > first0) || k0 < sink1)) return WIN_NONE;
    return (k0 >= first1 && k0 + kt <= end0) || k0 + kt <= sink0 ? WIN_ALL : WIN_SOME;
  }
};
__device__ __forceinline__ WinWave win_wave(const WindowProb &p, int q0, int len) {
  WinWave w;
  w.active = q0 < len;
  const WindowKeys a = window_keys(p, min(q0, len - 1), len), b = window_keys(p, min(q0 + 31, len - 1), len);
  w.first0 = a.first;
  w.first1 = b.first;
  w.end0 = a.end;
  w.end1 = b.end;
  w.sink0 = a.sink_end;
  w.sink1 = b.sink_end;
  return w;
}

// block of queries: key / value heads outermost, the query heads that share one innermost: workgroups that run together read the same
// keys.  Where a causal block's work grows with its place, the heavier half comes first, from the heaviest on, and then the lighter one
// from the lightest on: the two blocks that a compute unit gets of one run are as much work wherever it stands (2 x 2048 rows, 16 heads
// of 64: forward 43.5 -> 41.3 us against light and heavy in turn)
struct WinBlock {
  int b, h, g, r0;       // sample, query head, key / value head, first query
  bool first;            // of the query heads that share the key / value head
};
__device__ __forceinline__ WinBlock win_query_block(const WindowProb &p, int blk, int rows) {
  const Quotient hh = divide(blk, p.by_group), k = divide(hh.q, p.by_query_blocks), bg = divide(k.q, p.by_kv_heads);
  WinBlock w;
  w.b = bg.q;
  w.g = bg.r;
  w.h = bg.r * (int)p.by_group.d + hh.r;
  w.first = hh.r == 0;
  const int nb = (int)p.by_query_blocks.d, heavy = (nb + 1) >> 1;
  w.r0 = (p.causal && !p.window ? (k.r < heavy ? nb - 1 - k.r : k.r - heavy) : k.r) * rows;
  return w;
}

// a wave's transposed result (rows: columns of the head, lane: its query) times `mul` of the lane through its own piece of LDS to rows;
// rows at and behind `len` are written as zero.  LOW: what the rounding took off the values, rounded in its turn, to rows in front of len
template <typename T, int DH, bool LOW = false>
__device__ __forceinline__ void win_store_rows(unsigned char *lds, int wave, const f32x16 (&acc)[DH / 32], float mul, int q0, int len, int seq,
                                               int dh, GPP_G void *out, int64_t row0, int64_t ld, GPP_G void *out2, int64_t ld2, int64_t col0) {
  constexpr int ST = DH * (int)sizeof(T) + 16, EPC = 16 / sizeof(T);
  unsigned char *stage = lds + wave * 32 * ST;
  const int l = threadIdx.x & 63;
  if (LOW) seq = len;
#pragma unroll
  for (int d = 0; d < DH / 32; ++d)
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      T v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = acc[d][r + e] * mul;
        if constexpr (sizeof(T) == 2) v[e] = f32_to_bf16_bits(LOW ? x - bf16_bits_to_f32(f32_to_bf16_bits(x)) : x);
        else v[e] = x;
      }
      __builtin_memcpy(stage + (l & 31) * ST + (32 * d + win_acc_row(r)) * sizeof(T), v, sizeof(v));
    }
  __builtin_amdgcn_wave_barrier();
  const int cpr = dh / EPC;
  for (int c = l; c < 32 * (DH / EPC); c += 64) {
    const int row = c / (DH / EPC), k = c % (DH / EPC), q = q0 + row;
    if (k >= cpr || q >= seq) continue;
    u32x4 v = *(const u32x4 *)(stage + row * ST + k * 16);
    if (q >= len) v = (u32x4){0u, 0u, 0u, 0u};
    if (out) *(GPP_G u32x4 *)((GPP_G T *)out + (row0 + q) * ld + col0 + k * EPC) = v;
    if (out2) *(GPP_G u32x4 *)((GPP_G T *)out2 + (row0 + q) * ld2 + col0 + k * EPC) = v;
  }
}

// ROWS rows from w.r0 on of a head's Q, and of K and V where it is the first of those that share them, copied for the backward pass: read
// before the results are put together and written behind them
template <typename T, int DH, int ROWS>
struct WinKeep {
  static constexpr int EPC = 16 / sizeof(T), TPR = DH / EPC <= 8 ? 8 : (DH / EPC <= 16 ? 16 : 32), N = ROWS * TPR / 256;     // threads of a row, rows of a thread
  u32x4 v[3][N];
  template <typename Do>
  __device__ __forceinline__ void each(const WindowProb &p, const WinBlock &w, int64_t row0, const Do &what) {
    const int c = threadIdx.x % TPR * EPC, r = threadIdx.x / TPR;
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      if (k > 0 && !w.first) break;
      const int64_t col = (int64_t)(k == 0 ? w.h : p.heads + (k == 1 ? 0 : p.kv_heads) + w.g) * p.dh + c;
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (c < p.dh && w.r0 + r + i * (256 / TPR) < p.seq) what(v[k][i], row0 + w.r0 + r + i * (256 / TPR), col);
    }
  }
  __device__ __forceinline__ void load(const WindowProb &p, const GPP_G T *qkv, const WinBlock &w, int64_t row0) {
    each(p, w, row0, [&](u32x4 &x, int64_t row, int64_t col) { x = *(const GPP_G u32x4 *)(qkv + row * p.ld_qkv + col); });
  }
  __device__ __forceinline__ void store(const WindowProb &p, const WinBlock &w, int64_t row0) {
    each(p, w, row0, [&](u32x4 &x, int64_t row, int64_t col) { *(GPP_G u32x4 *)((GPP_G T *)p.qkv_keep + row * p.ld_keep + col) = x; });
  }
};

// A wave owns 32 queries.  KG = 1: a wave for every 32.  KG = 2: two waves share their queries and take one half of every tile of keys
// each; for launches of so few blocks that they would leave compute units idle.
template <typename T, int DH, int NW, int KG>
struct WinQueryCfg {
  typedef WinTile<T, DH, KG> C;
  static constexpr int QG = NW / KG, ROWS = 32 * QG;
  static constexpr int NB = C::RB == 128 ? 3 : 2;                                  // buffers: as many as leave room for two workgroups' waves
  static constexpr int CP = 2 * C::KT / C::RPG / NW;                               // copies of a wave per step
  static constexpr int OUT = ROWS * (DH * C::ES + 16), JOIN = KG == 2 ? QG * 32 * (DH + 2) * 4 : 0;
  static constexpr int TILES = 2 * NB * C::BYTES, LDS = TILES > OUT ? (TILES > JOIN ? TILES : JOIN) : (OUT > JOIN ? OUT : JOIN);
};

// What forward and dQ do with their tiles of K and V: a ring of NB buffers; step(K tile, V tile, first key)
template <typename Q, typename Stream, typename Copy, typename Step>
__device__ __forceinline__ void win_stream_keys(const WinRange &tiles, int nt, Stream &stream, const unsigned char *lds, int wave, const Copy &co,
                                                uint32_t lds0, const Step &step) {
  typedef typename Q::C C;
  uint32_t in = 2 * (Q::NB - 1) * C::BYTES, out = 0;       // buffers of the next copy and of this step
  for (int t = 0; t < nt; ++t) {
    if (Q::NB > 2 && t + Q::NB - 1 <= nt) copies_landed_barrier<(Q::NB - 2) * Q::CP>();
    else copies_landed_barrier<0>();
    if (t + Q::NB - 1 < nt) {
      stream.copy(co, lds0 + in, wave);
      in = in == 2 * (Q::NB - 1) * C::BYTES ? 0 : in + 2 * C::BYTES;
    }
    step(lds + out, lds + out + C::BYTES, tiles.tile(t) * C::KT);
    out = out == 2 * (Q::NB - 1) * C::BYTES ? 0 : out + 2 * C::BYTES;
  }
}

// ======================================================================= forward
// A workgroup's queries share the tiles of K and V; the softmax's running maximum and sum are of a lane's query, whose other 16 keys of 32
// the partner lane holds.
// (At two workgroups per compute unit heads of 128 in fp32 do not fit the 256 registers of a wave: forward spills 60 of them, dQ 20; the
// backward launch of both kinds, k_window_bwd_mfma, 6 with heads of 128 in bf16.)
template <typename T, int DH, int KG>
__global__ __launch_bounds__(256, 2) void k_window_fwd_mfma(const WindowProb *__restrict__ probs, int n, ExtPtrs ext, StageFlags *flags) {
  typedef WinTile<T, DH, KG> C;
  typedef WinFrag<T> F;
  typedef WinQueryCfg<T, DH, 4, KG> Q;
  constexpr int ROWS = Q::ROWS;
  __shared__ __attribute__((aligned(16))) unsigned char lds[Q::LDS];
  const int pi = find_prob(probs, n, blockIdx.x);
  const WindowProb p = probs[pi];
  win_fetch(p);
  const WinBlock w = win_query_block(p, win_spread(blockIdx.x - p.blk_begin, p.query_units, p.by_run), ROWS);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), qg = wave % Q::QG, kg = wave / Q::QG;
  const int len = __builtin_amdgcn_readfirstlane(window_length_checked(p, ext, w.b, w.h == 0 && w.r0 == 0 && threadIdx.x == 0, flags));
  const GPP_G T *qkv = (const GPP_G T *)(p.ext_qkv >= 0 ? ext.p[p.ext_qkv] : p.qkv);
  const int64_t row0 = (int64_t)w.b * p.seq;
  const GPP_G T *kbase = qkv + row0 * p.ld_qkv + (int64_t)(p.heads + w.g) * p.dh;
  const int q0 = w.r0 + 32 * qg, q = q0 + (lane & 31), qc = max(0, min(q, len - 1));
  const WinRange tiles = win_range<C::KT>(p, w.r0, min(w.r0 + ROWS, len) - 1, len);
  const WinCopy<T, DH, 4, KG> co = win_copy_offsets<T, DH, 4, KG>(wave, p.ld_qkv, p.dh);
  const uint32_t lds0 = lds_address((const uint16_t *)lds);
  WinKeyStream<T, DH, KG> stream(kbase, (int64_t)p.kv_heads * p.dh, p.ld_qkv, p.dh, tiles, len);
#pragma unroll
  for (int k = 0; k < Q::NB - 1; ++k)
    if (k < tiles.n) stream.copy(co, lds0 + 2 * k * C::BYTES, wave);
  const WinRows<T, DH> qf = win_rows<T, DH>(qkv, row0 + qc, p.ld_qkv, (int64_t)w.h * p.dh, p.dh);
  const WinLane<T, DH> at = win_lane<T, DH>();
  const WinWave mine = win_wave(p, q0, len);
  const WindowKeys keys = window_keys(p, qc, len);
  const float scale2 = p.scale * LOG2E;
  f32x16 o[C::DB];
#pragma unroll
  for (int d = 0; d < C::DB; ++d) o[d] = win_zero();
  float m = -INFINITY, l = 0.0f;     // running maximum (base 2, the same in a lane and its partner) and sum (in fp32 of this lane's share)

  // this wave's keys of a tile, N times 32
  auto part = [&](const unsigned char *tk, const unsigned char *tv, int k0, bool masked) {
    constexpr int N = C::SUB / KG;
    f32x16 st[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      st[i] = win_zero();
#pragma unroll
      for (int s = 0; s < C::KS; ++s) st[i] = F::mma(win_row_frag<T, DH>(at, tk, 32 * i, s), qf.f[s], st[i]);
    }
    if (masked) {
      asm volatile("");      // keeps this a branch
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int j = k0 + 32 * i;
        const uint32_t bits = win_bits(keys.first - j, keys.end - j, keys.sink_end - j);
#pragma unroll
        for (int r = 0; r < 16; ++r) st[i][r] = win_keep_bit(st[i][r], bits, r, -INFINITY);
      }
    }
    float mx = st[0][0];
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, st[i][r]);
    const float m_tile = win_half_max(mx) * scale2;
    // The maximum only keeps the exponentials in range: it follows where it grew by more than 2^8, which spares most tiles the
    // rescaling of the output
    if (__ballot(m_tile > m + 8.0f) != 0ull) {
      const float m_new = fmaxf(m, m_tile), alpha = __builtin_amdgcn_exp2f(m - (m_new == -INFINITY ? 0.0f : m_new));
      l *= alpha;
#pragma unroll
      for (int d = 0; d < C::DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= alpha;
      m = m_new;
    }
    const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        st[i][r] = __builtin_amdgcn_exp2f(fmaf(st[i][r], scale2, -ref));
        l += st[i][r];
      }
#pragma unroll
    for (int c = 0; c < 2 * N; ++c) {
      const typename F::type pf = F::pack(st[c >> 1], c & 1);
#pragma unroll
      for (int d = 0; d < C::DB; ++d) o[d] = F::mma(win_col_frag<T, DH>(at, tv, 16 * c, d), pf, o[d]);
    }
  };
  win_stream_keys<Q>(tiles, tiles.n, stream, lds, wave, co, lds0,
                         [&](const unsigned char *tk, const unsigned char *tv, int k0) {
    constexpr int N = C::SUB / KG;
    const int u = KG == 1 ? 0 : kg, sees = mine.sees(k0 + 32 * u, 32 * N);
    if (sees != WIN_NONE) part(tk + C::at(32) * u, tv + C::at(32) * u, k0 + 32 * u, sees == WIN_SOME);
  });
  WinKeep<T, DH, ROWS> keep;
  if (p.qkv_keep) keep.load(p, qkv, w, row0);
  __syncthreads();
  l = win_half_sum(l);
  if constexpr (KG == 2) {      // the second half's output, sum and maximum to the first half's waves
    float *join = (float *)lds + qg * 32 * (DH + 2) + lane;
    if (kg == 1) {
#pragma unroll
      for (int d = 0; d < C::DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) join[(16 * d + r) * 64] = o[d][r];
      if (lane < 32) {
        join[32 * DH] = m;
        join[32 * DH + 32] = l;
      }
    }
    __syncthreads();
    if (kg == 0) {
      const float m1 = join[32 * DH - (lane & 32)], l1 = join[32 * DH + 32 - (lane & 32)], m_new = fmaxf(m, m1), ref = m_new == -INFINITY ? 0.0f : m_new;
      const float a0 = __builtin_amdgcn_exp2f(m - ref), a1 = __builtin_amdgcn_exp2f(m1 - ref);
#pragma unroll
      for (int d = 0; d < C::DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] = o[d][r] * a0 + join[(16 * d + r) * 64] * a1;
      l = l * a0 + l1 * a1;
      m = m_new;
    }
    __syncthreads();
  }
  if (kg == 0) {
    if (p.lse && lane < 32 && q < len) p.lse[((int64_t)w.b * p.heads + w.h) * p.seq + q] = m + __builtin_amdgcn_logf(l);
    win_store_rows<T, DH>(lds, qg, o, 1.0f / l, q0, len, p.seq, p.dh, p.out, row0, p.ld_out, p.ext_out >= 0 ? (GPP_G void *)ext.p[p.ext_out] : nullptr,
                          p.ld_ext, (int64_t)w.h * p.dh);
    if constexpr (sizeof(T) == 2) {
      if (p.o_lo) {
        __builtin_amdgcn_wave_barrier();
        win_store_rows<T, DH, true>(lds, qg, o, 1.0f / l, q0, len, p.seq, p.dh, p.o_lo, row0, p.ld_lo, nullptr, 0, (int64_t)w.h * p.dh);
      }
    }
  }
  if (p.qkv_keep) keep.store(p, w, row0);
}

// ======================================================================= backward: dQ, and delta = rowsum(dO * O)
// (`local`: block of queries of the record; `lds`: Q::LDS bytes.  DELTA: the deltas are written for the dK / dV kernel behind this one.
// LOW: the record may have a lower half of O)
template <typename T, int DH, int NW, int KG, bool DELTA, bool LOW>
__device__ __forceinline__ void win_dq_body(const WindowProb &p, const ExtPtrs &ext, int local, unsigned char *lds) {
  typedef WinTile<T, DH, KG> C;
  typedef WinFrag<T> F;
  typedef WinQueryCfg<T, DH, NW, KG> Q;
  constexpr int ROWS = Q::ROWS;
  const WinBlock w = win_query_block(p, win_spread(local, p.query_units, p.by_run), ROWS);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), qg = wave % Q::QG, kg = wave / Q::QG;
  const int len = __builtin_amdgcn_readfirstlane(window_length(p, w.b));
  const GPP_G T *qkv = (const GPP_G T *)p.qkv;
  const int64_t row0 = (int64_t)w.b * p.seq;
  const GPP_G T *kbase = qkv + row0 * p.ld_qkv + (int64_t)(p.heads + w.g) * p.dh;
  const int q0 = w.r0 + 32 * qg, q = q0 + (lane & 31), qc = max(0, min(q, len - 1));
  const WinRange tiles = win_range<C::KT>(p, w.r0, min(w.r0 + ROWS, len) - 1, len);
  GPP_G void *dqkv = p.ext_out >= 0 ? (GPP_G void *)ext.p[p.ext_out] : p.out;
  const int nt = dqkv ? tiles.n : 0;
  const WinCopy<T, DH, NW, KG> co = win_copy_offsets<T, DH, NW, KG>(wave, p.ld_qkv, p.dh);
  const uint32_t lds0 = lds_address((const uint16_t *)lds);
  WinKeyStream<T, DH, KG> stream(kbase, (int64_t)p.kv_heads * p.dh, p.ld_qkv, p.dh, tiles, len);
#pragma unroll
  for (int k = 0; k < Q::NB - 1; ++k)
    if (k < nt) stream.copy(co, lds0 + 2 * k * C::BYTES, wave);
  const int64_t stat = ((int64_t)w.b * p.heads + w.h) * p.seq + qc;
  const WinRows<T, DH> qf = win_rows<T, DH>(qkv, row0 + qc, p.ld_qkv, (int64_t)w.h * p.dh, p.dh);
  const WinRows<T, DH> gf = win_rows<T, DH>(p.ext_dout >= 0 ? ext.p[p.ext_dout] : p.dout, row0 + qc, p.ld_dout, (int64_t)w.h * p.dh, p.dh);
  float delta = 0.0f;
  {
    const WinRows<T, DH> of = win_rows<T, DH>(p.o, row0 + qc, p.ld_o, (int64_t)w.h * p.dh, p.dh);
#pragma unroll
    for (int s = 0; s < C::KS; ++s) delta = F::dot(gf.f[s], of.f[s], delta);
    if constexpr (LOW) {
      if (p.o_lo) {
        const WinRows<T, DH> low = win_rows<T, DH>(p.o_lo, row0 + qc, p.ld_lo, (int64_t)w.h * p.dh, p.dh);
#pragma unroll
        for (int s = 0; s < C::KS; ++s) delta = F::dot(gf.f[s], low.f[s], delta);
      }
    }
    delta = win_half_sum(delta);
    if (DELTA && kg == 0 && lane < 32 && q < len) p.delta[stat] = -delta;      // (as the dK / dV kernel takes it)
  }
  const WinLane<T, DH> at = win_lane<T, DH>();
  const WinWave mine = win_wave(p, q0, len);
  WindowKeys keys = window_keys(p, qc, len);
  if (keys.count == 1) keys.end = keys.first = keys.sink_end = 0;      // a single key's probability is constant: no gradient
  const float scale2 = p.scale * LOG2E;
  const float lse = q0 < len ? p.lse[stat] : 0.0f;
  f32x16 dq[C::DB], minus;      // (dP's products are added to -delta)
#pragma unroll
  for (int d = 0; d < C::DB; ++d) dq[d] = win_zero();
#pragma unroll
  for (int r = 0; r < 16; ++r) minus[r] = -delta;

  win_stream_keys<Q>(tiles, nt, stream, lds, wave, co, lds0,
                         [&](const unsigned char *tk, const unsigned char *tv, int k0) {
#pragma unroll
    for (int u = 0; u < C::SUB; ++u) {
      if (KG == 2 && u != kg) continue;
      const int sees = mine.sees(k0 + 32 * u, 32);
      if (sees == WIN_NONE) continue;
      f32x16 st = win_zero(), dp = minus;
#pragma unroll
      for (int s = 0; s < C::KS; ++s) {
        st = F::mma(win_row_frag<T, DH>(at, tk, 32 * u, s), qf.f[s], st);
        dp = F::mma(win_row_frag<T, DH>(at, tv, 32 * u, s), gf.f[s], dp);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) st[r] = __builtin_amdgcn_exp2f(fmaf(st[r], scale2, -lse)) * dp[r];
      if (sees == WIN_SOME) {
        asm volatile("");
        const int j = k0 + 32 * u;
        const uint32_t bits = win_bits(keys.first - j, keys.end - j, keys.sink_end - j);
#pragma unroll
        for (int r = 0; r < 16; ++r) st[r] = win_keep_bit(st[r], bits, r, 0.0f);
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const typename F::type sf = F::pack(st, c);
#pragma unroll
        for (int d = 0; d < C::DB; ++d) dq[d] = F::mma(win_col_frag<T, DH>(at, tk, 32 * u + 16 * c, d), sf, dq[d]);
      }
    }
  });
  if (!dqkv) return;
  __syncthreads();
  if constexpr (KG == 2) {
    float *join = (float *)lds + qg * 32 * (DH + 2) + lane;
    if (kg == 1) {
#pragma unroll
      for (int d = 0; d < C::DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) join[(16 * d + r) * 64] = dq[d][r];
    }
    __syncthreads();
    if (kg == 0) {
#pragma unroll
      for (int d = 0; d < C::DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) dq[d][r] += join[(16 * d + r) * 64];
    }
    __syncthreads();
  }
  if (kg == 0)
    win_store_rows<T, DH>(lds, qg, dq, p.scale, q0, len, p.seq, p.dh, dqkv, row0, p.ld_out, nullptr, 0, (int64_t)w.h * p.dh);
}

// ======================================================================= backward: dK, dV
// The steps of a block of keys are the tiles of queries that see one of them, for every query head that shares the keys, head by
// head.  A block's steps go to one workgroup, or `parts` of at most `part_steps` to several, whose fp32 sums k_window_join adds in
// order.  Units of work: the first `whole` blocks unsplit, the other blocks part by part, then the blocks of the first
// tokens, which every query sees, part by part.
struct WinUnit {
  int b, g, c0, part;        // sample, key / value head, first key, part or -1: unsplit
  int slot;                  // of the parts of the launch
};
__device__ __forceinline__ WinUnit win_unit(const WindowProb &p, int idx) {
  const int rest = p.rest;     // regular blocks behind the whole ones
  WinUnit w;
  w.slot = idx - p.whole;
  w.part = -1;
  Quotient at;      // sample and head, block of keys
  if (idx < p.whole || w.slot < rest * p.parts) {
    Quotient k = {idx, 0};
    if (idx >= p.whole && p.parts > 1) {
      k = divide(w.slot, p.by_parts);
      w.part = k.r;
      k.q += p.whole;
    }
    at = divide(k.q, p.by_key_blocks);
    at.r += p.sink_blocks;
  } else {
    const Quotient k = divide(w.slot - rest * p.parts, p.by_sink_parts);
    if (p.sink_parts > 1) w.part = k.r;
    at = divide(k.q, p.by_sink_blocks);
  }
  const Quotient bg = divide(at.q, p.by_kv_heads);
  w.b = bg.q;
  w.g = bg.r;
  w.c0 = at.r * WIN_ROWS;
  return w;
}
struct WinSteps {
  int t0, nt, n;             // first tile of queries, tiles per head, steps in all
};
template <int KT>
__device__ __forceinline__ WinSteps win_steps(const WindowProb &p, int c0, int len) {
  WinSteps w = {0, 0, 0};
  if (c0 < len) {
    const int first = window_queries(p, c0, len).first;
    const int end = c0 < p.sinks ? len : window_queries(p, min(c0 + WIN_ROWS, len) - 1, len).end;
    w.t0 = first / KT;
    w.nt = (end - 1) / KT - w.t0 + 1;
    w.n = w.nt * (int)p.by_group.d;
  }
  return w;
}

// A wave owns 32 keys and, where a tile holds 64 queries, one half of them: the two waves of a SIMD that share their keys hide each
// other's chains (LDS reads -> score products -> exponentials -> gradient products), and add their sums at the end.  Two waves have 256
// registers each; with heads of more than 64 columns the sums take 128 of them, so V is then read from LDS like the tiles, K stays
// in registers.
// OWN: the deltas are formed here, from a tile of O beside the one of dO, instead of read from the dQ kernel in front of this one.
// LOW: records may have a lower half of O, a fourth tile; where the LDS does not hold one per buffer, there is one, and all
// waves have read it before the next is copied.
template <typename T, int DH, bool OWN, bool LOW = false>
struct WinKeyCfg {
  typedef WinTile<T, DH> C;
  static constexpr int QG = C::SUB, NW = 4 * QG;
  static constexpr bool LOW_ONE = LOW && C::RB > 128;
  static constexpr int STAT = (OWN ? 3 : 2) * C::BYTES + (LOW && !LOW_ONE ? C::BYTES : 0), BUF = STAT + 1024;       // Q, dO (and O), the log-sum-exps and deltas of the tile's queries
  static constexpr bool V_LDS = sizeof(T) == 2 && DH > 64;
  static constexpr int V_BYTES = V_LDS ? WIN_ROWS / C::RPG * C::GROUP : 0, ST = DH * C::ES + 16;
  static constexpr int JOIN = QG > 1 ? NW * 32 * DH * 4 : 0, OUT = NW * 32 * ST;    // over the tiles: a half of every wave's sums, rows of the result
  static constexpr int NB = C::RB == 128 ? 4 : (DH * C::ES > 256 || OWN ? 2 : 3);  // buffers, as many as the LDS of a compute unit's workgroups holds
  static constexpr int CP = (OWN ? 3 : 2) * C::KT / C::RPG / NW;                               // copies of a wave per step, at least
  static constexpr int LOW_AT = LOW_ONE ? NB * BUF + V_BYTES + NW * 128 : 3 * C::BYTES;         // of a buffer, or of all
  static constexpr int TILES = NB * BUF + V_BYTES + (OWN ? NW * 128 : 0) + (LOW_ONE ? C::BYTES : 0), LDS = TILES > JOIN ? (TILES > OUT ? TILES : OUT) : (JOIN > OUT ? JOIN : OUT);
};

template <typename T, int DH, bool OWN, bool LOW = false>
__device__ __forceinline__ void win_dkv_body(const WindowProb &p, const ExtPtrs &ext, int local, unsigned char *lds) {
  typedef WinTile<T, DH> C;
  typedef WinFrag<T> F;
  typedef WinKeyCfg<T, DH, OWN, LOW> K;
  GPP_G void *dqkv = p.ext_out >= 0 ? (GPP_G void *)ext.p[p.ext_out] : p.out;
  if (!dqkv) return;
  // (the unsplit units first, then the others)
  const WinUnit w = win_unit(p, local < p.whole ? win_spread(local, p.whole, p.by_key_blocks) : p.whole + win_spread(local - p.whole, p.units - p.whole, p.by_unit_run));
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), kg = wave & 3, qg = wave >> 2;
  const int len = __builtin_amdgcn_readfirstlane(window_length(p, w.b));
  const WinSteps st_ = win_steps<C::KT>(p, w.c0, len);
  const bool split = w.part >= 0;
  const int s0 = __builtin_amdgcn_readfirstlane(split ? w.part * p.part_steps : 0);
  const int s1 = __builtin_amdgcn_readfirstlane(split ? min(st_.n, s0 + p.part_steps) : st_.n);
  const int nt = __builtin_amdgcn_readfirstlane(st_.nt), t0 = __builtin_amdgcn_readfirstlane(st_.t0);
  if (split && s0 >= s1) return;                // (such a part is not added)
  const GPP_G T *qkv = (const GPP_G T *)p.qkv, *dout = (const GPP_G T *)(p.ext_dout >= 0 ? ext.p[p.ext_dout] : p.dout);
  const int64_t row0 = (int64_t)w.b * p.seq;
  const int h0 = w.g * (int)p.by_group.d;
  const int k0 = w.c0 + 32 * kg, k1 = min(k0 + 31, len - 1), kc = max(0, min(k0 + (lane & 31), len - 1));
  const int64_t kcol = (int64_t)(p.heads + w.g) * p.dh, vcol = kcol + (int64_t)p.kv_heads * p.dh;
  const WinCopy<T, DH, K::NW> cq = win_copy_offsets<T, DH, K::NW>(wave, p.ld_qkv, p.dh), cg = win_copy_offsets<T, DH, K::NW>(wave, p.ld_dout, p.dh);
  const WinCopy<T, DH, K::NW> cw = win_copy_offsets<T, DH, K::NW>(wave, OWN ? p.ld_o : 0, p.dh);      // (O's)
  const WinCopy<T, DH, K::NW> cl = win_copy_offsets<T, DH, K::NW>(wave, LOW ? p.ld_lo : 0, p.dh);
  const uint32_t lds0 = lds_address((const uint16_t *)lds);
  // of the next step to be copied: tile of its head, rows of the sample from there on, Q, dO, and (wave 0, 1) log-sum-exps or deltas
  int head = s0 < s1 ? s0 / nt : 0, tile = s0 - head * nt, rows = len - (t0 + tile) * C::KT;
  const GPP_G T *qn = qkv + (row0 + (t0 + tile) * C::KT) * p.ld_qkv + (int64_t)(h0 + head) * p.dh;
  const GPP_G T *gn = dout + (row0 + (t0 + tile) * C::KT) * p.ld_dout + (int64_t)(h0 + head) * p.dh;
  const GPP_G T *on = OWN ? (const GPP_G T *)p.o + (row0 + (t0 + tile) * C::KT) * p.ld_o + (int64_t)(h0 + head) * p.dh : nullptr;
  const GPP_G T *ln = LOW && p.o_lo ? (const GPP_G T *)p.o_lo + (row0 + (t0 + tile) * C::KT) * p.ld_lo + (int64_t)(h0 + head) * p.dh : nullptr;
  const GPP_G float *sn = (wave == 0 ? p.lse : p.delta) + ((int64_t)w.b * p.heads + h0 + head) * p.seq + (t0 + tile) * C::KT;
  const int64_t q_step = C::KT * p.ld_qkv, g_step = C::KT * p.ld_dout;
  const uint32_t q_whole = win_tile_bytes(C::KT, p.ld_qkv, p.dh, C::ES), q_tail = win_tile_bytes((len - 1) % C::KT + 1, p.ld_qkv, p.dh, C::ES);
  const int64_t o_step = C::KT * p.ld_o, l_step = C::KT * p.ld_lo;
  const uint32_t l_whole = win_tile_bytes(C::KT, p.ld_lo, p.dh, C::ES), l_tail = win_tile_bytes((len - 1) % C::KT + 1, p.ld_lo, p.dh, C::ES);
  const uint32_t o_whole = win_tile_bytes(C::KT, p.ld_o, p.dh, C::ES), o_tail = win_tile_bytes((len - 1) % C::KT + 1, p.ld_o, p.dh, C::ES);
  const uint32_t g_whole = win_tile_bytes(C::KT, p.ld_dout, p.dh, C::ES), g_tail = win_tile_bytes((len - 1) % C::KT + 1, p.ld_dout, p.dh, C::ES);
  auto copy_next = [&](int buf) {
    const bool full = rows >= C::KT;
    rsrc4 rq = win_rsrc(qn, full ? q_whole : q_tail), rg = win_rsrc(gn, full ? g_whole : g_tail);
    settle(rq, rg);
    win_copy(rq, cq, lds0 + buf * K::BUF, wave);
    win_copy(rg, cg, lds0 + buf * K::BUF + C::BYTES, wave);
    if constexpr (OWN) {
      rsrc4 ro = win_rsrc(on, full ? o_whole : o_tail), same = ro;
      settle(ro, same);
      win_copy(ro, cw, lds0 + buf * K::BUF + 2 * C::BYTES, wave);
      on += o_step;
    }
    if constexpr (LOW) {
      if (p.o_lo) {
        rsrc4 rl = win_rsrc(ln, full ? l_whole : l_tail), same = rl;
        settle(rl, same);
        win_copy(rl, cl, lds0 + (K::LOW_ONE ? 0 : buf * K::BUF) + K::LOW_AT, wave);
        ln += l_step;
      }
    }
    if (wave < (OWN ? 1 : 2)) {      // (queries behind the end: zero, as their rows)
      rsrc4 rs = win_rsrc(sn, (uint32_t)min(rows, C::KT) * 4), same = rs;
      settle(rs, same);
      lds_copy4(rs, lds0 + buf * K::BUF + K::STAT + wave * 512, lane * 4);
    }
    qn += q_step;
    gn += g_step;
    sn += C::KT;
    rows -= C::KT;
    if (++tile == nt) {      // the next head's first tile
      tile = 0;
      qn += p.dh - nt * q_step;
      gn += p.dh - nt * g_step;
      if (OWN) on += p.dh - nt * o_step;
      if (LOW) ln += p.dh - nt * l_step;
      sn += p.seq - nt * C::KT;
      rows += nt * C::KT;
    }
  };
  int now = tile;       // of the step that is being multiplied
  if constexpr (K::V_LDS) {
    if (s0 < s1) {      // 128 rows of V: two tiles' worth
      const WinCopy<T, DH, K::NW> cv = win_copy_offsets<T, DH, K::NW>(wave, p.ld_qkv, p.dh);
#pragma unroll
      for (int half = 0; half < WIN_ROWS / C::KT; ++half) {
        const int r0 = w.c0 + half * C::KT;
        rsrc4 rv = win_rsrc(qkv + (row0 + min(r0, len - 1)) * p.ld_qkv + vcol, win_tile_bytes(min(C::KT, len - r0), p.ld_qkv, p.dh, C::ES)), same = rv;
        settle(rv, same);
        win_copy(rv, cv, lds0 + K::NB * K::BUF + half * C::BYTES, wave);
      }
    }
  }
#pragma unroll
  for (int k = 0; k < K::NB - 1; ++k)
    if (s0 + k < s1) copy_next(k);
  const WindowQueries seen = window_queries(p, kc, len);
  const int win = (int)min(p.window ? p.window : (int64_t)p.seq, (int64_t)p.seq), nsink = (int)min(p.sinks, (int64_t)p.seq);
  // queries that see one key only have no gradient of their score: all of them, or the first
  const bool all_single = (win == 1 && nsink == 0) || len == 1, first_single = p.causal || (win == 1 && min(nsink, len) <= 1);
  const float scale2 = p.scale * LOG2E;
  // queries that see one of this wave's keys, and those that see all of them
  const int kl = max(0, k1);
  const int any_first = window_queries(p, min(k0, kl), len).first, any_end = k0 < len ? (k0 < nsink ? len : window_queries(p, kl, len).end) : 0;
  const int all_first = window_queries(p, kl, len).first, all_end = window_queries(p, k0 < nsink && nsink <= kl ? nsink : min(k0, kl), len).end;
  const WinLane<T, DH> at = win_lane<T, DH>();
  const WinRows<T, DH> kf = win_rows<T, DH>(qkv, row0 + kc, p.ld_qkv, kcol, p.dh);
  WinRows<T, DH> vf;
  if constexpr (!K::V_LDS) vf = win_rows<T, DH>(qkv, row0 + kc, p.ld_qkv, vcol, p.dh);
  f32x16 dk[C::DB], dv[C::DB];
#pragma unroll
  for (int d = 0; d < C::DB; ++d) dk[d] = dv[d] = win_zero();

  int in = K::NB - 1, out = 0;       // buffers of the next copy and of this step
  for (int s = s0; s < s1; ++s) {
    if (s + K::NB - 1 <= s1) copies_landed_barrier<(K::NB - 2) * K::CP>();
    else copies_landed_barrier<0>();
    const unsigned char *tq = lds + out * K::BUF, *tg = tq + C::BYTES;
    float own = 0.0f;
    if constexpr (LOW) {
      const unsigned char *low = K::LOW_ONE ? lds + K::LOW_AT : tq + K::LOW_AT;
      if (p.o_lo) {
#pragma unroll
        for (int x = 0; x < C::KS; ++x)
          own = F::dot(win_row_frag<T, DH>(at, tg + C::at(32) * qg, 0, x), win_row_frag<T, DH>(at, low + C::at(32) * qg, 0, x), own);
        if (K::LOW_ONE) __syncthreads();      // read by all: the next tile may come
      }
    }
    if (s + K::NB - 1 < s1) {
      copy_next(in);
      in = in + 1 == K::NB ? 0 : in + 1;
    }
    out = out + 1 == K::NB ? 0 : out + 1;
    const int i0 = (t0 + now) * C::KT + 32 * qg;
    now = now + 1 == nt ? 0 : now + 1;
    if (i0 >= any_end || i0 + 32 <= any_first) continue;
    const bool all = i0 >= all_first && min(i0 + 32, len) <= all_end;
    const float *tl = (const float *)(tq + K::STAT) + 32 * qg + 4 * (lane >> 5), *td = tl + 128;
    f32x16 st = win_zero(), dp = win_zero();
    if constexpr (!OWN) {      // dP - delta: the products are added to -delta
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const f32x4 minus = *(const f32x4 *)(td + 8 * k);
#pragma unroll
        for (int e = 0; e < 4; ++e) dp[4 * k + e] = minus[e];
      }
    }
#pragma unroll
    for (int x = 0; x < C::KS; ++x) {
      st = F::mma(win_row_frag<T, DH>(at, tq + C::at(32) * qg, 0, x), kf.f[x], st);
      const typename F::type g = win_row_frag<T, DH>(at, tg + C::at(32) * qg, 0, x);
      if constexpr (K::V_LDS) dp = F::mma(g, win_row_frag<T, DH>(at, lds + K::NB * K::BUF + C::at(32) * kg, 0, x), dp);
      else dp = F::mma(g, vf.f[x], dp);
      if constexpr (OWN) own = F::dot(g, win_row_frag<T, DH>(at, tg + C::BYTES + C::at(32) * qg, 0, x), own);
    }
    if constexpr (OWN) {       // of the lane's row; through a piece of LDS of the wave's own to the rows that the lane holds of the product
      float *mine = (float *)(lds + K::NB * K::BUF + K::V_BYTES) + 32 * wave;
      own = win_half_sum(own);
      if (lane < 32) mine[lane] = own;
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const f32x4 delta = *(const f32x4 *)(mine + 4 * (lane >> 5) + 8 * k);
#pragma unroll
        for (int e = 0; e < 4; ++e) dp[4 * k + e] -= delta[e];
      }
      __builtin_amdgcn_wave_barrier();
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const f32x4 lse = *(const f32x4 *)(tl + 8 * k);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = 4 * k + e;
        st[r] = __builtin_amdgcn_exp2f(fmaf(st[r], scale2, -lse[e]));
        dp[r] *= st[r];
      }
    }
    if (!all) {
      asm volatile("");      // keeps this a branch
      const uint32_t bits = win_bits(seen.first - i0, seen.end - i0, 0);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        st[r] = win_keep_bit(st[r], bits, r, 0.0f);
        dp[r] = win_keep_bit(dp[r], bits, r, 0.0f);
      }
      if (i0 == 0 && first_single && lane < 32) dp[0] = 0.0f;
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const typename F::type pf = F::pack(st, c), sf = F::pack(dp, c);
#pragma unroll
      for (int d = 0; d < C::DB; ++d) {
        dv[d] = F::mma(pf, win_col_frag<T, DH>(at, tg + C::at(32) * qg, 16 * c, d), dv[d]);
        dk[d] = F::mma(sf, win_col_frag<T, DH>(at, tq + C::at(32) * qg, 16 * c, d), dk[d]);
      }
    }
  }
  __syncthreads();
  // the waves that share keys give each other a half of the sums: the first takes dK, the second dV
  if constexpr (K::QG > 1) {
    float *sums = (float *)lds + kg * 32 * DH + lane, *theirs = sums + (1 - qg) * 4 * 32 * DH;
    sums += qg * 4 * 32 * DH;
#pragma unroll
    for (int d = 0; d < C::DB; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) sums[(d * 16 + r) * 64] = qg ? dk[d][r] : dv[d][r];
    __syncthreads();
#pragma unroll
    for (int d = 0; d < C::DB; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) dk[d][r] = (qg ? dv[d][r] : dk[d][r]) + theirs[(d * 16 + r) * 64];
    __syncthreads();
  }
  const float mk = all_single ? 0.0f : p.scale;
  unsigned char *stage = lds + wave * 32 * K::ST;
#pragma unroll
  for (int k = 0; k < 2 / K::QG; ++k) {
    const int which = K::QG > 1 ? qg : k;         // dK or dV
    f32x16(&acc)[C::DB] = K::QG > 1 || k == 0 ? dk : dv;
    const float mul = which ? 1.0f : mk;
    if (split) {     // [part of the launch][dK, dV][key][column] in fp32
      GPP_G float *part = p.partial + ((int64_t)w.slot * 2 + which) * WIN_ROWS * DH + (int64_t)(32 * kg) * DH + (lane & 31);
#pragma unroll
      for (int d = 0; d < C::DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) part[win_acc_row(r) * DH + 32 * d] = acc[d][r] * mul;
      continue;
    }
    // a wave turns its block of 32 keys in its own piece of LDS and writes whole pieces of rows
#pragma unroll
    for (int d = 0; d < C::DB; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        T *to = (T *)(stage + win_acc_row(r) * K::ST) + 32 * d + (lane & 31);
        if constexpr (sizeof(T) == 2) *to = f32_to_bf16_bits(acc[d][r] * mul);
        else *to = acc[d][r] * mul;
      }
    __builtin_amdgcn_wave_barrier();
    for (int c = lane; c < 32 * (DH / C::EPC); c += 64) {
      const int row = c / (DH / C::EPC), x = c % (DH / C::EPC);
      if (x * C::EPC >= p.dh || k0 + row >= p.seq) continue;
      u32x4 v = *(const u32x4 *)(stage + row * K::ST + x * 16);
      if (k0 + row >= len) v = (u32x4){0u, 0u, 0u, 0u};
      *(GPP_G u32x4 *)((GPP_G T *)dqkv + (row0 + k0 + row) * p.ld_out + (which ? vcol : kcol) + x * C::EPC) = v;
    }
    __builtin_amdgcn_wave_barrier();
  }
}

template <typename T, int DH>
__global__ __launch_bounds__((WinKeyCfg<T, DH, false>::NW * 64), (DH * sizeof(T) <= 256 ? 2 : 1)) void k_window_dkv_mfma(const WindowProb *__restrict__ probs,
                                                                                                              int n, ExtPtrs ext) {
  __shared__ __attribute__((aligned(16))) unsigned char lds[WinKeyCfg<T, DH, false>::LDS];
  const int pi = find_prob(probs, n, blockIdx.x);
  const WindowProb p = probs[pi];
  win_fetch(p);
  win_dkv_body<T, DH, false>(p, ext, blockIdx.x - p.blk_begin, lds);
}

// Small problems: dK / dV and dQ side by side in one launch, first the blocks of keys, then those of queries.  A launch of few
// workgroups is as long as the chain of one of them, and together they still find a compute unit each.
template <typename T, int DH, bool LOW>
__global__ __launch_bounds__((WinKeyCfg<T, DH, true>::NW * 64), (DH * sizeof(T) <= 256 ? 2 : 1)) void k_window_bwd_mfma(const WindowProb *__restrict__ probs,
                                                                                                             int n, ExtPtrs ext) {
  typedef WinKeyCfg<T, DH, true, LOW> K;
  typedef WinQueryCfg<T, DH, K::NW, 2> Q;
  __shared__ __attribute__((aligned(16))) unsigned char lds[K::LDS > Q::LDS ? K::LDS : Q::LDS];
  const int pi = find_prob(probs, n, blockIdx.x);
  const WindowProb p = probs[pi];
  win_fetch(p);
  const int local = blockIdx.x - p.blk_begin;
  if (local < p.units) win_dkv_body<T, DH, true, LOW>(p, ext, local, lds);
  else win_dq_body<T, DH, K::NW, 2, false, LOW>(p, ext, local - p.units, lds);
}

// The sums of a split block's parts, in order: four columns of a key per thread, DH / 4 workgroups per block (bound by memory; 12 us for
// 1 x 16384, window 4096, 2 key / value heads of 128: a few MB, most of it a launch and one trip to memory)
template <typename T, int DH>
__device__ __forceinline__ void win_join_body(const WindowProb &p, const ExtPtrs &ext, int local) {
  typedef WinTile<T, DH> C;
  GPP_G T *dqkv = (GPP_G T *)(p.ext_out >= 0 ? ext.p[p.ext_out] : p.out);
  if (!dqkv) return;
  const int rest = p.rest;
  const int regular = p.parts > 1 ? rest : 0;                     // split blocks that hold no first token
  const int blk = local / (DH / 4), piece = local % (DH / 4);
  const WinUnit w = win_unit(p, p.whole + (blk < regular ? blk * p.parts : rest * p.parts + (blk - regular) * p.sink_parts));
  const int first = w.slot, len = window_length(p, w.b);
  const int parts = (win_steps<C::KT>(p, w.c0, len).n + p.part_steps - 1) / p.part_steps;
  const int64_t row0 = (int64_t)w.b * p.seq, kcol = (int64_t)(p.heads + w.g) * p.dh, vcol = kcol + (int64_t)p.kv_heads * p.dh;
  const int u = piece * 256 + threadIdx.x, c = u % (DH / 4) * 4, row = u / (DH / 4) % WIN_ROWS, which = u / (DH / 4) / WIN_ROWS, key = w.c0 + row;
  if (key >= p.seq || c >= p.dh) return;
  f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
  if (key < len) {
    const GPP_G float *at = p.partial + ((int64_t)first * 2 + which) * WIN_ROWS * DH + (int64_t)row * DH + c;
#pragma unroll 8
    for (int k = 0; k < parts; ++k) sum += *(const GPP_G f32x4 *)(at + (int64_t)k * 2 * WIN_ROWS * DH);
  }
  T v[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (sizeof(T) == 2) v[e] = f32_to_bf16_bits(sum[e]);
    else v[e] = sum[e];
  }
  GPP_G T *to = dqkv + (row0 + key) * p.ld_out + (which ? vcol : kcol) + c;
  if constexpr (sizeof(T) == 2) {
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    u32x2 w2;
    __builtin_memcpy(&w2, v, 8);
    *(GPP_G u32x2 *)to = w2;
  } else {
    u32x4 w4;
    __builtin_memcpy(&w4, v, 16);
    *(GPP_G u32x4 *)to = w4;
  }
}

template <typename T, int DH>
__global__ __launch_bounds__(256) void k_window_join(const WindowProb *__restrict__ probs, int n, ExtPtrs ext) {
  const int pi = find_prob(probs, n, blockIdx.x);
  const WindowProb p = probs[pi];
  win_join_body<T, DH>(p, ext, blockIdx.x - p.blk_begin);
}

// (and, where dK and dV went first, the joining of their parts)
template <typename T, int DH, int KG>
__global__ __launch_bounds__(256, 2) void k_window_dq_mfma(const WindowProb *__restrict__ probs, int n, ExtPtrs ext) {
  __shared__ __attribute__((aligned(16))) unsigned char lds[WinQueryCfg<T, DH, 4, KG>::LDS];
  const int pi = find_prob(probs, n, blockIdx.x);
  const WindowProb p = probs[pi];
  win_fetch(p);
  const int local = blockIdx.x - p.blk_begin;
  if (local < p.query_units) win_dq_body<T, DH, 4, KG, true, sizeof(T) == 2>(p, ext, local, lds);
  else win_join_body<T, DH>(p, ext, local - p.query_units);
}

// ---- host ------------------------------------------------------------------------------------------------
// template head dimension of a record, or 0: the row-parallel kernels
int window_mfma_dh(const WindowProb &p) {
  const int es = p.dtype == DT_BF16 ? 2 : 4, epc = 16 / es;
  if (p.dtype == DT_I32 || p.out_dtype != p.dtype || p.dh > 128 || p.dh % epc) return 0;
  if ((p.ld_qkv | p.ld_out | p.ld_o | p.ld_dout | p.ld_ext) % epc) return 0;
  if (((uintptr_t)p.qkv | (uintptr_t)p.out | (uintptr_t)p.o | (uintptr_t)p.dout) & 15) return 0;
  if ((p.ld_qkv | p.ld_o | p.ld_dout) >= (1ll << 22)) return 0;        // a tile's offsets stay far inside 32 bits
  return p.dh <= 32 ? 32 : (p.dh <= 64 ? 64 : (p.dh <= 96 ? 96 : 128));
}
static int window_tile_rows(const WindowProb &p, int dh) { return dh * (p.dtype == DT_BF16 ? 2 : 4) > 256 ? 32 : 64; }
// Two waves per 32 queries where the blocks of 128 do not give every compute unit one, in fp32 two, whose products take sixteen times as
// long.  Step of 2 samples, bf16, heads of 64, window 128 / all earlier keys: 256 blocks 52 -> 48 / 88 -> 77 us, 512 blocks 70 -> 74 /
// 171 -> 161; heads of 128, window 256: 256 blocks 85 -> 82, 512 blocks 99 -> 112; fp32: 128 blocks 75 -> 63, 512 blocks 182 -> 175.
// In fp32 with heads of more than 64 columns two waves take a compute unit's whole LDS for their tiles of 64 keys: 1 x 2000 causal, heads of
// 128, 128 blocks 874 -> 612, heads of 96, 192 blocks 467 -> 378, 256 blocks 202 -> 220.
int window_key_groups(const WindowProb &p, int dh, int64_t blocks) {
  return blocks <= (p.dtype == DT_BF16 ? 256 : window_tile_rows(p, dh) == 64 ? 512 : 192) ? 2 : 1;
}
// whether the backward pass is one launch: its workgroups, one per compute unit, all run at once
bool window_one_backward(int64_t workgroups) { return workgroups <= 256; }
int window_one_rows(const WindowProb &p, int dh) { return window_tile_rows(p, dh) == 64 ? 128 : 64; }      // queries of a workgroup: 8 waves or 4, two for 32
// The same where blocks of keys, none of them split, leave half of the compute units to the blocks of queries (fewer steps than parts
// are made of: short samples, heads that share keys).  Step of 8 samples of 128 in bf16, 32 heads over 8: heads of 64 33.9 -> 27.9 us,
// of 128 51.1 -> 42.1, over 16 30.2 -> 26.2; as many units as compute units (over 32) 45.7 -> 48.4 with heads of 128; 512 blocks of
// queries 40.8 -> 39.0, 1024 of them 64.7 -> 68.9.
bool window_beside(int64_t query_blocks, int64_t key_units) { return query_blocks <= 512 && key_units <= 128; }
// Whether dK and dV, where they are split, go in front of dQ and form their own deltas: the joining of their parts is then in dQ's launch.
// What the deltas cost grows with the steps and with the rows.  Step of 4 x 512, window 128, bf16, 16 heads over 4, 256 blocks: heads of
// 64 48.1 -> 45.5 us, of 128 69.9 -> 73.8; 2 x 2048, window 512, heads of 64, 512 blocks: 84.7 -> 85.3; fp32 the same either way.
bool window_keys_first(int dtype, int dh, int64_t query_blocks) { return dtype == DT_BF16 && dh <= 64 && query_blocks <= 256; }
void window_plan_queries(WindowProb &p, int rows) {
  p.by_group = fast_div(p.heads / p.kv_heads);
  p.by_kv_heads = fast_div(p.kv_heads);
  p.by_query_blocks = fast_div((p.seq + rows - 1) / rows);
  p.by_run = fast_div((int64_t)p.by_group.d * p.by_query_blocks.d);
  p.query_units = (int32_t)((int64_t)p.batch * p.heads * ((p.seq + rows - 1) / rows));
}

// Cuts the key blocks of a launch (see WinUnit) into units, of which `slots` run at once: the first `whole` blocks stay in one piece,
// the others and the blocks of the first tokens, which take several times as long, go in parts of part_steps steps, which fill the
// gaps that whole blocks leave.  Of the pairs (whole, part_steps) the one with the least estimate, in steps.  Units of one size take
// their rounds; otherwise it is what a slot has to do, but no less than the rounds of whole blocks, plus half a part of unevenness.  A
// unit costs the time of some steps for its operands and its result (4 us: about four steps of 64 x 128 pairs in bf16, half a
// one in fp32), a part its sums' way through memory, the joining launch (5 us) the same for all.
// The sums take 64 MB or twice the gradient's bytes, whichever is more; the estimate alone would have cut 1 x 32768 causal rows of fp32, 4
// heads of 128 over 1, into 1074 MB of them.  In causal launches without a window, whose blocks hold less and less, many small parts only
// evened out that a contiguous eighth of the units went to each XCD.  Runs of one block's parts go round the XCDs instead (win_spread),
// and an odd number of them round the shader engines too (backward of that case: 2 / 4 / 8 parts 58 / 57 / 48 ms, 3 / 5 / 7 parts
// 46.4 / 44.0 / 42.8; contiguous, 32 parts 44.5).  Backward with 5 to 9 parts in bounds and as many as the estimate took without: that
// case 168 MB 44.0 ms, 1074 MB 44.5; bf16 8 heads of 128 over 1 168 MB 9.9 ms, 403 MB 10.7; 1 x 16384, 16 heads over 2 168 MB 4.54 ms,
// 268 MB 5.67; fp32 8 heads over 1 151 MB 23.7 ms, 688 MB 22.4.
// one_round: no more units than slots, if there is such a pair (units = 0: there is none).
void window_plan_parts(WindowProb &p, int dh, int slots, bool one_round) {
  const int64_t kt = window_tile_rows(p, dh), group = p.heads / p.kv_heads, seq = p.seq, nb = (seq + WIN_ROWS - 1) / WIN_ROWS;
  const int64_t win = p.window ? std::min<int64_t>(p.window, seq) : seq, bg = (int64_t)p.batch * p.kv_heads;
  const int64_t sb = p.window ? (std::min<int64_t>(p.sinks, seq) + WIN_ROWS - 1) / WIN_ROWS : 0;
  auto up = [](int64_t v, int64_t by) { return (v + by - 1) / by; };
  auto tiles = [&](int64_t queries) { return std::min<int64_t>(up(std::min(queries, seq), kt) + 1, up(seq, kt)); };
  const int64_t regular = group * tiles(WIN_ROWS - 1 + (p.causal ? win : 2 * win - 1)), every = group * tiles(seq), blocks = bg * (nb - sb);
  const bool triangle = p.causal && !p.window;       // half of the steps of a regular block, on average; the first blocks have most
  const bool wide = p.dtype != DT_BF16;
  const double start = wide ? 0.5 : 4.0, join = wide ? 0.75 : 6.0, sums = (wide ? 0.00005 : 0.00035) * dh;
  const double steps = (double)blocks * regular * (triangle ? 0.5 : 1.0) + (double)(bg * sb * every);
  const int64_t bytes = (int64_t)p.batch * seq * (p.heads + 2 * p.kv_heads) * p.dh * (wide ? 4 : 2), unit_bytes = 2 * WIN_ROWS * dh * 4;
  const int64_t most = std::max<int64_t>(64 << 20, 2 * bytes) / unit_bytes;
  double best = 1e300;
  p.units = 0;
  auto consider = [&](int64_t whole, int64_t part) {
    const int64_t rest = blocks - whole, parts = up(regular, part), sink_parts = sb ? up(every, part) : 1;
    const int64_t split = (parts > 1 ? rest * parts : 0) + (sink_parts > 1 ? bg * sb * sink_parts : 0);
    const int64_t units = whole + rest * parts + bg * sb * sink_parts;
    // (fewer than 2^32 threads in this launch and in the joining one; blocks that are not split always fit)
    if (units >= (1 << 23) || dh / 4 * ((parts > 1 ? rest : 0) + (sink_parts > 1 ? bg * sb : 0)) >= (1 << 23)) return;
    if (split && (units - whole > most || (triangle && parts % 2 == 0 && units > slots))) return;
    const double slot = (steps + start * (double)units) / slots;
    const double longest = std::max(whole ? (double)regular : 0.0, (double)std::min(part, std::max(rest ? regular : 0, sb ? every : 0))) + start;
    double t = std::max(slot, longest);
    if (!triangle && sb == 0 && (whole == 0 || rest == 0)) {
      t = (double)up(units, slots) * ((double)(rest == 0 ? regular : std::min(part, regular)) + start);
    } else if (triangle && whole == 0) {      // parts that hold something, while their rounds are few
      int64_t filled = 0;
      for (int64_t c = 0; c < nb; ++c) filled += up(group * (tiles(seq) - c * WIN_ROWS / kt), part);
      t = bg * filled <= 4 * slots ? (double)up(bg * filled, slots) * ((double)std::min(part, regular) + start) : t + 0.5 * (double)part;
    } else {
      if (!triangle) t = std::max(t, (double)up(whole, slots) * (regular + start));
      if (split) t += 0.5 * (double)part;
    }
    if (split) t += join + sums * (double)split;
    if (t >= best || (one_round && units > slots)) return;
    best = t;
    p.whole = (int32_t)whole;
    p.rest = (int32_t)rest;
    p.part_steps = (int32_t)part;
    p.parts = (int32_t)parts;
    p.sink_parts = (int32_t)sink_parts;
    p.units = (int32_t)units;
  };
  const int64_t least = wide ? 1 : 2;
  for (int64_t whole = blocks;; whole = triangle ? 0 : std::max<int64_t>(0, std::min(whole - 1, whole - slots / 8) / 8 * 8)) {
    for (int64_t k = 1; k <= 64; ++k) {
      consider(whole, std::max(least, up(regular, k)));
      if (sb) consider(whole, std::max(least, up(every, k)));
    }
    for (int64_t part = least; triangle && part <= 256; ++part) consider(whole, part);
    if (whole == 0) break;
  }
  p.sink_blocks = (int32_t)sb;
  p.by_key_blocks = fast_div(nb - sb);
  p.by_parts = fast_div(p.parts);
  p.by_unit_run = fast_div(triangle ? p.parts : nb - sb);
  p.by_sink_parts = fast_div(p.sink_parts);
  p.by_sink_blocks = fast_div(sb);
}
int window_mfma_key_blocks(const WindowProb &p) { return p.units; }
int window_join_blocks(const WindowProb &p, int dh) {
  const int64_t nb = (p.seq + WIN_ROWS - 1) / WIN_ROWS, bg = (int64_t)p.batch * p.kv_heads, sb = p.sink_blocks;
  return (int)(dh / 4 * ((p.parts > 1 ? bg * (nb - sb) - p.whole : 0) + (p.sink_parts > 1 ? bg * sb : 0)));
}
int64_t window_partial_bytes(const WindowProb &p, int dh) {
  return window_join_blocks(p, dh) ? (int64_t)(p.units - p.whole) * 2 * WIN_ROWS * dh * 4 : 0;
}
// workgroups of the dK / dV kernel that run at once: two waves per SIMD have the registers, four with heads of 32 columns in bf16
int window_key_slots(int dtype, int dh) { return dtype == DT_BF16 && dh == 32 ? 512 : 256; }

// GO(T, DH) for a storage type and template head dimension
#define WIN_INSTANCE(GO)                  \
  do {                                    \
    if (dtype == DT_BF16) {               \
      if (dh == 32) GO(uint16_t, 32);     \
      else if (dh == 64) GO(uint16_t, 64);\
      else if (dh == 96) GO(uint16_t, 96);\
      else GO(uint16_t, 128);             \
    } else {                              \
      if (dh == 32) GO(float, 32);        \
      else if (dh == 64) GO(float, 64);   \
      else if (dh == 96) GO(float, 96);   \
      else GO(float, 128);                \
    }                                     \
  } while (0)
#define WIN_QUERY_KERNEL(K, T, DH) (key_groups == 2 ? K<T, DH, 2> : K<T, DH, 1>)

void launch_window_fwd_mfma(const WindowProb *probs, int n, int total_blocks, int dtype, int dh, int key_groups, const ExtPtrs &ext, StageFlags *flags,
                            hipStream_t s) {
  if (total_blocks <= 0) return;
#define GO(T, DH) hipLaunchKernelGGL(WIN_QUERY_KERNEL(k_window_fwd_mfma, T, DH), dim3(total_blocks), dim3(256), 0, s, probs, n, ext, flags)
  WIN_INSTANCE(GO);
#undef GO
}
void launch_window_dq_mfma(const WindowProb *probs, int n, int total_blocks, int dtype, int dh, int key_groups, const ExtPtrs &ext, hipStream_t s) {
  if (total_blocks <= 0) return;
#define GO(T, DH) hipLaunchKernelGGL(WIN_QUERY_KERNEL(k_window_dq_mfma, T, DH), dim3(total_blocks), dim3(256), 0, s, probs, n, ext)
  WIN_INSTANCE(GO);
#undef GO
}
void launch_window_dkv_mfma(const WindowProb *probs, int n, int total_blocks, int dtype, int dh, const ExtPtrs &ext, hipStream_t s) {
  if (total_blocks <= 0) return;
#define GO(T, DH) hipLaunchKernelGGL((k_window_dkv_mfma<T, DH>), dim3(total_blocks), dim3((WinKeyCfg<T, DH, false>::NW * 64)), 0, s, probs, n, ext)
  WIN_INSTANCE(GO);
#undef GO
}
void launch_window_bwd_mfma(const WindowProb *probs, int n, int total_blocks, int dtype, int dh, bool low, const ExtPtrs &ext, hipStream_t s) {
  if (total_blocks <= 0) return;
#define GO(T, DH)                                                                                                         \
  hipLaunchKernelGGL((low ? k_window_bwd_mfma<T, DH, sizeof(T) == 2> : k_window_bwd_mfma<T, DH, false>), dim3(total_blocks), \
                     dim3((WinKeyCfg<T, DH, true>::NW * 64)), 0, s, probs, n, ext)
  WIN_INSTANCE(GO);
#undef GO
}
void launch_window_join(const WindowProb *probs, int n, int total_blocks, int dtype, int dh, const ExtPtrs &ext, hipStream_t s) {
  if (total_blocks <= 0) return;
#define GO(T, DH) hipLaunchKernelGGL((k_window_join<T, DH>), dim3(total_blocks), dim3(256), 0, s, probs, n, ext)
  WIN_INSTANCE(GO);
#undef GO
}

}  // namespace gpp
