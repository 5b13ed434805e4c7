// A tile of a paged cache (nt_cache.h) in the registers of a wave: loads, the rounding of 4-bit codes, the products.
#pragma once
#include "nt_cache.h"
#include "nt_kernels.h"

namespace nt {

// The running maximum of a row changes only where a score exceeds it by more than kSlack (as a logarithm of base 2): weights are up to
// 2^8 then, which no type here minds, and most tiles rescale nothing.
constexpr float kSlack = 8.f;
constexpr float kLeastScale = 1e-30f;  // for a scale of 0: the minus infinity of a key that is not seen stays one
constexpr float kLowest = -1e38f;  // maximum of no score; less than any that is a number

// What a workgroup has to do: the rows of sequence i in row tile rt of `rows` rows, the tiles of keys that one of them sees (those of the sinks, then
// those of the window), and how they are shared out.
struct Share {
  int s, len, m, R;                        // sequence, its length, new tokens, query rows
  long row0;
  int first, p_min, p_max, low;            // positions: of the first new token, of the rows; first key of the earliest window
  int sink_tiles, window_tile, tiles, per, shares;
  bool known;
  __device__ __forceinline__ Share(const CacheAttnArgs &a, int i, int rt, int rows) {
    s = a.r.seq ? a.r.seq[i] : i;
    row0 = a.r.first ? a.r.first[i] : i;
    m = a.r.first ? a.r.first[i + 1] - (int)row0 : 1;
    known = s >= 0 && s < a.c.max_seqs;
    len = known ? a.c.len[s] : 0;
    R = min(m, a.r.max_new) * a.group;
    first = len - m;
    p_min = first + rt * rows / a.group;
    p_max = first + min(rt * rows + rows - 1, R - 1) / a.group;
    low = a.window > 0 ? max(p_min - a.window + 1, 0) : 0;
    sink_tiles = (min(a.sinks, low) + kTile - 1) / kTile;
    window_tile = max(low / kTile, sink_tiles);
    tiles = p_max < 0 ? 0 : sink_tiles + max(p_max / kTile + 1 - window_tile, 0);
    per = max((tiles + a.splits - 1) / a.splits, a.least);
    shares = max((tiles + per - 1) / per, 1);
  }
};

// x of the column eight on (or back): the other of a row's head and tail
__device__ __forceinline__ float eight_on(float x) { return __uint_as_float(wave_dpp<0x128>(__float_as_uint(x))); }

// Head's and tail's sums of values, in the head's column.  Where an infinity is among the values the head's is one, and the tail's
// whatever its sign has made of it.
__device__ __forceinline__ float head_and_tail(float x) {
  const float y = x + eight_on(x);
  return fabsf(x) == __builtin_inff() ? x : y;
}

// x / l, zero where no key was seen
__device__ __forceinline__ void store_row(const CacheAttnArgs &a, const Share &w, int h, int row, int d, int dh, float x, float l) {
  if (row < w.R)
    io_store(a.out, a.out_type, (w.row0 + row / a.group) * a.ld_out + (long)(h * a.group + row % a.group) * dh + d, a.lo_offset, l == 0.f ? 0.f : x / l);
}

template <int KIND> struct FragType { typedef f16x8 type; typedef _Float16 elem; };
template <> struct FragType<CACHE_BF16> { typedef bf16x8 type; typedef __bf16 elem; };

__device__ __forceinline__ f32x4 mma(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
// eight codes as fp16 numbers (exact)
__device__ __forceinline__ void q4_unpack(uint32_t w, f16x2 (&x)[4]) {
  x[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.f, 0);
  x[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.f, 1);
  x[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.f, 2);
  x[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.f, 3);
}
__device__ __forceinline__ f16x8 q4_join(const f16x2 (&x)[4]) {
  f16x8 r;
#pragma unroll
  for (int j = 0; j < 8; j++) r[j] = x[j / 2][j % 2];
  return r;
}
// scale bytes i and j of w as fp16 numbers
template <int I, int J>
__device__ __forceinline__ f16x2 q4_scales(uint32_t w) {
  return __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(w, w, 0x000C000Cu | I << 8 | (uint32_t)J << 24));  // selector 12: a zero byte
}

// Keys of a tile, dims DW part .. DW part + DW - 1 of DH: fragment (t, c), c counted from there, for the first product
template <int KIND, int DH, int DW>
struct KeyTile {
  static constexpr int NC = DW / 32;
  uint4 x[KIND == CACHE_Q4 ? DW / 64 : 2 * NC];
  uint32_t sc[KIND == CACHE_Q4 ? 2 : 1];
  __device__ __forceinline__ void load(const char *tile, int lane, int part) {
    const uint4 *p = (const uint4 *)tile + lane;
    if constexpr (KIND != CACHE_Q4) {
#pragma unroll
      for (int t = 0; t < 2; t++)
#pragma unroll
        for (int c = 0; c < NC; c++) x[t * NC + c] = p[(t * (DH / 32) + part * NC + c) * 64];
    } else {
      static_assert(DW == 64 || DW == 128, "words of a token in one piece, or of both in one");
      const int r = lane & 15, tok = 8 * (r >> 2) + (r & 3);
#pragma unroll
      for (int i = 0; i < DW / 64; i++) x[i] = p[(i * (DH / 128) + part) * 64];
#pragma unroll
      for (int t = 0; t < 2; t++) {
        const char *s = tile + 32 * DH + (tok + 4 * t) * (DH / 32) + part * NC;
        sc[t] = NC == 2 ? *(const unsigned short *)s : *(const uint32_t *)s;
      }
    }
  }
  __device__ __forceinline__ typename FragType<KIND>::type frag(int t, int c) const {
    if constexpr (KIND != CACHE_Q4) {
      return __builtin_bit_cast(typename FragType<KIND>::type, x[t * NC + c]);
    } else {
      const int w = t * NC + c;
      f16x2 v[4];
      q4_unpack(((const uint32_t *)&x[w / 4])[w % 4], v);
      const f16x2 s = c == 0 ? q4_scales<0, 0>(sc[t]) : c == 1 ? q4_scales<1, 1>(sc[t]) : c == 2 ? q4_scales<2, 2>(sc[t]) : q4_scales<3, 3>(sc[t]);
#pragma unroll
      for (int j = 0; j < 4; j++) v[j] *= s;
      return q4_join(v);
    }
  }
};

// Values of a tile, the same dims: fragment n for the second product
template <int KIND, int DH, int DW>
struct ValueTile {
  static constexpr int NV = DW / 16;
  uint4 x[KIND == CACHE_Q4 ? NV / 4 : NV];
  uint2 sc[KIND == CACHE_Q4 ? NV / 2 : 1];
  __device__ __forceinline__ void load(const char *tile, int lane, int part) {
    const uint4 *p = (const uint4 *)(tile + (KIND == CACHE_Q4 ? 16 : 64) * DH) + part * (int)(sizeof(x) / 16) * 64 + lane;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(x) / 16); i++) x[i] = p[i * 64];
    if constexpr (KIND == CACHE_Q4) {
#pragma unroll
      for (int b = 0; b < NV / 2; b++) sc[b] = *(const uint2 *)(tile + 33 * DH + (part * (NV / 2) + b) * kTile + (lane >> 4) * 8);
    }
  }
  // Values of this lane's eight tokens that are no query's become zero, whatever they are: bit j of `keep` stays
  __device__ __forceinline__ void clear(uint32_t keep) {
    uint32_t m[4];
#pragma unroll
    for (int j = 0; j < 4; j++) m[j] = (keep >> (2 * j) & 1 ? 0xFFFFu : 0) | (keep >> (2 * j + 1) & 1 ? 0xFFFF0000u : 0);
    if constexpr (KIND != CACHE_Q4) {
#pragma unroll
      for (int i = 0; i < NV; i++) x[i].x &= m[0], x[i].y &= m[1], x[i].z &= m[2], x[i].w &= m[3];
    } else {  // a zero scale
      const uint32_t lo = (m[0] & 0xFF) | (m[0] >> 8 & 0xFF00) | (m[1] << 16 & 0xFF0000) | (m[1] & 0xFF000000u);
      const uint32_t hi = (m[2] & 0xFF) | (m[2] >> 8 & 0xFF00) | (m[3] << 16 & 0xFF0000) | (m[3] & 0xFF000000u);
#pragma unroll
      for (int b = 0; b < NV / 2; b++) sc[b].x &= lo, sc[b].y &= hi;
    }
  }
  __device__ __forceinline__ typename FragType<KIND>::type frag(int n) const {
    if constexpr (KIND != CACHE_Q4) {
      return __builtin_bit_cast(typename FragType<KIND>::type, x[n]);
    } else {
      f16x2 v[4];
      q4_unpack(((const uint32_t *)&x[n / 4])[n % 4], v);
      v[0] *= q4_scales<0, 1>(sc[n / 2].x);
      v[1] *= q4_scales<2, 3>(sc[n / 2].x);
      v[2] *= q4_scales<0, 1>(sc[n / 2].y);
      v[3] *= q4_scales<2, 3>(sc[n / 2].y);
      return q4_join(v);
    }
  }
};

// exponent bits all set
__device__ __forceinline__ bool no_number(_Float16 x) { return (__builtin_bit_cast(unsigned short, x) & 0x7C00) == 0x7C00; }
__device__ __forceinline__ bool no_number(__bf16 x) { return (__builtin_bit_cast(unsigned short, x) & 0x7F80) == 0x7F80; }
template <class F>
__device__ __forceinline__ bool any_no_number(F v) {
  bool b = false;
#pragma unroll
  for (int j = 0; j < 8; j++) b |= no_number(v[j]);
  return b;
}
// o += V^T P where some values are infinities or NaN, and some queries do not see all keys: bit j of `seen` says whether
// this lane's query sees its token j.  Infinities and NaN count for the queries that see them only, the rest is the product.
template <class F>
__device__ f32x4 mma_seen(F v, F p, uint32_t seen, f32x4 o) {
  F fin = v, up = v, down = v, nan = v, see = v;
#pragma unroll
  for (int j = 0; j < 8; j++) {
    const float x = (float)v[j];
    const bool bad = no_number(v[j]);
    if (bad) fin[j] = 0;
    up[j] = bad && x > 0.f ? 1 : 0;
    down[j] = bad && x < 0.f ? 1 : 0;
    nan[j] = x != x ? 1 : 0;
    see[j] = seen >> j & 1 ? 1 : 0;
  }
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  o = mma(fin, p, o);
  const f32x4 u = mma(up, see, zero), d = mma(down, see, zero), q = mma(nan, see, zero);
#pragma unroll
  for (int i = 0; i < 4; i++) {
    if (u[i] > 0.f) o[i] += __builtin_inff();
    if (d[i] > 0.f) o[i] -= __builtin_inff();
    if (q[i] > 0.f) o[i] = __builtin_nanf("");
  }
  return o;
}

}  // namespace nt
