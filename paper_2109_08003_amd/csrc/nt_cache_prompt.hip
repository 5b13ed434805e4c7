// Attention of many rows over a paged cache: prompts.
//
// A workgroup has a tile of query rows of one key/value head (rows: token, then head of the group) and walks the keys that they
// see, tile by tile: all its waves take part in bringing the next one to the LDS (16-bit tiles as they are, by loads
// that go there directly; 4-bit ones rounded back to fp16 once for all waves) while each computes on the present one for its own
// NQ x 16 rows, with the running maximum and sum of the softmax in registers.  As in the kernel for few rows, scores are S^T = K Q^T
// and weights enter O^T = V^T P^T from the registers they are made in.
//
// Rows of fp16 and bf16 are rounded to the cache's type for the products, weights likewise.  Rows of fp32 (WIDE) keep about twice those
// bits: as in the kernel for few rows, the sixteen columns of an instruction are then eight rows twice, heads and tails.
#include <algorithm>
#include <climits>

#include "nt_cache_frag.h"

namespace nt {
namespace {

constexpr long kFill = 512;  // workgroups that the chip holds at once

// Rows of a wave in tiles of 16, and waves.  Accumulators, queries, scores and weights of a wave are about
// NQ (DH / 4 + DH / 8 + 16) registers, and 256 let two waves share a SIMD; a fragment read from the LDS serves NQ products of 16
// clocks, and four SIMDs can read one in 32.  Two prompts of 6,000 tokens, TFLOP/s: 32 / 8 heads of 64 with NQ 2 / 3 / 4 619 / 645 /
// 594 (but 32 prompts of 1,000 with 8 heads 321 / 311 / 257); of 128, 8,200 tokens, 2 / 3 710 / 950; 16 / 4 of 256 with 2 x 4 / 2 x 8 /
// 1 x 8 877 / 865 / 717, in 4 bits, whose codes on the way take registers of each wave, 432 / 706 / 617; 8 / 2 of 512 with 1 x 8 /
// 1 x 4 690 / 432, in 4 bits 459 / 164.
template <int KIND, int DH> struct PromptShape { static constexpr int NQ = 1, NW = 8; };
template <int KIND> struct PromptShape<KIND, 64> { static constexpr int NQ = 2, NW = 4; };
template <int KIND> struct PromptShape<KIND, 128> { static constexpr int NQ = 3, NW = 4; };
template <int KIND> struct PromptShape<KIND, 256> { static constexpr int NQ = 2, NW = KIND == CACHE_Q4 ? 8 : 4; };

// 0xFFFF in the halves of w that are infinities or NaN: their exponent is all ones, and one more carries into the sign
template <typename E>
__device__ __forceinline__ uint32_t no_numbers(uint32_t w) {
  constexpr uint32_t one = __is_same(E, _Float16) ? 0x04000400u : 0x00800080u;
  const uint32_t b = ((w & 0x7FFF7FFFu) + one) & 0x80008000u;
  return (b << 1) - (b >> 15);
}

template <int KIND, int DH, bool WIDE>
__global__ __launch_bounds__((PromptShape<KIND, DH>::NW * 64), 2) void cache_prompt_kernel(CacheAttnArgs a, int spread) {
  typedef typename FragType<KIND>::type F;
  typedef typename FragType<KIND>::elem E;
  constexpr int NQ = PromptShape<KIND, DH>::NQ, NW = PromptShape<KIND, DH>::NW;
  constexpr int NC = DH / 32, NV = DH / 16, TB = 128 * DH, RT = WIDE ? 8 : 16, ROWS = NW * NQ * RT;
  // Fragments are read from the LDS two ahead of their products, the first values' before the softmax: 128 / 512 wide 934 -> 951 / 704 ->
  // 786 TFLOP/s.  Not where the registers are full (256 wide, 4 bits: 717 -> 304) or waves are many (64 wide, 4 bits: 626 -> 561).
  constexpr bool SOON = !(KIND == CACHE_Q4 && (DH == 64 || DH == 256));
  extern __shared__ __align__(1024) char lds[];  // [2][TB], before that the queries
  const CacheView &c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, g4 = lane >> 4, G = a.group;
  // row tiles of a head's sequence, and their shares, follow one another on one of the eight dies, whose cache they share; long ones
  // first
  const int b = blockIdx.x, j = spread ? b / 8 : b, split = j % a.splits, jt = j / a.splits;
  const int unit = spread ? jt / a.row_tiles * 8 + b % 8 : jt / a.row_tiles, rt = a.row_tiles - 1 - jt % a.row_tiles;
  const int h = unit % c.heads, i = unit / c.heads;
  if (i >= a.r.n) return;
  const Share w(a, i, rt, ROWS);
  const int s = w.s, R = w.R, first = w.first, p_min = w.p_min, p_max = w.p_max, low = w.low;
  const long row0 = w.row0;
  if ((!w.known || w.m < 0 || w.m > a.r.max_new || w.m > w.len) && h == 0 && rt == 0 && split == 0 && tid == 0) atomicOr(c.flags, 1);
  if (rt * ROWS >= R || split >= w.shares) return;
  const int t0 = split * w.per, t1 = min(t0 + w.per, w.tiles);
  auto tile_of = [&](int t) { return t < w.sink_tiles ? t : w.window_tile + t - w.sink_tiles; };

  // queries: rounded to the cache's type in the LDS, in the order in which the waves read them back.  A power of two brings the
  // largest of each to 1 .. 2: no overflow in fp16.
  __shared__ float lds_scale[ROWS];
  __shared__ int lds_strange;  // values that are no numbers were left out
  if (tid == 0) lds_strange = 0;
#pragma unroll 1
  for (int x = tid; x < ROWS * DH / 8; x += NW * 64) {
    const int r = x / (DH / 8), d = x % (DH / 8) * 8, row = rt * ROWS + r, tok = row / G;
    float v[8] = {}, big = 0.f;
    if (row < R) io_load8(a.q, a.type, (row0 + tok) * a.ld_q + (long)(h * G + row % G) * DH + d, a.vec, v);
#pragma unroll
    for (int k = 0; k < 8; k++) big = fmaxf(big, fabsf(v[k]));
#pragma unroll
    for (int k = 1; k < DH / 8; k *= 2) big = fmaxf(big, __shfl_xor(big, k, 64));
    const int ex = big > 0.f && big < __builtin_inff() ? min(max(ilogbf(big), -100), 126) : 0;
    if (d == 0) lds_scale[r] = fmaxf(ldexpf(fabsf(a.scale) * 1.44269504088896f, ex), kLeastScale);
    const float down = ldexpf(a.scale < 0.f ? -1.f : 1.f, -ex);
    F head, tail;
#pragma unroll
    for (int k = 0; k < 8; k++) {
      const float y = as_f32(v[k] * down);
      head[k] = (E)y;
      tail[k] = (E)(y - (float)head[k]);
    }
    F *to = (F *)lds + (r / RT * NC + d / 32) * 64 + d / 8 % 4 * 16 + r % RT;
    to[0] = head;
    if (WIDE) to[8] = tail;
  }
  __syncthreads();
  const int wave_row = rt * ROWS + wave * NQ * RT, own = col & (RT - 1);
  const float tails = col < 8 ? 0.f : 1.f;
  F q[NQ][NC];
  float to_log2[NQ];
  int pos[NQ];
#pragma unroll
  for (int k = 0; k < NQ; k++) {
    const int row = wave_row + k * RT + own;
    pos[k] = row < R ? first + row / G : -1;
    to_log2[k] = lds_scale[row - rt * ROWS];
#pragma unroll
    for (int e = 0; e < NC; e++) q[k][e] = ((const F *)lds)[((wave * NQ + k) * NC + e) * 64 + lane];
  }
  __syncthreads();
  // positions of the wave's rows
  const int w_min = wave_row < R ? first + wave_row / G : 0, w_max = wave_row < R ? first + min(wave_row + NQ * RT - 1, R - 1) / G : -1;
  const int w_low = a.window > 0 ? max(w_min - a.window + 1, 0) : 0;

  const int sub_bits = c.page_shift - 5;
  const int32_t *table = c.table + (long)s * c.width;
  const char *layer = c.pool + a.layer * c.layer_bytes;
  constexpr int kBytes = KIND == CACHE_Q4 ? 34 * DH : TB;
  auto page_of = [&](int t) { return t < t1 ? table[tile_of(t) >> sub_bits] : -1; };
  auto address = [&](int t, int page) {
    return layer + page * c.page_bytes + (long)((h << sub_bits) + (tile_of(t) & ((1 << sub_bits) - 1))) * kBytes;
  };

  // pieces of a 4-bit tile that a wave brings: 16 bytes a lane, four fragments
  constexpr int PIECES = DH / 32, MINE = KIND == CACHE_Q4 ? (PIECES + NW - 1) / NW : 1;
  uint4 code[MINE];
  uint32_t sc[MINE][4];
  auto fetch = [&](int t, int page, int buf) {
    if (page < 0) return;
    const char *at = address(t, page);
    if constexpr (KIND != CACHE_Q4) {
      for (int k = wave; k < TB / 1024; k += NW)
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(at + k * 1024 + lane * 16),
                                         (__attribute__((address_space(3))) void *)(lds + buf * TB + k * 1024), 16, 0, 0);
    } else {
#pragma unroll
      for (int y = 0; y < MINE; y++) {
        const int p = wave + y * NW;
        if (p >= PIECES) continue;
        code[y] = *(const uint4 *)(at + p * 1024 + lane * 16);
        if (p < PIECES / 2) {  // keys: words 4 p .. 4 p + 3
          const int tok = 8 * (col >> 2) + (col & 3);
          const char *scales = at + 32 * DH;
          if constexpr (NC == 2) {
            sc[y][0] = *(const unsigned short *)(scales + tok * NC);
            sc[y][1] = *(const unsigned short *)(scales + (tok + 4) * NC);
          } else {
            const int t = 4 * p / NC;
            sc[y][0] = *(const uint32_t *)(scales + (tok + 4 * t) * NC + 4 * p % NC);
          }
        } else {
          const char *scales = at + 33 * DH + (p - PIECES / 2) * 2 * kTile + g4 * 8;
          const uint2 u = *(const uint2 *)scales, v = *(const uint2 *)(scales + kTile);
          sc[y][0] = u.x, sc[y][1] = u.y, sc[y][2] = v.x, sc[y][3] = v.y;
        }
      }
    }
  };
  auto place = [&](int page, int buf) {  // 4 bits: what fetch left in registers
    if constexpr (KIND == CACHE_Q4) {
      if (page < 0) return;
#pragma unroll
      for (int y = 0; y < MINE; y++) {
        const int p = wave + y * NW;
        if (p >= PIECES) continue;
        char *to = lds + buf * TB + p * 4096 + lane * 16;
#pragma unroll
        for (int w = 0; w < 4; w++) {
          f16x2 v[4];
          q4_unpack(((const uint32_t *)&code[y])[w], v);
          if (p < PIECES / 2) {
            const uint32_t by = NC == 2 ? sc[y][w / 2] >> (8 * (w % 2)) : sc[y][0] >> (8 * w);
            const f16x2 f = q4_scales<0, 0>(by);
#pragma unroll
            for (int d = 0; d < 4; d++) v[d] *= f;
          } else {
#pragma unroll
            for (int d = 0; d < 4; d++) v[d] *= d % 2 ? q4_scales<2, 3>(sc[y][w / 2 * 2 + d / 2]) : q4_scales<0, 1>(sc[y][w / 2 * 2 + d / 2]);
          }
          *(f16x8 *)(to + w * 1024) = q4_join(v);
        }
      }
    }
  };

  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  F ones;
#pragma unroll
  for (int d = 0; d < 8; d++) ones[d] = (E)1.f;
  f32x4 o[NQ][NV];
  float top[NQ];
  f32x4 sum[NQ];  // of the weights as they are multiplied, in every row of a product with ones: a weight's rounding leaves a row of few keys exact
#pragma unroll
  for (int k = 0; k < NQ; k++) {
    top[k] = kLowest;
    sum[k] = zero;
#pragma unroll
    for (int n = 0; n < NV; n++) o[k][n] = zero;
  }

  int page = page_of(t0), next = page_of(t0 + 1);
  fetch(t0, page, 0);
  place(page, 0);
  // whether all rows of the workgroup see all keys of a tile
  auto seen_by_all = [&](int j0) { return j0 + kTile - 1 <= p_min && (a.window == 0 || j0 >= p_max - a.window + 1 || j0 + kTile <= a.sinks); };
  // Where they do not, the values of keys that none sees, and those that are no numbers, become zero in the LDS before the product.
  auto clean = [&](int j0, char *tile) {
    for (int k = tid; k < NV * 64; k += NW * 64) {
      uint4 *at = (uint4 *)(tile + 64 * DH) + k, v = *at;
      uint32_t *w = (uint32_t *)&v, bad = 0;
#pragma unroll
      for (int d = 0; d < 4; d++) {
        const int key = j0 + (k & 63) / 16 * 8 + 2 * d;
        w[d] &= ((key <= p_max) & ((key >= low) | (key < a.sinks)) ? 0xFFFFu : 0) |
                ((key + 1 <= p_max) & ((key + 1 >= low) | (key + 1 < a.sinks)) ? 0xFFFF0000u : 0);
        bad |= no_numbers<E>(w[d]);
        w[d] &= ~no_numbers<E>(w[d]);
      }
      if (bad) lds_strange = 1;
      *at = v;
    }
  };
  __syncthreads();
  for (int t = t0; t < t1; t++) {
    const int buf = (t - t0) & 1, j0 = tile_of(t) * kTile, after = page_of(t + 2);
    fetch(t + 1, next, buf ^ 1);
    if (page >= 0 && !seen_by_all(j0)) {
      clean(j0, lds + buf * TB);
      __syncthreads();
    }
    // unless there is nothing for this wave
    if (page >= 0 && j0 <= w_max && (j0 + kTile > w_low || j0 < a.sinks)) {
      const bool all_seen = j0 + kTile - 1 <= w_min && (a.window == 0 || j0 >= w_max - a.window + 1 || j0 + kTile <= a.sinks);
      const F *keys = (const F *)(lds + buf * TB) + lane, *values = keys + 4 * DH;
      f32x4 y[NQ][2];
#pragma unroll
      for (int k = 0; k < NQ; k++) y[k][0] = y[k][1] = zero;
      F kf[2];
      if (SOON) kf[0] = keys[0], kf[1] = keys[64];
#pragma unroll
      for (int e = 0; e < 2 * NC; e++) {
        const F now = SOON ? kf[e & 1] : keys[e * 64];
        if (SOON && e + 2 < 2 * NC) kf[e & 1] = keys[(e + 2) * 64];
#pragma unroll
        for (int k = 0; k < NQ; k++) y[k][e / NC] = mma(now, q[k][e % NC], y[k][e / NC]);
      }
      F vf[2];
      if (SOON) vf[0] = values[0], vf[1] = values[64];
      if (WIDE) {
#pragma unroll
        for (int k = 0; k < NQ; k++)
#pragma unroll
          for (int d = 0; d < 8; d++) y[k][d / 4][d % 4] += eight_on(y[k][d / 4][d % 4]);
      }
      if (!all_seen) {
#pragma unroll
        for (int k = 0; k < NQ; k++) {
          const int from = a.window > 0 ? pos[k] - a.window + 1 : 0;
#pragma unroll
          for (int d = 0; d < 8; d++) {
            const int key = j0 + g4 * 8 + d;
            y[k][d / 4][d % 4] = (key > pos[k]) | ((key < from) & (key >= a.sinks)) ? -__builtin_inff() : y[k][d / 4][d % 4];
          }
        }
      }
      F p[NQ];
#pragma unroll
      for (int k = 0; k < NQ; k++) {
        float z[8];
        auto weigh = [&]() {
          int big = INT_MIN;
#pragma unroll
          for (int d = 0; d < 8; d++) {
            z[d] = __builtin_fmaf(y[k][d / 4][d % 4], to_log2[k], -top[k]);
            big = max(big, __float_as_int(z[d]));  // of positive numbers the largest
          }
          return big;
        };
        if (__any(weigh() > __float_as_int(kSlack))) {  // some row: those that need it change their maximum, no other row depends on them
          float mx = y[k][0][0];
#pragma unroll
          for (int d = 1; d < 8; d++) mx = fmaxf(mx, y[k][d / 4][d % 4]);
          mx = wave_pair16(mx, mx, WaveMax{});
          mx = wave_pair32(mx, mx, WaveMax{}) * to_log2[k];
          const float up = mx - top[k] > kSlack ? mx : top[k], shrink = __builtin_amdgcn_exp2f(top[k] - up);
          top[k] = up;
          sum[k] *= shrink;
#pragma unroll
          for (int n = 0; n < NV; n++) o[k][n] *= shrink;
          weigh();
        }
#pragma unroll
        for (int d = 0; d < 8; d++) {
          const float x = __builtin_amdgcn_exp2f(z[d]);
          p[k][d] = WIDE ? (E)__builtin_fmaf(-(float)(E)x, tails, x) : (E)x;
        }
      }
#pragma unroll
      for (int k = 0; k < NQ; k++) sum[k] = mma(ones, p[k], sum[k]);
#pragma unroll
      for (int n = 0; n < NV; n++) {
        const F now = SOON ? vf[n & 1] : values[n * 64];
        if (SOON && n + 2 < NV) vf[n & 1] = values[(n + 2) * 64];
#pragma unroll
        for (int k = 0; k < NQ; k++) o[k][n] = mma(now, p[k], o[k][n]);
      }
    }
    place(next, buf ^ 1);
    page = next;
    next = after;
    __syncthreads();
  }
  const long part0 = ((long)((i * a.row_tiles + rt) * c.heads + h) * a.splits + split) * a.part_rows;
#pragma unroll
  for (int k = 0; k < NQ; k++) {
    const int row = wave_row + k * RT + own;
    float l = sum[k][0];
    if (WIDE) {
      l += eight_on(l);
#pragma unroll
      for (int n = 0; n < NV; n++)
#pragma unroll
        for (int d = 0; d < 4; d++) o[k][n][d] = head_and_tail(o[k][n][d]);
      if (col >= 8) continue;
    }
    if (row >= R) continue;
    if (w.shares > 1) {
      const long r = part0 + row - rt * ROWS;
#pragma unroll
      for (int n = 0; n < NV; n++) *(f32x4 *)(a.part + r * DH + n * 16 + g4 * 4) = o[k][n];
      if (g4 == 0) a.part_sums[r] = make_float2(top[k], l);
      continue;
    }
    const long at = (row0 + row / G) * a.ld_out + (long)(h * G + row % G) * DH + g4 * 4;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    auto rows = [&](auto *out) {
      typedef std::remove_pointer_t<decltype(out)> T;
      typedef T T4 __attribute__((ext_vector_type(4)));
      if (a.vec_out) {
#pragma unroll
        for (int n = 0; n < NV; n++) {
          T4 v;
#pragma unroll
          for (int d = 0; d < 4; d++) v[d] = (T)(l == 0.f ? 0.f : o[k][n][d] * inv);
          *(T4 *)(out + at + n * 16) = v;
        }
      } else {
#pragma unroll
        for (int n = 0; n < NV; n++)
#pragma unroll
          for (int d = 0; d < 4; d++) out[at + n * 16 + d] = (T)(l == 0.f ? 0.f : o[k][n][d] * inv);
      }
    };
    if (a.out_type == IO_F32) rows((float *)a.out);
    else if (a.out_type == IO_F16) rows((_Float16 *)a.out);
    else rows((__bf16 *)a.out);
  }
  if (!lds_strange || (WIDE && col >= 8)) return;
  // The infinities and NaN that were left out reach the rows that see them: a lane corrects what it has stored.
  for (int t = t0; t < t1; t++) {
    const int pg = page_of(t), j0 = tile_of(t) * kTile;
    if (pg < 0 || seen_by_all(j0)) continue;
    const char *at = address(t, pg);
    for (int key = 0; key < kTile; key++)
      for (int x = 0; x < DH / 4; x++) {
        const int dim = x / 4 * 16 + g4 * 4 + x % 4;
        float v;
        if constexpr (KIND == CACHE_Q4) {
          v = q4_scale(((const unsigned char *)at)[33 * DH + dim / 32 * kTile + key]);
          if (v == v) continue;
        } else {
          v = (float)((const E *)(at + 64 * DH))[value_elem(key, dim)];
          if (v - v == 0.f) continue;
        }
        for (int k = 0; k < NQ; k++) {
          const int row = wave_row + k * RT + own, p = row < R ? first + row / G : -1;
          if (j0 + key > p || (a.window > 0 && j0 + key < p - a.window + 1 && j0 + key >= a.sinks)) continue;
          if (w.shares > 1) {
            a.part[(part0 + row - rt * ROWS) * DH + dim] += v;
          } else {
            const long o = (row0 + row / G) * a.ld_out + (long)(h * G + row % G) * DH + dim;
            io_store(a.out, a.out_type, o, 0, io_load(a.out, a.out_type, o) + v);
          }
        }
      }
  }
}

template <int KIND, int DH>
struct PromptLaunch {
  static constexpr int kColumns = PromptShape<KIND, DH>::NW * PromptShape<KIND, DH>::NQ * 16, kTiles = 2 * 128 * DH, kQueries = kColumns * DH * 2;
  static constexpr int kLds = kTiles > kQueries ? kTiles : kQueries;  // first the queries, then the tiles
};

template <int KIND, int DH>
hipError_t launch(CacheAttnArgs a, long tiles, hipStream_t s) {
  const bool wide = a.type == IO_F32;
  const int rows = PromptLaunch<KIND, DH>::kColumns / (wide ? 2 : 1);
  a.row_tiles = (int)(((long)a.r.max_new * a.group + rows - 1) / rows);
  const long units = (long)a.r.n * a.c.heads, groups = units * a.row_tiles;
  // Shares of the keys where there are fewer workgroups than the chip holds, two to a CU, of kTurns tiles at least.
  constexpr int kTurns = 8;
  a.tile_rows = a.part_rows = rows;
  const long slots = a.part_floats / (rows * (DH + 2));
  a.splits = (int)std::max<long>(1, std::min({kFill / groups, tiles / kTurns, slots / groups, (long)kMaxSplits}));
  a.least = kTurns;
  a.part_sums = (float2 *)(a.part + slots * rows * DH);
  // spread over the dies by unit where that leaves none idle
  const int spread = units % 8 == 0 || units >= 64;
  const long blocks = (spread ? (units + 7) / 8 * 8 : units) * a.row_tiles * a.splits;
  const dim3 grid((unsigned)blocks), block(PromptShape<KIND, DH>::NW * 64);
  if (wide) hipLaunchKernelGGL((cache_prompt_kernel<KIND, DH, true>), grid, block, (PromptLaunch<KIND, DH>::kLds), s, a, spread);
  else hipLaunchKernelGGL((cache_prompt_kernel<KIND, DH, false>), grid, block, (PromptLaunch<KIND, DH>::kLds), s, a, spread);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess || a.splits == 1 ? e : launch_cache_join(a, s);
}

template <int KIND, int DH>
hipError_t prepare() {
  const hipError_t e = hipFuncSetAttribute((const void *)cache_prompt_kernel<KIND, DH, false>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                           PromptLaunch<KIND, DH>::kLds);
  return e != hipSuccess ? e : hipFuncSetAttribute((const void *)cache_prompt_kernel<KIND, DH, true>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                                   PromptLaunch<KIND, DH>::kLds);
}
template <int KIND>
hipError_t prepare_width(int dh) {
  switch (dh) {
    case 64: return prepare<KIND, 64>();
    case 128: return prepare<KIND, 128>();
    case 256: return prepare<KIND, 256>();
    default: return prepare<KIND, 512>();
  }
}

template <int KIND>
hipError_t launch_width(const CacheAttnArgs &a, long tiles, hipStream_t s) {
  switch (a.c.dh) {
    case 64: return launch<KIND, 64>(a, tiles, s);
    case 128: return launch<KIND, 128>(a, tiles, s);
    case 256: return launch<KIND, 256>(a, tiles, s);
    default: return launch<KIND, 512>(a, tiles, s);
  }
}

}  // namespace

hipError_t prepare_cache_prompt(int kind, int dh) {
  return kind == CACHE_Q4 ? prepare_width<CACHE_Q4>(dh) : kind == CACHE_F16 ? prepare_width<CACHE_F16>(dh) : prepare_width<CACHE_BF16>(dh);
}
hipError_t launch_cache_prompt(CacheAttnArgs a, long tiles, hipStream_t s) {
  if (a.c.kind == CACHE_Q4) return launch_width<CACHE_Q4>(a, tiles, s);
  return a.c.kind == CACHE_F16 ? launch_width<CACHE_F16>(a, tiles, s) : launch_width<CACHE_BF16>(a, tiles, s);
}

}  // namespace nt
