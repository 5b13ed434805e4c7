// Attention of few rows over a paged cache: single tokens, and any rows that are not worth the tiled kernel.
//
// A workgroup has eight query rows of one key/value head (rows: token, then head of the group) and a share of the keys that they see;
// each of its four waves walks tiles of 32 keys by itself with the running maximum and sum of the softmax, all in registers:
// S^T = K Q^T, the weights of a lane are the operand of O^T = V^T P^T as they are (nt_cache.h).  The sixteen columns of an
// instruction are eight queries twice: the head of the query (and of the weights) in the cache's type, and the tail against it, so that both
// products have twice the bits at no cost: reading the keys and values is what such a call is bound by.
// The waves meet in the LDS; where several workgroups share the keys of a row, a second launch joins what they left in memory.
#include <algorithm>
#include <climits>

#include "nt_cache_frag.h"

namespace nt {
namespace {

constexpr int kRows = 8, kWaves = 4, kFill = 1024;
// Waves that share a tile, 128 dims each, and so tiles in work at a time: beyond 128 dims the accumulators, keys and values of a
// wave would leave one wave to a SIMD.  Their parts of the scores are added through the LDS.
constexpr int parts_of(int dh) { return dh > 128 ? dh / 128 : 1; }

// One token's key and value in a tile of a head: eight dims to a thread.  Workgroups of the same head (more than eight query heads)
// may do the same at the same time: they write what the others write, and what else is in a word stays as it is.
template <int KIND, int DH>
__device__ void write_token(char *tile, int tok, const CacheAttnArgs &a, long row, int tid) {
  const int side = tid / (DH / 8), dim = tid % (DH / 8) * 8;
  if (side > 1) return;
  float x[8];
  io_load8(side ? a.v : a.k, a.type, row + dim, a.vec_kv, x);
  if constexpr (KIND == CACHE_Q4) {
    uint32_t codes;
    const int scale = q4_round(x, codes);
    uint32_t *words = (uint32_t *)(tile + 16 * DH);
    if (side == 0) {
      ((uint32_t *)tile)[q4_key_word(tok, dim, DH)] = codes;
      if (dim % 32 == 0) tile[32 * DH + tok * (DH / 32) + dim / 32] = (char)scale;
    } else {
#pragma unroll
      for (int j = 0; j < 8; j++) {
        uint32_t *to = words + q4_value_word(tok, dim + j);
        *to = (*to & ~(15u << (4 * (tok & 7)))) | (codes >> (4 * j) & 15) << (4 * (tok & 7));
      }
      if (dim % 32 == 0) tile[33 * DH + dim / 32 * kTile + tok] = (char)scale;
    }
  } else if (side == 0) {
    *(uint4 *)((unsigned short *)tile + key_elem(tok, dim, DH)) =
        make_uint4(half_bits<KIND>(x[0]) | half_bits<KIND>(x[1]) << 16, half_bits<KIND>(x[2]) | half_bits<KIND>(x[3]) << 16,
                   half_bits<KIND>(x[4]) | half_bits<KIND>(x[5]) << 16, half_bits<KIND>(x[6]) | half_bits<KIND>(x[7]) << 16);
  } else {
#pragma unroll
    for (int j = 0; j < 8; j++) ((unsigned short *)(tile + 64 * DH))[value_elem(tok, dim + j)] = (unsigned short)half_bits<KIND>(x[j]);
  }
}

// ONE: every sequence has one new token, so the rows of a workgroup see the same keys
template <int KIND, int DH, bool ONE>
__global__ __launch_bounds__(256, (ONE ? 2 : 1)) void cache_token_kernel(CacheAttnArgs a) {
  typedef typename FragType<KIND>::type F;
  typedef typename FragType<KIND>::elem E;
  constexpr int PARTS = parts_of(DH), GROUPS = kWaves / PARTS, DW = DH / PARTS, NC = DW / 32, NV = DW / 16;
  __shared__ float lds_o[GROUPS][kRows][DH + 4];
  __shared__ float lds_m[GROUPS][kRows], lds_l[GROUPS][kRows], lds_scale[kRows];
  __shared__ f32x4 lds_s[PARTS > 1 ? 2 : 1][PARTS > 1 ? kWaves : 1][2][PARTS > 1 ? 64 : 1];
  char *lds_q = (char *)lds_o;  // before the loop
  static_assert(sizeof(lds_o) >= DH * 32, "");
  const CacheView &c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, g4 = lane >> 4;
  const int part = wave % PARTS, mine = wave / PARTS;  // of a tile's dims, of the tiles in work
  const int split = blockIdx.x % a.splits, group = blockIdx.x / a.splits, h = group % c.heads, rt = group / c.heads % a.row_tiles,
            i = group / c.heads / a.row_tiles;
  const Share w(a, i, rt, kRows);
  const int G = a.group;
  if ((!w.known || w.m < 0 || w.m > a.r.max_new || w.m > w.len) && split == 0 && h == 0 && rt == 0 && tid == 0) atomicOr(c.flags, 1);
  if (rt * kRows >= w.R || split >= w.shares) return;
  const int t1 = min((split + 1) * w.per, w.tiles);

  if (ONE && a.k && split == w.shares - 1) {  // the newest token's key and value, to the tile that this workgroup has
    const bool given = w.known && w.m == 1 && c.slot[w.s] == i && c.base[w.s] == w.len - 1;
    if (given) {
      const int tile = w.first / kTile, page = c.table[(long)w.s * c.width + (tile >> (c.page_shift - 5))];
      if (page >= 0)
        write_token<KIND, DH>(c.pool + cache_tile_offset(c, a.layer, page, h, tile & ((1 << (c.page_shift - 5)) - 1), cache_tile_bytes(KIND, DH)),
                              w.first % kTile, a, w.row0 * a.ld_kv + (long)h * DH, tid);
    } else if (h == 0 && rt == 0 && tid == 0) {
      atomicOr(c.flags, 1);
    }
    __syncthreads();
  }
  // the queries: heads of the group in columns 0 .. 7, their tails in 8 .. 15.  A power of two brings the largest of each to
  // 1 .. 2: no overflow in fp16, and tails with all their bits.
  for (int x = tid; x < kRows * DH / 8; x += 256) {
    const int r = x / (DH / 8), d = x % (DH / 8) * 8, row = rt * kRows + r;
    float v[8] = {}, big = 0.f;
    if (row < w.R) io_load8(a.q, a.type, (w.row0 + row / G) * a.ld_q + (long)(h * G + row % G) * DH + d, a.vec, v);
#pragma unroll
    for (int k = 0; k < 8; k++) big = fmaxf(big, fabsf(v[k]));
#pragma unroll
    for (int k = 1; k < DH / 8; k *= 2) big = fmaxf(big, __shfl_xor(big, k, 64));
    const int e = big > 0.f && big < __builtin_inff() ? min(max(ilogbf(big), -100), 126) : 0;
    if (d == 0) lds_scale[r] = fmaxf(ldexpf(fabsf(a.scale) * 1.44269504088896f, e), kLeastScale);
    const float down = ldexpf(a.scale < 0.f ? -1.f : 1.f, -e);
    F head, tail;
#pragma unroll
    for (int k = 0; k < 8; k++) {
      const float y = as_f32(v[k] * down);
      head[k] = (E)y;
      tail[k] = (E)(y - (float)head[k]);
    }
    F *to = (F *)lds_q + d / 32 * 64 + d / 8 % 4 * 16 + r;
    to[0] = head;
    to[8] = tail;
  }
  const int row = rt * kRows + (col & 7);
  const int pos = row < w.R ? w.first + row / G : -1, low_own = a.window > 0 ? pos - a.window + 1 : 0;
  // the wave's first tile is on its way before the queries are there
  const int sub_bits = c.page_shift - 5;
  const int32_t *table = c.table + (long)w.s * c.width;
  auto tile_of = [&](int t) { return t < w.sink_tiles ? t : w.window_tile + t - w.sink_tiles; };
  auto page_of = [&](int t) { return t < t1 ? table[tile_of(t) >> sub_bits] : -1; };
  auto address = [&](int t, int page) {  // of a page that is not there: the first one's tile, which is then not looked at
    return c.pool + cache_tile_offset(c, a.layer, max(page, 0), h, tile_of(t) & ((1 << sub_bits) - 1), cache_tile_bytes(KIND, DH));
  };
  KeyTile<KIND, DH, DW> kt;
  ValueTile<KIND, DH, DW> vt;
  int t = split * w.per + mine;
  int page = page_of(t), page_next = page_of(t + GROUPS);
  if (t < t1) {
    const char *at = address(t, page);
    kt.load(at, lane, part);
    vt.load(at, lane, part);
  } else if (PARTS > 1) {  // a wave that has to meet the others all the same
    kt = {};
    vt = {};
  }
  __syncthreads();
  F q[NC];
#pragma unroll
  for (int k = 0; k < NC; k++) q[k] = ((const F *)lds_q)[(part * NC + k) * 64 + lane];
  const float to_log2 = lds_scale[col & 7], tails = col < 8 ? 0.f : 1.f;

  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  f32x4 o[NV];
#pragma unroll
  for (int n = 0; n < NV; n++) o[n] = zero;
  float top = kLowest, sum = 0.f;
  int turn = 0;
  for (; PARTS > 1 ? t - mine < t1 : t < t1; t += GROUPS) {  // waves that meet make the same number of turns
    const int j0 = tile_of(t) * kTile;
    f32x4 sc[2] = {zero, zero};
#pragma unroll
    for (int k = 0; k < NC; k++) {
      sc[0] = mma(kt.frag(0, k), q[k], sc[0]);
      sc[1] = mma(kt.frag(1, k), q[k], sc[1]);
    }
    // the next tile's keys take the place of these, its values that of these after the second product
    const char *next = address(min(t + GROUPS, t1 - 1), page_next);
    if (t + GROUPS < t1) kt.load(next, lane, part);
    const int page_after = page_of(t + 2 * GROUPS);
    if constexpr (PARTS > 1) {
      lds_s[turn][wave][0][lane] = sc[0];
      lds_s[turn][wave][1][lane] = sc[1];
      __syncthreads();
      sc[0] = sc[1] = zero;
#pragma unroll
      for (int k = 0; k < PARTS; k++) {
        sc[0] += lds_s[turn][mine * PARTS + k][0][lane];
        sc[1] += lds_s[turn][mine * PARTS + k][1][lane];
      }
      turn ^= 1;
    }
    float y[8];
#pragma unroll
    for (int j = 0; j < 8; j++) {
      const float x = sc[j / 4][j % 4];
      y[j] = x + eight_on(x);  // head and tail: columns 8 apart
    }
    const bool all_seen =
        page >= 0 && j0 + kTile - 1 <= w.p_min && (a.window == 0 || j0 >= w.p_max - a.window + 1 || j0 + kTile <= a.sinks);
    uint32_t seen = 0xFF;
    if (!all_seen) {
      uint32_t someone = 0;
      seen = 0;
#pragma unroll
      for (int j = 0; j < 8; j++) {
        const int key = j0 + g4 * 8 + j;
        const bool own = (page >= 0) & (key <= pos) & ((key >= low_own) | (key < a.sinks));
        const bool any = (page >= 0) & (key <= w.p_max) & ((key >= w.low) | (key < a.sinks));
        seen |= (own ? 1u : 0u) << j;
        someone |= (any ? 1u : 0u) << j;
        y[j] = own ? y[j] : -__builtin_inff();
      }
      vt.clear(someone);
    }
    float z[8];
    auto weigh = [&]() {
      int big = INT_MIN;
#pragma unroll
      for (int j = 0; j < 8; j++) {
        z[j] = __builtin_fmaf(y[j], to_log2, -top);
        big = max(big, __float_as_int(z[j]));  // of positive numbers the largest
      }
      return big;
    };
    if (__any(weigh() > __float_as_int(kSlack))) {  // some row: those that need it change their maximum, no other row depends on them
      float mx = y[0];
#pragma unroll
      for (int j = 1; j < 8; j++) mx = fmaxf(mx, y[j]);
      mx = wave_pair16(mx, mx, WaveMax{});
      mx = wave_pair32(mx, mx, WaveMax{}) * to_log2;
      const float up = mx - top > kSlack ? mx : top, shrink = __builtin_amdgcn_exp2f(top - up);
      top = up;
      sum *= shrink;
#pragma unroll
      for (int n = 0; n < NV; n++) o[n] *= shrink;
      weigh();
    }
    F p;
#pragma unroll
    for (int j = 0; j < 8; j++) {
      const float x = __builtin_amdgcn_exp2f(z[j]);
      sum += x;
      p[j] = (E)__builtin_fmaf(-(float)(E)x, tails, x);  // exact before it is rounded
    }
    bool bad = false;
    if (!ONE && !all_seen && w.p_min < w.p_max) {  // rows of different tokens: some see keys that others do not
#pragma unroll
      for (int n = 0; n < NV; n++) bad |= any_no_number(vt.frag(n));
    }
    if (!ONE && __any(bad)) {
#pragma unroll
      for (int n = 0; n < NV; n++) o[n] = mma_seen(vt.frag(n), p, seen, o[n]);
    } else {
#pragma unroll
      for (int n = 0; n < NV; n++) o[n] = mma(vt.frag(n), p, o[n]);
    }
    if (t + GROUPS < t1) vt.load(next, lane, part);
    page = page_next;
    page_next = page_after;
  }
  sum = wave_pair16(sum, sum, WaveAdd{});
  sum = wave_pair32(sum, sum, WaveAdd{});

  const long at = ((long)group * a.splits + split) * a.part_rows;
  __syncthreads();                                 // the last use of the LDS
  if (lane < 8 && part == 0) lds_m[mine][lane] = top, lds_l[mine][lane] = sum;
#pragma unroll
  for (int n = 0; n < NV; n++) {
    f32x4 x = o[n];
#pragma unroll
    for (int k = 0; k < 4; k++) x[k] = head_and_tail(x[k]);
    if (col < 8) *(f32x4 *)&lds_o[mine][col][part * DW + n * 16 + g4 * 4] = x;
  }
  __syncthreads();
  for (int x = tid; x < kRows * DH; x += 256) {
    const int r = x / DH, d = x % DH;
    if (rt * kRows + r >= w.R) break;
    float mx = lds_m[0][r];
#pragma unroll
    for (int k = 1; k < GROUPS; k++) mx = fmaxf(mx, lds_m[k][r]);
    float l = 0.f, y = 0.f;
#pragma unroll
    for (int k = 0; k < GROUPS; k++) {
      const float f = __builtin_amdgcn_exp2f(lds_m[k][r] - mx);
      l += f * lds_l[k][r];
      y += f * lds_o[k][r][d];
    }
    if (w.shares == 1) {
      store_row(a, w, h, rt * kRows + r, d, DH, y, l);
    } else {
      a.part[(at + r) * DH + d] = y;
      if (d == 0) a.part_sums[at + r] = make_float2(mx, l);
    }
  }
}

// Joins the shares of eight rows of a tile
template <int DH>
__global__ __launch_bounds__(256) void cache_join_kernel(CacheAttnArgs a) {
  __shared__ float lds_f[kRows][kMaxSplits], lds_l[kRows];
  const int tid = threadIdx.x, lane = tid & 63, group = blockIdx.x;
  const int h = group % a.c.heads, rt = group / a.c.heads % a.row_tiles, i = group / a.c.heads / a.row_tiles, r0 = blockIdx.y * kRows;
  const Share w(a, i, rt, a.tile_rows);
  const int first = rt * a.tile_rows + r0, rows = min(min(w.R - first, kRows), a.tile_rows - r0);
  if (rows <= 0 || w.shares == 1) return;
  const long at = (long)group * a.splits * a.part_rows + r0;
  static_assert(kMaxSplits == 64, "a share per lane");
  for (int r = tid >> 6; r < rows; r += 4) {  // weights of the shares
    const float2 ml = lane < w.shares ? a.part_sums[at + lane * a.part_rows + r] : make_float2(kLowest, 0.f);
    const float mx = wave_max(ml.x), f = __builtin_amdgcn_exp2f(ml.x - mx), l = wave_sum(f * ml.y);
    lds_f[r][lane] = f;
    if (lane == 0) lds_l[r] = l;
  }
  __syncthreads();
  for (int x = tid; x < rows * DH / 4; x += 256) {
    const int r = x / (DH / 4), d = x % (DH / 4) * 4;
    const f32x4 *from = (const f32x4 *)(a.part + (at + r) * DH + d);
    const int step = a.part_rows * (DH / 4);
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
    for (int k0 = 0; k0 < w.shares; k0 += 8) {  // eight loads under way
      f32x4 v[8];
#pragma unroll
      for (int k = 0; k < 8; k++) v[k] = from[(long)min(k0 + k, w.shares - 1) * step];
#pragma unroll
      for (int k = 0; k < 8; k++)
        if (k0 + k < w.shares) y += lds_f[r][k0 + k] * v[k];
    }
    const float l = lds_l[r];
    const int row = first + r;
    const long o = (w.row0 + row / a.group) * a.ld_out + (long)(h * a.group + row % a.group) * DH + d;
#pragma unroll
    for (int k = 0; k < 4; k++) io_store(a.out, a.out_type, o + k, a.lo_offset, l == 0.f ? 0.f : y[k] / l);
  }
}

template <int KIND, int DH>
hipError_t launch(CacheAttnArgs a, long tiles, hipStream_t s) {
  // Shares of the keys.  Up to 1,024 workgroups, four to a CU, as many as have a turn each; beyond that as many as have kTurns, so that
  // the longest sequences do not run on when the others are done: 64 sequences of 500 to 16,000 tokens, 8 heads, 235 us with two
  // shares and 218 with 15 (turns 2 / 4 / 8 / 16: 225 / 220 / 218 / 221); 256 in 4 bits, whose turns are shorter, 391 with one, 298
  // with 15 and 287 with 7.
  constexpr int kTurns = KIND == CACHE_Q4 ? 16 : 8;
  const long groups = (long)a.c.heads * a.row_tiles * a.r.n, at_once = kWaves / parts_of(DH);
  a.tile_rows = kRows;
  a.part_rows = (int)std::min<long>(kRows, (long)a.r.max_new * a.group);
  const long slots = a.part_floats / (a.part_rows * (DH + 2)), turns = (tiles + at_once - 1) / at_once;
  const long few = std::min(kFill / groups, turns), many = std::min(slots / groups, turns / kTurns);
  a.splits = (int)std::max<long>(1, std::min<long>(std::max(few, many), std::min<long>(kMaxSplits, slots / groups)));
  a.least = (int)(at_once * (few >= many ? 1 : kTurns));
  a.part_sums = (float2 *)(a.part + slots * a.part_rows * DH);
  const dim3 grid((unsigned)(groups * a.splits)), block(256);
  if (a.r.max_new == 1) hipLaunchKernelGGL((cache_token_kernel<KIND, DH, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((cache_token_kernel<KIND, DH, false>), grid, block, 0, s, a);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess || a.splits == 1 ? e : launch_cache_join(a, s);
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

hipError_t launch_cache_join(const CacheAttnArgs &a, hipStream_t s) {
  const dim3 grid((unsigned)((long)a.r.n * a.c.heads * a.row_tiles), (unsigned)((a.part_rows + kRows - 1) / kRows)), block(256);
  switch (a.c.dh) {
    case 64: hipLaunchKernelGGL(cache_join_kernel<64>, grid, block, 0, s, a); break;
    case 128: hipLaunchKernelGGL(cache_join_kernel<128>, grid, block, 0, s, a); break;
    case 256: hipLaunchKernelGGL(cache_join_kernel<256>, grid, block, 0, s, a); break;
    default: hipLaunchKernelGGL(cache_join_kernel<512>, grid, block, 0, s, a);
  }
  return hipGetLastError();
}
hipError_t launch_cache_token(CacheAttnArgs a, long tiles, hipStream_t s) {
  a.row_tiles = (int)(((long)a.r.max_new * a.group + kRows - 1) / kRows);
  if (a.c.kind == CACHE_Q4) return launch_width<CACHE_Q4>(a, tiles, s);
  return a.c.kind == CACHE_F16 ? launch_width<CACHE_F16>(a, tiles, s) : launch_width<CACHE_BF16>(a, tiles, s);
}

}  // namespace nt
