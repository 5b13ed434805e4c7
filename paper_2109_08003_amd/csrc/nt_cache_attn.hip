// Attention of few rows over a paged cache: single tokens, and any rows that are not worth the tiled kernel.
//
// A workgroup has eight query rows of one key/value head (rows: token, then head of the group) and a share of the keys that they see;
// each of its four waves walks tiles of 32 keys by itself with the running maximum and sum of the softmax, all in registers:
// S^T = K Q^T, the weights of a lane are the operand of O^T = V^T P^T as they are (nt_cache.h).  The sixteen columns of an
// instruction are eight queries twice: the head of the query (and of the weights) in the cache's type, and the tail against it, so that both
// products have twice the bits at no cost: reading the keys and values is what such a call is bound by.
// The waves meet in the LDS; where several workgroups share the keys of a row, a second launch joins what they left in memory.
#include "nt_cache_frag.h"

namespace nt {
namespace {

constexpr int kRows = 8, kWaves = 4;

// What a workgroup has to do: the rows of sequence i in row tile rt, the tiles of keys that one of them sees (those of the sinks, then
// those of the window), and how they are shared out.
struct Share {
  int s, len, m, R;                        // sequence, its length, new tokens, query rows
  long row0;
  int first, p_min, p_max, low;            // positions: of the first new token, of the rows; first key of the earliest window
  int sink_tiles, window_tile, tiles, per, shares;
  bool known;
  __device__ __forceinline__ Share(const CacheAttnArgs &a, int i, int rt) {
    s = a.r.seq ? a.r.seq[i] : i;
    row0 = a.r.first ? a.r.first[i] : i;
    m = a.r.first ? a.r.first[i + 1] - (int)row0 : 1;
    known = s >= 0 && s < a.c.max_seqs;
    len = known ? a.c.len[s] : 0;
    R = min(m, a.r.max_new) * a.group;
    first = len - m;
    p_min = first + rt * kRows / a.group;
    p_max = first + min(rt * kRows + kRows - 1, R - 1) / a.group;
    low = a.window > 0 ? max(p_min - a.window + 1, 0) : 0;
    sink_tiles = (min(a.sinks, low) + kTile - 1) / kTile;
    window_tile = max(low / kTile, sink_tiles);
    tiles = p_max < 0 ? 0 : sink_tiles + max(p_max / kTile + 1 - window_tile, 0);
    per = max((tiles + a.splits - 1) / a.splits, kWaves);
    shares = max((tiles + per - 1) / per, 1);
  }
};

// x / l, zero where no key was seen
__device__ __forceinline__ void store_row(const CacheAttnArgs &a, const Share &w, int h, int row, int d, int dh, float x, float l) {
  if (row < w.R)
    io_store(a.out, a.out_type, (w.row0 + row / a.group) * a.ld_out + (long)(h * a.group + row % a.group) * dh + d, a.lo_offset, l == 0.f ? 0.f : x / l);
}

template <int KIND, int DH>
__global__ __launch_bounds__(256) void cache_token_kernel(CacheAttnArgs a) {
  typedef typename FragType<KIND>::type F;
  typedef typename FragType<KIND>::elem E;
  constexpr int NC = DH / 32, NV = DH / 16, CH = DH < 256 ? DH : 256, LD = CH + 4;
  __shared__ float lds_o[kWaves][kRows][LD];
  __shared__ float lds_m[kWaves][kRows], lds_l[kWaves][kRows];
  const CacheView &c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, g4 = lane >> 4;
  const int split = blockIdx.x % a.splits, group = blockIdx.x / a.splits, h = group % c.heads, rt = group / c.heads % a.row_tiles,
            i = group / c.heads / a.row_tiles;
  const Share w(a, i, rt);
  const int G = a.group;
  if ((!w.known || w.m < 0 || w.m > a.r.max_new || w.m > w.len) && split == 0 && h == 0 && rt == 0 && tid == 0) atomicOr(c.flags, 1);
  if (rt * kRows >= w.R || split >= w.shares) return;
  const int t1 = min((split + 1) * w.per, w.tiles);

  // this lane's query: head g of the group in columns g and g + 8
  const int row = rt * kRows + (col & 7), tok = row / G;
  const bool real = row < w.R;
  const int pos = real ? w.first + tok : -1, low_own = a.window > 0 ? pos - a.window + 1 : 0;
  F q[NC];
  float to_log2;
  {
    float x[NC][8], top = 0.f;
#pragma unroll
    for (int k = 0; k < NC; k++) {
      if (real) io_load8(a.q, a.type, (w.row0 + tok) * a.ld_q + (long)(h * G + row % G) * DH + k * 32 + g4 * 8, a.vec, x[k]);
#pragma unroll
      for (int j = 0; j < 8; j++) {
        if (!real) x[k][j] = 0.f;
        top = fmaxf(top, fabsf(x[k][j]));
      }
    }
    top = wave_pair16(top, top, WaveMax{});
    top = wave_pair32(top, top, WaveMax{});
    // a power of two brings the largest of the query to 1 .. 2: no overflow in fp16, and a tail with all its bits
    const int e = top > 0.f && top < __builtin_inff() ? min(max(ilogbf(top), -100), 126) : 0;
    to_log2 = ldexpf(a.scale * 1.44269504088896f, e);
    const float down = ldexpf(1.f, -e);
#pragma unroll
    for (int k = 0; k < NC; k++)
#pragma unroll
      for (int j = 0; j < 8; j++) {
        const float y = as_f32(x[k][j] * down);
        const E head = (E)y;
        q[k][j] = col < 8 ? head : (E)(y - (float)head);
      }
  }

  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  f32x4 o[NV];
#pragma unroll
  for (int n = 0; n < NV; n++) o[n] = zero;
  float top = -__builtin_inff(), sum = 0.f;
  const int sub_bits = c.page_shift - 5;
  const int32_t *table = c.table + (long)w.s * c.width;
  for (int t = split * w.per + wave; t < t1; t += kWaves) {
    const int tile = t < w.sink_tiles ? t : w.window_tile + t - w.sink_tiles;
    const int page = table[tile >> sub_bits];
    if (page < 0) continue;
    const char *at = c.pool + cache_tile_offset(c, a.layer, page, h, tile & ((1 << sub_bits) - 1), cache_tile_bytes(KIND, DH));
    KeyTile<KIND, DH> kt;
    ValueTile<KIND, DH> vt;
    kt.load(at, lane);
    vt.load(at, lane);
    f32x4 sc[2] = {zero, zero};
#pragma unroll
    for (int k = 0; k < NC; k++) {
      sc[0] = mma(kt.frag(0, k), q[k], sc[0]);
      sc[1] = mma(kt.frag(1, k), q[k], sc[1]);
    }
    float y[8];
#pragma unroll
    for (int j = 0; j < 8; j++) {
      const float x = sc[j / 4][j % 4];
      y[j] = (x + __uint_as_float(wave_dpp<0x128>(__float_as_uint(x)))) * to_log2;  // head and tail: columns 8 apart
    }
    const int j0 = tile * kTile;
    const bool all_seen = j0 + kTile - 1 <= w.p_min && (a.window == 0 || j0 >= w.p_max - a.window + 1 || j0 + kTile <= a.sinks);
    uint32_t seen = 0xFF;
    if (!all_seen) {
      uint32_t someone = 0;
      seen = 0;
#pragma unroll
      for (int j = 0; j < 8; j++) {
        const int key = j0 + g4 * 8 + j;
        if (key <= pos && (key >= low_own || key < a.sinks)) seen |= 1u << j;
        else y[j] = -__builtin_inff();
        if (key <= w.p_max && (key >= w.low || key < a.sinks)) someone |= 1u << j;
      }
      vt.clear(someone);
    }
    float tile_top = y[0];
#pragma unroll
    for (int j = 1; j < 8; j++) tile_top = fmaxf(tile_top, y[j]);
    tile_top = wave_pair16(tile_top, tile_top, WaveMax{});
    tile_top = wave_pair32(tile_top, tile_top, WaveMax{});
    const float next = fmaxf(top, tile_top), from = next == -__builtin_inff() ? 0.f : next;
    const float shrink = __builtin_amdgcn_exp2f(top - from);
    top = next;
    sum *= shrink;
    F p;
#pragma unroll
    for (int j = 0; j < 8; j++) {
      const float x = __builtin_amdgcn_exp2f(y[j] - from);
      sum += x;
      const E head = (E)x;
      p[j] = col < 8 ? head : (E)(x - (float)head);
    }
#pragma unroll
    for (int n = 0; n < NV; n++) o[n] *= shrink;
    bool bad = false;
    if (!all_seen && w.p_min < w.p_max) {  // rows of different tokens: some see keys that others do not
#pragma unroll
      for (int n = 0; n < NV; n++) bad |= any_no_number(vt.frag(n));
    }
    if (__any(bad)) {
#pragma unroll
      for (int n = 0; n < NV; n++) o[n] = mma_seen(vt.frag(n), p, seen, o[n]);
    } else {
#pragma unroll
      for (int n = 0; n < NV; n++) o[n] = mma(vt.frag(n), p, o[n]);
    }
  }
  sum = wave_pair16(sum, sum, WaveAdd{});
  sum = wave_pair32(sum, sum, WaveAdd{});
  if (lane < 8) lds_m[wave][lane] = top, lds_l[wave][lane] = sum;

  float *part = a.part + ((long)group * a.splits + split) * kRows * (DH + 2);
#pragma unroll
  for (int d0 = 0; d0 < DH; d0 += CH) {
    __syncthreads();
#pragma unroll
    for (int n = 0; n < CH / 16; n++) {
      f32x4 x = o[d0 / 16 + n];
#pragma unroll
      for (int k = 0; k < 4; k++) x[k] += __uint_as_float(wave_dpp<0x128>(__float_as_uint(x[k])));
      if (col < 8) *(f32x4 *)&lds_o[wave][col][n * 16 + g4 * 4] = x;
    }
    __syncthreads();
    for (int x = tid; x < kRows * CH; x += 256) {
      const int r = x / CH, d = x % CH;
      float mx = lds_m[0][r];
#pragma unroll
      for (int k = 1; k < kWaves; k++) mx = fmaxf(mx, lds_m[k][r]);
      const float from = mx == -__builtin_inff() ? 0.f : mx;
      float l = 0.f, y = 0.f;
#pragma unroll
      for (int k = 0; k < kWaves; k++) {
        const float f = __builtin_amdgcn_exp2f(lds_m[k][r] - from);
        l += f * lds_l[k][r];
        y += f * lds_o[k][r][d];
      }
      if (w.shares == 1) {
        store_row(a, w, h, rt * kRows + r, d0 + d, DH, y, l);
      } else {
        float *to = part + r * (DH + 2);
        to[d0 + d] = y;
        if (d0 + d == 0) to[DH] = mx, to[DH + 1] = l;
      }
    }
  }
}

// Joins the shares of a row: a workgroup per tile of rows
template <int DH>
__global__ __launch_bounds__(256) void cache_join_kernel(CacheAttnArgs a) {
  __shared__ float lds_f[kMaxSplits][kRows], lds_l[kRows];
  const int tid = threadIdx.x, group = blockIdx.x, h = group % a.c.heads, rt = group / a.c.heads % a.row_tiles, i = group / a.c.heads / a.row_tiles;
  const Share w(a, i, rt);
  if (rt * kRows >= w.R || w.shares == 1) return;
  const float *part = a.part + (long)group * a.splits * kRows * (DH + 2);
  if (tid < kRows) {  // weights of the shares
    const float *p = part + tid * (DH + 2) + DH;
    float mx = -__builtin_inff();
    for (int k = 0; k < w.shares; k++) mx = fmaxf(mx, p[(long)k * kRows * (DH + 2)]);
    const float from = mx == -__builtin_inff() ? 0.f : mx;
    float l = 0.f;
    for (int k = 0; k < w.shares; k++) {
      const float f = __builtin_amdgcn_exp2f(p[(long)k * kRows * (DH + 2)] - from);
      lds_f[k][tid] = f;
      l += f * p[(long)k * kRows * (DH + 2) + 1];
    }
    lds_l[tid] = l;
  }
  __syncthreads();
  for (int x = tid; x < kRows * DH; x += 256) {
    const int r = x / DH, d = x % DH;
    float y = 0.f;
    for (int k = 0; k < w.shares; k++) y += lds_f[k][r] * part[((long)k * kRows + r) * (DH + 2) + d];
    store_row(a, w, h, rt * kRows + r, d, DH, y, lds_l[r]);
  }
}

template <int DH>
void join(const CacheAttnArgs &a, hipStream_t s) {
  if (a.splits > 1) hipLaunchKernelGGL(cache_join_kernel<DH>, dim3((unsigned)(a.c.heads * a.row_tiles * a.r.n)), dim3(256), 0, s, a);
}

template <int KIND>
hipError_t launch(const CacheAttnArgs &a, hipStream_t s) {
  const dim3 grid((unsigned)((long)a.splits * a.c.heads * a.row_tiles * a.r.n)), block(256);
  switch (a.c.dh) {
    case 64: hipLaunchKernelGGL((cache_token_kernel<KIND, 64>), grid, block, 0, s, a); join<64>(a, s); break;
    case 128: hipLaunchKernelGGL((cache_token_kernel<KIND, 128>), grid, block, 0, s, a); join<128>(a, s); break;
    case 256: hipLaunchKernelGGL((cache_token_kernel<KIND, 256>), grid, block, 0, s, a); join<256>(a, s); break;
    default: hipLaunchKernelGGL((cache_token_kernel<KIND, 512>), grid, block, 0, s, a); join<512>(a, s);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_token(const CacheAttnArgs &a, hipStream_t s) {
  if (a.c.kind == CACHE_Q4) return launch<CACHE_Q4>(a, s);
  return a.c.kind == CACHE_F16 ? launch<CACHE_F16>(a, s) : launch<CACHE_BF16>(a, s);
}

}  // namespace nt
