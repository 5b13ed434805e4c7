// Paged key/value caches: what the page kernels (nt_cache.hip) and the attention kernels (nt_cache_attn.hip,
// nt_cache_prompt.hip) share.
//
// Layout.  The unit is a tile: 32 tokens of one key/value head in one layer, keys and values, in the order in which the
// matrix instructions take them, so that every load of a wave is one contiguous KB and nothing is transposed on the way.
// Scores are formed as S^T = K Q^T and the output as O^T = V^T P^T (v_mfma_f32_16x16x32): a lane then holds a query's
// scores for the very keys whose weights it has to give to the second product.  With r = lane % 16 and g = lane / 16,
//   keys    fragment (t, c), t = 0, 1, c < width / 32:  lane holds dims 32 c + 8 g + (0 .. 7) of token 8 (r / 4) + 4 t + r % 4;
//           the product leaves in register i of lane (r, g) the score of token 8 g + 4 t + i for query r;
//   values  fragment n < width / 16:  lane holds tokens 8 g + (0 .. 7) of dim 16 n + r, against the weights of query r for the
//           same tokens, which are its scores of t = 0, then t = 1.
// 16-bit tiles: keys [t][c][lane][8], then values [n][lane][8].  4-bit tiles: a fragment is a word of eight codes per lane, lowest
// nibble first; keys [word / 4][lane][word % 4] with word = t (width / 32) + c, values likewise with word = n, then the scales,
// one byte each (the upper byte of an fp16 number): keys [token][width / 32], values [width / 32][token].
// A page is [head][tile of the page]; a layer is [page], layers follow one another.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace nt {

constexpr int kTile = 32;  // tokens
constexpr int kQ4ScaleMax = 0x71, kQ4ScaleMin = 0x04, kQ4ScaleNan = 0x7E;  // 10240, 2^-14, NaN as upper bytes of fp16 numbers

enum CacheKind { CACHE_F16 = 1, CACHE_BF16 = 2, CACHE_Q4 = 3 };
enum IoType { IO_F32 = 0, IO_F16 = 1, IO_BF16 = 2, IO_PLANES = 3 };  // PLANES (outputs): an fp16 head, and a tail lo_offset elements on

__host__ __device__ inline int cache_tile_bytes(int kind, int dh) { return kind == CACHE_Q4 ? 34 * dh : 128 * dh; }

struct CacheView {
  char *pool;
  long layer_bytes, page_bytes;
  int32_t kind, heads, dh, page_shift, n_pages, max_seqs, max_len, width;  // width: entries of a row of the page table
  int32_t *table;    // [max_seqs][width] pages, -1 = freed by a trim; entries behind a sequence's end mean nothing
  int32_t *len;      // [max_seqs]
  int32_t *base;     // [max_seqs] first of the tokens that the last reserve gave the sequence
  int32_t *slot;     // [max_seqs] its entry in that call
  int32_t *mark;     // [max_seqs] scratch: INT_MAX between calls
  int32_t *ref;      // [n_pages] sequences that hold the page
  uint32_t *used;    // [(n_pages + 31) / 32] bits: ref > 0
  int32_t *flags;    // [2]: an entry was skipped for its id or length / for want of pages
};
__host__ __device__ inline long cache_tile_offset(const CacheView &c, int layer, int page, int head, int sub, int tile_bytes) {
  return layer * c.layer_bytes + page * c.page_bytes + (long)((head << (c.page_shift - 5)) + sub) * tile_bytes;
}

// Sequences and rows of a call
struct CacheRows {
  int32_t n, max_new;
  const int32_t *seq, *first;
};

struct CacheWriteArgs {
  CacheView c;
  CacheRows r;
  int32_t layer, type, tiles;  // tiles: of a sequence's new tokens, at most
  const void *k, *v;
  long ld;
  int32_t vec;  // rows are 16-byte aligned
};
hipError_t launch_cache_write(const CacheWriteArgs &a, hipStream_t s);

struct CacheReadArgs {
  CacheView c;
  CacheRows r;
  int32_t layer, type, max_keys, tiles;
  void *k, *v;
  int32_t vec;  // 16-byte aligned
};
hipError_t launch_cache_read(const CacheReadArgs &a, hipStream_t s);

struct CacheAttnArgs {
  CacheView c;
  CacheRows r;
  int32_t layer, type, out_type, q_heads, group;  // group: query heads per key/value head
  const void *q, *k, *v;  // k, v (single tokens): written to the cache first, or null
  void *out;
  long ld_q, ld_kv, ld_out, lo_offset;
  float scale;
  int32_t window, sinks;
  int32_t vec, vec_kv, vec_out;  // rows are 16-byte aligned
  float *part;           // [share][row][dh], behind them {maximum, sum} [share][row]
  long part_floats;
  // set by the launchers: tiles of query rows of a sequence and their rows, workgroups that share their keys, tiles of keys that
  // each has at least, rows that a share leaves room for
  int32_t row_tiles, tile_rows, splits, least, part_rows;
  float2 *part_sums;
};
constexpr int kMaxSplits = 64;  // shares of one row's keys: a lane each in the join
constexpr long kPartFloats = 16l << 20;  // what the shares of a call leave for the join, at most: 512 of 192 rows of 128, 32,000 of four
// Queries in tiles of 8 (rows: token, then head of the group), each split over the keys, of which a row sees about `tiles` tiles.
hipError_t launch_cache_token(CacheAttnArgs a, long tiles, hipStream_t s);
// Tiles of 64 to 256 query rows, likewise
hipError_t launch_cache_prompt(CacheAttnArgs a, long tiles, hipStream_t s);
hipError_t prepare_cache_prompt(int kind, int dh);  // once on a device before the first: its LDS
hipError_t launch_cache_join(const CacheAttnArgs &a, hipStream_t s);  // what the shares of either have left

#ifdef __HIPCC__
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float io_load(const void *p, int type, long i) {
  if (type == IO_F32) return ((const float *)p)[i];
  if (type == IO_F16) return (float)((const _Float16 *)p)[i];
  return (float)((const __bf16 *)p)[i];
}
// eight consecutive elements
__device__ __forceinline__ void io_load8(const void *p, int type, long i, int vec, float (&x)[8]) {
  if (!vec) {
#pragma unroll
    for (int j = 0; j < 8; j++) x[j] = io_load(p, type, i + j);
  } else if (type == IO_F32) {
    const float4 a = *(const float4 *)((const float *)p + i), b = *(const float4 *)((const float *)p + i + 4);
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
  } else if (type == IO_F16) {
    const f16x8 a = *(const f16x8 *)((const _Float16 *)p + i);
#pragma unroll
    for (int j = 0; j < 8; j++) x[j] = (float)a[j];
  } else {
    const bf16x8 a = *(const bf16x8 *)((const __bf16 *)p + i);
#pragma unroll
    for (int j = 0; j < 8; j++) x[j] = (float)a[j];
  }
}
__device__ __forceinline__ void io_store(void *p, int type, long i, long lo, float x) {
  if (type == IO_F32) ((float *)p)[i] = x;
  else if (type == IO_BF16) ((__bf16 *)p)[i] = (__bf16)x;
  else {
    const _Float16 h = (_Float16)x;
    ((_Float16 *)p)[i] = h;
    if (type == IO_PLANES) ((_Float16 *)p)[i + lo] = (_Float16)(x - (float)h);
  }
}

// x as bits of the cache's 16-bit type
template <int KIND>
__device__ __forceinline__ uint32_t half_bits(float x) {
  if constexpr (KIND == CACHE_F16) return __builtin_bit_cast(unsigned short, (_Float16)x);
  else return __builtin_bit_cast(unsigned short, (__bf16)x);
}

// Places within a tile of a token and a dim: 16 bits (element) and 4 bits (nibble of the keys' or values' codes)
__device__ __forceinline__ int key_lane(int tok, int dim) { return ((dim >> 3) & 3) * 16 + (tok >> 3) * 4 + (tok & 3); }
__device__ __forceinline__ int key_elem(int tok, int dim, int dh) {
  return ((((tok >> 2) & 1) * (dh / 32) + (dim >> 5)) * 64 + key_lane(tok, dim)) * 8 + (dim & 7);
}
__device__ __forceinline__ int value_elem(int tok, int dim) { return ((dim >> 4) * 64 + (tok >> 3) * 16 + (dim & 15)) * 8 + (tok & 7); }
__device__ __forceinline__ int q4_word(int word, int lane) { return (word >> 2) * 256 + lane * 4 + (word & 3); }
__device__ __forceinline__ int q4_key_word(int tok, int dim, int dh) {
  return q4_word(((tok >> 2) & 1) * (dh / 32) + (dim >> 5), key_lane(tok, dim));
}
__device__ __forceinline__ int q4_value_word(int tok, int dim) { return q4_word(dim >> 4, (tok >> 3) * 16 + (dim & 15)); }

// The upper byte of an fp16 number as that number
__device__ __forceinline__ float q4_scale(int b) { return (float)__builtin_bit_cast(_Float16, (unsigned short)(b << 8)); }
// Scale of a block whose largest magnitude is `top` (not NaN): the smallest with 6 scale >= top.  top / 6 is rounded, so its leading
// three bits may be one step too low (never too high: a step is exact), which the product with 6, exact in fp32, shows.
__device__ __forceinline__ int q4_scale_byte(float top) {
  if (!(top <= 61440.f)) return kQ4ScaleMax;
  const int b = max((int)(__float_as_uint(top / 6.f) >> 21) - ((127 - 15) << 2), kQ4ScaleMin);
  return b + (6.f * q4_scale(b) < top ? 1 : 0);
}
// Code of x under that scale: borders times the scale are exact in fp32
__device__ __forceinline__ int q4_code(float x, float s) {
  const float a = fabsf(x);
  const int c = (a > 0.25f * s) + (a >= 0.75f * s) + (a > 1.25f * s) + (a >= 1.75f * s) + (a > 2.5f * s) + (a >= 3.5f * s) + (a > 5.f * s);
  return c | (x < 0.f ? 8 : 0);
}
// Eight values of a token, a quarter of a block whose other quarters the lanes ^ 1, ^ 2, ^ 3 have: scale byte and codes
__device__ __forceinline__ int q4_round(const float (&x)[8], uint32_t &codes) {
  float top = 0.f;
  bool nan = false;
#pragma unroll
  for (int j = 0; j < 8; j++) top = fmaxf(top, fabsf(x[j])), nan |= x[j] != x[j];
  if (nan) top = __builtin_nanf("");
#pragma unroll
  for (int m = 1; m < 4; m *= 2) {
    const float o = __shfl_xor(top, m, 64);
    top = top != top || o != o ? __builtin_nanf("") : fmaxf(top, o);
  }
  const int b = top != top ? kQ4ScaleNan : q4_scale_byte(top);
  const float s = q4_scale(b);
  codes = 0;
#pragma unroll
  for (int j = 0; j < 8; j++) codes |= (uint32_t)q4_code(x[j], s) << (4 * j);
  return b;
}
#endif

}  // namespace nt
