// Paged key/value caches: the C entry points and the kernels on pages (nt_cache.h has the layout).
//
// Which pages are free is a bit map beside a count of holders per page.  The calls that hand out pages begin with one workgroup
// that counts what every entry needs, sums the counts in the order of the entries and takes the lowest free pages: page tables then
// depend on nothing but the calls made.  64,000 pages are 8 KB of map, which that workgroup reads in two loads per thread.  What is
// left - rows of the page table, counts of holders, contents of pages - is done by launches over the whole chip.
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <new>

#include "../../include/nt.h"
#include "nt_cache_frag.h"
#include "nt_cache_host.h"
#include "nt_kernels.h"

namespace nt {

namespace {

constexpr int kPlan = 1024;  // threads of the workgroup that hands out pages

// Scratch of the calls that move pages
struct PageWork {
  int32_t *off;      // [max_seqs] first of an entry's new pages in `list`, -1 = the entry is skipped
  int32_t *list;     // [n_pages] new pages
  int32_t *from, *to;  // [n_pages] pages to be copied
  int32_t *info;     // [0] pages to be copied
  int32_t *row_len;  // [max_seqs] and
  int32_t *row;      // [max_seqs][width]: lengths and tables of the sources, before any target changes
};

__device__ __forceinline__ int atomic_read(const int32_t *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// Sum over the threads before this one; `all` is the sum over all.  Every thread of kPlan calls it.
__device__ __forceinline__ int block_scan(int x, int &all, int32_t (&lds)[kPlan / 64]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int s = x;
#pragma unroll
  for (int m = 1; m < 64; m *= 2) {
    const int o = __shfl_up(s, m, 64);
    if (lane >= m) s += o;
  }
  __syncthreads();  // the last use of lds
  if (lane == 63) lds[wave] = s;
  __syncthreads();
  int before = 0;
  all = 0;
#pragma unroll
  for (int w = 0; w < kPlan / 64; w++) {
    if (w < wave) before += lds[w];
    all += lds[w];
  }
  return before + s - x;
}
__device__ __forceinline__ int block_sum(int x, int32_t (&lds)[kPlan / 64]) {
  int all;
  block_scan(x, all, lds);
  return all;
}
__device__ __forceinline__ int block_max(int x, int32_t (&lds)[kPlan / 64]) {
  x = wave_fold(x, WaveMax{});
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
  __syncthreads();
  int m = INT_MIN;
#pragma unroll
  for (int w = 0; w < kPlan / 64; w++) m = max(m, lds[w]);
  return m;
}

__device__ __forceinline__ int words_of(const CacheView &c) { return (c.n_pages + 31) / 32; }
__device__ int count_free(const CacheView &c, int32_t (&lds)[kPlan / 64]) {
  int n = 0;
  for (int w = threadIdx.x; w < words_of(c); w += kPlan) n += __popc(~c.used[w]);
  return block_sum(n, lds);
}
// list[0 .. n) = the lowest n free pages, of which there are that many, now held once
__device__ void take_pages(const CacheView &c, int n, int32_t *list, int32_t (&lds)[kPlan / 64]) {
  for (int w0 = 0, done = 0; done < n && w0 < words_of(c); w0 += kPlan) {
    const int w = w0 + threadIdx.x;
    uint32_t free = w < words_of(c) ? ~c.used[w] : 0, got = 0;
    int all, at = done + block_scan(__popc(free), all, lds);
    for (; free && at < n; at++) {
      const uint32_t bit = free & -free;
      const int page = w * 32 + __ffs(bit) - 1;
      list[at] = page;
      c.ref[page] = 1;
      got |= bit;
      free ^= bit;
    }
    if (got) c.used[w] |= got;
    done += all;
  }
}
__device__ __forceinline__ void drop_page(const CacheView &c, int page) {
  if (page >= 0 && atomicSub(c.ref + page, 1) == 1) atomicAnd(c.used + (page >> 5), ~(1u << (page & 31)));
}
__device__ __forceinline__ int pages_of(const CacheView &c, int len) { return (len + (1 << c.page_shift) - 1) >> c.page_shift; }

// What is left of the entries of off[0 .. n) when `total` pages are wanted: entries that go beyond the free pages are
// skipped, the others' pages are taken.  need(i) >= 0 for entries that are not skipped already.
template <class Need>
__device__ void grant(const CacheView &c, int n, int total, const PageWork &w, int32_t (&lds)[kPlan / 64], Need need) {
  if (total <= 0) return;
  const int free = count_free(c, lds);
  int top = 0;
  for (int i = threadIdx.x; i < n; i += kPlan) {
    if (w.off[i] < 0) continue;
    const int k = need(i);
    if (k > 0 && k > free - w.off[i]) {
      w.off[i] = -1;
      atomicOr(c.flags + 1, 1);
    } else if (k > 0) {
      top = max(top, w.off[i] + k);
    }
  }
  top = block_max(top, lds);
  take_pages(c, top, w.list, lds);
  __syncthreads();
}

// ---- room for new tokens ---------------------------------------------------------------------------------------------

__global__ __launch_bounds__(kPlan) void cache_reserve_kernel(CacheView c, CacheRows r, PageWork w) {
  __shared__ int32_t lds[kPlan / 64];
  const int tid = threadIdx.x, n = r.n;
  auto id = [&](int i) { return r.seq ? r.seq[i] : i; };
  auto count = [&](int i) { return r.first ? r.first[i + 1] - r.first[i] : 1; };
  auto inside = [&](int s) { return s >= 0 && s < c.max_seqs; };
  if (r.seq) {
    for (int i = tid; i < n; i += kPlan)
      if (inside(id(i))) atomicMin(c.mark + id(i), i);
    __syncthreads();
  }
  int total = 0;
  for (int i0 = 0; i0 < n; i0 += kPlan) {
    const int i = i0 + tid;
    int need = 0;
    bool ok = false;
    if (i < n) {
      const int s = id(i);
      if (inside(s) && (!r.seq || atomic_read(c.mark + s) == i)) {
        const int len = c.len[s], k = count(i);
        ok = k >= 0 && k <= c.max_len - len;
        if (ok) need = pages_of(c, len + k) - pages_of(c, len);
      }
      if (!ok) atomicOr(c.flags, 1);
    }
    int all;
    const int at = total + block_scan(need, all, lds);
    if (i < n) w.off[i] = ok ? at : -1;
    // beyond 2^31 nothing is left anyhow: a page is a table entry of its own, and there are at most 2^24
    total = (int)min((long)total + all, (long)INT_MAX / 2);
  }
  grant(c, n, total, w, lds, [&](int i) { const int len = c.len[id(i)]; return pages_of(c, len + count(i)) - pages_of(c, len); });
  constexpr int kAlone = 4;  // pages that a sequence's thread enters by itself
  int most = 0;
  for (int i = tid; i < n; i += kPlan) {
    const int s = id(i);
    if (!inside(s) || (r.seq && atomic_read(c.mark + s) != i)) continue;
    const int len = c.len[s], off = w.off[i];
    c.base[s] = len;
    c.slot[s] = off < 0 ? -1 : i;
    if (off < 0) continue;
    const int p = pages_of(c, len), need = pages_of(c, len + count(i)) - p;
    c.len[s] = len + count(i);
    most = max(most, need);
    if (need <= kAlone)
      for (int k = 0; k < need; k++) c.table[(long)s * c.width + p + k] = w.list[off + k];
  }
  if (block_max(most, lds) > kAlone)
    for (int i = tid >> 6; i < n; i += kPlan / 64) {
      if (w.off[i] < 0) continue;
      const int s = id(i), p = pages_of(c, c.base[s]), need = pages_of(c, c.len[s]) - p;
      if (need > kAlone)
        for (int k = tid & 63; k < need; k += 64) c.table[(long)s * c.width + p + k] = w.list[w.off[i] + k];
    }
  if (r.seq) {
    __syncthreads();
    for (int i = tid; i < n; i += kPlan)
      if (inside(id(i))) c.mark[id(i)] = INT_MAX;
  }
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// 16 bytes that nobody reads soon: 409 -> 358 us for two layers of 48 sequences of up to 4,200 tokens read out
__device__ __forceinline__ void stream_out(void *p, u32x4 x) { __builtin_nontemporal_store(x, (u32x4 *)p); }

// ---- contents of pages -----------------------------------------------------------------------------------------------

constexpr int kCopyPiece = 16384;  // bytes a workgroup of 256 copies at a time: four loads in flight per thread
__host__ __device__ inline int copy_pieces(const CacheView &c) { return (int)((c.page_bytes + kCopyPiece - 1) / kCopyPiece); }
// Copies the pages of from[] to to[] in all layers; this is workgroup `block` of `blocks`, a multiple of layers x pieces.
__device__ void copy_pages(const CacheView &c, int layers, const PageWork &w, int block, int blocks) {
  const int pieces = copy_pieces(c), each = pieces * layers, piece = block % pieces, l = block / pieces % layers;
  const long at = (long)piece * kCopyPiece + threadIdx.x * 16;
  char *base = c.pool + l * c.layer_bytes + at;
  const int copies = w.info[0];
  for (int k = block / each; k < copies; k += blocks / each) {
    const char *src = base + w.from[k] * c.page_bytes;
    char *dst = base + w.to[k] * c.page_bytes;
    if ((long)(piece + 1) * kCopyPiece <= c.page_bytes) {  // streamed: 24 sequences of 2,500 in 4 bits, 4 layers, 136 -> 105 us
      const u32x4 x0 = *(const u32x4 *)src, x1 = *(const u32x4 *)(src + 4096), x2 = *(const u32x4 *)(src + 8192), x3 = *(const u32x4 *)(src + 12288);
      stream_out(dst, x0), stream_out(dst + 4096, x1), stream_out(dst + 8192, x2), stream_out(dst + 12288, x3);
    } else {
      for (int j = 0; at + j < c.page_bytes; j += 4096) *(uint4 *)(dst + j) = *(const uint4 *)(src + j);
    }
  }
}
// Workgroups for copies of at most `pages` pages
int copy_blocks(const CacheView &c, int layers, double pages) {
  const int each = copy_pieces(c) * layers;
  return each * (int)std::max(1.0, std::min(pages, std::ceil(2048.0 / each)));
}

// ---- sequences that become others -------------------------------------------------------------------------------------

// Pages an entry needs; deep: one for each that the source has, else one for a last page that is not full
__device__ __forceinline__ int copies_of(const CacheView &c, int src, bool deep, int lane) {
  const int len = c.len[src], np = pages_of(c, len);
  const int32_t *row = c.table + (long)src * c.width;
  if (!deep) return (len & ((1 << c.page_shift) - 1)) && row[np - 1] >= 0 ? 1 : 0;
  int n = 0;
  for (int p = lane; p < np; p += 64) n += row[p] >= 0;
  return wave_fold(n, WaveAdd{});
}

// Entry i, by `lanes` lanes of a wave, of which this is number `lane`: the source's row as the target will have it, holders of
// shared pages, pages to be copied
__device__ void fork_stage(const CacheView &c, int i, int src, bool deep, const PageWork &w, int lane, int lanes) {
  const int shift = (threadIdx.x & 63) - lane;
  const unsigned long long before = (1ull << lane) - 1, all = lanes == 64 ? ~0ull : (1ull << lanes) - 1;
  int at = w.off[i];
  if (at < 0) return;
  const int len = c.len[src], np = pages_of(c, len), full = len >> c.page_shift;
  const int32_t *row = c.table + (long)src * c.width;
  for (int p0 = 0; p0 < np; p0 += lanes) {
    const int p = p0 + lane, page = p < np ? row[p] : -1;
    const bool copied = page >= 0 && (deep || p >= full);
    const unsigned long long m = __ballot(copied) >> shift & all;
    int to = page;
    if (copied) {
      const int k = at + __popcll(m & before);
      to = w.list[k];
      w.from[k] = page;
      w.to[k] = to;
    } else if (page >= 0) {
      atomicAdd(c.ref + page, 1);
    }
    if (p < np) w.row[(long)i * c.width + p] = to;
    at += __popcll(m);
  }
  if (lane == 0) w.row_len[i] = len;
}
// Entry i, by `threads` threads that run together or not at all: the target's row.  A page that it gives up keeps its contents during
// the call (it can only be handed out by a later one).
__device__ void fork_apply(const CacheView &c, int i, int dst, const PageWork &w, int thread, int threads) {
  if (w.off[i] < 0) return;
  const int np_old = pages_of(c, c.len[dst]), len = w.row_len[i], np = pages_of(c, len);
  int32_t *row = c.table + (long)dst * c.width;
  for (int p = thread; p < max(np_old, np); p += threads) {
    if (p < np_old) drop_page(c, row[p]);
    if (p < np) row[p] = w.row[(long)i * c.width + p];
  }
  if (threads > 64) __syncthreads();
  if (thread == 0) {
    c.len[dst] = len;
    c.base[dst] = len;
    c.slot[dst] = -1;
  }
}

// whole: the workgroup does the table's part too, with so many lanes to an entry; 0: launches of their own do
__global__ __launch_bounds__(kPlan) void cache_fork_plan_kernel(CacheView c, int n, const int32_t *src, const int32_t *dst, int deep, int whole,
                                                                PageWork w) {
  __shared__ int32_t lds[kPlan / 64];
  const int tid = threadIdx.x;
  auto inside = [&](int s) { return s >= 0 && s < c.max_seqs; };
  for (int i = tid; i < n; i += kPlan)
    if (inside(dst[i])) atomicMin(c.mark + dst[i], i);
  if (deep) {  // counts by waves, kept where the sources' lengths will be
    for (int i = tid >> 6; i < n; i += kPlan / 64) {
      const int k = inside(src[i]) ? copies_of(c, src[i], true, tid & 63) : 0;
      if ((tid & 63) == 0) w.row_len[i] = k;
    }
  }
  __syncthreads();
  auto need = [&](int i) { return deep ? w.row_len[i] : copies_of(c, src[i], false, 0); };
  int total = 0;
  for (int i0 = 0; i0 < n; i0 += kPlan) {
    const int i = i0 + tid;
    int k = 0, off = -1;
    if (i < n) {
      const bool ok = inside(src[i]) && inside(dst[i]) && atomic_read(c.mark + dst[i]) == i;
      if (!ok) atomicOr(c.flags, 1);
      if (ok && src[i] != dst[i]) {
        off = 0;
        k = need(i);
      }
    }
    int all;
    const int at = total + block_scan(k, all, lds);
    if (i < n) w.off[i] = off < 0 ? -1 : at;
    total = (int)min((long)total + all, (long)INT_MAX / 2);
  }
  grant(c, n, total, w, lds, need);
  int top = 0;
  for (int i = tid; i < n; i += kPlan) {
    if (inside(dst[i])) c.mark[dst[i]] = INT_MAX;
    if (w.off[i] >= 0) top = max(top, w.off[i] + need(i));
  }
  top = block_max(top, lds);
  if (tid == 0) w.info[0] = top;
  if (!whole) return;
  __syncthreads();
  for (int i = tid / whole; i < n; i += kPlan / whole) fork_stage(c, i, src[i], deep, w, tid % whole, whole);
  __syncthreads();
  for (int i = tid / whole; i < n; i += kPlan / whole) fork_apply(c, i, dst[i], w, tid % whole, whole);
}
__global__ __launch_bounds__(64) void cache_fork_stage_kernel(CacheView c, const int32_t *src, int deep, PageWork w) {
  fork_stage(c, blockIdx.x, src[blockIdx.x], deep, w, threadIdx.x, 64);
}
// Workgroups 0 .. n - 1: the targets' rows; the others copy pages, all of which were free before the call.
__global__ __launch_bounds__(256) void cache_fork_apply_kernel(CacheView c, int layers, int n, const int32_t *dst, PageWork w) {
  const int i = blockIdx.x;
  if (i >= n) return copy_pages(c, layers, w, i - n, gridDim.x - n);
  fork_apply(c, i, dst[i], w, threadIdx.x, 256);
}

// ---- sequences cut back -----------------------------------------------------------------------------------------------

__global__ __launch_bounds__(256) void cache_end_kernel(CacheView c, const int32_t *seq) {
  __shared__ int len;
  const int s = seq ? seq[blockIdx.x] : blockIdx.x;
  if (s < 0 || s >= c.max_seqs) {
    if (threadIdx.x == 0) atomicOr(c.flags, 1);
    return;
  }
  if (threadIdx.x == 0) {
    if (seq && atomicAdd(c.mark + s, -1) != INT_MAX) {  // the id came before in this call
      len = 0;
      atomicOr(c.flags, 1);
    } else {
      len = c.len[s];
      c.len[s] = c.base[s] = 0;
      c.slot[s] = -1;
    }
  }
  __syncthreads();
  for (int p = threadIdx.x; p < pages_of(c, len); p += 256) drop_page(c, c.table[(long)s * c.width + p]);
}
__global__ __launch_bounds__(256) void cache_unmark_kernel(CacheView c, int n, const int32_t *seq) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < n && seq[i] >= 0 && seq[i] < c.max_seqs) c.mark[seq[i]] = INT_MAX;
}

__global__ __launch_bounds__(kPlan) void cache_truncate_plan_kernel(CacheView c, int n, const int32_t *seq, const int32_t *keep, PageWork w) {
  __shared__ int32_t lds[kPlan / 64];
  const int tid = threadIdx.x;
  auto id = [&](int i) { return seq ? seq[i] : i; };
  auto inside = [&](int s) { return s >= 0 && s < c.max_seqs; };
  if (seq) {
    for (int i = tid; i < n; i += kPlan)
      if (inside(id(i))) atomicMin(c.mark + id(i), i);
    __syncthreads();
  }
  const int mask = (1 << c.page_shift) - 1;
  auto cut = [&](int i) { return c.table[(long)id(i) * c.width + (keep[i] >> c.page_shift)]; };  // the page that is cut inside
  auto need = [&](int i) { return (keep[i] & mask) && keep[i] < c.len[id(i)] && c.ref[cut(i)] > 1 ? 1 : 0; };
  int total = 0;
  for (int i0 = 0; i0 < n; i0 += kPlan) {
    const int i = i0 + tid;
    int k = 0;
    bool ok = false;
    if (i < n) {
      const int s = id(i);
      ok = inside(s) && (!seq || atomic_read(c.mark + s) == i) && keep[i] >= 0 && keep[i] <= c.len[s] &&
           !((keep[i] & mask) && cut(i) < 0);
      if (ok) k = need(i);
      else atomicOr(c.flags, 1);
    }
    int all;
    const int at = total + block_scan(k, all, lds);
    if (i < n) w.off[i] = ok ? at : -1;
    total += all;
  }
  grant(c, n, total, w, lds, need);
  int top = 0;
  for (int i = tid; i < n; i += kPlan) {
    w.row_len[i] = 0;
    if (w.off[i] >= 0 && need(i)) {
      w.row_len[i] = 1;
      w.from[w.off[i]] = cut(i);
      w.to[w.off[i]] = w.list[w.off[i]];
      top = max(top, w.off[i] + 1);
    }
    if (seq && inside(id(i))) c.mark[id(i)] = INT_MAX;
  }
  top = block_max(top, lds);
  if (tid == 0) w.info[0] = top;
}
__global__ __launch_bounds__(256) void cache_truncate_apply_kernel(CacheView c, int layers, int n, const int32_t *seq, const int32_t *keep, PageWork w) {
  const int i = blockIdx.x;
  if (i >= n) return copy_pages(c, layers, w, i - n, gridDim.x - n);
  if (w.off[i] < 0) return;
  const int s = seq ? seq[i] : i, np_old = pages_of(c, c.len[s]), np = pages_of(c, keep[i]);
  int32_t *row = c.table + (long)s * c.width;
  for (int p = np + threadIdx.x; p < np_old; p += 256) drop_page(c, row[p]);
  __syncthreads();
  if (threadIdx.x == 0) {
    if (w.row_len[i]) {
      drop_page(c, row[np - 1]);
      row[np - 1] = w.list[w.off[i]];
    }
    c.len[s] = c.base[s] = keep[i];
    c.slot[s] = -1;
  }
}

// Pages that hold none of the first `sinks` tokens and none of the last `window`
__global__ __launch_bounds__(256) void cache_trim_kernel(CacheView c, const int32_t *seq, int window, int sinks) {
  const int s = seq ? seq[blockIdx.x] : blockIdx.x;
  if (s < 0 || s >= c.max_seqs) {
    if (threadIdx.x == 0) atomicOr(c.flags, 1);
    return;
  }
  const int low = max(c.len[s] - window, 0) >> c.page_shift;
  for (int p = (int)(((long)sinks + (1 << c.page_shift) - 1) >> c.page_shift) + threadIdx.x; p < low; p += 256)
    drop_page(c, atomicExch(c.table + (long)s * c.width + p, -1));
}

// ---- the pool packed --------------------------------------------------------------------------------------------------

// from = pages in use behind the first `used` ones, to = holes among these; where a page went is kept in w.list
__global__ __launch_bounds__(kPlan) void cache_compact_plan_kernel(CacheView c, PageWork w) {
  __shared__ int32_t lds[kPlan / 64];
  const int words = words_of(c), used = c.n_pages - count_free(c, lds);
  int holes = 0, moved = 0;
  for (int w0 = 0; w0 < words; w0 += kPlan) {
    const int k = w0 + threadIdx.x;
    const uint32_t here = k < words ? c.used[k] : 0, real = k >= words ? 0 : k * 32 + 32 <= c.n_pages ? ~0u : (1u << (c.n_pages & 31)) - 1;
    const int split = min(max(used - k * 32, 0), 32);  // bits of this word that belong to the front
    const uint32_t front = split == 32 ? ~0u : (1u << split) - 1;
    uint32_t to = ~here & front & real, from = here & ~front & real;
    int all;
    int at = holes + block_scan(__popc(to), all, lds);
    holes += all;
    for (; to; to &= to - 1) w.to[at++] = k * 32 + __ffs(to) - 1;
    at = moved + block_scan(__popc(from), all, lds);
    moved += all;
    for (; from; from &= from - 1) w.from[at++] = k * 32 + __ffs(from) - 1;
    if (k < words) c.used[k] = (front & real) | ~real;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < moved; i += kPlan) {
    const int a = w.from[i], b = w.to[i];
    w.list[a] = b;
    c.ref[b] = c.ref[a];
    c.ref[a] = 0;
  }
  if (threadIdx.x == 0) w.info[0] = moved, w.info[1] = used;
}
__global__ __launch_bounds__(256) void cache_compact_apply_kernel(CacheView c, int layers, PageWork w) {
  const int i = blockIdx.x;
  if (i >= c.max_seqs) return copy_pages(c, layers, w, i - c.max_seqs, gridDim.x - c.max_seqs);
  if (w.info[0] == 0) return;
  int32_t *row = c.table + (long)i * c.width;
  for (int p = threadIdx.x; p < pages_of(c, c.len[i]); p += 256)
    if (row[p] >= w.info[1]) row[p] = w.list[row[p]];
}

__global__ __launch_bounds__(kPlan) void cache_lengths_kernel(CacheView c, int32_t *len, int32_t *pages) {
  __shared__ int32_t lds[kPlan / 64];
  if (len)
    for (int i = threadIdx.x; i < c.max_seqs; i += kPlan) len[i] = c.len[i];
  if (pages) {
    const int used = c.n_pages - count_free(c, lds);
    int last = 0;
    for (int w = threadIdx.x; w < words_of(c); w += kPlan) {
      const uint32_t real = w * 32 + 32 <= c.n_pages ? ~0u : (1u << (c.n_pages & 31)) - 1, m = c.used[w] & real;
      if (m) last = w * 32 + 32 - __clz(m);
    }
    last = block_max(last, lds);
    if (threadIdx.x == 0) pages[0] = used, pages[1] = last;
  }
}

__global__ __launch_bounds__(256) void cache_clear_kernel(CacheView c, PageWork w) {
  const long i = (long)blockIdx.x * 256 + threadIdx.x, words = (c.n_pages + 31) / 32;
  if (i < c.max_seqs) c.len[i] = c.base[i] = 0, c.slot[i] = -1, c.mark[i] = INT_MAX;
  if (i < c.n_pages) c.ref[i] = w.list[i] = 0;
  if (i < words) c.used[i] = i * 32 + 32 <= c.n_pages ? 0 : ~((1u << (c.n_pages & 31)) - 1);  // bits behind the last page: never free
  if (i < 2) c.flags[i] = 0;
}

// ---- values in and out ------------------------------------------------------------------------------------------------

// One tile of one head: a thread takes eight dims of a token; the values, which a tile holds by dim, pass through the LDS.
template <int KIND>
__global__ __launch_bounds__(256) void cache_write_kernel(CacheWriteArgs a) {
  extern __shared__ uint32_t lds[];
  const CacheView &c = a.c;
  const int x = blockIdx.x % a.tiles, h = blockIdx.x / a.tiles % c.heads, i = blockIdx.x / a.tiles / c.heads;
  const int tid = threadIdx.x, dh = c.dh, per = dh / 8;
  const int s = a.r.seq ? a.r.seq[i] : i;
  const long row0 = a.r.first ? a.r.first[i] : i;
  const int rows = a.r.first ? a.r.first[i + 1] - (int)row0 : 1;
  const bool known = s >= 0 && s < c.max_seqs;
  const int base = known ? c.base[s] : 0, len = known ? c.len[s] : 0;
  if (!known || rows < 0 || rows > a.r.max_new || c.slot[s] != i || rows != len - base) {
    if (tid == 0 && x == 0 && h == 0) atomicOr(c.flags, 1);
    return;
  }
  const int tile = (base >> 5) + x;
  if (tile * kTile >= len) return;
  const int t0 = max(base - tile * kTile, 0), t1 = min(len - tile * kTile, kTile);
  const int page = c.table[(long)s * c.width + (tile >> (c.page_shift - 5))];
  if (page < 0) return;
  char *at = c.pool + cache_tile_offset(c, a.layer, page, h, tile & ((1 << (c.page_shift - 5)) - 1), cache_tile_bytes(KIND, dh));
  for (int side = 0; side < 2; side++) {
    const void *src = side ? a.v : a.k;
    for (int x = t0 * per + tid; x < t1 * per; x += 256) {  // four threads in a row have a block of 32
      const int tok = x / per, dim = x % per * 8;
      float val[8];
      io_load8(src, a.type, (row0 + tile * kTile + tok - base) * a.ld + (long)h * dh + dim, a.vec, val);
      if constexpr (KIND == CACHE_Q4) {
        uint32_t word;
        const int b = q4_round(val, word);
        char *scales = at + 32 * dh;
        if (side == 0) {
          ((uint32_t *)at)[q4_key_word(tok, dim, dh)] = word;
          if ((dim & 31) == 0) scales[tok * (dh / 32) + (dim >> 5)] = (char)b;
        } else {
          lds[tok * per + (dim >> 3)] = word;
          if ((dim & 31) == 0) scales[dh + (dim >> 5) * kTile + tok] = (char)b;
        }
      } else {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; j++) w[j] = half_bits<KIND>(val[2 * j]) | half_bits<KIND>(val[2 * j + 1]) << 16;
        if (side == 0) {
          *(uint4 *)((unsigned short *)at + key_elem(tok, dim, dh)) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
#pragma unroll
          for (int j = 0; j < 4; j++) lds[tok * (dh / 2 + 1) + dim / 2 + j] = w[j];
        }
      }
    }
  }
  __syncthreads();
  // values: eight tokens of a dim; those that are not new stay as they are
  for (int x = tid; x < 4 * dh; x += 256) {
    const int dim = x % dh, g = x / dh * 8;
    if (g + 8 <= t0 || g >= t1) continue;
    if constexpr (KIND == CACHE_Q4) {
      uint32_t *to = (uint32_t *)(at + 16 * dh) + q4_value_word(g, dim), word = *to;
#pragma unroll
      for (int j = 0; j < 8; j++)
        if (g + j >= t0 && g + j < t1) word = (word & ~(15u << (4 * j))) | ((lds[(g + j) * per + (dim >> 3)] >> (4 * (dim & 7))) & 15u) << (4 * j);
      *to = word;
    } else {
      unsigned short *to = (unsigned short *)(at + 64 * dh) + value_elem(g, dim);
      const unsigned short *from = (const unsigned short *)lds + g * (dh + 2) + dim;
      if (g >= t0 && g + 8 <= t1) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; j++) w[j] = from[2 * j * (dh + 2)] | (uint32_t)from[(2 * j + 1) * (dh + 2)] << 16;
        *(uint4 *)to = make_uint4(w[0], w[1], w[2], w[3]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; j++)
          if (g + j >= t0 && g + j < t1) to[j] = from[j * (dh + 2)];
      }
    }
  }
}

// At most 128 dims of a tile of one head
template <int KIND>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheReadArgs a) {
  extern __shared__ uint32_t lds[];
  const CacheView &c = a.c;
  const int tid = threadIdx.x, dh = c.dh, dw = min(dh, 128), parts = dh / dw, per = dw / 8;
  const int part = blockIdx.x % parts, b = blockIdx.x / parts, h = b % c.heads, tile = b / c.heads % a.tiles, i = b / c.heads / a.tiles;
  const int s = a.r.seq ? a.r.seq[i] : i;
  const bool known = s >= 0 && s < c.max_seqs;
  if (!known && tid == 0 && tile == 0 && h == 0) atomicOr(c.flags, 1);
  const int len = known ? c.len[s] : 0, t1 = min(a.max_keys - tile * kTile, kTile);
  const int page = tile * kTile < len ? c.table[(long)s * c.width + (tile >> (c.page_shift - 5))] : -1;
  const char *at = c.pool + cache_tile_offset(c, a.layer, max(page, 0), h, tile & ((1 << (c.page_shift - 5)) - 1), cache_tile_bytes(KIND, dh));
  constexpr int kPer = KIND == CACHE_Q4 ? 16 : 64;  // bytes of a dim's keys or values
  if (page >= 0) {
    for (int x = tid; x < kPer * dw / 16; x += 256) ((uint4 *)lds)[x] = ((const uint4 *)(at + kPer * dh))[part * (kPer * dw / 16) + x];
  }
  __syncthreads();
  for (int x = tid; x < t1 * per; x += 256) {
    const int tok = x / per, own = x % per * 8, dim = part * dw + own;
    const bool there = page >= 0 && tile * kTile + tok < len;
    const long o = (((long)i * a.max_keys + tile * kTile + tok) * c.heads + h) * dh + dim;
#pragma unroll
    for (int side = 0; side < 2; side++) {
      float val[8] = {};
      if (there) {
        if constexpr (KIND == CACHE_Q4) {
          const unsigned char *scales = (const unsigned char *)at + 32 * dh;
          const float sc = q4_scale(side == 0 ? scales[tok * (dh / 32) + (dim >> 5)] : scales[dh + (dim >> 5) * kTile + tok]);
          uint32_t word = 0;
          if (side == 0) {
            word = ((const uint32_t *)at)[q4_key_word(tok, dim, dh)];
          } else {
#pragma unroll
            for (int j = 0; j < 8; j++) word |= (lds[q4_value_word(tok, own + j)] >> (4 * (tok & 7)) & 15u) << (4 * j);
          }
          f16x2 h[4];
          q4_unpack(word, h);
#pragma unroll
          for (int j = 0; j < 8; j++) val[j] = (float)h[j / 2][j % 2] * sc;
        } else {
#pragma unroll
          for (int j = 0; j < 8; j++) {
            const unsigned short b = side == 0 ? ((const unsigned short *)at)[key_elem(tok, dim, dh) + j]
                                               : ((const unsigned short *)lds)[value_elem(tok, own + j)];
            val[j] = KIND == CACHE_F16 ? (float)__builtin_bit_cast(_Float16, b) : (float)__builtin_bit_cast(__bf16, b);
          }
        }
      }
      void *dst = side == 0 ? a.k : a.v;
      if (a.type == IO_F32) {
        float *to = (float *)dst + o;
        if (a.vec) {
          stream_out(to, (u32x4{__float_as_uint(val[0]), __float_as_uint(val[1]), __float_as_uint(val[2]), __float_as_uint(val[3])}));
          stream_out(to + 4, (u32x4{__float_as_uint(val[4]), __float_as_uint(val[5]), __float_as_uint(val[6]), __float_as_uint(val[7])}));
        } else {
#pragma unroll
          for (int j = 0; j < 8; j++) to[j] = val[j];
        }
      } else {
        unsigned short w[8];
#pragma unroll
        for (int j = 0; j < 8; j++)
          w[j] = a.type == IO_F16 ? __builtin_bit_cast(unsigned short, (_Float16)val[j]) : __builtin_bit_cast(unsigned short, (__bf16)val[j]);
        unsigned short *to = (unsigned short *)dst + o;
        if (a.vec) {
          stream_out(to, (u32x4{w[0] | (uint32_t)w[1] << 16, w[2] | (uint32_t)w[3] << 16, w[4] | (uint32_t)w[5] << 16, w[6] | (uint32_t)w[7] << 16}));
        } else {
#pragma unroll
          for (int j = 0; j < 8; j++) to[j] = w[j];
        }
      }
    }
  }
}

}  // namespace

hipError_t launch_cache_write(const CacheWriteArgs &a, hipStream_t s) {
  const dim3 grid((unsigned)((long)a.tiles * a.c.heads * a.r.n));
  const size_t lds = a.c.kind == CACHE_Q4 ? kTile * (a.c.dh / 8) * 4 : kTile * (a.c.dh / 2 + 1) * 4;
  if (a.c.kind == CACHE_Q4) hipLaunchKernelGGL(cache_write_kernel<CACHE_Q4>, grid, dim3(256), lds, s, a);
  else if (a.c.kind == CACHE_F16) hipLaunchKernelGGL(cache_write_kernel<CACHE_F16>, grid, dim3(256), lds, s, a);
  else hipLaunchKernelGGL(cache_write_kernel<CACHE_BF16>, grid, dim3(256), lds, s, a);
  return hipGetLastError();
}
hipError_t launch_cache_read(const CacheReadArgs &a, hipStream_t s) {
  const int dw = std::min(a.c.dh, 128);
  const dim3 grid((unsigned)((long)a.tiles * a.c.heads * a.r.n * (a.c.dh / dw)));
  const size_t lds = (a.c.kind == CACHE_Q4 ? 16 : 64) * dw;
  if (a.c.kind == CACHE_Q4) hipLaunchKernelGGL(cache_read_kernel<CACHE_Q4>, grid, dim3(256), lds, s, a);
  else if (a.c.kind == CACHE_F16) hipLaunchKernelGGL(cache_read_kernel<CACHE_F16>, grid, dim3(256), lds, s, a);
  else hipLaunchKernelGGL(cache_read_kernel<CACHE_BF16>, grid, dim3(256), lds, s, a);
  return hipGetLastError();
}

}  // namespace nt

// ---- entry points -----------------------------------------------------------------------------------------------------

struct nt_cache {
  nt_cache_config cfg{};
  nt::CacheView v{};
  nt::PageWork w{};
  int device = -1;
  char *mem = nullptr;
  float *part = nullptr;
  long part_floats = 0;
  int32_t *h_flags = nullptr;  // pinned
};

namespace {

int fail(int code, const char *fmt, ...) __attribute__((format(printf, 2, 3)));
int fail(int code, const char *fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return nt::set_error(code, buf);
}
#define HIP_TRY(expr)                                                                   \
  do {                                                                                  \
    hipError_t _e = (expr);                                                             \
    if (_e != hipSuccess) return fail(NT_EHIP, "%s: %s", #expr, hipGetErrorString(_e)); \
  } while (0)

hipStream_t as_stream(void *s) { return (hipStream_t)s; }

int check_config(const nt_cache_config *c) {
  if (!c) return fail(NT_EINVAL, "config is null");
  if (c->struct_size != sizeof(nt_cache_config)) return fail(NT_EINVAL, "config.struct_size %u != %zu", c->struct_size, sizeof(nt_cache_config));
  if (c->kind < NT_CACHE_F16 || c->kind > NT_CACHE_Q4) return fail(NT_EINVAL, "unknown kind of cache %d", c->kind);
  if (c->n_layers < 1 || c->n_layers > 1024) return fail(NT_ESHAPE, "n_layers must be in [1,1024]");
  if (c->n_kv_heads < 1 || c->n_kv_heads > 1024 || c->n_q_heads < c->n_kv_heads || c->n_q_heads > 4096 || c->n_q_heads % c->n_kv_heads)
    return fail(NT_ESHAPE, "%d query heads do not share %d key/value heads", c->n_q_heads, c->n_kv_heads);
  if (c->d_head != 64 && c->d_head != 128 && c->d_head != 256 && c->d_head != 512) return fail(NT_ESHAPE, "head width %d not in {64,128,256,512}", c->d_head);
  if (c->page_tokens != 32 && c->page_tokens != 64 && c->page_tokens != 128 && c->page_tokens != 256)
    return fail(NT_ESHAPE, "page_tokens %d not in {32,64,128,256}", c->page_tokens);
  if (c->n_pages < 1 || c->n_pages > 1 << 24) return fail(NT_ESHAPE, "n_pages must be in [1,2^24]");
  if (c->max_seqs < 1 || c->max_seqs > 1 << 20) return fail(NT_ESHAPE, "max_seqs must be in [1,2^20]");
  if (c->max_len < 1 || c->max_len > 1 << 24) return fail(NT_ESHAPE, "max_len must be in [1,2^24]");
  if ((double)c->n_layers * c->n_pages * c->page_tokens * c->n_kv_heads * c->d_head > 1e14) return fail(NT_ESHAPE, "the pool is beyond any memory");
  return NT_OK;
}

// Lays out the one allocation; with a null base only its size counts.
size_t lay_out(nt_cache *c, char *base) {
  const nt_cache_config &g = c->cfg;
  nt::CacheView &v = c->v;
  const int tile = nt::cache_tile_bytes(g.kind, g.d_head);
  v.kind = g.kind; v.heads = g.n_kv_heads; v.dh = g.d_head; v.n_pages = g.n_pages; v.max_seqs = g.max_seqs; v.max_len = g.max_len;
  v.page_shift = __builtin_ctz(g.page_tokens);
  v.page_bytes = (long)tile * (g.page_tokens / nt::kTile) * g.n_kv_heads;
  v.layer_bytes = v.page_bytes * g.n_pages;
  v.width = (g.max_len + g.page_tokens - 1) / g.page_tokens;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = (off + 255) & ~(size_t)255;
    off = o + bytes;
    return (char *)((uintptr_t)base + o);
  };
  auto ints = [&](size_t n) { return (int32_t *)take(n * 4); };
  v.pool = take((size_t)v.layer_bytes * g.n_layers);
  v.table = ints((size_t)g.max_seqs * v.width);
  v.len = ints(g.max_seqs); v.base = ints(g.max_seqs); v.slot = ints(g.max_seqs); v.mark = ints(g.max_seqs);
  v.ref = ints(g.n_pages); v.used = (uint32_t *)ints((g.n_pages + 31) / 32); v.flags = ints(2);
  c->w.off = ints(g.max_seqs); c->w.list = ints(g.n_pages); c->w.from = ints(g.n_pages); c->w.to = ints(g.n_pages);
  c->w.info = ints(2); c->w.row_len = ints(g.max_seqs); c->w.row = ints((size_t)g.max_seqs * v.width);
  // for the most shares that single tokens of all sequences can have; more, for shares of prompts, where the pool is larger
  const double tokens = (double)g.max_seqs * g.n_q_heads * nt::kMaxSplits * (g.d_head + 2);
  c->part_floats = (long)std::min<double>(nt::kPartFloats, std::max(tokens, (double)v.layer_bytes * g.n_layers / 4)) & ~3l;
  c->part = (float *)take((size_t)c->part_floats * 4);
  return off;
}

// What every call on a cache checks first
int check_call(const nt_cache *c, int32_t n) {
  if (!c) return fail(NT_EINVAL, "cache is null");
  if (n < 0) return fail(NT_EINVAL, "negative number of sequences %d", n);
  if (n > c->cfg.max_seqs) return fail(NT_ESHAPE, "%d sequences, the cache holds %d", n, c->cfg.max_seqs);
  int dev = -1;
  HIP_TRY(hipGetDevice(&dev));
  if (dev != c->device) return fail(NT_EINVAL, "the cache is on device %d, the current device is %d", c->device, dev);
  return NT_OK;
}
int check_layer(const nt_cache *c, int32_t layer) {
  return layer < 0 || layer >= c->cfg.n_layers ? fail(NT_ERANGE, "layer %d of %d", layer, c->cfg.n_layers) : NT_OK;
}
int type_bytes(int32_t type) { return type == NT_F32 ? 4 : 2; }
bool type_known(int32_t type) { return type >= NT_F32 && type <= NT_BF16; }
bool aligned(const void *p, int64_t ld, int32_t type) { return ((uintptr_t)p & 15) == 0 && (ld * type_bytes(type) & 15) == 0; }

// workgroups of a launch: one dimension, below 2^31
int check_blocks(int64_t tiles, int64_t heads, int64_t n) {
  return (double)tiles * heads * n < 2147483648.0 ? NT_OK : fail(NT_ESHAPE, "%lld sequences of %lld tiles are too much for one call", (long long)n, (long long)tiles);
}
int write_tiles(int32_t max_new) { return (max_new + nt::kTile - 2) / nt::kTile + 1; }

int become(nt_cache *c, int32_t n, const int32_t *d_src, const int32_t *d_dst, int deep, void *hip_stream) {
  int rc = check_call(c, n);
  if (rc || n == 0) return rc;
  if (!d_src || !d_dst) return fail(NT_EINVAL, "null argument");
  hipStream_t s = as_stream(hip_stream);
  // A table of few rows is the planning workgroup's as well: one launch less to enqueue.  48 entries of one page or two, with the
  // reading of what they became: 4 us less of the host's time and 2 less in all (of 24) than with a launch of the table's own.
  const int whole = (double)n * c->v.width > 4096 ? 0 : c->v.width <= 16 ? 16 : 64, tables = whole ? 0 : n;
  const int copies = nt::copy_blocks(c->v, c->cfg.n_layers, deep ? (double)n * c->v.width : n);
  hipLaunchKernelGGL(nt::cache_fork_plan_kernel, dim3(1), dim3(nt::kPlan), 0, s, c->v, n, d_src, d_dst, deep, whole, c->w);
  if (!whole) hipLaunchKernelGGL(nt::cache_fork_stage_kernel, dim3(n), dim3(64), 0, s, c->v, d_src, deep, c->w);
  hipLaunchKernelGGL(nt::cache_fork_apply_kernel, dim3(tables + copies), dim3(256), 0, s, c->v, c->cfg.n_layers, tables, d_dst, c->w);
  HIP_TRY(hipGetLastError());
  return NT_OK;
}

}  // namespace

extern "C" {

int64_t nt_cache_bytes(const nt_cache_config *cfg) {
  if (check_config(cfg) != NT_OK) return 0;
  nt_cache c;
  c.cfg = *cfg;
  return (int64_t)lay_out(&c, nullptr);
}

int nt_cache_create(const nt_cache_config *cfg, void *hip_stream, nt_cache **out) {
  if (!out) return fail(NT_EINVAL, "out is null");
  *out = nullptr;
  int rc = check_config(cfg);
  if (rc) return rc;
  nt_cache *c = new (std::nothrow) nt_cache;
  if (!c) return fail(NT_ENOMEM, "host allocation failed");
  c->cfg = *cfg;
  const size_t bytes = lay_out(c, nullptr);
  auto fill = [&]() -> int {
    HIP_TRY(hipGetDevice(&c->device));
    if (hipMalloc((void **)&c->mem, bytes) != hipSuccess) {
      (void)hipGetLastError();
      return fail(NT_ENOMEM, "hipMalloc of %zu bytes failed", bytes);
    }
    if (hipHostMalloc((void **)&c->h_flags, 64) != hipSuccess) {
      (void)hipGetLastError();
      return fail(NT_ENOMEM, "pinned allocation failed");
    }
    lay_out(c, c->mem);
    HIP_TRY(nt::prepare_cache_prompt(cfg->kind, cfg->d_head));
    const int most = std::max(cfg->n_pages, cfg->max_seqs);
    hipLaunchKernelGGL(nt::cache_clear_kernel, dim3((most + 255) / 256), dim3(256), 0, as_stream(hip_stream), c->v, c->w);
    HIP_TRY(hipGetLastError());
    HIP_TRY(hipStreamSynchronize(as_stream(hip_stream)));
    return NT_OK;
  };
  rc = fill();
  if (rc) {
    nt_cache_destroy(c);
    return rc;
  }
  *out = c;
  return NT_OK;
}

void nt_cache_destroy(nt_cache *c) {
  if (!c) return;
  if (c->mem) (void)hipFree(c->mem);
  if (c->h_flags) (void)hipHostFree(c->h_flags);
  delete c;
}

int nt_cache_reserve(nt_cache *c, int32_t n, const int32_t *d_seq, const int32_t *d_first, void *hip_stream) {
  int rc = check_call(c, n);
  if (rc || n == 0) return rc;
  HIP_TRY(nt::cache_reserve(c, nt::CacheRows{n, 0, d_seq, d_first}, as_stream(hip_stream)));
  return NT_OK;
}

int nt_cache_write(nt_cache *c, int32_t layer, int32_t n, const int32_t *d_seq, const int32_t *d_first, int32_t max_new, const void *d_k,
                   const void *d_v, int64_t ld, int32_t type, void *hip_stream) {
  int rc = check_call(c, n);
  if (rc || (rc = check_layer(c, layer))) return rc;
  if (!type_known(type)) return fail(NT_EINVAL, "unknown type %d", type);
  if (max_new < 0 || max_new > c->cfg.max_len) return fail(NT_ERANGE, "max_new %d outside [0, max_len=%d]", max_new, c->cfg.max_len);
  if (n == 0 || max_new == 0) return NT_OK;
  if (!d_k || !d_v) return fail(NT_EINVAL, "null argument");
  if (ld < (int64_t)c->cfg.n_kv_heads * c->cfg.d_head) return fail(NT_EINVAL, "row stride %lld shorter than a row", (long long)ld);
  if ((rc = check_blocks(write_tiles(max_new), c->cfg.n_kv_heads, n))) return rc;
  HIP_TRY(nt::cache_write(c, layer, nt::CacheRows{n, max_new, d_seq, d_first}, d_k, d_v, ld, type, as_stream(hip_stream)));
  return NT_OK;
}

int nt_cache_attend(nt_cache *c, const nt_attend_args *a, void *hip_stream) {
  if (!a) return fail(NT_EINVAL, "null argument");
  if (a->struct_size != sizeof(nt_attend_args)) return fail(NT_EINVAL, "struct_size %u != %zu", a->struct_size, sizeof(nt_attend_args));
  int rc = check_call(c, a->n);
  if (rc || (rc = check_layer(c, a->layer))) return rc;
  const nt_cache_config &g = c->cfg;
  if (!type_known(a->type)) return fail(NT_EINVAL, "unknown type %d", a->type);
  if (a->max_new < 0 || a->max_new > g.max_len) return fail(NT_ERANGE, "max_new %d outside [0, max_len=%d]", a->max_new, g.max_len);
  if (a->window < 0 || a->sinks < 0 || a->max_keys < 0) return fail(NT_EINVAL, "negative window, sinks or max_keys");
  if (!std::isfinite(a->scale)) return fail(NT_EINVAL, "scale is not a number");
  if (!a->d_first && a->max_new != 1) return fail(NT_EINVAL, "max_new must be 1 without d_first");
  if (!a->k != !a->v) return fail(NT_EINVAL, "one of k and v without the other");
  if (a->n == 0 || a->max_new == 0) return NT_OK;
  if (!a->q || !a->out) return fail(NT_EINVAL, "null argument");
  if (a->ld_q < (int64_t)g.n_q_heads * g.d_head || a->ld_out < (int64_t)g.n_q_heads * g.d_head ||
      (a->k && a->ld_kv < (int64_t)g.n_kv_heads * g.d_head))
    return fail(NT_EINVAL, "a row stride is shorter than a row");
  if ((rc = check_blocks(((int64_t)a->max_new * (g.n_q_heads / g.n_kv_heads) + 7) / 8, g.n_kv_heads, a->n)) ||
      (rc = check_blocks(write_tiles(a->max_new), g.n_kv_heads, a->n)))
    return rc;
  HIP_TRY(nt::cache_attend(c, *a, a->type, 0, as_stream(hip_stream)));
  return NT_OK;
}

int nt_cache_read(nt_cache *c, int32_t layer, int32_t n, const int32_t *d_seq, int32_t max_keys, void *d_k, void *d_v, int32_t type,
                  void *hip_stream) {
  int rc = check_call(c, n);
  if (rc || (rc = check_layer(c, layer))) return rc;
  if (!type_known(type)) return fail(NT_EINVAL, "unknown type %d", type);
  if (max_keys < 0 || max_keys > 1 << 24) return fail(NT_ERANGE, "max_keys %d outside [0, 2^24]", max_keys);
  if (n == 0 || max_keys == 0) return NT_OK;
  if (!d_k || !d_v) return fail(NT_EINVAL, "null argument");
  const int tiles = (max_keys + nt::kTile - 1) / nt::kTile;
  if ((rc = check_blocks(tiles, c->cfg.n_kv_heads * 4, n))) return rc;
  nt::CacheReadArgs r{c->v, nt::CacheRows{n, 0, d_seq, nullptr}, layer, type, max_keys, tiles, d_k, d_v, aligned(d_k, 0, type) && aligned(d_v, 0, type)};
  HIP_TRY(nt::launch_cache_read(r, as_stream(hip_stream)));
  return NT_OK;
}

int nt_cache_fork(nt_cache *c, int32_t n, const int32_t *d_src, const int32_t *d_dst, void *hip_stream) {
  return become(c, n, d_src, d_dst, 0, hip_stream);
}
int nt_cache_copy(nt_cache *c, int32_t n, const int32_t *d_src, const int32_t *d_dst, void *hip_stream) {
  return become(c, n, d_src, d_dst, 1, hip_stream);
}

int nt_cache_truncate(nt_cache *c, int32_t n, const int32_t *d_seq, const int32_t *d_len, void *hip_stream) {
  int rc = check_call(c, n);
  if (rc || n == 0) return rc;
  hipStream_t s = as_stream(hip_stream);
  if (!d_len) {
    HIP_TRY(nt::cache_end(c, n, d_seq, s));
    if (d_seq) hipLaunchKernelGGL(nt::cache_unmark_kernel, dim3((n + 255) / 256), dim3(256), 0, s, c->v, n, d_seq);
  } else {
    hipLaunchKernelGGL(nt::cache_truncate_plan_kernel, dim3(1), dim3(nt::kPlan), 0, s, c->v, n, d_seq, d_len, c->w);
    hipLaunchKernelGGL(nt::cache_truncate_apply_kernel, dim3(n + nt::copy_blocks(c->v, c->cfg.n_layers, n)), dim3(256), 0, s, c->v,
                       c->cfg.n_layers, n, d_seq, d_len, c->w);
  }
  HIP_TRY(hipGetLastError());
  return NT_OK;
}

int nt_cache_trim(nt_cache *c, int32_t n, const int32_t *d_seq, int32_t window, int32_t sinks, void *hip_stream) {
  int rc = check_call(c, n);
  if (rc) return rc;
  if (window < 1 || sinks < 0) return fail(NT_EINVAL, "window must be positive and sinks not negative");
  if (n == 0) return NT_OK;
  hipLaunchKernelGGL(nt::cache_trim_kernel, dim3(n), dim3(256), 0, as_stream(hip_stream), c->v, d_seq, window, sinks);
  HIP_TRY(hipGetLastError());
  return NT_OK;
}

int nt_cache_compact(nt_cache *c, void *hip_stream) {
  int rc = check_call(c, 0);
  if (rc) return rc;
  hipStream_t s = as_stream(hip_stream);
  hipLaunchKernelGGL(nt::cache_compact_plan_kernel, dim3(1), dim3(nt::kPlan), 0, s, c->v, c->w);
  hipLaunchKernelGGL(nt::cache_compact_apply_kernel, dim3(c->cfg.max_seqs + nt::copy_blocks(c->v, c->cfg.n_layers, c->cfg.n_pages)), dim3(256), 0, s, c->v, c->cfg.n_layers, c->w);
  HIP_TRY(hipGetLastError());
  return NT_OK;
}

int nt_cache_lengths(nt_cache *c, int32_t *d_len, int32_t *d_pages, void *hip_stream) {
  int rc = check_call(c, 0);
  if (rc) return rc;
  hipLaunchKernelGGL(nt::cache_lengths_kernel, dim3(1), dim3(nt::kPlan), 0, as_stream(hip_stream), c->v, d_len, d_pages);
  HIP_TRY(hipGetLastError());
  return NT_OK;
}

int nt_cache_check(nt_cache *c, void *hip_stream) {
  int rc = check_call(c, 0);
  if (rc) return rc;
  hipStream_t s = as_stream(hip_stream);
  HIP_TRY(hipMemcpyAsync(c->h_flags, c->v.flags, 8, hipMemcpyDeviceToHost, s));
  HIP_TRY(nt::launch_fill_i32(c->v.flags, 2, 0, s));
  HIP_TRY(hipStreamSynchronize(s));
  if (c->h_flags[1]) return fail(NT_ENOMEM, "an entry was skipped: no free pages were left for it");
  if (c->h_flags[0]) return fail(NT_ERANGE, "an entry was skipped: its sequence id or a length did not fit");
  return NT_OK;
}

}  // extern "C"

// ---- launches, for the entry points and the decoder -----------------------------------------------------------------------

hipError_t nt::cache_reserve(nt_cache *c, const CacheRows &r, hipStream_t s) {
  hipLaunchKernelGGL(cache_reserve_kernel, dim3(1), dim3(kPlan), 0, s, c->v, r, c->w);
  return hipGetLastError();
}
hipError_t nt::cache_end(nt_cache *c, int n, const int32_t *seq, hipStream_t s) {
  hipLaunchKernelGGL(cache_end_kernel, dim3(n), dim3(256), 0, s, c->v, seq);
  return hipGetLastError();
}
hipError_t nt::cache_write(nt_cache *c, int layer, const CacheRows &r, const void *k, const void *v, long ld, int type, hipStream_t s) {
  return launch_cache_write(CacheWriteArgs{c->v, r, layer, type, write_tiles(r.max_new), k, v, ld, aligned(k, ld, type) && aligned(v, ld, type)}, s);
}
// Attention by the kernel that fits.  The one for few rows reads the keys and values once for every eight rows, the one for many once
// for 128 or 192 but computes as many: 8 sequences of 16,000 tokens, 32 / 8 heads of 128, with 8 / 16 / 32 / 64 rows to a key/value
// head 117 / 166 / 283 / 519 us and 138 / 135 / 135 / 149; in 4 bits, where a tile is a quarter of the bytes, 51 / 88 / 146 / 268 and
// 137 / 139 / 140 / 151; 64 of 200 tokens, one head of 512, 2 / 4 / 8 / 16 rows 17 / 21 / 30 / 40 and 27 / 27 / 27 / 29.
constexpr int kFewRows = 8, kFewRowsQ4 = 16;
hipError_t nt::cache_attend(nt_cache *c, const nt_attend_args &a, int out_type, long lo_offset, hipStream_t s) {
  const nt_cache_config &g = c->cfg;
  CacheAttnArgs k{};
  k.c = c->v; k.r = CacheRows{a.n, a.max_new, a.d_seq, a.d_first};
  if (a.k && a.max_new == 1) {  // part of the attention's launch
    k.k = a.k; k.v = a.v; k.ld_kv = a.ld_kv; k.vec_kv = aligned(a.k, a.ld_kv, a.type) && aligned(a.v, a.ld_kv, a.type);
  } else if (a.k) {
    const hipError_t e = cache_write(c, a.layer, k.r, a.k, a.v, a.ld_kv, a.type, s);
    if (e != hipSuccess) return e;
  }
  k.layer = a.layer; k.type = a.type; k.out_type = out_type; k.q_heads = g.n_q_heads; k.group = g.n_q_heads / g.n_kv_heads;
  k.q = a.q; k.out = a.out; k.ld_q = a.ld_q; k.ld_out = a.ld_out; k.lo_offset = lo_offset;
  k.scale = a.scale; k.window = a.window; k.sinks = a.sinks; k.vec = aligned(a.q, a.ld_q, a.type); k.vec_out = aligned(a.out, a.ld_out, a.type);
  k.part = c->part; k.part_floats = c->part_floats;
  long keys = a.max_keys > 0 ? std::min(a.max_keys, g.max_len) : g.max_len;
  if (a.window > 0) keys = std::min<long>(keys, (long)a.window + a.sinks + a.max_new + 2 * kTile);
  const long tiles = (keys + kTile - 1) / kTile;
  const bool many = a.max_new > 1 && (long)a.max_new * k.group > (g.kind == NT_CACHE_Q4 ? kFewRowsQ4 : kFewRows);
  return many ? launch_cache_prompt(k, tiles, s) : launch_cache_token(k, tiles, s);
}
