// Eviction of the tokens that collected the least attention weight (include/grand.h: grand_cache_evict): the choice, one
// cluster of blocks per sequence and weight row, and the move of the kept tokens' rows.
//
// Choice: the keep - sinks - recent largest weights of the free tokens.  Weights become 32-bit keys in the order of the
// values.  Every block of a cluster has an equal run of the tokens and holds its keys in shared memory (where they fit; else
// it reads them anew); three passes count the keys' digits (11, 11 and 10 bits) from the top, each block adds up the
// cluster's counts, and narrow down to the smallest kept key T; then every key above T and the first ones equal to it are
// taken, in order of the tokens, each block knowing from the others' counts where its run of the list begins.  A token whose
// page is outside the pool is never kept; sinks and newest ones of that kind leave their places to the free tokens.
// Move: 2 x 2 x kept x row bytes, bound by memory.
#include <cooperative_groups.h>

#include "grand_cache.h"

namespace cg = cooperative_groups;

namespace grand {
namespace {

constexpr int kSelect = 1024, kBins = 2048, kMaxCluster = 8;   // (two digits a thread)
constexpr int kHeld = 24 * 1024;   // keys that a block holds
constexpr int kCopies = 8;

// Larger weight, larger key; -0 counts as 0 and a NaN as less than everything.  Key 0 is left to tokens without a page.
constexpr uint32_t kNoPage = 0;
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (!(w == w)) return 1u;
  const uint32_t u = __float_as_uint(w + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__global__ void __launch_bounds__(kSelect) select_kernel(const __grid_constant__ EvictArgs a) {
  extern __shared__ __align__(16) uint32_t shared[];   // counts; with a cluster the block's sums; keys
  // Weights crowd a few digits (the same powers of two, equal weights, zeros), and additions to one address wait for each
  // other: the lanes of a warp share kCopies counts of a digit.
  __shared__ uint32_t warp_sum[kSelect / 32], warp_equal[kSelect / 32];
  __shared__ uint32_t sh_digit, sh_left;
  __shared__ uint32_t counts[2];     // of this block's tokens: kept whatever the equal ones are, free and equal to T
  __shared__ uint32_t gaps;          // of its sinks and newest tokens: without a page
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = (int)cluster.block_rank(), blocks = (int)cluster.num_blocks();
  uint32_t* hist = shared;
  uint32_t* sums = hist + kCopies * kBins;              // of this block, one array for each pass: another block may still read the last one's
  uint32_t* held = blocks > 1 ? sums + 3 * kBins : sums;
  const int row = blockIdx.x / blocks, groups = (int)a.pool.groups, b = row / groups, g = row - b * groups;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  SeqView view = a.seq;
  view.cu = nullptr;
  const bool speaks = rank == 0 && g == 0 && tid == 0;
  const Seq s = load_seq(view, b, speaks ? a.status : nullptr);
  const int n = s.len, keep = (int)a.keep;
  int32_t* kept = a.kept + (int64_t)row * keep;
  const int32_t* table = a.seq.table + (int64_t)b * a.seq.table_stride;
  const bool fits = n <= keep;
  if (fits) {  // all stay if they have a page (every block looks at the whole table row: the cluster agrees)
    bool gap = false;
    for (int i = tid; i < (int)div_fast((uint32_t)(n + (int)a.pool.page.d - 1), a.pool.page); i += kSelect)
      gap |= page_of(table, (uint32_t)i, a.pool.num_pages, a.status) < 0;
    if (!__syncthreads_or(gap)) {
      if (speaks) a.lens_out[b] = n;
      for (int i = rank * kSelect + tid; i < keep; i += blocks * kSelect) kept[i] = i < n ? i : -1;
      return;
    }
  }
  // the free tokens (keep >= sinks + recent, so lo < hi); where all fit there are none
  const int lo = fits ? n : (int)a.sinks, hi = fits ? n : n - (int)a.recent;
  // this block's run: a multiple of 32 tokens per warp
  const int per_warp = (n + blocks * kSelect - 1) / (blocks * kSelect) * 32, per_block = per_warp * (kSelect / 32);
  const int j0 = min(rank * per_block, n), j1 = min(j0 + per_block, n);
  const int w0 = min(j0 + warp * per_warp, j1), w1 = min(w0 + per_warp, j1);   // and this warp's
  auto read_key = [&](int j) -> uint32_t {
    const uint32_t jp = div_fast((uint32_t)j, a.pool.page);
    const int p = page_of(table, jp, a.pool.num_pages, a.status);
    return p < 0 ? kNoPage : weight_key(__ldg(a.pool.weights + ((int64_t)p * groups + g) * a.pool.page.d + (j - (int)(jp * a.pool.page.d))));
  };
  const bool holds = per_block <= kHeld;
  auto key = [&](int j) -> uint32_t { return holds ? held[j - j0] : read_key(j); };
  auto is_free = [&](int j) { return j < w1 && j >= lo && j < hi; };
  uint32_t left = 0, prefix = 0;     // to take among the keys that start with `prefix`
  bool none = true, all = false;     // no free token is kept; all with a page are
  const int top = kBins - 2 - 2 * tid;   // the two digits of this thread, from the top
  uint32_t* mine = hist + (lane & (kCopies - 1)) * kBins;
  for (int i = tid; i < kCopies * kBins; i += kSelect) hist[i] = 0;
  if (tid == 0) gaps = 0;
  __syncthreads();
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    if (pass == 0) {
#pragma unroll 8
      for (int j = w0 + lane; j < w1; j += 32) {
        const uint32_t k = read_key(j);
        if (holds) held[j - j0] = k;
        if (k == kNoPage) {
          if (!is_free(j)) atomicAdd(&gaps, 1u);
        } else if (is_free(j)) {
          atomicAdd(&mine[k >> 21], 1u);
        }
      }
    } else {
      const int shift = pass == 1 ? 10 : 0;
#pragma unroll 4
      for (int j = w0 + lane; j < w1; j += 32) {
        const uint32_t k = key(j);
        if (is_free(j) && k != kNoPage && (k >> (pass == 1 ? 21 : 10)) == prefix) atomicAdd(&mine[(k >> shift) & (pass == 1 ? 2047u : 1023u)], 1u);
      }
    }
    __syncthreads();
    uint2 own = make_uint2(0, 0);
#pragma unroll
    for (int c = 0; c < kCopies; ++c) {
      uint2* h = reinterpret_cast<uint2*>(hist + c * kBins + top);
      own.x += h->x;
      own.y += h->y;
      *h = make_uint2(0, 0);
    }
    if (blocks > 1) {
      *reinterpret_cast<uint2*>(sums + pass * kBins + top) = own;
      cluster.sync();
      own = make_uint2(0, 0);
#pragma unroll
      for (int r = 0; r < kMaxCluster; ++r)
        if (r < blocks) {
          const uint2 v = *reinterpret_cast<const uint2*>(cluster.map_shared_rank(sums + pass * kBins, r) + top);
          own.x += v.x;
          own.y += v.y;
        }
    }
    if (pass == 0) {
      uint32_t without = gaps;
      if (blocks > 1) {
        without = 0;
        for (int r = 0; r < blocks; ++r) without += *cluster.map_shared_rank(&gaps, r);
      }
      left = (uint32_t)keep - ((uint32_t)(lo + n - hi) - without);
      none = left == 0;
    }
    // the digit at which the count from the top reaches `left`
    uint32_t incl = own.x + own.y;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, incl, o);
      if (lane >= o) incl += v;
    }
    if (lane == 31) warp_sum[warp] = incl;
    __syncthreads();
    uint32_t before = warp_sum[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, before, o);
      if (lane >= o) before += v;
    }
    if (pass == 0) {   // fewer free tokens than places?
      const uint32_t there = __shfl_sync(0xFFFFFFFFu, before, 31);
      all = there <= left;
      if (speaks) a.lens_out[b] = all ? keep - (int)(left - there) : keep;
    }
    before = __shfl_sync(0xFFFFFFFFu, before, warp) - warp_sum[warp];   // of the warps before this one
    const uint32_t above = before + incl - (own.x + own.y);
    if (above < left && left <= above + own.y) sh_digit = (uint32_t)top + 1, sh_left = left - above;
    else if (above + own.y < left && left <= above + own.y + own.x) sh_digit = (uint32_t)top, sh_left = left - above - own.y;
    __syncthreads();
    if (!none && !all) {
      prefix = (prefix << (pass == 0 ? 0 : pass == 1 ? 11 : 10)) | sh_digit;
      left = sh_left;
    }
  }
  if (none || all) prefix = none ? 0xFFFFFFFFu : kNoPage, left = 0;   // (no key is that large)
  // ---- how many tokens each warp's run has, and each block's, that are kept anyway (with a page, and not free or above T), and
  // how many are equal to T
  uint32_t above = 0, equal = 0;
#pragma unroll 4
  for (int j = w0 + lane; j < w1; j += 32) {
    const uint32_t k = key(j);
    if (k == kNoPage) continue;
    above += !is_free(j) || k > prefix;
    equal += is_free(j) && k == prefix;
  }
  above = __reduce_add_sync(0xFFFFFFFFu, above);
  equal = __reduce_add_sync(0xFFFFFFFFu, equal);
  if (lane == 0) warp_sum[warp] = above, warp_equal[warp] = equal;
  __syncthreads();
  uint32_t above0 = warp_sum[lane], equal0 = warp_equal[lane];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t u = __shfl_up_sync(0xFFFFFFFFu, above0, o), v = __shfl_up_sync(0xFFFFFFFFu, equal0, o);
    if (lane >= o) above0 += u, equal0 += v;
  }
  if (tid == 31) counts[0] = above0, counts[1] = equal0;
  above0 = __shfl_sync(0xFFFFFFFFu, above0, warp) - above;   // before this warp's run
  equal0 = __shfl_sync(0xFFFFFFFFu, equal0, warp) - equal;
  if (blocks > 1) {
    cluster.sync();
    for (int r = 0; r < rank; ++r) {
      const uint32_t* other = cluster.map_shared_rank(counts, r);
      above0 += other[0];
      equal0 += other[1];
    }
  } else {
    __syncthreads();
  }
  uint32_t at = above0 + min(equal0, left);   // kept before token w0
#pragma unroll 4
  for (int base = w0; base < w1; base += 32) {
    const int j = base + lane;
    const uint32_t k = j < w1 ? key(j) : kNoPage;
    const bool same = is_free(j) && k != kNoPage && k == prefix;
    const uint32_t me = __ballot_sync(0xFFFFFFFFu, same), below = (1u << lane) - 1;
    const bool take = k != kNoPage && (!is_free(j) || k > prefix || (same && equal0 + __popc(me & below) < left));
    equal0 += __popc(me);
    const uint32_t mt = __ballot_sync(0xFFFFFFFFu, take);
    const uint32_t to = at + __popc(mt & below);
    if (take && to < (uint32_t)keep) kept[to] = j;
    at += __popc(mt);
  }
  if (all) {   // behind the last: the tokens that are kept are the total of all blocks' runs
    uint32_t total = 0;
    for (int r = 0; r < blocks; ++r) total += blocks > 1 ? *cluster.map_shared_rank(counts, r) : counts[0];
    for (int i = (int)total + rank * kSelect + tid; i < keep; i += blocks * kSelect) kept[i] = -1;
  }
  if (blocks > 1) cluster.sync();  // no block leaves while another reads its counts
}

// Page and slot of token j; false if the table names no page of the pool.
__device__ __forceinline__ bool spot(const EvictArgs& a, const int32_t* row, int j, int& page, int& slot) {
  const uint32_t jp = div_fast((uint32_t)j, a.pool.page);
  page = page_of(row, jp, a.pool.num_pages, a.status);
  slot = j - (int)(jp * a.pool.page.d);
  return page >= 0;
}

// Into other pages: every kept row on its own.  A warp looks up 16 rows (one a lane, so that the three dependent reads of
// list, table and row overlap) and then moves their 16-byte pieces, four of the keys and four of the values at a time.
constexpr int kMoveRows = 16;
__global__ void __launch_bounds__(256) move_kernel(const __grid_constant__ EvictArgs a) {
  const int b = blockIdx.z, g = blockIdx.y, groups = gridDim.y;
  const int lane = threadIdx.x & 31;
  const int i0 = ((int)blockIdx.x * 8 + (int)(threadIdx.x >> 5)) * kMoveRows;
  if (i0 >= (int)a.keep) return;
  const int i = i0 + (lane & (kMoveRows - 1));
  const int j = i < (int)a.keep ? a.kept[((int64_t)b * groups + g) * a.keep + i] : -1;
  int sp = 0, ss = 0, dp = 0, ds = 0;
  const bool ok = j >= 0 && spot(a, a.seq.table + (int64_t)b * a.seq.table_stride, j, sp, ss) && spot(a, a.into + (int64_t)b * a.into_stride, i, dp, ds);
  if (ok && lane < kMoveRows)
    a.pool.weights[((int64_t)dp * groups + g) * a.pool.page.d + ds] = a.pool.weights[((int64_t)sp * groups + g) * a.pool.page.d + ss];
  const int h0 = groups == 1 ? 0 : g, heads = groups == 1 ? (int)a.pool.kv_heads : 1;
  const int per = (int)a.pool.dim / 8, total = heads * per;
  const int64_t from = ok ? sp * a.pool.page_stride + ss * a.pool.slot_stride : -1, to = dp * a.pool.page_stride + ds * a.pool.slot_stride;
  constexpr int kAhead = 4;
  for (int x0 = 0; x0 < kMoveRows * total; x0 += 32 * kAhead) {
    uint4 kk[kAhead], vv[kAhead];
    int64_t dst[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int x = x0 + u * 32 + lane, r = x / total, c = x - r * total, h = c / per;
      const int64_t f = __shfl_sync(0xFFFFFFFFu, from, r & (kMoveRows - 1)), t = __shfl_sync(0xFFFFFFFFu, to, r & (kMoveRows - 1));
      const int64_t e = (int64_t)(h0 + h) * a.pool.head_stride + (c - h * per) * 8;
      dst[u] = r < kMoveRows && f >= 0 ? (t + e) * 2 : -1;
      if (dst[u] >= 0) {
        kk[u] = *reinterpret_cast<const uint4*>(a.pool.k + (f + e) * 2);
        vv[u] = *reinterpret_cast<const uint4*>(a.pool.v + (f + e) * 2);
      }
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (dst[u] >= 0) {
        *reinterpret_cast<uint4*>(a.pool.k + dst[u]) = kk[u];
        *reinterpret_cast<uint4*>(a.pool.v + dst[u]) = vv[u];
      }
  }
}

// In place: a kept token never moves up (kept[i] >= i), so a block that goes through the tokens in order, reading a tile
// whole before it writes it, overwrites only rows that it has read.  Blocks share nothing: each has one 32-byte column
// of one head's keys or values, or the weights, of one sequence.
// A tile is two threads a row, kDeep rows a pair of threads: it waits for its reads, so large tiles pay (65,536 of 131,072
// tokens of 8 heads: 542 us with 256 threads and 4 rows, 338 with 512 and 8).
constexpr int kSlide = 512, kDeep = 8;
__global__ void __launch_bounds__(kSlide) slide_kernel(const __grid_constant__ EvictArgs a, uint32_t columns) {
  const int b = blockIdx.z, g = blockIdx.y, groups = gridDim.y;
  const int heads = groups == 1 ? (int)a.pool.kv_heads : 1;
  const uint32_t col = blockIdx.x % columns, which = blockIdx.x / columns;  // which: 2 x head + (keys | values); the last: weights
  const bool weights = which == 2u * heads;
  if (weights && col != 0) return;
  SeqView view = a.seq;
  view.cu = nullptr;
  const Seq s = load_seq(view, b, nullptr);
  if (a.lens_out[b] == s.len) return;  // nothing moves
  const int32_t* table = a.seq.table + (int64_t)b * a.seq.table_stride;
  const int32_t* kept = a.kept + ((int64_t)b * groups + g) * a.keep;
  const int64_t head_at = (int64_t)((groups == 1 ? 0 : g) + (int)(which >> 1)) * a.pool.head_stride + col * 16 + (threadIdx.x & 1) * 8;
  uint8_t* base = which & 1 ? a.pool.v : a.pool.k;
  const int chunks = weights ? 1 : min(2, (int)a.pool.dim / 8 - (int)col * 2);
  const bool used = (int)(threadIdx.x & 1) < chunks;
  // places of a tile's rows, looked up while the tile before it moves; to < 0: stays
  int64_t from[kDeep], to[kDeep];
  auto find = [&](int i0) {
#pragma unroll
    for (int u = 0; u < kDeep; ++u) {
      const int i = i0 + u * (kSlide / 2) + (int)(threadIdx.x >> 1);
      to[u] = -1;
      if (i < (int)a.keep && used) {
        const int j = kept[i];
        int sp, ss, dp, ds;
        if (j > i && spot(a, table, j, sp, ss) && spot(a, table, i, dp, ds)) {
          from[u] = weights ? ((int64_t)sp * groups + g) * a.pool.page.d + ss : (sp * a.pool.page_stride + ss * a.pool.slot_stride + head_at) * 2;
          to[u] = weights ? ((int64_t)dp * groups + g) * a.pool.page.d + ds : (dp * a.pool.page_stride + ds * a.pool.slot_stride + head_at) * 2;
        }
      }
    }
  };
  find(0);
  for (int i0 = 0; i0 < (int)a.keep; i0 += kDeep * kSlide / 2) {
    uint4 x[kDeep];
    int64_t dst[kDeep];
#pragma unroll
    for (int u = 0; u < kDeep; ++u) {
      dst[u] = to[u];
      if (to[u] >= 0) {
        if (weights) x[u].x = __float_as_uint(a.pool.weights[from[u]]);
        else x[u] = *reinterpret_cast<const uint4*>(base + from[u]);
      }
    }
    find(i0 + kDeep * kSlide / 2);
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kDeep; ++u)
      if (dst[u] >= 0) {
        if (weights) a.pool.weights[dst[u]] = __uint_as_float(x[u].x);
        else *reinterpret_cast<uint4*>(base + dst[u]) = x[u];
      }
    __syncthreads();
  }
}

}  // namespace

cudaError_t launch_evict(const EvictArgs& a, cudaStream_t s) {
  static SmemOptIn done;
  if (cudaError_t e = allow_dynamic_smem(reinterpret_cast<const void*>(select_kernel), ((kCopies + 3) * kBins + kHeld) * 4, &done)) return e;
  // Blocks per row: as many as the card has room for, up to 8; a block with less than 4,096 tokens only adds barriers.
  const uint64_t rows = (uint64_t)a.pool.groups * a.seq.batch, longest = a.seq.max_len;
  uint32_t blocks = 1;
  while (blocks < kMaxCluster && rows * blocks * 2 <= (uint64_t)sm_count() && longest >= 4096ull * 2 * blocks) blocks *= 2;
  const uint64_t per_block = (longest + blocks * kSelect - 1) / (blocks * kSelect) * kSelect;
  cudaLaunchConfig_t config{};
  config.gridDim = dim3((uint32_t)(rows * blocks));
  config.blockDim = dim3(kSelect);
  config.dynamicSmemBytes = ((kCopies + (blocks > 1 ? 3 : 0)) * kBins + (per_block < kHeld ? per_block : kHeld)) * 4;
  config.stream = s;
  cudaLaunchAttribute attribute{};
  attribute.id = cudaLaunchAttributeClusterDimension;
  attribute.val.clusterDim.x = blocks;
  attribute.val.clusterDim.y = attribute.val.clusterDim.z = 1;
  config.attrs = &attribute;
  config.numAttrs = 1;
  if (cudaError_t e = cudaLaunchKernelEx(&config, select_kernel, a)) return e;
  count_launches(1);
  if (a.into) {
    move_kernel<<<dim3((a.keep + 8 * kMoveRows - 1) / (8 * kMoveRows), a.pool.groups, a.seq.batch), 256, 0, s>>>(a);
  } else {
    const uint32_t heads = a.pool.groups == 1 ? a.pool.kv_heads : 1, columns = (a.pool.dim + 15) / 16;
    slide_kernel<<<dim3((2 * heads + 1) * columns, a.pool.groups, a.seq.batch), kSlide, 0, s>>>(a, columns);
  }
  count_launches(1);
  return cudaGetLastError();
}

}  // namespace grand
