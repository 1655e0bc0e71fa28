// What the tensor-core kernels of the token cache share: barriers in shared memory with bounded waits, tile loads of the
// paged pool, tile products (tcgen05) with operands in shared or tensor memory, and reads and writes of tensor memory.
#pragma once
#include <cuda.h>

#include "grand_cache_mma.cuh"

namespace grand {

// Tile loads see the pool as [entry, x, y, page] with x and y the slot and the head, the one with the smaller stride first.
// A load brings `rows` slots of one page and head, 64 entries (128 bytes) of each, into rows of 128 bytes whose 16-byte
// chunk c sits at place c ^ (row & 7).  `rows` is the largest power of two that divides the page size, at most 128.
// Where that is less than 4 and the pool is a plain list of rows (every stride a multiple of dim), the map is that list,
// and a load gathers four rows of it by their numbers: 2,048 queries over 16,384 tokens in pages of one take 980 us row by
// row and 327 so (141 in pages of 64).
struct PoolMaps {
  CUtensorMap k, v;
  uint32_t rows;         // 1 where rows are gathered
  uint32_t heads_first;  // x is the head
  uint32_t gather;       // 0, or the number of rows in the list, of which a page, a slot and a head are these steps:
  uint32_t page_step, slot_step, head_step;
};
// false: the pool's strides do not fit a map
bool make_pool_maps(const PoolView& pool, uint32_t dtype, PoolMaps* maps);
// Loads of `box_heads` heads of `box_tokens` tokens of a packed array [tokens, heads, dim], 64 entries of each.
bool make_rows_map(const void* x, int64_t token_stride, int64_t head_stride, uint32_t tokens, uint32_t heads, uint32_t dim, uint32_t dtype,
                   uint32_t box_heads, uint32_t box_tokens, CUtensorMap* map);

#ifdef __CUDACC__

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
      : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
// Waits for the completion of the barrier's phase of the given parity; after some seconds (a try suspends the thread for a
// while by itself) it raises `gave_up` for the whole block and returns false, as does every later wait.  The warps that
// issue copies and products then stop and wait for those in flight; the others go on without waiting, so that every
// barrier between them is still reached by all, and the block ends with void results and the status bit set.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int* gave_up) {
  if (bar_try(bar, parity)) return true;
#pragma unroll 1
  for (int i = 0; i < (1 << 20); ++i) {
    if (bar_try(bar, parity)) return true;
    if ((i & 15) == 15 && *gave_up) return false;
  }
  *gave_up = 1;
  return false;
}

__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* map, uint32_t bar, int e, int x, int y, int page) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
      ::"r"(dst), "l"(map), "r"(bar), "r"(e), "r"(x), "r"(y), "r"(page) : "memory");
}
__device__ __forceinline__ void load_gather(uint32_t dst, const CUtensorMap* map, uint32_t bar, int e, int r0, int r1, int r2, int r3) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];"
      ::"r"(dst), "l"(map), "r"(bar), "r"(e), "r"(r0), "r"(r1), "r"(r2), "r"(r3) : "memory");
}
__device__ __forceinline__ void load_rows(uint32_t dst, const CUtensorMap* map, uint32_t bar, int e, int head, int token) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
      ::"r"(dst), "l"(map), "r"(bar), "r"(e), "r"(head), "r"(token) : "memory");
}
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

__device__ __forceinline__ void tmem_alloc(uint32_t smem_addr, uint32_t columns) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr), "r"(columns) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(uint32_t tmem, uint32_t columns) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns));
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// Tile in shared memory in rows of 128 bytes as above, eight rows to a 1024-byte group.  As an operand whose products run
// along the row (K-major) the groups follow each other at 1024 bytes; as one whose products run across the rows
// (MN-major) `leading` is the distance of the next 64 entries of the row.  Layout 2 is the 128-byte swizzle.
__device__ __forceinline__ uint64_t smem_operand(uint32_t addr, uint32_t leading = 16) {
  return (uint64_t)((addr & 0x3FFFF) >> 4) | (uint64_t)(leading >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// 16-bit operands of one type, fp32 sums, M x N, B along its rows or across them
__host__ __device__ constexpr uint32_t mma_shape(bool bf16, int m, int n, bool b_across) {
  return 1u << 4 | (bf16 ? 1u : 0u) << 7 | (bf16 ? 1u : 0u) << 10 | (b_across ? 1u : 0u) << 16 | (uint32_t)(n >> 3) << 17 | (uint32_t)(m >> 4) << 24;
}
// (an operand's address lies in its low 14 bits, in units of 16 bytes, so a step through shared memory is an addition
// to its low word)
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t shape, uint32_t add) {
  asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
               ::"r"(d), "l"(a), "l"(b), "r"(shape), "r"(add) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t shape, uint32_t add) {
  asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
               ::"r"(d), "r"(a), "l"(b), "r"(shape), "r"(add) : "memory");
}
// One lane of a converged warp; the compiler knows that the code behind it runs once.
__device__ __forceinline__ bool elect_one() {
  uint32_t ok;
  asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xFFFFFFFF;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(ok));
  return ok != 0;
}

// 32 columns of this warp's 32 lanes: register i of a lane is its column i.
__device__ __forceinline__ void tmem_load32(uint32_t (&r)[32], uint32_t addr) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
        "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr));
}
__device__ __forceinline__ void tmem_load16(uint32_t (&r)[16], uint32_t addr) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                 "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(addr));
}
__device__ __forceinline__ void tmem_store16(uint32_t addr, const uint32_t (&r)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
               ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
                 "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void tmem_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Two 32-bit operations in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n.reg .b64 x, y, z;\nmov.b64 x, {%2, %3};\nmov.b64 y, {%4, %5};\nmov.b64 z, {%6, %7};\nfma.rn.f32x2 x, x, y, z;\nmov.b64 {%0, %1}, x;\n}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n.reg .b64 x, y;\nmov.b64 x, {%2, %3};\nmov.b64 y, {%4, %5};\nadd.rn.f32x2 x, x, y;\nmov.b64 {%0, %1}, x;\n}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}

__device__ __forceinline__ void group_sync(int t) {  // the 128 threads of warpgroup t, 0 or 1
  if (t == 0) asm volatile("bar.sync 1, 128;" ::: "memory");
  else asm volatile("bar.sync 2, 128;" ::: "memory");
}

__device__ __forceinline__ float max3_nan(float a, float b, float c) {  // a NaN if one of them is
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

__device__ __forceinline__ void pair_sync(int t) {  // the 256 threads of warpgroups 2 t and 2 t + 1
  if (t == 0) asm volatile("bar.sync 1, 256;" ::: "memory");
  else asm volatile("bar.sync 2, 256;" ::: "memory");
}

// Where the boxes of a tile of 128 keys lie: lane l looks up those that start at key j0 + (l + 32 i) * rows.  A box from
// `hi` on, or of a page outside the pool, gets the page behind the last, which loads as zeros.  Where rows are gathered, lane
// l looks up keys j0 + 4 l + i: `page` is the row's number in the list for head 0, or the one behind the last.  Returns (to
// every lane of its own) whether a page that it looked up is outside the pool.
struct Boxes {
  int page[4], slot[4];
};
__device__ __forceinline__ bool find_boxes(Boxes& b, const PoolView& pool, const int32_t* table, const PoolMaps& maps, int j0, int hi, int lane, uint32_t* status) {
  bool gap = false;
  auto look_up = [&](int j, int& slot) {
    const uint32_t jp = div_fast((uint32_t)j, pool.page);
    slot = j - (int)(jp * pool.page.d);
    const int p = page_of(table, jp, pool.num_pages, status);
    gap |= p < 0;
    return p;
  };
  if (maps.gather) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int j = j0 + 4 * lane + i;
      b.page[i] = -1;
      if (j < hi) {
        int slot;
        const int p = look_up(j, slot);
        if (p >= 0) b.page[i] = (int)(p * maps.page_step + slot * maps.slot_step);
      }
    }
    return gap;
  }
  const int n = 128 / (int)maps.rows;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int j = j0 + (lane + 32 * i) * (int)maps.rows;
    b.page[i] = (int)pool.num_pages;
    b.slot[i] = 0;
    if (lane + 32 * i < n && j < hi) {
      const int p = look_up(j, b.slot[i]);
      if (p >= 0) b.page[i] = p;
    }
  }
  return gap;
}
// One tile of 128 keys, COLS blocks of 64 entries, into `dst` (COLS x 16 KB).
template <int COLS>
__device__ __forceinline__ void load_boxes(const Boxes& b, const CUtensorMap* map, const PoolMaps& maps, int head, uint32_t dst, uint32_t bar, int lane) {
  if (maps.gather) {
    int r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = b.page[i] < 0 ? (int)maps.gather : b.page[i] + head * (int)maps.head_step;
#pragma unroll
    for (int c = 0; c < COLS; ++c) load_gather(dst + c * 16384 + lane * 512, map, bar, c * 64, r[0], r[1], r[2], r[3]);
    return;
  }
  const int n = 128 / (int)maps.rows;
  const bool heads_first = maps.heads_first;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int box = lane + 32 * i;
    if (box < n) {
#pragma unroll
      for (int c = 0; c < COLS; ++c)
        load_tile(dst + c * 16384 + box * maps.rows * 128, map, bar, c * 64, heads_first ? head : b.slot[i], heads_first ? b.slot[i] : head, b.page[i]);
    }
  }
}
#endif

}  // namespace grand
