// Attention of many query rows over a paged cache, on the tensor cores (include/grand.h: grand_cache_attend).
//
// For the rows of one kv head, 256 at a time as two tiles of 128: S = Q K^T with 128 keys, P = 2^(S scale log2(e) - m),
// O += P V.  For a tile of 128 x 128 at dim 128 the products take 1,024 cycles of the tensor cores and the exponentials
// 1,024 of their unit (16 a cycle); at dim 64 the products take half of that, and the exponentials bound it.
//
// One block per SM, five warpgroups.  One warp of the last brings keys and values in through a ring of tile loads that
// follow the page table; one lane of another issues the products.  Each row tile has the softmax of two warpgroups, one for
// either half of the keys: while they compute, the products of the other row tile run.  (With one warpgroup a row tile,
// 4,096 tokens of a prompt of 32,768 take 2.04 ms instead of 2.00, three ragged chunks of 700 65 us instead of 56; a lane a
// row tile to issue the products: 2.5 ms; a quarter of the exponentials as polynomials on the multiply-add units: no gain
// at dim 128, 2 % lost at 64.)  A thread has 64 scores of one row; the two of a row exchange their maxima through shared
// memory.  S and O stay in tensor memory: S0, S1, O0, O1 of 128 columns each; P takes the place of its S in the cache's type
// (the one rounding that O does not share with its own) and is the left operand of its product from there.  The running
// maximum that the exponents refer to is moved only when a row's has grown by 8 (a factor of 256), so O is read back and
// rescaled a few times per item instead of at every tile.
//
// The work is split into equal runs of key tiles as in the streaming kernel.
#include <type_traits>

#include "grand_attend_items.cuh"
#include "grand_tc.cuh"

namespace grand {
namespace {

constexpr int kRows = 256, kTile = 128, kTcWarps = 20, kThreads = kTcWarps * 32;

template <int DP>
struct Tc {
  static constexpr int kCols = DP / 64;                 // 64-entry column blocks
  static constexpr int kQ = kCols * 16384;              // bytes of 128 rows, of queries or of keys
  static constexpr int kRing = DP == 128 ? 5 : 8;       // tiles of keys or values in flight
  static constexpr int kShared = 2 * kQ + kRing * kQ;   // place of what the two sides of a row tile exchange
  static constexpr int kBytes = kShared + 2048;         // (with the kernel's static kilobyte all that a block can have)
};

// barriers
template <int RING>
struct Bars {
  uint32_t base;
  __device__ uint32_t full(int i) const { return base + 8 * i; }
  __device__ uint32_t empty(int i) const { return base + 8 * (RING + i); }
  __device__ uint32_t q(int t) const { return base + 8 * (2 * RING + t); }
  __device__ uint32_t s(int t) const { return base + 8 * (2 * RING + 2 + t); }
  __device__ uint32_t p(int t) const { return base + 8 * (2 * RING + 4 + t); }
  __device__ uint32_t o(int t) const { return base + 8 * (2 * RING + 6 + t); }
  __device__ uint32_t drain() const { return base + 8 * (2 * RING + 8); }
};

template <bool BF16, int DP>
__global__ void __launch_bounds__(kThreads, 1) attend_tc_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ PoolMaps maps) {
  using T = Tc<DP>;
  constexpr int RING = T::kRing, KS = DP / 16;
  extern __shared__ __align__(1024) uint8_t raw[];
  __shared__ __align__(8) uint64_t bar_mem[2 * RING + 9];
  __shared__ uint32_t tmem_at;
  __shared__ int gave_up;
  __shared__ uint32_t last_part[2];
  __shared__ volatile int gaps;   // the table named a page outside the pool for a token of this block's tiles
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t smem = (uint32_t)__cvta_generic_to_shared(raw);
  float* shared_row = reinterpret_cast<float*>(raw + T::kShared);   // [row tile][half of the keys][row]: maxima, at the end sums
  const uint32_t q_at = smem, ring_at = smem + 2 * T::kQ;
  Bars<RING> bars{(uint32_t)__cvta_generic_to_shared(bar_mem)};

  Run run;
  plan_run<kRows, kTile, kTcWarps>(a, 4, 8, run);
  if (!run.any) return;

  if (tid == 0) {
    gave_up = 0;
    gaps = 0;
    for (int i = 0; i < RING; ++i) bar_init(bars.full(i), 1), bar_init(bars.empty(i), 1);
    for (int t = 0; t < 2; ++t) bar_init(bars.q(t), 8), bar_init(bars.s(t), 1), bar_init(bars.p(t), 8), bar_init(bars.o(t), 1);
    bar_init(bars.drain(), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  if (warp == 16) tmem_alloc((uint32_t)__cvta_generic_to_shared(&tmem_at), 512);
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_at;
  Item it = run.it;
  int t0 = run.tile;
  long long at = run.first;
  const long long end = run.end;

  // 640 threads start with 96 registers each; a softmax thread holds 64 scores: 512 x 104 + 128 x 64 = 640 x 96
  if (warp >= 16) {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
  if (warp == 17) {
    // ---- keys and values in
    int stage = 0;
    uint32_t phase = 1;  // the ring starts empty
    Boxes now, next;
    const int32_t* table = a.seq.table + (int64_t)it.b * a.seq.table_stride;
    // (the flag is passed on by the barrier of the tile's load)
    auto look_up = [&](Boxes& boxes, int j0) {
      if (find_boxes(boxes, a.pool, table, maps, j0, it.hi, lane, a.status)) gaps = 1;
    };
    look_up(now, it.lo + t0 * kTile);
    bool ok = true;
    uint32_t issued = 0, parity = 0;  // stages that loads went to, and the parity of their last phase
    while (ok) {
      const int t1 = run.last(it, t0, at);
      for (int t = t0; t < t1 && ok; ++t) {
        if (t + 1 < t1) look_up(next, it.lo + (t + 1) * kTile);
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          if (!(ok = bar_wait(bars.empty(stage), phase, &gave_up))) break;
          if (lane == 0) bar_expect(bars.full(stage), T::kQ);
          issued |= 1u << stage;
          parity = (parity & ~(1u << stage)) | (phase ^ 1) << stage;
          __syncwarp();
          load_boxes<T::kCols>(now, kv ? &maps.v : &maps.k, maps, it.h, ring_at + stage * T::kQ, bars.full(stage), lane);
          if (++stage == RING) stage = 0, phase ^= 1;
        }
        now = next;
      }
      at += t1 - t0;
      if (at >= end) break;
      next_item<kRows, kTile>(a, it);
      t0 = 0;
      table = a.seq.table + (int64_t)it.b * a.seq.table_stride;
      look_up(now, it.lo);
    }
    if (!ok)  // after a wait that ran out: leave nothing in flight towards this block's memory
      for (int i = 0; i < RING; ++i) {
        const long long c = clock64();
        while ((issued >> i & 1) && !bar_try(bars.full(i), parity >> i & 1) && clock64() - c < 100000000ll) {
        }
      }
  } else if (warp == 16) {
    // ---- products
    constexpr uint32_t shape_s = mma_shape(BF16, 128, 128, false), shape_o = mma_shape(BF16, 128, DP, true);
    int stage = 0;
    uint32_t phase = 0;                         // of the ring's full barriers
    uint32_t n_item[2] = {0, 0}, n_tile[2] = {0, 0};  // items and tiles done by each row tile
    bool ok = true;
    const uint64_t q_op = smem_operand(q_at), ring_op = smem_operand(ring_at), v_op = smem_operand(ring_at, 16384);
    auto product_s = [&](int t, int k_stage) {
      const uint64_t qa = q_op + t * (T::kQ >> 4), kb = ring_op + k_stage * (T::kQ >> 4);
      const uint32_t d = tmem + t * 128;
      if (elect_one()) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          constexpr int kBlock = 16384 >> 4, kStep = 32 >> 4;
          mma_ss(d, qa + (ks >> 2) * kBlock + (ks & 3) * kStep, kb + (ks >> 2) * kBlock + (ks & 3) * kStep, shape_s, ks != 0);
        }
        tc_commit(bars.s(t));
      }
      __syncwarp();
    };
    auto product_o = [&](int t, int v_stage, bool add) {
      const uint64_t vb = v_op + v_stage * (T::kQ >> 4);
      const uint32_t d = tmem + 256 + t * 128, p = tmem + t * 128;
      if (elect_one()) {
        mma_ts(d, p, vb, shape_o, add);
#pragma unroll
        for (int ks = 1; ks < 8; ++ks) mma_ts(d, p + (ks >> 2) * 64 + (ks & 3) * 8, vb + ks * (2048 >> 4), shape_o, 1);  // P's halves begin 64 columns apart
        tc_commit(bars.o(t));
      }
      __syncwarp();
    };
    auto release = [&](int st) {
      if (elect_one()) tc_commit(bars.empty(st));
      __syncwarp();
    };
    // A token without a page takes no part.  Its key, loaded as zeros, becomes NaN, and so do its scores: the softmax of a tile
    // without such tokens has nothing to ask, and one that meets a NaN looks for them.
    auto mark_gaps = [&](int k_stage, int j) {
      if (!__any_sync(0xFFFFFFFFu, gaps)) return;   // (the warp decides as one: the flag may be raised for a later tile between two lanes' reads)
      const int32_t* table = a.seq.table + (int64_t)it.b * a.seq.table_stride;
      for (int r = lane; r < kTile; r += 32) {
        const int key = it.lo + j * kTile + r;
        if (key < it.hi && page_of(table, div_fast((uint32_t)key, a.pool.page), a.pool.num_pages, nullptr) < 0)
          for (int x = 0; x < 8 * T::kCols; ++x)
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(ring_at + k_stage * T::kQ + (x >> 3) * 16384 + r * 128 + (x & 7) * 16), "r"(-1) : "memory");
      }
      fence_async_smem();
      __syncwarp();
    };
    while (ok) {
      const int t1 = run.last(it, t0, at);
      const int tiles2 = it.m * (int)a.group.d - it.rt * kRows > 128 ? 2 : 1;   // row tiles with rows
      // S of the first keys
      if (!(ok = bar_wait(bars.full(stage), phase, &gave_up))) break;
      mark_gaps(stage, t0);
      for (int t = 0; t < tiles2; ++t) {
        if (!(ok = bar_wait(bars.q(t), n_item[t] & 1, &gave_up))) break;
        tc_fence_after();
        product_s(t, stage);
      }
      if (!ok) break;
      release(stage);
      if (++stage == RING) stage = 0, phase ^= 1;
      for (int j = t0; j < t1; ++j) {
        const int v_stage = stage;
        const uint32_t v_at = ring_at + v_stage * T::kQ;
        if (!(ok = bar_wait(bars.full(v_stage), phase, &gave_up))) break;
        if (++stage == RING) stage = 0, phase ^= 1;
        const int j0 = it.lo + j * kTile;
        if (j0 < it.len && it.len < j0 + kTile && it.len % (int)maps.rows) {
          // The box in which the sequence ends brought slots that hold no token; whatever they hold, it must not meet
          // the zeros of P (0 x NaN).
          const int r1 = (it.len - j0 + (int)maps.rows - 1) / (int)maps.rows * (int)maps.rows;
#pragma unroll
          for (int c = 0; c < T::kCols; ++c)
            for (int x = (it.len - j0) * 8 + lane; x < r1 * 8; x += 32)
              asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(v_at + c * 16384 + x * 16), "r"(0) : "memory");
          fence_async_smem();
          __syncwarp();
        }
        const bool more = j + 1 < t1;
        const int k_stage = stage;
        if (more) {
          if (!(ok = bar_wait(bars.full(k_stage), phase, &gave_up))) break;
          if (++stage == RING) stage = 0, phase ^= 1;
          mark_gaps(k_stage, j + 1);
        }
        for (int t = 0; t < tiles2; ++t) {
          if (!(ok = bar_wait(bars.p(t), n_tile[t] & 1, &gave_up))) break;
          ++n_tile[t];
          tc_fence_after();
          product_o(t, v_stage, j != t0);
          if (t + 1 == tiles2) release(v_stage);
          // (products are executed in the order they are issued in, so S may take the place of the P just read)
          if (more) product_s(t, k_stage);
        }
        if (!ok) break;
        if (more) release(k_stage);
      }
      for (int t = 0; t < tiles2; ++t) ++n_item[t];
      at += t1 - t0;
      if (at >= end || !ok) break;
      next_item<kRows, kTile>(a, it);
      t0 = 0;
    }
    if (!ok) {  // (likewise)
      if (lane == 0) tc_commit(bars.drain());
      const long long c = clock64();
      while (!bar_try(bars.drain(), 0) && clock64() - c < 100000000ll) {
      }
    }
  }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
    // ---- softmax of row tile t and half `side` of its keys, one row per thread
    const int t = warp >> 3, side = (warp >> 2) & 1, r_in = (warp & 3) * 32 + lane;
    const uint32_t lane_at = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t s_at = tmem + t * 128 + side * 64 + lane_at;           // S, and P in its first 32 columns
    constexpr int kSide = DP / 2;                                          // entries of the output that this side handles
    const uint32_t o_at = tmem + 256 + t * 128 + side * kSide + lane_at;
    const int dim = (int)a.pool.dim, kvh = (int)a.pool.kv_heads;
    const float scale = a.scale_log2;
    uint32_t n_tile = 0;
    while (true) {
      const int t1 = run.last(it, t0, at);
      const int rows = it.m * (int)a.group.d - it.rt * kRows - t * 128;   // of this row tile
      if (rows > 0) {
        const bool live = r_in < rows;
        const int r = it.rt * kRows + t * 128 + (live ? r_in : 0), tok = (int)div_fast(r, a.group), hq = it.h * (int)a.group.d + r - tok * (int)a.group.d;
        {  // half of this row of Q
          const uint16_t* q = static_cast<const uint16_t*>(a.q) + (int64_t)(it.row + tok) * a.q_tok + (int64_t)hq * a.q_head;
          const uint32_t to = q_at + t * T::kQ + r_in * 128;
#pragma unroll
          for (int k = 0; k < DP / 16; ++k) {
            const int c = side * (DP / 16) + k;
            uint4 x = make_uint4(0, 0, 0, 0);
            if (live && c * 8 < dim) x = __ldg(reinterpret_cast<const uint4*>(q + c * 8));
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + (c >> 3) * 16384 + (((c & 7) ^ (r_in & 7)) << 4)), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w) : "memory");
          }
          fence_async_smem();
          __syncwarp();
          if (lane == 0) bar_arrive(bars.q(t));
        }
        // the row sees keys low .. lim, counted from this side's first one of tile 0
        const int lim = (live ? (a.causal ? min(it.len - 1, it.len - it.m + tok) : it.len - 1) : 0x3FFFFFFF) - side * 64 - it.lo;
        const int low = live && a.window ? it.len - it.m + tok - (int)a.window + 1 - side * 64 - it.lo : -0x3FFFFFFF;
        float m = kNegInf;          // reference of the exponents, in units of log 2
        float2 l2 = make_float2(0.0f, 0.0f);
        for (int j = t0; j < t1; ++j, ++n_tile) {
          const int last = lim - j * kTile, first = low - j * kTile;   // the row sees scores first .. last of its 64
          bar_wait(bars.s(t), n_tile & 1, &gave_up);
          tc_fence_after();
          uint32_t s[2][32];
          tmem_load32(s[0], s_at);
          tmem_load32(s[1], s_at + 32);
          tmem_load_wait();
          float top[2] = {kNegInf, kNegInf};
#pragma unroll
          for (int i = 0; i < 32; i += 2)
#pragma unroll
            for (int c = 0; c < 2; ++c) top[c] = max3_nan(top[c], __uint_as_float(s[c][i]), __uint_as_float(s[c][i + 1]));
          float best = max3_nan(top[0], top[1], kNegInf) * scale;
          // Most tiles: every row of the warp sees every key, and all scores are finite.
          const bool plain = scale > 0.0f && last >= 63 && first <= 0 && fabsf(best) < __int_as_float(0x7F800000);
          const bool fast = __all_sync(0xFFFFFFFFu, plain);
          if (!fast) {
            const bool look = __any_sync(0xFFFFFFFFu, best != best);   // for tokens without a page, one of 32 a lane
            best = kNegInf;   // (a negative scale turns the order around; a NaN does not raise the maximum)
            auto mask = [&](int c, uint32_t gone) {
#pragma unroll
              for (int i = 0; i < 32; ++i) {
                // -inf in a masked place, whatever the key holds
                const float x = c * 32 + i > last || c * 32 + i < first || (gone >> i & 1) ? kNegInf : __uint_as_float(s[c][i]) * scale;
                s[c][i] = __float_as_uint(x);
                best = fmaxf(best, x);
              }
            };
            if (look) {
              const int32_t* table = a.seq.table + (int64_t)it.b * a.seq.table_stride;
              const int key = it.lo + j * kTile + side * 64 + lane;
#pragma unroll
              for (int c = 0; c < 2; ++c)
                mask(c, __ballot_sync(0xFFFFFFFFu, key + c * 32 < it.hi && page_of(table, div_fast((uint32_t)(key + c * 32), a.pool.page), a.pool.num_pages, nullptr) < 0));
            } else {
              mask(0, 0);
              mask(1, 0);
            }
          }
          {  // the row's maximum over both sides
            float* mine = shared_row + t * 256 + r_in;   // (read by all before the next S, which waits for their P)
            mine[side * 128] = best;
            pair_sync(t);
            best = fmaxf(best, mine[(side ^ 1) * 128]);
          }
          if (__any_sync(0xFFFFFFFFu, best > m + 8.0f)) {
            const float mn = best > m + 8.0f ? best : m;   // (rows stay independent of each other)
            const float f = mn == m ? 1.0f : exp2_fast(m - mn);
            m = mn;
            l2.x *= f;
            l2.y *= f;
            if (j != t0) {   // O holds the tiles before this one
              bar_wait(bars.o(t), (n_tile - 1) & 1, &gave_up);
              tc_fence_after();
#pragma unroll 1
              for (int c = 0; c < kSide / 16; ++c) {
                uint32_t o[16];
                tmem_load16(o, o_at + c * 16);
                tmem_load_wait();
#pragma unroll
                for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                tmem_store16(o_at + c * 16, o);
              }
            }
          }
          const float ref = m == kNegInf ? 0.0f : m - kLift<BF16>;
          const float2 sub = make_float2(-ref, -ref), mul = make_float2(scale, scale);
          auto exponentials = [&](auto is_fast) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              uint32_t p[16];
#pragma unroll
              for (int i = 0; i < 32; i += 2) {
                const float2 y = make_float2(__uint_as_float(s[c][i]), __uint_as_float(s[c][i + 1]));
                float2 x = decltype(is_fast)::value ? fma2(y, mul, sub) : add2(y, sub);
                x.x = exp2_fast(x.x);
                x.y = exp2_fast(x.y);
                l2 = add2(l2, x);
                p[i / 2] = pack2<BF16>(x.x, x.y);
              }
              tmem_store16(s_at + c * 16, p);
            }
          };
          if (fast) exponentials(std::true_type{});
          else exponentials(std::false_type{});
          tmem_store_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) bar_arrive(bars.p(t));
        }
        // ---- the item's rows, or their part
        float l = l2.x + l2.y;
        {  // the row's sum over both sides
          float* mine = shared_row + t * 256 + r_in;
          pair_sync(t);   // the last maxima are read
          mine[side * 128] = l;
          pair_sync(t);
          l = mine[0] + mine[128];
        }
        bar_wait(bars.o(t), (n_tile - 1) & 1, &gave_up);
        tc_fence_after();
        const int64_t out_row = (int64_t)(it.row + tok) * kvh * a.group.d + hq;
        auto emit = [&](int c0, const float (&v)[16], float f) {   // entries c0 .. c0 + 15 of this side
          uint16_t* out = static_cast<uint16_t*>(a.out) + out_row * dim;
          c0 += side * kSide;
#pragma unroll
          for (int i = 0; i < 16; i += 8)
            if (live && c0 + i < dim)
              *reinterpret_cast<uint4*>(out + c0 + i) = make_uint4(pack2<BF16>(v[i] * f, v[i + 1] * f), pack2<BF16>(v[i + 2] * f, v[i + 3] * f),
                                                                   pack2<BF16>(v[i + 4] * f, v[i + 5] * f), pack2<BF16>(v[i + 6] * f, v[i + 7] * f));
        };
        auto inverse = [](float sum) { return sum > 0.0f ? 1.0f / sum : (sum == 0.0f ? 0.0f : sum); };  // (a NaN stays one)
        const bool whole = t0 == 0 && t1 == it.tiles;
        if (whole) {
          const float f = inverse(l);
#pragma unroll 1
          for (int c = 0; c < kSide / 16; ++c) {
            uint32_t o[16];
            float v[16];
            tmem_load16(o, o_at + c * 16);
            tmem_load_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(o[i]);
            emit(c * 16, v, f);
          }
          if (live && a.lse && side == 0) a.lse[out_row] = (m - kLift<BF16> + log2f(l)) * kLn2;
        } else {
          // a part: entry-major, so that a warp's rows lie side by side
          constexpr uint64_t kPart = (uint64_t)(DP + 2) * 128;   // of one row tile
          float* slot = a.partial + ((uint64_t)blockIdx.x * 2 + (t0 == 0 ? 1 : 0)) * a.slot_floats + t * kPart + r_in;
#pragma unroll 1
          for (int c = 0; c < kSide / 16; ++c) {
            uint32_t o[16];
            tmem_load16(o, o_at + c * 16);
            tmem_load_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) __stcg(slot + (side * kSide + c * 16 + i) * 128, __uint_as_float(o[i]));
          }
          if (side == 0) {
            __stcg(slot + DP * 128, m);
            __stcg(slot + (DP + 1) * 128, l);
          }
          const long long item0 = at - t0, c0 = item0 / run.share, c1 = (item0 + it.tiles - 1) / run.share;
          __threadfence();
          pair_sync(t);
          if (r_in == 0 && side == 0) {
            const uint32_t n = atomicAdd(a.arrived + 2 * c0 + t, 1u);
            last_part[t] = n == (uint32_t)(c1 - c0);
            if (last_part[t]) a.arrived[2 * c0 + t] = 0;  // for the next call
          }
          pair_sync(t);
          if (last_part[t]) {
            __threadfence();
            // the item begins in the second slot of its first block and goes on in the first slots of the others
            const int parts = (int)(c1 - c0) + 1;
            const float* part0 = a.partial + ((uint64_t)c0 * 2 + 1) * a.slot_floats + t * kPart + r_in;
            const float* part1 = a.partial + (uint64_t)c0 * 2 * a.slot_floats + t * kPart + r_in;
            const uint64_t step = 2 * a.slot_floats;
#pragma unroll 1
            for (int k = 0; k < kSide / 32; ++k) {
              float top = kNegInf, sum = 0.0f, v[2][16];
#pragma unroll
              for (int i = 0; i < 32; ++i) v[i >> 4][i & 15] = 0.0f;
#pragma unroll 1
              for (int c = 0; c < parts; ++c) {   // one part's reads are in flight together
                const float* p = c == 0 ? part0 : part1 + c * step;
                const float pm = __ldcg(p + DP * 128), pl = __ldcg(p + (DP + 1) * 128);
                float x[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) x[i] = __ldcg(p + (side * kSide + k * 32 + i) * 128);
                const float up = fmaxf(top, pm), ref = up == kNegInf ? 0.0f : up, f = exp2_fast(top - ref), g = exp2_fast(pm - ref);
                top = up;
                sum = sum * f + pl * g;
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i >> 4][i & 15] = v[i >> 4][i & 15] * f + x[i] * g;
              }
              const float f = inverse(sum);
              emit(k * 32, v[0], f);
              emit(k * 32 + 16, v[1], f);
              if (live && a.lse && side == 0 && k == 0) a.lse[out_row] = (top - kLift<BF16> + log2f(sum)) * kLn2;
            }
          }
        }
        pair_sync(t);   // what the two sides share is read before it is written again
        // (the p barrier of the next item orders these reads of O before the product that overwrites it)
        tc_fence_before();
      }
      at += t1 - t0;
      if (at >= end) break;
      next_item<kRows, kTile>(a, it);
      t0 = 0;
    }
  }
  tc_fence_before();
  __syncthreads();
  if (tid == 0 && gave_up) atomicOr(a.status, (uint32_t)kGaveUp);
  if (warp == 16) tmem_free(tmem, 512);
}

template <bool BF16, int DP>
cudaError_t tc_at(const AttendArgs& a, const PoolMaps& maps, cudaStream_t s) {
  static SmemOptIn done;
  auto* kernel = attend_tc_kernel<BF16, DP>;
  if (cudaError_t e = allow_dynamic_smem(reinterpret_cast<const void*>(kernel), Tc<DP>::kBytes, &done)) return e;
  kernel<<<sm_count(), kThreads, Tc<DP>::kBytes, s>>>(a, maps);
  count_launches(1);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attend_tc(const AttendArgs& args, uint32_t dtype, cudaStream_t s) {
  AttendArgs a = args;
  a.slot_floats = kTcSlot;
  PoolMaps maps;
  if (!make_pool_maps(a.pool, dtype, &maps)) return launch_attend_stream(a, dtype, s);
  if (a.pool.dim <= 64) return dtype == 4 ? tc_at<true, 64>(a, maps, s) : tc_at<false, 64>(a, maps, s);
  return dtype == 4 ? tc_at<true, 128>(a, maps, s) : tc_at<false, 128>(a, maps, s);
}

}  // namespace grand
