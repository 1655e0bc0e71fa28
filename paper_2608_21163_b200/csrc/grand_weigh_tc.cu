// The attention weight that every cached token collects from many query rows, on the tensor cores (include/grand.h:
// grand_cache_weigh): w_j = decay w_j + sum_r 2^(scale log2(e) q_r.k_j - lse_r log2(e)).
//
// S^T = K Q^T, 128 keys on the long side (a key's scores lie in one lane of tensor memory, so one thread sums them) and up
// to 128 query rows on the other.  A pair costs 2 dim flops and one exponential: for a tile of 128 x 128 at dim 128 the
// products take 512 cycles of the tensor cores and the exponentials 1,024 at 16 a cycle, so the exponentials bound it.  Measured
// (four chunks of 1,024 tokens on up to 8,000) their unit is busy for two thirds of the time: every thread also reads -lse of every
// row from shared memory, 16 bytes for four exponentials, through the same queue.
//
// One block per SM: a warp that brings keys (once per item and kv head) and query rows (a ring) in, one that brings what
// the exponents need of each row, two lanes that issue the products into four score tiles in tensor memory, and four
// warpgroups that take the score tiles in turn.  (On the same chunks: two warpgroups that fetch the rows' data themselves 302 us of
// device time, four 307, with a warp of its own for that data 283, with the producers' loops shortened and two issuing lanes
// 265, with 256 keys to a tile of rows instead of 128 220.)  An item is a tile of 256 keys, two halves of 128, of one sequence and
// weight row; its tiles are the row tiles that see it, of each of its kv heads.  All tiles are numbered through and every block takes an
// equal run of them; parts of an item are joined in their order by the block that arrives last, so equal calls give equal
// bits.
#include "grand_attend_items.cuh"
#include "grand_tc.cuh"

namespace grand {
namespace {

constexpr int kHalf = 128, kTile = 2 * kHalf, kWarps = 20, kThreads = kWarps * 32, kKeyBufs = 2, kScores = 2, kColumns = 2 * kScores;

template <int DP>
struct Wt {
  static constexpr int kCols = DP / 64, kBytesTile = kCols * 16384;   // of 128 rows
  static constexpr int kRing = DP == 128 ? 2 : 4;
  static constexpr int kBytes = (2 * kKeyBufs + kRing) * kBytesTile + 1024;
};

struct KeyItem {
  int b, g, kt;          // sequence, weight row, key tile
  int len, row, m;
  int rt0, rts;          // row tiles that see it; none: the item is left out, or, with a decay, has one that is masked
  int heads;             // kv heads of a weight row
  __device__ int tiles() const { return rts * heads; }
};

__device__ __forceinline__ void open_keys(const WeighArgs& a, KeyItem& it, int b, uint32_t* status = nullptr) {
  const Seq s = load_seq(a.seq, b, status);
  it.b = b; it.len = s.len; it.row = s.row; it.m = s.m;
  it.g = it.kt = 0;
  it.heads = a.pool.groups == 1 ? (int)a.pool.kv_heads : 1;
}
__device__ __forceinline__ int key_tiles(const KeyItem& it) { return (it.len + kTile - 1) / kTile; }

// `tpt`: tokens of a row tile
__device__ __forceinline__ void set_rows(const WeighArgs& a, KeyItem& it, int tpt) {
  const int j0 = it.kt * kTile, past = it.len - it.m;   // token i sees j <= past + i, j > past + i - window
  int i0 = 0, i1 = it.m - 1;
  if (a.causal) {
    i0 = max(0, j0 - past);
    if (a.window) i1 = min(i1, j0 + kTile - 1 + (int)a.window - 1 - past);
  }
  it.rt0 = 0;
  it.rts = a.decay != 1.0f;
  if (i1 >= i0) it.rt0 = i0 / tpt, it.rts = i1 / tpt - it.rt0 + 1;
}
// Key tiles [0, n) of a sequence whose number of row tiles is that of the first: those that every row sees, or (with a window)
// that no row sees.
__device__ __forceinline__ int alike(const WeighArgs& a, const KeyItem& it, int tpt) {
  const int n = key_tiles(it), past = it.len - it.m;
  if (!a.causal || it.m == 0) return n;
  const long long edge = a.window ? (long long)past - (long long)a.window - kTile : past;  // a tile that ends before it is such a one
  return edge <= 0 ? 0 : (int)min((long long)n, edge / kTile);
}

template <bool WARP>
__device__ __forceinline__ long long key_seq_tiles(const WeighArgs& a, int b, int tpt, int lane, uint32_t* status) {
  KeyItem it{};
  open_keys(a, it, b, status);
  const int n = key_tiles(it), z = alike(a, it, tpt);
  long long sum = 0;
  for (it.kt = z + (WARP ? lane : 0); it.kt < n; it.kt += WARP ? 32 : 1) {
    set_rows(a, it, tpt);
    sum += it.tiles();
  }
  if (WARP)
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
  it.kt = 0;
  set_rows(a, it, tpt);
  return n == 0 ? 0 : sum + (long long)z * it.tiles();
}

// The next item with tiles.  Only called while tiles are left.
__device__ __forceinline__ void next_keys(const WeighArgs& a, KeyItem& it, int tpt) {
  while (true) {
    if (++it.kt >= key_tiles(it)) {
      if (++it.g >= (int)a.pool.groups) {
        if (it.b + 1 >= (int)a.seq.batch) return;
        open_keys(a, it, it.b + 1);
      }
      // key tiles that no row sees come first in a sequence: past all that are like the first
      it.kt = 0;
      if (it.len == 0) {
        it.kt = it.g = 0x3FFFFFFF;
        continue;
      }
      set_rows(a, it, tpt);
      if (it.rts == 0) it.kt = min(alike(a, it, tpt), key_tiles(it) - 1);
    }
    set_rows(a, it, tpt);
    if (it.rts > 0) return;
  }
}

template <int RING>
struct Bars {
  uint32_t base;
  __device__ uint32_t k_full(int i) const { return base + 8 * i; }
  __device__ uint32_t k_empty(int i) const { return base + 8 * (kKeyBufs + i); }
  __device__ uint32_t q_full(int i) const { return base + 8 * (2 * kKeyBufs + i); }
  __device__ uint32_t q_empty(int i) const { return base + 8 * (2 * kKeyBufs + RING + i); }
  __device__ uint32_t s_full(int i) const { return base + 8 * (2 * kKeyBufs + 2 * RING + i); }
  __device__ uint32_t s_empty(int i) const { return base + 8 * (2 * kKeyBufs + 2 * RING + 2 * kScores + i); }
  __device__ uint32_t c_full(int i) const { return base + 8 * (2 * kKeyBufs + 2 * RING + 4 * kScores + i); }
  __device__ uint32_t c_empty(int i) const { return base + 8 * (2 * kKeyBufs + 2 * RING + 4 * kScores + kColumns + i); }
  __device__ uint32_t drain() const { return base + 8 * (2 * kKeyBufs + 2 * RING + 4 * kScores + 2 * kColumns); }
  static constexpr int kCount = 2 * kKeyBufs + 2 * RING + 4 * kScores + 2 * kColumns + 1;
};

template <bool BF16, int DP>
__global__ void __launch_bounds__(kThreads, 1)
weigh_tc_kernel(const __grid_constant__ WeighArgs a, const __grid_constant__ PoolMaps maps, const __grid_constant__ CUtensorMap q_map, int tpt) {
  using T = Wt<DP>;
  constexpr int RING = T::kRing, KS = DP / 16;
  extern __shared__ uint8_t raw[];
  __shared__ __align__(8) uint64_t bar_mem[Bars<RING>::kCount];
  __shared__ uint32_t tmem_at;
  __shared__ int gave_up;
  __shared__ uint32_t last_part[2];
  __shared__ int sh_g, sh_kt, sh_tile;
  __shared__ float others[2][2][kHalf];                     // [buffer][half]: sums of warpgroups 2 and 3
  __shared__ __align__(16) float col_lse[kColumns][kHalf];   // of a score tile's rows: -lse in units of log 2,
  __shared__ __align__(16) int col_lim[kColumns][kHalf];      // and the last key they see (the first is a window before)
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t smem = ((uint32_t)__cvta_generic_to_shared(raw) + 1023) & ~1023u;
  const uint32_t k_at = smem, q_at = smem + 2 * kKeyBufs * T::kBytesTile;
  Bars<RING> bars{(uint32_t)__cvta_generic_to_shared(bar_mem)};
  const int group = (int)a.group.d, rows_t = tpt * group;   // rows of a row tile, at most 128

  Share share;
  if (!find_share<kWarps>((int)a.seq.batch, true, a.status, [&](int b, bool together, int l, uint32_t* status) {
        return (together ? key_seq_tiles<true>(a, b, tpt, l, status) : key_seq_tiles<false>(a, b, tpt, l, status)) * a.pool.groups;
      }, [](long long) { return 4ll; }, [](int, long long, int*) {}, share))
    return;
  if (warp == 0) {  // weight row and key tile of the first tile
    const long long n = key_seq_tiles<true>(a, share.b, tpt, lane, nullptr);
    long long off = share.off;
    const int g = (int)(off / n);
    off -= g * n;
    KeyItem it{};
    open_keys(a, it, share.b);
    const int tiles = key_tiles(it), z = alike(a, it, tpt);
    set_rows(a, it, tpt);
    const long long each = it.tiles();
    if (off < z * each) {
      if (lane == 0) sh_g = g, sh_kt = (int)(off / each), sh_tile = (int)(off % each);
    } else {
      off -= z * each;
      for (int base = z; base < tiles; base += 32) {
        it.kt = base + lane;
        long long c = 0;
        if (it.kt < tiles) {
          set_rows(a, it, tpt);
          c = it.tiles();
        }
        const long long incl = warp_scan(c, lane);
        if (off >= incl - c && off < incl) sh_g = g, sh_kt = it.kt, sh_tile = (int)(off - (incl - c));
        const long long all = __shfl_sync(0xFFFFFFFFu, incl, 31);
        if (off < all) break;
        off -= all;
      }
    }
  }
  if (tid == 0) {
    gave_up = 0;
    for (int i = 0; i < kKeyBufs; ++i) bar_init(bars.k_full(i), 1), bar_init(bars.k_empty(i), 2);
    for (int i = 0; i < RING; ++i) bar_init(bars.q_full(i), 1), bar_init(bars.q_empty(i), 1);
    for (int i = 0; i < 2 * kScores; ++i) bar_init(bars.s_full(i), 1), bar_init(bars.s_empty(i), 4);
    for (int i = 0; i < kColumns; ++i) bar_init(bars.c_full(i), 1), bar_init(bars.c_empty(i), 8);
    bar_init(bars.drain(), 2);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  // rows of the ring that no load reaches (a row tile of fewer than 128 rows) stay zero
  if (rows_t < 128)
    for (int x = tid; x < RING * T::kCols * (128 - rows_t) * 8; x += kThreads) {
      const int tile = x / ((128 - rows_t) * 8), in = x - tile * ((128 - rows_t) * 8);
      asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(q_at + tile * 16384 + rows_t * 128 + in * 16), "r"(0) : "memory");
    }
  fence_async_smem();
  if (warp == 16) tmem_alloc((uint32_t)__cvta_generic_to_shared(&tmem_at), 512);
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_at;
  KeyItem it{};
  open_keys(a, it, share.b);
  it.g = sh_g;
  it.kt = sh_kt;
  set_rows(a, it, tpt);
  int x0 = sh_tile;
  long long at = share.first;
  const long long end = share.end;

  // 640 threads start with 96 registers each: 512 x 104 + 128 x 64 = 640 x 96
  if (warp >= 16) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    // The block's run of tiles, kv head by kv head of its items: segment(kv head, first row tile, row tiles) is false if
    // a wait ran out.
    auto run_segments = [&](auto begin, auto segment) {
      while (true) {
        const int x1 = (int)min((long long)it.tiles(), x0 + (end - at));
        begin();
        for (int x = x0; x < x1;) {
          const int hi = x / it.rts, r = x - hi * it.rts, n = min(it.rts - r, x1 - x);
          if (!segment(it.g + hi, it.rt0 + r, n)) return false;   // (weight row g is kv head g, or all heads belong to row 0)
          x += n;
        }
        at += x1 - x0;
        if (at >= end) return true;
        next_keys(a, it, tpt);
        x0 = 0;
      }
    };
    if (warp == 18) {
      // ---- keys and query rows in
      int qs = 0, kb = 0;
      uint32_t q_phase = 1, k_phase = 1;
      uint32_t q_issued = 0, q_parity = 0, k_issued = 0, k_parity = 0;
      Boxes boxes[2];
      const bool ok = run_segments(
          [&] {
#pragma unroll
            for (int half = 0; half < 2; ++half)
              find_boxes(boxes[half], a.pool, a.seq.table + (int64_t)it.b * a.seq.table_stride, maps, it.kt * kTile + half * kHalf, it.len, lane, a.status);
          },
          [&](int h, int rt, int n) {
            if (!bar_wait(bars.k_empty(kb), k_phase, &gave_up)) return false;
            if (lane == 0) bar_expect(bars.k_full(kb), 2 * T::kBytesTile);
            k_issued |= 1u << kb;
            k_parity = (k_parity & ~(1u << kb)) | (k_phase ^ 1) << kb;
            __syncwarp();
#pragma unroll
            for (int half = 0; half < 2; ++half)
              load_boxes<T::kCols>(boxes[half], &maps.k, maps, h, k_at + (2 * kb + half) * T::kBytesTile, bars.k_full(kb), lane);
            if (++kb == kKeyBufs) kb = 0, k_phase ^= 1;
            for (int token = it.row + rt * tpt; n > 0; --n, token += tpt) {
              if (!bar_wait(bars.q_empty(qs), q_phase, &gave_up)) return false;
              q_issued |= 1u << qs;
              q_parity = (q_parity & ~(1u << qs)) | (q_phase ^ 1) << qs;
              if (elect_one()) {
                bar_expect(bars.q_full(qs), T::kCols * rows_t * 128);
#pragma unroll
                for (int c = 0; c < T::kCols; ++c)
                  load_rows(q_at + qs * T::kBytesTile + c * 16384, &q_map, bars.q_full(qs), c * 64, h * group, token);
              }
              __syncwarp();
              if (++qs == RING) qs = 0, q_phase ^= 1;
            }
            return true;
          });
      if (!ok) {  // after a wait that ran out: leave nothing in flight towards this block's memory
        const long long c = clock64();
        for (int i = 0; i < kKeyBufs; ++i)
          while ((k_issued >> i & 1) && !bar_try(bars.k_full(i), k_parity >> i & 1) && clock64() - c < 100000000ll) {
          }
        for (int i = 0; i < RING; ++i)
          while ((q_issued >> i & 1) && !bar_try(bars.q_full(i), q_parity >> i & 1) && clock64() - c < 100000000ll) {
          }
      }
    } else if (warp == 19) {
      // ---- what the rows of each score tile need: four neighbouring rows a lane, fetched two tiles ahead
      uint32_t n_done = 0;
      int t_in[4];            // token of the tile, -1: no row
      int64_t off[4];         // of its lse
      const int64_t per_token = (int64_t)a.pool.kv_heads * group;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int c = lane * 4 + k;
        t_in[k] = (int)div_fast((uint32_t)c, a.group);
        off[k] = t_in[k] * per_token + c - t_in[k] * group;
        if (c >= rows_t) t_in[k] = -1;
      }
      run_segments([] {}, [&](int h, int rt, int n) {
        const float* lse = a.lse + (int64_t)(it.row + rt * tpt) * per_token + h * group;
        int tok = rt * tpt;
        float next[2][4];
        auto fetch = [&](float (&x)[4], int ahead) {
#pragma unroll
          for (int k = 0; k < 4; ++k)
            x[k] = ahead < n && t_in[k] >= 0 && tok + ahead * tpt + t_in[k] < it.m ? __ldg(lse + ahead * tpt * per_token + off[k]) : kNegInf;
        };
        fetch(next[0], 0);
        fetch(next[1], 1);
        for (; n > 0; --n, ++n_done, tok += tpt, lse += tpt * per_token) {
          const int sb = (int)(n_done % kColumns);
          float x[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) x[k] = next[0][k], next[0][k] = next[1][k];
          fetch(next[1], 2);
          if (!bar_wait(bars.c_empty(sb), (n_done / kColumns & 1) ^ 1, &gave_up)) return false;
          float4 l;
          int4 s;
          float* lp = reinterpret_cast<float*>(&l);
          int* sp = reinterpret_cast<int*>(&s);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const bool sees = x[k] != kNegInf;   // (a row that attended nothing, or that is none, gives nothing)
            lp[k] = sees ? x[k] * -1.44269504088896340736f : kNegInf;
            sp[k] = !sees ? -0x3FFFFFFF : a.causal ? it.len - it.m + tok + t_in[k] : 0x3FFFFFFF;
          }
          *reinterpret_cast<float4*>(&col_lse[sb][lane * 4]) = l;
          *reinterpret_cast<int4*>(&col_lim[sb][lane * 4]) = s;
          __syncwarp();
          if (lane == 0) bar_arrive(bars.c_full(sb));
        }
        return true;
      });
    } else {
      // ---- products with every second row tile (one warp is behind: an instruction with its operands takes about 80
      // cycles to issue)
      constexpr uint32_t shape = mma_shape(BF16, 128, 128, false);
      const uint32_t w = warp - 16;
      int kb = kKeyBufs - 1;
      uint32_t k_phase = 1, n_done = 0;
      bool holds = false;   // a key tile is held
      const uint64_t k_op = smem_operand(k_at), q_op = smem_operand(q_at);
      const bool ok = run_segments([] {}, [&](int, int, int n) {
        if (holds && elect_one()) tc_commit(bars.k_empty(kb));
        __syncwarp();
        if (++kb == kKeyBufs) kb = 0, k_phase ^= 1;
        holds = true;
        if (!bar_wait(bars.k_full(kb), k_phase, &gave_up)) return false;
        const uint64_t ka = k_op + 2 * kb * (T::kBytesTile >> 4);
        for (; n > 0; --n, ++n_done) {
          if ((n_done & 1) != w) continue;
          const uint32_t qs = n_done % RING, sb = 2 * (n_done % kScores);
          if (!bar_wait(bars.q_full(qs), n_done / RING & 1, &gave_up)) return false;
          const uint64_t qb = q_op + qs * (T::kBytesTile >> 4);
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            if (!bar_wait(bars.s_empty(sb + half), (n_done / kScores & 1) ^ 1, &gave_up)) return false;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
              for (int ks = 0; ks < KS; ++ks) {
                constexpr int kBlock = 16384 >> 4, kStep = 32 >> 4;
                mma_ss(tmem + (sb + half) * 128, ka + half * (T::kBytesTile >> 4) + (ks >> 2) * kBlock + (ks & 3) * kStep,
                       qb + (ks >> 2) * kBlock + (ks & 3) * kStep, shape, ks != 0);
              }
              tc_commit(bars.s_full(sb + half));
              if (half) tc_commit(bars.q_empty(qs));
            }
            __syncwarp();
          }
        }
        return true;
      });
      // (what the last products still read is in use until the warpgroups have their scores)
      if (!ok) {
        if (lane == 0) tc_commit(bars.drain());
        const long long c = clock64();
        while (!bar_try(bars.drain(), 0) && clock64() - c < 100000000ll) {
        }
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
    // ---- sums; warpgroup w has the keys of half w & 1 and every second row tile, whose scores are always at the same place
    const int w = warp >> 2, half = w & 1, k_in = (warp & 3) * 32 + lane;
    const uint32_t s_at = tmem + w * 128 + ((uint32_t)((warp & 3) * 32) << 16);
    const float scale = a.scale_log2;
    const float2 mul = make_float2(scale, scale);
    const int window = a.window ? (int)a.window : 0x40000001;   // (no last key has a first one then)
    uint32_t n = 0;       // row tiles so far
    uint32_t mine = 0;    // of them, this warpgroup's
    uint32_t items = 0;
    while (true) {
      const int x1 = (int)min((long long)it.tiles(), x0 + (end - at));
      const int j0 = it.kt * kTile + half * kHalf, j = j0 + k_in, past = it.len - it.m;
      float2 sum = make_float2(0.0f, 0.0f);
      const int skip = (int)(((w >> 1) - n) & 1);        // the first tile of the run that is this warpgroup's
      int r = (x0 + skip) % it.rts;                      // row tile of tile x
      for (int x = x0 + skip; x < x1; x += 2, ++mine) {
        const int rt = it.rt0 + r;
        for (r += 2; r >= it.rts;) r -= it.rts;
        // every row of the tile there, and seeing every key of it?  Or none of them any?
        const bool clean = rows_t == 128 && (rt + 1) * tpt <= it.m && j0 + kHalf <= it.len &&
                           (!a.causal || (j0 + kHalf - 1 <= past + rt * tpt && (!a.window || j0 > past + (rt + 1) * tpt - 1 - (int)a.window)));
        const bool blank = j0 >= it.len || (a.causal && j0 > past + min((rt + 1) * tpt, it.m) - 1);
        const int cb = (w >> 1) + (int)(mine & 1) * kScores;   // (this is tile 2 mine + w / 2)
        bar_wait(bars.c_full(cb), mine >> 1 & 1, &gave_up);
        bar_wait(bars.s_full(w), mine & 1, &gave_up);
        tc_fence_after();
        if (blank) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) bar_arrive(bars.s_empty(w));
        } else {
#pragma unroll
          for (int part = 0; part < 2; ++part) {
            uint32_t s[2][32];
            tmem_load32(s[0], s_at + part * 64);
            tmem_load32(s[1], s_at + part * 64 + 32);
            tmem_load_wait();
            if (part == 1) {  // the scores are in registers
              tc_fence_before();
              __syncwarp();
              if (lane == 0) bar_arrive(bars.s_empty(w));
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              if (clean) {
#pragma unroll
                for (int i = 0; i < 32; i += 4) {
                  const float4 nl = *reinterpret_cast<const float4*>(&col_lse[cb][part * 64 + c * 32 + i]);
                  float2 p = fma2(make_float2(__uint_as_float(s[c][i]), __uint_as_float(s[c][i + 1])), mul, make_float2(nl.x, nl.y));
                  float2 q = fma2(make_float2(__uint_as_float(s[c][i + 2]), __uint_as_float(s[c][i + 3])), mul, make_float2(nl.z, nl.w));
                  p.x = exp2_fast(p.x); p.y = exp2_fast(p.y);
                  q.x = exp2_fast(q.x); q.y = exp2_fast(q.y);
                  sum = add2(sum, add2(p, q));
                }
              } else {
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                  const int col = part * 64 + c * 32 + i;
                  const float p = exp2_fast(fmaf(__uint_as_float(s[c][i]), scale, col_lse[cb][col]));
                  sum.x += j <= col_lim[cb][col] && j > col_lim[cb][col] - window ? p : 0.0f;
                }
              }
            }
          }
        }
        __syncwarp();
        if (lane == 0) bar_arrive(bars.c_empty(cb));
      }
      n += x1 - x0;
      // ---- the item's sums, or their part
      const float own = sum.x + sum.y;
      float(&other)[2][kHalf] = others[items++ & 1];   // (read before the barrier of the next item)
      if (w > 1) other[half][k_in] = own;
      asm volatile("bar.sync 5, 512;" ::: "memory");
      if (w < 2) {
        float all = own + other[half][k_in];
        bool write = x0 == 0 && x1 == it.tiles();
        if (!write) {
          const long long item0 = at - x0, c0 = item0 / share.share, c1 = (item0 + it.tiles() - 1) / share.share;
          const int entry = half * kHalf + k_in;
          __stcg(a.partial + ((uint64_t)blockIdx.x * 2 + (x0 == 0 ? 1 : 0)) * kTile + entry, all);
          __threadfence();
          group_sync(half);
          if (k_in == 0) {
            const uint32_t got = atomicAdd(a.arrived + 2 * c0 + half, 1u);
            last_part[half] = got == (uint32_t)(c1 - c0);
            if (last_part[half]) a.arrived[2 * c0 + half] = 0;  // for the next call
          }
          group_sync(half);
          write = last_part[half];
          if (write) {
            __threadfence();
            all = 0.0f;
            for (long long c = c0; c <= c1; ++c) all += __ldcg(a.partial + ((uint64_t)c * 2 + (c == c0 ? 1 : 0)) * kTile + entry);
          }
        }
        if (write && j < it.len) {
          const uint32_t jp = div_fast((uint32_t)j, a.pool.page);
          const int page = page_of(a.seq.table + (int64_t)it.b * a.seq.table_stride, jp, a.pool.num_pages, a.status);
          if (page >= 0) {
            float* to = a.pool.weights + ((int64_t)page * a.pool.groups + it.g) * a.pool.page.d + (j - (int)(jp * a.pool.page.d));
            *to = a.decay == 1.0f ? *to + all : *to * a.decay + all;
          }
        }
      }
      at += x1 - x0;
      if (at >= end) break;
      next_keys(a, it, tpt);
      x0 = 0;
    }
  }
  tc_fence_before();
  __syncthreads();
  if (tid == 0 && gave_up) atomicOr(a.status, (uint32_t)kGaveUp);
  if (warp == 16) tmem_free(tmem, 512);
}

template <bool BF16, int DP>
cudaError_t weigh_at(const WeighArgs& a, const PoolMaps& maps, const CUtensorMap& q, int tpt, cudaStream_t s) {
  static SmemOptIn done;
  auto* kernel = weigh_tc_kernel<BF16, DP>;
  if (cudaError_t e = allow_dynamic_smem(reinterpret_cast<const void*>(kernel), Wt<DP>::kBytes, &done)) return e;
  kernel<<<sm_count(), kThreads, Wt<DP>::kBytes, s>>>(a, maps, q, tpt);
  count_launches(1);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_weigh_tc(const WeighArgs& a, uint32_t dtype, cudaStream_t s) {
  PoolMaps maps;
  CUtensorMap q;
  const uint32_t group = a.group.d, tpt = 128 / group;   // (the caller has checked that a token's group fits)
  if (!make_pool_maps(a.pool, dtype, &maps) ||
      !make_rows_map(a.q, a.q_tok, a.q_head, a.seq.tokens, a.pool.kv_heads * group, a.pool.dim, dtype, group, tpt, &q))
    return launch_weigh_stream(a, dtype, s);
  if (a.pool.dim <= 64) return dtype == 4 ? weigh_at<true, 64>(a, maps, q, tpt, s) : weigh_at<false, 64>(a, maps, q, tpt, s);
  return dtype == 4 ? weigh_at<true, 128>(a, maps, q, tpt, s) : weigh_at<false, 128>(a, maps, q, tpt, s);
}

}  // namespace grand
