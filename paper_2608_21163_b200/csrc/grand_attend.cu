// Attention of a few query rows over a paged cache, streaming (include/grand.h: grand_cache_attend).
//
// For the rows of one kv head (group query heads x new tokens) o = sum_j p_j v_j / sum_j p_j with
// p_j = 2^(s_j - m), s_j = scale log2(e) q.k_j, in one pass over the keys with a running maximum m.  With few rows a key
// (4 dim bytes with its value) costs 4 rows dim flops, far below what the tensor cores sustain per byte, so up to 16 rows the
// bytes of the cache bound it: 64 sequences of up to 32,768 tokens read 6.7 TB/s.  A second tile of 16 rows doubles what a warp does
// between two loads, and that bounds it then (8 x 32,768 tokens of 8 heads: 16 rows 178 us, 32 rows 282, on the same
// bytes).  The kernel is a stream.  Every warp is a stream of its own - 16 keys and values at
// a time through a ring in shared memory that it alone fills and reads, with its own m, l and o - and needs no barrier
// but its own until a piece ends.
//
// Work split: the pieces (sequence, kv head, row tile) x (tiles of 16 keys a warp) are numbered through, and every block takes
// an equal run of them, so that long and short sequences fill the card alike.  A run covers parts of at most two items
// besides whole ones; the parts' sums go to the workspace, and the block that arrives last at an item joins its
// parts in their order (the result does not depend on who that is).
#include "grand_attend_items.cuh"

namespace grand {
namespace {

constexpr int kKeys = 16, kStages = 3;

template <int DP, int WARPS>
constexpr int stream_smem() {
  return WARPS * kStages * 2 * kKeys * RowLayout<DP>::kBytes;
}

template <bool BF16, int DP, int MT, int kWarps>
__global__ void __launch_bounds__(kWarps * 32, 8 / kWarps) attend_stream_kernel(const __grid_constant__ AttendArgs a) {
  constexpr int kTile = kWarps * kKeys, ROWS = 16 * MT, KS = DP / 16, NT = DP / 8;
  using L = RowLayout<DP>;
  constexpr int kRowsBytes = kKeys * L::kBytes;        // one stage's keys
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ float join_m[ROWS], join_l[ROWS];
  __shared__ uint32_t last_block;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int kvh = (int)a.pool.kv_heads, dim = (int)a.pool.dim;

  // A block takes two tiles at least, and items of up to five tiles whole: the join of parts through memory costs as much as
  // four of them (600 keys of 8 heads: 12.4 us whole, 16.8 in three parts; 1,000 keys: 20.4 whole, 15.2 in four).
  Run run;
  plan_run<ROWS, kTile, kWarps>(a, 2, 5, run);
  if (!run.any) return;
  Item& it = run.it;
  const long long share = run.share, end = run.end;
  long long at = run.first;
  int in_item = run.tile;
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + warp * (kStages * 2 * kRowsBytes);
  while (true) {
    // ---- one piece: tiles [t0, t1) of the item
    const int t0 = in_item, t1 = run.last(it, t0, at);
    const int rows = it.m * (int)a.group.d, r_base = it.rt * ROWS;
    const int32_t* table = a.seq.table + (int64_t)it.b * a.seq.table_stride;
    const int64_t head_at = (int64_t)it.h * a.pool.head_stride;

    uint32_t qf[MT][KS][4];
    int lim[MT][2];   // keys [low, lim] that the row attends (rows behind the last: all, for nothing)
    int low[MT][2];
    int lim_all = 0x7FFFFFFF, low_all = 0;   // ... that every row attends
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int r = r_base + mt * 16 + half * 8 + (lane >> 2);
        const bool ok = r < rows;
        const int tok = ok ? (int)div_fast(r, a.group) : 0, g = ok ? r - tok * (int)a.group.d : 0;
        lim[mt][half] = ok ? (a.causal ? min(it.len - 1, it.len - it.m + tok) : it.len - 1) : 0x7FFFFFFF;
        low[mt][half] = ok && a.window ? it.len - it.m + tok - (int)a.window + 1 : 0;
        lim_all = min(lim_all, lim[mt][half]);
        low_all = max(low_all, low[mt][half]);
        const uint16_t* q = static_cast<const uint16_t*>(a.q) + (int64_t)(it.row + tok) * a.q_tok + (int64_t)(it.h * (int)a.group.d + g) * a.q_head;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const int i = ks * 16 + (lane & 3) * 2;
          qf[mt][ks][half] = ok ? load_pair(q, i, dim) : 0u;
          qf[mt][ks][2 + half] = ok ? load_pair(q, i + 8, dim) : 0u;
        }
      }

    float o[MT][NT][4], m[MT][2], l[MT][2];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
      for (int i = 0; i < 2; ++i) m[mt][i] = kNegInf, l[mt][i] = 0.0f;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[mt][n][i] = 0.0f;
    }

    lim_all = __reduce_min_sync(0xFFFFFFFFu, lim_all);
    low_all = __reduce_max_sync(0xFFFFFFFFu, low_all);

    // tile t's 16 keys of this warp start at lo + t * kTile + warp * kKeys; lane r (and r + 16) looks up the place of key r:
    // -1 behind the last key, kNoPage where the table names no page of the pool (such a token takes no part)
    constexpr int64_t kNoPage = -2;
    auto place = [&](int t) -> int64_t {
      const int j = it.lo + t * kTile + warp * kKeys + (lane & 15);
      if (t >= t1 || j >= it.hi) return -1;
      const uint32_t jp = div_fast((uint32_t)j, a.pool.page);
      const int p = page_of(table, jp, a.pool.num_pages, a.status);
      return p < 0 ? kNoPage : p * a.pool.page_stride + (j - (int)(jp * a.pool.page.d)) * a.pool.slot_stride + head_at;
    };
    bool gaps = false;   // such a token is among the tiles fetched so far; which it is is then looked up again at its tile
    auto fetch = [&](int stage, int64_t where) {
      const uint32_t kd = ring + stage * 2 * kRowsBytes, vd = kd + kRowsBytes;
      gaps |= __any_sync(0xFFFFFFFFu, where == kNoPage);
      constexpr int C = L::kChunks, N = kKeys * C / 32;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int x = i * 32 + lane, r = x / C, c = x - r * C;
        const int64_t w = __shfl_sync(0xFFFFFFFFu, where, r);
        const bool ok = w >= 0 && c * 8 < dim;
        const int64_t at2 = ok ? (w + c * 8) * 2 : 0;
        copy16(kd + L::at(r, c), a.pool.k + at2, ok);
        copy16(vd + L::at(r, c), a.pool.v + at2, ok);
      }
    };
    int64_t next = place(t0);
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) {
      const int64_t now = next;
      next = place(t0 + s + 1);
      if (t0 + s < t1) fetch(s, now);
      copy_commit();
    }
    int stage = 0;
    for (int t = t0; t < t1; ++t) {
      copy_wait<kStages - 2>();
      __syncwarp();
      {
        // the stage that is filled now was read in the last round, by this warp
        const int64_t now = next;
        next = place(t + kStages);
        if (t + kStages - 1 < t1) fetch(stage == 0 ? kStages - 1 : stage - 1, now);
        copy_commit();
      }
      const uint32_t ks0 = ring + stage * 2 * kRowsBytes, vs0 = ks0 + kRowsBytes;
      stage = stage + 1 == kStages ? 0 : stage + 1;
      const int j0 = it.lo + t * kTile + warp * kKeys;
      const uint32_t gone = gaps ? __ballot_sync(0xFFFFFFFFu, place(t) == kNoPage) : 0u;   // bit r: key r is such a token

      float s[MT][2][4];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[mt][n][i] = 0.0f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        uint32_t kf[4];
        ldmatrix4(kf, ks0 + L::at(((lane >> 4) << 3) + (lane & 7), ks * 2 + ((lane >> 3) & 1)));
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          mma_m16n8k16<BF16>(s[mt][0], qf[mt][ks], kf[0], kf[1]);
          mma_m16n8k16<BF16>(s[mt][1], qf[mt][ks], kf[2], kf[3]);
        }
      }
      uint32_t pf[MT][4], pr[MT][4];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        float top[2] = {kNegInf, kNegInf};
        if (j0 + kKeys - 1 <= lim_all && j0 >= low_all && gone == 0) {
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[mt][n][i] *= a.scale_log2;
        } else {
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int r = n * 8 + (lane & 3) * 2 + (i & 1), j = j0 + r;
              // a masked place takes no part, whatever its key holds
              s[mt][n][i] = j <= lim[mt][i >> 1] && j >= low[mt][i >> 1] && !(gone >> r & 1) ? s[mt][n][i] * a.scale_log2 : kNegInf;
            }
        }
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) top[i >> 1] = fmaxf(top[i >> 1], s[mt][n][i]);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          top[i] = fmaxf(top[i], __shfl_xor_sync(0xFFFFFFFFu, top[i], 1));
          top[i] = fmaxf(top[i], __shfl_xor_sync(0xFFFFFFFFu, top[i], 2));
        }
        // The reference of the exponents follows the maximum only when it is 8 (a factor of 256) behind: the sums stay
        // far inside their range, and the output is rescaled a few times per sequence instead of at every step.
        if (__any_sync(0xFFFFFFFFu, top[0] > m[mt][0] + 8.0f || top[1] > m[mt][1] + 8.0f)) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float mn = top[i] > m[mt][i] + 8.0f ? top[i] : m[mt][i];   // (rows stay independent of each other)
            const float f = mn == m[mt][i] ? 1.0f : exp2_fast(m[mt][i] - mn);
            m[mt][i] = mn;
            l[mt][i] *= f;
#pragma unroll
            for (int n = 0; n < NT; ++n) o[mt][n][2 * i] *= f, o[mt][n][2 * i + 1] *= f;
          }
        }
        const float ref[2] = {m[mt][0] == kNegInf ? 0.0f : m[mt][0] - kLift<BF16>, m[mt][1] == kNegInf ? 0.0f : m[mt][1] - kLift<BF16>};
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            s[mt][n][i] = exp2_fast(s[mt][n][i] - ref[i >> 1]);
            l[mt][i >> 1] += s[mt][n][i];
          }
        // P as the sum of two 16-bit numbers: the tensor cores have time for both, and the output is then off by its
        // own rounding alone
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x = s[mt][i >> 1][(i & 1) * 2], y = s[mt][i >> 1][(i & 1) * 2 + 1];
          pf[mt][i] = pack2<BF16>(x, y);
          const float2 z = unpack2<BF16>(pf[mt][i]);
          pr[mt][i] = pack2<BF16>(x - z.x, y - z.y);
        }
      }
#pragma unroll
      for (int n = 0; n < NT; n += 2) {
        uint32_t vf[4];
        ldmatrix4_trans(vf, vs0 + L::at((((lane >> 3) & 1) << 3) + (lane & 7), n + (lane >> 4)));
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          mma_m16n8k16<BF16>(o[mt][n], pf[mt], vf[0], vf[1]);
          mma_m16n8k16<BF16>(o[mt][n + 1], pf[mt], vf[2], vf[3]);
          mma_m16n8k16<BF16>(o[mt][n], pr[mt], vf[0], vf[1]);
          mma_m16n8k16<BF16>(o[mt][n + 1], pr[mt], vf[2], vf[3]);
        }
      }
      __syncwarp();
    }
    copy_wait<0>();
    __syncthreads();  // the ring is free

    // ---- join the warps: row sums o [ROWS][DP], reference and sum per row and warp
    float* so = reinterpret_cast<float*>(smem);                  // [kWarps][ROWS][DP]
    static_assert(kWarps * ROWS * DP * 4 + kWarps * ROWS * 8 <= stream_smem<DP, kWarps>(), "the join fits the ring");
    float* sm = so + kWarps * ROWS * DP;
    float* sl = sm + kWarps * ROWS;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float x = l[mt][i];
        x += __shfl_xor_sync(0xFFFFFFFFu, x, 1);
        x += __shfl_xor_sync(0xFFFFFFFFu, x, 2);
        const int r = mt * 16 + i * 8 + (lane >> 2);
        if ((lane & 3) == 0) sm[warp * ROWS + r] = m[mt][i], sl[warp * ROWS + r] = x;
#pragma unroll
        for (int n = 0; n < NT; ++n)
          *reinterpret_cast<float2*>(so + (warp * ROWS + r) * DP + n * 8 + (lane & 3) * 2) = make_float2(o[mt][n][2 * i], o[mt][n][2 * i + 1]);
      }
    __syncthreads();
    if (tid < ROWS) {
      float top = kNegInf, sum = 0.0f;
      for (int w = 0; w < kWarps; ++w) top = fmaxf(top, sm[w * ROWS + tid]);
      for (int w = 0; w < kWarps; ++w) {
        const float f = top == kNegInf ? 0.0f : exp2_fast(sm[w * ROWS + tid] - top);
        sum += sl[w * ROWS + tid] * f;
        sm[w * ROWS + tid] = f;
      }
      join_m[tid] = top;
      join_l[tid] = sum;
    }
    __syncthreads();
    const int n_rows = min(ROWS, rows - r_base);
    const bool whole = t0 == 0 && t1 == it.tiles;
    auto emit = [&](int r, int c, float x, float y, float sum) {   // entries c and c + 1 of row r
      const int row = r_base + r, tok = (int)div_fast(row, a.group), g = row - tok * (int)a.group.d;
      const int64_t q = (int64_t)(it.row + tok) * kvh * a.group.d + it.h * (int)a.group.d + g;
      const float f = sum > 0.0f ? 1.0f / sum : (sum == 0.0f ? 0.0f : sum);  // (a NaN stays one)
      *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.out) + q * dim + c) = pack2<BF16>(x * f, y * f);
    };
    auto emit_lse = [&](int r, float top, float sum) {
      const int row = r_base + r, tok = (int)div_fast(row, a.group), g = row - tok * (int)a.group.d;
      if (a.lse) a.lse[(int64_t)(it.row + tok) * kvh * a.group.d + it.h * (int)a.group.d + g] = (top - kLift<BF16> + log2f(sum)) * kLn2;
    };
    float* slot = a.partial + ((uint64_t)blockIdx.x * 2 + (t0 == 0 ? 1 : 0)) * a.slot_floats;
    for (int x = tid; x < n_rows * (DP / 2); x += blockDim.x) {
      const int r = x / (DP / 2), c = (x - r * (DP / 2)) * 2;
      float v0 = 0.0f, v1 = 0.0f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float2 p = *reinterpret_cast<const float2*>(so + (w * ROWS + r) * DP + c);
        const float f = sm[w * ROWS + r];
        v0 += p.x * f;
        v1 += p.y * f;
      }
      if (!whole) *reinterpret_cast<float2*>(slot + r * DP + c) = make_float2(v0, v1);
      else if (c < dim) emit(r, c, v0, v1, join_l[r]);
    }
    if (tid < n_rows) {
      if (!whole) slot[ROWS * DP + tid] = join_m[tid], slot[ROWS * DP + ROWS + tid] = join_l[tid];
      else emit_lse(tid, join_m[tid], join_l[tid]);
    }
    if (!whole) {
      // the item's tiles are [item0, item0 + tiles) of all; its parts lie in the blocks c0 .. c1
      const long long item0 = at - t0;
      const long long c0 = item0 / share, c1 = (item0 + it.tiles - 1) / share;
      __threadfence();
      __syncthreads();
      if (tid == 0) {
        const uint32_t n = atomicAdd(a.arrived + c0, 1u);
        last_block = n == (uint32_t)(c1 - c0);
        if (last_block) a.arrived[c0] = 0;  // for the next call
      }
      __syncthreads();
      if (last_block) {
        __threadfence();
        const int parts = (int)(c1 - c0) + 1;
        const float* part0 = a.partial + ((uint64_t)c0 * 2 + 1) * a.slot_floats;    // the item begins in the second slot of its first block,
        const float* part1 = a.partial + (uint64_t)(c0 + 1) * 2 * a.slot_floats;    // and goes on in the first slots of the others
        const uint64_t step = 2 * a.slot_floats;
        if (tid < n_rows) {
          const float m0 = __ldcg(part0 + ROWS * DP + tid), l0 = __ldcg(part0 + ROWS * DP + ROWS + tid);
          float top = m0, sum = l0;
#pragma unroll 8
          for (int k = 0; k < parts - 1; ++k) {
            const float pm = __ldcg(part1 + k * step + ROWS * DP + tid), pl = __ldcg(part1 + k * step + ROWS * DP + ROWS + tid);
            const float up = fmaxf(top, pm), ref = up == kNegInf ? 0.0f : up;
            sum = sum * exp2_fast(top - ref) + pl * exp2_fast(pm - ref);
            top = up;
          }
          join_m[tid] = top;
          join_l[tid] = sum;
          emit_lse(tid, top, sum);
        }
        __syncthreads();
        for (int x = tid; x < n_rows * (DP / 2); x += blockDim.x) {
          const int r = x / (DP / 2), c = (x - r * (DP / 2)) * 2;
          const float ref = join_m[r] == kNegInf ? 0.0f : join_m[r];
          const float f0 = exp2_fast(__ldcg(part0 + ROWS * DP + r) - ref);
          const float2 y0 = __ldcg(reinterpret_cast<const float2*>(part0 + r * DP + c));
          float v0 = y0.x * f0, v1 = y0.y * f0;
#pragma unroll 8
          for (int k = 0; k < parts - 1; ++k) {
            const float* p = part1 + k * step;
            const float f = exp2_fast(__ldcg(p + ROWS * DP + r) - ref);
            const float2 y = __ldcg(reinterpret_cast<const float2*>(p + r * DP + c));
            v0 += y.x * f;
            v1 += y.y * f;
          }
          if (c < dim) emit(r, c, v0, v1, join_l[r]);
        }
      }
    }
    at += t1 - t0;
    if (at >= end) break;
    __syncthreads();  // the ring and the join's statistics are read to the end
    in_item = 0;
    next_item<ROWS, kTile>(a, it);
  }
}

template <bool BF16, int DP, int MT, int WARPS>
cudaError_t stream_at(const AttendArgs& a, cudaStream_t s) {
  static SmemOptIn done;
  auto* kernel = attend_stream_kernel<BF16, DP, MT, WARPS>;
  if (cudaError_t e = allow_dynamic_smem(reinterpret_cast<const void*>(kernel), stream_smem<DP, WARPS>(), &done)) return e;
  kernel<<<8 / WARPS * sm_count(), WARPS * 32, stream_smem<DP, WARPS>(), s>>>(a);
  count_launches(1);
  return cudaGetLastError();
}

template <bool BF16, int DP>
cudaError_t stream_dim(const AttendArgs& a, cudaStream_t s) {
  // one tile of 16 rows where a sequence's rows fit it
  const bool small = (uint64_t)a.seq.tokens * a.group.d <= (uint64_t)a.seq.batch * 16;
  // Few items: eight warps on each, which join in shared memory.  More than there are SMs: two blocks of four warps an SM,
  // so that one streams while the other is between items.
  const bool few = (uint64_t)a.seq.batch * a.pool.kv_heads <= (uint64_t)sm_count();
  if (few) return small ? stream_at<BF16, DP, 1, 8>(a, s) : stream_at<BF16, DP, 2, 8>(a, s);
  return small ? stream_at<BF16, DP, 1, 4>(a, s) : stream_at<BF16, DP, 2, 4>(a, s);
}

template <bool BF16>
cudaError_t stream_type(const AttendArgs& a, cudaStream_t s) {
  return a.pool.dim <= 64 ? stream_dim<BF16, 64>(a, s) : a.pool.dim <= 96 ? stream_dim<BF16, 96>(a, s) : stream_dim<BF16, 128>(a, s);
}

}  // namespace

cudaError_t launch_attend_stream(const AttendArgs& args, uint32_t dtype, cudaStream_t s) {
  AttendArgs a = args;
  a.slot_floats = kStreamSlot;
  return dtype == 4 ? stream_type<true>(a, s) : stream_type<false>(a, s);
}

}  // namespace grand
