// Rotary positions, alone and fused with the write of new tokens into the cache's pages.
//
// y_a = a c - b s, y_b = b c + a s for the pairs (a, b) of the first `rot` entries of a head: three flops an entry, so
// the bytes bound it (every entry is read once and written once; a table row is read once per token and serves all of
// its heads).  A unit is what one thread turns at a time: 16 bytes of each half (half layout) or 16 bytes of adjacent
// pairs.  A thread keeps its unit over several heads of one token, with the unit's cosines and sines in registers.
#include "grand_cache.h"

namespace grand {
namespace {

template <typename T>
__device__ __forceinline__ float to_f(T v) { return (float)v; }
template <typename T>
__device__ __forceinline__ T from_f(float v) { return (T)v; }
template <>
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
template <>
__device__ __forceinline__ __half from_f(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f(float v) { return __float2bfloat16_rn(v); }

template <typename T, int VEC>
struct Pack {
  T e[VEC];
};
template <typename T, int VEC>
__device__ __forceinline__ Pack<T, VEC> load_pack(const T* p) {
  Pack<T, VEC> r;
  if constexpr (VEC * sizeof(T) == 16) {
    *reinterpret_cast<uint4*>(&r) = *reinterpret_cast<const uint4*>(p);
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) r.e[i] = p[i];
  }
  return r;
}
template <typename T, int VEC>
__device__ __forceinline__ void store_pack(T* p, const Pack<T, VEC>& r) {
  if constexpr (VEC * sizeof(T) == 16) {
    *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(&r);
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) p[i] = r.e[i];
  }
}

// One pair, in one order of roundings: the wide and the narrow kernels give equal bits.
__device__ __forceinline__ void turn(float& a, float& b, float c, float s) {
  const float x = __fmaf_rn(a, c, -__fmul_rn(b, s)), y = __fmaf_rn(b, c, __fmul_rn(a, s));
  a = x;
  b = y;
}

// One thread's unit u of the heads [h0, heads) in steps of `step`, of one token.  VEC entries of T are 16 bytes, or 1
// where an offset or an alignment allows no more (INTER then handles one pair at a time).
template <typename T, int VEC, bool INTER>
struct Unit {
  static constexpr int kPer = INTER ? (VEC > 1 ? VEC / 2 : 1) : VEC;  // pairs per unit
  float c[kPer], s[kPer];
  int a, b;   // offsets of the unit's packs in a head; b < 0: copied, not turned
  __device__ __forceinline__ static uint32_t count(uint32_t dim, uint32_t rot) {
    return rot / 2 / kPer + (dim - rot) / VEC;
  }
  __device__ __forceinline__ void place(uint32_t u, uint32_t dim, uint32_t rot) {
    const uint32_t turned = rot / 2 / kPer;
    a = u < turned ? (INTER ? (int)(2 * kPer * u) : (int)(kPer * u)) : (int)(rot + (u - turned) * VEC);
    b = u >= turned ? -1 : INTER ? a : a + (int)(rot / 2);
  }
  // (wide units: the table and its rows' halves start on multiples of what is read at a time)
  __device__ __forceinline__ void angles(uint32_t u, uint32_t rot, const float* row, float sign) {
    if (b < 0) return;
    const float* p = row + u * kPer;
    if constexpr (kPer % 4 == 0) {
#pragma unroll
      for (int i = 0; i < kPer; i += 4) {
        *reinterpret_cast<float4*>(c + i) = __ldg(reinterpret_cast<const float4*>(p + i));
        *reinterpret_cast<float4*>(s + i) = __ldg(reinterpret_cast<const float4*>(p + rot / 2 + i));
      }
    } else {
#pragma unroll
      for (int i = 0; i < kPer; ++i) c[i] = __ldg(p + i), s[i] = __ldg(p + rot / 2 + i);
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) s[i] *= sign;
  }
  // a head's part of the unit: read, and turned and written
  struct Part {
    Pack<T, VEC> p, q;
  };
  __device__ __forceinline__ void read(Part& x, const T* from) const {
    x.p = load_pack<T, VEC>(from + a);
    if constexpr (!INTER) {
      if (b >= 0) x.q = load_pack<T, VEC>(from + b);
    } else if constexpr (VEC == 1) {
      if (b >= 0) x.q = load_pack<T, VEC>(from + a + 1);
    }
  }
  __device__ __forceinline__ void write(Part& x, T* to) const {
    if (b >= 0) {
      if constexpr (INTER && VEC > 1) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          float v = to_f(x.p.e[2 * i]), w = to_f(x.p.e[2 * i + 1]);
          turn(v, w, c[i], s[i]);
          x.p.e[2 * i] = from_f<T>(v);
          x.p.e[2 * i + 1] = from_f<T>(w);
        }
      } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          float v = to_f(x.p.e[i]), w = to_f(x.q.e[i]);
          turn(v, w, c[i], s[i]);
          x.p.e[i] = from_f<T>(v);
          x.q.e[i] = from_f<T>(w);
        }
        store_pack<T, VEC>(to + (INTER ? a + 1 : b), x.q);
      }
    }
    store_pack<T, VEC>(to + a, x.p);
  }
};

__device__ __forceinline__ const float* table_row(const RopeArgs& a, uint64_t t) {
  if (a.rot == 0) return a.table;
  int p = __ldg(a.positions + t);
  if (p < 0 || (uint64_t)p >= a.table_rows) {
    if (a.status) atomicOr(a.status, (uint32_t)kBadPosition);
    p = p < 0 ? 0 : (int)(a.table_rows - 1);
  }
  return a.table + (uint64_t)p * a.rot;
}

// A block covers blockDim.y tokens; the threadIdx.x of one token split into units and head lanes, and a thread takes
// kHeads heads at a time.  Everything it reads of them is asked for before the position and the table row, whose
// reads wait for each other (one head at a time, asked for last: 38 us instead of 23 on 8,191 tokens of 32 heads of 128).
constexpr int kHeads = 4;

template <typename T, int VEC, bool INTER>
__global__ void __launch_bounds__(256) rope_kernel(RopeArgs a) {
  using U = Unit<T, VEC, INTER>;
  const uint32_t units = U::count(a.dim, a.rot), lanes = blockDim.x / units;
  const uint32_t u0 = threadIdx.x % units, h0 = threadIdx.x / units;
  const uint64_t t = (uint64_t)blockIdx.x * blockDim.y + threadIdx.y;
  if (t >= a.tokens || h0 >= lanes) return;
  const T* x = static_cast<const T*>(a.x) + t * a.x_tok;
  T* y = static_cast<T*>(a.out) + t * a.o_tok;
  U unit;
  unit.place(u0, a.dim, a.rot);
  bool known = false;
  for (uint32_t h = h0; h < a.heads; h += lanes * kHeads) {
    typename U::Part part[kHeads];
#pragma unroll
    for (int i = 0; i < kHeads; ++i)
      if (h + i * lanes < a.heads) unit.read(part[i], x + (h + i * lanes) * a.x_head);
    if (!known) unit.angles(u0, a.rot, table_row(a, t), a.sign);
    known = true;
#pragma unroll
    for (int i = 0; i < kHeads; ++i)
      if (h + i * lanes < a.heads) unit.write(part[i], y + (h + i * lanes) * a.o_head);
  }
}

// The sequence of token t, the last whose first row is at most t, by a whole warp: 32 parts of the range at a time, so one
// read for up to 32 sequences where a search by halves waits for five.
__device__ __forceinline__ uint32_t find_seq(const int32_t* cu, uint32_t batch, int t) {
  uint32_t lo = 0, n = batch;
  const uint32_t lane = threadIdx.x & 31;
  while (n > 1) {
    const uint32_t step = (n + 31) / 32, at = lo + lane * step;
    const bool below = lane * step < n && __ldg(cu + at) <= t;
    const uint32_t hit = __ballot_sync(0xFFFFFFFFu, below);
    const uint32_t k = hit ? 31 - __clz(hit) : 0;
    const uint32_t end = lo + n;
    lo += k * step;
    n = min(step, end - lo);
  }
  return lo;
}

template <typename T, int VEC, bool INTER>
__global__ void __launch_bounds__(256) append_kernel(const __grid_constant__ AppendArgs a) {
  using U = Unit<T, VEC, INTER>;
  const uint32_t dim = a.pool.dim, kvh = a.pool.kv_heads, heads = a.q.heads + kvh;
  const uint32_t units = U::count(dim, a.q.rot), lanes = blockDim.x / units;
  const uint32_t u0 = threadIdx.x % units, h0 = threadIdx.x / units;
  const uint64_t t = (uint64_t)blockIdx.x * blockDim.y + threadIdx.y;   // (a warp has one token)
  if (t >= a.seq.tokens) return;
  const T* k = static_cast<const T*>(a.k) + t * a.k_tok;
  const T* v = static_cast<const T*>(a.v) + t * a.v_tok;
  const T* q = static_cast<const T*>(a.q.x) + t * a.q.x_tok;
  T* qo = static_cast<T*>(a.q.out) + t * a.q.o_tok;
  U unit;
  unit.place(u0, dim, a.q.rot);
  // the first round of what it moves, before all lookups
  typename U::Part part[kHeads];
  auto read = [&](uint32_t h) {
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
      const uint32_t hh = h + i * lanes;
      if (hh < heads) unit.read(part[i], hh < a.q.heads ? q + hh * a.q.x_head : k + (hh - a.q.heads) * a.k_head);
    }
  };
  if (h0 < lanes) read(h0);
  const uint32_t per = dim / VEC, values = kvh * per;
  Pack<T, VEC> value;
  auto value_at = [&](const T* base, uint32_t i, int64_t head_stride) {
    const uint32_t h = i / per;
    return base + h * head_stride + (i - h * per) * VEC;
  };
  if (threadIdx.x < values) value = load_pack<T, VEC>(value_at(v, threadIdx.x, a.v_head));
  const float* row = table_row(a.q, t);
  const uint32_t b = a.seq.cu ? find_seq(a.seq.cu, a.seq.batch, (int)t) : (uint32_t)t;
  if (h0 < lanes) unit.angles(u0, a.q.rot, row, a.q.sign);
  // The slot comes from the length and the bounds as they are: clipped ones would name the slot of another token.  A token whose
  // slot the table does not reach (or before the first), or whose sequence's bounds are not rows of this call, is dropped.
  const int len = a.seq.lens[b], lo = a.seq.cu ? a.seq.cu[b] : (int)b, hi = a.seq.cu ? a.seq.cu[b + 1] : lo + 1;
  const bool bounds = 0 <= lo && lo <= hi && hi <= (int)a.seq.tokens;
  const int slot = len - hi + (int)t;   // (used where 0 <= len and lo <= t < hi: no overflow)
  const bool mine = bounds && (int)t >= lo && (int)t < hi && len >= 0 && (uint32_t)slot < a.seq.max_len;
  if (!bounds || (uint32_t)len > a.seq.max_len) atomicOr(a.q.status, (uint32_t)kBadLength);
  int page = -1;
  uint32_t in_page = 0;
  if (mine) {
    const uint32_t jp = div_fast((uint32_t)slot, a.pool.page);
    in_page = (uint32_t)slot - jp * a.pool.page.d;
    page = page_of(a.seq.table + (int64_t)b * a.seq.table_stride, jp, a.pool.num_pages, a.q.status);
  }
  const int64_t at = page < 0 ? 0 : page * a.pool.page_stride + in_page * a.pool.slot_stride;
  T* kd = reinterpret_cast<T*>(a.pool.k) + at;
  T* vd = reinterpret_cast<T*>(a.pool.v) + at;
  if (h0 < lanes)
    for (uint32_t h = h0; h < heads; h += lanes * kHeads) {
      if (h != h0) read(h);
#pragma unroll
      for (int i = 0; i < kHeads; ++i) {
        const uint32_t hh = h + i * lanes;
        if (hh < a.q.heads) unit.write(part[i], qo + hh * a.q.o_head);
        else if (hh < heads && page >= 0) unit.write(part[i], kd + (hh - a.q.heads) * a.pool.head_stride);
      }
    }
  if (page < 0) return;
  for (uint32_t i = threadIdx.x; i < values; i += blockDim.x) {
    if (i != threadIdx.x) value = load_pack<T, VEC>(value_at(v, i, a.v_head));
    store_pack<T, VEC>(const_cast<T*>(value_at(vd, i, a.pool.head_stride)), value);
  }
  if (a.pool.weights)
    for (uint32_t g = threadIdx.x; g < a.pool.groups; g += blockDim.x)
      a.pool.weights[((int64_t)page * a.pool.groups + g) * a.pool.page.d + in_page] = 0.0f;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Threads per token and tokens per block: all heads in one round if 256 threads can, about 128 threads a block.
template <typename T, int VEC, bool INTER>
dim3 block_for(uint32_t dim, uint32_t rot, uint32_t heads, uint32_t copied) {
  constexpr int per = Unit<T, VEC, INTER>::kPer;
  const uint32_t units = rot / 2 / per + (dim - rot) / VEC;
  uint32_t lanes = (heads + kHeads - 1) / kHeads;
  if (lanes * units > 256) lanes = 256 / units;
  if (lanes == 0) lanes = 1;
  uint32_t x = lanes * units;
  if (copied) {   // whole warps; threads behind the last unit move values only
    if (x < copied) x = copied < 128 ? copied : 128;
    x = (x + 31) / 32 * 32;
  }
  uint32_t y = 128 / x;
  return dim3(x, y ? y : 1);
}

template <typename T, int VEC>
cudaError_t rope_at(const RopeArgs& a, cudaStream_t s) {
  const dim3 b = a.interleaved ? block_for<T, VEC, true>(a.dim, a.rot, a.heads, 0) : block_for<T, VEC, false>(a.dim, a.rot, a.heads, 0);
  const uint32_t grid = (uint32_t)((a.tokens + b.y - 1) / b.y);
  if (a.interleaved) rope_kernel<T, VEC, true><<<grid, b, 0, s>>>(a);
  else rope_kernel<T, VEC, false><<<grid, b, 0, s>>>(a);
  count_launches(1);
  return cudaGetLastError();
}

template <typename T, int VEC>
cudaError_t append_at(const AppendArgs& a, cudaStream_t s) {
  const uint32_t heads = a.q.heads + a.pool.kv_heads, copied = a.pool.kv_heads * a.pool.dim / VEC;
  const dim3 b = a.q.interleaved ? block_for<T, VEC, true>(a.pool.dim, a.q.rot, heads, copied)
                                 : block_for<T, VEC, false>(a.pool.dim, a.q.rot, heads, copied);
  const uint32_t grid = (a.seq.tokens + b.y - 1) / b.y;
  if (a.q.interleaved) append_kernel<T, VEC, true><<<grid, b, 0, s>>>(a);
  else append_kernel<T, VEC, false><<<grid, b, 0, s>>>(a);
  count_launches(1);
  return cudaGetLastError();
}

// Packs of 16 bytes need every offset that a unit starts at to be a multiple of them.
bool packs(const RopeArgs& a, uint32_t vec) {
  const uint32_t edge = a.interleaved ? a.rot : a.rot / 2;
  return aligned16(a.table) && edge % vec == 0 && a.dim % vec == 0 && (a.heads == 0 || (aligned16(a.x) && aligned16(a.out) && a.x_tok % vec == 0 &&
         a.x_head % vec == 0 && a.o_tok % vec == 0 && a.o_head % vec == 0));
}

}  // namespace

cudaError_t launch_rope(const RopeArgs& a, uint32_t dtype, cudaStream_t s) {
  if (dtype == 2) return packs(a, 4) ? rope_at<float, 4>(a, s) : rope_at<float, 1>(a, s);
  const bool wide = packs(a, 8);
  if (dtype == 3) return wide ? rope_at<__half, 8>(a, s) : rope_at<__half, 1>(a, s);
  return wide ? rope_at<__nv_bfloat16, 8>(a, s) : rope_at<__nv_bfloat16, 1>(a, s);
}

cudaError_t launch_append(const AppendArgs& a, uint32_t dtype, cudaStream_t s) {
  RopeArgs q = a.q;
  q.dim = a.pool.dim;
  const bool wide = packs(q, 8) && aligned16(a.k) && aligned16(a.v) && a.k_tok % 8 == 0 && a.k_head % 8 == 0 && a.v_tok % 8 == 0 &&
                    a.v_head % 8 == 0;  // (the pool's strides and addresses always allow it)
  if (dtype == 3) return wide ? append_at<__half, 8>(a, s) : append_at<__half, 1>(a, s);
  return wide ? append_at<__nv_bfloat16, 8>(a, s) : append_at<__nv_bfloat16, 1>(a, s);
}

}  // namespace grand
