// Pieces shared by the streaming kernels of the token cache: 16 x 8 x 16 tile products on 16-bit operands, asynchronous
// row copies into shared memory, and the layout of those rows.
#pragma once
#include "grand_cache.h"

namespace grand {

constexpr float kLn2 = 0.693147180559945309f;
constexpr float kNegInf = -__builtin_huge_valf();

// Unnormalised probabilities are 2^(s - m + kLift): a float16 has no numbers below 2^-24, so without the lift all keys whose probability is
// below 2^-25 of a row's largest would vanish from the output and stay in the sum.  m is at most 8 behind the maximum, so the
// largest number is 2^15, the last power of two that a float16 holds.  A bfloat16 has the range of 32 bits.
template <bool BF16>
constexpr float kLift = BF16 ? 0.0f : 7.0f;

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

template <bool BF16>
__device__ __forceinline__ void mma_m16n8k16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (BF16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// lo in the lower half
template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint32_t r;
  if constexpr (BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

template <bool BF16>
__device__ __forceinline__ float2 unpack2(uint32_t x) {
  if constexpr (BF16) return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xFFFF0000u));
  else return __half22float2(*reinterpret_cast<const __half2*>(&x));
}

// 16 bytes into shared memory, or zeros (the address is not read then)
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool ok) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// A row of DP 16-bit entries takes DP * 2 bytes rounded up to 128 or 256; its 16-byte chunk c sits at place c ^ (row & 7),
// so that the eight rows of an 8 x 8 matrix lie in eight different bank groups.
template <int DP>
struct RowLayout {
  static constexpr int kBytes = DP <= 64 ? 128 : 256;
  static constexpr int kChunks = DP / 8;
  __device__ __forceinline__ static uint32_t at(int row, int chunk) { return row * kBytes + ((chunk ^ (row & 7)) << 4); }
};

// Entries i and i + 1 of a row, zeros behind its end.
__device__ __forceinline__ uint32_t load_pair(const uint16_t* p, int i, int dim) {
  return i < dim ? __ldg(reinterpret_cast<const uint32_t*>(p + i)) : 0u;  // dim is even, i is even
}

}  // namespace grand
