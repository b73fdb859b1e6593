// attention_mfma.h - types, matrix instructions and cross-lane steps of the
// matrix-unit attention kernels.
//
// All of them compute the transposed products: scores^T = K Q^T and
// out^T += V^T P^T, so that a query row is a column of every accumulator and
// its maximum, sum and scale live in the lanes that hold the column.  The
// scores' accumulator layout (4 consecutive keys per lane) is also a valid
// layout of the second product's operand once both sides number the keys the
// same way, so that decode's and the prompts' weights never leave their
// registers; a latent cache's scores or weights pass through LDS, where waves
// share a row.
//
// The second product takes weights and values in one 16-bit type: a weight is
// rounded once, by at most half a step of that type, its sum (the divisor) is
// made of the weights before.  Against 64 bits the results are off 1.1 to 1.4
// times as far as those of a computation in 32 bits rounded once (8192 tokens:
// 0.0021 and 0.0016 relative, bf16's half step being 0.0039); two products, of
// a weight's upper and lower half, would take the second one's time twice.
#ifndef TOPKV_ATTENTION_MFMA_H_
#define TOPKV_ATTENTION_MFMA_H_

#include "attention.h"

namespace topkv_attend {

typedef float float2v __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef unsigned int uint2v __attribute__((ext_vector_type(2)));
typedef unsigned int uint4v __attribute__((ext_vector_type(4)));

template <int T> struct Elem;
template <> struct Elem<TOPKV_BF16> {
  typedef __bf16 type;
  typedef __bf16 vec8 __attribute__((ext_vector_type(8)));
  typedef __bf16 vec2 __attribute__((ext_vector_type(2)));
  static __device__ __forceinline__ float4v mfma16(vec8 a, vec8 b, float4v c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ float16v mfma32(vec8 a, vec8 b, float16v c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
  // two e4m3 values (exact in either 16-bit type)
  template <bool kHigh> static __device__ __forceinline__ vec2 from_fp8(uint32_t w) {
    return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, kHigh);
  }
};
template <> struct Elem<TOPKV_FP16> {
  typedef _Float16 type;
  typedef _Float16 vec8 __attribute__((ext_vector_type(8)));
  typedef _Float16 vec2 __attribute__((ext_vector_type(2)));
  static __device__ __forceinline__ float4v mfma16(vec8 a, vec8 b, float4v c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ float16v mfma32(vec8 a, vec8 b, float16v c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
  template <bool kHigh> static __device__ __forceinline__ vec2 from_fp8(uint32_t w) {
    return __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, kHigh);
  }
};

// Weights are exp2(score - reference).  Half floats lose what lies below 2^-14, which a long cache's many small weights
// may be together: their reference lies this far (in powers of two) below the largest score, so that the largest weight
// is 2^14, or 2^6 where the reference may fall 2^8 behind.
template <int T> constexpr float lift(float slack) { return T == TOPKV_FP16 ? 14.f - slack : 0.f; }

// The reference for a largest score x * scale: lowered by the lift, unless floats are so far apart there that it would
// fall further.  The product is rounded as exponent_of() rounds it.
template <int T>
__device__ __forceinline__ float reference(float x, float scale, float slack) {
#pragma clang fp contract(off)
  const float top = x * scale;
  if constexpr (lift<T>(0.f) == 0.f) return top;
  const float low = top - lift<T>(slack);
  return top - low > lift<T>(slack) ? top : low;
}

// Eight e4m3 values as eight of T.
template <int T>
__device__ __forceinline__ uint4v widen(uint2v w) {
  union {
    typename Elem<T>::vec2 h[4];
    uint4v v;
  } u;
  u.h[0] = Elem<T>::template from_fp8<false>(w[0]);
  u.h[1] = Elem<T>::template from_fp8<true>(w[0]);
  u.h[2] = Elem<T>::template from_fp8<false>(w[1]);
  u.h[3] = Elem<T>::template from_fp8<true>(w[1]);
  return u.v;
}

// Rows of NC 16-byte chunks in LDS: chunk c of row r is stored at place
// c ^ swizzle(r).  Both reads, 16 rows of one chunk and 4 rows of 4 chunks,
// then spread over all 64 banks (16 chunks): rows r, r + 1, .. start 16
// chunks apart (NC % 16 == 0) or 8 chunks apart (NC % 16 == 8).
template <int NC>
__device__ __forceinline__ int swizzle(int r) {
  static_assert(NC % 8 == 0, "a row is whole groups of 8 chunks");
  if constexpr (NC % 16 == 0) return (r & 3) << 2 | (r >> 2 & 3);
  else return (r >> 1 & 1) << 2 | (r >> 2 & 3);
}

// Four rows of 16 16-bit values, 4 of them given by each of 16 lanes (row
// lane / 4), returned by columns: lane i has column i.
__device__ __forceinline__ uint2v read_transposed(const char* lds) {
  typedef short4v __attribute__((address_space(3))) * P;
  union {
    short4v s;
    uint2v v;
  } u;
  u.s = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(lds));
  return u.v;
}

// Maximum and sum over the lanes that differ in bit 5, and in bits 4 and 5.
__device__ __forceinline__ float max_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float max_quarters(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return max_halves(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float sum_quarters(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return sum_halves(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// 16 bytes a lane from memory to LDS without registers in between: lane i's go
// to lds + 16 i (lds the same in all lanes; lanes that are off write nothing).
// The compiler does not see these loads: wait_loads() before their LDS is read.
// A scalar write of m0 needs a wait state before a load that takes its LDS
// address from it, and inside an asm text nobody else puts one there.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"   // that m0 is a register of the target's own is why it is named
__device__ __forceinline__ void load_to_lds(char* lds, const char* from) {
  typedef char __attribute__((address_space(3))) * L;
  const uint32_t to = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(L)lds);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(from) : "memory", "m0");
}
__device__ __forceinline__ void load_once_to_lds(char* lds, const char* from) {     // not kept in the L2
  typedef char __attribute__((address_space(3))) * L;
  const uint32_t to = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(L)lds);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off nt" ::"s"(to), "v"(from) : "memory", "m0");
}
#pragma clang diagnostic pop
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// The order of this wave's LDS accesses, for the compiler (the hardware keeps it).
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Running sums of a weight over the requests, each thread of the workgroup
// with a run of neighbours; find() is for the thread whose run holds an item.
template <class I>
struct Scan {
  int32_t lo, hi;      // the thread's requests
  I base, mine;        // weight before them and of them
  I total;

  __device__ bool holds(I item) const { return item >= base && item < base + mine; }
  // The request that item number `item` belongs to; base becomes its first item.
  template <class F> __device__ int32_t find(I item, F weight) {
    int32_t r = lo;
    for (I w = weight(r); item >= base + w && r + 1 < hi; w = weight(++r)) base += w;
    return r;
  }
};

template <class I, int kWaves, class F>
__device__ Scan<I> scan_requests(int32_t num_reqs, F weight) {
  __shared__ I s_sum[kWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int32_t per = (num_reqs + 64 * kWaves - 1) / (64 * kWaves);
  Scan<I> s;
  s.lo = threadIdx.x * per;
  s.hi = s.lo + per < num_reqs ? s.lo + per : num_reqs;
  s.mine = 0;
  for (int32_t r = s.lo; r < s.hi; ++r) s.mine += weight(r);
  I inc = s.mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const I x = __shfl_up(inc, d, 64);
    if (lane >= d) inc += x;
  }
  if (lane == 63) s_sum[wave] = inc;
  __syncthreads();
  s.base = inc - s.mine;
  s.total = 0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    if (i < wave) s.base += s_sum[i];
    s.total += s_sum[i];
  }
  return s;
}

}  // namespace topkv_attend

#endif  // TOPKV_ATTENTION_MFMA_H_
