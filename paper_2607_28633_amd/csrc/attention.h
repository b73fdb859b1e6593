// attention.h - what the attention kernels share (attention.hip: the calls and
// the general kernel; attention_decode.hip, attention_latent.hip, attention_prompt.hip: the matrix-unit kernels).
#ifndef TOPKV_ATTENTION_H_
#define TOPKV_ATTENTION_H_

#include <hip/hip_runtime.h>

#include <cstdint>

#include "topkv.h"

namespace topkv_attend {

// One call, validated.  Byte strides of the cache; element strides of q and out.
struct Args {
  const char* cache;          // layer and first KV head
  const int32_t* tables;      // [num_reqs][bt_stride]
  const int32_t* seq_lens;    // [num_reqs]
  const int32_t* q_starts;    // [num_reqs + 1], or null: one token per request
  const void* q;
  void* out;
  float* lse;                 // may be null
  int64_t num_pages;
  int64_t page_bytes, slot_bytes, head_bytes;
  int64_t value_bytes;        // from a key row to its value row
  int64_t q_stride, out_stride;
  int32_t page_size, bt_stride, num_reqs, total_q;
  uint32_t page_mul, page_shift;   // position / page_size = position * page_mul >> page_shift, positions below 2^30
  uint32_t group_mul, group_shift; // row / group likewise
  int32_t num_heads, kv_heads, group;
  int32_t head_dim, value_dim;
  int32_t window, sinks;
  float scale;                // scale * k_scale * log2(e): scores in powers of two
  float v_scale;
  int32_t dtype, kv_dtype;
  bool out_wide;              // rows of out on 16-byte addresses
};

constexpr int64_t kMostGroups = 1 << 23;   // workgroups of up to 512 threads in a launch of fewer than 2^32 threads
constexpr float kLn2 = 0.693147180559945309f;
constexpr float kLog2e = 1.44269504088896341f;

__device__ __forceinline__ int32_t clamped_len(const Args& a, int32_t r) {
  const int32_t n = a.seq_lens[r], cap = a.bt_stride * a.page_size;
  return n < 0 ? 0 : n > cap ? cap : n;
}

__device__ __forceinline__ int32_t clamped_start(const Args& a, int32_t r) {
  const int32_t s = a.q_starts[r];
  return s < 0 ? 0 : s > a.total_q ? a.total_q : s;
}

// The keys that positions [first, last] of a request see lie at positions
// [0, head) and [start, last + 1): numbered 0 .. head + last + 1 - start in
// that order.  Without a window head = start = 0.
struct Span {
  int32_t head, start, count;
};

__device__ __forceinline__ Span key_span(const Args& a, int32_t first, int32_t last) {
  Span s;
  const int32_t from = first < 0 ? 0 : first;
  s.start = (a.window > 0 && from >= a.window) ? from - a.window + 1 : 0;
  s.head = a.sinks < s.start ? a.sinks : s.start;
  s.count = last < 0 ? 0 : s.head + last + 1 - s.start;
  return s;
}

__device__ __forceinline__ int32_t key_position(const Span& s, int32_t i) { return i < s.head ? i : i - s.head + s.start; }

// j / page_size: with l = ceil(log2(page_size)) the multiplier ceil(2^(30 + l) / page_size) is at most 2^30 / page_size
// too large in 2^(30 + l), which no j below 2^30 can feel.
__device__ __forceinline__ uint32_t page_of(const Args& a, uint32_t j) {
  return (uint32_t)((uint64_t)j * a.page_mul >> a.page_shift);
}

// The new token that a row of a KV head's group belongs to.
__device__ __forceinline__ int32_t token_of(const Args& a, int32_t row) {
  return (int32_t)((uint64_t)(uint32_t)row * a.group_mul >> a.group_shift);
}

// Byte offset of position j's row from a.cache, or -1 when its page lies
// outside the pool.
__device__ __forceinline__ int64_t row_offset(const Args& a, const int32_t* __restrict__ table, int32_t j) {
  const uint32_t page = page_of(a, (uint32_t)j);
  const int32_t e = table[page];
  if (e < 0 || e >= a.num_pages) return -1;
  return (int64_t)e * a.page_bytes + (int64_t)((uint32_t)j - page * (uint32_t)a.page_size) * a.slot_bytes;
}

// x * scale - base with the product rounded before the difference, as it was where base was made of it: in one fused
// step the two differ by half a unit in the product's last place, whole powers of two once scores pass 24 bits.
__device__ __forceinline__ float exponent_of(float x, float scale, float base) {
#pragma clang fp contract(off)
  return x * scale - base;
}
__device__ __forceinline__ float weight_of(float x, float scale, float base) {
  return __builtin_amdgcn_exp2f(exponent_of(x, scale, base));
}

// One element of a row.
template <int T> struct Load;
template <> struct Load<TOPKV_BF16> {
  static constexpr int kBytes = 2;
  static __device__ __forceinline__ float at(const char* p) {
    return __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(p) << 16);
  }
};
template <> struct Load<TOPKV_FP16> {
  static constexpr int kBytes = 2;
  static __device__ __forceinline__ float at(const char* p) { return (float)*reinterpret_cast<const _Float16*>(p); }
};
template <> struct Load<TOPKV_FP8_E4M3> {
  static constexpr int kBytes = 1;
  static __device__ __forceinline__ float at(const char* p) {
    return __builtin_amdgcn_cvt_f32_fp8((int)*reinterpret_cast<const uint8_t*>(p), 0);
  }
};

}  // namespace topkv_attend

#endif  // TOPKV_ATTENTION_H_
