// attention.hip - attention of new tokens over a paged cache (declared in
// include/topkv.h): argument checks, and the general kernel that takes any
// geometry (odd head dims, rows off 16-byte alignment).
#include "attention.h"

#include <cmath>

#include "attention_internal.h"
#include "internal.h"

namespace topkv_attend {

constexpr int kWaves = 4;

template <int T>
__device__ __forceinline__ void store(void* p, int64_t i, float v) {
  if constexpr (T == TOPKV_BF16) {
    const __bf16 h = (__bf16)v;
    reinterpret_cast<__bf16*>(p)[i] = h;
  } else {
    reinterpret_cast<_Float16*>(p)[i] = (_Float16)v;
  }
}

// One wave per (token, query head): lanes over the head's elements, one key
// after the other with the running maximum and sum of the softmax.  Bound by
// the reduction over the wave and one key's latency, not by memory; it is
// what geometries run that the matrix-unit kernels do not take.
template <int QT, int KT, int NR>
__global__ __launch_bounds__(64 * kWaves) void kv_attention_general_kernel(Args a) {
  const int64_t row = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * kWaves + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (row >= (int64_t)a.total_q * a.num_heads) return;
  const int32_t token = (int32_t)(row / a.num_heads), head = (int32_t)(row - (int64_t)token * a.num_heads);
  int32_t r = token, pos;
  if (a.q_starts) {
    int32_t lo = 0, hi = a.num_reqs;                   // last request that starts at or before the token
    while (hi - lo > 1) {
      const int32_t mid = (lo + hi) >> 1;
      if (clamped_start(a, mid) <= token) lo = mid;
      else hi = mid;
    }
    r = lo;
    const int32_t end = clamped_start(a, r + 1);
    if (token < clamped_start(a, r) || token >= end) return;
    pos = clamped_len(a, r) - (end - token);
  } else {
    pos = clamped_len(a, r) - 1;
  }
  const int32_t* table = a.tables + (int64_t)r * a.bt_stride;
  const char* keys = a.cache + (int64_t)(head / a.group) * a.head_bytes;
  const char* qrow = static_cast<const char*>(a.q) + ((int64_t)token * a.q_stride + (int64_t)head * a.head_dim) * 2;
  float q[NR], acc[NR];
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    const int d = lane + 64 * i;
    q[i] = d < a.head_dim ? Load<QT>::at(qrow + 2 * d) : 0.f;
    acc[i] = 0.f;
  }
  float m = -INFINITY, l = 0.f;
  const Span span = key_span(a, pos, pos);
  for (int32_t i = 0; i < span.count; ++i) {
    const int64_t off = row_offset(a, table, key_position(span, i));
    if (off < 0) continue;
    const char* k = keys + off;
    float x = 0.f;
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const int d = lane + 64 * n;
      if (d < a.head_dim) x = fmaf(q[n], Load<KT>::at(k + d * Load<KT>::kBytes), x);
    }
#pragma unroll
    for (int s = 32; s; s >>= 1) x += __shfl_xor(x, s, 64);
    const float top = fmaxf(m, x * a.scale), safe = top == -INFINITY ? 0.f : top;
    const float keep = exp2f(m - safe), p = weight_of(x, a.scale, safe);
    m = top;
    l = l * keep + p;
    const char* v = k + a.value_bytes;
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const int d = lane + 64 * n;
      if (d < a.value_dim) acc[n] = fmaf(p, Load<KT>::at(v + d * Load<KT>::kBytes), acc[n] * keep);
    }
  }
  const float inv = l == 0.f ? 0.f : a.v_scale / l;
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    const int d = lane + 64 * n;
    if (d < a.value_dim) store<QT>(a.out, (int64_t)token * a.out_stride + (int64_t)head * a.value_dim + d, l == 0.f ? 0.f : acc[n] * inv);
  }
  if (a.lse && lane == 0) a.lse[(int64_t)token * a.num_heads + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

template <int QT, int KT>
void launch_general(const Args& a, hipStream_t stream) {
  const int64_t groups = ((int64_t)a.total_q * a.num_heads + kWaves - 1) / kWaves;
  const int64_t wide = groups < kMostGroups ? groups : kMostGroups;
  const dim3 grid((unsigned)wide, (unsigned)((groups + wide - 1) / wide));
  if (a.head_dim <= 256)
    hipLaunchKernelGGL(HIP_KERNEL_NAME(kv_attention_general_kernel<QT, KT, 4>), grid, dim3(64 * kWaves), 0, stream, a);
  else
    hipLaunchKernelGGL(HIP_KERNEL_NAME(kv_attention_general_kernel<QT, KT, 16>), grid, dim3(64 * kWaves), 0, stream, a);
}

topkv_status_t run_general(const Args& a, hipStream_t stream) {
  if (a.kv_dtype == TOPKV_FP8_E4M3) {
    if (a.dtype == TOPKV_BF16) launch_general<TOPKV_BF16, TOPKV_FP8_E4M3>(a, stream);
    else launch_general<TOPKV_FP16, TOPKV_FP8_E4M3>(a, stream);
  } else if (a.dtype == TOPKV_BF16) {
    launch_general<TOPKV_BF16, TOPKV_BF16>(a, stream);
  } else {
    launch_general<TOPKV_FP16, TOPKV_FP16>(a, stream);
  }
  return hipGetLastError() == hipSuccess ? TOPKV_OK : TOPKV_ERR_LAUNCH;
}

void divider(int32_t d, uint32_t* mul, uint32_t* shift) {
  int log2 = 0;
  while ((int64_t)1 << log2 < d) ++log2;
  *shift = 30 + log2;
  *mul = (uint32_t)((((uint64_t)1 << *shift) + d - 1) / d);
}

// Checks of the view and options, and the part of Args that follows from them.
topkv_status_t describe(const topkv_view_t* v, const topkv_attention_t* t, int32_t num_reqs, int32_t total_q, Args* a) {
  if (!v || !t) return TOPKV_ERR_INVALID_ARG;
  if (v->layout != TOPKV_LAYOUT_POOL && v->layout != TOPKV_LAYOUT_POOL_HEAD_MAJOR) return TOPKV_ERR_INVALID_ARG;
  const topkv_pool_t& p = v->pool;
  const topkv_status_t st = topkv_internal::pool_ok(&p);
  if (st != TOPKV_OK) return st;
  if (v->layer < 0 || v->layer >= p.num_layers || p.planes > 2 || v->bt_stride <= 0 || v->head_begin < 0 || v->reserved != 0)
    return TOPKV_ERR_INVALID_ARG;
  if ((t->dtype != TOPKV_BF16 && t->dtype != TOPKV_FP16) || (t->kv_dtype != t->dtype && t->kv_dtype != TOPKV_FP8_E4M3) ||
      p.elem_bytes != (t->kv_dtype == TOPKV_FP8_E4M3 ? 1 : 2))
    return TOPKV_ERR_INVALID_ARG;
  if (t->kv_heads <= 0 || t->kv_heads > p.num_heads - v->head_begin || t->num_heads <= 0 || t->num_heads % t->kv_heads != 0)
    return TOPKV_ERR_INVALID_ARG;
  if (t->value_dim <= 0 || (p.planes == 2 ? t->value_dim != p.head_dim : t->value_dim > p.head_dim)) return TOPKV_ERR_INVALID_ARG;
  if (t->window < 0 || t->sinks < 0 || t->reserved != 0 || t->reserved2 != 0.f) return TOPKV_ERR_INVALID_ARG;
  if (!std::isfinite(t->scale) || t->scale <= 0.f || !std::isfinite(t->k_scale) || t->k_scale <= 0.f ||
      !std::isfinite(t->v_scale))
    return TOPKV_ERR_INVALID_ARG;
  const float scale = t->scale * t->k_scale * kLog2e;
  if (!std::isfinite(scale) || scale <= 0.f) return TOPKV_ERR_INVALID_ARG;
  if (t->q_stride < (int64_t)t->num_heads * p.head_dim || t->out_stride < (int64_t)t->num_heads * t->value_dim)
    return TOPKV_ERR_INVALID_ARG;
  if (num_reqs < 0 || total_q < 0) return TOPKV_ERR_INVALID_ARG;
  if (p.head_dim > 1024 || num_reqs > TOPKV_MAX_BATCH_REQS || (int64_t)v->bt_stride * p.page_size >= (1 << 30) ||
      (int64_t)num_reqs * v->bt_stride * p.page_size > INT32_MAX || (int64_t)total_q * t->num_heads >= (1 << 30))
    return TOPKV_ERR_UNSUPPORTED;
  const int64_t elem = p.elem_bytes, plane = (int64_t)p.page_size * p.num_heads * p.head_dim * elem;
  const bool head_major = v->layout == TOPKV_LAYOUT_POOL_HEAD_MAJOR;
  a->slot_bytes = head_major ? p.head_dim * elem : (int64_t)p.num_heads * p.head_dim * elem;
  a->head_bytes = head_major ? (int64_t)p.page_size * p.head_dim * elem : p.head_dim * elem;
  a->page_bytes = plane * p.planes;
  a->value_bytes = p.planes == 2 ? plane : 0;
  a->cache = static_cast<const char*>(p.base) + (int64_t)v->layer * p.num_pages * a->page_bytes +
             (int64_t)v->head_begin * a->head_bytes;
  a->tables = v->block_tables;
  a->num_pages = p.num_pages;
  a->page_size = p.page_size;
  divider(p.page_size, &a->page_mul, &a->page_shift);
  divider(t->num_heads / t->kv_heads, &a->group_mul, &a->group_shift);
  a->bt_stride = v->bt_stride;
  a->num_reqs = num_reqs;
  a->total_q = total_q;
  a->num_heads = t->num_heads;
  a->kv_heads = t->kv_heads;
  a->group = t->num_heads / t->kv_heads;
  a->head_dim = p.head_dim;
  a->value_dim = t->value_dim;
  // A window as wide as the table hides nothing.  Narrower ones, and as many first tokens, leave every difference of a
  // position and either within 32 bits (a row may stand up to 2^30 before the request's first token).
  const int32_t cap = v->bt_stride * p.page_size;
  a->window = t->window < cap ? t->window : 0;
  a->sinks = a->window == 0 ? 0 : t->sinks < cap ? t->sinks : cap;
  a->scale = scale;
  a->v_scale = t->v_scale;
  a->dtype = t->dtype;
  a->kv_dtype = t->kv_dtype;
  a->q_stride = t->q_stride;
  a->out_stride = t->out_stride;
  return TOPKV_OK;
}

// Rows of q and the cache on 16-byte addresses (8 for an 8-bit cache).
bool aligned(const Args& a) {
  const uintptr_t unit = a.kv_dtype == TOPKV_FP8_E4M3 ? 8 : 16;
  return reinterpret_cast<uintptr_t>(a.cache) % unit == 0 && reinterpret_cast<uintptr_t>(a.q) % 16 == 0 &&
         a.q_stride % 8 == 0;
}

topkv_status_t attend(const topkv_view_t* cache, const topkv_attention_t* attn, int32_t num_reqs, const int32_t* seq_lens,
                      const int32_t* q_starts, bool decode, int32_t total_q, const void* q, void* out, float* lse,
                      void* workspace, int64_t workspace_bytes, hipStream_t stream) {
  Args a;
  const topkv_status_t st = describe(cache, attn, num_reqs, total_q, &a);
  if (st != TOPKV_OK) return st;
  const int64_t need = topkv_attention_workspace_bytes(cache, attn, num_reqs, total_q);
  if (workspace_bytes < need || (need > 0 && (!workspace || reinterpret_cast<uintptr_t>(workspace) % 16 != 0)))
    return TOPKV_ERR_INVALID_ARG;
  if (num_reqs == 0 || total_q == 0) return TOPKV_OK;
  if (!cache->block_tables || !seq_lens || !q || !out || (!decode && !q_starts)) return TOPKV_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(q) % 2 || reinterpret_cast<uintptr_t>(out) % 2 || reinterpret_cast<uintptr_t>(lse) % 4)
    return TOPKV_ERR_INVALID_ARG;
  a.seq_lens = seq_lens;
  a.q_starts = q_starts;
  a.q = q;
  a.out = out;
  a.lse = lse;
  a.out_wide = reinterpret_cast<uintptr_t>(out) % 16 == 0 && a.out_stride % 8 == 0;
  if (decode && decode_takes(a) && aligned(a)) return run_decode(a, workspace, stream);
  if (decode && latent_takes(a) && aligned(a)) return run_latent(a, workspace, stream);
  if (!decode && prompt_takes(a) && aligned(a)) return run_prompt(a, workspace, stream);
  return run_general(a, stream);
}

}  // namespace topkv_attend

extern "C" {

int64_t topkv_attention_workspace_bytes(const topkv_view_t* cache, const topkv_attention_t* attn, int32_t num_reqs,
                                        int32_t total_q) {
  topkv_attend::Args a;
  if (topkv_attend::describe(cache, attn, num_reqs, total_q, &a) != TOPKV_OK) return -1;
  const int64_t one = topkv_attend::decode_takes(a) ? topkv_attend::decode_workspace(a)
                      : topkv_attend::latent_takes(a) ? topkv_attend::latent_workspace(a)
                                                      : 0;
  const int64_t many = topkv_attend::prompt_workspace(a);
  return one > many ? one : many;
}

topkv_status_t topkv_attention_decode(const topkv_view_t* cache, const topkv_attention_t* attn, int32_t num_reqs,
                                      const int32_t* seq_lens, const void* q, void* out, float* lse, void* workspace,
                                      int64_t workspace_bytes, hipStream_t stream) {
  return topkv_attend::attend(cache, attn, num_reqs, seq_lens, nullptr, true, num_reqs, q, out, lse, workspace,
                                 workspace_bytes, stream);
}

topkv_status_t topkv_attention_prompt(const topkv_view_t* cache, const topkv_attention_t* attn, int32_t num_reqs,
                                      const int32_t* seq_lens, const int32_t* q_starts, int32_t total_q, const void* q,
                                      void* out, float* lse, void* workspace, int64_t workspace_bytes,
                                      hipStream_t stream) {
  return topkv_attend::attend(cache, attn, num_reqs, seq_lens, q_starts, false, total_q, q, out, lse, workspace,
                                 workspace_bytes, stream);
}

}  // extern "C"
