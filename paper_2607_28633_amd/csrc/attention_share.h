// attention_share.h - decode's division of a batch into equal shares, and the
// join of requests that were cut (attention_decode.hip, attention_latent.hip).
#ifndef TOPKV_ATTENTION_SHARE_H_
#define TOPKV_ATTENTION_SHARE_H_

#include "attention_mfma.h"

namespace topkv_attend {
namespace {

constexpr int kTile = 32;                // keys of a tile
constexpr int kLeast = 8;                // tiles of a share, at least: smaller pieces cost more to join than they save
constexpr int kSingle = 512;             // longest visible length that is never cut (one launch, no join)

constexpr int kMostShares = 512;

struct Plan {
  int32_t shares;      // wanted; 0: one per request, whatever its length
  float* part;         // [2 * share + 1 for a request's first piece][kv head][row of the group][value_dim]
  float2v* part_ml;    // the same without value_dim: maximum and sum
  bool by_request;     // what `cut` is indexed by: requests, or shares where these are fewer
  int4* cut;           // the request in pieces (of that number, or that starts in that share), its first share, how many (0: none)
};

struct Share {
  int32_t request;     // of the first tile; -1: the share is empty
  int32_t base;        // number of that request's first tile
  int32_t size;        // tiles of a share
  int32_t total;       // tiles of the batch
};

// Every request has at least one tile, so that those of no tokens are written too.
__device__ __forceinline__ int32_t tiles_of(const Args& a, int32_t r) {
  const int32_t p = clamped_len(a, r) - 1, n = key_span(a, p, p).count;
  return n < 1 ? 1 : (n + kTile - 1) / kTile;
}

template <int kWaves>
__device__ Share find_share(const Args& a, int32_t shares, int32_t share) {
  __shared__ Share s_got;
  if (threadIdx.x == 0) s_got.request = -1;
  const auto tiles = [&](int32_t r) { return tiles_of(a, r); };
  Scan<int32_t> n = scan_requests<int32_t, kWaves>(a.num_reqs, tiles);
  int32_t size = (n.total + shares - 1) / shares;
  size = size < kLeast ? kLeast : size;
  const int32_t first = share * size;
  if (n.holds(first)) {
    s_got.request = n.find(first, tiles);
    s_got.base = n.base;
  }
  __syncthreads();
  Share got = s_got;
  got.size = size;
  got.total = n.total;
  return got;
}

// Requests in pieces: one workgroup per (request or share, query head, 64 elements).
// The pieces' weights first, then their sum with the pieces over the waves and
// the elements over the lanes, so that no load waits for another.
constexpr int kJoinWaves = 8;

template <int T>
__global__ __launch_bounds__(64 * kJoinWaves) void kv_attention_join_kernel(Args a, Plan plan) {
  __shared__ float s_weight[kMostShares], s_sum[kJoinWaves], s_part[kJoinWaves][64];
  const int32_t entry = blockIdx.x / a.num_heads, head = blockIdx.x - entry * a.num_heads;
  const int4 cut = plan.cut[entry];
  const int32_t r = cut.x, share = cut.y, pieces = cut.z;
  if (pieces == 0) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t step = (int64_t)a.kv_heads * a.group;
  const int64_t at = 2 * (int64_t)share * step + head;            // piece k: slot 2 (first + k), the first one's next to it
  const int32_t d = blockIdx.y * 64 + lane;
  float top = -INFINITY;                                         // every wave over all chunks
  for (int32_t k = lane; k < pieces; k += 64) top = fmaxf(top, plan.part_ml[at + (k ? 2 * k : 1) * step][0]);
#pragma unroll
  for (int i = 32; i; i >>= 1) top = fmaxf(top, __shfl_xor(top, i, 64));
  const float base = top == -INFINITY ? 0.f : top;
  float sum = 0.f;
  for (int32_t k = threadIdx.x; k < pieces; k += 64 * kJoinWaves) {
    const float2v ml = plan.part_ml[at + (k ? 2 * k : 1) * step];
    const float f = __builtin_amdgcn_exp2f(ml[0] - base);
    s_weight[k] = f;
    sum += f * ml[1];
  }
#pragma unroll
  for (int i = 32; i; i >>= 1) sum += __shfl_xor(sum, i, 64);
  if (lane == 0) s_sum[wave] = sum;
  __syncthreads();
  float o = 0.f;
  if (d < a.value_dim) {
    const float* from = plan.part + at * a.value_dim + d;
    const int64_t row = step * a.value_dim;
#pragma unroll 8
    for (int32_t k = wave; k < pieces; k += kJoinWaves) o = fmaf(s_weight[k], from[(k ? 2 * k : 1) * row], o);
  }
  s_part[wave][lane] = o;
  __syncthreads();
  if (wave > 0) return;
  sum = 0.f;
  o = 0.f;
  for (int w = 0; w < kJoinWaves; ++w) {
    sum += s_sum[w];
    o += s_part[w][lane];
  }
  if (d < a.value_dim)
    static_cast<typename Elem<T>::type*>(a.out)[(int64_t)r * a.out_stride + (int64_t)head * a.value_dim + d] =
        (typename Elem<T>::type)(sum == 0.f ? 0.f : o * (a.v_scale / sum));
  if (a.lse && d == 0)
    a.lse[(int64_t)r * a.num_heads + head] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

int64_t up16(int64_t x) { return (x + 15) / 16 * 16; }

// Shares that a call wants, 0 where no request can be long enough to be cut.
int32_t shares_for(const Args& a, int32_t resident, int32_t units) {
  const int64_t seen = (int64_t)a.bt_stride * a.page_size;
  const int64_t most = a.window > 0 && (int64_t)a.window + a.sinks < seen ? (int64_t)a.window + a.sinks : seen;
  if (most <= kSingle) return 0;
  const int32_t n = resident / units;
  return n < 1 ? 1 : n;
}

int64_t plan_bytes(const Args& a, int32_t shares) {
  if (shares == 0) return 0;
  const int64_t rows = 2 * (int64_t)shares * a.num_heads;
  return up16(rows * a.value_dim * 4) + up16(rows * 8) + (int64_t)shares * 16;
}

Plan make_plan(const Args& a, int32_t shares, void* workspace) {
  Plan p = {};
  p.shares = shares;
  if (shares > 0) {
    const int64_t rows = 2 * (int64_t)shares * a.num_heads;
    char* at = static_cast<char*>(workspace);
    p.part = reinterpret_cast<float*>(at);
    at += up16(rows * a.value_dim * 4);
    p.part_ml = reinterpret_cast<float2v*>(at);
    at += up16(rows * 8);
    p.cut = reinterpret_cast<int4*>(at);
    p.by_request = a.num_reqs <= shares;
  }
  return p;
}

void launch_join(const Args& a, const Plan& p, hipStream_t stream) {
  if (p.shares == 0) return;
  const dim3 grid((unsigned)((p.by_request ? a.num_reqs : p.shares) * a.num_heads), (unsigned)((a.value_dim + 63) / 64));
  if (a.dtype == TOPKV_BF16)
    hipLaunchKernelGGL(kv_attention_join_kernel<TOPKV_BF16>, grid, dim3(64 * kJoinWaves), 0, stream, a, p);
  else
    hipLaunchKernelGGL(kv_attention_join_kernel<TOPKV_FP16>, grid, dim3(64 * kJoinWaves), 0, stream, a, p);
}

// Rows on addresses that the wide loads take.
bool rows_aligned(const Args& a) {
  const int64_t unit = a.kv_dtype == TOPKV_FP8_E4M3 ? 8 : 16;
  return a.head_dim % 8 == 0 && a.slot_bytes % unit == 0 && a.head_bytes % unit == 0 && a.page_bytes % unit == 0 &&
         a.value_bytes % unit == 0;
}

}  // namespace
}  // namespace topkv_attend

#endif  // TOPKV_ATTENTION_SHARE_H_
