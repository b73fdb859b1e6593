// attention_decode.hip - one new token per request on the matrix units.
//
// A request's group of query heads (up to 16 rows) reads each key and value
// once: 2 * group flops per cache element, so the kernel is bound by the
// cache's bytes.  A wave keeps the rows in registers and walks tiles of 32
// keys: the next tile is on its way to registers while the present one, in
// the wave's own piece of LDS, is multiplied; no barrier is needed on the way.
// The four waves of a workgroup take tiles in turn and join at the end.
//
// Few requests would leave most of the GPU idle, uneven ones would wait for
// the longest: the tiles of the whole batch, request after request, are cut
// into shares of one size, one for each workgroup that fits the GPU at once.
// A share may hold the end of one request, some whole ones and the start of
// another; requests cut into pieces are joined by a second kernel from partial
// results in 32 bits.  The cut follows the lengths on the device, not the
// width of the tables.
#include "attention_internal.h"
#include "attention_share.h"

namespace topkv_attend {

namespace {

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kRows = 16;                // query rows of a workgroup
constexpr int kStep = kTile * kWaves;    // keys of the waves' tiles together

// Shares, by the key width: as many workgroups as 256 CUs hold at once by their LDS (64 KiB at 128 elements, 128 KiB
// at 256).  131072 tokens, 8 heads of 128: 512 shares 97 us, 768 102, 1024 103; 262144 tokens, heads of 64, of which four
// workgroups fit a CU, 512 107 us, 768 112, 1024 105.
constexpr int resident(int KD) { return KD <= 128 ? 512 : 256; }

// KD, VD: key and value elements of a row, padded; kLatent: the value is the
// key row's front.  T: the inputs' type; kF8: the cache holds e4m3.
// kCut: the batch is cut into shares; otherwise a workgroup takes one request.
template <int T, bool kF8, int KD, int VD, bool kLatent, bool kCut>
__global__ __launch_bounds__(kThreads, resident(KD) / 256) void kv_attention_decode_kernel(Args a, Plan plan) {
  typedef typename Elem<T>::vec8 vec8;
  constexpr int NCK = KD / 8, NCV = VD / 8;                      // 16-byte chunks of a row in LDS
  constexpr int LK = kTile * NCK / 64, LV = kLatent ? 0 : kTile * NCV / 64;   // loads of a lane for a tile
  constexpr int kKeyBytes = kTile * KD * 2, kTileBytes = kKeyBytes + (kLatent ? 0 : kTile * VD * 2);
  constexpr int kPad = VD + 4;                                   // floats of a row in the final exchange
  constexpr int kWaveBytes = ((kTileBytes > kRows * kPad * 4 ? kTileBytes : kRows * kPad * 4) + 1023) / 1024 * 1024;
  __shared__ __attribute__((aligned(16))) char s_tile[kWaves * kWaveBytes];
  __shared__ float s_m[kWaves][kRows], s_l[kWaves][kRows];

  const int wave = threadIdx.x >> 6;
  const int32_t groups = (a.group + kRows - 1) / kRows;
  // Eight items side by side over the eight XCDs, an item's KV heads one after the other on one XCD: with the
  // heads side by side each XCD would read a narrow column of the cache through a few channels of its L2.
  const int32_t units = a.kv_heads * groups, eight = blockIdx.x / (8 * units), within = blockIdx.x - eight * 8 * units;
  const int32_t share = eight * 8 + (within & 7), sub = within >> 3;
  const int32_t kv_head = sub % a.kv_heads, first_row = sub / a.kv_heads * kRows;
  char* tile = s_tile + wave * kWaveBytes;
  const char* cache = a.cache + (int64_t)kv_head * a.head_bytes;
  const int32_t key_chunks = a.head_dim / 8;                     // of 8 elements
  const int32_t value_chunks = kLatent ? 0 : a.value_dim / 8;
  constexpr int kChunkBytes = kF8 ? 8 : 16;
  typedef typename std::conditional<kF8, uint2v, uint4v>::type Raw;

  Share sh = {share, 0, 0, 0};
  int32_t tile_at = 0, tile_end = 1;                             // tiles of the batch; uncut: the request as one
  if constexpr (kCut) {
    if (share >= plan.shares) return;
    sh = find_share<kWaves>(a, plan.shares, share);
    if (!plan.by_request && sub == 0 && threadIdx.x == 0) plan.cut[share] = make_int4(0, 0, 0, 0);
    if (sh.request < 0) return;
    tile_at = share * sh.size;
    tile_end = tile_at + sh.size < sh.total ? tile_at + sh.size : sh.total;
  } else {
    if (share >= a.num_reqs) return;
  }

  for (int32_t request = sh.request; tile_at < tile_end; ++request) {
  int lane = threadIdx.x & 63;
  if constexpr (kCut) asm volatile("" : "+v"(lane));             // addresses made from it stay in the loop: registers
  const int row = lane & 15, quad = lane >> 4;
  const int32_t pos = clamped_len(a, request) - 1;
  const Span span = key_span(a, pos, pos);
  int32_t begin = 0, end = span.count;
  bool whole = true, opens = false;
  if constexpr (kCut) {
    const int32_t tiles = span.count < 1 ? 1 : (span.count + kTile - 1) / kTile, from = tile_at - sh.base;
    const int32_t to = tile_end - sh.base < tiles ? tile_end - sh.base : tiles;
    opens = from == 0;
    whole = opens && to == tiles;
    begin = from * kTile;
    end = to * kTile < span.count ? to * kTile : span.count;
    if (opens && (!whole || plan.by_request) && sub == 0 && threadIdx.x == 0)
      plan.cut[plan.by_request ? request : share] =
          make_int4(request, share, whole ? 0 : (sh.base + tiles - 1) / sh.size - share + 1, 0);
    tile_at = sh.base + to;
    sh.base += tiles;
  } else {
    tile_at = tile_end;
  }

  // the query rows: lane (row, quad) holds elements quad * 8 .. + 7 of every 32
  vec8 q[KD / 32];
  {
    const int32_t h = first_row + row;
    const char* at = static_cast<const char*>(a.q) +
                     ((int64_t)request * a.q_stride + (int64_t)(kv_head * a.group + h) * a.head_dim) * 2;
#pragma unroll
    for (int s = 0; s < KD / 32; ++s) {
      const int d = s * 32 + quad * 8;
      union {
        uint4v w;
        vec8 v;
      } u;
      u.w = uint4v{0, 0, 0, 0};
      if (h < a.group && d < a.head_dim) u.w = *reinterpret_cast<const uint4v*>(at + 2 * d);
      q[s] = u.v;
    }
  }

  const int32_t* table = a.tables + (int64_t)request * a.bt_stride;
  if (key_chunks < NCK) {                                        // padding stays zero: loads leave it alone
#pragma unroll
    for (int i = 0; i < kWaveBytes / 1024; ++i)
      *reinterpret_cast<uint4v*>(tile + (i * 64 + lane) * 16) = uint4v{0, 0, 0, 0};
  }

  float4v acc[VD / 16];
#pragma unroll
  for (int t = 0; t < VD / 16; ++t) acc[t] = float4v{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;

  // The table entry of key (tile i's first + lane % 32) is asked for two tiles ahead and before the rows of the
  // next tile, so that its wait, a tile later, waits for nothing younger.
  auto ask = [&](int32_t first) -> int32_t {
    const int32_t v = first + (lane & 31);
    return v < end ? table[page_of(a, (uint32_t)key_position(span, v))] : -1;
  };
  auto locate = [&](int32_t first, int32_t entry) -> int64_t {
    const int32_t v = first + (lane & 31);
    if (v >= end || entry < 0 || entry >= a.num_pages) return -1;
    const uint32_t j = (uint32_t)key_position(span, v);
    return (int64_t)entry * a.page_bytes + (int64_t)(j - page_of(a, j) * (uint32_t)a.page_size) * a.slot_bytes;
  };
  // A long cache is read once and is better not kept in the L2 (131072 tokens, 8 heads of 128: 97 us, 108 without the
  // hint); short ones may still lie there.
  const auto load_row = [&](const char* from) -> Raw {
    if constexpr (kCut) return __builtin_nontemporal_load(reinterpret_cast<const Raw*>(from));
    else return *reinterpret_cast<const Raw*>(from);
  };
  Raw rk[LK], rv[LV > 0 ? LV : 1];
  auto fetch = [&](int64_t off) {
    const uint32_t safe_lo = off < 0 ? 0u : (uint32_t)off, safe_hi = off < 0 ? 0u : (uint32_t)(off >> 32);
#pragma unroll
    for (int i = 0; i < LK; ++i) {
      const int place = i * 64 + lane, r = place / NCK, c = (place - r * NCK) ^ swizzle<NCK>(r);
      const char* from = cache + ((int64_t)((uint64_t)(uint32_t)__shfl((int)safe_hi, r, 64) << 32 | (uint32_t)__shfl((int)safe_lo, r, 64)));
      if (c < key_chunks) rk[i] = load_row(from + c * kChunkBytes);
    }
#pragma unroll
    for (int i = 0; i < LV; ++i) {
      const int place = i * 64 + lane, r = place / NCV, c = (place - r * NCV) ^ swizzle<NCV>(r);
      const char* from = cache + a.value_bytes + ((int64_t)((uint64_t)(uint32_t)__shfl((int)safe_hi, r, 64) << 32 | (uint32_t)__shfl((int)safe_lo, r, 64)));
      if (c < value_chunks) rv[i] = load_row(from + c * kChunkBytes);
    }
  };
  // registers to LDS; rows without a key as zeros, whatever their place holds
  auto put = [&](uint32_t there) {
#pragma unroll
    for (int i = 0; i < LK; ++i) {
      const int place = i * 64 + lane, r = place / NCK, c = (place - r * NCK) ^ swizzle<NCK>(r);
      uint4v w;
      if constexpr (kF8) w = widen<T>(rk[i]);
      else w = rk[i];
      if (!(there >> r & 1)) w = uint4v{0, 0, 0, 0};
      if (c < key_chunks) *reinterpret_cast<uint4v*>(tile + place * 16) = w;
    }
#pragma unroll
    for (int i = 0; i < LV; ++i) {
      const int place = i * 64 + lane, r = place / NCV, c = (place - r * NCV) ^ swizzle<NCV>(r);
      uint4v w;
      if constexpr (kF8) w = widen<T>(rv[i]);
      else w = rv[i];
      if (!(there >> r & 1)) w = uint4v{0, 0, 0, 0};
      if (c < value_chunks) *reinterpret_cast<uint4v*>(tile + kKeyBytes + place * 16) = w;
    }
  };

  int32_t first = begin + wave * kTile;
  if (first < end) {
    int64_t off = locate(first, ask(first));
    int32_t entry = ask(first + kStep);
    fetch(off);
    for (; first < end; first += kStep) {
      const uint32_t there = (uint32_t)__ballot(off >= 0);       // bit k: key k of the tile is one
      put(there);
      wave_fence();
      off = locate(first + kStep, entry);
      if (first + kStep < end) {
        entry = ask(first + 2 * kStep);
        fetch(off);
      }
      // scores of 2 x 16 keys: lane (row, quad) gets keys 4 quad .. + 3 of each half
      float4v x[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        x[b] = float4v{0.f, 0.f, 0.f, 0.f};
        const int r = b * 16 + row;
#pragma unroll
        for (int s = 0; s < KD / 32; ++s) {
          const vec8 k = *reinterpret_cast<const vec8*>(tile + (r * NCK + ((s * 4 + quad) ^ swizzle<NCK>(r))) * 16);
          x[b] = Elem<T>::mfma16(k, q[s], x[b]);
        }
      }
      if (there != 0xffffffffu) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (!(there >> (b * 16 + quad * 4 + i) & 1)) x[b][i] = -INFINITY;
      }
      float top = fmaxf(fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[0][2], x[0][3])),
                        fmaxf(fmaxf(x[1][0], x[1][1]), fmaxf(x[1][2], x[1][3])));
      top = reference<T>(max_quarters(top), a.scale, 0.f);
      if (__any(top > m)) {                                      // some row's maximum rises
        const float up = fmaxf(m, top), fall = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - up);
        m = up;
        l *= fall;
#pragma unroll
        for (int t = 0; t < VD / 16; ++t) acc[t] *= fall;
      }
      const float base = m == -INFINITY ? 0.f : m;
      vec8 p;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float w = weight_of(x[b][i], a.scale, base);
          l += w;
          p[b * 4 + i] = (typename Elem<T>::type)w;              // rounded for the matrix units, its sum is not
        }
      // values by columns: lane (d, quad) takes keys 4 quad .. + 3 of each half, as the weights lie
      const char* values = tile + (kLatent ? 0 : kKeyBytes);
#pragma unroll
      for (int t = 0; t < VD / 16; ++t) {
        union {
          uint2v h[2];
          vec8 v;
        } u;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const int r = b * 16 + quad * 4 + (row >> 2), c = t * 2 + (row >> 1 & 1);
          constexpr int NC = kLatent ? NCK : NCV;
          u.h[b] = read_transposed(values + (r * NC + (c ^ swizzle<NC>(r))) * 16 + (row & 1) * 8);
        }
        acc[t] = Elem<T>::mfma16(u.v, p, acc[t]);
      }
      wave_fence();
    }
  }

  // the four waves' parts join in LDS
  l = sum_quarters(l);
  wave_fence();
  float* mine = reinterpret_cast<float*>(tile);
#pragma unroll
  for (int t = 0; t < VD / 16; ++t) *reinterpret_cast<float4v*>(mine + row * kPad + t * 16 + quad * 4) = acc[t];
  if (quad == 0) {
    s_m[wave][row] = m;
    s_l[wave][row] = l;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < kRows * (VD / 4); i += kThreads) {
    const int r = i / (VD / 4), d = (i - r * (VD / 4)) * 4;
    if (first_row + r >= a.group || d >= a.value_dim) continue;
    float top = s_m[0][r];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) top = fmaxf(top, s_m[w][r]);
    const float base = top == -INFINITY ? 0.f : top;
    float sum = 0.f;
    float4v o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(s_m[w][r] - base);
      if (s_m[w][r] == -INFINITY && s_l[w][r] == 0.f) continue;  // no key, or none that counts (a sum of NaN does)
      sum += f * s_l[w][r];
      o += *reinterpret_cast<const float4v*>(s_tile + w * kWaveBytes + (r * kPad + d) * 4) * f;
    }
    const int32_t head = kv_head * a.group + first_row + r;
    if (!whole) {
      const int64_t slot = (2 * (int64_t)share + opens) * a.num_heads + head;
      *reinterpret_cast<float4v*>(plan.part + slot * plan.part_dim + d) = o;
      if (d == 0) plan.part_ml[slot] = float2v{top, sum};
    } else {
      const float inv = sum == 0.f ? 0.f : a.v_scale / sum;
      typename Elem<T>::type* out =
          static_cast<typename Elem<T>::type*>(a.out) + (int64_t)request * a.out_stride + (int64_t)head * a.value_dim + d;
      for (int e = 0; e < 4; ++e)
        if (d + e < a.value_dim) out[e] = (typename Elem<T>::type)(sum == 0.f ? 0.f : o[e] * inv);
      if (a.lse && d == 0)
        a.lse[(int64_t)request * a.num_heads + head] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
    }
  }
  __syncthreads();                                               // the tiles' place is free again
  }
}

int32_t units(const Args& a) { return a.kv_heads * ((a.group + kRows - 1) / kRows); }

int32_t wanted_shares(const Args& a) { return shares_for(a, resident(a.head_dim), units(a)); }

template <int T, bool kF8>
void launch(const Args& a, const Plan& p, hipStream_t stream) {
  const int64_t items = p.shares > 0 ? p.shares : a.num_reqs;
  const dim3 grid((unsigned)((items + 7) / 8 * 8 * units(a))), block(kThreads);
  const bool latent = a.value_bytes == 0;
#define TOPKV_DECODE(KD, VD, LATENT)                                                                                         \
  do {                                                                                                                       \
    if (p.shares > 0)                                                                                                        \
      hipLaunchKernelGGL(HIP_KERNEL_NAME(kv_attention_decode_kernel<T, kF8, KD, VD, LATENT, true>), grid, block, 0, stream, a, p);  \
    else                                                                                                                     \
      hipLaunchKernelGGL(HIP_KERNEL_NAME(kv_attention_decode_kernel<T, kF8, KD, VD, LATENT, false>), grid, block, 0, stream, a, p); \
  } while (0)
  if (latent) TOPKV_DECODE(128, 128, true);
  else if (a.head_dim <= 64) TOPKV_DECODE(64, 64, false);
  else if (a.head_dim <= 128) TOPKV_DECODE(128, 128, false);
  else TOPKV_DECODE(256, 256, false);
#undef TOPKV_DECODE
  launch_join(a, p, stream);
}

}  // namespace

bool decode_takes(const Args& a) {
  const bool latent = a.value_bytes == 0;
  return rows_aligned(a) && a.head_dim <= (latent ? 128 : 256) && launchable(a, wanted_shares(a), units(a));
}

int64_t decode_workspace(const Args& a) { return plan_bytes(a, wanted_shares(a)); }

topkv_status_t run_decode(const Args& a, void* workspace, hipStream_t stream) {
  const Plan p = make_plan(a, wanted_shares(a), workspace);
  if (a.kv_dtype == TOPKV_FP8_E4M3) {
    if (a.dtype == TOPKV_BF16) launch<TOPKV_BF16, true>(a, p, stream);
    else launch<TOPKV_FP16, true>(a, p, stream);
  } else if (a.dtype == TOPKV_BF16) {
    launch<TOPKV_BF16, false>(a, p, stream);
  } else {
    launch<TOPKV_FP16, false>(a, p, stream);
  }
  return hipGetLastError() == hipSuccess ? TOPKV_OK : TOPKV_ERR_LAUNCH;
}

}  // namespace topkv_attend
