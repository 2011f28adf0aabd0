// Eviction from the cache by accumulated attention weight (part of kv_scatter.hip).
//
// evict_select: for every (request, KV head), which `keep` of L positions stay: the first n_first,
// the last n_recent, and of the others those of the greatest weight, the lower position first
// among equals.  One work-group finds the weight of the last one to stay by its bits, eight at a
// time from the top (a histogram of each eight in LDS), then writes the kept positions in order.
// kv_compact: the kept tokens' K and V into other blocks, position i of the result from position
// kept[i]; a head's tokens move on their own, so the same slot may hold another token for another
// head.  A work-group writes one block of one head.
#pragma once

#include "mx4.hpp"

namespace {

constexpr int kSelThreads = 1024;

// weights as integers of the same order: NaN lowest, -0 as 0
__device__ __forceinline__ uint32_t weight_key(float w) {
  const uint32_t b = __builtin_bit_cast(uint32_t, w + 0.f);
  if (w != w) return 0;
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__global__ __launch_bounds__(kSelThreads) void evict_select_kernel(
    const float* __restrict__ weights, int64_t w_stride, const int32_t* __restrict__ seq_lens, int hkv, int keep,
    int n_first, int n_recent, int32_t* __restrict__ kept, float* __restrict__ kept_weights, int64_t kw_stride) {
  __shared__ int hist[256];
  __shared__ int wave_take[kSelThreads / 64], wave_equal[kSelThreads / 64];
  __shared__ int pick, above;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, h = blockIdx.x, r = blockIdx.y;
  const int64_t seg = static_cast<int64_t>(r) * hkv + h;
  const float* w = weights + seg * w_stride;
  int32_t* out = kept + seg * keep;
  float* kw = kept_weights == nullptr ? nullptr : kept_weights + seg * kw_stride;
  const int len = static_cast<int>(min(static_cast<int64_t>(max(seq_lens[r], 0)), w_stride));
  const int n_kept = min(keep, len);
  const int lo = len <= keep ? 0 : n_first, hi = len <= keep ? 0 : len - n_recent;   // positions that compete
  int need = len <= keep ? 0 : keep - n_first - n_recent;                            // how many of them stay

  // the key of the last one to stay, and how many with that very key
  uint32_t prefix = 0;
  if (need > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      for (int i = lo + tid; i < hi; i += kSelThreads) {
        const uint32_t k = weight_key(w[i]);
        if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255u], 1);
      }
      __syncthreads();
      if (wave == 0) {       // the highest digit with at least `need` keys from it up
        int c[4], sum = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) { c[i] = hist[255 - (4 * lane + i)]; sum += c[i]; }
        int upto = sum;
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) {
          const int x = __shfl_up(upto, s);
          if (lane >= s) upto += x;
        }
        int before = upto - sum;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (before < need && before + c[i] >= need) { pick = 255 - (4 * lane + i); above = before; }
          before += c[i];
        }
      }
      __syncthreads();
      prefix |= static_cast<uint32_t>(pick) << shift;
      need -= above;
      __syncthreads();
    }
  } else {
    prefix = 0xffffffffu;    // no key is greater
  }

  // positions in order: greater keys, and the first `need` equal ones
  int at = 0, equal = 0;
  for (int i0 = 0; i0 < len; i0 += kSelThreads) {
    const int i = i0 + tid;
    const float x = i < len ? w[i] : 0.f;
    const bool held = i < len && (i < lo || i >= hi);
    const uint32_t k = weight_key(x);
    const bool eq = i < len && !held && need > 0 && k == prefix;
    const uint64_t eqs = __builtin_amdgcn_ballot_w64(eq);
    if (lane == 0) wave_equal[wave] = __builtin_popcountll(eqs);
    __syncthreads();
    int rank = equal + __builtin_popcountll(eqs & ((1ull << lane) - 1)), all = equal;
    for (int v = 0; v < kSelThreads / 64; ++v) {
      if (v < wave) rank += wave_equal[v];
      all += wave_equal[v];
    }
    const bool take = held || (i < len && !held && k > prefix) || (eq && rank < need);
    const uint64_t takes = __builtin_amdgcn_ballot_w64(take);
    if (lane == 0) wave_take[wave] = __builtin_popcountll(takes);
    __syncthreads();
    int dst = at + __builtin_popcountll(takes & ((1ull << lane) - 1)), next = at;
    for (int v = 0; v < kSelThreads / 64; ++v) {
      if (v < wave) dst += wave_take[v];
      next += wave_take[v];
    }
    if (take) {
      out[dst] = i;
      if (kw != nullptr) kw[dst] = x;
    }
    at = next;
    equal = all;
  }
  for (int i = n_kept + tid; i < keep; i += kSelThreads) {
    out[i] = -1;
    if (kw != nullptr) kw[i] = 0.f;
  }
}

// Where the 16 tokens of a destination block come from: slot of each, -1 for none.
__device__ __forceinline__ void source_slots(int32_t* src, const int32_t* kept, int keep, const int32_t* bt,
                                             int bt_stride, int64_t num_blocks, int b) {
  const int i = 16 * b + threadIdx.x;
  if (threadIdx.x < 16) {
    int32_t s = -1;
    const int32_t p = i < keep ? kept[i] : -1;
    if (p >= 0 && (p >> 4) < bt_stride) {
      const int32_t ph = bt[p >> 4];
      const bool ok = ph >= 0 && ph < num_blocks;
      ARCKV_CHECK_LANE(!ok, ARCKV_CHECK_BLOCK);
      s = ok ? ph * 16 + (p & 15) : -1;
    }
    src[threadIdx.x] = s;
  }
  __syncthreads();
}

template <int D>
__global__ __launch_bounds__(256) void kv_compact_kernel(
    uint16_t* __restrict__ k_pool, uint16_t* __restrict__ v_pool, const int32_t* __restrict__ block_tables,
    int bt_stride, const int32_t* __restrict__ kept, int keep, const int32_t* __restrict__ dst_tables, int dst_stride,
    int64_t num_blocks, int hkv) {
  __shared__ int32_t src[16];
  const int b = blockIdx.x / hkv, h = blockIdx.x % hkv, r = blockIdx.y, tid = threadIdx.x;
  source_slots(src, kept + (static_cast<int64_t>(r) * hkv + h) * keep, keep,
               block_tables + static_cast<int64_t>(r) * bt_stride, bt_stride, num_blocks, b);
  const int32_t db = dst_tables[static_cast<int64_t>(r) * dst_stride + b];
  const bool bad = db < 0 || db >= num_blocks;
  ARCKV_CHECK_WAVE(bad && src[0] >= 0 && tid < 64, ARCKV_CHECK_BLOCK);
  if (bad) return;
  const int64_t dst = (static_cast<int64_t>(db) * hkv + h) * 16 * D;
  constexpr int CH = D / 8;
  if (tid < 16 * CH) {
    const int t = tid / CH, c = tid % CH;
    const int32_t s = src[t];
    if (s >= 0)
      *reinterpret_cast<uint4*>(k_pool + dst + t * D + c * 8) =
          *reinterpret_cast<const uint4*>(k_pool + ((static_cast<int64_t>(s >> 4) * hkv + h) * 16 + (s & 15)) * D + c * 8);
  }
  if (tid < 2 * D) {
    const int d = tid >> 1, half = tid & 1;
    uint32_t x[8];
    bool all = true;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int32_t s = src[8 * half + j];
      all &= s >= 0;
      x[j] = s < 0 ? 0 : v_pool[((static_cast<int64_t>(s >> 4) * hkv + h) * D + d) * 16 + (s & 15)];
    }
    uint16_t* to = v_pool + dst + d * 16 + 8 * half;
    if (all) {
      *reinterpret_cast<uint4*>(to) = uint4{x[0] | x[1] << 16, x[2] | x[3] << 16, x[4] | x[5] << 16, x[6] | x[7] << 16};
    } else {                 // slots without a token keep what they hold
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (src[8 * half + j] >= 0) to[j] = static_cast<uint16_t>(x[j]);
    }
  }
}

template <int D>
__global__ __launch_bounds__(256) void kv_compact_mx4_kernel(
    uint8_t* __restrict__ pool, const int32_t* __restrict__ block_tables, int bt_stride,
    const int32_t* __restrict__ kept, int keep, const int32_t* __restrict__ dst_tables, int dst_stride,
    int64_t num_blocks, int hkv) {
  using L = mx4::Layout<D>;
  __shared__ int32_t src[16];
  const int b = blockIdx.x / hkv, h = blockIdx.x % hkv, r = blockIdx.y, tid = threadIdx.x;
  source_slots(src, kept + (static_cast<int64_t>(r) * hkv + h) * keep, keep,
               block_tables + static_cast<int64_t>(r) * bt_stride, bt_stride, num_blocks, b);
  const int32_t db = dst_tables[static_cast<int64_t>(r) * dst_stride + b];
  const bool bad = db < 0 || db >= num_blocks;
  ARCKV_CHECK_WAVE(bad && src[0] >= 0 && tid < 64, ARCKV_CHECK_BLOCK);
  if (bad) return;
  uint8_t* to = pool + (static_cast<int64_t>(db) * hkv + h) * L::kBytes;
  auto from = [&](int t) { return pool + (static_cast<int64_t>(src[t] >> 4) * hkv + h) * L::kBytes; };
  constexpr int WORDS = D / 8;
  if (tid < 16 * WORDS) {
    const int t = tid / WORDS, c = tid % WORDS;
    if (src[t] >= 0)
      *reinterpret_cast<uint32_t*>(to + t * L::kRow + 4 * c) =
          *reinterpret_cast<const uint32_t*>(from(t) + (src[t] & 15) * L::kRow + 4 * c);
  }
  if (tid < 16 * L::kGroups) {
    const int t = tid & 15, g = tid >> 4;
    if (src[t] >= 0) {
      to[L::kKScale + t * L::kGroups + g] = from(t)[L::kKScale + (src[t] & 15) * L::kGroups + g];
      to[L::kVScale + g * 16 + t] = from(t)[L::kVScale + g * 16 + (src[t] & 15)];
    }
  }
  if (tid < D) {
    const int half = tid / (D / 2), p = tid % (D / 2);
    uint32_t x[8];
    bool all = true;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int t = 8 * half + j, s = src[t];
      all &= s >= 0;
      x[j] = s < 0 ? 0 : from(t)[L::kV + ((s & 15) >> 3) * L::kHalf + 8 * p + (s & 7)];
    }
    uint8_t* at = to + L::kV + half * L::kHalf + 8 * p;
    if (all) {
      *reinterpret_cast<uint2*>(at) = uint2{x[0] | x[1] << 8 | x[2] << 16 | x[3] << 24, x[4] | x[5] << 8 | x[6] << 16 | x[7] << 24};
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (src[8 * half + j] >= 0) at[j] = static_cast<uint8_t>(x[j]);
    }
  }
}

int32_t check_compact(const char* fn, const void* pool, const void* pool2, const int32_t* block_tables,
                      int32_t bt_stride, const int32_t* kept, int32_t keep, const int32_t* dst_tables,
                      int32_t dst_stride, int32_t n_reqs, int64_t num_blocks, int32_t hkv, int32_t head_dim) {
  if (n_reqs < 0 || n_reqs > 65535 || keep < 0 || bt_stride < 0 || bt_stride > (1 << 26) || hkv < 1 ||
      num_blocks < 0 || num_blocks > (1LL << 27) || dst_stride < (static_cast<int64_t>(keep) + 15) / 16 ||
      (static_cast<int64_t>(keep) + 15) / 16 * hkv > INT32_MAX)
    return arckv::fail(ARCKV_EINVAL, "%s: bad sizes", fn);
  if (head_dim != 64 && head_dim != 128)
    return arckv::fail(ARCKV_EUNSUPPORTED, "%s: head_dim %d not in {64,128}", fn, head_dim);
  if (n_reqs == 0 || keep == 0) return ARCKV_OK;
  if (pool == nullptr || pool2 == nullptr || block_tables == nullptr || kept == nullptr || dst_tables == nullptr)
    return arckv::fail(ARCKV_EINVAL, "%s: NULL pointer", fn);
  if (reinterpret_cast<uintptr_t>(pool) % 16 != 0 || reinterpret_cast<uintptr_t>(pool2) % 16 != 0)
    return arckv::fail(ARCKV_EINVAL, "%s: pools must be 16-byte aligned", fn);
  return ARCKV_OK;
}

}  // namespace

extern "C" int32_t arckv_evict_select(const float* weights, int64_t w_stride, const int32_t* seq_lens, int32_t n_reqs,
                                      int32_t num_kv_heads, int32_t keep, int32_t n_first, int32_t n_recent,
                                      int32_t* kept, float* kept_weights, int64_t kw_stride, void* stream) {
  const char* fn = "evict_select";
  if (n_reqs < 0 || n_reqs > 65535 || num_kv_heads < 1 || keep < 0 || n_first < 0 || n_recent < 0 ||
      static_cast<int64_t>(n_first) + n_recent > keep || w_stride < 0 || w_stride > INT32_MAX / 2)
    return arckv::fail(ARCKV_EINVAL, "%s: bad sizes", fn);
  if (kept_weights != nullptr && kw_stride < keep)
    return arckv::fail(ARCKV_EINVAL, "%s: kw_stride %lld is less than keep %d", fn, (long long)kw_stride, keep);
  if (n_reqs == 0 || keep == 0) return ARCKV_OK;
  if ((weights == nullptr && w_stride > 0) || seq_lens == nullptr || kept == nullptr)
    return arckv::fail(ARCKV_EINVAL, "%s: NULL pointer", fn);
  hipLaunchKernelGGL(evict_select_kernel, dim3(num_kv_heads, n_reqs), dim3(kSelThreads), 0,
                     static_cast<hipStream_t>(stream), weights, w_stride, seq_lens, num_kv_heads, keep, n_first,
                     n_recent, kept, kept_weights, kw_stride);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return arckv::fail(ARCKV_EDEVICE, "%s: %s", fn, hipGetErrorString(e));
  return ARCKV_OK;
}

extern "C" int32_t arckv_kv_compact(void* k_pool, void* v_pool, const int32_t* block_tables, int32_t bt_stride,
                                    const int32_t* kept, int32_t keep, const int32_t* dst_tables, int32_t dst_stride,
                                    int32_t n_reqs, int64_t num_blocks, int32_t num_kv_heads, int32_t head_dim,
                                    void* stream) {
  const int32_t st = check_compact("kv_compact", k_pool, v_pool, block_tables, bt_stride, kept, keep, dst_tables,
                                   dst_stride, n_reqs, num_blocks, num_kv_heads, head_dim);
  if (st != ARCKV_OK || n_reqs == 0 || keep == 0) return st;
  const dim3 grid(static_cast<unsigned>((keep + 15) / 16) * num_kv_heads, n_reqs);
  auto* s = static_cast<hipStream_t>(stream);
  auto* k = static_cast<uint16_t*>(k_pool);
  auto* v = static_cast<uint16_t*>(v_pool);
  if (head_dim == 64)
    hipLaunchKernelGGL(kv_compact_kernel<64>, grid, dim3(256), 0, s, k, v, block_tables, bt_stride, kept, keep,
                       dst_tables, dst_stride, num_blocks, num_kv_heads);
  else
    hipLaunchKernelGGL(kv_compact_kernel<128>, grid, dim3(256), 0, s, k, v, block_tables, bt_stride, kept, keep,
                       dst_tables, dst_stride, num_blocks, num_kv_heads);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return arckv::fail(ARCKV_EDEVICE, "kv_compact: %s", hipGetErrorString(e));
  return ARCKV_OK;
}

extern "C" int32_t arckv_kv_compact_mx4(void* kv_pool, const int32_t* block_tables, int32_t bt_stride,
                                        const int32_t* kept, int32_t keep, const int32_t* dst_tables,
                                        int32_t dst_stride, int32_t n_reqs, int64_t num_blocks, int32_t num_kv_heads,
                                        int32_t head_dim, void* stream) {
  const int32_t st = check_compact("kv_compact_mx4", kv_pool, kv_pool, block_tables, bt_stride, kept, keep,
                                   dst_tables, dst_stride, n_reqs, num_blocks, num_kv_heads, head_dim);
  if (st != ARCKV_OK || n_reqs == 0 || keep == 0) return st;
  const dim3 grid(static_cast<unsigned>((keep + 15) / 16) * num_kv_heads, n_reqs);
  auto* s = static_cast<hipStream_t>(stream);
  auto* p = static_cast<uint8_t*>(kv_pool);
  if (head_dim == 64)
    hipLaunchKernelGGL(kv_compact_mx4_kernel<64>, grid, dim3(256), 0, s, p, block_tables, bt_stride, kept, keep,
                       dst_tables, dst_stride, num_blocks, num_kv_heads);
  else
    hipLaunchKernelGGL(kv_compact_mx4_kernel<128>, grid, dim3(256), 0, s, p, block_tables, bt_stride, kept, keep,
                       dst_tables, dst_stride, num_blocks, num_kv_heads);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return arckv::fail(ARCKV_EDEVICE, "kv_compact_mx4: %s", hipGetErrorString(e));
  return ARCKV_OK;
}
