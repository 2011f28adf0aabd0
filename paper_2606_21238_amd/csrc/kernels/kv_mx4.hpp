// K/V rows into the 4-bit paged pool and back (part of kv_scatter.hip).
//
// kv_scatter_mx4: pool[slot[t]] <- the codes and scales of (k_new[t], v_new[t]).  Four neighbouring
// lanes hold a group's 32 values, 8 each: the largest magnitude is one packed maximum and two
// lane exchanges away, and every load is 16 bytes of a row.
// kv_gather_mx4: the rows of `slots` as bf16.
// What bounds both is memory: 4 D bytes of rows per token and head against 17 / 16 D of codes.
#pragma once

#include "mx4.hpp"

namespace {

constexpr int kMx4Threads = 256;

template <int D>
__global__ __launch_bounds__(kMx4Threads) void kv_scatter_mx4_kernel(
    uint8_t* __restrict__ pool, const uint16_t* __restrict__ k_new, const uint16_t* __restrict__ v_new,
    const int32_t* __restrict__ slots, int64_t n_tokens, int64_t n_slots, int hkv) {
  using L = mx4::Layout<D>;
  constexpr int CH = D / 8;            // lanes of a row
  const int h = blockIdx.y;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * (kMx4Threads / CH) + threadIdx.x / CH;
  const int c = threadIdx.x % CH;
  const bool there = t < n_tokens;
  const int32_t s = there ? slots[t] : -1;
  ARCKV_CHECK_LANE(there && !(s >= 0 && s < n_slots), ARCKV_CHECK_SLOT);
  uint32_t k[4] = {}, v[4] = {};
  if (there) {
    const int64_t src = (t * hkv + h) * D + c * 8;
    __builtin_memcpy(k, __builtin_assume_aligned(k_new + src, 16), 16);
    __builtin_memcpy(v, __builtin_assume_aligned(v_new + src, 16), 16);
  }
  const uint32_t kb = mx4::scale_byte(mx4::group_top(k)), vb = mx4::scale_byte(mx4::group_top(v));
  const uint32_t kc = mx4::encode8(k, mx4::scale_value(kb)), vc = mx4::encode8(v, mx4::scale_value(vb));
  if (s < 0 || s >= n_slots) return;
  uint8_t* blk = pool + (static_cast<int64_t>(s >> 4) * hkv + h) * L::kBytes;
  const int tt = s & 15;
  *reinterpret_cast<uint32_t*>(blk + tt * L::kRow + c * 4) = kc;
  uint8_t* vp = blk + L::kV + (tt >> 3) * L::kHalf + c * 32 + (tt & 7);
#pragma unroll
  for (int i = 0; i < 4; ++i) vp[8 * i] = static_cast<uint8_t>(vc >> (8 * i));
  if (c % 4 == 0) {
    blk[L::kKScale + tt * L::kGroups + c / 4] = static_cast<uint8_t>(kb);
    blk[L::kVScale + (c / 4) * 16 + tt] = static_cast<uint8_t>(vb);
  }
}

template <int D>
__global__ __launch_bounds__(kMx4Threads) void kv_gather_mx4_kernel(
    const uint8_t* __restrict__ pool, uint16_t* __restrict__ k_out, uint16_t* __restrict__ v_out,
    const int32_t* __restrict__ slots, int64_t n_tokens, int64_t n_slots, int hkv) {
  using L = mx4::Layout<D>;
  constexpr int CH = D / 8;
  const int h = blockIdx.y;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * (kMx4Threads / CH) + threadIdx.x / CH;
  const int c = threadIdx.x % CH;
  if (t >= n_tokens) return;
  const int32_t s = slots[t];
  const bool ok = s >= 0 && s < n_slots;
  ARCKV_CHECK_LANE(!ok, ARCKV_CHECK_SLOT);
  uint32_t k[4] = {}, v[4] = {};
  if (ok) {
    const uint8_t* blk = pool + (static_cast<int64_t>(s >> 4) * hkv + h) * L::kBytes;
    const int tt = s & 15;
    const uint32_t kc = *reinterpret_cast<const uint32_t*>(blk + tt * L::kRow + c * 4);
    const uint8_t* vp = blk + L::kV + (tt >> 3) * L::kHalf + c * 32 + (tt & 7);
    const uint32_t vc = vp[0] | vp[8] << 8 | vp[16] << 16 | static_cast<uint32_t>(vp[24]) << 24;
    const float ks = mx4::scale_value(blk[L::kKScale + tt * L::kGroups + c / 4]);
    const float vs = mx4::scale_value(blk[L::kVScale + (c / 4) * 16 + tt]);
    k[0] = mx4::decode2<0>(kc, ks); k[1] = mx4::decode2<1>(kc, ks);
    k[2] = mx4::decode2<2>(kc, ks); k[3] = mx4::decode2<3>(kc, ks);
    v[0] = mx4::decode2<0>(vc, vs); v[1] = mx4::decode2<1>(vc, vs);
    v[2] = mx4::decode2<2>(vc, vs); v[3] = mx4::decode2<3>(vc, vs);
  }
  const int64_t dst = (t * hkv + h) * D + c * 8;
  __builtin_memcpy(__builtin_assume_aligned(k_out + dst, 16), k, 16);
  __builtin_memcpy(__builtin_assume_aligned(v_out + dst, 16), v, 16);
}

// the checks that both calls make
int32_t check_mx4_rows(const char* fn, const void* pool, const void* k, const void* v, const int32_t* slots,
                       int64_t n_tokens, int64_t num_blocks, int32_t hkv, int32_t head_dim) {
  if (n_tokens < 0 || n_tokens > INT32_MAX || num_blocks < 0 || num_blocks > (1LL << 27) || hkv < 1 || hkv > 65535)
    return arckv::fail(ARCKV_EINVAL, "%s: bad sizes", fn);
  if (head_dim != 64 && head_dim != 128)
    return arckv::fail(ARCKV_EUNSUPPORTED, "%s: head_dim %d not in {64,128}", fn, head_dim);
  if (n_tokens == 0) return ARCKV_OK;
  if (pool == nullptr || k == nullptr || v == nullptr || slots == nullptr)
    return arckv::fail(ARCKV_EINVAL, "%s: NULL pointer", fn);
  for (const void* p : {pool, k, v})
    if (reinterpret_cast<uintptr_t>(p) % 16 != 0)
      return arckv::fail(ARCKV_EINVAL, "%s: the pool and the rows must be 16-byte aligned", fn);
  return ARCKV_OK;
}

}  // namespace

extern "C" int64_t arckv_mx4_pool_bytes(int64_t num_blocks, int32_t num_kv_heads, int32_t head_dim) {
  if (num_blocks < 0 || num_kv_heads < 1 || (head_dim != 64 && head_dim != 128)) return -1;
  return num_blocks * num_kv_heads * 17 * head_dim;
}

extern "C" int32_t arckv_kv_scatter_mx4(void* kv_pool, const void* k_new, const void* v_new,
                                        const int32_t* slot_mapping, int64_t n_tokens, int64_t num_blocks,
                                        int32_t num_kv_heads, int32_t head_dim, void* stream) {
  const int32_t st = check_mx4_rows("kv_scatter_mx4", kv_pool, k_new, v_new, slot_mapping, n_tokens, num_blocks,
                                    num_kv_heads, head_dim);
  if (st != ARCKV_OK || n_tokens == 0) return st;
  const int per = kMx4Threads / (head_dim / 8);
  const dim3 grid(static_cast<unsigned>((n_tokens + per - 1) / per), num_kv_heads);
  auto* s = static_cast<hipStream_t>(stream);
  auto* pool = static_cast<uint8_t*>(kv_pool);
  auto* k = static_cast<const uint16_t*>(k_new);
  auto* v = static_cast<const uint16_t*>(v_new);
  if (head_dim == 64)
    hipLaunchKernelGGL(kv_scatter_mx4_kernel<64>, grid, dim3(kMx4Threads), 0, s, pool, k, v, slot_mapping,
                       n_tokens, num_blocks * 16, num_kv_heads);
  else
    hipLaunchKernelGGL(kv_scatter_mx4_kernel<128>, grid, dim3(kMx4Threads), 0, s, pool, k, v, slot_mapping,
                       n_tokens, num_blocks * 16, num_kv_heads);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return arckv::fail(ARCKV_EDEVICE, "kv_scatter_mx4: %s", hipGetErrorString(e));
  return ARCKV_OK;
}

extern "C" int32_t arckv_kv_gather_mx4(const void* kv_pool, void* k_out, void* v_out, const int32_t* slot_mapping,
                                       int64_t n_tokens, int64_t num_blocks, int32_t num_kv_heads,
                                       int32_t head_dim, void* stream) {
  const int32_t st = check_mx4_rows("kv_gather_mx4", kv_pool, k_out, v_out, slot_mapping, n_tokens, num_blocks,
                                    num_kv_heads, head_dim);
  if (st != ARCKV_OK || n_tokens == 0) return st;
  const int per = kMx4Threads / (head_dim / 8);
  const dim3 grid(static_cast<unsigned>((n_tokens + per - 1) / per), num_kv_heads);
  auto* s = static_cast<hipStream_t>(stream);
  auto* pool = static_cast<const uint8_t*>(kv_pool);
  auto* k = static_cast<uint16_t*>(k_out);
  auto* v = static_cast<uint16_t*>(v_out);
  if (head_dim == 64)
    hipLaunchKernelGGL(kv_gather_mx4_kernel<64>, grid, dim3(kMx4Threads), 0, s, pool, k, v, slot_mapping, n_tokens,
                       num_blocks * 16, num_kv_heads);
  else
    hipLaunchKernelGGL(kv_gather_mx4_kernel<128>, grid, dim3(kMx4Threads), 0, s, pool, k, v, slot_mapping, n_tokens,
                       num_blocks * 16, num_kv_heads);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return arckv::fail(ARCKV_EDEVICE, "kv_gather_mx4: %s", hipGetErrorString(e));
  return ARCKV_OK;
}
