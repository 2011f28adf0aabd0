// The attention weight that every cached token receives (part of prefill_attn.hip).
//
//   w[r][h][j] (+)= sum over the columns c of KV head h that see key j of exp(scale q_c . K[j] - lse_c)
//
// Keys are stationary: a wave holds 64 keys of one (request, KV head) as MFMA operands and the
// columns stream past them through LDS, 128 at a time.  S = Q . K^T with
// v_mfma_f32_32x32x16_bf16 puts one key on a lane and 16 columns in its registers, so the sum over
// columns is the lane's own; every weight is written once, by one lane, in one order, with no
// atomics.  A work-group of 8 waves takes KW x 64 keys; its 8 / KW waves of the same keys share
// the columns and add up through LDS at the end.
#pragma once

#include "mx4.hpp"

namespace {

constexpr int kWtCols = 128;    // columns in LDS at a time: 4 tiles of 32

template <int D, bool MX4, int KW>
__global__ __launch_bounds__(512, 2) void attn_weights_kernel(
    const uint8_t* __restrict__ pool, const uint16_t* __restrict__ q, const float* __restrict__ lse,
    const int32_t* __restrict__ block_tables, int bt_stride, const int32_t* __restrict__ cu_q,
    const int32_t* __restrict__ seq_lens, int64_t n_q, int64_t num_blocks, int hq, int hkv, int G, float scale_log2,
    float* __restrict__ weights, int64_t w_stride, int accumulate) {
  constexpr int kThreads = 512, CS = 8 / KW, KS = D / 16, TILES = kWtCols / 32;
  constexpr int kRowBytes = D * 2, kChunkBytes = kWtCols * kRowBytes;
  constexpr int NLD = kChunkBytes / (kThreads * 16);      // 16-byte loads of a thread for a chunk
  constexpr int kRowThreads = kRowBytes / 16, kRowsPer = kThreads / kRowThreads;
  __shared__ __attribute__((aligned(1024))) char qs[2][kChunkBytes];
  __shared__ __attribute__((aligned(16))) float ls[2][kWtCols];
  __shared__ float part[CS > 1 ? (CS - 1) * KW * 64 : 1];
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hg = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), kw = wave % KW, cs = wave / KW;
  const int kvh = blockIdx.x % hkv, r = blockIdx.y;
  const int q0 = cu_q[r], qlen = cu_q[r + 1] - q0, len = seq_lens[r], P = len - qlen;
  const int64_t bound = min(static_cast<int64_t>(min(len, bt_stride * 16)), w_stride);
  const int64_t wg_key = static_cast<int64_t>(blockIdx.x / hkv) * (KW * 64);
  if (wg_key >= bound) return;
  const int key0 = static_cast<int>(wg_key) + kw * 64;
  const int ncols = min(static_cast<int64_t>(qlen), max(n_q - q0, static_cast<int64_t>(0))) * G;
  // columns from the first that sees the work-group's first key
  const int first = static_cast<int>(min(static_cast<int64_t>(max(0, static_cast<int>(wg_key) - P)) * G, static_cast<int64_t>(ncols)));
  const int c_lo = first / kWtCols * kWtCols;

  // ---- the wave's keys: lane l32 of subtile s is key key0 + 32 s + l32 ---------------------------
  bf16x8_t kf[2][KS];
  const int32_t* bt = block_tables + static_cast<int64_t>(r) * bt_stride;
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const int key = key0 + 32 * s + l32;
    const int e = min(key, max(static_cast<int>(bound) - 1, 0)) >> 4;
    int32_t ph = bt[e];
    const bool bad = ph < 0 || ph >= num_blocks;
    ARCKV_CHECK_LANE(key < bound && bad && (key & 15) == 0 && hg == 0, ARCKV_CHECK_BLOCK);
    ph = bad ? 0 : ph;               // an entry out of range reads block 0
    const int64_t blk = static_cast<int64_t>(ph) * hkv + kvh;
    if constexpr (MX4) {
      using L = mx4::Layout<D>;
      const uint8_t* b = pool + blk * L::kBytes;
      uint32_t c[D / 16];
      __builtin_memcpy(c, __builtin_assume_aligned(b + (key & 15) * L::kRow + hg * (D / 4), 16), D / 4);
#pragma unroll
      for (int g = 0; g < D / 64; ++g) {
        const float sc = mx4::scale_value(b[L::kKScale + (key & 15) * L::kGroups + hg * (D / 64) + g]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t w = c[4 * g + i];
          kf[s][4 * g + i] = __builtin_bit_cast(bf16x8_t, u32x4_t{mx4::decode2<0>(w, sc), mx4::decode2<1>(w, sc),
                                                                  mx4::decode2<2>(w, sc), mx4::decode2<3>(w, sc)});
        }
      }
    } else {
      const uint8_t* b = pool + (blk * 16 + (key & 15)) * kRowBytes;
#pragma unroll
      for (int i = 0; i < KS; ++i) kf[s][i] = *reinterpret_cast<const bf16x8_t*>(b + 32 * i + 16 * hg);
    }
  }

  // ---- columns: rows of q and their sums, a chunk ahead in registers ---------------------------------
  u32x4_t qn[NLD];
  float ln = 0.f;
  auto fetch = [&](int c0) {
#pragma unroll
    for (int i = 0; i < NLD; ++i) {
      const int c = c0 + i * kRowsPer + tid / kRowThreads;
      const int tok = c / G;
      const int64_t row = static_cast<int64_t>(q0 + tok) * hq + kvh * G + (c - tok * G);
      qn[i] = u32x4_t{};
      if (c < ncols) __builtin_memcpy(&qn[i], q + row * D + (tid % kRowThreads) * 8, 16);
    }
    if (tid < kWtCols) {
      const int c = c0 + tid, tok = c / G;
      ln = c < ncols ? lse[static_cast<int64_t>(q0 + tok) * hq + kvh * G + (c - tok * G)] * 1.4426950408889634f : 0.f;
    }
  };
  auto put = [&](int buf) {
#pragma unroll
    for (int i = 0; i < NLD; ++i) {
      const int c = i * kRowsPer + tid / kRowThreads, ch = tid % kRowThreads;
      *reinterpret_cast<u32x4_t*>(qs[buf] + c * kRowBytes + ((ch ^ fk<D>(c)) * 16)) = qn[i];
    }
    if (tid < kWtCols) ls[buf][tid] = ln;
  };
  float acc[2] = {0.f, 0.f};
  int cmin[2];           // the first column that sees this lane's key
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const int64_t c = static_cast<int64_t>(max(0, key0 + 32 * s + l32 - P)) * G;
    cmin[s] = static_cast<int>(min(c, static_cast<int64_t>(INT32_MAX)));
  }
  const int64_t all_see = static_cast<int64_t>(max(0, key0 + 63 - P)) * G;   // columns from here on see every key of the wave

  if (c_lo < ncols) {
    fetch(c_lo);
    put(0);
  }
  __syncthreads();
  int buf = 0;
  for (int c0 = c_lo; c0 < ncols; c0 += kWtCols, buf ^= 1) {
    const bool more = c0 + kWtCols < ncols;
    if (more) fetch(c0 + kWtCols);
    for (int t = cs; t < TILES; t += CS) {
      const int cb = c0 + 32 * t;
      if (cb >= ncols) break;
      const char* qb = qs[buf] + 32 * t * kRowBytes;
      f32x16_t s[2];
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        const int ch = MX4 ? hg * KS + i : 2 * i + hg;
        const bf16x8_t a = *reinterpret_cast<const bf16x8_t*>(qb + l32 * kRowBytes + ((ch ^ fk<D>(l32)) * 16));
#pragma unroll
        for (int x = 0; x < 2; ++x)
          s[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, kf[x][i], i == 0 ? f32x16_t{} : s[x], 0, 0, 0);
      }
      const bool masked = cb < all_see || cb + 32 > ncols;
      float sum[2][4];
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4_t l4 = *reinterpret_cast<const f32x4_t*>(&ls[buf][32 * t + 8 * g + 4 * hg]);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          float p[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) p[j] = fast_exp2(fmaf(s[x][4 * g + j], scale_log2, -l4[j]));
          if (masked) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int c = cb + 8 * g + 4 * hg + j;
              p[j] = c >= cmin[x] && c < ncols ? p[j] : 0.f;
            }
          }
          sum[x][g] = (p[0] + p[1]) + (p[2] + p[3]);
        }
      }
#pragma unroll
      for (int x = 0; x < 2; ++x) acc[x] += (sum[x][0] + sum[x][1]) + (sum[x][2] + sum[x][3]);
    }
    if (more) put(buf ^ 1);
    __syncthreads();
  }
  // ---- the two halves of a key's columns, then the waves that shared the columns --------------------
  const float a0 = sum_halves(acc[0]), a1 = sum_halves(acc[1]);
  float total = hg == 0 ? a0 : a1;     // lane = key key0 + lane
  if constexpr (CS > 1) {
    if (cs > 0) part[((cs - 1) * KW + kw) * 64 + lane] = total;
    __syncthreads();
    if (cs > 0) return;
#pragma unroll
    for (int c = 1; c < CS; ++c) total += part[((c - 1) * KW + kw) * 64 + lane];
  }
  const int key = key0 + lane;
  if (key >= bound) return;
  float* w = weights + (static_cast<int64_t>(r) * hkv + kvh) * w_stride + key;
  *w = accumulate ? *w + total : total;
}

}  // namespace

extern "C" int32_t arckv_attention_weights(const void* k_pool, int32_t layout, const void* q, const float* lse,
                                           const int32_t* block_tables, int32_t bt_stride, const int32_t* cu_q,
                                           const int32_t* seq_lens, int32_t n_reqs, int64_t n_q, int64_t num_blocks,
                                           int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, float scale,
                                           float* weights, int64_t w_stride, int32_t accumulate, void* stream) {
  const char* fn = "attention_weights";
  if (layout != ARCKV_LAYOUT_V1 && layout != ARCKV_LAYOUT_MX4)
    return arckv::fail(ARCKV_EINVAL, "%s: layout %d is neither V1 nor MX4", fn, layout);
  const int32_t rc = check_attention(fn, n_reqs, n_q, num_blocks, 0, 0, arckv::kWideCols, num_q_heads, num_kv_heads,
                                     head_dim, bt_stride, scale, 0);
  if (rc != ARCKV_OK) return rc;
  if (w_stride < 0 || w_stride > INT32_MAX || n_reqs > 65535 || num_blocks > (1LL << 27) || bt_stride > (1 << 26))
    return arckv::fail(ARCKV_EINVAL, "%s: bad sizes", fn);
  if (n_reqs == 0 || w_stride == 0 || bt_stride == 0) return ARCKV_OK;
  if (k_pool == nullptr || block_tables == nullptr || cu_q == nullptr || seq_lens == nullptr || weights == nullptr ||
      (n_q > 0 && (q == nullptr || lse == nullptr)))
    return arckv::fail(ARCKV_EINVAL, "%s: NULL pointer", fn);
  if (reinterpret_cast<uintptr_t>(k_pool) % 16 != 0)
    return arckv::fail(ARCKV_EINVAL, "%s: the pool must be 16-byte aligned", fn);
  if (num_blocks == 0) return arckv::fail(ARCKV_EINVAL, "%s: num_blocks", fn);
  const int G = num_q_heads / num_kv_heads;
  const int64_t keys = std::min<int64_t>(w_stride, static_cast<int64_t>(bt_stride) * 16);
  const int KW = 8;
  const int64_t wgs = (keys + KW * 64 - 1) / (KW * 64) * num_kv_heads;
  if (wgs > INT32_MAX) return arckv::fail(ARCKV_EINVAL, "%s: too many keys", fn);
  const dim3 grid(static_cast<unsigned>(wgs), n_reqs);
  auto* st = static_cast<hipStream_t>(stream);
#define ARCKV_WEIGHTS(DD, MM, KK)                                                                              \
  hipLaunchKernelGGL((attn_weights_kernel<DD, MM, KK>), grid, dim3(512), 0, st, static_cast<const uint8_t*>(k_pool), \
                     static_cast<const uint16_t*>(q), lse, block_tables, bt_stride, cu_q, seq_lens, n_q, num_blocks,  \
                     num_q_heads, num_kv_heads, G, scale * 1.4426950408889634f, weights, w_stride, accumulate)
  const bool mx = layout == ARCKV_LAYOUT_MX4;
  if (head_dim == 64) {
    if (mx) ARCKV_WEIGHTS(64, true, 8); else ARCKV_WEIGHTS(64, false, 8);
  } else {
    if (mx) ARCKV_WEIGHTS(128, true, 8); else ARCKV_WEIGHTS(128, false, 8);
  }
#undef ARCKV_WEIGHTS
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return arckv::fail(ARCKV_EDEVICE, "%s: %s", fn, hipGetErrorString(e));
  return ARCKV_OK;
}
