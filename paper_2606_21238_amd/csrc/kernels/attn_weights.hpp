// The attention weight that every cached token receives (part of prefill_attn.hip).
//
//   w[r][h][j] (+)= sum over the columns c of KV head h that see key j of exp(scale q_c . K[j] - lse_c)
//
// Many columns: keys are stationary, a wave holds 32 keys of one (request, KV head) as MFMA operands and
// the columns stream past them through LDS, 128 at a time.  Few: columns are stationary and keys stream
// (which is which stands at the launch).  S = Q . K^T with v_mfma_f32_32x32x16_bf16 puts one key on two
// lanes, 16 columns in the registers of each, so the sum over columns is the lanes' own; every weight is
// written once, by one lane, in one order, with no atomics.
//
// Everything behind the products is fp32; lse goes to base 2 first (one rounding of it, 2^-24 of its size), so that an
// exponential takes one fused step, and the weights are 1.5e-7 to 2.3e-7 of their root mean square off the 64-bit ones
// (an fp32 form that subtracts first, one more step for each: 0.5e-7 to 0.8e-7).
//
// What bounds it: many columns, one exponential for each (column, key) beside 2 D products (half of the
// attention's): 2048 tokens on 32768, 64 / 8 heads of 128, 1.23 to 1.28 ms, 0.9 PFLOP/s; few, the keys' bytes: one
// token of each of 64 requests of 8192, 32 / 8, 68 us at 4 bits (half of the attention kernel's 128) and 220 in
// bf16 (5.0 TB/s).
#pragma once

#include "mx4.hpp"

namespace {

constexpr int kWtCols = 128;    // columns in LDS at a time: 4 tiles of 32
constexpr float kLog2e = 1.4426950408889634f;

// What a work-group needs of its request.
struct WtReq {
  int q0, P, ncols, bound;      // first row, cached tokens, columns, keys that get a weight
  const int32_t* bt;
};
__device__ __forceinline__ WtReq wt_request(int r, const int32_t* block_tables, int bt_stride, const int32_t* cu_q,
                                            const int32_t* seq_lens, int64_t n_q, int G, int64_t w_stride) {
  WtReq x;
  x.q0 = cu_q[r];
  const int qlen = cu_q[r + 1] - x.q0, len = seq_lens[r];
  x.P = len - qlen;
  x.ncols = static_cast<int>(min(static_cast<int64_t>(qlen), max(n_q - x.q0, static_cast<int64_t>(0)))) * G;
  x.bound = static_cast<int>(min(static_cast<int64_t>(min(len, bt_stride * 16)), w_stride));
  x.bt = block_tables + static_cast<int64_t>(r) * bt_stride;
  return x;
}

// One key's bytes as a lane holds them: lane l32 of a subtile of 32 keys has its key's dimensions of k-steps
// 0 .. KS - 1 of its half hg: 16 i + 8 hg .. (bf16 rows), hg D / 2 + 8 i .. (codes: one piece of a row).
template <int D, bool MX4>
struct WtKey {
  static constexpr int KS = D / 16;
  uint32_t c[MX4 ? D / 16 : D / 4];
  uint32_t sc[MX4 ? D / 64 : 1];

  __device__ __forceinline__ void load(const uint8_t* pool, int32_t ph, int64_t num_blocks, int hkv, int kvh, int key,
                                       int hg) {
    const bool bad = ph < 0 || ph >= num_blocks;
    ARCKV_CHECK_LANE(bad && (key & 15) == 0 && hg == 0, ARCKV_CHECK_BLOCK);
    const int64_t blk = static_cast<int64_t>(bad ? 0 : ph) * hkv + kvh;      // an entry out of range reads block 0
    if constexpr (MX4) {
      using L = mx4::Layout<D>;
      const uint8_t* b = pool + blk * L::kBytes;
      __builtin_memcpy(c, __builtin_assume_aligned(b + (key & 15) * L::kRow + hg * (D / 4), 16), D / 4);
#pragma unroll
      for (int g = 0; g < D / 64; ++g) sc[g] = b[L::kKScale + (key & 15) * L::kGroups + hg * (D / 64) + g];
    } else {
      const uint8_t* b = pool + (blk * 16 + (key & 15)) * (2 * D) + 16 * hg;
#pragma unroll
      for (int i = 0; i < KS; ++i) __builtin_memcpy(c + 4 * i, __builtin_assume_aligned(b + 32 * i, 16), 16);
    }
  }
  __device__ __forceinline__ bf16x8_t step(int i) const {
    if constexpr (MX4) {
      const float s = mx4::scale_value(sc[i / 4]);
      return __builtin_bit_cast(bf16x8_t, u32x4_t{mx4::decode2<0>(c[i], s), mx4::decode2<1>(c[i], s),
                                                  mx4::decode2<2>(c[i], s), mx4::decode2<3>(c[i], s)});
    } else {
      return __builtin_bit_cast(bf16x8_t, u32x4_t{c[4 * i], c[4 * i + 1], c[4 * i + 2], c[4 * i + 3]});
    }
  }
};
// the 16-byte chunk of a row of q that goes with k-step i
template <int D, bool MX4>
__device__ __forceinline__ int wt_chunk(int i, int hg) { return MX4 ? hg * (D / 16) + i : 2 * i + hg; }

// The weights of 32 columns for this lane's key, of S's 16 registers: register 4 g + j is column cb + 8 g + 4 hg + j.
template <bool MASKED, class Lse>
__device__ __forceinline__ float wt_sum(const f32x16_t& s, Lse lse, float scale_log2, int cb, int hg,
                                        int cmin, int ncols, int groups = 4) {
  float sum[4] = {};
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    if (g >= groups) break;                          // (uniform) the columns from 8 g on are not there
    const f32x4_t l4 = lse(g);
    float p[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) p[j] = fast_exp2(fmaf(s[4 * g + j], scale_log2, -l4[j]));
    if constexpr (MASKED) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int c = cb + 8 * g + 4 * hg + j;
        p[j] = c >= cmin && c < ncols ? p[j] : 0.f;
      }
    }
    sum[g] = (p[0] + p[1]) + (p[2] + p[3]);
  }
  return (sum[0] + sum[1]) + (sum[2] + sum[3]);
}

// the first column that sees a key
__device__ __forceinline__ int first_column(int64_t key, int P, int G) {
  return static_cast<int>(min(max(key - P, static_cast<int64_t>(0)) * G, static_cast<int64_t>(INT32_MAX)));
}

// Many columns: keys stay, columns stream.  n_split work-groups share a (request, KV head) in equal runs of
// subtiles of 32 keys; a work-group takes 8 of its subtiles at a time, one for each wave, and where fewer
// are left, 2 or 4 waves share a subtile's columns.
template <int D, bool MX4, bool ANY>
__global__ __launch_bounds__(512, 4) void attn_weights_kernel(
    const uint8_t* __restrict__ pool, const uint16_t* __restrict__ q, const float* __restrict__ lse,
    const int32_t* __restrict__ block_tables, int bt_stride, const int32_t* __restrict__ cu_q,
    const int32_t* __restrict__ seq_lens, int64_t n_q, int64_t num_blocks, int hq, int hkv, GroupDiv gd, float scale_log2,
    float* __restrict__ weights, int64_t w_stride, int accumulate, int n_split, int cols_from, int cols_to) {
  constexpr int kThreads = 512, KS = D / 16, TILES = kWtCols / 32;
  constexpr int kRowBytes = D * 2, kChunkBytes = kWtCols * kRowBytes;
  constexpr int NLD = kChunkBytes / (kThreads * 16);      // 16-byte loads of a thread for a chunk
  constexpr int kRowThreads = kRowBytes / 16, kWaveRows = 64 / kRowThreads;
  __shared__ __attribute__((aligned(1024))) char qs[2][kChunkBytes];
  __shared__ __attribute__((aligned(16))) float ls[2][kWtCols];
  __shared__ float part[6][2][64];                        // of the waves that only help
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hg = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kvh = blockIdx.x % hkv, r = blockIdx.y, G = static_cast<int>(gd.g);
  const WtReq rq = wt_request(r, block_tables, bt_stride, cu_q, seq_lens, n_q, G, w_stride);
  if (rq.ncols < cols_from || rq.ncols > cols_to) return;    // of the other kernel's
  float* const wrow = weights + (static_cast<int64_t>(r) * hkv + kvh) * w_stride;

  // Rows of q straight into LDS, chunk x of row c at x ^ fk(c); columns past the last load row 0, never used.
  // ANY: q at an address that is not a multiple of 16 goes through registers.
  float ln = 0.f;
  auto fetch = [&](int c0, int buf) {
#pragma unroll
    for (int i = 0; i < NLD; ++i) {
      const int at = i * (kThreads * 16) + wave * 1024;   // of the wave's 64 pieces of 16 bytes
      const int cl = at / kRowBytes + lane / kRowThreads, c = c0 + cl, tok = gd.tok(c);
      const int64_t row = c < rq.ncols ? static_cast<int64_t>(rq.q0 + tok) * hq + kvh * G + (c - tok * G) : 0;
      const uint16_t* src = q + row * D + (((lane % kRowThreads) ^ fk<D>(cl)) * 8);
      if constexpr (ANY) load_any16(src, qs[buf] + at + lane * 16);
      else load_lds16(src, (lds_void*)(qs[buf] + at));
    }
    if (tid < kWtCols) {
      const int c = c0 + tid, tok = gd.tok(c);
      ln = c < rq.ncols ? lse[static_cast<int64_t>(rq.q0 + tok) * hq + kvh * G + (c - tok * G)] * kLog2e : 0.f;
    }
  };
  auto landed = [&](int buf) {                            // this wave's part of a chunk is in LDS
    if (tid < kWtCols) ls[buf][tid] = ln;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  };
  static_assert(kWaveRows * kRowBytes == 1024, "a wave's load is whole rows");

  const int nsub = (rq.bound + 31) / 32;
  const int64_t share = blockIdx.x / hkv;
  const int sub1 = static_cast<int>((share + 1) * nsub / n_split);
  for (int sub = static_cast<int>(share * nsub / n_split), step; sub < sub1; sub += step) {
    step = min(sub1 - sub, 8);
    const int KW = step > 4 ? 8 : step > 2 ? 4 : 2, CS = 8 / KW;             // uniform
    const int kw = wave % KW, cs = wave / KW;
    const int64_t wg_key = static_cast<int64_t>(sub) * 32;
    const int key = sub * 32 + kw * 32 + l32;
    const bool mine = kw < step;                                             // a subtile of its own
    // keys and the first columns are asked for together
    WtKey<D, MX4> raw;
    raw.load(pool, rq.bt[min(key, rq.bound - 1) >> 4], num_blocks, hkv, kvh, key, hg);
    const int c_lo = min(first_column(wg_key, rq.P, G), rq.ncols) / kWtCols * kWtCols;
    const int cmin = first_column(key, rq.P, G);
    const int all_see = first_column(wg_key + kw * 32 + 31, rq.P, G);   // columns from here on see every key of the wave
    // sums of the tiles 0, 1, 2, 3 modulo 4 (of which a wave has every CS-th), added up in one order whoever has them
    float acc[TILES] = {};
    if (c_lo < rq.ncols) fetch(c_lo, 0);
    bf16x8_t kf[KS];
#pragma unroll
    for (int i = 0; i < KS; ++i) kf[i] = raw.step(i);
    if (c_lo < rq.ncols) landed(0);
    __syncthreads();
    int buf = 0;
    for (int c0 = c_lo; c0 < rq.ncols; c0 += kWtCols, buf ^= 1) {
      const bool more = c0 + kWtCols < rq.ncols;
      if (more) fetch(c0 + kWtCols, buf ^ 1);
      const int nt = mine ? min(TILES, (rq.ncols - c0 + 31) / 32) : 0;
      // rows start at multiples of 256 (D = 64: 128) bytes: the swizzled chunks are an exclusive or away
      const uint32_t a0 = l32 * kRowBytes + ((wt_chunk<D, MX4>(0, hg) ^ fk<D>(l32)) * 16);
      auto at = [&](int t, int i) {
        const char* qb = qs[buf] + t * (32 * kRowBytes);
        return *reinterpret_cast<const bf16x8_t*>(qb + (a0 ^ (wt_chunk<D, MX4>(i, 0) * 16)));
      };
      // a tile's first operands are read beside the exponentials of the tile before (as many as 128 registers hold)
      constexpr int kAhead = KS / 2 - (MX4 && D == 128 ? 1 : 0);
      bf16x8_t a[KS];
      auto read_first = [&](int t) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) a[i] = at(t, i);
      };
      if (cs < nt) read_first(cs);
#pragma unroll
      for (int k = 0; k < TILES; ++k) {
        const int t = cs + CS * k, cb = c0 + 32 * t;
        if (t >= nt) break;
#pragma unroll
        for (int i = kAhead; i < KS; ++i) a[i] = at(t, i);
        f32x16_t s;
#pragma unroll
        for (int i = 0; i < KS; ++i)
          s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i], kf[i], i == 0 ? f32x16_t{} : s, 0, 0, 0);
        if (t + CS < nt) read_first(t + CS);
        const float* lt = &ls[buf][32 * t + 4 * hg];
        auto l4 = [&](int g) { return *reinterpret_cast<const f32x4_t*>(lt + 8 * g); };
        if (cb < all_see || cb + 32 > rq.ncols) acc[k] += wt_sum<true>(s, l4, scale_log2, cb, hg, cmin, rq.ncols);
        else acc[k] += wt_sum<false>(s, l4, scale_log2, cb, hg, cmin, rq.ncols);
      }
      if (more) landed(buf ^ 1);
      __syncthreads();
    }
    float total = (acc[0] + acc[1]) + (acc[2] + acc[3]);
    if (CS > 1) {
      if (cs > 0) {
        part[wave - KW][0][lane] = acc[0];
        part[wave - KW][1][lane] = acc[1];
      }
      __syncthreads();
      if (CS == 2) total = (acc[0] + part[kw][0][lane]) + (acc[1] + part[kw][1][lane]);
      else total = (acc[0] + part[kw][0][lane]) + (part[kw + KW][0][lane] + part[kw + 2 * KW][0][lane]);
    }
    total = sum_halves(total);             // the other columns of the key
    if (cs == 0 && mine && hg == 0 && key < rq.bound) wrow[key] = accumulate ? wrow[key] + total : total;
  }
}

// Few columns (decode): columns stay, 32 of them in registers, and keys stream, 32 at a time for a wave,
// the next 32 on their way meanwhile.  Waves of n_split work-groups take a request's subtiles in turn.
template <int D, bool MX4>
__global__ __launch_bounds__(256, MX4 || D == 64 ? 4 : 3) void attn_weights_stream_kernel(
    const uint8_t* __restrict__ pool, const uint16_t* __restrict__ q, const float* __restrict__ lse,
    const int32_t* __restrict__ block_tables, int bt_stride, const int32_t* __restrict__ cu_q,
    const int32_t* __restrict__ seq_lens, int64_t n_q, int64_t num_blocks, int hq, int hkv, GroupDiv gd, float scale_log2,
    float* __restrict__ weights, int64_t w_stride, int accumulate, int n_split, int cols_from, int cols_to) {
  constexpr int KS = D / 16;
  const int lane = threadIdx.x & 63, l32 = lane & 31, hg = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kvh = blockIdx.x % hkv, r = blockIdx.y, G = static_cast<int>(gd.g);
  const WtReq rq = wt_request(r, block_tables, bt_stride, cu_q, seq_lens, n_q, G, w_stride);
  if (rq.ncols < cols_from || rq.ncols > cols_to) return;    // of the other kernel's
  float* const wrow = weights + (static_cast<int64_t>(r) * hkv + kvh) * w_stride;
  const int first = blockIdx.x / hkv * 4 + wave, by = 4 * n_split, nsub = (rq.bound + 31) / 32;
  if (first >= nsub) return;
  const int tiles = max((rq.ncols + 31) / 32, accumulate ? 0 : 1);
  for (int t = 0; t < tiles; ++t) {                  // more than 32 columns: pass after pass over the same keys
    const int cb = 32 * t, c = cb + l32, tok = gd.tok(c);
    const int64_t row = c < rq.ncols ? static_cast<int64_t>(rq.q0 + tok) * hq + kvh * G + (c - tok * G) : 0;
    WtKey<D, MX4> raw;
    float old = 0.f;
    auto fetch = [&](int sub, int32_t ph) {
      const int key = sub * 32 + l32;
      raw.load(pool, ph, num_blocks, hkv, kvh, key, hg);
      if ((accumulate || t > 0) && hg == 0) old = key < rq.bound ? wrow[key] : 0.f;
    };
    auto block = [&](int sub) { return rq.bt[min(sub * 32 + l32, rq.bound - 1) >> 4]; };
    fetch(first, block(first));
    int32_t ph = block(min(first + by, nsub - 1));
    bf16x8_t a[KS];
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      a[i] = bf16x8_t{};
      if (c < rq.ncols) __builtin_memcpy(&a[i], q + row * D + wt_chunk<D, MX4>(i, hg) * 8, 16);
    }
    // A column that is not there: q of zeros and a sum of infinity give a weight of zero, over finite keys.  Zero times
    // an infinite one is NaN, so with bf16 keys such columns are masked (of 4-bit keys what is not finite is NaN for the
    // columns that are there too).
    const float mine = c < rq.ncols ? lse[row] * kLog2e : INFINITY;
    f32x4_t l4[4];
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
      for (int j = 0; j < 4; ++j) l4[g][j] = __shfl(mine, 8 * g + 4 * hg + j);
    const int pos0 = rq.P + gd.tok(cb), groups = (min(32, rq.ncols - cb) + 7) / 8;
    for (int sub = first; sub < nsub; sub += by) {
      f32x16_t s;
#pragma unroll
      for (int i = 0; i < KS; ++i)
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i], raw.step(i), i == 0 ? f32x16_t{} : s, 0, 0, 0);
      const float was = old;
      if (sub + by < nsub) {
        fetch(sub + by, ph);
        ph = block(min(sub + 2 * by, nsub - 1));
      }
      const int key = sub * 32 + l32;
      const bool masked = sub * 32 + 31 > pos0 || (!MX4 && rq.ncols < cb + 8 * groups);
      auto sums = [&](int g) { return l4[g]; };
      const float mine32 = masked ? wt_sum<true>(s, sums, scale_log2, cb, hg, first_column(key, rq.P, G), rq.ncols, groups)
                                  : wt_sum<false>(s, sums, scale_log2, cb, hg, 0, rq.ncols, groups);
      const float total = sum_halves(mine32);
      if (hg == 0 && key < rq.bound) wrow[key] = was + total;
    }
  }
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
  const int64_t pairs = static_cast<int64_t>(n_reqs) * num_kv_heads;
  auto* st = static_cast<hipStream_t>(stream);
  const GroupDiv gd{static_cast<uint32_t>(G), G == 1 ? 0 : static_cast<uint32_t>(((1ull << 32) + G - 1) / G)};
  // work-groups for each (request, KV head): about `want` in all, at least `least` to a pair, each with `per` keys
  // or more
  auto split = [&](int64_t per, int64_t want, int64_t least) {
    return static_cast<int>(
        std::max<int64_t>(1, std::min((keys + per - 1) / per, std::max(least, (want + pairs - 1) / pairs))));
  };
#define ARCKV_WEIGHTS(KERNEL, THREADS, PER, WANT, LEAST, FROM, TO)                                             \
  do {                                                                                                         \
    const int ns = split(PER, WANT, LEAST);                                                                    \
    hipLaunchKernelGGL((KERNEL), dim3(static_cast<unsigned>(ns) * num_kv_heads, n_reqs), dim3(THREADS), 0, st, \
                       static_cast<const uint8_t*>(k_pool), static_cast<const uint16_t*>(q), lse, block_tables, \
                       bt_stride, cu_q, seq_lens, n_q, num_blocks, num_q_heads, num_kv_heads, gd,              \
                       scale * 1.4426950408889634f, weights, w_stride, accumulate, ns, FROM, TO);              \
  } while (0)
  // Which kernel takes a request.  Up to 32 columns (bf16) or 64 (4 bits) its keys may stream past them: a second
  // pass over bf16 keys costs more than what the other kernel's start does.  Streaming and stationary keys at 64
  // requests of 2000, 32 / 8 heads: 4 columns 44 and 52 us (bf16), 17 and 34 (4 bits); 32: 45 and 50, 20 and 30;
  // 48: 75 and 55, 31 and 38; 64: 76 and 55, 33 and 36; 128: 136 and 67, 59 and 51.  A batch of so few on average
  // streams; requests over the limit, which there may be where some have several rows, are a second launch's.
  const int limit = layout == ARCKV_LAYOUT_MX4 ? 64 : 32;
  const bool few = n_q * G <= static_cast<int64_t>(n_reqs) * limit;
  const bool mixed = few && n_q > n_reqs && n_q * G > limit;
  const bool any = reinterpret_cast<uintptr_t>(q) % 16 != 0;
  const int stream_to = mixed ? limit : INT32_MAX, stay_from = mixed ? limit + 1 : INT32_MIN;
  // Streaming: one round of the 1024 work-groups that fit at once, at least two to a pair and one for every 2048 keys
  // that a request may have, which is what its longest request takes (64 requests of 2000 at 4 bits, about 1024, 2048
  // and 4096 work-groups in all: 17, 19 and 21 us; of 8192: 65, 68 and 71; 256 ragged ones up to 3400, one and two to a
  // pair: 84 and 75; 64 lognormal ones up to 12000, two and seven: 82 and 33); bf16, whose keys are the bound, two
  // rounds (8 requests of 8000, 32 columns, 2048 and 4096: 28 and 34; 16 ragged ones up to 12000, 1024, 2048 and 4096:
  // 57, 51 and 49).
  // Stationary: about 512 (8 questions of 128 on 8192, 512, 1024 and 2048: 129, 141 and 146 us), but up to 4 to a pair
  // where its keys are over 1024 each, for one request may have most of the rows (64 requests of 2600, one of
  // them with 512 rows: 437 and 218 us, at the price of 73 and 79 us for 64 equal ones of 64 rows, 16 / 16 heads of
  // 64); beside a streaming launch 8 (one of 128 rows among 63 of one: 44 us, and 134 where it streams too; the
  // second launch costs 3 us where it finds no request).
  const int64_t least = std::max<int64_t>(2, (keys + 2047) / 2048);
  const int64_t least_stay = mixed ? 8 : std::min<int64_t>(4, (keys + 1023) / 1024);
#define ARCKV_WEIGHTS_DM(DD, MM)                                                                              \
  do {                                                                                                        \
    if (few) ARCKV_WEIGHTS((attn_weights_stream_kernel<DD, MM>), 256, 128, MM ? 1024 : 2048, least, INT32_MIN, stream_to); \
    if (!few || mixed) {                                                                                      \
      if (any) ARCKV_WEIGHTS((attn_weights_kernel<DD, MM, true>), 512, 64, 512, least_stay, stay_from, INT32_MAX);     \
      else ARCKV_WEIGHTS((attn_weights_kernel<DD, MM, false>), 512, 64, 512, least_stay, stay_from, INT32_MAX);        \
    }                                                                                                         \
  } while (0)
  if (head_dim == 64) {
    if (layout == ARCKV_LAYOUT_MX4) ARCKV_WEIGHTS_DM(64, true); else ARCKV_WEIGHTS_DM(64, false);
  } else {
    if (layout == ARCKV_LAYOUT_MX4) ARCKV_WEIGHTS_DM(128, true); else ARCKV_WEIGHTS_DM(128, false);
  }
#undef ARCKV_WEIGHTS_DM
#undef ARCKV_WEIGHTS
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return arckv::fail(ARCKV_EDEVICE, "%s: %s", fn, hipGetErrorString(e));
  return ARCKV_OK;
}
