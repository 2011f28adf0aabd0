// Eviction from the cache by accumulated attention weight (part of kv_scatter.hip).
//
// evict_select: for every (request, KV head), which `keep` of L positions stay: the first n_first,
// the last n_recent, and of the others those of the greatest weight, the lower position first
// among equals.  One work-group finds the weight of the last one to stay by its digits from the
// top, 12, 10 and 10 bits, each from a histogram in LDS (of the keys that share the digits before; 12
// bits first, because 8, the sign and most of the exponent, put most of the keys into a few bins, where
// additions wait for each other: 74 us for 32 rows of 32768, and 26), then writes the kept positions in order.
// What bounds it is that one work-group has a row: its read (128 KB at 32768), three passes of LDS additions
// and the barriers between, 24 to 26 us there; 512 ragged rows of up to 4096, two to a unit: 20 us.
// kv_compact: the kept tokens' K and V into other blocks, position i of the result from position
// kept[i]; a head's tokens move on their own, so the same slot may hold another token for another
// head.  A work-group writes one block (4 bits: four) of one head.  The bound is the lines it reads, not the tokens: a line
// of V is 4 dimensions of a block's 16 tokens (4 bits: 32 dimensions of 8 tokens), and comes in where one of them is kept.
// 64 requests of 192 to 16272 (2600 on average) down to 512, 1 token in 5, 8 heads of 128: four fifths of V's lines, 273 MB
// by that count, beside the kept rows of K, 66: 92 us for the 332 MB that are read and 132 written (5.05 TB/s).
// 4 requests of 32768 down to 4096, 1 in 8, at 4 bits: two thirds of V's lines and a quarter of K's, of which two tokens
// share one: 24.8 us for 66 and 18 MB (3.4 TB/s), gathered byte by byte.
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
__device__ __forceinline__ float key_weight(uint32_t k) {
  return __builtin_bit_cast(float, k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

constexpr int kSelWaves = kSelThreads / 64;

// KEYS: how many keys a thread holds, so rows of up to 1024 KEYS are read once.
template <int KEYS>
__global__ __launch_bounds__(kSelThreads, KEYS > 16 ? 4 : 8) void evict_select_kernel(
    const float* __restrict__ weights, int64_t w_stride, const int32_t* __restrict__ seq_lens, int hkv, int keep,
    int n_first, int n_recent, int32_t* __restrict__ kept, float* __restrict__ kept_weights, int64_t kw_stride) {
  // one histogram for every kCopies-th lane, side by side: fewer lanes of a wave meet at an address or a bank (one for
  // all: 25.0 against 24.3 us for 32 rows of 32768 uniform weights, 26.2 against 25.1 for 1024 of 2600)
  constexpr int kCopies = KEYS > 16 ? 4 : 2;
  __shared__ __attribute__((aligned(16))) int hist[4096][kCopies];
  __shared__ int wave_sum[kSelWaves], wave_take[kSelWaves], wave_equal[kSelWaves];
  __shared__ int pick, above;
  const int tid = threadIdx.x, lane = tid & 63, h = blockIdx.x, r = blockIdx.y;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t seg = static_cast<int64_t>(r) * hkv + h;
  const float* w = weights + seg * w_stride;
  int32_t* out = kept + seg * keep;
  float* kw = kept_weights == nullptr ? nullptr : kept_weights + seg * kw_stride;
  const int len = static_cast<int>(min(static_cast<int64_t>(max(seq_lens[r], 0)), w_stride));
  const int n_kept = min(keep, len);
  const int lo = len <= keep ? 0 : n_first, hi = len <= keep ? 0 : len - n_recent;   // positions that compete
  int need = len <= keep ? 0 : keep - n_first - n_recent;                            // how many of them stay

  // A wave has a run of positions, in tiles of KEYS x 64; the tile in its registers is read again only where
  // a run has several.  Positions past the run have the key 0.
  const int run = (len + kSelWaves * 64 - 1) / (kSelWaves * 64) * 64;
  const int from = min(wave * run, len), to = min(from + run, len);
  constexpr int kTile = KEYS * 64;
  const int tiles = (run + kTile - 1) / kTile;
  uint32_t key[KEYS];
  int have = -1;
  // f(u, i, key) for every position of the wave in order, four at a time past which there is nothing to do
  auto each = [&](auto f) {
    for (int t = 0; t < tiles; ++t) {
      const int i0 = from + t * kTile, n = min(run - t * kTile, kTile);
      if (have != t) {
#pragma unroll
        for (int u = 0; u < KEYS; u += 16) {
          if (64 * u >= n) break;
          float x[16];                     // 16 loads in flight
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            const int i = i0 + 64 * (u + v) + lane;
            x[v] = i < to ? w[i] : 0.f;
          }
#pragma unroll
          for (int v = 0; v < 16; ++v) key[u + v] = i0 + 64 * (u + v) + lane < to ? weight_key(x[v]) : 0;
        }
        have = t;
      }
#pragma unroll
      for (int u = 0; u < KEYS; u += 4) {
        if (64 * u >= n) break;
#pragma unroll
        for (int v = 0; v < 4; ++v) f(i0 + 64 * (u + v) + lane, key[u + v]);
      }
    }
  };

  // Most waves have a run of competing positions only, and need no look at a position.
  const bool inner = from >= lo && from + run <= hi;
  // the key of the last one to stay (its digits from the top), and how many with that very key
  uint32_t prefix = 0xffffffffu;           // nobody competes: no key is greater
  if (need > 0) {
    prefix = 0;
    constexpr int kShift[3] = {20, 10, 0}, kBits[3] = {12, 10, 10};
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = kShift[pass];
      constexpr int kPer = 4096 / kSelThreads;
      const int bins = 1 << kBits[pass];
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (i * kSelThreads < bins)
#pragma unroll
          for (int v = 0; v < kCopies; ++v) hist[i * kSelThreads + tid][v] = 0;
      __syncthreads();
      auto count = [&](uint32_t k) {
        if (pass == 0 || (k >> (shift + kBits[pass])) == (prefix >> (shift + kBits[pass])))
          atomicAdd(&hist[(k >> shift) & (bins - 1)][lane % kCopies], 1);
      };
      // (the key 0 of positions behind an inner run only adds to the lowest digit, where it decides nothing)
      if (inner) each([&](int, uint32_t k) { count(k); });
      else each([&](int i, uint32_t k) { if (i >= lo && i < min(hi, to)) count(k); });
      __syncthreads();
      // the highest digit with at least `need` keys from it up: a thread has `per` of them, thread 0 the highest
      const int per = bins / kSelThreads;    // 4, then 1
      int c[kPer], sum = 0;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        c[i] = 0;
#pragma unroll
        for (int v = 0; v < kCopies; ++v) c[i] += i < per ? hist[bins - 1 - (per * tid + i)][v] : 0;
        sum += c[i];
      }
      int upto = sum;
#pragma unroll
      for (int s = 1; s < 64; s <<= 1) {
        const int x = __shfl_up(upto, s);
        if (lane >= s) upto += x;
      }
      if (lane == 63) wave_sum[wave] = upto;
      __syncthreads();
      int before = upto - sum;
      for (int v = 0; v < wave; ++v) before += wave_sum[v];
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        if (before < need && before + c[i] >= need) {
          pick = bins - 1 - (per * tid + i);
          above = before;
        }
        before += c[i];
      }
      __syncthreads();
      prefix |= static_cast<uint32_t>(pick) << shift;
      need -= above;
    }
  }

  // Positions in order: greater keys, and the first `need` equal ones.  A wave counts its own, learns what the
  // waves before it have, and writes.
  auto classify = [&](int i, uint32_t k, bool& take, bool& eq) {
    const bool held = i < lo || i >= hi;
    take = i < to && (held || k > prefix);
    eq = i < to && !held && need > 0 && k == prefix;
  };
  const bool plain = inner && prefix != 0;   // (prefix 0, a NaN: the key of what is not there)
  int takes = 0, equals = 0;
  if (plain) {
    each([&](int, uint32_t k) {
      takes += __builtin_popcountll(__builtin_amdgcn_ballot_w64(k > prefix));
      equals += __builtin_popcountll(__builtin_amdgcn_ballot_w64(k == prefix));
    });
  } else {
    each([&](int i, uint32_t k) {
      bool take, eq;
      classify(i, k, take, eq);
      takes += __builtin_popcountll(__builtin_amdgcn_ballot_w64(take));
      equals += __builtin_popcountll(__builtin_amdgcn_ballot_w64(eq));
    });
  }
  if (lane == 0) {
    wave_take[wave] = takes;
    wave_equal[wave] = equals;
  }
  __syncthreads();
  int at = 0, equal = 0;                   // of the waves before
  for (int v = 0; v < wave; ++v) {
    at += wave_take[v] + min(wave_equal[v], max(need - equal, 0));
    equal += wave_equal[v];
  }
  auto put = [&](int i, uint32_t k, bool take) {
    const uint64_t all = __builtin_amdgcn_ballot_w64(take);
    if (take) {
      const int dst = at + __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(all >> 32),
                                                     __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(all), 0));
      out[dst] = i;
      if (kw != nullptr) kw[dst] = key_weight(k);
    }
    at += __builtin_popcountll(all);
  };
  if (plain && equals == 0) {
    each([&](int i, uint32_t k) { put(i, k, k > prefix); });
  } else {
    each([&](int i, uint32_t k) {
      bool take, eq;
      classify(i, k, take, eq);
      const uint64_t eqs = __builtin_amdgcn_ballot_w64(eq);
      take |= eq && equal + __builtin_popcountll(eqs & ((1ull << lane) - 1)) < need;
      equal += __builtin_popcountll(eqs);
      put(i, k, take);
    });
  }
  for (int i = n_kept + tid; i < keep; i += kSelThreads) {
    out[i] = -1;
    if (kw != nullptr) kw[i] = 0.f;
  }
}

// Where the 16 N tokens of the destination blocks from b on come from: slot of each, -1 for none.
template <int N>
__device__ __forceinline__ void source_slots(int32_t (&src)[16 * N], const int32_t* kept, int keep, const int32_t* bt,
                                             int bt_stride, int64_t num_blocks, int b) {
  const int i = 16 * b + threadIdx.x;
  if (threadIdx.x < 16 * N) {
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
  source_slots<1>(src, kept + (static_cast<int64_t>(r) * hkv + h) * keep, keep,
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

// A block has few bytes in 4 bits: a work-group takes 4, whose loads are in flight together (one block each:
// 27.5 us for 4 requests of 32768 down to 4096).
constexpr int kMoveBlocks = 4;

template <int D>
__global__ __launch_bounds__(256) void kv_compact_mx4_kernel(
    uint8_t* __restrict__ pool, const int32_t* __restrict__ block_tables, int bt_stride,
    const int32_t* __restrict__ kept, int keep, const int32_t* __restrict__ dst_tables, int dst_stride,
    int64_t num_blocks, int hkv) {
  using L = mx4::Layout<D>;
  constexpr int N = kMoveBlocks, WORDS = D / 8, VN = N * D / 256;
  __shared__ int32_t src[16 * N], dst[N];
  const int b = blockIdx.x / hkv * N, h = blockIdx.x % hkv, r = blockIdx.y, tid = threadIdx.x;
  if (tid >= 64 && tid < 64 + N) {
    const int n = tid - 64;
    const int32_t db = 16 * (b + n) < keep ? dst_tables[static_cast<int64_t>(r) * dst_stride + b + n] : -1;
    dst[n] = db >= 0 && db < num_blocks ? db : -1;
  }
  source_slots<N>(src, kept + (static_cast<int64_t>(r) * hkv + h) * keep, keep,
                  block_tables + static_cast<int64_t>(r) * bt_stride, bt_stride, num_blocks, b);
  ARCKV_CHECK_LANE(tid < N && dst[tid % N] < 0 && src[16 * (tid % N)] >= 0, ARCKV_CHECK_BLOCK);
  auto block = [&](int32_t ph) { return pool + (static_cast<int64_t>(ph) * hkv + h) * L::kBytes; };
  auto from = [&](int32_t s) { return block(s >> 4); };
  // loads: K codes, a word of a token; scales, one of a token and group; V codes, 8 tokens of a pair
  const int kt = tid / WORDS, kc = tid % WORDS;
  uint32_t kw[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int32_t s = tid < 16 * WORDS && dst[n] >= 0 ? src[16 * n + kt % 16] : -1;
    kw[n] = s < 0 ? 0 : *reinterpret_cast<const uint32_t*>(from(s) + (s & 15) * L::kRow + 4 * kc);
  }
  const int sn = tid / (16 * L::kGroups), st = tid % 16, sg = tid / 16 % L::kGroups;
  const int32_t ss = sn < N && dst[sn % N] >= 0 ? src[16 * (sn % N) + st] : -1;
  uint8_t ks = 0, vs = 0;
  if (ss >= 0) {
    ks = from(ss)[L::kKScale + (ss & 15) * L::kGroups + sg];
    vs = from(ss)[L::kVScale + sg * 16 + (ss & 15)];
  }
  uint32_t x[VN][8];
  bool all[VN];
#pragma unroll
  for (int m = 0; m < VN; ++m) {
    const int e = tid + 256 * m, n = e / D, half = e % D / (D / 2), p = e % (D / 2);
    all[m] = true;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int32_t s = dst[n] >= 0 ? src[16 * n + 8 * half + j] : -1;
      all[m] &= s >= 0;
      x[m][j] = s < 0 ? 0 : from(s)[L::kV + ((s & 15) >> 3) * L::kHalf + 8 * p + (s & 7)];
    }
  }
  // stores; slots without a token keep what they hold
#pragma unroll
  for (int n = 0; n < N; ++n)
    if (tid < 16 * WORDS && dst[n] >= 0 && src[16 * n + kt % 16] >= 0)
      *reinterpret_cast<uint32_t*>(block(dst[n]) + kt * L::kRow + 4 * kc) = kw[n];
  if (ss >= 0) {
    uint8_t* to = block(dst[sn % N]);
    to[L::kKScale + st * L::kGroups + sg] = ks;
    to[L::kVScale + sg * 16 + st] = vs;
  }
#pragma unroll
  for (int m = 0; m < VN; ++m) {
    const int e = tid + 256 * m, n = e / D, half = e % D / (D / 2), p = e % (D / 2);
    if (dst[n] < 0) continue;
    uint8_t* at = block(dst[n]) + L::kV + half * L::kHalf + 8 * p;
    if (all[m]) {
      *reinterpret_cast<uint2*>(at) = uint2{x[m][0] | x[m][1] << 8 | x[m][2] << 16 | x[m][3] << 24,
                                            x[m][4] | x[m][5] << 8 | x[m][6] << 16 | x[m][7] << 24};
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (src[16 * n + 8 * half + j] >= 0) at[j] = static_cast<uint8_t>(x[m][j]);
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
  // Keys of a thread: 16, and two work-groups to a unit, which reads rows of more than 16384 again for every pass;
  // 32 for such rows of a batch that leaves a unit to each.  32 and 16, us: 32 rows of 32768 24 and 34, 320 of them
  // 51 and 53; 256 rows of 16384 17.6 and 17.2, 320 of 4096 20 and 14, 1024 of 2600 38 and 25.
  const bool one = w_stride > 16384 && static_cast<int64_t>(n_reqs) * num_kv_heads <= 256;
#define ARCKV_SELECT(KEYS)                                                                                    \
  hipLaunchKernelGGL(evict_select_kernel<KEYS>, dim3(num_kv_heads, n_reqs), dim3(kSelThreads), 0,             \
                     static_cast<hipStream_t>(stream), weights, w_stride, seq_lens, num_kv_heads, keep,       \
                     n_first, n_recent, kept, kept_weights, kw_stride)
  if (one) ARCKV_SELECT(32); else ARCKV_SELECT(16);
#undef ARCKV_SELECT
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
  const dim3 grid(static_cast<unsigned>((static_cast<int64_t>(keep) + 15) / 16) * num_kv_heads, n_reqs);
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
  const int nb = static_cast<int>((static_cast<int64_t>(keep) + 15) / 16);
  const dim3 grid(static_cast<unsigned>((nb + kMoveBlocks - 1) / kMoveBlocks) * num_kv_heads, n_reqs);
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
