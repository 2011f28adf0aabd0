// K/V rows into the 4-bit paged pool and back (part of kv_scatter.hip).
//
// kv_scatter_mx4: pool[slot[t]] <- the codes and scales of (k_new[t], v_new[t]).  Four neighbouring
// lanes hold a group's 32 values, 8 each: the largest magnitude is one packed maximum and two
// lane exchanges away, and every load is 16 bytes of a row.  Of many tokens a work-group takes 64: 8 of
// them whose slots are the 8 of half a block (most of a prefill, wherever a request starts in the
// batch) send their V codes through LDS and out as 32 bytes a thread, transposed from 4 pairs of 8
// tokens; the others, and the tokens of a small batch, which spread over more work-groups, store single
// bytes.
// kv_gather_mx4: the rows of `slots` as bf16.  A thread takes 8 tokens; where their slots follow each
// other (through at most one end of half a block) it reads V as pieces of 32 bytes and transposes.
// What bounds both is memory: 4 D bytes of rows per token and head against 17 / 16 D of codes.  24576 tokens of 8
// heads of 128, in runs: 25.6 and 25.7 us, 4.95 TB/s (a byte or a token at a time: 39.6 and 33.3).
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
  ARCKV_CHECK_LANE(s != -1 && !(s >= 0 && s < n_slots), ARCKV_CHECK_SLOT);        // -1 names no slot
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

// dwords of four tokens, byte p for pair p -> dwords of four pairs, byte t for token t (and back)
__device__ __forceinline__ void transpose4(uint32_t (&x)[4]) {
  const uint32_t a = __builtin_amdgcn_perm(x[1], x[0], 0x05010400u), b = __builtin_amdgcn_perm(x[1], x[0], 0x07030602u);
  const uint32_t c = __builtin_amdgcn_perm(x[3], x[2], 0x05010400u), d = __builtin_amdgcn_perm(x[3], x[2], 0x07030602u);
  x[0] = __builtin_amdgcn_perm(c, a, 0x05040100u);
  x[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
  x[2] = __builtin_amdgcn_perm(d, b, 0x05040100u);
  x[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}

typedef uint32_t mx4_u32x4 __attribute__((ext_vector_type(4)));

template <int D>
__global__ __launch_bounds__(kMx4Threads) void kv_scatter_mx4_runs_kernel(
    uint8_t* __restrict__ pool, const uint16_t* __restrict__ k_new, const uint16_t* __restrict__ v_new,
    const int32_t* __restrict__ slots, int64_t n_tokens, int64_t n_slots, int hkv) {
  using L = mx4::Layout<D>;
  constexpr int CH = D / 8, kTokens = 64, kPer = kMx4Threads / CH, N = kTokens / kPer, kG = L::kGroups;
  __shared__ uint32_t vbuf[kTokens][CH + 1];
  __shared__ uint8_t ksb[kTokens][kG], vsb[kTokens][kG];
  __shared__ int32_t sslot[kTokens], run_tok[kTokens / 8], run_slot[kTokens / 8];
  __shared__ uint64_t covered;                      // bit t: token t belongs to a run
  __shared__ int n_runs;
  const int h = blockIdx.y, tid = threadIdx.x, c = tid % CH;
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * kTokens;
  mx4_u32x4 kr[N], vr[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {                     // past the last token its row again, not used
    const int64_t t = min(t0 + i * kPer + tid / CH, n_tokens - 1);
    const int64_t src = (t * hkv + h) * D + c * 8;
    kr[i] = __builtin_nontemporal_load(reinterpret_cast<const mx4_u32x4*>(k_new + src));
    vr[i] = __builtin_nontemporal_load(reinterpret_cast<const mx4_u32x4*>(v_new + src));
  }
  if (tid < kTokens) {
    const int64_t t = t0 + tid;
    const int32_t s = t < n_tokens ? slots[t] : -1;
    const bool ok = s >= 0 && s < n_slots;
    ARCKV_CHECK_LANE(s != -1 && !ok, ARCKV_CHECK_SLOT);
    sslot[tid] = ok ? s : -1;
  }
  __syncthreads();
  if (tid < kTokens) {                              // wave 0: the runs
    const int32_t s = sslot[tid];
    bool start = s >= 0 && (s & 7) == 0 && tid + 7 < kTokens;
    for (int j = 1; j < 8 && start; ++j) start = sslot[tid + j] == s + j;
    const uint64_t m = __builtin_amdgcn_ballot_w64(start);
    if (start) {
      const int r = __builtin_popcountll(m & ((1ull << tid) - 1));   // runs never overlap
      run_tok[r] = tid;
      run_slot[r] = s;
    }
    if (tid == 0) {
      uint64_t all = 0;
      for (int j = 0; j < 8; ++j) all |= m << j;
      covered = all;
      n_runs = __builtin_popcountll(m);
    }
  }
  auto block = [&](int32_t s) { return pool + (static_cast<int64_t>(s >> 4) * hkv + h) * L::kBytes; };
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int tl = i * kPer + tid / CH;
    const uint32_t k[4] = {kr[i][0], kr[i][1], kr[i][2], kr[i][3]}, v[4] = {vr[i][0], vr[i][1], vr[i][2], vr[i][3]};
    const uint32_t kb = mx4::scale_byte(mx4::group_top(k)), vb = mx4::scale_byte(mx4::group_top(v));
    const uint32_t kc = mx4::encode8(k, mx4::scale_value(kb));
    vbuf[tl][c] = mx4::encode8(v, mx4::scale_value(vb));
    if (c % 4 == 0) {
      ksb[tl][c / 4] = static_cast<uint8_t>(kb);
      vsb[tl][c / 4] = static_cast<uint8_t>(vb);
    }
    const int32_t s = sslot[tl];
    if (s >= 0) *reinterpret_cast<uint32_t*>(block(s) + (s & 15) * L::kRow + c * 4) = kc;
  }
  __syncthreads();
  const int nr = n_runs;
  const uint64_t in_run = covered;
  for (int e = tid; e < nr * CH; e += kMx4Threads) {           // V codes of the runs: 4 pairs of 8 tokens
    const int r = e / CH, ch = e % CH, tl = run_tok[r];
    const int32_t s = run_slot[r];
    uint32_t a[4], b[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      a[j] = vbuf[tl + j][ch];
      b[j] = vbuf[tl + 4 + j][ch];
    }
    transpose4(a);
    transpose4(b);
    auto* to = reinterpret_cast<mx4_u32x4*>(block(s) + L::kV + ((s & 15) >> 3) * L::kHalf + ch * 32);
    to[0] = mx4_u32x4{a[0], b[0], a[1], b[1]};
    to[1] = mx4_u32x4{a[2], b[2], a[3], b[3]};
  }
  for (int e = tid; e < nr * kG; e += kMx4Threads) {           // their V scales: a group of 8 tokens
    const int r = e / kG, g = e % kG, tl = run_tok[r];
    const int32_t s = run_slot[r];
    uint32_t x[2] = {0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j / 4] |= static_cast<uint32_t>(vsb[tl + j][g]) << (8 * (j % 4));
    *reinterpret_cast<uint2*>(block(s) + L::kVScale + g * 16 + (s & 8)) = uint2{x[0], x[1]};
  }
  for (int e = tid; e < kTokens * kG; e += kMx4Threads) {      // K scales, and V scales of the other tokens
    const int tl = e / kG, g = e % kG;
    const int32_t s = sslot[tl];
    if (s < 0) continue;
    block(s)[L::kKScale + (s & 15) * kG + g] = ksb[tl][g];
    if (!((in_run >> tl) & 1)) block(s)[L::kVScale + g * 16 + (s & 15)] = vsb[tl][g];
  }
  for (int e = tid; e < kTokens * CH; e += kMx4Threads) {      // V codes of the other tokens, byte by byte
    const int tl = e / CH, ch = e % CH;
    const int32_t s = sslot[tl];
    if (s < 0 || ((in_run >> tl) & 1)) continue;
    const uint32_t v = vbuf[tl][ch];
    uint8_t* vp = block(s) + L::kV + ((s & 15) >> 3) * L::kHalf + ch * 32 + (s & 7);
#pragma unroll
    for (int i = 0; i < 4; ++i) vp[8 * i] = static_cast<uint8_t>(v >> (8 * i));
  }
}

template <int D, int TOK>
__global__ __launch_bounds__(kMx4Threads) void kv_gather_mx4_kernel(
    const uint8_t* __restrict__ pool, uint16_t* __restrict__ k_out, uint16_t* __restrict__ v_out,
    const int32_t* __restrict__ slots, int64_t n_tokens, int64_t n_slots, int hkv) {
  using L = mx4::Layout<D>;
  constexpr int CH = D / 8;
  const int h = blockIdx.y, c = threadIdx.x % CH;
  const int64_t t0 = (static_cast<int64_t>(blockIdx.x) * (kMx4Threads / CH) + threadIdx.x / CH) * TOK;
  if (t0 >= n_tokens) return;
  const int n = static_cast<int>(min(n_tokens - t0, static_cast<int64_t>(TOK)));
  int32_t s[TOK];
  const uint8_t* blk[TOK];
#pragma unroll
  for (int j = 0; j < TOK; ++j) {
    const int32_t x = j < n ? slots[t0 + j] : -1;
    const bool ok = x >= 0 && x < n_slots;
    ARCKV_CHECK_LANE(j < n && !ok, ARCKV_CHECK_SLOT);
    s[j] = ok ? x : -1;
    blk[j] = pool + (static_cast<int64_t>(max(s[j], 0) >> 4) * hkv + h) * L::kBytes;
  }
  uint32_t kc[TOK], vc[TOK], kb[TOK], vb[TOK];
#pragma unroll
  for (int j = 0; j < TOK; ++j) {
    const int tt = s[j] & 15;
    kc[j] = s[j] >= 0 ? *reinterpret_cast<const uint32_t*>(blk[j] + tt * L::kRow + c * 4) : 0;
    kb[j] = s[j] >= 0 ? blk[j][L::kKScale + tt * L::kGroups + c / 4] : 0;
    vb[j] = s[j] >= 0 ? blk[j][L::kVScale + (c / 4) * 16 + tt] : 0;
  }
  // 8 tokens through at most one end of half a block: `a` of them are the last of the first half
  bool run = TOK == 8 && n == TOK;
  int a = 8;
  if constexpr (TOK == 8) {
    a = 8 - (s[0] & 7);
    run = run && s[0] >= 0;
#pragma unroll
    for (int j = 1; j < 8; ++j) run = run && s[j] >= 0 && (j == a ? (s[j] & 7) == 0 : s[j] == s[j - 1] + 1);
  }
  if (run) {
    if constexpr (TOK == 8) {
      auto half = [&](int j, uint32_t (&x)[8]) {
        const uint8_t* p = blk[j] + L::kV + ((s[j] & 15) >> 3) * L::kHalf + c * 32;
        __builtin_memcpy(x, __builtin_assume_aligned(p, 16), 32);
      };
      uint32_t x[8], y[8];
      half(0, x);
      half(7, y);                                   // the same half where a is 8
      // pair p: bytes 8 - a .. of the 16 that (x, y) hold, 8 of them
      uint32_t lo[4], hi[4];
      const int sh = 8 * (8 - a);                   // 0 .. 56
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        const uint64_t f = static_cast<uint64_t>(x[2 * p + 1]) << 32 | x[2 * p];
        const uint64_t g = static_cast<uint64_t>(y[2 * p + 1]) << 32 | y[2 * p];
        const uint64_t v = f >> sh | (sh == 0 ? 0 : g << (64 - sh));
        lo[p] = static_cast<uint32_t>(v);
        hi[p] = static_cast<uint32_t>(v >> 32);
      }
      transpose4(lo);
      transpose4(hi);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        vc[j] = lo[j];
        vc[4 + j] = hi[j];
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < TOK; ++j) {
      const uint8_t* vp = blk[j] + L::kV + ((s[j] & 15) >> 3) * L::kHalf + c * 32 + (s[j] & 7);
      vc[j] = s[j] < 0 ? 0 : vp[0] | vp[8] << 8 | vp[16] << 16 | static_cast<uint32_t>(vp[24]) << 24;
    }
  }
#pragma unroll
  for (int j = 0; j < TOK; ++j) {
    if (j >= n) break;
    const float ks = mx4::scale_value(kb[j]), vs = mx4::scale_value(vb[j]);
    mx4_u32x4 k{}, v{};
    if (s[j] >= 0) {
      k = mx4_u32x4{mx4::decode2<0>(kc[j], ks), mx4::decode2<1>(kc[j], ks), mx4::decode2<2>(kc[j], ks), mx4::decode2<3>(kc[j], ks)};
      v = mx4_u32x4{mx4::decode2<0>(vc[j], vs), mx4::decode2<1>(vc[j], vs), mx4::decode2<2>(vc[j], vs), mx4::decode2<3>(vc[j], vs)};
    }
    const int64_t dst = ((t0 + j) * hkv + h) * D + c * 8;
    *reinterpret_cast<mx4_u32x4*>(k_out + dst) = k;
    *reinterpret_cast<mx4_u32x4*>(v_out + dst) = v;
  }
}

// Whether there is enough to store or gather for the kernels that take runs of 8 tokens at a time: fewer work-groups,
// each with a longer chain of waits.  Alone and in runs, us (store; gather), 8 heads of 128: 1024 tokens 3.4 and
// 4.8; 3.9 and 5.6; 4096 6.6 and 6.6; 8.3 and 7.8; 8192 12.6 and 10.4; 14.0 and 10.8; 16384 22.0 and 16.2; 23.9 and
// 17.3.  16 heads of 64: 4096 5.5 and 6.1; 6.4 and 7.7; 8192 9.4 and 8.5; 10.7 and 10.9.
// (16384 tokens whose slots do not follow each other: 30.8 and 38.7; 25.6 and 30.3.)
bool many_mx4_rows(int64_t n_tokens, int32_t hkv, int32_t head_dim) { return n_tokens * hkv * head_dim > 1 << 22; }

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
  const bool runs = many_mx4_rows(n_tokens, num_kv_heads, head_dim);
  const int per = runs ? 64 : kMx4Threads / (head_dim / 8);
  const dim3 grid(static_cast<unsigned>((n_tokens + per - 1) / per), num_kv_heads);
  auto* s = static_cast<hipStream_t>(stream);
#define ARCKV_SCATTER_MX4(KERNEL)                                                                            \
  hipLaunchKernelGGL((KERNEL), grid, dim3(kMx4Threads), 0, s, static_cast<uint8_t*>(kv_pool),                \
                     static_cast<const uint16_t*>(k_new), static_cast<const uint16_t*>(v_new), slot_mapping, \
                     n_tokens, num_blocks * 16, num_kv_heads)
  if (head_dim == 64) {
    if (runs) ARCKV_SCATTER_MX4(kv_scatter_mx4_runs_kernel<64>); else ARCKV_SCATTER_MX4(kv_scatter_mx4_kernel<64>);
  } else {
    if (runs) ARCKV_SCATTER_MX4(kv_scatter_mx4_runs_kernel<128>); else ARCKV_SCATTER_MX4(kv_scatter_mx4_kernel<128>);
  }
#undef ARCKV_SCATTER_MX4
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
  const int tok = many_mx4_rows(n_tokens, num_kv_heads, head_dim) ? 8 : 1;      // tokens of a thread
  const int per = kMx4Threads / (head_dim / 8) * tok;
  const dim3 grid(static_cast<unsigned>((n_tokens + per - 1) / per), num_kv_heads);
  auto* s = static_cast<hipStream_t>(stream);
#define ARCKV_GATHER_MX4(DD, TT)                                                                              \
  hipLaunchKernelGGL((kv_gather_mx4_kernel<DD, TT>), grid, dim3(kMx4Threads), 0, s,                           \
                     static_cast<const uint8_t*>(kv_pool), static_cast<uint16_t*>(k_out),                     \
                     static_cast<uint16_t*>(v_out), slot_mapping, n_tokens, num_blocks * 16, num_kv_heads)
  if (head_dim == 64) {
    if (tok == 8) ARCKV_GATHER_MX4(64, 8); else ARCKV_GATHER_MX4(64, 1);
  } else {
    if (tok == 8) ARCKV_GATHER_MX4(128, 8); else ARCKV_GATHER_MX4(128, 1);
  }
#undef ARCKV_GATHER_MX4
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return arckv::fail(ARCKV_EDEVICE, "kv_gather_mx4: %s", hipGetErrorString(e));
  return ARCKV_OK;
}
