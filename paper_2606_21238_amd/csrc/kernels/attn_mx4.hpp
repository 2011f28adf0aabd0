// Prefix-cached paged attention over the 4-bit cache (part of prefill_attn.hip: work items,
// combine and column packing are those of the bf16 kernels).
//
//   o = softmax(scale * q . K^T) V over keys 0..position, K and V as the 4-bit pool stands for
//
// A wave takes 16 query columns of an item and its keys in chunks of 32, straight from the pool
// into registers: S^T = K . Q^T and O^T = V^T . P^T with v_mfma_f32_16x16x32_bf16, codes turned
// into bf16 (exactly) as operands.  Which keys and dimensions feed which operand row is chosen so
// that nothing is exchanged between lanes: lane (m, q4) = (lane % 16, lane / 16) holds
//   K row i of tile t in {0, 1}: key 8 (i / 4) + 4 t + i % 4 of the chunk, dimensions [q4 D/4, (q4 + 1) D/4);
//   S^T registers: keys 8 q4 + 4 t + r of column m, eight in a row, which is the B operand of P.V;
//   V^T row m of tile 4 j + i: dimension 64 j + 4 m + i, keys [8 q4, 8 q4 + 8);
//   O^T registers: dimensions 64 j + 16 q4 + 4 r + i of column m, 16 in a row.
#pragma once

#include "mx4.hpp"
#include "attn_mx4_wide.hpp"

namespace {

constexpr int kMx4Chunk = 32;   // keys of a chunk: two blocks

// Raw bytes of one chunk as a lane holds them.
template <int D>
struct Mx4Raw {
  static constexpr int W = D / 32, NJ = D / 64;
  uint32_t k[2][W], v[NJ][4], vs[NJ][2];
  uint32_t ks[2];
};

// Where a request's K and V are.
struct Mx4Keys {
  const uint8_t* pool;      // of the item's KV head: block 0
  int64_t blk_stride;       // bytes per physical block
  const cint32* bt;         // the request's block table
  int nblk;                 // entries of it that may be used
  uint32_t num_blocks;
};

template <int D>
__device__ __forceinline__ void mx4_load(const Mx4Keys& keys, int chunk, int lane, Mx4Raw<D>& raw) {
  using L = mx4::Layout<D>;
  const int m = lane & 15, q4 = lane >> 4;
  int64_t at[2];
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const int e = 2 * chunk + b;
    const int32_t ph = e < keys.nblk ? keys.bt[e] : 0;
    ARCKV_CHECK_WAVE(e < keys.nblk && static_cast<uint32_t>(ph) >= keys.num_blocks, ARCKV_CHECK_BLOCK);
    // an entry out of range reads block 0
    at[b] = static_cast<int64_t>(static_cast<uint32_t>(ph) >= keys.num_blocks ? 0 : ph) * keys.blk_stride;
  }
  const uint8_t* kb = keys.pool + (m >> 3 ? at[1] : at[0]);
  const uint8_t* vb = keys.pool + (q4 >> 1 ? at[1] : at[0]);
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int tt = 8 * ((m >> 2) & 1) + 4 * t + (m & 3);
    __builtin_memcpy(raw.k[t], __builtin_assume_aligned(kb + tt * L::kRow + q4 * (D / 8), D / 8), D / 8);
    raw.ks[t] = kb[L::kKScale + tt * L::kGroups + q4 * (D / 4) / 32];
  }
#pragma unroll
  for (int j = 0; j < Mx4Raw<D>::NJ; ++j) {
    __builtin_memcpy(raw.v[j], __builtin_assume_aligned(vb + L::kV + (q4 & 1) * L::kHalf + j * 256 + m * 16, 16), 16);
    __builtin_memcpy(raw.vs[j], __builtin_assume_aligned(vb + L::kVScale + (2 * j + (m >> 3)) * 16 + (q4 & 1) * 8, 8), 8);
  }
}

// Online softmax state of a wave: NT tiles of 16 columns.
template <int D, int NT>
struct Mx4State {
  static constexpr int NJ = D / 64, DT = D / 16, KS = D / 32;
  bf16x8_t q[NT][KS];
  f32x4_t o[NT][DT];
  float m[NT], l[NT];
  int pos[NT];             // the lane's query positions (-1: no column)
  int nan_key[NJ];         // first key whose V group of this lane's dimensions is NaN, of those in masked chunks

  __device__ __forceinline__ void reset() {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int t = 0; t < DT; ++t) o[n][t] = f32x4_t{};
      m[n] = -INFINITY;
      l[n] = 0.f;
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j) nan_key[j] = INT32_MAX;
  }
};

// A masked chunk: V of the keys past the request's end may be anything, and V of a key that only
// later columns see may be NaN.  Neither may meet a weight of zero in the product, so their scales
// are replaced; NaN comes back in the end, for the columns that see the first such key.
template <int D, int NT>
__device__ __forceinline__ void mx4_mask_v(Mx4State<D, NT>& st, Mx4Raw<D>& raw, int key0, int lane, int len) {
  const int m = lane & 15, q4 = lane >> 4;
#pragma unroll
  for (int j = 0; j < Mx4State<D, NT>::NJ; ++j) {
    int first = INT32_MAX;
#pragma unroll
    for (int k = 7; k >= 0; --k) {
      const int key = key0 + 8 * q4 + k, sh = 8 * (k & 3);
      uint32_t& w = raw.vs[j][k >> 2];
      const bool nan = ((w >> sh) & 255u) == mx4::kNanScale && key < len;
      first = nan ? key : first;
      if (nan || key >= len) w = (w & ~(255u << sh)) | (127u << sh);
    }
    if (__builtin_amdgcn_ballot_w64(first != INT32_MAX) == 0) continue;
#pragma unroll
    for (int g = 0; g < 2; ++g) {                      // group 2 j + g: of operand rows 8 g.., of lanes q4 / 2 = g
      int x = (m >> 3) == g ? first : INT32_MAX;
#pragma unroll
      for (int s = 1; s < 64; s <<= 1) x = min(x, __shfl_xor(x, s));
      if ((q4 >> 1) == g) st.nan_key[j] = min(st.nan_key[j], x);
    }
  }
}

// One chunk (keys key0 .. key0 + 31): S, softmax, O.
template <int D, int NT, bool MASKED>
__device__ __forceinline__ void mx4_chunk(Mx4State<D, NT>& st, Mx4Raw<D>& raw, int key0, int lane, int len,
                                          float scale_log2, bool first) {
  using S = Mx4State<D, NT>;
  const int q4 = lane >> 4;
  f32x4_t s[NT][2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const float ks = mx4::scale_value(raw.ks[t]);
#pragma unroll
    for (int step = 0; step < S::KS; ++step) {
      const uint32_t c = raw.k[t][step];
      const u32x4_t a = {mx4::decode2<0>(c, ks), mx4::decode2<1>(c, ks), mx4::decode2<2>(c, ks), mx4::decode2<3>(c, ks)};
#pragma unroll
      for (int n = 0; n < NT; ++n)
        s[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), st.q[n][step],
                                                          step == 0 ? f32x4_t{} : s[n][t], 0, 0, 0);
    }
  }
  bf16x8_t p[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    if constexpr (MASKED) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) s[n][t][r] = key0 + 8 * q4 + 4 * t + r > st.pos[n] ? -INFINITY : s[n][t][r];
    }
    // exponentials against the running maximum first: they are >= 0, so a lane whose sum is within
    // 2^kLazy has every term within it, and the maximum may stay (P is rounded to bf16, O and l
    // are fp32: a common factor costs neither precision nor range)
    auto exps = [&](float mu) {
      float sum = 0.f;
      uint32_t w[4];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const f32x2_t two = {fast_exp2(fmaf(s[n][t][2 * h], scale_log2, -mu)),
                               fast_exp2(fmaf(s[n][t][2 * h + 1], scale_log2, -mu))};
          sum += two[0];
          sum += two[1];
          w[2 * t + h] = __builtin_bit_cast(uint32_t, __builtin_convertvector(two, bf16x2_t));
        }
      p[n] = __builtin_bit_cast(bf16x8_t, u32x4_t{w[0], w[1], w[2], w[3]});
      return sum;
    };
    float sum = 0.f;
    bool pending = first;
    if (!first) {
      sum = exps(st.m[n] == -INFINITY ? 0.f : st.m[n]);
      pending = __builtin_amdgcn_ballot_w64(!(sum <= kLazySum)) != 0;   // also catches inf / NaN sums
    }
    if (pending) {
      float mx = -INFINITY;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) mx = fmaxf(mx, s[n][t][r]);
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = max_halves(mx) * scale_log2;
      const float m_new = fmaxf(st.m[n], mx);
      const float alpha = m_new == -INFINITY ? 1.f : fast_exp2(st.m[n] - m_new);
      st.m[n] = m_new;
      st.l[n] *= alpha;
#pragma unroll
      for (int t = 0; t < S::DT; ++t) st.o[n][t] *= alpha;
      sum = exps(m_new == -INFINITY ? 0.f : m_new);
    }
    st.l[n] += sum;
  }
  if constexpr (MASKED) mx4_mask_v<D, NT>(st, raw, key0, lane, len);
#pragma unroll
  for (int j = 0; j < S::NJ; ++j) {
    float vs[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) vs[k] = mx4::scale_value((raw.vs[j][k >> 2] >> (8 * (k & 3))) & 255u);
#pragma unroll
    for (int a = 0; a < 2; ++a) {                      // dimensions 64 j + 4 m + 2 a, + 1
      uint32_t x[8];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t c = raw.v[j][2 * a + h];
        x[4 * h] = mx4::decode2<0>(c, vs[4 * h]);
        x[4 * h + 1] = mx4::decode2<1>(c, vs[4 * h + 1]);
        x[4 * h + 2] = mx4::decode2<2>(c, vs[4 * h + 2]);
        x[4 * h + 3] = mx4::decode2<3>(c, vs[4 * h + 3]);
      }
      u32x4_t lo, hi;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        lo[k] = __builtin_amdgcn_perm(x[2 * k + 1], x[2 * k], 0x05040100u);
        hi[k] = __builtin_amdgcn_perm(x[2 * k + 1], x[2 * k], 0x07060302u);
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        st.o[n][4 * j + 2 * a] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, lo), p[n],
                                                                         st.o[n][4 * j + 2 * a], 0, 0, 0);
        st.o[n][4 * j + 2 * a + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, hi), p[n],
                                                                             st.o[n][4 * j + 2 * a + 1], 0, 0, 0);
      }
    }
  }
}

// Narrow tiles (128 columns): a work-group takes the list of kListItems items, a wave 16 columns.
template <int D>
__global__ __launch_bounds__(512) void mx4_attn_kernel(
    const uint8_t* __restrict__ pool, const uint16_t* __restrict__ q, uint16_t* __restrict__ out,
    float* __restrict__ lse_out, const int32_t* __restrict__ block_tables, int bt_stride,
    const int32_t* __restrict__ cu_q, const int32_t* __restrict__ seq_lens, int n_reqs,
    const Work* __restrict__ work, int64_t n_q, int64_t num_blocks, int hq, int hkv, int G, float scale_log2,
    float* __restrict__ ws_o, float* __restrict__ ws_lse, int64_t ws_slots) {
  using S = Mx4State<D, 1>;
  const int lane = threadIdx.x & 63, m16 = lane & 15, q4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  constexpr int kItems = arckv::kListItems, COLS = arckv::kNarrowCols;
  for (int i = 0; i < kItems; ++i) {
    const Work w = work[static_cast<int64_t>(blockIdx.x) * kItems + i];
    if (w.req < 0) return;                         // the end of the list
    const bool bad = w.req >= n_reqs || w.kvh < 0 || w.kvh >= hkv || w.col_start < 0;
    ARCKV_CHECK_WAVE(bad, ARCKV_CHECK_WORK);
    if (bad) continue;
    const int q0 = cu_q[w.req], qlen = cu_q[w.req + 1] - q0, len = seq_lens[w.req], ncols = qlen * G;
    const int local = wave * 16, c0 = w.col_start + local;
    if (c0 >= ncols) continue;
    const int col = c0 + m16, tok = col / G;
    const bool cval = col < ncols && q0 + tok < n_q;
    const int64_t row = cval ? static_cast<int64_t>(q0 + tok) * hq + w.kvh * G + col % G : 0;
    S st;
    st.reset();
    st.pos[0] = cval ? len - qlen + tok : -1;
#pragma unroll
    for (int s = 0; s < S::KS; ++s) {
      bf16x8_t x{};
      if (cval) __builtin_memcpy(&x, q + row * D + q4 * (D / 4) + 8 * s, 16);
      st.q[0][s] = x;
    }
    const int min_pos = len - qlen + c0 / G, max_pos = len - qlen + (min(c0 + 16, ncols) - 1) / G;
    const int kv_lo = max(w.kv_start, 0), kv_hi = min(w.kv_end, max_pos + 1);
    const Mx4Keys keys{pool + static_cast<int64_t>(w.kvh) * mx4::Layout<D>::kBytes,
                       static_cast<int64_t>(hkv) * mx4::Layout<D>::kBytes,
                       (const cint32*)(block_tables) + static_cast<int64_t>(w.req) * bt_stride,
                       min((len + 15) >> 4, bt_stride), static_cast<uint32_t>(num_blocks)};
    for (int k = kv_lo; k < kv_hi; k += kMx4Chunk) {
      Mx4Raw<D> raw;
      mx4_load<D>(keys, k / kMx4Chunk, lane, raw);
      if (k + kMx4Chunk - 1 > min_pos) mx4_chunk<D, 1, true>(st, raw, k, lane, len, scale_log2, k == kv_lo);
      else mx4_chunk<D, 1, false>(st, raw, k, lane, len, scale_log2, k == kv_lo);
    }
    float l = st.l[0] + __shfl_xor(st.l[0], 16);
    l = sum_halves(l);
    const float inv = l > 0.f ? 1.f / l : 0.f;          // a NaN sum stays NaN in O
    const float lse = l > 0.f ? st.m[0] + __log2f(l) : l == 0.f ? -INFINITY : l;
    if (!cval || (w.slot >= 0 && w.slot >= ws_slots)) continue;
    const int64_t prow = w.slot < 0 ? 0 : static_cast<int64_t>(w.slot) * COLS + local + m16;
#pragma unroll
    for (int j = 0; j < S::NJ; ++j) {
      const float by = st.nan_key[j] <= st.pos[0] ? __builtin_nanf("") : inv;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        f32x4_t v;
#pragma unroll
        for (int t = 0; t < 4; ++t) v[t] = st.o[0][4 * j + t][r] * by;
        const int d = 64 * j + 16 * q4 + 4 * r;
        if (w.slot < 0) store_out<true>(out + row * D + d, __builtin_convertvector(v, bf16x4_t));
        else *reinterpret_cast<f32x4_t*>(ws_o + prow * D + d) = v;
      }
    }
    if (q4 == 0) {
      if (w.slot >= 0) ws_lse[prow] = lse;
      else if (lse_out != nullptr) lse_out[row] = lse * kLn2;
    }
  }
}

}  // namespace

extern "C" int32_t arckv_prefill_attention_mx4(const void* kv_pool, const void* q, void* out, float* lse,
                                               const int32_t* block_tables, int32_t bt_stride, const int32_t* cu_q,
                                               const int32_t* seq_lens, int32_t n_reqs, int64_t n_q,
                                               int64_t num_blocks, const int32_t* work, int64_t n_work,
                                               int64_t n_combine, int32_t tile_cols, int32_t num_q_heads,
                                               int32_t num_kv_heads, int32_t head_dim, float scale, void* workspace,
                                               int64_t ws_bytes, void* stream) {
  const char* fn = "prefill_attention_mx4";
  const int32_t rc = check_attention(fn, n_reqs, n_q, num_blocks, n_work, n_combine, tile_cols, num_q_heads,
                                     num_kv_heads, head_dim, bt_stride, scale, ws_bytes);
  if (rc != ARCKV_OK || (n_work == 0 && n_combine == 0) || n_q == 0) return rc;
  if (kv_pool == nullptr || q == nullptr || out == nullptr || block_tables == nullptr || cu_q == nullptr ||
      seq_lens == nullptr || work == nullptr)
    return arckv::fail(ARCKV_EINVAL, "%s: NULL pointer", fn);
  if (reinterpret_cast<uintptr_t>(kv_pool) % 16 != 0 || reinterpret_cast<uintptr_t>(workspace) % 16 != 0)
    return arckv::fail(ARCKV_EINVAL, "%s: the pool and the workspace must be 16-byte aligned", fn);
  if (num_blocks > (1LL << 27)) return arckv::fail(ARCKV_EINVAL, "%s: num_blocks", fn);
  const int G = num_q_heads / num_kv_heads;
  const int64_t slot_bytes = static_cast<int64_t>(tile_cols) * (head_dim + 1) * 4;
  const int64_t ws_slots = workspace != nullptr ? ws_bytes / slot_bytes : 0;
  if (n_combine > 0 && ws_slots == 0)
    return arckv::fail(ARCKV_EINVAL, "%s: split plan needs a workspace", fn);
  float* ws_o = static_cast<float*>(workspace);
  float* ws_lse = ws_o == nullptr ? nullptr : ws_o + ws_slots * tile_cols * head_dim;
  auto* st = static_cast<hipStream_t>(stream);
  auto* pool = static_cast<const uint8_t*>(kv_pool);
  auto* qp = static_cast<const uint16_t*>(q);
  auto* op = static_cast<uint16_t*>(out);
  auto* wk = reinterpret_cast<const Work*>(work);
  const float scale_log2 = scale * 1.4426950408889634f;
  if (n_work > 0) {
    const bool any = (reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out)) % 16 != 0;
    // head_dim 64: two work-groups share a unit where the plan asks for it (an odd number of entries);
    // where it does not, LDS that nobody uses keeps each on a unit of its own
    const unsigned lds = head_dim == 64 && n_work % 2 == 0 ? 32 << 10 : 0;
    const GroupDiv gd{static_cast<uint32_t>(G), G == 1 ? 0 : static_cast<uint32_t>(((1ull << 32) + G - 1) / G)};
#define ARCKV_MX4(KERNEL, GRID, GG, LDS)                                                                           \
  hipLaunchKernelGGL((KERNEL), dim3(static_cast<unsigned>(GRID)), dim3(512), LDS, st, pool, qp, op, lse,        \
                     block_tables, bt_stride, cu_q, seq_lens, n_reqs, wk, n_q, num_blocks, num_q_heads,         \
                     num_kv_heads, GG, scale_log2, ws_o, ws_lse, ws_slots)
    if (tile_cols == arckv::kNarrowCols) {
      if (head_dim == 64) ARCKV_MX4(mx4_attn_kernel<64>, n_work / arckv::kListItems, G, 0);
      else ARCKV_MX4(mx4_attn_kernel<128>, n_work / arckv::kListItems, G, 0);
    } else if (head_dim == 64) {
      if (any) ARCKV_MX4((mx4_attn_wide_kernel<64, true>), n_work, gd, lds);
      else ARCKV_MX4((mx4_attn_wide_kernel<64, false>), n_work, gd, lds);
    } else {
      if (any) ARCKV_MX4((mx4_attn_wide_kernel<128, true>), n_work, gd, lds);
      else ARCKV_MX4((mx4_attn_wide_kernel<128, false>), n_work, gd, lds);
    }
#undef ARCKV_MX4
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return arckv::fail(ARCKV_EDEVICE, "%s: %s", fn, hipGetErrorString(e));
  }
  return combine_splits(fn, op, lse, wk + n_work, n_combine, cu_q, n_reqs, n_q, num_q_heads, G, head_dim,
                        tile_cols, ws_o, ws_lse, ws_slots, st);
}
