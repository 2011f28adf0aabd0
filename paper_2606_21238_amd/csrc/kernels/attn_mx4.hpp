// Prefix-cached paged attention over the 4-bit cache (part of prefill_attn.hip: work items,
// combine and column packing are those of the bf16 kernels).
//
//   o = softmax(scale * q . K^T) V over keys 0..position, K and V as the 4-bit pool stands for
//
// Narrow tiles, here: a wave takes 16 or 32 query columns of an item and its keys in chunks of 32, straight
// from the pool into registers: S^T = K . Q^T and O^T = V^T . P^T with v_mfma_f32_16x16x32_bf16, codes turned
// into bf16 (exactly) as operands.  Which keys and dimensions feed which operand row is chosen so
// that nothing is exchanged between lanes: lane (m, q4) = (lane % 16, lane / 16) holds
//   K row i of tile t in {0, 1}: key 8 (i / 4) + 4 t + i % 4 of the chunk, dimensions [q4 D/4, (q4 + 1) D/4);
//   S^T registers: keys 8 q4 + 4 t + r of column m, eight in a row, which is the B operand of P.V;
//   V^T row m of tile 4 j + i: dimension 64 j + 4 m + i, keys [8 q4, 8 q4 + 8);
//   O^T registers: dimensions 64 j + 16 q4 + 4 r + i of column m, 16 in a row.
//
// Probabilities enter P.V as bf16, the matrix unit's type, each off by at most 2^-8 of itself; O, the maxima and the sums
// (of the unrounded probabilities) are fp32.  That leaves outputs 0.0023 of their root mean square off the 64-bit ones, and
// rounding the output alone 0.0017; P as a sum of two bf16 parts would take the second products again.
//
// What bounds it is the pool's bytes, 17 / 64 of the bf16 kernel's: one new token of each of 64 requests of
// 2000 (32 / 8 heads of 128) 33.8 us, 4.15 TB/s with the launch, of 8192 128.5 us, 4.45 TB/s, where a large copy
// reaches 4.74; the bf16 kernel's decode takes 2.6 times as long at lognormal histories.  Small calls take the launch and a chain of
// round trips (list, lengths, table, codes, join): 8 requests of 400 10 us.
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

// The raw bytes of the chunk whose two blocks are at bytes at[0], at[1] of `pool` (block 0 of the KV head).
template <int D>
__device__ __forceinline__ void mx4_load(const uint8_t* pool, const int64_t (&at)[2], int lane, Mx4Raw<D>& raw) {
  using L = mx4::Layout<D>;
  const int m = lane & 15, q4 = lane >> 4;
  const uint8_t* kb = pool + (m >> 3 ? at[1] : at[0]);
  const uint8_t* vb = pool + (q4 >> 1 ? at[1] : at[0]);
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
  static constexpr int NJ = D / 64, DT = D / 16, KS = D / 32, kTiles = NT;
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
template <int D, int NT>
__device__ __forceinline__ void mx4_chunk(Mx4State<D, NT>& st, Mx4Raw<D>& raw, int key0, int lane, int len,
                                          float scale_log2, bool first, bool masked) {
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
    if (masked) {                                      // wave-uniform
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) s[n][t][r] = key0 + 8 * q4 + 4 * t + r > st.pos[n] ? -INFINITY : s[n][t][r];
    }
    // exponentials against the running maximum first: they are >= 0, so a lane whose sum is within
    // 2^kLazy has every term within it, and the maximum may stay (a common factor costs neither precision nor
    // range, in bf16 or fp32)
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
  if (masked) mx4_mask_v<D, NT>(st, raw, key0, lane, len);
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

// Narrow tiles: a work-group of 8 waves takes the list of kListItems items that the plan gave it.
//
// Lists whose items have at most 16 columns (decode): the items' chunks, one after the other, are cut
// into 8 equal runs, one for each wave, wherever the items end.  A wave keeps the bytes of three
// chunks in flight, across items too, and nothing waits for another wave until all are done: a
// wave's part of an item (at most 15 parts on a list) goes to LDS as (m, l, O), and one barrier later
// all threads join the parts.  (By item after item, as below: 41.3 instead of 33.8 us for 64 requests of
// 2000, 56 instead of 43 at 16 / 16 heads of 64.)
// Other lists: item after item, 32 columns for a wave, 8, 4 or 2 waves to the same columns, each with
// its run of the item's chunks, joined the same way.
struct Mx4Item {
  int req, kvh, col, slot, q0, ncols, P, len, kv_lo, n_chunks, first_chunk, min_pos;
};

template <int D>
__global__ __launch_bounds__(512) void mx4_attn_list_kernel(
    const uint8_t* __restrict__ pool, const uint16_t* __restrict__ q, uint16_t* __restrict__ out,
    float* __restrict__ lse_out, const int32_t* __restrict__ block_tables, int bt_stride,
    const int32_t* __restrict__ cu_q, const int32_t* __restrict__ seq_lens, int n_reqs,
    const Work* __restrict__ work, int64_t n_q, int64_t num_blocks, int hq, int hkv, GroupDiv gd, float scale_log2,
    float* __restrict__ ws_o, float* __restrict__ ws_lse, int64_t ws_slots) {
  constexpr int kCols = arckv::kNarrowCols, kItems = arckv::kListItems, kWaves = 8;
  constexpr int kPitch = D + 4;                      // floats of a row of parts: 16 columns, 16 bank groups
  __shared__ __attribute__((aligned(16))) float part_o[256 * kPitch];
  __shared__ float part_m[256], part_l[256];
  __shared__ Mx4Item items[kItems];
  const int tid = threadIdx.x, lane = tid & 63, m16 = lane & 15, q4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = static_cast<int>(gd.g);

  // ---- the list: entries up to the first idle one; an entry naming nothing of the batch has no columns ------
  {
    const Work w = work[static_cast<int64_t>(blockIdx.x) * kItems + (lane & 7)];
    const uint64_t idle = __builtin_amdgcn_ballot_w64(lane < kItems && w.req < 0);
    const bool live = (idle & ((2ull << (lane & 7)) - 1)) == 0;
    const bool bad = w.req >= n_reqs || w.kvh < 0 || w.kvh >= hkv || w.col_start < 0;
    ARCKV_CHECK_LANE(wave == 0 && lane < kItems && live && bad, ARCKV_CHECK_WORK);
    const bool ok = live && !bad;
    Mx4Item it{};
    if (ok) {
      it.req = w.req;
      it.kvh = w.kvh;
      it.col = w.col_start;
      it.slot = w.slot;
      it.q0 = cu_q[w.req];
      const int S = cu_q[w.req + 1] - it.q0;
      it.len = seq_lens[w.req];
      it.P = it.len - S;
      it.ncols = S * G;
      it.kv_lo = max(w.kv_start, 0);
      const int last = min(w.col_start + kCols, it.ncols) - 1;
      const int kv_hi = min(w.kv_end, it.P + gd.tok(max(last, 0)) + 1);
      it.n_chunks = last >= w.col_start && kv_hi > it.kv_lo ? (kv_hi - it.kv_lo + kMx4Chunk - 1) / kMx4Chunk : 0;
      it.min_pos = it.P + gd.tok(it.col);
    }
    int upto = it.n_chunks;
#pragma unroll
    for (int s = 1; s < kItems; s <<= 1) {
      const int x = __shfl_up(upto, s);
      if ((lane & 7) >= s) upto += x;
    }
    it.first_chunk = upto - it.n_chunks;
    if (tid < kItems) items[tid] = it;
  }
  __syncthreads();
  const int total = items[kItems - 1].first_chunk + items[kItems - 1].n_chunks;
  int most = 0;                                      // columns of the widest item
#pragma unroll
  for (int i = 0; i < kItems; ++i) most = max(most, min(items[i].ncols - items[i].col, kCols));
  if (most <= 0) return;
  const uint32_t nb32 = static_cast<uint32_t>(num_blocks);
  const int64_t blk_stride = static_cast<int64_t>(hkv) * mx4::Layout<D>::kBytes;

  // ---- a wave's run of chunks: its item, its place, and the two blocks of the chunk to load next ------------
  struct Cursor {
    int item, chunk, left, nblk;                     // chunk: of the item's key range; left: of the run
    const cint32* bt;
    const uint8_t* head;
    int32_t ph[2];
  };
  auto open = [&](Cursor& c, int i) {                // uniform: an item of the list
    c.item = i;
    const int req = __builtin_amdgcn_readfirstlane(items[i].req), len = __builtin_amdgcn_readfirstlane(items[i].len);
    c.bt = (const cint32*)(block_tables) + static_cast<int64_t>(req) * bt_stride +
           __builtin_amdgcn_readfirstlane(items[i].kv_lo) / 16;
    c.nblk = min((len + 15) >> 4, bt_stride) - __builtin_amdgcn_readfirstlane(items[i].kv_lo) / 16;
    c.head = pool + static_cast<int64_t>(__builtin_amdgcn_readfirstlane(items[i].kvh)) * mx4::Layout<D>::kBytes;
  };
  auto blocks = [&](Cursor& c) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int e = 2 * c.chunk + b;
      c.ph[b] = c.left > 0 && e < c.nblk ? c.bt[e] : 0;
    }
  };
  auto chunks_of = [&](int i) { return __builtin_amdgcn_readfirstlane(items[i].n_chunks); };
  auto step = [&](Cursor& c) {                       // on to the next chunk of the run
    --c.left;
    ++c.chunk;
    if (c.left > 0 && c.chunk == chunks_of(c.item)) {
      int i = c.item + 1;
      while (chunks_of(i) == 0) ++i;                 // the run has chunks left: an item follows
      c.chunk = 0;
      open(c, i);
    }
  };
  auto load = [&](Cursor& c, Mx4Raw<D>& raw) {       // the chunk at the cursor, then the cursor moves on
    int64_t at[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      ARCKV_CHECK_WAVE(c.left > 0 && static_cast<uint32_t>(c.ph[b]) >= nb32, ARCKV_CHECK_BLOCK);
      // an entry out of range reads block 0
      at[b] = static_cast<int64_t>(static_cast<uint32_t>(c.ph[b]) >= nb32 ? 0 : c.ph[b]) * blk_stride;
    }
    if (c.left > 0) mx4_load<D>(c.head, at, lane, raw);
    step(c);
    blocks(c);
  };
  auto begin = [&](int from, int to, int i, int chunk) {   // `to - from` chunks from chunk `chunk` of item i
    Cursor c{};
    c.left = to - from;
    c.chunk = chunk;
    open(c, i);
    blocks(c);
    return c;
  };
  // this lane's columns of an item: queries and positions
  auto take = [&](auto& st, int i, int col0) {
    using S = std::remove_reference_t<decltype(st)>;
    st.reset();
#pragma unroll
    for (int n = 0; n < S::kTiles; ++n) {
      const int col = items[i].col + col0 + 16 * n + m16, tok = gd.tok(col);
      const bool cval = col < items[i].ncols && items[i].q0 + tok < n_q;
      const int64_t row = cval ? static_cast<int64_t>(items[i].q0 + tok) * hq + items[i].kvh * G + (col - tok * G) : 0;
      st.pos[n] = cval ? items[i].P + tok : -1;
#pragma unroll
      for (int s = 0; s < S::KS; ++s) {
        bf16x8_t x{};
        if (cval) __builtin_memcpy(&x, q + row * D + q4 * (D / 4) + 8 * s, 16);
        st.q[n][s] = x;
      }
    }
  };
  // a wave's part of an item into rows row .. of the parts
  auto leave = [&](auto& st, int row) {
    using S = std::remove_reference_t<decltype(st)>;
#pragma unroll
    for (int n = 0; n < S::kTiles; ++n) {
      const int r0 = row + 16 * n + m16;
      const float l = sum_halves(st.l[n] + __shfl_xor(st.l[n], 16));
#pragma unroll
      for (int j = 0; j < S::NJ; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          f32x4_t v;
#pragma unroll
          for (int t = 0; t < 4; ++t) v[t] = st.nan_key[j] <= st.pos[n] ? __builtin_nanf("") : st.o[n][4 * j + t][r];
          *reinterpret_cast<f32x4_t*>(part_o + r0 * kPitch + 64 * j + 16 * q4 + 4 * r) = v;
        }
      if (q4 == 0) {
        part_m[r0] = st.m[n];
        part_l[r0] = l;
      }
    }
  };
  // joins the parts of column c of item i, four dimensions a thread: parts k in [k0, k1) are at rows
  // row + step * k, and is(k) says which of them there are
  auto join = [&](int i, int c, int d, int row, int step_rows, int k0, int k1, auto is) {
    const Mx4Item& it = items[i];
    const int col = it.col + c, tok = gd.tok(col);
    if (col >= it.ncols || it.q0 + tok >= n_q) return;
    float m = -INFINITY;
    for (int k = k0; k < k1; ++k)
      if (is(k)) m = fmaxf(m, part_m[row + step_rows * k]);
    f32x4_t o{};
    float l = 0.f;
    for (int k = k0; k < k1; ++k) {
      if (!is(k)) continue;
      const int r = row + step_rows * k;
      const float a = part_m[r] == -INFINITY ? 0.f : fast_exp2(part_m[r] - m);
      // (a part without a visible key has l = 0 and O = 0, a NaN one stays)
      l += a * part_l[r];
      o += a * *reinterpret_cast<const f32x4_t*>(part_o + r * kPitch + d);
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    const float lse = l > 0.f ? m + __log2f(l) : l == 0.f ? -INFINITY : l;
    o *= inv;
    const int64_t orow = static_cast<int64_t>(it.q0 + tok) * hq + it.kvh * G + (col - tok * G);
    if (it.slot < 0) {
      store_out<true>(out + orow * D + d, __builtin_convertvector(o, bf16x4_t));
      if (d == 0 && lse_out != nullptr) lse_out[orow] = lse * kLn2;
    } else if (it.slot < ws_slots) {
      const int64_t prow = static_cast<int64_t>(it.slot) * kCols + c;
      *reinterpret_cast<f32x4_t*>(ws_o + prow * D + d) = o;
      if (d == 0) ws_lse[prow] = lse;
    }
  };

  if (most <= 16) {
    // ---- decode: 8 equal runs over the whole list --------------------------------------------------------------
    const int from = total * wave / kWaves, to = total * (wave + 1) / kWaves;
    if (to > from) {
      int i = 0;
      while (items[i].first_chunk + items[i].n_chunks <= from) ++i;
      i = __builtin_amdgcn_readfirstlane(i);
      const int chunk0 = from - __builtin_amdgcn_readfirstlane(items[i].first_chunk);
      Cursor ld = begin(from, to, i, chunk0);
      Mx4Raw<D> raw[3];
      load(ld, raw[0]);
      load(ld, raw[1]);
      load(ld, raw[2]);
      Mx4State<D, 1> st;
      take(st, i, 0);
      int chunk = chunk0, n = chunks_of(i), left = to - from;
      bool fresh = true;
      int kv_lo = __builtin_amdgcn_readfirstlane(items[i].kv_lo), min_pos = __builtin_amdgcn_readfirstlane(items[i].min_pos);
      auto one = [&](Mx4Raw<D>& x) {
        const int key0 = kv_lo + chunk * kMx4Chunk;
        mx4_chunk<D, 1>(st, x, key0, lane, items[i].len, scale_log2, fresh, key0 + kMx4Chunk - 1 > min_pos);
        fresh = false;
        load(ld, x);
        ++chunk;
        if (--left == 0) {
          leave(st, (wave + i) * 16);
          return false;
        }
        if (chunk == n) {                            // the item ends inside the run
          leave(st, (wave + i) * 16);
          do ++i; while (chunks_of(i) == 0);
          take(st, i, 0);
          chunk = 0;
          n = chunks_of(i);
          kv_lo = __builtin_amdgcn_readfirstlane(items[i].kv_lo);
          min_pos = __builtin_amdgcn_readfirstlane(items[i].min_pos);
          fresh = true;
        }
        return true;
      };
      while (one(raw[0]) && one(raw[1]) && one(raw[2])) {}
    }
    __syncthreads();
    for (int e = tid; e < kItems * 16 * (D / 4); e += 512) {
      const int i = e / (16 * (D / 4)), c = e / (D / 4) % 16, d = 4 * (e % (D / 4));
      const int a = items[i].first_chunk, b = a + items[i].n_chunks;
      join(i, c, d, i * 16 + c, 16, 0, kWaves, [&](int w) {
        return max(total * w / kWaves, a) < min(total * (w + 1) / kWaves, b);
      });
    }
    return;
  }
  // ---- item after item: CW x 32 columns, 8 / CW runs of the item's chunks -----------------------------------------
  for (int i = 0; i < kItems; ++i) {
    const int cols = __builtin_amdgcn_readfirstlane(min(items[i].ncols - items[i].col, kCols)), n = chunks_of(i);
    if (cols <= 0) continue;
    const int CW = cols <= 32 ? 1 : cols <= 64 ? 2 : 4, KG = kWaves / CW;
    const int cw = wave % CW, kg = wave / CW;
    const int from = n * kg / KG, to = n * (kg + 1) / KG;
    Mx4State<D, 2> st;
    Cursor ld = begin(from, to, i, from);
    Mx4Raw<D> raw[2];
    load(ld, raw[0]);
    load(ld, raw[1]);
    take(st, i, 32 * cw);
    const int kv_lo = __builtin_amdgcn_readfirstlane(items[i].kv_lo), min_pos = __builtin_amdgcn_readfirstlane(items[i].min_pos);
    auto one = [&](int chunk, Mx4Raw<D>& x) {
      const int key0 = kv_lo + chunk * kMx4Chunk;
      mx4_chunk<D, 2>(st, x, key0, lane, items[i].len, scale_log2, chunk == from, key0 + kMx4Chunk - 1 > min_pos);
      load(ld, x);
    };
    int k = from;
    for (; k + 1 < to; k += 2) {
      one(k, raw[0]);
      one(k + 1, raw[1]);
    }
    if (k < to) one(k, raw[0]);
    leave(st, wave * 32);                            // rows (kg CW + cw) 32 ..: CW 32 rows for each run
    __syncthreads();
    for (int e = tid; e < cols * (D / 4); e += 512) {
      const int c = e / (D / 4);
      join(i, c, 4 * (e % (D / 4)), c, CW * 32, 0, KG, [&](int) { return true; });
    }
    __syncthreads();
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
    // where it does not, LDS that nobody uses keeps each on a unit of its own.  Alone and shared, us: 600 on
    // 30000, 64 / 8 heads 483 and 500; 2 turns of 640 on 17008, 32 / 4, 299 and 314; 12 prompts of 1100,
    // 16 / 16, 103 and 80; 2 turns of 2164 on 3920, 197 and 159.
    const unsigned lds = head_dim == 64 && n_work % 2 == 0 ? 32 << 10 : 0;
    const GroupDiv gd{static_cast<uint32_t>(G), G == 1 ? 0 : static_cast<uint32_t>(((1ull << 32) + G - 1) / G)};
#define ARCKV_MX4(KERNEL, GRID, GG, LDS)                                                                           \
  hipLaunchKernelGGL((KERNEL), dim3(static_cast<unsigned>(GRID)), dim3(512), LDS, st, pool, qp, op, lse,        \
                     block_tables, bt_stride, cu_q, seq_lens, n_reqs, wk, n_q, num_blocks, num_q_heads,         \
                     num_kv_heads, GG, scale_log2, ws_o, ws_lse, ws_slots)
    if (tile_cols == arckv::kNarrowCols) {
      if (head_dim == 64) ARCKV_MX4(mx4_attn_list_kernel<64>, n_work / arckv::kListItems, gd, 0);
      else ARCKV_MX4(mx4_attn_list_kernel<128>, n_work / arckv::kListItems, gd, 0);
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
