// Attention of a batch whose requests share long prefixes (part of prefill_attn.hip).
//
// The requests of a group hold the same first P tokens, in the same blocks.  All rows of the group see all of
// them, so the group's rows are the columns of one attention problem over those keys without a mask, and each K/V
// tile is read once for all of them, while a request's own keys [P, L) are its own.  Each part is
// cut into pieces of its keys, and a row's result joins its pieces by their log-sum-exp:
//   o = sum_i 2^(l_i - M) o_i / sum_i 2^(l_i - M),  M = max_i l_i,  o_i = softmax over piece i, l_i its lse.
//
//  * shared_plan_kernel (once a step; the layers share its plan): how many keys the groups share in truth (all
//    their rows must see them; whole tiles of 64), the cuts, and the work items, from lengths on the device.
//  * the shared keys: the attention kernels above, given a group as a request whose rows are those of
//    all its requests and whose length is P + rows, so that every row sees all keys below P.
//  * the own keys: shared_tail_kernel below for decode steps and few rows, the kernels above for more.
//  * shared_join_kernel: the join, and log-sum-exp.
#pragma once

namespace {

constexpr int kTailCols = 16;             // columns of an item of the tail kernel
constexpr int kTailThreads = 256;
constexpr int kTailPerUnit = 4;           // tail work-groups that a compute unit holds at a time
constexpr int kPlanThreads = 1024;
constexpr int kMaxPieceTiles = arckv::kMaxItemKeys / kBK;

// Sizes that the host fixes from the bounds of a batch; the plan's layout in ints.
struct SharedSizes {
  int tile_p, tile_o;                     // columns of an item over shared / own keys
  int64_t items_p, items_o;               // most items of each
  int64_t off_group, off_req, off_row, off_cu, off_len, off_work_p, off_work_o, n_ints;
  int64_t ws_floats;
};
// plan entries of a group / of a request: pieces are [i len, (i + 1) len) tiles of 64 keys from the part's start
struct Part {
  int32_t base, pieces, len, tiles, row0, rows, keys0, keys1;   // first slot; pieces; tiles of a piece; column tiles;
};                                                               // first row; rows; the part's keys [keys0, keys1)
static_assert(sizeof(Part) == 32, "eight ints");

SharedSizes shared_sizes(int64_t n_reqs, int64_t n_groups, int64_t max_q, int64_t max_group_q, int64_t max_new,
                         int64_t bt_stride, int hq, int hkv, int head_dim, int64_t num_cus) {
  SharedSizes z;
  const int64_t G = hq / hkv;
  z.tile_p = max_group_q * G <= arckv::kNarrowCols ? arckv::kNarrowCols : arckv::kWideCols;
  z.tile_o = max_new * G <= kTailCols ? kTailCols : max_new * G <= arckv::kNarrowCols ? arckv::kNarrowCols : arckv::kWideCols;
  const int64_t longest = (bt_stride * 16 + arckv::kMaxItemKeys - 1) / arckv::kMaxItemKeys;   // pieces at least
  auto items = [&](int64_t parts, int64_t cols, int64_t units) {
    const int64_t tiles = (max_q * G / cols + std::min(parts, max_q)) * hkv * std::max<int64_t>(longest, 1);
    return tiles <= units ? units : 2 * tiles;
  };
  z.items_p = n_groups > 0 ? items(n_groups, z.tile_p, num_cus) : 0;
  z.items_o = items(n_reqs, z.tile_o, z.tile_o == kTailCols ? kTailPerUnit * num_cus : num_cus);
  auto per = [](int tile) { return tile == arckv::kNarrowCols ? int64_t{arckv::kListItems} : int64_t{1}; };   // lists of one item
  int64_t at = 16;
  auto take = [&](int64_t n) { const int64_t o = at; at += (n + 15) / 16 * 16; return o; };
  z.off_group = take(n_groups * 8);
  z.off_req = take(n_reqs * 8);
  z.off_row = take(max_q * 2);
  z.off_cu = take(n_reqs + 1);
  z.off_len = take(n_reqs);
  z.off_work_p = take(z.items_p * ARCKV_WORK_INTS * per(z.tile_p));
  z.off_work_o = take(z.items_o * ARCKV_WORK_INTS * per(z.tile_o));
  z.n_ints = at;
  z.ws_floats = (z.items_p * z.tile_p + z.items_o * z.tile_o) * (head_dim + 1);
  return z;
}

// ---- the plan ---------------------------------------------------------------------------------

__device__ __forceinline__ int64_t shfl64(int64_t v, int src) {
  const int lo = __shfl(static_cast<int>(v), src), hi = __shfl(static_cast<int>(v >> 32), src);
  return static_cast<int64_t>(static_cast<uint64_t>(static_cast<uint32_t>(hi)) << 32 | static_cast<uint32_t>(lo));
}

struct PlanShared {
  int64_t wave[kPlanThreads / 64];
  int64_t items[kPlanThreads / 64][64];   // of every candidate cut, by the wave that counted
  int32_t top[kPlanThreads / 64];
  int32_t cap;
};

// Cuts n parts (column tiles and key tiles of part i from `size`) into at most `most` items: a piece has at most cap
// key tiles, where cap is the one of 64 (the longest part in 1, 2, .. 64 pieces) whose rounds of the chip take least: a round
// of `units` items takes its longest piece and `over` key tiles more.
template <class Size>
__device__ __forceinline__ int choose_cap(int n, int64_t most, int units, int min_cap, int over, Size size, PlanShared& sh) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int longest = 0;
  for (int i = tid; i < n; i += kPlanThreads) {
    int tiles, keys;
    size(i, tiles, keys);
    longest = max(longest, tiles > 0 ? keys : 0);
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) longest = max(longest, __shfl_xor(longest, d));
  __syncthreads();
  if (lane == 0) sh.top[wave] = longest;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) longest = max(longest, sh.top[w]);
  const int cap = min(max((longest + lane) / (lane + 1), min_cap), kMaxPieceTiles);
  int64_t items = 0;
  for (int i = wave; i < n; i += kPlanThreads / 64) {
    int tiles, keys;
    size(i, tiles, keys);
    items += static_cast<int64_t>(tiles) * ((keys + cap - 1) / cap);
  }
  sh.items[wave][lane] = items;
  __syncthreads();
  if (wave == 0) {
    items = 0;
    for (int w = 0; w < kPlanThreads / 64; ++w) items += sh.items[w][lane];
    const int64_t rounds = (items + units - 1) / units;
    int64_t cost = items <= most ? rounds * (cap + over) : INT64_MAX / 2;
    int best = lane;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
      const int64_t c = shfl64(cost, lane ^ d);
      const int b = __shfl(best, lane ^ d);
      if (c < cost || (c == cost && b < best)) {
        cost = c;
        best = b;
      }
    }
    const int chosen = __shfl(cap, best);
    if (lane == 0) sh.cap = chosen;
  }
  __syncthreads();
  return sh.cap;
}

// Exclusive sums over the threads of the work-group, and the total.
__device__ __forceinline__ int64_t sums_before(int64_t v, int64_t& total, PlanShared& sh) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t s = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t u = shfl64(s, max(lane - d, 0));
    if (lane >= d) s += u;
  }
  __syncthreads();
  if (lane == 63) sh.wave[wave] = s;
  __syncthreads();
  int64_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    if (w == wave) before = all;
    all += sh.wave[w];
  }
  total = all;
  return before + s - v;
}

// Pieces and slots of the parts, then their work items: item of part i, piece p, column tile c, head h at slot
// base + (p tiles + c) heads + h, so that items of the same keys lie `heads` apart (with 8 heads on one XCD).
template <class ReqOf>
__device__ void emit_items(Part* parts, int n, int cap, int hkv, int tile_cols, int per, Work* work, int64_t most, ReqOf req_of,
                           PlanShared& sh) {
  const int tid = threadIdx.x;
  int64_t at = 0;
  for (int i0 = 0; i0 < n; i0 += kPlanThreads) {
    const int i = i0 + tid;
    int64_t mine = 0, total;
    Part p = {};
    if (i < n) {
      p = parts[i];
      const int keys = p.tiles > 0 ? (p.keys1 - p.keys0 + kBK - 1) / kBK : 0;
      p.pieces = keys > 0 ? (keys + cap - 1) / cap : 0;
      p.len = p.pieces > 0 ? (keys + p.pieces - 1) / p.pieces : 0;
      p.pieces = p.pieces > 0 ? (keys + p.len - 1) / p.len : 0;
      mine = static_cast<int64_t>(p.pieces) * p.tiles * hkv;
    }
    const int64_t before = at + sums_before(mine, total, sh);
    if (i < n) {
      p.base = static_cast<int32_t>(min(before, most));
      if (before + mine > most) p.tiles = p.pieces = 0;     // (lengths or groups that pass the bounds: no slot for it)
      parts[i] = p;
    }
    at += total;
  }
  __syncthreads();
  const int64_t live = min(at, most);
  for (int64_t e = tid; e < most; e += kPlanThreads) {
    Work w = {-1, 0, 0, 0, 0, 0, 0, 0};
    if (e < live) {
      int lo = 0, hi = n - 1;               // the last part whose first slot is at most e
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (parts[mid].base <= e) lo = mid; else hi = mid - 1;
      }
      const Part p = parts[lo];
      if (p.tiles > 0) {
        const int k = static_cast<int>(e) - p.base;
        const int piece = k / (hkv * p.tiles);
        w.req = req_of(lo);
        w.kvh = k % hkv;
        w.col_start = k / hkv % p.tiles * tile_cols;
        w.kv_start = p.keys0 + piece * p.len * kBK;
        w.kv_end = min(w.kv_start + p.len * kBK, p.keys1);
        w.slot = static_cast<int32_t>(e);
      }
    }
    work[e * per] = w;
    if (per > 1) work[e * per + 1].req = -1;
  }
}

__global__ __launch_bounds__(kPlanThreads) void shared_plan_kernel(
    const int32_t* __restrict__ group_start, const int32_t* __restrict__ prefix_lens, int n_groups,
    const int32_t* __restrict__ cu_q, const int32_t* __restrict__ seq_lens, int n_reqs, int max_q, int bt_stride, int G,
    int hkv, int num_cus, SharedSizes z, int32_t* __restrict__ plan) {
  __shared__ PlanShared sh;
  const int tid = threadIdx.x;
  auto* groups = reinterpret_cast<Part*>(plan + z.off_group);
  auto* reqs = reinterpret_cast<Part*>(plan + z.off_req);
  auto* row_of = reinterpret_cast<int2*>(plan + z.off_row);
  int32_t* cu = plan + z.off_cu;
  int32_t* len = plan + z.off_len;
  auto row = [&](int r) { return min(max(cu_q[r], 0), max_q); };
  auto start = [&](int g) { return min(max(group_start[g], 0), n_reqs); };
  const int64_t room = static_cast<int64_t>(bt_stride) * 16;
  // ---- the groups' rows, and what they share as far as they say ------------------------------
  for (int g = tid; g < n_groups; g += kPlanThreads) {
    const int r0 = start(g), r1 = max(start(g + 1), r0);
    Part p = {};
    p.row0 = row(r0);
    p.rows = max(row(r1) - p.row0, 0);
    p.pieces = r0;                                     // until the cut: the group's first request
    p.keys1 = static_cast<int32_t>(min(static_cast<int64_t>(max(prefix_lens[g], 0)), room));
    groups[g] = p;
  }
  for (int r = tid; r <= n_reqs; r += kPlanThreads) {  // (entries that no group uses name no rows)
    cu[r] = 0;
    if (r < n_reqs) len[r] = 0;
  }
  __syncthreads();
  // ---- every row of a group has to see all of the shared keys --------------------------------
  // (a request's group is the last that starts at or before it, if it reaches that far)
  for (int r = tid; r < n_reqs; r += kPlanThreads) {
    int g = -1;
    if (n_groups > 0 && start(0) <= r) {
      int lo = 0, hi = n_groups - 1;
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (start(mid) <= r) lo = mid; else hi = mid - 1;
      }
      g = r < start(lo + 1) ? lo : -1;
    }
    const int L = max(seq_lens[r], 0), q0 = row(r), S = max(row(r + 1) - q0, 0);
    if (g >= 0 && S > 0) atomicMin(&groups[g].keys1, max(L - S, 0));
    Part p = {};
    p.row0 = q0;
    p.rows = S;
    p.keys1 = static_cast<int32_t>(min(static_cast<int64_t>(L), room));
    p.base = g;                                        // until the cut: the request's group
    reqs[r] = p;
  }
  __syncthreads();
  for (int g = tid; g < n_groups; g += kPlanThreads) {
    const int shared = __hip_atomic_load(&groups[g].keys1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) / kBK * kBK;
    Part& p = groups[g];
    p.tiles = shared > 0 ? static_cast<int>((static_cast<int64_t>(p.rows) * G + z.tile_p - 1) / z.tile_p) : 0;
    p.len = shared;
    if (p.tiles > 0) {                                 // the group as a request of the kernels above
      cu[p.pieces] = p.row0;
      cu[p.pieces + 1] = p.row0 + p.rows;
      len[p.pieces] = shared + p.rows;
    }
  }
  __syncthreads();
  for (int r = tid; r < n_reqs; r += kPlanThreads) {
    Part& p = reqs[r];
    const int g = p.base;
    p.keys0 = g >= 0 && p.rows > 0 ? groups[g].len : 0;
    p.tiles = p.keys1 > p.keys0 ? static_cast<int>((static_cast<int64_t>(p.rows) * G + z.tile_o - 1) / z.tile_o) : 0;
    for (int i = 0; i < p.rows; ++i) row_of[p.row0 + i] = make_int2(r, g);
  }
  __syncthreads();
  for (int g = tid; g < n_groups; g += kPlanThreads) groups[g].keys1 = groups[g].len;
  __syncthreads();
  // ---- the cuts and the items ------------------------------------------------------------------
  auto sizes = [&](const Part* parts) {
    return [=](int i, int& tiles, int& keys) {
      tiles = parts[i].tiles * hkv;
      keys = (parts[i].keys1 - parts[i].keys0 + kBK - 1) / kBK;
    };
  };
  auto per = [](int tile) { return tile == arckv::kNarrowCols ? arckv::kListItems : 1; };
  if (n_groups > 0) {
    const int cap = choose_cap(n_groups, z.items_p, num_cus, z.tile_p == arckv::kWideCols ? 8 : 4, 6, sizes(groups), sh);
    emit_items(groups, n_groups, cap, hkv, z.tile_p, per(z.tile_p), reinterpret_cast<Work*>(plan + z.off_work_p), z.items_p,
               [&](int g) { return start(g); }, sh);
  }
  const bool tail = z.tile_o == kTailCols;
  const int cap = choose_cap(n_reqs, z.items_o, tail ? kTailPerUnit * num_cus : num_cus, tail ? 4 : z.tile_o == arckv::kWideCols ? 8 : 4,
                             6, sizes(reqs), sh);
  emit_items(reqs, n_reqs, cap, hkv, z.tile_o, per(z.tile_o), reinterpret_cast<Work*>(plan + z.off_work_o), z.items_o,
             [](int r) { return r; }, sh);
}

// ---- the own keys of decode steps --------------------------------------------------------------
// An item is up to 16 columns (token x head of one KV group) of a request over a range of keys.  Too few columns to share
// a tile: K and V go from memory straight into the operands of v_mfma_f32_16x16x32_bf16, 32 keys a step, four waves taking
// every fourth step, and nothing passes through LDS but the waves' results at the end.  What bounds it is the
// bytes of K and V, and the chain of waits (item, lengths, table, keys) of items of a few steps; four work-groups share a
// compute unit.
//   S^T (16 keys x 16 columns, twice): lane (i = l % 16, g = l / 16) holds row i's dims 32 k + 8 g ..; row i of
//   product m is key 8 (i / 4) + 4 m + i % 4, so that the lane's results, rows 4 g + e, are the keys 8 g + 4 m + e
//   of its column: the eight keys that it holds as the operand of P.V.
//   O^T (16 dims x 16 columns): lane's V operand is dim 16 d + i, keys 8 g ..: 16 bytes of the dim-major block.
template <int D, int G>
__global__ __launch_bounds__(kTailThreads, 3) void shared_tail_kernel(
    const uint16_t* __restrict__ k_pool, const uint16_t* __restrict__ v_pool, const uint16_t* __restrict__ q,
    const int32_t* __restrict__ block_tables, int bt_stride, const int32_t* __restrict__ cu_q,
    const int32_t* __restrict__ seq_lens, int n_reqs, const Work* __restrict__ work, int64_t n_q, int64_t num_blocks, int hq,
    int hkv, float scale_log2, float* __restrict__ ws_o, float* __restrict__ ws_lse, int64_t ws_slots) {
  typedef float acc4 __attribute__((ext_vector_type(4)));
  constexpr int KS = D / 32, DM = D / 16, kWaves = kTailThreads / 64;
  constexpr int PO = D + 4;                               // a column's row of the waves' results (floats)
  __shared__ __attribute__((aligned(16))) float part_o[kWaves][kTailCols][PO];
  __shared__ float part_m[kWaves][kTailCols], part_l[kWaves][kTailCols];
  const Work w = work[blockIdx.x];
  if (w.req < 0 || w.req >= n_reqs || w.kvh < 0 || w.kvh >= hkv || w.col_start < 0 || w.slot < 0 || w.slot >= ws_slots) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i16 = lane & 15, g4 = lane >> 4;
  const int32_t* bt = block_tables + static_cast<int64_t>(w.req) * bt_stride;
  const int q0 = cu_q[w.req], S = cu_q[w.req + 1] - q0, L = seq_lens[w.req];
  const int P = L - S, ncols = S * G, held = min(L, bt_stride * 16);
  const int col = w.col_start + i16, tok = col / G;
  const bool cval = col < ncols && q0 + tok < n_q;
  const int pos = cval ? P + tok : -1;
  const int last_tok = (min(w.col_start + kTailCols, ncols) - 1) / G;
  const int kv_lo = max(w.kv_start, 0), kv_hi = min(min(w.kv_end, P + last_tok + 1), held);
  const int min_pos = P + w.col_start / G;
  const int steps = kv_hi > kv_lo ? (kv_hi - kv_lo + 31) / 32 : 0;
  const int nblk = (held + 15) >> 4;
  const uint32_t nb32 = static_cast<uint32_t>(min(num_blocks, static_cast<int64_t>(INT32_MAX)));
  const int64_t blk_stride = static_cast<int64_t>(hkv) * 16 * D;
  const int64_t head = static_cast<int64_t>(w.kvh) * 16 * D;

  bf16x8_t qf[KS];
  {
    const int64_t at = cval ? (static_cast<int64_t>(q0 + tok) * hq + w.kvh * G + col % G) * D : 0;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      u32x4_t v;
      __builtin_memcpy(&v, q + at + 32 * ks + 8 * g4, 16);
      qf[ks] = cval ? __builtin_bit_cast(bf16x8_t, v) : bf16x8_t{};
    }
  }
  auto block_of = [&](int b) -> int64_t {                 // (uniform)
    const int32_t ph = b < nblk ? bt[b] : 0;
    ARCKV_CHECK_WAVE(ph < 0 || ph >= num_blocks, ARCKV_CHECK_BLOCK);
    return (static_cast<uint32_t>(ph) >= nb32 ? 0 : ph) * blk_stride + head;
  };
  acc4 o[DM];
#pragma unroll
  for (int d = 0; d < DM; ++d) o[d] = acc4{};
  float m_run = -INFINITY, l_run = 0.f;
  for (int s = wave; s < steps; s += kWaves) {
    const int k0 = kv_lo + 32 * s;
    const int64_t b0 = block_of(k0 >> 4), b1 = block_of((k0 >> 4) + 1);
    bf16x8_t kf[2][KS], vf[DM];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const int key = 8 * (i16 >> 2) + 4 * m + (i16 & 3);
      const uint16_t* src = k_pool + (i16 >= 8 ? b1 : b0) + (key & 15) * D + 8 * g4;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) kf[m][ks] = *reinterpret_cast<const bf16x8_t*>(src + 32 * ks);
    }
    {
      const uint16_t* src = v_pool + (g4 >= 2 ? b1 : b0) + i16 * 16 + 8 * (g4 & 1);
#pragma unroll
      for (int d = 0; d < DM; ++d) vf[d] = *reinterpret_cast<const bf16x8_t*>(src + d * 256);
    }
    acc4 sc[2] = {acc4{}, acc4{}};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int m = 0; m < 2; ++m) sc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[m][ks], qf[ks], sc[m], 0, 0, 0);
    const int key0 = k0 + 8 * g4;
    if (k0 + 31 > min_pos || k0 + 32 > kv_hi) {           // (uniform) keys that some column does not see
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (key0 + j > pos || key0 + j >= kv_hi) sc[j / 4][j % 4] = -INFINITY;
    }
    if (k0 + 32 > held) {                                 // past the request's end the block may hold anything, NaN too
#pragma unroll
      for (int d = 0; d < DM; ++d) {
        u32x4_t v = __builtin_bit_cast(u32x4_t, vf[d]);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          v[j] = key0 + 2 * j >= held ? 0 : key0 + 2 * j + 1 >= held ? v[j] & 0xFFFFu : v[j];
        vf[d] = __builtin_bit_cast(bf16x8_t, v);
      }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int j = 0; j < 8; ++j) mx = fmaxf(mx, sc[j / 4][j % 4]);
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = max_halves(mx) * scale_log2;
    const float m_new = fmaxf(m_run, mx);
    const float mu = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = m_run == -INFINITY ? 0.f : fast_exp2(m_run - m_new);
    m_run = m_new;
    float p[8], sum = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      p[j] = fast_exp2(fmaf(sc[j / 4][j % 4], scale_log2, -mu));
      sum += p[j];
    }
    l_run = l_run * alpha + sum;
    // probabilities enter P.V as bf16 (off by at most 2^-8 of themselves); the sum is of the unrounded ones
    u32x4_t pw;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      pw[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{p[2 * j], p[2 * j + 1]}, bf16x2_t));
#pragma unroll
    for (int d = 0; d < DM; ++d) {
      o[d] *= alpha;
      o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[d], __builtin_bit_cast(bf16x8_t, pw), o[d], 0, 0, 0);
    }
  }
  // ---- the waves' results: lane holds dims 16 d + 4 g .. + 3 of its column ---------------------
  l_run += __shfl_xor(l_run, 16);
  l_run = sum_halves(l_run);
#pragma unroll
  for (int d = 0; d < DM; ++d) *reinterpret_cast<acc4*>(&part_o[wave][i16][16 * d + 4 * g4]) = o[d];
  if (g4 == 0) {
    part_m[wave][i16] = m_run;
    part_l[wave][i16] = l_run;
  }
  __syncthreads();
  constexpr int kPer = kTailCols * (D / 4) / kTailThreads;   // float4 of a thread
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int e = tid + k * kTailThreads, c = e / (D / 4), d4 = e % (D / 4);
    float m = -INFINITY;
#pragma unroll
    for (int v = 0; v < kWaves; ++v) m = fmaxf(m, part_m[v][c]);
    float l = 0.f;
    acc4 sum = {};
#pragma unroll
    for (int v = 0; v < kWaves; ++v) {
      const float a = part_m[v][c] == -INFINITY ? 0.f : fast_exp2(part_m[v][c] - m);
      l += a * part_l[v][c];
      sum += a * *reinterpret_cast<const acc4*>(&part_o[v][c][4 * d4]);
    }
    const int at = w.col_start + c;
    if (at >= ncols || q0 + at / G >= n_q) continue;
    const float inv = l > 0.f ? 1.f / l : 0.f;
    *reinterpret_cast<acc4*>(ws_o + (static_cast<int64_t>(w.slot) * kTailCols + c) * D + 4 * d4) = sum * inv;
    if (d4 == 0) ws_lse[static_cast<int64_t>(w.slot) * kTailCols + c] = l > 0.f ? m + __log2f(l) : l == 0.f ? -INFINITY : l;
  }
}

// ---- the join ------------------------------------------------------------------------------------
// D / 4 lanes have a row and head, four dims each.  Its pieces are first those over shared keys, then its own; their lse come in
// 16 at a time (a lane each), the pieces four at a time.  What bounds it is reading the partial results (fp32).
template <int D>
__global__ __launch_bounds__(256) void shared_join_kernel(uint16_t* __restrict__ out, float* __restrict__ lse_out,
                                                          const int32_t* __restrict__ plan, SharedSizes z,
                                                          const int32_t* __restrict__ cu_q, int n_reqs, int n_groups,
                                                          int64_t n_q, int hq, int hkv, int G, const float* __restrict__ ws_op,
                                                          const float* __restrict__ ws_lp, const float* __restrict__ ws_oo,
                                                          const float* __restrict__ ws_lo) {
  typedef float acc4 __attribute__((ext_vector_type(4)));
  constexpr int kLanes = D / 4, kRows = 256 / kLanes, kBatch = 16;
  const int64_t pair = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / kLanes;
  const int64_t t = pair / hq;
  const int h = static_cast<int>(pair % hq), kvh = h / G, d4 = threadIdx.x % kLanes;
  const int total = min(static_cast<int64_t>(max(cu_q[n_reqs], 0)), n_q);
  if (t >= total) return;
  const int2 of = reinterpret_cast<const int2*>(plan + z.off_row)[t];
  auto part = [&](int64_t off, int i, int n) {
    const Part p = i >= 0 && i < n ? reinterpret_cast<const Part*>(plan + off)[i] : Part{};
    return t >= p.row0 && t - p.row0 < p.rows ? p : Part{};
  };
  const Part pg = part(z.off_group, of.y, n_groups), pr = part(z.off_req, of.x, n_reqs);
  // row `col` of slot `base + (piece tiles + tile) hkv + kvh`
  auto place = [&](const Part& p, int tile_cols, int piece) -> int64_t {
    const int64_t c = (t - p.row0) * G + h % G;
    const int64_t tile = c / tile_cols;
    return (p.base + (static_cast<int64_t>(piece) * p.tiles + tile) * hkv + kvh) * tile_cols + c % tile_cols;
  };
  const int np = pg.tiles > 0 ? pg.pieces : 0, n = np + (pr.tiles > 0 ? pr.pieces : 0);
  const int64_t p0 = place(pg, z.tile_p, 0), ps = static_cast<int64_t>(pg.tiles) * hkv * z.tile_p;
  const int64_t r0 = place(pr, z.tile_o, 0), rs = static_cast<int64_t>(pr.tiles) * hkv * z.tile_o;
  float m = -INFINITY, sum = 0.f;
  acc4 acc = {};
  const int sub = threadIdx.x % kBatch;
  for (int i0 = 0; i0 < n; i0 += kBatch) {
    const int i = i0 + sub;
    float l = -INFINITY;
    if (i < n) l = i < np ? ws_lp[p0 + i * ps] : ws_lo[r0 + (i - np) * rs];
    float top = l;
#pragma unroll
    for (int d = kBatch / 2; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    const float m_new = fmaxf(m, top);
    const float mu = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = m == -INFINITY ? 0.f : fast_exp2(m - mu);
    const float wt = l == -INFINITY ? 0.f : fast_exp2(l - mu);
    m = m_new;
    sum *= alpha;
    acc *= alpha;
    const int nb = min(kBatch, n - i0);
    const int first = (threadIdx.x & 63) / kBatch * kBatch;
#pragma unroll 4
    for (int k = 0; k < nb; ++k) {
      const int j = i0 + k;
      const float* src = j < np ? ws_op + (p0 + j * ps) * D : ws_oo + (r0 + (j - np) * rs) * D;
      const float a = __shfl(wt, first + k);
      sum += a;
      acc += a * *reinterpret_cast<const acc4*>(src + 4 * d4);
    }
  }
  const float inv = sum > 0.f ? 1.f / sum : 0.f;
  store_out<true>(out + (t * hq + h) * D + 4 * d4, __builtin_convertvector(acc * inv, bf16x4_t));
  if (lse_out != nullptr && d4 == 0)
    lse_out[t * hq + h] = sum > 0.f ? (m + __log2f(sum)) * kLn2 : sum == 0.f ? -INFINITY : sum;
}

// What the three calls check of the bounds that they share.
int32_t check_shared(const char* fn, int32_t n_reqs, int32_t n_groups, int64_t max_q, int64_t max_group_q, int64_t max_new,
                     int32_t bt_stride, int32_t hq, int32_t hkv, int32_t head_dim, int32_t num_cus) {
  if (n_reqs < 0 || n_reqs > (1 << 20) || n_groups < 0 || n_groups > std::max(n_reqs, 1) || max_q < 0 || max_q > (1 << 24) ||
      max_group_q < 0 || max_group_q > max_q || max_new < 0 || max_new > max_q || bt_stride < 0 || bt_stride > (1 << 26) ||
      hq < 1 || hkv < 1 || hq % hkv != 0 || num_cus < 1 || num_cus > (1 << 16))
    return arckv::fail(ARCKV_EINVAL, "%s: bad sizes", fn);
  if (head_dim != 64 && head_dim != 128)
    return arckv::fail(ARCKV_EUNSUPPORTED, "%s: head_dim %d not in {64,128}", fn, head_dim);
  const int G = hq / hkv;
  if (G != 1 && G != 2 && G != 4 && G != 5 && G != 8)
    return arckv::fail(ARCKV_EUNSUPPORTED, "%s: group size %d not in {1,2,4,5,8}", fn, G);
  const SharedSizes z = shared_sizes(n_reqs, n_groups, max_q, max_group_q, max_new, bt_stride, hq, hkv, head_dim, num_cus);
  if (z.items_p > INT32_MAX / 512 || z.items_o > INT32_MAX / 512 || max_q * hq > INT32_MAX)
    return arckv::fail(ARCKV_EINVAL, "%s: a batch of %lld rows and %d requests needs too many work items", fn,
                       (long long)max_q, n_reqs);
  return ARCKV_OK;
}

}  // namespace

extern "C" int32_t arckv_shared_prefix_sizes(int32_t n_reqs, int32_t n_groups, int64_t max_q, int64_t max_group_q,
                                             int64_t max_new, int32_t bt_stride, int32_t num_q_heads, int32_t num_kv_heads,
                                             int32_t head_dim, int32_t num_cus, int64_t* plan_ints, int64_t* ws_bytes) {
  const int32_t rc = check_shared("shared_prefix_sizes", n_reqs, n_groups, max_q, max_group_q, max_new, bt_stride, num_q_heads,
                                  num_kv_heads, head_dim, num_cus);
  if (rc != ARCKV_OK) return rc;
  if (plan_ints == nullptr || ws_bytes == nullptr) return arckv::fail(ARCKV_EINVAL, "shared_prefix_sizes: NULL output");
  const SharedSizes z = shared_sizes(n_reqs, n_groups, max_q, max_group_q, max_new, bt_stride, num_q_heads, num_kv_heads,
                                     head_dim, num_cus);
  *plan_ints = z.n_ints;
  *ws_bytes = z.ws_floats * static_cast<int64_t>(sizeof(float));
  return ARCKV_OK;
}

extern "C" int32_t arckv_shared_prefix_plan(const int32_t* group_start, const int32_t* prefix_lens, int32_t n_groups,
                                            const int32_t* cu_q, const int32_t* seq_lens, int32_t n_reqs, int64_t max_q,
                                            int64_t max_group_q, int64_t max_new, int32_t bt_stride, int32_t num_q_heads,
                                            int32_t num_kv_heads, int32_t head_dim, int32_t num_cus, int32_t* plan,
                                            int64_t plan_ints, void* stream) {
  const int32_t rc = check_shared("shared_prefix_plan", n_reqs, n_groups, max_q, max_group_q, max_new, bt_stride, num_q_heads,
                                  num_kv_heads, head_dim, num_cus);
  if (rc != ARCKV_OK) return rc;
  if (n_reqs == 0 || max_q == 0) return ARCKV_OK;
  if (cu_q == nullptr || seq_lens == nullptr || plan == nullptr ||
      (n_groups > 0 && (group_start == nullptr || prefix_lens == nullptr)))
    return arckv::fail(ARCKV_EINVAL, "shared_prefix_plan: NULL pointer");
  if (reinterpret_cast<uintptr_t>(plan) % 16 != 0)
    return arckv::fail(ARCKV_EINVAL, "shared_prefix_plan: the plan must be 16-byte aligned");
  const SharedSizes z = shared_sizes(n_reqs, n_groups, max_q, max_group_q, max_new, bt_stride, num_q_heads, num_kv_heads,
                                     head_dim, num_cus);
  if (plan_ints < z.n_ints)
    return arckv::fail(ARCKV_ENOSPC, "shared_prefix_plan: %lld ints, and the plan needs %lld", (long long)plan_ints,
                       (long long)z.n_ints);
  hipLaunchKernelGGL(shared_plan_kernel, dim3(1), dim3(kPlanThreads), 0, static_cast<hipStream_t>(stream), group_start,
                     prefix_lens, n_groups, cu_q, seq_lens, n_reqs, static_cast<int>(max_q), bt_stride,
                     num_q_heads / num_kv_heads, num_kv_heads, num_cus, z, plan);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return arckv::fail(ARCKV_EDEVICE, "shared_prefix_plan: %s", hipGetErrorString(e));
  return ARCKV_OK;
}

extern "C" int32_t arckv_shared_prefix_attention(
    const void* k_pool, const void* v_pool, const void* q, void* out, float* lse, const int32_t* block_tables,
    int32_t bt_stride, const int32_t* cu_q, const int32_t* seq_lens, int32_t n_reqs, int32_t n_groups, int64_t max_q,
    int64_t max_group_q, int64_t max_new, int64_t num_blocks, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
    int32_t num_cus, float scale, const int32_t* plan, void* workspace, int64_t ws_bytes, void* stream) {
  const char* fn = "shared_prefix_attention";
  const int32_t rc = check_shared(fn, n_reqs, n_groups, max_q, max_group_q, max_new, bt_stride, num_q_heads, num_kv_heads,
                                  head_dim, num_cus);
  if (rc != ARCKV_OK) return rc;
  if (num_blocks < 1 || num_blocks > (int64_t{1} << 27) || !std::isfinite(scale) || scale <= 0.f)
    return arckv::fail(ARCKV_EINVAL, "%s: num_blocks %lld, scale %g", fn, (long long)num_blocks, static_cast<double>(scale));
  if (n_reqs == 0 || max_q == 0) return ARCKV_OK;
  if (k_pool == nullptr || v_pool == nullptr || q == nullptr || out == nullptr || block_tables == nullptr || cu_q == nullptr ||
      seq_lens == nullptr || plan == nullptr || workspace == nullptr)
    return arckv::fail(ARCKV_EINVAL, "%s: NULL pointer", fn);
  for (const void* p : {k_pool, v_pool, static_cast<const void*>(plan), static_cast<const void*>(workspace)})
    if (reinterpret_cast<uintptr_t>(p) % 16 != 0)
      return arckv::fail(ARCKV_EINVAL, "%s: pools, plan and workspace must be 16-byte aligned", fn);
  const SharedSizes z = shared_sizes(n_reqs, n_groups, max_q, max_group_q, max_new, bt_stride, num_q_heads, num_kv_heads,
                                     head_dim, num_cus);
  if (ws_bytes < z.ws_floats * static_cast<int64_t>(sizeof(float)))
    return arckv::fail(ARCKV_ENOSPC, "%s: workspace %lld bytes < %lld", fn, (long long)ws_bytes,
                       (long long)(z.ws_floats * sizeof(float)));
  auto* st = static_cast<hipStream_t>(stream);
  auto* kp = static_cast<const uint16_t*>(k_pool);
  auto* vp = static_cast<const uint16_t*>(v_pool);
  auto* qp = static_cast<const uint16_t*>(q);
  auto* op = static_cast<uint16_t*>(out);
  const float scale_log2 = scale * 1.4426950408889634f;
  const bool any_align = (reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out)) % 16 != 0;
  float* ws_op = static_cast<float*>(workspace);
  float* ws_oo = ws_op + z.items_p * z.tile_p * head_dim;
  float* ws_lp = ws_oo + z.items_o * z.tile_o * head_dim;
  float* ws_lo = ws_lp + z.items_p * z.tile_p;
  const int G = num_q_heads / num_kv_heads;
  auto go = [&](auto d_tag, auto g_tag) {
    constexpr int D = decltype(d_tag)::value, GG = decltype(g_tag)::value;
    // items over the keys of (cu, len): shared keys by the groups' rows, own keys by the requests'
    auto part = [&](int tile, int64_t items, const int32_t* work, const int32_t* cu, const int32_t* len, float* wo, float* wl) {
      auto* wk = reinterpret_cast<const Work*>(work);
      const dim3 grid(static_cast<unsigned>(items));
      if (tile == kTailCols)
        hipLaunchKernelGGL((shared_tail_kernel<D, GG>), grid, dim3(kTailThreads), 0, st, kp, vp, qp, block_tables, bt_stride, cu,
                           len, n_reqs, wk, max_q, num_blocks, num_q_heads, num_kv_heads, scale_log2, wo, wl, items);
      else if (tile == arckv::kWideCols && any_align)
        hipLaunchKernelGGL((prefill_attn_pp_kernel<D, GG, false, true>), grid, dim3(512), 0, st, kp, vp, qp, op, block_tables,
                           bt_stride, cu, len, n_reqs, wk, max_q, num_blocks, num_q_heads, num_kv_heads, scale_log2, wo, wl,
                           items, static_cast<float*>(nullptr));
      else if (tile == arckv::kWideCols)
        hipLaunchKernelGGL((prefill_attn_pp_kernel<D, GG, false, false>), grid, dim3(512), 0, st, kp, vp, qp, op, block_tables,
                           bt_stride, cu, len, n_reqs, wk, max_q, num_blocks, num_q_heads, num_kv_heads, scale_log2, wo, wl,
                           items, static_cast<float*>(nullptr));
      else if (any_align)
        hipLaunchKernelGGL((prefill_attn_list_kernel<D, GG, true>), grid, dim3(512), 0, st, kp, vp, qp, op, block_tables,
                           bt_stride, cu, len, n_reqs, wk, max_q, num_blocks, num_q_heads, num_kv_heads, scale_log2, wo, wl,
                           items, static_cast<float*>(nullptr));
      else
        hipLaunchKernelGGL((prefill_attn_list_kernel<D, GG, false>), grid, dim3(512), 0, st, kp, vp, qp, op, block_tables,
                           bt_stride, cu, len, n_reqs, wk, max_q, num_blocks, num_q_heads, num_kv_heads, scale_log2, wo, wl,
                           items, static_cast<float*>(nullptr));
    };
    if (z.items_p > 0) part(z.tile_p, z.items_p, plan + z.off_work_p, plan + z.off_cu, plan + z.off_len, ws_op, ws_lp);
    part(z.tile_o, z.items_o, plan + z.off_work_o, cu_q, seq_lens, ws_oo, ws_lo);
    constexpr int kRows = 256 / (D / 4);
    const int64_t pairs = max_q * num_q_heads;
    hipLaunchKernelGGL(shared_join_kernel<D>, dim3(static_cast<unsigned>((pairs + kRows - 1) / kRows)), dim3(256), 0, st, op, lse,
                       plan, z, cu_q, n_reqs, n_groups, max_q, num_q_heads, num_kv_heads, GG, ws_op, ws_lp, ws_oo, ws_lo);
  };
  auto with_g = [&](auto d_tag) {
    switch (G) {
      case 1: go(d_tag, std::integral_constant<int, 1>{}); break;
      case 2: go(d_tag, std::integral_constant<int, 2>{}); break;
      case 4: go(d_tag, std::integral_constant<int, 4>{}); break;
      case 5: go(d_tag, std::integral_constant<int, 5>{}); break;
      default: go(d_tag, std::integral_constant<int, 8>{}); break;
    }
  };
  if (head_dim == 64) with_g(std::integral_constant<int, 64>{}); else with_g(std::integral_constant<int, 128>{});
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return arckv::fail(ARCKV_EDEVICE, "%s: %s", fn, hipGetErrorString(e));
  return ARCKV_OK;
}
