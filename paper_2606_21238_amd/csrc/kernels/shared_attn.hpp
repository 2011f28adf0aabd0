// Attention of a batch whose requests share long prefixes (part of prefill_attn.hip).
//
// The requests of a group hold the same first P tokens, in the same blocks.  All rows of the group see all of
// them, so the group's rows are the columns of one attention problem over those keys without a mask, and each K/V
// tile is read once for all of them, while a request's own keys [P, L) are its own.  Each part is
// cut into pieces of its keys, and a row's result joins its pieces by their log-sum-exp:
//   o = sum_i 2^(l_i - M) o_i / sum_i 2^(l_i - M),  M = max_i l_i,  o_i = softmax over piece i, l_i its lse.
//
//  * shared_plan_kernel (once a step; the layers share its plan): how many keys the groups share in truth (all
//    their rows must see them; whole tiles of 64), the cuts, and the work items, from lengths on the device.  One work-group,
//    a chain of scans and searches: 20 us for 64 requests, 69 for 1000; none for short batches.
//  * the shared keys: the attention kernels above, given a group as a request whose rows are those of
//    all its requests and whose length is P + rows, so that every row sees all keys below P.  8192 tokens of 8 heads of 128
//    for 92 columns (34 MB, narrow tiles) 16 us, of which the stream is 6; 32768 tokens for 184 columns (134 MB, wide tiles) 40
//    us; 8192 tokens for 10240 columns (0.34 PFLOP, wide) 294 us, 1.17 PFLOP/s.
//  * the own keys: shared_tail_kernel below for decode steps and few rows, the kernels above for more.
//  * shared_join_kernel: the join, and log-sum-exp.
// Against the plan that reads every request's keys by itself (the attention call of a planned batch), us: 64 rows on 8192 + 300
// tokens (32 / 8 heads) 42 and 293; 32 on 32768 + 400 (64 / 8) 63 and 565; 96 in 8 groups on 4000 + 500 (40 / 8) 75 and 243; 16 x
// 128 on 8192 (40 / 8) 329 and 367.  Where nothing is shared it costs the join: 64 groups of one, 2048 + 300 tokens, 128 and 116.
#pragma once

namespace {

constexpr int kTailCols = 16;             // columns of an item of the tail kernel
constexpr int kTailPerUnit = 3;           // tail work-groups (of four waves) that a compute unit holds at a time
// Own keys of a request that are not cut: at most this many key steps set the launch's end, and fewer cuts leave fewer rows to
// the join.  us with 512 and 1024: 64 requests of 2000 own tokens 139 and 129, 32 of 900 79 and 73; 2 of 6000 31 and 34.
constexpr int kTailWhole = 1024;
constexpr int kPlanThreads = 1024;
constexpr int kMaxPieceTiles = arckv::kMaxItemKeys / kBK;

// Sizes that the host fixes from the bounds of a batch; the plan's layout in ints.
struct SharedSizes {
  int tile_p, tile_o;                     // columns of an item over shared / own keys
  int64_t items_p, items_o;               // most items of each
  int64_t off_group, off_req, off_row, off_list, off_cu, off_len, off_work_p, off_work_o, n_ints;
  int64_t ws_floats;
};
// Plan entry of a group / of a request.  Its units are (column tile, head) pairs, head fastest; the first `whole` of them
// have pieces_w pieces of len_w tiles of 64 keys, the others `pieces` of `len`, from the part's first key on.  Slots, from
// `base`: the whole units piece by piece, then the others piece by piece.
struct Part {
  int32_t base, tiles, whole, pieces_w, len_w, pieces, len, row0, rows, keys0, keys1, group;
};
constexpr int kPartInts = 12;
static_assert(sizeof(Part) == kPartInts * sizeof(int32_t), "twelve ints");

SharedSizes shared_sizes(int64_t n_reqs, int64_t n_groups, int64_t max_q, int64_t max_group_q, int64_t max_new,
                         int64_t bt_stride, int hq, int hkv, int head_dim, int64_t num_cus) {
  SharedSizes z;
  const int64_t G = hq / hkv;
  z.tile_p = max_group_q * G <= arckv::kNarrowCols ? arckv::kNarrowCols : arckv::kWideCols;
  z.tile_o = max_new * G <= kTailCols ? kTailCols : max_new * G <= arckv::kNarrowCols ? arckv::kNarrowCols : arckv::kWideCols;
  const int64_t longest = (bt_stride * 16 + arckv::kMaxItemKeys - 1) / arckv::kMaxItemKeys;   // pieces at least
  auto items = [&](int64_t parts, int64_t cols, int64_t units) {
    const int64_t tiles = (max_q * G / cols + std::min(parts, max_q)) * hkv * std::max<int64_t>(longest, 1);
    return 2 * tiles <= units ? units : tiles <= units ? 4 * tiles : tiles + 2 * units;
  };
  z.items_p = n_groups > 0 ? items(n_groups, z.tile_p, num_cus) : 0;
  z.items_o = items(n_reqs, z.tile_o, z.tile_o == kTailCols ? kTailPerUnit * num_cus : num_cus);
  auto per = [](int tile) { return tile == arckv::kNarrowCols ? int64_t{arckv::kListItems} : int64_t{1}; };   // lists of one item
  int64_t at = 16;
  auto take = [&](int64_t n) { const int64_t o = at; at += (n + 15) / 16 * 16; return o; };
  z.off_group = take(n_groups * kPartInts);
  z.off_req = take(n_reqs * kPartInts);
  z.off_row = take(max_q * 2);
  z.off_list = take(max_q);
  z.off_cu = take(n_reqs + 1);
  z.off_len = take(n_reqs);
  z.off_work_p = take(z.items_p * ARCKV_WORK_INTS * per(z.tile_p));
  z.off_work_o = take(z.items_o * ARCKV_WORK_INTS * per(z.tile_o));
  z.n_ints = at;
  z.ws_floats = (z.items_p * z.tile_p + z.items_o * z.tile_o) * (head_dim + 1);
  return z;
}

// Few and short requests read all of their keys in one launch, shared or not: the shared ones come from the caches
// then, and the launches that would save them cost more.  us, one launch and planned (32 / 8 heads of 128 unless stated;
// prefix + own tokens): 4 x 280 of 4 / 2 heads of 64 5.1 and 15.6; 16 x (256 + 100) 7.4 and 18.0; 64 x (256 + 100), 93 MB by
// request, 14.2 and 22.2; 64 x (512 + 300), 213 MB, 25.6 and 35.5; 64 x (896 + 100), 261 MB, 27.3 and 26.6; 256 x (64 + 30), 2048
// work-groups, 31.1 and 30.8; 16 x 1688 20.9 and 21.0; 4 x 1988 22.5 and 20.0.
constexpr int64_t kShortKeys = 1536, kShortBytes = int64_t{224} << 20, kShortGroups = 1024;
bool short_route(const SharedSizes& z, int64_t n_reqs, int64_t bt_stride, int hkv, int head_dim) {
  return z.tile_o == kTailCols && bt_stride * 16 <= kShortKeys && n_reqs * hkv <= kShortGroups &&
         n_reqs * bt_stride * 16 * hkv * head_dim * 4 <= kShortBytes;
}

// ---- the plan ---------------------------------------------------------------------------------

__device__ __forceinline__ int64_t shfl64(int64_t v, int src) {
  const int lo = __shfl(static_cast<int>(v), src), hi = __shfl(static_cast<int>(v >> 32), src);
  return static_cast<int64_t>(static_cast<uint64_t>(static_cast<uint32_t>(hi)) << 32 | static_cast<uint32_t>(lo));
}

constexpr int kPlanParts = 1024;          // groups and requests whose entries are made in LDS
struct PlanShared {
  Part parts[kPlanParts];
  uint32_t wave[kPlanThreads / 64];
  int64_t items[kPlanThreads / 64][64];   // of every candidate cut, by the wave that counted
  int32_t top[kPlanThreads / 64];
  int32_t cap;
};

// The most key tiles of a piece, for n parts (units to cut and key tiles of part i from `size`) in at most `most` items: of 64
// candidates (the longest part in 1, 2, .. 64 pieces) the one that takes least, in key tiles: a round of `units` items takes
// its longest piece and `over` tiles more, and an item's partial results take the chip w64 / 64 tiles to write and read (64
// rows of 32 / 8 heads of 128 on a shared prefix of 2048, 4096 and 8192: 34.6, 36.6 and 42.1 us with pieces of 4, 4 and 8
// tiles, 38.3, 39.5 and 44.3 with 8, 8 and 4).
template <class Size>
__device__ __forceinline__ int choose_cap(int n, int64_t most, int units, int min_cap, int over, int w64, Size size,
                                          PlanShared& sh) {
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
  const float inv = 1.f / static_cast<float>(cap);
#pragma unroll 2
  for (int i = wave; i < n; i += kPlanThreads / 64) {
    int tiles, keys;
    size(i, tiles, keys);
    const int x = keys + cap - 1;                       // below 2^24: the quotient by way of fp32 is at most 1 off
    int pieces = static_cast<int>(static_cast<float>(x) * inv);
    pieces -= pieces * cap > x;
    pieces += (pieces + 1) * cap <= x;
    items += static_cast<int64_t>(tiles) * pieces;
  }
  sh.items[wave][lane] = items;
  __syncthreads();
  if (wave == 0) {
    items = 0;
    for (int w = 0; w < kPlanThreads / 64; ++w) items += sh.items[w][lane];
    const int64_t rounds = (items + units - 1) / units;
    int64_t cost = items <= most ? rounds * (cap + over) * 64 + items * w64 : INT64_MAX / 2;
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

// Exclusive sums over the threads of the work-group, and the total; sums of more than 2^30 stay there (a batch within its bounds
// has fewer of whatever is counted).
__device__ __forceinline__ uint32_t add_sat(uint32_t a, uint32_t b) { return min(a + b, 1u << 30); }
__device__ __forceinline__ int64_t sums_before(int64_t value, int64_t& total, PlanShared& sh) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t s = static_cast<uint32_t>(min(value, int64_t{1} << 30));
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t u = __shfl_up(s, d);
    if (lane >= d) s = add_sat(s, u);
  }
  uint32_t before = __shfl_up(s, 1);
  if (lane == 0) before = 0;
  __syncthreads();
  if (lane == 63) sh.wave[wave] = s;
  __syncthreads();
  uint32_t earlier = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    if (w == wave) earlier = all;
    all = add_sat(all, sh.wave[w]);
  }
  total = all;
  return add_sat(earlier, before);
}

// The sum of a value of every thread.
__device__ __forceinline__ int64_t sum_threads(int64_t v, PlanShared& sh) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += shfl64(v, (threadIdx.x & 63) ^ d);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.items[threadIdx.x >> 6][0] = v;
  __syncthreads();
  v = 0;
  for (int w = 0; w < kPlanThreads / 64; ++w) v += sh.items[w][0];
  __syncthreads();
  return v;
}

// Pieces and slots of the parts, then their work items.  With more units than the chip takes at a time, whole rounds of
// them stay whole, but for those of more than a chip's unit's share of all keys, and only what is left is cut, so that it
// fills a last, shorter round (320 tiles of 128 key tiles on 256 units: 272 us, and 339 with every tile cut in two).  Units of the same keys lie `heads` apart: with 8 heads on one XCD.
// DIRECT: a unit of one piece that nothing joins has slot -1, and its kernel writes the result.
template <bool DIRECT, class ReqOf>
__device__ void emit_items(Part* parts, int n, int hkv, int units, int min_cap, int over, int w64, int tile_cols, int per, Work* work,
                           int64_t most, ReqOf req_of, PlanShared& sh) {
  const int tid = threadIdx.x;
  // (tiles of no keys count as one: the tail kernel's items of rows that see none)
  auto keys_of = [](const Part& p) { return p.tiles > 0 ? max((p.keys1 - p.keys0 + kBK - 1) / kBK, 1) : 0; };
  int64_t all = 0, total, first_sum = 0;
  int64_t load = 0;                                   // key tiles of this thread's parts
  int longest = 0;
  for (int i0 = 0; i0 < n; i0 += kPlanThreads) {
    const int i = i0 + tid, keys = i < n ? keys_of(parts[i]) : 0;
    const int64_t mine = keys > 0 ? static_cast<int64_t>(parts[i].tiles) * hkv : 0;
    load += mine * keys;
    longest = max(longest, keys);
    first_sum = sums_before(mine, total, sh);
    all += total;
  }
  const int64_t first_cut = all / units * units;      // units before this one stay whole
  const int64_t share = first_cut > 0 ? (sum_threads(load, sh) + units - 1) / units : kMaxPieceTiles;
  const int cap_w = static_cast<int>(min(max(share, static_cast<int64_t>(min_cap)), static_cast<int64_t>(kMaxPieceTiles)));
  bool longer = longest > cap_w;                      // a whole unit has several pieces
  int64_t at = 0, at_w = first_cut;                   // items of the whole units
  longer = __syncthreads_or(longer);
  if (longer) at_w = 0;
  for (int i0 = 0; i0 < n; i0 += kPlanThreads) {
    const int i = i0 + tid;
    const int keys = i < n ? keys_of(parts[i]) : 0;
    const int64_t mine = keys > 0 ? static_cast<int64_t>(parts[i].tiles) * hkv : 0;
    const int64_t before = n <= kPlanThreads ? first_sum : at + sums_before(mine, total, sh);
    at += total;
    int64_t items = 0;
    if (i < n) {
      Part& p = parts[i];
      p.whole = static_cast<int>(min(max(first_cut - before, int64_t{0}), mine));
      p.pieces_w = (keys + cap_w - 1) / cap_w;
      p.len_w = p.pieces_w > 0 ? (keys + p.pieces_w - 1) / p.pieces_w : 0;
      p.pieces_w = p.pieces_w > 0 ? (keys + p.len_w - 1) / p.len_w : 0;
      items = static_cast<int64_t>(p.whole) * p.pieces_w;
    }
    if (longer) {
      sums_before(items, total, sh);
      at_w += total;
    }
  }
  __syncthreads();
  const int cap = choose_cap(n, most - at_w, units, min_cap, over, w64, [=](int i, int& cut, int& keys) {
    keys = keys_of(parts[i]);
    cut = keys > 0 ? parts[i].tiles * hkv - parts[i].whole : 0;
  }, sh);
  at = 0;
  for (int i0 = 0; i0 < n; i0 += kPlanThreads) {
    const int i = i0 + tid;
    int64_t mine = 0;
    Part p = {};
    if (i < n) {
      p = parts[i];
      const int keys = keys_of(p);
      p.pieces = keys > 0 ? (keys + cap - 1) / cap : 0;
      p.len = p.pieces > 0 ? (keys + p.pieces - 1) / p.pieces : 0;
      p.pieces = p.pieces > 0 ? (keys + p.len - 1) / p.len : 0;
      mine = static_cast<int64_t>(p.whole) * p.pieces_w + (static_cast<int64_t>(p.tiles) * hkv - p.whole) * p.pieces;
    }
    const int64_t before = at + sums_before(mine, total, sh);
    if (i < n) {
      p.base = static_cast<int32_t>(min(before, most));
      if (before + mine > most) p.tiles = p.whole = p.pieces = 0;     // (lengths or groups that pass the bounds: no slot for it)
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
      int k = static_cast<int>(e) - p.base;
      const int whole_items = p.whole * p.pieces_w, cut = p.tiles * hkv - p.whole;
      const bool is_whole = k < whole_items;
      if (is_whole || cut > 0) {
        if (!is_whole) k -= whole_items;
        const int piece = k / (is_whole ? p.whole : cut), unit = k % (is_whole ? p.whole : cut) + (is_whole ? 0 : p.whole);
        const int len = is_whole ? p.len_w : p.len, pieces = is_whole ? p.pieces_w : p.pieces;
        w.req = req_of(lo);
        w.kvh = unit % hkv;
        w.col_start = unit / hkv * tile_cols;
        w.kv_start = p.keys0 + piece * len * kBK;
        w.kv_end = min(w.kv_start + len * kBK, p.keys1);
        w.slot = DIRECT && p.keys0 == 0 && pieces == 1 ? -1 : static_cast<int32_t>(e);
        w.pad0 = pieces;
      }
    }
    work[e * per] = w;
    if (per > 1) work[e * per + 1].req = -1;
  }
  __syncthreads();
}

__global__ __launch_bounds__(kPlanThreads) void shared_plan_kernel(
    const int32_t* __restrict__ group_start, const int32_t* __restrict__ prefix_lens, int n_groups,
    const int32_t* __restrict__ cu_q, const int32_t* __restrict__ seq_lens, int n_reqs, int max_q, int bt_stride, int G,
    int hkv, int num_cus, SharedSizes z, int32_t* __restrict__ plan) {
  __shared__ PlanShared sh;
  const int tid = threadIdx.x;
  // small batches are planned in LDS (the plan's entries are copied out at the end): every step below waits for the last
  const bool in_lds = n_groups + n_reqs <= kPlanParts;
  Part* const groups = in_lds ? sh.parts : reinterpret_cast<Part*>(plan + z.off_group);
  Part* const reqs = in_lds ? sh.parts + n_groups : reinterpret_cast<Part*>(plan + z.off_req);
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
    p.group = INT32_MAX;                               // of a group: its first request that has rows (below)
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
    if (g >= 0 && S > 0) {
      atomicMin(&groups[g].keys1, max(L - S, 0));
      if (q0 == row(start(g))) groups[g].group = r;    // the first of its group that has rows
      atomicAdd(&groups[g].whole, static_cast<int>((static_cast<int64_t>(S) * G + z.tile_o - 1) / z.tile_o));
    }
    Part p = {};
    p.row0 = q0;
    p.rows = S;
    p.keys1 = static_cast<int32_t>(min(static_cast<int64_t>(L), room));
    p.group = g;
    reqs[r] = p;
  }
  __syncthreads();
  for (int g = tid; g < n_groups; g += kPlanThreads) {
    int shared = __hip_atomic_load(&groups[g].keys1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) / kBK * kBK;
    const int apart = __hip_atomic_load(&groups[g].whole, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    Part& p = groups[g];
    // The shared keys are read through this request's table: one without rows may have ended, and its table name other blocks
    if (p.group >= n_reqs) shared = 0;
    const int together = static_cast<int>((static_cast<int64_t>(p.rows) * G + z.tile_p - 1) / z.tile_p);
    // Requests that fill their own wide tiles read their keys once for 256 columns anyhow: sharing that saves no more than
    // an eighth of the tiles is not worth a second item and the join (2 x 1024 rows on 16384: 978 us shared)
    if (z.tile_o == arckv::kWideCols && z.tile_p == arckv::kWideCols && 8 * apart <= 9 * together) shared = 0;
    p.tiles = shared > 0 ? together : 0;
    p.keys1 = shared;
    if (p.tiles > 0) {                                 // the group as a request of the kernels above
      cu[p.group] = p.row0;
      cu[p.group + 1] = p.row0 + p.rows;
      len[p.group] = shared + p.rows;
    }
  }
  __syncthreads();
  for (int r = tid; r < n_reqs; r += kPlanThreads) {
    Part& p = reqs[r];
    p.keys0 = p.group >= 0 && p.rows > 0 ? groups[p.group].keys1 : 0;
    // Rows without own keys: the tail kernel writes them too (there may be no join); in tiles they are the join's
    p.tiles = p.keys1 > p.keys0 || z.tile_o == kTailCols ? static_cast<int>((static_cast<int64_t>(p.rows) * G + z.tile_o - 1) / z.tile_o) : 0;
  }
  const int total = row(n_reqs);
  for (int t = tid; t < total; t += kPlanThreads) {    // a row's request and group
    int lo = 0, hi = n_reqs - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (reqs[mid].row0 <= t) lo = mid; else hi = mid - 1;
    }
    row_of[t] = make_int2(lo, reqs[lo].group);
  }
  __syncthreads();
  // ---- the cuts and the items ------------------------------------------------------------------
  auto tiles = [&](auto direct, Part* parts, int n, int tile, int64_t off, int64_t most, auto req_of) {
    const bool wide = tile == arckv::kWideCols;
    emit_items<decltype(direct)::value>(parts, n, hkv, num_cus, wide ? 4 : 2, wide ? 8 : 5, wide ? 2 : 1, tile,
                                        wide ? 1 : arckv::kListItems, reinterpret_cast<Work*>(plan + off), most, req_of, sh);
  };
  if (n_groups > 0)
    tiles(std::false_type{}, groups, n_groups, z.tile_p, z.off_work_p, z.items_p, [&](int g) { return groups[g].group; });
  if (z.tile_o == kTailCols)
    emit_items<false>(reqs, n_reqs, hkv, kTailPerUnit * num_cus, kTailWhole / kBK, 8, 0, kTailCols, 1,
                      reinterpret_cast<Work*>(plan + z.off_work_o), z.items_o, [](int r) { return r; }, sh);
  else
    tiles(std::true_type{}, reqs, n_reqs, z.tile_o, z.off_work_o, z.items_o, [](int r) { return r; });
  // ---- the rows that the join has to look at: those of several pieces, but for what the tail kernel joins itself
  if (tid == 0) sh.cap = 0;
  __syncthreads();
  for (int t = tid; t < total; t += kPlanThreads) {
    const int2 of = row_of[t];
    const Part& p = reqs[of.x];
    const bool cut = (p.whole > 0 && p.pieces_w > 1) || (p.tiles * hkv > p.whole && p.pieces > 1);
    const bool shared = z.tile_o != kTailCols && of.y >= 0 && groups[of.y].tiles > 0;
    if (cut || shared || p.tiles == 0) plan[z.off_list + atomicAdd(&sh.cap, 1)] = t;
  }
  if (in_lds)
    for (int i = tid; i < (n_groups + n_reqs) * kPartInts; i += kPlanThreads)
      plan[i < n_groups * kPartInts ? z.off_group + i : z.off_req + i - n_groups * kPartInts] = reinterpret_cast<int32_t*>(sh.parts)[i];
  __syncthreads();
  if (tid == 0) plan[0] = sh.cap;
}

// ---- joining pieces --------------------------------------------------------------------------------
// D / 4 lanes have a (row, head), four dims each: its partial results (fp32, normalised) and their lse (base 2).
typedef float acc4_t __attribute__((ext_vector_type(4)));
struct Joined {
  float m = -INFINITY, sum = 0.f;
  acc4_t acc = {};
};
// Adds pieces i0, i0 + step, .. < n.  Their lse come in 16 at a time (a lane each), the partial results eight at a time, the
// first eight beside the lse.
template <class Lse, class Row>
__device__ __forceinline__ void add_pieces(Joined& j, int i0, int step, int n, Lse lse_of, Row row_of) {
  constexpr int kBatch = 16, kLoad = 8;
  const int sub = threadIdx.x % kBatch, mine = (threadIdx.x & 63) / kBatch * kBatch;
  for (; i0 < n; i0 += step * kBatch) {
    const float l = i0 + sub * step < n ? lse_of(i0 + sub * step) : -INFINITY;
    acc4_t v[kLoad];
    auto load = [&](int k0) {
#pragma unroll
      for (int k = 0; k < kLoad; ++k) v[k] = i0 + (k0 + k) * step < n ? *row_of(i0 + (k0 + k) * step) : acc4_t{};
    };
    load(0);
    float top = l;
#pragma unroll
    for (int d = kBatch / 2; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    const float m_new = fmaxf(j.m, top);
    const float mu = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = j.m == -INFINITY ? 0.f : fast_exp2(j.m - mu);
    const float wt = l == -INFINITY ? 0.f : fast_exp2(l - mu);
    j.m = m_new;
    j.sum *= alpha;
    j.acc *= alpha;
#pragma unroll
    for (int k0 = 0; k0 < kBatch; k0 += kLoad) {
      if (k0 > 0) {
        if (i0 + k0 * step >= n) break;
        load(k0);
      }
#pragma unroll
      for (int k = 0; k < kLoad; ++k) {
        const float a = __shfl(wt, mine + k0 + k);          // (0 past the last piece)
        j.sum += a;
        j.acc += a * v[k];
      }
    }
  }
}
// another sum of exponentials (not normalised) into j
__device__ __forceinline__ void add_sum(Joined& j, float m, float sum, const acc4_t& acc) {
  const float m_new = fmaxf(j.m, m);
  const float a = j.m == -INFINITY ? 0.f : fast_exp2(j.m - m_new), b = m == -INFINITY ? 0.f : fast_exp2(m - m_new);
  j.m = m_new;
  j.sum = a * j.sum + b * sum;                            // (0 times a NaN stays NaN)
  j.acc = a * j.acc + b * acc;
}
__device__ __forceinline__ void write_joined(const Joined& j, uint16_t* out, float* lse_out, int64_t row_head, int d, int d4) {
  const float inv = j.sum > 0.f ? 1.f / j.sum : 0.f;
  store_out<true>(out + row_head * d + 4 * d4, __builtin_convertvector(j.acc * inv, bf16x4_t));
  if (lse_out != nullptr && d4 == 0)
    lse_out[row_head] = j.sum > 0.f ? (j.m + __log2f(j.sum)) * kLn2 : j.sum == 0.f ? -INFINITY : j.sum;
}
// Pieces of column `c` (row - row0 times G, and the head of the group) of a part, and where its first piece lies and how far
// apart they are, in columns.  (Tiles have a power of two of columns; the columns of all items are fewer than 2^31.)
__device__ __forceinline__ int pieces_of(const Part& p, uint32_t c, int kvh, int hkv, int tile_cols, int& first, int& step) {
  const int log_cols = __builtin_ctz(tile_cols);
  const int unit = static_cast<int>(c >> log_cols) * hkv + kvh, cut = p.tiles * hkv - p.whole;
  const bool whole = unit < p.whole;
  const int slot = p.base + (whole ? unit : p.whole * p.pieces_w + unit - p.whole);
  first = (slot << log_cols) + static_cast<int>(c & static_cast<uint32_t>(tile_cols - 1));
  step = (whole ? p.whole : cut) << log_cols;
  return p.tiles == 0 ? 0 : whole ? p.pieces_w : p.pieces;
}

// ---- the own keys of decode steps --------------------------------------------------------------
// An item is up to 16 columns (token x head of one KV group) of a request over a range of keys.  Too few columns to share
// a tile: K and V go from memory straight into the operands of v_mfma_f32_16x16x32_bf16, 32 keys a step, the waves taking
// steps in turn, and nothing passes through LDS but the waves' results at the end.  An item that has all of its columns' own
// keys joins them with the pieces over shared keys, which an earlier launch has written, and writes the result; one of
// several pieces writes a partial result.  What bounds it is the
// bytes of K and V (78 requests of 56 to 6500 own tokens, 40 / 8 heads, 225 MB and the shared pieces: 51 us), and the chain of
// waits (item, lengths, table, keys, join) of items of a few steps: 5 us without keys; three work-groups of four
// waves share a compute unit.  With fewer requests and heads than units (WAVES = 8) an item's keys are spread over twice the
// waves: 23 requests of 60 to 820 own tokens on a shared 8192 32.7 us in all, 33.7 with four; three times as many the same.
//   S^T (16 keys x 16 columns, twice): lane (i = l % 16, g = l / 16) holds row i's dims 32 k + 8 g ..; row i of
//   product m is key 8 (i / 4) + 4 m + i % 4, so that the lane's results, rows 4 g + e, are the keys 8 g + 4 m + e
//   of its column: the eight keys that it holds as the operand of P.V.
//   O^T (16 dims x 16 columns): lane's V operand is dim 16 d + i, keys 8 g ..: 16 bytes of the dim-major block.
// SHORT: no plan; a work-group has a request's columns for a head, and all of their keys, shared or not.
template <int D, int G, int WAVES, bool SHORT>
__global__ __launch_bounds__(64 * WAVES, 3) void shared_tail_kernel(
    const uint16_t* __restrict__ k_pool, const uint16_t* __restrict__ v_pool, const uint16_t* __restrict__ q,
    uint16_t* __restrict__ out, float* __restrict__ lse_out, const int32_t* __restrict__ block_tables, int bt_stride,
    const int32_t* __restrict__ cu_q, const int32_t* __restrict__ seq_lens, int n_reqs, int n_groups, int64_t n_q,
    int64_t num_blocks, int hq, int hkv, float scale_log2, const int32_t* __restrict__ plan, SharedSizes z,
    const float* __restrict__ ws_op, const float* __restrict__ ws_lp, float* __restrict__ ws_oo, float* __restrict__ ws_lo) {
  constexpr int KS = D / 32, DM = D / 16, LANES = D / 4, SETS = 64 * WAVES / LANES;
  constexpr int PO = D + 4;                               // a column's row of the waves' results (floats)
  __shared__ __attribute__((aligned(16))) float part_o[WAVES][kTailCols][PO];
  __shared__ float part_m[WAVES][kTailCols], part_l[WAVES][kTailCols];
  __shared__ acc4_t set_o[SHORT ? 1 : SETS][LANES];
  __shared__ float set_m[SETS], set_s[SETS];
  const int tid = threadIdx.x, lane = tid & 63;
  for (int item = blockIdx.x; SHORT || item < z.items_o; item += gridDim.x) {
    Work w = {static_cast<int>(blockIdx.x), static_cast<int>(blockIdx.y), 0, 0, INT32_MAX, 0, 1, 0};
    if constexpr (!SHORT) w = reinterpret_cast<const Work*>(plan + z.off_work_o)[item];
    if (w.req < 0 || w.req >= n_reqs || w.kvh < 0 || w.kvh >= hkv || w.col_start < 0 || (!SHORT && w.slot >= z.items_o)) {
      if constexpr (SHORT) return; else continue;
    }
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int i16 = lane & 15, g4 = lane >> 4;
    const int32_t* bt = block_tables + static_cast<int64_t>(w.req) * bt_stride;
    const int q0 = cu_q[w.req], S = cu_q[w.req + 1] - q0, L = seq_lens[w.req];
    const int P = L - S, ncols = S * G, held = min(L, bt_stride * 16), nblk = (held + 15) >> 4;
    const uint32_t nb32 = static_cast<uint32_t>(min(num_blocks, static_cast<int64_t>(INT32_MAX)));
    const int64_t blk_stride = static_cast<int64_t>(hkv) * 16 * D;
    const int64_t head = static_cast<int64_t>(w.kvh) * 16 * D;
    Part group = {};
    if constexpr (!SHORT) {
      const int g = reinterpret_cast<const Part*>(plan + z.off_req)[w.req].group;
      if (g >= 0 && g < n_groups && w.pad0 == 1) group = reinterpret_cast<const Part*>(plan + z.off_group)[g];
    }
    const int set = tid / LANES, d4 = tid % LANES;
    for (int col0 = w.col_start; col0 < (SHORT ? ncols : w.col_start + 1); col0 += kTailCols) {
      const int n_here = min(ncols - col0, kTailCols);      // columns that are there
      if (n_here <= 0) break;                               // (uniform)
      // ---- pieces over shared keys: sets_per sets of lanes have a column -------------------------
      const int sets_per = n_here * 8 <= SETS ? 8 : n_here * 4 <= SETS ? 4 : n_here * 2 <= SETS ? 2 : 1;
      auto shared = [&](int c, int from) {                  // into LDS: registers are short while the keys are read
        if constexpr (!SHORT) {
          Joined j;
          const int at = col0 + c;
          const int64_t row = q0 + at / G - group.row0;
          if (c < n_here && group.tiles > 0 && row >= 0 && row < group.rows) {
            int first, step;
            const int n = pieces_of(group, static_cast<uint32_t>(row * G + at % G), w.kvh, hkv, z.tile_p, first, step);
            add_pieces(j, from, sets_per, n, [&](int i) { return ws_lp[first + i * step]; },
                       [&](int i) { return reinterpret_cast<const acc4_t*>(ws_op + static_cast<int64_t>(first + i * step) * D + 4 * d4); });
          }
          set_o[set][d4] = j.acc;
          if (d4 == 0) {
            set_m[set] = j.m;
            set_s[set] = j.sum;
          }
        }
      };
      // ---- the keys ------------------------------------------------------------------------------
      const int col = col0 + i16, tok = col / G;
      const bool cval = col < ncols && q0 + tok < n_q;
      const int pos = cval ? P + tok : -1;
      const int last_tok = (col0 + n_here - 1) / G;
      const int kv_lo = max(w.kv_start, 0), kv_hi = min(min(w.kv_end, P + last_tok + 1), held);
      const int min_pos = P + col0 / G;
      const int steps = kv_hi > kv_lo ? (kv_hi - kv_lo + 31) / 32 : 0;
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
      auto entry = [&](int b) -> int32_t { return b < nblk ? bt[b] : 0; };      // (uniform)
      auto block_of = [&](int32_t ph) -> int64_t {
        ARCKV_CHECK_WAVE(ph < 0 || ph >= num_blocks, ARCKV_CHECK_BLOCK);
        return (static_cast<uint32_t>(ph) >= nb32 ? 0 : ph) * blk_stride + head;
      };
      acc4_t o[DM];
#pragma unroll
      for (int d = 0; d < DM; ++d) o[d] = acc4_t{};
      float m_run = -INFINITY, l_run = 0.f;
      int32_t e0 = 0, e1 = 0;                               // the next step's table entries, read a step ahead
      auto look_up = [&](int s) {
        if (s < steps) {
          e0 = entry((kv_lo + 32 * s) >> 4);
          e1 = entry(((kv_lo + 32 * s) >> 4) + 1);
        }
      };
      look_up(wave);
      shared(set / sets_per, set % sets_per);
      // (K/V a step ahead of their use, at 256 registers and two waves on a SIMD, measured no faster: 16.2 and 16.0 us for 23
      // requests of 60 to 820 own tokens)
      for (int s = wave; s < steps; s += WAVES) {
        const int k0 = kv_lo + 32 * s;
        const int64_t b0 = block_of(e0), b1 = block_of(e1);
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
        look_up(s + WAVES);
        acc4_t sc[2] = {acc4_t{}, acc4_t{}};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
          for (int m = 0; m < 2; ++m) sc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[m][ks], qf[ks], sc[m], 0, 0, 0);
        const int key0 = k0 + 8 * g4;
        if (k0 + 31 > min_pos || k0 + 32 > kv_hi) {         // (uniform) keys that some column does not see
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (key0 + j > pos || key0 + j >= kv_hi) sc[j / 4][j % 4] = -INFINITY;
        }
        if (k0 + 32 > held) {                               // past the request's end the block may hold anything, NaN too
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
      // ---- the waves' results: lane holds dims 16 d + 4 g .. + 3 of its column -------------------
      l_run += __shfl_xor(l_run, 16);
      l_run = sum_halves(l_run);
#pragma unroll
      for (int d = 0; d < DM; ++d) *reinterpret_cast<acc4_t*>(&part_o[wave][i16][16 * d + 4 * g4]) = o[d];
      if (g4 == 0) {
        part_m[wave][i16] = m_run;
        part_l[wave][i16] = l_run;
      }
      for (int c0 = 0; c0 < n_here; c0 += SETS / sets_per) {
        if (c0 > 0) shared(c0 + set / sets_per, set % sets_per);
        __syncthreads();
        const int c = c0 + set / sets_per;
        if (c < n_here && set % sets_per == 0 && q0 + (col0 + c) / G < n_q) {
          Joined mine;
          if constexpr (!SHORT)
            for (int k = 0; k < sets_per; ++k) add_sum(mine, set_m[set + k], set_s[set + k], set_o[set + k][d4]);
          Joined keys;
#pragma unroll
          for (int v = 0; v < WAVES; ++v)
            add_sum(keys, part_m[v][c], part_l[v][c], *reinterpret_cast<const acc4_t*>(&part_o[v][c][4 * d4]));
          if (SHORT || w.pad0 == 1) {
            add_sum(mine, keys.m, keys.sum, keys.acc);
            const int at = col0 + c;
            write_joined(mine, out, lse_out, static_cast<int64_t>(q0 + at / G) * hq + w.kvh * G + at % G, D, d4);
          } else {
            const float inv = keys.sum > 0.f ? 1.f / keys.sum : 0.f;
            const int64_t at = static_cast<int64_t>(w.slot) * kTailCols + c;
            *reinterpret_cast<acc4_t*>(ws_oo + at * D + 4 * d4) = keys.acc * inv;
            if (d4 == 0) ws_lo[at] = keys.sum > 0.f ? keys.m + __log2f(keys.sum) : keys.sum == 0.f ? -INFINITY : keys.sum;
          }
        }
        __syncthreads();
      }
    }
    if constexpr (SHORT) break;
  }
}

// ---- the join ------------------------------------------------------------------------------------
// What the items have not joined: rows over shared and own keys in tiles, and own keys in several pieces.  plan[0] says
// how many rows that may be, and its list which.  With few rows (SPLIT) a work-group has one row and head and its sets of lanes take the pieces in turn;
// otherwise it has a row and its sets take the heads.  What bounds it is reading the partial results (fp32): 2048 rows of 40
// heads of 128, 2.6 pieces each, 109 MB read and 21 written in 30 us; with few rows the two round trips (4 to 6 us).
constexpr int64_t kSplitPairs = 8192;   // most (row, head) pairs whose pieces are split over a work-group
template <int D, bool SPLIT>
__global__ __launch_bounds__(256) void shared_join_kernel(uint16_t* __restrict__ out, float* __restrict__ lse_out,
                                                          const int32_t* __restrict__ plan, SharedSizes z, int n_reqs, int n_groups,
                                                          int64_t n_q, int hq, int hkv, int G, const float* __restrict__ ws_op,
                                                          const float* __restrict__ ws_lp, const float* __restrict__ ws_oo,
                                                          const float* __restrict__ ws_lo) {
  constexpr int LANES = D / 4, SETS = 256 / LANES;
  __shared__ acc4_t set_o[SPLIT ? SETS : 1][LANES];
  __shared__ float set_m[SETS], set_s[SETS];
  const int set = threadIdx.x / LANES, d4 = threadIdx.x % LANES;
  const int at = SPLIT ? blockIdx.x / hq : blockIdx.x;
  if (at >= plan[0] || at >= n_q) return;
  const int64_t t = plan[z.off_list + at];
  if (t < 0 || t >= n_q) return;
  const int2 of = reinterpret_cast<const int2*>(plan + z.off_row)[t];
  auto part = [&](int64_t off, int i, int n) {
    const Part p = i >= 0 && i < n ? reinterpret_cast<const Part*>(plan + off)[i] : Part{};
    return t >= p.row0 && t - p.row0 < p.rows ? p : Part{};
  };
  const Part pg = part(z.off_group, of.y, n_groups), pr = part(z.off_req, of.x, n_reqs);
  for (int h = SPLIT ? blockIdx.x % hq : set; h < hq; h += SPLIT ? hq : SETS) {
    const int kvh = h / G;
    int p0, ps, r0, rs;
    const int np = pieces_of(pg, static_cast<uint32_t>((t - pg.row0) * G + h % G), kvh, hkv, z.tile_p, p0, ps);
    const int nr = pieces_of(pr, static_cast<uint32_t>((t - pr.row0) * G + h % G), kvh, hkv, z.tile_o, r0, rs);
    if (nr == 1 && (np == 0 || z.tile_o == kTailCols)) continue;     // its item has written the result
    Joined j;
    add_pieces(j, SPLIT ? set : 0, SPLIT ? SETS : 1, np + nr,
               [&](int i) { return i < np ? ws_lp[p0 + i * ps] : ws_lo[r0 + (i - np) * rs]; },
               [&](int i) {
                 return reinterpret_cast<const acc4_t*>((i < np ? ws_op : ws_oo) +
                                                        static_cast<int64_t>(i < np ? p0 + i * ps : r0 + (i - np) * rs) * D + 4 * d4);
               });
    if constexpr (SPLIT) {
      set_o[set][d4] = j.acc;
      if (d4 == 0) {
        set_m[set] = j.m;
        set_s[set] = j.sum;
      }
      __syncthreads();
      if (set > 0) return;
      for (int k = 1; k < SETS; ++k) add_sum(j, set_m[k], set_s[k], set_o[k][d4]);
    }
    write_joined(j, out, lse_out, t * hq + h, D, d4);
  }
}

// What the three calls check of the bounds that they share.
int32_t check_shared(const char* fn, int32_t n_reqs, int32_t n_groups, int64_t max_q, int64_t max_group_q, int64_t max_new,
                     int32_t bt_stride, int32_t hq, int32_t hkv, int32_t head_dim, int32_t num_cus) {
  if (n_reqs < 0 || n_reqs > (1 << 20) || n_groups < 0 || n_groups > std::max(n_reqs, 1) || max_q < 0 || max_q > (1 << 23) ||
      max_group_q < 0 || max_group_q > max_q || max_new < 0 || max_new > max_q || bt_stride < 0 || bt_stride > (1 << 25) ||
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
  const SharedSizes z = shared_sizes(n_reqs, n_groups, max_q, max_group_q, max_new, bt_stride, num_q_heads, num_kv_heads,
                                     head_dim, num_cus);
  if (n_reqs == 0 || max_q == 0) return ARCKV_OK;
  if (cu_q == nullptr || seq_lens == nullptr || plan == nullptr ||
      (n_groups > 0 && (group_start == nullptr || prefix_lens == nullptr)))
    return arckv::fail(ARCKV_EINVAL, "shared_prefix_plan: NULL pointer");
  if (reinterpret_cast<uintptr_t>(plan) % 16 != 0)
    return arckv::fail(ARCKV_EINVAL, "shared_prefix_plan: the plan must be 16-byte aligned");
  if (plan_ints < z.n_ints)
    return arckv::fail(ARCKV_ENOSPC, "shared_prefix_plan: %lld ints, and the plan needs %lld", (long long)plan_ints,
                       (long long)z.n_ints);
  if (short_route(z, n_reqs, bt_stride, num_kv_heads, head_dim)) return ARCKV_OK;     // the attention takes no plan
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
    auto part = [&](int tile, int64_t items, const int32_t* work, const int32_t* cu, const int32_t* len, float* wo, float* wl,
                    float* lse_out) {
      auto* wk = reinterpret_cast<const Work*>(work);
      const dim3 grid(static_cast<unsigned>(items));
      auto run = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(512), 0, st, kp, vp, qp, op, block_tables, bt_stride, cu, len, n_reqs, wk, max_q,
                           num_blocks, num_q_heads, num_kv_heads, scale_log2, wo, wl, items, lse_out);
      };
      if (tile == arckv::kWideCols && any_align) run(prefill_attn_pp_kernel<D, GG, false, true>);
      else if (tile == arckv::kWideCols) run(prefill_attn_pp_kernel<D, GG, false, false>);
      else if (any_align) run(prefill_attn_list_kernel<D, GG, true>);
      else run(prefill_attn_list_kernel<D, GG, false>);
    };
    auto tail = [&](auto waves, auto is_short, dim3 grid) {
      hipLaunchKernelGGL((shared_tail_kernel<D, GG, decltype(waves)::value, decltype(is_short)::value>), grid,
                         dim3(64 * decltype(waves)::value), 0, st, kp, vp, qp, op, lse, block_tables, bt_stride, cu_q, seq_lens, n_reqs,
                         n_groups, max_q, num_blocks, num_q_heads, num_kv_heads, scale_log2, plan, z, ws_op, ws_lp, ws_oo, ws_lo);
    };
    using W4 = std::integral_constant<int, 4>;
    using W8 = std::integral_constant<int, 8>;
    if (short_route(z, n_reqs, bt_stride, num_kv_heads, head_dim)) {
      tail(W8{}, std::true_type{}, dim3(static_cast<unsigned>(n_reqs), static_cast<unsigned>(num_kv_heads)));
      return;
    }
    if (z.items_p > 0) part(z.tile_p, z.items_p, plan + z.off_work_p, plan + z.off_cu, plan + z.off_len, ws_op, ws_lp, nullptr);
    if (z.tile_o != kTailCols) {
      part(z.tile_o, z.items_o, plan + z.off_work_o, cu_q, seq_lens, ws_oo, ws_lo, lse);
    } else {
      if (std::min<int64_t>(n_reqs, max_q) * num_kv_heads <= num_cus)
        tail(W8{}, std::false_type{}, dim3(static_cast<unsigned>(std::min<int64_t>(num_cus, z.items_o))));
      else tail(W4{}, std::false_type{}, dim3(static_cast<unsigned>(z.items_o)));
      if (bt_stride * 16 <= kTailWhole) return;           // no request's own keys can be cut
    }
    const int64_t pairs = max_q * num_q_heads;
    auto join = [&](auto split, int64_t groups) {
      hipLaunchKernelGGL((shared_join_kernel<D, decltype(split)::value>), dim3(static_cast<unsigned>(groups)), dim3(256), 0, st, op,
                         lse, plan, z, n_reqs, n_groups, max_q, num_q_heads, num_kv_heads, GG, ws_op, ws_lp, ws_oo, ws_lo);
    };
    if (pairs <= kSplitPairs) join(std::true_type{}, pairs); else join(std::false_type{}, max_q);
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
