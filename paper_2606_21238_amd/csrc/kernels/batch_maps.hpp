// A step's block and slot maps, made on the device from the requests' lengths (part of kv_scatter.hip).
//
// Requests in order: request r holds h tokens and wants w more, which takes b = ceil((h + w) / 16) - ceil(h / 16)
// blocks.  With B and W the running sums of b and w over the requests up to it, r gets its tokens if B fits the
// free blocks (or b = 0) and W the slots.  As the sums only grow, the requests that take blocks are the first ones
// that want any, and the blocks taken are the top of the free stack, in order.
//
// A few thousand integers: what bounds it is latency, so one work-group scans the requests, 1024 at a time, and
// writes lengths, offsets and table entries; up to kMapsInOne slots (a decode step) it writes those too, more are
// written by a second launch that finds a slot's request in cu_q.
#pragma once

namespace {

constexpr int kMapsThreads = 1024;
constexpr int kMapsInOne = 8192;      // most slots that the scanning work-group writes itself
constexpr int kMapsPer = 4;           // slots of a thread of the second launch

// What a request's tokens need.
struct Want {
  int64_t tokens, blocks;
};
__device__ __forceinline__ int64_t shfl_up64(int64_t v, int d) {
  const int lo = __shfl_up(static_cast<int>(v), d), hi = __shfl_up(static_cast<int>(v >> 32), d);
  return static_cast<int64_t>(static_cast<uint64_t>(static_cast<uint32_t>(hi)) << 32 | static_cast<uint32_t>(lo));
}

// Inclusive sums over the threads of the work-group, and the totals.
struct Scan {
  int64_t wave[kMapsThreads / 64];
};
__device__ __forceinline__ int64_t scan_threads(int64_t v, Scan& s, int64_t& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t u = shfl_up64(v, d);
    if (lane >= d) v += u;
  }
  __syncthreads();                                     // the last call's sums have been read
  if (lane == 63) s.wave[wave] = v;
  __syncthreads();
  int64_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kMapsThreads / 64; ++w) {
    if (w == wave) before = all;
    all += s.wave[w];
  }
  total = all;
  return before + v;
}

// The last index in [lo, hi] whose entry is at most t (entries grow; the entry at lo is).
template <class P>
__device__ __forceinline__ int last_at_most(P entry, int lo, int hi, int t) {
  while (lo < hi) {
    const int mid = lo + (hi - lo + 1) / 2;
    if (entry(mid) <= t) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// slot of the i-th new token of a request whose new tokens end at `len`
__device__ __forceinline__ int32_t slot_of(const int32_t* table, int64_t pos, int64_t num_blocks) {
  const int32_t b = table[pos >> 4];
  const bool bad = b < 0 || b >= num_blocks;
  ARCKV_CHECK_LANE(bad, ARCKV_CHECK_BLOCK);
  return bad ? -1 : b * 16 + static_cast<int32_t>(pos & 15);
}

template <bool SLOTS>
__global__ __launch_bounds__(kMapsThreads) void batch_maps_kernel(
    const int32_t* new_tokens, const int32_t* held, int32_t n_reqs, int32_t* block_tables, int32_t bt_stride,
    const int32_t* free_blocks, int64_t free_cap, const int32_t* free_count, int32_t* free_left, int32_t* cu_q,
    int32_t* seq_lens, const int32_t* true_offset, int32_t* true_lens, int32_t* slot_mapping, int32_t slot_cap,
    int64_t num_blocks) {
  __shared__ Scan s_tokens, s_blocks, s_taken;
  __shared__ int32_t cu[kMapsThreads + 1], upto[kMapsThreads + 1], first[kMapsThreads], pos0[kMapsThreads];
  __shared__ int32_t last_taker;
  const int tid = threadIdx.x;
  const int64_t avail = min(static_cast<int64_t>(max(*free_count, 0)), free_cap);
  int64_t tokens = 0, blocks = 0;       // wanted by the requests of earlier rounds
  int32_t taken = 0;                    // tokens that they got
  int64_t left = avail;
  for (int32_t r0 = 0; r0 < n_reqs; r0 += kMapsThreads) {
    const int32_t r = r0 + tid, n = min(n_reqs - r0, kMapsThreads);
    int32_t h = 0;
    Want w = {0, 0};
    if (tid < n) {
      const int32_t want = new_tokens[r];
      h = held[r];
      const bool can = want >= 0 && h >= 0 && static_cast<int64_t>(h) + want <= static_cast<int64_t>(bt_stride) * 16 &&
                       static_cast<int64_t>(h) + want <= INT32_MAX;
      if (can) w = {want, (static_cast<int64_t>(h) + want + 15) / 16 - (static_cast<int64_t>(h) + 15) / 16};
    }
    int64_t round_tokens, round_blocks, round_taken;
    const int64_t sum_tokens = tokens + scan_threads(w.tokens, s_tokens, round_tokens);
    const int64_t sum_blocks = blocks + scan_threads(w.blocks, s_blocks, round_blocks);
    const bool fits = (w.blocks == 0 || sum_blocks <= avail) && sum_tokens <= slot_cap;
    const int32_t get = fits ? static_cast<int32_t>(w.tokens) : 0;
    const int32_t use = fits ? static_cast<int32_t>(w.blocks) : 0;
    const int32_t sum_taken = taken + static_cast<int32_t>(scan_threads(get, s_taken, round_taken));
    if (tid == 0) last_taker = -1;
    cu[tid + 1] = sum_taken;
    first[tid] = static_cast<int32_t>((static_cast<int64_t>(max(h, 0)) + 15) / 16);
    pos0[tid] = h;
    if (tid == 0) cu[0] = taken;
    __syncthreads();
    // the blocks of the round's requests that take any: upto[i] behind request i (the same for those that take none)
    if (use > 0) atomicMax(&last_taker, tid);
    __syncthreads();
    const int32_t lt = last_taker;
    if (tid == 0) upto[0] = 0;
    upto[tid + 1] = tid <= lt ? static_cast<int32_t>(min(sum_blocks, avail) - blocks) : 0;
    __syncthreads();
    const int32_t round_use = lt >= 0 ? upto[lt + 1] : 0;
    if (tid < n) {
      seq_lens[r] = h + get;
      cu_q[r + 1] = sum_taken;
      if (true_lens != nullptr) true_lens[r] = h + get + true_offset[r];
      if (r == 0) cu_q[0] = 0;
    }
    for (int32_t e = tid; e < round_use; e += kMapsThreads) {
      // the request of block e: the first i with upto[i + 1] > e
      const int i = last_at_most([&](int k) { return upto[k]; }, 0, lt, e);
      block_tables[static_cast<int64_t>(r0 + i) * bt_stride + first[i] + (e - upto[i])] = free_blocks[left - 1 - e];
    }
    if constexpr (SLOTS) {
      __syncthreads();
      const int32_t t0 = cu[0], t1 = cu[n];
      for (int32_t t = t0 + tid; t < t1; t += kMapsThreads) {
        const int i = last_at_most([&](int k) { return cu[k]; }, 0, n - 1, t);
        slot_mapping[t] = slot_of(block_tables + static_cast<int64_t>(r0 + i) * bt_stride,
                                  static_cast<int64_t>(pos0[i]) + (t - cu[i]), num_blocks);
      }
    }
    tokens += round_tokens;
    blocks += round_blocks;
    taken += static_cast<int32_t>(round_taken);
    left -= round_use;
    __syncthreads();                                   // the round's arrays are no longer read
  }
  if (n_reqs == 0 && tid == 0) cu_q[0] = 0;
  if (tid == 0) *free_left = static_cast<int32_t>(left);
  if constexpr (SLOTS)
    for (int32_t t = taken + tid; t < slot_cap; t += kMapsThreads) slot_mapping[t] = -1;
}

// The slots of every new token, where there are many.
__global__ __launch_bounds__(256) void batch_slots_kernel(const int32_t* __restrict__ cu_q, const int32_t* __restrict__ seq_lens,
                                                          int32_t n_reqs, const int32_t* __restrict__ block_tables,
                                                          int32_t bt_stride, int32_t* __restrict__ slot_mapping,
                                                          int32_t slot_cap, int64_t num_blocks) {
  const int32_t t0 = blockIdx.x * (256 * kMapsPer);
  const int32_t total = cu_q[n_reqs];
  // the requests of the work-group's first and last slot bound the others'
  auto entry = [&](int k) { return cu_q[k]; };
  int lo = 0, hi = max(n_reqs - 1, 0);
  if (t0 < total) {
    lo = last_at_most(entry, lo, hi, t0);
    hi = last_at_most(entry, lo, hi, min(t0 + 256 * kMapsPer - 1, total - 1));
  }
#pragma unroll
  for (int k = 0; k < kMapsPer; ++k) {
    const int64_t t = static_cast<int64_t>(t0) + k * 256 + threadIdx.x;
    if (t >= slot_cap) return;
    int32_t slot = -1;
    if (t < total) {
      const int r = last_at_most(entry, lo, hi, static_cast<int>(t));
      slot = slot_of(block_tables + static_cast<int64_t>(r) * bt_stride,
                     static_cast<int64_t>(seq_lens[r]) - cu_q[r + 1] + t, num_blocks);
    }
    slot_mapping[t] = slot;
  }
}

}  // namespace

extern "C" int32_t arckv_batch_maps(const int32_t* new_tokens, const int32_t* held, int32_t n_reqs, int32_t* block_tables,
                                    int32_t bt_stride, const int32_t* free_blocks, int64_t free_cap, const int32_t* free_count,
                                    int32_t* free_left, int32_t* cu_q, int32_t* seq_lens, const int32_t* true_offset,
                                    int32_t* true_lens, int32_t* slot_mapping, int64_t slot_cap, int64_t num_blocks,
                                    void* stream) {
  if (n_reqs < 0 || n_reqs > (1 << 24) || bt_stride < 0 || free_cap < 0 || free_cap > INT32_MAX || slot_cap < 0 ||
      slot_cap > (1 << 30) || num_blocks < 1 || num_blocks > (int64_t{1} << 27))
    return arckv::fail(ARCKV_EINVAL, "batch_maps: bad sizes");
  if ((n_reqs > 0 && (new_tokens == nullptr || held == nullptr || seq_lens == nullptr ||
                      (block_tables == nullptr && bt_stride > 0))) ||
      (free_cap > 0 && free_blocks == nullptr) || free_count == nullptr || free_left == nullptr || cu_q == nullptr ||
      (slot_cap > 0 && slot_mapping == nullptr) || (true_lens != nullptr && true_offset == nullptr))
    return arckv::fail(ARCKV_EINVAL, "batch_maps: NULL pointer");
  auto* st = static_cast<hipStream_t>(stream);
  const int32_t cap = static_cast<int32_t>(slot_cap);
  if (cap <= kMapsInOne) {
    hipLaunchKernelGGL(batch_maps_kernel<true>, dim3(1), dim3(kMapsThreads), 0, st, new_tokens, held, n_reqs, block_tables,
                       bt_stride, free_blocks, free_cap, free_count, free_left, cu_q, seq_lens, true_offset, true_lens,
                       slot_mapping, cap, num_blocks);
  } else {
    hipLaunchKernelGGL(batch_maps_kernel<false>, dim3(1), dim3(kMapsThreads), 0, st, new_tokens, held, n_reqs, block_tables,
                       bt_stride, free_blocks, free_cap, free_count, free_left, cu_q, seq_lens, true_offset, true_lens,
                       slot_mapping, cap, num_blocks);
    hipLaunchKernelGGL(batch_slots_kernel, dim3(static_cast<unsigned>((cap + 256 * kMapsPer - 1) / (256 * kMapsPer))), dim3(256),
                       0, st, cu_q, seq_lens, n_reqs, block_tables, bt_stride, slot_mapping, cap, num_blocks);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return arckv::fail(ARCKV_EDEVICE, "batch_maps: %s", hipGetErrorString(e));
  return ARCKV_OK;
}
