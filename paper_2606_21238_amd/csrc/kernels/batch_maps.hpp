// A step's block and slot maps, made on the device from the requests' lengths (part of kv_scatter.hip).
//
// Requests in order: request r holds h tokens and wants w more, which takes b = ceil((h + w) / 16) - ceil(h / 16)
// blocks.  With B and W the running sums of b and w over the requests up to it, r gets its tokens if B fits the
// free blocks (or b = 0) and W the slots.  As the sums only grow, the requests that take blocks are the first ones
// that want any, and the blocks taken are the top of the free stack, in order.
//
// A few thousand integers: what bounds it is latency.  One work-group scans the requests and writes lengths and
// offsets; up to kMapsInOne slots (a decode step: 64 requests 4.9 us) it writes their table entries and slots too, more are
// left to a second launch, which counts the blocks of the requests before its own anew
// (they follow from seq_lens and cu_q): 4096 requests of 60 tokens 8.0 and 9.7 us, 50 with the table entries in the scan.
#pragma once

namespace {

constexpr int kMapsThreads = 1024;
// Most slots and requests whose maps the scanning work-group writes whole.  us in one launch and in two (inside a graph): 64
// requests of 16, 64 and 120 tokens 5.3, 7.4 and 9.4 against 10.7, 11.1 and 11.0; 2000 of one 9.3 and 14.6; 4000 of two 20.7 and 17.2.
constexpr int kMapsInOne = 8192, kMapsInOneReqs = 2048;

__device__ __forceinline__ int64_t shfl_up64(int64_t v, int d) {
  const int lo = __shfl_up(static_cast<int>(v), d), hi = __shfl_up(static_cast<int>(v >> 32), d);
  return static_cast<int64_t>(static_cast<uint64_t>(static_cast<uint32_t>(hi)) << 32 | static_cast<uint32_t>(lo));
}

// What requests want, in tokens and blocks; the sums of those that can never have theirs may pass 32 bits.
struct Want {
  int64_t tokens, blocks;
};
struct Scan {
  Want wave[kMapsThreads / 64];
};
// Inclusive sums over the threads of the work-group, and the totals.
__device__ __forceinline__ Want scan_threads(Want v, Scan& s, Want& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t t = shfl_up64(v.tokens, d), b = shfl_up64(v.blocks, d);
    if (lane >= d) {
      v.tokens += t;
      v.blocks += b;
    }
  }
  __syncthreads();                                     // the last call's sums have been read
  if (lane == 63) s.wave[wave] = v;
  __syncthreads();
  Want before = {0, 0}, all = {0, 0};
#pragma unroll
  for (int w = 0; w < kMapsThreads / 64; ++w) {
    if (w == wave) before = all;
    all.tokens += s.wave[w].tokens;
    all.blocks += s.wave[w].blocks;
  }
  total = all;
  return {before.tokens + v.tokens, before.blocks + v.blocks};
}
// blocks of `got` tokens behind `held` ones
__device__ __forceinline__ int32_t blocks_behind(int64_t held, int64_t got) {
  return static_cast<int32_t>((held + got + 15) / 16 - (held + 15) / 16);
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

// the slot of position pos: in block b, and by a request's table
__device__ __forceinline__ int32_t slot_in(int32_t b, int64_t pos, int64_t num_blocks) {
  const bool bad = b < 0 || b >= num_blocks;
  ARCKV_CHECK_LANE(bad, ARCKV_CHECK_BLOCK);
  return bad ? -1 : b * 16 + static_cast<int32_t>(pos & 15);
}
__device__ __forceinline__ int32_t slot_of(const int32_t* table, int64_t pos, int64_t num_blocks) {
  return slot_in(table[pos >> 4], pos, num_blocks);
}

// ALL: table entries and slots too; a request to a thread.  Otherwise four.
template <bool ALL>
__global__ __launch_bounds__(kMapsThreads) void batch_maps_kernel(
    const int32_t* new_tokens, const int32_t* held, int32_t n_reqs, int32_t* block_tables, int32_t bt_stride,
    const int32_t* free_blocks, int64_t free_cap, const int32_t* free_count, int32_t* free_left, int32_t* cu_q,
    int32_t* seq_lens, const int32_t* true_offset, int32_t* true_lens, int32_t* slot_mapping, int32_t slot_cap,
    int64_t num_blocks) {
  constexpr int kPer = ALL ? 1 : 4;
  __shared__ Scan sh, sh_taken;
  __shared__ int32_t cu[ALL ? kMapsThreads + 1 : 1], upto[ALL ? kMapsThreads + 1 : 1], pos0[ALL ? kMapsThreads : 1];
  const int tid = threadIdx.x;
  const int64_t avail = min(static_cast<int64_t>(max(*free_count, 0)), free_cap);
  Want wanted = {0, 0}, taken = {0, 0};                // by the requests of earlier rounds
  for (int32_t r0 = 0; r0 < n_reqs; r0 += kMapsThreads * kPer) {
    int32_t h[kPer], want[kPer];
    Want w[kPer], mine = {0, 0};
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int32_t r = r0 + tid * kPer + k;
      want[k] = r < n_reqs ? new_tokens[r] : 0;
      h[k] = r < n_reqs ? held[r] : 0;
    }
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int64_t to = static_cast<int64_t>(h[k]) + want[k];
      const bool can = want[k] >= 0 && h[k] >= 0 && to <= static_cast<int64_t>(bt_stride) * 16 && to <= INT32_MAX;
      w[k] = can ? Want{want[k], blocks_behind(h[k], want[k])} : Want{0, 0};
      mine.tokens += w[k].tokens;
      mine.blocks += w[k].blocks;
    }
    Want total, sum = scan_threads(mine, sh, total);
    sum.tokens += wanted.tokens - mine.tokens;         // of the requests before this thread's
    sum.blocks += wanted.blocks - mine.blocks;
    wanted.tokens += total.tokens;
    wanted.blocks += total.blocks;
    Want got = {0, 0}, before = sum;                   // tokens and blocks handed out before this thread's requests
    if (wanted.tokens > slot_cap || wanted.blocks > avail) {        // (uniform) not all fit
#pragma unroll
      for (int k = 0; k < kPer; ++k) {
        sum.tokens += w[k].tokens;
        sum.blocks += w[k].blocks;
        if (sum.tokens > slot_cap || (w[k].blocks > 0 && sum.blocks > avail)) w[k] = {0, 0};
        got.tokens += w[k].tokens;
        got.blocks += w[k].blocks;
      }
      before = scan_threads(got, sh_taken, total);
      before.tokens += taken.tokens - got.tokens;
      before.blocks += taken.blocks - got.blocks;
      taken.tokens += total.tokens;
      taken.blocks += total.blocks;
    } else {
      taken = wanted;
    }
    const int64_t left = avail - (taken.blocks - total.blocks);     // on the stack before this round
    int32_t at = static_cast<int32_t>(before.tokens);
    if (ALL && tid == 0) cu[0] = at, upto[0] = 0;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int32_t r = r0 + tid * kPer + k;
      const int32_t len = h[k] + static_cast<int32_t>(w[k].tokens);
      at += static_cast<int32_t>(w[k].tokens);
      if (r < n_reqs) {
        seq_lens[r] = len;
        cu_q[r + 1] = at;
        if (true_lens != nullptr) true_lens[r] = len + true_offset[r];
      }
    }
    if constexpr (ALL) {
      cu[tid + 1] = at;
      upto[tid + 1] = static_cast<int32_t>(before.blocks + w[0].blocks - (taken.blocks - total.blocks));
      pos0[tid] = h[0];
      __syncthreads();
      const int n = min(n_reqs - r0, kMapsThreads);
      for (int32_t e = tid; e < upto[n]; e += kMapsThreads) {
        const int i = last_at_most([&](int k) { return upto[k]; }, 0, n - 1, e);
        block_tables[static_cast<int64_t>(r0 + i) * bt_stride + (pos0[i] + 15) / 16 + (e - upto[i])] = free_blocks[left - 1 - e];
      }
      __syncthreads();
      const int32_t t1 = cu[n];
      for (int32_t t = cu[0] + tid; t < t1; t += kMapsThreads) {
        const int i = last_at_most([&](int k) { return cu[k]; }, 0, n - 1, t);
        slot_mapping[t] = slot_of(block_tables + static_cast<int64_t>(r0 + i) * bt_stride,
                                  static_cast<int64_t>(pos0[i]) + (t - cu[i]), num_blocks);
      }
      __syncthreads();                                 // the round's arrays are no longer read
    }
  }
  if (tid == 0) {
    cu_q[0] = 0;
    *free_left = static_cast<int32_t>(avail - taken.blocks);
  }
  if constexpr (ALL)
    for (int32_t t = static_cast<int32_t>(taken.tokens) + tid; t < slot_cap; t += kMapsThreads) slot_mapping[t] = -1;
}

// The table entries and slots of every new token, where there are many.  A work-group has kSlots of them.  Which blocks its
// requests take follows from the blocks of those before them, which it adds up itself; its own requests' offsets are
// summed kScanReqs at a time.
constexpr int kSlotThreads = 256, kSlots = 1024, kScanReqs = 1024;
__global__ __launch_bounds__(kSlotThreads) void batch_slots_kernel(
    const int32_t* __restrict__ cu_q, const int32_t* __restrict__ seq_lens, int32_t n_reqs, int32_t* block_tables,
    int32_t bt_stride, const int32_t* __restrict__ free_blocks, const int32_t* __restrict__ free_left,
    int32_t* __restrict__ slot_mapping, int32_t slot_cap, int64_t num_blocks) {
  __shared__ int32_t upto[kScanReqs + 1], cu[kScanReqs + 1], end[kScanReqs];
  __shared__ int32_t wave_sum[kSlotThreads / 64], sums[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int32_t t0 = blockIdx.x * kSlots, t1 = min(t0 + kSlots, slot_cap);
  const int32_t total = n_reqs > 0 ? cu_q[n_reqs] : 0;
  for (int32_t t = max(t0, total) + tid; t < t1; t += kSlotThreads) slot_mapping[t] = -1;
  if (t0 >= total) return;
  const int32_t last = min(t1, total) - 1;
  auto taken_by = [&](int r) {
    const int32_t got = cu_q[r + 1] - cu_q[r];
    return blocks_behind(static_cast<int64_t>(seq_lens[r]) - got, got);
  };
  // One pass over the requests: how many begin at or before the first slot and the last one, the blocks taken by those
  // that end there, and by all.
  if (tid < 4) sums[tid] = 0;
  __syncthreads();
  int32_t part[4] = {0, 0, 0, 0};
#pragma unroll 4
  for (int r = tid; r < n_reqs; r += kSlotThreads) {
    const int32_t c0 = cu_q[r], c1 = cu_q[r + 1], b = taken_by(r);
    part[0] += c0 <= t0;
    part[1] += c0 <= last;
    part[2] += c1 > c0 && c1 <= t0 ? b : 0;
    part[3] += c1 > c0 ? b : 0;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) part[k] += __shfl_xor(part[k], d);
    if (lane == 0) atomicAdd(&sums[k], part[k]);
  }
  __syncthreads();
  const int lo = sums[0] - 1, hi = sums[1] - 1;
  int32_t before = sums[2];
  const int64_t avail = static_cast<int64_t>(*free_left) + sums[3];
  constexpr int kPer = kScanReqs / kSlotThreads;
  for (int c0 = lo; c0 <= hi; c0 += kScanReqs) {
    const int n = min(hi + 1 - c0, kScanReqs);
    int32_t mine[kPer], sum = 0;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int i = tid * kPer + k;
      mine[k] = 0;
      if (i < n) {
        cu[i + 1] = cu_q[c0 + i + 1];
        end[i] = seq_lens[c0 + i];
        mine[k] = cu_q[c0 + i + 1] > cu_q[c0 + i] ? taken_by(c0 + i) : 0;
      }
      sum += mine[k];
    }
    if (tid == 0) cu[0] = cu_q[c0], upto[0] = before;
    int32_t up = sum;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int32_t u = __shfl_up(up, d);
      if (lane >= d) up += u;
    }
    if (lane == 63) wave_sum[wave] = up;
    __syncthreads();
    int32_t at = before + up - sum;
    for (int v = 0; v < wave; ++v) at += wave_sum[v];
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      at += mine[k];
      if (tid * kPer + k < n) upto[tid * kPer + k + 1] = at;
    }
    __syncthreads();
    for (int32_t t = max(t0, cu[0]) + tid; t <= min(last, cu[n] - 1); t += kSlotThreads) {
      const int i = last_at_most([&](int k) { return cu[k]; }, 0, n - 1, t);
      const int64_t pos = static_cast<int64_t>(end[i]) - cu[i + 1] + t;
      const int32_t held = end[i] - (cu[i + 1] - cu[i]);
      const int32_t first = (held + 15) / 16, c = static_cast<int32_t>(pos >> 4);
      int32_t* table = block_tables + static_cast<int64_t>(c0 + i) * bt_stride;
      if (c < first) {
        slot_mapping[t] = slot_of(table, pos, num_blocks);
      } else {
        const int32_t b = free_blocks[avail - 1 - (upto[i] + (c - first))];
        if ((pos & 15) == 0) table[c] = b;
        slot_mapping[t] = slot_in(b, pos, num_blocks);
      }
    }
    before = upto[n];
    __syncthreads();                                   // the arrays are no longer read
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
  if (cap <= kMapsInOne && n_reqs <= kMapsInOneReqs) {
    hipLaunchKernelGGL(batch_maps_kernel<true>, dim3(1), dim3(kMapsThreads), 0, st, new_tokens, held, n_reqs, block_tables,
                       bt_stride, free_blocks, free_cap, free_count, free_left, cu_q, seq_lens, true_offset, true_lens,
                       slot_mapping, cap, num_blocks);
  } else {
    hipLaunchKernelGGL(batch_maps_kernel<false>, dim3(1), dim3(kMapsThreads), 0, st, new_tokens, held, n_reqs, block_tables,
                       bt_stride, free_blocks, free_cap, free_count, free_left, cu_q, seq_lens, true_offset, true_lens,
                       slot_mapping, cap, num_blocks);
    if (cap > 0)                                       // without slots nobody has a token, nor takes a block
      hipLaunchKernelGGL(batch_slots_kernel, dim3(static_cast<unsigned>((cap + kSlots - 1) / kSlots)), dim3(kSlotThreads), 0, st,
                         cu_q, seq_lens, n_reqs, block_tables, bt_stride, free_blocks, free_left, slot_mapping, cap, num_blocks);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return arckv::fail(ARCKV_EDEVICE, "batch_maps: %s", hipGetErrorString(e));
  return ARCKV_OK;
}
