// Wide tiles (256 query columns) of attention over the 4-bit cache (part of prefill_attn.hip).
//
// The ping-pong of prefill_attn_pp_kernel: 8 waves of 32 columns; V(j) (mask, exponentials of tile j)
// of one half of the waves runs beside M(j) (O += V P, S(j + 1) = K Q^T) of the other.  A tile of 64
// keys is turned into bf16 once for all 8 waves, on its way from the pool to LDS: a thread holds 8
// bytes of K codes (16 dimensions of a token), 8 of V codes (2 dimensions of 8 tokens) and their scales,
// loaded in M(j) for tile j + 3, and in M(j + 1) writes them as bf16 into the stage of that tile, between
// the MFMAs.  (Codes in LDS and decoded by each wave for its own 32 columns would be 8 times the
// conversions: about 1.6 times the MFMAs' own time.)  LDS then holds what the bf16 kernel's does, in
// the same swizzled places.  Probabilities are rounded to bf16 for P.V, as in the narrow kernel.
//
// What bounds it is the matrix units with the conversions beside them: 2048 tokens on 32768, 64 / 8 heads of
// 128, 1.91 to 1.98 ms (1.15 to 1.19 PFLOP/s; the bf16 kernel 1.79, a large matrix product's rate 1.71).
// Without the loads it would take 1.81 (against 1.95 on the same card), without the conversions 1.69, without
// both 1.60.  8 questions of 128 on 8192, 40 / 8: 216 us (bf16 196): 192 items on 256 units.  12 prompts of 1100,
// 16 / 16 heads of 64: 72 us (bf16 64).  LDS operands 4 or 6 ahead and V writes without bank conflicts change
// nothing.
#pragma once

namespace {

// col / G for the group sizes there are, as a product (exact below 2^30)
struct GroupDiv {
  uint32_t g, mul;    // mul = ceil(2^32 / g), 0 for g = 1
  __device__ __forceinline__ int tok(int col) const {
    return mul == 0 ? col : static_cast<int>(__umulhi(static_cast<uint32_t>(col), mul));
  }
};

template <int D, bool ANY>
__global__ __launch_bounds__(512, D == 64 ? 4 : 1) void mx4_attn_wide_kernel(
    const uint8_t* __restrict__ pool, const uint16_t* __restrict__ q, uint16_t* __restrict__ out,
    float* __restrict__ lse_out, const int32_t* __restrict__ block_tables, int bt_stride,
    const int32_t* __restrict__ cu_q, const int32_t* __restrict__ seq_lens, int n_reqs,
    const Work* __restrict__ work, int64_t n_q, int64_t num_blocks, int hq, int hkv, GroupDiv gd, float scale_log2,
    float* __restrict__ ws_o, float* __restrict__ ws_lse, int64_t ws_slots) {
  using L4 = mx4::Layout<D>;
  constexpr int kThreads = 512;
  constexpr int kCols = arckv::kWideCols;
  constexpr int KSTEPS = D / 16;                 // k-steps of Q.K^T
  constexpr int DM = D / 32;                     // 32-row blocks of O^T
  constexpr int TILE = kBK * D * 2;              // bytes of one K (or V) tile in LDS
  constexpr int BLK_BYTES = 16 * D * 2;          // one block of one head, K or V, in LDS
  constexpr int NOP = 4 * DM + 2 * KSTEPS;       // MFMAs of a full M phase
  constexpr int PD = D == 64 ? 1 : 3;            // LDS operands in flight ahead of their MFMA
  constexpr int NB = D / 64;                     // dwords of K, V codes and V scales of a thread and tile
  constexpr int kTbl = arckv::kMaxItemKeys / 16;
  // Tile t is written in M(t - 2), half steps 2 t - 2 and 2 t - 1, over tile t - 3, last read in half step
  // 2 t - 3 (M(t - 3) of the second group), and first read in half step 2 t.
  constexpr int kSt = 3;
  __shared__ __attribute__((aligned(1024))) char smem[kSt * 2 * TILE];  // stage s: K, then V
  __shared__ int32_t tbl[kTbl];
  __shared__ int32_t nan_key[DM];                // first key of a masked tile whose V group is NaN

  const Work w = work[blockIdx.x];
  ARCKV_CHECK_WAVE(w.req >= n_reqs || (w.req >= 0 && (w.kvh < 0 || w.kvh >= hkv || w.col_start < 0)),
                   ARCKV_CHECK_WORK);
  if (w.req < 0 || w.req >= n_reqs || w.kvh < 0 || w.kvh >= hkv || w.col_start < 0) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int grp = wave >> 2;
  const int l32 = lane & 31, hg = lane >> 5;
  const int G = static_cast<int>(gd.g);
  // this wave's block of a tile, and its thread's number within the block's bytes
  const int wblk = wave >> 1;
  constexpr int kFirst = 3;
  const int32_t* bt = block_tables + static_cast<int64_t>(w.req) * bt_stride;
  const int b_lo = max(w.kv_start, 0) >> 4;
  const int b_hi = min(max((w.kv_end + kBK - 1) / kBK, 0) * (kBK / 16), bt_stride);   // past the item's last tile
  int32_t first_ph[kFirst];
#pragma unroll
  for (int k = 0; k < kFirst; ++k) {
    const int b = b_lo + k * (kBK / 16) + wblk;
    first_ph[k] = b < b_hi ? bt[b] : 0;
  }
  const int q0 = cu_q[w.req];
  const int S = cu_q[w.req + 1] - q0;
  const int L = seq_lens[w.req];
  const int P = L - S;
  const int ncols = S * G;
  const int nblk = min((L + 15) >> 4, bt_stride);

  const int col = w.col_start + wave * 32 + l32;
  const int tok = gd.tok(col);
  const bool cval = col < ncols && (q0 + tok) < n_q;
  const int pos = cval ? P + tok : -1;

  const int last_col = min(w.col_start + kCols, ncols) - 1;
  const int wg_max_pos = P + gd.tok(max(last_col, 0));
  const int wg_min_pos = P + gd.tok(w.col_start);
  const int kv_lo = max(w.kv_start, 0);
  const int kv_hi = min(w.kv_end, wg_max_pos + 1);
  const int ntiles = kv_hi > kv_lo && last_col >= w.col_start ? (kv_hi - kv_lo + kBK - 1) / kBK : 0;

  // ---- pool -> registers -> LDS -------------------------------------------------------------------
  // A thread's piece of its block.  K: 8 NB dimensions of token piece / 8; V: 2 dimensions of 4 NB tokens.
  // D = 64: 128 registers leave no room to keep what follows from it, so it is taken afresh for each use.
  struct Place {
    int piece, krow, kch, vpair, vhalf, vquad;
  };
  auto place = [&](bool fresh) {
    Place p;
    p.piece = (wave & 1) * 64 + (fresh ? lane_now() : lane);
    p.krow = wblk * 16 + p.piece / 8;                    // row of the tile, and 16-byte chunk of it
    p.kch = NB * (p.piece % 8);
    p.vpair = NB == 2 ? p.piece % 64 : (p.piece % 64) / 2;
    p.vhalf = wave & 1;
    p.vquad = NB == 2 ? 0 : p.piece % 2;
    return p;
  };
  const uint32_t head = static_cast<uint32_t>(w.kvh) * L4::kBytes;
  const int64_t blk_stride = static_cast<int64_t>(hkv) * L4::kBytes;
  const uint32_t nb32 = static_cast<uint32_t>(num_blocks);
  const int n_tbl = max(0, min(min(nblk - b_lo, ntiles * (kBK / 16)), kTbl));
  struct Raw { uint32_t k[NB], v[NB], vs[NB], ks; };
  int32_t next_v = 0;
  auto fetch_next = [&](int tile) {
    const int b = tile * (kBK / 16) + wblk;                          // relative to b_lo
    next_v = b < n_tbl ? tbl[b] : 0;
  };
  // one block of one head as a buffer: its address stays in scalar registers
  auto block_at = [&](int32_t ph) {
    ARCKV_CHECK_WAVE(ph < 0 || static_cast<uint32_t>(ph) >= nb32, ARCKV_CHECK_BLOCK);
    // wave-uniform; an entry out of range reads block 0
    const int32_t pb = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(ph) >= nb32 ? 0 : ph);
    return const_cast<uint8_t*>(pool) + (static_cast<int64_t>(pb) * blk_stride + head);
  };
  auto load = [&](uint8_t* base, Raw& x) {
    const __amdgpu_buffer_rsrc_t buf = __builtin_amdgcn_make_buffer_rsrc(base, 0, L4::kBytes, 0x00027000);
    const Place p = place(D == 64);
    const uint32_t c_ofs = p.piece * (4 * NB);           // of the codes of either
    const uint32_t ks_ofs = L4::kKScale + (p.piece / 8) * L4::kGroups + (p.piece % 8) * NB / 4;
    const uint32_t vs_ofs = L4::kVScale + (p.vpair / 16) * 16 + p.vhalf * 8 + p.vquad * 4;
    if constexpr (NB == 2) {
      const auto k = __builtin_amdgcn_raw_buffer_load_b64(buf, c_ofs, 0, 0);
      const auto v = __builtin_amdgcn_raw_buffer_load_b64(buf, L4::kV + c_ofs, 0, 0);
      const auto vs = __builtin_amdgcn_raw_buffer_load_b64(buf, vs_ofs, 0, 0);
#pragma unroll
      for (int i = 0; i < NB; ++i) { x.k[i] = k[i]; x.v[i] = v[i]; x.vs[i] = vs[i]; }
    } else {
      x.k[0] = __builtin_amdgcn_raw_buffer_load_b32(buf, c_ofs, 0, 0);
      x.v[0] = __builtin_amdgcn_raw_buffer_load_b32(buf, L4::kV + c_ofs, 0, 0);
      x.vs[0] = __builtin_amdgcn_raw_buffer_load_b32(buf, vs_ofs, 0, 0);
    }
    x.ks = __builtin_amdgcn_raw_buffer_load_b8(buf, ks_ofs, 0, 0);
  };
  // Before a masked tile is converted: V of the keys past the item's last (the prompt's end, or block 0 past
  // the last tile) may be anything, and V of a key that only later columns see may be NaN.  Neither may
  // meet a weight of zero, so their scales are replaced; NaN comes back at the end for the columns that
  // see the first such key.
  auto mask_v = [&](Raw& x, int tile) {
    const Place p = place(D == 64);
    int first = INT32_MAX;
#pragma unroll
    for (int k = 4 * NB - 1; k >= 0; --k) {
      const int key = kv_lo + tile * kBK + wblk * 16 + p.vhalf * 8 + p.vquad * 4 + k, sh = 8 * (k & 3);
      uint32_t& s = x.vs[k / 4];
      const bool nan = ((s >> sh) & 255u) == mx4::kNanScale && key < kv_hi;
      first = nan ? key : first;
      if (nan || key >= kv_hi) s = (s & ~(255u << sh)) | (127u << sh);
    }
    if (first != INT32_MAX) atomicMin(&nan_key[p.vpair / 16], first);
  };
  // conversions, in parts: NB 16-byte chunks of a K row, then 4 NB tokens of two dimensions of V
  constexpr int PARTS = 2 * NB + 2;
  uint32_t vx[4 * NB];
  auto convert = [&](const Raw& x, int st, int part) {          // st: byte offset of the tile's stage
    if (part < NB) {
      const float ks = mx4::scale_value(x.ks);
      const uint32_t c = x.k[part];
      const u32x4_t v = {mx4::decode2<0>(c, ks), mx4::decode2<1>(c, ks), mx4::decode2<2>(c, ks), mx4::decode2<3>(c, ks)};
      const Place p = place(D == 64);
      *reinterpret_cast<u32x4_t*>(smem + st + p.krow * 2 * D + (((p.kch + part) ^ fk<D>(p.krow)) * 16)) = v;
    } else if (part < 2 * NB) {
      const int i = part - NB;
      const uint32_t c = x.v[i], s = x.vs[i];
      vx[4 * i] = mx4::decode2<0>(c, mx4::scale_value(s & 255u));
      vx[4 * i + 1] = mx4::decode2<1>(c, mx4::scale_value((s >> 8) & 255u));
      vx[4 * i + 2] = mx4::decode2<2>(c, mx4::scale_value((s >> 16) & 255u));
      vx[4 * i + 3] = mx4::decode2<3>(c, mx4::scale_value(s >> 24));
    } else {
      const int d = part - 2 * NB;
      uint32_t v[2 * NB];
#pragma unroll
      for (int k = 0; k < 2 * NB; ++k) v[k] = __builtin_amdgcn_perm(vx[2 * k + 1], vx[2 * k], d == 0 ? 0x05040100u : 0x07060302u);
      const Place p = place(false);
      char* to = smem + st + TILE + wblk * BLK_BYTES + (2 * p.vpair + d) * 32 + ((p.vhalf ^ sv(2 * p.vpair)) * 16) + p.vquad * 8;
      __builtin_memcpy(__builtin_assume_aligned(to, 8 * NB), v, 8 * NB);
    }
  };
  // tiles that need the causal / prompt-end mask form a suffix of the key range
  auto tile_masked = [&](int t) {
    const int t0 = kv_lo + t * kBK;
    return (t0 + kBK - 1 > wg_min_pos) || (t0 + kBK > L);
  };

  f32x16_t o[DM];
#pragma unroll
  for (int md = 0; md < DM; ++md) o[md] = f32x16_t{};
  bf16x8_t qf[KSTEPS];              // Q^T operands of this lane's column
  f32x16_t sacc[2];                 // S^T of one tile: 2 blocks of 32 keys x this wave's columns
  uint32_t pw[4][4];                // P^T operands: 4 blocks of 16 keys, bf16 pairs
  float m_run = -INFINITY, l_run = 0.f;

  // ---- V phase (as in prefill_attn_pp_kernel) -------------------------------------------------------
  auto v_phase = [&](int j, auto masked) {
    const int t0 = kv_lo + j * kBK;
    if constexpr (decltype(masked)::value) {
#pragma unroll
      for (int mb = 0; mb < 2; ++mb)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int key = t0 + mb * 32 + 16 * (r >> 3) + 8 * hg + (r & 7);
          sacc[mb][r] = key > pos ? -INFINITY : sacc[mb][r];
        }
    }
    auto exps = [&](float mu) {
      float sum = -0.f;
#pragma unroll
      for (int mb = 0; mb < 2; ++mb)
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int jj = 0; jj < 4; ++jj) {
            const f32x2_t two = {fast_exp2(fmaf(sacc[mb][8 * half + 2 * jj], scale_log2, -mu)),
                                 fast_exp2(fmaf(sacc[mb][8 * half + 2 * jj + 1], scale_log2, -mu))};
            sum += two[0];
            sum += two[1];
            pw[2 * mb + half][jj] = __builtin_bit_cast(uint32_t, __builtin_convertvector(two, bf16x2_t));
          }
      return sum;
    };
    float lsum = 0.f;
    bool pending = true;
    if (j > 0) {
      lsum = exps(m_run == -INFINITY ? 0.f : m_run);
      pending = __builtin_amdgcn_ballot_w64(!(lsum <= kLazySum)) != 0;   // also catches inf / NaN sums
    }
    if (pending) {
      float m = -INFINITY;
#pragma unroll
      for (int mb = 0; mb < 2; ++mb)
#pragma unroll
        for (int r = 0; r < 16; ++r) m = fmaxf(m, sacc[mb][r]);
      const float mx = max_halves(m) * scale_log2;
      const float m_new = fmaxf(m_run, mx);
      const float alpha = m_new == -INFINITY ? 1.f : fast_exp2(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int md = 0; md < DM; ++md) o[md] *= alpha;
      lsum = exps(m_run == -INFINITY ? 0.f : m_run);
    }
    l_run += lsum;
  };

  // ---- M phase: V^T P, then K Q^T of the next tile, with the conversion of tile j + 2 between ----------
  // Bytes of tile j + 2, and of tile j + 3 on their way.  D = 64 has registers for one of them: its load
  // goes out once the conversion is through.
  // (Two sets that change places, in steps of two: a copy from one to the other would wait for the load.)
  constexpr bool kAhead = D == 128;
  Raw raw, next;
  // Byte offsets of the stages of tiles j, j + 1 and j + 2 of the step being run.
  int st0 = 0, st1 = 2 * TILE, st2 = 4 * TILE;
  auto m_phase = [&](Raw& cur, Raw& nxt, uint8_t* block) {
    // The lane's operand of V: rows l32 + 32 md of block sp, its half.  Of K: row pi(l32) + 32 mb, chunk 2 ks + hg
    // swizzled: stages and rows start at multiples of 256 (D = 64: 128) bytes, so chunks 2 ks on are an
    // exclusive or away.
    const char* const va = smem + (st0 + TILE + l32 * 32 + ((hg ^ sv(l32)) * 16));
    const uint32_t kr = pi_row(l32), ka = st1 + kr * (2 * D) + ((hg ^ fk<D>(kr)) * 16);
    auto op_at = [&](int n) -> bf16x8_t {
      if (n < 4 * DM) {
        const int sp = n / DM, md = n % DM;
        return *reinterpret_cast<const bf16x8_t*>(va + sp * BLK_BYTES + md * 1024);
      }
      const int ks = (n - 4 * DM) / 2, mb = (n - 4 * DM) % 2;
      return *reinterpret_cast<const bf16x8_t*>(smem + (ka ^ (ks * 32)) + mb * (64 * D));
    };
    constexpr int EVERY = NOP / (PARTS + 2);
    if constexpr (kAhead) load(block, nxt);
    bf16x8_t opv[NOP];
#pragma unroll
    for (int n = 0; n < PD; ++n) opv[n] = op_at(n);
#pragma unroll
    for (int n = 0; n < NOP; ++n) {
      if (n + PD < NOP) opv[n + PD] = op_at(n + PD);
      if (n < 4 * DM) {
        const int sp = n / DM, md = n % DM;
        const u32x4_t w4 = {pw[sp][0], pw[sp][1], pw[sp][2], pw[sp][3]};
        o[md] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(opv[n], __builtin_bit_cast(bf16x8_t, w4), o[md], 0, 0, 0);
      } else {
        const int ks = (n - 4 * DM) / 2, mb = (n - 4 * DM) % 2;
        sacc[mb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(opv[n], qf[ks], ks == 0 ? f32x16_t{} : sacc[mb], 0, 0, 0);
      }
      if (n % EVERY == EVERY / 2) {
        if (n / EVERY < PARTS) convert(cur, st2, n / EVERY);
        else if (n / EVERY == PARTS && !kAhead) load(block_at(__builtin_amdgcn_readfirstlane(next_v)), cur);
      }
    }
    // keep the operand reads PD ahead: DS reads, then one MFMA and one read at a time
    __builtin_amdgcn_sched_group_barrier(0x100, PD, 0);
#pragma unroll
    for (int n = 0; n < NOP - PD; ++n) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      // the loads of tile j + 3 after the first MFMAs: at the end of the phase they would come late
      if (kAhead && n < 4) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, PD, 0);
  };
  auto s_first = [&]() {
    const char* kb = smem;
#pragma unroll
    for (int ks = 0; ks < KSTEPS; ++ks)
#pragma unroll
      for (int mb = 0; mb < 2; ++mb) {
        const int r = mb * 32 + pi_row(l32);
        const int c = 2 * ks + hg;
        const bf16x8_t a = *reinterpret_cast<const bf16x8_t*>(kb + r * 2 * D + ((c ^ fk<D>(r)) * 16));
        sacc[mb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qf[ks], ks == 0 ? f32x16_t{} : sacc[mb], 0, 0, 0);
      }
  };
  auto pin_v = [&]() {
#pragma unroll
    for (int sp = 0; sp < 4; ++sp)
#pragma unroll
      for (int jj = 0; jj < 4; ++jj) asm volatile("" ::"v"(pw[sp][jj]));
    asm volatile("" ::"v"(l_run), "v"(m_run));
  };
  auto pin_m = [&]() {
#pragma unroll
    for (int md = 0; md < DM; ++md) asm volatile("" ::"v"(o[md][0]));
    asm volatile("" ::"v"(sacc[0][0]), "v"(sacc[1][0]));
  };
  auto barrier = [&]() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };

  // ---- prologue: table, queries (straight into the stages of tiles 1 and 2) and the first tiles ---------
  constexpr int QROWS = 512 / D;
  constexpr int QLD = 32 / QROWS;
  char* qst = smem + 2 * TILE + wave * (32 * D * 2);
  static_assert(8 * 32 * D * 2 == 2 * (2 * TILE), "the queries fill two stages");
  Raw raw1;
  if (tid < DM) nan_key[tid] = INT32_MAX;
  if (ntiles > 0) {
#pragma unroll
    for (int k = 0; k < kTbl / kThreads; ++k) {
      const int e = k * kThreads + wave * 64;          // wave-uniform
      if (e < n_tbl) load_lds4(bt + b_lo + min(e + lane, n_tbl - 1), (lds_void*)(tbl + e));
    }
    if (w.col_start + wave * 32 < ncols)
#pragma unroll
    for (int i = 0; i < QLD; ++i) {
      const int r = i * QROWS + lane / (D / 8);
      const int c = w.col_start + wave * 32 + r;       // columns past the request load row 0, never used
      const int t = gd.tok(c);
      const bool ok = c < ncols && (q0 + t) < n_q;
      const int64_t row = ok ? static_cast<int64_t>(q0 + t) * hq + w.kvh * G + (c - t * G) : 0;
      const uint16_t* src = q + row * D + (((lane % (D / 8)) ^ fk<D>(r)) * 8);
      if constexpr (ANY) load_any16(src, qst + i * 1024 + lane * 16);
      else load_lds16(src, (lds_void*)(qst + i * 1024));
    }
    auto first = [&](int t) { return b_lo + t * (kBK / 16) + wblk < nblk ? first_ph[t] : 0; };
    load(block_at(first(0)), raw);
    load(block_at(first(1)), raw1);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  }
  __syncthreads();                  // nan_key is set, table and queries are here
  if (ntiles > 0) {
#pragma unroll
    for (int ks = 0; ks < KSTEPS; ++ks)
      qf[ks] = cval ? *reinterpret_cast<const bf16x8_t*>(qst + l32 * (2 * D) + (((2 * ks + hg) ^ fk<D>(l32)) * 16))
                    : bf16x8_t{};
    if (tile_masked(0)) mask_v(raw, 0);
    if (tile_masked(1)) mask_v(raw1, 1);
#pragma unroll
    for (int p = 0; p < PARTS; ++p) convert(raw, st0, p);
    fetch_next(2);
    barrier();                                           // every wave has its queries
#pragma unroll
    for (int p = 0; p < PARTS; ++p) convert(raw1, st1, p);
    load(block_at(__builtin_amdgcn_readfirstlane(next_v)), raw);
    fetch_next(3);
    barrier();                                           // tiles 0 and 1 are there
    if (grp == 1) barrier();                             // half step 0: group 1 waits
    s_first();                                           // M(-1)
    pin_m();
    barrier();
    auto step = [&](int j, auto masked, Raw& cur, Raw& nxt) {
      uint8_t* block = nullptr;
      if constexpr (kAhead) block = block_at(__builtin_amdgcn_readfirstlane(next_v));    // of tile j + 3
      v_phase(j, masked);
      pin_v();
      barrier();
      // past the key range the table gives block 0 and the conversion writes a stage nobody reads
      if (tile_masked(j + 2)) mask_v(cur, j + 2);
      m_phase(cur, nxt, block);
      const int st3 = st0;
      st0 = st1;
      st1 = st2;
      st2 = st3;
      fetch_next(j + 4);
      pin_m();
      if (grp == 0 || j + 1 < ntiles) barrier();
    };
    int n_plain = ntiles;
    {
      int lo = 0, hi = ntiles;  // first masked tile, else ntiles
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (tile_masked(mid)) hi = mid; else lo = mid + 1;
      }
      n_plain = lo;
    }
    int j = 0;
    if constexpr (D == 128) asm volatile(".p2align 5");
    if constexpr (kAhead) {
      for (; j + 1 < n_plain; j += 2) {
        step(j, std::false_type{}, raw, next);
        step(j + 1, std::false_type{}, next, raw);
      }
      if (j < n_plain) {
        step(j, std::false_type{}, raw, next);
        raw = next;
        ++j;
      }
      for (; j < ntiles; ++j) {
        step(j, std::true_type{}, raw, next);
        raw = next;
      }
    } else {
      for (; j < n_plain; ++j) step(j, std::false_type{}, raw, raw);
      for (; j < ntiles; ++j) step(j, std::true_type{}, raw, raw);
    }
  }

  // ---- epilogue: O^T register r of block md holds dim 32 md + 8 (r / 4) + 4 hg + r % 4 ------
  const float lt = sum_halves(l_run);
  const float inv = lt > 0.f ? 1.f / lt : 0.f;
  const float lse = lt > 0.f ? m_run + __log2f(lt) : lt == 0.f ? -INFINITY : lt;   // a NaN stays
  const int le = D == 64 ? lane_now() : lane, r32 = le & 31, he = le >> 5;
  const int ce = w.col_start + wave * 32 + r32, te = gd.tok(ce);
  const bool ve = ce < ncols && (q0 + te) < n_q;
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");    // no wave reads the ring, nan_key is whole
#pragma unroll
  for (int md = 0; md < DM; ++md) o[md] *= nan_key[md] <= (ve ? P + te : -1) ? __builtin_nanf("") : inv;
  const int64_t rowe = ve ? static_cast<int64_t>(q0 + te) * hq + w.kvh * G + (ce - te * G) : 0;
  if (lse_out != nullptr && w.slot < 0 && ve && he == 0) lse_out[rowe] = lse * kLn2;
  if (w.slot >= ws_slots || w.col_start + wave * 32 >= ncols) return;
  // Through LDS ([column][dim], this wave's own rows), so that rows leave as whole 16-byte chunks.
  constexpr int EP = 2 * D + 16;                     // row pitch in bytes
  char* ep = smem + wave * (32 * EP);
  if (w.slot < 0) {
#pragma unroll
    for (int md = 0; md < DM; ++md)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        f32x4_t v;
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) v[jj] = o[md][4 * r4 + jj];
        *reinterpret_cast<bf16x4_t*>(ep + r32 * EP + (md * 32 + 8 * r4 + 4 * he) * 2) = __builtin_convertvector(v, bf16x4_t);
      }
#pragma unroll
    for (int i = 0; i < QLD; ++i) {
      const int r = i * QROWS + le / (D / 8), ch = le % (D / 8);
      const int c = w.col_start + wave * 32 + r, t = gd.tok(c);
      const u32x4_t v = *reinterpret_cast<const u32x4_t*>(ep + r * EP + ch * 16);
      if (c < ncols && (q0 + t) < n_q)
        store_out<ANY>(out + (static_cast<int64_t>(q0 + t) * hq + w.kvh * G + (c - t * G)) * D + ch * 8, v);
    }
    return;
  }
  float* po = ws_o + (static_cast<int64_t>(w.slot) * kCols + wave * 32) * D;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
#pragma unroll
    for (int m = 0; m < DM / 2; ++m)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        f32x4_t v;
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) v[jj] = o[half * (DM / 2) + m][4 * r4 + jj];
        *reinterpret_cast<f32x4_t*>(ep + r32 * EP + (m * 32 + 8 * r4 + 4 * he) * 4) = v;
      }
#pragma unroll
    for (int i = 0; i < QLD; ++i) {
      const int r = i * QROWS + le / (D / 8), ch = le % (D / 8);
      const int c = w.col_start + wave * 32 + r, t = gd.tok(c);
      const f32x4_t v = *reinterpret_cast<const f32x4_t*>(ep + r * EP + ch * 16);
      if (c < ncols && (q0 + t) < n_q)
        *reinterpret_cast<f32x4_t*>(po + static_cast<int64_t>(r) * D + half * (D / 2) + ch * 4) = v;
    }
  }
  if (ve && he == 0) ws_lse[static_cast<int64_t>(w.slot) * kCols + wave * 32 + r32] = lse;
}

}  // namespace
