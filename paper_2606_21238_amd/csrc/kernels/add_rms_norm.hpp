// The norm in front of the producer (part of qkv_rope.hip): residual addition and root-mean-square norm.
//
//   h = x + residual (fp32), residual_out = bf16(h)
//   y = h * rsqrt(mean(h^2) + eps) * weight (fp32, of the unrounded h)
//   out = bf16(y), or scale = max|y| / 448 for every row and out = e4m3(y / scale)
//
// One work-group has a row and holds it in registers as h, so each value is read once; what bounds it is
// the bytes of x, residual, residual_out and out: 25600 x 5120 in bf16 (1.05 GB) 178 us, 5.9 TB/s, 16384 x 4096 to 8 bits (0.47
// GB) 82 us, 5.8 TB/s, above a copy's 4.7 since more is read than written; 64 x 4096 3.0 us, a launch and two round trips (2.9
// inside a graph).  A row's squares are added in fp32: up to 40 in a thread, then by a tree of lanes and waves, always in the
// same order; where the sum leaves [2^-80, 2^100] (squares below or above fp32's numbers may be among them), once more of
// the row times a power of two, which rounds nothing that counts in it.
#pragma once

namespace {

constexpr int kNormMaxHidden = 32768;   // 1024 threads x 4 chunks x 8 values: all that 1024 threads' registers hold

constexpr int64_t kNormMaxRows = int64_t{1} << 21;     // rows of a launch (2^32 threads would be too many)
constexpr float kNormMinScale = 1.17549435e-38f;        // the smallest normal number: 1 / scale is finite

// Sums of squares outside these are taken again, of the row times 2^80 or 2^-80.  Below: a row's largest value is under 2^-40 (its
// square times 2^160 under 2^80) and at least bf16's smallest, 2^-133 (2^-106), and eps times 2^160 is under 2^80.  Above: it is at
// least 2^42 (the sum has 2^15 squares at most), so 2^-76 to 2^96 after, and eps times 2^-160 under 2^-32.
constexpr float kNormSmallSum = 0x1p-80f, kNormLargeSum = 0x1p100f, kNormUp = 0x1p80f, kNormDown = 0x1p-80f;

// 8 values of a row that follow each other.  ANY: at any bf16 address, 16 unaligned bytes in one access (5000 x 4097 in bf16
// takes 30 us, 93 with 2-byte accesses of neighbouring lanes; 5000 x 4096, aligned, 25), and the row may end inside the chunk.
template <int TH>
__device__ __forceinline__ int norm_at(int c) {
  return (c * TH + static_cast<int>(threadIdx.x)) * 8;
}
template <int TH, bool ANY>
__device__ __forceinline__ u32x4_t norm_load(const uint16_t* row, int c, int hidden) {
  const int at = norm_at<TH>(c);
  u32x4_t v = {0, 0, 0, 0};
  if constexpr (ANY) {
    if (at + 8 <= hidden) {
      __builtin_memcpy(&v, row + at, 16);
    } else {
#pragma unroll
      for (int j = 0; j < 7; ++j)
        if (at + j < hidden) v[j / 2] |= static_cast<uint32_t>(row[at + j]) << (16 * (j % 2));
    }
  } else {
    if (at < hidden) v = *reinterpret_cast<const u32x4_t*>(row + at);
  }
  return v;
}
template <int TH, bool ANY>
__device__ __forceinline__ void norm_store(uint16_t* row, int c, int hidden, const u32x4_t& v) {
  const int at = norm_at<TH>(c);
  if constexpr (ANY) {
    if (at + 8 <= hidden) {
      __builtin_memcpy(row + at, &v, 16);
    } else {
#pragma unroll
      for (int j = 0; j < 7; ++j)
        if (at + j < hidden) row[at + j] = static_cast<uint16_t>(v[j / 2] >> (16 * (j % 2)));
    }
  } else {
    if (at < hidden) *reinterpret_cast<u32x4_t*>(row + at) = v;
  }
}

// A value of every thread of the work-group, joined: op over the lanes of a wave, then over the waves.
template <int TH, class T, class Op>
__device__ __forceinline__ T join_threads(T v, T* scratch, Op op) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v = op(v, __shfl_xor(v, d));
  if constexpr (TH > 64) {
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
    __syncthreads();
    v = scratch[0];
#pragma unroll
    for (int w = 1; w < TH / 64; ++w) v = op(v, scratch[w]);
  }
  return v;
}

// TH threads a row, CH chunks of 8 values each.  Every read of a row comes before the first write to it, so
// out and residual_out may be x or residual.
template <int TH, int CH, bool ANY, bool E4M3>
__global__ __launch_bounds__(TH) void add_rms_norm_kernel(const uint16_t* x, int64_t x_stride, const uint16_t* residual,
                                                          uint16_t* residual_out, const uint16_t* __restrict__ weight,
                                                          int hidden, float eps, void* out, float* scales) {
  __shared__ float sum_of[TH / 64], again_of[TH / 64];
  __shared__ uint32_t top_of[TH / 64];
  const int64_t row = blockIdx.x;
  const uint16_t* xr = x + row * x_stride;
  u32x4_t xv[CH], rv[CH], wv[CH];
#pragma unroll
  for (int c = 0; c < CH; ++c) xv[c] = norm_load<TH, ANY>(xr, c, hidden);
  if (residual != nullptr) {
#pragma unroll
    for (int c = 0; c < CH; ++c) rv[c] = norm_load<TH, ANY>(residual + row * hidden, c, hidden);
  }
#pragma unroll
  for (int c = 0; c < CH; ++c) wv[c] = norm_load<TH, ANY>(weight, c, hidden);
  float h[CH][8];
  float ss = 0.f;
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      h[c][j] = bf16_to_f32(xv[c][j / 2] >> (16 * (j % 2)));
      if (residual != nullptr) h[c][j] += bf16_to_f32(rv[c][j / 2] >> (16 * (j % 2)));
      ss = fmaf(h[c][j], h[c][j], ss);
    }
  ss = join_threads<TH>(ss, sum_of, [](float a, float b) { return a + b; });
  if (residual_out != nullptr) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      u32x4_t v;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = pack_bf16(h[c][2 * j], h[c][2 * j + 1]);
      norm_store<TH, ANY>(residual_out + row * hidden, c, hidden, v);
    }
  }
  // Where eps >= 2^-80 what squares below 2^-126 lose does not count beside it.  A row times 2^80 is exact and stays so; times
  // 2^-80 its small values would lose bits, which y's factor takes up in the place.
  float down = 1.f;
  if (ss > kNormLargeSum || (ss < kNormSmallSum && eps < kNormSmallSum)) {        // (uniform, and not for a NaN)
    const float f = ss > kNormLargeSum ? kNormDown : kNormUp;
    ss = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float hf = h[c][j] * f;
        ss = fmaf(hf, hf, ss);
        if (f == kNormUp) h[c][j] = hf;
      }
    ss = join_threads<TH>(ss, again_of, [](float a, float b) { return a + b; });
    eps = eps * f * f;
    if (f == kNormDown) down = f;
  }
  const float r = 1.f / sqrtf(ss / static_cast<float>(hidden) + eps);
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int j = 0; j < 8; ++j) h[c][j] = h[c][j] * r * down * bf16_to_f32(wv[c][j / 2] >> (16 * (j % 2)));
  if constexpr (!E4M3) {
    auto* o = static_cast<uint16_t*>(out) + row * hidden;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      u32x4_t v;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = pack_bf16(h[c][2 * j], h[c][2 * j + 1]);
      norm_store<TH, ANY>(o, c, hidden, v);
    }
  } else {
    // the largest magnitude by its bits, in which a NaN is above all numbers: it makes the row's scale NaN
    uint32_t top = 0;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int j = 0; j < 8; ++j) top = max(top, __builtin_bit_cast(uint32_t, h[c][j]) & 0x7FFFFFFFu);
    top = join_threads<TH>(top, top_of, [](uint32_t a, uint32_t b) { return max(a, b); });
    float scale = __builtin_bit_cast(float, top) / 448.f;
    if (scale < kNormMinScale) scale = 0.f;
    if (threadIdx.x == 0) scales[row] = scale;
    // y / scale as a product with 1 / scale: off by 1.5 steps of fp32 from the quotient, far below e4m3's
    const float inv = scale == 0.f ? 0.f : 1.f / scale;
    auto* o = static_cast<uint8_t*>(out) + row * hidden;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      uint32_t w[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        float e[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float v = h[c][4 * k + j] * inv;
          e[j] = v != v ? v : fminf(fmaxf(v, -448.f), 448.f);
        }
        int b = __builtin_amdgcn_cvt_pk_fp8_f32(e[0], e[1], 0, false);
        w[k] = __builtin_amdgcn_cvt_pk_fp8_f32(e[2], e[3], b, true);
      }
      const int at = norm_at<TH>(c);
      const uint2 codes = make_uint2(w[0], w[1]);
      if constexpr (ANY) {
        if (at + 8 <= hidden) {
          __builtin_memcpy(o + at, &codes, 8);
        } else {
#pragma unroll
          for (int j = 0; j < 7; ++j)
            if (at + j < hidden) o[at + j] = static_cast<uint8_t>(w[j / 4] >> (8 * (j % 4)));
        }
      } else {
        if (at < hidden) *reinterpret_cast<uint2*>(o + at) = codes;
      }
    }
  }
}

template <bool ANY, bool E4M3>
void add_rms_norm_launch(const uint16_t* x, int64_t x_stride, const uint16_t* residual, uint16_t* residual_out,
                         const uint16_t* weight, int64_t n_tokens, int hidden, float eps, void* out, float* scales,
                         hipStream_t st) {
  const int chunks = (hidden + 7) / 8;
  auto go = [&](auto th, auto ch) {
    constexpr int TH = decltype(th)::value, CH = decltype(ch)::value;
    for (int64_t r = 0; r < n_tokens; r += kNormMaxRows)
      hipLaunchKernelGGL((add_rms_norm_kernel<TH, CH, ANY, E4M3>), dim3(static_cast<unsigned>(std::min(n_tokens - r, kNormMaxRows))),
                         dim3(TH), 0, st, x + r * x_stride, x_stride, residual == nullptr ? nullptr : residual + r * hidden,
                         residual_out == nullptr ? nullptr : residual_out + r * hidden, weight, hidden, eps,
                         static_cast<char*>(out) + r * hidden * (E4M3 ? 1 : 2), E4M3 ? scales + r : nullptr);
  };
  using std::integral_constant;
  using I1 = integral_constant<int, 1>;
  using I2 = integral_constant<int, 2>;
  using I4 = integral_constant<int, 4>;
  using I5 = integral_constant<int, 5>;
  using T64 = integral_constant<int, 64>;
  using T128 = integral_constant<int, 128>;
  using T256 = integral_constant<int, 256>;
  using T512 = integral_constant<int, 512>;
  using T1024 = integral_constant<int, 1024>;
  // Few rows: a chunk to a thread, so that a row's round trips are short (64 x 4096 2.9 us inside a graph, 3.3 with four chunks;
  // 256 x 4096 3.4 and 3.8; 512 x 5120 the same).  Otherwise the fewest threads that hold the row with four or five chunks each:
  // a work-group then has its loads, up to 15 of 16 bytes a thread, in flight at once, and fewer waves to join (5120 values on
  // 128 threads: no chunk idle).
  if (n_tokens <= 256 && chunks > 64 && chunks <= 1024) {
    if (chunks <= 128) go(T128{}, I1{});
    else if (chunks <= 256) go(T256{}, I1{});
    else if (chunks <= 512) go(T512{}, I1{});
    else go(T1024{}, I1{});
    return;
  }
  if (chunks <= 64) go(T64{}, I1{});
  else if (chunks <= 128) go(T64{}, I2{});
  else if (chunks <= 256) go(T64{}, I4{});
  else if (chunks <= 512) go(T128{}, I4{});
  else if (chunks <= 640) go(T128{}, I5{});
  else if (chunks <= 1024) go(T256{}, I4{});
  else if (chunks <= 2048) go(T512{}, I4{});
  else go(T1024{}, I4{});
}

}  // namespace

extern "C" int32_t arckv_add_rms_norm(const void* x, int64_t x_stride, const void* residual, void* residual_out,
                                      const void* weight, int64_t n_tokens, int32_t hidden, float eps, void* out,
                                      int32_t out_format, float* scales, void* stream) {
  if (n_tokens < 0 || n_tokens > INT32_MAX || hidden < 1 || x_stride < hidden || !std::isfinite(eps) || eps < 0.f)
    return arckv::fail(ARCKV_EINVAL, "add_rms_norm: bad sizes or eps");
  if (out_format != ARCKV_OUT_BF16 && out_format != ARCKV_OUT_E4M3)
    return arckv::fail(ARCKV_EINVAL, "add_rms_norm: out_format %d", out_format);
  if (hidden > kNormMaxHidden)
    return arckv::fail(ARCKV_EUNSUPPORTED, "add_rms_norm: hidden %d > %d", hidden, kNormMaxHidden);
  if ((residual == nullptr) != (residual_out == nullptr))
    return arckv::fail(ARCKV_EINVAL, "add_rms_norm: residual and residual_out go together");
  if (n_tokens == 0) return ARCKV_OK;
  const bool e4m3 = out_format == ARCKV_OUT_E4M3;
  if (x == nullptr || weight == nullptr || out == nullptr || (e4m3 && scales == nullptr))
    return arckv::fail(ARCKV_EINVAL, "add_rms_norm: NULL pointer");
  // outputs in the place of an input: only where a work-group writes what it alone has read, and not two in one place
  const bool apart = x_stride != hidden && n_tokens > 1;
  if (out == residual_out || (apart && (out == x || (residual_out != nullptr && residual_out == x))) ||
      (e4m3 && (out == x || out == residual)))
    return arckv::fail(ARCKV_EINVAL, "add_rms_norm: out, residual_out and the inputs overlap");
  uintptr_t all = reinterpret_cast<uintptr_t>(scales);
  if (all % 4 != 0) return arckv::fail(ARCKV_EINVAL, "add_rms_norm: scales must be 4-byte aligned");
  all = 0;
  for (const void* p : {x, residual, static_cast<const void*>(residual_out), weight}) all |= reinterpret_cast<uintptr_t>(p);
  if (all % 2 != 0 || (!e4m3 && reinterpret_cast<uintptr_t>(out) % 2 != 0))
    return arckv::fail(ARCKV_EINVAL, "add_rms_norm: rows must be 2-byte aligned");
  all |= static_cast<uintptr_t>(x_stride) * 2 | reinterpret_cast<uintptr_t>(out);
  const bool any = all % 16 != 0 || hidden % 8 != 0;
  auto run = [&](auto f) {
    f(static_cast<const uint16_t*>(x), x_stride, static_cast<const uint16_t*>(residual), static_cast<uint16_t*>(residual_out),
      static_cast<const uint16_t*>(weight), n_tokens, hidden, eps, out, scales, static_cast<hipStream_t>(stream));
  };
  if (e4m3) {
    if (any) run(add_rms_norm_launch<true, true>); else run(add_rms_norm_launch<false, true>);
  } else {
    if (any) run(add_rms_norm_launch<true, false>); else run(add_rms_norm_launch<false, false>);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return arckv::fail(ARCKV_EDEVICE, "add_rms_norm: %s", hipGetErrorString(e));
  return ARCKV_OK;
}
