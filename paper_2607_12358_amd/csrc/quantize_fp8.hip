// fp32 and bf16 values into e4m3 codes with a scale for each group of 128:
// activations by row (acid_quantize_fp8), LN-modulated rows
// (acid_ln_modulate_fp8) and weights by 128 x 128 block
// (acid_quantize_fp8_weight).
//
//   scale = max(max |x| / 448, 2^-126),  code = e4m3(x (1 / scale))
//
// Each is bound by HBM: every value is read once, held in registers while
// the group's largest is found, and written as one byte.
#include <algorithm>
#include <type_traits>

#include "fp8.h"

namespace acid {
namespace {

// ------------------------------------------------------------------- rows

struct RowsArgs {
  const void* x;
  uint8_t* codes;
  float* scales;
  int64_t x_ld, codes_ld, scales_ld, rows;
  int32_t K, groups;
};

// Eight neighbouring values as they were loaded.
template <typename T>
struct Eight;
template <>
struct Eight<bf16> {
  u32x4 w;
  __device__ __forceinline__ void load(const bf16* p) { w = *reinterpret_cast<const u32x4*>(p); }
  __device__ __forceinline__ void values(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
};
template <>
struct Eight<float> {
  f32x4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = *reinterpret_cast<const f32x4*>(p);
    b = *reinterpret_cast<const f32x4*>(p + 4);
  }
  __device__ __forceinline__ void values(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i] = a[i];
      v[4 + i] = b[i];
    }
  }
};

// A wave takes one group of 4 QUADS rows: sixteen lanes and eight values a lane to a row's
// group, four rows an instruction, all of them loaded before the first is used.  32760 bf16
// rows of 1536, 153 MB: 32 us, 4.7 TB/s; 77 fp32 rows of 1040: 2.0 us with four rows a wave, 4.5
// with 32, one quad after the other.
template <typename X, int QUADS>
__global__ __launch_bounds__(256) void quantize_fp8_rows_kernel(RowsArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t tile = item / a.groups;
  const int group = (int)(item - tile * a.groups);
  const int64_t row0 = tile * (4 * QUADS) + (lane >> 4);
  if (row0 - (lane >> 4) >= a.rows) return;
  const int k = group * kFp8Group + (lane & 15) * 8;
  const bool live = k < a.K;
  Eight<X> held[QUADS];
#pragma unroll
  for (int q = 0; q < QUADS; ++q)
    held[q].load((const X*)a.x + std::min(row0 + 4 * q, a.rows - 1) * a.x_ld + (live ? k : 0));
#pragma unroll
  for (int q = 0; q < QUADS; ++q) {
    const int64_t row = row0 + 4 * q;
    float v[8];
    held[q].values(v);
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = live ? v[i] : 0.f;
      most = max(most, abs_bits(v[i]));
    }
    const Fp8Scale s(row16_max(most));
    if (row < a.rows) {
      if (live) {
        uint2 w;
        w.x = to_fp8(v[0] * s.inv, v[1] * s.inv, v[2] * s.inv, v[3] * s.inv);
        w.y = to_fp8(v[4] * s.inv, v[5] * s.inv, v[6] * s.inv, v[7] * s.inv);
        *reinterpret_cast<uint2*>(a.codes + row * a.codes_ld + k) = w;
      }
      if ((lane & 15) == 0) a.scales[group * a.scales_ld + row] = s.scale;
    }
  }
}

template <typename X, int QUADS>
hipError_t launch_rows(const RowsArgs& a, hipStream_t s) {
  const int64_t items = (a.rows + 4 * QUADS - 1) / (4 * QUADS) * a.groups;
  hipLaunchKernelGGL((quantize_fp8_rows_kernel<X, QUADS>), dim3((unsigned)((items + 3) / 4)), dim3(256), 0, s, a);
  return hipGetLastError();
}

// ------------------------------------------------------------ LN-modulate

struct LnArgs {
  const float *x, *shift, *scale;
  uint8_t* codes;
  float* scales;
  int64_t x_ld, codes_ld, scales_ld, rows, rows_per_mod;
  int32_t hidden;
};

// Sum over the WAVES waves of a row.
template <int WAVES>
__device__ __forceinline__ float row_sum(float v, float* part) {
  v = lane_sum(v);
  if constexpr (WAVES > 1) {
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) v += part[w];
  }
  return v;
}

// A row a workgroup of WAVES waves, four values a lane at a time: 32 lanes hold a
// group.  Statistics in fp32, in two passes over the registers.  32760 rows of 1536, 253
// MB: 53 us, 4.8 TB/s, 47 of it without the modulation's vectors, which each row reads again
// from L2, and the scales, four bytes to a line.  (Two rows a workgroup that share both take
// as long, runs of eight with the next in flight 62; two or four waves a row 54 and 62.)  7
// rows of 4096: 3.4 us with four waves, 4.4 with two.
template <int WAVES, int CHUNKS>
__global__ __launch_bounds__(64 * WAVES) void ln_modulate_fp8_kernel(LnArgs a) {
  __shared__ float part[2][WAVES];
  const int64_t row = blockIdx.x, mod = a.rows_per_mod ? row / a.rows_per_mod * a.hidden : 0;
  const int tid = threadIdx.x, n4 = a.hidden / 4;
  const float inv_n = 1.0f / (float)a.hidden;
  auto inside = [&](int c) { return tid + 64 * WAVES * c < n4; };
  f32x4 v[CHUNKS], scale[CHUNKS], shift[CHUNKS];
  auto read = [&](f32x4 (&to)[CHUNKS], const float* from) {  // threads past the row's end: copies
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
      to[c] = *reinterpret_cast<const f32x4*>(from + 4 * (inside(c) ? tid + 64 * WAVES * c : 0));
  };
  read(v, a.x + row * a.x_ld);
  read(scale, a.scale + mod);
  read(shift, a.shift + mod);
  float sum = 0.f, squares = 0.f;
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) sum += inside(c) ? (v[c][0] + v[c][1]) + (v[c][2] + v[c][3]) : 0.f;
  const float mean = row_sum<WAVES>(sum, part[0]) * inv_n;
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[c][e] -= mean;
    const f32x4 q = v[c] * v[c];
    squares += inside(c) ? (q[0] + q[1]) + (q[2] + q[3]) : 0.f;
  }
  const float r = 1.0f / sqrtf(row_sum<WAVES>(squares, part[1]) * inv_n + 1e-6f);
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    const int i = tid + 64 * WAVES * c;
    f32x4 y;
    uint32_t most = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      y[e] = inside(c) ? fmaf(v[c][e] * r, 1.0f + scale[c][e], shift[c][e]) : 0.f;
      most = max(most, abs_bits(y[e]));
    }
    most = row16_max(most);
    const auto both = __builtin_amdgcn_permlane16_swap(most, most, false, false);  // the row of 16 lanes beside
    const Fp8Scale s(max(both[0], both[1]));
    if (inside(c)) {
      *reinterpret_cast<uint32_t*>(a.codes + row * a.codes_ld + 4 * i) =
          to_fp8(y[0] * s.inv, y[1] * s.inv, y[2] * s.inv, y[3] * s.inv);
      if (i % 32 == 0) a.scales[i / 32 * a.scales_ld + row] = s.scale;
    }
  }
}

template <int WAVES>
hipError_t launch_ln(const LnArgs& a, hipStream_t s) {
  const int chunks = (a.hidden / 4 + 64 * WAVES - 1) / (64 * WAVES);
#define LN(C) hipLaunchKernelGGL((ln_modulate_fp8_kernel<WAVES, C>), dim3((unsigned)a.rows), dim3(64 * WAVES), 0, s, a)
  if (chunks <= 2) LN(2);
  else if (chunks <= 4) LN(4);
  else if (chunks <= 6) LN(6);
  else LN(8);
#undef LN
  return hipGetLastError();
}

// ---------------------------------------------------------------- weights

// One 128 x 128 block a workgroup: thread t holds outputs t % 128 of 64
// inputs, half t / 128 of the block.  8960 x 1536, 69 MB: 15.5 us, 4.4 TB/s.
__global__ __launch_bounds__(256) void quantize_fp8_weight_kernel(const float* __restrict__ w, int N,
                                                                  int K, uint8_t* __restrict__ codes,
                                                                  float* __restrict__ scales) {
  __shared__ uint32_t part[4];
  const int col = threadIdx.x & 127, half = threadIdx.x >> 7;
  const int n = blockIdx.y * 128 + col, k0 = blockIdx.x * 128 + half * 64;
  const int left = std::min(64, K - k0);
  const float* p = w + (int64_t)k0 * N + n;
  float v[64];
  uint32_t most = 0;
#pragma unroll
  for (int j = 0; j < 64; ++j) {
    v[j] = n < N && j < left ? p[(int64_t)j * N] : 0.f;
    most = max(most, abs_bits(v[j]));
  }
  most = row16_max(most);
  most = max(most, (uint32_t)__shfl_xor((int)most, 16, 64));
  most = max(most, (uint32_t)__shfl_xor((int)most, 32, 64));
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = most;
  __syncthreads();
  const Fp8Scale s(max(max(part[0], part[1]), max(part[2], part[3])));
  if (threadIdx.x == 0) scales[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = s.scale;
  if (n >= N) return;
  uint8_t* out = codes + (int64_t)n * K + k0;
#pragma unroll
  for (int j = 0; j < 64; j += 16) {
    if (j >= left) break;  // K is whole 16s
    u32x4 c;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      c[e] = to_fp8(v[j + 4 * e] * s.inv, v[j + 4 * e + 1] * s.inv, v[j + 4 * e + 2] * s.inv,
                    v[j + 4 * e + 3] * s.inv);
    *reinterpret_cast<u32x4*>(out + j) = c;
  }
}

// What every call on e4m3 rows asks of their layout; of their number, that quantize_fp8_rows_kernel's
// workgroups, four of those 32 x 128 tiles each, have fewer than 2^32 threads in all.
acid_status check_rows(int64_t rows, int64_t K, int64_t x_ld, int64_t x_size, int64_t codes_ld,
                       int64_t scales_ld) {
  if (rows < 0 || K < 1) return set_error(ACID_ERR_INVALID_ARG, "fp8: rows < 0 or K < 1");
  if (K % 16 || K > (1 << 22) || (rows + 31) / 32 * fp8_groups(K) >= (1 << 26) - 3)
    return set_error(ACID_ERR_SHAPE,
                     "fp8: K %lld must be a multiple of 16, <= 2^22, and ceil(rows / 32) "
                     "ceil(K / 128) < 2^26 - 3", (long long)K);
  constexpr int64_t most = (int64_t)1 << 32;
  if (x_ld < K || x_ld * x_size % 16 || x_ld > most || codes_ld < K || codes_ld % 16 ||
      codes_ld > most)
    return set_error(ACID_ERR_SHAPE, "fp8: rows at least K apart, whole 16 bytes, at most 2^32");
  // (no rows have no scales: an empty matrix's stride means nothing)
  if (rows > 0 && (scales_ld < round_up(rows, 4) || scales_ld % 4 || scales_ld > most))
    return set_error(ACID_ERR_SHAPE, "fp8: scales' rows are round_up(rows, 4) or more apart, a multiple of 4");
  return ACID_OK;
}

struct Range {
  const void* p;
  int64_t rows, width, ld;
};
acid_status check_apart(const Range& x, std::initializer_list<Range> more, const Range& codes,
                        const Range& scales) {
  auto overlap = [](const Range& a, const Range& b) {
    return rows_overlap(a.p, a.rows, a.width, a.ld, b.p, b.rows, b.width, b.ld);
  };
  bool bad = overlap(codes, scales) || overlap(x, codes) || overlap(x, scales);
  for (const Range& m : more) bad = bad || overlap(m, codes) || overlap(m, scales);
  return bad ? set_error(ACID_ERR_INVALID_ARG, "fp8: codes or scales overlap another buffer") : ACID_OK;
}

}  // namespace
}  // namespace acid

using namespace acid;

extern "C" {

acid_status acid_quantize_fp8(int32_t x_dtype, int64_t rows, int32_t K, const void* x_dev,
                              int64_t x_ld, void* codes_dev, int64_t codes_ld, float* scales_dev,
                              int64_t scales_ld, hipStream_t stream) {
  if (x_dtype != ACID_F32 && x_dtype != ACID_BF16)
    return set_error(ACID_ERR_INVALID_ARG, "bad dtype %d", x_dtype);
  const int64_t size = x_dtype == ACID_BF16 ? 2 : 4;
  ACID_TRY(check_rows(rows, K, x_ld, size, codes_ld, scales_ld));
  if (rows == 0) return ACID_OK;
  if (!x_dev || !codes_dev || !scales_dev) return set_error(ACID_ERR_INVALID_ARG, "NULL argument");
  if (((uintptr_t)x_dev | (uintptr_t)codes_dev | (uintptr_t)scales_dev) % 16)
    return set_error(ACID_ERR_INVALID_ARG, "fp8: x, codes and scales must be 16-byte aligned");
  const int64_t groups = fp8_groups(K);
  ACID_TRY(check_apart({x_dev, rows, K * size, x_ld * size}, {}, {codes_dev, rows, K, codes_ld},
                       {scales_dev, groups, rows * 4, scales_ld * 4}));
  StreamDevice on;
  ACID_TRY(on.enter(stream));
  const RowsArgs a = {x_dev, (uint8_t*)codes_dev, scales_dev, x_ld, codes_ld, scales_ld, rows, K,
                      (int32_t)groups};
  // 32 rows a wave where that leaves each SIMD two waves, else four
  const bool many = (rows + 31) / 32 * groups >= 8 * device_cus();
  hipError_t e;
  if (x_dtype == ACID_BF16)
    e = many ? launch_rows<bf16, 8>(a, stream) : launch_rows<bf16, 1>(a, stream);
  else
    e = many ? launch_rows<float, 8>(a, stream) : launch_rows<float, 1>(a, stream);
  return e == hipSuccess ? ACID_OK : check_hip(e, "quantize fp8");
}

acid_status acid_ln_modulate_fp8(int64_t rows, int32_t hidden, const float* x_dev, int64_t x_ld,
                                 const float* shift_dev, const float* scale_dev,
                                 int64_t rows_per_mod, void* codes_dev, int64_t codes_ld,
                                 float* scales_dev, int64_t scales_ld, hipStream_t stream) {
  ACID_TRY(check_rows(rows, hidden, x_ld, 4, codes_ld, scales_ld));
  if (hidden > 8192 || rows > (1 << 23))
    return set_error(ACID_ERR_SHAPE, "fp8: hidden <= 8192, rows <= 2^23");
  if (rows_per_mod < 0) return set_error(ACID_ERR_INVALID_ARG, "rows_per_mod < 0");
  if (rows == 0) return ACID_OK;
  if (!x_dev || !shift_dev || !scale_dev || !codes_dev || !scales_dev)
    return set_error(ACID_ERR_INVALID_ARG, "NULL argument");
  if (((uintptr_t)x_dev | (uintptr_t)shift_dev | (uintptr_t)scale_dev | (uintptr_t)codes_dev |
       (uintptr_t)scales_dev) % 16)
    return set_error(ACID_ERR_INVALID_ARG, "fp8: every buffer must be 16-byte aligned");
  const int64_t mods = rows_per_mod ? (rows + rows_per_mod - 1) / rows_per_mod : 1, mb = mods * hidden * 4;
  ACID_TRY(check_apart({x_dev, rows, (int64_t)hidden * 4, x_ld * 4},
                       {{shift_dev, 1, mb, mb}, {scale_dev, 1, mb, mb}},
                       {codes_dev, rows, hidden, codes_ld},
                       {scales_dev, fp8_groups(hidden), rows * 4, scales_ld * 4}));
  StreamDevice on;
  ACID_TRY(on.enter(stream));
  const LnArgs a = {x_dev, shift_dev, scale_dev, (uint8_t*)codes_dev, scales_dev, x_ld, codes_ld,
                    scales_ld, rows, rows_per_mod, hidden};
  // One wave a row where there are two rows a SIMD, four for few rows.
  const bool many = rows >= 8 * device_cus();
  const hipError_t e = hidden <= 2048 && many   ? launch_ln<1>(a, stream)
                       : hidden <= 4096 && many ? launch_ln<2>(a, stream)
                                                : launch_ln<4>(a, stream);
  return e == hipSuccess ? ACID_OK : check_hip(e, "ln modulate fp8");
}

acid_status acid_quantize_fp8_weight(const float* w_dev, int32_t N, int32_t K, void* codes_dev,
                                     float* scales_dev, hipStream_t stream) {
  if (N < 1 || K < 1) return set_error(ACID_ERR_INVALID_ARG, "N and K must be >= 1");
  if (K % 16 || K > (1 << 22) || N > (1 << 22))
    return set_error(ACID_ERR_SHAPE, "fp8: K %d must be a multiple of 16, K and N <= 2^22", K);
  if (!w_dev || !codes_dev || !scales_dev) return set_error(ACID_ERR_INVALID_ARG, "NULL argument");
  if ((uintptr_t)codes_dev % 16 || ((uintptr_t)w_dev | (uintptr_t)scales_dev) % 4)
    return set_error(ACID_ERR_INVALID_ARG, "codes must be 16-byte aligned, w and scales 4-byte");
  const int64_t wb = (int64_t)N * K * 4, cb = (int64_t)N * K, sb = fp8_groups(N) * fp8_groups(K) * 4;
  ACID_TRY(check_apart({w_dev, 1, wb, wb}, {}, {codes_dev, 1, cb, cb}, {scales_dev, 1, sb, sb}));
  StreamDevice on;
  ACID_TRY(on.enter(stream));
  const dim3 grid((unsigned)fp8_groups(K), (unsigned)fp8_groups(N));
  hipLaunchKernelGGL(quantize_fp8_weight_kernel, grid, dim3(256), 0, stream, w_dev, N, K,
                     (uint8_t*)codes_dev, scales_dev);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? ACID_OK : check_hip(e, "quantize fp8 weight");
}

}  // extern "C"
