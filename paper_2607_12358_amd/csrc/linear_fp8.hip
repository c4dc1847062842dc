// Products of e4m3 rows and e4m3 weights with block scales (acid_linear_fp8):
//
//   y[m][n] = sum_b sa[b][m] sw[n / 128][b] (sum_{k in block b} a[m][k] w[n][k]) + bias[n]
//
// over blocks b of 128 inputs, and out = y, GELU(y) or residual + gate (.) y.  A
// block's inner sum starts from zero, and one fused multiply-add per value adds it to
// the fp32 accumulator with the block's scales.  The weights feed the matrix
// instruction's first operand, so a lane's results are one token's: its scale is one
// register.
//
// Two forms of the inner sum.  The 8-bit matrix instructions add eight neighbouring
// products at a time, aligned to the largest of them and cut below 2^-13 of it
// (measured; both the 32x32x64 and the older 32x32x16 do): random operands give sums
// that are 1.4e-5 off, against 2^-9 for the rounding to bf16 that follows and some 2^-5
// for the operands' own.  Outputs in bf16, and updates of a residual, take them.
// Plain fp32 outputs take the bf16 instruction on operands converted on the way, which
// is exact: products and sums in fp32.
#include <type_traits>

#include "fp8.h"

namespace acid {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

struct Fp8Args {
  const uint8_t *a, *w;
  const float *a_scales, *w_scales, *bias, *gate, *residual;
  void* out;
  int64_t a_ld, a_scales_ld, residual_ld, out_ld;
  int32_t M, N, K, groups, kind;
};

__device__ __forceinline__ f32x16 mfma64(const i32x8& w, const i32x8& a, const f32x16& c) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w, a, c, 0, 0, 0, 0, 0, 0);
}

// One output value out of its sum.
template <typename Out>
__device__ __forceinline__ Out finish(const Fp8Args& a, float y, int64_t m, int n) {
  if (a.bias) y += a.bias[n];
  if (a.kind == ACID_EPI_BIAS_GELU) {
    if constexpr (std::is_same_v<Out, bf16>)
      y = gelu_tanh_fast(y);
    else
      y = gelu_tanh(y);
  } else if (a.kind == ACID_EPI_GATE_RESIDUAL) {
    y = fmaf(a.gate[n], y, a.residual[m * a.residual_ld + n]);
  }
  return (Out)y;
}

// Sixteen e4m3 values as bf16.
__device__ __forceinline__ void to_bf16(const u32x4& c, bf16x8 (&v)[2]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const auto lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[i], 1.0f, false);
    const auto hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[i], 1.0f, true);
    v[i / 2][4 * (i % 2)] = lo[0];
    v[i / 2][4 * (i % 2) + 1] = lo[1];
    v[i / 2][4 * (i % 2) + 2] = hi[0];
    v[i / 2][4 * (i % 2) + 3] = hi[1];
  }
}

// 64 x 64 outputs a workgroup, 32 x 32 a wave, operands from global memory.
template <typename Out, bool EXACT>
__global__ __launch_bounds__(256) void linear_fp8_kernel(Fp8Args a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int lr = lane & 31, lg = lane >> 5;
  const int64_t m = (int64_t)blockIdx.x * 64 + (wave & 1) * 32 + lr;
  const int n0 = blockIdx.y * 64 + (wave >> 1) * 32;
  const int64_t mc = m < a.M ? m : a.M - 1;
  const int nc = n0 + lr < a.N ? n0 + lr : a.N - 1;
  const int nb = (n0 < a.N ? n0 : a.N - 1) / kFp8Group;
  f32x16 acc = {};
  for (int g = 0; g < a.groups; ++g) {
    u32x4 fw[4], fa[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int k = g * kFp8Group + 32 * j + 16 * lg;
      const bool in = k < a.K;  // K is whole 16s
      fw[j] = in ? *reinterpret_cast<const u32x4*>(a.w + (int64_t)nc * a.K + k) : u32x4{0, 0, 0, 0};
      fa[j] = in ? *reinterpret_cast<const u32x4*>(a.a + mc * a.a_ld + k) : u32x4{0, 0, 0, 0};
    }
    f32x16 sum = {};
    if constexpr (EXACT) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        bf16x8 bw[2], ba[2];
        to_bf16(fw[j], bw);
        to_bf16(fa[j], ba);
#pragma unroll
        for (int i = 0; i < 2; ++i)
          sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bw[i], ba[i], sum, 0, 0, 0);
      }
    } else {
      struct Pair { u32x4 v[2]; };
      sum = mfma64(__builtin_bit_cast(i32x8, Pair{fw[0], fw[1]}),
                   __builtin_bit_cast(i32x8, Pair{fa[0], fa[1]}), sum);
      sum = mfma64(__builtin_bit_cast(i32x8, Pair{fw[2], fw[3]}),
                   __builtin_bit_cast(i32x8, Pair{fa[2], fa[3]}), sum);
    }
    const float s = a.a_scales[g * a.a_scales_ld + mc] * a.w_scales[(int64_t)nb * a.groups + g];
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = fmaf(s, sum[r], acc[r]);
  }
  if (m >= a.M) return;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int n = n0 + 8 * (r >> 2) + 4 * lg + (r & 3);
    if (n < a.N) ((Out*)a.out)[m * a.out_ld + n] = finish<Out>(a, acc[r], m, n);
  }
}

}  // namespace
}  // namespace acid

using namespace acid;

extern "C" {

size_t acid_linear_fp8_workspace_needed(int64_t M, int32_t N, int32_t K) {
  (void)M;
  (void)N;
  (void)K;
  return 0;
}

acid_status acid_linear_fp8(const acid_linear_fp8_args* args, int64_t M, int32_t N, int32_t K,
                            hipStream_t stream) {
  if (!args) return set_error(ACID_ERR_INVALID_ARG, "NULL argument");
  const acid_linear_fp8_args& p = *args;
  if (p.out_dtype != ACID_F32 && p.out_dtype != ACID_BF16)
    return set_error(ACID_ERR_INVALID_ARG, "bad dtype %d", p.out_dtype);
  const bool update = p.kind == ACID_EPI_GATE_RESIDUAL;
  if (p.kind != ACID_EPI_BIAS && p.kind != ACID_EPI_BIAS_GELU && !update)
    return set_error(ACID_ERR_UNSUPPORTED, "fp8: epilogue %d is not BIAS, BIAS_GELU or GATE_RESIDUAL", p.kind);
  if (update && p.out_dtype != ACID_F32)
    return set_error(ACID_ERR_UNSUPPORTED, "fp8: GATE_RESIDUAL writes fp32");
  if (M < 0 || N < 1 || K < 1) return set_error(ACID_ERR_INVALID_ARG, "M < 0, N < 1 or K < 1");
  constexpr int64_t most = (int64_t)1 << 32;
  if (K % 16 || K > (1 << 22) || N > (1 << 22) || M > (1 << 24))
    return set_error(ACID_ERR_SHAPE, "fp8: K %d must be a multiple of 16, K and N <= 2^22, M <= 2^24", K);
  if (p.a_ld < K || p.a_ld % 16 || p.a_ld >= (1 << 24) || p.out_ld < N || p.out_ld > most ||
      (update && (p.residual_ld < N || p.residual_ld > most)))
    return set_error(ACID_ERR_SHAPE, "fp8: a_ld >= K, whole 16 bytes and < 2^24, out_ld and residual_ld >= N and <= 2^32");
  if (p.a_scales_ld < round_up(M, 4) || p.a_scales_ld % 4 || p.a_scales_ld > most)
    return set_error(ACID_ERR_SHAPE, "fp8: a_scales_ld >= round_up(M, 4), a multiple of 4");
  if (M == 0) return ACID_OK;
  if (!p.a || !p.w || !p.a_scales || !p.w_scales || !p.out || (update && (!p.gate || !p.residual)))
    return set_error(ACID_ERR_INVALID_ARG, "NULL argument");
  const int64_t os = p.out_dtype == ACID_BF16 ? 2 : 4;
  if (((uintptr_t)p.a | (uintptr_t)p.w | (uintptr_t)p.a_scales) % 16 || (uintptr_t)p.out % os ||
      ((uintptr_t)p.w_scales | (uintptr_t)p.bias | (update ? (uintptr_t)p.gate | (uintptr_t)p.residual : 0)) % 4)
    return set_error(ACID_ERR_INVALID_ARG, "fp8: a, its scales and w must be 16-byte aligned, the rest to an element");
  const int64_t groups = fp8_groups(K);
  const size_t need = acid_linear_fp8_workspace_needed(M, N, K);
  if (p.workspace_bytes < need)
    return set_error(ACID_ERR_SHAPE, "fp8: workspace of %zu bytes, %zu needed", p.workspace_bytes, need);
  if (need && (!p.workspace || (uintptr_t)p.workspace % 16))
    return set_error(ACID_ERR_INVALID_ARG, "fp8: workspace is NULL or not 16-byte aligned");
  const struct {
    const void* p;
    int64_t rows, width, ld;
  } in[] = {{p.a, M, K, p.a_ld},
            {p.w, 1, (int64_t)N * K, (int64_t)N * K},
            {p.a_scales, groups, M * 4, p.a_scales_ld * 4},
            {p.w_scales, 1, fp8_groups(N) * groups * 4, fp8_groups(N) * groups * 4},
            {p.bias, 1, (int64_t)N * 4, (int64_t)N * 4},
            {update ? p.gate : nullptr, 1, (int64_t)N * 4, (int64_t)N * 4},
            {update ? p.residual : nullptr, M, (int64_t)N * 4, p.residual_ld * 4}};
  for (const auto& i : in) {
    // the residual may be updated in place
    const bool same = update && i.p == p.residual && p.out == p.residual && p.out_ld == p.residual_ld;
    if (!same && rows_overlap(p.out, M, N * os, p.out_ld * os, i.p, i.rows, i.width, i.ld))
      return set_error(ACID_ERR_INVALID_ARG, "fp8: out overlaps an input");
    if (need && rows_overlap(p.workspace, 1, need, need, i.p, i.rows, i.width, i.ld))
      return set_error(ACID_ERR_INVALID_ARG, "fp8: workspace overlaps an input");
  }
  if (need && rows_overlap(p.workspace, 1, need, need, p.out, M, N * os, p.out_ld * os))
    return set_error(ACID_ERR_INVALID_ARG, "fp8: workspace overlaps out");
  StreamDevice on;
  ACID_TRY(on.enter(stream));
  const Fp8Args a = {(const uint8_t*)p.a, (const uint8_t*)p.w, p.a_scales, p.w_scales, p.bias, p.gate,
                     p.residual, p.out, p.a_ld, p.a_scales_ld, p.residual_ld, p.out_ld, (int32_t)M, N,
                     K, (int32_t)groups, p.kind};
  const dim3 grid((unsigned)((M + 63) / 64), (unsigned)((N + 63) / 64));
  if (p.out_dtype == ACID_BF16)
    hipLaunchKernelGGL((linear_fp8_kernel<bf16, false>), grid, dim3(256), 0, stream, a);
  else if (update)
    hipLaunchKernelGGL((linear_fp8_kernel<float, false>), grid, dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL((linear_fp8_kernel<float, true>), grid, dim3(256), 0, stream, a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? ACID_OK : check_hip(e, "linear fp8");
}

}  // extern "C"
