// The seam between two blocks in one pass over the rows (acid_residual_norm):
//
//   h' = res_scale h + gate (.) (N_post(y) (.) post_weight)
//   out = (N_pre(h') (.) pre_weight) (1 + scale) + shift
//
// N is LayerNorm (biased variance), RMS norm or nothing.  HBM-bound: y and h
// are read once, h' and out written once; a row stays in registers, in fp32,
// between its two norms.
#include <math.h>

#include <type_traits>

#include "common.h"

namespace acid {
namespace {

struct NormArgs {
  const float* h;
  const void* y;
  float* h_out;
  void* out;
  int64_t h_ld, y_ld, h_out_ld, out_ld;
  const float *post_weight, *gate, *pre_weight, *shift, *scale;
  int64_t rows, rows_per_mod;
  int32_t hidden, post, pre;
  float res_scale, eps;
};

struct Absent {};  // no y, or no out

__device__ __forceinline__ float4 load4(const float* p) {
  return *reinterpret_cast<const float4*>(p);
}
__device__ __forceinline__ float4 load4(const bf16* p) {
  const bf16x4 v = *reinterpret_cast<const bf16x4*>(p);
  return make_float4((float)v[0], (float)v[1], (float)v[2], (float)v[3]);
}
__device__ __forceinline__ void store4(float* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }
__device__ __forceinline__ void store4(bf16* p, float4 v) {
  bf16x4 b;
  b[0] = (bf16)v.x;
  b[1] = (bf16)v.y;
  b[2] = (bf16)v.z;
  b[3] = (bf16)v.w;
  *reinterpret_cast<bf16x4*>(p) = b;
}
__device__ __forceinline__ float sum4(float4 v) { return (v.x + v.y) + (v.z + v.w); }
__device__ __forceinline__ float4 mul4(float4 a, float4 b) {
  return make_float4(a.x * b.x, a.y * b.y, a.z * b.z, a.w * b.w);
}

// Sum of v over the WAVES waves of a row; `part` is one LDS array per sum.
template <int WAVES>
__device__ __forceinline__ float row_sum(float v, float* part) {
  v = wave_sum(v);
  if constexpr (WAVES > 1) {
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) v += part[w];
  }
  return v;
}

// v = N(v) (.) weight over a row of H values in CHUNKS float4 per thread.
// Statistics in fp32, in two passes over the registers (mean, then centred
// squares).  Threads past the row's end hold zeros and are left out.
template <int WAVES, int CHUNKS>
__device__ __forceinline__ void normalise(float4 (&v)[CHUNKS], int kind, int tid, int n4, float H,
                                          float eps, const float* __restrict__ weight,
                                          float (*part)[WAVES]) {
  if (kind != ACID_NORM_NONE) {
    float mean = 0.f;
    if (kind == ACID_NORM_LAYER) {
      float s = 0.f;
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c) s += sum4(v[c]);
      mean = row_sum<WAVES>(s, part[0]) / H;
    }
    float q = 0.f;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      v[c] = make_float4(v[c].x - mean, v[c].y - mean, v[c].z - mean, v[c].w - mean);
      const float t = sum4(mul4(v[c], v[c]));
      q += tid + 64 * WAVES * c < n4 ? t : 0.f;
    }
    const float r = 1.0f / sqrtf(row_sum<WAVES>(q, part[1]) / H + eps);
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) v[c] = mul4(v[c], make_float4(r, r, r, r));
  }
  if (weight) {
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      const int i = tid + 64 * WAVES * c;
      if (i < n4) v[c] = mul4(v[c], load4(weight + 4 * i));
    }
  }
}

template <int WAVES, int CHUNKS, typename Y, typename Out>
__global__ __launch_bounds__(256) void residual_norm_kernel(NormArgs a) {
  constexpr int ROWS = 4 / WAVES;  // rows of a workgroup
  __shared__ float part[4][WAVES];
  const int64_t row = (int64_t)blockIdx.x * ROWS + (WAVES == 1 ? threadIdx.x >> 6 : 0);
  const int tid = WAVES == 1 ? threadIdx.x & 63 : threadIdx.x;
  if (row >= a.rows) return;  // whole waves; with WAVES > 1 never
  const int n4 = a.hidden >> 2;
  const int64_t mod = a.rows_per_mod ? row / a.rows_per_mod : 0;
  const float H = (float)a.hidden;

  float4 h[CHUNKS];
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    const int i = tid + 64 * WAVES * c;
    h[c] = i < n4 ? load4(a.h + row * a.h_ld + 4 * i) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  if constexpr (!std::is_same_v<Y, Absent>) {
    float4 y[CHUNKS];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      const int i = tid + 64 * WAVES * c;
      y[c] = i < n4 ? load4((const Y*)a.y + row * a.y_ld + 4 * i)
                    : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    normalise<WAVES, CHUNKS>(y, a.post, tid, n4, H, a.eps, a.post_weight, part);
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      const int i = tid + 64 * WAVES * c;
      if (i < n4) {
        if (a.gate) y[c] = mul4(y[c], load4(a.gate + mod * a.hidden + 4 * i));
        h[c] = make_float4(fmaf(a.res_scale, h[c].x, y[c].x), fmaf(a.res_scale, h[c].y, y[c].y),
                           fmaf(a.res_scale, h[c].z, y[c].z), fmaf(a.res_scale, h[c].w, y[c].w));
        store4(a.h_out + row * a.h_out_ld + 4 * i, h[c]);
      }
    }
  }
  if constexpr (!std::is_same_v<Out, Absent>) {
    normalise<WAVES, CHUNKS>(h, a.pre, tid, n4, H, a.eps, a.pre_weight, part + 2);
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      const int i = tid + 64 * WAVES * c;
      if (i < n4) {
        float4 z = h[c];
        if (a.scale) {
          const float4 m = load4(a.scale + mod * a.hidden + 4 * i);
          z = mul4(z, make_float4(1.f + m.x, 1.f + m.y, 1.f + m.z, 1.f + m.w));
        }
        if (a.shift) {
          const float4 m = load4(a.shift + mod * a.hidden + 4 * i);
          z = make_float4(z.x + m.x, z.y + m.y, z.z + m.z, z.w + m.w);
        }
        store4((Out*)a.out + row * a.out_ld + 4 * i, z);
      }
    }
  }
}

template <typename Y, typename Out>
hipError_t launch(const NormArgs& a, hipStream_t s) {
  const int n4 = a.hidden / 4;
#define RN(W, C)                                                                            \
  hipLaunchKernelGGL((residual_norm_kernel<W, C, Y, Out>),                                  \
                     dim3((unsigned)((a.rows + 4 / W - 1) / (4 / W))), dim3(256), 0, s, a)
  if (n4 <= 64) RN(1, 1);
  else if (n4 <= 128) RN(1, 2);
  else if (n4 <= 256) RN(1, 4);
  else if (n4 <= 384) RN(1, 6);
  else if (n4 <= 512) RN(1, 8);
  else if (n4 <= 1024) RN(4, 4);
  else if (n4 <= 2048) RN(4, 8);
  else RN(4, 16);
#undef RN
  return hipGetLastError();
}

template <typename Y>
hipError_t launch_out(int out_dtype, const NormArgs& a, hipStream_t s) {
  if constexpr (!std::is_same_v<Y, Absent>) {
    if (!a.out) return launch<Y, Absent>(a, s);
  }
  return out_dtype == ACID_BF16 ? launch<Y, bf16>(a, s) : launch<Y, float>(a, s);
}

}  // namespace
}  // namespace acid

using namespace acid;

extern "C" acid_status acid_residual_norm(const acid_residual_norm_args* n, int64_t rows,
                                          int32_t hidden, hipStream_t stream) {
  if (!n) return set_error(ACID_ERR_INVALID_ARG, "residual norm args NULL");
  if (rows < 0) return set_error(ACID_ERR_INVALID_ARG, "rows < 0");
  if (hidden < 4 || hidden % 4 || hidden > 16384)
    return set_error(ACID_ERR_SHAPE, "hidden %d: multiple of 4 in [4, 16384]", hidden);
  if (rows > (int64_t)1 << 23)
    return set_error(ACID_ERR_SHAPE, "rows %lld: at most 2^23", (long long)rows);
  for (int kind : {n->post, n->pre})
    if (kind != ACID_NORM_NONE && kind != ACID_NORM_LAYER && kind != ACID_NORM_RMS)
      return set_error(ACID_ERR_INVALID_ARG, "bad norm kind %d", kind);
  for (int dt : {n->y_dtype, n->out_dtype})
    if (dt != ACID_F32 && dt != ACID_BF16)
      return set_error(ACID_ERR_INVALID_ARG, "bad dtype %d", dt);
  if (!(n->eps >= 0.f) || !std::isfinite(n->eps) || !std::isfinite(n->res_scale))
    return set_error(ACID_ERR_INVALID_ARG, "eps must be finite and >= 0, res_scale finite");
  if (n->rows_per_mod < 0) return set_error(ACID_ERR_INVALID_ARG, "rows_per_mod < 0");
  if (rows == 0) return ACID_OK;
  if (!n->h || (!n->y && !n->out) || (n->y && !n->h_out))
    return set_error(ACID_ERR_INVALID_ARG, "NULL argument: h, y with h_out, out without y");
  const struct {
    const char* name;
    const void* p;
    int64_t ld, size;
  } mats[] = {{"h", n->h, n->h_ld, 4},
              {"y", n->y, n->y_ld, n->y_dtype == ACID_BF16 ? 2 : 4},
              {"h_out", n->y ? n->h_out : nullptr, n->h_out_ld, 4},
              {"out", n->out, n->out_ld, n->out_dtype == ACID_BF16 ? 2 : 4}};
  for (const auto& m : mats) {
    if (!m.p) continue;
    if (m.ld < hidden || m.ld % 4 || m.ld > ((int64_t)1 << 32))
      return set_error(ACID_ERR_SHAPE, "%s: row stride %lld must be >= hidden, <= 2^32, a multiple of 4",
                       m.name, (long long)m.ld);
    if ((uintptr_t)m.p % (4 * m.size))
      return set_error(ACID_ERR_INVALID_ARG, "%s must be aligned to four of its elements", m.name);
  }
  if (((uintptr_t)n->post_weight | (uintptr_t)n->gate | (uintptr_t)n->pre_weight |
       (uintptr_t)n->shift | (uintptr_t)n->scale) % 16)
    return set_error(ACID_ERR_INVALID_ARG, "weights, gate, shift and scale must be 16-byte aligned");
  for (int w = 2; w < 4; ++w)  // what is written
    for (int r = 0; r < w; ++r) {
      const auto &x = mats[w], &z = mats[r];
      if (w == 2 && r == 0 && x.p == z.p && x.ld == z.ld) continue;  // h in place
      if (rows_overlap(x.p, rows, hidden * x.size, x.ld * x.size, z.p, rows, hidden * z.size,
                       z.ld * z.size))
        return set_error(ACID_ERR_INVALID_ARG, "%s overlaps %s", x.name, z.name);
    }
  const int64_t mods = n->rows_per_mod ? (rows + n->rows_per_mod - 1) / n->rows_per_mod : 1;
  const struct {
    const void* p;
    int64_t count;
  } vecs[] = {{n->post_weight, 1}, {n->gate, mods}, {n->pre_weight, 1}, {n->shift, mods},
              {n->scale, mods}};
  for (const auto& v : vecs)
    for (int w = 2; w < 4; ++w)
      if (rows_overlap(mats[w].p, rows, hidden * mats[w].size, mats[w].ld * mats[w].size, v.p, 1,
                       v.count * hidden * 4, v.count * hidden * 4))
        return set_error(ACID_ERR_INVALID_ARG, "%s overlaps a weight or modulation vector",
                         mats[w].name);
  StreamDevice on;
  ACID_TRY(on.enter(stream));
  const NormArgs a = {n->h, n->y, n->h_out, n->out, n->h_ld, n->y_ld, n->h_out_ld, n->out_ld,
                      n->post_weight, n->gate, n->pre_weight, n->shift, n->scale, rows,
                      n->rows_per_mod, hidden, n->post, n->pre, n->res_scale, n->eps};
  const hipError_t e = !n->y ? launch_out<Absent>(n->out_dtype, a, stream)
                       : n->y_dtype == ACID_BF16 ? launch_out<bf16>(n->out_dtype, a, stream)
                                                 : launch_out<float>(n->out_dtype, a, stream);
  return e == hipSuccess ? ACID_OK : check_hip(e, "residual norm");
}
