// The seam between two blocks in one pass over the rows (acid_residual_norm):
//
//   h' = res_scale h + gate (.) (N_post(y) (.) post_weight)
//   out = (N_pre(h') (.) pre_weight) (1 + scale) + shift
//
// N is LayerNorm (biased variance), RMS norm or nothing.  HBM-bound: y and h
// are read once, h' and out written once; a row stays in registers, in fp32,
// between its two norms.  32760 rows of 1536 (y and out bf16), 604 MB: 115 us, 5.2
// TB/s, where a 1 GiB copy makes 5.0 (with a modulation row for each, 1208 MB: 232);
// 4 rows of 4096: 4.0 us.  Short rows leave lanes of their one wave idle: 100000 of
// 64, 77 MB: 33 us.
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
// Four neighbouring values as they were loaded.
template <typename T>
struct Four {};
template <>
struct Four<float> {
  float4 v;
  __device__ __forceinline__ void load(const float* p) { v = load4(p); }
  __device__ __forceinline__ float4 value() const { return v; }
};
template <>
struct Four<bf16> {
  bf16x4 v;
  __device__ __forceinline__ void load(const bf16* p) { v = *reinterpret_cast<const bf16x4*>(p); }
  __device__ __forceinline__ float4 value() const {
    return make_float4((float)v[0], (float)v[1], (float)v[2], (float)v[3]);
  }
};
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

// Sum over a wave, in every lane: neighbours, fours, eights and rows of 16
// within the vector unit (each __shfl would take a trip through LDS).
__device__ __forceinline__ float lane_sum(float v) {
#define ADD_DPP(ctrl, rows)                                                                    \
  v += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), ctrl, rows, 0xf, false))
  ADD_DPP(0x111, 0xf);  // from the lane 1 before, in its row of 16
  ADD_DPP(0x112, 0xf);  // 2
  ADD_DPP(0x114, 0xf);  // 4
  ADD_DPP(0x118, 0xf);  // 8: the last lane of each row has its row's sum
  ADD_DPP(0x142, 0xa);  // rows 1 and 3 add the row before theirs
  ADD_DPP(0x143, 0xc);  // rows 2 and 3 add the first two
#undef ADD_DPP
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), 63));
}

// Sum over the WAVES waves of a row; `part` is one LDS array per sum.
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

// v = N(v) over a row of H values in CHUNKS float4 per thread.  Statistics in
// fp32, in two passes over the registers (mean, then centred squares).
// Threads past the row's end hold copies and are left out of the sums.
template <int WAVES, int CHUNKS>
__device__ __forceinline__ void normalise(float4 (&v)[CHUNKS], int kind, int tid, int n4, float H,
                                          float eps, float (*part)[WAVES]) {
  if (kind == ACID_NORM_NONE) return;
  float mean = 0.f;
  if (kind == ACID_NORM_LAYER) {
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) s += tid + 64 * WAVES * c < n4 ? sum4(v[c]) : 0.f;
    mean = row_sum<WAVES>(s, part[0]) / H;
  }
  float q = 0.f;
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    v[c] = make_float4(v[c].x - mean, v[c].y - mean, v[c].z - mean, v[c].w - mean);
    q += tid + 64 * WAVES * c < n4 ? sum4(mul4(v[c], v[c])) : 0.f;
  }
  const float r = 1.0f / sqrtf(row_sum<WAVES>(q, part[1]) / H + eps);
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) v[c] = mul4(v[c], make_float4(r, r, r, r));
}

// A workgroup of WAVES waves takes a run of `per` rows, one after the other.
// What the rows share (gate and post_weight as one factor, pre_weight and
// 1 + scale as one, shift) is read once a run, or where the modulation row
// changes, and the next row is loaded while a row is worked on: with all of it
// read for each row (the same bytes again from L2, three dependent waits a
// row) 32760 rows of 1536 took 145 us.  Loads past a row's end are of its last
// chunk, so that none of them waits under a branch; what they give is neither
// summed nor stored.
template <int WAVES, int CHUNKS, typename Y, typename Out>
__global__ __launch_bounds__(64 * WAVES) void residual_norm_kernel(NormArgs a, int per) {
  constexpr bool HAS_Y = !std::is_same_v<Y, Absent>, HAS_OUT = !std::is_same_v<Out, Absent>;
  __shared__ float part[2][4][WAVES];
  const int tid = threadIdx.x;
  int64_t row = (int64_t)blockIdx.x * per;
  const int64_t end = row + per < a.rows ? row + per : a.rows;
  const int n4 = a.hidden >> 2;
  const float H = (float)a.hidden;
  int at[CHUNKS];
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    const int i = tid + 64 * WAVES * c;
    at[c] = 4 * (i < n4 ? i : n4 - 1);
  }

  float4 h[CHUNKS], h_next[CHUNKS], y[CHUNKS];
  Four<Y> y_next[CHUNKS];
  float4 behind[CHUNKS], before[CHUNKS], shift[CHUNKS];
  auto load_row = [&](int64_t r) {
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) h_next[c] = load4(a.h + r * a.h_ld + at[c]);
    if constexpr (HAS_Y) {
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c) y_next[c].load((const Y*)a.y + r * a.y_ld + at[c]);
    }
  };
  auto load_mod = [&](int64_t mod) {
    float4 post[CHUNKS], pre[CHUNKS];
    auto load = [&](const float* p, int64_t r, float other, float4(&to)[CHUNKS]) {
      if (p) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) to[c] = load4(p + r * a.hidden + at[c]);
      } else {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) to[c] = make_float4(other, other, other, other);
      }
    };
    if constexpr (HAS_Y) {
      load(a.gate, mod, 1.f, behind);
      load(a.post_weight, 0, 1.f, post);
    }
    if constexpr (HAS_OUT) {
      load(a.scale, mod, 0.f, before);
      load(a.pre_weight, 0, 1.f, pre);
      load(a.shift, mod, 0.f, shift);
    }
    if constexpr (HAS_Y) {
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c) behind[c] = mul4(behind[c], post[c]);
    }
    if constexpr (HAS_OUT) {
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c)
        before[c] = mul4(pre[c], make_float4(1.f + before[c].x, 1.f + before[c].y,
                                             1.f + before[c].z, 1.f + before[c].w));
    }
  };
  load_row(row);
  int64_t mod = a.rows_per_mod ? row / a.rows_per_mod - 1 : -1, mod_end = row;
  for (int parity = 0; row < end; ++row, parity ^= 1) {
    if (row == mod_end) {  // the first row too
      load_mod(++mod);
      mod_end = a.rows_per_mod < a.rows && a.rows_per_mod ? (mod + 1) * a.rows_per_mod : a.rows;
    }
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      h[c] = h_next[c];
      if constexpr (HAS_Y) y[c] = y_next[c].value();
    }
    if (row + 1 < end) load_row(row + 1);
    if constexpr (HAS_Y) {
      normalise<WAVES, CHUNKS>(y, a.post, tid, n4, H, a.eps, part[parity]);
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c) {
        h[c] = make_float4(fmaf(a.res_scale, h[c].x, y[c].x * behind[c].x),
                           fmaf(a.res_scale, h[c].y, y[c].y * behind[c].y),
                           fmaf(a.res_scale, h[c].z, y[c].z * behind[c].z),
                           fmaf(a.res_scale, h[c].w, y[c].w * behind[c].w));
        if (tid + 64 * WAVES * c < n4) store4(a.h_out + row * a.h_out_ld + at[c], h[c]);
      }
    }
    if constexpr (HAS_OUT) {
      normalise<WAVES, CHUNKS>(h, a.pre, tid, n4, H, a.eps, part[parity] + 2);
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c)
        if (tid + 64 * WAVES * c < n4)
          store4((Out*)a.out + row * a.out_ld + at[c],
                 make_float4(fmaf(h[c].x, before[c].x, shift[c].x),
                             fmaf(h[c].y, before[c].y, shift[c].y),
                             fmaf(h[c].z, before[c].z, shift[c].z),
                             fmaf(h[c].w, before[c].w, shift[c].w)));
    }
  }
}

template <typename Y, typename Out>
hipError_t launch(const NormArgs& a, hipStream_t s) {
  const int n4 = a.hidden / 4;
  // Runs of up to four rows, of fewer where four would leave less than 1024
  // waves.  32760 rows of 1536 with 1 / 2 / 3 / 4 / 6 / 8 rows each: 122 / 113 /
  // 114 / 116 / 120 / 122 us; 8000 of 4096: 76 / 74 / 78 / 78 / 84 / 81; 4000 of 8192:
  // 99 / 84 / 85 / 79 / 82 / 80; 100000 of 64: 42 / 35 / 33 / 33 / 34 / 35; 1000 of 1024
  // (fp32): 5.5 / 6.7 / 7.9 / 8.6 / 11.0 / 13.3.
#define RN(W, C)                                                                               \
  do {                                                                                         \
    const int64_t most = a.rows / (1024 / W);                                                  \
    const int per = most < 1 ? 1 : most > 4 ? 4 : (int)most;                                   \
    hipLaunchKernelGGL((residual_norm_kernel<W, C, Y, Out>),                                   \
                       dim3((unsigned)((a.rows + per - 1) / per)), dim3(64 * W), 0, s, a, per); \
  } while (0)
  if (n4 <= 64) RN(1, 1);
  else if (n4 <= 128) RN(1, 2);
  else if (n4 <= 192) RN(1, 3);
  else if (n4 <= 256) RN(2, 2);
  else if (n4 <= 384) RN(2, 3);
  else if (n4 <= 512) RN(4, 2);
  else if (n4 <= 768) RN(4, 3);
  else if (n4 <= 1024) RN(4, 4);
  else if (n4 <= 1536) RN(8, 3);
  else RN(8, 4);
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
  if (hidden < 4 || hidden % 4 || hidden > 8192)
    return set_error(ACID_ERR_SHAPE, "hidden %d: multiple of 4 in [4, 8192]", hidden);
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
  const int64_t mods = n->rows_per_mod ? (rows - 1) / n->rows_per_mod + 1 : 1;
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
