// A projection's rows Q | K | V into attention's heads (acid_rotary_qkv): norm,
// rotation by the angles of positions with several axes, head-major Q and K, V
// transposed.
//
// Pair i of a head belongs to one axis; its angle is positions[axis][token]
// freqs[i], taken in 64 bits and in turns, so that far positions keep their
// fraction; sine and cosine of that are taken in 32 bits.  Bound by HBM: each row is
// read and written once.  32760 tokens of 12 + 12 + 12 heads of 128, bf16, norm over the row, 604
// MB: 127 us, 4.75 TB/s, where a copy makes 5.2; one token of 16 + 4 + 4 heads of 64: 4.3 us.
#include <cmath>
#include <type_traits>

#include "common.h"

namespace acid {
namespace {

struct HeadArgs {
  const void *q, *k, *v;
  void *q_out, *k_out, *vt;
  int64_t q_ld, k_ld, v_ld;
  int64_t q_head, q_row, q_seq, k_head, k_row, k_seq, vt_head, vt_row, vt_seq;
  const void* positions;
  int64_t positions_ld;
  const double* freqs;
  const float *q_weight, *k_weight, *q_bias, *k_bias;
  int64_t tokens, tiles, v_tiles, qk_groups;  // of a sequence; workgroups of Q and K
  int32_t heads, kv_heads, pairs, ends[3];  // ends of the first three axes' pairs
  int32_t norm, halves, float_positions, vt_wide;
  float q_scale, eps;
};

__device__ __forceinline__ void load8(const bf16* p, float* v) {
  const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load8(const float* p, float* v) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = a[i];
    v[4 + i] = b[i];
  }
}
// Streaming stores: Q and K are not read again before they have left L2 (131 -> 127 us; V^T's, of
// 128 bytes a row, take 16 us more so).
__device__ __forceinline__ void store8(bf16* p, const float* v) {
  bf16x8 w;
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = (bf16)v[i];
  __builtin_nontemporal_store(__builtin_bit_cast(u32x4, w), reinterpret_cast<u32x4*>(p));
}
__device__ __forceinline__ void store8(float* p, const float* v) {
  __builtin_nontemporal_store(f32x4{v[0], v[1], v[2], v[3]}, reinterpret_cast<f32x4*>(p));
  __builtin_nontemporal_store(f32x4{v[4], v[5], v[6], v[7]}, reinterpret_cast<f32x4*>(p + 4));
}

// Sixteen values of a head as they were loaded: two runs of eight.
template <typename T>
struct Held;
template <>
struct Held<bf16> {
  u32x4 v[2];
  __device__ __forceinline__ void load(const bf16* p, int d0, int d1) {
    v[0] = *reinterpret_cast<const u32x4*>(p + d0);
    v[1] = *reinterpret_cast<const u32x4*>(p + d1);
  }
  __device__ __forceinline__ void values(float* x) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[2 * i] = __uint_as_float(v[i / 4][i % 4] << 16);
      x[2 * i + 1] = __uint_as_float(v[i / 4][i % 4] & 0xffff0000u);
    }
  }
};
template <>
struct Held<float> {
  f32x4 v[4];
  __device__ __forceinline__ void load(const float* p, int d0, int d1) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      v[i] = *reinterpret_cast<const f32x4*>(p + d0 + 4 * i);
      v[2 + i] = *reinterpret_cast<const f32x4*>(p + d1 + 4 * i);
    }
  }
  __device__ __forceinline__ void values(float* x) const {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = v[i / 4][i % 4];
  }
};

// Sum over the lanes that hold one head of a token.
template <int LANES>
__device__ __forceinline__ float head_sum(float v) {
#define ADD_DPP(ctrl) \
  v += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), ctrl, 0xf, 0xf, false))
  ADD_DPP(0xB1);                             // the lane beside it
  ADD_DPP(0x4E);                             // the other two of its four
  if constexpr (LANES == 8) ADD_DPP(0x141);  // the other four of its eight
#undef ADD_DPP
  return v;
}

// Q and K of 64 / (D / 16) tokens: a lane holds sixteen values of a head, eight pairs, and
// the eight waves take the heads in turn.  Up to HELD heads a wave are loaded at once and
// stay in registers between their norm's sum and their rotation; past 32 heads of Q and K
// together the rest is read again.  The angles' sines and cosines are made once a token and
// shared by way of LDS, while the heads are on their way.  (At the size above: heads held, loads
// before the angles and 16-byte stores of V^T 140 us of 212, the lanes' order in a head and
// the layout in LDS 131, streaming stores 127.)
constexpr int kWaves = 8, HELD = 4;
template <typename In, typename Out, int D>
__device__ __forceinline__ void rotate_heads(const HeadArgs& a, int64_t group, float* lds) {
  constexpr int LANES = D / 16, TOKENS = 64 / LANES;
  float2* turns = reinterpret_cast<float2*>(lds);  // [8][64]: pair i of each lane's eight
  float* part = lds + TOKENS * D;                  // [2][kWaves][TOKENS]
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t seq = group / a.tiles, t0 = (group - seq * a.tiles) * TOKENS;
  const int o = lane % LANES, tt = lane / LANES;
  const int64_t t = t0 + tt < a.tokens ? t0 + tt : a.tokens - 1, row = seq * a.tokens + t;
  const bool live = t0 + tt < a.tokens;
  // this lane's two runs of eight dims, and its pairs, in two runs of four: neighbouring lanes
  // have neighbouring runs (of whole lines), but in halves past the pairs
  int d0 = 8 * o, d1 = D / 2 + d0, p0 = 4 * o, p1 = D / 4 + p0;
  if (a.halves) {
    p0 = 8 * o;
    p1 = p0 + 4;
    d0 = 8 * o < a.pairs ? 8 * o : 16 * o;  // 2 pairs + 16 (o - pairs / 8)
    d1 = d0 + (8 * o < a.pairs ? a.pairs : 8);
  }
  const int nq = a.q ? a.heads : 0, nk = a.k ? a.kv_heads : 0, n = nq + nk;
  auto source = [&](int u) {
    return u < nq ? (const In*)a.q + row * a.q_ld + u * D : (const In*)a.k + row * a.k_ld + (u - nq) * D;
  };
  Held<In> held[HELD];
#pragma unroll
  for (int i = 0; i < HELD; ++i)
    if (wave + kWaves * i < n) held[i].load(source(wave + kWaves * i), d0, d1);

  for (int i = tid; i < TOKENS * (D / 2); i += 64 * kWaves) {
    const int p = i % (D / 2);
    const int64_t ti = t0 + i / (D / 2);
    float2 cs = make_float2(1.f, 0.f);
    if (p < a.pairs && ti < a.tokens) {
      const int axis = (p >= a.ends[0]) + (p >= a.ends[1]) + (p >= a.ends[2]);
      const int64_t at = axis * a.positions_ld + seq * a.tokens + ti;
      const double pos = a.float_positions ? (double)((const float*)a.positions)[at]
                                           : (double)((const int32_t*)a.positions)[at];
      double turn = pos * (a.freqs[p] * 0.15915494309189535);  // 1 / (2 pi)
      turn -= rint(turn);
      sincospif(2.0f * (float)turn, &cs.y, &cs.x);
    }
    const int run = p / 4, lane_of = a.halves ? run / 2 : run % LANES, second = a.halves ? run % 2 : run / LANES;
    turns[(4 * second + p % 4) * 64 + i / (D / 2) * LANES + lane_of] = cs;
  }
  if (a.norm == ACID_HEAD_NORM_RMS_ROW) {
    float sums[2] = {0.f, 0.f};
    auto add = [&](const Held<In>& h, int u) {
      float v[16], s = 0.f;
      h.values(v);
#pragma unroll
      for (int i = 0; i < 16; ++i) s = fmaf(v[i], v[i], s);
      sums[0] += u < nq ? s : 0.f;
      sums[1] += u < nq ? 0.f : s;
    };
#pragma unroll
    for (int i = 0; i < HELD; ++i)
      if (wave + kWaves * i < n) add(held[i], wave + kWaves * i);
    for (int u = wave + kWaves * HELD; u < n; u += kWaves) {
      Held<In> h;
      h.load(source(u), d0, d1);
      add(h, u);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float s = head_sum<LANES>(sums[i]);
      if (o == 0) part[(i * kWaves + wave) * TOKENS + tt] = s;
    }
  }
  __syncthreads();
  float row_r[2] = {1.f, 1.f};
  if (a.norm == ACID_HEAD_NORM_RMS_ROW) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) s += part[(i * kWaves + w) * TOKENS + tt];
      row_r[i] = 1.0f / sqrtf(s / (float)((i ? a.kv_heads : a.heads) * D) + a.eps);
    }
  }
  float2 cs[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) cs[i] = turns[i * 64 + lane];

  auto finish = [&](const Held<In>& h, int u) {
    const bool is_q = u < nq;
    const int head = is_q ? u : u - nq;
    float v[16];
    h.values(v);
    if (a.norm != ACID_HEAD_NORM_NONE) {
      float r = is_q ? row_r[0] : row_r[1];
      const float* weight = is_q ? a.q_weight : a.k_weight;
      const float* bias = is_q ? a.q_bias : a.k_bias;
      if (a.norm == ACID_HEAD_NORM_RMS_ROW) {
        if (weight) weight += head * D;
      } else {
        if (a.norm == ACID_HEAD_NORM_LAYER) {
          float s = 0.f;
#pragma unroll
          for (int i = 0; i < 16; ++i) s += v[i];
          const float mean = head_sum<LANES>(s) / D;
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] -= mean;
        }
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) s = fmaf(v[i], v[i], s);
        r = 1.0f / sqrtf(head_sum<LANES>(s) / D + a.eps);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] *= r;
      auto each = [&](const float* p, auto f) {  // f(value, the column's)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const f32x4 w = *reinterpret_cast<const f32x4*>(p + (j < 2 ? d0 : d1 - 8) + 4 * j);
#pragma unroll
          for (int i = 0; i < 4; ++i) v[4 * j + i] = f(v[4 * j + i], w[i]);
        }
      };
      if (weight) each(weight, [](float x, float w) { return x * w; });
      if (bias) each(bias, [](float x, float b) { return x + b; });
    }
    const float scale = is_q ? a.q_scale : 1.f;
    auto turn = [&](float& x, float& y, int i) {
      const bool turned = (i < 4 ? p0 + i : p1 + i - 4) < a.pairs;
      const float nx = x * cs[i].x - y * cs[i].y, ny = x * cs[i].y + y * cs[i].x;
      x = scale * (turned ? nx : x);
      y = scale * (turned ? ny : y);
    };
    if (a.halves) {
#pragma unroll
      for (int i = 0; i < 8; ++i) turn(v[i], v[8 + i], i);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) turn(v[2 * i], v[2 * i + 1], i);
    }
    if (live) {
      Out* dst = is_q ? (Out*)a.q_out + seq * a.q_seq + head * a.q_head + t * a.q_row
                      : (Out*)a.k_out + seq * a.k_seq + head * a.k_head + t * a.k_row;
      store8(dst + d0, v);
      store8(dst + d1, v + 8);
    }
  };
#pragma unroll
  for (int i = 0; i < HELD; ++i)
    if (wave + kWaves * i < n) finish(held[i], wave + kWaves * i);
  for (int u = wave + kWaves * HELD; u < n; u += kWaves) {
    Held<In> h;
    h.load(source(u), d0, d1);
    finish(h, u);
  }
}

// V^T of 64 tokens and 64 dims of a head, by way of LDS: eight dims of a token a thread
// in, eight tokens of a dim out.  The eight tokens j of dim d lie at place j ^ (d / 8) % 8 of
// the dim's row, so that a wave's writes of one token's dims meet different banks.
template <typename In, typename Out, int D>
__device__ __forceinline__ void transpose_v(const HeadArgs& a, int64_t group, float* lds) {
  Out* tile = reinterpret_cast<Out*>(lds);
  const int tid = threadIdx.x, units = a.kv_heads * (D / 64);
  const int64_t per_seq = a.v_tiles * units, seq = group / per_seq, rest = group - seq * per_seq;
  const int part = (int)(rest % units);
  const int64_t t0 = rest / units * 64;
  const int head = part / (D / 64), dim0 = part % (D / 64) * 64;
  const int left = (int)(a.tokens - t0 < 64 ? a.tokens - t0 : 64);
  {
    const int r = tid / 8, c = tid % 8;
    float v[8];
    load8((const In*)a.v + (seq * a.tokens + t0 + (r < left ? r : left - 1)) * a.v_ld + head * D + dim0 + c * 8, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) tile[(c * 8 + e) * 64 + (r / 8 ^ c) * 8 + r % 8] = (Out)v[e];
  }
  __syncthreads();
  const int dim = tid / 8, c = tid % 8 * 8;
  const Out* from = tile + dim * 64 + (tid % 8 ^ dim / 8) * 8;
  Out* to = (Out*)a.vt + seq * a.vt_seq + head * a.vt_head + (dim0 + dim) * a.vt_row + t0 + c;
  if (a.vt_wide && c + 8 <= left) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(Out) / 2; ++i)
      reinterpret_cast<u32x4*>(to)[i] = reinterpret_cast<const u32x4*>(from)[i];
  } else {
    for (int e = 0; e < 8 && c + e < left; ++e) to[e] = from[e];
  }
}

template <typename In, typename Out, int D>
__global__ __launch_bounds__(64 * kWaves) void rotary_qkv_kernel(HeadArgs a) {
  constexpr int TURNS = 1024 / D * D + 2 * kWaves * (1024 / D), TILE = 64 * 64 * sizeof(Out) / 4;
  __shared__ __attribute__((aligned(16))) float lds[TURNS > TILE ? TURNS : TILE];
  if ((int64_t)blockIdx.x < a.qk_groups)
    rotate_heads<In, Out, D>(a, blockIdx.x, lds);
  else
    transpose_v<In, Out, D>(a, blockIdx.x - a.qk_groups, lds);
}

template <typename In, typename Out>
hipError_t launch(int d, const HeadArgs& a, unsigned grid, hipStream_t s) {
  if (d == 64)
    hipLaunchKernelGGL((rotary_qkv_kernel<In, Out, 64>), dim3(grid), dim3(64 * kWaves), 0, s, a);
  else
    hipLaunchKernelGGL((rotary_qkv_kernel<In, Out, 128>), dim3(grid), dim3(64 * kWaves), 0, s, a);
  return hipGetLastError();
}

// An output as rows of bytes, one for each token, head or sequence.
struct Rows {
  const void* p;
  int64_t rows, width, ld;
};

Rows input_rows(const void* p, int64_t rows, int64_t width, int64_t ld, int64_t size) {
  return {p, rows, width * size, ld * size};
}
Rows output_rows(const void* p, int64_t n_seq, int64_t heads, int64_t rows, int64_t width, int64_t head,
                 int64_t row, int64_t seq, int64_t size) {
  const int64_t token = (heads - 1) * head + width, whole = (rows - 1) * row + width;
  if (row >= token && (n_seq == 1 || seq == rows * row)) return {p, n_seq * rows, token * size, row * size};
  if (head >= whole && (n_seq == 1 || seq == heads * head)) return {p, n_seq * heads, whole * size, head * size};
  return {p, n_seq, ((heads - 1) * head + whole) * size, seq * size};
}
// Whether no two values of an output share an address: one axis within the
// other, and a sequence beyond both.
bool own_addresses(int64_t n_seq, int64_t heads, int64_t rows, int64_t width, int64_t head, int64_t row,
                   int64_t seq) {
  const bool head_major = row >= width && (heads == 1 || head >= (rows - 1) * row + width);
  const bool token_major = head >= width && (rows == 1 || row >= (heads - 1) * head + width);
  return (head_major || token_major) &&
         (n_seq == 1 || seq >= (heads - 1) * head + (rows - 1) * row + width);
}

}  // namespace
}  // namespace acid

using namespace acid;

extern "C" {

acid_status acid_rotary_qkv(const acid_rotary_qkv_args* args, int64_t n_seq, int64_t tokens,
                            hipStream_t stream) {
  if (!args) return set_error(ACID_ERR_INVALID_ARG, "NULL argument");
  const acid_rotary_qkv_args& p = *args;
  for (int dt : {p.in_dtype, p.out_dtype})
    if (dt != ACID_F32 && dt != ACID_BF16) return set_error(ACID_ERR_INVALID_ARG, "bad dtype %d", dt);
  if (p.norm < ACID_HEAD_NORM_NONE || p.norm > ACID_HEAD_NORM_RMS_ROW || (p.pairing != 0 && p.pairing != 1) ||
      (p.positions_f32 != 0 && p.positions_f32 != 1))
    return set_error(ACID_ERR_INVALID_ARG, "rotary: bad norm, pairing or positions_f32");
  if (!(p.eps >= 0.f) || !std::isfinite(p.eps) || !std::isfinite(p.q_scale))
    return set_error(ACID_ERR_INVALID_ARG, "rotary: eps must be >= 0, eps and q_scale finite");
  if (n_seq < 0 || tokens < 0) return set_error(ACID_ERR_INVALID_ARG, "n_seq < 0 or tokens < 0");
  if (!p.q != !p.q_out || !p.k != !p.k_out || !p.v != !p.vt)
    return set_error(ACID_ERR_INVALID_ARG, "rotary: each of q, k and v goes with its output");
  const int d = p.head_dim;
  if (d != 64 && d != 128) return set_error(ACID_ERR_SHAPE, "rotary: head_dim %d: 64 or 128", d);
  if (((p.q != nullptr) && (p.heads < 1 || p.heads > 1024)) ||
      ((p.k || p.v) && (p.kv_heads < 1 || p.kv_heads > 1024)))
    return set_error(ACID_ERR_SHAPE, "rotary: 1 to 1024 heads");
  if (p.axes < 1 || p.axes > 4) return set_error(ACID_ERR_SHAPE, "rotary: 1 to 4 axes");
  int pairs = 0;
  int32_t ends[4];
  for (int i = 0; i < 4; ++i) {
    const int n = i < p.axes ? p.sections[i] : 0;
    if (n < 0 || n > d / 2) return set_error(ACID_ERR_SHAPE, "rotary: sections are 0 to head_dim / 2 pairs");
    ends[i] = i + 1 < p.axes ? pairs + n : d;  // (the last axis has the rest)
    pairs += n;
  }
  if (pairs > d / 2 || (p.pairing == 1 && pairs % 8))
    return set_error(ACID_ERR_SHAPE, "rotary: %d pairs: at most head_dim / 2, in halves a multiple of 8", pairs);
  if (tokens > (1 << 30) || n_seq > (1 << 20) || n_seq * tokens > (1 << 30))
    return set_error(ACID_ERR_SHAPE, "rotary: at most 2^30 tokens, 2^20 sequences");
  const int64_t rows = n_seq * tokens, is = p.in_dtype == ACID_BF16 ? 2 : 4, os = p.out_dtype == ACID_BF16 ? 2 : 4;
  constexpr int64_t most = (int64_t)1 << 32;
  const struct {
    const void* in;
    int64_t ld, width;
  } ins[] = {{p.q, p.q_ld, (int64_t)p.heads * d}, {p.k, p.k_ld, (int64_t)p.kv_heads * d},
             {p.v, p.v_ld, (int64_t)p.kv_heads * d}};
  for (const auto& i : ins)
    if (i.in && (i.ld < i.width || i.ld * is % 16 || i.ld > most))
      return set_error(ACID_ERR_SHAPE, "rotary: rows at least heads * head_dim apart, whole 16 bytes, at most 2^32");
  struct {
    const void* out;
    int64_t heads, rows, width, head, row, seq;
  } outs[] = {{p.q_out, p.heads, tokens, d, p.q_head, p.q_row, p.q_seq},
              {p.k_out, p.kv_heads, tokens, d, p.k_head, p.k_row, p.k_seq},
              {p.vt, p.kv_heads, d, tokens, p.vt_head, p.vt_row, p.vt_seq}};
  if (rows == 0) return ACID_OK;
  for (int i = 0; i < 3; ++i) {
    auto& o = outs[i];
    if (!o.out) continue;
    constexpr int64_t far = (int64_t)1 << 40;
    auto out_of_range = [](int64_t n, int64_t stride) { return n > 1 && (stride < 0 || stride > far); };
    bool bad = out_of_range(o.heads, o.head) || out_of_range(o.rows, o.row) || out_of_range(n_seq, o.seq);
    // An axis of one entry may have any stride (a single token's heads are also its row's, one head's
    // tokens the matrix's): it counts as the least that keeps the entries apart.
    if (o.heads == 1) o.head = o.rows == 1 ? o.width : (o.rows - 1) * o.row + o.width;
    if (o.rows == 1) o.row = (o.heads - 1) * o.head + o.width;
    if (bad ||
        (i < 2 && (o.head * os % 16 || o.row * os % 16 || (n_seq > 1 && o.seq * os % 16))) ||
        !own_addresses(n_seq, o.heads, o.rows, o.width, o.head, o.row, o.seq))
      return set_error(ACID_ERR_SHAPE, "rotary: outputs' strides: values apart; of q_out and k_out whole 16 bytes");
  }
  if (!p.q && !p.k && !p.v) return ACID_OK;
  if ((p.q || p.k) && pairs && (!p.positions || !p.freqs)) return set_error(ACID_ERR_INVALID_ARG, "NULL argument");
  if ((p.q || p.k) && pairs && p.positions_ld < rows)
    return set_error(ACID_ERR_SHAPE, "rotary: positions' axes are n_seq * tokens or more apart");
  if (p.norm == ACID_HEAD_NORM_NONE && (p.q_weight || p.k_weight))
    return set_error(ACID_ERR_INVALID_ARG, "rotary: weights without a norm");
  if (p.norm != ACID_HEAD_NORM_LAYER && (p.q_bias || p.k_bias))
    return set_error(ACID_ERR_INVALID_ARG, "rotary: biases belong to the layer norm");
  if (((uintptr_t)p.q | (uintptr_t)p.k | (uintptr_t)p.v | (uintptr_t)p.q_out | (uintptr_t)p.k_out) % 16 ||
      (uintptr_t)p.vt % os || (uintptr_t)p.freqs % 8 || (uintptr_t)p.positions % 4 ||
      ((uintptr_t)p.q_weight | (uintptr_t)p.k_weight | (uintptr_t)p.q_bias | (uintptr_t)p.k_bias) % 16)
    return set_error(ACID_ERR_INVALID_ARG, "rotary: q, k, v, q_out, k_out, weights and biases must be 16-byte aligned, the rest to an element");
  const int64_t each = p.norm == ACID_HEAD_NORM_RMS_ROW;
  auto vec = [&](const void* v, int64_t n) { return Rows{v, 1, n * 4, n * 4}; };
  const Rows inputs[] = {input_rows(p.q, rows, (int64_t)p.heads * d, p.q_ld, is),
                         input_rows(p.k, rows, (int64_t)p.kv_heads * d, p.k_ld, is),
                         input_rows(p.v, rows, (int64_t)p.kv_heads * d, p.v_ld, is),
                         {p.positions, p.axes, rows * 4, p.positions_ld * 4},
                         {p.freqs, 1, pairs * 8, pairs * 8},
                         vec(p.q_weight, each ? (int64_t)p.heads * d : d),
                         vec(p.k_weight, each ? (int64_t)p.kv_heads * d : d),
                         vec(p.q_bias, d), vec(p.k_bias, d)};
  Rows written[3];
  for (int i = 0; i < 3; ++i) {
    const auto& o = outs[i];
    written[i] = o.out ? output_rows(o.out, n_seq, o.heads, o.rows, o.width, o.head, o.row, o.seq, os) : Rows{nullptr, 0, 0, 0};
  }
  auto overlap = [](const Rows& x, const Rows& y) {
    return rows_overlap(x.p, x.rows, x.width, x.ld, y.p, y.rows, y.width, y.ld);
  };
  for (int i = 0; i < 3; ++i) {
    const auto& o = outs[i];
    if (!o.out) continue;
    for (int j = 0; j < 9; ++j) {
      // Q and K may be turned in place: the same rows, of the same type
      const bool same = i < 2 && j == i && o.out == ins[i].in && is == os && (o.heads == 1 || o.head == d) &&
                        (tokens == 1 || o.row == ins[i].ld) && (n_seq == 1 || o.seq == tokens * ins[i].ld);
      if (!same && overlap(written[i], inputs[j]))
        return set_error(ACID_ERR_INVALID_ARG, "rotary: an output overlaps an input");
    }
    for (int j = 0; j < i; ++j)
      if (overlap(written[i], written[j])) return set_error(ACID_ERR_INVALID_ARG, "rotary: outputs overlap");
  }
  const int64_t tile = 1024 / d, tiles = (tokens + tile - 1) / tile, v_tiles = (tokens + 63) / 64;
  const int64_t qk = p.q || p.k ? n_seq * tiles : 0, vg = p.v ? n_seq * v_tiles * p.kv_heads * (d / 64) : 0;
  if (qk + vg >= (1 << 23))
    return set_error(ACID_ERR_SHAPE, "rotary: sequences, tokens and heads need %lld workgroups, at most 2^23 - 1",
                     (long long)(qk + vg));
  const int32_t vt_wide = ((uintptr_t)p.vt | (uintptr_t)(p.vt_row * os) | (uintptr_t)(p.vt_head * os) |
                           (uintptr_t)(p.vt_seq * os)) % 16 == 0;
  HeadArgs a = {p.q, p.k, p.v, p.q_out, p.k_out, p.vt, p.q_ld, p.k_ld, p.v_ld,
                p.q_head, p.q_row, p.q_seq, p.k_head, p.k_row, p.k_seq, p.vt_head, p.vt_row, p.vt_seq,
                p.positions, p.positions_ld, p.freqs, p.q_weight, p.k_weight, p.q_bias, p.k_bias,
                tokens, tiles, v_tiles, qk, p.heads, p.kv_heads, pairs, {ends[0], ends[1], ends[2]},
                p.norm, p.pairing, p.positions_f32, vt_wide, p.q_scale, p.eps};
  StreamDevice on;
  ACID_TRY(on.enter(stream));
  const unsigned grid = (unsigned)(qk + vg);
  hipError_t e;
  if (p.in_dtype == ACID_BF16)
    e = p.out_dtype == ACID_BF16 ? launch<bf16, bf16>(d, a, grid, stream) : launch<bf16, float>(d, a, grid, stream);
  else
    e = p.out_dtype == ACID_BF16 ? launch<float, bf16>(d, a, grid, stream) : launch<float, float>(d, a, grid, stream);
  return e == hipSuccess ? ACID_OK : check_hip(e, "rotary qkv");
}

}  // extern "C"
