// Causal linear attention with a decay for each head: whole sequences
// (acid_linear_attention) and one token a row (acid_linear_attention_step).
//
//   S_t = lambda S_{t-1} + k_t^T v_t,  o_t = scale q_t S_t,  lambda = exp(-slope)
//
// S is fp32 [d][d] (rows over k's columns, columns over v's).
#include "common.h"

namespace acid {
namespace {

// Where a sequence's or row's vectors lie, in elements.
struct Strides {
  int64_t seq, head, token;
};

struct RecurrentArgs {
  const void *q, *k, *v;
  void* o;
  Strides qs, ks, vs, os;
  int64_t v_col;  // distance of v's columns
  const float* slopes;
  const int32_t* lengths;  // tokens of each sequence, or null: all
  const int32_t* slots;    // step: state of each row, or null: its own index
  const float* state_in;
  float* state_out;
  int64_t tokens;  // of a sequence; step: rows
  int64_t n_slots;
  int32_t heads;
  float scale;
};

// First index in [from, to) whose slot is s, or -1; the same in every lane.
__device__ __forceinline__ int64_t find_slot(const int32_t* __restrict__ slots, int32_t s,
                                             int64_t from, int64_t to) {
  const int lane = threadIdx.x & 63;
  for (int64_t j = from; j < to; j += 64) {
    const bool hit = j + lane < to && slots[j + lane] == s;
    const uint64_t mask = __ballot(hit);
    if (mask) return j + __builtin_ctzll(mask);
  }
  return -1;
}

// The recurrence as it stands, one token after the other.  A workgroup owns
// 32 columns of one head's state: thread (rg, cg) holds rows rg + 32 i,
// columns 4 cg .. 4 cg + 3.
template <typename T, int D, bool STEP>
__global__ __launch_bounds__(256) void la_recurrent_kernel(RecurrentArgs a) {
  constexpr int R = D / 32;
  __shared__ float part[2][4][32];
  const int cg = threadIdx.x & 7, rg = threadIdx.x >> 3, wave = threadIdx.x >> 6;
  const int slice = blockIdx.x % R;
  const int head = (blockIdx.x / R) % a.heads;
  const int64_t seq = blockIdx.x / R / a.heads;

  int64_t slot = seq, t = 0, end = a.tokens;
  if constexpr (STEP) {
    t = seq;
    if (a.slots) {
      slot = a.slots[seq];
      if (slot < 0 || slot >= a.n_slots) return;  // padding
      // rows of one slot are one sequence's successive tokens: the first
      // row's workgroup takes them all
      if (find_slot(a.slots, (int32_t)slot, 0, seq) >= 0) return;
    }
  } else if (a.lengths) {
    const int64_t n = a.lengths[seq];
    end = n < 0 ? 0 : n < end ? n : end;
  }
  const T* q = (const T*)a.q + (STEP ? 0 : seq * a.qs.seq) + head * a.qs.head;
  const T* k = (const T*)a.k + (STEP ? 0 : seq * a.ks.seq) + head * a.ks.head;
  const T* v = (const T*)a.v + (STEP ? 0 : seq * a.vs.seq) + head * a.vs.head;
  T* o = (T*)a.o + (STEP ? 0 : seq * a.os.seq) + head * a.os.head;
  const int64_t at = (slot * a.heads + head) * (D * D) + slice * 32 + cg * 4;
  const float lambda = expf(-a.slopes[head]);

  float4 s[R];
#pragma unroll
  for (int i = 0; i < R; ++i)
    s[i] = a.state_in ? *reinterpret_cast<const float4*>(a.state_in + at + (rg + 32 * i) * D)
                      : make_float4(0.f, 0.f, 0.f, 0.f);
  int parity = 0;
  while (t >= 0 && t < end) {
    float4 vt;
    const T* vp = v + t * a.vs.token + (slice * 32 + cg * 4) * a.v_col;
    vt.x = (float)vp[0];
    vt.y = (float)vp[a.v_col];
    vt.z = (float)vp[2 * a.v_col];
    vt.w = (float)vp[3 * a.v_col];
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const float kt = (float)k[t * a.ks.token + rg + 32 * i];
      const float qt = (float)q[t * a.qs.token + rg + 32 * i];
      s[i].x = lambda * s[i].x + kt * vt.x;
      s[i].y = lambda * s[i].y + kt * vt.y;
      s[i].z = lambda * s[i].z + kt * vt.z;
      s[i].w = lambda * s[i].w + kt * vt.w;
      y.x += qt * s[i].x;
      y.y += qt * s[i].y;
      y.z += qt * s[i].z;
      y.w += qt * s[i].w;
    }
#pragma unroll
    for (int m = 8; m < 64; m <<= 1) {
      y.x += __shfl_xor(y.x, m, 64);
      y.y += __shfl_xor(y.y, m, 64);
      y.z += __shfl_xor(y.z, m, 64);
      y.w += __shfl_xor(y.w, m, 64);
    }
    if ((threadIdx.x & 63) < 8) *reinterpret_cast<float4*>(&part[parity][wave][cg * 4]) = y;
    __syncthreads();
    if (threadIdx.x < 32) {
      const float sum = (part[parity][0][threadIdx.x] + part[parity][1][threadIdx.x]) +
                        (part[parity][2][threadIdx.x] + part[parity][3][threadIdx.x]);
      o[t * a.os.token + slice * 32 + threadIdx.x] = (T)(a.scale * sum);
    }
    parity ^= 1;
    if constexpr (STEP)
      t = a.slots ? find_slot(a.slots, (int32_t)slot, t + 1, end) : -1;
    else
      ++t;
  }
  if (a.state_out) {
#pragma unroll
    for (int i = 0; i < R; ++i)
      *reinterpret_cast<float4*>(a.state_out + at + (rg + 32 * i) * D) = s[i];
  }
}

template <bool STEP>
hipError_t launch_recurrent(int dtype, int d, int64_t seqs, const RecurrentArgs& a,
                            hipStream_t s) {
  const dim3 grid((unsigned)(seqs * a.heads * (d / 32)));
#define LA(T, D) hipLaunchKernelGGL((la_recurrent_kernel<T, D, STEP>), grid, dim3(256), 0, s, a)
  if (dtype == ACID_BF16) {
    if (d == 64) LA(bf16, 64);
    else LA(bf16, 128);
  } else {
    if (d == 64) LA(float, 64);
    else LA(float, 128);
  }
#undef LA
  return hipGetLastError();
}

acid_status check_heads(int dtype, int64_t n, int heads, int d) {
  if (dtype != ACID_F32 && dtype != ACID_BF16)
    return set_error(ACID_ERR_INVALID_ARG, "bad dtype %d", dtype);
  if (n < 0 || heads < 1)
    return set_error(ACID_ERR_INVALID_ARG, "negative count of sequences, or n_heads < 1");
  if (d != 64 && d != 128)
    return set_error(ACID_ERR_SHAPE, "head_dim %d: supported 64 or 128", d);
  if (n > ((int64_t)1 << 24) || heads > (1 << 20) || n * heads >= ((int64_t)1 << 22))
    return set_error(ACID_ERR_SHAPE, "%lld sequences x n_heads %d exceeds the grid limit",
                     (long long)n, heads);
  return ACID_OK;
}

}  // namespace
}  // namespace acid

using namespace acid;

extern "C" {

size_t acid_linear_attention_workspace_bytes(int64_t n_seq, int32_t n_heads, int64_t seq_len,
                                             int32_t head_dim) {
  if (check_heads(ACID_BF16, n_seq, n_heads, head_dim) != ACID_OK || seq_len < 0) return 0;
  return 0;
}

acid_status acid_linear_attention(int32_t dtype, int64_t n_seq, int32_t n_heads, int64_t seq_len,
                                  int32_t head_dim, const void* q_dev, const void* k_dev,
                                  const void* vt_dev, int64_t vt_ld, const float* slopes_dev,
                                  const int32_t* lengths_dev, const float* state_in_dev,
                                  float* state_out_dev, float scale, void* o_dev,
                                  void* workspace_dev, size_t workspace_bytes,
                                  hipStream_t stream) {
  ACID_TRY(check_heads(dtype, n_seq, n_heads, head_dim));
  if (seq_len < 0) return set_error(ACID_ERR_INVALID_ARG, "seq_len < 0");
  if (seq_len > ((int64_t)1 << 31) - 64)
    return set_error(ACID_ERR_SHAPE, "seq_len %lld: below 2^31 - 63", (long long)seq_len);
  if (vt_ld < round_up(seq_len, 8) || vt_ld % 8 || vt_ld > ((int64_t)1 << 31))
    return set_error(ACID_ERR_SHAPE,
                     "vt_ld %lld must be a multiple of 8, >= round_up(L, 8) and <= 2^31",
                     (long long)vt_ld);
  if (n_seq == 0) return ACID_OK;
  if (!slopes_dev || (seq_len > 0 && (!q_dev || !k_dev || !vt_dev || !o_dev)))
    return set_error(ACID_ERR_INVALID_ARG, "NULL argument");
  if (((uintptr_t)q_dev | (uintptr_t)k_dev | (uintptr_t)vt_dev | (uintptr_t)o_dev |
       (uintptr_t)state_in_dev | (uintptr_t)state_out_dev | (uintptr_t)workspace_dev) % 16)
    return set_error(ACID_ERR_INVALID_ARG, "buffers must be 16-byte aligned");
  const int64_t size = dtype == ACID_BF16 ? 2 : 4, heads = n_seq * n_heads;
  const int64_t qkv = heads * seq_len * head_dim * size, vtb = heads * head_dim * vt_ld * size;
  const int64_t states = heads * head_dim * head_dim * 4;
  if (bytes_overlap(o_dev, qkv, q_dev, qkv) || bytes_overlap(o_dev, qkv, k_dev, qkv) ||
      bytes_overlap(o_dev, qkv, vt_dev, vtb) ||
      bytes_overlap(o_dev, qkv, state_in_dev, state_in_dev ? states : 0) ||
      bytes_overlap(o_dev, qkv, state_out_dev, state_out_dev ? states : 0))
    return set_error(ACID_ERR_INVALID_ARG, "o overlaps an input or a state");
  if (state_out_dev &&
      (bytes_overlap(state_out_dev, states, q_dev, qkv) ||
       bytes_overlap(state_out_dev, states, k_dev, qkv) ||
       bytes_overlap(state_out_dev, states, vt_dev, vtb)))
    return set_error(ACID_ERR_INVALID_ARG, "state_out overlaps an input");
  if (state_in_dev != state_out_dev &&
      bytes_overlap(state_in_dev, states, state_out_dev, states))
    return set_error(ACID_ERR_INVALID_ARG, "state_in and state_out: one buffer or apart");
  (void)workspace_bytes;
  StreamDevice on;
  ACID_TRY(on.enter(stream));
  RecurrentArgs a = {};
  a.q = q_dev;
  a.k = k_dev;
  a.v = vt_dev;
  a.o = o_dev;
  const int64_t d = head_dim;
  a.qs = a.ks = {n_heads * seq_len * d, seq_len * d, d};
  a.vs = {n_heads * d * vt_ld, d * vt_ld, 1};
  a.v_col = vt_ld;
  a.os = {seq_len * n_heads * d, d, n_heads * d};
  a.slopes = slopes_dev;
  a.lengths = lengths_dev;
  a.state_in = state_in_dev;
  a.state_out = state_out_dev;
  a.tokens = seq_len;
  a.heads = n_heads;
  a.scale = scale;
  const hipError_t e = launch_recurrent<false>(dtype, head_dim, n_seq, a, stream);
  return e == hipSuccess ? ACID_OK : check_hip(e, "linear attention");
}

acid_status acid_linear_attention_step(int32_t dtype, int64_t n_rows, int32_t n_heads,
                                       int32_t head_dim, const void* q_dev, int64_t q_ld,
                                       const void* k_dev, int64_t k_ld, const void* v_dev,
                                       int64_t v_ld, const float* slopes_dev,
                                       const int32_t* slots_dev, int64_t n_slots,
                                       const float* state_in_dev, float* state_out_dev,
                                       float scale, void* o_dev, int64_t o_ld,
                                       hipStream_t stream) {
  ACID_TRY(check_heads(dtype, n_rows, n_heads, head_dim));
  const int64_t width = (int64_t)n_heads * head_dim, size = dtype == ACID_BF16 ? 2 : 4;
  if (n_slots < 0 || n_slots > INT32_MAX || n_slots * n_heads >= ((int64_t)1 << 40) ||
      (!slots_dev && n_slots < n_rows))
    return set_error(ACID_ERR_SHAPE, "n_slots %lld: in [0, 2^31), times n_heads < 2^40, without slots >= n_rows",
                     (long long)n_slots);
  for (int64_t ld : {q_ld, k_ld, v_ld, o_ld})
    if (ld < width || ld * size % 16 || ld > ((int64_t)1 << 32))
      return set_error(ACID_ERR_SHAPE,
                       "row strides must be >= n_heads * head_dim, <= 2^32 and whole 16 bytes");
  if (n_rows == 0) return ACID_OK;
  if (!q_dev || !k_dev || !v_dev || !slopes_dev || !state_in_dev || !state_out_dev || !o_dev)
    return set_error(ACID_ERR_INVALID_ARG, "NULL argument");
  if (((uintptr_t)q_dev | (uintptr_t)k_dev | (uintptr_t)v_dev | (uintptr_t)o_dev |
       (uintptr_t)state_in_dev | (uintptr_t)state_out_dev) % 16)
    return set_error(ACID_ERR_INVALID_ARG, "buffers must be 16-byte aligned");
  const int64_t states = n_slots * width * head_dim * 4, w = width * size;
  const struct {
    const void* p;
    int64_t ld;
  } in[] = {{q_dev, q_ld}, {k_dev, k_ld}, {v_dev, v_ld}};
  for (const auto& i : in) {
    if (rows_overlap(o_dev, n_rows, w, o_ld * size, i.p, n_rows, w, i.ld * size))
      return set_error(ACID_ERR_INVALID_ARG, "o overlaps q, k or v");
    if (rows_overlap(state_out_dev, 1, states, states, i.p, n_rows, w, i.ld * size))
      return set_error(ACID_ERR_INVALID_ARG, "state_out overlaps q, k or v");
  }
  if (rows_overlap(state_in_dev, 1, states, states, o_dev, n_rows, w, o_ld * size) ||
      rows_overlap(state_out_dev, 1, states, states, o_dev, n_rows, w, o_ld * size))
    return set_error(ACID_ERR_INVALID_ARG, "o overlaps a state");
  if (state_in_dev != state_out_dev &&
      bytes_overlap(state_in_dev, states, state_out_dev, states))
    return set_error(ACID_ERR_INVALID_ARG, "state_in and state_out: one buffer or apart");
  StreamDevice on;
  ACID_TRY(on.enter(stream));
  RecurrentArgs a = {};
  a.q = q_dev;
  a.k = k_dev;
  a.v = v_dev;
  a.o = o_dev;
  a.qs = {0, head_dim, q_ld};
  a.ks = {0, head_dim, k_ld};
  a.vs = {0, head_dim, v_ld};
  a.os = {0, head_dim, o_ld};
  a.v_col = 1;
  a.slopes = slopes_dev;
  a.slots = slots_dev;
  a.n_slots = n_slots;
  a.state_in = state_in_dev;
  a.state_out = state_out_dev;
  a.tokens = n_rows;
  a.heads = n_heads;
  a.scale = scale;
  const hipError_t e = launch_recurrent<true>(dtype, head_dim, n_rows, a, stream);
  return e == hipSuccess ? ACID_OK : check_hip(e, "linear attention step");
}

}  // extern "C"
