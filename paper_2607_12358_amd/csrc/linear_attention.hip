// Causal linear attention with a decay for each head: whole sequences
// (acid_linear_attention) and one token a row (acid_linear_attention_step).
//
//   S_t = lambda S_{t-1} + k_t^T v_t,  o_t = scale q_t S_t,  lambda = exp(-slope)
//
// S is fp32 [d][d] (rows over k's columns, columns over v's).  Both forms move
// little more than they must: a token costs 4 d^2 operations a head for 4 d
// values, a single token reads and writes its states.
#include <float.h>
#include <math.h>

#include <type_traits>

#include "common.h"

namespace acid {
namespace {

// A value that is the same in every lane, kept in a scalar register.
__device__ __forceinline__ float uniform(float x) {
  return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x)));
}

// exp(-slope n), the decay over n tokens, as a sum of two fp32 values: a factor
// rounded once is off to the same side each time it is applied, and that adds
// up over a state's memory (one rounded factor a token, slope 1e-4, 8192 tokens:
// 1.8e-4 of the state).
struct Decay {
  float hi, lo;
  __device__ __forceinline__ Decay(float slope, double n) : Decay(exp(-(double)slope * n)) {}
  __device__ __forceinline__ explicit Decay(double w) {
    hi = uniform((float)w);
    lo = uniform((float)(w - (double)hi));
  }
  __device__ __forceinline__ float operator()(float x) const { return fmaf(x, hi, x * lo); }
  // decayed x + y; fmaf(x, hi, fmaf(x, lo, y)), where the compiler would copy each x
  // first (68 registers a lane in the step, past eight workgroups a CU; 60)
  __device__ __forceinline__ float operator()(float x, float y) const {
    const float rest = fmaf(x, lo, y);
    asm("v_fma_f32 %0, %0, %1, %2" : "+v"(x) : "s"(hi), "v"(rest));
    return x;
  }
};

struct StepArgs {
  const void *q, *k, *v;
  void* o;
  int64_t q_ld, k_ld, v_ld, o_ld;
  const float* slopes;
  const int32_t* slots;  // state of each row, or null: its own index
  const float* state_in;
  float* state_out;
  int64_t rows, n_slots;
  int32_t heads;
  float scale;
};

// First index in [from, to) whose slot is s, or -1; the same in every lane.
// Each row looks through all the others, so long lists are read AHEAD loads at
// a time: 16384 rows of one head (d = 64) 0.31 ms, with one load at a time 0.91, with
// no slots 0.08; 65536 rows 4.1, 13.1 and 0.42.  4096 and more are past what a
// batch of tokens has (256 rows of 12 heads: 62 us with slots, 61 without).
__device__ __forceinline__ int64_t find_slot(const int32_t* __restrict__ slots, int32_t s,
                                             int64_t from, int64_t to) {
  constexpr int AHEAD = 16;
  const int lane = threadIdx.x & 63;
  int64_t j = from;
  for (; j + 64 * AHEAD <= to; j += 64 * AHEAD) {
    int32_t v[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) v[i] = slots[j + 64 * i + lane];
    bool hit = false;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) hit |= v[i] == s;
    if (__ballot(hit)) break;
  }
  for (; j < to; j += 64) {
    const bool hit = j + lane < to && slots[j + lane] == s;
    const uint64_t mask = __ballot(hit);
    if (mask) return j + __builtin_ctzll(mask);
  }
  return -1;
}

// One token a row.  Bound by the states, read and written once: 256 rows of 12
// heads (d = 128), 391 MB, take 81 us, 4.8 TB/s.  A workgroup owns 32 columns of
// one head's state, so that one row of 12 heads still makes 48 of them (3.4 us):
// thread (rg, cg) holds rows rg + 32 i, columns 4 cg .. 4 cg + 3, and the sums over
// rows go over lanes, then over waves in LDS.
template <typename T, int D>
__global__ __launch_bounds__(256) void la_step_kernel(StepArgs a) {
  constexpr int R = D / 32;
  __shared__ float part[2][4][32];
  const int cg = threadIdx.x & 7, rg = threadIdx.x >> 3, wave = threadIdx.x >> 6;
  const int slice = blockIdx.x % R;
  const int head = (blockIdx.x / R) % a.heads;
  const int64_t row = blockIdx.x / R / a.heads;

  int64_t slot = row;
  if (a.slots) {
    slot = a.slots[row];
    if (slot < 0 || slot >= a.n_slots) return;  // padding
    // rows of one slot are one sequence's successive tokens: the first row's
    // workgroup takes them all
    if (find_slot(a.slots, (int32_t)slot, 0, row) >= 0) return;
  }
  const T* q = (const T*)a.q + head * D;
  const T* k = (const T*)a.k + head * D;
  const T* v = (const T*)a.v + head * D + slice * 32 + cg * 4;
  T* o = (T*)a.o + head * D + slice * 32;
  const int64_t at = (slot * a.heads + head) * (D * D) + slice * 32 + cg * 4;

  float4 s[R];
#pragma unroll
  for (int i = 0; i < R; ++i)
    s[i] = *reinterpret_cast<const float4*>(a.state_in + at + (rg + 32 * i) * D);
  const Decay decay(a.slopes[head], 1.0);
  int parity = 0;
  for (int64_t t = row; t >= 0;
       t = a.slots ? find_slot(a.slots, (int32_t)slot, t + 1, a.rows) : -1) {
    const T* vp = v + t * a.v_ld;
    const float4 vt = make_float4((float)vp[0], (float)vp[1], (float)vp[2], (float)vp[3]);
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const float kt = (float)k[t * a.k_ld + rg + 32 * i];
      const float qt = (float)q[t * a.q_ld + rg + 32 * i];
      s[i].x = decay(s[i].x, kt * vt.x);
      s[i].y = decay(s[i].y, kt * vt.y);
      s[i].z = decay(s[i].z, kt * vt.z);
      s[i].w = decay(s[i].w, kt * vt.w);
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
      o[t * a.o_ld + threadIdx.x] = (T)(a.scale * sum);
    }
    parity ^= 1;
  }
#pragma unroll
  for (int i = 0; i < R; ++i)
    *reinterpret_cast<float4*>(a.state_out + at + (rg + 32 * i) * D) = s[i];
}

constexpr int64_t kMaxSlotted = 65536;  // rows with slots, each of which looks through them all

hipError_t launch_step(int dtype, int d, const StepArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(a.rows * a.heads * (d / 32)));
#define LA(T, D) hipLaunchKernelGGL((la_step_kernel<T, D>), grid, dim3(256), 0, s, a)
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

// ---------------------------------------------------------- whole sequences
//
// In chunks of C = 64 tokens (i, j within a chunk):
//
//   O = scale (diag(lambda^(i+1)) Q S + ((Q K^T) (.) lambda^(i-j), j <= i) V)
//   S' = lambda^C S + sum_j k_j^T (lambda^(C-1-j) v_j)
//
// A workgroup of D / 16 waves takes a run of chunks of one head, S in the
// accumulators of its waves, each of which owns 16 of v's columns: [D][16] a
// wave, tiles of 16 x 16 whose lane (g, col) holds rows 4 g + i, column col.
// Two tiles' registers are then eight columns of k, 32 kk + 4 g .. + 3 and
// 32 kk + 16 + 4 g .. + 3: the operand of Q S as it stands, with no trip through
// LDS.  V is an operand as it lies in memory (vt's rows), read by its wave
// alone, so the decay goes onto V and not onto K, which all waves share.  O is
// formed transposed (rows: v's columns, columns: tokens), so that a lane
// stores four neighbouring values.
//
// LDS holds what the waves share, Q's and K's rows and the masked scores, and
// V's rows, each wave's its own; all are loaded there directly, a chunk ahead.
// K's operand of the outer products lies across those rows; bf16 reads it with
// the transposing LDS load.
//
// 12 heads of 32760 tokens (d = 128, bf16) take 163 us in three launches: the
// segments' states 51 us (239 MB), the scan of them 11 (62 MB) and the outputs 96
// (480 MB) at best, 4.7 to 5.4 TB/s where a copy makes 5.0 (medians of traced launches
// over two sets of inputs 57, 14 and 125).  K and V are read twice,
// because a segment's outputs need the states of those before it, and V's lines
// that two chunks share come from beyond L2 again for the second now and then
// (45 MB; the last reads of Q and K marked as such halve that, for no time here and
// 3% more with d = 64).  With all reads from L2 the outputs took 94 us for 97:
// the vector units issue for half of that time (S and the scores made into
// operands, V decayed), with 16 waves a CU to hide the rest: 80 KB of LDS and 128
// registers a lane are what two workgroups have.  One wave for 32 columns, half as
// many waves, took 115 us.  A workgroup alone on its CU takes 3.7 us a chunk (d =
// 64: 2.3), mostly LDS loads, products and barriers waiting on one another.
//
// Rounding.  A bf16 operand made from fp32 values would cost the output half
// of its accuracy, so scores and S go into their products as two bf16 parts
// (relative error 2^-16).  So does the decayed V where S is only read by the
// chunks that follow; where it is summed to an fp32 state that is returned, or
// carried to another segment, V goes in as three parts, which is exact.
constexpr int kChunk = 64;
constexpr int64_t kMaxTokens = (int64_t)1 << 28;
constexpr int kMaxAlone = 5;  // segments that make their own states

template <typename T>
struct Operand;  // eight values of the contracted index
template <>
struct Operand<bf16> {
  bf16x8 v;
};
template <>
struct Operand<float> {
  f32x4 a, b;
};

__device__ __forceinline__ Operand<bf16> load8(const bf16* p) {
  return {*reinterpret_cast<const bf16x8*>(p)};
}
__device__ __forceinline__ Operand<float> load8(const float* p) {
  return {reinterpret_cast<const f32x4*>(p)[0], reinterpret_cast<const f32x4*>(p)[1]};
}
// Values at and after index n become zeros, whatever they were.
__device__ __forceinline__ void keep_first(Operand<bf16>& x, int n) {
  const bf16x8 v = x.v;
#pragma unroll
  for (int e = 0; e < 8; ++e) x.v[e] = e < n ? v[e] : (bf16)0.0f;
}
__device__ __forceinline__ void keep_first(Operand<float>& x, int n) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x.a[e] = e < n ? x.a[e] : 0.f;
    x.b[e] = e + 4 < n ? x.b[e] : 0.f;
  }
}
__device__ __forceinline__ float sum8(const Operand<bf16>& x) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    s = __builtin_amdgcn_fdot2_f32_bf16((bf16x2){x.v[2 * i], x.v[2 * i + 1]},
                                        (bf16x2){(bf16)1.0f, (bf16)1.0f}, s, false);
  return s;
}
__device__ __forceinline__ float sum8(const Operand<float>& x) {
  const f32x4 s = x.a + x.b;
  return (s[0] + s[1]) + (s[2] + s[3]);
}
__device__ __forceinline__ bool finite(const Operand<bf16>& x, int e) {
  return fabsf((float)x.v[e]) <= FLT_MAX;
}
__device__ __forceinline__ bool finite(const Operand<float>& x, int e) {
  return fabsf(e < 4 ? x.a[e & 3] : x.b[e & 3]) <= FLT_MAX;
}
__device__ __forceinline__ void clear(Operand<bf16>& x, int e) { x.v[e] = (bf16)0.0f; }
__device__ __forceinline__ void clear(Operand<float>& x, int e) { (e < 4 ? x.a : x.b)[e & 3] = 0.f; }
__device__ __forceinline__ f32x4 mma(const Operand<bf16>& a, const Operand<bf16>& b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, b.v, c, 0, 0, 0);
}
// The fp32 instruction contracts one value a lane, so element e of both
// operands makes one product: the same 32 indices in another order.
__device__ __forceinline__ f32x4 mma(const Operand<float>& a, const Operand<float>& b, f32x4 c) {
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.a[e], b.a[e], c, 0, 0, 0);
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.b[e], b.b[e], c, 0, 0, 0);
  return c;
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// log2(e) slope: the decay over n tokens is exp2(-rate n).  Capped, so that an
// infinite slope still gives 1 over no tokens.
__device__ __forceinline__ float decay_rate(float slope) {
  const float c = slope * 1.44269504088896341f;
  return uniform(c > 1e30f ? 1e30f : c);
}

__device__ __forceinline__ void barrier_all() {  // loads into LDS included
  __builtin_amdgcn_s_waitcnt(0);
  asm volatile("s_barrier" ::: "memory");
}
__device__ __forceinline__ void wait_lds() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
}
__device__ __forceinline__ void barrier_lds() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// 64 rows of W values in LDS, in 16-byte chunks: chunk c of row r is at slot
// c ^ swizzle(r).  With 64 banks of four bytes, all of these hit each bank
// equally often: half chunks of 16 neighbouring rows (split_operand); two
// neighbouring chunks of rows 8 g + 0 .. 3 (bf16 across the rows) or four of rows
// 8 g (fp32 across the rows); whole chunks of 16 rows of scores and of V
// (score_operand; of bf16 rows of K and Q they would take two turns).
//
// Rows are a power of two long and the swizzle is linear in r's bits, so
// at(r ^ r1, x ^ x1) == at(r, x) ^ at(r1, x1): a lane keeps one address and
// every place it reads is that address with a constant's bits flipped (or, for
// rows that the swizzle does not see, at a constant distance).
template <typename T, int W, bool SCORES = false>
struct Rows {
  static constexpr int BYTES = W * (int)sizeof(T), CHUNK = 16 / (int)sizeof(T);
  static constexpr int TOTAL = kChunk * BYTES;
  static constexpr uint32_t swizzle(uint32_t r) {
    const uint32_t b0 = r & 1, b1 = r >> 1 & 1, b2 = r >> 2 & 1, b3 = r >> 3 & 1, b4 = r >> 4 & 1;
    return sizeof(T) == 4 ? b0 | b1 << 1 | b3 << 2 | (b2 ^ b4) << 3
           : W == kChunk && SCORES ? b1 | b2 << 1 | b3 << 2
           : BYTES == 256 ? b2 | b0 << 1 | b1 << 2 | b3 << 3
                          : b2 | b1 << 1 | b3 << 2;  // 128 bytes: odd rows lie in the other banks
  }
  static constexpr uint32_t at(uint32_t r, uint32_t x) {  // bytes
    return r * BYTES + (x / CHUNK ^ swizzle(r)) * 16 + x % CHUNK * (uint32_t)sizeof(T);
  }
  // what a step of 16 t rows, 16 t BYTES apart, flips besides
  static constexpr uint32_t tile_bits(uint32_t t) { return swizzle(16 * t) * 16; }
};

template <typename V>
__device__ __forceinline__ std::remove_volatile_t<V> lds_read(uint32_t at) {
  return *(const __attribute__((address_space(3))) V*)at;
}
template <typename V>
__device__ __forceinline__ void lds_write(uint32_t at, V v) {
  *(__attribute__((address_space(3))) V*)at = v;
}
// Keeps the addresses made from x out of registers across a loop.
__device__ __forceinline__ uint32_t afresh(uint32_t x) {
  asm volatile("" : "+v"(x));
  return x;
}

// The tile of rows c0 .. c0 + n - 1 (base: row c0) into LDS, rows past it as
// copies of the last one: sizeof(T) instructions of each of W / 16 waves.
template <typename T, int W>
__device__ __forceinline__ void load_rows(uint64_t base, int n, uint32_t lds, int wave,
                                          uint32_t lane) {
  typedef Rows<T, W> R;
  constexpr uint32_t SLOTS = W / R::CHUNK, ROWS = 64 / SLOTS;  // rows of an instruction
  const uint32_t r = lane / SLOTS, c = (lane % SLOTS ^ R::swizzle(r)) * 16;
#pragma unroll
  for (int i = 0; i < (int)sizeof(T); ++i) {
    const uint32_t piece = wave * (uint32_t)sizeof(T) + i, first = piece * ROWS;
    const uint32_t row = first + r < (uint32_t)n ? first + r : (uint32_t)n - 1;
    dma16(base, row * R::BYTES + (c ^ R::swizzle(first) * 16), lds + piece * 1024);
  }
}

// Operand along a row of scores: eight values from column 8 g (base: there) +
// X, X a multiple of 32.  `off`: a constant distance.
__device__ __forceinline__ Operand<bf16> score_operand(uint32_t base, int X, int off, bf16) {
  return {lds_read<bf16x8>((base ^ Rows<bf16, kChunk, true>::at(0, X)) + off)};
}
__device__ __forceinline__ Operand<float> score_operand(uint32_t base, int X, int off, float) {
  typedef Rows<float, kChunk, true> P;
  return {lds_read<f32x4>((base ^ P::at(0, X)) + off),
          lds_read<f32x4>((base ^ P::at(0, X + 4)) + off)};
}
// Operand along a row of Q or K: four values from column 4 g (base: there) + X
// and four from 16 further.
// (volatile: two loads must not become one that needs its halves moved)
template <int W>
__device__ __forceinline__ Operand<bf16> split_operand(uint32_t base, int X, int off, bf16) {
  const bf16x4 a = lds_read<volatile bf16x4>((base ^ Rows<bf16, W>::at(0, X)) + off);
  const bf16x4 b = lds_read<volatile bf16x4>((base ^ Rows<bf16, W>::at(0, X + 16)) + off);
  return {__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7)};
}
template <int W>
__device__ __forceinline__ Operand<float> split_operand(uint32_t base, int X, int off, float) {
  return {lds_read<f32x4>((base ^ Rows<float, W>::at(0, X)) + off),
          lds_read<f32x4>((base ^ Rows<float, W>::at(0, X + 16)) + off)};
}
// Operand across the rows: column X + lane % 16 of rows 8 g .. 8 g + 7, X a
// multiple of 16.  The transposing load hands the 16 lanes of a group the 16
// columns of four rows of which each lane has addressed four values.
template <typename T, int W>
__device__ __forceinline__ uint32_t column_base(uint32_t lane) {
  const uint32_t l = lane & 15, g = lane >> 4;
  return sizeof(T) == 2 ? Rows<T, W>::at(8 * g + (l >> 2), 4 * (l & 3)) : Rows<T, W>::at(8 * g, l);
}
template <int W>
__device__ __forceinline__ Operand<bf16> column_operand(uint32_t base, int X, int off, bf16) {
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) s16x4* Lds;
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)((base ^ Rows<bf16, W>::at(0, X)) + off));
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)((base ^ Rows<bf16, W>::at(4, X)) + off));
  return {__builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7))};
}
template <int W>
__device__ __forceinline__ Operand<float> column_operand(uint32_t base, int X, int off, float) {
  Operand<float> out;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    out.a[e] = lds_read<float>((base ^ Rows<float, W>::at(e, X)) + off);
    out.b[e] = lds_read<float>((base ^ Rows<float, W>::at(e + 4, X)) + off);
  }
  return out;
}

template <int D>
struct State {
  f32x4 t[D / 16];
};

// A wave's 16 columns of V for 64 tokens, vt's rows, by way of a part of LDS
// that is this wave's alone: loaded there as whole rows (straight into
// registers, 64 bytes of 16 rows at a time, took 5% longer and eight registers
// more), read as the operand they are, tokens 32 ks + 8 g .. + 7 in lane g.
template <typename T, int D>
struct ValueTile {
  typedef Rows<T, kChunk, true> R;
  static constexpr int BYTES = 16 * R::BYTES;  // of a wave
  Operand<T> v[2];
  // at: vt's first row of the wave, at token c0, of which n follow
  static __device__ __forceinline__ void load(const T* at, int64_t vt_ld, uint32_t n,
                                              uint32_t lds, uint32_t lane) {
    constexpr uint32_t SLOTS = R::BYTES / 16, ROWS = 64 / SLOTS;  // rows of an instruction
    const uint32_t r = lane / SLOTS, c = (lane % SLOTS ^ R::swizzle(r)) * 16;
    const uint32_t row = r * (uint32_t)(vt_ld * sizeof(T));
#pragma unroll
    for (uint32_t i = 0; i < 16 / ROWS; ++i) {
      const uint32_t t = c ^ R::swizzle(ROWS * i) * 16;
      // what is past the end is masked
      dma16(uniform_ptr(at + (int64_t)(ROWS * i) * vt_ld), row + (t < n * sizeof(T) ? t : 0),
            lds + i * 1024);
    }
  }
  __device__ __forceinline__ void read(uint32_t lds, uint32_t lane) {
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
      v[ks] = score_operand(lds + R::at(lane & 15, 8 * (lane >> 4)), 32 * ks, 0, T());
  }
  // tokens from n on become zeros
  __device__ __forceinline__ void mask(int n, int lane) {
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) keep_first(v[ks], n - 32 * ks - 8 * (lane >> 4));
  }
  // Whether any value of the wave's may be a NaN or an infinity: their sum is not finite.
  __device__ __forceinline__ bool spoilt() const {
    return __ballot(!(fabsf(sum8(v[0]) + sum8(v[1])) <= FLT_MAX)) != 0;
  }
  // The first token of the lane's column that is a NaN or an infinity (kChunk:
  // none); all such become zeros.
  __device__ __forceinline__ int take_spoilt(int lane) {
    int first = kChunk;
#pragma unroll
    for (int ks = 1; ks >= 0; --ks)
#pragma unroll
      for (int e = 7; e >= 0; --e)
        if (!finite(v[ks], e)) {
          first = 32 * ks + 8 * (lane >> 4) + e;
          clear(v[ks], e);
        }
#pragma unroll
    for (int m = 16; m < 64; m <<= 1) {
      const int other = __shfl_xor(first, m, 64);
      first = first < other ? first : other;
    }
    return first;
  }
};

// The decays over 7, 6, .. 0 tokens, the same in every lane.
struct Powers {
  float p[8];
  __device__ __forceinline__ explicit Powers(float rate) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      p[e] = uniform(exp2_fast(-rate * (float)(7 - e)));
  }
};

// x - hi's value i, exactly, where hi[i] is x cut or rounded to bf16.
template <int I>
__device__ __forceinline__ float rest(float x, bf16x2 hi) {
  const uint32_t u = __builtin_bit_cast(uint32_t, hi);
  return x - __uint_as_float(I ? u & 0xffff0000u : u << 16);
}
__device__ __forceinline__ bf16x2 rounded(float x0, float x1) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  return __builtin_convertvector((f32x2{x0, x1}), bf16x2);
}
__device__ __forceinline__ bf16x2 cut(float x0, float x1) {
  return __builtin_bit_cast(
      bf16x2, __builtin_amdgcn_perm(__float_as_uint(x1), __float_as_uint(x0), 0x07060302u));
}

// V times the tokens' decays, as operands whose sum it is: each product cut
// to its first eight significant bits, the next eight, the rest.  The last of two is
// rounded, since what is cut off would all be of one side (5e-6 of a long prompt's outputs).
template <int PARTS>
__device__ __forceinline__ void decayed(const Operand<bf16>& v, const float (&w)[8],
                                        Operand<bf16> (&out)[PARTS]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float x0 = (float)v.v[2 * i] * w[2 * i], x1 = (float)v.v[2 * i + 1] * w[2 * i + 1];
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
      const bf16x2 c = PARTS == 2 && p == 1 ? rounded(x0, x1) : cut(x0, x1);
      out[p].v[2 * i] = c[0];
      out[p].v[2 * i + 1] = c[1];
      if (p + 1 < PARTS) {
        x0 = rest<0>(x0, c);
        x1 = rest<1>(x1, c);
      }
    }
  }
}
template <int PARTS>
__device__ __forceinline__ void decayed(const Operand<float>& v, const float (&w)[8],
                                        Operand<float> (&out)[PARTS]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    out[0].a[e] = v.a[e] * w[e];
    out[0].b[e] = v.b[e] * w[4 + e];
  }
}

// S += K^T (decayed V) over 64 tokens; token t decays over last - t, last >= 63
// if WHOLE.  columns: K's tile plus column_base().
template <typename T, int D, int PARTS, bool WHOLE>
__device__ __forceinline__ void add_outer(State<D>& s, uint32_t columns, const ValueTile<T, D>& v,
                                          float rate, const Powers& pw, int last, int lane) {
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) {
    const int far = last - 32 * ks - 8 * (lane >> 4);  // of the lane's first token
    float w[8];
    if constexpr (WHOLE) {
      const float first = exp2_fast(-rate * (float)(far - 7));
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = first * pw.p[e];
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = exp2_fast(-rate * (float)(far > e ? far - e : 0));
    }
    Operand<T> b[PARTS];
    decayed(v.v[ks], w, b);
#pragma unroll
    for (int k0 = 0; k0 < D / 16; k0 += 4) {  // products on one accumulator stay apart
      Operand<T> a[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        a[k] = column_operand<D>(columns, 16 * (k0 + k), 32 * ks * Rows<T, D>::BYTES, T());
#pragma unroll
      for (int p = PARTS - 1; p >= 0; --p)
#pragma unroll
        for (int k = 0; k < 4; ++k) s.t[k0 + k] = mma(a[k], b[p], s.t[k0 + k]);
      if (D == 128) __builtin_amdgcn_sched_barrier(0);  // registers
    }
  }
}

struct ChunkArgs {
  const void *q, *k, *vt;
  void* o;
  int64_t vt_ld;
  const float* slopes;
  const int32_t* lengths;
  const float* state_in;
  float* state_out;
  float* slots;  // [n_seq][heads][segments][D][D], or null: each segment makes its own state
  int64_t tokens;
  int32_t heads, segments, segment;  // segment: tokens of one, a multiple of 64
  int32_t scanned;
  int32_t cut[kMaxAlone - 1];  // slots null: where segments 1 .. begin
  float scale;
};

__device__ __forceinline__ int64_t length_of(const int32_t* lengths, int64_t seq, int64_t tokens) {
  if (!lengths) return tokens;
  const int64_t n = lengths[seq];
  return n < 0 ? 0 : n < tokens ? n : tokens;
}

// A wave's share of a state in the workspace lies tile by tile as its lanes
// hold it; a caller's is [D][D].  f(tile, workspace index, row, column).
template <int D, typename F>
__device__ __forceinline__ void for_state(State<D>& s, F&& f) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int kt = 0; kt < D / 16; ++kt)
    f(s.t[kt], (wave * (D / 16) + kt) * 256 + lane * 4, 16 * kt + 4 * (lane >> 4),
      wave * 16 + (lane & 15));
}
template <int D>
__device__ __forceinline__ void read_state(State<D>& s, const float* p) {
  for_state(s, [&](f32x4& t, int, int row, int col) {
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = p[(row + i) * D + col];
  });
}
template <int D>
__device__ __forceinline__ void write_state(State<D>& s, float* p) {
  for_state(s, [&](f32x4& t, int, int row, int col) {
#pragma unroll
    for (int i = 0; i < 4; ++i) p[(row + i) * D + col] = t[i];
  });
}

template <int D>
__device__ __forceinline__ void fade(State<D>& s, const Decay& decay) {
  for_state(s, [&](f32x4& t, int, int, int) {
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = decay(t[i]);
  });
}

// Where there are too few heads to fill the chip, a sequence is cut into
// segments.  This kernel leaves in slot j + 1 what segment j adds to the state
// (segment 0: what it makes of state_in), for each segment that another
// follows, and in slot 0 state_in itself, which the outputs' kernel may
// overwrite in place.
template <typename T, int D>
__global__ __launch_bounds__(4 * D, sizeof(T) == 2 ? 4 : 2) void la_state_kernel(ChunkArgs a) {
  typedef Rows<T, D> R;
  typedef ValueTile<T, D> V;
  __shared__ __align__(1024) unsigned char rows[2 * R::TOTAL + 2 * (D / 16) * V::BYTES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int seg = blockIdx.x % (a.segments - 1);
  const int64_t hs = blockIdx.x / (a.segments - 1);  // sequence and head
  const int head = hs % a.heads;
  const int64_t len = length_of(a.lengths, hs / a.heads, a.tokens);
  const int64_t begin = (int64_t)seg * a.segment, end = begin + a.segment;
  float* slot = a.slots + (hs * a.segments + seg) * (D * D);
  State<D> s;
  if (seg == 0 && a.state_in && len > 0) {
    read_state(s, a.state_in + hs * (D * D));
    for_state(s, [&](f32x4& t, int at, int, int) { *reinterpret_cast<f32x4*>(slot + at) = t; });
  }
  if (end >= len) return;  // no segment follows
  constexpr int PARTS = sizeof(T) == 2 ? 3 : 1;
  const float rate = decay_rate(a.slopes[head]);
  const Powers pw(rate);
  if (seg == 0 && a.state_in) {
    fade(s, Decay(a.slopes[head], a.segment));
  } else {
    for_state(s, [&](f32x4& t, int, int, int) { t = f32x4{0.f, 0.f, 0.f, 0.f}; });
  }
  const T* k = (const T*)a.k + hs * a.tokens * D;
  const T* vt = (const T*)a.vt + (hs * D + wave * 16) * a.vt_ld;
  uint32_t buf = (uint32_t)(uintptr_t)(lds_void_t*)rows, next = buf + R::TOTAL;
  uint32_t v_buf = buf + 2 * R::TOTAL + wave * (2 * V::BYTES), v_next = v_buf + V::BYTES;
  load_rows<T, D>(uniform_ptr(k + begin * D), kChunk, buf, wave, lane);
  V::load(vt + begin, a.vt_ld, kChunk, v_buf, lane);
  for (int64_t c0 = begin; c0 < end; c0 += kChunk) {
    barrier_all();
    if (c0 + kChunk < end) {
      load_rows<T, D>(uniform_ptr(k + (c0 + kChunk) * D), kChunk, next, wave, lane);
      V::load(vt + c0 + kChunk, a.vt_ld, kChunk, v_next, lane);
    }
    V v;
    v.read(v_buf, lane);
    add_outer<T, D, PARTS, true>(s, afresh(buf + column_base<T, D>(lane)), v, rate, pw,
                                 (int)(end - 1 - c0), lane);
    uint32_t t = buf;
    buf = next;
    next = t;
    t = v_buf;
    v_buf = v_next;
    v_next = t;
  }
  for_state(s, [&](f32x4& t, int at, int, int) {
    *reinterpret_cast<f32x4*>(slot + D * D + at) = t;
  });
}

// Slot j becomes the state before segment j: x_j = lambda^segment x_{j-1} +
// slot j, in place, the chain in fp64 (a rounded factor would add up over the
// segments).
template <int D>
__global__ __launch_bounds__(256) void la_scan_kernel(ChunkArgs a) {
  constexpr int GROUPS = D * D / 512;
  const int64_t hs = blockIdx.x / GROUPS;
  const int64_t len = length_of(a.lengths, hs / a.heads, a.tokens);
  const int last = len > 0 ? (int)((len - 1) / a.segment) : 0;  // the sequence's last segment
  const double lambda = exp(-(double)a.slopes[hs % a.heads] * a.segment);
  float2* p = reinterpret_cast<float2*>(a.slots + hs * a.segments * (D * D)) +
              (blockIdx.x % GROUPS) * 256 + threadIdx.x;
  constexpr int STEP = D * D / 2;
  double x = 0.0, y = 0.0;
  int j = 1;
  for (; j + 7 <= last; j += 8) {
    float2 v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = p[(int64_t)(j + i) * STEP];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x = lambda * x + v[i].x;
      y = lambda * y + v[i].y;
      p[(int64_t)(j + i) * STEP] = make_float2((float)x, (float)y);
    }
  }
  for (; j <= last; ++j) {
    const float2 v = p[(int64_t)j * STEP];
    x = lambda * x + v.x;
    y = lambda * y + v.y;
    p[(int64_t)j * STEP] = make_float2((float)x, (float)y);
  }
}

// S as the two-part (fp32: whole) operand of Q S: columns 32 kk + 4 g .. + 3 and
// 32 kk + 16 + 4 g .. + 3 of k in lane g.
template <int D>
__device__ __forceinline__ void state_operand(const State<D>& s, int kk, Operand<bf16> (&out)[2]) {
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const f32x4 t = s.t[2 * kk + (e >> 2)];
    const float x0 = t[e & 3], x1 = t[(e & 3) + 1];
    const bf16x2 hi = rounded(x0, x1), lo = rounded(rest<0>(x0, hi), rest<1>(x1, hi));
    out[0].v[e] = hi[0];
    out[0].v[e + 1] = hi[1];
    out[1].v[e] = lo[0];
    out[1].v[e + 1] = lo[1];
  }
}
template <int D>
__device__ __forceinline__ void state_operand(const State<D>& s, int kk, Operand<float> (&out)[1]) {
  out[0] = {s.t[2 * kk], s.t[2 * kk + 1]};
}

// Four neighbouring scores of one token into LDS.
__device__ __forceinline__ void store_scores(uint32_t at, int part_stride, f32x4 v, bf16) {
  const bf16x2 h0 = rounded(v[0], v[1]), h1 = rounded(v[2], v[3]);
  const bf16x2 l0 = rounded(rest<0>(v[0], h0), rest<1>(v[1], h0));
  const bf16x2 l1 = rounded(rest<0>(v[2], h1), rest<1>(v[3], h1));
  lds_write(at, (bf16x4)__builtin_shufflevector(h0, h1, 0, 1, 2, 3));
  lds_write(at + part_stride, (bf16x4)__builtin_shufflevector(l0, l1, 0, 1, 2, 3));
}
__device__ __forceinline__ void store_scores(uint32_t at, int, f32x4 v, float) {
  lds_write(at, v);
}

__device__ __forceinline__ void store_out(bf16* p, f32x4 v) {
  *reinterpret_cast<bf16x4*>(p) = __builtin_convertvector(v, bf16x4);
}
__device__ __forceinline__ void store_out(float* p, f32x4 v) { *reinterpret_cast<f32x4*>(p) = v; }

// The outputs of one segment, from the state before it.  LAST: the sequence's
// last segment, which leaves the final state.
template <typename T, int D, bool LAST>
__device__ __forceinline__ void chunks_of(const ChunkArgs& a, unsigned char* rows, int seg,
                                          int64_t hs, int64_t len, int64_t begin, int64_t end) {
  constexpr int TWO = sizeof(T) == 2 ? 2 : 1;  // parts of scores and of S
  constexpr int PARTS = sizeof(T) == 2 ? (LAST ? 3 : 2) : 1;  // LAST: S is an output, in fp32
  typedef Rows<T, D> R;
  typedef Rows<T, kChunk, true> P;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int head = hs % a.heads;
  const int64_t seq = hs / a.heads;
  const float slope = a.slopes[head], rate = decay_rate(slope);

  const T* q = (const T*)a.q + hs * a.tokens * D;
  const T* k = (const T*)a.k + hs * a.tokens * D;
  const T* vt = (const T*)a.vt + (hs * D + wave * 16) * a.vt_ld;
  const int64_t o_ld = (int64_t)a.heads * D;
  T* o = (T*)a.o + seq * a.tokens * o_ld + head * D + wave * 16;
  const Powers pw(rate);
  // LDS: K's rows of this chunk and the next, Q's, V's (each wave its own),
  // the scores.  Q and V have one place each: the next chunk's are loaded once
  // all that is in it has been read.
  typedef ValueTile<T, D> V;
  uint32_t buf = (uint32_t)(uintptr_t)(lds_void_t*)rows, next = buf + R::TOTAL;
  const uint32_t q_at = buf + 2 * R::TOTAL, v_at = q_at + R::TOTAL + wave * V::BYTES;
  const uint32_t scores = q_at + R::TOTAL + (D / 16) * V::BYTES;
  V v;
  auto tokens = [&](int64_t c0) { return end - c0 < kChunk ? (int)(end - c0) : kChunk; };
  auto load_k = [&](int64_t c0, uint32_t to, int lane) {
    load_rows<T, D>(uniform_ptr(k + c0 * D), tokens(c0), to, wave, lane);
  };
  auto load_q = [&](int64_t c0, int lane) {
    load_rows<T, D>(uniform_ptr(q + c0 * D), tokens(c0), q_at, wave, lane);
  };
  auto load_v = [&](int64_t c0, int lane) { V::load(vt + c0, a.vt_ld, tokens(c0), v_at, lane); };
  const bool alone = seg > 0 && !a.slots;  // makes its own state
  if (begin < end && !alone) {
    const int lane = threadIdx.x & 63;
    load_k(begin, buf, lane);
    load_q(begin, lane);
    load_v(begin, lane);
  }

  State<D> s;
  if (alone) {
    // As la_state_kernel does, from the sequence's start; the last step brings
    // the first chunk's K and V.  V's second place is where Q's rows will be, of
    // which each wave loads the bytes that were its V's.
    const int lane = threadIdx.x & 63;
    constexpr int PARTS = sizeof(T) == 2 ? 3 : 1;
    static_assert((int)sizeof(T) * 1024 == V::BYTES, "Q's rows of a wave, V's place");
    uint32_t v_now = q_at + wave * V::BYTES, v_next = v_at;
    if (begin / kChunk % 2 == 0) {
      v_now = v_at;
      v_next = q_at + wave * V::BYTES;
    }
    load_k(0, buf, lane);
    V::load(vt, a.vt_ld, kChunk, v_now, lane);
    if (a.state_in) {
      read_state(s, a.state_in + hs * (D * D));
      fade(s, Decay(slope, (double)begin));
    } else {
      for_state(s, [&](f32x4& t, int, int, int) { t = f32x4{0.f, 0.f, 0.f, 0.f}; });
    }
    for (int64_t c0 = 0; c0 < begin; c0 += kChunk) {
      barrier_all();
      load_k(c0 + kChunk, next, lane);
      V::load(vt + c0 + kChunk, a.vt_ld, tokens(c0 + kChunk), v_next, lane);
      v.read(v_now, lane);
      add_outer<T, D, PARTS, true>(s, afresh(buf + column_base<T, D>(lane)), v, rate, pw,
                                   (int)(begin - 1 - c0), lane);
      uint32_t t = buf;
      buf = next;
      next = t;
      t = v_now;
      v_now = v_next;
      v_next = t;
    }
    wait_lds();
    load_q(begin, lane);
  } else if (seg == 0) {
    if (!a.state_in)
      for_state(s, [&](f32x4& t, int, int, int) { t = f32x4{0.f, 0.f, 0.f, 0.f}; });
    else if (a.slots && len > 0)
      for_state(s, [&](f32x4& t, int at, int, int) {
        t = *reinterpret_cast<const f32x4*>(a.slots + hs * a.segments * (D * D) + at);
      });
    else
      read_state(s, a.state_in + hs * (D * D));
  } else {
    const float* slot = a.slots + (hs * a.segments + seg) * (D * D);
    for_state(s, [&](f32x4& t, int at, int, int) {
      t = *reinterpret_cast<const f32x4*>(slot + at);
    });
    if (!a.scanned) {  // the segments before the last one, each with its decay
      const double step = exp(-(double)slope * a.segment);
      double w = step;
      for (int j = seg - 1; j > 0; --j, w *= step) {
        const Decay decay(w);
        for_state(s, [&](f32x4& t, int at, int, int) {
          const f32x4 x = *reinterpret_cast<const f32x4*>(slot - (int64_t)(seg - j) * (D * D) + at);
#pragma unroll
          for (int i = 0; i < 4; ++i) t[i] = decay(x[i], t[i]);
        });
      }
    }
  }
  // (made while the loads above are on their way)  Over a chunk, and over the ragged
  // one at a sequence's end; for a state that is only read by a segment's own bf16
  // outputs one part will do (2^-25 a chunk; what 288 GB hold gives a segment at most
  // 8600 of them, 2^-12 where a bf16 value is rounded by 2^-8).
  constexpr bool TWO_PART_DECAY = LAST || sizeof(T) == 4;
  const Decay whole(slope, kChunk), ragged(slope, (int)(end - begin) & (kChunk - 1));
  float tile_decay[4];
#pragma unroll
  for (int tt = 0; tt < 4; ++tt) tile_decay[tt] = uniform(a.scale * exp2_fast(-rate * (float)(16 * tt)));
  // the scores' tiles of this wave, 4 tq + st a digit: tokens 16 tq .., keys 16
  // st ..; the ten on and below the diagonal, the waves with one more than the
  // others on different SIMDs (wave w's is w % 4).  The two beside an even diagonal
  // tile are read too and stay zeros.
  constexpr int TILES = D == 64 ? 2 : 1;
  const uint32_t tiles =
      D == 64    ? (wave == 0 ? 0xf0 : wave == 1 ? 0xe54 : wave == 2 ? 0xa98 : 0xdc)
      : wave < 4 ? (wave == 0 ? 0x0 : wave == 1 ? 0x54 : wave == 2 ? 0x8 : 0x9)
                 : (wave == 4 ? 0xa : wave == 5 ? 0xc : wave == 6 ? 0xed : 0xf);
  const bool one_more = wave == 1 || wave == (D == 64 ? 2 : 6);
  if (wave < 2) {
    const int lane = threadIdx.x & 63, at = 32 * wave;
    store_scores(scores + P::at(at + (lane & 15), at + 16 + 4 * (lane >> 4)), P::TOTAL,
                 f32x4{0.f, 0.f, 0.f, 0.f}, T());
  }
  __builtin_amdgcn_s_waitcnt(0);  // S is here: no wait for it among the chunks' loads
  int64_t c0 = begin;
  // One chunk of n tokens: 64, or (WHOLE false) a sequence's last ones.
  auto chunk = [&](auto whole_chunk, int n, bool update) {
    constexpr bool WHOLE = decltype(whole_chunk)::value;
    // made afresh in each chunk: what follows from it is more than registers hold
    const uint32_t lane = afresh(threadIdx.x & 63), col = lane & 15, g = lane >> 4;
    barrier_all();
    const bool more = c0 + kChunk < end;
    if (more) load_k(c0 + kChunk, next, lane);
    v.read(v_at, lane);
    const uint32_t along = afresh(R::at(col, 4 * g));
    auto score_tile = [&](int i) {
      const uint32_t tq = tiles >> (4 * i + 2) & 3, st = tiles >> (4 * i) & 3;
      const uint32_t k_tile = (along ^ R::tile_bits(st)) + buf + 16 * st * R::BYTES;
      const uint32_t q_tile = (along ^ R::tile_bits(tq)) + q_at + 16 * tq * R::BYTES;
      Operand<T> kf[D / 32], qf[D / 32];
#pragma unroll
      for (int kk = 0; kk < D / 32; ++kk) {
        kf[kk] = split_operand<D>(k_tile, 32 * kk, 0, T());
        qf[kk] = split_operand<D>(q_tile, 32 * kk, 0, T());
      }
      const int far = (int)(16 * (tq - st) + col - 4 * g);  // from the lane's first key
      f32x4 w;
      if (D == 128 && st < tq) {
        const float last = a.scale * exp2_fast(-rate * (float)(far - 3));
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = last * pw.p[4 + i];
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = a.scale * exp2_fast(-rate * (float)(far - i));
      }
      f32x4 p = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < D / 32; ++kk) p = mma(kf[kk], qf[kk], p);
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i] = far >= i ? p[i] * w[i] : 0.f;
      store_scores(scores + P::at(16 * tq + col, 16 * st + 4 * g), P::TOTAL, p, T());
    };
#pragma unroll
    for (int i = 0; i < TILES; ++i) score_tile(i);
    if (one_more) score_tile(TILES);
    if (more) {
      wait_lds();  // v is in its registers
      load_v(c0 + kChunk, lane);
    }
    if (!WHOLE) v.mask(n, lane);
    f32x4 out[4];
#pragma unroll
    for (int tt = 0; tt < 4; ++tt) out[tt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk) {
      Operand<T> sf[TWO];
      state_operand(s, kk, sf);
      Operand<T> qf[4];
#pragma unroll
      for (int tt = 0; tt < 4; ++tt)
        qf[tt] = split_operand<D>((along ^ R::tile_bits(tt)) + q_at, 32 * kk, 16 * tt * R::BYTES, T());
#pragma unroll
      for (int p = TWO - 1; p >= 0; --p)
#pragma unroll
        for (int tt = 0; tt < 4; ++tt) out[tt] = mma(sf[p], qf[tt], out[tt]);
      if (D == 128) __builtin_amdgcn_sched_barrier(0);  // registers
    }
#pragma unroll
    for (int tt = 0; tt < 4; ++tt) out[tt] *= exp2_fast(-rate * (float)(col + 1)) * tile_decay[tt];
    barrier_lds();
    if (more) load_q(c0 + kChunk, lane);
    // A NaN or an infinity among V's tokens would reach the chunk's earlier outputs
    // too, whose weights for it are zeros: it is left out of V, and what comes of it is
    // a NaN in its column of S and in the outputs from its token on.
    if (__builtin_expect(v.spoilt(), 0)) {
      const float nan = __builtin_nanf("");
      const int first = v.take_spoilt(lane);
      if (first < kChunk) for_state(s, [&](f32x4& t, int, int, int) { t = f32x4{nan, nan, nan, nan}; });
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int from = __shfl(first, 4 * g + i, 64);
#pragma unroll
        for (int tt = 0; tt < 4; ++tt)
          if (16 * tt + (int)col >= from) out[tt][i] = nan;
      }
    }

    const uint32_t weights = afresh(scores + P::at(col, 8 * g));
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int p = TWO - 1; p >= 0; --p)
#pragma unroll
        for (int tt = 2 * ks; tt < 4; ++tt)
          out[tt] = mma(v.v[ks],
                        score_operand(weights ^ P::tile_bits(tt), 32 * ks,
                                      16 * tt * P::BYTES + p * P::TOTAL, T()),
                        out[tt]);
    if (D == 128) __builtin_amdgcn_sched_barrier(0);
    T* at = o + c0 * o_ld + col * o_ld + 4 * g;
#pragma unroll
    for (int tt = 0; tt < 4; ++tt) {
      if (WHOLE || 16 * tt + (int)col < n) store_out(at, out[tt]);
      at += 16 * o_ld;
    }
    if (update) {
      if constexpr (!WHOLE) fade(s, ragged);
      else if constexpr (TWO_PART_DECAY) fade(s, whole);
      else for_state(s, [&](f32x4& t, int, int, int) { t *= whole.hi; });
      add_outer<T, D, PARTS, WHOLE>(s, afresh(buf + column_base<T, D>(lane)), v, rate,
                                    pw, n - 1, lane);
    }
    const uint32_t t = buf;
    buf = next;
    next = t;
    c0 += kChunk;
  };
  while (c0 + kChunk <= end)
    chunk(std::true_type(), kChunk, (LAST && a.state_out) || c0 + kChunk < end);
  if constexpr (LAST) {
    if (c0 < end) chunk(std::false_type(), (int)(end - c0), a.state_out != nullptr);
    if (a.state_out) write_state(s, a.state_out + hs * (D * D));
  }
}

template <typename T, int D>
__global__ __launch_bounds__(4 * D, sizeof(T) == 2 ? 4 : 2) void la_chunk_kernel(ChunkArgs a) {
  __shared__ __align__(1024) unsigned char rows[3 * Rows<T, D>::TOTAL +
                                                (D / 16) * ValueTile<T, D>::BYTES +
                                                (sizeof(T) == 2 ? 2 : 1) * Rows<T, kChunk>::TOTAL];
  const int seg = blockIdx.x % a.segments;
  const int64_t hs = blockIdx.x / a.segments;
  const int64_t len = length_of(a.lengths, hs / a.heads, a.tokens);
  int64_t begin = (int64_t)seg * a.segment, end = begin + a.segment;
  if (!a.slots) {
    begin = seg > 0 ? a.cut[seg - 1] : 0;
    end = seg + 1 < a.segments ? a.cut[seg] : a.tokens;
  }
  if (end < len)
    chunks_of<T, D, false>(a, rows, seg, hs, len, begin, end);
  else if (seg == 0 || begin < len)
    chunks_of<T, D, true>(a, rows, seg, hs, len, begin, len);
}

// Tokens of a segment, a multiple of 64, and how many there are: as many as
// give each CU a workgroup, or two where they then have eight chunks each (one
// segment a head once the heads alone do).  With 256 / 512 workgroups: 12 x 4680
// tokens (d = 128) 42 / 50 us, but 12 x 32760 163 / 158, with d = 64 85 / 71, and 24 x
// 32760 313 / 306.
//
// A bf16 chunk takes about as long as its segment's state costs to write, sum and
// read, so segments have two unless there are few of them (one chunk / two,
// d = 128: 32 x 512 tokens 33 / 26 us, 16 x 640 24.7 / 22.6, but 8 x 1024 24.6 / 25.3,
// and with d = 64 4 x 1559 13.0 / 15.1), and up to four stay together (64 x 256: 26 in
// four segments, 23 in two, 20 in one).  An fp32 chunk takes three times as long
// (8 x 2000, d = 128: one 44 us, two 54).
struct Segments {
  int64_t tokens, count;
};
Segments segments_of(int dtype, int64_t heads, int64_t L) {
  const int64_t chunks = (L + kChunk - 1) / kChunk;
  const int64_t groups = heads * chunks >= 512 * 8 ? 512 : 256;
  const int64_t most = heads > 0 ? groups / heads : 1;
  const bool quick = dtype == ACID_BF16;
  if (chunks <= (quick ? 4 : 1) || most <= 1) return {chunks * kChunk, 1};
  int64_t per = (chunks + most - 1) / most;
  if (quick && per == 1 && heads * chunks > 128) per = 2;
  return {per * kChunk, (chunks + per - 1) / per};
}

// Up to this many segments the outputs' kernel adds those before its own
// itself; more take a scan, a launch of its own (folded / scanned, d = 128: 5
// segments of 48 x 1280 tokens 40.1 / 41.4 us, 6 of 40 x 1536 41.7 / 41.8, 8 of 32 x
// 2000 47.8 / 45.8; d = 64: 8 of 32 x 2000 25.1 / 26.2, 9 of 28 x 1728 22.7 / 21.9, 25
// of 4 x 1559 15.8 / 13.1; fp32, d = 64: 5 of 8 x 300 14.0 / 15.8, 10 of 8 x 600 16.7 /
// 15.8; d = 128: 7 of 8 x 400 30.4 / 30.3, 8 of 8 x 500 34.4 / 32.5).
int64_t most_folded(int d) { return d == 64 ? 8 : 6; }

// Segments that each make the state before them from the sequence's start: one
// launch and no workspace, but the last of n segments goes through K and V of
// all tokens (at r of the time that their outputs would take; cut for 0.3 to 0.5
// the times are within 5%, best for 0.3 with d = 64 and for 0.4 with 128).
constexpr double kStateShare = 0.4;
double alone_time(int64_t chunks, int n) {  // in chunks of outputs, of the longest segment
  return chunks * kStateShare / (1 - pow(1 - kStateShare, n));
}

// How many of those to use, or 0: where their time is less than that of the
// launches they save (three bf16 chunks of outputs, half an fp32 one) and of the
// form above.  That one / this, bf16: 16 heads of 509 tokens (d = 64) 12.6 / 10.4 us,
// 32 of 512 (d = 128) 23.5 / 17.8, 128 of 509 (d = 64) 20.5 / 16.1, 96 of 1000 (d =
// 128) 53.5 / 43.8, but 24 of 2045 (d = 128) 39 / 52; fp32: 100 of 300 (d = 64) 28.3 /
// 21.6, 128 of 500 (d = 128) 87.7 / 74.5, but 32 of 300 (d = 128) 34.3 / 39.4.
//
// Past 128 heads, with a segment each in the form above, two or three, of fp32
// (d = 64) from eight chunks on: bf16, d = 64: 150 of 500 24.1 / 19.9, 240 of 1000
// 43.2 / 37.0, 256 of 2000 78.8 / 68.6; fp32: 150 of 500 49 / 42, 256 of 1000 96 / 92,
// 200 of 130 21.7 / 22.4.  Heads of 128 fill a CU's LDS with two workgroups: bf16 takes
// three segments from eight chunks on (150 of 1000 67.4 / 61.1, of 300 26.4 / 28.4),
// two not at all while heads get one there (200 of 300 28.4 / 32.3, of 1000 68.6 / 71.7);
// fp32 150 of 500 110 / 118, 200 of 500 112 / 140.  Long sequences that get two
// workgroups a CU above keep them, but for heads of 128 that get four segments
// there and two here (128 of 4093 190 / 170), or two and two (200 of 2000 152 / 141).
int alone_of(int dtype, int64_t heads, int64_t L, int d) {
  const int64_t chunks = (L + kChunk - 1) / kChunk;
  const bool quick = dtype == ACID_BF16;
  if (chunks < 2 || heads < 1) return 0;
  if (heads > 128) {
    if (chunks < (quick ? 3 : 8) || (!quick && d == 128)) return 0;
    if (d == 128 && heads * chunks < 512 * 8 && (chunks < 8 || 512 / heads < 3)) return 0;
    return heads <= 256 ? (int)(512 / heads) : quick && d == 64 && heads <= 384 ? 2 : 0;
  }
  const int64_t most = 256 / heads;
  if (quick && heads * chunks >= 512 * 8) return d == 128 && 512 / heads <= 4 ? 2 : 0;
  const int64_t apart = chunks > 2 ? chunks - 1 : 2;
  const int n = (int)(most < apart ? most < kMaxAlone ? most : kMaxAlone
                                   : apart < kMaxAlone ? apart : kMaxAlone);
  int64_t per = (chunks + most - 1) / most;
  if (quick && per == 1 && heads * chunks > 128) per = 2;
  return alone_time(chunks, n) <= (quick ? 3 : 0.5) + (1 + kStateShare) * per ? n : 0;
}

// Where their segments begin, so that they end at the same time: segment j of c
// chunks after C others takes r C + c, and what is before segment j + 1 is
// C (1 - r) + that time.
void cut_alone(int64_t chunks, int n, int32_t (&cut)[kMaxAlone - 1]) {
  const double each = alone_time(chunks, n);
  double c = 0;
  for (int j = 0; j + 1 < n; ++j) {
    c = c * (1 - kStateShare) + each;
    const int64_t least = j ? cut[j - 1] / kChunk + 1 : 1, most = chunks - (n - 1 - j);
    const int64_t at = (int64_t)(c + 0.5);
    cut[j] = (int32_t)((at < least ? least : at > most ? most : at) * kChunk);
  }
}

template <typename T, int D>
hipError_t launch_chunks(const ChunkArgs& a, int64_t heads, hipStream_t s) {
  if (a.slots) {
    hipLaunchKernelGGL((la_state_kernel<T, D>), dim3((unsigned)(heads * (a.segments - 1))),
                       dim3(4 * D), 0, s, a);
    if (a.scanned)
      hipLaunchKernelGGL((la_scan_kernel<D>), dim3((unsigned)(heads * (D * D / 512))), dim3(256),
                         0, s, a);
  }
  hipLaunchKernelGGL((la_chunk_kernel<T, D>), dim3((unsigned)(heads * a.segments)), dim3(4 * D), 0,
                     s, a);
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
  // (an fp32 call has no fewer segments than a bf16 one)
  return acid_linear_attention_workspace_needed(ACID_F32, n_seq, n_heads, seq_len, head_dim, 1);
}

size_t acid_linear_attention_workspace_needed(int32_t dtype, int64_t n_seq, int32_t n_heads,
                                              int64_t seq_len, int32_t head_dim,
                                              int32_t in_place) {
  if (check_heads(dtype, n_seq, n_heads, head_dim) != ACID_OK || seq_len < 0 ||
      seq_len > kMaxTokens)
    return 0;
  const int64_t heads = n_seq * n_heads;
  if (!in_place && alone_of(dtype, heads, seq_len, head_dim) > 1) return 0;
  const Segments seg = segments_of(dtype, heads, seq_len);
  return seg.count > 1 ? (size_t)(seg.count * heads * head_dim * head_dim * 4) : 0;
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
  if (seq_len > kMaxTokens)
    return set_error(ACID_ERR_SHAPE, "seq_len %lld: at most 2^28", (long long)seq_len);
  if (vt_ld < round_up(seq_len, 8) || vt_ld % 8 || vt_ld > ((int64_t)1 << 28))
    return set_error(ACID_ERR_SHAPE,
                     "vt_ld %lld must be a multiple of 8, >= round_up(L, 8) and <= 2^28",
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
  const struct {
    const void* p;
    int64_t bytes;
  } small[] = {{slopes_dev, n_heads * (int64_t)4}, {lengths_dev, n_seq * 4}};
  for (const auto& v : small)
    if (bytes_overlap(o_dev, qkv, v.p, v.bytes) || bytes_overlap(state_out_dev, states, v.p, v.bytes))
      return set_error(ACID_ERR_INVALID_ARG, "o or state_out overlaps the slopes or the lengths");
  // (in place, a segment may end before another has read the state)
  const bool in_place = state_in_dev && state_in_dev == state_out_dev;
  const int alone = in_place ? 0 : alone_of(dtype, heads, seq_len, head_dim);
  const Segments seg = alone > 1 ? Segments{0, alone} : segments_of(dtype, heads, seq_len);
  const bool slots = alone <= 1 && seg.count > 1;
  if (slots) {
    const int64_t need = seg.count * states;
    if ((int64_t)workspace_bytes < need || !workspace_dev)
      return set_error(ACID_ERR_SHAPE, "workspace of %lld bytes, %lld needed",
                       (long long)(workspace_dev ? workspace_bytes : 0), (long long)need);
    for (const void* p : {q_dev, k_dev, (const void*)o_dev})
      if (bytes_overlap(workspace_dev, need, p, qkv))
        return set_error(ACID_ERR_INVALID_ARG, "the workspace overlaps q, k or o");
    if (bytes_overlap(workspace_dev, need, vt_dev, vtb) ||
        bytes_overlap(workspace_dev, need, state_in_dev, states) ||
        bytes_overlap(workspace_dev, need, state_out_dev, states))
      return set_error(ACID_ERR_INVALID_ARG, "the workspace overlaps vt or a state");
    for (const auto& v : small)
      if (bytes_overlap(workspace_dev, need, v.p, v.bytes))
        return set_error(ACID_ERR_INVALID_ARG, "the workspace overlaps the slopes or the lengths");
  }
  StreamDevice on;
  ACID_TRY(on.enter(stream));
  ChunkArgs a = {q_dev, k_dev, vt_dev, o_dev, vt_ld, slopes_dev, lengths_dev, state_in_dev,
                 state_out_dev, slots ? (float*)workspace_dev : nullptr, seq_len, n_heads,
                 (int32_t)seg.count, (int32_t)seg.tokens, seg.count > most_folded(head_dim), {},
                 scale};
  if (alone > 1) cut_alone((seq_len + kChunk - 1) / kChunk, alone, a.cut);
  hipError_t e;
  if (dtype == ACID_BF16)
    e = head_dim == 64 ? launch_chunks<bf16, 64>(a, heads, stream)
                       : launch_chunks<bf16, 128>(a, heads, stream);
  else
    e = head_dim == 64 ? launch_chunks<float, 64>(a, heads, stream)
                       : launch_chunks<float, 128>(a, heads, stream);
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
  if (slots_dev && n_rows > kMaxSlotted)
    return set_error(ACID_ERR_SHAPE, "n_rows %lld: with slots at most 65536", (long long)n_rows);
  if (n_slots < 0 || n_slots > INT32_MAX || n_slots * n_heads >= ((int64_t)1 << 40) ||
      (!slots_dev && n_slots < n_rows))
    return set_error(ACID_ERR_SHAPE, "n_slots %lld: in [0, 2^31), times n_heads < 2^40, without slots >= n_rows",
                     (long long)n_slots);
  for (int64_t ld : {q_ld, k_ld, v_ld, o_ld})
    if (ld < width || ld * size % 16 || ld > ((int64_t)1 << 32))
      return set_error(ACID_ERR_SHAPE,
                       "row strides must be >= n_heads * head_dim, <= 2^32 and whole 16 bytes");
  if (n_rows == 0 || n_slots == 0) return ACID_OK;  // (no slots: padding rows alone)
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
  const struct {
    const void* p;
    int64_t bytes;
  } small[] = {{slopes_dev, n_heads * (int64_t)4}, {slots_dev, n_rows * 4}};
  for (const auto& v : small)
    if (rows_overlap(o_dev, n_rows, w, o_ld * size, v.p, 1, v.bytes, v.bytes) ||
        bytes_overlap(state_out_dev, states, v.p, v.bytes))
      return set_error(ACID_ERR_INVALID_ARG, "o or state_out overlaps the slopes or the slots");
  if (state_in_dev != state_out_dev &&
      bytes_overlap(state_in_dev, states, state_out_dev, states))
    return set_error(ACID_ERR_INVALID_ARG, "state_in and state_out: one buffer or apart");
  StreamDevice on;
  ACID_TRY(on.enter(stream));
  const StepArgs a = {q_dev, k_dev, v_dev, o_dev, q_ld, k_ld, v_ld, o_ld, slopes_dev, slots_dev,
                      state_in_dev, state_out_dev, n_rows, n_slots, n_heads, scale};
  const hipError_t e = launch_step(dtype, head_dim, a, stream);
  return e == hipSuccess ? ACID_OK : check_hip(e, "linear attention step");
}

}  // extern "C"
