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
#include "tiles.h"

namespace acid {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

struct Fp8Args {
  const uint8_t *a, *w;
  const float *a_scales, *w_scales, *bias, *gate, *residual;
  void* out;
  int64_t a_ld, a_scales_ld, residual_ld, out_ld;
  int32_t M, N, K, groups, kind;
  bool vec;  // 16 bytes of outputs (and residual) may be read and written at once
};

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

// ------------------------------------------------------------------ tiles

struct Pair {
  u32x4 v[2];
};
typedef __attribute__((address_space(3))) const u32x4* lds_chunk_t;
__device__ __forceinline__ u32x4 lds16(uint32_t at) { return *(lds_chunk_t)at; }
__device__ __forceinline__ float lds4(uint32_t at) {
  return *(__attribute__((address_space(3))) const float*)at;
}

// As dma16, each lane from an address of its own.
__device__ __forceinline__ void dma16_from(const void* p, uint32_t lds_byte) {
  asm volatile(
      "s_mov_b32 m0, %1\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %0, off"
      :
      : "v"(p), "s"(lds_byte)
      : "memory");
}
__device__ const u32x4 kZeros = {0, 0, 0, 0};

// s_waitcnt vmcnt(n) alone
#define WAIT_DMA(n) __builtin_amdgcn_s_waitcnt(((n) & 15) | (7 << 4) | (15 << 8) | (((n) >> 4) << 14))
#define WAIT_LDS() __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14))

// WT x WF waves, each with TT x FF blocks of 16 tokens x 16 outputs.
template <int WT_, int WF_, int TT_, int FF_, int NST_, int OCC_>
struct Tile {
  static constexpr int WT = WT_, WF = WF_, TT = TT_, FF = FF_, NST = NST_, OCC = OCC_;
  static constexpr int TM = WT * TT * 16, TN = WF * FF * 16, WAVES = WT * WF;
  static constexpr int STAGE = (TM + TN) * kFp8Group;      // bytes of a stage's operands
  static constexpr int A_DMAS = TM / 32, DMAS = (TM + TN) / 32;  // of each of four waves
  static constexpr int LDS = NST * (STAGE + TM * 4);
  static_assert(WAVES >= 4 && TM % 32 == 0 && TN % 32 == 0 && FF % 2 == 0 && LDS <= 160 * 1024, "tile");
  static_assert((DMAS + 1) * (NST - 1) <= 63, "loads in flight");
};

// `rows` rows of COLS sums that lie in LDS, out: rows from m on, outputs from n on.
template <typename Out, int KIND, int COLS>
__device__ __forceinline__ void put_rows(const Fp8Args& a, uint32_t lds, int rows, int64_t m, int n, int lane) {
  constexpr int EACH = 16 / sizeof(Out), LANES = COLS / EACH, STEP = 64 / LANES, SLOTS = COLS / 4;
  const int r0 = lane / LANES, c = lane % LANES * EACH;
  n += c;
  const int left = (int)(a.M - m < rows ? a.M - m : rows);
  if (n >= a.N) return;
  float bias[EACH], gate[EACH];
#pragma unroll
  for (int e = 0; e < EACH; ++e) {
    const int ne = n + e < a.N ? n + e : a.N - 1;
    bias[e] = a.bias ? a.bias[ne] : 0.f;
    gate[e] = KIND == ACID_EPI_GATE_RESIDUAL ? a.gate[ne] : 0.f;
  }
  for (int r = r0; r < left; r += STEP) {
    float y[EACH];
#pragma unroll
    for (int q = 0; q < EACH / 4; ++q) {
      const f32x4 v = __builtin_bit_cast(f32x4, lds16(lds + r * (COLS * 4) + ((c / 4 + q) ^ (r & 15)) % SLOTS * 16));
#pragma unroll
      for (int e = 0; e < 4; ++e) y[4 * q + e] = v[e];
    }
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      y[e] += bias[e];
      if constexpr (KIND == ACID_EPI_BIAS_GELU) y[e] = std::is_same_v<Out, bf16> ? gelu_tanh_fast(y[e]) : gelu_tanh(y[e]);
    }
    Out* dst = (Out*)a.out + (m + r) * a.out_ld + n;
    const float* old = a.residual + (m + r) * a.residual_ld + n;
    if (a.vec) {
      if constexpr (KIND == ACID_EPI_GATE_RESIDUAL) {
        const f32x4 h = *reinterpret_cast<const f32x4*>(old);
#pragma unroll
        for (int e = 0; e < EACH; ++e) y[e] = fmaf(gate[e], y[e], h[e]);
      }
      if constexpr (std::is_same_v<Out, bf16>) {
        bf16x8 b;
#pragma unroll
        for (int e = 0; e < EACH; ++e) b[e] = (bf16)y[e];
        *reinterpret_cast<bf16x8*>(dst) = b;
      } else {
        *reinterpret_cast<f32x4*>(dst) = f32x4{y[0], y[1], y[2], y[3]};
      }
    } else {
#pragma unroll
      for (int e = 0; e < EACH; ++e)
        if (n + e < a.N) {
          if constexpr (KIND == ACID_EPI_GATE_RESIDUAL) y[e] = fmaf(gate[e], y[e], old[e]);
          dst[e] = (Out)y[e];
        }
    }
  }
}

// One output tile a workgroup.  A stage is one block of 128 inputs: a TM x 128
// and a TN x 128 byte tile and the tokens' scales, loaded straight into LDS (four
// waves issue the loads) NST - 1 stages ahead.  Row r's 16-byte chunk c lies at
// slot c ^ (r / 2 % 8), so that sixteen rows of one chunk cover all 64 banks.
// Inputs past K are loaded as zeros, rows past M and N as copies of the last.
// A lane's operand of a 16 x 16 x 128 product is chunks g and g + 4 (g its row of 16
// lanes) of both tiles' rows: any order of the inputs will do, if it is the same.
template <typename Out, int KIND, bool EXACT, typename T>
__global__ __launch_bounds__(64 * T::WAVES, T::OCC) void fp8_tile_kernel(Fp8Args a) {
  constexpr int TT = T::TT, FF = T::FF, TM = T::TM, TN = T::TN, NST = T::NST, DMAS = T::DMAS;
  __shared__ __attribute__((aligned(1024))) uint8_t lds_tiles[T::LDS];
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void_t*)lds_tiles);
  const uint32_t lds_scales = lds0 + NST * T::STAGE;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wt = wave % T::WT, wf = wave / T::WT, lr = lane & 15, lg = lane >> 4;

  const int tiles_n = (a.N + TN - 1) / TN;
  const uint32_t tiles_m = (a.M + TM - 1) / TM, tiles = tiles_m * tiles_n;
  int64_t tm;
  int tn;
  tile_coords(xcd_remap(blockIdx.x, tiles), tiles_m, tiles_n, tm, tn);
  const int64_t m0 = tm * TM;
  const int n0 = tn * TN, NS = a.groups;

  // loads of a stage: DMA i of wave w < 4 takes rows 32 i + 8 w .. + 7 of the tiles
  const int chunk = ((lane & 7) ^ lg ^ (4 * (wave & 1))) * 16;
  const uint32_t row0 = 8 * wave + (lane >> 3);
  const uint32_t a_ld = (uint32_t)a.a_ld, w_ld = (uint32_t)a.K;
  const uint32_t a_last = (uint32_t)(a.M - 1 - m0 < TM ? a.M - 1 - m0 : TM - 1) * a_ld;
  const uint32_t w_last = (uint32_t)(a.N - 1 - n0 < TN ? a.N - 1 - n0 : TN - 1) * w_ld;
  const uint64_t a_base = uniform_ptr(a.a + m0 * a.a_ld), w_base = uniform_ptr(a.w + (int64_t)n0 * a.K);
  const uint32_t s_off = (uint32_t)(4 * lane < a.M - 1 - m0 ? 4 * lane : ((a.M - 1 - m0) & ~3)) * 4;
  const uint64_t s_base = uniform_ptr(a.a_scales + m0);
  const int tail = a.K % kFp8Group;  // inputs of the last block, 0: all
  auto issue = [&](int st, uint32_t buf) {
    uint32_t row_off = row0 * a_ld, w_off = row0 * w_ld;
    asm volatile("" : "+v"(row_off), "+v"(w_off));  // not the offsets of all loads, kept in registers
    const uint32_t k0 = (uint32_t)st * kFp8Group, at0 = lds0 + buf * T::STAGE + (uint32_t)wave * 1024;
    if (tail && st == NS - 1) {
      const bool in = chunk < tail;
#pragma unroll 1
      for (int i = 0; i < DMAS; ++i) {
        const bool is_a = i < T::A_DMAS;
        const uint32_t off = is_a ? min(row_off + i * 32 * a_ld, a_last) : min(w_off + (i - T::A_DMAS) * 32 * w_ld, w_last);
        const uint8_t* at = reinterpret_cast<const uint8_t*>((is_a ? a_base : w_base) + k0) + off + chunk;
        dma16_from(in ? at : reinterpret_cast<const uint8_t*>(&kZeros), at0 + i * 4096);
      }
    } else {
#pragma unroll
      for (int i = 0; i < DMAS; ++i) {
        const bool is_a = i < T::A_DMAS;
        const uint32_t off = is_a ? min(row_off + i * 32 * a_ld, a_last) : min(w_off + (i - T::A_DMAS) * 32 * w_ld, w_last);
        dma16((is_a ? a_base : w_base) + k0, off + chunk, at0 + i * 4096);
      }
    }
    if (wave == 0 && lane < TM / 4)
      dma16(s_base + (uint64_t)st * a.a_scales_ld * 4, s_off, lds_scales + buf * (TM * 4));
  };
  // all but the `stages` youngest stages of this wave's loads have landed
  auto landed = [&](auto stages) {
    constexpr int S = decltype(stages)::value;
    if (wave == 0) WAIT_DMA((DMAS + 1) * S);
    else WAIT_DMA(DMAS * S);
  };

  // the outputs' scales, one stage a lane, 64 stages at a time
  const int nb = min(n0 + wf * (FF * 16), a.N - 1) / kFp8Group;
  const float* sw_at = a.w_scales + (int64_t)nb * a.groups;
  float sw = sw_at[min(lane, NS - 1)];

  const uint32_t swz = (uint32_t)((lg ^ (lr >> 1)) * 16);
  const uint32_t a_at = lds0 + (uint32_t)(wt * TT * 16 + lr) * kFp8Group + swz;
  const uint32_t w_at = lds0 + (uint32_t)(TM + wf * FF * 16 + lr) * kFp8Group + swz;
  const uint32_t s_at = lds_scales + (uint32_t)(wt * TT * 16 + lr) * 4;
  auto read = [&](uint32_t at, int block) {
    return Pair{{lds16(at + block * 2048), lds16((at ^ 64) + block * 2048)}};
  };

  f32x4 acc[FF][TT], part[TT];
  Pair fa[TT], fw[2];
  float s_old[TT], s_now[TT], s_next[TT];
  auto main_loop = [&](auto issues) {
  constexpr bool DMA = decltype(issues)::value;
  if constexpr (DMA) {
#pragma unroll
    for (int st = 0; st < NST; ++st)
      if (st < NS) issue(st, st);
    if (NS >= NST) landed(std::integral_constant<int, NST - 1>{});
    else WAIT_DMA(0);
  }
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
#pragma unroll
  for (int t = 0; t < TT; ++t) {
#pragma unroll
    for (int f = 0; f < FF; ++f) acc[f][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    part[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    fa[t] = read(a_at, t);
    s_old[t] = 0.f;
    s_now[t] = 0.f;
    s_next[t] = lds4(s_at + t * 64);
  }
  fw[0] = read(w_at, 0);

  uint32_t buf = 0, nxt = NST == 1 ? 0 : 1;
  for (int st = 0; st < NS; ++st) {
    if (st && st % 64 == 0) sw = sw_at[min(st + lane, NS - 1)];
    const float sw_now = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(sw), st % 64));
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      s_old[t] = s_now[t];
      s_now[t] = s_next[t] * sw_now;
    }
    const uint32_t cur_off = buf * T::STAGE, nxt_off = nxt * T::STAGE;
#pragma unroll
    for (int f = 0; f < FF; ++f) {
      if (f + 1 < FF) {
        fw[(f + 1) & 1] = read(w_at + cur_off, f + 1);
      } else {
        WAIT_LDS();  // the stage's last operands have arrived
        if constexpr (DMA) {
          if (st + NST - 1 < NS) landed(std::integral_constant<int, NST - 2>{});
          else WAIT_DMA(0);
        }
        __builtin_amdgcn_s_barrier();  // the next stage has landed, and this one's tiles are free
        asm volatile("" ::: "memory");
        fw[0] = read(w_at + nxt_off, 0);  // past the last stage: read and dropped
#pragma unroll
        for (int t = 0; t < TT; ++t) s_next[t] = lds4(s_at + nxt * (TM * 4) + t * 64);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        const int pf = (f + FF - 1) % FF;
#pragma unroll
        for (int r = 0; r < 4; ++r)
          acc[pf][t][r] = fmaf(f == 0 ? s_old[t] : s_now[t], part[t][r], acc[pf][t][r]);
        asm volatile("" : "+v"(acc[pf][t]));  // here, not where the loop ends
        if constexpr (EXACT) {
          f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            bf16x8 bw[2], ba[2];
            to_bf16(fw[f & 1].v[j], bw);
            to_bf16(fa[t].v[j], ba);
#pragma unroll
            for (int i = 0; i < 2; ++i)
              sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bw[i], ba[i], sum, 0, 0, 0);
          }
          part[t] = sum;
        } else {
          part[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
              __builtin_bit_cast(i32x8, fw[f & 1]), __builtin_bit_cast(i32x8, fa[t]),
              f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
        }
        if (f + 1 == FF) fa[t] = read(a_at + nxt_off, t);
        __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (DMA)
        if (f + 1 == FF && st + NST < NS) issue(st + NST, buf);
    }
    buf = nxt;
    nxt = nxt + 1 == NST ? 0 : nxt + 1;
  }
  };
  if (wave < 4) main_loop(std::true_type{});
  else main_loop(std::false_type{});
#pragma unroll
  for (int t = 0; t < TT; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) acc[FF - 1][t][r] = fmaf(s_now[t], part[t][r], acc[FF - 1][t][r]);

  // Out by way of LDS, whole rows of the wave's outputs at a time: two blocks of tokens in
  // a part of LDS that is this wave's alone (every load has landed, and what waves still
  // read past the last stage is dropped).  The 16-byte slot s of token i is at s ^ i % 16.
  constexpr int COLS = FF * 16, SLOTS = COLS / 4, PER = TT < 2 ? 1 : 2;
  static_assert(T::WAVES * PER * 16 * COLS * 4 <= T::LDS && TT % PER == 0, "outputs by way of LDS");
  const uint32_t mine = lds0 + (uint32_t)wave * (PER * 16 * COLS * 4);
  const int nw = n0 + wf * COLS;
#pragma unroll
  for (int t = 0; t < TT; t += PER) {
#pragma unroll
    for (int p = 0; p < PER; ++p)
#pragma unroll
      for (int f = 0; f < FF; ++f)
        *(__attribute__((address_space(3))) f32x4*)(mine + (p * 16 + lr) * (COLS * 4) + ((4 * f + lg) ^ lr) % SLOTS * 16) = acc[f][t + p];
    asm volatile("" ::: "memory");
    WAIT_LDS();
    put_rows<Out, KIND, COLS>(a, mine, PER * 16, m0 + (wt * TT + t) * 16, nw, lane);
    WAIT_LDS();
    asm volatile("" ::: "memory");
  }
}

template <typename Out, int KIND, bool EXACT, typename T>
hipError_t launch_tile(const Fp8Args& a, hipStream_t s) {
  const int64_t tiles = ((int64_t)a.M + T::TM - 1) / T::TM * ((a.N + T::TN - 1) / T::TN);
  hipLaunchKernelGGL((fp8_tile_kernel<Out, KIND, EXACT, T>), dim3((unsigned)tiles), dim3(64 * T::WAVES), 0, s, a);
  return hipGetLastError();
}

template <typename Out, int KIND, bool EXACT>
hipError_t launch(const Fp8Args& a, hipStream_t s) {
  if constexpr (EXACT)
    return launch_tile<Out, KIND, EXACT, Tile<4, 2, 4, 4, 2, 1>>(a, s);
  else
    return launch_tile<Out, KIND, EXACT, Tile<4, 2, 4, 8, 2, 1>>(a, s);
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
  if ((M + 63) / 64 * ((N + 63) / 64) >= (1 << 23))
    return set_error(ACID_ERR_SHAPE, "fp8: ceil(M / 64) * ceil(N / 64) must be below 2^23");
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
  const bool vec = N * os % 16 == 0 && p.out_ld * os % 16 == 0 && (uintptr_t)p.out % 16 == 0 &&
                   (!update || (p.residual_ld % 4 == 0 && (uintptr_t)p.residual % 16 == 0));
  const Fp8Args a = {(const uint8_t*)p.a, (const uint8_t*)p.w, p.a_scales, p.w_scales, p.bias, p.gate,
                     p.residual, p.out, p.a_ld, p.a_scales_ld, p.residual_ld, p.out_ld, (int32_t)M, N,
                     K, (int32_t)groups, p.kind, vec};
  hipError_t e;
  if (p.out_dtype == ACID_BF16)
    e = p.kind == ACID_EPI_BIAS ? launch<bf16, ACID_EPI_BIAS, false>(a, stream)
                                : launch<bf16, ACID_EPI_BIAS_GELU, false>(a, stream);
  else
    e = update                      ? launch<float, ACID_EPI_GATE_RESIDUAL, false>(a, stream)
        : p.kind == ACID_EPI_BIAS ? launch<float, ACID_EPI_BIAS, true>(a, stream)
                                  : launch<float, ACID_EPI_BIAS_GELU, true>(a, stream);
  return e == hipSuccess ? ACID_OK : check_hip(e, "linear fp8");
}

}  // extern "C"
