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
// products at a time, aligned to the largest of them, and drop towards zero what lies below
// 2^-13 of it (measured; both the 32x32x64 and the older 32x32x16 do): 7 2^-13 of the
// largest product at most.  Random operands give sums that are 1.4e-5 off, to no side;
// operands of one sign, sums 2.5e-6 too small.  The rounding to bf16 that may follow is 2^-9, and
// the operands' own are some 2^-5.  Outputs in bf16, and updates of a residual, take them.
// Plain fp32 outputs, and with ACID_FP8_EXACT all, take the bf16 instruction on operands
// converted on the way, which is exact: products and sums in fp32, in up to twice the time
// (us, 32760 x 1536 x 8960: bf16 759 for 368, fp32 776, onto a residual 826 for 447; x 1536 x
// 1536 onto a residual 180 for 130; 64 x 1536 x 8960 15.0 for 12.9).  An update of a residual
// costs more so than by acid_linear on operands of 16 bits (660 us), so exact ones are for
// who asks for them: they keep small products beside an outlier, or beside two that cancel.
//
// Microseconds on one MI355X, 8-bit products to bf16 (a register-only stream of the
// instruction makes 3.8 PFLOP/s, the library's product without block scales 2.4 to 3.3); the
// last line in a graph, the others calls in a row:
//   32760 x 4608 x 1536   227 (2.04 PFLOP/s)     8192 x 8192 x 8192  426 (2.58)
//   32760 x 1536 x 8960   367 (2.46); onto a residual in fp32 445
//   64 x 1536 x 8960  12.7   1 x 8960 x 1536  4.7    1 x 28672 x 8192  38.8 (6.1 TB/s)
// What bounds the large ones is cycles around the products.  At 32760 x 1536 x 8960 the matrix
// units are busy 61% of 5.7 M active cycles, the library's 81% of 4.25 M; our waves wait 26%
// of theirs, the library's 8%, with 11.3 M instructions of LDS for 6.9 M and 77 M of the
// vector units for 18 M (32760 x 4608 x 1536: 48% for 55%, and with a residual 47% of 7.4 M).  The clock is
// the power's, 1.6 to 1.9 GHz for both.  Parts left out for a timing took their time with
// them: loads of operands 15%, reads of LDS 20%, the scales' multiply-adds 8%, barriers 3%,
// the outputs 6%; leaving out the waits, wave priorities and other orders of the loads change
// nothing.  By the two bf16 times a stage is 1.67 us and a tile 5 more.  Four waves of 128 x 128 each
// would read a third less of LDS; that form has not been measured.

#include <algorithm>
#include <type_traits>

#include "fp8.h"
#include "fp8_form.h"
#include "tiles.h"

namespace acid {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

struct Fp8Args {
  const uint8_t *a, *w;
  const float *a_scales, *w_scales, *bias, *gate, *residual;
  void* out;
  int64_t a_ld, a_scales_ld, residual_ld, out_ld;
  float* partial;  // sums of parts of K, for fp8_reduce_kernel
  int32_t M, N, K, groups, split;
  bool whole;  // whole blocks of inputs, 16 bytes of outputs (and residual) at once
  bool wide;   // four outputs at once
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
// The same with four bytes a lane.
__device__ __forceinline__ void dma4_from(const void* p, uint32_t lds_byte) {
  asm volatile(
      "s_mov_b32 m0, %1\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dword %0, off"
      :
      : "v"(p), "s"(lds_byte)
      : "memory");
}
__device__ const u32x4 kZeros = {0, 0, 0, 0};

// s_waitcnt vmcnt(n) alone, and lgkmcnt(0) alone
#define WAIT_DMA(n) __builtin_amdgcn_s_waitcnt(((n) & 15) | (7 << 4) | (15 << 8) | (((n) >> 4) << 14))
#define WAIT_LDS() __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14))

constexpr int PARTIAL = -1;  // in the place of an epilogue: raw sums into a.partial

template <int N>
using I = std::integral_constant<int, N>;
template <int N, typename F>
__device__ __forceinline__ void each(F f) {  // f(I<0>), ..
  if constexpr (N > 0) {
    each<N - 1>(f);
    f(I<N - 1>{});
  }
}

// WT x WF waves, each with TT x FF blocks of 16 tokens x 16 outputs; OCC workgroups
// a CU.
template <int WT_, int WF_, int TT_, int FF_, int OCC_>
struct Tile {
  static constexpr int WT = WT_, WF = WF_, TT = TT_, FF = FF_, OCC = OCC_;
  static constexpr int TM = WT * TT * 16, TN = WF * FF * 16, WAVES = WT * WF;
  static constexpr int STAGE = (TM + TN) * kFp8Group;  // bytes of a stage's operands
  static constexpr int LDS = 2 * (STAGE + TM * 4) + WAVES * FF * 16 * 8;  // .. and bias and gate
  // A load fills 8 rows of 128 bytes.  A stage's part 0: the tokens, the first half of
  // each wave's outputs, the tokens' scales (one load of wave 0); part 1: the second
  // halves.  Loads of a wave:
  static constexpr int LOADS_A = TM / 8 / WAVES, LOADS_W = TN / 16 / WAVES, LOADS0 = LOADS_A + LOADS_W;
  // The eight rows of the outputs' tile that load i of wave w takes of its part's half are
  // 8 (rows_of(i) + rows_of_wave(w)) .. in part 0, FF of them further in part 1.
  static constexpr int rows_of(int i) { return WAVES >= FF ? i * (WAVES / FF) * 2 * FF : i / (FF / WAVES) * 2 * FF + i % (FF / WAVES) * WAVES; }
  static __device__ int rows_of_wave(int w) { return WAVES >= FF ? w / FF * 2 * FF + w % FF : w; }
  static_assert(WAVES % 4 == 0 && (WAVES % FF == 0 || FF % WAVES == 0) && FF % 4 == 0, "tile");
  static_assert(TM % (8 * WAVES) == 0 && TN % (16 * WAVES) == 0 && TM <= 256, "loads");
  static_assert(LDS * OCC <= 160 * 1024 && WAVES * OCC <= 32, "workgroups a CU");
};

// Outputs of one tile, a wave's blocks of 16 tokens x 16 outputs out of its sums: lane l has
// outputs 4 (l / 16) .. + 3 of token l % 16.
// Whole 16 bytes: fp32 as they are; two bf16 blocks side by side exchange halves between
// neighbouring rows of 16 lanes, so that each lane has eight outputs of one of them.
// Streaming stores: ordinary ones push the operands out of L2 (with groups of four token
// tiles for two, 32760 x 4608 x 1536 256 -> 232 us).
template <typename Out, int KIND, bool GENERAL, int TT, int FF>
__device__ __forceinline__ void put_tile(const Fp8Args& a, f32x4 (&acc)[FF][TT], int64_t m0, int n0,
                                         uint32_t columns, int lane) {
  asm volatile("" : "+v"(lane));  // nothing of this is kept in registers through the stages
  const int lr = lane & 15, lg = lane >> 4;
  auto column = [&](int which, int f) {  // bias (0) or gate (1) of this lane's four outputs
    return __builtin_bit_cast(f32x4, lds16(columns + (which * FF + f) * 64 + lg * 16));
  };
  auto finish = [&](f32x4 y, const f32x4& bias, const f32x4& gate, const f32x4& old) {
    y += bias;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      if constexpr (KIND == ACID_EPI_BIAS_GELU) y[r] = std::is_same_v<Out, bf16> ? gelu_tanh_fast(y[r]) : gelu_tanh(y[r]);
      if constexpr (KIND == ACID_EPI_GATE_RESIDUAL) y[r] = fmaf(gate[r], y[r], old[r]);
    }
    return y;
  };
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  if constexpr (GENERAL) {
#pragma unroll
    for (int f = 0; f < FF; ++f) {
      const f32x4 bias = column(0, f), gate = KIND == ACID_EPI_GATE_RESIDUAL ? column(1, f) : zero;
      const int n = n0 + f * 16 + 4 * lg;
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        const int64_t m = m0 + t * 16 + lr;
        f32x4 old = zero;
        if constexpr (KIND == ACID_EPI_GATE_RESIDUAL) {
          const float* at = a.residual + (m < a.M ? m : a.M - 1) * a.residual_ld;
#pragma unroll
          for (int r = 0; r < 4; ++r) old[r] = at[n + r < a.N ? n + r : a.N - 1];
        }
        const f32x4 y = finish(acc[f][t], bias, gate, old);
        Out* out = (Out*)a.out + m * a.out_ld + n;
        if (a.wide) {
          if (m < a.M && n < a.N) {
            if constexpr (std::is_same_v<Out, bf16>)
              *reinterpret_cast<bf16x4*>(out) = bf16x4{(bf16)y[0], (bf16)y[1], (bf16)y[2], (bf16)y[3]};
            else
              *reinterpret_cast<f32x4*>(out) = y;
          }
        } else if (m < a.M) {
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (n + r < a.N) out[r] = (Out)y[r];
        }
      }
    }
  } else if constexpr (std::is_same_v<Out, bf16>) {
    const int64_t at = (int64_t)lr * a.out_ld + (lg & 1) * 16 + (lg & 2) * 4;
    bf16* out = (bf16*)a.out + m0 * a.out_ld + n0 + at;
    const int left_m = (int)(a.M - m0 < TT * 16 ? a.M - m0 : TT * 16) - lr, left_n = a.N - n0 - (int)((lg & 1) * 16 + (lg & 2) * 4);
#pragma unroll
    for (int f = 0; f < FF; f += 2) {
      __builtin_amdgcn_sched_barrier(0);  // (not all of the tile's bias at once)
      const f32x4 bias[2] = {column(0, f), column(0, f + 1)};
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        uint32_t w[2][2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const f32x4 y = finish(acc[f + i][t], bias[i], zero, zero);
#pragma unroll
          for (int r = 0; r < 2; ++r) w[i][r] = __builtin_bit_cast(uint32_t, bf16x2{(bf16)y[2 * r], (bf16)y[2 * r + 1]});
        }
        const auto lo = __builtin_amdgcn_permlane16_swap(w[0][0], w[1][0], false, false);
        const auto hi = __builtin_amdgcn_permlane16_swap(w[0][1], w[1][1], false, false);
        if (t * 16 < left_m && f * 16 < left_n)
          __builtin_nontemporal_store(u32x4{lo[0], hi[0], lo[1], hi[1]},
                                      reinterpret_cast<u32x4*>(out + (int64_t)(t * 16) * a.out_ld + f * 16));
      }
    }
  } else {
    const int left_m = (int)(a.M - m0 < TT * 16 ? a.M - m0 : TT * 16) - lr, left_n = a.N - n0 - 4 * lg;
    float* out = (float*)a.out + (m0 + lr) * a.out_ld + n0 + 4 * lg;
    // the residual's values, AHEAD blocks ahead
    constexpr int AHEAD = KIND == ACID_EPI_GATE_RESIDUAL ? 10 : 1, BLOCKS = FF * TT;
    f32x4 old[AHEAD];
    auto read_old = [&](int i) {
      old[i % AHEAD] = zero;
      if constexpr (KIND == ACID_EPI_GATE_RESIDUAL) {
        const int f = i / TT, t = i % TT;
        const int64_t m = m0 + lr + (t * 16 < left_m ? t * 16 : left_m - 1);
        const int n = f * 16 < left_n ? n0 + 4 * lg + f * 16 : a.N - 4;
        if (left_m > 0) old[i % AHEAD] = *reinterpret_cast<const f32x4*>(a.residual + m * a.residual_ld + n);
      }
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) read_old(i);
    f32x4 bias, gate;
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i) {
      const int f = i / TT, t = i % TT;
      if (t == 0) {
        bias = column(0, f);
        gate = KIND == ACID_EPI_GATE_RESIDUAL ? column(1, f) : zero;
      }
      const f32x4 y = finish(acc[f][t], bias, gate, old[i % AHEAD]);
      if (i + AHEAD < BLOCKS) read_old(i + AHEAD);
      if (t * 16 < left_m && f * 16 < left_n)
        __builtin_nontemporal_store(y, reinterpret_cast<f32x4*>(out + (int64_t)(t * 16) * a.out_ld + f * 16));
    }
  }
}

// Output tiles, a workgroup's one after the other, or with PARTIAL parts of K of
// them; their stages form one stream.  A
// stage is one block of 128 inputs: a TM x 128 and a TN x 128 byte tile and the tokens'
// scales, loaded straight into one of two buffers in LDS.  Two barriers a stage: each frees
// what all waves have read, a half of its buffer (part 0, then part 1), which is then
// filled for the stage after the next, one load at a time between the products; so
// loads run one and a half stages ahead, into the next tile.  (32760 x 1536 x 8960, by one
// wave of each SIMD: one barrier a stage and loads at once behind it 451 us, two barriers 397,
// spread 391; by all waves, spread, from tile to tile 380.)
// Row r's 16-byte chunk c lies at slot c ^ (r / 2 % 8), so that sixteen rows of one
// chunk cover all 64 banks.  Rows past M and N are copies of the last.  A lane's operand of
// a 16 x 16 x 128 product is chunks g and g + 4 (g its row of 16 lanes) of both tiles'
// rows: any order of the inputs will do, if it is the same.
// GENERAL: K that is no whole blocks, or outputs that are no whole 16 bytes.  The
// short block comes first, its missing inputs loaded as zeros.
template <typename Out, int KIND, bool EXACT, bool GENERAL, typename T>
__global__ __launch_bounds__(64 * T::WAVES, T::OCC * T::WAVES / 4) void fp8_tile_kernel(Fp8Args a) {
  constexpr int TT = T::TT, FF = T::FF, TM = T::TM, TN = T::TN, HALF = FF / 2 * TT;
  __shared__ __attribute__((aligned(1024))) uint8_t lds_tiles[T::LDS];
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void_t*)lds_tiles);
  const uint32_t lds_scales = lds0 + 2 * T::STAGE;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wt = wave % T::WT, wf = wave / T::WT, lr = lane & 15, lg = lane >> 4;
  const uint32_t columns = lds_scales + 2 * TM * 4 + (uint32_t)wave * (FF * 128);  // bias, gate
  const int NS = a.groups, tiles_n = (a.N + TN - 1) / TN;
  const uint32_t tiles_m = (a.M + TM - 1) / TM, tiles = tiles_m * tiles_n, items = tiles * a.split;
  // A work item: tile (tm, tn), the blocks from `first` to before `end` of its order, where
  // a short block is the first.  Parts outermost, so that neighbours share operands.
  struct Item {
    uint32_t index;
    int64_t tm;
    int tn, first, end;
  };
  auto item_at = [&](uint32_t i) {
    Item r;
    r.index = xcd_remap(i < items ? i : blockIdx.x, items);
    const uint32_t part = KIND == PARTIAL ? r.index / tiles : 0;
    tile_coords<4>(r.index - part * tiles, tiles_m, tiles_n, r.tm, r.tn);
    r.first = KIND == PARTIAL ? (int)((int64_t)NS * part / a.split) : 0;
    r.end = KIND == PARTIAL ? (int)((int64_t)NS * (part + 1) / a.split) : NS;
    return r;
  };
  const int tail = GENERAL ? a.K % kFp8Group : 0;  // inputs of the short block, 0: none

  // ---- loads.  Where the next stage to be loaded lies:
  const int chunk = ((lane & 7) ^ lg ^ (4 * (wave & 1))) * 16;
  const uint32_t a_ld = (uint32_t)a.a_ld, w_ld = (uint32_t)a.K;
  const uint32_t a_row = (uint32_t)(8 * wave + (lane >> 3)) * a_ld;
  const uint32_t w_row = (uint32_t)(8 * T::rows_of_wave(wave) + (lane >> 3)) * w_ld;
  uint32_t a_off[T::LOADS_A], w_off[2][T::LOADS_W], s_off;  // of its tile's rows
  uint64_t a_from, w_from, s_from;  // its block
  const float* sw_from;             // its scale of this wave's outputs
  uint32_t next_item = blockIdx.x;
  int next_block, next_end;         // of that item's order
  auto enter_item = [&]() {
    const Item it = item_at(next_item);
    const int64_t m0 = it.tm * TM;
    const int n0 = it.tn * TN;
    const uint32_t a_last = (uint32_t)(a.M - 1 - m0 < TM ? a.M - 1 - m0 : TM - 1) * a_ld;
    const uint32_t w_last = (uint32_t)(a.N - 1 - n0 < TN ? a.N - 1 - n0 : TN - 1) * w_ld;
    each<T::LOADS_A>([&](auto i) { a_off[i()] = min(a_row + i() * 8 * T::WAVES * a_ld, a_last) + chunk; });
    each<T::LOADS_W>([&](auto i) {
      w_off[0][i()] = min(w_row + 8 * T::rows_of(i()) * w_ld, w_last) + chunk;
      w_off[1][i()] = min(w_row + 8 * (T::rows_of(i()) + FF) * w_ld, w_last) + chunk;
    });
    s_off = (uint32_t)(4 * lane < a.M - 1 - m0 ? 4 * lane : ((a.M - 1 - m0) & ~3)) * 4;
    next_block = it.first;
    next_end = it.end;
    const int first = !tail ? it.first : it.first ? it.first - 1 : NS - 1;
    a_from = uniform_ptr(a.a + m0 * a.a_ld) + (uint32_t)first * kFp8Group;
    w_from = uniform_ptr(a.w + (int64_t)n0 * a.K) + (uint32_t)first * kFp8Group;
    s_from = uniform_ptr(a.a_scales + m0) + (uint64_t)first * a.a_scales_ld * 4;
    sw_from = a.w_scales + (int64_t)(min(n0 + wf * (FF * 16), a.N - 1) / kFp8Group) * NS + first;
  };
  auto leave_stage = [&]() {  // all loads of a stage have been issued
    if (++next_block == next_end) {
      next_item += gridDim.x;
      enter_item();
      return;
    }
    if (tail && next_block == 1) {  // from the short block to the first
      a_from -= (uint32_t)(NS - 1) * kFp8Group;
      w_from -= (uint32_t)(NS - 1) * kFp8Group;
      s_from -= (uint64_t)(NS - 1) * a.a_scales_ld * 4;
      sw_from -= NS - 1;
    } else {
      a_from += kFp8Group;
      w_from += kFp8Group;
      s_from += (uint64_t)a.a_scales_ld * 4;
      sw_from += 1;
    }
  };
  auto copy = [&](uint64_t from, uint32_t off, uint32_t at) {
    if (GENERAL && tail && next_block == 0)
      dma16_from(chunk < tail ? reinterpret_cast<const uint8_t*>(from) + off : reinterpret_cast<const uint8_t*>(&kZeros), at);
    else
      dma16(from, off, at);
  };
  auto load = [&](auto part, auto index, uint32_t buf) {
    constexpr int PART = decltype(part)::value, i = decltype(index)::value;
    const uint32_t to = lds0 + buf * T::STAGE;
    if constexpr (PART == 0 && i < T::LOADS_A) {
      copy(a_from, a_off[i], to + (uint32_t)(i * T::WAVES + wave) * 1024);
    } else if constexpr (PART == 0 && i == T::LOADS0) {
      if (wave == 0 && lane < TM / 4) dma16(s_from, s_off, lds_scales + buf * (TM * 4));
    } else {
      constexpr int j = PART ? i : i - T::LOADS_A, rows = T::rows_of(j) + PART * FF;
      copy(w_from, w_off[PART][j], to + TM * kFp8Group + (uint32_t)(rows + T::rows_of_wave(wave)) * 1024);
    }
  };
  // a part's loads whose turn is slot S of SLOTS
  auto issue = [&](auto part, auto slot, auto slots, uint32_t buf) {
    constexpr int PART = decltype(part)::value, S = decltype(slot)::value, N = decltype(slots)::value;
    constexpr int LOADS = PART ? T::LOADS_W : T::LOADS0 + 1;
    each<LOADS>([&](auto index) {
      if constexpr (decltype(index)::value * N / LOADS == S) load(part, index, buf);
    });
  };
  // All but this wave's youngest loads, of so many parts 0 and 1, have landed.  (What else is in
  // flight, outputs of the last tile, makes the wait longer.)
  auto landed = [&](auto parts0, auto parts1) {
    constexpr int N0 = decltype(parts0)::value, N = T::LOADS0 * N0 + T::LOADS_W * decltype(parts1)::value;
    static_assert(N + N0 <= 63, "loads in flight");
    if (wave == 0) WAIT_DMA(N + N0);
    else WAIT_DMA(N);
  };

  // ---- operands
  const uint32_t swz = (uint32_t)((lg ^ (lr >> 1)) * 16);
  const uint32_t a_at = lds0 + (uint32_t)(wt * TT * 16 + lr) * kFp8Group + swz;
  const uint32_t w_at = lds0 + (uint32_t)(TM + wf * FF * 16 + lr) * kFp8Group + swz;
  const uint32_t s_at = lds_scales + (uint32_t)(wt * TT * 16 + lr) * 4;
  auto read = [&](uint32_t at, int block) {
    return Pair{{lds16(at + block * 2048), lds16((at ^ 64) + block * 2048)}};
  };
  f32x4 acc[FF][TT], part[TT];
  Pair fa[TT], fw[2];
  float s_now[TT], s_next[TT];

  // by way of the scalar cache: nothing that the loads in flight would be waited for
  auto outputs_scale = [&]() {
    return *(__attribute__((address_space(4))) const float*)uniform_ptr(sw_from);
  };
  enter_item();
  float sw_next = outputs_scale();
  issue(I<0>{}, I<0>{}, I<1>{}, 0);
  issue(I<1>{}, I<0>{}, I<1>{}, 0);
  leave_stage();
  issue(I<0>{}, I<0>{}, I<1>{}, 1);
  each<TT>([&](auto slot) { issue(I<1>{}, slot, I<HALF>{}, 1); });  // the rest: within the first stage
  auto first_operands = [&](uint32_t buf) {
    fw[0] = read(w_at + buf * T::STAGE, 0);
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      fa[t] = read(a_at + buf * T::STAGE, t);
      s_next[t] = lds4(s_at + buf * (TM * 4) + t * 64);
    }
  };
  landed(I<1>{}, I<1>{});  // part 0 of the first stage
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  first_operands(0);

  uint32_t buf = 0;
  for (uint32_t i = blockIdx.x; i < items; i += gridDim.x) {
    const Item it = item_at(i);
    const int64_t mw = it.tm * TM + wt * TT * 16;
    const int nw = it.tn * TN + wf * FF * 16;
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      s_now[t] = 0.f;  // what is left in `part` belongs to the last tile
#pragma unroll
      for (int f = 0; f < FF; ++f) acc[f][t] = f32x4{0.f, 0.f, 0.f, 0.f};
      part[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // bias and gate of the wave's outputs, for when the stages are done
    if constexpr (KIND != PARTIAL) {
      auto lay = [&](const float* v, uint32_t at) {
        if constexpr (GENERAL) {
#pragma unroll
          for (int j = 0; j < FF * 16; j += 64)
            dma4_from(v ? v + min(nw + j + lane, a.N - 1) : reinterpret_cast<const float*>(&kZeros), at + j * 4);
        } else if (lane < FF * 4) {
          dma16_from(v ? (const void*)(v + min(nw + 4 * lane, a.N - 4)) : &kZeros, at);
        }
      };
      lay(a.bias, columns);
      if constexpr (KIND == ACID_EPI_GATE_RESIDUAL) lay(a.gate, columns + FF * 64);
    }
    for (int st = it.first; st < it.end; ++st) {
      const uint32_t nxt = buf ^ 1, cur_off = buf * T::STAGE, nxt_off = nxt * T::STAGE;
      each<FF>([&](auto f_) {
        constexpr int f = decltype(f_)::value;
        if constexpr (f == 1) {  // (the sums that are added in f == 0 are the last stage's)
#pragma unroll
          for (int t = 0; t < TT; ++t) s_now[t] = s_next[t] * sw_next;
        }
        if constexpr (f + 1 == FF / 2) {
          sw_next = outputs_scale();
          leave_stage();
          WAIT_LDS();                   // this half's last operands have arrived
          landed(I<1>{}, I<1>{});       // part 1 of this stage: the next one's are younger
          __builtin_amdgcn_s_barrier();  // for all waves; part 0 of this buffer is free
          asm volatile("" ::: "memory");
        }
        if constexpr (f + 1 < FF) {
          fw[(f + 1) & 1] = read(w_at + cur_off, f + 1);
        } else {
          WAIT_LDS();
          landed(I<1>{}, I<1>{});       // part 0 of the next stage: its part 1 and part 0 of the one after are younger
          __builtin_amdgcn_s_barrier();  // part 1 of this buffer is free
          asm volatile("" ::: "memory");
          fw[0] = read(w_at + nxt_off, 0);
#pragma unroll
          for (int t = 0; t < TT; ++t) s_next[t] = lds4(s_at + nxt * (TM * 4) + t * 64);
        }
        __builtin_amdgcn_sched_barrier(0);
        each<TT>([&](auto t_) {
          constexpr int t = decltype(t_)::value, pf = (f + FF - 1) % FF;
#pragma unroll
          for (int r = 0; r < 4; ++r)
            acc[pf][t][r] = fmaf(s_now[t], part[t][r], acc[pf][t][r]);
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
          if constexpr (f + 1 == FF) fa[t] = read(a_at + nxt_off, t);
          if constexpr (f + 1 >= FF / 2 && f + 1 < FF)
            issue(I<0>{}, I<(f + 1 - FF / 2) * TT + t>{}, I<HALF>{}, buf);
          else if constexpr (f + 1 == FF)
            issue(I<1>{}, I<t>{}, I<HALF>{}, buf);
          else
            issue(I<1>{}, I<(f + 1) * TT + t>{}, I<HALF>{}, nxt);
          __builtin_amdgcn_sched_barrier(0);
        });
      });
      buf = nxt;
    }
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[FF - 1][t][r] = fmaf(s_now[t], part[t][r], acc[FF - 1][t][r]);
    if constexpr (KIND == PARTIAL) {
      f32x4* to = reinterpret_cast<f32x4*>(a.partial) + (int64_t)it.index * (TM * TN / 4) + tid;
#pragma unroll
      for (int f = 0; f < FF; ++f)
#pragma unroll
        for (int t = 0; t < TT; ++t) to[(f * TT + t) * (64 * T::WAVES)] = acc[f][t];
    } else {
      WAIT_DMA(T::LOADS0);  // bias and gate: this many loads were issued after them
      asm volatile("" ::: "memory");
      put_tile<Out, KIND, GENERAL, TT, FF>(a, acc, mw, nw, columns, lane);
      WAIT_LDS();  // bias and gate have been read
      asm volatile("" ::: "memory");
    }
    first_operands(buf);  // again: their registers held what is above
  }
  WAIT_DMA(0);  // the loads past the last stage land before the LDS is another workgroup's
}

// --------------------------------------------------------------- few rows

// A value of the output from its sum.
template <typename Out, int KIND>
__device__ __forceinline__ void put_one(const Fp8Args& a, float y, int64_t m, int n) {
  if (a.bias) y += a.bias[n];
  if constexpr (KIND == ACID_EPI_BIAS_GELU) y = std::is_same_v<Out, bf16> ? gelu_tanh_fast(y) : gelu_tanh(y);
  if constexpr (KIND == ACID_EPI_GATE_RESIDUAL) y = fmaf(a.gate[n], y, a.residual[m * a.residual_ld + n]);
  ((Out*)a.out)[m * a.out_ld + n] = (Out)y;
}

// Up to 32 rows, bound by reading the weights once.  A workgroup has 16 outputs; its WAVES
// waves take the blocks of inputs in turn, and their sums are added in wave order.  A wave's
// operands go by way of a part of LDS that is its own: whole lines, DEEP blocks ahead,
// laid out as the tiles' above (each lane's own 16 bytes straight into registers: 1 x 8960 x
// 1536 7.2 us for 4.7, 1 x 28672 x 8192 53 for 39, 16 rows of it 71 for 46).  Eight waves and
// two blocks ahead are best or within 11% from 4608 x 1536 to 28672 x 8192; four waves lose 25%
// where the inputs are long (1536 x 8960 6.2 us for 5.0), sixteen where they are short (5.1
// for 3.9).  X: eights of rows (LDS for one workgroup a CU with four, two with fewer).
template <typename Out, int KIND, bool EXACT, int WAVES, int DEEP, int X>
__global__ __launch_bounds__(64 * WAVES) void fp8_rows_kernel(Fp8Args a) {
  constexpr int BLOCK = 2048 + X * 1024 + 128, LOADS = 2 + X + 1, TT = (X + 1) / 2;
  __shared__ __attribute__((aligned(1024))) uint8_t ring[WAVES * DEEP * BLOCK];
  static_assert(sizeof(ring) >= WAVES * TT * 1024 && TT * 64 <= 128 && sizeof(ring) <= 160 * 1024 && LOADS * (DEEP - 1) <= 63, "ring");
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lr = lane & 15, lg = lane >> 4;
  const int n0 = blockIdx.x * 16, tail = a.K % kFp8Group;
  const uint32_t mine = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void_t*)ring) + wave * (DEEP * BLOCK);
  const int row = lane >> 3, chunk = ((lane & 7) ^ lg) * 16;
  const uint8_t* from[2 + X];  // rows `row` of the eights, outputs first
#pragma unroll
  for (int i = 0; i < 2; ++i) from[i] = a.w + (int64_t)std::min(n0 + 8 * i + row, a.N - 1) * a.K;
#pragma unroll
  for (int i = 0; i < X; ++i) from[2 + i] = a.a + (int64_t)std::min(8 * i + row, a.M - 1) * a.a_ld;
  const float* sw = a.w_scales + (int64_t)(n0 / kFp8Group) * a.groups;
  const float* sx = a.a_scales + std::min(4 * (lane & (4 * TT - 1)), (a.M - 1) & ~3);
  auto load = [&](int b, uint32_t at) {
#pragma unroll
    for (int i = 0; i < 2 + X; ++i) {
      const int k = chunk ^ (64 * (i & 1));  // rows 8 i ..: chunk c at slot c ^ (4 i + row / 2) % 8
      const bool in = !tail || b + 1 < a.groups || k < tail;
      dma16_from(in ? from[i] + (int64_t)b * kFp8Group + k : reinterpret_cast<const uint8_t*>(&kZeros), at + i * 1024);
    }
    if (lane < 4 * TT) dma16_from(sx + b * a.a_scales_ld, at + (2 + X) * 1024);
  };
  f32x4 acc[TT];
#pragma unroll
  for (int t = 0; t < TT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  const uint32_t swz = (uint32_t)((lg ^ (lr >> 1)) * 16);
#pragma unroll
  for (int i = 0; i < DEEP; ++i)
    if (wave + i * WAVES < a.groups) load(wave + i * WAVES, mine + i * BLOCK);
  uint32_t at = mine;
  for (int b = wave; b < a.groups; b += WAVES) {
    const float s_out = *(__attribute__((address_space(4))) const float*)uniform_ptr(sw + b);
    if (b + (DEEP - 1) * WAVES < a.groups) WAIT_DMA(LOADS * (DEEP - 1));
    else WAIT_DMA(0);
    asm volatile("" ::: "memory");
    const uint32_t w_at = at + lr * kFp8Group + swz, x_at = at + 2048 + lr % (8 * X) * kFp8Group + swz;
    const Pair w = {{lds16(w_at), lds16(w_at ^ 64)}};
    Pair x[TT];
    float scale[TT];
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      x[t] = Pair{{lds16(x_at + t * 2048), lds16((x_at ^ 64) + t * 2048)}};
      scale[t] = lds4(at + (2 + X) * 1024 + (t * 16 + lr) * 4) * s_out;
    }
    WAIT_LDS();
    asm volatile("" ::: "memory");
    if (b + DEEP * WAVES < a.groups) load(b + DEEP * WAVES, at);
    at = at + BLOCK == mine + DEEP * BLOCK ? mine : at + BLOCK;
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      f32x4 part = {0.f, 0.f, 0.f, 0.f};
      if constexpr (EXACT) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          bf16x8 bw[2], bx[2];
          to_bf16(w.v[j], bw);
          to_bf16(x[t].v[j], bx);
#pragma unroll
          for (int h = 0; h < 2; ++h)
            part = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bw[h], bx[h], part, 0, 0, 0);
        }
      } else {
        part = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
            __builtin_bit_cast(i32x8, w), __builtin_bit_cast(i32x8, x[t]), part, 0, 0, 0, 0, 0, 0);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[t][r] = fmaf(scale[t], part[r], acc[t][r]);
    }
  }
  __syncthreads();  // (every load has landed)
  float* sums = reinterpret_cast<float*>(ring);  // [wave][token][output]
#pragma unroll
  for (int t = 0; t < TT; ++t)
    *reinterpret_cast<f32x4*>(sums + (wave * TT + t) * 256 + lr * 16 + 4 * lg) = acc[t];
  __syncthreads();
  for (int i = threadIdx.x; i < a.M * 16; i += 64 * WAVES) {
    const int n = n0 + i % 16;
    if (n >= a.N) continue;
    float y = 0.f;
#pragma unroll
    for (int v = 0; v < WAVES; ++v) y += sums[v * TT * 256 + i];
    put_one<Out, KIND>(a, y, i / 16, n);
  }
}

template <typename Out, int KIND, bool EXACT>
hipError_t launch_rows(const Fp8Args& a, hipStream_t s) {
  constexpr int WAVES = 8, DEEP = 2;
  const dim3 grid((a.N + 15) / 16), block(64 * WAVES);
  if (a.M <= 8)
    hipLaunchKernelGGL((fp8_rows_kernel<Out, KIND, EXACT, WAVES, DEEP, 1>), grid, block, 0, s, a);
  else if (a.M <= 16)
    hipLaunchKernelGGL((fp8_rows_kernel<Out, KIND, EXACT, WAVES, DEEP, 2>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((fp8_rows_kernel<Out, KIND, EXACT, WAVES, DEEP, 4>), grid, block, 0, s, a);
  return hipGetLastError();
}

// The parts' sums of a split tile, added in order, then its outputs: four a thread.  Costs
// some 3.3 us, its launch for the most part, where the split saves more (64 x 1536 x 8960 in
// 64 x 64 tiles 28.6 us, in twelve parts 12.7).
template <typename Out, int KIND, typename T>
__global__ __launch_bounds__(256) void fp8_reduce_kernel(Fp8Args a) {
  constexpr int EACH = T::TM * T::TN / 4, THREADS = 64 * T::WAVES;
  const int tiles_n = (a.N + T::TN - 1) / T::TN;
  const uint32_t tiles_m = (a.M + T::TM - 1) / T::TM, tiles = tiles_m * tiles_n;
  const uint32_t tile = blockIdx.x / (EACH / 256);
  const int e = blockIdx.x % (EACH / 256) * 256 + threadIdx.x;
  int64_t tm;
  int tn;
  tile_coords<4>(tile, tiles_m, tiles_n, tm, tn);
  const int q = e / THREADS, wave = e % THREADS / 64, lane = e % 64;
  const int64_t m = tm * T::TM + (wave % T::WT * T::TT + q % T::TT) * 16 + (lane & 15);
  const int n = tn * T::TN + (wave / T::WT * T::FF + q / T::TT) * 16 + 4 * (lane >> 4);
  if (m >= a.M || n >= a.N) return;
  const f32x4* from = reinterpret_cast<const f32x4*>(a.partial) + (int64_t)tile * EACH + e;
  f32x4 y = from[0];
  for (int s = 1; s < a.split; s += 4) {  // four in flight; past the last: read again and dropped
    f32x4 v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = from[(int64_t)std::min(s + j, a.split - 1) * tiles * EACH];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (s + j < a.split) y += v[j];
  }
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (n + r < a.N) put_one<Out, KIND>(a, y[r], m, n + r);
}

template <typename Out, int KIND, bool EXACT, typename T>
hipError_t launch_tile(Fp8Args a, int split, hipStream_t s) {
  a.split = split;
  const int64_t tiles = ((int64_t)a.M + T::TM - 1) / T::TM * ((a.N + T::TN - 1) / T::TN);
  const dim3 grid((unsigned)std::min<int64_t>(tiles * split, device_cus() * T::OCC)), block(64 * T::WAVES);
  if constexpr (T::TM < 256) {
    if (split > 1) {
      if (a.K % kFp8Group == 0)
        hipLaunchKernelGGL((fp8_tile_kernel<float, PARTIAL, EXACT, false, T>), grid, block, 0, s, a);
      else
        hipLaunchKernelGGL((fp8_tile_kernel<float, PARTIAL, EXACT, true, T>), grid, block, 0, s, a);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
      hipLaunchKernelGGL((fp8_reduce_kernel<Out, KIND, T>), dim3((unsigned)(tiles * (T::TM * T::TN / 1024))), dim3(256), 0, s, a);
      return hipGetLastError();
    }
  }
  if (a.whole) {
    hipLaunchKernelGGL((fp8_tile_kernel<Out, KIND, EXACT, false, T>), grid, block, 0, s, a);
  } else {
    hipLaunchKernelGGL((fp8_tile_kernel<Out, KIND, EXACT, true, T>), grid, block, 0, s, a);
  }
  return hipGetLastError();
}

template <typename Out, int KIND, bool EXACT>
hipError_t launch(const Fp8Args& a, hipStream_t s) {
  const Fp8Form f = fp8_form(a.M, a.N, a.K, EXACT, device_cus());
  switch (f.tile) {
    case Fp8Tile::kRows: return launch_rows<Out, KIND, EXACT>(a, s);
    case Fp8Tile::k64: return launch_tile<Out, KIND, EXACT, Tile<4, 1, 1, 4, 4>>(a, f.split, s);
    case Fp8Tile::k128: return launch_tile<Out, KIND, EXACT, Tile<2, 2, 4, 4, 2>>(a, f.split, s);
    case Fp8Tile::k256: break;
  }
  if constexpr (EXACT) return hipErrorInvalidValue;  // (not one of its forms)
  else return launch_tile<Out, KIND, EXACT, Tile<4, 2, 4, 8, 1>>(a, 1, s);
}

}  // namespace
}  // namespace acid

using namespace acid;

extern "C" {

size_t acid_linear_fp8_workspace_needed(int64_t M, int32_t N, int32_t K) {
  if (M < 1 || N < 1 || K < 1 || K % 16 || M > (1 << 24) || N > (1 << 22) || K > (1 << 22)) return 0;
  const int64_t cus = device_cus();
  return sizeof(float) * (size_t)std::max(fp8_form(M, N, K, false, cus).floats, fp8_form(M, N, K, true, cus).floats);
}

acid_status acid_linear_fp8(const acid_linear_fp8_args* args, int64_t M, int32_t N, int32_t K,
                            hipStream_t stream) {
  if (!args) return set_error(ACID_ERR_INVALID_ARG, "NULL argument");
  const acid_linear_fp8_args& p = *args;
  if (p.out_dtype != ACID_F32 && p.out_dtype != ACID_BF16)
    return set_error(ACID_ERR_INVALID_ARG, "bad dtype %d", p.out_dtype);
  const int32_t kind = p.kind & ~ACID_FP8_EXACT;
  const bool update = kind == ACID_EPI_GATE_RESIDUAL;
  if (kind != ACID_EPI_BIAS && kind != ACID_EPI_BIAS_GELU && !update)
    return set_error(ACID_ERR_UNSUPPORTED, "fp8: epilogue %d is not BIAS, BIAS_GELU or GATE_RESIDUAL", kind);
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
  if (M > 0 && (p.a_scales_ld < round_up(M, 4) || p.a_scales_ld % 4 || p.a_scales_ld > most))
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
  const bool whole = K % kFp8Group == 0 && N * os % 16 == 0 && p.out_ld * os % 16 == 0 && (uintptr_t)p.out % 16 == 0 &&
                     (uintptr_t)p.bias % 16 == 0 &&
                     (!update || (p.residual_ld % 4 == 0 && ((uintptr_t)p.residual | (uintptr_t)p.gate) % 16 == 0));
  const bool wide = N % 4 == 0 && p.out_ld % 4 == 0 && (uintptr_t)p.out % (4 * os) == 0;
  const Fp8Args a = {(const uint8_t*)p.a, (const uint8_t*)p.w, p.a_scales, p.w_scales, p.bias, p.gate,
                     p.residual, p.out, p.a_ld, p.a_scales_ld, p.residual_ld, p.out_ld, (float*)p.workspace, (int32_t)M, N,
                     K, (int32_t)groups, 1, whole, wide};
  // 8-bit sums where a rounding to bf16 follows or the residual outweighs them, exact ones where asked for
  const bool exact = p.kind & ACID_FP8_EXACT;
  hipError_t e;
  if (update)
    e = exact ? launch<float, ACID_EPI_GATE_RESIDUAL, true>(a, stream) : launch<float, ACID_EPI_GATE_RESIDUAL, false>(a, stream);
  else if (p.out_dtype == ACID_F32)
    e = kind == ACID_EPI_BIAS ? launch<float, ACID_EPI_BIAS, true>(a, stream) : launch<float, ACID_EPI_BIAS_GELU, true>(a, stream);
  else if (exact)
    e = kind == ACID_EPI_BIAS ? launch<bf16, ACID_EPI_BIAS, true>(a, stream) : launch<bf16, ACID_EPI_BIAS_GELU, true>(a, stream);
  else
    e = kind == ACID_EPI_BIAS ? launch<bf16, ACID_EPI_BIAS, false>(a, stream) : launch<bf16, ACID_EPI_BIAS_GELU, false>(a, stream);
  return e == hipSuccess ? ACID_OK : check_hip(e, "linear fp8");
}

}  // extern "C"
