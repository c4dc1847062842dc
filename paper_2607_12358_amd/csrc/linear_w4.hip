// Few rows times 4-bit weights with group scales (acid_linear_w4), and the
// conversion of fp32 weights to them (acid_quantize_w4).
//
//   out[m][n] = act(sum_k x[m][k] (c[n][k] - 8) s[n][k / group] + bias[n])
//
// Bound by reading the codes once (HBM: 28672 x 8192 with groups of 128, 125 MB, 8
// bf16 rows, 26 us, 4.8 TB/s), so the layout is the one the matrix
// instruction takes: a tile is 16 outputs x 128 inputs, 1 KB, and lane l of
// the wave that reads it gets the 16 bytes of output l % 16 whose word j
// holds inputs 32 j + 8 (l / 16) .. + 7, its share of the j-th 16x16x32
// product.  Nibbles 0-3 and 4-7 of a word are its even and odd inputs, so
// one shift and one and-or turn two of them into a register pair of bf16.
#include <cfloat>
#include <cmath>
#include <type_traits>

#include "common.h"

namespace acid {
namespace {

// The eight codes of a word as bf16 values 16 + c: c sits in the top four
// mantissa bits of 16.0 (0x4180), exact.
__device__ __forceinline__ bf16x8 decode(uint32_t w) {
  u32x4 r;
  r[0] = ((w << 3) & 0x00780078u) | 0x41804180u;
  r[1] = ((w >> 1) & 0x00780078u) | 0x41804180u;
  r[2] = ((w >> 5) & 0x00780078u) | 0x41804180u;
  r[3] = ((w >> 9) & 0x00780078u) | 0x41804180u;
  return __builtin_bit_cast(bf16x8, r);
}

// Eight inputs of one operand row.  bf16 rows are taken as they are.  An
// fp32 row becomes three operand rows: the value cut to its first eight
// significant bits, the next eight, and the rest; their sum is exact, and the
// three products are added at the end.
__device__ __forceinline__ bf16x8 operand(const bf16x8 (&v)[1], int) { return v[0]; }
__device__ __forceinline__ bf16x8 operand(const f32x4 (&v)[2], int part) {
  const uint32_t less0 = part > 0 ? 0xffff0000u : 0u, less1 = part > 1 ? 0xffff0000u : 0u;
  uint32_t u[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = v[i / 4][i % 4];
    const float r = x - __uint_as_float(__float_as_uint(x) & less0);
    u[i] = __float_as_uint(r - __uint_as_float(__float_as_uint(r) & less1));
  }
  u32x4 out;  // the upper halves
#pragma unroll
  for (int i = 0; i < 4; ++i) out[i] = __builtin_amdgcn_perm(u[2 * i + 1], u[2 * i], 0x07060302u);
  return __builtin_bit_cast(bf16x8, out);
}

// The rows of one 128-input block, by way of a part of LDS that is one wave's
// alone: loaded there as whole lines, 1 KB an instruction, read as the operands
// they are.  (Each lane's own 16 bytes from L2, 64 of 16 rows an instruction: 16
// rows of 2048 x 28672 30 us for 18, 32 of 8192 x 8192 20 for 15; fp32, 4 rows of 2048
// x 28672 29 for 23, 32 of 1536 x 8960 32 for 28, but 64 of 8192 x 8192 83 for 86.)
// The 16-byte chunk c of row r is at slot c ^ swizzle(r), so that the rows of one
// chunk lie in different banks.
template <typename X>
struct Rows {
  typedef std::conditional_t<std::is_same_v<X, float>, f32x4, bf16x8> Chunk;
  static constexpr int CHUNKS = sizeof(X) * 8;     // of a row
  static constexpr int EIGHT = sizeof(X) / 2;      // of eight inputs
  static constexpr int PER_LOAD = 64 / CHUNKS;     // rows of an instruction
  static constexpr int MOST = std::is_same_v<X, float> ? 5 : 16;  // rows of a row tile
  static __host__ __device__ constexpr int loads(int rows) { return (rows + PER_LOAD - 1) / PER_LOAD; }
  static __device__ __forceinline__ int swizzle(int r) { return EIGHT * r; }
  // rows m0 .. of x (at input k0), `rows` of them
  static __device__ __forceinline__ void load(const X* x, int64_t x_ld, int rows, uint32_t lds,
                                              int lane) {
    for (int i = 0; i < loads(rows); ++i) {
      const int at = i * PER_LOAD + lane / CHUNKS, r = at < rows ? at : rows - 1;
      const X* p = x + r * x_ld + (lane % CHUNKS ^ swizzle(at)) % CHUNKS * (16 / (int)sizeof(X));
      asm volatile(
          "s_mov_b32 m0, %1\n\t"
          "s_nop 0\n\t"
          "global_load_lds_dwordx4 %0, off"
          :
          : "v"(p), "s"(__builtin_amdgcn_readfirstlane(lds + i * 1024))
          : "memory");
    }
  }
  // inputs 32 j + 8 g .. + 7 of row r
  static __device__ __forceinline__ void read(Chunk (&out)[EIGHT], uint32_t lds, int r, int j,
                                              int g) {
#pragma unroll
    for (int e = 0; e < EIGHT; ++e) {
      const int slot = (EIGHT * (4 * j + g) + e ^ swizzle(r)) % CHUNKS;
      out[e] = *(const __attribute__((address_space(3))) Chunk*)(lds + (r * CHUNKS + slot) * 16);
    }
  }
};

struct W4Args {
  const void* x;
  const uint8_t* codes;
  const float* scales;
  const float* bias;
  void* out;
  int64_t x_ld, out_ld;
  int32_t M, N, K, gelu;
};

// Sixteen waves pay where few tiles meet many blocks: 1536 x 8960, 8 / 16 waves, one
// row 7.2 / 5.9 us, four 7.1 / 6.3 (4608 x 1536, 8 / 12 waves: 3.8 / 4.2).
template <int NT, int MT>
constexpr int MOST_WAVES = NT * MT == 1 ? 16 : 8;

// A workgroup owns NT tiles of outputs and MT tiles of operand rows; its
// waves take the 128-input blocks in turn and their sums are added in wave
// order.  The matrix products give sum x (16 + c); one more product with the
// constant -24, shared by the output tiles, makes that sum x (c - 8) before
// the group's scale.  ONE: x is one bf16 row, each lane reads its operand itself.
template <typename X, typename Out, int GROUP, int NT, int MT, bool ONE>
__device__ __forceinline__ void products(const W4Args& a) {
  static_assert(!ONE || (std::is_same_v<X, bf16> && MT == 1), "one bf16 row");
  typedef Rows<X> R;
  constexpr int RPT = R::MOST;
  extern __shared__ __align__(1024) float red[];  // the rows; then sums, [wave][mt][nt][16][16]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int col = lane & 15, g = lane >> 4;
  const int KB = a.K / 128, tiles = (a.N + 15) / 16;
  const int tile0 = blockIdx.x * NT, m0 = blockIdx.y * (MT * RPT);
  const int part = std::is_same_v<X, float> ? col % 3 : 0;

  // operand row col: of row `row` of the tile; past the end a copy whose result is dropped
  const int row = std::is_same_v<X, float> ? (col < 15 ? col / 3 : 4) : col;
  const int loads = R::loads(a.M < RPT ? a.M : RPT);  // of a row tile
  const uint32_t lds = (uint32_t)(uintptr_t)(lds_void_t*)red +
                       wave * (MT * loads * 1024);
  int rows[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int left = a.M - m0 - mt * RPT;
    rows[mt] = left < RPT ? left : RPT;
  }
  const u32x4* codes[NT];
  const float* scales[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int64_t t = tile0 + nt < tiles ? tile0 + nt : tiles - 1;
    codes[nt] = reinterpret_cast<const u32x4*>(a.codes) + t * KB * 64 + lane;
    scales[nt] = a.scales + t * (a.K / GROUP) * 16 + col;
  }
  bf16x8 minus24;
#pragma unroll
  for (int i = 0; i < 8; ++i) minus24[i] = (bf16)-24.0f;

  f32x4 acc[MT][NT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) acc[mt][nt] = f32x4{0.f, 0.f, 0.f, 0.f};

  // a block's rows, codes and scales, one block ahead of the products
  u32x4 c_next[NT];
  float s_next[NT][128 / GROUP];
  auto load = [&](int b) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
      if (!ONE && rows[mt] > 0)
        R::load((const X*)a.x + (int64_t)(m0 + mt * RPT) * a.x_ld + b * 128, a.x_ld, rows[mt],
                lds + mt * loads * 1024, lane);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      c_next[nt] = codes[nt][b * 64];
#pragma unroll
      for (int i = 0; i < 128 / GROUP; ++i)
        s_next[nt][i] = scales[nt][(b * (128 / GROUP) + i) * 16];
    }
  };
  load(wave);  // there are no more waves than blocks
  for (int b = wave; b < KB; b += waves) {
    bf16x8 xf[MT][4];
    if constexpr (ONE) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        xf[0][j] = *reinterpret_cast<const bf16x8*>((const X*)a.x + b * 128 + 32 * j + 8 * g);
    } else {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          typename R::Chunk v[R::EIGHT];
          const int r = row < rows[mt] ? row : rows[mt] > 0 ? rows[mt] - 1 : 0;
          R::read(v, lds + mt * loads * 1024, r, j, g);
          xf[mt][j] = operand(v, part);
        }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
    u32x4 c[NT];
    float s[NT][128 / GROUP];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      c[nt] = c_next[nt];
#pragma unroll
      for (int i = 0; i < 128 / GROUP; ++i) s[nt][i] = s_next[nt][i];
    }
    if (b + waves < KB) load(b + waves);
    f32x4 off[MT], sum[MT][NT];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool first = j * 32 % GROUP == 0, last = (j + 1) * 32 % GROUP == 0;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
        off[mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            xf[mt][j], minus24, first ? f32x4{0.f, 0.f, 0.f, 0.f} : off[mt], 0, 0, 0);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const bf16x8 w = decode(c[nt][j]);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          sum[mt][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              xf[mt][j], w, first ? f32x4{0.f, 0.f, 0.f, 0.f} : sum[mt][nt], 0, 0, 0);
          if (last) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              acc[mt][nt][i] =
                  fmaf(s[nt][j * 32 / GROUP], sum[mt][nt][i] + off[mt][i], acc[mt][nt][i]);
          }
        }
      }
    }
  }
  __syncthreads();  // the rows have been read
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        red[((wave * MT + mt) * NT + nt) * 256 + (4 * g + i) * 16 + col] = acc[mt][nt][i];
  __syncthreads();
  for (int i = threadIdx.x; i < MT * NT * RPT * 16; i += blockDim.x) {
    const int c = i % 16, nt = i / 16 % NT, r = i / 16 / NT % RPT, mt = i / 16 / NT / RPT;
    const int n = (tile0 + nt) * 16 + c, m = m0 + mt * RPT + r;
    if (n >= a.N || m >= a.M) continue;
    float y = 0.f;
#pragma unroll 4
    for (int w = 0; w < waves; ++w) {
      const float* p = red + ((w * MT + mt) * NT + nt) * 256 + c;
      if constexpr (std::is_same_v<X, float>)
        y += (p[(3 * r + 2) * 16] + p[(3 * r + 1) * 16]) + p[3 * r * 16];
      else
        y += p[r * 16];
    }
    if (a.bias) y += a.bias[n];
    if constexpr (std::is_same_v<Out, bf16>) {
      if (a.gelu) y = gelu_tanh_fast(y);
    } else {
      if (a.gelu) y = gelu_tanh(y);
    }
    ((Out*)a.out)[m * a.out_ld + n] = (Out)y;
  }
}

template <typename X, typename Out, int GROUP, int NT, int MT>
__global__ __launch_bounds__(64 * (MOST_WAVES<NT, MT>)) void linear_w4_kernel(W4Args a) {
  products<X, Out, GROUP, NT, MT, false>(a);
}
template <typename Out, int GROUP>
__global__ __launch_bounds__(64 * (MOST_WAVES<1, 1>)) void linear_w4_row_kernel(W4Args a) {
  products<bf16, Out, GROUP, 1, 1, true>(a);
}

template <typename X, typename Out, int GROUP>
hipError_t launch(const W4Args& a, hipStream_t s) {
  constexpr int RPT = Rows<X>::MOST;
  const int tiles = (a.N + 15) / 16, KB = a.K / 128;
  const int loads = Rows<X>::loads(a.M < RPT ? a.M : RPT);
#define W4(NT, MT) W4_AS((linear_w4_kernel<X, Out, GROUP, NT, MT>), NT, MT)
#define W4_AS(KERNEL, NT, MT)                                                                 \
  do {                                                                                        \
    const int waves = KB < 8 ? KB : KB < 32 ? 8 : MOST_WAVES<NT, MT>;                         \
    hipLaunchKernelGGL(KERNEL,                                                                \
                       dim3((tiles + NT - 1) / NT, (a.M + MT * RPT - 1) / (MT * RPT)),        \
                       dim3(64 * waves), waves * MT * (loads > NT ? loads : NT) * 1024, s, a); \
  } while (0)
  // Two row tiles at once where there are two, so that codes are read and
  // decoded once for both.  Output tiles: as many as leave a workgroup for seven
  // CUs in eight, since each reads the rows (4 KB a block and row tile, to 1 KB of
  // codes an output tile).  1 / 16 / 32 bf16 rows: 28672 x 8192 26 / 35 / 55 us with one
  // output tile, 25 / 27 / 38 with four; 8192 x 28672 (512 tiles) 23 / 34 / 57 with one,
  // 22 / 29 / 41 with two, 34 / 40 / 55 with four; 14336 x 4096 (896) 8.4 / 10.2 / 14.9 with
  // two, 8.6 / 9.8 / 12.7 with four.  Four row tiles ran slower than two and two.
  const int groups = tiles * ((a.M + 2 * RPT - 1) / (2 * RPT));
  // One bf16 row has no lines to make whole, and where a CU has a workgroup at most
  // nothing hides a second trip.  By way of LDS / past it: 2048 x 28672 13.8 / 12.6 us,
  // 4096 x 14336 9.0 / 8.5, 1536 x 8960 6.2 / 5.9, 1024 x 2048 3.4 / 3.2, but 5000 x
  // 14336 (313 tiles) 14.6 / 16.5, 8960 x 1536 5.1 / 5.2, two rows of 2048 x 28672
  // 15.1 / 15.7, and groups of 64 and 32 of it 15.3 / 16.4 and 17.3 / 18.4.
  if constexpr (std::is_same_v<X, bf16> && GROUP == 128) {
    if (a.M == 1 && tiles <= 256) {
      W4_AS((linear_w4_row_kernel<Out, GROUP>), 1, 1);
      return hipGetLastError();
    }
  }
  if (a.M <= RPT) {
    if (groups >= 4 * 224) W4(4, 1);
    else if (groups >= 2 * 224) W4(2, 1);
    else W4(1, 1);
  } else {
    if (groups >= 4 * 224) W4(4, 2);
    else if (groups >= 2 * 224) W4(2, 2);
    else W4(1, 2);
  }
#undef W4
#undef W4_AS
  return hipGetLastError();
}

template <typename X, typename Out>
hipError_t launch_group(int group, const W4Args& a, hipStream_t s) {
  return group == 32   ? launch<X, Out, 32>(a, s)
         : group == 64 ? launch<X, Out, 64>(a, s)
                       : launch<X, Out, 128>(a, s);
}

// One thread per output and group: scale = max |w| / 7 (NaN if a weight of
// the group is not finite), code = w / scale rounded to nearest, ties to
// even, + 8.  Outputs past N, up to a whole tile, get scale 0 and code 8.  Reads w
// twice: 28672 x 8192 takes 408 us, where a copy of its 1.06 GB takes 214.
template <int GROUP>
__global__ __launch_bounds__(256) void quantize_w4_kernel(const float* __restrict__ w, int N,
                                                          int K, uint8_t* __restrict__ codes,
                                                          float* __restrict__ scales) {
  const int n = blockIdx.y * 256 + threadIdx.x, grp = blockIdx.x;
  const int64_t tile = n / 16;
  if (n >= (N + 15) / 16 * 16) return;
  const float* p = w + (int64_t)grp * GROUP * N + n;
  float most = 0.f;
  bool finite = true;
  if (n < N) {
    for (int k = 0; k < GROUP; ++k) {
      const float v = fabsf(p[(int64_t)k * N]);
      finite = finite && v <= FLT_MAX;
      most = fmaxf(most, v);
    }
  }
  const float scale = finite ? most / 7.0f : __builtin_nanf("");
  scales[(tile * (K / GROUP) + grp) * 16 + n % 16] = scale;
  for (int o = 0; o < GROUP / 8; ++o) {
    uint32_t word = 0x88888888u;
    if (n < N && scale > 0.f) {
      word = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float q = rintf(p[(int64_t)(8 * o + e) * N] / scale);
        const uint32_t c = (uint32_t)((int)fminf(fmaxf(q, -8.f), 7.f) + 8);
        word |= c << (4 * (e / 2 + 4 * (e % 2)));
      }
    }
    const int k = grp * GROUP + 8 * o, lane = k / 8 % 4 * 16 + n % 16;
    *reinterpret_cast<uint32_t*>(codes + ((tile * (K / 128) + k / 128) * 64 + lane) * 16 +
                                 k / 32 % 4 * 4) = word;
  }
}

acid_status check_w4_shape(int64_t N, int64_t K, int group) {
  if (N < 1 || K < 1) return set_error(ACID_ERR_INVALID_ARG, "N and K must be >= 1");
  if (group != 32 && group != 64 && group != 128)
    return set_error(ACID_ERR_SHAPE, "group %d: 32, 64 or 128", group);
  if (K % 128 || K > (1 << 22) || N > (1 << 22))
    return set_error(ACID_ERR_SHAPE, "w4: K %lld must be a multiple of 128, K and N <= 2^22",
                     (long long)K);
  return ACID_OK;
}

}  // namespace
}  // namespace acid

using namespace acid;

extern "C" {

acid_status acid_quantize_w4(const float* w_dev, int32_t N, int32_t K, int32_t group,
                             void* codes_dev, float* scales_dev, hipStream_t stream) {
  ACID_TRY(check_w4_shape(N, K, group));
  if (!w_dev || !codes_dev || !scales_dev) return set_error(ACID_ERR_INVALID_ARG, "NULL argument");
  if ((uintptr_t)w_dev % 4 || (uintptr_t)codes_dev % 16 || (uintptr_t)scales_dev % 4)
    return set_error(ACID_ERR_INVALID_ARG, "codes must be 16-byte aligned, w and scales 4-byte");
  const int64_t padded = round_up(N, 16), wb = (int64_t)N * K * 4, cb = padded * K / 2,
                sb = padded * (K / group) * 4;
  if (bytes_overlap(w_dev, wb, codes_dev, cb) || bytes_overlap(w_dev, wb, scales_dev, sb) ||
      bytes_overlap(codes_dev, cb, scales_dev, sb))
    return set_error(ACID_ERR_INVALID_ARG, "w, codes and scales overlap");
  StreamDevice on;
  ACID_TRY(on.enter(stream));
  const dim3 grid((unsigned)(K / group), (unsigned)((padded + 255) / 256));
#define QW(G) hipLaunchKernelGGL(quantize_w4_kernel<G>, grid, dim3(256), 0, stream, w_dev, N, K, (uint8_t*)codes_dev, scales_dev)
  if (group == 32) QW(32);
  else if (group == 64) QW(64);
  else QW(128);
#undef QW
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? ACID_OK : check_hip(e, "quantize w4");
}

acid_status acid_linear_w4(int32_t x_dtype, int64_t M, int32_t N, int32_t K, int32_t group,
                           const void* x_dev, int64_t x_ld, const void* codes_dev,
                           const float* scales_dev, const float* bias_dev, int32_t kind,
                           int32_t out_dtype, void* out_dev, int64_t out_ld, hipStream_t stream) {
  for (int dt : {x_dtype, out_dtype})
    if (dt != ACID_F32 && dt != ACID_BF16)
      return set_error(ACID_ERR_INVALID_ARG, "bad dtype %d", dt);
  if (kind != ACID_EPI_BIAS && kind != ACID_EPI_BIAS_GELU)
    return set_error(ACID_ERR_UNSUPPORTED, "w4: epilogue %d is not BIAS or BIAS_GELU", kind);
  if (M < 0) return set_error(ACID_ERR_INVALID_ARG, "M < 0");
  ACID_TRY(check_w4_shape(N, K, group));
  const int64_t xs = x_dtype == ACID_BF16 ? 2 : 4, os = out_dtype == ACID_BF16 ? 2 : 4;
  if (M > 65536) return set_error(ACID_ERR_SHAPE, "w4: M %lld: at most 65536 rows", (long long)M);
  if (x_ld < K || x_ld * xs % 16 || x_ld > ((int64_t)1 << 32) || out_ld < N ||
      out_ld > ((int64_t)1 << 32))
    return set_error(ACID_ERR_SHAPE,
                     "w4: x_ld >= K and whole 16 bytes, out_ld >= N, both <= 2^32");
  if (M == 0) return ACID_OK;
  if (!x_dev || !codes_dev || !scales_dev || !out_dev)
    return set_error(ACID_ERR_INVALID_ARG, "NULL argument");
  if (((uintptr_t)x_dev | (uintptr_t)codes_dev) % 16 || (uintptr_t)out_dev % os ||
      ((uintptr_t)scales_dev | (uintptr_t)bias_dev) % 4)
    return set_error(ACID_ERR_INVALID_ARG, "x and codes must be 16-byte aligned, the rest to an element");
  const int64_t padded = round_up(N, 16);
  const struct {
    const void* p;
    int64_t rows, width, ld;
  } in[] = {{x_dev, M, K * xs, x_ld * xs},
            {codes_dev, 1, padded * K / 2, padded * K / 2},
            {scales_dev, 1, padded * (K / group) * 4, padded * (K / group) * 4},
            {bias_dev, 1, (int64_t)N * 4, (int64_t)N * 4}};
  for (const auto& i : in)
    if (rows_overlap(out_dev, M, N * os, out_ld * os, i.p, i.rows, i.width, i.ld))
      return set_error(ACID_ERR_INVALID_ARG, "w4: out overlaps an input");
  StreamDevice on;
  ACID_TRY(on.enter(stream));
  const W4Args a = {x_dev, (const uint8_t*)codes_dev, scales_dev, bias_dev, out_dev, x_ld, out_ld,
                    (int32_t)M, N, K, kind == ACID_EPI_BIAS_GELU};
  hipError_t e;
  if (x_dtype == ACID_BF16)
    e = out_dtype == ACID_BF16 ? launch_group<bf16, bf16>(group, a, stream)
                               : launch_group<bf16, float>(group, a, stream);
  else
    e = out_dtype == ACID_BF16 ? launch_group<float, bf16>(group, a, stream)
                               : launch_group<float, float>(group, a, stream);
  return e == hipSuccess ? ACID_OK : check_hip(e, "linear w4");
}

}  // extern "C"
