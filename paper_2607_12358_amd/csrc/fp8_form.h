// Output tile and parts of K of a product of e4m3 operands: host code without any
// dependency, so that tests can compile it by itself.
#pragma once

#include <stdint.h>

#include <initializer_list>

namespace acid {

enum class Fp8Tile { kRows, k256, k128, k64 };
struct Fp8Form {
  Fp8Tile tile;
  int split;      // parts of K, each tile's sums left in the workspace and added by a second launch
  int64_t floats;  // of workspace
};
constexpr int kFp8FewRows = 16;

// The form with the least estimated time, in microseconds: base + rounds of workgroups x
// (once + blocks of 128 inputs x (least, or what a block costs a CU x the workgroups on it)); a
// round that is not full counts in part; a split adds a second launch and its bytes.  The
// constants are those that lose least against the best form of each of 185 measured shapes,
// 17 to 16000 rows, N 64 to 9600, K 128 to 8960: 0.7% on average (exact products 1.7%), 11% at most
// (28%); 256 x 256 tiles alone lose a factor of two.  Microseconds in a graph, weights in turn,
// 256 / 128 / 64, parts, and what the rule takes:
//     64 x 1536 x 8960:  89.5 /  42.0 /  28.6, 64 in 4 parts 13.2, 8 11.5, 12 12.7: 64 in 12
//    300 x 1536 x 8960:  92.7 /  42.8 /  29.1, 64 in 2 parts 20.8, 4 17.8, 8 19.6: 64 in 4
//    600 x 4608 x 1536:  23.4 /  11.8 /  11.5, 64 in 2 parts 25.3: 64
//   2048 x 1536 x 8960:  93.5 /  44.1 /  47.0, 128 in 2 parts 48.0, 3 53.3: 128 in 2
//   2500 x 4608 x 8960: 102.3 / 114.2 / 182.5: 256
//   4096 x 4608 x 1536:  47.2 /  36.8 /  53.6: 128
//   8200 x 1536 x 8960: 109.0 / 131.2 / 191.1: 256
// (64 x 128 tiles too would gain 0.8% on average; exact products, whose operands take twice the
// registers, in 256 x 128 tiles nothing.)  Up to 16 rows have a kernel of their own, and up to
// 32 where its workgroups, of 16 outputs and one a CU, take less than two rounds (its bf16
// outputs, then exact ones, / 64 x 64 tiles, parts among them):
//   32 x 1536 x 1536  3.3, 3.6 /  7.4,  8.5       32 x 8960 x 1536   8.3,  8.8 /  7.8, 10.9
//   32 x 4608 x 1536  6.0, 6.3 /  7.7, 10.8       32 x 8192 x 8192  20.6, 21.4 / 19.6, 22.5
//   32 x 1536 x 8960  7.5, 8.3 / 11.2, 13.5       32 x 28672 x 8192 64.7, 66.6 / 49.1, 57.8
inline Fp8Form fp8_form(int64_t M, int64_t N, int64_t K, bool exact, int64_t cus) {
  if (M <= kFp8FewRows || (M <= 2 * kFp8FewRows && (N + 15) / 16 < 2 * cus)) return {Fp8Tile::kRows, 1, 0};
  struct Times {
    Fp8Tile tile;
    int tm, tn, occ;
    double base, once, least, each, part;
  };
  static constexpr Times kTimes[] = {{Fp8Tile::k256, 256, 256, 1, 0, 10.0, 1.39, 1.39, 0.10},
                                     {Fp8Tile::k128, 128, 128, 2, 1.1, 2.4, 0.66, 0.50, 0.74},
                                     {Fp8Tile::k64, 64, 64, 4, 2.5, 0.70, 0.361, 0.193, 0.78}};
  static constexpr Times kExact[] = {{Fp8Tile::k128, 128, 128, 2, 0, 4.2, 1.23, 0.63, 0.91},
                                     {Fp8Tile::k64, 64, 64, 4, 2.9, 1.05, 0.66, 0.36, 0.93}};
  const int64_t blocks = (K + 127) / 128;
  Fp8Form f = {Fp8Tile::k128, 1, 0};
  double best = 1e300;
  for (int i = 0; i < (exact ? 2 : 3); ++i) {
    const Times& t = exact ? kExact[i] : kTimes[i];
    const int64_t tiles = (M + t.tm - 1) / t.tm * ((N + t.tn - 1) / t.tn), slots = cus * t.occ;
    for (int split : {1, 2, 3, 4, 6, 8, 12}) {
      const int64_t items = tiles * split;
      if (split > 1 && (t.tile == Fp8Tile::k256 || items > 2 * slots || blocks < 2 * split)) break;
      double q = (double)items / cus, x = (double)items / slots;
      q = q < 1 ? 1 : q > t.occ ? t.occ : q;
      double rounds = (1 - t.part) * (double)((items + slots - 1) / slots) + t.part * x;
      if (rounds < 1) rounds = 1;
      const double block = t.least > q * t.each ? t.least : q * t.each;
      double cost = t.base + rounds * (t.once * (0.5 + 0.5 * q) + block * (double)((blocks + split - 1) / split));
      if (split > 1) cost += 3.3 + (exact ? 1.23e-6 : 1.67e-6) * (double)(items * t.tm * t.tn);
      if (cost < best) {
        best = cost;
        f = {t.tile, split, split > 1 ? items * t.tm * t.tn : 0};
      }
    }
  }
  return f;
}

}  // namespace acid
