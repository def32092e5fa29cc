// Which kernel and tile takes a product whose Ker lies in 4 bits: from sizes, strides and
// alignments alone, on the host, so that what a call runs can be asked without a GPU.
#pragma once

#include <algorithm>

#include "routed.h"

namespace cnnlib {
namespace group {

// Rows shorter than a unit of 16 bytes (64 x 32 tiles through registers, by elements); both
// in 4 bits, past a buffer's 2^31 bytes or of a single block (64 x 32, by addresses).
constexpr int kShort4 = -1;

// What a kernel's tile of tm features by tn rows costs (microseconds, fitted to 155
// products on MI355X: 1 to 32 groups of 1 to 3000 rows, 512 to 4096 features each way,
// Ker cold): of s stages and n tiles a CU, once + max(s max(alone, n share), Ker's bytes
// at bw TB/s) + n ends.  The fit is older than the kernels: those of few rows, both kinds of
// tiles with both in 4 bits and the pipelined ones have become faster since, and a last round
// that is halved, or a tile of half the features, counts as a whole one here.  Of the
// present kernels, launched from a graph, the pick is 5 % (bf16 rows), 2 % (both in 4 bits)
// and 2 % (gradient) above the best one's time on average over the same sizes, and at worst
// 1.48, 1.39 and 1.36 times it (8 rows of 8 groups of 1024 x 2048: 7.0 and 4.7 us; 512 rows
// of 8 groups of 4096 x 4096: 31 and 23; the gradient of 320 of them: 63 and 46).
struct Cost4 {
  int tm, tn;
  double alone, share, ends, once, bw;
};

// Group sizes are not known here: of several groups, half a tile each is taken to be
// empty, and each to have one.
inline double cost_of(const Cost4& c, const GroupArgs& a, double stages, double ker_bytes, int cus) {
  const double groups = a.Ng < a.N ? a.Ng : a.N;
  double nt = (a.N + c.tn - 1) / c.tn;
  if (a.Ng > 1) nt = std::max(groups, (double)a.N / c.tn + 0.5 * groups);
  const double tiles = nt * ((a.M + c.tm - 1) / c.tm);
  const double n = 1 + (double)(int64_t)(tiles / cus - 1e-3);  // of the CU with most
  return c.once + std::max(stages * std::max(c.alone, n * c.share), ker_bytes / (c.bw * 1e6)) + n * c.ends;
}

// The cheapest of c[first ..]; `last`: one past those that may run.
template <int N>
inline int cheapest(const Cost4 (&c)[N], int first, int last, const GroupArgs& a, double stages, int cus) {
  const double ker = (a.Ng < a.N ? a.Ng : a.N) * 0.53125 * a.M * a.K;
  int best = first;
  double least = 1e30;
  for (int i = first; i < last; ++i) {
    const double t = cost_of(c[i], a, stages, ker, cus);
    if (t < least) {
      least = t;
      best = i;
    }
  }
  return best;
}

// Whether the byte offsets of a tile's rows, of any row that may be gathered and (the
// gradient's) of a group's Ker fit a buffer of 2^31.
constexpr int64_t kMostBytes = (1LL << 31) - 65536;
inline bool pipe4_fits(const GroupArgs& a, bool gradient) {
  return a.ldx < (1 << 22) && a.ldy < (1 << 22) && (!a.rows || a.Nsrc * a.ldy * 2 < kMostBytes) &&
         (!gradient || a.K * a.ldx * 2 < kMostBytes);
}

// Runs of 128 of k that group4_few asks for at a time: some for each wave.
inline int few4_runs(int Nb) { return Nb >= 64 ? 4 : 2; }

// bf16 rows.  Straight from memory: rows on 4-byte boundaries and of whole units, 16 blocks
// a row at least; the pipelined kernel besides: scales on 4-byte boundaries.
constexpr Cost4 kFwd4[] = {{64, 32, 0.380, 0.319, 0.00, 5.6, 4.6},  // through registers
                           {64, 64, 0.580, 0.437, 0.43, 3.8, 4.9},
                           {128, 128, 1.202, 1.015, 1.37, 3.8, 4.9},
                           {16, 16, 0.028, 0.116, 0.15, 5.9, 3.7},  // straight from memory
                           {64, 16, 0.176, 0.172, 0.16, 5.1, 6.7},
                           {64, 32, 0.166, 0.217, 0.31, 5.0, 5.8},
                           {128, 64, 0.683, 0.553, 1.60, 3.0, 6.0},
                           {256, 256, 1.592, 2.200, 4.17, 3.0, 2.0}};
inline int pick_fwd4(const GroupArgs& a, const Group4Args& b, int cus) {
  if (a.K < 8) return kShort4;
  const bool rows = ((uintptr_t)a.Y & 3) == 0 && a.K % 8 == 0 && b.Nb >= 16 && pipe4_fits(a, false) &&
                    a.Nsrc * a.ldy * 2 < kMostBytes;
  const bool pipe = rows && b.Nb % 4 == 0 && ((uintptr_t)b.xs & 3) == 0;
  const int first = rows ? 2 : 0, last = pipe ? 8 : rows ? 7 : 3;
  return cheapest(kFwd4, first, last, a, (a.K + 127) / 128, cus);
}

// Both in 4 bits.
constexpr Cost4 kFwd44[] = {{32, 32, 0.109, 0.229, 0.36, 5.6, 6.7},   {64, 32, 0.217, 0.356, 0.64, 5.1, 6.4},
                            {128, 32, 0.252, 0.497, 1.37, 4.3, 7.0},  {128, 64, 0.306, 0.681, 1.89, 4.0, 6.8},
                            {128, 128, 1.188, 1.146, 1.76, 3.7, 5.8}, {256, 256, 0.555, 1.253, 4.79, 3.0, 5.0}};
inline int pick_fwd44(const GroupArgs& a, const Group4Args& b, int cus) {
  if (!(pipe4_fits(a, false) && b.Nb >= 2 && a.Nsrc * a.ldy * 2 < kMostBytes)) return kShort4;
  const bool pipe = b.Nb % 4 == 0 && (((uintptr_t)b.xs | (uintptr_t)b.ys) & 3) == 0;
  GroupArgs values = a;
  values.K = 32 * b.Nb;
  return cheapest(kFwd44, 0, pipe ? 6 : 5, values, (b.Nb + 7) / 8, cus);
}

// The gradient of In.  Pipelined: dOut's rows on 4-byte boundaries and of whole units.
constexpr Cost4 kBwdIn4[] = {{64, 32, 0.269, 0.188, 0.00, 4.5, 2.6},
                             {64, 64, 0.350, 0.255, 0.19, 3.4, 2.2},
                             {128, 128, 0.771, 0.557, 1.02, 3.0, 4.5},
                             {256, 256, 0.728, 1.238, 3.70, 3.0, 1.8}};
inline int pick_bwd_in4(const GroupArgs& a, int cus) {
  if (a.K < 8) return kShort4;
  const bool pipe = ((uintptr_t)a.Y & 3) == 0 && a.K % 8 == 0 && pipe4_fits(a, true);
  return cheapest(kBwdIn4, 0, pipe ? 4 : 3, a, (a.K + 63) / 64, cus);
}

}  // namespace group
}  // namespace cnnlib
