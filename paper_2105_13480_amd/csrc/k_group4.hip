// Launches of the grouped products whose Ker lies in 4 bits: which kernel and tile.
#include <algorithm>

#include "group4_pipe.h"

namespace cnnlib {

namespace {

using namespace group;

// What a kernel's tile of tm features by tn rows costs (microseconds, fitted to 155
// products on MI355X: 1 to 32 groups of 1 to 3000 rows, 512 to 4096 features each way,
// Ker cold): of s stages and n tiles a CU, once + max(s max(alone, n share), Ker's bytes
// at bw TB/s) + n ends.  The least is within 1 to 3 % of the best kernel's time on
// average, 1.35 times it at worst.
struct Cost4 {
  int tm, tn;
  double alone, share, ends, once, bw;
};

// Group sizes are not known here: of several groups, half a tile each is taken to be
// empty, and each to have one.
double cost_of(const Cost4& c, const GroupArgs& a, double stages, double ker_bytes) {
  const double groups = a.Ng < a.N ? a.Ng : a.N;
  double nt = (a.N + c.tn - 1) / c.tn;
  if (a.Ng > 1) nt = std::max(groups, (double)a.N / c.tn + 0.5 * groups);
  const double tiles = nt * ((a.M + c.tm - 1) / c.tm);
  const double n = 1 + (double)(int64_t)(tiles / device_cus() - 1e-3);  // of the CU with most
  return c.once + std::max(stages * std::max(c.alone, n * c.share), ker_bytes / (c.bw * 1e6)) + n * c.ends;
}

// The cheapest of c[first ..]; `last`: one past those that may run.
template <int N> int cheapest(const Cost4 (&c)[N], int first, int last, const GroupArgs& a, double stages) {
  const double ker = (a.Ng < a.N ? a.Ng : a.N) * 0.53125 * a.M * a.K;
  int best = first;
  double least = 1e30;
  for (int i = first; i < last; ++i) {
    const double t = cost_of(c[i], a, stages, ker);
    if (t < least) {
      least = t;
      best = i;
    }
  }
  return best;
}

int64_t tiles_of(const GroupArgs& a, int tn) { return row_tiles(a.N, a.Ng, true, tn); }

// bf16 rows.  Straight from memory: rows on 4-byte boundaries and of whole units, 16 blocks
// a row at least; the pipelined kernel besides: scales on 4-byte boundaries.
constexpr Cost4 kFwd4[] = {{64, 32, 0.380, 0.319, 0.00, 5.6, 4.6},  // through registers
                           {64, 64, 0.580, 0.437, 0.43, 3.8, 4.9},
                           {128, 128, 1.202, 1.015, 1.37, 3.8, 4.9},
                           {16, 16, 0.028, 0.116, 0.15, 5.9, 3.7},  // straight from memory
                           {64, 16, 0.176, 0.172, 0.16, 5.1, 6.7},
                           {64, 32, 0.166, 0.217, 0.31, 5.0, 5.8},
                           {128, 64, 0.683, 0.553, 1.60, 3.0, 6.0},
                           {256, 256, 1.592, 2.200, 4.17, 3.0, 2.0}};  // pipelined

template <typename TO> hipError_t launch_fwd4(const GroupArgs& a, const Group4Args& b, hipStream_t stream) {
  constexpr bool OB = sizeof(TO) == 2;
  if (a.K < 8) return launch_tiles4<TO, kFwd, 64, 32, false>(a, b, tiles_of(a, 32), 16, stream);
  const bool rows = ((uintptr_t)a.Y & 3) == 0 && a.K % 8 == 0 && b.Nb >= 16 && pipe4_fits(a, kFwd) &&
                    a.Nsrc * a.ldy * 2 < kMostBytes;
  const bool pipe = rows && b.Nb % 4 == 0 && ((uintptr_t)b.xs & 3) == 0;
  const int first = rows ? 2 : 0, last = pipe ? 8 : rows ? 7 : 3;
  const int pick = cheapest(kFwd4, first, last, a, (a.K + 127) / 128);
  switch (pick) {
    case 0: return launch_tiles4<TO, kFwd, 64, 32>(a, b, tiles_of(a, 32), 16, stream);
    case 1: return launch_tiles4<TO, kFwd, 64, 64>(a, b, tiles_of(a, 64), 16, stream);
    case 2: return launch_tiles4<TO, kFwd, 128, 128>(a, b, tiles_of(a, 128), 8, stream);
    case 3: return launch_group4_few(a, b, OB, stream);
    case 7: return launch_pipe4<TO, kFwd>(a, b, tiles_of(a, 256), 4, stream);
    default: return launch_group4_rows(a, b, OB, pick == 4 ? 16 : pick == 5 ? 32 : 64, stream);
  }
}

// Both in 4 bits.
constexpr Cost4 kFwd44[] = {{32, 32, 0.109, 0.229, 0.36, 5.6, 6.7},   {64, 32, 0.217, 0.356, 0.64, 5.1, 6.4},
                            {128, 32, 0.252, 0.497, 1.37, 4.3, 7.0},  {128, 64, 0.306, 0.681, 1.89, 4.0, 6.8},
                            {128, 128, 1.188, 1.146, 1.76, 3.7, 5.8}, {256, 256, 0.555, 1.253, 4.79, 3.0, 5.0}};

template <typename TO> hipError_t launch_fwd44(const GroupArgs& a, const Group4Args& b, hipStream_t stream) {
  const bool buf = pipe4_fits(a, kFwd) && b.Nb >= 2 && a.Nsrc * a.ldy * 2 < kMostBytes;
  if (!buf) return launch_tiles44<TO, 64, 32, 2, 2, 4, false>(a, b, tiles_of(a, 32), 16, stream);
  const bool pipe = b.Nb % 4 == 0 && (((uintptr_t)b.xs | (uintptr_t)b.ys) & 3) == 0;
  GroupArgs values = a;
  values.K = 32 * b.Nb;
  // rings: more workgroups on a CU do more than more stages of each (1536 rows of 60
  // groups of 1536 x 2048 in 128 x 32 tiles, four stages, three, two: 36, 34 and 33 us with
  // the quantisation), but a lone one wants them
  switch (cheapest(kFwd44, 0, pipe ? 6 : 5, values, (b.Nb + 7) / 8)) {
    case 0: return launch_tiles44<TO, 32, 32, 2, 2, 4>(a, b, tiles_of(a, 32), 16, stream);
    case 1: return launch_tiles44<TO, 64, 32, 2, 2, 4>(a, b, tiles_of(a, 32), 16, stream);
    case 2: return launch_tiles44<TO, 128, 32, 4, 1, 3>(a, b, tiles_of(a, 32), 16, stream);
    case 3: return launch_tiles44<TO, 128, 64, 4, 1, 3>(a, b, tiles_of(a, 64), 16, stream);
    case 4: return launch_tiles44<TO, 128, 128, 2, 2, 2>(a, b, tiles_of(a, 128), 8, stream);
    default: return launch_pipe44<TO>(a, b, tiles_of(a, 256), 4, stream);
  }
}

// The gradient of In.  Pipelined: dOut's rows on 4-byte boundaries and of whole units.
constexpr Cost4 kBwdIn4[] = {{64, 32, 0.269, 0.188, 0.00, 4.5, 2.6},
                             {64, 64, 0.350, 0.255, 0.19, 3.4, 2.2},
                             {128, 128, 0.771, 0.557, 1.02, 3.0, 4.5},
                             {256, 256, 0.728, 1.238, 3.70, 3.0, 1.8}};

template <typename TO> hipError_t launch_bwd_in4(const GroupArgs& a, const Group4Args& b, hipStream_t stream) {
  if (a.K < 8) return launch_tiles4<TO, kBwdIn, 64, 32, false>(a, b, tiles_of(a, 32), 16, stream);
  const bool pipe = ((uintptr_t)a.Y & 3) == 0 && a.K % 8 == 0 && pipe4_fits(a, kBwdIn);
  switch (cheapest(kBwdIn4, 0, pipe ? 4 : 3, a, (a.K + 63) / 64)) {
    case 0: return launch_tiles4<TO, kBwdIn, 64, 32>(a, b, tiles_of(a, 32), 16, stream);
    case 1: return launch_tiles4<TO, kBwdIn, 64, 64>(a, b, tiles_of(a, 64), 16, stream);
    case 2: return launch_tiles4<TO, kBwdIn, 128, 128>(a, b, tiles_of(a, 128), 8, stream);
    default: return launch_pipe4<TO, kBwdIn>(a, b, tiles_of(a, 256), 4, stream);
  }
}

}  // namespace

hipError_t launch_group_fwd4(const GroupArgs& a, const Group4Args& b, bool bf16_out, hipStream_t stream) {
  if (b.ys) return bf16_out ? launch_fwd44<bf16_t>(a, b, stream) : launch_fwd44<float>(a, b, stream);
  return bf16_out ? launch_fwd4<bf16_t>(a, b, stream) : launch_fwd4<float>(a, b, stream);
}

hipError_t launch_group_bwd_in4(const GroupArgs& a, const Group4Args& b, bool bf16_out, hipStream_t stream) {
  return bf16_out ? launch_bwd_in4<bf16_t>(a, b, stream) : launch_bwd_in4<float>(a, b, stream);
}

}  // namespace cnnlib
