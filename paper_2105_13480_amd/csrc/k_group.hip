// Launches of the grouped products' tile kernel (group_kernel.h).
#include "group_pipe.h"

namespace cnnlib {

namespace {

using namespace group;

// Whether an operand can be copied straight to LDS, 16 bytes at a time: rows
// on 4-byte boundaries, and where its own index is last, whole units of it (k
// last: the kernel sees to the end of K).
bool copies_ok(const void* p, int64_t ld, int64_t extent, bool kc, int esize) {
  return ((uintptr_t)p & 3) == 0 && (ld * esize) % 4 == 0 && (kc || (extent * esize) % 16 == 0);
}

// Tiles that the worst split of Np rows into Ng groups and the rows past them
// needs: each non-empty group may leave one tile partly filled.
int64_t row_tiles(int64_t Np, int64_t Ng, bool groups, int TN) {
  if (!groups) return (Np + TN - 1) / TN;
  const int64_t parts = Ng + 1 < Np ? Ng + 1 : Np;
  return Np / TN + parts;
}

// Row tiles of TN rows of a launch.
template <int MODE> int64_t row_tiles_of(const GroupArgs& a, int TN) {
  if (MODE == kBwdKer) return (int64_t)a.Ng * ((a.N + TN - 1) / TN);
  return row_tiles(a.N, a.Ng, MODE != kAdapt, TN);
}

// What a tile costs (microseconds, measured on MI355X on products of one group
// with half a tile to four tiles a CU): `alone` for a stage of 128 bytes of k
// where a CU has one tile, `share` for a stage of each of several, `ends` for a
// tile's start and results, `once` for the launch.  A product of stages s and
// n tiles a CU takes once + s max(alone, n share) + n ends.  (The forward
// product's tiles of 64 x 64 and less have since become some 5 % quicker, alike.)
struct TileCost {
  int tm, tn;
  double alone, share, ends, once;
};
constexpr TileCost kBf16[] = {{256, 256, 1.33, 1.30, 10.5, 3.5},
                              {128, 128, 0.65, 0.50, 2.5, 4.0},
                              {64, 64, 0.28, 0.19, 1.1, 3.6},
                              {64, 32, 0.19, 0.137, 0.6, 4.6},
                              {32, 32, 0.17, 0.09, 0.4, 4.4}};
// fp32: the matrix unit's time at every size (2048 operations in 32 clocks)
constexpr TileCost kF32[] = {{0, 0, 0, 0, 0, 0},
                             {128, 128, 2.04, 2.06, 1.5, 7.5},
                             {64, 64, 0.67, 0.565, 1.0, 3.8},
                             {64, 32, 0.42, 0.33, 0.5, 3.6},
                             {32, 32, 0.30, 0.18, 0.4, 3.6}};

// The cheapest of the tile sizes from `first` on (0: with the pipelined
// kernel).  Group sizes are not known here: of several groups, half a tile each
// is taken to be empty.
template <typename T, int MODE> int pick_tile(const GroupArgs& a, int first, bool* crowded) {
  const TileCost* const c = sizeof(T) == 2 ? kBf16 : kF32;
  const int last = MODE == kBwdKer ? 2 : 4;
  const double cus = device_cus();
  int best = first;
  double least = 1e30;
  for (int i = first; i <= last; ++i) {
    const double mt = (a.M + c[i].tm - 1) / c[i].tm;
    double nt, k;
    if (MODE == kBwdKer) {
      nt = (double)a.Ng * ((a.N + c[i].tn - 1) / c[i].tn);
      k = (double)a.K / a.Ng;
    } else {
      nt = a.Ng == 1 ? (double)((a.N + c[i].tn - 1) / c[i].tn)
                     : (double)a.N / c[i].tn + 0.5 * (a.Ng < a.N ? a.Ng : a.N);
      k = a.K;
    }
    const double n = 1 + (double)(int64_t)(mt * nt / cus - 1e-3);  // of the CU with most
    const double stages = k * sizeof(T) / 128 + 1;
    const double t = c[i].once + stages * (n * c[i].share > c[i].alone ? n * c[i].share : c[i].alone) +
                     n * c[i].ends;
    if (t < least) {
      least = t;
      best = i;
      *crowded = n * (c[i].tm + c[i].tn) * 512 > 160 * 1024;
    }
  }
  return best;
}

// The tiles of 64 x 64 and less, by depth of their ring.  Where both operands
// have k last, a wave reads ahead and copies run the whole depth ahead: in bf16,
// whose stages are short, three stages let another workgroup onto a crowded CU
// (3000 rows of 6 groups of 768 x 512 8.6 us, 9.9 by four; 1500 of 4 of 3000 x 768
// 16.5 and 17.5; 17 rows of each of 28 of 4096 x 1024 48.3 and 49.6, or 35.4 and
// 33.5 where Ker is in the caches); four are better where all tiles fit (256 rows
// of 2048 x 2048 9.4 us, 11.1 by three) and in fp32 (3002 rows of 6 groups of
// 771 x 515 33.5 and 34.6).
template <typename T, typename TO, int MODE, int TM, int TN, bool WHOLE>
hipError_t launch_small(const GroupArgs& a, const AdaptArgs& ad, bool dma, bool crowded, Launch to) {
  const int64_t rt = row_tiles_of<MODE>(a, TN);
  if (!dma) return launch_tiles<T, TO, MODE, TM, TN, 2, 2, 0, WHOLE>(a, ad, rt, 16, to);
  if constexpr (sizeof(T) == 2 && (MODE == kFwd || MODE == kAdapt))
    if (crowded) return launch_tiles<T, TO, MODE, TM, TN, 2, 2, 3, WHOLE>(a, ad, rt, 16, to);
  return launch_tiles<T, TO, MODE, TM, TN, 2, 2, 4, WHOLE>(a, ad, rt, 16, to);
}

template <typename T, typename TO, int MODE, bool WHOLE>
hipError_t launch_sized(const GroupArgs& a, const AdaptArgs& ad, Launch to) {
  constexpr bool XKC = MODE == kFwd || MODE >= kAdapt, YKC = MODE != kBwdKer;
  const bool dma = copies_ok(a.X, a.ldx, a.M, XKC, sizeof(T)) && copies_ok(a.Y, a.ldy, a.N, YKC, sizeof(T));
  const bool pipe = sizeof(T) == 2 && WHOLE && dma && (MODE == kBwdKer || a.K % 8 == 0) && pipe_fits(a, MODE) &&
                    (MODE != kAdapt || ((uintptr_t)ad.B & 3) == 0);
  // fp32 through registers: 64 x 64 at most (gradient of In, 2000 rows of 2049 x
  // 2047 172 us, by 128 x 128 220, the other products alike; in bf16 56 and 71 there
  // but 187 and 162 at 8000 rows)
  const int first = pipe ? 0 : dma || sizeof(T) == 2 ? 1 : 2;
  bool crowded = false;
  const int pick = pick_tile<T, MODE>(a, first, &crowded);
  if constexpr (sizeof(T) == 2 && WHOLE)
    if (pick == 0) return launch_pipe<TO, MODE>(a, ad, row_tiles_of<MODE>(a, 256), 4, to);
  if (pick == 1) {
    const int64_t rt = row_tiles_of<MODE>(a, 128);
    if constexpr (sizeof(T) == 2)
      if (!dma) return launch_tiles<T, TO, MODE, 128, 128, 2, 2, 0, WHOLE>(a, ad, rt, 8, to);
    return launch_tiles<T, TO, MODE, 128, 128, 2, 2, 2, WHOLE>(a, ad, rt, 8, to);
  }
  if constexpr (MODE != kBwdKer) {
    if (pick == 4) return launch_small<T, TO, MODE, 32, 32, WHOLE>(a, ad, dma, crowded, to);
    if (pick == 3) return launch_small<T, TO, MODE, 64, 32, WHOLE>(a, ad, dma, crowded, to);
  }
  return launch_small<T, TO, MODE, 64, 64, WHOLE>(a, ad, dma, crowded, to);
}

template <typename T, typename TO, int MODE>
hipError_t launch_ranks(const GroupArgs& a, const AdaptArgs& ad, Launch to) {
  if constexpr (MODE == kAdapt)
    if (ad.nlp != ad.Nl) return launch_sized<T, TO, MODE, false>(a, ad, to);
  return launch_sized<T, TO, MODE, true>(a, ad, to);
}

template <int MODE>
hipError_t launch_typed(const GroupArgs& a, const AdaptArgs& ad, int dtype, Launch to) {
  switch (dtype) {
    case CNN_F32: return launch_ranks<float, float, MODE>(a, ad, to);
    case CNN_BF16: return launch_ranks<bf16_t, float, MODE>(a, ad, to);
    default: return launch_ranks<bf16_t, bf16_t, MODE>(a, ad, to);
  }
}

}  // namespace

hipError_t launch_group_fwd(const GroupArgs& a, int dtype, hipStream_t stream) {
  if (group_few_fits(a, dtype)) return launch_group_few(a, dtype, stream);
  return launch_typed<kFwd>(a, AdaptArgs{}, dtype, Launch{stream, false});
}
hipError_t launch_group_bwd_in(const GroupArgs& a, int dtype, hipStream_t stream) {
  return launch_typed<kBwdIn>(a, AdaptArgs{}, dtype, Launch{stream, false});
}
hipError_t launch_group_bwd_ker(const GroupArgs& a, int dtype, hipStream_t stream) {
  return launch_typed<kBwdKer>(a, AdaptArgs{}, dtype, Launch{stream, false});
}

namespace {

// Rows of the low-rank operand: the product grouped by adapter, whose ranks
// are few: tiles of 64 or 16 ranks by 32 rows.
template <typename T> hipError_t launch_down(const GroupArgs& a, const AdaptArgs& ad, Launch to) {
  GroupArgs h = a;
  h.X = ad.A;
  h.xgroup = (int64_t)ad.Nl * a.K;
  h.M = ad.Nl;
  h.Ng = ad.Na;
  const int64_t rt = row_tiles_of<kDown>(h, 32);
  const bool dma = copies_ok(h.X, h.ldx, h.M, true, sizeof(T)) && copies_ok(h.Y, h.ldy, h.N, true, sizeof(T));
  if (ad.Nl <= 16)
    return dma ? launch_tiles<T, T, kDown, 16, 32, 1, 2, 6>(h, ad, rt, 1, to)
               : launch_tiles<T, T, kDown, 16, 32, 1, 2, 0>(h, ad, rt, 1, to);
  return dma ? launch_tiles<T, T, kDown, 64, 32, 2, 2, 4>(h, ad, rt, 1, to)
             : launch_tiles<T, T, kDown, 64, 32, 2, 2, 0>(h, ad, rt, 1, to);
}

}  // namespace

hipError_t launch_adapt(const GroupArgs& a, const AdaptArgs& ad, int dtype, Launch to) {
  const hipError_t e =
      dtype == CNN_F32 ? launch_down<float>(a, ad, to) : launch_down<bf16_t>(a, ad, to);
  if (e != hipSuccess) return e;
  GroupArgs g = a;
  g.off = nullptr;
  g.Ng = 1;
  return launch_typed<kAdapt>(g, ad, dtype, to);
}

}  // namespace cnnlib
