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

template <typename T, typename TO, int MODE, bool WHOLE>
hipError_t launch_sized(const GroupArgs& a, const AdaptArgs& ad, hipStream_t stream) {
  constexpr bool XKC = MODE == kFwd || MODE == kAdapt, YKC = MODE != kBwdKer;
  const bool dma = copies_ok(a.X, a.ldx, a.M, XKC, sizeof(T)) && copies_ok(a.Y, a.ldy, a.N, YKC, sizeof(T));
  const int64_t rows = MODE == kBwdKer ? a.N : a.N / a.Ng;
  if constexpr (sizeof(T) == 2 && WHOLE)
    if (dma && rows >= 192 && a.M >= 192 && (MODE == kBwdKer || a.K % 8 == 0) && pipe_fits(a, MODE))
      return launch_pipe<TO, MODE>(a, ad, row_tiles_of<MODE>(a, 256), 4, stream);
  // results of 128 x 128 tiles: do they make a workgroup for each CU?
  const int64_t big = row_tiles_of<MODE>(a, 128) * ((a.M + 127) / 128);
  if (big >= 256) {
    if (dma)
      return launch_tiles<T, TO, MODE, 128, 128, 2, 2, 2, WHOLE>(a, ad, row_tiles_of<MODE>(a, 128), 8, stream);
    return launch_tiles<T, TO, MODE, 128, 128, 2, 2, 0, WHOLE>(a, ad, row_tiles_of<MODE>(a, 128), 8, stream);
  }
  if (dma)
    return launch_tiles<T, TO, MODE, 64, 64, 2, 2, 4, WHOLE>(a, ad, row_tiles_of<MODE>(a, 64), 16, stream);
  return launch_tiles<T, TO, MODE, 64, 64, 2, 2, 0, WHOLE>(a, ad, row_tiles_of<MODE>(a, 64), 16, stream);
}

template <typename T, typename TO, int MODE>
hipError_t launch_ranks(const GroupArgs& a, const AdaptArgs& ad, hipStream_t stream) {
  if constexpr (MODE == kAdapt)
    if (ad.nlp != ad.Nl) return launch_sized<T, TO, MODE, false>(a, ad, stream);
  return launch_sized<T, TO, MODE, true>(a, ad, stream);
}

template <int MODE>
hipError_t launch_typed(const GroupArgs& a, const AdaptArgs& ad, int dtype, hipStream_t stream) {
  switch (dtype) {
    case CNN_F32: return launch_ranks<float, float, MODE>(a, ad, stream);
    case CNN_BF16: return launch_ranks<bf16_t, float, MODE>(a, ad, stream);
    default: return launch_ranks<bf16_t, bf16_t, MODE>(a, ad, stream);
  }
}

}  // namespace

hipError_t launch_group_fwd(const GroupArgs& a, int dtype, hipStream_t stream) {
  if (group_few_fits(a)) return launch_group_few(a, dtype, stream);
  return launch_typed<kFwd>(a, AdaptArgs{}, dtype, stream);
}
hipError_t launch_group_bwd_in(const GroupArgs& a, int dtype, hipStream_t stream) {
  return launch_typed<kBwdIn>(a, AdaptArgs{}, dtype, stream);
}
hipError_t launch_group_bwd_ker(const GroupArgs& a, int dtype, hipStream_t stream) {
  return launch_typed<kBwdKer>(a, AdaptArgs{}, dtype, stream);
}

hipError_t launch_adapt(const GroupArgs& a, const AdaptArgs& ad, int dtype, hipStream_t stream) {
  const hipError_t e = launch_adapt_down(a, ad, dtype, stream);
  if (e != hipSuccess) return e;
  GroupArgs g = a;
  g.off = nullptr;
  g.Ng = 1;
  return launch_typed<kAdapt>(g, ad, dtype, stream);
}

}  // namespace cnnlib
