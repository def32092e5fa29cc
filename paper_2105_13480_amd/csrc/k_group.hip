// Launches of the grouped products' tile kernel (group_kernel.h).
#include "group_pipe.h"

namespace cnnlib {

namespace {

using namespace group;

// Whether copies of whole 16-byte units may be used: every row starts on a
// 16-byte boundary and holds whole units.
bool units_ok(const void* p, int64_t ld, int64_t extent, int esize) {
  return ((uintptr_t)p & 15) == 0 && (ld * esize) % 16 == 0 && (extent * esize) % 16 == 0;
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

template <typename T, typename TO, int MODE, bool DMA>
hipError_t launch_sized(const GroupArgs& a, const AdaptArgs& ad, hipStream_t stream) {
  if constexpr (sizeof(T) == 2 && DMA) {
    const int64_t rows = MODE == kBwdKer ? a.N : a.N / a.Ng;
    if (rows >= 192 && a.M >= 192 && pipe_fits(a, MODE) && ad.nlp == ad.Nl)
      return launch_pipe<TO, MODE>(a, ad, row_tiles_of<MODE>(a, 256), 4, stream);
  }
  if (MODE == kAdapt && ad.nlp != ad.Nl)
    return launch_tiles<T, TO, MODE, 128, 128, 2, 2, DMA, MODE != kAdapt>(
        a, ad, row_tiles_of<MODE>(a, 128), 8, stream);
  return launch_tiles<T, TO, MODE, 128, 128, 2, 2, DMA>(a, ad, row_tiles_of<MODE>(a, 128), 8, stream);
}

template <typename T, typename TO, int MODE>
hipError_t launch_aligned(const GroupArgs& a, const AdaptArgs& ad, hipStream_t stream) {
  // a KC operand's rows hold K values, an MC operand's the tile index
  const int64_t ex = MODE == kFwd || MODE == kAdapt ? a.K : a.M;
  const int64_t ey = MODE == kBwdKer ? a.N : a.K;
  if (units_ok(a.X, a.ldx, ex, sizeof(T)) && units_ok(a.Y, a.ldy, ey, sizeof(T)))
    return launch_sized<T, TO, MODE, true>(a, ad, stream);
  return launch_sized<T, TO, MODE, false>(a, ad, stream);
}

template <int MODE>
hipError_t launch_typed(const GroupArgs& a, const AdaptArgs& ad, int dtype, hipStream_t stream) {
  switch (dtype) {
    case CNN_F32: return launch_aligned<float, float, MODE>(a, ad, stream);
    case CNN_BF16: return launch_aligned<bf16_t, float, MODE>(a, ad, stream);
    default: return launch_aligned<bf16_t, bf16_t, MODE>(a, ad, stream);
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
