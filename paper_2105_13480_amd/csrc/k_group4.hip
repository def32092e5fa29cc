// Launches of the grouped products whose Ker lies in 4 bits (group4_kernel.h).
#include "group4_pipe.h"
#include <stdlib.h>

namespace cnnlib {

namespace {

using namespace group;

int pick_tile4(const GroupArgs& a, bool pipe) {
  if (const char* e = getenv("CNN_T4")) { int t = atoi(e); return t == 256 && !pipe ? 128 : t; }
  const int sizes[] = {128, 64};
  for (int t : sizes)
    if (((a.M + t - 1) / t) * ((int64_t)a.N / t + (a.Ng < a.N ? a.Ng : a.N)) >= device_cus()) return t;
  return 32;
}

template <typename TO, int MODE>
hipError_t launch_sized4(const GroupArgs& a, const Group4Args& b, hipStream_t stream) {
  const bool pipe = ((uintptr_t)a.Y & 3) == 0 && a.ldy % 2 == 0 && a.K % 8 == 0 && (MODE != kFwd || (b.Nb % 4 == 0 && ((uintptr_t)b.xs & 3) == 0)) && pipe4_fits(a, MODE);
  const int t = pick_tile4(a, pipe);
  if (t == 256) return launch_pipe4<TO, MODE>(a, b, row_tiles(a.N, a.Ng, true, 256), 4, stream);
  if (t == 128) return launch_tiles4<TO, MODE, 128, 128>(a, b, row_tiles(a.N, a.Ng, true, 128), 8, stream);
  if (t == 64) return launch_tiles4<TO, MODE, 64, 64>(a, b, row_tiles(a.N, a.Ng, true, 64), 16, stream);
  if (t == 65) return launch_tiles4<TO, MODE, 64, 32>(a, b, row_tiles(a.N, a.Ng, true, 32), 16, stream);
  if (t == 129) return launch_tiles4<TO, MODE, 128, 32>(a, b, row_tiles(a.N, a.Ng, true, 32), 16, stream);
  return launch_tiles4<TO, MODE, 32, 32>(a, b, row_tiles(a.N, a.Ng, true, 32), 16, stream);
}

template <typename TO> hipError_t launch_sized44(const GroupArgs& a, const Group4Args& b, hipStream_t stream) {
  const bool buf = pipe4_fits(a, kFwd) && b.Nb >= 2 && (int64_t)a.Nsrc * a.ldy * 2 < (1LL << 31) - 65536;
  if (!buf) return launch_tiles44<TO, 64, 32, 2, 2, 4, false>(a, b, row_tiles(a.N, a.Ng, true, 32), 16, stream);
  const int t = pick_tile4(a, buf && b.Nb % 4 == 0 && (((uintptr_t)b.xs | (uintptr_t)b.ys) & 3) == 0);
  if (t == 256) return launch_pipe44<TO>(a, b, row_tiles(a.N, a.Ng, true, 256), 4, stream);
  if (t == 128) return launch_tiles44<TO, 128, 128, 2, 2, 2>(a, b, row_tiles(a.N, a.Ng, true, 128), 8, stream);
  if (t == 64) return launch_tiles44<TO, 64, 64, 2, 2, 4>(a, b, row_tiles(a.N, a.Ng, true, 64), 16, stream);
  if (t == 65) return launch_tiles44<TO, 64, 32, 2, 2, 4>(a, b, row_tiles(a.N, a.Ng, true, 32), 16, stream);
  if (t == 129) return launch_tiles44<TO, 128, 32, 2, 2, 4>(a, b, row_tiles(a.N, a.Ng, true, 32), 16, stream);
  if (t == 130) return launch_tiles44<TO, 128, 64, 2, 2, 3>(a, b, row_tiles(a.N, a.Ng, true, 64), 16, stream);
  if (t == 131) return launch_tiles44<TO, 128, 32, 4, 1, 3>(a, b, row_tiles(a.N, a.Ng, true, 32), 16, stream);
  if (t == 132) return launch_tiles44<TO, 128, 128, 2, 2, 3>(a, b, row_tiles(a.N, a.Ng, true, 128), 8, stream);
  if (t == 140) return launch_tiles44<TO, 128, 64, 4, 1, 3>(a, b, row_tiles(a.N, a.Ng, true, 64), 16, stream);
  if (t == 141) return launch_tiles44<TO, 64, 64, 4, 1, 3>(a, b, row_tiles(a.N, a.Ng, true, 64), 16, stream);
  if (t == 142) return launch_tiles44<TO, 64, 32, 4, 1, 4>(a, b, row_tiles(a.N, a.Ng, true, 32), 16, stream);
  if (t == 143) return launch_tiles44<TO, 64, 64, 4, 1, 4>(a, b, row_tiles(a.N, a.Ng, true, 64), 16, stream);
  if (t == 144) return launch_tiles44<TO, 128, 32, 4, 1, 4>(a, b, row_tiles(a.N, a.Ng, true, 32), 16, stream);
  if (t == 145) return launch_tiles44<TO, 128, 32, 4, 1, 2>(a, b, row_tiles(a.N, a.Ng, true, 32), 16, stream);
  if (t == 146) return launch_tiles44<TO, 64, 32, 4, 1, 3>(a, b, row_tiles(a.N, a.Ng, true, 32), 16, stream);
  if (t == 149) return launch_tiles44<TO, 128, 64, 4, 1, 2>(a, b, row_tiles(a.N, a.Ng, true, 64), 16, stream);
  return launch_tiles44<TO, 32, 32, 2, 2, 4>(a, b, row_tiles(a.N, a.Ng, true, 32), 16, stream);
}

}  // namespace

hipError_t launch_group_fwd4(const GroupArgs& a, const Group4Args& b, bool bf16_out, hipStream_t stream) {
  const int t = pick_tile4(a, false);
  const bool ok = a.Nsrc * (int64_t)a.ldy * 2 < (1LL << 31) && (b.ys || (((uintptr_t)a.Y & 3) == 0 && a.K % 8 == 0));
  if (t == 16 && b.Nb >= 8 && (!b.ys || ok)) return launch_group4_few(a, b, bf16_out, stream);
  if (t > 1000 && ok && b.Nb >= 16) return launch_group4_rows(a, b, bf16_out, t > 2000 ? 128 : 64, t % 1000, stream);
  if (b.ys) return bf16_out ? launch_sized44<bf16_t>(a, b, stream) : launch_sized44<float>(a, b, stream);
  return bf16_out ? launch_sized4<bf16_t, kFwd>(a, b, stream) : launch_sized4<float, kFwd>(a, b, stream);
}

hipError_t launch_group_bwd_in4(const GroupArgs& a, const Group4Args& b, bool bf16_out, hipStream_t stream) {
  return bf16_out ? launch_sized4<bf16_t, kBwdIn>(a, b, stream) : launch_sized4<float, kBwdIn>(a, b, stream);
}

}  // namespace cnnlib
