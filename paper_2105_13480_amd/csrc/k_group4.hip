// Launches of the grouped products whose Ker lies in 4 bits (group4_kernel.h).
#include "group4_kernel.h"

namespace cnnlib {

namespace {

using namespace group;

// The largest tile of which the launch has one for every CU.
int pick_tile4(const GroupArgs& a) {
  const int sizes[] = {128, 64};
  for (int t : sizes)
    if (((a.M + t - 1) / t) * ((int64_t)a.N / t + (a.Ng < a.N ? a.Ng : a.N)) >= device_cus()) return t;
  return 32;
}

template <typename TO, int MODE>
hipError_t launch_sized4(const GroupArgs& a, const Group4Args& b, hipStream_t stream) {
  const int t = pick_tile4(a);
  if (t == 128) return launch_tiles4<TO, MODE, 128, 128>(a, b, row_tiles(a.N, a.Ng, true, 128), 8, stream);
  if (t == 64) return launch_tiles4<TO, MODE, 64, 64>(a, b, row_tiles(a.N, a.Ng, true, 64), 16, stream);
  return launch_tiles4<TO, MODE, 32, 32>(a, b, row_tiles(a.N, a.Ng, true, 32), 16, stream);
}

template <typename TO> hipError_t launch_sized44(const GroupArgs& a, const Group4Args& b, hipStream_t stream) {
  const int t = pick_tile4(a);
  if (t == 128) return launch_tiles44<TO, 128, 128, 2, 2, 2>(a, b, row_tiles(a.N, a.Ng, true, 128), 8, stream);
  if (t == 64) return launch_tiles44<TO, 64, 64, 2, 2, 4>(a, b, row_tiles(a.N, a.Ng, true, 64), 16, stream);
  return launch_tiles44<TO, 32, 32, 2, 2, 4>(a, b, row_tiles(a.N, a.Ng, true, 32), 16, stream);
}

}  // namespace

hipError_t launch_group_fwd4(const GroupArgs& a, const Group4Args& b, bool bf16_out, hipStream_t stream) {
  if (b.ys) return bf16_out ? launch_sized44<bf16_t>(a, b, stream) : launch_sized44<float>(a, b, stream);
  return bf16_out ? launch_sized4<bf16_t, kFwd>(a, b, stream) : launch_sized4<float, kFwd>(a, b, stream);
}

hipError_t launch_group_bwd_in4(const GroupArgs& a, const Group4Args& b, bool bf16_out, hipStream_t stream) {
  return bf16_out ? launch_sized4<bf16_t, kBwdIn>(a, b, stream) : launch_sized4<float, kBwdIn>(a, b, stream);
}

}  // namespace cnnlib
