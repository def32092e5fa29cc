// Launches of the grouped products whose Ker lies in 4 bits.
#include "group4_choice.h"
#include "group4_pipe.h"

namespace cnnlib {

namespace {

using namespace group;

int64_t tiles_of(const GroupArgs& a, int tn) { return row_tiles(a.N, a.Ng, true, tn); }

template <typename TO> hipError_t launch_fwd4(const GroupArgs& a, const Group4Args& b, hipStream_t stream) {
  constexpr bool OB = sizeof(TO) == 2;
  const int pick = pick_fwd4(a, b, device_cus());
  switch (pick) {
    case kShort4: return launch_tiles4<TO, kFwd, 64, 32, false>(a, b, tiles_of(a, 32), 16, stream);
    case 0: return launch_tiles4<TO, kFwd, 64, 32>(a, b, tiles_of(a, 32), 16, stream);
    case 1: return launch_tiles4<TO, kFwd, 64, 64>(a, b, tiles_of(a, 64), 16, stream);
    case 2: return launch_tiles4<TO, kFwd, 128, 128>(a, b, tiles_of(a, 128), 8, stream);
    case 3: return launch_group4_few(a, b, OB, stream);
    case 7: return launch_pipe4<TO, kFwd>(a, b, tiles_of(a, 256), 4, stream);
    default: return launch_group4_rows(a, b, OB, pick == 4 ? 16 : pick == 5 ? 32 : 64, stream);
  }
}

template <typename TO> hipError_t launch_fwd44(const GroupArgs& a, const Group4Args& b, hipStream_t stream) {
  // rings: more workgroups on a CU do more than more stages of each (1536 rows of 60
  // groups of 1536 x 2048 in 128 x 32 tiles, four stages, three, two: 36, 34 and 33 us with
  // the quantisation), but a lone one wants them
  switch (pick_fwd44(a, b, device_cus())) {
    case kShort4: return launch_tiles44<TO, 64, 32, 2, 2, 4, false>(a, b, tiles_of(a, 32), 16, stream);
    case 0: return launch_tiles44<TO, 32, 32, 2, 2, 4>(a, b, tiles_of(a, 32), 16, stream);
    case 1: return launch_tiles44<TO, 64, 32, 2, 2, 4>(a, b, tiles_of(a, 32), 16, stream);
    case 2: return launch_tiles44<TO, 128, 32, 4, 1, 3>(a, b, tiles_of(a, 32), 16, stream);
    case 3: return launch_tiles44<TO, 128, 64, 4, 1, 3>(a, b, tiles_of(a, 64), 16, stream);
    case 4: return launch_tiles44<TO, 128, 128, 2, 2, 2>(a, b, tiles_of(a, 128), 8, stream);
    default: return launch_pipe44<TO>(a, b, tiles_of(a, 256), 4, stream);
  }
}

template <typename TO> hipError_t launch_bwd_in4(const GroupArgs& a, const Group4Args& b, hipStream_t stream) {
  switch (pick_bwd_in4(a, device_cus())) {
    case kShort4: return launch_tiles4<TO, kBwdIn, 64, 32, false>(a, b, tiles_of(a, 32), 16, stream);
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
