// Host check of the half blocks that a stage of the products through registers reads of
// a row of codes and scales (csrc/group4_kernel.h): over rows of 1 to 9 blocks and the
// stages in flight past the last one too, every byte lies within the row, and a half block
// of the row is read where it lies.  Exits 1 on any mismatch.
#include <cstdio>
#include "group4_kernel.h"
using namespace cnnlib::group;
int main() {
  long n = 0, bad = 0;
  for (int Nb = 1; Nb <= 9; ++Nb)
    for (int k0 = 0; k0 <= 32 * Nb + 64 * 5; k0 += 64)
      for (int q = 0; q < 4; ++q) {
        const int base = half_base(q, Nb), step = half_step(16 * q, k0, 32 * Nb);
        const int code = base / 2 + (step >> 1), scale = base / 32 + (step >> 5);
        ++n;
        bool ok = code >= 0 && code + 8 <= 16 * Nb && scale >= 0 && scale < Nb;
        if (k0 + 16 * q < 32 * Nb) ok = ok && code == (k0 + 16 * q) / 2 && scale == (k0 + 16 * q) / 32;
        if (!ok) {
          ++bad;
          printf("blocks %d stage at %d half block %d: code byte %d of %d, scale %d\n", Nb, k0, q, code, 16 * Nb, scale);
        }
      }
  printf("checked %ld bad %ld\n", n, bad);
  return bad != 0;
}
