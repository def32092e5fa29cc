// Prints which kernel takes a product with a Ker in 4 bits (csrc/group4_choice.h) on a GPU
// of 256 CUs.  A line of standard input: Nt Np Ng Nc Nk, whether rows are gathered, and the
// lowest bits of the addresses of In (and dOut), KerScales and InScales.  A line of output:
// the picks with bf16 rows, with both in 4 bits and of the gradient, and the runs of
// group4_few where it is picked (else 0).
#include <cstdio>
#include "group4_choice.h"
using namespace cnnlib;
int main() {
  long long Nt, Np, Ng, Nc, Nk;
  int gathered, in, xs, ys;
  const int32_t rows = 0;
  while (scanf("%lld %lld %lld %lld %lld %d %d %d %d", &Nt, &Np, &Ng, &Nc, &Nk, &gathered, &in, &xs, &ys) == 9) {
    const int64_t Nb = (Nc + 31) / 32;
    const uintptr_t base = 4096;
    GroupArgs a = {};
    a.rows = gathered ? &rows : nullptr;
    a.Y = (const void*)(base + in);
    a.ldx = 8 * Nb; a.ldy = Nc; a.ldd = Nk;
    a.M = (int32_t)Nk; a.N = (int32_t)Np; a.K = (int32_t)Nc; a.Ng = (int32_t)Ng; a.Nsrc = (int32_t)Nt;
    Group4Args b = {(const uint8_t*)base + xs, nullptr, (int32_t)Nb};
    const int fwd = group::pick_fwd4(a, b, 256);
    GroupArgs c = a;
    c.Y = (const void*)base;
    c.ldy = 8 * Nb; c.K = (int32_t)(8 * Nb);
    b.ys = (const uint8_t*)base + ys;
    const int both = group::pick_fwd44(c, b, 256);
    GroupArgs d = a;
    d.rows = nullptr;
    d.ldy = Nk; d.ldd = Nc; d.M = (int32_t)Nc; d.K = (int32_t)Nk; d.Nsrc = (int32_t)Np;
    printf("%d %d %d %d\n", fwd, both, group::pick_bwd_in4(d, 256), fwd == 3 ? group::few4_runs((int)Nb) : 0);
  }
  return 0;
}
