// C ABI entry points of the routed contractions (include/cnn.h): argument
// validation and dispatch.  Every check happens before the first HIP call.
#include <hip/hip_runtime.h>
#include <stdarg.h>
#include <stdio.h>

#include <algorithm>

#include "routed.h"

using namespace cnnlib;

namespace {

int fail(int status, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
int fail(int status, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  return set_error(status, buf);
}

int launched(hipError_t e) {
  if (e == hipSuccess) return CNN_OK;
  if (e == hipErrorInvalidConfiguration)
    return fail(CNN_E_OVERFLOW, "more threads than a launch holds");
  return fail(CNN_E_HIP, "kernel launch: %s", hipGetErrorString(e));
}

// No exception leaves the library: host allocations are the only source.
template <typename F> int guarded(F f) {
  try {
    return f();
  } catch (...) {
    return CNN_E_HIP;
  }
}

struct Size {
  const char* name;
  int64_t value, least, most;
};
template <int N> int check_sizes(const Size (&s)[N]) {
  for (int i = 0; i < N; ++i) {
    if (s[i].value < s[i].least)
      return fail(CNN_E_SHAPE, "%s = %lld must be >= %lld", s[i].name, (long long)s[i].value,
                  (long long)s[i].least);
    if (s[i].value > s[i].most)
      return fail(CNN_E_OVERFLOW, "%s = %lld exceeds %lld", s[i].name, (long long)s[i].value,
                  (long long)s[i].most);
  }
  return CNN_OK;
}

constexpr int64_t kRows = 0x3fffffff;      // rows, features: 32-bit indexing with room for a tile
constexpr int64_t kFeatures = 0x3fffffff;
constexpr int64_t kGroups = 65535;
constexpr int64_t kExperts = 1024;         // experts of a router, adapters of a projection
constexpr int64_t kChoices = 16;
constexpr int64_t kRank = 4096;
constexpr int64_t kSequences = 1 << 20;
constexpr int64_t kGrid = 0x7fffffff;

int check_type(int dtype) {
  if (dtype != CNN_F32 && dtype != CNN_BF16 && dtype != CNN_BF16_OBF16)
    return fail(CNN_E_DTYPE, "unknown dtype %d", dtype);
  return CNN_OK;
}

// a b c of sizes >= 0, 2^62 where that or more is due: a product that wrapped
// would pass for a small one.
int64_t product(int64_t a, int64_t b, int64_t c) {
  constexpr int64_t most = 1LL << 62;
  int64_t r;
  if (!a || !b || !c) return 0;
  return __builtin_mul_overflow(a, b, &r) || __builtin_mul_overflow(r, c, &r) || r > most ? most : r;
}

// A tensor argument: NULL is allowed where it holds no element.
struct Buf {
  const char* name;
  const void* p;
  int64_t elems;
  int esize;
};
int check_bufs(const Buf* in, int n_in, const Buf* out, int n_out) {
  for (int i = 0; i < n_in + n_out; ++i) {
    const Buf& b = i < n_in ? in[i] : out[i - n_in];
    if (b.elems >= (1LL << 60)) return fail(CNN_E_OVERFLOW, "%s: element count exceeds 2^60", b.name);
    if (!b.p && b.elems > 0) return fail(CNN_E_NULL, "%s must be non-NULL", b.name);
  }
  for (int i = 0; i < n_out; ++i)
    for (int j = 0; j < n_in + n_out; ++j) {
      if (j == n_in + i) continue;
      const Buf& a = out[i];
      const Buf& b = j < n_in ? in[j] : out[j - n_in];
      if (!a.p || !b.p || !a.elems || !b.elems) continue;
      const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
      if (x < y + (uintptr_t)b.elems * b.esize && y < x + (uintptr_t)a.elems * a.esize)
        return fail(CNN_E_ALIAS, "%s overlaps %s", a.name, b.name);
    }
  return CNN_OK;
}
template <int NI, int NO> int check_bufs(const Buf (&in)[NI], const Buf (&out)[NO]) {
  return check_bufs(in, NI, out, NO);
}

int check_ws(const void* ws, int64_t have, int64_t need) {
  if (!need) return CNN_OK;
  if (!ws) return fail(CNN_E_NULL, "workspace of %lld bytes must be non-NULL", (long long)need);
  if (have < need)
    return fail(CNN_E_SHAPE, "workspace of %lld bytes, %lld needed", (long long)have, (long long)need);
  if ((uintptr_t)ws & 15) return fail(CNN_E_SHAPE, "workspace must be 16-byte aligned");
  return CNN_OK;
}

int check_grid(int64_t n) {
  if (n > kGrid) return fail(CNN_E_OVERFLOW, "%lld workgroups exceed the grid", (long long)n);
  return CNN_OK;
}

// Tiles of the smallest size (16 rows by 16 features, any group split).
int check_tiles(int64_t rows, int64_t groups, int64_t features) {
  return check_grid((rows / 16 + (groups + 1 < rows ? groups + 1 : rows)) * ((features + 15) / 16));
}

int check_route(int64_t Nt, int64_t Ng, int64_t Kt) {
  const Size s[] = {{"Nt", Nt, 0, kRows}, {"Ng", Ng, 1, kExperts}, {"Kt", Kt, 1, kChoices}};
  int st = check_sizes(s);
  if (st) return st;
  if (Kt > Ng) return fail(CNN_E_SHAPE, "Kt = %lld exceeds Ng = %lld", (long long)Kt, (long long)Ng);
  if (Nt * Kt > kRows) return fail(CNN_E_OVERFLOW, "Nt * Kt exceeds %lld", (long long)kRows);
  return CNN_OK;
}

int check_over(int over) {
  if (over != CNN_OVER_ALL && over != CNN_OVER_CHOSEN)
    return fail(CNN_E_UNSUPPORTED, "unknown weights %d", over);
  return CNN_OK;
}

// Tensors in 4 bits: the blocks of a row, codes on 16-byte boundaries.
int64_t blocks4(int64_t Nc) { return (Nc + 31) / 32; }
int check_codes(const char* name, const void* p) {
  if ((uintptr_t)p & 15) return fail(CNN_E_SHAPE, "%s must be 16-byte aligned", name);
  return CNN_OK;
}
// Products of Ker in 4 bits: bf16 rows (or rows in 4 bits), either result.
int check_type4(int dtype) {
  const int st = check_type(dtype);
  if (st) return st;
  if (dtype == CNN_F32) return fail(CNN_E_UNSUPPORTED, "no product of fp32 rows and a Ker in 4 bits");
  return CNN_OK;
}

int check_balance(int64_t Nt, int64_t Ng, int64_t Kt, int64_t Ns, bool bounds) {
  const int st = check_route(Nt, Ng, Kt);
  if (st) return st;
  const Size s[] = {{"Ns", Ns, 1, kSequences}};
  const int su = check_sizes(s);
  if (su) return su;
  if (!bounds && Ns != 1) return fail(CNN_E_SHAPE, "without Bounds, Ns = %lld must be 1", (long long)Ns);
  return CNN_OK;
}

int64_t round16(int64_t n) { return (n + 15) & ~(int64_t)15; }

int64_t route_ws_bytes(int64_t Nt, int64_t Ng) {
  int32_t chunk, nblocks;
  order_blocks(Nt, &chunk, &nblocks);
  return nblocks > 1 ? round16((int64_t)nblocks * Ng * 4) : 0;
}

// The adapted projection's workspace: few rows, the slices' sums; many, H and
// the order of the rows.
struct AdaptWs {
  int64_t few_h, h, counts, off, rows, total;
};
// For every type and alignment: whichever way the rows are taken, it fits.
AdaptWs adapt_ws(int64_t Nt, int64_t Nc, int64_t Nk, int64_t Na, int64_t Nl) {
  AdaptWs w = {};
  int64_t few = 0, ordered = 0;
  if (Nt <= kFewRows) {
    const FewPlan f = adapt_few_plan(Nt, Nc, Nk, 4);  // bf16 has no more slices
    w.few_h = round16(f.kh * Nt * Nl * 4);
    few = w.few_h + round16(f.ks * Nt * Nk * 4);
  }
  if (!adapt_few(Nt, Nc, Nk, true) || !adapt_few(Nt, Nc, Nk, false)) {
    int32_t chunk, nblocks;
    order_blocks(Nt, &chunk, &nblocks);
    w.h = round16(Nt * adapt_nlp(Nl, CNN_BF16) * 6);  // three bf16 parts, or fp32
    w.counts = round16((int64_t)nblocks * Na * 4);
    w.off = round16((Na + 1) * 4);
    w.rows = round16(Nt * 4);
    ordered = w.h + w.counts + w.off + 2 * w.rows;
  }
  w.total = few > ordered ? few : ordered;
  return w;
}

int check_adapt(int64_t Nt, int64_t Nc, int64_t Nk, int64_t Na, int64_t Nl) {
  const Size s[] = {{"Nt", Nt, 0, kRows}, {"Nc", Nc, 1, kFeatures}, {"Nk", Nk, 1, kFeatures},
                    {"Na", Na, 1, kExperts}, {"Nl", Nl, 1, kRank}};
  return check_sizes(s);
}

int check_group(int64_t Nt, int64_t Np, int64_t Ng, int64_t Nc, int64_t Nk, bool gathered) {
  const Size s[] = {{"Nt", Nt, 0, kRows}, {"Np", Np, 0, kRows}, {"Ng", Ng, 1, kGroups},
                    {"Nc", Nc, 1, kFeatures}, {"Nk", Nk, 1, kFeatures}};
  int st = check_sizes(s);
  if (st) return st;
  if (!gathered && Nt != Np)
    return fail(CNN_E_SHAPE, "without Rows, Nt = %lld must equal Np = %lld", (long long)Nt, (long long)Np);
  if (Np > 0 && Nt == 0) return fail(CNN_E_SHAPE, "Np = %lld rows of an empty In", (long long)Np);
  return CNN_OK;
}

}  // namespace

extern "C" {

int cnn_route_ws(int64_t Nt, int64_t Ng, int64_t Kt, int64_t* ws_bytes) {
  return guarded([&] {
    if (!ws_bytes) return fail(CNN_E_NULL, "ws_bytes must be non-NULL");
    int st = check_route(Nt, Ng, Kt);
    if (st) return st;
    *ws_bytes = route_ws_bytes(Nt, Ng);
    return (int)CNN_OK;
  });
}

int cnn_route(const void* Logits, int32_t* Choice, float* Gates, int32_t* Offsets, int32_t* Rows,
              int32_t* Slots, int64_t Nt, int64_t Ng, int64_t Kt, int dtype, int over,
              void* workspace, int64_t ws_bytes, void* stream) {
  return guarded([&] {
    int st;
    if ((st = check_route(Nt, Ng, Kt)) || (st = check_type(dtype)) || (st = check_over(over))) return st;
    const int64_t need = route_ws_bytes(Nt, Ng);
    const Buf in[] = {{"Logits", Logits, Nt * Ng, in_bytes(dtype)}};
    const Buf out[] = {{"Choice", Choice, Nt * Kt, 4}, {"Gates", Gates, Nt * Kt, 4},
                       {"Offsets", Offsets, Ng + 1, 4}, {"Rows", Rows, Nt * Kt, 4},
                       {"Slots", Slots, Nt * Kt, 4}, {"workspace", workspace, need, 1}};
    if ((st = check_ws(workspace, ws_bytes, need)) || (st = check_bufs(in, out))) return st;
    OrderArgs o = {};
    o.key = Choice;
    o.off = Offsets;
    o.rows = Rows;
    o.slots = Slots;
    o.counts = (int32_t*)workspace;
    o.Nt = (int32_t)Nt;
    o.Ng = (int32_t)Ng;
    o.Kt = (int32_t)Kt;
    order_blocks(Nt, &o.chunk, &o.nblocks);
    const RouteArgs a = {Logits, Gates, Choice, over == CNN_OVER_ALL};
    return launched(launch_route(a, o, dtype != CNN_F32, (hipStream_t)stream));
  });
}

int cnn_route_bwd(const void* Logits, const int32_t* Choice, const float* Gates,
                  const float* dGates, void* dLogits, int64_t Nt, int64_t Ng, int64_t Kt,
                  int dtype, int over, void* stream) {
  return guarded([&] {
    int st;
    if ((st = check_route(Nt, Ng, Kt)) || (st = check_type(dtype)) || (st = check_over(over))) return st;
    const Buf in[] = {{"Logits", Logits, Nt * Ng, in_bytes(dtype)}, {"Choice", Choice, Nt * Kt, 4},
                      {"Gates", Gates, Nt * Kt, 4}, {"dGates", dGates, Nt * Kt, 4}};
    const Buf out[] = {{"dLogits", dLogits, Nt * Ng, out_bytes(dtype)}};
    if ((st = check_bufs(in, out))) return st;
    if (!Nt) return (int)CNN_OK;
    return launched(launch_route_bwd(Logits, Choice, Gates, dGates, dLogits, Nt, (int)Ng, (int)Kt,
                                     dtype, over == CNN_OVER_ALL, (hipStream_t)stream));
  });
}

static int check_combine(int64_t Nt, int64_t Kt, int64_t Np, int64_t Nk, int dtype) {
  const Size s[] = {{"Nt", Nt, 0, kRows}, {"Kt", Kt, 1, kGroups}, {"Np", Np, 0, kRows},
                    {"Nk", Nk, 1, kFeatures}};
  int st;
  if ((st = check_sizes(s)) || (st = check_type(dtype))) return st;
  return check_grid(std::max(Nt * ((Nk + 3) / 4) / 256 + 1, Np + Nt * Kt / 256 + 2));
}

int cnn_combine(const void* In, const int32_t* Slots, const float* Gates, void* Out, int64_t Nt,
                int64_t Kt, int64_t Np, int64_t Nk, int dtype, void* stream) {
  return guarded([&] {
    int st = check_combine(Nt, Kt, Np, Nk, dtype);
    if (st) return st;
    const Buf in[] = {{"In", In, Np * Nk, in_bytes(dtype)}, {"Slots", Slots, Nt * Kt, 4},
                      {"Gates", Gates, Gates ? Nt * Kt : 0, 4}};
    const Buf out[] = {{"Out", Out, Nt * Nk, out_bytes(dtype)}};
    if ((st = check_bufs(in, out))) return st;
    if (!Nt) return (int)CNN_OK;
    return launched(launch_combine(In, Slots, Gates, Out, Nt, (int)Kt, Np, Nk, dtype,
                                   (hipStream_t)stream));
  });
}

int cnn_combine_bwd(const void* dOut, const void* In, const int32_t* Slots, const int32_t* Rows,
                    const float* Gates, void* dIn, float* dGates, int64_t Nt, int64_t Kt,
                    int64_t Np, int64_t Nk, int dtype, void* stream) {
  return guarded([&] {
    int st = check_combine(Nt, Kt, Np, Nk, dtype);
    if (st) return st;
    const Buf in[] = {{"dOut", dOut, Nt * Nk, in_bytes(dtype)}, {"In", In, Np * Nk, in_bytes(dtype)},
                      {"Slots", Slots, Nt * Kt, 4}, {"Rows", Rows, Np, 4},
                      {"Gates", Gates, Gates ? Nt * Kt : 0, 4}};
    const Buf out[] = {{"dIn", dIn, Np * Nk, out_bytes(dtype)},
                       {"dGates", dGates, dGates ? Nt * Kt : 0, 4}};
    if ((st = check_bufs(in, out))) return st;
    if (!Nt && !Np) return (int)CNN_OK;
    return launched(launch_combine_bwd(dOut, In, Slots, Rows, Gates, dIn, dGates, Nt, (int)Kt, Np,
                                       Nk, dtype, (hipStream_t)stream));
  });
}

int cnn_group_fwd(const void* In, const void* Ker, void* Out, const int32_t* Offsets,
                  const int32_t* Rows, int64_t Nt, int64_t Np, int64_t Ng, int64_t Nc, int64_t Nk,
                  int dtype, void* stream) {
  return guarded([&] {
    int st;
    if ((st = check_group(Nt, Np, Ng, Nc, Nk, Rows != nullptr)) || (st = check_type(dtype)) ||
        (st = check_tiles(Np, Ng, Nk)))
      return st;
    const Buf in[] = {{"In", In, Nt * Nc, in_bytes(dtype)}, {"Ker", Ker, product(Ng, Nk, Nc), in_bytes(dtype)},
                      {"Offsets", Offsets, Ng + 1, 4}, {"Rows", Rows, Rows ? Np : 0, 4}};
    const Buf out[] = {{"Out", Out, Np * Nk, out_bytes(dtype)}};
    if ((st = check_bufs(in, out))) return st;
    if (!Np) return (int)CNN_OK;
    GroupArgs a = {};
    a.X = Ker; a.Y = In; a.D = Out;
    a.off = Offsets; a.rows = Rows;
    a.ldx = Nc; a.ldy = Nc; a.ldd = Nk;
    a.xgroup = Nk * Nc;
    a.M = (int32_t)Nk; a.N = (int32_t)Np; a.K = (int32_t)Nc;
    a.Ng = (int32_t)Ng; a.Nsrc = (int32_t)Nt;
    return launched(launch_group_fwd(a, dtype, (hipStream_t)stream));
  });
}

int cnn_group_bwd_in(const void* dOut, const void* Ker, void* dIn, const int32_t* Offsets,
                     int64_t Np, int64_t Ng, int64_t Nc, int64_t Nk, int dtype, void* stream) {
  return guarded([&] {
    int st;
    if ((st = check_group(Np, Np, Ng, Nc, Nk, false)) || (st = check_type(dtype)) ||
        (st = check_tiles(Np, Ng, Nc)))
      return st;
    const Buf in[] = {{"dOut", dOut, Np * Nk, in_bytes(dtype)}, {"Ker", Ker, product(Ng, Nk, Nc), in_bytes(dtype)},
                      {"Offsets", Offsets, Ng + 1, 4}};
    const Buf out[] = {{"dIn", dIn, Np * Nc, out_bytes(dtype)}};
    if ((st = check_bufs(in, out))) return st;
    if (!Np) return (int)CNN_OK;
    GroupArgs a = {};
    a.X = Ker; a.Y = dOut; a.D = dIn;
    a.off = Offsets;
    a.ldx = Nc; a.ldy = Nk; a.ldd = Nc;
    a.xgroup = Nk * Nc;
    a.M = (int32_t)Nc; a.N = (int32_t)Np; a.K = (int32_t)Nk;
    a.Ng = (int32_t)Ng; a.Nsrc = (int32_t)Np;
    return launched(launch_group_bwd_in(a, dtype, (hipStream_t)stream));
  });
}

int cnn_group_bwd_ker(const void* dOut, const void* In, void* dKer, const int32_t* Offsets,
                      const int32_t* Rows, int64_t Nt, int64_t Np, int64_t Ng, int64_t Nc,
                      int64_t Nk, int dtype, void* stream) {
  return guarded([&] {
    int st;
    if ((st = check_group(Nt, Np, Ng, Nc, Nk, Rows != nullptr)) || (st = check_type(dtype)) ||
        (st = check_grid(product(Ng, (Nk + 63) / 64, (Nc + 63) / 64))))
      return st;
    const Buf in[] = {{"dOut", dOut, Np * Nk, in_bytes(dtype)}, {"In", In, Nt * Nc, in_bytes(dtype)},
                      {"Offsets", Offsets, Ng + 1, 4}, {"Rows", Rows, Rows ? Np : 0, 4}};
    const Buf out[] = {{"dKer", dKer, product(Ng, Nk, Nc), out_bytes(dtype)}};
    if ((st = check_bufs(in, out))) return st;
    GroupArgs a = {};
    a.X = In; a.Y = dOut; a.D = dKer;
    a.off = Offsets; a.rows = Rows;
    a.ldx = Nc; a.ldy = Nk; a.ldd = Nc;
    a.dgroup = Nk * Nc;
    a.M = (int32_t)Nc; a.N = (int32_t)Nk; a.K = (int32_t)Np;
    a.Ng = (int32_t)Ng; a.Nsrc = (int32_t)Nt;
    return launched(launch_group_bwd_ker(a, dtype, (hipStream_t)stream));
  });
}

int cnn_quantize4(const void* In, uint8_t* Codes, uint8_t* Scales, int64_t Nt, int64_t Nc, int dtype,
                  int rule, void* stream) {
  return guarded([&] {
    const Size s[] = {{"Nt", Nt, 0, kRows}, {"Nc", Nc, 1, kFeatures}};
    int st;
    if ((st = check_sizes(s)) || (st = check_type(dtype))) return st;
    if (rule != CNN_SCALE_FLOOR && rule != CNN_SCALE_UP) return fail(CNN_E_UNSUPPORTED, "unknown rule %d", rule);
    const Buf in[] = {{"In", In, Nt * Nc, in_bytes(dtype)}};
    const Buf out[] = {{"Codes", Codes, Nt * blocks4(Nc) * 16, 1}, {"Scales", Scales, Nt * blocks4(Nc), 1}};
    if ((st = check_codes("Codes", Codes)) || (st = check_bufs(in, out))) return st;
    if (!Nt) return (int)CNN_OK;
    return launched(launch_quantize4(In, Codes, Scales, Nt, Nc, dtype != CNN_F32, rule == CNN_SCALE_UP,
                                     (hipStream_t)stream));
  });
}

int cnn_dequantize4(const uint8_t* Codes, const uint8_t* Scales, void* Out, int64_t Nt, int64_t Nc,
                    int dtype, void* stream) {
  return guarded([&] {
    const Size s[] = {{"Nt", Nt, 0, kRows}, {"Nc", Nc, 1, kFeatures}};
    int st;
    if ((st = check_sizes(s)) || (st = check_type(dtype))) return st;
    const Buf in[] = {{"Codes", Codes, Nt * blocks4(Nc) * 16, 1}, {"Scales", Scales, Nt * blocks4(Nc), 1}};
    const Buf out[] = {{"Out", Out, Nt * Nc, in_bytes(dtype)}};
    if ((st = check_codes("Codes", Codes)) || (st = check_bufs(in, out))) return st;
    if (!Nt) return (int)CNN_OK;
    return launched(launch_dequantize4(Codes, Scales, Out, Nt, Nc, dtype != CNN_F32, (hipStream_t)stream));
  });
}

int cnn_group_fwd4(const void* In, const uint8_t* InScales, const uint8_t* Ker, const uint8_t* KerScales,
                   void* Out, const int32_t* Offsets, const int32_t* Rows, int64_t Nt, int64_t Np,
                   int64_t Ng, int64_t Nc, int64_t Nk, int dtype, void* stream) {
  return guarded([&] {
    int st;
    if ((st = check_group(Nt, Np, Ng, Nc, Nk, Rows != nullptr)) || (st = check_type4(dtype)) ||
        (st = check_tiles(Np, Ng, Nk)))
      return st;
    const int64_t Nb = blocks4(Nc);
    const Buf in[] = {{"In", In, InScales ? Nt * Nb * 16 : Nt * Nc, InScales ? 1 : 2},
                      {"InScales", InScales, InScales ? Nt * Nb : 0, 1},
                      {"Ker", Ker, product(Ng, Nk, 16 * Nb), 1}, {"KerScales", KerScales, product(Ng, Nk, Nb), 1},
                      {"Offsets", Offsets, Ng + 1, 4}, {"Rows", Rows, Rows ? Np : 0, 4}};
    const Buf out[] = {{"Out", Out, Np * Nk, out_bytes(dtype)}};
    if ((st = check_codes("Ker", Ker)) || (InScales && (st = check_codes("In", In))) ||
        (st = check_bufs(in, out)))
      return st;
    if (!Np) return (int)CNN_OK;
    GroupArgs a = {};
    a.X = Ker; a.Y = In; a.D = Out;
    a.off = Offsets; a.rows = Rows;
    a.ldx = 8 * Nb; a.ldy = InScales ? 8 * Nb : Nc; a.ldd = Nk;  // codes as 16-bit words
    a.xgroup = Nk * 8 * Nb;
    a.M = (int32_t)Nk; a.N = (int32_t)Np; a.K = (int32_t)(InScales ? 8 * Nb : Nc);
    a.Ng = (int32_t)Ng; a.Nsrc = (int32_t)Nt;
    const Group4Args b = {KerScales, InScales, (int32_t)Nb};
    return launched(launch_group_fwd4(a, b, dtype == CNN_BF16_OBF16, (hipStream_t)stream));
  });
}

int cnn_group_bwd_in4(const void* dOut, const uint8_t* Ker, const uint8_t* KerScales, void* dIn,
                      const int32_t* Offsets, int64_t Np, int64_t Ng, int64_t Nc, int64_t Nk, int dtype,
                      void* stream) {
  return guarded([&] {
    int st;
    if ((st = check_group(Np, Np, Ng, Nc, Nk, false)) || (st = check_type4(dtype)) ||
        (st = check_tiles(Np, Ng, Nc)))
      return st;
    const int64_t Nb = blocks4(Nc);
    const Buf in[] = {{"dOut", dOut, Np * Nk, 2}, {"Ker", Ker, product(Ng, Nk, 16 * Nb), 1},
                      {"KerScales", KerScales, product(Ng, Nk, Nb), 1}, {"Offsets", Offsets, Ng + 1, 4}};
    const Buf out[] = {{"dIn", dIn, Np * Nc, out_bytes(dtype)}};
    if ((st = check_codes("Ker", Ker)) || (st = check_bufs(in, out))) return st;
    if (!Np) return (int)CNN_OK;
    GroupArgs a = {};
    a.X = Ker; a.Y = dOut; a.D = dIn;
    a.off = Offsets;
    a.ldx = 8 * Nb; a.ldy = Nk; a.ldd = Nc;
    a.xgroup = Nk * 8 * Nb;
    a.M = (int32_t)Nc; a.N = (int32_t)Np; a.K = (int32_t)Nk;
    a.Ng = (int32_t)Ng; a.Nsrc = (int32_t)Np;
    const Group4Args b = {KerScales, nullptr, (int32_t)Nb};
    return launched(launch_group_bwd_in4(a, b, dtype == CNN_BF16_OBF16, (hipStream_t)stream));
  });
}

int cnn_balance_ws(int64_t Nt, int64_t Ng, int64_t Ns, int64_t* ws_bytes) {
  return guarded([&] {
    if (!ws_bytes) return fail(CNN_E_NULL, "ws_bytes must be non-NULL");
    const int st = check_balance(Nt, Ng, 1, Ns, true);
    if (st) return st;
    *ws_bytes = balance_ws_bytes(Nt, Ng, Ns);
    return (int)CNN_OK;
  });
}

int cnn_balance(const void* Logits, const int32_t* Choice, const int32_t* Bounds, int32_t* Counts,
                int32_t* Tokens, float* Loss, int64_t Nt, int64_t Ng, int64_t Kt, int64_t Ns, int dtype,
                void* workspace, int64_t ws_bytes, void* stream) {
  return guarded([&] {
    int st;
    if ((st = check_balance(Nt, Ng, Kt, Ns, Bounds != nullptr)) || (st = check_type(dtype))) return st;
    const int64_t need = balance_ws_bytes(Nt, Ng, Ns);
    const Buf in[] = {{"Logits", Logits, Nt * Ng, in_bytes(dtype)}, {"Choice", Choice, Nt * Kt, 4},
                      {"Bounds", Bounds, Bounds ? Ns + 1 : 0, 4}};
    const Buf out[] = {{"Counts", Counts, Ns * Ng, 4}, {"Tokens", Tokens, Ns, 4}, {"Loss", Loss, 2, 4},
                       {"workspace", workspace, need, 1}};
    if ((st = check_ws(workspace, ws_bytes, need)) || (st = check_bufs(in, out))) return st;
    BalanceArgs a = {};
    a.logits = Logits; a.choice = Choice; a.bounds = Bounds;
    a.counts = Counts; a.tokens = Tokens; a.loss = Loss;
    a.ws = workspace;
    a.Nt = (int32_t)Nt; a.Ng = (int32_t)Ng; a.Kt = (int32_t)Kt; a.Ns = (int32_t)Ns;
    order_blocks(Nt, &a.chunk, &a.nblocks);
    return launched(launch_balance(a, dtype != CNN_F32, (hipStream_t)stream));
  });
}

int cnn_balance_bwd(const void* Logits, const int32_t* Choice, const int32_t* Bounds,
                    const int32_t* Counts, const int32_t* Tokens, const float* dLoss, void* dLogits,
                    int64_t Nt, int64_t Ng, int64_t Kt, int64_t Ns, int dtype, int add, void* stream) {
  return guarded([&] {
    int st;
    if ((st = check_balance(Nt, Ng, Kt, Ns, Bounds != nullptr)) || (st = check_type(dtype))) return st;
    const Buf in[] = {{"Logits", Logits, Nt * Ng, in_bytes(dtype)}, {"Choice", Choice, Nt * Kt, 4},
                      {"Bounds", Bounds, Bounds ? Ns + 1 : 0, 4}, {"Counts", Counts, Ns * Ng, 4},
                      {"Tokens", Tokens, Ns, 4}, {"dLoss", dLoss, 2, 4}};
    const Buf out[] = {{"dLogits", dLogits, Nt * Ng, out_bytes(dtype)}};
    if ((st = check_bufs(in, out))) return st;
    if (!Nt) return (int)CNN_OK;
    BalanceArgs a = {};
    a.logits = Logits; a.choice = Choice; a.bounds = Bounds;
    a.counts = const_cast<int32_t*>(Counts); a.tokens = const_cast<int32_t*>(Tokens);
    a.dloss = dLoss; a.dlogits = dLogits;
    a.Nt = (int32_t)Nt; a.Ng = (int32_t)Ng; a.Kt = (int32_t)Kt; a.Ns = (int32_t)Ns;
    return launched(launch_balance_bwd(a, dtype, add != 0, (hipStream_t)stream));
  });
}

int cnn_adapt_ws(int64_t Nt, int64_t Nc, int64_t Nk, int64_t Na, int64_t Nl, int64_t* ws_bytes) {
  return guarded([&] {
    if (!ws_bytes) return fail(CNN_E_NULL, "ws_bytes must be non-NULL");
    int st = check_adapt(Nt, Nc, Nk, Na, Nl);
    if (st) return st;
    *ws_bytes = adapt_ws(Nt, Nc, Nk, Na, Nl).total;
    return (int)CNN_OK;
  });
}

int cnn_adapt_fwd(const void* In, const void* Ker, const void* A, const void* B,
                  const int32_t* Ids, const float* Scales, void* Out, int64_t Nt, int64_t Nc,
                  int64_t Nk, int64_t Na, int64_t Nl, int dtype, void* workspace,
                  int64_t ws_bytes, void* stream) {
  return guarded([&] {
    int st;
    if ((st = check_adapt(Nt, Nc, Nk, Na, Nl)) || (st = check_type(dtype)) ||
        (st = check_tiles(Nt, Na, Nk)))
      return st;
    const AdaptWs w = adapt_ws(Nt, Nc, Nk, Na, Nl);
    const int es = in_bytes(dtype);
    const Buf in[] = {{"In", In, Nt * Nc, es}, {"Ker", Ker, Nk * Nc, es}, {"A", A, product(Na, Nl, Nc), es},
                      {"B", B, product(Na, Nk, Nl), es}, {"Ids", Ids, Nt, 4},
                      {"Scales", Scales, Scales ? Na : 0, 4}};
    const Buf out[] = {{"Out", Out, Nt * Nk, out_bytes(dtype)}, {"workspace", workspace, w.total, 1}};
    if ((st = check_ws(workspace, ws_bytes, w.total)) || (st = check_bufs(in, out))) return st;
    if (!Nt) return (int)CNN_OK;
    char* p = (char*)workspace;
    GroupArgs a = {};
    a.X = Ker; a.Y = In; a.D = Out;
    a.ldx = Nc; a.ldy = Nc; a.ldd = Nk;
    a.M = (int32_t)Nk; a.N = (int32_t)Nt; a.K = (int32_t)Nc;
    a.Ng = 1; a.Nsrc = (int32_t)Nt;
    AdaptArgs ad = {};
    ad.A = A; ad.B = B; ad.ids = Ids; ad.scales = Scales;
    ad.Na = (int32_t)Na; ad.Nl = (int32_t)Nl;
    if (adapt_few(Nt, Nc, Nk, adapt_few_ring(Ker, In, Nc, es))) {
      ad.H = (float*)p;
      ad.part = (float*)(p + w.few_h);
      return launched(launch_adapt_few(a, ad, dtype, (hipStream_t)stream));
    }
    ad.Hp = p;
    ad.nlp = adapt_nlp(Nl, dtype);
    ad.hl = ad.nlp * adapt_parts(dtype);
    if ((st = launched(launch_adapt(a, ad, dtype, Launch{nullptr, true})))) return st;
    OrderArgs o = {};
    o.key = Ids;
    o.counts = (int32_t*)(p += w.h);
    o.off = (int32_t*)(p += w.counts);
    o.rows = (int32_t*)(p += w.off);
    o.keys = (int32_t*)(p += w.rows);
    o.Nt = (int32_t)Nt;
    o.Ng = (int32_t)Na;
    o.Kt = 1;
    o.place_none = 1;
    order_blocks(Nt, &o.chunk, &o.nblocks);
    if ((st = launched(launch_order(o, (hipStream_t)stream)))) return st;
    a.off = o.off;
    a.rows = o.rows;
    ad.ids = o.keys;
    return launched(launch_adapt(a, ad, dtype, Launch{(hipStream_t)stream, false}));
  });
}

}  // extern "C"
