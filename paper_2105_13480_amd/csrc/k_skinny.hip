// Products of few rows: grouped products with a few rows a group, and adapted
// projections of up to a few dozen rows (serving steps).
//
// Such a product is bound by reading Ker once: a workgroup takes 16 features
// by 16 RB rows, its waves share the contraction (wave w takes every NW-th
// 256-byte run of k), and both operands go straight from memory to the MFMA
// registers, no LDS and no barrier until the waves' sums meet: 16 rows of 64
// bytes a load, four loads a run.  Rows beyond a tile's last read a row that
// is there; their results are not stored.
#include "group_kernel.h"

namespace cnnlib {

namespace {

using namespace group;

// acc[f][b] += the 16 features of block f by the 16 rows of block b, over the
// runs of k that `wave` of `nw` takes in [k_lo, k_hi).  x, y: this lane's
// feature row (l % 16) and row of each block.
template <typename T, int FB, int RB>
__device__ __forceinline__ void few_rows_dot(const T* const (&x)[FB], const T* const (&y)[RB],
                                             int k_lo, int k_hi, int wave, int nw, int lane,
                                             f32x4_t (&acc)[FB][RB]) {
  constexpr int CE = 16 / (int)sizeof(T);
  constexpr int RUN = 16 * CE;
  const int G = lane >> 4;
  int k0 = k_lo + wave * RUN;
  for (; k0 + RUN <= k_hi; k0 += nw * RUN) {
    u32x4_t xf[FB][4], yf[RB][4];
#pragma unroll
    for (int f = 0; f < FB; ++f)
#pragma unroll
      for (int i = 0; i < 4; ++i) __builtin_memcpy(&xf[f][i], x[f] + k0 + (4 * i + G) * CE, 16);
#pragma unroll
    for (int b = 0; b < RB; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) __builtin_memcpy(&yf[b][i], y[b] + k0 + (4 * i + G) * CE, 16);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int f = 0; f < FB; ++f)
#pragma unroll
        for (int b = 0; b < RB; ++b) acc[f][b] = mma<T>(xf[f][i], yf[b][i], acc[f][b]);
  }
  if (k0 < k_hi) {  // the last, shorter run: what lies past k_hi is zero on both sides
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int k = k0 + (4 * i + G) * CE;
      u32x4_t xt[FB], yt[RB];
#pragma unroll
      for (int f = 0; f < FB; ++f) xt[f] = load_unit(x[f] + k, k_hi - k);
#pragma unroll
      for (int b = 0; b < RB; ++b) yt[b] = load_unit(y[b] + k, k_hi - k);
#pragma unroll
      for (int f = 0; f < FB; ++f)
#pragma unroll
        for (int b = 0; b < RB; ++b) acc[f][b] = mma<T>(xt[f], yt[b], acc[f][b]);
    }
  }
}

// The waves' sums in wave order: wave w returns the total of block w (f * RB
// + b), for w < FB * RB.  red: NW * FB * RB * 64 units.
template <int FB, int RB>
__device__ __forceinline__ f32x4_t sum_waves(f32x4_t* red, const f32x4_t (&acc)[FB][RB], int wave,
                                             int nw, int lane) {
#pragma unroll
  for (int f = 0; f < FB; ++f)
#pragma unroll
    for (int b = 0; b < RB; ++b) red[((f * RB + b) * nw + wave) * 64 + lane] = acc[f][b];
  __syncthreads();
  f32x4_t s = {0.f, 0.f, 0.f, 0.f};
  if (wave < FB * RB)
    for (int w = 0; w < nw; ++w) s += red[(wave * nw + w) * 64 + lane];
  return s;
}

constexpr int NW = 8;  // waves of a workgroup

template <typename T, typename TO, int RB>
__global__ __launch_bounds__(64 * NW) void group_few(GroupArgs a) {
  __shared__ f32x4_t red[NW * RB * 64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int MT = (a.M + 15) / 16;
  RowTile t;
  if (!find_tile<16 * RB>(a.off, a.Ng, a.N, MT, blockIdx.x, 1, &t)) return;
  const int l16 = lane & 15, G = lane >> 4;
  const int m0 = 16 * t.mt, n_valid = min(t.n1 - t.n0, 16 * RB);
  const bool live = t.g < a.Ng;

  const T* const X = reinterpret_cast<const T*>(a.X) + (live ? t.g : 0) * a.xgroup;
  const T* x[1] = {X + (int64_t)min(m0 + l16, a.M - 1) * a.ldx};
  const T* y[RB];
  uint32_t none = 0;  // blocks whose row of this lane is no row of In
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    int64_t r = t.n0 + min(16 * b + l16, n_valid - 1);
    if (a.rows) r = a.rows[r];
    if (r < 0 || r >= a.Nsrc) {
      none |= 1u << b;
      r = 0;
    }
    y[b] = reinterpret_cast<const T*>(a.Y) + r * a.ldy;
  }
  f32x4_t acc[1][RB];
#pragma unroll
  for (int b = 0; b < RB; ++b) acc[0][b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  if (live) few_rows_dot<T, 1, RB>(x, y, 0, a.K, wave, NW, lane, acc);
  f32x4_t s = sum_waves<1, RB>(red, acc, wave, NW, lane);

  const bool whole = ((uintptr_t)a.D & (4 * sizeof(TO) - 1)) == 0 && (a.ldd & 3) == 0;
  const int n = 16 * wave + l16;
  if (wave < RB && n < n_valid) {
    if (!live || (none >> wave & 1)) s = f32x4_t{0.f, 0.f, 0.f, 0.f};
    store4(reinterpret_cast<TO*>(a.D) + (t.n0 + n) * a.ldd, m0 + 4 * G, a.M, s, whole);
  }
}

// H[z][n][r] = sum over slice z of k of In[n, k] A[ids[n]][r, k] for the rows
// of a tile of 16: workgroup (tile, q, z) takes every Q-th of the adapters that
// the tile's rows name, 16 FB ranks at a time.
template <typename T, int FB>
__global__ __launch_bounds__(64 * NW) void adapt_few_down(GroupArgs a, AdaptArgs ad, int kslice) {
  __shared__ f32x4_t red[NW * FB * 64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, G = lane >> 4;
  const int n0 = 16 * blockIdx.x, n_valid = min(a.N - n0, 16);
  const int k_lo = blockIdx.z * kslice, k_hi = min(a.K, k_lo + kslice);
  const int n = n0 + min(l16, n_valid - 1);
  const int id = ad.ids[n];
  const T* y[1] = {reinterpret_cast<const T*>(a.Y) + (int64_t)n * a.ldy};
  float* const H = ad.H + (int64_t)blockIdx.z * a.N * ad.Nl;

  int last = -1;
  for (int q = 0;; ++q) {
    int next = id > last && id < ad.Na ? id : 0x7fffffff;
#pragma unroll
    for (int d = 8; d >= 1; d >>= 1) next = min(next, __shfl_xor(next, d));
    next = __builtin_amdgcn_readfirstlane(next);
    if (next == 0x7fffffff) break;
    last = next;
    if (q % (int)gridDim.y != (int)blockIdx.y) continue;
    const T* const A = reinterpret_cast<const T*>(ad.A) + (int64_t)next * ad.Nl * a.K;
    for (int r0 = 0; r0 < ad.Nl; r0 += 16 * FB) {
      const T* x[FB];
      f32x4_t acc[FB][1];
#pragma unroll
      for (int f = 0; f < FB; ++f) {
        x[f] = A + (int64_t)min(r0 + 16 * f + l16, ad.Nl - 1) * a.K;
        acc[f][0] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      }
      few_rows_dot<T, FB, 1>(x, y, k_lo, k_hi, wave, NW, lane, acc);
      const f32x4_t s = sum_waves<FB, 1>(red, acc, wave, NW, lane);
      if (wave < FB && l16 < n_valid && id == next)
        store4(H + (int64_t)n * ad.Nl, r0 + 16 * wave + 4 * G, ad.Nl, s, (ad.Nl & 3) == 0);
      __syncthreads();  // before the next sums overwrite `red`
    }
  }
}

// The projection of 16 features by all rows, plus each row's low-rank part:
// the ranks are shared by the waves like k, four at a time.
template <typename T, typename TO, int RB>
__global__ __launch_bounds__(64 * NW) void adapt_few_up(GroupArgs a, AdaptArgs ad) {
  __shared__ f32x4_t red[NW * RB * 64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, G = lane >> 4;
  const int m0 = 16 * blockIdx.x, n0 = 16 * RB * blockIdx.y;
  const int n_valid = min(a.N - n0, 16 * RB);
  const T* x[1] = {reinterpret_cast<const T*>(a.X) + (int64_t)min(m0 + l16, a.M - 1) * a.ldx};
  const T* y[RB];
  f32x4_t acc[1][RB];
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    const int n = n0 + min(16 * b + l16, n_valid - 1);
    y[b] = reinterpret_cast<const T*>(a.Y) + (int64_t)n * a.ldy;
    acc[0][b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    const int id = ad.ids[n];
    if (id >= 0 && id < ad.Na) {
      const float s = ad.scales ? ad.scales[id] : 1.f;
      const T* const B = reinterpret_cast<const T*>(ad.B) + (int64_t)id * a.M * ad.Nl;
      for (int r0 = 4 * wave; r0 < ad.Nl; r0 += 4 * NW) {
        float h[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          h[e] = 0.f;
          if (r0 + e < ad.Nl) {
            for (int z = 0; z < ad.kz; ++z)
              h[e] += ad.H[((int64_t)z * a.N + n) * ad.Nl + r0 + e];
            h[e] *= s;
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const T* const row = B + (int64_t)min(m0 + 4 * G + i, a.M - 1) * ad.Nl + r0;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (r0 + e < ad.Nl) acc[0][b][i] += h[e] * to_f32(row[e]);
        }
      }
    }
  }
  few_rows_dot<T, 1, RB>(x, y, 0, a.K, wave, NW, lane, acc);
  const f32x4_t s = sum_waves<1, RB>(red, acc, wave, NW, lane);
  const bool whole = ((uintptr_t)a.D & (4 * sizeof(TO) - 1)) == 0 && (a.ldd & 3) == 0;
  const int n = 16 * wave + l16;
  if (wave < RB && n < n_valid)
    store4(reinterpret_cast<TO*>(a.D) + (int64_t)(n0 + n) * a.ldd, m0 + 4 * G, a.M, s, whole);
}

template <typename T, typename TO>
hipError_t launch_few(const GroupArgs& a, int rb, hipStream_t stream) {
  const int64_t mt = (a.M + 15) / 16, parts = a.Ng + 1 < a.N ? a.Ng + 1 : a.N;
  const dim3 grid((uint32_t)((a.N / (16 * rb) + parts) * mt)), block(64 * NW);
  switch (rb) {
    case 1: group_few<T, TO, 1><<<grid, block, 0, stream>>>(a); break;
    case 2: group_few<T, TO, 2><<<grid, block, 0, stream>>>(a); break;
    default: group_few<T, TO, 4><<<grid, block, 0, stream>>>(a); break;
  }
  return hipGetLastError();
}

template <typename T, typename TO>
hipError_t launch_adapt_typed(const GroupArgs& a, const AdaptArgs& ad, hipStream_t stream) {
  constexpr int RUN = 256 / (int)sizeof(T);
  // slices of k of whole runs; the kernels add ad.kz partial sums
  const int kslice = (int)(((a.K + ad.kz - 1) / ad.kz + RUN - 1) / RUN) * RUN;
  const dim3 block(64 * NW);
  const dim3 gd((uint32_t)((a.N + 15) / 16), (uint32_t)(ad.Na < 16 ? ad.Na : 16), (uint32_t)ad.kz);
  if (ad.Nl <= 16)
    adapt_few_down<T, 1><<<gd, block, 0, stream>>>(a, ad, kslice);
  else if (ad.Nl <= 32)
    adapt_few_down<T, 2><<<gd, block, 0, stream>>>(a, ad, kslice);
  else
    adapt_few_down<T, 4><<<gd, block, 0, stream>>>(a, ad, kslice);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int rb = a.N <= 16 ? 1 : a.N <= 32 ? 2 : 4;
  const dim3 gu((uint32_t)((a.M + 15) / 16), (uint32_t)((a.N + 16 * rb - 1) / (16 * rb)));
  switch (rb) {
    case 1: adapt_few_up<T, TO, 1><<<gu, block, 0, stream>>>(a, ad); break;
    case 2: adapt_few_up<T, TO, 2><<<gu, block, 0, stream>>>(a, ad); break;
    default: adapt_few_up<T, TO, 4><<<gu, block, 0, stream>>>(a, ad); break;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_group_skinny(const GroupArgs& a, int dtype, int rb, hipStream_t stream) {
  switch (dtype) {
    case CNN_F32: return launch_few<float, float>(a, rb, stream);
    case CNN_BF16: return launch_few<bf16_t, float>(a, rb, stream);
    default: return launch_few<bf16_t, bf16_t>(a, rb, stream);
  }
}

bool adapt_few(int64_t Nt) { return Nt <= 64; }

int adapt_slices(int64_t Nc) {
  // a workgroup's eight waves take 256 bytes of k each in turn
  const int64_t n = Nc / 1024;
  return n < 1 ? 1 : n > 4 ? 4 : (int)n;
}

hipError_t launch_adapt_few(const GroupArgs& a, const AdaptArgs& ad, int dtype,
                            hipStream_t stream) {
  switch (dtype) {
    case CNN_F32: return launch_adapt_typed<float, float>(a, ad, stream);
    case CNN_BF16: return launch_adapt_typed<bf16_t, float>(a, ad, stream);
    default: return launch_adapt_typed<bf16_t, bf16_t>(a, ad, stream);
  }
}

}  // namespace cnnlib
