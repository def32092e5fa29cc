// The weighted return of the experts' rows to their tokens, and its gradient.
// Both are bound by moving the grouped rows once; everything is 16 bytes a lane,
// sums in fp32.  8192 rows of 2048 bf16 features: the return of four choices 36
// us (168 MB at 4.7 TB/s, a large copy's bytes at 5.5), the gradient of two
// (as many bytes) 29 us by itself.
#include "common.h"
#include "routed.h"

namespace cnnlib {

namespace {

// V consecutive values of a row as fp32; at most `n` of them are there.
template <typename T, int V> __device__ __forceinline__ void load_row(const T* p, int n, float (&v)[V]) {
  if (n >= V) {
    T raw[V];
    __builtin_memcpy(raw, p, V * sizeof(T));
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = to_f32(raw[i]);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = i < n ? to_f32(p[i]) : 0.f;
  }
}
template <typename T, int V> __device__ __forceinline__ void store_row(T* p, int n, const float (&v)[V]) {
  if (n >= V) {
    if constexpr (sizeof(T) == 2) {
      uint32_t raw[V / 2];
#pragma unroll
      for (int i = 0; i < V / 2; ++i) raw[i] = pk_bf16(v[2 * i], v[2 * i + 1]);
      __builtin_memcpy(p, raw, V * sizeof(T));
    } else {
      __builtin_memcpy(p, v, V * sizeof(T));
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < n) p[i] = from_f32<T>(v[i]);
  }
}

// Out[t] = sum_j gates[t, j] In[slots[t, j]], j in order, fp32.  A thread has V
// consecutive features of one row and reads them from all Kt rows at once: four
// rows in flight a thread, a workgroup's 2 KB of a row (bf16) in one piece.
// Stores past the caches were 6 % quicker here and slower in the gradient.
template <typename T, typename TO, int V>
__global__ __launch_bounds__(256) void combine_rows(const T* In, const int32_t* slots,
                                                    const float* gates, TO* Out, int64_t units,
                                                    int upr, int Kt, int64_t Np, int64_t Nk) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= units) return;
  const int64_t t = i / upr;
  const int64_t k = (i - t * upr) * V;
  const int n = (int)min<int64_t>(Nk - k, V);
  float acc[V];
#pragma unroll
  for (int e = 0; e < V; ++e) acc[e] = 0.f;
#pragma unroll 4
  for (int j = 0; j < Kt; ++j) {
    const int p = slots[t * Kt + j];
    const float g = gates ? gates[t * Kt + j] : 1.f;
    if (p >= 0 && p < Np) {
      float v[V];
      load_row<T, V>(In + p * Nk + k, n, v);
#pragma unroll
      for (int e = 0; e < V; ++e) acc[e] += g * v[e];
    }
  }
  store_row<TO, V>(Out + t * Nk + k, n, acc);
}

// W waves per place p: with t = rows[p] and j the choice whose slot p is,
// dIn[p] = gate dOut[t] and dGates[t, j] = dOut[t] . In[p]; zeros where no row
// has the place.  In the order of the places, In and dIn are read and written
// straight through, and dOut's rows (a Kt-th of the bytes) come from the caches
// the second time (in the order of the rows, a wave of each pair: 64 us where this
// takes 30).  The last workgroups clear dGates of the choices without a
// place.
template <typename T, typename TO, int V, int W>
__global__ __launch_bounds__(256) void combine_rows_bwd(const T* dOut, const T* In,
                                                        const int32_t* slots, const int32_t* rows,
                                                        const float* gates, TO* dIn, float* dGates,
                                                        int64_t Nt, int Kt, int64_t Np, int64_t Nk,
                                                        int64_t place_blocks) {
  __shared__ float sums[4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (blockIdx.x >= place_blocks) {
    const int64_t i = (blockIdx.x - place_blocks) * 256 + threadIdx.x;
    if (i < Nt * Kt && (slots[i] < 0 || slots[i] >= Np)) dGates[i] = 0.f;
    return;
  }
  const int64_t p = (int64_t)blockIdx.x * (4 / W) + wave / W;
  const bool there = p < Np;
  const int row = there ? __builtin_amdgcn_readfirstlane(rows[p]) : -1;
  // the choice of this place: the lanes look at Kt slots of the row
  int64_t pair = -1;
  if (row >= 0 && row < Nt)
    for (int j0 = 0; j0 < Kt && pair < 0; j0 += 64) {
      const uint64_t hit = __ballot(j0 + lane < Kt && slots[(int64_t)row * Kt + min(j0 + lane, Kt - 1)] == p);
      if (hit) pair = (int64_t)row * Kt + j0 + __ffsll((unsigned long long)hit) - 1;
    }
  float dot = 0.f;
  if (there) {
    TO* const out = dIn + p * Nk;
    if (pair < 0) {
      const float z[V] = {};
      for (int64_t k = ((wave % W) * 64 + lane) * V; k < Nk; k += W * 64 * V)
        store_row<TO, V>(out + k, (int)min<int64_t>(Nk - k, V), z);
    } else {
      const T* const drow = dOut + row * Nk;
      const T* const irow = In + p * Nk;
      const float g = gates ? gates[pair] : 1.f;
      auto columns = [&](int64_t k, int n) __attribute__((always_inline)) {
        float d[V], x[V];
        load_row<T, V>(irow + k, n, x);
        load_row<T, V>(drow + k, n, d);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          dot += d[e] * x[e];
          d[e] *= g;
        }
        store_row<TO, V>(out + k, n, d);
      };
      for (int64_t k = ((wave % W) * 64 + lane) * V; k < Nk; k += W * 64 * V) {
        if (k + V <= Nk) columns(k, V);
        else columns(k, (int)(Nk - k));
      }
    }
  }
  if (!dGates) return;
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) dot += __shfl_xor(dot, d);
  if (W > 1) {
    if (lane == 0) sums[wave] = dot;
    __syncthreads();
    dot = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) dot += sums[wave / W * W + w];
  }
  if (pair >= 0 && wave % W == 0 && lane == 0) dGates[pair] = dot;
}

template <typename T, typename TO>
hipError_t launch_fwd(const void* In, const int32_t* slots, const float* gates, void* Out,
                      int64_t Nt, int Kt, int64_t Np, int64_t Nk, hipStream_t stream) {
  constexpr int V = 16 / (int)sizeof(T);
  const int upr = (int)((Nk + V - 1) / V);
  const int64_t units = Nt * upr, blocks = (units + 255) / 256;
  const hipError_t e = grid_fits(blocks, 256);
  if (e != hipSuccess) return e;
  combine_rows<T, TO, V><<<dim3((uint32_t)blocks), dim3(256), 0, stream>>>(
      reinterpret_cast<const T*>(In), slots, gates, reinterpret_cast<TO*>(Out), units, upr, Kt, Np, Nk);
  return hipGetLastError();
}

template <typename T, typename TO>
hipError_t launch_bwd(const void* dOut, const void* In, const int32_t* slots, const int32_t* rows,
                      const float* gates, void* dIn, float* dGates, int64_t Nt, int Kt, int64_t Np,
                      int64_t Nk, hipStream_t stream) {
  constexpr int V = 16 / (int)sizeof(T);
  // a wave for each 64 V columns, up to four
  const int w = Nk <= 64 * V ? 1 : Nk <= 128 * V ? 2 : 4;
  const int64_t place_blocks = (Np * w + 3) / 4, clear_blocks = dGates ? (Nt * Kt + 255) / 256 : 0;
  if (!place_blocks && !clear_blocks) return hipSuccess;
  const hipError_t e = grid_fits(place_blocks + clear_blocks, 256);
  if (e != hipSuccess) return e;
  auto* const k = w == 1 ? combine_rows_bwd<T, TO, V, 1>
                  : w == 2 ? combine_rows_bwd<T, TO, V, 2> : combine_rows_bwd<T, TO, V, 4>;
  k<<<dim3((uint32_t)(place_blocks + clear_blocks)), dim3(256), 0, stream>>>(
      reinterpret_cast<const T*>(dOut), reinterpret_cast<const T*>(In), slots, rows, gates,
      reinterpret_cast<TO*>(dIn), dGates, Nt, Kt, Np, Nk, place_blocks);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_combine(const void* In, const int32_t* slots, const float* gates, void* Out,
                          int64_t Nt, int Kt, int64_t Np, int64_t Nk, int dtype,
                          hipStream_t stream) {
  switch (dtype) {
    case CNN_F32: return launch_fwd<float, float>(In, slots, gates, Out, Nt, Kt, Np, Nk, stream);
    case CNN_BF16: return launch_fwd<bf16_t, float>(In, slots, gates, Out, Nt, Kt, Np, Nk, stream);
    default: return launch_fwd<bf16_t, bf16_t>(In, slots, gates, Out, Nt, Kt, Np, Nk, stream);
  }
}

hipError_t launch_combine_bwd(const void* dOut, const void* In, const int32_t* slots,
                              const int32_t* rows, const float* gates, void* dIn, float* dGates,
                              int64_t Nt, int Kt, int64_t Np, int64_t Nk, int dtype,
                              hipStream_t stream) {
  switch (dtype) {
    case CNN_F32:
      return launch_bwd<float, float>(dOut, In, slots, rows, gates, dIn, dGates, Nt, Kt, Np, Nk, stream);
    case CNN_BF16:
      return launch_bwd<bf16_t, float>(dOut, In, slots, rows, gates, dIn, dGates, Nt, Kt, Np, Nk, stream);
    default:
      return launch_bwd<bf16_t, bf16_t>(dOut, In, slots, rows, gates, dIn, dGates, Nt, Kt, Np, Nk, stream);
  }
}

}  // namespace cnnlib
