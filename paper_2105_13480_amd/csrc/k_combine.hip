// The weighted return of the experts' rows to their tokens, and its gradient.
// Both are bound by moving the grouped rows once.
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
// consecutive features of one row and reads them from all Kt rows at once.
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

// One wave per token: dIn[p] = gate dOut[t] and dGates[t, j] = dOut[t] . In[p]
// for each of its Kt rows p.  The workgroups past the tokens' write zeros to
// the rows that no token has (rows[p] < 0).
template <typename T, typename TO, int V>
__global__ __launch_bounds__(256) void combine_rows_bwd(const T* dOut, const T* In,
                                                        const int32_t* slots, const int32_t* rows,
                                                        const float* gates, TO* dIn, float* dGates,
                                                        int64_t Nt, int Kt, int64_t Np, int64_t Nk,
                                                        int64_t token_blocks) {
  const int lane = threadIdx.x & 63;
  const int64_t b = blockIdx.x;
  if (b >= token_blocks) {
    const int64_t p0 = ((b - token_blocks) * 4 + (threadIdx.x >> 6)) * 64;
    uint64_t gone = __ballot(p0 + lane < Np && rows[min(p0 + lane, Np - 1)] < 0);
    while (gone) {
      const int64_t p = p0 + __ffsll((unsigned long long)gone) - 1;
      gone &= gone - 1;
      const float z[V] = {};
      for (int64_t k = lane * V; k < Nk; k += 64 * V)
        store_row<TO, V>(dIn + p * Nk + k, (int)min<int64_t>(Nk - k, V), z);
    }
    return;
  }
  const int64_t t = b * 4 + (threadIdx.x >> 6);
  if (t >= Nt) return;
  for (int j = 0; j < Kt; ++j) {
    const int p = slots[t * Kt + j];
    float dot = 0.f;
    if (p >= 0 && p < Np) {
      const float g = gates ? gates[t * Kt + j] : 1.f;
#pragma unroll 4
      for (int64_t k = lane * V; k < Nk; k += 64 * V) {
        const int n = (int)min<int64_t>(Nk - k, V);
        float d[V], x[V];
        load_row<T, V>(dOut + t * Nk + k, n, d);
        load_row<T, V>(In + p * Nk + k, n, x);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          dot += d[e] * x[e];
          d[e] *= g;
        }
        store_row<TO, V>(dIn + p * Nk + k, n, d);
      }
    }
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) dot += __shfl_xor(dot, s);
    if (lane == 0 && dGates) dGates[t * Kt + j] = dot;
  }
}

template <typename T, typename TO>
hipError_t launch_fwd(const void* In, const int32_t* slots, const float* gates, void* Out,
                      int64_t Nt, int Kt, int64_t Np, int64_t Nk, hipStream_t stream) {
  constexpr int V = 16 / (int)sizeof(T);
  const int upr = (int)((Nk + V - 1) / V);
  const int64_t units = Nt * upr;
  combine_rows<T, TO, V><<<dim3((uint32_t)((units + 255) / 256)), dim3(256), 0, stream>>>(
      reinterpret_cast<const T*>(In), slots, gates, reinterpret_cast<TO*>(Out), units, upr, Kt, Np, Nk);
  return hipGetLastError();
}

template <typename T, typename TO>
hipError_t launch_bwd(const void* dOut, const void* In, const int32_t* slots, const int32_t* rows,
                      const float* gates, void* dIn, float* dGates, int64_t Nt, int Kt, int64_t Np,
                      int64_t Nk, hipStream_t stream) {
  constexpr int V = 16 / (int)sizeof(T);
  const int64_t token_blocks = (Nt + 3) / 4, zero_blocks = (Np + 255) / 256;
  combine_rows_bwd<T, TO, V>
      <<<dim3((uint32_t)(token_blocks + zero_blocks)), dim3(256), 0, stream>>>(
          reinterpret_cast<const T*>(dOut), reinterpret_cast<const T*>(In), slots, rows, gates,
          reinterpret_cast<TO*>(dIn), dGates, Nt, Kt, Np, Nk, token_blocks);
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
