// The router's balance: counts of its choices per expert, the balance loss, the
// loss on the logits' size, and their gradient.
//
// Of a row that takes part (one with a choice and an allowed logit), p is the
// softmax over its allowed experts and z = log sum exp l.  Of a sequence s with
// T rows that take part and n[e] choices of expert e: f[e] = n[e] / sum n,
// P[e] = sum p[e] / T, and
//   Loss[0] = the mean over sequences with T > 0 of Ng sum_e f[e] P[e]
//   Loss[1] = sum z^2 / sum T
//   dl[e] = d0 Ng / (sequences T) p[e] (f[e] - sum p f) + d1 2 / (sum T) z p[e].
//
// Forward: a workgroup owns a run of rows and adds up p, z^2 and the choices of
// each sequence in it; the pair (workgroup b, sequence s) has place b + s, which
// no other pair shares since both only grow.  A second launch, a workgroup a
// sequence, adds a sequence's places in order and the last of them to finish adds
// up the sequences, in order too.  One workgroup and one sequence: one launch.
// Rows are held by 16 lanes (64 past 256 experts), as in the router.
#include "common.h"
#include "routed.h"

namespace cnnlib {

namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64;

template <int CTRL> __device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
// f(f(..)) over the row's LT lanes, the same in all of them.
template <int LT, typename F> __device__ __forceinline__ float over_row(float v, F f) {
  v = f(v, dpp<0xb1>(v));   // quad_perm 1,0,3,2
  v = f(v, dpp<0x4e>(v));   // quad_perm 2,3,0,1
  v = f(v, dpp<0x141>(v));  // row_half_mirror
  v = f(v, dpp<0x140>(v));  // row_mirror
  if constexpr (LT == 64) {
    v = f(v, __shfl_xor(v, 16));
    v = f(v, __shfl_xor(v, 32));
  }
  return v;
}
template <int LT> __device__ __forceinline__ float row_sum(float v) {
  return over_row<LT>(v, [](float a, float b) { return a + b; });
}

// The softmax p of a row over its allowed experts, E a lane (zero elsewhere);
// returns log sum exp.  `allowed`: some expert is.  +inf shares the whole weight
// with its kind.
template <typename T, int LT, int E>
__device__ __forceinline__ float softmax_row(const T* l, int Ng, int li, bool ok, float (&p)[E],
                                             bool* allowed) {
  float x[E], m = -INFINITY;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const int e = i * LT + li;
    const float v = ok && e < Ng ? to_f32(l[e]) : -INFINITY;
    x[i] = v > -INFINITY ? v : -INFINITY;  // NaN is not allowed either
    m = fmaxf(m, x[i]);
  }
  m = over_row<LT>(m, [](float a, float b) { return fmaxf(a, b); });
  *allowed = m > -INFINITY;
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    p[i] = !(x[i] > -INFINITY) ? 0.f : x[i] == m ? 1.f : expf(x[i] - m);
    s += p[i];
  }
  s = row_sum<LT>(s);
  const float inv = s > 0.f ? 1.f / s : 0.f;
#pragma unroll
  for (int i = 0; i < E; ++i) p[i] *= inv;
  return m + logf(s);
}

// The sequence of row t: the last that starts at or before it; -1: before the
// first, Ns: past the last.
__device__ __forceinline__ int sequence_of(const int32_t* bounds, int Ns, int t) {
  if (!bounds) return 0;
  int lo = 0, hi = Ns + 1;  // bounds[i] <= t for i < lo, > t for i >= hi
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (bounds[mid] <= t) lo = mid + 1; else hi = mid;
  }
  return lo - 1;
}

struct Parts {  // the workspace; `places` = workgroups + sequences
  float* p;       // [places][Ng]
  int32_t* n;     // [places][Ng]
  float* z;       // [places]
  int32_t* t;     // [places]
  float* loss;    // [Ns][2]: balance of each sequence, z^2
  int32_t* done;  // sequences that are added up
};
__host__ __device__ inline Parts parts_of(void* ws, int places, int Ng, int Ns) {
  Parts w;
  w.p = (float*)ws;
  w.n = (int32_t*)(w.p + (int64_t)places * Ng);
  w.z = (float*)(w.n + (int64_t)places * Ng);
  w.t = (int32_t*)(w.z + places);
  w.loss = (float*)(w.t + places);
  w.done = (int32_t*)(w.loss + 2 * (int64_t)Ns);
  return w;
}

struct Shared {
  int32_t hist[1024];
  float row[kWaves][1024];
  float z[kWaves + 1];  // [0] a result, the rest for sums
  int32_t t[kWaves + 1];
};

// The sum over the workgroup's threads, by waves and then in their order.
template <typename V> __device__ __forceinline__ V block_sum(V v, V* part) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  V s = part[0];
  for (int w = 1; w < kWaves; ++w) s += part[w];
  return s;
}

// The sums of one sequence's rows [t0, t1) in this workgroup: p into s.row[0],
// choices into s.hist, z^2 into s.z[0], rows into s.t[0].
template <typename T, int LT, int E>
__device__ void sum_rows(const BalanceArgs& a, Shared& s, int t0, int t1) {
  const int tid = threadIdx.x, li = tid % LT, lane = tid & 63, wave = tid >> 6;
  for (int e = tid; e < a.Ng; e += kThreads) s.hist[e] = 0;
  __syncthreads();
  float sum[E], z = 0.f;
  int rows = 0;
#pragma unroll
  for (int i = 0; i < E; ++i) sum[i] = 0.f;
  for (int tb = t0; tb < t1; tb += kThreads / LT) {
    const int t = tb + tid / LT;
    const bool ok = t < t1;
    const int64_t row = ok ? t : t0;
    float p[E];
    bool allowed;
    const float lse = softmax_row<T, LT, E>(reinterpret_cast<const T*>(a.logits) + row * a.Ng, a.Ng, li, ok, p, &allowed);
    const int c = ok && li < a.Kt ? a.choice[row * a.Kt + li] : -1;
    const bool mine = c >= 0 && c < a.Ng;
    if (mine) atomicAdd(&s.hist[c], 1);
    // whether one of the row's lanes has a choice
    const uint64_t any = __ballot(mine) >> (lane & ~(LT - 1));
    const bool part = allowed && (LT == 64 ? any : any & 0xffff) != 0;
#pragma unroll
    for (int i = 0; i < E; ++i) sum[i] += part ? p[i] : 0.f;
    z += part ? lse * lse : 0.f;
    rows += part;
  }
  // the rows that a wave holds side by side, then the waves in their order
  if constexpr (LT == 16) {
#pragma unroll
    for (int i = 0; i < E; ++i) {
      sum[i] += __shfl_xor(sum[i], 16);
      sum[i] += __shfl_xor(sum[i], 32);
    }
    z += __shfl_xor(z, 16);
    z += __shfl_xor(z, 32);
    rows += __shfl_xor(rows, 16);
    rows += __shfl_xor(rows, 32);
  }
  if (lane < LT)
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (i * LT + li < a.Ng) s.row[wave][i * LT + li] = sum[i];
  if (lane == 0) {
    s.z[wave] = z;
    s.t[wave] = rows;
  }
  __syncthreads();
  for (int e = tid; e < a.Ng; e += kThreads) {
    float v = s.row[0][e];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) v += s.row[w][e];
    s.row[0][e] = v;
  }
  if (tid == 0)
    for (int w = 1; w < kWaves; ++w) {
      s.z[0] += s.z[w];
      s.t[0] += s.t[w];
    }
  __syncthreads();
}

// The rows of sequence q, whatever the bounds are.
__device__ __forceinline__ void rows_of(const BalanceArgs& a, int q, int* lo, int* hi) {
  *lo = a.bounds ? min(max(a.bounds[q], 0), a.Nt) : 0;
  *hi = a.bounds ? min(max(a.bounds[q + 1], *lo), a.Nt) : a.Nt;
}

// The balance of a sequence from s.row[0] and s.hist, to all threads.
__device__ float sequence_loss(const BalanceArgs& a, Shared& s, int rows) {
  int n = 0;
  for (int e = threadIdx.x; e < a.Ng; e += kThreads) n += s.hist[e];
  const float total = (float)max(block_sum(n, s.t + 1), 1), live = (float)max(rows, 1);
  float fp = 0.f;
  for (int e = threadIdx.x; e < a.Ng; e += kThreads)
    fp += (float)s.hist[e] / total * (s.row[0][e] / live);
  return (float)a.Ng * block_sum(fp, s.z + 1);
}

// ONE: a single workgroup and sequence, which finishes the work.
template <typename T, int LT, int E, bool ONE>
__global__ __launch_bounds__(kThreads) void balance_rows(BalanceArgs a) {
  __shared__ Shared s;
  const int tid = threadIdx.x, b = blockIdx.x;
  if constexpr (ONE) {
    int lo, hi;
    rows_of(a, 0, &lo, &hi);
    sum_rows<T, LT, E>(a, s, lo, hi);
    const int rows = s.t[0];
    const float z = s.z[0], loss = sequence_loss(a, s, rows);
    for (int e = tid; e < a.Ng; e += kThreads) a.counts[e] = s.hist[e];
    if (tid == 0) {
      a.tokens[0] = rows;
      a.loss[0] = rows > 0 ? loss : 0.f;
      a.loss[1] = rows > 0 ? z / (float)rows : 0.f;
    }
  } else {
    const Parts w = parts_of(a.ws, a.nblocks + a.Ns, a.Ng, a.Ns);
    if (b == 0 && tid == 0) *w.done = 0;
    const int last = min(a.Nt, (b + 1) * a.chunk);
    for (int t = b * a.chunk; t < last;) {
      const int q = sequence_of(a.bounds, a.Ns, t);
      if (q >= a.Ns) break;
      // at least a row further, whatever the bounds are
      const int end = a.bounds ? min(last, max(a.bounds[q + 1], t + 1)) : last;
      if (q >= 0) {
        sum_rows<T, LT, E>(a, s, t, end);
        const int64_t at = b + q;
        for (int e = tid; e < a.Ng; e += kThreads) {
          w.p[at * a.Ng + e] = s.row[0][e];
          w.n[at * a.Ng + e] = s.hist[e];
        }
        if (tid == 0) {
          w.z[at] = s.z[0];
          w.t[at] = s.t[0];
        }
        __syncthreads();
      }
      t = end;
    }
  }
}

// A sequence's places added up, in order; the last sequence to finish adds up
// the losses.
__global__ __launch_bounds__(kThreads) void balance_sums(BalanceArgs a) {
  __shared__ Shared s;
  __shared__ int32_t last;
  const int tid = threadIdx.x, q = blockIdx.x;
  const Parts w = parts_of(a.ws, a.nblocks + a.Ns, a.Ng, a.Ns);
  int lo, hi;
  rows_of(a, q, &lo, &hi);
  // the workgroups that met it; thread (x, y): expert x of every ny-th of them
  const int b0 = lo / a.chunk, b1 = hi > lo ? (hi - 1) / a.chunk + 1 : b0;
  const int ny = min(kWaves, max(1, kThreads / a.Ng));
  for (int e = tid; e < a.Ng; e += kThreads) s.hist[e] = 0;
  __syncthreads();
  for (int i = tid; i < ny * a.Ng; i += kThreads) {
    const int x = i % a.Ng, y = i / a.Ng;
    float p = 0.f;
    int n = 0;
#pragma unroll 8
    for (int b = b0 + y; b < b1; b += ny) {
      p += w.p[(int64_t)(b + q) * a.Ng + x];
      n += w.n[(int64_t)(b + q) * a.Ng + x];
    }
    s.row[y][x] = p;
    atomicAdd(&s.hist[x], n);
  }
  float z = 0.f;
  int rows = 0;
  for (int b = b0 + tid; b < b1; b += kThreads) {
    z += w.z[b + q];
    rows += w.t[b + q];
  }
  z = block_sum(z, s.z);
  rows = block_sum(rows, s.t);
  for (int e = tid; e < a.Ng; e += kThreads) {
    float v = s.row[0][e];
    for (int y = 1; y < ny; ++y) v += s.row[y][e];
    s.row[0][e] = v;
    a.counts[(int64_t)q * a.Ng + e] = s.hist[e];
  }
  __syncthreads();
  const float loss = sequence_loss(a, s, rows);
  if (tid == 0) {
    a.tokens[q] = rows;
    w.loss[2 * (int64_t)q] = rows > 0 ? loss : 0.f;
    w.loss[2 * (int64_t)q + 1] = rows > 0 ? z : 0.f;
    __threadfence();
    last = atomicAdd(w.done, 1) == a.Ns - 1;
  }
  __syncthreads();
  if (!last) return;
  __threadfence();
  float balance = 0.f, squares = 0.f;
  int live = 0, total = 0;
  for (int i = tid; i < a.Ns; i += kThreads) {
    // written by other workgroups of this launch: past this one's caches
    balance += __hip_atomic_load(w.loss + 2 * (int64_t)i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    squares += __hip_atomic_load(w.loss + 2 * (int64_t)i + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const int t = __hip_atomic_load(a.tokens + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    live += t > 0;
    total += t;
  }
  balance = block_sum(balance, s.z);
  squares = block_sum(squares, s.z);
  live = block_sum(live, s.t);
  total = block_sum(total, s.t);
  if (tid == 0) {
    a.loss[0] = balance / (float)max(live, 1);
    a.loss[1] = squares / (float)max(total, 1);
  }
}

// One row by LT lanes; ADD: on top of what dLogits holds.
template <typename T, typename TO, int LT, int E, bool ADD>
__global__ __launch_bounds__(256) void balance_bwd(BalanceArgs a) {
  const int tid = threadIdx.x, lane = tid & 63, li = tid % LT;
  // sequences with rows that take part, and all such rows
  __shared__ int32_t part[2][4];
  int live = 0, total = 0;
  for (int i = tid; i < a.Ns; i += 256) {
    const int t = a.tokens[i];
    live += t > 0;
    total += t;
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    live += __shfl_xor(live, d);
    total += __shfl_xor(total, d);
  }
  if (lane == 0) {
    part[0][tid >> 6] = live;
    part[1][tid >> 6] = total;
  }
  __syncthreads();
  live = part[0][0] + part[0][1] + part[0][2] + part[0][3];
  total = part[1][0] + part[1][1] + part[1][2] + part[1][3];

  const int64_t t = (int64_t)blockIdx.x * (256 / LT) + tid / LT;
  const bool ok = t < a.Nt;
  const int64_t row = ok ? t : 0;
  float p[E];
  bool allowed;
  const float lse = softmax_row<T, LT, E>(reinterpret_cast<const T*>(a.logits) + row * a.Ng, a.Ng, li, ok, p, &allowed);
  const int c = ok && li < a.Kt ? a.choice[row * a.Kt + li] : -1;
  const uint64_t any = __ballot(c >= 0 && c < a.Ng) >> (lane & ~(LT - 1));
  const int q = sequence_of(a.bounds, a.Ns, (int)row);
  const bool in = allowed && (LT == 64 ? any : any & 0xffff) != 0 && q >= 0 && q < a.Ns;
  const int32_t* const n = a.counts + (int64_t)(in ? q : 0) * a.Ng;
  float f[E], sum = 0.f, pf = 0.f;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const int e = i * LT + li;
    f[i] = e < a.Ng ? (float)n[e] : 0.f;
    sum += f[i];
  }
  const float inv = 1.f / fmaxf(row_sum<LT>(sum), 1.f);
#pragma unroll
  for (int i = 0; i < E; ++i) {
    f[i] *= inv;
    pf += p[i] * f[i];
  }
  pf = row_sum<LT>(pf);
  const float rows = (float)max(a.tokens[in ? q : 0], 1);
  const float db = a.dloss[0] * (float)a.Ng / ((float)max(live, 1) * rows);
  const float dz = a.dloss[1] * 2.f / (float)max(total, 1) * lse;
  if (!ok) return;
  TO* const out = reinterpret_cast<TO*>(a.dlogits) + row * a.Ng;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const int e = i * LT + li;
    if (e >= a.Ng) continue;
    // an expert without weight gets nothing, also where the losses are not finite
    float d = in && p[i] != 0.f ? p[i] * (db * (f[i] - pf) + dz) : 0.f;
    if constexpr (ADD) d += to_f32(out[e]);
    out[e] = from_f32<TO>(d);
  }
}

template <typename T, int LT, int E> void launch_rows(const BalanceArgs& a, bool one, hipStream_t stream) {
  if (one) balance_rows<T, LT, E, true><<<dim3(1), dim3(kThreads), 0, stream>>>(a);
  else balance_rows<T, LT, E, false><<<dim3(a.nblocks), dim3(kThreads), 0, stream>>>(a);
}

template <typename T> hipError_t launch_fwd(const BalanceArgs& a, hipStream_t stream) {
  // one workgroup takes some rows for the price of the second launch
  const bool one = a.Ns == 1 && a.Nt <= kBalanceOne;
  if (a.Ng <= 32) launch_rows<T, 16, 2>(a, one, stream);
  else if (a.Ng <= 64) launch_rows<T, 16, 4>(a, one, stream);
  else if (a.Ng <= 128) launch_rows<T, 16, 8>(a, one, stream);
  else if (a.Ng <= 256) launch_rows<T, 16, 16>(a, one, stream);
  else launch_rows<T, 64, 16>(a, one, stream);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || one) return e;
  balance_sums<<<dim3(a.Ns), dim3(kThreads), 0, stream>>>(a);
  return hipGetLastError();
}

template <typename T, typename TO, bool ADD> hipError_t launch_bwd(const BalanceArgs& a, hipStream_t stream) {
  const int rows = a.Ng <= 256 ? 16 : 4;  // of a workgroup
  const int64_t blocks = ((int64_t)a.Nt + rows - 1) / rows;
  const hipError_t e = grid_fits(blocks, 256);
  if (e != hipSuccess) return e;
  auto* const k = a.Ng <= 32    ? balance_bwd<T, TO, 16, 2, ADD>
                  : a.Ng <= 64  ? balance_bwd<T, TO, 16, 4, ADD>
                  : a.Ng <= 128 ? balance_bwd<T, TO, 16, 8, ADD>
                  : a.Ng <= 256 ? balance_bwd<T, TO, 16, 16, ADD>
                                : balance_bwd<T, TO, 64, 16, ADD>;
  k<<<dim3((uint32_t)blocks), dim3(256), 0, stream>>>(a);
  return hipGetLastError();
}

template <typename T, typename TO> hipError_t launch_bwd(const BalanceArgs& a, bool add, hipStream_t stream) {
  return add ? launch_bwd<T, TO, true>(a, stream) : launch_bwd<T, TO, false>(a, stream);
}

}  // namespace

int64_t balance_ws_bytes(int64_t Nt, int64_t Ng, int64_t Ns) {
  int32_t chunk, nblocks;
  order_blocks(Nt, &chunk, &nblocks);
  return Ns == 1 && Nt <= kBalanceOne ? 0 : ((nblocks + Ns) * (8 * Ng + 8) + 8 * Ns + 4 + 15) & ~(int64_t)15;
}

hipError_t launch_balance(const BalanceArgs& a, bool bf16, hipStream_t stream) {
  return bf16 ? launch_fwd<bf16_t>(a, stream) : launch_fwd<float>(a, stream);
}

hipError_t launch_balance_bwd(const BalanceArgs& a, int dtype, bool add, hipStream_t stream) {
  switch (dtype) {
    case CNN_F32: return launch_bwd<float, float>(a, add, stream);
    case CNN_BF16: return launch_bwd<bf16_t, float>(a, add, stream);
    default: return launch_bwd<bf16_t, bf16_t>(a, add, stream);
  }
}

}  // namespace cnnlib
