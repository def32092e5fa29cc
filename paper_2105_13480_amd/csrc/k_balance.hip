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
//
// Bound by launches and by what waits for what within them (bounds, logits, sums), not by
// the 9 MB: 16384 rows of 128 experts in 37 sequences, bf16, rows 8.4 to 10.1 us, sums 5.6
// to 5.9, gradient 6.4 to 7.0 (a launch with nothing to do 2.5); 256 rows of 32 experts in
// fp32, one launch of 6.0 us (the two would be 8) and 3.8.  Sums of each workgroup are
// places of their own in the workspace, added up in order: atomic
// sums of floats would change from run to run.  Many short sequences take longer: a
// workgroup brings the sums of each of its together one by one, a workgroup of the second
// launch adds up one, and each wave of the gradient adds up all Tokens (the same rows in 4096
// sequences: rows 38 us, sums 100, gradient 14 to 25).
#include "common.h"
#include "routed.h"

namespace cnnlib {

namespace {

constexpr int kSumThreads = 1024;

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

__device__ __forceinline__ float to_f32(int32_t n) { return (float)n; }
using cnnlib::to_f32;

// E consecutive experts' values from `e` on of a row of Ng (`none` past its end and for
// a row that is not there).
template <int E, typename T, typename V>
__device__ __forceinline__ void load_experts(const T* row, int e, int Ng, bool ok, V none, V (&x)[E]) {
  if (ok && e + E <= Ng) {
    T v[E];
    __builtin_memcpy(v, row + e, sizeof(v));
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = (V)to_f32(v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = ok && e + i < Ng ? (V)to_f32(row[e + i]) : none;
  }
}
// Their softmax over the allowed experts (zero elsewhere); returns log sum exp.
// `allowed`: some expert is.  +inf shares the whole weight with its kind.
template <int LT, int E>
__device__ __forceinline__ float softmax_row(const float (&l)[E], float (&p)[E], bool* allowed) {
  float x[E], m = -INFINITY;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    x[i] = l[i] > -INFINITY ? l[i] : -INFINITY;  // NaN is not allowed either
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
// Whether one of the row's lanes has a choice.
template <int LT> __device__ __forceinline__ bool some_choice(bool mine) {
  const uint64_t any = __ballot(mine) >> (threadIdx.x & 63 & ~(LT - 1));
  return (LT == 64 ? any : any & 0xffff) != 0;
}

// Sequences by row, the same in the whole wave: find(t) is t's sequence (-1: before the
// first, Ns: past the last) and `end` the row after its last.  Starts are halved until
// 64 are left that may be t's; one load brings these, and find() asks for others only
// where they no longer reach.
struct Sequences {
  const int32_t* bounds;
  int Ns, first, v, end;  // v: bounds[first + lane]
  __device__ __forceinline__ void init(const int32_t* b, int Ns_) {
    bounds = b;
    Ns = Ns_;
    first = -1;
  }
  __device__ __forceinline__ int find(int t) {
    end = 0x7fffffff;
    if (!bounds) return 0;
    const int lane = threadIdx.x & 63;
    for (int tries = 0;; ++tries) {
      if (first >= 0) {
        const int n = __popcll(__ballot(first + lane <= Ns && v <= t));
        if (n < 64 || first + n > Ns || tries) {
          const int at = first + n;  // the first start past t
          if (at <= Ns) end = n < 64 ? __builtin_amdgcn_readlane(v, n) : __builtin_amdgcn_readfirstlane(bounds[at]);
          return at - 1;
        }
      }
      int lo = 0, hi = Ns + 1;  // bounds[i] <= t for i < lo, > t for i >= hi
      while (hi - lo > 64) {
        const int mid = (lo + hi) >> 1;
        if (__builtin_amdgcn_readfirstlane(bounds[mid]) <= t) lo = mid + 1; else hi = mid;
      }
      first = lo;
      v = bounds[min(lo + lane, Ns)];
    }
  }
};

struct Parts {  // the workspace; `places` = workgroups + sequences
  float* p;       // [places][Ng]
  int32_t* n;     // [places][Ng]
  float* z;       // [places]
  int32_t* t;     // [places]
  float* loss;    // [Ns][4]: balance of each sequence, z^2, rows
  int32_t* done;  // sequences that are added up
};
__host__ __device__ inline Parts parts_of(void* ws, int places, int Ng, int Ns) {
  Parts w;
  w.p = (float*)ws;
  w.n = (int32_t*)(w.p + (int64_t)places * Ng);
  w.z = (float*)(w.n + (int64_t)places * Ng);
  w.t = (int32_t*)(w.z + places);
  w.loss = (float*)(w.t + places);
  w.done = (int32_t*)(w.loss + 4 * (int64_t)Ns);
  return w;
}

// Sums over a wave.
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
  return v;
}
__device__ __forceinline__ int wave_sum(int v) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
  return v;
}

// The balance of a sequence of `rows` rows from its sums of p and its choices, by one wave.
__device__ __forceinline__ float sequence_loss(const float* p, const int32_t* n, int Ng, int rows) {
  const int lane = threadIdx.x & 63;
  int total = 0;
  for (int e = lane; e < Ng; e += 64) total += n[e];
  const float whole = (float)max(wave_sum(total), 1), live = (float)max(rows, 1);
  float fp = 0.f;
  for (int e = lane; e < Ng; e += 64) fp += (float)n[e] / whole * (p[e] / live);
  fp = wave_sum(fp);
  return rows > 0 ? (float)Ng * fp : 0.f;
}

// The rows of sequence q, whatever the bounds are.
__device__ __forceinline__ void rows_of(const BalanceArgs& a, int q, int* lo, int* hi) {
  *lo = a.bounds ? min(max(a.bounds[q], 0), a.Nt) : 0;
  *hi = a.bounds ? min(max(a.bounds[q + 1], *lo), a.Nt) : a.Nt;
}

// NT threads, LT lanes a row.  ONE: a single workgroup and sequence, which finishes the
// work.  Rows go through in blocks of NT / LT, whose weights are made once; a sequence's
// sums are brought together where it ends.
template <typename T, int NT, int LT, int E, bool ONE>
__global__ __launch_bounds__(NT) void balance_rows(BalanceArgs a) {
  constexpr int NW = NT / 64, ROWS = NT / LT;
  __shared__ float row[NW][LT * E], zs[NW];
  __shared__ int32_t hist[LT * E], ts[NW];
  const int tid = threadIdx.x, li = tid % LT, lane = tid & 63, wave = tid >> 6, b = blockIdx.x;
  const T* const logits = reinterpret_cast<const T*>(a.logits);
  const Parts w = parts_of(a.ws, a.nblocks + a.Ns, a.Ng, a.Ns);
  int t0 = b * a.chunk, last = min(a.Nt, t0 + a.chunk);
  if constexpr (ONE) rows_of(a, 0, &t0, &last);
  else if (b == 0 && tid == 0) *w.done = 0;
  // the first rows, before it is known whose they are
  float x[E];
  int t = t0 + tid / LT;
  load_experts<E>(logits + (int64_t)t * a.Ng, E * li, a.Ng, t < last, -INFINITY, x);
  int c = t < last && li < a.Kt ? a.choice[(int64_t)t * a.Kt + li] : -1;
  Sequences seq;
  int q = 0, end = last;
  if constexpr (!ONE) {
    seq.init(a.bounds, a.Ns);
    q = seq.find(t0);
    end = max(seq.end, t0 + 1);  // a row further, whatever the bounds are
  }
  for (int e = tid; e < a.Ng; e += NT) hist[e] = 0;
  __syncthreads();
  float sum[E], z = 0.f;
  int rows = 0;
#pragma unroll
  for (int i = 0; i < E; ++i) sum[i] = 0.f;
  // the sums of sequence q, and the next one's start at zero
  auto flush = [&]() __attribute__((always_inline)) {
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
      for (int i = 0; i < E; ++i) row[wave][E * li + i] = sum[i];
    if (lane == 0) {
      zs[wave] = z;
      ts[wave] = rows;
    }
    __syncthreads();
    const int64_t at = b + q;
    for (int e = tid; e < a.Ng; e += NT) {
      float v = row[0][e];
#pragma unroll
      for (int k = 1; k < NW; ++k) v += row[k][e];
      if constexpr (ONE) {
        row[0][e] = v;
        a.counts[e] = hist[e];
      } else {
        w.p[at * a.Ng + e] = v;
        w.n[at * a.Ng + e] = hist[e];
        hist[e] = 0;
      }
    }
    if (wave == 0) {
      const float zt = wave_sum(lane < NW ? zs[lane] : 0.f);
      const int n = wave_sum(lane < NW ? ts[lane] : 0);
      if (lane == 0) {
        if constexpr (ONE) {
          a.tokens[0] = ts[0] = n;
          a.loss[1] = n > 0 ? zt / (float)n : 0.f;
        } else {
          w.z[at] = zt;
          w.t[at] = n;
        }
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < E; ++i) sum[i] = 0.f;
    z = 0.f;
    rows = 0;
  };
  for (int tb = t0; tb < last && q < a.Ns; tb += ROWS) {
    // the next rows before these are summed up
    float next[E];
    const int tn = t + ROWS;
    load_experts<E>(logits + (int64_t)tn * a.Ng, E * li, a.Ng, tn < last, -INFINITY, next);
    const int cn = tn < last && li < a.Kt ? a.choice[(int64_t)tn * a.Kt + li] : -1;
    float p[E];
    bool allowed;
    const float lse = softmax_row<LT, E>(x, p, &allowed);
    const bool mine = c >= 0 && c < a.Ng;
    const bool part = some_choice<LT>(mine) && allowed;
    for (int lo = tb; lo < min(tb + ROWS, last) && q < a.Ns;) {
      const int hi = min(min(tb + ROWS, last), end);
      if (q >= 0 && t >= lo && t < hi) {
        if (mine) atomicAdd(&hist[c], 1);
#pragma unroll
        for (int i = 0; i < E; ++i) sum[i] += part ? p[i] : 0.f;
        z += part ? lse * lse : 0.f;
        rows += part;
      }
      lo = hi;
      if (!ONE && (hi == end || hi == last)) {
        if (q >= 0) flush();
        if (hi == last) break;
        q = seq.find(hi);
        end = max(seq.end, hi + 1);
      }
    }
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = next[i];
    c = cn;
    t = tn;
  }
  if constexpr (ONE) {
    flush();
    if (wave != 0) return;
    const float loss = sequence_loss(row[0], hist, a.Ng, ts[0]);
    if (lane == 0) a.loss[0] = loss;
  }
}

// A sequence's places added up, in order; the last sequence to finish adds up
// the losses.
__global__ __launch_bounds__(kSumThreads) void balance_sums(BalanceArgs a) {
  __shared__ float row[kSumThreads];
  __shared__ int32_t hist[1024];
  const int tid = threadIdx.x, lane = tid & 63, q = blockIdx.x;
  const Parts w = parts_of(a.ws, a.nblocks + a.Ns, a.Ng, a.Ns);
  int lo, hi;
  rows_of(a, q, &lo, &hi);
  // the workgroups that met it; thread (x, y): expert x of every ny-th of them
  const int b0 = lo / a.chunk, b1 = hi > lo ? (hi - 1) / a.chunk + 1 : b0;
  const int ny = kSumThreads / a.Ng, x = tid % a.Ng, y = tid / a.Ng;
  if (tid < a.Ng) hist[tid] = 0;
  __syncthreads();
  if (y < ny) {
    float p = 0.f;
    int n = 0;
#pragma unroll 8
    for (int b = b0 + y; b < b1; b += ny) {
      p += w.p[(int64_t)(b + q) * a.Ng + x];
      n += w.n[(int64_t)(b + q) * a.Ng + x];
    }
    row[tid] = p;
    atomicAdd(&hist[x], n);
  }
  __syncthreads();
  if (tid < a.Ng) {
    float v = row[tid];
    for (int k = 1; k < ny; ++k) v += row[k * a.Ng + tid];
    row[tid] = v;
    a.counts[(int64_t)q * a.Ng + tid] = hist[tid];
  }
  float z = 0.f;
  int rows = 0;
  if (tid < 64) {
    for (int b = b0 + lane; b < b1; b += 64) {
      z += w.z[b + q];
      rows += w.t[b + q];
    }
    z = wave_sum(z);
    rows = wave_sum(rows);
  }
  __syncthreads();
  if (tid >= 64) return;
  const float loss = sequence_loss(row, hist, a.Ng, rows);
  int done = 0;
  if (lane == 0) {
    a.tokens[q] = rows;
    __hip_atomic_store(w.loss + 4 * (int64_t)q, loss, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(w.loss + 4 * (int64_t)q + 1, rows > 0 ? z : 0.f, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(w.loss + 4 * (int64_t)q + 2, __int_as_float(rows), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    done = __hip_atomic_fetch_add(w.done, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
  }
  if (__builtin_amdgcn_readfirstlane(done) != a.Ns - 1) return;
  float balance = 0.f, squares = 0.f;
  int live = 0, total = 0;
  for (int i = lane; i < a.Ns; i += 64) {
    balance += __hip_atomic_load(w.loss + 4 * (int64_t)i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    squares += __hip_atomic_load(w.loss + 4 * (int64_t)i + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const int t = __float_as_int(__hip_atomic_load(w.loss + 4 * (int64_t)i + 2, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
    live += t > 0;
    total += t;
  }
  balance = wave_sum(balance);
  squares = wave_sum(squares);
  live = wave_sum(live);
  total = wave_sum(total);
  if (lane == 0) {
    a.loss[0] = balance / (float)max(live, 1);
    a.loss[1] = squares / (float)max(total, 1);
  }
}

// One row by LT lanes; ADD: on top of what dLogits holds.  Each wave finds out by itself
// how many sequences and rows take part, and its rows' sequences from the first one's.
template <typename T, typename TO, int LT, int E, bool ADD>
__global__ __launch_bounds__(256) void balance_bwd(BalanceArgs a) {
  const int tid = threadIdx.x, lane = tid & 63, li = tid % LT;
  const int first = blockIdx.x * (256 / LT) + (tid >> 6) * (64 / LT);  // the wave's first row
  const int t = first + lane / LT;
  if (first >= a.Nt) return;
  const bool ok = t < a.Nt;
  const int64_t row = ok ? t : first;
  float x[E], p[E];
  load_experts<E>(reinterpret_cast<const T*>(a.logits) + row * a.Ng, E * li, a.Ng, ok, -INFINITY, x);
  const int c = ok && li < a.Kt ? a.choice[row * a.Kt + li] : -1;
  const float d0 = a.dloss[0], d1 = a.dloss[1];
  int live = 0, total = 0;
  for (int i = lane; i < a.Ns; i += 64) {
    const int n = a.tokens[i];
    live += n > 0;
    total += n;
  }
  Sequences seq;
  seq.init(a.bounds, a.Ns);
  int q = seq.find(first);
  if (t >= seq.end) {  // a later one
    int lo = max(q, 0), hi = a.Ns + 1;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (a.bounds[mid] <= t) lo = mid + 1; else hi = mid;
    }
    q = lo - 1;
  }
  live = wave_sum(live);
  total = wave_sum(total);
  bool allowed;
  const float lse = softmax_row<LT, E>(x, p, &allowed);
  const bool in = some_choice<LT>(c >= 0 && c < a.Ng) && allowed && q >= 0 && q < a.Ns;
  const int s = in ? q : 0;
  const int32_t* const n = a.counts + (int64_t)s * a.Ng;
  float f[E], sum = 0.f, pf = 0.f;
  load_experts<E>(n, E * li, a.Ng, true, 0.f, f);
#pragma unroll
  for (int i = 0; i < E; ++i) sum += f[i];
  const float rows = (float)max(a.tokens[s], 1);
  // f stays the whole number n until the end: f - sum p f = (n - sum p n) / sum n
  const float choices = fmaxf(row_sum<LT>(sum), 1.f);
#pragma unroll
  for (int i = 0; i < E; ++i) pf += p[i] * f[i];
  pf = row_sum<LT>(pf);
  const float db = d0 * (float)a.Ng / ((float)max(live, 1) * rows * choices);
  const float dz = d1 * 2.f / (float)max(total, 1) * lse;
  if (!ok) return;
  TO* const out = reinterpret_cast<TO*>(a.dlogits) + row * a.Ng + E * li;
  float old[E];
  if constexpr (ADD) load_experts<E>(out, 0, a.Ng - E * li, true, 0.f, old);
  TO d[E];
#pragma unroll
  for (int i = 0; i < E; ++i) {
    // an expert without weight gets nothing, also where the losses are not finite
    float v = in && p[i] != 0.f ? p[i] * (db * (f[i] - pf) + dz) : 0.f;
    if constexpr (ADD) v += old[i];
    d[i] = from_f32<TO>(v);
  }
  if (E * (li + 1) <= a.Ng) {
    __builtin_memcpy(out, d, sizeof(d));
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (E * li + i < a.Ng) out[i] = d[i];
  }
}

template <typename T, int LT, int E> void launch_rows(const BalanceArgs& a, bool one, hipStream_t stream) {
  constexpr int NT = LT == 64 ? 512 : 1024;
  if (one) balance_rows<T, NT, LT, E, true><<<dim3(1), dim3(NT), 0, stream>>>(a);
  else balance_rows<T, NT, LT, E, false><<<dim3(a.nblocks), dim3(NT), 0, stream>>>(a);
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
  balance_sums<<<dim3(a.Ns), dim3(kSumThreads), 0, stream>>>(a);
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
  return Ns == 1 && Nt <= kBalanceOne ? 0 : ((nblocks + Ns) * (8 * Ng + 8) + 16 * Ns + 4 + 15) & ~(int64_t)15;
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
