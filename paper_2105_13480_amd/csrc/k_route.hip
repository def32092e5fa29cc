// The router: choice of experts, their weights, the grouped order, and the
// router's gradient.
//
// Choice: a row's logits are held by LT lanes (16, or 64 for more than 256
// experts), E of them a lane, as unsigned keys whose order is the logits';
// not-allowed ones (-inf, NaN) have key 0.  Each of the Kt largest is a
// maximum over the lanes by data-parallel moves, so every lane knows it: in
// bf16 of (16-bit key, ~expert) as one value, in fp32 of the key and then of
// the lowest expert that has it; ties go to the lowest expert.  Four rows a
// wave.  Bound by its instructions, some 70 a choice (16384 rows of 128 experts,
// eight choices, bf16: 7.6 to 8.8 us for 4 MB of logits, half of it issuing them on
// four waves a SIMD) and, for few rows, by the launch: up to 64 rows are chosen and
// ordered in one (16 rows of 32: 4 us).
//
// Order: a counting sort, stable.  A workgroup owns a chunk of rows; the
// chunk's counts per expert go to the workspace, then every workgroup adds up
// the counts before its own (all of them are read by each: at most 256 chunks
// by Ng, from L2, in place of a scan launch; 131072 pairs of 128 experts 6.9 us).
// Within 64 rows a place is the
// number of set bits below the row's in the expert's 64-bit mask: a row names
// an expert at most once, so no atomic's order shows in the result.
#include "common.h"
#include "routed.h"

namespace cnnlib {

namespace {

constexpr int kMaxExperts = 1024;
constexpr int kOrderThreads = 1024;

// Order-preserving key of a logit; 0: not allowed.
__device__ __forceinline__ uint32_t logit_key(float x) {
  if (!(x > -INFINITY)) return 0u;
  const uint32_t u = __float_as_uint(x + 0.f);  // -0 as +0: they tie
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_logit(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

template <int CTRL> __device__ __forceinline__ uint32_t dpp(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
// Exchange with the lane that step S of a butterfly over 16 lanes pairs: within
// pairs, quads, halves of 8 and 16 (each step's source holds the other side).
template <int S> __device__ __forceinline__ uint32_t partner16(uint32_t v) {
  if constexpr (S == 0) return dpp<0xb1>(v);        // quad_perm 1,0,3,2
  else if constexpr (S == 1) return dpp<0x4e>(v);   // quad_perm 2,3,0,1
  else if constexpr (S == 2) return dpp<0x141>(v);  // row_half_mirror
  else return dpp<0x140>(v);                        // row_mirror
}

template <int LT, typename F> __device__ __forceinline__ void butterfly(F step) {
  step([](uint32_t v) { return partner16<0>(v); });
  step([](uint32_t v) { return partner16<1>(v); });
  step([](uint32_t v) { return partner16<2>(v); });
  step([](uint32_t v) { return partner16<3>(v); });
  if constexpr (LT == 64) {
    step([](uint32_t v) { return (uint32_t)__shfl_xor((int)v, 16); });
    step([](uint32_t v) { return (uint32_t)__shfl_xor((int)v, 32); });
  }
}

template <int LT> __device__ __forceinline__ float row_sum(float s) {
  butterfly<LT>([&](auto from) { s += __uint_as_float(from(__float_as_uint(s))); });
  return s;
}

// e^(x - m), 1 at x = m (also where both are infinite).
__device__ __forceinline__ float weight_of(float x, float m) { return x == m ? 1.f : expf(x - m); }

// The largest (MAX) or least v of the row's lanes, in all of them.
template <int LT, bool MAX> __device__ __forceinline__ uint32_t row_best(uint32_t v) {
  butterfly<LT>([&](auto from) {
    const uint32_t o = from(v);
    v = MAX ? (o > v ? o : v) : (o < v ? o : v);
  });
  return v;
}

// Choice and weights of one row: lane j holds choice j (-1: none) and its weight.
template <typename T, int LT, int E>
__device__ __forceinline__ void choose_row(const T* logits, int Ng, int Kt, int over_all, int li,
                                           bool row_ok, int* choice, float* gate) {
  constexpr bool PACK = sizeof(T) == 2;
  uint32_t key[E];  // PACK: key in the upper half, ~expert in the lower
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const int e = i * LT + li;
    key[i] = row_ok && e < Ng ? logit_key(to_f32(logits[e])) : 0u;
  }
  float top = 0.f, total = 0.f;
  if (over_all) {
    uint32_t best = key[0];
#pragma unroll
    for (int i = 1; i < E; ++i) best = key[i] > best ? key[i] : best;
    best = row_best<LT, true>(best);
    top = best ? key_logit(best) : 0.f;
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (key[i] != 0u) s += weight_of(key_logit(key[i]), top);
    total = row_sum<LT>(s);
  }
  if constexpr (PACK)
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (key[i] != 0u) key[i] = (key[i] & 0xffff0000u) | (0xffffu ^ (uint32_t)(i * LT + li));
  uint32_t my_key = 0;
  int mine = -1;
  for (int j = 0; j < Kt; ++j) {
    uint32_t best = key[0];
#pragma unroll
    for (int i = 1; i < E; ++i) best = key[i] > best ? key[i] : best;
    best = row_best<LT, true>(best);
    int e;
    if constexpr (PACK) {
      e = (int)(0xffffu ^ (best & 0xffffu));
#pragma unroll
      for (int i = 0; i < E; ++i) key[i] = key[i] == best ? 0u : key[i];
      // the logit's key again: a negative bf16's has ones below
      best = best & 0x80000000u || !best ? best & 0xffff0000u : best | 0xffffu;
    } else {
      uint32_t lowest = ~0u;
#pragma unroll
      for (int i = E - 1; i >= 0; --i) lowest = key[i] == best ? (uint32_t)(i * LT + li) : lowest;
      e = (int)row_best<LT, false>(lowest);
#pragma unroll
      for (int i = 0; i < E; ++i) key[i] = e == i * LT + li ? 0u : key[i];
    }
    if (best != 0u) {
      const float x = key_logit(best);
      if (!over_all) {
        if (j == 0) top = x;
        total += weight_of(x, top);
      }
      if (li == j) {
        my_key = best;
        mine = e;
      }
    }
  }
  *choice = mine;
  *gate = mine >= 0 ? weight_of(key_logit(my_key), top) / total : 0.f;
}

// Shared memory of the ordering step.
struct OrderShared {
  int32_t base[kMaxExperts + 1];
  unsigned long long mask[kMaxExperts + 1];
  int32_t part[16];
};

// Places of the pairs of rows [t0, t1), in order, and what lies past the last
// pair.  All threads of the workgroup; s.base holds the first place of each key
// (key Ng: the rows without one).
__device__ void place_rows(const OrderArgs& o, OrderShared& s, int t0, int t1) {
  const int tid = threadIdx.x, nt = blockDim.x, Ng = o.Ng;
  const int bins = Ng + (o.place_none ? 1 : 0);
  for (int tb = t0; tb < t1; tb += 64) {
    for (int e = tid; e < bins; e += nt) s.mask[e] = 0ull;
    __syncthreads();
    const int n = min(64, t1 - tb) * o.Kt;
    for (int i = tid; i < n; i += nt) {
      int e = o.key[(int64_t)tb * o.Kt + i];
      if (e < 0 || e >= Ng) e = Ng;
      if (e < bins) atomicOr(&s.mask[e], 1ull << (i / o.Kt));
    }
    __syncthreads();
    for (int i = tid; i < n; i += nt) {
      const int64_t at = (int64_t)tb * o.Kt + i;
      const int r = i / o.Kt;
      int e = o.key[at];
      if (e < 0 || e >= Ng) e = Ng;
      int p = -1;
      if (e < bins) {
        p = s.base[e] + __popcll(s.mask[e] & ((1ull << r) - 1ull));
        o.rows[p] = tb + r;
        if (o.keys) o.keys[p] = e < Ng ? e : -1;
      }
      if (o.slots) o.slots[at] = p;
    }
    __syncthreads();
    for (int e = tid; e < bins; e += nt) s.base[e] += __popcll(s.mask[e]);
    __syncthreads();
  }
}

// s.base = exclusive sums of `count` over the keys; returns their total.
__device__ int scan_keys(OrderShared& s, int count, int bins) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int v = count;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  if (lane == 63) s.part[wave] = v;
  __syncthreads();
  int before = 0, total = 0;
  for (int w = 0; w < kOrderThreads / 64; ++w) {
    before += w < wave ? s.part[w] : 0;
    total += s.part[w];
  }
  if (tid < bins) s.base[tid] = before + v - count;
  __syncthreads();
  return total;
}

// One workgroup's choices; in one launch with the order where one workgroup
// takes all rows (ONE), else its counts go to the workspace.
template <typename T, int LT, int E, bool ONE>
__global__ __launch_bounds__(kOrderThreads) void route_choose(RouteArgs a, OrderArgs o) {
  __shared__ OrderShared s;
  __shared__ int32_t hist[kMaxExperts];
  const int tid = threadIdx.x, li = tid % LT;
  const int t0 = blockIdx.x * o.chunk, t1 = min(o.Nt, t0 + o.chunk);
  for (int e = tid; e < o.Ng; e += kOrderThreads) hist[e] = 0;
  __syncthreads();
  for (int t = t0 + tid / LT; t - tid / LT < t1; t += kOrderThreads / LT) {
    int choice;
    float gate;
    const bool ok = t < t1;
    choose_row<T, LT, E>(reinterpret_cast<const T*>(a.logits) + (int64_t)(ok ? t : 0) * o.Ng, o.Ng,
                         o.Kt, a.over_all, li, ok, &choice, &gate);
    if (ok && li < o.Kt) {
      a.choice[(int64_t)t * o.Kt + li] = choice;
      a.gates[(int64_t)t * o.Kt + li] = gate;
      if (choice >= 0) atomicAdd(&hist[choice], 1);
    }
  }
  __syncthreads();
  if constexpr (ONE) {
    const int total = scan_keys(s, tid < o.Ng ? hist[tid] : 0, o.Ng);
    for (int e = tid; e < o.Ng; e += kOrderThreads) o.off[e] = s.base[e];
    if (tid == 0) o.off[o.Ng] = total;
    for (int p = total + tid; p < o.Nt * o.Kt; p += kOrderThreads) o.rows[p] = -1;
    __syncthreads();  // s.base is read before it moves; choices are visible
    place_rows(o, s, t0, t1);
  } else {
    for (int e = tid; e < o.Ng; e += kOrderThreads) o.counts[(int64_t)blockIdx.x * o.Ng + e] = hist[e];
  }
}

// Counts of the keys of one chunk of rows.
__global__ __launch_bounds__(kOrderThreads) void order_count(OrderArgs o) {
  __shared__ int32_t hist[kMaxExperts];
  const int tid = threadIdx.x;
  const int t0 = blockIdx.x * o.chunk, t1 = min(o.Nt, t0 + o.chunk);
  for (int e = tid; e < o.Ng; e += kOrderThreads) hist[e] = 0;
  __syncthreads();
  for (int64_t i = (int64_t)t0 * o.Kt + tid; i < (int64_t)t1 * o.Kt; i += kOrderThreads) {
    const int e = o.key[i];
    if (e >= 0 && e < o.Ng) atomicAdd(&hist[e], 1);
  }
  __syncthreads();
  for (int e = tid; e < o.Ng; e += kOrderThreads) o.counts[(int64_t)blockIdx.x * o.Ng + e] = hist[e];
}

// Places of one chunk of rows, from the counts of all chunks, or (KEYS: few
// rows) from all keys.
template <bool KEYS>
__global__ __launch_bounds__(kOrderThreads) void order_place(OrderArgs o) {
  __shared__ OrderShared s;
  __shared__ int32_t whole[kMaxExperts], ahead[kMaxExperts];
  const int tid = threadIdx.x, Ng = o.Ng, b = blockIdx.x;
  const int t0 = b * o.chunk, t1 = min(o.Nt, t0 + o.chunk);
  for (int e = tid; e < Ng; e += kOrderThreads) whole[e] = ahead[e] = 0;
  __syncthreads();
  if constexpr (KEYS) {
    for (int i = tid; i < o.Nt * o.Kt; i += kOrderThreads) {
      const int e = o.key[i];
      if (e < 0 || e >= Ng) continue;
      atomicAdd(&whole[e], 1);
      if (i < t0 * o.Kt) atomicAdd(&ahead[e], 1);
    }
  }
  // thread (x, y): key x of every ny-th chunk
  const int ny = max(1, kOrderThreads / Ng), x = tid % Ng, y = tid / Ng;
  if (!KEYS && y < ny) {
    int w = 0, h = 0;
#pragma unroll 8
    for (int c = y; c < o.nblocks; c += ny) {
      const int v = o.counts[(int64_t)c * Ng + x];
      w += v;
      h += c < b ? v : 0;
    }
    atomicAdd(&whole[x], w);
    atomicAdd(&ahead[x], h);
  }
  __syncthreads();
  const int total = scan_keys(s, tid < Ng ? whole[tid] : 0, Ng);
  if (b == 0) {
    for (int e = tid; e < Ng; e += kOrderThreads) o.off[e] = s.base[e];
    if (tid == 0) o.off[Ng] = total;
  }
  __syncthreads();
  for (int e = tid; e < Ng; e += kOrderThreads) s.base[e] += ahead[e];
  if (o.place_none) {
    // rows without a key before this chunk: those before it less those with one
    if (tid == 0) {
      int with = 0;
      for (int e = 0; e < Ng; ++e) with += ahead[e];
      s.base[Ng] = total + t0 * o.Kt - with;
    }
  } else {
    const int64_t step = (int64_t)o.nblocks * kOrderThreads;
    for (int64_t p = total + (int64_t)b * kOrderThreads + tid; p < (int64_t)o.Nt * o.Kt; p += step)
      o.rows[p] = -1;
  }
  __syncthreads();
  place_rows(o, s, t0, t1);
}

// dLogits of one row from the gradients of its weights: with p the softmax the
// weights came from, dl[e] = p[e] ([e chosen] dg_e - sum_j g_j dg_j).  16 or 64
// lanes a row as in the choice; logits are read and gradients written once (8192
// rows of 64 experts, fp32: 4.6 us, two thirds of it launch and latency).
template <typename T, typename TO, int LT, int E>
__global__ __launch_bounds__(256) void route_bwd(const T* logits, const int32_t* choice,
                                                 const float* gates, const float* dgates,
                                                 TO* dlogits, int64_t Nt, int Ng, int Kt,
                                                 int over_all) {
  const int li = threadIdx.x % LT;
  const int64_t t = (int64_t)blockIdx.x * (256 / LT) + threadIdx.x / LT;
  const bool ok = t < Nt;
  const int64_t row = ok ? t : 0;
  const T* const l = logits + row * Ng;

  float p[E];
#pragma unroll
  for (int i = 0; i < E; ++i) p[i] = 0.f;
  if (over_all) {
    float x[E], m = -INFINITY;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int e = i * LT + li;
      const float v = e < Ng ? to_f32(l[e]) : -INFINITY;
      x[i] = v > -INFINITY ? v : -INFINITY;
      m = fmaxf(m, x[i]);
    }
    butterfly<LT>([&](auto from) { m = fmaxf(m, __uint_as_float(from(__float_as_uint(m)))); });
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      p[i] = x[i] > -INFINITY ? weight_of(x[i], m) : 0.f;
      s += p[i];
    }
    s = row_sum<LT>(s);
    const float inv = s > 0.f ? 1.f / s : 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) p[i] *= inv;
  }
  float inner = 0.f;
  for (int j = 0; j < Kt; ++j) {
    const int e = choice[row * Kt + j];
    if (e >= 0 && e < Ng) inner += gates[row * Kt + j] * dgates[row * Kt + j];
  }
  float d[E];
  bool some = false;
#pragma unroll
  for (int i = 0; i < E; ++i) d[i] = p[i] != 0.f ? -p[i] * inner : 0.f;  // inner may be infinite
  for (int j = 0; j < Kt; ++j) {
    const int e = choice[row * Kt + j];
    if (e < 0 || e >= Ng) continue;
    some = true;
    const float g = gates[row * Kt + j], dg = dgates[row * Kt + j];
    const float add = over_all ? g * dg : g * (dg - inner);
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (e == i * LT + li) d[i] += add;
  }
  if (ok)
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int e = i * LT + li;
      if (e < Ng) dlogits[row * Ng + e] = from_f32<TO>(some ? d[i] : 0.f);
    }
}

template <typename T, bool ONE>
hipError_t launch_choose(const RouteArgs& a, const OrderArgs& o, hipStream_t stream) {
  const dim3 grid(o.nblocks), block(kOrderThreads);
  const int per = (o.Ng + 15) / 16;
  if (per <= 2) route_choose<T, 16, 2, ONE><<<grid, block, 0, stream>>>(a, o);
  else if (per <= 4) route_choose<T, 16, 4, ONE><<<grid, block, 0, stream>>>(a, o);
  else if (per <= 8) route_choose<T, 16, 8, ONE><<<grid, block, 0, stream>>>(a, o);
  else if (per <= 16) route_choose<T, 16, 16, ONE><<<grid, block, 0, stream>>>(a, o);
  else route_choose<T, 64, 16, ONE><<<grid, block, 0, stream>>>(a, o);
  return hipGetLastError();
}

template <typename T, typename TO>
hipError_t launch_bwd(const void* logits, const int32_t* choice, const float* gates,
                      const float* dgates, void* dlogits, int64_t Nt, int Ng, int Kt, int over_all,
                      hipStream_t stream) {
  const T* const l = reinterpret_cast<const T*>(logits);
  TO* const d = reinterpret_cast<TO*>(dlogits);
  const int rows = Ng <= 256 ? 16 : 4;  // of a workgroup
  const int64_t blocks = (Nt + rows - 1) / rows;
  const hipError_t e = grid_fits(blocks, 256);
  if (e != hipSuccess) return e;
  auto* const k = Ng <= 64 ? route_bwd<T, TO, 16, 4> : Ng <= 256 ? route_bwd<T, TO, 16, 16> : route_bwd<T, TO, 64, 16>;
  k<<<dim3((uint32_t)blocks), dim3(256), 0, stream>>>(l, choice, gates, dgates, d, Nt, Ng, Kt, over_all);
  return hipGetLastError();
}

}  // namespace

void order_blocks(int64_t Nt, int32_t* chunk, int32_t* nblocks) {
  // whole runs of 64 rows, at most 256 workgroups, none of them empty
  const int64_t runs = Nt > 0 ? (Nt + 63) / 64 : 1, per = (runs + 255) / 256;
  *chunk = (int32_t)(per * 64);
  *nblocks = (int32_t)((runs + per - 1) / per);
}

hipError_t launch_order(const OrderArgs& o, hipStream_t stream) {
  // every workgroup counts all keys: two a thread, against another launch (at
  // eight a thread 16.6 us, in two launches 9.6)
  if ((int64_t)o.Nt * o.Kt <= 2 * kOrderThreads) {
    order_place<true><<<dim3(o.nblocks), dim3(kOrderThreads), 0, stream>>>(o);
    return hipGetLastError();
  }
  order_count<<<dim3(o.nblocks), dim3(kOrderThreads), 0, stream>>>(o);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  order_place<false><<<dim3(o.nblocks), dim3(kOrderThreads), 0, stream>>>(o);
  return hipGetLastError();
}

hipError_t launch_route(const RouteArgs& a, const OrderArgs& o, bool bf16, hipStream_t stream) {
  if (o.nblocks == 1)
    return bf16 ? launch_choose<bf16_t, true>(a, o, stream) : launch_choose<float, true>(a, o, stream);
  const hipError_t e =
      bf16 ? launch_choose<bf16_t, false>(a, o, stream) : launch_choose<float, false>(a, o, stream);
  if (e != hipSuccess) return e;
  order_place<false><<<dim3(o.nblocks), dim3(kOrderThreads), 0, stream>>>(o);
  return hipGetLastError();
}

hipError_t launch_route_bwd(const void* logits, const int32_t* choice, const float* gates,
                            const float* dgates, void* dlogits, int64_t Nt, int Ng, int Kt,
                            int dtype, int over_all, hipStream_t stream) {
  switch (dtype) {
    case CNN_F32:
      return launch_bwd<float, float>(logits, choice, gates, dgates, dlogits, Nt, Ng, Kt, over_all, stream);
    case CNN_BF16:
      return launch_bwd<bf16_t, float>(logits, choice, gates, dgates, dlogits, Nt, Ng, Kt, over_all, stream);
    default:
      return launch_bwd<bf16_t, bf16_t>(logits, choice, gates, dgates, dlogits, Nt, Ng, Kt, over_all, stream);
  }
}

}  // namespace cnnlib
