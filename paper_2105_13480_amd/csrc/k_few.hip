// Products of few rows: grouped products with a few rows a group (serving
// steps), and adapted projections of up to some hundred rows (adapt_few).
//
// Such a product is bound by reading Ker once: a workgroup takes some 16 features
// by 16 rows, its waves share the contraction (each of four takes every fourth
// 256-byte run of k), and both operands go straight from memory to the MFMA
// registers, no LDS and no barrier until the waves' sums meet: 16 rows of 64
// bytes a load, four loads a run.  Rows beyond a tile's last read a row that
// is there; their results are not stored.  8 rows of four choices among 20 of 32
// experts of 1024 x 2048, bf16: 15.8 us, 84 MB at 5.3 TB/s.
#include "group_kernel.h"

namespace cnnlib {

namespace {

using namespace group;

// A run's operands: four loads of 16 rows by 64 bytes of each block.
template <typename T, int FB, int RB> struct Run {
  static constexpr int CE = 16 / (int)sizeof(T), LEN = 16 * CE;
  u32x4_t x[FB][4], y[RB][4];

  // All loads before anything that waits for one.
  __device__ __forceinline__ void load(const T* const (&xp)[FB], const T* const (&yp)[RB], int k0,
                                       int G) {
#pragma unroll
    for (int f = 0; f < FB; ++f)
#pragma unroll
      for (int i = 0; i < 4; ++i) __builtin_memcpy(&x[f][i], xp[f] + k0 + (4 * i + G) * CE, 16);
#pragma unroll
    for (int b = 0; b < RB; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) __builtin_memcpy(&y[b][i], yp[b] + k0 + (4 * i + G) * CE, 16);
    __builtin_amdgcn_sched_barrier(0);
  }
  __device__ __forceinline__ void multiply(f32x4_t (&acc)[FB][RB]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int f = 0; f < FB; ++f)
#pragma unroll
        for (int b = 0; b < RB; ++b) acc[f][b] = mma<T>(x[f][i], y[b][i], acc[f][b]);
    __builtin_amdgcn_sched_barrier(0);
  }
};

// acc[f][b] += the 16 features of block f by the 16 rows of block b, over the
// runs of k that `wave` of `nw` takes in [0, K).  x, y: this lane's feature
// row (l % 16) and row of each block.  Where registers allow, a run's loads
// are issued before the last one's products.
template <typename T, int FB, int RB>
__device__ __forceinline__ void few_rows_dot(const T* const (&x)[FB], const T* const (&y)[RB],
                                             int K, int wave, int nw, int lane,
                                             f32x4_t (&acc)[FB][RB]) {
  typedef Run<T, FB, RB> R;
  const int G = lane >> 4, step = nw * R::LEN;
  int k0 = wave * R::LEN;
  R a;
  if constexpr (FB + RB <= 3) {
    R b;
    if (k0 + R::LEN <= K) a.load(x, y, k0, G);
    for (; k0 + R::LEN <= K; k0 += 2 * step) {
      const bool second = k0 + step + R::LEN <= K;
      if (second) b.load(x, y, k0 + step, G);
      a.multiply(acc);
      if (!second) {
        k0 += step;
        break;
      }
      if (k0 + 2 * step + R::LEN <= K) a.load(x, y, k0 + 2 * step, G);
      b.multiply(acc);
    }
  } else {
    for (; k0 + R::LEN <= K; k0 += step) {
      a.load(x, y, k0, G);
      a.multiply(acc);
    }
  }
  if (k0 < K) {  // the last, shorter run: what lies past K is zero on both sides
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int k = k0 + (4 * i + G) * R::CE;
#pragma unroll
      for (int f = 0; f < FB; ++f) a.x[f][i] = load_end(x[f], k, K);
#pragma unroll
      for (int b = 0; b < RB; ++b) a.y[b][i] = load_end(y[b], k, K);
    }
    a.multiply(acc);
  }
}

// Leaves the waves' sums where block_sum finds them.  red: nw * FB * RB * 64 units.
template <int FB, int RB>
__device__ __forceinline__ void leave_sums(f32x4_t* red, const f32x4_t (&acc)[FB][RB], int wave,
                                           int nw, int lane) {
#pragma unroll
  for (int f = 0; f < FB; ++f)
#pragma unroll
    for (int b = 0; b < RB; ++b) red[((f * RB + b) * nw + wave) * 64 + lane] = acc[f][b];
  __syncthreads();
}
// The waves' sums of block f * RB + b added in wave order.
__device__ __forceinline__ f32x4_t block_sum(const f32x4_t* red, int block, int nw, int lane) {
  f32x4_t s = {0.f, 0.f, 0.f, 0.f};
  for (int w = 0; w < nw; ++w) s += red[(block * nw + w) * 64 + lane];
  return s;
}

// This lane's feature rows from m0 on; past the last, the last.
template <typename T, int FB>
__device__ __forceinline__ void feature_rows(const T* X, int64_t ld, int m0, int M, int l16,
                                             const T* (&x)[FB]) {
#pragma unroll
  for (int f = 0; f < FB; ++f) x[f] = X + (int64_t)min(m0 + 16 * f + l16, M - 1) * ld;
}

template <int FB, int RB>
__device__ __forceinline__ void clear(f32x4_t (&acc)[FB][RB]) {
#pragma unroll
  for (int f = 0; f < FB; ++f)
#pragma unroll
    for (int b = 0; b < RB; ++b) acc[f][b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
}

// A tile of 16 features by 16 rows of a group.
constexpr int kFewWaves = 4;

template <typename T, typename TO>
__global__ __launch_bounds__(64 * kFewWaves) void group_few(GroupArgs a) {
  constexpr int NW = kFewWaves;
  __shared__ f32x4_t red[NW * 64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  RowTile t;
  if (!find_tile<16>(a.off, a.Ng, a.N, (a.M + 15) / 16, blockIdx.x, 1, &t)) return;
  const int l16 = lane & 15;
  const int m0 = 16 * t.mt, n_valid = min(t.n1 - t.n0, 16);
  const bool live = t.g < a.Ng;

  const T* x[1];
  feature_rows<T, 1>(reinterpret_cast<const T*>(a.X) + (live ? t.g : 0) * a.xgroup, a.ldx, m0, a.M, l16, x);
  int64_t r = t.n0 + min(l16, n_valid - 1);
  if (a.rows) r = a.rows[r];
  const bool there = r >= 0 && r < a.Nsrc;  // this lane's row is one of In
  const T* const y[1] = {reinterpret_cast<const T*>(a.Y) + (there ? r : 0) * a.ldy};
  f32x4_t acc[1][1];
  clear(acc);
  if (live) few_rows_dot<T, 1, 1>(x, y, a.K, wave, NW, lane, acc);
  leave_sums(red, acc, wave, NW, lane);
  if (wave != 0 || l16 >= n_valid) return;
  f32x4_t s = block_sum(red, 0, NW, lane);
  if (!live || !there) s = f32x4_t{0.f, 0.f, 0.f, 0.f};
  store4(reinterpret_cast<TO*>(a.D) + (t.n0 + l16) * a.ldd, m0 + 4 * (lane >> 4), a.M, s);
}

// Few adapted rows, first launch: partial sums of both products that read In.
// The first workgroups, (tile of 16 rows, q, z), take every Q-th of the
// adapters that the tile's rows name, 16 DF ranks at a time, over slice z of
// k: H[z][n][r] = sum_k In[n, k] A[ids[n]][r, k].  The rest, (block of 64
// features, TN rows, slice of k): part[z][n][m] = sum_k In[n, k] Ker[m, k].
// Neither waits for the other, and a slice is short, so that most of Ker is
// asked for at once.  RING: the projection's operands go through a ring of
// four stages in LDS (rows on 4-byte boundaries; 64 features read In a quarter
// as often as 16), else straight to the registers.  48 rows of 4096 x 4096 with
// 24 adapters of rank 16, bf16: 12 us for 34 MB of Ker and 3 of A, and 4.5 for the
// second launch; 333 rows of 1001 x 1537 in fp32 26 us, where the matrix unit is
// the bound (1 GFLOP, 8 us if its share were the same on every CU) and 6.
constexpr int kSumWaves = 4, kSumDepth = 4, kSumFeatures = 64;

template <typename T, int DF, int TN, bool RING>
__global__ __launch_bounds__(64 * kSumWaves) void adapt_few_sums(GroupArgs a, AdaptArgs ad, FewPlan f) {
  constexpr int NW = kSumWaves, NT = 64 * NW, RB = TN / 16;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  f32x4_t* const red = reinterpret_cast<f32x4_t*>(smem);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, G = lane >> 4;
  int bid = blockIdx.x;
  if (bid < f.downs) {
    const int z = bid % f.kh, q0 = bid / f.kh % f.q, n0 = 16 * (bid / (f.kh * f.q));
    const int k_lo = z * f.hslice, n_valid = min(a.N - n0, 16);
    const int K = min(a.K - k_lo, f.hslice);
    const int n = n0 + min(l16, n_valid - 1);
    const int id = ad.ids[n];
    const T* y[1] = {reinterpret_cast<const T*>(a.Y) + (int64_t)n * a.ldy + k_lo};
    float* const H = ad.H + ((int64_t)z * a.N + n) * ad.Nl;
    int last = -1;
    for (int q = 0;; ++q) {
      int next = id > last && id < ad.Na ? id : 0x7fffffff;
      next = __builtin_amdgcn_readfirstlane(row16_min(next));
      if (next == 0x7fffffff) break;
      last = next;
      if (q % f.q != q0) continue;
      const T* const A = reinterpret_cast<const T*>(ad.A) + (int64_t)next * ad.Nl * a.K + k_lo;
      for (int r0 = 0; r0 < ad.Nl; r0 += 16 * DF) {
        const T* x[DF];
        f32x4_t acc[DF][1];
        feature_rows<T, DF>(A, a.K, r0, ad.Nl, l16, x);
        clear(acc);
        few_rows_dot<T, DF, 1>(x, y, K, wave, NW, lane, acc);
        leave_sums(red, acc, wave, NW, lane);
        if (l16 < n_valid && id == next)
          for (int b = wave; b < DF; b += NW)
            store4(H, r0 + 16 * b + 4 * G, ad.Nl, block_sum(red, b, NW, lane));
        __syncthreads();  // before the next sums overwrite `red`
      }
    }
    return;
  }
  bid -= f.downs;
  const int z = bid / (f.blocks * f.rtiles), k_lo = z * f.kslice;
  const int m0 = kSumFeatures * (bid % f.blocks), n0 = TN * (bid / f.blocks % f.rtiles);
  const int n_valid = min(a.N - n0, TN);
  const int K = min(a.K - k_lo, f.kslice);
  const T* const X = reinterpret_cast<const T*>(a.X) + k_lo;
  const T* const Y = reinterpret_cast<const T*>(a.Y) + n0 * a.ldy + k_lo;
  float* const part = ad.part + ((int64_t)z * a.N + n0) * a.M;
  if constexpr (RING) {
    constexpr int TK = 128 / (int)sizeof(T), XU = 8 * kSumFeatures, STAGE = XU + 8 * TN;
    u32x4_t* const ring = reinterpret_cast<u32x4_t*>(smem);
    Stager<T, true, kSumFeatures, NT, false> sx;
    Stager<T, true, TN, NT, false> sy;
    constexpr int COPIES = sx.NU + sy.NU;
    Reader<T, true, kSumFeatures, 1> rx;
    Reader<T, true, TN, RB> ry;
    rx.init(16 * wave, lane);
    ry.init(0, lane);
    sx.init(tid, X, a.ldx, m0, min(a.M - m0, kSumFeatures), nullptr, 0);
    sy.init(tid, Y, a.ldy, 0, n_valid, nullptr, 0);
    f32x4_t acc[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b) acc[b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    // as in group_tiles (AHEAD); where k ends inside a unit, its last stage goes through
    // registers
    const bool ends_inside = K % (16 / (int)sizeof(T)) != 0;
    const int n_st = ends_inside ? K / TK : (K + TK - 1) / TK;
    auto copy = [&](int s) __attribute__((always_inline)) {
      u32x4_t* const dst = ring + s % kSumDepth * STAGE;
      sx.copy(tid, dst, s * TK, a.ldx, s < n_st ? K : 0, nullptr, 0);
      sy.copy(tid, dst + XU, s * TK, a.ldy, s < n_st ? K : 0, nullptr, 0);
    };
    u32x4_t xf[2][1][2], yf[2][RB][2];  // of this stage and the next
    auto read = [&](int at, const u32x4_t* stage) __attribute__((always_inline)) {
      rx.read(stage, xf[at]);
      ry.read(stage + XU, yf[at]);
    };
    auto multiply = [&](int at) __attribute__((always_inline)) {
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int b = 0; b < RB; ++b) acc[b] = mma<T>(xf[at][0][ks], yf[at][b][ks], acc[b]);
    };
#pragma unroll
    for (int s = 0; s < kSumDepth; ++s) copy(s);
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(COPIES * (kSumDepth - 1)) : "memory");
    read(0, ring);
    auto step = [&](auto at, int s) __attribute__((always_inline)) {
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(COPIES * (kSumDepth - 2)) : "memory");
      read(1 - at, ring + (s + 1) % kSumDepth * STAGE);
      copy(s + kSumDepth);
      multiply(at);
      interleave<T, RB * 2 * (sizeof(T) == 4 ? 4 : 1)>();
    };
    int s = 0;
    for (; s + 2 <= n_st; s += 2) {
      step(std::integral_constant<int, 0>{}, s);
      step(std::integral_constant<int, 1>{}, s + 1);
    }
    if (s < n_st) step(std::integral_constant<int, 0>{}, s);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the trailing (empty) copies
    if (ends_inside && n_st * TK < K) {
      sx.load(n_st * TK, a.ldx, K, nullptr, 0);
      sy.load(n_st * TK, a.ldy, K, nullptr, 0);
      __syncthreads();
      sx.commit(tid, ring, n_st * TK, a.ldx, K, nullptr, 0);
      sy.commit(tid, ring + XU, n_st * TK, a.ldy, K, nullptr, 0);
      __syncthreads();
      read(0, ring);
      multiply(0);
    }
#pragma unroll
    for (int b = 0; b < RB; ++b) {
      const int n = 16 * b + l16;
      if (n < n_valid) store4(part + (int64_t)n * a.M, m0 + 16 * wave + 4 * G, a.M, acc[b]);
    }
  } else {
    const T* y[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b) y[b] = Y + (int64_t)min(16 * b + l16, n_valid - 1) * a.ldy;
    // two blocks of features at a time
    for (int m = m0; m < min(m0 + kSumFeatures, a.M); m += 32) {
      const T* x[2];
      feature_rows<T, 2>(X, a.ldx, m, a.M, l16, x);
      f32x4_t acc[2][RB];
      clear(acc);
      few_rows_dot<T, 2, RB>(x, y, K, wave, NW, lane, acc);
      leave_sums(red, acc, wave, NW, lane);
      for (int blk = wave; blk < 2 * RB; blk += NW) {
        const int n = 16 * (blk % RB) + l16;
        if (n < n_valid)
          store4(part + (int64_t)n * a.M, m + 16 * (blk / RB) + 4 * G, a.M, block_sum(red, blk, NW, lane));
      }
      __syncthreads();
    }
  }
}

// Second launch: Out = the slices' sums, in order, and each row's low-rank
// part in fp32; a thread has four features of a row.
template <typename T, typename TO, int KS, int KH>
__global__ __launch_bounds__(256) void adapt_few_out(GroupArgs a, AdaptArgs ad) {
  int n, u;
  if (!unit_of_thread(blockIdx.x, threadIdx.x, a.N, (a.M + 3) / 4, &n, &u)) return;
  const int m = 4 * u;
  const int left = a.M - 1 - m;  // features after the first
  f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int z = 0; z < KS; ++z) {
    const float* const src = ad.part + ((int64_t)z * a.N + n) * a.M + m;
    f32x4_t p;
    if (left >= 3) {
      __builtin_memcpy(&p, src, 16);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) p[e] = src[min(e, left)];
    }
    sum += p;
  }
  const int id = ad.ids[n];
  if (id >= 0 && id < ad.Na) {
    const T* const B = reinterpret_cast<const T*>(ad.B) + ((int64_t)id * a.M + m) * ad.Nl;
    const float* const H = ad.H + (int64_t)n * ad.Nl;
    const int64_t hz = (int64_t)a.N * ad.Nl;
    f32x4_t d = {0.f, 0.f, 0.f, 0.f};
    auto ranks = [&](auto count, int r) __attribute__((always_inline)) {
      constexpr int R = count.value;
      float p[KH][R];
      T b[4][R];
#pragma unroll
      for (int z = 0; z < KH; ++z) __builtin_memcpy(p[z], H + z * hz + r, sizeof(p[z]));
#pragma unroll
      for (int e = 0; e < 4; ++e) __builtin_memcpy(b[e], B + (int64_t)min(e, left) * ad.Nl + r, sizeof(b[e]));
#pragma unroll
      for (int t = 0; t < R; ++t) {
        float h = p[0][t];
#pragma unroll
        for (int z = 1; z < KH; ++z) h += p[z][t];
#pragma unroll
        for (int e = 0; e < 4; ++e) d[e] += h * to_f32(b[e][t]);
      }
    };
    int r = 0;
#pragma unroll 2
    for (; r + 8 <= ad.Nl; r += 8) ranks(std::integral_constant<int, 8>{}, r);
    if (r + 4 <= ad.Nl) {
      ranks(std::integral_constant<int, 4>{}, r);
      r += 4;
    }
    if (r + 2 <= ad.Nl) {
      ranks(std::integral_constant<int, 2>{}, r);
      r += 2;
    }
    if (r < ad.Nl) ranks(std::integral_constant<int, 1>{}, r);
    const float s = ad.scales ? ad.scales[id] : 1.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] += s * d[e];
  }
  store4(reinterpret_cast<TO*>(a.D) + (int64_t)n * a.ldd, m, a.M, sum);
}

template <typename T, typename TO> hipError_t launch_few(const GroupArgs& a, hipStream_t stream) {
  const int64_t mt = (a.M + 15) / 16, parts = a.Ng + 1 < a.N ? a.Ng + 1 : a.N;
  const int64_t blocks = (a.N / 16 + parts) * mt;
  const hipError_t e = grid_fits(blocks, 64 * kFewWaves);
  if (e != hipSuccess) return e;
  group_few<T, TO><<<dim3((uint32_t)blocks), dim3(64 * kFewWaves), 0, stream>>>(a);
  return hipGetLastError();
}

template <typename T, int DF, int TN>
void launch_sums(const GroupArgs& a, const AdaptArgs& ad, const FewPlan& f, hipStream_t stream) {
  const dim3 grid((uint32_t)(f.downs + f.blocks * f.rtiles * f.ks)), block(64 * kSumWaves);
  const int red = 16 * 64 * kSumWaves * (DF > TN / 8 ? DF : TN / 8);
  if (adapt_few_ring(a.X, a.Y, a.K, sizeof(T))) {
    const int lds = kSumDepth * 8 * (kSumFeatures + TN) * 16;
    adapt_few_sums<T, DF, TN, true><<<grid, block, lds > red ? lds : red, stream>>>(a, ad, f);
  } else {
    adapt_few_sums<T, DF, TN, false><<<grid, block, red, stream>>>(a, ad, f);
  }
}

template <typename T, typename TO, int KS>
void launch_out(const GroupArgs& a, const AdaptArgs& ad, const FewPlan& f, hipStream_t stream) {
  const int64_t threads = (int64_t)a.N * ((a.M + 3) / 4);
  const dim3 grid((uint32_t)((threads + 255) / 256)), block(256);
  if (f.kh == 1) adapt_few_out<T, TO, KS, 1><<<grid, block, 0, stream>>>(a, ad);
  else adapt_few_out<T, TO, KS, 4><<<grid, block, 0, stream>>>(a, ad);
}

template <typename T, typename TO>
hipError_t launch_adapt_typed(const GroupArgs& a, const AdaptArgs& ad, hipStream_t stream) {
  constexpr int RUN = 256 / (int)sizeof(T);
  FewPlan f = adapt_few_plan(a.N, a.K, a.M, sizeof(T));
  // slices of k of whole runs; the last may be shorter or empty
  f.hslice = ((a.K + f.kh - 1) / f.kh + RUN - 1) / RUN * RUN;
  f.kslice = ((a.K + f.ks - 1) / f.ks + RUN - 1) / RUN * RUN;
  f.q = ad.Na < 16 ? ad.Na : 16;
  f.downs = (a.N + 15) / 16 * f.q * f.kh;
  // both launches before the first
  hipError_t e = grid_fits(f.downs + (int64_t)f.blocks * f.rtiles * f.ks, 64 * kSumWaves);
  if (e == hipSuccess) e = grid_fits(((int64_t)a.N * ((a.M + 3) / 4) + 255) / 256, 256);
  if (e != hipSuccess) return e;
  if (a.N <= 32) {
    if (ad.Nl <= 16) launch_sums<T, 1, 32>(a, ad, f, stream);
    else launch_sums<T, 4, 32>(a, ad, f, stream);
  } else {
    if (ad.Nl <= 16) launch_sums<T, 1, 64>(a, ad, f, stream);
    else launch_sums<T, 4, 64>(a, ad, f, stream);
  }
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  switch (f.ks) {
    case 1: launch_out<T, TO, 1>(a, ad, f, stream); break;
    case 2: launch_out<T, TO, 2>(a, ad, f, stream); break;
    case 4: launch_out<T, TO, 4>(a, ad, f, stream); break;
    default: launch_out<T, TO, 8>(a, ad, f, stream); break;
  }
  return hipGetLastError();
}

}  // namespace

// Up to eight rows a group, aligned rows, and two runs of k for each of the
// four waves: decoding steps.  bf16, at 32 rows of 20 groups, k 2048, 1024
// features: 16.1 us here, 17.2 by 64 x 32 tiles; with k 512 (49 rows of 38
// groups, 4096 features) 42 and 33; at 16 rows a group (512 rows of 28, k
// 1024, 4096 features) 60 and 49; odd k (1039, five rows a group) 40 and 21.
bool group_few_fits(const GroupArgs& a, int dtype) {
  return a.N <= 8 * (int64_t)a.Ng && a.K * in_bytes(dtype) >= 2048 && a.K * in_bytes(dtype) % 16 == 0 &&
         (((uintptr_t)a.X | (uintptr_t)a.Y) & 15) == 0;
}

hipError_t launch_group_few(const GroupArgs& a, int dtype, hipStream_t stream) {
  switch (dtype) {
    case CNN_F32: return launch_few<float, float>(a, stream);
    case CNN_BF16: return launch_few<bf16_t, float>(a, stream);
    default: return launch_few<bf16_t, bf16_t>(a, stream);
  }
}

// bf16 / fp32, us, rows as they come against the order of the adapters: 256 rows of
// 4096 x 4096, rank 16, 29 / 95 and 36 / 122; 400 rows 44 / 173 and 42 / 182; 333 of
// 2048 x 2048, rank 32, 25 / 66 and 27 / 68; 512 rows 32 / 83 and 27 / 77, but of
// 512 x 512, rank 8, 9.2 / 14 and 14 / 20.  Higher ranks were not measured and are
// no part of the rule.  Rows that are on no 4-byte boundary go
// straight to the registers: 1001 x 1537, rank 12, in bf16 at 128 rows 18 and 22, at
// 256 28 and 23.
bool adapt_few(int64_t Nt, int64_t Nc, int64_t Nk, bool ring) {
  if (!ring) return Nt <= 192;
  return Nt <= 352 || (Nt <= kFewRows && Nc * Nk <= 1 << 20);
}
bool adapt_few_ring(const void* Ker, const void* In, int64_t Nc, int es) {
  return (((uintptr_t)Ker | (uintptr_t)In) & 3) == 0 && Nc * es % 4 == 0;
}

FewPlan adapt_few_plan(int64_t Nt, int64_t Nc, int64_t Nk, int es) {
  FewPlan f = {};
  f.blocks = (int32_t)((Nk + kSumFeatures - 1) / kSumFeatures);
  f.rtiles = Nt <= 32 ? 1 : (int32_t)((Nt + 63) / 64);
  // slices of k, of some 200 values at least: a workgroup for each CU, or two of
  // slices that still have 16 stages, since the adapters' workgroups leave the
  // CUs unequal shares (256 workgroups of whole rows of 4096 in fp32: 156 us, two
  // slices 92; in bf16 32 and 27; short slices cost more than they even out:
  // 128 rows of 2048 x 2048 in bf16 15.2 us by four, 17.8 by eight)
  f.ks = 1;
  const int64_t wgs = (int64_t)f.blocks * f.rtiles;
  while (f.ks < 8 && Nc >= 384 * f.ks &&
         (f.ks * wgs < 256 || (f.ks * wgs < 512 && Nc * es >= 4096 * f.ks)))
    f.ks *= 2;
  f.kh = Nc >= 1024 ? 4 : 1;
  return f;
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
