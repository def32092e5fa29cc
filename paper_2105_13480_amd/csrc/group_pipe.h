// The pipelined tile kernel of the grouped products: 256 x 256 results of
// bf16 operands with rows on 4-byte boundaries, k (or, where it is last, the
// operand's own index) of whole units of 16 bytes.
//
// Eight waves of 128 (m) x 64 (n) results, two on each SIMD.  A stage is 64 of
// k: 64 KB of LDS in four halves (128 rows of Y, 128 of X, the other 128 of
// each), two stages in LDS.  A wave's results are four quarters, one per half
// of X and of Y, and a stage is four phases of one quarter, 16 MFMAs:
//   phase  reads from LDS       copies              products
//     0    X half 0             X half 1 of s + 1   X0 Y0
//     1    Y half 1             Y half 0 of s + 2   X0 Y1
//     2    X half 1             X half 0 of s + 2   X1 Y1
//     3    Y half 0 of s + 1    Y half 1 of s + 2   X1 Y0
// so that no phase reads more than its products take (8 or 4 KB a wave at 128
// bytes a clock against 256 clocks).  A phase is two slots between barriers,
// memory then products; waves 4 to 7 run one slot behind waves 0 to 3, so on
// each SIMD one wave feeds the matrix unit while the other reads.  A wave's
// reads are done by the end of its products slot, which the later waves end
// two slots after the earlier ones began to read: from the second phase after
// a read on, the half may be copied over.  That is six phases before it is
// read again, so every memory slot waits for all but its wave's last ten
// copies (copies beyond the end of k read zeros: the count always holds).
//
// Measured (bf16 results): 8192^3 711 us, 1546 TFLOP/s forward, 800 the gradient
// of In, 889 that of Ker; the transposing reads are waited for in their slot.  A
// stage takes 1.33 us (1.6 with both operands transposed), a tile's start and
// results 10: at k = 2048 and whole rounds of the 256 CUs (2048 tiles) 432 us,
// 1272 TFLOP/s, and a round more where the tiles do not divide.  Workgroups that
// stay for several tiles gained nothing: the results of one tile and the first
// copies of the next are still the same waves' work.
#pragma once

#include <type_traits>

#include "group_kernel.h"

namespace cnnlib {
namespace group {

constexpr int kPipeHalf = 1024;                  // units of a half: 128 rows of 64 of k
constexpr int kPipeRows = 4096;                  // source rows kept in LDS (gathered k)
constexpr int kPipeLds = 8 * kPipeHalf * 16;     // two stages
enum Half { kY0 = 0, kX0 = 1, kY1 = 2, kX1 = 3 };

// One operand: its copies to LDS and its reads from there.  KC: k last, rows
// may be gathered; else the tile's own index last, rows of k may be gathered.
// NB: blocks of 16 rows a wave reads from each half.
template <bool KC, bool GATHER, int NB> struct PipeOperand {
  const bf16_t* base;   // the tensor, or the tile's start
  uint32_t off[KC ? 4 : 2];  // bytes from base: rows half * 128 + j * 64 + tid / 8 | columns of a half
  int c8;               // KC: first k of this thread's unit within a stage
  int64_t ld;
  uint32_t frag[KC ? 2 : 1][KC ? 2 : 1];  // LDS bytes in half 0; KC: of each stage, each 32 of k

  // n: rows of the tile index that are there; index: source rows, if gathered.
  __device__ __forceinline__ void init(int tid, const bf16_t* b, int64_t i0, int n, int64_t ld_,
                                       const int32_t* index, int nsrc, int row0, int lane,
                                       uint32_t lds) {
    ld = ld_;
    const int l16 = lane & 15, G = lane >> 4;
    if constexpr (KC) {
      const int r0 = tid >> 3;
      c8 = 8 * ((tid & 7) ^ ((r0 >> 1) & 7));
      base = GATHER && index ? b : b + i0 * ld;
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        // a row that is not there reads one that is: its results are not
        // stored, or (no source row) stored as zeros
        int64_t r = min(h * 64 + r0, n - 1);
        if constexpr (GATHER)
          if (index) {
            r = index[i0 + r];
            if (r < 0 || r >= nsrc) r = 0;
          }
        off[h] = (uint32_t)((r * ld + c8) * 2);
      }
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
        frag[0][ks] = lds + (uint32_t)(((row0 + l16) * 8 + ((4 * ks + G) ^ ((l16 >> 1) & 7))) * 16);
    } else {
      const int k = tid >> 4, g = (k & 3) | ((k >> 1) & 4);
      const int c = (tid & 15) ^ (g << 1);
      base = b + i0;
      c8 = 0;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int col = h * 128 + 8 * c;
        off[h] = (uint32_t)(((GATHER && index ? 0 : k * ld) + (col < n ? col : 0)) * 2);
      }
      const int gr = (l16 >> 2) | ((G & 1) << 2);
      // block i lies at this ^ 32 i: row0 is a multiple of 16 NB, so i is in the
      // low bits of the pair of units alone
      frag[0][0] = lds + (uint32_t)((8 * G + (l16 >> 2)) * 256 + (((row0 >> 4) ^ gr) << 5) + (l16 & 3) * 8);
    }
    if constexpr (KC)
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) frag[1][ks] = frag[0][ks] + 4 * kPipeHalf * 16;
  }

  // The two copies of half `h` of the stage at k0 into dst (this wave's part).
  // CHECK: the stage may reach past K.  idx: bytes from base of the rows of k
  // this thread copies (~0: none), if they are gathered.
  template <bool CHECK>
  __device__ __forceinline__ void copy(int tid, int h, int k0, int K, u32x4_t* dst, bool gathered,
                                       const uint32_t (&idx)[2]) const {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const char* src;
      bool ok = true;
      if constexpr (KC) {
        src = reinterpret_cast<const char*>(base + k0) + off[2 * h + j];
        if constexpr (CHECK) ok = k0 + c8 < K;
      } else if (GATHER && gathered) {
        src = reinterpret_cast<const char*>(base) + idx[j] + off[h];
        ok = idx[j] != ~0u;
      } else {
        src = reinterpret_cast<const char*>(base + (int64_t)(k0 + 32 * j) * ld) + off[h];
        if constexpr (CHECK) ok = k0 + 32 * j + (tid >> 4) < K;
      }
      if (CHECK || (GATHER && !KC))
        src = ok ? src : reinterpret_cast<const char*>(zero_unit);
      copy16_lds(src, dst + 512 * j);
    }
  }

  template <int PAR> __device__ __forceinline__ void read(uint32_t half, u32x4_t (&f)[NB][2]) const {
    if constexpr (KC) {
#if defined(__HIP_DEVICE_COMPILE__)
      typedef const __attribute__((address_space(3))) char* lds_ptr;
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int i = 0; i < NB; ++i)
          f[i][ks] = *(const __attribute__((address_space(3))) u32x4_t*)(
              (lds_ptr)frag[PAR][ks] + (half + 2048 * i));
#endif
    } else {
      uint32_t q[NB], first = frag[0][0];
      asm volatile("" : "+v"(first));  // made anew each time: registers are short
#pragma unroll
      for (int i = 0; i < NB; ++i) q[i] = (first ^ (32u * i)) + (PAR * 4 * kPipeHalf * 16 + half);
      read_tr_blocks<1024, 8192>(q, f);
    }
  }
};

// The low-rank part of an adapted tile, added to acc, by runs of 64 of k as in
// the main loop (the same places in LDS, two runs at a time): adapter by
// adapter of the tile's rows, which are in the adapters' order, the rows of B
// (its parts' ranks over again) and the rows of H.  Only the adapter's own rows
// take its products, so what is not finite in B stays in them.  H in three parts
// takes 13 us a tile at rank 64 and 8 at rank 16 (8192 rows of 2048 x 4096, one
// adapter a tile; two 18 and 9).  In two parts, straight from memory, a quarter of
// the results at a time, it was 30 at rank 64.
template <typename TO>
__device__ __forceinline__ void pipe_low_rank(const GroupArgs& a, const AdaptArgs& ad,
                                              const Tile<bf16_t, TO>& w, int tid, int lane, int wave,
                                              u32x4_t* lds, uint32_t lds0, f32x4_t (&acc)[8][4]) {
  const int wm = wave >> 2, wn = wave & 3, l16 = lane & 15;
  const int r0 = tid >> 3, c8 = 8 * ((tid & 7) ^ ((r0 >> 1) & 7));
  PipeOperand<true, false, 4> X;
  PipeOperand<true, false, 2> Y;
  X.init(tid, nullptr, 0, 1, 0, nullptr, 0, wm * 64, lane, lds0);
  Y.init(tid, nullptr, 0, 1, 0, nullptr, 0, wn * 32, lane, lds0);
  const bf16_t* const H = reinterpret_cast<const bf16_t*>(ad.Hp) + (int64_t)w.n0 * ad.hl;
  for (int pos = 0; pos < w.n_valid;) {
    // the adapter of row `pos`, and the rows from there on that have it
    const int id = __builtin_amdgcn_readfirstlane(ad.ids[w.n0 + pos]);
    if (id < 0 || id >= ad.Na) break;  // rows without an adapter are last
    int end = pos;
    for (int b = pos & ~63; b < w.n_valid; b += 64) {
      const int n = b + lane;
      end += __popcll(__ballot(n >= pos && n < w.n_valid && ad.ids[w.n0 + min(n, w.n_valid - 1)] == id));
    }
    const bf16_t* const B = reinterpret_cast<const bf16_t*>(ad.B) + ((int64_t)id * a.M + w.m0) * ad.Nl;
    for (int k0 = 0; k0 < ad.hl; k0 += 128) {
      __syncthreads();  // every wave is done with what is there
#pragma unroll
      for (int par = 0; par < 2; ++par) {
        if (k0 + 64 * par >= ad.hl) break;
        const int k = k0 + 64 * par + c8;
        const bool ok = k < ad.hl;
        const int rank = k % ad.nlp;
#pragma unroll
        for (int q = 0; q < 4; ++q) {  // half q / 2, its rows from 64 (q % 2) on
          const int row = 64 * q + r0;
          u32x4_t* const dst = lds + par * 4 * kPipeHalf + 64 * wave + 512 * (q & 1);
          const bf16_t* const bx = B + min(row, w.m_valid - 1) * ad.Nl + rank;
          const bf16_t* const hy = H + min(row, w.n_valid - 1) * ad.hl + k;
          const char* const zero = reinterpret_cast<const char*>(zero_unit);
          copy16_lds(ok ? reinterpret_cast<const char*>(bx) : zero, dst + (q < 2 ? kX0 : kX1) * kPipeHalf);
          copy16_lds(ok ? reinterpret_cast<const char*>(hy) : zero, dst + (q < 2 ? kY0 : kY1) * kPipeHalf);
        }
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      auto products = [&](auto par) __attribute__((always_inline)) {
#pragma unroll
        for (int hm = 0; hm < 2; ++hm) {
          u32x4_t xf[4][2];
          X.template read<par.value>((hm ? kX1 : kX0) * kPipeHalf * 16, xf);
          const int k = k0 + 64 * par.value;
          if (k + 64 > ad.nlp) {  // some of it meets later parts
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
#pragma unroll
              for (int i = 0; i < 4; ++i)
                xf[i][ks] = met_by_part(xf[i][ks], k + 32 * ks + 8 * (lane >> 4) >= ad.nlp);
          }
#pragma unroll
          for (int hn = 0; hn < 2; ++hn) {
            const int n0 = hn * 128 + wn * 32;  // this wave's rows of the half
            if (n0 >= end || n0 + 32 <= pos) continue;
            u32x4_t yf[2][2];
            Y.template read<par.value>((hn ? kY1 : kY0) * kPipeHalf * 16, yf);
            const bool all = n0 >= pos && min(n0 + 32, w.n_valid) <= end;
            if (all) {
#pragma unroll
              for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                  for (int j = 0; j < 2; ++j)
                    acc[4 * hm + i][2 * hn + j] = mma<bf16_t>(xf[i][ks], yf[j][ks], acc[4 * hm + i][2 * hn + j]);
            } else {
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                const int n = n0 + 16 * j + l16;
                const bool own = n >= pos && n < end;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  f32x4_t sum = acc[4 * hm + i][2 * hn + j];
#pragma unroll
                  for (int ks = 0; ks < 2; ++ks) sum = mma<bf16_t>(xf[i][ks], yf[j][ks], sum);
#pragma unroll
                  for (int e = 0; e < 4; ++e)
                    acc[4 * hm + i][2 * hn + j][e] = own ? sum[e] : acc[4 * hm + i][2 * hn + j][e];
                }
              }
            }
          }
        }
      };
      products(std::integral_constant<int, 0>{});
      if (k0 + 64 < ad.hl) products(std::integral_constant<int, 1>{});
    }
    pos = end;
  }
}

template <typename TO, int MODE>
__global__ __launch_bounds__(512, 2) void group_pipe(GroupArgs a, AdaptArgs ad, int band) {
  typedef bf16_t T;
  constexpr bool XKC = MODE == kFwd || MODE == kAdapt, YKC = MODE != kBwdKer;
  constexpr bool XG = MODE == kBwdKer, YG = MODE == kFwd || MODE == kAdapt;

  extern __shared__ __attribute__((aligned(16))) char smem[];
  u32x4_t* const lds = reinterpret_cast<u32x4_t*>(smem);
  uint32_t* const idx = reinterpret_cast<uint32_t*>(smem + kPipeLds);

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int late = wave >> 2;  // one slot behind
  const int wm = wave >> 2, wn = wave & 3;
  auto xrow = [&](int i) { return (i >> 2) * 128 + wm * 64 + 16 * (i & 3); };
  auto yrow = [&](int j) { return (j >> 1) * 128 + wn * 32 + 16 * (j & 1); };

  Tile<T, TO> w;
  if (!setup_tile<T, TO, MODE, 256, 256>(a, band, &w)) return;

  f32x4_t acc[8][4];
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  const bool gather_k = XG && w.rows;
  PipeOperand<XKC, XG, 4> X;
  PipeOperand<YKC, YG, 2> Y;
  // the kernel has no other LDS: the ring starts at 0, as the blocks' addresses need
  const uint32_t lds0 = (uint32_t)(uintptr_t)LDS_AS(char, smem);

  // Runs of k: all of it, but for gathered rows of k as many as LDS holds.
  for (int kb = 0; kb < w.K; kb += kPipeRows) {
    const int K = gather_k ? min(w.K - kb, kPipeRows) : w.K;
    if (gather_k) {
      __syncthreads();  // every wave is done with the last run's rows
      for (int i = tid; i < kPipeRows + 192; i += 512) {
        const int r = i < K ? w.rows[kb + i] : -1;
        idx[i] = r >= 0 && r < a.Nsrc ? (uint32_t)(r * a.ldx * 2) : ~0u;
      }
      __syncthreads();
    }
    X.init(tid, w.X, w.m0, w.m_valid, a.ldx, gather_k ? w.rows : nullptr, 0, wm * 64, lane, lds0);
    Y.init(tid, w.Y + (gather_k ? kb * a.ldy : 0), w.n0, w.n_valid, a.ldy, YG ? w.rows : nullptr,
           a.Nsrc, wn * 32, lane, lds0);

    u32x4_t xf[4][2], y0[2][2], y1[2][2];
    uint32_t xi[2] = {0, 0};
    const uint32_t none[2] = {0, 0};
    auto fetch_rows = [&](int s) __attribute__((always_inline)) {
      if (XG && gather_k) {
        xi[0] = idx[64 * s + (tid >> 4)];
        xi[1] = idx[64 * s + 32 + (tid >> 4)];
      }
    };
    auto half_units = [&](int par, int h) { return lds + (par * 4 + h) * kPipeHalf + 64 * wave; };
    auto copy_x = [&](auto par, auto check, int s, int h) __attribute__((always_inline)) {
      X.template copy<check.value>(tid, h, 64 * s, K, half_units(par.value, h ? kX1 : kX0), gather_k, xi);
    };
    auto copy_y = [&](auto par, auto check, int s, int h) __attribute__((always_inline)) {
      Y.template copy<check.value>(tid, h, 64 * s, K, half_units(par.value, h ? kY1 : kY0), false, none);
    };
    // end of a memory slot: this wave's copies but the last ten have landed
    auto landed = [&]() __attribute__((always_inline)) {
      asm volatile("s_waitcnt vmcnt(10)\n\ts_barrier" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
    };
    // end of a products slot: this wave's reads are done
    auto done = [&]() __attribute__((always_inline)) {
      __builtin_amdgcn_sched_barrier(0);
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
    };
    auto products = [&](int hm, int hn, const u32x4_t(&yf)[2][2]) __attribute__((always_inline)) {
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j)
            acc[4 * hm + i][2 * hn + j] = mma<T>(xf[i][ks], yf[j][ks], acc[4 * hm + i][2 * hn + j]);
      __builtin_amdgcn_s_setprio(0);
    };
    // HALF: no row of Y half 1 is there, its phases only keep the step
    auto stage = [&](auto par, auto check, auto half, int s) __attribute__((always_inline)) {
      constexpr int P = par.value;
      constexpr bool HALF = half.value;
      std::integral_constant<int, 1 - P> other;
      X.template read<P>(kX0 * kPipeHalf * 16, xf);
      copy_x(other, check, s + 1, 1);
      landed();
      products(0, 0, y0);
      done();
      if constexpr (!HALF) Y.template read<P>(kY1 * kPipeHalf * 16, y1);
      copy_y(par, check, s + 2, 0);
      fetch_rows(s + 2);
      landed();
      if constexpr (!HALF) products(0, 1, y1);
      done();
      X.template read<P>(kX1 * kPipeHalf * 16, xf);
      copy_x(par, check, s + 2, 0);
      landed();
      if constexpr (!HALF) products(1, 1, y1);
      done();
      u32x4_t next[2][2];
      Y.template read<1 - P>(kY0 * kPipeHalf * 16, next);
      copy_y(par, check, s + 2, 1);
      landed();
      products(1, 0, y0);
      done();
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) y0[j][ks] = next[j][ks];
    };

    constexpr std::integral_constant<int, 0> even;
    constexpr std::integral_constant<int, 1> odd;
    constexpr std::integral_constant<bool, true> check;
    constexpr std::integral_constant<bool, false> whole;
    const int n_st = (K + 63) / 64;
    fetch_rows(0);
    copy_y(even, check, 0, 0);
    copy_x(even, check, 0, 0);
    copy_y(even, check, 0, 1);
    copy_x(even, check, 0, 1);
    fetch_rows(1);
    copy_y(odd, check, 1, 0);
    copy_x(odd, check, 1, 0);
    copy_y(odd, check, 1, 1);
    landed();
    Y.template read<0>(kY0 * kPipeHalf * 16, y0);
    done();
    if (late) done();
    // stages whose copies all lie within K, then the rest
    auto stages = [&](auto half) __attribute__((always_inline)) {
      int s = 0;
      for (; 64 * (s + 4) <= K; s += 2) {
        stage(even, whole, half, s);
        stage(odd, whole, half, s + 1);
      }
      for (; s < n_st; s += 2) {
        stage(even, check, half, s);
        if (s + 1 < n_st) stage(odd, check, half, s + 1);
      }
    };
    if (MODE != kBwdKer && w.n_valid <= 128) stages(std::integral_constant<bool, true>{});
    else stages(std::integral_constant<bool, false>{});
    if (!late) done();
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the trailing (empty) copies
    if (!gather_k) break;
  }

  if constexpr (MODE == kAdapt) pipe_low_rank<TO>(a, ad, w, tid, lane, wave, lds, lds0, acc);
  store_tile<T, TO, MODE, MODE == kFwd>(a, w, lane, acc, xrow, yrow);
}

// Whether the byte offsets of a tile's rows, or of any row that may be
// gathered, fit the kernel's 32 bits.
inline bool pipe_fits(const GroupArgs& a, int mode) {
  const int64_t ld = mode == kBwdKer ? a.ldx : a.ldy;
  return a.ldx < (1 << 22) && a.ldy < (1 << 22) && (!a.rows || a.Nsrc * ld * 2 < (1LL << 32) - 65536);
}

template <typename TO, int MODE>
hipError_t launch_pipe(const GroupArgs& a, const AdaptArgs& ad, int64_t row_tiles, int band,
                       Launch to) {
  auto* const k = group_pipe<TO, MODE>;
  const int64_t grid = row_tiles * ((a.M + 255) / 256);
  const hipError_t fit = grid_fits(grid, 512);
  if (fit != hipSuccess || to.dry) return fit;
  const hipError_t e = allow_max_lds(reinterpret_cast<const void*>(k));
  if (e != hipSuccess) return e;
  const int lds = kPipeLds + (MODE == kBwdKer && a.rows ? (kPipeRows + 192) * 4 : 0);
  k<<<dim3((uint32_t)grid), dim3(512), lds, to.stream>>>(a, ad, band);
  return hipGetLastError();
}

}  // namespace group
}  // namespace cnnlib
