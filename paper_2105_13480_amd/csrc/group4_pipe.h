// The pipelined 256 x 256 tile kernels of products with a Ker in 4 bits, in the
// phases of group_pipe (which see): eight waves, a stage in four phases of one quarter,
// waves 4 to 7 a slot behind.  Operands come by buffer instructions: one offset register
// a row (or one in all, where rows follow one another), scalar offsets for the rest, and
// zeros past the end (both offsets' sum is what is compared with it), since accumulators
// and operands leave no registers to spare, and a spill in the loop is a wait for
// everything in flight.
//
// Bound by the matrix unit and by a tile's start and results, 8 to 10 us in which the CU
// that it fills alone multiplies nothing (16384 x 2 rows of 16 groups of 4096 x 2048):
//   bf16 rows    465 us, 1180 TFLOP/s; one group of 8192 x 8192 1445, the library's bf16
//                product of that size 1330 to 1480
//   gradient     425 us, 1295 TFLOP/s; 1400
//   both 4 bits  209 us, 2630 TFLOP/s; 4330: a stage of 1.7 us (0.9 at the matrix unit's
//                rate).  Neither that nor LDS bounds the loop: both are busy for a
//                quarter of the kernel, some 42 % of the loop, one after the other as it
//                seems; why they do not overlap is not known.
// A last round of at most 128 tiles is halved by features (15550 rows of 8 groups of
// 2048 x 2048, 520 tiles: 141 us, now 131; one group of 1100 rows of 4096 x 4096 with both
// in 4 bits 32.1 and 24.5), and a tile without its second half of features does without
// its products (8000 rows of 2056 x 2048: 96 us, now 87).
// Workgroups that stay for several tiles (results are in the same order of waits as the
// next tile's copies) and stores past the caches gained nothing.
#pragma once

#include "group4_kernel.h"
#include "group_pipe.h"

namespace cnnlib {
namespace group {

__device__ __forceinline__ void write_lds(uint32_t at, u32x4_t v) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("ds_write_b128 %0, %1" ::"v"(at), "v"(v) : "memory");
#else
  (void)at;
  (void)v;
#endif
}

// LDS: Y's halves 0 and 1 of two stages, then X's.
constexpr int kHalfBytes = kPipeHalf * 16;
constexpr int kPipe4X = 4 * kHalfBytes;

// Where a lane's units of a half with k last lie: NB blocks of 16 rows from row0 on,
// 32 of k by 32.  PAIR: two units that follow one another (blocks of 4-bit values).
template <int NB, bool PAIR> struct PipeReads {
  uint32_t frag[2];  // LDS bytes of each sub-step's in half 0
  __device__ __forceinline__ void init(int row0, int lane, uint32_t lds) {
    const int l16 = lane & 15, G = lane >> 4;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
      frag[ks] = lds + (uint32_t)(((row0 + l16) * 8 + ((PAIR ? 2 * G + ks : 4 * ks + G) ^ ((l16 >> 1) & 7))) * 16);
  }
  // half: its bytes from the first, below 64 KB, where the instruction holds them.
  __device__ __forceinline__ void read(uint32_t half, u32x4_t (&f)[NB][2]) const {
#if defined(__HIP_DEVICE_COMPILE__)
    typedef const __attribute__((address_space(3))) char* lds_ptr;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int i = 0; i < NB; ++i)
        f[i][ks] = *(const __attribute__((address_space(3))) u32x4_t*)((lds_ptr)frag[ks] + (half + 2048 * i));
#endif
  }
};

// Copies of an operand's rows of 16-bit words, k last, to LDS; the rows may be gathered.
template <bool GATHER> struct PipeRows {
  __amdgpu_buffer_rsrc_t rsrc;
  uint32_t off[GATHER ? 4 : 1];  // bytes of this thread's rows 64 by 64, at its first k
  uint32_t step;                 // of 64 rows (rows that follow one another)
  int c8;                        // first k of this thread's unit within a stage

  // Rows [i0, i0 + n) of base, or index[i0 ..] of its nsrc rows.
  __device__ __forceinline__ void init(int tid, const bf16_t* base, int64_t i0, int n, int64_t ld,
                                       const int32_t* index, int nsrc) {
    const int r0 = tid >> 3;
    c8 = 8 * ((tid & 7) ^ ((r0 >> 1) & 7));
    step = (uint32_t)(64 * ld * 2);
    if (GATHER && index) rsrc = rsrc_of(base, nsrc * ld * 2);
    else rsrc = rsrc_of(base + i0 * ld, n * ld * 2);
#pragma unroll
    for (int h = 0; h < (GATHER ? 4 : 1); ++h) {
      int64_t r = 64 * h + r0;
      if (GATHER && index) {
        // a row that is not there reads one that is: its results are not stored, or
        // (no source row) stored as zeros
        r = index[i0 + min((int)r, n - 1)];
        if (r < 0 || r >= nsrc) r = 0;
      }
      off[h] = (uint32_t)((r * ld + c8) * 2);  // past the last row: zeros
    }
  }
  // Half h of the stage at k0 into dst (this wave's part).  CHECK: the stage may reach
  // past K.
  template <bool CHECK> __device__ __forceinline__ void copy(int h, int k0, int K, u32x4_t* dst) const {
    const bool ok = !CHECK || k0 + c8 < K;
#pragma unroll
    for (int j = 0; j < 2; ++j)
      buffer_lds(rsrc, dst + 512 * j, ok ? off[GATHER ? 2 * h + j : 0] : kNowhere,
                 (uint32_t)(2 * k0) + (GATHER ? 0u : (2 * h + j) * step));
  }
};

// A thread's part of a stage of Ker with c last on its way to LDS as bf16: of each half
// (64 rows of k by 128 of c), 16 values of a row.
struct PipeKer4 {
  __amdgpu_buffer_rsrc_t codes, scales;
  uint32_t dst;  // LDS bytes of its first unit within a half
  int Nb;
  u32x2_t code[2];
  uint32_t scale[2];

  // The group's codes and scales, K rows of them; the tile's first c.  A thread has 16
  // values of row k = tid / 8 from 16 (tid % 8) on; c past the row's blocks read the
  // next row: for results that are not stored.
  __device__ __forceinline__ void init(int tid, const uint8_t* c4, const uint8_t* s4, int Nb_, int m0, int K) {
    const int k = tid >> 3, g = (k & 3) | ((k >> 1) & 4);
    Nb = Nb_;
    codes = rsrc_of(c4 + m0 / 2, (int64_t)K * 16 * Nb - m0 / 2);
    scales = rsrc_words(s4 + m0 / 32, (int64_t)K * Nb - m0 / 32);
    dst = (uint32_t)(16 * (k * 16 + ((2 * (tid & 7)) ^ (g << 1))));
  }
  // Asks for half h of the stage at k0; past K zeros.
  __device__ __forceinline__ void load(int h, int k0) {
#if defined(__HIP_DEVICE_COMPILE__)
    uint32_t t = threadIdx.x;
    asm volatile("" : "+v"(t));  // offsets are made anew each time: registers are short
    const uint32_t row = (t >> 3) * (uint32_t)Nb;
    code[h] = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_raw_buffer_load_b64(codes, (int)(row * 16 + 8 * (t & 7)), (int)((uint32_t)k0 * 16u * (uint32_t)Nb + 64u * h), 0));
    scale[h] = __builtin_amdgcn_raw_buffer_load_b8(scales, (int)(row + ((t & 7) >> 1)), k0 * Nb + 4 * h, 0);
#endif
  }
  // Half h as it was asked for, as bf16 to LDS.
  __device__ __forceinline__ void write(int h, uint32_t half) const {
    const float s = scale4(scale[h]);
    write_lds(half + dst, bf16_of4(code[h][0], s));
    write_lds(half + (dst ^ 16u), bf16_of4(code[h][1], s));
  }
};

// What the kernels do at the end of a memory slot (this wave's copies and loads but
// the last N have landed) and of a products slot (its reads and writes are done).
template <int N> __device__ __forceinline__ void pipe_landed() {
  asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(N) : "memory");
  __builtin_amdgcn_sched_barrier(0);
}
__device__ __forceinline__ void pipe_done() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// The stages of n_st, two at a time: those whose copies all lie within K, the rest.
template <typename F> __device__ __forceinline__ void pipe_stages(int K, F stage) {
  constexpr std::integral_constant<int, 0> even;
  constexpr std::integral_constant<int, 1> odd;
  constexpr std::integral_constant<bool, true> check;
  constexpr std::integral_constant<bool, false> whole;
  const int n_st = (K + 63) / 64;
  int s = 0;
  for (; 64 * (s + 4) <= K; s += 2) {
    stage(even, whole, s);
    stage(odd, whole, s + 1);
  }
  for (; s < n_st; s += 2) {
    stage(even, check, s);
    if (s + 1 < n_st) stage(odd, check, s + 1);
  }
}

// run(X, Y): of that operand half 1 is not there, and its phases only keep the step (such
// a tile takes 0.73 to 0.77 of a whole one's time).
template <typename F> __device__ __forceinline__ void pipe_halves(int m_valid, int n_valid, F run) {
  constexpr std::integral_constant<bool, true> half;
  constexpr std::integral_constant<bool, false> whole;
  if (m_valid <= 128) {
    if (n_valid <= 128) run(half, half);
    else run(half, whole);
  } else {
    if (n_valid <= 128) run(whole, half);
    else run(whole, whole);
  }
}
// The launch's arguments with the tile's end for features.
__device__ __forceinline__ GroupArgs up_to(const GroupArgs& a, int end) {
  GroupArgs e = a;
  e.M = end;
  return e;
}

// bf16 rows, forward.  Ker stays in 4 bits in LDS and each wave turns what it reads into
// bf16 in its registers, in the slot in which the other waves multiply, so that X takes a
// quarter of the copies and reads: with bf16 in LDS these and the writes were as long as
// the products.  A wave has 64 (m) by 128 (n) results, so that it turns 64 rows of X, not
// 128.  A lane takes 16 values that follow one another, half a block; the other operand's
// lane the same.  A stage:
//   phase  reads from LDS            copies                          products
//     0    Y half 0, X1's codes      Y half 1 of s + 1               X0 Y0
//     1                              (even) X, scales of s + 2       X1 Y0
//     2    Y half 1                  Y half 0 of s + 2               X1 Y1
//     3    X0's codes of s + 1       -                               X0 Y1
// and X of s + 2 in an odd stage's phase 1; X0 and X1 become bf16 in phases 0 and 1, and X0
// is kept.  What is asked for in a phase is there in the sixth phase after it, so each wait
// leaves as many in flight as the five phases up to it have, by phases of two stages.
constexpr int kPipe4Codes = 4 * kHalfBytes;           // after Y: [stage % 4][256][32]
constexpr int kPipe4Scales = kPipe4Codes + 4 * 8192;  // [pair % 2][512][4], the second 256 not read
constexpr int kPipe4Lds = kPipe4Scales + 2 * 2048;
constexpr int kPipe4Waits[8] = {7, 7, 8, 6, 8, 7, 7, 5};

template <typename TO>
__global__ __launch_bounds__(512, 2) void group4_pipe(GroupArgs a, Group4Args b, int band) {
  typedef bf16_t T;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  u32x4_t* const lds = reinterpret_cast<u32x4_t*>(smem);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, G = lane >> 4;
  const int late = wave >> 2;  // one slot behind
  const int wm = wave & 3, wn = wave >> 2;
  auto xrow = [&](int i) { return (i >> 1) * 128 + wm * 32 + 16 * (i & 1); };
  auto yrow = [&](int j) { return (j >> 2) * 128 + wn * 64 + 16 * (j & 3); };

  Tile<T, TO> w;
  if (!setup_tile<T, TO, kFwd, 256, 256, true>(a, band, &w)) return;
  const int64_t g = w.g < a.Ng ? w.g : 0;

  f32x4_t acc[4][8];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  if (w.K > 0) {
    const uint32_t lds0 = (uint32_t)(uintptr_t)LDS_AS(char, smem);
    const int K = w.K, Kx = 32 * b.Nb;
    PipeRows<true> ys;
    PipeReads<4, true> Y;
    Y.init(wn * 64, lane, lds0);
    ys.init(tid, w.Y, w.n0, w.n_valid, a.ldy, w.rows, a.Nsrc);
    // this thread's part of X: 16 bytes of row tid / 2; and a row's four scales
    const int64_t x0 = g * a.M + w.m0;
    const __amdgpu_buffer_rsrc_t xr = rsrc_of(reinterpret_cast<const uint8_t*>(a.X) + x0 * 16 * b.Nb, (int64_t)w.m_valid * 16 * b.Nb);
    const __amdgpu_buffer_rsrc_t sr = rsrc_words(b.xs + x0 * b.Nb, (int64_t)w.m_valid * b.Nb);
    const uint32_t xoff = (uint32_t)((tid >> 1) * 16 * b.Nb + 16 * (tid & 1));
    // X of stage s, past the row's end zeros
    auto copy_x = [&](auto check, int s) __attribute__((always_inline)) {
      const bool ok = !check.value || 64 * s + 32 * (tid & 1) < Kx;
      buffer_lds(xr, lds + (kPipe4Codes + (s & 3) * 8192) / 16 + 64 * wave, ok ? xoff : kNowhere, 32u * s);
    };
    // the scales of stages 2 pair and the next, whole where some of it is the row's
    auto copy_scales = [&](int pair) __attribute__((always_inline)) {
#if defined(__HIP_DEVICE_COMPILE__)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(sr, LDS_AS(void, smem + kPipe4Scales + (pair & 1) * 2048 + 256 * wave), 4,
                                               (tid & 255) * b.Nb, 4 * pair, 0, 0);
#endif
    };
    auto copy_y = [&](auto par, auto check, int s, int h) __attribute__((always_inline)) {
      ys.template copy<check.value>(h, 64 * s, K, lds + (par.value * 2 + h) * kPipeHalf + 64 * wave);
    };
    const char* const xget = smem + kPipe4Codes + 32 * (wm * 32 + l16) + 8 * G;
    const char* const sget = smem + kPipe4Scales + 4 * (wm * 32 + l16) + (G >> 1);
    u32x2_t code[2];
    uint32_t scale[2];
    auto read_x = [&](int s, int h) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        code[i] = *reinterpret_cast<const u32x2_t*>(xget + (s & 3) * 8192 + 4096 * h + 512 * i);
        scale[i] = *reinterpret_cast<const uint8_t*>(sget + (s & 2) * 1024 + 2 * (s & 1) + 512 * h + 64 * i);
      }
    };
    u32x4_t x[2][2][2], yf[4][2];
    auto turn_x = [&](int h) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) x[h][i][ks] = bf16_of4(code[i][ks], scale4(scale[i]));
    };
    auto products = [&](int hm, int hn) __attribute__((always_inline)) {
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            acc[2 * hm + i][4 * hn + j] = mma<T>(x[hm][i][ks], yf[j][ks], acc[2 * hm + i][4 * hn + j]);
      __builtin_amdgcn_s_setprio(0);
    };
    constexpr std::integral_constant<int, 0> even;
    constexpr std::integral_constant<int, 1> odd;
    constexpr std::integral_constant<bool, true> check;
    copy_x(check, 0);
    copy_scales(0);
    copy_x(check, 1);
    copy_y(even, check, 0, 0);
    copy_y(even, check, 0, 1);
    copy_y(odd, check, 1, 0);
    pipe_landed<2>();
    read_x(0, 0);
    pipe_done();
    if (late) pipe_done();
    auto run = [&](auto one_x, auto one_y) __attribute__((always_inline)) {
      constexpr bool XHALF = one_x.value, HALF = one_y.value;
      pipe_stages(K, [&](auto par, auto chk, int s) __attribute__((always_inline)) {
        constexpr int P = par.value;
        std::integral_constant<int, 1 - P> other;
        Y.read(2 * P * kHalfBytes, yf);
        turn_x(0);
        if constexpr (!XHALF) read_x(s, 1);
        copy_y(other, chk, s + 1, 1);
        pipe_landed<kPipe4Waits[4 * P]>();
        products(0, 0);
        pipe_done();
        if constexpr (!XHALF) turn_x(1);
        copy_x(chk, s + 2);
        if constexpr (P == 0) copy_scales((s >> 1) + 1);
        pipe_landed<kPipe4Waits[4 * P + 1]>();
        if constexpr (!XHALF) products(1, 0);
        pipe_done();
        if constexpr (!HALF) Y.read((2 * P + 1) * kHalfBytes, yf);
        copy_y(par, chk, s + 2, 0);
        pipe_landed<kPipe4Waits[4 * P + 2]>();
        if constexpr (!HALF && !XHALF) products(1, 1);
        pipe_done();
        read_x(s + 1, 0);
        pipe_landed<kPipe4Waits[4 * P + 3]>();
        if constexpr (!HALF) products(0, 1);
        pipe_done();
      });
    };
    pipe_halves(w.m_valid, w.n_valid, run);
    if (!late) pipe_done();
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");  // the trailing copies
  }
  store_tile<T, TO, kFwd, true>(up_to(a, w.m0 + w.m_valid), w, lane, acc, xrow, yrow);
}

// The gradient of In.  Ker's part of a stage is 16 values a thread and half: codes and
// scale are asked for a stage before they become bf16 in LDS (8 instructions), beside the
// other waves' matrix instructions, and are read back transposed.  Waves of 64 (c) by 128
// results: half as many transposing reads as with 128 by 64.  A stage:
//   phase  reads from LDS   copies and loads                       products
//     0    Y half 0, X0     Y half 1 of s + 1                      X0 Y0
//     1    X1               X1 of s + 1 to LDS, the next asked for X1 Y0
//     2    Y half 1         Y half 0 of s + 2                      X1 Y1
//     3    -                X0 of s + 2 to LDS, the next asked for X0 Y1
// Two copies or loads a phase, and what is asked for there in the sixth phase after it (the
// loads, which the compiler waits for, in the fourth): a wait leaves ten in flight.
template <typename TO>
__global__ __launch_bounds__(512, 2) void group4_pipe_bwd_in(GroupArgs a, Group4Args b, int band) {
  typedef bf16_t T;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  u32x4_t* const lds = reinterpret_cast<u32x4_t*>(smem);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int late = wave >> 2;  // one slot behind
  const int wm = wave & 3, wn = wave >> 2;
  auto xrow = [&](int i) { return (i >> 1) * 128 + wm * 32 + 16 * (i & 1); };
  auto yrow = [&](int j) { return (j >> 2) * 128 + wn * 64 + 16 * (j & 3); };

  Tile<T, TO> w;
  if (!setup_tile<T, TO, kBwdIn, 256, 256, true>(a, band, &w)) return;
  const int64_t g = w.g < a.Ng ? w.g : 0;

  f32x4_t acc[4][8];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  if (w.K > 0) {
    const uint32_t lds0 = (uint32_t)(uintptr_t)LDS_AS(char, smem);
    const int K = w.K;
    PipeKer4 ker;
    PipeOperand<false, false, 2> X;  // its reads
    PipeRows<false> ys;
    PipeReads<4, false> Y;
    ker.init(tid, reinterpret_cast<const uint8_t*>(a.X) + g * K * 16 * b.Nb, b.xs + g * K * b.Nb, b.Nb, w.m0, K);
    X.init(tid, nullptr, 0, 1, 0, nullptr, 0, wm * 32, lane, lds0);
    Y.init(wn * 64, lane, lds0);
    ys.init(tid, w.Y, w.n0, w.n_valid, a.ldy, nullptr, 0);

    u32x4_t x0[2][2], x1[2][2], yf[4][2];
    auto half_of = [&](int par, int h) { return (uint32_t)(kPipe4X + (par * 2 + h) * kHalfBytes); };
    // half h of X of stage s to LDS, and the next one of it asked for
    auto put_x = [&](auto par, int s, int h) __attribute__((always_inline)) {
      ker.write(h, lds0 + half_of(par.value, h));
      ker.load(h, 64 * (s + 1));
    };
    auto copy_y = [&](auto par, auto check, int s, int h) __attribute__((always_inline)) {
      ys.template copy<check.value>(h, 64 * s, K, lds + (par.value * 2 + h) * kPipeHalf + 64 * wave);
    };
    auto products = [&](int hm, int hn, const u32x4_t(&xf)[2][2]) __attribute__((always_inline)) {
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            acc[2 * hm + i][4 * hn + j] = mma<T>(xf[i][ks], yf[j][ks], acc[2 * hm + i][4 * hn + j]);
      __builtin_amdgcn_s_setprio(0);
    };
    constexpr std::integral_constant<int, 0> even;
    constexpr std::integral_constant<int, 1> odd;
    constexpr std::integral_constant<bool, true> check;
    ker.load(0, 0);
    ker.load(1, 0);
    copy_y(even, check, 0, 0);
    copy_y(even, check, 0, 1);
    put_x(even, 0, 0);
    put_x(even, 0, 1);
    copy_y(odd, check, 1, 0);
    put_x(odd, 1, 0);
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    if (late) pipe_done();
    auto run = [&](auto one_x, auto one_y) __attribute__((always_inline)) {
      constexpr bool XHALF = one_x.value, HALF = one_y.value;
      pipe_stages(K, [&](auto par, auto chk, int s) __attribute__((always_inline)) {
        constexpr int P = par.value;
        std::integral_constant<int, 1 - P> other;
        Y.read(2 * P * kHalfBytes, yf);
        X.template read<0>(half_of(P, 0), x0);
        copy_y(other, chk, s + 1, 1);
        pipe_landed<10>();
        products(0, 0, x0);
        pipe_done();
        if constexpr (!XHALF) X.template read<0>(half_of(P, 1), x1);
        put_x(other, s + 1, 1);
        pipe_landed<10>();
        if constexpr (!XHALF) products(1, 0, x1);
        pipe_done();
        if constexpr (!HALF) Y.read((2 * P + 1) * kHalfBytes, yf);
        copy_y(par, chk, s + 2, 0);
        pipe_landed<10>();
        if constexpr (!HALF && !XHALF) products(1, 1, x1);
        pipe_done();
        put_x(par, s + 2, 0);
        pipe_landed<10>();
        if constexpr (!HALF) products(0, 1, x0);
        pipe_done();
      });
    };
    pipe_halves(w.m_valid, w.n_valid, run);
    if (!late) pipe_done();
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");  // the trailing copies
  }
  store_tile<T, TO, kBwdIn, false>(up_to(a, w.m0 + w.m_valid), w, lane, acc, xrow, yrow);
}

// Both operands in 4 bits: the same bytes a stage, 256 values of k, and so the same
// copies, reads and time a stage as in bf16, for four times the products.  Scales: of
// two stages at a time, a lane copies the 16 bytes of one row to LDS (waves 0 to 3 of
// X, the others of Y), eight phases before they are read.
constexpr int kPipe44Lds = kPipeLds + 2 * 512 * 16;

template <typename TO>
__global__ __launch_bounds__(512, 2) void group44_pipe(GroupArgs a, Group4Args b, int band) {
  typedef bf16_t T;  // codes as 16-bit words
  extern __shared__ __attribute__((aligned(16))) char smem[];
  u32x4_t* const lds = reinterpret_cast<u32x4_t*>(smem);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, G = lane >> 4;
  const int late = wave >> 2;  // one slot behind
  const int wm = wave >> 2, wn = wave & 3;
  auto xrow = [&](int i) { return (i >> 2) * 128 + wm * 64 + 16 * (i & 3); };
  auto yrow = [&](int j) { return (j >> 1) * 128 + wn * 32 + 16 * (j & 1); };

  Tile<T, TO> w;
  if (!setup_tile<T, TO, kFwd, 256, 256, true>(a, band, &w)) return;
  const int64_t g = w.g < a.Ng ? w.g : 0;

  f32x4_t acc[8][4];
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  if (w.K > 0) {
    const uint32_t lds0 = (uint32_t)(uintptr_t)LDS_AS(char, smem);
    const int K = w.K;
    PipeRows<false> xs;
    PipeRows<true> ys;
    PipeReads<4, true> X;
    PipeReads<2, true> Y;
    X.init(wm * 64, lane, lds0 + kPipe4X);
    Y.init(wn * 32, lane, lds0);
    xs.init(tid, w.X, w.m0, w.m_valid, a.ldx, nullptr, 0);
    ys.init(tid, w.Y, w.n0, w.n_valid, a.ldy, w.rows, a.Nsrc);
    // this lane's row of scales
    __amdgpu_buffer_rsrc_t srsrc;
    uint32_t soff = (uint32_t)((tid & 255) * b.Nb);
    if (wave < 4) {
      srsrc = rsrc_words(b.xs + (g * a.M + w.m0) * b.Nb, (int64_t)w.m_valid * b.Nb);
    } else if (w.rows) {
      int r = w.rows[w.n0 + min(tid & 255, w.n_valid - 1)];
      if (r < 0 || r >= a.Nsrc) r = 0;
      soff = (uint32_t)(r * b.Nb);
      srsrc = rsrc_words(b.ys, (int64_t)a.Nsrc * b.Nb);
    } else {
      srsrc = rsrc_words(b.ys + (int64_t)w.n0 * b.Nb, (int64_t)w.n_valid * b.Nb);
    }
    auto copy_scales = [&](int pair) __attribute__((always_inline)) {  // of stages 2 pair, 2 pair + 1
      buffer_lds(srsrc, lds + kPipeLds / 16 + (pair & 1) * 512 + 64 * wave, soff, (uint32_t)(16 * pair));
    };
    uint32_t sx[4], sy[4];
    const char* const sget = smem + kPipeLds + 2 * G + 16 * l16;
    // the scales of blocks 8 s + 2 G and the next of a block of rows; past the row's end
    // none (what the copy found there is another row's)
    auto scales = [&](auto check, int s, int row) __attribute__((always_inline)) -> uint32_t {
      const uint32_t v = *reinterpret_cast<const uint16_t*>(sget + (s & 2) * 4096 + (s & 1) * 8 + 16 * row);
      return !check.value || 8 * s + 2 * G < b.Nb ? v : 0u;
    };

    u32x4_t xf[4][2], y0[2][2], y1[2][2];
    auto half_units = [&](int par, int h) { return lds + (par * 2 + h) * kPipeHalf + 64 * wave; };
    auto copy_x = [&](auto par, auto check, int s, int h) __attribute__((always_inline)) {
      xs.template copy<check.value>(h, 64 * s, K, half_units(par.value, 4 + h));
    };
    auto copy_y = [&](auto par, auto check, int s, int h) __attribute__((always_inline)) {
      ys.template copy<check.value>(h, 64 * s, K, half_units(par.value, h));
    };
    auto products = [&](int hm, int hn, const u32x4_t(&yf)[2][2]) __attribute__((always_inline)) {
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          acc[4 * hm + i][2 * hn + j] =
              mma4<0>(xf[i][0], yf[j][0], acc[4 * hm + i][2 * hn + j], sx[i], sy[2 * hn + j]);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          acc[4 * hm + i][2 * hn + j] =
              mma4<1>(xf[i][1], yf[j][1], acc[4 * hm + i][2 * hn + j], sx[i], sy[2 * hn + j]);
      __builtin_amdgcn_s_setprio(0);
    };
    constexpr std::integral_constant<int, 0> even;
    constexpr std::integral_constant<int, 1> odd;
    constexpr std::integral_constant<bool, true> check;
    // X first: Y's copies wait for the rows' numbers
    copy_x(even, check, 0, 0);
    copy_x(even, check, 0, 1);
    copy_y(even, check, 0, 0);
    copy_scales(0);
    copy_y(even, check, 0, 1);
    copy_x(odd, check, 1, 0);
    copy_y(odd, check, 1, 0);
    copy_y(odd, check, 1, 1);
    pipe_landed<6>();
    Y.read(0, y0);
    pipe_done();
    if (late) pipe_done();
    auto run = [&](auto one_x, auto one_y) __attribute__((always_inline)) {
      constexpr bool XHALF = one_x.value, HALF = one_y.value;
      pipe_stages(K, [&](auto par, auto chk, int s) __attribute__((always_inline)) {
        constexpr int P = par.value;
        std::integral_constant<int, 1 - P> other;
        // scales first: reads come back in order, and the first product needs them
#pragma unroll
        for (int i = 0; i < 4; ++i) sx[i] = scales(chk, s, xrow(i));
#pragma unroll
        for (int j = 0; j < 2; ++j) sy[j] = scales(chk, s, 256 + yrow(j));
        __builtin_amdgcn_sched_barrier(0);
        X.read(2 * P * kHalfBytes, xf);
        if constexpr (P == 0) copy_scales((s >> 1) + 1);
        copy_x(other, chk, s + 1, 1);
        pipe_landed<10>();
        products(0, 0, y0);
        pipe_done();
        if constexpr (!HALF) {
#pragma unroll
          for (int j = 2; j < 4; ++j) sy[j] = scales(chk, s, 256 + yrow(j));
          __builtin_amdgcn_sched_barrier(0);
          Y.read((2 * P + 1) * kHalfBytes, y1);
        }
        copy_y(par, chk, s + 2, 0);
        pipe_landed<10>();
        if constexpr (!HALF) products(0, 1, y1);
        pipe_done();
        if constexpr (!XHALF) {
#pragma unroll
          for (int i = 0; i < 4; ++i) sx[i] = scales(chk, s, xrow(4 + i));
          __builtin_amdgcn_sched_barrier(0);
          X.read((2 * P + 1) * kHalfBytes, xf);
        }
        copy_x(par, chk, s + 2, 0);
        pipe_landed<10>();
        if constexpr (!HALF && !XHALF) products(1, 1, y1);
        pipe_done();
        u32x4_t next[2][2];
        Y.read(2 * (1 - P) * kHalfBytes, next);
        copy_y(par, chk, s + 2, 1);
        pipe_landed<10>();
        if constexpr (!XHALF) products(1, 0, y0);
        pipe_done();
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int ks = 0; ks < 2; ++ks) y0[j][ks] = next[j][ks];
      });
    };
    pipe_halves(w.m_valid, w.n_valid, run);
    if (!late) pipe_done();
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");  // the trailing (empty) copies
  }
  store_tile<T, TO, kFwd, true>(up_to(a, w.m0 + w.m_valid), w, lane, acc, xrow, yrow);
}

template <typename TO, int MODE>
hipError_t launch_pipe4(const GroupArgs& a, const Group4Args& b, int64_t row_tiles, int band, hipStream_t stream) {
  auto* const k = MODE == kFwd ? group4_pipe<TO> : group4_pipe_bwd_in<TO>;
  const int64_t grid = row_tiles * ((a.M + 255) / 256) + kRound / 2;
  hipError_t e = grid_fits(grid, 512);
  if (e == hipSuccess) e = allow_max_lds(reinterpret_cast<const void*>(k));
  if (e != hipSuccess) return e;
  k<<<dim3((uint32_t)grid), dim3(512), MODE == kFwd ? kPipe4Lds : kPipeLds, stream>>>(a, b, band);
  return hipGetLastError();
}

template <typename TO>
hipError_t launch_pipe44(const GroupArgs& a, const Group4Args& b, int64_t row_tiles, int band, hipStream_t stream) {
  auto* const k = group44_pipe<TO>;
  const int64_t grid = row_tiles * ((a.M + 255) / 256) + kRound / 2;
  hipError_t e = grid_fits(grid, 512);
  if (e == hipSuccess) e = allow_max_lds(reinterpret_cast<const void*>(k));
  if (e != hipSuccess) return e;
  k<<<dim3((uint32_t)grid), dim3(512), kPipe44Lds, stream>>>(a, b, band);
  return hipGetLastError();
}

}  // namespace group
}  // namespace cnnlib
