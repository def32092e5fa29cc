// Tile kernels of the grouped products whose Ker lies in 4 bits (gfx950): blocks
// of 32 values of c with a scale byte each, see k_block4.hip.
//
// With bf16 rows (group4_tiles) Ker's values become bf16 on their way into LDS,
// which is exact (a code has two significant bits, and its scale is a power of
// two), and are then what the bf16 kernel multiplies; both directions, since the
// conversion is the same whether c is summed over or is the result's index:
//   forward       X = Ker[g], rows of features, k = c
//   gradient, In  X = Ker[g], rows of k = features, the tile's index c
#pragma once

#include "group_kernel.h"

namespace cnnlib {
namespace group {

// 2^(s - 127) as the conversions take it: they read the exponent field alone, 0 is
// 2^-127 and 255 NaN.
__device__ __forceinline__ float scale4(uint32_t s) { return __uint_as_float(s << 23); }

// Eight values from a word of codes, as bf16.
__device__ __forceinline__ u32x4_t bf16_of4(uint32_t code, float scale) {
#if defined(__HIP_DEVICE_COMPILE__)
  return u32x4_t{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 0)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 1)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 2)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 3))};
#else
  (void)code;
  (void)scale;
  return u32x4_t{0u, 0u, 0u, 0u};
#endif
}

// An offset past the end of any buffer here (2^31 bytes at most), also with a scalar
// offset on top: it reads zeros.
constexpr uint32_t kNowhere = 0x80000000u;

// Bytes [0, n) from p on, both on 4-byte boundaries (rsrc_words: at any).
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc_of(const void* p, int64_t n) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, (int)n, 0x00020000);
}
__device__ __forceinline__ void buffer_lds(__amdgpu_buffer_rsrc_t r, u32x4_t* lds, uint32_t voff, uint32_t soff) {
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, LDS_AS(void, lds), 16, (int)voff, (int)soff, 0, 0);
#else
  (void)r;
  (void)lds;
  (void)voff;
  (void)soff;
#endif
}

// Half blocks of 16 values, of which a stage of 64 of k takes q = 0..3 of a row of Nb
// blocks: in the stage at k0, half block q reads the 16 values from half_base(q, Nb) +
// half_step(16 q, k0, 32 Nb) on.  What is not the row's reads its first half block or that
// of the first stage (a row of one block has two, and the bytes past it may be past the tensor).
__host__ __device__ constexpr int half_base(int q, int Nb) { return q < 2 * Nb ? 16 * q : 0; }
__host__ __device__ constexpr int half_step(int at, int k0, int nk) { return k0 + at < nk ? k0 : 0; }

// Stages R rows of features by 64 of k (KC) or 64 rows of k by R of c of a Ker in
// 4 bits as bf16: a thread takes half blocks (8 bytes, 16 values).
template <bool KC, int R, int NT, int SETS> struct Stager4 {
  static constexpr int ALL = 4 * R, NU = (ALL + NT - 1) / NT;
  static constexpr int U = KC ? 4 : R / 16;  // half blocks of a row of the stage
  const uint8_t* codes[NU];
  const uint8_t* scales[NU];
  int at[NU];        // KC: the half block's first k within a stage; else its row of k
  bool there[NU];    // !KC: the half block is one of the row's
  u32x2_t code[SETS][NU];
  uint32_t scale[SETS][NU];
  uint32_t gone[SETS];  // bit j: half block j of the set is not there

  // codes, scales: the group's; rows of Nb blocks; rows (KC) or c (else) [i0, i0 + n) are there.
  __device__ __forceinline__ void init(int tid, const uint8_t* c4, const uint8_t* s4, int Nb, int i0, int n) {
#pragma unroll
    for (int j = 0; j < NU; ++j) {
      const int u = min(j * NT + tid, ALL - 1), r = u / U, q = u % U;
      if constexpr (KC) {
        const int64_t row = i0 + min(r, n - 1);
        at[j] = 16 * q;
        codes[j] = c4 + row * 16 * Nb + half_base(q, Nb) / 2;
        scales[j] = s4 + row * Nb + half_base(q, Nb) / 32;
        there[j] = true;
      } else {
        at[j] = r;
        there[j] = i0 + 16 * q < 32 * Nb;
        codes[j] = c4 + (there[j] ? i0 / 2 + 8 * q : 0);
        scales[j] = s4 + (there[j] ? (i0 + 16 * q) / 32 : 0);
      }
    }
  }
  // nk: values of k (KC: of whole blocks).  What is not there is cleared when the
  // loads are waited for.
  template <int SET> __device__ __forceinline__ void load(int k0, int Nb, int nk) {
    gone[SET] = 0u;
#pragma unroll
    for (int j = 0; j < NU; ++j) {
      const bool in = k0 + at[j] < nk;
      gone[SET] |= (in && there[j] ? 0u : 1u) << j;
      if constexpr (KC) {
        const int k = half_step(at[j], k0, nk);
        __builtin_memcpy(&code[SET][j], codes[j] + (k >> 1), 8);
        scale[SET][j] = scales[j][k >> 5];
      } else {
        const int64_t k = min(k0 + at[j], nk - 1);
        __builtin_memcpy(&code[SET][j], codes[j] + k * 16 * Nb, 8);
        scale[SET][j] = scales[j][k * Nb];
      }
    }
  }
  template <int SET> __device__ __forceinline__ void commit(int tid, u32x4_t* lds) const {
#pragma unroll
    for (int j = 0; j < NU; ++j) {
      const int u = j * NT + tid, r = u / U, q = u % U;
      if (ALL % NT != 0 && u >= ALL) break;
      const bool in = !(gone[SET] >> j & 1);
      const float s = scale4(in ? scale[SET][j] : 0u);
      lds[unit_at<bf16_t, KC, R>(r, 2 * q)] = bf16_of4(in ? code[SET][j][0] : 0u, s);
      lds[unit_at<bf16_t, KC, R>(r, 2 * q + 1)] = bf16_of4(in ? code[SET][j][1] : 0u, s);
    }
  }
};

// TM x TN results by 2 x 2 waves, both operands through registers at any
// alignment of the rows, two stages in LDS and SETS in flight.  LONG: K is 8 at least.
//
// What bounds it: with one tile a CU how long a stage's loads take, so four stages of the
// small tiles are in flight (two, and a branch around them: 8 rows of 8 groups of
// 2048 x 2048 16.4 us, the gradient 20.1; four 11.3 and 12.8); with several, reads and
// writes of LDS, conversions and products, which a barrier a stage keeps from overlapping
// within a workgroup (400 rows of 32 groups of 2048 x 2048 in 128 x 128 tiles: 147 us,
// 730 TFLOP/s).  128 x 128 tiles have registers for two stages.  By 8 waves these are 8 to
// 20 % faster where a CU has one tile, and a quarter slower where it has more: not built as
// a tile of its own beside this one, between which the choice could tell.
template <typename TO, int MODE, int TM, int TN, int SETS, bool LONG>
__global__ __launch_bounds__(256, 2) void group4_tiles(GroupArgs a, Group4Args b, int band) {
  typedef bf16_t T;
  constexpr int NT = 256, WM = 2, WN = 2, TK = 64;
  constexpr bool XKC = MODE == kFwd, YG = MODE == kFwd;
  constexpr bool LATE = MODE == kBwdIn && SETS == 2;  // no registers for loads beside the products
  constexpr int NI = TM / WM / 16, NJ = TN / WN / 16;
  constexpr int XU = 8 * TM, STAGE = XU + 8 * TN;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  u32x4_t* const ring = reinterpret_cast<u32x4_t*>(smem);

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave % WM, wn = wave / WM;
  auto xrow = [&](int i) { return wm * (TM / WM) + 16 * i; };
  auto yrow = [&](int j) { return wn * (TN / WN) + 16 * j; };

  Tile<T, TO> w;
  if (!setup_tile<T, TO, MODE, TM, TN>(a, band, &w)) return;
  const int64_t g = w.g < a.Ng ? w.g : 0;
  const int rows_x = XKC ? a.M : a.K;  // rows of one group's Ker
  Stager4<XKC, TM, NT, SETS> sx;
  Stager<T, true, TN, NT, YG, SETS> sy;
  Reader<T, XKC, TM, NI> rx;
  Reader<T, true, TN, NJ> ry;
  rx.init(xrow(0), lane);
  ry.init(yrow(0), lane);

  f32x4_t acc[NI][NJ];
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  if (w.K > 0) {
    const uint8_t* const codes = reinterpret_cast<const uint8_t*>(a.X) + g * rows_x * 16 * b.Nb;
    sx.init(tid, codes, b.xs + g * rows_x * b.Nb, b.Nb, w.m0, w.m_valid);
    sy.init(tid, w.Y, a.ldy, w.n0, w.n_valid, YG ? w.rows : nullptr, a.Nsrc);
    const int xk = XKC ? 32 * b.Nb : w.K;
    const int n_st = (w.K + TK - 1) / TK;
    auto compute = [&](const u32x4_t* buf) __attribute__((always_inline)) {
      u32x4_t xf[NI][2], yf[NJ][2];
      rx.read(buf, xf);
      ry.read(buf + XU, yf);
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
          for (int j = 0; j < NJ; ++j) acc[i][j] = mma<T>(xf[i][ks], yf[j][ks], acc[i][j]);
    };
    // stages past the last are loaded too, from where there is something, and never used: a
    // branch around loads would have the compiler wait for all that are in flight
    auto load = [&](auto set, int s) __attribute__((always_inline)) {
      sx.template load<set.value>(s * TK, b.Nb, xk);
      sy.template load<set.value, LONG>(s * TK, a.ldy, w.K, nullptr, 0);
    };
    auto commit = [&](auto set, int s) __attribute__((always_inline)) {
      u32x4_t* const dst = ring + (s & 1) * STAGE;
      sx.template commit<set.value>(tid, dst);
      sy.template commit<set.value, LONG>(tid, dst + XU, s * TK, a.ldy, w.K, nullptr, 0);
    };
    auto step = [&](auto set, int s) __attribute__((always_inline)) {
      __syncthreads();  // stage s is there; every wave is done with stage s - 1
      std::integral_constant<int, (set.value + 1) % SETS> next;
      if constexpr (!LATE) load(set, s + SETS);
      compute(ring + (s & 1) * STAGE);
      if constexpr (LATE) {
        __builtin_amdgcn_sched_barrier(0);
        load(set, s + SETS);
      }
      commit(next, s + 1);
    };
    std::integral_constant<int, 0> s0;
    std::integral_constant<int, 1> s1;
    std::integral_constant<int, 2 % SETS> s2;
    std::integral_constant<int, 3 % SETS> s3;
    load(s0, 0);
    load(s1, 1);
    if constexpr (SETS > 2) {
      load(s2, 2);
      load(s3, 3);
    }
    commit(s0, 0);
    for (int s = 0;;) {
      step(s0, s);
      if (++s == n_st) break;
      step(s1, s);
      if (++s == n_st) break;
      if constexpr (SETS > 2) {
        step(s2, s);
        if (++s == n_st) break;
        step(s3, s);
        if (++s == n_st) break;
      }
    }
  }
  store_tile<T, TO, MODE, MODE == kFwd>(a, w, lane, acc, xrow, yrow);
}

template <typename TO, int MODE, int TM, int TN, bool LONG = true>
hipError_t launch_tiles4(const GroupArgs& a, const Group4Args& b, int64_t row_tiles, int band, hipStream_t stream) {
  auto* const k = group4_tiles<TO, MODE, TM, TN, (TM > 64 ? 2 : 4), LONG>;
  const int64_t grid = row_tiles * ((a.M + TM - 1) / TM);
  const hipError_t fit = grid_fits(grid, 256);
  if (fit != hipSuccess) return fit;
  const int lds = 2 * 8 * (TM + TN) * 16;
  k<<<dim3((uint32_t)grid), dim3(256), lds, stream>>>(a, b, band);
  return hipGetLastError();
}

// Both operands in 4 bits: a block of 32 is 16 bytes, which is what one lane gives
// the scaled matrix instruction (128 values of k by 16 rows: lane l has row l % 16,
// block l / 16 and its scale).  So rows of codes are staged as rows of eight bf16
// values a block are, straight to LDS, and a stage of 128 bytes holds 256 values.
// Lane l takes blocks 2 (l / 16) and the next, whose two scales it loads at once;
// the other operand's lane takes the same.
template <int NB, bool BUF> struct Scales4 {
  const uint8_t* p[BUF ? 1 : NB];  // this lane's rows
  __amdgpu_buffer_rsrc_t rsrc;
  uint32_t off[BUF ? NB : 1];

  // Scales of blocks `at` and the next of rows of Nb (2 at least with BUF, whose loads
  // know no branch), as load() found them; cut() clears what lies past the rows' end
  // (2^-127: the codes there are zeros).
  __device__ __forceinline__ void load(int at, int Nb, uint32_t (&s)[NB]) const {
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      if constexpr (BUF) {
#if defined(__HIP_DEVICE_COMPILE__)
        s[i] = __builtin_amdgcn_raw_buffer_load_b16(rsrc, (int)(off[i] + min(at, Nb - 2)), 0, 0);
#endif
      } else {
        s[i] = at + 1 < Nb ? (uint32_t)p[i][at] | (uint32_t)p[i][at + 1] << 8 : at < Nb ? p[i][at] : 0u;
      }
    }
  }
  __device__ __forceinline__ void cut(int at, int Nb, uint32_t (&s)[NB]) const {
    if constexpr (BUF)
#pragma unroll
      for (int i = 0; i < NB; ++i) s[i] = at + 2 <= Nb ? s[i] : at < Nb ? s[i] >> 8 : 0u;
  }
};

template <int KS>
__device__ __forceinline__ f32x4_t mma4(u32x4_t x, u32x4_t y, f32x4_t acc, uint32_t sx, uint32_t sy) {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef int i32x8_t __attribute__((ext_vector_type(8)));
  const i32x8_t p = {(int)x[0], (int)x[1], (int)x[2], (int)x[3], 0, 0, 0, 0};
  const i32x8_t q = {(int)y[0], (int)y[1], (int)y[2], (int)y[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(p, q, acc, 4, 4, KS, (int)sx, KS, (int)sy);
#else
  (void)x;
  (void)y;
  (void)sx;
  (void)sy;
  return acc;
#endif
}

// BUF: operands by buffer instructions (at most 2^31 bytes of each, two blocks a row at
// least); copies with addresses of their own beside loads make the compiler wait for
// all of both where it needs one.
//
// For few rows a group, bound by Ker's bytes (1536 rows in 60 groups of 1536 x 2048, 94 MB
// of codes: 30 us, 3.2 TB/s in 128 x 32 tiles): a workgroup's start (its tile, the rows'
// numbers, the first copies, 4 us) is as long as its eight stages.
template <typename TO, int TM, int TN, int WM, int WN, int DEPTH, bool BUF>
__global__ __launch_bounds__(64 * WM * WN, 2) void group44_tiles(GroupArgs a, Group4Args b, int band) {
  typedef bf16_t T;
  constexpr int NT = 64 * WM * WN, TK = 64;  // of 16-bit words: 256 values
  constexpr int NI = TM / WM / 16, NJ = TN / WN / 16;
  constexpr int XU = 8 * TM, STAGE = XU + 8 * TN;
  constexpr int NX = XU / NT, NY = 8 * TN / NT;  // units a thread copies
  static_assert(XU % NT == 0 && 8 * TN % NT == 0, "whole rounds");
  extern __shared__ __attribute__((aligned(16))) char smem[];
  u32x4_t* const ring = reinterpret_cast<u32x4_t*>(smem);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, G = lane >> 4;
  const int wm = wave % WM, wn = wave / WM;
  auto xrow = [&](int i) { return wm * (TM / WM) + 16 * i; };
  auto yrow = [&](int j) { return wn * (TN / WN) + 16 * j; };

  Tile<T, TO> w;
  if (!setup_tile<T, TO, kFwd, TM, TN>(a, band, &w)) return;
  const int64_t g = w.g < a.Ng ? w.g : 0;

  f32x4_t acc[NI][NJ];
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  if (w.K > 0) {
    const int Nb = b.Nb;
    const int64_t x0 = g * a.M + w.m0;
    // this thread's unit column, and its rows NT / 8 by NT / 8
    const int r0 = tid >> 3, c8 = 8 * ((tid & 7) ^ ((r0 >> 1) & 7));
    static_assert((NT / 8) % 16 == 0, "one unit column in all rows");
    // Y's rows of this thread's copies and of its lane's scales: their numbers are asked
    // for first, then X, which needs none
    int yrow_of[NY], srow_of[NJ];
    auto number = [&](int n) __attribute__((always_inline)) {
      const int r = w.n0 + min(n, w.n_valid - 1);
      return w.rows ? w.rows[r] : r;
    };
    auto source = [&](int r) __attribute__((always_inline)) -> int64_t { return r < 0 || r >= a.Nsrc ? 0 : r; };
#pragma unroll
    for (int j = 0; j < NY; ++j) yrow_of[j] = number(r0 + j * (NT / 8));
#pragma unroll
    for (int j = 0; j < NJ; ++j) srow_of[j] = number(yrow(j) + l16);
    const T* const X = reinterpret_cast<const T*>(a.X) + x0 * a.ldx + c8;
    const T* const Y = reinterpret_cast<const T*>(a.Y) + c8;
    __amdgpu_buffer_rsrc_t xr, yr;
    int64_t yat[NY];
    uint32_t xoff = 0;
    Scales4<NI, BUF> px;
    Scales4<NJ, BUF> py;
    if constexpr (BUF) {
      xr = rsrc_of(reinterpret_cast<const T*>(a.X) + x0 * a.ldx, (int64_t)w.m_valid * a.ldx * 2);
      yr = rsrc_of(a.Y, (int64_t)a.Nsrc * a.ldy * 2);
      px.rsrc = rsrc_words(b.xs + x0 * Nb, (int64_t)w.m_valid * Nb);
      py.rsrc = rsrc_words(b.ys, (int64_t)a.Nsrc * Nb);
      xoff = (uint32_t)((r0 * a.ldx + c8) * 2);
    }
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int m = min(xrow(i) + l16, w.m_valid - 1);
      if constexpr (BUF) px.off[i] = (uint32_t)(m * Nb);
      else px.p[i] = b.xs + (x0 + m) * Nb;
    }
    const int n_st = (w.K + TK - 1) / TK;
    // past K zeros, so that every wait counts the same
    auto copy_x = [&](int s) __attribute__((always_inline)) {
      u32x4_t* const dst = ring + (s % DEPTH) * STAGE + 64 * wave;
      const bool ok = s * TK + c8 < w.K;
#pragma unroll
      for (int j = 0; j < NX; ++j) {
        const int row = j * (NT / 8);
        if constexpr (BUF) buffer_lds(xr, dst + j * NT, ok ? xoff : kNowhere, (uint32_t)((row * a.ldx + s * TK) * 2));
        else copy16_lds(ok ? (const void*)(X + (int64_t)min(row + r0, w.m_valid - 1) * a.ldx + s * TK) : (const void*)zero_unit, dst + j * NT);
      }
    };
    auto copy_y = [&](int s) __attribute__((always_inline)) {
      u32x4_t* const dst = ring + (s % DEPTH) * STAGE + 64 * wave + XU;
      const bool ok = s * TK + c8 < w.K;
#pragma unroll
      for (int j = 0; j < NY; ++j) {
        if constexpr (BUF) buffer_lds(yr, dst + j * NT, ok ? (uint32_t)((yat[j] + c8) * 2) : kNowhere, (uint32_t)(2 * s * TK));
        else copy16_lds(ok ? (const void*)(Y + yat[j] + s * TK) : (const void*)zero_unit, dst + j * NT);
      }
    };
    uint32_t at[2][2];  // LDS bytes of this lane's units, by sub-step
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      at[0][ks] = 16 * unit_at<T, true, TM>(xrow(0) + l16, 2 * G + ks);
      at[1][ks] = 16 * unit_at<T, true, TN>(yrow(0) + l16, 2 * G + ks);
    }
    uint32_t fx[2][NI], fy[2][NJ];  // scales of this stage and the next
    px.load(2 * G, Nb, fx[0]);
#pragma unroll
    for (int s = 0; s < DEPTH - 1; ++s) copy_x(s);
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int64_t r = source(srow_of[j]);
      if constexpr (BUF) py.off[j] = (uint32_t)(r * Nb);
      else py.p[j] = b.ys + r * Nb;
    }
#pragma unroll
    for (int j = 0; j < NY; ++j) yat[j] = source(yrow_of[j]) * a.ldy;
    py.load(2 * G, Nb, fy[0]);
#pragma unroll
    for (int s = 0; s < DEPTH - 1; ++s) copy_y(s);
    // Stage s has landed and every wave is done with stage s - 1.  What may be in flight: the
    // copies of the stages between and, but for the second stage, the scales asked for with
    // them; of the first, Y's alone, since X's were all asked for before.
    constexpr int kFirst = (DEPTH - 2) * NY;
    constexpr int kSecond = DEPTH == 4 ? 2 * NY + NX : (DEPTH - 2) * (NX + NY);
    constexpr int kLater = (DEPTH - 2) * (NX + NY + (BUF ? NI + NJ : 0));
    auto step = [&](auto set, auto in_flight, int s) __attribute__((always_inline)) {
      constexpr int S = set.value;
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(in_flight.value) : "memory");
      px.load(8 * s + 8 + 2 * G, Nb, fx[1 - S]);
      py.load(8 * s + 8 + 2 * G, Nb, fy[1 - S]);
      copy_x(s + DEPTH - 1);
      copy_y(s + DEPTH - 1);
      const char* const buf = reinterpret_cast<const char*>(ring + (s % DEPTH) * STAGE);
      u32x4_t xf[NI][2], yf[NJ][2];
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
        for (int i = 0; i < NI; ++i) xf[i][ks] = *reinterpret_cast<const u32x4_t*>(buf + at[0][ks] + 2048 * i);
#pragma unroll
        for (int j = 0; j < NJ; ++j) yf[j][ks] = *reinterpret_cast<const u32x4_t*>(buf + 16 * XU + at[1][ks] + 2048 * j);
      }
      px.cut(8 * s + 2 * G, Nb, fx[S]);
      py.cut(8 * s + 2 * G, Nb, fy[S]);
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          acc[i][j] = mma4<0>(xf[i][0], yf[j][0], acc[i][j], fx[S][i], fy[S][j]);
          acc[i][j] = mma4<1>(xf[i][1], yf[j][1], acc[i][j], fx[S][i], fy[S][j]);
        }
    };
    static_assert(DEPTH <= 4, "two first stages");
    constexpr std::integral_constant<int, 0> even;
    constexpr std::integral_constant<int, 1> odd;
    constexpr std::integral_constant<int, kFirst> first;
    constexpr std::integral_constant<int, kSecond> second;
    constexpr std::integral_constant<int, kLater> later;
    step(even, first, 0);
    if (n_st > 1) step(odd, second, 1);
    int s = 2;
    for (; s + 2 <= n_st; s += 2) {
      step(even, later, s);
      step(odd, later, s + 1);
    }
    if (s < n_st) step(even, later, s);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the trailing (empty) copies
  }
  store_tile<T, TO, kFwd, true>(a, w, lane, acc, xrow, yrow);
}

template <typename TO, int TM, int TN, int WM, int WN, int DEPTH, bool BUF = true>
hipError_t launch_tiles44(const GroupArgs& a, const Group4Args& b, int64_t row_tiles, int band, hipStream_t stream) {
  auto* const k = group44_tiles<TO, TM, TN, WM, WN, DEPTH, BUF>;
  const int64_t grid = row_tiles * ((a.M + TM - 1) / TM);
  const hipError_t fit = grid_fits(grid, 64 * WM * WN);
  if (fit != hipSuccess) return fit;
  const int lds = DEPTH * 8 * (TM + TN) * 16;
  if (lds > 64 * 1024) {
    const hipError_t e = allow_max_lds(reinterpret_cast<const void*>(k));
    if (e != hipSuccess) return e;
  }
  k<<<dim3((uint32_t)grid), dim3(64 * WM * WN), lds, stream>>>(a, b, band);
  return hipGetLastError();
}

}  // namespace group
}  // namespace cnnlib
