// Grouped products of bf16 rows, few a group, with Ker in 4 bits, where Ker's bytes are
// the bound: its codes go straight from memory to the matrix registers, since the 16
// bytes of a block are what one lane gives (lane l: feature l % 16, block l / 16 of 128
// of k), and the rows are read so that each lane has the same 32 values.
//
// group4_few: 16 features by 16 rows a workgroup, whose four waves share k and add up
// in LDS: a few rows of long contractions (one group of 4096 x 4096, three rows: 8.0 us,
// by group4_rows 11.8), where no CU has enough workgroups otherwise.
// group4_rows: 64 features by 16 or 32 rows, or 128 by 64; each wave has its own features
// over all of k, and the rows come through a ring in LDS that the waves share.
#include "group4_choice.h"
#include "group4_kernel.h"

namespace cnnlib {

namespace {

using namespace group;

constexpr int kFewWaves = 4;

// A lane's blocks of one row over SB runs of 128 of k: the codes of block 4 i + lane /
// 16 of each run i, and the row's scales, which every lane of the row has (one load of
// them all; where the row ends inside, of its last 4 SB, so that no branch stands between
// these loads and the waits for earlier ones).
template <int SB> struct Blocks4 {
  u32x4_t code[SB];
  uint32_t scale[SB];

  // at: bytes of the row's codes in rsrc; first: block of the first run; past Nb zeros.
  // Rows have 4 SB blocks at least.
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t rsrc, uint32_t at, const uint8_t* scales, int first,
                                       int G, int Nb) {
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
    for (int i = 0; i < SB; ++i) {
      const bool in = first + 4 * i + G < Nb;
      code[i] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rsrc, (int)(in ? at + 16 * G : kNowhere), 16 * first + 64 * i, 0));
    }
    __builtin_memcpy(scale, scales + min(first, Nb - 4 * SB), 4 * SB);
#endif
  }
  // The scale byte of run i's block (in the low bits; others above it).
  __device__ __forceinline__ uint32_t scale_of(int i, int first, int G, int Nb) const {
    const int d = first - (Nb - 4 * SB);
    if (d <= 0) return scale[i] >> (8 * G);
    const int e = 4 * i + G + d;
    uint32_t v = 0u;
#pragma unroll
    for (int q = 0; q < SB; ++q) v = e >> 2 == q ? scale[q] : v;
    return v >> (8 * (e & 3));
  }
};

// Each wave takes every fourth SB runs of k; rows at any alignment.
template <typename TO, int SB>
__global__ __launch_bounds__(64 * kFewWaves) void group4_few(GroupArgs a, Group4Args b) {
  constexpr int NW = kFewWaves;
  __shared__ f32x4_t red[NW * 64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  RowTile t;
  if (!find_tile<16>(a.off, a.Ng, a.N, (a.M + 15) / 16, blockIdx.x, 1, &t)) return;
  const int l16 = lane & 15, G = lane >> 4;
  const int m0 = 16 * t.mt, n_valid = min(t.n1 - t.n0, 16), Nb = b.Nb;
  const bool live = t.g < a.Ng;

  int64_t r = t.n0 + min(l16, n_valid - 1);
  if (a.rows) r = a.rows[r];
  const bool there = r >= 0 && r < a.Nsrc;  // this lane's row is one of In
  if (!there) r = 0;
  f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
  if (live) {
    const int64_t x0 = (int64_t)t.g * a.M + m0;
    const int m_valid = min(a.M - m0, 16), m = min(l16, m_valid - 1);
    const __amdgpu_buffer_rsrc_t xr = rsrc_of(reinterpret_cast<const uint8_t*>(a.X) + x0 * 16 * Nb, (int64_t)m_valid * 16 * Nb);
    const uint8_t* const xs = b.xs + (x0 + m) * Nb;
    const bf16_t* const y = reinterpret_cast<const bf16_t*>(a.Y) + r * a.ldy;
    for (int first = 4 * SB * wave; first < Nb; first += 4 * SB * NW) {
      Blocks4<SB> x;
      u32x4_t v[SB][4];
      x.load(xr, (uint32_t)(m * 16 * Nb), xs, first, G, Nb);
      if (32 * (first + 4 * SB) <= a.K) {
#pragma unroll
        for (int i = 0; i < SB; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) __builtin_memcpy(&v[i][j], y + 32 * (first + 4 * i + G) + 8 * j, 16);
      } else {
#pragma unroll
        for (int i = 0; i < SB; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) v[i][j] = load_end(y, 32 * (first + 4 * i + G) + 8 * j, a.K);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < SB; ++i) {
        const float s = scale4(x.scale_of(i, first, G, Nb) & 255u);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc = mma<bf16_t>(bf16_of4(x.code[i][j], s), v[i][j], acc);
      }
    }
  }
  red[wave * 64 + lane] = acc;
  __syncthreads();
  if (wave != 0 || l16 >= n_valid) return;
  f32x4_t s = red[lane];
#pragma unroll
  for (int w = 1; w < NW; ++w) s += red[w * 64 + lane];
  if (!live || !there) s = f32x4_t{0.f, 0.f, 0.f, 0.f};
  store4(reinterpret_cast<TO*>(a.D) + (t.n0 + l16) * a.ldd, m0 + 4 * G, a.M, s);
}

// FB blocks of 16 features a wave, RB blocks of 16 rows.  A wave asks for SB runs of k of
// its features at a time, 64 SB bytes of each row in loads that follow one another, and
// for the next ones while it multiplies (a run at a time, 64 bytes of a row, half a
// line: 256 rows of two of 28 groups of 4096 x 1024 27.5 us in 64 x 32 tiles, this way
// 20.4, 3.3 TB/s; 8 rows of four of 20 of 1024 x 2048 in 64 x 16 13.1 and 9.0, half of it
// the start).  Four sets of codes in flight were slower (27.3 and 11.2): fewer waves fit,
// and a wait for the rows' copies is one for all older loads.  The rows come through a
// ring of four runs.
template <typename TO, int FB, int RB, int SB>
__global__ __launch_bounds__(256) void group4_rows(GroupArgs a, Group4Args b) {
  constexpr int TM = 64 * FB, TN = 16 * RB, D = 4;
  __shared__ u32x4_t ring[D * TN * 16];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  RowTile t;
  if (!find_tile<TN>(a.off, a.Ng, a.N, (a.M + TM - 1) / TM, blockIdx.x, 1, &t)) return;
  const int l16 = lane & 15, G = lane >> 4, Nb = b.Nb;
  const int m0 = TM * t.mt, n_valid = min(t.n1 - t.n0, TN);
  const bool live = t.g < a.Ng;

  f32x4_t acc[FB][RB];
#pragma unroll
  for (int f = 0; f < FB; ++f)
#pragma unroll
    for (int i = 0; i < RB; ++i) acc[f][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  if (live) {
    // this lane's features (past the last, the last)
    const int64_t x0 = (int64_t)t.g * a.M + m0;
    const int m_valid = min(a.M - m0, TM);
    const __amdgpu_buffer_rsrc_t xr = rsrc_of(reinterpret_cast<const uint8_t*>(a.X) + x0 * 16 * Nb, (int64_t)m_valid * 16 * Nb);
    uint32_t xoff[FB];
    const uint8_t* xs[FB];
#pragma unroll
    for (int f = 0; f < FB; ++f) {
      const int m = min(16 * (FB * wave + f) + l16, m_valid - 1);
      xoff[f] = (uint32_t)(m * 16 * Nb);
      xs[f] = b.xs + (x0 + m) * Nb;
    }
    // this thread's units of a run of rows
    const int c8 = 8 * ((tid & 15) ^ (tid >> 4));
    const __amdgpu_buffer_rsrc_t yr = rsrc_of(a.Y, (int64_t)a.Nsrc * 2 * a.ldy);
    uint32_t src[RB];
    int from[RB];  // the rows' numbers are asked for first, then codes, which need none
#pragma unroll
    for (int i = 0; i < RB; ++i) {
      from[i] = t.n0 + min(16 * i + (tid >> 4), n_valid - 1);
      if (a.rows) from[i] = a.rows[from[i]];
    }
    const int n_run = (Nb + 3) / 4;
    Blocks4<SB> x[2][FB];
    auto load = [&](auto set, int run) __attribute__((always_inline)) {  // the runs from `run` on
#pragma unroll
      for (int f = 0; f < FB; ++f) x[set.value][f].load(xr, xoff[f], xs[f], 4 * run, G, Nb);
    };
    // (copies with addresses of their own, beside loads, make the compiler wait for all
    // of both)
    auto copy_y = [&](int run) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < RB; ++i)
        buffer_lds(yr, ring + ((run & 3) * RB + i) * 256 + 64 * wave, 128 * run + c8 < a.K ? src[i] : kNowhere, 256u * run);
    };
    auto multiply = [&](auto set, auto at, int run0) __attribute__((always_inline)) {
      constexpr int I = at.value;
      const int run = run0 + I;
      // the two runs before this one asked for as many copies and loads after those of
      // this run (of the first of SB, whose codes are needed now too, the copies): it has
      // landed, then every wave's; every wave is done with the last run
      constexpr int X = I == 1 || I == 2 ? 1 : 0;
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(2 * RB + X * FB * (SB + 1)) : "memory");
      if constexpr (I == 0) load(std::integral_constant<int, 1 - set.value>{}, run0 + SB);
      copy_y(run + 3);
      if (run >= n_run) return;
      u32x4_t v[RB][4];
#pragma unroll
      for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i][j] = ring[((run & 3) * RB + i) * 256 + 16 * l16 + ((4 * G + j) ^ l16)];
#pragma unroll
      for (int f = 0; f < FB; ++f) {
        const float s = scale4(x[set.value][f].scale_of(I, 4 * run0, G, Nb) & 255u);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const u32x4_t w = bf16_of4(x[set.value][f].code[I][j], s);
#pragma unroll
          for (int i = 0; i < RB; ++i) acc[f][i] = mma<bf16_t>(w, v[i][j], acc[f][i]);
        }
      }
    };
    auto runs = [&](auto set, int run) __attribute__((always_inline)) {
      multiply(set, std::integral_constant<int, 0>{}, run);
      multiply(set, std::integral_constant<int, 1>{}, run);
      if constexpr (SB == 4) {
        multiply(set, std::integral_constant<int, 2>{}, run);
        multiply(set, std::integral_constant<int, 3>{}, run);
      }
    };
    load(std::integral_constant<int, 0>{}, 0);
#pragma unroll
    for (int i = 0; i < RB; ++i) {
      const int64_t r = from[i] < 0 || from[i] >= a.Nsrc ? 0 : from[i];
      src[i] = (uint32_t)((r * a.ldy + c8) * 2);
    }
    copy_y(0);
    copy_y(1);
    copy_y(2);
    for (int run = 0; run < n_run; run += 2 * SB) {
      runs(std::integral_constant<int, 0>{}, run);
      if (run + SB < n_run) runs(std::integral_constant<int, 1>{}, run + SB);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the trailing (empty) copies
  }
#pragma unroll
  for (int i = 0; i < RB; ++i) {
    const int n = 16 * i + l16;
    if (n >= n_valid) continue;
    bool there = live;
    if (live && a.rows) {
      const int r = a.rows[t.n0 + n];
      there = r >= 0 && r < a.Nsrc;
    }
    TO* const row = reinterpret_cast<TO*>(a.D) + (int64_t)(t.n0 + n) * a.ldd;
#pragma unroll
    for (int f = 0; f < FB; ++f) {
      const f32x4_t v = there ? acc[f][i] : f32x4_t{0.f, 0.f, 0.f, 0.f};
      store4(row, m0 + 16 * (FB * wave + f) + 4 * G, a.M, v);
    }
  }
}

template <typename TO> hipError_t launch_few(const GroupArgs& a, const Group4Args& b, hipStream_t stream) {
  const int64_t blocks = row_tiles(a.N, a.Ng, true, 16) * ((a.M + 15) / 16);
  const hipError_t e = grid_fits(blocks, 64 * kFewWaves);
  if (e != hipSuccess) return e;
  auto* const k = few4_runs(b.Nb) == 4 ? group4_few<TO, 4> : group4_few<TO, 2>;
  k<<<dim3((uint32_t)blocks), dim3(64 * kFewWaves), 0, stream>>>(a, b);
  return hipGetLastError();
}

template <typename TO, int FB, int RB, int SB>
hipError_t launch_rows(const GroupArgs& a, const Group4Args& b, hipStream_t stream) {
  const int64_t blocks = row_tiles(a.N, a.Ng, true, 16 * RB) * ((a.M + 64 * FB - 1) / (64 * FB));
  const hipError_t e = grid_fits(blocks, 256);
  if (e != hipSuccess) return e;
  group4_rows<TO, FB, RB, SB><<<dim3((uint32_t)blocks), dim3(256), 0, stream>>>(a, b);
  return hipGetLastError();
}

template <typename TO>
hipError_t launch_rows_sized(const GroupArgs& a, const Group4Args& b, int rows, hipStream_t stream) {
  switch (rows) {
    case 16: return launch_rows<TO, 1, 1, 4>(a, b, stream);
    case 32: return launch_rows<TO, 1, 2, 4>(a, b, stream);
    default: return launch_rows<TO, 2, 4, 2>(a, b, stream);
  }
}

}  // namespace

hipError_t launch_group4_few(const GroupArgs& a, const Group4Args& b, bool bf16_out, hipStream_t stream) {
  return bf16_out ? launch_few<bf16_t>(a, b, stream) : launch_few<float>(a, b, stream);
}

hipError_t launch_group4_rows(const GroupArgs& a, const Group4Args& b, bool bf16_out, int rows, hipStream_t stream) {
  return bf16_out ? launch_rows_sized<bf16_t>(a, b, rows, stream) : launch_rows_sized<float>(a, b, rows, stream);
}

}  // namespace cnnlib
