// The tile kernel of the grouped products (bf16 and fp32 MFMA, gfx950).
//
// One workgroup computes TM x TN results D[n][m] = sum_k X[m, k] Y[n, k] of
// one group.  m is the result's last index, so the MFMA's row operand is X
// and a lane ends up with four consecutive results of one row n.  Either
// operand may lie with k last (KC: rows of the tile, 128 bytes of k a stage)
// or with the tile's own index last (MC: rows of k, read from LDS by the
// transposing LDS read in bf16):
//   forward       X = Ker[g] (KC), Y = gathered In rows (KC)
//   gradient, In  X = Ker[g] (MC), Y = dOut rows (KC)
//   gradient, Ker X = gathered In rows (MC), Y = dOut rows (MC), k = the rows
//   down          X = A[a] (KC), Y = In rows in the order of their adapters (KC)
//   adapted       X = Ker, Y = In rows in the order of their adapters, one
//                 group, then the low-rank part
// Group sizes are read on the device, so the caller never waits for them: a
// workgroup finds its tile by adding up the groups' tile counts (a wave scans
// 64 groups at a time), and the launch has as many workgroups as the worst
// split of the rows into groups needs.  Rows past the last group are a last
// group without products: their results are zeros.
//
// LDS: each operand's stage is 8 units of 16 bytes per tile row (KC) or the
// same number laid out by k (MC).  Units are permuted within their row so
// that the 16 lanes of a read meet all 64 banks once.
//
// Bound by Ker's bytes where a group has few rows (17 rows a group of 28 experts
// of 4096 x 1024, bf16: 47.5 us, 240 MB at 5.1 TB/s), else by the matrix unit
// and by how the tiles fall on the CUs, which is why there are five tile sizes
// (3002 rows of 6 groups, 515 x 771, fp32: 31 to 35 us, 69 to 76 TFLOP/s).
#pragma once

#include <type_traits>

#include "common.h"
#include "routed.h"

namespace cnnlib {
namespace group {

enum Mode { kFwd = 0, kBwdIn = 1, kBwdKer = 2, kAdapt = 3, kDown = 4 };

#define LDS_AS(T, p) ((__attribute__((address_space(3))) T*)(p))
#define GLB_AS(T, p) ((__attribute__((address_space(1))) T*)(p))

// 16 zero bytes that copies of what lies outside a tensor read instead.
static __device__ __attribute__((aligned(16))) uint32_t zero_unit[4] = {0, 0, 0, 0};

__device__ __forceinline__ void copy16_lds(const void* src, void* lds) {
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_global_load_lds(GLB_AS(void, const_cast<void*>(src)), LDS_AS(void, lds), 16, 0, 0);
#else
  (void)src;
  (void)lds;
#endif
}

// `valid` (at most 16 / sizeof(T)) elements at any element alignment, the rest zeros.
template <typename T> __device__ __forceinline__ u32x4_t load_unit(const T* p, int valid) {
  constexpr int CE = 16 / (int)sizeof(T);
  u32x4_t v = {0u, 0u, 0u, 0u};
  if (valid >= CE) {
    __builtin_memcpy(&v, p, 16);
  } else if (valid > 0) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < CE; ++i)
        if (i < valid) v[i] = __builtin_bit_cast(uint32_t, p[i]);
    } else {
#pragma unroll
      for (int i = 0; i < CE; ++i)
        if (i < valid) v[i >> 1] |= (uint32_t)p[i] << (16 * (i & 1));
    }
  }
  return v;
}

// A unit without its first `e` elements, zeros after the others.
template <typename T> __device__ __forceinline__ u32x4_t drop_first(u32x4_t v, int e) {
  uint64_t lo = (uint64_t)v[1] << 32 | v[0], hi = (uint64_t)v[3] << 32 | v[2];
  const int bits = e * 8 * (int)sizeof(T);
  if (bits >= 128) return u32x4_t{0u, 0u, 0u, 0u};
  if (bits >= 64) {
    lo = hi >> (bits - 64);
    hi = 0;
  } else if (bits > 0) {
    lo = lo >> bits | hi << (64 - bits);
    hi >>= bits;
  }
  return u32x4_t{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}

// The unit from element k on of a row of n elements; zeros past its end.  Where
// the end is inside the unit, one load of the row's last 16 bytes (by elements,
// each load waited for before the next, it took a stage of its own: 28 groups of
// 17 rows of 4097 by 1023 features in bf16, gradient of In, 245 us).
template <typename T> __device__ __forceinline__ u32x4_t load_end(const T* row, int k, int n) {
  constexpr int CE = 16 / (int)sizeof(T);
  if (n < CE) return load_unit(row + k, n - k);
  const int start = min(k, n - CE);
  u32x4_t v;
  __builtin_memcpy(&v, row + start, 16);
  return drop_first<T>(v, k - start);
}

// Where unit `c` (16 bytes) of row `r` of an operand's stage lies.  KC: 8
// units a row, 16 rows of one unit column hit 16 distinct 16-byte columns.
// MC: R * sizeof(T) / 16 units a row of k; bf16 keeps pairs of units (the 32
// bytes a transposing read takes from a row) together and spreads the 8 rows
// that half a wave reads at once, fp32 keeps 64 bytes and spreads the four
// rows a wave reads at once.
template <typename T, bool KC, int R> __device__ __forceinline__ int unit_at(int r, int c) {
  if constexpr (KC) return r * 8 + (c ^ ((r >> 1) & 7));
  constexpr int U = R * (int)sizeof(T) / 16;
  if constexpr (sizeof(T) == 2) {
    const int g = U >= 16  ? (r & 3) | ((r >> 1) & 4)
                  : U == 8 ? ((r >> 1) & 1) | ((r >> 2) & 2)
                           : (r >> 3) & 1;
    static_assert(KC || U >= 4, "a pair of units to trade places with");
    return r * U + (c ^ (g << 1));
  } else {
    static_assert(KC || U >= 8, "four units to trade places with");
    return r * U + (c ^ (((r >> 2) & (U >= 16 ? 3 : 1)) << 2));
  }
}

// Stages one operand: R tile rows by TK values of k, 8 R units by NT threads.
// Rows of the tile past its last read one that is there (their results are not
// stored; source rows that are not there are stored as zeros).
template <typename T, bool KC, int R, int NT, bool GATHER, int SETS = 2> struct Stager {
  static constexpr int CE = 16 / (int)sizeof(T);
  static constexpr int TK = 128 / (int)sizeof(T);
  static constexpr int NU = 8 * R / NT;  // units a thread stages
  static constexpr int U = KC ? 8 : R / CE;
  static_assert(8 * R % NT == 0, "whole rounds");

  const T* p[NU];  // the unit's first element at k = 0, or (rows of k) of a row
  int at[NU];      // KC: the unit's first k within a stage; else its row of k
  int lim[KC ? 1 : NU];  // elements of the row from the unit's first
  bool wide;             // !KC: the row holds a unit; p is at most its last
  int src[GATHER && !KC ? NU : 1];
  u32x4_t regs[SETS][NU];
  uint32_t there[SETS];    // !KC: whether unit j's row of k is (bit j), of each set

  // base: the tensor at its first k; rows [i0, i0 + n) of the tile index are
  // there; ld: elements from row to row; index: source rows of a gathered
  // KC operand.
  __device__ __forceinline__ void init(int tid, const T* base, int64_t ld, int64_t i0, int n,
                                       const int32_t* index, int nsrc) {
    wide = i0 + n >= CE;
#pragma unroll
    for (int j = 0; j < NU; ++j) {
      const int u = j * NT + tid;
      const int r = u / U;
      const int c = unit_at<T, KC, R>(r, u % U) - r * U;  // the permutation is its own inverse
      if constexpr (KC) {
        int64_t row = i0 + min(r, n - 1);
        if constexpr (GATHER)
          if (index) {
            row = index[row];
            if (row < 0 || row >= nsrc) row = 0;
          }
        at[j] = c * CE;
        p[j] = base + row * ld + at[j];
      } else {
        at[j] = r;
        lim[j] = n - c * CE;
        p[j] = base + i0 + (wide ? min(c * CE, n - CE) : lim[j] > 0 ? c * CE : 0);
      }
    }
  }

  // Gathered rows of k: the source rows of the stage at k0 (of nk rows of k),
  // asked for a stage before they are used.
  __device__ __forceinline__ void fetch(int k0, int nk, const int32_t* index) {
    if constexpr (GATHER && !KC)
      if (index)
#pragma unroll
        for (int j = 0; j < NU; ++j) src[j] = index[max(min(k0 + at[j], nk - 1), 0)];
  }
  // The row that unit j reads in the stage at k0 (the one fetched); false: none.
  __device__ __forceinline__ bool row_of(int j, int k0, int nk, const int32_t* index, int nsrc,
                                         int64_t* row) const {
    const int k = k0 + at[j];
    bool ok = k < nk;
    *row = max(min(k, nk - 1), 0);  // the first is there even where nk = 0 asks for zeros
    if constexpr (GATHER)
      if (index) {
        *row = src[j];
        if (*row < 0 || *row >= nsrc) {
          *row = 0;
          ok = false;
        }
      }
    return ok;
  }

  // Straight to LDS, in whole units; what lies past K (nk) reads zeros.
  __device__ __forceinline__ void copy(int tid, u32x4_t* lds, int k0, int64_t ld, int nk,
                                       const int32_t* index, int nsrc) const {
#pragma unroll
    for (int j = 0; j < NU; ++j) {
      const T* src;
      bool ok;
      if constexpr (KC) {
        src = p[j] + k0;
        ok = k0 + at[j] < nk;
      } else {
        int64_t row;
        ok = row_of(j, k0, nk, index, nsrc, &row);
        src = p[j] + row * ld;
      }
      copy16_lds(ok ? (const void*)src : (const void*)zero_unit,
                 lds + j * NT + (__builtin_amdgcn_readfirstlane(tid) & ~63));
    }
  }

  // Through registers (one of SETS sets), at any alignment: loads, and later the
  // LDS writes.  LONG: K holds a unit, and no branch is around the loads.
  template <int SET = 0, bool LONG = false>
  __device__ __forceinline__ void load(int k0, int64_t ld, int nk, const int32_t* index, int nsrc) {
    u32x4_t(&reg)[NU] = regs[SET];
    // what is to be cut off or cleared is so when the loads are waited for, and
    // rows shorter than a unit are read only then
    if constexpr (KC) {
#pragma unroll
      for (int j = 0; j < NU; ++j) {
        if (LONG || nk >= CE) __builtin_memcpy(&reg[j], p[j] - at[j] + min(k0 + at[j], nk - CE), 16);
      }
    } else {
      there[SET] = 0;
#pragma unroll
      for (int j = 0; j < NU; ++j) {
        int64_t row;
        there[SET] |= (uint32_t)row_of(j, k0, nk, index, nsrc, &row) << j;
        if (wide) __builtin_memcpy(&reg[j], p[j] + row * ld, 16);
      }
    }
  }
  // Of the stage at k0, as it was loaded.
  template <int SET = 0, bool LONG = false>
  __device__ __forceinline__ void commit(int tid, u32x4_t* lds, int k0, int64_t ld, int nk,
                                         const int32_t* index, int nsrc) const {
#pragma unroll
    for (int j = 0; j < NU; ++j) {
      u32x4_t v = regs[SET][j];
      if constexpr (KC) {
        if (!LONG && nk < CE) v = load_unit(p[j] + k0, nk - k0 - at[j]);
        else if (k0 + TK > nk) v = drop_first<T>(v, max(k0 + at[j] + CE - nk, 0));
      } else {
        if (!wide) {
          int64_t row = max(min(k0 + at[j], nk - 1), 0);
          if (GATHER && index) {
            row = index[row];
            if (row < 0 || row >= nsrc) row = 0;  // cleared below
          }
          v = load_unit(p[j] + row * ld, lim[j]);
        } else if (lim[j] < CE) {
          v = drop_first<T>(v, CE - lim[j]);
        }
        if (!(there[SET] >> j & 1)) v = u32x4_t{0u, 0u, 0u, 0u};
      }
      lds[j * NT + tid] = v;
    }
  }
};

// The transposing reads of NB blocks of 16 tile rows at LDS addresses p[i]: for
// the 32 values of k from each of two starts KSTEP bytes apart, rows of k 0..3
// and 4..7 (KROWS bytes apart) of each 16 lanes.  Lane 4v + q of 16 reads row
// v, columns 4q .. 4q+3, and receives column l % 16 of the four rows.  One
// block that also waits for them, so the values are defined when it ends, and
// the compiler adds no wait for the copies to LDS that are in flight.
template <int KROWS, int KSTEP>
__device__ __forceinline__ void read_tr_blocks(const uint32_t (&p)[1], u32x4_t (&f)[1][2]) {
#if defined(__HIP_DEVICE_COMPILE__)
  u32x2_t r[4];
  asm volatile(
      "ds_read_b64_tr_b16 %0, %4\n\t"
      "ds_read_b64_tr_b16 %1, %4 offset:%5\n\t"
      "ds_read_b64_tr_b16 %2, %4 offset:%6\n\t"
      "ds_read_b64_tr_b16 %3, %4 offset:%7\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3])
      : "v"(p[0]), "n"(KROWS), "n"(KSTEP), "n"(KSTEP + KROWS)
      : "memory");
#pragma unroll
  for (int ks = 0; ks < 2; ++ks)
    f[0][ks] = u32x4_t{r[2 * ks][0], r[2 * ks][1], r[2 * ks + 1][0], r[2 * ks + 1][1]};
#else
  (void)p;
  (void)f;
#endif
}
template <int KROWS, int KSTEP>
__device__ __forceinline__ void read_tr_blocks(const uint32_t (&p)[2], u32x4_t (&f)[2][2]) {
#if defined(__HIP_DEVICE_COMPILE__)
  u32x2_t r[8];
  asm volatile(
      "ds_read_b64_tr_b16 %0, %8\n\t"
      "ds_read_b64_tr_b16 %1, %8 offset:%10\n\t"
      "ds_read_b64_tr_b16 %2, %9\n\t"
      "ds_read_b64_tr_b16 %3, %9 offset:%10\n\t"
      "ds_read_b64_tr_b16 %4, %8 offset:%11\n\t"
      "ds_read_b64_tr_b16 %5, %8 offset:%12\n\t"
      "ds_read_b64_tr_b16 %6, %9 offset:%11\n\t"
      "ds_read_b64_tr_b16 %7, %9 offset:%12\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]),
        "=&v"(r[7])
      : "v"(p[0]), "v"(p[1]), "n"(KROWS), "n"(KSTEP), "n"(KSTEP + KROWS)
      : "memory");
#pragma unroll
  for (int ks = 0; ks < 2; ++ks)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const u32x2_t lo = r[4 * ks + 2 * i], hi = r[4 * ks + 2 * i + 1];
      f[i][ks] = u32x4_t{lo[0], lo[1], hi[0], hi[1]};
    }
#else
  (void)p;
  (void)f;
#endif
}
template <int KROWS, int KSTEP>
__device__ __forceinline__ void read_tr_blocks(const uint32_t (&p)[4], u32x4_t (&f)[4][2]) {
#if defined(__HIP_DEVICE_COMPILE__)
  u32x2_t r[16];
  asm volatile(
      "ds_read_b64_tr_b16 %0, %16\n\t"
      "ds_read_b64_tr_b16 %1, %16 offset:%20\n\t"
      "ds_read_b64_tr_b16 %2, %17\n\t"
      "ds_read_b64_tr_b16 %3, %17 offset:%20\n\t"
      "ds_read_b64_tr_b16 %4, %18\n\t"
      "ds_read_b64_tr_b16 %5, %18 offset:%20\n\t"
      "ds_read_b64_tr_b16 %6, %19\n\t"
      "ds_read_b64_tr_b16 %7, %19 offset:%20\n\t"
      "ds_read_b64_tr_b16 %8, %16 offset:%21\n\t"
      "ds_read_b64_tr_b16 %9, %16 offset:%22\n\t"
      "ds_read_b64_tr_b16 %10, %17 offset:%21\n\t"
      "ds_read_b64_tr_b16 %11, %17 offset:%22\n\t"
      "ds_read_b64_tr_b16 %12, %18 offset:%21\n\t"
      "ds_read_b64_tr_b16 %13, %18 offset:%22\n\t"
      "ds_read_b64_tr_b16 %14, %19 offset:%21\n\t"
      "ds_read_b64_tr_b16 %15, %19 offset:%22\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]),
        "=&v"(r[7]), "=&v"(r[8]), "=&v"(r[9]), "=&v"(r[10]), "=&v"(r[11]), "=&v"(r[12]),
        "=&v"(r[13]), "=&v"(r[14]), "=&v"(r[15])
      : "v"(p[0]), "v"(p[1]), "v"(p[2]), "v"(p[3]), "n"(KROWS), "n"(KSTEP), "n"(KSTEP + KROWS)
      : "memory");
#pragma unroll
  for (int ks = 0; ks < 2; ++ks)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const u32x2_t lo = r[8 * ks + 2 * i], hi = r[8 * ks + 2 * i + 1];
      f[i][ks] = u32x4_t{lo[0], lo[1], hi[0], hi[1]};
    }
#else
  (void)p;
  (void)f;
#endif
}

// Reads a stage's operands of NB blocks of 16 tile rows from row0 on, for both
// sub-steps.  bf16: 32 values of k each, lane l row l % 16 and k = 8 (l / 16) +
// 0..7.  fp32: 16 values of k, element e of lane l is k = 4 (l / 16) + e, used
// by the e-th of four MFMAs.
template <typename T, bool KC, int R, int NB> struct Reader {
  uint32_t at[KC ? 2 : NB];

  __device__ __forceinline__ void init(int row0, int lane) {
    const int l16 = lane & 15, G = lane >> 4;
    if constexpr (KC) {
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) at[ks] = 16 * unit_at<T, true, R>(row0 + l16, 4 * ks + G);
    } else if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < NB; ++i)
        at[i] = 16 * unit_at<T, false, R>(8 * G + (l16 >> 2), (row0 >> 3) + 2 * i + ((l16 & 3) >> 1)) +
                8 * (l16 & 1);
    } else {
#pragma unroll
      for (int i = 0; i < NB; ++i)
        at[i] = 16 * unit_at<T, false, R>(4 * G, (row0 >> 2) + 4 * i + (l16 >> 2)) + 4 * (l16 & 3);
    }
  }
  __device__ __forceinline__ void read(const u32x4_t* lds, u32x4_t (&f)[NB][2]) const {
    const char* const base = reinterpret_cast<const char*>(lds);
    if constexpr (KC) {
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int i = 0; i < NB; ++i)
          f[i][ks] = *reinterpret_cast<const u32x4_t*>(base + at[ks] + 2048 * i);
    } else if constexpr (sizeof(T) == 2) {
      // the unit permutation is that of 4 and of 32 rows further on
      const uint32_t start = (uint32_t)(uintptr_t)LDS_AS(char, const_cast<char*>(base));
      uint32_t q[NB];
#pragma unroll
      for (int i = 0; i < NB; ++i) q[i] = start + at[i];
      read_tr_blocks<4 * 2 * R, 32 * 2 * R>(q, f);
    } else {
      // of the 3 rows further on, and of 16
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            f[i][ks][e] = *reinterpret_cast<const uint32_t*>(base + at[i] + (16 * ks + e) * 4 * R);
    }
  }
};

template <typename T>
__device__ __forceinline__ f32x4_t mma(u32x4_t x, u32x4_t y, f32x4_t acc) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, x),
                                                   __builtin_bit_cast(bf16x8_t, y), acc, 0, 0, 0);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x[e]), __uint_as_float(y[e]), acc,
                                                 0, 0, 0);
    return acc;
  }
}

// Four consecutive results from `m` of one row, as many as lie below M, at any
// element alignment.
template <typename TO>
__device__ __forceinline__ void store4(TO* row, int m, int M, f32x4_t v) {
  if (m + 4 <= M) {
    if constexpr (sizeof(TO) == 4) {
      __builtin_memcpy(row + m, &v, 16);
    } else {
      const u32x2_t p = {pk_bf16(v[0], v[1]), pk_bf16(v[2], v[3])};
      __builtin_memcpy(row + m, &p, 8);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (m + e < M) row[m + e] = from_f32<TO>(v[e]);
  }
}

// A row tile of the groups: its group (Ng: the rows past the last), the rows
// [n0, n1) of the group from the tile's first on, and its tile of m.
struct RowTile {
  int g, n0, n1, mt;
  int part;  // of a tile halved by features, 1 or 2; else 0
};
// Workgroups of a round of tiles that fill a CU each: MI355X's CUs.  Where a part of the
// GPU has fewer, tiles of other rounds than the last are halved: the same results, but
// later, since a half takes three quarters of a tile's time.
constexpr int kRound = 256;

// Rows of group g; group Ng is the rows past the last.
__device__ __forceinline__ void group_rows(const int32_t* off, int Ng, int Np, int g, int* lo,
                                           int* hi) {
  *lo = off[g];
  *hi = g < Ng ? off[g + 1] : Np;
}

// v of the lane that a data-parallel move names; 0 where there is none.
template <int CTRL, int ROWS = 0xf> __device__ __forceinline__ int move_lanes(int v) {
  return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false);
}

// Inclusive sum over the wave's lanes: within rows of 16 by shifts of 1, 2, 4
// and 8, then each row's last lane into the rows after it.
__device__ __forceinline__ int wave_scan(int v) {
  v += move_lanes<0x111>(v);
  v += move_lanes<0x112>(v);
  v += move_lanes<0x114>(v);
  v += move_lanes<0x118>(v);
  v += move_lanes<0x142, 0xa>(v);  // lane 15 of rows 0 and 2 into rows 1 and 3
  v += move_lanes<0x143, 0xc>(v);  // lane 31 into rows 2 and 3
  return v;
}

// The least v of each row of 16 lanes, in all of them.
__device__ __forceinline__ int row16_min(int v) {
  v = min(v, move_lanes<0xb1>(v));   // quad_perm 1,0,3,2
  v = min(v, move_lanes<0x4e>(v));   // quad_perm 2,3,0,1
  v = min(v, move_lanes<0x141>(v));  // row_half_mirror
  v = min(v, move_lanes<0x140>(v));  // row_mirror
  return v;
}

// The tile of workgroup `bid` of a launch over the groups' row tiles by MT
// tiles of m; false: none.  The rows past the last group come last and are
// spread over the XCDs by themselves: their tiles cost nothing, and among the
// others they leave one XCD idle and the rest a round more (15560 rows of 8
// groups and 819 without one, 2048 features: 64 row tiles in 149 us, now 117).
// SPLIT: whole row tiles come first, then those that a group's rows fill to
// more than half, then the rest, so that the launch ends on the cheaper ones
// (large tiles; small ones keep a group together, whose Ker they share).  Row
// tiles are walked in bands: `band` row tiles by every m tile, so that the
// tiles an XCD runs at a time share their rows of X and Y in its L2.  Offsets
// that are not an order (documented as the caller's duty) are found out by the
// wave that adds them up: no tile is then run.
// HALVES: a last round of few tiles has each of them twice, halved by features (the
// launch has kRound / 2 workgroups more).
template <int TN, bool SPLIT = false, bool HALVES = false>
__device__ __forceinline__ bool find_tile(const int32_t* off, int Ng, int Np, int MT, int bid,
                                          int band, RowTile* t) {
  const int lane = threadIdx.x & 63;
  int nt, j0, lo_g = 0, hi_g = Np;  // row tiles of the group, tile within it, its rows
  int first = 0;                    // the first of those row tiles
  t->g = 0;
  t->part = 0;
  if (!off) {
    nt = (Np + TN - 1) / TN;
    if (bid >= nt * MT) return false;
    j0 = xcd_remap(bid, nt * MT);
  } else {
    // up to 64 groups: one pass, else one for the totals and one for the tile.
    // Row tiles by kind: 0 all of them, or the whole ones; 1, 2 (one count in
    // each half of `parts`) those more and less than half filled
    int lo = 0, hi = 0, whole = 0, parts = 0, n_of[3] = {0, 0, 0};
    auto scan = [&](int base) __attribute__((always_inline)) {
      const int g = base + lane;
      lo = hi = 0;
      if (g < Ng) group_rows(off, Ng, Np, g, &lo, &hi);
      whole = wave_scan((hi - lo + (SPLIT ? 0 : TN - 1)) / TN);
      if (SPLIT) {
        const int part = (hi - lo) % TN;
        parts = wave_scan(part == 0 ? 0 : part > TN / 2 ? 1 : 0x10000);
      }
    };
    for (int base = 0; base < Ng; base += 64) {
      scan(base);
      if (__ballot(lo < 0 || hi < lo || hi > Np || (base + lane == 0 && lo != 0))) return false;
      n_of[0] += __builtin_amdgcn_readlane(whole, 63);
      const int both = __builtin_amdgcn_readlane(parts, 63);
      n_of[1] += both & 0xffff;
      n_of[2] += both >> 16;
    }
    if constexpr (HALVES) {
      const int all = (n_of[0] + n_of[1] + n_of[2]) * MT, left = all % kRound, at = bid - (all - left);
      if (left <= kRound / 2 && at >= 0) {
        if (at < 2 * left) t->part = 1 + (at & 1);
        bid -= t->part ? at - (at >> 1) : left;
      }
    }
    int kind = 0;
    while (kind < (SPLIT ? 3 : 1) && bid >= n_of[kind] * MT) bid -= n_of[kind++] * MT;
    if (kind == (SPLIT ? 3 : 1)) {
      lo_g = __builtin_amdgcn_readfirstlane(off[Ng]);
      nt = (Np - lo_g + TN - 1) / TN;
      if (bid >= nt * MT) return false;
      t->g = Ng;
      j0 = bid;
    } else {
      const int L = xcd_remap(bid, n_of[kind] * MT);
      int before = 0;
      for (int base = 0;; base += 64) {
        if (Ng > 64) scan(base);
        const int incl = kind == 0 ? whole : kind == 1 ? parts & 0xffff : parts >> 16;
        const uint64_t here = __ballot(L < (before + incl) * MT);
        if (here) {
          const int who = __ffsll((unsigned long long)here) - 1;
          lo_g = __builtin_amdgcn_readlane(lo, who);
          hi_g = __builtin_amdgcn_readlane(hi, who);
          nt = kind ? 1 : (hi_g - lo_g + (SPLIT ? 0 : TN - 1)) / TN;
          first = kind ? (hi_g - lo_g) / TN : 0;
          j0 = L - (before + __builtin_amdgcn_readlane(incl, who) - nt) * MT;
          t->g = base + who;
          break;
        }
        before += __builtin_amdgcn_readlane(incl, 63);
      }
    }
  }
  const int b = j0 / (band * MT), rb = min(band, nt - b * band), j = j0 - b * band * MT;
  t->mt = j / rb;
  t->n0 = lo_g + (first + b * band + j % rb) * TN;
  t->n1 = hi_g;
  return true;
}

// The group of the gradient of Ker's workgroup `bid`, tiles_per of them a
// group: the groups with most rows come first, for a tile's time is its
// group's rows.  Of more than 64 groups as they come.
__device__ __forceinline__ int group_by_rows(const int32_t* off, int Ng, int Np, int bid,
                                             int tiles_per) {
  const int lane = threadIdx.x & 63, want = bid / tiles_per;
  if (Ng > 64) return want;
  int lo = 0, hi = -1;
  if (lane < Ng) group_rows(off, Ng, Np, lane, &lo, &hi);
  const int rows = hi - lo;
  int rank = 0;
  for (int g = 0; g < Ng; ++g) {
    const int r = __builtin_amdgcn_readlane(rows, g);
    rank += r > rows || (r == rows && g < lane);
  }
  const uint64_t me = __ballot(lane < Ng && rank == want);
  return __ffsll((unsigned long long)me) - 1;
}

// Part `part` of h as the sum of bf16 values: the leading 8 bits of what the
// earlier parts left.  What is not finite is all in the first part.
__device__ __forceinline__ float bf16_part(float h, int part) {
  if (!(fabsf(h) < INFINITY)) return part == 0 ? to_f32(from_f32<bf16_t>(h)) : 0.f;
  float v = __uint_as_float(__float_as_uint(h) & 0xffff0000u);
  for (int i = 0; i < part; ++i) {
    h -= v;
    v = __uint_as_float(__float_as_uint(h) & 0xffff0000u);
  }
  return v;
}

// B's values as the later parts of H meet them (bf16): infinities and
// NaN are replaced by the type's largest value.  A later part may be zero, and
// zero times infinity would be NaN; the first part, which is zero only where H
// is (to 2^-133), gives what is due.  Finite values stay, and so does all of a first part's.
__device__ __forceinline__ u32x4_t met_by_part(u32x4_t b, bool later) {
  typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
  const u16x2_t most = __builtin_bit_cast(u16x2_t, later ? 0x7f7f7f7fu : 0x7fff7fffu);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const u16x2_t size = __builtin_bit_cast(u16x2_t, b[i] & 0x7fff7fffu);
    b[i] = (b[i] & 0x80008000u) | __builtin_bit_cast(uint32_t, __builtin_elementwise_min(size, most));
  }
  return b;
}

// A workgroup's tile: its operands and result from the tile's (and, for the
// gradient of Ker, the group's) start.
template <typename T, typename TO> struct Tile {
  const T* X;
  const T* Y;
  TO* D;
  const int32_t* rows;  // NULL, or the source rows of grouped rows n0 .. or of k = 0 ..
  int K, m0, m_valid, n0, n_valid, g;
};

template <typename T, typename TO, int MODE, int TM, int TN, bool HALVES = false>
__device__ __forceinline__ bool setup_tile(const GroupArgs& a, int band, Tile<T, TO>* w) {
  const int MT = (a.M + TM - 1) / TM;
  w->X = reinterpret_cast<const T*>(a.X);
  w->Y = reinterpret_cast<const T*>(a.Y);
  w->D = reinterpret_cast<TO*>(a.D);
  w->rows = a.rows;
  int mt, part = 0;
  if constexpr (MODE == kBwdKer) {
    const int NTL = (a.N + TN - 1) / TN;
    const int g = group_by_rows(a.off, a.Ng, a.K, blockIdx.x, MT * NTL);
    const int j0 = xcd_remap(blockIdx.x % (MT * NTL), MT * NTL);
    const int b = j0 / (band * MT), rb = min(band, NTL - b * band), j = j0 - b * band * MT;
    mt = j / rb;
    w->n0 = (b * band + j % rb) * TN;
    int lo, hi;
    group_rows(a.off, a.Ng, a.K, g, &lo, &hi);
    // clamped, so that no offset leads outside the tensors
    lo = min(max(__builtin_amdgcn_readfirstlane(lo), 0), a.K);
    w->K = min(max(__builtin_amdgcn_readfirstlane(hi), lo), a.K) - lo;
    w->n_valid = min(a.N - w->n0, TN);
    w->g = g;
    if (a.rows) w->rows += lo; else w->X += lo * a.ldx;
    w->Y += lo * a.ldy;
    w->D += g * a.dgroup + (int64_t)w->n0 * a.ldd;
  } else {
    RowTile t;
    if (!find_tile<TN, TN == 256, HALVES>(a.off, a.Ng, a.N, MT, blockIdx.x, band, &t)) return false;
    part = t.part;
    w->K = t.g < a.Ng ? a.K : 0;  // the rows past the last group: no products
    w->n0 = t.n0;
    w->g = t.g;
    w->n_valid = min(t.n1 - t.n0, TN);
    w->X += (t.g < a.Ng ? t.g : 0) * a.xgroup;
    // adapted rows go back to where they came from
    if constexpr (MODE < kAdapt) w->D += (int64_t)t.n0 * a.ldd;
    mt = t.mt;
  }
  w->m0 = mt * TM + (part == 2 ? TM / 2 : 0);
  w->m_valid = min(a.M - w->m0, part ? TM / 2 : TM);
  return !HALVES || w->m_valid > 0;
}

// Eight consecutive bf16 results from `m` of one row, as many as lie below M.
__device__ __forceinline__ void store8(bf16_t* row, int m, int M, u32x4_t v) {
  if (m + 8 <= M) {
    __builtin_memcpy(row + m, &v, 16);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (m + e < M) row[m + e] = (bf16_t)(v[e >> 1] >> (16 * (e & 1)));
  }
}

// Results acc[i][j] of 16 values of m from xrow(i) by 16 rows from yrow(j).
// MASK: rows whose source row is not there are stored as zeros.  A lane has
// four results of a row in each block: 16 bytes of fp32, 64 bytes a row and
// store.  In bf16 two neighbouring blocks trade the odd 16 lanes of the one for
// the even of the other, which makes it 16 and 64 bytes again (8 bytes a lane
// store at half the rate: 128 MB of results 40 us and, this way, 24).
template <typename T, typename TO, int MODE, bool MASK, int NI, int NJ, typename XR, typename YR>
__device__ __forceinline__ void store_tile(const GroupArgs& a, const Tile<T, TO>& w, int lane,
                                           f32x4_t (&acc)[NI][NJ], XR xrow, YR yrow) {
  const int l16 = lane & 15, G = lane >> 4;
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const int n = yrow(j) + l16;
    const bool there = n < w.n_valid;
    int64_t at = n;
    bool live = true;
    if constexpr (MASK || MODE == kAdapt) {
      if (w.rows) {
        const int r = w.rows[w.n0 + min(n, w.n_valid - 1)];
        if constexpr (MODE == kAdapt) at = r;
        live = r >= 0 && r < a.Nsrc;
      }
    }
    TO* const row = w.D + at * a.ldd;
    if constexpr (sizeof(TO) == 2 && NI % 2 == 0) {
      const bool eights = (a.M & 7) == 0;  // no row ends inside eight results
#pragma unroll
      for (int i = 0; i < NI; i += 2) {
        u32x4_t v;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t p = pk_bf16(acc[i][j][2 * e], acc[i][j][2 * e + 1]);
          const uint32_t q = pk_bf16(acc[i + 1][j][2 * e], acc[i + 1][j][2 * e + 1]);
          const auto r = __builtin_amdgcn_permlane16_swap(p, q, false, false);
          v[e] = live ? r[0] : 0u;
          v[2 + e] = live ? r[1] : 0u;
        }
        const int m = w.m0 + xrow(i) + 16 * (G & 1) + 8 * (G >> 1);
        if (there) {
          if (!eights) store8(row, m, a.M, v);
          else if (m < a.M) store8(row, m, m + 8, v);
        }
      }
    } else {
      const bool fours = (a.M & 3) == 0;  // no row ends inside four results
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int m = w.m0 + xrow(i) + 4 * G;
        f32x4_t v = acc[i][j];
        if constexpr (MASK)
          if (!live) v = f32x4_t{0.f, 0.f, 0.f, 0.f};
        if (there) {
          if (!fours) store4(row, m, a.M, v);
          else if (m < a.M) store4(row, m, m + 4, v);
        }
      }
    }
  }
}

// Rows of the low-rank operand from the results of In A^T: scaled, and in bf16
// as the sum of three bf16 values of 8 bits each, all 24 of the fp32 one, each
// part nlp ranks (zeros past M).  Two parts, for a bf16 result, cut off up to
// 2^-15 of a value, always with one sign: the result then was 1.0e-4 of its norm
// from that of an fp32 factor (rank 64, 2048 features), where the order of the
// sums makes 2e-5.
template <typename T, typename TO, int NI, int NJ, typename XR, typename YR>
__device__ __forceinline__ void store_parts(const GroupArgs& a, const AdaptArgs& ad,
                                            const Tile<T, TO>& w, int lane, f32x4_t (&acc)[NI][NJ],
                                            XR xrow, YR yrow) {
  constexpr int PARTS = sizeof(T) == 4 ? 1 : 3;
  const float scale = ad.scales ? ad.scales[w.g] : 1.f;
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const int n = yrow(j) + (lane & 15);
    T* const row = reinterpret_cast<T*>(ad.Hp) + (int64_t)(w.n0 + min(n, w.n_valid - 1)) * ad.hl;
    const int ranks = n < w.n_valid ? ad.nlp : 0;  // a multiple of four
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int m = w.m0 + xrow(i) + 4 * (lane >> 4);
      float h[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) h[e] = m + e < a.M ? acc[i][j][e] * scale : 0.f;
      if constexpr (sizeof(T) == 4) {
        if (m < ranks) __builtin_memcpy(row + m, h, 16);
      } else {
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
          bf16_t v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = (bf16_t)(__float_as_uint(bf16_part(h[e], p)) >> 16);
          if (m < ranks) __builtin_memcpy(row + p * ad.nlp + m, v, 8);
        }
      }
    }
  }
}

// The low-rank part of an adapted tile, added to acc: for each adapter that
// the wave's rows name, one more run of k over the parts of H.  Both operands
// come straight from memory (a few KB that the workgroup's waves share in
// their caches), so there is nothing to wait for but this wave's own loads.
// Each adapter's products go to its own rows only: another's infinities must
// not meet them, not even as products with zero.  Four by two blocks of acc
// at a time, so that no more is carried around the loops.
// WHOLE: Nl is a multiple of a unit, else B's rows are read by elements.
template <typename T, typename TO, bool WHOLE, int NI, int NJ, typename XR, typename YR>
__device__ __forceinline__ void low_rank(const GroupArgs& a, const AdaptArgs& ad,
                                         const Tile<T, TO>& w, int lane, f32x4_t (&acc)[NI][NJ],
                                         XR xrow, YR yrow) {
  constexpr int CE = 16 / (int)sizeof(T), STEP = 4 * CE;
  constexpr int BATCH = WHOLE ? 2 : 1;  // steps whose loads are in flight together
  constexpr int IB = NI < 4 ? NI : 4, JB = NJ < 2 ? NJ : 2;
  static_assert(NI % IB == 0 && NJ % JB == 0, "whole rounds of blocks");
  const u32x4_t zero = {0u, 0u, 0u, 0u};
  const int l16 = lane & 15, G = lane >> 4;
  const T* const H = reinterpret_cast<const T*>(ad.Hp) + (int64_t)w.n0 * ad.hl;
#pragma unroll
  for (int j0 = 0; j0 < NJ; j0 += JB) {
    int id_of[JB];  // adapter of this lane's rows; past the tile, the last row's
    uint32_t hrow[JB];
#pragma unroll
    for (int j = 0; j < JB; ++j) {
      const int n = min(yrow(j0 + j) + l16, w.n_valid - 1);
      id_of[j] = ad.ids[w.n0 + n];
      hrow[j] = (uint32_t)(n * ad.hl);
    }
#pragma unroll
    for (int i0 = 0; i0 < NI; i0 += IB) {
      uint32_t brow[IB];
#pragma unroll
      for (int i = 0; i < IB; ++i)
        brow[i] = (uint32_t)(min(xrow(i0 + i) + l16, w.m_valid - 1) * ad.Nl);
      int last = -1;
#pragma unroll 1
      for (;;) {
        int next = 0x7fffffff;  // the least adapter above the last one
#pragma unroll
        for (int j = 0; j < JB; ++j)
          if (id_of[j] > last && id_of[j] < ad.Na) next = min(next, id_of[j]);
        // the four rows of 16 lanes hold the same
        next = __builtin_amdgcn_readfirstlane(row16_min(next));
        if (next == 0x7fffffff) break;
        last = next;
        const T* const B = reinterpret_cast<const T*>(ad.B) + ((int64_t)next * a.M + w.m0) * ad.Nl;
#pragma unroll 1
        for (int k0 = 0; k0 < ad.hl; k0 += BATCH * STEP) {
          u32x4_t xf[BATCH][IB], yf[BATCH][JB];
          bool in[BATCH];
#pragma unroll
          for (int s = 0; s < BATCH; ++s) {
            in[s] = k0 + s * STEP + CE * G < ad.hl;
            const int kk = in[s] ? k0 + s * STEP + CE * G : 0, rank = kk % ad.nlp;
#pragma unroll
            for (int j = 0; j < JB; ++j) __builtin_memcpy(&yf[s][j], H + hrow[j] + kk, 16);
#pragma unroll
            for (int i = 0; i < IB; ++i) {
              const T* const row = B + brow[i];
              if constexpr (WHOLE) {
                __builtin_memcpy(&xf[s][i], row + rank, 16);
              } else {
                T v[CE];
#pragma unroll
                for (int e = 0; e < CE; ++e) v[e] = row[min(rank + e, ad.Nl - 1)];
#pragma unroll
                for (int e = 0; e < CE; ++e) v[e] = rank + e < ad.Nl ? v[e] : (T)0;
                __builtin_memcpy(&xf[s][i], v, 16);
              }
            }
          }
          __builtin_amdgcn_sched_barrier(0);
          if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int s = 0; s < BATCH; ++s)
#pragma unroll
              for (int i = 0; i < IB; ++i)
                xf[s][i] = met_by_part(xf[s][i], k0 + s * STEP + CE * G >= ad.nlp);
          }
#pragma unroll
          for (int j = 0; j < JB; ++j)
#pragma unroll
            for (int i = 0; i < IB; ++i) {
              f32x4_t sum = acc[i0 + i][j0 + j];
#pragma unroll
              for (int s = 0; s < BATCH; ++s)
                sum = mma<T>(in[s] ? xf[s][i] : zero, in[s] ? yf[s][j] : zero, sum);
#pragma unroll
              for (int e = 0; e < 4; ++e)
                acc[i0 + i][j0 + j][e] = id_of[j] == next ? sum[e] : acc[i0 + i][j0 + j][e];
            }
        }
      }
    }
  }
}

// The order of what follows the last wait: between a stage's MFMAS matrix
// instructions, its reads (two at a time), copies and their addresses, which a
// wave alone on its SIMD has nothing else to hide behind.  With more of the
// addresses to an instruction in bf16, whose are a quarter as many: 1000 rows of
// 2048 x 2048 16.5 us, in this order 16.0; fp32, 100 rows of 1024 x 1024 10.4 and 9.6.
template <typename T, int MFMAS> __device__ __forceinline__ void interleave() {
#pragma unroll
  for (int i = 0; i < MFMAS; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);                        // matrix
    __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);                      // LDS reads
    __builtin_amdgcn_sched_group_barrier(0x6, sizeof(T) == 4 ? 2 : 8, 0);  // vector, scalar
    __builtin_amdgcn_sched_group_barrier(0x10, 1, 0);                       // copies
  }
}

// TM x TN results by WM x WN waves.  DEPTH > 0: both operands are copied
// straight to LDS (rows on 4-byte boundaries), DEPTH - 1 stages ahead in a ring
// of DEPTH.  AHEAD: a wave reads a stage while it multiplies the one before, and
// the copies are a stage further ahead (64 x 64 and less: 3 to 11 % less time in
// the forward product at 100 to 3000 rows; 128 x 128 has no registers for it, and
// the transposing reads of bf16 are waited for where they are made).  Where K ends inside a unit, its last stage goes through registers.
// DEPTH 0: through registers, at any alignment, two stages in LDS and, in small tiles, two ahead.  WHOLE: see low_rank.
template <typename T, typename TO, int MODE, int TM, int TN, int WM, int WN, int DEPTH, bool WHOLE>
__global__ __launch_bounds__(64 * WM * WN, 2) void group_tiles(GroupArgs a, AdaptArgs ad, int band) {
  constexpr int NT = 64 * WM * WN;
  constexpr bool XKC = MODE == kFwd || MODE >= kAdapt, YKC = MODE != kBwdKer;
  constexpr bool XG = MODE == kBwdKer, YG = MODE == kFwd || MODE >= kAdapt;  // gathered operands
  constexpr int CE = 16 / (int)sizeof(T), TK = 8 * CE;
  constexpr int NI = TM / WM / 16, NJ = TN / WN / 16;
  constexpr int XU = 8 * TM, STAGE = XU + 8 * TN;
  constexpr bool AHEAD = TM < 128 && YKC && (XKC || sizeof(T) == 4);

  extern __shared__ __attribute__((aligned(16))) char smem[];
  u32x4_t* const ring = reinterpret_cast<u32x4_t*>(smem);

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave % WM, wn = wave / WM;
  auto xrow = [&](int i) { return wm * (TM / WM) + 16 * i; };
  auto yrow = [&](int j) { return wn * (TN / WN) + 16 * j; };

  Tile<T, TO> w;
  if (!setup_tile<T, TO, MODE, TM, TN>(a, band, &w)) return;
  Stager<T, XKC, TM, NT, XG> sx;
  Stager<T, YKC, TN, NT, YG> sy;
  const int32_t* const xrows = XG ? w.rows : nullptr;
  Reader<T, XKC, TM, NI> rx;
  Reader<T, YKC, TN, NJ> ry;
  rx.init(xrow(0), lane);
  ry.init(yrow(0), lane);

  f32x4_t acc[NI][NJ];
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  auto multiply = [&](const u32x4_t(&xf)[NI][2], const u32x4_t(&yf)[NJ][2]) __attribute__((always_inline)) {
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[i][j] = mma<T>(xf[i][ks], yf[j][ks], acc[i][j]);
  };
  auto compute = [&](const u32x4_t* buf) __attribute__((always_inline)) {
    u32x4_t xf[NI][2], yf[NJ][2];
    rx.read(buf, xf);
    ry.read(buf + XU, yf);
    multiply(xf, yf);
  };
  auto load = [&](auto set, int s) __attribute__((always_inline)) {
    sx.template load<set.value>(s * TK, a.ldx, w.K, xrows, a.Nsrc);
    sx.fetch((s + 1) * TK, w.K, xrows);
    sy.template load<set.value>(s * TK, a.ldy, w.K, nullptr, 0);
  };
  auto commit = [&](auto set, int s) __attribute__((always_inline)) {
    u32x4_t* const dst = ring + (s & 1) * STAGE;
    sx.template commit<set.value>(tid, dst, s * TK, a.ldx, w.K, xrows, a.Nsrc);
    sy.template commit<set.value>(tid, dst + XU, s * TK, a.ldy, w.K, nullptr, 0);
  };
  constexpr std::integral_constant<int, 0> even;
  constexpr std::integral_constant<int, 1> odd;

  if (w.K > 0) {
    sx.init(tid, w.X, a.ldx, w.m0, w.m_valid, nullptr, 0);
    sy.init(tid, w.Y, a.ldy, w.n0, w.n_valid, YG ? w.rows : nullptr, a.Nsrc);
    sx.fetch(0, w.K, xrows);
    if constexpr (DEPTH > 0) {
      constexpr int COPIES = sx.NU + sy.NU;  // of a thread and stage
      const bool ends_inside = (XKC || YKC) && w.K % CE != 0;
      const int n_st = ends_inside ? w.K / TK : (w.K + TK - 1) / TK;
      auto copy = [&](int s) __attribute__((always_inline)) {
        // past the last stage: zeros, so that every wait counts the same
        u32x4_t* const dst = ring + (s % DEPTH) * STAGE;
        const int K = s < n_st ? w.K : 0;
        sx.copy(tid, dst, s * TK, a.ldx, K, xrows, a.Nsrc);
        // before the other copies, so that waiting for it leaves those in flight
        sx.fetch((s + 1) * TK, w.K, xrows);
        sy.copy(tid, dst + XU, s * TK, a.ldy, K, nullptr, 0);
      };
#pragma unroll
      for (int s = 0; s < DEPTH - 1; ++s) copy(s);
      if constexpr (AHEAD) {
        copy(DEPTH - 1);
        u32x4_t xf[2][NI][2], yf[2][NJ][2];  // of this stage and the next
        asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(COPIES * (DEPTH - 1)) : "memory");
        rx.read(ring, xf[0]);
        ry.read(ring + XU, yf[0]);
        auto step = [&](auto at, int s) __attribute__((always_inline)) {
          // this wave's copies of stage s + 1 have landed (the later ones' may
          // be in flight) and it holds stage s; then every wave
          asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(COPIES * (DEPTH - 2)) : "memory");
          const u32x4_t* const next = ring + (s + 1) % DEPTH * STAGE;
          rx.read(next, xf[1 - at]);
          ry.read(next + XU, yf[1 - at]);
          copy(s + DEPTH);
          multiply(xf[at], yf[at]);
          interleave<T, NI * NJ * 2 * (sizeof(T) == 4 ? 4 : 1)>();
        };
        int s = 0;
        for (; s + 2 <= n_st; s += 2) {
          step(even, s);
          step(odd, s + 1);
        }
        if (s < n_st) step(even, s);
      } else {
        for (int s = 0; s < n_st; ++s) {
          // this wave's copies of stage s have landed (the later ones' may be in
          // flight), then every wave's; every wave is done with stage s - 1
          asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(COPIES * (DEPTH - 2)) : "memory");
          copy(s + DEPTH - 1);
          compute(ring + (s % DEPTH) * STAGE);
        }
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the trailing (empty) copies
      if (ends_inside && n_st * TK < w.K) {
        load(even, n_st);
        __syncthreads();
        sx.commit(tid, ring, n_st * TK, a.ldx, w.K, xrows, a.Nsrc);
        sy.commit(tid, ring + XU, n_st * TK, a.ldy, w.K, nullptr, 0);
        __syncthreads();
        compute(ring);
      }
    } else {
      const int n_st = (w.K + TK - 1) / TK;
      load(even, 0);
      if constexpr (TM < 128) {  // two stages in flight, one in each set of registers
        if (n_st > 1) load(odd, 1);
        commit(even, 0);
        auto step = [&](auto set, auto other, int s) __attribute__((always_inline)) {
          __syncthreads();  // stage s is there; every wave is done with stage s - 1
          if (s + 2 < n_st) load(set, s + 2);
          compute(ring + (s & 1) * STAGE);
          if (s + 1 < n_st) commit(other, s + 1);
        };
        int s = 0;
        for (; s + 2 <= n_st; s += 2) {
          step(even, odd, s);
          step(odd, even, s + 1);
        }
        if (s < n_st) step(even, odd, s);
      } else {
        commit(even, 0);
        for (int s = 0; s < n_st; ++s) {
          __syncthreads();
          if (s + 1 < n_st) load(even, s + 1);
          compute(ring + (s & 1) * STAGE);
          if (s + 1 < n_st) commit(even, s + 1);
        }
      }
    }
  }
  if constexpr (MODE == kDown) {
    if (w.g < a.Ng) store_parts<T, TO>(a, ad, w, lane, acc, xrow, yrow);
    return;
  }
  if constexpr (MODE == kAdapt) low_rank<T, TO, WHOLE>(a, ad, w, lane, acc, xrow, yrow);
  store_tile<T, TO, MODE, MODE == kFwd>(a, w, lane, acc, xrow, yrow);
}

// Tiles that the worst split of Np rows into Ng groups and the rows past them
// needs: each non-empty group may leave one tile partly filled.
inline int64_t row_tiles(int64_t Np, int64_t Ng, bool groups, int TN) {
  if (!groups) return (Np + TN - 1) / TN;
  const int64_t parts = Ng + 1 < Np ? Ng + 1 : Np;
  return Np / TN + parts;
}

template <typename T, typename TO, int MODE, int TM, int TN, int WM, int WN, int DEPTH, bool WHOLE = true>
hipError_t launch_tiles(const GroupArgs& a, const AdaptArgs& ad, int64_t row_tiles, int band,
                        Launch to) {
  auto* const k = group_tiles<T, TO, MODE, TM, TN, WM, WN, DEPTH, WHOLE>;
  const int64_t grid = row_tiles * ((a.M + TM - 1) / TM);
  const hipError_t fit = grid_fits(grid, 64 * WM * WN);
  if (fit != hipSuccess || to.dry) return fit;
  const int lds = (DEPTH > 0 ? DEPTH : 2) * 8 * (TM + TN) * 16;
  if (lds > 64 * 1024) {
    const hipError_t e = allow_max_lds(reinterpret_cast<const void*>(k));
    if (e != hipSuccess) return e;
  }
  k<<<dim3((uint32_t)grid), dim3(64 * WM * WN), lds, to.stream>>>(a, ad, band);
  return hipGetLastError();
}

}  // namespace group
}  // namespace cnnlib
