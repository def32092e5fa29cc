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
#pragma once

#include "common.h"
#include "routed.h"

namespace cnnlib {
namespace group {

enum Mode { kFwd = 0, kBwdIn = 1, kBwdKer = 2, kAdapt = 3 };

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
    const int g = U >= 16 ? (r & 3) | ((r >> 1) & 4) : ((r >> 1) & 1) | ((r >> 2) & 2);
    return r * U + (c ^ (g << 1));
  } else {
    return r * U + (c ^ (((r >> 2) & 3) << 2));
  }
}

// Stages one operand: R tile rows by TK values of k, 8 R units by NT threads.
template <typename T, bool KC, int R, int NT, bool DMA, bool GATHER> struct Stager {
  static constexpr int CE = 16 / (int)sizeof(T);
  static constexpr int TK = 128 / (int)sizeof(T);
  static constexpr int NU = 8 * R / NT;  // units a thread copies per stage
  static constexpr int U = KC ? 8 : R / CE;
  static_assert(8 * R % NT == 0, "whole rounds");

  const T* p[NU];   // the unit's first element at k = 0
  int lim[NU];      // KC: elements of k from the unit's first; MC: elements of the tile index
  int krow[NU];     // MC: row of k within a stage
  u32x4_t reg[DMA ? 1 : NU];

  // base: the tensor at its first k; rows [i0, i0 + n) of the tile index are
  // valid; ld: elements from row to row; K: extent of k (KC).
  // index: for a gathered KC operand, the source row of each tile row.
  __device__ __forceinline__ void init(int tid, const T* base, int64_t ld, int64_t i0, int n, int K,
                                       const int32_t* index, int nsrc) {
#pragma unroll
    for (int j = 0; j < NU; ++j) {
      const int u = j * NT + tid;
      const int r = u / U, pos = u % U;
      const int c = unit_at<T, KC, R>(r, pos) - r * U;  // the permutation is its own inverse
      if constexpr (KC) {
        int64_t row = i0 + r;
        bool ok = r < n;
        if constexpr (GATHER) {
          if (ok && index) {
            row = index[row];
            ok = row >= 0 && row < nsrc;
          }
        }
        p[j] = base + (ok ? row * ld : 0) + c * CE;
        lim[j] = ok ? K - c * CE : 0;
        krow[j] = 0;
      } else {
        p[j] = base + i0 + c * CE;
        lim[j] = n - c * CE;
        krow[j] = r;
      }
    }
  }

  // Source and valid elements of unit j of the stage at k0.  MC: `index` as
  // in init for the rows of k; nk rows of k in all.
  __device__ __forceinline__ const T* at(int j, int k0, int64_t ld, int nk, const int32_t* index,
                                         int nsrc, int* valid) const {
    if constexpr (KC) {
      *valid = lim[j] - k0;
      return p[j] + k0;
    } else {
      const int k = k0 + krow[j];
      int64_t row = k;
      bool ok = k < nk;
      if constexpr (GATHER) {
        if (ok && index) {
          row = index[k];
          ok = row >= 0 && row < nsrc;
        }
      }
      *valid = ok ? lim[j] : 0;
      return p[j] + (ok ? row * ld : 0);
    }
  }

  __device__ __forceinline__ void issue(int tid, u32x4_t* lds, int k0, int64_t ld, int nk,
                                        const int32_t* index, int nsrc) {
#pragma unroll
    for (int j = 0; j < NU; ++j) {
      int valid;
      const T* src = at(j, k0, ld, nk, index, nsrc, &valid);
      if constexpr (DMA) {
        // whole units only: a unit that starts inside a row ends inside it
        const void* from = valid > 0 ? (const void*)src : (const void*)zero_unit;
        copy16_lds(from, lds + j * NT + (__builtin_amdgcn_readfirstlane(tid) & ~63));
      } else {
        reg[j] = load_unit(src, valid);
      }
    }
  }
  __device__ __forceinline__ void commit(int tid, u32x4_t* lds) {
    if constexpr (!DMA) {
#pragma unroll
      for (int j = 0; j < NU; ++j) lds[j * NT + tid] = reg[j];
    }
  }
};

typedef short s16x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ u32x2_t read_tr(const bf16_t* p) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                         LDS_AS(s16x4_t, const_cast<bf16_t*>(p))));
#else
  (void)p;
  return u32x2_t{0u, 0u};
#endif
}

// The operand of 16 tile rows from i0 for the k sub-step ks.  bf16: 32 values
// of k, lane l row l % 16 and k = 8 (l / 16) + 0..7.  fp32: 16 values of k,
// element e of lane l is k = 4 (l / 16) + e, used by the e-th of four MFMAs.
template <typename T, bool KC, int R>
__device__ __forceinline__ u32x4_t read_frag(const u32x4_t* lds, int i0, int ks, int lane) {
  const int l16 = lane & 15, G = lane >> 4;
  if constexpr (KC) {
    return lds[unit_at<T, true, R>(i0 + l16, 4 * ks + G)];
  } else if constexpr (sizeof(T) == 2) {
    // 4 rows of k by 16 columns for each 16 lanes: lane 4v + q reads row v,
    // columns 4q .. 4q+3, and receives column l % 16 of the four rows
    const int k = 32 * ks + 8 * G + (l16 >> 2), q = l16 & 3;
    const bf16_t* base = reinterpret_cast<const bf16_t*>(lds);
    const bf16_t* a = base + 8 * unit_at<T, false, R>(k, (i0 >> 3) + (q >> 1)) + 4 * (q & 1);
    const bf16_t* b = base + 8 * unit_at<T, false, R>(k + 4, (i0 >> 3) + (q >> 1)) + 4 * (q & 1);
    const u32x2_t lo = read_tr(a), hi = read_tr(b);
    return u32x4_t{lo[0], lo[1], hi[0], hi[1]};
  } else {
    const uint32_t* base = reinterpret_cast<const uint32_t*>(lds);
    u32x4_t v;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      v[e] = base[4 * unit_at<T, false, R>(16 * ks + 4 * G + e, (i0 >> 2) + (l16 >> 2)) + (l16 & 3)];
    return v;
  }
}

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

// Four consecutive results from `m` of one row, as many as lie below M.
template <typename TO>
__device__ __forceinline__ void store4(TO* row, int m, int M, f32x4_t v, bool whole) {
  if (whole && m + 4 <= M) {
    if constexpr (sizeof(TO) == 4) {
      *reinterpret_cast<f32x4_t*>(row + m) = v;
    } else {
      *reinterpret_cast<u32x2_t*>(row + m) = u32x2_t{pk_bf16(v[0], v[1]), pk_bf16(v[2], v[3])};
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
};

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
// tiles of m; false: none.  Row tiles are walked in bands: `band` row tiles by
// every m tile, so that the tiles an XCD runs at a time share their rows of X
// and Y in its L2.  Offsets that are not an order (documented as the caller's
// duty) are found out by the wave that adds them up: no tile is then run.
template <int TN>
__device__ __forceinline__ bool find_tile(const int32_t* off, int Ng, int Np, int MT, int bid,
                                          int band, RowTile* t) {
  const int lane = threadIdx.x & 63;
  int nt, j0, lo_g = 0, hi_g = Np;  // row tiles of the group, tile within it, its rows
  t->g = 0;
  if (!off) {
    nt = (Np + TN - 1) / TN;
    if (bid >= nt * MT) return false;
    j0 = xcd_remap(bid, nt * MT);
  } else {
    // up to 63 groups: one pass, else one for the total and one for the tile
    int lo = 0, hi = 0, incl = 0, total = 0;
    for (int base = 0; base <= Ng; base += 64) {
      const int g = base + lane;
      lo = hi = 0;
      if (g <= Ng) group_rows(off, Ng, Np, g, &lo, &hi);
      if (__ballot(lo < 0 || hi < lo || hi > Np || (g == 0 && lo != 0))) return false;
      incl = wave_scan((hi - lo + TN - 1) / TN);
      total += __builtin_amdgcn_readlane(incl, 63);
    }
    if (bid >= total * MT) return false;
    const int L = xcd_remap(bid, total * MT);
    int before = 0;
    for (int base = 0;; base += 64) {
      if (Ng >= 64) {
        const int g = base + lane;
        lo = hi = 0;
        if (g <= Ng) group_rows(off, Ng, Np, g, &lo, &hi);
        incl = wave_scan((hi - lo + TN - 1) / TN);
      }
      const uint64_t here = __ballot(L < (before + incl) * MT);
      if (here) {
        const int who = __ffsll((unsigned long long)here) - 1;
        lo_g = __builtin_amdgcn_readlane(lo, who);
        hi_g = __builtin_amdgcn_readlane(hi, who);
        nt = (hi_g - lo_g + TN - 1) / TN;
        j0 = L - (before + __builtin_amdgcn_readlane(incl, who) - nt) * MT;
        t->g = base + who;
        break;
      }
      before += __builtin_amdgcn_readlane(incl, 63);
    }
  }
  const int b = j0 / (band * MT), rb = min(band, nt - b * band), j = j0 - b * band * MT;
  t->mt = j / rb;
  t->n0 = lo_g + (b * band + j % rb) * TN;
  t->n1 = hi_g;
  return true;
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

// A workgroup's tile: its operands and result from the tile's (and, for the
// gradient of Ker, the group's) start.
template <typename T, typename TO> struct Tile {
  const T* X;
  const T* Y;
  TO* D;
  const int32_t* rows;  // NULL, or the source rows of grouped rows n0 .. or of k = 0 ..
  int K, m0, m_valid, n0, n_valid;
};

template <typename T, typename TO, int MODE, int TM, int TN>
__device__ __forceinline__ bool setup_tile(const GroupArgs& a, int band, Tile<T, TO>* w) {
  const int MT = (a.M + TM - 1) / TM;
  w->X = reinterpret_cast<const T*>(a.X);
  w->Y = reinterpret_cast<const T*>(a.Y);
  w->D = reinterpret_cast<TO*>(a.D);
  w->rows = a.rows;
  int mt;
  if constexpr (MODE == kBwdKer) {
    const int NTL = (a.N + TN - 1) / TN;
    const int L = xcd_remap(blockIdx.x, gridDim.x);
    const int g = L / (MT * NTL);
    const int j0 = L - g * MT * NTL;
    const int b = j0 / (band * MT), rb = min(band, NTL - b * band), j = j0 - b * band * MT;
    mt = j / rb;
    w->n0 = (b * band + j % rb) * TN;
    int lo, hi;
    group_rows(a.off, a.Ng, a.K, g, &lo, &hi);
    // clamped, so that no offset leads outside the tensors
    lo = min(max(__builtin_amdgcn_readfirstlane(lo), 0), a.K);
    w->K = min(max(__builtin_amdgcn_readfirstlane(hi), lo), a.K) - lo;
    w->n_valid = min(a.N - w->n0, TN);
    if (a.rows) w->rows += lo; else w->X += lo * a.ldx;
    w->Y += lo * a.ldy;
    w->D += g * a.dgroup + (int64_t)w->n0 * a.ldd;
  } else {
    RowTile t;
    if (!find_tile<TN>(a.off, a.Ng, a.N, MT, blockIdx.x, band, &t)) return false;
    w->K = t.g < a.Ng ? a.K : 0;  // the rows past the last group: no products
    w->n0 = t.n0;
    w->n_valid = min(t.n1 - t.n0, TN);
    w->X += (t.g < a.Ng ? t.g : 0) * a.xgroup;
    // adapted rows go back to where they came from
    if constexpr (MODE != kAdapt) w->D += (int64_t)t.n0 * a.ldd;
    mt = t.mt;
  }
  w->m0 = mt * TM;
  w->m_valid = min(a.M - w->m0, TM);
  return true;
}

// Results acc[i][j] of 16 values of m from xrow(i) by 16 rows from yrow(j).
// MASK: rows whose source row is not there are stored as zeros.
template <typename T, typename TO, int MODE, bool MASK, int NI, int NJ, typename XR, typename YR>
__device__ __forceinline__ void store_tile(const GroupArgs& a, const Tile<T, TO>& w, int lane,
                                           f32x4_t (&acc)[NI][NJ], XR xrow, YR yrow) {
  const int l16 = lane & 15, m0 = w.m0 + 4 * (lane >> 4);
  // rows whose starts and ends let every four results be stored at once
  const bool whole = ((uintptr_t)a.D & (4 * sizeof(TO) - 1)) == 0 && (a.ldd & 3) == 0 && (a.M & 3) == 0;
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const int n = yrow(j) + l16;
    if (n >= w.n_valid) continue;
    int64_t at = n;
    bool live = true;
    if constexpr (MASK || MODE == kAdapt) {
      if (w.rows) {
        const int r = w.rows[w.n0 + n];
        if constexpr (MODE == kAdapt) at = r;
        live = r >= 0 && r < a.Nsrc;
      }
    }
    TO* const row = w.D + at * a.ldd;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int m = m0 + xrow(i);
      f32x4_t v = acc[i][j];
      if constexpr (MASK)
        if (!live) v = f32x4_t{0.f, 0.f, 0.f, 0.f};
      if (whole) {
        if (m < a.M) store4(row, m, a.M, v, true);
      } else {
        store4(row, m, a.M, v, false);
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
  const u32x4_t zero = {0u, 0u, 0u, 0u};
  const int l16 = lane & 15, G = lane >> 4;
  const T* const H = reinterpret_cast<const T*>(ad.Hp) + (int64_t)w.n0 * ad.hl;
#pragma unroll
  for (int j0 = 0; j0 < NJ; j0 += 2) {
    int id_of[2];  // adapter of this lane's rows; past the tile, the last row's
    uint32_t hrow[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int n = min(yrow(j0 + j) + l16, w.n_valid - 1);
      id_of[j] = ad.ids[w.n0 + n];
      hrow[j] = (uint32_t)(n * ad.hl);
    }
#pragma unroll
    for (int i0 = 0; i0 < NI; i0 += 4) {
      uint32_t brow[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        brow[i] = (uint32_t)(min(xrow(i0 + i) + l16, w.m_valid - 1) * ad.Nl);
      int last = -1;
#pragma unroll 1
      for (;;) {
        int next = 0x7fffffff;  // the least adapter above the last one
#pragma unroll
        for (int j = 0; j < 2; ++j)
          if (id_of[j] > last && id_of[j] < ad.Na) next = min(next, id_of[j]);
        // the four rows of 16 lanes hold the same
        next = __builtin_amdgcn_readfirstlane(row16_min(next));
        if (next == 0x7fffffff) break;
        last = next;
        const T* const B = reinterpret_cast<const T*>(ad.B) + ((int64_t)next * a.M + w.m0) * ad.Nl;
#pragma unroll 1
        for (int k0 = 0; k0 < ad.hl; k0 += BATCH * STEP) {
          u32x4_t xf[BATCH][4], yf[BATCH][2];
          bool in[BATCH];
#pragma unroll
          for (int s = 0; s < BATCH; ++s) {
            in[s] = k0 + s * STEP + CE * G < ad.hl;
            const int kk = in[s] ? k0 + s * STEP + CE * G : 0, rank = kk % ad.nlp;
#pragma unroll
            for (int j = 0; j < 2; ++j) __builtin_memcpy(&yf[s][j], H + hrow[j] + kk, 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
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
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
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

// TM x TN results by WM x WN waves.  DMA: both operands by 16-byte copies to
// LDS (16-byte aligned rows), else through registers.  WHOLE: see low_rank.
template <typename T, typename TO, int MODE, int TM, int TN, int WM, int WN, bool DMA, bool WHOLE>
__global__ __launch_bounds__(64 * WM * WN, 2) void group_tiles(GroupArgs a, AdaptArgs ad, int band) {
  constexpr int NT = 64 * WM * WN;
  constexpr bool XKC = MODE == kFwd || MODE == kAdapt, YKC = MODE != kBwdKer;
  constexpr bool XG = MODE == kBwdKer, YG = MODE == kFwd || MODE == kAdapt;  // gathered operands
  constexpr int TK = 128 / (int)sizeof(T);
  constexpr int KS = 2;  // sub-steps of a stage: 32 (bf16) or 16 (fp32) values of k
  constexpr int NI = TM / WM / 16, NJ = TN / WN / 16;
  constexpr int XU = 8 * TM, YU = 8 * TN;

  extern __shared__ __attribute__((aligned(16))) char smem[];
  u32x4_t* const buf0 = reinterpret_cast<u32x4_t*>(smem);
  u32x4_t* const buf1 = buf0 + XU + YU;

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave % WM, wn = wave / WM;
  auto xrow = [&](int i) { return wm * (TM / WM) + 16 * i; };
  auto yrow = [&](int j) { return wn * (TN / WN) + 16 * j; };

  Tile<T, TO> w;
  if (!setup_tile<T, TO, MODE, TM, TN>(a, band, &w)) return;
  Stager<T, XKC, TM, NT, DMA, XG> sx;
  Stager<T, YKC, TN, NT, DMA, YG> sy;
  sx.init(tid, w.X, a.ldx, w.m0, w.m_valid, w.K, nullptr, 0);
  sy.init(tid, w.Y, a.ldy, w.n0, w.n_valid, w.K, YG ? w.rows : nullptr, a.Nsrc);
  const int32_t* const xrows = XG ? w.rows : nullptr;

  f32x4_t acc[NI][NJ];
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  auto compute = [&](const u32x4_t* buf) __attribute__((always_inline)) {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      u32x4_t xf[NI], yf[NJ];
#pragma unroll
      for (int i = 0; i < NI; ++i) xf[i] = read_frag<T, XKC, TM>(buf, xrow(i), ks, lane);
#pragma unroll
      for (int j = 0; j < NJ; ++j) yf[j] = read_frag<T, YKC, TN>(buf + XU, yrow(j), ks, lane);
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[i][j] = mma<T>(xf[i], yf[j], acc[i][j]);
    }
  };

  const int n_st = (w.K + TK - 1) / TK;
  if (n_st > 0) {
    sx.issue(tid, buf0, 0, a.ldx, w.K, xrows, a.Nsrc);
    sy.issue(tid, buf0 + XU, 0, a.ldy, w.K, nullptr, 0);
    sx.commit(tid, buf0);
    sy.commit(tid, buf0 + XU);
  }
  for (int s = 0; s < n_st; ++s) {
    u32x4_t* const cur = s & 1 ? buf1 : buf0;
    u32x4_t* const nxt = s & 1 ? buf0 : buf1;
    // this stage has landed and every wave is done with the other buffer
    __syncthreads();
    if (s + 1 < n_st) {
      sx.issue(tid, nxt, (s + 1) * TK, a.ldx, w.K, xrows, a.Nsrc);
      sy.issue(tid, nxt + XU, (s + 1) * TK, a.ldy, w.K, nullptr, 0);
    }
    compute(cur);
    if (s + 1 < n_st) {
      sx.commit(tid, nxt);
      sy.commit(tid, nxt + XU);
    }
  }
  if constexpr (MODE == kAdapt) low_rank<T, TO, WHOLE>(a, ad, w, lane, acc, xrow, yrow);
  store_tile<T, TO, MODE, false>(a, w, lane, acc, xrow, yrow);
}

template <typename T, typename TO, int MODE, int TM, int TN, int WM, int WN, bool DMA, bool WHOLE = true>
hipError_t launch_tiles(const GroupArgs& a, const AdaptArgs& ad, int64_t row_tiles, int band,
                        hipStream_t stream) {
  auto* const k = group_tiles<T, TO, MODE, TM, TN, WM, WN, DMA, WHOLE>;
  const int lds = 2 * 8 * (TM + TN) * 16;
  if (lds > 64 * 1024) {
    const hipError_t e = allow_max_lds(reinterpret_cast<const void*>(k));
    if (e != hipSuccess) return e;
  }
  const int64_t grid = row_tiles * ((a.M + TM - 1) / TM);
  k<<<dim3((uint32_t)grid), dim3(64 * WM * WN), lds, stream>>>(a, ad, band);
  return hipGetLastError();
}

}  // namespace group
}  // namespace cnnlib
