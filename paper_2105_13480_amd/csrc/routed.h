// Internal declarations of the routed contractions (the cnn_route_*,
// cnn_combine_*, cnn_group_* and cnn_adapt_* entry points of include/cnn.h):
// the arguments of their kernels and the launches the entry points make.
#pragma once

#include "internal.h"

namespace cnnlib {

// A product over the groups of a routed tensor, or (off NULL) over one group.
// D[n][m] = sum_k X[m, k] Y[n, k] in the kernels' own terms: m the result's
// last index, n its row, k what is summed over.
struct GroupArgs {
  const void* X;
  const void* Y;
  void* D;
  const int32_t* off;   // Ng + 1 group starts, NULL: one group of all Np rows
  const int32_t* rows;  // row of In of each grouped row, NULL: the row itself
  int64_t ldx, ldy, ldd;  // elements from row to row
  int64_t xgroup, dgroup; // elements from group to group (0: none)
  int32_t M, N, K;      // extents of m, n and k; N (products over rows) or K (the
                        // gradient of Ker) is the number of grouped rows Np
  int32_t Ng;
  int32_t Nsrc;         // rows of the gathered tensor: rows outside [0, Nsrc) are zeros
};

// The low-rank part beside a product:
// D[n][m] += scales[a] sum_r H[n][r] B[a][m][r], H = In A[a]^T, a = ids[n].
struct AdaptArgs {
  const void* A;         // [Na][Nl][Nc]
  const void* B;         // [Na][Nk][Nl]
  const int32_t* ids;    // adapter of each row, in the order of H; outside [0, Na): none
  const float* scales;   // [Na] or NULL
  int32_t Na, Nl;
  // Many rows, in the order of their adapters: scaled H as operand rows of
  // `hl` elements, in bf16 the three bf16 parts of the fp32 values, `nlp` ranks
  // each (Nl up to a unit, zeros past it).
  void* Hp;
  int32_t nlp, hl;
  // Few rows, as they come: partial sums over slices of k.
  float* H;              // [kh][Nt][Nl]
  float* part;           // [ks][Nt][Nk]
};

// How an adapted product of few rows is split.
struct FewPlan {
  int32_t blocks, rtiles;  // of features and of rows
  int32_t ks, kh;  // slices of k of the projection and of H
  int32_t kslice, hslice, q, downs;  // set by the launch: their lengths, and H's workgroups
};

// Ranks of one part of an operand row of H, and the row's elements.
inline int adapt_nlp(int64_t Nl, int dtype) {
  return (int)(dtype == CNN_F32 ? (Nl + 3) & ~(int64_t)3 : (Nl + 7) & ~(int64_t)7);
}
inline int adapt_parts(int dtype) { return dtype == CNN_F32 ? 1 : 3; }

// The rows of a problem in the order of a key (experts of (row, choice) pairs,
// adapters of rows): a counting sort by workgroups of `chunk` rows.
struct OrderArgs {
  const int32_t* key;   // [Nt][Kt]; outside [0, Ng): none
  int32_t* off;         // [Ng + 1]
  int32_t* rows;        // [Nt Kt]: row of each place; -1 past off[Ng], or the rows without a key
  int32_t* slots;       // [Nt][Kt]: place of each pair, -1: none; may be NULL
  int32_t* keys;        // [Nt Kt]: key of each place (-1: none); may be NULL
  int32_t* counts;      // [nblocks][Ng + 1]
  int32_t Nt, Ng, Kt;
  int32_t chunk, nblocks;
  int32_t place_none;   // rows without a key get the places past off[Ng]
};

struct RouteArgs {
  const void* logits;
  float* gates;
  int32_t* choice;
  int32_t over_all;     // weights over all allowed experts, not the chosen ones
};

// A Ker in 4 bits beside GroupArgs, whose X then points to its codes: rows of Nb
// blocks of 16 bytes, and a scale byte each.
struct Group4Args {
  const uint8_t* xs;  // scales of X's blocks
  const uint8_t* ys;  // of Y's, if it is in 4 bits too; else NULL
  int32_t Nb;
};

// The router's balance.
struct BalanceArgs {
  const void* logits;     // [Nt][Ng]
  const int32_t* choice;  // [Nt][Kt]
  const int32_t* bounds;  // [Ns + 1], NULL: one sequence of all rows
  int32_t* counts;        // [Ns][Ng]
  int32_t* tokens;        // [Ns]
  float* loss;            // [2]
  const float* dloss;     // [2]
  void* dlogits;          // [Nt][Ng]
  void* ws;
  int32_t Nt, Ng, Kt, Ns;
  int32_t chunk, nblocks; // rows of a workgroup, workgroups
};
// Rows of one sequence that a single workgroup takes.
constexpr int64_t kBalanceOne = 256;

// Where a launch goes; `dry`: it is only seen whether its grid fits.
struct Launch {
  hipStream_t stream;
  bool dry;
};

// Rows of an ordering workgroup and the number of workgroups.
void order_blocks(int64_t Nt, int32_t* chunk, int32_t* nblocks);

hipError_t launch_route(const RouteArgs& a, const OrderArgs& o, bool bf16, hipStream_t stream);
hipError_t launch_order(const OrderArgs& o, hipStream_t stream);
hipError_t launch_route_bwd(const void* logits, const int32_t* choice, const float* gates,
                            const float* dgates, void* dlogits, int64_t Nt, int Ng, int Kt,
                            int dtype, int over_all, hipStream_t stream);
hipError_t launch_combine(const void* In, const int32_t* slots, const float* gates, void* Out,
                          int64_t Nt, int Kt, int64_t Np, int64_t Nk, int dtype,
                          hipStream_t stream);
hipError_t launch_combine_bwd(const void* dOut, const void* In, const int32_t* slots,
                              const int32_t* rows, const float* gates, void* dIn, float* dGates,
                              int64_t Nt, int Kt, int64_t Np, int64_t Nk, int dtype,
                              hipStream_t stream);
hipError_t launch_group_fwd(const GroupArgs& a, int dtype, hipStream_t stream);
hipError_t launch_group_bwd_in(const GroupArgs& a, int dtype, hipStream_t stream);
hipError_t launch_group_bwd_ker(const GroupArgs& a, int dtype, hipStream_t stream);
// Products of few rows a group, straight from memory.
bool group_few_fits(const GroupArgs& a, int dtype);
hipError_t launch_group_few(const GroupArgs& a, int dtype, hipStream_t stream);
// Whether an adapted product of Nt rows runs the few-rows kernels, which take
// the rows as they come.
constexpr int64_t kFewRows = 512;  // at most
bool adapt_few(int64_t Nt, int64_t Nc, int64_t Nk, bool ring);
bool adapt_few_ring(const void* Ker, const void* In, int64_t Nc, int es);  // rows on 4-byte boundaries
FewPlan adapt_few_plan(int64_t Nt, int64_t Nc, int64_t Nk, int es);
hipError_t launch_adapt_few(const GroupArgs& a, const AdaptArgs& ad, int dtype, hipStream_t stream);
// Rows in the order of their adapters (a.off, a.rows, ad.ids).
hipError_t launch_adapt(const GroupArgs& a, const AdaptArgs& ad, int dtype, Launch to);

int64_t balance_ws_bytes(int64_t Nt, int64_t Ng, int64_t Ns);
hipError_t launch_balance(const BalanceArgs& a, bool bf16, hipStream_t stream);
hipError_t launch_balance_bwd(const BalanceArgs& a, int dtype, bool add, hipStream_t stream);
hipError_t launch_quantize4(const void* In, uint8_t* Codes, uint8_t* Scales, int64_t Nt, int64_t Nc,
                            bool bf16, bool up, hipStream_t stream);
hipError_t launch_dequantize4(const uint8_t* Codes, const uint8_t* Scales, void* Out, int64_t Nt,
                              int64_t Nc, bool bf16, hipStream_t stream);
hipError_t launch_group_fwd4(const GroupArgs& a, const Group4Args& b, bool bf16_out, hipStream_t stream);
hipError_t launch_group_bwd_in4(const GroupArgs& a, const Group4Args& b, bool bf16_out, hipStream_t stream);

// bf16 rows, few a group, Ker in 4 bits straight from memory: 16 rows and features a
// workgroup (8 blocks a row at least), or 64 features by 16 or 32 rows, or 128 by 64
// (16 blocks; rows on 4-byte boundaries, of whole units, less than 2^31 bytes of them).
hipError_t launch_group4_few(const GroupArgs& a, const Group4Args& b, bool bf16_out, hipStream_t stream);
hipError_t launch_group4_rows(const GroupArgs& a, const Group4Args& b, bool bf16_out, int rows, hipStream_t stream);

}  // namespace cnnlib
