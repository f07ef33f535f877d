// Attention over key ranges: what its kernels share.
//
// Query i of a sample sees the keys [lo_i, hi_i).  The query heads of a group share a key head, so the rows that a kernel tiles are
// packed: row r of (sample, key head) is token r / G and head r % G of the group (G = heads / kv_heads), and a unit is the rows of
// tpt = TR / G whole tokens (TR = 128 rows on the tensor cores, 64 on the CUDA cores; less than TR rows where G does not divide it).
//
// The plan (device memory of the caller, made once per set of ranges):
//   rows   int2 [Bm][Sq]   the ranges clamped into [0, Sk); (0, 0) where nothing is left
//   units  int4 [Bm][nU]   of a unit's rows that see something: smallest lo, largest hi; of all its rows: largest lo, smallest hi
//   keys   int4 [Bm][nK]   of a tile of TR keys: first and one past the last unit that reaches into it; first and one past the last
//                          key (relative to the tile) that any unit's hull holds
//   runs   int4 [Bm][nK]   how many units reach into it; a run [first, last) of units of which every row sees the whole tile
//   order  int  [Bm][nI]   the forward's items (two units on the tensor cores, else one), those with the most keys first
// and where there are so few items that their key ranges are cut into pieces (smax > 1):
//   head   int  [2]        pieces of all items of all masks; tiles of keys in a piece
//   pieces int  [Bm][nI]   pieces of an item
//   work   int4 [...]      of a piece: mask, item, first tile, its number within the item
#pragma once

#include <algorithm>

#include <cuda.h>

#include "common.cuh"

namespace vmoba {
namespace range {

struct RDims {
  int B, Hq, Hk, G, d, Sq, Sk, Bm, dtype, es;
  float scale, cap;
  bool tc;            // tensor-core path
  int TR;             // rows of a unit at most, and keys of a tile
  int tpt;            // tokens of a unit
  int rows;           // rows of a (sample, key head): Sq * G
  int nU, nK, nI;     // units, key tiles, forward items per (sample, key head)
  int smax;           // pieces that an item's key range is cut into at most (1: none is)
  int reps;           // (sample, key head) pairs that share a mask's pieces
};

struct Plan {
  int2* rows;
  int4* units;
  int4* keys;
  int4* runs;
  int* order;
  int* head;
  int* pieces;
  int4* work;
};

struct Strides { long long b, t, h; };       // elements

__device__ __forceinline__ int mask_batch(const int Bm, int b) { return Bm > 1 ? b : 0; }

// Whether a unit with this record reaches into key tile t of TR keys.
__device__ __forceinline__ bool reaches(const int4& u, int t, int TR) { return u.y > u.x && u.x < (t + 1) * TR && u.y > t * TR; }

// Capped scores in the exp2 domain: c' tanh(a s), c' = cap * log2 e, a = scale / cap.
struct Cap {
  float c, twice_log2;           // c'; 2 log2 e times the factor that pre does not take
  float pre;                     // scores are multiplied by this first: 1 with a folded into all that follows, or a
  float most;                    // |score| up to this: by the polynomial
  float p[5], u[5];              // its coefficients of s, s^3, ...; of tanh alone
  float shift;                   // what stands for the rows' maximum where none is looked for (forward); else 0
};
constexpr float CAP_MOST = 96.0f;    // c' up to this: weights need no maximum
Cap make_cap(const RDims& D);      // attn_range_fwd.cu

// ---- tensor-core kernels (attn_range_fwd.cu, attn_range_bwd.cu)
struct FwdArgs {
  const void *q, *k, *v;
  void *o, *resid;           // resid: contiguous [B, Sq, Hq, d] or null
  float* lse;                // [B, Hq, Sq]
  Strides qs, ks, vs, os;
  float *part_o, *part_lse;  // [piece][B * Hk * rows][d], [piece][B * Hk * rows]
  int32_t* status;
};
struct BwdArgs {
  const void *q, *k, *v, *d_o;
  const float *lse, *Dv;     // Dv: [B * Hk * rows]
  Strides qs, ks, vs, dos, dks, dvs;
  void *dk, *dv;
  float* dq_acc;             // [parts][B * Hk * rows][d]
  int parts;
  int* turns;
  int32_t* status;
};

bool make_tmap_keys(CUtensorMap* map, const void* base, const RDims& D, const Strides& s);       // attn_range_fwd.cu
bool make_tmap_units(CUtensorMap* map, const void* base, const RDims& D, const Strides& s);
int tc_range_fwd(const RDims& D, const Plan& plan, const FwdArgs& a, cudaStream_t st);
int tc_range_bwd(const RDims& D, const Plan& plan, const BwdArgs& a, void* dq, const Strides& dqs, bool early, cudaStream_t st);
int tc_range_bwd_parts(const RDims& D);              // accumulators of dq
long long tc_range_bwd_turns(const RDims& D);        // words of `turns`, zero ahead of the kernel

}  // namespace range
}  // namespace vmoba
