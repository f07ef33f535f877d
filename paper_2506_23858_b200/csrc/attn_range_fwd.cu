// Tensor-core forward of attention over key ranges (bf16, head_dim 128).
//
// The wide forward of attn_tc_fwd.cu (two 128-row query tiles A and B that share every tile of K and V, one score buffer that they
// use in turn, softmax threads that hold a whole row of 128 scores) with the items of a plan: an item is two units of packed rows against
// the hull of their key ranges (or a piece of it, where there are few items), in tiles of 128 keys from the hull's first key on.  A unit
// takes part in the tiles that its own hull reaches; a score is compared with its row's range only in tiles where the unit's
// bounds say that some row needs it.
//
// Bound by the exponentials of two tiles and the one score buffer, as the dense forward is; the weights are rounded to bf16 (2^-8) for P V, and o
// is normalised by the sum of the rounded ones.  12 heads: 32,760 tokens by frames 2.85 ms (1210 TFLOP/s of the visible pairs), capped 3.5, and
// 4.1 in call after call on other inputs (power-capped); 13,440 tokens, eight clips packed, 257 us (985); a frame of 1,560 tokens against 31,200
// keys 315 us where the same call is repeated, 357 on other inputs each time, its pieces joined through memory; a token of each of four
// samples against 8K to 76K keys, four key heads, 362 MB, 76 us (4.8 TB/s).
//
// Every (item, unit) has at least one tile, masked as a whole if need be, and every tile at least one unit, so that no barrier skips a phase.
//
//   warp 0        TMA: K tiles into a ring of two stages, V tiles into one of three
//   warps 1, 2    MMA issuers: Q K^T; P V
//   warp 3        clears what the V tile of an item's last keys holds behind them: a weight of 0 times a value that is not finite
//                 would not be 0 (by the warp that issues P V, the clearing's code alone cost 8 % on tiles that need none)
//   warps 4-11    softmax of unit A, of unit B: thread = row
//   warps 12-15   Q tiles of the next item, o of the one before
//
// Capped scores: c tanh(x), x = scale s / c.  By the exponential unit that is an exponential and a reciprocal more per score, and the
// kernel is bound by that unit: a 33K clip by frames took 7.5 ms, 3.7 without the cap.  So tanh comes from the FMA pipe where a warp's
// scores allow (|x| <= 3/4): an odd polynomial of five terms, fitted to tanh for the smallest largest relative error (by reweighted least
// squares; 5.7e-7); larger scores take 1 - 2 / (1 + exp(2 x)).  So the time goes by the scores: the 33K clip, scores of a standard deviation of a tenth of
// the cap 3.5 ms, of half the cap and of the whole 6.8, where nearly every warp has one that is larger.
// And a cap bounds the weights: up to c' = c log2 e = 96 (caps of 66) exp2 of a score is a normal number, of no difference to the row's maximum but to one
// number for all rows: 0, or c' - 80 where that is more.  Weights of up to 2^80 leave room for sums of 2^17 of them times values of up to 2^29; they are
// 2^-112 at least.  So no maximum is looked for and nothing is rescaled.
#include <algorithm>

#include "attn_range.cuh"
#include "sm100.cuh"

namespace vmoba {
namespace range {
namespace tcf {

using namespace sm100;

constexpr int BM = 128, BN = 128, DH = 128;
constexpr int KST = 2, VST = 3;
constexpr int PANEL = BM * 128;      // bytes of one 64-column panel of a 128-row tile (16 KB)
constexpr int TILE = 2 * PANEL;      // bytes of a [128 x 128] bf16 tile (32 KB)
constexpr int THREADS = 512;         // warp groups {TMA, MMA, MMA, -}, A, B, loaders; registers 56, 200, 200, 56 (= 4 x 128)
constexpr uint32_t TMEM_COLS = 512;
constexpr uint32_t P_COL = 128, O_COL = 256;      // S at 0, P_X at 128 + 64 X, O_X at 256 + 128 X
constexpr float RESCALE_LOG2 = 8.0f;
constexpr float LOG2E = 1.4426950408889634f;

struct Smem {
  uint64_t k_full[KST], k_empty[KST], v_full[VST], v_empty[VST];
  uint64_t v_tail[VST];              // the V tile of an item's last keys has landed (warp 3 clears its rest and completes v_full)
  uint64_t s_full[2], p_ready[2];    // per unit: scores written (commit) / P written (128 arrivals)
  uint64_t s_free;                   // the score buffer has been read (128 arrivals of whichever unit used it)
  uint64_t o_done[2];                // per unit: P V of a key tile complete (commit)
  uint64_t ep_ready[2];              // per unit: an item's normalisers are in ep_inv / ep_lse (128 softmax arrivals)
  uint64_t o_free[2];                // per unit: epilogue has read them and the accumulator (128 arrivals)
  uint64_t q_full, q_empty;          // Q tiles of an item landed / no longer needed (commit)
  uint64_t drain[2];                 // (after a time-out only)
  uint32_t tmem_base;
  int abort_flag;
  float ep_inv[2][BM], ep_lse[2][BM];   // 1 / sum of the rounded weights (0: the row saw nothing), natural-log lse
};
constexpr size_t SMEM_BYTES = (2 /*Q*/ + KST + VST) * TILE + sizeof(Smem) + 32;
static_assert(SMEM_BYTES <= 232448, "range forward: shared memory");

struct Params {
  int B, Hk, G, Sq, Sk, Bm, tpt, nU, nI, cut, reps, n_items;
  int group;             // key heads (of all samples) whose items are taken together
  FastDiv by_reps, by_set, by_group, by_Hk, by_G;      // by_set: items of a group
  const int2* rows;
  const int4* units;
  const int* order;
  const int* head;
  const int4* work;
  float scale_log2;      // scores -> exp2 domain: scale * log2 e; 1 where they are capped first
  Cap cap;
  __nv_bfloat16 *o, *resid;
  Strides os;
  float* lse;
  float *part_o, *part_lse;
  int32_t* status;
};

struct Item {
  int b, hk, u0, nx, piece;
  int k_begin, keys;               // first key of the item's tiles, keys in them (0: all masked)
  int ntiles;
  int tb[2], te[2];                // per unit: its tiles
  int full_lo[2], full_hi[2];      // per unit: every row sees the keys between these
};

__device__ __forceinline__ Item decode_item(const Params& p, int item) {
  Item it;
  int bm, first = 0, len = INT32_MAX;
  it.piece = 0;
  if (p.cut) {
    const int entry = p.by_reps.div(item), rep = item - entry * p.reps;
    const int4 w = __ldg(p.work + entry);
    bm = w.x;
    it.b = p.Bm > 1 ? w.x : p.by_Hk.div(rep);
    it.hk = p.Bm > 1 ? rep : rep - it.b * p.Hk;
    it.u0 = 2 * w.y;
    first = w.z;
    len = __ldg(p.head + 1);
    it.piece = w.w;
  } else {
    const int set = p.by_set.div(item), r = item - set * p.group * p.nI, rank = p.by_group.div(r), bhk = set * p.group + (r - rank * p.group);
    it.b = p.by_Hk.div(bhk);
    it.hk = bhk - it.b * p.Hk;
    bm = mask_batch(p.Bm, it.b);
    it.u0 = 2 * __ldg(p.order + (long long)bm * p.nI + rank);
  }
  it.nx = it.u0 + 1 < p.nU ? 2 : 1;
  const int4* units = p.units + (long long)bm * p.nU + it.u0;
  const int4 a = __ldg(units), c = it.nx == 2 ? __ldg(units + 1) : make_int4(0, 0, 0, 0);
  int lo = a.x, hi = a.y;
  if (c.y > c.x) {
    lo = hi > lo ? min(lo, c.x) : c.x;
    hi = max(hi, c.y);
  }
  const int all = (max(hi - lo, 0) + BN - 1) / BN, tiles = max(min(len, all - first), 0);
  it.k_begin = lo + first * BN;
  it.keys = max(min(tiles * BN, hi - it.k_begin), 0);
  if (it.keys == 0) it.k_begin = 0;
  it.ntiles = max(tiles, 1);
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int4 u = x ? c : a;
    const int from = u.x - it.k_begin, to = min(u.y - it.k_begin, it.keys);
    it.tb[x] = max(from, 0) / BN;
    it.te[x] = (max(to, 0) + BN - 1) / BN;
    if (it.tb[x] >= it.te[x]) { it.tb[x] = 0; it.te[x] = 1; }
    it.full_lo[x] = u.z;
    it.full_hi[x] = u.w;
  }
  if (it.nx == 2) {                // no tile without a unit
    if (it.tb[0] > 0 && it.tb[1] > 0) { if (it.tb[0] <= it.tb[1]) it.tb[0] = 0; else it.tb[1] = 0; }
    if (it.te[0] < it.ntiles && it.te[1] < it.ntiles) { if (it.te[0] >= it.te[1]) it.te[0] = it.ntiles; else it.te[1] = it.ntiles; }
    if (it.te[0] < it.tb[1]) it.te[0] = it.tb[1];
    if (it.te[1] < it.tb[0]) it.te[1] = it.tb[0];
  } else {
    it.tb[0] = 0;
    it.te[0] = it.ntiles;
  }
  return it;
}
// A CTA's items, round after round: the items of a group of heads follow one another from the longest to the shortest, and the CTAs take
// them from the left and from the right in turn, so that who has the longest of one round has the shortest of the next.  (From the
// left only, the busiest CTA of 13K packed clips had 25 % more than the mean, of causal clips 27 to 56 %; so it is 1 to 7 %.)
__device__ __forceinline__ int item_at(int round) {
  return round * (int)gridDim.x + ((round & 1) ? (int)gridDim.x - 1 - (int)blockIdx.x : (int)blockIdx.x);
}
// decode_item(), known to be the same on all lanes of a warp (values from memory pass through a warp reduction).
__device__ __forceinline__ Item uniform_item(const Params& p, int item) {
  Item it = decode_item(p, item);
  auto u = [](int v) { return __reduce_max_sync(0xffffffffu, v); };
  it.nx = u(it.nx);
  it.keys = u(it.keys);
  it.ntiles = u(it.ntiles);
#pragma unroll
  for (int x = 0; x < 2; ++x) { it.tb[x] = u(it.tb[x]); it.te[x] = u(it.te[x]); }
  return it;
}
// Keys of tile t that the matrix products take: whole steps of 16, one at least.
__device__ __forceinline__ int key_steps(const Item& it, int t) { return (max(min(BN, it.keys - t * BN), 1) + 15) >> 4; }

// Whether the item's last tile ends inside a step of 16 keys.
__device__ __forceinline__ bool has_tail(const Item& it) { return it.keys == 0 || (it.keys & 15) != 0; }

__device__ __forceinline__ constexpr uint32_t koff(int ks) { return (uint32_t)(((ks >> 2) * PANEL + (ks & 3) * 32) >> 4); }
__device__ __forceinline__ constexpr uint32_t mnoff(int ks) { return (uint32_t)((ks * 2048) >> 4); }

__device__ __forceinline__ float rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// c' tanh(a s), less the shift, of 32 of a row's scores, in place.  Called by whole warps (which way is taken is the warp's choice).
__device__ __forceinline__ void cap_pair(float& x0, float& x1, const Cap& cap) {
  float z0, z1, r0 = cap.p[4], r1 = cap.p[4];
  mul2(z0, z1, x0, x1, x0, x1);
#pragma unroll
  for (int k = 3; k >= 0; --k) fma2(r0, r1, r0, r1, z0, z1, cap.p[k], cap.p[k]);
  fma2(x0, x1, r0, r1, x0, x1, -cap.shift, -cap.shift);
}
template <int N>
__device__ __forceinline__ bool polynomial_does(const uint32_t* sv, const Cap& cap) {
  float m0 = 0.f, m1 = 0.f;
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    m0 = max3(m0, fabsf(__uint_as_float(sv[i])), fabsf(__uint_as_float(sv[i + 1])));
    m1 = max3(m1, fabsf(__uint_as_float(sv[i + 2])), fabsf(__uint_as_float(sv[i + 3])));
  }
  return __all_sync(0xffffffffu, fmaxf(m0, m1) <= cap.most);
}
// APART: caps that may be large.  1 - 2 / (1 + exp(2 x)) is off by 1.6e-7 of the cap, and the scores of a warp's other rows need not be of its size:
// those that the polynomial does keep it.
template <bool APART>
__device__ __forceinline__ void cap32(uint32_t* sv, const Cap& cap) {
  if (polynomial_does<32>(sv, cap)) {
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
      float x0 = __uint_as_float(sv[i]), x1 = __uint_as_float(sv[i + 1]);
      cap_pair(x0, x1, cap);
      sv[i] = __float_as_uint(x0);
      sv[i + 1] = __float_as_uint(x1);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const float x = __uint_as_float(sv[i]), far = fmaf(-2.0f * cap.c, rcp(1.0f + ex2(x * cap.twice_log2)), cap.c - cap.shift);
      if (APART && fabsf(x) <= cap.most) {
        const float z = x * x;
        float r = cap.p[4];
#pragma unroll
        for (int k = 3; k >= 0; --k) r = fmaf(r, z, cap.p[k]);
        sv[i] = __float_as_uint(fmaf(r, x, -cap.shift));
      } else {
        sv[i] = __float_as_uint(far);
      }
    }
  }
}
// 32 scores from key i0 on of a row that sees n keys from key a on: those outside get a value.
__device__ __forceinline__ void mask32(uint32_t* sv, int i0, int a, int n, uint32_t value) {
  const int lo = min(max(a - i0, 0), 32), hi = min(max(a + n - i0, 0), 32);
  const uint32_t w = (hi ? 0xffffffffu >> (32 - hi) : 0u) & (lo < 32 ? 0xffffffffu << lo : 0u);
#pragma unroll
  for (int i = 0; i < 32; ++i)
    if (!(w >> i & 1)) sv[i] = value;
}
constexpr uint32_t MINUS_INF = 0xff800000u;

// p = 2^(s * scale - m) for 32 scores; bf16 pairs (keys 2i, 2i+1 -> word i).  s0/s1 collect the exact weights, r0/r1 the rounded ones (the
// tensor core multiplies the ROUNDED weights: o is normalised by their sum, so that the rounding perturbs the weights but never
// their total).
__device__ __forceinline__ void exp_pack32(const uint32_t* sv, float scale, float neg_m, uint32_t (&pk)[16], float& s0, float& s1, float& r0,
                                           float& r1) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    float p0, p1;
    fma2(p0, p1, __uint_as_float(sv[2 * i]), __uint_as_float(sv[2 * i + 1]), scale, scale, neg_m, neg_m);
    p0 = ex2(p0);
    p1 = ex2(p1);
    add2(s0, s1, s0, s1, p0, p1);
    pk[i] = pack_bf16(p0, p1);
    add_bf16_pair(r0, r1, pk[i]);
  }
}

// The same of capped scores, by the polynomial (FAST), or of scores that have been capped already.
template <bool FAST>
__device__ __forceinline__ void exp_capped32(const uint32_t* sv, const Cap& cap, uint32_t (&pk)[16], float& s0, float& s1, float& r0, float& r1) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    float p0 = __uint_as_float(sv[2 * i]), p1 = __uint_as_float(sv[2 * i + 1]);
    if (FAST) cap_pair(p0, p1, cap);
    p0 = ex2(p0);
    p1 = ex2(p1);
    add2(s0, s1, s0, s1, p0, p1);
    pk[i] = pack_bf16(p0, p1);
    add_bf16_pair(r0, r1, pk[i]);
  }
}

__device__ __forceinline__ void store8_resid(__nv_bfloat16* dst, __nv_bfloat16* rdst, const float (&v)[8]) {
  uint32_t h[4], r[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    h[k] = pack_bf16(v[2 * k], v[2 * k + 1]);
    r[k] = pack_bf16(v[2 * k] - __uint_as_float(h[k] << 16), v[2 * k + 1] - __uint_as_float(h[k] & 0xffff0000u));
  }
  *reinterpret_cast<uint4*>(dst) = make_uint4(h[0], h[1], h[2], h[3]);
  if (rdst) *reinterpret_cast<uint4*>(rdst) = make_uint4(r[0], r[1], r[2], r[3]);
}

// What a kernel does with the scores: nothing, caps them and goes by the cap's bound, caps them and looks for the maximum as without.
enum Mode { kPlain, kCapped, kCappedWide };

template <Mode MODE>
__global__ void __launch_bounds__(THREADS, 1)
attn_range_fwd_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                      const __grid_constant__ CUtensorMap tmQ, const Params p) {
  if (!grid_begin()) return;
  extern __shared__ uint8_t smem_raw[];
  // the swizzled tiles need 1024-byte alignment and there is no room for alignment slack
  if ((smem_u32(smem_raw) & 1023u) != 0) {
    if (threadIdx.x == 0) set_status(p.status, VMOBA_ERR_CUDA);
    return;
  }
  uint8_t* sQ = smem_raw;                  // [2 units][TILE]
  uint8_t* sK = sQ + 2 * TILE;             // [KST][TILE]
  uint8_t* sV = sK + KST * TILE;           // [VST][TILE]
  Smem* sm = reinterpret_cast<Smem*>(sV + VST * TILE);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  volatile int* abort_flag = &sm->abort_flag;

  if (threadIdx.x == 0) {
    for (int s = 0; s < KST; ++s) { mbar_init(&sm->k_full[s], 1); mbar_init(&sm->k_empty[s], 1); }
    for (int s = 0; s < VST; ++s) { mbar_init(&sm->v_full[s], 1); mbar_init(&sm->v_empty[s], 1); mbar_init(&sm->v_tail[s], 1); }
    for (int x = 0; x < 2; ++x) {
      mbar_init(&sm->s_full[x], 1); mbar_init(&sm->p_ready[x], 128);
      mbar_init(&sm->o_done[x], 1); mbar_init(&sm->o_free[x], 128); mbar_init(&sm->ep_ready[x], 128);
    }
    mbar_init(&sm->s_free, 128);
    mbar_init(&sm->q_full, 1); mbar_init(&sm->q_empty, 1);
    mbar_init(&sm->drain[0], 1); mbar_init(&sm->drain[1], 1);
    sm->abort_flag = 0;
    fence_barrier_init();
    prefetch_tmap(&tmK);
    prefetch_tmap(&tmV);
    prefetch_tmap(&tmQ);
  }
  // rows that a unit leaves over (the group's size does not divide 128): no copy writes them, and their scores have a say in the softmax
  // warps' votes
  for (int i = threadIdx.x; i < 2 * (BM - p.tpt * p.G) * 16; i += THREADS) {
    const int r = p.tpt * p.G + (i >> 5), at = i & 31;
    *reinterpret_cast<uint4*>(sQ + (at >> 4) * TILE + (at >> 3 & 1) * PANEL + r * 128 + (at & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
  }
  fence_async_proxy();
  if (warp == 1) {
    tmem_alloc(&sm->tmem_base, TMEM_COLS);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm->tmem_base;
  const int n_items = p.cut ? __ldg(p.head) * p.reps : p.n_items;
  constexpr uint32_t IDESC_PV = make_idesc_bf16(BM, DH, false, true);

  if (warp < 4) asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
  if (warp == 0) {
    // ------------------------------------------------------------------ TMA producer
    if (lane == 0) {
      uint32_t ks = 0, kp = 1, vs = 0, vp = 1;       // ring slots and the parities of their `empty` waits (the first pass at once)
      for (int round = 0, item; (item = item_at(round)) < n_items; ++round) {
        const Item it = decode_item(p, item);
        for (int t = 0; t < it.ntiles; ++t) {
          const int y = it.k_begin + t * BN;
          mbar_wait(&sm->k_empty[ks], kp, abort_flag, p.status);
          mbar_expect_tx(&sm->k_full[ks], TILE);
          tma_load_4d(sK + ks * TILE, &tmK, &sm->k_full[ks], 0, y, it.hk, it.b);
          tma_load_4d(sK + ks * TILE + PANEL, &tmK, &sm->k_full[ks], 64, y, it.hk, it.b);
          mbar_wait(&sm->v_empty[vs], vp, abort_flag, p.status);
          uint64_t* full = t == it.ntiles - 1 && has_tail(it) ? &sm->v_tail[vs] : &sm->v_full[vs];
          mbar_expect_tx(full, TILE);
          tma_load_4d(sV + vs * TILE, &tmV, full, 0, y, it.hk, it.b);
          tma_load_4d(sV + vs * TILE + PANEL, &tmV, full, 64, y, it.hk, it.b);
          // drain: every issued load must have landed before the CTA may exit (only matters after a timeout)
          if (*abort_flag) {
            mbar_wait(&sm->k_full[ks], kp ^ 1, abort_flag, p.status);
            mbar_wait(full, vp ^ 1, abort_flag, p.status);      // (of v_tail whatever phase: then v_full does not complete without it)
            mbar_wait(&sm->v_full[vs], vp ^ 1, abort_flag, p.status);
          }
          if (++ks == KST) { ks = 0; kp ^= 1; }
          if (++vs == VST) { vs = 0; vp ^= 1; }
        }
      }
    }
  } else if (warp <= 2) {
    // ------------------------------------------------------------------ MMA issuers: the whole warp walks the loop, one elected lane
    // issues (warp-uniform control flow; see elect_one); the lanes look at an operation's barriers at once.
    const bool leader = elect_one();
    const int n_items_u = __reduce_max_sync(0xffffffffu, n_items);
    auto wait3 = [&](uint64_t* b0, uint32_t p0, uint64_t* b1, uint32_t p1, bool third, uint64_t* b2, uint32_t p2) {
      const int which = lane & 3;
      uint32_t bar = smem_u32(b0), par = p0;
      if (which == 1) { bar = smem_u32(b1); par = p1; }
      if (which == 2 && third) { bar = smem_u32(b2); par = p2; }
      mbar_wait_lanes(bar, par, abort_flag, p.status);
      __syncwarp();
      tc_fence_after();
    };
    if (warp == 1) {
      uint32_t uses = 0, n = 0, slot = 0, par = 0;      // uses of the score buffer, items, K ring position
      const uint32_t lo_q = desc_lo(smem_u32(sQ), 16), lo_k = desc_lo(smem_u32(sK), 16);
      for (int item; (item = item_at((int)n)) < n_items_u; ++n) {
        const Item it = uniform_item(p, item);
        bool first = true;
        for (int t = 0; t < it.ntiles; ++t) {
          const uint32_t idesc = make_idesc_bf16(BM, 16 * key_steps(it, t), false, false);
          const uint32_t dk = lo_k + slot * (uint32_t)(TILE >> 4);
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            if (x >= it.nx || t < it.tb[x] || t >= it.te[x]) continue;
            // the score buffer has been read (its first use waits for a phase before the first: passes at once), the K tile
            // is there, and the item's Q tiles
            wait3(&sm->s_free, (uses + 1) & 1, &sm->k_full[slot], par, first, &sm->q_full, n & 1);
            first = false;
            ++uses;
            const uint32_t dq = lo_q + x * (uint32_t)(TILE >> 4);
#pragma unroll
            for (int ks = 0; ks < DH / 16; ++ks)
              if (leader) mma_ss_lo(tmem, dq + koff(ks), dk + koff(ks), idesc, ks > 0 ? 1u : 0u);
            if (leader) mma_commit(&sm->s_full[x]);
          }
          if (leader) mma_commit(&sm->k_empty[slot]);
          if (leader && t == it.ntiles - 1) mma_commit(&sm->q_empty);
          if (++slot == KST) { slot = 0; par ^= 1; }
        }
      }
    } else {
      uint32_t tcnt[2] = {0, 0}, ecnt[2] = {0, 0}, slot = 0, par = 0;      // per unit: P V and items done; V ring position
      const uint32_t lo_v = desc_lo(smem_u32(sV), PANEL);
      for (int round = 0, item; (item = item_at(round)) < n_items_u; ++round) {
        const Item it = uniform_item(p, item);
        for (int t = 0; t < it.ntiles; ++t) {
          const int ksteps = key_steps(it, t);
          const uint32_t mv = lo_v + slot * (uint32_t)(TILE >> 4);
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            if (x >= it.nx || t < it.tb[x] || t >= it.te[x]) continue;
            // P has been written, the V tile is there, the epilogue of the unit's previous item has read the accumulator
            wait3(&sm->p_ready[x], tcnt[x] & 1, &sm->v_full[slot], par, t == it.tb[x], &sm->o_free[x], (ecnt[x] + 1) & 1);
            tcnt[x] += 1;
#pragma unroll
            for (int ks = 0; ks < 8; ++ks)
              if (leader && ks < ksteps)   // P of keys 16 ks .. 16 ks + 15 sits in columns 8 ks .. of the unit's P buffer
                mma_ts_lo(tmem + O_COL + x * 128, tmem + P_COL + x * 64 + ks * 8, mv + mnoff(ks), IDESC_PV, (t > it.tb[x] || ks > 0) ? 1u : 0u);
            if (leader) mma_commit(&sm->o_done[x]);
          }
          if (leader) mma_commit(&sm->v_empty[slot]);
          if (++slot == VST) { slot = 0; par ^= 1; }
        }
        ecnt[0] += 1;
        if (it.nx == 2) ecnt[1] += 1;
      }
    }
    if (leader && *abort_flag) mma_drain(&sm->drain[warp - 1]);      // (nothing is under way when the CTA frees its TMEM)
  } else if (warp == 3) {
    // ------------------------------------------------------------------ V tiles that end inside a step of 16 keys
    uint32_t tiles = 0, par = 0;             // tiles so far; bit s: parity of slot s
    for (int round = 0, item; (item = item_at(round)) < n_items; ++round) {
      const Item it = decode_item(p, item);
      tiles += it.ntiles;
      if (!has_tail(it)) continue;
      const uint32_t slot = (tiles - 1) % VST;
      mbar_wait(&sm->v_tail[slot], par >> slot & 1, abort_flag, p.status);
      par ^= 1u << slot;
      const int t = it.ntiles - 1, from = max(it.keys - t * BN, 0);
      for (int r = from + (lane >> 4); r < 16 * key_steps(it, t); r += 2)
        *reinterpret_cast<uint4*>(sV + slot * TILE + (lane >> 3 & 1) * PANEL + r * 128 + (lane & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
      fence_async_proxy();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm->v_full[slot]);
    }
  } else if (warp >= 12) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    // ------------------------------------------------------------------ the Q tiles of item n, then o of item n - 1
    const int lt = (warp - 12) * 32 + lane;   // 0..127: row of a unit
    const int rows = p.tpt * p.G, rt = p.by_G.div(lt), rg = lt - rt * p.G;
    uint32_t n = 0;
    uint32_t tcs[2] = {0, 0}, eps[2] = {0, 0};        // per unit: P V and items done
    const long long all_rows = (long long)p.B * p.Hk * p.Sq * p.G;
    auto epilogue = [&](const Item& it) {
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        if (x >= it.nx) continue;
        const uint32_t o_tmem = tmem + ((uint32_t)((warp & 3) * 32) << 16) + O_COL + x * 128;
        const int tok = (it.u0 + x) * p.tpt + rt;
        const bool row_ok = lt < rows && tok < p.Sq;
        const long long head = (long long)it.hk * p.G + rg;
        const long long packed = ((long long)it.b * p.Hk + it.hk) * p.Sq * p.G + (long long)tok * p.G + rg + it.piece * all_rows;
        tcs[x] += it.te[x] - it.tb[x];
        mbar_wait(&sm->ep_ready[x], eps[x] & 1, abort_flag, p.status);
        eps[x] += 1;
        const float inv = sm->ep_inv[x][lt], row_lse = sm->ep_lse[x][lt];
        mbar_wait(&sm->o_done[x], (tcs[x] - 1) & 1, abort_flag, p.status);
        tc_fence_after();
        __nv_bfloat16* o_row = p.o + it.b * p.os.b + tok * p.os.t + head * p.os.h;
        __nv_bfloat16* r_row = p.resid ? p.resid + (((long long)it.b * p.Sq + tok) * p.Hk * p.G + head) * DH : nullptr;
#pragma unroll 1
        for (int c = 0; c < 8; ++c) {
          uint32_t ov[16];
          tmem_ld16(o_tmem + c * 16, ov);
          tmem_ld_wait();
          if (c == 7) {
            tc_fence_before();
            mbar_arrive(&sm->o_free[x]);
          }
          if (row_ok) {
            if (!p.cut) {
#pragma unroll
              for (int i = 0; i < 16; i += 8) {
                float v[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = inv == 0.f ? 0.f : __uint_as_float(ov[i + k]) * inv;
                store8_resid(o_row + i, r_row ? r_row + i : nullptr, v);
              }
              o_row += 16;
              if (r_row) r_row += 16;
            } else {
              float* to = p.part_o + packed * DH + 16 * c;
#pragma unroll
              for (int i = 0; i < 16; ++i) ov[i] = inv == 0.f ? 0u : __float_as_uint(__uint_as_float(ov[i]) * inv);
#pragma unroll
              for (int i = 0; i < 16; i += 4) *reinterpret_cast<uint4*>(to + i) = make_uint4(ov[i], ov[i + 1], ov[i + 2], ov[i + 3]);
            }
          }
        }
        if (row_ok) {
          if (!p.cut) p.lse[((long long)it.b * p.Hk * p.G + head) * p.Sq + tok] = row_lse;
          else p.part_lse[packed] = row_lse;
        }
      }
    };
    for (int item; (item = item_at((int)n)) < n_items; ++n) {
      if (lt == 0) {
        const Item it = decode_item(p, item);
        if (n >= 1) mbar_wait(&sm->q_empty, (n - 1) & 1, abort_flag, p.status);
        mbar_expect_tx(&sm->q_full, (uint32_t)(it.nx * rows * DH * 2));
        for (int x = 0; x < it.nx; ++x) {
          const int tok = (it.u0 + x) * p.tpt;
          tma_load_5d(sQ + x * TILE, &tmQ, &sm->q_full, 0, 0, tok, it.hk, it.b);
          tma_load_5d(sQ + x * TILE + PANEL, &tmQ, &sm->q_full, 64, 0, tok, it.hk, it.b);
        }
        if (*abort_flag) mbar_wait(&sm->q_full, n & 1, abort_flag, p.status);     // landed before the CTA may exit
      }
      __syncwarp();
      if (n >= 1) epilogue(decode_item(p, item_at((int)n - 1)));      // (read again: two items do not fit the registers)
    }
    if (n >= 1) epilogue(decode_item(p, item_at((int)n - 1)));
  } else if (warp >= 4) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
    // ------------------------------------------------------------------ softmax of one unit
    const int x = (warp - 4) >> 2;                  // unit of this warp group
    const int quad = warp & 3;                      // TMEM lane quarter this warp may access
    const int r = quad * 32 + lane;                 // row of the unit
    const int rt = p.by_G.div(r);
    const bool is_row = r < p.tpt * p.G;
    const uint32_t lane_addr = (uint32_t)(quad * 32) << 16;
    const uint32_t s_tmem = tmem + lane_addr;
    const uint32_t p_tmem = tmem + lane_addr + P_COL + x * 64;
    const uint32_t o_tmem = tmem + lane_addr + O_COL + x * 128;
    uint32_t tc = 0, items = 0;                      // key tiles and items done on this unit
    for (int round = 0, item; (item = item_at(round)) < n_items; ++round) {
      const Item it = decode_item(p, item);
      if (x >= it.nx) continue;
      const int tb = it.tb[x], te = it.te[x];
      // tiles in [all_lo, all_hi) are seen by every row as a whole
      const int all_lo = (max(it.full_lo[x] - it.k_begin, 0) + BN - 1) / BN, all_hi = max(min(it.full_hi[x] - it.k_begin, it.keys), 0) / BN;
      // of tile t, this row's range: first key and number of keys
      auto seen = [&](int t) {
        const int tok = (it.u0 + x) * p.tpt + rt;
        int2 r = make_int2(0, 0);
        if (is_row && tok < p.Sq) r = __ldg(p.rows + (long long)mask_batch(p.Bm, it.b) * p.Sq + tok);
        const int a = max(r.x - it.k_begin, 0) - t * BN;
        return make_int2(a, max(min(r.y - it.k_begin, it.keys) - t * BN - a, 0));
      };
      float m_used = MODE == kCapped ? p.cap.shift : -INFINITY, l = 0.f, l_r = 0.f;   // l: exact sum (for LSE); l_r: sum of the bf16-rounded weights
      for (int t = tb; t < te; ++t, ++tc) {
        mbar_wait(&sm->s_full[x], tc & 1, abort_flag, p.status);
        tc_fence_after();
        const int valid = min(BN, it.keys - t * BN);
        uint32_t sv[128];
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld32(s_tmem + 32 * c, *reinterpret_cast<uint32_t(*)[32]>(&sv[32 * c]));
        tmem_ld_wait();
        tc_fence_before();
        mbar_arrive(&sm->s_free);                    // the other unit's Q K^T may have the buffer
        if constexpr (MODE == kCapped) {
          // Tiles that every row sees as a whole, small scores: one run of instructions without a branch, in which the polynomial of some
          // scores (FMA pipe) goes beside the exponentials of others.
          const bool masked = t < all_lo || t >= all_hi;
          float s0 = 0.f, s1 = 0.f, r0 = 0.f, r1 = 0.f;
          auto p_free = [&]() {                              // P V of the tile before has read the P buffer
            if (tc > 0) {
              mbar_wait(&sm->o_done[x], (tc - 1) & 1, abort_flag, p.status);
              tc_fence_after();
            }
          };
          if (__builtin_expect(!masked && polynomial_does<128>(sv, p.cap), 1)) {
            uint32_t pk[4][16];
            exp_capped32<true>(sv, p.cap, pk[0], s0, s1, r0, r1);
            exp_capped32<true>(sv + 32, p.cap, pk[1], s0, s1, r0, r1);
            p_free();
            tmem_st16(p_tmem, pk[0]);
            tmem_st16(p_tmem + 16, pk[1]);
            exp_capped32<true>(sv + 64, p.cap, pk[2], s0, s1, r0, r1);
            tmem_st16(p_tmem + 32, pk[2]);
            exp_capped32<true>(sv + 96, p.cap, pk[3], s0, s1, r0, r1);
            tmem_st16(p_tmem + 48, pk[3]);
          } else {
            const int2 r = masked ? seen(t) : make_int2(0, BN);
            p_free();
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              if (c > 0 && 32 * c >= valid) continue;        // (uniform; P V takes the keys up to `valid` only)
              if (masked) mask32(sv + 32 * c, 32 * c, r.x, r.y, 0u);      // (what nobody sees has no say in how the others are capped)
              cap32<false>(sv + 32 * c, p.cap);
              if (masked) mask32(sv + 32 * c, 32 * c, r.x, r.y, MINUS_INF);
              uint32_t pk[16];
              exp_capped32<false>(sv + 32 * c, p.cap, pk, s0, s1, r0, r1);
              tmem_st16(p_tmem + 16 * c, pk);
            }
          }
          l += s0 + s1;
          l_r += r0 + r1;
          tmem_st_wait();
          tc_fence_before();
          mbar_arrive(&sm->p_ready[x]);
          continue;
        }
        if (MODE == kCappedWide) {
          const bool masked = t < all_lo || t >= all_hi;
          const int2 r = masked ? seen(t) : make_int2(0, BN);
#pragma unroll
          for (int c = 0; c < 4; ++c) {
#pragma unroll
            for (int i = 32 * c; i < 32 * c + 32; ++i) sv[i] = __float_as_uint(__uint_as_float(sv[i]) * p.cap.pre);
            if (masked) mask32(sv + 32 * c, 32 * c, r.x, r.y, 0u);
            cap32<true>(sv + 32 * c, p.cap);
          }
        }
        if (__builtin_expect(t < all_lo || t >= all_hi, 0)) {      // keys outside the row's range get score -inf
          const int2 r = seen(t);
#pragma unroll
          for (int c = 0; c < 4; ++c) mask32(sv + 32 * c, 32 * c, r.x, r.y, MINUS_INF);
        }
        float mx0 = -INFINITY, mx1 = -INFINITY, mx2 = -INFINITY, mx3 = -INFINITY;
#pragma unroll
        for (int i = 0; i < BN; i += 8) {
          mx0 = max3(mx0, __uint_as_float(sv[i]), __uint_as_float(sv[i + 1]));
          mx1 = max3(mx1, __uint_as_float(sv[i + 2]), __uint_as_float(sv[i + 3]));
          mx2 = max3(mx2, __uint_as_float(sv[i + 4]), __uint_as_float(sv[i + 5]));
          mx3 = max3(mx3, __uint_as_float(sv[i + 6]), __uint_as_float(sv[i + 7]));
        }
        const float scale = MODE == kPlain ? p.scale_log2 : 1.0f;
        const float mx = fmaxf(fmaxf(mx0, mx1), fmaxf(mx2, mx3)) * scale;      // exp2 domain from here on (the scale is positive)
        // lazy rescale: keep the old reference max unless the new one is more than 2^8 larger
        float factor = 1.0f;
        bool need = false;
        if (t == tb) {
          m_used = mx;
        } else if (mx > m_used + RESCALE_LOG2) {
          need = m_used > -INFINITY;                 // (else the row has seen nothing so far: its sums are 0)
          factor = need ? ex2(m_used - mx) : 1.0f;
          m_used = mx;
        }
        auto rescale_o = [&]() {                     // P V of the tile before is complete
#pragma unroll 1
          for (int c = 0; c < 8; ++c) {
            uint32_t ov[16];
            tmem_ld16(o_tmem + c * 16, ov);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) ov[i] = __float_as_uint(__uint_as_float(ov[i]) * factor);
            tmem_st16(o_tmem + c * 16, ov);
          }
        };
        float s0 = 0.f, s1 = 0.f, r0 = 0.f, r1 = 0.f;
        const float neg_m = m_used == -INFINITY ? 0.f : -m_used;
        {
          // the first half's weights stay in registers until P V of the tile before has read the P buffer
          uint32_t pk[2][16];
          exp_pack32(sv, scale, neg_m, pk[0], s0, s1, r0, r1);
          const uint32_t pv_done = mbar_test_wait(&sm->o_done[x], (tc + 1) & 1);      // (an early look, because the answer takes its time)
          if (valid > 32) exp_pack32(sv + 32, scale, neg_m, pk[1], s0, s1, r0, r1);
          if (tc > 0) {                              // (of the item before, where t is its first)
            if (!__all_sync(0xffffffffu, pv_done)) mbar_wait(&sm->o_done[x], (tc - 1) & 1, abort_flag, p.status);
            tc_fence_after();
            if (t > tb && __any_sync(0xffffffffu, need)) {
              rescale_o();
              l *= factor;
              l_r *= factor;
            }
          }
          tmem_st16(p_tmem, pk[0]);
          tmem_st16(p_tmem + 16, pk[1]);             // (whatever it holds where valid <= 32: P V does not read it)
        }
#pragma unroll
        for (int c = 2; c < 4; ++c) {
          if (32 * c < valid) {                      // (uniform; P V takes the keys up to `valid` only)
            uint32_t pk[16];
            exp_pack32(sv + 32 * c, scale, neg_m, pk, s0, s1, r0, r1);
            tmem_st16(p_tmem + 16 * c, pk);
          }
        }
        l += s0 + s1;
        l_r += r0 + r1;
        tmem_st_wait();
        tc_fence_before();
        mbar_arrive(&sm->p_ready[x]);
      }
      // ---- hand the row's normalisers to the epilogue warps, once they are through with the unit's previous item, and go on
      if (items >= 1) mbar_wait(&sm->o_free[x], (items - 1) & 1, abort_flag, p.status);
      sm->ep_inv[x][r] = l_r == 0.f ? 0.f : 1.0f / l_r;
      sm->ep_lse[x][r] = l == 0.f ? -INFINITY : (m_used + log2f(l)) * 0.6931471805599453f;
      mbar_arrive(&sm->ep_ready[x]);
      ++items;
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) tmem_dealloc(tmem, TMEM_COLS);
}

}  // namespace tcf

// K or V: {head_dim, tokens, heads, samples}, a tile of 128 tokens; Q or dO: {head_dim, heads of a group, tokens, key heads, samples}, a
// unit of packed rows.
bool make_tmap_keys(CUtensorMap* map, const void* base, const RDims& D, const Strides& s) {
  const uint64_t n[4] = {(uint64_t)D.d, (uint64_t)D.Sk, (uint64_t)D.Hk, (uint64_t)D.B};
  const uint64_t st[4] = {1, (uint64_t)s.t, (uint64_t)s.h, (uint64_t)s.b};
  const uint32_t box[4] = {64, 128, 1, 1};
  return sm100::make_tmap_bf16_strided(map, base, 4, n, st, box);
}
bool make_tmap_units(CUtensorMap* map, const void* base, const RDims& D, const Strides& s) {
  const uint64_t n[5] = {(uint64_t)D.d, (uint64_t)D.G, (uint64_t)D.Sq, (uint64_t)D.Hk, (uint64_t)D.B};
  const uint64_t st[5] = {1, (uint64_t)s.h, (uint64_t)s.t, (uint64_t)s.h * D.G, (uint64_t)s.b};
  const uint32_t box[5] = {64, (uint32_t)D.G, (uint32_t)D.tpt, 1, 1};
  return sm100::make_tmap_bf16_strided(map, base, 5, n, st, box);
}

// The polynomial's coefficients with the factors of score and result folded in.  Where the score's would leave fp32's range (caps of some
// hundred times what is usual, scales far from it) scores are multiplied by it first.  Scores of less than 10^-9 change no
// weight: tanh is taken of scale s / cap whatever the cap, and multiplied by 10^-9 at least, so that 1 / c' is a number of fp32's.
Cap make_cap(const RDims& D) {
  static const double k[5] = {0.9999994349, -0.333282515, 0.1325898302, -0.05005629744, 0.01292962787};
  Cap c = {};
  if (!(D.cap > 0.f)) return c;
  double a = std::min((double)D.scale / D.cap, 1e30);
  const double top = std::max((double)D.cap, 1e-9) * 1.4426950408889634;
  c.c = (float)top;
  c.pre = 1.f;
  if (!(a >= 2e-4 && a <= 1e3 && top <= 1e6)) { c.pre = (float)a; a = 1.0; }
  c.twice_log2 = (float)(2.0 * a * 1.4426950408889634);
  c.most = (float)(0.75 / a);
  c.shift = c.pre == 1.f && c.c <= CAP_MOST ? std::max(c.c - 80.0f, 0.0f) : 0.f;
  double f = a;
  for (int i = 0; i < 5; ++i, f *= a * a) {
    c.p[i] = (float)(k[i] * top * f);
    c.u[i] = (float)(k[i] * f);
  }
  return c;
}

// The more heads together, the evener the CTAs' shares; their keys and values have to stay in the L2 (126 MB).  33K clip by frames, capped: 4 of 12
// heads (67 MB) 3.71 ms, 6 (101 MB) 3.52, all (201 MB) 3.59.  Groups are equal ones: a prime number of heads that do not fit together goes head by
// head (causal, 1,600 tokens: 131 heads 168 us, 132 heads, two groups, 143).
static int group_of_heads(const RDims& D) {
  const long long all = (long long)D.B * D.Hk, one = (long long)D.Sk * D.d * 4;      // K and V of a head, bytes
  long long g = std::max<long long>(1, std::min<long long>(all, (101ll << 20) / one));
  while (all % g) --g;
  return (int)g;
}

int tc_range_fwd(const RDims& D, const Plan& plan, const FwdArgs& a, cudaStream_t st) {
  using namespace tcf;
  const long long items = (long long)D.B * D.Hk * D.nI * D.smax;      // (at most)
  if (items > (long long)INT32_MAX - 4096) return VMOBA_ERR_SHAPE;
  Params p;
  p.B = D.B; p.Hk = D.Hk; p.G = D.G; p.Sq = D.Sq; p.Sk = D.Sk; p.Bm = D.Bm; p.tpt = D.tpt; p.nU = D.nU; p.nI = D.nI;
  p.cut = D.smax > 1; p.reps = D.reps; p.n_items = (int)items;
  p.rows = plan.rows; p.units = plan.units; p.order = plan.order; p.head = plan.head; p.work = plan.work;
  p.group = group_of_heads(D);
  p.by_set = FastDiv(p.group * D.nI); p.by_group = FastDiv(p.group);
  p.by_reps = FastDiv(D.reps); p.by_Hk = FastDiv(D.Hk); p.by_G = FastDiv(D.G);
  p.scale_log2 = D.scale * LOG2E;
  p.cap = make_cap(D);
  p.o = (__nv_bfloat16*)a.o; p.resid = (__nv_bfloat16*)a.resid; p.os = a.os; p.lse = a.lse;
  p.part_o = a.part_o; p.part_lse = a.part_lse; p.status = a.status;
  CUtensorMap tmK, tmV, tmQ;
  if (!make_tmap_keys(&tmK, a.k, D, a.ks) || !make_tmap_keys(&tmV, a.v, D, a.vs) || !make_tmap_units(&tmQ, a.q, D, a.qs)) return VMOBA_ERR_CUDA;
  auto kernel = !(D.cap > 0.f)           ? attn_range_fwd_kernel<kPlain>
                : p.cap.c <= CAP_MOST && p.cap.pre == 1.f ? attn_range_fwd_kernel<kCapped>
                                      : attn_range_fwd_kernel<kCappedWide>;
  VMOBA_CUDA_OK(allow_smem(kernel, (int)SMEM_BYTES));
  launch_kernel(kernel, (unsigned)std::min<long long>(items, sm_count()), THREADS, SMEM_BYTES, st, tmK, tmV, tmQ, p);
  VMOBA_LAUNCH_OK(1);
  return VMOBA_OK;
}

}  // namespace range
}  // namespace vmoba
