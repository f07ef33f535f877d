// Tensor-core backward of attention over key ranges (bf16, head_dim 128): the dense backward of attn_tc_bwd.cu with the units that a key
// tile has to visit taken from the plan.
//
// A CTA takes one tile of 128 keys of a key head (by ticket) and streams the units of packed query rows that reach into it, all heads of the
// group among them, so that dK and dV of shared heads are sums inside the CTA and are written once.  Per unit, keys on the TMEM lanes:
//     S^T = K Q^T;  P^T = exp2(c S^T - lse), capped exp2(c' u - lse), u = tanh, 0 outside the range;  dV += P^T dO
//     dP^T = V dO^T;  dS^T = P^T (dP^T - D) (1 - u^2);  dK += dS^T Q;  dQ^T = K^T dS^T, added into an fp32 accumulator
// P and dS are rounded to bf16 (2^-8 each, once) for the products that the tensor cores do with them; in fp32 halves they would be twice
// the products, and dQ, dK and dV are rounded to the same type after that.  All sums, D and the weights under dS are fp32.
// The slope 1 - u^2 is taken into the fp32 weights that the second step keeps, at no register.  tanh comes from the forward's polynomial
// where a warp's scores allow, else from 1 - 2 / (1 + exp(2 x)): the same error in the weights and in the lse that they are divided by, so that
// it leaves their sum at one.  (With a term less, off by 4.4e-5 of a score, weights of scores of 300 were 1.3 % off, all to the same side.)
//
// Bound by the exponentials, the turns of dQ and the tensor cores' waits for both, as the dense backward is.  13,440 tokens x 12 heads: eight
// clips packed, 633 GFLOP, 866 us (730 TFLOP/s); two clips by frames, key heads shared by three, 1.04 ms (730), capped 1.26 ms (600), and 1.59 where
// scores have the cap's size.
//
// dQ of a unit is added key tile after key tile, so that the backward repeats bit for bit: a counter per unit says how many of the
// tiles of its hull (which are consecutive) have been added; the first one stores.  A tile waits for lower tickets only.  Units go
// from the last to the first: where hulls move forward with the queries (causal order, windows, clips) the lowest tile that a unit
// waits for then starts with it, or all tiles come to it at the same time.  (From the first to the last, the tiles of a causal clip's later
// frames waited for those of the first frame to get there: 13K tokens, two clips, 1.55 ms.)  Up to four
// accumulators (tile n of a unit's hull adds to accumulator n mod 4) where they fit 128 MB, see the dense backward.
//
// Rows of a unit that see nothing are brought in as zeros (asynchronous copies instead of the TMA tile), keys that no query sees are
// cleared in K: 0 times what they hold would not be 0 if it is not finite.
#include <algorithm>

#include "attn_range.cuh"
#include "sm100.cuh"

namespace vmoba {
namespace range {
namespace tcb {

using namespace sm100;

constexpr int BN = 128, DH = 128, QU = 128;
constexpr int PANEL = 128 * 128;             // bytes of one 64-column panel of a 128-row tile (16 KB)
constexpr int TILE = 2 * PANEL;              // [128 x 128] bf16 (32 KB)
constexpr uint32_t TMEM_COLS = 512;
constexpr uint32_t ST_COL = 0, DPT_COL = 128, DV_COL = 256, DK_COL = 384;
constexpr uint32_t ROW16 = 16u << 16;        // TMEM lanes 16 .. 31 of a warp's quarter
constexpr float LOG2E = 1.4426950408889634f;
constexpr int NQ = 3;                        // Q tiles in flight (one dO tile: see the dense backward)

struct Smem {
  uint64_t k_full, k_ready, v_full;                                // K landed / and cleared of keys that nobody sees; V landed
  uint64_t q_full[NQ], q_empty[NQ], do_full, do_empty;             // Q / dO rows of a unit (128 arrivals) / no longer needed (commit)
  uint64_t s_full, p_ready;                                        // S^T complete (commit) / P^T written (256 arrivals)
  uint64_t dp_full, ds_ready;                                      // dP^T complete (commit) / dS^T written (256 arrivals)
  uint64_t dq_full, dq_free;                                       // dQ^T complete (commit) / read out of TMEM (256 arrivals)
  uint64_t acc_done;                                               // dV / dK complete (commit)
  uint64_t turn_ok, rows_out, rows_seen;                           // it is this tile's turn / its dQ is on the way (256 arrivals) / and noted
  uint64_t drain;                                                  // (after a time-out only)
  uint32_t tmem_base;
  int ticket;
  int abort_flag;
  alignas(16) float lse2[NQ][QU];            // lse * log2 e, with the Q rows of a unit
  alignas(16) float negD[2][QU];             // -rowsum(dO * O), with its dO rows
};
// K, V, three Q tiles and a dO tile, the dS^T tile ([128 keys][128 queries] bf16)
constexpr size_t SMEM_BYTES = 7 * TILE + sizeof(Smem) + 32;
static_assert(SMEM_BYTES <= 232448, "range backward: shared memory");
// Warp groups: {TMA, MMA, turns, turns}, 4 Q loaders, 4 dO loaders, 2 x 4 compute, 2 x 4 dQ writers.  896 threads start with 72
// registers each: 2 x 112 + 2 x 80 + 3 x 40 = 7 x 72.
constexpr int THREADS = 896;
constexpr uint32_t IDESC_TN = make_idesc_bf16(128, 128, false, true);    // dV, dK: A from TMEM, B MN-major

struct Params {
  int B, Hk, G, Sq, Sk, Bm, tpt, nU, nK;
  const int2* rows;
  const int4* units;
  const int4 *keys, *runs;
  FastDiv by_G, by_tpt, by_rows, by_Hk, by_parts;
  const __nv_bfloat16 *q, *d_o;
  Strides qs, dos;
  const float *lse, *Dv;
  float scale;
  float to_exp2;               // scores, or tanh of capped ones, -> exp2 domain: scale * log2 e, or c'
  Cap cap;
  float cap_apart;             // |score| up to this: by the polynomial, whatever the others of the warp are; 0: as the warp's vote says
  float cap_masked;            // stands for tanh of a score outside its query's range: a weight of 0 and a finite slope
  __nv_bfloat16 *dk, *dv;
  Strides dks, dvs;
  int dkv_32;                  // rows of dk and dv are 32-byte aligned: they go out with 32-byte stores
  float* dq_acc;               // fp32 [parts][packed rows][head_dim]; columns in the order of the dQ writers: position
                               // 32 w + 4 r + a holds column 32 w + r + 8 a (r < 8, a < 4)
  int parts;
  int* turns;                  // [parts][B * Hk][nU], then the ticket; zero at the start
  int group;                   // heads whose key tiles are taken in turn
  int32_t* status;
};

struct Item {
  int bhk, b, hk, tile, key0, valid;
  int4 info;                   // first and one past the last unit, first and one past the last key that somebody sees
  int4 run;                    // units that reach into the tile; [y, z): units that see all of it
  const int4* units;
};
__device__ __forceinline__ Item decode(const Params& p, int ticket) {
  // groups of heads; in a group, the first key tile of every head, then the second ones
  Item it;
  const int per = p.group * p.nK, all = p.B * p.Hk, first = ticket / per * p.group, heads = min(p.group, all - first), r = ticket % per;
  it.tile = r / heads;
  it.bhk = first + r - it.tile * heads;
  it.b = it.bhk / p.Hk;
  it.hk = it.bhk - it.b * p.Hk;
  it.key0 = it.tile * BN;
  it.valid = min(BN, p.Sk - it.key0);
  const int bm = mask_batch(p.Bm, it.b);
  it.info = __ldg(p.keys + (long long)bm * p.nK + it.tile);
  it.run = __ldg(p.runs + (long long)bm * p.nK + it.tile);
  it.units = p.units + (long long)bm * p.nU;
  return it;
}

// Walks the units of an item, from the last to the first.  Where they are consecutive, as they nearly always are, no record is read on
// the way.
struct Walk {
  int u, first, tile;
  bool gaps;
  const int4* units;
  __device__ __forceinline__ explicit Walk(const Item& it)
      : u(it.info.y), first(it.info.x), tile(it.tile), gaps(it.run.x != it.info.y - it.info.x), units(it.units) {}
  __device__ __forceinline__ bool next() {
    --u;
    if (__builtin_expect(gaps, 0))
      while (u >= first && !reaches(__ldg(units + u), tile, BN)) --u;
    return u >= first;
  }
};
__device__ __forceinline__ int unit_rows(const Params& p, int u) { return min(p.tpt, p.Sq - u * p.tpt) * p.G; }

__device__ __forceinline__ void cp_async16(uint32_t smem_dst, const void* gsrc, uint32_t bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_dst), "l"(gsrc), "r"(bytes) : "memory");
}
__device__ __forceinline__ void red_add_v4(float* addr, float a, float b, float c, float d) {
  asm volatile("red.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(addr), "f"(a), "f"(b), "f"(c), "f"(d) : "memory");
}
__device__ __forceinline__ float rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Waits (bounded) until a turn counter has reached `turn`; the reductions of other threads follow a barrier.
__device__ __forceinline__ void turn_wait(const int* addr, int turn, volatile int* abort_flag, int32_t* status) {
  constexpr uint32_t kPolls = 1u << 22;
  const uint32_t limit = *abort_flag ? 16u : kPolls;
  for (uint32_t i = 0; i < limit; ++i) {
    int at;
    asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(at) : "l"(addr) : "memory");
    if (at >= turn) return;
    __nanosleep(32);
  }
  *abort_flag = 1;
  set_status(status, VMOBA_ERR_TIMEOUT);
}
// Passes the turn on, at device scope: behind the reductions of the threads whose barrier this one has waited for.
__device__ __forceinline__ void turn_pass(int* addr, int next) {
  asm volatile("fence.acq_rel.gpu;" ::: "memory");
  asm volatile("st.relaxed.gpu.global.s32 [%0], %1;" ::"l"(addr), "r"(next) : "memory");
}

__device__ __forceinline__ uint32_t lo_k(uint32_t tile_addr) { return desc_lo(tile_addr, 16); }
__device__ __forceinline__ uint32_t lo_mn(uint32_t tile_addr) { return desc_lo(tile_addr, PANEL); }
__device__ __forceinline__ constexpr uint32_t koff(int ks) { return (uint32_t)(((ks >> 2) * PANEL + (ks & 3) * 32) >> 4); }
__device__ __forceinline__ constexpr uint32_t mnoff(int ks) { return (uint32_t)((ks * 2048) >> 4); }

// Fragment shapes: see attn_tc_bwd.cu.
__device__ __forceinline__ void tmem_ld_16x256_x8(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x8.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_ld_16x256_x4(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_st_16x128_x4(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.16x128b.x4.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(r[0]),
               "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
__device__ __forceinline__ void stmatrix_x4(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d)
               : "memory");
}

// MULTI: several accumulators (with p.parts read in the one kernel, the case of one is slower).
template <bool CAP, bool MULTI>
__global__ void __launch_bounds__(THREADS, 1)
attn_range_bwd_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                      const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmO, const Params p) {
  if (!grid_begin()) return;
  extern __shared__ uint8_t smem_raw[];
  // the swizzled tiles need 1024-byte alignment and there is no room for alignment slack
  if ((smem_u32(smem_raw) & 1023u) != 0) {
    if (threadIdx.x == 0) set_status(p.status, VMOBA_ERR_CUDA);
    return;
  }
  uint8_t* sK = smem_raw;
  uint8_t* sV = smem_raw + TILE;
  uint8_t* sQ = smem_raw + 2 * TILE;           // [NQ]
  uint8_t* sO = smem_raw + (2 + NQ) * TILE;    // dO
  uint8_t* sDS = smem_raw + 6 * TILE;
  Smem* sm = reinterpret_cast<Smem*>(smem_raw + 7 * TILE);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  volatile int* abort_flag = &sm->abort_flag;
  auto wait = [&](uint64_t* bar, uint32_t parity) { return mbar_wait(bar, parity, abort_flag, p.status); };

  if (threadIdx.x == 0) {
    mbar_init(&sm->k_full, 1); mbar_init(&sm->k_ready, 1); mbar_init(&sm->v_full, 1);
    for (int b = 0; b < NQ; ++b) { mbar_init(&sm->q_full[b], 128); mbar_init(&sm->q_empty[b], 1); }
    mbar_init(&sm->do_full, 128); mbar_init(&sm->do_empty, 1);
    mbar_init(&sm->s_full, 1); mbar_init(&sm->p_ready, 256);
    mbar_init(&sm->dp_full, 1); mbar_init(&sm->ds_ready, 256);
    mbar_init(&sm->dq_full, 1); mbar_init(&sm->dq_free, 256);
    mbar_init(&sm->acc_done, 1); mbar_init(&sm->drain, 1);
    mbar_init(&sm->turn_ok, 1); mbar_init(&sm->rows_out, 256); mbar_init(&sm->rows_seen, 1);
    sm->abort_flag = 0;
    sm->ticket = atomicAdd(p.turns + (long long)(MULTI ? p.parts : 1) * p.B * p.Hk * p.nU, 1);
    fence_barrier_init();
    prefetch_tmap(&tmK);
    prefetch_tmap(&tmV);
  }
  // rows that a unit leaves over (the group's size does not divide 128): zeros, which no copy writes over
  for (int i = threadIdx.x; i < (NQ + 1) * (QU - p.tpt * p.G) * 16; i += THREADS) {
    const int r = p.tpt * p.G + i / ((NQ + 1) * 16), at = i % ((NQ + 1) * 16);
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
  const Item it = decode(p, sm->ticket);
  const bool some = it.info.y > it.info.x;       // somebody sees a key of this tile
  const long long all_rows = (long long)p.B * p.Hk * p.Sq * p.G;

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
    if (warp == 0) {
      // ---------------------------------------------------------------- TMA: the K and V tiles
      if (some) {
        if (lane == 0) {
          mbar_expect_tx(&sm->k_full, TILE);
          tma_load_4d(sK, &tmK, &sm->k_full, 0, it.key0, it.hk, it.b);
          tma_load_4d(sK + PANEL, &tmK, &sm->k_full, 64, it.key0, it.hk, it.b);
          mbar_expect_tx(&sm->v_full, TILE);
          tma_load_4d(sV, &tmV, &sm->v_full, 0, it.key0, it.hk, it.b);
          tma_load_4d(sV + PANEL, &tmV, &sm->v_full, 64, it.key0, it.hk, it.b);
        }
        __syncwarp();
        wait(&sm->k_full, 0);
        __syncwarp();
        if (it.info.z > 0 || it.info.w < BN) {             // keys that nobody sees
          for (int r = lane >> 4; r < BN; r += 2)
            if (r < it.info.z || r >= it.info.w)
              *reinterpret_cast<uint4*>(sK + (lane >> 3 & 1) * PANEL + r * 128 + (lane & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
          fence_async_proxy();
          __syncwarp();
        }
        if (lane == 0) mbar_arrive(&sm->k_ready);
        wait(&sm->v_full, 0);                              // landed before the CTA may exit, whatever the others do
      }
    } else if (warp == 1) {
      // ---------------------------------------------------------------- MMA issuer: the whole warp walks the loop, one elected lane
      // issues (warp-uniform control flow; see elect_one).  Order per unit and what overlaps it: see attn_tc_bwd.cu.
      const bool leader = elect_one();
      auto wwait = [&](uint64_t* bar, uint32_t parity) { wait(bar, parity); __syncwarp(); };
      auto uniform = [](int v) { return __reduce_max_sync(0xffffffffu, v); };
      Walk walk(it);
      walk.u = uniform(walk.u);
      walk.first = uniform(walk.first);
      walk.gaps = uniform(walk.gaps) != 0;
      // next unit's steps of 16 queries, or 0
      auto next = [&]() { return uniform(walk.next() ? (unit_rows(p, walk.u) + 15) >> 4 : 0); };
      uint32_t s_slot = 0, s_par = 0, k_slot = 0;      // Q ring: next unit's slot and parity for S^T, slot of the current dK
      const uint32_t kK = lo_k(smem_u32(sK)), kV = lo_k(smem_u32(sV)), mK = lo_mn(smem_u32(sK)), mS = lo_mn(smem_u32(sDS));
      const uint32_t kQ = lo_k(smem_u32(sQ)), kO = lo_k(smem_u32(sO)), mQ = lo_mn(smem_u32(sQ)), mO = lo_mn(smem_u32(sO));
      constexpr uint32_t STAGE = TILE >> 4;
      const int key_steps = uniform((it.valid + 15) >> 4);
      auto issue_s = [&](int steps) {
        wwait(&sm->q_full[s_slot], s_par);
        tc_fence_after();
        const uint32_t idesc = make_idesc_bf16(128, 16 * steps, false, false);
        const uint32_t b = kQ + s_slot * STAGE;
        if (++s_slot == NQ) { s_slot = 0; s_par ^= 1; }
#pragma unroll
        for (int ks = 0; ks < DH / 16; ++ks)
          if (leader) mma_ss_lo(tmem + ST_COL, kK + koff(ks), b + koff(ks), idesc, ks > 0 ? 1u : 0u);
        if (leader) mma_commit(&sm->s_full);
      };
      auto issue_dp = [&](uint32_t u, int steps) {
        wwait(&sm->do_full, u & 1);
        if (u >= 1) wwait(&sm->dq_free, (u - 1) & 1);          // the columns held dQ^T of the unit before
        tc_fence_after();
        const uint32_t idesc = make_idesc_bf16(128, 16 * steps, false, false);
#pragma unroll
        for (int ks = 0; ks < DH / 16; ++ks)
          if (leader) mma_ss_lo(tmem + DPT_COL, kV + koff(ks), kO + koff(ks), idesc, ks > 0 ? 1u : 0u);
        if (leader) mma_commit(&sm->dp_full);
      };
      auto issue_dv = [&](uint32_t u, int steps) {
        wwait(&sm->p_ready, u & 1);
        tc_fence_after();
#pragma unroll
        for (int ks = 0; ks < 8; ++ks)       // P^T of queries 64 h .. sits in columns 64 h .. 64 h + 31
          if (leader && ks < steps)
            mma_ts_lo(tmem + DV_COL, tmem + ST_COL + (ks >> 2) * 64 + (ks & 3) * 8, mO + mnoff(ks), IDESC_TN, (ks > 0 || u > 0) ? 1u : 0u);
        if (leader) mma_commit(&sm->do_empty);
      };
      int now = next();
      if (now) {
        wwait(&sm->k_ready, 0);
        int then = next();
        issue_s(now);
        wwait(&sm->v_full, 0);
        issue_dp(0, now);
        issue_dv(0, now);
        if (then) issue_s(then);
        for (uint32_t i = 0;; ++i) {
          wwait(&sm->ds_ready, i & 1);
          tc_fence_after();
          const uint32_t b = mQ + k_slot * STAGE;
#pragma unroll
          for (int ks = 0; ks < 8; ++ks)
            if (leader && ks < now)
              mma_ts_lo(tmem + DK_COL, tmem + DPT_COL + (ks >> 2) * 64 + (ks & 3) * 8, b + mnoff(ks), IDESC_TN, (ks > 0 || i > 0) ? 1u : 0u);
          if (leader) mma_commit(&sm->q_empty[k_slot]);
          if (++k_slot == NQ) k_slot = 0;
          // dQ^T over dP^T and dS^T: in order behind the dK MMAs that read dS^T there
          const uint32_t idesc = make_idesc_bf16(128, 16 * now, true, true);
#pragma unroll
          for (int ks = 0; ks < 8; ++ks)
            if (leader && ks < key_steps) mma_ss_lo(tmem + DPT_COL, mK + mnoff(ks), mS + mnoff(ks), idesc, ks > 0 ? 1u : 0u);
          if (leader) mma_commit(&sm->dq_full);
          if (!then) break;
          now = then;
          issue_dp(i + 1, now);
          issue_dv(i + 1, now);
          then = next();
          if (then) issue_s(then);
        }
        if (leader) mma_commit(&sm->acc_done);
      }
      if (leader && *abort_flag) mma_drain(&sm->drain);
    } else if (lane == 0) {
      // ---------------------------------------------------------------- turns: warp 3 waits for them, warp 2 passes them on.
      // Warp 3 lets the writers go on only when warp 2 has noted the end of the unit before: no barrier gets a phase ahead.
      Walk walk(it);
      for (uint32_t i = 0; walk.next(); ++i) {
        const int n = it.tile - __ldg(&it.units[walk.u].x) / BN, rank = MULTI ? p.by_parts.div(n) : n, part = MULTI ? n - rank * p.parts : 0;
        int* turn = p.turns + ((long long)part * p.B * p.Hk + it.bhk) * p.nU + walk.u;
        if (warp == 3) {
          if (rank > 0) turn_wait(turn, rank, abort_flag, p.status);
          if (i > 0) wait(&sm->rows_seen, (i - 1) & 1);
          mbar_arrive(&sm->turn_ok);
        } else {
          wait(&sm->rows_out, i & 1);
          mbar_arrive(&sm->rows_seen);
          turn_pass(turn, rank + 1);
        }
      }
    }
  } else if (warp < 12) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
    // ------------------------------------------------------------------ loaders: the Q rows of the units with their lse (warps
    // 4-7), the dO rows with -rowsum(dO * O) (warps 8-11); they run ahead.  One TMA tile where every row of the unit sees
    // something, else asynchronous 16-byte copies, eight threads per 128-byte half row, with zeros for the rows that do not.
    const bool is_q = warp < 8;
    const int lt = threadIdx.x & 127, r0 = 4 * (warp & 3) + (lane >> 3), chunk = lane & 7;      // rows r0 + 16 k
    const int rt = p.by_G.div(lt), rg = lt - rt * p.G;
    const int2* rows = p.rows + (long long)mask_batch(p.Bm, it.b) * p.Sq;
    Walk walk(it);
    float sc = 0.f;
    int least = 0;                             // smallest end of the unit's ranges (0: a row sees nothing)
    auto fetch = [&]() {
      least = __ldg(&it.units[walk.u].w);
      const int tok = walk.u * p.tpt + rt;
      sc = is_q ? INFINITY : 0.f;                          // rows that see nothing: P = exp2(-inf) = 0
      if (lt < p.tpt * p.G && tok < p.Sq && __ldg(&rows[tok].y) > 0)
        sc = is_q ? __ldg(p.lse + ((long long)it.b * p.Hk * p.G + it.hk * p.G + rg) * p.Sq + tok) * LOG2E
                  : -__ldg(p.Dv + (long long)it.bhk * p.Sq * p.G + (long long)tok * p.G + rg);
    };
    bool more = walk.next();
    if (more) fetch();
    uint32_t slot = 0, par = 1;
    for (uint32_t g = 0; more; ++g) {
      uint64_t* full = is_q ? &sm->q_full[slot] : &sm->do_full;
      // (the first waits pass at once: the parity of the phase before the first)
      wait(is_q ? &sm->q_empty[slot] : &sm->do_empty, par);
      // -rowsum(dO * O) of unit g goes to slot g % 2, which dS^T of unit g - 2 has left behind when dV of unit g - 1, which
      // follows P^T of unit g - 1, has freed the dO tile
      (is_q ? sm->lse2[slot] : sm->negD[g & 1])[lt] = sc;
      const int tok0 = walk.u * p.tpt;
      uint8_t* tile = is_q ? sQ + slot * TILE : sO;
      if (__builtin_expect(least > 0, 1)) {
        if (lt == 0) {
          const CUtensorMap* map = is_q ? &tmQ : &tmO;
          mbar_expect_tx(full, (uint32_t)(p.tpt * p.G * DH * 2));
          tma_load_5d(tile, map, full, 0, 0, tok0, it.hk, it.b);
          tma_load_5d(tile + PANEL, map, full, 64, 0, tok0, it.hk, it.b);
        } else {
          mbar_arrive(full);
        }
        more = walk.next();
        if (more) fetch();
        // drain: every issued load must have landed before the CTA may exit (only matters after a timeout)
        if (lt == 0 && *abort_flag) wait(full, par ^ 1);
      } else {
        const Strides& s = is_q ? p.qs : p.dos;
        const __nv_bfloat16* base = (is_q ? p.q : p.d_o) + it.b * s.b + (long long)it.hk * p.G * s.h + chunk * 8;
        const uint32_t dst = smem_u32(tile) + r0 * 128 + ((chunk ^ (r0 & 7)) << 4);
#pragma unroll 1
        for (int k = 0; k < 8; ++k) {
          const int r = r0 + 16 * k, rk = p.by_G.div(r), tok = tok0 + rk;
          const bool ok = r < p.tpt * p.G && tok < p.Sq && __ldg(&rows[min(tok, p.Sq - 1)].y) > 0;
          const __nv_bfloat16* row = ok ? base + tok * s.t + (r - rk * p.G) * s.h : base;
          cp_async16(dst + k * 2048, row, ok ? 16u : 0u);
          cp_async16(dst + k * 2048 + PANEL, row + 64, ok ? 16u : 0u);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        more = walk.next();
        if (more) fetch();
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        fence_async_proxy();
        mbar_arrive(full);
      }
      if (!is_q) par ^= 1;
      else if (++slot == NQ) { slot = 0; par ^= 1; }
    }
  } else if (warp >= 20) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 80;");
    // ------------------------------------------------------------------ dQ writers: dQ^T of a unit out of TMEM (lane = head-dim
    // index, 128 query columns; two warps per TMEM lane quarter, each taking 64 columns) into the accumulator; see attn_tc_bwd.cu.
    const int quad = warp & 3;
    const int qhalf = (warp - 20) >> 2;
    const uint32_t dq_tmem = tmem + ((uint32_t)(quad * 32) << 16) + DPT_COL + 64 * qhalf;
    float* acc_head = p.dq_acc + quad * 32 + (lane & ~3) + (long long)it.bhk * p.Sq * p.G * DH;
    Walk walk(it);
    for (uint32_t g = 0; walk.next(); ++g) {
      const int rows = unit_rows(p, walk.u), n = it.tile - __ldg(&it.units[walk.u].x) / BN;
      float* acc = acc_head + (long long)walk.u * p.tpt * p.G * DH;
      if constexpr (MULTI) acc += (long long)(n - p.by_parts.div(n) * p.parts) * all_rows * DH;
      wait(&sm->dq_full, g & 1);
      tc_fence_after();
      // everything out of TMEM first: the next dP^T waits for these columns
      uint32_t x[2][32];
      tmem_ld_16x256_x8(dq_tmem, x[0]);
      tmem_ld_16x256_x8(dq_tmem + ROW16, x[1]);
      tmem_ld_wait();
      tc_fence_before();
      mbar_arrive(&sm->dq_free);
      // A reduction holds its source registers until the load/store unit has taken them, so each has its own four.
      auto write_rows = [&](auto put) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int e = 0; e < 2; ++e) {        // query 8 j + 2 (lane % 4) + e of this half
            const int rw = 64 * qhalf + 8 * j + 2 * (lane & 3) + e;
            if (rw < rows)
              put(acc + rw * DH, __uint_as_float(x[0][4 * j + e]) * p.scale, __uint_as_float(x[0][4 * j + 2 + e]) * p.scale,
                  __uint_as_float(x[1][4 * j + e]) * p.scale, __uint_as_float(x[1][4 * j + 2 + e]) * p.scale);
          }
      };
      wait(&sm->turn_ok, g & 1);
      if (n < (MULTI ? p.parts : 1))
        write_rows([](float* to, float a, float b, float c, float d) { *reinterpret_cast<float4*>(to) = make_float4(a, b, c, d); });
      else
        write_rows([](float* to, float a, float b, float c, float d) { red_add_v4(to, a, b, c, d); });
      mbar_arrive(&sm->rows_out);
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 112;");
    // ------------------------------------------------------------------ compute: warp = 32 keys x half of the unit's queries
    const int quad = warp & 3;
    const int half = (warp - 12) >> 2;
    const uint32_t lane_addr = (uint32_t)(quad * 32) << 16;
    const int r = quad * 32 + lane;                // key row of the epilogue
    __nv_bfloat16* dk_row = p.dk + it.b * p.dks.b + (long long)(it.key0 + r) * p.dks.t + it.hk * p.dks.h;
    __nv_bfloat16* dv_row = p.dv + it.b * p.dvs.b + (long long)(it.key0 + r) * p.dvs.t + it.hk * p.dvs.h;
    if (!some) {
      // no query sees these keys: zero gradients
      if (r < it.valid) {
        const uint4 z = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          reinterpret_cast<uint4*>(dk_row)[half * 8 + i] = z;
          reinterpret_cast<uint4*>(dv_row)[half * 8 + i] = z;
        }
      }
    } else {
      const uint32_t st_t = tmem + lane_addr + ST_COL + 64 * half, dp_t = tmem + lane_addr + DPT_COL + 64 * half;
      // this lane's row address for stmatrix: matrices (keys 0-7, queries 8j), (keys 8-15, same), (keys 0-7, 8j + 8), ...
      const int mrow = quad * 32 + 8 * ((lane >> 3) & 1) + (lane & 7), mj = lane >> 4;
      const uint32_t ds_row = smem_u32(sDS) + half * PANEL + mrow * 128;
      const int key = quad * 32 + (lane >> 2);
      const int2* rows = p.rows + (long long)mask_batch(p.Bm, it.b) * p.Sq;
      uint32_t slot = 0, par = 0;                  // of the Q ring
      Walk walk(it);
      for (uint32_t g = 0; walk.next(); ++g) {
        const float2* lse2 = reinterpret_cast<const float2*>(sm->lse2[slot] + 64 * half) + (lane & 3);
        const float2* negD = reinterpret_cast<const float2*>(sm->negD[g & 1] + 64 * half) + (lane & 3);
        // What the unit's queries see of the tile.  Mostly all of it, or all the same keys of it ([lo, hi): a clip's or a frame's end):
        // then a thread masks by its four keys.  Else (apart) bounds: bytes {lo, hi} of queries 2 lane and 2 lane + 1 of this half.
        // (Every unit of a clip that begins inside a tile is masked there, and the clip's other tiles add dQ behind that one: with
        // bounds read and compared for each of them 13K tokens of two clips, capped, took 1406 us, so 1335.  The record brought by
        // the loaders, through shared memory: 1345, and 5 % more where nothing is masked.)
        const bool masked = walk.u < it.run.y || walk.u >= it.run.z, stale = CAP && unit_rows(p, walk.u) <= QU - 16;
        bool apart = stale;
        int lo = 0, hi = BN;
        if (__builtin_expect(masked, 0)) {
          const int4 u = __ldg(it.units + walk.u);
          auto rel = [&](int v) { return min(max(v - it.key0, 0), BN); };
          lo = rel(u.x);
          hi = rel(u.w);
          apart = apart || lo != rel(u.z) || hi != rel(u.y);
        }
        uint32_t bounds = 0;
        if (__builtin_expect(apart, 0)) {
#pragma unroll 1
          for (int e = 0; e < 2; ++e) {
            const int rw = 64 * half + 2 * lane + e, tok = walk.u * p.tpt + p.by_G.div(rw);
            if (rw < p.tpt * p.G && tok < p.Sq) {
              const int2 s = __ldg(rows + tok);
              bounds |= (uint32_t)(min(max(s.x - it.key0, 0), BN) | min(max(s.y - it.key0, 0), BN) << 8) << (16 * e);
            }
          }
        }
        wait(&sm->q_full[slot], par);                  // publishes lse2 of this unit
        if (++slot == NQ) { slot = 0; par ^= 1; }
        float2 l[8];                                   // (fetched before the wait: next to a busy tensor pipe a load takes its time)
#pragma unroll
        for (int j = 0; j < 8; ++j) l[j] = lse2[4 * j];
        wait(&sm->s_full, g & 1);
        tc_fence_after();
        // ---- P^T: thread holds keys key + 8 r (r = 0 .. 3) x queries 8 j + 2 (lane % 4) + {0, 1} of the half
        uint32_t pv[2][32];
        tmem_ld_16x256_x8(st_t, pv[0]);
        tmem_ld_16x256_x8(st_t + ROW16, pv[1]);
        tmem_ld_wait();
        // scores outside their query's range get a value
        auto mask = [&](uint32_t value) {
          if (apart) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const uint32_t w = __shfl_sync(0xffffffffu, bounds, 4 * j + (lane & 3));
#pragma unroll
              for (int e = 0; e < 2; ++e) {          // query e of the pair
                const int from = w >> (16 * e) & 0xff, n = (int)(w >> (16 * e + 8) & 0xff) - from, at = key - from;
#pragma unroll
                for (int k = 0; k < 4; ++k)          // key + 8 k
                  if ((unsigned)(at + 8 * k) >= (unsigned)n) pv[k >> 1][4 * j + 2 * (k & 1) + e] = value;
              }
            }
          } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const bool out = key + 8 * k < lo || key + 8 * k >= hi;
#pragma unroll
              for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                  if (out) pv[k >> 1][4 * j + 2 * (k & 1) + e] = value;
            }
          }
        };
        // (the rare cases' code is out of the way and short: beside the other roles' it does not fit the instruction cache)
        if constexpr (CAP) {
          // scores -> tanh (1 exactly where it is 1 to fp32, so that the slope is 0).  What no product has written (queries beyond the unit's)
          // has no say in how the others are capped
          if (__builtin_expect(stale, 0)) mask(0u);
          float m0 = 0.f, m1 = 0.f;
#pragma unroll
          for (int i = 0; i < 32; i += 2) {
            m0 = max3(m0, fabsf(__uint_as_float(pv[0][i])), fabsf(__uint_as_float(pv[0][i + 1])));
            m1 = max3(m1, fabsf(__uint_as_float(pv[1][i])), fabsf(__uint_as_float(pv[1][i + 1])));
          }
          if (__builtin_expect(__all_sync(0xffffffffu, fmaxf(m0, m1) <= p.cap.most), 1)) {
#pragma unroll
            for (int rh = 0; rh < 2; ++rh)
#pragma unroll
              for (int i = 0; i < 32; i += 2) {
                float x0 = __uint_as_float(pv[rh][i]), x1 = __uint_as_float(pv[rh][i + 1]), z0, z1, r0 = p.cap.u[4], r1 = p.cap.u[4];
                mul2(z0, z1, x0, x1, x0, x1);
#pragma unroll
                for (int k = 3; k >= 0; --k) fma2(r0, r1, r0, r1, z0, z1, p.cap.u[k], p.cap.u[k]);
                mul2(x0, x1, r0, r1, x0, x1);
                pv[rh][i] = __float_as_uint(x0);
                pv[rh][i + 1] = __float_as_uint(x1);
              }
          } else if (p.cap_apart > 0.0f) {           // (larger caps: score by score, as in the forward)
#pragma unroll
            for (int rh = 0; rh < 2; ++rh)
#pragma unroll
              for (int i = 0; i < 32; ++i) {
                const float x = __uint_as_float(pv[rh][i]) * p.cap.pre, z = x * x;
                const float near = x * fmaf(fmaf(fmaf(fmaf(p.cap.u[4], z, p.cap.u[3]), z, p.cap.u[2]), z, p.cap.u[1]), z, p.cap.u[0]);
                const float far = fmaf(rcp(1.0f + ex2(x * p.cap.twice_log2)), -2.0f, 1.0f);
                pv[rh][i] = __float_as_uint(fabsf(x) <= p.cap_apart ? near : far);
              }
          } else {
#pragma unroll
            for (int rh = 0; rh < 2; ++rh)
#pragma unroll
              for (int i = 0; i < 32; ++i)
                pv[rh][i] = __float_as_uint(fmaf(rcp(1.0f + ex2(__uint_as_float(pv[rh][i]) * p.cap.twice_log2)), -2.0f, 1.0f));
          }
          if (__builtin_expect(masked || stale, 0)) mask(__float_as_uint(p.cap_masked));
        } else {
          if (__builtin_expect(masked, 0)) mask(0xff800000u);
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          uint32_t pk[2][8];
#pragma unroll
          for (int jj = 0; jj < 4; ++jj) {
            const int j = 4 * c + jj;
#pragma unroll
            for (int rh = 0; rh < 2; ++rh)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                float x0 = __uint_as_float(pv[rh][4 * j + 2 * e]), x1 = __uint_as_float(pv[rh][4 * j + 2 * e + 1]), s0, s1;
                if constexpr (CAP) {                 // the slope
                  mul2(s0, s1, x0, x1, x0, x1);
                  fma2(s0, s1, s0, s1, -1.0f, -1.0f, 1.0f, 1.0f);
                }
                fma2(x0, x1, x0, x1, p.to_exp2, p.to_exp2, -l[j].x, -l[j].y);
                x0 = ex2(x0);
                x1 = ex2(x1);
                pk[rh][2 * jj + e] = pack_bf16(x0, x1);
                if constexpr (CAP) mul2(x0, x1, x0, x1, s0, s1);
                pv[rh][4 * j + 2 * e] = __float_as_uint(x0);
                pv[rh][4 * j + 2 * e + 1] = __float_as_uint(x1);
              }
          }
          tmem_st_16x128_x4(st_t + 16 * c, pk[0]);
          tmem_st_16x128_x4(st_t + ROW16 + 16 * c, pk[1]);
        }
        // negD of this unit (dV needs the dO rows anyway; asked before dV can run, so that the barrier cannot be a phase ahead)
        wait(&sm->do_full, g & 1);
        tmem_st_wait();
        tc_fence_before();
        mbar_arrive(&sm->p_ready);
        // ---- dS^T = P^T (dP^T - D).  The dS^T tile in shared memory is free: dP^T was issued behind the dQ^T that read it.
        float2 d[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) d[j] = negD[4 * j];
        wait(&sm->dp_full, g & 1);
        tc_fence_after();
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          uint32_t dp[2][16];
          tmem_ld_16x256_x4(dp_t + 32 * c, dp[0]);
          tmem_ld_16x256_x4(dp_t + ROW16 + 32 * c, dp[1]);
          tmem_ld_wait();
#pragma unroll
          for (int rh = 0; rh < 2; ++rh) {
            uint32_t dk_[8];
#pragma unroll
            for (int jj = 0; jj < 4; ++jj) {
              const int j = 4 * c + jj;
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const int at = key + 16 * rh + 8 * e;
                float x0, x1;
                add2(x0, x1, __uint_as_float(dp[rh][4 * jj + 2 * e]), __uint_as_float(dp[rh][4 * jj + 2 * e + 1]), d[j].x, d[j].y);
                mul2(x0, x1, x0, x1, __uint_as_float(pv[rh][4 * j + 2 * e]), __uint_as_float(pv[rh][4 * j + 2 * e + 1]));
                // (a key that nobody sees: its V row may hold anything)
                dk_[2 * jj + e] = at >= it.info.z && at < it.info.w ? pack_bf16(x0, x1) : 0u;
              }
            }
            tmem_st_16x128_x4(dp_t + rh * ROW16 + 16 * c, dk_);
#pragma unroll
            for (int m = 0; m < 2; ++m)
              stmatrix_x4(ds_row + rh * 16 * 128 + (((4 * c + 2 * m + mj) ^ (lane & 7)) << 4), dk_[4 * m], dk_[4 * m + 1], dk_[4 * m + 2],
                          dk_[4 * m + 3]);
          }
        }
        fence_async_proxy();
        tmem_st_wait();
        tc_fence_before();
        mbar_arrive(&sm->ds_ready);
      }
      // ---- epilogue: thread = key row; each half writes 64 of its 128 dV / dK columns
      wait(&sm->acc_done, 0);
      tc_fence_after();
#pragma unroll 1
      for (int pass = 0; pass < 4; ++pass) {      // dV columns, then dK columns, 32 at a time
        const int cgrp = half * 2 + (pass & 1);
        const bool is_dk = pass >= 2;
        uint32_t a[32];
        tmem_ld32(tmem + lane_addr + (is_dk ? DK_COL : DV_COL) + cgrp * 32, a);
        tmem_ld_wait();
        if (r < it.valid) {
          const float mul = is_dk ? p.scale : 1.0f;
          __nv_bfloat16* row = (is_dk ? dk_row : dv_row) + cgrp * 32;
#pragma unroll
          for (int i = 0; i < 32; i += 16) {      // sixteen bf16 = one 32-byte store (two 16-byte stores if unaligned)
            uint32_t hv[8];
#pragma unroll
            for (int k = 0; k < 8; ++k)
              hv[k] = pack_bf16(__uint_as_float(a[i + 2 * k]) * mul, __uint_as_float(a[i + 2 * k + 1]) * mul);
            if (p.dkv_32) {
              st_global_v8(row + i, hv[0], hv[1], hv[2], hv[3], hv[4], hv[5], hv[6], hv[7]);
            } else {
              *reinterpret_cast<uint4*>(row + i) = make_uint4(hv[0], hv[1], hv[2], hv[3]);
              *reinterpret_cast<uint4*>(row + i + 8) = make_uint4(hv[4], hv[5], hv[6], hv[7]);
            }
          }
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) tmem_dealloc(tmem, TMEM_COLS);
}

// The accumulators of dQ, added up in order, as bf16 rows of dq; rows that see nothing are zero.
__global__ void __launch_bounds__(256)
range_cast_kernel(const Params p, __nv_bfloat16* __restrict__ dq, const Strides dqs) {
  if (!grid_begin()) return;
  constexpr int R = 4;                         // rows of a warp whose loads are in flight together
  const int lane = threadIdx.x & 31;
  // this lane's output columns 4 lane .. 4 lane + 3 sit at positions at, at + 4, at + 8, at + 12: one line of the row
  const int at = (lane & ~7) * 4 + 16 * (lane & 1) + ((lane & 7) >> 1);
  const int per = p.Sq * p.G;
  const int all_rows = p.B * p.Hk * per;       // (at most 2^30)
  for (int row0 = (blockIdx.x * 8 + (threadIdx.x >> 5)) * R; row0 < all_rows; row0 += gridDim.x * 8 * R) {
    float4 v[R];
    long long to[R];
    int parts[R];
    int most = 0;
#pragma unroll
    for (int n = 0; n < R; ++n) {
      const int row = min(row0 + n, all_rows - 1), bhk = p.by_rows.div(row), r = row - bhk * per, tok = p.by_G.div(r), g = r - tok * p.G;
      const int b = p.by_Hk.div(bhk), hk = bhk - b * p.Hk, bm = mask_batch(p.Bm, b);
      to[n] = b * dqs.b + tok * dqs.t + (long long)(hk * p.G + g) * dqs.h + lane * 4;
      const int4 u = __ldg(p.units + (long long)bm * p.nU + p.by_tpt.div(tok));
      const int seen = __ldg(&p.rows[(long long)bm * p.Sq + tok].y);
      const float* from = p.dq_acc + (long long)row * DH + at;      // (read ahead of the answer whether the row has any)
      v[n] = make_float4(__ldg(from), __ldg(from + 4), __ldg(from + 8), __ldg(from + 12));
      parts[n] = seen > 0 ? min(p.parts, (u.y + BN - 1) / BN - u.x / BN) : 0;
      most = max(most, parts[n]);
      if (parts[n] == 0) v[n] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    for (int k = 1; k < most; ++k) {
#pragma unroll
      for (int n = 0; n < R; ++n)
        if (k < parts[n]) {
          const float* from = p.dq_acc + ((long long)k * all_rows + min(row0 + n, all_rows - 1)) * DH + at;
          v[n].x += __ldg(from); v[n].y += __ldg(from + 4); v[n].z += __ldg(from + 8); v[n].w += __ldg(from + 12);
        }
    }
#pragma unroll
    for (int n = 0; n < R; ++n)
      if (row0 + n < all_rows) store4(dq + to[n], v[n]);
  }
}

}  // namespace tcb

int tc_range_bwd_parts(const RDims& D) {
  const long long acc = (long long)D.B * D.Hk * D.rows * D.d * (long long)sizeof(float);
  return (int)std::max<long long>(1, std::min<long long>(std::min(4, D.nK), (128ll << 20) / acc));
}
long long tc_range_bwd_turns(const RDims& D) { return (long long)tc_range_bwd_parts(D) * D.B * D.Hk * D.nU + 1; }

int tc_range_bwd(const RDims& D, const Plan& plan, const BwdArgs& a, void* dq, const Strides& dqs, bool early, cudaStream_t st) {
  using namespace tcb;
  const long long items = (long long)D.B * D.Hk * D.nK;
  if (items > (long long)INT32_MAX - 4096) return VMOBA_ERR_SHAPE;
  Params p;
  p.B = D.B; p.Hk = D.Hk; p.G = D.G; p.Sq = D.Sq; p.Sk = D.Sk; p.Bm = D.Bm; p.tpt = D.tpt; p.nU = D.nU; p.nK = D.nK;
  p.rows = plan.rows; p.units = plan.units; p.keys = plan.keys; p.runs = plan.runs;
  p.by_G = FastDiv(D.G); p.by_tpt = FastDiv(D.tpt); p.by_rows = FastDiv(D.rows); p.by_Hk = FastDiv(D.Hk); p.by_parts = FastDiv(a.parts);
  p.q = (const __nv_bfloat16*)a.q; p.d_o = (const __nv_bfloat16*)a.d_o; p.qs = a.qs; p.dos = a.dos;
  p.lse = a.lse; p.Dv = a.Dv;
  p.scale = D.scale;
  p.cap = make_cap(D);
  p.to_exp2 = D.cap > 0.f ? p.cap.c : D.scale * LOG2E;
  p.cap_apart = p.cap.pre != 1.0f || p.cap.c > CAP_MOST ? p.cap.most : 0.f;
  if (p.cap.pre != 1.0f) p.cap.most = -1.0f;      // (the vote never finds for the polynomial: its scores have not been multiplied)
  // lse2 is -c' at least, so that -2 c' - 256 is a weight of 0, and its slope 1 - (2 + 256 / c')^2, of c' = 10^-9 at least
  p.cap_masked = D.cap > 0.f ? -2.0f - 256.0f / p.cap.c : 0.f;
  p.dk = (__nv_bfloat16*)a.dk; p.dv = (__nv_bfloat16*)a.dv; p.dks = a.dks; p.dvs = a.dvs;
  auto whole = [](const void* x, const Strides& s) {
    return reinterpret_cast<uintptr_t>(x) % 32 == 0 && s.b % 16 == 0 && s.t % 16 == 0 && s.h % 16 == 0;
  };
  p.dkv_32 = whole(a.dk, a.dks) && whole(a.dv, a.dvs);
  p.dq_acc = a.dq_acc; p.parts = a.parts; p.turns = a.turns; p.status = a.status;
  // Sixteen heads: their accumulators, Q and dO pass through the L2 once per SMs / 16 key tiles.  More where a head has so few
  // units that its tiles would come too slowly for the SMs.
  p.group = std::min(D.B * D.Hk, std::max(16, sm_count() / D.nU));
  CUtensorMap tmK, tmV, tmQ, tmO;
  if (!make_tmap_keys(&tmK, a.k, D, a.ks) || !make_tmap_keys(&tmV, a.v, D, a.vs) || !make_tmap_units(&tmQ, a.q, D, a.qs) ||
      !make_tmap_units(&tmO, a.d_o, D, a.dos))
    return VMOBA_ERR_CUDA;
  auto kernel = D.cap > 0.f ? (a.parts > 1 ? attn_range_bwd_kernel<true, true> : attn_range_bwd_kernel<true, false>)
                            : (a.parts > 1 ? attn_range_bwd_kernel<false, true> : attn_range_bwd_kernel<false, false>);
  VMOBA_CUDA_OK(allow_smem(kernel, (int)SMEM_BYTES));
  launch_kernel(early, kernel, (unsigned)items, THREADS, SMEM_BYTES, st, tmK, tmV, tmQ, tmO, p);
  const long long all_rows = (long long)D.B * D.Hk * D.rows;
  launch_kernel(early, range_cast_kernel, (unsigned)std::max<long long>(1, std::min<long long>((all_rows + 31) / 32, sm_count() * 16)), 256, 0, st,
                p, (__nv_bfloat16*)dq, dqs);
  VMOBA_LAUNCH_OK(2);
  return VMOBA_OK;
}

}  // namespace range
}  // namespace vmoba
