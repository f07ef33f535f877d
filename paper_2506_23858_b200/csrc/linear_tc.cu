// Matrix products on the tensor cores: bf16 operands, fp32 sums.
//
// Two CTAs of a cluster work on one tile of 256 x 256 sums: each holds 128 of its rows (its half of the accumulator in its own TMEM) and brings
// 128 rows and 128 columns of the operands, 64 summed indices at a time, into its shared memory; one thread of the pair issues the
// products of both (tcgen05.mma, cta_group::2).  Every byte loaded is used for 256 products, which is what L2 can feed: a lone CTA with a
// 128 x 256 tile asks it for half as much again.  Two accumulators alternate, so that eight warps finish one tile while the next
// is summed.  An operand whose summed index runs along its rows is read as it lies (MN-major tiles), so that no gradient needs a transpose.
// gated: the pair's columns are 128 of the gate (first CTA's half) and 128 of the factor.
// Where tiles would leave SMs idle, the summed index is cut into slices, whose sums a second kernel adds in a fixed order.
// Bound by the tensor pipe and, in long calls, the power limit: 32,760 tokens, 1,536 -> 4,608 channels 361 us (1.29 PFLOP/s; a launch on its own 291,
// the pipe 94 % busy); 5,120 -> 20,480 -> 5,120 10.5 ms (1.31); gradient of a weight of 8,208 x 1,536 over 13,440 tokens, on its own, 232 us (1.46).
#include <algorithm>

#include "linear.cuh"

namespace vmoba {
namespace linear {
namespace tc {

using namespace sm100;

constexpr int BM = 128, BN = 256, BK = 64;   // per CTA: rows of the accumulator; columns; summed indices of a stage
constexpr int MOST_STAGES = 5;               // four where results leave by rows, whose residual needs the room (no slower)
constexpr int HALF = 128 * BK * 2;           // bytes of one operand's half of a stage
constexpr int PANEL = 64 * 128;              // MN-major: 64 places of the tile x 64 summed indices
constexpr int THREADS = 384, EPI_WARPS = 8;
constexpr int STAGE_W = 64;                  // columns that a warp turns around in shared memory at a time

struct Args {
  Epilogue e;
  int Sm, rows_tiles, row_tiles, col_tiles;  // rows of a sample; tiles of rows per sample and of all; tiles of columns
  int N;                                     // columns of out
  int steps, items;                          // stages of the summed index; tiles and slices of tiles
  int whole, rest, per, splits;              // tiles worked out at once; the other ones, stages of their slices, slices of each
  int a_inner, b_inner, b_samples;           // columns of a head; samples of b (those of a come twice, if it has two planes)
  int step_inner;                            // stages per sample (kColsCols), per plane
  FastDiv by_rows_tiles, by_rest, by_group, by_a_inner, by_b_inner, by_step, by_wide;
  float* part;                               // [slice of a tile][256 rows][256 columns]
  int wide;                                  // columns of the sums
  int32_t* status;
};
constexpr long long PART = 2ll * BM * BN;    // floats of a slice of a tile
constexpr int TO_PART = 4;                   // floats at most from a 16-byte boundary, on which scratch begins, to a 32-byte one, as store_part has to have

struct Shared {
  uint64_t full[MOST_STAGES], empty[MOST_STAGES], acc_full[2], acc_empty[2], ahead[EPI_WARPS], drain;
  uint32_t tmem;
  int abort;
};
constexpr int STAGE_BYTES = 2 * HALF;
constexpr int TURN_BYTES = 32 * STAGE_W * 4;
constexpr int AHEAD_BYTES = 32 * STAGE_W * 2; // a warp's residual of the box to come
// How results leave: boxes written by TMA; rows of lanes where gate, residual or another order of the rows are in play; boxes that
// came by TMA where they are the slopes of an activation.
enum Store { kBoxes = 0, kRows = 1, kSlopes = 2 };
__host__ __device__ constexpr int stages_of(int store) { return store == kBoxes ? MOST_STAGES : MOST_STAGES - 1; }
__host__ __device__ constexpr int smem_of(int store) {
  return 1024 + stages_of(store) * STAGE_BYTES + EPI_WARPS * (TURN_BYTES + (store != kBoxes ? AHEAD_BYTES : 0)) + (int)sizeof(Shared);
}
static_assert(smem_of(kBoxes) <= 227 * 1024 && smem_of(kRows) <= 227 * 1024, "shared memory of a CTA");

__device__ __forceinline__ uint32_t cta_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_meet() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The address of the first CTA's barrier.
__device__ __forceinline__ uint32_t first_cta(const uint64_t* bar) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(smem_u32(bar)));
  return r;
}
// (What it says is that TMEM has been read, which tcgen05.wait::ld has seen to: no wider scope than the CTA's, whose release would wait for the
// thread's loads and stores under way.)
__device__ __forceinline__ void arrive_at(uint32_t cluster_bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
// Into this CTA's shared memory, completion counted by a barrier of either CTA.
__device__ __forceinline__ void pair_load_4d(uint32_t dst, const CUtensorMap* map, uint32_t cluster_bar, int x, int y, int z, int w) {
  asm volatile(
      "cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(cluster_bar), "r"(x), "r"(y), "r"(z), "r"(w)
      : "memory");
}
__device__ __forceinline__ void pair_mma(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
      "mov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(DESC_HI_SW128)
      : "memory");
}
__device__ __forceinline__ void tma_store_4d(const CUtensorMap* map, const void* smem_src, int x, int y, int z, int w) {
  asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.bulk_group [%0, {%2, %3, %4, %5}], [%1];" ::"l"(reinterpret_cast<uint64_t>(map)),
               "r"(smem_u32(smem_src)), "r"(x), "r"(y), "r"(z), "r"(w)
               : "memory");
}
// Arrives at the barriers of both CTAs when all products issued so far are done.
__device__ __forceinline__ void pair_commit(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)),
               "h"((uint16_t)3)
               : "memory");
}

// u += eight packed bf16
__device__ __forceinline__ void add_bf16x8(float (&u)[8], const uint4& v) {
  add_bf16_pair(u[0], u[1], v.x);
  add_bf16_pair(u[2], u[3], v.y);
  add_bf16_pair(u[4], u[5], v.z);
  add_bf16_pair(u[6], u[7], v.w);
}

// Sums over the warp's lanes of 32 numbers each: lane k gets that of x[k].  Half of what is left goes to the other half of the lanes at each step.
__device__ __forceinline__ float column_sum(float* x) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const bool high = lane & o;
#pragma unroll
    for (int k = 0; k < o; ++k) {
      const float keep = high ? x[k + o] : x[k], give = high ? x[k] : x[k + o];
      x[k] = keep + __shfl_xor_sync(0xffffffffu, give, o);
    }
  }
  return x[0];
}

struct Item {
  int slice, k0, k1;                         // -1: a whole tile; its stages
  int sample, row, col;                      // first row of the pair's tile in the sample; first column of out
};
// Tiles in groups of eight tiles of rows, down the rows first: the tiles that run at a time share rows and columns.
template <int KIND>
__device__ __forceinline__ Item item_of(const Args& p, int i) {
  constexpr int G = 8, COLS = KIND == kGated ? BN / 2 : BN;
  int t = i, slice = -1, k0 = 0, k1 = p.steps;
  if (i >= p.whole) {                        // slice after slice of the last tiles
    slice = i - p.whole;
    const int s = p.by_rest.div(slice);
    t = i - s * p.rest;
    k0 = s * p.per;
    k1 = min(k0 + p.per, p.steps);
  }
  const int group = p.by_group.div(t);       // (by G * col_tiles)
  t -= group * G * p.col_tiles;
  const int high = min(G, p.row_tiles - group * G);
  const int col = t / high, rt = group * G + t - col * high;
  const int sample = p.by_rows_tiles.div(rt);
  return {slice, k0, k1, sample, (rt - sample * p.rows_tiles) * 2 * BM, col * COLS};
}

// Columns of the sums that a tile works out: 256, fewer in the last tile of columns, by 64 (4,104 columns: 16 tiles and a quarter, not 17).
// Where columns are channels of heads (kColsCols), a box of 64 ends with the head that it begins in, and half of 192 columns begins in the middle
// of a head: all 256 there.  (Half of 64 begins there too, but needs no more than the box has.)
template <int FORM, int KIND>
__device__ __forceinline__ int columns_of(const Args& p, const Item& it) {
  if (KIND == kGated) return BN;
  const int cols = min(BN, (p.N - it.col + 63) & ~63);
  return FORM == kColsCols && cols == 192 && p.b_inner < p.N ? BN : cols;
}

// A warp's half of the columns of a slice of a tile, as they are; lane = row.
__device__ __forceinline__ void store_part(uint32_t tmem, float* to) {
#pragma unroll 1
  for (int c = 0; c < BN / 2; c += 32) {
    uint32_t v[32];
    tmem_ld32(tmem + c, v);
    tmem_ld_wait();
#pragma unroll
    for (int j = 0; j < 32; j += 8) st_global_v8(static_cast<void*>(to + c + j), v[j], v[j + 1], v[j + 2], v[j + 3], v[j + 4], v[j + 5], v[j + 6], v[j + 7]);
  }
}

template <int FORM, int KIND, int STORE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(THREADS, 1)
    pair_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ CUtensorMap tmOut,
                const __grid_constant__ CUtensorMap tmOut2, const __grid_constant__ CUtensorMap tmKept, const __grid_constant__ CUtensorMap tmKept2,
                const __grid_constant__ CUtensorMap tmAgain, Args p) {
  if (!grid_begin()) return;
  constexpr bool A_MN = FORM == kColsCols, B_MN = FORM != kRowsRows;
  constexpr int STAGES = stages_of(STORE);
  extern __shared__ char smem_raw[];
  char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  char* turn = smem + STAGES * STAGE_BYTES;
  char* ahead = turn + EPI_WARPS * TURN_BYTES;
  Shared* sm = reinterpret_cast<Shared*>(ahead + (STORE != kBoxes ? EPI_WARPS * AHEAD_BYTES : 0));
  volatile int* abort_flag = &sm->abort;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cta_rank();
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;

  if (warp == 0 && lane == 0) {
    for (int i = 0; i < STAGES; ++i) { mbar_init(&sm->full[i], 1); mbar_init(&sm->empty[i], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&sm->acc_full[i], 1); mbar_init(&sm->acc_empty[i], 2 * EPI_WARPS); }
    for (int i = 0; i < EPI_WARPS; ++i) mbar_init(&sm->ahead[i], 1);
    mbar_init(&sm->drain, 1);
    sm->abort = 0;
    fence_barrier_init();
    prefetch_tmap(&tmA);
    prefetch_tmap(&tmB);
  }
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sm->tmem)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_meet();
  tc_fence_after();
  const uint32_t tmem = sm->tmem;

  if (warp == 0) {
    // ------------------------------------------------------------------ loads of this CTA's halves
    if (lane == 0) {
      uint32_t slot = 0, par = 1, n = 0;     // (the first pass through the ring waits for nothing)
      for (int i = pair; i < p.items && !*abort_flag; i += pairs) {
        const Item it = item_of<KIND>(p, i);
        const int row = it.row + (int)rank * BM;
        // (the second CTA has the other half of the tile's columns, of the factor's where gated)
        const int col = KIND == kGated ? it.col + (int)rank * p.N : it.col + (int)rank * (columns_of<FORM, KIND>(p, it) / 2);
        for (int k = it.k0; k < it.k1; ++k) {
          if (!mbar_wait(&sm->empty[slot], par, abort_flag, p.status)) break;
          const uint32_t a = smem_u32(smem) + slot * STAGE_BYTES, b = a + HALF, bar = first_cta(&sm->full[slot]);
          if (rank == 0) mbar_expect_tx(&sm->full[slot], 2 * STAGE_BYTES);
          const int kb = p.by_step.div(k), ks = (k - kb * p.step_inner) * BK;      // sample or plane, and first index in it
          if (A_MN) {
            for (int h = 0; h < 2; ++h) {
              const int m = row + 64 * h, z = p.by_a_inner.div(m);
              pair_load_4d(a + h * PANEL, &tmA, bar, m - z * p.a_inner, ks, z, kb);
            }
          } else {
            const int z = p.by_a_inner.div(ks);
            pair_load_4d(a, &tmA, bar, ks - z * p.a_inner, row, z + kb, it.sample);
          }
          if (B_MN) {
            for (int h = 0; h < 2; ++h) {
              const int c = col + 64 * h, z = p.by_b_inner.div(c);
              pair_load_4d(b + h * PANEL, &tmB, bar, c - z * p.b_inner, ks, z, A_MN ? (kb < p.b_samples ? kb : kb - p.b_samples) : 0);
            }
          } else {
            pair_load_4d(b, &tmB, bar, ks, col, 0, 0);
          }
          ++n;
          if (++slot == STAGES) { slot = 0; par ^= 1; }
        }
      }
      // Every product that reads this CTA's stages has run, and the arrivals that say so have landed, before the CTA may exit; after
      // a time-out at least every load has landed (the first CTA's barriers count those of both).
      for (uint32_t i = 0; i < STAGES && i < n; ++i) {
        const uint32_t s = (slot + STAGES - 1 - i) % STAGES, use = (n - 1 - i) / STAGES;
        if (*abort_flag && rank == 0) mbar_wait(&sm->full[s], use & 1, abort_flag, p.status);
        mbar_wait(&sm->empty[s], use & 1, abort_flag, p.status);
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ products of the pair (the whole warp walks the loop, one lane issues)
    if (rank == 0) {
      const bool leader = elect_one();
      const uint32_t a_lo = desc_lo(smem_u32(smem), A_MN ? PANEL : 16), b_lo = desc_lo(smem_u32(smem) + HALF, B_MN ? PANEL : 16);
      uint32_t slot = 0, par = 0, n = 0;
      const int items = __reduce_max_sync(0xffffffffu, p.items);
      for (int i = pair; i < items; i += pairs, ++n) {
        const Item it = item_of<KIND>(p, i);
        const int k0 = it.k0, k1 = __reduce_max_sync(0xffffffffu, it.k1);
        const uint32_t acc = tmem + (n & 1) * BN;
        const uint32_t idesc = __reduce_max_sync(0xffffffffu, make_idesc_bf16(2 * BM, columns_of<FORM, KIND>(p, it), A_MN, B_MN));
        mbar_wait_warp(&sm->acc_empty[n & 1], ((n >> 1) & 1) ^ 1, abort_flag, p.status);
        tc_fence_after();
        for (int k = k0; k < k1; ++k) {
          mbar_wait_warp(&sm->full[slot], par, abort_flag, p.status);
          tc_fence_after();
          const uint32_t at = slot * (STAGE_BYTES >> 4);
#pragma unroll
          for (int s = 0; s < BK / 16; ++s)      // sixteen summed indices: 32 bytes of a row, or sixteen rows of 128 bytes
            if (leader) pair_mma(acc, a_lo + at + s * (A_MN ? 128 : 2), b_lo + at + s * (B_MN ? 128 : 2), idesc, k > k0 || s > 0 ? 1u : 0u);
          if (leader) pair_commit(&sm->empty[slot]);
          if (++slot == STAGES) { slot = 0; par ^= 1; }
        }
        if (leader) pair_commit(&sm->acc_full[n & 1]);
        if (*abort_flag) break;
      }
      if (leader && *abort_flag) {           // (nothing is under way when the pair frees its TMEM)
        pair_commit(&sm->drain);
        for (uint32_t i = 0; i < (1u << 16); ++i)
          if (mbar_try_wait(&sm->drain, 0)) break;
      }
    }
  }
  // What warps 4 to 11 do with slices of tiles, of which a pair has its last items.
  auto slices = [&](int i, uint32_t n) {
    const int quad = warp & 3, half = (warp - 4) >> 2;
    for (; i < p.items; i += pairs, ++n) {
      const Item it = item_of<KIND>(p, i);
      mbar_wait_warp(&sm->acc_full[n & 1], (n >> 1) & 1, abort_flag, p.status);
      tc_fence_after();
      store_part(tmem + ((uint32_t)(quad * 32) << 16) + (n & 1) * BN + half * (BN / 2),
                 p.part + it.slice * PART + ((int)rank * BM + quad * 32 + lane) * BN + half * (BN / 2));
      tc_fence_before();
      __syncwarp();
      if (lane == 0) arrive_at(first_cta(&sm->acc_empty[n & 1]));
    }
  };
  if (warp >= 4 && STORE == kBoxes) {
    // ------------------------------------------------------------------ sums to results, box by box: lane = row
    const int quad = warp & 3, half = (warp - 4) >> 2;
    const uint32_t lanes = tmem + ((uint32_t)(quad * 32) << 16);
    char* const mine = turn + (warp - 4) * TURN_BYTES;
    const Epilogue& e = p.e;
    constexpr int W = KIND == kGated ? 32 : 64, BOXES = 2;             // columns of a box; boxes of out per warp
    constexpr int COLS = KIND == kGated ? BN / 2 : BN;
    uint32_t n = 0, turns = 0;
    int i = pair;
    for (; i < p.whole; i += pairs, ++n) {
      const Item it = item_of<KIND>(p, i);
      const int row = it.row + (int)rank * BM + quad * 32;             // first row of the warp in the sample
      mbar_wait_warp(&sm->acc_full[n & 1], (n >> 1) & 1, abort_flag, p.status);
      tc_fence_after();
      // W numbers of the lane's row, packed, out through one of two buffers
      auto emit = [&](const CUtensorMap* map, int inner, const FastDiv& by_inner, const float (&u)[W], int c) {
        char* const buf = mine + (turns++ & 1) * (32 * 2 * W);
        if (lane == 0) bulk_wait_group_read<1>();                      // (of the two stores before this one the first has been read)
        __syncwarp();
#pragma unroll
        for (int j = 0; j < W / 8; ++j) {
          const int place = W == 64 ? j ^ (lane & 7) : j ^ ((lane >> 1) & 3);
          *reinterpret_cast<uint4*>(buf + lane * (2 * W) + place * 16) =
              make_uint4(pack_bf16(u[8 * j], u[8 * j + 1]), pack_bf16(u[8 * j + 2], u[8 * j + 3]), pack_bf16(u[8 * j + 4], u[8 * j + 5]),
                         pack_bf16(u[8 * j + 6], u[8 * j + 7]));
        }
        fence_async_proxy();
        __syncwarp();
        if (lane == 0) {
          if (row < p.Sm) {
            const int z = by_inner.div(c);
            tma_store_4d(map, buf, c - z * inner, row, z, it.sample);
          }
          bulk_commit_group();
        }
      };
#pragma unroll
      for (int ch = 0; ch < BOXES; ++ch) {
        const int at = half * (COLS / 2) + ch * W, c = it.col + at;
        if (c >= p.N) {                      // (uniform)
          if (ch == BOXES - 1) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive_at(first_cta(&sm->acc_empty[n & 1]));
          }
          continue;
        }
        uint32_t v[64];
        const uint32_t from = lanes + (n & 1) * BN + at;
        tmem_ld32(from, *reinterpret_cast<uint32_t(*)[32]>(&v[0]));
        tmem_ld32(KIND == kGated ? from + BN / 2 : from + 32, *reinterpret_cast<uint32_t(*)[32]>(&v[32]));
        tmem_ld_wait();
        if (ch == BOXES - 1) {               // the accumulator has been read
          tc_fence_before();
          __syncwarp();
          if (lane == 0) arrive_at(first_cta(&sm->acc_empty[n & 1]));
        }
        float u[W], w[W];                    // (w: gated)
#pragma unroll
        for (int k = 0; k < W; ++k) {
          u[k] = __uint_as_float(v[k]);
          if (KIND == kGated) w[k] = __uint_as_float(v[(32 + k) % 64]);
        }
        if constexpr (KIND != kPlain) {
          using T = __nv_bfloat16;
          auto add_bias = [&](float (&x)[W], const T* b) {             // (the same of all lanes; N is a multiple of 8)
#pragma unroll
            for (int j = 0; j < W; j += 8) {
              if (c + j >= p.N) break;
              float t[8];
              load_vec<8>(b + c + j, t);
#pragma unroll
              for (int k = 0; k < 8; k += 2) add2(x[j + k], x[j + k + 1], x[j + k], x[j + k + 1], t[k], t[k + 1]);
            }
          };
          if (e.bias) {
            add_bias(u, static_cast<const T*>(e.bias));
            if constexpr (KIND == kGated) add_bias(w, static_cast<const T*>(e.bias) + p.N);
          }
          if (e.kept) {
            emit(&tmKept, p.wide, p.by_wide, u, c);
            if constexpr (KIND == kGated) emit(&tmKept2, p.wide, p.by_wide, w, c);
          }
          by_activation(e.act, [&](auto act) {
#pragma unroll
            for (int k = 0; k < W; ++k) u[k] = activate<false, decltype(act)::value>(u[k]);
          });
          if constexpr (KIND == kGated)
#pragma unroll
            for (int k = 0; k < W; k += 2) mul2(u[k], u[k + 1], u[k], u[k + 1], w[k], w[k + 1]);
        }
        emit(&tmOut, e.inner, e.by_inner, u, c);
      }
    }
    slices(i, n);
    if (lane == 0) bulk_wait_group<0>();     // (the stores have been read from this CTA's memory and written before it exits)
  } else if (warp >= 4 && STORE == kRows) {
    // ------------------------------------------------------------------ sums to results by rows: gate, residual, order of the rows
    using T = __nv_bfloat16;
    const int quad = warp & 3, half = (warp - 4) >> 2;
    const uint32_t lanes = tmem + ((uint32_t)(quad * 32) << 16);
    float* mine = reinterpret_cast<float*>(turn + (warp - 4) * TURN_BYTES);
    const Epilogue& e = p.e;
    constexpr int W = KIND == kGated ? 32 : 64;        // columns of out at a time
    constexpr int PER_ROW = W / 8, ROWS = 32 / PER_ROW, TURNS = 32 / ROWS;
    const int lr = lane / PER_ROW, lc = (lane % PER_ROW) * 8;
    // four floats at place c4 of a row of the turned tile: rows apart by their number, so that neither rows nor columns meet in a bank
    auto place = [&](int r, int c4) { return reinterpret_cast<float4*>(mine + r * STAGE_W + ((c4 ^ (r & 7)) << 2)); };
    auto column = [&](int ch) { return KIND == kGated ? half * 64 + ch * 32 : half * 128 + ch * 64; };      // first column in the tile
    // A tile as a warp sees it; lane = row: its sample, token of out and group; the row of the gate where all rows have the same (nearly always).
    struct Place { Item it; int rows, b, t, g; long long first; const float* gate; };
    auto tile_of = [&](int i) {
      Place o;
      o.it = item_of<KIND>(p, i);
      const int local = o.it.row + (int)rank * BM + quad * 32;
      o.rows = p.Sm - local;
      o.first = (long long)o.it.sample * p.Sm + local;
      o.b = o.g = 0;
      o.t = -1;
      o.gate = nullptr;
      if (lane < o.rows) {
        const int r = (int)o.first + lane;
        o.b = e.by_S.div(r);
        o.t = r - o.b * e.S;
        if (e.perm) o.t = __ldg(e.perm + o.t);
      }
      return o;
    };
    auto settle = [&](Place& o) {            // (what hangs on the loaded place)
      if ((unsigned)o.t >= (unsigned)e.S) o.t = -1;
      if (!e.gate) return;
      if (o.t >= 0) o.g = e.by_gate.div(o.t);
      const unsigned some = __ballot_sync(0xffffffffu, o.t >= 0);
      const int from = some ? __ffs(some) - 1 : 0;
      const int b0 = __shfl_sync(0xffffffffu, o.b, from), g0 = __shfl_sync(0xffffffffu, o.g, from);
      if (__all_sync(0xffffffffu, o.t < 0 || (o.b == b0 && o.g == g0))) o.gate = e.gate + b0 * e.gb + g0 * e.gg;
    };
    const bool onto = e.residual != nullptr;
    // What a box of columns needs from memory is asked for a box ahead: beside the operands' loads it takes microseconds, and loads come back
    // in the order they were asked for.  So bias and gate of the next box and the places of the next tile's rows go ahead of the next box's
    // residual, a row of which is asked for, into shared memory, when the last one there has been used.
    uint4 bias_in[2];
    char* const mine_ahead = ahead + (warp - 4) * AHEAD_BYTES + lane * 16;       // (16 bytes per row and lane)
    float gate_in[8];
    auto load_residual = [&](const Place& o, int ch, int q) {
      const int c = o.it.col + column(ch) + lc;
      const int b = __shfl_sync(0xffffffffu, o.b, q * ROWS + lr), t = __shfl_sync(0xffffffffu, o.t, q * ROWS + lr);
      if (c < p.N && t >= 0)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(mine_ahead + q * 512)),
                     "l"(static_cast<const T*>(e.residual) + b * e.rb + t * e.rt + c)
                     : "memory");
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
    auto load_columns = [&](const Place& o, int ch) {
      const int c = o.it.col + column(ch) + lc;
      if (c >= p.N) return;
      if (e.bias) {
        bias_in[0] = __ldg(reinterpret_cast<const uint4*>(static_cast<const T*>(e.bias) + c));
        if (KIND == kGated) bias_in[1] = __ldg(reinterpret_cast<const uint4*>(static_cast<const T*>(e.bias) + e.cols + c));
      }
      if (o.gate) load_const<8>(o.gate + c, gate_in);
    };
    uint32_t n = 0;
    int i = pair;
    Place next;
    if (i < p.whole) {
      next = tile_of(i);
      settle(next);
      load_columns(next, 0);
      if (onto)
#pragma unroll
        for (int q = 0; q < TURNS; ++q) load_residual(next, 0, q);
    }
    for (; i < p.whole; i += pairs, ++n) {
      const Place now = next;
      const bool more = i + pairs < p.whole;
#pragma unroll
      for (int ch = 0; ch < 2; ++ch) {
        const int at = column(ch), c = now.it.col + at + lc;
        const bool col_ok = c < p.N;
        if (ch == 0) {
          mbar_wait_warp(&sm->acc_full[n & 1], (n >> 1) & 1, abort_flag, p.status);
          tc_fence_after();
        }
        const uint32_t from = lanes + (n & 1) * BN + at;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          uint32_t v[32];
          tmem_ld32(x == 0 ? from : KIND == kGated ? from + BN / 2 : from + 32, v);
          tmem_ld_wait();
          if (x == 0) {
            __syncwarp();                    // (the tile turned before has been read)
          } else if (ch == 1) {              // the accumulator has been read
            tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive_at(first_cta(&sm->acc_empty[n & 1]));
          }
#pragma unroll
          for (int j = 0; j < 8; ++j) *reinterpret_cast<uint4*>(place(lane, 8 * x + j)) = make_uint4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
        }
        __syncwarp();
        uint4 bias[2] = {bias_in[0], bias_in[1]};
        float gate[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) gate[x] = gate_in[x];
        if (ch == 0) {
          load_columns(now, 1);
          if (more) next = tile_of(i + pairs);
        } else if (more) {
          settle(next);
          load_columns(next, 0);
        }
#pragma unroll
        for (int q = 0; q < TURNS; ++q) {
          const int r = q * ROWS + lr;
          float u[8], w[8];
          {
            // a lane's eight columns are two places; which comes first alternates, so that the lanes of a row read apart
            const int c4 = lc / 4, swap = (lane >> 2) & 1;
            const float4 x = *place(r, c4 + swap), y = *place(r, c4 + (swap ^ 1));
            const float4 lo = swap ? y : x, hi = swap ? x : y;
            u[0] = lo.x; u[1] = lo.y; u[2] = lo.z; u[3] = lo.w; u[4] = hi.x; u[5] = hi.y; u[6] = hi.z; u[7] = hi.w;
            if (KIND == kGated) {
              const float4 a = *place(r, 8 + c4), b = *place(r, 9 + c4);
              w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w; w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
            }
          }
          if (onto) asm volatile("cp.async.wait_group %0;" ::"n"(TURNS - 1) : "memory");      // (the oldest of TURNS rows is here)
          const int b = __shfl_sync(0xffffffffu, now.b, r), t = __shfl_sync(0xffffffffu, now.t, r), g = __shfl_sync(0xffffffffu, now.g, r);
          if (col_ok && r < now.rows) {
            if (e.bias) {
              add_bf16x8(u, bias[0]);
              if (KIND == kGated) add_bf16x8(w, bias[1]);
            }
            if (e.kept) {
              T* kept = static_cast<T*>(e.kept) + (now.first + r) * p.wide + c;
              store_vec<8>(kept, u);
              if (KIND == kGated) store_vec<8>(kept + p.N, w);
            }
            by_activation(e.act, [&](auto act) {
#pragma unroll
              for (int x = 0; x < 8; ++x) u[x] = activate<false, decltype(act)::value>(u[x]);
            });
            if (KIND == kGated)
#pragma unroll
              for (int x = 0; x < 8; x += 2) mul2(u[x], u[x + 1], u[x], u[x + 1], w[x], w[x + 1]);
            if (t >= 0) {
              if (e.gate) {
                if (!now.gate) load_const<8>(e.gate + b * e.gb + g * e.gg + c, gate);
#pragma unroll
                for (int x = 0; x < 8; x += 2) mul2(u[x], u[x + 1], u[x], u[x + 1], gate[x], gate[x + 1]);
              }
              if (e.residual) add_bf16x8(u, *reinterpret_cast<const uint4*>(mine_ahead + q * 512));
              store_vec<8>(static_cast<T*>(e.out) + b * e.ob + t * e.ot + c, u);
            }
          }
          __syncwarp();
          if (onto) {
            if (ch == 0) load_residual(now, 1, q);
            else if (more) load_residual(next, 0, q);
            else asm volatile("cp.async.commit_group;" ::: "memory");
          }
        }
      }
    }
    slices(i, n);
  } else if (warp >= 4 && STORE == kSlopes) {
    // ------------------------------------------------------------------ sums d to d act'(u) and act(u) (gated: d v act'(u), d act(u); act(u) v)
    // Lane = row; everything comes and goes in boxes by TMA (by rows of lanes 77 million instructions instead of 50, in the same time).  Results take
    // the place of what they are made of, box after box of the columns in turns in one of two places: the next one is asked for into the other,
    // whose results have left.  (A box asked for into the place of one just read, behind no more than the warp's meeting, came before the last
    // reads of that: they need not have happened when the lanes meet, only before something is done with their values.)
    constexpr bool PAIR = KIND == kSlopeGated;
    constexpr int W = PAIR ? 32 : 64, BOXES = BN / 2 / W, BOX = 32 * 2 * W;      // columns of a box, boxes of a warp, bytes
    constexpr int IN = (PAIR ? 2 : 1) * BOX;                                     // u and v, then du and dv
    static_assert(2 * IN + BOX <= TURN_BYTES + AHEAD_BYTES, "two boxes and h");
    const int quad = warp & 3, half = (warp - 4) >> 2;
    const uint32_t lanes = tmem + ((uint32_t)(quad * 32) << 16);
    char* const places = turn + (warp - 4) * (TURN_BYTES + AHEAD_BYTES);
    char* const again = places + 2 * IN;                                         // h
    uint64_t* const here = &sm->ahead[warp - 4];
    const Epilogue& e = p.e;
    auto ask = [&](const Item& it, int ch, char* to) { // (one lane; places outside read as zeros)
      const int c = it.col + half * (BN / 2) + ch * W, row = it.row + (int)rank * BM + quad * 32;
      mbar_expect_tx(here, IN);
      tma_load_4d(to, &tmKept, here, c, row, 0, 0);
      if (PAIR) tma_load_4d(to + BOX, &tmKept2, here, c, row, 0, 0);
    };
    // 16-byte piece j of the lane's row of a box
    auto piece = [&](char* box, int j) {
      return reinterpret_cast<uint4*>(box + lane * (2 * W) + (W == 64 ? j ^ (lane & 7) : j ^ ((lane >> 1) & 3)) * 16);
    };
    uint32_t n = 0, boxes = 0;
    Item next = item_of<KIND>(p, pair);      // (tiles are whole here)
    if (lane == 0) ask(next, 0, places);
    for (int i = pair; i < p.items; i += pairs, ++n) {
      const Item now = next;
      const bool more = i + pairs < p.items;
      if (more) next = item_of<KIND>(p, i + pairs);
      const int row = now.row + (int)rank * BM + quad * 32;
      mbar_wait_warp(&sm->acc_full[n & 1], (n >> 1) & 1, abort_flag, p.status);
      tc_fence_after();
#pragma unroll 1
      for (int ch = 0; ch < BOXES; ++ch, ++boxes) {
        const int at = half * (BN / 2) + ch * W, c = now.col + at;
        float d[W];
#pragma unroll
        for (int x = 0; x < W / 32; ++x) {
          uint32_t v[32];
          tmem_ld32(lanes + (n & 1) * BN + at + 32 * x, v);
          tmem_ld_wait();
#pragma unroll
          for (int k = 0; k < 32; ++k) d[32 * x + k] = __uint_as_float(v[k]);
        }
        if (ch == BOXES - 1) {               // the accumulator has been read
          tc_fence_before();
          __syncwarp();
          if (lane == 0) arrive_at(first_cta(&sm->acc_empty[n & 1]));
        }
        mbar_wait_warp(here, boxes & 1, abort_flag, p.status);
        char* const box = places + (boxes & 1) * IN;
        if (lane == 0) {                     // the last results have left
          bulk_wait_group_read<0>();
          char* const other = places + (~boxes & 1) * IN;
          if (ch < BOXES - 1) ask(now, ch + 1, other);
          else if (more) ask(next, 0, other);
        }
        __syncwarp();
        float dv[PAIR ? W : 1];
        by_activation(e.act, [&](auto act) {
#pragma unroll
          for (int j = 0; j < W / 8; ++j) {
            float h[8], u[8], v[8];
            const uint4 uq = *piece(box, j), vq = PAIR ? *piece(box + BOX, j) : uq;
            const uint32_t uw[4] = {uq.x, uq.y, uq.z, uq.w};
            const uint32_t vw[4] = {vq.x, vq.y, vq.z, vq.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              u[2 * k] = __uint_as_float(uw[k] << 16);
              u[2 * k + 1] = __uint_as_float(uw[k] & 0xffff0000u);
              if (PAIR) { v[2 * k] = __uint_as_float(vw[k] << 16); v[2 * k + 1] = __uint_as_float(vw[k] & 0xffff0000u); }
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const float2 s = activate_slope<false, decltype(act)::value>(u[k]);
              float& x = d[8 * j + k];
              if (PAIR) {
                h[k] = s.x * v[k];
                dv[PAIR ? 8 * j + k : 0] = x * s.x;
                x *= v[k] * s.y;
              } else {
                h[k] = s.x;
                x *= s.y;
              }
            }
            auto put = [&](char* to, const float* f) {
              *piece(to, j) = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
            };
            put(box, d + 8 * j);
            if (PAIR) put(box + BOX, dv + (PAIR ? 8 * j : 0));
            if (e.again) put(again, h);
          }
        });
        fence_async_proxy();
        __syncwarp();
        if (lane == 0) {
          if (row < p.Sm && c < p.N) {
            tma_store_4d(&tmOut, box, c, row, 0, 0);
            if (PAIR) tma_store_4d(&tmOut2, box + BOX, c, row, 0, 0);
            if (e.again) tma_store_4d(&tmAgain, again, c, row, 0, 0);
          }
          bulk_commit_group();
        }
        if (e.col_sums && row < p.Sm) {      // of the warp's 32 rows (rows outside are zeros)
          float* to = e.col_sums + (long long)(row >> 5) * p.wide + c + lane;
#pragma unroll
          for (int x = 0; x < W / 32; ++x) {
            const float s = column_sum(d + 32 * x);
            if (c + 32 * x + lane < p.N) to[32 * x] = s;
          }
          if constexpr (PAIR) {
            const float s = column_sum(dv);
            if (c + lane < p.N) to[p.N] = s;
          }
        }
      }
    }
    if (lane == 0) bulk_wait_group<0>();
  }
  tc_fence_before();
  __syncthreads();
  cluster_meet();                            // (the first CTA has issued and waited for everything that reads the other's memory)
  if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

// [inner, S, heads, B] of a matrix, boxes of `cols` columns (64, 32) x `rows` rows.
bool map_of(CUtensorMap* map, const Matrix& m, int rows, int cols = 64) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  const cuuint64_t n[4] = {(cuuint64_t)m.inner, (cuuint64_t)m.S, (cuuint64_t)(m.cols / m.inner), (cuuint64_t)m.B};
  // (strides of dimensions of one address nothing, but have to be multiples of 16 bytes)
  const cuuint64_t stride[3] = {m.S > 1 ? (cuuint64_t)m.st * 2 : 16, m.cols > m.inner ? (cuuint64_t)m.sh * 2 : 16, m.B > 1 ? (cuuint64_t)m.sb * 2 : 16};
  const cuuint32_t box[4] = {(cuuint32_t)cols, (cuuint32_t)rows, 1, 1}, one[4] = {1, 1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(m.p), n, stride, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
            cols == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// Samples that follow one another at the tokens' distance are one, and so are samples of one token.
Matrix folded(Matrix m) {
  if (m.B > 1 && m.S == 1) { m.S = m.B; m.st = m.sb; m.B = 1; m.sb = 0; }
  if (m.B > 1 && m.sb == (long long)m.S * m.st) { m.S *= m.B; m.B = 1; m.sb = 0; }
  return m;
}

// Tiles worked out as a whole, in rounds of all pairs, and slices of the summed index of those that are left: as many as make the time least.
// A stage takes 0.28 us, a tile another one at its ends, a slice 1.5 more for its sums in memory; joining them is a launch and the
// sums' way through the L2.
constexpr int kPairs = 74;                   // of B200's SMs (a workspace's size goes by the shape alone)
struct Plan { int whole, rest, per, splits; };
Plan plan_of(long long tiles, int steps, bool cut) {
  Plan best{(int)tiles, 0, steps, 1};
  if (!cut) return best;
  double least = (double)((tiles + kPairs - 1) / kPairs) * (steps * 0.28 + 1.0);
  for (long long whole = tiles / kPairs * kPairs; whole >= 0 && whole >= tiles / kPairs * kPairs - kPairs; whole -= kPairs) {
    const long long rest = tiles - whole;
    for (int s = 2; s <= std::min(steps, 32) && rest * s <= 8 * kPairs; ++s) {
      const int per = (steps + s - 1) / s;
      if ((steps + per - 1) / per != s || rest == 0) continue;
      const double t = (double)(whole / kPairs) * (steps * 0.28 + 1.0) + (double)((rest * s + kPairs - 1) / kPairs) * (per * 0.28 + 2.5) + 3.0 + rest * s * 0.03;
      if (t < least * 0.97) {
        least = t;
        best = Plan{(int)whole, (int)rest, per, s};
      }
    }
  }
  return best;
}
// Stages of a product's summed index.
int steps_of(Form form, const Matrix& a, int planes) {
  return planes * (form == kColsCols ? a.B * ((a.S + BK - 1) / BK) : (a.cols + BK - 1) / BK);
}
// Tiles, of as many samples as do not follow one another.
long long tiles_of(const Product& p, int samples) {
  const int cols = p.e.kind == kGated ? BN / 2 : BN;
  const long long rows = (p.M / samples + 2 * BM - 1) / (2 * BM);
  return rows * samples * ((p.N + cols - 1) / cols);
}

// The slices' sums of the last tiles, and what becomes of them: CTAs of 256 pieces of eight columns.
template <int KIND>
__global__ void __launch_bounds__(256) join_tiles_kernel(Args p) {
  if (!grid_begin()) return;
  constexpr int COLS = KIND == kGated ? BN / 2 : BN, PER_TILE = 2 * BM * COLS / 8 / 256;
  const int tile = blockIdx.x / PER_TILE, piece = (blockIdx.x - tile * PER_TILE) * 256 + threadIdx.x;
  const int r = piece / (COLS / 8), c = piece % (COLS / 8) * 8;
  const Item it = item_of<KIND>(p, p.whole + tile);
  if (it.row + r >= p.Sm || it.col + c >= p.N) return;
  const float* from = p.part + tile * PART + r * BN + c;
  float u[8] = {}, v[8] = {};
#pragma unroll 2
  for (int s = 0; s < p.splits; ++s, from += p.rest * PART) {
    float t[8];
    load_vec<8>(from, t);
#pragma unroll
    for (int x = 0; x < 8; ++x) u[x] += t[x];
    if (KIND == kGated) {
      load_vec<8>(from + BN / 2, t);
#pragma unroll
      for (int x = 0; x < 8; ++x) v[x] += t[x];
    }
  }
  finish<__nv_bfloat16, 8, KIND>(p.e, OutRow<__nv_bfloat16>(p.e, it.sample * p.Sm + it.row + r), it.col + c, u, v);
}

struct Maps { CUtensorMap a, b, out, out2, kept, kept2, again; };      // (2: of the second half of the columns)

template <typename K>
int start(K kernel, int store, const Args& a, const Maps& m, cudaStream_t st) {
  VMOBA_CUDA_OK(allow_smem(kernel, smem_of(store)));
  launch_kernel(kernel, 2 * (unsigned)std::min(a.items, std::max(1, sm_count() / 2)), THREADS, (size_t)smem_of(store), st, m.a, m.b, m.out, m.out2,
                m.kept, m.kept2, m.again, a);
  VMOBA_LAUNCH_OK(1);
  return VMOBA_OK;
}
template <int FORM, int KIND>
int launch(const Args& a, const Maps& m, bool boxes, cudaStream_t st) {
  int rc;
  if constexpr (KIND == kPlain) rc = start(pair_kernel<FORM, KIND, kBoxes>, kBoxes, a, m, st);
  else rc = boxes ? start(pair_kernel<FORM, KIND, kBoxes>, kBoxes, a, m, st) : start(pair_kernel<FORM, KIND, kRows>, kRows, a, m, st);
  if (rc || a.splits == 1) return rc;
  launch_kernel(join_tiles_kernel<KIND>, (unsigned)a.rest * (2 * BM * (KIND == kGated ? BN / 2 : BN) / 8 / 256), 256, 0, st, a);
  VMOBA_LAUNCH_OK(1);
  return VMOBA_OK;
}

}  // namespace tc

// For the samples' rows in one or not: strides decide that.
size_t tc_scratch(const Product& p) {
  size_t most = 0;
  for (int apart = 0; apart < 2; ++apart) {
    Matrix a = p.a;
    if (!apart && a.B > 1) { a.S *= a.B; a.B = 1; }
    const tc::Plan plan = tc::plan_of(tc::tiles_of(p, p.form == kColsCols ? 1 : a.B), tc::steps_of(p.form, a, p.planes), p.e.kind < kSlope);
    if (plan.splits > 1) most = std::max(most, (size_t)plan.rest * plan.splits * (size_t)tc::PART + tc::TO_PART);
  }
  return most;
}

int tc_product(const Product& p, float* scratch, cudaStream_t st) {
  using namespace tc;
  Args a{};
  Matrix ma = p.a, mb = p.b;
  const int cols = p.e.kind == kGated ? BN / 2 : BN;
  a.e = p.e;
  a.N = p.N;
  a.wide = is_gated(p.e.kind) ? 2 * p.N : p.N;
  a.status = p.status;
  if (p.form == kColsCols) {
    if (folded(ma).B == 1 && folded(mb).B == 1) {
      ma = folded(ma);
      mb = folded(mb);
    }
    a.steps = steps_of(p.form, ma, p.planes);
    a.step_inner = (ma.S + BK - 1) / BK;
    a.b_samples = mb.B;
    if (p.planes == 2) {                     // (a plane's samples behind the other's)
      if (ma.B > 1 && p.plane != ma.B * ma.sb) return VMOBA_ERR_ARG;
      if (ma.B == 1) ma.sb = p.plane;
      ma.B *= 2;
    }
  }
  // how results leave, and (boxes) whether they lie so that all samples' rows can be taken for one's
  const bool slopes = p.e.kind >= kSlope, boxes = !p.e.gate && !p.e.residual && !p.e.perm && !slopes;
  const bool gated = p.e.kind == kGated;
  Matrix out{p.e.out, p.M / p.e.S, p.e.S, p.e.cols, p.e.inner, p.e.ob, p.e.ot, p.e.oh};
  Matrix kept{p.e.kept, out.B, out.S, a.wide, a.wide, (long long)out.S * a.wide, a.wide, 0};
  if (p.form != kColsCols) {
    if (!boxes || folded(out).B == 1) {
      ma = folded(ma);
      if (ma.B == 1) { out = folded(out); kept = folded(kept); }
    }
    a.steps = steps_of(p.form, ma, p.planes);
    a.step_inner = (ma.cols + BK - 1) / BK;
    if (p.planes == 2) {                     // (as a second head)
      ma.cols *= 2;
      ma.sh = p.plane;
    }
    a.Sm = ma.S;
  } else {
    a.Sm = p.M;
  }
  a.rows_tiles = (a.Sm + 2 * BM - 1) / (2 * BM);
  a.row_tiles = a.rows_tiles * (p.form == kColsCols ? 1 : ma.B);
  a.col_tiles = (p.N + cols - 1) / cols;
  const long long tiles = (long long)a.row_tiles * a.col_tiles;
  if (tiles > INT32_MAX - 4096) return VMOBA_ERR_SHAPE;
  const Plan plan = plan_of(tiles, a.steps, !slopes);      // (slopes' sums of rows are of whole sums)
  a.whole = plan.whole; a.rest = plan.rest; a.per = plan.per; a.splits = plan.splits;
  a.items = a.whole + a.rest * a.splits;
  a.part = scratch + reinterpret_cast<uintptr_t>(scratch) % 32 / sizeof(float);      // (0 or TO_PART)
  a.a_inner = ma.inner; a.b_inner = mb.inner;
  a.by_rows_tiles = FastDiv((unsigned)a.rows_tiles);
  a.by_rest = FastDiv((unsigned)std::max(1, a.rest));
  a.by_group = FastDiv((unsigned)(8 * a.col_tiles));
  a.by_a_inner = FastDiv((unsigned)ma.inner); a.by_b_inner = FastDiv((unsigned)mb.inner);
  a.by_step = FastDiv((unsigned)a.step_inner);
  a.by_wide = FastDiv((unsigned)a.wide);
  Maps m{};
  if (!map_of(&m.a, ma, p.form == kColsCols ? BK : BM) || !map_of(&m.b, mb, p.form == kRowsRows ? 128 : BK)) return VMOBA_ERR_CUDA;
  if (boxes || slopes) {                     // (gated: the halves on their own, so that a box of the first ends where it does)
    const bool two = is_gated(p.e.kind);
    const int box = two ? 32 : 64;
    auto halves = [&](const Matrix& all, const void* base, CUtensorMap* first, CUtensorMap* second) {
      Matrix x = all;
      x.p = base;
      x.cols = x.inner = p.N;
      if (!map_of(first, x, 32, box)) return false;
      x.p = static_cast<const char*>(base) + 2ll * p.N;
      return !two || map_of(second, x, 32, box);
    };
    if (slopes) {
      if (!halves(kept, p.e.kept, &m.kept, &m.kept2) || !halves(kept, p.e.out, &m.out, &m.out2)) return VMOBA_ERR_CUDA;
      if (p.e.again && !map_of(&m.again, folded(Matrix{p.e.again, out.B, out.S, p.N, p.N, (long long)out.S * p.N, p.N, 0}), 32, box)) return VMOBA_ERR_CUDA;
    } else {
      if (!map_of(&m.out, out, 32, box)) return VMOBA_ERR_CUDA;
      if (kept.p && !halves(kept, kept.p, &m.kept, &m.kept2)) return VMOBA_ERR_CUDA;
    }
  }
  if (p.form == kColsCols) return launch<kColsCols, kPlain>(a, m, boxes, st);
  if (p.e.kind == kSlope) return start(pair_kernel<kRowsCols, kSlope, kSlopes>, kSlopes, a, m, st);
  if (p.e.kind == kSlopeGated) return start(pair_kernel<kRowsCols, kSlopeGated, kSlopes>, kSlopes, a, m, st);
  if (p.form == kRowsCols) return launch<kRowsCols, kPlain>(a, m, boxes, st);
  return gated ? launch<kRowsRows, kGated>(a, m, boxes, st) : launch<kRowsRows, kForward>(a, m, boxes, st);
}

}  // namespace linear
}  // namespace vmoba
