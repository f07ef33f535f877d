// Matrix products on the tensor cores: bf16 operands, fp32 sums.
//
// Two CTAs of a cluster work on one tile of 256 x 256 sums: each holds 128 of its rows (its half of the accumulator in its own TMEM) and brings
// 128 rows and 128 columns of the operands, 64 summed indices at a time, into its shared memory; one thread of the pair issues the
// products of both (tcgen05.mma, cta_group::2).  Every byte loaded is used for 256 products, which is what L2 can feed: a lone CTA with a
// 128 x 256 tile asks it for half as much again.  Two accumulators alternate, so that eight warps finish one tile while the next
// is summed.  An operand whose summed index runs along its rows is read as it lies (MN-major tiles), so that no gradient needs a transpose.
// gated: the pair's columns are 128 of the gate (first CTA's half) and 128 of the factor.
// Where tiles would leave SMs idle, the summed index is cut into slices, whose sums a second kernel adds in a fixed order.
#include <algorithm>

#include "linear.cuh"

namespace vmoba {
namespace linear {
namespace tc {

using namespace sm100;

constexpr int BM = 128, BN = 256, BK = 64;   // per CTA: rows of the accumulator; columns; summed indices of a stage
constexpr int STAGES = 5;
constexpr int HALF = 128 * BK * 2;           // bytes of one operand's half of a stage
constexpr int PANEL = 64 * 128;              // MN-major: 64 places of the tile x 64 summed indices
constexpr int THREADS = 384, EPI_WARPS = 8;
constexpr int STAGE_W = 64;                  // columns that a warp turns around in shared memory at a time

struct Args {
  Epilogue e;
  int Sm, rows_tiles, row_tiles, col_tiles;  // rows of a sample; tiles of rows per sample and of all; tiles of columns
  int N;                                     // columns of out
  int steps, per, splits, items;             // stages of the summed index, of a slice; slices
  int a_inner, b_inner, step_inner;          // columns of a head; (kColsCols) stages per sample
  FastDiv by_rows_tiles, by_tiles, by_group, by_a_inner, by_b_inner, by_step;
  float* part;                               // [slice][row][column of the sums]
  int wide;                                  // columns of the sums
  long long part_rows;
  int32_t* status;
};

struct Shared {
  uint64_t full[STAGES], empty[STAGES], acc_full[2], acc_empty[2], drain;
  uint32_t tmem;
  int abort;
};
constexpr int STAGE_BYTES = 2 * HALF;
constexpr int TURN_BYTES = 32 * STAGE_W * 4;
constexpr int SMEM_BYTES = 1024 + STAGES * STAGE_BYTES + EPI_WARPS * TURN_BYTES + (int)sizeof(Shared);
static_assert(SMEM_BYTES <= 227 * 1024, "shared memory of a CTA");

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
__device__ __forceinline__ void arrive_at(uint32_t cluster_bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
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
// Arrives at the barriers of both CTAs when all products issued so far are done.
__device__ __forceinline__ void pair_commit(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)),
               "h"((uint16_t)3)
               : "memory");
}

struct Item {
  int split, sample, row, col;               // first row of the pair's tile in the sample; first column of out
};
// Tiles in groups of eight tiles of rows, down the rows first: the tiles that run at a time share rows and columns.
template <int KIND>
__device__ __forceinline__ Item item_of(const Args& p, int i) {
  constexpr int G = 8, COLS = KIND == kGated ? BN / 2 : BN;
  const int split = p.by_tiles.div(i);
  int t = i - split * p.row_tiles * p.col_tiles;
  const int group = p.by_group.div(t);       // (by G * col_tiles)
  t -= group * G * p.col_tiles;
  const int high = min(G, p.row_tiles - group * G);
  const int col = t / high, rt = group * G + t - col * high;
  const int sample = p.by_rows_tiles.div(rt);
  return {split, sample, (rt - sample * p.rows_tiles) * 2 * BM, col * COLS};
}

template <int FORM, int KIND>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(THREADS, 1)
    pair_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, Args p) {
  if (!grid_begin()) return;
  constexpr bool A_MN = FORM == kColsCols, B_MN = FORM != kRowsRows;
  extern __shared__ char smem_raw[];
  char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  char* turn = smem + STAGES * STAGE_BYTES;
  Shared* sm = reinterpret_cast<Shared*>(turn + EPI_WARPS * TURN_BYTES);
  volatile int* abort_flag = &sm->abort;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cta_rank();
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;

  if (warp == 0 && lane == 0) {
    for (int i = 0; i < STAGES; ++i) { mbar_init(&sm->full[i], 1); mbar_init(&sm->empty[i], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&sm->acc_full[i], 1); mbar_init(&sm->acc_empty[i], 2 * EPI_WARPS); }
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
        const int k0 = it.split * p.per, k1 = min(k0 + p.per, p.steps);
        const int row = it.row + (int)rank * BM;
        const int col = KIND == kGated ? it.col + (int)rank * p.N : it.col + (int)rank * (BN / 2);
        for (int k = k0; k < k1; ++k) {
          if (!mbar_wait(&sm->empty[slot], par, abort_flag, p.status)) break;
          const uint32_t a = smem_u32(smem) + slot * STAGE_BYTES, b = a + HALF, bar = first_cta(&sm->full[slot]);
          if (rank == 0) mbar_expect_tx(&sm->full[slot], 2 * STAGE_BYTES);
          int ks = 0, kb = 0;                // kColsCols: sample and first token of the stage
          if (A_MN) { kb = p.by_step.div(k); ks = (k - kb * p.step_inner) * BK; }
          if (A_MN) {
            for (int h = 0; h < 2; ++h) {
              const int m = row + 64 * h, z = p.by_a_inner.div(m);
              pair_load_4d(a + h * PANEL, &tmA, bar, m - z * p.a_inner, ks, z, kb);
            }
          } else {
            const int z = p.by_a_inner.div(k * BK);
            pair_load_4d(a, &tmA, bar, k * BK - z * p.a_inner, row, z, it.sample);
          }
          if (B_MN) {
            for (int h = 0; h < 2; ++h) {
              const int c = col + 64 * h, z = p.by_b_inner.div(c);
              pair_load_4d(b + h * PANEL, &tmB, bar, c - z * p.b_inner, A_MN ? ks : k * BK, z, kb);
            }
          } else {
            pair_load_4d(b, &tmB, bar, k * BK, col, 0, 0);
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
      constexpr uint32_t IDESC = make_idesc_bf16(2 * BM, BN, A_MN, B_MN);
      const uint32_t a_lo = desc_lo(smem_u32(smem), A_MN ? PANEL : 16), b_lo = desc_lo(smem_u32(smem) + HALF, B_MN ? PANEL : 16);
      uint32_t slot = 0, par = 0, n = 0;
      const int items = __reduce_max_sync(0xffffffffu, p.items);
      for (int i = pair; i < items; i += pairs, ++n) {
        const Item it = item_of<KIND>(p, i);
        const int k0 = it.split * p.per, k1 = __reduce_max_sync(0xffffffffu, min(k0 + p.per, p.steps));
        const uint32_t acc = tmem + (n & 1) * BN;
        mbar_wait_warp(&sm->acc_empty[n & 1], ((n >> 1) & 1) ^ 1, abort_flag, p.status);
        tc_fence_after();
        for (int k = k0; k < k1; ++k) {
          mbar_wait_warp(&sm->full[slot], par, abort_flag, p.status);
          tc_fence_after();
          const uint32_t at = slot * (STAGE_BYTES >> 4);
#pragma unroll
          for (int s = 0; s < BK / 16; ++s)      // sixteen summed indices: 32 bytes of a row, or sixteen rows of 128 bytes
            if (leader) pair_mma(acc, a_lo + at + s * (A_MN ? 128 : 2), b_lo + at + s * (B_MN ? 128 : 2), IDESC, k > k0 || s > 0 ? 1u : 0u);
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
  } else if (warp >= 4) {
    // ------------------------------------------------------------------ what becomes of the sums
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
    uint32_t n = 0;
    for (int i = pair; i < p.items; i += pairs, ++n) {
      const Item it = item_of<KIND>(p, i);
      const int local = it.row + (int)rank * BM + quad * 32;       // first row of the warp in the sample
      const int rows = p.Sm - local;                               // rows that there are
      const long long first = (long long)it.sample * p.Sm + local;
      // lane = row: its sample and token of out
      int ob = 0, ot = -1;
      if (lane < rows && !p.part) {
        const int r = (int)first + lane;
        ob = e.by_S.div(r);
        ot = r - ob * e.S;
        if (KIND != kPlain && e.perm) {
          ot = __ldg(e.perm + ot);
          if ((unsigned)ot >= (unsigned)e.S) ot = -1;
        }
      }
      bool there = false;
#pragma unroll 1
      for (int ch = 0; ch < 2; ++ch) {
        const int at = KIND == kGated ? half * 64 + ch * 32 : half * 128 + ch * 64;      // first column in the tile
        const int c = it.col + at + lc;
        const bool col_ok = c < p.N;
        uint4 res[TURNS];
        if (KIND != kPlain && e.residual && !p.part) {
#pragma unroll
          for (int q = 0; q < TURNS; ++q) {
            const int b = __shfl_sync(0xffffffffu, ob, q * ROWS + lr), t = __shfl_sync(0xffffffffu, ot, q * ROWS + lr);
            res[q] = make_uint4(0u, 0u, 0u, 0u);
            if (col_ok && t >= 0) res[q] = *reinterpret_cast<const uint4*>(static_cast<const T*>(e.residual) + b * e.rb + t * e.rt + c);
          }
        }
        float bias[8] = {}, bias2[8] = {};
        if (KIND != kPlain && e.bias && !p.part && col_ok) {
          load_vec<8>(static_cast<const T*>(e.bias) + c, bias);
          if (KIND == kGated) load_vec<8>(static_cast<const T*>(e.bias) + e.cols + c, bias2);
        }
        if (!there) {
          mbar_wait_warp(&sm->acc_full[n & 1], (n >> 1) & 1, abort_flag, p.status);
          tc_fence_after();
          there = true;
        }
        {
          uint32_t v[64];
          const uint32_t from = lanes + (n & 1) * BN + at;
          tmem_ld32(from, *reinterpret_cast<uint32_t(*)[32]>(&v[0]));
          tmem_ld32(KIND == kGated ? from + BN / 2 : from + 32, *reinterpret_cast<uint32_t(*)[32]>(&v[32]));
          tmem_ld_wait();
          if (ch == 1) {                     // the accumulator has been read
            tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive_at(first_cta(&sm->acc_empty[n & 1]));
          }
          __syncwarp();                      // (the tile turned before has been read)
#pragma unroll
          for (int j = 0; j < 16; ++j) *reinterpret_cast<uint4*>(place(lane, j)) = make_uint4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
          __syncwarp();
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
          if (p.part) {
            if (col_ok && r < rows) {
              float* to = p.part + ((long long)it.split * p.part_rows + first + r) * p.wide + c;
              store_vec<8>(to, u);
              if (KIND == kGated) store_vec<8>(to + p.N, w);
            }
            continue;
          }
          const int b = __shfl_sync(0xffffffffu, ob, r), t = __shfl_sync(0xffffffffu, ot, r);
          if (!col_ok || r >= rows) continue;
          if constexpr (KIND != kPlain) {
#pragma unroll
            for (int x = 0; x < 8; ++x) u[x] += bias[x];
            if (KIND == kGated) {
#pragma unroll
              for (int x = 0; x < 8; ++x) w[x] += bias2[x];
            }
            if (e.kept) {
              T* kept = static_cast<T*>(e.kept) + (first + r) * p.wide + c;
              store_vec<8>(kept, u);
              if (KIND == kGated) store_vec<8>(kept + p.N, w);
            }
#pragma unroll
            for (int x = 0; x < 8; ++x) {
              u[x] = activate<false>(e.act, u[x]);
              if (KIND == kGated) u[x] *= w[x];
            }
            if (t < 0) continue;
            if (e.gate) {
              float g[8];
              load_vec<8>(e.gate + b * e.gb + e.by_gate.div(t) * e.gg + c, g);
#pragma unroll
              for (int x = 0; x < 8; ++x) u[x] *= g[x];
            }
            if (e.residual) {
              const uint32_t rw[4] = {res[q].x, res[q].y, res[q].z, res[q].w};
#pragma unroll
              for (int x = 0; x < 4; ++x) add_bf16_pair(u[2 * x], u[2 * x + 1], rw[x]);
            }
          }
          const int h = e.inner == e.cols ? 0 : e.by_inner.div(c);
          store_vec<8>(static_cast<T*>(e.out) + b * e.ob + t * e.ot + h * e.oh + (c - h * e.inner), u);
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  cluster_meet();                            // (the first CTA has issued and waited for everything that reads the other's memory)
  if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

// The slices' sums, and what becomes of them.
template <int KIND>
__global__ void __launch_bounds__(256) join_kernel(Args p, FastDiv by_vecs, int vecs, int total) {
  if (!grid_begin()) return;
  const long long slice = p.part_rows * p.wide;
  for (int i = blockIdx.x * 256 + threadIdx.x; i < total; i += gridDim.x * 256) {
    const int r = by_vecs.div(i), c = (i - r * vecs) * 8;
    const float* from = p.part + (long long)r * p.wide + c;
    float u[8] = {}, v[8] = {};
    for (int s = 0; s < p.splits; ++s, from += slice) {
      float t[8];
      load_vec<8>(from, t);
#pragma unroll
      for (int x = 0; x < 8; ++x) u[x] += t[x];
      if (KIND == kGated) {
        load_vec<8>(from + p.N, t);
#pragma unroll
        for (int x = 0; x < 8; ++x) v[x] += t[x];
      }
    }
    finish<__nv_bfloat16, 8, KIND>(p.e, OutRow<__nv_bfloat16>(p.e, r), c, u, v);
  }
}

// [inner, S, heads, B] of a matrix, boxes of 64 columns x `rows` rows.
bool map_of(CUtensorMap* map, const Matrix& m, int rows) {
  const uint64_t n[4] = {(uint64_t)m.inner, (uint64_t)m.S, (uint64_t)(m.cols / m.inner), (uint64_t)m.B};
  // (strides of dimensions of one address nothing, but have to be multiples of 16 bytes)
  const uint64_t stride[4] = {1, m.S > 1 ? (uint64_t)m.st : 8, m.cols > m.inner ? (uint64_t)m.sh : 8, m.B > 1 ? (uint64_t)m.sb : 8};
  const uint32_t box[4] = {64, (uint32_t)rows, 1, 1};
  return make_tmap_bf16_strided(map, m.p, 4, n, stride, box);
}
// Samples that follow one another at the tokens' distance are one.
Matrix folded(Matrix m) {
  if (m.B > 1 && m.sb == (long long)m.S * m.st) { m.S *= m.B; m.B = 1; m.sb = 0; }
  return m;
}

// Slices of the summed index: as many as make the time least, in tiles' times: rounds of the pairs / slices, and what the slices' sums cost
// in memory (of a tile and slice, 256 KB out and in again at 6.5 TB/s shared by all, against a stage's 0.28 us).
int slices(long long tiles, int steps, int pairs) {
  int best = 1;
  double least = 1e30;
  for (int s = 1; s <= std::min(steps, 32); ++s) {
    const int per = (steps + s - 1) / s;
    if ((steps + per - 1) / per != s) continue;
    const double rounds = (double)((tiles * s + pairs - 1) / pairs);
    const double t = rounds * (per * 0.28 + 1.0) + (s > 1 ? 3.0 + tiles * s * 0.08 : 0.0);
    if (t < least * 0.97) { least = t; best = s; }
  }
  return best;
}

constexpr int kPairs = 74;                   // of B200's SMs (a workspace's size goes by the shape alone)
struct Plan { int steps, per, splits; long long tiles; };
Plan plan_of(const Product& p) {
  const int cols = p.e.kind == kGated ? BN / 2 : BN;
  Plan o;
  if (p.form == kColsCols) o.steps = p.a.B * ((p.a.S + BK - 1) / BK);
  else o.steps = (p.a.cols + BK - 1) / BK;
  o.tiles = (long long)((p.M + 2 * BM - 1) / (2 * BM)) * ((p.N + cols - 1) / cols);
  o.splits = slices(o.tiles, o.steps, kPairs);
  o.per = (o.steps + o.splits - 1) / o.splits;
  return o;
}

template <int FORM, int KIND>
int launch(const Args& a, const CUtensorMap& tmA, const CUtensorMap& tmB, cudaStream_t st) {
  auto kernel = pair_kernel<FORM, KIND>;
  VMOBA_CUDA_OK(allow_smem(kernel, SMEM_BYTES));
  launch_kernel(kernel, 2 * (unsigned)std::min(a.items, std::max(1, sm_count() / 2)), THREADS, SMEM_BYTES, st, tmA, tmB, a);
  VMOBA_LAUNCH_OK(1);
  if (a.splits > 1) {
    const long long vecs = a.N / 8, total = a.part_rows * vecs;
    launch_kernel(join_kernel<KIND>, (unsigned)std::min<long long>((total + 255) / 256, 16 * sm_count()), 256, 0, st, a, FastDiv((unsigned)vecs),
                  (int)vecs, (int)total);
    VMOBA_LAUNCH_OK(1);
  }
  return VMOBA_OK;
}

}  // namespace tc

size_t tc_scratch(const Product& p) {
  const tc::Plan plan = tc::plan_of(p);
  return plan.splits > 1 ? (size_t)plan.splits * p.M * p.N * (p.e.kind == kGated ? 2 : 1) : 0;
}

int tc_product(const Product& p, float* scratch, cudaStream_t st) {
  using namespace tc;
  Args a{};
  const Plan plan = plan_of(p);
  Matrix ma = p.a, mb = p.b;
  const int cols = p.e.kind == kGated ? BN / 2 : BN;
  a.e = p.e;
  a.N = p.N;
  a.wide = p.e.kind == kGated ? 2 * p.N : p.N;
  a.part_rows = p.M;
  a.status = p.status;
  a.splits = plan.splits; a.steps = plan.steps; a.per = plan.per;
  a.part = plan.splits > 1 ? scratch : nullptr;
  if (p.form == kColsCols) {
    if (folded(ma).B == 1 && folded(mb).B == 1) {
      ma = folded(ma);
      mb = folded(mb);
      a.steps = (ma.S + BK - 1) / BK;        // (no more than before)
      a.per = (a.steps + a.splits - 1) / a.splits;
      a.splits = (a.steps + a.per - 1) / a.per;
      if (a.splits == 1) a.part = nullptr;
    }
    a.step_inner = (ma.S + BK - 1) / BK;
    a.Sm = p.M;
  } else {
    ma = folded(ma);
    a.step_inner = 1;
    a.Sm = ma.S;
  }
  a.rows_tiles = (a.Sm + 2 * BM - 1) / (2 * BM);
  a.row_tiles = a.rows_tiles * (p.form == kColsCols ? 1 : ma.B);
  a.col_tiles = (p.N + cols - 1) / cols;
  const long long tiles = (long long)a.row_tiles * a.col_tiles;
  if (tiles * a.splits > INT32_MAX - 4096 || (a.splits > 1 && (long long)p.M * (p.N / 8) > INT32_MAX - (1 << 24))) return VMOBA_ERR_SHAPE;
  a.items = (int)(tiles * a.splits);
  a.a_inner = ma.inner; a.b_inner = mb.inner;
  a.by_rows_tiles = FastDiv((unsigned)a.rows_tiles);
  a.by_tiles = FastDiv((unsigned)tiles);
  a.by_group = FastDiv((unsigned)(8 * a.col_tiles));
  a.by_a_inner = FastDiv((unsigned)ma.inner); a.by_b_inner = FastDiv((unsigned)mb.inner);
  a.by_step = FastDiv((unsigned)a.step_inner);
  CUtensorMap tmA, tmB;
  if (!map_of(&tmA, ma, p.form == kColsCols ? BK : BM) || !map_of(&tmB, mb, p.form == kRowsRows ? 128 : BK)) return VMOBA_ERR_CUDA;
  if (p.form == kColsCols) return launch<kColsCols, kPlain>(a, tmA, tmB, st);
  if (p.form == kRowsCols) return launch<kRowsCols, kPlain>(a, tmA, tmB, st);
  return p.e.kind == kGated ? launch<kRowsRows, kGated>(a, tmA, tmB, st) : launch<kRowsRows, kForward>(a, tmA, tmB, st);
}

}  // namespace linear
}  // namespace vmoba
