// Attention over key ranges: the plan, the CUDA-core kernels (fp32, and bf16 with head_dim 64), the joining of split key ranges,
// and the entry points.
//
//   t = scale q.k, capped c tanh(t / c);  p = exp(t - lse) inside the range, else 0;  o = sum p v
//   D = rowsum(dO * O);  dV = P^T dO;  dT = P (dO V^T - D) (1 - (t / c)^2);  dQ = scale dT K;  dK = scale dT^T Q
//
// A mask that is one run of keys per query needs two words per query, and what a tile of queries and a tile of keys have to do
// with one another follows from four: smallest lo and largest hi (nothing outside is visited), largest lo and smallest hi (nothing
// inside is masked).  Keys that no query of a unit sees are not read.
#include "attn_range.cuh"

#include "attn_simt.cuh"

namespace vmoba {
namespace range {

using simt::dot_tiles;
using simt::add_weighted;
using simt::kLd;
using simt::kLdP;
using simt::kRows;
using simt::kThreads;
using simt::kTileFloats;

// ------------------------------------------------------------------------------ plan
// A warp per unit: clamps its tokens' ranges and takes the unit's four bounds.
__global__ void __launch_bounds__(256)
plan_units_kernel(const int2* __restrict__ in, Plan plan, RDims D) {
  if (!grid_begin()) return;
  const int lane = threadIdx.x & 31;
  const long long n = (long long)D.Bm * D.nU;
  for (long long w = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); w < n; w += (long long)gridDim.x * 8) {
    const long long bm = w / D.nU;
    const int u = (int)(w - bm * D.nU), t0 = u * D.tpt, t1 = min(t0 + D.tpt, D.Sq);
    int lo_min = INT32_MAX, hi_max = 0, lo_max = 0, hi_min = INT32_MAX;
    for (int t = t0 + lane; t < t1; t += 32) {
      int2 r = in[bm * D.Sq + t];
      r.x = max(r.x, 0);
      r.y = min(r.y, D.Sk);
      if (r.x >= r.y) r = make_int2(0, 0);
      plan.rows[bm * D.Sq + t] = r;
      if (r.y > 0) { lo_min = min(lo_min, r.x); hi_max = max(hi_max, r.y); }
      lo_max = max(lo_max, r.x);
      hi_min = min(hi_min, r.y);
    }
    lo_min = __reduce_min_sync(0xffffffffu, lo_min);
    hi_max = __reduce_max_sync(0xffffffffu, hi_max);
    lo_max = __reduce_max_sync(0xffffffffu, lo_max);
    hi_min = __reduce_min_sync(0xffffffffu, hi_min);
    if (hi_max == 0) lo_min = 0;
    if (lane == 0) plan.units[w] = make_int4(lo_min, hi_max, lo_max, hi_min);
  }
}

// Keys that a forward item (one or two units from u0 on) visits.
__device__ __forceinline__ int2 item_hull(const int4* units, int u0, int n) {
  const int4 a = units[u0];
  int2 h = make_int2(a.x, a.y);
  if (n > 1) {
    const int4 b = units[u0 + 1];
    if (h.y <= h.x) h = make_int2(b.x, b.y);
    else if (b.y > b.x) h = make_int2(min(h.x, b.x), max(h.y, b.y));
  }
  return h;
}

// Few items: their key ranges are cut into pieces of equally many tiles, as long as the SMs allow.  The length is the one of 32 (a whole
// number of rounds over the SMs if every item were a multiple of it) with the smallest time of its last round; a piece costs a fixed time and
// its rows' trip through memory, `fixed` tiles.  One block.
constexpr int kSms = 148;                      // (of the design: plan and scratch are functions of the shape and the ranges alone)
constexpr int kFewItems = 4 * kSms;
__device__ __forceinline__ void plan_pieces(const Plan& plan, const RDims& D) {
  __shared__ int tiles[kFewItems], sums[32], length, biggest;
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5, n = D.Bm * D.nI, per = D.tc ? 2 : 1;      // (n < kFewItems)
  if (t == 0) biggest = 1;
  __syncthreads();
  int mine = 0;
  if (t < n) {
    const int bm = t / D.nI, u0 = (t - bm * D.nI) * per;
    const int2 h = item_hull(plan.units + (long long)bm * D.nU, u0, min(per, D.nU - u0));
    mine = max((h.y - h.x + D.TR - 1) / D.TR, 1);
    tiles[t] = mine;
    atomicMax(&biggest, mine);
  }
  const int total = __reduce_add_sync(0xffffffffu, mine);      // (of the warp)
  if (lane == 0) sums[warp] = total;
  __syncthreads();
  if (warp == 0) {
    const long long all = (long long)__reduce_add_sync(0xffffffffu, sums[lane]) * D.reps;
    const float fixed = D.tc ? 1.5f + 2.0f * min(D.rows, 256) / 256.0f : 0.5f;
    const int len = max(max((int)((all + (long long)kSms * (lane + 1) - 1) / ((long long)kSms * (lane + 1))), (biggest + D.smax - 1) / D.smax), 1);
    long long pieces = 0;
    for (int i = 0; i < n; ++i) pieces += (tiles[i] + len - 1) / len;
    const float cost = (float)((pieces * D.reps + kSms - 1) / kSms) * ((float)len + fixed);
    float best = cost;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) best = fminf(best, __shfl_xor_sync(0xffffffffu, best, o));
    const int who = __ffs(__ballot_sync(0xffffffffu, cost == best)) - 1;
    if (lane == who) length = len;
  }
  __syncthreads();
  // The order: the first pieces of all items, the second ones, ...: what runs at the same time reads the same keys (a frame of 1,560 tokens
  // against 31,200, 12 heads, a cache larger than the L2, the same call again and again: 329 us item after item, so 309).
  const int len = length;
  if (t < n) {
    tiles[t] = (mine + len - 1) / len;
    plan.pieces[t] = tiles[t];
  }
  __syncthreads();
  for (int k = warp; k < D.smax; k += 32) {    // (an item has at most smax pieces)
    int before = 0;
    for (int i = lane; i < n; i += 32) before += min(tiles[i], k);
    before = __reduce_add_sync(0xffffffffu, before);
    for (int i0 = 0; i0 < n; i0 += 32) {
      const int i = i0 + lane;
      const bool has = i < n && tiles[i] > k;
      const uint32_t all = __ballot_sync(0xffffffffu, has);
      if (has) plan.work[before + __popc(all & ((1u << lane) - 1u))] = make_int4(i / D.nI, i % D.nI, k * len, k);
      before += __popc(all);
    }
    if (k == D.smax - 1 && lane == 0) {
      plan.head[0] = before;
      plan.head[1] = len;
    }
  }
}

// The first Bm blocks put a sample's items in order (bins of equal width by the number of keys, the fullest first; inside a bin in any
// order, which no result depends on), the next one cuts few items into pieces, the others walk the key tiles, a warp each.
constexpr int kBins = 1024;
__global__ void __launch_bounds__(1024)
plan_tiles_kernel(Plan plan, RDims D) {
  if (!grid_begin()) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if ((int)blockIdx.x < D.Bm) {
    __shared__ int bin[kBins];
    const int per = D.tc ? 2 : 1;
    const int4* units = plan.units + (long long)blockIdx.x * D.nU;
    int* order = plan.order + (long long)blockIdx.x * D.nI;
    auto bin_of = [&](int i) {
      const int2 h = item_hull(units, i * per, min(per, D.nU - i * per));
      return kBins - 1 - (int)((long long)max(h.y - h.x, 0) * (kBins - 1) / D.Sk);
    };
    bin[threadIdx.x] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < D.nI; i += 1024) atomicAdd(&bin[bin_of(i)], 1);
    __syncthreads();
    const int mine = bin[threadIdx.x];
    int before = mine;
    __shared__ int sums[32];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, before, o);
      if (lane >= o) before += x;
    }
    if (lane == 31) sums[warp] = before;
    __syncthreads();
    for (int w = 0; w < warp; ++w) before += sums[w];
    bin[threadIdx.x] = before - mine;
    __syncthreads();
    for (int i = threadIdx.x; i < D.nI; i += 1024) order[atomicAdd(&bin[bin_of(i)], 1)] = i;
    return;
  }
  if ((int)blockIdx.x == D.Bm) {
    if (D.smax > 1) plan_pieces(plan, D);
    return;
  }
  const long long n = (long long)D.Bm * D.nK, warps = (long long)(gridDim.x - D.Bm - 1) * 32;
  for (long long w = (long long)(blockIdx.x - D.Bm - 1) * 32 + warp; w < n; w += warps) {
    const long long bm = w / D.nK;
    const int t = (int)(w - bm * D.nK);
    const int4* units = plan.units + bm * D.nU;
    int first = INT32_MAX, last = -1, lo = INT32_MAX, hi = 0, count = 0, whole = INT32_MAX, until = D.nU;
    auto sees_all = [&](const int4& a) { return reaches(a, t, D.TR) && a.z <= t * D.TR && a.w >= (t + 1) * D.TR; };
    for (int u = lane; u < D.nU; u += 32) {
      const int4 a = units[u];
      if (!reaches(a, t, D.TR)) continue;
      first = min(first, u);
      last = max(last, u);
      lo = min(lo, a.x);
      hi = max(hi, a.y);
      ++count;
      if (sees_all(a)) whole = min(whole, u);
    }
    whole = __reduce_min_sync(0xffffffffu, whole);
    count = __reduce_add_sync(0xffffffffu, count);
    if (whole < D.nU)
      for (int u = whole + lane; u < D.nU; u += 32)
        if (!sees_all(units[u])) { until = u; break; }
    until = __reduce_min_sync(0xffffffffu, until);
    first = __reduce_min_sync(0xffffffffu, first);
    last = __reduce_max_sync(0xffffffffu, last);
    lo = __reduce_min_sync(0xffffffffu, lo);
    hi = __reduce_max_sync(0xffffffffu, hi);
    if (lane == 0) {
      plan.runs[w] = whole < D.nU ? make_int4(count, whole, until, 0) : make_int4(count, 0, 0, 0);
      plan.keys[w] = last < 0 ? make_int4(0, 0, 0, 0) : make_int4(first, last + 1, max(lo - t * D.TR, 0), min(hi - t * D.TR, D.TR));
    }
  }
}

// ------------------------------------------------------------------------------ CUDA-core kernels
// Tiles of 64 rows x 64 keys as in attn_simt.cuh: a thread has rows 4 ty + i and keys tx + 16 j of a tile of scores.
template <typename T, int DH>
struct RowRegs {
  static constexpr int V = DH / 4, N = kRows * V / kThreads;
  float4 x[N];
  template <typename RowOf>
  __device__ __forceinline__ void fetch(RowOf row_of) {           // row_of(r): its first element, or null for zeros
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int i = threadIdx.x + n * kThreads, r = i / V, c4 = i % V;
      const T* row = row_of(r);
      x[n] = row ? load4(row + c4 * 4) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
  }
  __device__ __forceinline__ void store(float* dst) const {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int i = threadIdx.x + n * kThreads, r = i / V, c4 = i % V;
      *reinterpret_cast<float4*>(dst + r * kLd<DH> + c4 * 4) = x[n];
    }
  }
};

__device__ __forceinline__ float capped(float s, float scale, float cap) {
  s *= scale;
  return cap > 0.f ? cap * tanhf(s / cap) : s;
}

// A unit's rows: token and range of each, in shared memory.
struct UnitRows { int tok[kRows]; int2 range[kRows]; };
__device__ __forceinline__ void load_unit(UnitRows& s, const RDims& D, const Plan& plan, int b, int u) {
  if (threadIdx.x < kRows) {
    const int r = threadIdx.x, t = u * D.tpt + r / D.G;
    const bool ok = r < D.tpt * D.G && t < D.Sq;
    s.tok[r] = ok ? t : -1;
    s.range[r] = ok ? plan.rows[(long long)mask_batch(D.Bm, b) * D.Sq + t] : make_int2(0, 0);
  }
}

// Forward: an item (64 packed rows, or a piece of their keys) per CTA and turn, one pass with the running maximum and sum.  Bound by the FMA
// pipe; with few items by the chain of tiles.  Then a cluster of C CTAs takes an item, every C-th tile each, and their parts are joined through one
// another's shared memory, in the order of the CTAs.  (Two samples of 256 tokens, two heads of 64 on one key head, fp32: 16 items, 20.5 us with a CTA
// each, 15 with four.)
template <typename T, int DH>
__global__ void __launch_bounds__(kThreads, 2)
range_fwd_kernel(const RDims D, const Plan plan, const FwdArgs a, const int C) {
  if (!grid_begin()) return;
  extern __shared__ __align__(16) float simt_smem[];
  float* Qs = simt_smem;
  float* KVs = Qs + kTileFloats<DH>;
  float* Ps = KVs + kTileFloats<DH>;
  __shared__ UnitRows rows;
  const int t = threadIdx.x, ty = t >> 4, tx = t & 15;
  const bool cut = D.smax > 1;
  const long long n_items = cut ? (long long)plan.head[0] * D.reps : (long long)D.B * D.Hk * D.nI, all_rows = (long long)D.B * D.Hk * D.rows;
  const int rank = blockIdx.x % C;
  for (long long item = blockIdx.x / C; item < n_items; item += gridDim.x / C) {
    int b, hk, u, piece = 0, first = 0, last = INT32_MAX;
    if (cut) {
      const int4 w = plan.work[item / D.reps];
      const int rep = (int)(item % D.reps);
      b = D.Bm > 1 ? w.x : rep / D.Hk;
      hk = D.Bm > 1 ? rep : rep % D.Hk;
      u = w.y;
      first = w.z;
      last = first + plan.head[1];
      piece = w.w;
    } else {
      const int bhk = (int)(item / D.nI);
      b = bhk / D.Hk;
      hk = bhk - b * D.Hk;
      u = plan.order[(long long)mask_batch(D.Bm, b) * D.nI + (item - (long long)bhk * D.nI)];
    }
    const int bhk = b * D.Hk + hk;
    const int4 info = plan.units[(long long)mask_batch(D.Bm, b) * D.nU + u];
    const int k_lo = info.x + first * kRows, k_hi = (int)min((long long)info.x + (long long)last * kRows, (long long)info.y);
    __syncthreads();
    load_unit(rows, D, plan, b, u);
    __syncthreads();
    const T* kb = reinterpret_cast<const T*>(a.k) + b * a.ks.b + hk * a.ks.h;
    const T* vb = reinterpret_cast<const T*>(a.v) + b * a.vs.b + hk * a.vs.h;
    const T* qb = reinterpret_cast<const T*>(a.q) + b * a.qs.b + (long long)hk * D.G * a.qs.h;
    RowRegs<T, DH> next;
    next.fetch([&](int r) { return rows.tok[r] < 0 ? nullptr : qb + rows.tok[r] * a.qs.t + (r % D.G) * a.qs.h; });
    next.store(Qs);
    float m_[4], l[4], acc[4][DH / 16];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      m_[i] = -INFINITY; l[i] = 0.f;
#pragma unroll
      for (int c = 0; c < DH / 16; ++c) acc[i][c] = 0.f;
    }
    const bool live = (ty & ~1) * 4 < D.tpt * D.G;    // (a warp has eight rows)
    for (long long t0 = k_lo + (long long)rank * kRows; t0 < k_hi; t0 += (long long)C * kRows) {
      const int nv = (int)min((long long)kRows, k_hi - t0);
      next.fetch([&](int r) { return r < nv ? kb + (t0 + r) * a.ks.t : nullptr; });
      __syncthreads();
      next.store(KVs);
      __syncthreads();
      next.fetch([&](int r) { return r < nv ? vb + (t0 + r) * a.vs.t : nullptr; });
      float corr[4];
      if (live) {
        float s[4][4];
        dot_tiles<DH>(Qs, KVs, ty, tx, nv, s);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int2 rg = rows.range[4 * ty + i];
          float mx = -INFINITY;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int key = (int)t0 + tx + 16 * j;
            s[i][j] = key >= rg.x && key < rg.y && tx + 16 * j < nv ? capped(s[i][j], D.scale, D.cap) : -INFINITY;
            mx = fmaxf(mx, s[i][j]);
          }
#pragma unroll
          for (int o = 8; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
          const float top = fmaxf(m_[i], mx), used = top == -INFINITY ? 0.f : top;
          corr[i] = expf(m_[i] - used);
          m_[i] = top;
          l[i] *= corr[i];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float p = expf(s[i][j] - used);
            l[i] += p;
            Ps[(4 * ty + i) * kLdP + tx + 16 * j] = p;
          }
        }
      }
      __syncthreads();
      next.store(KVs);
      __syncthreads();
      if (live) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int c = 0; c < DH / 16; ++c) acc[i][c] *= corr[i];
        add_weighted<DH>(Ps, KVs, ty, tx, kRows, acc);
      }
    }
    // four channels of a row: the sum of its weights times values, the maximum and the sum of the weights
    auto put = [&](int r, int col, const float4& sum, float m, float total) {
      const int tok = rows.tok[r], g = r % D.G;
      if (tok < 0) return;
      const bool none = total == 0.f;                // (no key: everything is 0 and lse -inf; a NaN stays one)
      const float inv = none ? 0.f : 1.0f / total, row_lse = none ? -INFINITY : m + logf(total);
      const long long packed = (long long)bhk * D.rows + (long long)tok * D.G + g, head = hk * D.G + g;
      const float4 x = make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv);
      if (!cut) {
        T* resid = a.resid ? reinterpret_cast<T*>(a.resid) + (((long long)b * D.Sq + tok) * D.Hq + head) * DH + col : nullptr;
        store4_resid(reinterpret_cast<T*>(a.o) + b * a.os.b + tok * a.os.t + head * a.os.h + col, resid, x);
      } else {
        store4(a.part_o + (piece * all_rows + packed) * DH + col, x);
      }
      if (col == 0) {
        if (!cut) a.lse[((long long)b * D.Hq + head) * D.Sq + tok] = row_lse;
        else a.part_lse[piece * all_rows + packed] = row_lse;
      }
    };
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], o);
    if (C == 1) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < DH / 64; ++c)
          put(4 * ty + i, 64 * c + 4 * tx, make_float4(acc[i][4 * c], acc[i][4 * c + 1], acc[i][4 * c + 2], acc[i][4 * c + 3]), m_[i], l[i]);
      continue;
    }
    cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
    __syncthreads();                                 // (values and weights have been read)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 4 * ty + i;
#pragma unroll
      for (int c = 0; c < DH / 64; ++c)
        *reinterpret_cast<float4*>(KVs + r * kLd<DH> + 64 * c + 4 * tx) = make_float4(acc[i][4 * c], acc[i][4 * c + 1], acc[i][4 * c + 2], acc[i][4 * c + 3]);
      if (tx == 0) { Ps[r] = m_[i]; Ps[kRows + r] = l[i]; }
    }
    cluster.sync();
    constexpr int V = DH / 4;
    for (int e = rank * kThreads + t; e < kRows * V; e += C * kThreads) {
      const int r = e / V, col = e % V * 4;
      float top = -INFINITY, total = 0.f;
      for (int n = 0; n < C; ++n) top = fmaxf(top, cluster.map_shared_rank(Ps, n)[r]);
      const float used = top == -INFINITY ? 0.f : top;
      float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int n = 0; n < C; ++n) {
        const float* stats = cluster.map_shared_rank(Ps, n);
        const float w = expf(stats[r] - used);
        const float4 x = *reinterpret_cast<const float4*>(cluster.map_shared_rank(KVs, n) + r * kLd<DH> + col);
        total = fmaf(w, stats[kRows + r], total);
        sum.x = fmaf(w, x.x, sum.x); sum.y = fmaf(w, x.y, sum.y); sum.z = fmaf(w, x.z, sum.z); sum.w = fmaf(w, x.w, sum.w);
      }
      put(r, col, sum, top, total);
    }
    cluster.sync();                                  // (nobody reads this CTA's part any more)
  }
}

// Joins the pieces of every row: W warps per row, warp w the pieces w, w + W, ...; the same order of sums in every call.  Bound by the
// latency of loads where rows are few (48 of 64 pieces each: 20 us with a warp per row), else by the L2, which the pieces come from.
template <typename T, int DH, int W>
__global__ void __launch_bounds__(256)
range_merge_kernel(const RDims D, const FastDiv by_rows, const FastDiv by_G, const FastDiv by_Hk, const FastDiv by_item, const Plan plan,
                   const FwdArgs a) {
  if (!grid_begin()) return;
  constexpr int C = DH / 32, AT_ONCE = 8;
  __shared__ float part[W > 1 ? W : 1][W > 1 ? DH + 32 : 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = warp % W;
  const int all_rows = D.B * D.Hk * D.rows;    // (at most 2^30)
  for (int row = blockIdx.x * (8 / W) + warp / W; row < all_rows; row += gridDim.x * (8 / W)) {
    const int bhk = by_rows.div(row), r = row - bhk * D.rows, tok = by_G.div(r), g = r - tok * D.G;
    const int b = by_Hk.div(bhk), head = (bhk - b * D.Hk) * D.G + g;
    const int n_pieces = __ldg(plan.pieces + (long long)mask_batch(D.Bm, b) * D.nI + by_item.div(tok));
    float lse[2], mx = -INFINITY;              // (n_pieces <= 64)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      lse[k] = lane + 32 * k < n_pieces ? __ldg(a.part_lse + (long long)(lane + 32 * k) * all_rows + row) : -INFINITY;
      mx = fmaxf(mx, lse[k]);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    const float used = mx == -INFINITY ? 0.f : mx;
#pragma unroll
    for (int k = 0; k < 2; ++k) lse[k] = expf(lse[k] - used);
    float total = 0.f, acc[C];
#pragma unroll
    for (int c = 0; c < C; ++c) acc[c] = 0.f;
    for (int s0 = sub; s0 < n_pieces; s0 += W * AT_ONCE) {
      float x[AT_ONCE][C];
#pragma unroll
      for (int k = 0; k < AT_ONCE; ++k) {
        const int s = s0 + k * W;
        const float* from = a.part_o + ((long long)s * all_rows + row) * DH + lane * C;
        if constexpr (C == 4) {
          const float4 v = s < n_pieces ? *reinterpret_cast<const float4*>(from) : make_float4(0.f, 0.f, 0.f, 0.f);
          x[k][0] = v.x; x[k][1] = v.y; x[k][2] = v.z; x[k][3] = v.w;
        } else {
          const float2 v = s < n_pieces ? *reinterpret_cast<const float2*>(from) : make_float2(0.f, 0.f);
          x[k][0] = v.x; x[k][1] = v.y;
        }
      }
#pragma unroll
      for (int k = 0; k < AT_ONCE; ++k) {
        const int s = s0 + k * W;
        const float w0 = __shfl_sync(0xffffffffu, lse[0], s & 31), w1 = __shfl_sync(0xffffffffu, lse[1], s & 31);
        const float w = s < n_pieces ? (s < 32 ? w0 : w1) : 0.f;
        total += w;
#pragma unroll
        for (int c = 0; c < C; ++c) acc[c] = fmaf(w, x[k][c], acc[c]);
      }
    }
    if constexpr (W > 1) {
      static_assert(W == 8, "a block per row");
      __syncthreads();                         // (the row before has been read)
#pragma unroll
      for (int c = 0; c < C; ++c) part[sub][lane * C + c] = acc[c];
      if (lane == 0) part[sub][DH] = total;
      __syncthreads();
      if (sub > 0) continue;
      total = 0.f;
#pragma unroll
      for (int c = 0; c < C; ++c) acc[c] = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        total += part[w][DH];
#pragma unroll
        for (int c = 0; c < C; ++c) acc[c] += part[w][lane * C + c];
      }
    }
    const bool none = total == 0.f;
    const float inv = none ? 0.f : 1.0f / total;
    T* o = reinterpret_cast<T*>(a.o) + b * a.os.b + tok * a.os.t + head * a.os.h + lane * C;
    T* resid = a.resid ? reinterpret_cast<T*>(a.resid) + (((long long)b * D.Sq + tok) * D.Hq + head) * DH + lane * C : nullptr;
#pragma unroll
    for (int c = 0; c < C; ++c) acc[c] *= inv;
    if constexpr (C == 4) {
      store4_resid(o, resid, make_float4(acc[0], acc[1], acc[2], acc[3]));
    } else {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const T h = from_f32<T>(acc[c]);
        o[c] = h;
        if (resid) resid[c] = from_f32<T>(acc[c] - to_f32<T>(h));
      }
    }
    if (lane == 0) a.lse[((long long)b * D.Hq + head) * D.Sq + tok] = none ? -INFINITY : mx + logf(total);
  }
}

// D = rowsum(dO * O) per packed row, 0 where the row sees nothing (whatever its dO holds).  zero_words: counters cleared on the way.
// A warp has four rows under way; nothing of a row's loads waits for another load (13,440 tokens x 12 heads: 51 us with the range looked at
// first and quotients by division).
template <typename T, int DH>
__global__ void __launch_bounds__(256)
range_rowdot_kernel(const RDims D, const FastDiv by_rows, const FastDiv by_G, const FastDiv by_Hk, const Plan plan, const T* __restrict__ o,
                    Strides os, const T* __restrict__ resid, const T* __restrict__ d_o, Strides dos, float* __restrict__ Dv,
                    int* __restrict__ zero_words, long long n_words) {
  if (!grid_begin()) return;
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < n_words; i += (long long)gridDim.x * blockDim.x)
    zero_words[i] = 0;
  constexpr int C = DH / 32, R = 4;            // channels per lane; rows of a warp
  const int lane = threadIdx.x & 31;
  const int all_rows = D.B * D.Hk * D.rows;    // (at most 2^30)
  for (int row0 = (blockIdx.x * 8 + (threadIdx.x >> 5)) * R; row0 < all_rows; row0 += gridDim.x * 8 * R) {
    float x[R][C], y[R][C], z[R][C];
    int seen[R];
#pragma unroll
    for (int n = 0; n < R; ++n) {
      const int row = min(row0 + n, all_rows - 1), bhk = by_rows.div(row), r = row - bhk * D.rows, tok = by_G.div(r), g = r - tok * D.G;
      const int b = by_Hk.div(bhk), head = (bhk - b * D.Hk) * D.G + g;
      seen[n] = __ldg(&plan.rows[(long long)mask_batch(D.Bm, b) * D.Sq + tok].y);
      auto get = [&](const T* from, float (&to)[C]) {
        if constexpr (C == 4) {
          const float4 v = load4(from + lane * 4);
          to[0] = v.x; to[1] = v.y; to[2] = v.z; to[3] = v.w;
        } else {
#pragma unroll
          for (int c = 0; c < C; ++c) to[c] = to_f32<T>(from[lane * C + c]);
        }
      };
      get(o + b * os.b + tok * os.t + head * os.h, x[n]);
      get(d_o + b * dos.b + tok * dos.t + head * dos.h, y[n]);
#pragma unroll
      for (int c = 0; c < C; ++c) z[n][c] = 0.f;
      if (resid) get(resid + (((long long)b * D.Sq + tok) * D.Hq + head) * DH, z[n]);
    }
    float s[R];
#pragma unroll
    for (int n = 0; n < R; ++n) {
      s[n] = 0.f;
#pragma unroll
      for (int c = 0; c < C; ++c) s[n] = fmaf(x[n][c] + z[n][c], y[n][c], s[n]);
    }
#pragma unroll
    for (int k = 16; k > 0; k >>= 1)
#pragma unroll
      for (int n = 0; n < R; ++n) s[n] += __shfl_xor_sync(0xffffffffu, s[n], k);
#pragma unroll
    for (int n = 0; n < R; ++n)
      if (lane == 0 && row0 + n < all_rows) Dv[row0 + n] = seen[n] > 0 ? s[n] : 0.f;
  }
}

// Scores of a tile as weights and slopes: p = exp(t - lse) inside the ranges, w = p (1 - (t / cap)^2).
__device__ __forceinline__ void weigh(float s, bool in, float lse, const RDims& D, float& p, float& w) {
  s *= D.scale;
  float slope = 1.f;
  if (D.cap > 0.f) {
    const float u = tanhf(s / D.cap);
    s = D.cap * u;
    slope = 1.f - u * u;
  }
  p = in ? expf(s - lse) : 0.f;
  w = in ? p * slope : 0.f;
}

// The gradients: one launch for dK / dV (an item is 64 keys of a key head, against the units that reach into them, all query heads of the
// group) and dQ (an item is a unit, against the tiles of its hull, which works S and dP out again).  Where that leaves SMs without
// an item, a cluster of C CTAs takes an item: each a C-th of what it streams, and their parts are added up through one another's shared
// memory in the order of the CTAs.  (Two samples of 256 tokens, two heads of 64: 24 items, 80 us with two launches and a CTA each, so 32.)
template <int DH> constexpr int kRangeBwdSmem = (4 * kTileFloats<DH> + kRows * kLdP) * 4;

// acc (rows 4 ty + i of a tile) of all CTAs of the cluster, summed: row r goes to put(r, column, four sums).  part: a tile in shared memory
// that nobody reads any more.
template <int DH, typename Put>
__device__ __forceinline__ void cluster_sum(int C, float (&acc)[4][DH / 16], float* part, int ty, int tx, Put put) {
  if (C == 1) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < DH / 64; ++c)
        put(4 * ty + i, 64 * c + 4 * tx, make_float4(acc[i][4 * c], acc[i][4 * c + 1], acc[i][4 * c + 2], acc[i][4 * c + 3]));
    return;
  }
  cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int c = 0; c < DH / 64; ++c)
      *reinterpret_cast<float4*>(part + (4 * ty + i) * kLd<DH> + 64 * c + 4 * tx) = make_float4(acc[i][4 * c], acc[i][4 * c + 1], acc[i][4 * c + 2], acc[i][4 * c + 3]);
  cluster.sync();
  constexpr int V = DH / 4;
  for (int e = (int)cluster.block_rank() * kThreads + threadIdx.x; e < kRows * V; e += C * kThreads) {
    const int r = e / V, col = e % V * 4;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int n = 0; n < C; ++n) {
      const float4 x = *reinterpret_cast<const float4*>(cluster.map_shared_rank(part, n) + r * kLd<DH> + col);
      a.x += x.x; a.y += x.y; a.z += x.z; a.w += x.w;
    }
    put(r, col, a);
  }
  cluster.sync();                              // (nobody reads this CTA's part any more)
}

template <typename T, int DH>
__device__ __forceinline__ void range_bwd_keys(const RDims& D, const Plan& plan, const BwdArgs& a, long long item, int rank, int C, float* smem, UnitRows& rows,
                                               float* s_lse, float* s_D) {
  float* Ks = smem;
  float* Vs = Ks + kTileFloats<DH>;
  float* Qs = Vs + kTileFloats<DH>;
  float* dOs = Qs + kTileFloats<DH>;
  float* Ps = dOs + kTileFloats<DH>;           // [key][query]: weights, then dT
  const int t = threadIdx.x, ty = t >> 4, tx = t & 15;
  const int bhk = (int)(item / D.nK), tile = (int)(item - (long long)bhk * D.nK), b = bhk / D.Hk, hk = bhk - b * D.Hk;
  const int4 info = plan.keys[(long long)mask_batch(D.Bm, b) * D.nK + tile];
  const int key0 = tile * kRows, keys = min(kRows, D.Sk - key0);
  float dk_[4][DH / 16], dv_[4][DH / 16];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int c = 0; c < DH / 16; ++c) dk_[i][c] = dv_[i][c] = 0.f;
  __syncthreads();                             // (the item before is through with the shared memory)
  {
    const T* kb = reinterpret_cast<const T*>(a.k) + b * a.ks.b + hk * a.ks.h;
    const T* vb = reinterpret_cast<const T*>(a.v) + b * a.vs.b + hk * a.vs.h;
    RowRegs<T, DH> x;
    x.fetch([&](int r) { return r >= info.z && r < info.w ? kb + (long long)(key0 + r) * a.ks.t : nullptr; });
    x.store(Ks);
    x.fetch([&](int r) { return r >= info.z && r < info.w ? vb + (long long)(key0 + r) * a.vs.t : nullptr; });
    x.store(Vs);
  }
  for (int u = info.x + rank; u < info.y; u += C) {
    if (!reaches(plan.units[(long long)mask_batch(D.Bm, b) * D.nU + u], tile, kRows)) continue;
    __syncthreads();
    load_unit(rows, D, plan, b, u);
    __syncthreads();
    if (t < kRows) {
      const int tok = rows.tok[t];
      const bool some = rows.range[t].y > 0;
      s_lse[t] = some ? a.lse[((long long)b * D.Hq + hk * D.G + t % D.G) * D.Sq + tok] : INFINITY;
      s_D[t] = some ? a.Dv[(long long)bhk * D.rows + (long long)tok * D.G + t % D.G] : 0.f;
    }
    {
      const T* qb = reinterpret_cast<const T*>(a.q) + b * a.qs.b + (long long)hk * D.G * a.qs.h;
      const T* ob = reinterpret_cast<const T*>(a.d_o) + b * a.dos.b + (long long)hk * D.G * a.dos.h;
      RowRegs<T, DH> x;
      x.fetch([&](int r) { return rows.range[r].y > 0 ? qb + rows.tok[r] * a.qs.t + (r % D.G) * a.qs.h : nullptr; });
      x.store(Qs);
      x.fetch([&](int r) { return rows.range[r].y > 0 ? ob + rows.tok[r] * a.dos.t + (r % D.G) * a.dos.h : nullptr; });
      x.store(dOs);
    }
    __syncthreads();
    float s[4][4], w[4][4];
    dot_tiles<DH>(Ks, Qs, ty, tx, kRows, s);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int r = tx + 16 * j, key = key0 + 4 * ty + i;
        const int2 rg = rows.range[r];
        weigh(s[i][j], key >= rg.x && key < rg.y, s_lse[r], D, s[i][j], w[i][j]);
        Ps[(4 * ty + i) * kLdP + r] = s[i][j];
      }
    __syncwarp();                              // (a warp reads its own eight rows)
    add_weighted<DH>(Ps, dOs, ty, tx, kRows, dv_);
    dot_tiles<DH>(Vs, dOs, ty, tx, kRows, s);
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) Ps[(4 * ty + i) * kLdP + tx + 16 * j] = w[i][j] * (s[i][j] - s_D[tx + 16 * j]);
    __syncwarp();
    add_weighted<DH>(Ps, Qs, ty, tx, kRows, dk_);
  }
  __syncthreads();                             // (K and V have been read)
  auto out = [&](void* to, const Strides& s, float scale) {
    return [=](int r, int col, const float4& x) {
      if (r < keys)
        store4(reinterpret_cast<T*>(to) + b * s.b + (long long)(key0 + r) * s.t + hk * s.h + col, make_float4(x.x * scale, x.y * scale, x.z * scale, x.w * scale));
    };
  };
  cluster_sum<DH>(C, dk_, Ks, ty, tx, out(a.dk, a.dks, D.scale));
  cluster_sum<DH>(C, dv_, Vs, ty, tx, out(a.dv, a.dvs, 1.0f));
}

template <typename T, int DH>
__device__ __forceinline__ void range_bwd_queries(const RDims& D, const Plan& plan, const BwdArgs& a, T* dq, const Strides& dqs, long long item, int rank,
                                                  int C, float* smem, UnitRows& rows) {
  float* Qs = smem;
  float* dOs = Qs + kTileFloats<DH>;
  float* Ks = dOs + kTileFloats<DH>;
  float* Vs = Ks + kTileFloats<DH>;
  float* Ps = Vs + kTileFloats<DH>;            // [query][key]: dT
  const int t = threadIdx.x, ty = t >> 4, tx = t & 15;
  const int bhk = (int)(item / D.nU), u = (int)(item - (long long)bhk * D.nU), b = bhk / D.Hk, hk = bhk - b * D.Hk;
  const int4 info = plan.units[(long long)mask_batch(D.Bm, b) * D.nU + u];
  __syncthreads();                             // (the item before is through with the shared memory)
  load_unit(rows, D, plan, b, u);
  __syncthreads();
  {
    const T* qb = reinterpret_cast<const T*>(a.q) + b * a.qs.b + (long long)hk * D.G * a.qs.h;
    const T* ob = reinterpret_cast<const T*>(a.d_o) + b * a.dos.b + (long long)hk * D.G * a.dos.h;
    RowRegs<T, DH> x;
    x.fetch([&](int r) { return rows.range[r].y > 0 ? qb + rows.tok[r] * a.qs.t + (r % D.G) * a.qs.h : nullptr; });
    x.store(Qs);
    x.fetch([&](int r) { return rows.range[r].y > 0 ? ob + rows.tok[r] * a.dos.t + (r % D.G) * a.dos.h : nullptr; });
    x.store(dOs);
  }
  float row_lse[4], row_D[4], acc[4][DH / 16];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = 4 * ty + i, tok = rows.tok[r];
    const bool some = rows.range[r].y > 0;
    row_lse[i] = some ? a.lse[((long long)b * D.Hq + hk * D.G + r % D.G) * D.Sq + tok] : INFINITY;
    row_D[i] = some ? a.Dv[(long long)bhk * D.rows + (long long)tok * D.G + r % D.G] : 0.f;
#pragma unroll
    for (int c = 0; c < DH / 16; ++c) acc[i][c] = 0.f;
  }
  const T* kb = reinterpret_cast<const T*>(a.k) + b * a.ks.b + hk * a.ks.h;
  const T* vb = reinterpret_cast<const T*>(a.v) + b * a.vs.b + hk * a.vs.h;
  for (long long t0 = info.x + (long long)rank * kRows; t0 < info.y; t0 += (long long)C * kRows) {
    const int nv = (int)min((long long)kRows, info.y - t0);
    RowRegs<T, DH> x, y;
    x.fetch([&](int r) { return r < nv ? kb + (t0 + r) * a.ks.t : nullptr; });
    y.fetch([&](int r) { return r < nv ? vb + (t0 + r) * a.vs.t : nullptr; });
    __syncthreads();
    x.store(Ks);
    y.store(Vs);
    __syncthreads();
    float p[4][4], s[4][4];
    dot_tiles<DH>(Qs, Ks, ty, tx, kRows, p);
    dot_tiles<DH>(dOs, Vs, ty, tx, kRows, s);
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int2 rg = rows.range[4 * ty + i];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int key = (int)t0 + tx + 16 * j;
        float w, none;
        weigh(p[i][j], key >= rg.x && key < rg.y, row_lse[i], D, none, w);
        Ps[(4 * ty + i) * kLdP + tx + 16 * j] = w * (s[i][j] - row_D[i]);
      }
    }
    __syncwarp();                              // (a warp reads its own eight rows)
    add_weighted<DH>(Ps, Ks, ty, tx, kRows, acc);
  }
  __syncthreads();                             // (Q has been read)
  cluster_sum<DH>(C, acc, Qs, ty, tx, [&](int r, int col, const float4& x) {
    const int tok = rows.tok[r];
    if (tok >= 0)
      store4(dq + b * dqs.b + tok * dqs.t + (long long)(hk * D.G + r % D.G) * dqs.h + col,
             make_float4(x.x * D.scale, x.y * D.scale, x.z * D.scale, x.w * D.scale));
  });
}

// A grid of whole clusters of C CTAs.
template <typename T, int DH>
__global__ void __launch_bounds__(kThreads, DH == 64 ? 2 : 1)
range_bwd_kernel(const RDims D, const Plan plan, const BwdArgs a, T* __restrict__ dq, const Strides dqs, const int C) {
  if (!grid_begin()) return;
  extern __shared__ __align__(16) float simt_smem[];
  __shared__ UnitRows rows;
  __shared__ float s_lse[kRows], s_D[kRows];
  const long long n_keys = (long long)D.B * D.Hk * D.nK, n_items = n_keys + (long long)D.B * D.Hk * D.nU;
  const int rank = blockIdx.x % C;
  for (long long item = blockIdx.x / C; item < n_items; item += gridDim.x / C) {
    if (item < n_keys) range_bwd_keys<T, DH>(D, plan, a, item, rank, C, simt_smem, rows, s_lse, s_D);
    else range_bwd_queries<T, DH>(D, plan, a, dq, dqs, item - n_keys, rank, C, simt_smem, rows);
  }
}

// ------------------------------------------------------------------------------ host
static int make_rdims(const vmoba_range_shape* s, RDims* o) {
  if (!s) return VMOBA_ERR_ARG;
  if (s->dtype != VMOBA_F32 && s->dtype != VMOBA_BF16) return VMOBA_ERR_ARG;
  if (s->B <= 0 || s->heads <= 0 || s->kv_heads <= 0 || s->Sq <= 0 || s->Sk <= 0) return VMOBA_ERR_SHAPE;
  if (s->head_dim != 64 && s->head_dim != 128) return VMOBA_ERR_SHAPE;
  if (s->heads % s->kv_heads || s->heads / s->kv_heads > 64) return VMOBA_ERR_SHAPE;
  if ((s->mask_batch != 1 && s->mask_batch != s->B) || s->mask_batch > 1 << 20) return VMOBA_ERR_SHAPE;      // (blocks of the plan)
  if (!(s->softmax_scale >= 0.f) || s->softmax_scale > 1e30f || !(s->softcap >= 0.f) || s->softcap > 1e30f) return VMOBA_ERR_ARG;
  if ((long long)s->B * s->heads > (1ll << 24) || (long long)s->B * s->heads * s->Sq > (1ll << 30) ||
      (long long)s->B * s->kv_heads * s->Sk > (1ll << 30))
    return VMOBA_ERR_SHAPE;
  o->B = s->B; o->Hq = s->heads; o->Hk = s->kv_heads; o->G = s->heads / s->kv_heads; o->d = s->head_dim;
  o->Sq = s->Sq; o->Sk = s->Sk; o->Bm = s->mask_batch; o->dtype = s->dtype;
  o->es = s->dtype == VMOBA_BF16 ? 2 : 4;
  o->scale = s->softmax_scale > 0.f ? s->softmax_scale : 1.0f / sqrtf((float)s->head_dim);
  o->cap = s->softcap;
  o->tc = o->dtype == VMOBA_BF16 && o->d == 128;
  o->TR = o->tc ? 128 : 64;
  o->tpt = o->TR / o->G;
  o->rows = s->Sq * o->G;
  o->nU = (s->Sq + o->tpt - 1) / o->tpt;
  o->nK = (s->Sk + o->TR - 1) / o->TR;
  o->nI = o->tc ? (o->nU + 1) / 2 : o->nU;
  // Fewer items than four for every SM: they are cut, where there is something to cut (a tile takes the tensor cores 2 us, the CUDA cores 4,
  // joining the pieces 5 to 10), eight pieces per SM at most on average and 64 of an item.  On the CUDA cores clusters do the same without
  // that, where eight CTAs for each item fill the SMs and there are up to eight tiles for every SM (fp32, heads of 64, 900 tokens x 2 heads: 45 us
  // in pieces, 29 by clusters; one token x 2 heads against 900 keys: 14 and 18; 1,200 queries x 4 heads of 128 against 1,900 keys: 196 and 288).
  const long long items = (long long)s->B * s->kv_heads * o->nI;
  const bool clusters = !o->tc && 8 * items >= kSms && items * o->nK <= 8 * kSms;
  o->smax = 1;
  if (items < kFewItems && o->nK >= 8 && !clusters) o->smax = (int)std::min<long long>(std::min(64, o->nK), (8 * kSms + items - 1) / items);
  o->reps = s->mask_batch == 1 ? s->B * s->kv_heads : s->kv_heads;
  return VMOBA_OK;
}

static Plan carve_plan(const RDims& D, const void* mem, size_t* bytes) {
  Carver c(const_cast<void*>(mem));
  Plan p = {};
  p.rows = c.take<int2>((size_t)D.Bm * D.Sq);
  p.units = c.take<int4>((size_t)D.Bm * D.nU);
  p.keys = c.take<int4>((size_t)D.Bm * D.nK);
  p.runs = c.take<int4>((size_t)D.Bm * D.nK);
  p.order = c.take<int>((size_t)D.Bm * D.nI);
  p.head = c.take<int>(2);
  if (D.smax > 1) {
    p.pieces = c.take<int>((size_t)D.Bm * D.nI);
    p.work = c.take<int4>((size_t)D.Bm * D.nI * D.smax);
  }
  if (bytes) *bytes = c.total();
  return p;
}

struct FwdWs { float *part_o, *part_lse; size_t bytes; Guards guards; };
static FwdWs carve_fwd(const RDims& D, void* ws) {
  Carver c(ws);
  FwdWs w = {};
  const size_t rows = (size_t)D.B * D.Hk * D.rows;
  if (D.smax > 1) {
    w.part_lse = c.take<float>(rows * D.smax);
    w.part_o = c.take<float>(rows * D.smax * D.d);
  }
  w.bytes = std::max<size_t>(c.total(), 256);
  w.guards = c.guards;
  return w;
}

struct BwdWs { float *Dv, *dq_acc; int* turns; size_t bytes; Guards guards; };
static BwdWs carve_bwd(const RDims& D, void* ws) {
  Carver c(ws);
  BwdWs w = {};
  w.Dv = c.take<float>((size_t)D.B * D.Hk * D.rows);
  if (D.tc) {
    w.dq_acc = c.take<float>((size_t)D.B * D.Hk * D.rows * D.d * tc_range_bwd_parts(D));
    w.turns = c.take<int>((size_t)tc_range_bwd_turns(D));
  }
  w.bytes = c.total();
  w.guards = c.guards;
  return w;
}

// Element strides of a tensor [B, S, heads, d]; those of dimensions of size one address nothing and are taken for dense ones.
static bool get_strides(const RDims& D, const int64_t s[3], int S, int heads, Strides* o) {
  if (!s) return false;
  const int per = 16 / D.es;
  long long st[3] = {s[0], s[1], s[2]};
  const int n[3] = {D.B, S, heads};
  if (heads == 1) st[2] = D.d;
  if (S == 1) st[1] = (long long)heads * D.d;
  if (D.B == 1) st[0] = (long long)S * heads * D.d;
  for (int i = 0; i < 3; ++i)
    if (st[i] < 0 || st[i] % per || (n[i] > 1 && st[i] < D.d) || st[i] > (1ll << 38)) return false;
  *o = {st[0], st[1], st[2]};
  return true;
}

static int grid_for(long long items, int per_sm) {
  return (int)std::max<long long>(1, std::min<long long>(items, (long long)sm_count() * per_sm));
}

// As for the CUDA-core kernels of the dense path: several of their CTAs share an SM, and long ones are not launched early.
static bool early_simt(const RDims& D) { return (double)D.B * D.Hq * D.Sq * D.Sk * D.d <= (double)(1 << 25); }
static bool early_rows(const RDims& D) { return (long long)D.B * D.Hq * D.Sq * D.d * D.es <= (16ll << 20); }

template <typename T, int DH>
static int forward(const RDims& D, const Plan& plan, FwdArgs a, cudaStream_t st) {
  if constexpr (sizeof(T) == 2 && DH == 128) {
    if (int rc = tc_range_fwd(D, plan, a, st)) return rc;
  } else {
    const long long items = (long long)D.B * D.Hk * D.nI * D.smax;
    VMOBA_CUDA_OK(allow_smem(range_fwd_kernel<T, DH>, simt::kFwdSmem<DH>));
    int C = 1;
    if (D.smax == 1)
      while (C < 8 && items * C * 2 <= 2 * kSms && D.nK >= 2 * C) C *= 2;
    if (C > 1)
      launch_cluster(early_simt(D), C, range_fwd_kernel<T, DH>, (int)items * C, kThreads, simt::kFwdSmem<DH>, st, D, plan, a, C);
    else
      launch_kernel(early_simt(D), range_fwd_kernel<T, DH>, grid_for(items, 8), kThreads, simt::kFwdSmem<DH>, st, D, plan, a, C);
    VMOBA_LAUNCH_OK(1);
  }
  if (D.smax > 1) {
    const long long rows = (long long)D.B * D.Hk * D.rows;
    const FastDiv by_rows(D.rows), by_G(D.G), by_Hk(D.Hk), by_item(D.tpt * (D.tc ? 2 : 1));
    if (rows <= 8 * kSms)                      // (a block per row, all of them at once)
      launch_kernel(early_rows(D), range_merge_kernel<T, DH, 8>, (int)rows, 256, 0, st, D, by_rows, by_G, by_Hk, by_item, plan, a);
    else
      launch_kernel(early_rows(D), range_merge_kernel<T, DH, 1>, grid_for((rows + 7) / 8, 16), 256, 0, st, D, by_rows, by_G, by_Hk, by_item,
                    plan, a);
    VMOBA_LAUNCH_OK(1);
  }
  return VMOBA_OK;
}

template <typename T, int DH>
static int backward(const RDims& D, const Plan& plan, const BwdArgs& a, const void* o, const Strides& os, const void* resid, float* Dv,
                    void* dq, const Strides& dqs, cudaStream_t st) {
  const long long all_rows = (long long)D.B * D.Hk * D.rows;
  launch_kernel(early_rows(D), range_rowdot_kernel<T, DH>, grid_for((all_rows + 31) / 32, 16), 256, 0, st, D, FastDiv(D.rows),
                FastDiv(D.G), FastDiv(D.Hk), plan, (const T*)o, os,
                (const T*)resid, (const T*)a.d_o, a.dos, Dv, a.turns, a.turns ? tc_range_bwd_turns(D) : 0ll);
  VMOBA_LAUNCH_OK(1);
  if constexpr (sizeof(T) == 2 && DH == 128) {
    return tc_range_bwd(D, plan, a, dq, dqs, early_rows(D), st);
  } else {
    VMOBA_CUDA_OK(allow_smem(range_bwd_kernel<T, DH>, kRangeBwdSmem<DH>));
    const long long items = (long long)D.B * D.Hk * (D.nK + D.nU), room = (long long)kSms * (DH == 64 ? 2 : 1);
    // The items that stream the most decide; of the others, which are short then, more come one after another.  (Room for all items at once
    // instead: 500 tokens x 2, eight heads of 64 on one key head, bf16, 469 us, so 158; 600 tokens, four of 128 on one, fp32, 363 and 124; but
    // 100 queries x 2 heads of 64 against 1,500 keys, fp32, 81 and 91.)
    const long long longest = (long long)D.B * D.Hk * std::min(D.nK, D.nU);
    int C = 1;
    while (C < 8 && longest * C * 2 <= room && std::max(D.nU, D.nK) >= 2 * C) C *= 2;
    const int grid = C * (int)std::max<long long>(1, std::min<long long>(items, (long long)sm_count() * 4 / C));
    if (C > 1) launch_cluster(early_simt(D), C, range_bwd_kernel<T, DH>, grid, kThreads, kRangeBwdSmem<DH>, st, D, plan, a, (T*)dq, dqs, C);
    else launch_kernel(early_simt(D), range_bwd_kernel<T, DH>, grid, kThreads, kRangeBwdSmem<DH>, st, D, plan, a, (T*)dq, dqs, C);
    VMOBA_LAUNCH_OK(1);
    return VMOBA_OK;
  }
}

#define VMOBA_RANGE_DISPATCH(rc, FN, ...)                                              \
  do {                                                                                 \
    if (D.dtype == VMOBA_BF16) {                                                       \
      rc = D.d == 128 ? FN<__nv_bfloat16, 128>(__VA_ARGS__) : FN<__nv_bfloat16, 64>(__VA_ARGS__); \
    } else {                                                                           \
      rc = D.d == 128 ? FN<float, 128>(__VA_ARGS__) : FN<float, 64>(__VA_ARGS__);      \
    }                                                                                  \
  } while (0)

}  // namespace range
}  // namespace vmoba

using namespace vmoba;
using namespace vmoba::range;

extern "C" size_t vmoba_range_plan_bytes(const vmoba_range_shape* shape) {
  RDims D;
  if (make_rdims(shape, &D)) return 0;
  size_t bytes;
  carve_plan(D, nullptr, &bytes);
  return bytes;
}

extern "C" int vmoba_range_plan(const vmoba_range_shape* shape, const int32_t* key_range, void* plan, size_t plan_bytes,
                                void* stream) {
  RDims D;
  if (int rc = make_rdims(shape, &D)) return rc;
  if (!key_range || !plan || !aligned16(plan) || (reinterpret_cast<uintptr_t>(key_range) & 7u)) return VMOBA_ERR_ARG;
  size_t need;
  const Plan p = carve_plan(D, plan, &need);
  if (plan_bytes < need) return VMOBA_ERR_WORKSPACE;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  launch_kernel(plan_units_kernel, grid_for(((long long)D.Bm * D.nU + 7) / 8, 8), 256, 0, st, reinterpret_cast<const int2*>(key_range), p, D);
  const long long tile_blocks = std::min<long long>(((long long)D.Bm * D.nK + 31) / 32, 2ll * sm_count());
  launch_kernel(plan_tiles_kernel, (unsigned)(D.Bm + 1 + tile_blocks), 1024, 0, st, p, D);
  VMOBA_LAUNCH_OK(2);
  return VMOBA_OK;
}

extern "C" size_t vmoba_range_workspace_bytes(const vmoba_range_shape* shape, int backward) {
  RDims D;
  if (make_rdims(shape, &D) || (backward != 0 && backward != 1)) return 0;
  return backward ? carve_bwd(D, nullptr).bytes : carve_fwd(D, nullptr).bytes;
}

extern "C" int vmoba_range_attn_fwd(const vmoba_range_shape* shape, const void* plan, const void* q, const int64_t q_strides[3],
                                    const void* k, const int64_t k_strides[3], const void* v, const int64_t v_strides[3], void* o,
                                    const int64_t o_strides[3], void* o_resid_or_null, float* lse, int32_t* dev_status, void* ws,
                                    size_t ws_bytes, void* stream) {
  RDims D;
  if (int rc = make_rdims(shape, &D)) return rc;
  if (!plan || !q || !k || !v || !o || !lse || !dev_status || !ws) return VMOBA_ERR_ARG;
  if (!aligned16(plan) || !aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o) || !aligned16(ws) || !aligned16(o_resid_or_null))
    return VMOBA_ERR_ARG;
  FwdArgs a = {};
  if (!get_strides(D, q_strides, D.Sq, D.Hq, &a.qs) || !get_strides(D, k_strides, D.Sk, D.Hk, &a.ks) ||
      !get_strides(D, v_strides, D.Sk, D.Hk, &a.vs) || !get_strides(D, o_strides, D.Sq, D.Hq, &a.os))
    return VMOBA_ERR_ARG;
  FwdWs w = carve_fwd(D, ws);
  if (ws_bytes < w.bytes) return VMOBA_ERR_WORKSPACE;
  a.q = q; a.k = k; a.v = v; a.o = o; a.resid = D.dtype == VMOBA_BF16 ? o_resid_or_null : nullptr; a.lse = lse;
  a.part_o = w.part_o; a.part_lse = w.part_lse; a.status = dev_status;
  const Plan p = carve_plan(D, plan, nullptr);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  VMOBA_GUARDS_ARM(w.guards, st);
  int rc;
  VMOBA_RANGE_DISPATCH(rc, forward, D, p, a, st);
  VMOBA_GUARDS_CHECK(w.guards, dev_status, st);
  return rc;
}

extern "C" int vmoba_range_attn_bwd(const vmoba_range_shape* shape, const void* plan, const void* q, const int64_t q_strides[3],
                                    const void* k, const int64_t k_strides[3], const void* v, const int64_t v_strides[3], const void* o,
                                    const int64_t o_strides[3], const void* o_resid_or_null, const float* lse, const void* d_o,
                                    const int64_t do_strides[3], void* dq, const int64_t dq_strides[3], void* dk,
                                    const int64_t dk_strides[3], void* dv, const int64_t dv_strides[3], int32_t* dev_status, void* ws,
                                    size_t ws_bytes, void* stream) {
  RDims D;
  if (int rc = make_rdims(shape, &D)) return rc;
  if (!plan || !q || !k || !v || !o || !lse || !d_o || !dq || !dk || !dv || !dev_status || !ws) return VMOBA_ERR_ARG;
  if (!aligned16(plan) || !aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o) || !aligned16(o_resid_or_null) ||
      !aligned16(d_o) || !aligned16(dq) || !aligned16(dk) || !aligned16(dv) || !aligned16(ws))
    return VMOBA_ERR_ARG;
  BwdArgs a = {};
  Strides os, dqs;
  if (!get_strides(D, q_strides, D.Sq, D.Hq, &a.qs) || !get_strides(D, k_strides, D.Sk, D.Hk, &a.ks) ||
      !get_strides(D, v_strides, D.Sk, D.Hk, &a.vs) || !get_strides(D, o_strides, D.Sq, D.Hq, &os) ||
      !get_strides(D, do_strides, D.Sq, D.Hq, &a.dos) || !get_strides(D, dq_strides, D.Sq, D.Hq, &dqs) ||
      !get_strides(D, dk_strides, D.Sk, D.Hk, &a.dks) || !get_strides(D, dv_strides, D.Sk, D.Hk, &a.dvs))
    return VMOBA_ERR_ARG;
  BwdWs w = carve_bwd(D, ws);
  if (ws_bytes < w.bytes) return VMOBA_ERR_WORKSPACE;
  a.q = q; a.k = k; a.v = v; a.d_o = d_o; a.lse = lse; a.Dv = w.Dv; a.dk = dk; a.dv = dv; a.status = dev_status;
  a.dq_acc = w.dq_acc; a.turns = w.turns;
  if (D.tc) a.parts = tc_range_bwd_parts(D);
  if (D.dtype != VMOBA_BF16) o_resid_or_null = nullptr;
  const Plan p = carve_plan(D, plan, nullptr);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  VMOBA_GUARDS_ARM(w.guards, st);
  int rc;
  VMOBA_RANGE_DISPATCH(rc, backward, D, p, a, o, os, o_resid_or_null, w.Dv, dq, dqs, st);
  VMOBA_GUARDS_CHECK(w.guards, dev_status, st);
  return rc;
}
