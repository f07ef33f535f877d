// What stands between two branches of a transformer block, in one pass over a token's channels, and its gradients in another.
//   z = y or post(y) * wp,   h = x + gate * z,   n = norm(h),   out = (n * w + b) * (1 + scale) + shift
// Backward, with dm = d_out (1 + scale) and r the norm's factor (1 / sqrt(var + eps)):
//   dh = d_h + r (dm w - n mean(dm w n) [- mean(dm w)]),   dz = gate * dh,   dy = dz, or through the post norm in the same way
//   with, per group of tokens that share a row of scale, shift and gate,   A = sum d_out n,   D = sum d_out,   E = sum dh post(y):
//   dscale = w A + b D,  dshift = D,  dgate = wp E,   dw = sum over groups (1 + scale) A,  db = sum (1 + scale) D,  dwp = sum gate E.
// Bound by HBM: forward x and y in, h and out out; backward d_out, d_h, h and y in, dx and dy out.  So rows come through a ring in shared
// memory, a bulk copy per tensor, and stay on the SM between the norms' trips through them; a thread keeps its channels over all rows of its
// CTA's chunk of a group, so that scale, shift and gate are loaded once and A, D and E add up in registers.  The chunks' sums are added by a second kernel in
// a fixed order.  Variances are taken about the mean of a thread's channels, and those means and variances put together.
#include <algorithm>

#include "linear.cuh"

namespace vmoba {
namespace norm {

using linear::load_vec;
using linear::store_vec;

constexpr int kMostChannels = 8192;
// Threads of a CTA that has a piece of eight channels for each: by the registers that many leave (85 and 102 each).  The backward has 128 with
// 256 threads at most, for four rows at a time on two CTAs of an SM (1,536 channels, 32,760 rows: 123 us; three CTAs with 102
// registers and two rows at a time: 157).  More channels than either has threads for are two pieces a thread, 512 threads at most: there the backward's 128
// registers leave 140 to 252 bytes of spills (8,192 channels, 4,000 rows: 196 us, 2.0 TB/s; 5,120 and 13,440: 184 us, 4.5).
constexpr int kFwdThreads = 768, kBwdThreads = 640, kBwdNarrow = 256;

struct Rows {
  const void* p;
  long long sb, st;
};
struct Params {
  int S, G, gt, C, pieces;
  int norm, post;
  float eps, mean;                           // mean: 1 / C
  Rows x, y, h, out;                         // forward; backward: h, y
  Rows d_out, d_h, dx, dy;
  const float *gate, *scale, *shift;
  long long gate_s[2], scale_s[2], shift_s[2];
  const float *weight, *bias, *post_weight;
  int cpg, chunk;                            // chunks per group, rows of a chunk
  int batch, stage_dh;                       // rows of a batch; whether d_h goes through the ring
  float* part;                               // [chunk][3][C]
  int32_t* status;
};

template <typename T>
__device__ __forceinline__ T* row_of(const Rows& r, int b, int t) {
  return static_cast<T*>(const_cast<void*>(r.p)) + b * r.sb + t * r.st;
}

__device__ __forceinline__ float warp_sum(float a) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
  return a;
}
__device__ __forceinline__ float2 warp_sum(float2 a) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    a.x += __shfl_xor_sync(0xffffffffu, a.x, o);
    a.y += __shfl_xor_sync(0xffffffffu, a.y, o);
  }
  return a;
}
// Eight channels at a time, in pairs: d = a b + c with a number or another piece for b and c.
struct Same { float v; __device__ __forceinline__ float operator[](int) const { return v; } };
template <typename B, typename C>
__device__ __forceinline__ void fma8(float (&d)[8], const float (&a)[8], const B& b, const C& c) {
#pragma unroll
  for (int k = 0; k < 8; k += 2) sm100::fma2(d[k], d[k + 1], a[k], a[k + 1], b[k], b[k + 1], c[k], c[k + 1]);
}
template <typename B>
__device__ __forceinline__ void mul8(float (&d)[8], const float (&a)[8], const B& b) {
#pragma unroll
  for (int k = 0; k < 8; k += 2) sm100::mul2(d[k], d[k + 1], a[k], a[k + 1], b[k], b[k + 1]);
}
template <typename B>
__device__ __forceinline__ void add8(float (&d)[8], const float (&a)[8], const B& b) {
#pragma unroll
  for (int k = 0; k < 8; k += 2) sm100::add2(d[k], d[k + 1], a[k], a[k + 1], b[k], b[k + 1]);
}
// s += a . b, and s += sum of a, in two halves
__device__ __forceinline__ void dot8(float2& s, const float (&a)[8], const float (&b)[8]) {
#pragma unroll
  for (int k = 0; k < 8; k += 2) sm100::fma2(s.x, s.y, a[k], a[k + 1], b[k], b[k + 1], s.x, s.y);
}
__device__ __forceinline__ void sum8(float2& s, const float (&a)[8]) {
#pragma unroll
  for (int k = 0; k < 8; k += 2) sm100::add2(s.x, s.y, s.x, s.y, a[k], a[k + 1]);
}

__device__ __forceinline__ void bulk_copy(uint32_t to, const void* from, uint32_t size, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to), "l"(from), "r"(size),
               "r"(sm100::smem_u32(bar))
               : "memory");
}

// What the kernels share.  A CTA takes the rows of one chunk of a group, a few at a time (a batch; the next one is on its way into the other half
// of the ring), a thread the same channels of all of them, so that scale, shift and gate are loaded once.  What a row's sums need of a
// thread's channels goes to shared memory, a warp adds up each row, and the threads go on with the sums: no lane adds up with
// another but in those warps.

// The rows of a CTA.
struct Chunk {
  int b, g, t0, t1;
  __device__ __forceinline__ explicit Chunk(const Params& p) {
    const int gi = blockIdx.x / p.cpg, j = blockIdx.x - gi * p.cpg;
    b = gi / p.G;
    g = gi - b * p.G;
    t0 = g * p.gt + j * p.chunk;
    t1 = min(min(t0 + p.chunk, (g + 1) * p.gt), p.S);
  }
};

// Sums of a row, of parts that the threads' channels give.
template <int P>
struct Sums {
  const Params& p;
  const int tpr;
  __device__ __forceinline__ explicit Sums(const Params& p) : p(p), tpr(blockDim.x) {}
  // channels of thread i
  __device__ __forceinline__ float n_of(int i) const {
    int n = 0;
#pragma unroll
    for (int k = 0; k < P; ++k) n += i + k * tpr < p.pieces;
    return 8.f * (float)n;
  }
  // a thread's channels of a row (0 where there are none): their sum and the sum of squares about their mean (about 0: root mean square)
  __device__ __forceinline__ float2 part(bool centred, const float (&v)[P][8], const bool (&mine)[P], float inv_n) const {
    float2 s = make_float2(0.f, 0.f), q = s;
    float mean = 0.f;
    if (centred) {
#pragma unroll
      for (int i = 0; i < P; ++i) sum8(s, v[i]);
      mean = (s.x + s.y) * inv_n;
    }
#pragma unroll
    for (int i = 0; i < P; ++i)
      if (P == 1 || mine[i]) {
        float d[8];
        add8(d, v[i], Same{-mean});
        dot8(q, d, d);
      }
    return make_float2(s.x + s.y, q.x + q.y);
  }
  // (one warp) mean and 1 / sqrt(variance + eps) of a row from the threads' parts
  __device__ __forceinline__ float2 stat(bool centred, const float2* part) const {
    const int lane = threadIdx.x & 31;
    float s = 0.f, q = 0.f;
    for (int i = lane; i < tpr; i += 32) { const float2 a = part[i]; s += a.x; q += a.y; }
    if (centred) {
      s = warp_sum(s) * p.mean;
      for (int i = lane; i < tpr; i += 32) {
        const float n = n_of(i), d = n > 0.f ? part[i].x * (P == 1 ? 0.125f : __fdividef(1.f, n)) - s : 0.f;
        q = fmaf(n * d, d, q);
      }
    }
    return make_float2(centred ? s : 0.f, 1.f / sqrtf(warp_sum(q) * p.mean + p.eps));
  }
  __device__ __forceinline__ float2 means(const float2* part) const {
    float2 s = make_float2(0.f, 0.f);
    for (int i = threadIdx.x & 31; i < tpr; i += 32) { const float2 a = part[i]; s.x += a.x; s.y += a.y; }
    s = warp_sum(s);
    return make_float2(s.x * p.mean, s.y * p.mean);
  }
};

// TS: the stream's type, T: the branch's.  P: pieces of eight channels per thread.
template <typename TS, typename T, int P, bool POST>
__global__ void __launch_bounds__(P == 1 ? kFwdThreads : 512, 1) norm_fwd_kernel(Params p) {
  if (!grid_begin()) return;
  constexpr int NB = P == 1 ? 4 : 2;
  extern __shared__ __align__(128) char s_rows[];
  __shared__ float2 s_stat[2][NB];
  __shared__ uint64_t s_full[2];
  __shared__ int s_abort;
  const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5, lane = threadIdx.x & 31, l = threadIdx.x, tpr = blockDim.x;
  const Chunk at(p);
  const Sums<P> sums(p);
  const bool layer = p.norm == VMOBA_NORM_LAYER, y_layer = POST && p.post == VMOBA_NORM_LAYER;
  const uint32_t bs = (uint32_t)p.C * sizeof(TS), bt = p.y.p ? (uint32_t)p.C * sizeof(T) : 0u, stride = (bs + bt + 127u) & ~127u;
  float2* const s_part = reinterpret_cast<float2*>(s_rows + 2 * p.batch * stride);      // [row][thread]
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) sm100::mbar_init(&s_full[i], 1);
    s_abort = 0;
    sm100::fence_barrier_init();
  }
  __syncthreads();
  auto ask = [&](int k) {                    // (one thread) for batch k
    const int first = at.t0 + k * p.batch, n = min(p.batch, at.t1 - first);
    if (n <= 0) return;
    uint64_t* bar = &s_full[k & 1];
    sm100::mbar_expect_tx(bar, (uint32_t)n * (bs + bt));
    uint32_t to = sm100::smem_u32(s_rows) + (k & 1) * p.batch * stride;
    for (int t = first; t < first + n; ++t, to += stride) {
      bulk_copy(to, row_of<const TS>(p.x, at.b, t), bs, bar);
      if (bt) bulk_copy(to + bs, row_of<const T>(p.y, at.b, t), bt, bar);
    }
  };
  if (threadIdx.x == 0) { ask(0); ask(1); }
  float fg[P][8], fm[P][8], fs[P][8];        // gate * post weight; (1 + scale) * weight; (1 + scale) * bias + shift
  bool mine[P];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int c = 8 * (l + i * tpr);
    mine[i] = c < p.C;
#pragma unroll
    for (int q = 0; q < 8; ++q) { fm[i][q] = fg[i][q] = 1.f; fs[i][q] = 0.f; }
    if (!mine[i]) continue;
    float f[8];
    if (p.gate) load_vec<8>(p.gate + at.b * p.gate_s[0] + at.g * p.gate_s[1] + c, fg[i]);
    if (p.post_weight) {
      load_vec<8>(p.post_weight + c, f);
      mul8(fg[i], fg[i], f);
    }
    if (p.scale) {
      load_vec<8>(p.scale + at.b * p.scale_s[0] + at.g * p.scale_s[1] + c, f);
      add8(fm[i], fm[i], f);
    }
    if (p.shift) load_vec<8>(p.shift + at.b * p.shift_s[0] + at.g * p.shift_s[1] + c, fs[i]);
    if (p.bias) {
      load_vec<8>(p.bias + c, f);
      fma8(fs[i], f, fm[i], fs[i]);
    }
    if (p.weight) {
      load_vec<8>(p.weight + c, f);
      mul8(fm[i], fm[i], f);
    }
  }
  const float inv_n = 1.f / fmaxf(sums.n_of(l), 1.f);
  const int batches = (at.t1 - at.t0 + p.batch - 1) / p.batch;
  for (int k = 0; k < batches; ++k) {
    const int first = at.t0 + k * p.batch, n = min(p.batch, at.t1 - first);
    const char* half = s_rows + (k & 1) * p.batch * stride;
    sm100::mbar_wait(&s_full[k & 1], (k >> 1) & 1, &s_abort, p.status);
    __syncwarp();
    if (POST) {
#pragma unroll
      for (int r = 0; r < NB; ++r) {
        if (r >= n) break;
        float y[P][8] = {};
#pragma unroll
        for (int i = 0; i < P; ++i)
          if (mine[i]) load_vec<8>(reinterpret_cast<const T*>(half + r * stride + bs) + 8 * (l + i * tpr), y[i]);
        s_part[r * tpr + l] = sums.part(y_layer, y, mine, inv_n);
      }
      __syncthreads();
      for (int r = warp; r < n; r += warps) {
        const float2 s = sums.stat(y_layer, s_part + r * tpr);
        if (lane == 0) s_stat[0][r] = s;
      }
      __syncthreads();
    }
    float h[NB][P][8];
#pragma unroll
    for (int r = 0; r < NB; ++r) {
      if (r >= n) break;
      const char* row = half + r * stride;
      const float2 sy = POST ? s_stat[0][r] : make_float2(0.f, 1.f);
      TS* h_row = row_of<TS>(p.h, at.b, first + r);
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const int c = 8 * (l + i * tpr);
        if (!mine[i]) {
#pragma unroll
          for (int q = 0; q < 8; ++q) h[r][i][q] = 0.f;
          continue;
        }
        load_vec<8>(reinterpret_cast<const TS*>(row) + c, h[r][i]);
        if (p.y.p) {
          float y[8];
          load_vec<8>(reinterpret_cast<const T*>(row + bs) + c, y);
          if (POST) {
            add8(y, y, Same{-sy.x});
            mul8(y, y, Same{sy.y});
          }
          fma8(h[r][i], y, fg[i], h[r][i]);
        }
        if (p.h.p) store_vec<8>(h_row + c, h[r][i]);
      }
      if (p.out.p) s_part[r * tpr + l] = sums.part(layer, h[r], mine, inv_n);
    }
    sm100::fence_async_proxy();              // (the thread's reads of the batch come ahead of the copy that takes its place, ..
    __syncthreads();                         //  .. all of them)
    if (threadIdx.x == 0) ask(k + 2);
    if (!p.out.p) continue;
    for (int r = warp; r < n; r += warps) {
      const float2 s = sums.stat(layer, s_part + r * tpr);
      if (lane == 0) s_stat[1][r] = s;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < NB; ++r) {
      if (r >= n) break;
      const float2 s = s_stat[1][r];
      T* out_row = row_of<T>(p.out, at.b, first + r);
#pragma unroll
      for (int i = 0; i < P; ++i) {
        if (!mine[i]) continue;
        float o[8];
        add8(o, h[r][i], Same{-s.x});
        mul8(o, o, Same{s.y});
        fma8(o, o, fm[i], fs[i]);
        store_vec<8>(out_row + 8 * (l + i * tpr), o);
      }
    }
  }
}

// (The backward with all warps adding up every row across their lanes: 3,400 instructions a row of 1,536 channels, 347 us for 32,760 of them; with
// a warp going through a whole row for its sums: 2,290 and 206 us; as it is: 1,720 and 123.)
struct alignas(16) RowSums { float mean, factor, along, level, y_mean, y_factor, y_along, y_level; };

template <typename TS, typename T, int P, bool POST, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == 256 ? 2 : 1) norm_bwd_kernel(Params p) {
  if (!grid_begin()) return;
  constexpr int NB = THREADS == 256 ? 4 : 2;
  extern __shared__ __align__(128) char s_rows[];
  __shared__ RowSums s_sums[NB];
  __shared__ uint64_t s_full[2];
  __shared__ int s_abort;
  const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5, lane = threadIdx.x & 31, l = threadIdx.x, tpr = blockDim.x;
  const Chunk chunk(p);
  const int b = chunk.b, g = chunk.g, t0 = chunk.t0, t1 = chunk.t1;
  const Sums<P> sums(p);
  const bool dh_here = p.stage_dh != 0, layer = p.norm == VMOBA_NORM_LAYER, y_layer = POST && p.post == VMOBA_NORM_LAYER;
  // bytes of a row of the stream's and of the branch's type; places in a slot: h, d_out, y, d_h; behind the ring the threads' parts of sums
  const uint32_t bs = (uint32_t)p.C * sizeof(TS), bt = (uint32_t)p.C * sizeof(T);
  const uint32_t at_d = bs, at_y = at_d + bt, at_dh = at_y + (p.y.p ? bt : 0u);
  const uint32_t bytes = at_dh + (dh_here ? bs : 0u), stride = (bytes + 127u) & ~127u;
  float2* const s_part = reinterpret_cast<float2*>(s_rows + 2 * p.batch * stride);      // [row][thread], and again for y
  float2* const s_part_y = s_part + p.batch * tpr;
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) sm100::mbar_init(&s_full[i], 1);
    s_abort = 0;
    sm100::fence_barrier_init();
  }
  __syncthreads();
  auto ask = [&](int k) {                    // (one thread) for batch k
    const int first = t0 + k * p.batch, n = min(p.batch, t1 - first);
    if (n <= 0) return;
    uint64_t* bar = &s_full[k & 1];
    sm100::mbar_expect_tx(bar, (uint32_t)n * bytes);
    uint32_t to = sm100::smem_u32(s_rows) + (k & 1) * p.batch * stride;
    for (int t = first; t < first + n; ++t, to += stride) {
      bulk_copy(to, row_of<const TS>(p.h, b, t), bs, bar);
      bulk_copy(to + at_d, row_of<const T>(p.d_out, b, t), bt, bar);
      if (p.y.p) bulk_copy(to + at_y, row_of<const T>(p.y, b, t), bt, bar);
      if (dh_here) bulk_copy(to + at_dh, row_of<const TS>(p.d_h, b, t), bs, bar);
    }
  };
  if (threadIdx.x == 0) { ask(0); ask(1); }
  float A[P][8] = {}, D[P][8] = {}, E[P][8] = {}, fm[P][8], fg[P][8];      // (1 + scale) * weight, gate * post weight
  bool mine[P];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int c = 8 * (l + i * tpr);
    mine[i] = c < p.C;
#pragma unroll
    for (int k = 0; k < 8; ++k) fm[i][k] = fg[i][k] = 1.f;
    if (!mine[i]) continue;
    float f[8];
    if (p.scale) {
      load_vec<8>(p.scale + b * p.scale_s[0] + g * p.scale_s[1] + c, f);
      add8(fm[i], fm[i], f);
    }
    if (p.weight) {
      load_vec<8>(p.weight + c, f);
      mul8(fm[i], fm[i], f);
    }
    if (p.gate) load_vec<8>(p.gate + b * p.gate_s[0] + g * p.gate_s[1] + c, fg[i]);
    if (p.post_weight) {
      load_vec<8>(p.post_weight + c, f);
      mul8(fg[i], fg[i], f);
    }
  }
  const float inv_n = 1.f / fmaxf(sums.n_of(l), 1.f);
  const int batches = (t1 - t0 + p.batch - 1) / p.batch;
  for (int k = 0; k < batches; ++k) {
    const int first = t0 + k * p.batch, n = min(p.batch, t1 - first);
    const char* half = s_rows + (k & 1) * p.batch * stride;
    sm100::mbar_wait(&s_full[k & 1], (k >> 1) & 1, &s_abort, p.status);
    __syncwarp();
    float h[NB][P][8];
    // ---- means and variances
#pragma unroll
    for (int r = 0; r < NB; ++r) {
      if (r >= n) break;
      const char* row = half + r * stride;
#pragma unroll
      for (int i = 0; i < P; ++i) {
        if (mine[i]) load_vec<8>(reinterpret_cast<const TS*>(row) + 8 * (l + i * tpr), h[r][i]);
        else
#pragma unroll
          for (int q = 0; q < 8; ++q) h[r][i][q] = 0.f;
      }
      s_part[r * tpr + l] = sums.part(layer, h[r], mine, inv_n);
      if (POST) {
        float y[P][8];
#pragma unroll
        for (int i = 0; i < P; ++i) {
          if (mine[i]) load_vec<8>(reinterpret_cast<const T*>(row + at_y) + 8 * (l + i * tpr), y[i]);
          else
#pragma unroll
            for (int q = 0; q < 8; ++q) y[i][q] = 0.f;
        }
        s_part_y[r * tpr + l] = sums.part(y_layer, y, mine, inv_n);
      }
    }
    __syncthreads();
    for (int r = warp; r < (POST ? 2 * n : n); r += warps) {
      RowSums& o = s_sums[r >= n ? r - n : r];
      if (r < n) {
        const float2 s = sums.stat(layer, s_part + r * tpr);
        if (lane == 0) { o.mean = s.x; o.factor = s.y; }
      } else {
        const float2 s = sums.stat(y_layer, s_part_y + (r - n) * tpr);
        if (lane == 0) { o.y_mean = s.x; o.y_factor = s.y; }
      }
    }
    __syncthreads();
    // ---- the norm's gradient: how much of it lies along n, and its level
#pragma unroll
    for (int r = 0; r < NB; ++r) {
      if (r >= n) break;
      const char* row = half + r * stride;
      const float mean = s_sums[r].mean, factor = s_sums[r].factor;
      float2 a = make_float2(0.f, 0.f), c = a;
#pragma unroll
      for (int i = 0; i < P; ++i) {
        if (!mine[i]) continue;
        float d[8];
        load_vec<8>(reinterpret_cast<const T*>(row + at_d) + 8 * (l + i * tpr), d);
        fma8(h[r][i], h[r][i], Same{factor}, Same{-mean * factor});
        fma8(A[i], d, h[r][i], A[i]);
        add8(D[i], D[i], d);
        mul8(d, d, fm[i]);
        dot8(a, d, h[r][i]);
        if (layer) sum8(c, d);
      }
      s_part[r * tpr + l] = make_float2(a.x + a.y, c.x + c.y);
    }
    __syncthreads();
    for (int r = warp; r < n; r += warps) {
      const float2 s = sums.means(s_part + r * tpr);
      if (lane == 0) { s_sums[r].along = s.x; s_sums[r].level = s.y; }
    }
    __syncthreads();
    // ---- dx, and without a post norm dy
#pragma unroll
    for (int r = 0; r < NB; ++r) {
      if (r >= n) break;
      const char* row = half + r * stride;
      const RowSums o = s_sums[r];
      TS* dx_row = row_of<TS>(p.dx, b, first + r);
      float2 a = make_float2(0.f, 0.f), c2 = a;
#pragma unroll
      for (int i = 0; i < P; ++i) {
        if (!mine[i]) continue;
        const int c = 8 * (l + i * tpr);
        float d[8], dh[8] = {};
        load_vec<8>(reinterpret_cast<const T*>(row + at_d) + c, d);
        if (dh_here) load_vec<8>(reinterpret_cast<const TS*>(row + at_dh) + c, dh);
        else if (p.d_h.p) load_vec<8>(row_of<const TS>(p.d_h, b, first + r) + c, dh);
        mul8(d, d, fm[i]);
        if (layer) add8(d, d, Same{-o.level});
        fma8(d, h[r][i], Same{-o.along}, d);
        fma8(dh, d, Same{o.factor}, dh);
        store_vec<8>(dx_row + c, dh);
        if (p.y.p) {
          float y[8];
          load_vec<8>(reinterpret_cast<const T*>(row + at_y) + c, y);
          if (POST) fma8(y, y, Same{o.y_factor}, Same{-o.y_mean * o.y_factor});
          fma8(E[i], dh, y, E[i]);
          mul8(dh, dh, fg[i]);
          if (POST) {
            dot8(a, dh, y);
            if (y_layer) sum8(c2, dh);
#pragma unroll
            for (int q = 0; q < 8; ++q) h[r][i][q] = dh[q];       // (n has done its work)
          } else if (p.dy.p) {
            store_vec<8>(row_of<T>(p.dy, b, first + r) + c, dh);
          }
        }
      }
      if (POST) s_part[r * tpr + l] = make_float2(a.x + a.y, c2.x + c2.y);
    }
    if (POST && p.dy.p) {
      __syncthreads();
      for (int r = warp; r < n; r += warps) {
        const float2 s = sums.means(s_part + r * tpr);
        if (lane == 0) { s_sums[r].y_along = s.x; s_sums[r].y_level = s.y; }
      }
      __syncthreads();
#pragma unroll
      for (int r = 0; r < NB; ++r) {
        if (r >= n) break;
        const RowSums o = s_sums[r];
        T* dy_row = row_of<T>(p.dy, b, first + r);
#pragma unroll
        for (int i = 0; i < P; ++i) {
          if (!mine[i]) continue;
          const int c = 8 * (l + i * tpr);
          float y[8];
          load_vec<8>(reinterpret_cast<const T*>(half + r * stride + at_y) + c, y);
          fma8(y, y, Same{o.y_factor}, Same{-o.y_mean * o.y_factor});
          fma8(y, y, Same{-o.y_along}, h[r][i]);
          if (y_layer) add8(y, y, Same{-o.y_level});
          mul8(y, y, Same{o.y_factor});
          store_vec<8>(dy_row + c, y);
        }
      }
    }
    sm100::fence_async_proxy();              // (as in the forward)
    __syncthreads();
    if (threadIdx.x == 0) ask(k + 2);
  }
  if (!p.part) return;
  float* part = p.part + (long long)blockIdx.x * 3 * p.C;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    if (!mine[i]) continue;
    const int c = 8 * (l + i * tpr);
    store_vec<8>(part + c, A[i]);
    store_vec<8>(part + p.C + c, D[i]);
    store_vec<8>(part + 2 * p.C + c, E[i]);
  }
}

struct GroupSums {
  int C, G, cpg, tiles;
  const float* part;
  float* by_group;                           // [group][3][C], for the vectors' gradients
  const float *weight, *bias, *post_weight;
  float *dgate, *dscale, *dshift;
};
// A CTA has 32 channels of a group, a warp every eighth chunk.
__global__ void __launch_bounds__(256) group_sums_kernel(GroupSums p) {
  if (!grid_begin()) return;
  __shared__ float s[3][8][33];
  const int g = blockIdx.x / p.tiles, lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = (blockIdx.x - g * p.tiles) * 32 + lane;
  float a[3] = {};
  if (c < p.C) {
    const float* from = p.part + (long long)g * p.cpg * 3 * p.C + c;
#pragma unroll 4
    for (int i = w; i < p.cpg; i += 8)
#pragma unroll
      for (int k = 0; k < 3; ++k) a[k] += from[((long long)i * 3 + k) * p.C];
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) s[k][w][lane] = a[k];
  __syncthreads();
  if (w != 0 || c >= p.C) return;
#pragma unroll
  for (int k = 0; k < 3; ++k)
#pragma unroll
    for (int i = 1; i < 8; ++i) a[k] += s[k][i][lane];
  const long long at = (long long)g * p.C + c;
  if (p.dscale) p.dscale[at] = a[0] * (p.weight ? __ldg(p.weight + c) : 1.f) + a[1] * (p.bias ? __ldg(p.bias + c) : 0.f);
  if (p.dshift) p.dshift[at] = a[1];
  if (p.dgate) p.dgate[at] = a[2] * (p.post_weight ? __ldg(p.post_weight + c) : 1.f);
  if (p.by_group)
#pragma unroll
    for (int k = 0; k < 3; ++k) p.by_group[((long long)g * 3 + k) * p.C + c] = a[k];
}

struct Vectors {
  int C, G, groups;                          // groups: of all samples
  const float *by_group, *gate, *scale;
  long long gate_s[2], scale_s[2];
  float *dweight, *dbias, *dpost;
};
__global__ void __launch_bounds__(256) vector_sums_kernel(Vectors p) {
  if (!grid_begin()) return;
  __shared__ float s[3][8][33];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  float a[3] = {};
  if (c < p.C) {
#pragma unroll 4
    for (int gi = w; gi < p.groups; gi += 8) {
      const int b = gi / p.G, g = gi - b * p.G;
      const float* from = p.by_group + (long long)gi * 3 * p.C + c;
      const float m = p.scale ? 1.f + __ldg(p.scale + b * p.scale_s[0] + g * p.scale_s[1] + c) : 1.f;
      const float f = p.gate ? __ldg(p.gate + b * p.gate_s[0] + g * p.gate_s[1] + c) : 1.f;
      a[0] = fmaf(__ldg(from), m, a[0]);
      a[1] = fmaf(__ldg(from + p.C), m, a[1]);
      a[2] = fmaf(__ldg(from + 2 * p.C), f, a[2]);
    }
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) s[k][w][lane] = a[k];
  __syncthreads();
  if (w != 0 || c >= p.C) return;
  float* const to[3] = {p.dweight, p.dbias, p.dpost};
#pragma unroll
  for (int k = 0; k < 3; ++k) {
#pragma unroll
    for (int i = 1; i < 8; ++i) a[k] += s[k][i][lane];
    if (to[k]) to[k][c] = a[k];
  }
}

// ---------------------------------------------------------------- host
struct Dims {
  int B, S, C, gt, G;
  bool bf16, stream_bf16;
};

static int make_dims(const vmoba_norm_shape* s, Dims* o) {
  if (!s) return VMOBA_ERR_ARG;
  for (int t : {s->dtype, s->stream_dtype})
    if (t != VMOBA_F32 && t != VMOBA_BF16) return VMOBA_ERR_ARG;
  if (s->norm != VMOBA_NORM_RMS && s->norm != VMOBA_NORM_LAYER) return VMOBA_ERR_ARG;
  if (s->post_norm < VMOBA_NORM_NONE || s->post_norm > VMOBA_NORM_LAYER || s->mod_tokens < 0 || !(s->eps >= 0.f) || s->eps > 1e30f) return VMOBA_ERR_ARG;
  if (s->B <= 0 || s->S <= 0 || s->C <= 0 || s->C % 8 || s->C > kMostChannels || (long long)s->B * s->S > (1ll << 30)) return VMOBA_ERR_SHAPE;
  if (s->dtype == VMOBA_F32 && s->stream_dtype == VMOBA_BF16) return VMOBA_ERR_NOT_IMPLEMENTED;
  o->B = s->B; o->S = s->S; o->C = s->C;
  o->gt = s->mod_tokens && s->mod_tokens < s->S ? s->mod_tokens : s->S;
  o->G = (s->S + o->gt - 1) / o->gt;
  o->bf16 = s->dtype == VMOBA_BF16; o->stream_bf16 = s->stream_dtype == VMOBA_BF16;
  return VMOBA_OK;
}

// Whether rows of a tensor (null: not there) can be addressed, and their strides.
static bool take(Rows* r, const void* p, const int64_t* st, const Dims& D, bool bf16, bool written) {
  *r = Rows{p, 0, 0};
  if (!p) return true;
  if (!st || !aligned16(p)) return false;
  const int n[2] = {D.B, D.S};
  for (int i = 0; i < 2; ++i) {
    if (n[i] == 1) continue;
    if (st[i] % (bf16 ? 8 : 4) || (!(st[i] == 0 && !written) && st[i] < D.C) || st[i] >= (1ll << 38)) return false;
  }
  r->sb = D.B > 1 ? st[0] : 0;
  r->st = D.S > 1 ? st[1] : 0;
  return true;
}
static bool take_params(Params* p, const vmoba_norm_params* m, const Dims& D) {
  const float* rows[3] = {m->gate, m->scale, m->shift};
  const int64_t* st[3] = {m->gate_strides, m->scale_strides, m->shift_strides};
  long long* to[3] = {p->gate_s, p->scale_s, p->shift_s};
  const int n[2] = {D.B, D.G};
  for (int k = 0; k < 3; ++k) {
    if (!rows[k]) continue;
    if (!aligned16(rows[k])) return false;
    for (int i = 0; i < 2; ++i) {
      if (n[i] > 1 && (st[k][i] % 4 || (st[k][i] != 0 && st[k][i] < D.C) || st[k][i] >= (1ll << 38))) return false;
      to[k][i] = n[i] > 1 ? st[k][i] : 0;
    }
  }
  if (!aligned16(m->weight) || !aligned16(m->bias) || !aligned16(m->post_weight)) return false;
  p->gate = m->gate; p->scale = m->scale; p->shift = m->shift;
  p->weight = m->weight; p->bias = m->bias; p->post_weight = m->post_weight;
  return true;
}
static Params params_of(const vmoba_norm_shape* s, const Dims& D) {
  Params p = {};
  p.S = D.S; p.G = D.G; p.gt = D.gt; p.C = D.C; p.pieces = D.C / 8;
  p.norm = s->norm; p.post = s->post_norm; p.eps = s->eps; p.mean = 1.f / (float)D.C;
  return p;
}

// Threads of a CTA, how many CTAs there are on an SM (of `warps` in all), and how the rows of a group are cut.
constexpr int kSms = 148, kFwdWarps = 24, kBwdWarps = 16;
struct Cut { int threads, pieces, ctas, cpg, chunk; long long chunks; };
static Cut cut_of(const Dims& D, int warps, int threads) {
  Cut c;
  const int pieces = D.C / 8;
  c.pieces = pieces <= threads ? 1 : 2;
  c.threads = ((pieces + c.pieces - 1) / c.pieces + 31) / 32 * 32;
  c.ctas = std::max(1, warps / (c.threads / 32));
  const long long run = (long long)kSms * c.ctas, groups = (long long)D.B * D.G;
  // chunks per group: the number whose rounds of CTAs take least, in rows (a chunk's beginning and end are worth about eight)
  long long least = INT64_MAX;
  c.chunk = D.gt;
  for (int rounds = 1; rounds <= 4; ++rounds) {
    const long long n = std::max<long long>(1, std::min<long long>(D.gt, rounds * run / groups)), rows = (D.gt + n - 1) / n;
    const long long cost = ((groups * ((D.gt + rows - 1) / rows) + run - 1) / run) * (rows + 8);
    if (cost < least) { least = cost; c.chunk = (int)rows; }
  }
  c.cpg = (D.gt + c.chunk - 1) / c.chunk;
  c.chunks = groups * c.cpg;
  return c;
}
struct Scratch { float *part, *by_group; Guards guards; size_t bytes; };
static Scratch scratch_of(const Dims& D, void* ws) {
  Carver c(ws);
  Scratch s;
  s.part = c.take<float>((size_t)cut_of(D, kBwdWarps, kBwdThreads).chunks * 3 * D.C);
  s.by_group = c.take<float>((size_t)D.B * D.G * 3 * D.C);
  s.guards = c.guards;
  s.bytes = c.total();
  return s;
}

template <typename TS, typename T>
static int go_fwd(const Dims& D, Params& p, cudaStream_t st) {
  const Cut c = cut_of(D, kFwdWarps, kFwdThreads);
  p.cpg = c.cpg; p.chunk = c.chunk;
  const size_t bytes = align_up((size_t)p.C * (sizeof(TS) + (p.y.p ? sizeof(T) : 0)), 128), parts = (size_t)c.threads * sizeof(float2);
  p.batch = (int)std::min<size_t>(c.pieces == 1 ? 4 : 2, std::max<size_t>(1, kSmemMost / c.ctas / (2 * bytes + parts)));
  auto go = [&](auto kernel) -> int {
    VMOBA_CUDA_OK(allow_smem(kernel, kSmemMost));
    launch_kernel(kernel, (unsigned)c.chunks, c.threads, p.batch * (2 * bytes + parts), st, p);
    VMOBA_LAUNCH_OK(1);
    return VMOBA_OK;
  };
  const bool post = p.y.p && p.post != VMOBA_NORM_NONE;
  if (c.pieces == 1) return post ? go(norm_fwd_kernel<TS, T, 1, true>) : go(norm_fwd_kernel<TS, T, 1, false>);
  return post ? go(norm_fwd_kernel<TS, T, 2, true>) : go(norm_fwd_kernel<TS, T, 2, false>);
}
template <typename TS, typename T>
static int go_bwd(const Cut& c, Params& p, cudaStream_t st) {
  p.cpg = c.cpg; p.chunk = c.chunk;
  // two rows at least in the ring and their parts behind it, d_h not through it where those would not fit (fp32, more than 6,880 channels)
  auto slot = [&](bool dh) {
    return align_up((size_t)p.C * ((dh ? 2 : 1) * sizeof(TS) + (p.y.p ? 2 : 1) * sizeof(T)), 128);
  };
  const size_t parts = (size_t)c.threads * 2 * sizeof(float2);
  static_assert(2 * kMostChannels * (sizeof(TS) + 2 * sizeof(T)) + 512 * 2 * sizeof(float2) <= kSmemMost, "rows without d_h always fit");
  p.stage_dh = p.d_h.p && 2 * slot(true) + parts <= (size_t)kSmemMost;
  const size_t bytes = slot(p.stage_dh != 0);
  p.batch = (int)std::min<size_t>(c.threads <= kBwdNarrow && c.pieces == 1 ? 4 : 2, std::max<size_t>(1, kSmemMost / c.ctas / (2 * bytes + parts)));
  auto go = [&](auto kernel) -> int {
    VMOBA_CUDA_OK(allow_smem(kernel, kSmemMost));
    launch_kernel(kernel, (unsigned)c.chunks, c.threads, p.batch * (2 * bytes + parts), st, p);
    VMOBA_LAUNCH_OK(1);
    return VMOBA_OK;
  };
  const bool post = p.y.p && p.post != VMOBA_NORM_NONE;
  if (c.pieces == 2) return post ? go(norm_bwd_kernel<TS, T, 2, true, 512>) : go(norm_bwd_kernel<TS, T, 2, false, 512>);
  if (c.threads <= kBwdNarrow) return post ? go(norm_bwd_kernel<TS, T, 1, true, kBwdNarrow>) : go(norm_bwd_kernel<TS, T, 1, false, kBwdNarrow>);
  return post ? go(norm_bwd_kernel<TS, T, 1, true, kBwdThreads>) : go(norm_bwd_kernel<TS, T, 1, false, kBwdThreads>);
}

}  // namespace norm
}  // namespace vmoba

using namespace vmoba;

extern "C" size_t vmoba_block_norm_workspace_bytes(const vmoba_norm_shape* shape) {
  norm::Dims D;
  return norm::make_dims(shape, &D) ? 0 : norm::scratch_of(D, nullptr).bytes;
}

extern "C" int vmoba_block_norm(const vmoba_norm_shape* shape, const vmoba_norm_params* params, const void* x, const int64_t x_strides[2],
                                const void* y, const int64_t y_strides[2], void* h, const int64_t h_strides[2], void* out,
                                const int64_t out_strides[2], int32_t* dev_status, void* stream) {
  norm::Dims D;
  if (int rc = norm::make_dims(shape, &D)) return rc;
  if (!params || !x || (!h && !out)) return VMOBA_ERR_ARG;
  norm::Params p = norm::params_of(shape, D);
  if (!norm::take_params(&p, params, D) || !norm::take(&p.x, x, x_strides, D, D.stream_bf16, false) ||
      !norm::take(&p.y, y, y_strides, D, D.bf16, false) || !norm::take(&p.h, h, h_strides, D, D.stream_bf16, true) ||
      !norm::take(&p.out, out, out_strides, D, D.bf16, true))
    return VMOBA_ERR_ARG;
  p.status = dev_status;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (!D.bf16) return norm::go_fwd<float, float>(D, p, st);
  return D.stream_bf16 ? norm::go_fwd<__nv_bfloat16, __nv_bfloat16>(D, p, st) : norm::go_fwd<float, __nv_bfloat16>(D, p, st);
}

extern "C" int vmoba_block_norm_bwd(const vmoba_norm_shape* shape, const vmoba_norm_params* params, const void* d_out,
                                    const int64_t d_out_strides[2], const void* h, const int64_t h_strides[2], const void* d_h,
                                    const int64_t d_h_strides[2], const void* y, const int64_t y_strides[2], void* dx,
                                    const int64_t dx_strides[2], void* dy, const int64_t dy_strides[2], const vmoba_norm_grads* grads,
                                    int32_t* dev_status, void* ws, size_t ws_bytes, void* stream) {
  norm::Dims D;
  if (int rc = norm::make_dims(shape, &D)) return rc;
  if (!params || !grads || !d_out || !h || !dx || !ws || !aligned16(ws) || (dy && !y)) return VMOBA_ERR_ARG;
  norm::Params p = norm::params_of(shape, D);
  if (!norm::take_params(&p, params, D) || !norm::take(&p.d_out, d_out, d_out_strides, D, D.bf16, false) ||
      !norm::take(&p.h, h, h_strides, D, D.stream_bf16, false) || !norm::take(&p.d_h, d_h, d_h_strides, D, D.stream_bf16, false) ||
      !norm::take(&p.y, y, y_strides, D, D.bf16, false) || !norm::take(&p.dx, dx, dx_strides, D, D.stream_bf16, true) ||
      !norm::take(&p.dy, dy, dy_strides, D, D.bf16, true))
    return VMOBA_ERR_ARG;
  // (a gradient of what is not there)
  if ((grads->gate && (!params->gate || !y)) || (grads->scale && !params->scale) || (grads->shift && !params->shift) ||
      (grads->weight && !params->weight) || (grads->bias && !params->bias) || (grads->post_weight && (!params->post_weight || !y)))
    return VMOBA_ERR_ARG;
  if (!aligned16(grads->gate) || !aligned16(grads->scale) || !aligned16(grads->shift) || !aligned16(grads->weight) ||
      !aligned16(grads->bias) || !aligned16(grads->post_weight))
    return VMOBA_ERR_ARG;
  const norm::Scratch s = norm::scratch_of(D, ws);
  if (ws_bytes < s.bytes) return VMOBA_ERR_WORKSPACE;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const norm::Cut cut = norm::cut_of(D, norm::kBwdWarps, norm::kBwdThreads);
  const bool vectors = grads->weight || grads->bias || grads->post_weight;
  const bool rows = grads->gate || grads->scale || grads->shift;
  p.part = vectors || rows ? s.part : nullptr;
  p.status = dev_status;
  VMOBA_GUARDS_ARM(s.guards, st);
  int rc;
  if (!D.bf16) rc = norm::go_bwd<float, float>(cut, p, st);
  else rc = D.stream_bf16 ? norm::go_bwd<__nv_bfloat16, __nv_bfloat16>(cut, p, st) : norm::go_bwd<float, __nv_bfloat16>(cut, p, st);
  if (rc) return rc;
  if (p.part) {
    const int tiles = (D.C + 31) / 32;
    const long long ctas = (long long)D.B * D.G * tiles;
    if (ctas > INT32_MAX) return VMOBA_ERR_SHAPE;
    const norm::GroupSums a{D.C, D.G, cut.cpg, tiles, s.part, vectors ? s.by_group : nullptr, p.weight, p.bias, p.post_weight, grads->gate,
                       grads->scale, grads->shift};
    launch_kernel(norm::group_sums_kernel, (unsigned)ctas, 256, 0, st, a);
    VMOBA_LAUNCH_OK(1);
    if (vectors) {
      norm::Vectors v{D.C, D.G, D.B * D.G, s.by_group, p.gate, p.scale, {}, {}, grads->weight, grads->bias, grads->post_weight};
      for (int i = 0; i < 2; ++i) { v.gate_s[i] = p.gate_s[i]; v.scale_s[i] = p.scale_s[i]; }
      launch_kernel(norm::vector_sums_kernel, (unsigned)tiles, 256, 0, st, v);
      VMOBA_LAUNCH_OK(1);
    }
  }
  VMOBA_GUARDS_CHECK(s.guards, dev_status, st);
  return VMOBA_OK;
}
