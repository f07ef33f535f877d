// What stands between two branches of a transformer block, in one pass over a token's channels, and its gradients in another.
//   z = y or post(y) * wp,   h = x + gate * z,   n = norm(h),   out = (n * w + b) * (1 + scale) + shift
// Backward, with dm = d_out (1 + scale) and r the norm's factor (1 / sqrt(var + eps)):
//   dh = d_h + r (dm w - n mean(dm w n) [- mean(dm w)]),   dz = gate * dh,   dy = dz, or through the post norm in the same way
//   with, per group of tokens that share a row of scale, shift and gate,   A = sum d_out n,   D = sum d_out,   E = sum dh post(y):
//   dscale = w A + b D,  dshift = D,  dgate = wp E,   dw = sum over groups (1 + scale) A,  db = sum (1 + scale) D,  dwp = sum gate E.
// Bound by HBM: forward x and y in, h and out out; backward d_out, d_h, h and y in, dx and dy out.  So a row stays on the SM between the norms'
// trips through it.  Forward, a row is taken by as few warps as hold it in three 8-channel pieces per thread, in registers, each group of warps on its
// own.  Backward, a thread keeps its channels over all rows of its CTA's chunk of a group, so that A, D and E add up in registers and scale and
// gate are loaded once; the rows come through a ring in shared memory, a bulk copy per tensor, so that the sums over a row (two meetings of the
// CTA, three with a post norm) wait for no memory.  The chunks' sums are added by a second kernel in a fixed order.
// Variances are taken about the mean of a warp's channels, and the warps' means and variances put together.
#include <algorithm>

#include "linear.cuh"

namespace vmoba {
namespace norm {

using linear::load_vec;
using linear::store_vec;

constexpr int kMostChannels = 8192;
constexpr int kFwdPieces = 3, kFwdWarps = 8;

struct Rows {
  const void* p;
  long long sb, st;
};
struct Params {
  int B, S, G, gt, C, pieces, rows;
  int norm, post;
  FastDiv by_S, by_gt;
  float eps, mean;                           // mean: 1 / C
  Rows x, y, h, out;                         // forward; backward: h, y
  Rows d_out, d_h, dx, dy;
  const float *gate, *scale, *shift;
  long long gate_s[2], scale_s[2], shift_s[2];
  const float *weight, *bias, *post_weight;
  int wpr, groups;                           // forward: warps per row, rows that a CTA has under way
  int cpg, chunk;                            // backward: chunks per group, rows of a chunk
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
__device__ __forceinline__ void meet(int barrier, int warps) {
  asm volatile("bar.sync %0, %1;" ::"r"(barrier), "r"(32 * warps) : "memory");
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

// Mean (0 for a root-mean-square norm) and 1 / sqrt(variance + eps) of a row, from those of its warps' channels.
struct Stat { float mean, factor; };
// What a warp has to say of its channels: their sum and the sum of squares about their mean (about 0: root mean square); n of them.
template <int P>
__device__ __forceinline__ float2 warp_stat(int kind, const float (&v)[P][8], const bool (&mine)[P], float n) {
  float s = 0.f, q = 0.f;
  if (kind == VMOBA_NORM_LAYER) {
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
      for (int k = 0; k < 8; ++k) s += v[i][k];            // (0 where there are no channels)
    s = warp_sum(s);
  }
  const float mean = n > 0.f ? __fdividef(s, n) : 0.f;
#pragma unroll
  for (int i = 0; i < P; ++i)
    if (mine[i])
#pragma unroll
      for (int k = 0; k < 8; ++k) { const float d = v[i][k] - mean; q = fmaf(d, d, q); }
  return make_float2(s, warp_sum(q));
}
// n_of: the number of channels of a warp.
template <typename N>
__device__ __forceinline__ Stat put_together(int kind, const float2* slot, int warps, N n_of, float inv_c, float eps) {
  float s = 0.f, q = 0.f;
  for (int w = 0; w < warps; ++w) { const float2 a = slot[w]; s += a.x; q += a.y; }
  const float mean = s * inv_c;
  if (kind == VMOBA_NORM_LAYER && warps > 1)
    for (int w = 0; w < warps; ++w) {
      const float n = n_of(w);
      if (n > 0.f) { const float d = __fdividef(slot[w].x, n) - mean; q = fmaf(n * d, d, q); }
    }
  return {kind == VMOBA_NORM_LAYER ? mean : 0.f, 1.f / sqrtf(q * inv_c + eps)};
}

// CTAs of the forward on an SM, by the registers of P pieces per thread.
__host__ __device__ constexpr int fwd_ctas(int P) { return P == 1 ? 4 : P <= 3 ? 3 : 2; }

// TS: the stream's type, T: the branch's.  P: pieces per thread.
template <typename TS, typename T, int P>
__global__ void __launch_bounds__(32 * kFwdWarps, fwd_ctas(P)) norm_fwd_kernel(Params p) {
  if (!grid_begin()) return;
  __shared__ float2 s_slots[2][2][kFwdWarps];
  const int group = (threadIdx.x >> 5) / p.wpr, warp = (threadIdx.x >> 5) - group * p.wpr, tpr = 32 * p.wpr;
  const int l = threadIdx.x - group * tpr;
  bool mine[P];
#pragma unroll
  for (int i = 0; i < P; ++i) mine[i] = 8 * (l + i * tpr) < p.C;
  // pieces of warp w: 32 of every run of tpr, as far as there are any
  auto n_of = [&](int w) {
    int n = 0;
#pragma unroll
    for (int i = 0; i < P; ++i) n += min(max(p.pieces - 32 * w - i * tpr, 0), 32);
    return 8.f * (float)n;
  };
  const float n_mine = n_of(warp);
  int turn = 0;                              // (a row may have a single meeting: the next one's numbers go elsewhere)
  auto stat = [&](int kind, const float (&v)[P][8], int which) {
    const float2 a = warp_stat<P>(kind, v, mine, n_mine);
    if (p.wpr == 1) return put_together(kind, &a, 1, n_of, p.mean, p.eps);
    float2* slot = &s_slots[turn][which][group * p.wpr];
    if ((threadIdx.x & 31) == 0) slot[warp] = a;
    meet(1 + group, p.wpr);
    return put_together(kind, slot, p.wpr, n_of, p.mean, p.eps);
  };
  for (int r = blockIdx.x * p.groups + group; r < p.rows; r += gridDim.x * p.groups, turn ^= 1) {
    const int b = p.by_S.div(r), t = r - b * p.S, g = p.by_gt.div(t);
    float h[P][8];
    const TS* x_row = row_of<const TS>(p.x, b, t);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      if (mine[i]) load_vec<8>(x_row + 8 * (l + i * tpr), h[i]);
      else
#pragma unroll
        for (int k = 0; k < 8; ++k) h[i][k] = 0.f;
    }
    if (p.y.p) {
      const T* y_row = row_of<const T>(p.y, b, t);
      float y[P][8];
#pragma unroll
      for (int i = 0; i < P; ++i) {
        if (mine[i]) load_vec<8>(y_row + 8 * (l + i * tpr), y[i]);
        else
#pragma unroll
          for (int k = 0; k < 8; ++k) y[i][k] = 0.f;
      }
      if (p.post != VMOBA_NORM_NONE) {
        const Stat s = stat(p.post, y, 0);
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
          for (int k = 0; k < 8; ++k) y[i][k] = (y[i][k] - s.mean) * s.factor;
      }
      const float* gate = p.gate ? p.gate + b * p.gate_s[0] + g * p.gate_s[1] : nullptr;
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const int c = 8 * (l + i * tpr);
        if (!mine[i]) continue;
        float f[8];
        if (p.post_weight) {
          load_vec<8>(p.post_weight + c, f);
#pragma unroll
          for (int k = 0; k < 8; ++k) y[i][k] *= f[k];
        }
        if (gate) {
          load_vec<8>(gate + c, f);
#pragma unroll
          for (int k = 0; k < 8; ++k) h[i][k] = fmaf(y[i][k], f[k], h[i][k]);
        } else {
#pragma unroll
          for (int k = 0; k < 8; ++k) h[i][k] += y[i][k];
        }
      }
    }
    if (p.h.p) {
      TS* h_row = row_of<TS>(p.h, b, t);
#pragma unroll
      for (int i = 0; i < P; ++i)
        if (mine[i]) store_vec<8>(h_row + 8 * (l + i * tpr), h[i]);
    }
    if (!p.out.p) continue;
    const Stat s = stat(p.norm, h, 1);
    const float* scale = p.scale ? p.scale + b * p.scale_s[0] + g * p.scale_s[1] : nullptr;
    const float* shift = p.shift ? p.shift + b * p.shift_s[0] + g * p.shift_s[1] : nullptr;
    T* out_row = row_of<T>(p.out, b, t);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int c = 8 * (l + i * tpr);
      if (!mine[i]) continue;
      float f[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) h[i][k] = (h[i][k] - s.mean) * s.factor;
      if (p.weight) {
        load_vec<8>(p.weight + c, f);
#pragma unroll
        for (int k = 0; k < 8; ++k) h[i][k] *= f[k];
      }
      if (p.bias) {
        load_vec<8>(p.bias + c, f);
#pragma unroll
        for (int k = 0; k < 8; ++k) h[i][k] += f[k];
      }
      if (scale) {
        load_vec<8>(scale + c, f);
#pragma unroll
        for (int k = 0; k < 8; ++k) h[i][k] = fmaf(h[i][k], f[k], h[i][k]);
      }
      if (shift) {
        load_vec<8>(shift + c, f);
#pragma unroll
        for (int k = 0; k < 8; ++k) h[i][k] += f[k];
      }
      store_vec<8>(out_row + c, h[i]);
    }
  }
}

// Backward.  A CTA takes the rows of one chunk, a few at a time (a batch; the next one is on its way into the other half of the ring), a thread the
// same channels of all of them.  What a row's sums need of a thread's channels goes to shared memory, a warp adds up each row, and the
// threads go on with the sums: no lane adds up with another but in those warps.  (All warps adding up every row across their lanes: 3,400
// instructions a row of 1,536 channels, 347 us for 32,760 of them; a warp going through a whole row for its sums: 2,290 and 206 us.)
__host__ __device__ constexpr int batch_rows(int P) { return P == 1 ? 4 : 2; }
struct alignas(16) RowSums { float mean, factor, along, level, y_mean, y_factor, y_along, y_level; };

template <typename TS, typename T, int P, bool POST>
__global__ void __launch_bounds__(P == 1 ? 256 : 512, P == 1 ? 2 : 1) norm_bwd_kernel(Params p) {
  if (!grid_begin()) return;
  constexpr int NB = batch_rows(P);
  extern __shared__ __align__(128) char s_rows[];
  __shared__ RowSums s_sums[NB];
  __shared__ uint64_t s_full[2];
  __shared__ int s_abort;
  const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5, lane = threadIdx.x & 31, l = threadIdx.x, tpr = blockDim.x;
  const int gi = blockIdx.x / p.cpg, j = blockIdx.x - gi * p.cpg, b = gi / p.G, g = gi - b * p.G;
  const int t0 = g * p.gt + j * p.chunk, t1 = min(min(t0 + p.chunk, (g + 1) * p.gt), p.S);
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
    auto copy = [&](uint32_t at, const void* from, uint32_t size) {
      asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to + at), "l"(from), "r"(size),
                   "r"(sm100::smem_u32(bar))
                   : "memory");
    };
    for (int t = first; t < first + n; ++t, to += stride) {
      copy(0, row_of<const TS>(p.h, b, t), bs);
      copy(at_d, row_of<const T>(p.d_out, b, t), bt);
      if (p.y.p) copy(at_y, row_of<const T>(p.y, b, t), bt);
      if (dh_here) copy(at_dh, row_of<const TS>(p.d_h, b, t), bs);
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
  // Channels of thread i, and their number over 8 of this one.
  auto n_of = [&](int i) {
    int n = 0;
#pragma unroll
    for (int k = 0; k < P; ++k) n += i + k * tpr < p.pieces;
    return 8.f * (float)n;
  };
  const float inv_n = 1.f / fmaxf(n_of(l), 1.f);
  // a thread's channels of a row: their sum and the sum of squares about their mean (about 0: root mean square)
  auto part_of = [&](bool centred, const float (&v)[P][8]) {
    float2 s = make_float2(0.f, 0.f), q = s;
    float mean = 0.f;
    if (centred) {
#pragma unroll
      for (int i = 0; i < P; ++i) sum8(s, v[i]);           // (0 where there are no channels)
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
  };
  // (one warp) mean and 1 / sqrt(variance + eps) of a row from the threads' parts
  auto stat_of = [&](bool centred, const float2* part, float* mean, float* factor) {
    float s = 0.f, q = 0.f;
    for (int i = lane; i < tpr; i += 32) { const float2 a = part[i]; s += a.x; q += a.y; }
    if (centred) {
      s = warp_sum(s) * p.mean;
      for (int i = lane; i < tpr; i += 32) {
        const float n = n_of(i), d = n > 0.f ? part[i].x * (P == 1 ? 0.125f : __fdividef(1.f, n)) - s : 0.f;
        q = fmaf(n * d, d, q);
      }
    }
    if (lane == 0) *mean = centred ? s : 0.f;
    *factor = 1.f / sqrtf(warp_sum(q) * p.mean + p.eps);
  };
  auto means_of = [&](const float2* part) {  // (one warp)
    float2 s = make_float2(0.f, 0.f);
    for (int i = lane; i < tpr; i += 32) { const float2 a = part[i]; s.x += a.x; s.y += a.y; }
    s = warp_sum(s);
    return make_float2(s.x * p.mean, s.y * p.mean);
  };
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
      s_part[r * tpr + l] = part_of(layer, h[r]);
      if (POST) {
        float y[P][8];
#pragma unroll
        for (int i = 0; i < P; ++i) {
          if (mine[i]) load_vec<8>(reinterpret_cast<const T*>(row + at_y) + 8 * (l + i * tpr), y[i]);
          else
#pragma unroll
            for (int q = 0; q < 8; ++q) y[i][q] = 0.f;
        }
        s_part_y[r * tpr + l] = part_of(y_layer, y);
      }
    }
    __syncthreads();
    for (int r = warp; r < (POST ? 2 * n : n); r += warps) {
      RowSums& o = s_sums[r >= n ? r - n : r];
      float factor;
      if (r < n) {
        stat_of(layer, s_part + r * tpr, &o.mean, &factor);
        if (lane == 0) o.factor = factor;
      } else {
        stat_of(y_layer, s_part_y + (r - n) * tpr, &o.y_mean, &factor);
        if (lane == 0) o.y_factor = factor;
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
      const float2 s = means_of(s_part + r * tpr);
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
        const float2 s = means_of(s_part + r * tpr);
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
    __syncthreads();                         // (everybody has read the batch and its sums)
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

struct Sums {
  int C, G, cpg, tiles;
  const float* part;
  float* by_group;                           // [group][3][C], for the vectors' gradients
  const float *weight, *bias, *post_weight;
  float *dgate, *dscale, *dshift;
};
// A CTA has 32 channels of a group, a warp every eighth chunk.
__global__ void __launch_bounds__(256) group_sums_kernel(Sums p) {
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
  if (c < p.C)
    for (int gi = w; gi < p.groups; gi += 8) {
      const int b = gi / p.G, g = gi - b * p.G;
      const float* from = p.by_group + (long long)gi * 3 * p.C + c;
      const float m = p.scale ? 1.f + __ldg(p.scale + b * p.scale_s[0] + g * p.scale_s[1] + c) : 1.f;
      const float f = p.gate ? __ldg(p.gate + b * p.gate_s[0] + g * p.gate_s[1] + c) : 1.f;
      a[0] = fmaf(from[0], m, a[0]);
      a[1] = fmaf(from[p.C], m, a[1]);
      a[2] = fmaf(from[2 * p.C], f, a[2]);
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
  p.B = D.B; p.S = D.S; p.G = D.G; p.gt = D.gt; p.C = D.C; p.pieces = D.C / 8; p.rows = D.B * D.S;
  p.norm = s->norm; p.post = s->post_norm; p.eps = s->eps; p.mean = 1.f / (float)D.C;
  p.by_S = FastDiv((unsigned)D.S); p.by_gt = FastDiv((unsigned)D.gt);
  return p;
}

// Backward: threads of a CTA, two of them on an SM where their warps are few; a group's rows cut into as many chunks as run at a time.
constexpr int kSms = 148;
struct Cut { int threads, pieces, ctas, cpg, chunk; long long chunks; };
static Cut cut_of(const Dims& D) {
  Cut c;
  const int pieces = D.C / 8;
  c.pieces = pieces <= 256 ? 1 : 2;
  c.threads = ((pieces + c.pieces - 1) / c.pieces + 31) / 32 * 32;
  c.ctas = std::max(1, 16 / (c.threads / 32));
  const long long run = (long long)kSms * c.ctas, groups = (long long)D.B * D.G;
  c.cpg = (int)std::max<long long>(1, std::min<long long>(D.gt, run / groups));
  c.chunk = (D.gt + c.cpg - 1) / c.cpg;
  c.cpg = (D.gt + c.chunk - 1) / c.chunk;
  c.chunks = groups * c.cpg;
  return c;
}
struct Scratch { float *part, *by_group; Guards guards; size_t bytes; };
static Scratch scratch_of(const Dims& D, void* ws) {
  Carver c(ws);
  Scratch s;
  s.part = c.take<float>((size_t)cut_of(D).chunks * 3 * D.C);
  s.by_group = c.take<float>((size_t)D.B * D.G * 3 * D.C);
  s.guards = c.guards;
  s.bytes = c.total();
  return s;
}

template <typename TS, typename T>
static int go_fwd(const Dims& D, Params& p, cudaStream_t st) {
  p.wpr = 1;
  while (p.wpr < kFwdWarps && p.pieces > 32 * p.wpr * kFwdPieces) p.wpr *= 2;
  const int per = (p.pieces + 32 * p.wpr - 1) / (32 * p.wpr);
  p.groups = std::min(kFwdWarps / p.wpr, p.rows);
  auto go = [&](auto pieces) {
    constexpr int P = decltype(pieces)::value;
    // as many CTAs as run at a time: they share the rows evenly
    const long long ctas = std::min<long long>(((long long)p.rows + p.groups - 1) / p.groups, (long long)fwd_ctas(P) * sm_count());
    launch_kernel(norm_fwd_kernel<TS, T, P>, (unsigned)ctas, 32 * p.wpr * p.groups, 0, st, p);
  };
  if (per <= 1) go(std::integral_constant<int, 1>{});
  else if (per == 2) go(std::integral_constant<int, 2>{});
  else if (per == 3) go(std::integral_constant<int, 3>{});
  else go(std::integral_constant<int, 4>{});
  VMOBA_LAUNCH_OK(1);
  return VMOBA_OK;
}
template <typename TS, typename T>
static int go_bwd(const Cut& c, Params& p, cudaStream_t st) {
  p.cpg = c.cpg; p.chunk = c.chunk;
  // two rows at least in the ring, d_h not through it where those would not fit (fp32, more than 6,900 channels)
  auto slot = [&](bool dh) {
    return align_up((size_t)p.C * ((dh ? 2 : 1) * sizeof(TS) + (p.y.p ? 2 : 1) * sizeof(T)), 128);
  };
  p.stage_dh = p.d_h.p && 2 * slot(true) <= (size_t)kSmemMost;
  const size_t bytes = slot(p.stage_dh != 0), parts = (size_t)c.threads * 2 * sizeof(float2);
  p.batch = (int)std::min<size_t>(batch_rows(c.pieces), std::max<size_t>(1, kSmemMost / c.ctas / (2 * bytes + parts)));
  auto go = [&](auto kernel) -> int {
    VMOBA_CUDA_OK(allow_smem(kernel, kSmemMost));
    launch_kernel(kernel, (unsigned)c.chunks, c.threads, p.batch * (2 * bytes + parts), st, p);
    VMOBA_LAUNCH_OK(1);
    return VMOBA_OK;
  };
  const bool post = p.y.p && p.post != VMOBA_NORM_NONE;
  if (c.pieces == 1) return post ? go(norm_bwd_kernel<TS, T, 1, true>) : go(norm_bwd_kernel<TS, T, 1, false>);
  return post ? go(norm_bwd_kernel<TS, T, 2, true>) : go(norm_bwd_kernel<TS, T, 2, false>);
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
                                const int64_t out_strides[2], void* stream) {
  norm::Dims D;
  if (int rc = norm::make_dims(shape, &D)) return rc;
  if (!params || !x || (!h && !out)) return VMOBA_ERR_ARG;
  norm::Params p = norm::params_of(shape, D);
  if (!norm::take_params(&p, params, D) || !norm::take(&p.x, x, x_strides, D, D.stream_bf16, false) ||
      !norm::take(&p.y, y, y_strides, D, D.bf16, false) || !norm::take(&p.h, h, h_strides, D, D.stream_bf16, true) ||
      !norm::take(&p.out, out, out_strides, D, D.bf16, true))
    return VMOBA_ERR_ARG;
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
  const norm::Cut cut = norm::cut_of(D);
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
    const norm::Sums a{D.C, D.G, cut.cpg, tiles, s.part, vectors ? s.by_group : nullptr, p.weight, p.bias, p.post_weight, grads->gate,
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
