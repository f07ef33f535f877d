// What stands between two branches of a transformer block, in one pass over a token's channels, and its gradients in another.
//   z = y or post(y) * wp,   h = x + gate * z,   n = norm(h),   out = (n * w + b) * (1 + scale) + shift
// Backward, with dm = d_out (1 + scale) and r the norm's factor (1 / sqrt(var + eps)):
//   dh = d_h + r (dm w - n mean(dm w n) [- mean(dm w)]),   dz = gate * dh,   dy = dz, or through the post norm in the same way
//   with, per group of tokens that share a row of scale, shift and gate,   A = sum d_out n,   D = sum d_out,   E = sum dh post(y):
//   dscale = w A + b D,  dshift = D,  dgate = wp E,   dw = sum over groups (1 + scale) A,  db = sum (1 + scale) D,  dwp = sum gate E.
// Bound by HBM: forward x and y in, h and out out; backward d_out, d_h, h and y in, dx and dy out.  So a row stays in registers between the
// norms' trips through it.  Forward, a row is taken by as few warps as hold it in six 8-channel pieces per thread, each group of warps on
// its own.  Backward, a thread keeps its channels over all rows of its CTA's chunk of a group, so that A, D and E add up in registers; the chunks' sums are
// added by a second kernel in a fixed order.  Variances are taken about the mean, in a second trip.
#include <algorithm>

#include "linear.cuh"

namespace vmoba {
namespace norm {

using linear::load_vec;
using linear::store_vec;

constexpr int kMostChannels = 8192;
constexpr int kFwdPieces = 6, kFwdWarps = 8;

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
  float* part;                               // [chunk][3][C]
};

template <typename T>
__device__ __forceinline__ T* row_of(const Rows& r, int b, int t) {
  return static_cast<T*>(const_cast<void*>(r.p)) + b * r.sb + t * r.st;
}

// Sums over the threads of a row, of two values.  slot: a pair per warp of the row; a call that takes the same one again has another
// call between (whose barrier no warp passes before it has read this one's).
__device__ __forceinline__ float2 row_sum(float a, float b, int warp, int warps, int barrier, float2* slot) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    a += __shfl_xor_sync(0xffffffffu, a, o);
    b += __shfl_xor_sync(0xffffffffu, b, o);
  }
  if (warps == 1) return make_float2(a, b);
  if ((threadIdx.x & 31) == 0) slot[warp] = make_float2(a, b);
  asm volatile("bar.sync %0, %1;" ::"r"(barrier), "r"(32 * warps) : "memory");
  float2 s = make_float2(0.f, 0.f);
  for (int w = 0; w < warps; ++w) { s.x += slot[w].x; s.y += slot[w].y; }
  return s;
}

// TS: the stream's type, T: the branch's.  P: pieces per thread.
template <typename TS, typename T, int P>
__global__ void __launch_bounds__(32 * kFwdWarps) norm_fwd_kernel(Params p) {
  if (!grid_begin()) return;
  __shared__ float2 s_slots[2][4][kFwdWarps];
  const int group = (threadIdx.x >> 5) / p.wpr, warp = (threadIdx.x >> 5) - group * p.wpr, tpr = 32 * p.wpr;
  const int l = threadIdx.x - group * tpr;
  int turn = 0;                              // (a row may have a single sum: the next one's goes elsewhere)
  auto sum = [&](float a, float b, int slot) { return row_sum(a, b, warp, p.wpr, 1 + group, &s_slots[turn][slot][group * p.wpr]); };
  for (int r = blockIdx.x * p.groups + group; r < p.rows; r += gridDim.x * p.groups, turn ^= 1) {
    const int b = p.by_S.div(r), t = r - b * p.S, g = p.by_gt.div(t);
    float h[P][8];
    const TS* x_row = row_of<const TS>(p.x, b, t);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int c = 8 * (l + i * tpr);
      if (c < p.C) load_vec<8>(x_row + c, h[i]);
      else
#pragma unroll
        for (int k = 0; k < 8; ++k) h[i][k] = 0.f;
    }
    if (p.y.p) {
      const T* y_row = row_of<const T>(p.y, b, t);
      float y[P][8];
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const int c = 8 * (l + i * tpr);
        if (c < p.C) load_vec<8>(y_row + c, y[i]);
        else
#pragma unroll
          for (int k = 0; k < 8; ++k) y[i][k] = 0.f;
      }
      float mean = 0.f, factor = 1.f;
      if (p.post == VMOBA_NORM_LAYER) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
          for (int k = 0; k < 8; ++k) s += y[i][k];
        mean = sum(s, 0.f, 0).x * p.mean;
      }
      if (p.post != VMOBA_NORM_NONE) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < P; ++i)
          if (8 * (l + i * tpr) < p.C)
#pragma unroll
            for (int k = 0; k < 8; ++k) { y[i][k] -= mean; s = fmaf(y[i][k], y[i][k], s); }
        factor = 1.f / sqrtf(sum(s, 0.f, 1).x * p.mean + p.eps);
      }
      const float* gate = p.gate ? p.gate + b * p.gate_s[0] + g * p.gate_s[1] : nullptr;
      TS* h_row = p.h.p ? row_of<TS>(p.h, b, t) : nullptr;
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const int c = 8 * (l + i * tpr);
        if (c >= p.C) continue;
        float f[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) y[i][k] *= factor;
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
        if (h_row) store_vec<8>(h_row + c, h[i]);
      }
    } else if (p.h.p) {
      TS* h_row = row_of<TS>(p.h, b, t);
#pragma unroll
      for (int i = 0; i < P; ++i)
        if (8 * (l + i * tpr) < p.C) store_vec<8>(h_row + 8 * (l + i * tpr), h[i]);
    }
    if (!p.out.p) continue;
    float mean = 0.f;
    if (p.norm == VMOBA_NORM_LAYER) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < P; ++i)
#pragma unroll
        for (int k = 0; k < 8; ++k) s += h[i][k];
      mean = sum(s, 0.f, 2).x * p.mean;
    }
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < P; ++i)
      if (8 * (l + i * tpr) < p.C)
#pragma unroll
        for (int k = 0; k < 8; ++k) { h[i][k] -= mean; s = fmaf(h[i][k], h[i][k], s); }
    const float factor = 1.f / sqrtf(sum(s, 0.f, 3).x * p.mean + p.eps);
    const float* scale = p.scale ? p.scale + b * p.scale_s[0] + g * p.scale_s[1] : nullptr;
    const float* shift = p.shift ? p.shift + b * p.shift_s[0] + g * p.shift_s[1] : nullptr;
    T* out_row = row_of<T>(p.out, b, t);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int c = 8 * (l + i * tpr);
      if (c >= p.C) continue;
      float f[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) h[i][k] *= factor;
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

// A CTA takes the rows of one chunk one after another; thread l the pieces l, l + blockDim.x ..
template <typename TS, typename T, int P>
__global__ void __launch_bounds__(P == 1 ? 256 : 512) norm_bwd_kernel(Params p) {
  if (!grid_begin()) return;
  __shared__ float2 s_slots[4][16];
  const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5, l = threadIdx.x, tpr = blockDim.x;
  auto sum = [&](float a, float b, int slot) { return row_sum(a, b, warp, warps, 0, s_slots[slot]); };
  const int gi = blockIdx.x / p.cpg, j = blockIdx.x - gi * p.cpg, b = gi / p.G, g = gi - b * p.G;
  const int t0 = g * p.gt + j * p.chunk, t1 = min(min(t0 + p.chunk, (g + 1) * p.gt), p.S);
  float A[P][8] = {}, D[P][8] = {}, E[P][8] = {};
  bool mine[P];
#pragma unroll
  for (int i = 0; i < P; ++i) mine[i] = 8 * (l + i * tpr) < p.C;
  const float* gate = p.gate ? p.gate + b * p.gate_s[0] + g * p.gate_s[1] : nullptr;
  const float* scale = p.scale ? p.scale + b * p.scale_s[0] + g * p.scale_s[1] : nullptr;
  for (int t = t0; t < t1; ++t) {
    float h[P][8] = {}, d[P][8] = {}, y[P][8] = {}, dh[P][8] = {};
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int c = 8 * (l + i * tpr);
      if (!mine[i]) continue;
      load_vec<8>(row_of<const TS>(p.h, b, t) + c, h[i]);
      load_vec<8>(row_of<const T>(p.d_out, b, t) + c, d[i]);
      if (p.y.p) load_vec<8>(row_of<const T>(p.y, b, t) + c, y[i]);
      if (p.d_h.p) load_vec<8>(row_of<const TS>(p.d_h, b, t) + c, dh[i]);
    }
    // means, then variances, of both norms
    float2 s = make_float2(0.f, 0.f);
    const bool means = p.norm == VMOBA_NORM_LAYER || (p.y.p && p.post == VMOBA_NORM_LAYER);
    if (means) {
#pragma unroll
      for (int i = 0; i < P; ++i)
#pragma unroll
        for (int k = 0; k < 8; ++k) { s.x += h[i][k]; s.y += y[i][k]; }
      s = sum(s.x, s.y, 0);
    }
    const float mean_h = p.norm == VMOBA_NORM_LAYER ? s.x * p.mean : 0.f, mean_y = p.post == VMOBA_NORM_LAYER ? s.y * p.mean : 0.f;
    s = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < P; ++i)
      if (mine[i])
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          h[i][k] -= mean_h;
          y[i][k] -= mean_y;
          s.x = fmaf(h[i][k], h[i][k], s.x);
          s.y = fmaf(y[i][k], y[i][k], s.y);
        }
    s = sum(s.x, s.y, 1);
    const float rh = 1.f / sqrtf(s.x * p.mean + p.eps), ry = p.post == VMOBA_NORM_NONE ? 1.f : 1.f / sqrtf(s.y * p.mean + p.eps);
    // the norm's gradient
    s = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      if (!mine[i]) continue;
      const int c = 8 * (l + i * tpr);
      float f[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        h[i][k] *= rh;
        A[i][k] = fmaf(d[i][k], h[i][k], A[i][k]);
        D[i][k] += d[i][k];
      }
      if (scale) {
        load_vec<8>(scale + c, f);
#pragma unroll
        for (int k = 0; k < 8; ++k) d[i][k] = fmaf(d[i][k], f[k], d[i][k]);
      }
      if (p.weight) {
        load_vec<8>(p.weight + c, f);
#pragma unroll
        for (int k = 0; k < 8; ++k) d[i][k] *= f[k];
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) { s.x = fmaf(d[i][k], h[i][k], s.x); s.y += d[i][k]; }
    }
    s = sum(s.x, s.y, 2);
    const float along = s.x * p.mean, level = p.norm == VMOBA_NORM_LAYER ? s.y * p.mean : 0.f;
    TS* dx_row = row_of<TS>(p.dx, b, t);
    s = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      if (!mine[i]) continue;
      const int c = 8 * (l + i * tpr);
#pragma unroll
      for (int k = 0; k < 8; ++k) dh[i][k] = fmaf(rh, d[i][k] - level - h[i][k] * along, dh[i][k]);
      store_vec<8>(dx_row + c, dh[i]);
      if (p.y.p) {
        float f[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          y[i][k] *= ry;
          E[i][k] = fmaf(dh[i][k], y[i][k], E[i][k]);
        }
        if (gate) {
          load_vec<8>(gate + c, f);
#pragma unroll
          for (int k = 0; k < 8; ++k) dh[i][k] *= f[k];
        }
        if (p.post_weight) {
          load_vec<8>(p.post_weight + c, f);
#pragma unroll
          for (int k = 0; k < 8; ++k) dh[i][k] *= f[k];
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) { s.x = fmaf(dh[i][k], y[i][k], s.x); s.y += dh[i][k]; }
      }
    }
    if (!p.dy.p) continue;
    T* dy_row = row_of<T>(p.dy, b, t);
    if (p.post != VMOBA_NORM_NONE) {
      s = sum(s.x, s.y, 3);
      s.x *= p.mean;
      s.y = p.post == VMOBA_NORM_LAYER ? s.y * p.mean : 0.f;
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
      if (!mine[i]) continue;
      if (p.post != VMOBA_NORM_NONE)
#pragma unroll
        for (int k = 0; k < 8; ++k) dh[i][k] = ry * (dh[i][k] - s.y - y[i][k] * s.x);
      store_vec<8>(dy_row + 8 * (l + i * tpr), dh[i]);
    }
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

// Backward: threads of a row's CTA, and how the rows of a group are cut: as many chunks as run at a time, 20 warps of an SM.
constexpr int kSms = 148;
struct Cut { int threads, pieces, cpg, chunk; long long chunks; };
static Cut cut_of(const Dims& D) {
  Cut c;
  const int pieces = D.C / 8;
  c.pieces = pieces <= 256 ? 1 : 2;
  c.threads = ((pieces + c.pieces - 1) / c.pieces + 31) / 32 * 32;
  const long long run = (long long)kSms * std::max(1, 20 / (c.threads / 32)), groups = (long long)D.B * D.G;
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
  while (p.pieces > 32 * p.wpr * kFwdPieces) p.wpr *= 2;
  const int per = (p.pieces + 32 * p.wpr - 1) / (32 * p.wpr);
  p.groups = std::min(kFwdWarps / p.wpr, p.rows);
  const unsigned ctas = (unsigned)std::min<long long>(((long long)p.rows + p.groups - 1) / p.groups, 4ll * sm_count());
  auto kernel = per <= 1 ? norm_fwd_kernel<TS, T, 1> : per <= 2 ? norm_fwd_kernel<TS, T, 2> : per <= 4 ? norm_fwd_kernel<TS, T, 4> : norm_fwd_kernel<TS, T, 6>;
  launch_kernel(kernel, ctas, 32 * p.wpr * p.groups, 0, st, p);
  VMOBA_LAUNCH_OK(1);
  return VMOBA_OK;
}
template <typename TS, typename T>
static int go_bwd(const Cut& c, Params& p, cudaStream_t st) {
  p.cpg = c.cpg; p.chunk = c.chunk;
  launch_kernel(c.pieces == 1 ? norm_bwd_kernel<TS, T, 1> : norm_bwd_kernel<TS, T, 2>, (unsigned)c.chunks, c.threads, 0, st, p);
  VMOBA_LAUNCH_OK(1);
  return VMOBA_OK;
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
                                    void* ws, size_t ws_bytes, void* stream) {
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
  VMOBA_GUARDS_CHECK(s.guards, nullptr, st);
  return VMOBA_OK;
}
