// Rotary positions of q and k, with the root-mean-square norm that video transformers put ahead of them, on the way into the
// layer; and the gradients on the way out.  With y = x r w, r = 1 / sqrt(mean(x^2) + eps) (or y = x), and pair i of a head turned by the
// angle a = pos[axis[i]] * freq[i]:
//   out0 = m (y0 cos a - y1 sin a),  out1 = m (y1 cos a + y0 sin a);   the other channels pass through.
// Backward: g = the gradient of out turned by -a (times m), then with s = w g:
//   dx = r (s - x r^2 mean(s x)),   dw = sum over tokens (norm per head: and heads) of g x r.
//
// Bound by HBM (a row of a token, all heads, is read once and written once, forward; the gradient, x and dx, backward), if the
// instructions are few enough.  So: a row is taken by as few warps as hold it in a few 16-byte vectors per thread, each warp or group of
// warps on its own, token after token, and stays in registers between the norm's two trips through it, while the next row is on its
// way; a thread has the same channels of every head, so that its sines and cosines are loaded once per token; angles are
// worked out once per token for all heads and tensors; the norm's weights lie in shared memory in the order of the registers; even and
// odd channels are apart, so that pairs turn by packed instructions.  Rows longer than that are read twice.
// An angle is formed and reduced in 64 bits, because a position of 10^6 times a frequency of one has no digit behind the point left in 32.
#include <algorithm>
#include <type_traits>

#include "common.cuh"
#include "sm100.cuh"

namespace vmoba {
namespace rotary {

using sm100::fma2;
using sm100::mul2;

constexpr int kMaxTensors = 4;
constexpr int kMaxWarps = 8;                 // of a row, and of a CTA
constexpr int kBwdWarps = 12;                // of the backward's CTAs, one per SM: 168 registers per thread
constexpr int kMaxPairs = 64;

struct Tensor {
  const void* src;                           // forward: x; backward: the gradient of the output
  const void* x;                             // backward with a norm: x
  void* dst;
  const float* w;                            // norm weights or null (ones)
  long long ss[3], xs[3], ds[3];             // element strides {batch, token, head} of src, x and dst
  unsigned ss1, xs1, ds1;                    // bytes from token to token where samples follow one another at that distance too, else 0
};

// The row of token g = (b, tok) of a tensor whose first row, from the thread's first channel on, is at `base`.
template <typename T>
__device__ __forceinline__ T* row_of(T* base, const long long (&s)[3], unsigned bytes, int g, int b, int tok) {
  using Byte = typename std::conditional<std::is_const<T>::value, const char, char>::type;
  if (bytes) return reinterpret_cast<T*>(reinterpret_cast<Byte*>(base) + (unsigned long long)(unsigned)g * bytes);
  return base + b * s[0] + tok * s[1];
}

struct Params {
  int B, S, heads, d;
  int W, bT, bH, bW, sb;
  FastDiv by_S, by_HW, by_W, by_bT, by_bH, by_bW;
  int HW, nH, nW;
  int n, turned;                             // tensors; the first `turned` of them are normed and rotated, the others only moved
  int pairs, axes, layout, norm, pos_batch;
  int full;                                  // every channel of a head belongs to a pair
  int src_bm, dst_bm;                        // src / dst is block-major (strides unused)
  float mscale, eps;
  const int* pos;
  const double* freq;
  const int* axis;
  int* perm;
  int wpr, groups;                           // warps per row, rows that a CTA has under way
  float* part;                               // backward: [tensor][CTA][weights] partial sums of dw
  Tensor t[kMaxTensors];
};

// Block-major position of raster token r (the inverse of Eq. 1).
__device__ __forceinline__ int block_pos(const Params& p, int r) {
  const int t = p.by_HW.div(r), r2 = r - t * p.HW, h = p.by_W.div(r2), w = r2 - h * p.W;
  const int jt = p.by_bT.div(t), jh = p.by_bH.div(h), jw = p.by_bW.div(w);
  const int block = (jt * p.nH + jh) * p.nW + jw;
  const int slot = ((t - jt * p.bT) * p.bH + (h - jh * p.bH)) * p.bW + (w - jw * p.bW);
  return block * p.sb + slot;
}

template <typename T>
struct Vec {
  static constexpr int E = 16 / (int)sizeof(T);
  static __device__ __forceinline__ void unpack(const uint4& u, float (&x)[E]) {
    if constexpr (E == 4) {
      x[0] = __uint_as_float(u.x); x[1] = __uint_as_float(u.y); x[2] = __uint_as_float(u.z); x[3] = __uint_as_float(u.w);
    } else {
      const uint32_t v[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(v[i] << 16); x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u); }
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&x)[E]) {
    if constexpr (E == 4) {
      return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    } else {
      uint32_t v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        v[i] = *reinterpret_cast<const uint32_t*>(&h);
      }
      return make_uint4(v[0], v[1], v[2], v[3]);
    }
  }
};

// The layouts, as far as the kernels tell them apart: half with whole vectors as partners, and with any number of pairs.
enum Layout { kInterleaved, kHalf, kHalfAny };

// cos and sin (times mscale) of a token's angles, by the threads of a group: the angle in turns, less whole ones.
struct alignas(16) Angles { float cs[kMaxPairs], sn[kMaxPairs]; };
// The pairs' frequencies in turns and axes, in shared memory, and the positions that a thread's pairs l, l + tpr (there are at most 64, and 32
// threads at least) take them at.
struct Frequencies { double f[kMaxPairs]; int axis[kMaxPairs]; };
__device__ __forceinline__ void stage_frequencies(const Params& p, Frequencies* to) {
  for (int i = threadIdx.x; i < p.pairs; i += blockDim.x) {
    to->f[i] = __ldg(p.freq + i) * 0.15915494309189533577;      // 1 / (2 pi)
    to->axis[i] = min(max(__ldg(p.axis + i), 0), p.axes - 1);
  }
}
struct Positions {
  int at[2];
  __device__ __forceinline__ void load(const Params& p, const Frequencies& f, int g, int l, int tpr) {
    const int at0 = p.pos_batch > 1 ? g : g - p.by_S.div(g) * p.S;
#pragma unroll
    for (int j = 0; j < 2; ++j)
      if (l + j * tpr < p.pairs) at[j] = __ldg(p.pos + (long long)at0 * p.axes + f.axis[l + j * tpr]);
  }
  __device__ __forceinline__ void angles(const Params& p, const Frequencies& f, int l, int tpr, Angles* ang) const {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int i = l + j * tpr;
      if (i >= p.pairs) continue;
      const double turns = (double)at[j] * f.f[i];
      float sn, cs;
      sincospif(2.0f * (float)(turns - rint(turns)), &sn, &cs);
      ang->cs[i] = cs * p.mscale;
      ang->sn[i] = sn * p.mscale;
    }
  }
};

// The channel, of a vector's, that a thread holds in place e: even ones ahead of odd ones where those are a pair.
template <int E, Layout L>
__device__ __forceinline__ constexpr int channel(int e) { return L != kInterleaved ? e : e < E / 2 ? 2 * e : 2 * e - E + 1; }

template <typename T, Layout L>
struct Row {
  static constexpr int E = Vec<T>::E;
  static __device__ __forceinline__ void unpack(const uint4& u, float (&x)[E]) {
    float y[E];
    Vec<T>::unpack(u, y);
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = y[channel<E, L>(e)];
  }
  static __device__ __forceinline__ uint4 pack(const float (&x)[E]) {
    float y[E];
#pragma unroll
    for (int e = 0; e < E; ++e) y[channel<E, L>(e)] = x[e];
    return Vec<T>::pack(y);
  }
};

// sum += a . b
template <int E>
__device__ __forceinline__ void dot(const float (&a)[E], const float (&b)[E], float& s0, float& s1) {
#pragma unroll
  for (int e = 0; e < E; e += 2) fma2(s0, s1, a[e], a[e + 1], b[e], b[e + 1], s0, s1);
}
template <int E>
__device__ __forceinline__ void times(float (&a)[E], const float (&b)[E]) {
#pragma unroll
  for (int e = 0; e < E; e += 2) mul2(a[e], a[e + 1], a[e], a[e + 1], b[e], b[e + 1]);
}
template <int E>
__device__ __forceinline__ void times(float (&a)[E], float b) {
#pragma unroll
  for (int e = 0; e < E; e += 2) mul2(a[e], a[e + 1], a[e], a[e + 1], b, b);
}

// What a thread's vectors, all of the same channels c0 .. c0 + E - 1 of a head, are turned by.  sign: -1 turns back.
template <int E, Layout L>
struct Turn {
  static constexpr int N = L == kInterleaved ? E / 2 : E;
  float cs[N], sn[N];
  uint32_t mine;                             // bit e: the channel in place e belongs to a pair
  __device__ __forceinline__ void load(const Params& p, const Angles& a, int c0, float sign) {
    mine = 0;
    if constexpr (L == kInterleaved) {
      if constexpr (E == 8) {
        const float4 c = *reinterpret_cast<const float4*>(a.cs + c0 / 2), s = *reinterpret_cast<const float4*>(a.sn + c0 / 2);
        cs[0] = c.x; cs[1] = c.y; cs[2] = c.z; cs[3] = c.w;
        sn[0] = s.x * sign; sn[1] = s.y * sign; sn[2] = s.z * sign; sn[3] = s.w * sign;
      } else {
        const float2 c = *reinterpret_cast<const float2*>(a.cs + c0 / 2), s = *reinterpret_cast<const float2*>(a.sn + c0 / 2);
        cs[0] = c.x; cs[1] = c.y;
        sn[0] = s.x * sign; sn[1] = s.y * sign;
      }
      if (!p.full) {
        const int n = min(max(p.pairs - c0 / 2, 0), N);
        mine = ((1u << n) - 1u) * ((1u << N) + 1u);
      }
    } else if constexpr (L == kHalf) {
      const bool second = c0 >= p.pairs;
      const int i = second ? c0 - p.pairs : c0;
      if (c0 < 2 * p.pairs) mine = (1u << E) - 1u;
      const float f = second ? sign : -sign;
#pragma unroll
      for (int e = 0; e < E; e += 4) {
        const int at = c0 < 2 * p.pairs ? i + e : 0;
        const float4 c = *reinterpret_cast<const float4*>(a.cs + at), s = *reinterpret_cast<const float4*>(a.sn + at);
        cs[e] = c.x; cs[e + 1] = c.y; cs[e + 2] = c.z; cs[e + 3] = c.w;
        sn[e] = s.x * f; sn[e + 1] = s.y * f; sn[e + 2] = s.z * f; sn[e + 3] = s.w * f;
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int c = c0 + e;
        const bool second = c >= p.pairs, ok = c < 2 * p.pairs;
        const int i = ok ? (second ? c - p.pairs : c) : 0;
        cs[e] = a.cs[i];
        sn[e] = a.sn[i] * (second ? sign : -sign);
        if (ok) mine |= 1u << e;
      }
    }
  }
  // Turns a vector and multiplies it by r (SCALED: not known to be 1).  buf (kHalfAny): 32 * E floats of the warp.  Called by whole warps.
  template <bool SCALED>
  __device__ __forceinline__ void apply(const Params& p, float (&y)[E], float r, int c0, float* buf) const {
    if constexpr (L == kInterleaved) {
      if (p.full) {
#pragma unroll
        for (int i = 0; i < N; i += 2) {     // (r times sine and cosine: the same of every vector of a row)
          const float c0 = cs[i] * r, c1 = cs[i + 1] * r, s0 = sn[i] * r, s1 = sn[i + 1] * r;
          float t0, t1, u0, u1;
          mul2(t0, t1, y[N + i], y[N + i + 1], -s0, -s1);
          mul2(u0, u1, y[i], y[i + 1], s0, s1);
          fma2(y[i], y[i + 1], y[i], y[i + 1], c0, c1, t0, t1);
          fma2(y[N + i], y[N + i + 1], y[N + i], y[N + i + 1], c0, c1, u0, u1);
        }
      } else {
        if (SCALED) times<E>(y, r);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float y0 = y[i], y1 = y[N + i];
          if (mine >> i & 1) {
            y[i] = fmaf(y0, cs[i], -y1 * sn[i]);
            y[N + i] = fmaf(y1, cs[i], y0 * sn[i]);
          }
        }
      }
    } else {
      if (SCALED) times<E>(y, r);
      float o[E];
      const int lane = threadIdx.x & 31;
      if constexpr (L == kHalf) {            // the partners of a vector are a vector of another lane of the same head
        const int by = p.pairs / E, from = (c0 < p.pairs ? lane + by : lane - by) & 31;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = __shfl_sync(0xffffffffu, y[e], from);
      } else {
        __syncwarp();
#pragma unroll
        for (int e = 0; e < E; ++e) buf[lane * E + e] = y[e];
        __syncwarp();
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = (mine >> e & 1) ? buf[lane * E + e + (c0 + e < p.pairs ? p.pairs : -p.pairs)] : 0.f;
      }
      if (p.full) {
#pragma unroll
        for (int e = 0; e < E; e += 2) {
          mul2(o[e], o[e + 1], o[e], o[e + 1], sn[e], sn[e + 1]);
          fma2(y[e], y[e + 1], y[e], y[e + 1], cs[e], cs[e + 1], o[e], o[e + 1]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (mine >> e & 1) y[e] = fmaf(y[e], cs[e], o[e] * sn[e]);
      }
    }
  }
};

// The warps of a group meet (barrier 1 + group).
__device__ __forceinline__ void meet(int group, int wpr) {
  if (wpr == 1) __syncwarp();
  else asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(32 * wpr) : "memory");
}

// Sums over the threads of a row, of one value or two.  slot: a pair of floats per warp of the group; the next call takes another one (a
// call that takes this one again is two barriers away).
template <bool TWO>
__device__ __forceinline__ float2 row_sum(float2 v, int group, int wpr, float2* slot) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
    if (TWO) v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
  }
  if (wpr == 1) return v;
  if ((threadIdx.x & 31) == 0) slot[(threadIdx.x >> 5) - group * wpr] = v;
  meet(group, wpr);
  float2 a = make_float2(0.f, 0.f);
  for (int w = 0; w < wpr; ++w) { a.x += slot[w].x; a.y += slot[w].y; }
  return a;
}
// Sums over the lanes of a head, of N vectors.
template <int N>
__device__ __forceinline__ void head_sums(float (&v)[N], int lanes) {
#pragma unroll 1
  for (int o = lanes >> 1; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
}

// The norm's weights in shared memory, in the order of a thread's registers: of `tensors` tensors, planes of four of a vector's E weights,
// `count` vectors each, of which `there` exist.  Ones where there are none.
template <int E, Layout L>
__device__ __forceinline__ void stage_weights(float4* to, const Tensor* t, int tensors, int count, int there) {
  constexpr int P = E / 4;
  for (int i = threadIdx.x; i < tensors * P * count; i += blockDim.x) {
    const int v = i % count, plane = i / count % P, k = i / (count * P);
    const float* w = t[k].w && v < there ? t[k].w + v * E : nullptr;
    float f[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int low = channel<E, L>(e), high = channel<E, L>(E - 4 + e);
      f[e] = w ? __ldg(w + (plane ? high : low)) : 1.f;
    }
    to[i] = make_float4(f[0], f[1], f[2], f[3]);
  }
}
template <int E>
__device__ __forceinline__ void staged_weights(const float4* from, int count, float (&f)[E]) {
#pragma unroll
  for (int e = 0; e < E; e += 4) {
    const float4 v = from[e / 4 * count];
    f[e] = v.x; f[e + 1] = v.y; f[e + 2] = v.z; f[e + 3] = v.w;
  }
}
template <int E, Layout L>
__device__ __forceinline__ void weights(const float* w, float (&f)[E]) {      // (from global memory)
#pragma unroll
  for (int e = 0; e < E; ++e) f[e] = w ? __ldg(w + channel<E, L>(e)) : 1.f;
}

// ------------------------------------------------------------------------------ forward
// A thread's place in a row: the vectors l, l + tpr, ... of all heads, the same channels of each.
struct Place {
  int group, l, tpr, V, nvec, c0, vshift, head0, heads_per;
  __device__ __forceinline__ Place(const Params& p, int E) {
    group = (int)(threadIdx.x >> 5) / p.wpr;
    tpr = 32 * p.wpr;
    l = threadIdx.x - group * tpr;
    V = p.d / E;
    nvec = p.heads * V;
    c0 = (l % V) * E;
    vshift = 31 - __clz(V);
    head0 = l >> vshift;
    heads_per = tpr >> vshift;
  }
};

// Rows that a group's threads hold in NV vectors each: 128 registers for six of them and the next row's, 16 warps per SM.
// q, k of 32,760 tokens x 12 heads of 128 into block order, 402 MB: 73 us, 600 warp instructions per row in 54 % of the issue slots (with a ring of
// asynchronous copies in shared memory, which every row is read from twice: 90); of 75,600 tokens x 40 heads, 3.1 GB: 556 us.
template <typename T, Layout L, int NV>
__global__ void __launch_bounds__(32 * kMaxWarps, 2)
rotary_fwd_kernel(const __grid_constant__ Params p) {
  if (!grid_begin()) return;
  constexpr int E = Vec<T>::E;
  extern __shared__ __align__(16) float4 w_all[];
  __shared__ Frequencies freq;
  __shared__ Angles ang[kMaxWarps][2];
  __shared__ float2 slot[2][kMaxWarps];
  __shared__ float exchange[L == kHalfAny ? kMaxWarps * 32 * E : 1];
  const Place at(p, E);
  const int l = at.l, tpr = at.tpr, group = at.group, c0 = at.c0;
  float* buf = L == kHalfAny ? exchange + (threadIdx.x >> 5) * 32 * E : exchange;
  const bool by_row = p.norm == VMOBA_ROTARY_NORM_ROW;
  const int n_w = by_row ? NV * tpr : at.V;
  stage_frequencies(p, &freq);
  if (p.norm != VMOBA_ROTARY_NORM_NONE) stage_weights<E, L>(w_all, p.t, p.turned, n_w, by_row ? at.nvec : at.V);
  __syncthreads();
  const float inv_n = 1.0f / (float)(by_row ? p.heads * p.d : p.d);
  const int have = l < at.nvec ? (at.nvec - l + tpr - 1) / tpr : 0;      // vectors of this thread
  const int tokens = p.B * p.S, step = gridDim.x * p.groups;
  int g = blockIdx.x * p.groups + group;
  if (g >= tokens) return;                   // (whole groups)
  uint4 next[NV];                            // the next row (those that the thread does not have stay zero)
#pragma unroll
  for (int i = 0; i < NV; ++i) next[i] = make_uint4(0u, 0u, 0u, 0u);
  auto fetch = [&](int g, int k) {
    if (g >= tokens) return;
    const Tensor& t = p.t[k];
    const int b = p.by_S.div(g);
    const T* from = row_of(reinterpret_cast<const T*>(t.src) + at.head0 * t.ss[2] + c0, t.ss, t.ss1, g, b, g - b * p.S);
    const long long apart = at.heads_per * t.ss[2];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (i < have) next[i] = __ldcs(reinterpret_cast<const uint4*>(from));
      from += apart;
    }
  };
  fetch(g, p.n - 1);
  Positions positions;
  positions.load(p, freq, g, l, tpr);
  positions.angles(p, freq, l, tpr, &ang[group][0]);
  int turn_buf = 0, sum_buf = 0;
  for (; g < tokens; g += step, turn_buf ^= 1) {
    meet(group, p.wpr);                      // (this token's angles)
    Turn<E, L> turn;
    turn.load(p, ang[group][turn_buf], c0, 1.f);
    if (g + step < tokens) positions.load(p, freq, g + step, l, tpr);
    const int b = p.by_S.div(g), tok = g - b * p.S, bm = p.dst_bm || p.perm ? block_pos(p, tok) : 0;
    if (p.perm && b == 0 && l == 0) p.perm[bm] = tok;
    // tensors from the last to the first: what the caller reads next comes last
#pragma unroll 1
    for (int k = p.n - 1; k >= 0; --k) {
      const Tensor& t = p.t[k];
      const long long to_head = p.dst_bm ? (long long)p.S * p.d : t.ds[2], to_next = at.heads_per * to_head;
      T* dst = reinterpret_cast<T*>(t.dst) + at.head0 * to_head + c0;
      dst = p.dst_bm ? dst + (unsigned long long)(unsigned)(b * p.heads * p.S + bm) * (unsigned)p.d : row_of(dst, t.ds, t.ds1, g, b, tok);
      const int gn = k > 0 ? g : g + step, kn = k > 0 ? k - 1 : p.n - 1;
      if (k >= p.turned) {                   // only moved
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          if (i < have) *reinterpret_cast<uint4*>(dst) = next[i];
          dst += to_next;
        }
        fetch(gn, kn);
        continue;
      }
      float y[NV][E];
#pragma unroll
      for (int i = 0; i < NV; ++i) Row<T, L>::unpack(next[i], y[i]);
      fetch(gn, kn);
      auto put = [&](int i) {
        if (i < have) *reinterpret_cast<uint4*>(dst) = Row<T, L>::pack(y[i]);
        dst += to_next;
      };
      if (by_row) {
        float s0 = 0.f, s1 = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) dot<E>(y[i], y[i], s0, s1);
        const float r = rsqrtf(fmaf(row_sum<false>(make_float2(s0 + s1, 0.f), group, p.wpr, slot[sum_buf] + group * p.wpr).x, inv_n, p.eps));
        sum_buf ^= 1;
        const float4* w = w_all + k * (E / 4) * n_w + l;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          float f[E];
          staged_weights<E>(w + i * tpr, n_w, f);
          times<E>(y[i], f);
          turn.template apply<true>(p, y[i], r, c0, buf);
          put(i);
        }
      } else if (p.norm == VMOBA_ROTARY_NORM_HEAD) {
        float f[E], sums[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          float s0 = 0.f, s1 = 0.f;
          dot<E>(y[i], y[i], s0, s1);
          sums[i] = s0 + s1;
        }
        head_sums<NV>(sums, at.V);
        staged_weights<E>(w_all + k * (E / 4) * n_w + c0 / E, n_w, f);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          times<E>(y[i], rsqrtf(fmaf(sums[i], inv_n, p.eps)));
          times<E>(y[i], f);
          turn.template apply<false>(p, y[i], 1.f, c0, buf);
          put(i);
        }
      } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          turn.template apply<false>(p, y[i], 1.f, c0, buf);
          put(i);
        }
      }
    }
    if (g + step < tokens) positions.angles(p, freq, l, tpr, &ang[group][turn_buf ^ 1]);
  }
}

// Longer rows: a CTA each, in trips of four vectors per thread, read once for the norm and once more for the result.
constexpr int kTrip = 4;
template <typename T, Layout L>
__global__ void __launch_bounds__(32 * kMaxWarps)
rotary_fwd_long_kernel(const __grid_constant__ Params p) {
  if (!grid_begin()) return;
  constexpr int E = Vec<T>::E;
  __shared__ Frequencies freq;
  __shared__ Angles ang[2];
  __shared__ float2 slot[2][kMaxWarps];
  __shared__ float exchange[L == kHalfAny ? kMaxWarps * 32 * E : 1];
  const Place at(p, E);
  const int l = at.l, tpr = at.tpr, c0 = at.c0;
  float* buf = L == kHalfAny ? exchange + (threadIdx.x >> 5) * 32 * E : exchange;
  const bool by_row = p.norm == VMOBA_ROTARY_NORM_ROW;
  Positions positions;
  stage_frequencies(p, &freq);
  __syncthreads();
  int turn_buf = 0, sum_buf = 0;
  for (int g = blockIdx.x; g < p.B * p.S; g += gridDim.x, turn_buf ^= 1) {
    positions.load(p, freq, g, l, tpr);
    positions.angles(p, freq, l, tpr, &ang[turn_buf]);
    meet(0, p.wpr);
    Turn<E, L> turn;
    turn.load(p, ang[turn_buf], c0, 1.f);
    const int b = p.by_S.div(g), tok = g - b * p.S, bm = p.dst_bm || p.perm ? block_pos(p, tok) : 0;
    if (p.perm && b == 0 && l == 0) p.perm[bm] = tok;
#pragma unroll 1
    for (int k = p.n - 1; k >= 0; --k) {
      const Tensor& t = p.t[k];
      const T* src = row_of(reinterpret_cast<const T*>(t.src) + at.head0 * t.ss[2] + c0, t.ss, t.ss1, g, b, tok);
      const long long to_head = p.dst_bm ? (long long)p.S * p.d : t.ds[2];
      T* dst = reinterpret_cast<T*>(t.dst) + at.head0 * to_head + c0;
      dst = p.dst_bm ? dst + (unsigned long long)(unsigned)(b * p.heads * p.S + bm) * (unsigned)p.d : row_of(dst, t.ds, t.ds1, g, b, tok);
      uint4 u[kTrip];
      auto fetch = [&](int v0) {
#pragma unroll
        for (int i = 0; i < kTrip; ++i) {
          u[i] = make_uint4(0u, 0u, 0u, 0u);
          if (v0 + l + i * tpr < at.nvec) u[i] = __ldcg(reinterpret_cast<const uint4*>(src + ((v0 >> at.vshift) + i * at.heads_per) * t.ss[2]));
        }
      };
      const bool turned = k < p.turned;
      float r = 1.f;
      if (turned && by_row) {
        float s0 = 0.f, s1 = 0.f;
        for (int v0 = 0; v0 < at.nvec; v0 += kTrip * tpr) {
          fetch(v0);
#pragma unroll
          for (int i = 0; i < kTrip; ++i) {
            float x[E];
            Vec<T>::unpack(u[i], x);
            dot<E>(x, x, s0, s1);
          }
        }
        r = rsqrtf(row_sum<false>(make_float2(s0 + s1, 0.f), 0, p.wpr, slot[sum_buf]).x / (float)(p.heads * p.d) + p.eps);
        sum_buf ^= 1;
      }
      for (int v0 = 0; v0 < at.nvec; v0 += kTrip * tpr) {
        fetch(v0);
#pragma unroll
        for (int i = 0; i < kTrip; ++i) {
          const int v = v0 + l + i * tpr;
          const bool there = v < at.nvec;
          float y[E];
          Row<T, L>::unpack(u[i], y);
          if (turned) {
            if (p.norm != VMOBA_ROTARY_NORM_NONE) {
              float f[E];
              weights<E, L>(t.w && there ? t.w + (by_row ? v * E : c0) : nullptr, f);
              if (!by_row) {
                float s[1], s1 = 0.f;
                s[0] = 0.f;
                dot<E>(y, y, s[0], s1);
                s[0] += s1;
                head_sums<1>(s, at.V);
                times<E>(y, rsqrtf(s[0] / (float)p.d + p.eps));
              }
              times<E>(y, f);
            }
            turn.template apply<true>(p, y, r, c0, buf);
          }
          if (there) *reinterpret_cast<uint4*>(dst + ((v0 >> at.vshift) + i * at.heads_per) * to_head) = Row<T, L>::pack(y);
        }
      }
    }
  }
}

// ------------------------------------------------------------------------------ backward
// blockIdx.y: tensor.  A thread has the same channels in every row that its group takes, and keeps their part of dw in registers (rows
// longer than that: in shared memory).  The parts of a CTA's groups, and of the CTAs (weight_sum_kernel), are added up in a
// fixed order: the results repeat bit for bit.
struct Gradients {                           // a tensor's rows, from a thread's first head on
  const Params& p;
  const Tensor& t;
  const Place& at;
  long long d_head;
  __device__ __forceinline__ Gradients(const Params& p, const Tensor& t, const Place& at)
      : p(p), t(t), at(at), d_head(p.src_bm ? (long long)p.S * p.d : t.ss[2]) {}
  template <typename T>
  __device__ __forceinline__ const T* d(int g, int b, int tok) const {
    const T* from = reinterpret_cast<const T*>(t.src) + at.head0 * d_head + at.c0;
    if (p.src_bm) return from + (unsigned long long)(unsigned)(b * p.heads * p.S + block_pos(p, tok)) * (unsigned)p.d;
    return row_of(from, t.ss, t.ss1, g, b, tok);
  }
  template <typename T>
  __device__ __forceinline__ const T* x(int g, int b, int tok) const {
    return row_of(reinterpret_cast<const T*>(t.x) + at.head0 * t.xs[2] + at.c0, t.xs, t.xs1, g, b, tok);
  }
  template <typename T>
  __device__ __forceinline__ T* dx(int g, int b, int tok) const {
    return row_of(reinterpret_cast<T*>(t.dst) + at.head0 * t.ds[2] + at.c0, t.ds, t.ds1, g, b, tok);
  }
};
// g -> dx, given x r: f g r - (x r) back, back = r^2 mean(x f g);  acc += g x r.
template <int E>
__device__ __forceinline__ void finish(float (&g)[E], const float (&xr)[E], const float (&f)[E], float r, float back, float (&acc)[E]) {
#pragma unroll
  for (int e = 0; e < E; e += 2) {
    fma2(acc[e], acc[e + 1], g[e], g[e + 1], xr[e], xr[e + 1], acc[e], acc[e + 1]);
    mul2(g[e], g[e + 1], g[e], g[e + 1], f[e], f[e + 1]);
    mul2(g[e], g[e + 1], g[e], g[e + 1], r, r);
    fma2(g[e], g[e + 1], xr[e], xr[e + 1], -back, -back, g[e], g[e + 1]);
  }
}
// x . x and x . (g f)
template <int E>
__device__ __forceinline__ void sums_of(const float (&x)[E], const float (&g)[E], const float (&f)[E], float (&s)[4]) {
  dot<E>(x, x, s[0], s[1]);
#pragma unroll
  for (int e = 0; e < E; e += 2) {
    float a, b;
    mul2(a, b, g[e], g[e + 1], f[e], f[e + 1]);
    fma2(s[2], s[3], x[e], x[e + 1], a, b, s[2], s[3]);
  }
}

// Keeps the compiler from carrying what it has made of u.
__device__ __forceinline__ void opaque(uint4& u) { asm volatile("" : "+r"(u.x), "+r"(u.y), "+r"(u.z), "+r"(u.w)); }

// Rows that a group's threads hold in NV vectors each: three of the gradient, x and dw, and the next row's two, in 168 registers, 12 warps per SM.
// q, k of 32,760 tokens x 12 heads of 128, norm per row, 604 MB: 131 us (128 registers and 16 warps: 156, the reloads of 40 registers per row).
template <typename T, Layout L, int NV>
__global__ void __launch_bounds__(32 * kBwdWarps, 1)
rotary_bwd_kernel(const __grid_constant__ Params p) {
  if (!grid_begin()) return;
  constexpr int E = Vec<T>::E;
  extern __shared__ __align__(16) float4 w_all[];                    // the weights; at the end [group][heads * d] sums
  __shared__ Frequencies freq;
  __shared__ Angles ang[kBwdWarps][2];
  __shared__ float2 slot[2][kBwdWarps];
  __shared__ float exchange[kBwdWarps * 32 * E];
  const Place at(p, E);
  const int l = at.l, tpr = at.tpr, group = at.group, c0 = at.c0;
  float* buf = exchange + (threadIdx.x >> 5) * 32 * E;
  const Tensor& t = p.t[blockIdx.y];
  const bool by_row = p.norm == VMOBA_ROTARY_NORM_ROW, normed = p.norm != VMOBA_ROTARY_NORM_NONE;
  const int row_ch = p.heads * p.d, n_w = by_row ? NV * tpr : at.V;
  const float inv_n = 1.0f / (float)(by_row ? row_ch : p.d);
  const float4* w_mine = w_all + (by_row ? l : c0 / E);
  stage_frequencies(p, &freq);
  if (normed) stage_weights<E, L>(w_all, &t, 1, n_w, by_row ? at.nvec : at.V);
  __syncthreads();
  float acc[NV][E];                          // (norm per head: all in acc[0])
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < E; ++e) acc[i][e] = 0.f;
  const Gradients rows(p, t, at);
  const int have = l < at.nvec ? (at.nvec - l + tpr - 1) / tpr : 0;
  const int tokens = p.B * p.S, step = gridDim.x * p.groups;
  int g = blockIdx.x * p.groups + group;
  if (g < tokens) {                          // (whole groups; all threads meet again at the end)
    uint4 next_d[NV], next_x[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) next_d[i] = next_x[i] = make_uint4(0u, 0u, 0u, 0u);
    auto fetch = [&](int g) {
      const int b = p.by_S.div(g), tok = g - b * p.S;
      const T* d = rows.d<T>(g, b, tok);
      const long long d_apart = at.heads_per * rows.d_head, x_apart = at.heads_per * t.xs[2];
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if (i < have) next_d[i] = __ldcs(reinterpret_cast<const uint4*>(d));
        d += d_apart;
      }
      if (normed) {
        const T* x = rows.x<T>(g, b, tok);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          if (i < have) next_x[i] = __ldcs(reinterpret_cast<const uint4*>(x));
          x += x_apart;
        }
      }
    };
    fetch(g);
    Positions positions;
    positions.load(p, freq, g, l, tpr);
    positions.angles(p, freq, l, tpr, &ang[group][0]);
    int turn_buf = 0;
    for (; g < tokens; g += step, turn_buf ^= 1) {
      meet(group, p.wpr);                    // (this token's angles)
      Turn<E, L> turn;
      turn.load(p, ang[group][turn_buf], c0, -1.f);
      const bool more = g + step < tokens;
      if (more) positions.load(p, freq, g + step, l, tpr);
      const int b = p.by_S.div(g), tok = g - b * p.S;
      const long long apart = at.heads_per * t.ds[2];
      T* dst = rows.dx<T>(g, b, tok);
      float y[NV][E];
      uint4 x_raw[NV];                       // (unpacked twice: 24 registers less)
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        Row<T, L>::unpack(next_d[i], y[i]);
        x_raw[i] = next_x[i];
      }
      if (more) fetch(g + step);
#pragma unroll
      for (int i = 0; i < NV; ++i) turn.template apply<false>(p, y[i], 1.f, c0, buf);
      float r, back;                         // 1 / rms; r^2 times the mean of x times its weighted gradient
      auto scales = [&](float xx, float xg) {
        r = rsqrtf(fmaf(xx, inv_n, p.eps));
        back = r * r * (xg * inv_n);
      };
      if (by_row) {
        float s[4] = {0.f, 0.f, 0.f, 0.f}, f[E];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          float x[E];
          staged_weights<E>(w_mine + i * tpr, n_w, f);
          Row<T, L>::unpack(x_raw[i], x);
          sums_of<E>(x, y[i], f, s);
        }
        const float2 total = row_sum<true>(make_float2(s[0] + s[1], s[2] + s[3]), group, p.wpr, slot[turn_buf] + group * p.wpr);
        scales(total.x, total.y);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          float x[E];
          opaque(x_raw[i]);
          staged_weights<E>(w_mine + i * tpr, n_w, f);
          Row<T, L>::unpack(x_raw[i], x);
          times<E>(x, r);
          finish<E>(y[i], x, f, r, back, acc[i]);
        }
      } else if (normed) {
        float sums[2 * NV], f[E];
        staged_weights<E>(w_mine, n_w, f);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          float s[4] = {0.f, 0.f, 0.f, 0.f};
          float x[E];
          Row<T, L>::unpack(x_raw[i], x);
          sums_of<E>(x, y[i], f, s);
          sums[2 * i] = s[0] + s[1];
          sums[2 * i + 1] = s[2] + s[3];
        }
        head_sums<2 * NV>(sums, at.V);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          scales(sums[2 * i], sums[2 * i + 1]);
          if (i >= have) r = back = 0.f;     // (beyond the row: without an eps r is infinite there, and dw is a sum over all vectors)
          float x[E];
          opaque(x_raw[i]);
          Row<T, L>::unpack(x_raw[i], x);
          times<E>(x, r);
          finish<E>(y[i], x, f, r, back, acc[0]);
        }
      }
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if (i < have) *reinterpret_cast<uint4*>(dst) = Row<T, L>::pack(y[i]);
        dst += apart;
      }
      if (more) positions.angles(p, freq, l, tpr, &ang[group][turn_buf ^ 1]);
    }
  }
  if (!normed) return;
  float* out = p.part + ((long long)blockIdx.y * gridDim.x + blockIdx.x) * (by_row ? row_ch : p.d);
  float* sums = by_row ? reinterpret_cast<float*>(w_all) : exchange;
  __syncthreads();                           // (the weights and the exchange buffers are free)
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (by_row) {
        if (i < have) sums[group * row_ch + (l + i * tpr) * E + channel<E, L>(e)] = acc[i][e];
      } else if (i == 0) {
        sums[threadIdx.x * E + channel<E, L>(e)] = acc[0][e];
      }
    }
  __syncthreads();
  if (by_row) {
    for (int i = threadIdx.x; i < row_ch; i += blockDim.x) {
      float a = 0.f;
      for (int q = 0; q < p.groups; ++q) a += sums[q * row_ch + i];
      out[i] = a;
    }
  } else {
    for (int c = threadIdx.x; c < p.d; c += blockDim.x) {            // threads c / E, c / E + V, ... hold channel c
      float a = 0.f;
      for (int q = c / E; q < (int)blockDim.x; q += at.V) a += sums[q * E + c % E];
      out[c] = a;
    }
  }
}

// Longer rows: a CTA each, read twice where the norm is theirs.  STAGED: the sums of dw (norm per row) lie in shared memory; else they grow where they
// end up, in the workspace (a channel's sum is one thread's).
template <typename T, Layout L, bool STAGED>
__global__ void __launch_bounds__(32 * kMaxWarps)
rotary_bwd_long_kernel(const __grid_constant__ Params p) {
  if (!grid_begin()) return;
  constexpr int E = Vec<T>::E;
  extern __shared__ __align__(16) float staged[];                    // [heads * d] (norm per row)
  __shared__ Frequencies freq;
  __shared__ Angles ang[2];
  __shared__ float2 slot[2][kMaxWarps];
  __shared__ float exchange[kMaxWarps * 32 * E];
  const Place at(p, E);
  const int l = at.l, tpr = at.tpr, c0 = at.c0;
  float* buf = exchange + (threadIdx.x >> 5) * 32 * E;
  const Tensor& t = p.t[blockIdx.y];
  const bool by_row = p.norm == VMOBA_ROTARY_NORM_ROW, normed = p.norm != VMOBA_ROTARY_NORM_NONE;
  const int row_ch = p.heads * p.d;
  const float inv_n = 1.0f / (float)(by_row ? row_ch : p.d);
  const Gradients rows(p, t, at);
  float* out = normed ? p.part + ((long long)blockIdx.y * gridDim.x + blockIdx.x) * (by_row ? row_ch : p.d) : nullptr;
  float* sums = STAGED ? staged : out;
  float acc[E];                              // (norm per head)
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.f;
  if (by_row)
    for (int i = l; i < row_ch; i += tpr) sums[i] = 0.f;
  Positions positions;
  stage_frequencies(p, &freq);
  __syncthreads();
  int turn_buf = 0;
  for (int g = blockIdx.x; g < p.B * p.S; g += gridDim.x, turn_buf ^= 1) {
    positions.load(p, freq, g, l, tpr);
    positions.angles(p, freq, l, tpr, &ang[turn_buf]);
    meet(0, p.wpr);
    Turn<E, L> turn;
    turn.load(p, ang[turn_buf], c0, -1.f);
    const int b = p.by_S.div(g), tok = g - b * p.S;
    const T *d = rows.d<T>(g, b, tok), *xs = normed ? rows.x<T>(g, b, tok) : nullptr;
    T* dst = rows.dx<T>(g, b, tok);
    // the vectors of the row: the gradient turned back, x and the weights
    auto each = [&](auto f) {
      for (int v0 = 0; v0 < at.nvec; v0 += tpr) {
        const int v = v0 + l, head = v0 >> at.vshift;
        const bool there = v < at.nvec;
        uint4 u = make_uint4(0u, 0u, 0u, 0u);
        float y[E], x[E], w[E];
        if (there) u = __ldcg(reinterpret_cast<const uint4*>(d + head * rows.d_head));
        Row<T, L>::unpack(u, y);
        turn.template apply<false>(p, y, 1.f, c0, buf);
        if (normed) {
          u = make_uint4(0u, 0u, 0u, 0u);
          if (there) u = __ldcg(reinterpret_cast<const uint4*>(xs + head * t.xs[2]));
          Row<T, L>::unpack(u, x);
          weights<E, L>(t.w && there ? t.w + (by_row ? v * E : c0) : nullptr, w);
        }
        f(v, head, there, y, x, w);
      }
    };
    float r = 1.f, back = 0.f;
    auto scales = [&](float xx, float xg) {
      r = rsqrtf(fmaf(xx, inv_n, p.eps));
      back = r * r * (xg * inv_n);
    };
    if (by_row) {
      float s[4] = {0.f, 0.f, 0.f, 0.f};
      each([&](int, int, bool, float (&y)[E], float (&x)[E], float (&w)[E]) { sums_of<E>(x, y, w, s); });
      const float2 total = row_sum<true>(make_float2(s[0] + s[1], s[2] + s[3]), 0, p.wpr, slot[turn_buf]);
      scales(total.x, total.y);
    }
    each([&](int v, int head, bool there, float (&y)[E], float (&x)[E], float (&w)[E]) {
      if (normed) {
        if (!by_row) {
          float s[4] = {0.f, 0.f, 0.f, 0.f};
          sums_of<E>(x, y, w, s);
          float two[2] = {s[0] + s[1], s[2] + s[3]};
          head_sums<2>(two, at.V);
          scales(two[0], two[1]);
          if (!there) r = back = 0.f;        // (as above)
        }
        times<E>(x, r);
        float part[E];
#pragma unroll
        for (int e = 0; e < E; ++e) part[e] = by_row ? (there ? sums[v * E + channel<E, L>(e)] : 0.f) : acc[e];
        finish<E>(y, x, w, r, back, part);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          if (!by_row) acc[e] = part[e];
          else if (there) sums[v * E + channel<E, L>(e)] = part[e];
        }
      }
      if (there) *reinterpret_cast<uint4*>(dst + head * t.ds[2]) = Row<T, L>::pack(y);
    });
  }
  if (!normed) return;
  __syncthreads();
  if (by_row) {
    if (STAGED)
      for (int i = l; i < row_ch; i += tpr) out[i] = sums[i];
    return;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) exchange[threadIdx.x * E + channel<E, L>(e)] = acc[e];
  __syncthreads();
  for (int c = threadIdx.x; c < p.d; c += blockDim.x) {
    float a = 0.f;
    for (int q = c / E; q < (int)blockDim.x; q += at.V) a += exchange[q * E + c % E];
    out[c] = a;
  }
}

// dw[tensor][i] = the sum of its parts in the order of the CTAs: 32 weights per block, a warp's lanes side by side, 32 runs of parts.
struct WeightOut { float* dw[kMaxTensors]; };
__global__ void __launch_bounds__(1024)
weight_sum_kernel(const float* __restrict__ part, int n_parts, int n_w, WeightOut o) {
  if (!grid_begin()) return;
  __shared__ double sums[32][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i = blockIdx.x * 32 + lane;
  const int run = (n_parts + 31) / 32, lo = warp * run, hi = min(lo + run, n_parts);
  const float* at = part + (long long)blockIdx.y * n_parts * n_w + i;
  double a = 0.0;
  if (i < n_w) {
#pragma unroll 8
    for (int k = lo; k < hi; ++k) a += (double)__ldg(at + (long long)k * n_w);
  }
  sums[warp][lane] = a;
  __syncthreads();
  if (warp == 0 && i < n_w) {
    a = 0.0;
    for (int k = 0; k < 32; ++k) a += sums[k][lane];
    if (o.dw[blockIdx.y]) o.dw[blockIdx.y][i] = (float)a;
  }
}

// ------------------------------------------------------------------------------ host
// How a row is laid over warps, up to `most` vectors per thread: with the most rows that a CTA of `warps` warps has under way, of equals in the
// fewest idle lanes (40 heads of 128: 549 us with four warps of five vectors, 618 with five of four; backward of 26 heads, norm per head, 54,543
// tokens: 923 us with seven warps of two vectors, the fewest idle lanes, 564 with five of three).  false: the row is longer than that, or
// its `tensors` weights are more than two CTAs of an SM have room for.
constexpr int kFwdVectors = 6, kBwdVectors = 3;
constexpr int kSmemMost = 96 * 1024;
static bool lay_out(const Dims& D, int most, int warps, int tensors, Params* p, int* nv) {
  const int nvec = D.heads * D.d * D.es / 16;
  int best = INT32_MAX;
  *nv = 0; p->groups = 0;
  for (int w = 1; w <= kMaxWarps; ++w) {
    const int v = (nvec + 32 * w - 1) / (32 * w), idle = w * 32 * v - nvec;
    if (v > most || warps / w < p->groups || (warps / w == p->groups && idle >= best)) continue;
    best = idle; *nv = v; p->wpr = w; p->groups = warps / w;
  }
  if (best < INT32_MAX &&
      (p->norm != VMOBA_ROTARY_NORM_ROW || (size_t)tensors * 32 * p->wpr * most * (16 / D.es) * sizeof(float) <= kSmemMost))
    return true;
  p->wpr = kMaxWarps; p->groups = 1;
  return false;
}
// CTAs that the SMs hold at once, `warps` of them each.
static long long resident(const Params& p, int warps) { return (long long)sm_count() * (warps / (p.wpr * p.groups)); }
// CTAs of the backward (per tensor); at most kMaxParts parts of dw.
constexpr int kMaxParts = 512;
static int bwd_ctas(const Dims& D, const Params& p) {
  return (int)std::min({((long long)D.B * D.S + p.groups - 1) / p.groups, (long long)kMaxParts, std::max(resident(p, kBwdWarps) / p.n, 1ll)});
}

static int check(const vmoba_shape* shape, const vmoba_rotary_spec* spec, Dims* D) {
  if (!spec) return VMOBA_ERR_ARG;
  if (int rc = make_dims(shape, D)) return rc;
  if ((long long)D->heads * D->d * D->es > INT32_MAX) return VMOBA_ERR_SHAPE;      // (a row's vectors are counted in 32 bits)
  if (spec->pairs < 0 || spec->pairs > D->d / 2) return VMOBA_ERR_SHAPE;
  if (spec->axes < 1 || spec->axes > 4) return VMOBA_ERR_SHAPE;
  if (spec->pos_batch != 1 && spec->pos_batch != D->B) return VMOBA_ERR_SHAPE;
  if (spec->layout != VMOBA_ROTARY_HALF && spec->layout != VMOBA_ROTARY_INTERLEAVED) return VMOBA_ERR_ARG;
  if (spec->norm < VMOBA_ROTARY_NORM_NONE || spec->norm > VMOBA_ROTARY_NORM_ROW) return VMOBA_ERR_ARG;
  if (!(spec->mscale > 0.f) || spec->mscale > 1e30f || !(spec->eps >= 0.f) || spec->eps > 1e30f) return VMOBA_ERR_ARG;
  return VMOBA_OK;
}

// Strides of a raster tensor: not negative, rows 16-byte aligned; of a tensor that is written also such that no two rows can
// share memory (a stride of zero over more than one).
static bool strides_ok(const Dims& D, const int64_t s[3], bool written) {
  const int per = 16 / D.es;
  const int n[3] = {D.B, D.S, D.heads};
  for (int i = 0; i < 3; ++i)
    if (s[i] < 0 || s[i] % per || (written && n[i] > 1 && s[i] < D.d)) return false;
  return true;
}

static unsigned token_bytes(const Dims& D, const long long s[3]) {
  const long long bytes = s[1] * D.es;
  return (D.B == 1 || s[0] == s[1] * D.S) && bytes <= 0xffffffffll ? (unsigned)bytes : 0u;
}

static void fill(const Dims& D, const vmoba_rotary_spec* spec, Params* p) {
  p->B = D.B; p->S = D.S; p->heads = D.heads; p->d = D.d;
  p->W = D.W; p->bT = D.bT; p->bH = D.bH; p->bW = D.bW; p->sb = D.sb; p->HW = D.H * D.W; p->nH = D.nH; p->nW = D.nW;
  p->by_S = FastDiv(D.S); p->by_HW = FastDiv(p->HW); p->by_W = FastDiv(D.W);
  p->by_bT = FastDiv(D.bT); p->by_bH = FastDiv(D.bH); p->by_bW = FastDiv(D.bW);
  p->pairs = spec->pairs; p->axes = spec->axes; p->layout = spec->layout; p->norm = spec->norm; p->pos_batch = spec->pos_batch;
  p->full = 2 * spec->pairs == D.d;
  p->mscale = spec->mscale; p->eps = spec->eps;
}

// Shared memory of the staged weights: whole vectors for all threads of a row, or one head's.
static size_t weight_bytes(const Dims& D, const Params& p, int nv, int tensors) {
  if (p.norm == VMOBA_ROTARY_NORM_NONE) return 0;
  return (size_t)tensors * (p.norm == VMOBA_ROTARY_NORM_ROW ? 32 * p.wpr * nv * (16 / D.es) : D.d) * sizeof(float);
}

// NV: vectors per thread; 0: the kernels for longer rows.
template <typename T, Layout L, int NV>
static int go_fwd(const Dims& D, const Params& p, cudaStream_t st) {
  const int threads = 32 * p.wpr * p.groups;
  const long long rows = ((long long)D.B * D.S + p.groups - 1) / p.groups;
  const unsigned ctas = (unsigned)std::min(rows, resident(p, 2 * kMaxWarps));
  if constexpr (NV == 0) {
    launch_kernel(early_rows(D), rotary_fwd_long_kernel<T, L>, ctas, threads, 0, st, p);
  } else {
    auto kernel = rotary_fwd_kernel<T, L, NV>;
    VMOBA_CUDA_OK(allow_smem(kernel, kSmemMost));
    launch_kernel(early_rows(D), kernel, ctas, threads, weight_bytes(D, p, NV, p.turned), st, p);
  }
  VMOBA_LAUNCH_OK(1);
  return VMOBA_OK;
}

constexpr int kLongSmemMost = 200 * 1024;

template <typename T, Layout L, int NV>
static int go_bwd(const Dims& D, const Params& p, const WeightOut& w, cudaStream_t st) {
  const int ctas = bwd_ctas(D, p), threads = 32 * p.wpr * p.groups;
  const int n_w = p.norm == VMOBA_ROTARY_NORM_ROW ? D.heads * D.d : D.d;
  const size_t sums = p.norm == VMOBA_ROTARY_NORM_ROW ? (size_t)p.groups * n_w * sizeof(float) : 0;
  if constexpr (NV == 0) {
    if (sums <= (size_t)kLongSmemMost) {
      auto kernel = rotary_bwd_long_kernel<T, L, true>;
      VMOBA_CUDA_OK(allow_smem(kernel, kLongSmemMost));
      launch_kernel(early_rows(D), kernel, dim3(ctas, p.n), threads, sums, st, p);
    } else {
      launch_kernel(early_rows(D), rotary_bwd_long_kernel<T, L, false>, dim3(ctas, p.n), threads, 0, st, p);
    }
  } else {
    auto kernel = rotary_bwd_kernel<T, L, NV>;
    VMOBA_CUDA_OK(allow_smem(kernel, kSmemMost));
    launch_kernel(early_rows(D), kernel, dim3(ctas, p.n), threads, std::max(sums, weight_bytes(D, p, NV, 1)), st, p);
  }
  VMOBA_LAUNCH_OK(1);
  if (p.norm != VMOBA_ROTARY_NORM_NONE) {
    launch_kernel(weight_sum_kernel, dim3((n_w + 31) / 32, p.n), 1024, 0, st, p.part, ctas, n_w, w);
    VMOBA_LAUNCH_OK(1);
  }
  return VMOBA_OK;
}

// The compiled variant of a shape: go(layout, vectors per thread).
template <typename T, int MOST, typename Go>
static int dispatch(const Dims& D, Params& p, int tensors, Go go) {
  int nv;
  const bool once = lay_out(D, MOST, MOST == kFwdVectors ? kMaxWarps : kBwdWarps, tensors, &p, &nv);
  auto with = [&](auto layout) {
    using std::integral_constant;
    if (!once) return go(layout, integral_constant<int, 0>{});
    if constexpr (decltype(layout)::value != kHalfAny) {      // (rare: one variant, with idle vectors)
      if (nv == 1) return go(layout, integral_constant<int, 1>{});
      if (nv == 2) return go(layout, integral_constant<int, 2>{});
      if constexpr (MOST > 3) {
        if (nv == 3) return go(layout, integral_constant<int, 3>{});
        if (nv == 4) return go(layout, integral_constant<int, 4>{});
        if (nv == 5) return go(layout, integral_constant<int, 5>{});
      }
    }
    return go(layout, integral_constant<int, MOST>{});
  };
  if (p.layout == VMOBA_ROTARY_INTERLEAVED) return with(std::integral_constant<Layout, kInterleaved>{});
  if (p.pairs % Vec<T>::E == 0) return with(std::integral_constant<Layout, kHalf>{});
  return with(std::integral_constant<Layout, kHalfAny>{});
}

template <typename T>
static int launch_fwd(const Dims& D, Params& p, cudaStream_t st) {
  return dispatch<T, kFwdVectors>(D, p, p.turned, [&](auto l, auto n) { return go_fwd<T, decltype(l)::value, decltype(n)::value>(D, p, st); });
}
template <typename T>
static int launch_bwd(const Dims& D, Params& p, const WeightOut& w, cudaStream_t st) {
  return dispatch<T, kBwdVectors>(D, p, 1, [&](auto l, auto n) { return go_bwd<T, decltype(l)::value, decltype(n)::value>(D, p, w, st); });
}

}  // namespace rotary
}  // namespace vmoba

using namespace vmoba;

extern "C" size_t vmoba_rotary_workspace_bytes(const vmoba_shape* shape, const vmoba_rotary_spec* spec, int32_t n) {
  Dims D;
  if (rotary::check(shape, spec, &D) || n < 1 || n > rotary::kMaxTensors) return 0;
  if (spec->norm == VMOBA_ROTARY_NORM_NONE) return 256;
  Carver c(nullptr);
  // (for as many parts as there can be: the size is a function of the shape alone)
  c.take<float>((size_t)n * std::min<long long>((long long)D.B * D.S, rotary::kMaxParts) * (spec->norm == VMOBA_ROTARY_NORM_ROW ? D.heads * D.d : D.d));
  return c.total();
}

extern "C" int vmoba_rotary(const vmoba_shape* shape, const vmoba_rotary_spec* spec, int32_t n, int32_t turned,
                            const void* const* src, const int64_t (*src_strides_bsh)[3], void* const* dst,
                            const int64_t (*dst_strides_bsh_or_null)[3], const float* const* weight_or_null,
                            const int32_t* positions, const double* freq, const int32_t* axis, int32_t* perm_or_null,
                            void* stream) {
  Dims D;
  if (int rc = rotary::check(shape, spec, &D)) return rc;
  if (n < 1 || n > rotary::kMaxTensors || turned < 0 || turned > n || !src || !src_strides_bsh || !dst) return VMOBA_ERR_ARG;
  if (spec->pairs > 0 && (!positions || !freq || !axis)) return VMOBA_ERR_ARG;
  rotary::Params p = {};
  rotary::fill(D, spec, &p);
  p.n = n; p.turned = turned; p.dst_bm = dst_strides_bsh_or_null == nullptr;
  p.pos = positions; p.freq = freq; p.axis = axis; p.perm = perm_or_null;
  for (int k = 0; k < n; ++k) {
    if (!src[k] || !dst[k] || !aligned16(src[k]) || !aligned16(dst[k])) return VMOBA_ERR_ARG;
    if (!rotary::strides_ok(D, src_strides_bsh[k], false)) return VMOBA_ERR_ARG;
    if (!p.dst_bm && !rotary::strides_ok(D, dst_strides_bsh_or_null[k], true)) return VMOBA_ERR_ARG;
    rotary::Tensor& t = p.t[k];
    t.src = src[k]; t.dst = dst[k];
    t.w = spec->norm != VMOBA_ROTARY_NORM_NONE && weight_or_null && k < turned ? weight_or_null[k] : nullptr;
    if (!aligned16(t.w)) return VMOBA_ERR_ARG;
    for (int i = 0; i < 3; ++i) { t.ss[i] = src_strides_bsh[k][i]; t.ds[i] = p.dst_bm ? 0 : dst_strides_bsh_or_null[k][i]; }
    t.ss1 = rotary::token_bytes(D, t.ss);
    t.ds1 = rotary::token_bytes(D, t.ds);
  }
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return D.dtype == VMOBA_BF16 ? rotary::launch_fwd<__nv_bfloat16>(D, p, st) : rotary::launch_fwd<float>(D, p, st);
}

extern "C" int vmoba_rotary_bwd(const vmoba_shape* shape, const vmoba_rotary_spec* spec, int32_t n, const void* const* d_out,
                                const int64_t (*d_out_strides_bsh_or_null)[3], const void* const* x_or_null,
                                const int64_t (*x_strides_bsh_or_null)[3], const float* const* weight_or_null, void* const* dx,
                                const int64_t (*dx_strides_bsh)[3], float* const* dweight_or_null, const int32_t* positions,
                                const double* freq, const int32_t* axis, void* ws, size_t ws_bytes, void* stream) {
  Dims D;
  if (int rc = rotary::check(shape, spec, &D)) return rc;
  const bool normed = spec->norm != VMOBA_ROTARY_NORM_NONE;
  if (n < 1 || n > rotary::kMaxTensors || !d_out || !dx || !dx_strides_bsh) return VMOBA_ERR_ARG;
  if (normed && (!x_or_null || !x_strides_bsh_or_null || !ws || !aligned16(ws))) return VMOBA_ERR_ARG;
  if (spec->pairs > 0 && (!positions || !freq || !axis)) return VMOBA_ERR_ARG;
  rotary::Params p = {};
  rotary::fill(D, spec, &p);
  p.n = n; p.turned = n; p.src_bm = d_out_strides_bsh_or_null == nullptr;
  p.pos = positions; p.freq = freq; p.axis = axis;
  rotary::WeightOut w = {};
  for (int k = 0; k < n; ++k) {
    rotary::Tensor& t = p.t[k];
    if (!d_out[k] || !dx[k] || !aligned16(d_out[k]) || !aligned16(dx[k])) return VMOBA_ERR_ARG;
    if (!p.src_bm && !rotary::strides_ok(D, d_out_strides_bsh_or_null[k], false)) return VMOBA_ERR_ARG;
    if (!rotary::strides_ok(D, dx_strides_bsh[k], true)) return VMOBA_ERR_ARG;
    t.src = d_out[k]; t.dst = dx[k];
    for (int i = 0; i < 3; ++i) {
      t.ss[i] = p.src_bm ? 0 : d_out_strides_bsh_or_null[k][i];
      t.ds[i] = dx_strides_bsh[k][i];
    }
    t.ss1 = rotary::token_bytes(D, t.ss);
    t.ds1 = rotary::token_bytes(D, t.ds);
    if (normed) {
      if (!x_or_null[k] || !aligned16(x_or_null[k]) || !rotary::strides_ok(D, x_strides_bsh_or_null[k], false)) return VMOBA_ERR_ARG;
      t.x = x_or_null[k];
      for (int i = 0; i < 3; ++i) t.xs[i] = x_strides_bsh_or_null[k][i];
      t.xs1 = rotary::token_bytes(D, t.xs);
      t.w = weight_or_null ? weight_or_null[k] : nullptr;
      if (!aligned16(t.w)) return VMOBA_ERR_ARG;
      w.dw[k] = dweight_or_null ? dweight_or_null[k] : nullptr;
    }
  }
  if (normed && ws_bytes < vmoba_rotary_workspace_bytes(shape, spec, n)) return VMOBA_ERR_WORKSPACE;
  p.part = static_cast<float*>(ws);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return D.dtype == VMOBA_BF16 ? rotary::launch_bwd<__nv_bfloat16>(D, p, w, st) : rotary::launch_bwd<float>(D, p, w, st);
}
