// Rotary positions of q and k, with the root-mean-square norm that video transformers put ahead of them, on the way into the
// layer; and the gradients on the way out.  With y = x r w, r = 1 / sqrt(mean(x^2) + eps) (or y = x), and pair i of a head turned by the
// angle a = pos[axis[i]] * freq[i]:
//   out0 = m (y0 cos a - y1 sin a),  out1 = m (y1 cos a + y0 sin a);   the other channels pass through.
// Backward: g = the gradient of out turned by -a (times m), then with s = w g:
//   dx = r (s - x r^2 mean(s x)),   dw = sum over tokens (norm per head: and heads) of g x r.
//
// Bound by HBM (a row of a token, all heads, is read once and written once, forward; the gradient, x and dx, backward) and, closely
// behind, by instruction issue.  So: a row is taken by as few warps as hold it in six 16-byte vectors per thread, each warp or
// group of warps on its own, token after token; a thread has the same channels of every head, so that its sines and cosines are
// loaded once per token; angles are worked out once per token for all heads and tensors; layouts and vectors per thread are compiled in.
// The norm's two trips through a row are one through memory: vectors come in by asynchronous copies into a ring of shared
// memory that each thread has to itself, rows ahead of their use; rows longer than that are read twice.
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
constexpr int kMaxWarps = 8;                 // of a CTA, and of a row
constexpr int kMaxPairs = 64;

struct Tensor {
  const void* src;                           // forward: x; backward: the gradient of the output
  const void* x;                             // backward with a norm: x
  void* dst;
  const float* w;                            // norm weights or null (ones)
  long long ss[3], xs[3], ds[3];             // element strides {batch, token, head} of src, x and dst
};

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
__device__ __forceinline__ void angles(const Params& p, int g, int l, int tpr, Angles* ang) {
  const int at0 = p.pos_batch > 1 ? g : g - p.by_S.div(g) * p.S;
#pragma unroll 1
  for (int pair = l; pair < p.pairs; pair += tpr) {
    const int at = __ldg(p.pos + (long long)at0 * p.axes + min(max(__ldg(p.axis + pair), 0), p.axes - 1));
    const double turns = (double)at * __ldg(p.freq + pair) * 0.15915494309189533577;      // 1 / (2 pi)
    float sn, cs;
    sincospif(2.0f * (float)(turns - rint(turns)), &sn, &cs);
    ang->cs[pair] = cs * p.mscale;
    ang->sn[pair] = sn * p.mscale;
  }
}

// A thread's ring: kDepth rows of its vectors.
constexpr int kDepth = 2;
__device__ __forceinline__ void copy16(uint4* to, const void* from, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from), "r"(there ? 16u : 0u) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// What a thread's vectors, all of the same channels c0 .. c0 + E - 1 of a head, are turned by.  sign: -1 turns back.
template <int E, Layout L>
struct Turn {
  float cs[L == kInterleaved ? E / 2 : E], sn[L == kInterleaved ? E / 2 : E];
  uint32_t mine;                             // bit e: channel c0 + e belongs to a pair
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
      const int n = 2 * p.pairs - c0;
      mine = n <= 0 ? 0u : n >= E ? (1u << E) - 1u : (1u << n) - 1u;
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
  // buf (kHalfAny): 32 * E floats of the warp.  Called by whole warps.
  __device__ __forceinline__ void apply(const Params& p, float (&y)[E], int c0, float* buf) const {
    if constexpr (L == kInterleaved) {
      auto turned = [&](bool all) {
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
          const float y0 = y[2 * i], y1 = y[2 * i + 1];
          if (all || (mine >> (2 * i) & 1)) {
            y[2 * i] = fmaf(y0, cs[i], -y1 * sn[i]);
            y[2 * i + 1] = fmaf(y1, cs[i], y0 * sn[i]);
          }
        }
      };
      if (p.full) turned(true);
      else turned(false);
    } else {
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
        for (int e = 0; e < E; ++e) y[e] = fmaf(y[e], cs[e], o[e] * sn[e]);
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

// Sum over the threads of a row.  slot: a pair of floats per warp of the group; the next call takes another one (a call that takes
// this one again is two barriers away).
__device__ __forceinline__ float2 row_sum(float2 v, int group, int wpr, float2* slot) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
    v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
  }
  if (wpr == 1) return v;
  if ((threadIdx.x & 31) == 0) slot[(threadIdx.x >> 5) - group * wpr] = v;
  meet(group, wpr);
  float2 a = make_float2(0.f, 0.f);
  for (int w = 0; w < wpr; ++w) { a.x += slot[w].x; a.y += slot[w].y; }
  return a;
}
__device__ __forceinline__ float2 head_sum(float2 v, int lanes) {
  for (int o = lanes >> 1; o > 0; o >>= 1) {
    v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
    v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
  }
  return v;
}

template <int E>
__device__ __forceinline__ void weights(const float* w, float (&x)[E]) {
#pragma unroll
  for (int e = 0; e < E; e += 4) {
    const float4 v = w ? __ldg(reinterpret_cast<const float4*>(w + e)) : make_float4(1.f, 1.f, 1.f, 1.f);
    x[e] = v.x; x[e + 1] = v.y; x[e + 2] = v.z; x[e + 3] = v.w;
  }
}

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

// ------------------------------------------------------------------------------ forward
// ONCE: the row fits the group's threads; else it is walked in trips, from global memory.
template <typename T, Layout L, int NV, bool ONCE>
__global__ void __launch_bounds__(32 * kMaxWarps, 3)
rotary_fwd_kernel(const __grid_constant__ Params p) {
  if (!grid_begin()) return;
  constexpr int E = Vec<T>::E;
  extern __shared__ __align__(16) uint4 ring[];                      // [kDepth][NV][threads]
  __shared__ Angles ang[kMaxWarps][2];
  __shared__ float2 slot[2][kMaxWarps];
  __shared__ float exchange[L == kHalfAny ? kMaxWarps * 32 * E : 1];
  const int warp = threadIdx.x >> 5, group = warp / p.wpr, tpr = 32 * p.wpr, l = threadIdx.x - group * tpr, threads = blockDim.x;
  float* buf = L == kHalfAny ? exchange + warp * 32 * E : exchange;
  uint4* mine = ring + threadIdx.x;
  const int V = p.d / E, nvec = p.heads * V, c0 = (l % V) * E, vshift = 31 - __clz(V), head0 = l >> vshift, heads_per = tpr >> vshift;
  const int per = NV * tpr;                  // vectors of a trip through a row
  const int tokens = p.B * p.S, step = gridDim.x * p.groups;
  // The row of (token, tensor): this thread's first vector.
  auto src_row = [&](int g, int k) {
    const Tensor& t = p.t[k];
    const int b = p.by_S.div(g);
    return reinterpret_cast<const T*>(t.src) + b * t.ss[0] + (long long)(g - b * p.S) * t.ss[1] + head0 * t.ss[2] + c0;
  };
  int g = blockIdx.x * p.groups + group;
  if (g >= tokens) return;                   // (whole groups)
  int ga = g, ka = p.n - 1;                  // the next row to ask for
  uint4* in = mine;                          // and its place
  auto ask = [&]() {
    if (ONCE) {
      if (ga < tokens) {
        const T* at = src_row(ga, ka);
        const long long apart = heads_per * p.t[ka].ss[2];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const bool there = l + i * tpr < nvec;
          copy16(in + i * threads, there ? at : reinterpret_cast<const T*>(p.t[ka].src), there);
          at += apart;
        }
        if (--ka < 0) { ka = p.n - 1; ga += step; }
      }
      copies_commit();
      in = in == mine ? mine + NV * threads : mine;      // (kDepth = 2)
    }
  };
  ask();
  ask();
  angles(p, g, l, tpr, &ang[group][0]);
  int turn_buf = 0, sum_buf = 0;
  const uint4* row = mine;
  for (; g < tokens; g += step, turn_buf ^= 1) {
    meet(group, p.wpr);                      // (this token's angles)
    Turn<E, L> turn;
    turn.load(p, ang[group][turn_buf], c0, 1.f);
    const int b = p.by_S.div(g), tok = g - b * p.S, bm = p.dst_bm || p.perm ? block_pos(p, tok) : 0;
    if (p.perm && b == 0 && l == 0) p.perm[bm] = tok;
    // tensors from the last to the first: what the caller reads next comes last
#pragma unroll 1
    for (int k = p.n - 1; k >= 0; --k) {
      if (ONCE) copies_wait<kDepth - 1>();
      const Tensor& t = p.t[k];
      auto vec = [&](int v0, int i) {
        if (ONCE) return row[i * threads];
        uint4 x = make_uint4(0u, 0u, 0u, 0u);
        if (v0 + l + i * tpr < nvec) x = __ldcg(reinterpret_cast<const uint4*>(src_row(g, k) + ((v0 >> vshift) + i * heads_per) * t.ss[2]));
        return x;
      };
      const bool turned = k < p.turned;
      const int norm = turned ? p.norm : VMOBA_ROTARY_NORM_NONE;
      float r_row = 1.f;
      if (norm == VMOBA_ROTARY_NORM_ROW) {
        float s0 = 0.f, s1 = 0.f;
        for (int v0 = 0; v0 < nvec; v0 += per) {
#pragma unroll
          for (int i = 0; i < NV; ++i) {
            float x[E];
            Vec<T>::unpack(vec(v0, i), x);
            dot<E>(x, x, s0, s1);
          }
          if (ONCE) break;
        }
        r_row = rsqrtf(row_sum(make_float2(s0 + s1, 0.f), group, p.wpr, slot[sum_buf] + group * p.wpr).x / (float)(p.heads * p.d) + p.eps);
        sum_buf ^= 1;
      }
      if (k == 0 && g + step < tokens) angles(p, g + step, l, tpr, &ang[group][turn_buf ^ 1]);
      const long long to_head = p.dst_bm ? (long long)p.S * p.d : t.ds[2], to_next = heads_per * to_head;
      T* dst = reinterpret_cast<T*>(t.dst) + (p.dst_bm ? ((long long)b * p.heads * p.S + bm) * p.d : b * t.ds[0] + tok * t.ds[1]) +
               head0 * to_head + c0;
      // the vectors of a trip, each through f
      auto each = [&](auto f) {
        for (int v0 = 0; v0 < nvec; v0 += per) {
          const float* w = t.w ? t.w + (norm == VMOBA_ROTARY_NORM_ROW ? (v0 + l) * E : c0) : nullptr;
#pragma unroll
          for (int i = 0; i < NV; ++i) {
            const bool there = v0 + l + i * tpr < nvec;
            if (__any_sync(0xffffffffu, there)) {
              float y[E];
              Vec<T>::unpack(vec(v0, i), y);
              f(y, there ? w : nullptr);
              if (there) *reinterpret_cast<uint4*>(dst) = Vec<T>::pack(y);
            }
            dst += to_next;
            if (w && norm == VMOBA_ROTARY_NORM_ROW) w += tpr * E;
          }
          if (ONCE) break;
        }
      };
      if (!turned) {
        each([&](float (&)[E], const float*) {});
      } else if (norm == VMOBA_ROTARY_NORM_ROW) {
        each([&](float (&y)[E], const float* w) {
          float f[E];
          weights<E>(w, f);
          times<E>(y, r_row);
          times<E>(y, f);
          turn.apply(p, y, c0, buf);
        });
      } else if (norm == VMOBA_ROTARY_NORM_HEAD) {
        each([&](float (&y)[E], const float* w) {
          float f[E], s0 = 0.f, s1 = 0.f;
          dot<E>(y, y, s0, s1);
          weights<E>(w, f);
          times<E>(y, rsqrtf(head_sum(make_float2(s0 + s1, 0.f), V).x / (float)p.d + p.eps));
          times<E>(y, f);
          turn.apply(p, y, c0, buf);
        });
      } else {
        each([&](float (&y)[E], const float*) { turn.apply(p, y, c0, buf); });
      }
      row = row == mine ? mine + NV * threads : mine;
      ask();                                 // (into the place of the row that has just been read)
    }
  }
}

// ------------------------------------------------------------------------------ backward
// blockIdx.y: tensor.  A thread has the same channels in every row that its group takes, and keeps their part of dw in registers (rows
// longer than that: in shared memory).  The parts of a CTA's groups, and of the CTAs (weight_sum_kernel), are added up in a
// fixed order: the results repeat bit for bit.
template <typename T, Layout L, int NV, bool ONCE>
__global__ void __launch_bounds__(32 * kMaxWarps, 2)
rotary_bwd_kernel(const __grid_constant__ Params p) {
  if (!grid_begin()) return;
  constexpr int E = Vec<T>::E;
  extern __shared__ __align__(16) uint4 ring[];                      // [kDepth][dy, x][NV][threads]; then, or instead, [group][heads * d]
  float* acc_row = reinterpret_cast<float*>(ring);
  __shared__ Angles ang[kMaxWarps][2];
  __shared__ float2 slot[2][kMaxWarps];
  __shared__ float exchange[kMaxWarps * 32 * E];
  const int warp = threadIdx.x >> 5, group = warp / p.wpr, tpr = 32 * p.wpr, l = threadIdx.x - group * tpr, threads = blockDim.x;
  float* buf = exchange + warp * 32 * E;
  uint4* mine = ring + threadIdx.x;
  const int V = p.d / E, nvec = p.heads * V, c0 = (l % V) * E, vshift = 31 - __clz(V), head0 = l >> vshift, heads_per = tpr >> vshift;
  const int per = NV * tpr;
  const Tensor& t = p.t[blockIdx.y];
  const int tokens = p.B * p.S, step = gridDim.x * p.groups;
  const bool by_row = p.norm == VMOBA_ROTARY_NORM_ROW, by_head = p.norm == VMOBA_ROTARY_NORM_HEAD, normed = by_row || by_head;
  const int row_ch = p.heads * p.d;
  const float inv_n = 1.0f / (float)(by_row ? row_ch : p.d);
  float acc[NV][E];
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < E; ++e) acc[i][e] = 0.f;
  float* mine_acc = acc_row + (long long)group * row_ch;
  if (by_row && !ONCE)
    for (int i = l; i < row_ch; i += tpr) mine_acc[i] = 0.f;
  const long long d_head = p.src_bm ? (long long)p.S * p.d : t.ss[2];
  auto d_row = [&](int g) {
    const int b = p.by_S.div(g), tok = g - b * p.S;
    return reinterpret_cast<const T*>(t.src) + (p.src_bm ? ((long long)b * p.heads * p.S + block_pos(p, tok)) * p.d : b * t.ss[0] + tok * t.ss[1]) +
           head0 * d_head + c0;
  };
  auto x_row = [&](int g) {
    const int b = p.by_S.div(g), tok = g - b * p.S;
    return reinterpret_cast<const T*>(t.x) + b * t.xs[0] + tok * t.xs[1] + head0 * t.xs[2] + c0;
  };
  int g = blockIdx.x * p.groups + group;
  if (g < tokens) {                          // (whole groups; all threads meet again at the end)
    int ga = g;
    uint4* in = mine;
    auto ask = [&]() {
      if (ONCE) {
        if (ga < tokens) {
          const T *d = d_row(ga), *x = normed ? x_row(ga) : nullptr;
#pragma unroll
          for (int i = 0; i < NV; ++i) {
            const bool there = l + i * tpr < nvec;
            copy16(in + i * threads, there ? d : reinterpret_cast<const T*>(t.src), there);
            if (normed) copy16(in + (NV + i) * threads, there ? x : reinterpret_cast<const T*>(t.x), there);
            d += heads_per * d_head;
            x += heads_per * t.xs[2];
          }
          ga += step;
        }
        copies_commit();
        in = in == mine ? mine + 2 * NV * threads : mine;      // (kDepth = 2)
      }
    };
    ask();
    ask();
    angles(p, g, l, tpr, &ang[group][0]);
    int turn_buf = 0;
    const uint4* row = mine;
    for (; g < tokens; g += step, turn_buf ^= 1) {
      meet(group, p.wpr);                    // (this token's angles)
      Turn<E, L> turn;
      turn.load(p, ang[group][turn_buf], c0, -1.f);
      if (ONCE) copies_wait<kDepth - 1>();
      auto vec_d = [&](int v0, int i) {
        if (ONCE) return row[i * threads];
        uint4 u = make_uint4(0u, 0u, 0u, 0u);
        if (v0 + l + i * tpr < nvec) u = __ldcg(reinterpret_cast<const uint4*>(d_row(g) + ((v0 >> vshift) + i * heads_per) * d_head));
        return u;
      };
      auto vec_x = [&](int v0, int i) {
        if (ONCE) return row[(NV + i) * threads];
        uint4 u = make_uint4(0u, 0u, 0u, 0u);
        if (v0 + l + i * tpr < nvec) u = __ldcg(reinterpret_cast<const uint4*>(x_row(g) + ((v0 >> vshift) + i * heads_per) * t.xs[2]));
        return u;
      };
      float r = 1.f, back = 0.f;             // 1 / rms; r^2 times the mean of x times its weighted gradient
      auto scales = [&](const float2& s) {
        r = rsqrtf(fmaf(s.x, inv_n, p.eps));
        back = r * r * (s.y * inv_n);
      };
      if (by_row) {
        float s0 = 0.f, s1 = 0.f, u0 = 0.f, u1 = 0.f;
        for (int v0 = 0; v0 < nvec; v0 += per) {
          const float* w = t.w ? t.w + (v0 + l) * E : nullptr;
#pragma unroll
          for (int i = 0; i < NV; ++i) {
            const bool there = v0 + l + i * tpr < nvec;
            if (__any_sync(0xffffffffu, there)) {
              float y[E], x[E], f[E];
              Vec<T>::unpack(vec_d(v0, i), y);
              turn.apply(p, y, c0, buf);
              Vec<T>::unpack(vec_x(v0, i), x);
              weights<E>(there ? w : nullptr, f);
              dot<E>(x, x, s0, s1);
              times<E>(y, f);
              dot<E>(x, y, u0, u1);
            }
            if (w) w += tpr * E;
          }
          if (ONCE) break;
        }
        scales(row_sum(make_float2(s0 + s1, u0 + u1), group, p.wpr, slot[turn_buf] + group * p.wpr));
      }
      if (g + step < tokens) angles(p, g + step, l, tpr, &ang[group][turn_buf ^ 1]);
      const int b = p.by_S.div(g), tok = g - b * p.S;
      T* dst = reinterpret_cast<T*>(t.dst) + b * t.ds[0] + tok * t.ds[1] + head0 * t.ds[2] + c0;
      for (int v0 = 0; v0 < nvec; v0 += per) {
        const float* w = t.w ? t.w + (by_row ? (v0 + l) * E : c0) : nullptr;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const bool there = v0 + l + i * tpr < nvec;
          if (__any_sync(0xffffffffu, there)) {
            float y[E];
            Vec<T>::unpack(vec_d(v0, i), y);
            turn.apply(p, y, c0, buf);
            if (normed) {
              float x[E], f[E];
              Vec<T>::unpack(vec_x(v0, i), x);
              weights<E>(there ? w : nullptr, f);
              float yw[E];
#pragma unroll
              for (int e = 0; e < E; e += 2) mul2(yw[e], yw[e + 1], y[e], y[e + 1], f[e], f[e + 1]);
              if (by_head) {
                float s0 = 0.f, s1 = 0.f, u0 = 0.f, u1 = 0.f;
                dot<E>(x, x, s0, s1);
                dot<E>(x, yw, u0, u1);
                scales(head_sum(make_float2(s0 + s1, u0 + u1), V));
              }
#pragma unroll
              for (int e = 0; e < E; e += 2) {
                mul2(y[e], y[e + 1], y[e], y[e + 1], r, r);
                if (by_row && !ONCE) {
                  if (there) {
                    float* a = mine_acc + (v0 + l + i * tpr) * E + e;
                    a[0] = fmaf(y[e], x[e], a[0]);
                    a[1] = fmaf(y[e + 1], x[e + 1], a[1]);
                  }
                } else {
                  fma2(acc[i][e], acc[i][e + 1], y[e], y[e + 1], x[e], x[e + 1], acc[i][e], acc[i][e + 1]);      // (zeros beyond the row)
                }
                fma2(y[e], y[e + 1], x[e], x[e + 1], -back, -back, yw[e], yw[e + 1]);
                mul2(y[e], y[e + 1], y[e], y[e + 1], r, r);
              }
            }
            if (there) *reinterpret_cast<uint4*>(dst) = Vec<T>::pack(y);
          }
          dst += heads_per * t.ds[2];
          if (w && by_row) w += tpr * E;
        }
        if (ONCE) break;
      }
      row = row == mine ? mine + 2 * NV * threads : mine;
      ask();
    }
  }
  if (!normed) return;
  const int n_w = by_row ? row_ch : p.d;
  float* out = p.part + ((long long)blockIdx.y * gridDim.x + blockIdx.x) * n_w;
  if (by_row) {
    copies_wait<0>();
    __syncthreads();                         // (the ring is free)
    if (ONCE) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < E; e += 4)
          if (l + i * tpr < nvec)
            *reinterpret_cast<float4*>(mine_acc + (l + i * tpr) * E + e) = make_float4(acc[i][e], acc[i][e + 1], acc[i][e + 2], acc[i][e + 3]);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < row_ch; i += threads) {
      float a = 0.f;
      for (int q = 0; q < p.groups; ++q) a += acc_row[(long long)q * row_ch + i];
      out[i] = a;
    }
  } else {
    __syncthreads();                         // (the exchange buffers are free)
#pragma unroll
    for (int e = 0; e < E; ++e) {
      float a = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i) a += acc[i][e];
      exchange[threadIdx.x * E + e] = a;
    }
    __syncthreads();
    for (int c = threadIdx.x; c < p.d; c += threads) {               // threads c / E, c / E + V, ... hold channel c
      float a = 0.f;
      for (int q = c / E; q < threads; q += V) a += exchange[q * E + c % E];
      out[c] = a;
    }
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
// How a row is laid over warps: up to six vectors per thread in the fewest idle lanes, of equals the fewest warps; CTAs of about eight
// warps.  false: the row is longer than that (eight warps, trips of four vectors per thread).
constexpr int kMaxNv = 6;
static bool lay_out(const Dims& D, Params* p, int* nv) {
  const int nvec = D.heads * D.d * D.es / 16;
  int best = INT32_MAX;
  *nv = 4; p->wpr = kMaxWarps; p->groups = 1;
  for (int w = 1; w <= kMaxWarps; ++w)
    for (int v = 1; v <= kMaxNv; ++v) {
      const int idle = w * 32 * v - nvec;
      if (idle >= 0 && idle < best) { best = idle; *nv = v; p->wpr = w; p->groups = kMaxWarps / w; }
    }
  return best < INT32_MAX;
}
// CTAs of the backward (per tensor); at most kMaxParts parts of dw.
constexpr int kMaxParts = 512;
static int bwd_ctas(const Dims& D, const Params& p) {
  return (int)std::min<long long>(((long long)D.B * D.S + p.groups - 1) / p.groups, std::min(kMaxParts, 2 * sm_count()));
}

static int check(const vmoba_shape* shape, const vmoba_rotary_spec* spec, Dims* D) {
  if (!spec) return VMOBA_ERR_ARG;
  if (int rc = make_dims(shape, D)) return rc;
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

static void fill(const Dims& D, const vmoba_rotary_spec* spec, Params* p) {
  p->B = D.B; p->S = D.S; p->heads = D.heads; p->d = D.d;
  p->W = D.W; p->bT = D.bT; p->bH = D.bH; p->bW = D.bW; p->sb = D.sb; p->HW = D.H * D.W; p->nH = D.nH; p->nW = D.nW;
  p->by_S = FastDiv(D.S); p->by_HW = FastDiv(p->HW); p->by_W = FastDiv(D.W);
  p->by_bT = FastDiv(D.bT); p->by_bH = FastDiv(D.bH); p->by_bW = FastDiv(D.bW);
  p->pairs = spec->pairs; p->axes = spec->axes; p->layout = spec->layout; p->norm = spec->norm; p->pos_batch = spec->pos_batch;
  p->full = 2 * spec->pairs == D.d;
  p->mscale = spec->mscale; p->eps = spec->eps;
}

template <typename T, Layout L, int NV, bool ONCE>
static int go_fwd(const Dims& D, const Params& p, cudaStream_t st) {
  auto kernel = rotary_fwd_kernel<T, L, NV, ONCE>;
  const int threads = 32 * p.wpr * p.groups;
  const long long ctas = ((long long)D.B * D.S + p.groups - 1) / p.groups;
  VMOBA_CUDA_OK(allow_smem(kernel, kDepth * NV * 32 * kMaxWarps * 16));
  launch_kernel(early_rows(D), kernel, (unsigned)std::min<long long>(ctas, 3ll * sm_count()), threads,
                ONCE ? (size_t)kDepth * NV * threads * 16 : 0, st, p);
  VMOBA_LAUNCH_OK(1);
  return VMOBA_OK;
}

static size_t bwd_smem(const Dims& D, const Params& p, int nv, bool once) {
  const size_t ring = once ? (size_t)2 * kDepth * nv * 32 * p.wpr * p.groups * 16 : 0;
  return std::max(ring, p.norm == VMOBA_ROTARY_NORM_ROW ? (size_t)p.groups * D.heads * D.d * sizeof(float) : 0);
}
constexpr int kBwdSmemMost = 200 * 1024;

template <typename T, Layout L, int NV, bool ONCE>
static int go_bwd(const Dims& D, const Params& p, const WeightOut& w, cudaStream_t st) {
  auto kernel = rotary_bwd_kernel<T, L, NV, ONCE>;
  const int ctas = bwd_ctas(D, p);
  const size_t smem = bwd_smem(D, p, NV, ONCE);
  if (smem > (size_t)kBwdSmemMost) return VMOBA_ERR_NOT_IMPLEMENTED;
  VMOBA_CUDA_OK(allow_smem(kernel, kBwdSmemMost));
  launch_kernel(early_rows(D), kernel, dim3(ctas, p.n), 32 * p.wpr * p.groups, smem, st, p);
  VMOBA_LAUNCH_OK(1);
  if (p.norm != VMOBA_ROTARY_NORM_NONE) {
    const int n_w = p.norm == VMOBA_ROTARY_NORM_ROW ? D.heads * D.d : D.d;
    launch_kernel(weight_sum_kernel, dim3((n_w + 31) / 32, p.n), 1024, 0, st, p.part, ctas, n_w, w);
    VMOBA_LAUNCH_OK(1);
  }
  return VMOBA_OK;
}

// The compiled variant of a shape: go(layout, vectors per thread, whether the row fits).
template <typename T, typename Go>
static int dispatch(const Dims& D, Params& p, Go go) {
  int nv;
  const bool once = lay_out(D, &p, &nv);
  auto with = [&](auto layout) {
    constexpr Layout L = decltype(layout)::value;
    auto pick = [&](auto n, auto o) { return go(layout, n, o); };
    using std::integral_constant;
    if (!once) return pick(integral_constant<int, 4>{}, std::false_type{});
    if constexpr (L == kHalfAny) {           // (rare: one variant, with idle vectors)
      return pick(integral_constant<int, kMaxNv>{}, std::true_type{});
    } else {
      switch (nv) {
        case 1: return pick(integral_constant<int, 1>{}, std::true_type{});
        case 2: return pick(integral_constant<int, 2>{}, std::true_type{});
        case 3: return pick(integral_constant<int, 3>{}, std::true_type{});
        case 4: return pick(integral_constant<int, 4>{}, std::true_type{});
        case 5: return pick(integral_constant<int, 5>{}, std::true_type{});
        default: return pick(integral_constant<int, 6>{}, std::true_type{});
      }
    }
  };
  if (p.layout == VMOBA_ROTARY_INTERLEAVED) return with(std::integral_constant<Layout, kInterleaved>{});
  if (p.pairs % Vec<T>::E == 0) return with(std::integral_constant<Layout, kHalf>{});
  return with(std::integral_constant<Layout, kHalfAny>{});
}

template <typename T>
static int launch_fwd(const Dims& D, Params& p, cudaStream_t st) {
  return dispatch<T>(D, p, [&](auto l, auto n, auto o) { return go_fwd<T, decltype(l)::value, decltype(n)::value, decltype(o)::value>(D, p, st); });
}
template <typename T>
static int launch_bwd(const Dims& D, Params& p, const WeightOut& w, cudaStream_t st) {
  return dispatch<T>(D, p, [&](auto l, auto n, auto o) { return go_bwd<T, decltype(l)::value, decltype(n)::value, decltype(o)::value>(D, p, w, st); });
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
    if (normed) {
      if (!x_or_null[k] || !aligned16(x_or_null[k]) || !rotary::strides_ok(D, x_strides_bsh_or_null[k], false)) return VMOBA_ERR_ARG;
      t.x = x_or_null[k];
      for (int i = 0; i < 3; ++i) t.xs[i] = x_strides_bsh_or_null[k][i];
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
