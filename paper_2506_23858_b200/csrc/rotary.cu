// Rotary positions of q and k, with the root-mean-square norm that video transformers put ahead of them, on the way into the
// layer; and the gradients on the way out.  With y = x r w, r = 1 / sqrt(mean(x^2) + eps) (or y = x), and pair i of a head turned by the
// angle a = pos[axis[i]] * freq[i]:
//   out0 = m (y0 cos a - y1 sin a),  out1 = m (y1 cos a + y0 sin a);   the other channels pass through.
// Backward: g = the gradient of out turned by -a (times m), then with s = w g:
//   dx = r (s - x r^2 mean(s x)),   dw = sum over tokens (norm per head: and heads) of g x r.
//
// Bound by HBM: a row of a token (all heads) is read once and written once, forward; the gradient, x and dx, backward.  The
// norm's two trips through a row are one through memory because the row stays in registers (up to eight 16-byte vectors per
// thread; longer rows are read twice).  A row is taken by 1, 2, 4 or 8 warps.  The angles of a token are worked out once for all heads and
// tensors of a CTA: product and reduction to (-pi, pi] in 64 bits, because a position of 10^6 times a frequency of one has no digit
// behind the point left in 32.
#include <algorithm>

#include "common.cuh"

namespace vmoba {
namespace rotary {

constexpr int kMaxTensors = 4;
constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int NV = 8;                        // 16-byte vectors of a row per thread and trip
constexpr int kMaxTok = 16;                  // tokens of a CTA at a time

struct Tensor {
  const void* src;                           // forward: x; backward: the gradient of the output
  const void* x;                             // backward with a norm: x
  void* dst;
  const float* w;                            // norm weights or null (ones)
  long long ss[3], xs[3], ds[3];             // element strides {batch, token, head} of src, x and dst
};

struct Params {
  int B, S, heads, d;
  int T, H, W, bT, bH, bW, nH, nW;
  int n, turned;                             // tensors; the first `turned` of them are normed and rotated, the others only moved
  int pairs, axes, layout, norm, pos_batch;
  int src_bm, dst_bm;                        // src / dst is block-major (strides unused)
  float mscale, eps;
  const int* pos;
  const double* freq;
  const int* axis;
  int* perm;
  int wpr;                                   // warps per row
  int tok;                                   // tokens per CTA and trip
  float* part;                               // backward: [tensor][CTA][weights] partial sums of dw
  Tensor t[kMaxTensors];
};

__host__ __device__ constexpr size_t ang_bytes(int tok, int pairs) { return ((size_t)tok * pairs * sizeof(float2) + 15) / 16 * 16; }

// Block-major position of raster token r (the inverse of Eq. 1).
__device__ __forceinline__ int block_pos(const Params& p, int r) {
  const int hw = p.H * p.W, t = r / hw, r2 = r - t * hw, h = r2 / p.W, w = r2 - h * p.W;
  const int jt = t / p.bT, jh = h / p.bH, jw = w / p.bW;
  const int block = (jt * p.nH + jh) * p.nW + jw;
  const int slot = ((t - jt * p.bT) * p.bH + (h - jh * p.bH)) * p.bW + (w - jw * p.bW);
  return block * (p.bT * p.bH * p.bW) + slot;
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

// cos and sin (times mscale) of the angles of `count` tokens from flat token index first on, into ang[token][pair].
__device__ __forceinline__ void angles(const Params& p, long long first, int count, float2* ang) {
  constexpr double kTurn = 6.283185307179586476925, kTurnLow = 2.4492935982947064e-16;      // 2 pi and what its double lacks
  for (int i = threadIdx.x; i < count * p.pairs; i += kThreads) {
    const int t = i / p.pairs, pair = i - t * p.pairs;
    const long long g = first + t;
    const int b = (int)(g / p.S), s = (int)(g - (long long)b * p.S);
    const int at = __ldg(p.pos + ((long long)(p.pos_batch > 1 ? b : 0) * p.S + s) * p.axes + min(max(__ldg(p.axis + pair), 0), p.axes - 1));
    const double a = (double)at * __ldg(p.freq + pair), turns = rint(a * (1.0 / kTurn));
    const float r = (float)fma(-turns, kTurnLow, fma(-turns, kTurn, a));
    float sn, cs;
    sincosf(r, &sn, &cs);
    ang[i] = make_float2(cs * p.mscale, sn * p.mscale);
  }
}

// What a thread's vectors, all of the same channels c0 .. c0 + E - 1 of a head, are turned by: out[e] = y[e] cs[e] + partner[e] sn[e].
template <int E>
struct Turn {
  float cs[E], sn[E];
  uint32_t mine;                             // bit e: channel c0 + e belongs to a pair
  __device__ __forceinline__ void load(const Params& p, const float2* ang, int c0, float sign) {
    mine = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int c = c0 + e;
      const bool second = p.layout == VMOBA_ROTARY_HALF ? c >= p.pairs : (c & 1) != 0;
      const int pair = p.layout == VMOBA_ROTARY_HALF ? (second ? c - p.pairs : c) : c >> 1;
      cs[e] = 1.f; sn[e] = 0.f;
      if (c < 2 * p.pairs) {
        const float2 a = ang[pair];
        cs[e] = a.x;
        sn[e] = second ? sign * a.y : -sign * a.y;
        mine |= 1u << e;
      }
    }
  }
};

// The partner of each of a thread's channels.  Interleaved: its neighbour.  Half: `pairs` channels away in the same head, whose
// vectors are in neighbouring lanes; by shuffles where whole vectors are partners (WHOLE), else through shared memory.
// Called by whole warps.
template <int E, bool WHOLE>
__device__ __forceinline__ void partners(const Params& p, const float (&y)[E], float (&o)[E], int c0, uint32_t mine, float* buf) {
  if (p.layout == VMOBA_ROTARY_INTERLEAVED) {
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = y[e ^ 1];
  } else if constexpr (WHOLE) {
    const int lane = threadIdx.x & 31, by = p.pairs / E;
    const int from = c0 < p.pairs ? lane + by : lane - by;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = __shfl_sync(0xffffffffu, y[e], from & 31);
  } else {
    const int lane = threadIdx.x & 31;
    __syncwarp();
#pragma unroll
    for (int e = 0; e < E; ++e) buf[lane * E + e] = y[e];
    __syncwarp();
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = (mine >> e & 1) ? buf[lane * E + e + (c0 + e < p.pairs ? p.pairs : -p.pairs)] : 0.f;
  }
}

// Sum over the threads of a row (all of the CTA call this); slot: two floats per warp.
__device__ __forceinline__ float2 row_sum(float2 v, int wpr, float2* slot) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
    v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
  }
  if (wpr == 1) return v;
  const int warp = threadIdx.x >> 5;
  __syncthreads();                           // (the row before has been read)
  if ((threadIdx.x & 31) == 0) slot[warp] = v;
  __syncthreads();
  float2 a = make_float2(0.f, 0.f);
  for (int w = warp / wpr * wpr; w < (warp / wpr + 1) * wpr; ++w) { a.x += slot[w].x; a.y += slot[w].y; }
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

// Where a row of a tensor begins and how far its heads lie apart, in elements.
struct RowAt { long long base, head; };
__device__ __forceinline__ RowAt row_at(const Params& p, bool bm, const long long (&s)[3], int b, int tok) {
  if (bm) return {((long long)b * p.heads * p.S + block_pos(p, tok)) * p.d, (long long)p.S * p.d};
  return {b * s[0] + tok * s[1], s[2]};
}

// ------------------------------------------------------------------------------ forward
template <typename T, bool WHOLE>
__global__ void __launch_bounds__(kThreads)
rotary_fwd_kernel(const __grid_constant__ Params p) {
  if (!grid_begin()) return;
  constexpr int E = Vec<T>::E;
  extern __shared__ __align__(16) uint8_t smem[];
  float2* ang = reinterpret_cast<float2*>(smem);                                  // [tok][pairs]
  __shared__ float2 slot[kWarps];
  __shared__ float exchange[WHOLE ? 1 : kWarps * 32 * E];
  const int warp = threadIdx.x >> 5;
  float* buf = WHOLE ? exchange : exchange + warp * 32 * E;
  const int V = p.d / E, nvec = p.heads * V, tpr = 32 * p.wpr, groups = kWarps / p.wpr;
  const int group = warp / p.wpr, l = threadIdx.x - group * tpr, c0 = (l % V) * E;
  const int vshift = 31 - __clz(V);
  const long long tokens = (long long)p.B * p.S, first = (long long)blockIdx.x * p.tok;
  const int count = (int)min((long long)p.tok, tokens - first);
  angles(p, first, count, ang);
  __syncthreads();
  const int rows = count * p.n, trips = (rows + groups - 1) / groups;
  for (int trip = 0; trip < trips; ++trip) {
    const int row = trip * groups + group;
    const bool ok = row < rows;
    // tensors from the last to the first, a token's rows behind one another: what the caller reads next comes last
    const int tk = ok ? row / p.n : 0, k = ok ? p.n - 1 - (row - tk * p.n) : 0;
    const long long g = first + tk;
    const int b = (int)(g / p.S), tok = (int)(g - (long long)b * p.S);
    const Tensor& t = p.t[k];
    const RowAt from = row_at(p, false, t.ss, b, tok), to = row_at(p, p.dst_bm, t.ds, b, tok);
    const T* src = reinterpret_cast<const T*>(t.src) + from.base + c0;
    T* dst = reinterpret_cast<T*>(t.dst) + to.base + c0;
    const bool turned = k < p.turned;
    if (p.perm && ok && k == 0 && b == 0 && l == 0) p.perm[block_pos(p, tok)] = tok;
    Turn<E> turn;
    turn.load(p, ang + tk * p.pairs, turned ? c0 : p.d, 1.f);
    uint4 raw[NV];
    auto load = [&](int v0) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int v = v0 + l + i * tpr;
        raw[i] = make_uint4(0u, 0u, 0u, 0u);
        if (ok && v < nvec) raw[i] = __ldcs(reinterpret_cast<const uint4*>(src + (long long)(v >> vshift) * from.head));
      }
    };
    const int per = NV * tpr;                // vectors of a trip through the row
    float r_row = 1.f;
    if (p.norm == VMOBA_ROTARY_NORM_ROW) {
      float2 sum = make_float2(0.f, 0.f);
      for (int v0 = 0; v0 < nvec; v0 += per) {
        load(v0);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          float x[E];
          Vec<T>::unpack(raw[i], x);
#pragma unroll
          for (int e = 0; e < E; ++e) sum.x = fmaf(x[e], x[e], sum.x);
        }
      }
      r_row = rsqrtf(row_sum(sum, p.wpr, slot).x / (float)(p.heads * p.d) + p.eps);
    }
    for (int v0 = 0; v0 < nvec; v0 += per) {
      if (p.norm != VMOBA_ROTARY_NORM_ROW || nvec > per) load(v0);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int v = v0 + l + i * tpr;
        if (v0 + (warp % p.wpr) * 32 + i * tpr >= nvec) break;      // (whole warps)
        const bool there = ok && v < nvec;
        float y[E];
        Vec<T>::unpack(raw[i], y);
        if (turned) {
          if (p.norm != VMOBA_ROTARY_NORM_NONE) {
            float r = r_row, w[E];
            if (p.norm == VMOBA_ROTARY_NORM_HEAD) {
              float2 sum = make_float2(0.f, 0.f);
#pragma unroll
              for (int e = 0; e < E; ++e) sum.x = fmaf(y[e], y[e], sum.x);
              r = rsqrtf(head_sum(sum, V).x / (float)p.d + p.eps);
              weights<E>(t.w ? t.w + c0 : nullptr, w);
            } else {
              weights<E>(t.w ? t.w + min(v, nvec - 1) * E : nullptr, w);
            }
#pragma unroll
            for (int e = 0; e < E; ++e) y[e] = y[e] * r * w[e];
          }
          if (p.pairs > 0) {
            float o[E];
            partners<E, WHOLE>(p, y, o, c0, turn.mine, buf);
#pragma unroll
            for (int e = 0; e < E; ++e)
              if (turn.mine >> e & 1) y[e] = fmaf(y[e], turn.cs[e], o[e] * turn.sn[e]);
          }
        }
        if (there) *reinterpret_cast<uint4*>(dst + (long long)(v >> vshift) * to.head) = Vec<T>::pack(y);
      }
    }
  }
}

// ------------------------------------------------------------------------------ backward
// blockIdx.y: tensor.  A CTA walks its share of the tokens and keeps its part of dw: norm over the row, in shared memory, a copy for
// each group of warps that takes a row (a thread owns its channels there); norm per head, in registers.  The parts are added up
// in a fixed order by weight_sum_kernel: the results repeat bit for bit.
template <typename T, bool WHOLE>
__global__ void __launch_bounds__(kThreads)
rotary_bwd_kernel(const __grid_constant__ Params p) {
  if (!grid_begin()) return;
  constexpr int E = Vec<T>::E;
  extern __shared__ __align__(16) uint8_t smem[];
  float2* ang = reinterpret_cast<float2*>(smem);                                  // [tok][pairs]
  float* acc_row = reinterpret_cast<float*>(smem + ang_bytes(p.tok, p.pairs));    // [group][heads * d]
  __shared__ float2 slot[kWarps];
  __shared__ float exchange[kWarps * 32 * E];
  const int warp = threadIdx.x >> 5;
  float* buf = exchange + warp * 32 * E;
  const int V = p.d / E, nvec = p.heads * V, tpr = 32 * p.wpr, groups = kWarps / p.wpr;
  const int group = warp / p.wpr, l = threadIdx.x - group * tpr, c0 = (l % V) * E;
  const int vshift = 31 - __clz(V);
  const Tensor& t = p.t[blockIdx.y];
  const long long tokens = (long long)p.B * p.S;
  const bool by_row = p.norm == VMOBA_ROTARY_NORM_ROW, by_head = p.norm == VMOBA_ROTARY_NORM_HEAD, normed = by_row || by_head;
  const int row_ch = p.heads * p.d;
  float acc[E];
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.f;
  if (by_row)
    for (int i = threadIdx.x; i < groups * row_ch; i += kThreads) acc_row[i] = 0.f;
  float* mine_acc = acc_row + (long long)group * row_ch;
  for (long long first = (long long)blockIdx.x * p.tok; first < tokens; first += (long long)gridDim.x * p.tok) {
    const int count = (int)min((long long)p.tok, tokens - first);
    __syncthreads();
    angles(p, first, count, ang);
    __syncthreads();
    const int trips = (count + groups - 1) / groups;
    for (int trip = 0; trip < trips; ++trip) {
      const int tk = trip * groups + group;
      const bool ok = tk < count;
      const long long g = first + (ok ? tk : 0);
      const int b = (int)(g / p.S), tok = (int)(g - (long long)b * p.S);
      const RowAt from = row_at(p, p.src_bm, t.ss, b, tok), at_x = row_at(p, false, t.xs, b, tok), to = row_at(p, false, t.ds, b, tok);
      const T* src = reinterpret_cast<const T*>(t.src) + from.base + c0;
      const T* xr = normed ? reinterpret_cast<const T*>(t.x) + at_x.base + c0 : nullptr;
      T* dst = reinterpret_cast<T*>(t.dst) + to.base + c0;
      Turn<E> turn;
      turn.load(p, ang + (ok ? tk : 0) * p.pairs, c0, -1.f);
      uint4 raw[NV], rawx[NV];
      auto load = [&](int v0) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const int v = v0 + l + i * tpr;
          raw[i] = rawx[i] = make_uint4(0u, 0u, 0u, 0u);
          if (ok && v < nvec) {
            raw[i] = __ldcs(reinterpret_cast<const uint4*>(src + (long long)(v >> vshift) * from.head));
            if (normed) rawx[i] = __ldcs(reinterpret_cast<const uint4*>(xr + (long long)(v >> vshift) * at_x.head));
          }
        }
      };
      auto turned_back = [&](const uint4& u, float (&y)[E]) {
        Vec<T>::unpack(u, y);
        if (p.pairs > 0) {
          float o[E];
          partners<E, WHOLE>(p, y, o, c0, turn.mine, buf);
#pragma unroll
          for (int e = 0; e < E; ++e)
            if (turn.mine >> e & 1) y[e] = fmaf(y[e], turn.cs[e], o[e] * turn.sn[e]);
        }
      };
      const int per = NV * tpr;
      const float2 zero = make_float2(0.f, 0.f);
      float2 sums = zero;                    // sum of squares of x, of x times its weighted gradient
      if (by_row) {
        for (int v0 = 0; v0 < nvec; v0 += per) {
          load(v0);
#pragma unroll
          for (int i = 0; i < NV; ++i) {
            if (v0 + (warp % p.wpr) * 32 + i * tpr >= nvec) break;
            const int v = v0 + l + i * tpr;
            float y[E], x[E], w[E];
            turned_back(raw[i], y);
            Vec<T>::unpack(rawx[i], x);
            weights<E>(t.w ? t.w + min(v, nvec - 1) * E : nullptr, w);
#pragma unroll
            for (int e = 0; e < E; ++e) {
              sums.x = fmaf(x[e], x[e], sums.x);
              sums.y = fmaf(x[e], y[e] * w[e], sums.y);
            }
          }
        }
        sums = row_sum(sums, p.wpr, slot);
      }
      for (int v0 = 0; v0 < nvec; v0 += per) {
        if (!by_row || nvec > per) load(v0);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          if (v0 + (warp % p.wpr) * 32 + i * tpr >= nvec) break;
          const int v = v0 + l + i * tpr;
          const bool there = ok && v < nvec;
          float y[E];
          turned_back(raw[i], y);
          if (normed) {
            float x[E], w[E];
            Vec<T>::unpack(rawx[i], x);
            weights<E>(!t.w ? nullptr : by_row ? t.w + min(v, nvec - 1) * E : t.w + c0, w);
            float2 s = sums;
            if (by_head) {
              s = zero;
#pragma unroll
              for (int e = 0; e < E; ++e) {
                s.x = fmaf(x[e], x[e], s.x);
                s.y = fmaf(x[e], y[e] * w[e], s.y);
              }
              s = head_sum(s, V);
            }
            const float n = (float)(by_row ? row_ch : p.d), r = rsqrtf(s.x / n + p.eps), back = r * r * (s.y / n);
            float dw[E];
#pragma unroll
            for (int e = 0; e < E; ++e) {
              dw[e] = y[e] * (x[e] * r);
              y[e] = r * fmaf(-x[e], back, y[e] * w[e]);
            }
            if (by_head) {
#pragma unroll
              for (int e = 0; e < E; ++e) acc[e] += there ? dw[e] : 0.f;
            } else if (there) {
#pragma unroll
              for (int e = 0; e < E; e += 4) {
                float4* a = reinterpret_cast<float4*>(mine_acc + v * E + e);
                float4 z = *a;
                z.x += dw[e]; z.y += dw[e + 1]; z.z += dw[e + 2]; z.w += dw[e + 3];
                *a = z;
              }
            }
          }
          if (there) *reinterpret_cast<uint4*>(dst + (long long)(v >> vshift) * to.head) = Vec<T>::pack(y);
        }
      }
    }
  }
  if (!normed) return;
  __syncthreads();
  const int n_w = by_row ? row_ch : p.d;
  float* out = p.part + ((long long)blockIdx.y * gridDim.x + blockIdx.x) * n_w;
  if (by_row) {
    for (int i = threadIdx.x; i < row_ch; i += kThreads) {
      float a = 0.f;
      for (int q = 0; q < groups; ++q) a += acc_row[(long long)q * row_ch + i];
      out[i] = a;
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) exchange[threadIdx.x * E + e] = acc[e];
    __syncthreads();
    for (int c = threadIdx.x; c < p.d; c += kThreads) {      // threads c / E, c / E + V, ... hold channel c
      float a = 0.f;
      for (int q = c / E; q < kThreads; q += V) a += exchange[q * E + c % E];
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
static int bwd_ctas(const Dims& D, int tok) {
  return (int)std::min<long long>(((long long)D.B * D.S + tok - 1) / tok, 2ll * sm_count());
}
static int tokens_per_cta(const Dims& D) {
  // as many as share their angles without leaving SMs short of work
  const long long per = (long long)D.B * D.S / ((long long)sm_count() * 8);
  int tok = 1;
  while (tok < kMaxTok && tok * 2 <= per) tok *= 2;
  return tok;
}
static int warps_per_row(const Dims& D) {
  const int nvec = D.heads * D.d * D.es / 16;
  int w = 1;
  while (w < kWarps && nvec > NV * 32 * w) w *= 2;
  return w;
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
  p->T = D.T; p->H = D.H; p->W = D.W; p->bT = D.bT; p->bH = D.bH; p->bW = D.bW; p->nH = D.nH; p->nW = D.nW;
  p->pairs = spec->pairs; p->axes = spec->axes; p->layout = spec->layout; p->norm = spec->norm; p->pos_batch = spec->pos_batch;
  p->mscale = spec->mscale; p->eps = spec->eps;
  p->wpr = warps_per_row(D);
  p->tok = tokens_per_cta(D);
}

static size_t bwd_smem(const Dims& D, const Params& p) {
  return ang_bytes(p.tok, p.pairs) +
         (p.norm == VMOBA_ROTARY_NORM_ROW ? (size_t)(kWarps / p.wpr) * D.heads * D.d * sizeof(float) : 0);
}
constexpr int kFwdSmem = kMaxTok * 64 * (int)sizeof(float2);

template <typename T>
static int launch_fwd(const Dims& D, const Params& p, cudaStream_t st) {
  const bool whole = p.layout == VMOBA_ROTARY_INTERLEAVED || p.pairs % Vec<T>::E == 0;
  const long long grid = ((long long)D.B * D.S + p.tok - 1) / p.tok;
  auto kernel = whole ? rotary_fwd_kernel<T, true> : rotary_fwd_kernel<T, false>;
  launch_kernel(early_rows(D), kernel, (unsigned)grid, kThreads, kFwdSmem, st, p);
  VMOBA_LAUNCH_OK(1);
  return VMOBA_OK;
}

template <typename T>
static int launch_bwd(const Dims& D, const Params& p, const WeightOut& w, cudaStream_t st) {
  const bool whole = p.layout == VMOBA_ROTARY_INTERLEAVED || p.pairs % Vec<T>::E == 0;
  const int ctas = bwd_ctas(D, p.tok);
  auto kernel = whole ? rotary_bwd_kernel<T, true> : rotary_bwd_kernel<T, false>;
  VMOBA_CUDA_OK(allow_smem(kernel, 200 * 1024));
  launch_kernel(early_rows(D), kernel, dim3(ctas, p.n), kThreads, bwd_smem(D, p), st, p);
  VMOBA_LAUNCH_OK(1);
  if (p.norm != VMOBA_ROTARY_NORM_NONE) {
    const int n_w = p.norm == VMOBA_ROTARY_NORM_ROW ? D.heads * D.d : D.d;
    launch_kernel(weight_sum_kernel, dim3((n_w + 31) / 32, p.n), 1024, 0, st, p.part, ctas, n_w, w);
    VMOBA_LAUNCH_OK(1);
  }
  return VMOBA_OK;
}

}  // namespace rotary
}  // namespace vmoba

using namespace vmoba;

extern "C" size_t vmoba_rotary_workspace_bytes(const vmoba_shape* shape, const vmoba_rotary_spec* spec, int32_t n) {
  Dims D;
  if (rotary::check(shape, spec, &D) || n < 1 || n > rotary::kMaxTensors) return 0;
  if (spec->norm == VMOBA_ROTARY_NORM_NONE) return 256;
  Carver c(nullptr);
  // (for as many CTAs as any device of 256 SMs runs: the size is a function of the shape alone)
  c.take<float>((size_t)n * std::min<long long>((long long)D.B * D.S, 512) * (spec->norm == VMOBA_ROTARY_NORM_ROW ? D.heads * D.d : D.d));
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
  if (rotary::bwd_smem(D, p) > 200 * 1024) return VMOBA_ERR_NOT_IMPLEMENTED;
  p.part = static_cast<float*>(ws);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return D.dtype == VMOBA_BF16 ? rotary::launch_bwd<__nv_bfloat16>(D, p, w, st) : rotary::launch_bwd<float>(D, p, w, st);
}
