// Matrix products of a transformer block with what stands behind them, shared by the kernels that compute them.
//   forward    out = residual + gate * act(x W^T + b), or act(x Wg^T + bg) * (x Wu^T + bu) in place of act(..)
//   backward   dx = du W,  dW = du^T x
// A product is one of three forms by where its summed index lies: kRowsRows  D[r][n] = sum_c A[r][c] B[n][c],
// kRowsCols  D[r][k] = sum_n A[r][n] B[n][k],  kColsCols  D[n][k] = sum_r A[r][n] B[r][k].
#pragma once

#include <type_traits>

#include "common.cuh"
#include "sm100.cuh"

namespace vmoba {
namespace linear {

enum Form { kRowsRows = 0, kRowsCols = 1, kColsCols = 2 };
// What becomes of sums: written; a layer's forward; that of a gated layer; the gradient of a layer's product from that of its output (kSlope,
// gated: kSlopeGated), together with the output itself.
enum Kind { kPlain = 0, kForward = 1, kGated = 2, kSlope = 3, kSlopeGated = 4 };

// A matrix in memory whose row r is token s of sample b, r = b * S + s; column c lies at (c / inner) * sh + c % inner of its row (inner: the
// channels of a head where heads are apart, else all columns).  Element strides.
struct Matrix {
  const void* p = nullptr;
  int B = 1, S = 1, cols = 0, inner = 0;
  long long sb = 0, st = 0, sh = 0;
};
inline Matrix dense(const void* p, int rows, int cols) { return Matrix{p, 1, rows, cols, cols, 0, cols, 0}; }

// What becomes of a sum.
struct Epilogue {
  int kind = kPlain, act = VMOBA_ACT_NONE;
  int cols = 0;                              // of out: of the sums, or half as many (kGated: gate and factor of column c are c and cols + c)
  int S = 1, inner = 0;
  FastDiv by_S, by_inner, by_gate;
  void* out = nullptr;
  long long ob = 0, ot = 0, oh = 0;
  const void* bias = nullptr;                // of the layer's type
  const float* gate = nullptr;
  long long gb = 0, gg = 0;
  const void* residual = nullptr;
  long long rb = 0, rt = 0;
  void* kept = nullptr;                      // sums with bias, ahead of the activation, dense in the order of x
  const int* perm = nullptr;                 // token of out for every token of x
  // kSlope*: out is dense [rows, cols or 2 cols], kept is read
  void* again = nullptr;                     // the layer's output, dense [rows, cols]
  float* col_sums = nullptr;                 // [rows / 32][cols or 2 cols]: sums of out by 32 rows
};
inline bool is_gated(int kind) { return kind == kGated || kind == kSlopeGated; }
inline void set_out(Epilogue* e, const Matrix& m) {
  e->S = m.S; e->by_S = FastDiv((unsigned)m.S);
  e->inner = m.inner; e->by_inner = FastDiv((unsigned)m.inner);
  e->out = const_cast<void*>(m.p); e->ob = m.sb; e->ot = m.st; e->oh = m.sh;
  e->cols = m.cols;
}

struct Product {
  Form form;
  Matrix a, b;
  Epilogue e;
  int M, N;                                  // of D; the summed index has a.cols (kRows*) or the rows of a
  int planes;                                // 2: a is the sum of two matrices, the second `plane` elements behind the first
  long long plane;
  bool bf16;
  int32_t* status;
};

// Scratch of a product (partial sums of slices of the summed index) and the product itself.
size_t product_scratch(const Product& p);
int run_product(const Product& p, float* scratch, cudaStream_t st);

// fp32 (linear_simt.cu), bf16 (linear_tc.cu), and of those the products of a few tokens with a weight (linear_few.cu).
size_t simt_scratch(const Product& p);
int simt_product(const Product& p, float* scratch, cudaStream_t st);
size_t tc_scratch(const Product& p);
int tc_product(const Product& p, float* scratch, cudaStream_t st);
bool few_takes(const Product& p);
int few_product(const Product& p, cudaStream_t st);

#ifdef __CUDACC__
// gelu in its tanh form, u s(2 k (u + c u^3)), and silu, u s(u), of the logistic function s = 1 / (1 + exp(-x)), whose exp overflows for very
// negative x, where s is zero, as it should be.  EXACT: to fp32's last places; else to 2^-20 or so, for results of 8 bits.
constexpr float kGeluK = 1.5957691216057308f, kGeluC = 0.044715f;      // 2 sqrt(2 / pi)
template <bool EXACT>
__device__ __forceinline__ float logistic(float x) {
  if constexpr (EXACT) {
    return 1.f / (1.f + expf(-x));
  } else {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + sm100::ex2(-1.4426950408889634f * x)));
    return r;
  }
}
template <bool EXACT, int ACT>
__device__ __forceinline__ float activate(float u) {
  if constexpr (ACT == VMOBA_ACT_NONE) return u;
  return u * logistic<EXACT>(ACT == VMOBA_ACT_SILU ? u : kGeluK * u * fmaf(kGeluC * u, u, 1.f));
}
// The activation and its slope, s + u s (1 - s) z' with z the argument of s.  (Far out s (1 - s) is zero and z' may be infinite: it is held below that.)
template <bool EXACT, int ACT>
__device__ __forceinline__ float2 activate_slope(float u) {
  if constexpr (ACT == VMOBA_ACT_NONE) return make_float2(u, 1.f);
  const float q = kGeluC * u * u, s = logistic<EXACT>(ACT == VMOBA_ACT_SILU ? u : kGeluK * u * (q + 1.f)), y = u * s, t = y * (1.f - s);
  if constexpr (ACT == VMOBA_ACT_SILU) return make_float2(y, s + t);
  return make_float2(y, fmaf(t, fminf(fmaf(3.f * kGeluK, q, kGeluK), 1e30f), s));
}
// f(activation), compiled for each.
template <typename F>
__device__ __forceinline__ void by_activation(int act, F f) {
  if (act == VMOBA_ACT_SILU) f(std::integral_constant<int, VMOBA_ACT_SILU>{});
  else if (act == VMOBA_ACT_GELU) f(std::integral_constant<int, VMOBA_ACT_GELU>{});
  else f(std::integral_constant<int, VMOBA_ACT_NONE>{});
}

template <int V>
__device__ __forceinline__ void load_vec(const float* p, float (&x)[V]) {
#pragma unroll
  for (int i = 0; i < V; i += 4) { const float4 v = load4(p + i); x[i] = v.x; x[i + 1] = v.y; x[i + 2] = v.z; x[i + 3] = v.w; }
}
// (of what no kernel of the call writes: these may move ahead of stores)
template <int V>
__device__ __forceinline__ void load_const(const float* p, float (&x)[V]) {
#pragma unroll
  for (int i = 0; i < V; i += 4) {
    const float4 v = __ldg(reinterpret_cast<const float4*>(p + i));
    x[i] = v.x; x[i + 1] = v.y; x[i + 2] = v.z; x[i + 3] = v.w;
  }
}
template <int V>
__device__ __forceinline__ void load_vec(const __nv_bfloat16* p, float (&x)[V]) {
  if constexpr (V == 8) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    const uint32_t v[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(v[i] << 16); x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u); }
  } else {
    const float4 v = load4(p);
    x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
  }
}
template <int V>
__device__ __forceinline__ void store_vec(float* p, const float (&x)[V]) {
#pragma unroll
  for (int i = 0; i < V; i += 4) store4(p + i, make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]));
}
template <int V>
__device__ __forceinline__ void store_vec(__nv_bfloat16* p, const float (&x)[V]) {
  if constexpr (V == 8) {
    uint32_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = sm100::pack_bf16(x[2 * i], x[2 * i + 1]);
    *reinterpret_cast<uint4*>(p) = make_uint4(v[0], v[1], v[2], v[3]);
  } else {
    store4(p, make_float4(x[0], x[1], x[2], x[3]));
  }
}

// A row of out: where it lies, with its residual and gate.  ok: false for a token that the permutation puts outside (its row is left out).
template <typename T>
struct OutRow {
  T* out;
  const T* residual;
  const float* gate;
  T* kept;
  bool ok;
  __device__ __forceinline__ OutRow(const Epilogue& e, int r) {
    const int b = e.by_S.div(r), s = r - b * e.S;
    int t = s;
    if (e.perm) t = __ldg(e.perm + s);
    ok = (unsigned)t < (unsigned)e.S;
    if (!ok) t = 0;
    out = static_cast<T*>(e.out) + b * e.ob + t * e.ot;
    residual = e.residual ? static_cast<const T*>(e.residual) + b * e.rb + t * e.rt : nullptr;
    gate = e.gate ? e.gate + b * e.gb + e.by_gate.div(t) * e.gg : nullptr;
    kept = e.kept ? static_cast<T*>(e.kept) + (long long)r * e.cols * (e.kind == kGated ? 2 : 1) : nullptr;
  }
};

// Columns c .. c + V - 1 (V divides every boundary) of a row of out from the sums; with kGated `v` are those of the factor.
template <typename T, int V, int KIND>
__device__ __forceinline__ void finish(const Epilogue& e, const OutRow<T>& row, int c, float (&u)[V], float (&v)[V]) {
  constexpr bool EXACT = sizeof(T) == 4;
  if constexpr (KIND != kPlain) {
    float t[V];
    if (e.bias) {
      load_vec<V>(static_cast<const T*>(e.bias) + c, t);
#pragma unroll
      for (int i = 0; i < V; ++i) u[i] += t[i];
      if constexpr (KIND == kGated) {
        load_vec<V>(static_cast<const T*>(e.bias) + e.cols + c, t);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] += t[i];
      }
    }
    if (row.kept) {
      store_vec<V>(row.kept + c, u);
      if constexpr (KIND == kGated) store_vec<V>(row.kept + e.cols + c, v);
    }
    by_activation(e.act, [&](auto act) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        u[i] = activate<EXACT, decltype(act)::value>(u[i]);
        if constexpr (KIND == kGated) u[i] *= v[i];
      }
    });
    if (row.gate) {
      load_vec<V>(row.gate + c, t);
#pragma unroll
      for (int i = 0; i < V; ++i) u[i] *= t[i];
    }
    if (row.residual) {
      load_vec<V>(row.residual + c, t);
#pragma unroll
      for (int i = 0; i < V; ++i) u[i] += t[i];
    }
  }
  if (!row.ok) return;
  const int h = e.inner == e.cols ? 0 : e.by_inner.div(c);
  store_vec<V>(row.out + h * e.oh + (c - h * e.inner), u);
}

// Sums of slices of the summed index: part[slice][row][column of the sums] (N columns, gated: twice as many).
struct Slices {
  const float* part;
  long long rows;
  int N, wide, count;
};
// ... added in order, and what becomes of them.
template <typename T, int KIND>
__global__ void __launch_bounds__(256) join_kernel(Slices p, Epilogue e, FastDiv by_vecs, int vecs, int total) {
  if (!grid_begin()) return;
  const long long slice = p.rows * p.wide;
  for (int i = blockIdx.x * 256 + threadIdx.x; i < total; i += gridDim.x * 256) {
    const int r = by_vecs.div(i), c = (i - r * vecs) * 8;
    const float* from = p.part + (long long)r * p.wide + c;
    float u[8] = {}, v[8] = {};
#pragma unroll 4
    for (int s = 0; s < p.count; ++s, from += slice) {
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
    finish<T, 8, KIND>(e, OutRow<T>(e, r), c, u, v);
  }
}
template <typename T, int KIND>
int join(const Slices& p, const Epilogue& e, cudaStream_t st) {
  const long long vecs = p.N / 8, total = p.rows * vecs;
  launch_kernel(join_kernel<T, KIND>, (unsigned)((total + 255) / 256 < 16 * sm_count() ? (total + 255) / 256 : 16 * sm_count()), 256, 0, st, p, e,
                FastDiv((unsigned)vecs), (int)vecs, (int)total);
  VMOBA_LAUNCH_OK(1);
  return VMOBA_OK;
}
#endif

}  // namespace linear
}  // namespace vmoba
