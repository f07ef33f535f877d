// Matrix products on the CUDA cores, in fp32: the operators' fp32 form.
// D tiles of 128 x 128 or 64 x 64 by CTAs of as many threads as there are 8 x 8 (4 x 4) pieces, 16 summed indices at a time through shared
// memory, the next 16 on their way in registers.  Where tiles are few the summed index is cut into slices, whose sums a second kernel adds in a
// fixed order.
#include <algorithm>

#include "linear.cuh"

namespace vmoba {
namespace linear {
namespace {

constexpr int BK = 16;

// Element (row r, column c) of a matrix, four columns at a time; zeros outside.
template <typename T>
__device__ __forceinline__ float4 fetch4(const Matrix& m, const FastDiv& by_S, const FastDiv& by_inner, int rows, int r, int c) {
  if (r >= rows || c >= m.cols) return make_float4(0.f, 0.f, 0.f, 0.f);
  const int b = m.B == 1 ? 0 : by_S.div(r), s = r - b * m.S;
  const int h = m.inner == m.cols ? 0 : by_inner.div(c);
  return load4(static_cast<const T*>(m.p) + b * m.sb + s * m.st + h * m.sh + (c - h * m.inner));
}

struct Args {
  Matrix a, b;
  FastDiv a_S, a_inner, b_S, b_inner;
  int a_rows, b_rows, M, N, K;
  int per, slices;                           // summed indices of a slice
  float* part;                               // [slice][row][column of the sums]
  Epilogue e;
};

// Threads THREADS, tile TM x TN, pieces of P x P: rows ty * P + .., columns tx * 4 + j * (TN / (P / 4)) + ..
template <typename T, int FORM, int KIND, int TILE, int P>
__global__ void __launch_bounds__((TILE / P) * (TILE / P)) product_kernel(Args p) {
  if (!grid_begin()) return;
  constexpr int THREADS = (TILE / P) * (TILE / P), SIDE = TILE / P, GROUPS = P / 4;
  constexpr bool TWO = KIND == kGated;
  constexpr int NB = TWO ? 2 : 1;
  constexpr int LOADS = TILE * BK / 4 / THREADS;
  __shared__ float sA[BK][TILE + 4];
  __shared__ float sB[NB][BK][TILE + 4];
  const int t = threadIdx.x, tx = t % SIDE, ty = t / SIDE;
  const int m0 = blockIdx.x * TILE, n0 = blockIdx.y * TILE;
  float acc[NB][P][P];
#pragma unroll
  for (int w = 0; w < NB; ++w)
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
      for (int j = 0; j < P; ++j) acc[w][i][j] = 0.f;
  float4 ra[LOADS], rb[NB][LOADS];
  // an operand's rows run along the tile (rows4: four summed indices of a row) or along the summed index (four places of the tile)
  constexpr bool A_ROWS = FORM != kColsCols, B_ROWS = FORM == kRowsRows;
  auto load = [&](int k0) {
#pragma unroll
    for (int l = 0; l < LOADS; ++l) {
      const int i = t + l * THREADS;
      if (A_ROWS) ra[l] = fetch4<T>(p.a, p.a_S, p.a_inner, p.a_rows, m0 + i / (BK / 4), k0 + i % (BK / 4) * 4);
      else ra[l] = fetch4<T>(p.a, p.a_S, p.a_inner, p.a_rows, k0 + i / (TILE / 4), m0 + i % (TILE / 4) * 4);
#pragma unroll
      for (int w = 0; w < NB; ++w) {
        if (B_ROWS) {
          const int n = n0 + i / (BK / 4);      // (the factor's rows of the weight follow the gate's)
          rb[w][l] = fetch4<T>(p.b, p.b_S, p.b_inner, w ? 2 * p.N : p.N, n < p.N ? n + w * p.N : 2 * p.N, k0 + i % (BK / 4) * 4);
        } else {
          rb[w][l] = fetch4<T>(p.b, p.b_S, p.b_inner, p.b_rows, k0 + i / (TILE / 4), n0 + i % (TILE / 4) * 4);
        }
      }
    }
  };
  auto put = [&](float (*s)[TILE + 4], bool rows, int i, float4 v) {
    if (rows) {
      const int r = i / (BK / 4), k = i % (BK / 4) * 4;
      s[k][r] = v.x; s[k + 1][r] = v.y; s[k + 2][r] = v.z; s[k + 3][r] = v.w;
    } else {
      *reinterpret_cast<float4*>(&s[i / (TILE / 4)][i % (TILE / 4) * 4]) = v;
    }
  };
  const int k_first = blockIdx.z * p.per, k_end = min(k_first + p.per, p.K);      // (per is a multiple of BK: nobody reads beyond a slice)
  load(k_first);
  for (int k0 = k_first; k0 < k_end; k0 += BK) {
    __syncthreads();
#pragma unroll
    for (int l = 0; l < LOADS; ++l) {
      put(sA, A_ROWS, t + l * THREADS, ra[l]);
#pragma unroll
      for (int w = 0; w < NB; ++w) put(sB[w], B_ROWS, t + l * THREADS, rb[w][l]);
    }
    __syncthreads();
    if (k0 + BK < k_end) load(k0 + BK);
#pragma unroll
    for (int k = 0; k < BK; ++k) {
      float a[P];
      load_vec<P>(&sA[k][ty * P], a);
#pragma unroll
      for (int w = 0; w < NB; ++w)
#pragma unroll
        for (int j = 0; j < GROUPS; ++j) {
          const float4 b = load4(&sB[w][k][tx * 4 + j * (TILE / GROUPS)]);
#pragma unroll
          for (int i = 0; i < P; ++i) {
            float (&c)[P] = acc[w][i];
            sm100::fma2(c[4 * j], c[4 * j + 1], a[i], a[i], b.x, b.y, c[4 * j], c[4 * j + 1]);
            sm100::fma2(c[4 * j + 2], c[4 * j + 3], a[i], a[i], b.z, b.w, c[4 * j + 2], c[4 * j + 3]);
          }
        }
    }
  }
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int r = m0 + ty * P + i;
    if (r >= p.M) break;
    if (p.part) {
      const int wide = TWO ? 2 * p.N : p.N;
      float* to = p.part + ((long long)blockIdx.z * p.M + r) * wide;
#pragma unroll
      for (int j = 0; j < GROUPS; ++j) {
        const int c = n0 + tx * 4 + j * (TILE / GROUPS);
        if (c >= p.N) continue;
#pragma unroll
        for (int w = 0; w < NB; ++w) store4(to + w * p.N + c, make_float4(acc[w][i][4 * j], acc[w][i][4 * j + 1], acc[w][i][4 * j + 2], acc[w][i][4 * j + 3]));
      }
      continue;
    }
    const OutRow<T> row(p.e, r);
#pragma unroll
    for (int j = 0; j < GROUPS; ++j) {
      const int c = n0 + tx * 4 + j * (TILE / GROUPS);
      if (c >= p.N) continue;
      float u[4], v[4] = {};
#pragma unroll
      for (int q = 0; q < 4; ++q) { u[q] = acc[0][i][4 * j + q]; if (TWO) v[q] = acc[NB - 1][i][4 * j + q]; }
      finish<T, 4, KIND>(p.e, row, c, u, v);
    }
  }
}

template <typename T, int FORM, int KIND, int TILE, int P>
int launch(const Args& a, cudaStream_t st) {
  launch_kernel(product_kernel<T, FORM, KIND, TILE, P>, dim3((unsigned)((a.M + TILE - 1) / TILE), (unsigned)((a.N + TILE - 1) / TILE), (unsigned)a.slices),
                (TILE / P) * (TILE / P), 0, st, a);
  VMOBA_LAUNCH_OK(1);
  return a.part ? join<T, KIND>(Slices{a.part, a.M, a.N, KIND == kGated ? 2 * a.N : a.N, a.slices}, a.e, st) : VMOBA_OK;
}

// Whether tiles are 128 x 128 (where that gives every SM one), and slices: up to four CTAs of the small tiles an SM, of 128 summed indices at least.
struct Cut { bool large; int per, slices; };
Cut cut_of(const Product& p) {
  constexpr int kSms = 148;                  // (a workspace's size goes by the shape alone)
  Cut c;
  const long long K = p.form == kColsCols ? (long long)p.a.B * p.a.S : p.a.cols;
  c.large = p.e.kind != kGated && (long long)((p.M + 127) / 128) * ((p.N + 127) / 128) >= kSms;
  const long long tiles = (long long)((p.M + 63) / 64) * ((p.N + 63) / 64);
  long long n = c.large ? 1 : std::max<long long>(1, std::min<long long>(4 * kSms / tiles, K / 128));
  c.per = (int)((K + n - 1) / n + BK - 1) / BK * BK;
  c.slices = (int)((K + c.per - 1) / c.per);
  return c;
}

int by_form(const Product& p, const Args& a, bool large, cudaStream_t st) {
  using T = float;
  if (p.form == kColsCols) return large ? launch<T, kColsCols, kPlain, 128, 8>(a, st) : launch<T, kColsCols, kPlain, 64, 4>(a, st);
  if (p.form == kRowsCols) return large ? launch<T, kRowsCols, kPlain, 128, 8>(a, st) : launch<T, kRowsCols, kPlain, 64, 4>(a, st);
  if (p.e.kind == kGated) return launch<T, kRowsRows, kGated, 64, 4>(a, st);
  return large ? launch<T, kRowsRows, kForward, 128, 8>(a, st) : launch<T, kRowsRows, kForward, 64, 4>(a, st);
}

}  // namespace

size_t simt_scratch(const Product& p) {
  const Cut c = cut_of(p);
  return c.slices > 1 ? (size_t)c.slices * p.M * p.N * (p.e.kind == kGated ? 2 : 1) : 0;
}

int simt_product(const Product& p, float* scratch, cudaStream_t st) {
  Args a;
  const Cut c = cut_of(p);
  a.per = c.per; a.slices = c.slices;
  a.part = c.slices > 1 ? scratch : nullptr;
  a.a = p.a; a.b = p.b; a.e = p.e; a.M = p.M; a.N = p.N;
  a.a_S = FastDiv((unsigned)p.a.S); a.a_inner = FastDiv((unsigned)p.a.inner);
  a.b_S = FastDiv((unsigned)p.b.S); a.b_inner = FastDiv((unsigned)p.b.inner);
  a.a_rows = p.a.B * p.a.S; a.b_rows = p.b.B * p.b.S;
  a.K = p.form == kColsCols ? a.a_rows : p.a.cols;
  return by_form(p, a, c.large, st);
}

}  // namespace linear
}  // namespace vmoba
