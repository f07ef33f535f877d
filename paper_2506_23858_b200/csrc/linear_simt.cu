// Matrix products on the CUDA cores, in fp32: the operators' fp32 form.
// D tiles of 128 x 128 (gated: 64 columns of either half), 128 x 32 or 64 x 64 by CTAs of as many threads as there are 8 x 8, 8 x 4 or 4 x 4
// pieces, 16 summed indices at a time through two places in shared memory, the next 16 on their way.  Where tiles are few the summed index is
// cut into slices, whose sums a second kernel adds in a fixed order.
#include <algorithm>

#include "linear.cuh"

namespace vmoba {
namespace linear {
namespace {

constexpr int BK = 16;

// Where element (row r, column c) of a matrix lies, the first of four columns; nullptr outside.  ROWS: one sample's rows of no heads (places of
// rows and columns worked out for any matrix took a sixth of the instructions).
template <typename T, bool ROWS>
__device__ __forceinline__ const T* place4(const Matrix& m, const FastDiv& by_S, const FastDiv& by_inner, int rows, int r, int c) {
  if (r >= rows || c >= m.cols) return nullptr;
  if (ROWS) return static_cast<const T*>(m.p) + r * m.st + c;
  const int b = m.B == 1 ? 0 : by_S.div(r), s = r - b * m.S;
  const int h = m.inner == m.cols ? 0 : by_inner.div(c);
  return static_cast<const T*>(m.p) + b * m.sb + s * m.st + h * m.sh + (c - h * m.inner);
}
// 16 bytes straight into shared memory; zeros where there is nothing.
__device__ __forceinline__ void bring(float* to, const float* from, const void* any) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(sm100::smem_u32(to)), "l"(from ? from : any), "r"(from ? 16 : 0) : "memory");
}

struct Args {
  Matrix a, b;
  FastDiv a_S, a_inner, b_S, b_inner;
  int a_rows, b_rows, M, N, K;
  int per, slices;                           // summed indices of a slice
  float* part;                               // [slice][row][column of the sums]
  Epilogue e;
};

// Bound by the issue of multiply-adds and what stands between them: 4,096 tokens, 2,048 channels in and out, forward 780 us (44 TFLOP/s), backward
// 1430 (48).  Two CTAs an SM, at 128 registers; operands that need no turning through registers as well 1500.
// Tiles of TM x TN (gated: TN columns of either half), a thread's piece PM x PN: rows ty * PM + .., columns tx * 4 + j * (TN / (PN / 4)) + ..
template <typename T, int FORM, int KIND, bool ROWS, int TM, int TN, int PM, int PN>
__global__ void __launch_bounds__((TM / PM) * (TN / PN), TM == 128 ? 512 / ((TM / PM) * (TN / PN)) : 0) product_kernel(Args p) {
  if (!grid_begin()) return;
  constexpr int SIDE = TN / PN, THREADS = (TM / PM) * SIDE, GROUPS = PN / 4;
  constexpr bool TWO = KIND == kGated;
  constexpr int NB = TWO ? 2 : 1;
  constexpr int LA = TM * BK / 4 / THREADS, LB = TN * BK / 4 / THREADS;
  __shared__ float sA[2][BK][TM + 4];
  __shared__ float sB[2][NB][BK][TN + 4];
  const int t = threadIdx.x, tx = t % SIDE, ty = t / SIDE;
  const int m0 = blockIdx.x * TM, n0 = blockIdx.y * TN;
  float acc[NB][PM][PN];
#pragma unroll
  for (int w = 0; w < NB; ++w)
#pragma unroll
    for (int i = 0; i < PM; ++i)
#pragma unroll
      for (int j = 0; j < PN; ++j) acc[w][i][j] = 0.f;
  // An operand's rows run along the tile (rows: four summed indices of a row, turned on their way through registers) or along the summed index
  // (four places of the tile, straight into shared memory).
  constexpr bool A_ROWS = FORM != kColsCols, B_ROWS = FORM == kRowsRows;
  float4 ra[A_ROWS ? LA : 1], rb[NB][B_ROWS ? LB : 1];
  auto load = [&](int k0, int to) {          // (the place `to` is written at once where the operand goes there directly)
#pragma unroll
    for (int l = 0; l < LA; ++l) {
      const int i = t + l * THREADS;
      if constexpr (A_ROWS) {
        const T* from = place4<T, ROWS>(p.a, p.a_S, p.a_inner, p.a_rows, m0 + i / (BK / 4), k0 + i % (BK / 4) * 4);
        ra[l] = from ? load4(from) : make_float4(0.f, 0.f, 0.f, 0.f);
      } else {
        bring(&sA[to][i / (TM / 4)][i % (TM / 4) * 4], place4<T, ROWS>(p.a, p.a_S, p.a_inner, p.a_rows, k0 + i / (TM / 4), m0 + i % (TM / 4) * 4), p.a.p);
      }
    }
#pragma unroll
    for (int l = 0; l < LB; ++l) {
      const int i = t + l * THREADS;
#pragma unroll
      for (int w = 0; w < NB; ++w) {
        if constexpr (B_ROWS) {
          const int n = n0 + i / (BK / 4);      // (the factor's rows of the weight follow the gate's)
          const T* from = place4<T, ROWS>(p.b, p.b_S, p.b_inner, w ? 2 * p.N : p.N, n < p.N ? n + w * p.N : 2 * p.N, k0 + i % (BK / 4) * 4);
          rb[w][l] = from ? load4(from) : make_float4(0.f, 0.f, 0.f, 0.f);
        } else {
          bring(&sB[to][w][i / (TN / 4)][i % (TN / 4) * 4], place4<T, ROWS>(p.b, p.b_S, p.b_inner, p.b_rows, k0 + i / (TN / 4), n0 + i % (TN / 4) * 4), p.b.p);
        }
      }
    }
  };
  auto turn = [&](auto& s, int i, float4 v) {
    const int r = i / (BK / 4), k = i % (BK / 4) * 4;
    s[k][r] = v.x; s[k + 1][r] = v.y; s[k + 2][r] = v.z; s[k + 3][r] = v.w;
  };
  const int k_first = blockIdx.z * p.per, k_end = min(k_first + p.per, p.K);      // (per is a multiple of BK: nobody reads beyond a slice)
  int at = 0;
  load(k_first, 0);
  for (int k0 = k_first; k0 < k_end; k0 += BK, at ^= 1) {
    if constexpr (A_ROWS)
#pragma unroll
      for (int l = 0; l < LA; ++l) turn(sA[at], t + l * THREADS, ra[l]);
    if constexpr (B_ROWS)
#pragma unroll
      for (int l = 0; l < LB; ++l)
#pragma unroll
        for (int w = 0; w < NB; ++w) turn(sB[at][w], t + l * THREADS, rb[w][l]);
    if constexpr (!A_ROWS || !B_ROWS) asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();                         // (and the place written next was read ahead of this)
    if (k0 + BK < k_end) load(k0 + BK, at ^ 1);
#pragma unroll
    for (int k = 0; k < BK; ++k) {
      float a[PM];
      load_vec<PM>(&sA[at][k][ty * PM], a);
#pragma unroll
      for (int w = 0; w < NB; ++w)
#pragma unroll
        for (int j = 0; j < GROUPS; ++j) {
          const float4 b = load4(&sB[at][w][k][tx * 4 + j * (TN / GROUPS)]);
#pragma unroll
          for (int i = 0; i < PM; ++i) {
            float (&c)[PN] = acc[w][i];
            sm100::fma2(c[4 * j], c[4 * j + 1], a[i], a[i], b.x, b.y, c[4 * j], c[4 * j + 1]);
            sm100::fma2(c[4 * j + 2], c[4 * j + 3], a[i], a[i], b.z, b.w, c[4 * j + 2], c[4 * j + 3]);
          }
        }
    }
  }
#pragma unroll
  for (int i = 0; i < PM; ++i) {
    const int r = m0 + ty * PM + i;
    if (r >= p.M) break;
    if (p.part) {
      const int wide = TWO ? 2 * p.N : p.N;
      float* to = p.part + ((long long)blockIdx.z * p.M + r) * wide;
#pragma unroll
      for (int j = 0; j < GROUPS; ++j) {
        const int c = n0 + tx * 4 + j * (TN / GROUPS);
        if (c >= p.N) continue;
#pragma unroll
        for (int w = 0; w < NB; ++w) store4(to + w * p.N + c, make_float4(acc[w][i][4 * j], acc[w][i][4 * j + 1], acc[w][i][4 * j + 2], acc[w][i][4 * j + 3]));
      }
      continue;
    }
    const OutRow<T> row(p.e, r);
#pragma unroll
    for (int j = 0; j < GROUPS; ++j) {
      const int c = n0 + tx * 4 + j * (TN / GROUPS);
      if (c >= p.N) continue;
      float u[4], v[4] = {};
#pragma unroll
      for (int q = 0; q < 4; ++q) { u[q] = acc[0][i][4 * j + q]; if (TWO) v[q] = acc[NB - 1][i][4 * j + q]; }
      finish<T, 4, KIND>(p.e, row, c, u, v);
    }
  }
}

template <int FORM, int KIND, int TM, int TN, int PM, int PN>
int launch(const Args& a, cudaStream_t st) {
  auto rows = [](const Matrix& m) { return m.B == 1 && m.inner == m.cols; };
  auto kernel = product_kernel<float, FORM, KIND, false, TM, TN, PM, PN>;
  if constexpr (FORM != kRowsRows)
    if (rows(a.a) && rows(a.b)) kernel = product_kernel<float, FORM, KIND, true, TM, TN, PM, PN>;
  launch_kernel(kernel, dim3((unsigned)((a.M + TM - 1) / TM), (unsigned)((a.N + TN - 1) / TN), (unsigned)a.slices),
                (TM / PM) * (TN / PN), 0, st, a);
  VMOBA_LAUNCH_OK(1);
  return a.part ? join<float, KIND>(Slices{a.part, a.M, a.N, KIND == kGated ? 2 * a.N : a.N, a.slices}, a.e, st) : VMOBA_OK;
}

// Tiles: of few columns for products that have no more; wide ones where those, cut into slices of 256 summed indices at least for two CTAs an
// SM, give every SM one and leave little of a tile empty (232 tokens, 3,248 -> 6,960 channels, the product of the input's gradient); small ones otherwise, in slices of 128
// for up to four CTAs an SM.
enum Tile { kWide, kNarrow, kSmall };
struct Cut { Tile tile; int per, slices; };
Cut cut_of(const Product& p) {
  constexpr int kSms = 148;                  // (a workspace's size goes by the shape alone)
  Cut c;
  const bool two = p.e.kind == kGated;
  const long long K = p.form == kColsCols ? (long long)p.a.B * p.a.S : p.a.cols;
  auto tiles = [&](int rows, int cols) { return (long long)((p.M + rows - 1) / rows) * ((p.N + cols - 1) / cols); };
  const int cols = two ? 64 : 128;
  const long long wide = tiles(128, cols), small = tiles(64, 64), cuts = std::max<long long>(1, std::min<long long>(2 * kSms / wide, K / 256));
  c.tile = p.N <= 32 && !two && p.M >= 128 ? kNarrow : wide * cuts >= kSms && wide * 2 * (cols / 64) * 4 <= small * 5 ? kWide : kSmall;
  const long long of = c.tile == kNarrow ? tiles(128, 32) : small;
  const long long n = c.tile == kWide ? cuts : std::max<long long>(1, std::min<long long>(4 * kSms / of, K / 128));
  c.per = (int)((K + n - 1) / n + BK - 1) / BK * BK;
  c.slices = (int)((K + c.per - 1) / c.per);
  return c;
}

template <int FORM, int KIND>
int by_tile(const Args& a, Tile tile, cudaStream_t st) {
  constexpr bool TWO = KIND == kGated;
  if constexpr (!TWO)
    if (tile == kNarrow) return launch<FORM, KIND, 128, 32, 8, 4>(a, st);
  return tile == kWide ? launch<FORM, KIND, 128, TWO ? 64 : 128, 8, TWO ? 4 : 8>(a, st) : launch<FORM, KIND, 64, 64, 4, 4>(a, st);
}
int by_form(const Product& p, const Args& a, Tile tile, cudaStream_t st) {
  if (p.form == kColsCols) return by_tile<kColsCols, kPlain>(a, tile, st);
  if (p.form == kRowsCols) return by_tile<kRowsCols, kPlain>(a, tile, st);
  return p.e.kind == kGated ? by_tile<kRowsRows, kGated>(a, tile, st) : by_tile<kRowsRows, kForward>(a, tile, st);
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
  auto one = [](Matrix m) {                  // samples that follow one another are one
    if (m.B > 1 && m.sb == (long long)m.S * m.st) { m.S *= m.B; m.B = 1; m.sb = 0; }
    return m;
  };
  a.a = one(p.a); a.b = one(p.b); a.e = p.e; a.M = p.M; a.N = p.N;
  a.a_S = FastDiv((unsigned)a.a.S); a.a_inner = FastDiv((unsigned)p.a.inner);
  a.b_S = FastDiv((unsigned)a.b.S); a.b_inner = FastDiv((unsigned)p.b.inner);
  a.a_rows = p.a.B * p.a.S; a.b_rows = p.b.B * p.b.S;
  a.K = p.form == kColsCols ? a.a_rows : p.a.cols;
  return by_form(p, a, c.tile, st);
}

}  // namespace linear
}  // namespace vmoba
