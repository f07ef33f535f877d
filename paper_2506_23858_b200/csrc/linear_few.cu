// Products of few tokens with a weight, x W^T: the weight is read once and everything else is small.
// Bound by HBM, and by how soon all of the weight is asked for.  A CTA has 16 rows of the weight (gated: of both halves), its eight warps
// every eighth run of 64 summed indices; a lane brings sixteen consecutive numbers of a row straight into the registers of the
// matrix instruction, whose summed indices may come in any order as long as x's come in the same.  The warps' sums are added in
// shared memory in a fixed order.
#include <algorithm>

#include "linear.cuh"

namespace vmoba {
namespace linear {
namespace few {

constexpr int WARPS = 8, ROWS = 16, STEP = 64, AHEAD = 4;      // loads of 16 bytes under way per row: AHEAD, two of a run

struct Args {
  Matrix x;
  const __nv_bfloat16* w;
  FastDiv by_S, by_inner;
  int M, N, K;
  Epilogue e;
};

__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_step(float (&d)[4], const uint4& lo, const uint4& hi, const uint4& x) {
  mma(d, lo.x, hi.x, lo.y, hi.y, x.x, x.y);
  mma(d, lo.z, hi.z, lo.w, hi.w, x.z, x.w);
}

// (the weight passes through once)
__device__ __forceinline__ uint4 load_once(const __nv_bfloat16* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.L2::128B.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

// NT: tokens / 8.
template <int NT, int KIND>
__global__ void __launch_bounds__(32 * WARPS) few_kernel(Args p) {
  if (!grid_begin()) return;
  constexpr int NB = KIND == kGated ? 2 : 1, TOKENS = 8 * NT, PITCH = ROWS * NB + 1;
  __shared__ float s_sum[WARPS][TOKENS][PITCH];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int n0 = blockIdx.x * ROWS;
  const __nv_bfloat16* w_row[NB][2];
  bool w_ok[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    w_ok[h] = n0 + g + 8 * h < p.N;
#pragma unroll
    for (int b = 0; b < NB; ++b) w_row[b][h] = p.w + ((long long)(w_ok[h] ? n0 + g + 8 * h : 0) + (long long)b * p.N) * p.K;
  }
  const __nv_bfloat16* x_row[NT];
  bool x_ok[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int r = 8 * j + g;
    x_ok[j] = r < p.M;
    const int b = x_ok[j] ? p.by_S.div(r) : 0, s = x_ok[j] ? r - b * p.x.S : 0;
    x_row[j] = static_cast<const __nv_bfloat16*>(p.x.p) + b * p.x.sb + s * p.x.st;
  }
  float acc[NB][NT][4] = {};
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  // load i of a trip: half of the lane's part of a run
  auto index = [&](int k0, int i) { return k0 + (i >> 1) * WARPS * STEP + 16 * t + 8 * (i & 1); };
  for (int k0 = warp * STEP; k0 < p.K; k0 += WARPS * STEP * (AHEAD / 2)) {
    uint4 w[AHEAD][NB][2], x[AHEAD][NT];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int k = index(k0, i);
      const bool in = k < p.K;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int h = 0; h < 2; ++h) w[i][b][h] = in && w_ok[h] ? load_once(w_row[b][h] + k) : zero;
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int k = index(k0, i);
      const bool in = k < p.K;
      const int z = in && p.x.inner != p.K ? p.by_inner.div(k) : 0;
      const long long at = z * p.x.sh + (k - z * p.x.inner);
#pragma unroll
      for (int j = 0; j < NT; ++j) x[i][j] = in && x_ok[j] ? __ldg(reinterpret_cast<const uint4*>(x_row[j] + at)) : zero;
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int b = 0; b < NB; ++b) mma_step(acc[b][j], w[i][b][0], w[i][b][1], x[i][j]);
  }
  // rows of the weight g and g + 8, tokens 2 t and 2 t + 1
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) s_sum[warp][8 * j + 2 * t + (i & 1)][b * ROWS + g + 8 * (i >> 1)] = acc[b][j][i];
  __syncthreads();
  for (int i = threadIdx.x; i < TOKENS * ROWS * NB; i += 32 * WARPS) {
    const int m = i / (ROWS * NB), c = i % (ROWS * NB);
    float a = 0.f;
#pragma unroll
    for (int v = 0; v < WARPS; ++v) a += s_sum[v][m][c];
    s_sum[0][m][c] = a;                      // (read and written by this thread alone)
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * p.M; i += 32 * WARPS) {
    const int m = i >> 1, c = (i & 1) * 8;
    if (n0 + c >= p.N) continue;
    float u[8], v[8] = {};
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      u[x] = s_sum[0][m][c + x];
      if (KIND == kGated) v[x] = s_sum[0][m][ROWS * (NB - 1) + c + x];
    }
    finish<__nv_bfloat16, 8, KIND>(p.e, OutRow<__nv_bfloat16>(p.e, m), n0 + c, u, v);
  }
}

template <int KIND>
int launch(const Args& a, cudaStream_t st) {
  const unsigned ctas = (unsigned)((a.N + ROWS - 1) / ROWS);
  auto kernel = a.M <= 8 ? few_kernel<1, KIND> : few_kernel<2, KIND>;
  launch_kernel(kernel, ctas, 32 * WARPS, 0, st, a);
  VMOBA_LAUNCH_OK(1);
  return VMOBA_OK;
}

}  // namespace few

// 16 tokens: 1,536 -> 9,216 channels 13 us, by tiles 19; 5,120 -> 20,480 53 and 68.  32 tokens: 18 and 19, 118 and 68.
bool few_takes(const Product& p) { return p.bf16 && p.form == kRowsRows && p.M <= 16; }

int few_product(const Product& p, cudaStream_t st) {
  few::Args a{p.a, static_cast<const __nv_bfloat16*>(p.b.p), FastDiv((unsigned)p.a.S), FastDiv((unsigned)p.a.inner), p.M, p.N, p.a.cols, p.e};
  return p.e.kind == kGated ? few::launch<kGated>(a, st) : few::launch<kForward>(a, st);
}

}  // namespace linear
}  // namespace vmoba
