// Linear layers and feed-forward blocks: entry points, and what their backward passes do ahead of the matrix products,
//   du = act'(u) * (gate * d_out)   (gated: da = v act'(u) .., dv = act(u) ..),   db = sum du,   dgate = sum over a group's tokens d_out act(u),
// which is one pass over d_out and what the forward kept: bound by HBM.  A warp takes 256 columns of a row, a CTA eight rows at a time
// of a chunk of one group, so that columns add up in registers; the chunks' sums are added by a second kernel in a fixed order.  (13,440 tokens of
// 1,536 channels with a gate: 31 us, 4.0 TB/s, 42 % of the issue slots.)
#include <algorithm>
#include <initializer_list>

#include "linear.cuh"

namespace vmoba {
namespace linear {
namespace {

struct Dims {
  int B, S, in, out, wide;                   // wide: rows of the weight
  int dtype, es, act, heads, gt, G;          // gt: tokens per row of the gate; G: rows per sample
  bool gated;
  long long rows;
};

int make_dims(const vmoba_linear_shape* s, Dims* o) {
  if (!s) return VMOBA_ERR_ARG;
  if (s->dtype != VMOBA_F32 && s->dtype != VMOBA_BF16) return VMOBA_ERR_ARG;
  if (s->activation < VMOBA_ACT_NONE || s->activation > VMOBA_ACT_SILU || s->gated < 0 || s->gated > 1) return VMOBA_ERR_ARG;
  if (s->B <= 0 || s->S <= 0 || s->in <= 0 || s->out <= 0 || s->in % 8 || s->out % 8) return VMOBA_ERR_SHAPE;
  if (s->in > (1 << 20) || s->out > (1 << 20) || (long long)s->B * s->S > (1ll << 30)) return VMOBA_ERR_SHAPE;
  if (s->heads < 0 || s->gate_tokens < 0) return VMOBA_ERR_ARG;
  if (s->heads && (s->in % s->heads || (s->in / s->heads != 64 && s->in / s->heads != 128))) return VMOBA_ERR_SHAPE;
  o->B = s->B; o->S = s->S; o->in = s->in; o->out = s->out; o->dtype = s->dtype; o->act = s->activation; o->heads = s->heads;
  o->gated = s->gated != 0;
  o->wide = o->gated ? 2 * s->out : s->out;
  o->es = s->dtype == VMOBA_BF16 ? 2 : 4;
  o->gt = s->gate_tokens && s->gate_tokens < s->S ? s->gate_tokens : s->S;
  o->G = (s->S + o->gt - 1) / o->gt;
  o->rows = (long long)s->B * s->S;
  return VMOBA_OK;
}

// Element strides {batch, token} of rows of `cols` elements that the kernels can address; dimensions of one are not looked at.
bool strides_ok(const int64_t* st, const Dims& D, int cols, bool zero_ok) {
  if (!st) return false;
  const int n[2] = {D.B, D.S};
  for (int i = 0; i < 2; ++i) {
    if (n[i] == 1) continue;
    if (st[i] % (16 / D.es)) return false;
    if (!(zero_ok && st[i] == 0) && (st[i] < cols || st[i] >= (1ll << 38))) return false;
  }
  return true;
}
Matrix raster(const void* p, const int64_t* st, const Dims& D, int cols) {
  return Matrix{p, D.B, D.S, cols, cols, D.B > 1 ? st[0] : 0, D.S > 1 ? st[1] : cols, 0};
}
// x: raster order through strides, or dense in block order.
Matrix input(const void* p, const int64_t* st, const Dims& D) {
  if (!D.heads) return raster(p, st, D, D.in);
  const int d = D.in / D.heads;
  return Matrix{p, D.B, D.S, D.in, d, (long long)D.heads * D.S * d, d, (long long)D.S * d};
}
bool gate_ok(const float* gate, const int64_t* gs, const Dims& D) {
  if (!gate) return true;
  if (!gs || !aligned16(gate)) return false;
  const int n[2] = {D.B, D.G};
  for (int i = 0; i < 2; ++i)
    if (n[i] > 1 && (gs[i] % 4 || (gs[i] != 0 && gs[i] < D.out) || gs[i] >= (1ll << 38))) return false;
  return true;
}

// ---------------------------------------------------------------- ahead of the backward's products
constexpr int kTile = 256;                   // columns of a CTA
// Rows of a chunk: eight per warp, two of them under way at once; fewer where there would be less than three CTAs for an SM.
int chunk_of(const Dims& D) {
  int rows = 64;
  while (rows > 8 && (long long)D.B * D.G * ((D.gt + rows - 1) / rows) * ((D.out + kTile - 1) / kTile) < 3 * 148) rows /= 2;
  return rows;
}

struct Prep {
  int S, G, gt, cpg, cols, act;              // cpg: chunks per group
  int chunk, tiles;                          // rows of a chunk; tiles of columns
  bool gated;
  FastDiv by_cpg, by_G, by_tiles;
  const void* d;
  long long db, dt;
  const void* kept;                          // [rows, cols or 2 cols] dense, in the order of x
  const float* gate;
  long long gb, gg;
  const int* inv;                            // place in the order of x of every token of d_out, or (by_place: a sample is one group, so that
  bool by_place;                             // its rows come in any order) token of d_out of every place
  void* du;                                  // as kept
  void* du_low;                              // what du's rounding left
  void* y;                                   // act(kept) again, [rows, cols]
  float* part_b;                             // [chunk][cols or 2 cols]
  float* part_g;                             // [chunk][cols]
};

// Eight numbers as they lie in memory.
template <typename T>
struct Packed {
  uint4 w[sizeof(T) / 2];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (auto& x : w) x = make_uint4(0u, 0u, 0u, 0u);
  }
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 2); ++i) w[i] = reinterpret_cast<const uint4*>(p)[i];
  }
  __device__ __forceinline__ void unpack(float (&x)[8]) const { load_vec<8>(reinterpret_cast<const T*>(w), x); }
};

template <typename T, bool GATED>
__global__ void __launch_bounds__(256, GATED ? 2 : 3) prep_kernel(Prep p) {
  if (!grid_begin()) return;
  constexpr bool EXACT = sizeof(T) == 4;
  __shared__ float s_sum[8][kTile];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // (tiles of columns next to one another in time)
  const int at_chunk = p.by_tiles.div(blockIdx.x), tile = blockIdx.x - at_chunk * p.tiles, c = tile * kTile + lane * 8;
  const int gi = p.by_cpg.div(at_chunk), j = at_chunk - gi * p.cpg;          // group of all samples' and chunk of it
  const int b = p.by_G.div(gi), g = gi - b * p.G;
  const int t0 = g * p.gt + j * p.chunk, t1 = min(min(t0 + p.chunk, (g + 1) * p.gt), p.S);
  const int wide = GATED ? 2 * p.cols : p.cols;
  float sb[8] = {}, sv[8] = {}, sg[8] = {};
  if (c < p.cols) {
    float gate[8];
    if (p.gate) load_vec<8>(p.gate + b * p.gb + g * p.gg + c, gate);
    const T* d_row = static_cast<const T*>(p.d) + b * p.db + c;
    constexpr int R = 2;
#pragma unroll 1
    for (int first = t0 + warp; first < t1; first += 8 * R) {
      Packed<T> d_in[R], u_in[R], v_in[R];
      long long row[R];
#pragma unroll
      for (int k = 0; k < R; ++k) {
        const int t = first + 8 * k;
        row[k] = -1;
        d_in[k].clear();
        u_in[k].clear();
        v_in[k].clear();
        if (t >= t1) continue;
        const int other = p.inv ? __ldg(p.inv + t) : t, at = p.by_place ? t : other, from = p.by_place ? other : t;
        if ((unsigned)at >= (unsigned)p.S) continue;
        row[k] = (long long)b * p.S + at;
        if ((unsigned)from >= (unsigned)p.S) continue;      // (a place without a token has no gradient, whatever was kept there)
        d_in[k].load(d_row + from * p.dt);
        if (p.kept) {
          u_in[k].load(static_cast<const T*>(p.kept) + row[k] * wide + c);
          if (GATED) v_in[k].load(static_cast<const T*>(p.kept) + row[k] * wide + p.cols + c);
        }
      }
#pragma unroll
      for (int k = 0; k < R; ++k) {
        const long long r = row[k];
        if (r < 0) continue;
        float d[8], u[8], v[8];
        d_in[k].unpack(d);
        if (p.kept) {
          u_in[k].unpack(u);
          if (GATED) v_in[k].unpack(v);
          float y[8];
          by_activation(p.act, [&](auto act) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float2 a = activate_slope<EXACT, decltype(act)::value>(u[i]);
              y[i] = GATED ? a.x * v[i] : a.x;
              sg[i] = fmaf(d[i], y[i], sg[i]);
              if (p.gate) d[i] *= gate[i];
              if (GATED) {
                const float dv = d[i] * a.x;
                d[i] *= a.y * v[i];
                v[i] = dv;
                sv[i] += dv;
              } else {
                d[i] *= a.y;
              }
            }
          });
          if (p.y) store_vec<8>(static_cast<T*>(p.y) + r * p.cols + c, y);
          if (GATED && p.du) store_vec<8>(static_cast<T*>(p.du) + r * wide + p.cols + c, v);
          if (GATED && sizeof(T) == 2 && p.du_low) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] -= to_f32<T>(from_f32<T>(v[i]));
            store_vec<8>(static_cast<T*>(p.du_low) + r * wide + p.cols + c, v);
          }
        } else if (p.gate) {
#pragma unroll
          for (int i = 0; i < 8; ++i) d[i] *= gate[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) sb[i] += d[i];
        if (p.du) store_vec<8>(static_cast<T*>(p.du) + r * wide + c, d);
        if (sizeof(T) == 2 && p.du_low) {
#pragma unroll
          for (int i = 0; i < 8; ++i) d[i] -= to_f32<T>(from_f32<T>(d[i]));
          store_vec<8>(static_cast<T*>(p.du_low) + r * wide + c, d);
        }
      }
    }
  }
  // the eight warps' sums, one set after another
  auto add_up = [&](const float (&s)[8], float* to) {
    __syncthreads();
    store_vec<8>(&s_sum[warp][lane * 8], s);
    __syncthreads();
    const int col = tile * kTile + threadIdx.x;
    if (col < p.cols) {
      float a = 0.f;
#pragma unroll
      for (int w = 0; w < 8; ++w) a += s_sum[w][threadIdx.x];
      to[col] = a;
    }
  };
  if (p.part_b) {
    add_up(sb, p.part_b + (long long)at_chunk * wide);
    if (GATED) add_up(sv, p.part_b + (long long)at_chunk * wide + p.cols);
  }
  if (p.part_g) add_up(sg, p.part_g + (long long)at_chunk * p.cols);
}

// Place in the order of x of every token, from the token of every place: the last one where it has several, -1 where it has none.  Places that
// no token leads to have a gradient of zero.
__global__ void __launch_bounds__(256) no_place_kernel(int S, int* inv, uint4* du, long long vecs) {
  if (!grid_begin()) return;
  const long long n = (long long)gridDim.x * 256;
  for (long long i = blockIdx.x * 256ll + threadIdx.x; i < S; i += n) inv[i] = -1;
  if (du)
    for (long long i = blockIdx.x * 256ll + threadIdx.x; i < vecs; i += n) du[i] = make_uint4(0u, 0u, 0u, 0u);
}
__global__ void __launch_bounds__(256) place_kernel(int S, const int* perm, int* inv) {
  if (!grid_begin()) return;
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < S) {
    const int t = __ldg(perm + i);
    if ((unsigned)t < (unsigned)S) atomicMax(inv + t, i);
  }
}

template <typename T>
int run_prep(Prep p, int chunks, cudaStream_t st) {
  p.tiles = (p.cols + kTile - 1) / kTile;
  p.by_tiles = FastDiv((unsigned)p.tiles);
  if ((long long)chunks * p.tiles > INT32_MAX) return VMOBA_ERR_SHAPE;
  const unsigned grid = (unsigned)(chunks * p.tiles);
  if (p.gated) launch_kernel(prep_kernel<T, true>, grid, 256, 0, st, p);
  else launch_kernel(prep_kernel<T, false>, grid, 256, 0, st, p);
  VMOBA_LAUNCH_OK(1);
  return VMOBA_OK;
}
int run_prep(const Prep& p, bool bf16, int chunks, cudaStream_t st) {
  return bf16 ? run_prep<__nv_bfloat16>(p, chunks, st) : run_prep<float>(p, chunks, st);
}
int chunks_of(const Dims& D) { return D.B * D.G * ((D.gt + chunk_of(D) - 1) / chunk_of(D)); }

}  // namespace

// ---------------------------------------------------------------- sums of chunks
// out[g][c] = sum over the `per` chunks of group g of part[chunk][c]: a CTA has 32 columns of a group, a warp every eighth chunk.  Two such sums
// in one launch.
struct ChunkSum {
  const float* part = nullptr;
  void* out = nullptr;
  int cols = 0, groups = 0, per = 0, tiles = 0, bf16 = 0;
};
__global__ void __launch_bounds__(256) sum_chunks_kernel(ChunkSum a, ChunkSum b) {
  if (!grid_begin()) return;
  __shared__ float s[8][33];
  const int first = a.tiles * a.groups;
  const bool second = (int)blockIdx.x >= first;
  const ChunkSum& p = second ? b : a;
  const int i = second ? blockIdx.x - first : blockIdx.x;
  const int g = i / p.tiles, c = (i - g * p.tiles) * 32 + (threadIdx.x & 31), w = threadIdx.x >> 5;
  float sum = 0.f;
  if (c < p.cols) {
    const float* from = p.part + (long long)g * p.per * p.cols + c;
#pragma unroll 8
    for (int k = w; k < p.per; k += 8) sum += from[(long long)k * p.cols];
  }
  s[w][threadIdx.x & 31] = sum;
  __syncthreads();
  if (w == 0 && c < p.cols) {
#pragma unroll
    for (int k = 1; k < 8; ++k) sum += s[k][threadIdx.x];
    const long long at = (long long)g * p.cols + c;
    if (p.bf16) static_cast<__nv_bfloat16*>(p.out)[at] = from_f32<__nv_bfloat16>(sum);
    else static_cast<float*>(p.out)[at] = sum;
  }
}
static int sum_chunks(ChunkSum a, ChunkSum b, cudaStream_t st) {
  a.tiles = (a.cols + 31) / 32;
  b.tiles = (b.cols + 31) / 32;
  const long long ctas = (long long)a.groups * a.tiles + (long long)b.groups * b.tiles;
  if (ctas > INT32_MAX) return VMOBA_ERR_SHAPE;
  if (ctas == 0) return VMOBA_OK;
  launch_kernel(sum_chunks_kernel, (unsigned)ctas, 256, 0, st, a, b);
  VMOBA_LAUNCH_OK(1);
  return VMOBA_OK;
}

size_t product_scratch(const Product& p) { return !p.bf16 ? simt_scratch(p) : few_takes(p) ? 0 : tc_scratch(p); }
int run_product(const Product& p, float* scratch, cudaStream_t st) {
  if (!p.bf16) return simt_product(p, scratch, st);
  return few_takes(p) ? few_product(p, st) : tc_product(p, scratch, st);
}

namespace {

// ---------------------------------------------------------------- the products of a layer
Product product(const Dims& D, Form form, const Matrix& a, const Matrix& b, int M, int N, int32_t* status) {
  Product p{};
  p.form = form; p.a = a; p.b = b; p.M = M; p.N = N;
  p.bf16 = D.dtype == VMOBA_BF16;
  p.planes = 1;
  p.status = status;
  return p;
}
// Dense rows of the layer's tokens.
Matrix tokens(const void* p, const Dims& D, int cols) { return Matrix{p, D.B, D.S, cols, cols, (long long)D.S * cols, cols, 0}; }

Product forward_product(const Dims& D, const Matrix& x, const void* w, const Matrix& out, int32_t* status) {
  Product p = product(D, kRowsRows, x, dense(w, D.wide, D.in), (int)D.rows, D.out, status);
  set_out(&p.e, out);
  p.e.kind = D.gated ? kGated : kForward;
  p.e.act = D.act;
  p.e.by_gate = FastDiv((unsigned)D.gt);
  return p;
}
Product dx_product(const Dims& D, const Matrix& du, const void* w, const Matrix& dx, int32_t* status) {
  Product p = product(D, kRowsCols, du, dense(w, D.wide, D.in), (int)D.rows, D.in, status);
  set_out(&p.e, dx);
  return p;
}
// The gradient of the product of the layer ahead (`up`, whose output this layer's input is) from du: through this layer's weight and that
// layer's activation.
Product slope_product(const Dims& D, const Dims& up, const Matrix& du, const void* w, const void* kept, const Matrix& d_up, int32_t* status) {
  Product p = dx_product(D, du, w, d_up, status);
  p.e.kind = up.gated ? kSlopeGated : kSlope;
  p.e.act = up.act;
  p.e.cols = up.out;
  p.e.kept = const_cast<void*>(kept);
  return p;
}
Product dw_product(const Dims& D, const Matrix& du, const Matrix& x, void* dw, int32_t* status) {
  Product p = product(D, kColsCols, du, x, D.wide, D.in, status);
  set_out(&p.e, dense(dw, D.wide, D.in));
  return p;
}
// Floats of scratch that the products of a layer need.
size_t forward_scratch(const Dims& D) {
  return product_scratch(forward_product(D, tokens(nullptr, D, D.in), nullptr, tokens(nullptr, D, D.out), nullptr));
}
size_t gradient_scratch(const Dims& D, int planes = 1) {
  const Matrix du = tokens(nullptr, D, D.wide), x = tokens(nullptr, D, D.in);
  Product dx = dx_product(D, du, nullptr, x, nullptr), dw = dw_product(D, du, x, nullptr, nullptr);
  size_t most = std::max(product_scratch(dx), product_scratch(dw));
  if (planes == 2) {
    dx.planes = dw.planes = 2;
    most = std::max(most, std::max(product_scratch(dx), product_scratch(dw)));
  }
  return most;
}

// The two layers of a feed-forward block.
Dims up_of(const Dims& D) { return D; }
Dims down_of(const Dims& D) {
  Dims o = D;
  o.in = D.out; o.out = o.wide = D.in; o.gated = false; o.act = VMOBA_ACT_NONE;
  return o;
}

// Gate, residual and output of a call.
struct Ends {
  const float* gate;
  const int64_t* gate_strides;
  const void* residual;
  const int64_t* residual_strides;
  void* out;
  const int64_t* out_strides;
  bool ok(const Dims& D) const {
    return out && aligned16(out) && aligned16(residual) && strides_ok(out_strides, D, D.out, false) &&
           (!residual || strides_ok(residual_strides, D, D.out, true)) && gate_ok(gate, gate_strides, D);
  }
  void give(const Dims& D, Epilogue* e) const {
    e->gate = gate;
    if (gate) { e->gb = D.B > 1 ? gate_strides[0] : 0; e->gg = D.G > 1 ? gate_strides[1] : 0; }
    e->residual = residual;
    if (residual) { e->rb = D.B > 1 ? residual_strides[0] : 0; e->rt = D.S > 1 ? residual_strides[1] : 0; }
  }
};

Prep prep_of(const Dims& D, const void* d, const int64_t* ds, const float* gate, const int64_t* gs, const void* kept) {
  Prep p{};
  p.S = D.S; p.G = D.G; p.gt = D.gt; p.chunk = chunk_of(D); p.cpg = (D.gt + p.chunk - 1) / p.chunk; p.cols = D.out; p.act = D.act; p.gated = D.gated;
  p.by_cpg = FastDiv((unsigned)p.cpg); p.by_G = FastDiv((unsigned)D.G);
  p.d = d; p.db = D.B > 1 ? ds[0] : 0; p.dt = D.S > 1 ? ds[1] : 0;
  p.kept = kept;
  p.gate = gate;
  if (gate) { p.gb = D.B > 1 ? gs[0] : 0; p.gg = D.G > 1 ? gs[1] : 0; }
  return p;
}
// Without a gate all tokens of a sample are one group.
Dims ungrouped(Dims D) {
  D.gt = D.S; D.G = 1;
  return D;
}

// Chunks of a layer's rows at most, with its groups or without.
size_t most_chunks(const Dims& D) { return (size_t)std::max(chunks_of(D), chunks_of(ungrouped(D))); }

// Planes of a layer's du in bf16.  Its rounding adds as much to the error of dx and dweight as their own has, however many terms their sums are of: root
// mean square against 64 bits 2.35e-3 at 128 tokens as at 32,760, and 1.66e-3, their own alone, with a second plane of what the rounding left.
// That doubles the products (a call of 13,440 tokens, 1,536 channels in and out: 122 us and 208), so it is there where it costs nothing: the host takes
// 28 to 31 us for a call and the device 11 to 28 with both planes (0.4 to 7 less with one, which is what a graph of such calls would gain).
// Beyond it shows: one token, 8,192 channels in and out 84 us a call and 103, 8 to 65,528 channels 36 and 46.
int planes_of(const Dims& D) {
  const bool few = D.rows * (D.wide + D.in) <= 1 << 16 && (long long)D.wide * D.in <= 1 << 22 && D.wide <= 1 << 13;
  return D.dtype == VMOBA_BF16 && few ? 2 : 1;
}

struct Scratch {
  int* inv;
  char *du, *dh, *du_up, *h;
  float *part_b, *part_g, *product;
  Guards guards;
  size_t bytes;
};
// The size that a call states: 256 says that it uses none of them, so that several calls can be given the same; more wherever it uses some.
size_t stated(const Carver& c) { return c.total() ? std::max<size_t>(c.total(), 512) : 256; }
Scratch linear_scratch(const Dims& D, bool backward, void* ws) {
  Carver c(ws);
  Scratch s{};
  if (backward) {
    s.inv = c.take<int>(D.heads ? D.S : 0);
    s.du = c.take<char>((size_t)D.rows * D.wide * D.es * planes_of(D));
    s.part_b = c.take<float>(most_chunks(D) * D.wide);
    s.part_g = c.take<float>(most_chunks(D) * D.out);
    s.product = c.take<float>(gradient_scratch(D, planes_of(D)));
  } else {
    s.product = c.take<float>(forward_scratch(D));
  }
  s.guards = c.guards;
  s.bytes = stated(c);
  return s;
}
Scratch ffn_scratch(const Dims& D, bool backward, void* ws) {
  const Dims up = up_of(D), down = down_of(D);
  Carver c(ws);
  Scratch s{};
  s.h = c.take<char>((size_t)D.rows * D.out * D.es);
  if (backward) {
    const bool bf16 = D.dtype == VMOBA_BF16;
    s.du = c.take<char>((size_t)D.rows * down.out * D.es * (bf16 ? 2 : 1));
    s.dh = c.take<char>(bf16 ? 0 : (size_t)D.rows * D.out * D.es);
    s.du_up = c.take<char>(bf16 || D.gated ? (size_t)D.rows * D.wide * D.es : 0);
    const size_t of_up = bf16 ? (size_t)(D.rows + 31) / 32 : 0;      // (bf16: sums by 32 rows)
    s.part_b = c.take<float>(std::max(std::max(most_chunks(up), of_up) * up.wide, most_chunks(down) * down.out));
    s.part_g = c.take<float>(most_chunks(down) * down.out);
    s.product = c.take<float>(std::max(gradient_scratch(up), gradient_scratch(down, bf16 ? 2 : 1)));
  } else {
    s.product = c.take<float>(std::max(forward_scratch(up), forward_scratch(down)));
  }
  s.guards = c.guards;
  s.bytes = stated(c);
  return s;
}

bool all_aligned(std::initializer_list<const void*> ps) {
  for (const void* p : ps)
    if (!aligned16(p)) return false;
  return true;
}

// du, and the sums of it (db) and of the gate's gradient.
int prepare(const Dims& D, Prep p, const Scratch& s, void* du, void* db, float* dgate, cudaStream_t st) {
  p.du = du;
  p.part_b = db ? s.part_b : nullptr;
  p.part_g = dgate ? s.part_g : nullptr;
  const int chunks = chunks_of(D);
  if (int rc = run_prep(p, D.dtype == VMOBA_BF16, chunks, st)) return rc;
  ChunkSum b, g;
  if (db) b = ChunkSum{s.part_b, db, D.wide, 1, chunks, 0, D.dtype == VMOBA_BF16};
  if (dgate) g = ChunkSum{s.part_g, dgate, D.out, D.B * D.G, p.cpg, 0, 0};
  return sum_chunks(b, g, st);
}

}  // namespace
}  // namespace linear
}  // namespace vmoba

using namespace vmoba;
using namespace vmoba::linear;

extern "C" size_t vmoba_linear_workspace_bytes(const vmoba_linear_shape* shape, int backward) {
  linear::Dims D;
  return linear::make_dims(shape, &D) ? 0 : linear_scratch(D, backward != 0, nullptr).bytes;
}

extern "C" int vmoba_linear(const vmoba_linear_shape* shape, const void* x, const int64_t x_strides[2], const void* weight, const void* bias,
                            const float* gate, const int64_t gate_strides[2], const void* residual, const int64_t residual_strides[2],
                            void* out, const int64_t out_strides[2], void* kept, const int32_t* perm, int32_t* dev_status, void* ws,
                            size_t ws_bytes, void* stream) {
  linear::Dims D;
  if (int rc = linear::make_dims(shape, &D)) return rc;
  const Ends ends{gate, gate_strides, residual, residual_strides, out, out_strides};
  if (!x || !weight || !ws || !all_aligned({x, weight, bias, kept, ws}) || !ends.ok(D)) return VMOBA_ERR_ARG;
  if (perm && !D.heads) return VMOBA_ERR_ARG;
  if (!D.heads && !strides_ok(x_strides, D, D.in, false)) return VMOBA_ERR_ARG;
  const Scratch s = linear_scratch(D, false, ws);
  if (ws_bytes < s.bytes) return VMOBA_ERR_WORKSPACE;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  Product p = forward_product(D, input(x, x_strides, D), weight, raster(out, out_strides, D, D.out), dev_status);
  p.e.bias = bias;
  p.e.kept = kept;
  p.e.perm = perm;
  ends.give(D, &p.e);
  VMOBA_GUARDS_ARM(s.guards, st);
  if (int rc = run_product(p, s.product, st)) return rc;
  VMOBA_GUARDS_CHECK(s.guards, dev_status, st);
  return VMOBA_OK;
}

extern "C" int vmoba_linear_bwd(const vmoba_linear_shape* shape, const void* d_out, const int64_t d_out_strides[2], const void* x,
                                const int64_t x_strides[2], const void* weight, const void* kept, const float* gate,
                                const int64_t gate_strides[2], void* dx, const int64_t dx_strides[2], void* dweight, void* dbias,
                                float* dgate, const int32_t* perm, int32_t* dev_status, void* ws, size_t ws_bytes, void* stream) {
  linear::Dims D;
  if (int rc = linear::make_dims(shape, &D)) return rc;
  if (!d_out || !ws || !all_aligned({d_out, x, weight, kept, dx, dweight, dbias, dgate, ws})) return VMOBA_ERR_ARG;
  if (!strides_ok(d_out_strides, D, D.out, false) || !gate_ok(gate, gate_strides, D)) return VMOBA_ERR_ARG;
  if ((dx && !weight) || (dweight && !x) || (perm && !D.heads) || (dgate && !gate)) return VMOBA_ERR_ARG;
  const bool acts = D.act != VMOBA_ACT_NONE || D.gated;
  if ((acts || dgate) && !kept) return VMOBA_ERR_ARG;
  if (!D.heads && dweight && !strides_ok(x_strides, D, D.in, false)) return VMOBA_ERR_ARG;
  if (!D.heads && dx && !strides_ok(dx_strides, D, D.in, false)) return VMOBA_ERR_ARG;
  const Scratch s = linear_scratch(D, true, ws);
  if (ws_bytes < s.bytes) return VMOBA_ERR_WORKSPACE;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (!gate) D = ungrouped(D);
  VMOBA_GUARDS_ARM(s.guards, st);
  Prep p = prep_of(D, d_out, d_out_strides, gate, gate_strides, acts || dgate ? kept : nullptr);
  // (nothing stands between d_out and du in the simplest layer)
  const bool apart = (acts || gate || perm) && (dx || dweight);
  const int planes = apart && (acts || gate) ? planes_of(D) : 1;
  const long long plane = D.rows * D.wide;
  if (planes == 2) p.du_low = s.du + plane * D.es;
  if (perm && D.G == 1) {
    p.inv = perm;
    p.by_place = true;
  } else if (perm) {
    launch_kernel(no_place_kernel, (unsigned)(4 * sm_count()), 256, 0, st, D.S, s.inv, apart ? reinterpret_cast<uint4*>(s.du) : nullptr,
                  planes * plane * D.es / 16);
    launch_kernel(place_kernel, (unsigned)((D.S + 255) / 256), 256, 0, st, D.S, perm, s.inv);
    VMOBA_LAUNCH_OK(2);
    p.inv = s.inv;
  }
  if (apart || dbias || dgate)
    if (int rc = prepare(D, p, s, apart ? s.du : nullptr, dbias, dgate, st)) return rc;
  const Matrix du = apart ? tokens(s.du, D, D.wide) : raster(d_out, d_out_strides, D, D.out);
  if (dx) {
    Product q = dx_product(D, du, weight, input(dx, dx_strides, D), dev_status);
    q.planes = planes;
    q.plane = plane;
    if (int rc = run_product(q, s.product, st)) return rc;
  }
  if (dweight) {
    Product q = dw_product(D, du, input(x, x_strides, D), dweight, dev_status);
    q.planes = planes;
    q.plane = plane;
    if (int rc = run_product(q, s.product, st)) return rc;
  }
  VMOBA_GUARDS_CHECK(s.guards, dev_status, st);
  return VMOBA_OK;
}

extern "C" size_t vmoba_ffn_workspace_bytes(const vmoba_linear_shape* shape, int backward) {
  linear::Dims D;
  return linear::make_dims(shape, &D) || D.heads ? 0 : ffn_scratch(D, backward != 0, nullptr).bytes;
}

extern "C" int vmoba_ffn(const vmoba_linear_shape* shape, const void* x, const int64_t x_strides[2], const void* w_up, const void* b_up,
                         const void* w_down, const void* b_down, const float* gate, const int64_t gate_strides[2], const void* residual,
                         const int64_t residual_strides[2], void* out, const int64_t out_strides[2], void* kept_up, void* kept_down,
                         int32_t* dev_status, void* ws, size_t ws_bytes, void* stream) {
  linear::Dims D;
  if (int rc = linear::make_dims(shape, &D)) return rc;
  if (D.heads) return VMOBA_ERR_ARG;
  const linear::Dims up = up_of(D), down = down_of(D);
  const Ends ends{gate, gate_strides, residual, residual_strides, out, out_strides};
  if (!x || !w_up || !w_down || !ws || !all_aligned({x, w_up, b_up, w_down, b_down, kept_up, kept_down, ws})) return VMOBA_ERR_ARG;
  if (!ends.ok(down) || !strides_ok(x_strides, up, up.in, false)) return VMOBA_ERR_ARG;
  const Scratch s = ffn_scratch(D, false, ws);
  if (ws_bytes < s.bytes) return VMOBA_ERR_WORKSPACE;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  VMOBA_GUARDS_ARM(s.guards, st);
  Product p = forward_product(up, input(x, x_strides, up), w_up, tokens(s.h, up, up.out), dev_status);
  p.e.bias = b_up;
  p.e.kept = kept_up;
  if (int rc = run_product(p, s.product, st)) return rc;
  p = forward_product(down, tokens(s.h, down, down.in), w_down, raster(out, out_strides, down, down.out), dev_status);
  p.e.bias = b_down;
  p.e.kept = kept_down;
  ends.give(down, &p.e);
  if (int rc = run_product(p, s.product, st)) return rc;
  VMOBA_GUARDS_CHECK(s.guards, dev_status, st);
  return VMOBA_OK;
}

extern "C" int vmoba_ffn_bwd(const vmoba_linear_shape* shape, const void* d_out, const int64_t d_out_strides[2], const void* x,
                             const int64_t x_strides[2], const void* w_up, const void* w_down, const void* kept_up, const void* kept_down,
                             const float* gate, const int64_t gate_strides[2], void* dx, const int64_t dx_strides[2], void* dw_up,
                             void* db_up, void* dw_down, void* db_down, float* dgate, int32_t* dev_status, void* ws, size_t ws_bytes,
                             void* stream) {
  linear::Dims D;
  if (int rc = linear::make_dims(shape, &D)) return rc;
  if (D.heads) return VMOBA_ERR_ARG;
  linear::Dims up = up_of(D), down = down_of(D);
  if (!d_out || !ws || !all_aligned({d_out, x, w_up, w_down, kept_up, kept_down, dx, dw_up, db_up, dw_down, db_down, dgate, ws})) return VMOBA_ERR_ARG;
  if (!strides_ok(d_out_strides, down, down.out, false) || !gate_ok(gate, gate_strides, down)) return VMOBA_ERR_ARG;
  const bool through = dx || dw_up || db_up;                       // the gradient of h is needed
  if ((through && (!w_down || !kept_up)) || (dx && !w_up) || (dw_up && !x) || (dw_down && !kept_up) || (dgate && (!gate || !kept_down)))
    return VMOBA_ERR_ARG;
  if ((dw_up && !strides_ok(x_strides, up, up.in, false)) || (dx && !strides_ok(dx_strides, up, up.in, false))) return VMOBA_ERR_ARG;
  const Scratch s = ffn_scratch(D, true, ws);
  if (ws_bytes < s.bytes) return VMOBA_ERR_WORKSPACE;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (!gate) down = ungrouped(down);
  up = ungrouped(up);
  VMOBA_GUARDS_ARM(s.guards, st);
  // Through the gate.  In bf16 what the rounding of gate * d_out leaves is kept as a second plane, and the products of it have both: rounded
  // here and again at the first product's gradient, dx and dw_up would be 1.7 times as far off as their own rounding leaves them, not 1.4.
  const bool bf16 = up.dtype == VMOBA_BF16;
  Prep p = prep_of(down, d_out, d_out_strides, gate, gate_strides, dgate ? kept_down : nullptr);
  const long long plane = down.rows * down.out;
  const bool dense_d = (down.S == 1 || d_out_strides[1] == down.out) && (down.B == 1 || d_out_strides[0] == (int64_t)down.S * down.out);
  const bool apart = (gate || (bf16 && !dense_d)) && (through || dw_down);
  const int planes = bf16 && gate && apart ? 2 : 1;
  if (planes == 2) p.du_low = s.du + plane * up.es;
  if (apart || db_down || dgate)
    if (int rc = prepare(down, p, s, apart ? s.du : nullptr, db_down, dgate, st)) return rc;
  const Matrix d_down = apart ? tokens(s.du, down, down.out) : raster(d_out, d_out_strides, down, down.out);
  // the gradient of h; from that, the activation's slope, that of the first product, and h again
  void* const d_up = bf16 || up.gated ? s.du_up : s.dh;
  if (through && bf16) {
    Product q = slope_product(down, up, d_down, w_down, kept_up, tokens(d_up, up, up.out), dev_status);
    q.planes = planes;
    q.plane = plane;
    q.e.again = dw_down ? s.h : nullptr;
    q.e.col_sums = db_up ? s.part_b : nullptr;
    if (int rc = run_product(q, s.product, st)) return rc;
    if (db_up)
      if (int rc = sum_chunks(ChunkSum{s.part_b, db_up, up.wide, 1, (int)((up.rows + 31) / 32), 0, 1}, {}, st)) return rc;
  } else if (through || dw_down) {           // (fp32: d_up in the place of dh, where it is not gated; for h alone any gradient does)
    if (through)
      if (int rc = run_product(dx_product(down, d_down, w_down, tokens(s.dh, down, down.in), dev_status), s.product, st)) return rc;
    const int64_t of_dh[2] = {(int64_t)up.S * up.out, up.out}, of_kept[2] = {(int64_t)up.S * up.wide, up.wide};
    p = prep_of(up, through ? (const void*)s.dh : kept_up, through ? of_dh : of_kept, nullptr, nullptr, kept_up);
    p.y = dw_down ? s.h : nullptr;
    if (int rc = prepare(up, p, s, dx || dw_up ? d_up : nullptr, db_up, nullptr, st)) return rc;
  }
  if (dw_down) {
    Product q = dw_product(down, d_down, tokens(s.h, down, down.in), dw_down, dev_status);
    q.planes = planes;
    q.plane = plane;
    if (int rc = run_product(q, s.product, st)) return rc;
  }
  const Matrix du = tokens(d_up, up, up.wide);
  if (dw_up)
    if (int rc = run_product(dw_product(up, du, input(x, x_strides, up), dw_up, dev_status), s.product, st)) return rc;
  if (dx)
    if (int rc = run_product(dx_product(up, du, w_up, input(dx, dx_strides, up), dev_status), s.product, st)) return rc;
  VMOBA_GUARDS_CHECK(s.guards, dev_status, st);
  return VMOBA_OK;
}
