// The gated feed-forward block's hidden values, out = act(x Wg') * (x Wu'), and its gradient:
//   dg = dout * u * act'(g),  du = dout * act(g),
//   dx = dg Wg + du Wu,  dWg = dg' x,  dWu = du' x,
// as tiled products on the matrix units with fp32 sums. The forward pass has both projections of
// a tile of hidden values in one block, whose epilogue multiplies them; the gradient forms g and u
// again in the same way (nothing is kept from the forward pass), its epilogue writes dg and du,
// rounded once as operands of the three products that follow.
//
// Tiles. Every product is taken transposed: the result's contiguous axis is the A operand's, so
// that a lane holds 4 consecutive values of a result's row. A step has 64 of the summed axis; an
// operand's tile in LDS has either its rows running along the summed axis (ROW) or the summed
// axis' rows running along its own (COL), which the transposing reads turn. Copies go to LDS
// directly, the next step's while this one's products run.
#include "layer_dev.h"

namespace bgp {
namespace {

constexpr int kStep = 64;              // of the summed axis
constexpr int kStepBytes = 2 * kStep;

// R rows of an operand, copied by WAVES wavefronts.
template <bool COL, int R, int WAVES>
struct Side;

template <int R, int WAVES>
struct Side<false, R, WAVES> {
  static constexpr int kBytes = R * kStepBytes;
  TileCopy<64, R, WAVES> copy;
  TileReader<64> reader;
  const char *base;
  int64_t stride;
  int rows, wave, lane;

  // rows row0.. of a matrix of `all` rows
  __device__ void init(const char *p, int64_t row0, int64_t all, int64_t row_stride, int w, int l) {
    base = p + row0 * row_stride;
    stride = row_stride;
    rows = (int)max((int64_t)0, min((int64_t)R, all - row0));
    wave = w, lane = l;
    copy.init(wave, lane, (int)stride, kStepBytes);
    reader.init(lane);
  }
  // k0.. of k
  __device__ void start(int64_t k0, int64_t k, uint32_t lds) const {
    const int64_t left = 2 * (k - k0);
    if (left >= kStepBytes) {
      copy.start(row_buffer(base + 2 * k0, 0, rows, stride, kStepBytes), lds);
    } else {
      TileCopy<64, R, WAVES> tail;
      tail.init(wave, lane, (int)stride, (int)left);
      tail.start(row_buffer(base + 2 * k0, 0, rows, stride, (int)left), lds);
    }
  }
  __device__ uint32_t at(uint32_t lds) const { return TileReader<64>::at(lds, reader.row); }
  // rows 32 i.., k = 16 s ..
  static __device__ u32x4 operand(uint32_t x, int i, int s) { return row_operand<64>(x, 32 * i, s); }
};

template <int R, int WAVES>
struct Side<true, R, WAVES> {
  static constexpr int kBytes = R * kStepBytes, kParts = R / 128, kPart = kStep * 256;
  TileCopy<128, kStep, WAVES> copy[kParts];
  const char *base;
  int64_t stride;
  int bytes;
  uint32_t col;

  // its rows row0.. of `all` are the columns of a matrix with the summed axis along rows
  __device__ void init(const char *p, int64_t row0, int64_t all, int64_t row_stride, int wave, int lane) {
    base = p + 2 * row0;
    stride = row_stride;
    bytes = (int)max((int64_t)0, min((int64_t)R, all - row0)) * 2;
#pragma unroll
    for (int i = 0; i < kParts; ++i) copy[i].init(wave, lane, (int)stride, bytes - 256 * i);
    // the transposing reads of lane half h: the step's rows 16 s + 8 h + 0..3 and + 4..7, so that k
    // runs as in a ROW operand (a row's swizzle differs by one piece between the two)
    const int q = 8 * (lane >> 5) + ((lane & 15) >> 2);
    const int piece = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    col = q * 256 + (piece ^ swizzle<128>(q)) * 16 + (lane & 1) * 8;
  }
  __device__ void start(int64_t k0, int64_t k, uint32_t lds) const {
    const int rows = (int)min((int64_t)kStep, k - k0);
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
      const int b = min(256, bytes - 256 * i);
      copy[i].start(row_buffer(base + 256 * i, k0, b > 0 ? rows : 0, stride, b), lds + i * kPart);
    }
  }
  __device__ uint32_t at(uint32_t lds) const { return TileReader<128>::at(lds, col); }
  static __device__ u32x4 operand(uint32_t x, int i, int s) {
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const uint32_t y = (x ^ ((i & 3) * 64)) + (i >> 2) * kPart + s * (16 * 256);
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)y);
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)((y ^ 16) + 4 * 256));
    const u32x2 ua = __builtin_bit_cast(u32x2, a), ub = __builtin_bit_cast(u32x2, b);
    return u32x4{ua[0], ua[1], ub[0], ub[1]};
  }
};

// Runs steps first .. end - 1: start(step, stage) copies, compute(stage) multiplies.
template <class Start, class Compute>
__device__ inline void run_steps(int first, int end, Start start, Compute compute) {
  if (first < end) start(first, 0);
  for (int i = first; i < end; ++i) {
    const int stage = (i - first) & 1;
    copies_barrier();                  // this step's copies are there, the other stage has been read
    if (i + 1 < end) start(i + 1, stage ^ 1);
    compute(stage);
  }
}

// Tile of a block: neighbours in m share an XCD's cache for the n side, eight m tiles to a group.
struct Tile {
  int m, n;
};
__device__ inline Tile tile_of(unsigned block, unsigned blocks, int nm, int nn) {
  // blocks go round the 8 XCDs: each gets a run of tiles
  const unsigned per = blocks / 8, more = blocks % 8, x = block % 8;
  const unsigned i = x * per + min(x, more) + block / 8;
  constexpr unsigned kGroup = 8;
  const unsigned group = i / (kGroup * nn), in = i - group * kGroup * nn;
  const unsigned size = min(kGroup, nm - group * kGroup);
  return {(int)(group * kGroup + in % size), (int)(in / size)};
}

// ------------------------------------------------------------------ activations
constexpr int kSilu = 0, kGelu = 1;   // GP_SILU, GP_GELU

// act(z) and its derivative. gelu's normal distribution function is 1/2 erfc(-z / sqrt(2)), and
// erfc(x) = e^(-x^2) t q(t), t = 1 / (1 + 0.375 x), for x >= 0, q a least-maximum fit of degree 6
// with a relative error of 6.4e-7: the tail keeps its digits, and the derivative has the same
// exponential.
template <int ACT>
__device__ inline void activation(float z, float &a, float &d) {
  if (ACT == kSilu) {
    const float p = __builtin_amdgcn_rcpf(1.f + fast_exp2(-kLog2e * z));
    a = z * p;
    d = p + a * (1.f - p);
  } else {
    const float x = fabsf(z) * 0.70710678f;
    const float t = __builtin_amdgcn_rcpf(fmaf(0.375f, x, 1.f));
    float q = -0.13509515f;
    q = fmaf(q, t, 0.38793566f);
    q = fmaf(q, t, -0.12959506f);
    q = fmaf(q, t, 0.28306065f);
    q = fmaf(q, t, 0.16666456f);
    q = fmaf(q, t, 0.21568926f);
    q = fmaf(q, t, 0.21133943f);
    const float e = fast_exp2(z * z * (-0.5f * kLog2e));
    const float tail = 0.5f * e * t * q;
    const float p = z < 0.f ? tail : 1.f - tail;
    a = z * p;
    d = fmaf(z * e, 0.39894228f, p);
  }
}

// ------------------------------------------------------------------ both projections
// BM rows of x and BN / 2 hidden values per block, WM x WN wavefronts, each of 32 hidden values.
template <class T, int BM, int BN, int WM, int WN, int ACT, bool GRAD>
__global__ __launch_bounds__(64 * WM * WN, 2) void gated_kernel(GatedGradArgs g, char *dg, char *du,
                                                             int nm, int nn) {
  constexpr int W = WM * WN, TM = BM / 32 / WM;
  static_assert(BN / 2 == 32 * WN);
  extern __shared__ char stages[];
  constexpr int kHalf = BN / 2 * kStepBytes, kStage = (BM + BN) * kStepBytes;
  const GatedArgs &a = g.f;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int wm = wave / WN, wn = wave % WN;
  const Tile t = tile_of(blockIdx.x, gridDim.x, nm, nn);
  const int64_t m0 = (int64_t)t.m * BM, n0 = (int64_t)t.n * (BN / 2);
  Side<false, BN / 2, W> gate, up;
  Side<false, BM, W> x;
  gate.init(a.w_gate, n0, a.hidden, a.gate_row, wave, lane);
  up.init(a.w_up, n0, a.hidden, a.up_row, wave, lane);
  x.init(a.x, m0, a.rows, a.x_row, wave, lane);
  const uint32_t lds = lds_address(stages);
  f32x16 acc[2][TM];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j) acc[i][j] = f32x16{0.f};
  run_steps(
      0, (a.width + kStep - 1) / kStep,
      [&](int step, int stage) {
        const int64_t k0 = (int64_t)step * kStep;
        const uint32_t to = lds + stage * kStage;
        gate.start(k0, a.width, to);
        up.start(k0, a.width, to + kHalf);
        x.start(k0, a.width, to + 2 * kHalf);
      },
      [&](int stage) {
        const uint32_t at = lds + stage * kStage;
        const uint32_t pg = gate.at(at + wn * (32 * kStepBytes)), pu = pg + kHalf;
        const uint32_t px = x.at(at + 2 * kHalf + wm * (BM / WM * kStepBytes));
#pragma unroll
        for (int s = 0; s < kStep / 16; ++s) {
          const u32x4 og = gate.operand(pg, 0, s), ou = up.operand(pu, 0, s);
#pragma unroll
          for (int j = 0; j < TM; ++j) {
            const u32x4 ox = x.operand(px, j, s);
            acc[0][j] = T::mfma(og, ox, acc[0][j]);
            acc[1][j] = T::mfma(ou, ox, acc[1][j]);
          }
        }
      });
  const int64_t n = n0 + 32 * wn;
  const int bytes = (int)min((int64_t)64, 2 * (a.hidden - n));
#pragma unroll
  for (int j = 0; j < TM; ++j) {
    const int64_t row = m0 + wm * (BM / WM) + 32 * j + (lane & 31);
    const bool ok = row < a.rows;
    f32x16 u = acc[0][j], v = acc[1][j];
    if constexpr (GRAD) {
      const char *dy = g.dout + row * g.dout_row + 2 * n;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int off = (8 * q + 4 * (lane >> 5)) * 2;
        u32x2 w = {0, 0};
        if (ok && off < bytes) w = *reinterpret_cast<const u32x2 *>(dy + off);
        const uint32_t w0 = w[0], w1 = w[1];
        const float y[4] = {T::lo(w0), T::hi(w0), T::lo(w1), T::hi(w1)};
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float f, d;
          activation<ACT>(u[4 * q + r], f, d);
          u[4 * q + r] = y[r] * v[4 * q + r] * d;
          v[4 * q + r] = y[r] * f;
        }
      }
      const int64_t to = row * ((int64_t)a.hidden * 2) + 2 * n;
      store_row<T, 1>(dg + to, ok, bytes, &u, 1.f, lane);
      store_row<T, 1>(du + to, ok, bytes, &v, 1.f, lane);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float f, d;
        activation<ACT>(u[i], f, d);
        u[i] = f * v[i];
      }
      store_row<T, 1>(a.out + row * a.out_row + 2 * n, ok, bytes, &u, 1.f, lane);
    }
  }
}

// ------------------------------------------------------------------ the gradient's products
// out[m][n] = sum over k of B(m, k) A(n, k), A in COL form.
// SEGMENTS 2: one output, the summed axis in two segments of k each with operands of their own
// (dx). 1: two outputs with operands of their own (dWg and dWu).
struct ProductArgs {
  const char *a[2], *b[2];
  int64_t a_row[2], b_row[2];
  char *out[2];
  int64_t out_row[2];
  float *part;                         // [output][split][m][n] fp32, with splits
  int64_t m, n, k;
  int nm, nn, splits;
};

template <class T, int BM, int BN, int WM, int WN, bool B_COL, int SEGMENTS>
__global__ __launch_bounds__(64 * WM * WN, 2) void product_kernel(ProductArgs p) {
  constexpr int W = WM * WN, TM = BM / 32 / WM, TN = BN / 32 / WN;
  extern __shared__ char stages[];
  constexpr int kStage = (BM + BN) * kStepBytes, kA = BN * kStepBytes;
  typedef Side<true, BN, W> ASide;
  typedef Side<B_COL, BM, W> BSide;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int wm = wave / WN, wn = wave % WN;
  const int output = blockIdx.y, split = blockIdx.z;
  const Tile t = tile_of(blockIdx.x, gridDim.x, p.nm, p.nn);
  const int64_t m0 = (int64_t)t.m * BM, n0 = (int64_t)t.n * BN;
  const int per = (int)((p.k + kStep - 1) / kStep), all = per * SEGMENTS;
  const int first = (int)((int64_t)all * split / p.splits);
  const int end = (int)((int64_t)all * (split + 1) / p.splits);
  ASide a;
  BSide b;
  int segment = SEGMENTS == 2 ? (first >= per) : output;
  a.init(p.a[segment], n0, p.n, p.a_row[segment], wave, lane);
  b.init(p.b[segment], m0, p.m, p.b_row[segment], wave, lane);
  const uint32_t lds = lds_address(stages);
  f32x16 acc[TN][TM];
#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j) acc[i][j] = f32x16{0.f};
  run_steps(
      first, end,
      [&](int step, int stage) {
        if (SEGMENTS == 2 && step >= per) {
          if (!segment) {
            segment = 1;
            a.init(p.a[1], n0, p.n, p.a_row[1], wave, lane);
            b.init(p.b[1], m0, p.m, p.b_row[1], wave, lane);
          }
          step -= per;
        }
        const int64_t k0 = (int64_t)step * kStep;
        a.start(k0, p.k, lds + stage * kStage);
        b.start(k0, p.k, lds + stage * kStage + kA);
      },
      [&](int stage) {
        const uint32_t pa = a.at(lds + stage * kStage), pb = b.at(lds + stage * kStage + kA);
#pragma unroll
        for (int s = 0; s < kStep / 16; ++s) {
          u32x4 oa[TN];
#pragma unroll
          for (int i = 0; i < TN; ++i) oa[i] = a.operand(pa, wn * TN + i, s);
#pragma unroll
          for (int j = 0; j < TM; ++j) {
            const u32x4 ob = b.operand(pb, wm * TM + j, s);
#pragma unroll
            for (int i = 0; i < TN; ++i) acc[i][j] = T::mfma(oa[i], ob, acc[i][j]);
          }
        }
      });
#pragma unroll
  for (int j = 0; j < TM; ++j) {
    const int64_t row = m0 + wm * (BM / WM) + 32 * j + (lane & 31);
    const bool ok = row < p.m;
#pragma unroll
    for (int i = 0; i < TN; ++i) {
      const int64_t n = n0 + wn * (BN / WN) + 32 * i;
      if (p.splits == 1) {
        store_row<T, 1>(p.out[output] + row * p.out_row[output] + 2 * n, ok,
                        (int)min((int64_t)64, 2 * (p.n - n)), &acc[i][j], 1.f, lane);
      } else {
        float *to = p.part + (((int64_t)output * p.splits + split) * p.m + row) * p.n + n;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int off = 8 * q + 4 * (lane >> 5);
          if (ok && n + off < p.n)
            *reinterpret_cast<f32x4 *>(to + off) =
                f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        }
      }
    }
  }
}

// out = the sum of the splits' parts, 8 values a thread.
template <class T>
__global__ __launch_bounds__(256) void product_add(ProductArgs p) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8, size = p.m * p.n;
  if (i >= size) return;
  const float *from = p.part + (int64_t)blockIdx.y * p.splits * size + i;
  f32x4 x = *reinterpret_cast<const f32x4 *>(from), y = *reinterpret_cast<const f32x4 *>(from + 4);
  for (int s = 1; s < p.splits; ++s) {
    const f32x4 *q = reinterpret_cast<const f32x4 *>(from + s * size);
    x += q[0], y += q[1];
  }
  const int64_t row = i / p.n;
  *reinterpret_cast<u32x4 *>(p.out[blockIdx.y] + row * p.out_row[blockIdx.y] + 2 * (i - row * p.n)) =
      u32x4{T::pack(x[0], x[1]), T::pack(x[2], x[3]), T::pack(y[0], y[1]), T::pack(y[2], y[3])};
}

// ------------------------------------------------------------------ launches
int64_t tiles(int64_t n, int size) { return (n + size - 1) / size; }
size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

// Tiles of 256 x 256 where they fill the device, else of 128 x 128.
bool use_big(int64_t m, int64_t n, int outputs) {
  return tiles(m, 256) * tiles(n, 256) * outputs >= kSeqCus;
}

template <class T, int BM, int BN, int WM, int WN, int ACT, bool GRAD>
hipError_t launch_projections(const GatedGradArgs &g, char *dg, char *du, hipStream_t s) {
  constexpr int kLds = 2 * (BM + BN) * kStepBytes;
  static LdsLimit limit;
  const void *f = reinterpret_cast<const void *>(gated_kernel<T, BM, BN, WM, WN, ACT, GRAD>);
  const hipError_t e = limit.set(f, kLds);
  if (e != hipSuccess) return e;
  const int nm = (int)tiles(g.f.rows, BM), nn = (int)tiles(g.f.hidden, BN / 2);
  gated_kernel<T, BM, BN, WM, WN, ACT, GRAD>
      <<<(unsigned)(nm * nn), 64 * WM * WN, kLds, s>>>(g, dg, du, nm, nn);
  return hipGetLastError();
}
template <class T, int ACT, bool GRAD>
hipError_t projections(const GatedGradArgs &g, char *dg, char *du, hipStream_t s) {
  if (use_big(g.f.rows, 2 * (int64_t)g.f.hidden, 1))
    return launch_projections<T, 256, 256, 2, 4, ACT, GRAD>(g, dg, du, s);
  return launch_projections<T, 128, 128, 2, 2, ACT, GRAD>(g, dg, du, s);
}
template <bool GRAD>
hipError_t by_type(const GatedGradArgs &g, char *dg, char *du, hipStream_t s) {
  if (g.f.fp16)
    return g.f.act == kSilu ? projections<Fp16, kSilu, GRAD>(g, dg, du, s)
                            : projections<Fp16, kGelu, GRAD>(g, dg, du, s);
  return g.f.act == kSilu ? projections<Bf16, kSilu, GRAD>(g, dg, du, s)
                          : projections<Bf16, kGelu, GRAD>(g, dg, du, s);
}

// Parts of the summed axis (`steps` of it): so many that the tiles fill the device, each of 8
// steps at least.
int splits_of(int64_t m, int64_t n, int outputs, int64_t steps) {
  const bool big = use_big(m, n, outputs);
  const int size = big ? 256 : 128;
  const int64_t have = tiles(m, size) * tiles(n, size) * outputs, want = big ? kSeqCus : 2 * kSeqCus;
  return (int)std::max<int64_t>(1, std::min<int64_t>(want / std::max<int64_t>(have, 1), steps / 8));
}
int splits_dx(int64_t rows, int64_t width, int64_t hidden) {
  return splits_of(rows, width, 1, 2 * tiles(hidden, kStep));
}
int splits_dw(int64_t rows, int64_t width, int64_t hidden) {
  return splits_of(hidden, width, 2, tiles(rows, kStep));
}

template <class T, int BM, int BN, int WM, int WN, bool B_COL, int SEGMENTS>
hipError_t launch_product(ProductArgs p, hipStream_t s) {
  constexpr int kLds = 2 * (BM + BN) * kStepBytes, kOutputs = SEGMENTS == 2 ? 1 : 2;
  static LdsLimit limit;
  const void *f = reinterpret_cast<const void *>(product_kernel<T, BM, BN, WM, WN, B_COL, SEGMENTS>);
  hipError_t e = limit.set(f, kLds);
  if (e != hipSuccess) return e;
  p.nm = (int)tiles(p.m, BM), p.nn = (int)tiles(p.n, BN);
  product_kernel<T, BM, BN, WM, WN, B_COL, SEGMENTS>
      <<<dim3((unsigned)(p.nm * p.nn), kOutputs, p.splits), 64 * WM * WN, kLds, s>>>(p);
  e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  product_add<T><<<dim3((unsigned)tiles(p.m * p.n, 256 * 8), kOutputs), 256, 0, s>>>(p);
  return hipGetLastError();
}
template <class T, bool B_COL, int SEGMENTS>
hipError_t product(const ProductArgs &p, hipStream_t s) {
  if (use_big(p.m, p.n, SEGMENTS == 2 ? 1 : 2))
    return launch_product<T, 256, 256, 2, 4, B_COL, SEGMENTS>(p, s);
  return launch_product<T, 128, 128, 2, 2, B_COL, SEGMENTS>(p, s);
}

template <class T>
hipError_t gradient(const GatedGradArgs &g, char *ws, hipStream_t s) {
  const GatedArgs &f = g.f;
  const size_t hidden_bytes = align256((size_t)f.rows * f.hidden * 2);
  char *dg = ws, *du = ws + hidden_bytes;
  float *part = reinterpret_cast<float *>(ws + 2 * hidden_bytes);
  const int64_t row = (int64_t)f.hidden * 2;
  hipError_t e;
  if (f.rows > 0) {
    if ((e = by_type<true>(g, dg, du, s)) != hipSuccess) return e;
    ProductArgs x = {{f.w_gate, f.w_up}, {dg, du}, {f.gate_row, f.up_row}, {row, row}, {g.dx, nullptr},
                     {g.dx_row, 0}, part, f.rows, f.width, f.hidden, 0, 0,
                     splits_dx(f.rows, f.width, f.hidden)};
    if ((e = product<T, false, 2>(x, s)) != hipSuccess) return e;
  }
  ProductArgs w = {{f.x, f.x}, {dg, du}, {f.x_row, f.x_row}, {row, row}, {g.dw_gate, g.dw_up},
                   {g.dgate_row, g.dup_row}, part, f.hidden, f.width, f.rows, 0, 0,
                   splits_dw(f.rows, f.width, f.hidden)};
  return product<T, true, 1>(w, s);
}

}  // namespace

hipError_t launch_gated(const GatedArgs &a, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  GatedGradArgs g = {};
  g.f = a;
  return by_type<false>(g, nullptr, nullptr, s);
}

bool gated_fits(int64_t rows, int64_t width, int64_t hidden, bool grad) {
  // (the smallest tiles; at most 512 threads a block)
  constexpr int64_t kMost = kMaxBlocks / 2;
  bool ok = tiles(rows, 128) * tiles(hidden, 64) <= kMost;
  if (grad)
    ok = ok && tiles(rows, 128) * tiles(width, 128) <= kMost &&
         tiles(hidden, 128) * tiles(width, 128) * 2 <= kMost &&
         tiles(std::max(rows, hidden) * width, 256 * 8) <= kMost;
  return ok;
}

size_t gated_grad_bytes(int32_t rows, int32_t width, int32_t hidden) {
  const int sx = splits_dx(rows, width, hidden), sw = splits_dw(rows, width, hidden);
  const size_t px = sx > 1 ? (size_t)sx * rows * width * 4 : 0;
  const size_t pw = sw > 1 ? (size_t)2 * sw * hidden * width * 4 : 0;
  return 2 * align256((size_t)rows * hidden * 2) + align256(std::max(px, pw));
}

hipError_t launch_gated_grad(const GatedGradArgs &g, void *ws, hipStream_t s) {
  return g.f.fp16 ? gradient<Fp16>(g, static_cast<char *>(ws), s)
                  : gradient<Bf16>(g, static_cast<char *>(ws), s);
}

}  // namespace bgp
