// Norms of rows: h = x + residual rounded as it is stored, mean m (0 without centring),
// s = 1 / sqrt(mean((h - m)^2) + eps), xh = (h - m) s, out = xh w + b; and their gradient,
//   g = dout w,  dx = s (g - mean(g) - xh mean(g xh)) + dsum   (no mean(g) without centring),
//   dw = sum over rows of dout xh,  db = sum over rows of dout.
// All of it in fp32; the deviations are taken from the mean first and squared then.
//
// Bound by memory: a row is read once into registers, its sums are taken there, and it is written
// once (wider rows are read again, from the cache). The gradient's blocks keep their rows' dw and db in
// registers too, and a second kernel adds the blocks' sums in a fixed order. 16,384 rows of 1,024 in
// bf16 with a residual: 28.3 us forward (4.7 TB/s), 28.2 back and 4.6 for the sums.
#include "layer_dev.h"

namespace bgp {
namespace {

// The weights' values e.. of a row, of the rows' type or fp32; `fill` where there are none.
template <class T>
__device__ inline void load_weights(const void *w, int dtype, int e, int width, float fill, float *v) {
  constexpr int V = Piece<T>::kV;
  if (!w) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = fill;
  } else if (V == 8 && dtype == GP_FP32) {
#pragma unroll
    for (int i = 0; i < V; i += 4) load_piece<Fp32>(w, e + i, width, v + i);
  } else {
    load_piece<T>(w, e, width, v);
  }
}

// ------------------------------------------------------------------ forward
// THREADS threads per row (64: four rows a block), NC pieces of a row per thread.
template <class T, int THREADS, int NC>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void norm_rows(NormArgs a) {
  constexpr int V = Piece<T>::kV;
  constexpr int kPer = THREADS < 256 ? 256 / THREADS : 1;
  __shared__ float lds[16];
  const int t = threadIdx.x % THREADS;
  const float inv = 1.f / (float)a.width;
  const int64_t step = (int64_t)gridDim.x * kPer;
  for (int64_t r = (int64_t)blockIdx.x * kPer + threadIdx.x / THREADS; r < a.rows; r += step) {
    const char *x = row_at<T>(a.x, r);
    float h[NC][V];
#pragma unroll
    for (int c = 0; c < NC; ++c) load_piece<T>(x, (c * THREADS + t) * V, a.width, h[c]);
    if (a.residual.data) {
      const char *q = row_at<T>(a.residual, r);
      char *to = const_cast<char *>(row_at<T>(a.sum, r));
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        float y[V];
        load_piece<T>(q, (c * THREADS + t) * V, a.width, y);
#pragma unroll
        for (int i = 0; i < V; ++i) y[i] += h[c][i];
        // (what is normalised is the sum as it is stored, as with two calls one after the other:
        // the gradient reads it from there)
        u32x4 p = Piece<T>::pack(y);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t u = p[i];
          p[i] = as_stored(u);
        }
        Piece<T>::unpack(p, h[c]);
        store_piece<T>(to, (c * THREADS + t) * V, a.width, h[c]);
        if (NC > 2) __builtin_amdgcn_sched_barrier(0);     // (not all at once: registers)
      }
    }
    float m = 0.f;
    if (a.centre) {
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < V; ++i) m += h[c][i];
      m = group_sum<THREADS>(m, lds) * inv;
    }
    float v = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        h[c][i] -= m;
        v += (c * THREADS + t) * V + i < a.width ? h[c][i] * h[c][i] : 0.f;
      }
    v = group_sum<THREADS>(v, lds) * inv;
    const float s = 1.f / sqrtf(v + a.eps);
    if (a.stats && t == 0) a.stats[2 * r] = m, a.stats[2 * r + 1] = s;
    char *to = const_cast<char *>(row_at<T>(a.out, r));
    // (the weights come from the cache for each row: kept in registers, they would take the places of
    // wavefronts that have rows on their way)
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int e = (c * THREADS + t) * V;
      float w[V], b[V];
      load_weights<T>(a.weight, a.weight_dtype, e, a.width, 1.f, w);
      load_weights<T>(a.bias, a.weight_dtype, e, a.width, 0.f, b);
#pragma unroll
      for (int i = 0; i < V; ++i) h[c][i] = h[c][i] * s * w[i] + b[i];
      store_piece<T>(to, e, a.width, h[c]);
      if (NC > 2) __builtin_amdgcn_sched_barrier(0);
    }
  }
}

// Rows of any width, a block each, which read the row again for each of its passes.
constexpr int kWideThreads = 1024;
template <class T>
__global__ __launch_bounds__(kWideThreads) void norm_wide(NormArgs a) {
  constexpr int V = Piece<T>::kV;
  __shared__ float lds[16];
  const float inv = 1.f / (float)a.width;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const char *x = row_at<T>(a.x, r);
    float m = 0.f, v = 0.f;
    const int64_t step = kWideThreads * V;
    if (a.residual.data) {
      const char *q = row_at<T>(a.residual, r);
      char *to = const_cast<char *>(row_at<T>(a.sum, r));
      for (int64_t e = threadIdx.x * V; e < a.width; e += step) {
        float y[V], z[V];
        load_piece<T>(x, e, a.width, y);
        load_piece<T>(q, e, a.width, z);
#pragma unroll
        for (int i = 0; i < V; ++i) y[i] += z[i];
        store_piece<T>(to, e, a.width, y);
      }
      x = to;      // (each thread reads what it wrote itself)
    }
    if (a.centre) {
      for (int64_t e = threadIdx.x * V; e < a.width; e += step) {
        float y[V];
        load_piece<T>(x, e, a.width, y);
#pragma unroll
        for (int i = 0; i < V; ++i) m += y[i];
      }
      m = group_sum<kWideThreads>(m, lds) * inv;
    }
    for (int64_t e = threadIdx.x * V; e < a.width; e += step) {
      float y[V];
      load_piece<T>(x, e, a.width, y, m);
#pragma unroll
      for (int i = 0; i < V; ++i) v += (y[i] - m) * (y[i] - m);
    }
    v = group_sum<kWideThreads>(v, lds) * inv;
    const float s = 1.f / sqrtf(v + a.eps);
    if (a.stats && threadIdx.x == 0) a.stats[2 * r] = m, a.stats[2 * r + 1] = s;
    char *to = const_cast<char *>(row_at<T>(a.out, r));
    for (int64_t e = threadIdx.x * V; e < a.width; e += step) {
      float y[V];
      load_piece<T>(x, e, a.width, y);
      float w[V], b[V];
      load_weights<T>(a.weight, a.weight_dtype, e, a.width, 1.f, w);
      load_weights<T>(a.bias, a.weight_dtype, e, a.width, 0.f, b);
#pragma unroll
      for (int i = 0; i < V; ++i) y[i] = (y[i] - m) * s * w[i] + b[i];
      store_piece<T>(to, e, a.width, y);
    }
  }
}

// ------------------------------------------------------------------ gradient
template <class T, int THREADS, int NC>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void norm_grad_rows(NormGradArgs a) {
  constexpr int V = Piece<T>::kV;
  constexpr int kPer = THREADS < 256 ? 256 / THREADS : 1;
  __shared__ float lds[16];
  __shared__ float acc[kPer > 1 ? 2 * NC * THREADS * V : 1];
  const int t = threadIdx.x % THREADS, row0 = threadIdx.x / THREADS;
  float w[NC][V], dw[NC][V], db[NC][V];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    load_weights<T>(a.weight, a.weight_dtype, (c * THREADS + t) * V, a.width, 1.f, w[c]);
#pragma unroll
    for (int i = 0; i < V; ++i) dw[c][i] = db[c][i] = 0.f;
  }
  const float inv = 1.f / (float)a.width;
  const int64_t step = (int64_t)gridDim.x * kPer;
  for (int64_t r = (int64_t)blockIdx.x * kPer + row0; r < a.rows; r += step) {
    const char *h = row_at<T>(a.h, r), *dy = row_at<T>(a.dout, r);
    const float m = a.stats[2 * r], s = a.stats[2 * r + 1];
    float xh[NC][V], g[NC][V];
    float sg = 0.f, sx = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      load_piece<T>(h, (c * THREADS + t) * V, a.width, xh[c], m);
      load_piece<T>(dy, (c * THREADS + t) * V, a.width, g[c]);
    }
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        xh[c][i] = (xh[c][i] - m) * s;
        dw[c][i] += g[c][i] * xh[c][i];
        db[c][i] += g[c][i];
        g[c][i] *= w[c][i];
        sg += g[c][i];
        sx += g[c][i] * xh[c][i];
      }
    sg = a.centre ? group_sum<THREADS>(sg, lds) * inv : 0.f;
    sx = group_sum<THREADS>(sx, lds) * inv;
    char *to = const_cast<char *>(row_at<T>(a.dx, r));
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int e = (c * THREADS + t) * V;
      float y[V];
#pragma unroll
      for (int i = 0; i < V; ++i) y[i] = (g[c][i] - sg - xh[c][i] * sx) * s;
      if (a.dsum.data) {
        float z[V];
        load_piece<T>(row_at<T>(a.dsum, r), e, a.width, z);
#pragma unroll
        for (int i = 0; i < V; ++i) y[i] += z[i];
      }
      store_piece<T>(to, e, a.width, y);
    }
  }
  if (!a.part) return;
  // the block's sums: of its rows' wavefronts one after another
  if constexpr (kPer > 1) {
    constexpr int kHalf = NC * THREADS * V;
    for (int k = 0; k < kPer; ++k) {
      if (row0 == k)
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const int e = (c * V + i) * THREADS + t;
            acc[e] = k ? acc[e] + dw[c][i] : dw[c][i];
            acc[kHalf + e] = k ? acc[kHalf + e] + db[c][i] : db[c][i];
          }
      __syncthreads();
    }
    if (row0) return;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int e = (c * V + i) * THREADS + t;
        dw[c][i] = acc[e], db[c][i] = acc[kHalf + e];
      }
  }
  float *to = a.part + (int64_t)blockIdx.x * 2 * a.width;
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      store_piece<Fp32>(to, (c * THREADS + t) * V + i, a.width, dw[c] + i);
      store_piece<Fp32>(to + a.width, (c * THREADS + t) * V + i, a.width, db[c] + i);
    }
}

// Wide rows: the means of g and g xh of each row, a block each ...
template <class T>
__global__ __launch_bounds__(kWideThreads) void norm_grad_sums(NormGradArgs a) {
  constexpr int V = Piece<T>::kV;
  __shared__ float lds[16];
  const float inv = 1.f / (float)a.width;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const char *h = row_at<T>(a.h, r), *dy = row_at<T>(a.dout, r);
    const float m = a.stats[2 * r], s = a.stats[2 * r + 1];
    float sg = 0.f, sx = 0.f;
    for (int64_t e = threadIdx.x * V; e < a.width; e += kWideThreads * V) {
      float x[V], g[V], w[V];
      load_piece<T>(h, e, a.width, x, m);
      load_piece<T>(dy, e, a.width, g);
      load_weights<T>(a.weight, a.weight_dtype, e, a.width, 1.f, w);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        g[i] *= w[i];
        sg += g[i];
        sx += g[i] * ((x[i] - m) * s);
      }
    }
    sg = a.centre ? group_sum<kWideThreads>(sg, lds) * inv : 0.f;
    sx = group_sum<kWideThreads>(sx, lds) * inv;
    if (threadIdx.x == 0) a.sums[2 * r] = sg, a.sums[2 * r + 1] = sx;
  }
}

// ... then strips of columns, over the rows of a block (blockIdx.y of gridDim.y).
template <class T>
__global__ __launch_bounds__(256) void norm_grad_strips(NormGradArgs a) {
  constexpr int V = Piece<T>::kV;
  const int64_t e = ((int64_t)blockIdx.x * 256 + threadIdx.x) * V;
  if (e >= a.width) return;
  float w[V], dw[V], db[V];
  load_weights<T>(a.weight, a.weight_dtype, e, a.width, 1.f, w);
#pragma unroll
  for (int i = 0; i < V; ++i) dw[i] = db[i] = 0.f;
  for (int64_t r = blockIdx.y; r < a.rows; r += gridDim.y) {
    float x[V], g[V], z[V];
    load_piece<T>(row_at<T>(a.h, r), e, a.width, x);
    load_piece<T>(row_at<T>(a.dout, r), e, a.width, g);
    if (a.dsum.data) load_piece<T>(row_at<T>(a.dsum, r), e, a.width, z);
    const float m = a.stats[2 * r], s = a.stats[2 * r + 1], sg = a.sums[2 * r], sx = a.sums[2 * r + 1];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float xh = (x[i] - m) * s;
      dw[i] += g[i] * xh;
      db[i] += g[i];
      x[i] = (g[i] * w[i] - sg - xh * sx) * s + (a.dsum.data ? z[i] : 0.f);
    }
    store_piece<T>(const_cast<char *>(row_at<T>(a.dx, r)), e, a.width, x);
  }
  if (!a.part) return;
  float *to = a.part + (int64_t)blockIdx.y * 2 * a.width;
#pragma unroll
  for (int i = 0; i < V; i += 4) {
    store_piece<Fp32>(to, e + i, a.width, dw + i);
    store_piece<Fp32>(to + a.width, e + i, a.width, db + i);
  }
}

// dw and db: the blocks' sums, 32 columns a block, 32 groups of threads of which each adds every 32nd.
constexpr int kAddColumns = 32;
__global__ __launch_bounds__(1024) void norm_grad_add(const float *part, int64_t parts, int width,
                                                      void *dweight, void *dbias, int dtype) {
  __shared__ float lds[32][kAddColumns + 1];
  const int col = threadIdx.x % kAddColumns, k0 = threadIdx.x / kAddColumns;
  const int64_t e = (int64_t)blockIdx.x * kAddColumns + col;
  void *to = blockIdx.y ? dbias : dweight;
  if (!to) return;
  float s = 0.f;
  if (e < width)
#pragma unroll 8
    for (int64_t k = k0; k < parts; k += 32) s += part[(2 * k + blockIdx.y) * width + e];
  lds[k0][col] = s;
  __syncthreads();
  if (k0 || e >= width) return;
  s = 0.f;
#pragma unroll
  for (int k = 0; k < 32; ++k) s += lds[k][col];
  store_any(dtype, to, e, s);
}

// ------------------------------------------------------------------ launches
// Threads per row and pieces per thread: the fewest threads that have no more pieces each than `most` (of
// 64, 256, 512 and 1024 threads). nc 0: the wide form.
struct Shape {
  int threads, nc;
};
constexpr int kThreads[4] = {64, 256, 512, 1024};
struct Most {
  int n[4];
};
// As many as registers have room for: 16,384 entries of 16 bits, 24,576 of fp32. (10,007 of fp32, 1,021 rows:
// 23.7 us forward and 28.5 back with 1024 threads; 24.9 and 33.7 with 512, five pieces each.)
template <class T>
constexpr Most kMostForward = Piece<T>::kV == 8 ? Most{{2, 2, 4, 0}} : Most{{4, 4, 4, 6}};
// (a gradient's block also keeps its sums of the weights' gradients in registers)
template <class T>
constexpr Most kMostGrad = Piece<T>::kV == 8 ? Most{{2, 2, 2, 2}} : Most{{4, 4, 4, 4}};
Shape shape_of(int64_t pieces, const Most &most) {
  for (int k = 0; k < 4; ++k) {
    const int64_t nc = (pieces + kThreads[k] - 1) / kThreads[k];
    if (nc <= most.n[k]) return {kThreads[k], (int)nc};
  }
  return {kWideThreads, 0};
}

int64_t pieces_of(int width, int dtype) {
  const int v = dtype == GP_FP32 ? 4 : 8;
  return ((int64_t)width + v - 1) / v;
}

int64_t row_blocks(const Shape &f, int64_t rows) {
  return f.threads == 64 ? (rows + 3) / 4 : rows;
}

// Blocks of a gradient's launch, which loops over its rows: as many as are resident at once. (16,384 rows of
// 1,024: 28.2 us with four of 256 threads a compute unit, 32.5 with three, 41.6 with two.)
int64_t resident(const Shape &f) {
  return (int64_t)kSeqCus * (f.threads == 1024 ? 1 : f.threads == 512 ? 2 : 4);
}

// f<threads, nc>() of a shape: those that shape_of gives, from the next smaller number of threads' last on.
template <class M, M &MOST, int K = 0, int NC = 1, class F>
void by_shape(const Shape &h, F f) {
  if constexpr (K < 4) {
    if constexpr (NC > MOST.n[K]) {
      constexpr int kNext = K < 3 ? K + 1 : K;
      by_shape<M, MOST, K + 1, K < 3 ? (MOST.n[K] * kThreads[K] + kThreads[kNext]) / kThreads[kNext] : 1>(h, f);
    } else if (h.threads == kThreads[K] && h.nc == NC) {
      f.template operator()<kThreads[K], NC>();
    } else {
      by_shape<M, MOST, K, NC + 1>(h, f);
    }
  }
}
Shape grad_shape(const NormGradArgs &a) {
  return shape_of(pieces_of(a.width, a.dtype), a.dtype == GP_FP32 ? kMostGrad<Fp32> : kMostGrad<Bf16>);
}

template <class T>
struct Forward {
  const NormArgs &a;
  unsigned blocks;
  hipStream_t s;
  template <int THREADS, int NC>
  void operator()() const {
    norm_rows<T, THREADS, NC><<<blocks, THREADS < 256 ? 256 : THREADS, 0, s>>>(a);
  }
};
template <class T>
struct Backward {
  const NormGradArgs &a;
  unsigned blocks;
  hipStream_t s;
  template <int THREADS, int NC>
  void operator()() const {
    norm_grad_rows<T, THREADS, NC><<<blocks, THREADS < 256 ? 256 : THREADS, 0, s>>>(a);
  }
};

template <class T>
void forward(const NormArgs &a, hipStream_t s) {
  const Shape f = shape_of(pieces_of(a.width, a.dtype), kMostForward<T>);
  const int64_t blocks = std::min(row_blocks(f, a.rows), kMaxBlocks / 4);
  if (!f.nc) norm_wide<T><<<(unsigned)std::min<int64_t>(a.rows, 2 * kSeqCus), kWideThreads, 0, s>>>(a);
  else by_shape<const Most, kMostForward<T>>(f, Forward<T>{a, (unsigned)blocks, s});
}

// Blocks that add up rows: of the row form, or the row groups of the strips.
int64_t grad_parts(const NormGradArgs &a, const Shape &f) {
  if (a.rows == 0) return 0;
  if (f.nc) return std::min(row_blocks(f, a.rows), resident(f));
  const int64_t strips = (pieces_of(a.width, a.dtype) + 255) / 256;
  return std::min<int64_t>(a.rows, std::max<int64_t>(1, 4 * kSeqCus / strips));
}

template <class T>
void backward(const NormGradArgs &a, const Shape &f, int64_t parts, hipStream_t s) {
  if (f.nc) {
    by_shape<const Most, kMostGrad<T>>(f, Backward<T>{a, (unsigned)parts, s});
    return;
  }
  const int64_t strips = (pieces_of(a.width, a.dtype) + 255) / 256;
  norm_grad_sums<T><<<(unsigned)std::min<int64_t>(a.rows, 2 * kSeqCus), kWideThreads, 0, s>>>(a);
  norm_grad_strips<T><<<dim3((unsigned)strips, (unsigned)parts), 256, 0, s>>>(a);
}

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

}  // namespace

hipError_t launch_norm(const NormArgs &a, hipStream_t s) {
  if (a.dtype == GP_BF16) forward<Bf16>(a, s);
  else if (a.dtype == GP_FP16) forward<Fp16>(a, s);
  else forward<Fp32>(a, s);
  return hipGetLastError();
}

size_t norm_grad_bytes(const NormGradArgs &a) {
  const Shape f = grad_shape(a);
  size_t n = 0;
  if (a.dweight || a.dbias) n += align256((size_t)grad_parts(a, f) * 2 * a.width * 4);
  if (!f.nc) n += align256((size_t)a.rows * 8);
  return n;
}

hipError_t launch_norm_grad(NormGradArgs a, void *ws, hipStream_t s) {
  const Shape f = grad_shape(a);
  const int64_t parts = grad_parts(a, f);
  char *at = static_cast<char *>(ws);
  const bool sums = a.dweight || a.dbias;
  a.part = sums ? reinterpret_cast<float *>(at) : nullptr;
  if (sums) at += align256((size_t)parts * 2 * a.width * 4);
  a.sums = reinterpret_cast<float *>(at);
  if (a.rows > 0) {
    if (a.dtype == GP_BF16) backward<Bf16>(a, f, parts, s);
    else if (a.dtype == GP_FP16) backward<Fp16>(a, f, parts, s);
    else backward<Fp32>(a, f, parts, s);
  }
  if (sums)
    norm_grad_add<<<dim3((unsigned)((a.width + kAddColumns - 1) / kAddColumns), 2), 1024, 0, s>>>(
        a.part, parts, a.width, a.dweight, a.dbias, a.weight_dtype);
  return hipGetLastError();
}

}  // namespace bgp
