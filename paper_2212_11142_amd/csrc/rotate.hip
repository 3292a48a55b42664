// Rotary positions: pair i of a head's rotated part, (i, i + n/2) or (2i, 2i + 1), turns by
// pos f_i: (a, b) -> magnitude (a cos - b sin, a sin + b cos); the other way for the gradient,
// which is the transposed map. What is behind the rotated part is copied.
//
// Bound by memory: each head is read and written once. The angle is taken in turns, as a product
// in 64 bits whose whole turns are dropped there, so that far positions lose none of its digits;
// sines and cosines of a block's rows are computed once for all their heads and kept in LDS.
#include "layer_dev.h"

namespace bgp {
namespace {

constexpr int kRotateThreads = 256;
constexpr int kTable = kRotateThreads; // pairs of a block's rows at most

// A block has `per` rows at a time. Items of a row: the heads of all parts, each in pieces of V pairs (and
// V values behind the rotated part); V divides rotated / 2 and dim - rotated.
template <class T, int V, bool INTERLEAVED>
__global__ __launch_bounds__(kRotateThreads) void rotate_kernel(RotateArgs a, int per) {
  constexpr int kSize = Piece<T>::kSize;
  __shared__ float cosine[kTable], sine[kTable];
  const int half = a.rotated / 2;
  const int turning = half / V, pieces = turning + (a.dim - a.rotated) / V;
  const int heads = a.part[0].heads + a.part[1].heads + a.part[2].heads;
  for (int64_t row0 = (int64_t)blockIdx.x * per; row0 < a.rows; row0 += (int64_t)gridDim.x * per) {
    const int rows = (int)min((int64_t)per, a.rows - row0);
    __syncthreads();                     // (the table before has been read)
    for (int i = threadIdx.x; i < rows * half; i += kRotateThreads) {
      const int r = i / half;
      const double turns = (double)a.positions[row0 + r] * a.turns[i - r * half];
      // in half turns: -1 .. 1
      const float t = (float)(2.0 * (turns - rint(turns)));
      float s, c;
      sincospif(t, &s, &c);
      cosine[i] = a.magnitude * c;
      sine[i] = a.magnitude * (a.inverse ? -s : s);
    }
    __syncthreads();
    const int items = rows * heads * pieces;
    for (int i = threadIdx.x; i < items; i += kRotateThreads) {
      const int piece = i % pieces;
      int head = i / pieces;
      const int r = head / heads;
      head -= r * heads;
      int p = 0;
      while (head >= a.part[p].heads) head -= a.part[p++].heads;
      const RotateArgs::Part &q = a.part[p];
      int64_t to = row0 + r;
      if (p > 0) {
        to = a.slots[to];
        if (to < 0 || to >= a.slot_rows) continue;
      }
      const char *x = q.in + (row0 + r) * q.in_row + head * q.in_head;
      char *y = q.out + to * q.out_row + head * q.out_head;
      struct alignas(V * kSize) Vec {
        char b[V * kSize];
      };
      auto at = [&](int e) { return *reinterpret_cast<const Vec *>(x + e * kSize); };
      auto put = [&](int e, const Vec &v) { *reinterpret_cast<Vec *>(y + e * kSize) = v; };
      if (piece >= turning) {
        const int e = a.rotated + (piece - turning) * V;
        put(e, at(e));
        continue;
      }
      const int e0 = INTERLEAVED ? 2 * V * piece : V * piece, e1 = INTERLEAVED ? e0 + V : e0 + half;
      Vec u = at(e0), w = at(e1);
      if (p < 2) {
        const float *c = cosine + r * half + piece * V, *s = sine + r * half + piece * V;
        Vec ou, ow;
#pragma unroll
        for (int k = 0; k < V; ++k) {
          const Vec &fa = INTERLEAVED && 2 * k >= V ? w : u, &fb = INTERLEAVED && 2 * k + 1 < V ? u : w;
          const float va = T::load(fa.b, INTERLEAVED ? 2 * k % V : k);
          const float vb = T::load(fb.b, INTERLEAVED ? (2 * k + 1) % V : k);
          Vec &ga = INTERLEAVED && 2 * k >= V ? ow : ou, &gb = INTERLEAVED && 2 * k + 1 < V ? ou : ow;
          T::store(ga.b, INTERLEAVED ? 2 * k % V : k, va * c[k] - vb * s[k]);
          T::store(gb.b, INTERLEAVED ? (2 * k + 1) % V : k, va * s[k] + vb * c[k]);
        }
        u = ou, w = ow;
      }
      put(e0, u);
      put(e1, w);
    }
  }
}

template <class T, int V>
void launch(const RotateArgs &a, hipStream_t s) {
  const int half = a.rotated / 2;
  // rows of a block: as many as its table has places for, fewer where that leaves the device idle
  const int64_t fill = std::max<int64_t>(1, a.rows / (2 * kSeqCus));
  const int per = (int)std::min<int64_t>(kTable / half, fill);
  const unsigned blocks = (unsigned)std::min<int64_t>(((int64_t)a.rows + per - 1) / per, kMaxBlocks);
  if (a.interleaved) rotate_kernel<T, V, true><<<blocks, kRotateThreads, 0, s>>>(a, per);
  else rotate_kernel<T, V, false><<<blocks, kRotateThreads, 0, s>>>(a, per);
}

template <class T>
void by_width(const RotateArgs &a, hipStream_t s) {
  const int n = (a.rotated / 2) | (a.dim - a.rotated);
  constexpr int V = Piece<T>::kV;
  if (n % V == 0) launch<T, V>(a, s);
  else if (n % 4 == 0) launch<T, 4>(a, s);
  else if (n % 2 == 0) launch<T, 2>(a, s);
  else launch<T, 1>(a, s);
}

}  // namespace

hipError_t launch_rotate(const RotateArgs &a, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  if (a.dtype == GP_BF16) by_width<Bf16>(a, s);
  else if (a.dtype == GP_FP16) by_width<Fp16>(a, s);
  else by_width<Fp32>(a, s);
  return hipGetLastError();
}

}  // namespace bgp
