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

// A block has `per` rows at a time, and their heads, of all parts, in pieces: with pairs (i, i + half) V
// values of either half, or V values behind the rotated part; interleaved V values, which are whole
// pairs. A thread keeps its piece of a head and goes through the heads; that there are many
// wavefronts keeps memory busy (2, 4 and 8 heads on a thread's way at once: 142, 159 and 190 us for 131,072 rows
// of 20 heads of 64 values in fp16, 32 of them rotated and interleaved, one 140: 4.8 TB/s; 190 too where a
// piece of interleaved pairs was two of V values, an instruction's loads 32 bytes apart).
template <class T, int V, bool INTERLEAVED>
__global__ __launch_bounds__(kRotateThreads) void rotate_kernel(RotateArgs a, int per) {
  constexpr int kSize = Piece<T>::kSize;
  struct alignas(V * kSize) Vec {
    char b[V * kSize];
  };
  __shared__ alignas(16) float cosine[kTable];
  __shared__ alignas(16) float sine[kTable];
  const int half = a.rotated / 2;
  const int turning = INTERLEAVED ? a.rotated / V : half / V;
  const int pieces = turning + (a.dim - a.rotated) / V, places = kRotateThreads / pieces;
  const int heads = a.part[0].heads + a.part[1].heads + a.part[2].heads;
  const int piece = threadIdx.x % pieces, place = threadIdx.x / pieces;
  // values e0.. and, with the halves apart, e1.. of a head
  const bool turns = piece < turning;
  const int e0 = turns ? V * piece : a.rotated + V * (piece - turning), e1 = e0 + half;
  const int angle = INTERLEAVED ? V / 2 * piece : V * piece;
  for (int64_t row0 = (int64_t)blockIdx.x * per; row0 < a.rows; row0 += (int64_t)gridDim.x * per) {
    const int rows = (int)min((int64_t)per, a.rows - row0);
    __syncthreads();                     // (the table before has been read)
    for (int i = threadIdx.x; i < rows * half; i += kRotateThreads) {
      const int r = i / half;
      const double turned = (double)a.positions[row0 + r] * a.turns[i - r * half];
      // in half turns: -1 .. 1
      const float t = (float)(2.0 * (turned - rint(turned)));
      float s, c;
      sincospif(t, &s, &c);
      cosine[i] = a.magnitude * c;
      sine[i] = a.magnitude * (a.inverse ? -s : s);
    }
    __syncthreads();
    if (place >= places) continue;
    int r = 0;
    for (int head = place;; head += places) {
      while (head >= heads) head -= heads, ++r;
      if (r >= rows) break;
      int h = head, p = 0;
      while (h >= a.part[p].heads) h -= a.part[p++].heads;
      const RotateArgs::Part &q = a.part[p];
      const int64_t row = row0 + r, to = p > 0 ? a.slots[row] : row;
      if (p > 0 && (to < 0 || to >= a.slot_rows)) continue;
      const char *x = q.in + row * q.in_row + h * q.in_head;
      char *y = q.out + to * q.out_row + h * q.out_head;
      Vec u = *reinterpret_cast<const Vec *>(x + e0 * kSize), w = u;
      if (!INTERLEAVED && turns) w = *reinterpret_cast<const Vec *>(x + e1 * kSize);
      if (turns && p < 2) {
        const float *c = cosine + r * half + angle, *s = sine + r * half + angle;
#pragma unroll
        for (int i = 0; i < (INTERLEAVED ? V / 2 : V); ++i) {
          const float f = T::load(u.b, INTERLEAVED ? 2 * i : i);
          const float g = INTERLEAVED ? T::load(u.b, 2 * i + 1) : T::load(w.b, i);
          T::store(u.b, INTERLEAVED ? 2 * i : i, f * c[i] - g * s[i]);
          if (INTERLEAVED) T::store(u.b, 2 * i + 1, f * s[i] + g * c[i]);
          else T::store(w.b, i, f * s[i] + g * c[i]);
        }
      }
      *reinterpret_cast<Vec *>(y + e0 * kSize) = u;
      if (!INTERLEAVED && turns) *reinterpret_cast<Vec *>(y + e1 * kSize) = w;
    }
  }
}

template <class T, int V, bool INTERLEAVED>
void launch(const RotateArgs &a, hipStream_t s) {
  // rows of a block: as many as its table has places for, fewer where that leaves the device idle
  const int64_t fill = std::max<int64_t>(1, a.rows / (2 * kSeqCus));
  const int per = (int)std::min<int64_t>(kTable / (a.rotated / 2), fill);
  const unsigned blocks = (unsigned)std::min<int64_t>(((int64_t)a.rows + per - 1) / per, kMaxBlocks);
  rotate_kernel<T, V, INTERLEAVED><<<blocks, kRotateThreads, 0, s>>>(a, per);
}

// The widest pieces that divide both parts of a head (and, with the halves apart, the rotated one's half).
template <class T>
void by_width(const RotateArgs &a, hipStream_t s) {
  constexpr int V = Piece<T>::kV;
  if (a.interleaved) {
    const int n = a.rotated | (a.dim - a.rotated);
    if (n % V == 0) launch<T, V, true>(a, s);
    else if (n % 4 == 0) launch<T, 4, true>(a, s);
    else launch<T, 2, true>(a, s);
    return;
  }
  const int n = (a.rotated / 2) | (a.dim - a.rotated);
  if (n % V == 0) launch<T, V, false>(a, s);
  else if (n % 4 == 0) launch<T, 4, false>(a, s);
  else if (n % 2 == 0) launch<T, 2, false>(a, s);
  else launch<T, 1, false>(a, s);
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
