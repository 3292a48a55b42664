// A step of AdamW over many tensors in one launch:
//   g = factor grad,  m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,
//   w = w - lr decay w - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps),
// in fp32 throughout; w is the master copy where there is one, and what is stored beside it is
// rounded from it.
//
// States in 8 bits: 256 values share a power of two, so that scaling rounds nothing. m is e4m3 and
// v e5m2 (v has no sign, but twice its exponent range), rounded to one of the two neighbours at
// random with the probabilities that keep their mean: rounded to the nearest, an average that moves
// by a thousandth of the way a step would never leave its code. Where that would do harm it is not
// random: an m below its smallest normal code goes to the nearest (a code taken by chance could be
// thousands of times the value, over a root of v just as small), and a v above 0 stays above 0.
//
// Bound by memory: every value is read and written once. A wavefront has a block of 256 values,
// four a lane; the tensors' table travels in the launch's arguments.
#include "layer_dev.h"

namespace bgp {
namespace {

constexpr int kShare = 256;            // values that share a scale: a wavefront's
constexpr int kWaves = 4;

// What a step's number and rate give: the averages' corrections.
__host__ __device__ inline AdamStep step_of(const AdamArgs &a, double t, double lr) {
  AdamStep s;
  s.lr_m = (float)(lr / (1.0 - pow(a.beta1, t)));
  s.root = (float)(1.0 / sqrt(1.0 - pow(a.beta2, t)));
  s.decay = (float)(lr * a.decay);
  return s;
}

// Philox4x32-10 (Salmon, Moraes, Dror, Shaw, SC 2011).
__device__ inline u32x4 philox(uint64_t quad, uint32_t t, uint32_t k0, uint32_t k1) {
  uint32_t c0 = (uint32_t)quad, c1 = (uint32_t)(quad >> 32), c2 = t, c3 = 0;
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t p = (uint64_t)0xD2511F53u * c0, q = (uint64_t)0xCD9E8D57u * c2;
    c0 = (uint32_t)(q >> 32) ^ c1 ^ k0;
    c1 = (uint32_t)q;
    c2 = (uint32_t)(p >> 32) ^ c3 ^ k1;
    c3 = (uint32_t)p;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return u32x4{c0, c1, c2, c3};
}

// The exponent of the largest magnitude of a block's values less `top`, -126 at least, as a power
// of two, and its inverse; 1 if all are 0. With a value that is not finite the scale is NaN, which
// makes the whole block NaN: codes have no such value.
__device__ inline void scale_of(float big, bool finite, int top, float &scale, float &inverse) {
  if (!finite) {
    scale = __builtin_nanf(""), inverse = 0.f;
  } else if (big == 0.f) {
    scale = inverse = 1.f;
  } else {
    const int k = max(ilogbf(big) - top, -126);
    scale = word_float((uint32_t)(k + 127) << 23);
    inverse = word_float((uint32_t)(127 - k) << 23);
  }
}

// The code of |x| on a grid of KEEP bits behind the leading one whose smallest normal number is
// 2^LOWEST: the upper neighbour if the place between the two, in 65536ths, and r reach 65536;
// below 2^LOWEST by `below` in r's place.
template <int KEEP, int LOWEST>
__device__ inline uint32_t code_of(float x, uint32_t r, uint32_t below) {
  constexpr int kLift = 23 - KEEP;
  if (x >= word_float((uint32_t)(LOWEST + 127) << 23))
    return ((__builtin_bit_cast(uint32_t, x) + (r << (kLift - 16))) >> kLift) -
           ((uint32_t)(LOWEST + 126) << KEEP);
  constexpr float kInv = (float)(1 << (KEEP - LOWEST));
  const float t = x * kInv, whole = floorf(t);           // (all of it exact)
  return (uint32_t)whole + (t - whole >= (float)(65536 - below) * (1.f / 65536.f));
}
// The value of a code.
template <int KEEP, int LOWEST>
__device__ inline float value_of(uint32_t code) {
  if (code >> KEEP) return word_float((code + ((uint32_t)(LOWEST + 126) << KEEP)) << (23 - KEEP));
  constexpr float kStep = 1.f / (float)(1 << (KEEP - LOWEST));
  return (float)code * kStep;
}

template <class T>
__device__ inline void load4(const void *p, int64_t i, bool whole, int left, float *v) {
  if (whole) {
    if constexpr (Piece<T>::kSize == 4) {
      Piece<T>::unpack(*reinterpret_cast<const u32x4_any *>(static_cast<const float *>(p) + i), v);
    } else {
      typedef u32x2 __attribute__((aligned(2))) pair;
      const u32x2 w = *reinterpret_cast<const pair *>(static_cast<const uint16_t *>(p) + i);
      const uint32_t a = w[0], b = w[1];
      v[0] = T::lo(a), v[1] = T::hi(a), v[2] = T::lo(b), v[3] = T::hi(b);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = k < left ? T::load(p, i + k) : 0.f;
  }
}
template <class T>
__device__ inline void store4(void *p, int64_t i, bool whole, int left, const float *v) {
  if (whole) {
    if constexpr (Piece<T>::kSize == 4) {
      *reinterpret_cast<u32x4_any *>(static_cast<float *>(p) + i) = Piece<T>::pack(v);
    } else {
      typedef u32x2 __attribute__((aligned(2))) pair;
      *reinterpret_cast<pair *>(static_cast<uint16_t *>(p) + i) =
          u32x2{T::pack(v[0], v[1]), T::pack(v[2], v[3])};
    }
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (k < left) T::store(p, i + k, v[k]);
  }
}
__device__ inline uint32_t load_codes(const void *p, int64_t i, bool whole, int left) {
  typedef uint32_t __attribute__((aligned(1))) word;
  const uint8_t *q = static_cast<const uint8_t *>(p) + i;
  if (whole) return *reinterpret_cast<const word *>(q);
  uint32_t w = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (k < left) w |= (uint32_t)q[k] << (8 * k);
  return w;
}
__device__ inline void store_codes(void *p, int64_t i, bool whole, int left, uint32_t w) {
  typedef uint32_t __attribute__((aligned(1))) word;
  uint8_t *q = static_cast<uint8_t *>(p) + i;
  if (whole) {
    *reinterpret_cast<word *>(q) = w;
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (k < left) q[k] = (uint8_t)(w >> (8 * k));
  }
}

// T: of the weights, G: of the gradients.
template <class T, class G, int BITS>
__global__ __launch_bounds__(64 * kWaves) void adamw_kernel(AdamArgs a, int64_t blocks) {
#pragma clang fp contract(off)
  __shared__ AdamStep shared;
  AdamStep s = a.s;
  if (a.step_dev || a.lr_dev) {        // (a power in 64 bits: once per block)
    if (threadIdx.x == 0)
      shared = step_of(a, (double)(a.step_dev ? *a.step_dev : a.step), a.lr_dev ? (double)*a.lr_dev : a.lr);
    __syncthreads();
    s = shared;
  }
  const float factor = a.factor ? *a.factor : 1.f;
  const float b1 = (float)a.beta1, c1 = (float)(1.0 - a.beta1);
  const float b2 = (float)a.beta2, c2 = (float)(1.0 - a.beta2), eps = (float)a.eps;
  const uint32_t step = (uint32_t)(a.step_dev ? *a.step_dev : a.step);
  const int lane = threadIdx.x % 64;
  int64_t b = (int64_t)blockIdx.x * kWaves + uniform(threadIdx.x / 64);
  for (; b < blocks; b += (int64_t)gridDim.x * kWaves) {
    // the tensor that has the block: the last one that starts at it or before
    int lo = 0, hi = a.n;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (a.t[mid].begin <= b) lo = mid;
      else hi = mid;
    }
    const AdamTensor t = a.t[uniform(lo)];
    const int64_t own = b - t.begin;
    const int64_t i = own * kShare + 4 * lane;
    const int left = (int)max((int64_t)0, min((int64_t)4, t.count - i));
    const bool whole = left == 4;
    float g[4], w[4], m[4], v[4];
    load4<G>(t.grad, i, whole, left, g);
    if (t.master) load4<Fp32>(t.master, i, whole, left, w);
    else load4<T>(t.param, i, whole, left, w);
    if constexpr (BITS == 32) {
      load4<Fp32>(t.m, i, whole, left, m);
      load4<Fp32>(t.v, i, whole, left, v);
    } else {
      const uint32_t cm = load_codes(t.m, i, whole, left), cv = load_codes(t.v, i, whole, left);
      const float sm = t.scales[2 * own], sv = t.scales[2 * own + 1];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t x = cm >> (8 * k) & 0xff, y = cv >> (8 * k) & 0xff;
        m[k] = value_of<3, -6>(x & 0x7f) * sm;
        m[k] = x & 0x80 ? -m[k] : m[k];
        v[k] = value_of<2, -14>(y & 0x7f) * sv;
      }
    }
    float big_m = 0.f, big_v = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      g[k] = g[k] * factor;
      m[k] = m[k] * b1 + g[k] * c1;
      v[k] = v[k] * b2 + g[k] * g[k] * c2;
      big_m = fmaxf(big_m, fabsf(m[k]));
      big_v = fmaxf(big_v, v[k]);
      w[k] = w[k] - w[k] * s.decay - m[k] * s.lr_m / (sqrtf(v[k]) * s.root + eps);
    }
    if (t.master) store4<Fp32>(t.master, i, whole, left, w);
    store4<T>(t.param, i, whole, left, w);
    if constexpr (BITS == 32) {
      store4<Fp32>(t.m, i, whole, left, m);
      store4<Fp32>(t.v, i, whole, left, v);
    } else {
      float sm, im, sv, iv;
      bool fm = true, fv = true;       // (fmaxf passes over a NaN)
#pragma unroll
      for (int k = 0; k < 4; ++k) fm &= fabsf(m[k]) < INFINITY, fv &= v[k] < INFINITY;
      scale_of(wave_max(big_m), __all(fm), 7, sm, im);
      scale_of(wave_max(big_v), __all(fv), 14, sv, iv);
      const u32x4 r = philox((t.first * kShare + (uint64_t)i) / 4, step, a.key0, a.key1);
      uint32_t cm = 0, cv = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t word = r[k];
        uint32_t x = code_of<3, -6>(fabsf(m[k]) * im, word & 0xffff, 32768);
        if (m[k] < 0.f) x |= 0x80;
        uint32_t y = code_of<2, -14>(v[k] * iv, word >> 16, word >> 16);
        if (v[k] > 0.f && y == 0) y = 1;
        cm |= (x & 0xff) << (8 * k);
        cv |= (y & 0xff) << (8 * k);
      }
      store_codes(t.m, i, whole, left, cm);
      store_codes(t.v, i, whole, left, cv);
      if (lane == 0) t.scales[2 * own] = sm, t.scales[2 * own + 1] = sv;
    }
  }
}

template <class T, class G>
void launch(AdamArgs a, int bits, hipStream_t s) {
  if (!a.step_dev && !a.lr_dev) a.s = step_of(a, (double)a.step, a.lr);
  int64_t blocks = 0;
  for (int i = 0; i < a.n; ++i) {
    a.t[i].begin = blocks;
    blocks += (a.t[i].count + kShare - 1) / kShare;
  }
  if (blocks == 0) return;
  const unsigned grid = (unsigned)std::min<int64_t>((blocks + kWaves - 1) / kWaves, 8 * kSeqCus);
  if (bits == 8) adamw_kernel<T, G, 8><<<grid, 64 * kWaves, 0, s>>>(a, blocks);
  else adamw_kernel<T, G, 32><<<grid, 64 * kWaves, 0, s>>>(a, blocks);
}

template <class T>
void by_gradient(const AdamArgs &a, int bits, hipStream_t s) {
  if (a.grad_dtype == GP_FP32) launch<T, Fp32>(a, bits, s);
  else launch<T, T>(a, bits, s);
}

}  // namespace

hipError_t launch_adamw(const AdamArgs &a, int bits, hipStream_t s) {
  if (a.dtype == GP_BF16) by_gradient<Bf16>(a, bits, s);
  else if (a.dtype == GP_FP16) by_gradient<Fp16>(a, bits, s);
  else launch<Fp32, Fp32>(a, bits, s);
  return hipGetLastError();
}

}  // namespace bgp
