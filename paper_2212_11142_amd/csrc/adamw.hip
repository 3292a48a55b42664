// A step of AdamW over many tensors in one launch:
//   g = factor grad,  m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,
//   w = w - lr decay w - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps),
// in fp32 throughout; w is the master copy where there is one, and what is stored beside it is
// rounded from it.
//
// States in 8 bits: 256 values share a power of two, so that scaling rounds nothing. m is e4m3 and
// v e5m2 (v has no sign, but twice its exponent range), rounded to one of the two neighbours at
// random with the probabilities that keep their mean: rounded to the nearest, an average that moves
// by a thousandth of the way a step would never leave its code, and one below the smallest normal
// codes, whose gradient has ended, would never reach 0 while v goes on falling beneath it. Where
// chance would do harm there is none: a v above 0 stays above 0, so that an m of its lowest code
// (2^-16 of the largest's) stands over a root of 2^-15 of the largest's at least, and an m below an
// eighth of its lowest code is 0.
//
// Bound by memory: every value is read and written once. A wavefront has 256 values, four a lane, or
// with 8-bit states two blocks of 256, eight a lane (four a lane, 4 bytes of codes each: 233 us instead of
// 228 for 63.5 M weights with master copies); the tensors' table travels in the launch's arguments.
#include "layer_dev.h"

namespace bgp {
namespace {

constexpr int kShare = 256;            // values that share a scale
constexpr int kWaves = 4;
constexpr float kLeast = 1.f / 4096;   // scaled m that are rounded at random: an eighth of the lowest code on
// Values of a lane.
template <int BITS>
constexpr int kLane = BITS == 8 ? 8 : 4;

// Largest value of a lane's half wavefront.
__device__ inline float half_max(float x) {
  x = fmaxf(x, moved<0xb1>(x));
  x = fmaxf(x, moved<0x4e>(x));
  x = fmaxf(x, moved<0x141>(x));
  x = fmaxf(x, moved<0x140>(x));
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const u32x2 r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return fmaxf(word_float(r[0]), word_float(r[1]));
}

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
// 2^LOWEST: the upper neighbour if the place between the two, in 65536ths, and r reach 65536.
template <int KEEP, int LOWEST>
__device__ inline uint32_t code_of(float x, uint32_t r) {
  constexpr int kLift = 23 - KEEP;
  if (x >= word_float((uint32_t)(LOWEST + 127) << 23))
    return ((__builtin_bit_cast(uint32_t, x) + (r << (kLift - 16))) >> kLift) -
           ((uint32_t)(LOWEST + 126) << KEEP);
  constexpr float kInv = (float)(1 << (KEEP - LOWEST));
  const float t = x * kInv, whole = floorf(t);           // (all of it exact)
  return (uint32_t)whole + (t - whole >= (float)(65536 - r) * (1.f / 65536.f));
}
// The value of a code.
template <int KEEP, int LOWEST>
__device__ inline float value_of(uint32_t code) {
  if (code >> KEEP) return word_float((code + ((uint32_t)(LOWEST + 126) << KEEP)) << (23 - KEEP));
  constexpr float kStep = 1.f / (float)(1 << (KEEP - LOWEST));
  return (float)code * kStep;
}

// The N values (4 or 8) from i on, of which `left` are the tensor's.
template <class T, int N>
__device__ inline void load_values(const void *p, int64_t i, int left, float *v) {
  const char *q = static_cast<const char *>(p) + i * Piece<T>::kSize;
  if (left < N) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = k < left ? T::load(q, k) : 0.f;
  } else if constexpr (Piece<T>::kV <= N) {
#pragma unroll
    for (int k = 0; k < N; k += Piece<T>::kV)
      Piece<T>::unpack(*reinterpret_cast<const u32x4_any *>(q + k * Piece<T>::kSize), v + k);
  } else {
    typedef u32x2 __attribute__((aligned(2))) pair;
    const u32x2 w = *reinterpret_cast<const pair *>(q);
    const uint32_t a = w[0], b = w[1];
    v[0] = T::lo(a), v[1] = T::hi(a), v[2] = T::lo(b), v[3] = T::hi(b);
  }
}
template <class T, int N>
__device__ inline void store_values(void *p, int64_t i, int left, const float *v) {
  char *q = static_cast<char *>(p) + i * Piece<T>::kSize;
  if (left < N) {
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (k < left) T::store(q, k, v[k]);
  } else if constexpr (Piece<T>::kV <= N) {
#pragma unroll
    for (int k = 0; k < N; k += Piece<T>::kV)
      *reinterpret_cast<u32x4_any *>(q + k * Piece<T>::kSize) = Piece<T>::pack(v + k);
  } else {
    typedef u32x2 __attribute__((aligned(2))) pair;
    *reinterpret_cast<pair *>(q) = u32x2{T::pack(v[0], v[1]), T::pack(v[2], v[3])};
  }
}
// Eight codes.
typedef u32x2 __attribute__((aligned(1))) codes_any;
__device__ inline u32x2 load_codes(const void *p, int64_t i, int left) {
  const uint8_t *q = static_cast<const uint8_t *>(p) + i;
  if (left == 8) return *reinterpret_cast<const codes_any *>(q);
  u32x2 w = {0, 0};
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (k < left) w[k / 4] |= (uint32_t)q[k] << (8 * (k % 4));
  return w;
}
__device__ inline void store_codes(void *p, int64_t i, int left, u32x2 w) {
  uint8_t *q = static_cast<uint8_t *>(p) + i;
  if (left == 8) {
    *reinterpret_cast<codes_any *>(q) = w;
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < left) q[k] = (uint8_t)(w[k / 4] >> (8 * (k % 4)));
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
  constexpr int N = kLane<BITS>;
  const int lane = threadIdx.x % 64;
  int64_t b = (int64_t)blockIdx.x * kWaves + uniform(threadIdx.x / 64);
  for (; b < blocks; b += (int64_t)gridDim.x * kWaves) {
    // the tensor that has the wavefront's values: the last one that starts at them or before
    int lo = 0, hi = a.n;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (a.t[mid].begin <= b) lo = mid;
      else hi = mid;
    }
    const AdamTensor t = a.t[uniform(lo)];
    const int64_t i = (b - t.begin) * (64 * N) + N * lane;
    const int left = (int)max((int64_t)0, min((int64_t)N, t.count - i));
    float g[N], w[N], m[N], v[N];
    load_values<G, N>(t.grad, i, left, g);
    if (t.master) load_values<Fp32, N>(t.master, i, left, w);
    else load_values<T, N>(t.param, i, left, w);
    const int64_t share = i / kShare;    // (8 bits: of half a wavefront)
    const bool any = share * kShare < t.count;
    if constexpr (BITS == 32) {
      load_values<Fp32, N>(t.m, i, left, m);
      load_values<Fp32, N>(t.v, i, left, v);
    } else {
      const u32x2 cm = load_codes(t.m, i, left), cv = load_codes(t.v, i, left);
      const float sm = any ? t.scales[2 * share] : 1.f, sv = any ? t.scales[2 * share + 1] : 1.f;
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const uint32_t x = cm[k / 4] >> (8 * (k % 4)) & 0xff, y = cv[k / 4] >> (8 * (k % 4)) & 0xff;
        m[k] = value_of<3, -6>(x & 0x7f) * sm;
        m[k] = x & 0x80 ? -m[k] : m[k];
        v[k] = value_of<2, -14>(y & 0x7f) * sv;
      }
    }
    float big_m = 0.f, big_v = 0.f;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      g[k] = g[k] * factor;
      m[k] = m[k] * b1 + g[k] * c1;
      v[k] = v[k] * b2 + g[k] * g[k] * c2;
      big_m = fmaxf(big_m, fabsf(m[k]));
      big_v = fmaxf(big_v, v[k]);
      w[k] = w[k] - w[k] * s.decay - m[k] * s.lr_m / (sqrtf(v[k]) * s.root + eps);
    }
    if (t.master) store_values<Fp32, N>(t.master, i, left, w);
    store_values<T, N>(t.param, i, left, w);
    if constexpr (BITS == 32) {
      store_values<Fp32, N>(t.m, i, left, m);
      store_values<Fp32, N>(t.v, i, left, v);
    } else {
      float sm, im, sv, iv;
      bool fm = true, fv = true;       // (fmaxf passes over a NaN)
#pragma unroll
      for (int k = 0; k < N; ++k) fm &= fabsf(m[k]) < INFINITY, fv &= v[k] < INFINITY;
      const uint64_t half = 0xffffffffull << (lane & 32);
      scale_of(half_max(big_m), (~__ballot(fm) & half) == 0, 7, sm, im);
      scale_of(half_max(big_v), (~__ballot(fv) & half) == 0, 14, sv, iv);
      const uint64_t quad = (t.first * kShare + (uint64_t)i) / 4;
      u32x2 cm = {0, 0}, cv = {0, 0};
#pragma unroll
      for (int k = 0; k < N; k += 4) {
        const u32x4 r = philox(quad + k / 4, step, a.key0, a.key1);
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          const uint32_t word = r[n];
          const float scaled = fabsf(m[k + n]) * im;
          uint32_t x = code_of<3, -6>(scaled, scaled < kLeast ? 0 : word & 0xffff);
          if (m[k + n] < 0.f) x |= 0x80;
          uint32_t y = code_of<2, -14>(v[k + n] * iv, word >> 16);
          if (v[k + n] > 0.f && y == 0) y = 1;
          cm[k / 4] |= (x & 0xff) << (8 * n);
          cv[k / 4] |= (y & 0xff) << (8 * n);
        }
      }
      store_codes(t.m, i, left, cm);
      store_codes(t.v, i, left, cv);
      if (any && lane % 32 == 0) t.scales[2 * share] = sm, t.scales[2 * share + 1] = sv;
    }
  }
}

template <class T, class G, int BITS>
void launch(AdamArgs a, hipStream_t s) {
  if (!a.step_dev && !a.lr_dev) a.s = step_of(a, (double)a.step, a.lr);
  constexpr int kPer = 64 * kLane<BITS>;
  int64_t blocks = 0;                  // wavefronts' values
  for (int i = 0; i < a.n; ++i) {
    a.t[i].begin = blocks;
    blocks += (a.t[i].count + kPer - 1) / kPer;
  }
  if (blocks == 0) return;
  const unsigned grid = (unsigned)std::min<int64_t>((blocks + kWaves - 1) / kWaves, 8 * kSeqCus);
  adamw_kernel<T, G, BITS><<<grid, 64 * kWaves, 0, s>>>(a, blocks);
}
template <class T, class G>
void launch(const AdamArgs &a, int bits, hipStream_t s) {
  if (bits == 8) launch<T, G, 8>(a, s);
  else launch<T, G, 32>(a, s);
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
