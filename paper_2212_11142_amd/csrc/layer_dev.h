// Device building blocks of the layers' kernels: rows of bf16, fp16 or fp32 as 16-byte pieces at
// any alignment of their type.
#pragma once
#include "layer.h"
#include "seq_dev.h"

namespace bgp {

// (a global load or store of 16 bytes may start at any address: unaligned access is on in the
// kernels' mode, and the compiler then takes one instruction for these types too)
typedef u32x4 __attribute__((aligned(2))) u32x4_any;

struct Fp32 {
  static __device__ float load(const void *p, int64_t i) { return static_cast<const float *>(p)[i]; }
  static __device__ void store(void *p, int64_t i, float v) { static_cast<float *>(p)[i] = v; }
};

// kV values of a piece of 16 bytes.
template <class T>
struct Piece {
  static constexpr int kV = 8, kSize = 2;
  static __device__ void unpack(u32x4 w, float *v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t u = w[i];
      v[2 * i] = T::lo(u), v[2 * i + 1] = T::hi(u);
    }
  }
  static __device__ u32x4 pack(const float *v) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = T::pack(v[2 * i], v[2 * i + 1]);
    return w;
  }
};
template <>
struct Piece<Fp32> {
  static constexpr int kV = 4, kSize = 4;
  static __device__ void unpack(u32x4 w, float *v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t u = w[i];
      v[i] = word_float(u);
    }
  }
  static __device__ u32x4 pack(const float *v) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(uint32_t, v[i]);
    return w;
  }
};

// The values e .. e + kV - 1 of a row of `width`; those past its end are `fill`.
template <class T>
__device__ inline void load_piece(const void *row, int e, int width, float *v, float fill = 0.f) {
  constexpr int V = Piece<T>::kV;
  if (e + V <= width) {
    Piece<T>::unpack(*reinterpret_cast<const u32x4_any *>(
                         static_cast<const char *>(row) + (int64_t)e * Piece<T>::kSize), v);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = e + i < width ? T::load(row, e + i) : fill;
  }
}
template <class T>
__device__ inline void store_piece(void *row, int e, int width, const float *v) {
  constexpr int V = Piece<T>::kV;
  if (e + V <= width) {
    *reinterpret_cast<u32x4_any *>(static_cast<char *>(row) + (int64_t)e * Piece<T>::kSize) =
        Piece<T>::pack(v);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (e + i < width) T::store(row, e + i, v[i]);
  }
}

// A value of a type that the launch gives.
__device__ inline void store_any(int dtype, void *p, int64_t i, float v) {
  if (dtype == GP_BF16) Bf16::store(p, i, v);
  else if (dtype == GP_FP16) Fp16::store(p, i, v);
  else Fp32::store(p, i, v);
}

template <class T>
__device__ inline const char *row_at(const Rows &x, int64_t r) {
  return static_cast<const char *>(x.data) + r * x.row * Piece<T>::kSize;
}

// Sum over the THREADS threads of a group (a wavefront, or the whole block through `lds` of one
// float per wavefront), on every one of them.
template <int THREADS>
__device__ inline float group_sum(float x, float *lds) {
  x = wave_sum(x);
  if constexpr (THREADS > 64) {
    const int wave = threadIdx.x / 64;
    __syncthreads();                     // (the sums before have been read)
    if (threadIdx.x % 64 == 0) lds[wave] = x;
    __syncthreads();
    x = 0.f;
#pragma unroll
    for (int i = 0; i < THREADS / 64; ++i) x += lds[i];
  }
  return x;
}

}  // namespace bgp
