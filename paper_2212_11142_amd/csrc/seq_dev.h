// Device building blocks of the sequence-surrogate kernels: matrix-instruction tiles of
// 16-bit operands, tile loads into LDS, and the masked, capped, biased scores.
//
// Tile forms. v_mfma_f32_32x32x16 takes A (row = lane % 32) and B (column = lane % 32) as
// 8 consecutive k per lane, k = 8 (lane / 32) + j, and gives D with column = lane % 32 and
// row = 8 g + 4 (lane / 32) + r in element 4 g + r. A product whose result is the B operand
// of the next one is therefore taken transposed (scores as keys x queries): a lane then
// holds 4 + 4 consecutive rows of each 16, which is the B operand of the next product up to
// the order of k, and k's order is free as long as A is read in the same one. So the
// probabilities never leave their lane's registers, and A (V, dO, Q, K with the summed
// axis along rows) comes out of LDS through the transposing read, 4 rows at a time.
#pragma once
#include "seq.h"

namespace bgp {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// ------------------------------------------------------------------ element types
struct Bf16 {
  static constexpr uint32_t kExp = 0x7f807f80u, kExpOne = 0x00800080u;
  static __device__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  // two values rounded to nearest even, the first in the low half
  static __device__ uint32_t pack(float a, float b) {
    return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
  }
  static __device__ float lo(uint32_t x) { return __builtin_bit_cast(float, x << 16); }
  static __device__ float hi(uint32_t x) { return __builtin_bit_cast(float, x & 0xffff0000u); }
  static __device__ float load(const void *p, int64_t i) {
    return __builtin_bit_cast(float, (uint32_t)static_cast<const uint16_t *>(p)[i] << 16);
  }
  static __device__ void store(void *p, int64_t i, float v) {
    static_cast<__bf16 *>(p)[i] = (__bf16)v;
  }
};
struct Fp16 {
  static constexpr uint32_t kExp = 0x7c007c00u, kExpOne = 0x04000400u;
  static __device__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
  static __device__ uint32_t pack(float a, float b) {
    return __builtin_bit_cast(uint32_t, f16x2{(_Float16)a, (_Float16)b});
  }
  static __device__ float lo(uint32_t x) { return (float)__builtin_bit_cast(f16x2, x)[0]; }
  static __device__ float hi(uint32_t x) { return (float)__builtin_bit_cast(f16x2, x)[1]; }
  static __device__ float load(const void *p, int64_t i) {
    return (float)static_cast<const _Float16 *>(p)[i];
  }
  static __device__ void store(void *p, int64_t i, float v) {
    static_cast<_Float16 *>(p)[i] = (_Float16)v;
  }
};

// The forward pass's probabilities are e^(score - m) times 2^shift, m the running maximum. It is
// raised, and the sums rescaled, only when a row's scores pass it by more than `slack` (in log 2):
// so the rescaling is skipped almost always, and what enters the second product reaches
// 2^(slack + shift). bf16 has fp32's range for that. fp16 ends at 2^16 and, below its normal
// numbers, rounds to multiples of 2^-24: with 2^15 for the largest a probability is off by its 11
// bits' rounding or by 2^-(25 + shift) of the maximum. Up to 4096 keys, 2^-32 each, that is 2^-20 of
// the largest |v| at most; more keys, each of which may have little, get 2^-39 (2^-19 at 2^20 keys)
// by raising the maximum more often. Slack 8 / 4 / 1: 1,048,576 rows over 512 keys 1481 / 1509 / 1562
// us (before 2^shift too), 13 documents of up to 1021 62 / 63.4 / 65.2, one of 16,384 1194 / 1195 /
// 1196.
constexpr int kManyKeys = 4096;
template <class T>
struct Probs {
  static __device__ float slack(int) { return 8.f; }
  static __device__ float shift(int) { return 0.f; }
};
template <>
struct Probs<Fp16> {
  static __device__ float slack(int lk) { return lk > kManyKeys ? 1.f : 8.f; }
  static __device__ float shift(int lk) { return 15.f - slack(lk); }
};

__device__ inline float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// (a parameter, not an element of a vector: __builtin_bit_cast takes those from the front)
__device__ inline float word_float(uint32_t x) { return __builtin_bit_cast(float, x); }

// Largest of three, NaN if one of them is: one instruction, and one that the compiler knows, so
// that it waits for the matrix and the transcendental instructions whose results these are.
// (fmaxf, which passes over a NaN, would first multiply each such operand by 1, against signalling
// NaN.)
__device__ inline float max3(float a, float b, float c) {
  return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);
}

// Sum and maximum over a lane and the one 32 away.
__device__ inline float sum_halves(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const u32x2 r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return word_float(r[0]) + word_float(r[1]);
}
__device__ inline float max_halves(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const u32x2 r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(word_float(r[0]), word_float(r[1]));
}

// Sum and maximum over the wavefront, on every lane, without LDS: neighbours, pairs, halves
// of 8 and rows of 16 mirrored, then rows and halves swapped.
template <int CTRL>
__device__ inline float moved(float x) {
  const int u = __builtin_bit_cast(int, x);
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(u, u, CTRL, 0xf, 0xf, false));
}
// over the four rows of 16 lanes
__device__ inline float sum_rows(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const u32x2 r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return sum_halves(word_float(r[0]) + word_float(r[1]));
}
// over a row of 16 lanes
__device__ inline float row_sum(float x) {
  x += moved<0xb1>(x);    // quad_perm 1 0 3 2
  x += moved<0x4e>(x);    // quad_perm 2 3 0 1
  x += moved<0x141>(x);   // row_half_mirror
  x += moved<0x140>(x);   // row_mirror
  return x;
}
__device__ inline float wave_sum(float x) { return sum_rows(row_sum(x)); }
__device__ inline float wave_max(float x) {
  x = fmaxf(x, moved<0xb1>(x));
  x = fmaxf(x, moved<0x4e>(x));
  x = fmaxf(x, moved<0x141>(x));
  x = fmaxf(x, moved<0x140>(x));
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const u32x2 r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return max_halves(fmaxf(word_float(r[0]), word_float(r[1])));
}

// ------------------------------------------------------------------ LDS tiles
// A tile is rows of DP 16-bit values without padding. The 16-byte pieces of a row are
// stored in the order piece ^ swizzle(row): then both the row reads (32 rows, one piece
// each half wavefront) and the transposing reads (4 rows x 4 pieces per half wavefront)
// touch all of LDS's 64 banks evenly.
template <int DP>
__device__ inline int swizzle(int row) {
  if (DP == 128) return ((row & 3) << 2) | ((row >> 2) & 3);
  return (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
}

// Rows r0.. of a matrix with `rows` rows from base (row stride `stride` bytes, `bytes` of
// each row used) as a buffer: reads past it, and of pieces past `bytes`, give zeros.
__device__ inline u32x4 row_buffer(const char *base, int64_t r0, int rows, int64_t stride,
                                   int bytes) {
  const uint64_t a = (uint64_t)base + (uint64_t)(r0 * stride);
  u32x4 d;
  d[0] = uniform((int)(uint32_t)a);
  d[1] = uniform((int)((uint32_t)(a >> 32) & 0xffffu));
  d[2] = uniform(rows > 0 ? (int)((rows - 1) * stride) + bytes : 0);
  d[3] = 0x00020000u;
  return d;
}

// Starts the copy of ROWS rows of a buffer into an LDS tile by WAVES wavefronts (`wave`
// is this one's number): each instruction moves 64 pieces of 16 bytes, and what is out of
// range arrives as zeros. Completion: wait_copies(). (s_nop: a scalar register that a vector
// instruction wrote, v_readfirstlane say, must be 5 cycles old when such an instruction reads it;
// the compiler counts none of them before inline assembly.)
template <int DP, int ROWS, int WAVES>
struct TileCopy {
  static constexpr int kPieces = DP / 8;               // pieces of a row
  static constexpr int kRowsPer = 64 / kPieces;        // rows an instruction moves
  static constexpr int kCount = ROWS / kRowsPer / WAVES;
  int voff[kCount];
  int lds0;

  __device__ void init(int wave, int lane, int stride, int bytes) {
#pragma unroll
    for (int i = 0; i < kCount; ++i) {
      const int row = (i * WAVES + wave) * kRowsPer + lane / kPieces;
      const int piece = (lane % kPieces) ^ swizzle<DP>(row);
      voff[i] = piece * 16 < bytes ? row * stride + piece * 16 : 0x7ffffff0;
    }
    lds0 = wave * 1024;
  }
  __device__ void start(u32x4 buf, uint32_t lds) const {
    constexpr int kStep = WAVES * 1024;
    const uint32_t m = uniform((int)(lds + lds0));
    if constexpr (kCount == 1) {
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                   ::"s"(m), "v"(voff[0]), "s"(buf)
                   : "memory");
    } else if constexpr (kCount == 2) {
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %2, %4, 0 offen lds\n\t"
                   "s_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %3, %4, 0 offen lds"
                   ::"s"(m), "s"(m + kStep), "v"(voff[0]), "v"(voff[1]), "s"(buf)
                   : "memory");
    } else {
      static_assert(kCount % 4 == 0);
#pragma unroll
      for (int i = 0; i < kCount; i += 4)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %4, %8, 0 offen lds\n\t"
                     "s_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %5, %8, 0 offen lds\n\t"
                     "s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %6, %8, 0 offen lds\n\t"
                     "s_mov_b32 m0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %7, %8, 0 offen lds"
                     ::"s"(m + i * kStep), "s"(m + (i + 1) * kStep), "s"(m + (i + 2) * kStep),
                     "s"(m + (i + 3) * kStep), "v"(voff[i]), "v"(voff[i + 1]), "v"(voff[i + 2]),
                     "v"(voff[i + 3]), "s"(buf)
                     : "memory");
    }
  }
};

// Until the copies that this wavefront started are in LDS, but for the last `left` of them.
template <int LEFT>
__device__ inline void wait_copies() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LEFT) : "memory");
}
// Joins the block: copies started by all wavefronts are in LDS, reads of LDS are done.
__device__ inline void copies_barrier() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

__device__ inline uint32_t lds_address(const void *p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void *)p;
}

// Operands out of LDS tiles. A lane's addresses differ from its first one by an XOR of the
// piece (the swizzle is one too) and by whole rows, so that two offsets per lane and one
// instruction per address do: kept ready for every piece, they would take the accumulators'
// registers.
template <int DP>
struct TileReader {
  uint32_t row, col;   // of this lane within a tile

  __device__ void init(int lane) {
    const int r = lane & 31;
    row = r * (DP * 2) + ((lane >> 5) ^ swizzle<DP>(r)) * 16;
    const int q = 4 * (lane >> 5) + ((lane & 15) >> 2);
    const int piece = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    col = q * (DP * 2) + (piece ^ swizzle<DP>(q)) * 16 + (lane & 1) * 8;
  }
  // an offset of the tile at LDS address `tile` (a multiple of 1024)
  static __device__ uint32_t at(uint32_t tile, uint32_t offset) {
    uint32_t x = tile + offset;
    asm volatile("" : "+v"(x));   // (not to be precomputed for every piece)
    return x;
  }
};

// A operand (32 rows from row0, k = 16 s + ..) of a tile whose rows run along k; x =
// at(tile, row).
template <int DP>
__device__ inline u32x4 row_operand(uint32_t x, int row0, int s) {
  typedef __attribute__((address_space(3))) const u32x4 lds_u32x4;
  return *(lds_u32x4 *)(uintptr_t)((x ^ (s * 32)) + row0 * (DP * 2));
}

// A operand of the transposed tile: rows of the operand are the columns 32 c.. of the tile,
// its k the tile's rows row0 + 16.. in the order of a D result's registers: lane half h has
// the rows row0 + 4 h + {0..3} and row0 + 8 + 4 h + {0..3}; x = at(tile, col).
template <int DP>
__device__ inline u32x4 col_operand(uint32_t x, int row0, int c) {
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (lds_s16x4 *)(uintptr_t)((x ^ (c * 64)) + row0 * (DP * 2)));
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (lds_s16x4 *)(uintptr_t)((x ^ (c * 64 + 32)) + (row0 + 8) * (DP * 2)));
  const u32x2 ua = __builtin_bit_cast(u32x2, a), ub = __builtin_bit_cast(u32x2, b);
  return u32x4{ua[0], ua[1], ub[0], ub[1]};
}

// B operand of 32 rows of a matrix in memory (column = row, k = 16 s + ..): one lane's
// pieces for all s; rows from `rows` on and values from `bytes` on are zero.
template <int DP>
__device__ inline void load_operand(const char *base, int64_t stride, int row, int rows, int bytes,
                                    int lane, u32x4 *out) {
#pragma unroll
  for (int s = 0; s < DP / 16; ++s) {
    const int off = (2 * s + (lane >> 5)) * 16;
    u32x4 v = {0, 0, 0, 0};
    if (row < rows && off < bytes)
      v = *reinterpret_cast<const u32x4 *>(base + (int64_t)row * stride + off);
    out[s] = v;
  }
}

// The two packed values as they are stored: what is computed from them then is computed from the
// numbers in memory. (The compiler may round a value once more for another use, from the product
// that it comes from instead of from that product's fp32 rounding: one step off at ties.)
__device__ inline uint32_t as_stored(uint32_t w) {
  asm("" : "+v"(w));
  return w;
}

// Writes a transposed result (D^T: element d = 32 c + 8 g + 4 (lane / 32) + r of the row at
// p, both lane halves of a row) as 16-byte pieces, times f; with REST also what the rounding to T
// took from each value, at `rest`.
template <class T, int DT, bool REST = false>
__device__ inline void store_row(char *p, bool ok, int bytes, const f32x16 *acc, float f, int lane,
                                 char *rest = nullptr) {
  const int h = lane >> 5;
#pragma unroll
  for (int c = 0; c < DT; ++c)
#pragma unroll
    for (int g = 0; g < 4; g += 2) {
      uint32_t w[4], e[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int k = 4 * (g + i / 2) + 2 * (i % 2);
        const float x = acc[c][k] * f, y = acc[c][k + 1] * f;
        w[i] = T::pack(x, y);
        if (REST) {
          w[i] = as_stored(w[i]);
          e[i] = T::pack(x - T::lo(w[i]), y - T::hi(w[i]));
        }
      }
      // lower half: all of piece g, upper half: all of piece g + 1
      auto store = [&](char *to, const uint32_t *v) {
        const u32x2 x = __builtin_amdgcn_permlane32_swap(v[0], v[2], false, false);
        const u32x2 y = __builtin_amdgcn_permlane32_swap(v[1], v[3], false, false);
        const int off = (32 * c + 8 * (g + h)) * 2;
        if (ok && off < bytes) *reinterpret_cast<u32x4 *>(to + off) = u32x4{x[0], y[0], x[1], y[1]};
      };
      store(p, w);
      if (REST) store(rest, e);
    }
}

// ------------------------------------------------------------------ values in masked places
// Nonzero if one of the 8 values is infinite or NaN (its exponent's carry goes into the
// place of the sign).
template <class T>
__device__ inline uint32_t nonfinite(u32x4 v) {
  uint32_t r = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) r |= (v[i] & T::kExp) + T::kExpOne;
  return r & 0x80008000u;
}
// The values with 0 in place of infinities and NaN.
template <class T>
__device__ inline u32x4 finite_part(u32x4 v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t t = (v[i] & T::kExp) + T::kExpOne;
    if (t & 0x8000u) v[i] &= 0xffff0000u;
    if (t & 0x80000000u) v[i] &= 0x0000ffffu;
  }
  return v;
}
// Sum of the infinities and NaN in column d of the rows r0..r1 - 1.
template <class T>
__device__ inline float nonfinite_sum(const char *base, int64_t stride, int r0, int r1, int d) {
  float x = 0.f;
  for (int r = r0; r < r1; ++r) {
    const float v = T::load(base + r * stride, d);
    if (!(__builtin_fabsf(v) < __builtin_inff())) x += v;
  }
  return x;
}

// ------------------------------------------------------------------ documents
struct DocTile {
  int doc, tile;  // doc < 0: past the last tile
  int b0, b1;     // the document's rows on the tiled side
};

// The tile-th tile of TILE rows of the documents with rows [b[d], e[d]) within 0..limit, in
// order. Every lane gets the same answer.
template <int TILE>
__device__ inline DocTile find_tile(const int32_t *b, const int32_t *e, int docs, int limit,
                                    int tile) {
  const int lane = threadIdx.x & 63;
  for (int d0 = 0; d0 < docs; d0 += 64) {
    int lo = 0, hi = 0;
    if (d0 + lane < docs) {
      lo = max(b[d0 + lane], 0);
      hi = max(min(e[d0 + lane], limit), lo);
    }
    const int n = (hi - lo + TILE - 1) / TILE;
    int inc = n;  // inclusive sum over the lanes
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(inc, o);
      if (lane >= o) inc += v;
    }
    const unsigned long long past = __ballot(inc > tile);
    if (past) {
      const int l = __ffsll(past) - 1;
      DocTile r;
      r.doc = d0 + l;
      r.b0 = uniform(__shfl(lo, l));
      r.b1 = uniform(__shfl(hi, l));
      r.tile = uniform(tile - __shfl(inc - n, l));
      return r;
    }
    tile -= uniform(__shfl(inc, 63));
  }
  return DocTile{-1, 0, 0, 0};
}

// ------------------------------------------------------------------ scores
// A score in units of log 2 is a x + b + bias. Without a cap x is the product itself. With one there
// are two forms of cap tanh(z / cap), z = scale times the product:
//   near: cap + 2 cap x, x = -1 / (1 + e^(2 z / cap)); exact at both ends, where the exponential is 0
//         or infinite, but off by up to cap 2^-22 in all between: 1.5e-5 at a cap of 64, 2e-3 at 1e4;
//   far:  x is the capped product itself, for |z| < cap / 4 as z times an even polynomial of z / cap
//         (the series of tanh; the first term left out is 9e-9 of it), else as cap (1 - 2 / (1 +
//         e^(2 z / cap))): off by 2^-21 of itself, for every cap. It takes longer: near / far,
//         13 documents of up to 1021 rows, 16 heads of 128, 57 / 68 us; training on 16 documents,
//         16 heads of 64, 229 / 265; 64 caches of up to 32,768 421 / 423.
enum CapKind { kCapNone = 0, kCapNear = 1, kCapFar = 2 };
// Documents of up to 8 keys, whose log-sums are little more than one score, take the far form for
// every cap (a log-sum of one key at a cap of 50 was off by 1.2e-6 of itself, of 8 keys by 6e-7; up
// to 32 keys the far form would cost 1000 documents 6 to 9%).
constexpr float kNearCap = 64.f;   // the largest cap of the near form
constexpr int kNearKeys = 8;       // documents of the near form have more
inline CapKind cap_kind(const AttnArgs &a) {
  if (!(a.cap > 0.f)) return kCapNone;
  return a.cap <= kNearCap && a.max_k > kNearKeys ? kCapNear : kCapFar;
}
struct ScoreScale {
  float c;   // near: the product's factor in the exponential; far: scale
  float a, b;
  float cap, inv;   // far: cap and 1 / cap
};
template <int CAP>
__device__ inline ScoreScale score_scale(float scale, float cap) {
  ScoreScale k = {};
  if (CAP == kCapNone) {
    k.a = scale * kLog2e;
  } else if (CAP == kCapNear) {
    k.b = cap * kLog2e;
    k.a = 2.f * k.b;
    // (finite, so that a product of 0 gives 0 with the smallest caps too)
    k.c = fminf(2.f * kLog2e * scale / cap, 3.4028234663852886e38f);
  } else {
    k.a = kLog2e;
    k.c = scale;
    k.cap = cap;
    k.inv = 1.f / cap;
  }
  return k;
}
template <int CAP>
__device__ inline float score_x(float s, const ScoreScale &k) {
  if (CAP == kCapNone) return s;
  if (CAP == kCapNear) return __builtin_amdgcn_rcpf(-(1.f + fast_exp2(s * k.c)));
  const float z = s * k.c, u = z * k.inv, v = u * u;
  float p = __builtin_fmaf(v, 62.f / 2835.f, -17.f / 315.f);
  p = __builtin_fmaf(p, v, 2.f / 15.f);
  p = __builtin_fmaf(p, v, -1.f / 3.f);
  const float near = __builtin_fmaf(z * v, p, z);
  const float t = __builtin_fmaf(-2.f, __builtin_amdgcn_rcpf(1.f + fast_exp2(u * (2.f * kLog2e))), 1.f);
  return v < 0.0625f ? near : k.cap * t;
}
// Derivative of the capped product, 1 - tanh^2, up to a constant that is left to the results: near
// 1 - (1 + 2 x)^2 = -4 (x + x^2).
template <int CAP>
constexpr float cap_factor() { return CAP == kCapNear ? -4.f : 1.f; }
template <int CAP>
__device__ inline float cap_slope(float x, const ScoreScale &k) {
  if (CAP == kCapNear) return __builtin_fmaf(x, x, x);
  const float t = x * k.inv;
  return __builtin_fmaf(-t, t, 1.f);
}

enum BiasKind { kBiasNone = 0, kBiasSlope = 1, kBiasTable = 2 };

// Room on both sides of the table's distances -reach..reach, so that a block of 32 keys and
// 32 queries of which any pair is nearer than reach reads the table without clamping.
constexpr int kLutPad = 64;
__host__ __device__ inline int lut_size(int reach) { return 2 * (reach + kLutPad) + 1; }

// Distance from which on keys ahead of a query share a bucket: the sides differ from distance 1 on,
// with one class a side (reach 0) too.
__device__ inline int ahead_reach(int reach) { return max(reach, 1); }

// Bucket of the distance delta = key - query position. (The starts past the last one are
// never reached, so that the comparisons go in eights.)
__device__ inline int bucket_of(const BucketMap &m, int delta) {
  const int a = m.two_sided ? (delta < 0 ? -delta : delta) : (delta < 0 ? -delta : 0);
  int b = 0;
  for (int t = 0; t < m.per_side; t += 8)
#pragma unroll
    for (int i = 0; i < 8; ++i) b += a >= m.start[t + i] ? 1 : 0;
  return b - 1 + ((m.two_sided && delta > 0) ? m.per_side : 0);
}
__host__ __device__ inline int bucket_count(const BucketMap &m) {
  return m.two_sided ? 2 * m.per_side : m.per_side;
}

// The buckets of the table's distances in LDS, and a head's biases (log 2 units) from them,
// each as `thread` of `threads`.
__device__ inline void fill_map(uint8_t *map, const BucketMap &m, int thread, int threads) {
  const int reach = m.start[m.per_side - 1], n = lut_size(reach);
  for (int i = thread; i < n; i += threads) map[i] = (uint8_t)bucket_of(m, i - (reach + kLutPad));
}
template <class T>
__device__ inline void fill_lut(float *lut, const uint8_t *map, const BucketMap &m, const void *table,
                                int head, int thread, int threads) {
  const int n = lut_size(m.start[m.per_side - 1]);
  const int64_t row = (int64_t)head * bucket_count(m);
#pragma unroll 4
  for (int i = thread; i < n; i += threads) lut[i] = T::load(table, row + map[i]) * kLog2e;
}
// LDS of a map, rounded up
__host__ __device__ inline int map_bytes(int reach) { return (lut_size(reach) + 15) / 16 * 16; }

// Offset of element e of a D result along its rows, without the lane half's 4.
constexpr int row_of(int e) { return 8 * (e >> 2) + (e & 3); }

// Puts the bias of 32 keys (from key0) on the 16 x of a lane whose query stands at pos; the
// block's positions are pos_lo..pos_lo + 31. Afterwards the scores are a x + b with the
// returned a (the same on all lanes) and b: what all of a lane's pairs share, or what every
// pair has, is left to those. `lut` is the head's table, `slope2` its slope, both in log 2
// units, steps[e] slope2 row_of(e).
struct Affine {
  float a, b;
};
template <int BIAS>
__device__ inline Affine add_bias(f32x16 &x, const ScoreScale &k, int key0, int pos, int pos_lo, int h,
                                  float slope2, const float *steps, const float *lut, int reach) {
  if (BIAS == kBiasSlope) {
    const float d0 = (float)(key0 + 4 * h - pos);
    if (key0 + 31 <= pos_lo) {  // no key ahead of a query: the bias is linear
      float a = k.a;
      asm volatile("" : "+v"(a));   // (an instruction takes one scalar register: the step's)
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] = __builtin_fmaf(x[e], a, steps[e]);
      return Affine{1.f, __builtin_fmaf(slope2, d0, k.b)};
    }
#pragma unroll
    for (int e = 0; e < 16; ++e)
      x[e] = __builtin_fmaf(x[e], k.a, -slope2 * __builtin_fabsf(d0 + (float)row_of(e)));
    return Affine{1.f, k.b};
  }
  if (BIAS == kBiasTable) {
    if (key0 + 31 - pos_lo <= -reach) return Affine{k.a, k.b + lut[0]};
    if (key0 - (pos_lo + 31) >= ahead_reach(reach)) return Affine{k.a, k.b + lut[lut_size(reach) - 1]};
    const float *p = lut + (key0 + 4 * h - pos + reach + kLutPad);
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = __builtin_fmaf(x[e], k.a, p[row_of(e)]);
    return Affine{1.f, k.b};
  }
  return Affine{k.a, k.b};
}
template <int BIAS>
__device__ inline void slope_steps(float *steps, float slope2) {
  if (BIAS != kBiasSlope) return;
#pragma unroll
  for (int e = 0; e < 16; ++e)
    steps[e] = __builtin_bit_cast(float, uniform(__builtin_bit_cast(int, slope2 * (float)row_of(e))));
}

}  // namespace bgp
