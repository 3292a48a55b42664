// The gated feed-forward block's hidden values, out = act(x Wg') * (x Wu'), and its gradient:
//   dg = dout * u * act'(g),  du = dout * act(g),
//   dx = dg Wg + du Wu,  dWg = dg' x,  dWu = du' x,
// as tiled products on the matrix units with fp32 sums. The forward pass has both projections of
// a tile of hidden values in one block, whose epilogue multiplies them; the gradient forms g and u
// again in the same way (nothing is kept from the forward pass), its epilogue writes dg and du,
// rounded once as operands of the three products that follow; in fp16 times a power of two.
//
// Tiles. Every product is taken transposed: the result's contiguous axis is the A operand's, so
// that a lane holds 4 consecutive values of a result's row. A step has 64 of the summed axis; an
// operand's tile in LDS has either its rows running along the summed axis (ROW) or the summed
// axis' rows running along its own (COL), which the transposing reads turn. Copies go to LDS
// directly, the next step's while this one's products run.
#include "gated_tiles.h"
#include "layer_dev.h"

namespace bgp {
namespace {

constexpr int kStep = 64;              // of the summed axis
constexpr int kStepBytes = 2 * kStep;

// Copies 64 pieces of 16 bytes of a buffer, a lane's at `offset`, to 1024 bytes of LDS. (s_nop: as for
// a tile's copies, a scalar register of the descriptor must be 5 cycles old.)
__device__ inline void copy_pieces(u32x4 buf, int offset, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               ::"s"(uniform((int)lds)), "v"(offset), "s"(buf)
               : "memory");
}

// R rows of an operand, copied by WAVES wavefronts. copy(i, ..): the i-th of a wavefront's kCopies
// instructions for a step that starts at k0; nothing is read if `on` is false.
template <bool COL, int R, int WAVES>
struct Side;

template <int R, int WAVES>
struct Side<false, R, WAVES> {
  typedef TileCopy<64, R, WAVES> Copy;
  static constexpr int kBytes = R * kStepBytes, kCopies = Copy::kCount, kReads = 1;
  Copy of;
  TileReader<64> reader;
  const char *base;
  int64_t stride;
  int rows, piece;

  // rows row0.. of a matrix of `all` rows
  __device__ void move(const char *p, int64_t row0, int64_t all) {
    base = p + row0 * stride;
    rows = (int)max((int64_t)0, min((int64_t)R, all - row0));
  }
  __device__ void init(const char *p, int64_t row0, int64_t all, int64_t row_stride, int wave, int lane) {
    stride = row_stride;
    move(p, row0, all);
    of.init(wave, lane, (int)stride, kStepBytes);
    reader.init(lane);
    // the piece of a row that this lane copies: the same in all its rows, which are WAVES * 8 apart
    piece = ((lane % 8) ^ swizzle<64>(wave * 8 + lane / 8)) * 16;
  }
  __device__ void copy(int i, bool on, int64_t k0, int64_t k, uint32_t lds) const {
    const int left = (int)min((int64_t)kStepBytes, 2 * (k - k0));
    copy_pieces(row_buffer(base + 2 * k0, 0, on ? rows : 0, stride, left),
                piece < left ? of.voff[i] : 0x7ffffff0, lds + of.lds0 + i * (WAVES * 1024));
  }
  __device__ uint32_t at(uint32_t lds) const { return TileReader<64>::at(lds, reader.row); }
  // rows 32 i.., k = 16 s ..
  static __device__ u32x4 operand(uint32_t x, int i, int s) { return row_operand<64>(x, 32 * i, s); }
};

template <int R, int WAVES>
struct Side<true, R, WAVES> {
  typedef TileCopy<128, kStep, WAVES> Copy;
  static constexpr int kBytes = R * kStepBytes, kParts = R / 128, kPart = kStep * 256;
  static constexpr int kCopies = kParts * Copy::kCount, kReads = 2;
  Copy of[kParts];
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
    for (int i = 0; i < kParts; ++i) of[i].init(wave, lane, (int)stride, bytes - 256 * i);
    // the transposing reads of lane half h: the step's rows 16 s + 8 h + 0..3 and + 4..7, so that k
    // runs as in a ROW operand (a row's swizzle differs by one piece between the two)
    const int q = 8 * (lane >> 5) + ((lane & 15) >> 2);
    const int piece = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    col = q * 256 + (piece ^ swizzle<128>(q)) * 16 + (lane & 1) * 8;
  }
  __device__ void copy(int i, bool on, int64_t k0, int64_t k, uint32_t lds) const {
    const int rows = (int)min((int64_t)kStep, k - k0), q = i / Copy::kCount, n = i % Copy::kCount;
    const int b = min(256, bytes - 256 * q);
    copy_pieces(row_buffer(base + 256 * q, k0, on && b > 0 ? rows : 0, stride, b), of[q].voff[n],
                lds + q * kPart + of[q].lds0 + n * (WAVES * 1024));
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

// Runs `count` steps, each 4 times 16 of the summed axis: after begin(step), called for one step after
// the other and for two past the last, copy(stage, i) is the i-th of a wavefront's COPIES copies,
// read(stage, s, i, operands) fetches the i-th of a quarter's READS operands, multiply(operands, i) is
// the i-th of its MFMAS products, and end(step, stage) follows a step's products and says whether it did
// anything.
//
// A quarter's operands are read while the one before is multiplied. The block meets in front of a step's
// last quarter, whose operands are in registers then: behind that barrier the next step's copies are
// there, and this step's place in LDS is free for the one after, whose copies go out one by one between
// the products of two quarters: a wavefront that asks for all at once waits for the units that take
// them, and its products with it (dx of 16,384 x 1,024 from 8,192: 229 us, 255 with the copies in one
// go; 239 where the lines were asked for two steps ahead, too). At the end of a step the second half of
// its place in LDS is unused until the block meets.
template <class Operands, int COPIES, int MFMAS, int READS, class Begin, class Copy, class Read, class Multiply,
          class End>
__device__ inline void run_steps(int64_t count, Begin begin, Copy copy, Read read, Multiply multiply, End end) {
  if (count <= 0) return;
  constexpr int kHalf = COPIES / 2;
  begin(0);
#pragma unroll
  for (int i = 0; i < COPIES; ++i) copy(0, i);
  begin(1);
#pragma unroll
  for (int i = 0; i < kHalf; ++i) copy(1, i);
  asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(kHalf) : "memory");
  Operands f, g;
  // multiplies `now` while the next quarter's operands are read, and copies `from`.. to stage `to`
  auto quarter = [&](const Operands &now, Operands &next, int stage, int s, int to, int from) {
#pragma unroll
    for (int i = 0; i < MFMAS; ++i) {
      multiply(now, i);
#pragma unroll
      for (int r = i * READS / MFMAS; r < (i + 1) * READS / MFMAS; ++r) read(stage, s, r, next);
      if (from >= 0 && (i + 1) * kHalf / MFMAS > i * kHalf / MFMAS)
        copy(to, from + i * kHalf / MFMAS);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
#pragma unroll
  for (int r = 0; r < READS; ++r) read(0, 0, r, f);
  for (int64_t i = 0; i < count; ++i) {
    const int stage = (int)i & 1;
    quarter(f, g, stage, 1, stage ^ 1, kHalf);
    quarter(g, f, stage, 2, 0, -1);
    quarter(f, g, stage, 3, 0, -1);
    begin(i + 2);
    copies_barrier();
    quarter(g, f, stage ^ 1, 0, stage, 0);
    // (operands read already do not stay in registers beside what end() does)
    if (end(i, stage))
#pragma unroll
      for (int r = 0; r < READS; ++r) read(stage ^ 1, 0, r, f);
  }
  // (what was asked for past the end: a block's place in LDS ends with it)
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

// ------------------------------------------------------------------ results
// A wavefront's 32 rows of 32 C columns on their way between registers, as the matrix units have
// them (4 consecutive values of a row a lane), and memory (rows of 64 C bytes, 16 bytes a lane),
// through its own place in LDS. (Stored from the registers at once, an instruction's 1024 bytes
// go to 32 rows instead of 16 / C.)
template <int C>
struct Exchange {
  static constexpr int kBytes = 32 * 64 * C, kPieces = 4 * C, kRows = 64 / kPieces, kCount = 32 / kRows;
  uint32_t lds;
  int lane;

  __device__ uint32_t at(int row, int piece) const {
    return lds + row * (64 * C) + (piece ^ (row & (kPieces - 1))) * 16;
  }
  // of a lane: values 32 c + 8 g + 4 (lane / 32) + 0..3 of row lane % 32
  __device__ void put(int c, int g, u32x2 v) const {
    typedef __attribute__((address_space(3))) u32x2 lds_u32x2;
    *(lds_u32x2 *)(uintptr_t)(at(lane & 31, 4 * c + g) + 8 * (lane >> 5)) = v;
  }
  __device__ u32x2 get(int c, int g) const {
    typedef __attribute__((address_space(3))) const u32x2 lds_u32x2;
    return *(lds_u32x2 *)(uintptr_t)(at(lane & 31, 4 * c + g) + 8 * (lane >> 5));
  }
  // of a lane: piece lane % kPieces of row kRows i + lane / kPieces
  __device__ void put_row(int i, u32x4 v) const {
    typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
    *(lds_u32x4 *)(uintptr_t)at(kRows * i + lane / kPieces, lane % kPieces) = v;
  }
  __device__ u32x4 get_row(int i) const {
    typedef __attribute__((address_space(3))) const u32x4 lds_u32x4;
    return *(lds_u32x4 *)(uintptr_t)at(kRows * i + lane / kPieces, lane % kPieces);
  }
  // Whether a lane's piece of rows kRows i .. is within `rows` and `bytes`, and its offset.
  __device__ bool within(int i, int64_t rows, int64_t bytes) const {
    return kRows * i + lane / kPieces < rows && lane % kPieces * 16 < bytes;
  }
  __device__ int64_t offset(int i, int64_t stride) const {
    return (kRows * i + lane / kPieces) * stride + lane % kPieces * 16;
  }
  // Writes what lies in LDS to the rows at p.
  __device__ void store(char *p, int64_t stride, int64_t rows, int64_t bytes) const {
    u32x4 v[kCount];
#pragma unroll
    for (int i = 0; i < kCount; ++i) v[i] = get_row(i);
#pragma unroll
    for (int i = 0; i < kCount; ++i)
      if (within(i, rows, bytes)) *reinterpret_cast<u32x4 *>(p + offset(i, stride)) = v[i];
  }
  template <class T>
  __device__ void put_all(const f32x16 *v) const {
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        put(c, g, u32x2{T::pack(v[c][4 * g], v[c][4 * g + 1]), T::pack(v[c][4 * g + 2], v[c][4 * g + 3])});
  }
};

// Two groups of W wavefronts have sums of the same tile, x, of different parts of the summed axis: each gives
// the other half of its own, through LDS, and keeps in x[0] the whole of x[0] (group 0) or x[1] (group 1).
template <int W>
constexpr int kHandOver = 2 * W * 8 * 1024;    // 8 pieces of 16 bytes a lane, both ways
template <int W>
__device__ inline void hand_over(uint32_t lds, int group, int wave, int lane, f32x16 (&x)[2][2]) {
  typedef __attribute__((address_space(3))) f32x4 lds_f32x4;
  const uint32_t at = lds + (wave * 8 * 64 + lane) * 16, half = W * 8 * 1024;
  const uint32_t to = at + (group ? half : 0), from = at + (group ? 0 : half);
  __syncthreads();                       // (all copies have landed, all operands have been read)
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    f32x16 a = x[0][i / 4], b = x[1][i / 4];
    f32x4 y;
#pragma unroll
    for (int r = 4 * (i % 4); r < 4 * (i % 4) + 4; ++r) {
      y[r % 4] = group ? +a[r] : +b[r];
      a[r] = group ? +b[r] : +a[r];
    }
    x[0][i / 4] = a;
    *(lds_f32x4 *)(uintptr_t)(to + i * 1024) = y;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const f32x4 y = *(lds_f32x4 *)(uintptr_t)(from + i * 1024);
#pragma unroll
    for (int r = 0; r < 4; ++r) x[0][i / 4][4 * (i % 4) + r] += y[r];
  }
}

// ------------------------------------------------------------------ activations
constexpr int kSilu = 0, kGelu = 1;   // GP_SILU, GP_GELU

// act(z) and its derivative. gelu: z Phi(z), where
// Phi(-|z|) = 1/2 erfc(|z| / sqrt(2)) = e^(-z^2 / 2) t q(t) / 2, t = 1 / (1 + 0.375 |z| / sqrt(2)), q a least-maximum
// fit of degree 6 to e^(x^2) erfc(x) / t with a relative error of 6.6e-7 up to |z| = 14.5 (at 0, with these fp32 constants;
// beyond, e^(-z^2 / 2) is 0): the tail keeps its digits, and the derivative has the same exponential.
template <int ACT>
__device__ inline void activation(float z, float &a, float &d) {
  if (ACT == kSilu) {
    const float p = __builtin_amdgcn_rcpf(1.f + fast_exp2(-kLog2e * z));
    a = z * p;
    d = p + a * (1.f - p);
  } else {
    const float t = __builtin_amdgcn_rcpf(fmaf(0.26516504f, fabsf(z), 1.f));
    float q = -0.5f * 0.13509515f;
    q = fmaf(q, t, 0.5f * 0.38793566f);
    q = fmaf(q, t, -0.5f * 0.12959506f);
    q = fmaf(q, t, 0.5f * 0.28306065f);
    q = fmaf(q, t, 0.5f * 0.16666456f);
    q = fmaf(q, t, 0.5f * 0.21568926f);
    q = fmaf(q, t, 0.5f * 0.21133943f);
    const float e = fast_exp2(z * z * (-0.5f * kLog2e));
    const float tail = e * (t * q);
    const float p = z < 0.f ? tail : 1.f - tail;
    a = z * p;
    d = fmaf(z * e, 0.39894228f, p);
  }
}

// ------------------------------------------------------------------ powers of two
// dg and du can be far outside of fp16's range where the gradients that come of them are not: each block of
// 64 rows and 64 hidden values has a power 2^e of its own, with which its largest finite magnitude is
// in 2^7 .. 2^15, so that what is 2^-21 of it still has all digits. The products' sums are kept at the power of
// the present step's block, and moved to the next one's where it is another: e goes in steps of 8, so that this is
// rare. (e of 40 at most: a larger one would save what is below 2^-65, and could bring sums of 2^87 to
// infinity.) Blocks of zeros have none. 16,384 rows of 1,024 x 4,096, gradient: 811 us, 772 without powers, 890 where
// every block has another than the next.
template <class T>
constexpr bool kPowers = false;
template <>
constexpr bool kPowers<Fp16> = true;
constexpr int kNoPower = 127, kMaxPower = 40, kPowerBlock = 64;

__device__ inline int power_of(float most) {
  const int k = (int)(__builtin_bit_cast(uint32_t, most) >> 23) - 127;
  return most > 0.f ? min((14 - k) >> 3 << 3, kMaxPower) : kNoPower;
}
__device__ inline float two_to(int e) { return e == kNoPower ? 1.f : word_float((uint32_t)(e + 127) << 23); }

// Largest finite magnitude of N sums, over the wavefront: with 0 times itself added, what is not finite is NaN,
// which fmaxf passes over.
template <int N>
__device__ inline float most_of(const f32x16 *x) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) m = fmaxf(m, fmaf(fabsf(x[i][r]), 0.f, fabsf(x[i][r])));
  return wave_max(m);
}

// ------------------------------------------------------------------ both projections
// What the gradient's products read: dg and du [rows][hidden], and their blocks' exponents [2][rows / 64][hidden / 64]
// (fp16).
struct HiddenGrads {
  char *dg, *du;
  int32_t *powers;
};
// BM rows of x and BN / 2 hidden values per block, WM x WN wavefronts, each of 32 C hidden values. With
// GROUPS 2 a block has two such groups of wavefronts, each with half of the summed axis and places in LDS of
// its own, and one tile: where tiles are few, what counts is how long a step takes, not how many run at once.
// The groups hand each other half of their sums in the end.
template <class T, int BM, int BN, int WM, int WN, int GROUPS, int ACT, bool GRAD>
__global__ __launch_bounds__(64 * WM * WN * GROUPS, 2) void gated_kernel(GatedGradArgs g, HiddenGrads to,
                                                                      int nm, int nn) {
  constexpr int W = WM * WN, TM = BM / 32 / WM, C = BN / 64 / WN;
  extern __shared__ char stages[];
  constexpr int kHalf = BN / 2 * kStepBytes, kStage = (BM + BN) * kStepBytes;
  typedef Exchange<C> Swap;
  // (the copies' second half is x's)
  static_assert(BM * kStepBytes >= W * Swap::kBytes);
  static_assert(2 * Side<false, BN / 2, W>::kCopies == Side<false, BM, W>::kCopies);
  const GatedArgs &a = g.f;
  const int lane = threadIdx.x & 63, waves = uniform(threadIdx.x >> 6);
  const int group = GROUPS > 1 ? waves / W : 0, wave = GROUPS > 1 ? waves % W : waves;
  const int wm = wave / WN, wn = wave % WN;
  const unsigned all = (unsigned)nm * nn;
  Tile t = tile_of(blockIdx.x, all, nm, nn);                // whose products are summed
  Tile next = t;                                            // whose operands are copied
  typedef Side<false, BN / 2, W> Half;
  typedef Side<false, BM, W> Whole;
  Half gate, up;
  Whole x;
  gate.init(a.w_gate, (int64_t)t.n * (BN / 2), a.hidden, a.gate_row, wave, lane);
  up.init(a.w_up, (int64_t)t.n * (BN / 2), a.hidden, a.up_row, wave, lane);
  x.init(a.x, (int64_t)t.m * BM, a.rows, a.x_row, wave, lane);
  const uint32_t lds = lds_address(stages) + group * (2 * kStage);
  f32x16 acc[TM][2][C];
  auto clear = [&] {
#pragma unroll
    for (int j = 0; j < TM; ++j)
#pragma unroll
      for (int i = 0; i < 2 * C; ++i) acc[j][i / C][i % C] = f32x16{0.f};
  };
  clear();
  struct Operands {
    u32x4 w[2][C], x[TM];
  };
  // The gradient: sums j become dg and du of rows 32 at .. of a wavefront's of tile `of` ...
  auto form = [&](int j, int at, const Tile &of, const Swap &swap) {
    const int64_t n = (int64_t)of.n * (BN / 2) + 32 * C * wn, bytes = 2 * (a.hidden - n);
    const int64_t row = (int64_t)of.m * BM + wm * (BM / WM) + 32 * at, rows = a.rows - row;
    f32x16 *u = acc[j][0], *v = acc[j][1];
    if constexpr (GRAD) {
      u32x4 dy[Swap::kCount];
#pragma unroll
      for (int i = 0; i < Swap::kCount; ++i) {
        dy[i] = u32x4{0, 0, 0, 0};
        if (swap.within(i, rows, bytes))
          dy[i] = *reinterpret_cast<const u32x4 *>(g.dout + row * g.dout_row + 2 * n +
                                                   swap.offset(i, g.dout_row));
      }
#pragma unroll
      for (int i = 0; i < Swap::kCount; ++i) swap.put_row(i, dy[i]);
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          __builtin_amdgcn_sched_barrier(0);       // (a few at a time: registers)
          const u32x2 w = swap.get(c, q);
          const uint32_t w0 = w[0], w1 = w[1];
          const float y[4] = {T::lo(w0), T::hi(w0), T::lo(w1), T::hi(w1)};
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            float f, d;
            activation<ACT>(u[c][4 * q + r], f, d);
            u[c][4 * q + r] = y[r] * v[c][4 * q + r] * d;
            v[c][4 * q + r] = y[r] * f;
          }
        }
      __builtin_amdgcn_wave_barrier();
    }
  };
  // ... which are scaled and stored; else the forward pass's results.
  float scale_g = 1.f, scale_u = 1.f;
  auto finish = [&](int j, int at, const Tile &of, const Swap &swap) {
    const int64_t n = (int64_t)of.n * (BN / 2) + 32 * C * wn, bytes = 2 * (a.hidden - n);
    const int64_t row = (int64_t)of.m * BM + wm * (BM / WM) + 32 * at, rows = a.rows - row;
    f32x16 *u = acc[j][0], *v = acc[j][1];
    if constexpr (GRAD) {
      if constexpr (kPowers<T>)
#pragma unroll
        for (int c = 0; c < C; ++c) u[c] *= scale_g, v[c] *= scale_u;
      const int64_t stride = (int64_t)a.hidden * 2, offset = row * stride + 2 * n;
      swap.template put_all<T>(u);
      __builtin_amdgcn_wave_barrier();
      swap.store(to.dg + offset, stride, rows, bytes);
      __builtin_amdgcn_wave_barrier();
      swap.template put_all<T>(v);
      __builtin_amdgcn_wave_barrier();
      swap.store(to.du + offset, stride, rows, bytes);
      __builtin_amdgcn_wave_barrier();
    } else {
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          float f, d;
          activation<ACT>(u[c][i], f, d);
          u[c][i] = f * v[c][i];
        }
      swap.template put_all<T>(u);
      __builtin_amdgcn_wave_barrier();
      swap.store(a.out + row * a.out_row + 2 * n, a.out_row, rows, bytes);
    }
  };
  // The powers of the dg and du that a wavefront has formed in sums 0 .. SUMS - 1; a block of 64 x 64 is one
  // wavefront's, or of all that have its rows.
  constexpr int SUMS = GROUPS > 1 ? 1 : TM;
  auto find_powers = [&](const Tile &of) {
    if constexpr (GRAD && kPowers<T>) {
      static_assert(BM / WM == kPowerBlock && (C == 2 || (C == 1 && WN == 2)));
      float big[2] = {0.f, 0.f};
#pragma unroll
      for (int j = 0; j < SUMS; ++j)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          big[q] = fmaxf(big[q], most_of<C>(acc[j][q]));
          __builtin_amdgcn_sched_barrier(0);
        }
      if constexpr (C == 1) {
        // (behind the stages, whose addresses are multiples of their rows' swizzles)
        typedef __attribute__((address_space(3))) float lds_float;
        lds_float *most = (lds_float *)(uintptr_t)(lds_address(stages) + 2 * GROUPS * kStage);
        if (lane < 2) most[2 * (group * W + wave) + lane] = big[lane];
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
          for (int i = 0; i < GROUPS * WN; ++i)
            big[q] = fmaxf(big[q], most[2 * (i / WN * W + wm * WN + i % WN) + q]);
      }
      const int eg = uniform(power_of(big[0])), eu = uniform(power_of(big[1]));
      scale_g = two_to(eg), scale_u = two_to(eu);
      const int64_t nr = (a.rows + kPowerBlock - 1) / kPowerBlock, nh = (a.hidden + kPowerBlock - 1) / kPowerBlock;
      const int64_t r = (int64_t)of.m * (BM / kPowerBlock) + wm;
      const int64_t h = ((int64_t)of.n * (BN / 2) + 32 * C * wn) / kPowerBlock;
      if (lane < 2 && group == 0 && (C == 2 || wn == 0) && r < nr && h < nh)
        to.powers[(lane * nr + r) * nh + h] = lane ? eu : eg;
    }
  };
  // a tile's steps follow those of the block's tile before without a pause. Each row of tiles starts at
  // another step: rows a power of two apart meet in few of the L2's channels (263 us without, 259 with it)
  const int total = (a.width + kStep - 1) / kStep, steps = (total + GROUPS - 1) / GROUPS;
  const int first = group * steps;                         // a group's steps
  const int mine = GROUPS > 1 ? max(1, min(steps, total - first)) : steps;
  unsigned index = blockIdx.x, current = blockIdx.x;       // of next and of t (two tiles apart, with one step a tile)
  int step = -1, left = steps;           // of next's, the one whose operands are copied; those left of t's
  int64_t k0 = 0;
  bool on = true;
  run_steps<Operands, 2 * Half::kCopies + Whole::kCopies, 2 * C * TM, TM + 2 * C>(
      GROUPS > 1 ? steps : (int64_t)steps * ((all - blockIdx.x + gridDim.x - 1) / gridDim.x),
      [&](int64_t) {
        ++step;
        if (GROUPS > 1) {
          on = step < steps && first + step < total;
        } else if (step == steps) {
          step = 0;
          index += gridDim.x;
          on = index < all;
          if (on) {
            next = tile_of(index, all, nm, nn);
            gate.move(a.w_gate, (int64_t)next.n * (BN / 2), a.hidden);
            up.move(a.w_up, (int64_t)next.n * (BN / 2), a.hidden);
            x.move(a.x, (int64_t)next.m * BM, a.rows);
          }
        }
        const int at = step + next.m % mine;
        k0 = on ? (int64_t)(first + (at >= mine ? at - mine : at)) * kStep : 0;
      },
      [&](int stage, int i) {
        const uint32_t to = lds + stage * kStage;
        constexpr int H = Half::kCopies;
        if (i < H) gate.copy(i, on, k0, a.width, to);
        else if (i < 2 * H) up.copy(i - H, on, k0, a.width, to + kHalf);
        else x.copy(i - 2 * H, on, k0, a.width, to + 2 * kHalf);
      },
      [&](int stage, int s, int i, Operands &o) {
        const uint32_t at = lds + stage * kStage;
        if (i < 2 * C)
          o.w[i / C][i % C] = gate.operand(gate.at(at + wn * (32 * C * kStepBytes)) + i / C * kHalf, i % C, s);
        else
          o.x[i - 2 * C] = x.operand(x.at(at + 2 * kHalf + wm * (BM / WM * kStepBytes)), i - 2 * C, s);
      },
      [&](const Operands &o, int i) {
        const int j = i / (2 * C), q = i % (2 * C) / C, c = i % C;
        acc[j][q][c] = T::mfma(o.w[q][c], o.x[j], acc[j][q][c]);
      },
      [&](int64_t, int stage) {
        if (GROUPS > 1 || --left) return false;
        left = steps;
        // (x's part of the stage: its copies go out last, after the block has met)
        int here = lane;
        if (GRAD) asm volatile("" : "+v"(here));         // (addresses are made here, not kept through the steps)
        const Swap swap = {lds + stage * kStage + 2 * kHalf + wave * Swap::kBytes, here};
        if constexpr (GRAD && kPowers<T>) {
#pragma unroll
          for (int j = 0; j < TM; ++j) {
            form(j, j, t, swap);
            __builtin_amdgcn_sched_barrier(0);           // (one at a time: registers)
          }
          find_powers(t);
        }
#pragma unroll
        for (int j = 0; j < TM; ++j) {
          if constexpr (!kPowers<T>) form(j, j, t, swap);
          finish(j, j, t, swap);
          __builtin_amdgcn_sched_barrier(0);
        }
        current += gridDim.x;
        if (current < all) t = tile_of(current, all, nm, nn);
        clear();
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        return true;
      });
  if constexpr (GROUPS > 1) {
    static_assert(GROUPS == 2 && TM == 2 && C == 1);
    static_assert(kHandOver<W> + 2 * W * Swap::kBytes <= 4 * kStage);
    const Swap swap = {lds_address(stages) + kHandOver<W> + (group * W + wave) * Swap::kBytes, lane};
    hand_over<W>(lds_address(stages), group, wave, lane, reinterpret_cast<f32x16 (&)[2][2]>(acc));
    form(0, group, t, swap);
    find_powers(t);
    finish(0, group, t, swap);
  }
}

// ------------------------------------------------------------------ few rows
// Both projections of up to 16 N rows a block: what counts is that the weights stream in. A block has 16
// hidden values; its wavefronts split the summed axis, each with four times 32 of it on its way at once,
// straight into the matrix units' registers, and are added up in LDS in order.
constexpr int kFewWaves = 8;

template <class T>
__device__ inline f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c);
template <>
__device__ inline f32x4 mfma16<Bf16>(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b),
                                                 c, 0, 0, 0);
}
template <>
__device__ inline f32x4 mfma16<Fp16>(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c,
                                                0, 0, 0);
}

template <class T, int N, int ACT>
__global__ __launch_bounds__(64 * kFewWaves) void gated_few(GatedArgs a) {
  constexpr int kUnroll = 4;
  // A lane has row lane % 16 of an operand, values 8 (lane / 16) .. of 32, and of a result row
  // (hidden value) 4 (lane / 16) + 0..3 and column (row of x) lane % 16.
  __shared__ f32x4 sums[kFewWaves][2 * N][64];
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int64_t n0 = (int64_t)blockIdx.x * 16, m0 = (int64_t)blockIdx.y * (16 * N);
  const int r = lane & 15, off = (lane >> 4) * 16;
  const int chunks = (a.width + 31) / 32, per = (chunks + kFewWaves - 1) / kFewWaves;
  const int first = wave * per, end = min(first + per, chunks);
  const int64_t n = min(n0 + r, (int64_t)a.hidden - 1);   // (results past the last are not stored)
  const char *src[2 + N];
  src[0] = a.w_gate + n * a.gate_row + off;
  src[1] = a.w_up + n * a.up_row + off;
#pragma unroll
  for (int j = 0; j < N; ++j) src[2 + j] = a.x + min(m0 + 16 * j + r, (int64_t)a.rows - 1) * a.x_row + off;
  f32x4 acc[2][N];
#pragma unroll
  for (int j = 0; j < N; ++j) acc[0][j] = acc[1][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int c = first; c < end; c += kUnroll) {
    u32x4 v[kUnroll][2 + N];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const bool in = c + u < end && (c + u) * 64 + off < 2 * a.width;
#pragma unroll
      for (int i = 0; i < 2 + N; ++i) {
        v[u][i] = u32x4{0, 0, 0, 0};
        if (in) v[u][i] = *reinterpret_cast<const u32x4 *>(src[i] + (int64_t)(c + u) * 64);
      }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        acc[0][j] = mfma16<T>(v[u][0], v[u][2 + j], acc[0][j]);
        acc[1][j] = mfma16<T>(v[u][1], v[u][2 + j], acc[1][j]);
      }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < N; ++j) sums[wave][i * N + j][lane] = acc[i][j];
  __syncthreads();
  // a wavefront joins 16 rows of x
  for (int j = wave; j < N; j += kFewWaves) {
    f32x4 g = sums[0][j][lane], u = sums[0][N + j][lane];
#pragma unroll
    for (int w = 1; w < kFewWaves; ++w) g += sums[w][j][lane], u += sums[w][N + j][lane];
    float f[4], d;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      activation<ACT>(g[i], f[i], d);
      f[i] *= u[i];
    }
    const int64_t row = m0 + 16 * j + r, to = n0 + 4 * (lane >> 4);
    if (row < a.rows && to < a.hidden)
      *reinterpret_cast<u32x2 *>(a.out + row * a.out_row + 2 * to) =
          u32x2{T::pack(f[0], f[1]), T::pack(f[2], f[3])};
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
  // fp16: exponents of B's blocks, one for 64 of m and a step: of the segment or output with power_all,
  // power_m and power_k apart
  const int32_t *powers;
  int64_t power_all, power_m, power_k;
  int64_t m, n, k;
  int nm, nn, splits;
};

template <class T, int BM, int BN, int WM, int WN, int GROUPS, bool B_COL, int SEGMENTS>
__device__ inline void product_tile(const ProductArgs &p, unsigned block) {
  constexpr int W = WM * WN, TM = BM / 32 / WM, TN = BN / 32 / WN;
  extern __shared__ char stages[];
  constexpr int kStage = (BM + BN) * kStepBytes, kA = BN * kStepBytes;
  typedef Side<true, BN, W> ASide;
  typedef Side<B_COL, BM, W> BSide;
  const int lane = threadIdx.x & 63, waves = uniform(threadIdx.x >> 6);
  const int group = GROUPS > 1 ? waves / W : 0, wave = GROUPS > 1 ? waves % W : waves;
  const int wm = wave / WN, wn = wave % WN;
  const unsigned all = (unsigned)p.nm * p.nn;
  const int part = (int)(block / all), output = part / p.splits, split = part % p.splits;
  const Tile t = tile_of(block - part * all, all, p.nm, p.nn);
  const int64_t m0 = (int64_t)t.m * BM, n0 = (int64_t)t.n * BN;
  const int per = (int)((p.k + kStep - 1) / kStep), steps = per * SEGMENTS;
  // a block's steps, or a group's: the first one's as many as the second's or one more
  const int begin = (int)((int64_t)steps * split / p.splits);
  const int behind = (int)((int64_t)steps * (split + 1) / p.splits), half = (behind - begin + 1) / 2;
  const int first = begin + group * half, end = GROUPS > 1 && group == 0 ? begin + half : behind;
  const int skew = !B_COL && end > first ? t.m % (end - first) : 0;
  ASide a;
  BSide b;
  int segment = SEGMENTS == 2 ? (first + skew >= per) : output;
  a.init(p.a[segment], n0, p.n, p.a_row[segment], wave, lane);
  b.init(p.b[segment], m0, p.m, p.b_row[segment], wave, lane);
  const uint32_t lds = lds_address(stages) + group * (2 * kStage);
  f32x16 acc[TM][TN];
#pragma unroll
  for (int j = 0; j < TM; ++j)
#pragma unroll
    for (int i = 0; i < TN; ++i) acc[j][i] = f32x16{0.f};
  struct Operands {
    u32x4 a[TN], b[TM];
  };
  // The power that a wavefront's sums are kept at, for each 64 of its m, and that of the next step. (Through the
  // constant address space: scalar loads, which no copy has to be waited for.)
  constexpr int POWERS = kPowers<T> ? BM / WM / kPowerBlock : 0;
  typedef __attribute__((address_space(4))) const int32_t const_int;
  int power[POWERS + 1] = {}, coming[POWERS + 1] = {};
  auto fetch = [&](int i) {
    if (POWERS == 0 || first + i >= end) return;
    int step = first + i + skew;
    step = step >= end ? step - (end - first) : step;
    const int of = SEGMENTS == 2 ? step >= per : output;
    step -= SEGMENTS == 2 ? of * per : 0;
#pragma unroll
    for (int q = 0; q < POWERS; ++q) {
      const int64_t block = min((m0 + wm * (BM / WM)) / kPowerBlock + q, (p.m - 1) / kPowerBlock);
      coming[q] = ((const_int *)(uintptr_t)p.powers)[of * p.power_all + block * p.power_m + step * p.power_k];
    }
  };
  // sums j .. of a 64 of m times 2^e
  auto lift = [&](int q, int e) {
    constexpr int kSums = kPowerBlock / 32;
#pragma unroll
    for (int j = q * kSums; j < (q + 1) * kSums; ++j)
#pragma unroll
      for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[j][i][r] = __builtin_amdgcn_ldexpf(acc[j][i][r], e);
  };
  fetch(0);
#pragma unroll
  for (int q = 0; q < POWERS; ++q) power[q] = coming[q] == kNoPower ? 0 : coming[q];
  fetch(1);
  bool on = true;                        // copies of a step that there is, from k0 on
  int64_t k0 = 0;
  run_steps<Operands, ASide::kCopies + BSide::kCopies, TM * TN, TN + TM>(
      GROUPS > 1 ? half : end - first,
      [&](int64_t i) {
        int step = first + (int)i;
        on = step < end;
        step += skew;
        step = step >= end ? step - (end - first) : step;
        if (SEGMENTS == 2) {
          const int now = step >= per;
          if (now != segment && on) {
            segment = now;
            a.init(p.a[now], n0, p.n, p.a_row[now], wave, lane);
            b.init(p.b[now], m0, p.m, p.b_row[now], wave, lane);
          }
          step -= now * per;
        }
        k0 = on ? (int64_t)step * kStep : 0;
      },
      [&](int stage, int i) {
        if (i < ASide::kCopies) a.copy(i, on, k0, p.k, lds + stage * kStage);
        else b.copy(i - ASide::kCopies, on, k0, p.k, lds + stage * kStage + kA);
      },
      [&](int stage, int s, int i, Operands &o) {
        if (i < TN) o.a[i] = a.operand(a.at(lds + stage * kStage), wn * TN + i, s);
        else o.b[i - TN] = b.operand(b.at(lds + stage * kStage + kA), wm * TM + i - TN, s);
      },
      [&](const Operands &o, int i) {
        acc[i / TN][i % TN] = T::mfma(o.a[i % TN], o.b[i / TN], acc[i / TN][i % TN]);
      },
      [&](int64_t i, int) {
#pragma unroll
        for (int q = 0; q < POWERS; ++q)
          if (coming[q] != power[q] && coming[q] != kNoPower) {
            lift(q, coming[q] - power[q]);
            power[q] = coming[q];
          }
        fetch((int)i + 2);
        return false;
      });
#pragma unroll
  for (int q = 0; q < POWERS; ++q) lift(q, -power[q]);
  typedef Exchange<TN> Swap;
  const int64_t n = n0 + wn * (BN / WN);
  auto finish = [&](int j, int at, const Swap &swap) {
    const int64_t row = m0 + wm * (BM / WM) + 32 * at;
    if (p.splits == 1) {
      swap.template put_all<T>(acc[j]);
      __builtin_amdgcn_wave_barrier();
      swap.store(p.out[output] + row * p.out_row[output] + 2 * n, p.out_row[output], p.m - row,
                 2 * (p.n - n));
      __builtin_amdgcn_wave_barrier();
    } else if (row + (lane & 31) < p.m) {
      float *to = p.part + (((int64_t)output * p.splits + split) * p.m + row + (lane & 31)) * p.n + n;
#pragma unroll
      for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int off = 32 * i + 8 * q + 4 * (lane >> 5);
          if (n + off < p.n)
            *reinterpret_cast<f32x4 *>(to + off) =
                f32x4{acc[j][i][4 * q], acc[j][i][4 * q + 1], acc[j][i][4 * q + 2], acc[j][i][4 * q + 3]};
        }
    }
  };
  if constexpr (GROUPS == 1) {
    static_assert(2 * kStage >= W * Swap::kBytes);
    const Swap swap = {lds + wave * Swap::kBytes, lane};
    __syncthreads();                     // (all of the block's operands have been read)
#pragma unroll
    for (int j = 0; j < TM; ++j) finish(j, j, swap);
  } else {
    static_assert(GROUPS == 2 && kHandOver<W> + 2 * W * Swap::kBytes <= 4 * kStage);
    const Swap swap = {lds_address(stages) + kHandOver<W> + (group * W + wave) * Swap::kBytes, lane};
    hand_over<W>(lds_address(stages), group, wave, lane, acc);
    finish(0, group, swap);
  }
}

// All three products in one launch, so that one kind's tiles fill up the places that the other's leave:
// first the `head` blocks of the kind with the longer tiles.
template <class T, int BM, int BN, int WM, int WN, int GROUPS>
__global__ __launch_bounds__(64 * WM * WN * GROUPS, 2) void products_kernel(ProductArgs x, ProductArgs w, int head,
                                                                bool x_first) {
  const bool front = (int)blockIdx.x < head;
  const unsigned block = front ? blockIdx.x : blockIdx.x - head;
  if (front == x_first) product_tile<T, BM, BN, WM, WN, GROUPS, false, 2>(x, block);
  else product_tile<T, BM, BN, WM, WN, GROUPS, true, 1>(w, block);
}

// out = the sum of the splits' parts, 8 values a thread: dx, dWg and dWu in turn (blockIdx.y).
template <class T>
__global__ __launch_bounds__(256) void product_add(ProductArgs x, ProductArgs w) {
  const ProductArgs &p = blockIdx.y ? w : x;
  const int output = blockIdx.y ? blockIdx.y - 1 : 0;
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8, size = p.m * p.n;
  if (i >= size || p.splits == 1) return;
  const float *from = p.part + (int64_t)output * p.splits * size + i;
  f32x4 u = *reinterpret_cast<const f32x4 *>(from), v = *reinterpret_cast<const f32x4 *>(from + 4);
  for (int s = 1; s < p.splits; ++s) {
    const f32x4 *q = reinterpret_cast<const f32x4 *>(from + s * size);
    u += q[0], v += q[1];
  }
  const int64_t row = i / p.n;
  *reinterpret_cast<u32x4 *>(p.out[output] + row * p.out_row[output] + 2 * (i - row * p.n)) =
      u32x4{T::pack(u[0], u[1]), T::pack(u[2], u[3]), T::pack(v[0], v[1]), T::pack(v[2], v[3])};
}

// ------------------------------------------------------------------ launches
int64_t tiles(int64_t n, int size) { return (n + size - 1) / size; }
size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

// Tiles of 256 x 256 where those of 128 x 128 are more than are resident at once. Measured, us, large and small:
// 2,048 x 1,024 x 2,048 (512 small tiles) 27.7 and 21.5, 4,096 x 1,024 x 1,024 (512) 28.4 and 27.0, 1,408 hidden
// values (704) 29.2 and 37.9, 2,048 (1,024) 33.9 and 41.4; 8,192 x 256 x 1,024 (1,024) 15.1 and 17.1.
bool use_big(int64_t rows, int64_t hidden) { return tiles(rows, 128) * tiles(hidden, 64) > 2 * kSeqCus; }

// Two groups of wavefronts a tile where each tile has a compute unit of its own, and sums long enough to pay
// for the exchange (1024 x 1024: from 1024 wide 10.3 us, 12.7 with one group; 256 wide 6.1 both; 64 wide 5.2 and 4.3).
bool use_groups(int64_t rows, int64_t width, int64_t hidden) {
  return width > 4 * kStep && tiles(rows, 128) * tiles(hidden, 64) <= kSeqCus;
}

template <class T, int BM, int BN, int WM, int WN, int GROUPS, int ACT, bool GRAD>
hipError_t launch_projections(const GatedGradArgs &g, const HiddenGrads &to, hipStream_t s) {
  constexpr int kMost = GRAD && kPowers<T> ? 2 * GROUPS * WM * WN * 4 : 0;
  constexpr int kLds = 2 * GROUPS * (BM + BN) * kStepBytes + kMost, kResident = kLdsBytes / kLds * kSeqCus;
  static LdsLimit limit;
  const void *f = reinterpret_cast<const void *>(gated_kernel<T, BM, BN, WM, WN, GROUPS, ACT, GRAD>);
  const hipError_t e = limit.set(f, kLds);
  if (e != hipSuccess) return e;
  const int nm = (int)tiles(g.f.rows, BM), nn = (int)tiles(g.f.hidden, BN / 2);
  gated_kernel<T, BM, BN, WM, WN, GROUPS, ACT, GRAD>
      <<<(unsigned)(GROUPS > 1 ? nm * nn : std::min(nm * nn, kResident)), 64 * WM * WN * GROUPS, kLds, s>>>(
          g, to, nm, nn);
  return hipGetLastError();
}
// Whether the weights stream past the rows: up to 32 rows, and more where a block for each 16 hidden values and
// 64 rows has a compute unit of its own. Measured, us, this form and tiles: 16 rows of 1,024 x 4,096 5.0 and
// 10.0, 64 rows 8.2 and 10.1, 96 rows (512 blocks) 13.1 and 10.2; 256 rows of 4,096 x 1,024 24.3 and 28.3, of
// 256 x 1,024 4.2 and 5.9; of 2,048 x 8,192 32 rows 18.1 and 21.1, 64 rows (512 blocks) 26.7 and 21.3.
bool use_few(int64_t rows, int64_t hidden) {
  return rows <= 32 || tiles(hidden, 16) * tiles(rows, 64) <= kSeqCus;
}
template <class T, int N, int ACT>
hipError_t launch_few(const GatedArgs &a, hipStream_t s) {
  gated_few<T, N, ACT><<<dim3((unsigned)tiles(a.hidden, 16), (unsigned)tiles(a.rows, 16 * N)), 64 * kFewWaves, 0, s>>>(a);
  return hipGetLastError();
}
template <class T, int ACT, bool GRAD>
hipError_t projections(const GatedGradArgs &g, const HiddenGrads &to, hipStream_t s) {
  if (!GRAD && use_few(g.f.rows, g.f.hidden)) {
    if (g.f.rows <= 16) return launch_few<T, 1, ACT>(g.f, s);
    if (g.f.rows <= 32) return launch_few<T, 2, ACT>(g.f, s);
    return launch_few<T, 4, ACT>(g.f, s);
  }
  if (use_big(g.f.rows, g.f.hidden))
    return launch_projections<T, 256, 256, 4, 2, 1, ACT, GRAD>(g, to, s);
  if (use_groups(g.f.rows, g.f.width, g.f.hidden))
    return launch_projections<T, 128, 128, 2, 2, 2, ACT, GRAD>(g, to, s);
  return launch_projections<T, 128, 128, 2, 2, 1, ACT, GRAD>(g, to, s);
}
template <bool GRAD>
hipError_t by_type(const GatedGradArgs &g, const HiddenGrads &to, hipStream_t s) {
  if (g.f.fp16)
    return g.f.act == kSilu ? projections<Fp16, kSilu, GRAD>(g, to, s) : projections<Fp16, kGelu, GRAD>(g, to, s);
  return g.f.act == kSilu ? projections<Bf16, kSilu, GRAD>(g, to, s) : projections<Bf16, kGelu, GRAD>(g, to, s);
}

// The products' tiles, and the parts of their summed axes.
struct Plan {
  bool big, groups;
  int sx, sw;                          // parts of dx's and of dW's summed axis
  int64_t nx, nw, lx, lw;              // blocks, and a block's steps
};
// Steps of a part at least: 1,021 x 520 x 1,368 in fp16 with one group of wavefronts a tile and 8 20.9 us and 5.2 for
// adding the parts, with 16 25.7 and 4.3, with 4 20.9 and 5.5; with two groups and 8 20.0 and 4.3, with 16 22.5 and 4.1.
constexpr int kLeast = 8;
Plan plan_of(int64_t rows, int64_t width, int64_t hidden, bool big, bool groups) {
  const int size = big ? 256 : 128;
  const int64_t tx = tiles(rows, size) * tiles(width, size), tw = 2 * tiles(hidden, size) * tiles(width, size);
  const int64_t lx = 2 * tiles(hidden, kStep), lw = tiles(rows, kStep);
  // a resident block's share of all steps: longer summed axes are split
  const int64_t places = big || groups ? kSeqCus : 2 * kSeqCus;
  const int64_t share = std::max<int64_t>(kLeast, tiles(tx * lx + tw * lw, places));
  Plan p;
  p.big = big, p.groups = groups;
  // (of no rows there is no dx to split: its parts would be added up by a launch without blocks)
  p.sx = tx > 0 ? (int)std::max<int64_t>(1, lx / share) : 1, p.sw = (int)std::max<int64_t>(1, lw / share);
  p.nx = tx * p.sx, p.nw = tw * p.sw;
  p.lx = tiles(lx, p.sx), p.lw = tiles(lw, p.sw);
  return p;
}
// By the time of a step of either size, measured with full tiles: 1.8 us of 256 x 256, one block a compute
// unit; 1.2 of 128 x 128, two. Two groups of wavefronts a tile where each block has a compute unit of its own and
// more steps than a few: the gradient of 1,021 x 2,048 x 512 36 us, 49 with one group; 1,024 x 1,024 x 1,024 33 and
// 39; 1,021 x 520 x 1,368 34.1 and 35.7 (fp16: 35.6 and 37.6); 128 x 64 x 64, of two steps, 12.1 and 11.3.
Plan plan_of(int64_t rows, int64_t width, int64_t hidden) {
  const Plan a = plan_of(rows, width, hidden, true, false), b = plan_of(rows, width, hidden, false, false);
  auto time = [](const Plan &p, double step, int places) {
    return step * std::max<double>((double)std::max(p.lx, p.lw), (double)(p.nx * p.lx + p.nw * p.lw) / places);
  };
  if (time(a, 1.8, kSeqCus) <= time(b, 1.2, 2 * kSeqCus)) return a;
  const Plan c = plan_of(rows, width, hidden, false, true);
  return c.nx + c.nw <= kSeqCus && std::max(c.lx, c.lw) > 4 ? c : b;
}
size_t part_bytes(const Plan &p, int64_t rows, int64_t width, int64_t hidden, bool x) {
  if (x) return p.sx > 1 ? align256((size_t)p.sx * rows * width * 4) : 0;
  return p.sw > 1 ? align256((size_t)2 * p.sw * hidden * width * 4) : 0;
}

size_t power_bytes(int64_t rows, int64_t hidden) {
  return align256((size_t)2 * tiles(rows, kPowerBlock) * tiles(hidden, kPowerBlock) * 4);
}

template <class T, int BM, int BN, int WM, int WN, int GROUPS>
hipError_t launch_products(ProductArgs x, ProductArgs w, const Plan &plan, hipStream_t s) {
  constexpr int kLds = 2 * GROUPS * (BM + BN) * kStepBytes;
  static LdsLimit limit;
  const void *f = reinterpret_cast<const void *>(products_kernel<T, BM, BN, WM, WN, GROUPS>);
  hipError_t e = limit.set(f, kLds);
  if (e != hipSuccess) return e;
  for (ProductArgs *p : {&x, &w}) p->nm = (int)tiles(p->m, BM), p->nn = (int)tiles(p->n, BN);
  const bool x_first = plan.lx > plan.lw;
  products_kernel<T, BM, BN, WM, WN, GROUPS><<<(unsigned)(plan.nx + plan.nw), 64 * WM * WN * GROUPS, kLds, s>>>(
      x, w, (int)(x_first ? plan.nx : plan.nw), x_first);
  e = hipGetLastError();
  if (e != hipSuccess || (x.splits == 1 && w.splits == 1)) return e;
  const int64_t most = std::max(x.splits > 1 ? x.m * x.n : 0, w.splits > 1 ? w.m * w.n : 0);
  product_add<T><<<dim3((unsigned)tiles(most, 256 * 8), 3), 256, 0, s>>>(x, w);
  return hipGetLastError();
}

template <class T>
hipError_t gradient(const GatedGradArgs &g, char *ws, hipStream_t s) {
  const GatedArgs &f = g.f;
  const Plan plan = plan_of(f.rows, f.width, f.hidden);
  const size_t hidden_bytes = align256((size_t)f.rows * f.hidden * 2);
  char *dg = ws, *du = ws + hidden_bytes;
  ws += 2 * hidden_bytes;
  int32_t *powers = reinterpret_cast<int32_t *>(ws);
  ws += f.fp16 ? power_bytes(f.rows, f.hidden) : 0;
  float *px = reinterpret_cast<float *>(ws);
  float *pw = reinterpret_cast<float *>(ws + part_bytes(plan, f.rows, f.width, f.hidden, true));
  const int64_t row = (int64_t)f.hidden * 2;
  const int64_t nr = tiles(f.rows, kPowerBlock), nh = tiles(f.hidden, kPowerBlock);
  if (f.rows > 0) {
    const hipError_t e = by_type<true>(g, {dg, du, powers}, s);
    if (e != hipSuccess) return e;
  }
  const ProductArgs x = {{f.w_gate, f.w_up}, {dg, du}, {f.gate_row, f.up_row}, {row, row}, {g.dx, nullptr},
                         {g.dx_row, 0}, px, powers, nr * nh, nh, 1, f.rows, f.width, f.hidden, 0, 0, plan.sx};
  const ProductArgs w = {{f.x, f.x}, {dg, du}, {f.x_row, f.x_row}, {row, row}, {g.dw_gate, g.dw_up},
                         {g.dgate_row, g.dup_row}, pw, powers, nr * nh, 1, nh, f.hidden, f.width, f.rows, 0, 0, plan.sw};
  if (plan.big) return launch_products<T, 256, 256, 2, 4, 1>(x, w, plan, s);
  return plan.groups ? launch_products<T, 128, 128, 2, 2, 2>(x, w, plan, s)
                     : launch_products<T, 128, 128, 2, 2, 1>(x, w, plan, s);
}

}  // namespace

hipError_t launch_gated(const GatedArgs &a, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  GatedGradArgs g = {};
  g.f = a;
  return by_type<false>(g, HiddenGrads{}, s);
}

bool gated_fits(int64_t rows, int64_t width, int64_t hidden, bool grad) {
  // (at most 512 threads a block)
  constexpr int64_t kMost = kMaxBlocks / 2;
  bool ok = tiles(rows, 128) * tiles(hidden, 64) <= kMost;
  if (grad && ok) {
    const Plan a = plan_of(rows, width, hidden);
    ok = a.nx + a.nw <= kMost && tiles(std::max(rows, hidden) * width, 256 * 8) <= kMost;
  }
  return ok;
}

size_t gated_grad_bytes(int32_t rows, int32_t width, int32_t hidden, bool fp16) {
  const Plan p = plan_of(rows, width, hidden);
  return 2 * align256((size_t)rows * hidden * 2) + (fp16 ? power_bytes(rows, hidden) : 0) +
         part_bytes(p, rows, width, hidden, true) +
         part_bytes(p, rows, width, hidden, false);
}

hipError_t launch_gated_grad(const GatedGradArgs &g, void *ws, hipStream_t s) {
  return g.f.fp16 ? gradient<Fp16>(g, static_cast<char *>(ws), s)
                  : gradient<Bf16>(g, static_cast<char *>(ws), s);
}

}  // namespace bgp
