// Gradients of the attention in attend.hip. With P = softmax(S), dP = dO V^T and
// D_i = dO_i . O_i:
//   dS = P (dP - D),  dbias = dS,  dZ = dS (1 - (z' / cap)^2)  (z' the capped product)
//   dQ = scale dZ K,  dK = scale dZ^T Q,  dV = P^T dO
// P is recomputed from the scores and the forward pass's log-sums. Two kinds of blocks, so
// that every sum has one owner and one order (no atomics): one goes over the queries for 128
// keys of a key head (all query heads of its group, in turn) and keeps dK and dV, the other
// goes over the keys for 128 queries of a head and keeps dQ and the head's table gradient.
// That costs 7 products of the pairs where one kind with atomic sums of dQ would take 5.
//
// Large calls are bound as the forward kernel is: 8192 rows, causal, 16 heads of 128, slopes:
// grad_pairs 950-1030 us for 0.96 TFLOP of its 7 products, 0.93 to 1.0 PFLOP/s (matrix units busy
// for half of the cycles). 8862 rows in 16 documents, 16 heads of 64 with 4 of keys, prefix masks,
// cap and table: 162 us, where neither unit is the bound (vector 53% of the cycles, matrix 16%):
// two wavefronts per SIMD go through a chain of product, scores and product, 32 queries or keys at
// a time. 3 documents of up to 333, 6 heads of 80 with 2 of keys: 35 us, narrow blocks of about
// eight such steps, each head's biases built anew (wavefronts wait for 54% of their cycles).
//
// fp16: P is kept times 2^12 and dS times a power of two from a bound of |dS| in the document and
// head, 2 max|dO_i| max|v_j|, so that neither leaves fp16's normal range; exact to undo.
#include <type_traits>

#include "seq_dev.h"

namespace bgp {
namespace {

constexpr int kThreads = 256;
constexpr float kP16 = 12.f;       // fp16: log2 of the factor of P
constexpr int kSkew = 16 * 64;      // floats of a wavefront's skewed values

// Queries of a step of dK and dV: as many as leave room for three blocks of head size 64, or
// two of 128, in LDS. With 64 / 32 at head size 64: 16 documents of up to 1024 236 / 247 us, one of
// 8192, 16 heads with 2 of keys, 961 / 996; one of 4096, 16 heads, a table, 264 / 255.
constexpr int kv_step(int dp, bool narrow) { return narrow || dp == 128 ? 32 : 64; }

// Starts the copy of one word per lane into LDS.
__device__ inline void copy_words(u32x4 buf, int voff, uint32_t lds) {
  const uint32_t m = uniform((int)lds);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dword %1, %2, 0 offen lds"
               ::"s"(m), "v"(voff), "s"(buf)
               : "memory");
}

// Adds the four wavefronts' results; true on the one (the first) that has the sum then.
template <int DT>
__device__ __forceinline__ bool add_waves(f32x16 *acc, char *lds) {
  f32x4 *x = reinterpret_cast<f32x4 *>(lds);   // [3][DT][4][64]
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  __syncthreads();
  if (wave) {
#pragma unroll
    for (int c = 0; c < DT; ++c)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        x[(((wave - 1) * DT + c) * 4 + g) * 64 + lane] =
            f32x4{acc[c][4 * g], acc[c][4 * g + 1], acc[c][4 * g + 2], acc[c][4 * g + 3]};
  }
  __syncthreads();
  if (wave) return false;
  for (int w = 0; w < 3; ++w)
#pragma unroll
    for (int c = 0; c < DT; ++c)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 y = x[((w * DT + c) * 4 + g) * 64 + lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[c][4 * g + e] += y[e];
      }
  return true;
}

// ------------------------------------------------------------------ rows
// rows[head][row] = {log-sum in units of log 2, D = dO . (O + what its rounding took)} of the
// documents' rows. For fp16 also the largest |dO_i|^2 and |v_j|^2 of each 16 rows of a document,
// at the first of them (bound: [heads][q_rows], then [kv_heads][k_rows]): what lies outside the
// documents, and rows that saw nothing, take no part. A wavefront per 16 rows and head, 16 lanes
// per row. D is a difference's other half in dS, so it takes O at full precision: the rounding of O
// alone would double the error of dQ and dK. Bound by reading the three: 8192 rows of 16 heads of
// 128, 101 MB, 18.1 us, 5.6 TB/s.
constexpr int kRowTile = 16;
constexpr int kRowBlocks = 16384;  // blocks of the row pass, at most
template <class T>
__device__ inline float dot8(u32x4 a, u32x4 b) {
  float x = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x = __builtin_fmaf(T::lo(a[i]), T::lo(b[i]), x);
    x = __builtin_fmaf(T::hi(a[i]), T::hi(b[i]), x);
  }
  return x;
}

template <class T>
__global__ __launch_bounds__(kThreads) void grad_rows(const AttnGradArgs a, int64_t q_units,
                                                      int64_t units) {
  constexpr int kTurns = kRowTile / 4;   // 4 rows at a time
  const int lane = threadIdx.x & 63, l16 = lane & 15;
  const bool in = l16 * 16 < a.f.bytes;
  const u32x4 zero = {};
  for (int64_t u = (int64_t)blockIdx.x * 4 + uniform(threadIdx.x >> 6); u < units;
       u += (int64_t)gridDim.x * 4) {
    const bool keys = u >= q_units;
    const int heads = keys ? a.f.kv_heads : a.f.heads;
    const int64_t n = keys ? u - q_units : u;
    const int head = (int)(n % heads), tile = (int)(n / heads);
    const DocTile t = keys ? find_tile<kRowTile>(a.f.kb, a.f.ke, a.f.docs, a.f.k_rows, tile)
                           : find_tile<kRowTile>(a.f.qb, a.f.qe, a.f.docs, a.f.q_rows, tile);
    if (t.doc < 0) continue;
    const int first = t.b0 + t.tile * kRowTile, rows = min(t.b1 - first, kRowTile);
    float top = 0.f;
    if (keys) {
      u32x4 v[kTurns];
#pragma unroll
      for (int i = 0; i < kTurns; ++i) {
        const int r = 4 * i + (lane >> 4);
        v[i] = zero;
        if (r < rows && in)
          v[i] = *reinterpret_cast<const u32x4 *>(a.f.v + (int64_t)(first + r) * a.f.v_row +
                                                  head * a.f.v_head + l16 * 16);
      }
#pragma unroll
      for (int i = 0; i < kTurns; ++i) {
        top = fmaxf(top, row_sum(dot8<T>(v[i], v[i])));
      }
    } else {
      u32x4 g[kTurns], o[kTurns], e[kTurns];
      float lse[kTurns];
#pragma unroll
      for (int i = 0; i < kTurns; ++i) {
        const int r = 4 * i + (lane >> 4);
        const int64_t row = first + r;
        lse[i] = r < rows ? a.f.lse[(int64_t)head * a.f.q_rows + row] : -__builtin_inff();
        g[i] = o[i] = e[i] = zero;
        if (r < rows && in) {
          g[i] = *reinterpret_cast<const u32x4 *>(a.dout + row * a.do_row + head * a.do_head + l16 * 16);
          o[i] = *reinterpret_cast<const u32x4 *>(a.f.o + row * a.f.o_row + head * a.f.o_head + l16 * 16);
          e[i] = *reinterpret_cast<const u32x4 *>(a.f.rest + row * a.f.rest_row +
                                                  head * a.f.rest_head + l16 * 16);
        }
      }
#pragma unroll
      for (int i = 0; i < kTurns; ++i) {
        const int r = 4 * i + (lane >> 4);
        const int64_t at = (int64_t)head * a.f.q_rows + first + r;
        const float d = row_sum(dot8<T>(g[i], o[i]) + dot8<T>(g[i], e[i]));
        if (l16 == 0 && r < rows) {
          // (a row that saw nothing: +inf, so that its P is 0)
          a.rows[2 * at] = lse[i] == -__builtin_inff() ? __builtin_inff() : lse[i] * kLog2e;
          a.rows[2 * at + 1] = d;
        }
        if (a.f.fp16 && lse[i] != -__builtin_inff()) top = fmaxf(top, row_sum(dot8<T>(g[i], g[i])));
      }
    }
    if (a.f.fp16) {
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      if (lane == 0)
        a.bound[keys ? (int64_t)a.f.heads * a.f.q_rows + (int64_t)head * a.f.k_rows + first
                     : (int64_t)head * a.f.q_rows + first] = top;
    }
  }
}

// Exponent e of the factor 2^e that dS is kept at, for a document's `heads` heads from `head` on
// of key head kvh: |dS| <= 2 max|dO_i| max|v_j| < 2^15 / 2^e over its rows q0.. (lq of them) and
// keys k0.. (lk).
__device__ inline int ds_exponent(const AttnGradArgs &a, int head, int heads, int kvh, int q0, int lq,
                                  int k0, int lk, float *red) {
  float x = 0.f, y = 0.f;
  const float *bq = a.bound + (int64_t)head * a.f.q_rows + q0;
  const float *bv = a.bound + (int64_t)a.f.heads * a.f.q_rows + (int64_t)kvh * a.f.k_rows + k0;
  for (int h = 0; h < heads; ++h)
#pragma unroll 4
    for (int i = threadIdx.x * kRowTile; i < lq; i += kThreads * kRowTile)
      x = fmaxf(x, bq[(int64_t)h * a.f.q_rows + i]);
#pragma unroll 4
  for (int i = threadIdx.x * kRowTile; i < lk; i += kThreads * kRowTile) y = fmaxf(y, bv[i]);
#pragma unroll
  for (int o = 32; o; o >>= 1) {
    x = fmaxf(x, __shfl_xor(x, o));
    y = fmaxf(y, __shfl_xor(y, o));
  }
  if ((threadIdx.x & 63) == 0) {
    red[threadIdx.x >> 6] = x;
    red[4 + (threadIdx.x >> 6)] = y;
  }
  __syncthreads();
  x = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  y = fmaxf(fmaxf(red[4], red[5]), fmaxf(red[6], red[7]));
  __syncthreads();
  const float b = 2.f * sqrtf(x) * sqrtf(y);
  if (!(b > 0.f) || !(b < __builtin_inff())) return 0;
  int e;
  frexpf(b, &e);            // b < 2^e
  return uniform(min(max(15 - e, -60), 60));
}

// dS's factor: a block's, the same for both kinds below.
template <class T>
struct GradScale {
  static constexpr bool kHalf = std::is_same<T, Fp16>::value;
  float ds_scale;
  int ds0;

  __device__ void init(const AttnGradArgs &g, int head, int heads, int kvh, int q0, int lq, int k0,
                       int lk, float *red) {
    ds0 = kHalf ? ds_exponent(g, head, heads, kvh, q0, lq, k0, lk, red) : 0;
    ds_scale = kHalf ? ldexpf(1.f, ds0) : 1.f;
  }
};

// dS is rounded to T as an operand. Over few rows those roundings do not average out, and with two
// keys, whose dS are each other's opposites, dQ and dK would be off by up to 2.3 times what rounding
// the results costs (1.4 to 1.5 times over many): in short documents a second term holds what the
// first one's rounding took. Without / with: 24 documents of 120 rows, 8 heads of 64, 36.2 / 37.0
// us; 200 of 100, 16 heads of 128 with 4 of keys, 385 / 391; one of 8192, which has one term but
// the instructions beside it, 1328 / 1342.
constexpr int kTwoTerms = 128;
__device__ inline bool short_document(int lq, int lk) { return max(lq, lk) <= kTwoTerms; }
template <class T>
__device__ inline u32x4 rest_of(const f32x16 &x, int k, u32x4 rounded) {
  u32x4 r;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const uint32_t s = as_stored(rounded[w]);
    r[w] = T::pack(x[8 * k + 2 * w] - T::lo(s), x[8 * k + 2 * w + 1] - T::hi(s));
  }
  return r;
}

// ------------------------------------------------------------------ dK, dV
// A lane's key is fixed, its elements are the queries 8 g + 4 h + r of 32: products are
// Q K^T (queries x keys), their results the operands of dV^T = dO^T P and dK^T = Q^T dZ.
// K stays in registers and V in LDS: with V in registers too the accumulators would spill.
//
// NARROW: a block has 32 keys, its wavefronts go over every fourth step of the queries with
// LDS buffers of their own, and their sums are added at the end.
//
// Where few key heads and documents make few blocks of many steps, `shares` blocks take a
// part of a tile's steps each and leave fp32 sums, which grad_shares adds in order.
template <class T, int DP, int CAP, int BIAS, bool NARROW>
__device__ __forceinline__ void grad_kv(const AttnGradArgs &ga, int id, char *lds,
                                        float *red) {
  constexpr int KS = DP / 16, DT = DP / 32;
  constexpr int kBQ = kv_step(DP, NARROW);     // queries of a step
  constexpr int kTile = kBQ * DP * 2;
  constexpr int kBK = NARROW ? 32 : 128;       // keys of a block
  constexpr int kParts = NARROW ? 4 : 1;       // wavefronts (or the block) with own steps
  const AttnArgs &a = ga.f;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), h = lane >> 5;
  const int part = NARROW ? wave : 0;
  // per part [2][Q, dO]; V; per part [2][rows of log-sum and D]; per part the table
  char *const tiles = lds + part * 4 * kTile;
  char *vt = lds + kParts * 4 * kTile;
  char *rows_lds = vt + kBK * DP * 2 + part * 2 * kBQ * 8;
  float *lut = reinterpret_cast<float *>(vt + kBK * DP * 2 + kParts * 2 * kBQ * 8);
  uint8_t *map = nullptr;
  if (BIAS == kBiasTable) {
    const int n = lut_size(a.buckets.start[a.buckets.per_side - 1]);
    map = reinterpret_cast<uint8_t *>(lut + kParts * n);
    lut += part * n;
  }

  const int share = id % ga.shares;
  id /= ga.shares;
  const int kvh = id % a.kv_heads;
  const DocTile t = find_tile<kBK>(a.kb, a.ke, a.docs, a.k_rows, id / a.kv_heads);
  if (t.doc < 0) return;
  const int lk = t.b1 - t.b0;
  const int q0 = max(a.qb[t.doc], 0);
  const int lq = max(min(a.qe[t.doc], a.q_rows) - q0, 0);
  const int prefix = (a.causal && a.prefix) ? a.prefix[t.doc] : 0;
  const int shift = lk - lq;
  const bool two_terms = short_document(lq, lk);
  const int j0 = t.tile * kBK;

  const int key_lo = NARROW ? j0 : j0 + 32 * wave, key = key_lo + (lane & 31);
  // queries that see key j: those from first(j) on
  auto first = [&](int j) { return (a.causal && j >= prefix) ? max(j - shift, 0) : 0; };
  auto limit = [&](int i) { return a.causal ? min(lk, max(i + shift + 1, prefix)) : lk; };
  const int i_start = first(j0) / kBQ * kBQ;
  const int i_wave = key_lo < lk ? first(key_lo) : lq;                 // any key of the wavefront
  const int i_whole = key_lo + 31 < lk ? first(key_lo + 31) : lq;      // all of its keys
  const int mine = key < lk ? first(key) : lq;
  const int steps = max((lq - i_start + kBQ - 1) / kBQ, 0);
  // this block's part of the group's heads' steps
  const int from = (int)((int64_t)steps * a.group * share / ga.shares);
  const int total = (int)((int64_t)steps * a.group * (share + 1) / ga.shares);

  TileReader<DP> rd;
  rd.init(lane);
  TileCopy<DP, kBQ, NARROW ? 1 : 4> qc, dc;
  qc.init(NARROW ? 0 : wave, lane, (int)a.q_row, a.bytes);
  dc.init(NARROW ? 0 : wave, lane, (int)ga.do_row, a.bytes);
  auto start = [&](int n, int buf) {
    const int head = kvh * a.group + n / steps, i = i_start + n % steps * kBQ;
    const int rows = min(lq - i, kBQ);
    qc.start(row_buffer(a.q + (int64_t)q0 * a.q_row + head * a.q_head, i, rows, a.q_row, a.bytes),
             lds_address(tiles) + buf * 2 * kTile);
    dc.start(row_buffer(ga.dout + (int64_t)q0 * ga.do_row + head * ga.do_head, i, rows, ga.do_row,
                        a.bytes),
             lds_address(tiles) + (buf * 2 + 1) * kTile);
    const int sixty4 = NARROW ? 0 : wave;
    if (sixty4 < kBQ / 32)
      copy_words(row_buffer(reinterpret_cast<const char *>(ga.rows) +
                                ((int64_t)head * a.q_rows + q0) * 8, i, rows, 8, 8),
                 // (32 log-sums, then their 32 D)
                 (sixty4 * 64 + 2 * (lane & 31) + h) * 4,
                 lds_address(rows_lds) + buf * kBQ * 8 + sixty4 * 256);
  };
  {
    TileCopy<DP, kBK, 4> vc;
    vc.init(wave, lane, (int)a.v_row, a.bytes);
    vc.start(row_buffer(a.v + (int64_t)t.b0 * a.v_row + kvh * a.v_head, j0, min(lk - j0, kBK),
                        a.v_row, a.bytes),
             lds_address(vt));
  }
  if (from + part < total) start(from + part, 0);

  u32x4 kf[KS];
  load_operand<DP>(a.k + (int64_t)t.b0 * a.k_row + kvh * a.k_head, a.k_row, key, lk, a.bytes, lane, kf);
  GradScale<T> ps;
  ps.init(ga, kvh * a.group, a.group, kvh, q0, lq, t.b0, lk, red);
  const ScoreScale sc = score_scale<CAP>(a.scale, a.cap);
  const float p0 = ps.kHalf ? kP16 : 0.f, ds_scale = ps.ds_scale * exp2f(-p0);
  const int reach = BIAS == kBiasTable ? a.buckets.start[a.buckets.per_side - 1] : 0;

  if (BIAS == kBiasTable) fill_map(map, a.buckets, threadIdx.x, kThreads);

  f32x16 dk[DT], dv[DT];
#pragma unroll
  for (int c = 0; c < DT; ++c) dk[c] = dv[c] = f32x16{};
  float slope2 = 0.f;

  copies_barrier();
  int head_now = -1;
  for (int n = from + part, buf = 0; n < total; n += kParts, buf ^= 1) {
    if (BIAS != kBiasNone && n / steps != head_now) {   // the next head
      head_now = n / steps;
      const int head = kvh * a.group + head_now;
      if (BIAS == kBiasSlope) slope2 = a.slopes[head] * kLog2e;
      if (BIAS == kBiasTable) {
        fill_lut<T>(lut, map, a.buckets, a.table, head, NARROW ? lane : threadIdx.x,
                    NARROW ? 64 : kThreads);
        if (!NARROW) __syncthreads();
      }
    }
    if (NARROW) {   // (the buffer that is filled next was read in the step before)
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (n + kParts < total) {
        start(n + kParts, buf ^ 1);
        wait_copies<2 * (kTile / 1024) + 1>();
      } else {
        wait_copies<0>();
      }
    } else if (n + 1 < total) {
      start(n + 1, buf ^ 1);
    }
#pragma unroll 1
    for (int sub = 0; sub < kBQ; sub += 32) {
      const int i0 = i_start + n % steps * kBQ + sub;
      if (i0 + 32 <= i_wave || i0 >= lq) continue;
      const uint32_t tile = lds_address(tiles) + buf * 2 * kTile;
      const uint32_t qr = rd.at(tile, rd.row), qc0 = rd.at(tile, rd.col);
      const uint32_t vr = rd.at(lds_address(vt), rd.row);
      const char *rows = rows_lds + (buf * kBQ + sub) * 8 + 16 * h;
      f32x16 s = {}, dp = {};
#pragma unroll
      for (int k = 0; k < KS; ++k) s = T::mfma(row_operand<DP>(qr, sub, k), kf[k], s);
#pragma unroll
      for (int k = 0; k < KS; ++k)
        dp = T::mfma(row_operand<DP>(qr + kTile, sub, k), row_operand<DP>(vr + (NARROW ? 0 : 32 * wave * DP * 2), 0, k), dp);
      const bool masked = i0 < i_whole || i0 + 32 > lq;
#pragma unroll
      for (int g = 0; g < 4; ++g) {   // (dP - D) dZ/dS first: the capped products then are done
        const f32x4 delta = *reinterpret_cast<const f32x4 *>(rows + 128 + 32 * g);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int e = 4 * g + r;
          s[e] = score_x<CAP>(s[e], sc);
          dp[e] -= delta[r];
          if (CAP) dp[e] *= cap_slope<CAP>(s[e], sc);
        }
      }
      // the distance falls with the query: add_bias's elements in the other direction
      Affine f = {sc.a, sc.b};
      if (BIAS == kBiasSlope) {
        const float d0 = (float)(key - shift - i0 - 4 * h);
#pragma unroll
        for (int e = 0; e < 16; ++e)
          s[e] = __builtin_fmaf(s[e], sc.a, -slope2 * __builtin_fabsf(d0 - (float)row_of(e)));
        f.a = 1.f;
      }
      if (BIAS == kBiasTable) {
        const int far_hi = key_lo + 31 - (i0 + shift), far_lo = key_lo - (i0 + 31 + shift);
        if (far_hi <= -reach || far_lo >= ahead_reach(reach)) {
          f.b += far_hi <= -reach ? lut[0] : lut[lut_size(reach) - 1];
        } else {
          const float *p = lut + (key - shift - i0 - 4 * h + reach + kLutPad);
#pragma unroll
          for (int e = 0; e < 16; ++e) s[e] = __builtin_fmaf(s[e], sc.a, p[-row_of(e)]);
          f.a = 1.f;
        }
      }
      const float off = f.b + p0;
      if (masked) {   // exp2(-inf) below
        const int lo = mine - i0 - 4 * h, hi = lq - i0 - 4 * h;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          if (row_of(e) < lo || row_of(e) >= hi) s[e] = -__builtin_inff();
          // a query that sees one key: dP - D is 0 but for the order of the sums
          if (limit(i0 + 4 * h + row_of(e)) == 1) dp[e] = 0.f;
        }
      }
      asm volatile("" ::: "memory");
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 lse = *reinterpret_cast<const f32x4 *>(rows + 32 * g);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int e = 4 * g + r;
          s[e] = fast_exp2(__builtin_fmaf(s[e], f.a, off - lse[r]));
          dp[e] *= ps.kHalf ? s[e] * ds_scale : s[e];
        }
      }
      u32x4 pr[2], dr[2];
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          pr[k][w] = T::pack(s[8 * k + 2 * w], s[8 * k + 2 * w + 1]);
          dr[k][w] = T::pack(dp[8 * k + 2 * w], dp[8 * k + 2 * w + 1]);
        }
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int c = 0; c < DT; ++c) {
          dv[c] = T::mfma(col_operand<DP>(qc0 + kTile, sub + 16 * k, c), pr[k], dv[c]);
          dk[c] = T::mfma(col_operand<DP>(qc0, sub + 16 * k, c), dr[k], dk[c]);
        }
      if (__builtin_expect(two_terms, 0)) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const u32x4 rest = rest_of<T>(dp, k, dr[k]);
#pragma unroll
          for (int c = 0; c < DT; ++c)
            dk[c] = T::mfma(col_operand<DP>(qc0, sub + 16 * k, c), rest, dk[c]);
        }
      }
    }
    if (!NARROW) copies_barrier();
  }
  if (NARROW) {
    copies_barrier();
    add_waves<DT>(dv, lds);
    if (!add_waves<DT>(dk, lds)) return;
  }
  const bool ok = key < lk;
  const float fv = exp2f(-p0), fk = a.scale * cap_factor<CAP>() * ldexpf(1.f, -ps.ds0);
  if (ga.shares > 1) {
    float *x = ga.kv_part + (((int64_t)share * a.k_rows + t.b0 + key) * a.kv_heads + kvh) * 2 * DP;
    if (ok) {
#pragma unroll
      for (int c = 0; c < DT; ++c)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          f32x4 k4, v4;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            k4[r] = dk[c][4 * g + r] * fk;
            v4[r] = dv[c][4 * g + r] * fv;
          }
          *reinterpret_cast<f32x4 *>(x + 32 * c + 8 * g + 4 * h) = k4;
          *reinterpret_cast<f32x4 *>(x + DP + 32 * c + 8 * g + 4 * h) = v4;
        }
    }
    return;
  }
  store_row<T, DT>(ga.dv + (int64_t)(t.b0 + key) * ga.dv_row + kvh * ga.dv_head, ok, a.bytes, dv,
                   fv, lane);
  store_row<T, DT>(ga.dk + (int64_t)(t.b0 + key) * ga.dk_row + kvh * ga.dk_head, ok, a.bytes, dk,
                   fk, lane);
}

// dK and dV from the shares' sums, in their order: a block per 32 keys and key head, all shares'
// loads under way at once. 2 shares of 8862 rows of 4 heads of 64, 36 MB, 8.6 us.
constexpr int kShareRows = 32;
template <class T, int DP>
__global__ __launch_bounds__(kThreads) void grad_shares(const AttnGradArgs ga) {
  const AttnArgs &a = ga.f;
  constexpr int kPieces = DP / 8;
  const int kvh = blockIdx.x % a.kv_heads;
  const DocTile t = find_tile<kShareRows>(a.kb, a.ke, a.docs, a.k_rows, blockIdx.x / a.kv_heads);
  if (t.doc < 0) return;
  for (int i = threadIdx.x; i < kShareRows * 2 * kPieces; i += kThreads) {
    const int row = t.tile * kShareRows + i / (2 * kPieces), piece = i % kPieces;
    const bool v = i / kPieces % 2;
    if (row >= t.b1 - t.b0 || piece * 16 >= a.bytes) continue;
    f32x4 lo = {}, hi = {};
#pragma unroll 4
    for (int s = 0; s < ga.shares; ++s) {
      const float *x = ga.kv_part + (((int64_t)s * a.k_rows + t.b0 + row) * a.kv_heads + kvh) * 2 * DP +
                       (v ? DP : 0) + piece * 8;
      lo += *reinterpret_cast<const f32x4 *>(x);
      hi += *reinterpret_cast<const f32x4 *>(x + 4);
    }
    char *to = v ? ga.dv + (int64_t)(t.b0 + row) * ga.dv_row + kvh * ga.dv_head
                 : ga.dk + (int64_t)(t.b0 + row) * ga.dk_row + kvh * ga.dk_head;
    *reinterpret_cast<u32x4 *>(to + piece * 16) =
        u32x4{T::pack(lo[0], lo[1]), T::pack(lo[2], lo[3]), T::pack(hi[0], hi[1]), T::pack(hi[2], hi[3])};
  }
}

// ------------------------------------------------------------------ dQ, table
// A lane's query is fixed, its elements are the keys, as in the forward kernel.
//
// Table gradient: the sums of dS by distance. Beyond the table's reach that is one sum per
// lane; within, a wavefront writes its values of dS into LDS skewed, so that a distance is a
// column, adds up the columns and adds those to its sums by distance (LDS atomics on those
// took 3.5 times as long).
//
// NARROW: a block has 32 queries, its wavefronts go over every fourth step of the keys.
template <class T, int DP, int CAP, int BIAS, bool NARROW>
__device__ __forceinline__ void grad_q(const AttnGradArgs &ga, int id, char *lds,
                                       float *red) {
  constexpr int KS = DP / 16, DT = DP / 32;
  constexpr int kBN = 32;                      // keys of a step
  constexpr int kTile = kBN * DP * 2;
  constexpr int kBM = NARROW ? 32 : 128;
  constexpr int kParts = NARROW ? 4 : 1;
  const AttnArgs &a = ga.f;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), h = lane >> 5;
  const int part = NARROW ? wave : 0;
  // per part [2][K, V]; [4] skewed values, biases, [4] sums by distance
  char *const kv_tiles = lds + part * 4 * kTile;
  float *skewed = reinterpret_cast<float *>(lds + kParts * 4 * kTile);
  float *lut = skewed + 4 * kSkew;

  const int kvh = id % a.kv_heads;
  id /= a.kv_heads;
  const int head = kvh * a.group + id % a.group, unit = id / a.group;
  const int nb = bucket_count(a.buckets);
  const DocTile t = find_tile<kBM>(a.qb, a.qe, a.docs, a.q_rows, unit);
  float *tout = nullptr;
  if (BIAS == kBiasTable) tout = ga.tpart + ((int64_t)unit * a.heads + head) * nb;
  if (t.doc < 0) {
    if (BIAS == kBiasTable)
      for (int b = threadIdx.x; b < nb; b += kThreads) tout[b] = 0.f;
    return;
  }
  const int lq = t.b1 - t.b0;
  const int k0 = max(a.kb[t.doc], 0);
  const int lk = max(min(a.ke[t.doc], a.k_rows) - k0, 0);
  const int prefix = (a.causal && a.prefix) ? a.prefix[t.doc] : 0;
  const int tiles = (lq + kBM - 1) / kBM;
  const int i0 = (tiles - 1 - t.tile) * kBM;

  const int row_lo = NARROW ? i0 : i0 + 32 * wave, row = row_lo + (lane & 31);
  const int shift = lk - lq;
  const bool two_terms = short_document(lq, lk);
  auto limit = [&](int i) { return a.causal ? min(lk, max(i + shift + 1, prefix)) : lk; };
  const bool ok = row < lq;
  const int lim = ok ? limit(row) : 0;
  const int lim_lo = row_lo + 31 < lq ? limit(row_lo) : 0;
  const int lim_hi = row_lo < lq ? limit(min(row_lo + 31, lq - 1)) : 0;
  const int n_tiles = (max(limit(min(i0 + kBM, lq) - 1), 0) + kBN - 1) / kBN;

  const char *kbase = a.k + (int64_t)k0 * a.k_row + kvh * a.k_head;
  const char *vbase = a.v + (int64_t)k0 * a.v_row + kvh * a.v_head;
  TileReader<DP> rd;
  rd.init(lane);
  TileCopy<DP, kBN, NARROW ? 1 : 4> kc, vc;
  kc.init(NARROW ? 0 : wave, lane, (int)a.k_row, a.bytes);
  vc.init(NARROW ? 0 : wave, lane, (int)a.v_row, a.bytes);
  auto start = [&](int tile, int buf) {
    const int n = min(lk - tile * kBN, kBN);
    kc.start(row_buffer(kbase, (int64_t)tile * kBN, n, a.k_row, a.bytes),
             lds_address(kv_tiles) + buf * 2 * kTile);
    vc.start(row_buffer(vbase, (int64_t)tile * kBN, n, a.v_row, a.bytes),
             lds_address(kv_tiles) + (buf * 2 + 1) * kTile);
  };
  if (part < n_tiles) start(part, 0);

  u32x4 qf[KS], df[KS];
  load_operand<DP>(a.q + (int64_t)t.b0 * a.q_row + head * a.q_head, a.q_row, row, lq, a.bytes, lane, qf);
  load_operand<DP>(ga.dout + (int64_t)t.b0 * ga.do_row + head * ga.do_head, ga.do_row, row, lq,
                   a.bytes, lane, df);
  const int64_t at = (int64_t)head * a.q_rows + t.b0 + row;
  // (a query that sees one key: dP - D is 0 but for the order of the sums)
  const float lse = ok && lim > 1 ? ga.rows[2 * at] : __builtin_inff();
  const float delta = ok ? ga.rows[2 * at + 1] : 0.f;
  GradScale<T> ps;
  ps.init(ga, head, 1, kvh, t.b0, lq, k0, lk, red);
  const ScoreScale sc = score_scale<CAP>(a.scale, a.cap);
  int reach = 0;
  float slope2 = 0.f;
  float *hist = nullptr, *skew = skewed + wave * kSkew;
  float far_l = 0.f, far_r = 0.f;              // behind and ahead of the table's reach
  if (BIAS == kBiasTable) {
    reach = a.buckets.start[a.buckets.per_side - 1];
    const int n = lut_size(reach);
    uint8_t *map = reinterpret_cast<uint8_t *>(lut + 5 * n);
    fill_map(map, a.buckets, threadIdx.x, kThreads);   // (each thread reads what it wrote)
    fill_lut<T>(lut, map, a.buckets, a.table, head, threadIdx.x, kThreads);
    hist = lut + n * (1 + wave);
    for (int i = lane; i < n; i += 64) hist[i] = 0.f;
    for (int i = lane; i < kSkew; i += 64) skew[i] = 0.f;
  }
  if (BIAS == kBiasSlope) slope2 = a.slopes[head] * kLog2e;
  float steps[16];
  slope_steps<BIAS>(steps, slope2);

  f32x16 acc[DT];
#pragma unroll
  for (int c = 0; c < DT; ++c) acc[c] = f32x16{};

  copies_barrier();
  for (int tile = part, buf = 0; tile < n_tiles; tile += kParts, buf ^= 1) {
    if (NARROW) {   // (as above)
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (tile + kParts < n_tiles) {
        start(tile + kParts, buf ^ 1);
        wait_copies<2 * (kTile / 1024)>();
      } else {
        wait_copies<0>();
      }
    } else if (tile + 1 < n_tiles) {
      start(tile + 1, buf ^ 1);
    }
    const int key0 = tile * kBN;
    if (key0 < lim_hi) {
      const uint32_t tile_at = lds_address(kv_tiles) + buf * 2 * kTile;
      const uint32_t kr = rd.at(tile_at, rd.row), kcol = rd.at(tile_at, rd.col);
      f32x16 s = {}, dp = {};
#pragma unroll
      for (int k = 0; k < KS; ++k) s = T::mfma(row_operand<DP>(kr, 0, k), qf[k], s);
#pragma unroll
      for (int k = 0; k < KS; ++k) dp = T::mfma(row_operand<DP>(kr + kTile, 0, k), df[k], dp);
      f32x16 z;   // x of the capped products
      if (CAP) {
#pragma unroll
        for (int e = 0; e < 16; ++e) z[e] = s[e] = score_x<CAP>(s[e], sc);
      }
      const Affine f = add_bias<BIAS>(s, sc, key0, row + shift, row_lo + shift, h, slope2, steps, lut, reach);
      if (key0 + 32 > lim_lo) {
        const int mine = lim - key0 - 4 * h;
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (row_of(e) >= mine) s[e] = -__builtin_inff();
      }
      const float off = f.b - lse;
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        dp[e] = fast_exp2(__builtin_fmaf(s[e], f.a, off)) * (dp[e] - delta);
        if (BIAS == kBiasTable) sum += dp[e];
      }
      if (BIAS == kBiasTable) {
        const int d_hi = key0 + 31 - (row_lo + shift), d_lo = key0 - (row_lo + 31 + shift);
        if (d_hi <= -reach) {
          far_l += sum;
        } else if (d_lo >= ahead_reach(reach)) {
          far_r += sum;
        } else {
          // 16 keys at a time: value (key k, query q) at [k][k - q + 31]; what lies outside
          // stays 0
          float *w = skew + 4 * h * 65 + 31 - (lane & 31);
          const float *r = skew + (lane >> 4) * 4 * 64 + (lane & 15) * 4;
          const int g = lane >> 4, d = (lane & 15) * 4 + g;   // this lane's column
          float *to = hist + d_lo + d + reach + kLutPad;
#pragma unroll
          for (int k16 = 0; k16 < 2; ++k16) {
#pragma unroll
            for (int e = 0; e < 8; ++e) w[(8 * (e >> 2) + (e & 3)) * 65] = dp[8 * k16 + e];
            f32x4 v = {};
#pragma unroll
            for (int k = 0; k < 4; ++k) v += *reinterpret_cast<const f32x4 *>(r + k * 64);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = sum_rows(v[k]);
            const float x = g == 0 ? v[0] : (g == 1 ? v[1] : (g == 2 ? v[2] : v[3]));
            if (d < 47) to[16 * k16] += x;
          }
        }
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        if (CAP) dp[e] *= cap_slope<CAP>(z[e], sc);
        if (ps.kHalf) dp[e] *= ps.ds_scale;
      }
      u32x4 dr[2];
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int w = 0; w < 4; ++w)
          dr[k][w] = T::pack(dp[8 * k + 2 * w], dp[8 * k + 2 * w + 1]);
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int c = 0; c < DT; ++c)
          acc[c] = T::mfma(col_operand<DP>(kcol, 16 * k, c), dr[k], acc[c]);
      if (__builtin_expect(two_terms, 0)) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const u32x4 rest = rest_of<T>(dp, k, dr[k]);
#pragma unroll
          for (int c = 0; c < DT; ++c) acc[c] = T::mfma(col_operand<DP>(kcol, 16 * k, c), rest, acc[c]);
        }
      }
    }
    if (!NARROW) copies_barrier();
  }
  bool writes = true;
  if (NARROW) {
    copies_barrier();
    writes = add_waves<DT>(acc, lds);
  }
  if (writes)
    store_row<T, DT>(ga.dq + (int64_t)(t.b0 + row) * ga.dq_row + head * ga.dq_head, ok, a.bytes,
                     acc, a.scale * cap_factor<CAP>() * ldexpf(1.f, -ps.ds0), lane);

  if (BIAS == kBiasTable) {
#pragma unroll
    for (int o = 32; o; o >>= 1) {
      far_l += __shfl_xor(far_l, o);
      far_r += __shfl_xor(far_r, o);
    }
    if (lane == 0) {
      red[2 * wave] = far_l;
      red[2 * wave + 1] = far_r;
    }
    __syncthreads();
    // the four wavefronts' sums by distance in the place of the first's
    const int n = lut_size(reach), mid = reach + kLutPad, per = a.buckets.per_side;
    float *all = lut + n;
    for (int i = threadIdx.x; i < n; i += kThreads)
      all[i] = (all[i] + all[n + i]) + (all[2 * n + i] + all[3 * n + i]);
    __syncthreads();
    // a wavefront per bucket in turn
    const float fl = (red[0] + red[2]) + (red[4] + red[6]), fr = (red[1] + red[3]) + (red[5] + red[7]);
    for (int b = wave; b < nb; b += 4) {
      const int k = b % per;
      const bool ahead = b >= per;             // the second half of a two-sided table
      const int to = k + 1 < per ? a.buckets.start[k + 1] : mid + 1;   // distances [from, to)
      float x = 0.f;
      for (int d = max(a.buckets.start[k], ahead ? 1 : 0) + lane; d < to; d += 64)
        x += all[mid + (ahead ? d : -d)];
      if (!a.buckets.two_sided && k == 0)      // keys ahead count as distance 0
        for (int d = 1 + lane; d <= mid; d += 64) x += all[mid + d];
#pragma unroll
      for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
      if (k + 1 == per) x += ahead ? fr : fl;
      if (!a.buckets.two_sided && k == 0) x += fr;
      if (lane == 0) tout[b] = x;
    }
  }
}

// Both in one launch, the longer-running blocks of dK and dV first. (In two
// launches each kind's last blocks would leave the device idle.)
template <class T, int DP, int CAP, int BIAS, bool NARROW>
__global__ __launch_bounds__(kThreads, NARROW && DP == 128 ? 1 : 2) void grad_pairs(const AttnGradArgs ga,
                                                          int kv_blocks) {
  extern __shared__ __align__(1024) char lds[];
  __shared__ float red[8];
  if ((int)blockIdx.x < kv_blocks)
    grad_kv<T, DP, CAP, BIAS, NARROW>(ga, blockIdx.x, lds, red);
  else
    grad_q<T, DP, CAP, BIAS, NARROW>(ga, blockIdx.x - kv_blocks, lds, red);
}

// dtable[head][b]: the tiles' partial sums, strided over the threads, then joined in a tree. 4 us,
// a launch's latency.
template <class T>
__global__ __launch_bounds__(256) void grad_table(const AttnGradArgs a, int units, int nb) {
  __shared__ float red[256];
  const int head = blockIdx.x / nb, b = blockIdx.x % nb;
  float x = 0.f;
  for (int u = threadIdx.x; u < units; u += 256)
    x += a.tpart[((int64_t)u * a.f.heads + head) * nb + b];
  red[threadIdx.x] = x;
  __syncthreads();
  for (int o = 128; o; o >>= 1) {
    if ((int)threadIdx.x < o) red[threadIdx.x] += red[threadIdx.x + o];
    __syncthreads();
  }
  if (threadIdx.x == 0) T::store(a.dtable, (int64_t)head * nb + b, red[0]);
}

int64_t bound_floats(const AttnArgs &f) {
  return f.fp16 ? (int64_t)f.q_rows * f.heads + (int64_t)f.k_rows * f.kv_heads : 0;
}

int64_t tile_bound(int64_t rows, int64_t docs, int64_t longest, int tile) {
  const int64_t x = rows / tile + docs, y = docs * ((longest + tile - 1) / tile);
  return x < y ? x : y;
}

// LDS of a block; lut: bytes of a head's table of biases, 0 without, and of the map to it.
constexpr int pair_bytes(int dp, bool narrow, int lut, int map) {
  const int step = kv_step(dp, narrow), parts = narrow ? 4 : 1;
  const int kv = parts * 4 * step * dp * 2 + (narrow ? 32 : 128) * dp * 2 +
                 parts * (2 * step * 8 + lut) + map;
  const int q = parts * 4 * 32 * dp * 2 + (lut ? 4 * kSkew * 4 + 5 * lut + map : 0);
  return kv > q ? kv : q;
}

// The narrow form's tiles where the wide one's blocks would leave compute units idle, if
// the table leaves room in LDS. Narrow / wide at n wide blocks, with a table: documents of 120
// rows, 8 heads of 64, n = 32 21.9 / 25.2 us, 128 30.4 / 26.8; 250 rows, 16 heads of 64 with 4 of
// keys, n = 160 45 / 60, 320 77 / 68; 500 rows, 8 heads of 128 with 2 of keys, n = 160 84 / 85,
// 320 137 / 96; 3 of 333, 6 heads of 80, n = 24 50 / 93.
constexpr int kNarrowBlocks = 160;
int pair_bytes(const AttnArgs &f, bool narrow) {
  const int dp = f.bytes <= 128 ? 64 : 128;
  if (f.buckets.per_side == 0) return pair_bytes(dp, narrow, 0, 0);
  const int reach = f.buckets.start[f.buckets.per_side - 1];
  return pair_bytes(dp, narrow, lut_size(reach) * 4, map_bytes(reach));
}
int tile_rows(const AttnArgs &f) {
  const int64_t wide = tile_bound(f.k_rows, f.docs, f.max_k, 128) * f.kv_heads +
                       tile_bound(f.q_rows, f.docs, f.max_q, 128) * f.heads;
  return wide <= kNarrowBlocks && pair_bytes(f, true) <= kLdsBytes - 1024 ? 32 : 128;
}

// Blocks that share a key tile's steps, so that the longest of them does not outlast the rest:
// about 384 blocks of keys in all (more with several query heads per key head, whose blocks are
// that much longer), none with less than 512 queries. Steps with 1 / 2 / 3 / 4 / 8 shares, D = 64,
// 4 heads per key head: 16 documents of 1024 at most (277 tiles) 258 / 230 / 231 / - / - us; 3 of
// 2000, 12 heads (141 tiles) - / 219 / 192 / 203 / 208; one of 4096, 12 heads (96 tiles) - / - / - /
// 234 / 259; D = 128, 2 key heads, 2 documents of 2500 (80 tiles) - / - / - / 244 / 290; one head
// per key head, one of 4096, 8 heads (256 tiles) 210 / 235 / 249 / - / -; 24 documents of 120 rows,
// 8 heads (184 tiles) 35 / - / 54 / - / -. Narrow blocks: about 192, with the more queries each the
// more there are. None / n shares: one of 1500 rows, 8 heads of 64 with 1 of keys (47 tiles) 144 /
// 74 (n = 4); of 120 (4 tiles) 34.5 / 28.4 (3); 1000 rows, 8 heads of 128 with 2 of keys (64 tiles)
// 97 / 75 (3); 4 documents of 250 (64 tiles), which this leaves whole, 47 / 53 (2).
constexpr int kShareQueries = 512, kShareBlocks = 384, kNarrowShares = 192;
int share_count(const AttnArgs &f) {
  const int tile = tile_rows(f);
  const int64_t blocks = ((int64_t)f.k_rows + tile - 1) / tile * f.kv_heads;
  if (blocks == 0 || f.q_rows == 0) return 1;
  const int64_t queries = (int64_t)f.group * f.max_q;
  int64_t s, most;
  if (tile == 32) {
    s = kNarrowShares / blocks;
    most = queries / (256 + 6 * blocks);
  } else {
    s = (kShareBlocks + (f.group > 1 ? blocks - 1 : 0)) / blocks;
    most = queries / kShareQueries;
  }
  if (s > most) s = most;
  if (s < 1) s = 1;
  return (int)(s < 8 ? s : 8);
}

// Blocks of the passes over the keys and over the queries.
struct PairGrid {
  int64_t kv, units, all;
};
PairGrid pair_grid(const AttnArgs &f, int tile, int shares) {
  PairGrid g;
  g.kv = tile_bound(f.k_rows, f.docs, f.max_k, tile) * f.kv_heads * shares;
  g.units = tile_bound(f.q_rows, f.docs, f.max_q, tile);
  g.all = g.kv + g.units * f.heads;
  return g;
}

template <class T, int DP, int CAP, int BIAS, bool NARROW>
hipError_t launch_form(const AttnGradArgs &a, hipStream_t s) {
  static LdsLimit limit;
  constexpr int kTile = NARROW ? 32 : 128;
  const int lds = pair_bytes(a.f, NARROW);
  hipError_t e = limit.set(reinterpret_cast<const void *>(&grad_pairs<T, DP, CAP, BIAS, NARROW>),
                           kLdsBytes - 1024);   // (the rest for what is static)
  if (e != hipSuccess) return e;
  const PairGrid g = pair_grid(a.f, kTile, a.shares);
  if (g.all > 0)
    grad_pairs<T, DP, CAP, BIAS, NARROW>
        <<<dim3((uint32_t)g.all), kThreads, lds, s>>>(a, (int)g.kv);
  if (a.shares > 1) {
    const int64_t n = tile_bound(a.f.k_rows, a.f.docs, a.f.max_k, kShareRows) * a.f.kv_heads;
    if (n > 0)   // (a cache of which no document has a row yet)
      grad_shares<T, DP><<<dim3((uint32_t)n), kThreads, 0, s>>>(a);
  }
  if (BIAS == kBiasTable) {
    const int nb = bucket_count(a.f.buckets);
    grad_table<T><<<dim3((uint32_t)(a.f.heads * nb)), 256, 0, s>>>(a, (int)g.units, nb);
  }
  return hipGetLastError();
}

template <class T, int DP, int CAP, int BIAS>
hipError_t launch(const AttnGradArgs &a, hipStream_t s) {
  if (tile_rows(a.f) == 32) return launch_form<T, DP, CAP, BIAS, true>(a, s);
  return launch_form<T, DP, CAP, BIAS, false>(a, s);
}

template <class T, int DP, int CAP>
hipError_t by_bias(const AttnGradArgs &a, hipStream_t s) {
  if (a.f.table) return launch<T, DP, CAP, kBiasTable>(a, s);
  if (a.f.slopes) return launch<T, DP, CAP, kBiasSlope>(a, s);
  return launch<T, DP, CAP, kBiasNone>(a, s);
}

template <class T, int DP>
hipError_t by_cap(const AttnGradArgs &a, hipStream_t s) {
  switch (cap_kind(a.f)) {
    case kCapNone: return by_bias<T, DP, kCapNone>(a, s);
    case kCapNear: return by_bias<T, DP, kCapNear>(a, s);
    default: return by_bias<T, DP, kCapFar>(a, s);
  }
}

}  // namespace

size_t attend_grad_bytes(const AttnArgs &f) {
  auto up = [](int64_t n) { return (n + 63) / 64 * 64; };
  int64_t n = up(2 * (int64_t)f.q_rows * f.heads);
  n += up(bound_floats(f));
  const int nb = bucket_count(f.buckets);
  n += up(tile_bound(f.q_rows, f.docs, f.max_q, tile_rows(f)) * f.heads * nb);
  const int shares = share_count(f);
  if (shares > 1) n += shares * (int64_t)f.k_rows * f.kv_heads * 2 * (f.bytes <= 128 ? 64 : 128);
  return (size_t)n * 4;
}

bool attend_grad_fits(const AttnArgs &f) {
  const int shares = share_count(f);
  const int64_t sums = shares > 1 ? tile_bound(f.k_rows, f.docs, f.max_k, kShareRows) * f.kv_heads : 0;
  return pair_grid(f, tile_rows(f), shares).all <= kMaxBlocks && sums <= kMaxBlocks;
}

hipError_t launch_attend_grad(const AttnGradArgs &args, void *ws, hipStream_t s) {
  AttnGradArgs a = args;
  auto up = [](int64_t n) { return (n + 63) / 64 * 64; };
  a.rows = static_cast<float *>(ws);
  a.bound = a.rows + up(2 * (int64_t)a.f.q_rows * a.f.heads);
  a.tpart = a.bound + up(bound_floats(a.f));
  a.kv_part = a.tpart + up(tile_bound(a.f.q_rows, a.f.docs, a.f.max_q, tile_rows(a.f)) * a.f.heads *
                           bucket_count(a.f.buckets));
  a.shares = share_count(a.f);
  const int64_t q_units = tile_bound(a.f.q_rows, a.f.docs, a.f.max_q, kRowTile) * a.f.heads;
  int64_t units = q_units;
  if (a.f.fp16) units += tile_bound(a.f.k_rows, a.f.docs, a.f.max_k, kRowTile) * a.f.kv_heads;
  int64_t blocks = (units + 3) / 4;
  if (blocks > kRowBlocks) blocks = kRowBlocks;
  if (blocks > 0) {
    if (a.f.fp16) grad_rows<Fp16><<<dim3((uint32_t)blocks), kThreads, 0, s>>>(a, q_units, units);
    else grad_rows<Bf16><<<dim3((uint32_t)blocks), kThreads, 0, s>>>(a, q_units, units);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (a.f.bytes <= 128) return a.f.fp16 ? by_cap<Fp16, 64>(a, s) : by_cap<Bf16, 64>(a, s);
  return a.f.fp16 ? by_cap<Fp16, 128>(a, s) : by_cap<Bf16, 128>(a, s);
}

}  // namespace bgp
