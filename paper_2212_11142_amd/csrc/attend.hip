// Attention over packed histories, general form: out_i = sum_j softmax_j(s_ij) v_j over the
// keys j < lim(i) of query i's document, s_ij = cap tanh(scale q_i.k_j / cap) + bias.
//
// One pass over the keys with a running maximum and sum. A block of 4 wavefronts takes 128
// queries of one head, a wavefront 32 of them; a wavefront's scores are the transposed
// product K Q^T (32 keys x 32 queries at a time), whose registers are the operand of the
// second product V^T P^T, so that only K and V go through LDS, and each once per block.
// lim(i) = min(Lk, max(position + 1, prefix)) covers the causal, prefix and document masks
// with one comparison per score, made only in tiles where some row's limit falls.
//
// Bound by the matrix units and by the scores' own instructions (an exponential, two fused
// multiply-adds, the maximum, the sum and half a conversion each) in turn. Measured: 16,384 rows,
// causal, 16 heads of 128, fp16, 1201 us, 0.92 PFLOP/s (a library product of 8192^3 has 1.11; the
// matrix units are busy for half of the cycles, the vector units for 65%); 1,048,576 rows over
// 512 keys, 8 heads of 64, bf16, 1456 us, 0.76 PFLOP/s (vector units 79%: at this head size half
// the products per score); 13 documents of up to 1021 rows, 16 heads of 128, cap and table, 57 us,
// where two blocks per compute unit leave both idle (vector units 50%, matrix units 22%; wavefronts
// wait for 42% of their cycles). More queries per wavefront or keys per tile would not fit the
// registers.
#include <type_traits>

#include "seq_dev.h"

namespace bgp {
namespace {

constexpr int kBM = 128;   // queries of a block
constexpr int kBN = 64;    // keys of a tile
constexpr int kThreads = 256;
// PARTS = 2: two groups of 4 wavefronts take every second tile each, with LDS buffers of their
// own, and the first adds up their sums at the end.
template <class T, int DP, int CAP, int BIAS, bool REST, int PARTS>
__global__ __launch_bounds__(kThreads * PARTS, 2) void attend_kernel(const AttnArgs a) {
  constexpr int KS = DP / 16;   // k-steps of the score product
  constexpr int DT = DP / 32;   // column blocks of V
  constexpr int kTile = kBN * DP * 2;
  extern __shared__ __align__(1024) char lds[];
  const int lane = threadIdx.x & 63, h = lane >> 5;
  const int wave = uniform(threadIdx.x >> 6) % 4, part = uniform(threadIdx.x >> 8);
  char *kt = lds + part * 4 * kTile, *vt = kt + 2 * kTile;
  float *lut = reinterpret_cast<float *>(lds + PARTS * 4 * kTile);

  // kv heads fastest: the blocks of one XCD (every 8th) then share few heads' keys; the
  // last tiles of a document, which see the most keys under a causal mask, come first
  int id = blockIdx.x;
  const int kvh = id % a.kv_heads;
  id /= a.kv_heads;
  const int head = kvh * a.group + id % a.group;
  const DocTile t = find_tile<kBM>(a.qb, a.qe, a.docs, a.q_rows, id / a.group);
  if (t.doc < 0) return;
  const int lq = t.b1 - t.b0;
  const int k0 = max(a.kb[t.doc], 0);
  const int lk = max(min(a.ke[t.doc], a.k_rows) - k0, 0);
  const int prefix = (a.causal && a.prefix) ? a.prefix[t.doc] : 0;
  const int tiles = (lq + kBM - 1) / kBM;
  const int i0 = (tiles - 1 - t.tile) * kBM;

  const int row_lo = i0 + 32 * wave;             // first query of the wavefront
  const int row = row_lo + (lane & 31);
  const int shift = lk - lq;                     // position of query 0
  auto limit = [&](int i) { return a.causal ? min(lk, max(i + shift + 1, prefix)) : lk; };
  const float slack = Probs<T>::slack(lk), p_shift = Probs<T>::shift(lk);
  const int lim = limit(row);
  const int lim_lo = limit(row_lo);                             // keys all rows see
  const int lim_hi = row_lo < lq ? limit(min(row_lo + 31, lq - 1)) : 0;  // keys any row sees
  const int lim_block = max(limit(min(i0 + kBM, lq) - 1), 0);
  const int n_tiles = (lim_block + kBN - 1) / kBN;

  const char *kbase = a.k + (int64_t)k0 * a.k_row + kvh * a.k_head;
  const char *vbase = a.v + (int64_t)k0 * a.v_row + kvh * a.v_head;
  TileReader<DP> rd;
  rd.init(lane);
  TileCopy<DP, kBN, 4> kc, vc;
  kc.init(wave, lane, (int)a.k_row, a.bytes);
  vc.init(wave, lane, (int)a.v_row, a.bytes);
  auto start = [&](int tile, int buf) {
    const int n = min(lk - tile * kBN, kBN);
    kc.start(row_buffer(kbase, (int64_t)tile * kBN, n, a.k_row, a.bytes),
             lds_address(kt) + buf * kTile);
    vc.start(row_buffer(vbase, (int64_t)tile * kBN, n, a.v_row, a.bytes),
             lds_address(vt) + buf * kTile);
  };
  if (part < n_tiles) start(part, 0);

  u32x4 qf[KS];
  load_operand<DP>(a.q + (int64_t)t.b0 * a.q_row + head * a.q_head, a.q_row, row, lq, a.bytes, lane,
                   qf);
  int reach = 0;
  float slope2 = 0.f;
  if (BIAS == kBiasTable) {
    reach = a.buckets.start[a.buckets.per_side - 1];
    uint8_t *map = reinterpret_cast<uint8_t *>(lut + lut_size(reach));
    fill_map(map, a.buckets, threadIdx.x, kThreads * PARTS);   // (each thread reads what it wrote)
    fill_lut<T>(lut, map, a.buckets, a.table, head, threadIdx.x, kThreads * PARTS);
  }
  if (BIAS == kBiasSlope) slope2 = a.slopes[head] * kLog2e;
  float steps[16];
  slope_steps<BIAS>(steps, slope2);
  const ScoreScale sc = score_scale<CAP>(a.scale, a.cap);

  f32x16 acc[DT];
#pragma unroll
  for (int c = 0; c < DT; ++c) acc[c] = f32x16{};
  float m = -__builtin_inff(), l = 0.f;   // l: this lane's half of the row's sum
  bool dirty = false;

  // one tile per part; `masked`: some row's limit may fall into it
  auto step = [&](int turn, auto masked_tile) {
    constexpr bool masked = decltype(masked_tile)::value;
    const int tile = turn * PARTS + part, buf = turn & 1, key0 = tile * kBN;
    if (tile + PARTS < n_tiles) start(tile + PARTS, buf ^ 1);
    if (key0 < lim_hi) {
      const uint32_t kb = rd.at(lds_address(kt) + buf * kTile, rd.row);
      const uint32_t vb = rd.at(lds_address(vt) + buf * kTile, rd.col);
      f32x16 s[2] = {f32x16{}, f32x16{}};
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        s[0] = T::mfma(row_operand<DP>(kb, 0, i), qf[i], s[0]);
        s[1] = T::mfma(row_operand<DP>(kb, 32, i), qf[i], s[1]);
      }
      Affine f[2];
      float top = -__builtin_inff();
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        if (CAP) {
#pragma unroll
          for (int e = 0; e < 16; ++e) s[b][e] = score_x<CAP>(s[b][e], sc);
        }
        f[b] = add_bias<BIAS>(s[b], sc, key0 + 32 * b, row + shift, row_lo + shift, h, slope2, steps,
                              lut, reach);
        if (masked) {
          const int mine = lim - key0 - 32 * b - 4 * h;
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (row_of(e) >= mine) s[b][e] = -__builtin_inff();
        }
        float t = max3(s[b][0], s[b][1], s[b][2]);
#pragma unroll
        for (int e = 3; e < 15; e += 2) t = max3(t, s[b][e], s[b][e + 1]);
        t = max3(t, s[b][15], s[b][15]);
        top = fmaxf(top, __builtin_fmaf(t, f[b].a, f[b].b));
      }
      top = max_halves(top);
      if (__any(top > m + slack)) {
        const float mn = top > m + slack ? top : m;
        const float r = mn == -__builtin_inff() ? 1.f : fast_exp2(m - mn);
        m = mn;
        l *= r;
#pragma unroll
        for (int c = 0; c < DT; ++c)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[c][e] *= r;
      }
      const float ms = (m == -__builtin_inff() ? 0.f : m) - p_shift;
      u32x4 p[kBN / 16];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const float off = f[b].b - ms;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          s[b][e] = fast_exp2(__builtin_fmaf(s[b][e], f[b].a, off));
          l += s[b][e];
        }
        // the probabilities are rounded to the operands' type for the second product (with
        // REST, a second term holds what that loses); the sum above is of the unrounded ones
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int w = 0; w < 4; ++w)
            p[2 * b + i][w] = T::pack(s[b][8 * i + 2 * w], s[b][8 * i + 2 * w + 1]);
      }
      // masked places may hold anything: 0 times an infinity or NaN would spoil the sums, so
      // in a tile with such values they are taken as 0 and added for who sees them at the end
      bool clean = true;
      if (masked && lim_lo < lk) {
        uint32_t bad = 0;
#pragma unroll 1   // (rolled and with the reads below kept apart: it must not cost registers)
        for (int i = 0; i < kBN / 16; ++i)
#pragma unroll
          for (int c = 0; c < DT; ++c)
            bad |= nonfinite<T>(col_operand<DP>(vb, 16 * i, c));
        clean = !__any(bad != 0);
        dirty |= !clean;
      }
#pragma unroll
      for (int i = 0; i < kBN / 16; ++i) {
        u32x4 rest;
        if (REST) {
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const int e = 8 * (i & 1) + 2 * w;
            rest[w] = T::pack(s[i >> 1][e] - T::lo(p[i][w]), s[i >> 1][e + 1] - T::hi(p[i][w]));
          }
        }
#pragma unroll
        for (int c = 0; c < DT; ++c) {
          u32x4 v = col_operand<DP>(vb, 16 * i, c);
          if (masked && !clean) v = finite_part<T>(v);
          acc[c] = T::mfma(v, p[i], acc[c]);
          if (REST) acc[c] = T::mfma(v, rest, acc[c]);
        }
      }
    }
    copies_barrier();
  };

  copies_barrier();
  const int turns = (n_tiles + PARTS - 1) / PARTS;
  const int whole = min(max(lim_lo, 0) / kBN, n_tiles) / PARTS;   // of tiles that every row sees
  for (int turn = 0; turn < whole; ++turn) step(turn, std::false_type{});
  for (int turn = whole; turn < turns; ++turn) step(turn, std::true_type{});

  l = sum_halves(l);
  if (PARTS == 2) {   // [wave][column block, quad][lane] of the other part's output; m, l; flags
    f32x4 *o = reinterpret_cast<f32x4 *>(lds) + wave * DT * 4 * 64 + lane;
    f32x2 *ml = reinterpret_cast<f32x2 *>(lds + 4 * DT * 4 * 64 * 16) + wave * 64 + lane;
    int *flag = reinterpret_cast<int *>(lds + 4 * DT * 4 * 64 * 16 + 4 * 64 * 8) + wave;
    if (part == 1) {
#pragma unroll
      for (int c = 0; c < DT; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          o[(4 * c + e) * 64] = f32x4{acc[c][4 * e], acc[c][4 * e + 1], acc[c][4 * e + 2], acc[c][4 * e + 3]};
      *ml = f32x2{m, l};
      if (lane == 0) *flag = dirty;
    }
    __syncthreads();
    if (part == 1) return;
    const f32x2 other = *ml;
    const float mn = fmaxf(m, other[0]), base = mn == -__builtin_inff() ? 0.f : mn;
    const float f0 = fast_exp2(m - base), f1 = fast_exp2(other[0] - base);
    m = mn;
    l = l * f0 + other[1] * f1;
    dirty |= *flag != 0;
#pragma unroll
    for (int c = 0; c < DT; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const f32x4 x = o[(4 * c + e) * 64];
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[c][4 * e + i] = acc[c][4 * e + i] * f0 + x[i] * f1;
      }
  }
  const bool ok = row < lq;
  const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);   // a NaN sum stays one
  store_row<T, DT, REST>(
      a.o + (int64_t)(t.b0 + row) * a.o_row + head * a.o_head, ok, a.bytes, acc, inv, lane,
      REST ? a.rest + (int64_t)(t.b0 + row) * a.rest_row + head * a.rest_head : nullptr);
  if (ok && h == 0)
    a.lse[(int64_t)head * a.q_rows + t.b0 + row] =
        l == 0.f ? -__builtin_inff() : (m - p_shift + __builtin_amdgcn_logf(l)) * kLn2;
  if (dirty) {
    __threadfence_block();
    const int first = whole * PARTS * kBN;   // from here on tiles were looked through
    for (int r = row_lo; r < min(row_lo + 32, lq); ++r)
      for (int d = lane; 2 * d < a.bytes; d += 64) {
        const float x = nonfinite_sum<T>(vbase, a.v_row, first, limit(r), d);
        char *o = a.o + (int64_t)(t.b0 + r) * a.o_row + head * a.o_head;
        if (x != 0.f) T::store(o, d, T::load(o, d) + x);
      }
  }
}

template <class T, int DP, int CAP, int BIAS, bool REST, int PARTS>
hipError_t launch_parts(const AttnArgs &a, int64_t blocks, hipStream_t s) {
  static LdsLimit limit;
  constexpr int kTiles = PARTS * 4 * kBN * DP * 2;
  int lds = kTiles;
  if (BIAS == kBiasTable) {
    const int reach = a.buckets.start[a.buckets.per_side - 1];
    lds += lut_size(reach) * 4 + map_bytes(reach);
  }
  hipError_t e = limit.set(reinterpret_cast<const void *>(&attend_kernel<T, DP, CAP, BIAS, REST, PARTS>),
                           kTiles + lut_size(kMaxReach) * 4 + map_bytes(kMaxReach));
  if (e != hipSuccess) return e;
  attend_kernel<T, DP, CAP, BIAS, REST, PARTS>
      <<<dim3((uint32_t)blocks), kThreads * PARTS, lds, s>>>(a);
  return hipGetLastError();
}

// Two groups of wavefronts per block while there is one block per compute unit; up to two, if
// most are of one document (under a causal mask its last blocks alone set the time then). Two
// groups / one, causal, at n blocks: 2048 rows, 16 heads of 128, n = 256 50.0 / 64.3 us; 3600 rows,
// n = 464 68.8 / 88.6; 4 documents of 1000, 8 heads of 64, n = 256 17.7 / 23.3; 4096 rows, 16 heads
// of 64, n = 512 54.9 / 68.8; 9 documents of 400, 8 heads of 128, n = 288 28.0 / 21.2; 12 of 500,
// 8 heads of 64 and slopes, n = 384 21.5 / 18.5.
bool use_parts(const AttnArgs &a, int64_t blocks) {
  const int64_t longest = (int64_t)((a.max_q + kBM - 1) / kBM) * a.heads;
  return blocks <= kSeqCus || (blocks <= 2 * kSeqCus && 2 * longest > blocks);
}

// An upper bound of the documents' tiles; the blocks past the last one end at once.
int64_t block_count(const AttnArgs &a) {
  const int64_t tiles = (int64_t)a.q_rows / kBM + a.docs;
  const int64_t by_max = (int64_t)a.docs * (((int64_t)a.max_q + kBM - 1) / kBM);
  return (tiles < by_max ? tiles : by_max) * a.heads;
}

template <class T, int DP, int CAP, int BIAS, bool REST>
hipError_t launch_form(const AttnArgs &a, hipStream_t s) {
  const int64_t blocks = block_count(a);
  if (blocks == 0) return hipSuccess;
  if (use_parts(a, blocks)) return launch_parts<T, DP, CAP, BIAS, REST, 2>(a, blocks, s);
  return launch_parts<T, DP, CAP, BIAS, REST, 1>(a, blocks, s);
}

template <class T, int DP, int CAP, int BIAS>
hipError_t launch(const AttnArgs &a, hipStream_t s) {
  if (a.rest) return launch_form<T, DP, CAP, BIAS, true>(a, s);
  return launch_form<T, DP, CAP, BIAS, false>(a, s);
}

template <class T, int DP, int CAP>
hipError_t by_bias(const AttnArgs &a, hipStream_t s) {
  if (a.table) return launch<T, DP, CAP, kBiasTable>(a, s);
  if (a.slopes) return launch<T, DP, CAP, kBiasSlope>(a, s);
  return launch<T, DP, CAP, kBiasNone>(a, s);
}

template <class T, int DP>
hipError_t by_cap(const AttnArgs &a, hipStream_t s) {
  switch (cap_kind(a)) {
    case kCapNone: return by_bias<T, DP, kCapNone>(a, s);
    case kCapNear: return by_bias<T, DP, kCapNear>(a, s);
    default: return by_bias<T, DP, kCapFar>(a, s);
  }
}

}  // namespace

bool attend_fits(const AttnArgs &a) { return block_count(a) <= kMaxBlocks; }

hipError_t launch_attend(const AttnArgs &a, hipStream_t s) {
  if (a.bytes <= 128) return a.fp16 ? by_cap<Fp16, 64>(a, s) : by_cap<Bf16, 64>(a, s);
  return a.fp16 ? by_cap<Fp16, 128>(a, s) : by_cap<Bf16, 128>(a, s);
}

}  // namespace bgp
