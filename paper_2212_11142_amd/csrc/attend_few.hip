// Attention of few query rows over long histories (one new row per run over a cache of keys
// and values): bound by reading K and V once, so the work is split over the keys.
//
// The group x queries rows that share a key head are the columns of one score tile (32 of
// them, fewer are padding: the matrix instructions have 10 times the rate that memory can
// feed). A block takes a range of keys, its 4 wavefronts take 32 keys each in turn, every
// one with LDS buffers and copies of its own and no barrier in the loop; a second kernel
// joins the blocks' sums in the order of the ranges. (Joining them in the first kernel's last
// block costs more than the launch it saves: what blocks hand over must pass the L2 of each
// XCD, 15.4 against 7.6 + 4.4 us for 4095 keys and 4 key heads of 128.)
//
// Measured, 16 heads of 128 with 4 of keys: 64 caches of up to 32,768 keys, 2.2 GB, 421 us, 5.3
// TB/s (reading alone reaches 6.3), 7 of them the join; 64 full ones, 4.3 GB, 767 us, 5.6 TB/s;
// one of 4095 keys, 8.4 MB, 7.7 us and 3.9 for the join, bound by the latency of a wavefront's one
// step (a block has 128 keys) and of the second launch.
#include "seq_dev.h"

namespace bgp {
namespace {

constexpr int kThreads = 256;
constexpr int kKeys = 32;      // keys of a wavefront's step
constexpr int kRows = 32;      // rows of a tile
// Keys of a block, at most: 64 caches of 32,768 at most, 4 key heads of 128, with 512 / 1024 /
// 2048 / unlimited: 445 / 429 / 445 / 442 us; the same, all full: 808 / 767 / 781 / 781.
constexpr int kFewChunk = 1024;
constexpr int kMaxValues = 4096;   // of the table for a group

constexpr int few_tiles(int dp) {
  const int tiles = 8 * kKeys * dp * 2, sums = 4 * kRows * (dp + 4) * 4;
  return tiles > sums ? tiles : sums;
}

struct FewPlan {
  int row_tiles, rows, chunk, chunks;  // rows: kept per tile; chunk: keys of a block
};

FewPlan plan(int docs, int kv_heads, int group, int max_q, int max_k) {
  FewPlan p;
  const int64_t r = (int64_t)group * max_q;
  p.row_tiles = (int)((r + kRows - 1) / kRows);
  p.rows = (int)(r < kRows ? r : kRows);
  const int64_t units = (int64_t)docs * kv_heads * p.row_tiles;
  auto up = [](int64_t x) { return (x + 127) / 128 * 128; };
  // Few rows: about 16 blocks per compute unit; where those would have less than 512 keys each,
  // one per compute unit, of 128 keys at least. Full tiles, whose sums are the larger: one per
  // compute unit.
  int64_t c = up(max_k * units / (16 * kSeqCus));
  if (r > kRows || c < 512) {
    c = up(max_k * units / kSeqCus);
    if (r <= kRows && c > 512) c = 512;
    if (c < 128) c = 128;
  }
  if (r <= kRows && c > kFewChunk) c = kFewChunk;
  // What the split saves, max_k - c keys of a block, has to pay for the second kernel and the
  // sums between them. Without / with: 192 rows of 16 heads of 128 9.3 / 14.6 us, 1024 rows
  // 19.6 / 50; 64 rows over 4096 keys, 8 heads of 128, 36 / 14; one row, 500 keys 9.1 / 9.1;
  // 64 rows of their own 1000 keys 24.8 / 28.7.
  // (max_k may be a loose bound, and the second kernel has a block per row: both grids fit, or
  // there is no second kernel)
  if (max_k - c <= 384 + units * p.rows / 4 || units * p.rows > kMaxBlocks)
    c = max_k > 0 ? up(max_k) : 128;
  if (c > 1 << 30) c = 1 << 30;
  const int64_t most = units > 0 && units < kMaxBlocks ? kMaxBlocks / units : 1;   // ranges
  const int64_t least = up((max_k + most - 1) / most);
  if (c < least) c = least;
  p.chunk = (int)c;
  p.chunks = (int)((max_k + c - 1) / c);
  if (p.chunks < 1) p.chunks = 1;
  return p;
}

// Workspace: per (document, kv head, row tile, chunk) the maxima and sums of its rows, then
// the unnormalised outputs [rows][DP].
struct Part {
  float *ml, *o;
};
__host__ __device__ inline Part part_of(void *base, const FewPlan &p, int64_t units) {
  float *f = static_cast<float *>(base);
  return Part{f, f + (units * p.chunks * p.rows * 2 + 63) / 64 * 64};
}

// Writes 4 columns of a finished row (sum l, times 2^p_shift, at the maximum m, in log 2 units).
template <class T, bool REST>
__device__ inline void write_quad(const AttnArgs &a, int row, int head, int d, f32x4 x, float m,
                                  float l, float p_shift) {
  const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);   // a NaN sum stays one
  x *= inv;
  if (2 * d < a.bytes) {
    const u32x2 w = {as_stored(T::pack(x[0], x[1])), as_stored(T::pack(x[2], x[3]))};
    *reinterpret_cast<u32x2 *>(a.o + (int64_t)row * a.o_row + head * a.o_head + 2 * d) = w;
    if (REST)
      *reinterpret_cast<u32x2 *>(a.rest + (int64_t)row * a.rest_row + head * a.rest_head + 2 * d) =
          u32x2{T::pack(x[0] - T::lo(w[0]), x[1] - T::hi(w[0])),
                T::pack(x[2] - T::lo(w[1]), x[3] - T::hi(w[1]))};
  }
  if (d == 0)
    a.lse[(int64_t)head * a.q_rows + row] =
        l == 0.f ? -__builtin_inff() : (m - p_shift + __builtin_amdgcn_logf(l)) * kLn2;
}

// A wavefront has room for one tile of K and one of V, asked for again as soon as they have
// been read: the eight wavefronts that a compute unit then holds keep more loads in flight than
// four with two tiles each (64 caches of 2048 keys, 4 key heads of 128: 48 against 58 us; one
// of 4095: 9.5 against 10.2).
template <class T, int DP, int CAP, int BIAS, bool REST>
__global__ __launch_bounds__(kThreads, 2) void few_kernel(const AttnArgs a, const FewPlan p,
                                                          void *part) {
  constexpr int KS = DP / 16, DT = DP / 32;
  constexpr int kTile = kKeys * DP * 2;
  constexpr int kCopies = kTile / 1024;             // copy instructions of a tile
  constexpr int kLine = DP + 4;                     // floats of a row in the join below
  extern __shared__ __align__(1024) char lds[];
  __shared__ float ml[4][kRows][2];
  __shared__ int any_dirty;
  // tiles (then the wavefronts' sums), the group's rows of the table, buckets by distance
  float *values = reinterpret_cast<float *>(lds + few_tiles(DP));

  int id = blockIdx.x;
  const int kvh = id % a.kv_heads;
  id /= a.kv_heads;
  const int chunk = id % p.chunks;
  id /= p.chunks;
  const int rt = id % p.row_tiles, doc = id / p.row_tiles;
  const int q0 = max(a.qb[doc], 0);
  const int lq = max(min(a.qe[doc], a.q_rows) - q0, 0);
  const int rows = min(a.group * lq - rt * kRows, kRows);
  if (rows <= 0) return;
  const int k0 = max(a.kb[doc], 0);
  const int lk = max(min(a.ke[doc], a.k_rows) - k0, 0);
  const int prefix = (a.causal && a.prefix) ? a.prefix[doc] : 0;
  const int shift = lk - lq;
  auto limit = [&](int i) { return a.causal ? min(lk, max(i + shift + 1, prefix)) : lk; };
  const float slack = Probs<T>::slack(lk), p_shift = Probs<T>::shift(lk);
  const int n_chunks = max((limit(lq - 1) + p.chunk - 1) / p.chunk, 1);
  if (chunk >= n_chunks || n_chunks > p.chunks) return;
  // a tile within one head has a range of the queries
  const int r_lo = rt * kRows, r_hi = r_lo + rows - 1;
  const bool one_head = r_lo / lq == r_hi / lq;
  const int lim_lo = limit(one_head ? r_lo % lq : 0), lim_hi = limit(one_head ? r_hi % lq : lq - 1);
  const int key_lo = chunk * p.chunk, key_hi = min(key_lo + p.chunk, lim_hi);

  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), h = lane >> 5;
  const int r = rt * kRows + (lane & 31);
  const bool live = (lane & 31) < rows;
  const int g = live ? r / lq : 0, i = live ? r % lq : 0;
  const int lim = live ? limit(i) : 0, pos = i + shift;
  const int head = kvh * a.group + g;

  const char *kbase = a.k + (int64_t)k0 * a.k_row + kvh * a.k_head;
  const char *vbase = a.v + (int64_t)k0 * a.v_row + kvh * a.v_head;
  TileReader<DP> rd;
  rd.init(lane);
  TileCopy<DP, kKeys, 1> kc, vc;
  kc.init(0, lane, (int)a.k_row, a.bytes);
  vc.init(0, lane, (int)a.v_row, a.bytes);
  char *mine = lds + wave * 2 * kTile;
  // (past the last key: nothing but zeros is copied, so that the waits below count evenly)
  auto start_k = [&](int key) {
    kc.start(row_buffer(kbase, key, key < key_hi ? min(lk - key, kKeys) : 0, a.k_row, a.bytes),
             lds_address(mine));
  };
  auto start_v = [&](int key) {
    vc.start(row_buffer(vbase, key, key < key_hi ? min(lk - key, kKeys) : 0, a.v_row, a.bytes),
             lds_address(mine) + kTile);
  };
  u32x4 qf[KS];   // (asked for before the tiles: their arrival is waited for in order)
  load_operand<DP>(a.q + (int64_t)(q0 + i) * a.q_row + head * a.q_head, 0, live ? 0 : 1, 1,
                   a.bytes, lane, qf);
  int key = key_lo + wave * kKeys;
  if (key < key_hi) {
    start_k(key);
    start_v(key);
  }

  int reach = 0, span = 1, nb = 0;
  float slope2 = 0.f, far = 0.f;
  uint8_t *map = nullptr;
  if (BIAS == kBiasTable) {   // buckets by distance -span..span
    reach = a.buckets.start[a.buckets.per_side - 1];
    span = ahead_reach(reach);
    nb = bucket_count(a.buckets);
    map = reinterpret_cast<uint8_t *>(values + a.group * nb);
    far = T::load(a.table, (int64_t)head * nb + a.buckets.per_side - 1) * kLog2e;
    if (key_hi + 31 - shift > -reach) {
      for (int d = threadIdx.x; d <= 2 * span; d += kThreads)
        map[d] = (uint8_t)bucket_of(a.buckets, d - span);
      for (int d = threadIdx.x; d < a.group * nb; d += kThreads)
        values[d] = T::load(a.table, (int64_t)kvh * a.group * nb + d) * kLog2e;
    }
  }
  if (BIAS == kBiasSlope) slope2 = a.slopes[head] * kLog2e;
  const ScoreScale sc = score_scale<CAP>(a.scale, a.cap);

  f32x16 acc[DT];
#pragma unroll
  for (int c = 0; c < DT; ++c) acc[c] = f32x16{};
  float m = -__builtin_inff(), l = 0.f;
  bool dirty = false;
  if (threadIdx.x == 0) any_dirty = 0;
  __syncthreads();

  const uint32_t kb = rd.at(lds_address(mine), rd.row);
  const uint32_t vb = rd.at(lds_address(mine) + kTile, rd.col);
  for (; key < key_hi; key += 4 * kKeys) {
    wait_copies<kCopies>();       // K has arrived
    f32x16 s = {};
#pragma unroll
    for (int k = 0; k < KS; ++k) s = T::mfma(row_operand<DP>(kb, 0, k), qf[k], s);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    start_k(key + 4 * kKeys);
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = __builtin_fmaf(score_x<CAP>(s[e], sc), sc.a, sc.b);
    if (BIAS == kBiasSlope) {
      const float d0 = (float)(key + 4 * h - pos);
#pragma unroll
      for (int e = 0; e < 16; ++e)
        s[e] = __builtin_fmaf(-slope2, __builtin_fabsf(d0 + (float)(8 * (e >> 2) + (e & 3))), s[e]);
    }
    if (BIAS == kBiasTable) {
      if (key + 31 - shift <= -reach) {             // every pair far behind
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] += far;
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int d = key + 4 * h - pos + 8 * (e >> 2) + (e & 3);
          s[e] += values[g * nb + map[min(max(d, -span), span) + span]];
        }
      }
    }
    const bool masked = key + kKeys > lim_lo;
    if (masked) {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (key + 4 * h + 8 * (e >> 2) + (e & 3) >= lim) s[e] = -__builtin_inff();
    }
    float top = s[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) top = fmaxf(top, s[e]);
    top = max_halves(top);
    if (__any(top > m + slack)) {
      const float mn = top > m + slack ? top : m;
      const float f = mn == -__builtin_inff() ? 1.f : fast_exp2(m - mn);
      m = mn;
      l *= f;
#pragma unroll
      for (int c = 0; c < DT; ++c)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[c][e] *= f;
    }
    const float ms = (m == -__builtin_inff() ? 0.f : m) - p_shift;
    u32x4 pr[2];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      s[e] = fast_exp2(s[e] - ms);
      l += s[e];
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int w = 0; w < 4; ++w) pr[k][w] = T::pack(s[8 * k + 2 * w], s[8 * k + 2 * w + 1]);
    wait_copies<kCopies>();       // V has
    bool clean = true;
    if (masked && lim_lo < lk) {                    // as in the general form
      uint32_t bad = 0;
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int c = 0; c < DT; ++c) bad |= nonfinite<T>(col_operand<DP>(vb, 16 * k, c));
      clean = !__any(bad != 0);
      dirty |= !clean;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      u32x4 rest;   // what the rounding of the probabilities lost
      if (REST) {
#pragma unroll
        for (int w = 0; w < 4; ++w)
          rest[w] = T::pack(s[8 * k + 2 * w] - T::lo(pr[k][w]), s[8 * k + 2 * w + 1] - T::hi(pr[k][w]));
      }
#pragma unroll
      for (int c = 0; c < DT; ++c) {
        u32x4 v = col_operand<DP>(vb, 16 * k, c);
        if (!clean) v = finite_part<T>(v);
        acc[c] = T::mfma(v, pr[k], acc[c]);
        if (REST) acc[c] = T::mfma(v, rest, acc[c]);
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    start_v(key + 4 * kKeys);
  }
  l = sum_halves(l);

  // join the four wavefronts
  copies_barrier();
  if (dirty) any_dirty = 1;
  float *o = reinterpret_cast<float *>(lds);        // [4][rows][kLine]
  if (live) {
    if (h == 0) {
      ml[wave][lane & 31][0] = m;
      ml[wave][lane & 31][1] = l;
    }
#pragma unroll
    for (int c = 0; c < DT; ++c)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        *reinterpret_cast<f32x4 *>(o + (wave * kRows + (lane & 31)) * kLine + 32 * c + 2 * e + 4 * h) =
            f32x4{acc[c][e], acc[c][e + 1], acc[c][e + 2], acc[c][e + 3]};
  }
  __syncthreads();
  constexpr int kQuads = DP / 4;
  const int d = (threadIdx.x % kQuads) * 4;
  const int64_t unit = ((int64_t)doc * a.kv_heads + kvh) * p.row_tiles + rt;
  const Part pt = part_of(part, p, (int64_t)a.docs * a.kv_heads * p.row_tiles);
  for (int q = threadIdx.x / kQuads; q < rows; q += kThreads / kQuads) {
    float mm = ml[0][q][0];
#pragma unroll
    for (int w = 1; w < 4; ++w) mm = fmaxf(mm, ml[w][q][0]);
    const float base = mm == -__builtin_inff() ? 0.f : mm;
    float ll = 0.f;
    f32x4 x = {};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = fast_exp2(ml[w][q][0] - base);
      ll += f * ml[w][q][1];
      x += f * *reinterpret_cast<f32x4 *>(o + (w * kRows + q) * kLine + d);
    }
    const int rr = rt * kRows + q, qi = rr % lq, qh = kvh * a.group + rr / lq;
    if (any_dirty) {
      const int first = max(max(lim_lo, 0) / kKeys * kKeys, key_lo);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (2 * (d + e) < a.bytes)
          x[e] += nonfinite_sum<T>(vbase, a.v_row, first, min(limit(qi), key_hi), d + e);
    }
    if (n_chunks == 1) {
      write_quad<T, REST>(a, q0 + qi, qh, d, x, mm, ll, p_shift);
    } else {
      const int64_t at = (unit * p.chunks + chunk) * p.rows + q;
      *reinterpret_cast<f32x4 *>(pt.o + at * DP + d) = x;
      if (d == 0) {
        pt.ml[2 * at] = mm;
        pt.ml[2 * at + 1] = ll;
      }
    }
  }
}

// Joins the ranges: one block per row, slices of threads take its ranges in turn, each with a running maximum
// (so that all loads are under way at once), then join in order. Bound by latency: 4.0 us for
// 16 rows of 32 ranges, 7.4 for 1024 rows.
template <class T, int DP, bool REST>
__global__ __launch_bounds__(kThreads) void few_join(const AttnArgs a, const FewPlan p, void *part) {
  constexpr int kQuads = DP / 4, kSlices = kThreads / kQuads;
  __shared__ f32x4 so[kSlices][kQuads];
  __shared__ float sml[kSlices][2];
  int id = blockIdx.x;
  const int q = id % p.rows;
  id /= p.rows;
  const int rt = id % p.row_tiles;
  id /= p.row_tiles;
  const int kvh = id % a.kv_heads, doc = id / a.kv_heads;
  const int q0 = max(a.qb[doc], 0);
  const int lq = max(min(a.qe[doc], a.q_rows) - q0, 0);
  const int r = rt * kRows + q;
  if (r >= a.group * lq) return;
  const int lk = max(min(a.ke[doc], a.k_rows) - max(a.kb[doc], 0), 0);
  const int n = (lk + p.chunk - 1) / p.chunk;   // the last query sees every key
  if (n <= 1 || n > p.chunks) return;           // written by the first kernel
  const Part pt = part_of(part, p, (int64_t)a.docs * a.kv_heads * p.row_tiles);
  const int64_t at =
      (((int64_t)doc * a.kv_heads + kvh) * p.row_tiles + rt) * p.chunks * (int64_t)p.rows + q;
  const int quad = threadIdx.x % kQuads, slice = threadIdx.x / kQuads;
  float mm = -__builtin_inff(), ll = 0.f;
  f32x4 x = {};
#pragma unroll 4
  for (int c = slice; c < n; c += kSlices) {
    const int64_t k = at + (int64_t)c * p.rows;
    const float mc = pt.ml[2 * k], lc = pt.ml[2 * k + 1];
    const f32x4 xc = *reinterpret_cast<const f32x4 *>(pt.o + k * DP + 4 * quad);
    const float top = fmaxf(mm, mc), base = top == -__builtin_inff() ? 0.f : top;
    const float f = fast_exp2(mm - base), fc = fast_exp2(mc - base);
    ll = ll * f + lc * fc;
    x = x * f + xc * fc;
    mm = top;
  }
  so[slice][quad] = x;
  if (quad == 0) {
    sml[slice][0] = mm;
    sml[slice][1] = ll;
  }
  __syncthreads();
  if (slice) return;
  float top = mm;
#pragma unroll
  for (int s = 1; s < kSlices; ++s) top = fmaxf(top, sml[s][0]);
  const float base = top == -__builtin_inff() ? 0.f : top;
  const float f0 = fast_exp2(mm - base);
  ll *= f0;
  x *= f0;
#pragma unroll
  for (int s = 1; s < kSlices; ++s) {
    const float f = fast_exp2(sml[s][0] - base);
    ll += f * sml[s][1];
    x += f * so[s][quad];
  }
  write_quad<T, REST>(a, q0 + r % lq, kvh * a.group + r / lq, 4 * quad, x, top, ll,
                      Probs<T>::shift(lk));
}

template <class T, int DP, int CAP, int BIAS, bool REST>
hipError_t launch_form(const AttnArgs &a, const FewPlan &p, void *part, hipStream_t s) {
  static LdsLimit limit;
  int lds = few_tiles(DP);
  if (BIAS == kBiasTable)
    lds += a.group * bucket_count(a.buckets) * 4 + 2 * a.buckets.start[a.buckets.per_side - 1] + 4;
  hipError_t e = limit.set(reinterpret_cast<const void *>(&few_kernel<T, DP, CAP, BIAS, REST>),
                           few_tiles(DP) + kMaxValues * 4 + 2 * kMaxReach + 4);
  if (e != hipSuccess) return e;
  const int64_t units = (int64_t)a.docs * a.kv_heads * p.row_tiles;
  few_kernel<T, DP, CAP, BIAS, REST>
      <<<dim3((uint32_t)(units * p.chunks)), kThreads, lds, s>>>(a, p, part);
  if (p.chunks > 1)
    few_join<T, DP, REST><<<dim3((uint32_t)(units * p.rows)), kThreads, 0, s>>>(a, p, part);
  return hipGetLastError();
}

template <class T, int DP, int CAP, int BIAS>
hipError_t launch(const AttnArgs &a, void *part, hipStream_t s) {
  const FewPlan p = plan(a.docs, a.kv_heads, a.group, a.max_q, a.max_k);
  if (a.rest) return launch_form<T, DP, CAP, BIAS, true>(a, p, part, s);
  return launch_form<T, DP, CAP, BIAS, false>(a, p, part, s);
}

template <class T, int DP, int CAP>
hipError_t by_bias(const AttnArgs &a, void *part, hipStream_t s) {
  if (a.table) return launch<T, DP, CAP, kBiasTable>(a, part, s);
  if (a.slopes) return launch<T, DP, CAP, kBiasSlope>(a, part, s);
  return launch<T, DP, CAP, kBiasNone>(a, part, s);
}

template <class T, int DP>
hipError_t by_cap(const AttnArgs &a, void *part, hipStream_t s) {
  switch (cap_kind(a)) {
    case kCapNone: return by_bias<T, DP, kCapNone>(a, part, s);
    case kCapNear: return by_bias<T, DP, kCapNear>(a, part, s);
    default: return by_bias<T, DP, kCapFar>(a, part, s);
  }
}

}  // namespace

// Small calls too: while the general form's blocks of 128 queries leave compute units idle,
// 32 rows per block with the keys split over its wavefronts finish sooner. This form / the
// general one at n of its blocks, causal: 16 heads of 128, n = 64 11.8 / 18.0 us, 128 22.4 / 27.9,
// 192 37.3 / 32.2; 8 heads of 64, n = 64 9.9 / 15.4, 160 22.1 / 29.1; 16 of 64, n = 192 18.5 /
// 21.3; documents of 200 rows, 8 heads of 64, n = 128 9.6 / 11.4, 192 10.9 / 9.5.
constexpr int kFewBlocks = 160;

bool attend_use_few(const AttnArgs &a) {
  if ((int64_t)a.group * bucket_count(a.buckets) > kMaxValues) return false;
  if ((int64_t)a.group * a.max_q <= kRows) return true;
  const int64_t x = (int64_t)a.q_rows / 128 + a.docs, y = (int64_t)a.docs * ((a.max_q + 127) / 128);
  return (x < y ? x : y) * a.heads <= kFewBlocks;
}

bool attend_few_fits(const AttnArgs &a) {
  const FewPlan p = plan(a.docs, a.kv_heads, a.group, a.max_q, a.max_k);
  return (int64_t)a.docs * a.kv_heads * p.row_tiles * p.chunks <= kMaxBlocks;
}

size_t attend_few_bytes(const AttnArgs &a) {
  const FewPlan p = plan(a.docs, a.kv_heads, a.group, a.max_q, a.max_k);
  if (p.chunks == 1) return 0;
  const int64_t units = (int64_t)a.docs * a.kv_heads * p.row_tiles;
  const Part pt = part_of(nullptr, p, units);
  return (size_t)((pt.o - pt.ml) + units * p.chunks * p.rows * (a.bytes <= 128 ? 64 : 128)) * 4;
}

hipError_t launch_attend_few(const AttnArgs &a, void *part, hipStream_t s) {
  if (a.bytes <= 128)
    return a.fp16 ? by_cap<Fp16, 64>(a, part, s) : by_cap<Bf16, 64>(a, part, s);
  return a.fp16 ? by_cap<Fp16, 128>(a, part, s) : by_cap<Bf16, 128>(a, part, s);
}

}  // namespace bgp
