// Attention of few query rows over long histories (one new row per run over a cache of keys
// and values): bound by reading K and V once, so the work is split over the keys.
//
// The group x queries rows that share a key head are the columns of one score tile (32 of
// them, fewer are padding: the matrix instructions have 10 times the rate that memory can
// feed). A block takes a range of keys, its 4 wavefronts take 32 keys each in turn, every
// one with LDS buffers and copies of its own and no barrier in the loop; the blocks' sums
// are joined by a second kernel in the order of the ranges.
#include "seq_dev.h"

namespace bgp {
namespace {

constexpr int kThreads = 256;
constexpr int kKeys = 32;      // keys of a wavefront's step
constexpr int kRows = 32;      // rows of a tile
constexpr float kSlack = 8.f;  // as in the general form

struct FewPlan {
  int row_tiles, rows, chunk, chunks;  // rows: kept per tile; chunk: keys of a block
};

FewPlan plan(int docs, int kv_heads, int group, int max_q, int max_k) {
  FewPlan p;
  const int64_t r = (int64_t)group * max_q;
  p.row_tiles = (int)((r + kRows - 1) / kRows);
  p.rows = (int)(r < kRows ? r : kRows);
  const int64_t units = (int64_t)docs * kv_heads * p.row_tiles;
  // about 8 blocks per compute unit if the keys allow it, none under 128 keys
  int64_t c = ((int64_t)max_k * units / (8 * (int64_t)kSeqCus) + 127) / 128 * 128;
  if (c < 128) c = 128;
  if (c > 4096) c = 4096;
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
__host__ __device__ inline Part part_of(float *base, const FewPlan &p, int64_t units) {
  return Part{base, base + ((units * p.chunks * p.rows * 2 + 63) / 64) * 64};
}

template <class T, int DP, bool CAP, int BIAS>
__global__ __launch_bounds__(kThreads, 1) void few_kernel(const AttnArgs a, const FewPlan p,
                                                          float *part) {
  constexpr int KS = DP / 16, DT = DP / 32;
  constexpr int kTile = kKeys * DP * 2;
  constexpr int kCopies = 2 * (kTile / 1024);       // copy instructions of a step
  constexpr int kLine = DP + 4;                     // floats of a row in the join below
  extern __shared__ __align__(1024) char lds[];
  __shared__ float ml[4][kRows][2];
  __shared__ int any_dirty;
  uint8_t *map = reinterpret_cast<uint8_t *>(lds + 16 * kTile);

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
  const int lim_lo = limit(0), lim_hi = limit(lq - 1);
  const int n_chunks = max((lim_hi + p.chunk - 1) / p.chunk, 1);
  if (chunk >= n_chunks || n_chunks > p.chunks) return;
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
  char *mine = lds + wave * 4 * kTile;              // K, V of two steps
  auto start = [&](int key, int buf) {
    const int n = min(lk - key, kKeys);
    kc.start(row_buffer(kbase, key, n, a.k_row, a.bytes), lds_address(mine) + buf * 2 * kTile);
    vc.start(row_buffer(vbase, key, n, a.v_row, a.bytes),
             lds_address(mine) + (buf * 2 + 1) * kTile);
  };
  int key = key_lo + wave * kKeys;
  if (key < key_hi) start(key, 0);

  u32x4 qf[KS];
  load_operand<DP>(a.q + (int64_t)(q0 + i) * a.q_row + head * a.q_head, 0, live ? 0 : 1, 1,
                   a.bytes, lane, qf);
  int reach = 0, nb = 0;
  float slope2 = 0.f, far = 0.f;
  if (BIAS == kBiasTable) {   // buckets by distance -reach..reach
    reach = a.buckets.start[a.buckets.per_side - 1];
    nb = a.buckets.two_sided ? 2 * a.buckets.per_side : a.buckets.per_side;
    far = T::load(a.table, (int64_t)head * nb + a.buckets.per_side - 1) * kLog2e;
    if (key_hi + 31 - shift > -reach)
      for (int d = threadIdx.x; d <= 2 * reach; d += kThreads)
        map[d] = (uint8_t)bucket_of(a.buckets, d - reach);
  }
  if (BIAS == kBiasSlope) slope2 = a.slopes[head] * kLog2e;
  ScoreScale sc;
  sc.cap2 = a.cap * kLog2e;
  sc.c = CAP ? 2.f * kLog2e * a.scale / a.cap : a.scale * kLog2e;

  f32x16 acc[DT];
#pragma unroll
  for (int c = 0; c < DT; ++c) acc[c] = f32x16{};
  float m = -__builtin_inff(), l = 0.f;
  bool dirty = false;
  if (threadIdx.x == 0) any_dirty = 0;
  __syncthreads();

  for (int buf = 0; key < key_hi; key += 4 * kKeys, buf ^= 1) {
    // the buffer that is filled next was read in the step before
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (key + 4 * kKeys < key_hi) {
      start(key + 4 * kKeys, buf ^ 1);
      wait_copies<kCopies>();
    } else {
      wait_copies<0>();
    }
    const uint32_t kb = rd.at(lds_address(mine) + buf * 2 * kTile, rd.row);
    const uint32_t vb = rd.at(lds_address(mine) + (buf * 2 + 1) * kTile, rd.col);
    f32x16 s = {};
#pragma unroll
    for (int k = 0; k < KS; ++k) s = T::mfma(row_operand<DP>(kb, 0, k), qf[k], s);
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = scaled<CAP>(s[e], sc);
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
          const int b = map[min(max(d, -reach), reach) + reach];
          s[e] += T::load(a.table, (int64_t)head * nb + b) * kLog2e;
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
    if (__any(top > m + kSlack)) {
      const float mn = top > m + kSlack ? top : m;
      const float f = mn == -__builtin_inff() ? 1.f : fast_exp2(m - mn);
      m = mn;
      l *= f;
#pragma unroll
      for (int c = 0; c < DT; ++c)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[c][e] *= f;
    }
    const float ms = m == -__builtin_inff() ? 0.f : m;
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
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int c = 0; c < DT; ++c) {
        u32x4 v = col_operand<DP>(vb, 16 * k, c);
        if (!clean) v = finite_part<T>(v);
        acc[c] = T::mfma(v, pr[k], acc[c]);
      }
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
      const float inv = ll > 0.f ? 1.f / ll : (ll == 0.f ? 0.f : ll);
      if (2 * d < a.bytes)
        *reinterpret_cast<u32x2 *>(a.o + (int64_t)(q0 + qi) * a.o_row + qh * a.o_head + 2 * d) =
            u32x2{T::pack(x[0] * inv, x[1] * inv), T::pack(x[2] * inv, x[3] * inv)};
      if (d == 0)
        a.lse[(int64_t)qh * a.q_rows + q0 + qi] =
            ll == 0.f ? -__builtin_inff() : (mm + __builtin_amdgcn_logf(ll)) * kLn2;
    } else {
      const int64_t units = (int64_t)a.docs * a.kv_heads * p.row_tiles;
      const Part pt = part_of(part, p, units);
      const int64_t at =
          ((((int64_t)doc * a.kv_heads + kvh) * p.row_tiles + rt) * p.chunks + chunk) * p.rows + q;
      *reinterpret_cast<f32x4 *>(pt.o + at * DP + d) = x;
      if (d == 0) {
        pt.ml[2 * at] = mm;
        pt.ml[2 * at + 1] = ll;
      }
    }
  }
}

// One block per row: the sums of its ranges, in their order.
template <class T, int DP>
__global__ __launch_bounds__(256) void few_join(const AttnArgs a, const FewPlan p, float *part) {
  constexpr int kQuads = DP / 4, kSlices = 256 / kQuads;
  __shared__ f32x4 so[kSlices][kQuads];
  __shared__ float sm[4];
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
  const int prefix = (a.causal && a.prefix) ? a.prefix[doc] : 0;
  const int lim_hi = a.causal ? min(lk, max(lk, prefix)) : lk;
  const int n = (lim_hi + p.chunk - 1) / p.chunk;
  if (n <= 1 || n > p.chunks) return;               // written by the first kernel
  const int i = r % lq, head = kvh * a.group + r / lq;
  const int64_t units = (int64_t)a.docs * a.kv_heads * p.row_tiles;
  const Part pt = part_of(part, p, units);
  const int64_t at =
      ((((int64_t)doc * a.kv_heads + kvh) * p.row_tiles + rt) * p.chunks) * (int64_t)p.rows + q;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float mm = -__builtin_inff();
  for (int c = threadIdx.x; c < n; c += 256) mm = fmaxf(mm, pt.ml[2 * (at + (int64_t)c * p.rows)]);
#pragma unroll
  for (int o = 32; o; o >>= 1) mm = fmaxf(mm, __shfl_xor(mm, o));
  if (lane == 0) sm[wave] = mm;
  __syncthreads();
  mm = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3]));
  const float base = mm == -__builtin_inff() ? 0.f : mm;
  const int quad = threadIdx.x % kQuads, slice = threadIdx.x / kQuads;
  f32x4 x = {};
  float ll = 0.f;
  for (int c = slice; c < n; c += kSlices) {
    const int64_t k = at + (int64_t)c * p.rows;
    const float f = fast_exp2(pt.ml[2 * k] - base);
    ll += f * pt.ml[2 * k + 1];
    x += f * *reinterpret_cast<const f32x4 *>(pt.o + k * DP + 4 * quad);
  }
  so[slice][quad] = x;
  __shared__ float ssum[kSlices];
  if (quad == 0) ssum[slice] = ll;
  __syncthreads();
  if (slice) return;
  ll = 0.f;
  x = f32x4{};
#pragma unroll
  for (int s = 0; s < kSlices; ++s) {
    ll += ssum[s];
    x += so[s][quad];
  }
  const float inv = ll > 0.f ? 1.f / ll : (ll == 0.f ? 0.f : ll);
  if (8 * quad < a.bytes)
    *reinterpret_cast<u32x2 *>(a.o + (int64_t)(q0 + i) * a.o_row + head * a.o_head + 8 * quad) =
        u32x2{T::pack(x[0] * inv, x[1] * inv), T::pack(x[2] * inv, x[3] * inv)};
  if (quad == 0)
    a.lse[(int64_t)head * a.q_rows + q0 + i] =
        ll == 0.f ? -__builtin_inff() : (mm + __builtin_amdgcn_logf(ll)) * kLn2;
}

template <class T, int DP, bool CAP, int BIAS>
hipError_t launch(const AttnArgs &a, float *part, hipStream_t s) {
  static LdsLimit limit;
  const FewPlan p = plan(a.docs, a.kv_heads, a.group, a.max_q, a.max_k);
  int lds = 16 * kKeys * DP * 2;
  const int join = 4 * kRows * (DP + 4) * 4;
  if (lds < join) lds = join;
  const int most = lds + 2 * kMaxReach + 4;
  if (BIAS == kBiasTable) lds += 2 * a.buckets.start[a.buckets.per_side - 1] + 4;
  hipError_t e = limit.set(reinterpret_cast<const void *>(&few_kernel<T, DP, CAP, BIAS>), most);
  if (e != hipSuccess) return e;
  const int64_t units = (int64_t)a.docs * a.kv_heads * p.row_tiles;
  few_kernel<T, DP, CAP, BIAS>
      <<<dim3((uint32_t)(units * p.chunks)), kThreads, lds, s>>>(a, p, part);
  if (p.chunks > 1)
    few_join<T, DP><<<dim3((uint32_t)(units * p.rows)), 256, 0, s>>>(a, p, part);
  return hipGetLastError();
}

template <class T, int DP>
hipError_t by_bias(const AttnArgs &a, float *part, hipStream_t s) {
  const int bias = a.table ? kBiasTable : (a.slopes ? kBiasSlope : kBiasNone);
  if (a.cap > 0.f) {
    if (bias == kBiasTable) return launch<T, DP, true, kBiasTable>(a, part, s);
    if (bias == kBiasSlope) return launch<T, DP, true, kBiasSlope>(a, part, s);
    return launch<T, DP, true, kBiasNone>(a, part, s);
  }
  if (bias == kBiasTable) return launch<T, DP, false, kBiasTable>(a, part, s);
  if (bias == kBiasSlope) return launch<T, DP, false, kBiasSlope>(a, part, s);
  return launch<T, DP, false, kBiasNone>(a, part, s);
}

}  // namespace

bool attend_use_few(int32_t docs, int32_t kv_heads, int32_t group, int32_t max_q, int32_t max_k) {
  (void)docs, (void)kv_heads, (void)max_k;
  return (int64_t)group * max_q <= kRows;
}

size_t attend_few_bytes(int32_t docs, int32_t kv_heads, int32_t group, int32_t max_q, int32_t max_k,
                        int32_t dim) {
  const FewPlan p = plan(docs, kv_heads, group, max_q, max_k);
  const int64_t units = (int64_t)docs * kv_heads * p.row_tiles;
  if (p.chunks == 1) return 0;
  const int64_t rows = units * p.chunks * p.rows;
  return (size_t)((rows * 2 + 63) / 64 * 64 + rows * (dim <= 64 ? 64 : 128)) * 4;
}

hipError_t launch_attend_few(const AttnArgs &a, float *part, hipStream_t s) {
  if (a.bytes <= 128)
    return a.fp16 ? by_bias<Fp16, 64>(a, part, s) : by_bias<Bf16, 64>(a, part, s);
  return a.fp16 ? by_bias<Fp16, 128>(a, part, s) : by_bias<Bf16, 128>(a, part, s);
}

}  // namespace bgp
