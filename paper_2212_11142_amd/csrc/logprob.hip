// Log probability of a given entry, entropy and best alternatives of rows of logits, and the
// gradient of the first two. With m = max x, d_v = c (x_v - m) (c the scale), A = sum e^d,
// B = sum e^d d:  lse = c m + log A,  logp = d_t - log A,  H = log A - B / A (a sum of terms
// of one sign, so that a peaked row's entropy keeps its digits).
//
// Bound by reading the logits once: a wavefront keeps a short row in registers, a block goes
// once over a long one with a running maximum, and where rows are few several blocks share
// one. The alternatives come from the same pass: every thread remembers its largest entry;
// the k-th largest of 64 (or 256) groups' entries bounds the k-th best from below, so that
// only the few threads above it look at their entries again. Order: larger value, then lower
// index; a NaN is no alternative.
#include <type_traits>

#include "seq_dev.h"

namespace bgp {
namespace {

constexpr int kThreads = 256;
constexpr int kList = 1024;        // candidates for the alternatives (8 blocks fit LDS)
constexpr int kOwners = 512;       // groups of entries that may hold candidates
// Alternatives up to which 64 groups' bound is taken instead of 256 groups'. Even a row of equal
// entries then lists 32 (k - 1) + 1 candidates at most in a block per row (8 (k - 1) + 1 with 256).
// With 64 / 256 groups: 40 alternatives of one row of 10,000 10.9 / 12.7 us, of 200 rows of
// 131,072 38.6 / 30.7.
constexpr int kSixtyFour = 32;
// Widest row of the one-wavefront form (64 entries a lane). 16,384 rows, this form / a block per
// row: 1100 wide bf16 14.3 / 54.6 us, with 5 alternatives 24.1 / 115; 4096 wide bf16 26.4 / 43.0,
// 38.1 / 95.9; 4096 wide fp32 42.3 / 41.1, 45.4 / 70.5.
constexpr int kWaveWidth = 4096;
constexpr float kLowest = -3.4028234663852886e38f;

enum { kBf16 = GP_BF16, kFp16 = GP_FP16, kFp32 = GP_FP32 };

// Largest number of three and of two (a NaN is passed over). fmaxf would first multiply each
// operand that was loaded by 1, against signalling NaN. The compiler does not wait before inline
// assembly for the results of transcendental instructions: none may be an operand here.
__device__ inline float top3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
__device__ inline float top2(float a, float b) {
  float r;
  asm("v_max_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}

template <int DT>
struct Elem {
  static constexpr int kVec = 8, kSize = 2;
};
template <>
struct Elem<kFp32> {
  static constexpr int kVec = 4, kSize = 4;
};

template <int DT>
__device__ inline float load_one(const char *p, int64_t i) {
  if (DT == kBf16) return Bf16::load(p, i);
  if (DT == kFp16) return Fp16::load(p, i);
  return reinterpret_cast<const float *>(p)[i];
}

// 16 bytes of entries at any alignment of an entry
template <int DT>
__device__ inline void load_vec(const char *p, float *x) {
  u32x4 v;
  if (DT == kFp32) {
    typedef float f4u __attribute__((ext_vector_type(4), aligned(4)));
    const f4u f = *reinterpret_cast<const f4u *>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = f[i];
    return;
  }
  typedef uint32_t u4u __attribute__((ext_vector_type(4), aligned(2)));
  const u4u w = *reinterpret_cast<const u4u *>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = w[i];
    x[2 * i] = DT == kBf16 ? Bf16::lo(v[i]) : Fp16::lo(v[i]);
    x[2 * i + 1] = DT == kBf16 ? Bf16::hi(v[i]) : Fp16::hi(v[i]);
  }
}

// entries v * kVec.. of a range [0, n) (past it: `fill`)
template <int DT>
__device__ inline void load_some(const char *p, int64_t v, int64_t n, float fill, float *x) {
  constexpr int kVec = Elem<DT>::kVec;
  if ((v + 1) * kVec <= n) {
    load_vec<DT>(p + v * 16, x);
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i) x[i] = v * kVec + i < n ? load_one<DT>(p, v * kVec + i) : fill;
  }
}

// A row (or a block's range of one) from p on as aligned vectors: entry i is at place i +
// skip, the first vector lacks its first `skip` places. (Vectors across 16-byte boundaries
// cost about a seventh of the rate.)
template <int DT>
struct Aligned {
  const char *p;
  int skip;
  int64_t end;      // places
  __device__ Aligned(const char *row, int64_t n) {
    skip = (int)((uintptr_t)row % 16) / Elem<DT>::kSize;
    p = row - skip * Elem<DT>::kSize;
    end = n + skip;
  }
  __device__ int64_t vectors() const { return (end + Elem<DT>::kVec - 1) / Elem<DT>::kVec; }
  __device__ bool whole(int64_t v) const {
    return v * Elem<DT>::kVec >= skip && (v + 1) * Elem<DT>::kVec <= end;
  }
  __device__ void load(int64_t v, float fill, float *x) const {
    constexpr int kVec = Elem<DT>::kVec;
    if (whole(v)) {
      load_vec<DT>(p + v * 16, x);
    } else {
#pragma unroll
      for (int i = 0; i < kVec; ++i)
        x[i] = v * kVec + i >= skip && v * kVec + i < end ? load_one<DT>(p, v * kVec + i) : fill;
    }
  }
};

// Sort key of an entry: larger for a larger value, then for a lower index; 0 for a NaN.
__device__ inline uint64_t key_of(float x, int64_t index) {
  if (x != x) return 0;
  const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.f);
  const uint32_t o = (b & 0x80000000u) ? ~b : b | 0x80000000u;
  return (uint64_t)o << 32 | (0xffffffffu - (uint32_t)index);
}
__device__ inline float key_value(uint64_t k) {
  const uint32_t o = (uint32_t)(k >> 32);
  return __builtin_bit_cast(float, (o & 0x80000000u) ? o & 0x7fffffffu : ~o);
}
__device__ inline int64_t key_index(uint64_t k) { return 0xffffffffu - (uint32_t)k; }

// Running sums at the maximum m (raw units; kLowest before the first entry). A term's
// exponent is d = fl(x c2 - r), one instruction, with r = fl(m c2) in m c2's place; what r is
// off by is taken out of the sums' logarithm. Where m is so large that this would be many
// units, and in short rows (`exact`, where reading hides the instruction: a row of one entry
// then gives exact zeros), d = (x - m) c2.
struct Sums {
  float m, a, b;
  bool exact = false;
};
__device__ inline bool near_zero(float r) { return __builtin_fabsf(r) <= 1e6f; }
// the reference less m c2
__device__ inline float ref_error(float m, float c2) {
  const float r = m * c2;
  return near_zero(r) ? -__builtin_fmaf(m, c2, -r) : 0.f;
}
__device__ inline void raise(Sums &s, float m, float c2) {
  const float d = fmaxf(__builtin_fmaf(s.m - m, c2, ref_error(s.m, c2) - ref_error(m, c2)),
                        -1e4f);   // (finite: the sums may be 0)
  const float f = fast_exp2(d);
  s.b = (s.b + s.a * d) * f;
  s.a *= f;
  s.m = m;
}
__device__ inline void add(Sums &s, float d) {
  const float e = fast_exp2(d);
  s.a += e;
  s.b = __builtin_fmaf(e, top2(d, -200.f), s.b);   // (a ruled out entry: 0 times -200)
}
template <int M, int N>
__device__ inline void add_all(Sums &s, const float (&x)[M][N], float c2) {
  const float r = s.m * c2;
  if (!s.exact && near_zero(r)) {
#pragma unroll
    for (int i = 0; i < M * N; ++i) add(s, __builtin_fmaf(x[i / N][i % N], c2, -r));
  } else {
#pragma unroll
    for (int i = 0; i < M * N; ++i) add(s, (x[i / N][i % N] - s.m) * c2);
  }
}
__device__ inline Sums joined(Sums x, Sums y, float c2) {
  const float m = fmaxf(x.m, y.m);
  raise(x, m, c2);
  raise(y, m, c2);
  return Sums{m, x.a + y.a, x.b + y.b};
}

__device__ inline uint64_t shfl_xor64(uint64_t v, int o) {
  return (uint64_t)__shfl_xor((uint32_t)(v >> 32), o) << 32 | __shfl_xor((uint32_t)v, o);
}
__device__ inline uint64_t max64(uint64_t a, uint64_t b) { return a > b ? a : b; }

struct RowOut {
  float lse, logp, entropy, log_sum;   // (log_sum: of e^(scale (x - m)))
};
// (rounding aside, neither is below 0; a NaN stays one)
__device__ inline float not_below_0(float x) { return x < 0.f ? 0.f : x; }
// log of the sum of e^(scale (x - m))
__device__ inline float log_sum(const Sums &s, float c2) {
  return not_below_0(s.exact ? logf(s.a) : __builtin_fmaf(kLn2, ref_error(s.m, c2), logf(s.a)));
}
// x_t: the given entry (only read if there is one)
__device__ inline RowOut finish(const Sums &s, float scale, bool has, float xt) {
  RowOut r;
  if (s.a == 0.f) {      // nothing but ruled out entries
    const float inf = __builtin_inff();
    return RowOut{-inf, has ? -inf : 0.f, 0.f, -inf};
  }
  const float c2 = scale * kLog2e, la = log_sum(s, c2);
  r.lse = __builtin_fmaf(scale, s.m, la);
  r.logp = has ? __builtin_fmaf(scale, xt - s.m, -la) : 0.f;
  r.entropy = not_below_0(logf(s.a) - kLn2 * (s.b / s.a));
  r.log_sum = la;
  return r;
}
__device__ inline float alt_logp(const Sums &s, float scale, float x) {
  if (s.a == 0.f) return -__builtin_inff();
  return __builtin_fmaf(scale, x - s.m, -log_sum(s, scale * kLog2e));
}
__device__ inline float alt_logp(const Sums &s, float scale, uint64_t key) {
  return key ? alt_logp(s, scale, key_value(key)) : __builtin_nanf("");
}

// A row's target and its logit, asked for before the sums.
struct Target {
  bool has;
  float x;
};
template <int DT>
__device__ inline Target target_of(const LogprobArgs &a, int64_t row, const char *p) {
  const int64_t t = a.target ? a.target[row] : -1;
  const bool has = t >= 0 && t < a.width;
  return Target{has, has ? load_one<DT>(p, t) : 0.f};
}

__device__ inline void write_row(const LogprobArgs &a, int64_t row, const Sums &s, const Target &t) {
  const RowOut r = finish(s, a.scale, t.has, t.x);
  if (a.logp) a.logp[row] = r.logp;
  if (a.entropy) a.entropy[row] = r.entropy;
  if (a.lse) a.lse[row] = r.lse;
  if (a.norm) {
    a.norm[2 * row] = s.m;
    a.norm[2 * row + 1] = r.log_sum;
  }
}

// ------------------------------------------------------------------ short rows
// One wavefront per row, the row in registers (VL vectors a lane). The alternatives one by
// one: the maximum of the lanes' maxima, the first vector and lane that hold it (so the lowest
// index), which strike the entry out. Bound by reading: 65,536 rows of 512, fp32, 134 MB, 22.1 us,
// 6.1 TB/s; alternatives cost 1.7 us each at 16,384 rows of 500, 1.8 of 2048.
template <int DT, int VL>
__global__ __launch_bounds__(kThreads) void logprob_wave(const LogprobArgs a) {
  constexpr int kVec = Elem<DT>::kVec;
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= a.rows) return;
  const char *p = static_cast<const char *>(a.x) + row * a.row * Elem<DT>::kSize;
  const float c2 = a.scale * kLog2e;
  const Target given = target_of<DT>(a, row, p);
  float x[VL][kVec], top[VL];     // (top: of a vector)
  float m = kLowest;
  auto top_of = [&](const float *y) {
    float t = top3(y[0], y[1], y[2]);
#pragma unroll
    for (int i = 3; i < kVec; i += 2) t = top3(t, y[i], y[i + 1 < kVec ? i + 1 : i]);
    return t;
  };
#pragma unroll
  for (int v = 0; v < VL; ++v) load_some<DT>(p, v * 64 + lane, a.width, -__builtin_inff(), x[v]);
#pragma unroll
  for (int v = 0; v < VL; ++v) {
    top[v] = top_of(x[v]);
    m = top2(m, top[v]);
  }
  Sums s{wave_max(m), 0.f, 0.f, true};
  add_all(s, x, c2);
  s.a = wave_sum(s.a);
  s.b = wave_sum(s.b);
  if (lane == 0) write_row(a, row, s, given);
  bool more = true;
  for (int k0 = 0; k0 < a.top; k0 += 64) {    // lane k of 64 keeps alternative k0 + k
    float value = 0.f;
    int at = -1;
    for (int k = 0; k < min(a.top - k0, 64) && more; ++k) {
      float best = top[0];
#pragma unroll
      for (int v = 1; v < VL; ++v) best = top2(best, top[v]);
      best = wave_max(best);
      more = false;
#pragma unroll
      for (int v = 0; v < VL; ++v) {
        const uint64_t same = more ? 0 : __ballot(top[v] == best);
        if (same) {
          const int owner = __builtin_ctzll(same);
          int i0 = 0;
#pragma unroll
          for (int i = kVec - 1; i >= 0; --i) i0 = x[v][i] == best ? i : i0;
          const int index = (v * 64 + owner) * kVec + __builtin_amdgcn_readlane(i0, owner);
#pragma unroll
          for (int i = 0; i < kVec; ++i)
            if (lane == owner && i == i0) x[v][i] = __builtin_nanf("");
          if (lane == owner) top[v] = top_of(x[v]);
          // (past the row's end there are entries of -inf, after all of its own)
          more = index < a.width;
          if (lane == k && more) {
            value = best;
            at = index;
          }
        }
      }
    }
    if (k0 + lane < a.top) {
      a.top_logp[row * a.top + k0 + lane] = at < 0 ? __builtin_nanf("") : alt_logp(s, a.scale, value);
      a.top_id[row * a.top + k0 + lane] = at;
    }
  }
}

// ------------------------------------------------------------------ alternatives of a block
struct TopShared {
  uint64_t group[kThreads];
  uint64_t list[kList];
  uint64_t best[4];
  int owners[kOwners];
  int n_owners, n_list;
};

// The k-th largest of the block's keys of groups of 256 / G threads (0 if fewer than k);
// nonzero keys are distinct. With 64 groups one wavefront compares them from its registers.
__device__ inline uint64_t bound_from_below(TopShared &sh, uint64_t mine, int k) {
  if (threadIdx.x == 0) {
    sh.n_owners = sh.n_list = 0;
    sh.best[0] = 0;
  }
  if (k <= kSixtyFour) {
    uint64_t g = max64(mine, shfl_xor64(mine, 1));
    g = max64(g, shfl_xor64(g, 2));
    if (threadIdx.x % 4 == 0) sh.group[threadIdx.x / 4] = g;
    __syncthreads();
    if (threadIdx.x < 64) {
      const uint64_t own = sh.group[threadIdx.x];
      const uint32_t lo = (uint32_t)own, hi = (uint32_t)(own >> 32);
      int rank = 0;
#pragma unroll
      for (int i = 0; i < 64; ++i) {
        const uint64_t other = (uint64_t)__builtin_amdgcn_readlane(hi, i) << 32 |
                               (uint32_t)__builtin_amdgcn_readlane(lo, i);
        rank += other > own ? 1 : 0;
      }
      if (own && rank == k - 1) sh.best[0] = own;
    }
  } else {
    sh.group[threadIdx.x] = mine;
    __syncthreads();
    int rank = 0;
#pragma unroll 8
    for (int i = 0; i < kThreads; ++i) rank += sh.group[i] > mine ? 1 : 0;
    if (mine && rank == k - 1) sh.best[0] = mine;
  }
  __syncthreads();
  return sh.best[0];
}

__device__ inline void offer(TopShared &sh, uint64_t key, uint64_t bound) {
  if (key && key >= bound) {
    const int at = atomicAdd(&sh.n_list, 1);
    if (at < kList) sh.list[at] = key;
  }
}

// Calls out(k, key) for the k best of the listed keys, in order (the list's own order, which
// depends on the wavefronts' timing, does not matter).
template <class Out>
__device__ inline void rank_list(TopShared &sh, int n, int k, Out out) {
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const uint64_t own = sh.list[i];
    int rank = 0;
#pragma unroll 4
    for (int j = 0; j < n; ++j) rank += sh.list[j] > own ? 1 : 0;
    if (rank < k) out(rank, own);
  }
  for (int r = n + threadIdx.x; r < k; r += kThreads) out(r, (uint64_t)0);
}

// More entries above the bound than the list holds (possible where many of the best fall on
// few threads): one pass over the entries [0, n) at p per alternative.
template <int DT, class Out>
__device__ inline void by_passes(TopShared &sh, const char *p, int64_t n, int k, Out out) {
  constexpr int kVec = Elem<DT>::kVec;
  const int64_t nv = (n + kVec - 1) / kVec;
  uint64_t last = ~0ull;
  for (int r = 0; r < k; ++r) {
    uint64_t b = 0;
    for (int64_t w = threadIdx.x; w < nv; w += kThreads) {
      float x[kVec];
      load_some<DT>(p, w, n, __builtin_nanf(""), x);
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const uint64_t key = key_of(x[i], w * kVec + i);
        if (key < last) b = max64(b, key);
      }
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) b = max64(b, shfl_xor64(b, o));
    if ((threadIdx.x & 63) == 0) sh.best[threadIdx.x >> 6] = b;
    __syncthreads();
    last = max64(max64(sh.best[0], sh.best[1]), max64(sh.best[2], sh.best[3]));
    __syncthreads();
    if (threadIdx.x == 0) out(r, last);
  }
}

// ------------------------------------------------------------------ long rows
// A block per row. Bound by reading and by the sums' instructions (an exponential, three others and
// the maximum per entry), 70 to 79% of the cycles: 8191 rows of 32,001, bf16, 524 MB, 122 us, 4.3 TB/s;
// 2048 rows of 49,999, fp16, with 5 alternatives, 205 MB, 51 us, 4.0 TB/s.
// A thread's share of a block's range [0, n) at p (index `first` of the row on): its sums, and
// with KEYS the key of its largest entry.
template <int DT, bool KEYS>
__device__ __forceinline__ Sums range_pass(const char *p, int64_t first, int64_t n, float c2,
                                           uint64_t *key) {
  constexpr int kVec = Elem<DT>::kVec, kUnroll = 4;
  const Aligned<DT> row(p, n);
  const int64_t nv = row.vectors();
  const float inf = __builtin_inff();
  Sums s{kLowest, 0.f, 0.f};
  float best = -inf;                    // largest entry of this thread,
  int64_t best_v = threadIdx.x;         // and the first of its vectors that holds it
  auto batch = [&](int64_t v0, auto whole) {
    constexpr bool kWhole = decltype(whole)::value;
    float x[kUnroll][kVec], top[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int64_t v = v0 + u * kThreads;
      if (kWhole) load_vec<DT>(row.p + v * 16, x[u]);
      else row.load(v, -inf, x[u]);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      top[u] = top3(x[u][0], x[u][1], x[u][2]);
#pragma unroll
      for (int i = 3; i < kVec; i += 2) top[u] = top3(top[u], x[u][i], x[u][i + 1 < kVec ? i + 1 : i]);
      if (KEYS) {
        if (top[u] > best) {
          best = top[u];
          best_v = v0 + u * kThreads;
        }
      } else {
        best = top2(best, top[u]);
      }
    }
    raise(s, top2(s.m, best), c2);
    add_all(s, x, c2);
  };
  int64_t v = threadIdx.x;
  if (!row.whole(v) && v < nv) {
    batch(v, std::false_type{});
    v += kUnroll * kThreads;
  }
  for (; row.whole(v + (kUnroll - 1) * kThreads); v += kUnroll * kThreads) batch(v, std::true_type{});
  for (; v < nv; v += kUnroll * kThreads) batch(v, std::false_type{});
  if (KEYS) {
    auto key_at = [&](int64_t w) {
      float x[kVec];
      row.load(w, __builtin_nanf(""), x);
      uint64_t k = 0;
#pragma unroll
      for (int i = 0; i < kVec; ++i) k = max64(k, key_of(x[i], first + w * kVec + i - row.skip));
      return k;
    };
    *key = best_v < nv ? key_at(best_v) : 0;
    // where a vector of NaN came first, and nothing above -inf after it: the first with a number
    if (__builtin_expect(*key == 0, 0))
#pragma unroll 1
      for (int64_t w = best_v + kThreads; w < nv && *key == 0; w += kThreads) *key = key_at(w);
  }
  return s;
}

// The block's sums, the same on every thread.
__device__ inline Sums block_sums(Sums s, float c2, float (*red)[3]) {
  raise(s, wave_max(s.m), c2);
  s.a = wave_sum(s.a);
  s.b = wave_sum(s.b);
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) {
    red[wave][0] = s.m;
    red[wave][1] = s.a;
    red[wave][2] = s.b;
  }
  __syncthreads();
  s = Sums{red[0][0], red[0][1], red[0][2]};
#pragma unroll
  for (int w = 1; w < 4; ++w) s = joined(s, Sums{red[w][0], red[w][1], red[w][2]}, c2);
  return s;
}

template <int DT, bool KEYS>
__global__ __launch_bounds__(kThreads) void logprob_row(const LogprobArgs a) {
  constexpr int kVec = Elem<DT>::kVec, kAhead = 2;
  __shared__ float red[4][3];
  const int64_t row = blockIdx.x;
  const char *p = static_cast<const char *>(a.x) + row * a.row * Elem<DT>::kSize;
  const float c2 = a.scale * kLog2e;
  const Target given = target_of<DT>(a, row, p);
  uint64_t mine = 0;
  const Sums s = block_sums(range_pass<DT, KEYS>(p, 0, a.width, c2, &mine), c2, red);
  if (threadIdx.x == 0) write_row(a, row, s, given);
  if (!KEYS) return;
  __shared__ TopShared sh;
  const uint64_t bound = bound_from_below(sh, mine, a.top);
  if (mine && mine >= bound) sh.owners[atomicAdd(&sh.n_owners, 1)] = threadIdx.x;
  __syncthreads();
  // all of the block look through those threads' vectors
  const Aligned<DT> all(p, a.width);
  const int turns = (int)((all.vectors() + kThreads - 1) / kThreads);
  const int items = sh.n_owners * turns;
  for (int n0 = threadIdx.x; n0 < items; n0 += kAhead * kThreads) {
    float x[kAhead][kVec];
    int64_t w[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int n = n0 + u * kThreads;
      w[u] = n < items ? sh.owners[n / turns] + (int64_t)(n % turns) * kThreads : all.vectors();
      all.load(w[u], __builtin_nanf(""), x[u]);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
#pragma unroll
      for (int i = 0; i < kVec; ++i) offer(sh, key_of(x[u][i], w[u] * kVec + i - all.skip), bound);
  }
  __syncthreads();
  auto out = [&](int r, uint64_t k) {
    a.top_logp[row * a.top + r] = alt_logp(s, a.scale, k);
    a.top_id[row * a.top + r] = k ? key_index(k) : -1;
  };
  const int n = sh.n_list;
  if (n <= kList) rank_list(sh, n, a.top, out);
  else by_passes<DT>(sh, p, a.width, a.top, out);
}

// ------------------------------------------------------------------ rows shared by blocks
struct SplitPlan {
  int parts;       // blocks of a row
  int64_t chunk;   // entries of a block
};
// One block per row where that fills the device, or where the rows are too short to pay for the
// second kernel; fewer parts of more rows save less. Split / not, bf16, 5 alternatives: 1 row of
// 40,000 11.1 / 11.4 us, of 60,000 11.2 / 13.2, of 131,072 11.7 / 17.4; 40 rows of 60,000 13.3 /
// 13.6; 100 of 60,000 14.9 / 13.7, of 80,000 16.3 / 15.8, of 131,072 18.2 / 18.3; 200 of 60,000
// 18.3 / 14.0, of 131,072 23.4 / 24.4; 300 of 20,000 14.5 / 11.9.
constexpr int kSplitWidth = 49152;
SplitPlan split_plan(int32_t rows, int32_t width) {
  SplitPlan p{1, width};
  if (rows >= kSeqCus || width <= kSplitWidth + 256 * (int64_t)rows) return p;
  int64_t parts = (4 * (int64_t)kSeqCus + rows - 1) / rows;
  // A part has at least 4096 entries (2 vectors of 2-byte entries per thread): shorter ones save
  // less than their keys cost the joining block, longer ones leave too few loads in flight. With
  // at least 2048, 4096, 8192: 8 rows of 131,072 bf16, 20 alternatives, 16.0, 14.0, 13.4 us;
  // 3 rows of 11,419, 33 alternatives, 18.0, 16.6, 20.3; 21 rows of 53,830 without, 9.6, 9.7, 9.6.
  const int64_t most = width / 4096;
  if (parts > most) parts = most;
  if (parts < 2) return p;
  p.chunk = ((width + parts - 1) / parts + 63) / 64 * 64;
  p.parts = (int)((width + p.chunk - 1) / p.chunk);
  return p;
}

// Groups of threads that a block leaves the best keys of.
__host__ __device__ inline int key_groups(int top) {
  return top == 0 ? 0 : (top <= kSixtyFour ? 64 : kThreads);
}

// Every block leaves its range's sums and the keys of its groups of threads; a second kernel
// joins them, one block per row. Bound by latency: 8 rows of 131,072, bf16, 20 alternatives,
// 5.0 us and 9.9 for the join, whose choice of the alternatives is a chain of four passes over
// LDS and of two over the candidates' memory.
struct PartSpace {
  uint64_t *keys;    // [rows][parts][groups]
  float *sums;       // [rows][parts][4]
};
__host__ __device__ inline PartSpace part_space(void *ws, int64_t rows, int parts, int top) {
  PartSpace s;
  s.keys = static_cast<uint64_t *>(ws);
  s.sums = reinterpret_cast<float *>(s.keys + rows * parts * key_groups(top));
  return s;
}

template <int DT, bool KEYS>
__global__ __launch_bounds__(kThreads) void logprob_part(const LogprobArgs a, SplitPlan sp,
                                                         void *ws) {
  __shared__ float red[4][3];
  const int64_t row = blockIdx.x / sp.parts;
  const int part = blockIdx.x % sp.parts;
  const PartSpace sc = part_space(ws, a.rows, sp.parts, a.top);
  const char *p = static_cast<const char *>(a.x) + row * a.row * Elem<DT>::kSize;
  const float c2 = a.scale * kLog2e;
  const int64_t lo = part * sp.chunk, hi = lo + sp.chunk < a.width ? lo + sp.chunk : a.width;
  uint64_t mine = 0;
  Sums s = range_pass<DT, KEYS>(p + lo * Elem<DT>::kSize, lo, hi - lo, c2, &mine);
  if (KEYS) {
    if (a.top <= kSixtyFour) {
      mine = max64(mine, shfl_xor64(mine, 1));
      mine = max64(mine, shfl_xor64(mine, 2));
      if (threadIdx.x % 4 == 0) sc.keys[(int64_t)blockIdx.x * 64 + threadIdx.x / 4] = mine;
    } else {
      sc.keys[(int64_t)blockIdx.x * kThreads + threadIdx.x] = mine;
    }
  }
  s = block_sums(s, c2, red);
  if (threadIdx.x == 0)
    *reinterpret_cast<f32x4 *>(sc.sums + 4 * (int64_t)blockIdx.x) = f32x4{s.m, s.a, s.b, 0.f};
}

template <int DT, bool KEYS>
__global__ __launch_bounds__(kThreads) void logprob_join(const LogprobArgs a, SplitPlan sp,
                                                         void *ws) {
  constexpr int kVec = Elem<DT>::kVec;
  __shared__ float red[4][3];
  const int64_t row = blockIdx.x;
  const PartSpace sc = part_space(ws, a.rows, sp.parts, a.top);
  const char *p = static_cast<const char *>(a.x) + row * a.row * Elem<DT>::kSize;
  const float c2 = a.scale * kLog2e;
  const Target given = target_of<DT>(a, row, p);
  uint64_t mine = 0;
  const int groups = key_groups(a.top), n = sp.parts * groups;
  const uint64_t *kr = sc.keys + row * n;
  if (KEYS) {
#pragma unroll 4
    for (int i = threadIdx.x; i < n; i += kThreads) mine = max64(mine, kr[i]);
  }
  Sums s{kLowest, 0.f, 0.f};
  for (int i = threadIdx.x; i < sp.parts; i += kThreads) {
    const f32x4 q = *reinterpret_cast<const f32x4 *>(sc.sums + 4 * (row * sp.parts + i));
    s = joined(s, Sums{q[0], q[1], q[2]}, c2);
  }
  s = block_sums(s, c2, red);
  if (threadIdx.x == 0) write_row(a, row, s, given);
  if (!KEYS) return;
  __shared__ TopShared sh;
  uint64_t bound = bound_from_below(sh, mine, a.top);
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const uint64_t k = kr[i];
    if (k && k >= bound) {
      const int at = atomicAdd(&sh.n_owners, 1);
      if (at < kOwners) sh.owners[at] = i;
    }
  }
  __syncthreads();
  auto out = [&](int r, uint64_t k) {
    a.top_logp[row * a.top + r] = alt_logp(s, a.scale, k);
    a.top_id[row * a.top + r] = k ? key_index(k) : -1;
  };
  int owners = sh.n_owners;
  if (owners <= kOwners) {
    if (owners > 2 * a.top) {
      // Many groups, as where many entries are equal: the k-th of their keys is a bound too, and
      // k groups have keys above it. (A row of 131,072 equal entries without: 720 us, 20 passes.)
      for (int i = threadIdx.x; i < owners; i += kThreads) sh.list[i] = kr[sh.owners[i]];
      __syncthreads();
      int keep[kOwners / kThreads];
#pragma unroll
      for (int u = 0; u < kOwners / kThreads; ++u) {
        const int i = threadIdx.x + u * kThreads;
        keep[u] = -1;
        if (i < owners) {
          const uint64_t own = sh.list[i];
          int rank = 0;
          for (int j = 0; j < owners; ++j) rank += sh.list[j] > own ? 1 : 0;
          if (rank < a.top) keep[u] = sh.owners[i];
          if (rank == a.top - 1) sh.best[1] = own;
        }
      }
      if (threadIdx.x == 0) sh.n_owners = 0;
      __syncthreads();
      bound = sh.best[1];
#pragma unroll
      for (int u = 0; u < kOwners / kThreads; ++u)
        if (keep[u] >= 0) sh.owners[atomicAdd(&sh.n_owners, 1)] = keep[u];
      __syncthreads();
      owners = a.top;
    }
    // `per` vectors side by side every 256 of the group's block
    const int per = kThreads / groups;
    const int turns = (int)((sp.chunk / kVec + 1 + kThreads - 1) / kThreads);
    const int items = owners * turns * per;
    for (int i = threadIdx.x; i < items; i += kThreads) {
      const int g = sh.owners[i / (turns * per)];
      const int64_t from = (g / groups) * sp.chunk;
      const int64_t v = (int64_t)(i / per % turns) * kThreads + g % groups * per + i % per;
      const int64_t len = from + sp.chunk < a.width ? sp.chunk : a.width - from;
      const Aligned<DT> range(p + from * Elem<DT>::kSize, len);
      float x[kVec];
      range.load(v, __builtin_nanf(""), x);
#pragma unroll
      for (int e = 0; e < kVec; ++e) offer(sh, key_of(x[e], from + v * kVec + e - range.skip), bound);
    }
    __syncthreads();
    if (sh.n_list <= kList) {
      rank_list(sh, sh.n_list, a.top, out);
      return;
    }
  }
  __syncthreads();
  by_passes<DT>(sh, p, a.width, a.top, out);
}

// ------------------------------------------------------------------ gradient
// dx_v = c [ g (1[v = t] - p_v) - h p_v (log p_v + H) ]: one pass, each block a range of a
// row (or, for short rows, each wavefront a row). Bound by reading x and writing dx: 65,536 rows of
// 512, fp32, 268 MB, 42.0 us, 6.4 TB/s (part of x still in the caches); 8191 rows of 32,001, bf16,
// 1.05 GB, 201 us, 5.2 TB/s (a copy reaches 5.15).
template <int DT>
__device__ inline void store_vec(char *p, const float *y) {
  if (DT == kFp32) {
    typedef float f4u __attribute__((ext_vector_type(4), aligned(4)));
    *reinterpret_cast<f4u *>(p) = f4u{y[0], y[1], y[2], y[3]};
    return;
  }
  typedef uint32_t u4u __attribute__((ext_vector_type(4), aligned(2)));
  u4u w;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = DT == kBf16 ? Bf16::pack(y[2 * i], y[2 * i + 1]) : Fp16::pack(y[2 * i], y[2 * i + 1]);
  *reinterpret_cast<u4u *>(p) = w;
}
template <int DT>
__device__ inline void store_one(char *p, int64_t i, float y) {
  if (DT == kBf16) Bf16::store(p, i, y);
  else if (DT == kFp16) Fp16::store(p, i, y);
  else reinterpret_cast<float *>(p)[i] = y;
}

template <int DT>
__global__ __launch_bounds__(kThreads) void logprob_grad(const LogprobArgs a, int per_row,
                                                         int threads) {
  constexpr int kVec = Elem<DT>::kVec;
  // `threads` of the block's 256 share a row
  const int64_t unit = (int64_t)blockIdx.x * (kThreads / threads) + threadIdx.x / threads;
  // the last rows first: the caches hold them still from the forward pass
  const int64_t row = a.rows - 1 - unit / per_row;
  if (row < 0) return;
  const int64_t first = unit % per_row * threads + threadIdx.x % threads;
  const int64_t step = (int64_t)per_row * threads;
  const char *p = static_cast<const char *>(a.x) + row * a.row * Elem<DT>::kSize;
  char *q = static_cast<char *>(a.dx) + row * a.dx_row * Elem<DT>::kSize;
  // log p = c x - lse; with the maximum and the log-sum apart c (x - m) - log_sum, whose error does
  // not grow with what the row's logits have in common
  const float m = a.norm ? a.norm[2 * row] : 0.f, lse = a.norm ? a.norm[2 * row + 1] : a.lse[row];
  const bool none = lse == -__builtin_inff();
  const int64_t t = a.target ? a.target[row] : -1;
  const bool has = !none && t >= 0 && t < a.width && a.g_logp;
  const float g = has ? a.g_logp[row] * a.scale : 0.f;
  const float eh = (!none && a.g_entropy) ? a.g_entropy[row] * a.scale : 0.f;
  const float H = (!none && a.g_entropy) ? a.entropy[row] : 0.f;
  const float w = __builtin_fmaf(eh, H, g);
  const Aligned<DT> in(p, a.width);
  q -= in.skip * Elem<DT>::kSize;
  for (int64_t v = first; v < in.vectors(); v += step) {
    float x[kVec];
    in.load(v, -__builtin_inff(), x);
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      const float lp = __builtin_fmaf(x[i] - m, a.scale, -lse);
      const float pr = fast_exp2(lp * kLog2e);
      // -p (g + h (log p + H)), 0 for a ruled out entry
      float y = -pr * __builtin_fmaf(eh, fmaxf(lp, -1e30f), w);
      if (none) y = 0.f;
      if (v * kVec + i - in.skip == t) y += g;
      x[i] = y;
    }
    if (in.whole(v)) {
      store_vec<DT>(q + v * 16, x);
    } else {
#pragma unroll
      for (int i = 0; i < kVec; ++i)
        if (v * kVec + i >= in.skip && v * kVec + i < in.end) store_one<DT>(q, v * kVec + i, x[i]);
    }
  }
}

template <int DT>
hipError_t forward(const LogprobArgs &a, void *ws, hipStream_t s) {
  constexpr int kVec = Elem<DT>::kVec;
  if (a.width <= kWaveWidth) {
    const dim3 grid((uint32_t)((a.rows + 3) / 4));
    const int vl = (a.width + 64 * kVec - 1) / (64 * kVec);
    if (vl <= 1) logprob_wave<DT, 1><<<grid, kThreads, 0, s>>>(a);
    else if (vl <= 2) logprob_wave<DT, 2><<<grid, kThreads, 0, s>>>(a);
    else if (vl <= 4) logprob_wave<DT, 4><<<grid, kThreads, 0, s>>>(a);
    else if (vl <= 8) logprob_wave<DT, 8><<<grid, kThreads, 0, s>>>(a);
    else logprob_wave<DT, kWaveWidth / (64 * kVec)><<<grid, kThreads, 0, s>>>(a);
    return hipGetLastError();
  }
  const SplitPlan sp = split_plan(a.rows, a.width);
  const dim3 grid((uint32_t)((int64_t)a.rows * sp.parts));
  if (sp.parts == 1) {
    if (a.top) logprob_row<DT, true><<<grid, kThreads, 0, s>>>(a);
    else logprob_row<DT, false><<<grid, kThreads, 0, s>>>(a);
  } else {
    const dim3 rows((uint32_t)a.rows);
    if (a.top) {
      logprob_part<DT, true><<<grid, kThreads, 0, s>>>(a, sp, ws);
      logprob_join<DT, true><<<rows, kThreads, 0, s>>>(a, sp, ws);
    } else {
      logprob_part<DT, false><<<grid, kThreads, 0, s>>>(a, sp, ws);
      logprob_join<DT, false><<<rows, kThreads, 0, s>>>(a, sp, ws);
    }
  }
  return hipGetLastError();
}

template <int DT>
hipError_t gradient(const LogprobArgs &a, hipStream_t s) {
  constexpr int kVec = Elem<DT>::kVec;
  const int64_t nv = (a.width + kVec - 1) / kVec;
  // A wavefront per row below 512 vectors, a block per row from there on; more blocks per row (each
  // thread 4 vectors at least) while the rows do not fill the device. 16,384 rows, a wavefront / a
  // block each: 512 bf16 10.4 / 19.3 us, 2048 bf16 23.5 / 30.1, 4096 bf16 46.5 / 44.3, 2048 fp32
  // 45.8 / 42.8. Several blocks / one per row: 8 of 131,072 4.9 / 30, 300 of 65,536 16.4 / 25.3.
  const int threads = nv < 512 ? 64 : kThreads;
  int64_t per_row = 1;
  if (threads == kThreads) {
    const int64_t want = (8 * (int64_t)kSeqCus + a.rows - 1) / a.rows, most = nv / (4 * kThreads);
    per_row = want < most ? want : most;
    if (per_row < 1) per_row = 1;
  }
  const int64_t units = (int64_t)a.rows * per_row, per = kThreads / threads;
  logprob_grad<DT><<<dim3((uint32_t)((units + per - 1) / per)), kThreads, 0, s>>>(a, (int)per_row,
                                                                                  threads);
  return hipGetLastError();
}

}  // namespace

size_t logprob_bytes(int32_t rows, int32_t width, int32_t top) {
  if (width <= kWaveWidth) return 0;
  const SplitPlan sp = split_plan(rows, width);
  if (sp.parts == 1) return 0;
  return (size_t)rows * sp.parts * (key_groups(top) * 8 + 16);
}

// A launch has fewer than 2^32 threads, up to 256 for each row: more rows take several launches.
// (Rows that several blocks share are fewer.)
constexpr int32_t kLaunchRows = 1 << 23;

LogprobArgs rows_from(const LogprobArgs &a, int32_t r) {
  LogprobArgs b = a;
  const int64_t size = a.dtype == kFp32 ? 4 : 2;
  b.rows = a.rows - r < kLaunchRows ? a.rows - r : kLaunchRows;
  b.x = static_cast<const char *>(a.x) + r * a.row * size;
  if (a.target) b.target = a.target + r;
  if (a.logp) b.logp = a.logp + r;
  if (a.entropy) b.entropy = a.entropy + r;
  if (a.lse) b.lse = a.lse + r;
  if (a.norm) b.norm = a.norm + 2 * (int64_t)r;
  if (a.top_logp) b.top_logp = a.top_logp + r * (int64_t)a.top;
  if (a.top_id) b.top_id = a.top_id + r * (int64_t)a.top;
  if (a.g_logp) b.g_logp = a.g_logp + r;
  if (a.g_entropy) b.g_entropy = a.g_entropy + r;
  if (a.dx) b.dx = static_cast<char *>(a.dx) + r * a.dx_row * size;
  return b;
}

hipError_t launch_logprob(const LogprobArgs &a, void *ws, hipStream_t s) {
  hipError_t e = hipSuccess;
  for (int64_t r = 0; r < a.rows && e == hipSuccess; r += kLaunchRows) {
    const LogprobArgs b = rows_from(a, (int32_t)r);
    e = a.dtype == kBf16   ? forward<kBf16>(b, ws, s)
        : a.dtype == kFp16 ? forward<kFp16>(b, ws, s)
                           : forward<kFp32>(b, ws, s);
  }
  return e;
}

hipError_t launch_logprob_grad(const LogprobArgs &a, hipStream_t s) {
  hipError_t e = hipSuccess;
  for (int64_t r = 0; r < a.rows && e == hipSuccess; r += kLaunchRows) {
    const LogprobArgs b = rows_from(a, (int32_t)r);
    e = a.dtype == kBf16   ? gradient<kBf16>(b, s)
        : a.dtype == kFp16 ? gradient<kFp16>(b, s)
                           : gradient<kFp32>(b, s);
  }
  return e;
}

}  // namespace bgp
