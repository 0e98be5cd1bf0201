// What a row of logits says about a token (grpo_top.h): the given token's log-prob, the entropy and the n likeliest
// alternatives, in one pass over the row, and the gradient of all three, in another.
//
// Forward.  Each thread walks its vectors, U of them (a chunk) at a time, and keeps, relative to its running maximum m and in
// units of log 2,
//   s = sum 2^w, t = sum 2^w w, w = (z - m) log2(e) / tau,
// over the words (z > -1e8).  m also bounds the alternatives: the n-th largest of the threads' maxima (of 1,024 threads, of
// four lanes') is a lower bound L of the n-th largest word.  The maximum of each chunk of four neighbouring lanes is kept
// in LDS, and only the chunks whose maximum is >= L, n of them unless words repeat, are read a second time; their words
// >= L (n and a few) go to a list in LDS, and a word's place is the number of list words in front of it.  Where words repeat
// so often that the list or the number of chunks is too small, the n-th largest word is found by bisection with counts over
// the row.  HBM-bound for long rows of which there are many: bf16 [8,000, 151,936] with 8 alternatives 380 us, 6.4 TB/s.
// Where rows are few and long, a row is cut into parts of their own workgroups, and a second launch joins them.
//
// Backward.  A streaming pass: dlogits_v = p_v (A log2 p_v + B) with A, B of the row; the words with a coefficient of their
// own (the action, the alternatives) are formed apart in fp64 and stored over it by the thread that stored their vector.
#include <float.h>
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>

#include "device.h"
#include "grpo_top.h"
#include "host.h"

namespace grpo {

constexpr int kMostGroups = 256;  // chunks of four lanes that are read again
constexpr int kTopCap = 1024;     // words the list holds (a quarter of them for rows of one wave)
constexpr int kShort = 128;       // words that are ranked against one another at once
constexpr uint32_t kNothing = 0;  // the key of no word (a word's is larger)

// A row's part of a workgroup: its sums relative to max, in units of log 2.
struct TopPart {
  double s, t;
  float max;
  float pad;
};

struct TopArgs {
  const void* logits;
  int64_t ld;
  int V, n;
  const float* tau_rows;
  float tau_all;
  const int32_t* actions;
  float* logp;
  float* entropy;
  int32_t* ids;
  float* top_logp;
  grpo_top_row* rows;
  int32_t* flags;
  int parts, part_cols;  // workgroups to a row and their columns
  TopPart* part;         // ws [T][parts]
  uint64_t* part_keys;   // ws [T][parts][n]
};

// Order of words: fp32 values as whole numbers (-0 as 0), the larger the greater; below them the index, the lower the
// greater.  bf16 words' lower 16 bits say nothing, and the first 16 are an order by themselves.
__device__ __forceinline__ uint32_t order_of(float z) {
  const uint32_t b = __float_as_uint(z + 0.f);
  return (b >> 31) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t k) {
  return __uint_as_float((k >> 31) ? k & 0x7fffffffu : ~k);
}
__device__ __forceinline__ uint64_t key_of(float z, int idx) {
  return ((uint64_t)order_of(z) << 32) | (0xffffffffu - (uint32_t)idx);
}
__device__ __forceinline__ bool is_word(float z) { return z > kShiftMin; }

// A thread's sums relative to the shift m sc - rest: w = z sc - m sc + rest.  Near: m sc is small enough that c = -m sc,
// rounded, is a shift to half a unit, rest its rounding, and w one fma, whose error is relative to w; otherwise the
// difference z - m comes first and rest is 0.  A chunk's words are summed in fp32, the chunks in fp64: weights that repeat are
// all rounded the same way (rows of two values, log S with fp32 throughout: off by 3e-6 over 782 words of a thread, by 3e-5
// over 5,860), and two additions to 32 words cost no time that could be measured.
constexpr float kNear = 4194304.f;
__device__ __forceinline__ float rest_of(float m, float sc) {
  const float c = -(m * sc);
  return fabsf(c) < kNear ? fmaf(m, sc, c) : 0.f;
}
struct Sums {
  double s = 0.0, t = 0.0;
  float m = kShiftMin, c = 0.f, rest = 0.f;
  float cs = 0.f, ct = 0.f;  // of the chunk
  bool near = false;

  __device__ __forceinline__ void raise(float mn, float sc) {
    if (mn > m) {
      c = -(mn * sc);
      near = fabsf(c) < kNear;
      const float r = near ? fmaf(mn, sc, c) : 0.f;
      const float dl = fmaf(m - mn, sc, r - rest), f = __builtin_amdgcn_exp2f(dl);
      t = f == 0.f ? 0.0 : (double)f * fma((double)dl, s, t);
      s *= (double)f;
      m = mn;
      rest = r;
    }
  }
  __device__ __forceinline__ void join() {
    s += (double)cs;
    t += (double)ct;
    cs = ct = 0.f;
  }
  // A word at the shift, near and above -1e8; a NaN makes s NaN.
  __device__ __forceinline__ void fold_near(float z, float sc) {
    const float w = fmaf(z, sc, c), e = __builtin_amdgcn_exp2f(w);
    cs += e;
    ct = fmaf(e, w, ct);
  }
  // Any element: a masked word, and one so far below the shift that w may pass fp32's range, adds 2^-200 = 0; a NaN is neither.
  __device__ __forceinline__ void fold(float z, float sc) {
    float w = fmaf(z - m, sc, rest);
    w = z <= kShiftMin || w < -200.f ? -200.f : w;
    const float e = __builtin_amdgcn_exp2f(w);
    cs += e;
    ct = fmaf(e, w, ct);
  }
};

__device__ __forceinline__ float min3f(float a, float b, float c) {  // as max3f (device.h)
  float r;
  asm("v_min3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
template <typename Tin>
__device__ __forceinline__ float vec_min(const u32x4& x, float m) {
  if constexpr (sizeof(Tin) == 2) {
    const float a = min3f(bf16_lo(x[0]), bf16_hi(x[0]), bf16_lo(x[1]));
    const float b = min3f(bf16_hi(x[1]), bf16_lo(x[2]), bf16_hi(x[2]));
    const float c = min3f(bf16_lo(x[3]), bf16_hi(x[3]), m);
    return min3f(a, b, c);
  } else {
    return min3f(min3f(m, __uint_as_float(x[0]), __uint_as_float(x[1])), __uint_as_float(x[2]), __uint_as_float(x[3]));
  }
}

// log2(e) / tau, NaN for a temperature out of range (which then makes the row's sums NaN).
__device__ __forceinline__ float scale_of(float tau) {
  return tau >= 1e-6f && tau <= 1e6f ? kLog2e / tau : NAN;
}

constexpr int kSlices = 32;  // chunks, or runs of chunks, of a lane that have a maximum of their own

// The thread that finishes a row: of the second wave, beside the first one's search for the bound.
template <int NT>
constexpr int kFinisher = NT > 64 ? 64 : 0;

template <int NT>
struct TopSmem {
  float m[NT / 64];
  double s[NT / 64], t[NT / 64];
  double log_sum;
  static constexpr int kTops = NT < 256 ? NT : 256;
  uint16_t top[kTops];                // upper 16 bits of the order of each thread's (1,024 threads: four's) maximum
  uint16_t group[kSlices * NT / 4];   // and of four lanes' chunk
  uint32_t bound;                     // and of L
  int n_groups, count;
  int wave_count[NT / 64];
  uint16_t groups[kMostGroups];
  static constexpr int kCap = NT > 64 ? kTopCap : kTopCap / 4;
  uint64_t list[kCap];
  uint64_t first[kShort];
  int n_first;
};

// All threads' sums joined in fp64, in every thread: S = sum 2^w and T / S at the shift M sc of the row's maximum M.  The sums stay
// at the shift of the thread's, the wave's and the row's maximum until they are joined; then they are divided by the weight
// that the maximum was added with (2^rest, as the hardware rounds it), so that it weighs 1, S is at least 1 and no log-prob is
// above 0.  One thread needs them: `divide`.
template <int NT>
__device__ __forceinline__ void join_threads(const Sums& a, float sc, TopSmem<NT>& sm, bool divide, float& M, double& S,
                                             double& mean) {
  constexpr int NW = NT / 64;
  static_assert(NW <= 16, "one wave to a lane of 16");
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  M = wave_max_dpp(a.m);
  float rest = rest_of(M, sc);
  const float dl = fmaf(a.m - M, sc, rest - a.rest), f = __builtin_amdgcn_exp2f(dl);
  S = wave_sum_dpp((double)f * a.s);
  double T = wave_sum_dpp(f == 0.f ? 0.0 : (double)f * (a.t + (double)dl * a.s));
  if (NW > 1 && lane == 0) {
    sm.m[wv] = M;
    sm.s[wv] = S;
    sm.t[wv] = T;
  }
  __syncthreads();
  if constexpr (NW > 1) {
    const int q = lane & 15;
    const bool in = q < NW;
    const float mq = in ? sm.m[q] : -INFINITY;
    M = row16_max(mq);
    rest = rest_of(M, sc);
    const float dq = in ? fmaf(mq - M, sc, rest - rest_of(mq, sc)) : 0.f, g = in ? __builtin_amdgcn_exp2f(dq) : 0.f;
    S = row16_sum(in ? (double)g * sm.s[q] : 0.0);
    T = row16_sum(g == 0.f ? 0.0 : (double)g * (sm.t[q] + (double)dq * sm.s[q]));
  }
  if (divide) {
    mean = T / S - (double)rest;
    // S / own by its residual, twice: exact where they are equal
    const float own = __builtin_amdgcn_exp2f(rest);
    const double inv = (double)__builtin_amdgcn_rcpf(own);
    double s1 = S * inv;
    s1 = fma(fma(-(double)own, s1, S), inv, s1);
    S = fma(fma(-(double)own, s1, S), inv, s1);
  }
}

// What the row comes to, from the joined sums, and its outputs: one thread.  za: the logit of the action act.
__device__ inline grpo_top_row finish_row(const TopArgs& a, int t, int act, float za, float tau, float M, double S,
                                          double mean) {
  grpo_top_row r;
  const bool act_ok = act >= 0 && act < a.V;
  const bool bad_tau = !(tau >= 1e-6f && tau <= 1e6f), bad = isnan(S) || isnan(M) || M == INFINITY || bad_tau;
  r.temperature = tau;
  int flags = act_ok ? 0 : GRPO_FLAG_ACTION;
  if (bad) {
    r.log_sum = NAN;
    r.max = NAN;
    r.entropy = NAN;
    r.logp = act_ok ? NAN : 0.f;
    flags |= bad_tau ? GRPO_FLAG_SETTING : GRPO_FLAG_NONFINITE;
  } else if (S == 0.0) {
    r.log_sum = -INFINITY;
    r.max = -INFINITY;
    r.entropy = 0.f;
    r.logp = act_ok ? -INFINITY : 0.f;
    flags |= GRPO_FLAG_NONFINITE;
  } else {
    r.log_sum = log(S);
    r.max = M;
    r.entropy = fmaxf((float)(r.log_sum - mean * kLn2), 0.f);  // S >= 1, mean <= 0 but for rounding
    r.logp = !act_ok ? 0.f : is_word(za) ? (float)(((double)za - (double)M) / (double)tau - r.log_sum) : -INFINITY;
  }
  if (flags && a.flags) atomicOr(a.flags, flags);
  if (a.logp) a.logp[t] = r.logp;
  if (a.entropy) a.entropy[t] = r.entropy;
  // Below fp32's range it is -inf, by which the backward call knows a masked word.
  if (act_ok && is_word(za) && !bad) r.logp = fmaxf(r.logp, -FLT_MAX);
  if (a.rows) a.rows[t] = r;
  return r;
}

// Where a list word goes: a final row's outputs, or a part's keys.
struct TopOut {
  int32_t* ids;      // the row's, or NULL
  float* logp;
  uint64_t* keys;    // the part's, or NULL
  double max, tau, log_sum;
  int c0;
  __device__ __forceinline__ void put(int j, uint64_t key) const {
    const uint32_t idx = 0xffffffffu - (uint32_t)key;
    if (keys) {
      keys[j] = key;
      return;
    }
    if (ids) ids[j] = (int)idx;
    if (logp) logp[j] = (float)(((double)value_of((uint32_t)(key >> 32)) - max) / tau - log_sum);
  }
  __device__ __forceinline__ void none(int j, bool bad) const {
    if (keys) keys[j] = kNothing;
    if (ids) ids[j] = -1;
    if (logp) logp[j] = bad ? NAN : -INFINITY;
  }
};

// The n-th largest of 64 `per` 16-bit keys, those of a lane the first `per` in k: one wave.
template <int PER>
__device__ __forceinline__ uint32_t nth_largest(const uint32_t (&k)[PER], int per, int n) {
  uint32_t p = 0;
#pragma unroll 1
  for (int b = 15; b >= 0; --b) {
    const uint32_t c = p | (1u << b);
    int cnt = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (i < per) cnt += __popcll(__ballot(k[i] >= c));
    if (cnt >= n) p = c;
  }
  return p;
}

// The list's first n words in order; the rest of the n places empty.  Every thread of the workgroup.  Of a long list the
// words below the n-th largest (by the upper 16 bits of their order) are left out before they are ranked.
template <int NT, class Smem>
__device__ __forceinline__ void rank_list(Smem& sm, int c, int n, const TopOut& out) {
  const int tid = threadIdx.x;
  const uint64_t* list = sm.list;
  int k = c;
  if (c > kShort) {
    constexpr int PER = Smem::kCap / 64;
    if (tid < 64) {
      uint32_t key[PER];
#pragma unroll
      for (int i = 0; i < PER; ++i) key[i] = tid + 64 * i < c ? (uint32_t)(sm.list[tid + 64 * i] >> 48) : 0u;
      const uint32_t b = nth_largest(key, (c + 63) / 64, n);
      if (tid == 0) {
        sm.bound = b;
        sm.n_first = 0;
      }
    }
    __syncthreads();
    const uint32_t b = sm.bound;
    for (int i = tid; i < c; i += NT) {
      const uint64_t key = sm.list[i];
      if ((uint32_t)(key >> 48) < b) continue;
      const int at = atomicAdd(&sm.n_first, 1);
      if (at < kShort) sm.first[at] = key;
    }
    __syncthreads();
    if (sm.n_first <= kShort) {
      list = sm.first;
      k = sm.n_first;
    }
  }
  for (int i = tid; i < k; i += NT) {
    const uint64_t key = list[i];
    int rank = 0;
    for (int j0 = 0; j0 < k; j0 += 8) {  // eight reads of the LDS at a time
#pragma unroll
      for (int j = 0; j < 8; ++j) rank += j0 + j < k && list[min(j0 + j, k - 1)] > key;
    }
    if (rank < n) out.put(rank, key);
  }
  for (int j = c + tid; j < n; j += NT) out.none(j, false);
}

// The sum of v over the workgroup, in every thread.
template <int NT, class Smem>
__device__ __forceinline__ int block_sum(int v, Smem& sm) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  __syncthreads();  // the last use of wave_count is over
  if ((threadIdx.x & 63) == 0) sm.wave_count[threadIdx.x >> 6] = v;
  __syncthreads();
  int sum = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) sum += sm.wave_count[w];
  return sum;
}

// The n likeliest of a row (or part) with more than n words >= the bound, whatever repeats in it: the n-th largest value by
// bisection between the bound and the maximum, each step a count over the row; then the words above it (fewer than n) and
// the first of those that equal it.
template <typename Tin, int NT>
__device__ __forceinline__ void top_by_counts(const Tin* row, int cols, int n, float M, TopSmem<NT>& sm, const TopOut& out) {
  constexpr int EPV = 16 / (int)sizeof(Tin), SH = sizeof(Tin) == 2 ? 16 : 0;
  typedef typename VecAt<Tin>::type u32x4_any;
  const int tid = threadIdx.x, nvec = cols / EPV, tiles = (nvec + NT - 1) / NT, n_edge = cols - nvec * EPV;
  const float ez = tid < n_edge ? load_elem(row + nvec * EPV + tid) : -INFINITY;
  auto rank_of = [](float z) { return is_word(z) ? order_of(z) >> SH : 0u; };
  uint32_t lo = (sm.bound << 16) >> SH, hi = (order_of(M) >> SH) + 1;  // count(>= lo) >= n > count(>= hi)
  while (hi - lo > 1) {
    const uint32_t mid = lo + (hi - lo) / 2;
    int cnt = rank_of(ez) >= mid;
#pragma unroll 1
    for (int q = 0; q < tiles; ++q) {
      const int vi = q * NT + tid;
      if (vi >= nvec) break;
      const u32x4 x = *reinterpret_cast<const u32x4_any*>(row + (int64_t)vi * EPV);
#pragma unroll
      for (int e = 0; e < EPV; ++e) cnt += rank_of(elem<Tin>(x, e)) >= mid;
    }
    if (block_sum<NT>(cnt, sm) >= n) lo = mid;
    else hi = mid;
  }
  __syncthreads();
  if (tid == 0) sm.count = 0;
  __syncthreads();
  uint64_t* equal = sm.list + GRPO_TOP_MAX;
  int n_equal = 0;  // words that equal lo so far, in index order
  auto take = [&](float z, int idx, int& at) {
    const uint32_t r = rank_of(z);
    if (r > lo) sm.list[atomicAdd(&sm.count, 1)] = key_of(z, out.c0 + idx);
    else if (r == lo) {
      if (at < n) equal[at] = key_of(z, out.c0 + idx);
      ++at;
    }
  };
#pragma unroll 1
  for (int q = 0; q <= tiles; ++q) {  // the last tile: the row's last words
    const int vi = q * NT + tid;
    const bool vec = q < tiles && vi < nvec;
    u32x4 x = {0u, 0u, 0u, 0u};
    if (vec) x = *reinterpret_cast<const u32x4_any*>(row + (int64_t)vi * EPV);
    const bool edge = q == tiles && tid < n_edge;
    int here = 0;
    if (vec) {
#pragma unroll
      for (int e = 0; e < EPV; ++e) here += rank_of(elem<Tin>(x, e)) == lo;
    } else if (edge) {
      here = rank_of(ez) == lo;
    }
    int before = here;  // inclusive prefix over the wave
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(before, o, 64);
      if ((tid & 63) >= o) before += v;
    }
    __syncthreads();
    if ((tid & 63) == 63) sm.wave_count[tid >> 6] = before;
    __syncthreads();
    int at = n_equal + before - here;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
      if (w < (tid >> 6)) at += sm.wave_count[w];
      n_equal += sm.wave_count[w];
    }
    if (vec) {
#pragma unroll
      for (int e = 0; e < EPV; ++e) take(elem<Tin>(x, e), vi * EPV + e, at);
    } else if (edge) {
      take(ez, nvec * EPV + tid, at);
    }
  }
  __syncthreads();
  const int above = sm.count;  // < n
  if (tid < above) {
    const uint64_t key = sm.list[tid];
    int rank = 0;
    for (int j = 0; j < above; ++j) rank += sm.list[j] > key;
    out.put(rank, key);
  }
  if (tid >= above && tid < n) out.put(tid, equal[tid - above]);
}

// One workgroup to a row, or (PART) to a part of it.  Seven waves to a SIMD: left to itself the compiler takes the registers of six
// (20,000 x 1,000 bf16 words with 64 alternatives: 151 us against 132).
template <typename Tin, int NT, bool PART>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(NT == 1024 ? 8 : 7))) void k_top(const TopArgs a,
                                                                                                  int row0) {
  constexpr int EPV = 16 / (int)sizeof(Tin), U = 4, QUADS = NT / 4;
  typedef typename VecAt<Tin>::type u32x4_any;
  __shared__ TopSmem<NT> sm;
  const int tid = threadIdx.x;
  const int t = row0 + (int)(PART ? blockIdx.x / (unsigned)a.parts : blockIdx.x);
  const int part = PART ? (int)(blockIdx.x % (unsigned)a.parts) : 0;
  const int c0 = PART ? part * a.part_cols : 0, cols = PART ? min(a.part_cols, a.V - c0) : a.V;
  const Tin* row = static_cast<const Tin*>(a.logits) + (int64_t)t * a.ld + c0;
  const float tau = a.tau_rows ? a.tau_rows[t] : a.tau_all, sc = scale_of(tau);
  const int n = a.n, nvec = cols / EPV, n_edge = cols - nvec * EPV;
  const int chunks = (nvec + NT * U - 1) / (NT * U), run = max(1, (chunks + kSlices - 1) / kSlices);  // of chunks, a slice
  if (tid == 0) sm.n_groups = sm.count = 0;
  const float ez = tid < n_edge ? load_elem(row + nvec * EPV + tid) : -INFINITY;
  int act = -1;
  float za = -INFINITY;  // the action's logit, for the thread that finishes the row
  if (!PART && tid == kFinisher<NT>) {
    act = a.actions[t];
    if (act >= 0 && act < a.V) za = load_elem(row + act);
  }
  Sums sum;
  sum.raise(ez, sc);
  sum.fold(ez, sc);
  sum.join();
  float gm = -INFINITY;
  for (int q = 0; q < chunks; ++q) {
    const int base = q * NT * U + tid;
    float cm = -INFINITY, cn = INFINITY;
    auto words = [&](const u32x4& x) {
      if (sum.near && cn > kShiftMin) {
#pragma unroll
        for (int e = 0; e < EPV; ++e) sum.fold_near(elem<Tin>(x, e), sc);
      } else {
#pragma unroll
        for (int e = 0; e < EPV; ++e) sum.fold(elem<Tin>(x, e), sc);
      }
    };
    if ((q + 1) * NT * U <= nvec) {
      u32x4 x[U];
#pragma unroll
      for (int u = 0; u < U; ++u)  // non-temporal: 6.4 TB/s of long bf16 rows against 5.6
        x[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_any*>(row + (int64_t)(base + u * NT) * EPV));
#pragma unroll
      for (int u = 0; u < U; ++u) {
        cm = vec_max<Tin>(x[u], cm);
        cn = vec_min<Tin>(x[u], cn);
      }
      sum.raise(cm, sc);
      if (sum.near && cn > kShiftMin) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int e = 0; e < EPV; ++e) sum.fold_near(elem<Tin>(x[u], e), sc);
      } else {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int e = 0; e < EPV; ++e) sum.fold(elem<Tin>(x[u], e), sc);
      }
      sum.join();
    } else {
#pragma unroll 1
      for (int vi = base; vi < nvec; vi += NT) {
        const u32x4 x = *reinterpret_cast<const u32x4_any*>(row + (int64_t)vi * EPV);
        cm = vec_max<Tin>(x, cm);
        cn = vec_min<Tin>(x, cn);
        sum.raise(cm, sc);
        words(x);
        sum.join();
      }
    }
    if (n > 0) {
      cm = fmaxf(cm, dpp_f32v<0xB1>(cm));
      gm = fmaxf(gm, fmaxf(cm, dpp_f32v<0x4E>(cm)));  // of the four lanes
      if ((q + 1) % run == 0 || q + 1 == chunks) {
        if ((tid & 3) == 0) sm.group[q / run * QUADS + (tid >> 2)] = is_word(gm) ? (uint16_t)(order_of(gm) >> 16) : 0;
        gm = -INFINITY;
      }
    }
  }
  constexpr int PER = NT / TopSmem<NT>::kTops;
  static_assert(PER == 1 || PER == 4, "a thread, or four lanes");
  float tm = sum.m;
  if constexpr (PER == 4) {
    tm = fmaxf(tm, dpp_f32v<0xB1>(tm));
    tm = fmaxf(tm, dpp_f32v<0x4E>(tm));
  }
  if (tid % PER == 0) sm.top[tid / PER] = (uint16_t)(order_of(tm) >> 16);
  float M;
  double S, mean = 0.0;
  join_threads<NT>(sum, sc, sm, tid == kFinisher<NT>, M, S, mean);
  const bool bad = isnan(S) || isnan(M) || M == INFINITY || isnan(sc), some = !bad && S > 0.0;
  if (PART) {
    if (tid == kFinisher<NT>)
      a.part[(int64_t)t * a.parts + part] = TopPart{bad ? (double)NAN : S, some ? mean * S : 0.0, some ? M : kShiftMin, 0.f};
  } else if (tid == kFinisher<NT>) {
    const grpo_top_row r = finish_row(a, t, act, za, tau, M, S, mean);
    sm.log_sum = r.log_sum;
  }
  if (n == 0) return;
  if (tid < 64 && some) {
    constexpr int K = TopSmem<NT>::kTops / 64;
    uint32_t k[K];
#pragma unroll
    for (int i = 0; i < K; ++i) k[i] = sm.top[tid + 64 * i];
    const uint32_t p = nth_largest(k, K, n);
    if (tid == 0) sm.bound = p;
  }
  __syncthreads();
  TopOut out;
  const int64_t at = (int64_t)t * n;
  out.ids = !PART && a.ids ? a.ids + at : nullptr;
  out.logp = !PART && a.top_logp ? a.top_logp + at : nullptr;
  out.keys = PART ? a.part_keys + ((int64_t)t * a.parts + part) * n : nullptr;
  out.max = M;
  out.tau = tau;
  out.log_sum = PART ? 0.0 : sm.log_sum;
  out.c0 = c0;
  if (!some) {
    if (tid < n) out.none(tid, bad);
    return;
  }
  const uint32_t bound = sm.bound;
  const float least = value_of(bound << 16);
  auto take = [&](float z, int idx) {
    if (z >= least && is_word(z)) {
      const int i = atomicAdd(&sm.count, 1);
      if (i < sm.kCap) sm.list[i] = key_of(z, c0 + idx);
    }
  };
  if (tid < n_edge) take(ez, nvec * EPV + tid);
  const int slices = (chunks + run - 1) / run;
  for (int i = tid; i < slices * QUADS; i += NT)
    if (sm.group[i] >= bound) {
      const int g = atomicAdd(&sm.n_groups, 1);
      if (g < kMostGroups) sm.groups[g] = (uint16_t)i;
    }
  __syncthreads();
  const int ng = sm.n_groups;
  bool fits = ng <= kMostGroups;
  if (fits) {
    const int per = run * U * 4, items = ng * per;
    for (int i = tid; i < items; i += NT) {
      const int gi = i / per, r = i - gi * per, g = sm.groups[gi];
      const int vi = (g / QUADS * run * U + r / 4) * NT + g % QUADS * 4 + r % 4;
      if (vi >= nvec) continue;
      const u32x4 x = *reinterpret_cast<const u32x4_any*>(row + (int64_t)vi * EPV);
      if (!(vec_max<Tin>(x, -INFINITY) >= least)) continue;
#pragma unroll
      for (int e = 0; e < EPV; ++e) take(elem<Tin>(x, e), vi * EPV + e);
    }
    __syncthreads();
    fits = sm.count <= sm.kCap;
  }
  if (fits) rank_list<NT>(sm, sm.count, n, out);
  else top_by_counts<Tin, NT>(row, cols, n, M, sm, out);
}

// A row's parts joined: one workgroup to a row.
constexpr int kJoinNT = 256;
struct JoinSmem {
  static constexpr int kCap = kTopCap;
  uint64_t list[kCap];
  uint64_t first[kShort];
  double log_sum;
  uint32_t bound;
  int count, n_first;
};
template <typename Tin>
__global__ __launch_bounds__(kJoinNT) void k_top_join(const TopArgs a) {
  constexpr int PER = kTopCap / kJoinNT;
  __shared__ JoinSmem sm;
  __shared__ uint16_t sh_top[kTopCap];
  const int t = blockIdx.x, tid = threadIdx.x, lane = tid & 63, n = a.n, c = a.parts * n;
  const float tau = a.tau_rows ? a.tau_rows[t] : a.tau_all, sc = scale_of(tau);
  const uint64_t* keys = a.part_keys + (int64_t)t * c;
  uint64_t mine[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) mine[i] = tid + kJoinNT * i < c ? keys[tid + kJoinNT * i] : kNothing;
  TopPart p{0.0, 0.0, kShiftMin, 0.f};
  if (lane < a.parts) p = a.part[(int64_t)t * a.parts + lane];
  int act = -1;
  float za = -INFINITY;
  if (tid == 64) {
    act = a.actions[t];
    if (act >= 0 && act < a.V) za = load_elem(static_cast<const Tin*>(a.logits) + (int64_t)t * a.ld + act);
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) sh_top[tid + kJoinNT * i] = (uint16_t)(mine[i] >> 48);
  if (tid == 0) sm.count = 0;
  // every wave for itself
  const float M = wave_max_dpp(p.max);
  const float d = (p.max - M) * sc, f = __builtin_amdgcn_exp2f(d);
  const double S = wave_sum_dpp((double)f * p.s);
  const double Tsum = wave_sum_dpp(f == 0.f ? 0.0 : (double)f * (p.t + (double)d * p.s));
  const bool bad = isnan(S) || isnan(sc), some = !bad && S > 0.0;
  if (tid == 64) sm.log_sum = finish_row(a, t, act, za, tau, M, S, Tsum / S).log_sum;
  if (n == 0) return;
  __syncthreads();
  if (tid < 64 && some) {
    uint32_t k[kTopCap / 64];
#pragma unroll
    for (int i = 0; i < kTopCap / 64; ++i) k[i] = sh_top[tid + 64 * i];
    const uint32_t b = nth_largest(k, (c + 63) / 64, n);
    if (tid == 0) sm.bound = b;
  }
  __syncthreads();
  TopOut out;
  const int64_t at = (int64_t)t * n;
  out.ids = a.ids ? a.ids + at : nullptr;
  out.logp = a.top_logp ? a.top_logp + at : nullptr;
  out.keys = nullptr;
  out.max = M;
  out.tau = tau;
  out.log_sum = sm.log_sum;
  out.c0 = 0;
  if (!some) {
    if (tid < n) out.none(tid, bad);
    return;
  }
  const uint32_t bound = sm.bound;
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (mine[i] != kNothing && (uint32_t)(mine[i] >> 48) >= bound) sm.list[atomicAdd(&sm.count, 1)] = mine[i];
  __syncthreads();
  rank_list<kJoinNT>(sm, sm.count, n, out);
}

// ---- the gradient ---------------------------------------------------------------
struct TopBwdArgs {
  const void* logits;
  void* dlogits;
  int64_t ld;
  int V, blocks;  // blocks of columns to a row
  int n;
  const int32_t* actions;
  const int32_t* ids;
  const grpo_top_row* rows;
  const float* dlogp;
  const float* dent;
  const float* dtop;
};

constexpr int kTopBwdCols = 8192;

// One workgroup to COLS columns of a row.  A word's log2 p is formed from z - max, which keeps the exponent's
// rounding small whatever max and tau are.
template <typename Tin, int NT, int COLS>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(4, 8))) void k_top_bwd(const TopBwdArgs a, int row0) {
  constexpr int EPV = 16 / (int)sizeof(Tin), U = COLS / NT / EPV;
  typedef typename VecAt<Tin>::type u32x4_any;
  __shared__ double sh_sum;
  // this workgroup's words with a coefficient: their columns, gradients and the threads that store their vectors
  __shared__ int sh_col[GRPO_TOP_MAX + 8], sh_owner[GRPO_TOP_MAX + 8];
  __shared__ float sh_d[GRPO_TOP_MAX + 8];
  __shared__ int sh_count;
  const int t = row0 + (int)(blockIdx.x / (unsigned)a.blocks), b = (int)(blockIdx.x % (unsigned)a.blocks);
  const int tid = threadIdx.x, n = a.n;
  const Tin* row = static_cast<const Tin*>(a.logits) + (int64_t)t * a.ld;
  Tin* drow = static_cast<Tin*>(a.dlogits) + (int64_t)t * a.ld;
  const int c0 = b * COLS, c1 = min(c0 + COLS, a.V), edge = a.V / EPV * EPV;
  const int n_edge = b == a.blocks - 1 ? a.V - edge : 0;
  u32x4 x[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int col = c0 + (i * NT + tid) * EPV;
    if (col + EPV <= a.V) x[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_any*>(row + col));
  }
  const float ez = tid < n_edge ? load_elem(row + edge + tid) : 0.f;
  const grpo_top_row r = a.rows[t];
  const bool nan = isnan(r.log_sum), none = r.max == -INFINITY;
  const double g = a.dent ? (double)a.dent[t] : 0.0, inv = 1.0 / (double)r.temperature;
  if (tid < 64) {
    const int act = a.actions[t];
    const bool act_on = a.dlogp && act >= 0 && act < a.V && r.logp > -INFINITY;
    const float d_act = act_on ? a.dlogp[t] : 0.f;
    int id = -1;
    float up = 0.f;
    if (tid < n) {
      id = a.ids[(int64_t)t * n + tid];
      if (id >= 0 && id < a.V) up = a.dtop[(int64_t)t * n + tid];
      else id = -1;
    }
    const double C = wave_sum_dpp((double)up) + (double)d_act;
    // the words with a coefficient of their own in these columns, each once, in fp64
    auto special = [&](int col, double c) {
      if (col < c0 || col >= c1) return;
      const float z = load_elem(row + col);
      double d = 0.0;
      if (is_word(z)) {
        const double lp = ((double)z - (double)r.max) * inv - r.log_sum;
        d = (c - exp(lp) * (C + g * (lp + (double)r.entropy))) * inv;
      }
      const int i = atomicAdd(&sh_count, 1);
      sh_col[i] = col;
      sh_d[i] = (float)d;
      sh_owner[i] = col >= edge ? col - edge : (col - c0) / EPV % NT;
    };
    if (tid == 0) {
      sh_sum = C;
      sh_count = 0;
    }
    if (!nan && !none) {
      double c = (double)up + (act_on && id == act ? (double)d_act : 0.0);
      bool twice = false, again = false;  // a word that is listed more than once; an earlier one of it does it
      for (int j0 = 0; j0 < n; j0 += 8) {
#pragma unroll
        for (int j = 0; j < 8; ++j) twice |= __builtin_amdgcn_readlane(id, j0 + j) == id && j0 + j != tid;
      }
      if (__ballot(twice && id >= 0)) {
        for (int j = 0; j < n; ++j) {
          const bool same = __builtin_amdgcn_readlane(id, j) == id && j != tid;
          c += same ? (double)__builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, up), j)) : 0.0;
          again |= same && j < tid;
        }
      }
      const bool listed = __ballot(id == act) != 0;
      if (id >= 0 && !again) special(id, c);
      if (tid == 0 && act_on && !listed) special(act, (double)d_act);
    }
  }
  __syncthreads();
  auto store = [&](auto value) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int col = c0 + (i * NT + tid) * EPV;
      if (col + EPV <= a.V) {
        u32x4 o;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          if constexpr (sizeof(Tin) == 2) o[q] = pack_bf16(value(bf16_lo(x[i][q])), value(bf16_hi(x[i][q])));
          else o[q] = __float_as_uint(value(__uint_as_float(x[i][q])));
        }
        __builtin_nontemporal_store(o, reinterpret_cast<u32x4_any*>(drow + col));
        asm volatile("s_nop 1" ::: "memory");  // the store has read its data before its registers are reused
      }
    }
    if (tid < n_edge) store_elem(drow + edge + tid, value(ez));
  };
  if (nan || none) {
    const float v = nan ? NAN : 0.f;
    store([&](float) { return v; });
    return;
  }
  // p (A log2 p + B)
  const double C = sh_sum;
  const float sc = kLog2e / r.temperature, l2 = (float)(r.log_sum / kLn2), top = r.max;
  const float A = (float)(-g * kLn2 * inv), B = (float)(-(C + g * (double)r.entropy) * inv);
  store([&](float z) {
    // a masked word's, and any so small that A times it may pass fp32's range, weigh nothing
    const float w = z <= kShiftMin ? -200.f : fmaxf(fmaf(z - top, sc, -l2), -200.f);
    return __builtin_amdgcn_exp2f(w) * fmaf(w, A, B);
  });
  // by the thread that stored the word's place, after that store
  const int count = sh_count;
  for (int i0 = 0; i0 < count; i0 += 8) {
    int mine = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) mine |= (i0 + i < count && sh_owner[i0 + i] == tid) << i;
    for (; mine; mine &= mine - 1) {
      const int i = i0 + __ffs(mine) - 1;
      store_elem(drow + sh_col[i], sh_d[i]);
    }
  }
}

__global__ void k_clear_top_flag(int32_t* f) { *f = 0; }

// ---- host -----------------------------------------------------------------------

static bool bad_top_shape(int64_t T, int64_t V, int64_t ld, int32_t n) {
  return T < 0 || T >= ((int64_t)1 << 31) || V < 1 || V > GRPO_TOP_MAX_V || ld < V || n < 0 || n > GRPO_TOP_MAX;
}

// How many workgroups a row goes to.  Up to 48 rows of more than 16,384 words are cut, each into at most 16 parts; then a row
// has 1,024 threads up to 400 rows (about as many as the chip takes at once), 256 beyond (us, the call with 8 alternatives
// of 151,936 bf16 words, which the caches do not hold: T = 1 cut in 4, 8, 16, 32, 64: 22.0, 20.3, 18.2, 17.5, 16.0, whole with
// 1,024 threads 21.7, with 256 31.7; T = 16: 22.3, 19.4, 17.6, 18.4, 18.7, 22.2, 32.2; T = 64: 23.8, 21.1, 21.2, 24.7, 29.5,
// 22.8, 31.8; T = 256 whole 27.9 and 34.2, T = 512 48.3 and 39.3, T = 1,024 82.6 and 60.4).
constexpr int64_t kFewTopRows = 48, kSomeTopRows = 400;
// Short rows of which there are many go to one wave each (us, one wave and 256 threads, bf16: V = 1,000 T = 1,024 without
// alternatives 7.5 and 7.2, with 8 11.2 and 10.5, T = 4,096 9.5 and 13.1, 14 and 21, T = 20,000 23 and 42, 38 and 77, with 33
// 55 and 99; the gradient at T = 20,000 22 and 37, 31 and 60, with 64 49 and 110), but for more than 48 alternatives, which
// the 64 lanes' maxima bound badly (with 64 at V = 4,000 T = 20,000 294 and 157).
constexpr int64_t kOneWaveTopBytes = 8192, kManyTopRows = 2048;
struct TopPlan {
  int parts, cols;
};
static TopPlan top_plan(int64_t T, int64_t V, int32_t n) {
  TopPlan p{1, (int)V};
  if (T <= 0 || T > kFewTopRows || V <= 16384) return p;
  const int64_t parts = std::min<int64_t>({V / 8192, (int64_t)16, n ? (int64_t)(kTopCap / n) : (int64_t)16});
  if (parts < 2) return p;
  p.cols = (int)(((V + parts - 1) / parts + 7) / 8 * 8);
  p.parts = (int)((V + p.cols - 1) / p.cols);
  return p;
}

static size_t top_part_bytes(int64_t T, const TopPlan& p) { return align_up(sizeof(TopPart) * (size_t)T * p.parts); }

constexpr int64_t kTopRowsPerLaunch = 1 << 20;  // a launch's threads stay below 2^32

template <typename Tin, int NT>
static void launch_top_rows(const TopArgs& a, int64_t T, hipStream_t s) {
  for (int64_t r = 0; r < T; r += kTopRowsPerLaunch)
    hipLaunchKernelGGL((k_top<Tin, NT, false>), dim3((unsigned)std::min(kTopRowsPerLaunch, T - r)), dim3(NT), 0, s, a,
                       (int)r);
}

template <typename Tin>
static void launch_top(const TopArgs& a, int64_t T, hipStream_t s) {
  if (a.parts > 1) {
    hipLaunchKernelGGL((k_top<Tin, 256, true>), dim3((unsigned)(T * a.parts)), dim3(256), 0, s, a, 0);
    hipLaunchKernelGGL(k_top_join<Tin>, dim3((unsigned)T), dim3(kJoinNT), 0, s, a);
    return;
  }
  if (a.V * (int64_t)sizeof(Tin) <= kOneWaveTopBytes && T >= kManyTopRows && a.n <= 48) launch_top_rows<Tin, 64>(a, T, s);
  else if (T > kSomeTopRows || a.V <= 16384) launch_top_rows<Tin, 256>(a, T, s);
  else launch_top_rows<Tin, 1024>(a, T, s);
}

}  // namespace grpo

using namespace grpo;

extern "C" size_t grpo_token_logp_top_workspace_bytes(int64_t T, int64_t V, int32_t n) {
  if (bad_top_shape(T, V, V, n)) return 0;
  const TopPlan p = top_plan(T, V, n);
  return p.parts == 1 ? 0 : top_part_bytes(T, p) + align_up(sizeof(uint64_t) * (size_t)T * p.parts * n);
}

extern "C" int grpo_token_logp_top(const void* logits, int32_t dtype, int64_t T, int64_t V, int64_t ld,
                                   const float* temperature, float temperature_all, const int32_t* actions, int32_t n,
                                   float* logp, float* entropy, int32_t* top_ids, float* top_logp, grpo_top_row* rows,
                                   int32_t* error_flags, void* ws, size_t ws_bytes, hipStream_t s) {
  if (bad_top_shape(T, V, ld, n)) return GRPO_ERR_SHAPE;
  if (T > 0 && (!logits || !actions)) return GRPO_ERR_ARG;
  if (!temperature && !(temperature_all >= 1e-6f && temperature_all <= 1e6f)) return GRPO_ERR_ARG;
  if (dtype != GRPO_F32 && dtype != GRPO_BF16) return GRPO_ERR_DTYPE;
  if (!aligned(logits, dtype == GRPO_BF16 ? 2 : 4) || !aligned(temperature, 4) || !aligned(actions, 4) ||
      !aligned(logp, 4) || !aligned(entropy, 4) || !aligned(top_ids, 4) || !aligned(top_logp, 4) || !aligned(rows, 8) ||
      !aligned(error_flags, 4))
    return GRPO_ERR_ALIGN;
  const TopPlan p = top_plan(T, V, n);
  if (p.parts > 1) {
    if (!ws || ws_bytes < grpo_token_logp_top_workspace_bytes(T, V, n)) return GRPO_ERR_WORKSPACE;
    if (!aligned(ws, 16)) return GRPO_ERR_ALIGN;
  }
  if (error_flags) hipLaunchKernelGGL(k_clear_top_flag, dim3(1), dim3(1), 0, s, error_flags);
  if (T > 0) {
    TopArgs a{logits, ld, (int)V, n, temperature, temperature_all, actions, logp, entropy, top_ids, top_logp, rows,
              error_flags, p.parts, p.cols, nullptr, nullptr};
    if (!top_ids && !top_logp) a.n = 0;
    if (p.parts > 1) {
      a.part = static_cast<TopPart*>(ws);
      a.part_keys = reinterpret_cast<uint64_t*>(static_cast<char*>(ws) + top_part_bytes(T, p));
    }
    if (dtype == GRPO_BF16) launch_top<uint16_t>(a, T, s);
    else launch_top<float>(a, T, s);
  }
  return hipGetLastError() == hipSuccess ? GRPO_OK : GRPO_ERR_HIP;
}

extern "C" int grpo_token_logp_top_bwd(const void* logits, int32_t dtype, int64_t T, int64_t V, int64_t ld,
                                       const int32_t* actions, int32_t n, const int32_t* top_ids,
                                       const grpo_top_row* rows, const float* dlogp, const float* dentropy,
                                       const float* dtop, void* dlogits, hipStream_t s) {
  if (bad_top_shape(T, V, ld, n)) return GRPO_ERR_SHAPE;
  if (T > 0 && (!logits || !actions || !rows || !dlogits || (dtop && n > 0 && !top_ids))) return GRPO_ERR_ARG;
  if (dtype != GRPO_F32 && dtype != GRPO_BF16) return GRPO_ERR_DTYPE;
  const size_t esz = dtype == GRPO_BF16 ? 2 : 4;
  if (!aligned(logits, esz) || !aligned(dlogits, esz) || !aligned(actions, 4) || !aligned(top_ids, 4) ||
      !aligned(rows, 8) || !aligned(dlogp, 4) || !aligned(dentropy, 4) || !aligned(dtop, 4))
    return GRPO_ERR_ALIGN;
  if (T > 0 && rows_overlap(logits, dlogits, T, V, ld, esz)) return GRPO_ERR_ARG;
  // Rows of one wave's reach go to one wave each.
  const bool one_wave = V * (int64_t)esz <= kOneWaveTopBytes && T >= kManyTopRows;
  const int blocks = one_wave ? 1 : (int)((V + kTopBwdCols - 1) / kTopBwdCols);
  const int64_t per = std::max<int64_t>(1, ((int64_t)1 << 23) / blocks);  // a launch's threads stay below 2^32
  for (int64_t r = 0; r < T; r += per) {
    const TopBwdArgs a{logits, dlogits, ld, (int)V, blocks, dtop ? n : 0, actions, top_ids, rows, dlogp, dentropy, dtop};
    const unsigned grid = (unsigned)(std::min(per, T - r) * blocks);
    auto go = [&](auto kernel, int nt) { hipLaunchKernelGGL(kernel, dim3(grid), dim3((unsigned)nt), 0, s, a, (int)r); };
    if (dtype == GRPO_BF16) {
      if (one_wave) go(k_top_bwd<uint16_t, 64, 4096>, 64);
      else go(k_top_bwd<uint16_t, 256, kTopBwdCols>, 256);
    } else {
      if (one_wave) go(k_top_bwd<float, 64, 2048>, 64);
      else go(k_top_bwd<float, 256, kTopBwdCols>, 256);
    }
  }
  return hipGetLastError() == hipSuccess ? GRPO_OK : GRPO_ERR_HIP;
}
