// The policy as a rollout samples from it (grpo_sampling.h): per row, the words that temperature, top-k, top-p and min-p
// keep, an action drawn from them or the log-prob of a given one, and that log-prob's gradient.
//
// The kept words are a prefix of the row in the order (logit descending, index ascending), so a row's cut is a threshold
// and, among the words that equal it, a last index.  With w = exp((z - max z) / tau), S its sum:
//   top-k  the prefix of k words: a count;
//   top-p  the shortest prefix of weight >= p S: a weight;
//   min-p  z >= max z + tau log(min_p): a threshold at once.
// Counts are exact; weights and their sums are fp64 (exp2_neg below), because with 150,000 words of about equal weight a
// word's share is 7e-6 of the sum, and an error of 1e-8 in the sums would draw another word in one row of a thousand.
//
// A row is cut into tiles of kTile words, each reduced in a wave's registers to its maximum, its count of live words and
// its sum of weights relative to its own maximum: one pass over memory, of any number of waves per row.  Then one
// workgroup per row works on the tiles' records and re-reads only the tiles that it needs:
//   nothing cut     a draw picks its tile by the tiles' sums and re-reads that one;
//   few candidates  a lower bound of the threshold (the k-th largest of the partial maxima; for top-p, the weight below
//                   which all live words together weigh less than (1 - p) S; min-p's own) leaves at most kCap words:
//                   they are gathered in LDS, sorted, and the cut read off their prefix sums;
//   many            histograms: words fall into kBins bins of a quarter of a power of two of weight, each bin's count
//                   and weight are summed, the bin that holds the cut is split again by the bits of its logits until at
//                   most kCap words (gathered and sorted) or one repeated value are left.
// Histogram weights are integers (weight relative to the bin's top, in 2^-44), so that atomics in any order give one sum.
#include <hip/hip_runtime.h>
#include <float.h>
#include <math.h>

#include <algorithm>

#include "device.h"
#include "grpo_sampling.h"
#include "host.h"

namespace grpo {

constexpr int kTile = 2048;        // words of a tile: 32 per lane
constexpr int kMaxTiles = GRPO_SAMPLING_MAX_V / kTile;
constexpr int kSubs = 8;           // partial maxima of a tile, each over 8 lanes' words
constexpr int kMaxSubs = 1024;     // partial maxima (or tiles' maxima) that bound the k-th largest word
constexpr int kCap = 2048;         // words that are sorted in LDS
constexpr int kBins = 128, kCols = 32;
constexpr int kNT = 512, kNW = kNT / 64;
constexpr float kLiveMin = -99999992.f;  // the smallest float above -1e8: the lowest live logit
constexpr double kLog2e64 = 1.4426950408889634074;

struct TileRec {
  double sum;
  float sub[kSubs];
  int32_t live;
  int32_t bad;
};

struct RowArgs {
  const void* logits;
  int64_t ld;
  int V, tiles;
  grpo_sampling par;
  const float* u;          // draws
  const int32_t* actions;  // given actions
  int32_t* actions_out;
  float* logp;             // nullable
  int32_t* n_kept;         // nullable
  grpo_sampling_row* rows; // nullable
  int32_t* flags;          // nullable
  TileRec* recs;           // [T][tiles] where the tiles are reduced by a launch of their own
};

// ---- numbers -------------------------------------------------------------------

// 2^t for t <= 0, relative error below 1e-15 (0 for t < -1021; exactly 1 at 0): 2^n by the exponent bits, 2^f for
// |f| <= 1/2 by its Chebyshev interpolant (f times a polynomial of degree 9, plus 1).
template <bool FAR = true>
__device__ __forceinline__ double exp2_neg(double t) {
  constexpr double kRound = 6755399441055744.0;  // 1.5 2^52: adding it leaves rint(t) in the low bits
  const double y = t + kRound;
  const double f = t - (y - kRound);
  double p = 7.070976083807186e-09;
  p = fma(p, f, 1.0205905476607851e-07);
  p = fma(p, f, 1.3215451644483806e-06);
  p = fma(p, f, 1.525267292453816e-05);
  p = fma(p, f, 0.00015403530424751012);
  p = fma(p, f, 0.0013333558200795041);
  p = fma(p, f, 0.00961812910761869);
  p = fma(p, f, 0.05550410866465167);
  p = fma(p, f, 0.24022650695910075);
  p = fma(p, f, 0.6931471805599462);
  p = fma(p, f, 1.0);
  const uint64_t n = __builtin_bit_cast(uint64_t, y) << 52;
  const double r = __builtin_bit_cast(double, __builtin_bit_cast(uint64_t, p) + n);
  return FAR && !(t >= -1021.0) ? 0.0 : r;
}

// Unsigned integers in the order of the floats (-0 counts as 0), and back.
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float((k & 0x80000000u) ? k ^ 0x80000000u : ~k);
}

__device__ __forceinline__ float min3f(float a, float b, float c) {
  float r;
  asm("v_min3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

__device__ __forceinline__ double scan_add(double v) {  // inclusive, over the wave
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double n = __shfl_up(v, o, 64);
    if (lane >= o) v += n;
  }
  return v;
}
__device__ __forceinline__ int scan_add(int v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int n = __shfl_up(v, o, 64);
    if (lane >= o) v += n;
  }
  return v;
}

// ---- a row's settings -----------------------------------------------------------
struct Settings {
  float tau, p, min_p;
  int k;
  double c;  // log2(e) / tau
  bool ok, greedy;
};

__device__ __forceinline__ Settings load_settings(const grpo_sampling& g, int t) {
  Settings s;
  s.tau = g.temperature ? g.temperature[t] : g.temperature_all;
  s.k = g.top_k ? g.top_k[t] : g.top_k_all;
  s.p = g.top_p ? g.top_p[t] : g.top_p_all;
  s.min_p = g.min_p ? g.min_p[t] : g.min_p_all;
  s.greedy = s.tau == 0.f;
  s.ok = (s.greedy || (s.tau >= 1e-6f && s.tau <= 1e6f)) && s.p >= 0.f && s.p <= 1.f && s.min_p >= 0.f && s.min_p <= 1.f;
  s.c = s.ok && !s.greedy ? kLog2e64 / (double)s.tau : 1.0;
  return s;
}

// What a tile's sum of weights is for: nothing, a cut or a draw (fp64), or a log-prob alone (fp32 terms, like the other
// log-probs of this library).
enum SumMode { kNoSum, kSum64, kSum32 };
__device__ __forceinline__ SumMode sum_mode(const Settings& s, int V, bool draw) {
  if (!s.ok || s.greedy || (s.k > 0 && s.k < V)) return kNoSum;
  if (s.p < 1.f) return kSum64;
  if (s.min_p > 0.f) return kNoSum;
  return draw ? kSum64 : kSum32;
}

// ---- tiles ----------------------------------------------------------------------
// Vector j of lane l holds the tile's words (64 j + l) EPV ..., as element e of 16 bytes; the hardware takes vector loads
// at any alignment, so a row may start at any element.  Words past the row's end read as -inf.
template <typename Tin>
struct Tile {
  static constexpr int EPV = 16 / (int)sizeof(Tin), NV = kTile / 64 / EPV;
  u32x4 v[NV];

  __device__ __forceinline__ static int col(int tile, int j, int e) {
    return tile * kTile + (j * 64 + (threadIdx.x & 63)) * EPV + e;
  }
  // Vector j of a tile that the row's end may cut.
  __device__ __forceinline__ static u32x4 load_one(const Tin* row, int V, int tile, int j) {
    typedef typename VecAt<Tin>::type u32x4_any;
    const int c0 = col(tile, j, 0);
    if (c0 + EPV <= V) return *reinterpret_cast<const u32x4_any*>(row + c0);
    u32x4 r;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if constexpr (sizeof(Tin) == 2) {
        const uint32_t lo = c0 + 2 * q < V ? row[c0 + 2 * q] : 0xff80u;
        const uint32_t hi = c0 + 2 * q + 1 < V ? row[c0 + 2 * q + 1] : 0xff80u;
        r[q] = lo | (hi << 16);
      } else {
        r[q] = c0 + q < V ? __float_as_uint(row[c0 + q]) : 0xff800000u;
      }
    }
    return r;
  }
  __device__ __forceinline__ void load(const Tin* row, int V, int tile) {
    typedef typename VecAt<Tin>::type u32x4_any;
    if ((tile + 1) * kTile <= V) {
#pragma unroll
      for (int j = 0; j < NV; ++j) v[j] = *reinterpret_cast<const u32x4_any*>(row + col(tile, j, 0));
    } else {
#pragma unroll 1
      for (int j = 0; j < NV; ++j) {
        const u32x4 r = load_one(row, V, tile, j);
#pragma unroll
        for (int i = 0; i < NV; ++i)
          if (i == j) v[i] = r;
      }
    }
  }
  __device__ __forceinline__ float at(int j, int e) const { return elem<Tin>(v[j], e); }
};

struct TileStats {
  double sum;   // of weights relative to max; every lane
  float sub;    // the maximum over this lane's group of 8 lanes
  float max;    // every lane
  int live;     // every lane
  bool bad;     // a NaN or +inf; every lane
};

template <typename Tin>
__device__ __forceinline__ TileStats tile_stats(const Tile<Tin>& x, SumMode mode, double c) {
  constexpr int NV = Tile<Tin>::NV, EPV = Tile<Tin>::EPV;
  TileStats s;
  float mx = -INFINITY, mn = INFINITY;
  bool nan = false;
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int e = 0; e < EPV; e += 2) {
      const float p = x.at(j, e), q = x.at(j, e + 1);
      nan |= __builtin_isunordered(p, q);
      mx = max3f(mx, p, q);
      mn = min3f(mn, p, q);
    }
  float g = fmaxf(mx, dpp_f32v<0xB1>(mx));
  g = fmaxf(g, dpp_f32v<0x4E>(g));
  s.sub = fmaxf(g, dpp_f32v<0x141>(g));
  s.max = wave_max_dpp(mx);
  const float lo = -wave_max_dpp(-mn);
  s.bad = __any(nan) || s.max == INFINITY;
  s.sum = 0.0;
  s.live = kTile;
  const bool all_live = lo >= kLiveMin;
  if (!all_live) {
    s.live = 0;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < EPV; ++e) s.live += __popcll(__ballot(x.at(j, e) >= kLiveMin));
  }
  if (mode == kNoSum || s.bad || s.live == 0) return s;
  if (mode == kSum64) {
    const double m = (double)s.max;
    double sum = 0.0;
    if (all_live && (m - (double)lo) * c < 1000.0) {
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < EPV; ++e) sum += exp2_neg<false>(((double)x.at(j, e) - m) * c);
    } else {
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < EPV; ++e) {
          const float z = x.at(j, e);
          sum += z >= kLiveMin ? exp2_neg(((double)z - m) * c) : 0.0;
        }
    }
    s.sum = wave_sum_dpp(sum);
  } else {
    const float c32 = (float)c;
    float sum = 0.f;
    if (all_live) {
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < EPV; ++e) sum += __builtin_amdgcn_exp2f((x.at(j, e) - s.max) * c32);
    } else {
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < EPV; ++e) {
          const float z = x.at(j, e);
          sum += z >= kLiveMin ? __builtin_amdgcn_exp2f((z - s.max) * c32) : 0.f;
        }
    }
    s.sum = wave_sum_dpp((double)sum);
  }
  return s;
}

// The tiles of few rows, one wave each, spread over the whole chip.
template <typename Tin>
__global__ __launch_bounds__(256) void k_sample_tiles(const RowArgs a, int n_waves, bool draw) {
  const int w = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (w >= n_waves) return;
  const int t = w / a.tiles, tile = w - t * a.tiles;
  const Settings st = load_settings(a.par, t);
  Tile<Tin> x;
  x.load(static_cast<const Tin*>(a.logits) + (int64_t)t * a.ld, a.V, tile);
  const TileStats s = tile_stats<Tin>(x, sum_mode(st, a.V, draw), st.c);
  TileRec* r = a.recs + w;
  if ((lane & 7) == 0) r->sub[lane >> 3] = s.sub;
  if (lane == 0) {
    r->sum = s.sum;
    r->live = s.live;
    r->bad = s.bad;
  }
}

// ---- one row --------------------------------------------------------------------
struct Cut {
  float thr;    // kept: z > thr, or z == thr and index <= tie
  int tie;
  double mass;  // weight of the prefix that ends there
};

struct RowShared {
  union {
    struct {
      unsigned long long mass[kBins * kCols];
      uint32_t count[kBins * kCols];
    } h;
    struct {
      unsigned long long key[kCap];
      double cum[kCap];
    } l;
    int tcount[kMaxTiles];
  };
  double tsum[kMaxTiles];
  float tmax[kMaxTiles];
  float sub[kMaxSubs];
  double bin_mass[2][kBins];
  int bin_count[2][kBins];
  double wd[kNW];
  int wi[kNW];
  // broadcast
  int n, bin, i0;
  uint32_t key;
  double d0;
};

// Workgroup reductions, the same value in every thread; `sh.w*` may be reused after them.
__device__ __forceinline__ double block_sum(RowShared& sh, double v) {
  v = wave_sum_dpp(v);
  if ((threadIdx.x & 63) == 0) sh.wd[threadIdx.x >> 6] = v;
  __syncthreads();
  double r = 0.0;
#pragma unroll
  for (int i = 0; i < kNW; ++i) r += sh.wd[i];
  __syncthreads();
  return r;
}
template <typename F>
__device__ __forceinline__ int block_reduce_int(RowShared& sh, int v, F f) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = f(v, __shfl_xor(v, o, 64));
  if ((threadIdx.x & 63) == 0) sh.wi[threadIdx.x >> 6] = v;
  __syncthreads();
  int r = sh.wi[0];
#pragma unroll
  for (int i = 1; i < kNW; ++i) r = f(r, sh.wi[i]);
  __syncthreads();
  return r;
}
__device__ __forceinline__ int block_sum_int(RowShared& sh, int v) {
  return block_reduce_int(sh, v, [](int a, int b) { return a + b; });
}
__device__ __forceinline__ int block_min_int(RowShared& sh, int v) {
  return block_reduce_int(sh, v, [](int a, int b) { return min(a, b); });
}
__device__ __forceinline__ int block_max_int(RowShared& sh, int v) {
  return block_reduce_int(sh, v, [](int a, int b) { return max(a, b); });
}
// Inclusive scan over the workgroup's threads; total in every thread.
__device__ __forceinline__ double block_scan(RowShared& sh, double v, double& total) {
  const int wv = threadIdx.x >> 6;
  v = scan_add(v);
  if ((threadIdx.x & 63) == 63) sh.wd[wv] = v;
  __syncthreads();
  double before = 0.0, all = 0.0;
#pragma unroll
  for (int i = 0; i < kNW; ++i) {
    if (i < wv) before += sh.wd[i];
    all += sh.wd[i];
  }
  __syncthreads();
  total = all;
  return before + v;
}

// Sorts the n keys in sh.l.key, largest first, padded with zeros to a power of two.
__device__ __forceinline__ void sort_list(RowShared& sh, int n) {
  const int tid = threadIdx.x;
  int P = 2;
  while (P < n) P <<= 1;
  for (int i = n + tid; i < P; i += kNT) sh.l.key[i] = 0ull;
  __syncthreads();
  for (int k = 2; k <= P; k <<= 1) {
    for (int j = k >> 1; j > 0; j >>= 1) {
      for (int q = tid; q < (P >> 1); q += kNT) {
        const int i = ((q & ~(j - 1)) << 1) | (q & (j - 1));
        const unsigned long long x = sh.l.key[i], y = sh.l.key[i | j];
        if ((x < y) == ((i & k) == 0)) {
          sh.l.key[i] = y;
          sh.l.key[i | j] = x;
        }
      }
      __syncthreads();
    }
  }
}

template <typename Tin>
struct RowWork {
  RowShared& sh;
  const Tin* row;
  int V, tiles;
  float m;   // the row's maximum
  double c;  // log2(e) / tau
  float x_lo;  // words below it are not looked at

  // f(vector, j) over a tile's vectors, the next one's load in flight: for the passes whose work per word is long.
  template <typename F>
  __device__ __forceinline__ void each_vector(int tile, F f) const {
    u32x4 x = Tile<Tin>::load_one(row, V, tile, 0);
#pragma unroll 1
    for (int j = 0; j < Tile<Tin>::NV; ++j) {
      const u32x4 next = Tile<Tin>::load_one(row, V, tile, min(j + 1, Tile<Tin>::NV - 1));
      f(x, j);
      x = next;
    }
  }

  __device__ __forceinline__ double t2(float z) const { return ((double)z - (double)m) * c; }
  __device__ __forceinline__ double weight(float z) const { return exp2_neg(t2(z)); }

  // The words of [lo, hi] appended to the list while it has room; returns how many there are, or more than kCap.
  __device__ __forceinline__ int gather(float lo, float hi) {
    const int tid = threadIdx.x, lane = tid & 63;
    if (tid == 0) sh.n = 0;
    __syncthreads();
    for (int tile = tid >> 6; tile < tiles; tile += kNW) {
      if (sh.tmax[tile] < lo) continue;
      if (__builtin_amdgcn_readfirstlane(*(volatile int*)&sh.n) > kCap) break;
      Tile<Tin> x;
      x.load(row, V, tile);
#pragma unroll
      for (int j = 0; j < Tile<Tin>::NV; ++j) {
        if (!__any(vec_max<Tin>(x.v[j], -INFINITY) >= lo)) continue;
#pragma unroll
        for (int e = 0; e < Tile<Tin>::EPV; ++e) {
          const float z = x.at(j, e);
          const bool in = z >= lo && z <= hi;
          const uint64_t mask = __ballot(in);
          if (mask) {
            int at = 0;
            if (lane == 0) at = atomicAdd(&sh.n, __popcll(mask));
            at = __builtin_amdgcn_readfirstlane(at) + (int)__popcll(mask & ((1ull << lane) - 1));
            if (in && at < kCap)
              sh.l.key[at] = ((unsigned long long)order_key(z) << 32) | (uint32_t)~x.col(tile, j, e);
          }
        }
      }
    }
    __syncthreads();
    const int n = sh.n;
    __syncthreads();
    return n;
  }

  __device__ __forceinline__ float list_value(int i) const { return key_value((uint32_t)(sh.l.key[i] >> 32)); }
  __device__ __forceinline__ int list_index(int i) const { return (int)~(uint32_t)sh.l.key[i]; }

  // sh.l.cum = the prefix sums of the list's weights, from `base` on.
  __device__ __forceinline__ void scan_list(int n, double base) {
    for (int i0 = 0; i0 < n; i0 += kNT) {
      const int i = i0 + threadIdx.x;
      double total;
      const double v = block_scan(sh, i < n ? weight(list_value(i)) : 0.0, total);
      if (i < n) sh.l.cum[i] = base + v;
      base += total;
    }
    __syncthreads();
  }

  // The least r >= 1 with cum[r - 1] >= target, or n.
  __device__ __forceinline__ int first_reaching(int n, double target) {
    int r = n;
    for (int i = threadIdx.x; i < n; i += kNT)
      if (sh.l.cum[i] >= target) {
        r = i + 1;
        break;
      }
    return block_min_int(sh, r);
  }

  __device__ __forceinline__ int bin_of(float z) const {
    const double q = -4.0 * t2(z);
    return q < (double)(kBins - 1) ? (int)q : kBins - 1;
  }

  // Histogram `to`: the words of [lo, hi] by bins of a quarter power of two of weight (top = 0), or by the bits of their
  // keys below `top`, `shift` bits to a bin.  Weights relative to the bin's top, in 2^-44, then in units of the row's.
  __device__ __forceinline__ void histogram(int to, float lo, float hi, uint32_t top, int shift) {
    const int tid = threadIdx.x, colm = tid & (kCols - 1);
    for (int i = tid; i < kBins * kCols; i += kNT) {
      sh.h.mass[i] = 0ull;
      sh.h.count[i] = 0u;
    }
    __syncthreads();
    const double t_top = top ? t2(key_value(top)) : 0.0;
    for (int tile = tid >> 6; tile < tiles; tile += kNW) {
      if (sh.tmax[tile] < lo) continue;
      each_vector(tile, [&](const u32x4& x, int) {
#pragma unroll
        for (int e = 0; e < Tile<Tin>::EPV; ++e) {
          const float z = elem<Tin>(x, e);
          if (z >= lo && z <= hi) {
            const double t = t2(z);
            int b;
            double rel;
            if (top) {
              b = min((int)((top - order_key(z)) >> shift), kBins - 1);
              rel = t - t_top;
            } else {
              b = bin_of(z);
              rel = fma((double)b, 0.25, t);
            }
            const double y = exp2_neg(fmin(rel, 0.0)) + 256.0;  // the weight in 2^-44 in the low bits
            const unsigned long long w = __builtin_bit_cast(unsigned long long, y) & 0xfffffffffffffull;
            atomicAdd(&sh.h.mass[b * kCols + colm], w);
            atomicAdd(&sh.h.count[b * kCols + colm], 1u);
          }
        }
      });
    }
    __syncthreads();
    // four threads to a bin, eight columns each
    static_assert(kNT == 4 * kBins && kCols == 32, "threads to bins");
    const int b = tid >> 2, q = (tid & 3) * (kCols / 4);
    double mass = 0.0;
    int count = 0;
#pragma unroll
    for (int i = 0; i < kCols / 4; ++i) {
      const int at = b * kCols + q + ((i + (tid >> 2)) & (kCols / 4 - 1));
      mass += (double)sh.h.mass[at] * 0x1p-44;
      count += (int)sh.h.count[at];
    }
    mass += __shfl_xor(mass, 1, 64);
    mass += __shfl_xor(mass, 2, 64);
    count += __shfl_xor(count, 1, 64);
    count += __shfl_xor(count, 2, 64);
    if ((tid & 3) == 0) {
      sh.bin_mass[to][b] = mass * exp2_neg(top ? t_top : -0.25 * b);
      sh.bin_count[to][b] = count;
    }
    __syncthreads();
  }

  // The first bin of histogram `of` up to which count0 (mass0) and the bins' counts (masses) reach the target, or the
  // last one that holds a word; count0 and mass0 then end before it.
  __device__ __forceinline__ int find_bin(int of, bool by_mass, int& count0, double& mass0, int k, double target,
                                          int& in_bin) {
    const int tid = threadIdx.x, lane = tid & 63;
    if (tid < 64) {
      const int c0 = sh.bin_count[of][2 * lane], c1 = sh.bin_count[of][2 * lane + 1];
      const double m0 = sh.bin_mass[of][2 * lane], m1 = sh.bin_mass[of][2 * lane + 1];
      const int ce = scan_add(c0 + c1) - (c0 + c1) + count0;
      double me = __shfl_up(scan_add(m0 + m1), 1, 64);
      me = (lane == 0 ? 0.0 : me) + mass0;
      const bool at0 = c0 > 0 && (by_mass ? me + m0 >= target : ce + c0 >= k);
      const bool at1 = c1 > 0 && (by_mass ? me + m0 + m1 >= target : ce + c0 + c1 >= k);
      const uint64_t any = __ballot(at0 || at1), held = __ballot(c0 + c1 > 0);
      const int l = any ? __ffsll((unsigned long long)any) - 1 : 63 - __clzll((long long)(held | 1ull));
      if (lane == l) {
        const bool first = any ? at0 : c1 == 0;
        sh.bin = 2 * lane + (first ? 0 : 1);
        sh.i0 = first ? ce : ce + c0;
        sh.d0 = first ? me : me + m0;
        sh.n = first ? c0 : c1;
      }
    }
    __syncthreads();
    const int b = sh.bin;
    count0 = sh.i0;
    mass0 = sh.d0;
    in_bin = sh.n;
    __syncthreads();
    return b;
  }

  // Wave 0: the tile's r-th word (from 1) that equals z, by index.
  __device__ __forceinline__ int nth_equal(int tile, float z, int r) {
    int found = 0;
    each_vector(tile, [&](const u32x4& x, int j) {
      int n = 0;
#pragma unroll
      for (int e = 0; e < Tile<Tin>::EPV; ++e) n += elem<Tin>(x, e) == z;
      const int incl = scan_add(n);
      const int all = __builtin_amdgcn_readlane(incl, 63);
      if (r >= 1 && r <= all) {
        const int l = __ffsll((unsigned long long)__ballot(incl >= r)) - 1;
        int left = r - (incl - n), col = 0;
#pragma unroll
        for (int e = 0; e < Tile<Tin>::EPV; ++e) {
          const bool same = elem<Tin>(x, e) == z;
          left -= same;
          if (left == 0 && same) col = Tile<Tin>::col(tile, j, e);
        }
        found = __builtin_amdgcn_readlane(col, l);
      }
      r -= all;
    });
    return found;
  }

  // The index of the r-th word of the row that equals z.
  __device__ __forceinline__ int tie_index(float z, int r) {
    const int tid = threadIdx.x;
    for (int tile = tid >> 6; tile < tiles; tile += kNW) {
      int n = 0;
      if (sh.tmax[tile] >= z) {
        Tile<Tin> x;
        x.load(row, V, tile);
#pragma unroll
        for (int j = 0; j < Tile<Tin>::NV; ++j)
#pragma unroll
          for (int e = 0; e < Tile<Tin>::EPV; ++e) n += __popcll(__ballot(x.at(j, e) == z));
      }
      if ((tid & 63) == 0) sh.tcount[tile] = n;
    }
    __syncthreads();
    if (tid < 64) {
      int left = r, at = -1;
      for (int i0 = 0; i0 < tiles && at < 0; i0 += 64) {
        const int n = i0 + tid < tiles ? sh.tcount[i0 + tid] : 0;
        const int incl = scan_add(n);
        const uint64_t mask = __ballot(incl >= left);
        if (mask) {
          const int l = __ffsll((unsigned long long)mask) - 1;
          left -= __builtin_amdgcn_readlane(incl - n, l);
          at = i0 + l;
        } else {
          left -= __builtin_amdgcn_readlane(incl, 63);
        }
      }
      const int col = at < 0 ? V : nth_equal(at, z, left);
      if (tid == 0) sh.i0 = col;
    }
    __syncthreads();
    const int col = sh.i0;
    __syncthreads();
    return col;
  }

  // The cut after the k-th word, or after the shortest prefix of weight `target`, from histogram 0.
  __device__ __forceinline__ Cut select(bool by_mass, int k, double target) {
    int count0 = 0, cnt;
    double mass0 = 0.0;
    const int b = find_bin(0, by_mass, count0, mass0, k, target, cnt);
    // the keys that fall into bin b: bin_of only falls as the key grows
    auto lowest = [&](int bin) {
      uint32_t lo = order_key(x_lo), hi = order_key(m);
      while (lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2;
        if (bin_of(key_value(mid)) <= bin) hi = mid;
        else lo = mid + 1;
      }
      return lo;
    };
    constexpr uint32_t kMinusZero = 0x7fffffffu;  // the key that no word has: -0 counts as 0
    uint32_t klo = lowest(b), khi = b == 0 ? order_key(m) : lowest(b - 1) - 1;
    while (cnt > kCap && klo < khi) {
      const int bits = 32 - __clz((int)(khi - klo));
      const int shift = max(0, bits - 7);
      histogram(1, key_value(klo), key_value(khi), khi, shift);
      const int q = find_bin(1, by_mass, count0, mass0, k, target, cnt);
      khi -= (uint32_t)q << shift;
      klo = max(klo, khi - ((1u << shift) - 1));
      khi -= khi == kMinusZero;  // as a bound it would let the zeros in
    }
    Cut cut;
    if (cnt > kCap) {  // one value, more often than the list holds
      cut.thr = key_value(klo);
      const double w = weight(cut.thr);
      int r = cnt;
      if (!by_mass) r = k - count0;
      else if (w > 0.0) r = (int)fmin(ceil((target - mass0) / w), (double)cnt);
      r = max(1, min(r, cnt));
      cut.mass = mass0 + (double)r * w;
      cut.tie = r == cnt ? V : tie_index(cut.thr, r);
      return cut;
    }
    const int n = gather(key_value(klo), key_value(khi));
    sort_list(sh, n);
    scan_list(n, mass0);
    const int r = by_mass ? first_reaching(n, target) : max(1, min(k - count0, n));
    cut.thr = list_value(r - 1);
    cut.tie = list_index(r - 1);
    cut.mass = sh.l.cum[r - 1];
    __syncthreads();
    return cut;
  }

  __device__ __forceinline__ bool kept(float z, int col, float thr, int tie) const {
    return z > thr || (z == thr && col <= tie);
  }

  // Wave 0: the tile's first kept word at which the kept weights pass `left`, or its last kept word.
  __device__ __forceinline__ int pick(int tile, double left, float thr, int tie) {
    int found = -1, last = -1;
    each_vector(tile, [&](const u32x4& x, int j) {
      double w[Tile<Tin>::EPV], s = 0.0;
      int mine = -1;
#pragma unroll
      for (int e = 0; e < Tile<Tin>::EPV; ++e) {
        const float z = elem<Tin>(x, e);
        const int col = Tile<Tin>::col(tile, j, e);
        w[e] = kept(z, col, thr, tie) ? weight(z) : 0.0;
        if (w[e] > 0.0) mine = col;
        s += w[e];
      }
      const double incl = scan_add(s), excl = incl - s;
      const uint64_t mask = __ballot(s > 0.0 && incl > left);
      if (mask && found < 0) {
        const int l = __ffsll((unsigned long long)mask) - 1;
        double run = excl;
        int col = -1;
#pragma unroll
        for (int e = 0; e < Tile<Tin>::EPV; ++e) {
          run += w[e];
          if (col < 0 && w[e] > 0.0 && run > left) col = Tile<Tin>::col(tile, j, e);
        }
        if (col < 0) col = mine;  // the lane's own sum in another order
        found = __builtin_amdgcn_readlane(col, l);
      }
      const uint64_t some = __ballot(mine >= 0);
      if (some) last = __builtin_amdgcn_readlane(mine, 63 - __clzll((long long)some));
      left -= readlane_f64(incl, 63);
    });
    return found >= 0 ? found : last;
  }

  // The first kept word at which the kept weights pass u times their sum, from the tiles' sums in sh.tsum.
  __device__ __forceinline__ int draw(double target, float thr, int tie) {
    double before = 0.0;
    int at = INT_MAX, last = -1;
    for (int i0 = 0; i0 < tiles && at == INT_MAX; i0 += kNT) {
      const int i = i0 + threadIdx.x;
      const double v = i < tiles ? sh.tsum[i] : 0.0;
      double total;
      const double incl = before + block_scan(sh, v, total);
      const bool here = v > 0.0 && incl > target;
      at = block_min_int(sh, here ? i : INT_MAX);
      if (i == at) sh.d0 = target - (incl - v);
      last = max(last, block_max_int(sh, v > 0.0 ? i : -1));
      before += total;
    }
    __syncthreads();
    if (threadIdx.x < 64) {
      const bool there = at != INT_MAX;
      const int col = pick(there ? at : last, there ? sh.d0 : (double)INFINITY, thr, tie);
      if (threadIdx.x == 0) sh.i0 = col;
    }
    __syncthreads();
    return sh.i0;
  }

  // A lower bound of the k-th largest of the n partial maxima in sh.sub, and so of the row's k-th word.
  __device__ __forceinline__ float kth_bound(int n, int k) {
    if (threadIdx.x < 64) {
      const int lane = threadIdx.x;
      uint32_t key[kMaxSubs / 64];
#pragma unroll
      for (int i = 0; i < kMaxSubs / 64; ++i) key[i] = i * 64 + lane < n ? order_key(sh.sub[i * 64 + lane]) : 0u;
      uint32_t t = 0;
#pragma unroll 1
      for (int bit = 31; bit >= 12; --bit) {
        const uint32_t cand = t | (1u << bit);
        int have = 0;
#pragma unroll
        for (int i = 0; i < kMaxSubs / 64; ++i) have += __popcll(__ballot(key[i] >= cand));
        if (have >= k) t = cand;
      }
      if (lane == 0) sh.key = t;
    }
    __syncthreads();
    const uint32_t t = sh.key;
    __syncthreads();
    return t > order_key(kLiveMin) ? key_value(t) : kLiveMin;
  }

  // The smallest float whose weight is at least min_p: t2(z) >= log2(min_p).
  __device__ __forceinline__ float min_p_bound(double l) const {
    float z = fminf((float)((double)m + l / c), m);
    for (int i = 0; i < 8 && t2(z) >= l; ++i) z = nextafterf(z, -INFINITY);
    for (int i = 0; i < 64 && !(t2(z) >= l) && z < m; ++i) z = nextafterf(z, INFINITY);
    return z;
  }
};

template <typename Tin, bool FUSED, bool DRAW>
__global__ __launch_bounds__(kNT) __attribute__((amdgpu_waves_per_eu(4, 4))) void k_sample_row(const RowArgs a, int row0) {
  __shared__ RowShared sh;
  const int t = row0 + blockIdx.x, tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const Tin* row = static_cast<const Tin*>(a.logits) + (int64_t)t * a.ld;
  const Settings st = load_settings(a.par, t);
  float u = 0.f;
  bool ok = st.ok;
  int act = -1;
  if (DRAW) {
    u = a.u[t];
    ok = ok && u >= 0.f && u < 1.f;
  } else {
    act = a.actions[t];
  }
  const bool act_ok = DRAW || (act >= 0 && act < a.V);
  const bool k_on = st.k > 0 && st.k < a.V, p_on = st.p < 1.f, m_on = st.min_p > 0.f;
  const int subs = a.tiles * kSubs <= kMaxSubs ? a.tiles * kSubs : a.tiles <= kMaxSubs ? a.tiles : 0;
  const bool fine = a.tiles * kSubs <= kMaxSubs;

  // the tiles' records
  float m = -INFINITY;
  int live = 0, bad = 0;
  if (FUSED) {
    const SumMode mode = sum_mode(st, a.V, DRAW);
    for (int tile = wv; tile < a.tiles; tile += kNW) {
      Tile<Tin> x;
      x.load(row, a.V, tile);
      const TileStats s = tile_stats<Tin>(x, mode, st.c);
      if (fine && (lane & 7) == 0) sh.sub[tile * kSubs + (lane >> 3)] = s.sub;
      if (lane == 0) {
        if (!fine && subs) sh.sub[tile] = s.max;
        sh.tsum[tile] = s.sum;
        sh.tmax[tile] = s.max;
        live += s.live;
      }
      m = fmaxf(m, s.max);
      bad |= s.bad;
    }
  } else {
    for (int i = tid; i < a.tiles; i += kNT) {
      const TileRec r = a.recs[(int64_t)t * a.tiles + i];
      float mx = r.sub[0];
#pragma unroll
      for (int q = 1; q < kSubs; ++q) mx = fmaxf(mx, r.sub[q]);
      if (fine) {
#pragma unroll
        for (int q = 0; q < kSubs; ++q) sh.sub[i * kSubs + q] = r.sub[q];
      } else if (subs) {
        sh.sub[i] = mx;
      }
      sh.tsum[i] = r.sum;
      sh.tmax[i] = mx;
      live += r.live;
      bad |= r.bad;
      m = fmaxf(m, mx);
    }
  }
  __syncthreads();
  live = block_sum_int(sh, live);
  bad = block_max_int(sh, bad);
  m = key_value((uint32_t)block_max_int(sh, (int)(order_key(m) ^ 0x80000000u)) ^ 0x80000000u);

  grpo_sampling_row out;
  out.max = m;
  out.temperature = st.tau;
  out.threshold = INFINITY;
  out.tie = -1;
  out.n_kept = 0;
  out.sum = 0.0;
  out.logp = -INFINITY;
  int flag = 0;
  if (!ok || bad) {
    out.sum = NAN;
    out.logp = NAN;
    flag = ok ? GRPO_FLAG_NONFINITE : GRPO_FLAG_SETTING;
  } else if (live == 0) {
    flag = GRPO_FLAG_NONFINITE;
  } else {
    RowWork<Tin> w{sh, row, a.V, a.tiles, m, st.c, kLiveMin};
    float thr = -1e8f;  // kept: above it
    int tie = -1, n = live;
    double S = 0.0;
    if (st.greedy) {
      int first = INT_MAX;
      for (int i = tid; i < a.tiles; i += kNT)
        if (sh.tmax[i] == m) {
          first = i;
          break;
        }
      first = block_min_int(sh, first);
      if (wv == 0) {
        const int col = w.nth_equal(first, m, 1);
        if (lane == 0) sh.i0 = col;
      }
      __syncthreads();
      thr = m;
      tie = sh.i0;
      n = 1;
      S = 1.0;
      if (DRAW) act = tie;
    } else {
      // the tiles' sums relative to the row's maximum
      double total = 0.0;
      for (int i = tid; i < a.tiles; i += kNT) {
        const double v = sh.tmax[i] >= kLiveMin ? sh.tsum[i] * w.weight(sh.tmax[i]) : 0.0;
        sh.tsum[i] = v;
        total += v;
      }
      S = block_sum(sh, total);
      bool drawn = !DRAW;
      if (k_on || p_on || m_on) {
        const int k = min(st.k, live);
        const float z_min = m_on ? w.min_p_bound(log2((double)st.min_p)) : kLiveMin;
        float x_lo = k_on && p_on ? kLiveMin : fmaxf(z_min, kLiveMin);  // top-p of top-k needs the first k words' sum
        if (k_on && k <= subs) x_lo = fmaxf(x_lo, w.kth_bound(subs, k));
        if (p_on && !k_on) {
          // all words lighter than (1 - p) S / live together weigh less than (1 - p) S
          const double l = log2((double)live / ((1.0 - (double)st.p) * S)) + 0.01;
          const double z = (double)m - l / st.c;
          float zf = fminf((float)z, m);
          if ((double)zf > z) zf = nextafterf(zf, -INFINITY);
          x_lo = fmaxf(x_lo, zf);
        }
        w.x_lo = x_lo;
        const int listed = w.gather(x_lo, INFINITY);
        if (listed <= kCap) {
          sort_list(sh, listed);
          w.scan_list(listed, 0.0);
          n = k_on ? min(k, listed) : listed;
          if (p_on) {
            const double Sk = k_on ? sh.l.cum[n - 1] : S;
            n = min(n, w.first_reaching(listed, (double)st.p * Sk));
          }
          if (m_on) {
            int c = 0;
            for (int i = tid; i < listed; i += kNT) c += w.list_value(i) >= z_min;
            n = min(n, block_sum_int(sh, c));
          }
          n = max(n, 1);
          thr = w.list_value(n - 1);
          tie = w.list_index(n - 1);
          S = sh.l.cum[n - 1];
          __syncthreads();
          if (DRAW) {
            // the kept words in the order of their indices, smallest first: keys that fall as the index grows
            for (int i = tid; i < n; i += kNT) {
              const unsigned long long q = sh.l.key[i];
              sh.l.key[i] = (q << 32) | (q >> 32);
            }
            __syncthreads();
            sort_list(sh, n);
            double before = 0.0;
            int at = INT_MAX, last = 0;
            const double target = (double)u * S;
            for (int i0 = 0; i0 < n && at == INT_MAX; i0 += kNT) {
              const int i = i0 + tid;
              const double v = i < n ? w.weight(key_value((uint32_t)sh.l.key[i])) : 0.0;
              double all;
              const double incl = before + block_scan(sh, v, all);
              at = block_min_int(sh, v > 0.0 && incl > target ? i : INT_MAX);
              last = max(last, block_max_int(sh, v > 0.0 ? i : 0));
              before += all;
            }
            act = (int)~(uint32_t)(sh.l.key[at == INT_MAX ? last : at] >> 32);
            drawn = true;
          }
        } else {
          thr = kLiveMin;
          tie = a.V;
          auto narrow = [&](float z, int i) {
            if (z > thr || (z == thr && i < tie)) {
              thr = z;
              tie = i;
            }
          };
          if (k_on || p_on) {
            w.histogram(0, x_lo, INFINITY, 0u, 0);
            double Sk = S;
#pragma unroll 1
            for (int by_mass = 0; by_mass < 2; ++by_mass) {
              if (by_mass ? !p_on : !k_on) continue;
              const Cut cut = w.select(by_mass, k, (double)st.p * Sk);
              narrow(cut.thr, cut.tie);
              Sk = cut.mass;
            }
          }
          if (m_on) narrow(z_min, a.V);
          // the kept words' sums, tile by tile in the order of the indices
          int kept_here = 0;
          for (int tile = wv; tile < a.tiles; tile += kNW) {
            double s = 0.0;
            if (sh.tmax[tile] >= thr) {
              w.each_vector(tile, [&](const u32x4& x, int j) {
#pragma unroll
                for (int e = 0; e < Tile<Tin>::EPV; ++e) {
                  const float z = elem<Tin>(x, e);
                  if (w.kept(z, Tile<Tin>::col(tile, j, e), thr, tie)) {
                    s += w.weight(z);
                    ++kept_here;
                  }
                }
              });
              s = wave_sum_dpp(s);
            }
            if (lane == 0) sh.tsum[tile] = s;
          }
          __syncthreads();
          double sum = 0.0;
          for (int i = tid; i < a.tiles; i += kNT) sum += sh.tsum[i];
          S = block_sum(sh, sum);
          n = block_sum_int(sh, kept_here);
        }
      }
      if (!drawn) act = w.draw((double)u * S, thr, tie);
    }
    if (tid == 0) {
      out.threshold = thr;
      out.tie = tie;
      out.n_kept = n;
      out.sum = S;
      if (act_ok) {
        const float z = load_elem(row + act);
        if (z >= kLiveMin && w.kept(z, act, thr, tie))
          out.logp = st.greedy ? 0.f : (float)(((double)z - (double)m) / (double)st.tau - log(S));
      }
    }
  }
  if (tid == 0) {
    if (!act_ok) {
      out.logp = 0.f;
      flag |= GRPO_FLAG_ACTION;
    }
    if (DRAW) a.actions_out[t] = out.n_kept > 0 ? act : -1;
    if (a.logp) a.logp[t] = out.logp;
    if (a.n_kept) a.n_kept[t] = out.n_kept;
    if (a.rows) a.rows[t] = out;
    if (a.flags && flag) atomicOr(a.flags, flag);
  }
}

// ---- the gradient ---------------------------------------------------------------
struct BwdArgs {
  const void* logits;
  void* dlogits;
  int64_t ld;
  int V, blocks;  // blocks of columns to a row
  const int32_t* actions;
  const grpo_sampling_row* rows;
  const float* dlogp;
};

constexpr int kBwdNT = 256, kBwdCols = 8192;

// One workgroup to kBwdCols columns of a row, all loads in flight before the first store: a streaming pass, bound by
// the 2 + 2 (bf16) or 4 + 4 bytes per word.
template <typename Tin>
__global__ __launch_bounds__(kBwdNT) __attribute__((amdgpu_waves_per_eu(4, 8))) void k_sampled_bwd(const BwdArgs a, int row0) {
  constexpr int EPV = 16 / (int)sizeof(Tin), U = kBwdCols / kBwdNT / EPV;
  typedef typename VecAt<Tin>::type u32x4_any;
  const int t = row0 + (int)(blockIdx.x / (unsigned)a.blocks), b = (int)(blockIdx.x % (unsigned)a.blocks);
  const int tid = threadIdx.x;
  const Tin* row = static_cast<const Tin*>(a.logits) + (int64_t)t * a.ld;
  Tin* drow = static_cast<Tin*>(a.dlogits) + (int64_t)t * a.ld;
  const grpo_sampling_row r = a.rows[t];
  const int act = a.actions[t];
  const bool nan = isnan(r.sum);
  const bool none = !nan && (act < 0 || act >= a.V || !(r.logp > -INFINITY) || !(r.temperature > 0.f));
  const double scale = none ? 0.0 : nan ? (double)NAN : (double)a.dlogp[t] / (double)r.temperature;
  // d_v = -scale P(v), P(v) = 2^((z - max) c - log2 S); formed from z - max, which keeps the exponent's rounding small
  const float c = (float)(kLog2e64 / (double)r.temperature);
  const float l = none || nan ? 0.f : (float)log2(r.sum);
  const float neg = (float)-scale;
  const int c0 = b * kBwdCols;
  // Words that equal the threshold are kept up to r.tie: all of this workgroup's, none, or (mixed) some of them.
  const float least = r.tie < c0 ? nextafterf(r.threshold, INFINITY) : r.threshold;
  const bool mixed = r.tie >= c0 && r.tie < c0 + kBwdCols;
  auto one = [&](float z, int col, bool ties) {
    const bool in = z >= least && !(ties && z == r.threshold && col > r.tie);
    return in ? neg * __builtin_amdgcn_exp2f(fmaf(z - r.max, c, -l)) : 0.f;
  };
  auto vec = [&](const u32x4& x, int col, bool ties) {
    u32x4 o;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if constexpr (sizeof(Tin) == 2)
        o[q] = pack_bf16(one(bf16_lo(x[q]), col + 2 * q, ties), one(bf16_hi(x[q]), col + 2 * q + 1, ties));
      else
        o[q] = __float_as_uint(one(__uint_as_float(x[q]), col + q, ties));
    }
    return o;
  };
  // the action's own, formed in fp64; read before any store, which may be to the same place
  const bool has_act = act >= c0 && act < min(c0 + kBwdCols, a.V);
  float d_act = 0.f;
  if (has_act) {
    const float z = load_elem(row + act);
    d_act = none ? 0.f : (float)(scale * (1.0 - exp(((double)z - (double)r.max) / (double)r.temperature) / r.sum));
    __syncthreads();
  }
  const int edge = a.V / EPV * EPV;  // the row's last words, fewer than a vector holds, one to a thread
  const int n_edge = b == a.blocks - 1 ? a.V - edge : 0;
  u32x4 x[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int col = c0 + (i * kBwdNT + tid) * EPV;
    if (col + EPV <= a.V) x[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_any*>(row + col));
  }
  const float ez = tid < n_edge ? load_elem(row + edge + tid) : 0.f;
  auto store = [&](auto value) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int col = c0 + (i * kBwdNT + tid) * EPV;
      if (col + EPV <= a.V) {
        __builtin_nontemporal_store(value(x[i], col), reinterpret_cast<u32x4_any*>(drow + col));
        asm volatile("s_nop 1" ::: "memory");  // the store has read its data before its registers are reused
      }
    }
  };
  if (none || nan) {
    const float v = none ? 0.f : NAN;
    const uint32_t w = sizeof(Tin) == 2 ? pack_bf16(v, v) : __float_as_uint(v);
    store([&](const u32x4&, int) { return u32x4{w, w, w, w}; });
    if (tid < n_edge) store_elem(drow + edge + tid, v);
    return;
  }
  if (mixed) store([&](const u32x4& v, int col) { return vec(v, col, true); });
  else store([&](const u32x4& v, int col) { return vec(v, col, false); });
  if (tid < n_edge) store_elem(drow + edge + tid, one(ez, edge + tid, mixed));
  // the thread that stored the action's place, after that store
  if (has_act && tid == (act >= edge ? act - edge : (act - c0) / EPV % kBwdNT)) store_elem(drow + act, d_act);
}

__global__ void k_clear_sampling_flag(int32_t* f) { *f = 0; }

// ---- host -----------------------------------------------------------------------

// Whether the tiles are reduced by a launch of their own.
static bool split_rows(int64_t T, int64_t V) { return T < 192 && V > kNW * kTile; }

static int check_settings(const grpo_sampling* g) {
  if (!g) return GRPO_ERR_ARG;
  if (!g->temperature && !(g->temperature_all == 0.f || (g->temperature_all >= 1e-6f && g->temperature_all <= 1e6f)))
    return GRPO_ERR_ARG;
  if (!g->top_p && !(g->top_p_all >= 0.f && g->top_p_all <= 1.f)) return GRPO_ERR_ARG;
  if (!g->min_p && !(g->min_p_all >= 0.f && g->min_p_all <= 1.f)) return GRPO_ERR_ARG;
  if (!aligned(g->temperature, 4) || !aligned(g->top_k, 4) || !aligned(g->top_p, 4) || !aligned(g->min_p, 4))
    return GRPO_ERR_ALIGN;
  return GRPO_OK;
}

static bool bad_shape(int64_t T, int64_t V, int64_t ld) {
  return T < 0 || T >= ((int64_t)1 << 31) || V < 1 || V > GRPO_SAMPLING_MAX_V || ld < V;
}

template <typename Tin, bool DRAW>
static void launch_rows(const RowArgs& a, int64_t T, hipStream_t s) {
  if (split_rows(T, a.V)) {
    const int waves = (int)T * a.tiles;
    hipLaunchKernelGGL(k_sample_tiles<Tin>, dim3((unsigned)(waves + 3) / 4), dim3(256), 0, s, a, waves, DRAW);
    hipLaunchKernelGGL((k_sample_row<Tin, false, DRAW>), dim3((unsigned)T), dim3(kNT), 0, s, a, 0);
    return;
  }
  constexpr int64_t kRows = 1 << 20;  // a launch's threads stay below 2^32
  for (int64_t r = 0; r < T; r += kRows)
    hipLaunchKernelGGL((k_sample_row<Tin, true, DRAW>), dim3((unsigned)std::min(kRows, T - r)), dim3(kNT), 0, s, a,
                       (int)r);
}

template <bool DRAW>
static int sample_call(const void* logits, int32_t dtype, int64_t T, int64_t V, int64_t ld, const grpo_sampling* par,
                       const float* u, const int32_t* actions, int32_t* actions_out, float* logp, int32_t* n_kept,
                       grpo_sampling_row* rows, int32_t* flags, void* ws, size_t ws_bytes, hipStream_t s) {
  if (bad_shape(T, V, ld)) return GRPO_ERR_SHAPE;
  if (T > 0 && (!logits || (DRAW ? !u || !actions_out : !actions))) return GRPO_ERR_ARG;
  int st = check_settings(par);
  if (st != GRPO_OK) return st;
  if (dtype != GRPO_F32 && dtype != GRPO_BF16) return GRPO_ERR_DTYPE;
  if (!aligned(logits, dtype == GRPO_BF16 ? 2 : 4) || !aligned(u, 4) || !aligned(actions, 4) || !aligned(actions_out, 4) ||
      !aligned(logp, 4) || !aligned(n_kept, 4) || !aligned(rows, 8) || !aligned(flags, 4))
    return GRPO_ERR_ALIGN;
  if (T > 0 && split_rows(T, V)) {
    if (!ws || ws_bytes < grpo_sampling_workspace_bytes(T, V)) return GRPO_ERR_WORKSPACE;
    if (!aligned(ws, 16)) return GRPO_ERR_ALIGN;
  }
  if (flags) hipLaunchKernelGGL(k_clear_sampling_flag, dim3(1), dim3(1), 0, s, flags);
  if (T > 0) {
    const RowArgs a{logits, ld,     (int)V, (int)((V + kTile - 1) / kTile), *par,  u, actions, actions_out,
                    logp,   n_kept, rows,   flags, static_cast<TileRec*>(ws)};
    if (dtype == GRPO_BF16) launch_rows<uint16_t, DRAW>(a, T, s);
    else launch_rows<float, DRAW>(a, T, s);
  }
  return hipGetLastError() == hipSuccess ? GRPO_OK : GRPO_ERR_HIP;
}

}  // namespace grpo

using namespace grpo;

extern "C" size_t grpo_sampling_workspace_bytes(int64_t T, int64_t V) {
  if (bad_shape(T, V, V)) return 0;
  const size_t recs = split_rows(T, V) ? sizeof(TileRec) * (size_t)T * (size_t)((V + kTile - 1) / kTile) : 0;
  return align_up(std::max(recs, (size_t)1));
}

extern "C" int grpo_sample(const void* logits, int32_t dtype, int64_t T, int64_t V, int64_t ld,
                           const grpo_sampling* par, const float* u, int32_t* actions, float* logp, int32_t* n_kept,
                           int32_t* error_flags, void* ws, size_t ws_bytes, hipStream_t s) {
  return sample_call<true>(logits, dtype, T, V, ld, par, u, nullptr, actions, logp, n_kept, nullptr, error_flags, ws,
                           ws_bytes, s);
}

extern "C" int grpo_sampled_logp(const void* logits, int32_t dtype, int64_t T, int64_t V, int64_t ld,
                                 const grpo_sampling* par, const int32_t* actions, float* logp, int32_t* n_kept,
                                 grpo_sampling_row* rows, int32_t* error_flags, void* ws, size_t ws_bytes,
                                 hipStream_t s) {
  return sample_call<false>(logits, dtype, T, V, ld, par, nullptr, actions, nullptr, logp, n_kept, rows, error_flags,
                            ws, ws_bytes, s);
}

extern "C" int grpo_sampled_logp_bwd(const void* logits, int32_t dtype, int64_t T, int64_t V, int64_t ld,
                                     const int32_t* actions, const grpo_sampling_row* rows, const float* dlogp,
                                     void* dlogits, hipStream_t s) {
  if (bad_shape(T, V, ld)) return GRPO_ERR_SHAPE;
  if (T > 0 && (!logits || !actions || !rows || !dlogp || !dlogits)) return GRPO_ERR_ARG;
  if (dtype != GRPO_F32 && dtype != GRPO_BF16) return GRPO_ERR_DTYPE;
  const size_t esz = dtype == GRPO_BF16 ? 2 : 4;
  if (!aligned(logits, esz) || !aligned(dlogits, esz) || !aligned(actions, 4) || !aligned(rows, 8) || !aligned(dlogp, 4))
    return GRPO_ERR_ALIGN;
  const int blocks = (int)((V + kBwdCols - 1) / kBwdCols);
  const int64_t per = std::max<int64_t>(1, ((int64_t)1 << 23) / blocks);  // a launch's threads stay below 2^32
  for (int64_t r = 0; r < T; r += per) {
    const BwdArgs a{logits, dlogits, ld, (int)V, blocks, actions, rows, dlogp};
    const unsigned grid = (unsigned)(std::min(per, T - r) * blocks);
    if (dtype == GRPO_BF16) hipLaunchKernelGGL(k_sampled_bwd<uint16_t>, dim3(grid), dim3(kBwdNT), 0, s, a, (int)r);
    else hipLaunchKernelGGL(k_sampled_bwd<float>, dim3(grid), dim3(kBwdNT), 0, s, a, (int)r);
  }
  return hipGetLastError() == hipSuccess ? GRPO_OK : GRPO_ERR_HIP;
}
