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
// A row is cut into tiles, each reduced in a wave's registers to its maximum, its count of live words and
// its sum of weights relative to its own maximum: one pass over memory, of any number of waves per row.  Then one
// workgroup per row works on the tiles' records and re-reads only the tiles that it needs:
//   nothing cut     a draw picks its tile by the tiles' sums and re-reads that one;
//   few candidates  a lower bound of the threshold (the k-th largest of the partial maxima; for top-p, the weight below
//                   which all live words together weigh less than (1 - p) S; min-p's own) leaves at most kCap words: they
//                   are gathered in LDS, and the cut is read off the sorted words' prefix sums (up to kSorted), or found
//                   as in the last case, in the list instead of the row;
//   many, bf16      a count of each value (bf16 logits below 64 in size have 5,377 that are told apart); counts times weights,
//                   summed from the top, give the cut, and a table of the values' weights the tiles' kept sums;
//   many, else      counts by fine bins of weight say which bin holds the cut, and one more pass gathers that bin's words
//                   and sums the words above them; where they do not (a value that repeats, one bin for many words),
//                   histograms: words fall into kBins bins, each bin's count and weight are summed, the bin that holds the
//                   cut is split again by the bits of its logits until at most kSorted words (gathered and sorted) or one
//                   repeated value are left.
// Histogram weights are integers (weight relative to the bin's top, in 2^-42 or finer), so that atomics in any order give one
// sum.
//
// A pass over a row by its own workgroup is bound by its instructions, not by memory: about 6 us for 32,003 fp32 words where
// tiles are reduced or words counted, 13 us where each word's fp64 weight is summed, two rows on a CU (a CU's share of the
// memory would bring them in 11 us for both).  The loops over a tile's vectors are rolled: unrolled, the kernel waits for its
// own instructions.
#include <hip/hip_runtime.h>
#include <float.h>
#include <math.h>

#include <algorithm>

#include "device.h"
#include "grpo_sampling.h"
#include "host.h"

namespace grpo {

constexpr int kTileVecs = 4;       // a tile: 4 vectors of 16 bytes per lane, 2,048 bf16 words or 1,024 of fp32
constexpr int kSubs = 8;           // partial maxima of a tile in its record, each over 8 lanes' words

// What a row's workgroup of NT threads holds in LDS, and so how many rows a CU works on at once: two with 512 threads (one
// with 1,024), four with 256 for rows of at most 16,384 words.
template <int NT>
struct RowShape {
  static constexpr int kMaxSubs = 1280;  // partial maxima (or tiles' maxima) that bound the k-th largest word
  static constexpr int kCap = 2048;      // words that a list holds
  static constexpr int kSorted = 256;    // words that are sorted
  static constexpr int kBins = 1024, kCols = 2;  // bins of 32 to a power of two of weight, each in kCols copies
  static constexpr int kMaxWords = GRPO_SAMPLING_MAX_V;
  static constexpr int kUnitBits = 42;  // a bin's weights are in 2^-kUnitBits
  static constexpr bool kValueTable = true;  // room for the counts of bf16 values
};
template <>
struct RowShape<256> {
  static constexpr int kMaxSubs = 1024, kCap = 1024, kSorted = 256, kBins = 512, kCols = 1, kMaxWords = 16384;
  static constexpr int kUnitBits = 44;
  static constexpr bool kValueTable = false;
};
constexpr int kMaxNW = 16;
constexpr float kLimit = 64.f;     // logits that the count of values takes: below it in size
constexpr float kLiveMin = -99999992.f;  // the smallest float above -1e8: the lowest live logit
constexpr double kLog2e64 = 1.4426950408889634074;

struct TileRec {
  double sum;
  float sub[kSubs];
  float lo;       // the least live logit
  int32_t live;
  int32_t bad;
  int32_t pad;
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

// Inclusive sums over the wave, by lane moves within rows of 16 (row_shr), then from row to row (row_bcast).
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_rows(int x) {
  return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xF, ROWS == 0xF);
}
template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ double dpp_rows(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = (uint32_t)dpp_rows<CTRL, ROWS>((int)(uint32_t)u);
  const uint32_t hi = (uint32_t)dpp_rows<CTRL, ROWS>((int)(uint32_t)(u >> 32));
  return __builtin_bit_cast(double, (uint64_t)lo | ((uint64_t)hi << 32));
}
template <typename T>
__device__ __forceinline__ T scan_add(T v) {
  v += dpp_rows<0x111, 0xF>(v);
  v += dpp_rows<0x112, 0xF>(v);
  v += dpp_rows<0x114, 0xF>(v);
  v += dpp_rows<0x118, 0xF>(v);
  v += dpp_rows<0x142, 0xA>(v);
  v += dpp_rows<0x143, 0xC>(v);
  return v;
}

// A value that every lane has, in scalar registers.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ float uniform(float v) { return __uint_as_float((uint32_t)uniform((int)__float_as_uint(v))); }
__device__ __forceinline__ double uniform(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = (uint32_t)uniform((int)(uint32_t)u), hi = (uint32_t)uniform((int)(uint32_t)(u >> 32));
  return __builtin_bit_cast(double, (uint64_t)lo | ((uint64_t)hi << 32));
}

template <typename F>
__device__ __forceinline__ int wave_reduce(int v, F f) {
  v = f(v, (int)dpp_u32<0xB1>((uint32_t)v));
  v = f(v, (int)dpp_u32<0x4E>((uint32_t)v));
  v = f(v, (int)dpp_u32<0x141>((uint32_t)v));
  v = f(v, (int)dpp_u32<0x140>((uint32_t)v));
  return f(f(__builtin_amdgcn_readlane(v, 0), __builtin_amdgcn_readlane(v, 16)),
           f(__builtin_amdgcn_readlane(v, 32), __builtin_amdgcn_readlane(v, 48)));
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

// How a tile's weights are summed: not at all, exactly enough for a cut or a draw (fp64), for a log-prob alone, and for a
// first estimate of a cut (fp32 terms, like the other log-probs of this library; off by less than kSum32Error), or by
// counting the row's values.
enum SumMode { kNoSum, kSum64, kSum32, kCount };
constexpr double kSum32Error = 1e-5;
__device__ __forceinline__ SumMode sum_mode(const Settings& s, int V, bool draw, bool fused, bool by_value, int subs) {
  if (!s.ok || s.greedy) return kNoSum;
  const bool k_on = s.k > 0 && s.k < V;
  if (fused && by_value && (k_on ? s.k > subs : s.p < 1.f || s.min_p > 0.f)) return kCount;
  if (k_on) return kNoSum;
  if (s.p < 1.f) return fused ? kSum32 : kSum64;
  if (s.min_p > 0.f) return kNoSum;
  return draw ? kSum64 : kSum32;
}

// ---- tiles ----------------------------------------------------------------------
// Vector j of lane l holds the tile's words (64 j + l) EPV ..., as element e of 16 bytes; the hardware takes vector loads
// at any alignment, so a row may start at any element.  Words past the row's end read as -inf.
template <typename Tin>
struct Tile {
  static constexpr int EPV = 16 / (int)sizeof(Tin), NV = kTileVecs, kWords = 64 * EPV * NV;
  u32x4 v[NV];

  __device__ __forceinline__ static int col(int tile, int j, int e, int lane = threadIdx.x & 63) {
    return tile * kWords + (j * 64 + lane) * EPV + e;
  }
  // The vector at column c0, which the row's end may cut.
  __device__ __forceinline__ static u32x4 load_one(const Tin* row, int V, int c0) {
    typedef typename VecAt<Tin>::type u32x4_any;
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
  __device__ __forceinline__ void load(const Tin* row, int V, int tile, int lane = threadIdx.x & 63) {
    typedef typename VecAt<Tin>::type u32x4_any;
    if (__all((tile + 1) * kWords <= V)) {
#pragma unroll
      for (int j = 0; j < NV; ++j) v[j] = *reinterpret_cast<const u32x4_any*>(row + col(tile, j, 0, lane));
    } else {
#pragma unroll 1
      for (int j = 0; j < NV; ++j) {
        const u32x4 r = load_one(row, V, col(tile, j, 0, lane));
#pragma unroll
        for (int i = 0; i < NV; ++i)
          if (i == j) v[i] = r;
      }
    }
  }
  __device__ __forceinline__ float at(int j, int e) const { return elem<Tin>(v[j], e); }
  // Vector j, the same j in every lane: a loop over them that is not unrolled keeps the code short, which most of this
  // file is bound by where a row is worked on by one workgroup (code is fetched once by each).
  __device__ __forceinline__ u32x4 vec(int j) const {
    u32x4 r = v[0];
    asm("" : "+v"(r));  // registers chosen between, not a place in memory
#pragma unroll
    for (int i = 1; i < NV; ++i) {
      u32x4 q = v[i];
      asm("" : "+v"(q));
      r = j == i ? q : r;
    }
    return r;
  }
};

struct TileStats {
  double sum;   // of weights relative to max; every lane
  float own;    // the maximum of this lane's words
  float sub;    // over its group of 8 lanes
  float max;    // every lane
  float lo;     // the least live logit; every lane
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
  s.own = mx;
  float g = fmaxf(mx, dpp_f32v<0xB1>(mx));
  g = fmaxf(g, dpp_f32v<0x4E>(g));
  s.sub = fmaxf(g, dpp_f32v<0x141>(g));
  s.max = wave_max_dpp(mx);
  float lo = -wave_max_dpp(-mn);
  s.bad = __any(nan) || s.max == INFINITY;
  s.sum = 0.0;
  s.live = Tile<Tin>::kWords;
  const bool all_live = lo >= kLiveMin;
  if (!all_live) {
    s.live = 0;
    mn = INFINITY;
#pragma unroll 1
    for (int j = 0; j < NV; ++j) {
      const u32x4 v = x.vec(j);
#pragma unroll
      for (int e = 0; e < EPV; ++e) {
        const float z = elem<Tin>(v, e);
        s.live += __popcll(__ballot(z >= kLiveMin));
        if (z >= kLiveMin) mn = fminf(mn, z);
      }
    }
    lo = -wave_max_dpp(-mn);
  }
  s.lo = lo;
  if (mode == kNoSum || mode == kCount || s.bad || s.live == 0) return s;
  if (mode == kSum64) {
    const double m = (double)s.max;
    double sum = 0.0;
    if (all_live && (m - (double)lo) * c < 1000.0) {
#pragma unroll 1
      for (int j = 0; j < NV; ++j) {
        const u32x4 v = x.vec(j);
#pragma unroll
        for (int e = 0; e < EPV; ++e) sum += exp2_neg<false>(((double)elem<Tin>(v, e) - m) * c);
      }
    } else {
#pragma unroll 1
      for (int j = 0; j < NV; ++j) {
        const u32x4 v = x.vec(j);
#pragma unroll
        for (int e = 0; e < EPV; ++e) {
          const float z = elem<Tin>(v, e);
          sum += z >= kLiveMin ? exp2_neg(((double)z - m) * c) : 0.0;
        }
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
#pragma unroll 1
      for (int j = 0; j < NV; ++j) {
        const u32x4 v = x.vec(j);
#pragma unroll
        for (int e = 0; e < EPV; ++e) {
          const float z = elem<Tin>(v, e);
          sum += z >= kLiveMin ? __builtin_amdgcn_exp2f((z - s.max) * c32) : 0.f;
        }
      }
    }
    s.sum = wave_sum_dpp((double)sum);
  }
  return s;
}

// The tiles of few rows, one wave each, spread over the whole chip.  bf16 [1, 151,936]: 4.5 us, a launch's latency; [64,
// 151,936]: 14 us, bound by the fp64 weights of a row with nothing cut (19 MB: 3.5 us).
template <typename Tin>
__global__ __launch_bounds__(256) void k_sample_tiles(const RowArgs a, int n_waves, bool draw) {
  const int w = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (w >= n_waves) return;
  const int t = w / a.tiles, tile = w - t * a.tiles;
  const Settings st = load_settings(a.par, t);
  Tile<Tin> x;
  x.load(static_cast<const Tin*>(a.logits) + (int64_t)t * a.ld, a.V, tile);
  const TileStats s = tile_stats<Tin>(x, sum_mode(st, a.V, draw, false, false, 0), st.c);
  TileRec* r = a.recs + w;
  if ((lane & 7) == 0) r->sub[lane >> 3] = s.sub;
  if (lane == 0) {
    r->sum = s.sum;
    r->lo = s.lo;
    r->live = s.live;
    r->bad = s.bad;
  }
}

// ---- one row --------------------------------------------------------------------
// bf16 logits below kLimit in size, by value: `i` counts the steps from 2^-15 up, 0 is anything smaller in size, and
// kSteps + 1 is what does not count (masked words); a word's bin is kMid + i or kMid - i by its sign.
constexpr int kStepLo = 0x3800;                       // the bits of 2^-15
constexpr int kSteps = 0x4280 - kStepLo;              // of kLimit, less those
constexpr int kMid = kSteps + 1, kValues = 2 * kMid + 1;
typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
// Both bins of a pair of words, less kMid; `least` is 0 where one of either half was kMid itself.
__device__ __forceinline__ s16x2 value_bins(uint32_t w, u16x2& least) {
  u16x2 i = __builtin_bit_cast(u16x2, w & 0x7fff7fffu);
  i = __builtin_elementwise_sub_sat(i, (u16x2)(unsigned short)(kStepLo - 1));
  least = __builtin_elementwise_min(least, i);
  i = __builtin_elementwise_min(i, (u16x2)(unsigned short)kMid);
  const s16x2 sign = __builtin_bit_cast(s16x2, w) >> (s16x2)(short)15;
  return (__builtin_bit_cast(s16x2, i) ^ sign) - sign;
}
__device__ __forceinline__ float bin_value(int bin) {
  const int i = bin - kMid, mag = (i < 0 ? -i : i) + kStepLo - 1;
  return i == 0 ? 0.f : __uint_as_float(((uint32_t)mag << 16) | (i < 0 ? 0x80000000u : 0u));
}

// The bin of a logit below kLimit in size, less kMid.
__device__ __forceinline__ int bin_index(float z) {
  const int mag = (int)((__float_as_uint(z) & 0x7fffffffu) >> 16), i = max(0, mag - (kStepLo - 1));
  return z < 0.f ? -i : i;
}

struct Cut {
  float thr;    // kept: z > thr, or z == thr and index <= tie
  int tie;
  double mass;  // the prefix that ends there: its weight, its words
  int count;
};

constexpr int kMidWords = 1 << 20;  // as many words of bin kMid do not fit their sum

template <bool TABLE>
struct ValueTable {
  double weight[kValues];
  uint32_t count[kValues];
  unsigned long long mid;  // the weight of the words of bin kMid, in 2^-44 of the next bin's
};
template <>
struct ValueTable<false> {};

template <int NT>
struct RowShared {
  typedef RowShape<NT> Shape;
  union {
    struct {
      unsigned long long mass[Shape::kBins * Shape::kCols];
      uint32_t count[Shape::kBins * Shape::kCols];
      double bin_mass[Shape::kBins];
      int bin_count[Shape::kBins];
      unsigned long long key[Shape::kCap];      // a list of words: order_key, ~index
      unsigned long long some[Shape::kSorted];  // a few of them
      unsigned long long sorted[Shape::kSorted];
      double cum[Shape::kSorted];               // prefix sums of the sorted ones' weights
    } h;
    ValueTable<Shape::kValueTable> v;
  };
  float sub[Shape::kMaxSubs];
  uint16_t block[Shape::kMaxSubs];
  double wd[2][kMaxNW];
  int wi[2][kMaxNW];
  float wf[2][kMaxNW];
  uint32_t radix[256];
  // broadcast
  int n, bin, i0;
  uint32_t key, key2;
  double d0;
};

// A tile's record in LDS, `tiles` of each after RowShared.
struct RowTiles {
  double* sum;
  float* max;
  int* count;
};
__host__ __device__ constexpr size_t row_tile_bytes(int tiles) { return (size_t)tiles * 16; }

template <typename Tin, int NT>
struct RowWork {
  typedef RowShape<NT> Shape;
  static constexpr int NW = NT / 64, NV = Tile<Tin>::NV, EPV = Tile<Tin>::EPV;
  static constexpr int kBins = Shape::kBins, kCols = Shape::kCols, kCap = Shape::kCap, kSorted = Shape::kSorted;
  static constexpr int kMaxTiles = (Shape::kMaxWords + Tile<Tin>::kWords - 1) / Tile<Tin>::kWords;
  static constexpr bool kByValue = sizeof(Tin) == 2 && Shape::kValueTable;
  RowShared<NT>& sh;
  RowTiles rec;
  const Tin* row;
  int V, tiles;
  float m;   // the row's maximum
  double c;  // log2(e) / tau
  float x_lo;  // words below it are not looked at
  int per;     // partial maxima of a tile: 64, 8 or 1, each over 64 / per lanes' words
  bool fine;   // sh.sub holds them

  int turn = 0;  // which of the two sets of sh.w* the next reduction takes

  // ---- over the workgroup: the same value in every thread.  One barrier each: a set is written again after the next
  // reduction's barrier, when every wave has read it. ----
  __device__ __forceinline__ double block_sum(double v) {
    const int b = turn, lane = threadIdx.x & 63;
    turn ^= 1;
    v = wave_sum_dpp(v);
    if (lane == 0) sh.wd[b][threadIdx.x >> 6] = v;
    __syncthreads();
    return readlane_f64(row16_sum(lane < NW ? sh.wd[b][lane] : 0.0), 0);
  }
  template <typename F>
  __device__ __forceinline__ int block_reduce(int v, F f) {  // f(a, a) = a
    const int b = turn, lane = threadIdx.x & 63;
    turn ^= 1;
    v = wave_reduce(v, f);
    if (lane == 0) sh.wi[b][threadIdx.x >> 6] = v;
    __syncthreads();
    return wave_reduce(sh.wi[b][lane & (NW - 1)], f);
  }
  __device__ __forceinline__ int block_sum(int v) {
    const int b = turn, lane = threadIdx.x & 63;
    turn ^= 1;
    v = scan_add(v);
    if (lane == 63) sh.wi[b][threadIdx.x >> 6] = v;
    __syncthreads();
    return __builtin_amdgcn_readlane(scan_add(lane < NW ? sh.wi[b][lane] : 0), 63);
  }
  __device__ __forceinline__ int block_min(int v) {
    return block_reduce(v, [](int a, int b) { return min(a, b); });
  }
  __device__ __forceinline__ int block_max(int v) {
    return block_reduce(v, [](int a, int b) { return max(a, b); });
  }
  // Sums of a count and a weight over the threads up to this one.
  __device__ __forceinline__ void block_scan(int& n, double& v, int& all_n, double& all_v) {
    const int wv = threadIdx.x >> 6, b = turn;
    turn ^= 1;
    n = scan_add(n);
    v = scan_add(v);
    if ((threadIdx.x & 63) == 63) {
      sh.wi[b][wv] = n;
      sh.wd[b][wv] = v;
    }
    __syncthreads();
    const int lane = threadIdx.x & 63, w = uniform(wv);
    const int wn = scan_add(lane < NW ? sh.wi[b][lane] : 0);
    const double wd = scan_add(lane < NW ? sh.wd[b][lane] : 0.0);
    all_n = __builtin_amdgcn_readlane(wn, 63);
    all_v = readlane_f64(wd, 63);
    if (w > 0) {
      n += __builtin_amdgcn_readlane(wn, w - 1);
      v += readlane_f64(wd, w - 1);
    }
  }
  __device__ __forceinline__ double block_scan(double v, double& all) {
    int n = 0, all_n;
    block_scan(n, v, all_n, all);
    return v;
  }

  // ---- over the row ----

  // f(tile's words, tile) for each of this wave's tiles that `want` names, the next one's loads in flight.
  template <typename P, typename F>
  __device__ __forceinline__ void each_tile(P want, F f) const {
    auto next = [&](int t) {
      while (t < tiles && !want(t)) t += NW;
      return t;
    };
    int tile = tiles, after = next(uniform((int)(threadIdx.x >> 6)));
    Tile<Tin> x;
    do {
      Tile<Tin> y;
      if (after < tiles) y.load(row, V, after);
      if (tile < tiles) f(x, tile);
      x = y;
      tile = after;
      after = next(after + NW);
    } while (tile < tiles);
  }

  // The same with f(vector, tile, j) for each of their vectors, then done(tile).
  template <typename P, typename F, typename G>
  __device__ __forceinline__ void each_vector(P want, F f, G done) const {
    each_tile(want, [&](const Tile<Tin>& x, int tile) {
      if constexpr (EPV == 8) {
#pragma unroll 1
        for (int j = 0; j < NV; ++j) f(x.vec(j), tile, j);
      } else {  // two at a time: eight words to overlap
#pragma unroll 1
        for (int j = 0; j < NV; j += 2) {
          f(x.vec(j), tile, j);
          f(x.vec(j + 1), tile, j + 1);
        }
      }
      done(tile);
    });
  }

  __device__ __forceinline__ double t2(float z) const { return ((double)z - (double)m) * c; }
  __device__ __forceinline__ double weight(float z) const { return exp2_neg(t2(z)); }
  __device__ __forceinline__ bool kept(float z, int col, float thr, int tie) const {
    return z > thr || (z == thr && col <= tie);
  }

  // ---- a list of words in LDS ----

  // The words of [lo, hi] in `list`, in no order; returns how many there are, or more than it has room for.  As many lanes
  // as a partial maximum is over read their words again, only of those that reach lo; without partial maxima, of every
  // tile that does.
  __device__ __forceinline__ int gather(unsigned long long* list, int room, float lo, float hi) {
    const int tid = threadIdx.x, lane = tid & 63;
    __syncthreads();
    if (tid == 0) sh.n = sh.bin = 0;
    __syncthreads();
    const int wide = 64 / per;  // lanes that read a block
    int blocks = tiles * per;
    if (fine) {
      for (int i = tid; i < blocks; i += NT)
        if (sh.sub[i] >= lo) sh.block[atomicAdd(&sh.bin, 1)] = (uint16_t)i;
      __syncthreads();
      blocks = uniform(sh.bin);
    }
    // this thread's block of round g0: its tile and the lane whose words it reads, or -1
    auto block_at = [&](int g0) {
      const int g = g0 + tid / wide;
      if (g >= blocks) return -1;
      const int b = fine ? sh.block[g] : g;
      return rec.max[b / per] >= lo ? b : -1;
    };
    auto lane_of = [&](int b) { return max(b, 0) % per * wide + tid % wide; };
    Tile<Tin> x, y;
    int block = block_at(0);
    if (__any(block >= 0)) x.load(row, V, max(block, 0) / per, lane_of(block));
    for (int g0 = 0; g0 < blocks; g0 += NT / wide) {
      if (uniform(*(volatile int*)&sh.n) > room) break;
      const int next = block_at(g0 + NT / wide);
      if (__any(next >= 0)) y.load(row, V, max(next, 0) / per, lane_of(next));
      int mine = 0;
      if (block >= 0) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
          for (int e = 0; e < EPV; ++e) mine += x.at(j, e) >= lo && x.at(j, e) <= hi;
      }
      const int incl = scan_add(mine), all = __builtin_amdgcn_readlane(incl, 63);
      if (all > 0) {
        int at = 0;
        if (lane == 0) at = atomicAdd(&sh.n, all);
        at = uniform(at);
        if (at + all > room) break;
        at += incl - mine;
        if (mine > 0) {
          const int tile = block / per, own = lane_of(block);
#pragma unroll
          for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < EPV; ++e) {
              const float z = x.at(j, e);
              if (z >= lo && z <= hi)
                list[at++] = ((unsigned long long)order_key(z) << 32) | (uint32_t)~Tile<Tin>::col(tile, j, e, own);
            }
        }
      }
      x = y;
      block = next;
    }
    __syncthreads();
    return uniform(sh.n);
  }

  __device__ __forceinline__ static float word_of(unsigned long long key) { return key_value((uint32_t)(key >> 32)); }
  __device__ __forceinline__ static int index_of(unsigned long long key) { return (int)~(uint32_t)key; }

  // `to` = the n <= kSorted keys of `from`, all different, largest first; by_index: by the index alone, lowest first.  A
  // key's place is the number of larger ones, which kEach threads count.
  template <bool BY_INDEX>
  __device__ __forceinline__ void sort_words(const unsigned long long* from, unsigned long long* to, int n) const {
    constexpr int kEach = NT / kSorted;
    const int tid = threadIdx.x, i = tid / kEach;
    const unsigned long long mine = i < n ? from[i] : 0ull;
    int place = 0;
    if (i < n)
      for (int q = tid % kEach; q < n; q += kEach)
        place += BY_INDEX ? (uint32_t)from[q] > (uint32_t)mine : from[q] > mine;
#pragma unroll
    for (int o = 1; o < kEach; o <<= 1) place += __shfl_xor(place, o, 64);
    if (i < n && tid % kEach == 0) to[place] = mine;
    __syncthreads();
  }

  // sh.h.cum = the prefix sums of the n sorted words' weights, from `base` on.
  __device__ __forceinline__ void scan_sorted(int n, double base) {
    const int tid = threadIdx.x;
    double total;
    const double v = block_scan(tid < n ? weight(word_of(sh.h.sorted[tid])) : 0.0, total);
    if (tid < n) sh.h.cum[tid] = base + v;
    __syncthreads();
  }

  // The least r >= 1 with cum[r - 1] >= target, or n.
  __device__ __forceinline__ int first_reaching(int n, double target) {
    const int tid = threadIdx.x;
    return block_min(tid < n && sh.h.cum[tid] >= target ? tid + 1 : n);
  }

  // ---- one value's words ----

  // Wave 0: the tile's r-th word (from 1) that equals z, by index.
  __device__ __forceinline__ int nth_equal(int tile, float z, int r) const {
    int found = 0;
    Tile<Tin> x;
    x.load(row, V, tile);
#pragma unroll 1
    for (int j = 0; j < NV; ++j) {
      const u32x4 v = x.vec(j);
      int n = 0;
#pragma unroll
      for (int e = 0; e < EPV; ++e) n += elem<Tin>(v, e) == z;
      const int incl = scan_add(n);
      const int all = __builtin_amdgcn_readlane(incl, 63);
      if (r >= 1 && r <= all) {
        const int l = __ffsll((unsigned long long)__ballot(incl >= r)) - 1;
        int left = r - (incl - n), col = 0;
#pragma unroll
        for (int e = 0; e < EPV; ++e) {
          const bool same = elem<Tin>(v, e) == z;
          left -= same;
          if (left == 0 && same) col = Tile<Tin>::col(tile, j, e);
        }
        found = __builtin_amdgcn_readlane(col, l);
      }
      r -= all;
    }
    return found;
  }

  // rec.count = each tile's words that equal z.
  __device__ __forceinline__ void count_equal(float z) const {
    for (int i = threadIdx.x; i < tiles; i += NT)
      if (!(rec.max[i] >= z)) rec.count[i] = 0;
    int n = 0;
    each_vector([&](int tile) { return rec.max[tile] >= z; },
                [&](const u32x4& v, int, int) {
#pragma unroll
                  for (int e = 0; e < EPV; ++e) n += __popcll(__ballot(elem<Tin>(v, e) == z));
                },
                [&](int tile) {
                  if ((threadIdx.x & 63) == 0) rec.count[tile] = n;
                  n = 0;
                });
    __syncthreads();
  }

  // The index of the r-th word of the row that equals z, from rec.count; rec.count then holds the tiles' words among
  // the first r.
  __device__ __forceinline__ int tie_index(float z, int r) const {
    const int lane = threadIdx.x;
    if (lane < 64) {
      int left = r, at = -1, at_left = 0;
      for (int i0 = 0; i0 < tiles; i0 += 64) {
        const int n = i0 + lane < tiles ? rec.count[i0 + lane] : 0;
        const int incl = scan_add(n);
        const uint64_t mask = __ballot(incl >= left);
        if (at < 0 && mask) {
          const int l = __ffsll((unsigned long long)mask) - 1;
          at_left = left - __builtin_amdgcn_readlane(incl - n, l);
          at = i0 + l;
        }
        if (i0 + lane < tiles) rec.count[i0 + lane] = max(0, min(n, left - (incl - n)));
        left -= __builtin_amdgcn_readlane(incl, 63);
      }
      const int col = at < 0 ? V : nth_equal(at, z, at_left);
      if (lane == 0) sh.i0 = col;
    }
    __syncthreads();
    const int col = uniform(sh.i0);
    __syncthreads();
    return col;
  }

  // ---- histograms of weight ----

  static constexpr double kPerOctave = kBins / 32;
  // How many 1/kPerOctave of an octave (a power of two of weight) a word lies below the maximum.
  __device__ __forceinline__ double steps(float z) const { return ((double)m - (double)z) * (c * kPerOctave); }
  __device__ __forceinline__ int bin_of(float z) const { return (int)fmin(steps(z), (double)(kBins - 1)); }

  // A bin's weights are summed in 64 bits, in each copy half the row's words at most (lanes of one parity): 2^21 of weight
  // 1 in 2^-42 are 2^63.  Rounding to 2^-42 is off by 1.2e-13 of a word's weight at most (2^-43 of 2^(-1/32)).
  static constexpr int kUnitBits = Shape::kUnitBits;
  static_assert((uint64_t)(Shape::kMaxWords / kCols) <= 1ull << (63 - kUnitBits), "a bin that holds all words");
  static constexpr double kOver = (double)(1ull << (52 - kUnitBits));  // kOver + w: w in the low bits, in 2^-kUnitBits

  // The low bits of y in [1, 2) or [kOver, 2 kOver).
  __device__ __forceinline__ static unsigned long long fixed(double y) {
    return __builtin_bit_cast(unsigned long long, y) & 0xfffffffffffffull;
  }

  // The words of [lo, hi], of the row or of its list (listed >= 0), counted and weighed by bins of 1/kPerOctave octave of
  // weight (TOP), or by the bits of their keys below `top`, `shift` bits to a bin; into sh.h.bin_count and bin_mass.
  // Weights are added relative to the bin's top.  The last bin by weight, which has no lower end and may hold most of a
  // row, is added up in registers.
  template <bool TOP>
  __device__ __forceinline__ void histogram(int listed, float lo, float hi, uint32_t top, int shift) {
    const int tid = threadIdx.x, copy = tid & (kCols - 1);
    __syncthreads();
    for (int i = tid; i < kBins * kCols; i += NT) {
      sh.h.mass[i] = 0ull;
      sh.h.count[i] = 0u;
    }
    __syncthreads();
    const double t_top = TOP ? 0.0 : t2(key_value(top));
    int rest = 0;
    double rest_mass = 0.0;
    auto add = [&](float z) {
      int b;
      double y;
      if constexpr (TOP) {
        const double q = steps(z);
        b = (int)fmin(q, (double)(kBins - 1));
        const double x = q - (double)b;
        if constexpr (kBins == 1024) {  // 2^(-x / 32) for the rest x, by its interpolant of degree 5: off by 1.2e-16
          y = fma(x, -3.930921700473334e-11, 9.172082236776783e-09);
          y = fma(x, y, -1.6938507235263203e-06);
          y = fma(x, y, 0.00023459619814393515);
          y = fma(x, y, -0.021660849392493294);
          y = fma(x, y, 1.0 + kOver);
        } else {
          y = exp2_neg(x * (-1.0 / kPerOctave)) + kOver;
        }
        if (b == kBins - 1) {
          const double r = exp2_neg(x * (-1.0 / kPerOctave));
          if (listed < 0) {
            ++rest;
            rest_mass += r;
            return;
          }
          y = r + kOver;
        }
      } else {
        b = min((int)((top - order_key(z)) >> shift), kBins - 1);
        y = exp2_neg(fmin(t2(z) - t_top, 0.0)) + kOver;
      }
      atomicAdd(&sh.h.mass[b * kCols + copy], fixed(y));
      atomicAdd(&sh.h.count[b * kCols + copy], 1u);
    };
    if (listed >= 0) {
      for (int i = tid; i < listed; i += NT) {
        const float z = word_of(sh.h.key[i]);
        if (z >= lo && z <= hi) add(z);
      }
    } else {
      each_vector(
          [&](int tile) { return rec.max[tile] >= lo; },
          [&](const u32x4& x, int, int) {
#pragma unroll
            for (int e = 0; e < EPV; ++e) {
              const float z = elem<Tin>(x, e);
              if (z >= lo && (TOP || z <= hi)) add(z);
            }
          },
          [](int) {});
    }
    __syncthreads();
    rest = block_sum(rest);
    rest_mass = block_sum(rest_mass);
    for (int b = tid; b < kBins; b += NT) {
      int count = 0;
      double mass = 0.0;
#pragma unroll
      for (int i = 0; i < kCols; ++i) {
        mass += (double)sh.h.mass[b * kCols + i] * (1.0 / (double)(1ull << kUnitBits));
        count += (int)sh.h.count[b * kCols + i];
      }
      if (TOP && b == kBins - 1) {
        mass += rest_mass;
        count += rest;
      }
      sh.h.bin_mass[b] = mass * exp2_neg(TOP ? (double)b * (-1.0 / kPerOctave) : t_top);
      sh.h.bin_count[b] = count;
    }
    __syncthreads();
  }

  // The first bin up to which count0 (mass0) and the bins' counts (weights) reach the target, or the last one that holds a
  // word; count0 and mass0 then end before it.
  __device__ __forceinline__ int find_bin(bool by_mass, int& count0, double& mass0, int k, double target, int& in_bin) {
    constexpr int kEach = kBins / NT;
    const int tid = threadIdx.x;
    int n = 0, all_n;
    double w = 0.0, all_w;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      n += sh.h.bin_count[tid * kEach + i];
      w += sh.h.bin_mass[tid * kEach + i];
    }
    const int mine = n;
    const double my_w = w;
    block_scan(n, w, all_n, all_w);
    n += count0;
    w += mass0;
    const int first = block_min(mine > 0 && (by_mass ? w >= target : n >= k) ? tid : INT_MAX);
    const int at = first != INT_MAX ? first : block_max(mine > 0 ? tid : -1);
    if (tid == at) {
      n -= mine;
      w -= my_w;
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int b = tid * kEach + i, q = sh.h.bin_count[b];
        if (q == 0) continue;
        sh.bin = b;  // the last one with a word, where rounding leaves the target above them
        sh.i0 = n;
        sh.d0 = w;
        sh.n = q;
        n += q;
        w += sh.h.bin_mass[b];
        if (by_mass ? w >= target : n >= k) break;
      }
    }
    __syncthreads();
    const int b = uniform(sh.bin);
    count0 = uniform(sh.i0);
    mass0 = uniform(sh.d0);
    in_bin = uniform(sh.n);
    __syncthreads();
    return b;
  }

  // The words of [lo, hi] in sh.h.some, and rec.sum = the tiles' weights of the words above hi; returns how many there are
  // (at most kSorted, as the caller knows).  ALL: also `all`, the weight of this thread's live words.
  template <bool ALL>
  __device__ __forceinline__ int gather_and_sum(float lo, float hi, double& all) {
    const bool far = ALL || t2(hi) < -1000.0;
    const float least = ALL ? kLiveMin : lo;
    double s = 0.0;
    __syncthreads();
    if (threadIdx.x == 0) sh.n = 0;
    for (int i = threadIdx.x; i < tiles; i += NT)
      if (!(rec.max[i] >= least)) rec.sum[i] = 0.0;
    __syncthreads();
    each_vector([&](int tile) { return rec.max[tile] >= least; },
                [&](const u32x4& x, int tile, int j) {
#pragma unroll
                  for (int e = 0; e < EPV; ++e) {
                    const float z = elem<Tin>(x, e);
                    const double t = t2(z), w = exp2_neg<false>(far ? fmax(t, -1022.0) : t);
                    const double v = far && t < -1021.0 ? 0.0 : w;
                    if (ALL && z >= kLiveMin) all += v;
                    if (z > hi) s += v;
                    if (z >= lo && z <= hi)
                      sh.h.some[min(atomicAdd(&sh.n, 1), kSorted - 1)] =
                          ((unsigned long long)order_key(z) << 32) | (uint32_t)~Tile<Tin>::col(tile, j, e);
                  }
                },
                [&](int tile) {
                  s = wave_sum_dpp(s);
                  if ((threadIdx.x & 63) == 0) rec.sum[tile] = s;
                  s = 0.0;
                });
    __syncthreads();
    return min(uniform(sh.n), kSorted);
  }

  // A weight w <= 1 in 2^-51, at least one of them if it is not 0: sums of up to 4,096 fit 64 bits, in any order.
  __device__ __forceinline__ static unsigned long long fine_fixed(double w) {
    return max(fixed(fma(w, 0.5, 1.0)), (unsigned long long)(w > 0.0));
  }

  // rec.sum += the weights of the first r sorted words, each in its tile.  The histograms' memory is free by now.
  __device__ __forceinline__ void add_sorted(int r) {
    static_assert(sizeof(sh.h.mass) + sizeof(sh.h.count) + sizeof(sh.h.bin_mass) + sizeof(sh.h.bin_count) >=
                      8 * kMaxTiles, "an integer for each tile");
    const int tid = threadIdx.x;
    unsigned long long* sum = sh.h.mass;
    for (int i = tid; i < tiles; i += NT) sum[i] = 0ull;
    __syncthreads();
    if (tid < r) {
      const unsigned long long key = sh.h.sorted[tid];
      atomicAdd(sum + index_of(key) / Tile<Tin>::kWords, fine_fixed(weight(word_of(key))));
    }
    __syncthreads();
    for (int i = tid; i < tiles; i += NT) rec.sum[i] += (double)sum[i] * 0x1p-51;
    __syncthreads();
  }

  static constexpr uint32_t kMinusZero = 0x7fffffffu;  // the key that no word has: -0 counts as 0

  // The keys, from `least`'s up, that `bin` takes to b0 .. b1; it only falls as the key grows.  Waves 0 and 1 look for one
  // end each, a lane trying one of 64 keys between the ends.
  template <typename F>
  __device__ __forceinline__ void keys_of(int b0, int b1, float least, F bin, uint32_t& klo, uint32_t& khi) {
    if (threadIdx.x < 128) {
      const bool top = uniform((int)(threadIdx.x >> 6));
      uint32_t lo = order_key(least), hi = order_key(m);
      if (top && b0 == 0) lo = ++hi;
      while (lo < hi) {
        const uint32_t step = (hi - lo) / 64 + 1, key = lo + (threadIdx.x & 63) * step;
        const uint64_t mask = __ballot(key >= hi || bin(key_value(key)) <= (top ? b0 - 1 : b1));
        const uint32_t l = mask ? (uint32_t)__ffsll((unsigned long long)mask) - 1 : 64;
        if (l < 64) hi = min(hi, lo + l * step);
        if (l > 0) lo = lo + (l - 1) * step + 1;
      }
      if ((threadIdx.x & 63) == 0) *(top ? &sh.key2 : &sh.key) = top ? lo - 1 : lo;
    }
    __syncthreads();
    klo = (uint32_t)uniform((int)sh.key);
    khi = (uint32_t)uniform((int)sh.key2);
  }

  // ---- a cut by counts alone ----
  // The row's words are counted by fine bins of weight.  Counts say exactly where the k-th word is.  For a weight, the
  // bins' counts times their middles say where the words below the cut, all lighter than it, weigh what is to be left out:
  // within a bin or so, since no heavy word adds to the error.  One pass then gathers these bins' words and sums the ones
  // above them in fp64, and the cut is accepted if the sums confirm that it lies among them.  A count is one 32-bit LDS
  // atomic per word, a histogram's weight a 64-bit one besides, which bounds it (fp32 [500, 32,003], top-p 0.9, two rows on
  // a CU: 6 us and 24 us for that pass; the whole call 62 us and 74 us).

  static constexpr int kFine = 2 * kBins * kCols;  // bins, in the histograms' memory
  __device__ __forceinline__ int fine_of(float z, float cf) const {
    return (int)fminf((m - z) * cf, (float)(kFine - 1));
  }

  // The last bin, without a lower end, is not counted.
  __device__ __forceinline__ void count_fine(float cf) {
    uint32_t* bins = reinterpret_cast<uint32_t*>(sh.h.mass);
    __syncthreads();
    for (int i = threadIdx.x; i < kFine; i += NT) bins[i] = 0u;
    __syncthreads();
    each_vector([&](int tile) { return rec.max[tile] >= kLiveMin; },
                [&](const u32x4& x, int, int) {
#pragma unroll
                  for (int e = 0; e < EPV; ++e) {
                    const float z = elem<Tin>(x, e);
                    const int b = fine_of(z, cf);
                    if (z >= kLiveMin && b < kFine - 1) atomicAdd(bins + b, 1u);
                  }
                },
                [](int) {});
    __syncthreads();
  }

  // The bins b0 .. b1 that hold the k-th word, or the word with the share `out` of the weight S (0: of `whole`) below it among
  // the words that weigh `whole` by the middles of their bins (0: all of them); the words before them and in them.  By k,
  // `whole` comes back as what the first k words weigh.  False where the cut is below the counted bins or too many words
  // are in these.
  __device__ __forceinline__ bool find_fine(bool by_mass, int k, double out, double S, double octave, double& whole, int& b0,
                                            int& b1, int& before, int& cnt) {
    constexpr int kEach = kFine / NT;
    const uint32_t* bins = reinterpret_cast<const uint32_t*>(sh.h.mass);
    const int tid = threadIdx.x;
    const double w0 = exp2_neg((tid * kEach + 0.5) * -octave), step = exp2_neg(-octave);
    int n = 0, all_n;
    double e = 0.0, all_e, w = w0;
#pragma unroll
    for (int i = 0; i < kEach; ++i, w *= step) {
      const int q = (int)bins[tid * kEach + i];
      n += q;
      e += q * w;
    }
    const int mine = n;
    const double my_e = e;
    block_scan(n, e, all_n, all_e);
    const double among = whole > 0.0 ? whole : all_e, target = among - out * (S > 0.0 ? S : among);
    const int at = block_min(mine > 0 && (by_mass ? e >= target : n >= k) ? tid : INT_MAX);
    if (at == INT_MAX) return false;
    if (tid == at) {
      n -= mine;
      e -= my_e;
      w = w0;
#pragma unroll 1
      for (int i = 0; i < kEach; ++i, w *= step) {
        const int q = (int)bins[tid * kEach + i];
        if (q == 0) continue;
        sh.bin = tid * kEach + i;
        sh.i0 = n;
        sh.d0 = by_mass ? (target - e) / (q * w) : e + (k - n) * w;  // how far into the bin; the first k words' weight
        n += q;
        e += q * w;
        if (by_mass ? e >= target : n >= k) break;
      }
    }
    __syncthreads();
    const double d = uniform(sh.d0);
    b0 = b1 = uniform(sh.bin);
    before = uniform(sh.i0);
    cnt = (int)bins[b0];
    if (!by_mass) whole = d;
    if (by_mass && d < 0.25 && b0 > 0) {
      const int q = (int)bins[--b0];
      before -= q;
      cnt += q;
    }
    if (by_mass && d > 0.75) cnt += (int)bins[min(++b1, kFine - 1)];
    cnt = uniform(cnt);
    before = uniform(before);
    return b1 < kFine - 1 && cnt <= kSorted;
  }

  // The cut after k words, and among these (k_on; else all words, which weigh about S, 0 where that is not known) after
  // the share p of their weight; `least` is the row's least live word.  sums: rec.sum = the tiles' kept weights.  False
  // where counts do not find it.
  __device__ __forceinline__ bool fine_cut(float least, bool k_on, int k, bool p_on, double p, double S, bool exact, bool sums,
                                           Cut& cut) {
    // A count may end anywhere: the bins go down to the row's least live word.  Words lighter than 2^-32 of the first are
    // not what a share depends on.
    const double down = -t2(least) + 0.01, octave = (k_on ? down : fmin(down, 32.0)) / (kFine - 2);  // of a bin
    const float cf = (float)(c / octave);
    double whole = 0.0, Sk = S;
    int r = 0;
    count_fine(cf);
#pragma unroll 1
    for (int by_mass = !k_on; by_mass <= (int)p_on; ++by_mass) {
      int b0, b1, before, cnt;
      if (!find_fine(by_mass, k, 1.0 - p, Sk, octave, whole, b0, b1, before, cnt)) return false;
      uint32_t klo, khi;
      keys_of(b0, b1, kLiveMin, [&](float z) { return fine_of(z, cf); }, klo, khi);
      khi -= khi == kMinusZero;
      const float lo = key_value(klo), hi = key_value(khi);
      const bool total = by_mass && !k_on && !exact;
      double all = 0.0;
      const int n = total ? gather_and_sum<true>(lo, hi, all) : gather_and_sum<false>(lo, hi, all);
      if (total) Sk = block_sum(all);
      const double above = tile_sum(), target = p * Sk;
      sort_words<false>(sh.h.some, sh.h.sorted, n);
      scan_sorted(n, above);
      if (by_mass) {
        if (before > 0 && !(above < target)) return false;
        r = first_reaching(n, target);
        if (!(uniform(sh.h.cum[r - 1]) >= target)) return false;
      } else {
        r = k - before;
      }
      const unsigned long long last = sh.h.sorted[r - 1];
      cut.thr = uniform(word_of(last));
      cut.tie = uniform(index_of(last));
      cut.mass = Sk = uniform(sh.h.cum[r - 1]);
      cut.count = before + r;
      __syncthreads();
    }
    if (sums) add_sorted(r);
    return true;
  }

  // The cut after the k-th word, or after the shortest prefix of weight `target`, among the words from x_lo up (all in the
  // list where listed >= 0), whose histogram<true> is made.  `sums`: rec.sum is wanted too, and true comes back in it where
  // it holds the tiles' kept weights.
  __device__ __forceinline__ Cut select(int listed, bool by_mass, int k, double target, bool& sums) {
    int count0 = 0, cnt;
    double mass0 = 0.0;
    const bool want = sums && listed < 0;
    sums = false;
    const int b = find_bin(by_mass, count0, mass0, k, target, cnt);
    uint32_t klo, khi;
    keys_of(b, b, x_lo, [&](float z) { return bin_of(z); }, klo, khi);
    while (cnt > kSorted && klo < khi) {
      const int bits = 32 - __clz((int)(khi - klo));
      constexpr int kBinBits = 31 - __builtin_clz(kBins);
      const int shift = max(0, bits - kBinBits);
      histogram<false>(listed, key_value(klo), key_value(khi), khi, shift);
      const int q = find_bin(by_mass, count0, mass0, k, target, cnt);
      khi -= (uint32_t)q << shift;
      klo = max(klo, khi - ((1u << shift) - 1));
      khi -= khi == kMinusZero;  // as a bound it would let the zeros in
    }
    Cut cut;
    const float lo = key_value(klo), hi = key_value(khi);
    if (cnt > kSorted) {  // one value
      cut.thr = lo;
      const double w = weight(lo);
      int r = cnt;
      if (!by_mass) r = k - count0;
      else if (w > 0.0) r = (int)fmin(ceil((target - mass0) / w), (double)cnt);
      r = max(1, min(r, cnt));
      cut.mass = mass0 + (double)r * w;
      cut.count = count0 + r;
      cut.tie = V;
      if (r < cnt) {
        count_equal(lo);
        cut.tie = tie_index(lo, r);
      }
      return cut;
    }
    int n;
    if (listed >= 0) {
      const int tid = threadIdx.x;
      if (tid == 0) sh.n = 0;
      __syncthreads();
      for (int i = tid; i < listed; i += NT) {
        const unsigned long long key = sh.h.key[i];
        const float z = word_of(key);
        if (z >= lo && z <= hi) sh.h.some[min(atomicAdd(&sh.n, 1), kSorted - 1)] = key;
      }
      __syncthreads();
      n = min(uniform(sh.n), kSorted);
    } else if (want) {
      double none = 0.0;
      n = gather_and_sum<false>(lo, hi, none);
    } else {
      n = gather(sh.h.some, kSorted, lo, hi);
    }
    sort_words<false>(sh.h.some, sh.h.sorted, n);
    scan_sorted(n, mass0);
    const int r = by_mass ? first_reaching(n, target) : max(1, min(k - count0, n));
    const unsigned long long last = sh.h.sorted[r - 1];
    cut.thr = uniform(word_of(last));
    cut.tie = uniform(index_of(last));
    cut.mass = uniform(sh.h.cum[r - 1]);
    cut.count = count0 + r;
    __syncthreads();
    if (want) {
      add_sorted(r);
      sums = true;
    }
    return cut;
  }

  // rec.sum = the tiles' kept weights, all kept words in the list; their sum and number.  Added as integers.
  __device__ __forceinline__ double list_sums(int listed, float thr, int tie, int& n) {
    const int tid = threadIdx.x;
    unsigned long long* sum = reinterpret_cast<unsigned long long*>(rec.sum);
    for (int i = tid; i < tiles; i += NT) sum[i] = 0ull;
    __syncthreads();
    int here = 0;
    for (int i = tid; i < listed; i += NT) {
      const unsigned long long key = sh.h.key[i];
      const float z = word_of(key);
      const int col = index_of(key);
      if (kept(z, col, thr, tie)) {
        atomicAdd(sum + col / Tile<Tin>::kWords, fine_fixed(weight(z)));
        ++here;
      }
    }
    __syncthreads();
    double s = 0.0;
    for (int i = tid; i < tiles; i += NT) {
      const double v = (double)sum[i] * 0x1p-51;
      rec.sum[i] = v;
      s += v;
    }
    n = block_sum(here);
    return block_sum(s);
  }

  // The sum of rec.sum.
  __device__ __forceinline__ double tile_sum() {
    double sum = 0.0;
    for (int i = threadIdx.x; i < tiles; i += NT) sum += rec.sum[i];
    return block_sum(sum);
  }

  // rec.sum = the tiles' kept weights; their sum, and the number of kept words.  In a tile before the last kept one's all
  // words that equal the threshold are kept, after it none; in its own they are added by their index.
  __device__ __forceinline__ double kept_sums(float thr, int tie, int& n) {
    const int tie_tile = tie < 0 ? -1 : tie / Tile<Tin>::kWords;
    const float above = nextafterf(thr, INFINITY);
    const double w_thr = weight(thr);
    const bool far = t2(thr) < -1000.0;
    int here = 0;
    double s = 0.0;
    for (int i = threadIdx.x; i < tiles; i += NT)
      if (!(rec.max[i] >= thr)) rec.sum[i] = 0.0;
    each_vector([&](int tile) { return rec.max[tile] >= thr; },
                [&](const u32x4& x, int tile, int j) {
                  const float least = tile < tie_tile ? thr : above;
#pragma unroll
                  for (int e = 0; e < EPV; ++e) {
                    const float z = elem<Tin>(x, e);
                    if (z >= least) {
                      const double t = t2(z), w = exp2_neg<false>(far ? fmax(t, -1022.0) : t);
                      s += far && t < -1021.0 ? 0.0 : w;
                      ++here;
                    }
                  }
                  if (tile == tie_tile) {
#pragma unroll
                    for (int e = 0; e < EPV; ++e)
                      if (elem<Tin>(x, e) == thr && Tile<Tin>::col(tile, j, e) <= tie) {
                        s += w_thr;
                        ++here;
                      }
                  }
                },
                [&](int tile) {
                  s = wave_sum_dpp(s);
                  if ((threadIdx.x & 63) == 0) rec.sum[tile] = s;
                  s = 0.0;
                });
    __syncthreads();
    n = block_sum(here);
    return tile_sum();
  }

  // ---- the count of bf16 values ----

  // f(word) for the words of bin kMid among a tile's: 1 in 80,000 of normal logits.
  template <typename F>
  __device__ __forceinline__ void each_mid(const Tile<Tin>& x, u16x2 least, F f) const {
    if (!__any(least.x == 0 || least.y == 0)) return;
#pragma unroll 1
    for (int j = 0; j < NV; ++j) {
      const u32x4 v = x.vec(j);
#pragma unroll
      for (int e = 0; e < EPV; ++e)
        if (fabsf(elem<Tin>(v, e)) < bin_value(kMid + 1)) f(elem<Tin>(v, e));
    }
  }

  __device__ __forceinline__ void clear_values() const {
    for (int i = threadIdx.x; i < kValues; i += NT) sh.v.count[i] = 0u;
    if (threadIdx.x == 0) sh.v.mid = 0ull;
    __syncthreads();
  }

  // A tile's words added to the counts of values.
  __device__ __forceinline__ void count_values(const Tile<Tin>& x) const {
    u16x2 least = (u16x2)(unsigned short)1;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const s16x2 b = value_bins(x.v[j][q], least);
        atomicAdd(&sh.v.count[kMid + b.x], 1u);
        atomicAdd(&sh.v.count[kMid + b.y], 1u);
      }
    each_mid(x, least, [&](float z) {
      const double y = exp2_neg(((double)z - (double)bin_value(kMid + 1)) * c) + 256.0;
      atomicAdd(&sh.v.mid, __builtin_bit_cast(unsigned long long, y) & 0xfffffffffffffull);
    });
  }

  struct ValueCut {
    float thr;
    int n, r, of;  // kept words; of the `of` words that equal thr the first r (r = of = 0: all)
    double S;
  };

  // The row's cut from the counts of values.  False where it falls among the words of bin kMid, which are not told apart, or
  // where these are too many for their sum or too light for its unit.
  __device__ __forceinline__ bool cut_values(bool k_on, int k, bool p_on, double p, float z_min, ValueCut& out) {
    constexpr int kEach = (kValues + NT - 1) / NT;
    const int tid = threadIdx.x;
    const double mid_top = t2(bin_value(kMid + 1));
    // each thread kEach bins, from the largest value down; the last one holds the masked words
    double mid = 0.0;
    // Without words of bin kMid the maximum may lie far below them, and their weight beyond the range of exp2_neg.  With one,
    // the maximum is above -2^-15: 2^89 at most, which exp2_neg forms as well.
    if (const int n_mid = uniform((int)sh.v.count[kMid])) {
      const double unit = 0x1p-44 * exp2_neg(mid_top);
      mid = (double)sh.v.mid * unit;
      // Each is off by half a unit, which below a temperature of 2e-5 may be as much as such a word weighs; the kept words'
      // sum is at least 1, and at least `mid` where they are kept.
      if (n_mid >= kMidWords || n_mid * (0.5 * unit) > 0x1p-43 * fmax(1.0, mid)) return false;
    }
    auto bin_at = [&](int i) { return kValues - 1 - (tid * kEach + i); };
    int q[kEach], my_n = 0;
    double w[kEach], my_m = 0.0;  // counts, weights of the bins
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int b = bin_at(i);
      q[i] = b >= 1 ? (int)sh.v.count[b] : 0;
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int b = bin_at(i);
      w[i] = 0.0;
      if (b >= 0) {
        const double one = q[i] > 0 && b != kMid ? weight(bin_value(b)) : 0.0;
        sh.v.weight[b] = one;
        w[i] = b == kMid ? mid : (double)q[i] * one;
      }
      my_n += q[i];
      my_m += w[i];
    }
    int cn = my_n, all_n;
    double cm = my_m, all_m;
    block_scan(cn, cm, all_n, all_m);
    const int n0 = cn - my_n;
    const double m0 = cm - my_m;
    // the first bin up to which the counts (weights) reach the target
    auto find = [&](bool by_mass, int k_, double target, int& count0, double& mass0, int& have) {
      const int first = block_min(my_n > 0 && (by_mass ? m0 + my_m >= target : n0 + my_n >= k_) ? tid : INT_MAX);
      if (first == INT_MAX) return -1;
      if (tid == first) {
        int a = n0;
        double v = m0;
        bool over = false;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
          if (q[i] > 0 && !over) {
            sh.bin = bin_at(i);  // the last one with a word, where the sum in another order does not reach
            sh.i0 = a;
            sh.d0 = v;
            sh.n = q[i];
            a += q[i];
            v += w[i];
            over = by_mass ? v >= target : a >= k_;
          }
        }
      }
      __syncthreads();
      count0 = uniform(sh.i0);
      mass0 = uniform(sh.d0);
      have = uniform(sh.n);
      const int b = uniform(sh.bin);
      __syncthreads();
      return b;
    };
    int n = all_n;
    double S = all_m;
    float thr = kLiveMin;
    int r = 0, cnt = 0;  // of the cut's value, r words of cnt are kept (0: all)
#pragma unroll 1
    for (int by_mass = 0; by_mass < 2; ++by_mass) {
      if (by_mass ? !p_on : !(k_on && k < all_n)) continue;
      const double target = p * S;
      int count0, have;
      double mass0;
      const int b = find(by_mass, k, target, count0, mass0, have);
      if (b == kMid) return false;
      if (b < 0) continue;  // rounding left the target above all words
      const double one = uniform(sh.v.weight[b]);
      int need = k - count0;
      if (by_mass) need = one > 0.0 ? max(1, (int)fmin(ceil((target - mass0) / one), (double)have)) : have;
      if (count0 + need >= n) continue;
      thr = bin_value(b);
      cnt = have;
      r = need;
      n = count0 + need;
      S = mass0 + (double)need * one;
    }
    if (z_min > thr) {
      if (fabsf(z_min) < bin_value(kMid + 1)) return false;
      int qn = 0;
      double qm = 0.0;
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int b = bin_at(i);
        if (b >= 1 && bin_value(b) >= z_min) {
          qn += q[i];
          qm += w[i];
        }
      }
      n = block_sum(qn);
      S = block_sum(qm);
      thr = z_min;
      cnt = r = 0;
    }
    out = ValueCut{thr, n, r, cnt, S};
    __syncthreads();
    return true;
  }

  // The last kept index of the cut's value.
  __device__ __forceinline__ int value_tie(const ValueCut& cut) const {
    if (cut.r >= cut.of) return V;
    count_equal(cut.thr);
    return tie_index(cut.thr, cut.r);
  }

  // rec.sum = the tiles' kept weights, from the table that cut_values leaves; the last kept index of the cut's value.
  __device__ __forceinline__ int value_sums(const ValueCut& cut) const {
    const int tid = threadIdx.x, lane = tid & 63;
    const float thr = cut.thr;
    const bool partial = cut.r < cut.of;
    // 0 below the cut; the cut's own value apart where it is kept in part
    const double w_thr = weight(thr);
    for (int b = tid; b < kValues; b += NT) {
      if ((b < 1 || (b != kMid && !(partial ? bin_value(b) > thr : bin_value(b) >= thr)))) sh.v.weight[b] = 0.0;
    }
    const bool mid_kept = 0.f >= thr;
    __syncthreads();
    for (int i = tid; i < tiles; i += NT)
      if (!(rec.max[i] >= thr)) {
        rec.sum[i] = 0.0;
        rec.count[i] = 0;
      }
    // words below the cut all read one place, the bin below it: no bank has to answer twice for them
    const int at = thr > -kLimit ? bin_index(thr) : 1 - kMid;
    const s16x2 floor2 = (s16x2)(short)(at - 1), at2 = (s16x2)(short)at;
    each_tile([&](int tile) { return rec.max[tile] >= thr; },
              [&](const Tile<Tin>& x, int tile) {
                double s = 0.0;
                u16x2 least = (u16x2)(unsigned short)1, other = (u16x2)(unsigned short)0;
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                  for (int q = 0; q < 4; ++q) {
                    s16x2 b = value_bins(x.v[j][q], least);
                    if (partial)
                      other += __builtin_elementwise_min(__builtin_bit_cast(u16x2, b ^ at2), (u16x2)(unsigned short)1);
                    b = __builtin_elementwise_max(b, floor2);
                    s += sh.v.weight[kMid + b.x];
                    s += sh.v.weight[kMid + b.y];
                  }
                if (mid_kept) each_mid(x, least, [&](float z) { s += weight(z); });
                s = wave_sum_dpp(s);
                const int same = __builtin_amdgcn_readlane(scan_add(EPV * NV - (int)other.x - (int)other.y), 63);
                if (lane == 0) {
                  rec.sum[tile] = s;
                  rec.count[tile] = same;
                }
              });
    __syncthreads();
    int tie = V;
    if (partial) {
      tie = tie_index(thr, cut.r);
      for (int i = tid; i < tiles; i += NT) rec.sum[i] += (double)rec.count[i] * w_thr;
      __syncthreads();
    }
    return tie;
  }

  // ---- draws ----

  // The same among the first n sorted words.
  __device__ __forceinline__ int draw_sorted(int n, double target) {
    const int tid = threadIdx.x;
    sort_words<true>(sh.h.sorted, sh.h.some, n);
    const double v = tid < n ? weight(word_of(sh.h.some[tid])) : 0.0;
    double all;
    const double incl = block_scan(v, all);
    int at = block_min(v > 0.0 && incl > target ? tid : INT_MAX);
    if (at == INT_MAX) at = block_max(v > 0.0 ? tid : 0);
    return uniform(index_of(sh.h.some[at]));
  }

  // The first kept word at which the kept weights pass `target`, from the tiles' sums in rec.sum: its tile, then its
  // words, a few to a thread; the last kept word where rounding leaves none.
  __device__ __forceinline__ int draw(double target, float thr, int tie) {
    constexpr int kEach = (Tile<Tin>::kWords + NT - 1) / NT;
    const int tid = threadIdx.x;
    double left = target, total;
    int tile = -1, last = -1;
    for (int i0 = 0; i0 < tiles && tile < 0; i0 += NT) {
      const int i = i0 + tid;
      const double v = i < tiles ? rec.sum[i] : 0.0;
      const double incl = block_scan(v, total);
      const int at = block_min(v > 0.0 && incl > left ? i : INT_MAX);
      if (at != INT_MAX) {
        if (i == at) sh.d0 = left - (incl - v);
        __syncthreads();
        left = uniform(sh.d0);
        tile = at;
      } else {
        left -= total;
        last = max(last, block_max(v > 0.0 ? i : -1));
      }
    }
    if (tile < 0) {
      tile = last;
      left = INFINITY;
    }
    const int col0 = tile * Tile<Tin>::kWords + tid * kEach;
    auto word = [&](int e) {
      const int col = col0 + e;
      if (tid * kEach + e >= Tile<Tin>::kWords || col >= V) return 0.0;
      const float z = load_elem(row + col);
      return z >= kLiveMin && kept(z, col, thr, tie) ? weight(z) : 0.0;
    };
    double s = 0.0;
#pragma unroll 4
    for (int e = 0; e < kEach; ++e) s += word(e);
    if (tid == 0) sh.i0 = min(tile * Tile<Tin>::kWords, V - 1);  // a place in the row, whatever the sums
    const double incl = block_scan(s, total);
    int at = block_min(s > 0.0 && incl > left ? tid : INT_MAX);
    if (at == INT_MAX) at = block_max(s > 0.0 ? tid : -1);
    if (tid == at) {
      double run = incl - s;
      int col = col0;
#pragma unroll 1
      for (int e = 0; e < kEach; ++e) {
        const double v = word(e);
        run += v;
        if (v > 0.0) col = col0 + e;  // the last one where the sum in another order does not pass
        if (v > 0.0 && run > left) break;
      }
      sh.i0 = col;
    }
    __syncthreads();
    return uniform(sh.i0);
  }

  // ---- bounds ----

  // A lower bound of the k-th largest of the n partial maxima in sh.sub, and so of the row's k-th word: the upper 16 bits
  // of its key, 8 at a time.
  __device__ __forceinline__ float kth_bound(int n, int k) const {
    const int tid = threadIdx.x;
    uint32_t t = 0;
#pragma unroll 1
    for (int shift = 24; shift >= 16; shift -= 8) {
      for (int i = tid; i < 256; i += NT) sh.radix[i] = 0u;
      __syncthreads();
      for (int i = tid; i < n; i += NT) {
        const uint32_t key = order_key(sh.sub[i]);
        if (shift == 24 || (key ^ t) >> 24 == 0) atomicAdd(&sh.radix[(key >> shift) & 255], 1u);
      }
      __syncthreads();
      if (tid < 64) {  // four bins to a lane, from the largest down
        int q[4], sum = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          q[i] = (int)sh.radix[255 - (tid * 4 + i)];
          sum += q[i];
        }
        int before = scan_add(sum) - sum;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (before < k && before + q[i] >= k) {
            sh.key = t | (uint32_t)(255 - (tid * 4 + i)) << shift;
            sh.i0 = before;
          }
          before += q[i];
        }
      }
      __syncthreads();
      t = (uint32_t)uniform((int)sh.key);
      k -= uniform(sh.i0);
    }
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

// A row's outputs; an action outside the vocabulary has log-prob 0.
__device__ __forceinline__ void write_row(const RowArgs& a, int t, grpo_sampling_row out, bool act_ok, int flag) {
  if (!act_ok) {
    out.logp = 0.f;
    flag |= GRPO_FLAG_ACTION;
  }
  if (a.logp) a.logp[t] = out.logp;
  if (a.n_kept) a.n_kept[t] = out.n_kept;
  if (a.rows) a.rows[t] = out;
  if (a.flags && flag) atomicOr(a.flags, flag);
}

// One workgroup per row.  FUSED: it reduces the row's tiles itself; else their records are there (split_now).  A few words to
// look at: latency, a dozen steps between barriers (bf16 [1, 151,936], k = 50 with p = 0.95: 12.5 us after the tiles' 4.5);
// many: the passes over the row (top-p 0.9: fp32 [500, 32,003] 62 us = 1.0 TB/s, bf16 [256, 151,936] 48 us = 1.6 TB/s; a
// setting per row, log-probs: bf16 [2,000, 151,669] 0.19 ms = 3.1 TB/s).  128 VGPRs, for two rows of 512
// threads to a CU, at the price of 32 to 128 bytes of scratch per lane: 7 to 47 VGPRs, and 85 to 121 SGPRs in others' lanes.
template <typename Tin, bool FUSED, bool DRAW, int NT>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(4, 4))) void k_sample_row(const RowArgs a, int row0) {
  __shared__ RowShared<NT> sh;
  extern __shared__ double tile_mem[];
  typedef RowWork<Tin, NT> Work;
  constexpr int NW = NT / 64;
  const int t = row0 + blockIdx.x, tid = threadIdx.x, lane = tid & 63, wv = uniform(tid >> 6);
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
  constexpr int kMaxSubs = Work::Shape::kMaxSubs, kCap = Work::kCap, kSorted = Work::kSorted, kBins = Work::kBins;
  const int per = FUSED && a.tiles * 64 <= kMaxSubs ? 64 : a.tiles * kSubs <= kMaxSubs ? kSubs : 1;
  const bool fine = a.tiles * per <= kMaxSubs;
  const int subs = fine ? a.tiles * per : 0;
  const RowTiles rec{tile_mem, reinterpret_cast<float*>(tile_mem + a.tiles),
                     reinterpret_cast<int*>(tile_mem + a.tiles) + a.tiles};
  Work w{sh, rec, row, a.V, a.tiles, 0.f, st.c, kLiveMin, per, fine};

  // the tiles' records
  float m = -INFINITY, lo = INFINITY;
  int live = 0;
  bool bad = false;
  const SumMode mode = sum_mode(st, a.V, DRAW, FUSED, Work::kByValue, subs);
  if (FUSED) {
    if constexpr (Work::kByValue) {
      if (mode == kCount) w.clear_values();
    }
    w.each_tile([](int) { return true; },
                [&](const Tile<Tin>& x, int tile) {
                  if constexpr (Work::kByValue) {
                    if (mode == kCount) w.count_values(x);
                  }
                  const TileStats s = tile_stats<Tin>(x, mode, st.c);
                  if (per == 64) sh.sub[tile * 64 + lane] = s.own;
                  else if (per == kSubs && (lane & 7) == 0) sh.sub[tile * kSubs + (lane >> 3)] = s.sub;
                  if (lane == 0) {
                    if (per == 1 && fine) sh.sub[tile] = s.max;
                    rec.sum[tile] = s.sum;
                    rec.max[tile] = s.max;
                  }
                  live += s.live;
                  m = fmaxf(m, s.max);
                  lo = fminf(lo, s.lo);
                  bad |= s.bad;
                });
    if (lane != 0) live = 0;
  } else {
    for (int i = tid; i < a.tiles; i += NT) {
      const TileRec r = a.recs[(int64_t)t * a.tiles + i];
      float mx = r.sub[0];
#pragma unroll
      for (int q = 1; q < kSubs; ++q) mx = fmaxf(mx, r.sub[q]);
      if (per == kSubs) {
#pragma unroll
        for (int q = 0; q < kSubs; ++q) sh.sub[i * kSubs + q] = r.sub[q];
      } else if (fine) {
        sh.sub[i] = mx;
      }
      rec.sum[i] = r.sum;
      rec.max[i] = mx;
      live += r.live;
      m = fmaxf(m, mx);
      lo = fminf(lo, r.lo);
      bad |= r.bad != 0;
    }
  }
  {  // over the workgroup, together
    m = wave_max_dpp(m);
    lo = -wave_max_dpp(-lo);
    live = __builtin_amdgcn_readlane(scan_add(live), 63);
    const bool any_bad = __any(bad);
    if (lane == 0) {
      sh.wf[0][wv] = m;
      sh.wf[1][wv] = lo;
      sh.wi[0][wv] = live;
      sh.wi[1][wv] = any_bad;
    }
    __syncthreads();
    const int q = lane & (NW - 1);
    m = uniform(row16_max(sh.wf[0][q]));
    lo = uniform(-row16_max(-sh.wf[1][q]));
    live = __builtin_amdgcn_readlane(scan_add(lane < NW ? sh.wi[0][lane] : 0), 63);
    bad = __any(sh.wi[1][q] != 0);
    __syncthreads();  // both sets are free again
  }
  w.m = m;

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
    float thr = -1e8f;  // kept: above it
    int tie = -1, n = live;
    double S = 0.0;
    bool drawn = !DRAW;
    if (st.greedy) {
      int first = INT_MAX;
      for (int i = tid; i < a.tiles; i += NT)
        if (rec.max[i] == m) {
          first = i;
          break;
        }
      first = w.block_min(first);
      if (wv == 0) {
        const int col = w.nth_equal(first, m, 1);
        if (lane == 0) sh.i0 = col;
      }
      __syncthreads();
      thr = m;
      tie = uniform(sh.i0);
      n = 1;
      S = 1.0;
      if (DRAW) act = tie;
      drawn = true;
    } else {
      if (mode == kSum64 || mode == kSum32) {  // the tiles' sums relative to the row's maximum
        double total = 0.0;
        for (int i = tid; i < a.tiles; i += NT) {
          const double v = rec.max[i] >= kLiveMin ? rec.sum[i] * w.weight(rec.max[i]) : 0.0;
          rec.sum[i] = v;
          total += v;
        }
        S = w.block_sum(total);
      }
      if (k_on || p_on || m_on) {
        const int k = min(st.k, live);
        const double p = (double)st.p;
        const float z_min = m_on ? fmaxf(w.min_p_bound(log2((double)st.min_p)), kLiveMin) : kLiveMin;
        float x_lo = k_on && p_on ? kLiveMin : z_min;  // top-p of top-k needs the first k words' sum
        if (k_on && k <= subs) x_lo = fmaxf(x_lo, w.kth_bound(subs, k));
        if (p_on && !k_on && mode != kCount) {
          // all words lighter than (1 - p) S / live together weigh less than (1 - p) S; 0.01 covers S's error
          const double l = log2((double)live / ((1.0 - p) * S)) + 0.01;
          const double z = (double)m - l / st.c;
          float zf = fminf((float)z, m);
          if ((double)zf > z) zf = nextafterf(zf, -INFINITY);
          x_lo = fmaxf(x_lo, zf);
        }
        w.x_lo = x_lo;
        int listed = -1;
        if (mode != kCount) listed = x_lo > kLiveMin || live <= kCap ? w.gather(sh.h.key, kCap, x_lo, INFINITY) : live;
        bool cut_known = false;
        if constexpr (Work::kByValue) {
          if ((mode == kCount || listed > kCap) && m < kLimit && lo > -kLimit) {
            if (mode != kCount) {
              w.clear_values();
              w.each_tile([](int) { return true; }, [&](const Tile<Tin>& x, int) { w.count_values(x); });
              __syncthreads();
            }
            typename Work::ValueCut cut;
            cut_known = w.cut_values(k_on, k, p_on, p, z_min, cut);
            if (cut_known) {
              thr = cut.thr;
              n = cut.n;
              S = cut.S;
              if (n - cut.r + cut.of <= kSorted) listed = w.gather(sh.h.key, kCap, thr, INFINITY);
              else if (DRAW) tie = w.value_sums(cut);
              else tie = w.value_tie(cut);
            }
          }
        }
        if (listed > kCap) listed = -1;
        const bool exact = mode == kSum64;  // S
        const double p_lo = exact || k_on ? p : p * (1.0 - kSum32Error), p_hi = exact || k_on ? p : p * (1.0 + kSum32Error);
        if (listed >= 0 && listed <= kSorted) {
          w.template sort_words<false>(sh.h.key, sh.h.sorted, listed);
          if (!cut_known) {
            w.scan_sorted(listed, 0.0);
            n = k_on ? min(k, listed) : listed;
            if (p_on) {
              if (k_on) S = uniform(sh.h.cum[n - 1]);
              int np = w.first_reaching(listed, p_lo * S);
              if (!(uniform(sh.h.cum[np - 1]) >= p_hi * S) && p_lo < p_hi) {
                int all;
                S = w.kept_sums(kLiveMin, a.V, all);
                np = w.first_reaching(listed, p * S);
              }
              n = min(n, np);
            }
            if (m_on) n = min(n, w.block_sum((int)(tid < listed && Work::word_of(sh.h.sorted[tid]) >= z_min)));
            n = max(n, 1);
            S = uniform(sh.h.cum[n - 1]);
          }
          const unsigned long long last_word = sh.h.sorted[n - 1];
          thr = uniform(Work::word_of(last_word));
          tie = uniform(Work::index_of(last_word));
          if (DRAW) {
            act = w.draw_sorted(n, (double)u * S);
            drawn = true;
          }
        } else if (!cut_known) {
          thr = kLiveMin;
          tie = a.V;
          auto narrow = [&](float z, int i) {
            if (z > thr || (z == thr && i < tie)) {
              thr = z;
              tie = i;
            }
          };
          bool summed = false;  // rec.sum holds the tiles' kept weights
          Cut by_counts;
          if ((k_on || p_on) && listed < 0 && w.fine_cut(lo, k_on, k, p_on, p, S, exact, DRAW, by_counts)) {
            narrow(by_counts.thr, by_counts.tie);
            S = by_counts.mass;
            n = by_counts.count;
            summed = DRAW;
          } else if (k_on || p_on) {
            const bool sum_all = p_on && !k_on && !exact && listed < 0;  // S from the histogram: all live words
            if (sum_all) w.x_lo = x_lo = kLiveMin;
            double Sk = S;
            bool sums = false;
#pragma unroll 1
            for (int by_mass = !k_on, again = 0; by_mass <= (int)p_on; ++by_mass) {
              w.template histogram<true>(listed, x_lo, INFINITY, 0u, 0);
              if (sum_all) {
                double q = 0.0;
                for (int i = tid; i < kBins; i += NT) q += sh.h.bin_mass[i];
                Sk = w.block_sum(q);
              }
              const bool sure = sum_all || again;
              sums = DRAW && by_mass == (int)p_on;
              const Cut cut = w.select(listed, by_mass, k, (sure ? p : p_lo) * Sk, sums);
              if (by_mass && !sure && p_lo < p_hi && !(cut.mass >= p_hi * Sk)) {  // S has to be exact: once more
                int all;
                Sk = w.kept_sums(kLiveMin, a.V, all);
                again = 1;
                --by_mass;
                continue;
              }
              narrow(cut.thr, cut.tie);
              Sk = S = cut.mass;
              n = cut.count;
            }
            summed = sums;
          }
          if (m_on && (z_min > thr || !(k_on || p_on))) {
            narrow(z_min, a.V);
            summed = false;
            n = INT_MAX;
          }
          if (listed >= 0 && (DRAW || n == INT_MAX)) S = w.list_sums(listed, thr, tie, n);
          else if (summed) S = w.tile_sum();
          else if (DRAW || n == INT_MAX) S = w.kept_sums(thr, tie, n);
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
    if (DRAW) a.actions_out[t] = out.n_kept > 0 ? act : -1;
    write_row(a, t, out, act_ok, flag);
  }
}

// ---- log-probs of rows with nothing cut -------------------------------------------
// One workgroup to a row, read once: a thread's 32 (bf16) or 16 weights at a time summed in fp32, relative to its running
// maximum, and these sums in fp64.  HBM-bound: bf16 [8,000, 151,936] in 0.50 ms = 4.9 TB/s (the row kernel's own first pass
// takes 0.51 ms for it), fp32 [192, 1,024] in 4.8 us.
template <typename Tin>
__global__ __launch_bounds__(256) void k_tempered_logp(const RowArgs a, int row0) {
  constexpr int NT = 256, NW = NT / 64, EPV = 16 / (int)sizeof(Tin), U = 4;
  typedef typename VecAt<Tin>::type u32x4_any;
  __shared__ float sh_m[NW];
  __shared__ double sh_s[NW];
  __shared__ int sh_n[NW], sh_bad[NW];
  const int t = row0 + blockIdx.x, tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const Tin* row = static_cast<const Tin*>(a.logits) + (int64_t)t * a.ld;
  const int act = a.actions[t], nvec = a.V / EPV;
  const bool act_ok = act >= 0 && act < a.V;
  const float act_z = act_ok ? load_elem(row + act) : 0.f;
  const float tau = a.par.temperature_all;
  const double c = kLog2e64 / (double)tau;
  const float c32 = (float)c;
  float m = kLiveMin;
  double s = 0.0;
  int dead = 0;
  bool nan = false;
  auto raise = [&](float z) {  // the running maximum
    s *= exp2_neg(((double)m - (double)z) * c);
    m = z;
  };
  auto one = [&](float z) {  // a word by itself
    nan |= z != z;
    if (!(z >= kLiveMin)) {
      ++dead;
      return;
    }
    if (z > m) raise(z);
    s += (double)__builtin_amdgcn_exp2f((z - m) * c32);
  };
  for (int base = tid; base < nvec; base += NT * U) {
    u32x4 x[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int v = min(base + i * NT, nvec - 1);
      x[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_any*>(row + (int64_t)v * EPV));
    }
    float hi = -INFINITY, lo = INFINITY;
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int e = 0; e < EPV; e += 2) {
        const float p = elem<Tin>(x[i], e), q = elem<Tin>(x[i], e + 1);
        nan |= __builtin_isunordered(p, q);
        hi = max3f(hi, p, q);
        lo = min3f(lo, p, q);
      }
    const bool whole = base + (U - 1) * NT < nvec;
    if (__all(whole && lo >= kLiveMin)) {
      if (hi > m) raise(hi);
      float some = 0.f;
#pragma unroll
      for (int i = 0; i < U; ++i)
#pragma unroll
        for (int e = 0; e < EPV; ++e) some += __builtin_amdgcn_exp2f((elem<Tin>(x[i], e) - m) * c32);
      s += (double)some;
    } else {
      for (int v = base; v < min(base + U * NT, nvec); v += NT)
        for (int e = 0; e < EPV; ++e) one(load_elem(row + (int64_t)v * EPV + e));
    }
  }
  if (tid < a.V - nvec * EPV) one(load_elem(row + nvec * EPV + tid));
  const float mw = wave_max_dpp(m);
  const double sw = wave_sum_dpp(s * exp2_neg(((double)m - (double)mw) * c));
  dead = __builtin_amdgcn_readlane(scan_add(dead), 63);
  const bool bad = __any(nan) || mw == INFINITY;
  if (lane == 0) {
    sh_m[wv] = mw;
    sh_s[wv] = sw;
    sh_n[wv] = dead;
    sh_bad[wv] = bad;
  }
  __syncthreads();
  if (tid != 0) return;
  float M = sh_m[0];
#pragma unroll
  for (int i = 1; i < NW; ++i) M = fmaxf(M, sh_m[i]);
  double S = 0.0;
  int n = a.V, any_bad = 0;
#pragma unroll
  for (int i = 0; i < NW; ++i) {
    S += sh_s[i] * exp2_neg(((double)sh_m[i] - (double)M) * c);
    n -= sh_n[i];
    any_bad |= sh_bad[i];
  }
  grpo_sampling_row out;
  out.max = M;
  out.temperature = tau;
  out.threshold = n > 0 && !any_bad ? -1e8f : INFINITY;
  out.tie = -1;
  out.n_kept = any_bad ? 0 : n;
  out.sum = any_bad ? (double)NAN : n > 0 ? S : 0.0;
  out.logp = any_bad ? NAN : -INFINITY;
  if (n > 0 && !any_bad && act_ok && act_z >= kLiveMin)
    out.logp = (float)(((double)act_z - (double)M) / (double)tau - log(S));
  write_row(a, t, out, act_ok, any_bad || n == 0 ? GRPO_FLAG_NONFINITE : 0);
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
// the 2 + 2 (bf16) or 4 + 4 bytes per word: bf16 [8,000, 151,936] in 0.82-0.86 ms = 5.7-5.9 TB/s, fp32 [3,001, 32,003], whose rows
// start at any element, in 0.12 ms = 6.6 TB/s (the forward pass left part of it cached).
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

// Whether the tiles may be reduced by a launch of their own, which needs a workspace.
static bool split_rows(int64_t T, int64_t V) { return T > 0 && T < 192 && V > 16384; }

static int tile_count(int64_t V, bool bf16) {
  const int words = bf16 ? Tile<uint16_t>::kWords : Tile<float>::kWords;
  return (int)((V + words - 1) / words);
}

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

constexpr int64_t kRowsPerLaunch = 1 << 20;  // a launch's threads stay below 2^32

template <typename Tin, bool FUSED, bool DRAW, int NT>
static void launch_row_kernel(const RowArgs& a, int64_t T, hipStream_t s) {
  for (int64_t r = 0; r < T; r += kRowsPerLaunch)
    hipLaunchKernelGGL((k_sample_row<Tin, FUSED, DRAW, NT>), dim3((unsigned)std::min(kRowsPerLaunch, T - r)), dim3(NT),
                       row_tile_bytes(a.tiles), s, a, (int)r);
}

// Whether rows go to workgroups of 256 threads, four on a CU, and not to ones of 512 or 1,024.  Up to 16,384 words a small
// top-k is found among the partial maxima that such a workgroup holds, 64 to a tile (us, 256 against 512 threads, bf16, k = 50
// with p = 0.95: V = 2,000 T = 4 12 and 13, T = 3,000 37 and 76; V = 16,384 T = 4 13 and 14, T = 3,000 49 and 85).  A larger k
// is not, and the rule does not look at it: V = 16,384, k = 2,000 T = 4 bf16 30 and 22, fp32 30 and 24, T = 3,000 134 and 140,
// 142 and 184; with p = 0.95 T = 4 44 and 23, 45 and 36, T = 3,000 210 and 149, 221 and 276.  A top-p alone goes
// through more of the row, which few rows do faster with more threads (V = 16,384, T = 200: bf16 35 and 29, fp32 34 and
// 30) and many with more rows at once (T = 3,000: V = 2,048 bf16 56 and 104; V = 8,000 bf16 90 and 127; V = 16,384 fp32
// 118 and 161), but for bf16 rows beyond 8,192 words, whose values the large workgroup counts (126 and 120; T = 600 60 and
// 39).  fp32 [200, 8,000] is on the wrong side of that: 28 and 31.
template <typename Tin>
static bool short_rows(const RowArgs& a, int64_t T) {
  if (a.V > RowShape<256>::kMaxWords) return false;
  if (a.par.top_k || a.par.top_k_all > 0 || a.V <= 2048) return true;
  return T > 512 && (a.V <= 8192 || sizeof(Tin) == 4);
}

// Whether nothing is cut anywhere, which the host sees where no setting is an array.
static bool nothing_cut(const grpo_sampling& p, int V) {
  return !p.temperature && !p.top_k && !p.top_p && !p.min_p && p.temperature_all > 0.f &&
         (p.top_k_all <= 0 || p.top_k_all >= V) && p.top_p_all == 1.f && p.min_p_all == 0.f;
}

// Whether the tiles are reduced by a launch of their own, which spreads a row over the chip but lets the row's workgroup
// see each tile's record alone.  Where nothing is cut that is all it needs (us, two launches against one: V = 17,000
// bf16 T = 1 14 and 15; V = 152,064 T = 1 13 and 38, T = 64 21 and 39, T = 191 36 and 41).  A cut reads the row again:
// two launches pay for the longest of few rows (fp32 top-p: V = 50,000 T = 64 51 and 48; V = 152,064 T = 1 89 and 93,
// T = 191 123 and 110; bf16 k = 50 with p = 0.95: T = 1 17 and 21, T = 128 25 and 24), and not for a bf16 row with a top-p
// alone, which one launch counts by value as it reads it first (T = 1 49 and 43, T = 64 60 and 44).
template <typename Tin>
static bool split_now(const RowArgs& a, int64_t T) {
  const grpo_sampling& p = a.par;
  if (!split_rows(T, a.V)) return false;
  if (nothing_cut(p, a.V)) return true;
  const bool counted = sizeof(Tin) == 2 && (p.top_k || p.top_k_all <= 0) && (p.top_p || p.top_p_all < 1.f);
  return T <= 64 && a.V > 65536 && !counted;
}

template <typename Tin, bool DRAW>
static void launch_rows(const RowArgs& a, int64_t T, hipStream_t s) {
  if (split_now<Tin>(a, T)) {
    const int waves = (int)T * a.tiles;
    hipLaunchKernelGGL(k_sample_tiles<Tin>, dim3((unsigned)(waves + 3) / 4), dim3(256), 0, s, a, waves, DRAW);
    launch_row_kernel<Tin, false, DRAW, 1024>(a, T, s);
  } else if (!DRAW && nothing_cut(a.par, a.V)) {
    for (int64_t r = 0; r < T; r += kRowsPerLaunch)
      hipLaunchKernelGGL(k_tempered_logp<Tin>, dim3((unsigned)std::min(kRowsPerLaunch, T - r)), dim3(256), 0, s, a,
                         (int)r);
  } else if (short_rows<Tin>(a, T)) {
    launch_row_kernel<Tin, true, DRAW, 256>(a, T, s);
  } else if (T <= 256 && (a.V > RowShape<256>::kMaxWords || sizeof(Tin) == 2)) {
    // one row per CU: all its waves for that row (us, 1,024 against 512 threads, top-p alone: V = 8,000 T = 200 bf16 25 and
    // 30, fp32 35 and 32; V = 152,064 T = 191 bf16 48 and 53, fp32 111 and 141; T = 400 bf16 93 and 77, fp32 212 and 194)
    launch_row_kernel<Tin, true, DRAW, 1024>(a, T, s);
  } else {
    launch_row_kernel<Tin, true, DRAW, 512>(a, T, s);
  }
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
  if (split_rows(T, V)) {
    if (!ws || ws_bytes < grpo_sampling_workspace_bytes(T, V)) return GRPO_ERR_WORKSPACE;
    if (!aligned(ws, 16)) return GRPO_ERR_ALIGN;
  }
  if (flags) hipLaunchKernelGGL(k_clear_sampling_flag, dim3(1), dim3(1), 0, s, flags);
  if (T > 0) {
    const RowArgs a{logits, ld,     (int)V, tile_count(V, dtype == GRPO_BF16), *par,  u, actions, actions_out,
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
  return split_rows(T, V) ? align_up(sizeof(TileRec) * (size_t)T * (size_t)tile_count(V, false)) : 0;
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
  if (T > 0 && rows_overlap(logits, dlogits, T, V, ld, esz)) return GRPO_ERR_ARG;
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
