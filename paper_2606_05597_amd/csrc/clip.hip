// The gradients' common norm and their clipping to it (grpo_clip.h).
//
// The tensors lie one behind the other in units of kUnit elements; a workgroup takes units `gridDim.x` apart and finds
// each one's tensor by its first unit in the table, so that the launch is the same for one large tensor and for many
// small ones.  Memory-bound: 4 (fp32) or 2 bytes are read per element for the norm, and read again and written for the
// clipping.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>
#include <new>

#include "device.h"
#include "grpo_clip.h"
#include "host.h"

namespace grpo {

constexpr int kUnit = 8192;  // elements of a unit: 32 per thread, 128 bytes of fp32 in flight
constexpr int kClipNT = 256;

struct GradEntry {
  const void* data;
  void* out;
  int64_t n;
  int64_t unit0;  // its first unit; a tensor without elements has none
  int32_t dtype, out_dtype;
};

// The entry of unit u: the last one whose unit0 is not above it (entries without units share the next one's unit0 and
// come before it).
__device__ __forceinline__ int entry_of(const GradEntry* tab, int lo, int n, int64_t u) {
  int hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (tab[mid].unit0 <= u) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// Addresses read from the table, said to be global memory's (a generic address takes the slower flat path).
#define GRPO_GLOBAL __attribute__((address_space(1)))
typedef const GRPO_GLOBAL float* gf32;
typedef const GRPO_GLOBAL uint16_t* gbf16;
typedef GRPO_GLOBAL float* gf32o;
typedef GRPO_GLOBAL uint16_t* gbf16o;

// Eight elements at any element-aligned address, as fp32.
template <bool STREAM>
__device__ __forceinline__ void load8(gf32 p, float (&x)[8]) {
  const GRPO_GLOBAL u32x4_a4* q = (const GRPO_GLOBAL u32x4_a4*)p;
  const u32x4 a = STREAM ? __builtin_nontemporal_load(q) : q[0], b = STREAM ? __builtin_nontemporal_load(q + 1) : q[1];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[e] = __uint_as_float(a[e]);
    x[4 + e] = __uint_as_float(b[e]);
  }
}
template <bool STREAM>
__device__ __forceinline__ void load8(gbf16 p, float (&x)[8]) {
  const GRPO_GLOBAL u32x4_a2* q = (const GRPO_GLOBAL u32x4_a2*)p;
  const u32x4 a = STREAM ? __builtin_nontemporal_load(q) : *q;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = bf16_lo(a[e]);
    x[2 * e + 1] = bf16_hi(a[e]);
  }
}
__device__ __forceinline__ void store8(gf32o p, const float (&x)[8]) {
  u32x4 a, b;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    a[e] = __float_as_uint(x[e]);
    b[e] = __float_as_uint(x[4 + e]);
  }
  __builtin_nontemporal_store(a, (GRPO_GLOBAL u32x4_a4*)p);
  __builtin_nontemporal_store(b, (GRPO_GLOBAL u32x4_a4*)(p + 4));
  asm volatile("s_nop 1" ::: "memory");  // the stores have read their data before its registers are reused
}
__device__ __forceinline__ void store8(gbf16o p, const float (&x)[8]) {
  u32x4 a;
#pragma unroll
  for (int e = 0; e < 4; ++e) a[e] = pack_bf16(x[2 * e], x[2 * e + 1]);
  __builtin_nontemporal_store(a, (GRPO_GLOBAL u32x4_a2*)p);
  asm volatile("s_nop 1" ::: "memory");
}

__device__ __forceinline__ float load1(gf32 p) { return *p; }
__device__ __forceinline__ float load1(gbf16 p) { return bf16_to_f32(*p); }
__device__ __forceinline__ void store1(gf32o p, float v) { *p = v; }
__device__ __forceinline__ void store1(gbf16o p, float v) { *p = (uint16_t)(pack_bf16(v, 0.f) & 0xffffu); }

constexpr int kVecs = kUnit / kClipNT / 8;  // of 8 elements, to a thread

// Sums one unit's squares: fp32 squares can pass fp32's range at both ends, fp64 ones cannot.
template <typename P>
__device__ __forceinline__ double unit_sumsq(P p, int n) {
  const int tid = threadIdx.x, nv = n / 8;
  float x[kVecs][8];
  double s = 0.0;
  if (n == kUnit) {
#pragma unroll
    for (int q = 0; q < kVecs; ++q) load8<false>(p + (q * kClipNT + tid) * 8, x[q]);
  } else {
#pragma unroll
    for (int q = 0; q < kVecs; ++q) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[q][e] = 0.f;
      if (q * kClipNT + tid < nv) load8<false>(p + (q * kClipNT + tid) * 8, x[q]);
    }
    const float edge = tid < n - nv * 8 ? load1(p + nv * 8 + tid) : 0.f;
    s = (double)edge * (double)edge;
  }
#pragma unroll
  for (int q = 0; q < kVecs; ++q)
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fma((double)x[q][e], (double)x[q][e], s);
  return s;
}

// HBM-bound, or by the memory-side cache where the gradients fit it: 545 M fp32 elements in 0.35 ms = 6.2 TB/s, 60 M in
// 37 us = 6.6 TB/s; 24 small tensors in 3.7 us.
__global__ __launch_bounds__(kClipNT) void k_grad_sumsq(const GradEntry* __restrict__ tab, int n_tab, int64_t units,
                                                        double* __restrict__ partials) {
  __shared__ double sh[kClipNT / 64];
  const int tid = threadIdx.x;
  double s = 0.0;
  int at = 0;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    at = entry_of(tab, at, n_tab, u);
    const GradEntry e = tab[at];
    const int64_t first = (u - e.unit0) * kUnit;
    const int n = (int)min((int64_t)kUnit, e.n - first);
    s += e.dtype == GRPO_F32 ? unit_sumsq((gf32)e.data + first, n) : unit_sumsq((gbf16)e.data + first, n);
  }
  s = wave_sum_dpp(s);
  if ((tid & 63) == 0) sh[tid >> 6] = s;
  __syncthreads();
  if (tid == 0) partials[blockIdx.x] = (sh[0] + sh[1]) + (sh[2] + sh[3]);
  // slots that no workgroup has
  for (unsigned i = gridDim.x + blockIdx.x * kClipNT + tid; i < GRPO_GRAD_PARTIALS; i += gridDim.x * kClipNT)
    partials[i] = 0.0;
}

// A factor f 2^e: e is 0 but for factors near fp32's subnormals, which hold fewer bits than the products do.
struct Factor {
  float f;
  int e;
  __device__ __forceinline__ bool is_one() const { return f == 1.f && e == 0; }
};
__device__ __forceinline__ float operator*(float x, Factor k) { return __builtin_amdgcn_ldexpf(x * k.f, k.e); }
__device__ __forceinline__ Factor factor_of(double f) {
  if (f >= 0x1p-100 || f == 0.0) return Factor{(float)f, 0};
  int e;
  const double r = frexp(f, &e);  // [1/2, 1)
  return Factor{(float)r, e};
}

template <bool STREAM, typename Pi, typename Po>
__device__ __forceinline__ void unit_scale(Pi p, Po o, int n, Factor f) {
  const int tid = threadIdx.x, nv = n / 8;
  float x[kVecs][8];
  if (n == kUnit) {
#pragma unroll
    for (int q = 0; q < kVecs; ++q) load8<STREAM>(p + (q * kClipNT + tid) * 8, x[q]);
#pragma unroll
    for (int q = 0; q < kVecs; ++q) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[q][e] = x[q][e] * f;
      store8(o + (q * kClipNT + tid) * 8, x[q]);
    }
    return;
  }
#pragma unroll
  for (int q = 0; q < kVecs; ++q)
    if (q * kClipNT + tid < nv) load8<STREAM>(p + (q * kClipNT + tid) * 8, x[q]);
  const float edge = tid < n - nv * 8 ? load1(p + nv * 8 + tid) : 0.f;
#pragma unroll
  for (int q = 0; q < kVecs; ++q)
    if (q * kClipNT + tid < nv) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[q][e] = x[q][e] * f;
      store8(o + (q * kClipNT + tid) * 8, x[q]);
    }
  if (tid < n - nv * 8) store1(o + nv * 8 + tid, edge * f);
}

// BIG: more bytes of gradients than the memory-side cache holds.  They are then taken from the last unit back, so that what
// the sum of squares read last is still there, and past the caches otherwise; fewer are read from that cache as they lie.
// Norm and clipping, both ways (us): 545 M elements, fp32 to bf16, 938 so and 955 in order through the caches (the clipping
// 0.58 ms = 5.6 TB/s); in place, 160 MB of fp32 84 and 76, 264 MB 136 and 120, 320 MB 165 and 174, 480 MB 254 and 286; of
// bf16 160 MB 77 and 73, 268 MB 127 and 120, 300 MB 139 and 141, 400 MB 184 and 223.
template <bool BIG>
__global__ __launch_bounds__(kClipNT) void k_grad_clip(const GradEntry* __restrict__ tab, int n_tab, int64_t units,
                                                       bool in_place, const double* __restrict__ partials,
                                                       double max_norm, float* __restrict__ norm_out,
                                                       int32_t* __restrict__ flags) {
  __shared__ double sh[kClipNT / 64];
  const int tid = threadIdx.x;
  double s = 0.0;
#pragma unroll
  for (int i = 0; i < GRPO_GRAD_PARTIALS / kClipNT; ++i) s += partials[i * kClipNT + tid];
  s = wave_sum_dpp(s);
  if ((tid & 63) == 0) sh[tid >> 6] = s;
  __syncthreads();
  const double norm = sqrt((sh[0] + sh[1]) + (sh[2] + sh[3]));
  const bool finite = isfinite(norm);
  const Factor f = factor_of(finite ? fmin(1.0, max_norm / (norm + GRPO_CLIP_EPS)) : 1.0);
  if (blockIdx.x == 0 && tid == 0) {
    if (norm_out) *norm_out = (float)norm;
    if (flags) *flags = finite ? 0 : GRPO_FLAG_NONFINITE;
  }
  if (in_place && f.is_one()) return;
  for (int64_t v = blockIdx.x; v < units; v += gridDim.x) {
    const int64_t u = BIG ? units - 1 - v : v;
    const GradEntry e = tab[entry_of(tab, 0, n_tab, u)];
    const int64_t first = (u - e.unit0) * kUnit;
    const int n = (int)min((int64_t)kUnit, e.n - first);
    if (e.data == e.out && f.is_one()) continue;
    if (e.dtype == GRPO_F32) {
      if (e.out_dtype == GRPO_F32) unit_scale<BIG>((gf32)e.data + first, (gf32o)e.out + first, n, f);
      else unit_scale<BIG>((gf32)e.data + first, (gbf16o)e.out + first, n, f);
    } else {
      if (e.out_dtype == GRPO_F32) unit_scale<BIG>((gbf16)e.data + first, (gf32o)e.out + first, n, f);
      else unit_scale<BIG>((gbf16)e.data + first, (gbf16o)e.out + first, n, f);
    }
  }
}

constexpr int64_t kMaxGrads = 1 << 20;
constexpr int64_t kCacheBytes = 256 << 20;  // the memory-side cache

static unsigned clip_grid(int64_t units) { return (unsigned)std::max<int64_t>(1, std::min<int64_t>(units, GRPO_GRAD_PARTIALS)); }

static int check_layout(const grpo_grad_layout* l, const void* table, const double* partials) {
  if (!l || !partials || l->n < 0 || l->n > kMaxGrads || l->units < 0 || l->units >= ((int64_t)1 << 31) ||
      l->bytes < 0 || (l->n > 0 && !table) || (l->n == 0 && l->units > 0))
    return GRPO_ERR_ARG;
  if (!aligned(table, 8) || !aligned(partials, 8)) return GRPO_ERR_ALIGN;
  return GRPO_OK;
}

}  // namespace grpo

using namespace grpo;

extern "C" size_t grpo_grad_table_bytes(int32_t n) {
  return n < 0 || n > kMaxGrads ? 0 : sizeof(GradEntry) * (size_t)std::max(n, 1);
}

extern "C" int grpo_grad_table(const grpo_grad* grads, int32_t n, void* table, size_t table_bytes,
                               grpo_grad_layout* layout) {
  if (n < 0 || n > kMaxGrads) return GRPO_ERR_SHAPE;
  if (!table || !layout || (n > 0 && !grads)) return GRPO_ERR_ARG;
  if (table_bytes < grpo_grad_table_bytes(n)) return GRPO_ERR_WORKSPACE;
  if (!aligned(table, 8)) return GRPO_ERR_ALIGN;
  // Memory ranges: what is written may meet nothing else, what is only read may overlap.
  struct Range {
    uintptr_t begin, end;
    bool written;
  };
  Range* ranges = new (std::nothrow) Range[2 * (size_t)std::max(n, 1)];
  if (!ranges) return GRPO_ERR_WORKSPACE;
  GradEntry* tab = static_cast<GradEntry*>(table);
  int64_t unit = 0, bytes = 0;
  int32_t in_place = 1;
  size_t nr = 0;
  int st = GRPO_OK;
  for (int32_t i = 0; i < n && st == GRPO_OK; ++i) {
    const grpo_grad& g = grads[i];
    if ((g.dtype != GRPO_F32 && g.dtype != GRPO_BF16) || (g.out_dtype != GRPO_F32 && g.out_dtype != GRPO_BF16)) {
      st = GRPO_ERR_DTYPE;
    } else if (g.n < 0 || g.n >= ((int64_t)1 << 40)) {
      st = GRPO_ERR_SHAPE;
    } else if (g.n > 0 && (!g.data || !g.out || (g.data == g.out && g.dtype != g.out_dtype))) {
      st = GRPO_ERR_ARG;
    } else {
      const size_t a = g.dtype == GRPO_F32 ? 4 : 2, b = g.out_dtype == GRPO_F32 ? 4 : 2;
      if (g.n > 0 && (!aligned(g.data, a) || !aligned(g.out, b))) st = GRPO_ERR_ALIGN;
      tab[i] = GradEntry{g.data, g.out, g.n, unit, g.dtype, g.out_dtype};
      unit += (g.n + kUnit - 1) / kUnit;
      bytes += g.n * (int64_t)a;
      if (unit >= ((int64_t)1 << 31)) st = GRPO_ERR_SHAPE;
      if (g.n > 0) {
        const uintptr_t d = (uintptr_t)g.data, o = (uintptr_t)g.out;
        ranges[nr++] = Range{o, o + (uintptr_t)g.n * b, true};
        if (g.data != g.out) {
          in_place = 0;
          ranges[nr++] = Range{d, d + (uintptr_t)g.n * a, false};
        }
      }
    }
  }
  if (st == GRPO_OK) {
    std::sort(ranges, ranges + nr, [](const Range& x, const Range& y) { return x.begin < y.begin; });
    uintptr_t read_end = 0, write_end = 0;  // the furthest ends so far
    for (size_t i = 0; i < nr; ++i) {
      if (ranges[i].begin < write_end || (ranges[i].written && ranges[i].begin < read_end)) st = GRPO_ERR_SHAPE;
      uintptr_t& end = ranges[i].written ? write_end : read_end;
      end = std::max(end, ranges[i].end);
    }
  }
  delete[] ranges;
  if (st != GRPO_OK) return st;
  layout->n = n;
  layout->in_place = in_place;
  layout->units = unit;
  layout->bytes = bytes;
  return GRPO_OK;
}

extern "C" int grpo_grad_sumsq(const grpo_grad_layout* layout, const void* table, double* partials, hipStream_t s) {
  const int st = check_layout(layout, table, partials);
  if (st != GRPO_OK) return st;
  hipLaunchKernelGGL(k_grad_sumsq, dim3(clip_grid(layout->units)), dim3(kClipNT), 0, s,
                     static_cast<const GradEntry*>(table), layout->n, layout->units, partials);
  return hipGetLastError() == hipSuccess ? GRPO_OK : GRPO_ERR_HIP;
}

extern "C" int grpo_grad_clip(const grpo_grad_layout* layout, const void* table, const double* partials,
                              double max_norm, float* norm_out, int32_t* error_flags, hipStream_t s) {
  const int st = check_layout(layout, table, partials);
  if (st != GRPO_OK) return st;
  if (!(max_norm >= 0.0)) return GRPO_ERR_ARG;
  if (!aligned(norm_out, 4) || !aligned(error_flags, 4)) return GRPO_ERR_ALIGN;
  const auto kernel = layout->bytes > kCacheBytes ? k_grad_clip<true> : k_grad_clip<false>;
  hipLaunchKernelGGL(kernel, dim3(clip_grid(layout->units)), dim3(kClipNT), 0, s, static_cast<const GradEntry*>(table),
                     layout->n, layout->units, layout->in_place != 0, partials, max_norm, norm_out, error_flags);
  return hipGetLastError() == hipSuccess ? GRPO_OK : GRPO_ERR_HIP;
}
