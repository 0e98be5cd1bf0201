// A product with bias, activation and residual in its epilogue, and its gradient (grpo_linear.h).
//
//   y  [M, N] = x W           dx [M, K] = dz W^T          dW [K, N] = x^T dz, or [N, K] = dz^T x
// Few rows go to the kernel below, which is as fast as W can be read; everything else to tiles (linear_tiles.hip), which take
// operands whichever way they lie.  Only where rows are not whole aligned vectors of 16 bytes is an operand copied for the
// tiles.  A product with too few tiles for the chip is split along its sum, the splits' sums are joined by a launch of their
// own.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "gemm.h"
#include "host.h"
#include "linear.h"
#include "overlap.h"

namespace grpo {

// ---- few rows ---------------------------------------------------------------------
// Up to 16 rows, or 32 where W's rows run along the outputs (KN): a product is then as long as reading W once takes.  A wave
// goes down its part of the summed dimension over 128 outputs, W's vectors from memory straight into the operands of
// v_mfma_f32_16x16x32_bf16 (a lane: 8 consecutive k of one column):
//   KN: a lane reads 8 columns of 8 rows of W and turns them in its registers (v_perm), so that fragment c holds its
//     column c;
//   rows of W along the sum: fragment c is of row 8 (lane % 16) + c, of which four lanes read 128 bytes (64 bytes at a time,
//     the other half of each line came from memory again: 271 us instead of 186 at 3,584 x 151,936).
// Either way a lane ends with 8 consecutive outputs.  The waves of a workgroup, each with its part of the sum, are added
// through the LDS in their order.  W's rows may start at any element.
// us by rows (1, 16, 32; 6 TB/s of W: 182 and 38): 3,584 x 151,936 KN 180, 187, 200, else 186, 194; 3,584 x 32,000 41, 41, 43
// and 42, 43.  Tiles take 196 and 45 for 33 rows.
typedef float lin_acc4 __attribute__((ext_vector_type(4)));

struct FewArgs {
  const uint16_t* x;  // [M, K]
  const uint16_t* w;
  int64_t ldx, ldw;
  int M, K, N;
  int strips;     // of 128 outputs
  int splits;     // workgroups that share a strip's sum; > 1: their sums go to part [splits][M][N]
  int wave_k;     // summed over by a wave, a multiple of 64
  float* part;
  Epilogue e;
};

constexpr int kFewWaves = 8, kFewCols = 128;

template <int ACT, bool PART>
__device__ __forceinline__ void few_out(const FewArgs& a, int split, int m, int n, float (&v)[8]) {
  if constexpr (PART) {
    float* o = a.part + ((int64_t)split * a.M + m) * a.N + n;
    if (n + 8 <= a.N) store8(o, 0, false, v);
    else
      for (int q = 0; q < 8; ++q)
        if (n + q < a.N) o[q] = v[q];
  } else {
    float bias[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) bias[q] = a.e.bias && n + q < a.N ? load_any(a.e.bias, n + q, a.e.bias_bf16) : 0.f;
    finish8<ACT>(a.e, m, n, a.N, bias, v);
  }
}

// 8 elements p[0 .. 7], those from `left` on zeros and unread: the last 8 before p + left (which have to be there) moved down.
__device__ __forceinline__ u32x4 load_vec(const uint16_t* p, int left) {
  const int past = 8 - min(left, 8);
  if (past >= 8) return u32x4{0u, 0u, 0u, 0u};
  const u32x4 v = *reinterpret_cast<const u32x4_a2*>(p - past);
  return __builtin_bit_cast(u32x4, __builtin_bit_cast(unsigned __int128, v) >> (16 * past));
}

template <int MB, bool KN, int ACT, bool PART>
__global__ __launch_bounds__(64 * kFewWaves) void k_lin_few(const FewArgs a) {
  __shared__ float red[kFewWaves][32][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int strip = blockIdx.x % a.strips, split = blockIdx.x / a.strips;
  const int n = strip * kFewCols + 8 * (lane & 15);  // the lane's 8 outputs
  const int kl = (KN ? 8 : 16) * (lane >> 4);        // and its place in a step
  const int k0 = (split * kFewWaves + wave) * a.wave_k, k1 = min(k0 + a.wave_k, a.K);
  lin_acc4 acc[MB][8];
#pragma unroll
  for (int b = 0; b < MB; ++b)
#pragma unroll
    for (int c = 0; c < 8; ++c) acc[b][c] = lin_acc4{0.f, 0.f, 0.f, 0.f};
  // byte offsets from the strip's and step's start, which are the wave's alone
  uint32_t xo[MB], wo[KN ? 1 : 8];
#pragma unroll
  for (int b = 0; b < MB; ++b) xo[b] = 2u * ((uint32_t)min(16 * b + (lane & 15), a.M - 1) * (uint32_t)a.ldx + (uint32_t)kl);
  // the lane's columns (KN: of N >= 8, the last 8 where fewer are left, computed twice) or rows of W
  const uint16_t* wb = KN ? a.w : a.w + (int64_t)strip * kFewCols * a.ldw;
  if constexpr (KN) {
    wo[0] = 2u * ((uint32_t)kl * (uint32_t)a.ldw + (uint32_t)min(n, a.N - 8));
  } else {
#pragma unroll
    for (int c = 0; c < 8; ++c)
      wo[c] = 2u * ((uint32_t)(min(n + c, a.N - 1) - strip * kFewCols) * (uint32_t)a.ldw + (uint32_t)kl);
  }
  auto w_at = [&](int c, int k) {
    const uint16_t* base = KN ? wb + (int64_t)(k + c) * a.ldw : wb + k;
    return reinterpret_cast<const uint16_t*>(reinterpret_cast<const char*>(base) + wo[KN ? 0 : c]);
  };
  auto x_at = [&](int b, int k) {
    return reinterpret_cast<const uint16_t*>(reinterpret_cast<const char*>(a.x + k) + xo[b]);
  };
  auto multiply = [&](const u32x4 (&wv)[8], const u32x4 (&xv)[MB]) {
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      u32x4 f;
      if constexpr (KN) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          f[j] = __builtin_amdgcn_perm(wv[2 * j + 1][c >> 1], wv[2 * j][c >> 1], c & 1 ? 0x07060302u : 0x05040100u);
      } else {
        f = wv[c];
      }
#pragma unroll
      for (int b = 0; b < MB; ++b)
        acc[b][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(g_bf16x8, xv[b]),
                                                            __builtin_bit_cast(g_bf16x8, f), acc[b][c], 0, 0, 0);
    }
  };
  // A step's vectors, H for each output and row: 8 of 32 k (KN) or, so that four lanes read 128 bytes of a row of W, 16 of 64.
  // Two steps are in flight.
  constexpr int H = KN ? 1 : 2, STEP = 32 * H;
  u32x4 w0[H][8], w1[H][8], x0[H][MB], x1[H][MB];
  auto load = [&](u32x4 (&wv)[H][8], u32x4 (&xv)[H][MB], int k) {
#pragma unroll
    for (int c = 0; c < 8; ++c)
#pragma unroll
      for (int h = 0; h < H; ++h) wv[h][c] = *reinterpret_cast<const u32x4_a2*>(w_at(c, k + 8 * h));
#pragma unroll
    for (int b = 0; b < MB; ++b)
#pragma unroll
      for (int h = 0; h < H; ++h) xv[h][b] = *reinterpret_cast<const u32x4_a2*>(x_at(b, k + 8 * h));
  };
  auto step = [&](const u32x4 (&wv)[H][8], const u32x4 (&xv)[H][MB]) {
#pragma unroll
    for (int h = 0; h < H; ++h) multiply(wv[h], xv[h]);
  };
  int k = k0, left = max(0, k1 - k0) / STEP;
  if (left > 0) load(w0, x0, k);
  while (left >= 2) {
    load(w1, x1, k + STEP);
    step(w0, x0);
    if (left > 2) load(w0, x0, k + 2 * STEP);
    step(w1, x1);
    k += 2 * STEP;
    left -= 2;
  }
  if (left) {
    step(w0, x0);
    k += STEP;
  }
  if (k < k1) {  // the last, shorter step
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const int rest = k1 - k - kl - 8 * h;
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        if constexpr (KN) w0[h][c] = c < rest ? *reinterpret_cast<const u32x4_a2*>(w_at(c, k)) : u32x4{0u, 0u, 0u, 0u};
        else w0[h][c] = load_vec(w_at(c, k + 8 * h), rest);
      }
#pragma unroll
      for (int b = 0; b < MB; ++b) x0[h][b] = load_vec(x_at(b, k + 8 * h), rest);
    }
    step(w0, x0);
  }
#pragma unroll
  for (int b = 0; b < MB; ++b) {
    if (b) __syncthreads();
#pragma unroll
    for (int c = 0; c < 8; ++c)
#pragma unroll
      for (int r = 0; r < 4; ++r) red[wave][r * 8 + c][lane] = acc[b][c][r];
    __syncthreads();
    // row 4 (l / 16) + r of the block, outputs of lane l
    if (tid < 256) {
      const int l = tid & 63, r = tid >> 6, m = 16 * b + 4 * (l >> 4) + r;
      const int no = strip * kFewCols + 8 * (l & 15);
      if (m < a.M && no < a.N) {
        float v[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          float sum = red[0][r * 8 + c][l];
#pragma unroll
          for (int q = 1; q < kFewWaves; ++q) sum += red[q][r * 8 + c][l];
          v[c] = sum;
        }
        // columns computed from N - 8 on: the ones from `no` on
        if (KN && no + 8 > a.N) {
          float u[8];
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            u[c] = 0.f;
#pragma unroll
            for (int d = 0; d < 8; ++d)
              if (d == c + no + 8 - a.N) u[c] = v[d];
          }
#pragma unroll
          for (int c = 0; c < 8; ++c) v[c] = u[c];
        }
        few_out<ACT, PART>(a, split, m, no, v);
      }
    }
  }
}

// The sums of the splits joined in their order, then the epilogue: a wave to 512 columns of a row.
template <int ACT>
__global__ __launch_bounds__(256) void k_lin_join(const float* __restrict__ part, int splits, int M, int N,
                                                  const Epilogue e) {
  const int n = (blockIdx.x * 64 + (threadIdx.x & 63)) * 8;
  if (n >= N) return;
  float bias[8];
#pragma unroll
  for (int q = 0; q < 8; ++q) bias[q] = e.bias && n + q < N ? load_any(e.bias, n + q, e.bias_bf16) : 0.f;
  for (int m = blockIdx.y * 4 + (threadIdx.x >> 6); m < M; m += gridDim.y * 4) {
    float v[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] = 0.f;
#pragma unroll 2
    for (int s = 0; s < splits; ++s) {
      const float* p = part + ((int64_t)s * M + m) * N + n;
      float u[8];
      if (n + 8 <= N) load8(p, 0, false, u);
      else
#pragma unroll
        for (int q = 0; q < 8; ++q) u[q] = n + q < N ? p[q] : 0.f;
#pragma unroll
      for (int q = 0; q < 8; ++q) v[q] += u[q];
    }
    finish8<ACT>(e, m, n, N, bias, v);
  }
}

// ---- operands laid out anew -----------------------------------------------------
// dst = src [lines, length] (lines ld apart) in lines of `vecs` whole vectors, ending in zeros.
struct LayOut {
  const uint16_t* src;
  int64_t ld;
  uint16_t* dst;
  int length, vecs;
  uint32_t total;  // vectors of all lines
};

// Both operands of a product in one launch, a thread to a vector: a streaming pass, 322 us for 687 MB of rows of 3,259
// elements (an element to a thread, 485).
__global__ __launch_bounds__(256) void k_lin_copy(const LayOut a, const LayOut b) {
  uint32_t i = blockIdx.x * 256u + threadIdx.x;
  const bool first = i < a.total;
  const LayOut& o = first ? a : b;
  if (!first) i -= a.total;
  if (i >= o.total) return;
  const uint32_t line = i / (uint32_t)o.vecs, c = (i - line * (uint32_t)o.vecs) * 8;
  const uint16_t* p = o.src + line * o.ld + c;
  const int left = o.length - (int)c;
  u32x4 v = {0u, 0u, 0u, 0u};
  if (left >= 8) {
    v = *reinterpret_cast<const u32x4_a2*>(p);
  } else {
#pragma unroll
    for (int q = 0; q < 7; ++q)
      if (q < left) v[q >> 1] |= (uint32_t)p[q] << (16 * (q & 1));
  }
  reinterpret_cast<u32x4*>(o.dst)[i] = v;
}

// ---- dz -------------------------------------------------------------------------
struct DzArgs {
  const void* dy;  // [M, N], rows lddy apart
  int64_t lddy;
  const float* z;  // [M, N] or NULL (no activation)
  uint16_t* dz;    // [M, lddz] or NULL, zeros past column N
  int64_t lddz;
  float* part;     // [blocks of rows][N] column sums, or NULL
  void* dbias;     // their place where there is one block
  bool dbias_bf16;
  int M, N;
  int rows;  // whose column sums are one fp32 partial
  bool dy_bf16;
};
// A workgroup to `rows` rows of 256 columns, a thread to 8 columns of every eighth row, two rows' loads in flight: a
// streaming pass.  The column sums of a thread's rows are joined through the LDS.
// dz is stored as bf16, what the matrix cores take, whatever dy's type: half a step in each term of dx and dW, whose own
// rounding is as large (4,001 x 3,584 x 3,584 with gelu: off by 2.3e-3 of the norm against 1.7e-3 of one rounding).  A second
// bf16 part would keep 16 bits and double both products.  dbias is summed before.
// 64 rows, or 16 where that leaves the chip without work (1,113 x 2,856: 11 us with 64).
static int dz_rows(int64_t M, int64_t N) { return (M + 63) / 64 * ((N + 255) / 256) >= 1024 ? 64 : 16; }

template <int ACT>
__global__ __launch_bounds__(256) void k_lin_dz(const DzArgs a) {
  __shared__ float sh[8][256];
  const int cl = threadIdx.x & 31, rl = threadIdx.x >> 5, n = blockIdx.x * 256 + 8 * cl;
  const int blocks = (a.M + a.rows - 1) / a.rows, k = min(8, a.N - n);
  for (int b = blockIdx.y; b < blocks; b += gridDim.y) {
    const int end = min(a.M, (b + 1) * a.rows);
    float sum[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) sum[q] = 0.f;
    auto row = [&](int m, float (&v)[8], float (&z)[8]) {
      const int64_t od = m * a.lddy + n, oz = (int64_t)m * a.N + n;
      if (k == 8) {
        load8(a.dy, od, a.dy_bf16, v);
        if (ACT != GRPO_ACT_NONE) load8(a.z, oz, false, z);
      } else {
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          v[q] = q < k ? load_any(a.dy, od + q, a.dy_bf16) : 0.f;
          z[q] = ACT != GRPO_ACT_NONE && q < k ? a.z[oz + q] : 0.f;
        }
      }
    };
    auto out = [&](int m, float (&v)[8], const float (&z)[8]) {
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        if (ACT != GRPO_ACT_NONE) v[q] *= slope_of<ACT>(z[q]);
        sum[q] += v[q];
      }
      if (a.dz) store8(a.dz, m * a.lddz + n, true, v);
    };
    if (n < a.N) {
      for (int m = b * a.rows + rl; m < end; m += 16) {
        float v0[8], z0[8], v1[8], z1[8];
        row(m, v0, z0);
        if (m + 8 < end) row(m + 8, v1, z1);
        out(m, v0, z0);
        if (m + 8 < end) out(m + 8, v1, z1);
      }
    }
    if (a.dbias) {
      __syncthreads();
#pragma unroll
      for (int q = 0; q < 8; ++q) sh[rl][8 * cl + q] = sum[q];
      __syncthreads();
      const int c = threadIdx.x;
      float s = sh[0][c];
#pragma unroll
      for (int q = 1; q < 8; ++q) s += sh[q][c];
      const int col = blockIdx.x * 256 + c;
      if (col >= a.N) continue;
      if (blocks == 1) store_any(a.dbias, col, s, a.dbias_bf16);
      else a.part[(int64_t)b * a.N + col] = s;
    }
  }
}

// dbias from the partial sums, added in fp64, each quarter of them in the order of the rows.
__global__ __launch_bounds__(256) void k_lin_dbias(const float* __restrict__ part, int blocks, int N, void* dbias,
                                                   bool bf16) {
  __shared__ double sh[4][64];
  const int c = threadIdx.x & 63, l = threadIdx.x >> 6, n = blockIdx.x * 64 + c;
  double sum = 0.0;
  if (n < N) {
#pragma unroll 8
    for (int b = l; b < blocks; b += 4) sum += (double)part[(int64_t)b * N + n];
  }
  sh[l][c] = sum;
  __syncthreads();
  if (l == 0 && n < N) store_any(dbias, n, (float)((sh[0][c] + sh[1][c]) + (sh[2][c] + sh[3][c])), bf16);
}

// ---- host -----------------------------------------------------------------------
constexpr int64_t kCus = 256;
constexpr int64_t kMostLin = 8388352;  // 2^23 - 256: 256 rows of an operand stay below 4 GB

static int64_t up8(int64_t x) { return (x + 7) / 8 * 8; }

// Whether rows of C elements, ld apart, can be loaded as whole aligned vectors.
static bool whole(const void* p, int64_t C, int64_t ld) {
  return C % 8 == 0 && ld % 8 == 0 && ld <= kMostLin && aligned(p, 16);
}

// An operand of a product: `rows` rows whose `cols` elements are summed over, as it lies (TileOperand).
struct Operand {
  const uint16_t* src;
  int64_t ld, rows, cols;
  bool turned;  // src is [cols, rows]
  bool padded;  // its lines end in zeros up to a multiple of 8
  int64_t lines() const { return turned ? cols : rows; }
  int64_t length() const { return padded ? up8(turned ? rows : cols) : turned ? rows : cols; }
  bool copied() const { return !whole(src, length(), ld); }  // where tiles read it
  size_t bytes() const { return copied() ? align_up(2 * (size_t)lines() * (size_t)up8(length())) : 0; }
};

// The operands as tiles read them, from ws on where they are copied.
static void lay_out(const Operand& a, const Operand& b, char*& ws, TileArgs& t, hipStream_t s) {
  LayOut l[2];
  int64_t lines[2], most[2];
  const Operand* o[2] = {&a, &b};
  TileOperand* to[2] = {&t.a, &t.b};
  for (int i = 0; i < 2; ++i) {
    const bool copied = o[i]->copied();
    uint16_t* dst = reinterpret_cast<uint16_t*>(ws);
    if (copied) ws += o[i]->bytes();
    const int64_t length = o[i]->length(), vecs = up8(length) / 8;
    *to[i] = copied ? TileOperand{dst, vecs * 8, o[i]->turned} : TileOperand{o[i]->src, o[i]->ld, o[i]->turned};
    l[i] = LayOut{o[i]->src, o[i]->ld, dst, (int)length, (int)vecs, 0u};
    lines[i] = copied ? o[i]->lines() : 0;
    most[i] = std::max<int64_t>(1, ((int64_t)1 << 30) / vecs);  // lines of a launch, whose threads stay below 2^32
  }
  while (lines[0] > 0 || lines[1] > 0) {
    int64_t n[2];
    for (int i = 0; i < 2; ++i) {
      n[i] = std::min(lines[i], most[i]);
      l[i].total = (uint32_t)(n[i] * l[i].vecs);
    }
    hipLaunchKernelGGL(k_lin_copy, dim3((l[0].total + l[1].total + 255u) / 256u), dim3(256), 0, s, l[0], l[1]);
    for (int i = 0; i < 2; ++i) {
      lines[i] -= n[i];
      l[i].src += n[i] * l[i].ld;
      l[i].dst += n[i] * l[i].vecs * 8;
    }
  }
}

// Tile shape and splits of the shortest launch, by what a CU was seen to take (us): for 64 summed over of a tile, with as
// many tiles beside it as the CU holds (`full`, of `slots`) or alone; for a tile's first loads and its epilogue; for the
// splits' sums, written, read and joined by a launch of their own.  Measured with bf16 operands of either layout (us, 256 x
// 256, 128 x 128, 64 x 128 and 192 x 256 tiles): 8,192 x 3,584 x 3,584 182, 200, 253, 216; 300 x 32,000 x 3,584 100, 115, 134,
// 82; 128 x 32,000 x 3,584 81, 50, 49, 66 and split in two 53, 42, 58, 48; 512 x 2,048 x 2,048 48, 22, 24, 40 and in two 29,
// 15, 16, 25; 2,048 x 3,584 x 151,936 whole 3,480, 2,359, 4,233, in two (256 x 256) 1,937.
static void plan_tiles(int64_t M, int64_t N, int64_t K, int& shape, int& splits, int& range) {
  static const struct {
    int slots;
    double full, alone, ends;
  } kCost[] = {{1, 1.70, 1.45, 9.0}, {2, 0.56, 0.78, 3.0}, {3, 0.36, 0.74, 2.0}, {1, 1.30, 1.12, 8.0}};
  const int64_t slabs = (K + 63) / 64;
  double best = 0.0;
  for (int s = 0; s < 4; ++s) {
    const TileShape& t = kTileShapes[s];
    const int64_t tiles = ((M + t.m - 1) / t.m) * ((N + t.n - 1) / t.n);
    for (int64_t k = 1; k <= 16 && (k == 1 || (k * 4 <= slabs && tiles * k <= 8 * kCus)); ++k) {
      const int64_t per = (slabs + k - 1) / k;
      if ((k - 1) * per >= slabs) continue;
      const int64_t rounds = (tiles * k + kCus - 1) / kCus, turns = (rounds + kCost[s].slots - 1) / kCost[s].slots;
      double us = std::max((double)rounds * (per * kCost[s].full + kCost[s].ends / 2),
                           (double)turns * (per * kCost[s].alone + kCost[s].ends));
      if (k > 1) us += 4.0 + (double)k * M * N * 8.0 / 5e6;
      if (best == 0.0 || us < best) {
        best = us;
        shape = s;
        splits = (int)k;
        range = (int)per * 64;
      }
    }
  }
}

// How a product is done: by the kernel for few rows, in `splits` parts of the summed dimension, or by tiles.
struct ProductPlan {
  bool few;
  int shape, splits;
  int range;    // few: the part of the sum of a wave; tiles: of a split
  size_t part;  // bytes of the splits' sums
};
static ProductPlan product_plan(const Operand& a, const Operand& b) {
  ProductPlan p{};
  p.splits = 1;
  const int64_t K = a.cols;
  p.few = a.rows <= (b.turned ? 32 : 16) && !a.turned && K >= 8 && (!b.turned || b.rows >= 8) && a.ld <= kMostLin &&
          b.ld <= kMostLin;
  if (p.few) {
    const int64_t strips = (b.rows + kFewCols - 1) / kFewCols, steps = (K + 63) / 64;
    // workgroups for the whole chip, of waves that have at least 2 steps each
    const int64_t most = std::max<int64_t>(1, steps / (2 * kFewWaves));
    p.splits = (int)std::max<int64_t>(1, std::min<int64_t>({most, kCus / strips, 32}));
    const int64_t waves = (int64_t)p.splits * kFewWaves;
    p.range = (int)((steps + waves - 1) / waves * 64);
  } else {
    plan_tiles(a.rows, b.rows, K, p.shape, p.splits, p.range);
  }
  if (p.splits > 1) p.part = align_up(4 * (size_t)p.splits * (size_t)a.rows * (size_t)b.rows);
  return p;
}

// go(the activation as a constant).
template <class F>
static void with_act(int act, F&& go) {
  switch (act) {
    case GRPO_ACT_RELU: return go(std::integral_constant<int, GRPO_ACT_RELU>());
    case GRPO_ACT_GELU: return go(std::integral_constant<int, GRPO_ACT_GELU>());
    case GRPO_ACT_GELU_TANH: return go(std::integral_constant<int, GRPO_ACT_GELU_TANH>());
    case GRPO_ACT_SILU: return go(std::integral_constant<int, GRPO_ACT_SILU>());
    default: return go(std::integral_constant<int, GRPO_ACT_NONE>());
  }
}

static size_t product_bytes(const Operand& a, const Operand& b) {
  const ProductPlan p = product_plan(a, b);
  return p.part + (p.few ? 0 : a.bytes() + b.bytes());
}

template <int ACT>
static void launch_few(const FewArgs& f, bool kn, hipStream_t s) {
  const dim3 grid((unsigned)(f.strips * f.splits)), block(64 * kFewWaves);
  auto go = [&](auto mb, auto is_kn) {
    constexpr int MB = decltype(mb)::value;
    constexpr bool KN = decltype(is_kn)::value;
    if (f.splits > 1) hipLaunchKernelGGL((k_lin_few<MB, KN, GRPO_ACT_NONE, true>), grid, block, 0, s, f);
    else hipLaunchKernelGGL((k_lin_few<MB, KN, ACT, false>), grid, block, 0, s, f);
  };
  const std::integral_constant<int, 1> one;
  if (!kn) go(one, std::false_type());
  else if (f.M <= 16) go(one, std::true_type());
  else go(std::integral_constant<int, 2>(), std::true_type());
}

static void join_splits(const float* part, int splits, int M, int N, const Epilogue& e, hipStream_t s) {
  const dim3 grid((unsigned)((N + 511) / 512), (unsigned)std::min((M + 3) / 4, 16384)), block(256);
  auto go = [&](auto act) { hipLaunchKernelGGL(k_lin_join<decltype(act)::value>, grid, block, 0, s, part, splits, M, N, e); };
  with_act(e.act, go);
}

// C [a.rows, b.rows] = A B^T with the epilogue e.
static void launch_product(const Operand& a, const Operand& b, const Epilogue& e, char* ws, hipStream_t s) {
  const ProductPlan p = product_plan(a, b);
  const int M = (int)a.rows, N = (int)b.rows, K = (int)a.cols;
  float* part = reinterpret_cast<float*>(ws);
  ws += p.part;
  if (p.few) {
    const FewArgs f{a.src, b.src, a.ld, b.ld, M, K, N, (N + kFewCols - 1) / kFewCols, p.splits, p.range, part, e};
    with_act(e.act, [&](auto act) { launch_few<decltype(act)::value>(f, b.turned, s); });
  } else {
    TileArgs t;
    lay_out(a, b, ws, t, s);
    t.M = M;
    t.N = N;
    t.K = K;
    t.splits = p.splits;
    t.split_k = p.range;
    t.part = part;
    t.e = e;
    launch_tiles(t, p.shape, s);
  }
  if (p.splits > 1) join_splits(part, p.splits, M, N, e, s);
}

static bool is_dtype(int32_t d) { return d == GRPO_F32 || d == GRPO_BF16; }
static size_t size_of(int32_t d) { return d == GRPO_BF16 ? 2 : 4; }

static int check_op(const grpo_linear_op* op) {
  if (!op || op->act < GRPO_ACT_NONE || op->act > GRPO_ACT_SILU || (op->w_out_in != 0 && op->w_out_in != 1))
    return GRPO_ERR_ARG;
  if (op->M < 0 || op->M > kMostLin || op->K < 1 || op->K > kMostLin || op->N < 1 || op->N > kMostLin ||
      op->ldx < op->K || op->ldw < (op->w_out_in ? op->K : op->N))
    return GRPO_ERR_SHAPE;
  return GRPO_OK;
}

static Operand x_rows(const grpo_linear_op& op) {
  return Operand{static_cast<const uint16_t*>(op.x), op.ldx, op.M, op.K, false, false};
}
static Operand w_as_nk(const grpo_linear_op& op) {
  return Operand{static_cast<const uint16_t*>(op.w), op.ldw, op.N, op.K, op.w_out_in == 0, false};
}
static Operand w_as_kn(const grpo_linear_op& op) {
  return Operand{static_cast<const uint16_t*>(op.w), op.ldw, op.K, op.N, op.w_out_in == 1, false};
}

static ByteRows x_bytes(const grpo_linear_op& op) { return ByteRows(op.x, op.M, op.K, op.ldx, 2); }
static ByteRows w_bytes(const grpo_linear_op& op) {
  return op.w_out_in ? ByteRows(op.w, op.N, op.K, op.ldw, 2) : ByteRows(op.w, op.K, op.N, op.ldw, 2);
}

// What the backward call does and keeps: dz, dbias's partial sums, and what the product at hand needs (dW's comes after dx's on
// the stream and takes the same place).
struct BwdPlan {
  bool make_dz;  // dz is not dy as it lies
  size_t dz, part;
  Operand dz_rows, dz_cols, x_cols, w;
  size_t total;
};
static BwdPlan bwd_plan(const grpo_linear_op& op, const void* dy, int64_t lddy, int32_t dy_dtype,
                        const grpo_linear_grads& g) {
  BwdPlan p{};
  const bool products = g.dx || g.dw;
  p.make_dz = products && (op.act != GRPO_ACT_NONE || dy_dtype != GRPO_BF16 || !whole(dy, op.N, lddy));
  p.dz = p.make_dz ? align_up(2 * (size_t)op.M * (size_t)up8(op.N)) : 0;
  const int64_t rows = dz_rows(op.M, op.N);
  p.part = g.dbias ? align_up(4 * (size_t)((op.M + rows - 1) / rows) * (size_t)op.N) : 0;
  const uint16_t* dz = p.make_dz ? nullptr : static_cast<const uint16_t*>(dy);  // its place in the workspace is aligned as NULL is
  const int64_t ld = p.make_dz ? up8(op.N) : lddy;
  p.dz_rows = Operand{dz, ld, op.M, op.N, false, p.make_dz};
  p.dz_cols = Operand{dz, ld, op.N, op.M, true, p.make_dz};
  p.x_cols = Operand{static_cast<const uint16_t*>(op.x), op.ldx, op.K, op.M, true, false};
  p.w = w_as_kn(op);
  const size_t dx = g.dx ? product_bytes(p.dz_rows, p.w) : 0;
  const size_t dw = g.dw ? product_bytes(op.w_out_in ? p.dz_cols : p.x_cols, op.w_out_in ? p.x_cols : p.dz_cols) : 0;
  p.total = p.dz + p.part + std::max(dx, dw);
  return p;
}

static int check_bwd(const grpo_linear_op* op, int64_t lddy, int32_t dy_dtype, const grpo_linear_grads* g) {
  const int st = check_op(op);
  if (st != GRPO_OK) return st;
  if (!g || (g->accumulate_dw != 0 && g->accumulate_dw != 1)) return GRPO_ERR_ARG;
  if (lddy < op->N) return GRPO_ERR_SHAPE;
  if (!is_dtype(dy_dtype) || (g->dw && !is_dtype(g->dw_dtype)) || (g->dbias && !is_dtype(op->bias_dtype)))
    return GRPO_ERR_DTYPE;
  if (g->dw && g->accumulate_dw && g->dw_dtype != GRPO_F32) return GRPO_ERR_ARG;
  return GRPO_OK;
}

// n elements of 2 bytes.
__global__ __launch_bounds__(256) void k_lin_zero(uint16_t* p, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) p[i] = 0;
}
static void zero_fill(void* p, int64_t n, size_t esz, hipStream_t s) {
  n *= (int64_t)(esz / 2);
  hipLaunchKernelGGL(k_lin_zero, dim3((unsigned)std::min<int64_t>(4096, (n + 255) / 256)), dim3(256), 0, s,
                     static_cast<uint16_t*>(p), n);
}

}  // namespace grpo

using namespace grpo;

extern "C" size_t grpo_linear_workspace_bytes(const grpo_linear_op* op) {
  if (check_op(op) != GRPO_OK || op->M == 0) return 0;
  return product_bytes(x_rows(*op), w_as_nk(*op));
}

extern "C" int grpo_linear(const grpo_linear_op* op, const void* residual, int64_t ldr, void* y, int64_t ldy,
                           int32_t y_dtype, float* z, void* ws, size_t ws_bytes, hipStream_t s) {
  const int st = check_op(op);
  if (st != GRPO_OK) return st;
  if (op->M > 0 && (!op->x || !op->w || !y)) return GRPO_ERR_ARG;
  if (ldy < op->N || (residual && ldr < op->N)) return GRPO_ERR_SHAPE;
  if (!is_dtype(y_dtype) || (op->bias && !is_dtype(op->bias_dtype))) return GRPO_ERR_DTYPE;
  if (!aligned(op->x, 2) || !aligned(op->w, 2) || !aligned(y, size_of(y_dtype)) || !aligned(z, 4) ||
      !aligned(residual, size_of(y_dtype)) || (op->bias && !aligned(op->bias, size_of(op->bias_dtype))))
    return GRPO_ERR_ALIGN;
  if (residual == y && residual && ldr != ldy) return GRPO_ERR_ARG;
  const size_t need = grpo_linear_workspace_bytes(op);
  if (need > 0) {
    if (!ws || ws_bytes < need) return GRPO_ERR_WORKSPACE;
    if (!aligned(ws, 16)) return GRPO_ERR_ALIGN;
  }
  if (op->M > 0) {
    const ByteRows x = x_bytes(*op), w = w_bytes(*op), b(op->bias, 1, op->N, op->N, size_of(op->bias_dtype)),
                   r(residual, op->M, op->N, ldr, size_of(y_dtype)), out(y, op->M, op->N, ldy, size_of(y_dtype)),
                   zs(z, op->M, op->N, op->N, 4);
    if (rows_share(out, x) || rows_share(out, w) || rows_share(out, b) || (residual != y && rows_share(out, r)) ||
        rows_share(zs, x) || rows_share(zs, w) || rows_share(zs, b) || rows_share(zs, r) || rows_share(zs, out))
      return GRPO_ERR_ARG;
    char* at = static_cast<char*>(ws);
    const Epilogue e{y, ldy, op->bias, residual, ldr, z, op->act, y_dtype == GRPO_BF16, op->bias_dtype == GRPO_BF16, false};
    launch_product(x_rows(*op), w_as_nk(*op), e, at, s);
  }
  return hipGetLastError() == hipSuccess ? GRPO_OK : GRPO_ERR_HIP;
}

extern "C" size_t grpo_linear_bwd_workspace_bytes(const grpo_linear_op* op, const void* dy, int64_t lddy,
                                                  int32_t dy_dtype, const grpo_linear_grads* grads) {
  if (check_bwd(op, lddy, dy_dtype, grads) != GRPO_OK || op->M == 0) return 0;
  return bwd_plan(*op, dy, lddy, dy_dtype, *grads).total;
}

extern "C" int grpo_linear_bwd(const grpo_linear_op* op, const void* dy, int64_t lddy, int32_t dy_dtype, const float* z,
                               const grpo_linear_grads* grads, void* ws, size_t ws_bytes, hipStream_t s) {
  const int st = check_bwd(op, lddy, dy_dtype, grads);
  if (st != GRPO_OK) return st;
  const grpo_linear_grads& g = *grads;
  const bool act = op->act != GRPO_ACT_NONE, work = g.dx || g.dw || g.dbias;
  if (op->M > 0 && work && (!dy || (act && !z))) return GRPO_ERR_ARG;
  if (op->M > 0 && ((g.dx && !op->w) || (g.dw && !op->x))) return GRPO_ERR_ARG;
  if (!aligned(op->x, 2) || !aligned(op->w, 2) || !aligned(dy, size_of(dy_dtype)) || !aligned(z, 4) || !aligned(g.dx, 2) ||
      (g.dw && !aligned(g.dw, size_of(g.dw_dtype))) || (g.dbias && !aligned(g.dbias, size_of(op->bias_dtype))))
    return GRPO_ERR_ALIGN;
  const size_t need = grpo_linear_bwd_workspace_bytes(op, dy, lddy, dy_dtype, grads);
  if (need > 0) {
    if (!ws || ws_bytes < need) return GRPO_ERR_WORKSPACE;
    if (!aligned(ws, 16)) return GRPO_ERR_ALIGN;
  }
  if (op->M == 0) {
    if (g.dw && !g.accumulate_dw) zero_fill(g.dw, op->K * op->N, size_of(g.dw_dtype), s);
    if (g.dbias) zero_fill(g.dbias, op->N, size_of(op->bias_dtype), s);
    return hipGetLastError() == hipSuccess ? GRPO_OK : GRPO_ERR_HIP;
  }
  const ByteRows out[3] = {ByteRows(g.dx, op->M, op->K, op->K, 2),
                           ByteRows(g.dw, op->K, op->N, op->N, size_of(g.dw_dtype)),
                           ByteRows(g.dbias, 1, op->N, op->N, size_of(op->bias_dtype))};
  const ByteRows in[4] = {ByteRows(dy, op->M, op->N, lddy, size_of(dy_dtype)), ByteRows(act ? z : nullptr, op->M, op->N, op->N, 4),
                          x_bytes(*op), w_bytes(*op)};
  const bool read[4] = {true, true, g.dw != nullptr, g.dx != nullptr};
  for (int i = 0; i < 3; ++i) {
    for (int j = 0; j < 4; ++j)
      if (read[j] && rows_share(out[i], in[j])) return GRPO_ERR_ARG;
    if (rows_share(out[i], out[(i + 1) % 3])) return GRPO_ERR_ARG;
  }
  BwdPlan p = bwd_plan(*op, dy, lddy, dy_dtype, g);
  char* at = static_cast<char*>(ws);
  uint16_t* dz = p.make_dz ? reinterpret_cast<uint16_t*>(at) : nullptr;
  at += p.dz;
  float* part = g.dbias ? reinterpret_cast<float*>(at) : nullptr;
  at += p.part;
  if (dz || part) {
    const int rows = dz_rows(op->M, op->N), blocks = (int)((op->M + rows - 1) / rows);
    const DzArgs a{dy,   lddy,    act ? z : nullptr,             dz,         up8(op->N),
                   part, g.dbias, op->bias_dtype == GRPO_BF16, (int)op->M, (int)op->N, rows,
                   dy_dtype == GRPO_BF16};
    const dim3 grid((unsigned)((up8(op->N) + 255) / 256), (unsigned)std::min(blocks, 16384));
    with_act(op->act, [&](auto kind) { hipLaunchKernelGGL(k_lin_dz<decltype(kind)::value>, grid, dim3(256), 0, s, a); });
    if (part && blocks > 1)
      hipLaunchKernelGGL(k_lin_dbias, dim3((unsigned)((op->N + 63) / 64)), dim3(256), 0, s, part, blocks, (int)op->N,
                         g.dbias, op->bias_dtype == GRPO_BF16);
  }
  if (dz) p.dz_rows.src = p.dz_cols.src = dz;
  if (g.dx) {
    const Epilogue e{g.dx, op->K, nullptr, nullptr, 0, nullptr, GRPO_ACT_NONE, true, false, false};
    launch_product(p.dz_rows, p.w, e, at, s);
  }
  if (g.dw) {
    const Epilogue e{g.dw, op->w_out_in ? op->K : op->N, nullptr, nullptr, 0, nullptr, GRPO_ACT_NONE,
                     g.dw_dtype == GRPO_BF16, false, g.accumulate_dw == 1};
    launch_product(op->w_out_in ? p.dz_cols : p.x_cols, op->w_out_in ? p.x_cols : p.dz_cols, e, at, s);
  }
  return hipGetLastError() == hipSuccess ? GRPO_OK : GRPO_ERR_HIP;
}
