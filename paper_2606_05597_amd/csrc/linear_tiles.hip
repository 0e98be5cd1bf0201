// The tiled products of grpo_linear.h: C[m, n] = sum_k A[m, k] B[n, k], the tiles, accumulators and DMA into LDS of gemm.h, for
// operands that lie with the summed dimension contiguous or across it.
//
// An operand that lies across ("turned": row k holds its values for all m) goes into LDS as it is, 64 rows of a tile's
// columns, and is turned where its fragments are read: ds_read_b64_tr_b16 takes 8 bytes from each of 16 lanes, four k of 16
// columns, and gives each lane one column's four.  The 16-byte slots of four consecutive rows are exchanged so that a read's 256
// bytes lie in different banks.  So no transposed copy of x, W or dz is ever made.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "gemm.h"
#include "linear.h"

namespace grpo {

typedef short lin_s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) lin_s16x4 lin_lds_s16x4;

// One operand's part of a tile: R rows (m or n), W of them a wave's, in blocks of 32; NW waves load it.
template <int R, int W, int NW, bool TURNED>
struct Side {
  static constexpr int Q = R / 8 / NW;           // DMA instructions per wave and slab
  static constexpr int NB = W / 32;              // fragments of a wave
  static constexpr int READS = TURNED ? 2 * NB : NB;
  static constexpr int SLOTS = R / 8;            // turned: 16-byte slots of a row k
  static constexpr int BYTES = R * 128;          // of a slab
  const uint16_t* base;
  int64_t ld;
  int rows, K;        // rows of the tile that exist; the summed dimension's end
  int wave, lane;
  uint32_t off[NB];   // turned: LDS byte offsets of the wave's fragments in a slab
  uint32_t row_off;   // otherwise: of its first row
  int sw[4];

  __device__ __forceinline__ void init(const TileOperand& o, int row0, int total, int K_, int wave_, int lane_, int first) {
    base = o.p + (TURNED ? (int64_t)row0 : (int64_t)row0 * o.ld);
    ld = o.ld;
    rows = min(R, (TURNED ? (total + 7) / 8 * 8 : total) - row0);
    K = TURNED ? K_ : (K_ + 7) / 8 * 8;
    wave = wave_;
    lane = lane_;
    if constexpr (TURNED) {
      const int i = lane & 15, k = 8 * (lane >> 5) + (i >> 2);  // row k of the first read
      const int x = exchange(k);
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const int slot = (((first / 32 + b) ^ x) << 2) | (((lane >> 4) & 1) << 1) | ((i & 3) >> 1);
        off[b] = (uint32_t)(k * R * 2 + slot * 16 + (i & 1) * 8);
      }
    } else {
      const int fr = lane & 31, hi = lane >> 5;
      row_off = (uint32_t)(first + fr) * 128u;
#pragma unroll
      for (int s = 0; s < 4; ++s) sw[s] = ((2 * s + hi) ^ lds_swizzle(fr)) * 16;
    }
  }

  // How many fours of slots row k's are exchanged by.  Rows of 256 or 512 bytes begin at the same bank, those of 128 or 384
  // at two in turn.
  static __device__ __forceinline__ int exchange(int k) { return R % 128 == 0 ? k & 3 : (k >> 1) & 1; }

  // Slab k0 .. k0 + 63 into LDS at byte address `at`.
  __device__ __forceinline__ void issue(uint32_t at, int k0) const {
    if constexpr (TURNED) {
      const int left = min(64, K - k0);
      const g_u32x4 rs = buffer_rsrc(base + (int64_t)k0 * ld, (uint32_t)(((int64_t)(left - 1) * ld + rows) * 2));
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        const int i = q * NW + wave, v = i * 64 + lane, k = v / SLOTS, s = v % SLOTS;
        const int col = (s ^ (exchange(k) << 2)) * 8;
        dma16(at + (uint32_t)i * 1024u, col < rows ? (uint32_t)(k * ld + col) * 2u : kOobOffset, rs);
      }
    } else {
      const g_u32x4 rs = buffer_rsrc(base, (uint32_t)(((int64_t)(rows - 1) * ld + K) * 2));
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        const int i = q * NW + wave, row = i * 8 + (lane >> 3), kv = (lane & 7) ^ lds_swizzle(row);
        dma16(at + (uint32_t)i * 1024u, k0 + kv * 8 < K ? (uint32_t)(row * ld + k0 + kv * 8) * 2u : kOobOffset, rs);
      }
    }
  }

  // The fragments of k-substep s (16 of the slab's 64) of the slab at byte address `at`.
  __device__ __forceinline__ void read(g_bf16x8 (&f)[NB], uint32_t at, int s) const {
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      if constexpr (TURNED) {
        const uint32_t p = at + off[b] + (uint32_t)(s * 16 * R * 2);
        const lin_s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lin_lds_s16x4*>(p));
        const lin_s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lin_lds_s16x4*>(p + 4 * R * 2));
        f[b] = __builtin_bit_cast(g_bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
      } else {
        typedef __attribute__((address_space(3))) g_bf16x8 frag;
        f[b] = *reinterpret_cast<const frag*>(at + row_off + (uint32_t)(b * 32 * 128) + (uint32_t)sw[s]);
      }
    }
  }
};

// Bound by the matrix cores and their power: 59% busy at the 1.9 GHz that 256 x 256 tiles of random numbers leave the chip
// (1,170 TFLOP/s); with all operands in the L2 no faster, with zeros for numbers 1,400 TFLOP/s.  LDS reads take 23% of its
// cycles, without bank conflicts.
template <class C, bool AT, bool BT>
__device__ __forceinline__ void lin_mainloop(const TileArgs& t, int m0, int n0, int kb, int ke,
                                             g_f32x16 (&acc)[C::IB][C::JB], uint32_t lds0) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / C::WGN, wn = wave % C::WGN;
  typedef Side<C::BM, C::WTM, C::NW, AT> SA;
  typedef Side<C::BN, C::WTN, C::NW, BT> SB;
  SA a;
  SB b;
  a.init(t.a, m0, t.M, min(t.K, ke), wave, lane, wm * C::WTM);
  b.init(t.b, n0, t.N, min(t.K, ke), wave, lane, wn * C::WTN);
  constexpr uint32_t kStage = SA::BYTES + SB::BYTES;
  auto issue = [&](int buf, int k0) {
    a.issue(lds0 + buf * kStage, k0);
    b.issue(lds0 + buf * kStage + SA::BYTES, k0);
  };
#pragma unroll
  for (int i = 0; i < C::IB; ++i)
#pragma unroll
    for (int j = 0; j < C::JB; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  g_bf16x8 fa[2][C::IB], fb[2][C::JB];
  auto read = [&](int f, int buf, int s) {
    a.read(fa[f], lds0 + buf * kStage, s);
    b.read(fb[f], lds0 + buf * kStage + SA::BYTES, s);
  };
  // the MFMAs of one fragment set, with the LDS reads of the next one between them
  auto mma = [&](int f) {
#pragma unroll
    for (int i = 0; i < C::IB; ++i)
#pragma unroll
      for (int j = 0; j < C::JB; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[f][i], fb[f][j], acc[i][j], 0, 0, 0);
    constexpr int NR = SA::READS + SB::READS, NM = C::IB * C::JB;
    constexpr int TWO = NR > NM ? NR - NM : 0, ONE = NR > NM ? NM - TWO : NR;
#pragma unroll
    for (int x = 0; x < TWO; ++x) {
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);  // two LDS reads
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // one MFMA
    }
#pragma unroll
    for (int x = 0; x < ONE; ++x) {
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    }
    if constexpr (NM > TWO + ONE) __builtin_amdgcn_sched_group_barrier(0x008, NM - TWO - ONE, 0);
  };
  const int nk = (ke - kb + 63) / 64;
  issue(0, kb);
  if (nk > 1) issue(1, kb + 64);
  wait_vm0();
  barrier();
  read(0, 0, 0);
  for (int kt = 0; kt < nk; ++kt) {
    const int buf = kt & 1;
    read(1, buf, 1);
    mma(0);
    read(0, buf, 2);
    mma(1);
    read(1, buf, 3);
    mma(0);
    wait_lgkm0();  // this wave's reads of slab kt are done
    wait_vm0();    // this wave's DMA of slab kt + 1 has landed
    barrier();     // ... and every wave's
    // Eight waves' loads go out behind the MFMAs, which then are not held up by the waves' first reads of the next slab
    // waiting behind them (8,192 x 3,584 x 3,584: 186 us against 199); four waves' before (128 x 128 tiles 247 and 261).
    constexpr bool LATE = C::NW == 8;
    if (!LATE && kt + 2 < nk) issue(buf, kb + (kt + 2) * 64);
    if (kt + 1 < nk) read(0, buf ^ 1, 0);
    mma(1);
    if (LATE && kt + 2 < nk) issue(buf, kb + (kt + 2) * 64);
  }
}

typedef float lin_f32x4 __attribute__((ext_vector_type(4)));

// What lanes of a wave stored to LDS before is what others of it read after.
__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A wave's sums, 32 rows at a time, through its own part of the LDS into rows of 16-byte vectors: out of the registers
// they would be stored 64 bytes to a row.  FULL: the tile's columns lie inside C; what is added to the rows is then on its
// way before the 32 rows before them are done (nothing else on the CU hides a load here: 8 rows at a time, each waiting for
// its own, 8,192 x 3,584 x 3,584 with a residual took 235 us).
template <class C, int ACT, bool FULL>
__device__ __forceinline__ void finish_tile(const Epilogue& e, int m0, int n0, int M, int N,
                                            const g_f32x16 (&acc)[C::IB][C::JB], float* lds) {
  constexpr int LD = C::WTN + 4, LPR = C::WTN / 8, RPS = 64 / LPR, STEPS = 32 / RPS;  // lanes to a row, rows to a step
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / C::WGN, wn = wave % C::WGN;
  float* mine = lds + wave * 32 * LD;
  const int cl = lane % LPR * 8, n = n0 + wn * C::WTN + cl, mw = m0 + wm * C::WTM + lane / LPR;
  float bias[8];
#pragma unroll
  for (int q = 0; q < 8; ++q) bias[q] = e.bias && n + q < N ? load_any(e.bias, n + q, e.bias_bf16) : 0.f;
  const void* more = e.residual ? e.residual : e.accumulate ? e.out : nullptr;
  const int64_t ldm = e.residual ? e.ldr : e.ldo;
  Raw8 r[2][STEPS];
  auto fetch = [&](int i) {
#pragma unroll
    for (int q = 0; q < STEPS; ++q) r[i & 1][q].load(more, min(mw + i * 32 + q * RPS, M - 1) * ldm + n, e.out_bf16);
  };
  if (FULL && more) fetch(0);
#pragma unroll
  for (int i = 0; i < C::IB; ++i) {
    if (FULL && more && i + 1 < C::IB) fetch(i + 1);
#pragma unroll
    for (int j = 0; j < C::JB; ++j)
#pragma unroll
      for (int k = 0; k < 16; ++k) mine[(8 * (k >> 2) + 4 * (lane >> 5) + (k & 3)) * LD + j * 32 + (lane & 31)] = acc[i][j][k];
    wave_order();
    auto step = [&](int q) {
      const int m = mw + i * 32 + q * RPS;
      if (m >= M || (!FULL && n >= N)) return;
      float v[8];
      const lin_f32x4* src = reinterpret_cast<const lin_f32x4*>(mine + (q * RPS + lane / LPR) * LD + cl);
      const lin_f32x4 a = src[0], b = src[1];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        v[k] = a[k];
        v[k + 4] = b[k];
      }
      if constexpr (FULL) finish_whole8<ACT>(e, m, n, N, bias, more ? &r[i & 1][q] : nullptr, v);
      else finish8<ACT>(e, m, n, N, bias, v);
    };
    if constexpr (FULL) {
#pragma unroll
      for (int q = 0; q < STEPS; ++q) step(q);
    } else {
#pragma unroll 1
      for (int q = 0; q < STEPS; ++q) step(q);
    }
    wave_order();
  }
}

template <class C, int ACT>
__device__ __forceinline__ void finish(const Epilogue& e, int m0, int n0, int M, int N, const g_f32x16 (&acc)[C::IB][C::JB],
                                       float* lds) {
  if (n0 + C::BN <= N) finish_tile<C, ACT, true>(e, m0, n0, M, N, acc, lds);
  else finish_tile<C, ACT, false>(e, m0, n0, M, N, acc, lds);
}

template <class C, bool AT, bool BT, int ACT>
__global__ __launch_bounds__(C::NT) void k_lin_tiles(const TileArgs t) {
  constexpr int kEpi = (int)sizeof(float) * C::NW * 32 * (C::WTN + 4);
  __shared__ __attribute__((aligned(16))) uint16_t lds[(kEpi > C::LDS_BYTES ? kEpi : C::LDS_BYTES) / 2];
  int tm, tn, split;
  const int tiles_m = (t.M + C::BM - 1) / C::BM, tiles_n = (t.N + C::BN - 1) / C::BN;
  if (!gemm_tile_of(blockIdx.x, gridDim.x, tiles_m, tiles_n, t.splits, tm, tn, split)) return;
  const int m0 = tm * C::BM, n0 = tn * C::BN, kb = split * t.split_k, ke = min(kb + t.split_k, t.K);
  g_f32x16 acc[C::IB][C::JB];
  const uint32_t lds0 = (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint16_t*)lds);
  lin_mainloop<C, AT, BT>(t, m0, n0, kb, ke, acc, lds0);
  __syncthreads();  // every wave's last reads are done
  if (t.splits > 1) {
    Epilogue e{};
    e.out = t.part + (int64_t)split * t.M * t.N;
    e.ldo = t.N;
    finish<C, GRPO_ACT_NONE>(e, m0, n0, t.M, t.N, acc, reinterpret_cast<float*>(lds));
  } else {
    finish<C, ACT>(t.e, m0, n0, t.M, t.N, acc, reinterpret_cast<float*>(lds));
  }
}

template <class C, bool AT, bool BT, int ACT>
static void launch(const TileArgs& t, hipStream_t s) {
  const int64_t tiles = (int64_t)((t.M + C::BM - 1) / C::BM) * ((t.N + C::BN - 1) / C::BN) * t.splits;
  hipLaunchKernelGGL((k_lin_tiles<C, AT, BT, ACT>), dim3((unsigned)((tiles + 7) / 8 * 8)), dim3(C::NT), 0, s, t);
}

template <class C>
static void launch_shape(const TileArgs& t, hipStream_t s) {
  if (t.a.turned) return launch<C, true, true, GRPO_ACT_NONE>(t, s);  // dW alone
  const int act = t.splits > 1 ? (int)GRPO_ACT_NONE : t.e.act;
  auto with = [&](auto bt) {
    constexpr bool BT = decltype(bt)::value;
    switch (act) {
      case GRPO_ACT_RELU: return launch<C, false, BT, GRPO_ACT_RELU>(t, s);
      case GRPO_ACT_GELU: return launch<C, false, BT, GRPO_ACT_GELU>(t, s);
      case GRPO_ACT_GELU_TANH: return launch<C, false, BT, GRPO_ACT_GELU_TANH>(t, s);
      case GRPO_ACT_SILU: return launch<C, false, BT, GRPO_ACT_SILU>(t, s);
      default: return launch<C, false, BT, GRPO_ACT_NONE>(t, s);
    }
  };
  if (t.b.turned) with(std::true_type());
  else with(std::false_type());
}

void launch_tiles(const TileArgs& t, int shape, hipStream_t s) {
  switch (shape) {
    case 0: return launch_shape<GemmCfg<256, 256, 2, 4>>(t, s);
    case 1: return launch_shape<GemmCfg<128, 128, 2, 2>>(t, s);
    case 2: return launch_shape<GemmCfg<64, 128, 1, 2>>(t, s);
    default: return launch_shape<GemmCfg<192, 256, 2, 4>>(t, s);
  }
}

}  // namespace grpo
