// Linear layers in 8-bit floating point: e4m3 codes with one fp32 scale per token and 128 inputs for the activations, one per
// 128 x 128 tile for the weights (the paper's deployments run their projections and FFNs in low-bit formats and fuse GEMM + GELU and
// GEMM + residual).
//     y[m,n] = sum_g sx[g,m] sw[n/128,g] sum_{k in group g} x8[m,k] w8[n,k],   out = bf16(act(y + bias[n]) + residual[m,n])
//   quantize_rows_kernel, quantize_tiles_kernel   the codes (HBM-bound passes)
//   linear_kernel                                 the product
#include <type_traits>

#include "tc_ptx.cuh"

namespace sva {

// ------------------------------------------------------------------ quantisers
// 16 consecutive values of a row of K from channel c (zeros beyond K); the row is 16-byte aligned and c a multiple of 16
__device__ __forceinline__ void lin_load16(const __nv_bfloat16* row, int c, int K, uint4 (&u)[2]) {
  u[0] = u[1] = make_uint4(0u, 0u, 0u, 0u);
  if (c + 16 <= K) {
    u[0] = __ldg(reinterpret_cast<const uint4*>(row + c));
    u[1] = __ldg(reinterpret_cast<const uint4*>(row + c + 8));
  } else if (c < K) {
    uint32_t w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t lo = c + 2 * e < K ? __ldg(reinterpret_cast<const unsigned short*>(row) + c + 2 * e) : 0u;
      const uint32_t hi = c + 2 * e + 1 < K ? __ldg(reinterpret_cast<const unsigned short*>(row) + c + 2 * e + 1) : 0u;
      w[e] = lo | hi << 16;
    }
    u[0] = make_uint4(w[0], w[1], w[2], w[3]);
    u[1] = make_uint4(w[4], w[5], w[6], w[7]);
  }
}
__device__ __forceinline__ float lin_scale(float amax) { return amax == 0.f ? 1.0f : div_by_448(amax); }
// the codes of 16 values: the correctly rounded fp32 quotients, rounded to e4m3
__device__ __forceinline__ uint4 lin_codes(const uint4 (&u)[2], float s) {
  const uint32_t w[8] = {u[0].x, u[0].y, u[0].z, u[0].w, u[1].x, u[1].y, u[1].z, u[1].w};
  uint32_t c[4];
  if (div_fast_ok(s)) {
    const float r = __frcp_rn(s);
    const uint64_t neg2 = pack2(-s, -s), r2 = pack2(r, r);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      c[e] = e4m3x4(div_fast2(pack2(bf16lo(w[2 * e]), bf16hi(w[2 * e])), neg2, r2),
                    div_fast2(pack2(bf16lo(w[2 * e + 1]), bf16hi(w[2 * e + 1])), neg2, r2));
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      c[e] = __byte_perm(e4m3x2(div_any(bf16lo(w[2 * e]), s), div_any(bf16hi(w[2 * e]), s)),
                         e4m3x2(div_any(bf16lo(w[2 * e + 1]), s), div_any(bf16hi(w[2 * e + 1]), s)), 0x5410);
  }
  return make_uint4(c[0], c[1], c[2], c[3]);
}

// A CTA takes 32 rows x GROUPS groups: 8 lanes per row and group, so that a group's maximum is three shuffles and the 32 scales of
// a group leave side by side; a thread has GROUPS groups of its row in flight.  HBM-bound: 47 616 x 4 096 86 us = 6.8 TB/s.
template <int GROUPS>
__global__ void __launch_bounds__(256)
quantize_rows_kernel(const __nv_bfloat16* __restrict__ x, int M, int K, long long xs, uint8_t* __restrict__ x8, long long x8s,
                     float* __restrict__ scale, long long ss, int group_tiles) {
  grid_dep_launch();
  const int zero = grid_dep_wait();
  const int lane = threadIdx.x & 7, Kb = (K + 127) / 128;
  const int g0 = (int)(blockIdx.x % group_tiles) * GROUPS;
  const int m = (int)(blockIdx.x / group_tiles) * 32 + (threadIdx.x >> 3) + zero;
  const bool there = m < M;
  const __nv_bfloat16* row = x + (long long)(there ? m : 0) * xs;
  uint4 u[GROUPS][2];
#pragma unroll
  for (int i = 0; i < GROUPS; ++i) lin_load16(row, (g0 + i) * 128 + lane * 16, there ? K : 0, u[i]);
#pragma unroll
  for (int i = 0; i < GROUPS; ++i) {
    float amax = bf16_amax(u[i][0], u[i][1]);
#pragma unroll
    for (int o = 4; o; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
    const int c = (g0 + i) * 128 + lane * 16;
    if (!there || g0 + i >= Kb) continue;
    const float s = lin_scale(amax);
    if (c < K) *reinterpret_cast<uint4*>(x8 + (long long)m * x8s + c) = lin_codes(u[i], s);
    if (lane == 0) scale[(long long)(g0 + i) * ss + m] = s;
  }
}

// One CTA per 128 x 128 tile, which stays in registers between the maximum and the cast: 47 616 x 4 096 112 us = 5.2 TB/s, 24 576 x 4 096 61 us
// (once per weight).
__global__ void __launch_bounds__(256)
quantize_tiles_kernel(const __nv_bfloat16* __restrict__ w, int N, int K, long long ws, uint8_t* __restrict__ w8, long long w8s,
                      float* __restrict__ scale, long long ss, int Kb) {
  __shared__ float part[8];
  const int zero = grid_dep_wait();
  const int g = (int)(blockIdx.x % Kb), J = (int)(blockIdx.x / Kb), c = g * 128 + (threadIdx.x & 7) * 16 + zero;
  uint4 u[4][2];
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int n = J * 128 + i * 32 + (threadIdx.x >> 3);
    lin_load16(w + (long long)(n < N ? n : 0) * ws, c, n < N ? K : 0, u[i]);
    amax = fmaxf(amax, bf16_amax(u[i][0], u[i][1]));
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = amax;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) amax = fmaxf(amax, part[i]);
  const float s = lin_scale(amax);
  if (threadIdx.x == 0) scale[(long long)J * ss + g] = s;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int n = J * 128 + i * 32 + (threadIdx.x >> 3);
    if (n < N && c < K) *reinterpret_cast<uint4*>(w8 + (long long)n * w8s + c) = lin_codes(u[i], s);
  }
}

// ------------------------------------------------------------------ the product
struct LinearParams {
  const float *xs, *ws, *bias;
  const __nv_bfloat16* residual;
  __nv_bfloat16* out;
  long long xs_stride, ws_stride, out_stride, res_stride;
  int M, N, Kb, debug;
  int32_t* status;
  bool wide;                                              // rows of out begin on 32 bytes
};

// GELU (tanh form) 0.5 y (1 + tanh u) = y / (1 + exp(-2u)), u = sqrt(2/pi) (y + 0.044715 y^3); SiLU y / (1 + exp(-y)).
// The denominator, with the exponent formed in base 2 and kept below 2^60, so that the product of two denominators has a reciprocal that is a
// normal number; the numerator is kept above -64 (a NaN stays one), so that what is left of values that far out is below 2^-54.
template <int ACT>
__device__ __forceinline__ float lin_denominator(float y) {
  constexpr float LOG2E = 1.4426950408889634f, C = -2.f * 0.7978845608028654f * LOG2E;
  return 1.f + ex2(fminf(ACT == SVA_ACT_GELU ? y * fmaf(C * 0.044715f, y * y, C) : -LOG2E * y, 60.f));
}
__device__ __forceinline__ float lin_rcp(float d) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(d));
  return r;
}
__device__ __forceinline__ float lin_numerator(float y) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(y), "f"(-64.f));
  return r;
}
template <int ACT>
__device__ __forceinline__ float lin_act(float y) {
  return ACT == SVA_ACT_NONE ? y : lin_numerator(y) * lin_rcp(lin_denominator<ACT>(y));
}
// two at a time, one reciprocal for both: exponentials and reciprocals leave the SM at 16 a cycle, 4 096 cycles for two of each of 256 x 128 values.
// 8 192 x 2 048 x 8 192, us, in a short run: none 129, SiLU 146, GELU 150; 1 024 x 2 048 x 2 048: 9.5, 10.3, 10.6.
template <int ACT>
__device__ __forceinline__ void lin_act2(float& a, float& b) {
  if (ACT == SVA_ACT_NONE) return;
  const float da = lin_denominator<ACT>(a), db = lin_denominator<ACT>(b), r = lin_rcp(da * db);
  a = lin_numerator(a) * (r * db);
  b = lin_numerator(b) * (r * da);
}

__device__ __forceinline__ bool lin_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag));      // (a warp gives up together)
}

// A wait has run out: copies and MMAs still in flight get time to land before shared memory and TMEM go away.
static __device__ __noinline__ void lin_settle() {
  const long long t0 = clock64();
  while (clock64() - t0 < 2000000LL) __nanosleep(1000);
}

// Tiles in an order in which CTAs that run side by side share rows of x and of w: LIN_GROUP tile rows at a time, down each column.
static constexpr int LIN_GROUP = 16;
__device__ __forceinline__ void lin_tile(int i, int mt, int nt, int& m, int& n) {
  const int per = LIN_GROUP * nt, g = i / per, rows = min(LIN_GROUP, mt - g * LIN_GROUP), r = i - g * per;
  m = g * LIN_GROUP + r % rows;
  n = r / rows;
}

// Persistent CTAs, one per SM.  x and w tiles of 128 inputs come through a ring by TMA; the tensor cores multiply a group of 128 inputs
// into one of the accumulators in tensor memory; the sum warps take each group's product out, times its two scales, and add it up in
// registers, fp32 throughout.
//   PAIR   two CTAs make a tile of 256 tokens x 256 weights rows: each stages its 128 tokens and half of the weights rows, the first issues
//          the MMAs of both (cta_group::2): 32 KB from the L2 per CTA and group where a CTA by itself would need 48 KB for its 128 x 256
//   else   a CTA makes 128 x 128: problems that are too small to fill the device with pairs
//   SPLIT  the CTAs of a cluster take every split-th group of a 128 x 128 tile each and join their sums through distributed shared memory, in
//          the order of the CTAs: few tiles with many inputs
// Warps: eight sum, a thread owning one token and half of the tile's columns; then one that loads, one that issues the MMAs, one that brings the
// scales, and in a pair one that sees to the staging tiles (bias, residual, stores), else one that loads too: x and w have a warp each.
// A turn of any of these roles takes some 600 cycles of its own (barriers asked, instructions with their operands issued, barriers told), also
// where it waits for nothing: a pair's MMAs for one group of inputs take 512, those of a 128 x 128 tile 256.  So a turn of a CTA by itself is two
// groups, in loads, MMAs, scales and sums alike: 640 -> 470 cycles per group (1 024 x 16 384 x 2 048: 48.4 -> 37.2 us); two groups in the MMAs
// alone, the barriers asked a turn ahead or loads left out had changed nothing.  Its results go straight from the registers: there is no room
// for staging tiles beside three stages of two groups.
namespace lin {
constexpr uint32_t A_BYTES = 128 * 128, GROUP = 2 * A_BYTES;
constexpr uint32_t OUT_BYTES = 128 * 128;                 // staging tile, 128 tokens x 64 columns of bf16
constexpr int BUFS = 2, ACC = 256, SLOTS = 2 * BUFS;      // accumulators and their columns; scale slots, a float per column quarter and token
template <bool PAIR> struct Shape {
  static constexpr int SIDE = PAIR ? 256 : 128, COLS = SIDE / 2, SUM_WARPS = 8;      // columns of a sum warp
  static constexpr int TURN = PAIR ? 1 : 2;                 // groups of inputs per stage and accumulator
  static constexpr int UNITS = SIDE / 128;                  // an accumulator is one or two units with barriers of their own
  static constexpr int THREADS = 32 * (SUM_WARPS + 4);
  static constexpr int STAGES = PAIR ? 4 : 3, AHEAD = PAIR ? 2 : 4;      // groups whose scales are fetched together
  static constexpr uint32_t STAGE = TURN * GROUP, OUT = STAGES * STAGE;
  static constexpr int SMEM = 1024 + OUT + (PAIR ? SIDE / 64 * OUT_BYTES : 0);
  // registers of a thread that sums and of the others; the launch has 168 for each
  static constexpr int SUM_REGS = 216, HELPER_REGS = 72;
  static_assert(32 * SUM_WARPS * SUM_REGS + 128 * HELPER_REGS <= THREADS * 168, "setmaxnreg draws on the registers of the launch");
  static_assert(PAIR || SIDE * SIDE * 4 <= OUT, "the ring takes the sums that are exchanged");
};
}

template <bool PAIR, int ACT, bool SPLIT>
__global__ void __launch_bounds__(lin::Shape<PAIR>::THREADS, 1)
linear_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_o,
              const __grid_constant__ CUtensorMap tm_r, const LinearParams prm, int split) {
  using namespace lin;
  using S = Shape<PAIR>;
  constexpr int STAGES = S::STAGES, SIDE = S::SIDE, COLS = S::COLS, UNITS = S::UNITS, TURN = S::TURN, LOADER = S::SUM_WARPS;
  constexpr uint32_t STAGE = S::STAGE;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  __shared__ __align__(8) unsigned long long bars[2 * STAGES + 2 * BUFS * UNITS + 4];
  __shared__ __align__(16) float bias_s[2][COLS];
  __shared__ float scale_s[SLOTS][256];                    // x_scale * w_scale: [weights block of 128, or group][token]
  __shared__ uint32_t tmem_base_s;
  __shared__ int abort_s;
  volatile int* abort_flag = &abort_s;
  const uint32_t sbase = smem_u32(smem);
  const uint32_t bar_full = smem_u32(&bars[0]), bar_empty = bar_full + 8 * STAGES, bar_acc = bar_empty + 8 * STAGES;
  const uint32_t bar_free = bar_acc + 8 * BUFS * UNITS, bar_ready = bar_free + 8 * BUFS * UNITS, bar_staged = bar_ready + 16;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = PAIR ? (int)(blockIdx.x & 1) : 0, part = SPLIT ? (int)blockIdx.x % split : 0;
  const int first = PAIR ? (int)(blockIdx.x >> 1) : SPLIT ? (int)blockIdx.x / split : (int)blockIdx.x;
  const int mt = (prm.M + SIDE - 1) / SIDE, nt = (prm.N + SIDE - 1) / SIDE, tiles = mt * nt;
  const int step = PAIR ? (int)(gridDim.x >> 1) : SPLIT ? tiles : (int)gridDim.x;
  // this CTA's groups of inputs: all, or part, part + split, ... of them
  const int Kb = SPLIT ? (prm.Kb - part + split - 1) / split : prm.Kb;
  auto group = [&](int g) { return SPLIT ? part + g * split : g; };
  if (threadIdx.x == 0) {
    for (int i = 0; i < STAGES; ++i) { mbar_init(bar_full + 8 * i, PAIR ? 1 : 2); mbar_init(bar_empty + 8 * i, 1); }
    for (int i = 0; i < BUFS * UNITS; ++i) {              // full: by the MMAs and the scales; free: by eight warps, a pair's four in each CTA
      mbar_init(bar_acc + 8 * i, 2);
      mbar_init(bar_free + 8 * i, 8);
    }
    for (int i = 0; i < 2; ++i) { mbar_init(bar_ready + 8 * i, 1); mbar_init(bar_staged + 8 * i, 4); }
    abort_s = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    prefetch_tmap(&tm_x);
    prefetch_tmap(&tm_w);
    if (PAIR) prefetch_tmap(&tm_o);
    if (PAIR && prm.residual) prefetch_tmap(&tm_r);
  }
  if (warp == LOADER + 1) {
    if (PAIR) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_s)), "r"(512u) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_s)), "r"(512u) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  tc_fence_before();
  __syncthreads();
  if (PAIR) cluster_sync_all();                           // the other CTA's barriers are there
  tc_fence_after();
  const uint32_t tmem = tmem_base_s;
  const int zero = grid_dep_wait();

  if (warp >= LOADER) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(S::HELPER_REGS));
    if (warp == LOADER || (!PAIR && warp == LOADER + 3)) {
      // ---- loads; in a pair, the first CTA's barrier waits for the bytes of both; else a warp loads x, another w
      const uint32_t bar_lead = PAIR ? mapa(bar_full, 0) : bar_full;
      const bool loads_w = warp != LOADER;
      bool ok = true;
      int st = 0;
      uint32_t ph = 0;
      for (int i = first; i < tiles && ok; i += step) {
        int m, n;
        lin_tile(i, mt, nt, m, n);
        const int m0 = m * SIDE + rank * 128, n0 = n * SIDE + rank * 64;
        for (int g = 0; g < Kb; g += TURN) {
          ok = lin_wait(bar_empty + 8 * st, ph ^ 1u, abort_flag);
          if (!ok) break;
          if ((prm.debug & 1024) && g > 0) break;                              // test aid: the ring runs dry
          if (lane == 0) {
            const uint32_t dst = sbase + st * STAGE;
            if (PAIR) {
              if (rank == 0) mbar_expect_tx(bar_full + 8 * st, 2 * STAGE);
              tma_load_2d_pair(dst, &tm_x, bar_lead + 8 * st, g * 128, m0);
              tma_load_2d_pair(dst + A_BYTES, &tm_w, bar_lead + 8 * st, g * 128, n0);               // this CTA's half of unit 0,
              tma_load_2d_pair(dst + A_BYTES + 64 * 128, &tm_w, bar_lead + 8 * st, g * 128, n0 + 128);       // of unit 1
            } else {
              const CUtensorMap* tm = loads_w ? &tm_w : &tm_x;
              const uint32_t to = dst + (loads_w ? A_BYTES : 0u);
              const int row = loads_w ? n0 : m0;
              mbar_expect_tx(bar_full + 8 * st, (g + 1 < Kb ? 2 : 1) * A_BYTES);
              tma_load_2d(to, tm, bar_full + 8 * st, group(g) * 128, row);
              if (g + 1 < Kb && !(prm.debug & 1024)) tma_load_2d(to + GROUP, tm, bar_full + 8 * st, group(g + 1) * 128, row);
            }
          }
          __syncwarp();
          if (++st == STAGES) { st = 0; ph ^= 1u; }
        }
      }
      // in a pair, the MMAs' arrivals from the first CTA are all here before this one may go
      for (int s = 0; PAIR && ok && s < STAGES; ++s) {
        ok = lin_wait(bar_empty + 8 * st, ph ^ 1u, abort_flag);
        if (++st == STAGES) { st = 0; ph ^= 1u; }
      }
    } else if (warp == LOADER + 1 && rank == 0) {
      // ---- MMAs
      // A unit is 128 columns of the accumulator: 128 weights rows, in a pair 64 staged by each CTA.
      constexpr uint32_t IDESC = instr_desc(SIDE, 128, 0, false);
      const uint32_t el = elect_one();
      const uint64_t ad0 = smem_desc(sbase, 16, 1024), bd0 = smem_desc(sbase + A_BYTES, 16, 1024);
      bool ok = true;
      int st = 0, buf = 0;
      uint32_t ph = 0, bph = 0;
      for (int i = first; i < tiles && ok; i += step) {
        for (int g = 0; g < Kb && ok; g += TURN) {
          ok = lin_wait(bar_full + 8 * st, ph, abort_flag);
          const uint64_t ad = ad0 + (uint64_t)(st * (STAGE >> 4)), bd = bd0 + (uint64_t)(st * (STAGE >> 4));
#pragma unroll
          for (int u = 0; u < UNITS; ++u) {
            const int at = buf * UNITS + u;
            ok = ok && lin_wait(bar_free + 8 * at, bph ^ 1u, abort_flag);
            if (!ok) break;
            tc_fence_after();
            if (PAIR) {
#pragma unroll
              for (int kk = 0; kk < 4; ++kk)
                tc_mma_ss_f8_pair(tmem + at * 128, ad + 2 * kk, bd + u * (64 * 128 >> 4) + 2 * kk, IDESC, kk > 0 ? 1u : 0u, el);
              tc_commit_pair(bar_acc + 8 * at, el);
            } else {
#pragma unroll
              for (int kk = 0; kk < 4; ++kk) tc_mma_ss_f8(tmem + buf * ACC, ad + 2 * kk, bd + 2 * kk, IDESC, kk > 0 ? 1u : 0u, el);
              if (g + 1 < Kb) {
#pragma unroll
                for (int kk = 0; kk < 4; ++kk)
                  tc_mma_ss_f8(tmem + buf * ACC + 128, ad + (GROUP >> 4) + 2 * kk, bd + (GROUP >> 4) + 2 * kk, IDESC, kk > 0 ? 1u : 0u, el);
              }
              tc_commit(bar_acc + 8 * at, el);
            }
          }
          if (!ok) break;
          if (PAIR) tc_commit_pair(bar_empty + 8 * st, el); else tc_commit(bar_empty + 8 * st, el);
          if (++st == STAGES) { st = 0; ph ^= 1u; }
          if (++buf == BUFS) { buf = 0; bph ^= 1u; }
        }
      }
    } else if (warp == LOADER + 2) {
      // ---- scales: a lane has four tokens'; AHEAD groups' values are on their way while as many are handed over
      // A slot is free when the accumulator of BUFS turns ago is full: its MMAs began when the sum warps had given back the one of 2 BUFS
      // turns ago, whose scales were in the slot.
      constexpr int BLOCKS = SIDE / 128, AHEAD = S::AHEAD;
      int i = first, g = 0, c = 0;                           // next group to fetch, turns handed over
      const float *xs[4], *ws[BLOCKS];
      auto place = [&]() {
        int m, n;
        lin_tile(i, mt, nt, m, n);
        // (rows and columns that do not exist hold zeros: any scale will do)
#pragma unroll
        for (int j = 0; j < 4; ++j) xs[j] = prm.xs + min(m * SIDE + rank * 128 + 32 * j + lane, prm.M - 1) + zero;
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) ws[b] = prm.ws + min(n * BLOCKS + b, (prm.N - 1) / 128) * prm.ws_stride + zero;
      };
      if (i < tiles) place();
      struct Some { float x[AHEAD][4], w[AHEAD][BLOCKS]; int n; };
      auto fetch = [&](Some& t) {
        t.n = 0;
        if (i >= tiles) return;
        t.n = min(AHEAD, Kb - g);
#pragma unroll
        for (int q = 0; q < AHEAD; ++q) {
          const int at = group(min(g + q, Kb - 1));
#pragma unroll
          for (int j = 0; j < 4; ++j) t.x[q][j] = __ldg(xs[j] + at * prm.xs_stride);
#pragma unroll
          for (int b = 0; b < BLOCKS; ++b) t.w[q][b] = __ldg(ws[b] + at);
        }
        g += AHEAD;
        if (g >= Kb) {
          g = 0;
          i += step;
          if (i < tiles) place();
        }
      };
      auto hand_over = [&](const Some& t) {
#pragma unroll
        for (int q = 0; q < AHEAD; q += TURN) {
          if (q >= t.n) break;
          if (c >= BUFS) {
#pragma unroll
            for (int u = 0; u < UNITS; ++u)
              if (!lin_wait(bar_acc + 8 * (UNITS * (c % BUFS) + u), (uint32_t)(c / BUFS - 1) & 1u, abort_flag)) return false;
          }
#pragma unroll
          for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
            for (int j = 0; j < 4; ++j) scale_s[c % SLOTS][b * 128 + 32 * j + lane] = t.x[q][j] * t.w[q][b];
          if (TURN == 2) {                                   // (a group that does not exist: any scale will do)
#pragma unroll
            for (int j = 0; j < 4; ++j) scale_s[c % SLOTS][128 + 32 * j + lane] = t.x[q + TURN - 1][j] * t.w[q + TURN - 1][0];
          }
          __syncwarp();
          if (lane < UNITS) mbar_arrive(bar_acc + 8 * (UNITS * (c % BUFS) + lane));
          ++c;
        }
        return true;
      };
      Some a, b;
      fetch(a);
      while (a.n) {
        fetch(b);
        if (!hand_over(a) || !b.n) break;
        fetch(a);
        if (!hand_over(b)) break;
      }
    } else if (PAIR && warp == LOADER + 3) {
      // ---- staging tiles: the bias of their columns, what the result is added to, the stores
      bool ok = true;
      uint32_t ph = 0;
      for (int i = first; i < tiles && ok; i += step) {
        int m, n;
        lin_tile(i, mt, nt, m, n);
        const int m0 = m * SIDE + rank * 128;
        for (int h = 0; h < 2; ++h) {
          const int n0 = n * SIDE + h * COLS;
          for (int c = lane; c < COLS; c += 32) bias_s[h][c] = prm.bias && n0 + c < prm.N ? __ldg(prm.bias + n0 + c + zero) : 0.f;
          __syncwarp();
          if (lane == 0) {
            if (prm.residual) {                              // comes to where the result will be staged
              mbar_expect_tx(bar_ready + 8 * h, COLS / 64 * OUT_BYTES);
              for (int j = 0; j < COLS / 64; ++j)
                tma_load_2d(sbase + S::OUT + (h * (COLS / 64) + j) * OUT_BYTES, &tm_r, bar_ready + 8 * h, n0 + j * 64, m0);
            } else {
              mbar_arrive(bar_ready + 8 * h);
            }
          }
        }
        for (int h = 0; h < 2 && ok; ++h) {
          const int n0 = n * SIDE + h * COLS;
          ok = lin_wait(bar_staged + 8 * h, ph, abort_flag);
          if (ok && lane == 0 && m0 < prm.M) {
            for (int j = 0; j < COLS / 64; ++j)
              if (n0 + j * 64 < (prm.N & ~7)) tma_store_2d(&tm_o, sbase + S::OUT + (h * (COLS / 64) + j) * OUT_BYTES, n0 + j * 64, m0);
            bulk_commit();
          }
        }
        ph ^= 1u;
        if (lane == 0) bulk_wait_read0();                    // the staging tiles have been read
        __syncwarp();
      }
      if (lane == 0) bulk_wait0();
    }
    __syncwarp();
    if (SPLIT) cluster_sync_all();                        // (the sum warps' barrier below)
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(S::SUM_REGS));
    // ---- sums and epilogue
    const int wg = warp >> 2, row = (warp & 3) * 32 + lane;
    // (a pair's CTA: each group of four warps has a unit of its own, the other's half a group's time later; else half of the columns)
    const uint32_t taddr = tmem + ((uint32_t)((warp & 3) * 32) << 16) + wg * COLS;
    const float* scale = &scale_s[0][(PAIR ? wg * 128 : 0) + row];
    uint8_t* stage = smem + S::OUT + wg * (COLS / 64) * OUT_BYTES;
    const uint32_t free_lead = PAIR ? mapa(bar_free, 0) : bar_free;
    bool ok = true;
    int buf = 0, slot = 0;
    uint32_t bph = 0, rph = 0;
    // 64 columns come out at once and are added up; whether the next group's are there is asked before the last sums and used after them
    // (a wait whose answer is used at once costs a sum warp 100 to 250 cycles even where there is nothing to wait for).
    // 8 192 x 4 096 x 4 096, cycles per group of a pair: MMAs and loads alone 560 (MMAs of 256 columns) to 660 (of 128), with the accumulator
    // read 650, with the sums 768.  The MMA warp finds its barriers passed in nine turns of ten: what is left is the pace of the MMAs, which warps
    // that multiply and add without having anything to do with the product slow down as much (660 -> 890), and which goes with the power drawn:
    // 122 us = 2.25 PFLOP/s in a run of 20, 138 in one of 2 000, 107 with codes of zeros.  128 columns read between sums 32 at a time, no units:
    // 870; sixteen sum warps of 64 columns: 1 000.
    const uint32_t first_lane = lane == 0;
    uint32_t there = 0u;
    for (int i = first; i < tiles; i += step) {
      uint64_t acc[COLS / 2];
#pragma unroll
      for (int c = 0; c < COLS / 2; ++c) acc[c] = 0ull;
#pragma unroll 1
      for (int g = 0; g < Kb; g += TURN) {
        const int at = PAIR ? buf * UNITS + wg : buf;
        if (!__all_sync(0xffffffffu, there)) ok = lin_wait(bar_acc + 8 * at, bph, abort_flag);
        if (!ok) break;
        tc_fence_after();
        auto give_back = [&]() {
          tc_fence_before();
          if (PAIR) mbar_arrive_cluster_if(free_lead + 8 * at, first_lane);
          else mbar_arrive_if(bar_free + 8 * at, first_lane);
          const bool wraps = buf + 1 == BUFS;
          there = mbar_test(bar_acc + 8 * (wraps ? at - buf * UNITS : at + UNITS), wraps ? bph ^ 1u : bph);
        };
        auto add = [&](const uint32_t (&v)[64], float s, uint64_t* to) {
          const uint64_t s2 = pack2(s, s);
#pragma unroll
          for (int e = 0; e < 32; ++e) to[e] = fma2(pack2(__uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1])), s2, to[e]);
        };
        const uint32_t from = taddr + buf * ACC;
        uint32_t v[64];
        tmem_ld32(from, v);
        tmem_ld32(from + 32, v + 32);
        const float s = scale[slot * 256];
        tc_wait_ld64(v);
        if (PAIR) {
          add(v, s, acc);
          tmem_ld32(from + 64, v);
          tmem_ld32(from + 96, v + 32);
          tc_wait_ld64(v);
          give_back();
          add(v, s, acc + 32);
        } else if (g + 1 < Kb) {
          uint32_t w[64];                                    // the second group comes out while the first is added
          tmem_ld32(from + 128, w);
          tmem_ld32(from + 160, w + 32);
          const float s1 = scale[slot * 256 + 128];
          add(v, s, acc);
          tc_wait_ld64(w);
          give_back();
          add(w, s1, acc);
        } else {
          give_back();
          add(v, s, acc);
        }
        if (++buf == BUFS) { buf = 0; bph ^= 1u; }
        if (++slot == SLOTS) slot = 0;
      }
      int m, n;
      lin_tile(i, mt, nt, m, n);
      // eight columns of a token, straight to where they belong
      auto finish8 = [&](float (&y)[8], int tok, int col) {
        if (col >= prm.N) return;
        if (prm.bias) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (col + e < prm.N) y[e] += __ldg(prm.bias + col + e + zero);
        }
#pragma unroll
        for (int e = 0; e < 8; e += 2) lin_act2<ACT>(y[e], y[e + 1]);
        if (tok >= prm.M) return;
        __nv_bfloat16* to = prm.out + (long long)tok * prm.out_stride + col;
        const __nv_bfloat16* add = prm.residual + (long long)tok * prm.res_stride + col;
        if (col + 8 <= prm.N) {
          if (prm.residual) {
            const uint4 u = *reinterpret_cast<const uint4*>(add);
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) { y[2 * e] += bf16lo(w[e]); y[2 * e + 1] += bf16hi(w[e]); }
          }
          *reinterpret_cast<uint4*>(to) = make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
        } else {
#pragma unroll
          for (int e = 0; e < 7; ++e)
            if (col + e < prm.N) to[e] = __float2bfloat16_rn(y[e] + (prm.residual ? __bfloat162float(add[e]) : 0.f));
        }
      };
      if (SPLIT) {
        // the sums of the cluster's CTAs: everybody's into its own ring (which the MMAs are done with), then each finishes a part of the columns
        float* mine = reinterpret_cast<float*>(smem);
        if (ok) {
#pragma unroll
          for (int c = 0; c < COLS / 2; ++c) {
            float lo, hi;
            unpack2(acc[c], lo, hi);
            mine[(wg * COLS + 2 * c) * 128 + row] = lo;
            mine[(wg * COLS + 2 * c + 1) * 128 + row] = hi;
          }
        }
        __syncwarp();
        cluster_sync_all();
        if (!ok) break;
        auto join = [&](auto split_tag) {
          constexpr int Q = decltype(split_tag)::value, W = COLS / Q;          // columns of a thread
          const int c0 = part * 2 * W + wg * W;
          float v[Q][W];
#pragma unroll
          for (int q = 0; q < Q; ++q) {
            const uint32_t from = mapa(sbase + (uint32_t)(c0 * 128 + row) * 4u, q);
#pragma unroll
            for (int c = 0; c < W; ++c) v[q][c] = ld_cluster_f32(from + c * 512);
          }
#pragma unroll
          for (int c = 0; c < W; c += 8) {
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              y[e] = v[0][c + e];
#pragma unroll
              for (int q = 1; q < Q; ++q) y[e] += v[q][c + e];
            }
            finish8(y, m * SIDE + row, n * SIDE + c0 + c);
          }
        };
        if (split == 2) join(std::integral_constant<int, 2>{});
        else if (split == 4) join(std::integral_constant<int, 4>{});
        else join(std::integral_constant<int, 8>{});
        break;
      }
      if (!PAIR) {
        if (!ok) break;
        const int tok = m * SIDE + row, col = n * SIDE + wg * COLS;
        // straight code where all columns are there (what is optional in its midst ran at the pace of instruction fetches)
        auto straight = [&](auto bias_tag, auto res_tag) {
          constexpr bool BIAS = decltype(bias_tag)::value, RES = decltype(res_tag)::value;
          const bool there = tok < prm.M;
          const uint4* add = reinterpret_cast<const uint4*>(prm.residual + (RES ? (long long)(there ? tok : 0) * prm.res_stride + col : 0));
          uint4 r[COLS / 8], o[COLS / 8];
#pragma unroll
          for (int q = 0; q < COLS / 8; ++q) r[q] = RES ? add[q] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
          for (int q = 0; q < COLS / 8; ++q) {
            float y[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) unpack2(acc[q * 4 + e], y[2 * e], y[2 * e + 1]);
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (BIAS) y[e] += __ldg(prm.bias + col + q * 8 + e + zero);
#pragma unroll
            for (int e = 0; e < 8; e += 2) lin_act2<ACT>(y[e], y[e + 1]);
            const uint32_t w[4] = {r[q].x, r[q].y, r[q].z, r[q].w};
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (RES) { y[2 * e] += bf16lo(w[e]); y[2 * e + 1] += bf16hi(w[e]); }
            o[q] = make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
          }
          uint4* to = reinterpret_cast<uint4*>(prm.out + (long long)tok * prm.out_stride + col);
          if (!there) return;
          if (prm.wide) {
#pragma unroll
            for (int q = 0; q < COLS / 8; q += 2) stg32(to + q, o[q], o[q + 1]);
          } else {
#pragma unroll
            for (int q = 0; q < COLS / 8; ++q) to[q] = o[q];
          }
        };
        if (col + COLS <= prm.N) {
          if (prm.bias && prm.residual) straight(std::true_type{}, std::true_type{});
          else if (prm.bias) straight(std::true_type{}, std::false_type{});
          else if (prm.residual) straight(std::false_type{}, std::true_type{});
          else straight(std::false_type{}, std::false_type{});
        } else {
#pragma unroll
          for (int c = 0; c < COLS; c += 8) {
            float y[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) unpack2(acc[c / 2 + e], y[2 * e], y[2 * e + 1]);
            finish8(y, tok, col + c);
          }
        }
        continue;
      }
      const int m1 = m * SIDE + rank * 128, n1 = n * SIDE + wg * COLS;
      ok = ok && lin_wait(bar_ready + 8 * wg, rph, abort_flag);
      if (!ok) break;
      rph ^= 1u;
      // (two straight pieces of code without a branch: 16 times 8 columns with the optional parts in their midst ran at the pace of
      // instruction fetches, 4 000 cycles per tile)
      auto finish = [&](auto res_tag) {
        constexpr bool RES = decltype(res_tag)::value;
#pragma unroll
        for (int q = 0; q < COLS / 8; ++q) {                 // 8 columns at a time
          const float4 b0 = *reinterpret_cast<const float4*>(&bias_s[wg][q * 8]), b1 = *reinterpret_cast<const float4*>(&bias_s[wg][q * 8 + 4]);
          const float b[8] = {b0.x, b0.y, b0.z, b0.w, b1.x, b1.y, b1.z, b1.w};
          uint4* to = reinterpret_cast<uint4*>(stage + (q >> 3) * OUT_BYTES + row * 128 + (((q & 7) ^ (row & 7)) << 4));
          float y[8];
#pragma unroll
          for (int e = 0; e < 4; ++e) unpack2(acc[q * 4 + e], y[2 * e], y[2 * e + 1]);
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] += b[e];
#pragma unroll
          for (int e = 0; e < 8; e += 2) lin_act2<ACT>(y[e], y[e + 1]);
          if (RES) {
            const uint4 u = *to;
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) { y[2 * e] += bf16lo(w[e]); y[2 * e + 1] += bf16hi(w[e]); }
          }
          *to = make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
        }
      };
      if (prm.residual) finish(std::true_type{}); else finish(std::false_type{});
      // columns behind the last whole 16 bytes, which the tile store would overrun: a thread its row's
      const int last = (prm.N & ~7) - n1;
      if ((prm.N & 7) && last >= 0 && last < COLS && m1 + row < prm.M) {
        const __nv_bfloat16* from =
            reinterpret_cast<const __nv_bfloat16*>(stage + (last >> 6) * OUT_BYTES + row * 128 + ((((last >> 3) & 7) ^ (row & 7)) << 4));
        for (int e = 0; e < (prm.N & 7); ++e) prm.out[(long long)(m1 + row) * prm.out_stride + n1 + last + e] = from[e];
      }
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_staged + 8 * wg);
    }
  }
  __syncthreads();
  if (*abort_flag) lin_settle();
  tc_fence_before();
  __syncthreads();
  if (PAIR || SPLIT) cluster_sync_all();                  // nothing arrives at, and nobody reads from, a CTA that has gone
  if (threadIdx.x == 0 && *abort_flag && prm.status) atomicOr(prm.status, SVA_DEV_TIMEOUT);
  if (warp == LOADER + 1) {
    tc_fence_after();
    if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
}

// ------------------------------------------------------------------ few tokens
// Up to 64 tokens (conditioning vectors, a decoded token, a short prompt): the weights are the work, read once.  The weights rows are the
// M of the MMA and the tokens its N, so that a CTA takes 128 rows and no MMA row is empty; a cluster of CTAs splits the inputs of its 128 rows
// between them, so that small layers fill the device too, and joins the sums through distributed shared memory in the order of its CTAs
// (no workspace, no atomics: results repeat).  Several CTAs share an SM: what has to be in flight for the HBM is spread over all of them.
// 2 x 4 096 x 24 576 with its quantiser 21.2 us, 100 MB of weights.
// Warps 0-3: a thread sums one weights row for T tokens.  Warp 4 loads, warp 5 issues the MMAs.
namespace few {
constexpr int THREADS = 192, STAGES = 4, BUFS = 4;
template <int T> struct Shape {
  // CTAs per SM; groups whose scales are fetched together (four, for 16 tokens, would not leave room for a third CTA)
  static constexpr int PER_SM = T == 16 ? 3 : 2, AHEAD = T == 16 ? 2 : 4;
  static constexpr uint32_t STAGE = 128 * 128 + T * 128, COLUMNS = BUFS * T;      // (T columns per accumulator: 64 .. 256 in all)
  static constexpr int SMEM = 1024 + STAGES * STAGE;
  static_assert(T * 128 * 4 <= STAGES * STAGE, "the ring takes the sums that are exchanged");
};
}

template <int T>
__global__ void __launch_bounds__(few::THREADS, few::Shape<T>::PER_SM)
linear_few_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_w, const LinearParams prm, int split, int act) {
  using namespace few;
  using S = Shape<T>;
  constexpr int AHEAD = S::AHEAD;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  __shared__ __align__(8) unsigned long long bars[2 * STAGES + 2 * BUFS];
  __shared__ __align__(16) float scale_s[2][4][AHEAD][T];  // a warp's own copy of some groups' scales, to be read four at a time
  __shared__ uint32_t tmem_base_s;
  __shared__ int abort_s;
  volatile int* abort_flag = &abort_s;
  const uint32_t sbase = smem_u32(smem);
  const uint32_t bar_full = smem_u32(&bars[0]), bar_empty = bar_full + 8 * STAGES, bar_acc = bar_empty + 8 * STAGES, bar_free = bar_acc + 8 * BUFS;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = blockIdx.x % split, J = blockIdx.x / split;
  // this CTA's groups of inputs: rank, rank + split, ...: a cluster's CTAs read pieces of the weights rows that lie side by side
  const int mine_n = rank < prm.Kb ? (prm.Kb - rank + split - 1) / split : 0;
  if (threadIdx.x == 0) {
    for (int i = 0; i < STAGES; ++i) { mbar_init(bar_full + 8 * i, 1); mbar_init(bar_empty + 8 * i, 1); }
    for (int i = 0; i < BUFS; ++i) { mbar_init(bar_acc + 8 * i, 1); mbar_init(bar_free + 8 * i, 4); }
    abort_s = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    prefetch_tmap(&tm_x);
    // the weights can be on their way to the L2 while the kernel before this one (the quantiser of the tokens) still runs
    for (int i = 0; i < min(mine_n, STAGES); ++i) tma_prefetch_2d(&tm_w, (rank + i * split) * 128, J * 128);
  }
  if (warp == 5) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_s)), "r"(S::COLUMNS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_base_s;
  const int zero = grid_dep_wait();
  float acc[T];
#pragma unroll
  for (int t = 0; t < T; ++t) acc[t] = 0.f;
  bool ok = true;
  if (warp == 4) {
    for (int i = 0; i < mine_n; ++i) {
      const int st = i % STAGES, g = rank + i * split;
      ok = lin_wait(bar_empty + 8 * st, (uint32_t)(i / STAGES + 1) & 1u, abort_flag);
      if (!ok) break;
      if ((prm.debug & 1024) && i > 0) break;                                 // test aid: the ring runs dry
      if (lane == 0) {
        mbar_expect_tx(bar_full + 8 * st, S::STAGE);
        tma_load_2d(sbase + st * S::STAGE, &tm_w, bar_full + 8 * st, g * 128, J * 128);
        tma_load_2d(sbase + st * S::STAGE + 128 * 128, &tm_x, bar_full + 8 * st, g * 128, 0);
      }
      __syncwarp();
    }
  } else if (warp == 5) {
    constexpr uint32_t IDESC = instr_desc(128, T, 0, false);
    const uint32_t el = elect_one();
    const uint64_t ad0 = smem_desc(sbase, 16, 1024), bd0 = smem_desc(sbase + 128 * 128, 16, 1024);
    for (int i = 0; i < mine_n; ++i) {
      const int st = i % STAGES, buf = i % BUFS;
      ok = lin_wait(bar_free + 8 * buf, (uint32_t)(i / BUFS + 1) & 1u, abort_flag) &&
           lin_wait(bar_full + 8 * st, (uint32_t)(i / STAGES) & 1u, abort_flag);
      if (!ok) break;
      tc_fence_after();
      const uint64_t ad = ad0 + (uint64_t)(st * (S::STAGE >> 4)), bd = bd0 + (uint64_t)(st * (S::STAGE >> 4));
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) tc_mma_ss_f8(tmem + buf * T, ad + 2 * kk, bd + 2 * kk, IDESC, kk > 0 ? 1u : 0u, el);
      tc_commit(bar_empty + 8 * st, el);
      tc_commit(bar_acc + 8 * buf, el);
    }
  } else {
    const uint32_t taddr = tmem + ((uint32_t)(warp * 32) << 16);
    // a lane has a token's scale (tokens that do not exist hold zeros: any scale will do), times the weights'
    constexpr int PER = T > 32 ? 2 : 1;
    const float* xs[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) xs[j] = prm.xs + min((lane + 32 * j) % T, prm.M - 1) + zero;
    const float* ws = prm.ws + J * prm.ws_stride + zero;
    // The scales of AHEAD groups at a time, fetched while those before them are used (one group ahead, a fetch of 800 cycles was what a group took).
    float nx[AHEAD][PER], nw[AHEAD];
    auto fetch = [&](int i) {
#pragma unroll
      for (int q = 0; q < AHEAD; ++q) {
        const int at = rank + min(i + q, mine_n - 1) * split;
#pragma unroll
        for (int j = 0; j < PER; ++j) nx[q][j] = __ldg(xs[j] + at * prm.xs_stride);
        nw[q] = __ldg(ws + at);
      }
    };
    if (mine_n) fetch(0);
#pragma unroll 1
    for (int i = 0; i < mine_n; ++i) {
      const int buf = i % BUFS;
      float (*block)[T] = scale_s[i / AHEAD & 1][warp];     // (the other one may still be read by a lane that is behind)
      if (i % AHEAD == 0) {
#pragma unroll
        for (int q = 0; q < AHEAD; ++q)
#pragma unroll
          for (int j = 0; j < PER; ++j)
            if (lane < T) block[q][lane + 32 * j] = nx[q][j] * nw[q];
        if (i + AHEAD < mine_n) fetch(i + AHEAD);
        __syncwarp();
      }
      const float* s = block[i % AHEAD];
      ok = lin_wait(bar_acc + 8 * buf, (uint32_t)(i / BUFS) & 1u, abort_flag);
      if (!ok) break;
      tc_fence_after();
      constexpr int C = T < 32 ? T : 32;                    // tokens taken out of the accumulator at a time
#pragma unroll
      for (int c = 0; c < T / C; ++c) {
        uint32_t v[C];
        if constexpr (C == 32) tmem_ld32(taddr + buf * T + c * C, v);
        else tmem_ld16(taddr + buf * T + c * C, v);
        float4 f[C / 4];                                    // (read while the accumulator is on its way)
#pragma unroll
        for (int e = 0; e < C / 4; ++e) f[e] = *reinterpret_cast<const float4*>(s + c * C + 4 * e);
        if constexpr (C == 32) tc_wait_ld32(v);
        else tc_wait_ld16(v);
        if (c + 1 == T / C) {
          tc_fence_before();
          mbar_arrive_if(bar_free + 8 * buf, lane == 0);
        }
#pragma unroll
        for (int e = 0; e < C; e += 4) {
          float* a = acc + c * C + e;
          a[0] = fmaf(__uint_as_float(v[e]), f[e / 4].x, a[0]);
          a[1] = fmaf(__uint_as_float(v[e + 1]), f[e / 4].y, a[1]);
          a[2] = fmaf(__uint_as_float(v[e + 2]), f[e / 4].z, a[2]);
          a[3] = fmaf(__uint_as_float(v[e + 3]), f[e / 4].w, a[3]);
        }
      }
    }
  }
  // ---- join: each CTA of the cluster finishes T / split tokens
  const int n = J * 128 + (int)threadIdx.x;
  auto finish = [&](float y, int t) {
    if (t >= prm.M || n >= prm.N) return;
    if (prm.bias) y += __ldg(prm.bias + n + zero);
    y = act == SVA_ACT_GELU ? lin_act<SVA_ACT_GELU>(y) : act == SVA_ACT_SILU ? lin_act<SVA_ACT_SILU>(y) : y;
    if (prm.residual) y += __bfloat162float(prm.residual[(long long)t * prm.res_stride + n]);
    prm.out[(long long)t * prm.out_stride + n] = __float2bfloat16_rn(y);
  };
  if (split == 1) {
    if (warp < 4 && ok) {
#pragma unroll
      for (int t = 0; t < T; ++t) finish(acc[t], t);
    }
  } else {
    float* mine = reinterpret_cast<float*>(smem);                              // (the MMAs that read the ring are done: their sums are here)
    if (warp < 4 && ok) {
#pragma unroll
      for (int t = 0; t < T; ++t) mine[t * 128 + threadIdx.x] = acc[t];
    }
    __syncwarp();
    cluster_sync_all();
    // sixteen values on their way at a time: a read of another CTA's shared memory takes several hundred cycles
    auto join = [&](auto split_tag) {
      constexpr int SPLIT = decltype(split_tag)::value, BATCH = 16 / SPLIT < T / SPLIT ? 16 / SPLIT : T / SPLIT;
#pragma unroll 1
      for (int t = rank * (T / SPLIT); t < (rank + 1) * (T / SPLIT) && t < prm.M; t += BATCH) {
        float v[BATCH][SPLIT];
#pragma unroll
        for (int e = 0; e < BATCH; ++e)
#pragma unroll
          for (int q = 0; q < SPLIT; ++q) v[e][q] = ld_cluster_f32(mapa(sbase + (uint32_t)((t + e) * 128 + threadIdx.x) * 4u, q));
#pragma unroll
        for (int e = 0; e < BATCH; ++e) {
          float y = v[e][0];
#pragma unroll
          for (int q = 1; q < SPLIT; ++q) y += v[e][q];
          finish(y, t + e);
        }
      }
    };
    if (warp < 4 && ok) {
      if (split == 2) join(std::integral_constant<int, 2>{});
      else if (split == 4) join(std::integral_constant<int, 4>{});
      else join(std::integral_constant<int, 8>{});
    }
    __syncwarp();
    cluster_sync_all();                                                         // nobody's sums go before they were read
  }
  if (*abort_flag) lin_settle();
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag && prm.status) atomicOr(prm.status, SVA_DEV_TIMEOUT);
  if (warp == 5) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::COLUMNS) : "memory");
  }
}

// ------------------------------------------------------------------ host side
typedef CUresult (*lin_encode_fn_t)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                    const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                    CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static lin_encode_fn_t lin_encode() {
  static lin_encode_fn_t fn = nullptr;
  if (!fn) {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult qres;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &qres) != cudaSuccess ||
        qres != cudaDriverEntryPointSuccess)
      return nullptr;
    fn = reinterpret_cast<lin_encode_fn_t>(p);
  }
  return fn;
}
// rows x inner map (elements of elem bytes, byte stride between rows), box = 128 bytes x box_rows, 128-byte swizzle
static int lin_map(CUtensorMap* map, const void* ptr, long long inner, long long rows, long long stride, int elem, int box_rows) {
  lin_encode_fn_t enc = lin_encode();
  if (!enc) return SVA_ERR_CUDA;
  cuuint64_t dims[2] = {(cuuint64_t)inner, (cuuint64_t)rows};
  cuuint64_t st[1] = {(cuuint64_t)stride};
  cuuint32_t box[2] = {(cuuint32_t)(128 / elem), (cuuint32_t)box_rows};
  cuuint32_t estr[2] = {1, 1};
  return enc(map, elem == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(ptr), dims, st, box, estr,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS ? SVA_OK : SVA_ERR_CUDA;
}

static int g_debug_lin = 0;
void lin_set_debug_mode(int v) { g_debug_lin = v; }
int lin_set_wait_limit(long long cycles) { return set_wait_limit(cycles); }

static int lin_sms(int* sms) {
  static int cached[64];
  static DeviceOnce once;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return SVA_ERR_CUDA;
  const int rc = once.run([&] {
    return cudaDeviceGetAttribute(&cached[dev], cudaDevAttrMultiProcessorCount, dev) == cudaSuccess && cached[dev] > 0;
  });
  *sms = cached[dev];
  return rc;
}

int launch_quantize_rows(const sva_linear_t* p, const void* x, void* x8, float* x_scale, cudaStream_t st) {
  const int Kb = (p->K + 127) / 128;
  const long long rows = (p->M + 31) / 32;
  // Four groups per thread keep 128 bytes of it in flight; where that leaves SMs idle, one group and four times the CTAs.
  const bool four = rows * ((Kb + 3) / 4) >= 148;
  const int tiles = four ? (Kb + 3) / 4 : Kb;
  if (rows * tiles > 0x7fffffffLL) return SVA_ERR_UNSUPPORTED;
  note_choice(four ? 4 : 1);
  return launch_dep(four ? quantize_rows_kernel<4> : quantize_rows_kernel<1>, dim3((unsigned)(rows * tiles)), 256, 0, st, (const __nv_bfloat16*)x,
                    p->M, p->K, (long long)p->x_stride, (uint8_t*)x8, (long long)p->x8_stride, x_scale, (long long)p->x_scale_stride, tiles);
}

int launch_quantize_tiles(const sva_linear_t* p, const void* w, void* w8, float* w_scale, cudaStream_t st) {
  const int Kb = (p->K + 127) / 128;
  const long long tiles = (long long)Kb * ((p->N + 127) / 128);
  if (tiles > 0x7fffffffLL) return SVA_ERR_UNSUPPORTED;
  return launch_dep(quantize_tiles_kernel, dim3((unsigned)tiles), 256, 0, st, (const __nv_bfloat16*)w, p->N, p->K, (long long)p->w_stride,
                    (uint8_t*)w8, (long long)p->w8_stride, w_scale, (long long)p->w_scale_stride, Kb);
}

// How many clusters of `ctas` CTAs of a kernel the current device, or the part of it that this process has, holds at once.
template <typename K>
static int lin_clusters(K kern, int threads, int smem, int ctas) {
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = (unsigned)ctas;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  int n = 0;
  if (cudaOccupancyMaxActiveClusters(&n, kern, &cfg) == cudaSuccess) return n;
  (void)cudaGetLastError();
  return 0;
}

// split: CTAs that share the inputs of a tile (SPLIT only)
template <bool PAIR, int ACT, bool SPLIT = false>
static int launch_linear_tiles(const sva_linear_t* p, const void* x8, const void* w8, void* out, const LinearParams& prm, int sms,
                               cudaStream_t st) {
  static DeviceOnce once;
  static int held[64][4];                                   // clusters of 1, 2, 4, 8 CTAs
  auto kern = linear_kernel<PAIR, ACT, SPLIT>;
  using S = lin::Shape<PAIR>;
  constexpr int SIDE = S::SIDE, CTAS = PAIR ? 2 : 1, SMEM = S::SMEM;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return SVA_ERR_CUDA;
  int rc = once.run([&] {
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM) != cudaSuccess) return false;
    for (int j = 1; j < (SPLIT ? 4 : PAIR ? 2 : 1); ++j) held[dev][j] = lin_clusters(kern, S::THREADS, SMEM, 1 << j);
    return true;
  });
  if (rc) return rc;
  if (PAIR && (held[dev][1] == 0 || prm.debug & 64)) return launch_linear_tiles<false, ACT>(p, x8, w8, out, prm, sms, st);
  const long long tiles = (long long)((p->M + SIDE - 1) / SIDE) * ((p->N + SIDE - 1) / SIDE);
  int split = 1;
  if (SPLIT) {
    // As many as all tiles' clusters run at once with, if that saves more than the joining of the sums takes, some fourteen groups' time, and
    // leaves a CTA two turns.  us, without / split in 2, 4, 8: 65 x 4 096 x 4 096 11.2 / 10.1, 9.5, 9.6, 512 x 4 096 x 2 048 12.3 / 10.8, but
    // 65 x 2 048 x 1 024 (sixteen groups) 7.5 / 8.0, 7.7, 8.5, 100 x 1 024 x 512 6.1 / 7.0, 7.4, 8.1.
    for (int j = 1; j < 4 && !(prm.debug & 64) && tiles <= held[dev][j]; ++j)
      if (prm.Kb > (prm.Kb + (1 << j) - 1) / (1 << j) + 14 && prm.Kb >= 4 << j) split = 1 << j;
    if (split == 1) return launch_linear_tiles<false, ACT>(p, x8, w8, out, prm, sms, st);
  }
  CUtensorMap tx, tw, to, tr;
  if ((rc = lin_map(&tx, x8, p->K, p->M, p->x8_stride, 1, 128))) return rc;
  if ((rc = lin_map(&tw, w8, p->K, p->N, p->w8_stride, 1, PAIR ? 64 : 128))) return rc;
  // (a tile store writes whole 16-byte pieces, also beyond an inner extent that ends within one: it gets the whole pieces only; there are some,
  // since pairs never need fewer rounds for up to 128 columns)
  to = tr = tx;
  if (PAIR && (rc = lin_map(&to, out, p->N & ~7, p->M, 2 * p->out_stride, 2, 128))) return rc;
  if (PAIR && prm.residual && (rc = lin_map(&tr, prm.residual, p->N, p->M, 2 * p->residual_stride, 2, 128))) return rc;
  if (tiles > 0x7fffffffLL - sms) return SVA_ERR_UNSUPPORTED;
  note_choice(PAIR ? 4 : SPLIT ? 3 : 2);
  const long long most = sms / CTAS;
  const int per = SPLIT ? split : CTAS;
  return launch_dep_cluster(per, kern, dim3((unsigned)(per * (SPLIT || tiles < most ? tiles : most))), S::THREADS, SMEM, st, tx, tw, to, tr, prm,
                            split);
}

template <bool PAIR, bool SPLIT = false>
static int launch_linear_act(const sva_linear_t* p, const void* x8, const void* w8, void* out, const LinearParams& prm, int sms, cudaStream_t st) {
  return p->act == SVA_ACT_GELU ? launch_linear_tiles<PAIR, SVA_ACT_GELU, SPLIT>(p, x8, w8, out, prm, sms, st)
       : p->act == SVA_ACT_SILU ? launch_linear_tiles<PAIR, SVA_ACT_SILU, SPLIT>(p, x8, w8, out, prm, sms, st)
                                : launch_linear_tiles<PAIR, SVA_ACT_NONE, SPLIT>(p, x8, w8, out, prm, sms, st);
}

template <int T>
static int launch_linear_few(const sva_linear_t* p, const void* x8, const void* w8, const LinearParams& prm, int sms, cudaStream_t st) {
  using S = few::Shape<T>;
  static DeviceOnce once;
  static int largest[64];                                   // CTAs in a cluster
  auto kern = linear_few_kernel<T>;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return SVA_ERR_CUDA;
  int rc = once.run([&] {
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM) != cudaSuccess) return false;
    largest[dev] = 1;
    for (int c = 2; c <= 8 && lin_clusters(kern, few::THREADS, S::SMEM, c) > 0; c *= 2) largest[dev] = c;
    return true;
  });
  if (rc) return rc;
  CUtensorMap tx, tw;
  if ((rc = lin_map(&tx, x8, p->K, p->M, p->x8_stride, 1, T))) return rc;
  if ((rc = lin_map(&tw, w8, p->K, p->N, p->w8_stride, 1, 128))) return rc;
  const int rows = (p->N + 127) / 128;
  // The inputs are split while all CTAs still run at once: the HBM then has the most in flight, and all end together.
  const int most = prm.debug & 64 ? 1 : largest[dev];     // (test aid: as on a device that holds no clusters)
  int split = 1;
  while (split < most && 2 * split <= prm.Kb && (long long)rows * split * 2 <= (long long)sms * S::PER_SM) split *= 2;
  note_choice(1);
  return launch_dep_cluster(split, kern, dim3((unsigned)(rows * split)), few::THREADS, S::SMEM, st, tx, tw, prm, split, p->act);
}

int launch_linear(const sva_linear_t* p, const void* x8, const float* x_scale, const void* w8, const float* w_scale, void* out,
                  const float* bias, const void* residual, int32_t* status, cudaStream_t st) {
  int sms = 0, rc = lin_sms(&sms);
  if (rc) return rc;
  LinearParams prm;
  prm.xs = x_scale; prm.ws = w_scale; prm.bias = bias;
  prm.residual = (const __nv_bfloat16*)residual; prm.out = (__nv_bfloat16*)out;
  prm.xs_stride = p->x_scale_stride; prm.ws_stride = p->w_scale_stride; prm.out_stride = p->out_stride; prm.res_stride = p->residual_stride;
  prm.M = p->M; prm.N = p->N; prm.Kb = (p->K + 127) / 128;
  prm.debug = g_debug_lin;
  prm.status = status;
  prm.wide = (reinterpret_cast<uintptr_t>(out) & 31u) == 0 && (p->out_stride & 15) == 0;
  if (p->M <= 16) return launch_linear_few<16>(p, x8, w8, prm, sms, st);
  if (p->M <= 32) return launch_linear_few<32>(p, x8, w8, prm, sms, st);
  if (p->M <= 64) return launch_linear_few<64>(p, x8, w8, prm, sms, st);
  // A pair takes some 770 cycles for a group of inputs of its 256 x 256, a CTA by itself 470 for its 128 x 128: whichever needs less for its
  // rounds over the device.  us, in pairs / without: 1 024 x 2 048 x 4 096 13.8 / 14.8 (one round, two), 768 x 4 096 x 4 096 20.1 / 22.1 (one, two),
  // 1 024 x 2 048 x 6 144 21.7 / 20.6 (two, three), 2 048 x 4 096 x 4 096 35.6 / 41.3 (two, four), 512 x 2 048 x 2 048 12.3 / 8.5 (one each).
  auto rounds = [&](long long side, int places) {
    return (((p->M + side - 1) / side) * ((p->N + side - 1) / side) + places - 1) / places;
  };
  if (5 * rounds(256, sms > 1 ? sms / 2 : 1) <= 3 * rounds(128, sms)) return launch_linear_act<true>(p, x8, w8, out, prm, sms, st);
  return 2 * rounds(128, 1) <= sms ? launch_linear_act<false, true>(p, x8, w8, out, prm, sms, st)
                                   : launch_linear_act<false>(p, x8, w8, out, prm, sms, st);
}

}  // namespace sva
