// Linear layers in 8-bit floating point: e4m3 codes with one fp32 scale per token and 128 inputs for the activations, one per
// 128 x 128 tile for the weights (the paper's deployments run their projections and FFNs in low-bit formats and fuse GEMM + GELU and
// GEMM + residual).
//     y[m,n] = sum_g sx[g,m] sw[n/128,g] sum_{k in group g} x8[m,k] w8[n,k],   out = bf16(act(y + bias[n]) + residual[m,n])
//   quantize_rows_kernel, quantize_tiles_kernel   the codes (HBM-bound passes)
//   linear_kernel                                 the product
#include "tc_ptx.cuh"

namespace sva {

// ------------------------------------------------------------------ quantisers
__device__ __noinline__ float lin_div_slow(float a, float b) { return __fdiv_rn(a, b); }

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
__device__ __forceinline__ float lin_amax(const uint4 (&u)[2]) {
  const uint32_t w[8] = {u[0].x, u[0].y, u[0].z, u[0].w, u[1].x, u[1].y, u[1].z, u[1].w};
  uint32_t m = 0u;
#pragma unroll
  for (int e = 0; e < 8; ++e) asm("max.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(m), "r"(w[e] & 0x7fff7fffu));
  return __uint_as_float(max(m << 16, m & 0xffff0000u));
}
__device__ __forceinline__ float lin_scale(float amax) { return amax == 0.f ? 1.0f : __fdiv_rn(amax, 448.0f); }
// the codes of 16 values: the correctly rounded fp32 quotients, rounded to e4m3
__device__ __forceinline__ uint4 lin_codes(const uint4 (&u)[2], float s) {
  const uint32_t w[8] = {u[0].x, u[0].y, u[0].z, u[0].w, u[1].x, u[1].y, u[1].z, u[1].w};
  uint32_t c[4];
  if (div_fast_ok(s)) {
    const float r = __frcp_rn(s);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      c[e] = __byte_perm(e4m3x2(div_fast(bf16lo(w[2 * e]), s, r), div_fast(bf16hi(w[2 * e]), s, r)),
                         e4m3x2(div_fast(bf16lo(w[2 * e + 1]), s, r), div_fast(bf16hi(w[2 * e + 1]), s, r)), 0x5410);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      c[e] = __byte_perm(e4m3x2(lin_div_slow(bf16lo(w[2 * e]), s), lin_div_slow(bf16hi(w[2 * e]), s)),
                         e4m3x2(lin_div_slow(bf16lo(w[2 * e + 1]), s), lin_div_slow(bf16hi(w[2 * e + 1]), s)), 0x5410);
  }
  return make_uint4(c[0], c[1], c[2], c[3]);
}

// A CTA takes 32 rows x GROUPS groups: 8 lanes per row and group, so that a group's maximum is three shuffles and the 32 scales of
// a group leave side by side; a thread has GROUPS groups of its row in flight.
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
    float amax = lin_amax(u[i]);
#pragma unroll
    for (int o = 4; o; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
    const int c = (g0 + i) * 128 + lane * 16;
    if (!there || g0 + i >= Kb) continue;
    const float s = lin_scale(amax);
    if (c < K) *reinterpret_cast<uint4*>(x8 + (long long)m * x8s + c) = lin_codes(u[i], s);
    if (lane == 0) scale[(long long)(g0 + i) * ss + m] = s;
  }
}

// One CTA per 128 x 128 tile, which stays in registers between the maximum and the cast.
__global__ void __launch_bounds__(256)
quantize_tiles_kernel(const __nv_bfloat16* __restrict__ w, int N, int K, long long ws, uint8_t* __restrict__ w8, long long w8s,
                      float* __restrict__ scale, long long ss) {
  __shared__ float part[8];
  const int zero = grid_dep_wait();
  const int g = blockIdx.x, J = blockIdx.y, c = g * 128 + (threadIdx.x & 7) * 16 + zero;
  uint4 u[4][2];
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int n = J * 128 + i * 32 + (threadIdx.x >> 3);
    lin_load16(w + (long long)(n < N ? n : 0) * ws, c, n < N ? K : 0, u[i]);
    amax = fmaxf(amax, lin_amax(u[i]));
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
  long long xs_stride, ws_stride, out_stride;
  int M, N, Kb, debug;
  int32_t* status;
};

// GELU (tanh form) 0.5 y (1 + tanh u) = y / (1 + exp(-2u)), u = sqrt(2/pi) (y + 0.044715 y^3); SiLU y / (1 + exp(-y)).  The exponent is
// formed in base 2 and kept below 2^126, where its reciprocal is still a normal number.
template <int ACT>
__device__ __forceinline__ float lin_act(float y) {
  if (ACT == SVA_ACT_NONE) return y;
  constexpr float LOG2E = 1.4426950408889634f, C = -2.f * 0.7978845608028654f * LOG2E;
  const float z = ACT == SVA_ACT_GELU ? y * fmaf(C * 0.044715f, y * y, C) : -LOG2E * y;
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + ex2(fminf(z, 126.f))));
  return y * r;
}

__device__ __forceinline__ bool lin_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag));      // (a warp gives up together)
}

// A barrier of the four warps of one epilogue group (id 1 or 2), and whether all of them may go on.
__device__ __forceinline__ bool lin_group_all(bool ok, int id) {
  uint32_t r;
  asm volatile("{\n.reg .pred p, q;\nsetp.ne.b32 p, %1, 0;\nbarrier.cta.red.and.pred q, %2, 128, p;\nselp.u32 %0, 1, 0, q;\n}"
               : "=r"(r) : "r"((uint32_t)ok), "r"(id) : "memory");
  return r != 0u;
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
// into one of the accumulators in tensor memory; eight warps take each group's product out, times its two scales, and add it up in
// registers, fp32 throughout.
//   PAIR   two CTAs make a tile of 256 tokens x 256 weights rows: each stages its 128 tokens and half of the weights rows, the first issues
//          the MMAs of both (cta_group::2): 32 KB from the L2 per CTA and group where a CTA by itself would need 48 KB for its
//          128 x 256; what bounds that is the way from the L2.
//   else   a CTA makes 128 x 128: problems that are too small to fill the device with pairs.
// Warps 0-7: a thread owns one token and half of the tile's columns.  Warp 8 loads, warp 9 issues the MMAs.
namespace lin {
constexpr int THREADS = 384;                              // (warps 10 and 11 only complete a warpgroup)
constexpr int SUM_REGS = 232, HELPER_REGS = 40;
static_assert(256 * SUM_REGS + 128 * HELPER_REGS <= THREADS * 168, "setmaxnreg draws on the registers of the launch");
constexpr uint32_t A_BYTES = 128 * 128, STAGE = 2 * A_BYTES;
constexpr uint32_t OUT_BYTES = 128 * 128;                 // staging tile, 128 tokens x 64 columns of bf16
template <bool PAIR> struct Shape {                       // (227 KB: the staging tiles of all columns, the rest is ring)
  static constexpr int OUTS = PAIR ? 4 : 2, STAGES = PAIR ? 5 : 6;
  static constexpr uint32_t OUT = STAGES * STAGE;
  static constexpr int SMEM = 1024 + OUT + OUTS * OUT_BYTES;
};
}

template <bool PAIR, int ACT>
__global__ void __launch_bounds__(lin::THREADS, 1)
linear_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_o,
              const __grid_constant__ CUtensorMap tm_r, const LinearParams prm) {
  using namespace lin;
  using S = Shape<PAIR>;
  constexpr int STAGES = S::STAGES;
  constexpr int BM = PAIR ? 256 : 128, BN = PAIR ? 256 : 128, BUFS = 512 / BN, COLS = BN / 2;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  __shared__ __align__(8) unsigned long long bars[2 * STAGES + 2 * BUFS + 2];
  __shared__ uint32_t tmem_base_s;
  __shared__ int abort_s;
  volatile int* abort_flag = &abort_s;
  const uint32_t sbase = smem_u32(smem);
  const uint32_t bar_full = smem_u32(&bars[0]), bar_empty = bar_full + 8 * STAGES, bar_acc = bar_empty + 8 * STAGES, bar_free = bar_acc + 8 * BUFS,
                 bar_res = bar_free + 8 * BUFS;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = PAIR ? (int)(blockIdx.x & 1) : 0, first = PAIR ? (int)(blockIdx.x >> 1) : (int)blockIdx.x;
  const int step = PAIR ? (int)(gridDim.x >> 1) : (int)gridDim.x;
  const int mt = (prm.M + BM - 1) / BM, nt = (prm.N + BN - 1) / BN, tiles = mt * nt, Kb = prm.Kb;
  if (threadIdx.x == 0) {
    for (int i = 0; i < STAGES; ++i) { mbar_init(bar_full + 8 * i, 1); mbar_init(bar_empty + 8 * i, 1); }
    for (int i = 0; i < BUFS; ++i) { mbar_init(bar_acc + 8 * i, 1); mbar_init(bar_free + 8 * i, PAIR ? 16 : 8); }
    for (int i = 0; i < 2; ++i) mbar_init(bar_res + 8 * i, 1);
    abort_s = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    prefetch_tmap(&tm_x);
    prefetch_tmap(&tm_w);
    prefetch_tmap(&tm_o);
    if (prm.residual) prefetch_tmap(&tm_r);
  }
  if (warp == 9) {
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

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(HELPER_REGS));
    if (warp == 8) {
      // ---- loads; in a pair, the first CTA's barrier waits for the bytes of both
      const uint32_t bar_lead = PAIR ? mapa(bar_full, 0) : bar_full;
      bool ok = true;
      int st = 0;
      uint32_t ph = 0;
      for (int i = first; i < tiles && ok; i += step) {
        int m, n;
        lin_tile(i, mt, nt, m, n);
        const int m0 = m * BM + rank * 128, n0 = n * BN + rank * 128;
        for (int g = 0; g < Kb; ++g) {
          ok = lin_wait(bar_empty + 8 * st, ph ^ 1u, abort_flag);
          if (!ok) break;
          if ((prm.debug & 1024) && g > 0) break;                              // test aid: the ring runs dry
          if (lane == 0) {
            const uint32_t dst = sbase + st * STAGE;
            if (PAIR) {
              if (rank == 0) mbar_expect_tx(bar_full + 8 * st, 2 * STAGE);
              tma_load_2d_pair(dst, &tm_x, bar_lead + 8 * st, g * 128, m0);
              tma_load_2d_pair(dst + A_BYTES, &tm_w, bar_lead + 8 * st, g * 128, n0);
            } else {
              mbar_expect_tx(bar_full + 8 * st, STAGE);
              tma_load_2d(dst, &tm_x, bar_full + 8 * st, g * 128, m0);
              tma_load_2d(dst + A_BYTES, &tm_w, bar_full + 8 * st, g * 128, n0);
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
    } else if (warp == 9 && rank == 0) {
      // ---- MMAs
      constexpr uint32_t IDESC = instr_desc(BM, BN, 0, false);
      const uint32_t el = elect_one();
      const uint64_t ad0 = smem_desc(sbase, 16, 1024), bd0 = smem_desc(sbase + A_BYTES, 16, 1024);
      bool ok = true;
      int st = 0, buf = 0;
      uint32_t ph = 0, bph = 0;
      for (int i = first; i < tiles && ok; i += step) {
        for (int g = 0; g < Kb; ++g) {
          ok = lin_wait(bar_free + 8 * buf, bph ^ 1u, abort_flag) && lin_wait(bar_full + 8 * st, ph, abort_flag);
          if (!ok) break;
          tc_fence_after();
          const uint64_t ad = ad0 + (uint64_t)(st * (STAGE >> 4)), bd = bd0 + (uint64_t)(st * (STAGE >> 4));
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) {
            if (PAIR) tc_mma_ss_f8_pair(tmem + buf * BN, ad + 2 * kk, bd + 2 * kk, IDESC, kk > 0 ? 1u : 0u, el);
            else tc_mma_ss_f8(tmem + buf * BN, ad + 2 * kk, bd + 2 * kk, IDESC, kk > 0 ? 1u : 0u, el);
          }
          if (PAIR) {
            tc_commit_pair(bar_empty + 8 * st, el);
            tc_commit_pair(bar_acc + 8 * buf, el);
          } else {
            tc_commit(bar_empty + 8 * st, el);
            tc_commit(bar_acc + 8 * buf, el);
          }
          if (++st == STAGES) { st = 0; ph ^= 1u; }
          if (++buf == BUFS) { buf = 0; bph ^= 1u; }
        }
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(SUM_REGS));
    // ---- sums and epilogue
    const int wg = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t taddr = tmem + ((uint32_t)((warp & 3) * 32) << 16) + wg * COLS;
    const bool leader = (threadIdx.x & 127) == 0;
    uint8_t* stage = smem + S::OUT + wg * (COLS / 64) * OUT_BYTES;
    const uint32_t free_lead = PAIR ? mapa(bar_free, 0) : bar_free, res = bar_res + 8 * wg;
    bool ok = true;
    int buf = 0;
    uint32_t bph = 0, rph = 0;
    // scales of two groups at hand, those of the next two (of the next tile's first two, towards a tile's end) on their way
    // (rows and columns that do not exist hold zeros: any scale will do)
    const float *xs, *ws;
    int m0, n0;
    auto place = [&](int i) {
      int m, n;
      lin_tile(i, mt, nt, m, n);
      m0 = m * BM + rank * 128;
      n0 = n * BN + wg * COLS;
      xs = prm.xs + min(m0 + row, prm.M - 1) + zero;
      ws = prm.ws + min(n0 / 128, (prm.N - 1) / 128) * prm.ws_stride + zero;
    };
    float x0, x1, w0, w1;
    auto fetch = [&](int g) {
      const int ga = min(g, Kb - 1), gb = min(g + 1, Kb - 1);
      x0 = __ldg(xs + ga * prm.xs_stride); w0 = __ldg(ws + ga);
      x1 = __ldg(xs + gb * prm.xs_stride); w1 = __ldg(ws + gb);
    };
    place(first);
    fetch(0);
    for (int i = first; i < tiles; i += step) {
      const int m1 = m0, n1 = n0;                            // this tile's place (m0, n0 move on to the next before its epilogue)
      if (leader) {
        bulk_wait_read0();                                   // the staging tiles' last stores have been read
        if (prm.residual) {                                  // what the result is added to comes to where it will be staged
          mbar_expect_tx(res, COLS / 64 * OUT_BYTES);
#pragma unroll
          for (int h = 0; h < COLS / 64; ++h) tma_load_2d(smem_u32(stage) + h * OUT_BYTES, &tm_r, res, n1 + h * 64, m1);
        }
      }
      float acc[COLS];
#pragma unroll
      for (int c = 0; c < COLS; ++c) acc[c] = 0.f;
      float s0 = 0.f, s1 = 0.f;
#pragma unroll 1
      for (int g = 0; g < Kb; ++g) {
        if (!(g & 1)) {
          s0 = x0 * w0;
          s1 = x1 * w1;
          fetch(g + 2);
        }
        const float s = g & 1 ? s1 : s0;
        ok = lin_wait(bar_acc + 8 * buf, bph, abort_flag);
        if (!ok) break;
        tc_fence_after();
        uint32_t v[2][32];
        tmem_ld32(taddr + buf * BN, v[0]);
#pragma unroll
        for (int c = 0; c < COLS / 32; ++c) {
          tc_wait_ld32(v[c & 1]);
          if (c + 1 < COLS / 32) {
            tmem_ld32(taddr + buf * BN + (c + 1) * 32, v[(c + 1) & 1]);
          } else {                                           // all of it is in registers
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
              if (PAIR) mbar_arrive_cluster(free_lead + 8 * buf);
              else mbar_arrive(bar_free + 8 * buf);
            }
          }
#pragma unroll
          for (int e = 0; e < 32; ++e) acc[c * 32 + e] = fmaf(__uint_as_float(v[c & 1][e]), s, acc[c * 32 + e]);
        }
        if (++buf == BUFS) { buf = 0; bph ^= 1u; }
      }
      if (i + step < tiles) {
        place(i + step);
        fetch(0);
      }
      if (prm.residual) {
        ok = ok && lin_wait(res, rph, abort_flag);
        rph ^= 1u;
      }
      ok = lin_group_all(ok, 1 + wg);                        // (the four warps go on together or not at all: there is a barrier below)
      if (!ok) break;
      const int tok = m1 + row;
#pragma unroll
      for (int q = 0; q < COLS / 8; ++q) {                   // 8 columns at a time
        const int c = n1 + q * 8;
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = acc[q * 8 + e];
        if (prm.bias) {
          if (c + 8 <= prm.N) {
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] += __ldg(prm.bias + c + e);
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (c + e < prm.N) y[e] += __ldg(prm.bias + c + e);
          }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = lin_act<ACT>(y[e]);
        uint4* to = reinterpret_cast<uint4*>(stage + (q >> 3) * OUT_BYTES + row * 128 + (((q & 7) ^ (row & 7)) << 4));
        if (prm.residual) {
          const uint4 u = *to;
          const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) { y[2 * e] += bf16lo(w[e]); y[2 * e + 1] += bf16hi(w[e]); }
        }
        if (c < prm.N && c + 8 > prm.N && tok < prm.M) {     // columns behind the last whole 16 bytes, which the tile store would overrun
#pragma unroll
          for (int e = 0; e < 7; ++e)
            if (c + e < prm.N) prm.out[(long long)tok * prm.out_stride + c + e] = __float2bfloat16_rn(y[e]);
        }
        *to = make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
      }
      fence_async_smem();
      lin_group_all(true, 1 + wg);
      if (leader && m1 < prm.M) {
#pragma unroll
        for (int h = 0; h < COLS / 64; ++h)
          if (n1 + h * 64 < (prm.N & ~7)) tma_store_2d(&tm_o, smem_u32(stage) + h * OUT_BYTES, n1 + h * 64, m1);
        bulk_commit();
      }
    }
    if (leader) bulk_wait0();
  }
  __syncthreads();
  if (*abort_flag) lin_settle();
  tc_fence_before();
  __syncthreads();
  if (PAIR) cluster_sync_all();                           // nothing arrives at a CTA that has gone
  if (threadIdx.x == 0 && *abort_flag && prm.status) atomicOr(prm.status, SVA_DEV_TIMEOUT);
  if (warp == 9) {
    tc_fence_after();
    if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
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
  return launch_dep(four ? quantize_rows_kernel<4> : quantize_rows_kernel<1>, dim3((unsigned)(rows * tiles)), 256, 0, st, (const __nv_bfloat16*)x,
                    p->M, p->K, (long long)p->x_stride, (uint8_t*)x8, (long long)p->x8_stride, x_scale, (long long)p->x_scale_stride, tiles);
}

int launch_quantize_tiles(const sva_linear_t* p, const void* w, void* w8, float* w_scale, cudaStream_t st) {
  const dim3 grid((p->K + 127) / 128, (p->N + 127) / 128);
  if (grid.y > 65535) return SVA_ERR_UNSUPPORTED;
  return launch_dep(quantize_tiles_kernel, grid, 256, 0, st, (const __nv_bfloat16*)w, p->N, p->K, (long long)p->w_stride, (uint8_t*)w8,
                    (long long)p->w8_stride, w_scale, (long long)p->w_scale_stride);
}

template <bool PAIR, int ACT>
static int launch_linear_tiles(const sva_linear_t* p, const void* x8, const void* w8, void* out, const LinearParams& prm, int sms,
                               cudaStream_t st) {
  static DeviceOnce once;
  auto kern = linear_kernel<PAIR, ACT>;
  constexpr int SIDE = PAIR ? 256 : 128, CTAS = PAIR ? 2 : 1, SMEM = lin::Shape<PAIR>::SMEM;
  int rc = once.run([&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM) == cudaSuccess; });
  if (rc) return rc;
  CUtensorMap tx, tw, to, tr;
  if ((rc = lin_map(&tx, x8, p->K, p->M, p->x8_stride, 1, 128))) return rc;
  if ((rc = lin_map(&tw, w8, p->K, p->N, p->w8_stride, 1, 128))) return rc;
  // (a tile store writes whole 16-byte pieces, also beyond an inner extent that ends within one: it gets the whole pieces only)
  if ((rc = lin_map(&to, out, p->N < 8 ? 8 : p->N & ~7, p->M, 2 * p->out_stride, 2, 128))) return rc;
  tr = to;
  if (prm.residual && (rc = lin_map(&tr, prm.residual, p->N, p->M, 2 * p->residual_stride, 2, 128))) return rc;
  const long long tiles = (long long)((p->M + SIDE - 1) / SIDE) * ((p->N + SIDE - 1) / SIDE);
  if (tiles > 0x7fffffffLL - sms) return SVA_ERR_UNSUPPORTED;
  const long long most = sms / CTAS;
  return launch_dep_cluster(CTAS, kern, dim3((unsigned)(CTAS * (tiles < most ? tiles : most))), lin::THREADS, SMEM, st, tx, tw, to, tr, prm);
}

template <bool PAIR>
static int launch_linear_act(const sva_linear_t* p, const void* x8, const void* w8, void* out, const LinearParams& prm, int sms, cudaStream_t st) {
  return p->act == SVA_ACT_GELU ? launch_linear_tiles<PAIR, SVA_ACT_GELU>(p, x8, w8, out, prm, sms, st)
       : p->act == SVA_ACT_SILU ? launch_linear_tiles<PAIR, SVA_ACT_SILU>(p, x8, w8, out, prm, sms, st)
                                : launch_linear_tiles<PAIR, SVA_ACT_NONE>(p, x8, w8, out, prm, sms, st);
}

int launch_linear(const sva_linear_t* p, const void* x8, const float* x_scale, const void* w8, const float* w_scale, void* out,
                  const float* bias, const void* residual, int32_t* status, cudaStream_t st) {
  int sms = 0, rc = lin_sms(&sms);
  if (rc) return rc;
  LinearParams prm;
  prm.xs = x_scale; prm.ws = w_scale; prm.bias = bias;
  prm.residual = (const __nv_bfloat16*)residual; prm.out = (__nv_bfloat16*)out;
  prm.xs_stride = p->x_scale_stride; prm.ws_stride = p->w_scale_stride; prm.out_stride = p->out_stride;
  prm.M = p->M; prm.N = p->N; prm.Kb = (p->K + 127) / 128;
  prm.debug = g_debug_lin;
  prm.status = status;
  const long long pairs = (long long)((p->M + 255) / 256) * ((p->N + 255) / 256);
  return pairs >= sms / 2 ? launch_linear_act<true>(p, x8, w8, out, prm, sms, st) : launch_linear_act<false>(p, x8, w8, out, prm, sms, st);
}

}  // namespace sva
