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
  long long xs_stride, ws_stride, out_stride, res_stride;
  int M, N, K, Kb, act, debug;
  int32_t* status;
};

__device__ __forceinline__ float lin_act(float y, int act) {
  if (act == SVA_ACT_GELU) {                              // 0.5 y (1 + tanh u) = y / (1 + exp(-2u)), u = sqrt(2/pi) (y + 0.044715 y^3)
    const float u = 0.7978845608028654f * (y + 0.044715f * y * y * y);
    return __fdividef(y, 1.f + __expf(fminf(-2.f * u, 80.f)));
  }
  if (act == SVA_ACT_SILU) return __fdividef(y, 1.f + __expf(fminf(-y, 80.f)));
  return y;
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

// One persistent CTA per SM, output tiles of 128 tokens x BN weights rows.  x and w tiles of 128 inputs come through a ring by TMA; the tensor cores
// multiply a group of 128 inputs into one of 512/BN accumulators in tensor memory; eight warps take each group's product out, times its
// two scales, and add it up in registers, fp32 throughout.
// Warps 0-7: a thread owns one token and BN/2 columns.  Warp 8 loads, warp 9 issues the MMAs.
namespace lin {
constexpr int THREADS = 320;
constexpr uint32_t A_BYTES = 128 * 128;
template <int BN> struct Shape {
  static constexpr uint32_t STAGE = A_BYTES + BN * 128;
  static constexpr int STAGES = BN == 256 ? 4 : 6, BUFS = 512 / BN, COLS = BN / 2;
  static constexpr uint32_t OUT = STAGES * STAGE, OUT_BYTES = 128 * 128;       // two staging tiles, 128 tokens x 64 columns
  static constexpr int SMEM = 1024 + OUT + 2 * OUT_BYTES;
};
}

template <int BN>
__global__ void __launch_bounds__(lin::THREADS, 1)
linear_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_o,
              const LinearParams prm) {
  using S = lin::Shape<BN>;
  constexpr int STAGES = S::STAGES, BUFS = S::BUFS, COLS = S::COLS;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  __shared__ __align__(8) unsigned long long bars[2 * STAGES + 2 * BUFS];
  __shared__ uint32_t tmem_base_s;
  __shared__ int abort_s;
  volatile int* abort_flag = &abort_s;
  const uint32_t sbase = smem_u32(smem);
  const uint32_t bar_full = smem_u32(&bars[0]), bar_empty = bar_full + 8 * STAGES, bar_acc = bar_empty + 8 * STAGES, bar_free = bar_acc + 8 * BUFS;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int mt = (prm.M + 127) / 128, nt = (prm.N + BN - 1) / BN, tiles = mt * nt, Kb = prm.Kb;
  if (threadIdx.x == 0) {
    for (int i = 0; i < STAGES; ++i) { mbar_init(bar_full + 8 * i, 1); mbar_init(bar_empty + 8 * i, 1); }
    for (int i = 0; i < BUFS; ++i) { mbar_init(bar_acc + 8 * i, 1); mbar_init(bar_free + 8 * i, 8); }
    abort_s = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    prefetch_tmap(&tm_x);
    prefetch_tmap(&tm_w);
    prefetch_tmap(&tm_o);
  }
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_s)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_base_s;
  const int zero = grid_dep_wait();

  if (warp == 8) {
    // ---- loads
    bool ok = true;
    int st = 0;
    uint32_t ph = 0;
    for (int i = blockIdx.x; i < tiles && ok; i += gridDim.x) {
      int m, n;
      lin_tile(i, mt, nt, m, n);
      for (int g = 0; g < Kb; ++g) {
        ok = lin_wait(bar_empty + 8 * st, ph ^ 1u, abort_flag);
        if (!ok) break;
        if ((prm.debug & 1024) && g > 0) break;                                // test aid: the ring runs dry
        if (lane == 0) {
          const uint32_t dst = sbase + st * S::STAGE, bar = bar_full + 8 * st;
          mbar_expect_tx(bar, S::STAGE);
          tma_load_2d(dst, &tm_x, bar, g * 128, m * 128);
          tma_load_2d(dst + lin::A_BYTES, &tm_w, bar, g * 128, n * BN);
        }
        __syncwarp();
        if (++st == STAGES) { st = 0; ph ^= 1u; }
      }
    }
  } else if (warp == 9) {
    // ---- MMAs
    constexpr uint32_t IDESC = instr_desc(128, BN, 0, false);
    const uint32_t el = elect_one();
    const uint64_t ad0 = smem_desc(sbase, 16, 1024), bd0 = smem_desc(sbase + lin::A_BYTES, 16, 1024);
    bool ok = true;
    int st = 0, buf = 0;
    uint32_t ph = 0, bph = 0;
    for (int i = blockIdx.x; i < tiles && ok; i += gridDim.x) {
      for (int g = 0; g < Kb; ++g) {
        ok = lin_wait(bar_free + 8 * buf, bph ^ 1u, abort_flag) && lin_wait(bar_full + 8 * st, ph, abort_flag);
        if (!ok) break;
        tc_fence_after();
        const uint64_t ad = ad0 + (uint64_t)(st * (S::STAGE >> 4)), bd = bd0 + (uint64_t)(st * (S::STAGE >> 4));
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) tc_mma_ss_f8(tmem + buf * BN, ad + 2 * kk, bd + 2 * kk, IDESC, kk > 0 ? 1u : 0u, el);
        tc_commit(bar_empty + 8 * st, el);
        tc_commit(bar_acc + 8 * buf, el);
        if (++st == STAGES) { st = 0; ph ^= 1u; }
        if (++buf == BUFS) { buf = 0; bph ^= 1u; }
      }
    }
  } else {
    // ---- sums and epilogue
    const int wg = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t taddr = tmem + ((uint32_t)((warp & 3) * 32) << 16) + wg * COLS;
    const bool leader = (threadIdx.x & 127) == 0;
    uint8_t* stage = smem + S::OUT + wg * S::OUT_BYTES;
    bool ok = true;
    int buf = 0;
    uint32_t bph = 0;
    for (int i = blockIdx.x; i < tiles; i += gridDim.x) {
      int m, n;
      lin_tile(i, mt, nt, m, n);
      const int tok = m * 128 + row, n0 = n * BN + wg * COLS;
      // (rows and columns that do not exist hold zeros: any scale will do)
      const float* xs = prm.xs + min(tok, prm.M - 1) + zero;
      const float* ws = prm.ws + min(n0 / 128, (prm.N - 1) / 128) * prm.ws_stride + zero;
      uint64_t acc[COLS / 2];
#pragma unroll
      for (int c = 0; c < COLS / 2; ++c) acc[c] = 0ull;
      float next[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) next[j] = j < Kb ? __ldg(xs + j * prm.xs_stride) * __ldg(ws + j) : 0.f;
      for (int g0 = 0; g0 < Kb && ok; g0 += 4) {
        float cur[4], nx[4], nw[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          cur[j] = next[j];
          const int g = min(g0 + 4 + j, Kb - 1);
          nx[j] = __ldg(xs + g * prm.xs_stride);
          nw[j] = __ldg(ws + g);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (g0 + j >= Kb) break;
          ok = lin_wait(bar_acc + 8 * buf, bph, abort_flag);
          if (!ok) break;
          tc_fence_after();
          const uint64_t s2 = pack2(cur[j], cur[j]);
          uint32_t v[2][16];
          tmem_ld16(taddr + buf * BN, v[0]);
#pragma unroll
          for (int c = 0; c < COLS / 16; ++c) {
            tc_wait_ld16(v[c & 1]);
            if (c + 1 < COLS / 16) tmem_ld16(taddr + buf * BN + (c + 1) * 16, v[(c + 1) & 1]);
#pragma unroll
            for (int e = 0; e < 8; ++e)
              acc[c * 8 + e] = fma2(pack2(__uint_as_float(v[c & 1][2 * e]), __uint_as_float(v[c & 1][2 * e + 1])), s2, acc[c * 8 + e]);
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar_free + 8 * buf);
          if (++buf == BUFS) { buf = 0; bph ^= 1u; }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) next[j] = nx[j] * nw[j];
      }
      ok = lin_group_all(ok, 1 + wg);                        // (the four warps go on together or not at all: there are barriers below)
      if (!ok) break;
#pragma unroll
      for (int half = 0; half < COLS / 64; ++half) {
        if (leader) bulk_wait_read0();                       // the staging tile's last store has been read
        lin_group_all(true, 1 + wg);
        const int c0 = n0 + half * 64;
#pragma unroll
        for (int q = 0; q < 8; ++q) {                        // 8 columns at a time
          const int c = c0 + q * 8;
          float y[8];
#pragma unroll
          for (int e = 0; e < 4; ++e) unpack2(acc[half * 32 + q * 4 + e], y[2 * e], y[2 * e + 1]);
          if (prm.bias) {
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] += c + e < prm.N ? __ldg(prm.bias + c + e) : 0.f;
          }
          if (prm.act) {
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = lin_act(y[e], prm.act);
          }
          if (prm.residual && tok < prm.M && c < prm.N) {
            const __nv_bfloat16* r = prm.residual + (long long)tok * prm.res_stride + c;
            if (c + 8 <= prm.N) {
              const uint4 u = __ldg(reinterpret_cast<const uint4*>(r));
              const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
              for (int e = 0; e < 4; ++e) { y[2 * e] += bf16lo(w[e]); y[2 * e + 1] += bf16hi(w[e]); }
            } else {
              for (int e = 0; e < 8; ++e)
                if (c + e < prm.N) y[e] += __bfloat162float(r[e]);
            }
          }
          if (c < prm.N && c + 8 > prm.N && tok < prm.M) {   // columns behind the last whole 16 bytes, which the tile store would overrun
            for (int e = 0; e < 7; ++e)
              if (c + e < prm.N) prm.out[(long long)tok * prm.out_stride + c + e] = __float2bfloat16_rn(y[e]);
          }
          *reinterpret_cast<uint4*>(stage + row * 128 + ((q ^ (row & 7)) << 4)) =
              make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
        }
        fence_async_smem();
        lin_group_all(true, 1 + wg);
        if (leader && c0 < (prm.N & ~7)) {
          tma_store_2d(&tm_o, smem_u32(stage), c0, m * 128);
          bulk_commit();
        }
      }
    }
    if (leader) bulk_wait0();
  }
  __syncthreads();
  if (*abort_flag) lin_settle();
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag && prm.status) atomicOr(prm.status, SVA_DEV_TIMEOUT);
  if (warp == 9) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
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

template <int BN>
static int launch_linear_bn(const sva_linear_t* p, const void* x8, const void* w8, void* out, const LinearParams& prm, int sms, cudaStream_t st) {
  using S = lin::Shape<BN>;
  static DeviceOnce once;
  auto kern = linear_kernel<BN>;
  int rc = once.run([&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM) == cudaSuccess; });
  if (rc) return rc;
  CUtensorMap tx, tw, to;
  if ((rc = lin_map(&tx, x8, p->K, p->M, p->x8_stride, 1, 128))) return rc;
  if ((rc = lin_map(&tw, w8, p->K, p->N, p->w8_stride, 1, BN))) return rc;
  // (a tile store writes whole 16-byte pieces, also beyond an inner extent that ends within one: it gets the whole pieces only)
  if ((rc = lin_map(&to, out, p->N < 8 ? 8 : p->N & ~7, p->M, 2 * p->out_stride, 2, 128))) return rc;
  const long long tiles = (long long)((p->M + 127) / 128) * ((p->N + BN - 1) / BN);
  if (tiles > 0x7fffffffLL - sms) return SVA_ERR_UNSUPPORTED;
  return launch_dep(kern, dim3((unsigned)(tiles < sms ? tiles : sms)), lin::THREADS, S::SMEM, st, tx, tw, to, prm);
}

int launch_linear(const sva_linear_t* p, const void* x8, const float* x_scale, const void* w8, const float* w_scale, void* out,
                  const float* bias, const void* residual, int32_t* status, cudaStream_t st) {
  int sms = 0, rc = lin_sms(&sms);
  if (rc) return rc;
  LinearParams prm;
  prm.xs = x_scale; prm.ws = w_scale; prm.bias = bias;
  prm.residual = (const __nv_bfloat16*)residual; prm.out = (__nv_bfloat16*)out;
  prm.xs_stride = p->x_scale_stride; prm.ws_stride = p->w_scale_stride; prm.out_stride = p->out_stride; prm.res_stride = p->residual_stride;
  prm.M = p->M; prm.N = p->N; prm.K = p->K; prm.Kb = (p->K + 127) / 128; prm.act = p->act;
  prm.debug = g_debug_lin;
  prm.status = status;
  const long long wide = (long long)((p->M + 127) / 128) * ((p->N + 255) / 256);
  return wide >= sms ? launch_linear_bn<256>(p, x8, w8, out, prm, sms, st) : launch_linear_bn<128>(p, x8, w8, out, prm, sms, st);
}

}  // namespace sva
