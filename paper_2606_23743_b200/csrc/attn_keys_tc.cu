// Attention of many rows over many keys (sva_cached_attn_fwd, sva_cross_attn_fwd) on the tensor cores.
//
// A pair of CTAs (cta_group::2) takes items: 512 rows (four tiles of 128) of one key head, and a range of its key tiles of 128.  A row is a query of one
// of the heads that share the key head; a tile holds the `group` heads of 128 / group tokens.  Each CTA has two of the row tiles, w = 0 and 1, and half of
// each key tile: 64 keys of K, half of the channels of V.  The MMAs (256 rows, the w-th tiles of both CTAs) read both halves; so a key tile is brought
// in, and where it is codes converted, once for 512 rows, and of what shared memory can deliver the operands take two thirds where a CTA by itself would take
// all of it.  Roles:
//   warp  0          (first CTA) issues the MMAs of both
//   warps 1-7        bf16 keys: 1 brings in K, 2 V and 3 Q (TMA); 3 also puts zeros into rows of V that are left out
//                    cached keys: all seven read codes, convert them to fp16 (exactly) and store them in the layout that TMA would leave
//   warps 8-11, 12-15   softmax of tile 0 and of tile 1; thread <-> row <-> TMEM lane.  Also the epilogue, and for cached keys the Q tile
// A key tile is worked on in halves h of 64 keys: S_wh = Q_w K_h^T (A, B from shared memory), P_wh over the columns of S_wh, O_w += P_wh V_h (A from TMEM,
// V as an MN-major B operand).  TMEM: S_0 | S_1 | O_0 | O_1, 128 columns each.  Once a group has handed over P_wh, the issuer lets P V_wh and the next
// tile's S_wh follow one another, and the group goes on with the other half, whose S is there by then: its exponentials never wait for an MMA that
// waits for them (with whole tiles the way from P to the next S took 1 200 to 1 700 cycles of 4 000).  The next S_wh overwrites P_wh, which P V_wh before
// it reads: MMAs run in the order of their issue.
//
// The reference m of a row's exponentials follows its maximum lazily: a tile's first exponentials are taken with the m so far and its maximum beside
// them; only when that is more than LAZY powers of two above m are they done again, and O rescaled (probabilities reach 2^LAZY; sums are fp32).
// Probabilities have the operands' type, which is V's: bf16 beside bf16 keys (2^-8 of each weight; a second term as in attn_keys.cu would be half as many
// MMAs again, and its subtractions and stores the softmax warps', which are what bounds the kernel), fp16 beside codes.  Row sums take them unrounded.
// Cached keys: K's scale is a factor of the logits, log2 of V's an addend (both per 16 keys), see attn_keys.cu; P is fp16 and at most 2^(UP + LAZY).
//
// 24 heads x 4 680 queries x 32 760 cached keys: 2.2 ms = 0.84 PFLOP/s; 2 x 24 heads x 32 760 queries x 512 bf16 keys 490 us.  What bounds it is the softmax warps' own latency, in
// this arrangement (attn_sm100.cu has as many warps per scheduler and takes some 1 460 cycles for a 128 x 128 tile and SM, this kernel 2 000): a scheduler has
// one of each group, and no pipe is more than half busy (tensor 52 %, issue 44 %, exponentials 39 %).
//
// Every wait is bounded; when one runs out all roles leave, the CTA reports SVA_DEV_TIMEOUT and its rows are not stored.
#include <cuda_fp16.h>

#include "attn_keys.cuh"
#include "tc_ptx.cuh"

namespace sva {

namespace kt {
constexpr int THREADS = 512;
constexpr int SOFTMAX_REGS = 168, HELPER_REGS = 88;
static_assert(256 * SOFTMAX_REGS + 256 * HELPER_REGS <= THREADS * 128, "setmaxnreg draws on the registers of the launch");
constexpr int KT = 128;                               // keys of a tile
constexpr int PANEL = 128 * 128;                      // Q: 128 rows x 128 bytes (64 channels)
constexpr int STAGES = 4;
constexpr int SCALE_RING = 8;                         // (one more than the stages is enough)
constexpr float LAZY = 7.0f;
constexpr int POLY = 0b01000100;                      // pairs of eight whose exponentials are polynomials
constexpr float UP_F16 = 8.0f;                        // log2 of a probability at the reference (fp16: 2^15 at most)
constexpr int CONVERTERS = 7;                         // warps (cached keys)
// shared memory (bytes from a 1024-byte boundary): Q tiles | K stages | V stages | control | 2 KB per softmax warp on O's way out
template <int D> struct Smem {
  static constexpr int TILE = D / 64 * PANEL, HALF = TILE / 2;      // of Q; of K or V, a CTA's half of a key tile
  static constexpr int K = 2 * TILE, V = K + STAGES * HALF, CTRL = V + STAGES * HALF, OUT = CTRL + 2048, BYTES = OUT + 8 * 2048 + 1024;
};
// control block: barriers (8 bytes each), then TMEM base and abort flag, then the scales' ring
enum { K_FULL = 0, K_EMPTY = 32, V_LAND = 64, V_FULL = 96, V_EMPTY = 128, Q_FULL = 160, Q_EMPTY = 176, S_FULL = 192, P_FULL = 224, PV_DONE = 256,
       O_DONE = 272, O_FREE = 288, TMEM_BASE = 304, ABORT = 308, SCALES = 512 };      // (S_FULL, P_FULL: [w][h])
// SCALES: [ring][8 chunks of 16 keys]{k scale, log2 v scale, 1 / v scale, -}
}  // namespace kt

struct KeysTcParams {
  KeysParams k;
  int tokens;                                         // of a row tile: 128 / group
  int quads;                                          // fours of row tiles per key head
  uint32_t items;
  int k_each_h, k_each_b, v_each_h, v_each_b;         // 0: heads / items share K, V (the maps then have one)
  bool wide;                                          // 32-byte stores into o
  int debug;
};

// An item: queries [t0, t0 + 4 * tokens) of (b, hk), key tiles [j0, j1).  Tile w of CTA r begins with query t0 + (2 w + r) tokens.
struct KeysItem {
  int b, hk, quad, split, keys, queries, t0, j0, j1;
  bool two;                                           // tiles w = 1 have rows
};

// D[tmem of both CTAs] (+)= A[each CTA's shared memory: its 128 rows] * B[half of the columns from each], 16-bit operands
__device__ __forceinline__ void tc_mma_ss_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc, uint32_t elected) {
  asm volatile("{\n.reg .pred p, q;\nsetp.ne.b32 p, %4, 0;\nsetp.ne.b32 q, %5, 0;\n"
               "@q tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}"
               ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc), "r"(elected) : "memory");
}
// the same with A in each CTA's tensor memory
__device__ __forceinline__ void tc_mma_ts_pair(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc, uint32_t elected) {
  asm volatile("{\n.reg .pred p, q;\nsetp.ne.b32 p, %4, 0;\nsetp.ne.b32 q, %5, 0;\n"
               "@q tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;\n}"
               ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(acc), "r"(elected) : "memory");
}
__device__ __forceinline__ void tma_load_4d_pair_if(uint32_t dst, const CUtensorMap* map, uint32_t mapped_bar, int c0, int c1, int c2, int c3, uint32_t elected) {
  asm volatile(
      "{\n.reg .pred q;\nsetp.ne.b32 q, %7, 0;\n"
      "@q cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];\n}"
      ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(mapped_bar), "r"(elected) : "memory");
}
__device__ __forceinline__ uint32_t f16_pair(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// Eight codes as fp16 values.  (By way of shifts and masks it would take eight operations for four codes on a pipe of half the rate: 25 codes
// per cycle and SM, this 57.)
__device__ __forceinline__ uint4 f16_of_codes(uint32_t x, uint32_t y) {
  uint4 r;
  asm("{\n\t.reg .b16 a, b, c, d;\n\tmov.b32 {a, b}, %4;\n\tmov.b32 {c, d}, %5;\n\t"
      "cvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\tcvt.rn.f16x2.e4m3x2 %2, c;\n\tcvt.rn.f16x2.e4m3x2 %3, d;\n\t}"
      : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(x), "r"(y));
  return r;
}

// Bounded wait of a warp, as mbar_wait, but suspended until the phase completes (or for as long as the hardware likes) where it polls: a
// group's way from its last P to its next S goes through six of them.
__device__ __forceinline__ uint32_t mbar_suspend(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(done) : "r"(bar), "r"(parity) : "memory");
  return done;
}
__device__ __forceinline__ bool keys_wait_long(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  const uint32_t t0 = (uint32_t)clock();
  do {
    if (__all_sync(0xffffffffu, mbar_suspend(bar, parity))) return true;
  } while (!__any_sync(0xffffffffu, *abort_flag || (uint32_t)clock() - t0 > g_wait_limit));
  *abort_flag = 1;
  return false;
}
__device__ __forceinline__ bool keys_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  if (__all_sync(0xffffffffu, mbar_suspend(bar, parity))) return true;
  return keys_wait_long(bar, parity, abort_flag);
}
// the larger of three, a NaN if there is one
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
  float y;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
// What a logit of codes is multiplied by, a row's factor times a page's scale of K; not 0, so that a logit of -inf (a key that is left out) stays one.
__device__ __forceinline__ float logit_factor(float row, float page) { return fmaxf(row * page, 1.17549435e-38f); }
// 0, and of a NaN or +infinity a NaN
__device__ __forceinline__ float nan_if_endless(float x) {
  x = max_nan(x, -3.402823466e38f);
  return x - x;
}
// 2^x of two values on the FMA and integer pipes, x <= 126: 2^floor(x) by the exponent field, the rest by a polynomial with the value 1 at 0 (the
// smallest relative error on [0, 1) of its degree: 8.3e-8; 1.5e-7 as evaluated).  Below -127 exactly 0.
__device__ __forceinline__ uint64_t ex2_poly(uint64_t x2) {
  float x0, x1, t0, t1, p0, p1;
  unpack2(x2, x0, x1);
  const uint64_t x = pack2(fmaxf(x0, -127.f), fmaxf(x1, -127.f));
  const uint64_t magic = pack2(12582912.f, 12582912.f), unmagic = pack2(-12582912.f, -12582912.f), minus = pack2(-1.f, -1.f);
  uint64_t t;
  asm("add.rm.f32x2 %0, %1, %2;" : "=l"(t) : "l"(x), "l"(magic));       // floor(x) in the low bits
  const uint64_t f = fma2(add2(t, unmagic), minus, x);
  uint64_t p = fma2(f, pack2(0.0018671302823349833f, 0.0018671302823349833f), pack2(0.009017029777169228f, 0.009017029777169228f));
  p = fma2(f, p, pack2(0.05579991266131401f, 0.05579991266131401f));
  p = fma2(f, p, pack2(0.24016444385051727f, 0.24016444385051727f));
  p = fma2(f, p, pack2(0.6931512951850891f, 0.6931512951850891f));
  p = fma2(f, p, pack2(1.f, 1.f));
  unpack2(t, t0, t1);
  unpack2(p, p0, p1);
  return pack2(__uint_as_float(__float_as_uint(p0) + (__float_as_uint(t0) << 23)), __uint_as_float(__float_as_uint(p1) + (__float_as_uint(t1) << 23)));
}

// Item i; false where it has no rows.
__device__ __forceinline__ bool item_at(const KeysTcParams& prm, uint32_t i, KeysItem& x) {
  const KeysParams& k = prm.k;
  x.quad = (int)(i % (uint32_t)prm.quads); i /= (uint32_t)prm.quads;
  x.split = 0;
  if (k.splits > 1) { x.split = (int)(i % (uint32_t)k.splits); i /= (uint32_t)k.splits; }
  x.hk = (int)(i % (uint32_t)k.Hk);
  x.b = (int)(i / (uint32_t)k.Hk);
  x.keys = seq_keys(k, x.b);
  x.queries = seq_queries(k, x.b);
  x.t0 = x.quad * 4 * prm.tokens;
  if (x.t0 >= x.queries) return false;
  x.two = x.t0 + 2 * prm.tokens < x.queries;
  const int end = keys_seen(k, x.keys, x.queries, min(x.t0 + (x.two ? 4 : 2) * prm.tokens, x.queries) - 1);
  const int tiles = (end + kt::KT - 1) / kt::KT;
  x.j0 = 0;
  x.j1 = tiles;
  if (k.splits > 1) {
    // (at most 2^24 tiles and as many splits as SMs)
    x.j0 = (int)((uint32_t)tiles * (uint32_t)x.split / (uint32_t)k.splits);
    x.j1 = (int)((uint32_t)tiles * (uint32_t)(x.split + 1) / (uint32_t)k.splits);
  }
  return true;
}
// The next item at or after i (a pair's are as far apart as there are pairs) that has key tiles; false at the end.
__device__ __forceinline__ bool next_item(const KeysTcParams& prm, uint32_t& i, KeysItem& x) {
  for (; i < prm.items; i += gridDim.x / 2)
    if (item_at(prm, i, x) && x.j0 < x.j1) return true;
  return false;
}

template <int D, bool PAGED>
__global__ void __launch_bounds__(kt::THREADS, 1)
keys_tc_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
               const KeysTcParams prm) {
  using namespace kt;
  constexpr int TILE = Smem<D>::TILE, HALF = Smem<D>::HALF, OFF_K = Smem<D>::K, OFF_V = Smem<D>::V, PANELS = D / 64;
  constexpr int KPANEL = 64 * 128;                                            // K: 64 rows x 128 bytes
  constexpr int VROW = D;                                                     // V: bytes of a row, D / 2 channels
  constexpr int FMT = PAGED ? 0 : 1;                                          // fp16 or bf16 operands
  constexpr uint32_t IDESC_S = instr_desc(256, 64, FMT, false), IDESC_O = instr_desc(256, D, FMT, true);
  constexpr float UP = PAGED ? UP_F16 : 0.f;
  constexpr uint32_t COL_S = 0, COL_O = 256;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const uint32_t sbase = smem_u32(smem), cb = sbase + Smem<D>::CTRL;
  uint8_t* ctrl = smem + Smem<D>::CTRL;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(ctrl + ABORT);
  float4* scales = reinterpret_cast<float4*>(ctrl + SCALES);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rank = (int)(blockIdx.x & 1);

  if (threadIdx.x == 0) {
    for (int i = 0; i < STAGES; ++i) {
      mbar_init(cb + K_FULL + 8 * i, PAGED ? 2 * CONVERTERS : 1);
      mbar_init(cb + K_EMPTY + 8 * i, 1);
      mbar_init(cb + V_LAND + 8 * i, 1);
      mbar_init(cb + V_FULL + 8 * i, PAGED ? 2 * CONVERTERS : 2);
      mbar_init(cb + V_EMPTY + 8 * i, 1);
    }
    for (int w = 0; w < 2; ++w) {
      mbar_init(cb + Q_FULL + 8 * w, PAGED ? 8 : 1);                          // (8: the warps of a group, in both CTAs)
      mbar_init(cb + Q_EMPTY + 8 * w, 1);
      for (int h = 0; h < 2; ++h) {
        mbar_init(cb + S_FULL + 16 * w + 8 * h, 1);
        mbar_init(cb + P_FULL + 16 * w + 8 * h, 8);
      }
      mbar_init(cb + PV_DONE + 8 * w, 1);
      mbar_init(cb + O_DONE + 8 * w, 1);
      mbar_init(cb + O_FREE + 8 * w, 8);
    }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
    if (!PAGED) { prefetch_tmap(&tm_q); prefetch_tmap(&tm_k); prefetch_tmap(&tm_v); }
  }
  if (warp == 0) {
    __syncwarp();
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(cb + TMEM_BASE), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();                                                         // the other CTA's barriers are there
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, *reinterpret_cast<volatile uint32_t*>(ctrl + TMEM_BASE), 0);
  const uint32_t lead = mapa(cb, 0);                                          // the first CTA's barriers: what both CTAs bring the issuer
  const int zero = grid_dep_wait();
  if (PAGED) report_long(prm.k, zero);
  uint32_t at = (blockIdx.x >> 1) + (uint32_t)zero;
  const uint32_t pairs = gridDim.x / 2;
  KeysItem it;
  bool ok = true;
  auto wait = [&](uint32_t bar, uint32_t use) -> bool { return keys_wait(bar, use & 1u, abort_flag); };

  if (warp < 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(HELPER_REGS));
    if (warp == 0 && rank == 0) {
      // ------------------------------------------------------------------------------------------------ issuer
      const uint32_t el = elect_one();
      const uint64_t qd0 = smem_desc(sbase, 16, 1024), kd0 = smem_desc(sbase + OFF_K, 16, 1024);
      const uint64_t vd0 = D == 128 ? smem_desc(sbase + OFF_V, 16, 1024) : smem_desc_sw64(sbase + OFF_V);
      uint32_t kn = 0, vn = 0, qn[2] = {0, 0}, pn[2] = {0, 0}, on[2] = {0, 0};      // uses so far
      auto issue_s = [&](int w, int h, bool first, bool last) -> bool {      // from the K tile in use number kn
        if (first && !wait(cb + Q_FULL + 8 * w, qn[w]++)) return false;
        tc_fence_after();
        const uint64_t qd = qd0 + (uint64_t)(w * (TILE >> 4)), kd = kd0 + (uint64_t)((kn % STAGES) * (HALF >> 4) + h * (32 * 128 >> 4));
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
          tc_mma_ss_pair(tmem + COL_S + 128 * w + 64 * h, qd + (uint64_t)((kk / 4) * (PANEL >> 4) + (kk % 4) * 2),
                         kd + (uint64_t)((kk / 4) * (KPANEL >> 4) + (kk % 4) * 2), IDESC_S, kk > 0 ? 1u : 0u, el);
        tc_commit_pair(cb + S_FULL + 16 * w + 8 * h, el);
        if (last) tc_commit_pair(cb + Q_EMPTY + 8 * w, el);
        return true;
      };
      auto issue_pv = [&](int w, int h, bool first, bool last) -> bool {     // with the V tile in use number vn
        if (!wait(cb + P_FULL + 16 * w + 8 * h, pn[w])) return false;
        if (h == 1) ++pn[w];
        if (first && on[w] > 0 && !wait(cb + O_FREE + 8 * w, on[w] - 1u)) return false;
        if (first) ++on[w];
        tc_fence_after();
        const uint64_t vd = vd0 + (uint64_t)((vn % STAGES) * (HALF >> 4) + h * 4 * VROW);
#pragma unroll
        for (int kk = 0; kk < KT / 32; ++kk)                          // 16 keys = 16 rows of V
          tc_mma_ts_pair(tmem + COL_O + 128 * w, tmem + COL_S + 128 * w + 64 * h + 8 * kk, vd + (uint64_t)(kk * VROW), IDESC_O, !first || kk > 0 ? 1u : 0u, el);
        tc_commit_pair(cb + PV_DONE + 8 * w, el);
        if (last) tc_commit_pair(cb + O_DONE + 8 * w, el);
        return true;
      };
      // S of the first tile of an item
      auto begin = [&](const KeysItem& x) -> bool {
        if (!wait(cb + K_FULL + 8 * (kn % STAGES), kn / STAGES)) return false;
        const bool last = x.j1 - x.j0 == 1;
        if (!issue_s(0, 0, true, false) || !issue_s(0, 1, false, last)) return false;
        if (x.two && (!issue_s(1, 0, true, false) || !issue_s(1, 1, false, last))) return false;
        tc_commit_pair(cb + K_EMPTY + 8 * (kn % STAGES), el);
        ++kn;
        return true;
      };
      // (an item's numbers by way of a shuffle: the compiler then knows them to be the same for the warp, and can keep descriptors in uniform registers)
      auto next = [&]() -> bool {
        const bool more = next_item(prm, at, it);
        it.j0 = __shfl_sync(0xffffffffu, it.j0, 0);
        it.j1 = __shfl_sync(0xffffffffu, it.j1, 0);
        it.two = __shfl_sync(0xffffffffu, (int)it.two, 0) != 0;
        return __shfl_sync(0xffffffffu, (int)more, 0) != 0;
      };
      bool more = next();
      if (more) ok = begin(it);
      while (more && ok) {
        for (int j = it.j0; j < it.j1 && ok; ++j) {
          const bool first = j == it.j0, last = j + 1 == it.j1;
          // (both tiles first: they are there long before P is, and between P and S nothing is waited for)
          ok = wait(cb + V_FULL + 8 * (vn % STAGES), vn / STAGES) && (last || wait(cb + K_FULL + 8 * (kn % STAGES), kn / STAGES));
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int h = i >> 1, w = i & 1;
            if (!ok || (w == 1 && !it.two)) continue;
            ok = issue_pv(w, h, first && h == 0, last && h == 1) && (last || issue_s(w, h, false, h == 1 && j + 2 == it.j1));
          }
          if (!ok) break;
          tc_commit_pair(cb + V_EMPTY + 8 * (vn % STAGES), el);
          ++vn;
          if (!last) {
            tc_commit_pair(cb + K_EMPTY + 8 * (kn % STAGES), el);
            ++kn;
          }
        }
        if (!ok) break;
        at += pairs;
        more = next();
        if (more) ok = begin(it);
      }
    } else if (warp > 0 && warp < 4 && !PAGED) {
      const uint32_t el = elect_one();
      uint32_t n = 0;
      if (warp < 3) {
        // ---------------------------------------------------------------------------------------------- K, V (bf16)
        const uint32_t empty = cb + (warp == 1 ? K_EMPTY : V_EMPTY);
        for (; ok && next_item(prm, at, it); at += pairs) {
          for (int j = it.j0; j < it.j1 && ok; ++j, ++n) {
            const uint32_t s = n % STAGES, use = n / STAGES;
            if (use > 0) ok = wait(empty + 8 * s, use - 1u);
            if (!ok || ((prm.debug & 2048) && n >= 1)) { ok = false; break; }       // (test aid: later tiles never come)
            if (warp == 1) {
              if (rank == 0) mbar_expect_tx_if(cb + K_FULL + 8 * s, 2 * HALF, el);
#pragma unroll
              for (int p = 0; p < PANELS; ++p)
#pragma unroll
                for (int h = 0; h < 2; ++h)                             // of each half's 64 keys this CTA's 32
                  tma_load_4d_pair_if(sbase + OFF_K + s * HALF + p * KPANEL + h * 32 * 128, &tm_k, lead + K_FULL + 8 * s, 64 * p,
                                      j * KT + 64 * h + 32 * rank, it.hk * prm.k_each_h, it.b * prm.k_each_b, el);
            } else {
              mbar_expect_tx_if(cb + V_LAND + 8 * s, HALF, el);
              tma_load_4d_if(sbase + OFF_V + s * HALF, &tm_v, cb + V_LAND + 8 * s, D / 2 * rank, j * KT, it.hk * prm.v_each_h, it.b * prm.v_each_b, el);
            }
          }
        }
        // (the MMAs' arrivals from the first CTA are all here before this one may go)
        for (uint32_t i = n > STAGES ? n - STAGES : 0; ok && i < n; ++i) ok = wait(empty + 8 * (i % STAGES), i / STAGES);
      } else {
        // ---------------------------------------------------------------------------------------------- Q; rows of V that are left out
        const uint32_t bytes = (uint32_t)(prm.tokens * prm.k.group) * 128 * PANELS;
        uint32_t qn[2] = {0, 0};
        for (; ok && next_item(prm, at, it); at += pairs) {
          for (int w = 0; w < (it.two ? 2 : 1) && ok; ++w) {
            if (qn[w] > 0) ok = wait(cb + Q_EMPTY + 8 * w, qn[w] - 1u);
            if (!ok) break;
            ++qn[w];
            if (rank == 0) mbar_expect_tx_if(cb + Q_FULL + 8 * w, 2 * bytes, el);
#pragma unroll
            for (int p = 0; p < PANELS; ++p)
              tma_load_4d_pair_if(sbase + w * TILE + p * PANEL, &tm_q, lead + Q_FULL + 8 * w, 64 * p, it.hk * prm.k.group,
                                  it.t0 + (2 * w + rank) * prm.tokens, it.b, el);
          }
          for (int j = it.j0; j < it.j1 && ok; ++j, ++n) {
            const uint32_t s = n % STAGES;
            ok = wait(cb + V_LAND + 8 * s, n / STAGES);
            if (!ok) break;
            if (prm.k.mask || (it.keys < prm.k.S && (j + 1) * KT > it.keys)) {
              // zeros, whatever they hold: their probabilities are 0, and 0 times a NaN is one
#pragma unroll 1
              for (int row = lane; row < KT; row += 32) {
                const int key = j * KT + row;
                bool out = key >= it.keys;
                if (!out && prm.k.mask) out = __ldg(prm.k.mask + it.b * prm.k.mask_stride + key) == 0;
                if (out) {
#pragma unroll
                  for (int e = 0; e < VROW; e += 16) *reinterpret_cast<uint4*>(smem + OFF_V + s * HALF + row * VROW + e) = make_uint4(0u, 0u, 0u, 0u);
                }
              }
              fence_async_smem();
              __syncwarp();
            }
            mbar_arrive_cluster_if(lead + V_FULL + 8 * s, lane == 0);
          }
        }
        for (int w = 0; w < 2 && ok; ++w)
          if (qn[w] > 0) ok = wait(cb + Q_EMPTY + 8 * w, qn[w] - 1u);
      }
    } else if (warp > 0 && PAGED) {
      // ------------------------------------------------------------------------------------------------ K, V (codes)
      // Units of 512 bytes: K's 64 keys 8 at a time and 64 channels at a time, then V's 128 keys (this CTA's half of the channels) 8 at a time (D = 64: 16).  A
      // lane has 16 codes of a row; its two 16-byte stores meet all banks with those of its neighbours.  Warp a takes units a, a + 7, ...
      constexpr int KU = 8 * PANELS, VU = D == 128 ? 16 : 8, UNITS = KU + VU, EACH = (UNITS + CONVERTERS - 1) / CONVERTERS;
      const KeysParams& k = prm.k;
      const int a = warp - 1;
      uint32_t n = 0;
      // lane c < 8 knows chunk c of 16 keys: its page (-1: none, or named wrongly), its first row there, its scales
      struct Place { KeysItem it; uint32_t at; int j; bool more; int id; long long row; };
      auto look_up = [&](Place& x) {
        x.id = -1;
        x.row = 0;
        const int key = x.j * KT + lane * 16;
        if (x.more && lane < 8 && key < x.it.keys) {
          const int e = key / k.page;
          x.id = e < k.max_pages ? __ldg(k.table + x.it.b * k.table_stride + e) : -1;
          if (x.id < 0 || x.id >= k.pages) {
            x.id = -1;
            if (k.status) atomicOr(k.status, SVA_DEV_BAD_INDEX);
          } else {
            x.row = ((long long)x.id * k.Hk + x.it.hk) * k.page + (key - e * k.page);
          }
        }
      };
      auto step_on = [&](Place& x) {
        if (++x.j == x.it.j1) {
          x.at += pairs;
          x.more = next_item(prm, x.at, x.it);
          x.j = x.it.j0;
        }
      };
      // where a unit's lane finds its codes, and puts the values (from the stage's beginning)
      auto unit_of = [&](int u, int& key, int& byte, int& to0, int& to1) {
        if (u < KU) {
          const int sub = lane >> 2, piece = lane & 3, row = u / PANELS * 8 + sub, p = u % PANELS;
          key = (row & 32) * 2 + 32 * rank + (row & 31);                     // (of each half's 64 keys this CTA's 32)
          byte = 64 * p + 16 * piece;
          const int line = p * KPANEL + row * 128;
          to0 = line + (((2 * piece) ^ (row & 7)) << 4);
          to1 = line + (((2 * piece + 1) ^ (row & 7)) << 4);
        } else if (D == 128) {
          const int sub = lane >> 2, piece = lane & 3;
          key = (u - KU) * 8 + sub;
          byte = 64 * rank + 16 * piece;
          to0 = key * 128 + (((2 * piece) ^ (key & 7)) << 4);
          to1 = key * 128 + (((2 * piece + 1) ^ (key & 7)) << 4);
        } else {
          const int sub = lane >> 1, piece = lane & 1;
          key = (u - KU) * 16 + sub;
          byte = 32 * rank + 16 * piece;
          to0 = key * 64 + (((2 * piece) ^ (key >> 1 & 3)) << 4);
          to1 = key * 64 + (((2 * piece + 1) ^ (key >> 1 & 3)) << 4);
        }
      };
      auto load = [&](const Place& x, int u, uint4& r) {
        int key, byte, to0, to1;
        unit_of(u, key, byte, to0, to1);
        const long long row = __shfl_sync(0xffffffffu, x.row, key >> 4);
        const int id = __shfl_sync(0xffffffffu, x.id, key >> 4);
        r = make_uint4(0u, 0u, 0u, 0u);
        if (id >= 0 && x.j * KT + key < x.it.keys)
          r = __ldg(reinterpret_cast<const uint4*>((u < KU ? k.k : k.v) + (row + (key & 15)) * D + byte));
      };
      auto store = [&](uint32_t s, int u, const uint4& r) {
        int key, byte, to0, to1;
        unit_of(u, key, byte, to0, to1);
        uint8_t* stage = smem + (u < KU ? OFF_K : OFF_V) + s * HALF;
        *reinterpret_cast<uint4*>(stage + to0) = f16_of_codes(r.x, r.y);
        *reinterpret_cast<uint4*>(stage + to1) = f16_of_codes(r.z, r.w);
      };
      uint4 r[EACH];                                                              // one tile ahead, its pages looked up another tile ahead
      float ks = 1.f, vs = 1.f;
      bool named = false;
      auto fetch_scales = [&](const Place& x) {
        named = x.id >= 0;
        if (named) {
          ks = __ldg(k.k_scale + (long long)x.id * k.Hk + x.it.hk);
          vs = __ldg(k.v_scale + (long long)x.id * k.Hk + x.it.hk);
        }
      };
      Place nx;                                                                   // the next tile to be fetched
      nx.at = at;
      nx.more = next_item(prm, nx.at, nx.it);
      nx.j = nx.it.j0;
      bool more = nx.more;                                                        // ... and whether one has been
      if (more) {
        look_up(nx);
#pragma unroll
        for (int i = 0; i < EACH; ++i)
          if (a + CONVERTERS * i < UNITS) load(nx, a + CONVERTERS * i, r[i]);
        fetch_scales(nx);
        step_on(nx);
        look_up(nx);
      }
      while (more) {
        const uint32_t s = n % STAGES, use = n / STAGES;
        if (use > 0) ok = wait(cb + K_EMPTY + 8 * s, use - 1u);
        if (!ok || ((prm.debug & 2048) && n >= 1)) { ok = false; break; }         // (test aid: later tiles never come)
        // A chunk on a page with a scale that is a NaN or infinite: its keys become NaNs, which masks take out of S for the rows that do not see them, its
        // values zeros, which spoil no row
        const bool good = named && max_nan(fabsf(ks), fabsf(vs)) < INFINITY;
        if (const uint32_t bad = __ballot_sync(0xffffffffu, named && !good)) {
#pragma unroll
          for (int i = 0; i < EACH; ++i) {
            const int u = a + CONVERTERS * i;
            int key, byte, to0, to1;
            unit_of(u, key, byte, to0, to1);
            if (bad >> (key >> 4 & 7) & 1u) r[i].x = r[i].y = r[i].z = r[i].w = u < KU ? 0x7f7f7f7fu : 0u;
          }
        }
        if (a == 0 && lane < 8) {
          // (pages that are named wrongly: left out)
          const float v = good ? v_scale_floor(vs) : 1.f;
          scales[(n % SCALE_RING) * 8 + lane] = make_float4(good ? ks : 1.f, named ? log2f(v) : -INFINITY, 1.f / v, 0.f);
        }
        more = nx.more;
        bool k_out = false;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
          const int u = a + CONVERTERS * i;
          if (u >= KU && !k_out) {                                                // (uniform in a warp)
            k_out = true;
            fence_async_smem();
            __syncwarp();
            mbar_arrive_cluster_if(lead + K_FULL + 8 * s, lane == 0);
            if (use > 0) ok = ok && wait(cb + V_EMPTY + 8 * s, use - 1u);
          }
          if (u < UNITS) {
            store(s, u, r[i]);
            if (more) load(nx, u, r[i]);
          }
        }
        if (!ok) break;
        fence_async_smem();
        __syncwarp();
        mbar_arrive_cluster_if(lead + V_FULL + 8 * s, lane == 0);
        if (more) {
          fetch_scales(nx);
          step_on(nx);
          look_up(nx);
        }
        ++n;
      }
      // (the MMAs' arrivals from the first CTA are all here before this one may go)
      for (uint32_t i = n > STAGES ? n - STAGES : 0; ok && i < n; ++i)
        ok = wait(cb + K_EMPTY + 8 * (i % STAGES), i / STAGES) && wait(cb + V_EMPTY + 8 * (i % STAGES), i / STAGES);
    }
  } else {
    // ------------------------------------------------------------------------------------------------ softmax
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(SOFTMAX_REGS));
    const KeysParams& k = prm.k;
    const int w = (warp >> 2) - 2, row = (warp & 3) * 32 + lane;
    const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16, sole = lane == 0;
    const uint32_t s_tmem = tmem + lane_addr + COL_S + 128 * w, o_tmem = tmem + lane_addr + COL_O + 128 * w;
    uint32_t fn = 0, hn = 0, qn = 0, dn = 0, tn = 0;                          // halves of S fetched, of P handed over, Q tiles, items, and key tiles of all items so far
    // where a row's output goes
    const int tok = row / k.group, head = row % k.group, mine_from = (2 * w + rank) * prm.tokens + tok;
    auto out_row = [&](const KeysItem& x, int t) -> long long { return x.b * k.so.b + (long long)(x.hk * k.group + head) * k.so.h + (long long)t * k.so.n; };
    auto lse_at = [&](const KeysItem& x, int t) -> float* { return k.lse + ((long long)x.b * k.Hq + x.hk * k.group + head) * k.M + t; };
    auto part_row = [&](const KeysItem& x) -> long long {
      return (x.split * ((long long)k.B * k.Hk * k.tiles) + ((long long)x.b * k.Hk + x.hk) * k.tiles + 4 * x.quad + 2 * w + rank) * 128 + row;
    };
    // (an item without keys: zeros; a split without: an empty part)
    auto empty_item = [&](const KeysItem& x) {
      const int t = x.t0 + mine_from;
      if (tok >= prm.tokens || t >= x.queries) return;
      if (k.splits > 1) {
        k.part_ml[part_row(x)] = make_float2(0.f, 0.f);
        return;
      }
      uint4* dst = reinterpret_cast<uint4*>(k.o + 2 * out_row(x, t));
      for (int e = 0; e < D / 8; ++e) dst[e] = make_uint4(0u, 0u, 0u, 0u);
      if (k.lse) *lse_at(x, t) = -INFINITY;
    };
    // this group's next item (one that has tiles for it), others on the way: key tiles are counted, rows without keys answered
    auto advance = [&](KeysItem& x) -> bool {
      for (; at < prm.items; at += pairs) {
        if (!item_at(prm, at, x) || (w == 1 && !x.two && x.j0 >= x.j1)) continue;
        if (x.j0 >= x.j1) { empty_item(x); continue; }
        if (w == 1 && !x.two) { tn += (uint32_t)(x.j1 - x.j0); continue; }
        return true;
      }
      return false;
    };
    float q_scale = 1.f;                                                      // power of two that Q's row was divided by (cached keys)
    // cached keys: the group's Q rows as fp16 into shared memory
    auto put_q = [&](const KeysItem& x) -> bool {
      const int t = x.t0 + mine_from;
      const bool there = tok < prm.tokens && t < x.queries;
      const uint4* src = reinterpret_cast<const uint4*>(k.q + 2 * (x.b * k.sq.b + (long long)(x.hk * k.group + head) * k.sq.h + (long long)t * k.sq.n));
      auto piece = [&](int e) -> uint4 { return there ? __ldg(src + e) : make_uint4(0u, 0u, 0u, 0u); };
      uint32_t top = 0u;
#pragma unroll 4
      for (int e = 0; e < D / 8; ++e) {
        const uint4 u = piece(e);
        const uint32_t a = max(max(u.x & 0x7fff7fffu, u.x << 16 & 0x7fffffffu), max(u.y & 0x7fff7fffu, u.y << 16 & 0x7fffffffu)),
                       c = max(max(u.z & 0x7fff7fffu, u.z << 16 & 0x7fffffffu), max(u.w & 0x7fff7fffu, u.w << 16 & 0x7fffffffu));
        top = max(top, max(a, c));
      }
      const uint32_t ex = top >> 23;
      const bool odd = ex == 0u || ex > 252u;                                 // (zeros; infinities, NaNs)
      const float down = odd ? 1.f : __uint_as_float((254u - ex) << 23);
      q_scale = odd ? 1.f : __uint_as_float(ex << 23);
      if (qn > 0 && !wait(cb + Q_EMPTY + 8 * w, qn - 1u)) return false;
      uint8_t* line = smem + w * TILE + row * 128;
#pragma unroll 2
      for (int e = 0; e < D / 8; ++e) {
        const uint4 u = piece(e);
        const uint4 h = make_uint4(f16_pair(bf16lo(u.x) * down, bf16hi(u.x) * down), f16_pair(bf16lo(u.y) * down, bf16hi(u.y) * down),
                                   f16_pair(bf16lo(u.z) * down, bf16hi(u.z) * down), f16_pair(bf16lo(u.w) * down, bf16hi(u.w) * down));
        *reinterpret_cast<uint4*>(line + (e / 8) * PANEL + (((e & 7) ^ (row & 7)) << 4)) = h;
      }
      fence_async_smem();
      __syncwarp();
      mbar_arrive_cluster_if(lead + Q_FULL + 8 * w, sole);
      ++qn;
      return true;
    };

    // (What happens once per item stands here once, and in loops that are not unrolled: the tile's own code is what the instruction cache is for.)
    bool mine = false, begun = false;
    int t = 0;
    float m = 0.f, l = 0.f;
    KeysItem done;
    while (true) {
      const bool more = advance(it);
      // the next item's Q first, so that its S can start
      if (PAGED && more && !put_q(it)) break;
      if (begun) {
        // ---- epilogue
        if (!wait(cb + O_DONE + 8 * w, dn)) break;
        ++dn;
        tc_fence_after();
        const float inv = l != 0.f ? 1.f / l : 0.f;
        const bool parts = k.splits > 1;
        const long long pr = parts && mine ? part_row(done) : 0;
        if (!parts) {
          uint8_t* dst = k.o + 2 * (mine ? out_row(done, t) : 0);
#pragma unroll 1
          for (int c = 0; c < D; c += 32) {
            uint32_t ov[32];
            tmem_ld32(o_tmem + c, ov);
            tc_wait_ld32(ov);
#pragma unroll
            for (int e = 0; e < 16; ++e) ov[e] = pack_bf16(__uint_as_float(ov[2 * e]) * inv, __uint_as_float(ov[2 * e + 1]) * inv);
            if (mine) {
              uint4* d4 = reinterpret_cast<uint4*>(dst + 2 * c);
#pragma unroll
              for (int e = 0; e < 16; e += 8) {
                const uint4 lo = make_uint4(ov[e], ov[e + 1], ov[e + 2], ov[e + 3]), hi = make_uint4(ov[e + 4], ov[e + 5], ov[e + 6], ov[e + 7]);
                if (prm.wide) {
                  stg32(d4 + e / 4, lo, hi);
                } else {
                  d4[e / 4] = lo;
                  d4[e / 4 + 1] = hi;
                }
              }
            }
          }
        } else {
          // A lane has a row of D floats; 64 bytes of each of the warp's 32 rows at a time go through shared memory, so that four lanes store them side by
          // side (a clip's chunk, four splits: 2 121 -> 2 060 us.  Rows of bf16 leave sooner from their lanes: a clip over two prompts 408 us, this way 428)
          uint8_t* mine_out = reinterpret_cast<uint8_t*>(k.part_o + pr * D);
          uint8_t* rows_out[4];                                               // rows 8 i + lane / 4; null: not there
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const unsigned long long a = __shfl_sync(0xffffffffu, (unsigned long long)(mine ? mine_out : nullptr), 8 * i + (lane >> 2));
            rows_out[i] = a ? reinterpret_cast<uint8_t*>(a) + 16 * (lane & 3) : nullptr;
          }
          uint8_t* way = smem + Smem<D>::OUT + (warp - 8) * 2048;
#pragma unroll 1
          for (int c = 0; c < D / 16; ++c) {
            uint32_t ov[16];
            tmem_ld16(o_tmem + 16 * c, ov);
            tc_wait_ld16(ov);
            // (16-byte pieces of a row's 64 bytes, turned by the row so that neither side meets a bank twice)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              *reinterpret_cast<uint4*>(way + lane * 64 + ((e ^ (lane >> 1 & 3)) << 4)) = make_uint4(ov[4 * e], ov[4 * e + 1], ov[4 * e + 2], ov[4 * e + 3]);
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int from = 8 * i + (lane >> 2);
              const uint4 u = *reinterpret_cast<const uint4*>(way + from * 64 + (((lane & 3) ^ (from >> 1 & 3)) << 4));
              if (rows_out[i]) *reinterpret_cast<uint4*>(rows_out[i] + 64 * c) = u;
            }
            __syncwarp();
          }
        }
        tc_fence_before();
        __syncwarp();
        mbar_arrive_cluster_if(lead + O_FREE + 8 * w, sole);
        const float m_fin = (m > -INFINITY ? m : 0.f) - UP;                   // (of a NaN 0 too: what splits are joined by is a number)
        if (mine && parts) k.part_ml[pr] = make_float2(m_fin, l);
        if (mine && !parts && k.lse) *lse_at(done, t) = l != 0.f ? (m_fin + log2f(l)) * 0.6931471805599453f : -INFINITY;
      }
      if (!more) break;
      begun = true;
      t = it.t0 + mine_from;
      mine = tok < prm.tokens && t < it.queries;
      const int seen = mine ? keys_seen(k, it.keys, it.queries, t) : it.keys;
      const float cc = k.scale_log2 * q_scale;
      m = -INFINITY;
      l = 0.f;
      uint32_t sv[64], pv[16];
      // half number i of the item on its way from tensor memory
      auto fetch = [&](int i) -> bool {
        const uint32_t h = fn & 1u, sh = s_tmem + 64 * h;
        if (!wait(cb + S_FULL + 16 * w + 8 * h, fn >> 1)) return false;
        ++fn;
        tc_fence_after();
        // keys that a row does not see: -inf into S (rare, and short: the half's own code is what the groups' time goes into)
        const int key0 = it.j0 * KT + 64 * i, valid = seen - key0;
        const bool masked = !PAGED && k.mask != nullptr;
        if (masked || __any_sync(0xffffffffu, valid < 64)) {
#pragma unroll 1
          for (int e0 = 0; e0 < 64; e0 += 32) {
            const int v = valid - e0;
            uint32_t bits = v >= 32 ? 0xffffffffu : v <= 0 ? 0u : (1u << v) - 1u, x[32];
            if (masked) {
              const int key = key0 + e0 + lane;
              bits &= __ballot_sync(0xffffffffu, key < it.keys && __ldg(k.mask + it.b * k.mask_stride + key) != 0);
            }
            tmem_ld32(sh + e0, x);
            tc_wait_ld32(x);
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (!(bits >> e & 1u)) x[e] = 0xff800000u;
            tmem_st32(sh + e0, x);
          }
          tc_wait_st();
        }
        tmem_ld32(sh, sv);
        tmem_ld32(sh + 32, sv + 32);
        return true;
      };
      const int halves = 2 * (it.j1 - it.j0);
      if (!fetch(0)) { ok = false; break; }
#pragma unroll 1
      for (int i = 0; i < halves; ++i) {
        const int h = i & 1;
        const float4* sc = scales + ((tn + (uint32_t)(i >> 1)) % SCALE_RING) * 8;
        const uint32_t sh = s_tmem + 64 * h;
        {
          tc_wait_ld64(sv);
          // P = 2^(S c + a - ref) of 32 keys and their sum (cached keys: over V's scale).  Of eight pairs POLY's go the way of ex2_poly: the exponentials' pipe
          // would be busy for as long as the MMAs take with all of them
          auto exps = [&](int q, float ref) -> float {
            float sum = 0.f;
#pragma unroll
            for (int g = 2 * q; g < 2 * q + 2; ++g) {
              const float4 f = PAGED ? sc[4 * h + g] : make_float4(1.f, 0.f, 1.f, 0.f);
              const float c = PAGED ? logit_factor(cc, f.x) : cc, nm = PAGED ? f.y - ref : -ref;
              const uint64_t c2 = pack2(c, c), nm2 = pack2(nm, nm);
              uint64_t sum2 = pack2(0.f, 0.f);
#pragma unroll
              for (int e = 0; e < 16; e += 2) {
                uint64_t p2 = fma2(pack2(__uint_as_float(sv[16 * g + e]), __uint_as_float(sv[16 * g + e + 1])), c2, nm2);
                float p0, p1;
                if (POLY >> (e / 2) & 1) {
                  p2 = ex2_poly(p2);
                  unpack2(p2, p0, p1);
                } else {
                  unpack2(p2, p0, p1);
                  p0 = ex2(p0);
                  p1 = ex2(p1);
                  p2 = pack2(p0, p1);
                }
                sum2 = add2(sum2, p2);
                pv[8 * (g - 2 * q) + e / 2] = PAGED ? f16_pair(p0, p1) : pack_bf16(p0, p1);
              }
              float s0, s1;
              unpack2(sum2, s0, s1);
              sum = PAGED ? fmaf(s0 + s1, f.z, sum) : sum + (s0 + s1);
            }
            return sum;
          };
          auto maximum = [&]() -> float {
            float mx = -INFINITY;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
              float a = __uint_as_float(sv[16 * g]), b = __uint_as_float(sv[16 * g + 1]);
#pragma unroll
              for (int e = 2; e < 14; e += 4) {
                a = max3_nan(a, __uint_as_float(sv[16 * g + e]), __uint_as_float(sv[16 * g + e + 1]));
                b = max3_nan(b, __uint_as_float(sv[16 * g + e + 2]), __uint_as_float(sv[16 * g + e + 3]));
              }
              a = max3_nan(a, __uint_as_float(sv[16 * g + 14]), __uint_as_float(sv[16 * g + 15]));
              if (PAGED) {
                const float4 f = sc[4 * h + g];
                mx = max_nan(mx, fmaf(max_nan(a, b), logit_factor(cc, f.x), f.y));
              } else {
                mx = max3_nan(mx, a, b);
              }
            }
            return PAGED ? mx : mx * cc;
          };
          auto reference = [&]() -> float { return (m > -INFINITY ? m : 0.f) - UP; };
          const bool first = i == 0;
          // (a logit that is a NaN or +infinity makes the row's sum, and with it the row, a NaN, whatever the exponentials make of it: ex2_poly takes a
          // NaN for -127)
          if (first) {
            m = maximum();
            l = nan_if_endless(m);
          }
          float ref = reference(), sum = exps(0, ref);
          if (!first) {
            const float mx = maximum();
            l += nan_if_endless(mx);
            if (__any_sync(0xffffffffu, mx > m + LAZY)) {
              // (O is at rest once P V of the half before has completed)
              if (!wait(cb + PV_DONE + 8 * w, hn - 1u)) { ok = false; break; }
              tc_fence_after();
              float f = 1.f;
              if (mx > m + LAZY) {
                f = ex2(m - mx);
                m = mx;
                l *= f;
              }
#pragma unroll 1
              for (int c = 0; c < D; c += 16) {
                tmem_ld16(o_tmem + c, pv);
                tc_wait_ld16(pv);
#pragma unroll
                for (int e = 0; e < 16; ++e) pv[e] = __float_as_uint(__uint_as_float(pv[e]) * f);
                tmem_st16(o_tmem + c, pv);
              }
              ref = reference();
              sum = exps(0, ref);
            }
          }
          l += sum;
          tmem_st16(sh, pv);
          l += exps(1, ref);
          tmem_st16(sh + 16, pv);
          tc_wait_st();
          tc_fence_before();
          __syncwarp();
          mbar_arrive_cluster_if(lead + P_FULL + 16 * w + 8 * h, sole);
          ++hn;
          if (i + 1 < halves && !fetch(i + 1)) { ok = false; break; }
        }
      }
      if (!ok) break;
      tn += (uint32_t)(it.j1 - it.j0);
      done = it;
      at += pairs;
    }
    if (PAGED && ok && qn > 0) (void)wait(cb + Q_EMPTY + 8 * w, qn - 1u);     // (as the loaders do)
  }

  // ---------------------------------------------------------------- tear-down
  __syncthreads();
  if (*abort_flag) {
    // copies and MMAs still in flight land before shared memory and TMEM go away
    const long long t0 = clock64();
    while (clock64() - t0 < 2000000) {}
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();                                                         // nothing arrives at a CTA that has gone
  if (warp == 0) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
  if (threadIdx.x == 0 && *abort_flag && prm.k.status) atomicOr(prm.k.status, SVA_DEV_TIMEOUT);
}

// ---------------------------------------------------------------------------------------------------------------- host side
typedef CUresult (*keys_encode_t)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static keys_encode_t keys_encode() {
  static const keys_encode_t fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) p = nullptr;
    return reinterpret_cast<keys_encode_t>(p);
  }();
  return fn;
}
// 4-D map of bf16, box of box0 channels (64, or 32: the swizzle's span) and of the next two dimensions; sizes and element strides of dimensions 1 to 3
static int keys_map(CUtensorMap* map, const void* ptr, int d, const long long n[3], const long long s[3], int box0, int box1, int box2) {
  const keys_encode_t enc = keys_encode();
  if (!enc) return SVA_ERR_CUDA;
  const cuuint64_t dims[4] = {(cuuint64_t)d, (cuuint64_t)n[0], (cuuint64_t)n[1], (cuuint64_t)n[2]};
  cuuint64_t strides[3];
  for (int i = 0; i < 3; ++i) strides[i] = n[i] > 1 ? 2 * (cuuint64_t)s[i] : 2 * (cuuint64_t)d;      // (a dimension of one may carry any)
  const cuuint32_t box[4] = {(cuuint32_t)box0, (cuuint32_t)box1, (cuuint32_t)box2, 1}, each[4] = {1, 1, 1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(ptr), dims, strides, box, each, CU_TENSOR_MAP_INTERLEAVE_NONE,
             box0 == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS ? SVA_OK : SVA_ERR_CUDA;
}

static int g_debug_keys = 0;
void keys_set_debug_mode(int v) { g_debug_keys = v; }
int keys_set_wait_limit(long long cycles) { return set_wait_limit(cycles); }

template <int D, bool PAGED>
static int launch_tc(const KeysTcParams& prm, const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, int sms, cudaStream_t st) {
  static DeviceOnce once;
  auto kern = keys_tc_kernel<D, PAGED>;
  const int rc = once.run([&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kt::Smem<D>::BYTES) == cudaSuccess; });
  if (rc) return rc;
  const unsigned pairs = prm.items < (unsigned)(sms / 2) ? prm.items : (unsigned)(sms / 2);
  return launch_dep_cluster(2, kern, dim3(2 * pairs), kt::THREADS, kt::Smem<D>::BYTES, st, tq, tk, tv, prm);
}

int launch_keys_tc(const KeysParams& k, bool paged, int sms, cudaStream_t st) {
  KeysTcParams prm = {};
  prm.k = k;
  prm.tokens = 128 / k.group;
  prm.quads = (k.tiles + 3) / 4;
  const long long items = (long long)k.B * k.Hk * prm.quads * k.splits;
  if (items > 0x7fffffffLL) return SVA_ERR_UNSUPPORTED;
  prm.items = (uint32_t)items;
  prm.wide = (reinterpret_cast<uintptr_t>(k.o) & 31u) == 0 && ((k.so.b | k.so.h | k.so.n) & 15) == 0;
  prm.debug = g_debug_keys;
  CUtensorMap tq = {}, tk = {}, tv = {};
  if (!paged) {
    // (row tiles: the group's heads of each token side by side)
    const long long qn[3] = {k.Hq, k.M, k.B}, qs[3] = {k.sq.h, k.sq.n, k.sq.b};
    int rc = keys_map(&tq, k.q, k.d, qn, qs, 64, k.group, prm.tokens);
    const int hk = k.sk.h == 0 ? 1 : k.Hk, bk = k.sk.b == 0 ? 1 : k.B, hv = k.sv.h == 0 ? 1 : k.Hk, bv = k.sv.b == 0 ? 1 : k.B;
    prm.k_each_h = hk > 1; prm.k_each_b = bk > 1; prm.v_each_h = hv > 1; prm.v_each_b = bv > 1;
    const long long kn[3] = {k.S, hk, bk}, ks[3] = {k.sk.n, k.sk.h, k.sk.b}, vn[3] = {k.S, hv, bv}, vs[3] = {k.sv.n, k.sv.h, k.sv.b};
    if (!rc) rc = keys_map(&tk, k.k, k.d, kn, ks, 64, kt::KT / 4, 1);
    if (!rc) rc = keys_map(&tv, k.v, k.d, vn, vs, k.d / 2, kt::KT, 1);
    if (rc) return rc;
  }
  if (paged) return k.d == 128 ? launch_tc<128, true>(prm, tq, tk, tv, sms, st) : launch_tc<64, true>(prm, tq, tk, tv, sms, st);
  return k.d == 128 ? launch_tc<128, false>(prm, tq, tk, tv, sms, st) : launch_tc<64, false>(prm, tq, tk, tv, sms, st);
}

}  // namespace sva
