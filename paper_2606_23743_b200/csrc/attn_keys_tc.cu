// Attention of many rows over many keys (sva_cached_attn_fwd, sva_cross_attn_fwd) on the tensor cores.
//
// A CTA takes items: 256 rows (two tiles of 128) of one key head, and a range of its key tiles of 128.  A row is a query of one of the heads that
// share the key head; a tile holds the `group` heads of 128 / group tokens.  Both tiles use each key tile, so that it is brought in (and, where it
// is codes, converted) once for 256 rows.  Roles:
//   warp  0          issues the MMAs;  warp 1  brings in Q for bf16 keys (TMA)
//   warps 4-7        bf16 keys: 4 brings in K and 5 V (TMA), 6 and 7 put zeros into rows of V that are left out
//                    cached keys: all four read codes, convert them to fp16 (exactly) and store them in the layout that TMA would leave
//   warps 8-11, 12-15   softmax of tile 0 and of tile 1; thread <-> row <-> TMEM lane.  Also the epilogue, and for cached keys the Q tile
// Per key tile j and row tile w: S_w = Q_w K^T (A, B from shared memory), P_w over the columns of S_w, O_w += P_w V (A from TMEM, V as an MN-major
// B operand).  TMEM: S_0 | S_1 | O_0 | O_1, 128 columns each.  The issuing order is P V_0(j), S_0(j+1), P V_1(j), S_1(j+1): while one group computes its
// exponentials the MMAs of the other run.  S_w(j+1) overwrites P_w(j), which P V_w(j) before it reads: MMAs run in the order of their issue.
//
// The reference m of a row's exponentials follows its maximum lazily: O is rescaled only when a tile's maximum is more than LAZY powers of two above m
// (probabilities reach 2^LAZY; sums are fp32).  Cached keys: K's scale is a factor of the logits, log2 of V's an addend (both per 16 keys), see
// attn_keys.cu; P is fp16 and lies at 2^(UP + LAZY) at most.
//
// Every wait is bounded; when one runs out all roles leave, the CTA reports SVA_DEV_TIMEOUT and its rows are not stored.
#include <cuda_fp16.h>

#include "attn_keys.cuh"
#include "tc_ptx.cuh"

namespace sva {

namespace kt {
constexpr int THREADS = 512;
constexpr int KT = 128;                               // keys of a tile
constexpr int PANEL = 128 * 128;                      // 128 rows x 128 bytes (64 channels)
constexpr int STAGES = 2;
constexpr int SCALE_RING = 4;
constexpr float LAZY = 7.0f;
constexpr int POLY = 0b10010010;                      // pairs of eight whose exponentials are polynomials
constexpr float UP_F16 = 8.0f;                        // log2 of a probability at the reference (fp16: 2^15 at most)
// shared memory (bytes from a 1024-byte boundary): Q tiles | K stages | V stages | control
template <int D> struct Smem {
  static constexpr int TILE = D / 64 * PANEL, K = 2 * TILE, V = K + STAGES * TILE, CTRL = V + STAGES * TILE, BYTES = CTRL + 1024 + 1024;
};
// control block: barriers (8 bytes each, pairs), then TMEM base and abort flag, then the scales' ring
enum { K_FULL = 0, K_EMPTY = 16, V_LAND = 32, V_FULL = 48, V_EMPTY = 64, Q_FULL = 80, Q_EMPTY = 96, S_FULL = 112, P_FULL = 128, O_DONE = 144,
       O_FREE = 160, P_HALF = 176, TMEM_BASE = 192, ABORT = 196, SCALES = 256 };      // SCALES: [ring][8 chunks of 16 keys]{k scale, log2 v scale, 1 / v scale, -}
}  // namespace kt

struct KeysTcParams {
  KeysParams k;
  int tokens;                                         // of a row tile: 128 / group
  int pairs;                                          // pairs of row tiles per key head
  uint32_t items;
  int k_each_h, k_each_b, v_each_h, v_each_b;         // 0: heads / items share K, V (the maps then have one)
  bool wide;                                          // 32-byte stores into o
  int debug;
};

// An item: rows [t0, t0 + 2 * tokens) of (b, hk), key tiles [j0, j1).
struct KeysItem {
  int b, hk, pair, split, keys, queries, t0, j0, j1;
  bool two;                                           // the second tile has rows
};

__device__ __forceinline__ void tc_mma_ss_16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc, uint32_t elected) {
  asm volatile("{\n.reg .pred p, q;\nsetp.ne.b32 p, %4, 0;\nsetp.ne.b32 q, %5, 0;\n"
               "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
               ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc), "r"(elected) : "memory");
}
__device__ __forceinline__ uint32_t f16_pair(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// Codes 0, 1 (sel 0x1404) or 2, 3 (0x3424) of four as fp16 values, times 2^-8: a code's exponent and significand are moved to where fp16 has
// them, which is exact for denormals too.  (The conversion instruction shares its pipe with the exponentials.)
__device__ __forceinline__ uint32_t f16_of_codes(uint32_t codes, uint32_t sel) {
  const uint32_t x = __byte_perm(codes, 0u, sel);
  return (x & 0x80008000u) | (x >> 1 & 0x3f803f80u);
}
constexpr float CODE_UNIT = 256.0f;                   // what those values are to be multiplied by

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
  x.pair = (int)(i % (uint32_t)prm.pairs); i /= (uint32_t)prm.pairs;
  x.split = 0;
  if (k.splits > 1) { x.split = (int)(i % (uint32_t)k.splits); i /= (uint32_t)k.splits; }
  x.hk = (int)(i % (uint32_t)k.Hk);
  x.b = (int)(i / (uint32_t)k.Hk);
  x.keys = seq_keys(k, x.b);
  x.queries = seq_queries(k, x.b);
  x.t0 = x.pair * 2 * prm.tokens;
  if (x.t0 >= x.queries) return false;
  x.two = x.t0 + prm.tokens < x.queries;
  const int end = keys_seen(k, x.keys, x.queries, min(x.t0 + (x.two ? 2 : 1) * prm.tokens, x.queries) - 1);
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
// The next item at or after i (a CTA's are gridDim.x apart) that has key tiles; false at the end.
__device__ __forceinline__ bool next_item(const KeysTcParams& prm, uint32_t& i, KeysItem& x) {
  for (; i < prm.items; i += gridDim.x)
    if (item_at(prm, i, x) && x.j0 < x.j1) return true;
  return false;
}

template <int D, bool PAGED>
__global__ void __launch_bounds__(kt::THREADS, 1)
keys_tc_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
               const KeysTcParams prm) {
  using namespace kt;
  constexpr int TILE = Smem<D>::TILE, OFF_K = Smem<D>::K, OFF_V = Smem<D>::V, PANELS = D / 64;
  constexpr int FMT = PAGED ? 0 : 1;                                          // fp16 or bf16 operands
  constexpr uint32_t IDESC_S = instr_desc(128, 128, FMT, false), IDESC_O = instr_desc(128, D, FMT, true);
  constexpr float UP = PAGED ? UP_F16 : 0.f;
  constexpr uint32_t COL_S = 0, COL_O = 256;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const uint32_t sbase = smem_u32(smem), cb = sbase + Smem<D>::CTRL;
  uint8_t* ctrl = smem + Smem<D>::CTRL;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(ctrl + ABORT);
  float4* scales = reinterpret_cast<float4*>(ctrl + SCALES);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int w = 0; w < 2; ++w) {
      mbar_init(cb + K_FULL + 8 * w, PAGED ? 4 : 1);
      mbar_init(cb + K_EMPTY + 8 * w, 1);
      mbar_init(cb + V_LAND + 8 * w, 1);
      mbar_init(cb + V_FULL + 8 * w, PAGED ? 4 : 2);
      mbar_init(cb + V_EMPTY + 8 * w, 1);
      mbar_init(cb + Q_FULL + 8 * w, PAGED ? 128 : 1);
      mbar_init(cb + Q_EMPTY + 8 * w, 1);
      mbar_init(cb + S_FULL + 8 * w, 1);
      mbar_init(cb + P_HALF + 8 * w, 128);
      mbar_init(cb + P_FULL + 8 * w, 128);
      mbar_init(cb + O_DONE + 8 * w, 1);
      mbar_init(cb + O_FREE + 8 * w, 128);
    }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  if (!PAGED && warp == 1 && lane == 0) { prefetch_tmap(&tm_q); prefetch_tmap(&tm_k); prefetch_tmap(&tm_v); }
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(cb + TMEM_BASE), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(ctrl + TMEM_BASE);
  uint32_t at = blockIdx.x + (uint32_t)grid_dep_wait();
  KeysItem it;
  bool ok = true;

  if (warp < 4) {
    if (warp == 0) {
      // ------------------------------------------------------------------------------------------------ issuer
      const uint32_t el = elect_one();
      const uint64_t qd0 = smem_desc(sbase, 16, 1024), kd0 = smem_desc(sbase + OFF_K, 16, 1024),
                     vd0 = smem_desc(sbase + OFF_V, PANEL, 1024);
      uint32_t kn = 0, vn = 0, qn[2] = {0, 0}, pn[2] = {0, 0}, on[2] = {0, 0};      // uses so far
      auto wait = [&](uint32_t bar, uint32_t use) { return __all_sync(0xffffffffu, mbar_wait(bar, use & 1u, abort_flag)) != 0; };
      auto issue_s = [&](int w, bool first, bool last) -> bool {      // from the K tile in use number kn
        if (first && !wait(cb + Q_FULL + 8 * w, qn[w]++)) return false;
        tc_fence_after();
        const uint64_t qd = qd0 + (uint64_t)(w * (TILE >> 4)), kd = kd0 + (uint64_t)((kn & 1u) * (TILE >> 4));
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          const uint64_t off = (uint64_t)((kk / 4) * (PANEL >> 4) + (kk % 4) * 2);
          tc_mma_ss_16(tmem + COL_S + 128 * w, qd + off, kd + off, IDESC_S, kk > 0 ? 1u : 0u, el);
        }
        tc_commit(cb + S_FULL + 8 * w, el);
        if (last) tc_commit(cb + Q_EMPTY + 8 * w, el);
        return true;
      };
      auto issue_pv = [&](int w, bool first, bool last) -> bool {     // with the V tile in use number vn
        if (!wait(cb + P_HALF + 8 * w, pn[w])) return false;
        if (first && on[w] > 0 && !wait(cb + O_FREE + 8 * w, on[w] - 1u)) return false;
        if (first) ++on[w];
        const uint64_t vd = vd0 + (uint64_t)((vn & 1u) * (TILE >> 4));
#pragma unroll
        for (int i = 0; i < KT / 16; ++i) {
          // 16 keys = 16 rows of 128 bytes; in the order in which P is made, 32 keys at a time: quarters 0, 3, 1, 2, each where its S was
          const int quarter = i < 2 ? 0 : i < 4 ? 3 : i / 2 - 1, kk = 2 * quarter + (i & 1);
          if (i == KT / 32 && !wait(cb + P_FULL + 8 * w, pn[w]++)) return false;
          if (i % (KT / 32) == 0) tc_fence_after();
          tc_mma_ts(tmem + COL_O + 128 * w, tmem + COL_S + 128 * w + 32 * quarter + 8 * (i & 1), vd + (uint64_t)(kk * 128), IDESC_O,
                    !first || i > 0 ? 1u : 0u, el);
        }
        if (last) tc_commit(cb + O_DONE + 8 * w, el);
        return true;
      };
      // S of the first tile of an item, both row tiles
      auto begin = [&](const KeysItem& x) -> bool {
        if (!wait(cb + K_FULL + 8 * (kn & 1u), kn >> 1)) return false;
        const bool last = x.j1 - x.j0 == 1;
        if (!issue_s(0, true, last) || (x.two && !issue_s(1, true, last))) return false;
        tc_commit(cb + K_EMPTY + 8 * (kn & 1u), el);
        ++kn;
        return true;
      };
      bool more = next_item(prm, at, it);
      if (more) ok = begin(it);
      while (more && ok) {
        for (int j = it.j0; j < it.j1 && ok; ++j) {
          const bool first = j == it.j0, last = j + 1 == it.j1;
          ok = wait(cb + V_FULL + 8 * (vn & 1u), vn >> 1) && issue_pv(0, first, last);
          if (ok && !last) {
            ok = wait(cb + K_FULL + 8 * (kn & 1u), kn >> 1) && issue_s(0, false, j + 2 == it.j1);
          }
          if (ok && it.two) ok = issue_pv(1, first, last);
          if (!ok) break;
          tc_commit(cb + V_EMPTY + 8 * (vn & 1u), el);
          ++vn;
          if (!last) {
            if (it.two) ok = issue_s(1, false, j + 2 == it.j1);
            if (!ok) break;
            tc_commit(cb + K_EMPTY + 8 * (kn & 1u), el);
            ++kn;
          }
        }
        if (!ok) break;
        at += gridDim.x;
        more = next_item(prm, at, it);
        if (more) ok = begin(it);
      }
    } else if (warp == 1 && !PAGED) {
      // ------------------------------------------------------------------------------------------------ Q (bf16 keys)
      const uint32_t el = elect_one();
      const uint32_t bytes = (uint32_t)(prm.tokens * prm.k.group) * 128 * PANELS;
      uint32_t qn[2] = {0, 0};
      for (; ok && next_item(prm, at, it); at += gridDim.x) {
        for (int w = 0; w < (it.two ? 2 : 1) && ok; ++w) {
          if (qn[w] > 0) ok = __all_sync(0xffffffffu, mbar_wait(cb + Q_EMPTY + 8 * w, (qn[w] - 1u) & 1u, abort_flag));
          if (!ok) break;
          ++qn[w];
          const uint32_t bar = cb + Q_FULL + 8 * w;
          mbar_expect_tx_if(bar, bytes, el);
#pragma unroll
          for (int p = 0; p < PANELS; ++p)
            tma_load_4d_if(sbase + w * TILE + p * PANEL, &tm_q, bar, 64 * p, it.hk * prm.k.group, it.t0 + w * prm.tokens, it.b, el);
        }
      }
    }
  } else if (warp < 8) {
    if (!PAGED) {
      // ------------------------------------------------------------------------------------------------ K, V (bf16)
      uint32_t n = 0;
      const uint32_t el = elect_one();
      for (; ok && next_item(prm, at, it); at += gridDim.x) {
        for (int j = it.j0; j < it.j1 && ok; ++j, ++n) {
          const uint32_t s = n & 1u, use = n >> 1;
          if (warp < 6) {
            const uint32_t empty = cb + (warp == 4 ? K_EMPTY : V_EMPTY) + 8 * s, full = cb + (warp == 4 ? K_FULL : V_LAND) + 8 * s;
            if (use > 0) ok = __all_sync(0xffffffffu, mbar_wait(empty, (use - 1u) & 1u, abort_flag));
            if (!ok || ((prm.debug & 2048) && n >= 1)) { ok = false; break; }     // (test aid: later tiles never come)
            mbar_expect_tx_if(full, TILE, el);
#pragma unroll
            for (int p = 0; p < PANELS; ++p) {
              if (warp == 4) tma_load_4d_if(sbase + OFF_K + s * TILE + p * PANEL, &tm_k, full, 64 * p, j * KT, it.hk * prm.k_each_h, it.b * prm.k_each_b, el);
              else tma_load_4d_if(sbase + OFF_V + s * TILE + p * PANEL, &tm_v, full, 64 * p, j * KT, it.hk * prm.v_each_h, it.b * prm.v_each_b, el);
            }
          } else {
            // rows of V whose keys are left out: zeros, whatever they hold (their probabilities are 0, and 0 times a NaN is one)
            ok = __all_sync(0xffffffffu, mbar_wait(cb + V_LAND + 8 * s, use & 1u, abort_flag));
            if (!ok) break;
            if (prm.k.mask || (it.keys < prm.k.S && (j + 1) * KT > it.keys)) {
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const int row = (warp - 6) * 64 + 32 * i + lane, key = j * KT + row;
                bool out = key >= it.keys;
                if (!out && prm.k.mask) out = __ldg(prm.k.mask + it.b * prm.k.mask_stride + key) == 0;
                if (out) {
#pragma unroll
                  for (int p = 0; p < PANELS; ++p)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                      *reinterpret_cast<uint4*>(smem + OFF_V + s * TILE + p * PANEL + row * 128 + ((e ^ (row & 7)) << 4)) = make_uint4(0u, 0u, 0u, 0u);
                }
              }
              fence_async_smem();
              __syncwarp();
            }
            if (lane == 0) mbar_arrive(cb + V_FULL + 8 * s);
          }
        }
      }
    } else {
      // ------------------------------------------------------------------------------------------------ K, V (codes)
      // A warp converts 32 keys: chunks 2 wl and 2 wl + 1 of 16.  Four lanes hold 64 bytes of a row, 8 rows at a time: their 16-byte stores meet all banks.
      const KeysParams& k = prm.k;
      const int wl = warp - 4, piece = lane & 3, sub = lane >> 2;
      uint32_t n = 0;
      auto pages_of = [&](const KeysItem& x, int j, int id[2]) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int key = j * KT + wl * 32 + c * 16;
          id[c] = -1;
          if (key < x.keys) {
            const int e = key / k.page;
            id[c] = e < k.max_pages ? __ldg(k.table + x.b * k.table_stride + e) : -1;
            if (id[c] < 0 || id[c] >= k.pages) {
              id[c] = -1;
              if (lane == 0 && k.status) atomicOr(k.status, SVA_DEV_BAD_INDEX);
            }
          }
        }
      };
      // raw codes of a tile: [chunk][8 rows][panel]
      auto load = [&](const uint8_t* codes, const KeysItem& x, int j, const int id[2], uint4 (&r)[4 * PANELS]) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int key = j * KT + wl * 32 + c * 16;
          const long long row = ((long long)id[c] * k.Hk + x.hk) * k.page + (key - key / k.page * k.page);
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int p = 0; p < PANELS; ++p) {
              uint4& u = r[(2 * c + h) * PANELS + p];
              u = make_uint4(0u, 0u, 0u, 0u);
              if (id[c] >= 0 && key + 8 * h + sub < x.keys)
                u = __ldg(reinterpret_cast<const uint4*>(codes + (row + 8 * h + sub) * D + 64 * p + 16 * piece));
            }
        }
      };
      auto store = [&](uint8_t* tile, const uint4 (&r)[4 * PANELS]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int row = wl * 32 + 8 * i + sub;
#pragma unroll
          for (int p = 0; p < PANELS; ++p) {
            const uint4 u = r[i * PANELS + p];
            uint8_t* line = tile + p * PANEL + row * 128;
            *reinterpret_cast<uint4*>(line + (((2 * piece) ^ (row & 7)) << 4)) =
                make_uint4(f16_of_codes(u.x, 0x1404u), f16_of_codes(u.x, 0x3424u), f16_of_codes(u.y, 0x1404u), f16_of_codes(u.y, 0x3424u));
            *reinterpret_cast<uint4*>(line + (((2 * piece + 1) ^ (row & 7)) << 4)) =
                make_uint4(f16_of_codes(u.z, 0x1404u), f16_of_codes(u.z, 0x3424u), f16_of_codes(u.w, 0x1404u), f16_of_codes(u.w, 0x3424u));
          }
        }
      };
      auto wait = [&](uint32_t bar, uint32_t use) { return __all_sync(0xffffffffu, mbar_wait(bar, use & 1u, abort_flag)) != 0; };
      // one tile ahead in registers, its pages looked up another tile ahead
      struct Place { KeysItem it; uint32_t at; int j; bool more; int id[2]; };
      auto look_up = [&](Place& x) { if (x.more) pages_of(x.it, x.j, x.id); };
      auto step_on = [&](Place& x) {
        if (++x.j == x.it.j1) {
          x.at += gridDim.x;
          x.more = next_item(prm, x.at, x.it);
          x.j = x.it.j0;
        }
      };
      uint4 kr[4 * PANELS], vr[4 * PANELS];
      float ks = 1.f, vs = 1.f;                                                   // (lanes 0 and 1: of their chunk)
      bool named = false;
      auto fetch_scales = [&](const Place& x) {
        const int id = lane == 0 ? x.id[0] : x.id[1];
        named = id >= 0;
        if (lane < 2 && named) {
          ks = __ldg(k.k_scale + (long long)id * k.Hk + x.it.hk);
          vs = __ldg(k.v_scale + (long long)id * k.Hk + x.it.hk);
        }
      };
      Place nx;                                                                   // the next tile to be fetched
      nx.at = at;
      nx.more = next_item(prm, nx.at, nx.it);
      nx.j = nx.it.j0;
      bool more = nx.more;                                                        // ... and whether one has been
      look_up(nx);
      if (more) {
        load(k.k, nx.it, nx.j, nx.id, kr);
        load(k.v, nx.it, nx.j, nx.id, vr);
        fetch_scales(nx);
        step_on(nx);
        look_up(nx);
      }
      while (more) {
        const uint32_t s = n & 1u, use = n >> 1;
        if (use > 0) ok = wait(cb + K_EMPTY + 8 * s, use - 1u);
        if (!ok || ((prm.debug & 2048) && n >= 1)) break;                         // (test aid: later tiles never come)
        if (lane < 2) {
          // (K of zeros alone, scale 0: any scale will do but one that makes -inf a NaN; pages that are named wrongly: left out)
          const float v = named ? v_scale_floor(vs) : 1.f;
          scales[(n & (SCALE_RING - 1)) * 8 + 2 * wl + lane] =
              make_float4(!named || ks == 0.f ? 1.f : ks * CODE_UNIT, named ? log2f(v) : -INFINITY, 1.f / v, 0.f);
        }
        more = nx.more;
        store(smem + OFF_K + s * TILE, kr);
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(cb + K_FULL + 8 * s);
        if (more) load(k.k, nx.it, nx.j, nx.id, kr);
        if (use > 0) ok = wait(cb + V_EMPTY + 8 * s, use - 1u);
        if (!ok) break;
        store(smem + OFF_V + s * TILE, vr);
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(cb + V_FULL + 8 * s);
        if (more) {
          load(k.v, nx.it, nx.j, nx.id, vr);
          fetch_scales(nx);
          step_on(nx);
          look_up(nx);
        }
        ++n;
      }
    }
  } else {
    // ------------------------------------------------------------------------------------------------ softmax
    const KeysParams& k = prm.k;
    const int w = (warp >> 2) - 2, row = (warp & 3) * 32 + lane;
    const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t s_tmem = tmem + lane_addr + COL_S + 128 * w, o_tmem = tmem + lane_addr + COL_O + 128 * w;
    uint32_t sn = 0, qn = 0, dn = 0, tn = 0;                                  // S tiles, Q tiles, items, and key tiles of all items so far
    // where a row's output goes
    const int tok = row / k.group, head = row % k.group;
    auto out_row = [&](const KeysItem& x, int t) -> long long { return x.b * k.so.b + (long long)(x.hk * k.group + head) * k.so.h + (long long)t * k.so.n; };
    auto lse_at = [&](const KeysItem& x, int t) -> float* { return k.lse + ((long long)x.b * k.Hq + x.hk * k.group + head) * k.M + t; };
    auto part_row = [&](const KeysItem& x) -> long long {
      return (x.split * ((long long)k.B * k.Hk * k.tiles) + ((long long)x.b * k.Hk + x.hk) * k.tiles + 2 * x.pair + w) * 128 + row;
    };
    // (an item without keys: zeros; a split without: an empty part)
    auto empty_item = [&](const KeysItem& x) {
      const int t = x.t0 + w * prm.tokens + tok;
      if (tok >= prm.tokens || t >= x.queries) return;
      if (k.splits > 1) {
        k.part_ml[part_row(x)] = make_float2(0.f, 0.f);
        return;
      }
      uint4* dst = reinterpret_cast<uint4*>(k.o + 2 * out_row(x, t));
      for (int e = 0; e < D / 8; ++e) dst[e] = make_uint4(0u, 0u, 0u, 0u);
      if (k.lse) *lse_at(x, t) = -INFINITY;
    };
    // this group's next item (one that has a tile for it), others on the way: key tiles are counted, rows without keys answered
    auto advance = [&](KeysItem& x) -> bool {
      for (; at < prm.items; at += gridDim.x) {
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
      const int t = x.t0 + w * prm.tokens + tok;
      const bool there = tok < prm.tokens && t < x.queries;
      uint32_t q[D / 2];
      const uint8_t* src = k.q + 2 * (x.b * k.sq.b + (long long)(x.hk * k.group + head) * k.sq.h + (long long)t * k.sq.n);
      uint32_t top = 0u;
#pragma unroll
      for (int e = 0; e < D / 8; ++e) {
        const uint4 u = there ? __ldg(reinterpret_cast<const uint4*>(src) + e) : make_uint4(0u, 0u, 0u, 0u);
        q[4 * e] = u.x; q[4 * e + 1] = u.y; q[4 * e + 2] = u.z; q[4 * e + 3] = u.w;
      }
#pragma unroll
      for (int e = 0; e < D / 2; ++e) top = max(top, max(q[e] & 0x7fffu, q[e] >> 16 & 0x7fffu));
      const uint32_t ex = top >> 7;
      const bool odd = ex == 0u || ex > 252u;                                 // (zeros; infinities, NaNs)
      const float down = odd ? 1.f : __uint_as_float((254u - ex) << 23);
      q_scale = odd ? 1.f : __uint_as_float(ex << 23);
      if (qn > 0 && !__all_sync(0xffffffffu, mbar_wait(cb + Q_EMPTY + 8 * w, (qn - 1u) & 1u, abort_flag))) return false;
      uint8_t* line = smem + w * TILE + row * 128;
#pragma unroll
      for (int e = 0; e < D / 8; ++e) {
        uint32_t h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = f16_pair(bf16lo(q[4 * e + i]) * down, bf16hi(q[4 * e + i]) * down);
        *reinterpret_cast<uint4*>(line + (e / 8) * PANEL + (((e & 7) ^ (row & 7)) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
      }
      fence_async_smem();
      mbar_arrive(cb + Q_FULL + 8 * w);
      ++qn;
      return true;
    };

    bool more = advance(it);
    if (PAGED && more) ok = put_q(it);
    while (more && ok) {
      const int t = it.t0 + w * prm.tokens + tok;
      const bool mine = tok < prm.tokens && t < it.queries;
      const int seen = mine ? keys_seen(k, it.keys, it.queries, t) : it.keys;
      const float cc = k.scale_log2 * q_scale;
      float m = -INFINITY, l = 0.f;
      for (int j = it.j0; j < it.j1; ++j, ++tn) {
        if (!__all_sync(0xffffffffu, mbar_wait(cb + S_FULL + 8 * w, sn & 1u, abort_flag))) { ok = false; break; }
        ++sn;
        tc_fence_after();
        // keys that a row does not see: -inf into S (rare, and short: the tile's own code is what the groups' time goes into)
        const int valid = seen - j * KT;
        const bool masked = !PAGED && k.mask != nullptr;
        if (masked || __any_sync(0xffffffffu, valid < KT)) {
#pragma unroll 1
          for (int i = 0; i < 4; ++i) {
            const int v = valid - 32 * i;
            uint32_t bits = v >= 32 ? 0xffffffffu : v <= 0 ? 0u : (1u << v) - 1u, x[32];
            if (masked) {
              const int key = j * KT + 32 * i + lane;
              bits &= __ballot_sync(0xffffffffu, key < it.keys && __ldg(k.mask + it.b * k.mask_stride + key) != 0);
            }
            tmem_ld32(s_tmem + 32 * i, x);
            tc_wait_ld32(x);
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (!(bits >> e & 1u)) x[e] = 0xff800000u;
            tmem_st32(s_tmem + 32 * i, x);
          }
          tc_wait_st();
        }
        // P = 2^(S c + a - ref) of 32 keys, put where their S was, and their sum (cached keys: over V's scale).  Of eight pairs POLY's go the way of
        // ex2_poly: the exponentials' pipe would be busy for as long as the MMAs take with all of them
        const float4* sc = scales + (tn & (SCALE_RING - 1)) * 8;
        uint32_t pv[16];
        auto exps = [&](int h, const uint32_t* x, float ref) -> float {
          float sum = 0.f;
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            const float4 f = PAGED ? sc[2 * h + g] : make_float4(1.f, 0.f, 1.f, 0.f);
            const float c = PAGED ? cc * f.x : cc, nm = PAGED ? f.y - ref : -ref;
            const uint64_t c2 = pack2(c, c), nm2 = pack2(nm, nm);
            uint64_t sum2 = pack2(0.f, 0.f);
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
              uint64_t p2 = fma2(pack2(__uint_as_float(x[16 * g + e]), __uint_as_float(x[16 * g + e + 1])), c2, nm2);
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
              pv[8 * g + e / 2] = PAGED ? f16_pair(p0, p1) : pack_bf16(p0, p1);
            }
            float s0, s1;
            unpack2(sum2, s0, s1);
            sum = PAGED ? fmaf(s0 + s1, f.z, sum) : sum + (s0 + s1);
          }
          return sum;
        };
        auto maximum = [&](int h, const uint32_t* x, float mx) -> float {
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            float a = __uint_as_float(x[16 * g]), b = __uint_as_float(x[16 * g + 1]);
#pragma unroll
            for (int e = 2; e < 14; e += 4) {
              a = max3_nan(a, __uint_as_float(x[16 * g + e]), __uint_as_float(x[16 * g + e + 1]));
              b = max3_nan(b, __uint_as_float(x[16 * g + e + 2]), __uint_as_float(x[16 * g + e + 3]));
            }
            a = max3_nan(a, __uint_as_float(x[16 * g + 14]), __uint_as_float(x[16 * g + 15]));
            if (PAGED) {
              const float4 f = sc[2 * h + g];
              mx = max_nan(mx, fmaf(max_nan(a, b), cc * f.x, f.y));
            } else {
              mx = max3_nan(mx, a, b);
            }
          }
          return mx;
        };
        auto reference = [&]() -> float { return (m == -INFINITY ? 0.f : m) - UP; };
        // Quarters of 32 keys.  The maximum of all four is taken beside the first one's exponentials (of an item's first tile: before them), which
        // are done again where it has outgrown the reference.  The second and third are read twice for that: the whole tile would take 128 registers.
        uint32_t x[32], y[32];
        tmem_ld32(s_tmem, x);
        tmem_ld32(s_tmem + 32, y);
        tc_wait_ld32(x);
        tc_wait_ld32(y);
        float mx = maximum(1, y, maximum(0, x, -INFINITY)), sum = 0.f;
        const bool first = j == it.j0;
        tmem_ld32(s_tmem + 64, y);
        if (!first) sum = exps(0, x, reference());
        tc_wait_ld32(y);
        mx = maximum(2, y, mx);
        tmem_ld32(s_tmem + 96, y);
        tc_wait_ld32(y);
        mx = maximum(3, y, mx);
        if (!PAGED) mx *= cc;
        if (first) m = mx;
        else if (mx != mx) l = mx;                                            // (a NaN: the row's sum, and with it the row, becomes one)
        if (first || __any_sync(0xffffffffu, mx > m + LAZY)) {
          // (P V of the tile before has completed: S of this one came after it)
          if (!first) {
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
          }
          sum = exps(0, x, reference());
        }
        const float ref = reference();
        tmem_st16(s_tmem, pv);
        tmem_ld32(s_tmem + 32, x);
        sum += exps(3, y, ref);
        tmem_st16(s_tmem + 96, pv);
        tc_wait_st();
        tc_wait_ld32(x);
        tc_fence_before();
        mbar_arrive(cb + P_HALF + 8 * w);
        tmem_ld32(s_tmem + 64, y);
        sum += exps(1, x, ref);
        tmem_st16(s_tmem + 32, pv);
        tc_wait_ld32(y);
        sum += exps(2, y, ref);
        tmem_st16(s_tmem + 64, pv);
        l += sum;
        tc_wait_st();
        tc_fence_before();
        mbar_arrive(cb + P_FULL + 8 * w);
      }
      if (!ok) break;
      // ---- epilogue; the next item's Q first, so that its S can start
      const KeysItem done = it;
      at += gridDim.x;
      more = advance(it);
      if (PAGED && more && !put_q(it)) { ok = false; break; }
      if (!__all_sync(0xffffffffu, mbar_wait(cb + O_DONE + 8 * w, dn & 1u, abort_flag))) { ok = false; break; }
      ++dn;
      tc_fence_after();
      constexpr float UNIT = PAGED ? CODE_UNIT : 1.f;
      const float inv = l != 0.f ? UNIT / l : 0.f;
      if (k.splits > 1) {
        const long long pr = mine ? part_row(done) : 0;
        auto scaled = [](uint32_t x) -> uint32_t { return __float_as_uint(__uint_as_float(x) * UNIT); };
#pragma unroll 1
        for (int c = 0; c < D; c += 32) {
          uint32_t ov[32];
          tmem_ld32(o_tmem + c, ov);
          tc_wait_ld32(ov);
          if (mine) {
            float* dst = k.part_o + pr * D + c;
#pragma unroll
            for (int e = 0; e < 32; e += 4) *reinterpret_cast<uint4*>(dst + e) = 
                  make_uint4(scaled(ov[e]), scaled(ov[e + 1]), scaled(ov[e + 2]), scaled(ov[e + 3]));
          }
        }
        tc_fence_before();
        mbar_arrive(cb + O_FREE + 8 * w);
        if (mine) k.part_ml[pr] = make_float2((m == -INFINITY ? 0.f : m) - UP, l);
      } else {
        uint8_t* dst = k.o + 2 * (mine ? out_row(done, t) : 0);
#pragma unroll 1
        for (int c = 0; c < D; c += 32) {
          uint32_t ov[32], h[16];
          tmem_ld32(o_tmem + c, ov);
          tc_wait_ld32(ov);
#pragma unroll
          for (int e = 0; e < 16; ++e) h[e] = pack_bf16(__uint_as_float(ov[2 * e]) * inv, __uint_as_float(ov[2 * e + 1]) * inv);
          if (mine) {
            uint4* d4 = reinterpret_cast<uint4*>(dst + 2 * c);
#pragma unroll
            for (int e = 0; e < 16; e += 8) {
              const uint4 lo = make_uint4(h[e], h[e + 1], h[e + 2], h[e + 3]), hi = make_uint4(h[e + 4], h[e + 5], h[e + 6], h[e + 7]);
              if (prm.wide) {
                stg32(d4 + e / 4, lo, hi);
              } else {
                d4[e / 4] = lo;
                d4[e / 4 + 1] = hi;
              }
            }
          }
        }
        tc_fence_before();
        mbar_arrive(cb + O_FREE + 8 * w);
        if (mine && k.lse) *lse_at(done, t) = l != 0.f ? ((m == -INFINITY ? 0.f : m) - UP + log2f(l)) * 0.6931471805599453f : -INFINITY;
      }
    }
  }

  // ---------------------------------------------------------------- tear-down
  if (*abort_flag) {
    // copies and MMAs still in flight land before shared memory and TMEM go away
    const long long t0 = clock64();
    while (clock64() - t0 < 2000000) {}
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 0) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
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
// 4-D map of bf16, 64 channels (128 bytes, swizzled) x box of the next two dimensions; sizes and element strides of dimensions 1 to 3
static int keys_map(CUtensorMap* map, const void* ptr, int d, const long long n[3], const long long s[3], int box1, int box2) {
  const keys_encode_t enc = keys_encode();
  if (!enc) return SVA_ERR_CUDA;
  const cuuint64_t dims[4] = {(cuuint64_t)d, (cuuint64_t)n[0], (cuuint64_t)n[1], (cuuint64_t)n[2]};
  cuuint64_t strides[3];
  for (int i = 0; i < 3; ++i) strides[i] = n[i] > 1 ? 2 * (cuuint64_t)s[i] : 2 * (cuuint64_t)d;      // (a dimension of one may carry any)
  const cuuint32_t box[4] = {64, (cuuint32_t)box1, (cuuint32_t)box2, 1}, each[4] = {1, 1, 1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(ptr), dims, strides, box, each, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS ? SVA_OK : SVA_ERR_CUDA;
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
  const unsigned grid = prm.items < (unsigned)sms ? prm.items : (unsigned)sms;
  return launch_dep(kern, dim3(grid), kt::THREADS, kt::Smem<D>::BYTES, st, tq, tk, tv, prm);
}

int launch_keys_tc(const KeysParams& k, bool paged, int sms, cudaStream_t st) {
  KeysTcParams prm = {};
  prm.k = k;
  prm.tokens = 128 / k.group;
  prm.pairs = (k.tiles + 1) / 2;
  const long long items = (long long)k.B * k.Hk * prm.pairs * k.splits;
  if (items > 0x7fffffffLL) return SVA_ERR_UNSUPPORTED;
  prm.items = (uint32_t)items;
  prm.wide = (reinterpret_cast<uintptr_t>(k.o) & 31u) == 0 && ((k.so.b | k.so.h | k.so.n) & 15) == 0;
  prm.debug = g_debug_keys;
  CUtensorMap tq = {}, tk = {}, tv = {};
  if (!paged) {
    // (row tiles: the group's heads of each token side by side)
    const long long qn[3] = {k.Hq, k.M, k.B}, qs[3] = {k.sq.h, k.sq.n, k.sq.b};
    int rc = keys_map(&tq, k.q, k.d, qn, qs, k.group, prm.tokens);
    const int hk = k.sk.h == 0 ? 1 : k.Hk, bk = k.sk.b == 0 ? 1 : k.B, hv = k.sv.h == 0 ? 1 : k.Hk, bv = k.sv.b == 0 ? 1 : k.B;
    prm.k_each_h = hk > 1; prm.k_each_b = bk > 1; prm.v_each_h = hv > 1; prm.v_each_b = bv > 1;
    const long long kn[3] = {k.S, hk, bk}, ks[3] = {k.sk.n, k.sk.h, k.sk.b}, vn[3] = {k.S, hv, bv}, vs[3] = {k.sv.n, k.sv.h, k.sv.b};
    if (!rc) rc = keys_map(&tk, k.k, k.d, kn, ks, kt::KT, 1);
    if (!rc) rc = keys_map(&tv, k.v, k.d, vn, vs, kt::KT, 1);
    if (rc) return rc;
  }
  if (paged) return k.d == 128 ? launch_tc<128, true>(prm, tq, tk, tv, sms, st) : launch_tc<64, true>(prm, tq, tk, tv, sms, st);
  return k.d == 128 ? launch_tc<128, false>(prm, tq, tk, tv, sms, st) : launch_tc<64, false>(prm, tq, tk, tv, sms, st);
}

}  // namespace sva
