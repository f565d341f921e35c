// Attention of few rows over many keys (sva_cached_attn_fwd, sva_cross_attn_fwd): one token or a few per sequence.
//
// Bound by the keys' bytes: every key is read once per tile of 16 rows (cached keys: 8), straight into the registers of the warp that uses it, and enters
// mma.sync products (m16n8k16).  A row of a tile is a token times one of the heads that share the keys.  A warp takes 16 keys at a time, in turn with
// the others of its CTA.  In which order the products run over channels is free, so each thread takes whole 16-byte pieces of a row and the
// operand fragments are cut from them.  The warps' sums meet in shared memory; ranges of a long axis (splits) meet in a second kernel.
//
// e4m3 codes are converted to fp16, exactly; Q is scaled by a power of two per row into fp16's range, P = 2^(s + log2 v_scale - m + P_UP) with a
// reference m of what is in the exponent: weights whose products with codes of any pages add up as they are; the row sum takes 1 / v_scale per group.
#include <cuda_fp16.h>

#include "attn_keys.cuh"
#include "tc_ptx.cuh"

namespace sva {

static constexpr int FEW_ROWS = 16, FEW_KEYS = 16, FEW_WARPS = 8, FEW_THREADS = FEW_WARPS * 32;
static constexpr int PAGED_ROWS = 8, PAGED_WARPS = 4, PAGED_CTAS = 3;      // (CTAs per SM)
// fp16 probabilities: log2 of one at the reference, and how far above it they may go
static constexpr float P_UP = 10.0f, FEW_LAZY = 4.0f;

__device__ __forceinline__ void mma_f16(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// four e4m3 codes -> two pairs of fp16 values
__device__ __forceinline__ void codes_f16x4(uint32_t codes, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=r"(lo), "=r"(hi) : "r"(codes));
}
// an 8 x 8 matrix of 16-bit values that lies over a warp as MMA fragments do, transposed
__device__ __forceinline__ uint32_t turn8x8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// ---- cached keys: up to eight rows per tile
// The products are taken the other way round, keys (S^T = K Q^T) and channels (O^T = V^T P^T) as the MMA's 16 rows and the queries as its 8 columns: half
// the MMAs, accumulators and Q of 16 rows, so that twelve warps with the next group's codes in flight share an SM.  P is turned by movmatrix on its way.
// The reference m follows the maximum lazily: only when a weight is more than FEW_LAZY powers of two above it is the group's maximum taken.
// Eight sequences of up to 131 071 tokens (unequal ones), 8 key heads of 128, four query heads each, a pass among others: 376 to 397 us = 4.2 TB/s; the same
// call by itself over and over, when it was built, 320, and with 16 rows per tile, eight warps per SM and the maximum in every group 653.  What is left is latency: a group is on its way for as long as the group before it is worked on.
template <int D>
__global__ void __launch_bounds__(PAGED_WARPS * 32, PAGED_CTAS)
keys_paged_few_kernel(const KeysParams prm) {
  constexpr int KSTEPS = D / 16, MT = D / 16;
  constexpr int KP = D / 64, VB = D / 8;                                  // 16-byte pieces of a key row per thread; bytes of a value row
  extern __shared__ float smem_f[];                                       // [warps][8][D] then [warps][8] x 2
  const int zero = grid_dep_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  report_long(prm, zero);
  uint32_t at = blockIdx.x + (uint32_t)zero;
  const int tile = (int)(at % (uint32_t)prm.tiles); at /= (uint32_t)prm.tiles;
  const int split = (int)(at % (uint32_t)prm.splits); at /= (uint32_t)prm.splits;
  const int hk = (int)(at % (uint32_t)prm.Hk), b = (int)(at / (uint32_t)prm.Hk);
  const int keys = seq_keys(prm, b), queries = seq_queries(prm, b);
  const int row_first = tile * PAGED_ROWS, rows = queries * prm.group;
  if (row_first >= rows) return;
  const int end = keys_seen(prm, keys, queries, (min(row_first + PAGED_ROWS, rows) - 1) / prm.group);
  const int groups = (end + FEW_KEYS - 1) / FEW_KEYS;
  const int g_lo = (int)((long long)groups * split / prm.splits), g_hi = (int)((long long)groups * (split + 1) / prm.splits);

  struct Group { uint4 k[2][KP], v[4]; float ks, vs; uint32_t there; };
  const int per_page = prm.page / FEW_KEYS;
  const int32_t* table = prm.table + b * prm.table_stride;
  // page id of a group; -1: named wrongly
  auto page_of = [&](int gi, int& in_page) -> int {
    if (gi >= g_hi) return 0;
    const int e = gi / per_page;
    in_page = gi - e * per_page;
    const int id = e < prm.max_pages ? __ldg(table + e) : -1;
    return id >= prm.pages ? -1 : id;
  };
  auto load = [&](int gi, int id, int in_page, Group& x) {
    x.there = 0u;
    if (gi >= g_hi) return;
    if (id < 0) {
      if (lane == 0 && prm.status) atomicOr(prm.status, SVA_DEV_BAD_INDEX);
      return;
    }
    const int left = keys - gi * FEW_KEYS;
    x.there = left >= FEW_KEYS ? 0xffffu : (1u << left) - 1u;
    const long long head = (long long)id * prm.Hk + hk, row = head * prm.page + in_page * FEW_KEYS;
    const uint8_t *kp = prm.k + row * D, *vp = prm.v + row * D;
    x.ks = __ldg(prm.k_scale + head);
    x.vs = __ldg(prm.v_scale + head);
    // keys g and g + 8; values of keys 2c, 2c + 1, 2c + 8, 2c + 9.  Rows that are not there are not read: zeros, whatever they hold
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int e = 0; e < KP; ++e)
        x.k[n][e] = x.there >> (g + 8 * n) & 1u ? __ldg(reinterpret_cast<const uint4*>(kp + (g + 8 * n) * D + (e * 4 + c) * 16))
                                                : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const int key = 2 * c + (n & 1) + 8 * (n >> 1);
      x.v[n] = make_uint4(0u, 0u, 0u, 0u);
      if (x.there >> key & 1u) {
        if (VB >= 16) {
          x.v[n] = __ldg(reinterpret_cast<const uint4*>(vp + key * D + g * 16));
        } else {
          const uint2 u = __ldg(reinterpret_cast<const uint2*>(vp + key * D + g * 8));
          x.v[n].x = u.x; x.v[n].y = u.y;
        }
      }
    }
  };
  auto word = [](const uint4& u, int i) -> uint32_t { return i == 0 ? u.x : i == 1 ? u.y : i == 2 ? u.z : u.w; };

  Group x, y;
  int gi = g_lo + warp, in_page = 0;
  {
    const int id = page_of(gi, in_page);
    load(gi, id, in_page, x);
  }
  int id = page_of(gi + PAGED_WARPS, in_page);

  // Q: B fragments of row g.  Channels of step s, thread c: piece (s / 4) * 4 + c of 16, from (s % 4) * 4 on.  Each row times a power of two
  uint32_t qb[KSTEPS][2];
  float mine_scale = prm.scale_log2;
  {
    const int r = min(row_first + g, rows - 1), t = r / prm.group, h = hk * prm.group + r % prm.group;
    const uint8_t* q = prm.q + 2 * (b * prm.sq.b + h * prm.sq.h + (long long)t * prm.sq.n);
    uint32_t top = 0u;
#pragma unroll
    for (int s = 0; s < KSTEPS; ++s) {
      const uint2 u = __ldg(reinterpret_cast<const uint2*>(q + 2 * (((s / 4) * 4 + c) * 16 + (s % 4) * 4)));
      qb[s][0] = u.x;
      qb[s][1] = u.y;
      top = max(max(top, max(u.x & 0x7fffu, u.x >> 16 & 0x7fffu)), max(u.y & 0x7fffu, u.y >> 16 & 0x7fffu));
    }
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const uint32_t ex = top >> 7;
    const bool odd = ex == 0u || ex > 252u;                               // (zeros; infinities, NaNs)
    const float down = odd ? 1.f : __uint_as_float((254u - ex) << 23);
    mine_scale *= odd ? 1.f : __uint_as_float(ex << 23);
#pragma unroll
    for (int s = 0; s < KSTEPS; ++s)
#pragma unroll
      for (int e = 0; e < 2; ++e) qb[s][e] = pack_f16(bf16lo(qb[s][e]) * down, bf16hi(qb[s][e]) * down);
  }
  // my columns of S^T and O^T are rows 2c and 2c + 1: logits' scale, what they see
  float cc[2], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
  int seen[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    cc[i] = __shfl_sync(0xffffffffu, mine_scale, (2 * c + i) * 4);
    seen[i] = keys_seen(prm, keys, queries, min(row_first + 2 * c + i, rows - 1) / prm.group);
  }
  const int seen_least = keys_seen(prm, keys, queries, row_first / prm.group);
  float acc[MT][4];
#pragma unroll
  for (int t = 0; t < MT; ++t) acc[t][0] = acc[t][1] = acc[t][2] = acc[t][3] = 0.f;

  auto step = [&](int gi, Group& x) {
    if (x.there == 0u) return;                                            // (a page that is named wrongly: nothing was read)
    float s[4] = {0.f, 0.f, 0.f, 0.f};                                    // (key g, rows 2c, 2c + 1), (key g + 8, the same)
#pragma unroll
    for (int i = 0; i < KSTEPS; ++i) {
      uint32_t a[4];
      codes_f16x4(word(x.k[0][i / 4], i % 4), a[0], a[2]);
      codes_f16x4(word(x.k[1][i / 4], i % 4), a[1], a[3]);
      mma_f16(s, a, qb[i][0], qb[i][1]);
    }
    // a page with a scale that is a NaN or infinite: logits of NaN for the rows that see it, values of zeros, which spoil no other row
    if (!(fabsf(x.ks) < INFINITY && fabsf(x.vs) < INFINITY)) {            // (uniform in a warp)
      s[0] = s[1] = s[2] = s[3] = __int_as_float(0x7fc00000);
      x.ks = x.vs = 1.f;
#pragma unroll
      for (int n = 0; n < 4; ++n) x.v[n] = make_uint4(0u, 0u, 0u, 0u);
    }
    const float vs = v_scale_floor(x.vs), lv = __log2f(vs), inv_vs = __frcp_rn(vs);
    float p[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) p[e] = fmaf(s[e], cc[e & 1] * x.ks, lv);
    if (x.there != 0xffffu || (gi + 1) * FEW_KEYS > seen_least) {         // (uniform in a warp)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int key = g + 8 * (e >> 1);
        if (!(x.there >> key & 1u) || gi * FEW_KEYS + key >= seen[e & 1]) p[e] = -INFINITY;
      }
    }
    const float t0 = fmaxf(p[0], p[2]), t1 = fmaxf(p[1], p[3]);
    if (__any_sync(0xffffffffu, t0 > m[0] + FEW_LAZY || t1 > m[1] + FEW_LAZY)) {
      float top[2] = {t0, t1};
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], o));
        if (top[i] > m[i]) {
          const float down = ex2(m[i] - top[i]);                          // (0 where m was -inf)
          m[i] = top[i];
          l[i] *= down;
#pragma unroll
          for (int t = 0; t < MT; ++t) {
            acc[t][i] *= down;
            acc[t][i + 2] *= down;
          }
        }
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) p[e] = ex2(p[e] - ((m[e & 1] == -INFINITY ? 0.f : m[e & 1]) - P_UP));
    l[0] = fmaf(p[0] + p[2], inv_vs, l[0]);
    l[1] = fmaf(p[1] + p[3], inv_vs, l[1]);
    const uint32_t b0 = turn8x8(pack_f16(p[0], p[1])), b1 = turn8x8(pack_f16(p[2], p[3]));
#pragma unroll
    for (int t = 0; t < MT; t += 2) {                                     // four channels of each of the four rows: two tiles' rows g and g + 8
      const uint32_t w0 = word(x.v[0], t / 2), w1 = word(x.v[1], t / 2), w2 = word(x.v[2], t / 2), w3 = word(x.v[3], t / 2);
      uint32_t a[4], d[4];
      codes_f16x4(__byte_perm(w0, w1, 0x5140), a[0], a[1]);
      codes_f16x4(__byte_perm(w2, w3, 0x5140), a[2], a[3]);
      codes_f16x4(__byte_perm(w0, w1, 0x7362), d[0], d[1]);
      codes_f16x4(__byte_perm(w2, w3, 0x7362), d[2], d[3]);
      mma_f16(acc[t], a, b0, b1);
      mma_f16(acc[t + 1], d, b0, b1);
    }
  };
  // the group after this one is on its way while this one is used, and the page of the one after that is looked up
  while (gi < g_hi) {
    load(gi + PAGED_WARPS, id, in_page, y);
    id = page_of(gi + 2 * PAGED_WARPS, in_page);
    step(gi, x);
    gi += PAGED_WARPS;
    if (gi >= g_hi) break;
    load(gi + PAGED_WARPS, id, in_page, x);
    id = page_of(gi + 2 * PAGED_WARPS, in_page);
    step(gi, y);
    gi += PAGED_WARPS;
  }

  // ---- the warps' sums.  Of tile t, row g is channel g * D/8 + 2 t, row g + 8 the next
  float* so = smem_f + warp * PAGED_ROWS * D;
  float* sm = smem_f + PAGED_WARPS * PAGED_ROWS * D;                        // m [warps][8], l [warps][8]
#pragma unroll
  for (int i = 0; i < 2; ++i) {
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], o);
    if (g == 0) {
      sm[warp * PAGED_ROWS + 2 * c + i] = m[i] == -INFINITY ? 0.f : m[i];
      sm[(PAGED_WARPS + warp) * PAGED_ROWS + 2 * c + i] = l[i];
    }
#pragma unroll
    for (int t = 0; t < MT; t += 2)
      *reinterpret_cast<float4*>(so + (2 * c + i) * D + g * (D / 8) + 2 * t) = make_float4(acc[t][i], acc[t][i + 2], acc[t + 1][i], acc[t + 1][i + 2]);
  }
  __syncthreads();
  constexpr int EACH = PAGED_ROWS * D / (PAGED_WARPS * 32);                      // channels per thread: 4 or 2
  const int row = threadIdx.x / (D / EACH), ch = threadIdx.x % (D / EACH) * EACH;
  float top = -INFINITY, total = 0.f, out[EACH];
#pragma unroll
  for (int w = 0; w < PAGED_WARPS; ++w)
    if (sm[(PAGED_WARPS + w) * PAGED_ROWS + row] != 0.f) top = fmaxf(top, sm[w * PAGED_ROWS + row]);
#pragma unroll
  for (int e = 0; e < EACH; ++e) out[e] = 0.f;
#pragma unroll
  for (int w = 0; w < PAGED_WARPS; ++w) {
    const float lw = sm[(PAGED_WARPS + w) * PAGED_ROWS + row];
    if (lw != 0.f) {
      const float f = ex2(sm[w * PAGED_ROWS + row] - top);
      total = fmaf(lw, f, total);
#pragma unroll
      for (int e = 0; e < EACH; ++e) out[e] = fmaf(smem_f[(w * PAGED_ROWS + row) * D + ch + e], f, out[e]);
    }
  }
  if (prm.splits > 1) {
    const long long unit = ((long long)b * prm.Hk + hk) * prm.tiles + tile, all = (long long)prm.B * prm.Hk * prm.tiles * PAGED_ROWS;
    const long long mine = split * all + unit * PAGED_ROWS + row;
#pragma unroll
    for (int e = 0; e < EACH; e += 2) *reinterpret_cast<float2*>(prm.part_o + mine * D + ch + e) = make_float2(out[e], out[e + 1]);
    if (ch == 0) prm.part_ml[mine] = make_float2(top, total);
    return;
  }
  const int r = row_first + row;
  if (r >= rows) return;
  const int t = r / prm.group, h = hk * prm.group + r % prm.group;
  const float inv = total != 0.f ? 1.f / total : 0.f;
  uint32_t* dst = reinterpret_cast<uint32_t*>(prm.o + 2 * (b * prm.so.b + h * prm.so.h + (long long)t * prm.so.n + ch));
#pragma unroll
  for (int e = 0; e < EACH; e += 2) dst[e / 2] = pack_bf16(out[e] * inv, out[e + 1] * inv);
  if (ch == 0 && prm.lse) prm.lse[((long long)b * prm.Hq + h) * prm.M + t] = total != 0.f ? (top - P_UP + log2f(total)) * 0.6931471805599453f : -INFINITY;
}

// ---- bf16 keys: sixteen rows per tile; P needs no shuffle, being A of the second product as it leaves the first.  It enters as two bf16 terms (MMA operands
// have one type, V's), so that 16 of its bits count: the kernel waits for its loads, and the second product is hidden behind them
template <int D>
__global__ void __launch_bounds__(FEW_THREADS, 1)
keys_few_kernel(const KeysParams prm) {
  constexpr int KSTEPS = D / 16, NT = D / 8;
  // 16-byte pieces of a row that a thread holds: of a key (4 threads per row), of a value row (8 threads per row)
  constexpr int KP = D / 32, VP = D / 64;
  extern __shared__ float smem_f[];                                       // [warps][16][D] then [warps][16] x 2
  const int zero = grid_dep_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  long long at = (long long)blockIdx.x + zero;
  const int tile = (int)(at % prm.tiles); at /= prm.tiles;
  const int split = (int)(at % prm.splits); at /= prm.splits;
  const int hk = (int)(at % prm.Hk), b = (int)(at / prm.Hk);
  const int keys = seq_keys(prm, b), queries = seq_queries(prm, b);
  const long long row_first = (long long)tile * FEW_ROWS, rows = (long long)queries * prm.group;
  if (row_first >= rows) return;
  const int last_t = (int)(min(row_first + FEW_ROWS, rows) - 1) / prm.group;
  const int end = keys_seen(prm, keys, queries, last_t);
  const int groups = (end + FEW_KEYS - 1) / FEW_KEYS;
  const int g_lo = (int)((long long)groups * split / prm.splits), g_hi = (int)((long long)groups * (split + 1) / prm.splits);

  // my two rows (g, g + 8): where their queries are, what they see
  const uint8_t* qrow[2];
  int seen[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const long long r = min(row_first + g + 8 * i, rows - 1);
    const int t = (int)(r / prm.group), h = hk * prm.group + (int)(r % prm.group);
    qrow[i] = prm.q + 2 * (b * prm.sq.b + h * prm.sq.h + (long long)t * prm.sq.n);
    seen[i] = keys_seen(prm, keys, queries, t);
  }
  // Q: A fragments.  Channels of step s, thread c: piece (s / 2) * 4 + c of 8, from (s % 2) * 4 on
  uint32_t qa[KSTEPS][4];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int s = 0; s < KSTEPS; ++s) {
      const uint2 u = __ldg(reinterpret_cast<const uint2*>(qrow[i] + 2 * (((s / 2) * 4 + c) * 8 + (s % 2) * 4)));
      qa[s][i] = u.x;
      qa[s][2 + i] = u.y;
    }

  float acc[NT][4], more[NT][4];                                          // (more: of P's second term)
#pragma unroll
  for (int t = 0; t < NT; ++t) acc[t][0] = acc[t][1] = acc[t][2] = acc[t][3] = more[t][0] = more[t][1] = more[t][2] = more[t][3] = 0.f;
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};

  struct Group { uint4 k[2][KP], v[4][VP]; uint32_t there; };
  auto load = [&](int gi, Group& x) {
    const int key0 = gi * FEW_KEYS;
    x.there = keys - key0 >= FEW_KEYS ? 0xffffu : (1u << (keys - key0)) - 1u;
    const uint8_t *kp = prm.k + 2 * (b * prm.sk.b + hk * prm.sk.h + (long long)key0 * prm.sk.n),
                  *vp = prm.v + 2 * (b * prm.sv.b + hk * prm.sv.h + (long long)key0 * prm.sv.n);
    const long long ks_row = 2 * prm.sk.n, vs_row = 2 * prm.sv.n;
    if (prm.mask) {
      const bool on = lane < FEW_KEYS && (x.there >> lane & 1u) && __ldg(prm.mask + b * prm.mask_stride + key0 + lane) != 0;
      x.there = __ballot_sync(0xffffffffu, on);
    }
    // keys g and g + 8; values of keys 2c, 2c + 1, 2c + 8, 2c + 9.  Rows that are not there are not read: zeros, whatever they hold
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int e = 0; e < KP; ++e)
        x.k[n][e] = x.there >> (g + 8 * n) & 1u ? __ldg(reinterpret_cast<const uint4*>(kp + (g + 8 * n) * ks_row + (e * 4 + c) * 16))
                                                : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const int key = 2 * c + (n & 1) + 8 * (n >> 1);
      const bool on = x.there >> key & 1u;
#pragma unroll
      for (int e = 0; e < VP; ++e)
        x.v[n][e] = on ? __ldg(reinterpret_cast<const uint4*>(vp + key * vs_row + (e * 8 + g) * 16)) : make_uint4(0u, 0u, 0u, 0u);
    }
  };
  auto word = [](const uint4& u, int i) -> uint32_t { return i == 0 ? u.x : i == 1 ? u.y : i == 2 ? u.z : u.w; };

  auto step = [&](int gi, const Group& x) {
    float s[2][4];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
#pragma unroll
      for (int i = 0; i < KSTEPS; ++i) {
        mma_bf16(s[n], qa[i], word(x.k[n][i / 2], 2 * (i % 2)), word(x.k[n][i / 2], 2 * (i % 2) + 1));
      }
    }
    const int key0 = gi * FEW_KEYS;
    uint32_t p[2][2], rest[2][2];                                         // [n tile][row]
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float y[4], top = -INFINITY;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int key = (e >> 1) * 8 + 2 * c + (e & 1);
        y[e] = s[e >> 1][2 * i + (e & 1)] * prm.scale_log2;
        if (!(x.there >> key & 1u) || key0 + key >= seen[i]) y[e] = -INFINITY;
        top = fmaxf(top, y[e]);
      }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      if (top > m[i]) {                                                   // (all four threads of the row)
        const float down = ex2(m[i] - top);                               // (0 where m was -inf)
        m[i] = top;
        l[i] *= down;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          acc[t][2 * i] *= down;
          acc[t][2 * i + 1] *= down;
          more[t][2 * i] *= down;
          more[t][2 * i + 1] *= down;
        }
      }
      const float ref = m[i] == -INFINITY ? 0.f : m[i];
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        y[e] = ex2(y[e] - ref);
        sum += y[e];
      }
      l[i] += sum;
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        p[n][i] = pack_bf16(y[2 * n], y[2 * n + 1]);
        rest[n][i] = pack_bf16(y[2 * n] - bf16lo(p[n][i]), y[2 * n + 1] - bf16hi(p[n][i]));
      }
    }
    const uint32_t pa[4] = {p[0][0], p[0][1], p[1][0], p[1][1]}, pr[4] = {rest[0][0], rest[0][1], rest[1][0], rest[1][1]};
#pragma unroll
    for (int t = 0; t < NT; t += 4) {                                     // four channels of each of the four rows
#pragma unroll
      for (int e = 0; e < 2; ++e) {                                       // two words of two channels
        const int piece = t / 8, i = (t / 4 % 2) * 2 + e;
        const uint32_t w0 = word(x.v[0][piece], i), w1 = word(x.v[1][piece], i), w2 = word(x.v[2][piece], i), w3 = word(x.v[3][piece], i);
        const uint32_t lo01 = __byte_perm(w0, w1, 0x5410), lo23 = __byte_perm(w2, w3, 0x5410), hi01 = __byte_perm(w0, w1, 0x7632),
                       hi23 = __byte_perm(w2, w3, 0x7632);
        mma_bf16(acc[t + 2 * e], pa, lo01, lo23);
        mma_bf16(acc[t + 2 * e + 1], pa, hi01, hi23);
        mma_bf16(more[t + 2 * e], pr, lo01, lo23);
        mma_bf16(more[t + 2 * e + 1], pr, hi01, hi23);
      }
    }
  };

  for (int gi = g_lo + warp; gi < g_hi; gi += FEW_WARPS) {
    Group x;
    load(gi, x);
    step(gi, x);
  }

  // (the second term's products with an infinite value may have the other sign, or none: the first term's stand for those)
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[t][e] += fabsf(more[t][e]) < INFINITY ? more[t][e] : 0.f;

  // ---- the warps' sums: each thread's columns n = 2c, 2c + 1 of tile t are channels of its own order
  float* so = smem_f + warp * FEW_ROWS * D;
  float* sm = smem_f + FEW_WARPS * FEW_ROWS * D;                          // m [warps][16], l [warps][16]
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
    l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
    if (c == 0) {
      sm[warp * FEW_ROWS + g + 8 * i] = m[i] == -INFINITY ? 0.f : m[i];
      sm[(FEW_WARPS + warp) * FEW_ROWS + g + 8 * i] = l[i];
    }
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const int col = 2 * c + n;
#pragma unroll
      for (int t = 0; t < NT; t += 4) {
        const int ch = (t / 8) * 64 + col * 8 + t % 8;
        *reinterpret_cast<float4*>(so + (g + 8 * i) * D + ch) =
            make_float4(acc[t][2 * i + n], acc[t + 1][2 * i + n], acc[t + 2][2 * i + n], acc[t + 3][2 * i + n]);
      }
    }
  }
  __syncthreads();
  constexpr int EACH = FEW_ROWS * D / FEW_THREADS;                        // channels per thread: 8 or 4
  const int row = threadIdx.x / (D / EACH), ch = threadIdx.x % (D / EACH) * EACH;
  float top = -INFINITY, total = 0.f, out[EACH];
#pragma unroll
  for (int w = 0; w < FEW_WARPS; ++w)
    if (sm[(FEW_WARPS + w) * FEW_ROWS + row] != 0.f) top = fmaxf(top, sm[w * FEW_ROWS + row]);
#pragma unroll
  for (int e = 0; e < EACH; ++e) out[e] = 0.f;
#pragma unroll
  for (int w = 0; w < FEW_WARPS; ++w) {
    const float lw = sm[(FEW_WARPS + w) * FEW_ROWS + row];
    if (lw != 0.f) {
      const float f = ex2(sm[w * FEW_ROWS + row] - top);
      total = fmaf(lw, f, total);
#pragma unroll
      for (int e = 0; e < EACH; ++e) out[e] = fmaf(smem_f[(w * FEW_ROWS + row) * D + ch + e], f, out[e]);
    }
  }
  if (prm.splits > 1) {
    const long long unit = ((long long)b * prm.Hk + hk) * prm.tiles + tile, all = (long long)prm.B * prm.Hk * prm.tiles * FEW_ROWS;
    const long long mine = split * all + unit * FEW_ROWS + row;
#pragma unroll
    for (int e = 0; e < EACH; e += 4) *reinterpret_cast<float4*>(prm.part_o + mine * D + ch + e) = make_float4(out[e], out[e + 1], out[e + 2], out[e + 3]);
    if (ch == 0) prm.part_ml[mine] = make_float2(top, total);
    return;
  }
  const long long r = row_first + row;
  if (r >= rows) return;
  const int t = (int)(r / prm.group), h = hk * prm.group + (int)(r % prm.group);
  const float inv = total != 0.f ? 1.f / total : 0.f;
  uint32_t w[EACH / 2];
#pragma unroll
  for (int e = 0; e < EACH; e += 2) w[e / 2] = pack_bf16(out[e] * inv, out[e + 1] * inv);
  uint8_t* dst = prm.o + 2 * (b * prm.so.b + h * prm.so.h + (long long)t * prm.so.n + ch);
  if (EACH == 8) *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[EACH / 2 - 2], w[EACH / 2 - 1]);
  else *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
  if (ch == 0 && prm.lse)
    prm.lse[((long long)b * prm.Hq + h) * prm.M + t] = total != 0.f ? (top + log2f(total)) * 0.6931471805599453f : -INFINITY;
}

// The splits' sums of a row: [splits][rows of all][D].  WARPS warps take the splits in turn: one where there are up to
// eight of them, the four of a CTA for more (rows are then few, and the loads' latency is what they wait for).  Tiles have rows_per rows, of
// which those of `tokens` tokens are used (the kernels for few rows: all, tokens that go over a tile's end among them, tokens 0); up: what
// the references lie below the exponents.
static constexpr int JOIN_THREADS = 128;
template <int D, int WARPS>
__global__ void __launch_bounds__(JOIN_THREADS)
keys_join_kernel(const KeysParams prm, int rows_per, int tokens, float up) {
  constexpr int EACH = D / 32;
  __shared__ float sums[WARPS][D], tops[WARPS], totals[WARPS];
  static_assert(WARPS == 1 || WARPS == JOIN_THREADS / 32, "a row's warps meet at the CTA's barrier");
  const int zero = grid_dep_wait();
  const int warp = (threadIdx.x >> 5) % WARPS, lane = threadIdx.x & 31;
  const long long per_head = (long long)prm.tiles * rows_per, all = (long long)prm.B * prm.Hk * per_head;
  const long long mine = (long long)blockIdx.x * (JOIN_THREADS / 32 / WARPS) + (threadIdx.x >> 5) / WARPS + zero, unit = mine / per_head;
  if (mine >= all) return;
  long long r = mine % per_head;
  const int hk = (int)(unit % prm.Hk), b = (int)(unit / prm.Hk);
  if (tokens) {
    const int in_tile = (int)(r % rows_per);
    if (in_tile >= tokens * prm.group) return;
    r = r / rows_per * tokens * prm.group + in_tile;
  }
  if (r >= (long long)seq_queries(prm, b) * prm.group) return;
  float top = -INFINITY, total = 0.f, out[EACH];
#pragma unroll
  for (int e = 0; e < EACH; ++e) out[e] = 0.f;
  // 32 of the warp's splits at a time: each lane has the reference and the row sum of one, so that the loop's loads wait for nothing
#pragma unroll 1
  for (int base = warp; base < prm.splits; base += 32 * WARPS) {
    const int s = base + lane * WARPS;
    const float2 ml = s < prm.splits ? prm.part_ml[s * all + mine] : make_float2(0.f, 0.f);
    float now = ml.y != 0.f ? ml.x : -INFINITY;
#pragma unroll
    for (int o = 16; o; o >>= 1) now = fmaxf(now, __shfl_xor_sync(0xffffffffu, now, o));
    now = fmaxf(now, top);
    if (now == -INFINITY) continue;                                       // (nothing but empty splits so far)
    const float old = ex2(top - now), factor = ml.y != 0.f ? ex2(ml.x - now) : 0.f;
    float part = ml.y != 0.f ? ml.y * factor : 0.f;
#pragma unroll
    for (int o = 16; o; o >>= 1) part += __shfl_xor_sync(0xffffffffu, part, o);
    top = now;
    total = fmaf(total, old, part);
#pragma unroll
    for (int e = 0; e < EACH; ++e) out[e] *= old;
    const uint32_t there = __ballot_sync(0xffffffffu, ml.y != 0.f);      // (of an empty split nothing is written)
    const float* x = prm.part_o + (base * all + mine) * D + lane * EACH;
    const int n = min(32, (prm.splits - base + WARPS - 1) / WARPS);
#pragma unroll 8
    for (int i = 0; i < n; ++i) {
      const float f = __shfl_sync(0xffffffffu, factor, i);
#pragma unroll
      for (int e = 0; e < EACH; e += 2) {
        const float2 u = there >> i & 1u ? *reinterpret_cast<const float2*>(x + (long long)i * WARPS * all * D + e) : make_float2(0.f, 0.f);
        out[e] = fmaf(u.x, f, out[e]);
        out[e + 1] = fmaf(u.y, f, out[e + 1]);
      }
    }
  }
  if (WARPS > 1) {
#pragma unroll
    for (int e = 0; e < EACH; ++e) sums[warp][lane * EACH + e] = out[e];
    if (lane == 0) {
      tops[warp] = top;
      totals[warp] = total;
    }
    __syncthreads();
    if (warp != 0) return;
  }
#pragma unroll
  for (int w = 1; w < WARPS; ++w)
    if (totals[w] != 0.f) {
      const float now = fmaxf(top, tops[w]), f = ex2(tops[w] - now), old = ex2(top - now);
      top = now;
      total = fmaf(total, old, totals[w] * f);
#pragma unroll
      for (int e = 0; e < EACH; ++e) out[e] = fmaf(out[e], old, sums[w][lane * EACH + e] * f);
    }
  const int t = (int)(r / prm.group), h = hk * prm.group + (int)(r % prm.group);
  const float inv = total != 0.f ? 1.f / total : 0.f;
  uint32_t* dst = reinterpret_cast<uint32_t*>(prm.o + 2 * (b * prm.so.b + h * prm.so.h + (long long)t * prm.so.n + lane * EACH));
#pragma unroll
  for (int e = 0; e < EACH; e += 2) dst[e / 2] = pack_bf16(out[e] * inv, out[e + 1] * inv);
  if (lane == 0 && prm.lse) prm.lse[((long long)b * prm.Hq + h) * prm.M + t] = total != 0.f ? (top - up + log2f(total)) * 0.6931471805599453f : -INFINITY;
}

template <int D>
static int launch_join(const KeysParams& prm, int rows_per, int tokens, float up, cudaStream_t st) {
  const long long rows = (long long)prm.B * prm.Hk * prm.tiles * rows_per;
  if (prm.splits <= 8) return launch_dep(keys_join_kernel<D, 1>, dim3((unsigned)((rows + 3) / 4)), JOIN_THREADS, 0, st, prm, rows_per, tokens, up);
  return launch_dep(keys_join_kernel<D, 4>, dim3((unsigned)rows), JOIN_THREADS, 0, st, prm, rows_per, tokens, up);
}

template <int D, bool PAGED>
static int launch_few(const KeysParams& prm, cudaStream_t st) {
  static DeviceOnce once;
  constexpr int ROWS = PAGED ? PAGED_ROWS : FEW_ROWS, WARPS = PAGED ? PAGED_WARPS : FEW_WARPS, SMEM = WARPS * ROWS * (D + 2) * 4;
  auto kern = PAGED ? keys_paged_few_kernel<D> : keys_few_kernel<D>;
  int rc = once.run([&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM) == cudaSuccess; });
  if (rc) return rc;
  const long long ctas = (long long)prm.B * prm.Hk * prm.tiles * prm.splits;
  if (ctas > 0x7fffffffLL) return SVA_ERR_UNSUPPORTED;
  rc = launch_dep(kern, dim3((unsigned)ctas), WARPS * 32, SMEM, st, prm);
  return rc || prm.splits == 1 ? rc : launch_join<D>(prm, ROWS, 0, PAGED ? P_UP : 0.f, st);
}

// ---------------------------------------------------------------------------------------------------------------- plan, workspace
// How a call is cut: row tiles of 16 or of 128, and splits of the key axis where there are fewer of them than the device has room for.
struct KeysPlan {
  bool tc;                                  // tensor memory, 128 rows
  int tokens, sms;                          // (tc) tokens of a tile
  long long tiles, units, all;              // per key head; of the call; rows of all tiles
  int splits;
  size_t o_bytes, total;                    // of the workspace
};
static int device_sms() {
  static std::atomic<int> sms[64];
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 148;
  if ((n = sms[dev].load(std::memory_order_relaxed)) > 0) return n;
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) {
    (void)cudaGetLastError();
    return 148;
  }
  sms[dev].store(n, std::memory_order_relaxed);
  return n;
}
static KeysPlan keys_plan(int B, int Hk, int group, int M, long long S, int d, bool paged, bool maps) {
  KeysPlan k = {};
  k.sms = device_sms();
  const long long rows = (long long)M * group;
  // Rows of a key head, few-row kernel against many-row kernel, us.  Cached keys, eight sequences of 65 536 tokens, 8 key heads of 128: 8 rows 239 / 1 025, 16:
  // 470 / 1 024, 20: 676 / 1 025, 32: 898 / 1 025, 48: 1 320 / 1 025; 64 sequences of 2 048: 16 rows 140 / 234, 20: 183 / 236, 32: 228 / 238, 64: 436 / 240; two of
  // 32 768, 24 heads: 16 rows 170 / 406, 24: 240 / 409, 32: 348 / 406, 64: 662 / 409.  So from 17 to 32 rows the few-row kernel would be the faster one too, by 4 to
  // 70 %, and neither is near what the codes take (164, 41, 62): such calls lack a kernel of their own.  bf16 keys, 2 x 24 heads x 512 keys: 16 rows
  // 11.6 / 11.8, 17: 18.9 / 11.8, 32: 19.2 / 11.7; 16 heads x 8 192 keys of 64: 16 rows 23.6 / 33.0, 32: 30.7 / 32.3, 33: 36.6 / 33.1.
  k.tc = maps && group <= 128 && rows > (paged ? 2 * PAGED_ROWS : 2 * FEW_ROWS);
  k.tokens = k.tc ? 128 / group : 0;
  const int per = k.tc ? 128 : paged ? PAGED_ROWS : FEW_ROWS;
  k.tiles = k.tc ? (M + k.tokens - 1) / k.tokens : (rows + per - 1) / per;
  k.units = (long long)B * Hk * k.tiles;
  k.all = k.units * per;
  if (k.tc) {
    // The number of splits for which the pairs of SMs are done first: a pair's share of the items and one more, for the last round and for items of
    // unequal length, each as long as its key tiles and some 2 tiles more; and for more than one split the partial sums: 512 KB of HBM traffic per item, 3 / 74 of the 2 us that a pair takes for a tile.  At least four key tiles per split.
    // (24 heads x 4 680 queries x 32 760 keys, 240 items for 74 pairs: 2 418 us in one split, 2 179 in four.)
    const long long items = (long long)B * Hk * ((k.tiles + 3) / 4), pairs = k.sms / 2 > 0 ? k.sms / 2 : 1, tiles = (S + 127) / 128;
    double best = 0.0;
    k.splits = 1;
    for (int n = 1; n <= 64 && (n == 1 || tiles / n >= 4); ++n) {
      const double share = (double)(items * n) / (double)pairs, rounds = share <= 1.0 ? 1.0 : share + 1.0;
      const double time = rounds * ((double)((tiles + n - 1) / n) + 2.0) + (n > 1 ? 3.0 + 3.0 * d / 128 * n * (double)items / (double)pairs : 0.0);
      if (n == 1 || time < best) {
        best = time;
        k.splits = n;
      }
    }
  } else {
    // at least 256 keys per split; CTAs for four rounds, with cached keys (three per SM) two.  (Two sequences of 65 536 tokens / eight of up to 131 071, 8 key
    // heads, us: 6 CTAs' worth per SM 78 / 320, 7: 94 / 348, 9: 87 / 322, 12: 98 / 312; CTAs of eight warps, two per SM, 4: 86 / 376, 8: 100 / 372.)
    long long splits = k.units > 0 ? k.sms * (paged ? 2 * PAGED_CTAS : 4) / k.units : 1;
    if (splits > S / 256) splits = S / 256;
    k.splits = (int)(splits < 1 ? 1 : splits);
  }
  if (k.splits > 1) {
    k.o_bytes = (size_t)k.splits * k.all * d * 4;
    k.total = k.o_bytes + (size_t)k.splits * k.all * 8;
  }
  return k;
}
static KeysPlan cached_plan(const sva_kv_cache_t* c, const sva_cached_attn_t* p) {
  return keys_plan(p->B, c->H, p->Hq / c->H, p->M, (long long)p->max_pages * c->page, c->d, true, true);
}
// (tensor maps know no stride of 0 along tokens, none of 0 along Q's heads and items, and strides below 2^40 bytes)
static KeysPlan cross_plan(const sva_cross_attn_t* p) {
  auto fits = [](const int64_t s[3]) { return s[0] < (1LL << 38) && s[1] < (1LL << 38) && s[2] < (1LL << 38); };
  const bool maps = p->S > 0 && (p->N == 1 || p->q_stride[2] > 0) && (p->Hq == 1 || p->q_stride[1] > 0) && (p->B == 1 || p->q_stride[0] > 0) &&
                    (p->S == 1 || (p->k_stride[2] > 0 && p->v_stride[2] > 0)) && fits(p->q_stride) && fits(p->k_stride) && fits(p->v_stride);
  return keys_plan(p->B, p->Hk, p->Hq / p->Hk, p->N, p->S, p->d, false, maps);
}

size_t cached_attn_workspace_bytes(const sva_kv_cache_t* c, const sva_cached_attn_t* p) { return cached_plan(c, p).total; }
size_t cross_attn_workspace_bytes(const sva_cross_attn_t* p) { return cross_plan(p).total; }

static int launch_keys(KeysParams& prm, bool paged, const KeysPlan& plan, void* ws, cudaStream_t st) {
  if (plan.all > 0x7fffffffLL) return SVA_ERR_UNSUPPORTED;
  prm.tiles = (int)plan.tiles;
  prm.splits = plan.splits;
  prm.part_o = static_cast<float*>(ws);
  prm.part_ml = reinterpret_cast<float2*>(static_cast<uint8_t*>(ws) + plan.o_bytes);
  note_choice(plan.tc ? 128 : paged ? PAGED_ROWS : FEW_ROWS);
  if (plan.tc) {
    const int rc = launch_keys_tc(prm, paged, plan.sms, st);
    if (rc || prm.splits == 1) return rc;
    return prm.d == 128 ? launch_join<128>(prm, 128, plan.tokens, 0.f, st) : launch_join<64>(prm, 128, plan.tokens, 0.f, st);
  }
  if (paged) return prm.d == 128 ? launch_few<128, true>(prm, st) : launch_few<64, true>(prm, st);
  return prm.d == 128 ? launch_few<128, false>(prm, st) : launch_few<64, false>(prm, st);
}

static int check_space(const KeysPlan& plan, const void* ws, size_t ws_bytes) {
  if (plan.total == 0) return SVA_OK;
  if (!ws || ws_bytes < plan.total) return SVA_ERR_WORKSPACE;
  return reinterpret_cast<uintptr_t>(ws) & 255u ? SVA_ERR_ALIGNMENT : SVA_OK;
}

int launch_cached_attn(const sva_kv_cache_t* c, const sva_cached_attn_t* p, const void* q, const int32_t* table, const int32_t* lengths,
                       const int32_t* counts, void* o, float* lse, int32_t* status, void* ws, size_t ws_bytes, cudaStream_t st) {
  const KeysPlan plan = cached_plan(c, p);
  int rc = check_space(plan, ws, ws_bytes);
  if (rc) return rc;
  KeysParams prm = {};
  prm.q = (const uint8_t*)q; prm.o = (uint8_t*)o; prm.lse = lse;
  prm.sq = make_strides(p->q_stride); prm.so = make_strides(p->o_stride);
  prm.B = p->B; prm.Hq = p->Hq; prm.Hk = c->H; prm.group = p->Hq / c->H; prm.M = p->M; prm.d = c->d;
  prm.causal = p->causal;
  prm.scale_log2 = (p->softmax_scale > 0.f ? p->softmax_scale : 1.0f / sqrtf((float)c->d)) * 1.4426950408889634f;
  prm.lengths = lengths; prm.counts = counts;
  prm.k = (const uint8_t*)c->k_codes; prm.v = (const uint8_t*)c->v_codes;
  prm.k_scale = c->k_scale; prm.v_scale = c->v_scale;
  prm.table = table; prm.table_stride = p->table_stride;
  const long long most = (long long)p->max_pages * c->page;
  prm.S = (int)(most < 0x7fffff00LL ? most : 0x7fffff00LL);
  prm.page = c->page; prm.pages = c->pages; prm.max_pages = p->max_pages;
  prm.status = status;
  return launch_keys(prm, true, plan, ws, st);
}

int launch_cross_attn(const sva_cross_attn_t* p, const void* q, const void* k, const void* v, const int32_t* lengths, const uint8_t* mask, void* o,
                      float* lse, int32_t* status, void* ws, size_t ws_bytes, cudaStream_t st) {
  const KeysPlan plan = cross_plan(p);
  int rc = check_space(plan, ws, ws_bytes);
  if (rc) return rc;
  KeysParams prm = {};
  prm.q = (const uint8_t*)q; prm.o = (uint8_t*)o; prm.lse = lse;
  prm.sq = make_strides(p->q_stride); prm.so = make_strides(p->o_stride);
  prm.sk = make_strides(p->k_stride); prm.sv = make_strides(p->v_stride);
  prm.B = p->B; prm.Hq = p->Hq; prm.Hk = p->Hk; prm.group = p->Hq / p->Hk; prm.M = p->N; prm.d = p->d;
  prm.scale_log2 = (p->softmax_scale > 0.f ? p->softmax_scale : 1.0f / sqrtf((float)p->d)) * 1.4426950408889634f;
  prm.lengths = lengths;
  prm.k = (const uint8_t*)k; prm.v = (const uint8_t*)v;
  prm.mask = mask; prm.mask_stride = p->mask_stride;
  prm.S = p->S;
  prm.status = status;
  return launch_keys(prm, false, plan, ws, st);
}

}  // namespace sva
