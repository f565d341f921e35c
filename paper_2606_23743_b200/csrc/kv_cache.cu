// Quantised K/V cache: rows of K and V (one token of one head, d values) as e4m3 codes with an fp32 scale, or as 4-bit codes with an e4m3
// scale per 16 channels and an fp32 scale, in pages of `page` tokens, [pages][H][page][...].  A token has a slot
// (page id * page + place in the page); writing quantises into slots, reading collects a sequence's pages into the [B,H,N,d] tensors that the
// attention calls take.
//
// Both are HBM-bound streaming passes, the 4-bit cast also by its instructions.  d/16 lanes own a row, 16 channels each (one 4-bit scale block),
// so that a row's maximum is a few shuffles; a thread looks its token's slot up once and then has some heads' rows in flight.
// 24 heads of 32 760 tokens, us, one call after another: e4m3 written 91 = 6.7 TB/s, read 95 = 6.4; 4-bit 86 = 6.1 and 83 = 6.3; heads of 64: e4m3 48.2
// and 49.9, 4-bit 47.4 and 44.4.
#include <cuda_fp4.h>

#include "common.cuh"

namespace sva {

static constexpr int CACHE_THREADS = 256;
static constexpr int CACHE_HEADS = 4;                     // rows in flight per thread

struct CacheArrays {                                      // one of K, V
  uint8_t* codes;
  float* scale;
  uint8_t* sf;
};

struct CacheParams {
  CacheArrays k, v;
  uint8_t *xk, *xv;                                       // bf16 tensors, read or written
  Strides sk, sv;
  const int32_t *slots, *table, *lengths;
  long long table_stride, tokens;                         // tokens: B * T, or B * N
  long long slot_count;
  int H, T, page, pages, max_pages, chunk, chunks;        // chunk: heads per CTA, chunks: CTAs per token tile and tensor
  int32_t* status;
  bool wide;                                              // 32-byte stores into the bf16 tensors
};

// row of (page, head, place) among all rows
__device__ __forceinline__ long long cache_row(const CacheParams& prm, long long page, int h, int place) {
  return (page * prm.H + h) * prm.page + place;
}

// The casts of a lane's 16 values by general divisions: rows whose scale is far out (zero, infinite, NaN, 1e-12 and less) or has a significand of ones.
struct Cast { uint4 codes; float scale; uint32_t sf; };
template <bool FP4>
__device__ __noinline__ Cast cache_cast_any(uint4 a, uint4 b, float amax, float own) {
  const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  Cast o;
  o.codes = make_uint4(0u, 0u, 0u, 0u);
  o.sf = 0u;
  uint32_t c[4] = {0u, 0u, 0u, 0u};
  o.scale = amax == 0.f ? 1.0f : __fdiv_rn(amax, FP4 ? 2688.0f : 448.0f);
  float unit = o.scale;
  if (FP4) {
    o.sf = (uint32_t)__nv_cvt_float_to_fp8(__fdiv_rn(__fdiv_rn(own, 6.0f), o.scale), __NV_SATFINITE, __NV_E4M3);
    unit = __fmul_rn(e4m3_to_float(o.sf), o.scale);
    if (!(unit > 0.f)) {
      o.sf = 0u;
      return o;
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float lo = __fdiv_rn(bf16lo(w[e]), unit), hi = __fdiv_rn(bf16hi(w[e]), unit);
    if (FP4) c[e >> 2] |= ((uint32_t)__nv_cvt_float2_to_fp4x2(make_float2(lo, hi), __NV_E2M1, cudaRoundNearest) & 0xffu) << (8 * (e & 3));
    else c[e >> 1] |= e4m3x2(lo, hi) << (16 * (e & 1));
  }
  o.codes = make_uint4(c[0], c[1], c[2], c[3]);
  return o;
}

// The same with quotients from reciprocals (div_fast).  In a row whose amax is in [2^-38, 2^60] every divisor is in div_fast's range, and a 4-bit
// block's maximum that is too small for it gives a scale of zero in any case.
template <bool FP4>
__device__ __forceinline__ Cast cache_cast(const uint4& a, const uint4& b, float amax, float own) {
  const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  Cast o;
  o.scale = div_fast(amax, FP4 ? 2688.0f : 448.0f, FP4 ? 1.0f / 2688.0f : 1.0f / 448.0f);
  o.sf = 0u;
  float unit = o.scale, rcp = __frcp_rn(o.scale);
  bool ones = (__float_as_uint(o.scale) & 0x7fffffu) == 0x7fffffu;
  if (FP4) {
    o.sf = (uint32_t)__nv_cvt_float_to_fp8(div_fast(div_fast(own, 6.0f, 1.0f / 6.0f), o.scale, rcp), __NV_SATFINITE, __NV_E4M3);
    unit = __fmul_rn(e4m3_to_float(o.sf), o.scale);
    rcp = __frcp_rn(unit);
    ones |= (__float_as_uint(unit) & 0x7fffffu) == 0x7fffffu;
  }
  if (!(amax >= 3.637978807091713e-12f && amax <= 1.152921504606847e18f) || ones) return cache_cast_any<FP4>(a, b, amax, own);
  const uint64_t neg2 = pack2(-unit, -unit), r2 = pack2(rcp, rcp);
  uint64_t y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = div_fast2(pack2(bf16lo(w[e]), bf16hi(w[e])), neg2, r2);
  if (FP4) {
    o.codes = make_uint4(o.sf ? e2m1x8(y[0], y[1], y[2], y[3]) : 0u, o.sf ? e2m1x8(y[4], y[5], y[6], y[7]) : 0u, 0u, 0u);
  } else {
    o.codes = make_uint4(e4m3x4(y[0], y[1]), e4m3x4(y[2], y[3]), e4m3x4(y[4], y[5]), e4m3x4(y[6], y[7]));
  }
  return o;
}

template <int LANES, bool FP4>
__global__ void __launch_bounds__(CACHE_THREADS)
cache_write_kernel(const CacheParams prm) {
  const int zero = grid_dep_wait();
  const int which = blockIdx.x & 1, part = (int)((blockIdx.x >> 1) % prm.chunks);
  const long long t = (long long)((blockIdx.x >> 1) / prm.chunks) * (CACHE_THREADS / LANES) + threadIdx.x / LANES + zero;
  const int lane = threadIdx.x % LANES;
  const CacheArrays out = which ? prm.v : prm.k;
  const Strides s = which ? prm.sv : prm.sk;
  // (all lanes of a row share its token; the shuffles below are taken by every thread)
  long long slot = -1;
  if (t < prm.tokens) slot = __ldg(prm.slots + t);
  if (slot >= prm.slot_count) {
    if (lane == 0 && part == 0 && prm.status) atomicOr(prm.status, SVA_DEV_BAD_INDEX);
    slot = -1;
  }
  const bool there = slot >= 0;
  const long long b = there ? t / prm.T : 0, n = there ? t - b * prm.T : 0;
  const long long page = there ? slot / prm.page : 0;
  const int place = there ? (int)(slot - page * prm.page) : 0;
  const int hb = part * prm.chunk, he = there ? min(hb + prm.chunk, prm.H) : 0;
  const uint8_t* src = (which ? prm.xv : prm.xk) + 2 * (b * s.b + n * s.n + hb * s.h + lane * 16);
  const long long row = cache_row(prm, page, hb, place);
  constexpr int BYTES = FP4 ? 8 : 16;
  uint8_t *codes = out.codes + (row * LANES + lane) * BYTES, *sf = FP4 ? out.sf + row * LANES + lane : nullptr;
  float* scale = out.scale + row;
  for (int h0 = hb; h0 < hb + prm.chunk; h0 += CACHE_HEADS) {
    uint4 in[CACHE_HEADS][2];
#pragma unroll
    for (int i = 0; i < CACHE_HEADS; ++i) {
      in[i][0] = in[i][1] = make_uint4(0u, 0u, 0u, 0u);
      if (h0 + i < he) {
        in[i][0] = __ldg(reinterpret_cast<const uint4*>(src));
        in[i][1] = __ldg(reinterpret_cast<const uint4*>(src) + 1);
      }
      src += 2 * s.h;
    }
#pragma unroll
    for (int i = 0; i < CACHE_HEADS; ++i) {
      // (4-bit codes have no NaN: one that is there becomes the row's scale; as bits, since a maximum of floats would lose it)
      const float own = bf16_amax<FP4>(in[i][0], in[i][1]);
      uint32_t amax = __float_as_uint(own);
#pragma unroll
      for (int o = LANES / 2; o; o >>= 1) amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, o));
      if (h0 + i < he) {
        const Cast x = cache_cast<FP4>(in[i][0], in[i][1], __uint_as_float(amax), own);
        if (lane == 0) *scale = x.scale;
        if (FP4) {
          *sf = (uint8_t)x.sf;
          *reinterpret_cast<uint2*>(codes) = make_uint2(x.codes.x, x.codes.y);
        } else {
          *reinterpret_cast<uint4*>(codes) = x.codes;
        }
      }
      codes += (long long)prm.page * LANES * BYTES;
      if (FP4) sf += (long long)prm.page * LANES;
      scale += prm.page;
    }
  }
}

template <int LANES, bool FP4>
__global__ void __launch_bounds__(CACHE_THREADS, 5)
cache_read_kernel(const CacheParams prm) {
  const int zero = grid_dep_wait();
  const int which = blockIdx.x & 1, part = (int)((blockIdx.x >> 1) % prm.chunks);
  const long long t = (long long)((blockIdx.x >> 1) / prm.chunks) * (CACHE_THREADS / LANES) + threadIdx.x / LANES + zero;
  const int lane = threadIdx.x % LANES;
  if (t >= prm.tokens) return;
  const CacheArrays in = which ? prm.v : prm.k;
  const Strides s = which ? prm.sv : prm.sk;
  const long long b = t / prm.T;
  const int n = (int)(t - b * prm.T), at = n / prm.page;
  bool there = n < __ldg(prm.lengths + b);
  long long page = 0;
  if (there) {
    page = at < prm.max_pages ? __ldg(prm.table + b * prm.table_stride + at) : -1;
    if (page < 0 || page >= prm.pages) {
      if (lane == 0 && part == 0 && prm.status) atomicOr(prm.status, SVA_DEV_BAD_INDEX);
      there = false;
    }
  }
  const int place = n - at * prm.page, hb = part * prm.chunk, he = min(hb + prm.chunk, prm.H);
  uint8_t* dst = (which ? prm.xv : prm.xk) + 2 * (b * s.b + (long long)n * s.n + lane * 16);
  for (int h0 = hb; h0 < he; h0 += CACHE_HEADS) {
    uint4 codes[CACHE_HEADS];
    float scale[CACHE_HEADS];
    uint32_t sf[CACHE_HEADS];
#pragma unroll
    for (int i = 0; i < CACHE_HEADS; ++i) {
      codes[i] = make_uint4(0u, 0u, 0u, 0u);
      scale[i] = 0.f;
      sf[i] = 0u;
      if (there && h0 + i < he) {
        const long long row = cache_row(prm, page, h0 + i, place);
        scale[i] = __ldg(in.scale + row);
        if (FP4) {
          const uint2 c = __ldg(reinterpret_cast<const uint2*>(in.codes + (row * LANES + lane) * 8));
          codes[i].x = c.x; codes[i].y = c.y;
          sf[i] = __ldg(in.sf + row * LANES + lane);
        } else {
          codes[i] = __ldg(reinterpret_cast<const uint4*>(in.codes + (row * LANES + lane) * 16));
        }
      }
    }
#pragma unroll
    for (int i = 0; i < CACHE_HEADS; ++i) {
      if (h0 + i >= he) continue;
      uint32_t o[8];
      const uint32_t w[4] = {codes[i].x, codes[i].y, codes[i].z, codes[i].w};
      const float unit = FP4 ? e4m3_to_float(sf[i]) : 1.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float2 x;
        if (FP4) {
          const __half2_raw h = __nv_cvt_fp4x2_to_halfraw2((__nv_fp4x2_storage_t)(w[e >> 2] >> (8 * (e & 3)) & 0xffu), __NV_E2M1);
          x = __half22float2(__half2(h));
          x.x *= unit; x.y *= unit;                         // exact: 2 by 4 significant bits
        } else {
          x = e4m3x2_to_float2(w[e >> 1] >> (16 * (e & 1)) & 0xffffu);
        }
        const __nv_bfloat162 v = __floats2bfloat162_rn(__fmul_rn(x.x, scale[i]), __fmul_rn(x.y, scale[i]));
        o[e] = *reinterpret_cast<const uint32_t*>(&v);
      }
      uint4* row = reinterpret_cast<uint4*>(dst + 2 * (h0 + i) * s.h);
      const uint4 lo = make_uint4(o[0], o[1], o[2], o[3]), hi = make_uint4(o[4], o[5], o[6], o[7]);
      // 2 x 47 616 tokens x 32 heads, e4m3: 373 us in stores of 16 bytes, which touch every sector twice, 360 in stores of 32; (loads of 32 in the
      // other kernel: 354 us, of 16, the L1 having the other half, 347)
      if (prm.wide) {
        stg32(row, lo, hi);
      } else {
        row[0] = lo;
        row[1] = hi;
      }
    }
  }
}

// whether every row of a tensor begins on 32 bytes
static bool rows_on_32(const void* x, const Strides& s) {
  return (reinterpret_cast<uintptr_t>(x) & 31u) == 0 && ((s.b | s.h | s.n) & 15) == 0;
}

static int launch_cache(bool write, CacheParams& prm, const sva_kv_cache_t* c, cudaStream_t st) {
  prm.k = CacheArrays{(uint8_t*)c->k_codes, c->k_scale, (uint8_t*)c->k_sf};
  prm.v = CacheArrays{(uint8_t*)c->v_codes, c->v_scale, (uint8_t*)c->v_sf};
  prm.H = c->H; prm.page = c->page; prm.pages = c->pages;
  prm.wide = rows_on_32(prm.xk, prm.sk) && rows_on_32(prm.xv, prm.sv);
  const int lanes = c->d / 16;
  const long long tiles = (prm.tokens + CACHE_THREADS / lanes - 1) / (CACHE_THREADS / lanes);
  // Heads per CTA: eight, whose second half's loads find the slots and the table at hand, where the grid comes to sixteen CTAs per SM all the
  // same.  2 x 47 616 tokens x 32 heads, e4m3, written / read, us: four heads 375 / 358, eight 347 / 360, sixteen 350 / 362;
  // 24 x 32 760 tokens, 4-bit: 114 / 88, 106 / 86, 108 / 88.
  prm.chunk = 2 * CACHE_HEADS;
  if (2 * tiles * ((c->H + prm.chunk - 1) / prm.chunk) < 148 * 16) prm.chunk = CACHE_HEADS;
  prm.chunks = (c->H + prm.chunk - 1) / prm.chunk;
  const long long ctas = 2 * tiles * prm.chunks;
  if (ctas > 0x7fffffffLL) return SVA_ERR_UNSUPPORTED;
  note_choice(prm.chunk);
  const bool fp4 = c->format == SVA_CACHE_FP4;
  auto kern = write ? (lanes == 8 ? (fp4 ? cache_write_kernel<8, true> : cache_write_kernel<8, false>)
                                  : (fp4 ? cache_write_kernel<4, true> : cache_write_kernel<4, false>))
                    : (lanes == 8 ? (fp4 ? cache_read_kernel<8, true> : cache_read_kernel<8, false>)
                                  : (fp4 ? cache_read_kernel<4, true> : cache_read_kernel<4, false>));
  return launch_dep(kern, dim3((unsigned)ctas), CACHE_THREADS, 0, st, prm);
}

int launch_cache_write(const sva_kv_cache_t* c, const void* k, const void* v, const int64_t ks[3], const int64_t vs[3], int B, int T,
                       const int32_t* slots, int32_t* status, cudaStream_t st) {
  CacheParams prm = {};
  prm.xk = (uint8_t*)k; prm.xv = (uint8_t*)v;
  prm.sk = make_strides(ks); prm.sv = make_strides(vs);
  prm.slots = slots;
  prm.tokens = (long long)B * T; prm.T = T;
  prm.slot_count = (long long)c->pages * c->page;
  prm.status = status;
  return launch_cache(true, prm, c, st);
}

int launch_cache_read(const sva_kv_cache_t* c, const int32_t* table, int64_t table_stride, int max_pages, const int32_t* lengths, int B, int N,
                      void* k, void* v, const int64_t ks[3], const int64_t vs[3], int32_t* status, cudaStream_t st) {
  CacheParams prm = {};
  prm.xk = (uint8_t*)k; prm.xv = (uint8_t*)v;
  prm.sk = make_strides(ks); prm.sv = make_strides(vs);
  prm.table = table; prm.table_stride = table_stride; prm.max_pages = max_pages; prm.lengths = lengths;
  prm.tokens = (long long)B * N; prm.T = N;
  prm.status = status;
  return launch_cache(false, prm, c, st);
}

}  // namespace sva
