// Appending to the K/V cache whose e4m3 codes share one scale per page and head (sva.h: SVA_CACHE_E4M3_PAGE).
//
// A CTA owns one page of one head of K or V: it reads the page's new rows once, keeps them in registers while their largest magnitude is found, and
// writes their codes.  Where that outgrows the scale of rows that are there already, the CTA reads their codes and writes them again under the
// new one: at most d bytes a row, and only in the page that a sequence ended in.  d/16 lanes own a row, 16 channels each; up to APPEND_PASSES
// rows per lane stay in registers, which is a call's part of the page up to 1 024 tokens (512 for d = 128); rows behind them are read twice.
// HBM-bound: 2 d bytes of a row are read and d written.  A call is sized by its new rows: one token for each of 64 sequences, 8 heads of 128, takes 2.8 us where
// no scale grows; where all of them do, one warp re-expresses each page in turns of four rows, 5.7 us with pages of 64 tokens, 17.7 with 256 and 133 with 1 024.
#include "common.cuh"

namespace sva {

static constexpr int APPEND_PASSES = 4;

struct AppendParams {
  uint8_t *k_codes, *v_codes;
  float *k_scale, *v_scale;
  const uint8_t *xk, *xv;
  Strides sk, sv;
  const int32_t *table, *lengths, *counts;
  long long table_stride;
  int H, T, page, pages, max_pages, touched;      // touched: pages that T tokens can lie on
  int32_t* status;
};

// 16 values over s, as e4m3 codes (s = 0: all values are zeros)
__device__ __noinline__ uint4 codes16_any(uint4 a, uint4 b, float s) {
  const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  uint32_t c[4] = {0u, 0u, 0u, 0u};
  if (s == 0.f) return make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
  for (int e = 0; e < 8; ++e) c[e >> 1] |= e4m3x2(__fdiv_rn(bf16lo(w[e]), s), __fdiv_rn(bf16hi(w[e]), s)) << (16 * (e & 1));
  return make_uint4(c[0], c[1], c[2], c[3]);
}
__device__ __forceinline__ uint4 codes16(const uint4& a, const uint4& b, uint64_t neg2, uint64_t r2) {
  const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  uint64_t y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = div_fast2(pack2(bf16lo(w[e]), bf16hi(w[e])), neg2, r2);
  return make_uint4(e4m3x4(y[0], y[1]), e4m3x4(y[2], y[3]), e4m3x4(y[4], y[5]), e4m3x4(y[6], y[7]));
}

template <int LANES>
__global__ void __launch_bounds__(1024)
cache_append_kernel(const AppendParams prm) {
  __shared__ uint32_t warp_amax[32];
  const int zero = grid_dep_wait();
  // head fastest: CTAs side by side read neighbouring heads of the same tokens
  long long at = (long long)blockIdx.x + zero;
  const int h = (int)(at % prm.H); at /= prm.H;
  const int which = (int)(at & 1); at >>= 1;
  const int j = (int)(at % prm.touched);
  const int b = (int)(at / prm.touched);
  const long long held = max(__ldg(prm.lengths + b), 0);
  const int count = prm.counts ? min(max(__ldg(prm.counts + b), 0), prm.T) : prm.T;
  const long long place = held / prm.page + j;                       // page of the sequence
  const long long begin = place * prm.page;
  // rows of this page: old ones are places below lo, new ones [lo, hi)
  const int lo = (int)max(held - begin, 0LL);
  const int hi = (int)min((long long)prm.page, held + count - begin);
  if (lo >= hi) return;                                              // nothing of the call lies here (the whole CTA)
  const int id = place < prm.max_pages ? __ldg(prm.table + b * prm.table_stride + place) : -1;
  if (id < 0 || id >= prm.pages) {
    if (threadIdx.x == 0 && h == 0 && which == 0 && prm.status) atomicOr(prm.status, SVA_DEV_BAD_INDEX);
    return;
  }
  const Strides s = which ? prm.sv : prm.sk;
  const int lane = threadIdx.x % LANES, row0 = threadIdx.x / LANES, step = blockDim.x / LANES;
  const uint8_t* src = (which ? prm.xv : prm.xk) + 2 * (b * s.b + h * s.h + lane * 16);
  const long long first = begin - held;                              // token of the call at place 0 (may be negative)
  const long long head = (long long)id * prm.H + h;
  uint8_t* codes = (which ? prm.v_codes : prm.k_codes) + (head * prm.page * LANES + lane) * 16;
  float* scale = (which ? prm.v_scale : prm.k_scale) + head;

  uint4 in[APPEND_PASSES][2];
  uint32_t amax = 0u;
#pragma unroll
  for (int i = 0; i < APPEND_PASSES; ++i) {
    in[i][0] = in[i][1] = make_uint4(0u, 0u, 0u, 0u);
    const int row = lo + row0 + i * step;
    if (row < hi) {
      const uint4* p = reinterpret_cast<const uint4*>(src + 2 * (first + row) * s.n);
      in[i][0] = __ldg(p);
      in[i][1] = __ldg(p + 1);
    }
  }
#pragma unroll
  for (int i = 0; i < APPEND_PASSES; ++i) amax = max(amax, __float_as_uint(bf16_amax<true>(in[i][0], in[i][1])));
  for (int row = lo + row0 + APPEND_PASSES * step; row < hi; row += step) {          // (pages beyond what the registers hold)
    const uint4* p = reinterpret_cast<const uint4*>(src + 2 * (first + row) * s.n);
    amax = max(amax, __float_as_uint(bf16_amax<true>(__ldg(p), __ldg(p + 1))));
  }
  // (as bits: magnitudes are ordered as their bits are, NaN above infinity)
#pragma unroll
  for (int o = 16; o; o >>= 1) amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, o));
  if (blockDim.x > 32) {
    if ((threadIdx.x & 31) == 0) warp_amax[threadIdx.x >> 5] = amax;
    __syncthreads();
    for (int w = 0; w < (int)blockDim.x / 32; ++w) amax = max(amax, warp_amax[w]);
  }
  const float old_scale = lo > 0 ? *scale : 0.f;
  float now = div_by_448(__uint_as_float(amax));
  if (!(now >= old_scale)) now = isnan(now) ? now : old_scale;       // (the larger; a NaN of either stays)
  if (lo > 0) {
    __syncthreads();                                                 // (every thread has the old scale)
    if (now > old_scale) {
      const float ratio = __fdiv_rn(old_scale, now);
      for (int row = row0; row < lo; row += step) {
        uint4* c = reinterpret_cast<uint4*>(codes + (long long)row * LANES * 16);
        const uint4 was = *c;
        uint32_t w[4] = {was.x, was.y, was.z, was.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 x = e4m3x2_to_float2(w[e] & 0xffffu), y = e4m3x2_to_float2(w[e] >> 16);
          w[e] = e4m3x2(__fmul_rn(x.x, ratio), __fmul_rn(x.y, ratio)) | e4m3x2(__fmul_rn(y.x, ratio), __fmul_rn(y.y, ratio)) << 16;
        }
        *c = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
  }
  if (threadIdx.x == 0) *scale = now;
  const bool fast = div_fast_ok(now);
  const float rcp = fast ? __frcp_rn(now) : 0.f;
  const uint64_t neg2 = pack2(-now, -now), r2 = pack2(rcp, rcp);
#pragma unroll
  for (int i = 0; i < APPEND_PASSES; ++i) {
    const int row = lo + row0 + i * step;
    if (row < hi)
      *reinterpret_cast<uint4*>(codes + (long long)row * LANES * 16) = fast ? codes16(in[i][0], in[i][1], neg2, r2) : codes16_any(in[i][0], in[i][1], now);
  }
  for (int row = lo + row0 + APPEND_PASSES * step; row < hi; row += step) {
    const uint4* p = reinterpret_cast<const uint4*>(src + 2 * (first + row) * s.n);
    const uint4 a = __ldg(p), c = __ldg(p + 1);
    *reinterpret_cast<uint4*>(codes + (long long)row * LANES * 16) = fast ? codes16(a, c, neg2, r2) : codes16_any(a, c, now);
  }
}

int launch_cache_append(const sva_kv_cache_t* c, const void* k, const void* v, const int64_t ks[3], const int64_t vs[3], int B, int T,
                        const int32_t* table, int64_t table_stride, int max_pages, const int32_t* lengths, const int32_t* counts, int32_t* status,
                        cudaStream_t st) {
  AppendParams prm = {};
  prm.k_codes = (uint8_t*)c->k_codes; prm.v_codes = (uint8_t*)c->v_codes;
  prm.k_scale = c->k_scale; prm.v_scale = c->v_scale;
  prm.xk = (const uint8_t*)k; prm.xv = (const uint8_t*)v;
  prm.sk = make_strides(ks); prm.sv = make_strides(vs);
  prm.table = table; prm.lengths = lengths; prm.counts = counts;
  prm.table_stride = table_stride;
  prm.H = c->H; prm.T = T; prm.page = c->page; prm.pages = c->pages; prm.max_pages = max_pages;
  prm.touched = (int)(((long long)T + c->page - 2) / c->page) + 1;
  prm.status = status;
  const int lanes = c->d / 16;
  // rows of a page, or of a call that is shorter, over APPEND_PASSES passes
  const int rows = T < c->page ? T : c->page;
  long long threads = (long long)((rows + APPEND_PASSES - 1) / APPEND_PASSES) * lanes;
  threads = threads < 1024 ? (threads + 31) / 32 * 32 : 1024;
  const long long ctas = 2LL * prm.H * prm.touched * B;
  if (ctas > 0x7fffffffLL) return SVA_ERR_UNSUPPORTED;
  return launch_dep(lanes == 8 ? cache_append_kernel<8> : cache_append_kernel<4>, dim3((unsigned)ctas), dim3((unsigned)threads), 0, st, prm);
}

}  // namespace sva
