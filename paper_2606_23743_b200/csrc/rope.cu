// Rotary positions of Q and K as a call of its own (the fused prologue covers whole heads in the interleaved layout from a table of cosines
// behind an RMS norm; this one rotates what a projection wrote, in either layout, the whole head or a part of it, from integer positions
// on one to three axes, and back again).
//
// Pair j of a token at position p turns by p * theta_j.  theta_j / 2 pi is held as a 64-bit fraction of a turn, step_j; p * step_j
// modulo 2^64 is the phase with whole turns taken off, exactly, for any 32-bit position: an fp32 product p * theta_j would be off by p * 2^-24
// radians (0.06 at a million).  Its upper 32 bits go to fp32 (error 2^-25 turns) and on to sincospif.
//
// HBM-bound: 2 bytes read and 2 written per element.  A thread owns the same channels of one token in several heads, so that
// the phases are made once per token and HEADS rows are in flight.
#include "common.cuh"

namespace sva {

static constexpr int ROPE_THREADS = 256;
static constexpr int ROPE_HEADS = 4;                      // rows in flight per thread

struct RopeParams {
  const uint8_t *q, *k;
  uint8_t *qo, *ko;
  Strides sq, sk, sqo, sko;
  const unsigned long long* steps;
  const int32_t* pos;
  long long pos_axis, pos_batch;
  int Hq, Hk, N, d, half, end0, end1;                    // half = pairs; pairs below end0 turn with axis 0, below end1 with axis 1
  long long tokens;                                       // B * N
  int chunk, q_chunks, chunks;                            // heads per CTA; CTAs per token tile for Q, and for Q and K
  float factor, sin_factor;
};

struct Turn { float c, s; };
__device__ __forceinline__ Turn rope_turn(const RopeParams& prm, const unsigned long long* steps, const int32_t* pos, int pair) {
  Turn t = {1.f, 0.f};                                    // channels that are not rotated
  if (pair < prm.half) {
    const long long p = __ldg(pos + (pair < prm.end0 ? 0 : pair < prm.end1 ? prm.pos_axis : 2 * prm.pos_axis));
    const unsigned long long phase = (unsigned long long)p * __ldg(steps + pair);
    float s, c;
    sincospif((float)(int)(phase >> 32) * 4.656612873077393e-10f, &s, &c);       // 2^-31: half turns
    t.c = c * prm.factor;
    t.s = s * prm.sin_factor;
  }
  return t;
}

__device__ __forceinline__ void rope_pair(float& a, float& b, const Turn& t) {
  const float x = a;
  a = x * t.c - b * t.s;
  b = b * t.c + x * t.s;
}

// Unpacks, packs 8 bf16 values.
__device__ __forceinline__ void rope_load8(const uint4& u, float (&x)[8]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) { x[2 * e] = bf16lo(w[e]); x[2 * e + 1] = bf16hi(w[e]); }
}
__device__ __forceinline__ uint4 rope_store8(const float (&x)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(x[2 * e], x[2 * e + 1]);
    w[e] = *reinterpret_cast<const uint32_t*>(&v);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// A thread owns 8 channels (a 16-byte vector), the lanes of a token lie in one warp.
// FORM 0: interleaved, 4 pairs.
// FORM 1: half layout whose halves are whole vectors: 8 pairs, whose other halves a lane of the same token holds: they come by shuffles.
// FORM 2: half layout otherwise: the partners lie at no fixed place of a vector: they come through shared memory.
// In forms 1 and 2 all lanes of a token have read a row before any of them writes it, so in place is safe.
template <int FORM>
__global__ void __launch_bounds__(ROPE_THREADS, FORM == 2 ? 3 : 4)
rope_kernel(const RopeParams prm, int lanes) {
  __shared__ __align__(16) uint8_t stage[FORM == 2 ? ROPE_HEADS * ROPE_THREADS * 16 : 16];
  const int zero = grid_dep_wait();
  const int tile_chunk = blockIdx.x % prm.chunks;
  const long long tile = blockIdx.x / prm.chunks;
  const int u = threadIdx.x % lanes, c0 = u * 8;
  const long long t = tile * (ROPE_THREADS / lanes) + threadIdx.x / lanes + zero;
  const bool mine = t < prm.tokens && c0 < prm.d;
  const long long b = mine ? t / prm.N : 0, n = mine ? t - b * prm.N : 0;
  const bool is_k = tile_chunk >= prm.q_chunks;
  const int h0 = (is_k ? tile_chunk - prm.q_chunks : tile_chunk) * prm.chunk, h1 = min(h0 + prm.chunk, is_k ? prm.Hk : prm.Hq);
  const Strides si = is_k ? prm.sk : prm.sq, so = is_k ? prm.sko : prm.sqo;
  const uint8_t* src = (is_k ? prm.k : prm.q) + 2 * (b * si.b + n * si.n + c0);
  uint8_t* dst = (is_k ? prm.ko : prm.qo) + 2 * (b * so.b + n * so.n + c0);

  uint4 in[ROPE_HEADS];
  auto load = [&](int h) {
#pragma unroll
    for (int i = 0; i < ROPE_HEADS; ++i) {
      in[i] = make_uint4(0u, 0u, 0u, 0u);
      if (mine && h + i < h1) in[i] = *reinterpret_cast<const uint4*>(src + 2 * (h + i) * si.h);
    }
  };
  load(h0);
  Turn turn[FORM == 0 ? 4 : 8];                           // one per pair, or one per channel
  const int32_t* pos = prm.pos + b * prm.pos_batch + n;
  const unsigned long long* steps = prm.steps + zero;
#pragma unroll
  for (int e = 0; e < (FORM == 0 ? 4 : 8); ++e) {
    const int c = c0 + e;
    if (FORM == 0) {
      turn[e] = mine ? rope_turn(prm, steps, pos, c0 / 2 + e) : Turn{1.f, 0.f};
    } else {
      turn[e] = mine && c < 2 * prm.half ? rope_turn(prm, steps, pos, c < prm.half ? c : c - prm.half) : Turn{1.f, 0.f};
      if (c < prm.half) turn[e].s = -turn[e].s;           // first of a pair: a c - b s; second: b c + a s
    }
  }
  const int words = prm.half - c0 / 2;                    // 4-byte words of the vector that are rotated, if fewer than 4
  // the lane that has the other halves (form 1)
  const int other = c0 < prm.half ? u + prm.half / 8 : c0 < 2 * prm.half ? u - prm.half / 8 : u;
  const int from = (threadIdx.x & 31) - u + other;
  for (int h = h0; h < h1; h += ROPE_HEADS) {
    if (h > h0) load(h);
    if (FORM == 2) {
#pragma unroll
      for (int i = 0; i < ROPE_HEADS; ++i) *reinterpret_cast<uint4*>(stage + (i * ROPE_THREADS + threadIdx.x) * 16) = in[i];
      __syncwarp();
    }
#pragma unroll
    for (int i = 0; i < ROPE_HEADS; ++i) {
      float x[8];
      rope_load8(in[i], x);
      if (FORM == 0) {
#pragma unroll
        for (int e = 0; e < 4; ++e) rope_pair(x[2 * e], x[2 * e + 1], turn[e]);
      } else if (FORM == 1) {
        uint4 w;
        w.x = __shfl_sync(0xffffffffu, in[i].x, from);
        w.y = __shfl_sync(0xffffffffu, in[i].y, from);
        w.z = __shfl_sync(0xffffffffu, in[i].z, from);
        w.w = __shfl_sync(0xffffffffu, in[i].w, from);
        float y[8];
        rope_load8(w, y);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = x[e] * turn[e].c + y[e] * turn[e].s;
      } else {
        // the token's row begins at its first lane's vector
        const __nv_bfloat16* held = reinterpret_cast<const __nv_bfloat16*>(stage + (i * ROPE_THREADS + threadIdx.x - u) * 16);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int c = c0 + e;
          if (c < 2 * prm.half) x[e] = x[e] * turn[e].c + __bfloat162float(held[c < prm.half ? c + prm.half : c - prm.half]) * turn[e].s;
        }
      }
      uint4 o = rope_store8(x);
      if (words < 4) {                                     // what is not rotated keeps its bits
        if (words < 1) o.x = in[i].x;
        if (words < 2) o.y = in[i].y;
        if (words < 3) o.z = in[i].z;
        o.w = in[i].w;
      }
      if (mine && h + i < h1) *reinterpret_cast<uint4*>(dst + 2 * (h + i) * so.h) = o;
    }
    if (FORM == 2) __syncwarp();
  }
}

int launch_rope(const sva_rope_t* p, const void* q, const void* k, const void* steps, const int32_t* positions, void* q_out, void* k_out,
                cudaStream_t st) {
  RopeParams prm;
  prm.q = (const uint8_t*)q; prm.k = (const uint8_t*)k; prm.qo = (uint8_t*)q_out; prm.ko = (uint8_t*)k_out;
  prm.sq = make_strides(p->q_stride); prm.sk = make_strides(p->k_stride);
  prm.sqo = make_strides(p->q_out_stride); prm.sko = make_strides(p->k_out_stride);
  prm.steps = (const unsigned long long*)steps;
  prm.pos = positions;
  prm.pos_axis = p->pos_stride[0]; prm.pos_batch = p->pos_stride[1];
  prm.Hq = p->Hq; prm.Hk = k ? p->Hk : 0; prm.N = p->N; prm.d = p->d; prm.half = p->rotary_dim / 2;
  prm.end0 = p->axis_pairs[0];
  prm.end1 = p->axis_pairs[0] + p->axis_pairs[1];
  prm.tokens = (long long)p->B * p->N;
  prm.factor = p->factor;
  prm.sin_factor = p->inverse ? -p->factor : p->factor;

  const int form = p->layout == SVA_ROPE_INTERLEAVED ? 0 : prm.half % 8 == 0 ? 1 : 2;
  int lanes = 1;
  while (lanes < prm.d / 8) lanes *= 2;
  const long long tiles = (prm.tokens + ROPE_THREADS / lanes - 1) / (ROPE_THREADS / lanes);
  // Heads per CTA: they share the phases, but the grid should come to eight CTAs per SM; fewer than a thread has in flight gain nothing.
  // 2 x 8 191 tokens, 32 + 8 heads: up to 32 heads 56.8 us, up to 16 53.4, but 8 192 tokens x 16 + 16 heads then 28.6 instead of 23.8;
  // 1 024 tokens x 8 + 8: one head per CTA 10.7, four 4.6.
  prm.chunk = 8 * ROPE_HEADS;
  auto ctas = [&](int chunk) { return tiles * ((prm.Hq + chunk - 1) / chunk + (prm.Hk + chunk - 1) / chunk); };
  while (prm.chunk > ROPE_HEADS && ctas(prm.chunk) < 148 * 8) prm.chunk /= 2;
  prm.q_chunks = (prm.Hq + prm.chunk - 1) / prm.chunk;
  prm.chunks = prm.q_chunks + (prm.Hk + prm.chunk - 1) / prm.chunk;
  if (tiles * prm.chunks > 0x7fffffffLL) return SVA_ERR_UNSUPPORTED;
  auto kern = form == 0 ? rope_kernel<0> : form == 1 ? rope_kernel<1> : rope_kernel<2>;
  return launch_dep(kern, dim3((unsigned)(tiles * prm.chunks)), ROPE_THREADS, 0, st, prm, lanes);
}

}  // namespace sva
