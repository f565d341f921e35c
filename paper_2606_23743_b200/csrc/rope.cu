// Rotary positions of Q and K as a call of its own (the fused prologue covers whole heads in the interleaved layout from a table of cosines
// behind an RMS norm; this one rotates what a projection wrote, in either layout, the whole head or a part of it, from integer positions
// on one to three axes, and back again).
//
// Pair j of a token at position p turns by p * theta_j.  theta_j / 2 pi is held as a 64-bit fraction of a turn, step_j; p * step_j
// modulo 2^64 is the phase with whole turns taken off, exactly, for any 32-bit position: an fp32 product p * theta_j would be off by p * 2^-24
// radians (0.06 at a million).  Its upper 32 bits go to fp32 (error 2^-25 turns) and on to sincospif.
//
// HBM-bound: 2 bytes read and 2 written per element.  A thread owns the same channels of one token in several heads, so that
// the phases are made once per token and ROPE_HEADS rows are in flight.  24 + 24 heads of 32 760 tokens 126 us = 6.4 TB/s.
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

// A thread owns 8 channels, the lanes of a token lie in one warp.
// FORM 0: interleaved: a 16-byte vector, 4 pairs.
// FORM 1: half layout whose halves are whole 8-byte pieces: 4 pairs again, from one piece of each half; behind the rotated channels 16 bytes.
// FORM 2: half layout otherwise: a 16-byte vector, whose partners lie at no fixed place of another: they come through shared memory.  All
// lanes of a token have read a row before any of them writes it, so in place is safe (in the other forms a thread writes what it read).  Eight
// phases per thread and the way through shared memory: 24 + 24 heads of 32 760 tokens, 74 of 128 channels 176 us = 4.6 TB/s, 64 channels (form 1) 125.
// Form 1 with 16-byte vectors and the partners by shuffles, twice the phases and half the loads: 2 x 8 191 tokens, 32 + 8 heads of 64 rotated
// channels of 128 61.4 us, so 56.7; 16 + 16 heads of 128, 8 190 tokens, 29.6, so 24.1; one token of
// 8 x (32 + 8) heads 3.9, so 2.7.
template <int FORM>
__global__ void __launch_bounds__(ROPE_THREADS, FORM == 2 ? 3 : 4)
rope_kernel(const RopeParams prm, int lanes) {
  __shared__ __align__(16) uint8_t stage[FORM == 2 ? ROPE_HEADS * ROPE_THREADS * 16 : 16];
  const int zero = grid_dep_wait();
  const int tile_chunk = blockIdx.x % prm.chunks;
  const long long tile = blockIdx.x / prm.chunks;
  const int u = threadIdx.x % lanes;
  const bool split = FORM == 1 && u < prm.half / 4;       // the thread's channels lie in two places
  const int c0 = split ? u * 4 : u * 8, c1 = split ? c0 + prm.half : c0 + 4;          // its first channel, its fifth
  const long long t = tile * (ROPE_THREADS / lanes) + threadIdx.x / lanes + zero;
  const bool mine = t < prm.tokens && u * 8 < prm.d;
  const long long b = mine ? t / prm.N : 0, n = mine ? t - b * prm.N : 0;
  const bool is_k = tile_chunk >= prm.q_chunks;
  const int h0 = (is_k ? tile_chunk - prm.q_chunks : tile_chunk) * prm.chunk, h1 = min(h0 + prm.chunk, is_k ? prm.Hk : prm.Hq);
  const Strides si = is_k ? prm.sk : prm.sq, so = is_k ? prm.sko : prm.sqo;
  const uint8_t* src = (is_k ? prm.k : prm.q) + 2 * (b * si.b + n * si.n + c0);
  uint8_t* dst = (is_k ? prm.ko : prm.qo) + 2 * (b * so.b + n * so.n + c0);

  const int far = 2 * (c1 - c0);                          // bytes

  uint4 in[ROPE_HEADS];
  auto load = [&](int h) {
#pragma unroll
    for (int i = 0; i < ROPE_HEADS; ++i) {
      in[i] = make_uint4(0u, 0u, 0u, 0u);
      if (!mine || h + i >= h1) continue;
      const uint8_t* row = src + 2 * (h + i) * si.h;
      if (FORM == 1) {
        const uint2 a = *reinterpret_cast<const uint2*>(row), b = *reinterpret_cast<const uint2*>(row + far);
        in[i] = make_uint4(a.x, a.y, b.x, b.y);
      } else {
        in[i] = *reinterpret_cast<const uint4*>(row);
      }
    }
  };
  load(h0);
  Turn turn[FORM == 2 ? 8 : 4];                           // one per pair, or one per channel
  const int32_t* pos = prm.pos + b * prm.pos_batch + n;
  const unsigned long long* steps = prm.steps + zero;
#pragma unroll
  for (int e = 0; e < (FORM == 2 ? 8 : 4); ++e) {
    if (FORM == 2) {
      const int c = c0 + e;
      turn[e] = mine && c < 2 * prm.half ? rope_turn(prm, steps, pos, c < prm.half ? c : c - prm.half) : Turn{1.f, 0.f};
      if (c < prm.half) turn[e].s = -turn[e].s;           // first of a pair: a c - b s; second: b c + a s
    } else {
      turn[e] = mine ? rope_turn(prm, steps, pos, 4 * u + e) : Turn{1.f, 0.f};
    }
  }
  const int words = FORM == 1 ? (split ? 4 : 0) : prm.half - c0 / 2;          // 4-byte words of the thread that are rotated, if fewer than 4
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
#pragma unroll
        for (int e = 0; e < 4; ++e) rope_pair(x[e], x[e + 4], turn[e]);
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
      if (!mine || h + i >= h1) continue;
      uint8_t* row = dst + 2 * (h + i) * so.h;
      if (FORM == 1) {
        *reinterpret_cast<uint2*>(row) = make_uint2(o.x, o.y);
        *reinterpret_cast<uint2*>(row + far) = make_uint2(o.z, o.w);
      } else {
        *reinterpret_cast<uint4*>(row) = o;
      }
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

  const int form = p->layout == SVA_ROPE_INTERLEAVED ? 0 : prm.half % 4 == 0 ? 1 : 2;
  int lanes = 1;
  while (lanes < prm.d / 8) lanes *= 2;
  const long long tiles = (prm.tokens + ROPE_THREADS / lanes - 1) / (ROPE_THREADS / lanes);
  // Heads per CTA, which share the phases: equal shares of the heads, of up to 24, or fewer while there are not two CTAs per SM; fewer than a
  // thread has in flight gain nothing.
  // us, up to 32 / 16 / 8 / 4: 2 x 8 191 tokens of 32 + 8 heads 56.9 / 53.1 / 52.7 / 64.4, 4 096 of 40 + 8 18.9 / 17.5 / 17.5 / 21.8, 64 of
  // 32 + 8 7.0 / 4.7 / 3.5 / 2.9; 32 760 of 24 + 24, 24 heads 126.2, 16 128.4, 12 128.0.  Where 16 leave less than two CTAs per SM, them / the
  // rule: 1 000 of 32 + 8 6.4 / 5.7, 2 048 of 24 + 24 10.4 / 8.7, but 1 024 of 16 + 16 4.5 / 5.3.
  const int most = prm.Hq > prm.Hk ? prm.Hq : prm.Hk, shares = most / 24 + (most % 24 != 0);
  auto whole = [](int heads) { return (heads + ROPE_HEADS - 1) / ROPE_HEADS * ROPE_HEADS; };
  prm.chunk = whole(most / shares + (most % shares != 0));
  auto ctas = [&](int chunk) { return tiles * ((prm.Hq + chunk - 1) / chunk + (prm.Hk + chunk - 1) / chunk); };
  while (prm.chunk > ROPE_HEADS && ctas(prm.chunk) < 148 * 2) prm.chunk = whole(prm.chunk / 2);
  prm.q_chunks = (prm.Hq + prm.chunk - 1) / prm.chunk;
  prm.chunks = prm.q_chunks + (prm.Hk + prm.chunk - 1) / prm.chunk;
  if (tiles * prm.chunks > 0x7fffffffLL) return SVA_ERR_UNSUPPORTED;
  note_choice(prm.chunk);
  auto kern = form == 0 ? rope_kernel<0> : form == 1 ? rope_kernel<1> : rope_kernel<2>;
  return launch_dep(kern, dim3((unsigned)(tiles * prm.chunks)), ROPE_THREADS, 0, st, prm, lanes);
}

}  // namespace sva
