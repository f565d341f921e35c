// Attention whose keys are not its queries' own tokens (sva_cached_attn_fwd, sva_cross_attn_fwd): what the kernels share.
#pragma once
#include "common.cuh"

namespace sva {

// Rows of work: query head hk * group + g of token t is row t * group + g of cached (key) head hk, so that heads which share keys share tiles.
struct KeysParams {
  const uint8_t* q;                         // bf16
  uint8_t* o;
  float* lse;
  Strides sq, so, sk, sv;
  int B, Hq, Hk, group, M, d;
  int causal;
  float scale_log2;                         // softmax_scale * log2(e)
  const int32_t *lengths, *counts;          // may be null
  // bf16 keys: tensors, a mask; cached keys: codes, scales, pages
  const uint8_t *k, *v;
  const float *k_scale, *v_scale;
  const uint8_t* mask;
  long long mask_stride;
  const int32_t* table;
  long long table_stride;
  int S;                                    // keys that there can be: of the tensors, or max_pages * page
  int page, pages, max_pages;
  int32_t* status;
  // a long axis in splits: partial results [split][row of all] (row of all: ((b * Hk + hk) * tiles + tile) * rows per tile + row)
  int splits, tiles;
  float* part_o;
  float2* part_ml;
};

// Queries and keys of a sequence.
__device__ __forceinline__ int seq_keys(const KeysParams& prm, int b) {
  return prm.lengths ? min(max(__ldg(prm.lengths + b), 0), prm.S) : prm.S;
}
__device__ __forceinline__ int seq_queries(const KeysParams& prm, int b) {
  return prm.counts ? min(max(__ldg(prm.counts + b), 0), prm.M) : prm.M;
}
// Cached keys: a sequence that is longer than its table has pages for is reported (by the first CTA; zero: of grid_dep_wait).
__device__ __forceinline__ void report_long(const KeysParams& prm, int zero) {
  if (blockIdx.x != 0 || !prm.status) return;
  for (int b = (int)threadIdx.x + zero; b < prm.B; b += (int)blockDim.x)
    if (__ldg(prm.lengths + b) > prm.S) atomicOr(prm.status, SVA_DEV_BAD_INDEX);
}
// keys that query t of a sequence sees (causal: up to its own position)
__device__ __forceinline__ int keys_seen(const KeysParams& prm, int keys, int queries, int t) {
  return prm.causal ? min(keys, max(keys - queries + t + 1, 0)) : keys;
}
// scales of V as the kernels use them: their logarithm is added to the logits, so that the largest weight of P V is the reference whatever
// the pages' scales are; 2^-80 stands for less (a page of zeros has scale 0)
__device__ __forceinline__ float v_scale_floor(float s) { return s < 8.271806125530277e-25f ? 8.271806125530277e-25f : s; }

int launch_keys_tc(const KeysParams& prm, bool paged, int sms, cudaStream_t st);

}  // namespace sva
