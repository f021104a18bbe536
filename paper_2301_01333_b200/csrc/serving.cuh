// Declarations shared by the host side (gc_serving.cu) and the kernels of the served attention block.
#pragma once
#include <cuda_bf16.h>
#include <math.h>

#include "gc_internal.h"

namespace gc {

// Status word values of the checks the device makes (the bounded waits use those of ptx.cuh).
enum : uint32_t {
  DEV_BAD_SLOT = 0x201,
  DEV_BAD_PAGE = 0x202,
  DEV_BAD_LENGTH = 0x203,
  DEV_BAD_OFFSETS = 0x204,
  DEV_LARGE_VALUE = 0x205,
  DEV_LARGE_SCORE = 0x206,
};

// Scores times log2(e) above which weights could leave fp32: 2^26 log2(e).  (Exponents are taken relative to a reference rounded to 2^-24
// of itself.  What that is off by, up to 3 binades here and 60 at 2^30, all weights of a row carry as a common factor.)
// Infinite scores are another matter: their rows are NaN.
constexpr float LARGEST_SCORE = 0x1p26f * 1.4426950408889634f;
__device__ __forceinline__ bool score_too_large(float s) { return fabsf(s) > LARGEST_SCORE && fabsf(s) < INFINITY; }

// Launches of this block follow one another closely: each may be set up while the kernel before it on the stream still runs
// (programmatic dependent launch), and every thread of every kernel passes wait_for_predecessor() before it touches global memory
// or returns - also where it has nothing to do: a kernel that ended without waiting would let the one behind it overtake the
// one before it.  A kernel that takes tensor memory lets the next one start only once every one of its blocks has it, with a
// barrier in between: a block of the next kernel could take the columns first, and the two would wait for each other.
__device__ __forceinline__ void wait_for_predecessor() {
  asm volatile("griddepcontrol.launch_dependents;\n\tgriddepcontrol.wait;" ::: "memory");
}
template <typename... P, typename... A>
cudaError_t launch_following(void (*kern)(P...), dim3 grid, int threads, size_t smem, cudaStream_t s, A&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(static_cast<unsigned>(threads));
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, static_cast<P>(args)...);
}

struct Kv4AttnParams {
  int B, n, Hq, Hk, g;              // g: query heads per key/value head; columns of a unit = n * g
  int page_shift, max_len;
  int64_t num_pages, table_stride;
  float c;                          // scale * log2(e)
  int block, ctas;                  // tokens per block (a multiple of 128) of the row of blocks that `ctas` CTAs share out
  int col_chunks;                   // chunks the columns of a (sequence, head) are taken in
  int solo;                         // 1: a warp per (sequence, head, chunk), nothing split
  const __nv_bfloat16* q;
  int64_t qb, qn, qh;
  __nv_bfloat16* o;
  int64_t ob, on, oh;
  const int* table;
  const int* lengths;
  const uint8_t* k_codes;
  const uint32_t* k_params;         // one (lo, scale) pair per word
  const uint8_t* v_codes;
  const uint32_t* v_params;
  float* ws;
  uint32_t* status;
};
// Columns (query, head) one CTA of the kernel for this many columns covers.
int attn_kv4_cols(int columns);
// Resident CTAs per SM the split of the work is planned for.
int attn_kv4_resident(int head_dim, int group, int cols);
cudaError_t launch_attn_kv4(const Kv4AttnParams& p, int head_dim, int group, cudaStream_t s);

struct PromptParams {
  int B, Hq, Hk, D, causal;
  int64_t q_tokens, k_tokens;
  float c;                          // scale * log2(e)
  __nv_bfloat16* o;
  int64_t o_tok, o_head;
  const int* cu_q;
  const int* cu_k;
  uint32_t* status;
};
// tmQ / tmK / tmV: 3-D maps (head dimension, heads, tokens), boxes of 64 x 1 x 128, 128-byte swizzle
cudaError_t launch_attn_prompt(const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV, const PromptParams& p,
                               int num_sms, cudaStream_t s);

cudaError_t launch_qk_norm_rope(const gc_qk_norm_rope_t& d, int num_sms, cudaStream_t s);
cudaError_t launch_kv4_append(const gc_kv4_cache_t& c, int dtype, int64_t tokens, const gc_heads_t& k, const gc_heads_t& v,
                              const int64_t* slots, cudaStream_t s);
cudaError_t launch_kv4_read(const gc_kv4_cache_t& c, int dtype, int64_t tokens, const gc_heads_t& k, const gc_heads_t& v,
                            const int64_t* slots, cudaStream_t s);

}  // namespace gc
