// Host-only argument checks of the libspecfp8 C ABI.  No HIP here: every
// check runs before anything is enqueued, so argument errors never touch the
// device (and can be exercised on a machine without a GPU).
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "../../include/spec_fp8.h"

namespace specfp8 {

spec_status check_quantize(const void* x, int64_t rows, int64_t cols, int64_t ld_x, int in_kind, int mode,
                           const float* scales, const void* q, int64_t ld_q);
spec_status check_silu_mul(const void* x, int64_t rows, int64_t cols, int64_t ld_x, const void* h,
                           int64_t ld_h);
spec_status check_clip_count(const void* x, int64_t rows, int64_t cols, int64_t ld_x, const float* scale,
                             const void* count);
spec_status check_gemm(const void* a, int64_t lda, const float* a_scale, int a_mode, const void* w,
                       int64_t ldw, const float* w_scale, int w_mode, int64_t M, int64_t N, int64_t K,
                       const void* y, int64_t ldy, int out_dtype);
spec_status check_kv_cache_write(const void* k, int64_t ld_k, const void* v, int64_t ld_v,
                                 const int64_t* slot_mapping, int64_t T, int64_t H, int64_t D, int64_t num_slots,
                                 int mode, const float* k_scale, const float* v_scale, const void* k_cache,
                                 const void* v_cache);
spec_status check_rms_norm(const void* x, int64_t ld_x, const void* residual, int64_t ld_residual, const void* weight,
                           float eps, int64_t rows, int64_t cols, int mode, const float* scales, const void* q,
                           int64_t ld_q, const void* sum, int64_t ld_sum, const void* y, int64_t ld_y);
spec_status check_rope_kv_cache_write(const void* q, int64_t ld_q, const void* k, int64_t ld_k, const void* v,
                                      int64_t ld_v, const int32_t* positions, const double* inv_freq, int64_t R,
                                      int pairs, const int64_t* slot_mapping, int64_t T, int64_t Hq, int64_t H,
                                      int64_t D, int64_t num_slots, int mode, const float* k_scale,
                                      const float* v_scale, const void* k_cache, const void* v_cache,
                                      const void* q_out, int64_t ld_q_out, const void* k_out, int64_t ld_k_out);
spec_status check_fp4_quantize(const void* x, int64_t rows, int64_t cols, int64_t ld_x, const void* q, int64_t ld_q,
                               const void* scales, int64_t ld_scales);
spec_status check_gemm_fp4(const void* a, int64_t lda, const float* a_scale, int a_mode, const void* w, int64_t ldw,
                           const void* w_scale, int64_t ld_w_scale, int64_t M, int64_t N, int64_t K, const void* y,
                           int64_t ldy, int out_dtype);
spec_status check_kv_cache_read(const void* k_cache, const void* v_cache, const float* k_scale, const float* v_scale,
                                int mode, const int64_t* slot_mapping, int64_t T, int64_t H, int64_t D,
                                int64_t num_slots, const void* k, int64_t ld_k, const void* v, int64_t ld_v);
spec_status check_paged_attention(const void* q, int64_t ld_q, const void* k_cache, const void* v_cache,
                                  const float* k_scale, const float* v_scale, int mode, const int32_t* block_tables,
                                  int64_t ld_tables, int64_t max_blocks, const int32_t* kv_lens, const int32_t* cu_q,
                                  const uint64_t* tree_mask, int64_t N, int64_t T, int64_t B, int64_t Hq, int64_t H,
                                  int64_t D, int64_t block_size, int64_t num_blocks, float scale, const void* out,
                                  int64_t ld_out);
spec_status check_prompt_attention(const void* q, int64_t ld_q, const void* k, int64_t ld_k, const void* v,
                                   int64_t ld_v, const int32_t* cu_seqlens, int64_t T, int64_t B, int64_t Hq,
                                   int64_t H, int64_t D, float scale, const void* out, int64_t ld_out);
spec_status check_logit_stats(int64_t M, int64_t V, float temperature, const void* logits, int64_t ld_logits,
                              const float* stats, int64_t ld_stats, int64_t n_groups);
spec_status check_accept_stats(const float* target_stats, int64_t n_stats, int64_t ld_stats, int64_t B);
spec_status check_accept_tree(const void* target_logits, const int32_t* parents, const int32_t* tokens,
                              const float* uniforms, int64_t B, int64_t N, int64_t V, float temperature,
                              const int32_t* out_tokens, const int32_t* accepted_nodes,
                              const int32_t* num_accepted);
spec_status check_tree_mask(const int32_t* parents, int64_t B, int64_t N, const uint64_t* mask,
                            const int32_t* depth);
spec_status check_accept(const void* target_logits, const void* draft_logits, const int32_t* draft_tokens,
                         const float* uniforms, int64_t B, int64_t k, int64_t V, float temperature,
                         const int32_t* out_tokens, const int32_t* num_accepted);

}  // namespace specfp8
