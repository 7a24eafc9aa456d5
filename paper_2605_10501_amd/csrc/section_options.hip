// Sections with options: the entry points, and the table of what the executor (section.hip) calls for them.
#include "launch.h"

namespace {
const SectionOps kOps = {ms_k_embedding_scaled_forward, ms_k_embedding_sorted_backward, ms_k_embedding_sorted_backward_scratch_bytes,
                         ms_k_qk_norm_rope_forward, ms_k_qk_norm_rope_backward, ms_k_qk_norm_rope_backward_scratch_bytes,
                         ms_k_norm_fp8, ms_k_fp8_quantize, ms_k_gemm_fp8, ms_k_gemm_fp8_swiglu, ms_k_gemm_fp8_swiglu_scratch_bytes,
                         ms_k_swiglu_fp8};
}

extern "C" size_t ms_section_workspace_bytes_with(const ms_section_config *cfg, const ms_section_options *options, int32_t max_tokens,
                                                  int32_t max_seqlen, int32_t need_backward) {
    const SectionOptions o = {options, nullptr, &kOps};
    return section_workspace(cfg, options ? &o : nullptr, max_tokens, max_seqlen, need_backward != 0);
}

extern "C" ms_status ms_section_forward_with(const ms_section_config *cfg, const ms_section_options *options, const ms_section_ptrs *weights,
                                             const ms_batch *batch, const void *x_in, void *h_out, void *workspace_dev, size_t workspace_bytes,
                                             void *stream) {
    const SectionOptions o = {options, nullptr, &kOps};
    return section_forward(cfg, options ? &o : nullptr, weights, batch, x_in, h_out, workspace_dev, workspace_bytes, stream);
}

extern "C" ms_status ms_section_forward_backward_with(const ms_section_config *cfg, const ms_section_options *options,
                                                      const ms_layer_options *option_grads, const ms_section_ptrs *weights,
                                                      const ms_section_ptrs *grads, const ms_batch *batch, const void *x_in, void *h_out,
                                                      const void *d_h_out, const ms_kd_config *kd, const void *h_teacher, void *d_w_student,
                                                      float *loss_dev, float *kl_per_token_dev, void *d_x_in, void *workspace_dev,
                                                      size_t workspace_bytes, void *stream) {
    const SectionOptions o = {options, option_grads, &kOps};
    return section_forward_backward(cfg, options ? &o : nullptr, weights, grads, batch, x_in, h_out, d_h_out, kd, h_teacher, d_w_student, loss_dev,
                                    kl_per_token_dev, d_x_in, workspace_dev, workspace_bytes, stream);
}
