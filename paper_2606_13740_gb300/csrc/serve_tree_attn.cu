// Attention by bits (include/dllm_serve_drafts.h, dllm_serve_tree_attention); the kernels: serve_attn.cuh.
#include "serve_attn.cuh"

namespace dllm {

cudaError_t launch_serve_tree_attention(const ServeShape& s, const dllm_serve_tables& t, const ServeAttnArgs& a, int sms,
                                        cudaStream_t st) {
    return go_any<true>(s, t, a, sms, st);
}

}  // namespace dllm
