// Attention by the plan's lengths (include/dllm_serve.h, dllm_serve_attention); the kernels: serve_attn.cuh.
#include "serve_attn.cuh"

namespace dllm {

size_t serve_partial_bytes(const ServeShape& s) {
    return static_cast<size_t>(2 * kServeCtas) * kServeRows * (s.hd * sizeof(float) + sizeof(float2));
}

cudaError_t launch_serve_attention(const ServeShape& s, const dllm_serve_tables& t, const ServeAttnArgs& a, int sms,
                                   cudaStream_t st) {
    return go_any<false>(s, t, a, sms, st);
}

}  // namespace dllm
