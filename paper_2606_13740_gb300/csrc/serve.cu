// Entry points of the serving operators (include/dllm_serve.h): argument checks, buffer layout, launches.
#include "serve_args.cuh"

using namespace dllm;

extern "C" {

int dllm_serve_layout(const dllm_serve_config* cfg, void* mem, dllm_serve_tables* out, size_t* bytes) {
    ServeShape s;
    if (const char* why = shape_of(cfg, &s)) return fail(DLLM_EINVAL, "serve config: %s", why);
    if (mem && !aligned(mem, 16)) return fail(DLLM_EINVAL, "serve buffers must be 16-byte aligned");
    size_t at = 0;
    auto take = [&](size_t n) {
        char* p = mem ? static_cast<char*>(mem) + at : nullptr;
        at += serve_round(n);
        return p;
    };
    const size_t B = s.max_batch, R = s.max_rows;
    dllm_serve_tables t;
    t.table = reinterpret_cast<int32_t*>(take(B * s.max_pages * 4));
    t.held = reinterpret_cast<int32_t*>(take(B * 4));
    t.ring = reinterpret_cast<int32_t*>(take(static_cast<size_t>(s.n_pages) * 4));
    t.ring_pos = reinterpret_cast<int32_t*>(take(8));
    t.shared = reinterpret_cast<int32_t*>(take(B * 4));
    t.row_start = reinterpret_cast<int32_t*>(take((B + 1) * 4));
    t.n_keys = reinterpret_cast<int32_t*>(take(B * 4));
    t.slot = reinterpret_cast<int32_t*>(take(R * 4));
    t.pos = reinterpret_cast<int32_t*>(take(R * 4));
    t.req = reinterpret_cast<int32_t*>(take(R * 4));
    t.status = reinterpret_cast<int32_t*>(take(16));
    t.work = reinterpret_cast<int32_t*>(take(serve_arrays(s, nullptr, nullptr)));
    const size_t attn = serve_partial_bytes(s), fork = serve_fork_bytes(s);
    t.partials = reinterpret_cast<float*>(take(attn > fork ? attn : fork));
    if (out) *out = t;
    if (bytes) *bytes = at;
    return DLLM_OK;
}

int dllm_serve_reset(const dllm_serve_config* cfg, const dllm_serve_tables* t, void* stream) {
    ServeShape s;
    if (const char* why = shape_of(cfg, &s)) return fail(DLLM_EINVAL, "serve config: %s", why);
    if (!whole(t)) return fail(DLLM_EINVAL, "serve tables: null or misaligned buffer");
    return launched(launch_serve_reset(s, *t, static_cast<cudaStream_t>(stream)), "serve reset");
}

int dllm_serve_plan(const dllm_serve_config* cfg, const dllm_serve_tables* t, const int32_t* len, const int32_t* q_len,
                    int batch, int rows, int prefix_len, int causal, void* stream) {
    ServeShape s;
    if (const char* why = shape_of(cfg, &s)) return fail(DLLM_EINVAL, "serve config: %s", why);
    if (!whole(t) || !len || !q_len || !words(len, q_len)) return fail(DLLM_EINVAL, "serve plan: null or misaligned buffer");
    if (batch < 1 || batch > s.max_batch) return fail(DLLM_EINVAL, "serve plan: batch must be 1 to max_batch");
    if (rows < 0 || rows > s.max_rows) return fail(DLLM_EINVAL, "serve plan: rows must be 0 to max_rows");
    if (prefix_len < 0 || prefix_len > 0x3fffffff) return fail(DLLM_EINVAL, "serve plan: prefix_len must be 0 to 2^30 - 1");
    const int sms = sm_count();
    if (sms <= 0) return fail(DLLM_ECUDA, "no CUDA device");
    return launched(launch_serve_plan(s, *t, len, q_len, batch, rows, prefix_len, causal != 0, sms,
                                      static_cast<cudaStream_t>(stream)),
                    "serve plan");
}

int dllm_serve_qk_norm_rope(const dllm_serve_config* cfg, const dllm_serve_tables* t, const void* q, const void* k,
                            const void* v, int in_dtype, int64_t ldq, int64_t ldk, int64_t ldv, const float* q_gain,
                            const float* k_gain, float eps, const float* theta, void* q_out, int64_t ld_out, void* kc,
                            void* vc, int rows, void* stream) {
    ServeShape s;
    if (const char* why = shape_of(cfg, &s)) return fail(DLLM_EINVAL, "serve config: %s", why);
    if (!whole(t) || !theta || !kc || !vc || (rows > 0 && (!q || !k || !v || !q_out)))
        return fail(DLLM_EINVAL, "qk_norm_rope: null buffer, or misaligned tables");
    if (in_dtype != s.dtype && in_dtype != DLLM_F32)
        return fail(DLLM_EINVAL, "qk_norm_rope: in_dtype must be the config's dtype or DLLM_F32");
    if (rows < 0 || rows > s.max_rows) return fail(DLLM_EINVAL, "qk_norm_rope: rows must be 0 to max_rows");
    if (!(eps >= 0.0f)) return fail(DLLM_EINVAL, "qk_norm_rope: eps must not be negative");
    const int64_t qd = static_cast<int64_t>(s.H) * s.hd, kvd = static_cast<int64_t>(s.Hkv) * s.hd;
    if (ldq < qd || ldk < kvd || ldv < kvd || ld_out < qd || (ldq | ldk | ldv | ld_out) % 8)
        return fail(DLLM_EINVAL, "qk_norm_rope: strides must be multiples of 8, and no less than a row");
    for (const void* p : {q, k, v, static_cast<const void*>(q_out), static_cast<const void*>(kc), static_cast<const void*>(vc)})
        if (!aligned(p, 16)) return fail(DLLM_EINVAL, "qk_norm_rope: buffers must be 16-byte aligned");
    if (!aligned(q_gain, 16) || !aligned(k_gain, 16) || !aligned(theta, 4))
        return fail(DLLM_EINVAL, "qk_norm_rope: gains must be 16-byte aligned");
    if (q_out == q && (in_dtype != s.dtype || ldq != ld_out))
        return fail(DLLM_EINVAL, "qk_norm_rope: in place, q_out has q's type and stride");
    if (rows == 0) return DLLM_OK;
    const int sms = sm_count();
    if (sms <= 0) return fail(DLLM_ECUDA, "no CUDA device");
    const ServeNormArgs a{q, k, v, ldq, ldk, ldv, ld_out, q_gain, k_gain, theta, eps, q_out, kc, vc, t->slot, t->pos, t->status, rows};
    return launched(launch_serve_norm(s, a, in_dtype, sms, static_cast<cudaStream_t>(stream)), "qk_norm_rope");
}

int dllm_serve_attention(const dllm_serve_config* cfg, const dllm_serve_tables* t, const void* q, int64_t ldq,
                         const void* kc, const void* vc, const int32_t* prefix_pages, int n_prefix, float scale,
                         void* out, float* lse, int rows, void* stream) {
    ServeShape s;
    ServeAttnArgs a;
    if (const char* why = shape_of(cfg, &s)) return fail(DLLM_EINVAL, "serve config: %s", why);
    if (const char* why = attention_of(s, t, q, ldq, kc, vc, prefix_pages, n_prefix, scale, out, lse, rows, &a))
        return fail(DLLM_EINVAL, "serve attention: %s", why);
    if (rows == 0) return DLLM_OK;
    const int sms = sm_count();
    if (sms <= 0) return fail(DLLM_ECUDA, "no CUDA device");
    return launched(launch_serve_attention(s, *t, a, sms, static_cast<cudaStream_t>(stream)), "serve attention");
}

int dllm_serve_check(const dllm_serve_tables* t, int* bits, void* stream) {
    if (!t || !t->status) return fail(DLLM_EINVAL, "serve check: null buffer");
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int b = 0;
    cudaError_t e = cudaMemcpyAsync(&b, t->status, 4, cudaMemcpyDeviceToHost, st);
    if (e == cudaSuccess) e = cudaMemsetAsync(t->status, 0, 4, st);
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    if (e != cudaSuccess) return fail(DLLM_ECUDA, "serve check: %s", cudaGetErrorString(e));
    if (bits) *bits = b;
    if (b & DLLM_SERVE_TIMEOUT) return fail(DLLM_ETIMEOUT, "bounded device wait ran out");
    if (b & DLLM_SERVE_PAGES) return fail(DLLM_ECAPACITY, "the pool of pages ran out (status bits %d)", b);
    if (b) return fail(DLLM_EINVAL, "serve status bits %d", b);
    return DLLM_OK;
}

int dllm_serve_logits_bytes(int rows, int vocab, size_t* bytes) {
    if (!bytes || rows < 0 || vocab < 1 || vocab > 1 << 28) return fail(DLLM_EINVAL, "serve logits: bad sizes");
    *bytes = serve_logits_bytes(rows, vocab);
    return DLLM_OK;
}

int dllm_serve_logits(const dllm_serve_logits_args* a, void* stream) {
    if (!a || (a->rows > 0 && !a->logits)) return fail(DLLM_EINVAL, "serve logits: null buffer");
    if (a->rows < 0 || a->vocab < 1 || a->vocab > 1 << 28) return fail(DLLM_EINVAL, "serve logits: bad sizes");
    if (a->ld < a->vocab || (a->out && a->ld_out < a->vocab)) return fail(DLLM_EINVAL, "serve logits: a row is shorter than the vocabulary");
    if (a->dtype != DLLM_F32 && a->dtype != DLLM_BF16 && a->dtype != DLLM_F16) return fail(DLLM_EINVAL, "serve logits: unknown dtype");
    if (a->mask_id < -1 || a->mask_id >= a->vocab) return fail(DLLM_EINVAL, "serve logits: mask_id outside the vocabulary");
    const size_t size = a->dtype == DLLM_F32 ? 4 : 2;
    if (!aligned(a->logits, size) || !aligned(a->out, size) ||
        !words(a->req, a->hist, a->hist_len, a->rep, a->freq, a->pres, a->bias_ids, a->bias, a->bias_len, a->grammar,
               a->grammar_row, a->cur, a->x0, a->conf, a->tokconf))
        return fail(DLLM_EINVAL, "serve logits: misaligned buffer");
    if (a->out && a->out == a->logits && a->ld_out != a->ld) return fail(DLLM_EINVAL, "serve logits: in place, ld_out is ld");
    if ((a->hist || a->bias_ids) && a->n_req < 1) return fail(DLLM_EINVAL, "serve logits: n_req must be positive");
    if (a->hist && (a->hist_ld < 0 || a->hist_ld >= 1 << 20)) return fail(DLLM_EINVAL, "serve logits: hist_ld must be below 2^20");
    if (a->bias_ids && (!a->bias || a->bias_ld < 0 || a->bias_ld >= 4096))
        return fail(DLLM_EINVAL, "serve logits: bias_ids come with bias, bias_ld below 4096");
    if (a->grammar && (!a->grammar_row || a->n_grammar < 0)) return fail(DLLM_EINVAL, "serve logits: grammar comes with grammar_row");
    if (a->tokconf && !a->cur) return fail(DLLM_EINVAL, "serve logits: tokconf comes with cur");
    if (a->rows == 0) return DLLM_OK;
    if (!a->out && !a->x0 && !a->conf && !a->tokconf) return fail(DLLM_EINVAL, "serve logits: nothing to write");
    if (!a->ws || !aligned(a->ws, 16) || a->ws_bytes < serve_logits_bytes(a->rows, a->vocab))
        return fail(DLLM_EINVAL, "serve logits: workspace missing, misaligned or too small");
    const int sms = sm_count();
    if (sms <= 0) return fail(DLLM_ECUDA, "no CUDA device");
    return launched(launch_serve_logits(*a, sms, static_cast<cudaStream_t>(stream)), "serve logits");
}

}  // extern "C"
