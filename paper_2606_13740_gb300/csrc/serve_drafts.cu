// Entry points of the operators for drafts and continuations (include/dllm_serve_drafts.h): argument checks, launches.
#include "serve_args.cuh"

using namespace dllm;

namespace {

// The caches of the layers: what is wrong with them, or null.
const char* caches_of(void* const* kc, void* const* vc, int n_layers, ServeCaches* c) {
    if (!kc || !vc) return "null caches";
    if (n_layers < 1 || n_layers > kServeLayers) return "n_layers must be 1 to 128";
    c->n = n_layers;
    constexpr int kPlaces = 1024;  // of a table by address, to find one that is there twice
    const void* seen[kPlaces] = {};
    for (int i = 0; i < 2 * n_layers; ++i) {
        void* p = i & 1 ? vc[i >> 1] : kc[i >> 1];
        if (!p || !aligned(p, 16)) return "a cache is null, or not 16-byte aligned";
        (i & 1 ? c->v : c->k)[i >> 1] = p;
        size_t at = (reinterpret_cast<uintptr_t>(p) >> 4) * 2654435761u >> 7 & (kPlaces - 1);
        for (; seen[at]; at = (at + 1) & (kPlaces - 1))
            if (seen[at] == p) return "a cache is there twice";
        seen[at] = p;
    }
    return nullptr;
}

}  // namespace

extern "C" {

int dllm_serve_tree(const dllm_serve_config* cfg, const dllm_serve_tables* t, const int32_t* parent, uint32_t* mask, int words_,
                    int rows, void* stream) {
    ServeShape s;
    if (const char* why = shape_of(cfg, &s)) return fail(DLLM_EINVAL, "serve config: %s", why);
    if (!whole(t) || (rows > 0 && (!parent || !mask)) || !words(parent, mask))
        return fail(DLLM_EINVAL, "serve tree: null or misaligned buffer");
    if (rows < 0 || rows > s.max_rows) return fail(DLLM_EINVAL, "serve tree: rows must be 0 to max_rows");
    if (words_ < 1 || words_ > 1024) return fail(DLLM_EINVAL, "serve tree: words must be 1 to 1024");
    if (rows == 0) return DLLM_OK;
    const int sms = sm_count();
    if (sms <= 0) return fail(DLLM_ECUDA, "no CUDA device");
    return launched(launch_serve_tree(s, *t, parent, mask, words_, rows, sms, static_cast<cudaStream_t>(stream)), "serve tree");
}

int dllm_serve_tree_attention(const dllm_serve_config* cfg, const dllm_serve_tables* t, const void* q, int64_t ldq,
                              const void* kc, const void* vc, const int32_t* prefix_pages, int n_prefix, float scale,
                              const uint32_t* mask, int words_, void* out, float* lse, int rows, void* stream) {
    ServeShape s;
    ServeAttnArgs a;
    if (const char* why = shape_of(cfg, &s)) return fail(DLLM_EINVAL, "serve config: %s", why);
    if (const char* why = attention_of(s, t, q, ldq, kc, vc, prefix_pages, n_prefix, scale, out, lse, rows, &a))
        return fail(DLLM_EINVAL, "serve tree attention: %s", why);
    if (words_ < 1 || words_ > 1 << 16) return fail(DLLM_EINVAL, "serve tree attention: words must be 1 to 2^16");
    if ((rows > 0 && !mask) || !words(mask)) return fail(DLLM_EINVAL, "serve tree attention: null or misaligned mask");
    if (rows == 0) return DLLM_OK;
    a.mask = mask;
    a.words = words_;
    const int sms = sm_count();
    if (sms <= 0) return fail(DLLM_ECUDA, "no CUDA device");
    return launched(launch_serve_tree_attention(s, *t, a, sms, static_cast<cudaStream_t>(stream)), "serve tree attention");
}

int dllm_serve_accept(const dllm_serve_config* cfg, const dllm_serve_tables* t, const int32_t* parent, const int32_t* ids,
                      const int32_t* x0, int batch, int rows, int max_len, int32_t* keep, int32_t* n, int32_t* next,
                      void* stream) {
    ServeShape s;
    if (const char* why = shape_of(cfg, &s)) return fail(DLLM_EINVAL, "serve config: %s", why);
    if (!whole(t) || (rows > 0 && (!parent || !ids || !x0)) || !keep || !n || !next || !words(parent, ids, x0, keep, n, next))
        return fail(DLLM_EINVAL, "serve accept: null or misaligned buffer");
    if (batch < 1 || batch > s.max_batch) return fail(DLLM_EINVAL, "serve accept: batch must be 1 to max_batch");
    if (rows < 0 || rows > s.max_rows) return fail(DLLM_EINVAL, "serve accept: rows must be 0 to max_rows");
    if (max_len < 1 || max_len > 1 << 22) return fail(DLLM_EINVAL, "serve accept: max_len must be 1 to 2^22");
    const ServeAcceptArgs a{parent, ids, x0, batch, rows, max_len, keep, n, next};
    return launched(launch_serve_accept(s, *t, a, static_cast<cudaStream_t>(stream)), "serve accept");
}

int dllm_serve_compact(const dllm_serve_config* cfg, const dllm_serve_tables* t, void* const* kc, void* const* vc, int n_layers,
                       const int32_t* first, const int32_t* keep, int keep_ld, const int32_t* n, int batch, void* stream) {
    ServeShape s;
    ServeCaches c;
    if (const char* why = shape_of(cfg, &s)) return fail(DLLM_EINVAL, "serve config: %s", why);
    if (!whole(t) || !first || (keep_ld > 0 && !keep) || !n || !words(first, keep, n)) return fail(DLLM_EINVAL, "serve compact: null or misaligned buffer");
    if (const char* why = caches_of(kc, vc, n_layers, &c)) return fail(DLLM_EINVAL, "serve compact: %s", why);
    if (batch < 1 || batch > s.max_batch) return fail(DLLM_EINVAL, "serve compact: batch must be 1 to max_batch");
    if (keep_ld < 0) return fail(DLLM_EINVAL, "serve compact: negative keep_ld");
    const int sms = sm_count();
    if (sms <= 0) return fail(DLLM_ECUDA, "no CUDA device");
    const ServeCompactArgs a{first, keep, n, keep_ld, batch};
    return launched(launch_serve_compact(s, *t, c, a, sms, static_cast<cudaStream_t>(stream)), "serve compact");
}

int dllm_serve_fork(const dllm_serve_config* cfg, const dllm_serve_tables* t, void* const* kc, void* const* vc, int n_layers,
                    const int32_t* src, const int32_t* len, int batch, void* stream) {
    ServeShape s;
    ServeCaches c;
    if (const char* why = shape_of(cfg, &s)) return fail(DLLM_EINVAL, "serve config: %s", why);
    if (!whole(t) || !src || !len || !words(src, len)) return fail(DLLM_EINVAL, "serve fork: null or misaligned buffer");
    if (const char* why = caches_of(kc, vc, n_layers, &c)) return fail(DLLM_EINVAL, "serve fork: %s", why);
    if (batch < 1 || batch > s.max_batch) return fail(DLLM_EINVAL, "serve fork: batch must be 1 to max_batch");
    const int sms = sm_count();
    if (sms <= 0) return fail(DLLM_ECUDA, "no CUDA device");
    return launched(launch_serve_fork(s, *t, c, src, len, batch, sms, static_cast<cudaStream_t>(stream)), "serve fork");
}

int dllm_serve_logprobs(const dllm_serve_logprobs_args* a, void* stream) {
    if (!a || (a->rows > 0 && !a->logits)) return fail(DLLM_EINVAL, "serve logprobs: null buffer");
    if (a->rows < 0 || a->vocab < 1 || a->vocab > 1 << 28) return fail(DLLM_EINVAL, "serve logprobs: bad sizes");
    if (a->ld < a->vocab) return fail(DLLM_EINVAL, "serve logprobs: a row is shorter than the vocabulary");
    if (a->dtype != DLLM_F32 && a->dtype != DLLM_BF16 && a->dtype != DLLM_F16) return fail(DLLM_EINVAL, "serve logprobs: unknown dtype");
    if (a->mask_id < -1 || a->mask_id >= a->vocab) return fail(DLLM_EINVAL, "serve logprobs: mask_id outside the vocabulary");
    if (!aligned(a->logits, a->dtype == DLLM_F32 ? 4 : 2) || !words(a->tokens, a->lp, a->entropy, a->lse, a->top_ids, a->top_lp))
        return fail(DLLM_EINVAL, "serve logprobs: misaligned buffer");
    if (a->n_tokens < 0 || a->n_tokens > 1 << 20 || a->n_top < 0 || a->n_top > 32)
        return fail(DLLM_EINVAL, "serve logprobs: n_tokens must be 0 to 2^20, n_top 0 to 32");
    if (a->rows == 0) return DLLM_OK;
    if ((a->n_tokens && (!a->tokens || !a->lp)) || (a->n_top && (!a->top_ids || !a->top_lp)))
        return fail(DLLM_EINVAL, "serve logprobs: tokens come with lp, n_top with top_ids and top_lp");
    if (!a->n_tokens && !a->n_top && !a->lse && !a->entropy) return fail(DLLM_EINVAL, "serve logprobs: nothing to write");
    const int sms = sm_count();
    if (sms <= 0) return fail(DLLM_ECUDA, "no CUDA device");
    return launched(launch_serve_logprobs(*a, sms, static_cast<cudaStream_t>(stream)), "serve logprobs");
}

}  // extern "C"
