// Checks of arguments that the serving operators' entry points share: the config, the tables, pointers, errors.
#pragma once

#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "serve.cuh"

void dllm_set_noctx_error(const char* msg);

namespace dllm {

inline int fail(int code, const char* fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    try {
        dllm_set_noctx_error(buf);
    } catch (...) {  // no memory for the message
    }
    return code;
}

inline int sm_count() {
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    return n;
}

inline bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
// 32-bit values, or null
template <typename... P>
bool words(const P*... p) {
    static_assert(((sizeof(P) == 4) && ...), "");
    return (aligned(p, 4) && ...);
}

// Fills s from cfg; what is wrong with it, or null.
inline const char* shape_of(const dllm_serve_config* c, ServeShape* s) {
    if (!c) return "null config";
    if (c->max_batch < 1 || c->max_batch > kServeMaxBatch) return "max_batch must be 1 to 4096";
    if (c->max_rows < 1 || c->max_rows > 1 << 22) return "max_rows must be 1 to 2^22";
    int lg = 4;
    while (lg < 8 && (1 << lg) != c->page) ++lg;
    if ((1 << lg) != c->page) return "page must be 16, 32, 64, 128 or 256";
    if (c->n_pages < 1 || static_cast<long long>(c->n_pages) * c->page > 0x7fffffffll) return "n_pages * page must be 1 to 2^31 - 1";
    if (c->max_pages < 1 || static_cast<long long>(c->max_pages) * c->page > 0x7fffffffll)
        return "max_pages * page must be 1 to 2^31 - 1";
    if (c->head_dim != 64 && c->head_dim != 128) return "head_dim must be 64 or 128";
    if (c->n_heads < 1 || c->n_kv_heads < 1 || c->n_heads % c->n_kv_heads || c->n_heads / c->n_kv_heads > kServeRows ||
        c->n_heads > 1 << 16)
        return "n_heads must be 1 to 65536, and n_kv_heads divide it in groups of at most 128";
    if (c->dtype != DLLM_BF16 && c->dtype != DLLM_F16) return "dtype must be DLLM_BF16 or DLLM_F16";
    const long long dense = static_cast<long long>(c->n_kv_heads) * c->page * c->head_dim;
    if (c->page_stride != 0 && (c->page_stride < dense || c->page_stride % 8 || c->page_stride >= 1ll << 38))
        return "page_stride must be 0, or a multiple of 8 of at least n_kv_heads * page * head_dim";
    s->max_batch = c->max_batch;
    s->max_rows = c->max_rows;
    s->page = c->page;
    s->page_log2 = lg;
    s->n_pages = c->n_pages;
    s->max_pages = c->max_pages;
    s->H = c->n_heads;
    s->Hkv = c->n_kv_heads;
    s->hd = c->head_dim;
    s->G = c->n_heads / c->n_kv_heads;
    s->tile_tokens = kServeRows / s->G;
    s->dtype = c->dtype;
    s->page_stride = c->page_stride ? c->page_stride : dense;
    s->max_tiles = (c->max_rows + s->tile_tokens - 1) / s->tile_tokens;
    // Blocks of a plan.  No page in two rows of the table: as many as the pool has, and a request's last one may be one key.
    // After a fork each request may see as much as the pool has; of these up to kServeSharedBlocks.
    auto blocks = [&](int pages) { return (static_cast<long long>(pages) * c->page + kServeBlock - 1) / kServeBlock; };
    const long long apart = blocks(c->n_pages) + c->max_batch;
    const long long together = c->max_batch * blocks(c->max_pages < c->n_pages ? c->max_pages : c->n_pages);
    const long long shared = together < kServeSharedBlocks ? together : kServeSharedBlocks;
    s->max_blocks = static_cast<int>(apart > shared ? apart : shared);
    return nullptr;
}

inline bool whole(const dllm_serve_tables* t) {
    return t && t->table && t->held && t->ring && t->ring_pos && t->shared && t->row_start && t->n_keys && t->slot && t->pos && t->req &&
           t->status && t->work && t->partials &&
           words(t->table, t->held, t->ring, t->ring_pos, t->shared, t->row_start, t->n_keys, t->slot, t->pos, t->req, t->status) &&
           aligned(t->work, 16) && aligned(t->partials, 16);
}

// An attention's arguments: what is wrong with them, or null.
inline const char* attention_of(const ServeShape& s, const dllm_serve_tables* t, const void* q, int64_t ldq, const void* kc,
                                const void* vc, const int32_t* prefix_pages, int n_prefix, float scale, void* out, float* lse,
                                int rows, ServeAttnArgs* a) {
    if (!whole(t) || !kc || !vc || (rows > 0 && (!q || !out)) || (n_prefix > 0 && !prefix_pages))
        return "null buffer, or misaligned tables";
    if (rows < 0 || rows > s.max_rows) return "rows must be 0 to max_rows";
    if (n_prefix < 0) return "negative n_prefix";
    if (!(scale > 0.0f) || !std::isfinite(scale)) return "scale must be positive";
    if (ldq < static_cast<int64_t>(s.H) * s.hd || ldq % 8 || ldq >= 1ll << 38)
        return "ldq must be a multiple of 8, and no less than a row";
    for (const void* p : {q, kc, vc, static_cast<const void*>(out)})
        if (!aligned(p, 16)) return "buffers must be 16-byte aligned";
    if (!aligned(out, 32)) return "out must be 32-byte aligned";
    if (!words(prefix_pages, lse)) return "prefix_pages and lse must be 4-byte aligned";
    *a = ServeAttnArgs{q, kc, vc, ldq, prefix_pages, n_prefix, scale, out, lse, rows, nullptr, 0};
    return nullptr;
}

inline int launched(cudaError_t e, const char* what) {
    return e == cudaSuccess ? DLLM_OK : fail(DLLM_ECUDA, "%s launch: %s", what, cudaGetErrorString(e));
}

}  // namespace dllm
