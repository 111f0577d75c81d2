// What the serving operators (include/dllm_serve.h) share: the config in the form the kernels take, and
// the layout of the attention's work list, which the plan writes and the attention reads.
#pragma once

#include <cuda_fp16.h>

#include "../../include/dllm.h"
#include "../../include/dllm_serve_drafts.h"
#include "common.cuh"
#include "internal.h"

namespace dllm {

constexpr int kServeMaxBatch = 4096;
constexpr int kServeBlock = 64;    // keys of a block of the work list
constexpr int kServeRows = 128;    // query rows of an attention tile (UMMA M)
constexpr int kServeSharedBlocks = 1 << 22;  // of a plan whose requests share pages (2^28 keys, 128 MB of the work list)
constexpr int kServeCtas = 320;    // CTAs that the attention's work is cut for, at most: two on each of 160 SMs

// A config with its defaults filled in.
struct ServeShape {
    int max_batch, max_rows, page, page_log2, n_pages, max_pages;
    int H, Hkv, hd, G;       // G: query heads of a K/V head
    int tile_tokens;         // tokens of an attention tile: kServeRows / G, their G heads side by side
    int dtype;
    long long page_stride;
    int max_tiles, max_blocks;
};

// The work list.  Rows (token, query head of the group) of a K/V head are cut into tiles of tile_tokens
// tokens; tile x K/V head is a unit.  A unit's keys are steps of up to 64: the prefix's blocks, then the
// own blocks of the requests that have rows in the tile, which stand side by side in the block arrays.
// All units' steps in order (tile, head, step) are cut into `ctas` runs of equal cost, one a CTA.
struct ServeWork {
    int ticket;          // CTAs of a plan that have read the state
    int ctas;
    int causal;
    int prefix_len;
    int prefix_blocks;
    int tiles;
    int rows;            // new tokens covered
    int joins;           // units that several CTAs share
    long long total;     // steps of all units
    int shape[6];        // what the list was made for (serve_same_shape)
    int batch;           // requests of the plan
    int pad[3];
};
static_assert(sizeof(ServeWork) % 16 == 0, "the arrays behind it are 16-byte aligned");

// Whether a work list was made for this config (calls with another one find its arrays elsewhere, or want larger
// partials behind it).
__host__ __device__ inline void serve_key(const ServeShape& s, int* key) {
    key[0] = s.Hkv;
    key[1] = s.G;
    key[2] = s.page;
    key[3] = s.max_tiles;
    key[4] = s.max_blocks;
    key[5] = s.hd;
}
__device__ inline bool serve_same_shape(const ServeShape& s, const ServeWork& w) {
    int key[6];
    serve_key(s, key);
    bool same = true;
    for (int i = 0; i < 6; ++i) same = same && key[i] == w.shape[i];
    return same;
}

struct ServeArrays {
    ServeWork* head;
    int* left_out;        // [kServeMaxBatch]: whether dllm_serve_tree has found a request's tree wrong since the plan
    int4* join;           // [joins]: the unit's tile and K/V head, the first and the last CTA that holds a part of it
    int4* cta;            // [kServeCtas][2]: tile, K/V head, step within the unit, number of steps; the tile's entry
    int4* info;           // [max_blocks]: first and last + 1 row of the request, the block's first key, n_keys - rows
    int4* pages;          // [max_blocks]: up to four pages (page < 64), or page and first place in it
    int2* tile;           // [max_tiles]: its first own block, its steps
};

__host__ __device__ inline size_t serve_round(size_t n) { return (n + 255) / 256 * 256; }

// Carves the work list; null base: sizes only.
__host__ __device__ inline size_t serve_arrays(const ServeShape& s, void* base, ServeArrays* out) {
    size_t at = 0;
    char* b = static_cast<char*>(base);
    ServeArrays r;
    r.head = reinterpret_cast<ServeWork*>(b + at);
    at += serve_round(sizeof(ServeWork));
    r.left_out = reinterpret_cast<int*>(b + at);
    at += serve_round(sizeof(int) * kServeMaxBatch);
    r.join = reinterpret_cast<int4*>(b + at);
    at += serve_round(sizeof(int4) * kServeCtas);
    r.cta = reinterpret_cast<int4*>(b + at);
    at += serve_round(sizeof(int4) * 2 * kServeCtas);
    r.info = reinterpret_cast<int4*>(b + at);
    at += serve_round(sizeof(int4) * s.max_blocks);
    r.pages = reinterpret_cast<int4*>(b + at);
    at += serve_round(sizeof(int4) * s.max_blocks);
    r.tile = reinterpret_cast<int2*>(b + at);
    at += serve_round(sizeof(int2) * s.max_tiles);
    if (out) *out = r;
    return at;
}

// The 16-bit types of the cache.
template <typename T>
struct Half2;
template <>
struct Half2<__nv_bfloat16> {
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<uint32_t*>(&v);
    }
    static __device__ __forceinline__ float2 unpack(uint32_t u) {
        return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
    }
};
template <>
struct Half2<__half> {
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        __half2 v = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<uint32_t*>(&v);
    }
    static __device__ __forceinline__ float2 unpack(uint32_t u) { return __half22float2(*reinterpret_cast<__half2*>(&u)); }
};

// A launch that begins while the one before it in the stream ends: the kernel calls pdl_wait before it reads or
// writes anything that another launch may have to do with.
template <typename... P, typename... A>
cudaError_t serve_launch(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, A... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}

cudaError_t launch_serve_reset(const ServeShape& s, const dllm_serve_tables& t, cudaStream_t st);
cudaError_t launch_serve_plan(const ServeShape& s, const dllm_serve_tables& t, const int* len, const int* q_len,
                              int batch, int rows, int prefix_len, int causal, int sms, cudaStream_t st);
struct ServeNormArgs {
    const void *q, *k, *v;
    long long ldq, ldk, ldv, ld_out;
    const float *q_gain, *k_gain, *theta;
    float eps;
    void *q_out, *kc, *vc;
    const int *slot, *pos;
    int* status;
    int rows;
};
cudaError_t launch_serve_norm(const ServeShape& s, const ServeNormArgs& a, int in_dtype, int sms, cudaStream_t st);
struct ServeAttnArgs {
    const void *q, *kc, *vc;
    long long ldq;
    const int* prefix_pages;
    int n_prefix;
    float scale;
    void* out;
    float* lse;
    int rows;
    const uint32_t* mask;  // [rows][words]: new tokens that a row sees (null: by the plan's causal)
    int words;
};
cudaError_t launch_serve_attention(const ServeShape& s, const dllm_serve_tables& t, const ServeAttnArgs& a, int sms,
                                   cudaStream_t st);
cudaError_t launch_serve_tree_attention(const ServeShape& s, const dllm_serve_tables& t, const ServeAttnArgs& a, int sms,
                                        cudaStream_t st);
size_t serve_partial_bytes(const ServeShape& s);
size_t serve_logits_bytes(int rows, int vocab);
cudaError_t launch_serve_logits(const dllm_serve_logits_args& a, int sms, cudaStream_t st);
cudaError_t launch_serve_tree(const ServeShape& s, const dllm_serve_tables& t, const int* parent, uint32_t* mask, int words,
                              int rows, int sms, cudaStream_t st);
struct ServeAcceptArgs {
    const int *parent, *ids, *x0;
    int batch, rows, max_len;
    int *keep, *n, *next;
};
cudaError_t launch_serve_accept(const ServeShape& s, const dllm_serve_tables& t, const ServeAcceptArgs& a, cudaStream_t st);
// The caches of a model's layers.
constexpr int kServeLayers = 128;
struct ServeCaches {
    void *k[kServeLayers], *v[kServeLayers];
    int n;
};
struct ServeCompactArgs {
    const int *first, *keep, *n;
    int keep_ld, batch;
};
cudaError_t launch_serve_compact(const ServeShape& s, const dllm_serve_tables& t, const ServeCaches& c,
                                 const ServeCompactArgs& a, int sms, cudaStream_t st);
size_t serve_fork_bytes(const ServeShape& s);  // of the tables' partials
cudaError_t launch_serve_fork(const ServeShape& s, const dllm_serve_tables& t, const ServeCaches& c, const int* src,
                              const int* len, int batch, int sms, cudaStream_t st);
cudaError_t launch_serve_logprobs(const dllm_serve_logprobs_args& a, int sms, cudaStream_t st);

}  // namespace dllm
