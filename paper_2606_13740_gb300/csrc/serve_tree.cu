// Trees of drafted tokens (include/dllm_serve_drafts.h): who sees whom from the parents (dllm_serve_tree), and the path
// that the decisions bear out (dllm_serve_accept).
#include "serve.cuh"

namespace dllm {

namespace {

constexpr int kThreads = 128;
constexpr int kStaged = 2048;  // parents of a tree held in shared memory; those past them are read from the cache

// The rows of request b that there are.
__device__ __forceinline__ int2 rows_of(const dllm_serve_tables& t, int b, int rows) {
    const int r0 = t.row_start[b], r1 = t.row_start[b + 1];
    const int lo = min(max(r0, 0), rows);
    return make_int2(lo, min(max(r1, lo), rows));
}

// A CTA takes a request, a thread its tokens: from each it walks to the root, which numbers the bits downwards, so that
// a row's words are made one by one and written once.  Bound: latency, of the plan's row starts, the parents and
// the walk (a load from shared memory a step).  Measured in a graph: a tree of 26 2.5 us, 800 trees of up to 64 4.8.
__global__ void __launch_bounds__(kThreads) k_serve_tree(const __grid_constant__ ServeShape s,
                                                         const __grid_constant__ dllm_serve_tables t, const int* parent,
                                                         uint32_t* mask, int words, int rows) {
    __shared__ int staged[kStaged];
    ServeArrays w;
    serve_arrays(s, t.work, &w);
    pdl_wait();
    pdl_launch_dependents();
    const bool same = serve_same_shape(s, *w.head);
    const int batch = same ? min(w.head->batch, s.max_batch) : 0, there = same ? min(rows, w.head->rows) : 0;
    if (!same && w.head->ctas && blockIdx.x == 0 && threadIdx.x == 0) atomicOr(t.status, DLLM_SERVE_STATE);
    // rows that are padding
    for (long long i = static_cast<long long>(there) * words + blockIdx.x * kThreads + threadIdx.x;
         i < static_cast<long long>(rows) * words; i += static_cast<long long>(gridDim.x) * kThreads)
        mask[i] = 0;
    for (int b = blockIdx.x; b < batch; b += gridDim.x) {
        const int2 r = rows_of(t, b, there);
        const int n = r.y - r.x, was = w.left_out[b];
        if (n == 0) continue;
        const int* par = parent + r.x;
        bool bad = n > 32ll * words;
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += kThreads) {
            const int p = par[i];
            bad |= p < -1 || p >= i;
            if (i < kStaged) staged[i] = p;
        }
        // (a request whose rows the plan has left out in part is of no use)
        const bool wrong = __syncthreads_or(bad);
        if (threadIdx.x == 0 && was != wrong) w.left_out[b] = wrong;
        if (wrong) {
            if (threadIdx.x == 0) atomicOr(t.status, DLLM_SERVE_TREE);
            for (long long i = threadIdx.x; i < static_cast<long long>(n) * words; i += kThreads)
                mask[static_cast<long long>(r.x) * words + i] = 0;
            if (t.slot[r.x] >= 0) {  // (an earlier tree of the same plan may have moved them)
                for (int i = 1 + threadIdx.x; i < n; i += kThreads) t.pos[r.x + i] = t.pos[r.x] + i;
            }
            continue;
        }
        const bool refused = t.slot[r.x] < 0;
        const int pos0 = t.pos[r.x];  // (token 0 follows none: its position stays)
        for (int i = threadIdx.x; i < n; i += kThreads) {
            uint32_t* row = mask + static_cast<long long>(r.x + i) * words;
            int at = words - 1, depth = -1;  // the word that is made
            uint32_t bits = 0;
            for (int j = i; j >= 0; j = j < kStaged ? staged[j] : par[j]) {
                for (; at > j >> 5; --at) {
                    row[at] = bits;
                    bits = 0;
                }
                bits |= 1u << (j & 31);
                ++depth;
            }
            for (; at >= 0; --at) {
                row[at] = bits;
                bits = 0;
            }
            if (!refused) t.pos[r.x + i] = pos0 + depth;
        }
    }
}

// A warp takes a request and goes down the path, 32 tokens looked at side by side.  A request that the plan has refused, or
// whose tree was wrong, has no path: its rows have attended to nothing that a decision could come from.  Bound: latency, two
// trips to L2 a token of the path (the decision, then the children's parents and ids).  32 trees of up to 61, 4 us of the 9.6
// that it takes with the compaction behind it.
__global__ void __launch_bounds__(kThreads) k_serve_accept(const __grid_constant__ ServeShape s,
                                                           const __grid_constant__ dllm_serve_tables t,
                                                           const __grid_constant__ ServeAcceptArgs a) {
    ServeArrays w;
    serve_arrays(s, t.work, &w);
    const int lane = threadIdx.x & 31, b = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    pdl_wait();
    pdl_launch_dependents();
    if (b >= a.batch) return;
    const bool same = serve_same_shape(s, *w.head);
    if (!same && w.head->ctas && b == 0 && lane == 0) atomicOr(t.status, DLLM_SERVE_STATE);
    const int left_out = w.left_out[b];
    int2 r = make_int2(0, 0);
    if (same && b < w.head->batch) r = rows_of(t, b, min(a.rows, w.head->rows));
    const int n = r.y - r.x;
    int* keep = a.keep + static_cast<long long>(b) * a.max_len;
    const int slot = n > 0 ? t.slot[r.x] : -1;  // (looked at behind the walk, which does not wait for it)
    int node = n > 0 ? 0 : -1, len = 0, next = -1;
    while (node >= 0) {
        if (lane == 0) keep[len] = node;
        ++len;
        next = a.x0[r.x + node];
        if (len == a.max_len) break;
        int child = -1;
        for (int i0 = (node + 1) & ~31; i0 < n; i0 += 32) {
            const int i = i0 + lane;
            const bool hit = i > node && i < n && a.parent[r.x + i] == node && a.ids[r.x + i] == next;
            const uint32_t any = __ballot_sync(0xffffffffu, hit);
            if (any) {
                child = i0 + __ffs(any) - 1;
                break;
            }
        }
        node = child;
    }
    if (slot < 0 || left_out) {
        len = 0;
        next = -1;
    }
    __syncwarp();
    for (int i = len + lane; i < a.max_len; i += 32) keep[i] = -1;
    if (lane == 0) {
        a.n[b] = len;
        a.next[b] = next;
    }
}

}  // namespace

cudaError_t launch_serve_tree(const ServeShape& s, const dllm_serve_tables& t, const int* parent, uint32_t* mask, int words,
                              int rows, int sms, cudaStream_t st) {
    // (the plan's batch is on the device; a request has a row, or nothing to do)
    const int most = rows < s.max_batch ? rows : s.max_batch, fill = 16 * sms;
    return serve_launch(k_serve_tree, dim3(most < fill ? most : fill), kThreads, 0, st, s, t, parent, mask, words, rows);
}

cudaError_t launch_serve_accept(const ServeShape& s, const dllm_serve_tables& t, const ServeAcceptArgs& a, cudaStream_t st) {
    constexpr int kWarps = kThreads / 32;
    return serve_launch(k_serve_accept, dim3((a.batch + kWarps - 1) / kWarps), kThreads, 0, st, s, t, a);
}

}  // namespace dllm
