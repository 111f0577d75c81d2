// Pages of the serving cache between steps (include/dllm_serve_drafts.h): kept places moved together in all layers
// (dllm_serve_compact), and requests that continue others on shared pages (dllm_serve_fork).
#include "serve.cuh"

namespace dllm {

namespace {

// ---------------------------------------------------------------------------------------------- compact
constexpr int kMoveThreads = 256;
constexpr int kMoveWarps = kMoveThreads / 32;

// A warp takes a request, a layer's K or V, and a head: places in ascending order, 32 at a time, all of them loaded
// before the first is stored.  A place moves down or stays, so what is stored lies below all that is yet to be loaded.
template <int HD>
__global__ void __launch_bounds__(kMoveThreads) k_serve_compact(const __grid_constant__ ServeShape s,
                                                                const __grid_constant__ dllm_serve_tables t,
                                                                const __grid_constant__ ServeCaches c,
                                                                const __grid_constant__ ServeCompactArgs a) {
    constexpr int kLanes = HD / 8, kAtOnce = 32 / kLanes;  // lanes of a row of 16-byte pieces, rows of a warp's load
    ServeArrays w;
    serve_arrays(s, t.work, &w);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int columns = 2 * c.n * s.Hkv;
    const long long units = static_cast<long long>(a.batch) * columns;
    pdl_wait();
    pdl_launch_dependents();
    for (long long unit = static_cast<long long>(blockIdx.x) * kMoveWarps + warp; unit < units;
         unit += static_cast<long long>(gridDim.x) * kMoveWarps) {
        const int b = static_cast<int>(unit / columns), col = static_cast<int>(unit % columns);
        const int n = a.n[b], first = a.first[b], held = t.held[b];
        if (n == 0) continue;
        const int* keep = a.keep + static_cast<long long>(b) * a.keep_ld;
        const int* table = t.table + static_cast<size_t>(b) * s.max_pages;
        const long long end = static_cast<long long>(min(max(held, 0), s.max_pages)) << s.page_log2;  // places there are
        // the list ascends, its places are there and in the pool; the first that moves
        bool bad = n < 0 || n > a.keep_ld || first < 0;
        int from = n, bits = 0;
        if (!bad) {
            int last = -1;
            for (int i0 = 0; i0 < n; i0 += 32) {
                const int i = i0 + lane, k = i < n ? keep[i] : 0x7fffffff;
                int before = __shfl_up_sync(0xffffffffu, k, 1);
                if (lane == 0) before = last;
                last = __shfl_sync(0xffffffffu, k, 31);
                if (i < n) {
                    bad |= k <= before || k < 0 || first + static_cast<long long>(k) >= end;
                    if (k != i) from = min(from, i);
                }
            }
            from = __reduce_min_sync(0xffffffffu, from);
        }
        if (__any_sync(0xffffffffu, bad)) {
            bits = DLLM_SERVE_TREE;
        } else if (from == n) {
            continue;
        } else if ((first + from) >> s.page_log2 < w.shared[b]) {
            bits = DLLM_SERVE_SHARED;
        } else {
            bool out = false;  // a page that is not of the pool
            const int p1 = (first + keep[n - 1]) >> s.page_log2;
            for (int p = ((first + from) >> s.page_log2) + lane; p <= p1; p += 32) out |= table[p] < 0 || table[p] >= s.n_pages;
            if (__any_sync(0xffffffffu, out)) bits = DLLM_SERVE_STATE;
        }
        if (bits) {
            if (lane == 0 && col == 0) atomicOr(t.status, bits);
            continue;
        }
        uint4* cache = static_cast<uint4*>(col & 1 ? c.v[(col >> 1) / s.Hkv] : c.k[(col >> 1) / s.Hkv]) +
                       static_cast<long long>((col >> 1) % s.Hkv) * s.page * kLanes + lane % kLanes;
        auto row = [&](int place) {  // of the cache, in 16-byte pieces
            return static_cast<long long>(table[place >> s.page_log2]) * (s.page_stride / 8) + (place & (s.page - 1)) * kLanes;
        };
        for (int i0 = from; i0 < n; i0 += 32) {
            const int i = i0 + lane;
            long long src = 0, dst = 0;
            if (i < n) {
                src = row(first + keep[i]);
                dst = row(first + i);
            }
            uint4 x[32 / kAtOnce];
#pragma unroll
            for (int k = 0; k < 32 / kAtOnce; ++k) {
                const long long at = __shfl_sync(0xffffffffu, src, k * kAtOnce + lane / kLanes);
                if (i0 + k * kAtOnce + lane / kLanes < n) x[k] = cache[at];
            }
            __syncwarp();
#pragma unroll
            for (int k = 0; k < 32 / kAtOnce; ++k) {
                const long long at = __shfl_sync(0xffffffffu, dst, k * kAtOnce + lane / kLanes);
                if (i0 + k * kAtOnce + lane / kLanes < n) cache[at] = x[k];
            }
            __syncwarp();
        }
    }
}

// ---------------------------------------------------------------------------------------------- fork
constexpr int kForkThreads = 1024;
constexpr int kForkWarps = kForkThreads / 32;
constexpr int kForkCtas = 8;  // a cluster

// The bookkeeping's workspace.
constexpr int kOld = 1 << 30, kKept = 1 << 29, kCount = kKept - 1;
struct ForkArrays {
    int* head;    // [0]: jobs, [1]: a page number outside the pool, [2 ..]: pages given back, a CTA each
    int4* job;    // [max_batch]: page, its copy, places
    int* mark;    // [n_pages]: rows that hold the page in full after the fork; held before it; its last writer keeps it
    int* writer;  // [n_pages]: max_batch - the first request that goes on writing to it
    int* stage;   // [max_batch][max_pages]: the rows after the fork
};
__host__ __device__ inline size_t fork_arrays(const ServeShape& s, void* base, ForkArrays* out) {
    size_t at = 0;
    char* b = static_cast<char*>(base);
    ForkArrays r;
    r.head = reinterpret_cast<int*>(b + at);
    at += 256;
    r.job = reinterpret_cast<int4*>(b + at);
    at += serve_round(sizeof(int4) * s.max_batch);
    r.mark = reinterpret_cast<int*>(b + at);
    at += serve_round(sizeof(int) * s.n_pages);
    r.writer = reinterpret_cast<int*>(b + at);
    at += serve_round(sizeof(int) * s.n_pages);
    r.stage = reinterpret_cast<int*>(b + at);
    at += serve_round(sizeof(int) * static_cast<size_t>(s.max_batch) * s.max_pages);
    if (out) *out = r;
    return at;
}

__device__ __forceinline__ void cluster_barrier() {
    __syncthreads();  // (the barrier wants whole warps)
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ int cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return static_cast<int>(r);
}
__device__ __forceinline__ int cluster_size() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return static_cast<int>(r);
}
// Sum over the block of the values before this thread's; total in sum.
__device__ __forceinline__ int block_before(int v, int* buf, int* sum) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int upto = v;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const int o = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += o;
    }
    __syncthreads();
    if (lane == 31) buf[warp] = upto;
    __syncthreads();
    int before = 0, all = 0;
    for (int w = 0; w < kForkWarps; ++w) {
        const int x = buf[w];
        if (w < warp) before += x;
        all += x;
    }
    *sum = all;
    return before + upto - v;
}

// The tables.  One cluster: every CTA looks at all requests, the rows and the pages are shared out, marks go through L2
// between cluster barriers.  Nothing that others read is changed before it is known that the fork can be carried out.
__global__ void __launch_bounds__(kForkThreads) k_serve_fork(const __grid_constant__ ServeShape s,
                                                             const __grid_constant__ dllm_serve_tables t, const int* src,
                                                             const int* len, int batch) {
    __shared__ int s_src[kServeMaxBatch], s_last[kServeMaxBatch];  // the request continued; the last page, if partly filled
    __shared__ int s_scan[kForkWarps];
    const int rank = cluster_rank(), ctas = cluster_size(), tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int lg = s.page_log2, page = s.page, M = s.max_pages;
    ServeArrays w;
    serve_arrays(s, t.work, &w);
    ForkArrays f;
    fork_arrays(s, t.partials, &f);
    pdl_wait();
    pdl_launch_dependents();

    // ------------------------------------------------ what is asked for
    const int head0 = t.ring_pos[0], free0 = t.ring_pos[1];
    const int free_n = min(max(free0, 0), s.n_pages);
    const int head = static_cast<int>(static_cast<unsigned>(max(head0, 0)) % static_cast<unsigned>(s.n_pages));
    int bits = free0 != free_n || head0 != head ? DLLM_SERVE_STATE : 0;
    auto held_of = [&](int b) { return min(max(t.held[b], 0), M); };
    for (int b = tid; b < s.max_batch; b += kForkThreads)
        if (t.held[b] < 0 || t.held[b] > M) bits |= DLLM_SERVE_STATE;
    for (int b = tid; b < batch; b += kForkThreads) {
        int from = src[b], last = -1;
        const int n = len[b];
        if (from < 0 || from >= s.max_batch || n < 0) {
            bits |= DLLM_SERVE_LENGTHS;
            from = 0;
        } else {
            const int need = static_cast<int>((static_cast<long long>(n) + page - 1) >> lg);
            if (need > held_of(from)) {
                bits |= DLLM_SERVE_LENGTHS;
            } else if (n & (page - 1)) {
                last = t.table[static_cast<size_t>(from) * M + (n >> lg)];
                if (last < 0 || last >= s.n_pages) bits |= DLLM_SERVE_STATE;
                else if (rank == 0) f.writer[last] = 0;
            }
        }
        s_src[b] = from;
        s_last[b] = last;
    }
    const int p0 = static_cast<int>(static_cast<long long>(s.n_pages) * rank / ctas);
    const int p1 = static_cast<int>(static_cast<long long>(s.n_pages) * (rank + 1) / ctas);
    for (int p = p0 + tid; p < p1; p += kForkThreads) f.mark[p] = 0;
    if (rank == 0 && tid < 2) f.head[tid] = 0;
    const bool shape_bad = __syncthreads_or(bits) != 0;
    cluster_barrier();
    auto refuse = [&](int why) {
        if (rank == 0) {
            if (why) atomicOr(t.status, why);
            if (tid == 0) {
                t.status[1] = batch;
                t.status[2] = t.status[3] = 0;
            }
        }
    };
    if (shape_bad) return refuse(bits);

    // ------------------------------------------------ who holds what
    bool out = false;
    for (int r = rank * kForkWarps + warp; r < s.max_batch; r += ctas * kForkWarps) {
        const int held = held_of(r);
        const int* row = t.table + static_cast<size_t>(r) * M;
        for (int i = lane; i < held; i += 32) {
            const int p = row[i];
            if (p < 0 || p >= s.n_pages) out = true;
            else if (r < batch) atomicOr(f.mark + p, kOld);
            else atomicAdd(f.mark + p, 1);
        }
        if (r >= batch) continue;
        const int full = len[r] >> lg;
        const int* from = t.table + static_cast<size_t>(s_src[r]) * M;
        for (int i = lane; i < full; i += 32) {
            const int p = from[i];
            f.stage[static_cast<size_t>(r) * M + i] = p;
            if (p < 0 || p >= s.n_pages) out = true;
            else atomicAdd(f.mark + p, 1);
        }
    }
    if (rank == 0) {
        for (int b = tid; b < batch; b += kForkThreads)
            if (s_last[b] >= 0) atomicMax(f.writer + s_last[b], s.max_batch - b);
    }
    if (out) f.head[1] = 1;
    cluster_barrier();
    if (f.head[1]) return refuse(tid == 0 ? DLLM_SERVE_STATE : 0);

    // ------------------------------------------------ the last pages: kept, or copied
    const int per = (batch + kForkThreads - 1) / kForkThreads;
    const int b0 = min(batch, tid * per), b1 = min(batch, b0 + per);
    auto copied = [&](int b) {
        const int p = s_last[b];
        return p >= 0 && ((f.mark[p] & kCount) > 0 || f.writer[p] != s.max_batch - b);
    };
    int mine = 0, taken;
    for (int b = b0; b < b1; ++b) mine += copied(b);
    int nth = block_before(mine, s_scan, &taken);
    if (taken > free_n) return refuse(tid == 0 ? DLLM_SERVE_PAGES : 0);
    auto free_page = [&](int k) { return t.ring[(static_cast<unsigned>(head) + k) % static_cast<unsigned>(s.n_pages)]; };
    for (int k = tid; k < taken; k += kForkThreads) out |= free_page(k) < 0 || free_page(k) >= s.n_pages;
    if (__syncthreads_or(out)) return refuse(tid == 0 ? DLLM_SERVE_STATE : 0);
    for (int b = b0; b < b1; ++b) {
        const int p = s_last[b];
        if (p < 0) continue;
        if (copied(b)) {
            const int to = free_page(nth);
            if (rank == 0) f.job[nth] = make_int4(p, to, len[b] & (page - 1), 0);
            s_last[b] = to;
            ++nth;
        } else if (rank == 0) {
            atomicOr(f.mark + p, kKept);
        }
    }
    cluster_barrier();  // (and the state is read)

    // ------------------------------------------------ the rows
    for (int r = rank * kForkWarps + warp; r < s.max_batch; r += ctas * kForkWarps) {
        int* row = t.table + static_cast<size_t>(r) * M;
        const int held = held_of(r), n = r < batch ? len[r] : 0, full = r < batch ? n >> lg : held;
        const int need = r < batch ? static_cast<int>((static_cast<long long>(n) + page - 1) >> lg) : held;
        int shared = 0;
        for (int i = lane; i < max(need, r < batch ? held : 0); i += 32) {
            if (i < full) {
                const int p = r < batch ? f.stage[static_cast<size_t>(r) * M + i] : row[i];
                if ((f.mark[p] & kCount) > 1) shared = i + 1;
                if (r < batch) row[i] = p;
            } else {
                row[i] = i < need ? s_last[r] : -1;
            }
        }
        shared = __reduce_max_sync(0xffffffffu, shared);
        __syncwarp();
        if (lane == 0) {
            w.shared[r] = shared;
            if (r < batch) {
                t.held[r] = need;
                t.n_keys[r] = n;
            }
        }
    }

    // ------------------------------------------------ the ring
    int n_back = 0;
    for (int p = p0 + tid; p < p1; p += kForkThreads) n_back += (f.mark[p] & (kCount | kKept | kOld)) == kOld;
    int given;
    block_before(n_back, s_scan, &given);
    if (tid == 0) f.head[2 + rank] = given;
    cluster_barrier();
    int at = free_n, all = 0;
    for (int c = 0; c < ctas; ++c) {
        if (c < rank) at += f.head[2 + c];
        all += f.head[2 + c];
    }
    for (int q = p0; q < p1; q += kForkThreads) {
        const int p = q + tid;
        const bool back = p < p1 && (f.mark[p] & (kCount | kKept | kOld)) == kOld;
        int here;
        const int before = block_before(back, s_scan, &here);
        if (back) t.ring[(static_cast<unsigned>(head) + at + before) % static_cast<unsigned>(s.n_pages)] = p;
        at += here;
    }
    if (rank == 0 && tid == 0) {
        f.head[0] = taken;
        t.ring_pos[0] = static_cast<int>((static_cast<unsigned>(head) + taken) % static_cast<unsigned>(s.n_pages));
        t.ring_pos[1] = min(free_n - taken + all, s.n_pages);
        t.status[1] = 0;
        t.status[2] = taken;
        t.status[3] = all;
    }
}

// The copies: a warp takes a job, a layer's K or V and a head, whose places lie side by side.
__global__ void __launch_bounds__(kMoveThreads) k_serve_copy(const __grid_constant__ ServeShape s,
                                                             const __grid_constant__ dllm_serve_tables t,
                                                             const __grid_constant__ ServeCaches c) {
    constexpr int kAhead = 8;
    ForkArrays f;
    fork_arrays(s, t.partials, &f);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, columns = 2 * c.n * s.Hkv, row = s.hd / 8;
    pdl_wait();
    pdl_launch_dependents();
    const long long units = static_cast<long long>(f.head[0]) * columns;
    for (long long unit = static_cast<long long>(blockIdx.x) * kMoveWarps + warp; unit < units;
         unit += static_cast<long long>(gridDim.x) * kMoveWarps) {
        const int4 j = f.job[unit / columns];
        const int col = static_cast<int>(unit % columns);
        uint4* cache = static_cast<uint4*>(col & 1 ? c.v[(col >> 1) / s.Hkv] : c.k[(col >> 1) / s.Hkv]) +
                       static_cast<long long>((col >> 1) % s.Hkv) * s.page * row;
        const uint4* from = cache + j.x * (s.page_stride / 8);
        uint4* to = cache + j.y * (s.page_stride / 8);
        const int n = j.z * row;
        for (int i0 = lane; i0 < n; i0 += 32 * kAhead) {
            uint4 x[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                if (i0 + 32 * k < n) x[k] = from[i0 + 32 * k];
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                if (i0 + 32 * k < n) to[i0 + 32 * k] = x[k];
        }
    }
}

}  // namespace

cudaError_t launch_serve_compact(const ServeShape& s, const dllm_serve_tables& t, const ServeCaches& c,
                                 const ServeCompactArgs& a, int sms, cudaStream_t st) {
    const long long units = 2ll * c.n * s.Hkv * a.batch, ctas = (units + kMoveWarps - 1) / kMoveWarps;
    const dim3 grid(static_cast<unsigned>(ctas < 8ll * sms ? ctas : 8ll * sms));
    return s.hd == 128 ? serve_launch(k_serve_compact<128>, grid, kMoveThreads, 0, st, s, t, c, a)
                       : serve_launch(k_serve_compact<64>, grid, kMoveThreads, 0, st, s, t, c, a);
}

size_t serve_fork_bytes(const ServeShape& s) { return fork_arrays(s, nullptr, nullptr); }

cudaError_t launch_serve_fork(const ServeShape& s, const dllm_serve_tables& t, const ServeCaches& c, const int* src,
                              const int* len, int batch, int sms, cudaStream_t st) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = cfg.blockDim = dim3(1);
    cfg.gridDim.x = kForkCtas;
    cfg.blockDim.x = kForkThreads;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cfg.gridDim.x;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    cudaError_t e = cudaLaunchKernelEx(&cfg, k_serve_fork, s, t, src, len, batch);
    if (e != cudaSuccess) return e;
    const long long units = 2ll * c.n * s.Hkv * batch, ctas = (units + kMoveWarps - 1) / kMoveWarps;
    return serve_launch(k_serve_copy, dim3(static_cast<unsigned>(ctas < 8ll * sms ? ctas : 8ll * sms)), kMoveThreads, 0, st, s, t, c);
}

}  // namespace dllm
