// Pages of the serving cache between steps (include/dllm_serve_drafts.h): kept places moved together in all layers
// (dllm_serve_compact), and requests that continue others on shared pages (dllm_serve_fork).
#include "serve.cuh"

namespace dllm {

namespace {

// ---------------------------------------------------------------------------------------------- compact
constexpr int kMoveThreads = 256;
constexpr int kMoveWarps = kMoveThreads / 32;

// A request's column is a layer's K or V and a head.  Its places are moved in ascending order, a step of them at a
// time, all of a step loaded before the first is stored.  A place moves down or stays, so what is stored lies below all that
// is yet to be loaded, and loads may run ahead.  A list that ascends from 0 begins with the places that stay.
// Bound: memory, for long lists.  Measured in a graph, 28 layers of 4 heads of 128: 6 requests of 500 to 2000 keep two
// thirds 79.6 us (484 MB: 6.1 TB/s; a warp a column took 2 times that, a CTA a column without steps ahead 1.2 times); paths of
// up to 16 of 32 requests, with their finding, 9.6 (a column's chain: lengths, list, pages, values).
struct Column {
    const int* keep;
    const int* table;
    uint4* cache;  // of the lane's 16 bytes
    int n, first, from;
};

// What request b asks for.  Threads: a warp's or a CTA's (THREADS of them, me one of them).  False: nothing to move.
template <int HD, int THREADS>
__device__ __forceinline__ bool column_of(const ServeShape& s, const dllm_serve_tables& t, const ServeCaches& c,
                                          const ServeCompactArgs& a, int b, int col, int me, int* s_stay,
                                          Column* out) {
    constexpr int kLanes = HD / 8;
    constexpr bool kWarp = THREADS == 32;
    auto any = [&](bool v) { return kWarp ? __any_sync(0xffffffffu, v) != 0 : __syncthreads_or(v) != 0; };
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int n = a.n[b], first = a.first[b], held = t.held[b], shared = t.shared[b];
    if (n == 0) return false;
    const int* keep = a.keep + static_cast<long long>(b) * a.keep_ld;
    const int* table = t.table + static_cast<size_t>(b) * s.max_pages;
    const long long end = static_cast<long long>(min(max(held, 0), s.max_pages)) << s.page_log2;  // places there are
    // the list ascends, its places are there and in the pool; how many of them stay
    bool bad = n < 0 || n > a.keep_ld || first < 0;
    int from = 0, bits = 0;
    if (!bad) {
#pragma unroll 4
        for (int i = me; i < n; i += THREADS) {
            const int k = keep[i], below = i ? keep[i - 1] : -1;
            bad |= k <= below || first + static_cast<long long>(k) >= end;
            from += k == i;
        }
    }
    from = __reduce_add_sync(0xffffffffu, from);
    if (!kWarp && lane == 0) s_stay[warp] = from;
    if (any(bad)) {
        bits = DLLM_SERVE_TREE;
    } else {
        if (!kWarp) {
            from = 0;
            for (int i = 0; i < THREADS / 32; ++i) from += s_stay[i];
        }
        if (from == n) return false;
        bool out_of = false;  // a page that is not of the pool
        const int p1 = (first + keep[n - 1]) >> s.page_log2;
        for (int p = ((first + from) >> s.page_log2) + me; p <= p1; p += THREADS) out_of |= table[p] < 0 || table[p] >= s.n_pages;
        if (any(out_of)) bits = DLLM_SERVE_STATE;
        if ((first + from) >> s.page_log2 < shared) bits = DLLM_SERVE_SHARED;
    }
    if (bits) {
        if (me == 0 && col == 0) atomicOr(t.status, bits);
        return false;
    }
    out->keep = keep;
    out->table = table;
    out->n = n;
    out->first = first;
    out->from = from;
    out->cache = static_cast<uint4*>(col & 1 ? c.v[(col >> 1) / s.Hkv] : c.k[(col >> 1) / s.Hkv]) +
                 static_cast<long long>((col >> 1) % s.Hkv) * s.page * kLanes + lane % kLanes;
    return true;
}
// A place's row of the cache, in 16-byte pieces.
template <int HD>
__device__ __forceinline__ long long row_of(const ServeShape& s, const Column& u, int place) {
    return static_cast<long long>(u.table[place >> s.page_log2]) * (s.page_stride / 8) + (place & (s.page - 1)) * (HD / 8);
}

// Short lists (an accepted path): a warp a column.  (80 registers, so that three CTAs fit an SM: 4 words are spilled.)
template <int HD>
__global__ void __launch_bounds__(kMoveThreads, 3)
    k_serve_compact(const __grid_constant__ ServeShape s, const __grid_constant__ dllm_serve_tables t,
                    const __grid_constant__ ServeCaches c, const __grid_constant__ ServeCompactArgs a) {
    constexpr int kLanes = HD / 8, kAtOnce = 32 / kLanes;  // lanes of a row of 16-byte pieces, rows of a warp's load
    constexpr int kLoads = 8, kStep = kLoads * kAtOnce;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, nth = lane / kLanes;
    const int columns = 2 * c.n * s.Hkv;
    const long long units = static_cast<long long>(a.batch) * columns;
    pdl_wait();
    pdl_launch_dependents();
    for (long long unit = static_cast<long long>(blockIdx.x) * kMoveWarps + warp; unit < units;
         unit += static_cast<long long>(gridDim.x) * kMoveWarps) {
        Column u;
        if (!column_of<HD, 32>(s, t, c, a, static_cast<int>(unit / columns), static_cast<int>(unit % columns), lane, nullptr, &u))
            continue;
        for (int i0 = u.from; i0 < u.n; i0 += kStep) {
            long long src = 0, dst = 0;
            if (lane < kStep && i0 + lane < u.n) {
                src = row_of<HD>(s, u, u.first + u.keep[i0 + lane]);
                dst = row_of<HD>(s, u, u.first + i0 + lane);
            }
            uint4 x[kLoads];
#pragma unroll
            for (int k = 0; k < kLoads; ++k) {
                const long long at = __shfl_sync(0xffffffffu, src, k * kAtOnce + nth);
                if (i0 + k * kAtOnce + nth < u.n) x[k] = u.cache[at];
            }
            __syncwarp();
#pragma unroll
            for (int k = 0; k < kLoads; ++k) {
                const long long at = __shfl_sync(0xffffffffu, dst, k * kAtOnce + nth);
                if (i0 + k * kAtOnce + nth < u.n) u.cache[at] = x[k];
            }
            __syncwarp();
        }
    }
}

// Long lists: a CTA a column, steps copied ahead into shared memory, each lane what it stores itself.
constexpr int kMoveStages = 3, kMoveLoads = 8;
constexpr int kMoveSmem = kMoveStages * kMoveWarps * kMoveLoads * 32 * 16;
template <int HD>
__global__ void __launch_bounds__(kMoveThreads, 2)
    k_serve_compact_long(const __grid_constant__ ServeShape s, const __grid_constant__ dllm_serve_tables t,
                         const __grid_constant__ ServeCaches c, const __grid_constant__ ServeCompactArgs a) {
    constexpr int kLanes = HD / 8, kAtOnce = 32 / kLanes;
    constexpr int kRows = kMoveLoads * kAtOnce, kStep = kRows * kMoveWarps;  // of a warp, of a CTA
    extern __shared__ __align__(16) uint4 ring[];
    __shared__ int s_stay[kMoveWarps];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, nth = lane / kLanes;
    const int columns = 2 * c.n * s.Hkv;
    const long long units = static_cast<long long>(a.batch) * columns;
    uint4* const mine = ring + warp * (kMoveLoads * 32) + lane;
    pdl_wait();
    pdl_launch_dependents();
    for (long long unit = blockIdx.x; unit < units; unit += gridDim.x) {
        Column u;
        if (column_of<HD, kMoveThreads>(s, t, c, a, static_cast<int>(unit / columns), static_cast<int>(unit % columns),
                                        threadIdx.x, s_stay, &u)) {
            const int begin = u.from + warp * kRows;
            long long src = 0;
            auto look = [&](int i0) {  // the rows that a step's places come from, a lane a place
                if (lane < kRows && i0 + lane < u.n) src = row_of<HD>(s, u, u.first + u.keep[i0 + lane]);
            };
            auto ask = [&](int i0, int stage) {  // a step's copies, and the rows of the step after it
#pragma unroll
                for (int k = 0; k < kMoveLoads; ++k) {
                    const long long at = __shfl_sync(0xffffffffu, src, k * kAtOnce + nth);
                    if (i0 + k * kAtOnce + nth < u.n) cp_async16(mine + (stage * kMoveWarps * kMoveLoads + k) * 32, u.cache + at);
                }
                cp_async_commit();
                look(i0 + kStep);
            };
            look(begin);
#pragma unroll
            for (int k = 0; k < kMoveStages; ++k) ask(begin + k * kStep, k);
            int stage = 0;
            for (int i0 = begin; i0 - begin < u.n - u.from; i0 += kStep) {
                long long dst = 0;
                if (lane < kRows && i0 + lane < u.n) dst = row_of<HD>(s, u, u.first + i0 + lane);
                cp_async_wait<kMoveStages - 1>();
                __syncthreads();  // all warps have the step
#pragma unroll
                for (int k = 0; k < kMoveLoads; ++k) {
                    const long long at = __shfl_sync(0xffffffffu, dst, k * kAtOnce + nth);
                    if (i0 + k * kAtOnce + nth < u.n) u.cache[at] = mine[(stage * kMoveWarps * kMoveLoads + k) * 32];
                }
                ask(i0 + kMoveStages * kStep, stage);
                stage = stage + 1 == kMoveStages ? 0 : stage + 1;
            }
            cp_async_wait<0>();
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------------------------- fork
constexpr int kForkCtas = 8;  // a cluster
template <bool SMALL>
constexpr int kForkThreads = SMALL ? 512 : 1024;
// One CTA with all of it in shared memory, for so many requests, and places of the rows with half the pool's pages (the
// launch has the measurements).
constexpr int kSmallBatch = 256, kSmallWork = 6144;
constexpr int kSmallPages = 2 * kSmallWork, kSmallStage = kSmallWork;
size_t fork_smem(const ServeShape& s, bool small) {
    return sizeof(int) * (5 * static_cast<size_t>(s.max_batch) + (small ? 2 * static_cast<size_t>(s.n_pages) + kSmallStage : 0));
}
constexpr size_t kForkSmem[2] = {sizeof(int) * 5 * kServeMaxBatch,
                                 sizeof(int) * (5 * kSmallBatch + 2 * kSmallPages + kSmallStage)};  // the most of any call

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
template <int WARPS>
__device__ __forceinline__ int block_before(int v, int* buf, int* sum) {
    static_assert(WARPS <= 32, "a lane for each warp's sum");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    auto scan = [&](int x) {
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const int o = __shfl_up_sync(0xffffffffu, x, d);
            if (lane >= d) x += o;
        }
        return x;
    };
    const int upto = scan(v);
    __syncthreads();
    if (lane == 31) buf[warp] = upto;
    __syncthreads();
    const int warps = scan(lane < WARPS ? buf[lane] : 0);
    *sum = __shfl_sync(0xffffffffu, warps, 31);
    const int before = __shfl_sync(0xffffffffu, warps, (warp + 31) & 31);
    return (warp ? before : 0) + upto - v;
}
// The tables.  One cluster: every CTA looks at all requests, the rows and the pages are shared out, marks go through L2
// between cluster barriers; or (SMALL) one CTA, marks in shared memory.  Nothing that others read is changed before it is
// known that the fork can be carried out.
// Bound: latency of its phases: two trips to memory, the marks, a scan.  Measured in a graph with the copies: four beams of a
// small request 5.6 us by one CTA (10.4 by the cluster), 16 groups of 6 beams of a 28-layer cache 32.3 by the cluster (33.1 by one
// CTA; 163 MB copied in 22.5); by the cluster, with one layer of 4 heads, 1500 requests of 11 pages 50, 4096 of 5 84, 16 of 6250
// 160.  Threads of the one CTA, four beams and, by it too, the groups, each pass with a graph's launch: 128 5.8 and 45, 256 5.9
// and 38.5, 512 6.0 and 36.3, 1024 6.4 and 36.0.
template <bool SMALL>
__global__ void __launch_bounds__(kForkThreads<SMALL>, 1) k_serve_fork(const __grid_constant__ ServeShape s,
                                                             const __grid_constant__ dllm_serve_tables t, const int* src,
                                                             const int* len, int batch, int row_lanes) {
    extern __shared__ int smem[];
    constexpr int kThreads = kForkThreads<SMALL>, kWarps = kThreads / 32;
    __shared__ int s_scan[kWarps];
    const int B = s.max_batch, M = s.max_pages, lg = s.page_log2, page = s.page, tid = threadIdx.x;
    // of the requests: the one continued, its length, pages held before; the last page, if partly filled; pages shared
    int *s_src = smem, *s_len = s_src + B, *s_held = s_len + B, *s_last = s_held + B, *s_shared = s_last + B;
    const int rank = SMALL ? 0 : cluster_rank(), ctas = SMALL ? 1 : cluster_size();
    ForkArrays f;
    fork_arrays(s, t.partials, &f);
    int* const mark = SMALL ? smem + 5 * B : f.mark;
    int* const writer = SMALL ? smem + 5 * B + s.n_pages : f.writer;
    int* const stage = SMALL ? smem + 5 * B + 2 * s.n_pages : f.stage;
    auto barrier = [] {
        if (SMALL) __syncthreads();
        else cluster_barrier();
    };
    const int p0 = static_cast<int>(static_cast<long long>(s.n_pages) * rank / ctas);
    const int p1 = static_cast<int>(static_cast<long long>(s.n_pages) * (rank + 1) / ctas);
    if (SMALL) {
        for (int p = tid; p < s.n_pages; p += kThreads) mark[p] = writer[p] = 0;
    }
    pdl_wait();
    pdl_launch_dependents();

    // ------------------------------------------------ what is asked for
    const int head0 = t.ring_pos[0], free0 = t.ring_pos[1];
    int bits = 0;
    for (int b = tid; b < B; b += kThreads) {
        const int held = t.held[b], from = b < batch ? src[b] : b, n = b < batch ? len[b] : 0;
        const bool bad = from < 0 || from >= B || n < 0;
        if (held < 0 || held > M) bits |= DLLM_SERVE_STATE;
        if (bad) bits |= DLLM_SERVE_LENGTHS;
        s_held[b] = min(max(held, 0), M);
        s_src[b] = bad ? 0 : from;
        s_len[b] = bad ? 0 : n;
        s_shared[b] = 0;
    }
    const int free_n = min(max(free0, 0), s.n_pages);
    const unsigned head = static_cast<unsigned>(max(head0, 0)) % static_cast<unsigned>(s.n_pages);
    if (free0 != free_n || head0 != static_cast<int>(head)) bits |= DLLM_SERVE_STATE;
    auto free_page = [&](int k) { return t.ring[(head + k) % static_cast<unsigned>(s.n_pages)]; };
    const int ring0 = tid < min(batch, free_n) ? free_page(tid) : 0;  // (asked for ahead of its use)
    if (!SMALL) {
        for (int p = p0 + tid; p < p1; p += kThreads) mark[p] = writer[p] = 0;
    }
    if (rank == 0 && tid < 2) f.head[tid] = 0;
    barrier();

    // ------------------------------------------------ who holds what; row_lanes threads a row
    for (int b = tid; b < batch; b += kThreads) {
        const int n = s_len[b], from = s_src[b];
        int last = -1;
        if ((static_cast<long long>(n) + page - 1) >> lg > s_held[from]) {
            bits |= DLLM_SERVE_LENGTHS;
        } else if (n & (page - 1)) {
            last = t.table[static_cast<size_t>(from) * M + (n >> lg)];
            if (last < 0 || last >= s.n_pages) bits |= DLLM_SERVE_STATE;
            else if (rank == 0) atomicMax(writer + last, B - b);
        }
        s_last[b] = last;
    }
    const int sub = tid % row_lanes, row0 = rank * (kThreads / row_lanes) + tid / row_lanes;
    const int rows = ctas * (kThreads / row_lanes);
    bool out = false;
    for (int r = row0; r < B; r += rows) {
        const int held = s_held[r], full = min(s_len[r] >> lg, s_held[s_src[r]]);
        const int* row = t.table + static_cast<size_t>(r) * M;
        const int* from = t.table + static_cast<size_t>(s_src[r]) * M;
        const bool more = r >= batch;  // a row that stays
        for (int i = sub; i < max(held, full); i += row_lanes) {
            const int p = i < held ? row[i] : 0, q = i < full ? from[i] : 0;
            if (p < 0 || p >= s.n_pages || q < 0 || q >= s.n_pages) {
                out = true;
                continue;
            }
            if (i < held) {
                if (more) atomicAdd(mark + p, 1);
                else atomicOr(mark + p, kOld);
            }
            if (i < full) {
                atomicAdd(mark + q, 1);
                stage[static_cast<size_t>(r) * M + i] = q;
            }
        }
    }
    if (tid < min(batch, free_n) && (ring0 < 0 || ring0 >= s.n_pages)) out = true;
    for (int k = kThreads + tid; k < min(batch, free_n); k += kThreads) out |= free_page(k) < 0 || free_page(k) >= s.n_pages;
    if (out) bits |= DLLM_SERVE_STATE;
    bool wrong = __syncthreads_or(bits) != 0;
    if (!SMALL) {
        if (wrong) f.head[1] = 1;
        barrier();
        wrong = f.head[1];
    }
    auto refuse = [&](int why) {
        if (why) atomicOr(t.status, why);
        if (rank == 0 && tid == 0) {
            t.status[1] = batch;
            t.status[2] = t.status[3] = 0;
        }
    };
    if (wrong) return refuse(bits);

    // ------------------------------------------------ the last pages: kept, or copied
    const int per = (batch + kThreads - 1) / kThreads;
    const int b0 = min(batch, tid * per), b1 = min(batch, b0 + per);
    auto copied = [&](int b) {
        const int p = s_last[b];
        return p >= 0 && ((mark[p] & kCount) > 0 || writer[p] != B - b);
    };
    int mine = 0, taken;
    for (int b = b0; b < b1; ++b) mine += copied(b);
    int nth = block_before<kWarps>(mine, s_scan, &taken);
    if (taken > free_n) return refuse(rank == 0 && tid == 0 ? DLLM_SERVE_PAGES : 0);
    for (int b = b0; b < b1; ++b) {
        const int p = s_last[b];
        if (p < 0) continue;
        if (copied(b)) {
            const int to = free_page(nth);
            if (rank == 0) f.job[nth] = make_int4(p, to, s_len[b] & (page - 1), 0);
            s_last[b] = to;
            ++nth;
        } else if (rank == 0) {
            atomicOr(mark + p, kKept);
        }
    }
    barrier();  // (and the state is read)

    // ------------------------------------------------ the rows
    for (int r = row0; r < B; r += rows) {
        int* row = t.table + static_cast<size_t>(r) * M;
        const bool more = r >= batch;
        const int held = s_held[r], n = s_len[r], full = more ? held : n >> lg, need = more ? held : (n >> lg) + ((n & (page - 1)) != 0);
        int shared = 0;
        for (int i = sub; i < max(need, held); i += row_lanes) {
            if (i < full) {
                const int p = more ? row[i] : stage[static_cast<size_t>(r) * M + i];
                if ((mark[p] & kCount) > 1) shared = i + 1;
                if (!more) row[i] = p;
            } else {
                row[i] = i < need ? s_last[r] : -1;
            }
        }
        if (shared) atomicMax(s_shared + r, shared);
        if (sub == 0 && !more) {
            t.held[r] = need;
            t.n_keys[r] = n;
        }
    }

    // ------------------------------------------------ the ring
    int n_back = 0;
    for (int p = p0 + tid; p < p1; p += kThreads) n_back += (mark[p] & (kCount | kKept | kOld)) == kOld;
    int given, all = 0, at = free_n;
    block_before<kWarps>(n_back, s_scan, &given);
    for (int r = row0; r < B; r += rows)
        if (sub == 0) t.shared[r] = s_shared[r];
    if (SMALL) {
        all = given;
    } else {
        if (tid == 0) f.head[2 + rank] = given;
        barrier();
        for (int c = 0; c < ctas; ++c) {
            if (c < rank) at += f.head[2 + c];
            all += f.head[2 + c];
        }
    }
    for (int q = p0; q < p1 && given; q += kThreads) {
        const int p = q + tid;
        const bool back = p < p1 && (mark[p] & (kCount | kKept | kOld)) == kOld;
        int here;
        const int before = block_before<kWarps>(back, s_scan, &here);
        if (back) t.ring[(head + at + before) % static_cast<unsigned>(s.n_pages)] = p;
        at += here;
    }
    if (rank == 0 && tid == 0) {
        f.head[0] = taken;
        t.ring_pos[0] = static_cast<int>((head + taken) % static_cast<unsigned>(s.n_pages));
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
    // By the width of the list's rows, as their lengths are on the device.  Measured in a graph, heads of 128, a warp against a
    // CTA a column: 32 requests of 4 heads and 28 layers 41 and 77 us at 64 places, 76 and 102 at 128, 152 and 154 at 256, 584
    // and 549 at 1024; 4 requests 6.5 and 10.0, 10.3 and 12.1, 23.8 and 17.9, 120 and 77; 32 of 32 heads and layers 321 and 652,
    // 629 and 871, 1245 and 1357, 4953 and 4930.  (Of a wide row little of which is used, 3 places: 6.6 and 57, 3.1 and 9.0.)
    const bool small = a.keep_ld <= 128;
    const long long units = 2ll * c.n * s.Hkv * a.batch, ctas = small ? (units + kMoveWarps - 1) / kMoveWarps : units;
    const dim3 grid(static_cast<unsigned>(ctas < 64ll * sms ? ctas : 64ll * sms));
    if (small)
        return s.hd == 128 ? serve_launch(k_serve_compact<128>, grid, kMoveThreads, 0, st, s, t, c, a)
                           : serve_launch(k_serve_compact<64>, grid, kMoveThreads, 0, st, s, t, c, a);
    const auto kernel = s.hd == 128 ? k_serve_compact_long<128> : k_serve_compact_long<64>;
    const cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void*>(kernel), cudaFuncAttributeMaxDynamicSharedMemorySize, kMoveSmem);
    if (e != cudaSuccess) return e;
    return serve_launch(kernel, grid, kMoveThreads, kMoveSmem, st, s, t, c, a);
}

size_t serve_fork_bytes(const ServeShape& s) { return fork_arrays(s, nullptr, nullptr); }

cudaError_t launch_serve_fork(const ServeShape& s, const dllm_serve_tables& t, const ServeCaches& c, const int* src,
                              const int* len, int batch, int sms, cudaStream_t st) {
    int row_lanes = 1;  // threads a row: as many as it may hold pages, up to a warp
    while (row_lanes < 32 && row_lanes < s.max_pages) row_lanes *= 2;
    // One CTA goes over the rows 512 places at a time, and over the pool.  Measured in a graph, one CTA against the cluster, beams
    // in fours: 4 requests of 4 pages 6.2 and 10.6 us; 16 of 63 6.9 and 10.6, in a pool of 10284 13.1 and 13.5; 64 of 16 9.7 and
    // 11.8, of 63 12.0 and 13.1, in a pool of 11136 17.9 and 13.7; 128 of 16 13.1 and 12.3; 256 of 16 19.8 and 12.8, of 63
    // 29.5 and 13.5; 1000 of 11 38.0 and 16.2.
    const long long places = static_cast<long long>(s.max_batch) * ((s.max_pages + row_lanes - 1) / row_lanes * row_lanes);
    const bool small = s.max_batch <= kSmallBatch && places + s.n_pages / 2 <= kSmallWork;
    const auto kernel = small ? k_serve_fork<true> : k_serve_fork<false>;
    // (always the most of any call, so that host threads do not lower it between another's asking and launch)
    cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void*>(kernel), cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         static_cast<int>(kForkSmem[small]));
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(small ? 1 : kForkCtas);
    cfg.blockDim = dim3(small ? kForkThreads<true> : kForkThreads<false>);
    cfg.dynamicSmemBytes = fork_smem(s, small);
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cfg.gridDim.x;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = small ? 1 : 2;
    e = cudaLaunchKernelEx(&cfg, kernel, s, t, src, len, batch, row_lanes);
    if (e != cudaSuccess) return e;
    const long long units = 2ll * c.n * s.Hkv * batch, ctas = (units + kMoveWarps - 1) / kMoveWarps;
    return serve_launch(k_serve_copy, dim3(static_cast<unsigned>(ctas < 8ll * sms ? ctas : 8ll * sms)), kMoveThreads, 0, st, s, t, c);
}

}  // namespace dllm
