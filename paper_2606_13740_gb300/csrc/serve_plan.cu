// The plan of a serving step: pages taken and given back, slots and positions of the new tokens, and the
// attention's work list, from the requests' lengths (include/dllm_serve.h, dllm_serve_plan).
//
// Everything follows from four running sums over the requests: new tokens, pages taken, pages given back,
// blocks of 64 keys.  Each CTA makes all four by itself in shared memory (up to 4096 requests: a few
// thousand cycles, less than a round of launches or of waiting for one another would cost), then fills its
// share of the rows, pages and blocks, the owner of an item found by binary search in the sums, so that
// one long request among many short ones spreads over all CTAs.  CTA 0 cuts the attention's work instead.
// The state that all of them read (held, ring_pos) is replaced by the CTA that ends last.  Pages come from
// the ring's front and go to its end, so that what a plan takes and what it gives back never meet: the
// free pages and those given back fit into the ring together.
#include "serve.cuh"

namespace dllm {

namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kMost = 0x7fffffff;

struct PlanArgs {
    ServeShape s;
    dllm_serve_tables t;
    const int* len;
    const int* q_len;
    int batch, rows, prefix_len, causal, max_ctas;
};

__device__ __forceinline__ int clip(long long v) { return static_cast<int>(v < kMost ? v : kMost); }

// Exclusive sums over the block of N values a thread; totals in sum.  buf: [N][kWarps].
template <int N>
__device__ __forceinline__ void block_scan(long long (&v)[N], long long (&sum)[N], long long* buf) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    long long own[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        own[i] = v[i];
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const long long o = __shfl_up_sync(0xffffffffu, v[i], d);
            if (lane >= d) v[i] += o;
        }
        if (lane == 31) buf[i * kWarps + warp] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        long long before = 0;
        sum[i] = 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const long long x = buf[i * kWarps + w];
            if (w < warp) before += x;
            sum[i] += x;
        }
        v[i] += before - own[i];
    }
    __syncthreads();
}

// b with a[b] <= k < a[b + 1]; a[0] <= k < a[n].
template <typename T>
__device__ __forceinline__ int find(const T* a, int n, T k) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a[mid] <= k) lo = mid;
        else hi = mid;
    }
    return lo;
}

// What a request wants, apart from the others.
struct Wants {
    int rows, held, need;  // new tokens, pages held and wanted
    bool bad, state;       // its lengths make no sense, or its held does not
};
__device__ __forceinline__ Wants wants(const PlanArgs& a, int b) {
    const int L = __ldg(a.len + b), q = __ldg(a.q_len + b), held = a.t.held[b];
    Wants w;
    w.rows = max(q, 0);
    w.state = held < 0 || held > a.s.max_pages;
    w.held = min(max(held, 0), a.s.max_pages);
    const long long need = (static_cast<long long>(L) + q + a.s.page - 1) >> a.s.page_log2;
    w.bad = w.state || L < 0 || q < 0 || need > a.s.max_pages;
    w.need = w.bad ? w.held : static_cast<int>(need);
    return w;
}

__global__ void __launch_bounds__(kThreads) k_serve_plan(const __grid_constant__ PlanArgs a) {
    extern __shared__ long long smem[];
    const int B = a.batch;
    long long* scan_buf = smem;                          // [4][kWarps]
    long long* tile_sum = scan_buf + 4 * kWarps;         // [kThreads + 1], CTA 0
    int* first_row = reinterpret_cast<int*>(tile_sum + kThreads + 1);  // [B + 1] each: sums before a request
    int* first_grow = first_row + B + 1;
    int* first_shrink = first_grow + B + 1;
    int* first_block = first_shrink + B + 1;
    uint8_t* refused = reinterpret_cast<uint8_t*>(first_block + B + 1);  // [B]
    __shared__ int s_taken, s_refused, s_last;

    const dllm_serve_tables& t = a.t;
    const int n_pages = a.s.n_pages, page = a.s.page, lg = a.s.page_log2;
    ServeArrays w;
    serve_arrays(a.s, t.work, &w);
    if (threadIdx.x == 0) s_taken = s_refused = 0;
    int bits = 0;

    // ------------------------------------------------ the sums
    const int per = (B + kThreads - 1) / kThreads;
    const int b0 = min(B, static_cast<int>(threadIdx.x) * per), b1 = min(B, b0 + per);
    const int head0 = t.ring_pos[0], free0 = t.ring_pos[1];
    const int free_n = min(max(free0, 0), n_pages);
    const int head = static_cast<int>(static_cast<unsigned>(max(head0, 0)) % static_cast<unsigned>(n_pages));
    if (free0 != free_n || head0 != head) bits |= DLLM_SERVE_STATE;
    long long run[3] = {0, 0, 0}, all[3];
    for (int b = b0; b < b1; ++b) {
        const Wants x = wants(a, b);
        run[0] += x.rows;
        run[1] += max(x.need - x.held, 0);
        run[2] += max(x.held - x.need, 0);
    }
    block_scan(run, all, scan_buf);
    int taken = 0, n_refused = 0;
    long long blocks[1] = {0}, all_blocks[1];
    for (int b = b0; b < b1; ++b) {
        const Wants x = wants(a, b);
        const int grow = max(x.need - x.held, 0);
        first_row[b] = clip(run[0]);
        first_grow[b] = clip(run[1]);
        first_shrink[b] = clip(run[2]);
        run[0] += x.rows;
        run[1] += grow;
        run[2] += max(x.held - x.need, 0);
        const bool no = x.bad || (grow > 0 && run[1] > free_n);
        if (x.state) bits |= DLLM_SERVE_STATE;
        else if (x.bad) bits |= DLLM_SERVE_LENGTHS;
        else if (no) bits |= DLLM_SERVE_PAGES;
        if (!no && grow > 0) taken = max(taken, static_cast<int>(run[1]));
        n_refused += no;
        refused[b] = no;
        // a request without new tokens has no rows to see its keys
        if (!no && x.rows > 0) blocks[0] += (__ldg(a.len + b) + x.rows + kServeBlock - 1) / kServeBlock;
    }
    if (taken) atomicMax(&s_taken, taken);
    if (n_refused) atomicAdd(&s_refused, n_refused);
    block_scan(blocks, all_blocks, scan_buf);
    if (all_blocks[0] > a.s.max_blocks) bits |= DLLM_SERVE_STATE;  // more keys than the pool has places
    for (int b = b0; b < b1; ++b) {
        first_block[b] = static_cast<int>(min(blocks[0], static_cast<long long>(a.s.max_blocks)));
        const Wants x = wants(a, b);
        if (!refused[b] && x.rows > 0) blocks[0] += (__ldg(a.len + b) + x.rows + kServeBlock - 1) / kServeBlock;
    }
    if (threadIdx.x == 0) {
        first_row[B] = clip(all[0]);
        first_grow[B] = clip(all[1]);
        first_shrink[B] = clip(all[2]);
        first_block[B] = static_cast<int>(min(all_blocks[0], static_cast<long long>(a.s.max_blocks)));
    }
    __syncthreads();
    taken = s_taken;
    const int given = min(first_shrink[B], n_pages), n_blocks = first_block[B];
    const int rows = min(first_row[B], a.rows);
    if (all[0] > a.rows) bits |= DLLM_SERVE_ROWS;

    // page idx of request b after the plan (b not refused, idx below its need)
    auto page_of = [&](int b, int idx) {
        const int h = t.held[b];
        if (idx < h) return t.table[static_cast<size_t>(b) * a.s.max_pages + idx];
        return t.ring[(static_cast<unsigned>(head) + first_grow[b] + (idx - h)) % static_cast<unsigned>(n_pages)];
    };

    if (blockIdx.x == 0) {
        // -------------------------------------------- row starts, key counts, the attention's work
        for (int b = threadIdx.x; b <= B; b += kThreads) {
            t.row_start[b] = first_row[b];
            if (b < B) t.n_keys[b] = refused[b] ? 0 : __ldg(a.len + b) + __ldg(a.q_len + b);
        }
        const int tt = a.s.tile_tokens, tiles = (rows + tt - 1) / tt;
        const int pb = (a.prefix_len + kServeBlock - 1) / kServeBlock;
        long long carry = 0;
        for (int base = 0; base < tiles; base += kThreads) {
            const int tile = base + threadIdx.x;
            long long steps[1] = {0}, sum[1];
            if (tile < tiles) {
                const int tok0 = tile * tt, tok1 = min(tok0 + tt, rows) - 1;
                const int r0 = find(first_row, B, tok0), r1 = find(first_row, B, tok1);
                const int s0 = first_block[r0];
                int s1 = first_block[r1 + 1];
                if (a.causal) {  // the tile's last row sees no further
                    const int seen = __ldg(a.len + r1) + tok1 - first_row[r1] + 1;
                    s1 = min(s1, first_block[r1] + (max(seen, 0) + kServeBlock - 1) / kServeBlock);
                }
                steps[0] = pb + s1 - s0;
                w.tile_first[tile] = steps[0] ? s0 : -1;
                steps[0] = max(steps[0], 1ll);
            }
            block_scan(steps, sum, scan_buf);
            if (tile < tiles) {
                w.tile_cum[tile] = carry + steps[0];
                if (tiles <= kThreads) tile_sum[tile] = steps[0];
            }
            carry += sum[0];
        }
        if (threadIdx.x == 0) {
            w.tile_cum[tiles] = carry;
            tile_sum[min(tiles, kThreads)] = carry;
        }
        __syncthreads();
        const long long total = carry * a.s.Hkv;
        const int ctas = static_cast<int>(min((total + 1) / 2, static_cast<long long>(a.max_ctas)));
        for (int c = threadIdx.x; c < kServeCtas; c += kThreads) {
            int4 d = make_int4(0, 0, 0, 0);
            if (c < ctas) {
                const long long x = c * total / ctas, y = (c + 1) * total / ctas;
                const long long* sums = tiles <= kThreads ? tile_sum : w.tile_cum;
                // tile: the one whose units (all heads) hold step x
                d.x = find(sums, tiles, x / a.s.Hkv);
                const long long steps = sums[d.x + 1] - sums[d.x], in = x - sums[d.x] * a.s.Hkv;
                d.y = static_cast<int>(in / steps);
                d.z = static_cast<int>(in - d.y * steps);
                d.w = static_cast<int>(y - x);
            }
            w.cta[c] = d;
        }
        if (threadIdx.x == 0) {
            w.head->ctas = ctas;
            w.head->causal = a.causal;
            w.head->prefix_len = a.prefix_len;
            w.head->prefix_blocks = pb;
            w.head->tiles = tiles;
            w.head->rows = rows;
            w.head->total = total;
            serve_key(a.s, w.head->shape);
            t.status[1] = s_refused;
            t.status[2] = taken;
            t.status[3] = given;
        }
    }
    if (blockIdx.x > 0 || gridDim.x == 1) {
        // -------------------------------------------- rows, pages, blocks
        const int first = (gridDim.x == 1 ? 0 : blockIdx.x - 1) * kThreads + threadIdx.x;
        const int step = (gridDim.x == 1 ? 1 : gridDim.x - 1) * kThreads;
        for (int r = first; r < a.rows; r += step) {
            int slot = -1, pos = 0, req = -1;
            if (r < rows) {
                req = find(first_row, B, r);
                if (!refused[req]) {
                    const int at = __ldg(a.len + req) + r - first_row[req];
                    const int p = page_of(req, at >> lg);
                    if (p >= 0 && p < n_pages) slot = p * page + (at & (page - 1));
                    else bits |= DLLM_SERVE_STATE;
                    pos = a.prefix_len + at;
                }
            }
            t.slot[r] = slot;
            t.pos[r] = pos;
            t.req[r] = req;
        }
        for (int k = first; k < taken; k += step) {
            const int b = find(first_grow, B, k);
            const int idx = t.held[b] + k - first_grow[b];
            t.table[static_cast<size_t>(b) * a.s.max_pages + idx] =
                t.ring[(static_cast<unsigned>(head) + k) % static_cast<unsigned>(n_pages)];
        }
        for (int k = first; k < given; k += step) {
            const int b = find(first_shrink, B, k);
            const int idx = wants(a, b).need + k - first_shrink[b];
            int* p = t.table + static_cast<size_t>(b) * a.s.max_pages + idx;
            t.ring[(static_cast<unsigned>(head) + free_n + k) % static_cast<unsigned>(n_pages)] = *p;
            *p = -1;
        }
        for (int k = first; k < n_blocks; k += step) {
            const int b = find(first_block, B, k), key0 = (k - first_block[b]) * kServeBlock;
            const int L = __ldg(a.len + b), q = __ldg(a.q_len + b);
            w.info[k] = make_int4(first_row[b], first_row[b + 1], key0, L);
            int4 p = make_int4(-1, -1, -1, -1);
            if (page >= kServeBlock) {
                p.x = page_of(b, key0 >> lg);
                p.y = key0 & (page - 1);
            } else {
                int* pp = &p.x;
                const int last = (L + q - 1) >> lg;
                for (int i = 0; i < kServeBlock >> lg; ++i)
                    if ((key0 >> lg) + i <= last) pp[i] = page_of(b, (key0 >> lg) + i);
            }
            w.pages[k] = p;
        }
    }
    if (bits) atomicOr(t.status, bits);

    // ------------------------------------------------ the state, once every CTA has read it
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        s_last = atomicAdd(&w.head->ticket, 1) == static_cast<int>(gridDim.x) - 1;
    }
    __syncthreads();
    if (!s_last) return;
    for (int b = threadIdx.x; b < B; b += kThreads)
        if (!refused[b]) t.held[b] = wants(a, b).need;
    if (threadIdx.x == 0) {
        t.ring_pos[0] = static_cast<int>((static_cast<unsigned>(head) + taken) % static_cast<unsigned>(n_pages));
        t.ring_pos[1] = min(free_n - taken + given, n_pages);
        w.head->ticket = 0;
    }
}

__global__ void k_serve_reset(ServeShape s, dllm_serve_tables t) {
    const size_t i0 = blockIdx.x * static_cast<size_t>(blockDim.x) + threadIdx.x, n = static_cast<size_t>(gridDim.x) * blockDim.x;
    for (size_t i = i0; i < static_cast<size_t>(s.max_batch) * s.max_pages; i += n) t.table[i] = -1;
    for (size_t i = i0; i < s.max_batch; i += n) t.held[i] = t.n_keys[i] = 0;
    for (size_t i = i0; i <= s.max_batch; i += n) t.row_start[i] = 0;
    for (size_t i = i0; i < s.n_pages; i += n) t.ring[i] = static_cast<int>(i);
    for (size_t i = i0; i < s.max_rows; i += n) {
        t.slot[i] = t.req[i] = -1;
        t.pos[i] = 0;
    }
    if (i0 < 4) t.status[i0] = 0;
    if (i0 < 2) t.ring_pos[i0] = i0 ? s.n_pages : 0;
    if (i0 < sizeof(ServeWork) / 4) t.work[i0] = 0;
}

size_t plan_smem(int batch) {
    return sizeof(long long) * (4 * kWarps + kThreads + 1) + sizeof(int) * 4 * (static_cast<size_t>(batch) + 1) + batch;
}

}  // namespace

cudaError_t launch_serve_reset(const ServeShape& s, const dllm_serve_tables& t, cudaStream_t st) {
    k_serve_reset<<<152, 512, 0, st>>>(s, t);
    return cudaGetLastError();
}

cudaError_t launch_serve_plan(const ServeShape& s, const dllm_serve_tables& t, const int* len, const int* q_len,
                              int batch, int rows, int prefix_len, int causal, int sms, cudaStream_t st) {
    if (plan_smem(batch) > 48 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void*>(k_serve_plan),
                                                   cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                   static_cast<int>(plan_smem(kServeMaxBatch)));
        if (e != cudaSuccess) return e;
    }
    PlanArgs a{s, t, len, q_len, batch, rows, prefix_len, causal, 2 * sms < kServeCtas ? 2 * sms : kServeCtas};
    // one CTA for the work list, and one for every eight items a thread of the others
    const long long items = rows + 64ll * batch;
    long long fill = (items + 8 * kThreads - 1) / (8 * kThreads);
    if (fill > sms - 1) fill = sms - 1;
    if (fill < 1) fill = 1;
    k_serve_plan<<<static_cast<unsigned>(1 + fill), kThreads, plan_smem(batch), st>>>(a);
    return cudaGetLastError();
}

}  // namespace dllm
