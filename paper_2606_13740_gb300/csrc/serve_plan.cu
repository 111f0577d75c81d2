// The plan of a serving step: pages taken and given back, slots and positions of the new tokens, and the
// attention's work list, from the requests' lengths (include/dllm_serve.h, dllm_serve_plan).
//
// Everything follows from running sums over the requests: new tokens, pages taken, pages given back, blocks
// of 64 keys, steps of the attention.  Each CTA makes them all by itself in shared memory (up to 4096
// requests: a few thousand cycles, less than a round of launches or of waiting for one another would cost),
// then fills its share of the rows, pages, blocks and tiles, the owner of an item found by binary search in
// the sums, so that one long request among many short ones spreads over all CTAs.  (One CTA that summed over
// the tiles took 30 us for 19500 of them.)  The state that all CTAs read (held, ring_pos) is replaced by the
// CTA that has read it last.  Pages come from the ring's front and go to its end, so that what a plan takes and what
// it gives back never meet: the free pages and those given back fit into the ring together.
// Bound: latency of that chain.  Measured in a graph: 16 requests of 32 tokens 8.1 us, 1000 ragged prompts 15.0; the CTA that cuts the
// runs ends last, so that fewer or more items a thread for the others change nothing.
#include "serve.cuh"

namespace dllm {

namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kMost = 0x7fffffff;
constexpr int kStart = 10, kPrefix = 5, kOwnStep = 6;  // cost of a unit's start, of a prefix and of an own step (heads of 128)
constexpr int kLeast = 12;                             // of a run

struct PlanArgs {
    ServeShape s;
    dllm_serve_tables t;
    const int* len;
    const int* q_len;
    int batch, rows, prefix_len, causal, max_ctas;
};

// An input: a plain load, which stays behind pdl_wait (a read-only one need not).
__device__ __forceinline__ int load_in(const int* p) { return *p; }
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
    const int L = load_in(a.len + b), q = load_in(a.q_len + b), held = a.t.held[b];
    Wants w;
    w.rows = max(q, 0);
    w.state = held < 0 || held > a.s.max_pages;
    w.held = min(max(held, 0), a.s.max_pages);
    const long long own = static_cast<long long>(L) + q, need = (own + a.s.page - 1) >> a.s.page_log2;
    w.bad = w.state || L < 0 || q < 0 || need > a.s.max_pages || a.prefix_len + own > kMost;
    w.need = w.bad ? w.held : static_cast<int>(need);
    return w;
}

// sum of floor((x + k d) / m), k = 0 .. n - 1: the lattice points under a line.  Whole parts of d / m and x / m come
// out as a closed form; what is left is counted along the other axis, which trades m and d (the reciprocity of such sums,
// Graham, Knuth and Patashnik, Concrete Mathematics, 3.5), so that the steps are those of Euclid's algorithm.
__device__ long long floor_sum(long long n, long long m, long long d, long long x) {
    long long sum = 0;
    while (n > 0) {
        sum += n * (n - 1) / 2 * (d / m) + n * (x / m);
        d %= m;
        x %= m;
        const long long top = d * n + x;  // the line's end; below it the points are counted by columns of height 1
        if (top < m) break;
        n = top / m;
        x = top % m;
        const long long t = m;
        m = d;
        d = t;
    }
    return sum;
}

// Shared memory of a CTA: the sums before each request, and what is read of the requests.
struct Sums {
    long long *scan, *steps;  // [3][kWarps]; [B + 1]: own steps of the tiles of the requests before
    int *row, *grow, *shrink, *block;  // [B + 1]
    int *len, *held;                   // [B]
    uint8_t* refused;                  // [B]
    __device__ Sums(void* base, int B) {
        scan = static_cast<long long*>(base);
        steps = scan + 3 * kWarps;
        row = reinterpret_cast<int*>(steps + B + 1);
        grow = row + B + 1;
        shrink = grow + B + 1;
        block = shrink + B + 1;
        len = block + B + 1;
        held = len + B;
        refused = reinterpret_cast<uint8_t*>(held + B);
    }
};
// static shared memory of k_serve_plan, at most: its two arrays and a few words (a launch counts it too)
constexpr size_t kStaticSmem = sizeof(long long) * (kServeCtas + 1 + kThreads) + 256;
size_t plan_smem(int B) {
    return sizeof(long long) * (3 * kWarps + B + 1) + sizeof(int) * (4 * (static_cast<size_t>(B) + 1) + 2 * B) + B;
}

__global__ void __launch_bounds__(kThreads) k_serve_plan(const __grid_constant__ PlanArgs a) {
    extern __shared__ long long smem[];
    const int B = a.batch;
    const Sums u(smem, B);
    __shared__ int s_taken, s_refused, s_last, s_joins;
    __shared__ long long begin[kServeCtas + 1], sampled[kThreads];  // a run's first step among all; costs before some tiles

    const dllm_serve_tables& t = a.t;
    const int n_pages = a.s.n_pages, page = a.s.page, lg = a.s.page_log2, tt = a.s.tile_tokens;
    ServeArrays w;
    serve_arrays(a.s, t.work, &w);
    if (threadIdx.x == 0) s_taken = s_refused = 0;
    int bits = 0;
    pdl_wait();

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
    block_scan(run, all, u.scan);
    int taken = 0, n_refused = 0;
    // Blocks of a request that has rows to see them; a refused one has an empty block, so that every tile has a
    // step.  And their steps, tile by tile: all blocks in the last of its tiles (and, not causal, in all of
    // them); causal, in the tiles before, up to the tile's last row.
    auto blocks_of = [&](int rows, int L, bool no) { return rows == 0 ? 0 : no ? 1 : static_cast<int>((static_cast<unsigned>(L) + rows + kServeBlock - 1) / kServeBlock); };
    auto steps_of = [&](int n_blocks, int row0, int rows, int L, bool no, int tiles) {  // of its first `tiles` tiles
        if (rows == 0) return 0ll;
        // tiles but the last (a row's number past 2^31, of a request that is refused, is past the plan's rows)
        const unsigned end = static_cast<unsigned>(row0) + static_cast<unsigned>(rows) - 1u;
        const int first = row0 / tt, whole = static_cast<int>(min(end / static_cast<unsigned>(tt), kMost - 1u)) - first;
        if (!a.causal || no) return static_cast<long long>(n_blocks) * min(tiles, whole + 1);
        const long long seen = static_cast<long long>(L) - row0 + (first + 1ll) * tt;  // keys, first tile
        return floor_sum(min(tiles, whole), kServeBlock, tt, seen + kServeBlock - 1) + (tiles > whole ? n_blocks : 0);
    };
    long long more[2] = {0, 0}, all_more[2];
    for (int b = b0; b < b1; ++b) {
        const Wants x = wants(a, b);
        const int grow = max(x.need - x.held, 0), L = load_in(a.len + b);
        u.row[b] = clip(run[0]);
        u.grow[b] = clip(run[1]);
        u.shrink[b] = clip(run[2]);
        u.len[b] = L;
        u.held[b] = x.held;
        run[1] += grow;
        const bool no = x.bad || (grow > 0 && run[1] > free_n);
        if (x.state) bits |= DLLM_SERVE_STATE;
        else if (x.bad) bits |= DLLM_SERVE_LENGTHS;
        else if (no) bits |= DLLM_SERVE_PAGES;
        if (!no && grow > 0) taken = max(taken, static_cast<int>(run[1]));
        n_refused += no;
        u.refused[b] = no;
        const int n = blocks_of(x.rows, L, no);
        more[0] += n;
        more[1] += steps_of(n, u.row[b], x.rows, L, no, kMost);
        run[0] += x.rows;
        run[2] += max(x.held - x.need, 0);
    }
    if (taken) atomicMax(&s_taken, taken);
    if (n_refused) atomicAdd(&s_refused, n_refused);
    block_scan(more, all_more, u.scan);
    for (int b = b0; b < b1; ++b) {
        u.block[b] = clip(more[0]);
        u.steps[b] = more[1];
        const int rows = max(load_in(a.q_len + b), 0), n = blocks_of(rows, u.len[b], u.refused[b]);
        more[0] += n;
        more[1] += steps_of(n, u.row[b], rows, u.len[b], u.refused[b], kMost);
    }
    if (threadIdx.x == 0) {
        u.row[B] = clip(all[0]);
        u.grow[B] = clip(all[1]);
        u.shrink[B] = clip(all[2]);
        u.block[B] = clip(all_more[0]);
        u.steps[B] = all_more[1];
    }
    __syncthreads();
    // The CTA has read the state (held is in shared memory): the last one to say so replaces it.  By a thread that
    // has no run to find; its ticket is looked at when all else is done.
    int ticket = 0;
    if (threadIdx.x == kThreads - 1) {
        __threadfence();
        ticket = atomicAdd(&w.head->ticket, 1);
    }
    auto need_of = [&](int b) {  // pages wanted by a request that is not refused
        return static_cast<int>((static_cast<long long>(u.len[b]) + load_in(a.q_len + b) + page - 1) >> lg);
    };
    taken = s_taken;
    const int given = min(u.shrink[B], n_pages), rows = min(u.row[B], a.rows);
    if (all[0] > a.rows) bits |= DLLM_SERVE_ROWS;
    const bool fits = all_more[0] <= a.s.max_blocks;  // else there are more keys than the pool has places: no work list
    if (!fits) bits |= DLLM_SERVE_STATE;
    const int n_blocks = fits ? u.block[B] : 0, tiles = fits ? (rows + tt - 1) / tt : 0;
    const int pb = (a.prefix_len + kServeBlock - 1) / kServeBlock;

    // page idx of request b after the plan (b not refused, idx below its need)
    auto page_of = [&](int b, int idx) {
        const int h = u.held[b];
        if (idx < h) return t.table[static_cast<size_t>(b) * a.s.max_pages + idx];
        return t.ring[(static_cast<unsigned>(head) + u.grow[b] + (idx - h)) % static_cast<unsigned>(n_pages)];
    };
    // steps of a K/V head's tiles before tile i
    auto cum = [&](int i) {
        const long long own = static_cast<long long>(i) * tt;
        long long n = static_cast<long long>(i) * pb;
        if (own >= u.row[B]) return n + u.steps[B];
        const int b = find(u.row, B, static_cast<int>(own));
        return n + u.steps[b] + steps_of(u.block[b + 1] - u.block[b], u.row[b], u.row[b + 1] - u.row[b], u.len[b], u.refused[b],
                                         i - u.row[b] / tt);
    };

    if (blockIdx.x == 0) {
        // -------------------------------------------- row starts, the CTAs' runs
        for (int b = threadIdx.x; b <= B; b += kThreads) t.row_start[b] = u.row[b];
        // The cost of a unit: its start, its prefix steps, its own steps; of all units of the tiles before tile i.
        // (Measured at heads of 128, in prefix steps of 0.78 us: an own step 1.17, a unit's start and end 1.5 to 2.7.  Cut by steps
        // alone, the CTAs of 16 windows of 32 under 4096 shared keys ended between 34 and 47 us.)
        auto cost_of = [&](int i, long long steps) {  // of tile i, with cum(i)
            return i * (kStart + kPrefix * static_cast<long long>(pb)) + kOwnStep * (steps - static_cast<long long>(i) * pb);
        };
        // at kThreads tiles side by side, so that a run's search goes over few of the others
        const int stride = (tiles + kThreads - 1) / kThreads, samples = tiles ? (tiles + stride - 1) / stride : 0;
        if (static_cast<int>(threadIdx.x) < samples) sampled[threadIdx.x] = cost_of(threadIdx.x * stride, cum(threadIdx.x * stride));
        const long long per_head = tiles ? cum(tiles) : 0, total = per_head * a.s.Hkv, all_cost = cost_of(tiles, per_head) * a.s.Hkv;
        // (no run of less than two steps, so that only a run that begins where a unit does may be empty)
        const int ctas = static_cast<int>(min(all_cost ? max(all_cost / kLeast, 1ll) : 0ll, static_cast<long long>(a.max_ctas)));
        int4 d = make_int4(0, 0, 0, 0), e = d;
        long long unit0 = 0;  // the first step of the unit that this thread's run begins in
        static_assert(kServeCtas < kThreads, "a thread a run");
        const int c = threadIdx.x;
        __syncthreads();
        if (c <= kServeCtas) {
            begin[c] = total;
            if (c < ctas) {
                const long long x = all_cost / ctas * c + all_cost % ctas * c / ctas, own = x / a.s.Hkv;
                int lo = samples > 1 ? find(sampled, samples, own) * stride : 0, hi = min(lo + stride, tiles);
                while (hi - lo > 1) {  // the tile whose units (all heads) hold cost x
                    const int mid = (lo + hi) >> 1;
                    if (cost_of(mid, cum(mid)) <= own) lo = mid;
                    else hi = mid;
                }
                const long long steps0 = cum(lo), steps1 = lo + 1 == tiles ? per_head : cum(lo + 1), steps = steps1 - steps0;
                const long long at = cost_of(lo, steps0), unit = cost_of(lo + 1, steps1) - at, in = x - at * a.s.Hkv;
                d.x = lo;
                d.y = static_cast<int>(in / unit);
                const long long o = max(in - d.y * unit - kStart, 0ll);
                d.z = static_cast<int>(o < kPrefix * static_cast<long long>(pb) ? o / kPrefix : pb + (o - kPrefix * static_cast<long long>(pb)) / kOwnStep);
                unit0 = steps0 * a.s.Hkv + d.y * steps;
                begin[c] = unit0 + d.z;
                e = make_int4(u.block[find(u.row, B, lo * tt)], static_cast<int>(steps), 0, 0);
            }
        }
        if (threadIdx.x == 0) s_joins = 0;
        __syncthreads();
        if (c < kServeCtas) {
            if (c < ctas) d.w = static_cast<int>(begin[c + 1] - begin[c]);
            w.cta[2 * c] = d;
            w.cta[2 * c + 1] = e;
            // a unit's second part: a run that begins inside it, the one before (the last that begins at or before
            // the unit does) holding its first step
            if (c < ctas && c > 0 && d.z > 0 && begin[c - 1] <= unit0)
                w.join[atomicAdd(&s_joins, 1)] = make_int4(d.x, d.y, c - 1, find(begin, ctas, unit0 + e.y - 1));
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            w.head->ctas = ctas;
            w.head->causal = a.causal;
            w.head->prefix_len = a.prefix_len;
            w.head->prefix_blocks = pb;
            w.head->tiles = tiles;
            w.head->rows = fits ? rows : 0;
            w.head->total = total;
            w.head->joins = s_joins;
            serve_key(a.s, w.head->shape);
            t.status[1] = s_refused;
            t.status[2] = taken;
            t.status[3] = given;
        }
    } else {
        // -------------------------------------------- rows, pages, blocks, tiles
        const int first = (blockIdx.x - 1) * kThreads + threadIdx.x, step = (gridDim.x - 1) * kThreads;
        for (int r = first; r < a.rows; r += step) {
            int slot = -1, pos = 0, req = -1;
            if (r < rows) {
                req = find(u.row, B, r);
                if (!u.refused[req]) {
                    const int at = u.len[req] + r - u.row[req];
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
            const int b = find(u.grow, B, k);
            const int idx = u.held[b] + k - u.grow[b];
            t.table[static_cast<size_t>(b) * a.s.max_pages + idx] =
                t.ring[(static_cast<unsigned>(head) + k) % static_cast<unsigned>(n_pages)];
        }
        for (int k = first; k < given; k += step) {
            const int b = find(u.shrink, B, k);
            const int idx = need_of(b) + k - u.shrink[b];
            int* p = t.table + static_cast<size_t>(b) * a.s.max_pages + idx;
            t.ring[(static_cast<unsigned>(head) + free_n + k) % static_cast<unsigned>(n_pages)] = *p;
            *p = -1;
        }
        for (int k = first; k < n_blocks; k += step) {
            const int b = find(u.block, B, k), key0 = (k - u.block[b]) * kServeBlock;
            const int q = u.row[b + 1] - u.row[b], L = u.refused[b] ? -q : u.len[b];  // (refused: no keys)
            w.info[k] = make_int4(u.row[b], u.row[b + 1], key0, L);
            int4 p = make_int4(-1, page >= kServeBlock ? key0 & (page - 1) : -1, -1, -1);
            if (!u.refused[b]) {
                if (page >= kServeBlock) {
                    p.x = page_of(b, key0 >> lg);
                } else {
                    int* pp = &p.x;
                    const int last = (L + q - 1) >> lg;
                    for (int i = 0; i < kServeBlock >> lg; ++i)
                        if ((key0 >> lg) + i <= last) pp[i] = page_of(b, (key0 >> lg) + i);
                }
            }
            w.pages[k] = p;
            if (!u.refused[b]) {  // pages outside the pool read as zeros, and are reported
                const int n_own = page >= kServeBlock ? 1 : min(kServeBlock >> lg, ((L + q - 1) >> lg) - (key0 >> lg) + 1);
                const int id[4] = {p.x, n_own > 1 ? p.y : 0, n_own > 2 ? p.z : 0, n_own > 3 ? p.w : 0};
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (id[i] < 0 || id[i] >= n_pages) bits |= DLLM_SERVE_STATE;
            }
        }
        for (int k = first; k < tiles; k += step)
            w.tile[k] = make_int2(u.block[find(u.row, B, k * tt)], static_cast<int>(cum(k + 1) - cum(k)));
    }
    if (bits) atomicOr(t.status, bits);

    // ------------------------------------------------ the state, by the CTA that read it last (and the key counts, which
    // may be the next plan's lengths)
    if (threadIdx.x == kThreads - 1) s_last = ticket == static_cast<int>(gridDim.x) - 1;
    __syncthreads();
    if (!s_last) return;
    for (int b = threadIdx.x; b < B; b += kThreads) {
        if (!u.refused[b]) t.held[b] = need_of(b);
        t.n_keys[b] = u.refused[b] ? 0 : u.len[b] + load_in(a.q_len + b);
    }
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

}  // namespace

cudaError_t launch_serve_reset(const ServeShape& s, const dllm_serve_tables& t, cudaStream_t st) {
    k_serve_reset<<<152, 512, 0, st>>>(s, t);
    return cudaGetLastError();
}

cudaError_t launch_serve_plan(const ServeShape& s, const dllm_serve_tables& t, const int* len, const int* q_len,
                              int batch, int rows, int prefix_len, int causal, int sms, cudaStream_t st) {
    if (plan_smem(batch) + kStaticSmem > 48 * 1024) {  // has to be asked for: the most of any batch
        const cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void*>(k_serve_plan),
                                                   cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                   static_cast<int>(plan_smem(kServeMaxBatch)));
        if (e != cudaSuccess) return e;
    }
    PlanArgs a{s, t, len, q_len, batch, rows, prefix_len, causal, 2 * sms < kServeCtas ? 2 * sms : kServeCtas};
    // one CTA for the runs, and one for every two items a thread of the others
    const long long items = rows + 64ll * batch;
    long long fill = (items + 2 * kThreads - 1) / (2 * kThreads);
    if (fill > sms - 1) fill = sms - 1;
    if (fill < 1) fill = 1;
    return serve_launch(k_serve_plan, dim3(static_cast<unsigned>(1 + fill)), kThreads, plan_smem(batch), st, a);
}

}  // namespace dllm
