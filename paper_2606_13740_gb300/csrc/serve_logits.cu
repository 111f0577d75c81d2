// Logits of a serving step: penalties for repeated ids, biases, grammar masks, and the decision, in one
// pass over them (include/dllm_serve.h, dllm_serve_logits).
//
// A CTA takes a stretch of the vocabulary for some rows.  What the rows' request asks for there (how often
// an id stands in its history, which of its biases names it) is one 32-bit word an id in shared memory, made
// once for all the request's rows in the CTA: count in the low 20 bits, 1 + index of the bias above; and a bit
// an id says whether there is anything.  Sums, maxima and bits do not depend on the order in which threads
// add them.  Then warps stream the rows, several to a row where rows are few, and keep a running maximum, sum
// of exponentials and argmax in registers.  The ids asked for, few among many, leave that stream and are
// taken 32 at a time from a list, in a fixed order: treated in the stream, they cost a warp the division for
// nearly every 512 ids (20 instructions an id, 69 us for 512 rows of 126464).  k_merge joins a row's
// stretches.  Bound: memory (logits once in, once out when asked for) and, with long lists, what each CTA does before it
// streams: words, history, list.  Measured in a graph: 512 rows of 126464 32-bit ids 61.5 us (262 MB, 4.3 TB/s; 47 with
// nothing asked for; 1024 CTAs on 608 places, DRAM 58 % busy, issue slots 44); 96 single bf16 rows of 152064 ids with
// 5000 ids of history each, written out, 38.2 us (11 with nothing asked for, in L2).
// (Clusters of 8 stretches that each read an eighth of a history and count in one another's shared memory: 61 us, as half
// of a history falls into one stretch, which all of the cluster then waits for.)
#include "serve.cuh"

namespace dllm {

namespace {

constexpr int kThreads = 256;  // at most
constexpr int kWarps = kThreads / 32;
constexpr int kChunk = 8192;  // ids of a stretch, at most: 32 KB of words
constexpr int kGroup = 128;   // ids that a warp takes side by side, 4 a lane
constexpr int kGroups = 4;    // of these in flight together
constexpr int kPiece = kGroup * kGroups;
constexpr int kCountBits = 20;
constexpr float kLog2e = 1.4426950408889634f;

struct alignas(16) Part {
    float m, s;  // largest z, sum of exp(z - m)
    int arg, pad;
};

// How a call is cut: stretches of `chunk` ids, `rows_cta` rows a CTA of `warps` warps, `split` warps a row and
// stretch.
struct Cut {
    int chunk, chunks, rows_cta, warps, split;
    int list;  // places for the ids that a stretch may be asked for
};

// 2^x by the special function unit; below 2^-126: 0 (nothing beside the largest, 1)
__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
template <typename T>
struct Io;
template <>
struct Io<float> {
    typedef float4 Raw;  // four values as they lie in memory
    static __device__ __forceinline__ float get(const float* p) { return *p; }
    static __device__ __forceinline__ void put(float* p, float v) { *p = v; }
    static __device__ __forceinline__ void floats(Raw f, float* v) { v[0] = f.x, v[1] = f.y, v[2] = f.z, v[3] = f.w; }
    static __device__ __forceinline__ void put4(float* p, const float* v) {
        *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    }
};
template <typename T>
struct Io16 {
    typedef uint2 Raw;
    static __device__ __forceinline__ float get(const T* p) { return static_cast<float>(*p); }
    static __device__ __forceinline__ void floats(Raw u, float* v) {
        const float2 a = Half2<T>::unpack(u.x), b = Half2<T>::unpack(u.y);
        v[0] = a.x, v[1] = a.y, v[2] = b.x, v[3] = b.y;
    }
    static __device__ __forceinline__ void put4(T* p, const float* v) {
        uint2 u;
        u.x = Half2<T>::pack(v[0], v[1]);
        u.y = Half2<T>::pack(v[2], v[3]);
        *reinterpret_cast<uint2*>(p) = u;
    }
};
template <>
struct Io<__nv_bfloat16> : Io16<__nv_bfloat16> {
    static __device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
};
template <>
struct Io<__half> : Io16<__half> {
    static __device__ __forceinline__ void put(__half* p, float v) { *p = __float2half_rn(v); }
};

// exp(a - m), 0 for a = -inf whatever m
__device__ __forceinline__ float exp_below(float a, float m) { return a == -INFINITY ? 0.0f : exp2f((a - m) * kLog2e); }

// Bits of the ids: the 16 words of a 512-id piece in the order (quarter of 32 lanes, group), so that a lane's
// four words, one a group, lie side by side.  (Its own inverse.)
__device__ __forceinline__ int bit_word(int w) { return (w & ~15) | ((w & 3) << 2) | ((w >> 2) & 3); }

// A running sum of exp(z - ref).  ref is the first values' maximum and moves only when a value exceeds it by more
// than 40, so that a warp seldom leaves its straight path (with the running maximum itself some lane of 32 has a
// new one at nearly every step of 512 ids).  Where ref log2(e) is a finite number (plain) the sum is of
// 2^(z log2(e) - hi), hi the rounded ref log2(e): one FMA an exponent, as exact for a large ref as for a small one,
// and total() makes good what the rounding of hi took.  Else (the type's lowest value, infinities) it is of
// exp(z - ref) itself.
struct Running {
    float ref = -INFINITY, hi = 0.0f, s = 0.0f;
    __device__ bool plain() const { return fabsf(hi) < INFINITY; }
    __device__ float rest() const { return fmaf(ref, kLog2e, -hi); }  // ref log2(e) - hi
    __device__ float total() const { return ref == -INFINITY || !plain() ? s : s * ex2(-rest()); }
    __device__ bool above(float y) const { return y > ref + 40.0f; }
    __device__ void raise(float y) {
        s = total() * exp_below(ref, y);
        ref = y;
        hi = y * kLog2e;
        if (plain()) s *= ex2(rest());
    }
    __device__ float weight(float y) const { return plain() ? ex2(fmaf(y, kLog2e, -hi)) : exp_below(y, ref); }
};

template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads, 4) k_logits(const __grid_constant__ dllm_serve_logits_args a, Cut cut,
                                                     Part* __restrict__ part, float* __restrict__ zcur) {
    extern __shared__ __align__(16) uint32_t word[];  // [cut.chunk]
    uint32_t* bits = word + cut.chunk;                // [cut.chunk / 32], in the order of bit_word
    uint16_t* list = reinterpret_cast<uint16_t*>(bits + cut.chunk / 32);  // [cut.list]: the ids asked for
    __shared__ int s_count[kWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = cut.warps * 32;
    const int v0 = blockIdx.y * cut.chunk, v1 = min(a.vocab, v0 + cut.chunk), n = v1 - v0;
    const int row0 = blockIdx.x * cut.rows_cta, row1 = min(a.rows, row0 + cut.rows_cta);
    const int words = (a.vocab + 31) / 32, pieces = (n + kPiece - 1) / kPiece;

    pdl_wait();  // (inputs by plain loads, which stay behind it)
    int r0 = row0;
    while (r0 < row1) {
        // the run of rows of one request (without lists: all rows)
        const int req = a.req ? a.req[r0] : r0;
        int r1 = a.hist || a.bias_ids ? r0 + 1 : row1;
        while (r1 < row1 && (a.req ? a.req[r1] : r1) == req) ++r1;
        const bool asks = req >= 0 && req < a.n_req && (a.hist || a.bias_ids);
        int n_list = 0;
        if (asks) {
            const int n_bias = !a.bias_ids ? 0 : a.bias_len ? min(max(a.bias_len[req], 0), a.bias_ld) : a.bias_ld;
            const int n_hist = !a.hist ? 0 : a.hist_len ? min(max(a.hist_len[req], 0), a.hist_ld) : a.hist_ld;
            for (int i = tid; i < (cut.chunk + cut.chunk / 32) / 4; i += threads) reinterpret_cast<uint4*>(word)[i] = make_uint4(0, 0, 0, 0);
            // the history in whole 16-byte pieces, and what is before and behind them; the first of them on their way
            // while the biases are marked
            const int* h = a.hist + static_cast<size_t>(req) * a.hist_ld;
            const int lead = min(n_hist, static_cast<int>((16 - reinterpret_cast<uintptr_t>(h) % 16) % 16 / 4));
            const int n4 = (n_hist - lead) / 4, tail = n_hist - lead - 4 * n4;
            const int4* h4 = reinterpret_cast<const int4*>(h + lead);
            constexpr int kAhead = 4;
            int4 x[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) x[k] = tid + k * threads < n4 ? h4[tid + k * threads] : make_int4(-1, -1, -1, -1);
            const int* ids = a.bias_ids + static_cast<size_t>(req) * a.bias_ld;
            int id = tid < n_bias ? ids[tid] : -1;
            __syncthreads();
            for (int i = tid; i < n_bias; i += threads, id = i < n_bias ? ids[i] : -1) {
                const unsigned v = static_cast<unsigned>(id - v0);
                if (v < static_cast<unsigned>(n) && id >= 0) {
                    atomicMax(&word[v], static_cast<uint32_t>(i + 1) << kCountBits);
                    atomicOr(&bits[bit_word(v >> 5)], 1u << (v & 31));
                }
            }
            __syncthreads();
            auto count = [&](int id) {
                const unsigned v = static_cast<unsigned>(id - v0);
                if (v < static_cast<unsigned>(n) && id >= 0) {
                    atomicAdd(&word[v], 1u);
                    atomicOr(&bits[bit_word(v >> 5)], 1u << (v & 31));
                }
            };
            if (tid < lead) count(h[tid]);
            if (tid < tail) count(h[lead + 4 * n4 + tid]);
            for (int i = tid;;) {
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    if (i + k * threads >= n4) break;
                    count(x[k].x);
                    count(x[k].y);
                    count(x[k].z);
                    count(x[k].w);
                }
                i += kAhead * threads;
                if (i >= n4) break;
#pragma unroll
                for (int k = 0; k < kAhead; ++k) x[k] = i + k * threads < n4 ? h4[i + k * threads] : make_int4(-1, -1, -1, -1);
            }
            __syncthreads();
            // the list, in the order of the bits
            int base = 0;
            for (int i0 = 0; i0 < 16 * pieces; i0 += threads) {
                const int i = i0 + tid;
                uint32_t b = i < 16 * pieces ? bits[i] : 0u;
                const int c = __popc(b);
                int upto = c;
#pragma unroll
                for (int d = 1; d < 32; d *= 2) {
                    const int o = __shfl_up_sync(0xffffffffu, upto, d);
                    if (lane >= d) upto += o;
                }
                if (lane == 31) s_count[warp] = upto;
                __syncthreads();
                int at = base + upto - c;
                for (int w = 0; w < cut.warps; ++w) {
                    if (w < warp) at += s_count[w];
                    base += s_count[w];
                }
                for (const int v = bit_word(i) * 32; b; b &= b - 1) list[at++] = static_cast<uint16_t>(v + __ffs(b) - 1);
                __syncthreads();
            }
            n_list = base;
        }
        const float rep = asks && a.rep ? a.rep[req] : 1.0f;
        const float freq = asks && a.freq ? a.freq[req] : 0.0f;
        const float pres = asks && a.pres ? a.pres[req] : 0.0f;
        const float* bias = a.bias_ids && asks ? a.bias + static_cast<size_t>(req) * a.bias_ld : nullptr;

        // warp jobs: (row, share of the stretch), shares of whole pieces
        const int jobs = (r1 - r0) * cut.split;
        for (int job0 = 0; job0 < jobs; job0 += cut.warps) {
            const bool mine = job0 + warp < jobs;  // else nothing to do but the barrier
            const int job = mine ? job0 + warp : 0, row = r0 + job / cut.split, share = job % cut.split;
            const int p0 = pieces * share / cut.split, p1 = mine ? pieces * (share + 1) / cut.split : p0;
            const T* src = static_cast<const T*>(a.logits) + static_cast<size_t>(row) * a.ld + v0;
            T* dst = a.out ? static_cast<T*>(a.out) + static_cast<size_t>(row) * a.ld_out + v0 : nullptr;
            const int g = a.grammar ? a.grammar_row[row] : -1;
            const uint32_t* allow = g >= 0 && g < a.n_grammar ? a.grammar + static_cast<size_t>(g) * words + v0 / 32 : nullptr;
            const int cur = a.cur ? a.cur[row] - v0 : -1, mask = a.mask_id < 0 ? -1 : a.mask_id - v0;
            Running run;
            // the stream's largest value, and the first piece that has it; that of ids taken one by one, and the id
            float best = -INFINITY, best_one = -INFINITY;
            int best_piece = -1, arg = kChunk;

            // The stream: the whole pieces; what is in the list is left out, and the mask id of the decision.
            const int pm = mask >= 0 && mask < n ? mask / kPiece : -1, pw = min(p1, n / kPiece);
            auto load = [&](const T* p, float (&z)[kGroups][4]) {
#pragma unroll
                for (int u = 0; u < kGroups; ++u) {
                    if constexpr (VEC) {
                        Io<T>::floats(*reinterpret_cast<const typename Io<T>::Raw*>(p + u * kGroup), z[u]);
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i) z[u][i] = Io<T>::get(p + u * kGroup + i);
                    }
                }
            };
            auto asked_of = [&](int q) {  // bit 4 u + i: value i of group u is in the list
                const uint4 b = *reinterpret_cast<const uint4*>(bits + 16 * q + 4 * (lane >> 3));
                const int sh = 4 * lane & 31;
                return !(b.x | b.y | b.z | b.w) ? 0u
                                                : ((b.x >> sh) & 15u) | ((b.y >> sh) & 15u) << 4 | ((b.z >> sh) & 15u) << 8 |
                                                      ((b.w >> sh) & 15u) << 12;
            };
            auto only_allowed = [&](int q, float (&z)[kGroups][4]) {
#pragma unroll
                for (int u = 0; u < kGroups; ++u) {
                    const uint32_t ok = allow[16 * q + 4 * u + (lane >> 3)] >> (4 * lane & 31);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!((ok >> i) & 1u)) z[u][i] = -INFINITY;
                }
            };
            auto stream = [&](auto with_list, auto with_grammar, auto with_out) {
                float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                const T* ps = src + p0 * kPiece + 4 * lane;
                for (int q = p0; q < pw; ++q, ps += kPiece) {
                    float z[kGroups][4];
                    load(ps, z);
                    uint32_t todo = 0;
                    if constexpr (decltype(with_list)::value) todo = asked_of(q);
                    if constexpr (decltype(with_grammar)::value) only_allowed(q, z);
                    if constexpr (decltype(with_out)::value) {
                        T* pd = dst + q * kPiece + 4 * lane;
#pragma unroll
                        for (int u = 0; u < kGroups; ++u) {  // (those in the list too, whose values follow)
                            if constexpr (VEC) {
                                Io<T>::put4(pd + u * kGroup, z[u]);
                            } else {
#pragma unroll
                                for (int i = 0; i < 4; ++i) Io<T>::put(pd + u * kGroup + i, z[u][i]);
                            }
                        }
                    }
                    if constexpr (decltype(with_list)::value) {
                        if (todo) {
#pragma unroll
                            for (int u = 0; u < kGroups; ++u)
#pragma unroll
                                for (int i = 0; i < 4; ++i)
                                    if ((todo >> (4 * u + i)) & 1u) z[u][i] = -INFINITY;
                        }
                    }
                    if (q == pm) {
#pragma unroll
                        for (int u = 0; u < kGroups; ++u)
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if (mask == q * kPiece + u * kGroup + 4 * lane + i) z[u][i] = -INFINITY;
                    }
                    float mx = z[0][0];
#pragma unroll
                    for (int u = 0; u < kGroups; ++u) mx = fmaxf(fmaxf(fmaxf(mx, z[u][0]), z[u][1]), fmaxf(z[u][2], z[u][3]));
                    if (mx > best) {
                        best = mx;
                        best_piece = q;
                    }
                    if (run.above(mx)) {
                        run.s += (s[0] + s[1]) + (s[2] + s[3]);
                        s[0] = s[1] = s[2] = s[3] = 0.0f;
                        run.raise(mx);
                    }
#pragma unroll
                    for (int u = 0; u < kGroups; ++u)
#pragma unroll
                        for (int i = 0; i < 4; ++i) s[i] += ex2(fmaf(z[u][i], kLog2e, -run.hi));
                }
                run.s += (s[0] + s[1]) + (s[2] + s[3]);
            };
            const std::true_type yes;
            const std::false_type no;
            if (asks) {
                if (allow) dst ? stream(yes, yes, yes) : stream(yes, yes, no);
                else dst ? stream(yes, no, yes) : stream(yes, no, no);
            } else {
                if (allow) dst ? stream(no, yes, yes) : stream(no, yes, no);
                else dst ? stream(no, no, yes) : stream(no, no, no);
            }
            // One id with its value, all asked of it done: into out, the decision, the sum.
            auto one = [&](int v, float y) {
                if (allow && !((allow[v >> 5] >> (v & 31)) & 1u)) y = -INFINITY;
                if (dst) Io<T>::put(dst + v, y);
                if (v == cur) zcur[row] = y;
                if (v == mask) y = -INFINITY;
                if (y > best_one) {
                    best_one = y;
                    arg = v;
                } else if (y == best_one) {
                    arg = min(arg, v);
                }
                if (run.above(y)) run.raise(y);
                run.s += run.weight(y);
            };
            auto by_ones = [&](int p) {  // a piece that is not whole
                const int end = min(n, (p + 1) * kPiece);
                for (int v = p * kPiece + lane; v < end; v += 4 * 32) {
                    float y[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) y[i] = v + 32 * i < end ? Io<T>::get(src + v + 32 * i) : 0.0f;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (v + 32 * i < end && (!asks || !word[v + 32 * i])) one(v + 32 * i, y[i]);
                }
            };
            if (__any_sync(0xffffffffu, !run.plain())) {  // (the stream's exponents are for finite ones)
                run = Running();
                best = -INFINITY;
                for (int p = p0; p < p1; ++p) by_ones(p);
            } else if (pw < p1) {
                by_ones(pw);
            }
            // the current id, if the stream had it
            if (lane == 0 && cur >= p0 * kPiece && cur < min(n, p1 * kPiece) && !(asks && word[cur]))
                zcur[row] = allow && !((allow[cur >> 5] >> (cur & 31)) & 1u) ? -INFINITY : Io<T>::get(src + cur);
            // The ids asked for, spread over the row's warps whatever pieces they lie in (half of a history falls into
            // a few hundred ids).  Their stores come behind the stream's, which wrote them as they were, so that their
            // values are there still where out is logits.  Four gathers a lane in flight.
            if (asks) {
                if (cut.split > 1 && a.out) __syncthreads();
                else __syncwarp();
                constexpr int kIds = 4;
                for (int k0 = mine ? share * 32 + lane : n_list; k0 < n_list; k0 += kIds * 32 * cut.split) {
                    int v[kIds];
                    float y[kIds];
#pragma unroll
                    for (int i = 0; i < kIds; ++i) {
                        const int k = k0 + i * 32 * cut.split;
                        v[i] = k < n_list ? list[k] : -1;
                        y[i] = v[i] >= 0 ? Io<T>::get(src + v[i]) : -INFINITY;
                    }
#pragma unroll
                    for (int i = 0; i < kIds; ++i) {
                        if (v[i] < 0) break;
                        const uint32_t x = word[v[i]], c = x & ((1u << kCountBits) - 1), nth = x >> kCountBits;
                        float f = y[i];
                        if (c) {
                            f = f > 0.0f ? __fdiv_rn(f, rep) : __fmul_rn(f, rep);
                            f = __fsub_rn(f, __fadd_rn(__fmul_rn(freq, static_cast<float>(c)), pres));
                        }
                        if (nth) f = __fadd_rn(f, bias[nth - 1]);
                        one(v[i], f);
                    }
                }
            }
            // the warp's lanes: the largest value, its first id, the sum
            float m = fmaxf(best, best_one);
#pragma unroll
            for (int d = 16; d; d /= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
            if (best_one != m) arg = kChunk;
            if (best == m && best_piece >= 0) {
                float z[kGroups][4];
                load(src + best_piece * kPiece + 4 * lane, z);
                if (allow) only_allowed(best_piece, z);
                const uint32_t todo = asks ? asked_of(best_piece) : 0u;
#pragma unroll
                for (int u = kGroups - 1; u >= 0; --u)
#pragma unroll
                    for (int i = 3; i >= 0; --i)
                        {
                        const int v = best_piece * kPiece + 4 * lane + u * kGroup + i;
                        if (z[u][i] == m && v != mask && !((todo >> (4 * u + i)) & 1u)) arg = min(arg, v);
                    }
            }
            __syncwarp();
            arg = __reduce_min_sync(0xffffffffu, arg);
            float sum = run.total() * exp_below(run.ref, m);
            if (run.ref == -INFINITY) sum = run.s;  // nothing but -inf: 0, or NaN
#pragma unroll
            for (int d = 16; d; d /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            if (lane == 0 && mine)
                part[(static_cast<size_t>(row) * cut.chunks + blockIdx.y) * cut.split + share] =
                    Part{m, sum, arg < kChunk ? v0 + arg : -1, 0};
        }
        __syncthreads();
        r0 = r1;
    }
}

// A warp joins a row's parts (in order of ids).  A row whose grammar there is not, which allows no id, has passed
// k_logits as one without a grammar: here it gets its -inf and its decision.
template <typename T>
__global__ void __launch_bounds__(128) k_merge(const __grid_constant__ dllm_serve_logits_args a, int parts,
                                               const Part* part, const float* zcur) {
    pdl_wait();
    const int row = blockIdx.x * 4 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (row >= a.rows) return;
    const int g = a.grammar ? a.grammar_row[row] : -1;  // (looked at when the parts are there)
    float m = -INFINITY, s = 0.0f;
    int arg = a.vocab;
    constexpr int kAtOnce = 8;
    for (int i0 = lane; i0 < parts; i0 += 32 * kAtOnce) {
        Part p[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k)
            p[k] = i0 + 32 * k < parts ? part[static_cast<size_t>(row) * parts + i0 + 32 * k] : Part{-INFINITY, 0.0f, 0, 0};
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const float mx = fmaxf(m, p[k].m);
            s = s * (m == mx ? 1.0f : exp_below(m, mx)) + p[k].s * (p[k].m == mx ? 1.0f : exp_below(p[k].m, mx));
            if (p[k].m > m) arg = p[k].arg;
            m = mx;
        }
    }
#pragma unroll
    for (int d = 16; d; d /= 2) {
        const float om = __shfl_xor_sync(0xffffffffu, m, d), os = __shfl_xor_sync(0xffffffffu, s, d);
        const int oa = __shfl_xor_sync(0xffffffffu, arg, d);
        const float mx = fmaxf(m, om);
        s = s * (m == mx ? 1.0f : exp_below(m, mx)) + os * (om == mx ? 1.0f : exp_below(om, mx));
        arg = om > m ? oa : om < m ? arg : min(arg, oa);
        m = mx;
    }
    if (g >= 0 && g >= a.n_grammar) {
        if (a.out) {
            T* z = static_cast<T*>(a.out) + static_cast<size_t>(row) * a.ld_out;
            for (int v = lane; v < a.vocab; v += 32) Io<T>::put(z + v, -INFINITY);
        }
        m = -INFINITY;
        s = 0.0f;
    }
    if (lane) return;
    const bool some = s != 0.0f;  // (NaN too)
    if (a.x0) a.x0[row] = m > -INFINITY ? arg : -1;
    if (a.conf) a.conf[row] = some ? 1.0f / s : 0.0f;
    if (a.tokconf && a.cur) {
        const int cur = a.cur[row];
        const bool there = cur >= 0 && cur < a.vocab && cur != a.mask_id;
        a.tokconf[row] = there && some ? exp_below(zcur[row], m > -INFINITY ? m : 0.0f) / s : 0.0f;
    }
}

// Rows of a request share its words and the reading of its lists; CTAs enough to fill the GPU (four an SM run at a
// time) come first.  Measured, 512 rows of 126464 ids in requests of 32, by rows a CTA and ids a stretch: 32 and
// 8192 274 us (an earlier form), 8 and 8192 60, 8 and 4096 72, 4 and 8192 69.  Single rows: a CTA of four warps each;
// 96 of 152064 ids and 5000 of history: stretches of 4096 39 us, 8192 34, 16384 44.
Cut logits_cut(int rows, int vocab, int n_req, long long asked, int sms) {
    Cut c;
    const int per = n_req > 0 ? rows / n_req : kWarps;
    c.rows_cta = per < 1 ? 1 : per > 32 ? 32 : per;
    if (c.rows_cta > rows) c.rows_cta = rows;
    c.chunk = kChunk;
    auto ctas = [&] {
        return static_cast<long long>((rows + c.rows_cta - 1) / c.rows_cta) * ((vocab + c.chunk - 1) / c.chunk);
    };
    while (c.rows_cta > kWarps && ctas() < 6ll * sms) c.rows_cta = (c.rows_cta + 1) / 2;
    while (c.chunk > 4096 && ctas() < 4ll * sms) c.chunk /= 2;
    while (c.chunk > 2048 && ctas() < sms) c.chunk /= 2;
    c.chunks = (vocab + c.chunk - 1) / c.chunk;
    c.warps = c.rows_cta < 4 ? 4 : kWarps;
    const int most = c.chunk / kPiece;
    c.split = (c.warps + c.rows_cta - 1) / c.rows_cta;
    if (c.split > most) c.split = most;
    c.list = static_cast<int>(asked < c.chunk ? (asked + 7) / 8 * 8 : c.chunk);
    return c;
}

template <typename T>
cudaError_t go(const dllm_serve_logits_args& a, const Cut& c, Part* part, float* zcur, cudaStream_t st) {
    const dim3 grid((a.rows + c.rows_cta - 1) / c.rows_cta, c.chunks);
    const int smem = c.chunk * 4 + c.chunk / 8 + c.list * 2;
    const bool vec = reinterpret_cast<uintptr_t>(a.logits) % (4 * sizeof(T)) == 0 && a.ld % 4 == 0 &&
                     reinterpret_cast<uintptr_t>(a.out) % (4 * sizeof(T)) == 0 && (!a.out || a.ld_out % 4 == 0);
    const auto kernel = vec ? k_logits<T, true> : k_logits<T, false>;
    cudaError_t e = cudaSuccess;
    // with s_count over 48 KB it has to be asked for: the most of any call, so that host threads, whose limit is one and
    // the same, do not lower it between another's asking and launch
    constexpr int kMostSmem = kChunk * 4 + kChunk / 8 + kChunk * 2;
    if (smem + static_cast<int>(sizeof(int)) * kWarps > 48 * 1024)
        e = cudaFuncSetAttribute(reinterpret_cast<const void*>(kernel), cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSmem);
    if (e != cudaSuccess) return e;
    e = serve_launch(kernel, grid, c.warps * 32, smem, st, a, c, part, zcur);
    if (e != cudaSuccess || !(a.x0 || a.conf || a.tokconf || (a.grammar && a.out))) return e;
    return serve_launch(k_merge<T>, dim3((a.rows + 3) / 4), 128, 0, st, a, c.chunks * c.split, static_cast<const Part*>(part),
                        static_cast<const float*>(zcur));
}

}  // namespace

size_t serve_logits_bytes(int rows, int vocab) {
    // the most parts that a cut makes of a row: eight of each 8192 ids, or one of each 512
    const size_t parts = static_cast<size_t>((vocab + kChunk - 1) / kChunk) * kWarps * 2;
    return serve_round(static_cast<size_t>(rows) * 4) + serve_round(static_cast<size_t>(rows) * parts * sizeof(Part));
}

cudaError_t launch_serve_logits(const dllm_serve_logits_args& a, int sms, cudaStream_t st) {
    const long long asked = (a.hist ? a.hist_ld : 0) + (a.bias_ids ? a.bias_ld : 0);
    const Cut c = logits_cut(a.rows, a.vocab, a.hist || a.bias_ids ? a.n_req : 0, asked, sms);
    float* zcur = static_cast<float*>(a.ws);
    Part* part = reinterpret_cast<Part*>(static_cast<char*>(a.ws) + serve_round(static_cast<size_t>(a.rows) * 4));
    return a.dtype == DLLM_F32    ? go<float>(a, c, part, zcur, st)
           : a.dtype == DLLM_BF16 ? go<__nv_bfloat16>(a, c, part, zcur, st)
                                  : go<__half>(a, c, part, zcur, st);
}

}  // namespace dllm
