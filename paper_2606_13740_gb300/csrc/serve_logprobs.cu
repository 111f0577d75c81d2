// Log probabilities from logits (include/dllm_serve_drafts.h, dllm_serve_logprobs): the normaliser, the entropy, given
// tokens and the largest ones, from one read of the logits.
//
// A cluster takes a row, its warps steps of it that they copy ahead into shared memory (cp.async, each lane what it
// reads itself, so that nobody waits for another).  A warp keeps the largest logit m it has met and, of all the others, sums
//   s = sum 2^y,  t = sum 2^y y,  y = z log2(e) - c
// against a reference c that moves only when a value exceeds it by more than 8.  The largest is never among the sums,
// so that log1p(s) of a row in which one id has nearly everything keeps its digits; as a step (2 KB of ids) seldom brings a new
// one, it is looked for a step at a time.  Where m log2(e) may not be a number (10^37 and more) the sums are of exp(z - m)
// itself.  Parts meet in the same way.  The largest ids: each group of ids (a step, or more where that makes over 1024 groups)
// leaves its maximum; where n_top groups, at least, reach a value, the n_top largest ids are no less and lie in groups that
// reach it (of many that just reach it the first do).  These are read again, and what is no less is ranked.
// Bound: memory, and at the end of a row the latency of that.  Measured in a graph, passes in a row: 512 rows of 126464 32-bit ids
// 45.9 us (259 MB: 5.6 TB/s; a kernel that does nothing but read them 39.6), with 20 alternatives 52.5; 1501 rows of 152064 bf16 ids
// 79.9 (456 MB: 5.7 TB/s; 67 to read them); one row of 126464 with 5 alternatives 7.0.  Rows that do not begin at 16 bytes go id by
// id, without copies ahead: 1500 rows of 50257 bf16 ids 105 us, of 50264 36.  (Loads a step ahead in registers instead: 62 and 94.  Clamping only where -inf was met: more code than the
// instruction cache holds, 120 for the bf16 rows.  Every largest value met kept out one by one: 93 and 110.)
#include "serve.cuh"

namespace dllm {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kCluster = 8;              // CTAs of a row, at most
constexpr int kSpans = 4;                // 16-byte pieces of a lane in a step
constexpr int kStages = 3;               // steps of a warp on their way
constexpr int kGroups = 1024;            // of a row, at most
constexpr int kChosen = 64;              // groups that may hold one of the largest, at most
constexpr int kRanked = 256;             // ids that may be among the largest: so many are ranked, more of them thinned out first
constexpr int kList = 6144;
constexpr int kRing = kWarps * kStages * kSpans * 32;  // 16-byte pieces
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kFar = -150.0f;          // exp of it is 0 in 32 bits
constexpr float kFar2 = -216.0f;         // 2^ that too
constexpr float kLowest = -3.402823466e38f;
constexpr float kWide = 1e37f;           // values whose product with log2(e) is safely a number
constexpr float kLn2 = 0.6931471805599453f;

struct alignas(16) Part {
    float m, s, t, pad;  // the largest logit; of the others the sums against m
};

// Values side by side in 16 bytes of memory.
template <typename T>
struct Raw {
    static constexpr int kPer = 8;
    static __device__ __forceinline__ void floats(const uint4& u, float* v) {
        const uint32_t x[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = Half2<T>::unpack(x[i]);
            v[2 * i] = f.x;
            v[2 * i + 1] = f.y;
        }
    }
};
template <>
struct Raw<float> {
    static constexpr int kPer = 4;
    static __device__ __forceinline__ void floats(const uint4& u, float* v) {
        v[0] = __uint_as_float(u.x), v[1] = __uint_as_float(u.y), v[2] = __uint_as_float(u.z), v[3] = __uint_as_float(u.w);
    }
};
template <typename T>
constexpr int kSpan = 32 * Raw<T>::kPer;         // ids that a warp takes side by side
template <typename T>
constexpr int kPiece = kSpan<T> * kSpans;        // a warp's step

__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// the larger; NaN if one is
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// 2 values at a time
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("{\n .reg .b64 a, b, d;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n"
        " add.rn.f32x2 d, a, b;\n mov.b64 {%0, %1}, d;\n}\n"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{\n .reg .b64 a, b, c, d;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n mov.b64 c, {%6, %7};\n"
        " fma.rn.f32x2 d, a, b, c;\n mov.b64 {%0, %1}, d;\n}\n"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float finite(float x) { return fminf(fmaxf(x, kLowest), -kLowest); }

// A lane's share of the sums, against ref.
struct Sums {
    float ref = kLowest, s = 0.0f, t = 0.0f;
    __device__ __forceinline__ void add(float z) {
        const float d = max_nan(z - ref, kFar), e = ex2(d * kLog2e);
        s += e;
        t = fmaf(e, d, t);
    }
    __device__ __forceinline__ void add(float s2, float t2, float ref2) {  // sums against another reference
        const float d = ref2 - ref, e = ex2(fmaxf(d, kFar) * kLog2e);
        s = fmaf(s2, e, s);
        t += e > 0.0f ? fmaf(s2, d, t2) * e : t2 * 0.0f;  // (0, or NaN)
    }
    __device__ __forceinline__ void move(float to) {  // the reference; to finite
        const Sums old = *this;
        ref = to;
        s = t = 0.0f;
        add(old.s, old.t, old.ref);
    }
};

// The same against c in powers of 2: y of z is fma(z, log2(e), -c), so that the rounding of c is no error.
struct Sums2 {
    float c = 0.0f, s = 0.0f, t = 0.0f;
    __device__ __forceinline__ void move(float to) {  // to z = `to`
        const float d = fmaf(-to, kLog2e, c), e = ex2(fmaxf(d, kFar2));
        t = fmaf(s, fmaxf(d, kFar2), t) * e;
        s *= e;
        c = fmaf(to, kLog2e, 0.0f);
        // (c is rounded: what its rounding leaves of d)
        const float r = fmaf(to, kLog2e, -c), f = ex2(r);
        t = fmaf(s, r, t) * f;
        s *= f;
    }
};

__device__ __forceinline__ float warp_max(float x) {  // (NaN passed over)
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// Joins parts, one a lane (those without: m -inf, s and t 0).  All lanes get the result.
__device__ __forceinline__ Part join_warp(const Part& p) {
    const float m = warp_max(p.m);
    const bool holder = (threadIdx.x & 31) == __ffs(__ballot_sync(0xffffffffu, p.m == m)) - 1;
    Sums v;
    v.ref = finite(m);
    v.add(p.s, p.t, finite(p.m));
    if (!holder) v.add(p.m);
#pragma unroll
    for (int d = 16; d; d /= 2) {
        v.s += __shfl_xor_sync(0xffffffffu, v.s, d);
        v.t += __shfl_xor_sync(0xffffffffu, v.t, d);
    }
    return Part{m, v.s, v.t, 0.0f};
}

// Ids of a row side by side, one by one.
template <typename T>
__device__ __forceinline__ void load_some(const T* src, int v, int vocab, float* z) {
#pragma unroll
    for (int i = 0; i < Raw<T>::kPer; ++i) z[i] = v + i < vocab ? static_cast<float>(src[v + i]) : -INFINITY;
}
// Whether (value, id) comes before another among the largest.
__device__ __forceinline__ bool before(float z, int v, float z2, int v2) { return z > z2 || (z == z2 && v < v2); }

struct More {
    float z[kList];
    int v[kList];
};
// Shared memory of a CTA.  The steps on their way, and when all have been taken what the ending of a row needs.
struct Shared {
    alignas(16) float top[kGroups];  // the groups' maxima
    Part part[kCluster * kWarps];    // of the row's warps
    Part all;
    int group[kChosen], n_groups, n, count[64];
    float least;
    alignas(16) float z[kRanked];  // ids that may be among the largest
    int v[kRanked];
    float best[kWarps];
    int id[kWarps];
    union {
        alignas(16) uint4 ring[kRing];
        More more;
    };
};
static_assert(4 * (sizeof(Shared) + 1024) <= 228 * 1024, "four CTAs an SM");

// The logit of a row's token i, -inf for ids that are none.
template <typename T>
__device__ __forceinline__ float logit_of(const dllm_serve_logprobs_args& a, int row, const T* src, int i) {
    const int v = a.tokens[static_cast<long long>(row) * a.n_tokens + i];
    return v >= 0 && v < a.vocab && v != a.mask_id ? static_cast<float>(src[v]) : -INFINITY;
}

// Values in an order of whole numbers; -inf and NaN: 0.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);  // (-0 is 0)
    return x > -INFINITY ? (b >> 31 ? ~b : b | 0x80000000u) : 0u;
}

// A value that k of n, at least, reach, as a key: the k-th largest of the lanes' two largest each (0: they are less).  By one
// warp; both: 64 words of shared memory, 16-byte aligned.
__device__ __forceinline__ uint32_t bound_of(const float* x, int n, int k, uint32_t* both) {
    const int lane = threadIdx.x & 31;
    uint32_t top = 0, next = 0;
    for (int i = lane; i < n; i += 32) {
        const uint32_t v = key_of(x[i]);
        next = max(next, min(v, top));
        top = max(top, v);
    }
    both[lane] = top;
    both[32 + lane] = next;
    __syncwarp();
    int reach = 0, reach2 = 0;  // how many are no less
#pragma unroll
    for (int i = 0; i < 64; i += 4) {
        const uint4 o = *reinterpret_cast<const uint4*>(both + i);
        reach += (o.x >= top) + (o.y >= top) + (o.z >= top) + (o.w >= top);
        reach2 += (o.x >= next) + (o.y >= next) + (o.z >= next) + (o.w >= next);
    }
    return __reduce_max_sync(0xffffffffu, reach >= k ? top : reach2 >= k ? next : 0u);
}
// The number of a key (of none: the lowest).
__device__ __forceinline__ float number_of(uint32_t key) {
    return key > 1 ? __uint_as_float(key >> 31 ? key & 0x7fffffffu : ~key) : kLowest;
}

// A warp chooses groups whose maxima reach a value that k of them, at least, reach (all where there are less), in order of their
// numbers.  Where it lets more than 2 k through (many equal ones), the k-th largest of all is found bit by bit, and of those
// equal to it the first are taken.
__device__ __forceinline__ void choose(Shared& sh, int groups, int k) {
    const int lane = threadIdx.x & 31;
    uint32_t least = max(bound_of(sh.top, groups, k, reinterpret_cast<uint32_t*>(sh.z)), 1u);
    auto reach = [&](uint32_t from) {  // how many are no less
        int n = 0;
        for (int g = lane; g < groups; g += 32) n += key_of(sh.top[g]) >= from;
        return __reduce_add_sync(0xffffffffu, n);
    };
    int equal = groups;  // how many of those equal to it are taken
    if (reach(least) > 2 * k) {
        least = 0;
        for (uint32_t bit = 1u << 31; bit; bit >>= 1)
            if (reach(least | bit) >= k) least |= bit;
        equal = k - reach(least + 1);
    }
    int n = 0;
    for (int g0 = 0; g0 < groups; g0 += 32) {
        const uint32_t x = g0 + lane < groups ? key_of(sh.top[g0 + lane]) : 0u;
        const uint32_t same = __ballot_sync(0xffffffffu, x == least), low = (1u << lane) - 1;
        const bool in = x > least || (x == least && __popc(same & low) < equal);
        const uint32_t ins = __ballot_sync(0xffffffffu, in);
        if (in) sh.group[n + __popc(ins & low)] = g0 + lane;
        n += __popc(ins);
        equal -= __popc(same);
    }
    if (lane == 0) {
        sh.n_groups = n;
        sh.least = number_of(least);
    }
}

// f of the values side by side (the first of id v) that are no less than least.
template <int N, typename F>
__device__ __forceinline__ void look(const float (&z)[N], int v, float least, int mask_id, const F& f) {
    float mx = z[0];
#pragma unroll
    for (int c = 1; c < N; ++c) mx = fmaxf(mx, z[c]);
    if (!(mx >= least)) return;
#pragma unroll
    for (int c = 0; c < N; ++c)
        if (z[c] >= least && v + c != mask_id) f(v + c, z[c]);
}

// The row's values from the parts of its `warps` warps and the groups' maxima, which lie in sh.  (z_token: the logit of the
// thread's token.)
template <typename T, bool VEC>
__device__ __forceinline__ void finish(const dllm_serve_logprobs_args& a, int row, const T* src, int group_pieces, int groups,
                                       int warps, float z_token, Shared& sh) {
    constexpr int kPer = Raw<T>::kPer, kLoads = kPiece<T> / kPer;  // 16-byte loads of a step
    const Part nothing{-INFINITY, 0.0f, 0.0f, 0.0f};
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int k = min(a.n_top, groups);
    __syncthreads();
    if (warp == 0) {
        Part all = nothing;
        for (int i = 0; i < warps; i += 32) {
            const Part p = join_warp(i + lane < warps ? sh.part[i + lane] : nothing);
            if (lane == i / 32) all = p;
        }
        all = join_warp(all);
        if (lane == 0) {
            sh.all = all;
            sh.n = 0;
        }
        sh.count[lane] = sh.count[lane + 32] = 0;
    } else if (warp == 1 && k) {
        choose(sh, groups, k);
    }
    __syncthreads();
    // ------------------------------------------------ the chosen groups, their first loads asked for
    const int n_groups = k ? sh.n_groups : 0;
    float least = k && k == a.n_top ? sh.least : kLowest;
    const int total = n_groups * group_pieces * kLoads;
    static_assert(kThreads % kLoads == 0, "a load's place in its step is the thread's own");
    auto id_of = [&](int i) {
        const int piece = i / kLoads, g = group_pieces == 1 ? piece : piece / group_pieces;
        return (sh.group[g] * group_pieces + piece - g * group_pieces) * kPiece<T> + i % kLoads * kPer;
    };
    auto ask = [&](int i0) {  // for a thread's own, up to a ring full
        for (int i = i0 + tid; i < min(total, i0 + kRing); i += kThreads) {
            const int v = id_of(i);
            if (VEC && v + kPer <= a.vocab) cp_async16(sh.ring + (i - i0), src + v);
        }
        cp_async_commit();
    };
    static_assert(kRing <= 32 * kThreads, "a bit for each of a thread's loads");
    ask(0);

    const Part all = sh.all;
    const bool none = all.m == -INFINITY && all.s == 0.0f, above = all.m == INFINITY;
    const float m = all.m, log_rest = log1pf(all.s);
    auto lp_of = [&](float z) {
        if (z == -INFINITY || none) return all.s == all.s ? -INFINITY : all.s;
        if (above) return z == INFINITY || all.s != all.s ? __int_as_float(0x7fffffff) : -INFINITY;
        return (z - m) - log_rest;
    };
    if (tid == 0) {
        if (a.lse) a.lse[row] = none ? -INFINITY : above && all.s == all.s ? INFINITY : m + log_rest;
        if (a.entropy) a.entropy[row] = none ? 0.0f : above ? __int_as_float(0x7fffffff) : log_rest - all.t / (1.0f + all.s);
    }
    for (int i = tid; i < a.n_tokens; i += kThreads)
        a.lp[static_cast<long long>(row) * a.n_tokens + i] = lp_of(i == tid ? z_token : logit_of<T>(a, row, src, i));
    if (!k) return;

    // ------------------------------------------------ the largest
    for (int i0 = 0; i0 < total; i0 += kRing) {
        cp_async_wait<0>();
        // first which of the thread's loads hold one at all
        auto get = [&](int i, float (&z)[kPer]) {
            const int v = id_of(i);
            if (VEC && v + kPer <= a.vocab) Raw<T>::floats(sh.ring[i - i0], z);
            else load_some(src, v, a.vocab, z);
            if (static_cast<unsigned>(a.mask_id - v) < kPer) {
#pragma unroll
                for (int c = 0; c < kPer; ++c)
                    if (v + c == a.mask_id) z[c] = -INFINITY;
            }
            return v;
        };
        const int mine = (min(total - i0, kRing) - tid + kThreads - 1) / kThreads;
        uint32_t hits = 0;
        float most = -INFINITY;
#pragma unroll 4
        for (int u = 0; u < mine; ++u) {
            float z[kPer];
            get(i0 + tid + u * kThreads, z);
            float mx = z[0];
#pragma unroll
            for (int c = 1; c < kPer; ++c) mx = fmaxf(mx, z[c]);
            hits |= static_cast<uint32_t>(mx >= least) << u;
            most = fmaxf(most, mx);
        }
        if (a.n_top > 1 && groups < 4 * a.n_top && i0 == 0) {  // few groups for the ids wanted: what so many threads reach is a better limit
            sh.top[tid] = most;
            __syncthreads();
            if (warp == 0) {
                const uint32_t key = bound_of(sh.top, kThreads, a.n_top, reinterpret_cast<uint32_t*>(sh.z));
                if (lane == 0) sh.least = number_of(key);
            }
            __syncthreads();
            least = fmaxf(least, sh.least);
        }
        for (; hits; hits &= hits - 1) {
            float z[kPer];
            const int v = get(i0 + tid + (__ffs(hits) - 1) * kThreads, z);
            look(z, v, least, a.mask_id, [&](int id, float x) {
                const int at = atomicAdd(&sh.n, 1);
                if (at < kRanked) {
                    sh.z[at] = x;
                    sh.v[at] = id;
                }
            });
        }
        if (i0 + kRing < total) ask(i0 + kRing);
    }
    __syncthreads();
    const int n = sh.n;
    int* ids = a.top_ids + static_cast<long long>(row) * a.n_top;
    float* lps = a.top_lp + static_cast<long long>(row) * a.n_top;
    if (n <= kRanked) {
        if (tid < n) {
            const float z = sh.z[tid];
            const int v = sh.v[tid];
            int rank = 0;
#pragma unroll 4
            for (int j = 0; j < n; ++j) rank += before(sh.z[j], sh.v[j], z, v);
            if (rank < a.n_top) {
                ids[rank] = v;
                lps[rank] = lp_of(z);
            }
        }
        for (int r = n + tid; r < a.n_top; r += kThreads) {
            ids[r] = -1;
            lps[r] = -INFINITY;
        }
        return;
    }
    // Many equal ones, or a small vocabulary: from memory again.
    auto each = [&](const auto& f) {
#pragma unroll 1
        for (int i = tid; i < total; i += kThreads) {
            const int v = id_of(i);
            float z[kPer];
            if (VEC && v + kPer <= a.vocab) Raw<T>::floats(*reinterpret_cast<const uint4*>(src + v), z);
            else load_some(src, v, a.vocab, z);
            look(z, v, least, a.mask_id, f);
        }
    };
    if (n <= kList) {
        __syncthreads();  // (all know n)
        if (tid == 0) sh.n = 0;
        __syncthreads();
        each([&](int id, float x) {
            const int at = atomicAdd(&sh.n, 1);
            sh.more.z[at] = x;
            sh.more.v[at] = id;
        });
        __syncthreads();
        // The n_top largest (value, id), which are all different, bit by bit.
        auto pair_of = [&](int i) {
            return static_cast<unsigned long long>(key_of(sh.more.z[i])) << 32 | static_cast<uint32_t>(~sh.more.v[i]);
        };
        unsigned long long from = 0;
        for (int bit = 63; bit >= 0; --bit) {
            const unsigned long long x = from | 1ull << bit;
            int c = 0;
            for (int i = tid; i < n; i += kThreads) c += pair_of(i) >= x;
            c = __reduce_add_sync(0xffffffffu, c);
            if (lane == 0 && c) atomicAdd(&sh.count[bit], c);
            __syncthreads();
            c = sh.count[bit];
            if (c >= a.n_top) from = x;
            if (c == a.n_top) break;
        }
        if (tid == 0) sh.n = 0;
        __syncthreads();
        for (int i = tid; i < n; i += kThreads)
            if (pair_of(i) >= from) sh.group[atomicAdd(&sh.n, 1)] = i;
        __syncthreads();
        if (tid < a.n_top) {
            const int at = sh.group[tid];
            const float z = sh.more.z[at];
            const int v = sh.more.v[at];
            int rank = 0;
            for (int j = 0; j < a.n_top; ++j) rank += before(sh.more.z[sh.group[j]], sh.more.v[sh.group[j]], z, v);
            ids[rank] = v;
            lps[rank] = lp_of(z);
        }
        return;
    }
    // More equal ones than there are places: the largest below the one before, one by one.
    float z0 = INFINITY;
    int v0 = -1;
    for (int r = 0; r < a.n_top; ++r) {
        float bz = -INFINITY;
        int bv = a.vocab;
        each([&](int v, float z) {
            if (before(z0, v0, z, v) && before(z, v, bz, bv)) {
                bz = z;
                bv = v;
            }
        });
#pragma unroll
        for (int d = 16; d; d /= 2) {
            const float oz = __shfl_xor_sync(0xffffffffu, bz, d);
            const int ov = __shfl_xor_sync(0xffffffffu, bv, d);
            if (before(oz, ov, bz, bv)) {
                bz = oz;
                bv = ov;
            }
        }
        if (lane == 0) {
            sh.best[warp] = bz;
            sh.id[warp] = bv;
        }
        __syncthreads();
        z0 = sh.best[0];
        v0 = sh.id[0];
        for (int i = 1; i < kWarps; ++i)
            if (before(sh.best[i], sh.id[i], z0, v0)) {
                z0 = sh.best[i];
                v0 = sh.id[i];
            }
        if (tid == 0) {
            ids[r] = v0;
            lps[r] = lp_of(z0);
        }
        __syncthreads();
    }
}

// A cluster takes a row.  Its warps take turns at the groups, so that it reads in order (1501 rows of 152064 bf16 ids 82.5 ->
// 80.5 us); its first CTA ends it.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 4 ? 4 : 3)
    k_logprobs(const __grid_constant__ dllm_serve_logprobs_args a, int group_pieces, int groups) {
    constexpr int kPer = Raw<T>::kPer, kValues = kSpans * kPer;
    extern __shared__ __align__(16) uint8_t smem[];
    Shared& sh = *reinterpret_cast<Shared*>(smem);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int row = blockIdx.y, share = blockIdx.x * kWarps + warp, shares = gridDim.x * kWarps;
    if (gridDim.x > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;");  // (the first CTA is there)
    // steps of the row, whole ones; the warp's: those of groups share, share + shares, ...
    const int q1 = (a.vocab + kPiece<T> - 1) / kPiece<T>, qw = VEC ? a.vocab / kPiece<T> : 0;
    const int skip = (shares - 1) * group_pieces;
    int q = share * group_pieces, asked = q, stage = 0, to = 0;
    pdl_wait();
    pdl_launch_dependents();
    const T* src = static_cast<const T*>(a.logits) + row * a.ld;
    uint4* const mine = sh.ring + warp * (kStages * kSpans * 32) + lane;
    const T* ps = src + static_cast<size_t>(q) * kPiece<T> + lane * kPer;
    int asked_left = group_pieces;  // of the group
    auto ask = [&] {  // for the next whole step (a group of copies in any case, to count)
        if (asked < qw) {
#pragma unroll
            for (int u = 0; u < kSpans; ++u) cp_async16(mine + to * (kSpans * 32) + u * 32, ps + u * kSpan<T>);
        }
        cp_async_commit();
        ++asked;
        ps += kPiece<T>;
        if (--asked_left == 0) {
            asked_left = group_pieces;
            asked += skip;
            ps += static_cast<size_t>(skip) * kPiece<T>;
        }
        to = to + 1 == kStages ? 0 : to + 1;
    };
#pragma unroll
    for (int i = 0; i < kStages; ++i) ask();
    const float z_token = blockIdx.x == 0 && static_cast<int>(threadIdx.x) < a.n_tokens ? logit_of<T>(a, row, src, threadIdx.x) : 0.0f;
    Shared* first = &sh;  // the first CTA's
    if (gridDim.x > 1) {
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
        uint64_t at;
        asm("mapa.u64 %0, %1, 0;" : "=l"(at) : "l"(&sh));
        first = reinterpret_cast<Shared*>(at);
    }
    float m = -INFINITY, best = -INFINITY;  // the warp's; the group's
    Sums2 sums;                             // while -10^37 < m < 10^37
    Sums wide;                              // else
    const int mask_piece = a.mask_id >= 0 ? a.mask_id / kPiece<T> : -1;
    int left = group_pieces;  // steps of the group
    for (int g = share; q < q1;) {
        uint4* at = mine + stage * (kSpans * 32);
        cp_async_wait<kStages - 1>();
        if (q >= qw) {  // one by one
#pragma unroll 1
            for (int u = 0; u < kSpans; ++u) {
                const int v = q * kPiece<T> + u * kSpan<T> + kPer * lane;
#pragma unroll
                for (int i = 0; i < kPer; ++i)
                    reinterpret_cast<T*>(at + u * 32)[i] = v + i < a.vocab ? src[v + i] : static_cast<T>(-INFINITY);
            }
        }
        if (q == mask_piece) {
            const int in = a.mask_id % kPiece<T>, span = in / kSpan<T>, of = in % kSpan<T>;
            if (of / kPer == lane) reinterpret_cast<T*>(at + span * 32)[of % kPer] = static_cast<T>(-INFINITY);
        }
        asm volatile("" ::: "memory");  // (stored as values, loaded as 16 bytes)
        float z[kValues];
#pragma unroll
        for (int u = 0; u < kSpans; ++u) Raw<T>::floats(at[u * 32], z + u * kPer);
        float mx = z[0];
#pragma unroll
        for (int i = 1; i + 1 < kValues; i += 2) mx = max3(mx, z[i], z[i + 1]);
        mx = fmaxf(mx, z[kValues - 1]);
        const float wm = warp_max(mx), old = m;
        const bool more = wm > m;
        if (more) {  // the new m stays out, the old one comes in its place
            if (lane == __ffs(__ballot_sync(0xffffffffu, mx == wm)) - 1) {
                float seek = wm;
#pragma unroll
                for (int i = 0; i < kValues; ++i) {
                    const bool hit = z[i] == seek;
                    z[i] = hit ? old : z[i];
                    seek = hit ? __int_as_float(0x7fffffff) : seek;
                }
            }
            __syncwarp();
            m = wm;
            if (fabsf(m) < kWide) {
                if (!(fabsf(old) < kWide)) {  // (what there was is nothing beside it, unless it is NaN)
                    sums.s = sums.t = wide.s * 0.0f + wide.t * 0.0f;
                    sums.c = m * kLog2e;
                } else if (fmaf(m, kLog2e, -sums.c) > 8.0f) {
                    sums.move(m);
                }
            } else {
                if (fabsf(old) < kWide) wide.s = wide.t = sums.s * 0.0f + sums.t * 0.0f;
                wide.move(finite(m));
            }
        }
        if (fabsf(m) < kWide) {
            // (clamped, so that -inf gives 0 times a number)
            const float2 nc = make_float2(-sums.c, -sums.c), l2 = make_float2(kLog2e, kLog2e);
            float2 s2 = make_float2(0.0f, 0.0f), t2 = s2;
#pragma unroll
            for (int i = 0; i < kValues; i += 2) {
                float2 y = fma2(make_float2(z[i], z[i + 1]), l2, nc), e;
                y.x = max_nan(y.x, kFar2);
                y.y = max_nan(y.y, kFar2);
                e.x = ex2(y.x);
                e.y = ex2(y.y);
                s2 = add2(s2, e);
                t2 = fma2(e, y, t2);
            }
            sums.s += s2.x + s2.y;
            sums.t += t2.x + t2.y;
        } else if (m == -INFINITY) {
            bool odd = false;
#pragma unroll
            for (int i = 0; i < kValues; ++i) odd |= z[i] != z[i];
            if (odd) wide.s = wide.t = __int_as_float(0x7fffffff);
        } else {
            bool out = more && lane == __ffs(__ballot_sync(0xffffffffu, mx == wm)) - 1;  // (the step's one new m)
            if (out) wide.add(old);
#pragma unroll 1
            for (int i = 0; i < kValues; ++i) {
                const float x = static_cast<float>(reinterpret_cast<const T*>(at + i / kPer * 32)[i % kPer]);
                if (out && x == wm) out = false;
                else wide.add(x);
            }
        }
        stage = stage + 1 == kStages ? 0 : stage + 1;
        ask();
        best = fmaxf(best, wm);
        ++q;
        if (--left == 0 || q == q1) {
            if (lane == 0 && a.n_top) first->top[g] = best;
            best = -INFINITY;
            left = group_pieces;
            q += skip;
            g += shares;
        }
    }
    cp_async_wait<0>();
    // the lanes' sums, against m
    if (fabsf(m) < kWide) {
        const float d = fmaf(-m, kLog2e, sums.c), e = ex2(d);
        wide.s = sums.s * e;
        wide.t = fmaf(sums.s, d, sums.t) * e * kLn2;
    } else {
        wide.move(finite(m));
    }
#pragma unroll
    for (int d = 16; d; d /= 2) {
        wide.s += __shfl_xor_sync(0xffffffffu, wide.s, d);
        wide.t += __shfl_xor_sync(0xffffffffu, wide.t, d);
    }
    if (lane == 0) first->part[share] = Part{m, wide.s, wide.t, 0.0f};
    if (gridDim.x > 1) {
        __syncwarp();
        asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
        if (blockIdx.x) return;
    }
    finish<T, VEC>(a, row, src, group_pieces, groups, shares, z_token, sh);
}

template <typename T>
cudaError_t go(const dllm_serve_logprobs_args& a, int sms, cudaStream_t st) {
    constexpr int kRows = 65535;  // of a launch: a grid has no more rows of blocks
    const int pieces = (a.vocab + kPiece<T> - 1) / kPiece<T>, group_pieces = (pieces + kGroups - 1) / kGroups;
    const int groups = (pieces + group_pieces - 1) / group_pieces;
    const bool vec = reinterpret_cast<uintptr_t>(a.logits) % 16 == 0 && a.ld % Raw<T>::kPer == 0;
    const auto kernel = vec ? k_logprobs<T, true> : k_logprobs<T, false>;
    cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void*>(kernel), cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         static_cast<int>(sizeof(Shared)));
    if (e != cudaSuccess) return e;
    for (int r0 = 0; r0 < a.rows; r0 += kRows) {
        dllm_serve_logprobs_args b = a;
        b.rows = a.rows - r0 < kRows ? a.rows - r0 : kRows;
        b.logits = static_cast<const T*>(a.logits) + r0 * a.ld;
        if (a.tokens) b.tokens = a.tokens + static_cast<long long>(r0) * a.n_tokens;
        if (a.lp) b.lp = a.lp + static_cast<long long>(r0) * a.n_tokens;
        if (a.entropy) b.entropy = a.entropy + r0;
        if (a.lse) b.lse = a.lse + r0;
        if (a.top_ids) b.top_ids = a.top_ids + static_cast<long long>(r0) * a.n_top;
        if (a.top_lp) b.top_lp = a.top_lp + static_cast<long long>(r0) * a.n_top;
        // CTAs of a row: up to eight while they are no more than 7 for 4 SMs, each with a group a warp at least.  (Measured
        // for 1, 2, 4, 8, 20 alternatives wanted: 16 rows of 126464 32-bit ids 15.8, 12.0, 10.0, 9.5 us; 76 rows 16.8, 13.9, 15.9,
        // 17.5; 152 rows 19.6, 19.4, 23.6, 24.1; 608 rows 56.6, 61.2, 57.7, 67.1; bf16 rows of 152064, 128 of them 17.8, 20.4,
        // 20.4, 24.2; 1500 of them 97, 118, 144, 195.)
        int ctas = 1;
        while (ctas < kCluster && 8ll * ctas * b.rows <= 7ll * sms && ctas * kWarps < groups) ctas *= 2;
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3(ctas, b.rows);
        cfg.blockDim = dim3(kThreads);
        cfg.dynamicSmemBytes = sizeof(Shared);
        cfg.stream = st;
        cudaLaunchAttribute at[2];
        at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at[0].val.programmaticStreamSerializationAllowed = 1;
        at[1].id = cudaLaunchAttributeClusterDimension;
        at[1].val.clusterDim.x = ctas;
        at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
        cfg.attrs = at;
        cfg.numAttrs = 2;
        e = cudaLaunchKernelEx(&cfg, kernel, b, group_pieces, groups);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace

cudaError_t launch_serve_logprobs(const dllm_serve_logprobs_args& a, int sms, cudaStream_t st) {
    return a.dtype == DLLM_F32    ? go<float>(a, sms, st)
           : a.dtype == DLLM_BF16 ? go<__nv_bfloat16>(a, sms, st)
                                  : go<__half>(a, sms, st);
}

}  // namespace dllm
