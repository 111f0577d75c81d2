// Log probabilities from logits (include/dllm_serve_drafts.h, dllm_serve_logprobs): the normaliser, the entropy, given
// tokens and the largest ones, from one read of the logits.
//
// Warps stream stretches of a row.  A lane keeps the largest logit m it has met and, of all the others, the sums
//   s = sum exp(z - ref),  t = sum exp(z - ref) (z - ref)
// against a reference that moves only when a value exceeds it by more than 8: of each new value and m the smaller
// goes into the sums, so that the largest is never among them, and log1p(s) of a row in which one id has nearly
// everything keeps its digits.  Parts meet in the same way in k_logprobs_row (a CTA a row), which turns them into the
// row's values.  The largest ids: each group of ids (512, or more where that makes over 1024 groups) leaves its maximum; the
// n_top largest ids lie in the n_top groups with the largest maxima (of equal ones the first), as each of these has
// one value at least as large as any value outside.  They are read again, and what is not below the smallest of the
// chosen maxima is ranked.
// Bound: memory.
#include "serve.cuh"

namespace dllm {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kSpan = 128;               // ids that a warp takes side by side, 4 a lane
constexpr int kSpans = 4;                // of these in flight together
constexpr int kPiece = kSpan * kSpans;   // a warp's step
constexpr int kGroups = 1024;            // of a row, at most
constexpr int kTop = 32;
constexpr int kList = 1024;              // ids that are ranked side by side
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kFar = -150.0f;          // exp of it is 0 in 32 bits
constexpr float kLowest = -3.402823466e38f;

struct alignas(16) Part {
    float m, s, t, pad;  // the largest logit; of the others the sums against m
};

template <typename T>
struct Vec4;  // four values as they lie in memory
template <>
struct Vec4<float> {
    static __device__ __forceinline__ void load(const float* p, float* v) {
        const float4 f = *reinterpret_cast<const float4*>(p);
        v[0] = f.x, v[1] = f.y, v[2] = f.z, v[3] = f.w;
    }
};
template <typename T>
struct Vec4 {
    static __device__ __forceinline__ void load(const T* p, float* v) {
        const uint2 u = *reinterpret_cast<const uint2*>(p);
        const float2 a = Half2<T>::unpack(u.x), b = Half2<T>::unpack(u.y);
        v[0] = a.x, v[1] = a.y, v[2] = b.x, v[3] = b.y;
    }
};

__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// the smaller, the larger; NaN if one is
__device__ __forceinline__ float min_nan(float a, float b) {
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// The running sums of a lane.
struct Sums {
    float m = -INFINITY, ref = kLowest, s = 0.0f, t = 0.0f;
    __device__ __forceinline__ void add(float z) {
        const float lo = min_nan(z, m);
        m = fmaxf(m, z);
        const float d = max_nan(lo - ref, kFar), e = ex2(d * kLog2e);
        s += e;
        t = fmaf(e, d, t);
    }
    __device__ __forceinline__ void move(float to) {  // the reference; to finite
        const float d = ref - to, e = ex2(fmaxf(d, kFar) * kLog2e);
        t = e > 0.0f ? (t + s * d) * e : t * 0.0f;  // (0, or NaN)
        s *= e;
        ref = to;
    }
    __device__ __forceinline__ void look(float mx) {  // before values up to mx are added
        if (mx > ref + 8.0f || (ref == kLowest && mx > ref)) move(fminf(mx, -kLowest));
    }
};

// Joins the lanes' (or parts') sums: afterwards m is the largest of all, s and t are against it, and the largest values
// of the others are among them.  All lanes get the result.
__device__ __forceinline__ Part join_warp(Sums v) {
    float m = v.m;
#pragma unroll
    for (int d = 16; d; d /= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    const uint32_t have = __ballot_sync(0xffffffffu, v.m == m);
    const bool holder = (threadIdx.x & 31) == __ffs(have) - 1;
    const float to = fminf(fmaxf(m, kLowest), -kLowest);
    v.move(to);
    if (!holder) {
        const float d = fmaxf(v.m - to, kFar), e = ex2(d * kLog2e);
        v.s += e;
        v.t = fmaf(e, d, v.t);
    }
#pragma unroll
    for (int d = 16; d; d /= 2) {
        v.s += __shfl_xor_sync(0xffffffffu, v.s, d);
        v.t += __shfl_xor_sync(0xffffffffu, v.t, d);
    }
    return Part{m, v.s, v.t, 0.0f};
}

// A warp takes some groups of a row that lie side by side.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) k_logprobs(const __grid_constant__ dllm_serve_logprobs_args a, int group_pieces,
                                                       int groups, int shares, Part* part, float* top) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int row = blockIdx.y, share = blockIdx.x * kWarps + warp;
    pdl_wait();
    pdl_launch_dependents();
    if (share >= shares) return;
    const T* src = static_cast<const T*>(a.logits) + row * a.ld;
    const int g0 = static_cast<int>(static_cast<long long>(groups) * share / shares);
    const int g1 = static_cast<int>(static_cast<long long>(groups) * (share + 1) / shares);
    Sums sums;
    for (int g = g0; g < g1; ++g) {
        float best = -INFINITY;
        for (int q = g * group_pieces; q < (g + 1) * group_pieces; ++q) {
            const int v0 = q * kPiece + 4 * lane;
            float z[kSpans][4];
            if (VEC && (q + 1) * kPiece <= a.vocab) {
#pragma unroll
                for (int u = 0; u < kSpans; ++u) Vec4<T>::load(src + v0 + u * kSpan, z[u]);
            } else {
#pragma unroll
                for (int u = 0; u < kSpans; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        z[u][i] = v0 + u * kSpan + i < a.vocab ? static_cast<float>(src[v0 + u * kSpan + i]) : -INFINITY;
            }
            if (a.mask_id >= 0 && a.mask_id / kPiece == q) {
#pragma unroll
                for (int u = 0; u < kSpans; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (v0 + u * kSpan + i == a.mask_id) z[u][i] = -INFINITY;
            }
            float mx = z[0][0];
#pragma unroll
            for (int u = 0; u < kSpans; ++u) mx = fmaxf(fmaxf(fmaxf(mx, z[u][0]), z[u][1]), fmaxf(z[u][2], z[u][3]));
            best = fmaxf(best, mx);
            sums.look(mx);
#pragma unroll
            for (int u = 0; u < kSpans; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) sums.add(z[u][i]);
        }
        if (a.n_top) {
#pragma unroll
            for (int d = 16; d; d /= 2) best = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, d));
            if (lane == 0) top[static_cast<size_t>(row) * groups + g] = best;
        }
    }
    const Part p = join_warp(sums);
    if (lane == 0) part[static_cast<size_t>(row) * shares + share] = p;
}

// Whether (value, id) comes before another among the largest.
__device__ __forceinline__ bool before(float z, int v, float z2, int v2) { return z > z2 || (z == z2 && v < v2); }

template <typename T>
__global__ void __launch_bounds__(kThreads) k_logprobs_row(const __grid_constant__ dllm_serve_logprobs_args a, int group_pieces,
                                                           int groups, int shares, const Part* part, const float* top) {
    __shared__ float s_top[kGroups], s_z[kList];
    __shared__ int s_group[kTop], s_v[kList], s_n;
    __shared__ Part s_part[kWarps];
    __shared__ float s_best[kWarps];
    __shared__ int s_id[kWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, row = blockIdx.x;
    pdl_wait();
    pdl_launch_dependents();
    const T* src = static_cast<const T*>(a.logits) + row * a.ld;
    // ------------------------------------------------ the parts
    Sums sums;
    for (int i = tid; i < shares; i += kThreads) {
        const Part p = part[static_cast<size_t>(row) * shares + i];
        sums.look(p.m);
        sums.add(p.m);
        const float d = fminf(fmaxf(p.m, kLowest), -kLowest) - sums.ref, e = ex2(fmaxf(d, kFar) * kLog2e);
        sums.s += p.s * e;
        sums.t += e > 0.0f ? (p.t + p.s * d) * e : p.t * 0.0f;
    }
    Part all = join_warp(sums);
    if (lane == 0) s_part[warp] = all;
    if (a.n_top)
        for (int i = tid; i < groups; i += kThreads) s_top[i] = top[static_cast<size_t>(row) * groups + i];
    if (tid < kTop) s_group[tid] = -1;
    if (tid == 0) s_n = 0;
    __syncthreads();
    sums = Sums();
    if (lane < kWarps) {
        const Part p = s_part[lane];
        sums.m = p.m;
        sums.ref = fminf(fmaxf(p.m, kLowest), -kLowest);
        sums.s = p.s;
        sums.t = p.t;
    }
    all = join_warp(sums);
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
    for (int i = tid; i < a.n_tokens; i += kThreads) {
        const long long at = static_cast<long long>(row) * a.n_tokens + i;
        const int v = a.tokens[at];
        a.lp[at] = lp_of(v >= 0 && v < a.vocab && v != a.mask_id ? static_cast<float>(src[v]) : -INFINITY);
    }
    if (!a.n_top) return;

    // ------------------------------------------------ the groups that hold the largest
    const int k = min(a.n_top, groups);
    for (int g = tid; g < groups; g += kThreads) {
        const float x = s_top[g];
        int rank = 0;
        for (int i = 0; i < groups; ++i) rank += before(s_top[i], i, x, g);
        if (rank < k && x > -INFINITY) s_group[rank] = g;
    }
    __syncthreads();
    int n_groups = 0;
    while (n_groups < k && s_group[n_groups] >= 0) ++n_groups;
    const float least = n_groups == a.n_top ? s_top[s_group[n_groups - 1]] : -INFINITY;
    const int size = group_pieces * kPiece;
    auto each = [&](auto&& f) {  // of the groups' ids
        for (int g = 0; g < n_groups; ++g) {
            const int v0 = s_group[g] * size, v1 = min(a.vocab, v0 + size);
            for (int v = v0 + tid; v < v1; v += kThreads)
                if (v != a.mask_id) f(v, static_cast<float>(src[v]));
        }
    };
    each([&](int v, float z) {
        if (z >= least && z > -INFINITY) {
            const int at = atomicAdd(&s_n, 1);
            if (at < kList) {
                s_z[at] = z;
                s_v[at] = v;
            }
        }
    });
    __syncthreads();
    const int n = s_n;
    int* ids = a.top_ids + static_cast<long long>(row) * a.n_top;
    float* lps = a.top_lp + static_cast<long long>(row) * a.n_top;
    if (n <= kList) {
        for (int i = tid; i < n; i += kThreads) {
            int rank = 0;
            for (int j = 0; j < n; ++j) rank += before(s_z[j], s_v[j], s_z[i], s_v[i]);
            if (rank < a.n_top) {
                ids[rank] = s_v[i];
                lps[rank] = lp_of(s_z[i]);
            }
        }
    } else {
        // too many equal or allowed ones: the largest below the one before, one by one
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
                s_best[warp] = bz;
                s_id[warp] = bv;
            }
            __syncthreads();
            z0 = s_best[0];
            v0 = s_id[0];
            for (int i = 1; i < kWarps; ++i)
                if (before(s_best[i], s_id[i], z0, v0)) {
                    z0 = s_best[i];
                    v0 = s_id[i];
                }
            if (tid == 0) {
                ids[r] = v0;
                lps[r] = lp_of(z0);
            }
            __syncthreads();
        }
    }
    for (int r = n + tid; r < a.n_top; r += kThreads) {
        ids[r] = -1;
        lps[r] = -INFINITY;
    }
}

// Groups of a row, and the warps that share them.
struct Cut {
    int group_pieces, groups, shares;
};
Cut logprobs_cut(int rows, int vocab, int sms) {
    Cut c;
    const int pieces = (vocab + kPiece - 1) / kPiece;
    c.group_pieces = (pieces + kGroups - 1) / kGroups;
    c.groups = (pieces + c.group_pieces - 1) / c.group_pieces;
    // as many warps a row as fill the GPU (16 an SM), none of less than a group
    const long long want = (16ll * sms + rows - 1) / rows;
    c.shares = static_cast<int>(want < c.groups ? want : c.groups);
    c.shares = (c.shares + kWarps - 1) / kWarps * kWarps;
    if (c.shares > c.groups) c.shares = c.groups;
    return c;
}

constexpr int kRows = 65535;  // of a launch
size_t most_of(int rows, int vocab) {  // groups of a launch, at most
    const size_t pieces = (static_cast<size_t>(vocab) + kPiece - 1) / kPiece;
    return (rows < kRows ? rows : kRows) * (pieces < kGroups ? pieces : kGroups);
}
size_t part_bytes(int rows, int vocab) { return serve_round(sizeof(Part) * most_of(rows, vocab)); }

template <typename T>
cudaError_t go(const dllm_serve_logprobs_args& a, int sms, cudaStream_t st) {
    // (a grid has 65535 rows of blocks at most)
    const Cut c = logprobs_cut(a.rows < kRows ? a.rows : kRows, a.vocab, sms);
    Part* part = static_cast<Part*>(a.ws);
    float* top = reinterpret_cast<float*>(static_cast<char*>(a.ws) + part_bytes(a.rows, a.vocab));
    const bool vec = reinterpret_cast<uintptr_t>(a.logits) % (4 * sizeof(T)) == 0 && a.ld % 4 == 0;
    const auto kernel = vec ? k_logprobs<T, true> : k_logprobs<T, false>;
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
        cudaError_t e = serve_launch(kernel, dim3((c.shares + kWarps - 1) / kWarps, b.rows), kThreads, 0, st, b, c.group_pieces,
                                     c.groups, c.shares, part, top);
        if (e == cudaSuccess)
            e = serve_launch(k_logprobs_row<T>, dim3(b.rows), kThreads, 0, st, b, c.group_pieces, c.groups, c.shares, part, top);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace

size_t serve_logprobs_bytes(int rows, int vocab) {
    return part_bytes(rows, vocab) + serve_round(sizeof(float) * most_of(rows, vocab));
}

cudaError_t launch_serve_logprobs(const dllm_serve_logprobs_args& a, int sms, cudaStream_t st) {
    return a.dtype == DLLM_F32    ? go<float>(a, sms, st)
           : a.dtype == DLLM_BF16 ? go<__nv_bfloat16>(a, sms, st)
                                  : go<__half>(a, sms, st);
}

}  // namespace dllm
