// Logits of a serving step: penalties for repeated ids, biases, grammar masks, and the decision, in one
// pass over them (include/dllm_serve.h, dllm_serve_logits).
//
// A CTA takes a stretch of the vocabulary for some rows.  What the rows' request asks for there (how often
// an id stands in its history, which of its biases names it) is one 32-bit word an id in shared memory, made
// once for all the request's rows in the CTA: count in the low 20 bits, 1 + index of the bias above.  Both
// are integers (a sum and a maximum), so the order in which threads add them does not matter.  Then warps
// stream the rows, several to a row where rows are few, and keep a running maximum, sum of exponentials and
// argmax in registers; k_merge joins a row's stretches.  Bound: memory (logits once in, once out when asked
// for); with single rows, latency.
#include "serve.cuh"

namespace dllm {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kChunk = 8192;  // ids of a stretch, at most: 32 KB of words
constexpr int kGroup = 128;   // ids that a warp takes side by side, 4 a lane
constexpr int kGroups = 4;    // of these in flight together
constexpr int kCountBits = 20;
constexpr float kLog2e = 1.4426950408889634f;

struct Part {
    float m, s;  // largest z, sum of exp(z - m)
    int arg, pad;
};

// How a call is cut: stretches of `chunk` ids, `rows_cta` rows a CTA, `split` warps a row and stretch.
struct Cut {
    int chunk, chunks, rows_cta, split;
};

__device__ __forceinline__ float2 sub2(float2 a, float b) {
    float2 d;
    asm("{\n .reg .b64 a, b, d;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %4};\n"
        " sub.rn.f32x2 d, a, b;\n mov.b64 {%0, %1}, d;\n}\n"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("{\n .reg .b64 a, b, d;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n"
        " add.rn.f32x2 d, a, b;\n mov.b64 {%0, %1}, d;\n}\n"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float b) {
    float2 d;
    asm("{\n .reg .b64 a, b, d;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %4};\n"
        " mul.rn.f32x2 d, a, b;\n mov.b64 {%0, %1}, d;\n}\n"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b));
    return d;
}
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
    static __device__ __forceinline__ float get(const float* p) { return *p; }
    static __device__ __forceinline__ void put(float* p, float v) { *p = v; }
    static __device__ __forceinline__ void get4(const float* p, float* v) {
        const float4 f = *reinterpret_cast<const float4*>(p);
        v[0] = f.x, v[1] = f.y, v[2] = f.z, v[3] = f.w;
    }
    static __device__ __forceinline__ void put4(float* p, const float* v) {
        *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    }
};
template <typename T>
struct Io16 {
    static __device__ __forceinline__ float get(const T* p) { return static_cast<float>(*p); }
    static __device__ __forceinline__ void get4(const T* p, float* v) {
        const uint2 u = *reinterpret_cast<const uint2*>(p);
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

template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) k_logits(const __grid_constant__ dllm_serve_logits_args a, Cut cut,
                                                     Part* __restrict__ part, float* __restrict__ zcur) {
    extern __shared__ __align__(16) uint32_t word[];  // [cut.chunk]
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int v0 = blockIdx.y * cut.chunk, v1 = min(a.vocab, v0 + cut.chunk), n = v1 - v0;
    const int row0 = blockIdx.x * cut.rows_cta, row1 = min(a.rows, row0 + cut.rows_cta);
    const int words = (a.vocab + 31) / 32;

    int r0 = row0;
    while (r0 < row1) {
        // the run of rows of one request
        const int req = a.req ? __ldg(a.req + r0) : r0;
        int r1 = r0 + 1;
        while (r1 < row1 && (a.req ? __ldg(a.req + r1) : r1) == req) ++r1;
        const bool asks = req >= 0 && req < a.n_req && (a.hist || a.bias_ids);
        if (asks) {
            for (int i = tid; i < (n + 3) / 4; i += kThreads) reinterpret_cast<uint4*>(word)[i] = make_uint4(0, 0, 0, 0);
            __syncthreads();
            if (a.bias_ids) {
                const int len = a.bias_len ? min(max(__ldg(a.bias_len + req), 0), a.bias_ld) : a.bias_ld;
                for (int i = tid; i < len; i += kThreads) {
                    const unsigned v = static_cast<unsigned>(__ldg(a.bias_ids + static_cast<size_t>(req) * a.bias_ld + i) - v0);
                    if (v < static_cast<unsigned>(n)) atomicMax(&word[v], static_cast<uint32_t>(i + 1) << kCountBits);
                }
                __syncthreads();
            }
            if (a.hist) {
                const int len = a.hist_len ? min(max(__ldg(a.hist_len + req), 0), a.hist_ld) : a.hist_ld;
                const int* h = a.hist + static_cast<size_t>(req) * a.hist_ld;
                auto count = [&](int id) {
                    const unsigned v = static_cast<unsigned>(id - v0);
                    if (v < static_cast<unsigned>(n)) atomicAdd(&word[v], 1u);
                };
                // whole 16-byte pieces, and what is before and behind them
                const int lead = min(len, static_cast<int>((16 - reinterpret_cast<uintptr_t>(h) % 16) % 16 / 4));
                const int4* h4 = reinterpret_cast<const int4*>(h + lead);
                const int n4 = (len - lead) / 4;
                if (tid < lead) count(__ldg(h + tid));
                if (tid < len - lead - 4 * n4) count(__ldg(h + lead + 4 * n4 + tid));
#pragma unroll 2
                for (int i = tid; i < n4; i += kThreads) {
                    const int4 x = __ldg(h4 + i);
                    count(x.x);
                    count(x.y);
                    count(x.z);
                    count(x.w);
                }
            }
            __syncthreads();
        }
        const float rep = asks && a.rep ? __ldg(a.rep + req) : 1.0f;
        const float freq = asks && a.freq ? __ldg(a.freq + req) : 0.0f;
        const float pres = asks && a.pres ? __ldg(a.pres + req) : 0.0f;
        const float* bias = a.bias_ids && asks ? a.bias + static_cast<size_t>(req) * a.bias_ld : nullptr;

        // warp jobs: (row, share of the stretch), shares of whole groups
        for (int job = warp; job < (r1 - r0) * cut.split; job += kWarps) {
            const int row = r0 + job / cut.split, share = job % cut.split, groups = (n + kGroup - 1) / kGroup;
            const int g0 = groups * share / cut.split * kGroup, g1 = min(n, groups * (share + 1) / cut.split * kGroup);
            const T* src = static_cast<const T*>(a.logits) + static_cast<size_t>(row) * a.ld + v0;
            T* dst = a.out ? static_cast<T*>(a.out) + static_cast<size_t>(row) * a.ld_out + v0 : nullptr;
            const int g = a.grammar ? __ldg(a.grammar_row + row) : -1;
            const uint32_t* allow = g >= 0 && g < a.n_grammar ? a.grammar + static_cast<size_t>(g) * words + v0 / 32 : nullptr;
            const int cur = a.cur ? __ldg(a.cur + row) - v0 : -1, mask = a.mask_id < 0 ? -1 : a.mask_id - v0;
            float m = -INFINITY;
            float2 s[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
            int arg = kChunk;
            for (int base = g0; base < g1; base += kGroup * kGroups) {
                const int i0 = base + 4 * lane;
                float z[kGroups][4];
                // (a warp's groups lie whole in the stretch but for the vocabulary's end)
                const bool whole = VEC && base + kGroup * kGroups <= g1;
                if (whole) {
#pragma unroll
                    for (int u = 0; u < kGroups; ++u) Io<T>::get4(src + i0 + u * kGroup, z[u]);
                } else {
#pragma unroll
                    for (int u = 0; u < kGroups; ++u)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            z[u][i] = i0 + u * kGroup + i < g1 ? Io<T>::get(src + i0 + u * kGroup + i) : -INFINITY;
                }
                if (asks) {
#pragma unroll
                    for (int u = 0; u < kGroups; ++u) {
                        if (!whole && i0 + u * kGroup >= g1) break;
                        const uint4 x = *reinterpret_cast<const uint4*>(word + i0 + u * kGroup);
                        if (x.x | x.y | x.z | x.w) {
                            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const uint32_t c = w[i] & ((1u << kCountBits) - 1), k = w[i] >> kCountBits;
                                if (c) {
                                    const float f = z[u][i] > 0.0f ? __fdiv_rn(z[u][i], rep) : __fmul_rn(z[u][i], rep);
                                    z[u][i] = __fsub_rn(f, __fadd_rn(__fmul_rn(freq, static_cast<float>(c)), pres));
                                }
                                if (k) z[u][i] = __fadd_rn(z[u][i], __ldg(bias + k - 1));
                            }
                        }
                    }
                }
                if (allow) {
#pragma unroll
                    for (int u = 0; u < kGroups; ++u) {
                        if (!whole && i0 + u * kGroup >= g1) break;
                        const uint32_t ok = __ldg(allow + ((i0 + u * kGroup) >> 5)) >> (i0 & 31);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (!((ok >> i) & 1u)) z[u][i] = -INFINITY;
                    }
                }
                if (dst) {
                    if (whole) {
#pragma unroll
                        for (int u = 0; u < kGroups; ++u) Io<T>::put4(dst + i0 + u * kGroup, z[u]);
                    } else {
#pragma unroll
                        for (int u = 0; u < kGroups; ++u)
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if (i0 + u * kGroup + i < g1) Io<T>::put(dst + i0 + u * kGroup + i, z[u][i]);
                    }
                }
                // the current id's logit, and the mask id out of the decision
                if (static_cast<unsigned>(cur - base) < kGroup * kGroups && cur < g1) {
#pragma unroll
                    for (int u = 0; u < kGroups; ++u)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (cur == i0 + u * kGroup + i) zcur[row] = z[u][i];
                }
                if (static_cast<unsigned>(mask - base) < kGroup * kGroups) {
#pragma unroll
                    for (int u = 0; u < kGroups; ++u)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (mask == i0 + u * kGroup + i) z[u][i] = -INFINITY;
                }
                float mx = -INFINITY;
#pragma unroll
                for (int u = 0; u < kGroups; ++u) mx = fmaxf(mx, fmaxf(fmaxf(z[u][0], z[u][1]), fmaxf(z[u][2], z[u][3])));
                if (mx > m) {  // rare after the first groups
                    const float al = exp_below(m, mx);
                    s[0] = make_float2((s[0].x + s[0].y + s[1].x + s[1].y) * al, 0.0f);
                    s[1] = make_float2(0.0f, 0.0f);
                    m = mx;
#pragma unroll
                    for (int u = kGroups - 1; u >= 0; --u)
#pragma unroll
                        for (int i = 3; i >= 0; --i)
                            if (z[u][i] == mx) arg = i0 + u * kGroup + i;
                }
                // (the difference first: z and m may be the type's lowest value, whose product overflows)
                const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
                for (int u = 0; u < kGroups; ++u) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float2 e = mul2(sub2(make_float2(z[u][2 * i], z[u][2 * i + 1]), ref), kLog2e);
                        e.x = ex2(e.x);
                        e.y = ex2(e.y);
                        s[i] = add2(s[i], e);
                    }
                }
            }
            float sum = (s[0].x + s[0].y) + (s[1].x + s[1].y);
            // the warp's lanes: largest z, of equal ones the lowest id
#pragma unroll
            for (int d = 16; d; d /= 2) {
                const float om = __shfl_xor_sync(0xffffffffu, m, d), os = __shfl_xor_sync(0xffffffffu, sum, d);
                const int oa = __shfl_xor_sync(0xffffffffu, arg, d);
                const float mx = fmaxf(m, om);
                sum = sum * (m == mx ? 1.0f : exp_below(m, mx)) + os * (om == mx ? 1.0f : exp_below(om, mx));
                arg = om > m ? oa : om < m ? arg : min(arg, oa);
                m = mx;
            }
            if (lane == 0)
                part[(static_cast<size_t>(row) * cut.chunks + blockIdx.y) * cut.split + share] =
                    Part{m, sum, arg < kChunk ? v0 + arg : -1, 0};
        }
        __syncthreads();
        r0 = r1;
    }
}

// A warp joins a row's parts (in order of ids).
__global__ void __launch_bounds__(128) k_merge(const __grid_constant__ dllm_serve_logits_args a, int parts,
                                               const Part* __restrict__ part, const float* __restrict__ zcur) {
    pdl_wait();
    const int row = blockIdx.x * 4 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (row >= a.rows) return;
    float m = -INFINITY, s = 0.0f;
    int arg = a.vocab;
    for (int i = lane; i < parts; i += 32) {
        const Part p = part[static_cast<size_t>(row) * parts + i];
        const float mx = fmaxf(m, p.m);
        s = s * (m == mx ? 1.0f : exp_below(m, mx)) + p.s * (p.m == mx ? 1.0f : exp_below(p.m, mx));
        if (p.m > m) arg = p.arg;
        m = mx;
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

// Rows of a request share its words and the reading of its lists; CTAs enough to fill the GPU come first.
// (512 rows of 126464 ids in 32-row CTAs of 8192 ids, 256 of them: 274 us.)
Cut logits_cut(int rows, int vocab, int n_req, int sms) {
    Cut c;
    const int per = n_req > 0 ? rows / n_req : 1;
    c.rows_cta = per < 1 ? 1 : per > 32 ? 32 : per;
    c.chunk = kChunk;
    auto ctas = [&] {
        return static_cast<long long>((rows + c.rows_cta - 1) / c.rows_cta) * ((vocab + c.chunk - 1) / c.chunk);
    };
    while (c.rows_cta > kWarps && ctas() < 6ll * sms) c.rows_cta = (c.rows_cta + 1) / 2;
    while (c.chunk > 2048 && ctas() < sms) c.chunk /= 2;
    c.chunks = (vocab + c.chunk - 1) / c.chunk;
    const int most = c.chunk / (kGroup * kGroups);
    c.split = (kWarps + c.rows_cta - 1) / c.rows_cta;
    if (c.split > most) c.split = most;
    return c;
}

template <typename T>
cudaError_t go(const dllm_serve_logits_args& a, const Cut& c, Part* part, float* zcur, cudaStream_t st) {
    const dim3 grid((a.rows + c.rows_cta - 1) / c.rows_cta, c.chunks);
    const bool vec = reinterpret_cast<uintptr_t>(a.logits) % (4 * sizeof(T)) == 0 && a.ld % 4 == 0 &&
                     reinterpret_cast<uintptr_t>(a.out) % (4 * sizeof(T)) == 0 && (!a.out || a.ld_out % 4 == 0);
    if (vec) k_logits<T, true><<<grid, kThreads, c.chunk * 4, st>>>(a, c, part, zcur);
    else k_logits<T, false><<<grid, kThreads, c.chunk * 4, st>>>(a, c, part, zcur);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess || !(a.x0 || a.conf || a.tokconf)) return e;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((a.rows + 3) / 4);
    cfg.blockDim = dim3(128);
    cfg.stream = st;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, k_merge, a, c.chunks * c.split, static_cast<const Part*>(part), static_cast<const float*>(zcur));
}

}  // namespace

size_t serve_logits_bytes(int rows, int vocab) {
    // the most parts that a cut makes of a row: eight of each 8192 ids, or one of each 512
    const size_t parts = static_cast<size_t>((vocab + kChunk - 1) / kChunk) * kWarps * 2;
    return serve_round(static_cast<size_t>(rows) * 4) + serve_round(static_cast<size_t>(rows) * parts * sizeof(Part));
}

cudaError_t launch_serve_logits(const dllm_serve_logits_args& a, int sms, cudaStream_t st) {
    const Cut c = logits_cut(a.rows, a.vocab, a.hist || a.bias_ids ? a.n_req : 0, sms);
    float* zcur = static_cast<float*>(a.ws);
    Part* part = reinterpret_cast<Part*>(static_cast<char*>(a.ws) + serve_round(static_cast<size_t>(a.rows) * 4));
    return a.dtype == DLLM_F32    ? go<float>(a, c, part, zcur, st)
           : a.dtype == DLLM_BF16 ? go<__nv_bfloat16>(a, c, part, zcur, st)
                                  : go<__half>(a, c, part, zcur, st);
}

}  // namespace dllm
