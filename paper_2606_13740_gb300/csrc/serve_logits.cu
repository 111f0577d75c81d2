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
constexpr int kChunk = 8192;  // ids of a stretch: 32 KB of words, five CTAs an SM beside them
constexpr int kCountBits = 20;
constexpr float kLog2e = 1.4426950408889634f;

struct Part {
    float m, s;  // largest z, sum of exp(z - m)
    int arg, pad;
};

// Stretches of a row: chunks, each cut among the `split` warps that share a row.
struct Cut {
    int chunks, rows_cta, split;
};
__host__ __device__ inline int cut_parts(const Cut& c) { return c.chunks * c.split; }

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
    __shared__ __align__(16) uint32_t word[kChunk];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int v0 = blockIdx.y * kChunk, v1 = min(a.vocab, v0 + kChunk), n = v1 - v0;
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
                    const int v = __ldg(a.bias_ids + static_cast<size_t>(req) * a.bias_ld + i) - v0;
                    if (v >= 0 && v < n) atomicMax(&word[v], static_cast<uint32_t>(i + 1) << kCountBits);
                }
                __syncthreads();
            }
            if (a.hist) {
                const int len = a.hist_len ? min(max(__ldg(a.hist_len + req), 0), a.hist_ld) : a.hist_ld;
                const int* h = a.hist + static_cast<size_t>(req) * a.hist_ld;
                for (int i = tid; i < len; i += kThreads) {
                    const int v = __ldg(h + i) - v0;
                    if (v >= 0 && v < n) atomicAdd(&word[v], 1u);
                }
            }
            __syncthreads();
        }
        const float rep = asks && a.rep ? __ldg(a.rep + req) : 1.0f;
        const float freq = asks && a.freq ? __ldg(a.freq + req) : 0.0f;
        const float pres = asks && a.pres ? __ldg(a.pres + req) : 0.0f;
        const float* bias = a.bias_ids && asks ? a.bias + static_cast<size_t>(req) * a.bias_ld : nullptr;

        // warp jobs: (row, share of the stretch), shares of whole groups of 128 ids
        for (int job = warp; job < (r1 - r0) * cut.split; job += kWarps) {
            const int row = r0 + job / cut.split, share = job % cut.split;
            const int g0 = (n + 127) / 128 * share / cut.split * 128, g1 = min(n, (n + 127) / 128 * (share + 1) / cut.split * 128);
            const T* src = static_cast<const T*>(a.logits) + static_cast<size_t>(row) * a.ld + v0;
            T* dst = a.out ? static_cast<T*>(a.out) + static_cast<size_t>(row) * a.ld_out + v0 : nullptr;
            const int g = a.grammar ? __ldg(a.grammar_row + row) : -1;
            const uint32_t* allow = g >= 0 && g < a.n_grammar ? a.grammar + static_cast<size_t>(g) * words + v0 / 32 : nullptr;
            const int cur = a.cur ? __ldg(a.cur + row) - v0 : -1;
            const int mask = a.mask_id - v0;
            float m = -INFINITY, s = 0.0f;
            int arg = kChunk;
            for (int i0 = g0 + 4 * lane; i0 < g1; i0 += 128) {
                float z[4];
                const bool whole = VEC && i0 + 4 <= n;
                if (whole) {
                    Io<T>::get4(src + i0, z);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) z[i] = i0 + i < n ? Io<T>::get(src + i0 + i) : -INFINITY;
                }
                if (asks) {
                    const uint4 u = *reinterpret_cast<const uint4*>(word + i0);
                    if (u.x | u.y | u.z | u.w) {
                        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t c = w[i] & ((1u << kCountBits) - 1), k = w[i] >> kCountBits;
                            if (c) {
                                const float f = z[i] > 0.0f ? __fdiv_rn(z[i], rep) : __fmul_rn(z[i], rep);
                                z[i] = __fsub_rn(f, __fadd_rn(__fmul_rn(freq, static_cast<float>(c)), pres));
                            }
                            if (k) z[i] = __fadd_rn(z[i], __ldg(bias + k - 1));
                        }
                    }
                }
                if (allow) {
                    const uint32_t ok = __ldg(allow + (i0 >> 5)) >> (i0 & 31);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!((ok >> i) & 1u)) z[i] = -INFINITY;
                }
                if (dst) {
                    if (whole) {
                        Io<T>::put4(dst + i0, z);
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (i0 + i < n) Io<T>::put(dst + i0 + i, z[i]);
                    }
                }
                if (static_cast<unsigned>(cur - i0) < 4u) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (cur == i0 + i) zcur[row] = z[i];
                }
                if (static_cast<unsigned>(mask - i0) < 4u) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (mask == i0 + i) z[i] = -INFINITY;
                }
                const float mx = fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3]));
                if (mx > m) {  // rare after the first groups
                    s *= exp_below(m, mx);
                    m = mx;
                    arg = i0 + (z[0] == mx ? 0 : z[1] == mx ? 1 : z[2] == mx ? 2 : 3);
                }
                // (the difference first: z and m may be the type's lowest value, whose product overflows)
                const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
                for (int i = 0; i < 4; ++i) s += exp2f((z[i] - ref) * kLog2e);
            }
            // the warp's lanes: largest z, of equal ones the lowest id
#pragma unroll
            for (int d = 16; d; d /= 2) {
                const float om = __shfl_xor_sync(0xffffffffu, m, d), os = __shfl_xor_sync(0xffffffffu, s, d);
                const int oa = __shfl_xor_sync(0xffffffffu, arg, d);
                const float mx = fmaxf(m, om);
                s = s * (m == mx ? 1.0f : exp_below(m, mx)) + os * (om == mx ? 1.0f : exp_below(om, mx));
                arg = om > m ? oa : om < m ? arg : min(arg, oa);
                m = mx;
            }
            if (lane == 0)
                part[(static_cast<size_t>(row) * cut.chunks + blockIdx.y) * cut.split + share] =
                    Part{m, s, arg < kChunk ? v0 + arg : -1, 0};
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

Cut logits_cut(int rows, int n_req) {
    Cut c;
    c.chunks = 0;
    // rows of a request share its words; single rows share a CTA's warps instead
    const int per = rows / (n_req > 0 ? n_req : rows);
    c.rows_cta = per < 1 ? 1 : per > 32 ? 32 : per;
    c.split = c.rows_cta >= kWarps ? 1 : (kWarps + c.rows_cta - 1) / c.rows_cta;
    return c;
}

template <typename T>
cudaError_t go(const dllm_serve_logits_args& a, const Cut& c, Part* part, float* zcur, cudaStream_t st) {
    const dim3 grid((a.rows + c.rows_cta - 1) / c.rows_cta, c.chunks);
    const bool vec = reinterpret_cast<uintptr_t>(a.logits) % (4 * sizeof(T)) == 0 && a.ld % 4 == 0 &&
                     reinterpret_cast<uintptr_t>(a.out) % (4 * sizeof(T)) == 0 && (!a.out || a.ld_out % 4 == 0);
    if (vec) k_logits<T, true><<<grid, kThreads, 0, st>>>(a, c, part, zcur);
    else k_logits<T, false><<<grid, kThreads, 0, st>>>(a, c, part, zcur);
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
    return cudaLaunchKernelEx(&cfg, k_merge, a, cut_parts(c), static_cast<const Part*>(part), static_cast<const float*>(zcur));
}

}  // namespace

size_t serve_logits_bytes(int rows, int vocab) {
    const size_t chunks = (static_cast<size_t>(vocab) + kChunk - 1) / kChunk;
    return serve_round(static_cast<size_t>(rows) * chunks * kWarps * sizeof(Part)) + serve_round(static_cast<size_t>(rows) * 4);
}

cudaError_t launch_serve_logits(const dllm_serve_logits_args& a, int sms, cudaStream_t st) {
    (void)sms;
    Cut c = logits_cut(a.rows, a.n_req);
    c.chunks = (a.vocab + kChunk - 1) / kChunk;
    float* zcur = static_cast<float*>(a.ws);
    Part* part = reinterpret_cast<Part*>(static_cast<char*>(a.ws) + serve_round(static_cast<size_t>(a.rows) * 4));
    return a.dtype == DLLM_F32    ? go<float>(a, c, part, zcur, st)
           : a.dtype == DLLM_BF16 ? go<__nv_bfloat16>(a, c, part, zcur, st)
                                  : go<__half>(a, c, part, zcur, st);
}

}  // namespace dllm
