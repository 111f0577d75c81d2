// Queries and keys of a step's rows: RMSNorm of each head, rotate-half RoPE, and keys and values to their
// slots of the paged cache, in one pass (include/dllm_serve.h, dllm_serve_qk_norm_rope).
//
// A head of hd features is held by hd / 16 lanes, each with the 8 features from 8 l on and the 8 from
// hd / 2 + 8 l on: the rotation's partners are in one thread, loads and stores are 16 bytes a lane, and the
// mean of squares takes two or three shuffles.  A warp takes heads of one row, so that the row's hd / 2
// angles are made once a warp (one or two a lane) and travel by shuffles.  The angle is position x theta in
// 64 bits, reduced to a part of a turn before it is rounded to 32 bits: the rotation is as exact at position
// 10^6 as at 1.  Bound: memory, each value once in and once out.
#include "serve.cuh"

namespace dllm {

namespace {

constexpr int kWarpsPerCta = 8;

template <typename T>
__device__ __forceinline__ void load8(const T* p, float* v) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = Half2<T>::unpack(w[i]);
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}
template <>
__device__ __forceinline__ void load8<float>(const float* p, float* v) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float4 f = reinterpret_cast<const float4*>(p)[i];
        v[4 * i] = f.x;
        v[4 * i + 1] = f.y;
        v[4 * i + 2] = f.z;
        v[4 * i + 3] = f.w;
    }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float* v) {
    uint4 u;
    u.x = Half2<T>::pack(v[0], v[1]);
    u.y = Half2<T>::pack(v[2], v[3]);
    u.z = Half2<T>::pack(v[4], v[5]);
    u.w = Half2<T>::pack(v[6], v[7]);
    *reinterpret_cast<uint4*>(p) = u;
}

// parts: warps that share a row.  Not __restrict__ / read-only for q: q_out may be q (a warp reads a head
// before it writes it, and nobody else reads it).
template <int HD, typename TI, typename TO>
__global__ void __launch_bounds__(kWarpsPerCta * 32) k_serve_norm(ServeShape s, ServeNormArgs a, int parts) {
    constexpr int kLanes = HD / 16, kHeads = 32 / kLanes;  // lanes of a head, heads of a warp's pass
    const int lane = threadIdx.x & 31, l = lane % kLanes, sub = lane / kLanes;
    const long long wid = static_cast<long long>(blockIdx.x) * kWarpsPerCta + (threadIdx.x >> 5);
    const long long row = wid / parts;
    const int part = static_cast<int>(wid - row * parts);
    if (row >= a.rows) return;
    const int H = s.H, Hkv = s.Hkv;
    const int pos = __ldg(a.pos + row);
    int slot = __ldg(a.slot + row);
    if (slot >= s.n_pages * s.page) {
        if (lane == 0) atomicOr(a.status, DLLM_SERVE_SLOT);
        slot = -1;
    }

    // cos and sin of pairs lane, lane + 32; then those of pairs 8 l .. 8 l + 7
    float cs[8], sn[8];
    {
        float c[HD / 64], d[HD / 64];
#pragma unroll
        for (int i = 0; i < HD / 64; ++i) {
            const double turns = static_cast<double>(pos) * (static_cast<double>(__ldg(a.theta + lane + 32 * i)) * 0.15915494309189533577);
            sincospif(2.0f * static_cast<float>(turns - rint(turns)), &d[i], &c[i]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int p = 8 * l + i, src = p & 31;
            cs[i] = __shfl_sync(0xffffffffu, c[0], src);
            sn[i] = __shfl_sync(0xffffffffu, d[0], src);
            if constexpr (HD == 128) {
                const float c1 = __shfl_sync(0xffffffffu, c[1], src), d1 = __shfl_sync(0xffffffffu, d[1], src);
                if (p >= 32) {
                    cs[i] = c1;
                    sn[i] = d1;
                }
            }
        }
    }

    TO* kc = static_cast<TO*>(a.kc);
    TO* vc = static_cast<TO*>(a.vc);
    const long long at = slot < 0 ? 0 : (slot >> s.page_log2) * s.page_stride + static_cast<long long>(slot & (s.page - 1)) * HD;
    const int heads = H + 2 * Hkv;
    for (int h0 = part * kHeads; h0 < heads; h0 += parts * kHeads) {
        const int h = h0 + sub;
        const bool is_q = h < H, is_k = !is_q && h < H + Hkv, live = h < heads && (is_q || slot >= 0);
        float x[8], y[8];
        if (live) {
            const TI* src = is_q   ? static_cast<const TI*>(a.q) + row * a.ldq + static_cast<long long>(h) * HD
                            : is_k ? static_cast<const TI*>(a.k) + row * a.ldk + static_cast<long long>(h - H) * HD
                                   : static_cast<const TI*>(a.v) + row * a.ldv + static_cast<long long>(h - H - Hkv) * HD;
            load8(src + 8 * l, x);
            load8(src + HD / 2 + 8 * l, y);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = y[i] = 0.0f;
        }
        float ss = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss += x[i] * x[i] + y[i] * y[i];
#pragma unroll
        for (int d = 1; d < kLanes; d *= 2) ss += __shfl_xor_sync(0xffffffffu, ss, d);
        if (!live) continue;
        TO* dst;
        if (is_q || is_k) {
            const float r = rsqrtf(ss * (1.0f / HD) + a.eps);
            const float* gain = is_q ? a.q_gain : a.k_gain;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float u = x[i] * r, w = y[i] * r;
                if (gain) {
                    u *= __ldg(gain + 8 * l + i);
                    w *= __ldg(gain + HD / 2 + 8 * l + i);
                }
                x[i] = u * cs[i] - w * sn[i];
                y[i] = w * cs[i] + u * sn[i];
            }
            dst = is_q ? static_cast<TO*>(a.q_out) + row * a.ld_out + static_cast<long long>(h) * HD
                       : kc + at + static_cast<long long>(h - H) * s.page * HD;
        } else {
            dst = vc + at + static_cast<long long>(h - H - Hkv) * s.page * HD;
        }
        store8(dst + 8 * l, x);
        store8(dst + HD / 2 + 8 * l, y);
    }
}

template <int HD, typename TI, typename TO>
cudaError_t go(const ServeShape& s, const ServeNormArgs& a, int sms, cudaStream_t st) {
    constexpr int kHeads = 32 / (HD / 16);
    const int passes = (s.H + 2 * s.Hkv + kHeads - 1) / kHeads;
    // few rows: a warp for each pass; many: a warp for a whole row, whose angles are made once
    long long parts = (static_cast<long long>(sms) * 64 + a.rows - 1) / a.rows;
    if (parts > passes) parts = passes;
    const long long ctas = (a.rows * parts + kWarpsPerCta - 1) / kWarpsPerCta;
    k_serve_norm<HD, TI, TO><<<static_cast<unsigned>(ctas), kWarpsPerCta * 32, 0, st>>>(s, a, static_cast<int>(parts));
    return cudaGetLastError();
}
template <int HD>
cudaError_t go_types(const ServeShape& s, const ServeNormArgs& a, int in_dtype, int sms, cudaStream_t st) {
    if (s.dtype == DLLM_BF16)
        return in_dtype == DLLM_F32 ? go<HD, float, __nv_bfloat16>(s, a, sms, st)
                                    : go<HD, __nv_bfloat16, __nv_bfloat16>(s, a, sms, st);
    return in_dtype == DLLM_F32 ? go<HD, float, __half>(s, a, sms, st) : go<HD, __half, __half>(s, a, sms, st);
}

}  // namespace

cudaError_t launch_serve_norm(const ServeShape& s, const ServeNormArgs& a, int in_dtype, int sms, cudaStream_t st) {
    return s.hd == 128 ? go_types<128>(s, a, in_dtype, sms, st) : go_types<64>(s, a, in_dtype, sms, st);
}

}  // namespace dllm
