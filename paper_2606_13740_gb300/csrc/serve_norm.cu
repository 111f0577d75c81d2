// Queries and keys of a step's rows: RMSNorm of each head, rotate-half RoPE, and keys and values to their
// slots of the paged cache, in one pass (include/dllm_serve.h, dllm_serve_qk_norm_rope).
//
// A head of hd features is held by hd / 16 lanes, each with the 8 features from 8 l on and the 8 from
// hd / 2 + 8 l on: the rotation's partners are in one thread, loads and stores are 16 bytes a lane, and the
// mean of squares takes two or three shuffles.  A warp takes heads of one row, the next ones loading while
// it works on a pass, and makes the row's hd / 2 angles once, one or two a lane, shared through shared memory.
// An angle is position x theta as an integer: theta / 2 pi in units of 2^-64 of a turn, so that the product's
// whole turns fall off its top and the rotation is as exact at position 10^6 as at 1.  (In 64-bit floating
// point, of which the SM does two operations a cycle, the angles of 1201 rows took a fifth of the call.)
// Bound: memory, each value once in and once out.  Measured in a graph: 16384 rows of 96 heads of 128 (805 MB)
// 131.3 us, 6.1 TB/s, and from 32 bits (1208 MB) 199.6, 6.05 TB/s, though that form spills some 70 bytes a thread; 32
// rows 2.8 us, the latency of a row; 1201 rows of 36 heads 7.6 us (751 CTAs, and 80 registers leave places for 456).
#include "serve.cuh"

namespace dllm {

namespace {

constexpr int kWarpsPerCta = 8;

// 8 values as they lie in memory, and as floats
template <typename T>
struct Raw8 {
    uint4 u;
    __device__ __forceinline__ void load(const T* p) { u = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void get(float* v) const {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = Half2<T>::unpack(w[i]);
            v[2 * i] = f.x;
            v[2 * i + 1] = f.y;
        }
    }
};
template <>
struct Raw8<float> {
    float4 f[2];
    __device__ __forceinline__ void load(const float* p) {
        f[0] = reinterpret_cast<const float4*>(p)[0];
        f[1] = reinterpret_cast<const float4*>(p)[1];
    }
    __device__ __forceinline__ void get(float* v) const {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            v[4 * i] = f[i].x;
            v[4 * i + 1] = f[i].y;
            v[4 * i + 2] = f[i].z;
            v[4 * i + 3] = f[i].w;
        }
    }
};
// theta / 2 pi in units of 2^-64 of a turn, whole turns dropped: theta is a whole number below 2^24 times a
// power of two, the number's product with the first 64 bits of 1 / 2 pi is exact, and what the bits behind
// them would add is below 2^-40 / 2^23 of a turn a position (theta <= 1).
__device__ __forceinline__ unsigned long long turns_of(float theta) {
    const uint32_t u = __float_as_uint(theta);
    const int e = static_cast<int>((u >> 23) & 255u);
    const unsigned long long mant = (u & 0x7fffffu) | (e ? 0x800000u : 0u), per = 0x28be60db9391054aull;
    const unsigned long long lo = mant * per, hi = __umul64hi(mant, per);
    const int sh = 150 - max(e, 1);  // theta = mant 2^-sh
    unsigned long long t;
    if (sh <= 0) t = sh > -64 ? lo << -sh : 0;
    else if (sh < 64) t = (hi << (64 - sh)) | (lo >> sh);
    else t = sh < 128 ? hi >> (sh - 64) : 0;
    return u >> 31 ? 0ull - t : t;
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
__global__ void __launch_bounds__(kWarpsPerCta * 32, 3) k_serve_norm(ServeShape s, ServeNormArgs a, int parts) {
    constexpr int kLanes = HD / 16, kHeads = 32 / kLanes;  // lanes of a head, heads of a warp's pass
    const int lane = threadIdx.x & 31, l = lane % kLanes, sub = lane / kLanes;
    const long long wid = static_cast<long long>(blockIdx.x) * kWarpsPerCta + (threadIdx.x >> 5);
    const long long row = wid / parts;
    const int part = static_cast<int>(wid - row * parts);
    pdl_wait();
    if (row >= a.rows) return;
    const int H = s.H, Hkv = s.Hkv;
    const int pos = a.pos[row];
    int slot = a.slot[row];
    if (slot >= s.n_pages * s.page) {
        if (lane == 0) atomicOr(a.status, DLLM_SERVE_SLOT);
        slot = -1;
    }

    const int heads = H + 2 * Hkv, step = parts * kHeads;
    struct Pass {
        Raw8<TI> x, y;
    };
    auto fetch = [&](int h, Pass& r) {  // head h of q, k and v in a row
        if (h >= heads || (h >= H && slot < 0)) return;
        const TI* src = h < H         ? static_cast<const TI*>(a.q) + row * a.ldq + static_cast<long long>(h) * HD
                        : h < H + Hkv ? static_cast<const TI*>(a.k) + row * a.ldk + static_cast<long long>(h - H) * HD
                                      : static_cast<const TI*>(a.v) + row * a.ldv + static_cast<long long>(h - H - Hkv) * HD;
        r.x.load(src + 8 * l);
        r.y.load(src + HD / 2 + 8 * l);
    };
    // two passes on their way while a third is worked on
    Pass r0, r1;
    int h = part * kHeads + sub;
    fetch(h, r0);
    fetch(h + step, r1);

    __shared__ float4 angles[kWarpsPerCta][2][HD / 8];  // cosines, sines
    {
        float* c = reinterpret_cast<float*>(angles[threadIdx.x >> 5][0]);
        float* d = reinterpret_cast<float*>(angles[threadIdx.x >> 5][1]);
#pragma unroll
        for (int i = lane; i < HD / 2; i += 32) {
            const unsigned long long turn = turns_of(a.theta[i]) * static_cast<unsigned long long>(static_cast<long long>(pos));
            // the part of a turn, -1/2 .. 1/2, in units of pi
            sincospif(static_cast<float>(static_cast<int>(turn >> 32)) * 4.656612873077393e-10f, d + i, c + i);
        }
        __syncwarp();
    }

    TO* kc = static_cast<TO*>(a.kc);
    TO* vc = static_cast<TO*>(a.vc);
    const long long at = slot < 0 ? 0 : (slot >> s.page_log2) * s.page_stride + static_cast<long long>(slot & (s.page - 1)) * HD;
    auto work = [&](int h, Pass& r) {
        const bool is_q = h < H, is_k = !is_q && h < H + Hkv, live = h < heads && (is_q || slot >= 0);
        float x[8], y[8];
        r.x.get(x);
        r.y.get(y);
        fetch(h + 2 * step, r);
        float ss = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss += x[i] * x[i] + y[i] * y[i];
#pragma unroll
        for (int d = 1; d < kLanes; d *= 2) ss += __shfl_xor_sync(0xffffffffu, ss, d);
        if (!live) return;
        TO* dst;
        if (is_q || is_k) {
            const float scale = rsqrtf(ss * (1.0f / HD) + a.eps);
            const float* gain = is_q ? a.q_gain : a.k_gain;
            const float4 *pc = angles[threadIdx.x >> 5][0] + 2 * l, *pd = angles[threadIdx.x >> 5][1] + 2 * l;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float4 c4 = pc[k], d4 = pd[k];
                const float c[4] = {c4.x, c4.y, c4.z, c4.w}, d[4] = {d4.x, d4.y, d4.z, d4.w};
                float gx[4] = {1.0f, 1.0f, 1.0f, 1.0f}, gy[4] = {1.0f, 1.0f, 1.0f, 1.0f};
                if (gain) {
                    const float4 g4 = reinterpret_cast<const float4*>(gain + 8 * l)[k], h4 = reinterpret_cast<const float4*>(gain + HD / 2 + 8 * l)[k];
                    gx[0] = g4.x, gx[1] = g4.y, gx[2] = g4.z, gx[3] = g4.w;
                    gy[0] = h4.x, gy[1] = h4.y, gy[2] = h4.z, gy[3] = h4.w;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float u = x[4 * k + i] * scale * gx[i], w = y[4 * k + i] * scale * gy[i];
                    x[4 * k + i] = u * c[i] - w * d[i];
                    y[4 * k + i] = w * c[i] + u * d[i];
                }
            }
            dst = is_q ? static_cast<TO*>(a.q_out) + row * a.ld_out + static_cast<long long>(h) * HD
                       : kc + at + static_cast<long long>(h - H) * s.page * HD;
        } else {
            dst = vc + at + static_cast<long long>(h - H - Hkv) * s.page * HD;
        }
        store8(dst + 8 * l, x);
        store8(dst + HD / 2 + 8 * l, y);
    };
    const int passes = (heads - part * kHeads + step - 1) / step;  // the warp's
    for (int i = 0; i < passes; i += 2, h += 2 * step) {
        work(h, r0);
        if (i + 1 < passes) work(h + step, r1);
    }
}

template <int HD, typename TI, typename TO>
cudaError_t go(const ServeShape& s, const ServeNormArgs& a, int sms, cudaStream_t st) {
    constexpr int kHeads = 32 / (HD / 16);
    const int passes = (s.H + 2 * s.Hkv + kHeads - 1) / kHeads;
    // Few rows: a warp for each pass; many: half a row a warp, which makes the row's angles for that.  (1201 rows of 9
    // passes: 9 warps a row 8.6 us, 5 7.6; 16384 rows of 24: one 134, two 130.)
    long long parts = (static_cast<long long>(sms) * 32 + a.rows - 1) / a.rows;
    if (parts < 2) parts = 2;
    if (parts > passes) parts = passes;
    const long long ctas = (a.rows * parts + kWarpsPerCta - 1) / kWarpsPerCta;
    return serve_launch(k_serve_norm<HD, TI, TO>, dim3(static_cast<unsigned>(ctas)), kWarpsPerCta * 32, 0, st, s, a, static_cast<int>(parts));
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
