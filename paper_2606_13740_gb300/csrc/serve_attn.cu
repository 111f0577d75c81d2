// Attention of a serving step's rows over the shared prefix and each request's own pages
// (include/dllm_serve.h, dllm_serve_attention): one warp a (row, query head), 32 keys at a time, a lane
// a key for the scores and hd / 32 features a lane for the values.
#include "serve.cuh"

namespace dllm {

namespace {

template <int HD, typename T>
__global__ void __launch_bounds__(128) k_serve_attn(ServeShape s, dllm_serve_tables t, ServeAttnArgs a) {
    constexpr int kF = HD / 32;  // features of a lane
    __shared__ float sq[4][HD];
    ServeArrays w;
    serve_arrays(s, t.work, &w);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long wid = static_cast<long long>(blockIdx.x) * 4 + warp;
    const int row = static_cast<int>(wid / s.H), h = static_cast<int>(wid % s.H), hk = h / s.G;
    if (row >= a.rows) return;
    T* out = static_cast<T*>(a.out) + (static_cast<size_t>(row) * s.H + h) * HD;
    const T* q = static_cast<const T*>(a.q) + row * a.ldq + h * HD;
    for (int i = lane; i < HD; i += 32) sq[warp][i] = static_cast<float>(q[i]) * a.scale;
    __syncwarp();
    const int req = row < w.head->rows ? t.req[row] : -1;
    float m = -INFINITY, l = 0.0f, o[kF] = {};
    const T* kc = static_cast<const T*>(a.kc);
    const T* vc = static_cast<const T*>(a.vc);
    auto span = [&](const int* pages, int n_list, int n) {
        for (int k0 = 0; k0 < n; k0 += 32) {
            const int k = k0 + lane;
            long long at = -1;
            float z = -INFINITY;
            if (k < n) {
                const int idx = k >> s.page_log2, p = idx < n_list ? pages[idx] : -1;
                z = 0.0f;
                if (p >= 0 && p < s.n_pages) {
                    at = p * s.page_stride + (static_cast<long long>(hk) * s.page + (k & (s.page - 1))) * HD;
                    for (int c = 0; c < HD; c += 8) {
                        const uint4 u = *reinterpret_cast<const uint4*>(kc + at + c);
                        const uint32_t x[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float2 f = Half2<T>::unpack(x[i]);
                            z += f.x * sq[warp][c + 2 * i] + f.y * sq[warp][c + 2 * i + 1];
                        }
                    }
                }
            }
            float mx = z;
#pragma unroll
            for (int d = 16; d; d /= 2) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
            mx = fmaxf(mx, m);
            const float ref = mx == -INFINITY ? 0.0f : mx, al = expf(m - ref), p = expf(z - ref);
            float sum = p;
#pragma unroll
            for (int d = 16; d; d /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            l = l * al + sum;
            m = mx;
#pragma unroll
            for (int i = 0; i < kF; ++i) o[i] *= al;
            for (int j = 0; j < min(32, n - k0); ++j) {
                const long long aj = __shfl_sync(0xffffffffu, at, j);
                const float pj = __shfl_sync(0xffffffffu, p, j);
                if (aj < 0) continue;
#pragma unroll
                for (int i = 0; i < kF; ++i) o[i] += pj * static_cast<float>(vc[aj + lane * kF + i]);
            }
        }
    };
    if (req >= 0) {
        span(a.prefix_pages, a.n_prefix, w.head->prefix_len);
        const int q_len = t.row_start[req + 1] - t.row_start[req];
        int n = t.n_keys[req];
        if (n > 0 && w.head->causal) n += row - t.row_start[req] + 1 - q_len;
        span(t.table + static_cast<size_t>(req) * s.max_pages, s.max_pages, n);
    }
    const float il = l > 0.0f || l != l ? 1.0f / l : 0.0f;
#pragma unroll
    for (int i = 0; i < kF; i += 2)
        *reinterpret_cast<uint32_t*>(out + lane * kF + i) = Half2<T>::pack(o[i] * il, o[i + 1] * il);
    if (a.lse && lane == 0) a.lse[static_cast<size_t>(row) * s.H + h] = m + logf(l);
}

template <int HD, typename T>
cudaError_t go(const ServeShape& s, const dllm_serve_tables& t, const ServeAttnArgs& a, cudaStream_t st) {
    const long long ctas = (static_cast<long long>(a.rows) * s.H + 3) / 4;
    k_serve_attn<HD, T><<<static_cast<unsigned>(ctas), 128, 0, st>>>(s, t, a);
    return cudaGetLastError();
}

}  // namespace

size_t serve_partial_bytes(const ServeShape& s) {
    return 0;
}

cudaError_t launch_serve_attention(const ServeShape& s, const dllm_serve_tables& t, const ServeAttnArgs& a, int sms,
                                   cudaStream_t st) {
    (void)sms;
    if (s.dtype == DLLM_BF16)
        return s.hd == 128 ? go<128, __nv_bfloat16>(s, t, a, st) : go<64, __nv_bfloat16>(s, t, a, st);
    return s.hd == 128 ? go<128, __half>(s, t, a, st) : go<64, __half>(s, t, a, st);
}

}  // namespace dllm
