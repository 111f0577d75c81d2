// Attention of a serving step's rows over the shared prefix and each request's own pages
// (include/dllm_serve.h, dllm_serve_attention; with bits that say which new tokens a row sees,
// include/dllm_serve_drafts.h, dllm_serve_tree_attention) on the 5th-generation tensor cores.
//
// A tile is 128 query rows of one K/V head: tile_tokens tokens of the packed batch, whatever requests they
// belong to, with the head's G query heads side by side.  So the prefix's keys and values are loaded once
// for all the requests in the tile.  After the prefix the tile goes through its requests' own blocks of 64
// keys, one request after another: only that request's rows are live then, and the tensor cores leave the
// others' lanes of O as they are (disable-output-lane), so that one request's values, NaN included, never
// reach another's rows.  The plan has cut all tiles' steps into runs of equal cost, one a CTA (serve.cuh); a unit
// (tile, K/V head) that a CTA holds whole is written out, the parts of the others go to a workspace, where
// k_serve_join joins them in the order of their keys.  Per step j:
//   S_j = Q K_j^T         tcgen05.mma, Q and K_j in shared memory (K-major), S_j in tensor memory
//   P_j = exp2(S_j - m)   one thread a query row; P_j (16 bit) written back over S_j
//   O  += P_j V_j         tcgen05.mma, P_j from tensor memory, V_j in shared memory (MN-major)
// The running maximum m is the first block's, and moves only where a block's sum of P passes 2^12 (no maximum is
// looked for otherwise); only then are O and the row's sum rescaled.  P, a floating-point number, loses nothing by
// being larger than 1, and stays far below what f16 holds.  P is rounded to the cache's type, as the tensor
// cores take it; the sum is of the unrounded values.  Warps 0-3: softmax and output (a thread a row); warps 4
// and 7: TMA loads of Q and K, and of V, a box a page and 64 features; warps 5 and 6: the MMAs of S and of
// P V.  (With one warp for the loads and one for the MMAs each spent 2000 cycles a step on them, twice what
// the tensor cores and the softmax take.)
// Keys past a request's end, and those that a row's bits or its place leave out, score -inf.  The values of keys past the
// end, which may be anything, are set to 0 in shared memory.  In a block that rows see in part, values that are infinities or
// NaN are set to 0 as well, as 0 times them would reach the rows that do not see them, and added at the unit's end for
// those that do.  The warp of P V does this while the softmax is at work.  (By the softmax's warps 5 causal prompts under
// 2000 take 111.1 us for 109.6, side by side.)  Keys of a request that has rows in several tiles keep their place in L2 (64 ragged trees, 28
// heads over 4: 79 -> 71 us; for all requests, 16 windows under 4096 shared keys lose 2.6), others leave it first.
// Bound: 0.78 us a step, in which S, softmax and P V of a tile wait for one another, the SM's two CTAs side by side.
// (Of the 128 registers that two CTAs leave a thread, 3 words are spilled in every form.)  Measured in a graph, passes in a
// row, join included: 16 windows of 32 under 4096 shared keys, 32 heads of 128, 55.9 us (189 MB at least: 3.4 TB/s); 96 tokens
// under 8001, 28 heads over 4, 39.5 us (151 MB, 3.8 TB/s); 5 causal prompts under 2000, 110.4 us (127 GFLOP: 1.15 PFLOP/s); one
// token under 300 keys 9.1 us.  By bits: trees of 48 of 16 requests under 2048 shared and up to 1000 own keys, 32 heads, 53.6 us
// (164 MB at least: 3.1 TB/s); 64 ragged trees of up to 61 over up to 2500 own keys, 28 heads over 4, f16, 66.6 us (176 MB, 2.6
// TB/s; own keys are read for 2.7 tiles a request, so that L2 gives 434 MB).
#pragma once

#include "serve.cuh"

namespace dllm {

namespace {

constexpr int kThreads = 256;
constexpr int kHalfQ = kServeRows * 128;    // bytes of 64 features of the Q tile
constexpr int kHalfKV = kServeBlock * 128;  // and of a K or V block
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kSumMax = 4096.0f;  // of a row's P in a block, before its m moves

template <int HD>
constexpr int kStages = HD == 128 ? 2 : 4;  // K/V blocks in flight, two CTAs an SM
// The barriers and flags of a CTA, behind its tiles.  (No static shared memory: two CTAs fill an SM's 228 KB.)
template <int NB>
struct Sync {
    uint64_t qfull, qempty, drain[2], sfull[2], pfull[2], pvdone[2], kfull[NB], vfull[NB], kempty[NB], vempty[NB];
    uint32_t tmem;
    int abort;
    int odd;  // infinities or NaN were taken out of a block of V
};
// (768: from the 256-byte alignment that dynamic shared memory has here to the tiles' 1024)
template <int HD>
constexpr int kSmem = 768 + HD / 64 * (kHalfQ + 2 * kStages<HD> * kHalfKV) + static_cast<int>(sizeof(Sync<kStages<HD>>));
static_assert(kSmem<128> <= 228 * 1024 / 2 - 1024 && kSmem<64> <= 228 * 1024 / 2 - 1024, "two CTAs an SM");

struct Maps {
    CUtensorMap q;  // [rows][Hkv][G][hd], box: 64 features, the group, one head, tile_tokens rows
    CUtensorMap k;  // [n_pages][Hkv * page][hd], box: 64 features of up to 64 places of a page
    CUtensorMap v;
};

__device__ __forceinline__ uint64_t sw128(uint32_t saddr, uint32_t lbo, uint32_t sbo) {
    uint64_t d = 0;
    d |= static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4);
    d |= static_cast<uint64_t>((lbo >> 4) & 0x3FFFu) << 16;
    d |= static_cast<uint64_t>((sbo >> 4) & 0x3FFFu) << 32;
    d |= static_cast<uint64_t>(1u) << 46;  // descriptor version for tcgen05
    d |= static_cast<uint64_t>(2u) << 61;  // 128-byte swizzle
    return d;
}
// D += A B with A from tensor memory, B from shared memory; the lanes of D whose bit in off is set keep
// their value.
__device__ __forceinline__ void umma_tmem_a_masked(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint4 off) {
    asm volatile(
        "{\n .reg .pred p;\n setp.eq.b32 p, 0, 0;\n"
        " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, {%4, %5, %6, %7}, p;\n}\n" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"(off.x), "r"(off.y), "r"(off.z), "r"(off.w)
        : "memory");
}
__device__ __forceinline__ void tmem_st_32u(uint32_t taddr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, "
        "%14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
        "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
        "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tma_3d(void* dst, const CUtensorMap* tm, int x, int y, int z, uint64_t* bar, uint64_t pol) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint"
        " [%0], [%1, {%3, %4, %5}], [%2], %6;" ::"r"(smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(tm)), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z), "l"(pol)
        : "memory");
}
__device__ __forceinline__ void tma_4d(void* dst, const CUtensorMap* tm, int x, int y, int z, int w, uint64_t* bar,
                                       uint64_t pol) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint"
        " [%0], [%1, {%3, %4, %5, %6}], [%2], %7;" ::"r"(smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(tm)), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z), "r"(w), "l"(pol)
        : "memory");
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{\n .reg .b64 a, b, c, d;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n mov.b64 c, {%6, %7};\n"
        " fma.rn.f32x2 d, a, b, c;\n mov.b64 {%0, %1}, d;\n}\n"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
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
__device__ __forceinline__ void st_32b(void* p, const uint32_t* v) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]),
                 "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
}
// 16 registers per thread -> its lane, 16 columns; tmem_wait_st waits for all of a warp's stores
__device__ __forceinline__ void tmem_st_32x16_async(uint32_t taddr, const float* v) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, "
        "%15, %16};" ::"r"(taddr),
        "r"(__float_as_uint(v[0])), "r"(__float_as_uint(v[1])), "r"(__float_as_uint(v[2])), "r"(__float_as_uint(v[3])),
        "r"(__float_as_uint(v[4])), "r"(__float_as_uint(v[5])), "r"(__float_as_uint(v[6])), "r"(__float_as_uint(v[7])),
        "r"(__float_as_uint(v[8])), "r"(__float_as_uint(v[9])), "r"(__float_as_uint(v[10])),
        "r"(__float_as_uint(v[11])), "r"(__float_as_uint(v[12])), "r"(__float_as_uint(v[13])),
        "r"(__float_as_uint(v[14])), "r"(__float_as_uint(v[15]))
        : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// 2^x by the special function unit; below 2^-126: 0
__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// bits lo .. hi - 1 (any ints)
__device__ __forceinline__ uint32_t bit_run(int lo, int hi) {
    lo = min(max(lo, 0), 32);
    hi = min(max(hi, lo), 32);
    const uint32_t up = hi == 32 ? 0xffffffffu : (1u << hi) - 1u;
    return lo == 32 ? 0u : up & ~((1u << lo) - 1u);
}

// Which of 64 keys a row of bits m (words of them) lets it see, the first key being new token d of the request; keys
// before token 0 all of them.  d > -64.
__device__ __forceinline__ uint64_t seen_bits(const uint32_t* m, int words, int d) {
    auto word = [&](int i) { return i < words ? m[i] : 0u; };
    if (d >= 0) {
        const int i = d >> 5;
        const uint32_t a = word(i), b = word(i + 1), c = word(i + 2);
        return static_cast<uint64_t>(__funnelshift_r(b, c, d & 31)) << 32 | __funnelshift_r(a, b, d & 31);
    }
    return (static_cast<uint64_t>(word(1)) << 32 | word(0)) << -d | ((1ull << -d) - 1);
}
// Whether a live row of a block (f: its info, valid: its keys) may see less than all of it, in the tile from token tok0 on.
template <bool TREE>
__device__ __forceinline__ bool sees_partly(const int4& f, int valid, int tok0, int causal) {
    if (TREE && f.w < f.z + valid) return true;  // new tokens among its keys
    return causal && f.w + max(tok0, f.x) - f.x + 1 - f.z < valid;
}
// The first n of 64 bits.
__device__ __forceinline__ uint64_t low_bits(int n) { return n >= 64 ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1; }

// Which of two 16-bit values are infinities or NaN: bits 15 and 31.
template <typename T>
__device__ __forceinline__ uint32_t odd_halves(uint32_t u) {
    constexpr uint32_t kExp = std::is_same<T, __half>::value ? 0x7c007c00u : 0x7f807f80u;
    constexpr uint32_t kOne = std::is_same<T, __half>::value ? 0x04000400u : 0x00800080u;
    return ((u & kExp) + kOne) & 0x80008000u;
}

// One CTA's run of steps, unit by unit: the same walk in every role.
struct Walk {
    const int2* tiles;
    int n_tiles, Hkv, tile, hk, step, left;
    int n, own0, steps;  // steps of the current segment; the tile's first own block, its unit's steps
    int2 next;           // of the next tile, asked for a unit ahead
    __device__ Walk(const ServeArrays& w, int Hkv_, int cta) : tiles(w.tile), n_tiles(w.head->tiles), Hkv(Hkv_) {
        const int4 d = w.cta[2 * cta], e = w.cta[2 * cta + 1];
        tile = d.x;
        hk = d.y;
        step = d.z;
        left = d.w;
        next = make_int2(e.x, e.y);
        enter();
        n = min(left, steps - step);
    }
    __device__ void enter() {
        own0 = next.x;
        steps = next.y;
        next = tiles[min(tile + 1, n_tiles - 1)];
    }
    __device__ bool whole() const { return step == 0 && n == steps; }
    // to the next segment; false: that was the last
    __device__ bool advance() {
        left -= n;
        if (left <= 0) return false;
        step = 0;
        if (++hk == Hkv) {
            hk = 0;
            ++tile;
            enter();
        }
        n = min(left, steps);
        return n > 0;
    }
};

template <int HD, typename T, bool TREE>
__global__ void __launch_bounds__(kThreads, 2)
    k_serve_attn(const __grid_constant__ Maps maps, const __grid_constant__ ServeShape s,
                 const __grid_constant__ dllm_serve_tables t, const __grid_constant__ ServeAttnArgs a) {
    constexpr int NB = kStages<HD>, kParts = HD / 64;
    constexpr int kQ = kParts * kHalfQ, kKV = kParts * kHalfKV;
    ServeArrays w;
    serve_arrays(s, t.work, &w);
    const int cta = blockIdx.x;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *sQ = smem, *sK = sQ + kQ, *sV = sK + NB * kKV;
    Sync<NB>& sy = *reinterpret_cast<Sync<NB>*>(sV + NB * kKV);
    uint64_t &qfull = sy.qfull, &qempty = sy.qempty;
    uint64_t *drain = sy.drain, *sfull = sy.sfull, *pfull = sy.pfull, *pvdone = sy.pvdone;
    uint64_t *kfull = sy.kfull, *vfull = sy.vfull, *kempty = sy.kempty, *vempty = sy.vempty;
    int& s_abort = sy.abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        mbar_init(&qfull, 1);
        mbar_init(&qempty, 1);
        mbar_init(&drain[0], 1);
        mbar_init(&drain[1], 1);
        for (int i = 0; i < NB; ++i) {
            mbar_init(&kfull[i], 1);
            mbar_init(&vfull[i], 1);
            mbar_init(&kempty[i], 1);
            mbar_init(&vempty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sfull[i], 1);
            mbar_init(&pfull[i], 4);
            mbar_init(&pvdone[i], 1);
        }
        s_abort = sy.odd = 0;
        mbar_fence_init();
    }
    if (warp == 4) {
        tmem_alloc(&sy.tmem, 256);  // O: columns 0 .. HD - 1; S and P: 128 .. 191, 192 .. 255
        tmem_relinquish();
    }
    // rows past the tile's tokens (groups that do not divide 128) stay zero: ordinary scores, never read
    for (int i = s.G * s.tile_tokens * 8 + static_cast<int>(threadIdx.x); i < kServeRows * 8; i += kThreads) {
#pragma unroll
        for (int h = 0; h < kParts; ++h) reinterpret_cast<uint4*>(sQ + h * kHalfQ)[i] = make_uint4(0, 0, 0, 0);
    }
    fence_proxy_async_smem();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sy.tmem;
    if (threadIdx.x == 0) {
        tma_prefetch_desc(&maps.q);
        tma_prefetch_desc(&maps.k);
        tma_prefetch_desc(&maps.v);
    }
    // All before this may run while the launch before ends; from here on data and the plan are read (by plain loads:
    // read-only ones need not stay behind the wait).
    pdl_wait();
    pdl_launch_dependents();
    const bool same = serve_same_shape(s, *w.head);  // else the plan of another config, or none
    const int rows = same ? min(w.head->rows, a.rows) : 0, ctas = same ? w.head->ctas : 0;
    const int prefix_blocks = w.head->prefix_blocks, prefix_len = w.head->prefix_len, causal = w.head->causal;
    if (!same && w.head->ctas && threadIdx.x == 0 && cta == 0) atomicOr(t.status, DLLM_SERVE_STATE);
    // rows that are padding
    for (long long i = static_cast<long long>(rows) * s.H * (HD / 8) + static_cast<long long>(cta) * kThreads + threadIdx.x;
         i < static_cast<long long>(a.rows) * s.H * (HD / 8); i += static_cast<long long>(gridDim.x) * kThreads) {
        reinterpret_cast<uint4*>(a.out)[i] = make_uint4(0, 0, 0, 0);
        if (a.lse && i % (HD / 8) == 0) a.lse[i / (HD / 8)] = -INFINITY;
    }
    if (cta >= ctas) {  // (the whole CTA)
        __syncthreads();
        if (warp == 4) tmem_dealloc(tmem, 256);
        return;
    }

    // The load and MMA warps run their loops whole, the outcomes of their waits voted, and one elected lane
    // issues.  Barrier phases count the steps j of the whole run, across its segments.
    auto wait_all = [&](uint64_t* bar, uint32_t parity) {
        return __all_sync(0xffffffffu, mbar_wait(bar, parity, &s_abort, t.status)) != 0;
    };
    Walk at(w, s.Hkv, cta);
    if (warp == 4 || warp == 7) {
        // ------------------------------------------------ loads
        const bool leader = elect_one(), is_k = warp == 4;
        const CUtensorMap* tm = is_k ? &maps.k : &maps.v;
        const uint64_t once = policy_evict_first(), often = policy_evict_last(), again = policy_evict_normal();
        const int lg = s.page_log2, page = s.page, boxes = page < kServeBlock ? kServeBlock >> lg : 1;
        const int n_prefix = min(a.n_prefix, (prefix_len + page - 1) >> lg);
        if (static_cast<long long>(a.n_prefix) * page < prefix_len && cta == 0 && is_k && leader)
            atomicOr(t.status, DLLM_SERVE_PREFIX);
        uint8_t* ring = is_k ? sK : sV;
        uint64_t *full = is_k ? kfull : vfull, *empty = is_k ? kempty : vempty;
        // pages of a segment's step (-1: none, the copy fills in zeros): up to four, or one and the place in it
        auto pages_of = [&](int step) {
            int4 p = make_int4(-1, -1, -1, -1);
            if (step < prefix_blocks) {
                const int i = step * kServeBlock >> lg;
                bool out = false;  // a page that is not of the pool
                auto page_at = [&](int k) {
                    if (k >= n_prefix) return -1;
                    const int id = a.prefix_pages[k];
                    out |= id < 0 || id >= s.n_pages;
                    return id;
                };
                p.x = page_at(i);
                if (page >= kServeBlock) {
                    p.y = step * kServeBlock & (page - 1);
                } else {
                    p.y = page_at(i + 1);
                    if (boxes == 4) {
                        p.z = page_at(i + 2);
                        p.w = page_at(i + 3);
                    }
                }
                if (out) atomicOr(t.status, DLLM_SERVE_PREFIX);
            } else {
                p = w.pages[at.own0 + step - prefix_blocks];
            }
            return p;
        };
        // whether a step's keys are those of a request that has rows in other tiles too
        auto shared_of = [&](int step) {
            if (step < prefix_blocks) return false;
            const int4 f = w.info[at.own0 + step - prefix_blocks];
            return f.x < at.tile * s.tile_tokens || f.y > (at.tile + 1) * s.tile_tokens;
        };
        int j = 0, seg = 0;
        bool ok = true;
        do {
            if (at.left <= 0) break;
            if (is_k) {
                if (seg > 0 && !wait_all(&qempty, static_cast<uint32_t>((seg - 1) & 1))) break;
                if (leader) {
                    mbar_arrive_expect_tx(&qfull, static_cast<uint32_t>(kParts * 128 * s.G * s.tile_tokens));
#pragma unroll
                    for (int p = 0; p < kParts; ++p)
                        tma_4d(sQ + p * kHalfQ, &maps.q, 64 * p, 0, at.hk, at.tile * s.tile_tokens, &qfull, once);
                }
                ++seg;
            }
            int4 cur, nxt = make_int4(-1, 0, -1, -1);
            bool more = false;
            uint32_t reread = 0;
            if (lane < at.n) {
                nxt = pages_of(at.step + lane);
                more = shared_of(at.step + lane);
            }
            for (int i = 0; i < at.n; ++i) {
                if ((i & 31) == 0) {
                    cur = nxt;
                    reread = __ballot_sync(0xffffffffu, more);
                    if (i + 32 + lane < at.n) {
                        nxt = pages_of(at.step + i + 32 + lane);
                        more = shared_of(at.step + i + 32 + lane);
                    }
                }
                const int p0 = __shfl_sync(0xffffffffu, cur.x, i & 31), p1 = __shfl_sync(0xffffffffu, cur.y, i & 31);
                const int p2 = __shfl_sync(0xffffffffu, cur.z, i & 31), p3 = __shfl_sync(0xffffffffu, cur.w, i & 31);
                const int st = j % NB;
                if (j >= NB && !wait_all(&empty[st], static_cast<uint32_t>((j / NB - 1) & 1))) {
                    ok = false;
                    break;
                }
                if (leader) {
                    const uint64_t pol = at.step + i < prefix_blocks ? often : reread >> (i & 31) & 1u ? again : once;
                    uint8_t* dst = ring + st * kKV;
                    const int y = at.hk * page;
                    mbar_arrive_expect_tx(&full[st], kKV);
#pragma unroll
                    for (int h = 0; h < kParts; ++h) {
                        uint8_t* d = dst + h * kHalfKV;
                        if (boxes == 1) {
                            tma_3d(d, tm, 64 * h, y + p1, p0, &full[st], pol);
                        } else {
                            tma_3d(d, tm, 64 * h, y, p0, &full[st], pol);
                            tma_3d(d + page * 128, tm, 64 * h, y, p1, &full[st], pol);
                            if (boxes == 4) {
                                tma_3d(d + page * 256, tm, 64 * h, y, p2, &full[st], pol);
                                tma_3d(d + page * 384, tm, 64 * h, y, p3, &full[st], pol);
                            }
                        }
                    }
                }
                ++j;
            }
        } while (ok && at.advance());
        if (leader && *const_cast<volatile int*>(&s_abort)) {
            // the copies in flight land before the shared memory is released (one deadline for all)
            const long long t0 = spin_clock();
            auto land = [&](uint64_t* bar, int phase) {
                while (!mbar_try_wait(bar, static_cast<uint32_t>(phase & 1)) && spin_clock() - t0 < kWaitLimitCycles) {
                }
            };
            if (seg) land(&qfull, seg - 1);
            for (int k = max(0, j - NB); k < j; ++k) land(&full[k % NB], k / NB);
        }
    } else if (warp >= 5) {
        // ------------------------------------------------ MMA issue
        const bool leader = elect_one();
        const uint32_t t_o = __shfl_sync(0xffffffffu, tmem, 0), t_s = t_o + 128;
        constexpr uint32_t kType = std::is_same<T, __half>::value ? 0u : (1u << 7) | (1u << 10);
        constexpr uint32_t kShape = (1u << 4) | kType | (static_cast<uint32_t>(kServeRows >> 4) << 24);
        int j = 0;
        bool ok = true;
        if (warp == 5) {
            constexpr uint32_t id_s = kShape | (static_cast<uint32_t>(kServeBlock >> 3) << 17);
            const uint64_t qd = sw128(smem_u32(sQ), 16, 1024), kd = sw128(smem_u32(sK), 16, 1024);
            int seg = 0;
            do {
                if (at.left <= 0) break;
                ok = wait_all(&qfull, static_cast<uint32_t>(seg++ & 1));
                for (int i = 0; i < at.n && ok; ++i, ++j) {
                    const int st = j % NB, sb = j % 2;
                    ok = wait_all(&kfull[st], static_cast<uint32_t>((j / NB) & 1));
                    // S_j goes where P_{j-2} was: its P V must be done
                    if (ok && j >= 2) ok = wait_all(&pvdone[sb], static_cast<uint32_t>(((j - 2) / 2) & 1));
                    if (!ok) break;
                    tc_fence_after();
                    if (leader) {
                        const uint64_t kds = kd + static_cast<uint64_t>(st * (kKV >> 4));
#pragma unroll
                        for (int k = 0; k < HD / 16; ++k)
                            umma_bf16(t_s + static_cast<uint32_t>(sb * 64),
                                      qd + static_cast<uint64_t>(((k >> 2) * kHalfQ + (k & 3) * 32) >> 4),
                                      kds + static_cast<uint64_t>(((k >> 2) * kHalfKV + (k & 3) * 32) >> 4), id_s, k > 0 ? 1u : 0u);
                        umma_commit(&sfull[sb]);
                        umma_commit(&kempty[st]);
                        if (i + 1 == at.n) umma_commit(&qempty);  // the segment's last use of Q
                    }
                    __syncwarp();
                }
            } while (ok && at.advance());
        } else {
            constexpr uint32_t id_o = kShape | (static_cast<uint32_t>(HD >> 3) << 17) | (1u << 16);  // V is MN-major
            const uint64_t vd = sw128(smem_u32(sV), kHalfKV, 1024);
            do {
                if (at.left <= 0) break;
                // of a step: first and last + 1 live lane, keys that there are, whether rows see less than those
                const int tok0 = at.tile * s.tile_tokens;
                auto live_of = [&](int step) {
                    int lo = 0, hi = kServeRows, valid = kServeBlock;
                    bool partly = false;
                    if (step < prefix_blocks) {
                        valid = min(valid, prefix_len - step * kServeBlock);
                    } else {
                        const int4 f = w.info[at.own0 + step - prefix_blocks];
                        lo = max(f.x - tok0, 0) * s.G;
                        hi = min(f.y - tok0, s.tile_tokens) * s.G;
                        valid = max(min(valid, f.w + f.y - f.x - f.z), 0);
                        partly = sees_partly<TREE>(f, valid, tok0, causal);
                    }
                    return lo | hi << 8 | valid << 16 | static_cast<int>(partly) << 24;
                };
                int cur, nxt = 0;
                if (lane < at.n) nxt = live_of(at.step + lane);
                for (int i = 0; i < at.n; ++i, ++j) {
                    if ((i & 31) == 0) {
                        cur = nxt;
                        if (i + 32 + lane < at.n) nxt = live_of(at.step + i + 32 + lane);
                    }
                    const int x = __shfl_sync(0xffffffffu, cur, i & 31);
                    const int lo = x & 255, hi = x >> 8 & 255, valid = x >> 16 & 255;
                    const uint4 off = make_uint4(~bit_run(lo, hi), ~bit_run(lo - 32, hi - 32), ~bit_run(lo - 64, hi - 64),
                                                 ~bit_run(lo - 96, hi - 96));
                    const int st = j % NB, sb = j % 2;
                    ok = wait_all(&vfull[st], static_cast<uint32_t>((j / NB) & 1));
                    if (!ok) break;
                    if (valid < kServeBlock || x >> 24) {
                        // While the softmax is at work: the values of keys that are not there become 0; so do infinities
                        // and NaN that some row must not see (its P is 0, but they would come through the MMA all
                        // the same), which the rows that see them get at the unit's end.
                        uint4* v4 = reinterpret_cast<uint4*>(sV + st * kKV);
                        if (x >> 24) {
                            uint32_t odd = 0;
                            auto bits = [](uint32_t u) { return odd_halves<T>(u); };
#pragma unroll 4
                            for (int k = lane; k < valid * 8; k += 32) {
#pragma unroll
                                for (int h = 0; h < kParts; ++h) {
                                    const uint4 y = v4[h * (kHalfKV / 16) + k];
                                    odd |= bits(y.x) | bits(y.y) | bits(y.z) | bits(y.w);
                                }
                            }
                            if (odd) {
#pragma unroll 1
                                for (int k = lane; k < valid * 8; k += 32) {
                                    for (int h = 0; h < kParts; ++h) {
                                        uint4& y = v4[h * (kHalfKV / 16) + k];
                                        y.x &= ~((bits(y.x) >> 15) * 0xffffu);
                                        y.y &= ~((bits(y.y) >> 15) * 0xffffu);
                                        y.z &= ~((bits(y.z) >> 15) * 0xffffu);
                                        y.w &= ~((bits(y.w) >> 15) * 0xffffu);
                                    }
                                }
                                *const_cast<volatile int*>(&sy.odd) = 1;
                            }
                        }
                        for (int k = valid * 8 + lane; k < kServeBlock * 8; k += 32) {
#pragma unroll
                            for (int h = 0; h < kParts; ++h) v4[h * (kHalfKV / 16) + k] = make_uint4(0, 0, 0, 0);
                        }
                        __threadfence_block();
                        fence_proxy_async_smem();
                        __syncwarp();
                    }
                    ok = wait_all(&pfull[sb], static_cast<uint32_t>((j / 2) & 1));
                    if (!ok) break;
                    tc_fence_after();
                    if (leader) {
                        const uint64_t vds = vd + static_cast<uint64_t>(st * (kKV >> 4));
#pragma unroll
                        for (int k = 0; k < kServeBlock / 16; ++k)
                            umma_tmem_a_masked(t_o, t_s + static_cast<uint32_t>(sb * 64 + k * 8),
                                               vds + static_cast<uint64_t>((k * 2048) >> 4), id_o, off);
                        umma_commit(&pvdone[sb]);
                        umma_commit(&vempty[st]);
                    }
                    __syncwarp();
                }
            } while (ok && at.advance());
        }
        // every MMA is done before the CTA gives back tensor memory and shared memory
        if (leader) {
            umma_commit(&drain[warp - 5]);
            const long long t0 = spin_clock();
            while (!mbar_try_wait(&drain[warp - 5], 0) && spin_clock() - t0 < kWaitLimitCycles) {
            }
        }
        __syncwarp();
    } else {
        // ------------------------------------------------ softmax, output
        const int r = threadIdx.x;  // row of the tile = lane of tensor memory
        const int tok_off = r / s.G, g = r - tok_off * s.G;
        const uint32_t lane_off = static_cast<uint32_t>(warp * 32) << 16;
        const uint32_t t_o = tmem + lane_off, t_s = tmem + 128 + lane_off;
        const float sl2 = a.scale * 1.4426950408889634f;
        const int full_blocks = prefix_len / kServeBlock;
        auto wait = [&](uint64_t* bar, uint32_t parity) {
            return __all_sync(0xffffffffu, mbar_wait(bar, parity, &s_abort, t.status)) != 0;
        };
        int j = 0;
        bool ok = true;
        do {
            if (at.left <= 0) break;
            const int tok = at.tile * s.tile_tokens + tok_off;
            const bool there = tok_off < s.tile_tokens && tok < rows;
            float m = -INFINITY, l = 0.0f;
            // of the request whose own keys are at hand: keys from the step's block on, its new tokens, which of them the row is
            int n_left = 0, q_rows = 0, nth = 0;
            {
                uint32_t zero[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) zero[i] = 0u;
#pragma unroll
                for (int c = 0; c < HD; c += 32) tmem_st_32u(t_o + static_cast<uint32_t>(c), zero);
            }
            for (int i = 0; i < at.n; ++i, ++j) {
                const int step = at.step + i, sb = j % 2;
                // Keys of the block that there are, and that this row sees.  A row that is not live (of another
                // request) computes on, unmasked, and keeps its m and l: its lane of O is not written.
                int valid = kServeBlock, seen = kServeBlock;
                bool live = true, masked = false, some = true, any_live = true;
                uint64_t bits = ~0ull;  // TREE: those keys
                if (step >= full_blocks) {
                    if (step < prefix_blocks) {
                        valid = seen = prefix_len - step * kServeBlock;
                    } else {
                        if (n_left <= 0) {  // (a request's blocks follow one another)
                            const int4 f = w.info[at.own0 + step - prefix_blocks];
                            q_rows = f.y - f.x;
                            nth = tok - f.x;
                            n_left = f.w + q_rows - f.z;
                        }
                        valid = min(kServeBlock, n_left);
                        live = there && static_cast<unsigned>(nth) < static_cast<unsigned>(q_rows);
                        seen = causal ? min(valid, n_left - q_rows + nth + 1) : valid;
                        if constexpr (TREE) {
                            if (live && q_rows - n_left + valid > 0)
                                bits = seen_bits(a.mask + static_cast<size_t>(tok) * a.words, a.words, q_rows - n_left);
                        }
                        n_left -= kServeBlock;
                    }
                    if constexpr (TREE) {
                        bits &= low_bits(seen);
                        seen = __popcll(bits);
                    }
                    masked = __any_sync(0xffffffffu, live && seen < kServeBlock);
                    some = __any_sync(0xffffffffu, live && seen > 0);
                    any_live = __any_sync(0xffffffffu, live);
                }
                ok = wait(&sfull[sb], static_cast<uint32_t>((j / 2) & 1));
                if (!ok) break;
                tc_fence_after();
                const uint32_t ts = t_s + static_cast<uint32_t>(sb * 64);
                if (some) {
                    float v[64];
                    tmem_ld_32x64(ts, v);
                    if (masked) {
#pragma unroll
                        for (int k = 0; k < 64; ++k)
                            if (TREE ? !((k < 32 ? static_cast<uint32_t>(bits) >> k : static_cast<uint32_t>(bits >> 32) >> (k - 32)) & 1u)
                                     : k >= seen)
                                v[k] = -INFINITY;
                    }
                    // P and its sum with the m there is; a row whose m is too small for the block, or not yet there, takes
                    // the block's maximum, and the warp makes P again
                    float sum = 0.0f;
                    auto weigh = [&] {
                        const float ref = m == -INFINITY ? 0.0f : -m;
                        const float2 sl = make_float2(sl2, sl2), nm = make_float2(ref, ref);
                        float2 ls[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            float pk[16];
#pragma unroll
                            for (int k = 0; k < 16; ++k) {
                                float2 e = fma2(make_float2(v[32 * h + 2 * k], v[32 * h + 2 * k + 1]), sl, nm);
                                e.x = ex2(e.x);
                                e.y = ex2(e.y);
                                ls[k & 1] = add2(ls[k & 1], e);
                                pk[k] = __uint_as_float(Half2<T>::pack(e.x, e.y));
                            }
                            tmem_st_32x16_async(ts + static_cast<uint32_t>(16 * h), pk);
                        }
                        sum = (ls[0].x + ls[0].y) + (ls[1].x + ls[1].y);
                    };
                    weigh();
                    const bool redo = live && (m == -INFINITY ? seen > 0 : !(sum <= kSumMax));
                    if (__any_sync(0xffffffffu, redo)) {
                        float mi[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
                        for (int k = 4; k < 64; k += 4) {
#pragma unroll
                            for (int u = 0; u < 4; ++u) mi[u] = fmaxf(mi[u], v[k + u]);
                        }
                        const float mx = fmaxf(fmaxf(mi[0], mi[1]), fmaxf(mi[2], mi[3])) * sl2;
                        const bool up = redo && mx > m;
                        if (__any_sync(0xffffffffu, up && m != -INFINITY)) {
                            ok = wait(&pvdone[(j - 1) % 2], static_cast<uint32_t>(((j - 1) / 2) & 1));
                            if (!ok) break;
                            tc_fence_after();
                            const float al = up && m != -INFINITY ? ex2(m - mx) : 1.0f;
                            float o[16];
#pragma unroll 1
                            for (int c = 0; c < HD; c += 16) {
                                tmem_ld_32x16(t_o + static_cast<uint32_t>(c), o);
#pragma unroll
                                for (int k = 0; k < 16; ++k) o[k] *= al;
                                tmem_st_32x16(t_o + static_cast<uint32_t>(c), o);
                            }
                            l *= al;
                        }
                        if (up) m = mx;
                        tmem_wait_st();  // (nothing else orders two stores to the same columns)
                        weigh();
                    }
                    if (live) l += sum;
                    tmem_wait_st();
                } else if (any_live) {
                    // rows of the block's request, all before its keys: nothing, but their lanes do take part
                    uint32_t zero[32];
#pragma unroll
                    for (int k = 0; k < 32; ++k) zero[k] = 0u;
                    tmem_st_32u(ts, zero);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&pfull[sb]);
            }
            if (!ok) break;
            // O after the segment's last P V
            ok = wait(&pvdone[(j - 1) % 2], static_cast<uint32_t>(((j - 1) / 2) & 1));
            if (!ok) break;
            tc_fence_after();
            if (__any_sync(0xffffffffu, *const_cast<volatile int*>(&sy.odd))) {
                // The infinities and NaN of blocks that are seen in part, from the cache: whatever its weight, one
                // that a row sees makes the feature what it is itself.  (sy.odd may be of another segment: then
                // nothing is found.)
                const T* vc = static_cast<const T*>(a.vc) + static_cast<long long>(at.hk) * s.page * HD;
#pragma unroll 1
                for (int c = 0; c < HD; c += 16) {
                    float o[16];
                    tmem_ld_32x16(t_o + static_cast<uint32_t>(c), o);
#pragma unroll 1
                    for (int step = max(at.step, prefix_blocks); step < at.step + at.n; ++step) {
                        const int4 f = w.info[at.own0 + step - prefix_blocks], pg = w.pages[at.own0 + step - prefix_blocks];
                        const int valid = min(kServeBlock, f.w + f.y - f.x - f.z);
                        if (!there || tok < f.x || tok >= f.y || !sees_partly<TREE>(f, valid, at.tile * s.tile_tokens, causal)) continue;
                        const int seen = causal ? min(valid, f.w + tok - f.x + 1 - f.z) : valid;
                        uint64_t bits = ~0ull;
                        if constexpr (TREE) bits = seen_bits(a.mask + static_cast<size_t>(tok) * a.words, a.words, f.z - f.w);
#pragma unroll 1
                        for (int k = 0; k < seen; ++k) {
                            if (TREE && !((bits >> k) & 1)) continue;
                            const int nth = s.page >= kServeBlock ? 0 : k >> s.page_log2;
                            const int id = nth == 0 ? pg.x : nth == 1 ? pg.y : nth == 2 ? pg.z : pg.w;
                            const int place = s.page >= kServeBlock ? pg.y + k : k & (s.page - 1);
                            if (id < 0 || id >= s.n_pages) continue;
                            const uint32_t* v = reinterpret_cast<const uint32_t*>(vc + id * s.page_stride + static_cast<long long>(place) * HD + c);
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                const uint32_t u = v[i], odd = odd_halves<T>(u);
                                const float2 x = Half2<T>::unpack(u);
                                if (odd & 0x8000u) o[2 * i] += x.x;
                                if (odd & 0x80000000u) o[2 * i + 1] += x.y;
                            }
                        }
                    }
                    __syncwarp();
                    tmem_st_32x16(t_o + static_cast<uint32_t>(c), o);
                }
            }
            const bool whole = at.whole();
            const float il = l != 0.0f ? 1.0f / l : 0.0f;
            const long long row_head = static_cast<long long>(tok) * s.H + at.hk * s.G + g;
            const size_t slot = 2 * static_cast<size_t>(cta) + (at.step == 0 ? 1 : 0);  // an end of the run: its first or last unit
            if (whole) {
                // (32 bytes a store, a sector each: the rows of a group lie head_dim values apart)
                T* op = static_cast<T*>(a.out) + row_head * HD;
#pragma unroll 1
                for (int c = 0; c < HD; c += 32) {
                    float o[32];
                    tmem_ld_32x32(t_o + static_cast<uint32_t>(c), o);
                    uint32_t x[16];
#pragma unroll
                    for (int k = 0; k < 16; ++k) x[k] = Half2<T>::pack(o[2 * k] * il, o[2 * k + 1] * il);
                    if (there) {
                        st_32b(op + c, x);
                        st_32b(op + c + 16, x + 8);
                    }
                }
                if (there && a.lse) a.lse[row_head] = (m + log2f(l)) * kLn2;
            } else {
                // [features / 4][rows][4]: a warp's store is 512 bytes in a row
                float4* pp = reinterpret_cast<float4*>(t.partials) + slot * kServeRows * (HD / 4) + r;
                if (__any_sync(0xffffffffu, l != 0.0f)) {
#pragma unroll 1
                    for (int c = 0; c < HD; c += 32) {
                        float o[32];
                        tmem_ld_32x32(t_o + static_cast<uint32_t>(c), o);
                        if (l != 0.0f) {
#pragma unroll
                            for (int k = 0; k < 8; ++k)
                                pp[(c / 4 + k) * kServeRows] = make_float4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
                        }
                    }
                }
                float2* ml = reinterpret_cast<float2*>(t.partials + static_cast<size_t>(2 * kServeCtas) * kServeRows * HD);
                ml[slot * kServeRows + r] = make_float2(m, l);
            }
            tc_fence_before();
        } while (at.advance());
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 4) tmem_dealloc(tmem, 256);
}

// Joins the parts of units that several CTAs share, in the order of their keys: blocks take a unit and 16
// features at a time, a thread a row.  A part is its CTA's first (the unit begins before its run) or its last.
// Bound by the trips to L2 that depend on one another: the unit, the rows' maxima and sums, the parts.  (Joined
// by the warp that stores the last part instead, one SM's loads in flight take longer than this launch: 96
// tokens under 8001 keys 41 -> 71 us.)
constexpr int kJoinBlocks = 6;  // of an SM
template <int HD, typename T>
__global__ void __launch_bounds__(kServeRows, kJoinBlocks) k_serve_join(const __grid_constant__ ServeShape s,
                                                                        const __grid_constant__ dllm_serve_tables t,
                                                                        const __grid_constant__ ServeAttnArgs a) {
    constexpr int kBatch = 2;  // parts whose loads are in flight together
    ServeArrays w;
    serve_arrays(s, t.work, &w);
    // (the plan was there before the launch that this one overlaps with waited for it)
    const int items = serve_same_shape(s, *w.head) ? w.head->joins * (HD / 16) : 0, rows = min(w.head->rows, a.rows);
    const int r = threadIdx.x, tok_off = r / s.G, g = r - tok_off * s.G;
    int4 d = static_cast<int>(blockIdx.x) < items ? w.join[blockIdx.x / (HD / 16)] : make_int4(0, 0, 0, 0);
    pdl_wait();
    for (int item = blockIdx.x; item < items;) {
        const int f0 = item % (HD / 16) * 16, first = d.z, last = d.w, n = d.x * s.tile_tokens + tok_off;
        const long long row_head = static_cast<long long>(n) * s.H + d.y * s.G + g;
        item += gridDim.x;
        if (item < items) d = w.join[item / (HD / 16)];
        if (tok_off >= s.tile_tokens || n >= rows) continue;
        const float2* ml = reinterpret_cast<const float2*>(t.partials + static_cast<size_t>(2 * kServeCtas) * kServeRows * HD) + r;
        const float4* pp = reinterpret_cast<const float4*>(t.partials) + static_cast<size_t>(f0 / 4) * kServeRows + r;
        auto slot = [&](int k) { return (2 * static_cast<size_t>(k) + (k == first ? 1 : 0)) * kServeRows; };
        float acc[16] = {}, M = -INFINITY, L = 0.0f;
        float2 x[kBatch];
        auto fetch = [&](int k0) {
#pragma unroll
            for (int i = 0; i < kBatch; ++i) x[i] = k0 + i <= last ? ml[slot(k0 + i)] : make_float2(-INFINITY, 0.0f);
        };
        fetch(first);
        for (int k0 = first; k0 <= last; k0 += kBatch) {
            float4 v[kBatch][4];
            float wt[kBatch], mx = M;
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    v[i][u] = x[i].y != 0.0f ? pp[slot(k0 + i) * (HD / 4) + u * kServeRows] : make_float4(0.f, 0.f, 0.f, 0.f);
                mx = fmaxf(mx, x[i].x);
            }
            const float ref = mx == -INFINITY ? 0.0f : mx, al = M == -INFINITY ? 0.0f : exp2f(M - ref);
            M = mx;
            L *= al;
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                wt[i] = x[i].y != 0.0f ? exp2f(x[i].x - ref) : 0.0f;
                L += x[i].y * wt[i];
            }
            fetch(k0 + kBatch);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                float4 o = make_float4(acc[4 * u] * al, acc[4 * u + 1] * al, acc[4 * u + 2] * al, acc[4 * u + 3] * al);
#pragma unroll
                for (int i = 0; i < kBatch; ++i) {
                    o.x += v[i][u].x * wt[i];
                    o.y += v[i][u].y * wt[i];
                    o.z += v[i][u].z * wt[i];
                    o.w += v[i][u].w * wt[i];
                }
                acc[4 * u] = o.x;
                acc[4 * u + 1] = o.y;
                acc[4 * u + 2] = o.z;
                acc[4 * u + 3] = o.w;
            }
        }
        const float il = L != 0.0f ? 1.0f / L : 0.0f;
        uint32_t o[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) o[k] = Half2<T>::pack(acc[2 * k] * il, acc[2 * k + 1] * il);
        st_32b(static_cast<T*>(a.out) + row_head * HD + f0, o);
        if (a.lse && f0 == 0) a.lse[row_head] = (M + log2f(L)) * kLn2;
    }
}

template <bool TREE, int HD, typename T>
cudaError_t go(const ServeShape& s, const dllm_serve_tables& t, const ServeAttnArgs& a, int sms, cudaStream_t st) {
    constexpr bool f16 = std::is_same<T, __half>::value;
    Maps maps;
    const uint64_t e = 2, page_rows = static_cast<uint64_t>(s.Hkv) * s.page;
    const uint64_t qdims[4] = {HD, static_cast<uint64_t>(s.G), static_cast<uint64_t>(s.Hkv), static_cast<uint64_t>(a.rows)};
    const uint64_t qstr[3] = {HD * e, s.G * HD * e, a.ldq * e};
    const uint32_t qbox[4] = {64, static_cast<uint32_t>(s.G), 1, static_cast<uint32_t>(s.tile_tokens)};
    const uint64_t kdims[3] = {HD, page_rows, static_cast<uint64_t>(s.n_pages)};
    const uint64_t kstr[2] = {HD * e, s.page_stride * e};
    const uint32_t kbox[3] = {64, static_cast<uint32_t>(s.page < kServeBlock ? s.page : kServeBlock), 1};
    if (!make_tmap_16bit(&maps.q, a.q, f16, 4, qdims, qstr, qbox) || !make_tmap_16bit(&maps.k, a.kc, f16, 3, kdims, kstr, kbox) ||
        !make_tmap_16bit(&maps.v, a.vc, f16, 3, kdims, kstr, kbox))
        return cudaErrorInvalidValue;
    // (an attribute of the function in the current device's context; a call takes about a microsecond)
    cudaError_t err = cudaFuncSetAttribute(reinterpret_cast<const void*>(k_serve_attn<HD, T, TREE>),
                                           cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem<HD>);
    if (err != cudaSuccess) return err;
    const int ctas = 2 * sms < kServeCtas ? 2 * sms : kServeCtas;
    err = serve_launch(k_serve_attn<HD, T, TREE>, dim3(ctas), kThreads, kSmem<HD>, st, maps, s, t, a);
    if (err != cudaSuccess) return err;
    return serve_launch(k_serve_join<HD, T>, dim3(kJoinBlocks * sms), kServeRows, 0, st, s, t, a);
}
template <bool TREE>
cudaError_t go_any(const ServeShape& s, const dllm_serve_tables& t, const ServeAttnArgs& a, int sms, cudaStream_t st) {
    if (s.dtype == DLLM_BF16)
        return s.hd == 128 ? go<TREE, 128, __nv_bfloat16>(s, t, a, sms, st) : go<TREE, 64, __nv_bfloat16>(s, t, a, sms, st);
    return s.hd == 128 ? go<TREE, 128, __half>(s, t, a, sms, st) : go<TREE, 64, __half>(s, t, a, sms, st);
}

}  // namespace

}  // namespace dllm
