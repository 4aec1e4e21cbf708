// Attention over a paged cache in fp32 arithmetic throughout: the path of fp32 caches.
//
// One block takes a run of key tiles of one row unit (see Plan), both products on the fp32 pipes from shared memory, the
// running maximum and sum of the softmax in registers. Two kernels:
//   many rows (RU = d): a thread holds up to d / 16 rows (1, 2, 4 or 8, as many as the unit's rows need) x 4 scores of a
//     tile of 64 tokens and as many rows x d / 16 columns of the numerator; the 16 threads of a row are half a warp, so row
//     reductions are four shuffles. Bound by what shared memory delivers (8 rows: 12 16-byte loads for 128 multiply-adds,
//     4 rows: 8 for 64), then by the fp32 pipes. K and V are copied (cp.async) as soon as the one before has been read: K
//     during P V, V during the next Q K^T. At d = 128 one block of 128 rows an SM against two of 64: 860 and 920 us (1000
//     new tokens x 32 heads behind 1000 to 1700 others, 32 TFLOP/s); at d = 64 two blocks of 64 rows are ahead, 192 and 200.
//   few rows (RU = 8): single tokens and drafts, where the cache is read once and the copies must never stop. A warp is on
//     its own with a quarter of the tile's tokens: its lanes share the tokens' scores for all rows, then each holds
//     D / 32 columns of the numerator; the next tile is copied (cp.async) meanwhile, three blocks an SM, and the warps'
//     results are joined at the end of the run.
#pragma once
#include "subgen_paged.cuh"

namespace sgk {

constexpr int kSimtLead = 1;

template <int D>
struct SimtSmem {
    static constexpr int RU = D, KT = 64, NT = 256, BLOCKS = D == 64 ? 2 : 1;
    float Q[RU][D];
    float K[KT][D + 4];                               // + 4: sixteen threads read sixteen rows at once
    float V[KT][D];
    float P[RU][KT];
    int bad, flag;
};
template <int D>
struct FewSmem {
    static constexpr int RU = 8, KT = D == 128 ? 32 : 64, NT = 128, BLOCKS = 3, SPLIT = NT / KT;    // SPLIT lanes share a token
    float Q[RU][D];
    float K[2][KT][D + 4 * SPLIT];                    // eight lanes read all 32 banks
    float V[2][KT][D];
    float P[NT / 32][KT / 4][RU];                     // [warp][token][row]
    float2 stat[NT / 32][RU];
    int bad, flag;
};

// 16 bytes, or zeros
__device__ __forceinline__ void copy16(void* to, const void* from, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from), "r"(there ? 16 : 0) : "memory");
}

// Tile t of a run into shared memory, K or V or (one loop, one look at the page) both: tokens behind the end and unusable
// pages as zeros. One group of copies.
template <int KT, int D, int NT, bool HAS_K, bool HAS_V>
__device__ __forceinline__ void bring_tile(const PagedView& P, const Seg& g, int t, float* K, int k_stride, float* V, int* bad) {
    constexpr int LPR = D / 4;
    const bool pre = t < g.kp;
    const int base = (pre ? t : t - g.kp) * KT, limit = pre ? g.e.P : g.e.S;
    const int* tab = pre ? g.e.ptab : g.e.stab;
#pragma unroll 4
    for (int p = threadIdx.x; p < KT * LPR; p += NT) {
        const int j = p / LPR, piece = p % LPR, pos = base + j;
        long long off = 0;
        bool there = pos < limit;
        if (there) {
            const int id = __ldg(tab + (pos >> P.page_shift));
            there = id >= 0 && id < P.pages;
            if (there) off = id * P.ps + g.head * P.hs + (pos & ((1 << P.page_shift) - 1)) * P.ts + piece * 4;
            else *bad = 1;
        }
        if (HAS_K) copy16(K + j * k_stride + piece * 4, (const float*)P.K + off, there);
        if (HAS_V) copy16(V + j * D + piece * 4, (const float*)P.V + off, there);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
}
template <int RU, int D, int NT>
__device__ __forceinline__ void bring_queries(const Attend& a, const Seg& g, float (*Q)[D]) {
    for (int p = threadIdx.x; p < RU * (D / 4); p += NT) {
        const int r = p / (D / 4), piece = p % (D / 4);
        float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
        if (r < g.rows) {
            const int row = g.ru * RU + r, tok = g.e.tok0 + (row >> a.g_shift), h = (g.head << a.g_shift) + (row & ((1 << a.g_shift) - 1));
            f = __ldg(reinterpret_cast<const float4*>((const float*)a.q.p + tok * a.q.ts + h * a.q.hs) + piece);
        }
        *reinterpret_cast<float4*>(&Q[r][piece * 4]) = f;
    }
}
// Where row r of a run goes: the output, or its place among the partials.
template <int RU, int D>
__device__ __forceinline__ float* result_row(const Attend& a, const Seg& g, int r) {
    if (!g.direct) return a.part + (long long)(g.slot + r) * D;
    const int row = g.ru * RU + r;
    return (float*)a.o.p + (g.e.tok0 + (row >> a.g_shift)) * a.o.ts + ((g.head << a.g_shift) + (row & ((1 << a.g_shift) - 1))) * a.o.hs;
}

// R rows of a tile by one warp (few rows): scores of its KT / 4 tokens, weights, numerator.
template <int D, int R>
__device__ __forceinline__ void few_tile(FewSmem<D>& sm, int at, int first, const int* lim, float c, float* m, float* l, float (*acc)[D / 32]) {
    typedef FewSmem<D> S;
    constexpr int SPLIT = S::SPLIT, TOK = S::KT / 4, VL = D / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, split = lane % SPLIT, tok = lane / SPLIT, j = warp * TOK + tok;
    float s[R];
#pragma unroll
    for (int r = 0; r < R; ++r) s[r] = 0.f;
#pragma unroll 4
    for (int f = 0; f < D / 4 / SPLIT; ++f) {
        const int e = (f * SPLIT + split) * 4;
        const float4 k = *reinterpret_cast<const float4*>(&sm.K[at][j][e]);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float4 q = *reinterpret_cast<const float4*>(&sm.Q[r][e]);
            s[r] = fmaf(q.x, k.x, fmaf(q.y, k.y, fmaf(q.z, k.z, fmaf(q.w, k.w, s[r]))));
        }
    }
    bool rise = false;
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
        for (int o = 1; o < SPLIT; o <<= 1) s[r] += __shfl_xor_sync(0xffffffffu, s[r], o);
        s[r] = first + j < lim[r] ? s[r] * c : -INFINITY;
        rise |= s[r] > m[r];
    }
    if (__any_sync(0xffffffffu, rise)) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float top = fmaxf(m[r], s[r]);
#pragma unroll
            for (int o = SPLIT; o < 32; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            const float al = top == -INFINITY ? 1.f : exp2f(m[r] - top);
            m[r] = top;
            l[r] *= al;
#pragma unroll
            for (int i = 0; i < VL; ++i) acc[r][i] *= al;
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const float p = s[r] == -INFINITY ? 0.f : exp2f(s[r] - m[r]);
        l[r] += p;                                                   // of this lane's tokens
        if (split == 0) sm.P[warp][tok][r] = p;
    }
    __syncwarp();
#pragma unroll 4
    for (int t = 0; t < TOK; ++t) {
        float p[R], v[VL];
#pragma unroll
        for (int r = 0; r < R; r += 4) {
            const float4 x = *reinterpret_cast<const float4*>(&sm.P[warp][t][r]);
            p[r] = x.x; p[r + 1] = x.y; p[r + 2] = x.z; p[r + 3] = x.w;
        }
        if constexpr (VL == 4) {
            const float4 x = *reinterpret_cast<const float4*>(&sm.V[at][warp * TOK + t][lane * 4]);
            v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
        } else {
            const float2 x = *reinterpret_cast<const float2*>(&sm.V[at][warp * TOK + t][lane * 2]);
            v[0] = x.x; v[1] = x.y;
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = 0; i < VL; ++i) acc[r][i] = fmaf(p[r], v[i], acc[r][i]);
    }
    __syncwarp();
}

template <int D>
__global__ void __launch_bounds__(FewSmem<D>::NT, FewSmem<D>::BLOCKS) paged_attend_few_kernel(PagedView P, Attend a) {
    typedef FewSmem<D> S;
    constexpr int RU = S::RU, KT = S::KT, NT = S::NT, NW = NT / 32, VL = D / 32;
    extern __shared__ __align__(16) unsigned char dyn[];
    S& sm = *reinterpret_cast<S*>(dyn);
    Plan<RU, KT, 0, kSimtLead> plan(P, a);
    plan.build(dyn + ((sizeof(S) + 15) & ~(size_t)15), &sm.flag, gridDim.x);
    pdl_trigger();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int x = blockIdx.x * plan.chunk;
    const int x1 = min(plan.total, x + plan.chunk);
    while (x < x1) {
        const Seg g = plan.next(x, x1, blockIdx.x);
        if (g.tile0 >= g.tile1) continue;
        __syncthreads();
        if (tid == 0) sm.bad = g.e.bad;
        __syncthreads();
        auto bring = [&](int t) {
            const int at = (t - g.tile0) & 1;
            bring_tile<KT, D, NT, true, true>(P, g, t, &sm.K[at][0][0], D + 4 * S::SPLIT, &sm.V[at][0][0], &sm.bad);
        };
        bring(g.tile0);
        bring_queries<RU, D, NT>(a, g, sm.Q);
        float m[RU], l[RU], acc[RU][VL];
        int own[RU];
#pragma unroll
        for (int r = 0; r < RU; ++r) {
            m[r] = -INFINITY;
            l[r] = 0.f;
            own[r] = plan.own_limit(g.e, g.ru * RU + r);
#pragma unroll
            for (int i = 0; i < VL; ++i) acc[r][i] = 0.f;
        }
        for (int t = g.tile0; t < g.tile1; ++t) {
            if (t + 1 < g.tile1) {
                bring(t + 1);
                asm volatile("cp.async.wait_group 1;" ::: "memory");
            } else {
                asm volatile("cp.async.wait_group 0;" ::: "memory");
            }
            __syncthreads();
            const bool pre = t < g.kp;
            int lim[RU];
#pragma unroll
            for (int r = 0; r < RU; ++r) lim[r] = pre ? g.e.P : own[r];
            const int first = (pre ? t : t - g.kp) * KT, at = (t - g.tile0) & 1;
            if (g.rows <= 4) few_tile<D, 4>(sm, at, first, lim, a.c, m, l, acc);
            else few_tile<D, 8>(sm, at, first, lim, a.c, m, l, acc);
            __syncthreads();                                         // the stage may be filled again
        }
        const bool bad = sm.bad != 0;
        if (bad && tid == 0) paged_status(P, kStPage);
        // join the four warps: their numerators where K was
        float (*join)[RU][D] = reinterpret_cast<float (*)[RU][D]>(&sm.K[0][0][0]);
        static_assert(sizeof(float) * NW * RU * D <= sizeof(sm.K), "the warps' numerators fit");
#pragma unroll
        for (int r = 0; r < RU; ++r) {
#pragma unroll
            for (int o = S::SPLIT; o < 32; o <<= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], o);
            if (lane == 0) sm.stat[warp][r] = make_float2(m[r], l[r]);
#pragma unroll
            for (int i = 0; i < VL; ++i) join[warp][r][lane * VL + i] = acc[r][i];
        }
        __syncthreads();
        for (int r = warp; r < g.rows; r += NW) {
            float M = -INFINITY, L = 0.f, z[VL];
#pragma unroll
            for (int i = 0; i < VL; ++i) z[i] = 0.f;
#pragma unroll
            for (int k = 0; k < NW; ++k) M = fmaxf(M, sm.stat[k][r].x);
#pragma unroll
            for (int k = 0; k < NW; ++k) {
                const float f = sm.stat[k][r].x == -INFINITY ? 0.f : exp2f(sm.stat[k][r].x - M);
                L = fmaf(sm.stat[k][r].y, f, L);
#pragma unroll
                for (int i = 0; i < VL; ++i) z[i] = fmaf(join[k][r][lane * VL + i], f, z[i]);
            }
            if (bad) L = NAN;
            const float f = !g.direct ? 1.f : plan.inverse(L, g.e.P, g.e, g.ru * RU + r);
            float* y = result_row<RU, D>(a, g, r) + lane * VL;
            if (!g.direct && lane == 0) a.stat[g.slot + r] = make_float2(M, L);
            if constexpr (VL == 4) *reinterpret_cast<float4*>(y) = make_float4(z[0] * f, z[1] * f, z[2] * f, z[3] * f);
            else *reinterpret_cast<float2*>(y) = make_float2(z[0] * f, z[1] * f);
        }
    }
}

// One tile against 16 * R rows (many rows); thread (tx, ty) has rows ty + 16 i, tokens tx + 16 j and columns tx * 4 + 64 b.
// K of the tile is there, V on its way; asks for K and V of the next one when these have been read.
template <int D, int R>
__device__ __forceinline__ void simt_tile(SimtSmem<D>& sm, const PagedView& P, const Seg& g, int t, const int* own, float c, float* m, float* l,
                                          float (*acc)[D / 16]) {
    typedef SimtSmem<D> S;
    constexpr int KT = S::KT, NT = S::NT, TK = KT / 16;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const bool pre = t < g.kp, more = t + 1 < g.tile1;
    const int base = (pre ? t : t - g.kp) * KT;
    float s[R][TK];
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
        for (int j = 0; j < TK; ++j) s[i][j] = 0.f;
#pragma unroll 4
    for (int e = 0; e < D; e += 4) {
        float4 kv[TK];
#pragma unroll
        for (int j = 0; j < TK; ++j) kv[j] = *reinterpret_cast<const float4*>(&sm.K[tx + 16 * j][e]);
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const float4 qv = *reinterpret_cast<const float4*>(&sm.Q[ty + 16 * i][e]);
#pragma unroll
            for (int j = 0; j < TK; ++j) s[i][j] = fmaf(qv.x, kv[j].x, fmaf(qv.y, kv[j].y, fmaf(qv.z, kv[j].z, fmaf(qv.w, kv[j].w, s[i][j]))));
        }
    }
    __syncthreads();                                                 // K has been read
    if (more) {
        bring_tile<KT, D, NT, true, false>(P, g, t + 1, &sm.K[0][0], D + 4, nullptr, &sm.bad);
        asm volatile("cp.async.wait_group 1;" ::: "memory");         // V of this tile
    } else {
        asm volatile("cp.async.wait_group 0;" ::: "memory");
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int lim = (pre ? g.e.P : own[i]) - base;
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < TK; ++j) {
            s[i][j] = tx + 16 * j < lim ? s[i][j] * c : -INFINITY;
            top = fmaxf(top, s[i][j]);
        }
#pragma unroll
        for (int off = 8; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
        const float mn = fmaxf(m[i], top), b = mn == -INFINITY ? 0.f : mn;
        const float al = exp2f(m[i] - b);
        m[i] = mn;
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < TK; ++j) {
            const float p = exp2f(s[i][j] - b);
            sum += p;
            sm.P[ty + 16 * i][tx + 16 * j] = p;
        }
        l[i] = l[i] * al + sum;                                      // this thread's share; the 16 are added at the end
#pragma unroll
        for (int j = 0; j < D / 16; ++j) acc[i][j] *= al;
    }
    __syncthreads();                                                 // V is there for all (P would need its half-warp only)
#pragma unroll 4
    for (int j = 0; j < KT; j += 4) {
        float4 p[R];
#pragma unroll
        for (int i = 0; i < R; ++i) p[i] = *reinterpret_cast<const float4*>(&sm.P[ty + 16 * i][j]);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
#pragma unroll
            for (int b = 0; b < D / 64; ++b) {
                const float4 v = *reinterpret_cast<const float4*>(&sm.V[j + q][b * 64 + tx * 4]);
#pragma unroll
                for (int i = 0; i < R; ++i) {
                    const float w = q == 0 ? p[i].x : q == 1 ? p[i].y : q == 2 ? p[i].z : p[i].w;
                    acc[i][b * 4 + 0] = fmaf(w, v.x, acc[i][b * 4 + 0]);
                    acc[i][b * 4 + 1] = fmaf(w, v.y, acc[i][b * 4 + 1]);
                    acc[i][b * 4 + 2] = fmaf(w, v.z, acc[i][b * 4 + 2]);
                    acc[i][b * 4 + 3] = fmaf(w, v.w, acc[i][b * 4 + 3]);
                }
            }
        }
    }
    __syncthreads();                                                 // V has been read
    if (more) bring_tile<KT, D, NT, false, true>(P, g, t + 1, nullptr, 0, &sm.V[0][0], &sm.bad);
}

template <int D>
__global__ void __launch_bounds__(SimtSmem<D>::NT, SimtSmem<D>::BLOCKS) paged_attend_simt_kernel(PagedView P, Attend a) {
    typedef SimtSmem<D> S;
    constexpr int RU = S::RU, KT = S::KT, NT = S::NT, RPT = RU / 16;
    static_assert(NT == 256, "16 x 16 threads");
    extern __shared__ __align__(16) unsigned char dyn[];
    S& sm = *reinterpret_cast<S*>(dyn);
    Plan<RU, KT, 0, kSimtLead> plan(P, a);
    plan.build(dyn + ((sizeof(S) + 15) & ~(size_t)15), &sm.flag, gridDim.x);
    pdl_trigger();
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    int x = blockIdx.x * plan.chunk;
    const int x1 = min(plan.total, x + plan.chunk);
    while (x < x1) {
        const Seg g = plan.next(x, x1, blockIdx.x);
        if (g.tile0 >= g.tile1) continue;
        __syncthreads();
        if (tid == 0) sm.bad = g.e.bad;
        __syncthreads();
        bring_tile<KT, D, NT, true, false>(P, g, g.tile0, &sm.K[0][0], D + 4, nullptr, &sm.bad);
        bring_tile<KT, D, NT, false, true>(P, g, g.tile0, nullptr, 0, &sm.V[0][0], &sm.bad);
        bring_queries<RU, D, NT>(a, g, sm.Q);
        float m[RPT], l[RPT], acc[RPT][D / 16];
        int own[RPT];
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
            m[i] = -INFINITY;
            l[i] = 0.f;
            own[i] = plan.own_limit(g.e, g.ru * RU + ty + 16 * i);
#pragma unroll
            for (int j = 0; j < D / 16; ++j) acc[i][j] = 0.f;
        }
        for (int t = g.tile0; t < g.tile1; ++t) {
            asm volatile("cp.async.wait_group 1;" ::: "memory");     // K of this tile
            __syncthreads();
            if (g.rows <= 16) simt_tile<D, 1>(sm, P, g, t, own, a.c, m, l, acc);
            else if (g.rows <= 32) simt_tile<D, 2>(sm, P, g, t, own, a.c, m, l, acc);
            else if (RU == 64 || g.rows <= 64) simt_tile<D, 4>(sm, P, g, t, own, a.c, m, l, acc);
            else simt_tile<D, RU / 16>(sm, P, g, t, own, a.c, m, l, acc);
        }
        const bool bad = sm.bad != 0;                                // last written before the last tile's barriers
        if (bad && tid == 0) paged_status(P, kStPage);
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
#pragma unroll
            for (int off = 8; off > 0; off >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], off);
            const int r = ty + 16 * i;
            if (bad) l[i] = NAN;
            if (r < g.rows) {
                const float f = !g.direct ? 1.f : plan.inverse(l[i], g.e.P, g.e, g.ru * RU + r);
                float* y = result_row<RU, D>(a, g, r);
                if (!g.direct && tx == 0) a.stat[g.slot + r] = make_float2(m[i], l[i]);
#pragma unroll
                for (int b = 0; b < D / 64; ++b)
                    *reinterpret_cast<float4*>(y + b * 64 + tx * 4) = make_float4(acc[i][b * 4] * f, acc[i][b * 4 + 1] * f, acc[i][b * 4 + 2] * f, acc[i][b * 4 + 3] * f);
            }
        }
    }
}

}  // namespace sgk
