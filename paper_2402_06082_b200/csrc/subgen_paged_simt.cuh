// Attention over a paged cache in fp32 arithmetic throughout: the path of fp32 caches.
//
// One block takes a run of key tiles of one row unit (see Plan): RU query rows against KT tokens at a time, both products
// on the fp32 pipes from shared memory, the running maximum and sum of the softmax in registers. A thread holds RPT rows x
// KT / 16 scores of a tile and RPT rows x D / 16 columns of the numerator; the 16 threads of a row are half a warp, so row
// reductions are four shuffles.
// Two sizes. RU = 16 for single tokens and drafts, where the cache is read once and 16 rows of arithmetic per byte stay
// below what the memory takes: what counts is latency, so the next tile is copied (cp.async) while this one is worked on,
// in blocks small enough for three an SM. RU = 64 for many rows, where each value read from shared memory serves four rows
// and two blocks an SM cover for each other's copies.
#pragma once
#include "subgen_paged.cuh"

namespace sgk {

constexpr int kSimtLead = 1;

template <int D, int RU> struct SimtShape {
    static constexpr int KT = RU == 16 && D == 128 ? 32 : 64, STAGES = RU == 16 ? 2 : 1, NT = RU == 16 ? 128 : 256, BLOCKS = RU == 16 ? 3 : 2;
};
template <int D, int RU>
struct SimtSmem {
    typedef SimtShape<D, RU> S;
    float Q[RU][D];
    float K[S::STAGES][S::KT][D + 4];                 // + 4: sixteen threads read sixteen rows at once
    float V[S::STAGES][S::KT][D];
    float P[RU][S::KT];
    int bad, flag;
};

// 16 bytes, or zeros
__device__ __forceinline__ void copy16(void* to, const void* from, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from), "r"(there ? 16 : 0) : "memory");
}

template <int D, int RU>
__global__ void __launch_bounds__(SimtShape<D, RU>::NT) paged_attend_simt_kernel(PagedView P, Attend a) {
    typedef SimtShape<D, RU> S;
    constexpr int KT = S::KT, NT = S::NT, TK = KT / 16, TY = NT / 16, RPT = RU / TY, LPR = D / 4;
    static_assert(RPT * TY == RU, "rows divide");
    extern __shared__ __align__(16) unsigned char dyn[];
    SimtSmem<D, RU>& sm = *reinterpret_cast<SimtSmem<D, RU>*>(dyn);
    Plan<RU, KT, false, kSimtLead> plan(P, a);
    plan.build(dyn + ((sizeof(SimtSmem<D, RU>) + 15) & ~(size_t)15), &sm.flag, gridDim.x);
    pdl_trigger();
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    int x = blockIdx.x * plan.chunk;
    const int x1 = min(plan.total, x + plan.chunk);
    while (x < x1) {
        const Seg g = plan.next(x, x1, blockIdx.x);
        if (g.tile0 >= g.tile1) continue;
        const int row0 = g.ru * RU;
        __syncthreads();
        if (tid == 0) sm.bad = g.e.bad;
        __syncthreads();
        // tile t into a stage; tokens behind the end and unusable pages as zeros
        auto bring = [&](int t, int stage) {
            const bool pre = t < g.kp;
            const int base = (pre ? t : t - g.kp) * KT, limit = pre ? g.e.P : g.e.S;
            const int* tab = pre ? g.e.ptab : g.e.stab;
            for (int p = tid; p < KT * LPR; p += NT) {
                const int j = p / LPR, piece = p % LPR, pos = base + j;
                long long off = 0;
                bool there = pos < limit;
                if (there) {
                    const int id = __ldg(tab + (pos >> P.page_shift));
                    there = id >= 0 && id < P.pages;
                    if (there) off = id * P.ps + g.head * P.hs + (pos & ((1 << P.page_shift) - 1)) * P.ts + piece * 4;
                    else sm.bad = 1;
                }
                copy16(&sm.K[stage][j][piece * 4], (const float*)P.K + off, there);
                copy16(&sm.V[stage][j][piece * 4], (const float*)P.V + off, there);
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        bring(g.tile0, 0);
        for (int p = tid; p < RU * LPR; p += NT) {
            const int r = p / LPR, piece = p % LPR;
            float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
            if (r < g.rows) {
                const int row = row0 + r, tok = g.e.tok0 + (row >> a.g_shift), h = (g.head << a.g_shift) + (row & ((1 << a.g_shift) - 1));
                f = __ldg(reinterpret_cast<const float4*>((const float*)a.q.p + tok * a.q.ts + h * a.q.hs) + piece);
            }
            *reinterpret_cast<float4*>(&sm.Q[r][piece * 4]) = f;
        }
        float m[RPT], l[RPT], acc[RPT][D / 16];
        int own[RPT];
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
            m[i] = -INFINITY;
            l[i] = 0.f;
            own[i] = plan.own_limit(g.e, row0 + ty * RPT + i);
#pragma unroll
            for (int j = 0; j < D / 16; ++j) acc[i][j] = 0.f;
        }
        for (int t = g.tile0; t < g.tile1; ++t) {
            const bool pre = t < g.kp;
            const int base = (pre ? t : t - g.kp) * KT, limit = pre ? g.e.P : g.e.S, at = (t - g.tile0) % S::STAGES;
            if (S::STAGES > 1 && t + 1 < g.tile1) {
                bring(t + 1, (t + 1 - g.tile0) % S::STAGES);
                asm volatile("cp.async.wait_group 1;" ::: "memory");
            } else {
                if (S::STAGES == 1 && t > g.tile0) bring(t, 0);
                asm volatile("cp.async.wait_group 0;" ::: "memory");
            }
            __syncthreads();
            float s[RPT][TK];
#pragma unroll
            for (int i = 0; i < RPT; ++i)
#pragma unroll
                for (int j = 0; j < TK; ++j) s[i][j] = 0.f;
#pragma unroll 4
            for (int e = 0; e < D; e += 4) {
                float4 kv[TK];
#pragma unroll
                for (int j = 0; j < TK; ++j) kv[j] = *reinterpret_cast<const float4*>(&sm.K[at][tx + 16 * j][e]);
#pragma unroll
                for (int i = 0; i < RPT; ++i) {
                    const float4 qv = *reinterpret_cast<const float4*>(&sm.Q[ty * RPT + i][e]);
#pragma unroll
                    for (int j = 0; j < TK; ++j)
                        s[i][j] = fmaf(qv.x, kv[j].x, fmaf(qv.y, kv[j].y, fmaf(qv.z, kv[j].z, fmaf(qv.w, kv[j].w, s[i][j]))));
                }
            }
#pragma unroll
            for (int i = 0; i < RPT; ++i) {
                const int lim = (pre ? limit : own[i]) - base;
                float top = -INFINITY;
#pragma unroll
                for (int j = 0; j < TK; ++j) {
                    s[i][j] = tx + 16 * j < lim ? s[i][j] * a.c : -INFINITY;
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
                    sm.P[ty * RPT + i][tx + 16 * j] = p;
                }
                l[i] = l[i] * al + sum;                              // this thread's share; the 16 are added at the end
#pragma unroll
                for (int j = 0; j < D / 16; ++j) acc[i][j] *= al;
            }
            __syncwarp();                                            // a row's scores come from and go to one half-warp
#pragma unroll 4
            for (int j = 0; j < KT; j += 4) {
                float4 p[RPT];
#pragma unroll
                for (int i = 0; i < RPT; ++i) p[i] = *reinterpret_cast<const float4*>(&sm.P[ty * RPT + i][j]);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
#pragma unroll
                    for (int b = 0; b < D / 64; ++b) {
                        const float4 v = *reinterpret_cast<const float4*>(&sm.V[at][j + q][b * 64 + tx * 4]);
#pragma unroll
                        for (int i = 0; i < RPT; ++i) {
                            const float w = q == 0 ? p[i].x : q == 1 ? p[i].y : q == 2 ? p[i].z : p[i].w;
                            acc[i][b * 4 + 0] = fmaf(w, v.x, acc[i][b * 4 + 0]);
                            acc[i][b * 4 + 1] = fmaf(w, v.y, acc[i][b * 4 + 1]);
                            acc[i][b * 4 + 2] = fmaf(w, v.z, acc[i][b * 4 + 2]);
                            acc[i][b * 4 + 3] = fmaf(w, v.w, acc[i][b * 4 + 3]);
                        }
                    }
                }
            }
            __syncthreads();                                         // the stage may be filled again
        }
        const bool bad = sm.bad != 0;
        if (bad && tid == 0) paged_status(P, kStPage);
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
#pragma unroll
            for (int off = 8; off > 0; off >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], off);
            const int r = ty * RPT + i;
            if (bad) l[i] = NAN;
            if (r < g.rows) {
                const int row = row0 + r;
                const float f = !g.direct ? 1.f : l[i] == 0.f ? 0.f : 1.f / l[i];
                float* y = g.direct ? (float*)a.o.p + (g.e.tok0 + (row >> a.g_shift)) * a.o.ts + ((g.head << a.g_shift) + (row & ((1 << a.g_shift) - 1))) * a.o.hs
                                    : a.part + (long long)(g.slot + r) * D;
                if (!g.direct && tx == 0) a.stat[g.slot + r] = make_float2(m[i], l[i]);
#pragma unroll
                for (int b = 0; b < D / 64; ++b)
                    *reinterpret_cast<float4*>(y + b * 64 + tx * 4) = make_float4(acc[i][b * 4] * f, acc[i][b * 4 + 1] * f, acc[i][b * 4 + 2] * f, acc[i][b * 4 + 3] * f);
            }
        }
    }
}

}  // namespace sgk
