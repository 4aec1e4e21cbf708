// Attention over a paged bf16 cache on the 5th-generation tensor cores.
//
// A block takes a run of key tiles (128 tokens) of one row unit (up to 256 query rows, see Plan) and is one pipeline
// of ten warps around two score buffers in tensor memory:
//   producer (warp 8)    walks the block's share of the plan, publishes the runs, and brings Q, K and V by TMA: one copy
//                        per page and 64 columns into the 128-byte-swizzled layout the MMA reads; a ring of tiles
//   issuer (warp 9)      S = Q K^T (M = 128 rows, N = 128 tokens), O += P V (P from tensor memory, V as it lies: tokens
//                        along K, columns contiguous), both tcgen05.mma bf16 -> fp32
//   softmax (warps 0-3, 4-7)  one thread per row: read S, running maximum and sum, P in bf16 over S, finally O out
// A job is one tile against 128 rows; job c uses score buffer, numerator and softmax group c & 1, and S of job c + 2 is
// issued right after P V of job c, so the tensor cores work for one group while the other exponentiates. More than 128
// rows: both halves of the unit take every tile in turn. Up to 128: the groups take alternate tiles of the same rows
// and leave two partial results, so a single sequence's tiles overlap just as well.
// The numerator is rescaled only when a row's maximum has risen by more than 2^8 over the one in use (weights up to 256
// are as exact in bf16, and the sum is fp32); S of job c comes after P V of job c - 2 in the issue order, so a group
// that has S may change its numerator.
// V rows behind the sequence's end hold whatever the page holds; 0 * NaN would spoil the sum, so the issuer's lanes
// clear them in the sequence's last tile. Scores of such tokens are masked by selection.
// Every wait is bounded: when one gives up, the block sets SUBGEN_ST_TIMEOUT, waits for its copies and MMAs (bounded),
// frees its tensor memory and returns.
#pragma once
#include <cuda.h>

#include "subgen_paged.cuh"

namespace sgk {

constexpr int kPtThreads = 320, kPtRU = 256, kPtKT = 128, kPtRing = 4;
constexpr unsigned kPtSpins = 1u << 20;

struct SegRec {
    long long slot;
    int tile0, tile1, kp, rows, head, ru, tok0, nq, S, P, direct, bad;   // tile1 < 0: no more
};

template <int D>
struct PtSmem {                                       // after a 1024-byte aligned base
    static constexpr int kTile = 128 * D * 2, kSlots = 131072 / kTile;
    unsigned char Q[2][kTile];                        // [64-column half][row][128 B swizzled]
    unsigned char KV[kSlots][kTile];                  // K, V, K, V, ...: [half][token][128 B swizzled]
    SegRec seg[kPtRing];
    unsigned long long q_full[2], q_empty[2], kv_full[kSlots], kv_empty[kSlots], s_full[2], p_full[2], o_full[2], o_empty[2],
        seg_full[kPtRing], seg_empty[kPtRing], drain;
    unsigned tmem;
    int failed, flag;
};

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(unsigned long long* b, unsigned count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(b)), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(unsigned long long* b) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(b)) : "memory");
}
__device__ __forceinline__ void bar_expect(unsigned long long* b, unsigned bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(b)), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(unsigned long long* b, unsigned parity) {
    unsigned ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}\n"
                 : "=r"(ok) : "r"(smem_u32(b)), "r"(parity) : "memory");
    return ok != 0;
}
// Bounded; false (and *failed set) when it gives up or another warp has.
__device__ __forceinline__ bool bar_wait(unsigned long long* b, unsigned parity, int* failed) {
    if (bar_try(b, parity)) return true;
    for (unsigned i = 0; i < kPtSpins; ++i) {
        if (bar_try(b, parity)) return true;
        if ((i & 15) == 15 && *reinterpret_cast<volatile int*>(failed)) return false;
    }
    *reinterpret_cast<volatile int*>(failed) = 1;
    return false;
}
__device__ __forceinline__ void tma_load_4d(void* dst, const CUtensorMap* map, int x, int y, int z, int w, unsigned long long* bar) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(smem_u32(dst)), "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void tma_load_3d(void* dst, const CUtensorMap* map, int x, int y, int z, unsigned long long* bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(smem_u32(dst)), "l"(map), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void tc_commit(unsigned long long* b) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(b)) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// shared-memory operand: rows of 128 bytes, 128-byte swizzle, 8-row groups 1024 bytes apart. lbo: bytes between 64-column
// blocks where the contiguous axis is the MMA's N (V); not used where it is K (Q, K).
__device__ __forceinline__ uint64_t tc_desc(uint32_t addr, uint32_t lbo) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(lbo >> 4) << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ void tc_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accum) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, {%5, %5, %5, %5}, p;\n\t}\n"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accum), "r"(0u) : "memory");
}
__device__ __forceinline__ void tc_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accum) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, {%5, %5, %5, %5}, p;\n\t}\n"
                 ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accum), "r"(0u) : "memory");
}
#define SGK_R8(v, i) "=r"(v[i]), "=r"(v[i + 1]), "=r"(v[i + 2]), "=r"(v[i + 3]), "=r"(v[i + 4]), "=r"(v[i + 5]), "=r"(v[i + 6]), "=r"(v[i + 7])
#define SGK_I8(v, i) "r"(v[i]), "r"(v[i + 1]), "r"(v[i + 2]), "r"(v[i + 3]), "r"(v[i + 4]), "r"(v[i + 5]), "r"(v[i + 6]), "r"(v[i + 7])
__device__ __forceinline__ void tc_ld32(uint32_t addr, uint32_t* v) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n"
                 : SGK_R8(v, 0), SGK_R8(v, 8), SGK_R8(v, 16), SGK_R8(v, 24) : "r"(addr) : "memory");
}
__device__ __forceinline__ void tc_st32(uint32_t addr, const uint32_t* v) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
                 "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};\n"
                 ::"r"(addr), SGK_I8(v, 0), SGK_I8(v, 8), SGK_I8(v, 16), SGK_I8(v, 24) : "memory");
}
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ float ex2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

template <int D>
__global__ void __launch_bounds__(kPtThreads, 1)
paged_attend_tc_kernel(PagedView P, Attend a, const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                       const __grid_constant__ CUtensorMap mv) {
    typedef PtSmem<D> Smem;
    constexpr int NS = Smem::kSlots, HALVES = D / 64;
    constexpr uint32_t kIdescS = (1u << 4) | (1u << 7) | (1u << 10) | ((128u >> 3) << 17) | ((128u >> 4) << 24);
    constexpr uint32_t kIdescO = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((128u >> 4) << 24);
    extern __shared__ unsigned char dyn_raw[];
    unsigned char* base = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(dyn_raw) + 1023) & ~(uintptr_t)1023);
    Smem& sm = *reinterpret_cast<Smem*>(base);
    typedef Plan<kPtRU, kPtKT, true> PlanT;
    PlanT plan(P, a);
    plan.build(base + ((sizeof(Smem) + 15) & ~(size_t)15), &sm.flag, gridDim.x);
    pdl_trigger();
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    long long x = (long long)blockIdx.x * plan.chunk;
    const long long x1 = min(plan.total, x + plan.chunk);
    if (x >= x1) return;

    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sm.tmem)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            bar_init(&sm.q_full[i], 1); bar_init(&sm.q_empty[i], 1);
            bar_init(&sm.s_full[i], 1); bar_init(&sm.p_full[i], 4);
            bar_init(&sm.o_full[i], 1); bar_init(&sm.o_empty[i], 4);
        }
        for (int i = 0; i < NS; ++i) { bar_init(&sm.kv_full[i], 1); bar_init(&sm.kv_empty[i], 1); }
        for (int i = 0; i < kPtRing; ++i) { bar_init(&sm.seg_full[i], 1); bar_init(&sm.seg_empty[i], 9); }
        bar_init(&sm.drain, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        sm.failed = 0;
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sm.tmem;

    if (warp == 8) {
        // ---- producer ----
        unsigned ns = 0, nq = 0, nk = 0;              // runs, query tiles and ring tiles so far
        const int pb = min(1 << P.page_shift, 128), chunks = 128 / pb;   // tokens one copy brings; copies for a half tile
        bool ok = true;
        while (ok) {
            SegRec r;
            const int* ptab = nullptr;
            const int* stab = nullptr;
            r.tile1 = -1;
            while (x < x1) {
                const Seg g = plan.next(x, x1, blockIdx.x);
                if (g.tile0 >= g.tile1) continue;
                r = SegRec{g.slot, g.tile0, g.tile1, g.kp, g.rows, g.head, g.ru, g.e.tok0, g.e.nq, g.e.S, g.e.P, g.direct, g.e.bad};
                ptab = g.e.ptab;
                stab = g.e.stab;
                break;
            }
            const int slot = ns % kPtRing;
            if (ns >= kPtRing && !(ok = bar_wait(&sm.seg_empty[slot], (ns / kPtRing - 1) & 1, &sm.failed))) break;
            if (lane == 0) {
                sm.seg[slot] = r;
                bar_arrive(&sm.seg_full[slot]);
            }
            ++ns;
            if (r.tile1 < 0) break;
            const int sub = r.rows > 128 ? 2 : 1;
            for (int i = 0; i < sub && ok; ++i, ++nq) {
                const int qs = nq & 1;
                if (nq >= 2 && !(ok = bar_wait(&sm.q_empty[qs], (nq / 2 - 1) & 1, &sm.failed))) break;
                if (lane == 0) {
                    bar_expect(&sm.q_full[qs], Smem::kTile);
                    for (int h = 0; h < HALVES; ++h)
                        tma_load_3d(sm.Q[qs] + h * 16384, &mq, h * 64, r.head * a.G, r.tok0 + (r.ru * kPtRU + i * 128) / a.G, &sm.q_full[qs]);
                }
            }
            for (int t = r.tile0; t < r.tile1 && ok; ++t) {
                const bool pre = t < r.kp;
                const int first = (pre ? t : t - r.kp) * kPtKT, limit = pre ? r.P : r.S;
                // lane: chunk = lane / HALVES, half = lane % HALVES
                const int chunk = lane / HALVES, half = lane % HALVES, pos = first + chunk * pb;
                bool mine = chunk < chunks && pos < limit;
                int id = 0;
                if (mine) {
                    id = __ldg((pre ? ptab : stab) + (pos >> P.page_shift));
                    if (id < 0 || id >= P.pages) { mine = false; id = -1; }
                }
                if (__any_sync(0xffffffffu, id < 0) && lane == 0) {
                    *reinterpret_cast<volatile int*>(&sm.seg[slot].bad) = 1;
                    paged_status(P, kStPage);
                }
                const unsigned bytes = __popc(__ballot_sync(0xffffffffu, mine)) * (unsigned)pb * 128u;
                for (int kv = 0; kv < 2; ++kv, ++nk) {
                    const int s = nk % NS;
                    if (nk >= NS && !(ok = bar_wait(&sm.kv_empty[s], (nk / NS - 1) & 1, &sm.failed))) break;
                    if (lane == 0) bar_expect(&sm.kv_full[s], bytes);
                    __syncwarp();
                    if (mine)
                        tma_load_4d(sm.KV[s] + half * 16384 + chunk * pb * 128, kv ? &mv : &mk, half * 64, pos & ((1 << P.page_shift) - 1),
                                    r.head, id, &sm.kv_full[s]);
                }
            }
        }
        // copies in flight write shared memory: they have to be done before the block ends
        for (unsigned i = nk > (unsigned)NS ? nk - NS : 0; i < nk; ++i)
            for (unsigned j = 0; j < kPtSpins && !bar_try(&sm.kv_full[i % NS], (i / NS) & 1); ++j) {}
        for (unsigned i = nq > 2 ? nq - 2 : 0; i < nq; ++i)
            for (unsigned j = 0; j < kPtSpins && !bar_try(&sm.q_full[i & 1], (i / 2) & 1); ++j) {}
    } else if (warp == 9) {
        // ---- issuer ----
        struct Cursor { int tile, tile0, tile1, kp, dual, sub, P, S; unsigned seg, q, kv; bool done; };
        auto enter = [&](Cursor& c) {                  // the run that c.seg counts to
            const int slot = c.seg % kPtRing;
            if (!bar_wait(&sm.seg_full[slot], (c.seg / kPtRing) & 1, &sm.failed)) { c.done = true; return; }
            const SegRec& r = sm.seg[slot];
            c.tile = c.tile0 = r.tile0; c.tile1 = r.tile1; c.kp = r.kp; c.dual = r.rows > 128; c.sub = 0; c.P = r.P; c.S = r.S;
            c.done = r.tile1 < 0;
        };
        Cursor qk = {0, 0, 0, 0, 0, 0, 0, 0, 0u, 0u, 0u, false}, pv = qk;
        unsigned jobs_qk = 0, jobs_pv = 0, segs[2] = {0u, 0u};        // segs: runs whose numerator each group has begun
        bool ok = true;
        auto issue_qk = [&]() {
            if (qk.done || !ok) return;
            const unsigned w = jobs_qk & 1, qt = qk.q + qk.sub, ks = 2 * qk.kv, s = ks % NS;
            if (qk.tile == qk.tile0 && !(ok = bar_wait(&sm.q_full[qt & 1], (qt / 2) & 1, &sm.failed))) return;
            if (!(ok = bar_wait(&sm.kv_full[s], (ks / NS) & 1, &sm.failed))) return;
            const bool last_sub = qk.sub == qk.dual;
            if (lane == 0) {
                tc_fence_after();
                const uint32_t qa = smem_u32(sm.Q[qt & 1]), ka = smem_u32(sm.KV[s]);
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {
                    const uint32_t off = (uint32_t)((i >> 2) * 16384 + (i & 3) * 32);
                    tc_mma_ss(tmem + w * 128u, tc_desc(qa + off, 16), tc_desc(ka + off, 16), kIdescS, i ? 1u : 0u);
                }
                tc_commit(&sm.s_full[w]);
                if (last_sub) tc_commit(&sm.kv_empty[s]);
                if (qk.tile == qk.tile1 - 1) tc_commit(&sm.q_empty[qt & 1]);
            }
            __syncwarp();
            ++jobs_qk;
            if (!last_sub) { qk.sub = 1; return; }
            qk.sub = 0;
            ++qk.kv;
            if (++qk.tile == qk.tile1) {
                qk.q += 1 + qk.dual;
                ++qk.seg;
                enter(qk);
            }
        };
        enter(qk);
        enter(pv);
        issue_qk();
        issue_qk();
        while (!pv.done && ok) {
            const unsigned w = jobs_pv & 1, vs = 2 * pv.kv + 1, s = vs % NS;
            const int i = pv.tile - pv.tile0;
            const bool fresh = pv.dual ? i == 0 : i < 2, last_sub = pv.sub == pv.dual;
            const bool final = pv.dual ? pv.tile == pv.tile1 - 1 : pv.tile >= pv.tile1 - 2;
            if (!(ok = bar_wait(&sm.kv_full[s], (vs / NS) & 1, &sm.failed))) break;
            if (pv.sub == 0) {
                const bool pre = pv.tile < pv.kp;
                const int nv = pre ? pv.P - pv.tile * kPtKT : pv.S - (pv.tile - pv.kp) * kPtKT;
                if (nv < kPtKT) {                      // the sequence ends in this tile: clear what lies behind
                    for (int p = lane; p < (kPtKT - nv) * 8 * HALVES; p += 32) {
                        const int row = nv + p / (8 * HALVES), c = p % (8 * HALVES);
                        *reinterpret_cast<uint4*>(sm.KV[s] + (c >> 3) * 16384 + row * 128 + (c & 7) * 16) = make_uint4(0, 0, 0, 0);
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                }
            }
            if (!(ok = bar_wait(&sm.p_full[w], (jobs_pv / 2) & 1, &sm.failed))) break;
            if (fresh) {
                if (segs[w] && !(ok = bar_wait(&sm.o_empty[w], (segs[w] - 1) & 1, &sm.failed))) break;
                ++segs[w];
            }
            if (lane == 0) {
                tc_fence_after();
                const uint32_t va = smem_u32(sm.KV[s]);
#pragma unroll
                for (int k = 0; k < kPtKT / 16; ++k)
                    tc_mma_ts(tmem + 256u + w * (uint32_t)D, tmem + w * 128u + k * 8u, tc_desc(va + k * 2048u, 16384), kIdescO, fresh && !k ? 0u : 1u);
                if (last_sub) tc_commit(&sm.kv_empty[s]);
                if (final) tc_commit(&sm.o_full[w]);
            }
            __syncwarp();
            ++jobs_pv;
            if (!last_sub) pv.sub = 1;
            else {
                pv.sub = 0;
                ++pv.kv;
                if (++pv.tile == pv.tile1) {
                    if (lane == 0) bar_arrive(&sm.seg_empty[pv.seg % kPtRing]);
                    ++pv.seg;
                    enter(pv);
                }
            }
            issue_qk();
        }
        if (lane == 0) tc_commit(&sm.drain);          // the MMAs read shared memory: done before the block ends
        for (unsigned j = 0; j < kPtSpins && !bar_try(&sm.drain, 0); ++j) {}
    } else {
        // ---- softmax ----
        const int w = warp >> 2, row128 = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tS = tmem + lanes + (uint32_t)w * 128u, tO = tmem + lanes + 256u + (uint32_t)(w * D);
        unsigned ns = 0, job = 0, mine = 0, segs = 0;  // runs, jobs of both groups, jobs and runs of this one
        bool ok = true;
        while (ok) {
            const int slot = ns % kPtRing;
            if (!(ok = bar_wait(&sm.seg_full[slot], (ns / kPtRing) & 1, &sm.failed))) break;
            const SegRec& r = sm.seg[slot];
            const int tile0 = r.tile0, tile1 = r.tile1, kp = r.kp, rows = r.rows;
            if (tile1 < 0) break;
            const int dual = rows > 128, tiles = tile1 - tile0, order = (w - (int)job) & 1;   // order: this group's half, or turn
            const int row = dual ? order * 128 + row128 : row128;
            const bool live = row < rows, some = (row & ~31) < rows;
            const int urow = r.ru * kPtRU + row;
            Entry e;
            e.S = r.S; e.nq = r.nq;
            const int own = plan.own_limit(e, urow);
            float m = -INFINITY, l = 0.f;              // m: the maximum in use
            bool begun = false;
            for (int t = tile0 + (dual ? 0 : order); t < tile1; t += 2 - dual) {
                if (!(ok = bar_wait(&sm.s_full[w], mine & 1, &sm.failed))) break;
                if (some) {
                    tc_fence_after();
                    uint32_t raw[128];
                    float s[128];
#pragma unroll
                    for (int i = 0; i < 4; ++i) tc_ld32(tS + i * 32, raw + i * 32);
                    tc_wait_ld();
#pragma unroll
                    for (int i = 0; i < 128; ++i) s[i] = __uint_as_float(raw[i]);
                    const bool pre = t < kp;
                    const int lim = pre ? r.P - t * kPtKT : own - (t - kp) * kPtKT;
                    if (__any_sync(0xffffffffu, lim < kPtKT)) {
#pragma unroll
                        for (int i = 0; i < 128; ++i) s[i] = i < lim ? s[i] : -INFINITY;
                    }
                    float m0 = s[0], m1 = s[1], m2 = s[2], m3 = s[3];
#pragma unroll
                    for (int i = 4; i < 128; i += 4) {
                        m0 = fmaxf(m0, s[i]); m1 = fmaxf(m1, s[i + 1]); m2 = fmaxf(m2, s[i + 2]); m3 = fmaxf(m3, s[i + 3]);
                    }
                    const float top = fmaxf(m, fmaxf(fmaxf(m0, m1), fmaxf(m2, m3)));
                    const bool rise = (top - m) * a.c > 8.f || (m == -INFINITY && top > m);
                    if (__any_sync(0xffffffffu, rise)) {
                        const float f = rise ? ex2_approx((m - top) * a.c) : 1.f;      // 0 when there was no maximum yet
                        if (rise) m = top;
                        l *= f;
                        if (begun) {
                            uint32_t o[32];
#pragma unroll
                            for (int i = 0; i < D / 32; ++i) {
                                tc_ld32(tO + i * 32, o);
                                tc_wait_ld();
#pragma unroll
                                for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
                                tc_st32(tO + i * 32, o);
                            }
                            tc_wait_st();
                        }
                    }
                    const float off = m == -INFINITY ? 0.f : -m * a.c;
                    float l0 = 0.f, l1 = 0.f, l2 = 0.f, l3 = 0.f;
                    uint32_t p[64];
#pragma unroll
                    for (int i = 0; i < 128; i += 4) {
                        const float p0 = ex2_approx(fmaf(s[i], a.c, off)), p1 = ex2_approx(fmaf(s[i + 1], a.c, off));
                        const float p2 = ex2_approx(fmaf(s[i + 2], a.c, off)), p3 = ex2_approx(fmaf(s[i + 3], a.c, off));
                        l0 += p0; l1 += p1; l2 += p2; l3 += p3;
                        const __nv_bfloat162 a0 = __floats2bfloat162_rn(p0, p1), a1 = __floats2bfloat162_rn(p2, p3);
                        p[i / 2] = *reinterpret_cast<const uint32_t*>(&a0);
                        p[i / 2 + 1] = *reinterpret_cast<const uint32_t*>(&a1);
                    }
                    l += (l0 + l1) + (l2 + l3);
                    tc_st32(tS, p);
                    tc_st32(tS + 32, p + 32);
                    tc_wait_st();
                    tc_fence_before();
                }
                begun = true;
                __syncwarp();
                if (lane == 0) bar_arrive(&sm.p_full[w]);
                ++mine;
            }
            if (!ok) break;
            job += dual ? 2 * tiles : tiles;
            ++ns;
            if (begun) {
                if (!(ok = bar_wait(&sm.o_full[w], segs & 1, &sm.failed))) break;
                ++segs;
                if (some) {
                    tc_fence_after();
                    if (*reinterpret_cast<const volatile int*>(&r.bad)) l = NAN;
                    const int G = a.G, tok = r.tok0 + urow / G, head = r.head * G + urow % G;
                    const long long at = r.slot + (dual || order == 0 ? row : rows + row);
                    const bool direct = r.direct;
                    const float f = direct ? (l == 0.f ? 0.f : 1.f / l) : 1.f;
                    uint32_t o[32];
                    __nv_bfloat16* y = (__nv_bfloat16*)a.o.p + tok * a.o.ts + head * a.o.hs;
                    if (live && !direct) a.stat[at] = make_float2(m * a.c, l);
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) {
                        __syncwarp();
                        tc_ld32(tO + i * 32, o);
                        tc_wait_ld();
                        if (live && direct) {
#pragma unroll
                            for (int j = 0; j < 32; j += 8) {
                                uint4 v;
                                uint32_t* vv = &v.x;
#pragma unroll
                                for (int k = 0; k < 4; ++k) {
                                    const __nv_bfloat162 b = __floats2bfloat162_rn(__uint_as_float(o[j + 2 * k]) * f, __uint_as_float(o[j + 2 * k + 1]) * f);
                                    vv[k] = *reinterpret_cast<const uint32_t*>(&b);
                                }
                                *reinterpret_cast<uint4*>(y + i * 32 + j) = v;
                            }
                        } else if (live) {
                            uint4* z = reinterpret_cast<uint4*>(a.part + at * D + i * 32);
#pragma unroll
                            for (int j = 0; j < 8; ++j) z[j] = make_uint4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
                        }
                    }
                    __syncwarp();
                    tc_fence_before();
                }
                __syncwarp();
                if (lane == 0) bar_arrive(&sm.o_empty[w]);
            }
            if (lane == 0) bar_arrive(&sm.seg_empty[slot]);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 9) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
    if (tid == 0 && sm.failed) paged_status(P, kStTimeout);
}

}  // namespace sgk
