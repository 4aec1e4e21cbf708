// Attention over a paged bf16 cache on the 5th-generation tensor cores.
//
// A block takes a run of key tiles (128 tokens) of one row unit (up to 256 query rows, see Plan) and is one pipeline
// of warps around two score buffers in tensor memory:
//   planner (warp 11)    walks the block's share of the plan and publishes its runs
//   producer (warp 8)    brings Q, K and V by TMA: one copy per page (K: and 64 columns) into the 128-byte-swizzled
//                        layouts the MMA reads; a ring of tiles
//   issuers (warps 9-10) S = Q K^T (M = 128 rows, N = 128 tokens), O += P V (P from tensor memory, V as it lies: tokens
//                        along K, columns contiguous), both tcgen05.mma bf16 -> fp32
//   softmax (warps 0-3, 4-7)  one thread per row: read S, running maximum and sum, P in bf16 over S, finally O out
// A job is one tile against 128 rows; job c uses score buffer, numerator and softmax group c & 1, and S of job c + 2 is
// issued right after P V of job c, so the tensor cores work for one group while the other exponentiates. More than 128
// rows: both halves of the unit take every tile in turn. Up to 128: the groups take alternate tiles of the same rows
// and leave two partial results, so a single sequence's tiles overlap just as well. Up to 32 rows (single tokens, drafts):
// Q lies in shared memory four times, so that every warp of a group has all rows in its lanes of tensor memory and
// takes a quarter of the tile's tokens (the other quarters of its P are zero); the four numerators are added through
// shared memory at the end of the run. The chain score -> weight -> product is then a quarter as long.
// HAND: the second group hands the rows of such a unit over to the first, warp to warp, so that a run leaves one result,
// and a whole sequence nothing for the merge.
// The numerator is rescaled only when a row's maximum has risen by more than 2^8 over the one in use (weights up to 256
// are as exact in bf16, and the sum is fp32); S of job c comes after P V of job c - 2 in the issue order, so a group
// that has S may change its numerator.
// V rows behind the sequence's end hold whatever the page holds; 0 * NaN would spoil the sum, so the issuer's lanes
// clear them in the sequence's last tile. Scores of such tokens are masked by selection.
// Every wait is bounded: when one gives up, the block sets SUBGEN_ST_TIMEOUT, waits for its copies and MMAs (bounded),
// frees its tensor memory and returns.
#pragma once
#include <cuda.h>

#include <type_traits>

#include "subgen_paged.cuh"

namespace sgk {

constexpr int kPtThreads = 384, kPtRU = 256, kPtKT = 128, kPtRing = 8, kPtLead = 2;
constexpr int kPtPoly = 2;                            // of 8 pairs of weights, those exponentiated on the fp32 pipe
constexpr unsigned kPtSpins = 1u << 20;

struct SegRec {
    const int *ptab, *stab;
    int slot, tile0, tile1, kp, rows, head, ru, tok0, nq, S, P, direct, bad;   // tile1 < 0: no more
};

template <int D>
struct PtSmem {                                       // after a 1024-byte aligned base
    static constexpr int kTile = 128 * D * 2, kSlots = 131072 / kTile;
    unsigned char Q[2][kTile];                        // [64-column half][row][128 B swizzled]
    unsigned char KV[kSlots][kTile];                  // K, V, K, V, ...; K: [half][token][128 B swizzled], V: also by pages
    float join[2][4][4][D];                           // [group][warp][row][column]: numerators of four rows to be added
    float2 join_stat[2][4][32];                       // maximum in use, sum
    float hand[4][2][D];                              // [warp][which][column]: a row's numerator from the second group to the first
    float2 hand_stat[4][2];
    SegRec seg[kPtRing];
    unsigned long long q_full[2], q_empty[2], kv_full[kSlots], kv_empty[kSlots], s_full[2], p_full[2], o_full[2], o_empty[2], join_bar[2], hand_full[4][2], hand_empty[4][2],
        seg_full[kPtRing], seg_empty[kPtRing], drain;
    unsigned tmem;
    int failed, flag, turns[2];                       // turns: tiles shared by both groups that a group's issuer has done with
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
__device__ __forceinline__ bool bar_test(unsigned long long* b, unsigned parity) {       // does not wait
    unsigned ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}\n"
                 : "=r"(ok) : "r"(smem_u32(b)), "r"(parity) : "memory");
    return ok != 0;
}
// By a whole warp, with one answer for all lanes. Bounded; false (and *failed set) when it gives up or another warp has.
__device__ __forceinline__ bool bar_wait(unsigned long long* b, unsigned parity, int* failed) {
    bool done = bar_try(b, parity);
    for (unsigned i = 0; i < kPtSpins && !done; ++i) {
        done = bar_try(b, parity);
        if ((i & 15) == 15 && *reinterpret_cast<volatile int*>(failed)) break;
    }
    if (__all_sync(0xffffffffu, done)) return true;
    *reinterpret_cast<volatile int*>(failed) = 1;
    return false;
}
// Waits until *count, which only grows, is `target` or more; as bar_wait. A count, not a barrier: one group's issuer may be two
// turns ahead of the other's wait (the last of one run and the first of the next), and a barrier's parity would then stand for
// a turn that never comes.
__device__ __forceinline__ bool count_wait(const int* count, int target, int* failed) {
    bool done = *reinterpret_cast<const volatile int*>(count) >= target;
    for (unsigned i = 0; i < 8 * kPtSpins && !done; ++i) {
        done = *reinterpret_cast<const volatile int*>(count) >= target;
        if ((i & 255) == 255 && *reinterpret_cast<volatile int*>(failed)) break;
    }
    if (__all_sync(0xffffffffu, done)) return true;
    *reinterpret_cast<volatile int*>(failed) = 1;
    return false;
}
__device__ __forceinline__ void tma_load_4d(void* dst, const CUtensorMap* map, int x, int y, int z, int w, unsigned long long* bar) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(smem_u32(dst)), "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void tma_load_5d(void* dst, const CUtensorMap* map, int x, int y, int z, int w, int v, unsigned long long* bar) {
    asm volatile("cp.async.bulk.tensor.5d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
                 ::"r"(smem_u32(dst)), "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(v), "r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void tma_load_3d(void* dst, const CUtensorMap* map, int x, int y, int z, unsigned long long* bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(smem_u32(dst)), "l"(map), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// Issued by a whole warp in step; one lane is elected inside. The election sits in the assembly, as a predicate, because an
// MMA's operands have to be in uniform registers: behind a branch on the election the compiler takes them for divergent
// and each MMA costs some 90 cycles to issue instead of 64 (128 x 128 x 16).
__device__ __forceinline__ void tc_commit(unsigned long long* b) {
    asm volatile("{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
                 "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}\n" ::"r"(smem_u32(b)) : "memory");
}
// Shared-memory operands: rows of 128 bytes, 128-byte swizzle, 8-row groups 1024 bytes apart. The descriptor's low word is
// address >> 4 | distance of 64-column blocks >> 4 << 16 (used where the contiguous axis is the MMA's N: V).
constexpr uint32_t kDescHigh = 64u | (1u << 14) | (2u << 29);
#define SGK_MMA_S(off, p) "add.u32 al, %1, " #off ";\n\tadd.u32 bl, %2, " #off ";\n\tmov.b64 a, {al, %4};\n\tmov.b64 b, {bl, %4};\n\t" \
                          "@e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, " #p ";\n\t"
#define SGK_MMA_O(i, off, p) "add.u32 al, %1, " #i ";\n\t" off "mov.b64 b, {bl, %4};\n\t" \
                             "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [al], b, %3, " #p ";\n\t"
// S = Q K^T over d in steps of 16: 32 bytes of a row, the second 64 columns 16 KB behind
template <int D>
__device__ __forceinline__ void tc_scores(uint32_t d, uint32_t q, uint32_t k, uint32_t idesc) {
    asm volatile("{\n\t.reg .pred e, z, o;\n\t.reg .b64 a, b;\n\t.reg .b32 al, bl;\n\t"
                 "elect.sync _|e, 0xffffffff;\n\tsetp.ne.b32 z, 0, 0;\n\tsetp.eq.b32 o, 0, 0;\n\t"
                 SGK_MMA_S(0, z) SGK_MMA_S(2, o) SGK_MMA_S(4, o) SGK_MMA_S(6, o) "}\n"
                 ::"r"(d), "r"((q >> 4) | (1u << 16)), "r"((k >> 4) | (1u << 16)), "r"(idesc), "r"(kDescHigh) : "memory");
    if constexpr (D == 128)
        asm volatile("{\n\t.reg .pred e, o;\n\t.reg .b64 a, b;\n\t.reg .b32 al, bl;\n\t"
                     "elect.sync _|e, 0xffffffff;\n\tsetp.eq.b32 o, 0, 0;\n\t"
                     SGK_MMA_S(1024, o) SGK_MMA_S(1026, o) SGK_MMA_S(1028, o) SGK_MMA_S(1030, o) "}\n"
                     ::"r"(d), "r"((q >> 4) | (1u << 16)), "r"((k >> 4) | (1u << 16)), "r"(idesc), "r"(kDescHigh) : "memory");
}
// O (+)= P V over half a tile's tokens in steps of 16: 8 columns of P each; V's low word, and how far behind it the second
// 16 and the second 32 tokens lie (in units of 16 bytes)
__device__ __forceinline__ void tc_output(uint32_t d, uint32_t p, uint32_t v, uint32_t second, uint32_t third, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred e, z, o;\n\t.reg .b64 b;\n\t.reg .b32 al, bl;\n\t"
                 "elect.sync _|e, 0xffffffff;\n\tsetp.ne.b32 z, %5, 0;\n\tsetp.eq.b32 o, 0, 0;\n\t"
                 SGK_MMA_O(0, "mov.u32 bl, %2;\n\t", z) SGK_MMA_O(8, "add.u32 bl, %2, %6;\n\t", o)
                 SGK_MMA_O(16, "add.u32 bl, %2, %7;\n\t", o) SGK_MMA_O(24, "add.u32 bl, bl, %6;\n\t", o) "}\n"
                 ::"r"(d), "r"(p), "r"(v), "r"(idesc), "r"(kDescHigh), "r"(accumulate), "r"(second), "r"(third) : "memory");
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
__device__ __forceinline__ void tc_st16(uint32_t addr, const uint32_t* v) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};\n"
                 ::"r"(addr), SGK_I8(v, 0), SGK_I8(v, 8) : "memory");
}
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(0xffffffffu, x, 0); }
// two fp32 operations in one instruction
__device__ __forceinline__ float2 fma2(float2 x, float2 y, float2 z) {
    float2 r;
    asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
        "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}\n"
        : "=f"(r.x), "=f"(r.y) : "f"(x.x), "f"(x.y), "f"(y.x), "f"(y.y), "f"(z.x), "f"(z.y));
    return r;
}
__device__ __forceinline__ float2 add2(float2 x, float2 y) {
    float2 r;
    asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}\n"
        : "=f"(r.x), "=f"(r.y) : "f"(x.x), "f"(x.y), "f"(y.x), "f"(y.y));
    return r;
}
// 2^(x + 1/2) for x <= 7.5 on the fp32 pipe: 2^round(x) by the exponent, 2^(x - round(x) + 1/2) in [1, 2) by the cubic with the
// least relative error (Remez, 7.5e-5: a fiftieth of a bf16 half step, which the weight is rounded to). The half is what lets
// x end at -127.5: with r = -127 the exponent field is 0 and the value a denormal, 7e-42 at the end, which bf16 rounds to 0. So
// a masked token's weight is 0 and its V of any finite size adds nothing (2^-126 of bf16's lowest value would be 4).
__device__ __forceinline__ float2 exp2_poly(float2 x) {
    x = make_float2(fmaxf(x.x, -127.4990234375f), fmaxf(x.y, -127.4990234375f));      // -127.5 + 2^-10: the cubic is above 1
    const float2 r = add2(x, make_float2(12582912.f, 12582912.f));        // 1.5 * 2^23: the rounded integer in the low bits
    const float2 f = fma2(add2(r, make_float2(-12582912.f, -12582912.f)), make_float2(-1.f, -1.f), x);
    float2 y = fma2(f, make_float2(0.07802452f, 0.07802452f), make_float2(0.34310395f, 0.34310395f));
    y = fma2(y, f, make_float2(0.98041904f, 0.98041904f));
    y = fma2(y, f, make_float2(1.4141119f, 1.4141119f));
    return make_float2(__int_as_float(__float_as_int(y.x) + (__float_as_int(r.x) << 23)),
                       __int_as_float(__float_as_int(y.y) + (__float_as_int(r.y) << 23)));
}
// the largest, or NaN if there is one
__device__ __forceinline__ float max3(float x, float y, float z) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(x), "f"(y), "f"(z));
    return r;
}
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ float ex2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Pages of 16 tokens: the copies of a tile (16 for K, 16 for V at d = 128) become what the producer spends its time on, so V
// comes with both 64-column halves of a page in one (long sequences 428 -> 405 us; pages of 64 lose 5 % by it: the bigger
// copies arrive later).
__host__ __device__ __forceinline__ bool paired(const PagedView& P, int d) { return d == 128 && P.page_shift == 4; }

template <int D, bool HAND>
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
    typedef Plan<kPtRU, kPtKT, HAND ? 2 : 1, kPtLead> PlanT;
    const int tid = threadIdx.x, lane = tid & 31, warp = uniform(tid >> 5);
    pdl_trigger();
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sm.tmem)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (tid == 256) {
        for (const CUtensorMap* m : {&mq, &mk, &mv}) asm volatile("prefetch.tensormap [%0];" ::"l"(m) : "memory");
        for (int i = 0; i < 2; ++i) {
            bar_init(&sm.q_full[i], 1); bar_init(&sm.q_empty[i], 2);
            bar_init(&sm.s_full[i], 1); bar_init(&sm.p_full[i], 4);
            bar_init(&sm.o_full[i], 1); bar_init(&sm.o_empty[i], 4);
            bar_init(&sm.join_bar[i], 4);
            sm.turns[i] = 0;
        }
        for (int i = 0; i < NS; ++i) { bar_init(&sm.kv_full[i], 1); bar_init(&sm.kv_empty[i], 2); }
        for (int i = 0; i < kPtRing; ++i) { bar_init(&sm.seg_full[i], 1); bar_init(&sm.seg_empty[i], 11); }
        bar_init(&sm.drain, 2);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        sm.failed = 0;
    }
    if (HAND && warp == 10 && lane < 16) {
        bar_init((lane & 8 ? &sm.hand_empty[0][0] : &sm.hand_full[0][0]) + (lane & 7), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    tc_fence_before();
    PlanT plan(P, a);
    plan.build(base + ((sizeof(Smem) + 15) & ~(size_t)15), &sm.flag, gridDim.x);
    tc_fence_after();
    int x = blockIdx.x * plan.chunk;
    const int x1 = min(plan.total, x + plan.chunk);
    const uint32_t tmem = (uint32_t)uniform((int)sm.tmem);

    // registers: three groups of four warps were launched with 168 a thread; 2 x 208 + 88 = 3 x 168
    if (x >= x1) {
        // nothing of the line is left for this block
    } else if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
        if (warp == 11) {
            // ---- planner ----
            unsigned ns = 0;
            while (true) {
                SegRec r;
                r.tile1 = -1;
                while (x < x1) {
                    const Seg g = plan.next(x, x1, blockIdx.x);
                    if (g.tile0 >= g.tile1) continue;
                    r = SegRec{g.e.ptab, g.e.stab, g.slot, g.tile0, g.tile1, g.kp, g.rows, g.head, g.ru, g.e.tok0, g.e.nq, g.e.S, g.e.P, g.direct, g.e.bad};
                    break;
                }
                const int slot = ns % kPtRing;
                if (ns >= kPtRing && !bar_wait(&sm.seg_empty[slot], (ns / kPtRing - 1) & 1, &sm.failed)) break;
                if (lane == 0) {
                    sm.seg[slot] = r;
                    bar_arrive(&sm.seg_full[slot]);
                }
                __syncwarp();
                ++ns;
                if (r.tile1 < 0) break;
            }
        } else if (warp == 8) {
            // ---- producer ----
            unsigned ns = 0, nq = 0, nk = 0;          // runs, query tiles and ring tiles so far
            const int pb = min(1 << P.page_shift, 128), chunks = 128 / pb;   // tokens one copy brings; copies for a half tile
            const int chunk = lane / HALVES, half = lane % HALVES;           // this lane's copy of a tile
            const bool pairs = paired(P, D);
            bool ok = true;
            while (ok) {
                const int slot = ns % kPtRing;
                if (!(ok = bar_wait(&sm.seg_full[slot], (ns / kPtRing) & 1, &sm.failed))) break;
                SegRec& r = sm.seg[slot];
                const int tile0 = uniform(r.tile0), tile1 = uniform(r.tile1), kp = uniform(r.kp), head = uniform(r.head), P_ = r.P, S_ = r.S;
                const int *ptab = r.ptab, *stab = r.stab;
                if (tile1 < 0) break;
                // the page of this lane's copy of tile t: -2 nothing to bring, -1 outside the pool
                auto page_of = [&](int t) {
                    const bool pre = t < kp;
                    const int pos = (pre ? t : t - kp) * kPtKT + chunk * pb;
                    if (t >= tile1 || chunk >= chunks || pos >= (pre ? P_ : S_)) return -2;
                    const int id = __ldg((pre ? ptab : stab) + (pos >> P.page_shift));
                    return id < 0 || id >= P.pages ? -1 : id;
                };
                int id = page_of(tile0);
                const int sub = r.rows > 128 ? 2 : 1;
                for (int i = 0; i < sub && ok; ++i, ++nq) {
                    const int qs = nq & 1;
                    if (nq >= 2 && !(ok = bar_wait(&sm.q_empty[qs], (nq / 2 - 1) & 1, &sm.failed))) break;
                    if (lane == 0) bar_expect(&sm.q_full[qs], Smem::kTile);
                    __syncwarp();
                    if (lane < 4 * HALVES) {           // 32 rows at a time, or the same 32 four times
                        const int step = r.rows > 32 ? 32 >> a.g_shift : 0, tok = r.tok0 + ((r.ru * kPtRU + i * 128) >> a.g_shift);
                        tma_load_3d(sm.Q[qs] + (lane >> 2) * 16384 + (lane & 3) * 4096, &mq, (lane >> 2) * 64, head << a.g_shift,
                                    tok + (lane & 3) * step, &sm.q_full[qs]);
                    }
                }
                for (int t = tile0; t < tile1 && ok; ++t) {
                    const int following = page_of(t + 1);        // asked for a tile early
                    const int row = ((t < kp ? t : t - kp) * kPtKT) & ((1 << P.page_shift) - 1);   // pieces of a page start at 0
                    if (__any_sync(0xffffffffu, id == -1) && lane == 0) {
                        *reinterpret_cast<volatile int*>(&r.bad) = 1;
                        paged_status(P, kStPage);
                    }
                    const unsigned bytes = __popc(__ballot_sync(0xffffffffu, id >= 0)) * (unsigned)pb * 128u;
                    for (int kv = 0; kv < 2; ++kv, ++nk) {
                        const int s = nk % NS;
                        if (nk >= NS && !(ok = bar_wait(&sm.kv_empty[s], (nk / NS - 1) & 1, &sm.failed))) break;
                        if (lane == 0) bar_expect(&sm.kv_full[s], bytes);
                        __syncwarp();
                        if (id < 0) continue;
                        if (!pairs || !kv) tma_load_4d(sm.KV[s] + half * 16384 + chunk * pb * 128, kv ? &mv : &mk, half * 64, row, head, id, &sm.kv_full[s]);
                        else if (!half) tma_load_5d(sm.KV[s] + chunk * pb * 256, &mv, 0, row, 0, head, id, &sm.kv_full[s]);
                    }
                    id = following;
                }
                __syncwarp();
                if (lane == 0) bar_arrive(&sm.seg_empty[slot]);
                ++ns;
            }
            // copies in flight write shared memory: they have to be done before the block ends
            for (unsigned i = nk > (unsigned)NS ? nk - NS : 0; i < nk; ++i)
                for (unsigned j = 0; j < kPtSpins && !bar_try(&sm.kv_full[i % NS], (i / NS) & 1); ++j) {}
            for (unsigned i = nq > 2 ? nq - 2 : 0; i < nq; ++i)
                for (unsigned j = 0; j < kPtSpins && !bar_try(&sm.q_full[i & 1], (i / 2) & 1); ++j) {}
        } else {
            // ---- issuers ----
            // Everything here is the same in all lanes, and said so by shuffles and votes. One warp per group, so that a wait
            // of one leaves no gap in the tensor pipe.
            const int w = warp - 9;
            // V lies as K does, or, in pairs, by pages of 16 tokens and in each of those [half][token][128 B]: in units of 16
            // bytes, how far apart the halves are, and how far on the second 16, 32 and 64 tokens
            const bool pairs = paired(P, D);
            const uint32_t apart = pairs ? 128u : 1024u, second = pairs ? 256u : 128u, third = 2 * second, upper = 4 * second;
            struct Cursor { int tile, tile0, tile1, kp, dual, order, rows, P, S, seg, q, kv, jobs, done; };
            bool ok = true;
            auto wait = [&](unsigned long long* b, int parity) { return bar_wait(b, (unsigned)parity, &sm.failed); };
            // The first run from c.seg on in which this group has a job. `release`: give up those in which it has none.
            auto enter = [&](Cursor& c, bool release) {
                while (true) {
                    const int slot = c.seg % kPtRing;
                    if (!(ok = wait(&sm.seg_full[slot], (c.seg / kPtRing) & 1))) { c.done = 1; return; }
                    const SegRec& r = sm.seg[slot];
                    c.tile0 = uniform(r.tile0); c.tile1 = uniform(r.tile1); c.kp = uniform(r.kp);
                    c.rows = uniform(r.rows); c.P = uniform(r.P); c.S = uniform(r.S);
                    c.dual = c.rows > 128 ? 1 : 0;
                    c.order = (w - c.jobs) & 1;
                    c.done = c.tile1 < 0 ? 1 : 0;
                    c.tile = c.tile0 + (c.dual ? 0 : c.order);
                    if (c.done || c.tile < c.tile1) return;
                    // one tile, and the other group's: the query tile counts both groups all the same (once it is there,
                    // or the arrival would count for the tile that had its place before)
                    if (!release && !(ok = wait(&sm.q_full[c.q & 1], (c.q / 2) & 1))) { c.done = 1; return; }
                    if (lane == 0) bar_arrive(release ? &sm.seg_empty[slot] : &sm.q_empty[c.q & 1]);
                    __syncwarp();
                    ++c.seg; ++c.q; ++c.kv; ++c.jobs;
                }
            };
            auto leave = [&](Cursor& c) {
                const int tiles = c.tile1 - c.tile0;
                c.q += 1 + c.dual;
                c.kv += tiles;
                c.jobs += tiles << c.dual;
                ++c.seg;
            };
            Cursor qk = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0}, pv = qk;
            int segs = 0, mine = 0, turns = 0;         // runs whose numerator the group has begun, products with V, those of shared tiles
            // Whether Q and K of the next S are there: asked before P V is issued, so that S can follow without a wait.
            auto issue_ready = [&]() {
                if (qk.done) return false;
                const int qt = qk.q + (qk.dual ? qk.order : 0), ks = 2 * (qk.kv + qk.tile - qk.tile0), s = ks % NS;
                const bool q = qk.tile >= qk.tile0 + 2 || bar_test(&sm.q_full[qt & 1], (qt / 2) & 1);
                return (bool)__all_sync(0xffffffffu, q && bar_test(&sm.kv_full[s], (ks / NS) & 1));
            };
            auto issue_qk = [&](bool there) {
                if (qk.done || !ok) return;
                const int qt = qk.q + (qk.dual ? qk.order : 0), ks = 2 * (qk.kv + qk.tile - qk.tile0), s = ks % NS, step = 2 - qk.dual;
                if (!there) {
                    if (qk.tile < qk.tile0 + 2 && !(ok = wait(&sm.q_full[qt & 1], (qt / 2) & 1))) return;
                    if (!(ok = wait(&sm.kv_full[s], (ks / NS) & 1))) return;
                }
                const bool last = qk.tile + step >= qk.tile1;
                const uint32_t qa = smem_u32(sm.Q[qt & 1]), ka = smem_u32(sm.KV[s]);
                tc_fence_after();
                tc_scores<D>(tmem + w * 128u, qa, ka, kIdescS);
                tc_commit(&sm.s_full[w]);
                tc_commit(&sm.kv_empty[s]);            // a slot counts two: both groups', or this one's twice
                if (!qk.dual) tc_commit(&sm.kv_empty[s]);
                if (last) {
                    tc_commit(&sm.q_empty[qt & 1]);
                    if (qk.dual) tc_commit(&sm.q_empty[qt & 1]);
                }
                __syncwarp();
                qk.tile += step;
                if (last) {
                    leave(qk);
                    enter(qk, false);
                }
            };
            enter(qk, false);
            enter(pv, true);
            issue_qk(false);
            while (!pv.done && ok) {
                const int vs = 2 * (pv.kv + pv.tile - pv.tile0) + 1, s = vs % NS, step = 2 - pv.dual;
                const bool fresh = pv.tile < pv.tile0 + step, last = pv.tile + step >= pv.tile1;
                if (!(ok = wait(&sm.kv_full[s], (vs / NS) & 1))) break;
                const bool pre = pv.tile < pv.kp;
                const int nv = pre ? pv.P - pv.tile * kPtKT : pv.S - (pv.tile - pv.kp) * kPtKT;
                if (nv < kPtKT) {                      // the sequence ends in this tile: clear what lies behind
                    for (int p = lane; p < (kPtKT - nv) * 8 * HALVES; p += 32) {
                        const int row = nv + p / (8 * HALVES), c = p % (8 * HALVES);
                        const int at = pairs ? (row >> 4) * 4096 + (c >> 3) * 2048 + (row & 15) * 128 : (c >> 3) * 16384 + row * 128;
                        *reinterpret_cast<uint4*>(sm.KV[s] + at + (c & 7) * 16) = make_uint4(0, 0, 0, 0);
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                }
                if (fresh) {
                    if (segs && !(ok = wait(&sm.o_empty[w], (segs - 1) & 1))) break;
                    ++segs;
                }
                const uint32_t va = (smem_u32(sm.KV[s]) >> 4) | (apart << 16);
                const uint32_t first = fresh ? 0u : 1u;
                const bool k_there = issue_ready();
                // Two groups on the same tiles take turns, P V and the next S of one, then of the other. Left to themselves
                // both pairs run interleaved, end together, and the tensor pipe waits while both groups exponentiate.
                const bool turn = pv.dual && (pv.order || pv.tile != pv.tile0);
                if (turn && !(ok = count_wait(&sm.turns[1 - w], turns + pv.order, &sm.failed))) break;
                if (!(ok = wait(&sm.p_full[w], mine & 1))) break;
                tc_fence_after();
                const uint32_t td = tmem + 256u + w * (uint32_t)D, tp = tmem + w * 128u;
                tc_output(td, tp, va, second, third, kIdescO, first);
                tc_output(td, tp + 32u, va + upper, second, third, kIdescO, 1u);
                tc_commit(&sm.kv_empty[s]);
                if (!pv.dual) tc_commit(&sm.kv_empty[s]);
                if (last) tc_commit(&sm.o_full[w]);
                __syncwarp();
                pv.tile += step;
                issue_qk(k_there);
                ++mine;
                turns += pv.dual;
                if (pv.dual && lane == 0) *reinterpret_cast<volatile int*>(&sm.turns[w]) = turns;
                if (last) {
                    __syncwarp();
                    if (lane == 0) bar_arrive(&sm.seg_empty[pv.seg % kPtRing]);
                    __syncwarp();
                    leave(pv);
                    enter(pv, true);
                }
            }
            tc_commit(&sm.drain);                     // the MMAs read shared memory: done before the block ends
            __syncwarp();
            for (unsigned j = 0; j < kPtSpins && !bar_try(&sm.drain, 0); ++j) {}
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
        // ---- softmax ----
        const int w = warp >> 2, quarter = warp & 3;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        const uint32_t tS = tmem + lanes + (uint32_t)w * 128u, tO = tmem + lanes + 256u + (uint32_t)(w * D);
        unsigned ns = 0, job = 0, mine = 0, segs = 0;  // runs, jobs of both groups, jobs and runs of this one
        bool ok = true;
        float m = 0.f, l = 0.f, edge = 0.f, off = 0.f, cr = 0.f;   // of this thread's row: the maximum in use, the sum, the score
                                                       // from which on the maximum is replaced, -m * cr, c or less
        const float margin = 8.f / a.c;
        bool begun = false, live = false;              // live: the row is one of the unit's (other lanes may hold anything)
        unsigned joins = 0, hands = 0;                 // hands: rows that this warp has handed over or taken
        auto joined = [&]() {                          // the group's four warps have come here
            __syncwarp();
            if (lane == 0) bar_arrive(&sm.join_bar[w]);
            return ok = bar_wait(&sm.join_bar[w], joins++ & 1, &sm.failed);
        };
        // A new maximum of the row: keep the one in use, or change to the new one and rescale.
        auto raise = [&](float top) {
            const bool rise = live && !(top <= edge);  // a NaN becomes the maximum, and the sum NaN with it
            if (__any_sync(0xffffffffu, rise)) {
                const float f = rise ? ex2_approx((m - top) * a.c) : 1.f;              // 0 when there was no maximum yet
                if (rise) {
                    m = top;
                    edge = top + margin;
                    // -m * c is rounded once more than s * c + off: by 2^-4 at 2^20, by more than any exponent holds at 2^31. A
                    // score is no better known there (d sums rounded to 2^-24 of it), so from 2^21 on a factor that is smaller
                    // by a power of two does as well: scores that sums over d = 64 can tell apart stay 17 octaves apart. Sums
                    // are joined by c as ever.
                    const int e = max((__float_as_int(top * a.c) >> 23) & 255, 127 + 20);
                    cr = a.c * __int_as_float((127 + 127 + 20 - e) << 23);
                    off = -top * cr;
                }
                l *= f;
                if (begun) {
                    uint32_t o[32];
#pragma unroll 1
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
        };
        // N scores of the row -> bf16 weights, two to a register; adds them to the sum
        auto weigh = [&](auto count, const uint32_t* s, uint32_t* p) {
            constexpr int N = decltype(count)::value;
            const float2 cc = make_float2(cr, cr), oo = make_float2(off, off), oh = make_float2(off - 0.5f, off - 0.5f);
            float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                float2 x = fma2(make_float2(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])), cc, i % 8 < kPtPoly ? oh : oo);
                if (i % 8 < kPtPoly) x = exp2_poly(x);
                else x = make_float2(ex2_approx(x.x), ex2_approx(x.y));
                sum[i & 1] = add2(sum[i & 1], x);
                const __nv_bfloat162 b = __float22bfloat162_rn(x);
                p[i] = *reinterpret_cast<const uint32_t*>(&b);
            }
            sum[0] = add2(sum[0], sum[1]);
            l += sum[0].x + sum[0].y;
        };
        auto largest = [&](auto count, const uint32_t* s) {
            constexpr int N = decltype(count)::value;
            float t[4] = {m, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int i = 0; i < N; i += 8) {
#pragma unroll
                for (int j = 0; j < 4; ++j) t[j] = max3(t[j], __uint_as_float(s[i + 2 * j]), __uint_as_float(s[i + 2 * j + 1]));
            }
            return max3(max3(t[0], t[1], t[2]), t[3], t[3]);
        };
        while (ok) {
            const int slot = ns % kPtRing;
            if (!(ok = bar_wait(&sm.seg_full[slot], (ns / kPtRing) & 1, &sm.failed))) break;
            const SegRec& r = sm.seg[slot];
            const int tile0 = r.tile0, tile1 = r.tile1, kp = r.kp, rows = r.rows;
            if (tile1 < 0) break;
            const int dual = rows > 128, tiles = tile1 - tile0, order = (w - (int)job) & 1;   // order: this group's half, or turn
            const bool quad = rows <= 32;
            const int row = quad ? lane : (dual ? order * 128 : 0) + quarter * 32 + lane;
            const bool some = quad || (row & ~31) < rows;
            live = row < rows;
            const int urow = r.ru * kPtRU + row, P_ = r.P;
            Entry e;
            e.S = r.S; e.nq = r.nq;
            const int own = plan.own_limit(e, urow);
            m = edge = -INFINITY;
            l = off = 0.f;
            cr = a.c;
            begun = false;
            for (int t = tile0 + (dual ? 0 : order); t < tile1; t += 2 - dual) {
                const bool pre = t < kp;
                const int lim = pre ? P_ - t * kPtKT : own - (t - kp) * kPtKT;        // tokens of the tile that the row sees
                const bool cut = __any_sync(0xffffffffu, lim < kPtKT);
                if (!(ok = bar_wait(&sm.s_full[w], mine & 1, &sm.failed))) break;
                if (quad) {
                    tc_fence_after();
                    uint32_t s[32], p[16];
                    tc_ld32(tS + quarter * 32, s);
                    tc_wait_ld();
                    if (cut) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) s[i] = quarter * 32 + i < lim ? s[i] : 0xff800000u;
                    }
                    raise(largest(std::integral_constant<int, 32>(), s));
                    weigh(std::integral_constant<int, 32>(), s, p);
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[i] = 0;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (j == quarter) tc_st16(tS + j * 16, p);
                        else tc_st16(tS + j * 16, s);
                    }
                    tc_wait_st();
                    tc_fence_before();
                } else if (some) {
                    tc_fence_after();
                    uint32_t s[128];
#pragma unroll
                    for (int i = 0; i < 4; ++i) tc_ld32(tS + i * 32, s + i * 32);
                    tc_wait_ld();
                    if (cut) {
#pragma unroll
                        for (int i = 0; i < 128; ++i) s[i] = i < lim ? s[i] : 0xff800000u;
                    }
                    raise(largest(std::integral_constant<int, 128>(), s));
                    uint32_t p[64];
                    weigh(std::integral_constant<int, 128>(), s, p);
                    tc_st32(tS, p);
                    tc_st32(tS + 32, p + 32);
                    tc_wait_st();
                    tc_fence_before();
                }
                begun = true;
                __syncwarp();
                if (lane == 0) {
                    bar_arrive(&sm.p_full[w]);
                }
                ++mine;
            }
            if (!ok) break;
            job += dual ? 2 * tiles : tiles;
            ++ns;
            if (begun) {
                // no score above -infinity here, or one that is not finite
                if (!(fabsf(m * a.c) < INFINITY)) l = m == -INFINITY ? 0.f : NAN;
                // a whole row without weights: nothing to see (0), or nothing but scores of -infinity (NaN, as the formula's)
                const float none = P_ > 0 || own > 0 ? NAN : 0.f;
                if (!(ok = bar_wait(&sm.o_full[w], segs & 1, &sm.failed))) break;
                ++segs;
                const int gs = a.g_shift, bad = *reinterpret_cast<const volatile int*>(&r.bad);
                const bool direct = r.direct;
                const int slot0 = r.slot + (order == 0 || !PlanT::twice(rows) ? 0 : rows);
                if (quad) {
                    // the four warps' numerators, four rows at a time: [warp][row][column] in shared memory, added by one
                    // thread for four columns
                    tc_fence_after();
                    sm.join_stat[w][quarter][lane] = make_float2(m, l);
                    uint32_t o[D];
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) tc_ld32(tO + i * 32, o + i * 32);
                    tc_wait_ld();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(&sm.o_empty[w]);
                    for (int r0 = 0; r0 < rows; r0 += 4) {
                        // before the next four rows; the next run's numerators come after everybody's weights for it
                        if (r0 && !joined()) break;
                        if (lane >= r0 && lane < r0 + 4) {
                            uint4* z = reinterpret_cast<uint4*>(&sm.join[w][quarter][lane - r0][0]);
#pragma unroll
                            for (int j = 0; j < D / 4; ++j) z[j] = make_uint4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
                        }
                        if (!joined()) break;
                        const int rr = r0 + quarter;             // a warp per row
                        const float rr_none = __shfl_sync(0xffffffffu, none, rr & 31);
                        if (rr < rows) {
                            float2 st[4];
                            float M = -INFINITY, L = 0.f;
#pragma unroll
                            for (int k = 0; k < 4; ++k) { st[k] = sm.join_stat[w][k][rr]; M = fmaxf(M, st[k].x); }
                            const float base = M == -INFINITY ? 0.f : M;
                            float z[D / 32];
#pragma unroll
                            for (int j = 0; j < D / 32; ++j) z[j] = 0.f;
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const float f = ex2_approx((st[k].x - base) * a.c);
                                L = fmaf(st[k].y, f, L);
#pragma unroll
                                for (int j = 0; j < D / 32; ++j) z[j] = fmaf(sm.join[w][k][quarter][j * 32 + lane], f, z[j]);
                            }
                            if (bad) L = NAN;
                            if (HAND && tiles > 1) {                     // the other group has the other tiles' share of the row
                                const int at = hands & 1, parity = (hands >> 1) & 1;
                                ++hands;
                                if (w) {
                                    if (hands > 2 && !(ok = bar_wait(&sm.hand_empty[quarter][at], parity ^ 1, &sm.failed))) break;
#pragma unroll
                                    for (int j = 0; j < D / 32; ++j) sm.hand[quarter][at][j * 32 + lane] = z[j];
                                    if (lane == 0) sm.hand_stat[quarter][at] = make_float2(M, L);
                                    __syncwarp();
                                    if (lane == 0) bar_arrive(&sm.hand_full[quarter][at]);
                                    continue;
                                }
                                if (!(ok = bar_wait(&sm.hand_full[quarter][at], parity, &sm.failed))) break;
                                const float2 other = sm.hand_stat[quarter][at];
                                const float both = fmaxf(M, other.x), b = both == -INFINITY ? 0.f : both;
                                const float f = ex2_approx((M - b) * a.c), fo = ex2_approx((other.x - b) * a.c);
                                M = both;
                                L = L * f + other.y * fo;
#pragma unroll
                                for (int j = 0; j < D / 32; ++j) z[j] = fmaf(sm.hand[quarter][at][j * 32 + lane], fo, z[j] * f);
                                __syncwarp();
                                if (lane == 0) bar_arrive(&sm.hand_empty[quarter][at]);
                            }
                            const int gr = r.ru * kPtRU + rr, tok = r.tok0 + (gr >> gs), head = (r.head << gs) + (gr & ((1 << gs) - 1));
                            if (direct) {
                                const float f = L == 0.f ? rr_none : 1.f / L;
                                __nv_bfloat16* y = (__nv_bfloat16*)a.o.p + tok * a.o.ts + head * a.o.hs;
#pragma unroll
                                for (int j = 0; j < D / 32; ++j) y[j * 32 + lane] = __float2bfloat16_rn(z[j] * f);
                            } else {
                                float* y = a.part + (long long)(slot0 + rr) * D;
#pragma unroll
                                for (int j = 0; j < D / 32; ++j) y[j * 32 + lane] = z[j];
                                if (lane == 0) a.stat[slot0 + rr] = make_float2(M * a.c, L);
                            }
                        }
                    }
                } else if (some) {
                    tc_fence_after();
                    if (bad) l = NAN;
                    const int tok = r.tok0 + (urow >> gs), head = (r.head << gs) + (urow & ((1 << gs) - 1));
                    const float f = direct ? (l == 0.f ? none : 1.f / l) : 1.f;
                    __nv_bfloat16* y = (__nv_bfloat16*)a.o.p + tok * a.o.ts + head * a.o.hs;
                    if (live && !direct) a.stat[slot0 + row] = make_float2(m * a.c, l);
                    __syncwarp();
                    uint32_t o[D];
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) tc_ld32(tO + i * 32, o + i * 32);
                    tc_wait_ld();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(&sm.o_empty[w]);
                    if (live && direct) {
#pragma unroll
                        for (int j = 0; j < D; j += 8) {
                            uint4 v;
                            uint32_t* vv = &v.x;
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const __nv_bfloat162 b = __floats2bfloat162_rn(__uint_as_float(o[j + 2 * k]) * f, __uint_as_float(o[j + 2 * k + 1]) * f);
                                vv[k] = *reinterpret_cast<const uint32_t*>(&b);
                            }
                            *reinterpret_cast<uint4*>(y + j) = v;
                        }
                    } else if (live) {
                        uint4* z = reinterpret_cast<uint4*>(a.part + (long long)(slot0 + row) * D);
#pragma unroll
                        for (int j = 0; j < D / 4; ++j) z[j] = make_uint4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
                    }
                } else {
                    __syncwarp();
                    if (lane == 0) bar_arrive(&sm.o_empty[w]);
                }
                __syncwarp();
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
