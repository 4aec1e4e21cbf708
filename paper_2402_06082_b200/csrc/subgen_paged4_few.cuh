// Attention over a cache in 4-bit cells for few query rows a sequence: single tokens and drafts.
//
// out = softmax(scale q K^T) V with K, V = value / 8 of Cell4, exact in fp16, straight from registers into mma m16n8k16 (fp16
// operands, fp32 sums). Per byte of the cache there is little time: 4.5 bits a value at the HBM rate are 2304 bytes (a cell of
// 16 tokens, K and V) every 98 cycles of an SM, 392 of a scheduler. So codes are expanded once, by 11 instructions for 8 of
// them, in the lane whose fragment needs them, and never written anywhere:
//   S^T = K Q^T   A = 16 tokens x 16 coordinates. The contraction's order is free: lane (g, t) of a quad row takes the row's bytes
//                 t * D / 8 ..., 2 * D / 8 coordinates on end, one 16-byte load, and Q's fragment is loaded to match.
//   O^T += V^T P^T  A = 16 coordinates x 16 tokens: the lane takes 4 tokens' bytes g * D / 16 ..., and two tokens' words are interleaved
//                 by halves (one byte permutation for 4 pairs), since a pair of this fragment is two tokens of one coordinate.
// Rows (tokens x heads of a KV head) are the 8 columns, NT times; P changes from S's layout to its own by movmatrix. fp32
// queries and weights are split into two fp16 (22 bits), which doubles the columns or products (PIECES).
// Row r of the 16 is token r ^ (r >> 1 & 1) of the cell: then neither the loads of K nor those of V meet the same banks more
// than twice.
// Queries are scaled by a power of two (largest magnitude to [2^14, 2^15)), so fp16 holds what bf16 does down to 2^-29 of it.
// Weights are 2^(score - reference + 6), the reference a maximum that is replaced (and the sums rescaled) only when a score is
// 2^8 above it: at most 2^14, and what fp16 loses at the other end is below 2^-31 of the largest.
//
// A block: 4 warps, two cells each of every tile of 128 tokens (two chains of products at a time), and one that walks the block's share of the plan and brings tiles by
// bulk copies (a page's cells lie on end) and the runs' queries. At the end of a run the 4 results are joined through shared
// memory. Bound by the instructions of the expansion and their latency (counted: 300 a cell, of which 139 fp32 and fp16, 111
// logic, 16 products; issue slots 65 % busy with 12 warps an SM, neither pipe above 50 %): 131072 tokens x 8 heads x 128 in 45 us,
// 29 to 32 of it by the tokens (4.7 to 5.3 TB/s), the rest start, end and merge. Measured on the way (one long sequence / 64
// sequences of up to 8191, us): shifts and masks as written 53 / 114; shifts to the left as multiply-adds 51 / 106; mask and exponent
// in registers 47 / 93; two cells a warp, three blocks of 4 warps 45 / 89; third tile 44 / 86; 8 warps in two blocks of 96
// registers 45 / 92; U = 1 in 18 warps 47 / 93.
// Every wait is bounded: when one gives up, the block sets SUBGEN_ST_TIMEOUT, waits for its copies (bounded) and returns.
#pragma once
#include <type_traits>

#include "subgen_paged_tc.cuh"

namespace sgk {

constexpr int kP4Warps = 4, kP4Cells = 2, kP4Threads = 32 * (kP4Warps + 1), kP4KT = 16 * kP4Warps * kP4Cells, kP4Lead = 2, kP4Runs = 2;
constexpr float kP4Shift = 6.f, kP4Margin = 8.f;

template <typename T, int D, int NT, int TILES>
struct P4Smem {
    static constexpr int RU = 8 * NT, kTile = kP4Warps * kP4Cells * Cell4<D>::kBytes, kTiles = TILES, kQRow = D * (int)sizeof(T) + 16, kJoin = D + 4;
    unsigned char tile[kTiles][kTile];
    unsigned char q[RU][kQRow];                       // of one run: free again as soon as it is in registers
    float join[kP4Warps][RU][kJoin];
    float2 stat[kP4Warps][RU];                        // reference * factor, sum
    float factor[RU];                                 // of a row's scores
    SegRec run[kP4Runs];
    unsigned long long full[kTiles], empty[kTiles], run_full[kP4Runs], run_empty[kP4Runs], q_full, q_ready, q_empty, joined, read;
    int failed, flag;
};
template <int NT> constexpr int kP4Blocks = NT == 1 ? 3 : 2;

__device__ __forceinline__ void mma_f16(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {         // 8 x 8 pairs of halves
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ uint32_t halves(float x, float y) {
    const __half2 h = __floats2half2_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// what the rounding to fp16 took off
__device__ __forceinline__ uint32_t rest(float x, float y, uint32_t h) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
    return halves(x - f.x, y - f.y);
}

template <typename T, int D, int NT, int TILES>
__global__ void __launch_bounds__(kP4Threads, kP4Blocks<NT>) paged4_attend_few_kernel(PagedView P, Attend a) {
    typedef P4Smem<T, D, NT, TILES> S;
    typedef Cell4<D> C;
    constexpr int RU = S::RU, NW = kP4Warps, U = kP4Cells, PIECES = sizeof(T) == 4 ? 2 : 1, KS = D / 16, MT = D / 16;
    extern __shared__ __align__(128) unsigned char dyn4[];
    S& sm = *reinterpret_cast<S*>(dyn4);
    const int tid = threadIdx.x, lane = tid & 31, warp = uniform(tid >> 5);
    pdl_trigger();
    if (tid == 0) {
        for (int i = 0; i < S::kTiles; ++i) { bar_init(&sm.full[i], 1); bar_init(&sm.empty[i], NW); }
        for (int i = 0; i < kP4Runs; ++i) { bar_init(&sm.run_full[i], 1); bar_init(&sm.run_empty[i], NW); }
        bar_init(&sm.q_full, 1);
        bar_init(&sm.q_ready, NW);
        bar_init(&sm.q_empty, NW);
        bar_init(&sm.joined, NW);
        bar_init(&sm.read, NW);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        sm.failed = 0;
    }
    Plan<RU, kP4KT, 0, kP4Lead> plan(P, a);
    plan.build(dyn4 + ((sizeof(S) + 15) & ~(size_t)15), &sm.flag, gridDim.x);        // barriers of the block inside
    int x = blockIdx.x * plan.chunk;
    const int x1 = min(plan.total, x + plan.chunk);
    if (x >= x1) return;                                             // the same for the whole block

    if (warp == NW) {
        // ---- plan and copies ----
        unsigned ns = 0, nt = 0;
        const int pb = min(1 << P.page_shift, kP4KT);                // tokens a copy brings at most
        bool ok = true;
        while (ok) {
            SegRec r;
            r.tile1 = -1;
            while (x < x1) {
                const Seg g = plan.next(x, x1, blockIdx.x);
                if (g.tile0 >= g.tile1) continue;
                r = SegRec{g.e.ptab, g.e.stab, g.slot, g.tile0, g.tile1, g.kp, g.rows, g.head, g.ru, g.e.tok0, g.e.nq, g.e.S, g.e.P, g.direct, g.e.bad};
                break;
            }
            const int slot = ns % kP4Runs;
            if (ns >= kP4Runs && !(ok = bar_wait(&sm.run_empty[slot], (ns / kP4Runs - 1) & 1, &sm.failed))) break;
            const bool last = r.tile1 < 0;
            if (lane == 0) {
                sm.run[slot] = r;
                bar_arrive(&sm.run_full[slot]);
            }
            __syncwarp();
            if (last) break;
            if (ns && !(ok = bar_wait(&sm.q_empty, (ns - 1) & 1, &sm.failed))) break;
            if (lane == 0) bar_expect(&sm.q_full, (unsigned)r.rows * (unsigned)(D * sizeof(T)));
            __syncwarp();
            if (lane < r.rows) {                                     // RU <= 32
                const int gr = r.ru * RU + lane, tok = r.tok0 + (gr >> a.g_shift), head = (r.head << a.g_shift) + (gr & ((1 << a.g_shift) - 1));
                bulk_load(sm.q[lane], (const T*)a.q.p + tok * a.q.ts + head * a.q.hs, D * sizeof(T), &sm.q_full);
            }
            ++ns;
            // this lane's copy of tile t: tokens [pos, pos + 16 * cells) of a page; -1 a page outside the pool, cells 0: nothing
            auto copy_of = [&](int t, int* cells, int* row) {
                const bool pre = t < r.kp;
                const int pos = (pre ? t : t - r.kp) * kP4KT + lane * pb, len = pre ? r.P : r.S;
                *cells = 0;
                *row = pos & ((1 << P.page_shift) - 1);
                if (t >= r.tile1 || lane * pb >= kP4KT || pos >= len) return -2;
                *cells = min(pb, len - pos + 15) >> 4;
                const int id = __ldg((pre ? r.ptab : r.stab) + (pos >> P.page_shift));
                return id < 0 || id >= P.pages ? -1 : id;
            };
            int cells, row, id = copy_of(r.tile0, &cells, &row);
            for (int t = r.tile0; t < r.tile1; ++t, ++nt) {
                int cells2, row2;
                const int id2 = copy_of(t + 1, &cells2, &row2);      // asked for a tile early
                const int s = nt % S::kTiles;
                if (nt >= S::kTiles && !(ok = bar_wait(&sm.empty[s], (nt / S::kTiles - 1) & 1, &sm.failed))) break;
                if (__any_sync(0xffffffffu, id == -1)) {
                    if (lane == 0) {
                        *reinterpret_cast<volatile int*>(&sm.run[slot].bad) = 1;     // before this tile's barrier
                        paged_status(P, kStPage);
                    }
                }
                const unsigned bytes = id >= 0 ? cells * C::kBytes : 0u, all = __reduce_add_sync(0xffffffffu, bytes);
                if (lane == 0) bar_expect(&sm.full[s], all);
                __syncwarp();
                if (bytes)
                    bulk_load(sm.tile[s] + (lane * pb >> 4) * C::kBytes, P.K + id * P.ps + r.head * P.hs + (row >> 4) * C::kBytes, bytes, &sm.full[s]);
                id = id2; cells = cells2; row = row2;
            }
        }
        // copies in flight write shared memory: they have to be done before the block ends
        for (unsigned i = nt > (unsigned)S::kTiles ? nt - S::kTiles : 0; i < nt; ++i)
            for (unsigned j = 0; j < kPtSpins && !bar_try(&sm.full[i % S::kTiles], (i / S::kTiles) & 1); ++j) {}
        if (ns)
            for (unsigned j = 0; j < kPtSpins && !bar_try(&sm.q_full, (ns - 1) & 1); ++j) {}
    } else {
        // ---- products ----
        const int g = lane >> 2, t = lane & 3;
        const int tk0 = g ^ (g >> 1 & 1), tv0 = 2 * t ^ (t & 1), tv1 = (2 * t + 1) ^ (t & 1);        // tokens of rows g, 2t, 2t + 1
        const Consts4 consts;
        unsigned ns = 0, nt = 0;
        bool ok = true;
        while (ok) {
            const int slot = ns % kP4Runs;
            if (!(ok = bar_wait(&sm.run_full[slot], (ns / kP4Runs) & 1, &sm.failed))) break;
            const SegRec& r = sm.run[slot];
            const int tile0 = r.tile0, tile1 = r.tile1, kp = r.kp, rows = r.rows;
            if (tile1 < 0) break;
            // queries, to fp16 where they lie, a warp a row (fp32: the rest behind), and from there every warp's fragments: row g of column
            // block n, coordinates t * D / 4 ... (Each warp on its own, all in registers, was four times the work in straight code, which
            // short calls spend their time on fetching.)
            if (!(ok = bar_wait(&sm.q_full, ns & 1, &sm.failed))) break;
#pragma unroll 1
            for (int row = warp; row < RU; row += NW) {
                constexpr int VL = D / 32;
                float f[VL];
                unsigned top = 0;
#pragma unroll
                for (int i = 0; i < VL; ++i) {
                    f[i] = row < rows ? to_float(reinterpret_cast<const T*>(sm.q[row])[lane * VL + i]) : 0.f;
                    top = max(top, __float_as_uint(f[i]) & 0x7fffffffu);
                }
                top = __reduce_max_sync(0xffffffffu, top);
                // 2^(14 - e) and its reciprocal, both normal numbers; a row that is not finite becomes NaN
                const int ex = min(max((int)(top >> 23), 15), 254);
                const float up = top >= 0x7f800000u ? NAN : __uint_as_float((unsigned)(268 - ex) << 23);
                __syncwarp();
#pragma unroll
                for (int i = 0; i < VL; i += 2) {
                    const float u0 = f[i] * up, u1 = f[i + 1] * up;
                    const uint32_t h = halves(u0, u1);
                    uint32_t* to = reinterpret_cast<uint32_t*>(sm.q[row]) + (lane * VL + i) / 2;
                    to[0] = h;
                    if constexpr (PIECES == 2) to[D / 2] = rest(u0, u1, h);
                }
                const float cc = a.c * 8.f * __uint_as_float((unsigned)(ex - 14) << 23);
                // not 0, which times -infinity would be NaN, nor infinite, which times 0 would be
                if (lane == 0) sm.factor[row] = fminf(fmaxf(cc, 1.1754944e-38f), 3.4028235e38f);
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // the next run's queries come by a copy
            __syncwarp();
            if (lane == 0) bar_arrive(&sm.q_ready);
            if (!(ok = bar_wait(&sm.q_ready, ns & 1, &sm.failed))) break;
            uint32_t q[NT][PIECES][KS * 2];
            float c[NT][2];                                          // exponent per unit of a score, of columns 2t and 2t + 1
            int own[NT][2];
            Entry e;
            e.S = r.S; e.nq = r.nq;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
#pragma unroll
                for (int p = 0; p < PIECES; ++p)
#pragma unroll
                    for (int i = 0; i < KS * 2; i += 4)
                        *reinterpret_cast<uint4*>(&q[n][p][i]) = *reinterpret_cast<const uint4*>(sm.q[n * 8 + g] + p * 2 * D + t * (D / 2) + i * 4);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    c[n][j] = sm.factor[n * 8 + 2 * t + j];
                    own[n][j] = plan.own_limit(e, r.ru * RU + n * 8 + 2 * t + j);
                }
            }
            __syncwarp();
            if (lane == 0) bar_arrive(&sm.q_empty);
            const int own_least = plan.own_limit(e, r.ru * RU);
            float acc[NT][MT][4], m[NT][2], ref[NT][2], edge[NT][2], l[NT][2];      // ref: m, or 0 where there is none
#pragma unroll
            for (int n = 0; n < NT; ++n) {
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[n][i][j] = 0.f;
#pragma unroll
                for (int j = 0; j < 2; ++j) { m[n][j] = edge[n][j] = -INFINITY; ref[n][j] = l[n][j] = 0.f; }
            }
            for (int ti = tile0; ti < tile1; ++ti, ++nt) {
                const int s = nt % S::kTiles;
                const bool pre = ti < kp;
                // cells u * NW + warp of the tile; all of them even if the last ones hold no tokens: their scores are masked, their values 0
                const int base = (pre ? ti : ti - kp) * kP4KT + warp * 16, have = (pre ? r.P : r.S) - base;      // tokens from this warp's first cell on
                if (!(ok = bar_wait(&sm.full[s], (nt / S::kTiles) & 1, &sm.failed))) break;
                if (have > 0) {
                    const unsigned char* const tile = sm.tile[s] + warp * C::kBytes;
                    const bool tail = have < 16 * NW * (U - 1) + 16;
                    float sc[U][NT][4];
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const unsigned char* cell = tile + u * NW * C::kBytes;
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int j = 0; j < 4; ++j) sc[u][n][j] = 0.f;
                        constexpr int W = D / 32;                    // words of 8 codes
                        uint32_t k0[W], k1[W], s0, s1;
                        const unsigned char *y0 = cell + tk0 * C::kCodes + t * (W * 4), *y1 = y0 + 8 * C::kCodes;
                        const unsigned char *z0 = cell + C::kScaleAt + tk0 * C::kScales + t * (W / 2), *z1 = z0 + 8 * C::kScales;
                        if constexpr (W == 4) {
                            *reinterpret_cast<uint4*>(k0) = *reinterpret_cast<const uint4*>(y0);
                            *reinterpret_cast<uint4*>(k1) = *reinterpret_cast<const uint4*>(y1);
                            s0 = *reinterpret_cast<const unsigned short*>(z0);
                            s1 = *reinterpret_cast<const unsigned short*>(z1);
                        } else {
                            *reinterpret_cast<uint2*>(k0) = *reinterpret_cast<const uint2*>(y0);
                            *reinterpret_cast<uint2*>(k1) = *reinterpret_cast<const uint2*>(y1);
                            s0 = *z0;
                            s1 = *z1;
                        }
                        __half2 f0[W / 2], o0[W / 2], f1[W / 2], o1[W / 2];
#pragma unroll
                        for (int w = 0; w < W / 2; ++w) {
                            scale_pair4(__byte_perm(s0, 0, 0x4040 + w * 0x0101), consts, &f0[w], &o0[w]);
                            scale_pair4(__byte_perm(s1, 0, 0x4040 + w * 0x0101), consts, &f1[w], &o1[w]);
                        }
#pragma unroll
                        for (int w = 0; w < W; ++w) {
                            uint32_t x0[4], x1[4];
                            pairs4(k0[w], f0[w / 2], o0[w / 2], consts, x0);
                            pairs4(k1[w], f1[w / 2], o1[w / 2], consts, x1);
#pragma unroll
                            for (int n = 0; n < NT; ++n)
#pragma unroll
                                for (int p = PIECES - 1; p >= 0; --p) {
                                    mma_f16(sc[u][n], x0[0], x1[0], x0[1], x1[1], q[n][p][4 * w], q[n][p][4 * w + 1]);
                                    mma_f16(sc[u][n], x0[2], x1[2], x0[3], x1[3], q[n][p][4 * w + 2], q[n][p][4 * w + 3]);
                                }
                        }
                    }
                    // limits: what a row does not see is -infinity
                    if (tail || (!pre && own_least - base < 16 * NW * (U - 1) + 16)) {
#pragma unroll
                        for (int u = 0; u < U; ++u)
#pragma unroll
                            for (int n = 0; n < NT; ++n)
#pragma unroll
                                for (int j = 0; j < 2; ++j) {
                                    const int lim = (pre ? have : own[n][j] - base) - 16 * NW * u;
                                    if (tk0 >= lim) sc[u][n][j] = -INFINITY;
                                    if (tk0 + 8 >= lim) sc[u][n][j + 2] = -INFINITY;
                                }
                    }
                    float high[NT][2];
                    bool rise = false;
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            high[n][j] = m[n][j];
#pragma unroll
                            for (int u = 0; u < U; ++u) high[n][j] = max3(high[n][j], sc[u][n][j], sc[u][n][j + 2]);
                            rise |= !(high[n][j] <= edge[n][j]);     // a NaN too
                        }
                    if (__any_sync(0xffffffffu, rise)) {
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int j = 0; j < 2; ++j) {
                                float top = high[n][j];
#pragma unroll
                                for (int off = 4; off < 32; off <<= 1) top = max3(top, top, __shfl_xor_sync(0xffffffffu, top, off));
                                if (!(top <= edge[n][j])) {          // the same for the column's 8 lanes
                                    const float f = ex2_approx((m[n][j] - top) * c[n][j]);       // 0 where there was none yet
                                    m[n][j] = ref[n][j] = top;
                                    edge[n][j] = top + kP4Margin / c[n][j];
                                    l[n][j] *= f;
#pragma unroll
                                    for (int i = 0; i < MT; ++i) { acc[n][i][j] *= f; acc[n][i][j + 2] *= f; }
                                }
                            }
                    }
                    uint32_t p[U][NT][PIECES][2];
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            float w[4];
#pragma unroll
                            for (int j = 0; j < 2; ++j) {
                                w[j] = ex2_approx(fmaf(sc[u][n][j] - ref[n][j], c[n][j], kP4Shift));
                                w[j + 2] = ex2_approx(fmaf(sc[u][n][j + 2] - ref[n][j], c[n][j], kP4Shift));
                                l[n][j] += w[j] + w[j + 2];
                            }
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                const uint32_t h = halves(w[2 * k], w[2 * k + 1]);
                                p[u][n][0][k] = transposed(h);
                                if constexpr (PIECES == 2) p[u][n][1][k] = transposed(rest(w[2 * k], w[2 * k + 1], h));
                            }
                        }
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const unsigned char* cell = tile + u * NW * C::kBytes + C::kHalf;
                        constexpr int W = D / 64;                    // words of 8 codes a token
                        uint32_t v[4][W], sv[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int tok = (i & 1 ? tv1 : tv0) + (i >> 1) * 8;
                            const unsigned char* y = cell + tok * C::kCodes + g * (W * 4);
                            if constexpr (W == 2) *reinterpret_cast<uint2*>(v[i]) = *reinterpret_cast<const uint2*>(y);
                            else v[i][0] = *reinterpret_cast<const uint32_t*>(y);
                            sv[i] = *(cell + C::kScaleAt + tok * C::kScales + (g * W >> 1));
                        }
                        if (tail) {                                  // whatever lies there: 0 times it would be NaN where it is NaN
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if ((i & 1 ? tv1 : tv0) + (i >> 1) * 8 + 16 * NW * u >= have) sv[i] = 0;
                        }
                        __half2 f0, o0, f1, o1;
                        scale_pair4(sv[1] * consts.f64k + sv[0], consts, &f0, &o0);
                        scale_pair4(sv[3] * consts.f64k + sv[2], consts, &f1, &o1);
#pragma unroll
                        for (int w = 0; w < W; ++w) {
                            uint32_t a0[4], a1[4], a2[4], a3[4];
                            pairs4(__byte_perm(v[0][w], v[1][w], 0x5410), f0, o0, consts, a0);
                            pairs4(__byte_perm(v[0][w], v[1][w], 0x7632), f0, o0, consts, a1);
                            pairs4(__byte_perm(v[2][w], v[3][w], 0x5410), f1, o1, consts, a2);
                            pairs4(__byte_perm(v[2][w], v[3][w], 0x7632), f1, o1, consts, a3);
#pragma unroll
                            for (int i = 0; i < 4; ++i)
#pragma unroll
                                for (int n = 0; n < NT; ++n)
#pragma unroll
                                    for (int k = PIECES - 1; k >= 0; --k) mma_f16(acc[n][w * 4 + i], a0[i], a1[i], a2[i], a3[i], p[u][n][k][0], p[u][n][k][1]);
                        }
                    }
                }
                __syncwarp();
                if (lane == 0) bar_arrive(&sm.empty[s]);
            }
            if (!ok) break;
            // the run's end: the warps' results joined
            if (ns && !(ok = bar_wait(&sm.read, (ns - 1) & 1, &sm.failed))) break;       // the run before has been read
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float sum = l[n][j];
#pragma unroll
                    for (int off = 4; off < 32; off <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
                    const int row = n * 8 + 2 * t + j;
                    if (g == 0) sm.stat[warp][row] = make_float2(m[n][j] * c[n][j], sum);
                    float4* y = reinterpret_cast<float4*>(&sm.join[warp][row][g * (D / 8)]);
#pragma unroll
                    for (int i = 0; i < MT; i += 2) y[i / 2] = make_float4(acc[n][i][j], acc[n][i][j + 2], acc[n][i + 1][j], acc[n][i + 1][j + 2]);
                }
            __syncwarp();
            if (lane == 0) bar_arrive(&sm.joined);
            if (!(ok = bar_wait(&sm.joined, ns & 1, &sm.failed))) break;
            const bool bad = *reinterpret_cast<const volatile int*>(&r.bad) != 0;
            for (int row = warp; row < rows; row += NW) {
                float M = -INFINITY, L = 0.f, z[D / 32];
#pragma unroll
                for (int i = 0; i < D / 32; ++i) z[i] = 0.f;
#pragma unroll
                for (int k = 0; k < NW; ++k) { const float y = sm.stat[k][row].x; M = max3(M, y, y); }
                const float base = M == -INFINITY ? 0.f : M;
#pragma unroll
                for (int k = 0; k < NW; ++k) {
                    const float2 st = sm.stat[k][row];
                    const float f = ex2_approx(st.x - base);
                    L = fmaf(st.y, f, L);
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) z[i] = fmaf(sm.join[k][row][lane * (D / 32) + i], f, z[i]);
                }
                // every score finite, but none of them times the scale: as the other caches, NaN
                if (!(fabsf(M) < INFINITY)) L = M == -INFINITY && L == 0.f ? 0.f : NAN;
                if (bad) L = NAN;
                const int gr = r.ru * RU + row, tok = r.tok0 + (gr >> a.g_shift), head = (r.head << a.g_shift) + (gr & ((1 << a.g_shift) - 1));
                if (r.direct) {
                    Entry ee;
                    ee.S = r.S; ee.nq = r.nq;
                    const float f = 8.f * plan.inverse(L, r.P, ee, gr);
                    T* y = (T*)a.o.p + tok * a.o.ts + head * a.o.hs + lane * (D / 32);
                    if constexpr (sizeof(T) == 4) {
                        if constexpr (D == 128) *reinterpret_cast<float4*>(y) = make_float4(z[0] * f, z[1] * f, z[2] * f, z[3] * f);
                        else *reinterpret_cast<float2*>(y) = make_float2(z[0] * f, z[1] * f);
                    } else {
#pragma unroll
                        for (int i = 0; i < D / 64; ++i) reinterpret_cast<__nv_bfloat162*>(y)[i] = __floats2bfloat162_rn(z[2 * i] * f, z[2 * i + 1] * f);
                    }
                } else {
                    const int at = r.slot + row;
                    float* y = a.part + (long long)at * D + lane * (D / 32);
                    if constexpr (D == 128) *reinterpret_cast<float4*>(y) = make_float4(z[0] * 8.f, z[1] * 8.f, z[2] * 8.f, z[3] * 8.f);
                    else *reinterpret_cast<float2*>(y) = make_float2(z[0] * 8.f, z[1] * 8.f);
                    if (lane == 0) a.stat[at] = make_float2(M, L);
                }
            }
            __syncwarp();
            if (lane == 0) { bar_arrive(&sm.read); bar_arrive(&sm.run_empty[slot]); }
            ++ns;
        }
    }
    __syncthreads();
    if (tid == 0 && sm.failed) paged_status(P, kStTimeout);
}

}  // namespace sgk
