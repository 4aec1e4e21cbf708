// Paged exact cache: what its kernels share (descriptors, the division of an attention call's work), and the kernel
// that norms and rotates heads and writes new tokens into pages.
#pragma once
#include <stdint.h>

#include <type_traits>

#include "subgen_device.cuh"

namespace sgk {

constexpr int kStTimeout = 4, kStPage = 8, kStSize = 16;     // SUBGEN_ST_TIMEOUT, SUBGEN_ST_PAGE, SUBGEN_ST_SIZE

struct HeadsView {                                    // [tokens, heads, d]: unit stride along d, strides in elements
    void* p;
    long long ts, hs;
};

struct PagedView {
    char *K, *V;                                      // element (page, head, row, x) at page * ps + head * hs + row * ts + x
    long long ps, hs, ts;
    int pages, page_shift, Hkv;
    int B, groups;                                    // sequences; groups of them that share a prefix (0: none do)
    const int *cu_q, *lengths, *table;                // [B+1], [B], [B, table_stride]
    const int *cu_group, *prefix_len, *prefix_table;  // [groups+1], [groups], [groups, prefix_stride]
    int table_stride, prefix_stride;
    int* status;                                      // may be NULL
};

__device__ __forceinline__ void paged_status(const PagedView& P, int bit) {
    if (P.status) atomicOr(P.status, bit);
}

// ---- norms, rotation, append --------------------------------------------------------------------
//
// y = rot(pos, w * x / sqrt(mean(x^2) + eps)) per head, pairs (a, b) -> (a cos - b sin, b cos + a sin); fp32 inside, one
// rounding at the end. The angle of pair i is pos * f_i; f_i comes as word_i = round(f_i / 2pi * 2^64), so pos * word_i
// mod 2^64 is the angle's fraction of a turn, off by 2^-33 of a turn at most for positions below 2^32 (a product in fp32
// would be off by 2^-24 * pos radians). Its top 32 bits, converted to fp32 half turns, go through sincospi: the conversion
// rounds to 24 bits, 2^-26 of a turn near half a turn, as much as fp32 holds of an angle; more would take a second product
// and a correction for each pair (fp32 results are 6.9e-8 from the exact ones, 6.3e-8 with 64-bit angles).
//
// Memory bound: each element is read once and written once (n = 16384, 64 heads, d = 128, bf16: 537 MB, floor 83 us).
// A row (one head of one token) is held by D / 16 bytes / 2 lanes, each with two 16-byte pieces that contain both
// members of its pairs, so the rotation needs no exchange and the norm a few shuffles. A warp stays with one token and
// walks over its heads: the sines are computed once per token and lane, and the loads of U row groups go out before the
// first is used. With few tokens a token's heads are dealt to several warps (`parts`), which repeat the sines but shorten
// the chain; then U = 1. U = 4 in 96 registers: 97 to 102 us for the above by the box (5.3 to 5.5 TB/s), 158 us for 19.7 K
// tokens x 96 heads appended to pages (6.1 TB/s of 6.5 measured for a copy); U = 1 took 132 and 201, U = 2 103 and 162.
struct NormRope {
    HeadsView q, k, v, qo, ko;                        // ko: unless the keys go into pages
    int n, H, Hkv, parts;
    const int* positions;                             // may be NULL when the keys go into pages
    const unsigned long long* words;                  // NULL: no rotation
    int rot, interleaved;
    const void *wq, *wk;                              // NULL: no norm
    float eps;
    int fresh;                                        // qo holds nothing yet: a token that is left out becomes NaN
};

constexpr int kNrThreads = 128;

// Index of the last i in [0, count) with edges[i] <= x, or -1; -2 where edges that are above x come before ones that are
// not. One warp, all lanes get it.
__device__ __forceinline__ int warp_find(const int* edges, int count, int x) {
    int found = 0;
    bool over = false, broken = false;
    for (int i = 0; i < count; i += 32) {
        const int j = i + (threadIdx.x & 31);
        const unsigned below = __ballot_sync(0xffffffffu, j < count && __ldg(edges + j) <= x);
        broken |= (below & (below + 1)) != 0 || (over && below);
        over |= below != 0xffffffffu;
        found += __popc(below);
    }
    return broken ? -2 : found - 1;
}

// The group of sequence b; -1 where none or several claim it. Edges that fall, do not start at 0 or do not end at B set the
// status. One warp, all lanes get it.
__device__ __forceinline__ int warp_group(const PagedView& P, int b) {
    int found = -1, claims = 0;
    bool broken = false;
    for (int i = 0; i < P.groups; i += 32) {
        const int g = i + (threadIdx.x & 31);
        bool mine = false;
        if (g < P.groups) {
            const int e0 = __ldg(P.cu_group + g), e1 = __ldg(P.cu_group + g + 1);
            mine = e0 <= b && b < e1;
            broken |= e1 < e0 || (g == 0 && e0 != 0) || (g == P.groups - 1 && e1 != P.B);
        }
        const unsigned who = __ballot_sync(0xffffffffu, mine);
        claims += __popc(who);
        if (who) found = i + __ffs(who) - 1;
    }
    if (__any_sync(0xffffffffu, broken) && (threadIdx.x & 31) == 0) paged_status(P, kStPage);
    return claims == 1 ? found : -1;
}

template <typename T, int VE>
__device__ __forceinline__ uint4 pack_row(const float* f) {
    uint4 r;
    if constexpr (sizeof(T) == 4) {
        r = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    } else {
        uint32_t* w = &r.x;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * e], f[2 * e + 1]);
            w[e] = *reinterpret_cast<const uint32_t*>(&h);
        }
    }
    return r;
}

template <typename T, int D, bool PAGED, int U>
__global__ void __launch_bounds__(kNrThreads, U > 1 ? 5 : 1) norm_rope_kernel(NormRope a, PagedView P) {
    constexpr int VE = 16 / sizeof(T), LPR = D / VE / 2, RPW = 32 / LPR;
    const int lane = threadIdx.x & 31, l = lane % LPR, sub = lane / LPR;
    const long long w = (long long)blockIdx.x * (kNrThreads / 32) + (threadIdx.x >> 5);
    const int tok = (int)(w / a.parts), part = (int)(w % a.parts);
    if (tok >= a.n) return;

    long long slot = -1;                                             // element offset of the token's row in head 0 of its page
    long long pos = 0;                                               // prefix and own tokens together may pass 2^31
    if constexpr (PAGED) {
        const int b = warp_find(P.cu_q, P.B + 1, tok);
        const int start = b >= 0 && b < P.B ? __ldg(P.cu_q + b) : 0, end = b >= 0 && b < P.B ? __ldg(P.cu_q + b + 1) : 0;
        if (w == 0 && lane == 0 && (__ldg(P.cu_q) < 0 || __ldg(P.cu_q + P.B) > a.n)) paged_status(P, kStPage);    // no token may tell
        auto leave_out = [&]() {                                     // the token: nothing is written
            if (lane == 0) paged_status(P, kStPage);
            if (!a.fresh || !a.q.p) return;
            for (int i = part * 32 + lane; i < a.H * (D / VE); i += a.parts * 32)
                *reinterpret_cast<uint4*>((T*)a.qo.p + tok * a.qo.ts + i / (D / VE) * a.qo.hs + i % (D / VE) * VE) = make_uint4(~0u, ~0u, ~0u, ~0u);
        };
        if (b == -2 || start < 0 || end > a.n) return leave_out();
        if (b < 0 || b >= P.B) return;                               // before the first sequence, behind the last
        const long long place = (long long)__ldg(P.lengths + b) - end + tok, pg = place >> P.page_shift;
        const int own = (int)place;
        if (place >= 0 && pg < P.table_stride) {
            const int id = __ldg(P.table + (long long)b * P.table_stride + pg);
            if (id >= 0 && id < P.pages) slot = (long long)id * P.ps + (long long)(own & ((1 << P.page_shift) - 1)) * P.ts;
        }
        if (slot < 0 && lane == 0) paged_status(P, kStPage);
        pos = own;
        if (a.positions) pos = __ldg(a.positions + tok);
        else if (P.groups && a.words) {                              // its prefix comes before it
            const int g = warp_group(P, b), len = g >= 0 ? __ldg(P.prefix_len + g) : -1;
            if (len < 0 || len > (long long)P.prefix_stride << P.page_shift) return leave_out();     // no position
            pos += len;
        }
    } else {
        if (a.words) pos = __ldg(a.positions + tok);
    }

    // this lane's two pieces; rotated lanes hold pairs l*VE .. l*VE+VE-1
    const int rl = a.words ? a.rot / (2 * VE) : 0;                   // lanes of a row that rotate
    const bool turn = l < rl;
    int ca, cb;                                                      // pieces
    if (!turn || a.interleaved) { ca = 2 * l; cb = 2 * l + 1; }      // also the pieces behind the rotated ones
    else { ca = l; cb = l + rl; }
    float co[VE], si[VE];
    if (turn) {
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            const unsigned long long turns = (unsigned long long)pos * __ldg(a.words + l * VE + e);
            sincospif((float)(int)(turns >> 32) * 4.656612873077393e-10f, &si[e], &co[e]);   // 2^-31: half turns
        }
    }

    // This warp's share of the token's rows, numbered queries, keys, values in steps of RPW.
    const int gq = (a.H + RPW - 1) / RPW, gk = (a.Hkv + RPW - 1) / RPW, total = gq + (PAGED ? 2 : 1) * gk;
    const int per = (total + a.parts - 1) / a.parts, g0 = part * per, g1 = min(total, g0 + per);

    // Groups [lo, hi) of one kind: 0 queries, 1 keys, 2 values.
    auto run = [&](auto kind_, int lo, int hi, const HeadsView& src, T* dst, long long dst_hs, const T* wt) {
        constexpr int KIND = decltype(kind_)::value;
        const int heads = KIND == 0 ? a.H : a.Hkv;
        const T* x = (const T*)src.p + tok * src.ts;
        uint4 wa = make_uint4(0, 0, 0, 0), wb = wa;
        if (KIND < 2 && wt) {
            wa = __ldg(reinterpret_cast<const uint4*>(wt + ca * VE));
            wb = __ldg(reinterpret_cast<const uint4*>(wt + cb * VE));
        }
        for (int g = lo; g < hi; g += U) {
            uint4 ra[U], rb[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {                            // all loads first
                const int h = (g + u) * RPW + sub;
                ra[u] = rb[u] = make_uint4(0, 0, 0, 0);
                if (g + u < hi && h < heads) {
                    ra[u] = *reinterpret_cast<const uint4*>(x + h * src.hs + ca * VE);
                    rb[u] = *reinterpret_cast<const uint4*>(x + h * src.hs + cb * VE);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int h = (g + u) * RPW + sub;
                if (KIND < 2 && (wt || turn)) {                      // else the bits go through as they are
                    float xa[VE], xb[VE];
                    Elem<T>::unpack(ra[u], xa);
                    Elem<T>::unpack(rb[u], xb);
                    if (wt) {
                        float ss = 0.f;
#pragma unroll
                        for (int e = 0; e < VE; ++e) ss = fmaf(xa[e], xa[e], fmaf(xb[e], xb[e], ss));
#pragma unroll
                        for (int off = LPR / 2; off > 0; off >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, off);
                        const float r = rsqrtf(ss * (1.f / D) + a.eps);
                        float fa[VE], fb[VE];
                        Elem<T>::unpack(wa, fa);
                        Elem<T>::unpack(wb, fb);
#pragma unroll
                        for (int e = 0; e < VE; ++e) { xa[e] *= r * fa[e]; xb[e] *= r * fb[e]; }
                    }
                    if (turn) {
                        if (a.interleaved) {
#pragma unroll
                            for (int e = 0; e < VE / 2; ++e) {
                                const float p0 = xa[2 * e], p1 = xa[2 * e + 1], r0 = xb[2 * e], r1 = xb[2 * e + 1];
                                xa[2 * e] = p0 * co[e] - p1 * si[e];
                                xa[2 * e + 1] = p1 * co[e] + p0 * si[e];
                                xb[2 * e] = r0 * co[VE / 2 + e] - r1 * si[VE / 2 + e];
                                xb[2 * e + 1] = r1 * co[VE / 2 + e] + r0 * si[VE / 2 + e];
                            }
                        } else {
#pragma unroll
                            for (int e = 0; e < VE; ++e) {
                                const float p0 = xa[e], p1 = xb[e];
                                xa[e] = p0 * co[e] - p1 * si[e];
                                xb[e] = p1 * co[e] + p0 * si[e];
                            }
                        }
                    }
                    ra[u] = pack_row<T, VE>(xa);
                    rb[u] = pack_row<T, VE>(xb);
                }
                if (g + u < hi && h < heads) {
                    *reinterpret_cast<uint4*>(dst + h * dst_hs + ca * VE) = ra[u];
                    *reinterpret_cast<uint4*>(dst + h * dst_hs + cb * VE) = rb[u];
                }
            }
        }
    };
    if (a.q.p) run(std::integral_constant<int, 0>(), g0, min(g1, gq), a.q, (T*)a.qo.p + tok * a.qo.ts, a.qo.hs, (const T*)a.wq);
    if (a.k.p && (!PAGED || slot >= 0))
        run(std::integral_constant<int, 1>(), max(g0 - gq, 0), min(g1 - gq, gk), a.k, PAGED ? (T*)P.K + slot : (T*)a.ko.p + tok * a.ko.ts,
            PAGED ? P.hs : a.ko.hs, (const T*)a.wk);
    if (PAGED && slot >= 0)
        run(std::integral_constant<int, 2>(), max(g0 - gq - gk, 0), g1 - gq - gk, a.v, (T*)P.V + slot, P.hs, (const T*)nullptr);
}

// ---- the division of an attention call's work ---------------------------------------------------
//
// out = softmax(scale q [Kp; Ko]^T) [Vp; Vo]: every query row (a new token's head) sees its group's prefix p in full and
// of its sequence's own tokens o those up to its own position (causal) or all. Entries of the plan, per KV head:
// groups first (their prefix against the rows of all their sequences at once: the prefix is read once per row unit),
// then sequences (own tokens against the sequence's rows). An entry's rows (tokens x G heads, in packed order, so a
// group's rows are one range of tokens) are cut into row units of RU rows, each unit's keys into tiles of KT tokens.
// A unit with tiles has weight LEAD (what starting and ending a run costs, in tiles) plus 1 for each tile, or 2 where
// more than half of 128 or 256 rows are in use. All weights of all heads lie on one line; block c takes [c * chunk, (c+1) * chunk)
// of it, so every block has the same work whatever the lengths are, and a unit that several blocks share leaves one
// partial result (numerator, largest score, sum) per block.
// A group folds its prefix into the sequences' entries (own tiles follow the prefix's tiles there) when that costs no
// tensor work: one sequence in it, or at least RU / 2 rows per sequence, so that the row units are full without
// packing several sequences into one; that spares the rows' second partial.
constexpr int kPlanMax = 1024;                        // groups + sequences of one call
constexpr long long kPlanWeight = 1 << 30;            // the line is shorter: of full units 10^13 (query row, key) pairs in bf16,
                                                      // 10^11 where 8 fp32 rows meet 32 tokens

struct Entry {
    int tok0, rows;                                   // first token; rows = tokens * G
    int P, S, nq;                                     // prefix tokens and own tokens to see; new tokens
    const int *ptab, *stab;                           // page tables of the two
    int bad;                                          // a length beyond its page table: the rows become NaN
};
struct Seg {                                          // a run of tiles of one row unit
    Entry e;
    int entry, head, ru, rows, tile0, tile1, tiles, kp;   // rows of the unit; kp: tiles of the prefix
    bool direct;                                      // the unit's whole result: goes to `out` as it is
    int slot;                                         // row of the partials otherwise
};

struct Attend {
    HeadsView q, o;
    int n, H, g_shift, causal;                        // H / Hkv = 1 << g_shift
    float c;                                          // scale * log2(e)
    float* part;                                      // [slots][D] numerators
    float2* stat;                                     // [slots] largest score * c, sum
    int fresh;                                        // o holds nothing yet: NaN where nothing can be computed
};

template <int RU, int KT, int DUAL, int LEAD>
struct Plan {
    const PagedView& P;
    const Attend& a;
    const int* tscan;                                 // [E+1] weights before each entry, per head
    const int* sscan;                                 // [E+1] partial slots before each entry, per head
    int E;
    int head_w, total, chunk;
    int broken;                                       // nothing is computed: 1 cu_q or cu_group is not what it has to be, 2 a line too long

    __device__ Plan(const PagedView& P_, const Attend& a_) : P(P_), a(a_) {}

    __device__ __forceinline__ bool folds(int g, int* t0, int* t1) const {
        const int b0 = min(max(__ldg(P.cu_group + g), 0), P.B), b1 = min(max(__ldg(P.cu_group + g + 1), 0), P.B);
        *t0 = __ldg(P.cu_q + b0);
        *t1 = __ldg(P.cu_q + b1);
        return b1 - b0 <= 1 || (((long long)*t1 - *t0) << a.g_shift) >= (long long)(b1 - b0) * (RU / 2);
    }
    __device__ __forceinline__ int clipped(int len, int stride, int* bad) const {
        const long long cap = (long long)stride << P.page_shift;
        if (len < 0 || len > cap) { *bad = 1; return len < 0 ? 0 : (int)cap; }
        return len;
    }
    __device__ __forceinline__ int group_of(int b) const {
        int lo = 0, hi = P.groups - 1;
#pragma unroll 1
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (__ldg(P.cu_group + mid) <= b) lo = mid; else hi = mid - 1;
        }
        return lo;
    }
    __device__ __forceinline__ Entry entry(int i) const {
        Entry e;
        e.bad = 0;
        e.ptab = e.stab = nullptr;
        if (i < P.groups) {
            int t0, t1;
            const bool f = folds(i, &t0, &t1);
            e.tok0 = t0;
            e.nq = t1 - t0;
            e.rows = f ? 0 : e.nq << a.g_shift;
            e.P = clipped(__ldg(P.prefix_len + i), P.prefix_stride, &e.bad);
            e.S = 0;
            e.ptab = P.prefix_table + (long long)i * P.prefix_stride;
            return e;
        }
        const int b = i - P.groups;
        e.tok0 = __ldg(P.cu_q + b);
        e.nq = __ldg(P.cu_q + b + 1) - e.tok0;
        e.rows = e.nq << a.g_shift;
        e.P = 0;
        e.S = clipped(__ldg(P.lengths + b), P.table_stride, &e.bad);
        e.stab = P.table + (long long)b * P.table_stride;
        if (P.groups) {
            const int g = group_of(b);
            int t0, t1;
            if (folds(g, &t0, &t1)) {
                e.P = clipped(__ldg(P.prefix_len + g), P.prefix_stride, &e.bad);
                e.ptab = P.prefix_table + (long long)g * P.prefix_stride;
            }
        }
        return e;
    }
    // Units of up to 128 rows, whose tiles two groups of a block share, leave two partials (DUAL 1), or one where the block
    // joins them (DUAL 2: units of up to 32 rows).
    __device__ static __forceinline__ int twice(int rows) { return DUAL && rows <= RU / 2 && (DUAL == 1 || rows > 32) ? 1 : 0; }
    // own tokens that row r of an entry sees
    __device__ __forceinline__ int own_limit(const Entry& e, int r) const {
        if (!a.causal) return e.S;
        const int lim = e.S - e.nq + 1 + (r >> a.g_shift);
        return lim < 0 ? 0 : lim > e.S ? e.S : lim;
    }
    // 1 / sum of row r, which sees `prefix` tokens before its own. A sum of 0: nothing to see, and the result is 0, or nothing
    // but scores of -infinity, and it is NaN as the formula's.
    __device__ __forceinline__ float inverse(float sum, int prefix, const Entry& e, int r) const {
        if (sum == 0.f) return prefix > 0 || own_limit(e, r) > 0 ? NAN : 0.f;
        return 1.f / sum;
    }
    __device__ __forceinline__ int unit_rows(const Entry& e, int ru) const { return min(RU, e.rows - ru * RU); }
    __device__ __forceinline__ int prefix_tiles(const Entry& e) const { return (e.P + KT - 1) / KT; }
    __device__ __forceinline__ int unit_tiles(const Entry& e, int ru) const {
        const int last = min(e.rows, (ru + 1) * RU) - 1;
        return prefix_tiles(e) + (own_limit(e, last) + KT - 1) / KT;
    }
    __device__ static __forceinline__ int shift(int rows) { return RU >= 128 && rows > RU / 2 ? 1 : 0; }     // a tile weighs 1 << shift
    __device__ __forceinline__ int unit_weight(int tiles, int rows) const { return tiles ? LEAD + (tiles << shift(rows)) : 0; }
    // tiles of a unit before position p of its weight
    __device__ static __forceinline__ int tile_at(int p, int sh) { return p <= LEAD ? 0 : (p - LEAD + sh) >> sh; }

    // All threads of the block. sm: 8 bytes for each of E + 1; flag: one int of shared memory.
    __device__ void build(void* sm, int* flag, int nblk) {
        E = P.groups + P.B;
        int* t = (int*)sm;
        int* s = t + E + 1;
        // entry() reads these one after the other: asked for at once, so that it finds them in L1
        auto touch = [](const int* p) { int x; asm volatile("ld.global.nc.b32 %0, [%1];" : "=r"(x) : "l"(p)); };
#pragma unroll 1
        for (int b = threadIdx.x; b < P.B; b += blockDim.x) { touch(P.cu_q + b); touch(P.lengths + b); }
#pragma unroll 1
        for (int g = threadIdx.x; g < P.groups; g += blockDim.x) { touch(P.cu_group + g); touch(P.prefix_len + g); }
        if (threadIdx.x == 0) *flag = 0;
        __syncthreads();
#pragma unroll 1
        for (int i = threadIdx.x; i < E; i += blockDim.x) {
            const Entry e = entry(i);
            // a group's rows too: the loop below is as long as they are many
            bool bad = e.tok0 < 0 || e.nq < 0 || (long long)e.tok0 + e.nq > a.n;
            if (i < P.groups) {
                const int b0 = __ldg(P.cu_group + i), b1 = __ldg(P.cu_group + i + 1);
                bad |= b0 < 0 || b1 < b0 || b1 > P.B || (i == 0 && b0 != 0) || (i == P.groups - 1 && b1 != P.B);
            }
            long long w = 0;
            int sl = 0;
            if (bad) *flag = 1;
            else {
#pragma unroll 1
                for (int ru = 0; ru * RU < e.rows; ++ru) {
                    const int rows = unit_rows(e, ru);
                    w += unit_weight(unit_tiles(e, ru), rows);
                    sl = ru * RU + (rows << twice(rows));
                }
            }
            t[i + 1] = (int)(w > kPlanWeight ? kPlanWeight : w);
            s[i + 1] = sl;
        }
        __syncthreads();
        if (threadIdx.x < 32) {
            // Sums that stay at kPlanWeight once they reach it. A lane has `per` entries in a row (an odd number, so that the lanes
            // are in different banks). Loops as they stand: a block starts with no code in its caches, and each new 128 bytes of
            // it (8 instructions) cost over 300 cycles; unrolled, 32 entries at a time, this took 3500 to 11000.
            const int lane = threadIdx.x, per = (E + 31) / 32 | 1, i0 = lane * per, i1 = min(E, i0 + per);
            unsigned x = 0, y = 0;
#pragma unroll 1
            for (int i = i0; i < i1; ++i) { x = min(x + t[i + 1], (unsigned)kPlanWeight); y += s[i + 1]; }
            unsigned at = x, as = y;
#pragma unroll 1
            for (int off = 1; off < 32; off <<= 1) {
                const unsigned xo = __shfl_up_sync(0xffffffffu, at, off), yo = __shfl_up_sync(0xffffffffu, as, off);
                at = lane >= off ? min(at + xo, (unsigned)kPlanWeight) : at;
                as += lane >= off ? yo : 0;
            }
            const unsigned all = __shfl_sync(0xffffffffu, at, 31);
            at = __shfl_up_sync(0xffffffffu, at, 1);
            as -= y;
            if (lane == 0) at = 0;
#pragma unroll 1
            for (int i = i0; i < i1; ++i) {
                at = min(at + t[i + 1], (unsigned)kPlanWeight);
                as += s[i + 1];
                t[i + 1] = (int)at;
                s[i + 1] = (int)as;
            }
            if (lane == 0) {
                t[0] = s[0] = 0;
                if (!*flag && (long long)all * P.Hkv >= kPlanWeight) *flag = 2;
            }
        }
        __syncthreads();
        broken = *flag;
        tscan = t;
        sscan = s;
        head_w = broken ? 0 : t[E];
        total = head_w * P.Hkv;
        chunk = total ? (total + nblk - 1) / nblk : 1;
    }
    __device__ __forceinline__ int slot_of(int i, int ru, int h, int blk) const {
        return h * sscan[E] + sscan[i] + ru * RU + blk * RU;
    }
    __device__ __forceinline__ bool is_direct(const Entry& e, int i, int rows, int tiles) const {
        if (i < P.groups || (P.groups && !e.ptab)) return false;     // partials of the group's entry join in
        return tiles == 1 || !twice(rows);
    }
    // The run of tiles that starts at x (< x1 <= total) on the line; moves x behind it. May be empty (tile0 == tile1).
    __device__ Seg next(int& x, int x1, int blk) const {
        Seg g;
        g.head = x / head_w;
        int r = x - g.head * head_w;
        int lo = 0, hi = E - 1;
#pragma unroll 1
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (tscan[mid] <= r) lo = mid; else hi = mid - 1;
        }
        g.entry = lo;
        r -= tscan[lo];
        g.e = entry(lo);
        g.kp = prefix_tiles(g.e);
        int ru = 0, w;
#pragma unroll 1
        while (true) {
            g.rows = unit_rows(g.e, ru);
            g.tiles = unit_tiles(g.e, ru);
            w = unit_weight(g.tiles, g.rows);
            if (r < w) break;
            r -= w;
            ++ru;
        }
        g.ru = ru;
        const int take = min(x1 - x, w - r), sh = shift(g.rows);
        g.tile0 = tile_at(r, sh);
        g.tile1 = tile_at(r + take, sh);
        x += take;
        g.direct = g.tile0 == 0 && g.tile1 == g.tiles && is_direct(g.e, g.entry, g.rows, g.tiles);
        g.slot = slot_of(g.entry, ru, g.head, blk);
        return g;
    }
};

// Joins the partials of every row that has some (rows whose result went out directly are left alone) and writes 0 for
// rows that see nothing, NaN for rows of a sequence whose lengths or pages are unusable. An item is up to `part` rows of a row
// unit of a sequence and KV head; a block's threads first sort out its items that have anything to join (most prompt rows
// do not), which needs the plan alone and so runs while the attention kernel's last blocks finish. A row's partials are
// dealt to WPR warps (as many as the block has left for the item's rows, so that one sequence's long list is read by all
// of them); a lane looks after one partial's weight, then the warp adds the numerators, and the warps of a row join
// through shared memory. Latency, not bandwidth, is what counts here: one pass over the own and the prefix partials
// together, and registers for three blocks an SM.
constexpr int kMergeThreads = 256, kMergeBlocks = 3;

// All rows of an output. Out of line: no part of what the kernel's code caches hold.
template <typename T, int D>
__device__ __noinline__ void fill_nan(T* o, long long ts, long long hs, int n, int H) {
    constexpr int PIECES = D * (int)sizeof(T) / 16;
    const long long count = (long long)n * H * PIECES, step = (long long)gridDim.x * blockDim.x;
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < count; i += step) {
        const long long row = i / PIECES;
        *reinterpret_cast<uint4*>(o + row / H * ts + row % H * hs + i % PIECES * (16 / (int)sizeof(T))) = make_uint4(~0u, ~0u, ~0u, ~0u);
    }
}

template <typename T, int D, int RU, int KT, int DUAL, int LEAD>
__global__ void __launch_bounds__(kMergeThreads, kMergeBlocks) paged_merge_kernel(PagedView P, Attend a, int nblk, int part) {
    constexpr int NW = kMergeThreads / 32, VL = D / 32;
    extern __shared__ __align__(16) unsigned char sm_plan[];
    __shared__ int flag, units;
    __shared__ int4 todo[kMergeThreads];              // head, sequence, first row, where its unit starts on the line
    __shared__ int todo_warp[NW];
    __shared__ float join[NW][D];
    __shared__ float2 join_stat[NW];
    typedef Plan<RU, KT, DUAL, LEAD> PlanT;
    PlanT plan(P, a);
    plan.build(sm_plan, &flag, nblk);
    int* uscan = (int*)sm_plan + 2 * (plan.E + 1);    // [B+1] parts before each sequence
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (plan.broken) {
        if (blockIdx.x == 0 && tid == 0) paged_status(P, plan.broken == 2 ? kStSize : kStPage);
        pdl_wait();                                   // this kernel's end stands for the attention kernel's
        if (a.fresh) fill_nan<T, D>((T*)a.o.p, a.o.ts, a.o.hs, a.n, a.H);
        return;
    }
    if (warp == 0) {
        const int per = (P.B + 31) / 32 | 1, b0 = lane * per, b1 = min(P.B, b0 + per);
        int x = 0;
#pragma unroll 1
        for (int b = b0; b < b1; ++b) {
            const int y = (((__ldg(P.cu_q + b + 1) - __ldg(P.cu_q + b)) << a.g_shift) + part - 1) / part;
            uscan[b + 1] = y;
            x += y;
        }
        int at = x;
#pragma unroll 1
        for (int off = 1; off < 32; off <<= 1) {
            const int xo = __shfl_up_sync(0xffffffffu, at, off);
            if (lane >= off) at += xo;
        }
        if (lane == 31) units = at;
        at -= x;
#pragma unroll 1
        for (int b = b0; b < b1; ++b) { at += uscan[b + 1]; uscan[b + 1] = at; }
        if (lane == 0) uscan[0] = 0;
    }
    __syncthreads();
    const int items = units * P.Hkv, chunk = plan.chunk;
    // first position of the line that belongs to row unit ru of a sequence's entry
    auto unit_start = [&](const Entry& e, int ei, int h, int ru) {
        int u0 = h * plan.head_w + plan.tscan[ei];
#pragma unroll 1
        for (int k = 0; k < ru; ++k) u0 += plan.unit_weight(plan.unit_tiles(e, k), RU);
        return u0;
    };
    bool waited = false;
    for (int first = 0; first * gridDim.x + blockIdx.x < items; first += kMergeThreads) {
        bool need = false;
        const int mine = (first + tid) * gridDim.x + blockIdx.x;
        int4 what = make_int4(0, 0, 0, 0);
        if (mine < items) {
            const int h = mine / units, u = mine - h * units;
            int lo = 0, hi = P.B - 1;
#pragma unroll 1
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (uscan[mid] <= u) lo = mid; else hi = mid - 1;
            }
            const int b = lo, row0 = (u - uscan[lo]) * part, ei = P.groups + b, ru = row0 / RU;
            const Entry e = plan.entry(ei);
            const int rows = plan.unit_rows(e, ru), tiles = plan.unit_tiles(e, ru), w = plan.unit_weight(tiles, rows), u0 = unit_start(e, ei, h, ru);
            // a direct unit went out whole if the block that holds its first tile also holds the last
            need = !tiles || !plan.is_direct(e, ei, rows, tiles) ||
                   PlanT::tile_at(min(((u0 + LEAD) / chunk + 1) * chunk, u0 + w) - u0, PlanT::shift(rows)) != tiles;
            what = make_int4(h, b, row0, u0);
        }
        const unsigned some = __ballot_sync(0xffffffffu, need);
        __syncthreads();                                             // the list before this one is done with
        if (lane == 0) todo_warp[warp] = __popc(some);
        __syncthreads();
        int before = 0, count = 0;
        for (int k = 0; k < NW; ++k) { before += k < warp ? todo_warp[k] : 0; count += todo_warp[k]; }
        if (need) todo[before + __popc(some & ((1u << lane) - 1u))] = what;
        __syncthreads();
        if (!waited) { pdl_wait(); waited = true; }
        for (int it = 0; it < count; ++it) {
            const int h = todo[it].x, b = todo[it].y, row0 = todo[it].z, u0 = todo[it].w;
            const int ei = P.groups + b, ru = row0 / RU;
            const Entry e = plan.entry(ei);
            const int rows = plan.unit_rows(e, ru), tiles = plan.unit_tiles(e, ru), w = plan.unit_weight(tiles, rows), sh = PlanT::shift(rows);
            const int c0 = u0 / chunk, c1 = w ? (u0 + w - 1) / chunk : c0 - 1;
            const int per = PlanT::twice(rows), own = (c1 - c0 + 1) << per;
            int g = -1;
            Entry ge;
            ge.bad = ge.rows = ge.tok0 = ge.P = 0;
            if (P.groups) {
                g = plan.group_of(b);
                ge = plan.entry(g);
                if (!ge.rows) g = -1;                                // folded (or no rows)
            }
            const int bad = e.bad | (g >= 0 ? ge.bad : 0), pt = g >= 0 ? plan.prefix_tiles(ge) : 0;
            if (bad && tid == 0) paged_status(P, kStPage);
            const int rows_begin = row0 - ru * RU, rows_end = min(rows, rows_begin + part), here = rows_end - rows_begin;
            const int wpr = here > 4 ? 1 : here > 2 ? NW / 4 : here > 1 ? NW / 2 : NW;      // warps per row
            for (int r0 = rows_begin; r0 < rows_end; r0 += NW / wpr) {
                const int r = r0 + warp / wpr, sub = warp % wpr;
                float acc[VL], m = -INFINITY, l = 0.f;
#pragma unroll
                for (int j = 0; j < VL; ++j) acc[j] = 0.f;
                if (r < rows_end) {
                    // partials: 1 or 2 (`per`) of every block of the unit's, then of the prefix's run on the line
                    int v0 = 0, vw = 0, vrows = RU, vper = 0, vc = 0, vslot = 0, all = own;
                    if (pt) {
                        const int prow = ru * RU + r + ((e.tok0 - ge.tok0) << a.g_shift), pru = prow / RU;
                        vrows = plan.unit_rows(ge, pru);
                        vw = plan.unit_weight(pt, vrows);
                        v0 = h * plan.head_w + plan.tscan[g] + pru * plan.unit_weight(pt, RU);
                        vper = PlanT::twice(vrows);
                        vc = v0 / chunk;
                        vslot = plan.slot_of(g, pru, h, 0) + prow - pru * RU;
                        all += ((v0 + vw - 1) / chunk - vc + 1) << vper;
                    }
                    const int oslot = plan.slot_of(ei, ru, h, 0) + r;
#pragma unroll 1
                    for (int i0 = 0; i0 < all; i0 += wpr * 32) {
                        const int i = i0 + lane * wpr + sub;
                        const bool pre = i >= own;
                        const int k = pre ? i - own : i, p = pre ? vper : per, c = (pre ? vc : c0) + (k >> p), second = k & ((1 << p) - 1);
                        const int z0 = pre ? v0 : u0, zw = pre ? vw : w, zrows = pre ? vrows : rows, zsh = PlanT::shift(zrows);
                        const int t0 = PlanT::tile_at(max(c * chunk, z0) - z0, zsh), t1 = PlanT::tile_at(min((c + 1) * chunk, z0 + zw) - z0, zsh);
                        const bool have = i < all && t1 - t0 > second;
                        const int slot = (pre ? vslot : oslot) + c * RU + (second ? zrows : 0);
                        float2 st = make_float2(-INFINITY, 0.f);
                        if (have) st = __ldcg(a.stat + slot);
                        float top = st.x;
#pragma unroll 1
                        for (int off = 16; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
                        const float mn = fmaxf(m, top), bs = mn == -INFINITY ? 0.f : mn, al = exp2f(m - bs);
                        const float f = have ? exp2f(st.x - bs) : 0.f;
                        float sum = have ? st.y * f : 0.f;
#pragma unroll 1
                        for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
                        m = mn;
                        l = l * al + sum;
#pragma unroll
                        for (int j = 0; j < VL; ++j) acc[j] *= al;
                        unsigned left = __ballot_sync(0xffffffffu, have);
                        // W numerators, all loads in flight
                        auto add = [&](auto width) {
                            constexpr int W = decltype(width)::value;
                            float x[W][VL], fx[W];
#pragma unroll
                            for (int q = 0; q < W; ++q) {
                                const int src = left ? __ffs(left) - 1 : -1;
                                left &= left - 1;
                                const int s = __shfl_sync(0xffffffffu, slot, src & 31);
                                fx[q] = __shfl_sync(0xffffffffu, f, src & 31);
                                if (src < 0) fx[q] = 0.f;
#pragma unroll
                                for (int j = 0; j < VL; ++j) x[q][j] = 0.f;
                                if (src >= 0) {
                                    const float* y = a.part + (long long)s * D + lane * VL;
                                    if constexpr (VL == 4) {
                                        const float4 v = __ldcg(reinterpret_cast<const float4*>(y));
                                        x[q][0] = v.x; x[q][1] = v.y; x[q][2] = v.z; x[q][3] = v.w;
                                    } else {
                                        const float2 v = __ldcg(reinterpret_cast<const float2*>(y));
                                        x[q][0] = v.x; x[q][1] = v.y;
                                    }
                                }
                            }
#pragma unroll
                            for (int q = 0; q < W; ++q)
#pragma unroll
                                for (int j = 0; j < VL; ++j) acc[j] = fmaf(x[q][j], fx[q], acc[j]);
                        };
                        while (left) {
                            if (__popc(left) > 3) add(std::integral_constant<int, 8>());
                            else add(std::integral_constant<int, 3>());
                        }
                    }
                }
                if (wpr > 1) {
                    __syncthreads();
                    if (lane == 0) join_stat[warp] = make_float2(m, l);
#pragma unroll
                    for (int j = 0; j < VL; ++j) join[warp][lane * VL + j] = acc[j];
                    __syncthreads();
                    float mm = -INFINITY;
#pragma unroll 1
                    for (int k = 0; k < wpr; ++k) mm = fmaxf(mm, join_stat[warp - sub + k].x);
                    const float bs = mm == -INFINITY ? 0.f : mm;
                    l = 0.f;
#pragma unroll
                    for (int j = 0; j < VL; ++j) acc[j] = 0.f;
#pragma unroll 1
                    for (int k = 0; k < wpr; ++k) {
                        const float2 st = join_stat[warp - sub + k];
                        const float f = exp2f(st.x - bs);
                        l = fmaf(st.y, f, l);
#pragma unroll
                        for (int j = 0; j < VL; ++j) acc[j] = fmaf(join[warp - sub + k][lane * VL + j], f, acc[j]);
                    }
                }
                if (r >= rows_end || sub) continue;
                const int row = ru * RU + r;
                float inv = 1.f / l;                                 // l is NaN where a page was unusable
                if (__builtin_expect(l == 0.f, 0)) {
                    int b2 = b;                                      // told anew, so that nothing is kept for it
                    asm volatile("" : "+r"(b2));
                    const Entry e2 = plan.entry(P.groups + b2);
                    inv = plan.inverse(l, P.groups ? __ldg(P.prefix_len + plan.group_of(b2)) : 0, e2, row);
                }
                if (bad) inv = NAN;
                const int tok = e.tok0 + (row >> a.g_shift), head = (h << a.g_shift) + (row & ((1 << a.g_shift) - 1));
                T* y = (T*)a.o.p + tok * a.o.ts + head * a.o.hs + lane * VL;
                if constexpr (sizeof(T) == 4) {
                    if constexpr (VL == 4) *reinterpret_cast<float4*>(y) = make_float4(acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
                    else *reinterpret_cast<float2*>(y) = make_float2(acc[0] * inv, acc[1] * inv);
                } else {
#pragma unroll
                    for (int j = 0; j < VL / 2; ++j)
                        reinterpret_cast<__nv_bfloat162*>(y)[j] = __floats2bfloat162_rn(acc[2 * j] * inv, acc[2 * j + 1] * inv);
                }
            }
        }
    }
    if (!waited) pdl_wait();
}

}  // namespace sgk
