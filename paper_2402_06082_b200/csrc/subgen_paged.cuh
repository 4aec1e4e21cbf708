// Paged exact cache: what its kernels share (descriptors, the division of an attention call's work), and the kernel
// that norms and rotates heads and writes new tokens into pages.
#pragma once
#include <stdint.h>

#include "subgen_device.cuh"

namespace sgk {

constexpr int kStTimeout = 4, kStPage = 8;            // SUBGEN_ST_TIMEOUT, SUBGEN_ST_PAGE

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
// mod 2^64 is the angle's fraction of a turn, exact to 2^-33 of a turn for every 31-bit position (a product in fp32
// would be off by 2^-24 * pos radians), and the top 32 bits go through sincospi.
//
// Memory bound: each element is read once and written once (n = 16384, 64 heads, d = 128, bf16: 537 MB, floor 83 us).
// A row (one head of one token) is held by D / 16 bytes / 2 lanes, each with two 16-byte pieces that contain both
// members of its pairs, so the rotation needs no exchange and the norm a few shuffles. A warp stays with one token and
// walks over its heads: the sines are computed once per token and lane. With few tokens a token's heads are dealt to
// several warps (`parts`), which repeat the sines but shorten the chain.
struct NormRope {
    HeadsView q, k, v, qo, ko;                        // ko: unless the keys go into pages
    int n, H, Hkv, parts;
    const int* positions;                             // may be NULL when the keys go into pages
    const unsigned long long* words;                  // NULL: no rotation
    int rot, interleaved;
    const void *wq, *wk;                              // NULL: no norm
    float eps;
};

constexpr int kNrThreads = 256;

// index of the last i in [0, count) with edges[i] <= x, or -1; edges non-decreasing. One warp, all lanes get it.
__device__ __forceinline__ int warp_find(const int* edges, int count, int x) {
    int found = 0;
    for (int i = 0; i < count; i += 32) {
        const int j = i + (threadIdx.x & 31);
        found += __popc(__ballot_sync(0xffffffffu, j < count && __ldg(edges + j) <= x));
    }
    return found - 1;
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

template <typename T, int D, bool PAGED>
__global__ void __launch_bounds__(kNrThreads) norm_rope_kernel(NormRope a, PagedView P) {
    constexpr int VE = 16 / sizeof(T), LPR = D / VE / 2, RPW = 32 / LPR;
    const int lane = threadIdx.x & 31, l = lane % LPR, sub = lane / LPR;
    const long long w = (long long)blockIdx.x * (kNrThreads / 32) + (threadIdx.x >> 5);
    const int tok = (int)(w / a.parts), part = (int)(w % a.parts);
    if (tok >= a.n) return;

    long long slot = -1;                                             // element offset of the token's row in head 0 of its page
    int pos = 0;
    if constexpr (PAGED) {
        const int b = warp_find(P.cu_q, P.B + 1, tok);
        if (b < 0 || b >= P.B) return;                               // behind the last sequence
        const int own = __ldg(P.lengths + b) - __ldg(P.cu_q + b + 1) + tok;
        const int pg = own >> P.page_shift;
        if (own >= 0 && pg < P.table_stride) {
            const int id = __ldg(P.table + (long long)b * P.table_stride + pg);
            if (id >= 0 && id < P.pages) slot = (long long)id * P.ps + (long long)(own & ((1 << P.page_shift) - 1)) * P.ts;
        }
        if (slot < 0 && lane == 0) paged_status(P, kStPage);
        pos = own;
        if (a.positions) pos = __ldg(a.positions + tok);
        else if (P.groups) {
            const int g = warp_find(P.cu_group, P.groups + 1, b);
            if (g >= 0 && g < P.groups) pos += __ldg(P.prefix_len + g);
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
            const unsigned long long turns = (unsigned long long)(long long)pos * __ldg(a.words + l * VE + e);
            sincospif((float)(int)(turns >> 32) * 4.656612873077393e-10f, &si[e], &co[e]);   // 2^-31: half turns
        }
    }

    const int heads = a.H + (PAGED ? 2 : 1) * a.Hkv;
    const int per = (heads + a.parts * RPW - 1) / (a.parts * RPW) * RPW;
    const int end = min(heads, (part + 1) * per);
    for (int h0 = part * per; h0 < end; h0 += RPW) {
        const int h = h0 + sub;
        const int kind = h < a.H ? 0 : h < a.H + a.Hkv ? 1 : 2;
        const int hh = kind == 0 ? h : h - a.H - (kind - 1) * a.Hkv;
        const HeadsView& src = kind == 0 ? a.q : kind == 1 ? a.k : a.v;
        const bool live = h < end && src.p != nullptr && (!PAGED || kind == 0 || slot >= 0);
        float xa[VE], xb[VE];
        const T* x = (const T*)src.p + tok * src.ts + hh * src.hs;
        uint4 ra = make_uint4(0, 0, 0, 0), rb = ra;
        if (live) { ra = *reinterpret_cast<const uint4*>(x + ca * VE); rb = *reinterpret_cast<const uint4*>(x + cb * VE); }
        Elem<T>::unpack(ra, xa);
        Elem<T>::unpack(rb, xb);
        const T* wt = (const T*)(kind == 0 ? a.wq : kind == 1 ? a.wk : nullptr);
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < VE; ++e) ss = fmaf(xa[e], xa[e], fmaf(xb[e], xb[e], ss));
#pragma unroll
        for (int off = LPR / 2; off > 0; off >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, off);
        if (wt) {
            const float r = 1.f / sqrtf(ss * (1.f / D) + a.eps);
            float wa[VE], wb[VE];
            Elem<T>::unpack(__ldg(reinterpret_cast<const uint4*>(wt + ca * VE)), wa);
            Elem<T>::unpack(__ldg(reinterpret_cast<const uint4*>(wt + cb * VE)), wb);
#pragma unroll
            for (int e = 0; e < VE; ++e) { xa[e] *= r * wa[e]; xb[e] *= r * wb[e]; }
        }
        if (turn && kind < 2) {
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
        if (!live) continue;
        T* y;
        if (kind == 0) y = (T*)a.qo.p + tok * a.qo.ts + hh * a.qo.hs;
        else if (PAGED) y = (T*)(kind == 1 ? P.K : P.V) + slot + hh * P.hs;
        else y = (T*)a.ko.p + tok * a.ko.ts + hh * a.ko.hs;
        const bool copy = kind == 2 || (!wt && !turn);               // untouched bits go through as they are
        *reinterpret_cast<uint4*>(y + ca * VE) = copy ? ra : pack_row<T, VE>(xa);
        *reinterpret_cast<uint4*>(y + cb * VE) = copy ? rb : pack_row<T, VE>(xb);
    }
}

// ---- the division of an attention call's work ---------------------------------------------------
//
// out = softmax(scale q [Kp; Ko]^T) [Vp; Vo]: every query row (a new token's head) sees its group's prefix p in full and
// of its sequence's own tokens o those up to its own position (causal) or all. Entries of the plan, per KV head:
// groups first (their prefix against the rows of all their sequences at once: the prefix is read once per group),
// then sequences (own tokens against the sequence's rows). An entry's rows (tokens x G heads, in packed order, so a
// group's rows are one range of tokens) are cut into row units of RU rows, each unit's keys into tiles of KT tokens.
// A unit's tiles carry weight 2 when both halves of its rows are in use. All weights of all heads lie on one line;
// block c takes [c * chunk, (c+1) * chunk) of it, so every block has the same work whatever the lengths are, and a
// unit that several blocks share leaves one partial result (numerator, largest score, sum) per block.
// A group folds its prefix into the sequences' entries (own tiles follow the prefix's tiles there) when that costs no
// tensor work: one sequence in it, or at least RU / 2 rows per sequence, so that the row units are full without
// packing several sequences into one; that spares the rows' second partial.
constexpr int kPlanMax = 2048;                        // groups + sequences of one call

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
    long long slot;                                   // row of the partials otherwise
};

struct Attend {
    HeadsView q, o;
    int n, H, G, causal;
    float c;                                          // scale * log2(e)
    float* part;                                      // [slots][D] numerators
    float2* stat;                                     // [slots] largest score * c, sum
    long long slots;
};

template <int RU, int KT, bool DUAL>
struct Plan {
    const PagedView& P;
    const Attend& a;
    const long long* tscan;                           // [E+1] weights before each entry, per head
    const int* sscan;                                 // [E+1] partial slots before each entry, per head
    int E, nblk;
    long long head_w, total, chunk;
    bool broken;                                      // cu_q or cu_group is not what it has to be: nothing is computed

    __device__ Plan(const PagedView& P_, const Attend& a_) : P(P_), a(a_) {}

    __device__ __forceinline__ bool folds(int g, int* b0, int* t0, int* t1) const {
        *b0 = __ldg(P.cu_group + g);
        const int b1 = __ldg(P.cu_group + g + 1);
        *t0 = __ldg(P.cu_q + *b0);
        *t1 = __ldg(P.cu_q + b1);
        return b1 - *b0 <= 1 || (long long)(*t1 - *t0) * a.G >= (long long)(b1 - *b0) * (RU / 2);
    }
    __device__ __forceinline__ int clipped(int len, int stride, int* bad) const {
        const long long cap = (long long)stride << P.page_shift;
        if (len < 0 || len > cap) { *bad = 1; return len < 0 ? 0 : (int)cap; }
        return len;
    }
    __device__ Entry entry(int i) const {
        Entry e;
        e.bad = 0;
        e.ptab = e.stab = nullptr;
        if (i < P.groups) {
            int b0, t0, t1;
            const bool f = folds(i, &b0, &t0, &t1);
            e.tok0 = t0;
            e.nq = t1 - t0;
            e.rows = f ? 0 : e.nq * a.G;
            e.P = clipped(__ldg(P.prefix_len + i), P.prefix_stride, &e.bad);
            e.S = 0;
            e.ptab = P.prefix_table + (long long)i * P.prefix_stride;
            return e;
        }
        const int b = i - P.groups;
        e.tok0 = __ldg(P.cu_q + b);
        e.nq = __ldg(P.cu_q + b + 1) - e.tok0;
        e.rows = e.nq * a.G;
        e.P = 0;
        e.S = clipped(__ldg(P.lengths + b), P.table_stride, &e.bad);
        e.stab = P.table + (long long)b * P.table_stride;
        if (P.groups) {
            const int g = group_of(b);
            int b0, t0, t1;
            if (folds(g, &b0, &t0, &t1)) {
                e.P = clipped(__ldg(P.prefix_len + g), P.prefix_stride, &e.bad);
                e.ptab = P.prefix_table + (long long)g * P.prefix_stride;
            }
        }
        return e;
    }
    __device__ __forceinline__ int group_of(int b) const {
        int lo = 0, hi = P.groups - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (__ldg(P.cu_group + mid) <= b) lo = mid; else hi = mid - 1;
        }
        return lo;
    }
    // own tokens that row r of an entry sees
    __device__ __forceinline__ int own_limit(const Entry& e, int r) const {
        if (!a.causal) return e.S;
        const int lim = e.S - e.nq + 1 + r / a.G;
        return lim < 0 ? 0 : lim > e.S ? e.S : lim;
    }
    __device__ __forceinline__ int unit_rows(const Entry& e, int ru) const { return min(RU, e.rows - ru * RU); }
    __device__ __forceinline__ int prefix_tiles(const Entry& e) const { return (e.P + KT - 1) / KT; }
    __device__ __forceinline__ int unit_tiles(const Entry& e, int ru) const {
        const int last = min(e.rows, (ru + 1) * RU) - 1;
        return prefix_tiles(e) + (own_limit(e, last) + KT - 1) / KT;
    }
    __device__ static __forceinline__ int weight(int rows) { return DUAL && rows > RU / 2 ? 2 : 1; }

    // All threads of the block. sm: 12 bytes for each of E + 1, 8-byte aligned; flag: one int of shared memory.
    __device__ void build(void* sm, int* flag, int nblk_) {
        E = P.groups + P.B;
        nblk = nblk_;
        long long* t = (long long*)sm;
        int* s = (int*)(t + E + 1);
        if (threadIdx.x == 0) *flag = 0;
        __syncthreads();
        bool bad = false;
        for (int b = threadIdx.x; b <= P.B; b += blockDim.x) {
            const int x = __ldg(P.cu_q + b);
            bad |= b == 0 ? x < 0 : x < __ldg(P.cu_q + b - 1);
            bad |= x > a.n;
        }
        for (int g = threadIdx.x; g <= P.groups && P.groups; g += blockDim.x) {
            const int x = __ldg(P.cu_group + g);
            bad |= g == 0 ? x != 0 : x < __ldg(P.cu_group + g - 1);
            bad |= g == P.groups ? x != P.B : x > P.B;
        }
        if (bad) *flag = 1;
        __syncthreads();
        broken = *flag != 0;
        if (!broken) {
            for (int i = threadIdx.x; i < E; i += blockDim.x) {
                const Entry e = entry(i);
                long long w = 0;
                int sl = 0;
                for (int ru = 0; ru * RU < e.rows; ++ru) {
                    const int rows = unit_rows(e, ru);
                    w += (long long)unit_tiles(e, ru) * weight(rows);
                    sl = ru * RU + (DUAL && rows <= RU / 2 ? 2 * rows : rows);
                }
                t[i + 1] = w;
                s[i + 1] = sl;
            }
        }
        __syncthreads();
        if (threadIdx.x < 32 && !broken) {
            long long at = 0;
            int as = 0;
            for (int i0 = 0; i0 < E; i0 += 32) {
                const int i = i0 + (int)threadIdx.x;
                long long x = i < E ? t[i + 1] : 0;
                int y = i < E ? s[i + 1] : 0;
#pragma unroll
                for (int off = 1; off < 32; off <<= 1) {
                    const long long xo = __shfl_up_sync(0xffffffffu, x, off);
                    const int yo = __shfl_up_sync(0xffffffffu, y, off);
                    if ((int)threadIdx.x >= off) { x += xo; y += yo; }
                }
                if (i < E) { t[i + 1] = at + x; s[i + 1] = as + y; }
                at += __shfl_sync(0xffffffffu, x, 31);
                as += __shfl_sync(0xffffffffu, y, 31);
            }
            if (threadIdx.x == 0) { t[0] = 0; s[0] = 0; }
        }
        __syncthreads();
        tscan = t;
        sscan = s;
        head_w = broken ? 0 : t[E];
        total = head_w * P.Hkv;
        chunk = total ? (total + nblk - 1) / nblk : 1;
    }
    // first position of the line that belongs to row unit ru of entry i, head h
    __device__ long long unit_start(const Entry& e, int i, int ru, int h) const {
        long long x = h * head_w + tscan[i];
        for (int k = 0; k < ru; ++k) x += (long long)unit_tiles(e, k) * weight(RU);
        return x;
    }
    __device__ __forceinline__ long long slot_of(int i, int ru, int h, int blk) const {
        return (long long)h * sscan[E] + sscan[i] + (long long)ru * RU + (long long)blk * RU;
    }
    __device__ __forceinline__ bool is_direct(const Entry& e, int i, int rows, int tiles, int tile0, int tile1) const {
        if (tile0 != 0 || tile1 != tiles || i < P.groups) return false;
        if (P.groups && !e.ptab) return false;                       // the prefix's partials come from the group's entry
        return !DUAL || rows > RU / 2 || tiles == 1;
    }
    // The run of tiles that starts at x (< x1 <= total) on the line; moves x behind it. May be empty (tile0 == tile1).
    __device__ Seg next(long long& x, long long x1, int blk) const {
        Seg g;
        g.head = (int)(x / head_w);
        long long r = x - (long long)g.head * head_w;
        int lo = 0, hi = E - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (tscan[mid] <= r) lo = mid; else hi = mid - 1;
        }
        g.entry = lo;
        r -= tscan[lo];
        g.e = entry(lo);
        g.kp = prefix_tiles(g.e);
        int ru = 0, w;
        while (true) {
            g.rows = unit_rows(g.e, ru);
            g.tiles = unit_tiles(g.e, ru);
            w = weight(g.rows);
            if (r < (long long)g.tiles * w) break;
            r -= (long long)g.tiles * w;
            ++ru;
        }
        g.ru = ru;
        const long long left = (long long)g.tiles * w - r;
        const long long take = x1 - x < left ? x1 - x : left;
        g.tile0 = (int)((r + w - 1) / w);
        g.tile1 = (int)((r + take + w - 1) / w);
        x += take;
        g.direct = is_direct(g.e, g.entry, g.rows, g.tiles, g.tile0, g.tile1);
        g.slot = slot_of(g.entry, ru, g.head, blk);
        return g;
    }
};

// Joins the partials of every row that has some (rows whose result went out directly are left alone) and writes 0 for
// rows that see nothing, NaN for rows of a sequence whose lengths or pages are unusable. One block per row unit of a
// sequence and KV head, a warp per row; the largest score first, then one pass over the numerators.
constexpr int kMergeThreads = 256;

template <typename T, int D, int RU, int KT, bool DUAL>
__global__ void __launch_bounds__(kMergeThreads) paged_merge_kernel(PagedView P, Attend a, int nblk) {
    extern __shared__ __align__(16) unsigned char sm_plan[];
    __shared__ int flag;
    __shared__ int units;
    typedef Plan<RU, KT, DUAL> PlanT;
    PlanT plan(P, a);
    plan.build(sm_plan, &flag, nblk);
    int* uscan = (int*)(sm_plan + 12 * (plan.E + 1));  // [B+1] row units before each sequence
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (!plan.broken) {
        for (int b = tid; b < P.B; b += kMergeThreads)
            uscan[b + 1] = ((__ldg(P.cu_q + b + 1) - __ldg(P.cu_q + b)) * a.G + RU - 1) / RU;
    }
    __syncthreads();
    if (warp == 0) {
        int at = 0;
        for (int i0 = 0; i0 < P.B && !plan.broken; i0 += 32) {
            int x = i0 + lane < P.B ? uscan[i0 + lane + 1] : 0;
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                const int xo = __shfl_up_sync(0xffffffffu, x, off);
                if (lane >= off) x += xo;
            }
            if (i0 + lane < P.B) uscan[i0 + lane + 1] = at + x;
            at += __shfl_sync(0xffffffffu, x, 31);
        }
        if (lane == 0) { uscan[0] = 0; units = at; }
    }
    __syncthreads();
    if (plan.broken) {
        if (blockIdx.x == 0 && tid == 0) paged_status(P, kStPage);
        return;
    }
    pdl_wait();
    const int items = units * P.Hkv;
    for (int item = blockIdx.x; item < items; item += gridDim.x) {
        const int h = item / units, u = item % units;
        int lo = 0, hi = P.B - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (uscan[mid] <= u) lo = mid; else hi = mid - 1;
        }
        const int b = lo, ru = u - uscan[lo], ei = P.groups + b;
        const Entry e = plan.entry(ei);
        const int rows = plan.unit_rows(e, ru), tiles = plan.unit_tiles(e, ru), w = PlanT::weight(rows);
        const long long u0 = plan.unit_start(e, ei, ru, h), u1 = u0 + (long long)tiles * w;
        const int c0 = (int)(u0 / plan.chunk);
        int c1 = tiles ? (int)((u1 - 1) / plan.chunk) : c0 - 1;
        if (c1 > c0 && ((long long)c1 * plan.chunk - u0 + w - 1) / w >= tiles) --c1;     // its share is half a tile: the block before did it
        if (c0 == c1 && plan.is_direct(e, ei, rows, tiles, 0, tiles)) continue;
        int g = -1;
        Entry ge;
        if (P.groups) {
            g = plan.group_of(b);
            ge = plan.entry(g);
            if (!ge.rows) g = -1;                                    // folded (or no rows)
        }
        const int bad = e.bad | (g >= 0 ? ge.bad : 0);
        if (bad && lane == 0) paged_status(P, kStPage);
        for (int r = warp; r < rows; r += kMergeThreads / 32) {
            const int row = ru * RU + r, tok = e.tok0 + row / a.G, head = h * a.G + row % a.G;
            float acc[D / 32], m = -INFINITY, l = 0.f;
#pragma unroll
            for (int j = 0; j < D / 32; ++j) acc[j] = 0.f;
            // two passes over the partials: fn(slot)
            auto each = [&](auto fn) {
                for (int c = c0; c <= c1; ++c) {
                    const long long a0 = max((long long)c * plan.chunk, u0) - u0, a1 = min((long long)(c + 1) * plan.chunk, u1) - u0;
                    const int t0 = (int)((a0 + w - 1) / w), t1 = (int)((a1 + w - 1) / w);
                    if (t0 >= t1) continue;
                    const long long s = plan.slot_of(ei, ru, h, c) + r;
                    fn(s);
                    if (DUAL && rows <= RU / 2 && t1 - t0 > 1) fn(s + rows);
                }
                if (g >= 0) {
                    const int prow = row + (e.tok0 - ge.tok0) * a.G, pru = prow / RU, pr = prow % RU;
                    const int prows = plan.unit_rows(ge, pru), pt = plan.prefix_tiles(ge), pw = PlanT::weight(prows);
                    if (pt) {
                        const long long v0 = (long long)h * plan.head_w + plan.tscan[g] + (long long)pru * pt * PlanT::weight(RU);
                        const long long v1 = v0 + (long long)pt * pw;
                        const int d0 = (int)(v0 / plan.chunk), d1 = (int)((v1 - 1) / plan.chunk);
                        for (int c = d0; c <= d1; ++c) {
                            const long long a0 = max((long long)c * plan.chunk, v0) - v0, a1 = min((long long)(c + 1) * plan.chunk, v1) - v0;
                            const int t0 = (int)((a0 + pw - 1) / pw), t1 = (int)((a1 + pw - 1) / pw);
                            if (t0 >= t1) continue;
                            const long long s = plan.slot_of(g, pru, h, c) + pr;
                            fn(s);
                            if (DUAL && prows <= RU / 2 && t1 - t0 > 1) fn(s + prows);
                        }
                    }
                }
            };
            each([&](long long s) { m = fmaxf(m, __ldcg(a.stat + s).x); });
            const float base = m == -INFINITY ? 0.f : m;
            each([&](long long s) {
                const float2 st = __ldcg(a.stat + s);
                const float f = exp2f(st.x - base);
                l += st.y * f;
                if constexpr (D == 128) {
                    const float4 x = __ldcg(reinterpret_cast<const float4*>(a.part + s * D) + lane);
                    acc[0] = fmaf(x.x, f, acc[0]); acc[1] = fmaf(x.y, f, acc[1]); acc[2] = fmaf(x.z, f, acc[2]); acc[3] = fmaf(x.w, f, acc[3]);
                } else {
                    const float2 x = __ldcg(reinterpret_cast<const float2*>(a.part + s * D) + lane);
                    acc[0] = fmaf(x.x, f, acc[0]); acc[1] = fmaf(x.y, f, acc[1]);
                }
            });
            float inv = l == 0.f ? 0.f : 1.f / l;                    // l is NaN where a page was unusable
            if (bad) inv = NAN;
            T* y = (T*)a.o.p + tok * a.o.ts + head * a.o.hs + lane * (D / 32);
            if constexpr (sizeof(T) == 4) {
                if constexpr (D == 128) *reinterpret_cast<float4*>(y) = make_float4(acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
                else *reinterpret_cast<float2*>(y) = make_float2(acc[0] * inv, acc[1] * inv);
            } else {
#pragma unroll
                for (int j = 0; j < D / 64; ++j)
                    reinterpret_cast<__nv_bfloat162*>(y)[j] = __floats2bfloat162_rn(acc[2 * j] * inv, acc[2 * j + 1] * inv);
            }
        }
    }
}

}  // namespace sgk
