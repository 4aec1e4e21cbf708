// Cache in 4-bit cells: tokens by their slots as dense keys and values; and the tables of a step.
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>

#include "subgen_paged.cuh"

namespace sgk {

// ---- load ---------------------------------------------------------------------------------------
//
// Row (token, head, K or V) = d / 2 code bytes and d / 16 scale bytes -> d values of T, exact. Memory bound: 4.5 bits read, 16 or
// 32 written per value. A lane takes 8 values (4 bytes and a scale byte), so that a warp writes whole rows by 16-byte pieces. It
// stays with one head and one of K and V and goes from token to token, kLoadAhead of them at a time, slots two turns ahead and codes
// one: the place of a row among a token's is told once. 32768 tokens x 8 heads x 128 to bf16: 34 us, 5.0 TB/s (rows numbered over all
// tokens, 3 times the instructions, 45; without the turns ahead 39; ordinary stores 35; 5 or 6 blocks an SM 39, 44; a block's tokens
// on end 36).
struct Load4 {
    const char* pool;
    long long ps, hs;                                 // bytes
    const long long* slots;
    int n, Hkv, pages, page_shift;
    int at_once;                                      // tokens that a block takes at a time, where it holds all rows of one
    HeadsView k, v;                                   // p NULL: not wanted
    int* status;
};

constexpr int kLoadThreads = 256, kLoadAhead = 4, kLoadBlocks = 4;

template <typename T, int D>
__global__ void __launch_bounds__(kLoadThreads, kLoadBlocks) paged4_load_kernel(Load4 a) {
    constexpr int LPR = D / 8, RPB = kLoadThreads / LPR;             // lanes a row, rows a block
    const int l = threadIdx.x % LPR, rows = 2 * a.Hkv, row = threadIdx.x / LPR;
    const int mine = row / rows, i = blockIdx.y * RPB + row - mine * rows;       // token of those taken at once; which of its rows
    if (mine >= a.at_once || i >= rows) return;
    const int kv = i >= a.Hkv ? 1 : 0, h = i - kv * a.Hkv;
    const HeadsView& y = kv ? a.v : a.k;
    if (!y.p) return;
    const int step = gridDim.x * a.at_once;                          // from one of this lane's tokens to the next
    int tok = blockIdx.x * a.at_once + mine;
    T* z = (T*)y.p + h * y.hs + tok * y.ts + l * 8;
    const long long z_step = step * y.ts;
    const char* const from = a.pool + h * a.hs + kv * Cell4<D>::kHalf;
    const Consts4Bf16 consts;
    constexpr int A = kLoadAhead;
    long long slot[A];
    uint32_t code[2][A], scale[2][A];
    auto slots = [&](int t) {
#pragma unroll
        for (int u = 0; u < A; ++u) slot[u] = t + u * step < a.n ? __ldg(a.slots + t + u * step) : -1;
    };
    auto codes = [&](int b) {
#pragma unroll
        for (int u = 0; u < A; ++u) {
            code[b][u] = scale[b][u] = 0;                            // a slot below 0: zeros
            const long long page = slot[u] >> a.page_shift;
            if (page >= a.pages) {
                scale[b][u] = 255u;
                if (h == 0 && l == 0 && (!kv || !a.k.p) && a.status) atomicOr(a.status, kStPage);        // once a token, K wanted or not
            } else if (page >= 0) {
                const int id = (int)page, at = (int)slot[u] & ((1 << a.page_shift) - 1);
                const char* cell = from + id * a.ps + (at >> 4) * Cell4<D>::kBytes;
                code[b][u] = __ldcs(reinterpret_cast<const uint32_t*>(cell + (at & 15) * Cell4<D>::kCodes) + l);
                scale[b][u] = __ldg(reinterpret_cast<const unsigned char*>(cell) + Cell4<D>::kScaleAt + (at & 15) * Cell4<D>::kScales + l / 2);
            }
        }
    };
    auto values = [&](int b) {
#pragma unroll
        for (int u = 0; u < A; ++u) {
            if (tok >= a.n) return;
            uint32_t s[2], x[4];
            scale_bf16_4(scale[b][u], 0, s);
            pairs4_bf16(code[b][u], s[0], consts, x);
            if constexpr (sizeof(T) == 4) {
                __stcs(reinterpret_cast<uint4*>(z), make_uint4(x[0] << 16, x[0] & 0xffff0000u, x[1] << 16, x[1] & 0xffff0000u));
                __stcs(reinterpret_cast<uint4*>(z + 4), make_uint4(x[2] << 16, x[2] & 0xffff0000u, x[3] << 16, x[3] & 0xffff0000u));
            } else {
                __stcs(reinterpret_cast<uint4*>(z), make_uint4(x[0], x[1], x[2], x[3]));
            }
            tok += step;
            z += z_step;
        }
    };
    // slots two turns ahead, codes one
    slots(tok);
    codes(0);
    slots(tok + A * step);
    while (tok < a.n) {
        codes(1);
        slots(tok + 2 * A * step);
        values(0);
        if (tok >= a.n) break;
        codes(0);
        slots(tok + 2 * A * step);
        values(1);
    }
}

// ---- the tables of a step -----------------------------------------------------------------------
//
// Row b of the table has ceil(lengths[b] / page) pages. Rows that ended give theirs back to the stack of free pages, in order of
// rows and places; then rows with new tokens take what they lack from its top, in the same order; then every new token gets
// its slot and position. A row is served if its pages, with those of all rows before it, are there, its tokens with those
// before it fit into n, and its pages fit into the table.
// Latency bound (some KB of lengths, sums over 1024 rows, one dependent read of the stack): one cluster. Each of its blocks
// makes the sums over all rows for itself (a thread a row), and they share out pages and tokens; between giving back and
// taking lies the one barrier of the cluster, and whatever a block changes in place it changes behind it. One block where
// there is little to share. Slots and positions of many tokens are left to a second kernel, since a cluster has 8 SMs only: with
// 118000 new tokens in 1024 rows it took 29 us for both, bound by their instructions.
struct PageStep {
    int B, n, pages, page_shift, stride;
    int *table, *free;
    const int *free_count, *lengths, *added, *ended, *first;
    int *free_count_out, *lengths_out, *cu_q, *positions, *sources;       // sources may be NULL
    long long* slots;
    int* status;
    int split;                                        // slots and positions are the second kernel's
};

constexpr int kStepThreads = 1024, kStepCluster = 8, kSlotThreads = 256;

// Inclusive sums of K numbers over the block, and their totals. Sums stay at kStepMost once they reach it.
constexpr unsigned kStepMost = 0x7fffffffu;
template <int K>
__device__ __forceinline__ void block_scan(unsigned* x, unsigned (*sums)[32], unsigned* all) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll 1
    for (int off = 1; off < 32; off <<= 1)
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const unsigned y = __shfl_up_sync(0xffffffffu, x[k], off);
            if (lane >= off) x[k] = min(x[k] + y, kStepMost);
        }
    __syncthreads();                                                 // what was there has been read
    if (lane == 31)
#pragma unroll
        for (int k = 0; k < K; ++k) sums[k][warp] = x[k];
    __syncthreads();
    unsigned w[K];
#pragma unroll
    for (int k = 0; k < K; ++k) w[k] = sums[k][lane];                // 32 warps
#pragma unroll 1
    for (int off = 1; off < 32; off <<= 1)
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const unsigned y = __shfl_up_sync(0xffffffffu, w[k], off);
            if (lane >= off) w[k] = min(w[k] + y, kStepMost);
        }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const unsigned before = __shfl_sync(0xffffffffu, w[k], warp ? warp - 1 : 0);
        all[k] = __shfl_sync(0xffffffffu, w[k], 31);
        if (warp) x[k] = min(x[k] + before, kStepMost);
    }
}
// The last row whose sum is at most i, for the warp's 32 numbers that follow each other; r: such a row of an earlier number, the
// same in all lanes. Long rows need one look; else each lane searches.
__device__ __forceinline__ int row_from(const int* scan, int B, int i, int r) {
    if (__all_sync(0xffffffffu, r + 1 >= B || scan[r + 1] > i)) return r;
    int hi = B - 1;
    while (r < hi) {
        const int mid = (r + hi + 1) >> 1;
        if (scan[mid] <= i) r = mid; else hi = mid - 1;
    }
    return r;
}
// f(i, row) for the warp's share of the numbers below `count`, 32 of them at a time. (Several turns under way at once hide the loads of
// one another, but take more code, and a launch runs through it cold, each 128 bytes some 300 cycles: 64 rows with a token each
// 8.2 us like this, 10.2 with four turns; 1024 rows with 118000 tokens 16.4, 17.2 with two and 20.5 with four.)
template <typename F>
__device__ __forceinline__ void share_out(const int* scan, int B, int count, F f) {
    const unsigned warps = gridDim.x * (blockDim.x / 32), per = (((unsigned)count + warps - 1) / warps + 31) & ~31u;     // a count may be 2^31 - 1
    const unsigned long long from = (unsigned long long)(blockIdx.x * (blockDim.x / 32) + (threadIdx.x >> 5)) * per;
    const unsigned end = (unsigned)min((unsigned long long)count, from + per);
    int r = 0;
#pragma unroll 1
    for (unsigned i0 = (unsigned)min((unsigned long long)count, from); i0 < end; i0 += 32) {
        const unsigned i = i0 + (threadIdx.x & 31);
        const int mine = row_from(scan, B, (int)min(i, end - 1), r);
        r = __shfl_sync(0xffffffffu, mine, 0);                       // numbers grow, rows do
        if (i < end) f((int)i, mine);
    }
}

// source: of token i among those asked for
__device__ __forceinline__ void put_slot(const PageStep& a, int i, bool there, int id, int place, int lead, int source) {
    const bool sound = id >= 0 && id < a.pages;
    if (there && !sound && a.status) atomicOr(a.status, kStPage);
    a.slots[i] = there && sound ? ((long long)id << a.page_shift) + (place & ((1 << a.page_shift) - 1)) : -1;
    a.positions[i] = there ? place + lead : 0;
    if (a.sources) a.sources[i] = there ? (int)min((unsigned)source, (unsigned)a.n - 1) : 0;
}

__global__ void __launch_bounds__(kStepThreads) page_step_kernel(PageStep a) {
    pdl_trigger();
    __shared__ unsigned sums[3][32];
    __shared__ int back[kPlanMax], cu[kPlanMax], take[kPlanMax], kept[kPlanMax], held[kPlanMax], lead[kPlanMax], ask[kPlanMax];
    const int b = threadIdx.x, page = 1 << a.page_shift, me = blockIdx.x, blocks = gridDim.x;
    const bool mine = b < a.B;
    int len = 0, add = 0, raw = 0, wrong = 0;
    bool end = false, sound = true;
    if (mine) {
        len = __ldg(a.lengths + b);
        add = __ldg(a.added + b);
        raw = max(add, 0);
        end = a.ended && __ldg(a.ended + b) != 0;
        lead[b] = a.first ? __ldg(a.first + b) : 0;
        sound = len >= 0 && len <= (long long)a.stride << a.page_shift;
        if (!sound || add < 0) { wrong |= kStPage; add = 0; }
        end = end && sound;
    }
    int count = *a.free_count;
    if (count < 0 || count > a.pages) { wrong |= kStPage; count = 0; }
    const int mine_back = end ? (int)(((long long)len + page - 1) >> a.page_shift) : 0;
    const int stay = end ? 0 : len, has = sound ? (int)(((long long)stay + page - 1) >> a.page_shift) : 0;
    const int want = sound ? (int)((((long long)stay + add + page - 1) >> a.page_shift) - has) : 0;
    unsigned asked[3] = {(unsigned)mine_back, (unsigned)want, (unsigned)add}, all[3];
    block_scan<3>(asked, sums, all);
    const int returned = min((int)all[0], a.pages - count);
    if ((int)all[0] > returned) wrong |= kStPage;                    // more pages than there are
    const int top = count + returned;
    const bool fits = (want == 0 || (asked[1] <= (unsigned)top && asked[1] < kStepMost)) && (add == 0 || (asked[2] <= (unsigned)a.n && asked[2] < kStepMost)) &&
                      (long long)has + want <= a.stride;
    if (mine && !fits) wrong |= kStCapacity;
    const int given = fits ? add : 0, got = fits ? want : 0;
    unsigned served[2] = {(unsigned)given, (unsigned)got}, totals[2];
    block_scan<2>(served, sums, totals);
    const int tokens = (int)totals[0], taken = (int)totals[1], at = (int)served[0] - given, from = (int)served[1] - got;
    if (mine) {
        back[b] = (int)asked[0] - mine_back;                        // (a whole table has fewer than kStepMost)
        cu[b] = at;
        take[b] = from;
        kept[b] = stay;
        held[b] = has;
    }
    if (a.sources && !a.split) {                                     // tokens asked for before each row, whatever its length says
        unsigned before[1] = {(unsigned)raw}, sum[1];
        block_scan<1>(before, sums, sum);
        ask[b] = (int)before[0] - raw;
    }
    __syncthreads();
    // a warp's pages and tokens follow each other (searched for one by one, all threads apart, 1024 rows with 118000 new tokens took
    // 31 us: 8 SMs' instructions)
    share_out(back, a.B, returned, [&](int i, int r) { a.free[count + i] = __ldcg(a.table + (long long)r * a.stride + i - back[r]); });
    __syncwarp();
    if (blocks > 1) {
        asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    } else {
        __syncthreads();
    }
    if (me == 0) {
        if (mine) {
            a.lengths_out[b] = sound ? stay + given : len;
            a.cu_q[b] = at;
        }
        if (threadIdx.x == 0) {
            a.cu_q[a.B] = tokens;
            *a.free_count_out = top - taken;
        }
        if (wrong && a.status) atomicOr(a.status, wrong);
    }
    share_out(take, a.B, taken, [&](int i, int r) { a.table[(long long)r * a.stride + held[r] + i - take[r]] = __ldcg(a.free + top - 1 - i); });
    if (a.split) return;
    share_out(cu, a.B, a.n, [&](int i, int r) {
        const int place = kept[r] + i - cu[r], p = place >> a.page_shift;
        int id = -1;
        if (i < tokens) id = p < held[r] ? __ldcg(a.table + (long long)r * a.stride + p) : __ldcg(a.free + top - 1 - (take[r] + p - held[r]));
        put_slot(a, i, i < tokens, id, place, lead[r], a.sources ? ask[r] + i - cu[r] : 0);
    });
}

// Slots and positions from the step's results: offsets, lengths and tables, the new tokens among them.
__global__ void __launch_bounds__(kSlotThreads) page_slots_kernel(PageStep a) {
    __shared__ int cu[kPlanMax + 1], ask[kPlanMax];
    __shared__ unsigned sums[kSlotThreads / 32];
    pdl_wait();
    for (int b = threadIdx.x; b <= a.B; b += kSlotThreads) cu[b] = __ldcg(a.cu_q + b);
    if (a.sources) {                                                 // tokens asked for before each row, a thread a few rows
        constexpr int R = kPlanMax / kSlotThreads;
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        unsigned add[R], sum = 0;
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const int b = threadIdx.x * R + k;
            add[k] = b < a.B ? max(__ldg(a.added + b), 0) : 0;
            sum += add[k];                                           // (may pass 31 bits behind the last token that an input of n rows has)
        }
        unsigned at = sum;
#pragma unroll 1
        for (int off = 1; off < 32; off <<= 1) {
            const unsigned y = __shfl_up_sync(0xffffffffu, at, off);
            if (lane >= off) at += y;
        }
        if (lane == 31) sums[warp] = at;
        __syncthreads();
        for (int k = 0; k < warp; ++k) at += sums[k];
        at -= sum;
#pragma unroll
        for (int k = 0; k < R; ++k) { ask[threadIdx.x * R + k] = (int)at; at += add[k]; }
    }
    __syncthreads();
    const int tokens = cu[a.B];
    share_out(cu, a.B, a.n, [&](int i, int r) {
        int id = -1, place = 0, lead = 0, source = 0;
        if (i < tokens) {
            place = __ldcg(a.lengths_out + r) - cu[r + 1] + i;
            lead = a.first ? __ldg(a.first + r) : 0;
            id = __ldcg(a.table + (long long)r * a.stride + (place >> a.page_shift));
            if (a.sources) source = ask[r] + i - cu[r];
        }
        put_slot(a, i, i < tokens, id, place, lead, source);
    });
}

}  // namespace sgk
