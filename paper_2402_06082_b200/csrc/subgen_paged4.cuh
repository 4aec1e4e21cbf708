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
// one: the place of a row among a token's is told once (rows numbered over all tokens took 3 times the instructions, 45 us for
// 32768 tokens x 8 heads x 128 in bf16).
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
                if (i == 0 && l == 0 && a.status) atomicOr(a.status, kStPage);
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
                *reinterpret_cast<uint4*>(z) = make_uint4(x[0] << 16, x[0] & 0xffff0000u, x[1] << 16, x[1] & 0xffff0000u);
                *reinterpret_cast<uint4*>(z + 4) = make_uint4(x[2] << 16, x[2] & 0xffff0000u, x[3] << 16, x[3] & 0xffff0000u);
            } else {
                *reinterpret_cast<uint4*>(z) = make_uint4(x[0], x[1], x[2], x[3]);
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
// there is little to share.
struct PageStep {
    int B, n, pages, page_shift, stride;
    int *table, *free;
    const int *free_count, *lengths, *added, *ended, *first;
    int *free_count_out, *lengths_out, *cu_q, *positions;
    long long* slots;
    int* status;
};

constexpr int kStepThreads = 1024, kStepCluster = 8;

// exclusive sums of x over the block; *all: the total
__device__ __forceinline__ long long block_scan(long long x, long long* sums, long long* all) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    long long s = x;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, s, off);
        if (lane >= off) s += y;
    }
    __syncthreads();                                                 // what was there has been read
    if (lane == 31) sums[warp] = s;
    __syncthreads();
    long long w = sums[lane];                                        // 32 warps
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, w, off);
        if (lane >= off) w += y;
    }
    *all = __shfl_sync(0xffffffffu, w, 31);
    const long long before = __shfl_sync(0xffffffffu, w, warp ? warp - 1 : 0);
    return s - x + (warp ? before : 0);
}
// the last row whose sum is at most i
__device__ __forceinline__ int row_of(const int* scan, int B, int i) {
    int lo = 0, hi = B - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (scan[mid] <= i) lo = mid; else hi = mid - 1;
    }
    return lo;
}

__global__ void __launch_bounds__(kStepThreads) page_step_kernel(PageStep a) {
    __shared__ long long sums[32];
    __shared__ int back[kPlanMax], cu[kPlanMax], take[kPlanMax], kept[kPlanMax], held[kPlanMax], lead[kPlanMax];
    const int b = threadIdx.x, page = 1 << a.page_shift, me = blockIdx.x, blocks = gridDim.x;
    const bool mine = b < a.B;
    int len = 0, add = 0, wrong = 0;
    bool end = false, sound = true;
    if (mine) {
        len = __ldg(a.lengths + b);
        add = __ldg(a.added + b);
        end = a.ended && __ldg(a.ended + b) != 0;
        lead[b] = a.first ? __ldg(a.first + b) : 0;
        sound = len >= 0 && len <= (long long)a.stride << a.page_shift;
        if (!sound || add < 0) { wrong |= kStPage; add = 0; }
        end = end && sound;
    }
    int count = *a.free_count;
    if (count < 0 || count > a.pages) { wrong |= kStPage; count = 0; }
    long long all;
    const int mine_back = end ? (int)(((long long)len + page - 1) >> a.page_shift) : 0;
    const long long before = block_scan(mine_back, sums, &all);
    int returned = (int)min(all, (long long)(a.pages - count));
    if (returned < all) wrong |= kStPage;                            // more pages than there are
    const int top = count + returned;
    const int stay = end ? 0 : len, has = sound ? (int)(((long long)stay + page - 1) >> a.page_shift) : 0;
    const long long want = sound ? (((long long)stay + add + page - 1) >> a.page_shift) - has : 0;
    long long none;
    const long long pages_before = block_scan(want, sums, &none), tokens_before = block_scan(add, sums, &none);
    const bool fits = (want == 0 || pages_before + want <= top) && (add == 0 || tokens_before + add <= a.n) && has + want <= a.stride;
    if (mine && !fits) wrong |= kStCapacity;
    const int given = fits ? add : 0, got = fits ? (int)want : 0;
    long long tokens, taken;
    const int at = (int)block_scan(given, sums, &tokens), from = (int)block_scan(got, sums, &taken);
    if (mine) {
        back[b] = (int)min(before, (long long)INT32_MAX);
        cu[b] = at;
        take[b] = from;
        kept[b] = stay;
        held[b] = has;
    }
    __syncthreads();
    const int stride = blocks * kStepThreads, i0 = me * kStepThreads + threadIdx.x;
    for (int i = i0; i < returned; i += stride) {
        const int r = row_of(back, a.B, i);
        a.free[count + i] = __ldcg(a.table + (long long)r * a.stride + i - back[r]);
    }
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
            a.cu_q[a.B] = (int)tokens;
            *a.free_count_out = top - (int)taken;
        }
        if (wrong && a.status) atomicOr(a.status, wrong);
    }
    for (int i = i0; i < taken; i += stride) {
        const int r = row_of(take, a.B, i);
        a.table[(long long)r * a.stride + held[r] + i - take[r]] = __ldcg(a.free + top - 1 - i);
    }
    for (int i = i0; i < a.n; i += stride) {
        long long slot = -1;
        int position = 0;
        if (i < tokens) {
            const int r = row_of(cu, a.B, i), place = kept[r] + i - cu[r], p = place >> a.page_shift;
            const int id = p < held[r] ? __ldcg(a.table + (long long)r * a.stride + p) : __ldcg(a.free + top - 1 - (take[r] + p - held[r]));
            if (id >= 0 && id < a.pages) slot = ((long long)id << a.page_shift) + (place & (page - 1));
            else if (a.status) atomicOr(a.status, kStPage);
            position = place + lead[r];
        }
        a.slots[i] = slot;
        a.positions[i] = position;
    }
}

}  // namespace sgk
