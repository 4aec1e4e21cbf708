// Cache in 4-bit cells: tokens by their slots as dense keys and values; and the tables of a step.
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>

#include "subgen_paged.cuh"

namespace sgk {

// ---- load ---------------------------------------------------------------------------------------
//
// Row (token, head, K or V) = d / 2 code bytes and d / 16 scale bytes -> d values of T, exact. Memory bound: 4.5 bits read, 16 or
// 32 written per value. A lane takes 8 values (4 bytes and a scale byte), so that a warp writes whole rows by 16-byte pieces,
// and kLoadAhead rows' loads go out before the first is used.
struct Load4 {
    const char* pool;
    long long ps, hs;                                 // bytes
    const long long* slots;
    int n, Hkv, pages, page_shift;
    HeadsView k, v;                                   // p NULL: not wanted
    int* status;
};

constexpr int kLoadThreads = 256, kLoadAhead = 4;

template <typename T, int D>
__global__ void __launch_bounds__(kLoadThreads) paged4_load_kernel(Load4 a) {
    constexpr int LPR = D / 8, RPB = kLoadThreads / LPR;             // lanes a row, rows a block and turn
    const int l = threadIdx.x % LPR, per = a.Hkv * 2;
    const long long rows = (long long)a.n * per, first = (long long)blockIdx.x * (RPB * kLoadAhead) + threadIdx.x / LPR;
    uint32_t code[kLoadAhead], scale[kLoadAhead];
    T* to[kLoadAhead];
#pragma unroll
    for (int u = 0; u < kLoadAhead; ++u) {
        const long long r = first + u * RPB;
        to[u] = nullptr;
        if (r >= rows) continue;
        const int tok = (int)(r / per), i = (int)(r - (long long)tok * per), kv = i >= a.Hkv ? 1 : 0, h = i - kv * a.Hkv;
        const HeadsView& y = kv ? a.v : a.k;
        if (!y.p) continue;
        to[u] = (T*)y.p + tok * y.ts + h * y.hs + l * 8;
        const long long slot = __ldg(a.slots + tok), page = slot >> a.page_shift;
        code[u] = 0;
        scale[u] = 0;                                                // a slot below 0: zeros
        if (slot < 0) continue;
        if (page >= a.pages) {
            scale[u] = 255u;
            if (i == 0 && l == 0 && a.status) atomicOr(a.status, kStPage);
            continue;
        }
        const int row = (int)(slot & ((1 << a.page_shift) - 1));
        const char* cell = a.pool + page * a.ps + h * a.hs + (row >> 4) * Cell4<D>::kBytes + kv * Cell4<D>::kHalf;
        code[u] = __ldcs(reinterpret_cast<const uint32_t*>(cell + (row & 15) * Cell4<D>::kCodes) + l);
        scale[u] = *reinterpret_cast<const unsigned char*>(cell + Cell4<D>::kScaleAt + (row & 15) * Cell4<D>::kScales + l / 2);
    }
    const Consts4 consts;
#pragma unroll
    for (int u = 0; u < kLoadAhead; ++u) {
        if (!to[u]) continue;
        __half2 s, o;
        scale_pair4(scale[u] * 0x00010001u, consts, &s, &o);
        uint32_t x[4];
        pairs4(code[u], s, o, consts, x);
        float f[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 y = __half22float2(*reinterpret_cast<const __half2*>(&x[j]));
            f[2 * j] = y.x * 8.f;
            f[2 * j + 1] = y.y * 8.f;
        }
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<float4*>(to[u]) = make_float4(f[0], f[1], f[2], f[3]);
            *reinterpret_cast<float4*>(to[u] + 4) = make_float4(f[4], f[5], f[6], f[7]);
        } else {
            *reinterpret_cast<uint4*>(to[u]) = pack_row<T, 8>(f);
        }
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
