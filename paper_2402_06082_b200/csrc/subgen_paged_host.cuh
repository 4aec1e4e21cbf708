// Host helpers of the paged calls: checks of arguments, launches that the exact and the 4-bit cache have in common.
#pragma once
#include <cuda.h>
#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include <initializer_list>

#include "../../include/subgen.h"
#include "subgen_paged.cuh"

using namespace sgk;

int sgk_set_error(int code, const char* text);

namespace {

int fail(int code, const char* fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    return sgk_set_error(code, buf);
}

#define CUDA_TRY(expr)                                                                      \
    do {                                                                                    \
        cudaError_t err__ = (expr);                                                         \
        if (err__ != cudaSuccess) return fail(SUBGEN_ECUDA, "%s: %s", #expr, cudaGetErrorString(err__)); \
    } while (0)

constexpr int kSMs = 148;
constexpr int kMaxDevices = 64;

bool misaligned(const void* p) { return ((uintptr_t)p & 15) != 0; }
size_t elem(int dtype) { return dtype == SUBGEN_DTYPE_FP32 ? 4 : 2; }
bool odd_stride(int64_t s, int dtype) { return (s * (int64_t)elem(dtype)) % 16 != 0; }

// Also makes the kernel's view of it; the stride of an axis of one is not looked at.
int check_heads(const char* fn, const char* name, const subgen_heads* x, int n, int heads, int d, int dtype, HeadsView* v) {
    if (!x->p) return fail(SUBGEN_EINVAL, "%s: %s must not be NULL", fn, name);
    *v = HeadsView{x->p, n == 1 ? (int64_t)heads * d : x->token_stride, heads == 1 ? d : x->head_stride};
    if (v->ts <= 0 || v->hs <= 0) return fail(SUBGEN_EINVAL, "%s: %s: strides must be positive", fn, name);
    if (misaligned(x->p) || odd_stride(v->ts, dtype) || odd_stride(v->hs, dtype))
        return fail(SUBGEN_EINVAL, "%s: %s: pointer and strides must be multiples of 16 bytes", fn, name);
    return SUBGEN_OK;
}

// An output whose rows overlap each other, or that starts where an input does and lies otherwise (`same`: the one that it may be).
// Outputs that overlap an input further on are the caller's to avoid.
int check_output(const char* fn, const char* name, const HeadsView& o, int n, int heads, int d, const HeadsView& same,
                 std::initializer_list<const void*> others) {
    bool overlap = (n > 1 && o.ts < d) || (heads > 1 && o.hs < d);
    // rows (t, h) and (t + dt, h - dh) are dt * ts - dh * hs apart; where one axis lies within a step of the other there are none
    if (!overlap && o.ts < (heads - 1) * o.hs + d && o.hs < (n - 1) * o.ts + d)
        for (long long dh = 1; dh < heads && !overlap; ++dh) {
            const long long dt = dh * o.hs / o.ts, off = dh * o.hs - dt * o.ts;
            overlap = (dt > 0 && dt < n && off < d) || (dt + 1 < n && o.ts - off < d);
        }
    if (overlap) return fail(SUBGEN_EINVAL, "%s: %s: rows overlap", fn, name);
    if (o.p == same.p && (o.ts != same.ts || o.hs != same.hs))
        return fail(SUBGEN_EINVAL, "%s: %s: an output that is its input must have its strides", fn, name);
    for (const void* p : others)
        if (p && o.p == p) return fail(SUBGEN_EINVAL, "%s: %s must not be another tensor of the call", fn, name);
    return SUBGEN_OK;
}

int check_shape(const char* fn, int n, int H, int Hkv, int d, int dtype) {
    if (dtype != SUBGEN_DTYPE_FP32 && dtype != SUBGEN_DTYPE_BF16) return fail(SUBGEN_EINVAL, "%s: unknown dtype", fn);
    if (d != 64 && d != 128) return fail(SUBGEN_EINVAL, "%s: d must be 64 or 128", fn);
    if (n < 0 || H <= 0 || Hkv <= 0) return fail(SUBGEN_EINVAL, "%s: n must be >= 0, the numbers of heads positive", fn);
    if ((long long)n * (H + 2LL * Hkv) > 0x1fffffffLL) return fail(SUBGEN_EINVAL, "%s: too many rows in one call", fn);
    return SUBGEN_OK;
}

int check_rope(const char* fn, const subgen_rope* r, int d) {
    if (!r->words) return SUBGEN_OK;
    if (r->rotary_dim <= 0 || r->rotary_dim > d || r->rotary_dim % 16)
        return fail(SUBGEN_EINVAL, "%s: rotary_dim must be a multiple of 16 and at most d", fn);
    return SUBGEN_OK;
}

int check_norm(const char* fn, const void* wq, const void* wk, float eps) {
    if (misaligned(wq) || misaligned(wk)) return fail(SUBGEN_EINVAL, "%s: norm weights must be 16-byte aligned", fn);
    if ((wq || wk) && !(eps >= 0.f && isfinite(eps))) return fail(SUBGEN_EINVAL, "%s: eps must be finite and >= 0", fn);
    return SUBGEN_OK;
}

// The batch of a call on pages of `page` tokens.
int check_batch(const char* fn, const subgen_batch* b, int page) {
    if (b->B < 0 || b->groups < 0 || (long long)b->B + b->groups > kPlanMax)
        return fail(SUBGEN_EINVAL, "%s: B and groups must be >= 0, together at most %d", fn, kPlanMax);
    if (b->B && (!b->cu_q || !b->lengths || !b->table || b->table_stride <= 0))
        return fail(SUBGEN_EINVAL, "%s: cu_q, lengths and table must not be NULL, table_stride must be positive", fn);
    if (b->groups && (!b->cu_group || !b->prefix_len || !b->prefix_table || b->prefix_stride <= 0))
        return fail(SUBGEN_EINVAL, "%s: cu_group, prefix_len and prefix_table must not be NULL, prefix_stride must be positive", fn);
    const long long cap = 0x7fffffffLL - 1024;        // a token's index rounded up to tiles stays an int
    if ((long long)b->table_stride * page > cap || (b->groups && (long long)b->prefix_stride * page > cap))
        return fail(SUBGEN_EINVAL, "%s: a page table must hold fewer than 2^31 - 1024 tokens", fn);
    return SUBGEN_OK;
}

int check_cache(const char* fn, const subgen_pages* c, const subgen_batch* b, PagedView* v) {
    if (!c || !b) return fail(SUBGEN_EINVAL, "%s: cache and batch must not be NULL", fn);
    if (!c->K || !c->V) return fail(SUBGEN_EINVAL, "%s: K and V must not be NULL", fn);
    if (c->page < 16 || c->page > 1024 || (c->page & (c->page - 1)))
        return fail(SUBGEN_EINVAL, "%s: page must be a power of two, 16 to 1024", fn);
    if (c->pages <= 0) return fail(SUBGEN_EINVAL, "%s: pages must be positive", fn);
    if (c->page_stride <= 0 || c->head_stride <= 0 || c->row_stride < c->d)
        return fail(SUBGEN_EINVAL, "%s: the strides of the pool must be positive, row_stride at least d", fn);
    if (misaligned(c->K) || misaligned(c->V) || odd_stride(c->page_stride, c->dtype) || odd_stride(c->head_stride, c->dtype) ||
        odd_stride(c->row_stride, c->dtype))
        return fail(SUBGEN_EINVAL, "%s: the pool's pointers and strides must be multiples of 16 bytes", fn);
    const int rc = check_batch(fn, b, c->page);
    if (rc) return rc;
    int shift = 0;
    while ((1 << shift) < c->page) ++shift;
    *v = PagedView{(char*)c->K, (char*)c->V, c->page_stride, c->head_stride, c->row_stride, c->pages, shift, c->Hkv,
                   b->B, b->groups, b->cu_q, b->lengths, b->table, b->cu_group, b->prefix_len, b->prefix_table,
                   b->table_stride, b->prefix_stride, c->status};
    return SUBGEN_OK;
}

int this_device(int* dev) {
    CUDA_TRY(cudaGetDevice(dev));
    if (*dev < 0 || *dev >= kMaxDevices) return fail(SUBGEN_EINVAL, "device index %d not supported", *dev);
    return SUBGEN_OK;
}

// ---- norms, rotation, append ----
template <typename T, int D, int PAGED>
int launch_norm_rope(NormRope a, const PagedView& P, cudaStream_t st) {
    static bool done[kMaxDevices];
    int dev, rc = this_device(&dev);
    if (rc) return rc;
    if (!done[dev]) {                                 // loads both, so that a call of any size may be captured later
        cudaFuncAttributes at;
        CUDA_TRY(cudaFuncGetAttributes(&at, norm_rope_kernel<T, D, PAGED, 4>));
        CUDA_TRY(cudaFuncGetAttributes(&at, norm_rope_kernel<T, D, PAGED, 1>));
        done[dev] = true;
    }
    constexpr int RPW = 32 / (D / (16 / (int)sizeof(T)) / 2);
    const int groups = (a.H + RPW - 1) / RPW + (PAGED ? 2 : 1) * ((a.Hkv + RPW - 1) / RPW);
    // enough warps to fill the SMs (16 a SM); beyond that a token stays with one warp
    const int want = (kSMs * 16 + a.n - 1) / a.n;
    a.parts = want < 1 ? 1 : want > groups ? groups : want;
    const long long warps = (long long)a.n * a.parts;
    const unsigned blocks = (unsigned)((warps + kNrThreads / 32 - 1) / (kNrThreads / 32));
    if (a.parts == 1) norm_rope_kernel<T, D, PAGED, 4><<<blocks, kNrThreads, 0, st>>>(a, P);
    else norm_rope_kernel<T, D, PAGED, 1><<<blocks, kNrThreads, 0, st>>>(a, P);
    CUDA_TRY(cudaGetLastError());
    return SUBGEN_OK;
}

template <int PAGED>
int norm_rope(const NormRope& a, const PagedView& P, int d, int dtype, cudaStream_t st) {
    const bool f32 = dtype == SUBGEN_DTYPE_FP32;
    if (d == 64) return f32 ? launch_norm_rope<float, 64, PAGED>(a, P, st) : launch_norm_rope<__nv_bfloat16, 64, PAGED>(a, P, st);
    return f32 ? launch_norm_rope<float, 128, PAGED>(a, P, st) : launch_norm_rope<__nv_bfloat16, 128, PAGED>(a, P, st);
}

void fill_norm_rope(NormRope* a, const subgen_qk_args* x, int H, int Hkv) {
    a->n = x->n; a->H = H; a->Hkv = Hkv;
    a->positions = x->positions;
    a->words = (const unsigned long long*)x->rope.words;
    a->rot = x->rope.rotary_dim; a->interleaved = x->rope.interleaved;
    a->wq = x->wq; a->wk = x->wk; a->eps = x->eps; a->fresh = x->fresh != 0;
}

// ---- attention ----
constexpr size_t plan_bytes(int E) { return ((size_t)8 * (E + 1) + 15) & ~(size_t)15; }

long long slot_count(const PagedView& P, int n, int H) {
    // every row once per entry it belongs to; up to 128 rows of an entry's last unit twice, where the two groups of a block
    // share its tiles; and a unit of up to 256 rows (64 where a launch has more blocks) for every block that shares a unit
    // with the block before it
    const long long rows = (long long)n * H, unit = 128LL * P.Hkv;
    auto entries = [&](long long count) { return rows + (rows < unit * count ? rows : unit * count); };
    return entries(P.B) + (P.groups ? entries(P.groups) : 0) + 256LL * kSMs;
}

// The arguments of an attention call, as its kernels take them (left alone where n or P.B is 0).
int check_attend(const char* fn, const subgen_attend_args* x, const PagedView& P, int d, int dtype, Attend* a) {
    const int n = x->n, H = x->H;
    const int G = H / P.Hkv;
    if (H % P.Hkv || (G != 1 && G != 2 && G != 4 && G != 8)) return fail(SUBGEN_EINVAL, "%s: H / Hkv must be 1, 2, 4 or 8", fn);
    if (!(x->scale > 0.f) || !isfinite(x->scale * 1.4426950408889634f)) return fail(SUBGEN_EINVAL, "%s: scale must be positive and finite", fn);
    if (n == 0 || P.B == 0) return SUBGEN_OK;      // (nothing to do)
    HeadsView vq, vo;
    int rc = check_heads(fn, "q", &x->q, n, H, d, dtype, &vq);
    if (!rc) rc = check_heads(fn, "out", &x->out, n, H, d, dtype, &vo);
    if (rc) return rc;
    if (vo.p == vq.p) return fail(SUBGEN_EINVAL, "%s: out must not be q", fn);
    const long long slots = slot_count(P, n, H);
    // (the merge counts parts of rows for each sequence and KV head, those without new tokens among them)
    if (slots > 0x7fffffffLL || (long long)n * H + (long long)P.B * P.Hkv > 0x7f000000LL) return fail(SUBGEN_EINVAL, "%s: too many rows in one call", fn);
    const size_t need = (size_t)slots * (d * sizeof(float) + sizeof(float2));
    if (!x->workspace || ((uintptr_t)x->workspace & 255) || x->workspace_bytes < need)
        return fail(SUBGEN_ENOMEM, "%s: the workspace must be 256-byte aligned and hold %zu bytes", fn, need);
    rc = check_output(fn, "out", vo, n, H, d, vq, {P.K, P.V});
    if (rc) return rc;
    const int g_shift = G == 1 ? 0 : G == 2 ? 1 : G == 4 ? 2 : 3;
    *a = Attend{vq, vo, n, H, g_shift, x->causal != 0, x->scale * 1.4426950408889634f, (float*)x->workspace,
                (float2*)((float*)x->workspace + slots * d), x->fresh != 0};
    return SUBGEN_OK;
}

// Once per device: loads a kernel and the merge that follows it, so that both may be captured later.
template <typename K, typename M>
int opt_in(K kern, M merge, size_t smem) {
    cudaFuncAttributes at;
    CUDA_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    CUDA_TRY(cudaFuncGetAttributes(&at, merge));
    return SUBGEN_OK;
}

template <typename T, int D, int RU, int KT, int DUAL, int LEAD>
int launch_merge(const PagedView& P, const Attend& a, int blocks, cudaStream_t st) {
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof cfg);
    // parts of a row unit that a block joins at a time: as few rows as let the blocks that fit take all of them at once, up
    // to 16 for prompts, most of whose rows need none (RU is a multiple of each)
    const long long rows = (long long)a.n * a.H, once = kSMs * kMergeBlocks;
    int part = 1;
    while (part < 16 && part < RU && rows > once * part) part *= 2;
    const long long units = ((long long)P.B + ((long long)a.n << a.g_shift) / part) * P.Hkv;
    cfg.gridDim = dim3((unsigned)(units < kSMs * kMergeBlocks ? units : kSMs * kMergeBlocks));
    cfg.blockDim = dim3(kMergeThreads);
    cfg.dynamicSmemBytes = plan_bytes(P.B + P.groups) + (size_t)4 * (P.B + 1);
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    CUDA_TRY(cudaLaunchKernelEx(&cfg, paged_merge_kernel<T, D, RU, KT, DUAL, LEAD>, P, a, blocks, part));
    return SUBGEN_OK;
}

// ---- tensor maps (bf16 attention) ----
typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled() {
    static const EncodeTiled f = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult r;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &r) != cudaSuccess || r != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            p = nullptr;
        }
        return (EncodeTiled)p;
    }();
    return f;
}

// extents and strides from the second axis on; the innermost is d, boxes are 64 columns (128 bytes) wide
int make_map(CUtensorMap* m, void* p, int rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box) {
    const EncodeTiled f = encode_tiled();
    if (!f) return fail(SUBGEN_ECUDA, "cuTensorMapEncodeTiled is not available");
    const cuuint32_t ones[5] = {1, 1, 1, 1, 1};
    const CUresult r = f(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank, p, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                         CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return fail(SUBGEN_ECUDA, "cuTensorMapEncodeTiled failed (%d): strides of 2^40 bytes or more?", (int)r);
    return SUBGEN_OK;
}

}  // namespace
