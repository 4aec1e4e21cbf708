// Host side of the head norms with rotation and of the paged exact cache (see include/subgen.h).
#include "../../include/subgen.h"

#include <cuda.h>
#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include <initializer_list>

#include "subgen_paged.cuh"
#include "subgen_paged_simt.cuh"
#include "subgen_paged_tc.cuh"

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
    if (b->B < 0 || b->groups < 0 || (long long)b->B + b->groups > kPlanMax)
        return fail(SUBGEN_EINVAL, "%s: B and groups must be >= 0, together at most %d", fn, kPlanMax);
    if (b->B && (!b->cu_q || !b->lengths || !b->table || b->table_stride <= 0))
        return fail(SUBGEN_EINVAL, "%s: cu_q, lengths and table must not be NULL, table_stride must be positive", fn);
    if (b->groups && (!b->cu_group || !b->prefix_len || !b->prefix_table || b->prefix_stride <= 0))
        return fail(SUBGEN_EINVAL, "%s: cu_group, prefix_len and prefix_table must not be NULL, prefix_stride must be positive", fn);
    const long long cap = 0x7fffffffLL - 1024;        // a token's index rounded up to tiles stays an int
    if ((long long)b->table_stride * c->page > cap || (b->groups && (long long)b->prefix_stride * c->page > cap))
        return fail(SUBGEN_EINVAL, "%s: a page table must hold fewer than 2^31 - 1024 tokens", fn);
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
template <typename T, int D, bool PAGED>
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

template <bool PAGED>
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
size_t plan_bytes(int E) { return ((size_t)8 * (E + 1) + 15) & ~(size_t)15; }

long long slot_count(const PagedView& P, int n, int H) {
    // every row once per entry it belongs to; up to 128 rows of an entry's last unit twice, where the two groups of a block
    // share its tiles; and a unit of up to 256 rows (64 where a launch has more blocks) for every block that shares a unit
    // with the block before it
    const long long rows = (long long)n * H, unit = 128LL * P.Hkv;
    auto entries = [&](long long count) { return rows + (rows < unit * count ? rows : unit * count); };
    return entries(P.B) + (P.groups ? entries(P.groups) : 0) + 256LL * kSMs;
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

template <typename S, int D, typename K>
int attend_fp32_with(K kern, const PagedView& P, const Attend& a, cudaStream_t st) {
    constexpr size_t tile = (sizeof(S) + 15) & ~(size_t)15;
    const int blocks = kSMs * S::BLOCKS;
    static_assert(S::RU * S::BLOCKS <= 256, "slot_count");
    kern<<<blocks, S::NT, tile + plan_bytes(P.B + P.groups), st>>>(P, a);
    CUDA_TRY(cudaGetLastError());
    return launch_merge<float, D, S::RU, S::KT, 0, kSimtLead>(P, a, blocks, st);
}
template <typename S, int D, typename K>
int opt_in_fp32(K kern) {
    return opt_in(kern, paged_merge_kernel<float, D, S::RU, S::KT, 0, kSimtLead>, ((sizeof(S) + 15) & ~(size_t)15) + plan_bytes(kPlanMax));
}

template <int D>
int attend_fp32(const PagedView& P, const Attend& a, cudaStream_t st) {
    static bool done[kMaxDevices];
    int dev, rc = this_device(&dev);
    if (!rc && !done[dev]) {                          // both kinds, whichever this call takes
        rc = opt_in_fp32<FewSmem<D>, D>(paged_attend_few_kernel<D>);
        if (!rc) rc = opt_in_fp32<SimtSmem<D>, D>(paged_attend_simt_kernel<D>);
        done[dev] = !rc;
    }
    if (rc) return rc;
    // Up to 8 rows a sequence on average: one pass over the cache with little arithmetic to it (16 sequences of 2000 tokens,
    // 8 heads, 8 rows each: 93 us against 216; 12 rows, which take two units there: 191 against 218, but 110 against 82 at
    // d = 64 behind a shared prefix). The mean is all that is looked at: a chunk of a prompt among many single tokens, or many of
    // those behind one prefix, comes in units of 8 rows here, each of which reads all that it sees.
    if (((long long)a.n << a.g_shift) <= 8LL * P.B) return attend_fp32_with<FewSmem<D>, D>(paged_attend_few_kernel<D>, P, a, st);
    return attend_fp32_with<SimtSmem<D>, D>(paged_attend_simt_kernel<D>, P, a, st);
}

// ---- attention, bf16: tensor maps over the pool and the queries ----
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

template <int D>
int attend_tc(const PagedView& P, const Attend& a, cudaStream_t st) {
    typedef __nv_bfloat16 T;
    static bool done[kMaxDevices];
    constexpr size_t fixed = 1024 + ((sizeof(PtSmem<D>) + 15) & ~(size_t)15);
    int dev, rc = this_device(&dev);
    if (!rc && !done[dev]) {                          // both kinds, whichever this call takes
        rc = opt_in(paged_attend_tc_kernel<D, false>, paged_merge_kernel<T, D, kPtRU, kPtKT, 1, kPtLead>, fixed + plan_bytes(kPlanMax));
        if (!rc) rc = opt_in(paged_attend_tc_kernel<D, true>, paged_merge_kernel<T, D, kPtRU, kPtKT, 2, kPtLead>, fixed + plan_bytes(kPlanMax));
        done[dev] = !rc;
    }
    if (rc) return rc;
    CUtensorMap mq, mk, mv;
    {
        const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)a.H, (cuuint64_t)a.n};
        const cuuint64_t strides[2] = {(cuuint64_t)a.q.hs * 2, (cuuint64_t)a.q.ts * 2};
        const cuuint32_t box[3] = {64, 1u << a.g_shift, 32u >> a.g_shift};       // 32 rows
        rc = make_map(&mq, a.q.p, 3, dims, strides, box);
    }
    const int page = 1 << P.page_shift;
    const cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)page, (cuuint64_t)P.Hkv, (cuuint64_t)P.pages};
    const cuuint64_t strides[3] = {(cuuint64_t)P.ts * 2, (cuuint64_t)P.hs * 2, (cuuint64_t)P.ps * 2};
    const cuuint32_t box[4] = {64, (cuuint32_t)(page < 128 ? page : 128), 1, 1};
    if (!rc) rc = make_map(&mk, P.K, 4, dims, strides, box);
    if (!rc && !paired(P, D)) rc = make_map(&mv, P.V, 4, dims, strides, box);
    if (!rc && paired(P, D)) {                        // both 64-column halves of a page's rows in one copy
        const cuuint64_t dims5[5] = {64, (cuuint64_t)page, 2, (cuuint64_t)P.Hkv, (cuuint64_t)P.pages};
        const cuuint64_t strides5[4] = {strides[0], 128, strides[1], strides[2]};
        const cuuint32_t box5[5] = {64, box[1], 2, 1, 1};
        rc = make_map(&mv, P.V, 5, dims5, strides5, box5);
    }
    if (rc) return rc;
    const size_t smem = fixed + plan_bytes(P.B + P.groups);
    // The two groups' results of a unit of up to 32 rows are joined in the block where most units are one block's: no prefixes
    // and a unit for each block at least (128 sequences of 1024 tokens, 8 KV heads: 107 -> 102 us; but 95 -> 98 with
    // prefixes, whose partials go to the merge anyway, and 15.4 -> 16.1 for one short sequence, all of it split).
    if (!P.groups && (long long)P.B * P.Hkv >= kSMs) {
        paged_attend_tc_kernel<D, true><<<kSMs, kPtThreads, smem, st>>>(P, a, mq, mk, mv);
        CUDA_TRY(cudaGetLastError());
        return launch_merge<T, D, kPtRU, kPtKT, 2, kPtLead>(P, a, kSMs, st);
    }
    paged_attend_tc_kernel<D, false><<<kSMs, kPtThreads, smem, st>>>(P, a, mq, mk, mv);
    CUDA_TRY(cudaGetLastError());
    return launch_merge<T, D, kPtRU, kPtKT, 1, kPtLead>(P, a, kSMs, st);
}

}  // namespace

extern "C" {

int subgen_rope_words(const double* f, int count, uint64_t* words) {
    if (!f || !words || count < 0) return fail(SUBGEN_EINVAL, "subgen_rope_words: invalid argument");
    for (int i = 0; i < count; ++i) {
        if (!isfinite(f[i])) return fail(SUBGEN_EINVAL, "subgen_rope_words: f[%d] is not finite", i);
        const long double turns = (long double)f[i] / 6.283185307179586476925286766559005768L;
        const long double frac = turns - floorl(turns);                       // [0, 1)
        const long double w = roundl(frac * 18446744073709551616.0L);
        words[i] = w >= 18446744073709551616.0L ? 0 : (uint64_t)w;
    }
    return SUBGEN_OK;
}

int subgen_qk_norm_rope(const subgen_qk_args* x, void* stream) {
    const char* fn = "subgen_qk_norm_rope";
    if (!x) return fail(SUBGEN_EINVAL, "%s: args must not be NULL", fn);
    const bool has_q = x->q.p, has_k = x->k.p;
    int rc = check_shape(fn, x->n, has_q || !has_k ? x->H : 1, has_k || !has_q ? x->Hkv : 1, x->d, x->dtype);
    if (!rc) rc = check_rope(fn, &x->rope, x->d);
    if (!rc) rc = check_norm(fn, x->wq, x->wk, x->eps);
    if (rc || x->n == 0) return rc;
    if (!has_q && !has_k) return fail(SUBGEN_EINVAL, "%s: q and k must not both be NULL", fn);
    NormRope a;
    memset(&a, 0, sizeof a);
    if (has_q) rc = check_heads(fn, "q", &x->q, x->n, x->H, x->d, x->dtype, &a.q);
    if (!rc && has_q) rc = check_heads(fn, "q_out", &x->q_out, x->n, x->H, x->d, x->dtype, &a.qo);
    if (!rc && has_k) rc = check_heads(fn, "k", &x->k, x->n, x->Hkv, x->d, x->dtype, &a.k);
    if (!rc && has_k) rc = check_heads(fn, "k_out", &x->k_out, x->n, x->Hkv, x->d, x->dtype, &a.ko);
    if (!rc && x->rope.words && !x->positions) rc = fail(SUBGEN_EINVAL, "%s: a rotation needs positions", fn);
    if (!rc && has_q) rc = check_output(fn, "q_out", a.qo, x->n, x->H, x->d, a.q, {a.k.p, a.ko.p});
    if (!rc && has_k) rc = check_output(fn, "k_out", a.ko, x->n, x->Hkv, x->d, a.k, {a.q.p});
    if (rc) return rc;
    fill_norm_rope(&a, x, has_q ? x->H : 0, has_k ? x->Hkv : 0);
    PagedView none;
    memset(&none, 0, sizeof none);
    return norm_rope<false>(a, none, x->d, x->dtype, (cudaStream_t)stream);
}

int subgen_paged_append(const subgen_pages* cache, const subgen_batch* batch, const subgen_qk_args* x, void* stream) {
    const char* fn = "subgen_paged_append";
    PagedView P;
    if (!cache || !batch || !x) return fail(SUBGEN_EINVAL, "%s: cache, batch and args must not be NULL", fn);
    const bool has_q = x->q.p;
    const int Hkv = cache->Hkv, d = cache->d, dtype = cache->dtype;
    int rc = check_shape(fn, x->n, has_q ? x->H : 1, Hkv, d, dtype);
    if (!rc) rc = check_cache(fn, cache, batch, &P);
    if (!rc) rc = check_rope(fn, &x->rope, d);
    if (!rc) rc = check_norm(fn, x->wq, x->wk, x->eps);
    if (rc || x->n == 0 || batch->B == 0) return rc;
    NormRope a;
    memset(&a, 0, sizeof a);
    rc = check_heads(fn, "k", &x->k, x->n, Hkv, d, dtype, &a.k);
    if (!rc) rc = check_heads(fn, "v", &x->v, x->n, Hkv, d, dtype, &a.v);
    if (!rc && has_q) rc = check_heads(fn, "q", &x->q, x->n, x->H, d, dtype, &a.q);
    if (!rc && has_q) rc = check_heads(fn, "q_out", &x->q_out, x->n, x->H, d, dtype, &a.qo);
    if (!rc && has_q) rc = check_output(fn, "q_out", a.qo, x->n, x->H, d, a.q, {a.k.p, a.v.p, P.K, P.V});
    if (rc) return rc;
    fill_norm_rope(&a, x, has_q ? x->H : 0, Hkv);
    return norm_rope<true>(a, P, d, dtype, (cudaStream_t)stream);
}

size_t subgen_paged_workspace_bytes(const subgen_pages* cache, const subgen_batch* batch, int n, int H) {
    const char* fn = "subgen_paged_workspace_bytes";
    PagedView P;
    if (!cache || !batch) { fail(SUBGEN_EINVAL, "%s: cache and batch must not be NULL", fn); return 0; }
    if (check_shape(fn, n, H, cache->Hkv, cache->d, cache->dtype) || check_cache(fn, cache, batch, &P)) return 0;
    return (size_t)slot_count(P, n, H) * (cache->d * sizeof(float) + sizeof(float2));
}

int subgen_paged_attend(const subgen_pages* cache, const subgen_batch* batch, const subgen_attend_args* x, void* stream) {
    const char* fn = "subgen_paged_attend";
    PagedView P;
    if (!cache || !batch || !x) return fail(SUBGEN_EINVAL, "%s: cache, batch and args must not be NULL", fn);
    const int n = x->n, H = x->H, d = cache->d;
    int rc = check_shape(fn, n, H, cache->Hkv, d, cache->dtype);
    if (!rc) rc = check_cache(fn, cache, batch, &P);
    if (rc) return rc;
    const int G = H / cache->Hkv;
    if (H % cache->Hkv || (G != 1 && G != 2 && G != 4 && G != 8)) return fail(SUBGEN_EINVAL, "%s: H / Hkv must be 1, 2, 4 or 8", fn);
    if (!(x->scale > 0.f) || !isfinite(x->scale * 1.4426950408889634f)) return fail(SUBGEN_EINVAL, "%s: scale must be positive and finite", fn);
    if (n == 0 || batch->B == 0) return SUBGEN_OK;
    HeadsView vq, vo;
    rc = check_heads(fn, "q", &x->q, n, H, d, cache->dtype, &vq);
    if (!rc) rc = check_heads(fn, "out", &x->out, n, H, d, cache->dtype, &vo);
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
    Attend a = {vq, vo, n, H, g_shift, x->causal != 0, x->scale * 1.4426950408889634f, (float*)x->workspace,
                (float2*)((float*)x->workspace + slots * d), x->fresh != 0};
    cudaStream_t st = (cudaStream_t)stream;
    if (cache->dtype == SUBGEN_DTYPE_BF16) return d == 64 ? attend_tc<64>(P, a, st) : attend_tc<128>(P, a, st);
    return d == 64 ? attend_fp32<64>(P, a, st) : attend_fp32<128>(P, a, st);
}

}  // extern "C"
