// Host side of the head norms with rotation and of the paged exact cache (see include/subgen.h).
#include "../../include/subgen.h"

#include "subgen_paged_host.cuh"
#include "subgen_paged_simt.cuh"
#include "subgen_paged_tc.cuh"

namespace {

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
    return norm_rope<0>(a, none, x->d, x->dtype, (cudaStream_t)stream);
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
    return norm_rope<1>(a, P, d, dtype, (cudaStream_t)stream);
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
    Attend a;
    rc = check_attend(fn, x, P, d, cache->dtype, &a);
    if (rc || n == 0 || batch->B == 0) return rc;
    cudaStream_t st = (cudaStream_t)stream;
    if (cache->dtype == SUBGEN_DTYPE_BF16) return d == 64 ? attend_tc<64>(P, a, st) : attend_tc<128>(P, a, st);
    return d == 64 ? attend_fp32<64>(P, a, st) : attend_fp32<128>(P, a, st);
}

}  // extern "C"
