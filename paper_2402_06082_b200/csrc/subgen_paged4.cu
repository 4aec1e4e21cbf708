// Host side of the paged cache in 4 bits and of the tables of a step (see include/subgen.h).
#include "subgen_paged_host.cuh"
#include "subgen_paged4.cuh"
#include "subgen_paged4_few.cuh"
#include "subgen_paged_tc.cuh"

namespace {

size_t cell_bytes(int d) { return d == 64 ? Cell4<64>::kBytes : Cell4<128>::kBytes; }

int check_pages(const char* fn, int pages, int page) {
    if (page < 16 || page > 1024 || (page & (page - 1))) return fail(SUBGEN_EINVAL, "%s: page must be a power of two, 16 to 1024", fn);
    if (pages <= 0) return fail(SUBGEN_EINVAL, "%s: pages must be positive", fn);
    return SUBGEN_OK;
}
int shift_of(int page) {
    int shift = 0;
    while ((1 << shift) < page) ++shift;
    return shift;
}

// The stride of an axis of one is not looked at.
int check_pool(const char* fn, const subgen_pages4* c, PagedView* v) {
    if (!c->pool) return fail(SUBGEN_EINVAL, "%s: pool must not be NULL", fn);
    const int rc = check_pages(fn, c->pages, c->page);
    if (rc) return rc;
    const int64_t bytes = (int64_t)(c->page / 16) * (int64_t)cell_bytes(c->d);
    const int64_t hs = c->Hkv == 1 ? bytes : c->head_stride, ps = c->pages == 1 ? bytes * c->Hkv : c->page_stride;
    if (hs < bytes || ps < bytes) return fail(SUBGEN_EINVAL, "%s: the pool's strides must be at least %lld bytes", fn, (long long)bytes);
    if (misaligned(c->pool) || hs % 16 || ps % 16) return fail(SUBGEN_EINVAL, "%s: the pool's pointer and strides must be multiples of 16 bytes", fn);
    memset(v, 0, sizeof *v);
    v->K = v->V = (char*)c->pool;
    v->ps = ps; v->hs = hs;
    v->pages = c->pages; v->page_shift = shift_of(c->page); v->Hkv = c->Hkv;
    v->status = c->status;
    return SUBGEN_OK;
}

int check_cache4(const char* fn, const subgen_pages4* c, const subgen_batch* b, PagedView* v) {
    int rc = check_pool(fn, c, v);
    if (!rc) rc = check_batch(fn, b, c->page);
    if (rc) return rc;
    v->B = b->B; v->groups = b->groups;
    v->cu_q = b->cu_q; v->lengths = b->lengths; v->table = b->table;
    v->cu_group = b->cu_group; v->prefix_len = b->prefix_len; v->prefix_table = b->prefix_table;
    v->table_stride = b->table_stride; v->prefix_stride = b->prefix_stride;
    return SUBGEN_OK;
}

template <typename T, int D>
int launch_load(Load4 a, cudaStream_t st) {
    constexpr int RPB = kLoadThreads / (D / 8);
    const int rows = 2 * a.Hkv;
    a.at_once = rows < RPB ? RPB / rows : 1;
    const long long groups = (rows + RPB - 1) / RPB, tokens = ((long long)a.n + a.at_once - 1) / a.at_once;
    if (groups > 65535) return fail(SUBGEN_EINVAL, "subgen_paged4_load: too many heads");
    const long long once = (kSMs * kLoadBlocks + groups - 1) / groups, blocks = tokens < once ? tokens : once;       // all blocks at once
    paged4_load_kernel<T, D><<<dim3((unsigned)blocks, (unsigned)groups), kLoadThreads, 0, st>>>(a);
    CUDA_TRY(cudaGetLastError());
    return SUBGEN_OK;
}

// ---- attention ----
template <typename T, int D, int NT, int TILES>
constexpr size_t few_smem() { return (sizeof(P4Smem<T, D, NT, TILES>) + 15) & ~(size_t)15; }

// Tiles in flight. A third one where the plan (8 bytes a sequence) leaves room for it with all blocks there at once: 64 sequences 89 -> 86 us.
// Without room (256 sequences of 1024 tokens) a third of the blocks would run after the others. By size of the rest it fits never, always
// or with small plans (bf16, D = 128, units of 8 rows: up to 233 sequences and prefixes).
template <typename T, int D, int NT>
struct Few {
    static constexpr size_t kRoom = 233472 / kP4Blocks<NT> - 1024;   // shared memory of a block
    static constexpr bool kThree = few_smem<T, D, NT, 3>() + plan_bytes(1) <= kRoom, kTwo = few_smem<T, D, NT, 3>() + plan_bytes(kPlanMax) > kRoom;
    static_assert(few_smem<T, D, NT, 2>() + plan_bytes(kPlanMax) <= kRoom, "two tiles always fit");
};

template <typename T, int D, int NT>
int opt_in_few() {
    int rc = SUBGEN_OK;
    if constexpr (Few<T, D, NT>::kThree)
        rc = opt_in(paged4_attend_few_kernel<T, D, NT, 3>, paged_merge_kernel<T, D, 8 * NT, kP4KT, 0, kP4Lead>, few_smem<T, D, NT, 3>() + plan_bytes(kPlanMax));
    if constexpr (Few<T, D, NT>::kTwo)
        if (!rc) rc = opt_in(paged4_attend_few_kernel<T, D, NT, 2>, paged_merge_kernel<T, D, 8 * NT, kP4KT, 0, kP4Lead>, few_smem<T, D, NT, 2>() + plan_bytes(kPlanMax));
    return rc;
}
template <typename T, int D, int NT>
int attend_few(const PagedView& P, const Attend& a, cudaStream_t st) {
    typedef Few<T, D, NT> F;
    constexpr int blocks = kSMs * kP4Blocks<NT>;
    static_assert(8 * NT * kP4Blocks<NT> <= 256, "slot_count");
    const size_t plan = plan_bytes(P.B + P.groups);
    bool three = F::kThree;
    if (F::kTwo) three = three && few_smem<T, D, NT, 3>() + plan <= F::kRoom;
    if constexpr (F::kThree)
        if (three) paged4_attend_few_kernel<T, D, NT, 3><<<blocks, kP4Threads, few_smem<T, D, NT, 3>() + plan, st>>>(P, a);
    if constexpr (F::kTwo)
        if (!three) paged4_attend_few_kernel<T, D, NT, 2><<<blocks, kP4Threads, few_smem<T, D, NT, 2>() + plan, st>>>(P, a);
    CUDA_TRY(cudaGetLastError());
    return launch_merge<T, D, 8 * NT, kP4KT, 0, kP4Lead>(P, a, blocks, st);
}

// fp32 queries: units of 8 rows whatever the call. With more rows a sequence every unit reads and expands the cache for itself: 32 heads of
// 128 on 8 KV heads, 2047 prompt tokens 999 us (bytes and products 62), 4 x 512 behind 4096 shared ones 1350 (88); one token behind
// 131072 54 (bf16 45).
template <int D>
int attend4_fp32(const PagedView& P, const Attend& a, cudaStream_t st) {
    static bool done[kMaxDevices];
    int dev, rc = this_device(&dev);
    if (!rc && !done[dev]) {
        rc = opt_in_few<float, D, 1>();
        done[dev] = !rc;
    }
    return rc ? rc : attend_few<float, D, 1>(P, a, st);
}

template <int D>
int attend4_bf16(const PagedView& P, const Attend& a, cudaStream_t st) {
    typedef __nv_bfloat16 T;
    static bool done[kMaxDevices];
    constexpr size_t fixed = 1024 + ((sizeof(PtSmem<D, true>) + 15) & ~(size_t)15);
    int dev, rc = this_device(&dev);
    if (!rc && !done[dev]) {                          // all kinds, whichever this call takes
        rc = opt_in_few<T, D, 1>();
        if (!rc) rc = opt_in_few<T, D, 2>();
        if (!rc) rc = opt_in(paged_attend_tc_kernel<D, false, true>, paged_merge_kernel<T, D, kPtRU, kPtKT, 1, kPtLead>, fixed + plan_bytes(kPlanMax));
        done[dev] = !rc;
    }
    if (rc) return rc;
    // By the mean of rows a sequence, or a group where several sequences share a prefix. 16 sequences of 8192 tokens, 8 KV heads, in
    // units of 8 rows / units of 16 / units of 256 on the other tensor cores: 4 rows 46 / 56 / 101 us, 8 rows 45 / 56 / 102, 12 rows
    // 73 / 58 / 105, 24 rows 101 / 97 / 113, 32 rows 131 / 99 / 121. A prefix of 32768 tokens before single tokens (4 rows each): 2
    // sequences 31 / 27 / 43, 4 45 / 29 / 48, 8 75 / 41 / 58.
    // The mean is all that the host knows, so a prompt among many single tokens takes the units of the others: 255 tokens behind 1000 each
    // with a prompt of 1500 319 us (in units of 16), with one of 2000 320 (in units of 256); the tokens alone 88, the prompt of 1500 alone 84.
    const long long rows = (long long)a.n << a.g_shift;
    const bool shared = P.groups && P.groups < P.B;
    if (!shared && rows <= 8LL * P.B) return attend_few<T, D, 1>(P, a, st);
    if (rows <= 32LL * (shared ? P.groups : P.B)) return attend_few<T, D, 2>(P, a, st);
    CUtensorMap mq;
    const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)a.H, (cuuint64_t)a.n};
    const cuuint64_t strides[2] = {(cuuint64_t)a.q.hs * 2, (cuuint64_t)a.q.ts * 2};
    const cuuint32_t box[3] = {64, 1u << a.g_shift, 32u >> a.g_shift};           // 32 rows
    rc = make_map(&mq, a.q.p, 3, dims, strides, box);
    if (rc) return rc;
    paged_attend_tc_kernel<D, false, true><<<kSMs, kPtThreads4, fixed + plan_bytes(P.B + P.groups), st>>>(P, a, mq, mq, mq);
    CUDA_TRY(cudaGetLastError());
    return launch_merge<T, D, kPtRU, kPtKT, 1, kPtLead>(P, a, kSMs, st);
}

}  // namespace

extern "C" {

int subgen_paged4_append(const subgen_pages4* cache, const subgen_batch* batch, const subgen_qk_args* x, void* stream) {
    const char* fn = "subgen_paged4_append";
    PagedView P;
    if (!cache || !batch || !x) return fail(SUBGEN_EINVAL, "%s: cache, batch and args must not be NULL", fn);
    const bool has_q = x->q.p;
    const int Hkv = cache->Hkv, d = cache->d, dtype = x->dtype;
    int rc = check_shape(fn, x->n, has_q ? x->H : 1, Hkv, d, dtype);
    if (!rc) rc = check_cache4(fn, cache, batch, &P);
    if (!rc) rc = check_rope(fn, &x->rope, d);
    if (!rc) rc = check_norm(fn, x->wq, x->wk, x->eps);
    if (rc || x->n == 0 || batch->B == 0) return rc;
    NormRope a;
    memset(&a, 0, sizeof a);
    rc = check_heads(fn, "k", &x->k, x->n, Hkv, d, dtype, &a.k);
    if (!rc) rc = check_heads(fn, "v", &x->v, x->n, Hkv, d, dtype, &a.v);
    if (!rc && has_q) rc = check_heads(fn, "q", &x->q, x->n, x->H, d, dtype, &a.q);
    if (!rc && has_q) rc = check_heads(fn, "q_out", &x->q_out, x->n, x->H, d, dtype, &a.qo);
    if (!rc && has_q) rc = check_output(fn, "q_out", a.qo, x->n, x->H, d, a.q, {a.k.p, a.v.p, P.K});
    if (rc) return rc;
    fill_norm_rope(&a, x, has_q ? x->H : 0, Hkv);
    return norm_rope<2>(a, P, d, dtype, (cudaStream_t)stream);
}

int subgen_paged4_load(const subgen_pages4* cache, const int64_t* slots, int n, const subgen_heads* K, const subgen_heads* V, int dtype, void* stream) {
    const char* fn = "subgen_paged4_load";
    PagedView P;
    if (!cache || !K || !V) return fail(SUBGEN_EINVAL, "%s: cache, K and V must not be NULL", fn);
    const int Hkv = cache->Hkv, d = cache->d;
    int rc = check_shape(fn, n, 1, Hkv, d, dtype);
    if (!rc) rc = check_pool(fn, cache, &P);
    if (rc || n == 0) return rc;
    if (!slots || ((uintptr_t)slots & 7)) return fail(SUBGEN_EINVAL, "%s: slots must not be NULL and be 8-byte aligned", fn);
    if (!K->p && !V->p) return fail(SUBGEN_EINVAL, "%s: K and V must not both be without a pointer", fn);
    Load4 a;
    memset(&a, 0, sizeof a);
    const HeadsView none = {nullptr, 0, 0};
    if (K->p) rc = check_heads(fn, "K", K, n, Hkv, d, dtype, &a.k);
    if (!rc && V->p) rc = check_heads(fn, "V", V, n, Hkv, d, dtype, &a.v);
    if (!rc && K->p) rc = check_output(fn, "K", a.k, n, Hkv, d, none, {a.v.p, P.K, slots});
    if (!rc && V->p) rc = check_output(fn, "V", a.v, n, Hkv, d, none, {a.k.p, P.K, slots});
    if (rc) return rc;
    a.pool = P.K; a.ps = P.ps; a.hs = P.hs;
    a.slots = (const long long*)slots;
    a.n = n; a.Hkv = Hkv; a.pages = P.pages; a.page_shift = P.page_shift; a.status = P.status;
    cudaStream_t st = (cudaStream_t)stream;
    if (dtype == SUBGEN_DTYPE_FP32) return d == 64 ? launch_load<float, 64>(a, st) : launch_load<float, 128>(a, st);
    return d == 64 ? launch_load<__nv_bfloat16, 64>(a, st) : launch_load<__nv_bfloat16, 128>(a, st);
}

size_t subgen_paged4_workspace_bytes(const subgen_pages4* cache, const subgen_batch* batch, int n, int H) {
    const char* fn = "subgen_paged4_workspace_bytes";
    PagedView P;
    if (!cache || !batch) { fail(SUBGEN_EINVAL, "%s: cache and batch must not be NULL", fn); return 0; }
    if (check_shape(fn, n, H, cache->Hkv, cache->d, SUBGEN_DTYPE_BF16) || check_cache4(fn, cache, batch, &P)) return 0;
    return (size_t)slot_count(P, n, H) * (cache->d * sizeof(float) + sizeof(float2));
}

int subgen_paged4_attend(const subgen_pages4* cache, const subgen_batch* batch, const subgen_attend_args* x, int dtype, void* stream) {
    const char* fn = "subgen_paged4_attend";
    PagedView P;
    if (!cache || !batch || !x) return fail(SUBGEN_EINVAL, "%s: cache, batch and args must not be NULL", fn);
    const int n = x->n, H = x->H, d = cache->d;
    int rc = check_shape(fn, n, H, cache->Hkv, d, dtype);
    if (!rc) rc = check_cache4(fn, cache, batch, &P);
    if (rc) return rc;
    Attend a;
    rc = check_attend(fn, x, P, d, dtype, &a);
    if (rc || n == 0 || batch->B == 0) return rc;
    cudaStream_t st = (cudaStream_t)stream;
    if (dtype == SUBGEN_DTYPE_BF16) return d == 64 ? attend4_bf16<64>(P, a, st) : attend4_bf16<128>(P, a, st);
    return d == 64 ? attend4_fp32<64>(P, a, st) : attend4_fp32<128>(P, a, st);
}

int subgen_page_step(const subgen_page_step_args* x, void* stream) {
    const char* fn = "subgen_page_step";
    if (!x) return fail(SUBGEN_EINVAL, "%s: args must not be NULL", fn);
    int rc = check_pages(fn, x->pages, x->page);
    if (rc) return rc;
    if (x->B < 1 || x->B > kPlanMax || x->n < 0) return fail(SUBGEN_EINVAL, "%s: B must be 1 to %d, n >= 0", fn, kPlanMax);
    if (!x->table || !x->free_pages || !x->free_count || !x->lengths || !x->added || !x->free_count_out || !x->lengths_out || !x->cu_q ||
        (x->n && (!x->slots || !x->positions)))
        return fail(SUBGEN_EINVAL, "%s: only ended, first, status and sources may be NULL", fn);
    if (x->table_stride <= 0 || (long long)x->table_stride * x->page > 0x7fffffffLL - 1024)
        return fail(SUBGEN_EINVAL, "%s: table_stride must be positive, a row of fewer than 2^31 - 1024 tokens", fn);
    if ((long long)x->B * x->table_stride >= 0x7fffffffLL) return fail(SUBGEN_EINVAL, "%s: a table must hold fewer than 2^31 - 1 pages", fn);
    if ((uintptr_t)x->slots & 7) return fail(SUBGEN_EINVAL, "%s: slots must be 8-byte aligned", fn);
    PageStep a;
    a.B = x->B; a.n = x->n; a.pages = x->pages; a.page_shift = shift_of(x->page); a.stride = x->table_stride;
    a.table = x->table; a.free = x->free_pages;
    a.free_count = x->free_count; a.lengths = x->lengths; a.added = x->added; a.ended = x->ended; a.first = x->first;
    a.free_count_out = x->free_count_out; a.lengths_out = x->lengths_out; a.cu_q = x->cu_q; a.positions = x->positions; a.sources = x->sources;
    a.slots = (long long*)x->slots;
    a.status = x->status;
    // Slots and positions: in the one kernel / by the second (us a call, in a graph): 64 rows with 64 tokens 5.2 / 6.4, 4096 6.3 / 6.9; 128 rows with
    // 8192 6.5 / 7.0; 1024 rows with 8192 7.2 / 8.4, 16384 8.3 / 8.4, 112640 19.1 / 8.1.
    a.split = x->n > 4 * kStepThreads;
    static bool done[kMaxDevices];
    int dev;
    rc = this_device(&dev);
    if (rc) return rc;
    if (!done[dev]) {                                 // loads both, so that a call of any size may be captured later
        cudaFuncAttributes at;
        CUDA_TRY(cudaFuncGetAttributes(&at, page_step_kernel));
        CUDA_TRY(cudaFuncGetAttributes(&at, page_slots_kernel));
        done[dev] = true;
    }
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof cfg);
    // Something to share out. One block / the cluster: 64 rows with a token each 5.2 / 5.7, 256 5.5 / 6.0; 64 rows with 2048 tokens 6.7 / 6.3,
    // 4096 7.9 / 6.3. Pages that rows give back are not known here: 4 x 512 of them 6.5 / 6.7, 8 x 1024 8.5 / 6.9, 65536 25.8 / 7.9.
    const int blocks = x->n > kStepThreads || x->B > 128 ? kStepCluster : 1;
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(kStepThreads);
    cfg.stream = (cudaStream_t)stream;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)blocks;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    CUDA_TRY(cudaLaunchKernelEx(&cfg, page_step_kernel, a));
    if (!a.split) return SUBGEN_OK;
    const int parts = (x->n - 1) / kSlotThreads + 1;      // a turn a warp
    cfg.gridDim = dim3((unsigned)(parts < 4 * kSMs ? parts : 4 * kSMs));
    cfg.blockDim = dim3(kSlotThreads);
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    CUDA_TRY(cudaLaunchKernelEx(&cfg, page_slots_kernel, a));
    return SUBGEN_OK;
}

}  // extern "C"
