// The calls around a hit: append new keys and values to the paged pool, attend to what it holds.
// Host side: checks of the arguments, scratch, choice of kernel, launches.
// Included at the end of lsmkv.cu (needs the context's internals).
#pragma once

#include <cudaTypedefs.h>

namespace {

// The pools these calls take.
bool serve_geom_ok(const lsmkv_ctx *ctx, uint32_t layer, uint32_t dtype)
{
    const lsmkv_geom_t &g = ctx->geom;
    return g.elem_bytes == 2 && g.head_dim % 8 == 0 && g.head_dim <= 256 && layer < g.n_layers &&
           (dtype == LSMKV_BF16 || dtype == LSMKV_F16);
}

bool seqs_ok(const lsmkv_seqs_t *s)
{
    return s && s->n_seq && s->max_new && s->new_off && s->kv_len && s->page_off && s->page_table;
}

bool rows_ok(const lsmkv_rows_t *r)
{
    return r && r->data && aligned16(r->data) && r->token_stride % 8 == 0 && r->head_stride % 8 == 0 &&
           r->token_stride <= 0xFFFFFFFFull && r->head_stride <= 0xFFFFFFFFull;
}

// Whether two sets of rows are the same ones (strides of an extent of one aside).
bool rows_same(const lsmkv_rows_t &a, const lsmkv_rows_t &b, uint64_t n_new, uint32_t heads)
{
    return a.data == b.data && (n_new == 1 || a.token_stride == b.token_stride) &&
           (heads == 1 || a.head_stride == b.head_stride);
}

// Whether the memory of two sets of rows may meet. Rows that lie side by side in the tokens of one
// buffer do not.
bool rows_meet(const lsmkv_rows_t &a, const lsmkv_rows_t &b, uint64_t n_new, uint32_t heads, uint32_t head_dim)
{
    auto span = [&](const lsmkv_rows_t &r) { return 2 * ((heads - 1ull) * r.head_stride + head_dim); };
    auto begin = [&](const lsmkv_rows_t &r) { return reinterpret_cast<uintptr_t>(r.data); };
    auto end = [&](const lsmkv_rows_t &r) { return begin(r) + 2 * (n_new - 1) * r.token_stride + span(r); };
    if (begin(a) >= end(b) || begin(b) >= end(a)) return false;
    const uint64_t period = 2 * a.token_stride;
    if (a.token_stride == b.token_stride && span(a) <= period && span(b) <= period) {
        const uint64_t ahead = begin(b) >= begin(a) ? (begin(b) - begin(a)) % period
                                                    : (period - (begin(a) - begin(b)) % period) % period;
        return ahead < span(a) || ahead + span(b) > period;      // b's token begins so far behind one of a's
    }
    return true;
}

SeqArgs seq_args(const lsmkv_seqs_t *s)
{
    SeqArgs a;
    a.n_new = s->n_new;
    a.n_seq = s->n_seq;
    a.max_new = s->max_new;
    a.new_off = s->new_off;
    a.kv_len = s->kv_len;
    a.page_off = s->page_off;
    a.page_table = s->page_table;
    return a;
}

// A launch of an attend call: behind another one of the same call (follows) it may start before
// that one has ended (the kernels wait for it themselves).
template <typename... P, typename... A>
cudaError_t start(lsmkv_ctx *ctx, cudaStream_t s, bool follows, void (*kern)(P...), dim3 grid, unsigned threads,
                  size_t smem, const A &...args)
{
    cudaLaunchAttribute early;
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t c = {};
    c.gridDim = grid;
    c.blockDim = threads;
    c.dynamicSmemBytes = smem;
    c.stream = s;
    c.attrs = &early;
    c.numAttrs = follows ? 1 : 0;
    ++ctx->launches;
    return cudaLaunchKernelEx(&c, kern, args...);
}

template <typename T, int DP, int NB>
cudaError_t start_few(lsmkv_ctx *ctx, cudaStream_t s, bool follows, const AttendJob &job)
{
    using Sh = FewShape<DP, NB>;
    return start(ctx, s, follows, k_attend_few<T, DP, NB>, (unsigned)ctx->sm_count, Sh::kThreads, Sh::kSmem, job);
}

// rows8: no row tile has more than 8 rows.
template <typename T>
int launch_few(lsmkv_ctx *ctx, cudaStream_t s, bool follows, const AttendJob &job, bool rows8)
{
    if (job.head_dim <= 64)
        CU(ctx, (rows8 ? start_few<T, 64, 1> : start_few<T, 64, 2>)(ctx, s, follows, job));
    else if (job.head_dim <= 128)
        CU(ctx, (rows8 ? start_few<T, 128, 1> : start_few<T, 128, 2>)(ctx, s, follows, job));
    else
        CU(ctx, (rows8 ? start_few<T, 256, 1> : start_few<T, 256, 2>)(ctx, s, follows, job));
    return LSMKV_OK;
}

// A tensor map of 16-bit floats, swizzled; dims and box from the innermost on, strides in elements
// of the dimensions behind it.
template <int R>
bool make_map(uint32_t dtype, const void *base, const uint64_t (&dims)[R], const uint64_t (&strides)[R - 1],
              const uint32_t (&box)[R], CUtensorMap *map)
{
    static const PFN_cuTensorMapEncodeTiled_v12000 encode = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) !=
                cudaSuccess || found != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            p = nullptr;
        }
        return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
    }();
    if (!encode) return false;
    cuuint64_t d[R], st[R - 1];
    cuuint32_t bx[R], step[R];
    for (int i = 0; i < R; ++i) {
        if (dims[i] == 0 || dims[i] > 0x7FFFFFFFull) return false;       // coordinates are 32-bit
        d[i] = dims[i];
        bx[i] = box[i];
        step[i] = 1;
        if (i) st[i - 1] = strides[i - 1] * 2;
    }
    return encode(map, dtype == LSMKV_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, R,
                  const_cast<void *>(base), d, st, bx, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T>
int launch_many(lsmkv_ctx *ctx, cudaStream_t s, bool follows, AttendJob &job)
{
    const unsigned sm = (unsigned)ctx->sm_count;
    // Tokens of a box: the largest power of two that divides the page, at most 64. The swizzle's
    // unit is 8 rows, so boxes of fewer than 8 are out and cp.async takes such pages.
    const lsmkv_geom_t &g = ctx->geom;
    const uint32_t dtype = std::is_same<T, __half>::value ? LSMKV_F16 : LSMKV_BF16;
    job.box_rows = std::min(g.page_tokens & (~g.page_tokens + 1), 64u);
    CUtensorMap map, q_map;
    std::memset(&map, 0, sizeof(map));
    std::memset(&q_map, 0, sizeof(q_map));
    // (the map's address is filled in by the kernel, which finds it in the pool's table)
    const uint64_t row = (uint64_t)g.n_kv_heads * g.head_dim, D = g.head_dim;
    bool boxes = job.box_rows >= 8 && job.num_pages < 0x7FFFFFFFull / g.page_tokens;
    // A box with all elements of a head, where they are whole blocks of 64: half as many boxes at
    // head_dim 128, and the engine's time goes by boxes (pages of 16: 909 -> 1005 TFLOP/s at 8k keys).
    job.wide_boxes = D % 64 == 0;
    if (boxes && job.wide_boxes)
        boxes = make_map<5>(dtype, ctx->d_attend, {64, 8, D / 64, job.num_pages * g.page_tokens / 8, g.n_kv_heads},
                            {row, 64, 8 * row, D}, {64, 8, (uint32_t)D / 64, job.box_rows / 8, 1}, &map);
    else if (boxes)
        boxes = make_map<3>(dtype, ctx->d_attend, {D, g.n_kv_heads, job.num_pages * g.page_tokens}, {D, row},
                            {64, 1, job.box_rows}, &map);
    // The 128 rows of half a tile are a box of queries when the heads of a KV head divide them.
    job.q_boxes = boxes && job.group <= 128 && (job.group & (job.group - 1)) == 0 &&
                  make_map<3>(dtype, job.q, {D, job.n_q_heads, job.seqs.n_new}, {job.q_hs, job.q_ts},
                              {64, job.group, 128 / job.group}, &q_map);
    if (job.head_dim <= 64)
        CU(ctx, start(ctx, s, follows, boxes ? k_attend_many<T, 64, true> : k_attend_many<T, 64, false>, sm,
                      ManyShape<64>::kThreads, ManyShape<64>::kSmem, job, map, q_map));
    else
        CU(ctx, start(ctx, s, follows, boxes ? k_attend_many<T, 128, true> : k_attend_many<T, 128, false>, sm,
                      ManyShape<128>::kThreads, ManyShape<128>::kSmem, job, map, q_map));
    CU(ctx, start(ctx, s, true, k_attend_merge<T>, dim3(sm, 256 / kMergeBlockRows), 256, 0, job));
    return LSMKV_OK;
}

// The tcgen05 kernel takes heads of up to 128 elements.
bool many_takes(const lsmkv_ctx *ctx) { return ctx->geom.head_dim <= 128; }

// Whether a sequence of max_new new tokens has more rows than one tile of the few-row kernel.
bool many_rows(const lsmkv_ctx *ctx, uint32_t max_new, uint32_t group)
{
    return many_takes(ctx) && (uint64_t)max_new * group > 16;
}

uint32_t part_dp(const lsmkv_ctx *ctx)
{
    return ctx->geom.head_dim <= 64 ? 64 : ctx->geom.head_dim <= 128 ? 128 : 256;
}

// The groups' common keys, all groups by one kernel: whatever their rows, reading the keys once
// is what counts. A batch of at most 64 rows in all goes by the few-row kernel all the same: its up
// to four row tiles find the keys in L2, and it starts and ends faster (one group of 8 sequences,
// G = 4, 1024 common tokens: 26.6 us a call against 30.9).
template <typename T>
int launch_prefix(lsmkv_ctx *ctx, cudaStream_t s, AttendJob &job)
{
    job.prefix_pass = 1;
    job.rows_lo = 0;
    job.rows_hi = 0xFFFFFFFFu;
    const uint64_t rows = job.seqs.n_new * job.group;
    job.beside = 0;
    const int rc = many_takes(ctx) && rows > 64 ? launch_many<T>(ctx, s, false, job)
                                                 : launch_few<T>(ctx, s, false, job, rows <= 8);
    job.prefix_pass = 0;
    return rc;
}

// The sequences: those of few rows and those of many, each by its kernel.
template <typename T>
int launch_own(lsmkv_ctx *ctx, cudaStream_t s, AttendJob &job)
{
    // Up to 16 rows are one tile of the few-row kernel; beyond, it would read the keys once for
    // every 16 rows, where the many-row kernel reads them once for 256.
    const bool mma = many_takes(ctx);
    job.rows_lo = 0;
    job.rows_hi = mma ? 16 : 0xFFFFFFFFu;
    const uint64_t most = (uint64_t)job.seqs.max_new * job.group;
    float *const many_parts = job.parts;
    job.parts = job.few_parts;
    const int rc = launch_few<T>(ctx, s, job.skip != nullptr, job, most <= 8);
    job.parts = many_parts;
    if (rc != LSMKV_OK || !many_rows(ctx, job.seqs.max_new, job.group)) return rc;
    // side by side, unless a prefix pass is still ahead of both
    job.beside = job.skip == nullptr;
    job.rows_lo = 16;
    job.rows_hi = 0xFFFFFFFFu;
    return launch_many<T>(ctx, s, true, job);
}

// Two part slots of so many rows for every CTA.
size_t part_bytes(const lsmkv_ctx *ctx, uint32_t rows)
{
    return (size_t)ctx->sm_count * 2 * rows * (part_dp(ctx) + 2) * 4;
}

// Scratch of the attend kernels for n_seq sequences: counters, descriptors of cut tiles, tensor
// maps, the spans' beginnings, the items' tiles, parts. Returns its size.
size_t place_attend(const lsmkv_ctx *ctx, void *at, uint32_t n_seq, AttendJob *job)
{
    IoLayout l(at);
    const size_t sm = (size_t)ctx->sm_count;
    job->arrived = reinterpret_cast<unsigned int *>(l.take<unsigned char>(attend_counter_bytes(ctx)));
    job->cuts = l.take<CutDesc>(sm);
    job->maps = l.take<unsigned char>(sm * 256);
    job->span_begin = l.take<uint64_t>(sm + 1);
    job->few_parts = l.take<float>(part_bytes(ctx, 16) / 4);
    job->parts = many_takes(ctx) ? l.take<float>(part_bytes(ctx, 256) / 4) : job->few_parts;
    job->tile_base = l.take<uint32_t>((size_t)n_seq + 1);
    return l.at;
}

int ensure_attend(lsmkv_ctx *ctx, cudaStream_t s, uint32_t n_seq, AttendJob *job)
{
    const size_t bytes = place_attend(ctx, nullptr, n_seq, job);
    if (!ctx->d_attend || bytes > ctx->attend_cap) {
        // room for a few sequences more than asked for: a growing batch does not allocate every time
        const int rc = enlarge_scratch(ctx, &ctx->d_attend, &ctx->attend_cap, bytes + 16384, __LINE__);
        if (rc != LSMKV_OK) return rc;
        const cudaError_t e = cudaMemsetAsync(ctx->d_attend, 0, attend_counter_bytes(ctx), s);
        if (e != cudaSuccess) {
            release_scratch(ctx, &ctx->d_attend, &ctx->attend_cap, __LINE__);
            return cuda_fail(ctx, e, __LINE__);
        }
    }
    place_attend(ctx, ctx->d_attend, n_seq, job);
    return LSMKV_OK;
}

int attend(lsmkv_ctx *ctx, void *stream, uint32_t layer, uint32_t dtype, const lsmkv_seqs_t *seqs,
           const lsmkv_groups_t *groups, uint32_t n_q_heads, const lsmkv_rows_t *q,
           const lsmkv_pool_t *pool, float scale, const lsmkv_rows_t *out, float *lse_out)
{
    if (!ctx || !seqs) return LSMKV_EINVAL;
    if (!serve_geom_ok(ctx, layer, dtype)) return LSMKV_EINVAL;
    if (seqs->n_new == 0) return LSMKV_OK;
    if (!seqs_ok(seqs) || !rows_ok(q) || !rows_ok(out) || !pool || !pool->kv_ptrs) return LSMKV_EINVAL;
    if (n_q_heads == 0 || n_q_heads % ctx->geom.n_kv_heads != 0 || !std::isfinite(scale)) return LSMKV_EINVAL;
    // rows are numbered in 32 bits: new tokens, and rows under a KV head up to whole tiles
    if (seqs->n_new > 0x7FFFFFFFull || seqs->n_new * (n_q_heads / ctx->geom.n_kv_heads) > 0xFFFFFF00ull)
        return LSMKV_EINVAL;
    if (groups && groups->n_group && (!groups->group_off || !groups->shared_pages)) return LSMKV_EINVAL;
    if (groups && groups->n_group > seqs->n_seq) return LSMKV_EINVAL;
    const bool shared = groups && groups->n_group;
    DeviceGuard guard(ctx->device);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    AttendJob job;
    std::memset(&job, 0, sizeof(job));
    int rc = ensure_attend(ctx, s, seqs->n_seq, &job);
    if (rc != LSMKV_OK) return rc;
    job.seqs = seq_args(seqs);
    job.kv_ptrs = pool->kv_ptrs;
    job.num_pages = pool->num_pages;
    job.layer = layer;
    job.n_layers = ctx->geom.n_layers;
    job.page_tokens = ctx->geom.page_tokens;
    job.n_kv_heads = ctx->geom.n_kv_heads;
    job.head_dim = ctx->geom.head_dim;
    job.n_q_heads = n_q_heads;
    job.group = n_q_heads / ctx->geom.n_kv_heads;
    job.rows_lo = 0;
    job.rows_hi = 0xFFFFFFFFu;
    job.q = q->data;
    job.q_ts = q->token_stride;
    job.q_hs = q->head_stride;
    job.out = out->data;
    job.o_ts = out->token_stride;
    job.o_hs = out->head_stride;
    job.lse = lse_out;
    job.scale_log2 = scale * kLog2e;
    job.dp = part_dp(ctx);
    job.wait_cycles = ctx->wait_cycles;
    job.test_drop = ctx->test_drop_piece < 0 ? ~0ull : (uint64_t)ctx->test_drop_piece;
    job.st = ctx->d_status;
    if (shared) {
        const uint64_t heads = seqs->n_new * n_q_heads;
        auto place = [&](void *at) {
            IoLayout l(at);
            job.skip = l.take<uint32_t>(seqs->n_seq);
            job.pre_o = l.take<float>(heads * ctx->geom.head_dim);
            job.pre_lse = l.take<float>(heads);
            return l.at;
        };
        const size_t bytes = place(nullptr);
        if (!ctx->d_prefix || bytes > ctx->prefix_cap) {
            rc = enlarge_scratch(ctx, &ctx->d_prefix, &ctx->prefix_cap, bytes, __LINE__);
            if (rc != LSMKV_OK) return rc;
        }
        place(ctx->d_prefix);
        job.n_group = groups->n_group;
        job.group_off = groups->group_off;
        job.shared_pages = groups->shared_pages;
    }
    LaunchTimer timer(ctx, s, LSMKV_K_ATTEND);
    // Where the output lies over the queries: rows over themselves are fine, each is written after it was
    // read. But a row of a many-row tile that comes out undefined beside later tokens may be computed once more from its
    // query, which must not have become output by then; and in another layout a row lies over other rows.
    if (rows_meet(*q, *out, seqs->n_new, n_q_heads, ctx->geom.head_dim) &&
        ((many_rows(ctx, seqs->max_new, job.group) && seqs->max_new > 1) ||
         !rows_same(*q, *out, seqs->n_new, n_q_heads))) {
        const uint64_t pieces = seqs->n_new * n_q_heads * (ctx->geom.head_dim / 8);
        if (!ctx->d_queries || pieces * 16 > ctx->queries_cap) {
            rc = enlarge_scratch(ctx, &ctx->d_queries, &ctx->queries_cap, pieces * 16, __LINE__);
            if (rc != LSMKV_OK) return rc;
        }
        k_gather_rows<<<merge_grid(ctx, pieces), 256, 0, s>>>(
            static_cast<const uint4 *>(q->data), q->token_stride / 8, q->head_stride / 8, seqs->n_new, n_q_heads,
            ctx->geom.head_dim / 8, static_cast<uint4 *>(ctx->d_queries));
        ++ctx->launches;
        CU(ctx, cudaGetLastError());
        job.q = ctx->d_queries;
        job.q_hs = ctx->geom.head_dim;
        job.q_ts = (uint64_t)n_q_heads * ctx->geom.head_dim;
    }
    const bool bf = dtype == LSMKV_BF16;
    if (shared) {
        rc = bf ? launch_prefix<__nv_bfloat16>(ctx, s, job) : launch_prefix<__half>(ctx, s, job);
        if (rc != LSMKV_OK) return rc;
    }
    return bf ? launch_own<__nv_bfloat16>(ctx, s, job) : launch_own<__half>(ctx, s, job);
}

}  // namespace

extern "C" int lsmkv_append_batch(lsmkv_ctx *ctx, void *stream, uint32_t layer, uint32_t dtype,
                                  const lsmkv_seqs_t *seqs, const lsmkv_rows_t *k,
                                  const lsmkv_rows_t *v, const lsmkv_pool_t *pool,
                                  const lsmkv_rope_t *rope, uint32_t n_q_heads,
                                  const lsmkv_rows_t *q_in, const lsmkv_rows_t *q_out,
                                  const void *q_norm, const void *k_norm, float eps)
{
    if (!ctx || !seqs) return LSMKV_EINVAL;
    if (!serve_geom_ok(ctx, layer, dtype)) return LSMKV_EINVAL;
    if (seqs->n_new == 0) return LSMKV_OK;
    if (!seqs_ok(seqs) || !rows_ok(k) || !rows_ok(v) || !pool || !pool->kv_ptrs) return LSMKV_EINVAL;
    if (n_q_heads ? !rows_ok(q_in) || !rows_ok(q_out) : q_in || q_out || q_norm) return LSMKV_EINVAL;
    if (!aligned16(q_norm) || !aligned16(k_norm)) return LSMKV_EINVAL;
    if ((q_norm || k_norm) && !(eps >= 0.f && std::isfinite(eps))) return LSMKV_EINVAL;
    const lsmkv_geom_t &g = ctx->geom;
    if (rope && (!rope->table || !aligned16(rope->table) || rope->rot_dim % 2 || rope->rot_dim == 0 ||
                 rope->rot_dim > g.head_dim || rope->interleaved > 1))
        return LSMKV_EINVAL;
    if (n_q_heads > 0x10000u || seqs->n_new > 0x7FFFFFFFull) return LSMKV_EINVAL;
    AppendJob job;
    std::memset(&job, 0, sizeof(job));
    job.seqs = seq_args(seqs);
    job.kv_ptrs = pool->kv_ptrs;
    job.num_pages = pool->num_pages;
    job.layer = layer;
    job.n_layers = g.n_layers;
    job.page_tokens = g.page_tokens;
    job.n_kv_heads = g.n_kv_heads;
    job.head_dim = g.head_dim;
    job.n_q_heads = n_q_heads;
    job.k = k->data;
    job.k_ts = k->token_stride;
    job.k_hs = k->head_stride;
    job.v = v->data;
    job.v_ts = v->token_stride;
    job.v_hs = v->head_stride;
    if (n_q_heads) {
        job.q = q_in->data;
        job.q_ts = q_in->token_stride;
        job.q_hs = q_in->head_stride;
        job.q_out = q_out->data;
        job.o_ts = q_out->token_stride;
        job.o_hs = q_out->head_stride;
    }
    if (rope) {
        job.table = rope->table;
        job.positions = rope->positions;
        job.n_pos = rope->n_pos;
        job.rot_dim = rope->rot_dim;
        job.interleaved = rope->interleaved;
    }
    job.q_norm = q_norm;
    job.k_norm = k_norm;
    job.eps = eps;
    job.st = ctx->d_status;

    DeviceGuard guard(ctx->device);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    LaunchTimer timer(ctx, s, LSMKV_K_ATTEND);
    const uint32_t slots = n_q_heads + 2 * g.n_kv_heads;
    // Whole 16-byte pieces on both sides of a pair (or no pair that leaves its piece): vector
    // form. Otherwise element by element.
    const bool vec = job.rot_dim % (job.interleaved ? 8 : 16) == 0;
    const bool bf = dtype == LSMKV_BF16;
    if (vec) {
        const uint32_t lanes = job.interleaved || !job.rot_dim
                                   ? (g.head_dim / 8 + 1) / 2
                                   : job.rot_dim / 16 + (g.head_dim - job.rot_dim + 15) / 16;
        while ((1u << job.lane_log2) < lanes) ++job.lane_log2;
        // as many tokens a block as one round of blocks, four a SM, leaves; at most one a warp
        const uint64_t round = (uint64_t)ctx->sm_count * 4;
        job.tokens = (uint32_t)std::min<uint64_t>(kAppendWarps, (seqs->n_new + round - 1) / round);
        const uint64_t grid = (seqs->n_new + job.tokens - 1) / job.tokens;
        // (that form has more registers: two blocks a SM; 512 tokens of 36 heads 8.9 us, 7.3 without)
        auto kern = seqs->n_new <= (uint64_t)ctx->sm_count * 2
                        ? (bf ? k_append<__nv_bfloat16, true> : k_append<__half, true>)
                        : (bf ? k_append<__nv_bfloat16, false> : k_append<__half, false>);
        kern<<<(unsigned)grid, kAppendWarps * 32, 0, s>>>(job);
    } else {
        // as many warps a token as keep the GPU busy
        const uint64_t fill = (uint64_t)ctx->sm_count * 16;
        job.parts = (uint32_t)std::min<uint64_t>((fill + seqs->n_new - 1) / seqs->n_new, slots);
        const uint64_t grid = (seqs->n_new * job.parts + 3) / 4;
        (bf ? k_append_elements<__nv_bfloat16> : k_append_elements<__half>)<<<(unsigned)grid, 128, 0, s>>>(job);
    }
    ++ctx->launches;
    CU(ctx, cudaGetLastError());
    return LSMKV_OK;
}

extern "C" int lsmkv_attend_batch(lsmkv_ctx *ctx, void *stream, uint32_t layer, uint32_t dtype,
                                  const lsmkv_seqs_t *seqs, uint32_t n_q_heads,
                                  const lsmkv_rows_t *q, const lsmkv_pool_t *pool, float scale,
                                  const lsmkv_rows_t *out, float *lse_out)
{
    return attend(ctx, stream, layer, dtype, seqs, nullptr, n_q_heads, q, pool, scale, out, lse_out);
}

extern "C" int lsmkv_attend_shared_batch(lsmkv_ctx *ctx, void *stream, uint32_t layer,
                                         uint32_t dtype, const lsmkv_seqs_t *seqs,
                                         const lsmkv_groups_t *groups, uint32_t n_q_heads,
                                         const lsmkv_rows_t *q, const lsmkv_pool_t *pool,
                                         float scale, const lsmkv_rows_t *out, float *lse_out)
{
    if (!groups) return LSMKV_EINVAL;
    return attend(ctx, stream, layer, dtype, seqs, groups, n_q_heads, q, pool, scale, out, lse_out);
}
