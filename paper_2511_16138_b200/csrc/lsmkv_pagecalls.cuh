// The page calls: release, fork, compaction, copies. Host side: checks of the arguments, scratch, launches.
// Included at the end of lsmkv.cu (needs the context's internals).
#pragma once

namespace {

bool tables_ok(const lsmkv_tables_t *t)
{
    return t->kv_len && t->page_off && (t->page_table || !t->n_entries);
}

TableArgs table_args(const lsmkv_tables_t *t)
{
    TableArgs a;
    a.n_entries = t->n_entries;
    a.n_seq = t->n_seq;
    a.kv_len = t->kv_len;
    a.page_off = t->page_off;
    a.page_table = t->page_table;
    return a;
}

// Slabs as the movers take them, and the launch shape: one CTA a SM, a warp for every stage.
struct Mover {
    SlabArgs a;
    unsigned grid, threads;
    size_t smem;
};

Mover slab_mover(const lsmkv_ctx *ctx, const lsmkv_pool_t *pool)
{
    const lsmkv_geom_t &g = ctx->geom;
    Mover m;
    m.a.kv_ptrs = pool->kv_ptrs;
    m.a.num_pages = pool->num_pages;
    m.a.buffers = 2 * g.n_layers;
    m.a.page_bytes = (uint32_t)ctx->page_bytes;
    m.a.body_bytes = ctx->pool8 ? ctx->codes.code_bytes : (uint32_t)ctx->page_bytes;
    m.a.page_tokens = g.page_tokens;
    const uint64_t piece = std::min<uint64_t>((uint64_t)ctx->copy_stage_bytes, ctx->page_bytes);
    m.a.piece_bytes = (uint32_t)piece;
    m.a.wait_cycles = ctx->wait_cycles;
    m.a.test_drop = ctx->test_drop_piece < 0 ? ~0ull : (uint64_t)ctx->test_drop_piece;
    m.a.st = ctx->d_status;
    const size_t stride = (piece + 127) & ~size_t(127);
    unsigned stages = (unsigned)ctx->copy_stages;
    while (stages > 1 && stages * (stride + 8) + 1024 > (size_t)ctx->max_smem_optin) --stages;
    m.grid = (unsigned)ctx->sm_count;
    m.threads = stages * 32;
    m.smem = stages * (stride + 8);
    return m;
}

int ensure_pages(lsmkv_ctx *ctx, size_t bytes)
{
    if (ctx->d_pages && bytes <= ctx->pages_cap) return LSMKV_OK;
    return enlarge_scratch(ctx, &ctx->d_pages, &ctx->pages_cap, bytes, __LINE__);
}

bool pool_ok(const lsmkv_pool_t *pool) { return pool && pool->kv_ptrs && pool->num_pages < 0xFFFFFFFFull; }

}  // namespace

extern "C" int lsmkv_release_batch(lsmkv_ctx *ctx, void *stream, const lsmkv_tables_t *tables, uint32_t *refs,
                                   uint64_t num_pages)
{
    if (!ctx || !tables) return LSMKV_EINVAL;
    if (tables->n_seq == 0) return LSMKV_OK;
    if (!tables_ok(tables) || !refs || num_pages >= 0xFFFFFFFFull || tables->n_seq > 0x7FFFFFFFu) return LSMKV_EINVAL;
    DeviceGuard guard(ctx->device);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    LaunchTimer timer(ctx, s, LSMKV_K_PLAN);
    k_release<<<tables->n_seq, 256, 0, s>>>(table_args(tables), ctx->geom.page_tokens, num_pages,
                                            reinterpret_cast<int *>(refs), ctx->d_status);
    ++ctx->launches;
    CU(ctx, cudaGetLastError());
    return LSMKV_OK;
}

extern "C" int lsmkv_fork_batch(lsmkv_ctx *ctx, void *stream, const lsmkv_tables_t *parents, const uint32_t *parent,
                                const lsmkv_tables_t *children, uint32_t *refs, const lsmkv_pool_t *pool)
{
    if (!ctx || !parents || !children) return LSMKV_EINVAL;
    if (children->n_seq == 0) return LSMKV_OK;
    if (!tables_ok(parents) || !tables_ok(children) || !parent || !refs || !pool_ok(pool)) return LSMKV_EINVAL;
    if (children->n_seq > 0x7FFFFFFFu) return LSMKV_EINVAL;
    DeviceGuard guard(ctx->device);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const size_t n = children->n_seq;
    const int rc = ensure_pages(ctx, n * 8);
    if (rc != LSMKV_OK) return rc;
    const Mover m = slab_mover(ctx, pool);
    ForkJob j;
    j.parents = table_args(parents);
    j.kids = table_args(children);
    j.parent = parent;
    j.refs = reinterpret_cast<int *>(refs);
    j.rank = static_cast<uint32_t *>(ctx->d_pages);
    j.fresh = j.rank + n;
    j.a = m.a;
    LaunchTimer timer(ctx, s, LSMKV_K_PACK);
    CU(ctx, start(ctx, s, false, k_fork_plan, 1, 1024, 0, j));
    CU(ctx, start(ctx, s, true, k_fork, m.grid, m.threads, m.smem, j));
    return LSMKV_OK;
}

extern "C" int lsmkv_compact_pages(lsmkv_ctx *ctx, void *stream, const uint32_t *refs, uint32_t *refs_out,
                                   const uint32_t *page_table, uint32_t *page_table_out, uint64_t n_entries,
                                   const lsmkv_pool_t *pool, uint64_t *n_live_out)
{
    if (!ctx || !pool_ok(pool) || !refs || !refs_out) return LSMKV_EINVAL;
    if (n_entries && (!page_table || !page_table_out)) return LSMKV_EINVAL;
    DeviceGuard guard(ctx->device);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const size_t n = pool->num_pages;
    // moves are no more than half of the pages
    const int rc = ensure_pages(ctx, 16 + (n / 2 + 1) * 8 + n * 4);
    if (rc != LSMKV_OK) return rc;
    const Mover m = slab_mover(ctx, pool);
    CompactJob j;
    j.refs = refs;
    j.refs_out = refs_out;
    j.table = page_table;
    j.table_out = page_table_out;
    j.n_entries = n_entries;
    j.n_live_out = n_live_out;
    j.moves = static_cast<uint64_t *>(ctx->d_pages);
    j.src = reinterpret_cast<uint32_t *>(j.moves + 2);
    j.dst = j.src + n / 2 + 1;
    j.rank = j.dst + n / 2 + 1;
    j.a = m.a;
    LaunchTimer timer(ctx, s, LSMKV_K_PACK);
    CU(ctx, start(ctx, s, false, k_compact_plan, 1, 1024, 0, j));
    CU(ctx, start(ctx, s, true, k_compact, m.grid, m.threads, m.smem, j));
    return LSMKV_OK;
}

extern "C" int lsmkv_copy_pages(lsmkv_ctx *ctx, void *stream, const uint32_t *src, const uint32_t *dst, uint64_t n,
                                const lsmkv_pool_t *pool)
{
    if (!ctx || !pool_ok(pool)) return LSMKV_EINVAL;
    if (n == 0) return LSMKV_OK;
    if (!src || !dst || n > 0xFFFFFFFFull) return LSMKV_EINVAL;
    DeviceGuard guard(ctx->device);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const Mover m = slab_mover(ctx, pool);
    LaunchTimer timer(ctx, s, LSMKV_K_PACK);
    k_copy_pages<<<m.grid, m.threads, m.smem, s>>>(m.a, src, dst, n);
    ++ctx->launches;
    CU(ctx, cudaGetLastError());
    return LSMKV_OK;
}
