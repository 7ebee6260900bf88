// Pages of a pool and who uses them: release, fork, compaction, copies.
//
// A counter a page holds how many entries of the caller's page tables name it; 0 = free. Release counts
// the entries of sequences down. Fork gives a child its parent's whole pages (counted up) and, where the
// parent ends inside a page, a page of its own with the rows that are filled; free pages are taken from the
// lowest on, in the children's order. Compaction moves the used pages behind the first n (n used pages in all) to
// the free ones among the first n, k-th to k-th in ascending order, and rewrites tables and counters.
// Every result is determined: ranks come from prefix sums, counters are sums.
//
// The bookkeeping is a few loads a page, by one CTA; what costs is moving slabs, at the copy's rate: lane 0 of every
// warp runs a shared-memory stage of its own through the copy engine, as the pack and unpack kernels do.
// Measured: compaction of 1000 pages of 2 MB of which 600 are used, 1.02 GB read and written, 180 us, 5.7 TB/s; release
// and fork of 64 prompts four ways, 0.53 GB, 76 us.
#pragma once
#include "lsmkv_attend.cuh"
#include "lsmkv_copy.cuh"

namespace lsmkv {

struct TableArgs {
    uint64_t n_entries;
    uint32_t n_seq;
    uint32_t *kv_len;
    const uint64_t *page_off;
    uint32_t *page_table;
};

// Where slabs lie and how they are moved.
struct SlabArgs {
    void *const *kv_ptrs;
    uint64_t num_pages;
    uint32_t buffers;            // 2 L
    uint32_t page_bytes, body_bytes, page_tokens;   // body: without the scales of an 8-bit pool
    uint32_t piece_bytes;
    long long wait_cycles;
    uint64_t test_drop;
    DevStatus *st;
};

struct TableSeq {
    uint64_t page0;
    uint32_t kv, pages;          // tokens; entries in use
    bool ok;
};

__device__ __forceinline__ TableSeq load_table(const TableArgs &t, uint32_t i, uint32_t page_tokens)
{
    TableSeq s;
    const uint64_t p0 = t.page_off[i], p1 = t.page_off[i + 1];
    s.kv = t.kv_len[i];
    s.page0 = p0;
    s.ok = p0 <= p1 && p1 <= t.n_entries && s.kv < 0x80000000u && (p1 - p0) * page_tokens >= s.kv;
    s.pages = s.ok ? (s.kv + page_tokens - 1) / page_tokens : 0u;
    return s;
}

// ---- moving slabs ------------------------------------------------------------------------------

// Pieces 0 .. total, dealt out over the grid's warps; resolve(p, piece) says what piece p is, or that
// there is none. One lane a warp; smem: a stage a warp, then a barrier each.
template <typename Resolve>
__device__ __forceinline__ void copy_pieces(const SlabArgs &a, uint64_t total, unsigned char *smem, Resolve resolve)
{
    const uint32_t n_stage = blockDim.x >> 5, warp = threadIdx.x >> 5;
    const uint32_t stride = (a.piece_bytes + 127u) & ~127u;
    const uint32_t sbuf = smem_addr(smem + (size_t)warp * stride);
    const uint32_t bar = smem_addr(smem + (size_t)n_stage * stride) + warp * 8;
    if (lane_id() != 0) return;
    asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" :: "r"(bar) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    const uint64_t workers = (uint64_t)gridDim.x * n_stage;
    uint32_t parity = 0;
    for (uint64_t p = (uint64_t)blockIdx.x * n_stage + warp; p < total; p += workers) {
        Piece pc;
        if (!resolve(p, pc)) continue;
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" :: "r"(bar), "r"(pc.bytes) : "memory");
        if (p != a.test_drop)    // (test hook: nothing is started, nothing is in flight when the wait gives up)
            asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                         :: "r"(sbuf), "l"(pc.src), "r"(pc.bytes), "r"(bar) : "memory");
        if (!mbar_wait_bounded(bar, parity, a.wait_cycles)) {
            // one more bounded wait, so that no copy still writes this shared memory when the warp leaves
            st_flag(a.st, LSMKV_ST_WAIT_EXPIRED, p);
            mbar_wait_bounded(bar, parity, a.wait_cycles);
            break;
        }
        parity ^= 1u;
        asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;"
                     :: "l"(pc.dst), "r"(sbuf), "r"(pc.bytes) : "memory");
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    }
    asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
}

// Pool buffer number b, or null (reported) when it is not aligned.
__device__ __forceinline__ unsigned char *slab_buffer(const SlabArgs &a, uint32_t b)
{
    unsigned char *const buf = static_cast<unsigned char *>(a.kv_ptrs[b]);
    if (!(reinterpret_cast<uintptr_t>(buf) & 15u)) return buf;
    st_flag(a.st, LSMKV_ST_MISALIGNED, b);
    return nullptr;
}

// ---- release -----------------------------------------------------------------------------------

__global__ __launch_bounds__(256) void k_release(const TableArgs t, uint32_t page_tokens, uint64_t num_pages, int *refs,
                                                 DevStatus *st)
{
    const uint32_t i = blockIdx.x;
    const TableSeq s = load_table(t, i, page_tokens);
    if (!s.ok && threadIdx.x == 0) st_flag(st, LSMKV_ST_BAD_COUNT, i);
    for (uint32_t k = threadIdx.x; k < s.pages; k += 256) {
        const uint32_t page = t.page_table[s.page0 + k];
        if (page >= num_pages) {
            st_flag(st, LSMKV_ST_BAD_PAGE, s.page0 + k);
        } else if (atomicSub(&refs[page], 1) <= 0) {
            // nobody used it: back to where it was, whatever the others do meanwhile
            atomicAdd(&refs[page], 1);
            st_flag(st, LSMKV_ST_BAD_COUNT, i);
        }
    }
}

// ---- fork --------------------------------------------------------------------------------------

constexpr uint32_t kNoPage = 0xFFFFFFFFu;

struct ForkJob {
    TableArgs parents, kids;
    const uint32_t *parent;
    int *refs;
    uint32_t *rank;              // of a child among those that take a page; kNoPage: takes none
    uint32_t *fresh;             // the pages taken; kNoPage: there was none left
    SlabArgs a;
};

struct Fork {
    TableSeq from;
    uint64_t to0;
    uint32_t tail;               // filled rows of the last page, 0: it is whole
    bool ok;
};

__device__ __forceinline__ Fork load_fork(const ForkJob &j, uint32_t c)
{
    Fork f;
    const uint32_t i = j.parent[c];
    const uint64_t q0 = j.kids.page_off[c], q1 = j.kids.page_off[c + 1];
    f.ok = i < j.parents.n_seq;
    f.tail = 0;
    f.to0 = q0;
    if (!f.ok) return f;
    f.from = load_table(j.parents, i, j.a.page_tokens);
    f.ok = f.from.ok && q0 <= q1 && q1 <= j.kids.n_entries && q1 - q0 >= f.from.pages;
    if (f.ok) f.tail = f.from.kv % j.a.page_tokens;
    return f;
}

// One CTA: the children that take a page are numbered, and the lowest free pages become theirs.
__global__ __launch_bounds__(1024) void k_fork_plan(const __grid_constant__ ForkJob j)
{
    __shared__ uint64_t scan[32];
    const uint32_t tid = threadIdx.x;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    uint32_t want = 0;
    for (uint32_t c0 = 0; c0 < j.kids.n_seq; c0 += 1024) {
        const uint32_t c = c0 + tid;
        bool takes = false;
        if (c < j.kids.n_seq) {
            const Fork f = load_fork(j, c);
            if (!f.ok) st_flag(j.a.st, LSMKV_ST_BAD_COUNT, c);
            // (a page that is not there is passed on as it is)
            takes = f.ok && f.tail && j.parents.page_table[f.from.page0 + f.from.pages - 1] < j.a.num_pages;
        }
        uint64_t all;
        const uint64_t upto = block_scan<1024>(takes, scan, &all);
        if (c < j.kids.n_seq) j.rank[c] = takes ? want + (uint32_t)upto - 1 : kNoPage;
        want += (uint32_t)all;
    }
    uint32_t found = 0;
    constexpr uint32_t kEach = 8;
    for (uint64_t p0 = 0; p0 < j.a.num_pages && found < want; p0 += 1024 * kEach) {
        uint32_t mine = 0;       // bit k: page p0 + tid * kEach + k is free
#pragma unroll
        for (uint32_t k = 0; k < kEach; ++k) {
            const uint64_t p = p0 + (uint64_t)tid * kEach + k;
            if (p < j.a.num_pages && j.refs[p] == 0) mine |= 1u << k;
        }
        uint64_t all;
        uint32_t r = found + (uint32_t)block_scan<1024>(__popc(mine), scan, &all) - __popc(mine);
#pragma unroll
        for (uint32_t k = 0; k < kEach; ++k) {
            if (!(mine >> k & 1)) continue;
            if (r < want) {
                const uint64_t p = p0 + (uint64_t)tid * kEach + k;
                j.fresh[r] = (uint32_t)p;
                j.refs[p] = 1;
            }
            ++r;
        }
        found += (uint32_t)all;
    }
    for (uint32_t r = found + tid; r < want; r += 1024) j.fresh[r] = kNoPage;
}

__global__ __launch_bounds__(1024) void k_fork(const __grid_constant__ ForkJob j)
{
    extern __shared__ __align__(128) unsigned char smem[];
    follow_launch();
    // tables and counters: a CTA takes every gridDim-th child
    for (uint32_t c = blockIdx.x; c < j.kids.n_seq; c += gridDim.x) {
        const Fork f = load_fork(j, c);
        if (!f.ok) continue;
        const uint32_t rank = j.rank[c];
        const uint32_t shared = rank == kNoPage ? f.from.pages : f.from.pages - 1;
        for (uint32_t k = threadIdx.x; k < shared; k += blockDim.x) {
            const uint32_t page = j.parents.page_table[f.from.page0 + k];
            j.kids.page_table[f.to0 + k] = page;
            if (page < j.a.num_pages) atomicAdd(&j.refs[page], 1);
            else st_flag(j.a.st, LSMKV_ST_BAD_PAGE, f.from.page0 + k);
        }
        if (threadIdx.x == 0) {
            j.kids.kv_len[c] = f.from.kv;
            if (rank != kNoPage) {
                const uint32_t page = j.fresh[rank];
                j.kids.page_table[f.to0 + shared] = page;
                if (page == kNoPage) st_flag(j.a.st, LSMKV_ST_NO_PAGE, c);
            }
        }
    }
    // the filled rows of last pages: pieces of the codes, then the scales
    const SlabArgs &a = j.a;
    const uint32_t body_pieces = (a.body_bytes + a.piece_bytes - 1) / a.piece_bytes;
    const uint32_t extra = (a.page_bytes - a.body_bytes + a.piece_bytes - 1) / a.piece_bytes;
    const uint32_t per_slab = body_pieces + extra, row = a.body_bytes / a.page_tokens;
    copy_pieces(a, (uint64_t)j.kids.n_seq * a.buffers * per_slab, smem, [&](uint64_t p, Piece &pc) {
        const uint64_t slab = p / per_slab;
        const uint32_t piece = (uint32_t)(p - slab * per_slab);
        const uint32_t c = (uint32_t)(slab / a.buffers), b = (uint32_t)(slab - (uint64_t)c * a.buffers);
        const uint32_t rank = j.rank[c];
        if (rank == kNoPage || j.fresh[rank] == kNoPage) return false;
        const Fork f = load_fork(j, c);
        // whole 16 bytes: the last row's end may take a little of the next one's with it
        const uint32_t end = piece < body_pieces ? (uint32_t)(((uint64_t)f.tail * row + 15) & ~15ull) : a.page_bytes;
        const uint32_t off = piece < body_pieces ? piece * a.piece_bytes
                                                 : a.body_bytes + (piece - body_pieces) * a.piece_bytes;
        if (off >= end) return false;
        unsigned char *const buf = slab_buffer(a, b);
        if (!buf) return false;
        const uint64_t src = j.parents.page_table[f.from.page0 + f.from.pages - 1];
        pc.src = buf + src * a.page_bytes + off;
        pc.dst = buf + (uint64_t)j.fresh[rank] * a.page_bytes + off;
        pc.bytes = min(a.piece_bytes, end - off);
        return true;
    });
}

// ---- compaction and copies ---------------------------------------------------------------------

struct CompactJob {
    const uint32_t *refs;
    uint32_t *refs_out;
    const uint32_t *table;
    uint32_t *table_out;
    uint64_t n_entries;
    uint64_t *n_live_out;        // optional
    uint64_t *moves;             // [2]: moves, used pages
    uint32_t *src, *dst;         // of the moves
    uint32_t *rank;              // of a used page behind the first n among the moves
    SlabArgs a;
};

// One CTA: counts the used pages, then numbers the used ones behind the first n and the free ones ahead.
__global__ __launch_bounds__(1024) void k_compact_plan(const __grid_constant__ CompactJob j)
{
    __shared__ uint64_t scan[32];
    constexpr uint32_t kEach = 16;
    const uint32_t tid = threadIdx.x;
    const uint64_t N = j.a.num_pages;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    uint64_t n = 0;
    for (uint64_t p0 = tid; p0 < N; p0 += 1024 * kEach) {        // (so many loads in flight)
#pragma unroll
        for (uint32_t k = 0; k < kEach; ++k)
            if (p0 + k * 1024 < N) n += j.refs[p0 + k * 1024] != 0;
    }
    {
        uint64_t all;
        block_scan<1024>(n, scan, &all);
        n = all;
    }
    uint32_t to = 0, from = 0;   // numbered so far
    for (uint64_t p0 = 0; p0 < N; p0 += 1024 * kEach) {
        uint32_t mine = 0;       // bit k: page k of this thread's moves, or is moved to
        uint32_t ahead = 0;      // of them the pages among the first n
#pragma unroll
        for (uint32_t k = 0; k < kEach; ++k) {
            const uint64_t p = p0 + (uint64_t)tid * kEach + k;
            if (p >= N) continue;
            const bool used = j.refs[p] != 0;
            if (p < n ? !used : used) {
                mine |= 1u << k;
                if (p < n) ahead |= 1u << k;
            }
        }
        const uint64_t both = (uint64_t)__popc(mine & ~ahead) << 32 | __popc(ahead);
        uint64_t all;
        const uint64_t before = block_scan<1024>(both, scan, &all) - both;
        uint32_t t = to + (uint32_t)before, f = from + (uint32_t)(before >> 32);
#pragma unroll
        for (uint32_t k = 0; k < kEach; ++k) {
            if (!(mine >> k & 1)) continue;
            const uint32_t p = (uint32_t)(p0 + (uint64_t)tid * kEach + k);
            if (ahead >> k & 1) {
                j.dst[t++] = p;
            } else {
                j.rank[p] = f;
                j.src[f++] = p;
            }
        }
        to += (uint32_t)all;
        from += (uint32_t)(all >> 32);
    }
    if (tid == 0) {
        j.moves[0] = from;
        j.moves[1] = n;
        if (j.n_live_out) *j.n_live_out = n;
    }
}

__global__ __launch_bounds__(1024) void k_compact(const __grid_constant__ CompactJob j)
{
    extern __shared__ __align__(128) unsigned char smem[];
    follow_launch();
    const uint64_t moves = j.moves[0], n = j.moves[1], N = j.a.num_pages;
    const uint64_t threads = (uint64_t)gridDim.x * blockDim.x, me = (uint64_t)blockIdx.x * blockDim.x + threadIdx.x;
    for (uint64_t x = me; x < j.n_entries; x += threads) {
        const uint32_t page = j.table[x];
        uint32_t to = page;
        if (page >= N) st_flag(j.a.st, LSMKV_ST_BAD_PAGE, x);
        // (a page that nobody counts stays where it is named)
        else if (page >= n && j.rank[page] < moves && j.src[j.rank[page]] == page) to = j.dst[j.rank[page]];
        j.table_out[x] = to;
    }
    // counters; in place too: a page that is moved or moved to is one thread's
    for (uint64_t k = me; k < moves; k += threads) {
        const uint32_t from = j.src[k], to = j.dst[k], r = j.refs[from];
        j.refs_out[to] = r;
        j.refs_out[from] = 0;
    }
    if (j.refs_out != j.refs)
        for (uint64_t p = me; p < N; p += threads) {
            const uint32_t r = j.refs[p];
            if ((p < n) == (r != 0)) j.refs_out[p] = r;
        }
    const SlabArgs &a = j.a;
    const uint32_t per_slab = (a.page_bytes + a.piece_bytes - 1) / a.piece_bytes;
    copy_pieces(a, moves * a.buffers * per_slab, smem, [&](uint64_t p, Piece &pc) {
        const uint64_t slab = p / per_slab;
        const uint32_t off = (uint32_t)(p - slab * per_slab) * a.piece_bytes;
        const uint64_t k = slab / a.buffers;
        unsigned char *const buf = slab_buffer(a, (uint32_t)(slab - k * a.buffers));
        if (!buf) return false;
        pc.src = buf + (uint64_t)j.src[k] * a.page_bytes + off;
        pc.dst = buf + (uint64_t)j.dst[k] * a.page_bytes + off;
        pc.bytes = min(a.piece_bytes, a.page_bytes - off);
        return true;
    });
}

// Pages src[i] -> dst[i].
__global__ __launch_bounds__(1024) void k_copy_pages(const __grid_constant__ SlabArgs a, const uint32_t *src,
                                                     const uint32_t *dst, uint64_t n)
{
    extern __shared__ __align__(128) unsigned char smem[];
    const uint32_t per_slab = (a.page_bytes + a.piece_bytes - 1) / a.piece_bytes;
    copy_pieces(a, n * a.buffers * per_slab, smem, [&](uint64_t p, Piece &pc) {
        const uint64_t slab = p / per_slab;
        const uint32_t off = (uint32_t)(p - slab * per_slab) * a.piece_bytes;
        const uint64_t i = slab / a.buffers;
        const uint32_t from = src[i], to = dst[i];
        if (from >= a.num_pages || to >= a.num_pages) {
            if (off == 0) st_flag(a.st, LSMKV_ST_BAD_PAGE, i);
            return false;
        }
        unsigned char *const buf = slab_buffer(a, (uint32_t)(slab - i * a.buffers));
        if (!buf || from == to) return false;
        pc.src = buf + (uint64_t)from * a.page_bytes + off;
        pc.dst = buf + (uint64_t)to * a.page_bytes + off;
        pc.bytes = min(a.piece_bytes, a.page_bytes - off);
        return true;
    });
}

}  // namespace lsmkv
