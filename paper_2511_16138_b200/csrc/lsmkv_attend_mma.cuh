// Attention over the paged pool, kernel for many rows: the score and value products on the
// tensor cores' tcgen05 path, for head_dim up to 128.
//
// A row tile is 256 rows, two halves of 128 (one TMEM lane a row). A persistent CTA walks its span
// of units (key tiles of 128 keys); its warps have roles that run side by side:
//   loaders (3 warps)  gather the tile's queries, then keys and values of one key tile after the
//                      other through a ring of stages, in the 128-byte-swizzled layout that the
//                      matrix unit reads. Pages of a multiple of 8 tokens come by the copy engine
//                      in boxes of up to 64 tokens, others by 16-byte cp.async, each to its place
//   issuer (1 warp)    S_x = Q_x K^T of the next key tile and O_x += P_x V of this one, for the
//                      halves x in turn: while one half's softmax runs, the other half's products do
//   softmax (2 x 4 warps) a thread owns a row: scores from TMEM, running maximum and sum in
//                      registers, weights back to TMEM over the scores, where they are the
//                      A operand of the value product. The sums in TMEM are rescaled only when the
//                      maximum grew by more than 2^8 (weights stay below 2^8, sums in 32 bits).
// Bound by the chain of a half -- scores, softmax (1.9k cycles for 128 x 128 alone), value product,
// next scores -- that alternates with the other's: 2.5k to 3k cycles for a tile of 256 x 128, whose
// products take 2048 at head_dim 128 (8192 operations a cycle and SM) and whose exponentials as many (16
// a cycle and SM). Measured: two requests of 32768 tokens, the last 1024 new, 64/8 heads of 128, 2.16
// TFLOP: 1.94 ms, 1.11 PFLOP/s, of which a library product reaches 1.63 in a burst and 1.40 sustained.
// Taking some exponentials by a polynomial on the multiply-add units lengthened the chain (1.83 -> 1.84
// to 1.98 ms).
// Every wait is bounded; one that runs out ends all roles and is reported.
#pragma once
#include <cuda.h>

#include <type_traits>

#include "lsmkv_attend.cuh"

namespace lsmkv {

template <int DP>
struct ManyShape {
    static constexpr int kM = 256, kKeys = 128;
    static constexpr int kStages = DP == 128 ? 5 : 8;
    static constexpr uint32_t kTileBytes = 128 * DP * 2;
    static constexpr int kLoaders = 2;         // warps that share a block's rows, by cp.async
    // 8 softmax warps, then a warpgroup of loaders and the issuer. 384 threads start with
    // 168 registers each (64512); 256 x 208 + 128 x 80 = 63488 of them are in use afterwards.
    static constexpr int kThreads = 12 * 32;
    static constexpr int kSoftmaxRegs = 208, kOtherRegs = 80;
    static constexpr size_t kSmem = 1024 + (size_t)(2 + kStages) * kTileBytes;
    static_assert(kStages >= 4, "both halves' keys and values in flight");
};

__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(bar), "r"(count) : "memory");
}

__device__ __forceinline__ void mbar_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(bar) : "memory");
}

// Bounded wait that also ends when another role gave up.
__device__ __forceinline__ bool mbar_wait_or_stop(uint32_t bar, uint32_t parity, long long limit,
                                                  volatile uint32_t *stop)
{
    const long long t0 = clock64();
    for (uint32_t it = 0;; ++it) {
        uint32_t ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
        if (ok) return true;
        if ((it & 15u) == 15u) {
            if (*stop) return false;
            if (clock64() - t0 > limit) {
                *stop = 1;
                return false;
            }
        }
    }
}

// Shared-memory operand descriptors of 128-byte-swizzled tiles: cells of 8 rows x 64 elements (1024
// bytes), cells of the next 8 rows `group` bytes on, of the next 64 elements `half` bytes on. K-major
// (rows are M or N, elements run along K; `half` is the caller's to add) and MN-major (elements run
// along N, rows along K).
__device__ __forceinline__ uint64_t desc_k_major(uint32_t addr, uint32_t group)
{
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | (1ull << 16) | ((uint64_t)(group >> 4) << 32) | (1ull << 46) |
           (2ull << 61);
}

__device__ __forceinline__ uint64_t desc_mn_major(uint32_t addr, uint32_t group, uint32_t half)
{
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(half >> 4) << 16) | ((uint64_t)(group >> 4) << 32) |
           (1ull << 46) | (2ull << 61);
}

// True on one lane of a converged warp, always the same one.
__device__ __forceinline__ bool elect_one()
{
    uint32_t p;
    asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(p));
    return p != 0;
}

__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
}

__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t add)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 :: "r"(d), "r"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
}

// The barrier is arrived at when all products issued so far are done.
__device__ __forceinline__ void mma_commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];"
                 :: "r"(bar) : "memory");
}

// The key (or value) buffer of a layer as the copy engine sees it: elements, heads, tokens. The
// host knows all of it but the address, which lies in the pool's table on the device: a warp puts
// it into a copy of the map and publishes that for its CTA.
__device__ __forceinline__ void publish_map(void *dst, unsigned char *work, const CUtensorMap &map,
                                            const void *address)
{
    const uint32_t lane = threadIdx.x & 31;
    reinterpret_cast<uint32_t *>(work)[lane] = reinterpret_cast<const uint32_t *>(&map)[lane];
    __syncwarp();
    if (lane == 0)
        asm volatile("tensormap.replace.tile.global_address.shared::cta.b1024.b64 [%0], %1;"
                     :: "r"(smem_addr(work)), "l"(address) : "memory");
    __syncwarp();
    asm volatile("tensormap.cp_fenceproxy.global.shared::cta.tensormap::generic.release.gpu.sync.aligned [%0], [%1], 128;"
                 :: "l"(dst), "r"(smem_addr(work)) : "memory");
    asm volatile("fence.proxy.tensormap::generic.acquire.gpu [%0], 128;" :: "l"(dst) : "memory");
}

__device__ __forceinline__ void tma_box(uint32_t dst, const void *map, int e, int head, int token, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
                 "[%0], [%1, {%2, %3, %4}], [%5];"
                 :: "r"(dst), "l"(map), "r"(e), "r"(head), "r"(token), "r"(bar) : "memory");
}

// All elements of a head of several tokens: elements, tokens mod 8, blocks of 64 elements, tokens
// div 8, heads.
__device__ __forceinline__ void tma_wide_box(uint32_t dst, const void *map, int head, int group, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
                 "[%0], [%1, {%2, %2, %2, %3, %4}], [%5];"
                 :: "r"(dst), "l"(map), "r"(0), "r"(group), "r"(head), "r"(bar) : "memory");
}

__device__ __forceinline__ void tmem_ld32(uint32_t addr, float *v)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]),
          "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]),
          "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]),
          "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
        : "r"(addr) : "memory");
}

__device__ __forceinline__ void tmem_st32(uint32_t addr, const float (&v)[32])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};"
        :: "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]),
           "f"(v[8]), "f"(v[9]), "f"(v[10]), "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15]),
           "f"(v[16]), "f"(v[17]), "f"(v[18]), "f"(v[19]), "f"(v[20]), "f"(v[21]), "f"(v[22]), "f"(v[23]),
           "f"(v[24]), "f"(v[25]), "f"(v[26]), "f"(v[27]), "f"(v[28]), "f"(v[29]), "f"(v[30]), "f"(v[31]),
           "r"(addr) : "memory");
}

__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t (&v)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
        :: "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]),
           "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]),
           "r"(addr) : "memory");
}

// Loaded values may be used behind the wait only: this ties them to its place.
__device__ __forceinline__ void tmem_pin32(float *v)
{
    asm volatile("" : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]),
                      "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]));
    asm volatile("" : "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]), "+f"(v[23]),
                      "+f"(v[24]), "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]), "+f"(v[30]), "+f"(v[31]));
}

__device__ __forceinline__ float max3(float a, float b, float c)
{
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// A tile of up to 128 rows is one half; so that both halves' pipelines work, the key tiles of a
// cut then go to the halves in turn, over the same queries, and the first half's threads merge
// the two sums at the end.
__device__ __forceinline__ bool shares_rows(const Cut &p) { return p.rows <= 128; }

// Key tiles of half x in a cut: of the tile's first half the last row may see fewer.
__device__ __forceinline__ uint32_t half_tiles(const AttendJob &j, const Item &it, const Cut &p, uint32_t x,
                                               uint32_t M, uint32_t tile)
{
    const uint32_t n = p.k1 - p.k0;
    if (shares_rows(p)) return (n + 1 - x) / 2;
    if (x) return n;
    const uint32_t e = (token_limit(it, (p.rt * M + 127) / j.group) - it.kv0 + tile - 1) / tile;
    return e <= p.k0 ? 0 : e >= p.k1 ? n : e - p.k0;
}

// The cut tile that starts in a CTA's span, for the merge behind the kernel; rows = 0: none.
struct CutDesc {
    Item it;
    Cut p;
    uint32_t c0, c1;             // its parts
};

// Merge of the cut tiles: a block takes 32 rows of one, a thread four elements of four rows at a
// time, their parts' loads in flight together. Latency decides (two or three parts a row: 13 us with
// cold caches for 148 tiles of 256 rows at head_dim 64, 19 MB); done by the last CTA to arrive at
// a tile instead, it took that CTA 40 us and more.
constexpr uint32_t kMergeBlockRows = 32;
template <typename T>
__global__ __launch_bounds__(256) void k_attend_merge(const __grid_constant__ AttendJob j)
{
    constexpr int R = 4;
    follow_launch();
    const CutDesc &c = j.cuts[blockIdx.x];
    const uint32_t rows = c.p.rows, r0 = blockIdx.y * kMergeBlockRows;
    if (r0 >= rows) return;
    const uint32_t c0 = c.c0, c1 = c.c1, DP = j.dp, M = 256;
    const uint32_t quads = j.head_dim / 4, step = 256 / quads;
    const uint32_t d = threadIdx.x % quads * 4, first = threadIdx.x / quads;
    if (first >= step) return;
    const uint32_t end = min(r0 + kMergeBlockRows, rows);
    for (uint32_t r = r0 + first; r < end; r += R * step) {
        Quad sum[R];
#pragma unroll
        for (int k = 0; k < R; ++k) {
            sum[k].acc = make_float4(0.f, 0.f, 0.f, 0.f);
            sum[k].m = -INFINITY;
            sum[k].l = 0.f;
        }
        for (uint32_t x = c0; x <= c1; ++x) {
            const float *s = part_slot(j, 2ull * x + (x == c0 ? 1 : 0), M, DP);
            float pm[R], pl[R];
            float4 o[R];
#pragma unroll
            for (int k = 0; k < R; ++k) {
                const uint32_t row = min(r + k * step, end - 1);
                pm[k] = __ldcg(s + (uint64_t)M * DP + row);
                pl[k] = __ldcg(s + (uint64_t)M * (DP + 1) + row);
                o[k] = __ldcg(reinterpret_cast<const float4 *>(s + (uint64_t)row * DP + d));
            }
#pragma unroll
            for (int k = 0; k < R; ++k)
                if (pl[k] != 0.f) add_quad(sum[k], o[k], pm[k], pl[k]);   // else no key of it was the row's
        }
#pragma unroll 1
        for (int k = 0; k < R; ++k) {
            const uint32_t row = r + k * step;
            const Quad q = k == 0 ? sum[0] : k == 1 ? sum[1] : k == 2 ? sum[2] : sum[3];
            if (row < end) finish_row4<T>(j, c.it, c.p.kv_head, c.p.rt * M + row, d, q.acc, q.m, q.l);
        }
    }
}

// ---- rows that came out undefined ---------------------------------------------------------------
//
// A row may have come out undefined for a value that only later rows of its tile see (see add_undefined). When
// a CTA is done and has met undefined rows, its softmax warps go through its cuts once more: a scan of
// the values that some rows of the cut see and others do not (at most 256 keys) finds the last undefined
// one, and only rows that end ahead of it are computed anew, over the cut's keys alone; all others are undefined by
// themselves and stay. So an undefined value that its rows see costs the scan; one that rows beside them do
// not see, their share of the CTA's work once more, at the rate of m16n8k16 products. Nobody waits for the
// softmax warps by then, so no bounded wait depends on how long it takes, and the pipeline's shared
// memory is theirs. Measured, 1024 new tokens behind 30000, 64/8 heads of 128, 0.81 ms: 0.80 with a NaN in the first
// value, 3.6 with one in the last (248 rows of eight CTAs over all keys; 14 with the fragments straight from
// memory). In the merge launch instead, its registers lengthened that launch by 3.6 us in every call.

// Barriers of the 256 threads of the softmax warps; the second tells whether a condition holds for all of them.
__device__ __forceinline__ void softmax_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

__device__ __forceinline__ bool softmax_all(bool c)
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.and.pred q, 1, 256, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"((uint32_t)c) : "memory");
    return r != 0;
}

template <int DP>
struct RedoShape {
    static constexpr uint32_t kKeys = 64;                    // keys of a stage
    static constexpr uint32_t kRow = DP * 2 + 16;            // 16 bytes more: ldmatrix without conflicts
    static constexpr uint32_t kHalf = kKeys * kRow;          // keys, then values
    static constexpr uint32_t kOffsets = 4 * kHalf;          // behind two stages: places of two stages' keys
    static constexpr uint32_t kBehind = kOffsets + 2 * kKeys * 8;
    static_assert(kBehind + 4 <= ManyShape<DP>::kSmem - 1024, "within the pipeline's shared memory");
};

// 16 rows a warp from row r0 of the cut's tile on, 128 in all; smem: RedoShape's, free.
template <typename T, int DP, int M, int TILE>
__device__ __forceinline__ void redo_rows(const AttendJob &j, const Walk<M, TILE> &cw, float *slot, uint32_t r0,
                                          unsigned char *smem, uint32_t behind)
{
    using Sh = RedoShape<DP>;
    constexpr uint64_t kNone = ~0ull;
    const Item &it = cw.it;
    const uint32_t tid = threadIdx.x, lane = tid & 31, g = lane >> 2, c4 = lane & 3, D = j.head_dim, G = j.group;
    const uint32_t kv_head = cw.p.kv_head, r1 = min(r0 + 128, cw.p.rows), row_base = cw.p.rt * M;
    const uint32_t key0 = it.kv0 + cw.p.k0 * TILE;
    const uint32_t key_end = min(token_limit(it, (row_base + r1 - 1) / G), it.kv0 + cw.p.k1 * TILE);
    if (key_end <= key0) return;                 // (no row here has a key in the cut)
    // a warp's rows; this lane's are g and g + 8
    const uint32_t w0 = r0 + (tid >> 5) * 16, n_rows = w0 < r1 ? min(r1 - w0, 16u) : 0;
    const uint32_t t0 = n_rows ? (row_base + w0) / G : 0, t1 = n_rows ? (row_base + w0 + n_rows - 1) / G : 0;
    const uint32_t lim_first = token_limit(it, t0);
    uint32_t lim[2], q[DP / 16][4];
    bool anew[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const bool in = g + 8 * h < n_rows;
        const uint32_t R = row_base + (in ? w0 + g + 8 * h : 0);
        lim[h] = in ? token_limit(it, R / G) : it.kv0;
        anew[h] = in && lim[h] < behind;
        const T *row = static_cast<const T *>(j.q) + (it.row0 + R / G) * j.q_ts + (uint64_t)(kv_head * G + R % G) * j.q_hs;
#pragma unroll
        for (int x = 0; x < DP / 8; ++x)
            q[x >> 1][h + 2 * (x & 1)] =
                in && x * 8u < D ? *reinterpret_cast<const uint32_t *>(row + x * 8 + c4 * 2) : 0u;
    }
    uint64_t *const offsets = reinterpret_cast<uint64_t *>(smem + Sh::kOffsets);
    const uint32_t n_stages = (key_end - key0 + Sh::kKeys - 1) / Sh::kKeys;
    auto look_up = [&](uint32_t st) {            // places of stage st's keys
        const uint32_t k = key0 + st * Sh::kKeys + tid;
        if (tid >= Sh::kKeys) return;
        uint64_t at = kNone;                     // zeros
        if (k < key_end) {
            const uint32_t page = j.seqs.page_table[it.page0 + k / j.page_tokens];
            if (page < j.num_pages)
                at = (((uint64_t)page * j.page_tokens + k % j.page_tokens) * j.n_kv_heads + kv_head) * D;
        }
        offsets[(st & 1) * Sh::kKeys + tid] = at;
    };
    const uint32_t base = smem_addr(smem);
    auto load = [&](uint32_t st) {
        const T *const kbuf = static_cast<const T *>(j.kv_ptrs[j.layer]);
        const T *const vbuf = static_cast<const T *>(j.kv_ptrs[j.n_layers + j.layer]);
        const uint32_t dst = base + (st & 1) * 2 * Sh::kHalf;
        for (uint32_t x = tid; x < Sh::kKeys * (DP / 8); x += 256) {
            const uint32_t r = x / (DP / 8), c = x % (DP / 8);
            const uint64_t at = offsets[(st & 1) * Sh::kKeys + r];
            const bool in = at != kNone && c * 8 < D;
            const uint64_t e = in ? at + c * 8 : 0;
            cp_async16(dst + r * Sh::kRow + c * 16, kbuf + e, in);
            cp_async16(dst + Sh::kHalf + r * Sh::kRow + c * 16, vbuf + e, in);
        }
    };
    float o[DP / 8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
    for (int x = 0; x < DP / 8; ++x) o[x][0] = o[x][1] = o[x][2] = o[x][3] = 0.f;
    bool done = !__any_sync(~0u, anew[0] || anew[1]);
    softmax_sync();                              // whatever lay here is read
    look_up(0);
    softmax_sync();
    load(0);
    look_up(1);
    for (uint32_t st = 0; st < n_stages; ++st) {
        asm volatile("cp.async.wait_all;" ::: "memory");
        if (softmax_all(done)) break;
        if (st + 1 < n_stages) load(st + 1);
        look_up(st + 2);
        if (done) continue;
        const uint32_t ks = base + (st & 1) * 2 * Sh::kHalf, vs = ks + Sh::kHalf;
#pragma unroll 1
        for (uint32_t sub = 0; sub < Sh::kKeys; sub += 32) {
            const uint32_t key = key0 + st * Sh::kKeys + sub;
            if (key >= key_end) break;
            float s[4][4] = {};                  // keys 8 n ..
#pragma unroll
            for (int x = 0; x < DP / 16; ++x)    // elements 16 x ..
#pragma unroll
                for (int n = 0; n < 4; n += 2) {
                    uint32_t f[4];
                    ldmatrix4(ks + (sub + n * 8 + (lane & 7) + (lane >> 4) * 8) * Sh::kRow + (2 * x + (lane >> 3 & 1)) * 16, f);
                    mma16816<T>(s[n], q[x], f[0], f[1]);
                    mma16816<T>(s[n + 1], q[x], f[2], f[3]);
                }
            float top[2] = {m[0], m[1]};
#pragma unroll
            for (int n = 0; n < 4; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[n][e] = key + 8 * n + 2 * c4 + (e & 1) < min(lim[e >> 1], key_end) ? s[n][e] * j.scale_log2 : -INFINITY;
                    top[e >> 1] = fmaxf(top[e >> 1], s[n][e]);
                }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                top[h] = fmaxf(top[h], __shfl_xor_sync(~0u, top[h], 1));
                top[h] = fmaxf(top[h], __shfl_xor_sync(~0u, top[h], 2));
                const float ref = top[h] == -INFINITY ? 0.f : top[h];
                if (__any_sync(~0u, top[h] > m[h])) {
                    const float f = exp2f(m[h] - ref);
                    m[h] = top[h];
                    l[h] *= f;
#pragma unroll
                    for (int x = 0; x < DP / 8; ++x) {
                        o[x][2 * h] *= f;
                        o[x][2 * h + 1] *= f;
                    }
                }
#pragma unroll
                for (int n = 0; n < 4; ++n)
#pragma unroll
                    for (int e = 2 * h; e < 2 * h + 2; ++e) {
                        s[n][e] = exp2f(s[n][e] - ref);
                        l[h] += s[n][e];
                    }
            }
            uint32_t p[2][4];                    // (rounded to the values' type, as everywhere)
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                p[n >> 1][2 * (n & 1)] = Half2<T>::down(s[n][0], s[n][1]);
                p[n >> 1][2 * (n & 1) + 1] = Half2<T>::down(s[n][2], s[n][3]);
            }
            auto value_fragment = [&](int x, int k, uint32_t (&f)[4]) {      // elements 16 x .., keys 16 k ..
                ldmatrix4t(vs + (sub + k * 16 + (lane & 15)) * Sh::kRow + (2 * x + (lane >> 4)) * 16, f);
            };
            if (key + 32 <= lim_first) {
#pragma unroll
                for (int x = 0; x < DP / 16; ++x)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        uint32_t f[4];
                        value_fragment(x, k, f);
                        mma16816<T>(o[2 * x], p[k], f[0], f[1]);
                        mma16816<T>(o[2 * x + 1], p[k], f[2], f[3]);
                    }
            } else {
                // keys that some of these rows do not see: token by token
                for (uint32_t t = t0; t <= t1; ++t) {
                    const uint32_t lim_t = token_limit(it, t);
#pragma unroll
                    for (int x = 0; x < DP / 16; ++x) {
                        float part[2][4] = {};
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            uint32_t f[4];
                            value_fragment(x, k, f);
                            const uint32_t k0 = key + k * 16 + 2 * c4;
                            const uint32_t m0 = (k0 < lim_t ? 0xFFFFu : 0u) | (k0 + 1 < lim_t ? 0xFFFF0000u : 0u);
                            const uint32_t m1 = (k0 + 8 < lim_t ? 0xFFFFu : 0u) | (k0 + 9 < lim_t ? 0xFFFF0000u : 0u);
                            mma16816<T>(part[0], p[k], f[0] & m0, f[1] & m1);
                            mma16816<T>(part[1], p[k], f[2] & m0, f[3] & m1);
                        }
#pragma unroll
                        for (int n = 0; n < 2; ++n)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (lim[e >> 1] == lim_t) o[2 * x + n][e] += part[n][e];
                    }
                }
            }
        }
        if (st % 4 != 3 && st + 1 != n_stages) continue;
        // rows undefined in all their elements are right as they are
        bool lost[2] = {true, true};
#pragma unroll
        for (int x = 0; x < DP / 8; ++x)
#pragma unroll
            for (int e = 0; e < 4; ++e) lost[e >> 1] = lost[e >> 1] && (x * 8u >= D || isnan(o[x][e]));
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const unsigned votes = __ballot_sync(~0u, lost[h]);
            if ((votes >> (lane & 28) & 15) == 15) anew[h] = false;
        }
        done = !__any_sync(~0u, anew[0] || anew[1]);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        l[h] += __shfl_xor_sync(~0u, l[h], 1);
        l[h] += __shfl_xor_sync(~0u, l[h], 2);
        const uint32_t r = w0 + g + 8 * h;
        // elements 8 x + 2 c4, + 1 of two x: a lane and its neighbour turn them into four of one
#pragma unroll
        for (int x = 0; x < DP / 8; x += 2) {
            const bool odd = c4 & 1;
            float give[2] = {odd ? o[x][2 * h] : o[x + 1][2 * h], odd ? o[x][2 * h + 1] : o[x + 1][2 * h + 1]};
            float keep[2] = {odd ? o[x + 1][2 * h] : o[x][2 * h], odd ? o[x + 1][2 * h + 1] : o[x][2 * h + 1]};
            give[0] = __shfl_xor_sync(~0u, give[0], 1);
            give[1] = __shfl_xor_sync(~0u, give[1], 1);
            const float4 acc = odd ? make_float4(give[0], give[1], keep[0], keep[1])
                                   : make_float4(keep[0], keep[1], give[0], give[1]);
            const uint32_t d = (x + odd) * 8 + (c4 >> 1) * 4;
            if (!anew[h] || d >= D) continue;
            if (slot)
                __stcg(reinterpret_cast<float4 *>(slot + (uint64_t)r * DP + d), acc);
            else
                finish_row4_call<T>(j, it, kv_head, row_base + r, d, acc, m[h], l[h]);
        }
        if (slot && anew[h] && c4 == 0) {
            __stcg(slot + (uint64_t)M * DP + r, m[h]);
            __stcg(slot + (uint64_t)M * (DP + 1) + r, l[h]);
        }
    }
}

// The cuts of a CTA once more, by its softmax warps.
template <typename T, int DP, int M, int TILE>
__device__ __noinline__ void redo_cuts(const AttendJob &j, const Span span, unsigned char *smem)
{
    uint32_t *const behind = reinterpret_cast<uint32_t *>(smem + RedoShape<DP>::kBehind);
    const T *const vbuf = static_cast<const T *>(j.kv_ptrs[j.n_layers + j.layer]);
    const uint32_t tid = threadIdx.x, pieces = j.head_dim / 8;
    Walk<M, TILE> cw;
    cw.start(j, span);
    while (cw.next(j, span)) {
        const Item &it = cw.it;
        if (!it.causal || it.tokens < 2) continue;
        const uint32_t row_base = cw.p.rt * M;
        const uint32_t from = max(token_limit(it, row_base / j.group), it.kv0 + cw.p.k0 * TILE);
        const uint32_t end = min(token_limit(it, (row_base + cw.p.rows - 1) / j.group), it.kv0 + cw.p.k1 * TILE);
        if (end <= from) continue;
        softmax_sync();
        if (tid == 0) *behind = 0;
        softmax_sync();
        for (uint32_t x = tid; x < (end - from) * pieces; x += 256) {
            const uint32_t k = from + x / pieces, page = j.seqs.page_table[it.page0 + k / j.page_tokens];
            if (page >= j.num_pages) continue;
            const uint64_t at = (((uint64_t)page * j.page_tokens + k % j.page_tokens) * j.n_kv_heads + cw.p.kv_head) * j.head_dim;
            uint32_t sum = 0;
            add_undefined<T>(*reinterpret_cast<const uint4 *>(vbuf + at + x % pieces * 8), sum);
            if (was_undefined(sum)) atomicMax(behind, k + 1);
        }
        softmax_sync();
        const uint32_t last = *behind;
        const bool whole = cw.p.k0 == 0 && cw.p.k1 == cw.p.units;
        float *slot = whole ? nullptr : part_slot(j, 2ull * span.rank + (cw.p.k0 == 0 ? 1 : 0), M, DP);
        for (uint32_t r0 = 0; r0 < cw.p.rows && token_limit(it, (row_base + r0) / j.group) < last; r0 += 128)
            redo_rows<T, DP>(j, cw, slot, r0, smem, last);
    }
}

template <typename T, int DP, bool kBoxes>
__global__ __launch_bounds__(ManyShape<DP>::kThreads, 1)
void k_attend_many(const __grid_constant__ AttendJob j, const __grid_constant__ CUtensorMap map,
                   const __grid_constant__ CUtensorMap q_map)
{
    using Sh = ManyShape<DP>;
    constexpr int kChunks = DP / 8;
    constexpr uint32_t kBlock = 128 * 128;      // bytes of one block of 128 rows x 64 elements
    constexpr uint32_t kIssuer = 10;            // its warp
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t bars[3 * Sh::kStages + 14];
    __shared__ uint32_t tmem_slot;
    __shared__ __align__(128) unsigned char map_work[128];
    __shared__ volatile uint32_t stop, undefined[8];   // (a softmax warp's rows have come out undefined)
    __shared__ float half_m[128], half_l[128];   // the second half's statistics, when the halves share rows
    const uint32_t tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    const uint32_t G = j.group, D = j.head_dim;
    // (what comes behind may count on the launch before this one: nobody leaves ahead of it)
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (!j.beside) wait_launch();
    if (tid == 0) j.cuts[blockIdx.x].p.rows = 0;

    const T *const kbuf = static_cast<const T *>(j.kv_ptrs[j.layer]);
    const T *const vbuf = static_cast<const T *>(j.kv_ptrs[j.n_layers + j.layer]);
    const Span span = find_span<Sh::kThreads, true>(j, j.prefix_pass ? j.n_group : j.seqs.n_seq, Sh::kM, Sh::kKeys,
                                                    reinterpret_cast<uint32_t *>(smem_raw));
    // the loads of the waves lay where the copy engine writes queries later; ordered by the barrier below
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    if ((reinterpret_cast<uintptr_t>(kbuf) | reinterpret_cast<uintptr_t>(vbuf)) & 15u) {
        if (blockIdx.x == 0 && tid == 0) st_flag(j.st, LSMKV_ST_MISALIGNED, 0);
        wait_launch();
        return;
    }
    if (span.begin >= span.end && !span.waves) {
        wait_launch();
        return;
    }

    const uint32_t base = (smem_addr(smem_raw) + 1023u) & ~1023u;
    const uint32_t q_s = base, ring = base + 2 * Sh::kTileBytes;
    const uint32_t bar0 = smem_addr(bars);
    auto full = [&](uint32_t s) { return bar0 + 8 * s; };
    auto empty = [&](uint32_t s) { return bar0 + 8 * (Sh::kStages + s); };
    const uint32_t q_full = bar0 + 8 * (2 * Sh::kStages), q_empty = q_full + 8;
    auto s_full = [&](uint32_t x) { return q_empty + 8 + 8 * x; };
    auto p_full = [&](uint32_t x) { return q_empty + 24 + 8 * x; };
    auto o_full = [&](uint32_t x) { return q_empty + 40 + 8 * x; };
    const uint32_t half_bar = q_empty + 56, half_read = q_empty + 64, done_bar = q_empty + 72,
                   spare_bar = q_empty + 80;
    auto p_half = [&](uint32_t x) { return q_empty + 88 + 8 * x; };
    auto landed = [&](uint32_t s) { return q_empty + 104 + 8 * s; };   // boxes that are still to be wiped
    if (tid == 0) {
        mbar_init(half_bar, 128);
        mbar_init(half_read, 128);
        mbar_init(done_bar, 1);
        mbar_init(spare_bar, 32 * Sh::kLoaders);
        for (int s = 0; s < Sh::kStages; ++s) {
            mbar_init(full(s), kBoxes ? 1 : 32 * Sh::kLoaders);
            mbar_init(empty(s), 1);
            mbar_init(landed(s), 1);
        }
        mbar_init(q_full, kBoxes && j.q_boxes ? 1 : 32 * Sh::kLoaders);
        mbar_init(q_empty, 1);
        for (int x = 0; x < 2; ++x) {
            mbar_init(s_full(x), 1);
            mbar_init(p_half(x), 4);
            mbar_init(p_full(x), 4);
            mbar_init(o_full(x), 1);
        }
        stop = 0;
        for (int x = 0; x < 8; ++x) undefined[x] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (w == Sh::kThreads / 32 - 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     :: "r"(smem_addr(&tmem_slot)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    unsigned char *const maps = reinterpret_cast<unsigned char *>(j.maps) + blockIdx.x * 256;
    if (kBoxes && w == 8) {
        publish_map(maps, map_work, map, kbuf);
        publish_map(maps + 128, map_work, map, vbuf);
        if (lane < 2) asm volatile("prefetch.tensormap [%0];" :: "l"(maps + lane * 128) : "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    // layout of keys and values in their stages: cells of all elements of 8 tokens side by side, as
    // wide boxes leave them, or block after block of 64 elements, like the queries
    const bool wide = kBoxes && j.wide_boxes;
    const uint32_t kv_group = wide ? 1024 * (DP / 64) : 1024, kv_half = wide ? 1024 : kBlock;
    // columns: scores (and weights over them) of the halves at 0 and 128, sums at 256 and 384
    auto wait = [&](uint32_t bar, uint32_t parity) { return mbar_wait_or_stop(bar, parity, j.wait_cycles, &stop); };
    // for roles whose lanes act together: all of a warp go on, or none
    auto wait_warp = [&](uint32_t bar, uint32_t parity) { return (bool)__all_sync(~0u, wait(bar, parity)); };
    using CutWalk = Walk<Sh::kM, Sh::kKeys>;

    if (w < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" :: "n"(Sh::kSoftmaxRegs));
        // ---- softmax: a thread owns row `row` of half x
        const uint32_t x = w >> 2, row = tid & 127;
        const uint32_t lane_base = (w & 3) << 21;            // lanes 32 (w % 4) ..
        const uint32_t s_t = tmem + lane_base + x * 128, o_t = tmem + lane_base + 256 + x * 128;
        const float c = fmaxf(fabsf(j.scale_log2), 1e-37f);  // a negative scale negates the products
        if ((D + 15) / 16 * 16 < DP) {
            // columns of the sums that no product writes: they are read with the others, and an earlier kernel
            // may have left anything there
            float zero[32] = {};
            for (int ch = 0; ch < DP / 32; ++ch) tmem_st32(o_t + ch * 32, zero);
        }
        uint32_t s_cnt = 0, o_cnt = 0, half_cnt = 0;
        bool half_due = false;       // second half: its sums of the cut before are still to be read
        CutWalk cw;
        cw.start(j, span);
        while (cw.next(j, span)) {
            const uint32_t n = half_tiles(j, cw.it, cw.p, x, Sh::kM, Sh::kKeys);
            const bool both = shares_rows(cw.p);                   // the halves share rows
            const uint32_t first = both ? 0 : x * 128, step = both ? 2 : 1;
            const uint32_t row_base = cw.p.rt * Sh::kM + first;
            const bool real = first + row < cw.p.rows;
            const uint32_t lim = real ? token_limit(cw.it, (row_base + row) / G) : 0x7FFFFFFFu;
            const uint32_t lim_first = token_limit(cw.it, row_base / G);
            float m = -INFINITY, l = 0.f;
            bool alive = true;
            for (uint32_t t = 0; t < n; ++t) {
                if (!(alive = wait_warp(s_full(x), s_cnt & 1))) break;
                ++s_cnt;
                tc_fence_after();
                const uint32_t key = cw.it.kv0 + (cw.p.k0 + (both ? x : 0) + t * step) * Sh::kKeys;
                const bool masked = key + Sh::kKeys > lim_first;
                const int see = masked ? (int)(lim > key ? lim - key : 0u) : Sh::kKeys;   // keys of the tile
                float v[Sh::kKeys];
#pragma unroll
                for (int ch = 0; ch < 4; ++ch) tmem_ld32(s_t + ch * 32, v + ch * 32);
                tmem_wait_ld();
#pragma unroll
                for (int ch = 0; ch < 4; ++ch) tmem_pin32(v + ch * 32);
                if (masked) {
#pragma unroll
                    for (int e = 0; e < Sh::kKeys; ++e)
                        if (e >= see) v[e] = -INFINITY;
                }
                float tops[4];
#pragma unroll
                for (int ch = 0; ch < 4; ++ch) {
                    tops[ch] = fmaxf(v[ch * 32], v[ch * 32 + 1]);
#pragma unroll
                    for (int e = 2; e < 32; e += 2) tops[ch] = max3(tops[ch], v[ch * 32 + e], v[ch * 32 + e + 1]);
                }
                const float top = fmaxf(max3(tops[0], tops[1], tops[2]), tops[3]) * c;
                float fix = 1.f;
                if (t == 0) {
                    m = top;
                } else if (top > m + 8.f) {
                    fix = exp2f(m - top);
                    m = top;
                    l *= fix;
                }
                const float neg = m == -INFINITY ? 0.f : -m;
                if (__any_sync(~0u, fix != 1.f)) {
                    // the value product of the tile before is done: its scores came after it
#pragma unroll 1
                    for (int ch = 0; ch < DP / 32; ++ch) {
                        float o[32];
                        tmem_ld32(o_t + ch * 32, o);
                        tmem_wait_ld();
                        tmem_pin32(o);
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] *= fix;
                        tmem_st32(o_t + ch * 32, o);
                    }
                }
                if (half_due) {
                    // the weights let the issuer overwrite the sums that the first half merges
                    if (!(alive = wait_warp(half_read, half_cnt & 1))) break;
                    ++half_cnt;
                    half_due = false;
                }
                float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                const float2 cc = make_float2(c, c), nn = make_float2(neg, neg);
#pragma unroll
                for (int ch = 0; ch < 4; ++ch) {
                    uint32_t pk[16];
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        float2 x = fma2(make_float2(v[ch * 32 + e], v[ch * 32 + e + 1]), cc, nn);
                        x.x = exp2f(x.x);
                        x.y = exp2f(x.y);
                        sum[(e >> 1) & 1] = add2(sum[(e >> 1) & 1], x);
                        // the weights are rounded to the values' type: the tensor cores take both in one
                        pk[e / 2] = Half2<T>::down(x.x, x.y);
                    }
                    if (ch == 2) {
                        // the weights of the first 64 keys are in place: their product may begin
                        tmem_wait_st();
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(p_half(x));
                    }
                    tmem_st16(s_t + ch * 16, pk);
                }
                l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full(x));
            }
            if (alive && n) {
                alive = wait_warp(o_full(x), o_cnt & 1);
                ++o_cnt;
                tc_fence_after();
            }
            if (!alive) break;
            const bool whole = cw.p.k0 == 0 && cw.p.k1 == cw.p.units;
            float *slot = whole ? nullptr
                                : part_slot(j, 2ull * span.rank + (cw.p.k0 == 0 ? 1 : 0), Sh::kM, DP);
            float f0 = 1.f, f1 = 0.f;            // weights of the two halves' sums, when they share rows
            const bool two = both && cw.p.k1 - cw.p.k0 > 1;
            if (two && x) {
                if (half_due) {                  // (no key tile in the cuts since)
                    if (!(alive = wait_warp(half_read, half_cnt & 1))) break;
                    ++half_cnt;
                }
                half_m[row] = m;
                half_l[row] = l;
                tc_fence_before();
                mbar_arrive(half_bar);
                half_due = true;
            } else if (two) {
                if (!(alive = wait_warp(half_bar, half_cnt & 1))) break;
                ++half_cnt;
                tc_fence_after();
                const float m1 = half_m[row], top = fmaxf(m, m1);
                f0 = part_weight(m, top);
                f1 = part_weight(m1, top);
                l = l * f0 + half_l[row] * f1;
                m = top;
            }
            if (first < cw.p.rows && (n || whole) && !(both && x)) {
                // most rows: nothing to merge, l > 0
                const bool plain = !j.prefix_pass && !cw.it.skip && l != 0.f;
                const float inv = 1.f / l;
                const uint32_t R = row_base + (real ? row : 0);
                const uint64_t out_row = cw.it.row0 + R / G;
                const uint32_t out_head = cw.p.kv_head * G + R % G;
                bool lost = false;
#pragma unroll 1
                for (int ch = 0; ch < DP / 32; ++ch) {
                    float v[32];
                    __syncwarp();
                    if (n) {
                        tmem_ld32(o_t + ch * 32, v);
                        tmem_wait_ld();
                        tmem_pin32(v);
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = 0.f;
                    }
                    if (two) {
                        float v1[32];
                        tmem_ld32(o_t + 128 + ch * 32, v1);
                        tmem_wait_ld();
                        tmem_pin32(v1);
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = v[e] * f0 + v1[e] * f1;
                    }
                    if (!real) continue;
                    float all = 0.f;
#pragma unroll
                    for (int e = 0; e < 32; ++e) all += v[e];
                    lost |= isnan(all);
                    if (!whole) {
#pragma unroll
                        for (int e = 0; e < 32; e += 4)
                            __stcg(reinterpret_cast<float4 *>(slot + (uint64_t)(first + row) * DP + ch * 32 + e),
                                   make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]));
                    } else if (plain) {
                        T *const dst = static_cast<T *>(j.out) + out_row * j.o_ts + out_head * j.o_hs + ch * 32;
#pragma unroll
                        for (int e = 0; e < 32; e += 8) {
                            if (ch * 32 + e >= D) continue;
                            uint4 pk;
                            pk.x = Half2<T>::down(v[e] * inv, v[e + 1] * inv);
                            pk.y = Half2<T>::down(v[e + 2] * inv, v[e + 3] * inv);
                            pk.z = Half2<T>::down(v[e + 4] * inv, v[e + 5] * inv);
                            pk.w = Half2<T>::down(v[e + 6] * inv, v[e + 7] * inv);
                            *reinterpret_cast<uint4 *>(dst + e) = pk;
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; e += 4)
                            if (ch * 32 + e < D)
                                finish_row4_call<T>(j, cw.it, cw.p.kv_head, row_base + row, ch * 32 + e,
                                                    make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]), m, l);
                    }
                }
                if (plain && real && whole && j.lse)
                    j.lse[out_row * j.n_q_heads + out_head] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
                __syncwarp();
                if (lost) undefined[w] = 1;
                tc_fence_before();
            }
            if (two && !x) mbar_arrive(half_read);
            if (!whole && real && !(both && x)) {
                __stcg(slot + (uint64_t)Sh::kM * DP + first + row, m);
                __stcg(slot + (uint64_t)Sh::kM * (DP + 1) + first + row, l);
            }
            if (!whole && cw.p.k0 == 0 && tid == 0) {
                CutDesc &c = j.cuts[blockIdx.x];
                c.it = cw.it;
                c.p = cw.p;
                c.c0 = c.c1 = span.rank;
                while (j.span_begin[c.c1 + 1] < cw.p.tile0 + cw.p.units) ++c.c1;
            }
        }
        // The softmax warps' part in the pipeline is done, and with it all products and all copies.
        softmax_sync();
        bool any = false;
        for (int k = 0; k < 8; ++k) any |= undefined[k] != 0;
        if (softmax_all(any && !stop))
            redo_cuts<T, DP, Sh::kM, Sh::kKeys>(j, span, smem_raw + (base - smem_addr(smem_raw)));
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" :: "n"(Sh::kOtherRegs));
    }
    if (w >= 8 && w != kIssuer) {
        // ---- loaders. With boxes: warp 8 keys and values, warp 9 queries (and warp 11, if by
        // cp.async) and what is left to wipe. Otherwise warps 8 and 9 everything, half the rows each.
        constexpr int kSets = 4 / Sh::kLoaders;              // sets of 32 rows a warp takes of a block of 128
        const uint32_t r0 = ((kBoxes ? w == 11 : w == 9) ? 1 : 0) * 32 * kSets;
        const uint64_t tok_stride = (uint64_t)j.n_kv_heads * D;
        uint32_t stage = 0, laps = 0, q_cnt = 0, wiped = 0;     // wiped: a parity per stage
        bool alive = kBoxes ? w != 11 || !j.q_boxes : w != 11;

        // The barrier is arrived at, for this thread, when its copies so far have landed; the
        // issuer's proxy fence behind its wait makes them visible to the matrix unit.
        auto hand_over = [&](uint32_t bar) {
            asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" :: "r"(bar) : "memory");
        };
        auto expect = [&](uint32_t bar, uint32_t bytes) {
            asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;"
                         :: "r"(bar), "r"(bytes) : "memory");
        };
        // 32 rows of a block of 128 from row `first` on; row r at src + off(lane r), if ok(lane r).
        // Four lanes take 64 bytes of a row, eight rows at a time: with the swizzle (piece c of row r
        // at c ^ r % 8) a lane's places differ by constants.
        uint32_t piece_at[2], bytes[kChunks / 4];
#pragma unroll
        for (int y = 0; y < 2; ++y)
            piece_at[y] = (lane >> 2) * 128 + (((y * 4 + (lane & 3)) ^ (lane >> 2)) << 4);
#pragma unroll
        for (int y = 0; y < kChunks / 4; ++y) bytes[y] = (y * 4 + (lane & 3)) * 8 < D ? 16 : 0;
        auto copy_rows = [&](uint32_t dst, const T *src, uint64_t off, bool ok, uint32_t first) {
            const uint32_t lo = (uint32_t)off, hi = (uint32_t)(off >> 32) | (ok ? 0u : 0x80000000u);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = i * 8 + (lane >> 2);
                const uint32_t h = __shfl_sync(~0u, hi, r);
                const bool in = !(h >> 31);
                const uint64_t o = ((uint64_t)(h & 0x7FFFFFFFu) << 32) | __shfl_sync(~0u, lo, r);
                const T *row = src + o + (lane & 3) * 8;
                const uint32_t at = dst + (first + i * 8) * 128;
#pragma unroll
                for (int y = 0; y < kChunks / 4; ++y)
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"
                                 :: "r"(at + piece_at[y & 1] + (y >> 1) * kBlock),
                                    "l"(bytes[y] ? row + y * 32 : src), "r"(in ? bytes[y] : 0u) : "memory");
            }
        };
        auto take_stage = [&]() {
            alive = alive && wait_warp(empty(stage), (laps & 1) ^ 1);
            return alive;
        };
        // the barrier of the stage that is filled next (test hook: another one's)
        auto stage_bar = [&]() {
            return blockIdx.x == 0 && (uint64_t)laps * Sh::kStages + stage == j.test_drop ? spare_bar : full(stage);
        };
        auto next_stage = [&]() {
            if (++stage == Sh::kStages) {
                stage = 0;
                ++laps;
            }
        };

        CutWalk cw;
        cw.start(j, span);
        while (alive && cw.next(j, span)) {
            const Item &it = cw.it;
            const uint32_t row_base = cw.p.rt * Sh::kM;
            const uint32_t n = cw.p.k1 - cw.p.k0;
            const uint32_t key0 = it.kv0 + cw.p.k0 * Sh::kKeys;
            const uint32_t key_end = min(token_limit(it, (row_base + cw.p.rows - 1) / G), key0 + n * Sh::kKeys);
            // Boxes are whole: rows behind the last key hold whatever the page holds there, or what
            // the stage held before. Keys are masked, but a value times zero need not be zero.
            const bool ragged = kBoxes && key_end < key0 + n * Sh::kKeys;
            // the queries, once the products of the cut before have read theirs
            auto fetch_queries = [&]() {
                if (!(alive = wait_warp(q_empty, (q_cnt & 1) ^ 1))) return;
                ++q_cnt;
                const uint32_t halves = cw.p.rows > 128 ? 2 : 1;
                if (kBoxes && j.q_boxes) {
                    if (lane == 0) {
                        expect(q_full, halves * Sh::kTileBytes);
                        for (uint32_t x = 0; x < halves; ++x)
                            for (int e = 0; e < DP / 64; ++e)
                                tma_box(q_s + x * Sh::kTileBytes + e * kBlock, &q_map, e * 64, (int)(cw.p.kv_head * G),
                                        (int)(it.row0 + (row_base + x * 128) / G), q_full);
                    }
                    __syncwarp();
                    return;
                }
                for (uint32_t x = 0; x < halves; ++x) {
#pragma unroll
                    for (int y = 0; y < kSets; ++y) {
                        const uint32_t r = x * 128 + r0 + y * 32 + lane;
                        const bool in = r < cw.p.rows;
                        const uint32_t R = row_base + (in ? r : 0);
                        const uint64_t q_off =
                            (it.row0 + R / G) * j.q_ts + (uint64_t)(cw.p.kv_head * G + R % G) * j.q_hs;
                        copy_rows(q_s + x * Sh::kTileBytes, static_cast<const T *>(j.q), q_off, in, r0 + y * 32);
                    }
                }
                hand_over(q_full);
            };
            // page id of key k; kNone for a key that is not loaded
            constexpr uint32_t kNone = 0xFFFFFFFFu;
            auto page_of = [&](uint32_t k) -> uint32_t {
                if (k >= key_end) return kNone;
                const uint64_t entry = it.page0 + k / j.page_tokens;
                const uint32_t page = j.seqs.page_table[entry];
                if (page < j.num_pages) return page;
                st_flag(j.st, LSMKV_ST_BAD_PAGE, entry);
                return kBoxes ? (uint32_t)j.num_pages : kNone;    // the copy engine reads zeros there
            };
            if (kBoxes && w != 8) {
                fetch_queries();
                if (w != 9) continue;
                // the last values of the cut: stage of position 2n - 1 from here
                stage += 2 * n - 1;
                laps += stage / Sh::kStages;
                stage %= Sh::kStages;
                if (ragged && alive) {
                    if (!(alive = wait_warp(landed(stage), (wiped >> stage) & 1))) break;
                    wiped ^= 1u << stage;
                    const uint32_t at = ring + stage * Sh::kTileBytes;
                    const uint32_t last0 = key0 + (n - 1) * Sh::kKeys;
                    const uint32_t first = key_end > last0 ? key_end - last0 : 0;
                    for (uint32_t y = first * 8 + lane; y < Sh::kKeys * 8; y += 32)
#pragma unroll
                        for (int e = 0; e < DP / 64; ++e)
                            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};"
                                         :: "r"(at + e * kv_half + (y >> 6) * kv_group + (y & 63) * 16), "r"(0)
                                         : "memory");
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) mbar_arrive(full(stage));
                }
                next_stage();
            } else if (kBoxes) {
                // lane g takes tokens [g box_rows, (g + 1) box_rows) of every key tile, one page's
                const uint32_t g0 = lane * j.box_rows;
                uint32_t page = g0 < Sh::kKeys ? page_of(key0 + g0) : kNone;
                for (uint32_t t = 0; t < n; ++t) {
                    const uint32_t k = key0 + t * Sh::kKeys + g0;
                    const bool ok = page != kNone;
                    const int token = (int)(page * j.page_tokens + k % j.page_tokens);
                    if (t + 1 < n && g0 < Sh::kKeys) page = page_of(k + Sh::kKeys);
                    const uint32_t total = __popc(__ballot_sync(~0u, ok)) * (DP / 64) * j.box_rows * 128;
#pragma unroll
                    for (int kv = 0; kv < 2; ++kv) {
                        if (!take_stage()) break;
                        const uint32_t bar = kv && ragged && t + 1 == n ? landed(stage) : stage_bar();
                        if (lane == 0) expect(bar, total);
                        __syncwarp();
                        if (ok && wide) {
                            tma_wide_box(ring + stage * Sh::kTileBytes + (g0 >> 3) * kv_group, maps + kv * 128,
                                         (int)cw.p.kv_head, token >> 3, bar);
                        } else if (ok) {
#pragma unroll
                            for (int e = 0; e < DP / 64; ++e)
                                tma_box(ring + stage * Sh::kTileBytes + e * kBlock + g0 * 128, maps + kv * 128, e * 64,
                                        (int)cw.p.kv_head, token, bar);
                        }
                        next_stage();
                    }
                    if (!alive) break;
                }
            } else {
                uint32_t page[kSets];                            // a tile ahead of the copies
#pragma unroll
                for (int y = 0; y < kSets; ++y) page[y] = page_of(key0 + r0 + y * 32 + lane);
                for (uint32_t t = 0; t < n; ++t) {
                    uint64_t off[kSets];
                    bool ok[kSets];
#pragma unroll
                    for (int y = 0; y < kSets; ++y) {
                        const uint32_t k = key0 + t * Sh::kKeys + r0 + y * 32 + lane;
                        ok[y] = page[y] != kNone;
                        off[y] = ok[y] ? ((uint64_t)page[y] * j.page_tokens + k % j.page_tokens) * tok_stride +
                                             (uint64_t)cw.p.kv_head * D
                                       : 0;
                        if (t + 1 < n) page[y] = page_of(k + Sh::kKeys);
                    }
#pragma unroll
                    for (int kv = 0; kv < 2; ++kv) {
                        if (!take_stage()) break;
#pragma unroll
                        for (int y = 0; y < kSets; ++y)
                            copy_rows(ring + stage * Sh::kTileBytes, kv ? vbuf : kbuf, off[y], ok[y], r0 + y * 32);
                        hand_over(stage_bar());
                        next_stage();
                        if (t == 0 && kv == 0) fetch_queries();
                        if (!alive) break;
                    }
                    if (!alive) break;
                }
            }
        }
        if (kBoxes && w == 8) {
            // boxes still under way write shared memory: let them land
            for (int s = 0; s < Sh::kStages; ++s) {
                const uint32_t lap = laps + (stage > (uint32_t)s ? 1 : 0);        // times this stage was filled
                if (lap) (void)mbar_wait_bounded(full(s), (lap - 1) & 1, j.wait_cycles);
            }
        }
        if (kBoxes && w == 9 && j.q_boxes && q_cnt)
            (void)mbar_wait_bounded(q_full, (q_cnt - 1) & 1, j.wait_cycles);      // boxes of queries likewise
    } else if (w == kIssuer) {
        // ---- issuer: the warp walks together, one lane waits and issues
        const uint32_t type = std::is_same<T, __half>::value ? 0u : 1u;
        const uint32_t common = (1u << 4) | (type << 7) | (type << 10) | (8u << 24);   // f32 sums, M = 128
        const uint32_t k_steps = (D + 15) / 16, n_out = k_steps * 16;
        const uint32_t id_s = common | ((Sh::kKeys / 8) << 17) | (j.scale_log2 < 0.f ? 1u << 13 : 0u);
        const uint32_t id_o = common | ((n_out / 8) << 17) | (1u << 16);
        const bool leader = elect_one();
        const bool fenced = !kBoxes;
        // places in the ring: keys of tile t at 2 t, values behind them
        struct Place {
            uint32_t st, ph;
            __device__ __forceinline__ void step(uint32_t by)
            {
                st += by;
                if (st >= Sh::kStages) {
                    st -= Sh::kStages;
                    ph ^= 1;
                }
            }
        };
        Place kp = {0, 0};
        uint32_t q_par = 0, p_par = 0;
        const uint64_t q_desc = desc_k_major(q_s, 1024), k_desc = desc_k_major(ring, kv_group),
                       v_desc = desc_mn_major(ring, kv_group, kv_half);
        // cp.async wrote through another proxy than the matrix unit reads through
        auto wait_tile = [&](const Place &at) {
            if (!wait(full(at.st), at.ph)) return false;
            if (fenced) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            return true;
        };
        auto scores = [&](uint32_t x, uint32_t q, uint32_t st) {      // S_x = Q_q K^T
            const uint64_t a = q_desc + q * (Sh::kTileBytes >> 4), b = k_desc + st * (Sh::kTileBytes >> 4);
#pragma unroll
            for (uint32_t k = 0; k < DP / 16; ++k) {
                // 64 elements a block, 16 a step
                if (k < k_steps)
                    mma_ss(tmem + x * 128, a + (k >> 2) * (kBlock >> 4) + (k & 3) * 2,
                           b + (k >> 2) * (kv_half >> 4) + (k & 3) * 2, id_s, k != 0);
            }
            mma_commit(s_full(x));
        };
        // O_x += P_x V, the first 64 keys as soon as their weights are there
        auto values = [&](uint32_t x, uint32_t st, bool add) {
            const uint64_t b = v_desc + st * (Sh::kTileBytes >> 4);
            const uint32_t par = (p_par >> x) & 1;
            p_par ^= 1u << x;
#pragma unroll
            for (uint32_t h = 0; h < 2; ++h) {
                if (!wait(h ? p_full(x) : p_half(x), par)) return false;
                tc_fence_after();
#pragma unroll
                for (uint32_t k = h * 4; k < h * 4 + 4; ++k)
                    mma_ts(tmem + 256 + x * 128, tmem + x * 128 + k * 8, b + k * (2 * kv_group >> 4), id_o, add || k != 0);
            }
            return true;
        };
        auto run_cut = [&](uint32_t n, uint32_t n0, uint32_t n1, bool both) -> bool {
            Place vp = kp;
            vp.step(1);
            if (!wait(q_full, q_par)) return false;
            q_par ^= 1;
            if (!kBoxes || !j.q_boxes) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            if (both) {
                // tile t belongs to half t % 2
                for (uint32_t t = 0; t < n + 2; ++t) {
                    const uint32_t x = t & 1;
                    if (t >= 2) {
                        if (!wait_tile(vp) || !values(x, vp.st, t >= 4)) return false;
                        mma_commit(empty(vp.st));
                        if (t >= n) mma_commit(o_full(x));
                        vp.step(2);
                    }
                    if (t < n) {
                        if (!wait_tile(kp)) return false;
                        scores(x, 0, kp.st);
                        mma_commit(empty(kp.st));
                        if (t + 1 == n) mma_commit(q_empty);
                        kp.step(2);
                    }
                }
                return true;
            }
            if (!wait_tile(kp)) return false;
            if (n0) scores(0, 0, kp.st);
            if (n1) scores(1, 1, kp.st);
            mma_commit(empty(kp.st));
            if (n == 1) mma_commit(q_empty);
            kp.step(2);
            for (uint32_t t = 0; t < n; ++t) {
                const bool more = t + 1 < n;
                if (!wait_tile(vp) || (more && !wait_tile(kp))) return false;
#pragma unroll
                for (uint32_t x = 0; x < 2; ++x) {
                    const uint32_t nx = x ? n1 : n0;
                    if (t < nx && !values(x, vp.st, t != 0)) return false;
                    if (t + 1 < nx) scores(x, x, kp.st);
                    else if (t + 1 == nx) mma_commit(o_full(x));
                }
                mma_commit(empty(vp.st));
                vp.step(2);
                if (more) {
                    mma_commit(empty(kp.st));
                    if (t + 2 == n) mma_commit(q_empty);
                    kp.step(2);
                }
            }
            return true;
        };
        CutWalk cw;
        cw.start(j, span);
        while (cw.next(j, span)) {
            bool ok = true;
            if (leader)
                ok = run_cut(cw.p.k1 - cw.p.k0, half_tiles(j, cw.it, cw.p, 0, Sh::kM, Sh::kKeys),
                             half_tiles(j, cw.it, cw.p, 1, Sh::kM, Sh::kKeys), shares_rows(cw.p));
            if (!__all_sync(~0u, ok)) break;
        }
        // products still under way read shared memory and write TMEM: let them end
        if (leader) {
            mma_commit(done_bar);
            (void)mbar_wait_bounded(done_bar, 0, j.wait_cycles);
        }
    }
    __syncwarp();
    asm volatile("cp.async.wait_all;" ::: "memory");
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (w == Sh::kThreads / 32 - 1)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem), "r"(512u) : "memory");
    if (tid == 0 && stop) st_flag(j.st, LSMKV_ST_WAIT_EXPIRED, blockIdx.x);
    wait_launch();
}

}  // namespace lsmkv
