// Attention over the paged pool, kernel for many rows: the score and value products on the
// tensor cores' tcgen05 path, for head_dim up to 128.
//
// A row tile is 256 rows, two halves of 128 (one TMEM lane a row). A persistent CTA walks its span
// of units (key tiles of 128 keys); its warps have roles that run side by side:
//   loaders (2 warps)  gather the tile's queries, then keys and values of one key tile after the
//                      other through a ring of stages: 16-byte cp.async, each to its place in the
//                      128-byte-swizzled layout that the matrix unit reads, so that any page size
//                      and any page order costs the same
//   issuer (1 warp)    S_x = Q_x K^T of the next key tile and O_x += P_x V of this one, for the
//                      halves x in turn: while one half's softmax runs, the other half's products do
//   softmax (2 x 4 warps) a thread owns a row: scores from TMEM, running maximum and sum in
//                      registers, weights back to TMEM over the scores, where they are the
//                      A operand of the value product. The sums in TMEM are rescaled only when the
//                      maximum grew by more than 2^8 (weights stay below 2^8, sums in 32 bits).
// Bound by the exponentials and the tensor cores together: a 128 x 128 tile takes 1024 cycles of
// either (16 exponentials a cycle and SM; 8192 operations a cycle and SM at head_dim 128).
// Every wait is bounded; one that runs out ends all roles and is reported.
#pragma once
#include <type_traits>

#include "lsmkv_attend.cuh"

namespace lsmkv {

template <int DP>
struct ManyShape {
    static constexpr int kM = 256, kKeys = 128;
    static constexpr int kStages = DP == 128 ? 5 : 8;
    static constexpr int kLag = 3;             // copy groups in flight per loader thread
    static constexpr uint32_t kTileBytes = 128 * DP * 2;
    static constexpr int kLoaders = 2;         // warps
    static constexpr int kThreads = (8 + kLoaders + 1) * 32;   // 11 warps: 168 registers each
    static constexpr size_t kSmem = 1024 + (size_t)(2 + kStages) * kTileBytes;
    static_assert(kLag <= kStages - 2, "a stage must be handed over before the ring blocks on it");
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

// Shared-memory operand descriptors of 128-byte-swizzled tiles [rows][64 elements], one block of
// 128 rows after the other. K-major (rows are M or N, elements run along K): groups of 8 rows are
// 1024 bytes apart. MN-major (elements run along N, rows along K): blocks of 64 elements are
// `block` bytes apart, groups of 8 rows 1024.
__device__ __forceinline__ uint64_t desc_k_major(uint32_t addr)
{
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | (1ull << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}

__device__ __forceinline__ uint64_t desc_mn_major(uint32_t addr, uint32_t block)
{
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(block >> 4) << 16) | (64ull << 32) |
           (1ull << 46) | (2ull << 61);
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

__device__ __forceinline__ void tmem_ld32(uint32_t addr, float (&v)[32])
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

__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// Key tiles of half x in a cut: the first half's last row may see fewer than the second's.
__device__ __forceinline__ uint32_t half_tiles(const AttendJob &j, const Item &it, const Cut &p, uint32_t x,
                                               uint32_t M, uint32_t tile)
{
    const uint32_t n = p.k1 - p.k0;
    if (p.rows <= 128) return x ? 0 : n;
    if (x) return n;
    const uint32_t e = (token_limit(it, (p.rt * M + 127) / j.group) - it.kv0 + tile - 1) / tile;
    return e <= p.k0 ? 0 : e >= p.k1 ? n : e - p.k0;
}

template <typename T, int DP>
__global__ __launch_bounds__(ManyShape<DP>::kThreads, 1) void k_attend_many(const __grid_constant__ AttendJob j)
{
    using Sh = ManyShape<DP>;
    constexpr int kChunks = DP / 8;
    constexpr uint32_t kBlock = 128 * 128;      // bytes of one block of 128 rows x 64 elements
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t bars[2 * Sh::kStages + 11];
    __shared__ uint32_t tmem_slot;
    __shared__ volatile uint32_t stop, last_part;
    const uint32_t tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    const uint32_t G = j.group, D = j.head_dim;

    const T *const kbuf = static_cast<const T *>(j.kv_ptrs[j.layer]);
    const T *const vbuf = static_cast<const T *>(j.kv_ptrs[j.n_layers + j.layer]);
    if ((reinterpret_cast<uintptr_t>(kbuf) | reinterpret_cast<uintptr_t>(vbuf)) & 15u) {
        if (blockIdx.x == 0 && tid == 0) st_flag(j.st, LSMKV_ST_MISALIGNED, 0);
        return;
    }
    const Span span = find_span<Sh::kThreads>(j, j.prefix_pass ? j.n_group : j.seqs.n_seq, Sh::kM, Sh::kKeys);
    if (span.begin >= span.end) return;

    const uint32_t base = (smem_addr(smem_raw) + 1023u) & ~1023u;
    const uint32_t q_s = base, ring = base + 2 * Sh::kTileBytes;
    const uint32_t bar0 = smem_addr(bars);
    auto full = [&](uint32_t s) { return bar0 + 8 * s; };
    auto empty = [&](uint32_t s) { return bar0 + 8 * (Sh::kStages + s); };
    const uint32_t q_full = bar0 + 8 * (2 * Sh::kStages), q_empty = q_full + 8;
    auto s_full = [&](uint32_t x) { return q_empty + 8 + 8 * x; };
    auto p_full = [&](uint32_t x) { return q_empty + 24 + 8 * x; };
    auto o_full = [&](uint32_t x) { return q_empty + 40 + 8 * x; };
    const uint32_t part_bar = q_empty + 56, done_bar = q_empty + 64, spare_bar = q_empty + 72;
    if (tid == 0) {
        mbar_init(part_bar, 256);
        mbar_init(done_bar, 1);
        mbar_init(spare_bar, 32 * Sh::kLoaders);
        for (int s = 0; s < Sh::kStages; ++s) {
            mbar_init(full(s), 32 * Sh::kLoaders);
            mbar_init(empty(s), 1);
        }
        mbar_init(q_full, 32 * Sh::kLoaders);
        mbar_init(q_empty, 1);
        for (int x = 0; x < 2; ++x) {
            mbar_init(s_full(x), 1);
            mbar_init(p_full(x), 128);
            mbar_init(o_full(x), 1);
        }
        stop = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (w == Sh::kThreads / 32 - 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     :: "r"(smem_addr(&tmem_slot)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    // columns: scores (and weights over them) of the halves at 0 and 128, sums at 256 and 384
    auto wait = [&](uint32_t bar, uint32_t parity) { return mbar_wait_or_stop(bar, parity, j.wait_cycles, &stop); };
    // for roles whose lanes act together: all of a warp go on, or none
    auto wait_warp = [&](uint32_t bar, uint32_t parity) { return (bool)__all_sync(~0u, wait(bar, parity)); };
    using CutWalk = Walk<Sh::kM, Sh::kKeys>;

    if (w < 8) {
        // ---- softmax: a thread owns row `row` of half x
        const uint32_t x = w >> 2, row = tid & 127;
        const uint32_t lane_base = (w & 3) << 21;            // lanes 32 (w % 4) ..
        const uint32_t s_t = tmem + lane_base + x * 128, o_t = tmem + lane_base + 256 + x * 128;
        const float c = fmaxf(fabsf(j.scale_log2), 1e-37f);  // a negative scale negates the products
        uint32_t s_cnt = 0, o_cnt = 0, part_cnt = 0;
        CutWalk cw;
        cw.start(j, span);
        while (cw.next(j, span)) {
            const uint32_t n = half_tiles(j, cw.it, cw.p, x, Sh::kM, Sh::kKeys);
            const uint32_t row_base = cw.p.rt * Sh::kM + x * 128;
            const bool real = x * 128 + row < cw.p.rows;
            const uint32_t lim = real ? token_limit(cw.it, (row_base + row) / G) : 0x7FFFFFFFu;
            const uint32_t lim_first = token_limit(cw.it, row_base / G);
            float m = -INFINITY, l = 0.f;
            bool alive = true;
            for (uint32_t t = 0; t < n; ++t) {
                if (!(alive = wait_warp(s_full(x), s_cnt & 1))) break;
                ++s_cnt;
                tc_fence_after();
                const uint32_t key = cw.it.kv0 + (cw.p.k0 + t) * Sh::kKeys;
                const bool masked = key + Sh::kKeys > lim_first;
                const int see = masked ? (int)(lim > key ? lim - key : 0u) : Sh::kKeys;   // keys of the tile
                float top = -INFINITY;
#pragma unroll
                for (int ch = 0; ch < 4; ++ch) {
                    float v[32];
                    tmem_ld32(s_t + ch * 32, v);
                    tmem_wait_ld();
                    if (masked) {
#pragma unroll
                        for (int e = 0; e < 32; ++e) top = fmaxf(top, ch * 32 + e < see ? v[e] : -INFINITY);
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; ++e) top = fmaxf(top, v[e]);
                    }
                }
                top *= c;
                float fix = 1.f;
                if (t == 0) {
                    m = top;
                } else if (top > m + 8.f) {
                    fix = exp2f(m - top);
                    m = top;
                    l *= fix;
                }
                if (__any_sync(~0u, fix != 1.f)) {
                    // the value product of the tile before is done: its scores came after it
#pragma unroll 1
                    for (int ch = 0; ch < DP / 32; ++ch) {
                        float v[32];
                        tmem_ld32(o_t + ch * 32, v);
                        tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] *= fix;
                        tmem_st32(o_t + ch * 32, v);
                    }
                    tmem_wait_st();
                }
                const float neg = m == -INFINITY ? 0.f : -m;
                float sum0 = 0.f, sum1 = 0.f;
#pragma unroll
                for (int ch = 0; ch < 4; ++ch) {
                    float v[32];
                    uint32_t pk[16];
                    tmem_ld32(s_t + ch * 32, v);
                    tmem_wait_ld();
                    if (masked) {
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (ch * 32 + e >= see) v[e] = -INFINITY;
                    }
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        const float a = exp2f(fmaf(v[e], c, neg)), b = exp2f(fmaf(v[e + 1], c, neg));
                        sum0 += a;
                        sum1 += b;
                        // the weights are rounded to the values' type: the tensor cores take both in one
                        pk[e / 2] = Half2<T>::down(a, b);
                    }
                    tmem_st16(s_t + ch * 16, pk);
                }
                l += sum0 + sum1;
                tmem_wait_st();
                tc_fence_before();
                mbar_arrive(p_full(x));
            }
            if (alive && n) {
                alive = wait_warp(o_full(x), o_cnt & 1);
                ++o_cnt;
                tc_fence_after();
            }
            if (!alive) break;
            const bool whole = cw.p.k0 == 0 && cw.p.k1 == cw.p.units;
            float *slot = whole ? nullptr
                                : part_slot(j, 2ull * blockIdx.x + (cw.p.k0 == 0 ? 1 : 0), Sh::kM, DP);
            if (x * 128 < cw.p.rows && (n || whole)) {
#pragma unroll 1
                for (int ch = 0; ch < DP / 32; ++ch) {
                    float v[32];
                    __syncwarp();
                    if (n) {
                        tmem_ld32(o_t + ch * 32, v);
                        tmem_wait_ld();
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = 0.f;
                    }
                    if (real) {
#pragma unroll
                        for (int e = 0; e < 32; e += 4) {
                            const uint32_t d = ch * 32 + e;
                            const float4 acc = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
                            if (d >= D) continue;
                            if (whole)
                                finish_row4<T>(j, cw.it, cw.p, row_base + row, d, acc, m, l);
                            else
                                __stcg(reinterpret_cast<float4 *>(slot + (uint64_t)(x * 128 + row) * DP + d), acc);
                        }
                    }
                }
                tc_fence_before();
            }
            if (!whole) {
                if (real) {
                    __stcg(slot + (uint64_t)Sh::kM * DP + x * 128 + row, m);
                    __stcg(slot + (uint64_t)Sh::kM * (DP + 1) + x * 128 + row, l);
                }
                // as deliver_part, for the 256 threads of this role and with bounded waits
                const uint32_t c0 = (uint32_t)(cw.p.tile0 / span.per);
                __threadfence();
                mbar_arrive(part_bar);
                if (!(alive = wait_warp(part_bar, part_cnt & 1))) break;
                ++part_cnt;
                if (tid == 0) {
                    const uint32_t c1 = (uint32_t)((cw.p.tile0 + cw.p.units - 1) / span.per);
                    __threadfence();
                    last_part = atomicAdd(&j.arrived[c0], 1u) == c1 - c0;
                    if (last_part) j.arrived[c0] = 0;
                    __threadfence();
                }
                mbar_arrive(part_bar);
                if (!(alive = wait_warp(part_bar, part_cnt & 1))) break;
                ++part_cnt;
                if (last_part) {
                    __threadfence();
                    merge_parts<T, 256>(j, cw.it, cw.p, span.per, Sh::kM, DP);
                }
            }
        }
    } else if (w < 8 + Sh::kLoaders) {
        // ---- loaders
        constexpr int kSets = 4 / Sh::kLoaders;              // sets of 32 rows a warp takes of a block of 128
        const uint32_t r0 = (w - 8) * 32 * kSets;
        const uint64_t tok_stride = (uint64_t)j.n_kv_heads * D;
        uint32_t stage = 0, laps = 0, q_cnt = 0;
        uint32_t fifo[Sh::kLag] = {};
        uint32_t pending = 0;
        bool alive = true;

        auto hand_over = [&](uint32_t bar) {
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            mbar_arrive(bar);
        };
        auto push = [&](uint32_t bar) {                      // a group of copies that ends at `bar`
            asm volatile("cp.async.commit_group;" ::: "memory");
            if (pending == Sh::kLag) {
                asm volatile("cp.async.wait_group %0;" :: "n"(Sh::kLag) : "memory");
                hand_over(fifo[0]);
            } else {
                ++pending;
            }
#pragma unroll
            for (int k = 0; k + 1 < Sh::kLag; ++k) fifo[k] = fifo[k + 1];
            fifo[Sh::kLag - 1] = bar;
        };
        auto flush = [&]() {
            asm volatile("cp.async.wait_group 0;" ::: "memory");
#pragma unroll
            for (int k = 0; k < Sh::kLag; ++k)
                if (k + pending >= Sh::kLag) hand_over(fifo[k]);
            pending = 0;
        };
        // 32 rows of a block, row r at src + off(lane r): 16-byte pieces to their swizzled places
        auto copy_rows = [&](uint32_t dst, const T *src, uint64_t off, bool ok, uint32_t first) {
            const unsigned live = __ballot_sync(~0u, ok);
            const uint32_t lo = (uint32_t)off, hi = (uint32_t)(off >> 32);
#pragma unroll
            for (int y = 0; y < kChunks; ++y) {
                const uint32_t piece = y * 32 + lane, r = piece / kChunks, ck = piece % kChunks;
                const uint64_t o = ((uint64_t)__shfl_sync(~0u, hi, r) << 32) | __shfl_sync(~0u, lo, r);
                const bool in = ((live >> r) & 1u) && ck * 8 < D;
                const uint32_t at = dst + (ck >> 3) * kBlock + (first + r) * 128 + (((ck & 7) ^ (r & 7)) << 4);
                cp_async16(at, src + (in ? o + ck * 8 : 0), in);
            }
        };
        auto take_stage = [&]() {
            alive = alive && wait_warp(empty(stage), (laps & 1) ^ 1);
            return alive;
        };
        // hands the stage just filled to the issuer
        auto push_stage = [&]() {
            push(blockIdx.x == 0 && (uint64_t)laps * Sh::kStages + stage == j.test_drop ? spare_bar : full(stage));
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
            const uint32_t key_end = min(token_limit(it, (row_base + cw.p.rows - 1) / G),
                                         it.kv0 + cw.p.k1 * Sh::kKeys);
            auto page_of = [&](uint32_t t, int set) -> uint32_t {
                const uint32_t k = it.kv0 + (cw.p.k0 + t) * Sh::kKeys + r0 + set * 32 + lane;
                if (k >= key_end) return 0xFFFFFFFFu;
                const uint64_t entry = it.page0 + k / j.page_tokens;
                const uint32_t page = j.seqs.page_table[entry];
                if (page >= j.num_pages) {
                    st_flag(j.st, LSMKV_ST_BAD_PAGE, entry);
                    return 0xFFFFFFFFu;
                }
                return page;
            };
            const uint32_t n = cw.p.k1 - cw.p.k0;
            uint32_t page[kSets];                            // a tile ahead of the copies
#pragma unroll
            for (int y = 0; y < kSets; ++y) page[y] = page_of(0, y);
            for (uint32_t t = 0; t < n; ++t) {
                uint64_t off[kSets];
                bool ok[kSets];
#pragma unroll
                for (int y = 0; y < kSets; ++y) {
                    const uint32_t k = it.kv0 + (cw.p.k0 + t) * Sh::kKeys + r0 + y * 32 + lane;
                    ok[y] = page[y] != 0xFFFFFFFFu;
                    off[y] = ok[y] ? ((uint64_t)page[y] * j.page_tokens + k % j.page_tokens) * tok_stride +
                                         (uint64_t)cw.p.kv_head * D
                                   : 0;
                    if (t + 1 < n) page[y] = page_of(t + 1, y);
                }
                if (!take_stage()) break;
#pragma unroll
                for (int y = 0; y < kSets; ++y)
                    copy_rows(ring + stage * Sh::kTileBytes, kbuf, off[y], ok[y], r0 + y * 32);
                push_stage();
                if (t == 0) {
                    // the queries, once the products of the cut before have read theirs
                    flush();
                    if (!(alive = wait_warp(q_empty, (q_cnt & 1) ^ 1))) break;
                    ++q_cnt;
                    for (uint32_t x = 0; x < 2 && x * 128 < cw.p.rows; ++x) {
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
                    push(q_full);
                }
                if (!take_stage()) break;
#pragma unroll
                for (int y = 0; y < kSets; ++y)
                    copy_rows(ring + stage * Sh::kTileBytes, vbuf, off[y], ok[y], r0 + y * 32);
                push_stage();
            }
        }
        flush();
    } else {
        // ---- issuer: the warp walks and waits together, one lane issues
        const uint32_t type = std::is_same<T, __half>::value ? 0u : 1u;
        const uint32_t common = (1u << 4) | (type << 7) | (type << 10) | (8u << 24);   // f32 sums, M = 128
        const uint32_t k_steps = (D + 15) / 16, n_out = k_steps * 16;
        const uint32_t id_s = common | ((Sh::kKeys / 8) << 17) | (j.scale_log2 < 0.f ? 1u << 13 : 0u);
        const uint32_t id_o = common | ((n_out / 8) << 17) | (1u << 16);
        uint32_t pos = 0;             // tiles taken from the ring: keys and values in turn
        uint32_t q_cnt = 0, p_cnt[2] = {0, 0};
        bool alive = true;
        auto stage_of = [&](uint32_t at) { return at % Sh::kStages; };
        auto lap_of = [&](uint32_t at) { return (at / Sh::kStages) & 1; };
        auto scores = [&](uint32_t x, uint32_t st) {
            if (lane) return;
            const uint64_t a = desc_k_major(q_s + x * Sh::kTileBytes), b = desc_k_major(ring + st * Sh::kTileBytes);
            for (uint32_t k = 0; k < k_steps; ++k) {
                const uint64_t step = (k >> 2) * (kBlock >> 4) + (k & 3) * 2;   // 64 elements a block, 16 a step
                mma_ss(tmem + x * 128, a + step, b + step, id_s, k != 0);
            }
        };
        auto values = [&](uint32_t x, uint32_t st, bool add) {
            if (lane) return;
            const uint64_t b = desc_mn_major(ring + st * Sh::kTileBytes, kBlock);
            for (uint32_t k = 0; k < Sh::kKeys / 16; ++k)
                mma_ts(tmem + 256 + x * 128, tmem + x * 128 + k * 8, b + k * (2048 >> 4), id_o, add || k != 0);
        };
        auto commit = [&](uint32_t bar) {
            if (lane == 0) mma_commit(bar);
        };
        CutWalk cw;
        cw.start(j, span);
        while (alive && cw.next(j, span)) {
            const uint32_t n = cw.p.k1 - cw.p.k0;
            const uint32_t nx[2] = {half_tiles(j, cw.it, cw.p, 0, Sh::kM, Sh::kKeys),
                                    half_tiles(j, cw.it, cw.p, 1, Sh::kM, Sh::kKeys)};
            const uint32_t at = pos;
            pos += 2 * n;
            if (!(alive = wait_warp(q_full, q_cnt & 1))) break;
            ++q_cnt;
            if (!(alive = wait_warp(full(stage_of(at)), lap_of(at)))) break;
            tc_fence_after();
            for (uint32_t x = 0; x < 2; ++x)
                if (nx[x]) {
                    scores(x, stage_of(at));
                    commit(s_full(x));
                }
            commit(empty(stage_of(at)));
            if (n == 1) commit(q_empty);
            for (uint32_t t = 0; t < n && alive; ++t) {
                const uint32_t v_at = at + 2 * t + 1, k_at = v_at + 1;
                if (!(alive = wait_warp(full(stage_of(v_at)), lap_of(v_at)))) break;
                bool key_here = false;
                for (uint32_t x = 0; x < 2; ++x) {
                    if (t < nx[x]) {
                        if (!(alive = wait_warp(p_full(x), p_cnt[x] & 1))) break;
                        ++p_cnt[x];
                        tc_fence_after();
                        values(x, stage_of(v_at), t != 0);
                    }
                    if (t + 1 < nx[x]) {
                        if (!key_here && !(alive = wait_warp(full(stage_of(k_at)), lap_of(k_at)))) break;
                        key_here = true;
                        scores(x, stage_of(k_at));
                        commit(s_full(x));
                    } else if (t + 1 == nx[x]) {
                        commit(o_full(x));
                    }
                }
                if (!alive) break;
                commit(empty(stage_of(v_at)));
                if (t + 1 < n) {
                    commit(empty(stage_of(k_at)));
                    if (t + 2 == n) commit(q_empty);
                }
            }
        }
        // products still under way read shared memory and write TMEM: let them end
        commit(done_bar);
        (void)mbar_wait_bounded(done_bar, 0, j.wait_cycles);
    }
    __syncwarp();
    asm volatile("cp.async.wait_all;" ::: "memory");
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (w == Sh::kThreads / 32 - 1)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem), "r"(512u) : "memory");
    if (tid == 0 && stop) st_flag(j.st, LSMKV_ST_WAIT_EXPIRED, blockIdx.x);
}

}  // namespace lsmkv
