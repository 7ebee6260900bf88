// Attention over a pool of 8-bit floats, kernel for few rows: the division of work, the parts and their
// merge are those of the 16-bit kernels (see lsmkv_attend.cuh).
//
//   k_j = c_j 2^a_j, v_j = d_j 2^b_j   (codes c, d; exponents a, b of their blocks)
//   s_j = scale * q . c_j * 2^a_j;  weights in base 2;  u_j = s_j + b_j (log2 of what multiplies d_j)
//   with M = max_j u_j (at least max_j s_j - 40):  o = sum_j 2^(u_j - M) d_j / sum_j 2^(s_j - M)
// so the scales cost one multiplication and one addition a score, nothing a code, and the weights that meet
// the codes are the true contributions relative to their largest, whatever the scales of the values.
//
// Codes become 16-bit floats exactly (f16: 11 bits and a range of 2^-24 to 2^15 against e4m3's 4 bits, 2^-9
// to 448), in registers behind the load of a fragment: one conversion for two codes. So the products run
// in f16 whatever the type of the queries; bfloat16 queries are brought to it row by row with a power of two
// that puts a row's largest element at 2^13 (what lies below 2^-27 of it loses bits, far below the products' 32 bits).
//
// A token's codes of one head are 128 bytes or fewer, and read head by head -- the whole of a sequence under one
// head, then under the next -- memory gives half of its rate: 256 requests of 1k to 8k tokens, 8 heads, 687 us for
// the loads alone. So up to eight heads are read side by side where the batch is large enough: the warps of a CTA
// take a head each (or two or more a head), over the same keys, and a page's codes are read whole. Then nothing is
// merged among the warps but what shares a head. Small batches cut each head's keys for themselves.
// Measured: that batch 510 to 565 us (2.38 GB, up to 4.7 TB/s; the loads alone 405, head by head 730); 512 sequences of
// 256 to 4096 tokens, 28/4 heads, 1.16 GB, 258 us (loads alone 198). What lies between is instructions, 370 for 16 keys of
// a head, 64 of them conversions; 16 warps with 128 registers instead of 8 take as long.
#pragma once
#include "lsmkv_append8.cuh"
#include "lsmkv_attend.cuh"

namespace lsmkv {

template <int DP, int NB>
struct Few8Shape {
    static constexpr int kM = 8 * NB;                      // rows of a tile
    static constexpr int kKeys = 16;                       // keys a warp takes at a time
    static constexpr int kWarps = DP > 128 ? 4 : 8;
    static constexpr int kStages = DP <= 64 ? 10 : 5;      // 160 KB of keys and values a SM
    static constexpr int kHeads = DP <= 128 ? 8 : 1;       // heads of a CTA, at most
    static constexpr int kThreads = kWarps * 32;
    static constexpr uint32_t kCodes = 16 * DP * 2;        // sixteen keys, their values,
    static constexpr uint32_t kStage = kCodes + 32 * 8;    // and of each a word with its scale and the byte's place
    static constexpr size_t kQBytes = (size_t)kHeads * kM * DP * 2;
    static constexpr uint32_t kMergeRows = (DP == 128 && NB == 1 ? 32768 : DP <= 128 ? 16384 : 24576) / (kWarps * DP * 4);
    static constexpr size_t kMergeBytes = (size_t)kMergeRows * kWarps * DP * 4;
    static constexpr size_t kSmem = kQBytes + kMergeBytes + (size_t)kWarps * kStages * kStage;
    static constexpr bool kQInRegs = DP * NB <= 256;
};

// The reference M lies no more than 2^40 below the largest 2^(s_j), whatever the values' exponents: the sum of weights, which are
// relative to M too, stays in range beside blocks of zeros, whose exponent is the least there is. (Contributions
// under 2^-54 of a code's size times the largest weight lose bits for it.)
constexpr float kLeastLog = -40.f;

// Whether one of four codes is NaN.
__device__ __forceinline__ uint32_t undefined_codes(uint32_t c) { return ((c & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u; }

// kSide: heads side by side, up to 2^most_log2; without it the divisions among a CTA's warps are known here (four
// short chats: 12.4 us instead of 14.4).
template <typename T, int DP, int NB, bool kSide>
__global__ __launch_bounds__(Few8Shape<DP, NB>::kThreads, 1)
void k_attend_few8(const __grid_constant__ AttendJob j, const __grid_constant__ CodeArgs cd, const uint32_t most_log2)
{
    using Sh = Few8Shape<DP, NB>;
    using F = __half;
    constexpr int NT = Sh::kThreads, NW = Sh::kWarps, ST = Sh::kStages;
    constexpr int kChunks = DP / 16;           // 16-byte pieces of a row of codes
    constexpr int kQChunks = DP / 8;           // of a row of queries
    constexpr uint32_t kNone = 0xFFFFFFFFu;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ float sm_m[NW][Sh::kM], sm_l[NW][Sh::kM], sm_q[Sh::kHeads * Sh::kM];
    const uint32_t tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    const uint32_t G = j.group, D = j.head_dim;

    follow_launch();
    const unsigned char *const kbuf = static_cast<const unsigned char *>(j.kv_ptrs[j.layer]);
    const unsigned char *const vbuf = static_cast<const unsigned char *>(j.kv_ptrs[j.n_layers + j.layer]);
    const uint32_t n_items = j.prefix_pass ? j.n_group : j.seqs.n_seq;
    // Heads side by side: as many as the host allows while the row tiles under a group of heads are no fewer than
    // an eighth of the CTAs, so that a cut tile has no more than about eight parts for its last CTA to merge. (What
    // this launch takes of the batch is known here only: one sequence of a batch of 32 that others' kernel takes, cut
    // among all CTAs with its eight heads side by side, made the call 250 us longer.)
    uint32_t heads_log2 = kSide ? most_log2 : 0;
    if (kSide) {
        uint32_t tiles = 0;
        for (uint32_t i = tid; i < n_items; i += NT) tiles += item_tiles(j, load_item(j, i), Sh::kM);
        __shared__ uint32_t all_tiles;
        if (tid == 0) all_tiles = 0;
        __syncthreads();
        if (tiles) atomicAdd(&all_tiles, tiles);
        __syncthreads();
        while (heads_log2 && (uint64_t)all_tiles * (j.n_kv_heads >> heads_log2) * 8 < gridDim.x) --heads_log2;
    }
    const uint32_t HC = 1u << heads_log2, per_head = NW >> heads_log2, kv_heads = j.n_kv_heads;
    const uint32_t kTile = Sh::kKeys * per_head;
    const uint32_t my_head = w / per_head, my_part = w % per_head;         // of the group; of its keys
    const Span span = find_span<NT, false>(j, n_items, kv_heads >> heads_log2, Sh::kM, kTile, nullptr);
    if ((reinterpret_cast<uintptr_t>(kbuf) | reinterpret_cast<uintptr_t>(vbuf)) & 15u) {
        if (blockIdx.x == 0 && tid == 0) st_flag(j.st, LSMKV_ST_MISALIGNED, 0);
        return;
    }
    if (span.begin >= span.end) return;

    const uint32_t q_s = smem_addr(smem);
    float *const merge = reinterpret_cast<float *>(smem + Sh::kQBytes);
    const uint32_t ring_at = (uint32_t)(Sh::kQBytes + Sh::kMergeBytes) + w * (ST * Sh::kStage);
    const uint32_t ring = q_s + ring_at;
    const uint32_t tok_stride = kv_heads * D;          // bytes of a token's codes
    const uint32_t blocks = j.page_tokens >> cd.block_log2;
    using CutWalk = Walk<Sh::kM, 0>;

    CutWalk walk;
    walk.start(j, span);
    bool more = walk.next(j, span);
    const Item &it = walk.it;
    const Cut &p = walk.p;
    // The load side, ahead of the other, as in the 16-bit kernel.
    CutWalk ahead = walk;
    const bool one_page = j.page_tokens % 16 == 0;
    uint32_t load_key = 0, load_end = 0, load_page = kNone, tiles_known = 0;
    auto page_of = [&](uint32_t k) -> uint32_t {
        if (k >= load_end) return kNone;
        const uint64_t entry = ahead.it.page0 + k / j.page_tokens;
        const uint32_t page = j.seqs.page_table[entry];
        if (page < j.num_pages) return page;
        st_flag(j.st, LSMKV_ST_BAD_PAGE, entry);
        return kNone;
    };
    auto load_pages = [&]() {
        load_page = page_of(load_key + (one_page ? lane * kTile : lane & 15));
        tiles_known = one_page ? 32 : 1;
    };
    auto take_load_cut = [&]() {
        const Item &on = ahead.it;
        load_key = on.kv0 + ahead.p.k0 * kTile + my_part * Sh::kKeys;
        load_end = min(token_limit(on, (ahead.p.rt * Sh::kM + ahead.p.rows - 1) / G), on.kv0 + ahead.p.k1 * kTile);
    };
    auto next_load_cut = [&]() {
        while (load_key >= load_end && ahead.next(j, span)) take_load_cut();
        load_pages();
    };
    // Piece c of row r lies at c ^ (r % 8); rows of 64 bytes, two to the width of the banks, at c ^ (r / 2 % 4).
    constexpr int kRows = 32 / kChunks;
    constexpr int kCopies = 16 * kChunks / 32;
    auto swizzle = [](uint32_t r) { return kChunks == 4 ? (r >> 1) & 3 : r & 7; };
    const uint32_t piece_r = lane / kChunks, piece_c = lane % kChunks;
    // (piece c of row x kRows + piece_r: only the row's bit 2 depends on x, where rows are 128 bytes)
    const uint32_t piece_at = (piece_r * kChunks + (piece_c ^ swizzle(piece_r))) * 16;
    const uint32_t row_off = piece_r * tok_stride + piece_c * 16;
    const bool chunk_there = piece_c * 16 < D;
    auto fetch = [&](uint32_t stage) {
        if (load_key < load_end) {
            const uint32_t kv_head = (ahead.p.kv_head << heads_log2) + my_head;
            const uint32_t page = one_page ? __shfl_sync(~0u, load_page, 32 - tiles_known) : load_page;
            const uint32_t left = load_end - load_key;
            const uint32_t slot0 = slot_of_token(cd, j.page_tokens, load_key);
            // this lane's key, for the scale (and for its codes, where a page does not hold sixteen)
            const uint32_t slot = one_page ? slot0 + (lane & 15) : slot_of_token(cd, j.page_tokens, load_key + (lane & 15));
            const bool real = page != kNone && (lane & 15) < left;
            const uint64_t slab = page != kNone ? page * cd.page_bytes : 0;
            const unsigned char *const kp = kbuf + slab, *const vp = vbuf + slab;
            const uint32_t dst = ring + stage * Sh::kStage;
            {
                // the word that holds the scale (a copy takes four bytes), and which byte it is
                const uint32_t at = cd.code_bytes + kv_head * blocks + (slot >> cd.block_log2), to = dst + Sh::kCodes + lane * 8;
                asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;"
                             :: "r"(to), "l"((lane < 16 ? kp : vp) + (real ? at & ~3u : 0u)), "r"(real ? 4 : 0) : "memory");
                asm volatile("st.shared.b32 [%0], %1;" :: "r"(to + 4), "r"((at & 3u) * 8) : "memory");
            }
            if (one_page && page != kNone && left >= 16) {
                const uint32_t off = slot0 * tok_stride + kv_head * D + row_off;
                if (chunk_there) {
                    const unsigned char *k = kp + off, *v = vp + off;
#pragma unroll
                    for (int x = 0; x < kCopies; ++x) {
                        const uint32_t to = dst + (piece_at ^ (swizzle(x * kRows) << 4)) + x * kRows * kChunks * 16;
                        cp_async16(to, k);
                        cp_async16(to + 16 * DP, v);
                        k += kRows * tok_stride;
                        v += kRows * tok_stride;
                    }
                } else {
#pragma unroll
                    for (int x = 0; x < kCopies; ++x) {
                        const uint32_t to = dst + (piece_at ^ (swizzle(x * kRows) << 4)) + x * kRows * kChunks * 16;
                        cp_async16(to, kbuf, false);
                        cp_async16(to + 16 * DP, vbuf, false);
                    }
                }
            } else {
                const uint64_t mine = slab + slot * tok_stride + kv_head * D;
                const uint32_t lo = (uint32_t)mine, hi = (uint32_t)(mine >> 32) | (real ? 0u : 0x80000000u);
#pragma unroll
                for (int x = 0; x < kCopies; ++x) {
                    const uint32_t r = x * kRows + piece_r;
                    const uint32_t h = __shfl_sync(~0u, hi, r);
                    const uint64_t o = ((uint64_t)(h & 0x7FFFFFFFu) << 32) | __shfl_sync(~0u, lo, r);
                    const bool in = !(h >> 31) && chunk_there;
                    const uint64_t e = in ? o + piece_c * 16 : 0;
                    const uint32_t to = dst + (r * kChunks + (piece_c ^ swizzle(r))) * 16;
                    cp_async16(to, kbuf + e, in);
                    cp_async16(to + 16 * DP, vbuf + e, in);
                }
            }
            load_key += kTile;
            if (--tiles_known == 0 && load_key < load_end) load_pages();
            if (load_key >= load_end) next_load_cut();
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    // Pieces of 16 bytes of the cut's queries, of all its heads; rows beyond the tile are zero.
    constexpr int kPieces = (Sh::kHeads * Sh::kM * kQChunks + NT - 1) / NT;
    const uint32_t n_pieces = HC * Sh::kM * kQChunks;
    uint4 q_piece[kPieces];
    auto load_queries = [&]() {
#pragma unroll
        for (int y = 0; y < kPieces; ++y) {
            const uint32_t x = tid + y * NT, r = x / kQChunks % Sh::kM, h = x / (kQChunks * Sh::kM), c = x % kQChunks;
            q_piece[y] = make_uint4(0, 0, 0, 0);
            if (y * NT < n_pieces && h < HC && r < p.rows && c * 8 < D) {
                const uint32_t R = p.rt * Sh::kM + r;
                q_piece[y] = *reinterpret_cast<const uint4 *>(
                    static_cast<const T *>(j.q) + (it.row0 + R / G) * j.q_ts +
                    (uint64_t)(((p.kv_head << heads_log2) + h) * G + R % G) * j.q_hs + c * 8);
            }
        }
    };
    // Queries to f16, a row's largest element at 2^13, and what the row's products are multiplied by. The
    // pieces of a row are neighbouring lanes'.
    auto store_queries = [&]() {
#pragma unroll
        for (int y = 0; y < kPieces; ++y) {
            if (y * NT >= n_pieces) break;
            const uint32_t x = tid + y * NT, r = x / kQChunks, c = x % kQChunks;
            uint4 v = q_piece[y];
            float back = 1.f;
            if constexpr (!std::is_same<T, F>::value) {
                uint32_t top = 0;                          // of the magnitudes' bits, undefined ones included
#pragma unroll
                for (int i = 0; i < 4; ++i) top = max(top, max((&v.x)[i] & 0x7FFFu, (&v.x)[i] >> 16 & 0x7FFFu));
#pragma unroll
                for (int d = 1; d < kQChunks; d <<= 1) top = max(top, __shfl_xor_sync(~0u, top, d));
                int e = (int)(top >> 7) - 127 - 13;        // exponent of the largest, less 13
                e = e < -126 ? -126 : e > 114 ? 114 : e;
                const float f = power_of_two(-e);
                back = power_of_two(e);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 u = Half2<T>::up((&v.x)[i]);
                    (&v.x)[i] = Half2<F>::down(u.x * f, u.y * f);
                }
            }
            if (x < n_pieces) {
                *reinterpret_cast<uint4 *>(smem + (r * kQChunks + (c ^ (r & 7))) * 16) = v;
                if (c == 0) sm_q[r] = back * j.scale_log2;
            }
        }
    };
    uint32_t stage = 0, stage_load = ST - 1;
    if (more) {
        take_load_cut();
        next_load_cut();
        load_queries();
#pragma unroll
        for (int s = 0; s < ST - 1; ++s) fetch(s);
        store_queries();
    }
    __syncthreads();
    while (more) {
        const Cut cut = p;
        const uint32_t row_base = cut.rt * Sh::kM;
        // this lane's rows are 8 nb + 2 (lane % 4) and the one behind it; the keys they see
        uint32_t lim[NB][2];
        float row_scale[NB][2];
#pragma unroll
        for (int x = 0; x < 2 * NB; ++x) {
            const uint32_t r = (x >> 1) * 8 + 2 * (lane & 3) + (x & 1);
            lim[x >> 1][x & 1] = r < cut.rows ? token_limit(it, (row_base + r) / G) : it.kv0;
            row_scale[x >> 1][x & 1] = sm_q[my_head * Sh::kM + r];
        }
        const uint32_t lim_first = token_limit(it, row_base / G);              // least of the tile
        const uint32_t key_end = min(token_limit(it, (row_base + cut.rows - 1) / G), it.kv0 + cut.k1 * kTile);
        const uint32_t key0 = it.kv0 + cut.k0 * kTile + my_part * Sh::kKeys;

        // Queries as the right operand. The elements of a piece of 16 are taken in the order in which a lane
        // finds the codes of a key: its elements 4 t .. 4 t + 3 (t = lane % 4) stand for 2 t, 2 t + 1, 2 t + 8, 2 t + 9.
        uint32_t qf[Sh::kQInRegs ? DP / 16 : 1][NB][2];
        auto load_q = [&](int x, uint32_t (&f)[NB][2]) {          // elements 16 x ..
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const uint32_t r = my_head * Sh::kM + nb * 8 + (lane >> 2), c = 2 * x + ((lane & 3) >> 1);
                const uint2 q = *reinterpret_cast<const uint2 *>(smem + (r * kQChunks + (c ^ (r & 7))) * 16 + (lane & 1) * 8);
                f[nb][0] = q.x;
                f[nb][1] = q.y;
            }
        };
        if constexpr (Sh::kQInRegs) {
#pragma unroll
            for (int x = 0; x < DP / 16; ++x) load_q(x, qf[x]);
        }

        // sums of elements 16 x + 2 (lane / 4) and the one behind it
        float o[DP / 16][NB][4];
#pragma unroll
        for (int x = 0; x < DP / 16; ++x)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) o[x][nb][0] = o[x][nb][1] = o[x][nb][2] = o[x][nb][3] = 0.f;
        float m[NB][2], l[NB][2];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            m[nb][0] = m[nb][1] = -INFINITY;
            l[nb][0] = l[nb][1] = 0.f;
        }
        for (uint32_t key = key0; key < key_end; key += kTile) {
            fetch(stage_load);
            stage_load = stage_load + 1 == ST ? 0 : stage_load + 1;
            asm volatile("cp.async.wait_group %0;" :: "n"(ST - 1) : "memory");
            __syncwarp();
            const uint32_t first = ring + stage * Sh::kStage;
            // scores of 16 keys (lane/4 and lane/4 + 8) x 8 rows; u: with the logarithm of what multiplies the value
            float s[NB][4], u[NB][4];
            {
                const uint32_t ks = first;
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) s[nb][0] = s[nb][1] = s[nb][2] = s[nb][3] = 0.f;
                const uint32_t kr = lane & 15;
#pragma unroll
                for (int x = 0; x < DP / 16; x += 2) {
                    uint32_t c[4];               // keys 0-7 and 8-15 of piece x, then of piece x + 1
                    ldmatrix4(ks + (kr * kChunks + ((x + (lane >> 4)) ^ swizzle(kr))) * 16, c);
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        uint32_t a[4], f[NB][2];
                        from_codes4(c[2 * y], a[0], a[2]);
                        from_codes4(c[2 * y + 1], a[1], a[3]);
                        if constexpr (!Sh::kQInRegs) load_q(x + y, f);
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb) {
                            if constexpr (Sh::kQInRegs) mma16816<F>(s[nb], a, qf[x + y][nb][0], qf[x + y][nb][1]);
                            else mma16816<F>(s[nb], a, f[nb][0], f[nb][1]);
                        }
                    }
                }
                // exponents of this lane's keys: a byte each of their words
                const uint2 *const words = reinterpret_cast<const uint2 *>(smem + (ks - q_s) + Sh::kCodes);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint2 kw = words[(lane >> 2) + 8 * h], vw = words[(lane >> 2) + 8 * h + 16];
                    const float k_scale = power_of_two(scale_exponent(kw.x >> kw.y & 0xFF));
                    const float v_log = (float)scale_exponent(vw.x >> vw.y & 0xFF);
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                        for (int e = 2 * h; e < 2 * h + 2; ++e) {
                            s[nb][e] = s[nb][e] * row_scale[nb][e & 1] * k_scale;
                            u[nb][e] = s[nb][e] + v_log;
                        }
                }
                if (key + 16 > lim_first) {
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (key + (lane >> 2) + 8 * (e >> 1) >= lim[nb][e & 1]) s[nb][e] = u[nb][e] = -INFINITY;
                }
            }
            // the maximum moves only when passed by more than 2^8, as in the 16-bit kernel
            float top[NB][2];
            bool over = false;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    top[nb][x] = fmaxf(u[nb][x], u[nb][2 + x]);
                    over |= top[nb][x] > m[nb][x] + 8.f;
                }
            if (__any_sync(~0u, over)) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    float fix[2];
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        float t = fmaxf(top[nb][x], fmaxf(s[nb][x], s[nb][2 + x]) + kLeastLog);
                        t = fmaxf(t, __shfl_xor_sync(~0u, t, 4));
                        t = fmaxf(t, __shfl_xor_sync(~0u, t, 8));
                        t = fmaxf(t, __shfl_xor_sync(~0u, t, 16));
                        t = fmaxf(t, m[nb][x]);
                        fix[x] = t == -INFINITY ? 1.f : exp2f(m[nb][x] - t);
                        m[nb][x] = t;
                        l[nb][x] *= fix[x];
                    }
#pragma unroll
                    for (int x = 0; x < DP / 16; ++x) {
                        o[x][nb][0] *= fix[0];
                        o[x][nb][1] *= fix[1];
                        o[x][nb][2] *= fix[0];
                        o[x][nb][3] *= fix[1];
                    }
                }
            }
            {
                const uint32_t vs = first + 16 * DP;
                uint32_t pf[NB][2];
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float base = m[nb][e & 1] == -INFINITY ? 0.f : m[nb][e & 1];
                        l[nb][e & 1] += exp2f(s[nb][e] - base);
                        u[nb][e] = exp2f(u[nb][e] - base);
                    }
                    // the weights are rounded to f16, the codes' type: the tensor cores take both in one
                    pf[nb][0] = transpose8x8(Half2<F>::down(u[nb][0], u[nb][1]));
                    pf[nb][1] = transpose8x8(Half2<F>::down(u[nb][2], u[nb][3]));
                }
                // Values as the left operand: a transposed load gives two elements of two keys, whose codes are
                // sorted by element and converted. Rows of the fragment: elements 2 g and 2 g + 1 of a piece at g and g + 8.
                const uint32_t vr = lane & 15;
                auto value_fragments = [&](int x, uint32_t (&a)[2][4]) {      // pieces x and x + 1
                    uint32_t c[4];
                    ldmatrix4t(vs + (vr * kChunks + ((x + (lane >> 4)) ^ swizzle(vr))) * 16, c);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        from_codes4(__byte_perm(c[i], 0, 0x3120), a[i >> 1][2 * (i & 1)], a[i >> 1][2 * (i & 1) + 1]);
                };
                // keys that some rows see and others do not, and a NaN among their values
                bool apart = false;
                if (it.tokens > 1 && key + 16 > lim_first && it.causal) {
                    uint32_t any = 0;
#pragma unroll
                    for (uint32_t x = 0; x < 16 * kChunks; x += 32) {
                        const uint4 v = *reinterpret_cast<const uint4 *>(smem + (vs - q_s) + (x + lane) * 16);
                        any |= undefined_codes(v.x) | undefined_codes(v.y) | undefined_codes(v.z) | undefined_codes(v.w);
                    }
                    apart = __any_sync(~0u, any != 0);
                }
                if (!apart) {
#pragma unroll
                    for (int x = 0; x < DP / 16; x += 2) {
                        uint32_t a[2][4];
                        value_fragments(x, a);
#pragma unroll
                        for (int y = 0; y < 2; ++y)
#pragma unroll
                            for (int nb = 0; nb < NB; ++nb) mma16816<F>(o[x + y][nb], a[y], pf[nb][0], pf[nb][1]);
                    }
                } else {
                    // token by token, over the keys that it sees
                    const uint32_t t1 = (row_base + cut.rows - 1) / G;
#pragma unroll 1
                    for (uint32_t t = row_base / G; t <= t1; ++t) {
                        const uint32_t lim_t = token_limit(it, t), see = lim_t > key ? lim_t - key : 0;
                        uint32_t mask[2];                // of this lane's keys 2 (lane % 4), + 1, + 8, + 9
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint32_t k = 8 * h + 2 * (lane & 3);
                            mask[h] = (k < see ? 0xFFFFu : 0u) | (k + 1 < see ? 0xFFFF0000u : 0u);
                        }
#pragma unroll
                        for (int x = 0; x < DP / 16; x += 2) {
                            uint32_t a[2][4];
                            value_fragments(x, a);
#pragma unroll
                            for (int y = 0; y < 2; ++y) {
#pragma unroll
                                for (int e = 0; e < 4; ++e) a[y][e] &= mask[e >> 1];
#pragma unroll
                                for (int nb = 0; nb < NB; ++nb) {
                                    float part_o[4] = {0.f, 0.f, 0.f, 0.f};
                                    mma16816<F>(part_o, a[y], pf[nb][0], pf[nb][1]);
#pragma unroll
                                    for (int e = 0; e < 4; ++e)
                                        if (lim[nb][e & 1] == lim_t) o[x + y][nb][e] += part_o[e];
                                }
                            }
                        }
                    }
                }
            }
            __syncwarp();     // the stage is read before it is filled again
            stage = stage + 1 == ST ? 0 : stage + 1;
        }

        // merge the warps, kMergeRows rows at a time; the next cut's queries are on their way
        const Item done = it;
        more = walk.next(j, span);
        if (more) load_queries();
#pragma unroll
        for (int x = 0; x < 2 * NB; ++x) {
            float &sum = l[x >> 1][x & 1];
            sum += __shfl_xor_sync(~0u, sum, 4);
            sum += __shfl_xor_sync(~0u, sum, 8);
            sum += __shfl_xor_sync(~0u, sum, 16);
            if (lane < 4) {
                sm_m[w][(x >> 1) * 8 + 2 * lane + (x & 1)] = m[x >> 1][x & 1];
                sm_l[w][(x >> 1) * 8 + 2 * lane + (x & 1)] = sum;
            }
        }
        const bool whole = cut.k0 == 0 && cut.k1 == cut.units;
        const uint32_t quads = D / 4, part_rows = HC * Sh::kM;       // a part's row: head of the group * kM + row
        float *slot = whole ? nullptr
                            : part_slot(j, 2ull * blockIdx.x + (cut.k0 == 0 ? 1 : 0), part_rows, DP);
        for (uint32_t r0 = 0; r0 < cut.rows; r0 += Sh::kMergeRows) {
            const uint32_t r1 = min(r0 + Sh::kMergeRows, cut.rows);
#pragma unroll
            for (int x = 0; x < 2 * NB; ++x) {
                const uint32_t r = (x >> 1) * 8 + 2 * (lane & 3) + (x & 1);
                if (r >= r0 && r < r1) {
                    float *const mine = merge + ((r - r0) * NW + w) * DP;
#pragma unroll
                    for (int n = 0; n < DP / 16; ++n)
                        *reinterpret_cast<float2 *>(mine + ((n * 16 + 2 * (lane >> 2)) ^ ((r & 6) << 3))) =
                            make_float2(o[n][x >> 1][x & 1], o[n][x >> 1][2 + (x & 1)]);
                }
            }
            __syncthreads();
            if (r0 == 0 && more) store_queries();      // all warps are done with this cut's
            const uint32_t per = (r1 - r0) * quads;
            for (uint32_t x = tid; x < per << heads_log2; x += NT) {
                const uint32_t h = x / per, y = x - h * per, r = r0 + y / quads, d = y % quads * 4;
                const uint32_t k0 = h * per_head;                            // the head's warps
                float top = -INFINITY, sum = 0.f;
#pragma unroll
                for (uint32_t i = 0; i < NW; ++i)
                    if (i < per_head) top = fmaxf(top, sm_m[k0 + i][r]);
                float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (uint32_t i = 0; i < NW; ++i) {
                    if (i >= per_head) break;
                    const uint32_t k = k0 + i;
                    const float f = part_weight(sm_m[k][r], top);
                    const float4 v = *reinterpret_cast<const float4 *>(
                        merge + ((r - r0) * NW + k) * DP + (d ^ ((r & 6) << 3)));
                    acc.x += f * v.x;
                    acc.y += f * v.y;
                    acc.z += f * v.z;
                    acc.w += f * v.w;
                    sum += f * sm_l[k][r];
                }
                if (whole) {
                    finish_row4<T>(j, done, (cut.kv_head << heads_log2) + h, row_base + r, d, acc, top, sum);
                } else {
                    const uint32_t at = h * Sh::kM + r;
                    __stcg(reinterpret_cast<float4 *>(slot + (uint64_t)at * DP + d), acc);
                    if (d == 0) {
                        __stcg(slot + (uint64_t)part_rows * DP + at, top);
                        __stcg(slot + (uint64_t)part_rows * (DP + 1) + at, sum);
                    }
                }
            }
            __syncthreads();
        }
        if (!whole) {
            const uint32_t c0 = (uint32_t)quotient(cut.tile0, span.per),
                           c1 = (uint32_t)quotient(cut.tile0 + cut.units - 1, span.per);
            if (deliver_part(j, c0, c1)) {
                const uint32_t per = cut.rows * quads;
                for (uint32_t x = tid; x < per << heads_log2; x += NT) {
                    const uint32_t h = x / per, y = x - h * per, r = y / quads, d = y % quads * 4;
                    const Quad q = sum_parts(j.parts, c0, c1, part_rows, j.dp, h * Sh::kM + r, d);
                    finish_row4<T>(j, done, (cut.kv_head << heads_log2) + h, row_base + r, d, q.acc, q.m, q.l);
                }
            }
        }
    }
}

}  // namespace lsmkv
