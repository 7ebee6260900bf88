// Attention over the paged pool: what both kernels share (the batch as a list of row tiles and
// its division among the CTAs, partial results and their merge), and the kernel for few rows.
//
// For a row (query of one head at position p) with keys k_j, values v_j, j <= p:
//   m = max_j s_j, s_j = scale * q . k_j;  l = sum_j exp(s_j - m);  o = sum_j exp(s_j - m) v_j / l
// The sums can be taken in parts: parts (m_1, l_1, o_1), (m_2, l_2, o_2) merge into
//   m = max(m_1, m_2), l = l_1 e^(m_1-m) + l_2 e^(m_2-m), o = likewise
// so one pass over the keys suffices, and the keys of a row may be split among warps and CTAs.
// Exponents are kept in base 2 (scale * log2 e is folded into the scores).
//
// Division of work. The query heads of one KV head read the same keys, so a row tile is up to M
// rows of one sequence under one KV head (row r = token r / G, head r % G), and its cost is the
// number of key tiles that its last row sees. All tiles in a row -- sequence, KV head, row tile,
// key tile -- form one line of units that is cut into equal spans, one per CTA: no CTA has more
// than the total over the CTAs, rounded up, whatever the lengths. (The last spans may be shorter or
// empty: with few units a CTA the rounding shows, 149 units on 148 CTAs keep half of them busy. In
// the many-row kernel whole tiles may come first, see find_span; every tile's length holds one unit
// for what its beginning and end cost, kTileCost.) A row tile cut by a span's end leaves parts in
// scratch, merged in order by whoever comes after (the CTA that delivers the last part in the few-row
// kernel, a launch of its own behind the many-row kernel), so that results do not depend on timing.
// Every CTA finds its span by itself, from the lengths: no launch before, and nothing for the host to
// know.
#pragma once
#include <type_traits>

#include "lsmkv_append.cuh"
#include "lsmkv_copy.cuh"

namespace lsmkv {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct AttendJob {
    SeqArgs seqs;
    void *const *kv_ptrs;
    uint64_t num_pages;
    uint32_t layer, n_layers, page_tokens, n_kv_heads, head_dim, n_q_heads, group;   // group = G
    uint32_t rows_lo, rows_hi;   // this launch takes the items with rows_lo < rows * G <= rows_hi
    const void *q;
    void *out;
    uint64_t q_ts, q_hs, o_ts, o_hs;
    float *lse;
    float scale_log2;
    // Shared prefixes. prefix_pass: the items are the groups, results go to pre_o / pre_lse, and
    // skip[] is filled; otherwise, with skip set, sequence i starts behind its skip[i] tokens and
    // merges the prefix pass's result into its own.
    uint32_t prefix_pass, n_group;
    const uint32_t *group_off, *shared_pages;
    uint32_t *skip;
    float *pre_o;                // f32 [n_new][n_q_heads][head_dim]
    float *pre_lse;              // f32 [n_new][n_q_heads], base 2
    uint32_t dp;                 // elements of a part's row
    float *parts;                // two slots per CTA
    float *few_parts;            // (host side: the few-row kernel's, which may run beside the other)
    unsigned int *arrived;       // few rows: one counter per CTA, zero between calls
    struct CutDesc *cuts;        // many rows: the cut tile that starts in a CTA's span
    uint64_t *span_begin;        // many rows: where the spans begin on the line, and its end
    uint32_t *tile_base;         // many rows: row tiles ahead of every item
    void *maps;                  // many rows: two tensor maps per CTA
    uint32_t box_rows;           // tokens of a box, dividing page_tokens
    uint32_t beside;             // the launch before has nothing for this one: wait for it at the end
    uint32_t wide_boxes;         // a box has all elements of a head, not 64
    uint32_t q_boxes;            // the queries come by boxes too
    long long wait_cycles;
    uint64_t test_drop;          // test hook: ~0 = off
    DevStatus *st;
    uint32_t pair_bytes;         // of an element of a key and its value: 4, or 2 in an 8-bit pool
    uint32_t q_gathered;         // 8-bit pools, many rows: the queries are f16 rows [kv_head][token, head of the group]
    const float *q_back;         // their rows' factors (null: 1)
};

// An item: a sequence, or in the prefix pass a group.
struct Item {
    uint64_t row0, page0;
    uint32_t tokens;             // new tokens
    uint32_t kv0, kv1;           // keys [kv0, kv1)
    bool causal;
    bool ok;
    uint32_t skip;               // own pass: tokens whose result the prefix pass has
};

__device__ __forceinline__ uint32_t shared_tokens(const AttendJob &j, uint32_t g)
{
    const uint32_t a = j.group_off[g], b = j.group_off[g + 1];
    if (a >= b || b > j.seqs.n_seq || b - a < 2) return 0;
    const uint64_t p0 = j.seqs.page_off[a], p1 = j.seqs.page_off[a + 1];
    const uint64_t want = j.shared_pages[g];
    if (p1 < p0 || want > p1 - p0 || want * j.page_tokens >= 0x80000000ull) return 0;
    return (uint32_t)(want * j.page_tokens);
}

__device__ __forceinline__ Item load_item(const AttendJob &j, uint32_t i)
{
    Item it;
    if (j.prefix_pass) {
        const uint32_t a = j.group_off[i], b = j.group_off[i + 1];
        it.kv0 = 0;
        it.kv1 = shared_tokens(j, i);
        it.causal = false;
        it.skip = 0;
        it.ok = true;
        it.tokens = 0;
        it.row0 = it.page0 = 0;
        if (it.kv1) {
            const uint64_t r0 = j.seqs.new_off[a], r1 = j.seqs.new_off[b];
            it.ok = r0 <= r1 && r1 <= j.seqs.n_new;
            it.row0 = r0;
            it.tokens = it.ok ? (uint32_t)(r1 - r0) : 0u;
            it.page0 = j.seqs.page_off[a];
        }
        return it;
    }
    const SeqInfo s = load_seq(j.seqs, i, j.page_tokens);
    it.row0 = s.row0;
    it.page0 = s.page0;
    it.tokens = s.rows;
    it.ok = s.ok;
    it.kv0 = 0;
    it.kv1 = s.kv;
    it.causal = true;
    it.skip = 0;
    if (j.skip) {
        // a member with a new token inside the shared part goes by itself
        const uint32_t k = j.skip[i];
        if (s.ok && s.kv >= s.rows && k <= s.kv - s.rows) it.skip = it.kv0 = k;
    }
    return it;
}

// Keys that token t of an item sees: [kv0, limit).
__device__ __forceinline__ uint32_t token_limit(const Item &it, uint32_t t)
{
    if (!it.causal) return it.kv1;
    const int64_t p = (int64_t)it.kv1 - (int64_t)it.tokens + (int64_t)t + 1;
    return p > (int64_t)it.kv0 ? (uint32_t)p : it.kv0;
}

// Key tiles of `tile` keys for row tile rt (M rows): at least one, so that rows without keys are
// written too.
__device__ __forceinline__ uint32_t tile_units(const Item &it, uint32_t rt, uint32_t M, uint32_t G,
                                               uint32_t tile)
{
    uint32_t t = (rt * M + M - 1) / G;
    if (t >= it.tokens) t = it.tokens - 1;
    const uint32_t n = (token_limit(it, t) - it.kv0 + tile - 1) / tile;
    return n ? n : 1u;
}

__device__ __forceinline__ uint32_t item_tiles(const AttendJob &j, const Item &it, uint32_t M)
{
    const uint64_t rows = (uint64_t)it.tokens * j.group;
    if (rows <= j.rows_lo || rows > j.rows_hi) return 0;
    return (uint32_t)((rows + M - 1) / M);
}

// A tile's length on the line: its units and one more, about what its beginning and end cost (its
// queries, the merge of the warps, the result: 5k cycles, where a unit of the few-row kernel takes
// 2.9k). No work lies in that last unit.
constexpr uint32_t kTileCost = 1;

// Units of one KV head of an item.
__device__ __forceinline__ uint64_t item_units(const AttendJob &j, const Item &it, uint32_t M,
                                               uint32_t tile)
{
    const uint32_t n = item_tiles(j, it, M);
    if (!n) return 0;
    if (!it.causal) return (uint64_t)n * (tile_units(it, 0, M, j.group, tile) + kTileCost);
    uint64_t u = 0;
    for (uint32_t rt = 0; rt < n; ++rt) u += tile_units(it, rt, M, j.group, tile) + kTileCost;
    return u;
}

// A CTA's place on the line of units.
struct Span {
    uint64_t begin, end, per;    // units [begin, end); units per CTA (equal spans)
    uint32_t item;               // the item that holds `begin`
    uint64_t before;             // units ahead of that item
    uint32_t waves;              // whole row tiles that the CTA takes first
    uint32_t rank;               // number of its span among those that are not empty
    uint32_t heads, tile;        // of the line: KV heads, or groups of them, and keys of a unit
};

// A call's launches follow each other closely: each lets the next one start while it still runs
// and itself waits, first of all, for what the one before has written.
__device__ __forceinline__ void wait_launch() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

__device__ __forceinline__ void follow_launch()
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    wait_launch();
}

// 64-bit division takes hundreds of cycles; most quotients here are of small numbers.
__device__ __forceinline__ uint64_t quotient(uint64_t a, uint64_t b)
{
    return (a | b) >> 32 ? a / b : (uint32_t)a / (uint32_t)b;
}

// Inclusive sum over a CTA's threads, and the total; scratch: NT / 32 words of shared memory.
template <int NT>
__device__ __forceinline__ uint64_t block_scan(uint64_t mine, uint64_t *scratch, uint64_t *total)
{
    const uint32_t lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    uint64_t incl = mine;
    for (int d = 1; d < 32; d <<= 1) {
        const uint64_t o = __shfl_up_sync(~0u, incl, d);
        if ((int)lane >= d) incl += o;
    }
    __syncthreads();             // an earlier scan's words are read
    if (lane == 31) scratch[w] = incl;
    __syncthreads();
    uint64_t all = 0, ahead = 0;
#pragma unroll
    for (int k = 0; k < NT / 32; ++k) {
        if (k < (int)w) ahead += scratch[k];
        all += scratch[k];
    }
    *total = all;
    return ahead + incl;
}

// Where a CTA's work lies. Called by all threads of a CTA (NT of them, a multiple of 32, at most
// 1024). n items.
// kWaves: where there are more row tiles than CTAs, the CTAs first take whole tiles in turn, wave
// by wave -- tiles of one sequence and head side by side, so that the CTAs read the same keys at
// the same time and L2 has them -- and only the tiles that are left are cut into spans, which even
// out what the waves left uneven. (Two requests of 32768 tokens, 1024 new, 64/8 heads, 0.27 GB of
// keys and values: spans alone read 6.1 GB from memory and take 2.40 ms, with waves 0.35 GB and
// 2.12 ms.) Keys that L2 holds anyway need none, and spans even out better (six prompts of 700 to
// 3000 tokens, 45 MB: 133 us against 147). load: gridDim words of shared memory.
constexpr uint64_t kL2Keeps = 64ull << 20;   // bytes of keys and values, of 126 MB
template <int NT, bool kWaves>
__device__ Span find_span(const AttendJob &j, uint32_t n, uint32_t heads, uint32_t M, uint32_t tile, uint32_t *load)
{
    __shared__ uint64_t scan[NT / 32];
    __shared__ uint64_t found_before, mine_begin, mine_end;
    __shared__ unsigned long long all_bytes;
    __shared__ uint32_t found_item, mine_rank, all_tiles;
    const uint32_t tid = threadIdx.x, N = gridDim.x;
    const uint32_t each = (n + NT - 1) / NT;
    const uint32_t i0 = tid * each < n ? tid * each : n;
    const uint32_t i1 = i0 + each < n ? i0 + each : n;
    uint64_t mine = 0, first = 0;
    uint32_t tiles = 0;
    uint64_t bytes = 0;
    for (uint32_t i = i0; i < i1; ++i) {
        const Item it = load_item(j, i);
        const uint64_t u = item_units(j, it, M, tile) * heads;
        // (a group left out for its offsets holds a sequence that the own pass reports)
        if (!it.ok && !j.prefix_pass && blockIdx.x == 0) st_flag(j.st, LSMKV_ST_BAD_COUNT, i);
        if (i == i0) first = u;
        mine += u;
        if (kWaves && item_tiles(j, it, M)) {
            tiles += item_tiles(j, it, M) * heads;
            bytes += (uint64_t)(it.kv1 - it.kv0) * heads * j.head_dim * j.pair_bytes;
        }
    }
    const bool may_wave = kWaves && !j.prefix_pass;
    if (may_wave) {
        if (tid == 0) {
            all_bytes = 0;
            all_tiles = 0;
        }
        __syncthreads();
        if (tiles) {
            atomicAdd(&all_bytes, (unsigned long long)bytes);
            atomicAdd(&all_tiles, tiles);
        }
    }
    uint64_t total;
    const uint64_t incl = block_scan<NT>(mine, scan, &total);
    Span s;
    s.per = quotient(total + N - 1, N);
    s.begin = s.per * blockIdx.x;
    s.end = s.begin + s.per;
    if (s.end > total) s.end = total;
    if (s.begin > total) s.begin = total;
    s.waves = 0;
    s.rank = blockIdx.x;
    s.heads = heads;
    s.tile = tile;
    uint32_t waves = may_wave && all_bytes > kL2Keeps ? all_tiles / N : 0;
    if (kWaves && !waves) {
        // equal spans; every CTA writes all of span_begin, the same values, and reads its own
        for (uint32_t c = tid; c <= N; c += NT) j.span_begin[c] = c * s.per < total ? c * s.per : total;
    }
    if (waves) {
        uint64_t ignored;
        uint32_t base = (uint32_t)(block_scan<NT>(tiles, scan, &ignored) - tiles);
        // (tile_base likewise)
        for (uint32_t i = i0; i < i1; ++i) {
            j.tile_base[i] = base;
            base += item_tiles(j, load_item(j, i), M) * heads;
        }
        if (i1 == n && i0 < i1) j.tile_base[n] = base;
        uint64_t capacity = s.per;                       // of CTA tid, behind its waves
        const uint32_t team = n < NT ? NT / n : 1;       // threads that go through an item's tiles
        while (waves) {
            for (uint32_t c = tid; c < N; c += NT) load[c] = 0;
            __syncthreads();
            for (uint32_t i = tid / team; i < n; i += NT / team) {
                const Item it = load_item(j, i);
                const uint32_t nt = item_tiles(j, it, M), p0 = j.tile_base[i];
                for (uint32_t q = tid % team; q < nt * heads && p0 + q < waves * N; q += team)
                    atomicAdd(&load[(p0 + q) % N], tile_units(it, q % nt, M, j.group, tile) + kTileCost);
            }
            __syncthreads();
            // no CTA may have more than its share already
            if (!__syncthreads_or(tid < N && load[tid] > s.per)) break;
            waves /= 2;
        }
        if (waves) capacity = tid < N ? s.per - load[tid] : 0;
        if (tid >= N) capacity = 0;
        uint64_t sum;
        const uint64_t taken = waves && tid < N ? load[tid] : 0;
        block_scan<NT>(taken, scan, &sum);               // units of the waves: the line goes on there
        const uint64_t upto = sum + block_scan<NT>(capacity, scan, &ignored);
        const uint64_t b = upto - capacity < total ? upto - capacity : total, e = upto < total ? upto : total;
        const uint32_t rank = (uint32_t)block_scan<NT>(b < e, scan, &ignored) - (b < e);
        if (b < e) j.span_begin[rank] = b;
        if (tid == 0) j.span_begin[ignored] = total;
        if (tid == blockIdx.x) {
            mine_begin = b;
            mine_end = e;
            mine_rank = rank;
        }
        __syncthreads();
        s.begin = mine_begin;
        s.end = mine_end;
        s.rank = mine_rank;
        s.waves = waves;
    }
    uint64_t at = incl - mine;
    if (j.prefix_pass) {
        // for the own pass: a CTA fills in every gridDim-th group's members
        for (uint32_t g = blockIdx.x + tid * N; g < n; g += N * NT) {
            const uint32_t a = j.group_off[g], b = j.group_off[g + 1];
            if (a > b || b > j.seqs.n_seq) {
                st_flag(j.st, LSMKV_ST_BAD_COUNT, g);
                continue;
            }
            const Item it = load_item(j, g);
            const uint32_t k = item_tiles(j, it, M) ? it.kv1 : 0;
            for (uint32_t i = a; i < b; ++i) j.skip[i] = k;
        }
        if (tid == 0 && blockIdx.x == 0 &&
            (j.group_off[0] != 0 || j.group_off[j.n_group] != j.seqs.n_seq))
            st_flag(j.st, LSMKV_ST_BAD_COUNT, j.n_group);
    }
    if (s.begin < s.end && at <= s.begin && s.begin < at + mine) {
        uint32_t i = i0;
        if (each > 1 && at + first <= s.begin) {
            at += first;
            for (i = i0 + 1; i < i1; ++i) {
                const uint64_t u = item_units(j, load_item(j, i), M, tile) * heads;
                if (at + u > s.begin) break;
                at += u;
            }
        }
        found_item = i;
        found_before = at;
    }
    __syncthreads();
    s.item = found_item;
    s.before = found_before;
    return s;
}

// The first item behind i that has units (there is one when the span is not done), looked for by
// the lanes of every warp together: a launch may pass over many items that are not its own.
__device__ __forceinline__ uint32_t next_item(const AttendJob &j, uint32_t i, uint32_t n, uint32_t M, Item *it)
{
    const uint32_t lane = threadIdx.x & 31;
    for (uint32_t base = i + 1; base < n; base += 32) {
        const unsigned some =
            __ballot_sync(~0u, base + lane < n && item_tiles(j, load_item(j, base + lane), M) != 0);
        if (some) {
            const uint32_t k = base + __ffs(some) - 1;
            *it = load_item(j, k);
            return k;
        }
    }
    return i;
}

// One row tile of the line and the piece of it that lies in a CTA's span.
struct Cut {
    uint32_t kv_head, rt, rows;  // rows of the tile
    uint64_t tile0;              // units ahead of the tile
    uint32_t units;              // of the whole tile
    uint32_t k0, k1;             // key tiles [k0, k1) of it are this CTA's
};

// Walks a CTA's whole tiles and the cuts of its span. All threads of a warp go through it together. TILE keys a
// unit, 0: the span says how many, and of how many heads.
template <int M, int TILE>
struct Walk {
    static __device__ __forceinline__ uint32_t tile_keys(const Span &s) { return TILE ? TILE : s.tile; }
    uint64_t u;                  // next unit
    uint32_t i, tiles;           // item, its row tiles
    uint32_t wave;               // whole tiles taken so far
    Item it;
    Cut p;
    bool begun;

    __device__ __forceinline__ void start(const AttendJob &j, const Span &s)
    {
        wave = 0;
        i = 0xFFFFFFFFu;
        u = s.begin;
        begun = false;
        if (!s.waves) start_span(j, s);
    }
    __device__ __forceinline__ void start_span(const AttendJob &j, const Span &s)
    {
        if (s.begin >= s.end) return;
        i = s.item;
        it = load_item(j, i);
        tiles = item_tiles(j, it, M);
        // the tile that holds unit s.begin
        const uint64_t per_head = item_units(j, it, M, tile_keys(s));
        const uint64_t rel = u - s.before;
        p.kv_head = (uint32_t)quotient(rel, per_head);
        uint64_t at = rel - (uint64_t)p.kv_head * per_head;
        p.tile0 = s.before + (uint64_t)p.kv_head * per_head;
        p.rt = 0;
        while (true) {
            p.units = tile_units(it, p.rt, M, j.group, tile_keys(s));
            if (at < p.units + kTileCost || p.rt + 1 >= tiles) break;
            at -= p.units + kTileCost;
            p.tile0 += p.units + kTileCost;
            ++p.rt;
        }
    }
    __device__ __forceinline__ void count_rows(const AttendJob &j)
    {
        const uint64_t rows = (uint64_t)it.tokens * j.group - (uint64_t)p.rt * M;
        p.rows = rows < M ? (uint32_t)rows : M;
    }
    // whole tile number `at` of the batch
    __device__ __forceinline__ void take_tile(const AttendJob &j, const Span &s, uint32_t at)
    {
        uint32_t lo = 0, hi = j.seqs.n_seq;      // tile_base[lo] <= at < tile_base[hi]
        while (hi - lo > 1) {
            const uint32_t mid = (lo + hi) / 2;
            if (j.tile_base[mid] <= at) lo = mid;
            else hi = mid;
        }
        if (lo != i) {
            i = lo;
            it = load_item(j, i);
            tiles = item_tiles(j, it, M);
        }
        const uint32_t rel = at - j.tile_base[i];
        p.kv_head = rel / tiles;
        p.rt = rel - p.kv_head * tiles;
        p.tile0 = 0;
        p.units = tile_units(it, p.rt, M, j.group, tile_keys(s));
        p.k0 = 0;
        p.k1 = p.units;
        count_rows(j);
    }
    __device__ __forceinline__ bool next(const AttendJob &j, const Span &s)
    {
        if (wave < s.waves) {
            take_tile(j, s, wave++ * gridDim.x + blockIdx.x);
            return true;
        }
        if (s.waves && wave == s.waves) {
            ++wave;
            start_span(j, s);
        }
        while (u < s.end) {
            if (begun) {
                p.tile0 = u;
                if (++p.rt == tiles) {
                    p.rt = 0;
                    if (++p.kv_head == (TILE ? j.n_kv_heads : s.heads)) {
                        p.kv_head = 0;
                        i = next_item(j, i, j.prefix_pass ? j.n_group : j.seqs.n_seq, M, &it);
                        tiles = item_tiles(j, it, M);
                    }
                }
                p.units = tile_units(it, p.rt, M, j.group, tile_keys(s));
            }
            begun = true;
            p.k0 = (uint32_t)(u - p.tile0);
            const uint64_t end = p.tile0 + p.units;
            u = end + kTileCost < s.end ? end + kTileCost : s.end;
            if (p.k0 >= p.units) continue;      // the span begins behind the tile's last unit
            p.k1 = (uint32_t)((end < s.end ? end : s.end) - p.tile0);
            count_rows(j);
            return true;
        }
        return false;
    }
};

// ---- partial results: per slot, M rows of sums, then M maxima and M sums of weights ----------

__device__ __forceinline__ float *part_slot(const AttendJob &j, uint64_t slot, uint32_t M, uint32_t DP)
{
    return j.parts + slot * ((uint64_t)M * (DP + 2));
}

// A part is empty when its sum of weights is zero (m is -inf then, the sums are not looked at). An undefined
// score never becomes the maximum, so a part of undefined scores alone has m = -inf too, but l and the
// sums are NaN: it counts, and NaN times a weight of zero keeps the row undefined.
// 2^(m - top), 0 for m = -inf
__device__ __forceinline__ float part_weight(float m, float top)
{
    return m == -INFINITY ? 0.f : exp2f(m - top);
}

struct Quad {
    float4 acc;
    float m, l;
};

__device__ __forceinline__ void add_quad(Quad &a, const float4 &o, float m, float l)
{
    const float top = fmaxf(a.m, m);
    const float f = part_weight(a.m, top), g = part_weight(m, top);
    a.acc.x = a.acc.x * f + o.x * g;
    a.acc.y = a.acc.y * f + o.y * g;
    a.acc.z = a.acc.z * f + o.z * g;
    a.acc.w = a.acc.w * f + o.w * g;
    a.l = a.l * f + l * g;
    a.m = top;
}

// Parts c0..c1 of a cut tile, four elements of row r, merged in order; four parts in flight. (Out
// of line, like what else ends a row: the loops that come before want the registers.)
__device__ __noinline__ Quad sum_parts(const float *parts, uint32_t c0, uint32_t c1, uint32_t M, uint32_t DP,
                                       uint32_t r, uint32_t d)
{
    constexpr int U = 4;
    Quad sum;
    sum.acc = make_float4(0.f, 0.f, 0.f, 0.f);
    sum.m = -INFINITY;
    sum.l = 0.f;
    for (uint32_t c = c0; c <= c1; c += U) {
        float pm[U], pl[U];
        float4 o[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            pl[u] = 0.f;
            if (c + u > c1) continue;
            const float *s = parts + (2ull * (c + u) + (c + u == c0 ? 1 : 0)) * ((uint64_t)M * (DP + 2));
            pm[u] = __ldcg(s + (uint64_t)M * DP + r);
            pl[u] = __ldcg(s + (uint64_t)M * (DP + 1) + r);
            o[u] = __ldcg(reinterpret_cast<const float4 *>(s + (uint64_t)r * DP + d));
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (pl[u] != 0.f) add_quad(sum, o[u], pm[u], pl[u]);   // else no key of it was the row's
    }
    return sum;
}

// A row tile's products also run over keys that only later rows of it see, with weight zero: an
// infinite or undefined value there would make the sum undefined although the row must not see it.
// Whether there is one among eight elements: a running sum of zero times each, which stays zero or does not.
template <typename T>
__device__ __forceinline__ void add_undefined(const uint4 &v, uint32_t &sum)
{
    using Pair = typename std::conditional<std::is_same<T, __half>::value, __half2, __nv_bfloat162>::type;
    const uint32_t zero = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t x = (&v.x)[i];
        const Pair r = __hfma2(*reinterpret_cast<const Pair *>(&x), *reinterpret_cast<const Pair *>(&zero),
                               *reinterpret_cast<const Pair *>(&sum));
        sum = *reinterpret_cast<const uint32_t *>(&r);
    }
}

__device__ __forceinline__ bool was_undefined(uint32_t sum) { return (sum & 0x7FFF7FFFu) != 0; }

// Write four elements of finished row R of the item: acc = sum of weighted values relative to
// 2^m, l the sum of weights. Merges the prefix pass's result first when there is one.
template <typename T>
__device__ __forceinline__ void finish_row4(const AttendJob &j, const Item &it, uint32_t kv_head, uint32_t R,
                                            uint32_t d, float4 acc, float m, float l)
{
    const uint64_t row = it.row0 + R / j.group;
    const uint32_t sub = R % j.group, head = kv_head * j.group + sub;
    const uint64_t flat = row * j.n_q_heads + head;
    if (it.skip) {
        Quad sum;
        sum.acc = acc;
        sum.m = m;
        sum.l = l;
        const float pm = j.pre_lse[flat];
        add_quad(sum, *reinterpret_cast<const float4 *>(j.pre_o + flat * j.head_dim + d), pm,
                 pm == -INFINITY ? 0.f : 1.f);
        acc = sum.acc;
        m = sum.m;
        l = sum.l;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    acc.x *= inv; acc.y *= inv; acc.z *= inv; acc.w *= inv;
    if (l == 0.f) acc = make_float4(0.f, 0.f, 0.f, 0.f);
    const float lse2 = l == 0.f ? -INFINITY : m + log2f(l);
    if (j.prefix_pass) {
        *reinterpret_cast<float4 *>(j.pre_o + flat * j.head_dim + d) = acc;
        if (d == 0) j.pre_lse[flat] = lse2;
        return;
    }
    uint2 v;
    v.x = Half2<T>::down(acc.x, acc.y);
    v.y = Half2<T>::down(acc.z, acc.w);
    *reinterpret_cast<uint2 *>(static_cast<T *>(j.out) + row * j.o_ts + head * j.o_hs + d) = v;
    if (d == 0 && j.lse) j.lse[flat] = lse2 * kLn2;
}

// The same out of line, where the call site is unrolled.
template <typename T>
__device__ __noinline__ void finish_row4_call(const AttendJob &j, const Item &it, uint32_t kv_head, uint32_t R,
                                              uint32_t d, float4 acc, float m, float l)
{
    finish_row4<T>(j, it, kv_head, R, d, acc, m, l);
}

// Merge rows [r0, r1) of a cut tile with parts c0..c1, by NT threads.
template <typename T, int NT>
__device__ __forceinline__ void merge_parts(const AttendJob &j, const Item &it, const Cut &p, uint32_t c0,
                                            uint32_t c1, uint32_t M, uint32_t r0, uint32_t r1)
{
    const uint32_t quads = j.head_dim / 4;
    for (uint32_t x = threadIdx.x; x < (r1 - r0) * quads; x += NT) {
        const uint32_t r = r0 + x / quads, d = x % quads * 4;
        const Quad q = sum_parts(j.parts, c0, c1, M, j.dp, r, d);
        finish_row4<T>(j, it, p.kv_head, p.rt * M + r, d, q.acc, q.m, q.l);
    }
}

// The CTA has written its part of a cut tile: true for all its threads when it is the last one.
__device__ __forceinline__ bool deliver_part(const AttendJob &j, uint32_t c0, uint32_t c1)
{
    __shared__ uint32_t last;
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) {
        last = atomicAdd(&j.arrived[c0], 1u) == c1 - c0;
        if (last) j.arrived[c0] = 0;      // ready for the next call
    }
    __syncthreads();
    if (last) __threadfence();
    return last;
}

// ---- few rows ---------------------------------------------------------------------------------
//
// Bound by memory: a decode step reads every key and value once and does 4 G operations a byte.
// A row tile is NB blocks of 8 rows. The products are taken the other way round, S^T = K Q^T and
// O^T = V^T P^T, with the keys (or the elements) as the 16 rows of an m16n8k16 fragment and 8
// queries as its columns: with 16 query rows, of which a decode step has G, the products cost twice
// as much, and the legacy matrix path is slow enough here for that to show beside the memory.
// P^T goes from accumulator to operand layout by movmatrix.
// A warp takes 16 keys at a time in a private ring of ST stages fed by cp.async (no barrier in the
// loop: the warps of a CTA share nothing until the cut's end), and the NW warps of a CTA take the
// key tiles in turn. One CTA a SM, and the ring runs ahead over the cuts' ends: the next cut's
// keys travel while this one's warps merge, which is what short sequences need. Measured: 256 requests
// of 1k to 8k tokens, 32/8 heads of 128, 4.76 GB: 727 us, 6.55 TB/s; 512 of 256 to 4096 tokens, 28/4
// heads, 2.29 GB: 367 us, 6.2 TB/s (435 with the ring ending with each cut's keys and 16 query rows).

__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src, bool real)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"
                 :: "r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}

__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(dst), "l"(src) : "memory");
}

__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}

__device__ __forceinline__ void ldmatrix4t(uint32_t addr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}

template <typename T> __device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4],
                                                               uint32_t b0, uint32_t b1);
template <> __device__ __forceinline__ void mma16816<__nv_bfloat16>(float (&c)[4], const uint32_t (&a)[4],
                                                                    uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
                 "{%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <> __device__ __forceinline__ void mma16816<__half>(float (&c)[4], const uint32_t (&a)[4],
                                                             uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
                 "{%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t transpose8x8(uint32_t v)
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}

template <int DP, int NB>
struct FewShape {
    static constexpr int kM = 8 * NB;                      // rows of a tile
    static constexpr int kKeys = 16;                       // keys a warp takes at a time
    static constexpr int kWarps = DP <= 128 ? 8 : 4;
    static constexpr int kStages = DP <= 64 ? 6 : 3;       // 192 KB of keys and values a SM
    static constexpr int kThreads = kWarps * 32;
    static constexpr uint32_t kStage = kKeys * DP * 2 * 2; // K then V
    static constexpr size_t kQBytes = kM * DP * 2;
    // rows merged at a time: all of them where they fit beside the ring
    static constexpr uint32_t kMergeRows = (NB == 1 && DP <= 128 ? 32768 : 24576) / (kWarps * DP * 4);
    static constexpr size_t kMergeBytes = (size_t)kMergeRows * kWarps * DP * 4;
    static constexpr size_t kSmem = kQBytes + kMergeBytes + (size_t)kWarps * kStages * kStage;
    // operand fragments of the queries stay in registers while there are few
    static constexpr bool kQInRegs = DP * NB <= 256;
};

template <typename T, int DP, int NB>
__global__ __launch_bounds__(FewShape<DP, NB>::kThreads, 1) void k_attend_few(const __grid_constant__ AttendJob j)
{
    using Sh = FewShape<DP, NB>;
    constexpr int NT = Sh::kThreads, NW = Sh::kWarps, ST = Sh::kStages;
    constexpr int kChunks = DP / 8;            // 16-byte pieces of a row
    constexpr uint32_t kTile = Sh::kKeys * NW, kNone = 0xFFFFFFFFu;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ float sm_m[NW][Sh::kM], sm_l[NW][Sh::kM];
    const uint32_t tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    const uint32_t G = j.group, D = j.head_dim;

    follow_launch();
    const T *const kbuf = static_cast<const T *>(j.kv_ptrs[j.layer]);
    const T *const vbuf = static_cast<const T *>(j.kv_ptrs[j.n_layers + j.layer]);
    const uint32_t n_items = j.prefix_pass ? j.n_group : j.seqs.n_seq;
    const Span span = find_span<NT, false>(j, n_items, j.n_kv_heads, Sh::kM, kTile, nullptr);
    if ((reinterpret_cast<uintptr_t>(kbuf) | reinterpret_cast<uintptr_t>(vbuf)) & 15u) {
        if (blockIdx.x == 0 && tid == 0) st_flag(j.st, LSMKV_ST_MISALIGNED, 0);
        return;
    }
    if (span.begin >= span.end) return;

    const uint32_t q_s = smem_addr(smem);
    float *const merge = reinterpret_cast<float *>(smem + Sh::kQBytes);
    const uint32_t ring = q_s + (uint32_t)(Sh::kQBytes + Sh::kMergeBytes) + w * (ST * Sh::kStage);
    const uint64_t tok_stride = (uint64_t)j.n_kv_heads * D;
    using CutWalk = Walk<Sh::kM, (int)kTile>;

    CutWalk walk;
    walk.start(j, span);
    bool more = walk.next(j, span);
    const Item &it = walk.it;
    const Cut &p = walk.p;
    // The load side, ahead of the other: its cut, and this warp's next 16-key tile. Where such a
    // tile lies in one page, a lane holds the page id of one of the next 32 tiles; else, of key
    // lane % 16 of the next tile.
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
        load_key = on.kv0 + ahead.p.k0 * kTile + w * Sh::kKeys;
        load_end = min(token_limit(on, (ahead.p.rt * Sh::kM + ahead.p.rows - 1) / G), on.kv0 + ahead.p.k1 * kTile);
    };
    auto next_load_cut = [&]() {
        while (load_key >= load_end && ahead.next(j, span)) take_load_cut();
        load_pages();
    };
    // Piece c = lane % kChunks of rows kRows x + lane / kChunks: whole rows side by side (256 bytes in
    // one request at head_dim 128), swizzled (piece c of row r at c ^ r % 8).
    constexpr int kRows = 32 / kChunks > 0 ? 32 / kChunks : 1;
    constexpr int kCopies = 16 * kChunks / 32;
    const uint32_t piece_r = lane / kChunks, piece_c = lane % kChunks;
    const uint32_t piece_at = (piece_r * kChunks + (piece_c ^ piece_r)) * 16;
    const uint64_t step = kRows * tok_stride;
    auto fetch = [&](uint32_t stage) {
        if (load_key < load_end) {
            const uint32_t k = load_key + (one_page ? 0 : lane & 15);
            const uint32_t page = one_page ? __shfl_sync(~0u, load_page, 32 - tiles_known) : load_page;
            const bool real = page != kNone;
            const uint32_t left = load_end - load_key;
            uint64_t off = real ? ((uint64_t)page * j.page_tokens + k % j.page_tokens) * tok_stride +
                                      (uint64_t)ahead.p.kv_head * D
                                : 0;
            load_key += kTile;
            if (--tiles_known == 0 && load_key < load_end) load_pages();
            const uint32_t dst = ring + stage * Sh::kStage;
            if (one_page) {
                // the rows of the tile lie one behind the other
                off += piece_r * tok_stride + piece_c * 8;
                const bool there = real && piece_c * 8 < D;
                const T *kp = kbuf + off, *vp = vbuf + off;
#pragma unroll
                for (int x = 0; x < kCopies; ++x) {
                    const uint32_t r = x * kRows;            // and piece_r more
                    const bool in = there && r + piece_r < left;
                    const uint32_t to = dst + r * kChunks * 16 + (piece_at ^ ((r & 7) << 4));
                    cp_async16(to, in ? kp : kbuf, in);
                    cp_async16(to + Sh::kKeys * DP * 2, in ? vp : vbuf, in);
                    kp += step;
                    vp += step;
                }
            } else {
                const uint32_t lo = (uint32_t)off, hi = (uint32_t)(off >> 32) | (real ? 0u : 0x80000000u);
#pragma unroll
                for (int x = 0; x < kCopies; ++x) {
                    const uint32_t r = x * kRows + piece_r;
                    const uint32_t h = __shfl_sync(~0u, hi, r);
                    const uint64_t o = ((uint64_t)(h & 0x7FFFFFFFu) << 32) | __shfl_sync(~0u, lo, r);
                    const bool in = !(h >> 31) && piece_c * 8 < D;
                    const uint64_t e = in ? o + piece_c * 8 : 0;
                    const uint32_t to = dst + x * kRows * kChunks * 16 + (piece_at ^ (((x * kRows) & 7) << 4));
                    cp_async16(to, kbuf + e, in);
                    cp_async16(to + Sh::kKeys * DP * 2, vbuf + e, in);
                }
            }
            if (load_key >= load_end) next_load_cut();
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    // a 16-byte piece (or several, at few threads) of the tile's queries a thread; rows beyond
    // the tile are zero
    constexpr int kPieces = (Sh::kM * kChunks + NT - 1) / NT;
    uint4 q_piece[kPieces];
    auto load_queries = [&]() {
#pragma unroll
        for (int y = 0; y < kPieces; ++y) {
            const uint32_t x = tid + y * NT, r = x / kChunks, c = x % kChunks;
            q_piece[y] = make_uint4(0, 0, 0, 0);
            if (r < p.rows && c * 8 < D) {
                const uint32_t R = p.rt * Sh::kM + r;
                q_piece[y] = *reinterpret_cast<const uint4 *>(static_cast<const T *>(j.q) + (it.row0 + R / G) * j.q_ts +
                                                              (uint64_t)(p.kv_head * G + R % G) * j.q_hs + c * 8);
            }
        }
    };
    auto store_queries = [&]() {
#pragma unroll
        for (int y = 0; y < kPieces; ++y) {
            const uint32_t x = tid + y * NT, r = x / kChunks, c = x % kChunks;
            if (r < Sh::kM) *reinterpret_cast<uint4 *>(smem + (r * kChunks + (c ^ (r & 7))) * 16) = q_piece[y];
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
#pragma unroll
        for (int x = 0; x < 2 * NB; ++x) {
            const uint32_t r = (x >> 1) * 8 + 2 * (lane & 3) + (x & 1);
            lim[x >> 1][x & 1] = r < cut.rows ? token_limit(it, (row_base + r) / G) : it.kv0;
        }
        const uint32_t lim_first = token_limit(it, row_base / G);              // least of the tile
        const uint32_t key_end = min(token_limit(it, (row_base + cut.rows - 1) / G), it.kv0 + cut.k1 * kTile);
        const uint32_t key0 = it.kv0 + cut.k0 * kTile + w * Sh::kKeys;

        // queries as the right operand: 16 elements x 8 rows a fragment, two fragments a load
        uint32_t qf[Sh::kQInRegs ? DP / 16 : 1][NB][2];
        auto load_q = [&](int x, uint32_t (&f)[2][NB][2]) {       // elements 32 x ..
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const uint32_t r = nb * 8 + (lane & 7), ck = 4 * x + (lane >> 3);
                uint32_t q[4];
                ldmatrix4(q_s + (r * kChunks + (ck ^ (r & 7))) * 16, q);
                f[0][nb][0] = q[0];
                f[0][nb][1] = q[1];
                f[1][nb][0] = q[2];
                f[1][nb][1] = q[3];
            }
        };
        if constexpr (Sh::kQInRegs) {
#pragma unroll
            for (int x = 0; x < DP / 32; ++x) load_q(x, *reinterpret_cast<uint32_t(*)[2][NB][2]>(&qf[2 * x]));
        }

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
            const uint32_t ks = ring + stage * Sh::kStage;
            const uint32_t vs = ks + Sh::kKeys * DP * 2;

            // scores of 16 keys (lane/4 and lane/4 + 8) x 8 rows
            float s[NB][4];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) s[nb][0] = s[nb][1] = s[nb][2] = s[nb][3] = 0.f;
            {
                const uint32_t kr = lane & 15;
                uint32_t f[2][NB][2];
#pragma unroll
                for (int x = 0; x < DP / 16; ++x) {
                    uint32_t a[4];
                    ldmatrix4(ks + (kr * kChunks + ((2 * x + (lane >> 4)) ^ (kr & 7))) * 16, a);
                    if constexpr (!Sh::kQInRegs) {
                        if (x % 2 == 0) load_q(x / 2, f);
                    }
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) {
                        if constexpr (Sh::kQInRegs) mma16816<T>(s[nb], a, qf[x][nb][0], qf[x][nb][1]);
                        else mma16816<T>(s[nb], a, f[x & 1][nb][0], f[x & 1][nb][1]);
                    }
                }
            }
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[nb][e] *= j.scale_log2;
            if (key + Sh::kKeys > lim_first) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (key + (lane >> 2) + 8 * (e >> 1) >= lim[nb][e & 1]) s[nb][e] = -INFINITY;
            }
            // The maximum that the weights refer to is the row's over all lanes. It moves only when
            // a score passes it by more than 2^8: most tiles need one vote, no exchange.
            bool over = false;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int x = 0; x < 2; ++x) over |= fmaxf(s[nb][x], s[nb][2 + x]) > m[nb][x] + 8.f;
            if (__any_sync(~0u, over)) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    float fix[2];
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        float t = fmaxf(s[nb][x], s[nb][2 + x]);
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
            uint32_t pf[NB][2];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float base = m[nb][e & 1] == -INFINITY ? 0.f : m[nb][e & 1];
                    s[nb][e] = exp2f(s[nb][e] - base);
                    l[nb][e & 1] += s[nb][e];
                }
                // the weights are rounded to the values' type: the tensor cores take both in one
                pf[nb][0] = transpose8x8(Half2<T>::down(s[nb][0], s[nb][1]));
                pf[nb][1] = transpose8x8(Half2<T>::down(s[nb][2], s[nb][3]));
            }
            const uint32_t vr = (lane & 7) + ((lane >> 4) << 3);
            auto value_fragment = [&](int x, uint32_t (&a)[4]) {
                ldmatrix4t(vs + (vr * kChunks + ((2 * x + ((lane >> 3) & 1)) ^ (vr & 7))) * 16, a);
            };
            // A tile with keys that some rows see and others do not, and an undefined value among them
            // (16 keys at the end of a sequence with several new tokens, at most two warps' tiles)
            bool apart = false;
            if (it.tokens > 1 && key + Sh::kKeys > lim_first && it.causal) {
                uint32_t sum = 0;
#pragma unroll
                for (uint32_t x = 0; x < Sh::kKeys * kChunks; x += 32)
                    add_undefined<T>(*reinterpret_cast<const uint4 *>(smem + (vs - q_s) + (x + lane) * 16), sum);
                apart = __any_sync(~0u, was_undefined(sum));
            }
            if (!apart) {
#pragma unroll
                for (int x = 0; x < DP / 16; ++x) {
                    uint32_t a[4];
                    value_fragment(x, a);
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) mma16816<T>(o[x][nb], a, pf[nb][0], pf[nb][1]);
                }
            } else {
                // token by token, over the keys that it sees
                const uint32_t t1 = (row_base + cut.rows - 1) / G;
                for (uint32_t t = row_base / G; t <= t1; ++t) {
                    const uint32_t lim_t = token_limit(it, t), see = lim_t > key ? lim_t - key : 0;
                    uint32_t mask[2];                // of this lane's keys 2 (lane % 4), + 1, + 8, + 9
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t k = 8 * h + 2 * (lane & 3);
                        mask[h] = (k < see ? 0xFFFFu : 0u) | (k + 1 < see ? 0xFFFF0000u : 0u);
                    }
#pragma unroll
                    for (int x = 0; x < DP / 16; ++x) {
                        uint32_t a[4];
                        value_fragment(x, a);
#pragma unroll
                        for (int e = 0; e < 4; ++e) a[e] &= mask[e >> 1];
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb) {
                            float part[4] = {0.f, 0.f, 0.f, 0.f};
                            mma16816<T>(part, a, pf[nb][0], pf[nb][1]);
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (lim[nb][e & 1] == lim_t) o[x][nb][e] += part[e];
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
        const uint32_t quads = D / 4;
        float *slot = whole ? nullptr
                            : part_slot(j, 2ull * blockIdx.x + (cut.k0 == 0 ? 1 : 0), Sh::kM, DP);
        for (uint32_t r0 = 0; r0 < cut.rows; r0 += Sh::kMergeRows) {
            const uint32_t r1 = min(r0 + Sh::kMergeRows, cut.rows);
#pragma unroll
            for (int x = 0; x < 2 * NB; ++x) {
                const uint32_t r = (x >> 1) * 8 + 2 * (lane & 3) + (x & 1);
                if (r >= r0 && r < r1) {
                    float *const mine = merge + ((r - r0) * NW + w) * DP;
#pragma unroll
                    for (int n = 0; n < DP / 16; ++n) {
                        mine[(n * 16 + (lane >> 2)) ^ ((r & 6) << 2)] = o[n][x >> 1][x & 1];
                        mine[(n * 16 + 8 + (lane >> 2)) ^ ((r & 6) << 2)] = o[n][x >> 1][2 + (x & 1)];
                    }
                }
            }
            __syncthreads();
            if (r0 == 0 && more) store_queries();      // all warps are done with this cut's
            for (uint32_t x = tid; x < (r1 - r0) * quads; x += NT) {
                const uint32_t r = r0 + x / quads, d = x % quads * 4;
                float top = -INFINITY, sum = 0.f;
#pragma unroll
                for (int k = 0; k < NW; ++k) top = fmaxf(top, sm_m[k][r]);
                float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int k = 0; k < NW; ++k) {
                    const float f = part_weight(sm_m[k][r], top);
                    const float4 v = *reinterpret_cast<const float4 *>(
                        merge + ((r - r0) * NW + k) * DP + (d ^ ((r & 6) << 2)));
                    acc.x += f * v.x;
                    acc.y += f * v.y;
                    acc.z += f * v.z;
                    acc.w += f * v.w;
                    sum += f * sm_l[k][r];
                }
                if (whole) {
                    finish_row4<T>(j, done, cut.kv_head, row_base + r, d, acc, top, sum);
                } else {
                    __stcg(reinterpret_cast<float4 *>(slot + (uint64_t)r * DP + d), acc);
                    if (d == 0) {
                        __stcg(slot + (uint64_t)Sh::kM * DP + r, top);
                        __stcg(slot + (uint64_t)Sh::kM * (DP + 1) + r, sum);
                    }
                }
            }
            __syncthreads();
        }
        if (!whole) {
            const uint32_t c0 = (uint32_t)quotient(cut.tile0, span.per),
                           c1 = (uint32_t)quotient(cut.tile0 + cut.units - 1, span.per);
            if (deliver_part(j, c0, c1)) merge_parts<T, NT>(j, done, cut, c0, c1, Sh::kM, 0, cut.rows);
        }
    }
}

// Rows of a strided tensor to contiguous ones, 16 bytes at a time.
__global__ void k_gather_rows(const uint4 *src, uint64_t token_stride, uint64_t head_stride, uint64_t n_new,
                              uint32_t heads, uint32_t pieces, uint4 *dst)
{
    const uint64_t all = n_new * heads * pieces;
    for (uint64_t x = (uint64_t)blockIdx.x * blockDim.x + threadIdx.x; x < all; x += (uint64_t)gridDim.x * blockDim.x) {
        const uint64_t row = x / pieces, t = row / heads;
        dst[x] = src[t * token_stride + (row - t * heads) * head_stride + (x - row * pieces)];
    }
}

}  // namespace lsmkv
