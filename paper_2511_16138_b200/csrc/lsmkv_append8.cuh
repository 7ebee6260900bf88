// Append to a pool of 8-bit floats: the new tokens' keys (after norm and rotation) and values are
// rounded to e4m3 codes with a power-of-two scale for each block of B tokens and head; the queries get
// norm and rotation beside them, as in the 16-bit append.
//
//   e = least exponent with max |x| <= 448 * 2^e over the finite elements of the block's new tokens
//   e = max(e, the block's) where the block holds earlier tokens, whose codes follow: c <- rn(c * 2^(e_old - e))
//   c = rn_e4m3(x * 2^-e); infinities and NaN become NaN codes and do not count for e
//
// Why powers of two: a code keeps its relative precision whatever the scale, so nothing is lost against
// a scale of full precision, and a block whose scale grows is rounded again only where a code falls below
// e4m3's normal range. Arithmetic is in 32 bits up to the one rounding.
//
// Its floor is memory: 2 bytes an element in, 1 out (queries 2 and 2). A scale needs all of a block's tokens of a
// head, so the unit of work is that: a warp loads the block's rows, takes their maximum by shuffles, and keeps them in
// registers until they are written. A CTA takes a block of all heads, keys and values, and looks up place and angles
// once; other CTAs take the queries, a few tokens each. Measured: 64 turns of 256 to 1024 tokens, 28 + 2 x 4 heads of
// 128 with norms, 0.73 GB: 181 us, 4.0 TB/s, of which the queries alone take 125 (5 TB/s); the blocks wait for their
// lookups, loads and maxima one after another.
#pragma once
#include "lsmkv_attend.cuh"

namespace lsmkv {

constexpr int kScaleMin = -100, kScaleMax = 100;   // exponents of a block's scale

// A layer's 8-bit buffers: page slabs of codes [page_tokens][heads][head_dim], then scale bytes
// [heads][page_tokens / B] (exponent + 127).
struct CodeArgs {
    uint64_t page_bytes;
    uint32_t code_bytes;     // of a slab: page_tokens * heads * head_dim
    uint32_t block_log2;     // B
    uint32_t page_log2;      // of page_tokens; 32: it is no power of two
};

// Page of a sequence's token, and its slot there. (A division takes tens of instructions.)
__device__ __forceinline__ uint32_t page_of_token(const CodeArgs &c, uint32_t page_tokens, uint32_t t)
{
    return c.page_log2 < 32 ? t >> c.page_log2 : t / page_tokens;
}

__device__ __forceinline__ uint32_t slot_of_token(const CodeArgs &c, uint32_t page_tokens, uint32_t t)
{
    return c.page_log2 < 32 ? t & (page_tokens - 1) : t % page_tokens;
}

__device__ __forceinline__ int scale_exponent(uint32_t byte)
{
    const int e = (int)byte - 127;
    return e < kScaleMin ? kScaleMin : e > kScaleMax ? kScaleMax : e;
}

__device__ __forceinline__ float power_of_two(int e) { return __int_as_float((e + 127) << 23); }

// Least e with x <= 448 * 2^e = 1.75 * 2^(e + 8), from the bits of x >= 0.
__device__ __forceinline__ int least_exponent(float x)
{
    const int e = ((__float_as_int(x) + 0x1FFFFF) >> 23) - 135;
    return e < kScaleMin ? kScaleMin : e > kScaleMax ? kScaleMax : e;
}

// Two codes, the first in the low byte.
__device__ __forceinline__ uint32_t to_codes2(float a, float b)
{
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(b), "f"(a));
    return r;
}

__device__ __forceinline__ uint32_t to_codes4(float a, float b, float c, float d)
{
    return to_codes2(a, b) | (to_codes2(c, d) << 16);
}

// Four codes as 16-bit floats: the first two, the last two. Exact.
__device__ __forceinline__ void from_codes4(uint32_t c, uint32_t &lo, uint32_t &hi)
{
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
        : "=r"(lo), "=r"(hi) : "r"(c));
}

// Four codes times 2^-by, by in 1..200. (From 2^-19 on every code becomes zero: 448 2^-19 is less than half of the
// least one, 2^-9. 2^-126 is the least factor that 32 bits hold.)
__device__ __forceinline__ uint32_t shrink_codes4(uint32_t c, int by)
{
    uint32_t lo, hi;
    from_codes4(c, lo, hi);
    const float2 a = Half2<__half>::up(lo), b = Half2<__half>::up(hi);
    const float f = power_of_two(-min(by, 126));
    return to_codes4(a.x * f, a.y * f, b.x * f, b.y * f);
}

constexpr float kLargest = 3.4028234664e38f;

// x times 0 is NaN for an infinity (and no compiler may drop it here)
__device__ __forceinline__ float infinite_to_nan(float x)
{
    float y;
    asm("fma.rn.f32 %0, %1, 0f00000000, %1;" : "=f"(y) : "f"(x));
    return y;
}

struct Append8Job {
    AppendJob a;
    CodeArgs c;
    uint32_t q_blocks;       // CTAs that take queries
    uint32_t per_seq;        // block slots a sequence, 0: as many as its length asks for (see find_block)
};

// The block that a CTA takes: `count` new tokens from row t0 on, in slots [slot, slot + count) of a page, of
// which the first `have` behind `begin` are held already.
struct BlockPlace {
    uint64_t t0;
    uint32_t page, begin, have, count, pos;
};

// Block slot g of the batch. A sequence of n new tokens touches at most n / B + 2 blocks, and with
// slots from new_off / B + 2 i on every sequence has that many: no launch before, nothing for the host to
// know. Batches of one token each, and others where it takes no more, have per_seq slots a sequence.
__device__ __forceinline__ bool find_block(const Append8Job &J, uint32_t g, BlockPlace *p, bool report)
{
    // (there are at least as many slots as sequences: every sequence is checked by one CTA)
    if (report && g < J.a.seqs.n_seq && !load_seq(J.a.seqs, g, J.a.page_tokens).ok)
        st_flag(J.a.st, LSMKV_ST_BAD_COUNT, g);
    const AppendJob &j = J.a;
    const uint32_t lb = J.c.block_log2, B = 1u << lb, lane = lane_id();
    uint32_t i, k;
    if (J.per_seq) {
        i = g / J.per_seq;
        k = g - i * J.per_seq;
    } else {
        auto base = [&](uint32_t s) { return (uint32_t)(j.seqs.new_off[s] >> lb) + 2 * s; };
        uint32_t lo = 0, hi = j.seqs.n_seq;                  // base(lo) <= g < base(hi), or hi == n_seq
        while (hi - lo > 1) {
            const uint32_t span = hi - lo;
            const uint32_t at = lo + (uint32_t)((uint64_t)span * (lane + 1) / 33);
            const unsigned below = __ballot_sync(~0u, base(at) <= g);
            const int last = 31 - __clz(below);
            const uint32_t new_lo = last < 0 ? lo : lo + (uint32_t)((uint64_t)span * (last + 1) / 33);
            const uint32_t new_hi = last == 31 ? hi : lo + (uint32_t)((uint64_t)span * (last + 2) / 33);
            lo = new_lo;
            hi = new_hi > new_lo ? new_hi : new_lo + 1;
        }
        i = lo;
        const uint32_t b = base(i);
        if (b > g) return false;                             // (offsets that do not ascend)
        k = g - b;
    }
    const SeqInfo s = load_seq(j.seqs, i, j.page_tokens);
    if (!s.ok) return false;
    const int64_t p0 = (int64_t)s.kv - (int64_t)s.rows;      // position of the first new token
    const uint32_t first = p0 > 0 ? (uint32_t)p0 : 0u;
    const uint64_t begin = ((uint64_t)(first >> lb) + k) << lb;      // position of the block
    if (begin >= s.kv || s.rows == 0) return false;
    const uint32_t from = max((uint32_t)begin, first), to = min((uint32_t)begin + B, s.kv);
    const uint64_t entry = s.page0 + (uint32_t)begin / j.page_tokens;
    p->page = j.seqs.page_table[entry];
    if (p->page >= j.num_pages) {
        if (report) st_flag(j.st, LSMKV_ST_BAD_PAGE, entry);
        return false;
    }
    p->t0 = s.row0 + (uint64_t)((int64_t)from - p0);
    p->pos = from;
    p->begin = (uint32_t)begin % j.page_tokens;
    p->have = from - (uint32_t)begin;
    p->count = to - from;
    return true;
}

// Row of the rotation table of new token t at position pos; ~0 when there is none (reported).
__device__ __forceinline__ uint64_t angle_row(const AppendJob &j, uint64_t t, uint32_t pos, bool report)
{
    const uint64_t r = j.positions ? (uint64_t)j.positions[t] : (uint64_t)pos;
    if (!j.table || r < j.n_pos) return r;
    if (report) st_flag(j.st, LSMKV_ST_BAD_COUNT, t);
    return ~0ull;
}

// A lane's part of a head: two 16-byte pieces, chosen as in the 16-bit append so that every pair of
// elements lies in one lane.
struct LanePieces {
    uint32_t l, pa, pb, turned, angle_at;
    bool has_a, has_b, split;
    __device__ __forceinline__ LanePieces(const AppendJob &j, unsigned lane)
    {
        const uint32_t half = j.rot_dim / 2, pieces = j.head_dim / 8;
        l = lane & ((1u << j.lane_log2) - 1);
        split = !j.interleaved && j.rot_dim;
        if (split && l < half / 8) {
            pa = l;
            pb = l + half / 8;
        } else if (split) {
            pa = j.rot_dim / 8 + 2 * (l - half / 8);
            pb = pa + 1;
        } else {
            pa = 2 * l;
            pb = pa + 1;
        }
        has_a = pa < pieces;
        has_b = pb < pieces;
        turned = split ? (l < half / 8 ? 8u : 0u) : half > pa * 4 ? min(8u, half - pa * 4) : 0u;
        angle_at = split ? pa * 8 : pa * 4;
    }
};

// Sixteen elements of a lane, in 32 bits, and what happens to them.
template <typename T>
struct LaneRow {
    float2 x[4], y[4];
    __device__ __forceinline__ void take(const uint4 &a, const uint4 &b)
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[e] = Half2<T>::up((&a.x)[e]);
            y[e] = Half2<T>::up((&b.x)[e]);
        }
    }
    // all lanes of the head take part
    __device__ __forceinline__ void norm(const AppendJob &j, const float2 (&wa)[4], const float2 (&wb)[4])
    {
        float2 sum = mul2(x[0], x[0]), more = mul2(y[0], y[0]);
#pragma unroll
        for (int e = 1; e < 4; ++e) {
            sum = fma2(x[e], x[e], sum);
            more = fma2(y[e], y[e], more);
        }
        sum = add2(sum, more);
        float all = sum.x + sum.y;
        for (uint32_t d = 1u << j.lane_log2 >> 1; d; d >>= 1) all += __shfl_xor_sync(~0u, all, d);
        const float scale = rsqrtf(all / (float)j.head_dim + j.eps);
        const float2 sc = make_float2(scale, scale);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[e] = mul2(mul2(x[e], sc), wa[e]);
            y[e] = mul2(mul2(y[e], sc), wb[e]);
        }
    }
    __device__ __forceinline__ void turn(const LanePieces &p, const float *row, uint32_t half)
    {
        row += p.angle_at;
        if (p.split && p.turned) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 c = *reinterpret_cast<const float2 *>(row + 2 * e);
                const float2 s = *reinterpret_cast<const float2 *>(row + half + 2 * e);
                const float2 minus = make_float2(-s.x, -s.y);
                const float2 t = fma2(y[e], minus, mul2(x[e], c));
                y[e] = fma2(y[e], c, mul2(x[e], s));
                x[e] = t;
            }
        } else if (!p.split) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if ((uint32_t)e < p.turned) {
                    float2 &v = e < 4 ? x[e] : y[e - 4];
                    const float c = row[e], s = row[half + e], t = v.x;
                    v.x = t * c - v.y * s;
                    v.y = v.y * c + t * s;
                }
            }
        }
    }
    __device__ __forceinline__ float largest(bool &undefined) const
    {
        float m = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float2 v = e < 4 ? x[e] : y[e - 4];
            const float a = fabsf(v.x), b = fabsf(v.y);
            undefined |= !(a <= kLargest) || !(b <= kLargest);
            m = fmaxf(m, a <= kLargest ? a : 0.f);
            m = fmaxf(m, b <= kLargest ? b : 0.f);
        }
        return m;
    }
};

template <typename T>
__device__ __forceinline__ void load_weights(const void *weights, const LanePieces &p, float2 (&wa)[4], float2 (&wb)[4])
{
    const uint4 *wv = static_cast<const uint4 *>(weights);
    const uint4 a = p.has_a ? wv[p.pa] : make_uint4(0, 0, 0, 0), b = p.has_b ? wv[p.pb] : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        wa[e] = Half2<T>::up((&a.x)[e]);
        wb[e] = Half2<T>::up((&b.x)[e]);
    }
}

// Scale of a block of one head after the new tokens, whose largest finite element is `top` (in all
// lanes): the exponent, with the codes of `have` earlier tokens brought to it.
__device__ __forceinline__ int settle_scale(unsigned char *block, uint64_t row_bytes, uint32_t head_dim, uint32_t have,
                                            unsigned char *scale, float top)
{
    const unsigned lane = lane_id();
    int e = least_exponent(top);
    if (have) {
        const int old = scale_exponent(*scale);
        if (old >= e) {
            e = old;
        } else {
            const uint32_t words = head_dim / 4;
            for (uint32_t x = lane; x < have * words; x += 32) {
                const uint32_t r = x / words;
                uint32_t *at = reinterpret_cast<uint32_t *>(block + r * row_bytes) + (x - r * words);
                *at = shrink_codes4(*at, e - old);
            }
        }
    }
    __syncwarp();                // every lane has read the old scale
    if (lane == 0) *scale = (unsigned char)(e + 127);
    return e;
}

constexpr int kAppend8Warps = 8;

// Queries of j.tokens tokens from row t0 on, by a CTA: places and angles looked up first, then a head a lane group and
// pass, the next pass's pieces loaded ahead.
template <typename T>
__device__ __forceinline__ void append_queries(const AppendJob &j, uint32_t t0, float (*angles)[256], TokenPlace *places)
{
    const unsigned lane = lane_id(), w = threadIdx.x >> 5;
    const uint32_t half = j.rot_dim / 2, groups = 32u >> j.lane_log2, sub = lane >> j.lane_log2;
    const LanePieces lp(j, lane);
    const uint4 none = make_uint4(0, 0, 0, 0);
    const uint32_t here = min((uint32_t)j.seqs.n_new - t0, j.tokens);
    const uint32_t n = j.n_q_heads, rows = here * n, stride = kAppend8Warps * groups;
    const T *const q = static_cast<const T *>(j.q);
    T *const out = static_cast<T *>(j.q_out);
    uint32_t r = w * groups + sub, tok = r / n, h = r - tok * n;
    uint4 a = none, b = none;
    auto fetch = [&](uint4 &x, uint4 &y) {
        x = y = none;
        if (tok >= here) return;
        const uint4 *src = reinterpret_cast<const uint4 *>(q + (uint64_t)(t0 + tok) * j.q_ts + (uint64_t)h * j.q_hs);
        if (lp.has_a) x = src[lp.pa];
        if (lp.has_b) y = src[lp.pb];
    };
    fetch(a, b);
    if (w < here) {
        const TokenPlace at = place_token(j, t0 + w, lane, false);
        if (lane == 0) places[w] = at;
        if (at.state == 2)
            for (uint32_t e = lane * 4; e < j.rot_dim; e += 128)
                *reinterpret_cast<float4 *>(&angles[w][e]) =
                    *reinterpret_cast<const float4 *>(j.table + at.angle * j.rot_dim + e);
    }
    __syncthreads();
    float2 wa[4], wb[4];
    if (j.q_norm) load_weights<T>(j.q_norm, lp, wa, wb);
    for (uint32_t r0 = w * groups; r0 < rows; r0 += stride) {
        const uint32_t on = tok, head = h;
        h += stride;
        while (h >= n) {
            h -= n;
            ++tok;
        }
        uint4 na, nb;
        fetch(na, nb);
        const int state = on < here ? places[on].state : 0;
        LaneRow<T> v;
        v.take(a, b);
        if (j.q_norm) v.norm(j, wa, wb);
        if (half && state == 2) v.turn(lp, angles[on], half);
        if (state) {
            // what neither norm nor rotation touched keeps its bits; padding is zero
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (j.q_norm || (uint32_t)e < lp.turned) (&a.x)[e] = Half2<T>::down(v.x[e].x, v.x[e].y);
                if (j.q_norm || (uint32_t)e + 4 < lp.turned) (&b.x)[e] = Half2<T>::down(v.y[e].x, v.y[e].y);
            }
            if (state == 1) a = b = none;
            uint4 *dst = reinterpret_cast<uint4 *>(out + (uint64_t)(t0 + on) * j.o_ts + (uint64_t)head * j.o_hs);
            if (lp.has_a) dst[lp.pa] = a;
            if (lp.has_b) dst[lp.pb] = b;
        }
        a = na;
        b = nb;
    }
}

// The queries alone, of large batches: at 80 registers three CTAs a SM, where the blocks of keys and values take
// 128. (The turns above: 207 us in one launch.)
template <typename T>
__global__ __launch_bounds__(kAppend8Warps * 32, 3) void k_append8_queries(const __grid_constant__ AppendJob j)
{
    __shared__ __align__(16) float angles[kAppend8Warps][256];
    __shared__ TokenPlace places[kAppend8Warps];
    follow_launch();             // (the blocks of keys and values may start beside)
    append_queries<T>(j, blockIdx.x * j.tokens, angles, places);
}

// Keys and values of block slot g, by a CTA: a warp takes a head's keys or values at a time.
template <typename T, int kPasses>
__device__ __forceinline__ void append_block(const Append8Job &J, uint32_t g, float (*angles)[256], uint32_t &stored)
{
    const AppendJob &j = J.a;
    const unsigned lane = lane_id(), w = threadIdx.x >> 5;
    const uint32_t half = j.rot_dim / 2, D = j.head_dim, H = j.n_kv_heads;
    const uint32_t groups = 32u >> j.lane_log2, sub = lane >> j.lane_log2;
    const LanePieces lp(j, lane);
    const uint4 none = make_uint4(0, 0, 0, 0);

    unsigned char *const kbuf = static_cast<unsigned char *>(j.kv_ptrs[j.layer]);
    unsigned char *const vbuf = static_cast<unsigned char *>(j.kv_ptrs[j.n_layers + j.layer]);
    if ((reinterpret_cast<uintptr_t>(kbuf) | reinterpret_cast<uintptr_t>(vbuf)) & 15u) {
        if (threadIdx.x == 0) st_flag(j.st, LSMKV_ST_MISALIGNED, 0);
        return;
    }
    BlockPlace p;
    if (!find_block(J, g, &p, threadIdx.x == 0)) return;
    // a unit: a head's keys, or its values; the first one's rows are under way while the angles are looked up
    uint4 a[kPasses], b[kPasses];
    auto fetch = [&](uint32_t u) {
        const uint32_t h = u < H ? u : u - H;
        const T *const src = u < H ? static_cast<const T *>(j.k) + h * j.k_hs : static_cast<const T *>(j.v) + h * j.v_hs;
        const uint64_t ts = u < H ? j.k_ts : j.v_ts;
#pragma unroll
        for (int s = 0; s < kPasses; ++s) {
            const uint32_t k = s * groups + sub;
            a[s] = b[s] = none;
            if (k < p.count) {
                const uint4 *row = reinterpret_cast<const uint4 *>(src + (p.t0 + k) * ts);
                if (lp.has_a) a[s] = row[lp.pa];
                if (lp.has_b) b[s] = row[lp.pb];
            }
        }
    };
    if (w < 2 * H) fetch(w);
    if (threadIdx.x == 0) stored = 0;
    __syncthreads();
    for (uint32_t k = w; k < p.count; k += kAppend8Warps) {
        const uint64_t row = angle_row(j, p.t0 + k, p.pos + k, lane == 0);
        if (row == ~0ull) continue;
        if (lane == 0) atomicOr(&stored, 1u << k);
        for (uint32_t e = lane * 4; e < j.rot_dim; e += 128)
            *reinterpret_cast<float4 *>(&angles[k][e]) = *reinterpret_cast<const float4 *>(j.table + row * j.rot_dim + e);
    }
    __syncthreads();
    const uint32_t real = stored, blocks = j.page_tokens >> J.c.block_log2;
    if (!real) return;
    const uint64_t row_bytes = (uint64_t)H * D, slab = (uint64_t)p.page * J.c.page_bytes;
    float2 wa[4], wb[4];
    if (j.k_norm) load_weights<T>(j.k_norm, lp, wa, wb);
    for (uint32_t u = w; u < 2 * H; u += kAppend8Warps) {
        const bool key = u < H;
        const uint32_t h = key ? u : u - H;
        if (u != w) fetch(u);
        LaneRow<T> v[kPasses];
        float top = 0.f;
        bool undefined = false;
#pragma unroll
        for (int s = 0; s < kPasses; ++s) {
            if (s * groups >= p.count) break;                // (the same for all lanes)
            const uint32_t k = s * groups + sub;
            const bool in = k < 16 && (real >> k & 1);
            if (!in) a[s] = b[s] = none;                     // (a token left out counts for nothing)
            v[s].take(a[s], b[s]);
            if (key && j.k_norm) v[s].norm(j, wa, wb);
            if (key && half && in) v[s].turn(lp, angles[k], half);
            top = fmaxf(top, v[s].largest(undefined));
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
        undefined = __any_sync(~0u, undefined);
        unsigned char *const buf = (key ? kbuf : vbuf) + slab;
        unsigned char *const block = buf + p.begin * row_bytes + (uint64_t)h * D;
        const int e = settle_scale(block, row_bytes, D, p.have,
                                   buf + J.c.code_bytes + h * blocks + (p.begin >> J.c.block_log2), top);
        const float f = power_of_two(-e);
        const float2 ff = make_float2(f, f);
#pragma unroll
        for (int s = 0; s < kPasses; ++s) {
            const uint32_t k = s * groups + sub;
            if (s * groups >= p.count) break;
            if (k >= 16 || !(real >> k & 1)) continue;
            float2 x[4], y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[i] = mul2(v[s].x[i], ff);
                y[i] = mul2(v[s].y[i], ff);
                if (undefined) {
                    x[i] = make_float2(infinite_to_nan(x[i].x), infinite_to_nan(x[i].y));
                    y[i] = make_float2(infinite_to_nan(y[i].x), infinite_to_nan(y[i].y));
                }
            }
            unsigned char *const dst = block + (p.have + k) * row_bytes;
            if (lp.has_a)
                *reinterpret_cast<uint2 *>(dst + lp.pa * 8) = make_uint2(
                    to_codes4(x[0].x, x[0].y, x[1].x, x[1].y), to_codes4(x[2].x, x[2].y, x[3].x, x[3].y));
            if (lp.has_b)
                *reinterpret_cast<uint2 *>(dst + lp.pb * 8) = make_uint2(
                    to_codes4(y[0].x, y[0].y, y[1].x, y[1].y), to_codes4(y[2].x, y[2].y, y[3].x, y[3].y));
        }
    }
}

// kPasses: passes of a warp over the rows of a block of tokens, at most; one is enough for single tokens, whose
// CTAs then fit four to a SM.
template <typename T, int kPasses>
__global__ __launch_bounds__(kAppend8Warps * 32, kPasses == 1 ? 4 : kPasses <= 4 ? 2 : 1)
void k_append8(const __grid_constant__ Append8Job J)
{
    __shared__ __align__(16) float angles[16][256];          // cosines and sines of the tokens
    __shared__ TokenPlace places[kAppend8Warps];
    __shared__ uint32_t stored;                              // bit k: token k of the block has its angles
    if (blockIdx.x < J.q_blocks) append_queries<T>(J.a, blockIdx.x * J.a.tokens, angles, places);
    else append_block<T, kPasses>(J, blockIdx.x - J.q_blocks, angles, stored);
    wait_launch();               // what comes behind may count on the queries' launch too
}

// Element form, for rotations whose halves are not whole 16-byte pieces: a warp takes a block of a head,
// its tokens one after the other and twice (for the maximum, then to write), a lane every 32nd pair.
template <typename T>
__global__ __launch_bounds__(128) void k_append8_elements(const __grid_constant__ Append8Job J)
{
    const AppendJob &j = J.a;
    const unsigned lane = lane_id(), w = threadIdx.x >> 5;
    const uint32_t half = j.rot_dim / 2, D = j.head_dim, H = j.n_kv_heads;
    // visit(element, value) for all elements of a row after norm and rotation, those of this lane
    auto row_values = [&](const T *src, const T *wt, const float *row, auto visit) {
        float scale = 1.f;
        if (wt) {
            float sum = 0.f;
            for (uint32_t e = lane; e < D; e += 32) {
                const float x = Half2<T>::up1(src[e]);
                sum += x * x;
            }
            for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(~0u, sum, d);
            scale = rsqrtf(sum / (float)D + j.eps);
        }
        auto at = [&](uint32_t e) { return Half2<T>::up1(src[e]) * (wt ? scale * Half2<T>::up1(wt[e]) : 1.f); };
        uint32_t done = 0;
        if (row) {
            for (uint32_t e = lane; e < half; e += 32) {
                const uint32_t ia = j.interleaved ? 2 * e : e, ib = j.interleaved ? 2 * e + 1 : e + half;
                const float p = at(ia), q = at(ib), c = row[e], s = row[half + e];
                visit(ia, p * c - q * s);
                visit(ib, q * c + p * s);
            }
            done = j.rot_dim;
        }
        for (uint32_t e = done + lane; e < D; e += 32) visit(e, at(e));
    };
    if (blockIdx.x < J.q_blocks) {
        const uint64_t row = (uint64_t)blockIdx.x * 4 + w;
        if (row >= j.seqs.n_new * j.n_q_heads) return;
        const uint64_t t = row / j.n_q_heads;
        const uint32_t h = (uint32_t)(row - t * j.n_q_heads);
        const TokenPlace at = place_token(j, t, lane, false);
        T *const dst = static_cast<T *>(j.q_out) + t * j.o_ts + h * j.o_hs;
        const T *const src = static_cast<const T *>(j.q) + t * j.q_ts + h * j.q_hs;
        if (at.state == 1)
            for (uint32_t e = lane; e < D; e += 32) dst[e] = Half2<T>::down1(0.f);
        // (without a norm, what lies behind the rotation passes through 32 bits and back unchanged)
        else if (at.state == 2)
            row_values(src, static_cast<const T *>(j.q_norm), half ? j.table + at.angle * j.rot_dim : nullptr,
                       [&](uint32_t e, float x) { dst[e] = Half2<T>::down1(x); });
        return;
    }
    unsigned char *const kbuf = static_cast<unsigned char *>(j.kv_ptrs[j.layer]);
    unsigned char *const vbuf = static_cast<unsigned char *>(j.kv_ptrs[j.n_layers + j.layer]);
    if ((reinterpret_cast<uintptr_t>(kbuf) | reinterpret_cast<uintptr_t>(vbuf)) & 15u) {
        if (threadIdx.x == 0) st_flag(j.st, LSMKV_ST_MISALIGNED, 0);
        return;
    }
    BlockPlace p;
    if (!find_block(J, blockIdx.x - J.q_blocks, &p, threadIdx.x == 0)) return;
    const uint32_t blocks = j.page_tokens >> J.c.block_log2;
    const uint64_t row_bytes = (uint64_t)H * D, slab = (uint64_t)p.page * J.c.page_bytes;
    for (uint32_t u = w; u < 2 * H; u += 4) {
        const bool key = u < H;
        const uint32_t h = key ? u : u - H;
        const T *const src = key ? static_cast<const T *>(j.k) + h * j.k_hs : static_cast<const T *>(j.v) + h * j.v_hs;
        const uint64_t ts = key ? j.k_ts : j.v_ts;
        const T *const wt = key ? static_cast<const T *>(j.k_norm) : nullptr;
        uint32_t real = 0;
        float top = 0.f;
        for (uint32_t k = 0; k < p.count; ++k) {
            const uint64_t row = angle_row(j, p.t0 + k, p.pos + k, u == 0 && lane == 0);
            if (row == ~0ull) continue;
            real |= 1u << k;
            row_values(src + (p.t0 + k) * ts, wt, key && half ? j.table + row * j.rot_dim : nullptr,
                       [&](uint32_t, float x) {
                           if (fabsf(x) <= kLargest) top = fmaxf(top, fabsf(x));
                       });
        }
        if (!real) continue;
        for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
        unsigned char *const buf = (key ? kbuf : vbuf) + slab;
        unsigned char *const block = buf + p.begin * row_bytes + (uint64_t)h * D;
        const float f = power_of_two(-settle_scale(block, row_bytes, D, p.have,
                                                   buf + J.c.code_bytes + h * blocks + (p.begin >> J.c.block_log2), top));
        for (uint32_t k = 0; k < p.count; ++k) {
            if (!(real >> k & 1)) continue;
            const uint64_t row = angle_row(j, p.t0 + k, p.pos + k, false);
            unsigned char *const dst = block + (p.have + k) * row_bytes;
            row_values(src + (p.t0 + k) * ts, wt, key && half ? j.table + row * j.rot_dim : nullptr,
                       [&](uint32_t e, float x) { dst[e] = (unsigned char)to_codes2(infinite_to_nan(x * f), 0.f); });
        }
    }
}

}  // namespace lsmkv
