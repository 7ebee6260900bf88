// Append: the keys and values of new tokens enter the paged pool, keys (and the queries beside
// them) after the norm of each head and the position rotation, in one pass over the projections.
//
//   y = x * rsqrt(mean(x^2) + eps) * w           (norm, per head, optional)
//   (a, b) -> (a cos p - b sin p, b cos p + a sin p)   (rotation, per pair, optional)
//
// Its floor is memory: every element is read once and written once. Large batches reach 0.78 of the copy's
// rate; the counters name neither memory (58 % of its peak) nor issue (63 % of the slots) as the bound, but
// the wait for loads (long scoreboard): they run one pass ahead, at 64 registers a thread, of which the loop
// spills 84 bytes. A lane always holds whole element pairs of a head, so no pair crosses lanes.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "lsmkv_common.cuh"

namespace lsmkv {

template <typename T> struct Half2;
template <> struct Half2<__nv_bfloat16> {
    static __device__ __forceinline__ float2 up(uint32_t v)
    {
        return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u));
    }
    static __device__ __forceinline__ uint32_t down(float a, float b)
    {
        __nv_bfloat162 r = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<uint32_t *>(&r);
    }
    static __device__ __forceinline__ float up1(__nv_bfloat16 v) { return __bfloat162float(v); }
    static __device__ __forceinline__ __nv_bfloat16 down1(float v) { return __float2bfloat16_rn(v); }
};
template <> struct Half2<__half> {
    static __device__ __forceinline__ float2 up(uint32_t v)
    {
        return __half22float2(*reinterpret_cast<__half2 *>(&v));
    }
    static __device__ __forceinline__ uint32_t down(float a, float b)
    {
        __half2 r = __floats2half2_rn(a, b);
        return *reinterpret_cast<uint32_t *>(&r);
    }
    static __device__ __forceinline__ float up1(__half v) { return __half2float(v); }
    static __device__ __forceinline__ __half down1(float v) { return __float2half_rn(v); }
};

// Two operations of a kind in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 d;
    asm("{\n\t.reg .b64 x, y, z, w;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\t"
        "fma.rn.f32x2 w, x, y, z;\n\tmov.b64 {%0, %1}, w;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}

__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    float2 d;
    asm("{\n\t.reg .b64 x, y, w;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\t"
        "add.rn.f32x2 w, x, y;\n\tmov.b64 {%0, %1}, w;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}

__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    float2 d;
    asm("{\n\t.reg .b64 x, y, w;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\t"
        "mul.rn.f32x2 w, x, y;\n\tmov.b64 {%0, %1}, w;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}

// The batch as the kernels take it.
struct SeqArgs {
    uint64_t n_new;
    uint32_t n_seq, max_new;
    const uint64_t *new_off;
    const uint32_t *kv_len;
    const uint64_t *page_off;
    const uint32_t *page_table;
};

// One sequence's descriptor, checked; rows = 0 for one that breaks the rules.
struct SeqInfo {
    uint64_t row0;       // its first row of q, k, v, out
    uint64_t page0;      // its first entry of page_table
    uint32_t rows, kv;   // new tokens; tokens in all
    bool ok;
};

__device__ __forceinline__ SeqInfo load_seq(const SeqArgs &a, uint32_t i, uint32_t page_tokens)
{
    SeqInfo s;
    const uint64_t r0 = a.new_off[i], r1 = a.new_off[i + 1];
    const uint64_t p0 = a.page_off[i], p1 = a.page_off[i + 1];
    s.kv = a.kv_len[i];
    s.row0 = r0;
    s.page0 = p0;
    s.ok = r0 <= r1 && r1 <= a.n_new && r1 - r0 <= a.max_new && p0 <= p1 &&
           s.kv < 0x80000000u && (p1 - p0) * page_tokens >= s.kv &&
           (i + 1 != a.n_seq || r1 == a.n_new);
    s.rows = s.ok ? (uint32_t)(r1 - r0) : 0u;
    return s;
}

struct AppendJob {
    SeqArgs seqs;
    void *const *kv_ptrs;
    uint64_t num_pages;
    uint32_t layer, n_layers, page_tokens, n_kv_heads, head_dim, n_q_heads;
    const void *k, *v, *q;
    void *q_out;
    uint64_t k_ts, k_hs, v_ts, v_hs, q_ts, q_hs, o_ts, o_hs;
    const float *table;
    const uint32_t *positions;
    uint64_t n_pos;
    uint32_t rot_dim, interleaved;
    const void *q_norm, *k_norm;
    float eps;
    uint32_t tokens;     // vector form: tokens of a block
    uint32_t parts;      // element form: warps that share a token's heads
    uint32_t lane_log2;  // vector form: lanes per head, as a power of two
    DevStatus *st;
};

// The sequence of row t: the largest i with new_off[i] <= t, found by the warp's lanes together
// (33 parts a trip: two trips up to 1088 sequences). A batch of one token each needs one look.
__device__ __forceinline__ uint32_t find_seq(const uint64_t *off, uint32_t n_seq, uint64_t n_new,
                                             uint64_t t, unsigned lane)
{
    if (n_seq == n_new && off[t] <= t && off[t + 1] > t) return (uint32_t)t;
    uint32_t lo = 0, hi = n_seq;   // off[lo] <= t, and off[hi] > t or hi == n_seq
    while (hi - lo > 1) {
        const uint32_t span = hi - lo;
        const uint32_t at = lo + (uint32_t)((uint64_t)span * (lane + 1) / 33);
        const unsigned below = __ballot_sync(~0u, off[at] <= t);
        const int last = 31 - __clz(below);   // -1 when no lane is at or below t
        const uint32_t new_lo = last < 0 ? lo : lo + (uint32_t)((uint64_t)span * (last + 1) / 33);
        const uint32_t new_hi = last == 31 ? hi : lo + (uint32_t)((uint64_t)span * (last + 2) / 33);
        // spans below 33 repeat probes; a trip always narrows the range
        lo = new_lo;
        hi = new_hi > new_lo ? new_hi : new_lo + 1;
    }
    return lo;
}

// What a token's warp needs to know beyond its data. state: 0 = left out, 1 = padding, 2 = real
struct TokenPlace {
    int state;
    uint64_t slot;       // page * page_tokens + slot in page; ~0 when its page id is bad
    uint64_t angle;      // row of the rotation table
};

__device__ __forceinline__ TokenPlace place_token(const AppendJob &j, uint64_t t, unsigned lane,
                                                  bool report)
{
    TokenPlace r;
    r.state = 0;
    r.slot = ~0ull;
    r.angle = 0;
    const uint32_t i = find_seq(j.seqs.new_off, j.seqs.n_seq, j.seqs.n_new, t, lane);
    const SeqInfo s = load_seq(j.seqs, i, j.page_tokens);
    if (!s.ok || t < s.row0 || t >= s.row0 + s.rows) {
        if (report && lane == 0) st_flag(j.st, LSMKV_ST_BAD_COUNT, i);
        return r;
    }
    const int64_t p = (int64_t)s.kv - (int64_t)s.rows + (int64_t)(t - s.row0);
    if (p < 0) {
        r.state = 1;
        return r;
    }
    r.angle = j.positions ? (uint64_t)j.positions[t] : (uint64_t)p;
    if (j.table && r.angle >= j.n_pos) {
        if (report && lane == 0) st_flag(j.st, LSMKV_ST_BAD_COUNT, t);
        return r;
    }
    const uint64_t entry = s.page0 + (uint32_t)p / j.page_tokens;
    const uint32_t page = j.seqs.page_table[entry];
    if (page < j.num_pages)
        r.slot = (uint64_t)page * j.page_tokens + (uint32_t)p % j.page_tokens;
    else if (report && lane == 0)
        st_flag(j.st, LSMKV_ST_BAD_PAGE, entry);
    r.state = 2;
    return r;
}

// Source and destination of head slot h (queries first, then keys, then values) of row t;
// kind: 0 query, 1 key, 2 value.
template <typename T>
__device__ __forceinline__ const T *head_src(const AppendJob &j, uint64_t t, uint32_t h, int *kind)
{
    if (h < j.n_q_heads) {
        *kind = 0;
        return static_cast<const T *>(j.q) + t * j.q_ts + h * j.q_hs;
    }
    h -= j.n_q_heads;
    if (h < j.n_kv_heads) {
        *kind = 1;
        return static_cast<const T *>(j.k) + t * j.k_ts + h * j.k_hs;
    }
    h -= j.n_kv_heads;
    *kind = 2;
    return static_cast<const T *>(j.v) + t * j.v_ts + h * j.v_hs;
}

template <typename T>
__device__ __forceinline__ T *head_dst(const AppendJob &j, uint64_t t, uint32_t h,
                                       const TokenPlace &at, T *kbuf, T *vbuf)
{
    if (h < j.n_q_heads) return static_cast<T *>(j.q_out) + t * j.o_ts + h * j.o_hs;
    if (at.slot == ~0ull) return nullptr;
    h -= j.n_q_heads;
    T *const base = h < j.n_kv_heads ? kbuf : vbuf;
    if (h >= j.n_kv_heads) h -= j.n_kv_heads;
    return base + (at.slot * j.n_kv_heads + h) * j.head_dim;
}

// Vector form. 2^lane_log2 lanes per head, two 16-byte pieces a lane: for half-split pairs the
// lanes below rot_dim/16 hold piece l and its partner piece l + rot_dim/16; all others (and
// interleaved pairs, which lie inside a piece) hold neighbouring pieces.
// A block takes `tokens` tokens: its warps first look up the tokens' places and angles, one each,
// then go through all query heads, all keys, all values, a head per lane group and pass, the next
// pass's pieces loaded ahead. Measured on 64 turns of 256 to 1024 tokens (41k in all) with 28 + 2 x 4
// heads of 128 and norms, 0.77 GB: 152 us, 5.1 TB/s; with kinds, addresses and weights worked out head
// by head (400 instructions a pass of four heads) 174 us; a warp per token, its angles in registers, 208.
// kOne: a token a block, for small batches: the first pass of all three kinds is loaded before
// anything is looked up.
constexpr int kAppendWarps = 8;
template <typename T, bool kOne>
__global__ __launch_bounds__(kAppendWarps * 32, kOne ? 2 : 4) void k_append(const __grid_constant__ AppendJob j)
{
    __shared__ TokenPlace places[kAppendWarps];
    __shared__ __align__(16) float angles[kAppendWarps][256];    // cosines and sines of the tokens
    const unsigned lane = lane_id(), w = threadIdx.x >> 5;
    const uint32_t t0 = blockIdx.x * j.tokens;
    const uint32_t here = min((uint32_t)j.seqs.n_new - t0, j.tokens);
    T *const kbuf = static_cast<T *>(j.kv_ptrs[j.layer]);
    T *const vbuf = static_cast<T *>(j.kv_ptrs[j.n_layers + j.layer]);

    const uint32_t lanes = 1u << j.lane_log2, groups = 32u >> j.lane_log2;
    const uint32_t l = lane & (lanes - 1), pieces = j.head_dim / 8, half = j.rot_dim / 2;
    const bool split = !j.interleaved && j.rot_dim;
    uint32_t pa, pb;      // this lane's pieces; >= pieces: none
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
    const bool has_a = pa < pieces, has_b = pb < pieces;
    // pairs (P, Q) of this lane that are turned: all, none, or (interleaved) the first few
    const uint32_t turned = split ? (l < half / 8 ? 8u : 0u) : half > pa * 4 ? min(8u, half - pa * 4) : 0u;
    const uint32_t angle_at = split ? pa * 8 : pa * 4;
    const float per_element = 1.f / (float)j.head_dim;
    const uint32_t stride = kAppendWarps * groups, r0 = w * groups + (lane >> j.lane_log2);

    auto fetch = [&](const T *src, uint32_t ts, uint32_t hs, uint32_t tok, uint32_t h, uint4 &a, uint4 &b) {
        a = b = make_uint4(0, 0, 0, 0);
        if (tok >= here) return;
        const uint4 *row = reinterpret_cast<const uint4 *>(src + ((uint64_t)(t0 + tok) * ts + (uint64_t)h * hs));
        if (has_a) a = row[pa];
        if (has_b) b = row[pb];
    };
    auto put = [&](T *dst, uint64_t off, const uint4 &a, const uint4 &b) {
        uint4 *row = reinterpret_cast<uint4 *>(dst + off);
        if (has_a) row[pa] = a;
        if (has_b) row[pb] = b;
    };
    // All heads of a kind, in passes of `stride` heads: work(token of the block, head, pieces). The
    // lanes of a warp stay together until its last lane group has no head left.
    auto first_pass = [&](const T *src, uint32_t ts, uint32_t hs, uint32_t n, uint4 &a, uint4 &b) {
        fetch(src, ts, hs, r0 / n, r0 % n, a, b);
    };
    uint4 q_a, q_b, k_a, k_b, v_a, v_b;
    if (kOne) {
        if (j.n_q_heads) first_pass(static_cast<const T *>(j.q), (uint32_t)j.q_ts, (uint32_t)j.q_hs, j.n_q_heads, q_a, q_b);
        first_pass(static_cast<const T *>(j.k), (uint32_t)j.k_ts, (uint32_t)j.k_hs, j.n_kv_heads, k_a, k_b);
        first_pass(static_cast<const T *>(j.v), (uint32_t)j.v_ts, (uint32_t)j.v_hs, j.n_kv_heads, v_a, v_b);
    }
    auto sweep = [&](const T *src, uint32_t ts, uint32_t hs, uint32_t n, uint4 &a, uint4 &b, auto work) {
        uint32_t tok = r0 / n, h = r0 - tok * n;
        uint4 na, nb;
        if (!kOne) fetch(src, ts, hs, tok, h, a, b);
        while (__any_sync(~0u, tok < here)) {
            const uint32_t on = tok, at = h;
            h += stride;
            while (h >= n) {
                h -= n;
                ++tok;
            }
            fetch(src, ts, hs, tok, h, na, nb);
            work(on, at, a, b);
            a = na;
            b = nb;
        }
    };
    if (w < here) {
        const TokenPlace at = place_token(j, t0 + w, lane, true);
        if (lane == 0) places[w] = at;
        if (at.state == 2)
            for (uint32_t e = lane * 4; e < j.rot_dim; e += 128)
                *reinterpret_cast<float4 *>(&angles[w][e]) =
                    *reinterpret_cast<const float4 *>(j.table + at.angle * j.rot_dim + e);
    }
    if (((reinterpret_cast<uintptr_t>(kbuf) | reinterpret_cast<uintptr_t>(vbuf)) & 15u)) {
        if (threadIdx.x == 0) st_flag(j.st, LSMKV_ST_MISALIGNED, 0);
        return;
    }
    __syncthreads();

    // norm and rotation of the queries or keys, then write(token, head, place, pieces)
    auto turn_heads = [&](const T *src, uint32_t ts, uint32_t hs, uint32_t n, uint4 &a0, uint4 &b0, const void *weights, auto write) {
        float2 wa[4], wb[4];
        if (weights) {
            const uint4 *wv = static_cast<const uint4 *>(weights);
            const uint4 qa = has_a ? wv[pa] : make_uint4(0, 0, 0, 0), qb = has_b ? wv[pb] : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                wa[e] = Half2<T>::up((&qa.x)[e]);
                wb[e] = Half2<T>::up((&qb.x)[e]);
            }
        }
        sweep(src, ts, hs, n, a0, b0, [&](uint32_t tok, uint32_t h, uint4 &a, uint4 &b) {
            uint32_t *ra = &a.x, *rb = &b.x;
            float2 x[4], y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[e] = Half2<T>::up(ra[e]);
                y[e] = Half2<T>::up(rb[e]);
            }
            float scale = 1.f;
            if (weights) {
                float2 sum = mul2(x[0], x[0]), more = mul2(y[0], y[0]);
#pragma unroll
                for (int e = 1; e < 4; ++e) {
                    sum = fma2(x[e], x[e], sum);
                    more = fma2(y[e], y[e], more);
                }
                sum = add2(sum, more);
                float all = sum.x + sum.y;
                for (uint32_t d = lanes >> 1; d; d >>= 1) all += __shfl_xor_sync(~0u, all, d);
                scale = rsqrtf(all * per_element + j.eps);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[e] = mul2(x[e], wa[e]);
                    y[e] = mul2(y[e], wb[e]);
                }
            }
            if (tok >= here) return;
            const float *row = angles[tok] + angle_at;
            if (split && turned) {
                const float2 minus = make_float2(-1.f, -1.f);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float4 cs = *reinterpret_cast<const float4 *>(row + (e & 2) * 2);
                    const float4 ss = *reinterpret_cast<const float4 *>(row + half + (e & 2) * 2);
                    const float2 c = e & 1 ? make_float2(cs.z, cs.w) : make_float2(cs.x, cs.y);
                    const float2 s = e & 1 ? make_float2(ss.z, ss.w) : make_float2(ss.x, ss.y);
                    const float2 p = fma2(mul2(y[e], s), minus, mul2(x[e], c));
                    y[e] = fma2(y[e], c, mul2(x[e], s));
                    x[e] = p;
                }
            } else if (!split) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if ((uint32_t)e < turned) {
                        float2 &v = e < 4 ? x[e] : y[e - 4];
                        const float c = row[e], s = row[half + e], p = v.x;
                        v.x = p * c - v.y * s;
                        v.y = v.y * c + p * s;
                    }
                }
            }
            // what neither norm nor rotation touched keeps its bits
            const float2 sc = make_float2(scale, scale);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (weights) {
                    x[e] = mul2(x[e], sc);
                    y[e] = mul2(y[e], sc);
                }
                if (weights || (uint32_t)e < turned) ra[e] = Half2<T>::down(x[e].x, x[e].y);
                if (weights || (uint32_t)e + 4 < turned) rb[e] = Half2<T>::down(y[e].x, y[e].y);
            }
            write(tok, h, a, b);
        });
    };
    // slot of a stored token, ~0 for one that is not stored
    auto slot_of = [&](uint32_t tok) { return places[tok].state == 2 ? places[tok].slot : ~0ull; };
    const uint32_t D = j.head_dim, H = j.n_kv_heads;
    if (j.n_q_heads)
        turn_heads(static_cast<const T *>(j.q), (uint32_t)j.q_ts, (uint32_t)j.q_hs, j.n_q_heads, q_a, q_b, j.q_norm,
                   [&](uint32_t tok, uint32_t h, uint4 &a, uint4 &b) {
                       const int state = places[tok].state;
                       if (state == 1) a = b = make_uint4(0, 0, 0, 0);      // padding
                       if (state)
                           put(static_cast<T *>(j.q_out),
                               (uint64_t)(t0 + tok) * (uint32_t)j.o_ts + (uint64_t)h * (uint32_t)j.o_hs, a, b);
                   });
    turn_heads(static_cast<const T *>(j.k), (uint32_t)j.k_ts, (uint32_t)j.k_hs, H, k_a, k_b, j.k_norm,
               [&](uint32_t tok, uint32_t h, uint4 &a, uint4 &b) {
                   const uint64_t slot = slot_of(tok);
                   if (slot != ~0ull) put(kbuf, (slot * H + h) * D, a, b);
               });
    sweep(static_cast<const T *>(j.v), (uint32_t)j.v_ts, (uint32_t)j.v_hs, H, v_a, v_b,
          [&](uint32_t tok, uint32_t h, uint4 &a, uint4 &b) {
              if (tok >= here) return;
              const uint64_t slot = slot_of(tok);
              if (slot != ~0ull) put(vbuf, (slot * H + h) * D, a, b);
          });
}

// Element form, for rotations whose halves are not whole 16-byte pieces: a warp takes a head at
// a time, a lane every 32nd pair, then every 32nd element behind the rotation.
template <typename T>
__global__ __launch_bounds__(128) void k_append_elements(const AppendJob j)
{
    const unsigned lane = lane_id();
    const uint64_t warp = (uint64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    const uint64_t t = warp / j.parts;
    const uint32_t part = (uint32_t)(warp % j.parts);
    if (t >= j.seqs.n_new) return;
    T *const kbuf = static_cast<T *>(j.kv_ptrs[j.layer]);
    T *const vbuf = static_cast<T *>(j.kv_ptrs[j.n_layers + j.layer]);
    if (((reinterpret_cast<uintptr_t>(kbuf) | reinterpret_cast<uintptr_t>(vbuf)) & 15u)) {
        if (lane == 0) st_flag(j.st, LSMKV_ST_MISALIGNED, 0);
        return;
    }
    const TokenPlace at = place_token(j, t, lane, part == 0);
    if (at.state == 0) return;
    const uint32_t slots = j.n_q_heads + 2 * j.n_kv_heads, half = j.rot_dim / 2, D = j.head_dim;
    const float *row = j.table + at.angle * j.rot_dim;
    for (uint32_t h = part; h < slots; h += j.parts) {
        int kind;
        const T *src = head_src<T>(j, t, h, &kind);
        T *dst = head_dst<T>(j, t, h, at, kbuf, vbuf);
        if (at.state == 1) {
            if (kind == 0)
                for (uint32_t e = lane; e < D; e += 32) dst[e] = Half2<T>::down1(0.f);
            continue;
        }
        if (!dst) continue;
        const T *w = static_cast<const T *>(kind == 0 ? j.q_norm : kind == 1 ? j.k_norm : nullptr);
        float scale = 1.f;
        if (w) {
            float sum = 0.f;
            for (uint32_t e = lane; e < D; e += 32) {
                const float x = Half2<T>::up1(src[e]);
                sum += x * x;
            }
            for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(~0u, sum, d);
            scale = rsqrtf(sum / (float)D + j.eps);
        }
        uint32_t done = 0;
        if (kind < 2 && half) {
            for (uint32_t e = lane; e < half; e += 32) {
                const uint32_t ia = j.interleaved ? 2 * e : e;
                const uint32_t ib = j.interleaved ? 2 * e + 1 : e + half;
                float p = Half2<T>::up1(src[ia]), q = Half2<T>::up1(src[ib]);
                if (w) {
                    p *= scale * Half2<T>::up1(w[ia]);
                    q *= scale * Half2<T>::up1(w[ib]);
                }
                const float c = row[e], s = row[half + e];
                dst[ia] = Half2<T>::down1(p * c - q * s);
                dst[ib] = Half2<T>::down1(q * c + p * s);
            }
            done = j.rot_dim;
        }
        for (uint32_t e = done + lane; e < D; e += 32)
            dst[e] = w ? Half2<T>::down1(Half2<T>::up1(src[e]) * (scale * Half2<T>::up1(w[e]))) : src[e];
    }
}

}  // namespace lsmkv
