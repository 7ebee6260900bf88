// Append: the keys and values of new tokens enter the paged pool, keys (and the queries beside
// them) after the norm of each head and the position rotation, in one pass over the projections.
//
//   y = x * rsqrt(mean(x^2) + eps) * w           (norm, per head, optional)
//   (a, b) -> (a cos p - b sin p, b cos p + a sin p)   (rotation, per pair, optional)
//
// Bound by memory: every element is read once and written once. A warp owns a part of the heads
// of one token: a lane always holds the same element pairs of a head, so the token's cosines and
// sines are fetched once into registers and serve all its heads, and no pair crosses lanes. The
// loads of the heads are issued before the token's sequence is looked up, because only the
// destination and the angle depend on it.
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
    uint32_t parts;      // warps that share a token's heads
    uint32_t lane_log2;  // vector form: lanes per head, as a power of two
    DevStatus *st;
};

// The sequence of row t: the largest i with new_off[i] <= t, found by the warp's lanes together
// (33 parts a trip: two trips up to 1088 sequences). A batch of equal lengths needs one guess.
__device__ __forceinline__ uint32_t find_seq(const uint64_t *off, uint32_t n_seq, uint64_t n_new,
                                             uint64_t t, unsigned lane)
{
    const uint32_t guess = n_seq == n_new ? (uint32_t)t : (uint32_t)(t * n_seq / n_new);
    if (off[guess] <= t && off[guess + 1] > t) return guess;
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
// A warp's U heads-per-lane-group loads are in flight together.
template <typename T, int U>
__global__ __launch_bounds__(128) void k_append(const AppendJob j)
{
    const unsigned lane = lane_id();
    const uint64_t warp = (uint64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    const uint64_t t = warp / j.parts;
    const uint32_t part = (uint32_t)(warp % j.parts);
    if (t >= j.seqs.n_new) return;
    T *const kbuf = static_cast<T *>(j.kv_ptrs[j.layer]);
    T *const vbuf = static_cast<T *>(j.kv_ptrs[j.n_layers + j.layer]);

    const uint32_t slots = j.n_q_heads + 2 * j.n_kv_heads;
    const uint32_t lanes = 1u << j.lane_log2, groups = 32u >> j.lane_log2;
    const uint32_t l = lane & (lanes - 1), g = lane >> j.lane_log2;
    const uint32_t pieces = j.head_dim / 8;
    const uint32_t half = j.rot_dim / 2;
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

    TokenPlace at;
    float c[8], s[8];
    bool known = false;
    const uint32_t step = groups * j.parts;
    for (uint32_t h0 = part * groups; h0 < slots; h0 += step * U) {
        uint4 a[U], b[U];
        int kind[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t h = h0 + u * step + g;
            a[u] = b[u] = make_uint4(0, 0, 0, 0);
            kind[u] = 3;
            if (h < slots) {
                const uint4 *src = reinterpret_cast<const uint4 *>(head_src<T>(j, t, h, &kind[u]));
                if (has_a) a[u] = src[pa];
                if (has_b) b[u] = src[pb];
            }
        }
        if (!known) {
            known = true;
            at = place_token(j, t, lane, part == 0);
            if (((reinterpret_cast<uintptr_t>(kbuf) | reinterpret_cast<uintptr_t>(vbuf)) & 15u)) {
                if (lane == 0) st_flag(j.st, LSMKV_ST_MISALIGNED, 0);
                return;
            }
            if (at.state == 0) return;
#pragma unroll
            for (int e = 0; e < 8; ++e) { c[e] = 1.f; s[e] = 0.f; }
            if (at.state == 2 && j.rot_dim) {
                const float *row = j.table + at.angle * j.rot_dim;
                // half-split: eight pairs of pieces a and b; interleaved: four pairs of each
                const uint32_t first = split ? pa * 8 : pa * 4;
                const uint32_t n_a = split ? (l < half / 8 ? 8u : 0u)
                                           : (first < half ? min(8u, half - first) : 0u);
#pragma unroll
                for (int e = 0; e < 8; e += 4) {
                    if ((uint32_t)e < n_a) {
                        const float4 cc = *reinterpret_cast<const float4 *>(row + first + e);
                        const float4 ss = *reinterpret_cast<const float4 *>(row + half + first + e);
                        c[e] = cc.x; c[e + 1] = cc.y; c[e + 2] = cc.z; c[e + 3] = cc.w;
                        s[e] = ss.x; s[e + 1] = ss.y; s[e + 2] = ss.z; s[e + 3] = ss.w;
                    }
                }
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t h = h0 + u * step + g;
            const void *w = kind[u] == 0 ? j.q_norm : kind[u] == 1 ? j.k_norm : nullptr;
            const bool touch = kind[u] < 2 && (w || j.rot_dim);
            float scale = 1.f;
            // the sum of squares needs every lane of the warp, whatever its head's kind
            if (j.q_norm || j.k_norm) {
                float sum = 0.f;
                const uint32_t *ra = &a[u].x, *rb = &b[u].x;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 x = Half2<T>::up(ra[e]), y = Half2<T>::up(rb[e]);
                    sum += x.x * x.x + x.y * x.y + y.x * y.x + y.y * y.y;
                }
                for (uint32_t d = lanes >> 1; d; d >>= 1) sum += __shfl_xor_sync(~0u, sum, d);
                if (w) scale = rsqrtf(sum / (float)j.head_dim + j.eps);
            }
            if (touch && at.state == 2) {
                float x[16];
                uint32_t *ra = &a[u].x, *rb = &b[u].x;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 p = Half2<T>::up(ra[e]), q = Half2<T>::up(rb[e]);
                    x[2 * e] = p.x; x[2 * e + 1] = p.y;
                    x[8 + 2 * e] = q.x; x[8 + 2 * e + 1] = q.y;
                }
                if (w) {
                    const uint4 *wv = static_cast<const uint4 *>(w);
                    const uint4 wa = has_a ? wv[pa] : make_uint4(0, 0, 0, 0);
                    const uint4 wb = has_b ? wv[pb] : make_uint4(0, 0, 0, 0);
                    const uint32_t *qa = &wa.x, *qb = &wb.x;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float2 p = Half2<T>::up(qa[e]), q = Half2<T>::up(qb[e]);
                        x[2 * e] *= scale * p.x; x[2 * e + 1] *= scale * p.y;
                        x[8 + 2 * e] *= scale * q.x; x[8 + 2 * e + 1] *= scale * q.y;
                    }
                }
                if (split && l < half / 8) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float p = x[e], q = x[8 + e];
                        x[e] = p * c[e] - q * s[e];
                        x[8 + e] = q * c[e] + p * s[e];
                    }
                } else if (!split && j.rot_dim) {
                    const uint32_t first = pa * 4;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        if (first + e < half) {
                            const float p = x[2 * e], q = x[2 * e + 1];
                            x[2 * e] = p * c[e] - q * s[e];
                            x[2 * e + 1] = q * c[e] + p * s[e];
                        }
                    }
                }
                // elements that neither norm nor rotation touched keep their bits
                const uint32_t turned = split ? (l < half / 8 ? 8u : 0u)
                                              : half > pa * 4 ? half - pa * 4 : 0u;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (w || (uint32_t)e < turned) ra[e] = Half2<T>::down(x[2 * e], x[2 * e + 1]);
                    if (w || (uint32_t)e + 4 < turned)
                        rb[e] = Half2<T>::down(x[8 + 2 * e], x[8 + 2 * e + 1]);
                }
            }
            if (kind[u] == 3) continue;
            if (at.state == 1) {
                if (kind[u] != 0) continue;
                a[u] = b[u] = make_uint4(0, 0, 0, 0);
            }
            uint4 *dst = reinterpret_cast<uint4 *>(head_dst<T>(j, t, h, at, kbuf, vbuf));
            if (!dst) continue;
            if (has_a) dst[pa] = a[u];
            if (has_b) dst[pb] = b[u];
        }
    }
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
