// gk_append.cuh -- new keys and values into the paged cache, rotated on the way (gk_append).
//
// The unit of work is an ITEM: 16 dimensions of one head of one token, the 8 + 8 values of 8 rotation
// pairs (two 16-byte pieces, rotary_dim/2 apart, or adjacent where pairs are), so that a lane loads,
// turns and stores whole vectors and neighbouring lanes touch neighbouring addresses.
#pragma once

#include "gk_seq.cuh"

namespace gk {

struct RopeDev {
    const float *cos_sin;  // null: no rotation
    const int32_t *positions;
    uint32_t max_pos, R, interleaved, axes;
    uint32_t end0, end1;  // pairs below end0 turn by axis 0, below end1 by axis 1, the others by axis 2
};

struct RowsDev {
    const __nv_bfloat16 *p;
    uint64_t tok, head;  // elements
};

struct AppendParams {
    SeqsDev seqs;
    LayerDev cache;
    RopeDev rope;
    RowsDev q, k, v;
    __nv_bfloat16 *q_out;
    uint64_t qo_tok, qo_head;
    uint32_t Hq;
    uint32_t chunks;         // items per head row: D / 16
    FastDiv by_chunks;
    FastDiv by_row;          // items per token of the flat part of the grid
    uint32_t shared_scale;   // fp8: K and V of a page and head share one scale
    uint32_t unit_ctas, head_groups;  // fp8: CTAs that append pages; the flat part follows them
    uint32_t unit_slots;
};

constexpr int kAppendThreads = 128;
constexpr int kAppendWarps = kAppendThreads / 32;

struct Item {
    float x[16];
    uint32_t d0, d1;  // first dimensions of its two pieces
};

__device__ __forceinline__ void item_dims(const AppendParams &P, uint32_t c, bool rotated, Item &it, bool &turn)
{
    const uint32_t R = rotated ? P.rope.R : 0u;
    turn = 16u * c < R;
    if (turn && !P.rope.interleaved) {
        it.d0 = 8u * c;
        it.d1 = (R >> 1) + 8u * c;
    } else {
        it.d0 = 16u * c;
        it.d1 = 16u * c + 8u;
    }
}

__device__ __forceinline__ void unpack8(const uint4 &u, float *x)
{
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}

__device__ __forceinline__ uint4 pack8(const float *x)
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t *>(&b);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Turns the 8 pairs of chunk c of row i.  Every product is rounded by itself (no fused multiply-add): the
// result is then the textbook expression's, bit for bit, whatever compiler or library computes that.
__device__ __forceinline__ void turn_item(const AppendParams &P, uint32_t i, int pos, uint32_t c, Item &it, bool &bad)
{
    const RopeDev &r = P.rope;
    int row[3] = {pos, pos, pos};
    if (r.positions) {
#pragma unroll
        for (int a = 0; a < 3; ++a)
            if ((uint32_t)a < r.axes) row[a] = __ldg(r.positions + (uint64_t)a * P.seqs.n_tokens + i);
            else row[a] = row[0];
    }
    const uint32_t p0 = 8u * c, half = r.R >> 1;
    bad = false;
#pragma unroll
    for (int a = 0; a < 3; ++a) bad |= (uint32_t)row[a] >= r.max_pos;
    float cs[8], sn[8];
    if (bad) {
        const float nan = __int_as_float(0x7fc00000);
#pragma unroll
        for (int e = 0; e < 16; ++e) it.x[e] = nan;
        return;
    }
    const uint32_t ax0 = p0 < r.end0 ? 0u : p0 < r.end1 ? 1u : 2u;
    const uint32_t last = p0 + 7u;
    const uint32_t ax7 = last < r.end0 ? 0u : last < r.end1 ? 1u : 2u;
    if (ax0 == ax7) {
        const float *t = r.cos_sin + (uint64_t)(ax0 == 0u ? row[0] : ax0 == 1u ? row[1] : row[2]) * r.R + p0;
        *reinterpret_cast<float4 *>(cs) = __ldg(reinterpret_cast<const float4 *>(t));
        *reinterpret_cast<float4 *>(cs + 4) = __ldg(reinterpret_cast<const float4 *>(t) + 1);
        *reinterpret_cast<float4 *>(sn) = __ldg(reinterpret_cast<const float4 *>(t + half));
        *reinterpret_cast<float4 *>(sn + 4) = __ldg(reinterpret_cast<const float4 *>(t + half) + 1);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t p = p0 + e;
            const float *t = r.cos_sin + (uint64_t)(p < r.end0 ? row[0] : p < r.end1 ? row[1] : row[2]) * r.R + p;
            cs[e] = __ldg(t);
            sn[e] = __ldg(t + half);
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int ia = r.interleaved ? 2 * e : e, ib = r.interleaved ? 2 * e + 1 : e + 8;
        const float a = it.x[ia], b = it.x[ib];
        it.x[ia] = __fsub_rn(__fmul_rn(a, cs[e]), __fmul_rn(b, sn[e]));
        it.x[ib] = __fadd_rn(__fmul_rn(b, cs[e]), __fmul_rn(a, sn[e]));
    }
}

__device__ __forceinline__ void load_item(const RowsDev &r, uint64_t i, uint32_t h, Item &it)
{
    const __nv_bfloat16 *p = r.p + i * r.tok + h * r.head;
    const uint4 a = __ldg(reinterpret_cast<const uint4 *>(p + it.d0));
    const uint4 b = __ldg(reinterpret_cast<const uint4 *>(p + it.d1));
    unpack8(a, it.x);
    unpack8(b, it.x + 8);
}

// Page id of a token, or -1 (status raised) where the table holds none.
__device__ __forceinline__ int page_of(const AppendParams &P, uint32_t s, uint32_t page)
{
    int g = -1;
    if (page < P.seqs.max_pages) g = __ldg(P.seqs.page_table + (uint64_t)s * P.seqs.table_stride + page);
    if ((uint32_t)g >= P.cache.num_pages) {
        g = -1;
        if (P.seqs.status) P.seqs.status[s] = 2;  // GK_JOB_PAGE_TABLE
    }
    return g;
}

// The flat part: items of queries (and, into a bf16 cache, of keys and values), one per lane.
template <bool FP8>
__device__ __forceinline__ void append_flat(const AppendParams &P, uint32_t idx)
{
    const uint32_t i = P.by_row.div(idx);
    if (i >= P.seqs.n_tokens) return;
    const uint32_t in_row = idx - i * P.by_row.d;
    uint32_t h = P.by_chunks.div(in_row);
    const uint32_t c = in_row - h * P.chunks;
    int kind = 0;  // query, key, value
    if (h >= P.Hq) {
        h -= P.Hq;
        kind = 1;
        if (h >= P.cache.H) {
            h -= P.cache.H;
            kind = 2;
        }
    }
    Item it;
    bool turn, bad = false;
    item_dims(P, c, kind != 2, it, turn);
    load_item(kind == 0 ? P.q : kind == 1 ? P.k : P.v, i, h, it);
    const uint32_t s = seq_of_row(P.seqs, i);
    const SeqSpan sp = seq_span(P.seqs, s);
    const int pos = sp.kv - sp.q_len + (int)i - sp.q0;
    if (turn) turn_item(P, i, pos, c, it, bad);
    if (bad && P.seqs.status) P.seqs.status[s] = 5;  // GK_SEQ_POSITION
    uint8_t *dst;
    if (kind == 0) {
        dst = reinterpret_cast<uint8_t *>(P.q_out + (uint64_t)i * P.qo_tok + h * P.qo_head);
    } else {
        if (pos < 0) return;
        const uint32_t page = P.cache.by_T.div((uint32_t)pos);
        const int g = page_of(P, s, page);
        if (g < 0) return;
        dst = (kind == 1 ? P.cache.k : P.cache.v) + (uint64_t)g * P.cache.page +
              (uint64_t)((uint32_t)pos - page * P.cache.T) * P.cache.tok + (uint64_t)h * P.cache.head;
    }
    *reinterpret_cast<uint4 *>(dst + 2u * it.d0) = pack8(it.x);
    *reinterpret_cast<uint4 *>(dst + 2u * it.d1) = pack8(it.x + 8);
}

__device__ __forceinline__ float finite_size(float x)
{
    const float a = fabsf(x);
    return a <= 3.402823466e38f ? a : 0.f;  // false for infinities and NaN
}

__device__ __forceinline__ uint2 pack_e4m3(const float *x, float inv)
{
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint32_t h[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            float2 f = make_float2(__fmul_rn(x[4 * i + 2 * j], inv), __fmul_rn(x[4 * i + 2 * j + 1], inv));
            if (isinf(f.x)) f.x = __int_as_float(0x7fc00000);  // the conversion would store the largest value
            if (isinf(f.y)) f.y = __int_as_float(0x7fc00000);
            h[j] = __nv_cvt_float2_to_fp8x2(f, __NV_SATFINITE, __NV_E4M3);
        }
        w[i] = h[0] | (h[1] << 16);
    }
    return make_uint2(w[0], w[1]);
}

// e4m3 values times a power of two not above 1, rounded to nearest
__device__ __forceinline__ uint32_t rescale_e4m3(uint32_t w, float f)
{
    uint32_t out = 0;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w >> (16 * j)), __NV_E4M3);
        float2 v = __half22float2(__half2(h));
        v.x *= f;
        v.y *= f;
        out |= (uint32_t)__nv_cvt_float2_to_fp8x2(v, __NV_SATFINITE, __NV_E4M3) << (16 * j);
    }
    return out;
}

// The new scale of a page and head, and what earlier rows are multiplied by (1 if they keep their bytes).
__device__ __forceinline__ float grown_scale(float big, float old, bool has_rows, float &shrink)
{
    const bool kept = has_rows && old > 0.f && old <= 3.402823466e38f;
    const float base = kept ? old : 1.f;
    int k = 0;
    if (big > 0.f) {
        const uint32_t r = __float_as_uint(__fdiv_rn(big, __fmul_rn(448.f, base)));
        // least k with r <= 2^k; a quotient below the smallest normal number counts as that
        k = max((int)(r >> 23), 1) - 127 + ((r & 0x7fffffu) != 0u && (r >> 23) != 0u ? 1 : 0);
        k = min(max(k, -126), 127);
    }
    if (kept) k = max(k, 0);
    const float scale = __fmul_rn(base, __uint_as_float((uint32_t)(k + 127) << 23));
    shrink = kept ? exp2f((float)-k) : 0.f;
    return scale;
}

// fp8: one warp appends one head (K and V) of one page.  Two passes over the page's new rows (the second finds
// them in L1/L2): the largest value decides the scale before anything is stored.
__device__ __forceinline__ void append_unit(const AppendParams &P, uint32_t slot, uint32_t h, int lane)
{
    const uint32_t T = P.cache.T;
    uint32_t s, u;
    if (!P.seqs.q_start) {
        s = slot;
        u = 0;
    } else {
        // sequence s owns the slots from q_start[s]/T + 2s on: as many as its rows can touch pages
        uint32_t lo = 0, hi = P.seqs.n_seqs;
        while (hi - lo > 1u) {
            const uint32_t mid = (lo + hi) >> 1;
            const uint32_t q = (uint32_t)min(max(__ldg(P.seqs.q_start + mid), 0), (int)P.seqs.n_tokens);
            if (P.cache.by_T.div(q) + 2u * mid <= slot) lo = mid;
            else hi = mid;
        }
        s = lo;
        const uint32_t q = (uint32_t)min(max(__ldg(P.seqs.q_start + s), 0), (int)P.seqs.n_tokens);
        u = slot - (P.cache.by_T.div(q) + 2u * s);
    }
    const SeqSpan sp = seq_span(P.seqs, s);
    const int start = max(sp.kv - sp.q_len, 0);
    const uint32_t page = P.cache.by_T.div((uint32_t)start) + u;
    const int a = max(start, (int)(page * T)), b = min(sp.kv, (int)min((uint64_t)(page + 1u) * T, (uint64_t)0x7fffffff));
    if (a >= b || sp.q_len <= 0) return;
    const int g = page_of(P, s, page);
    if (g < 0) return;
    const uint32_t rows = (uint32_t)(b - a), fill = (uint32_t)a - page * T;
    const uint32_t i0 = (uint32_t)(sp.q0 + a - (sp.kv - sp.q_len));  // row of the first token
    const uint32_t n_items = rows * P.chunks;

    float big[2] = {0.f, 0.f};
    bool any_bad = false;
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
        for (uint32_t j = lane; j < n_items; j += 32u) {
            const uint32_t t = P.by_chunks.div(j), c = j - t * P.chunks;
            Item it;
            bool turn, bad = false;
            item_dims(P, c, kv == 0, it, turn);
            load_item(kv == 0 ? P.k : P.v, i0 + t, h, it);
            if (turn) turn_item(P, i0 + t, a + (int)t, c, it, bad);
            any_bad |= bad;
#pragma unroll
            for (int e = 0; e < 16; ++e) big[kv] = fmaxf(big[kv], finite_size(it.x[e]));
        }
        big[kv] = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(big[kv])));
    }
    if (any_bad && P.seqs.status) P.seqs.status[s] = 5;  // GK_SEQ_POSITION
    if (P.shared_scale) big[0] = big[1] = fmaxf(big[0], big[1]);

    float scale[2], shrink[2];
    scale[0] = grown_scale(big[0], P.cache.ks[(uint64_t)g * P.cache.s_page + h], fill > 0u, shrink[0]);
    if (P.shared_scale) {
        scale[1] = scale[0];
        shrink[1] = shrink[0];
    } else {
        scale[1] = grown_scale(big[1], P.cache.vs[(uint64_t)g * P.cache.s_page + h], fill > 0u, shrink[1]);
    }
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
        uint8_t *base = (kv ? P.cache.v : P.cache.k) + (uint64_t)g * P.cache.page + (uint64_t)h * P.cache.head;
        if (fill > 0u && shrink[kv] != 1.f) {
            for (uint32_t j = lane; j < fill * P.chunks; j += 32u) {
                const uint32_t t = P.by_chunks.div(j), c = j - t * P.chunks;
                uint4 *w = reinterpret_cast<uint4 *>(base + (uint64_t)t * P.cache.tok + 16u * c);
                uint4 x = *w;
                x.x = rescale_e4m3(x.x, shrink[kv]);
                x.y = rescale_e4m3(x.y, shrink[kv]);
                x.z = rescale_e4m3(x.z, shrink[kv]);
                x.w = rescale_e4m3(x.w, shrink[kv]);
                *w = x;
            }
        }
        const float inv = __fdiv_rn(1.f, scale[kv]);
        for (uint32_t j = lane; j < n_items; j += 32u) {
            const uint32_t t = P.by_chunks.div(j), c = j - t * P.chunks;
            Item it;
            bool turn, bad;
            item_dims(P, c, kv == 0, it, turn);
            load_item(kv == 0 ? P.k : P.v, i0 + t, h, it);
            if (turn) turn_item(P, i0 + t, a + (int)t, c, it, bad);
            uint8_t *dst = base + (uint64_t)(fill + t) * P.cache.tok;
            *reinterpret_cast<uint2 *>(dst + it.d0) = pack_e4m3(it.x, inv);
            *reinterpret_cast<uint2 *>(dst + it.d1) = pack_e4m3(it.x + 8, inv);
        }
    }
    __syncwarp();
    if (lane == 0) {
        P.cache.ks[(uint64_t)g * P.cache.s_page + h] = scale[0];
        if (!P.shared_scale) P.cache.vs[(uint64_t)g * P.cache.s_page + h] = scale[1];
    }
}

template <bool FP8>
__global__ void __launch_bounds__(kAppendThreads) append_kernel(const AppendParams P)
{
    uint32_t cta = blockIdx.x;
    if (FP8) {
        if (cta < P.unit_ctas) {
            const uint32_t slot = cta / P.head_groups;
            const uint32_t h = (cta - slot * P.head_groups) * kAppendWarps + (threadIdx.x >> 5);
            if (h < P.cache.H) append_unit(P, slot, h, threadIdx.x & 31);
            return;
        }
        cta -= P.unit_ctas;
    }
    append_flat<FP8>(P, cta * kAppendThreads + threadIdx.x);
}

}  // namespace gk
