// gk_attend.cuh -- attention of few rows over the paged cache (gk_attention): a few query rows per key
// head read the whole cache of their sequence once, so the kernel is bound by memory.
//
//   out = sum_t w_t V_t / sum_t w_t,  w_t = exp(scale * q.K_t - m)
//
// in one pass with a running maximum m: when it rises, what has been summed is multiplied by
// exp(m_old - m_new).
//
// Work.  An ITEM is (sequence, 16 query rows, key head); a query row is a (token, head of the group) pair, so
// the heads that share a key head share its loads.  An item's tokens are cut into tiles of 4 warps x TK
// tokens; the tiles of all items lie in one line, and every CTA takes an equal stretch of that
// line.  No length, ragged or not, leaves a part of the GPU idle.  A CTA's stretch may begin and end inside an
// item: the parts then go to the workspace, and the CTA that delivers an item's last part joins them in
// the order of the line.
//
// A warp works alone: its own ring of stages filled by its own 16-byte asynchronous copies, its own
// running maximum, sum and output; warps meet only at the end of an item.
#pragma once

#include "gk_seq.cuh"

namespace gk {

struct AttendParams {
    SeqsDev seqs;
    LayerDev cache;
    const __nv_bfloat16 *q;
    uint64_t q_tok, q_head;
    __nv_bfloat16 *out;
    uint64_t o_tok, o_head;
    float *lse;
    uint32_t Hq, G;    // query heads, query heads per key head
    FastDiv by_G;
    float scale_log2;  // scale * log2(e)
    uint32_t causal, window;
    uint32_t *counters;  // one per CTA: parts delivered of the item that begins in it and ends in a later one
    float *parts;        // two slots per CTA
};

constexpr int kAttendWarps = 4;
constexpr int kAttendThreads = 32 * kAttendWarps;
constexpr int kAttendStages = 3;
constexpr int kAttendRows = 16;

template <bool FP8, int DP>
struct AttendCfg {
    static constexpr int E = FP8 ? 1 : 2;
    static constexpr int TK = FP8 ? 32 : 16;         // tokens of a stage
    static constexpr int TILE = kAttendWarps * TK;   // tokens of a tile
    static constexpr int CPR = DP * E / 16;          // 16-byte pieces of a row
    static constexpr int KV_BYTES = TK * DP * E;
    static constexpr int SCALE_BYTES = FP8 ? 2 * TK * 4 : 0;
    static constexpr int STAGE_BYTES = 2 * KV_BYTES + SCALE_BYTES;
    static constexpr int PART_FLOATS = kAttendRows * DP + 2 * kAttendRows;  // outputs, maxima, sums
    static constexpr int SMEM = kAttendWarps * kAttendStages * STAGE_BYTES;
    static_assert(STAGE_BYTES >= kAttendRows * DP * 4, "a stage also holds a warp's output at an item's end");
};

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool take)
{
    const int n = take ? 16 : 0;  // 0 bytes read: 16 zeros written
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void *src, bool take)
{
    const int n = take ? 4 : 0;
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t a)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t a)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}

// D[16x8] += A[16x16] B[16x8], bf16 or f16 operands, fp32 accumulators
template <bool F16>
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if (F16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ float fast_exp2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ uint32_t bf16x2(float lo, float hi)
{
    const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&b);
}
__device__ __forceinline__ uint32_t f16x2(float lo, float hi)
{
    const __half2 b = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&b);
}
// two e4m3 values (the low half of w) as f16, exactly
__device__ __forceinline__ uint32_t e4m3_to_f16(uint32_t w)
{
    uint32_t r;
    asm("{ .reg .b16 t; cvt.u16.u32 t, %1; cvt.rn.f16x2.e4m3x2 %0, t; }" : "=r"(r) : "r"(w));
    return r;
}

// Where the 16-byte piece c of row r of a tile with CPR pieces per row lies: pieces are exchanged within a row so that
// the 8 rows of one ldmatrix, and the 4 lanes x 2 rows of one 16-byte read, fall on different banks.
template <int CPR>
__device__ __forceinline__ uint32_t piece(uint32_t r, uint32_t c)
{
    if (CPR >= 8) return (r * CPR + (c ^ (((r & 1u) << 2) | ((r >> 1) & 3u)))) * 16u;
    return (r * CPR + (c ^ ((r >> 1) & 3u))) * 16u;
}

// A sequence as this kernel walks it.
struct SeqWork {
    int q0, q_len, kv;  // rows, tokens
    int first;          // first token of the first tile
    int tiles;          // tiles of every item of the sequence
    int items;          // 16-row blocks x key heads
    bool bad;           // longer than its page table
};

template <int TILE>
__device__ __forceinline__ SeqWork seq_work(const AttendParams &P, uint32_t s)
{
    const SeqSpan sp = seq_span(P.seqs, s);
    SeqWork w;
    w.q0 = sp.q0;
    w.q_len = sp.q_len;
    w.kv = sp.kv;
    w.bad = (uint64_t)sp.kv > (uint64_t)P.seqs.max_pages * P.cache.T;
    w.items = (int)(((uint32_t)sp.q_len * P.G + (kAttendRows - 1)) / kAttendRows * P.cache.H);
    int lo = 0;
    if (P.window) lo = (int)max(0ll, (long long)sp.kv - sp.q_len + 1 - (long long)P.window);
    w.first = lo / TILE * TILE;
    w.tiles = w.bad ? 1 : max(1, (w.kv - w.first + TILE - 1) / TILE);  // an empty sequence still has its rows' zeros to write
    return w;
}

// A place in the line of tiles.
struct TilePos {
    uint32_t s;
    int item, tile;
    SeqWork w;
};

template <int TILE>
__device__ __forceinline__ void next_tile(const AttendParams &P, TilePos &c)
{
    if (++c.tile < c.w.tiles) return;
    c.tile = 0;
    if (++c.item < c.w.items) return;
    c.item = 0;
    do {
        if (++c.s >= P.seqs.n_seqs) return;
        c.w = seq_work<TILE>(P, c.s);
    } while (c.w.items == 0);
}

// Rows of a 16-row block and the tokens that any of them attends to.
struct BlockSpan {
    int row0;    // first row (token * G + head of the group)
    int h;       // key head
    int lo, hi;  // tokens that some row of the block attends to
    bool mixed;  // its rows do not all attend to the same tokens
};

__device__ __forceinline__ BlockSpan block_span(const AttendParams &P, const SeqWork &w, int item)
{
    BlockSpan b;
    const int blk = item / (int)P.cache.H;
    b.h = item - blk * (int)P.cache.H;
    b.row0 = blk * kAttendRows;
    const int rows = w.q_len * (int)P.G;
    const int j0 = (int)P.by_G.div((uint32_t)b.row0);
    const int j1 = (int)P.by_G.div((uint32_t)min(b.row0 + kAttendRows, rows) - 1u);
    const int at = w.kv - w.q_len;
    b.hi = P.causal ? max(0, at + j1 + 1) : w.kv;
    b.lo = P.window ? (int)max(0ll, (long long)at + j0 + 1 - (long long)P.window) : 0;
    b.mixed = j0 != j1 && (P.causal || P.window);
    return b;
}

// What a lane knows about "its" token of the next stage to be loaded.
struct TokenMeta {
    int64_t at;       // byte offset of the token's row from the layer's k or v, or -1: no token here
    uint32_t s_at;    // unused without scales
    bool bad;         // a page id that the table should have held is missing
};

template <bool FP8, int DP>
__device__ __forceinline__ TokenMeta token_meta(const AttendParams &P, const TilePos &c, int warp, int lane)
{
    using C = AttendCfg<FP8, DP>;
    TokenMeta m{-1, 0, c.w.bad};
    const int tok = c.w.first + c.tile * C::TILE + warp * C::TK + lane;
    const BlockSpan b = block_span(P, c.w, c.item);
    if (lane < C::TK && tok >= b.lo && tok < b.hi && !c.w.bad) {
        const uint32_t page = P.cache.by_T.div((uint32_t)tok);
        const int g = __ldg(P.seqs.page_table + (uint64_t)c.s * P.seqs.table_stride + page);
        if ((uint32_t)g < P.cache.num_pages) {
            m.at = (int64_t)((uint64_t)g * P.cache.page + (uint64_t)((uint32_t)tok - page * P.cache.T) * P.cache.tok +
                             (uint64_t)b.h * P.cache.head);
            m.s_at = (uint32_t)g;
        } else {
            m.bad = true;
        }
    }
    return m;
}

template <bool FP8, int DP>
__device__ __forceinline__ void load_stage(const AttendParams &P, uint32_t stage, const TokenMeta &m, int h, int lane)
{
    using C = AttendCfg<FP8, DP>;
    const uint32_t pieces = P.cache.D * C::E / 16u;
#pragma unroll
    for (int i = 0; i < C::TK * C::CPR / 32; ++i) {
        const uint32_t j = (uint32_t)lane + 32u * i, r = j / C::CPR, c = j % C::CPR;
        const int64_t at = __shfl_sync(0xffffffffu, m.at, (int)r);
        const bool take = at >= 0 && c < pieces;
        const uint64_t off = take ? (uint64_t)at + 16u * c : 0u;
        const uint32_t d = stage + piece<C::CPR>(r, c);
        copy16(d, P.cache.k + off, take);
        copy16(d + C::KV_BYTES, P.cache.v + off, take);
    }
    if (FP8 && lane < C::TK) {
        const uint64_t off = m.at >= 0 ? (uint64_t)m.s_at * P.cache.s_page + (uint32_t)h : 0u;
        copy4(stage + 2 * C::KV_BYTES + 4 * lane, P.cache.ks + off, m.at >= 0);
        copy4(stage + 2 * C::KV_BYTES + 4 * (C::TK + lane), P.cache.vs + off, m.at >= 0);
    }
}

// Rows g and g + 8 of a 16-row block, as a lane sees them.
struct LaneRows {
    int lo[2], hi[2];  // tokens that the row attends to (none: hi <= lo)
    float mul[2];      // scale * log2(e), times the row's power of two with f16 queries
};

template <bool FP8, int DP>
__device__ __forceinline__ void load_queries(const AttendParams &P, const SeqWork &w, const BlockSpan &b, int lane,
                                             uint32_t (&qa)[DP / 16][4], LaneRows &lr)
{
    const int g = lane >> 2, t = lane & 3;
    const int rows = w.q_len * (int)P.G, at = w.kv - w.q_len;
    const uint32_t D = P.cache.D;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int r = b.row0 + g + 8 * half;
        const bool live = r < rows;
        const uint32_t j = P.by_G.div((uint32_t)(live ? r : 0));
        const uint32_t head = (uint32_t)b.h * P.G + (uint32_t)((live ? r : 0) - (int)(j * P.G));
        const __nv_bfloat16 *p = P.q + (uint64_t)(w.q0 + j) * P.q_tok + (uint64_t)head * P.q_head;
        const int pos = at + (int)j;
        lr.hi[half] = !live ? 0 : P.causal ? max(0, pos + 1) : w.kv;
        lr.lo[half] = P.window ? (int)max(0ll, (long long)pos + 1 - (long long)P.window) : 0;
        lr.mul[half] = P.scale_log2;
        if (!FP8) {
            // k-step s, dimensions 16s + 2t, +1 and 16s + 8 + 2t, +1
#pragma unroll
            for (int s = 0; s < DP / 16; ++s)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t d = 16u * s + 8u * e + 2u * t;
                    qa[s][half + 2 * e] = live && d < D ? __ldg(reinterpret_cast<const uint32_t *>(p + d)) : 0u;
                }
        } else {
            // A lane's 16-byte pieces of a key row are 16 consecutive dimensions, so queries are dealt out
            // alike (the order of the dimensions in a dot product is free): k-step 4j + s takes dimensions
            // 64j + 16t + 4s ..+3.  bf16 queries become f16 after a division by the row's power of two: exact
            // but for values 2^-14 below the row's largest.
            uint32_t raw[DP / 16][2];
            uint32_t top = 0;
#pragma unroll
            for (int s = 0; s < DP / 16; ++s) {
                const uint32_t d = 64u * (s / 4) + 16u * t + 4u * (s % 4);
                uint2 u = make_uint2(0u, 0u);
                if (live && d < D) u = __ldg(reinterpret_cast<const uint2 *>(p + d));
                raw[s][0] = u.x;
                raw[s][1] = u.y;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t a = raw[s][e] & 0x7fffu, c = (raw[s][e] >> 16) & 0x7fffu;
                    if (a < 0x7f80u) top = max(top, a);
                    if (c < 0x7f80u) top = max(top, c);
                }
            }
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const int ex = min(max((int)(top >> 7) - 127, -126), 126);
            const float down = __uint_as_float((uint32_t)(127 - ex) << 23);
            lr.mul[half] *= __uint_as_float((uint32_t)(127 + ex) << 23);
#pragma unroll
            for (int s = 0; s < DP / 16; ++s)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    qa[s][half + 2 * e] = f16x2(__uint_as_float(raw[s][e] << 16) * down,
                                                __uint_as_float(raw[s][e] & 0xffff0000u) * down);
        }
    }
}

// A warp's running state of one item.
template <int DP>
struct Running {
    float o[DP / 8][4];
    float m[2], l[2];  // rows g, g + 8; l is this lane's share of the sum
    float vref;        // fp8: outputs are held divided by this, the largest value scale seen
};

// f16 weights are multiplied by 2^12 so that small ones keep their bits; outputs carry the factor until the end.
constexpr float kWeightUp = 4096.f;

// Dimension of element e of accumulator n, for lane position t.
template <bool FP8>
__device__ __forceinline__ int out_dim(int n, int e, int t)
{
    // fp8: accumulators 2i and 2i + 1 hold the even and the odd dimensions of 16i ..+15
    if (FP8) return 16 * (n >> 1) + 2 * (2 * t + (e & 1)) + (n & 1);
    return 8 * n + 2 * t + (e & 1);
}

// Does a stage's V hold an infinity or NaN?
template <bool FP8, int DP>
__device__ __forceinline__ bool values_not_finite(const uint8_t *v, int lane)
{
    using C = AttendCfg<FP8, DP>;
    bool found = false;
    for (int i = lane; i < C::KV_BYTES / 4; i += 32) {
        const uint32_t w = *reinterpret_cast<const uint32_t *>(v + 4 * i);
        if (FP8) found |= __vcmpeq4(w & 0x7f7f7f7fu, 0x7f7f7f7fu) != 0u;
        else found |= (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
    }
    return __any_sync(0xffffffffu, found);
}

template <bool FP8, int DP>
__device__ __forceinline__ void add_values_by_element(const uint8_t *v, const float (&s)[AttendCfg<FP8, DP>::TK / 8][4],
                                                      Running<DP> &R, int lane)
{
    using C = AttendCfg<FP8, DP>;
    const int t = lane & 3;
#pragma unroll
    for (int n8 = 0; n8 < C::TK / 8; ++n8)
#pragma unroll 1
        for (int k = 0; k < 8; ++k) {
            float w[2];
#pragma unroll
            for (int half = 0; half < 2; ++half)
                w[half] = __shfl_sync(0xffffffffu, (k & 1) ? s[n8][1 + 2 * half] : s[n8][2 * half], (lane & ~3) | (k >> 1));
#pragma unroll
            for (int n = 0; n < DP / 8; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int d = out_dim<FP8>(n, e, t) * C::E;
                    const uint8_t *p = v + piece<C::CPR>(8 * n8 + k, d / 16) + d % 16;
                    float x;
                    if (FP8) x = __half2float(__half(__nv_cvt_fp8_to_halfraw(*p, __NV_E4M3)));
                    else x = __bfloat162float(*reinterpret_cast<const __nv_bfloat16 *>(p));
                    if (w[e >> 1] != 0.f) R.o[n][e] += w[e >> 1] * x;
                }
        }
}

template <bool FP8, int DP>
__device__ __forceinline__ void attend_stage(const AttendParams &P, uint32_t stage, const uint8_t *stage_ptr, int tok0,
                                             const uint32_t (&qa)[DP / 16][4], const LaneRows &lr, Running<DP> &R, bool mixed, int lane)
{
    using C = AttendCfg<FP8, DP>;
    const int t = lane & 3;
    float s[C::TK / 8][4];
#pragma unroll
    for (int n = 0; n < C::TK / 8; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[n][e] = 0.f;
    // scores
#pragma unroll
    for (int n = 0; n < C::TK / 8; ++n) {
        if (!FP8) {
            const uint32_t r = 8u * n + (lane & 7);
#pragma unroll
            for (int k = 0; k < DP / 32; ++k) {
                uint32_t b[4];
                ldmatrix4(b, stage + piece<C::CPR>(r, 4u * k + (lane >> 3)));
                mma16816<false>(s[n], qa[2 * k], b[0], b[1]);
                mma16816<false>(s[n], qa[2 * k + 1], b[2], b[3]);
            }
        } else {
            const uint32_t r = 8u * n + (lane >> 2);
#pragma unroll
            for (int j = 0; j < DP / 64; ++j) {
                const uint4 u = *reinterpret_cast<const uint4 *>(stage_ptr + piece<C::CPR>(r, 4u * j + t));
                const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    mma16816<true>(s[n], qa[4 * j + k], e4m3_to_f16(w[k]), e4m3_to_f16(w[k] >> 16));
            }
        }
    }
    // scale, mask, running maximum
    const float *scales = reinterpret_cast<const float *>(stage_ptr + 2 * C::KV_BYTES);
    float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int n = 0; n < C::TK / 8; ++n) {
        float ks[2] = {1.f, 1.f};
        if (FP8) {
            const float2 f = *reinterpret_cast<const float2 *>(scales + 8 * n + 2 * t);
            ks[0] = f.x;
            ks[1] = f.y;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int half = e >> 1, tok = tok0 + 8 * n + 2 * t + (e & 1);
            float x = s[n][e] * lr.mul[half];
            if (FP8) x *= ks[e & 1];
            if (tok < lr.lo[half] || tok >= lr.hi[half]) x = -INFINITY;
            s[n][e] = x;
            top[half] = fmaxf(top[half], x);
        }
    }
    float vtop = 0.f;
    if (FP8) {
        vtop = lane < C::TK ? fabsf(scales[C::TK + lane]) : 0.f;
        if (!(vtop <= 3.402823466e38f)) vtop = 0.f;  // a scale that is no number counts only where it is used
        vtop = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(vtop)));
    }
    bool rise = FP8 && vtop > R.vref;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        top[half] = fmaxf(top[half], __shfl_xor_sync(0xffffffffu, top[half], 1));
        top[half] = fmaxf(top[half], __shfl_xor_sync(0xffffffffu, top[half], 2));
        rise |= top[half] > R.m[half];
    }
    if (__any_sync(0xffffffffu, rise)) {
        float down_v = 1.f;
        if (FP8 && vtop > R.vref) {
            down_v = R.vref / vtop;
            R.vref = vtop;
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const float m = fmaxf(R.m[half], top[half]);
            const float down = m == R.m[half] ? 1.f : fast_exp2(R.m[half] - m);
            R.m[half] = m;
            R.l[half] *= down;
#pragma unroll
            for (int n = 0; n < DP / 8; ++n) {
                R.o[n][2 * half] *= down * down_v;
                R.o[n][2 * half + 1] *= down * down_v;
            }
        }
    }
    // weights
    const float ref[2] = {R.m[0] == -INFINITY ? 0.f : R.m[0], R.m[1] == -INFINITY ? 0.f : R.m[1]};
    const float up = FP8 ? (R.vref > 0.f ? kWeightUp / R.vref : 0.f) : 1.f;
#pragma unroll
    for (int n = 0; n < C::TK / 8; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            s[n][e] = fast_exp2(s[n][e] - ref[e >> 1]);
            R.l[e >> 1] += s[n][e];
        }
    if (FP8) {
#pragma unroll
        for (int n = 0; n < C::TK / 8; ++n) {
            const float2 f = *reinterpret_cast<const float2 *>(scales + C::TK + 8 * n + 2 * t);
            const float v0 = f.x * up, v1 = f.y * up;
            // a token that a row does not attend to stays 0 whatever its scale is
            s[n][0] = s[n][0] == 0.f ? 0.f : s[n][0] * v0;
            s[n][1] = s[n][1] == 0.f ? 0.f : s[n][1] * v1;
            s[n][2] = s[n][2] == 0.f ? 0.f : s[n][2] * v0;
            s[n][3] = s[n][3] == 0.f ? 0.f : s[n][3] * v1;
        }
    }
    // outputs
    const uint32_t vbase = stage + C::KV_BYTES;
    if (mixed && values_not_finite<FP8, DP>(stage_ptr + C::KV_BYTES, lane)) {
        // 0 * infinity would reach rows that do not attend to the token: element by element, by weight
        add_values_by_element<FP8, DP>(stage_ptr + C::KV_BYTES, s, R, lane);
        return;
    }
#pragma unroll
    for (int k = 0; k < C::TK / 16; ++k) {
        const uint32_t r = 16u * k + (lane & 15);
        if (!FP8) {
            // a weight goes in as its upper 16 bits and the bf16 of the rest: rounding weights to 8 bits would add as much
            // error as the rounding of the result, and the tensor pipe has the time.  Neither part is negative, nor 0
            // unless the weight is, so that an infinite V stays what it is.
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float a = s[2 * k + (e >> 1)][2 * (e & 1)], b = s[2 * k + (e >> 1)][2 * (e & 1) + 1];
                hi[e] = __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632);
                const float la = a - __uint_as_float(__float_as_uint(a) & 0xffff0000u);
                const float lb = b - __uint_as_float(__float_as_uint(b) & 0xffff0000u);
                lo[e] = bf16x2(fmaxf(la, a * 0x1p-24f), fmaxf(lb, b * 0x1p-24f));
            }
#pragma unroll
            for (int n = 0; n < DP / 16; ++n) {
                uint32_t b[4];
                ldmatrix4_trans(b, vbase + piece<C::CPR>(r, 2u * n + (lane >> 4)));
                mma16816<false>(R.o[2 * n], hi, b[0], b[1]);
                mma16816<false>(R.o[2 * n], lo, b[0], b[1]);
                mma16816<false>(R.o[2 * n + 1], hi, b[2], b[3]);
                mma16816<false>(R.o[2 * n + 1], lo, b[2], b[3]);
            }
        } else {
            uint32_t a[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) a[e] = f16x2(s[2 * k + (e >> 1)][2 * (e & 1)], s[2 * k + (e >> 1)][2 * (e & 1) + 1]);
            // transposing 16-bit pairs of e4m3 values: a register holds dimensions 2g, 2g + 1 of token 2t, then of
            // token 2t + 1; its bytes 0, 2 and 1, 3 are the operands for the even and the odd dimensions
#pragma unroll
            for (int n = 0; n < DP / 32; ++n) {
                uint32_t b[4];
                ldmatrix4_trans(b, vbase + piece<C::CPR>(r, 2u * n + (lane >> 4)));
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t x = __byte_perm(b[2 * e], 0, 0x3120), y = __byte_perm(b[2 * e + 1], 0, 0x3120);
                    mma16816<true>(R.o[4 * n + 2 * e], a, e4m3_to_f16(x), e4m3_to_f16(y));
                    mma16816<true>(R.o[4 * n + 2 * e + 1], a, e4m3_to_f16(x >> 16), e4m3_to_f16(y >> 16));
                }
            }
        }
    }
}

template <int DP>
__device__ __forceinline__ void write_row_piece(const AttendParams &P, const SeqWork &w, const BlockSpan &b, int row, int d,
                                                const float4 &v)
{
    const int r = b.row0 + row;
    const uint32_t j = P.by_G.div((uint32_t)r);
    const uint32_t head = (uint32_t)b.h * P.G + (uint32_t)(r - (int)(j * P.G));
    if (d < (int)P.cache.D)
        *reinterpret_cast<uint2 *>(P.out + (uint64_t)(w.q0 + j) * P.o_tok + (uint64_t)head * P.o_head + d) =
            make_uint2(bf16x2(v.x, v.y), bf16x2(v.z, v.w));
}

__device__ __forceinline__ void write_lse(const AttendParams &P, const SeqWork &w, const BlockSpan &b, int row, float m, float l)
{
    const int r = b.row0 + row;
    const uint32_t j = P.by_G.div((uint32_t)r);
    const uint32_t head = (uint32_t)b.h * P.G + (uint32_t)(r - (int)(j * P.G));
    if (P.lse) P.lse[(uint64_t)(w.q0 + j) * P.Hq + head] = l == 0.f ? -INFINITY : m * 0.69314718055994531f + logf(l);
}

template <bool FP8, int DP>
__global__ void __launch_bounds__(kAttendThreads, DP <= 128 ? 2 : 1) attend_kernel(const AttendParams P)
{
    using C = AttendCfg<FP8, DP>;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ long long sh_total[kAttendWarps];
    __shared__ long long sh_at;
    __shared__ uint32_t sh_seq;
    __shared__ float sh_m[kAttendWarps][kAttendRows], sh_l[kAttendWarps][kAttendRows];
    __shared__ uint32_t sh_last;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    // the length of the line of tiles, and where this CTA's stretch of it begins
    long long total = 0;
    for (uint32_t s0 = 0; s0 < P.seqs.n_seqs; s0 += kAttendThreads) {
        long long n = 0;
        if (s0 + tid < P.seqs.n_seqs) {
            const SeqWork w = seq_work<C::TILE>(P, s0 + tid);
            n = (long long)w.items * w.tiles;
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) n += __shfl_xor_sync(0xffffffffu, n, o);
        if (lane == 0) sh_total[warp] = n;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kAttendWarps; ++i) total += sh_total[i];
        __syncthreads();
    }
    if (total == 0) return;
    const long long ctas = total < (long long)gridDim.x ? total : (long long)gridDim.x;
    if ((long long)blockIdx.x >= ctas) return;
    const long long begin = total * blockIdx.x / ctas, end = total * (blockIdx.x + 1) / ctas;
    {
        long long before = 0;
        for (uint32_t s0 = 0; s0 < P.seqs.n_seqs; s0 += kAttendThreads) {
            long long n = 0;
            if (s0 + tid < P.seqs.n_seqs) {
                const SeqWork w = seq_work<C::TILE>(P, s0 + tid);
                n = (long long)w.items * w.tiles;
            }
            long long incl = n;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long x = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += x;
            }
            if (lane == 31) sh_total[warp] = incl;
            __syncthreads();
            long long base = before;
            for (int i = 0; i < warp; ++i) base += sh_total[i];
            const long long lo = base + incl - n;
            if (n > 0 && begin >= lo && begin < lo + n) {
                sh_seq = s0 + tid;
                sh_at = lo;
            }
            for (int i = 0; i < kAttendWarps; ++i) before += sh_total[i];
            __syncthreads();
            if (before > begin) break;
        }
    }

    TilePos comp;
    comp.s = sh_seq;
    comp.w = seq_work<C::TILE>(P, comp.s);
    {
        const long long off = begin - sh_at;
        comp.item = (int)(off / comp.w.tiles);
        comp.tile = (int)(off - (long long)comp.item * comp.w.tiles);
    }
    TilePos load = comp;  // runs ahead of comp
    const int n_tiles = (int)(end - begin);
    const uint32_t ring = smem_addr(smem) + warp * kAttendStages * C::STAGE_BYTES;
    const uint8_t *ring_ptr = smem + warp * kAttendStages * C::STAGE_BYTES;

    TokenMeta meta = token_meta<FP8, DP>(P, load, warp, lane);
    uint32_t bad_stages = 0;  // bit s: the load in stage s met a missing page
    int loaded = 0;
    auto issue = [&](int stage) {
        if (loaded < n_tiles) {
            const int h = load.item % (int)P.cache.H;
            load_stage<FP8, DP>(P, ring + stage * C::STAGE_BYTES, meta, h, lane);
            const bool bad = __any_sync(0xffffffffu, meta.bad);
            bad_stages = (bad_stages & ~(1u << stage)) | ((bad ? 1u : 0u) << stage);
            if (bad && lane == 0 && P.seqs.status) P.seqs.status[load.s] = 2;  // GK_JOB_PAGE_TABLE
            if (++loaded < n_tiles) {
                next_tile<C::TILE>(P, load);
                meta = token_meta<FP8, DP>(P, load, warp, lane);
            }
        }
        copy_commit();
    };
#pragma unroll
    for (int i = 0; i < kAttendStages; ++i) issue(i);

    uint32_t qa[DP / 16][4];
    LaneRows lr;
    Running<DP> R;
    BlockSpan b;
    bool fresh = true;
    int stage = 0;
    const int g = lane >> 2, t = lane & 3;
    long long item_first = begin - comp.tile;  // place of the item's first tile in the line
    for (int n = 0; n < n_tiles; ++n) {
        if (fresh) {
            b = block_span(P, comp.w, comp.item);
            load_queries<FP8, DP>(P, comp.w, b, lane, qa, lr);
#pragma unroll
            for (int i = 0; i < DP / 8; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) R.o[i][e] = 0.f;
            R.m[0] = R.m[1] = -INFINITY;
            R.l[0] = R.l[1] = 0.f;
            R.vref = 0.f;
            fresh = false;
        }
        copy_wait<kAttendStages - 1>();
        __syncwarp();
        attend_stage<FP8, DP>(P, ring + stage * C::STAGE_BYTES, ring_ptr + stage * C::STAGE_BYTES,
                              comp.w.first + comp.tile * C::TILE + warp * C::TK, qa, lr, R, b.mixed, lane);
        if ((bad_stages >> stage) & 1u) R.l[0] = R.l[1] = __int_as_float(0x7fc00000);
        __syncwarp();
        const bool item_ends = comp.tile + 1 == comp.w.tiles;
        if (item_ends || n + 1 == n_tiles) {
            // the four warps' results meet: each in the stage that it has just used up
            float *mine = reinterpret_cast<float *>(smem + (warp * kAttendStages + stage) * C::STAGE_BYTES);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                R.l[half] += __shfl_xor_sync(0xffffffffu, R.l[half], 1);
                R.l[half] += __shfl_xor_sync(0xffffffffu, R.l[half], 2);
                if (t == 0) {
                    sh_m[warp][g + 8 * half] = R.m[half];
                    sh_l[warp][g + 8 * half] = R.l[half];
                }
            }
            const float back = FP8 ? R.vref * (1.f / kWeightUp) : 1.f;
#pragma unroll
            for (int i = 0; i < DP / 8; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    mine[(g + 8 * (e >> 1)) * DP + out_dim<FP8>(i, e, t)] = R.o[i][e] * back;
            __syncthreads();
            const bool whole = item_ends && item_first >= begin;
            const int rows = min(kAttendRows, comp.w.q_len * (int)P.G - b.row0);
            const bool starts_before = item_first < begin;
            float *part = P.parts + (uint64_t)(2u * blockIdx.x + (starts_before ? 0u : 1u)) * C::PART_FLOATS;
            for (int i = tid; i < rows * (DP / 4); i += kAttendThreads) {
                const int row = i / (DP / 4), d = 4 * (i - row * (DP / 4));
                float m = sh_m[0][row];
#pragma unroll
                for (int w = 1; w < kAttendWarps; ++w) m = fmaxf(m, sh_m[w][row]);
                const float ref = m == -INFINITY ? 0.f : m;
                float l = 0.f;
                float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < kAttendWarps; ++w) {
                    const float f = fast_exp2(sh_m[w][row] - ref);
                    const float4 x = *reinterpret_cast<const float4 *>(
                        smem + (w * kAttendStages + stage) * C::STAGE_BYTES + (row * DP + d) * 4);
                    l += f * sh_l[w][row];
                    v.x += f * x.x;
                    v.y += f * x.y;
                    v.z += f * x.z;
                    v.w += f * x.w;
                }
                if (whole) {
                    const float inv = l == 0.f ? 0.f : 1.f / l;
                    write_row_piece<DP>(P, comp.w, b, row, d, make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv));
                    if (d == 0) write_lse(P, comp.w, b, row, m, l);
                } else {
                    *reinterpret_cast<float4 *>(part + row * DP + d) = v;
                    if (d == 0) {
                        part[kAttendRows * DP + row] = m;
                        part[kAttendRows * DP + kAttendRows + row] = l;
                    }
                }
            }
            if (!whole) {
                // the CTAs that share the item: those whose stretches hold its first and its last tile
                const long long item_last = item_first + comp.w.tiles - 1;
                const uint32_t c0 = (uint32_t)(((item_first + 1) * ctas - 1) / total);
                const uint32_t c1 = (uint32_t)(((item_last + 1) * ctas - 1) / total);
                __threadfence();
                __syncthreads();
                if (tid == 0) {
                    const uint32_t seen = atomicAdd(P.counters + c0, 1u);
                    sh_last = seen == c1 - c0;
                    if (seen == c1 - c0) P.counters[c0] = 0u;  // ready for the next call
                }
                __syncthreads();
                if (sh_last) {
                    __threadfence();
                    for (int i = tid; i < rows * (DP / 4); i += kAttendThreads) {
                        const int row = i / (DP / 4), d = 4 * (i - row * (DP / 4));
                        float m = -INFINITY, l = 0.f;
                        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
                        for (uint32_t c = c0; c <= c1; ++c) {
                            const float *p = P.parts + (uint64_t)(2u * c + (c == c0 ? 1u : 0u)) * C::PART_FLOATS;
                            const float pm = __ldcg(p + kAttendRows * DP + row), pl = __ldcg(p + kAttendRows * DP + kAttendRows + row);
                            const float4 x = __ldcg(reinterpret_cast<const float4 *>(p + row * DP + d));
                            const float nm = fmaxf(m, pm), ref = nm == -INFINITY ? 0.f : nm;
                            const float a = fast_exp2(m - ref), f = fast_exp2(pm - ref);
                            l = a * l + f * pl;
                            v.x = a * v.x + f * x.x;
                            v.y = a * v.y + f * x.y;
                            v.z = a * v.z + f * x.z;
                            v.w = a * v.w + f * x.w;
                            m = nm;
                        }
                        const float inv = l == 0.f ? 0.f : 1.f / l;
                        write_row_piece<DP>(P, comp.w, b, row, d, make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv));
                        if (d == 0) write_lse(P, comp.w, b, row, m, l);
                    }
                }
            }
            __syncthreads();
            fresh = true;
        }
        issue(stage);
        stage = stage + 1 == kAttendStages ? 0 : stage + 1;
        if (n + 1 < n_tiles) {
            if (item_ends) item_first += comp.w.tiles;
            next_tile<C::TILE>(P, comp);
        }
    }
    copy_wait<0>();
}

}  // namespace gk
