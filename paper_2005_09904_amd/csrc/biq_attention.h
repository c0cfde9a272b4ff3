// Attention over the paged 8-bit cache (biq_attention).
//
//   s_t = scale q.k_t,  m = max s_t,  l = sum exp(s_t - m),  o = (1/l) sum exp(s_t - m) v_t
//
// in one pass over the tokens with a running m, l and o.  A wave takes 64 tokens (4 blocks of 16) at a time and computes the
// transposed products, so that nothing crosses lanes between the two of them:
//   S^T = K Q^T   4 tiles of 16 tokens x 16 rows.  Row m of tile t is token 16 (m / 4) + 4 t + m % 4, so that the 16 sums of a
//                 lane (16 x 16 x 32 MFMA: lane l holds column l % 16, rows 4 (l / 16) ..) are the 16 tokens of block l / 16:
//                 one scale per lane for the keys, one for the values.
//   O^T = V^T P^T The lane's probabilities are the right operand as they lie (k index 8 (l / 16) + j of step h is token
//                 16 (l / 16) + 8 h + j), and the left operand wants the 16 tokens of block l / 16 at one element: 16 adjacent
//                 bytes of the cache's value layout.
// The order of the elements along k of Q K^T is free as well: a lane reads 16 adjacent bytes of a key.
#pragma once

#include "biq_serve.h"

namespace biq {

struct AttendParams {
    Cache cache;
    Ragged ragged;
    Rows q, out;
    float* lse;
    float* part;             // splits > 1: [row * q_heads + head][split][dim] sums, then [..][split][2] maximum and sum
    long long part_stats;    // floats before the maxima
    int q_heads, group, causal, window;
    int units;               // seqs * heads * splits
    int splits, split_tokens, row_tiles;
    float scale;             // scale * log2(e)
};

// Tokens that a tile of rows sees, in whole steps of 64: [base, end).
struct TokenSpan { int base, end; };
__device__ __forceinline__ TokenSpan token_span(const AttendParams& p, int len, int pos_first, int pos_last) {
    TokenSpan t;
    int lo = p.window > 0 ? pos_first - p.window + 1 : 0;
    lo = lo < 0 ? 0 : lo;
    t.base = lo & ~63;
    t.end = p.causal ? pos_last + 1 : len;
    t.end = t.end < t.base ? t.base : t.end;
    return t;
}
// Splits of that span that have tokens (one at least).  The last split takes what is left, whatever the length.
__device__ __forceinline__ int active_splits(const AttendParams& p, TokenSpan t) {
    const int n = (t.end - t.base + p.split_tokens - 1) / p.split_tokens;
    return n < 1 ? 1 : n > p.splits ? p.splits : n;
}

// Terms of 8 floats as bf16, each the upper half of what is left (the last one rounded): 8 bits of significand a term.
template <int TERMS>
__device__ __forceinline__ void bf16_terms(const float (&x)[8], bf16x8 (&out)[TERMS]) {
    float r[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) r[j] = x[j];
#pragma unroll
    for (int t = 0; t < TERMS; ++t) {
        union { bf16x8 v; uint32_t w[4]; } o;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (t == TERMS - 1) {
                union { bf16x2 v; uint32_t w; } c;
                c.v = __builtin_convertvector((f32x2){r[2 * j], r[2 * j + 1]}, bf16x2);
                o.w[j] = c.w;
            } else {
                o.w[j] = __builtin_amdgcn_perm(__float_as_uint(r[2 * j + 1]), __float_as_uint(r[2 * j]), 0x07060302);
                r[2 * j] -= __uint_as_float(__float_as_uint(r[2 * j]) & 0xffff0000u);
                r[2 * j + 1] -= __uint_as_float(__float_as_uint(r[2 * j + 1]) & 0xffff0000u);
            }
        }
        out[t] = o.v;
    }
}

template <int TYPE>
__device__ __forceinline__ void load_q8(const Rows& q, long long at, float (&x)[8]) {
    if (q.quads) {
        const f32x4 a = load_elem4<TYPE>(q.data, at), b = load_elem4<TYPE>(q.data, at + 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) { x[j] = a[j]; x[4 + j] = b[j]; }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = load_elem<TYPE>(q.data, at + j);
    }
}

template <int TYPE> struct AttendTerms { static constexpr int value = TYPE == BIQ_F32 ? 3 : TYPE == BIQ_F16 ? 2 : 1; };

__device__ __forceinline__ float exp2_raw(float x) { return __builtin_amdgcn_exp2f(x); }

// Few rows of a sequence and head (one token with its heads, drafted tokens).  The waves of a workgroup hold the same rows and take
// steps of 64 tokens in turn, straight from memory to registers: every code is used by one wave only.  The waves' sums are
// joined through LDS.  CH: 64 elements of a head each; NT: tiles of 16 rows.
template <int TYPE, int FMT, int CH, int NT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void attend_rows_kernel(const AttendParams p) {
    constexpr int TERMS = AttendTerms<TYPE>::value;
    constexpr int ROWS = 16 * NT;
    extern __shared__ float lds[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int col = lane & 15, grp = lane >> 4;
    // row tiles of a unit follow each other on one XCD: they read the same tokens
    const int xcd = blockIdx.x % kXcds, at = blockIdx.x / kXcds;
    const int unit = at / p.row_tiles * kXcds + xcd, tile = at % p.row_tiles;
    if (unit >= p.units) return;
    const int split = unit % p.splits, head = unit / p.splits % p.cache.heads, seq = unit / p.splits / p.cache.heads;
    const int2 range = p.ragged.range(seq);
    const int len = p.cache.length(seq);
    const int rows_here = range.y * p.group - tile * ROWS;      // (token, head of the group), heads fastest
    if (rows_here <= 0) return;
    const int i_first = tile * ROWS / p.group;
    const int i_last = (tile * ROWS + (rows_here < ROWS ? rows_here : ROWS) - 1) / p.group;
    const int pos0 = len - range.y;                             // token of row 0 (negative: before the first token)
    const TokenSpan span = token_span(p, len, pos0 + i_first, pos0 + i_last);
    const int splits_here = active_splits(p, span);
    if (split >= splits_here) return;
    const int begin = span.base + split * p.split_tokens;
    const int end = split == splits_here - 1 ? span.end : begin + p.split_tokens;

    const int dim = p.cache.dim;
    // rows of this lane's columns, and what they see
    long long row_of[NT];
    int head_of[NT], lo[NT], hi[NT];
    bf16x8 q[NT][CH][2][TERMS];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int rr = tile * ROWS + n * 16 + col;
        const bool there = n * 16 + col < rows_here;
        const int i = rr / p.group;
        row_of[n] = there ? range.x + i : -1;
        head_of[n] = head * p.group + (rr - i * p.group);
        hi[n] = p.causal ? pos0 + i : len - 1;
        lo[n] = p.window > 0 ? pos0 + i - p.window + 1 : 0;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                const int d = c * 64 + grp * 16 + h * 8;
                if (there && d < dim) load_q8<TYPE>(p.q, row_of[n] * p.q.row_stride + head_of[n] * p.q.head_stride + d, x);
                bf16_terms<TERMS>(x, q[n][c][h]);
            }
    }
    // tokens that every row of the tile sees
    const int all_lo = p.window > 0 ? pos0 + i_last - p.window + 1 : 0;
    const int all_hi = p.causal ? pos0 + i_first : len - 1;

    f32x4 o[NT][CH * 4];
    float m[NT], l[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        m[n] = -INFINITY;
        l[n] = 0.f;
#pragma unroll
        for (int t = 0; t < CH * 4; ++t) o[n][t] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }

    const long long codes = p.cache.codes_bytes();
    const int kblock = col >> 2;                                // block of this lane's key rows, 0 .. 3
    // key rows of the lane in tile t: token 4 t + col % 4 of its block
    u32x4 kc[4][CH];
    float ks = 0.f, vs = 0.f;
    const uint8_t* vbase = p.cache.store;
    int valid = 0;

    auto locate_and_load_keys = [&](int t0) {
        const int kb = (t0 >> 4) + kblock, vb = (t0 >> 4) + grp;
        const int kp = p.cache.page_number(seq, kb), vp = p.cache.page_number(seq, vb);
        // (without a page: codes of page 0, hidden below)
        const uint8_t* kbase = p.cache.page(kp < 0 ? 0 : kp) + static_cast<long long>(p.cache.block_in_page(kb, head)) * (kCacheBlock * dim);
        const uint8_t* page = p.cache.page(vp < 0 ? 0 : vp);
        const int vblock = p.cache.block_in_page(vb, head);
        vbase = page + codes + static_cast<long long>(vblock) * (kCacheBlock * dim);
        const float* scales = reinterpret_cast<const float*>(page + 2 * codes) + vblock;
        valid = vp < 0 ? 0 : len - vb * kCacheBlock;
        valid = valid < 0 ? 0 : valid > kCacheBlock ? kCacheBlock : valid;
        ks = valid ? scales[0] : 0.f;
        vs = valid ? scales[p.cache.heads * p.cache.page_blocks] : 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            int d = c * 64 + grp * 16;
            d = d < dim ? d : 0;                                // (against zeros of q)
#pragma unroll
            for (int t = 0; t < 4; ++t)
                kc[t][c] = *reinterpret_cast<const u32x4*>(kbase + (4 * t + (col & 3)) * dim + d);
        }
    };

    int t0 = begin + wave * 64;
    if (t0 < end) locate_and_load_keys(t0);
    for (; t0 < end; t0 += 64 * WAVES) {
        // values of this step
        u32x4 vc[CH * 4];
#pragma unroll
        for (int t = 0; t < CH * 4; ++t) {
            const int d = t * 16 < dim ? t * 16 + col : col;    // (beyond the head: sums that are not stored)
            vc[t] = *reinterpret_cast<const u32x4*>(vbase + d * kCacheBlock);
        }
        const float kscale = ks * p.scale, vscale = vs;
        const int nvalid = valid;
        // scores
        f32x4 s[NT][4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
            for (int n = 0; n < NT; ++n) s[n][t] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const bf16x8 k = codes_bf16<FMT>(kc[t][c][2 * h], kc[t][c][2 * h + 1]);
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < TERMS; ++e)
                            s[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[n][c][h][e], s[n][t], 0, 0, 0);
                }
        }
        // keys of the next step
        const int tn = t0 + 64 * WAVES;
        if (tn < end) locate_and_load_keys(tn);

        const bool whole = t0 + 63 <= all_hi && t0 >= all_lo && __all(nvalid == kCacheBlock);
        if (!whole) {
            // codes of tokens that the sequence does not have may be anything
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int left = nvalid - 4 * w;                // tokens of this dword
                const uint32_t mask = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
#pragma unroll
                for (int t = 0; t < CH * 4; ++t) vc[t][w] &= mask;
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int first = t0 + grp * kCacheBlock;           // token of the lane's sum 0
            float x[16];
            float top = -INFINITY;
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                x[j] = s[n][j >> 2][j & 3] * kscale;
                if (!whole && (first + j < lo[n] || first + j > hi[n] || j >= nvalid)) x[j] = -INFINITY;
                top = fmaxf(top, x[j]);
            }
            const float now = fmaxf(m[n], max_over_groups(top));
            const float ref = now == -INFINITY ? 0.f : now;     // (nothing seen yet)
            const float keep = exp2_raw(m[n] - ref);
            m[n] = now;
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const bool seen = whole || x[j] != -INFINITY;
                const float e = exp2_raw(x[j] - ref);
                sum += e;
                x[j] = seen ? e * vscale : 0.f;                 // (a hidden token's scale may be NaN)
            }
            l[n] = l[n] * keep + sum;
#pragma unroll
            for (int t = 0; t < CH * 4; ++t) o[n][t] *= keep;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float y[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = x[8 * h + j];
                bf16x8 pt[TERMS];
                bf16_terms<TERMS>(y, pt);
#pragma unroll
                for (int t = 0; t < CH * 4; ++t) {
                    const bf16x8 v = codes_bf16<FMT>(vc[t][2 * h], vc[t][2 * h + 1]);
#pragma unroll
                    for (int e = 0; e < TERMS; ++e)
                        o[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pt[e], o[n][t], 0, 0, 0);
                }
            }
        }
    }

    // ---- the waves' sums, joined -------------------------------------------------------------------
    float top[NT], total[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        total[n] = sum_over_groups(l[n]);
        top[n] = m[n];
    }
    if constexpr (WAVES > 1) {
        float* stats = lds;                                     // [wave][ROWS][2]
        float* slots = lds + WAVES * ROWS * 2;                  // [WAVES / 2][NT * CH * 4][64][4]
#pragma unroll
        for (int n = 0; n < NT; ++n)
            if (grp == 0) {
                stats[(wave * ROWS + n * 16 + col) * 2] = m[n];
                stats[(wave * ROWS + n * 16 + col) * 2 + 1] = total[n];
            }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float t = -INFINITY;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) t = fmaxf(t, stats[(w * ROWS + n * 16 + col) * 2]);
            const float ref = t == -INFINITY ? 0.f : t;
            float sum = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w)
                sum += stats[(w * ROWS + n * 16 + col) * 2 + 1] * exp2_raw(stats[(w * ROWS + n * 16 + col) * 2] - ref);
            const float f = exp2_raw(m[n] - ref);
            top[n] = t;
            total[n] = sum;
#pragma unroll
            for (int i = 0; i < CH * 4; ++i) o[n][i] *= f;
        }
        // halves of the waves are added, over and over
        for (int half = WAVES / 2; half > 0; half /= 2) {
            if (half < WAVES / 2) __syncthreads();
            if (wave >= half && wave < 2 * half) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < CH * 4; ++i)
                        *reinterpret_cast<f32x4*>(slots + (((wave - half) * NT + n) * (CH * 4) + i) * 256 + lane * 4) = o[n][i];
            }
            __syncthreads();
            if (wave < half) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < CH * 4; ++i)
                        o[n][i] += *reinterpret_cast<const f32x4*>(slots + ((wave * NT + n) * (CH * 4) + i) * 256 + lane * 4);
            }
        }
        if (wave != 0) return;
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        if (row_of[n] < 0) continue;
        const long long rh = row_of[n] * p.q_heads + head_of[n];
        if (p.splits > 1) {
            float* part = p.part + (rh * p.splits + split) * dim;
#pragma unroll
            for (int i = 0; i < CH * 4; ++i)
                if (i * 16 < dim) *reinterpret_cast<f32x4*>(part + i * 16 + grp * 4) = o[n][i];
            if (grp == 0) {
                float* st = p.part + p.part_stats + (rh * p.splits + split) * 2;
                st[0] = top[n];
                st[1] = total[n];
            }
            continue;
        }
        const float inv = total[n] == 0.f ? 0.f : 1.f / total[n];
        const long long to = row_of[n] * p.out.row_stride + head_of[n] * p.out.head_stride + grp * 4;
#pragma unroll
        for (int i = 0; i < CH * 4; ++i)
            if (i * 16 < dim) {
                const f32x4 r = o[n][i] * inv;
                if (p.out.quads) store_elem4<TYPE>(p.out.data, to + i * 16, r);
                else
#pragma unroll
                    for (int j = 0; j < 4; ++j) store_elem<TYPE>(p.out.data, to + i * 16 + j, r[j]);
            }
        if (p.lse && grp == 0) p.lse[rh] = total[n] == 0.f ? -INFINITY : (top[n] + __log2f(total[n])) * 0.69314718055994531f;
    }
}

// The splits of a row's tokens, joined: 16 lanes a row and head, elements 4 lane, 4 lane + 64, ..
template <int TYPE>
__global__ __launch_bounds__(256) void attend_join_kernel(const AttendParams p, int tile_rows) {
    const long long rh = (static_cast<long long>(blockIdx.x) * 256 + threadIdx.x) >> 4;
    const int lane = threadIdx.x & 15;
    if (rh >= static_cast<long long>(p.ragged.rows) * p.q_heads) return;
    const int row = static_cast<int>(rh / p.q_heads), head = static_cast<int>(rh - static_cast<long long>(row) * p.q_heads);
    // the row's sequence
    const int seqs = p.units / (p.cache.heads * p.splits);
    int seq;
    if (!p.ragged.starts) {
        seq = row / p.ragged.max_rows;
    } else {
        int a = 0, e = seqs;                                    // last sequence that starts at or before the row
        while (e - a > 1) {
            const int mid = (a + e) / 2;
            if (p.ragged.starts[mid] <= row) a = mid; else e = mid;
        }
        seq = a;
    }
    const int2 range = p.ragged.range(seq);
    const int i = row - range.x;
    if (i < 0 || i >= range.y) return;                          // a row of no sequence
    const int len = p.cache.length(seq), pos0 = len - range.y;
    // the tile of rows that it was computed in
    const int tile = (i * p.group + head % p.group) / tile_rows;
    const int last = (tile + 1) * tile_rows < range.y * p.group ? (tile + 1) * tile_rows : range.y * p.group;
    const TokenSpan span = token_span(p, len, pos0 + tile * tile_rows / p.group, pos0 + (last - 1) / p.group);
    const int n = active_splits(p, span);
    const float* st = p.part + p.part_stats + rh * p.splits * 2;
    float top = -INFINITY;
    for (int k = 0; k < n; ++k) top = fmaxf(top, st[2 * k]);
    const float ref = top == -INFINITY ? 0.f : top;
    float total = 0.f;
    for (int k = 0; k < n; ++k) total += st[2 * k + 1] * exp2_raw(st[2 * k] - ref);
    const float inv = total == 0.f ? 0.f : 1.f / total;
    const float* part = p.part + rh * p.splits * p.cache.dim;
    for (int d = lane * 4; d < p.cache.dim; d += 64) {
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        for (int k = 0; k < n; ++k)
            acc += *reinterpret_cast<const f32x4*>(part + static_cast<long long>(k) * p.cache.dim + d) * exp2_raw(st[2 * k] - ref);
        acc *= inv;
        const long long to = row * p.out.row_stride + head * p.out.head_stride + d;
        if (p.out.quads) store_elem4<TYPE>(p.out.data, to, acc);
        else
#pragma unroll
            for (int j = 0; j < 4; ++j) store_elem<TYPE>(p.out.data, to + j, acc[j]);
    }
    if (p.lse && lane == 0) p.lse[rh] = total == 0.f ? -INFINITY : (top + __log2f(total)) * 0.69314718055994531f;
}

}  // namespace biq
