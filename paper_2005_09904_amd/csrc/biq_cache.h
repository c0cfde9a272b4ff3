// The cache's writer and reader (biq_cache_append, biq_cache_read).
//
// A wave has one block of 16 tokens of one head, keys or values.  Its lanes hold what they write: of the keys 16 adjacent
// elements of a token, of the values the 16 tokens at one element, 16 bytes of codes either way, so the codes that are there
// already come with one load to the lanes that may have to round them anew.
#pragma once

#include "biq_serve.h"

namespace biq {

struct Rotation {
    const float* angles;     // NULL: none
    int positions, rot, interleaved;
};

// Element d of a turned row: x[d], its partner and the sign of its sine.  a c - b s and a s + b c, each operation rounded.
__device__ __forceinline__ float turned(float x, float partner, float c, float s, bool second) {
#pragma clang fp contract(off)
    const float xc = x * c, ps = partner * s;
    return second ? ps + xc : xc - ps;
}

struct AppendParams {
    Cache cache;
    Ragged ragged;
    Rows k, v;
    Rotation rotation;
    int seqs, blocks;        // blocks: the most that a sequence's rows can touch
};

// The block's new scale and the factors for new values and old codes.  bits: largest magnitude of the new values as an integer
// (NaN and infinities above all numbers).
struct BlockScale { float scale, fresh, kept; };
template <int FMT>
__device__ __forceinline__ BlockScale block_scale(uint32_t bits, float old) {
    const float amax = __uint_as_float(bits);
    float scale;
    if constexpr (FMT == BIQ_CACHE_INT8) {
        scale = amax / 127.0f;
    } else {
        // 448 = 1.75 * 2^8: exponent - 8, one more for a larger significand
        const uint32_t e = (bits >> 23) - 8u + ((bits & 0x7fffffu) > 0x600000u ? 1u : 0u);
        scale = __uint_as_float(e << 23);
    }
    if (bits < 0x0d800000u) scale = 0.f;                        // below 2^-100
    scale = scale > old ? scale : old;
    BlockScale r;
    if (bits >= 0x7f800000u || old != old) {
        r.scale = __uint_as_float(0x7fc00000u);
        r.fresh = r.kept = 0.f;
    } else {
        r.scale = scale;
        r.fresh = scale > 0.f ? 1.0f / scale : 0.f;
        r.kept = scale > 0.f ? old / scale : 0.f;
    }
    return r;
}

__device__ __forceinline__ uint32_t max_over_wave(uint32_t x) {
#pragma unroll
    for (int d = 32; d > 0; d /= 2) {
        const uint32_t y = __shfl_xor(x, d);
        x = x > y ? x : y;
    }
    return x;
}

// 16 values and 16 old codes -> 16 codes.  fresh: which are new; the others before `old` tokens are kept.
template <int FMT>
__device__ __forceinline__ u32x4 encode16(const float (&x)[16], u32x4 codes, uint32_t fresh, uint32_t old, BlockScale s) {
    u32x4 out;
    float y[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        y[0] = code_value<FMT, 0>(codes[w]);
        y[1] = code_value<FMT, 1>(codes[w]);
        y[2] = code_value<FMT, 2>(codes[w]);
        y[3] = code_value<FMT, 3>(codes[w]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t bit = 1u << (4 * w + i);
            y[i] = (fresh & bit) ? x[4 * w + i] * s.fresh : (old & bit) ? y[i] * s.kept : 0.f;
        }
        out[w] = s.scale != s.scale ? 0u : encode4<FMT>(y[0], y[1], y[2], y[3]);
    }
    return out;
}

template <int TYPE, int FMT, int CH>
__global__ __launch_bounds__(256) void cache_append_kernel(const AppendParams p) {
    const int lane = threadIdx.x & 63;
    const int kinds = 2 * p.cache.heads;
    const long long unit = static_cast<long long>(blockIdx.x) * 4 + (threadIdx.x >> 6);
    const int kind = static_cast<int>(unit % kinds);
    const int j = static_cast<int>(unit / kinds % p.blocks), seq = static_cast<int>(unit / kinds / p.blocks);
    if (seq >= p.seqs) return;
    const int head = kind >> 1;
    const bool values = kind & 1;
    const int2 range = p.ragged.range(seq);
    const int len = p.cache.length(seq), pos0 = len - range.y;
    const int b = (pos0 < 0 ? 0 : pos0) / kCacheBlock + j, t0 = b * kCacheBlock;
    if (range.y <= 0 || t0 >= len) return;
    const int number = p.cache.page_number(seq, b);
    if (number < 0) return;
    uint8_t* page = p.cache.page(number);
    const int block = p.cache.block_in_page(b, head), dim = p.cache.dim;
    const long long codes = p.cache.codes_bytes();
    uint8_t* base = page + (values ? codes : 0) + static_cast<long long>(block) * (kCacheBlock * dim);
    float* scale_at = reinterpret_cast<float*>(page + 2 * codes) + (values ? p.cache.heads * p.cache.page_blocks : 0) + block;
    // tokens of the block: [0, old) are there, [old, end) are new
    int old = pos0 - t0, end = len - t0;
    old = old < 0 ? 0 : old;
    end = end > kCacheBlock ? kCacheBlock : end;
    const float old_scale = old > 0 ? *scale_at : 0.f;
    const Rows& src = values ? p.v : p.k;
    const long long first = (range.x + static_cast<long long>(t0 - pos0)) * src.row_stride + head * src.head_stride;   // token t0

    float x[CH][16];
    u32x4 there[CH];
    uint32_t bits = 0;
    const int units = dim / 16;                                 // of a token
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int n = lane + 64 * c;                            // keys: unit n % units of token n / units; values: element n
        there[c] = (u32x4){0u, 0u, 0u, 0u};
#pragma unroll
        for (int i = 0; i < 16; ++i) x[c][i] = 0.f;
        if (n >= dim) continue;
        if (old > 0) there[c] = *reinterpret_cast<const u32x4*>(base + n * 16);
        if (values) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (i >= old && i < end) x[c][i] = load_elem<TYPE>(src.data, first + i * src.row_stride + n);
        } else {
            const int i = n / units, d0 = (n - i * units) * 16;
            if (i >= old && i < end) {
                const long long at = first + i * src.row_stride;
#pragma unroll
                for (int e = 0; e < 16; e += 4) {
                    if (src.quads) {
                        const f32x4 q = load_elem4<TYPE>(src.data, at + d0 + e);
#pragma unroll
                        for (int f = 0; f < 4; ++f) x[c][e + f] = q[f];
                    } else {
#pragma unroll
                        for (int f = 0; f < 4; ++f) x[c][e + f] = load_elem<TYPE>(src.data, at + d0 + e + f);
                    }
                }
                const int rot = p.rotation.rot;
                if (p.rotation.angles && d0 < rot) {
                    const int pos = t0 + i, half = rot / 2;
                    const bool known = pos < p.rotation.positions;
                    const float* angles = p.rotation.angles + static_cast<long long>(known ? pos : 0) * rot;
#pragma unroll
                    for (int e = 0; e < 16; e += 2) {
                        // elements d, d + 1 of the head
                        const int d = d0 + e;
                        if (d >= rot) continue;
                        float a = x[c][e], b2 = x[c][e + 1];
                        if (p.rotation.interleaved) {
                            const f32x2 cs = *reinterpret_cast<const f32x2*>(angles + d);
                            x[c][e] = turned(a, b2, cs[0], cs[1], false);
                            x[c][e + 1] = turned(b2, a, cs[0], cs[1], true);
                        } else {
#pragma unroll
                            for (int f = 0; f < 2; ++f) {
                                const int df = d + f;                                   // (< rot: rot is even)
                                const bool second = df >= half;
                                const int pair = second ? df - half : df;
                                const float partner = load_elem<TYPE>(src.data, at + (second ? pair : df + half));
                                x[c][e + f] = turned(x[c][e + f], partner, angles[2 * pair], angles[2 * pair + 1], second);
                            }
                        }
                        if (!known) x[c][e] = x[c][e + 1] = __uint_as_float(0x7fc00000u);
                    }
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint32_t u = __float_as_uint(x[c][i]) & 0x7fffffffu;
            bits = bits > u ? bits : u;
        }
    }
    const BlockScale s = block_scale<FMT>(max_over_wave(bits), old_scale);
    const uint32_t is_old = (1u << old) - 1u, is_new = ((1u << end) - 1u) & ~is_old;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int n = lane + 64 * c;
        if (n >= dim) continue;
        uint32_t mine_old = is_old, mine_new = is_new;
        if (!values) {                                          // one token in all 16 codes
            const int i = n / units;
            mine_old = (is_old >> i) & 1u ? 0xffffu : 0u;
            mine_new = (is_new >> i) & 1u ? 0xffffu : 0u;
        }
        *reinterpret_cast<u32x4*>(base + n * 16) = encode16<FMT>(x[c], there[c], mine_new, mine_old, s);
    }
    if (lane == 0) *scale_at = s.scale;
}

struct ReadParams {
    Cache cache;
    Ragged ragged;
    Rows k, v;
    int seqs, blocks;
};

template <int TYPE, int FMT, int CH>
__global__ __launch_bounds__(256) void cache_read_kernel(const ReadParams p) {
    const int lane = threadIdx.x & 63;
    const int kinds = 2 * p.cache.heads;
    const long long unit = static_cast<long long>(blockIdx.x) * 4 + (threadIdx.x >> 6);
    const int kind = static_cast<int>(unit % kinds);
    const int j = static_cast<int>(unit / kinds % p.blocks), seq = static_cast<int>(unit / kinds / p.blocks);
    if (seq >= p.seqs) return;
    const int head = kind >> 1;
    const bool values = kind & 1;
    const int2 range = p.ragged.range(seq);
    const int len = p.cache.length(seq), pos0 = len - range.y;
    const int b = (pos0 >> 4) + j;                              // (rounded down: below 0 before the first token)
    const long long t0 = static_cast<long long>(b) * kCacheBlock;
    if (range.y <= 0 || t0 >= len) return;
    const int number = b < 0 ? -1 : p.cache.page_number(seq, b);
    const int dim = p.cache.dim;
    const uint8_t* base = nullptr;
    float scale = 0.f;
    if (number >= 0) {
        const uint8_t* page = p.cache.page(number);
        const int block = p.cache.block_in_page(b, head);
        const long long codes = p.cache.codes_bytes();
        base = page + (values ? codes : 0) + static_cast<long long>(block) * (kCacheBlock * dim);
        scale = reinterpret_cast<const float*>(page + 2 * codes)[(values ? p.cache.heads * p.cache.page_blocks : 0) + block];
    }
    const Rows& dst = values ? p.v : p.k;
    const long long first = (range.x + (t0 - pos0)) * dst.row_stride + head * dst.head_stride;
    const int from = pos0 > t0 ? static_cast<int>(pos0 - t0) : 0;
    const int to = len - t0 < kCacheBlock ? static_cast<int>(len - t0) : kCacheBlock;
    const int units = dim / 16;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int n = lane + 64 * c;
        if (n >= dim) continue;
        float x[16];
        u32x4 w = {0u, 0u, 0u, 0u};
        if (base) w = *reinterpret_cast<const u32x4*>(base + n * 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[4 * i] = code_value<FMT, 0>(w[i]) * scale;
            x[4 * i + 1] = code_value<FMT, 1>(w[i]) * scale;
            x[4 * i + 2] = code_value<FMT, 2>(w[i]) * scale;
            x[4 * i + 3] = code_value<FMT, 3>(w[i]) * scale;
        }
        if (!base)
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = 0.f;
        if (values) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (i >= from && i < to) store_elem<TYPE>(dst.data, first + i * dst.row_stride + n, x[i]);
        } else {
            const int i = n / units, d0 = (n - i * units) * 16;
            if (i < from || i >= to) continue;
            const long long at = first + i * dst.row_stride + d0;
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                if (dst.quads) store_elem4<TYPE>(dst.data, at + e, (f32x4){x[e], x[e + 1], x[e + 2], x[e + 3]});
                else
#pragma unroll
                    for (int f = 0; f < 4; ++f) store_elem<TYPE>(dst.data, at + e + f, x[e + f]);
            }
        }
    }
}

}  // namespace biq
