// The cache's writer and reader (biq_cache_append, biq_cache_read).
//
// A wave has one block of 16 tokens of one head, keys or values.  Its lanes hold what they write: of the keys 16 adjacent
// elements of a token, of the values the 16 tokens at one element, 16 bytes of codes either way, so the codes that are there
// already come with one load to the lanes that may have to round them anew.
//
// The writer waits for loads that depend on each other (lengths, rows, page, angles; a wave lives 8 us): 10300 tokens of 8 heads of
// 128 (bf16 to fp8, 63 MB) take 25 us, 2.5 TB/s, one token of 64 sequences 7 us.  The reader is bound by its writes: 105 MB (to
// fp32) take 20.5 us, 5.1 TB/s.
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

// 16 and 2 adjacent elements of a row.
template <int TYPE>
__device__ __forceinline__ void load16(const Rows& src, long long at, float (&x)[16]) {
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
        if (src.quads) {
            const f32x4 q = load_elem4<TYPE>(src.data, at + e);
#pragma unroll
            for (int f = 0; f < 4; ++f) x[e + f] = q[f];
        } else {
#pragma unroll
            for (int f = 0; f < 4; ++f) x[e + f] = load_elem<TYPE>(src.data, at + e + f);
        }
    }
}
template <int TYPE>
__device__ __forceinline__ f32x2 load2(const Rows& src, long long at) {
    typedef typename Elem<TYPE>::T V __attribute__((ext_vector_type(2), aligned(4)));
    if (src.quads) return __builtin_convertvector(*reinterpret_cast<const V*>(static_cast<const typename Elem<TYPE>::T*>(src.data) + at), f32x2);
    return (f32x2){load_elem<TYPE>(src.data, at), load_elem<TYPE>(src.data, at + 1)};
}

// Elements d0 .. d0 + 15 of a key turned by the angles of its position (row `at` of src).
template <int TYPE>
__device__ __forceinline__ void turn16(const Rows& src, long long at, const Rotation& r, int pos, int d0, float (&x)[16]) {
    const int rot = r.rot, half = rot / 2;
    if (d0 >= rot) return;
    const bool known = pos < r.positions;
    const float* angles = r.angles + static_cast<long long>(known ? pos : 0) * rot;
    if (r.interleaved) {
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
            if (d0 + e >= rot) continue;
            const f32x2 cs = *reinterpret_cast<const f32x2*>(angles + d0 + e);
            const float a = x[e], b = x[e + 1];
            x[e] = turned(a, b, cs[0], cs[1], false);
            x[e + 1] = turned(b, a, cs[0], cs[1], true);
        }
    } else if (half % 16 == 0) {                                // partners are 16 adjacent elements as well
        const bool second = d0 >= half;
        const int p0 = second ? d0 - half : d0;
        float y[16];
        load16<TYPE>(src, at + (second ? p0 : d0 + half), y);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const f32x2 cs = *reinterpret_cast<const f32x2*>(angles + 2 * (p0 + e));
            x[e] = turned(x[e], y[e], cs[0], cs[1], second);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int d = d0 + e;
            if (d >= rot) continue;
            const bool second = d >= half;
            const int pair = second ? d - half : d;
            x[e] = turned(x[e], load_elem<TYPE>(src.data, at + (second ? pair : d + half)), angles[2 * pair], angles[2 * pair + 1], second);
        }
    }
    if (!known)
#pragma unroll
        for (int e = 0; e < 16; ++e)
            if (d0 + e < rot) x[e] = __uint_as_float(0x7fc00000u);
}

__device__ __forceinline__ uint32_t most_bits(const float (&x)[16], uint32_t bits) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const uint32_t u = __float_as_uint(x[i]) & 0x7fffffffu;
        bits = bits > u ? bits : u;
    }
    return bits;
}

// A block of a sequence: tokens [0, old) are there, [old, end) are new.  find() looks up where it lies (codes stays NULL where
// there is no page); the new rows are requested before.
struct BlockPlace {
    const Cache& cache;
    int seq, b, head;
    bool values;
    long long first;         // element of the source's token 0 of the block
    int t0, old, end;
    uint8_t* codes;
    float* scale;
    __device__ __forceinline__ bool find() {
        const int number = cache.page_number(seq, b);
        if (number < 0) return false;
        uint8_t* page = cache.page(number);
        const int block = cache.block_in_page(b, head);
        const long long all = cache.codes_bytes();
        codes = page + (values ? all : 0) + static_cast<long long>(block) * (kCacheBlock * cache.dim);
        scale = reinterpret_cast<float*>(page + 2 * all) + (values ? cache.heads * cache.page_blocks : 0) + block;
        return true;
    }
};

// Keys: lane n has unit n % units (16 elements) of token n / units.
template <int TYPE, int FMT, int CH>
__device__ __forceinline__ void append_keys(const AppendParams& p, BlockPlace& b, int lane, int dim) {
    const int units = dim / 16;
    float x[CH][16];
    u32x4 there[CH];
    uint32_t bits = 0;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int n = lane + 64 * c, i = n / units, d0 = (n - i * units) * 16;
#pragma unroll
        for (int e = 0; e < 16; ++e) x[c][e] = 0.f;
        if (i >= b.old && i < b.end) load16<TYPE>(p.k, b.first + i * p.k.row_stride + d0, x[c]);
    }
    if (!b.find()) return;
    const float old_scale = b.old > 0 ? *b.scale : 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int n = lane + 64 * c;
        there[c] = (u32x4){0u, 0u, 0u, 0u};
        if (b.old > 0 && n < dim) there[c] = *reinterpret_cast<const u32x4*>(b.codes + n * 16);
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int n = lane + 64 * c, i = n / units, d0 = (n - i * units) * 16;
        if (p.rotation.angles && i >= b.old && i < b.end) turn16<TYPE>(p.k, b.first + i * p.k.row_stride, p.rotation, b.t0 + i, d0, x[c]);
        bits = most_bits(x[c], bits);
    }
    const BlockScale s = block_scale<FMT>(max_over_wave(bits), old_scale);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int n = lane + 64 * c, i = n / units;
        if (n >= dim) continue;
        *reinterpret_cast<u32x4*>(b.codes + n * 16) = encode16<FMT>(x[c], there[c], i >= b.old && i < b.end ? 0xffffu : 0u, i < b.old ? 0xffffu : 0u, s);
    }
    if (lane == 0) *b.scale = s.scale;
}

// Values: lane n has the 16 tokens at elements 2 n and 2 n + 1 (so that a row is read 4 or 8 bytes a lane).
template <int TYPE, int FMT, int CH>
__device__ __forceinline__ void append_values(const AppendParams& p, BlockPlace& b, int lane, int dim) {
    constexpr int PARTS = (CH + 1) / 2;
    float x[PARTS][2][16];
    u32x4 there[PARTS][2];
    uint32_t bits = 0;
#pragma unroll
    for (int c = 0; c < PARTS; ++c) {
        const int d = 2 * (lane + 64 * c);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            f32x2 v = {0.f, 0.f};
            if (i >= b.old && i < b.end && d < dim) v = load2<TYPE>(p.v, b.first + i * p.v.row_stride + d);
            x[c][0][i] = v[0];
            x[c][1][i] = v[1];
        }
    }
    if (!b.find()) return;
    const float old_scale = b.old > 0 ? *b.scale : 0.f;
#pragma unroll
    for (int c = 0; c < PARTS; ++c)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int d = 2 * (lane + 64 * c);
            there[c][h] = (u32x4){0u, 0u, 0u, 0u};
            if (b.old > 0 && d < dim) there[c][h] = *reinterpret_cast<const u32x4*>(b.codes + (d + h) * 16);
        }
#pragma unroll
    for (int c = 0; c < PARTS; ++c) bits = most_bits(x[c][1], most_bits(x[c][0], bits));
    const BlockScale s = block_scale<FMT>(max_over_wave(bits), old_scale);
    const uint32_t is_old = (1u << b.old) - 1u, is_new = ((1u << b.end) - 1u) & ~is_old;
#pragma unroll
    for (int c = 0; c < PARTS; ++c) {
        const int d = 2 * (lane + 64 * c);
        if (d >= dim) continue;
#pragma unroll
        for (int h = 0; h < 2; ++h)
            *reinterpret_cast<u32x4*>(b.codes + (d + h) * 16) = encode16<FMT>(x[c][h], there[c][h], is_new, is_old, s);
    }
    if (lane == 0) *b.scale = s.scale;
}

template <int TYPE, int FMT, int CH>
__global__ __launch_bounds__(256) void cache_append_kernel(const AppendParams p) {
    const int lane = threadIdx.x & 63;
    // (sequence, block) pairs and, four waves of a workgroup, the heads' keys and values
    const int kinds = 2 * p.cache.heads, parts = (kinds + 3) / 4;
    const int pair = blockIdx.x / parts, kind = (blockIdx.x - pair * parts) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int seq = pair / p.blocks, j = pair - seq * p.blocks;
    if (kind >= kinds) return;
    const int head = kind >> 1;
    const int2 range = p.ragged.range(seq);
    const int len = p.cache.length(seq), pos0 = len - range.y;
    const int b = (pos0 < 0 ? 0 : pos0) / kCacheBlock + j, t0 = b * kCacheBlock;
    if (range.y <= 0 || t0 >= len) return;
    const bool values = kind & 1;
    const Rows& src = values ? p.v : p.k;
    const int dim = p.cache.dim;
    BlockPlace at = {p.cache, seq, b, head, values,
                     (range.x + static_cast<long long>(t0 - pos0)) * src.row_stride + head * src.head_stride, t0,
                     pos0 - t0 < 0 ? 0 : pos0 - t0, len - t0 < kCacheBlock ? len - t0 : kCacheBlock, nullptr, nullptr};
    if (values) append_values<TYPE, FMT, CH>(p, at, lane, dim);
    else append_keys<TYPE, FMT, CH>(p, at, lane, dim);
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
    const int kinds = 2 * p.cache.heads, parts = (kinds + 3) / 4;
    const int pair = blockIdx.x / parts, kind = (blockIdx.x - pair * parts) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int seq = pair / p.blocks, j = pair - seq * p.blocks;
    if (kind >= kinds) return;
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
