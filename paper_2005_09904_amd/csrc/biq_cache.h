// The cache's writer and reader (biq_cache_append, biq_cache_read).
//
// A wave has one block of 16 tokens of one head, keys or values.  Its lanes hold what they write: of the keys 16 adjacent
// elements of a token, of the values the 16 tokens at one element, 16 bytes of codes either way, so the codes that are there
// already come with one load to the lanes that may have to round them anew.
//
// The writer waits for loads that depend on each other (lengths, page; then rows, angles and codes, all requested before the first
// is used: 17.5 us instead of 26): 8755 tokens of 8 heads of 128 (bf16 to fp8, 54 MB) take 17.5 us, 3.1 TB/s, one token of 64
// sequences 6.2 us.  The reader is bound by its writes where there are many: 90 MB (to fp32) take 20.8 us, 4.3 TB/s.
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
    unsigned first;          // first workgroup of this launch
};

// The block's new scale and the factors for new values and old codes.  bits: largest magnitude of the new values as an integer
// (NaN and infinities above all numbers).
struct BlockScale { float scale, fresh, kept; };
template <int FMT>
__device__ __forceinline__ BlockScale block_scale(uint32_t bits, float old) {
    const float amax = __uint_as_float(bits);
    float scale;
    if constexpr (FMT == BIQ_CACHE_INT8) {
        // a product with the rounded constant, as biq.h says: what a division by 127 becomes in tensor programs on GPUs, so that their
        // codes and these agree where x / scale is halfway between two (the correctly rounded quotient differs in its last bit now and then)
        scale = amax * (1.0f / 127.0f);
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

// Largest of a wave's numbers: within rows of 16 lanes, then over the rows' ends; lane 63 has it.
__device__ __forceinline__ uint32_t max_over_wave(uint32_t x) {
    auto with = [&](int y) { x = x > static_cast<uint32_t>(y) ? x : static_cast<uint32_t>(y); };
    with(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), 0x111, 0xf, 0xf, true));       // row_shr:1, 2, 4, 8
    with(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), 0x112, 0xf, 0xf, true));
    with(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), 0x114, 0xf, 0xf, true));
    with(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), 0x118, 0xf, 0xf, true));
    with(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), 0x142, 0xa, 0xf, false));      // row_bcast:15 to rows 1 and 3
    with(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), 0x143, 0xc, 0xf, false));      // row_bcast:31 to rows 2 and 3
    return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(x), 63));
}

// The bytes of 16 codes whose bit is set; zeros for the others.
__device__ __forceinline__ u32x4 chosen_codes(u32x4 codes, uint32_t bits) {
#pragma unroll
    for (int w = 0; w < 4; ++w) codes[w] &= ((bits >> (4 * w) & 15u) * 0x00204081u & 0x01010101u) * 255u;
    return codes;
}

// 16 values and 16 codes -> 16 codes.  fresh: the values that count; the others are +0, as are the codes of these.
template <int FMT>
__device__ __forceinline__ u32x4 encode16(const float (&x)[16], u32x4 codes, uint32_t fresh, BlockScale s) {
    u32x4 out;
    float y[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        y[0] = code_value<FMT, 0>(codes[w]);
        y[1] = code_value<FMT, 1>(codes[w]);
        y[2] = code_value<FMT, 2>(codes[w]);
        y[3] = code_value<FMT, 3>(codes[w]);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            y[i] = __uint_as_float(__float_as_uint(y[i]) | __float_as_uint(x[4 * w + i])) * ((fresh >> (4 * w + i) & 1u) ? s.fresh : s.kept);
        out[w] = s.scale != s.scale ? 0u : encode4<FMT>(y[0], y[1], y[2], y[3]);
    }
    return out;
}

// Elements d0 .. d0 + 15 of a key (raw; row `at` of src) turned by the angles of its position.
template <int TYPE>
__device__ __forceinline__ void turn16(const Rows& src, long long at, const Rotation& r, int pos, int d0, bool used, const Elems<TYPE, 16>& raw, float (&x)[16]) {
    const int rot = r.rot, half = rot / 2;
    if (!r.angles || d0 >= rot || !used) {
        raw.get(x, used);
        return;
    }
    const bool known = pos < r.positions;
    const float* angles = r.angles + static_cast<long long>(known ? pos : 0) * rot;
    if (r.interleaved) {
        f32x2 cs[8];
#pragma unroll
        for (int e = 0; e < 16; e += 2) cs[e / 2] = *reinterpret_cast<const f32x2*>(angles + (d0 + e < rot ? d0 + e : d0));
        raw.get(x, true);
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
            if (d0 + e >= rot) continue;
            const float a = x[e], b = x[e + 1];
            x[e] = turned(a, b, cs[e / 2][0], cs[e / 2][1], false);
            x[e + 1] = turned(b, a, cs[e / 2][0], cs[e / 2][1], true);
        }
    } else if (half % 16 == 0) {                                // partners are 16 adjacent elements as well
        const bool second = d0 >= half;
        const int p0 = second ? d0 - half : d0;
        Elems<TYPE, 16> partners;
        partners.request(static_cast<const typename Elem<TYPE>::T*>(src.data) + at + (second ? p0 : d0 + half));
        f32x2 cs[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) cs[e] = *reinterpret_cast<const f32x2*>(angles + 2 * (p0 + e));
        raw.get(x, true);
        float y[16];
        partners.get(y, true);
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = turned(x[e], y[e], cs[e][0], cs[e][1], second);
    } else {
        raw.get(x, true);
#pragma unroll
        for (int q = 0; q < 16; q += 4) {                       // (four at a time: registers)
            Elems<TYPE, 1> partners[4];
            f32x2 cs[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int d = d0 + q + e < rot ? d0 + q + e : d0, pair = d < half ? d : d - half;
                partners[e].request(static_cast<const typename Elem<TYPE>::T*>(src.data) + at + (d < half ? d + half : pair));
                cs[e] = *reinterpret_cast<const f32x2*>(angles + 2 * pair);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float y[1];
                partners[e].get(y, true);
                if (d0 + q + e < rot) x[q + e] = turned(x[q + e], y[0], cs[e][0], cs[e][1], d0 + q + e >= half);
            }
            __builtin_amdgcn_sched_barrier(0);
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

// A block of a sequence: tokens [0, old) are there, [old, end) are new.  find() looks up where it lies (scalar loads), if it has a
// page; then codes, rows and angles are requested together.
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

// Keys: lane n has unit n % units (16 elements) of token n / units.  Lanes without a new token request one that there is.
template <int TYPE, int FMT, int CH>
__device__ __forceinline__ void append_keys(const AppendParams& p, const BlockPlace& b, int lane, int dim) {
    const int units = dim / 16;
    Elems<TYPE, 16> raw[CH];
    u32x4 there[CH];
    const float old_scale = b.old > 0 ? *b.scale : 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int n = lane + 64 * c, i = n / units, d0 = (n - i * units) * 16, row = i < b.old ? b.old : i < b.end ? i : b.end - 1;
        raw[c].request(static_cast<const typename Elem<TYPE>::T*>(p.k.data) + b.first + row * p.k.row_stride + d0);
        there[c] = (u32x4){0u, 0u, 0u, 0u};
        if (b.old > 0 && n < dim) there[c] = *reinterpret_cast<const u32x4*>(b.codes + n * 16);
    }
    float x[CH][16];
    uint32_t bits = 0;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int n = lane + 64 * c, i = n / units, d0 = (n - i * units) * 16;
        turn16<TYPE>(p.k, b.first + i * p.k.row_stride, p.rotation, b.t0 + i, d0, i >= b.old && i < b.end, raw[c], x[c]);
        bits = most_bits(x[c], bits);
    }
    const BlockScale s = block_scale<FMT>(max_over_wave(bits), old_scale);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int n = lane + 64 * c, i = n / units;
        if (n >= dim) continue;
        const u32x4 kept = i < b.old ? there[c] : (u32x4){0u, 0u, 0u, 0u};
        *reinterpret_cast<u32x4*>(b.codes + n * 16) = encode16<FMT>(x[c], kept, i >= b.old ? 0xffffu : 0u, s);
    }
    if (lane == 0) *b.scale = s.scale;
}

// Values: lane n has the 16 tokens at elements 2 n and 2 n + 1 (so that a row is read 4 or 8 bytes a lane).  Tokens that are not
// new stand for one that is, lanes beyond the head for its first one.
template <int TYPE, int FMT, int CH>
__device__ __forceinline__ void append_values(const AppendParams& p, const BlockPlace& b, int lane, int dim) {
    typedef typename Elem<TYPE>::T T;
    constexpr int PARTS = (CH + 1) / 2;
    Elems<TYPE, 2> raw[PARTS][16];
    u32x4 there[PARTS][2];
    const float old_scale = b.old > 0 ? *b.scale : 0.f;
#pragma unroll
    for (int c = 0; c < PARTS; ++c) {
        const int d = 2 * (lane + 64 * c);
        typedef const __attribute__((address_space(1))) T* Row;
        Row row = (Row)(static_cast<const T*>(p.v.data) + b.first + b.old * p.v.row_stride);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if (i > 0) row += i > b.old && i < b.end ? p.v.row_stride : 0;
            asm("" : "+s"(row));                                // (an address of the wave: no lane adds its offset to 64 bits)
            raw[c][i].request((const T*)row + static_cast<uint32_t>(d < dim ? d : 0));
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            there[c][h] = (u32x4){0u, 0u, 0u, 0u};
            if (b.old > 0 && d < dim) there[c][h] = *reinterpret_cast<const u32x4*>(b.codes + (d + h) * 16);
        }
    }
    float x[PARTS][2][16];
    uint32_t bits = 0;
#pragma unroll
    for (int c = 0; c < PARTS; ++c) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float two[2];
            raw[c][i].get(two, i >= b.old && i < b.end);        // (lanes beyond the head: numbers of the block, no matter)
            x[c][0][i] = two[0];
            x[c][1][i] = two[1];
        }
        bits = most_bits(x[c][1], most_bits(x[c][0], bits));
    }
    const BlockScale s = block_scale<FMT>(max_over_wave(bits), old_scale);
    const uint32_t is_old = (1u << b.old) - 1u;
#pragma unroll
    for (int c = 0; c < PARTS; ++c) {
        const int d = 2 * (lane + 64 * c);
        if (d >= dim) continue;
#pragma unroll
        for (int h = 0; h < 2; ++h)
            *reinterpret_cast<u32x4*>(b.codes + (d + h) * 16) = encode16<FMT>(x[c][h], chosen_codes(there[c][h], is_old), ~is_old, s);
    }
    if (lane == 0) *b.scale = s.scale;
}

template <int TYPE, int FMT, int CH>
__global__ __launch_bounds__(256) void cache_append_kernel(const AppendParams p) {
    const int lane = threadIdx.x & 63;
    // (sequence, block) pairs and, four waves of a workgroup, the heads' keys and values
    const int kinds = 2 * p.cache.heads, parts = (kinds + 3) / 4;
    const int group = p.first + blockIdx.x, pair = group / parts, kind = (group - pair * parts) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int seq = pair / p.blocks, j = pair - seq * p.blocks;
    if (kind >= kinds) return;
    const int head = kind >> 1;
    const RowRange range = p.ragged.range(seq, p.cache.length(seq));
    const int pos0 = range.token, end = pos0 + range.count;     // tokens of the rows
    const int b = (pos0 < 0 ? 0 : pos0) / kCacheBlock + j, t0 = b * kCacheBlock;
    if (range.count <= 0 || t0 >= end) return;
    const bool values = kind & 1;
    const Rows& src = values ? p.v : p.k;
    const int dim = p.cache.dim;
    BlockPlace at = {p.cache, seq, b, head, values,
                     (range.first + static_cast<long long>(t0 - pos0)) * src.row_stride + head * src.head_stride, t0,
                     pos0 - t0 < 0 ? 0 : pos0 - t0, end - t0 < kCacheBlock ? end - t0 : kCacheBlock, nullptr, nullptr};
    if (!at.find()) return;
    if (values) append_values<TYPE, FMT, CH>(p, at, lane, dim);
    else append_keys<TYPE, FMT, CH>(p, at, lane, dim);
}

struct ReadParams {
    Cache cache;
    Ragged ragged;
    Rows k, v;
    int seqs, blocks;
    unsigned first;
};

template <int TYPE, int FMT, int CH>
__global__ __launch_bounds__(256) void cache_read_kernel(const ReadParams p) {
    const int lane = threadIdx.x & 63;
    const int kinds = 2 * p.cache.heads, parts = (kinds + 3) / 4;
    const int group = p.first + blockIdx.x, pair = group / parts, kind = (group - pair * parts) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int seq = pair / p.blocks, j = pair - seq * p.blocks;
    if (kind >= kinds) return;
    const int head = kind >> 1;
    const bool values = kind & 1;
    const RowRange range = p.ragged.range(seq, p.cache.length(seq));
    const int pos0 = range.token, end = pos0 + range.count;
    const int b = (pos0 >> 4) + j;                              // (rounded down: below 0 before the first token)
    const long long t0 = static_cast<long long>(b) * kCacheBlock;
    if (range.count <= 0 || t0 >= end) return;
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
    const long long first = (range.first + (t0 - pos0)) * dst.row_stride + head * dst.head_stride;
    const int from = pos0 > t0 ? static_cast<int>(pos0 - t0) : 0;
    const int to = end - t0 < kCacheBlock ? static_cast<int>(end - t0) : kCacheBlock;
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
