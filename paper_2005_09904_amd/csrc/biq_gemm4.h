// Products with 4-bit weights (biq_gemm4), their layout and quantiser.
//
//   Y[b][i] = sum over groups g of scale[i][g] * sum over the group's j of code[i][j] X[b][j]
//
// Layout: records of 16 rows and 128 elements of each, all records of 16 rows one after the other.  A record holds 64 x 16 bytes
// of codes, then the bfloat16 scales [rows / 4][128 / group][4].  Lane l of a wave takes the l-th 16 bytes: row l % 16, and of each of
// the four spans of 32 elements the 8 from 8 (l / 16) on (a dword): the left operand of one 16 x 16 x 32 product per dword, whose
// 32 elements belong to one group.  A dword holds code + 8 of element 2 i in its bits 4 i and of element 2 i + 1 in its bits
// 16 + 4 i: ((w >> 4 i) & 0x000f000f) | 0x64006400 is two 16-bit floats 1024 + code + 8.  (Small whole numbers set under the exponent of
// 1024 instead of converted: published for 8- and 4-bit weights in arXiv 2211.10017.)
// What is missing of the last rows and elements has code 0 and scale 0.
#pragma once

#include "biq_serve.h"

namespace biq {

constexpr int kBlock4 = 128;                         // elements of a record's rows
constexpr int kWaves4 = 8;                           // waves of a workgroup
constexpr int kInt8 = 3, kFp8 = 4;                   // types of X beside biq_type: codes

struct Gemm4Params {
    const uint8_t* weights;
    const void* x;
    const float* x_scales;   // [batch][x_groups], codes only
    void* y;
    float* part;             // [splits][batch][16 tiles] sums of shares of the blocks (many vectors)
    long long x_stride, y_stride;
    int m, n, batch, blocks, tiles;
    int record;              // bytes of a record
    int x_group, x_groups;   // elements of a group of X's scales (0: the row), groups of a row
    int y_type;
    int splits;              // waves (many vectors: workgroups) that share a tile's blocks
    int columns;             // vectors of a workgroup
    unsigned first;
};

__device__ __forceinline__ float bf16_up(uint32_t bits) { return __uint_as_float(bits << 16); }

// 8 codes as 16-bit floats (exact): 4 bits below the exponent of 1024 are 1024 + u, those above them 1024 + 16 u, both u = code + 8.
// Masks are kept in registers, one of them a vector's, as an instruction takes one constant.
struct Masks4 {
    uint32_t low, high, exponent;
    __device__ __forceinline__ Masks4() : low(0x000f000fu), high(0x00f000f0u), exponent(0x64006400u) {
        asm("" : "+v"(low));
        asm("" : "+v"(high));
        asm("" : "+s"(exponent));
    }
};
__device__ __forceinline__ f16x8 weights_f16(uint32_t w, const Masks4& m) {
    union { f16x8 v; f16x2 p[4]; uint32_t w[4]; } r;
    const uint32_t w8 = w >> 8;
    r.w[0] = (w & m.low) | m.exponent;
    r.w[1] = (w & m.high) | m.exponent;
    r.w[2] = (w8 & m.low) | m.exponent;
    r.w[3] = (w8 & m.high) | m.exponent;
    const f16x2 sixteenth = {0.0625f16, 0.0625f16}, less = {-72.0f16, -72.0f16};
    r.p[0] -= (f16x2){1032.0f16, 1032.0f16};
    r.p[2] -= (f16x2){1032.0f16, 1032.0f16};
    r.p[1] = __builtin_elementwise_fma(r.p[1], sixteenth, less);
    r.p[3] = __builtin_elementwise_fma(r.p[3], sixteenth, less);
    return r.v;
}

// ---- laying out ---------------------------------------------------------------------------------------------

// One thread per dword of codes; scale(row, group) is asked for once per scale.
template <typename Code, typename Scale>
__device__ __forceinline__ void lay_out4(uint8_t* record, int tile, int block, int dword, int m, int n, int group, const Code& code, const Scale& scale) {
    const int lane = dword >> 2, j = dword & 3, row = tile * 16 + (lane & 15), e0 = block * kBlock4 + 32 * j + 8 * (lane >> 4);
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int c = row < m && e0 + i < n ? code(row, e0 + i) : 0;
        w |= static_cast<uint32_t>(c + 8) << (i & 1 ? 16 + 4 * (i >> 1) : 4 * (i >> 1));
    }
    reinterpret_cast<uint32_t*>(record)[dword] = w;
    const int per = kBlock4 / group;                            // scales of a row in a record
    if (dword < 16 * per) {
        const int r = tile * 16 + dword / (4 * per) * 4 + (dword & 3), g = block * per + dword / 4 % per;
        const bool there = r < m && g * group < n;
        reinterpret_cast<uint16_t*>(record + 1024)[dword] = there ? scale(r, g) : 0;
    }
}

// To bfloat16, to nearest, ties to even (NaN stays one).
__device__ __forceinline__ uint16_t bf16_bits(float x) {
    union { __bf16 h; uint16_t u; } r;
    r.h = static_cast<__bf16>(x);
    return r.u;
}

struct Pack4Params {
    const int8_t* codes;     // [m][n]
    const void* source;      // the quantiser's W [m][n]
    const float* scales;     // [m][groups]
    uint8_t* packed;
    float* out;              // biq_unpack4's W
    long long stride;
    int m, n, group, groups, blocks, record;
    unsigned first;
};

static __global__ __launch_bounds__(256) void pack4_kernel(const Pack4Params p) {
    const long long at = p.first + blockIdx.x;
    const int tile = static_cast<int>(at / p.blocks), block = static_cast<int>(at - static_cast<long long>(tile) * p.blocks);
    lay_out4(p.packed + at * p.record, tile, block, threadIdx.x, p.m, p.n, p.group,
             [&](int r, int e) {
                 const int c = p.codes[static_cast<long long>(r) * p.n + e];
                 return c < -8 ? -8 : c > 7 ? 7 : c;
             },
             [&](int r, int g) { return bf16_bits(p.scales[static_cast<long long>(r) * p.groups + g]); });
}

// scale = (largest magnitude of the group) * (1 / 7) to bfloat16, codes rn(w * (1 / scale)) in -8 .. 7; groups below 2^-100: zeros;
// groups with an infinity or a NaN: NaN.  A workgroup per record: scales first, through LDS.
template <int TYPE>
__global__ __launch_bounds__(256) void quantize4_kernel(const Pack4Params p) {
    __shared__ float scales[64], factors[64];                   // [group in the record][row]
    const long long at = p.first + blockIdx.x;
    const int tile = static_cast<int>(at / p.blocks), block = static_cast<int>(at - static_cast<long long>(tile) * p.blocks);
    {
        // 16 threads a row, 8 elements each: 4, 8 or 16 of them are a group
        const int row = tile * 16 + (threadIdx.x >> 4), e0 = block * kBlock4 + 8 * (threadIdx.x & 15);
        uint32_t most = 0;
        for (int i = 0; i < 8; ++i) {
            const float x = row < p.m && e0 + i < p.n ? load_elem<TYPE>(p.source, row * p.stride + e0 + i) : 0.f;
            const uint32_t bits = __float_as_uint(x) & 0x7fffffffu;
            most = most > bits ? most : bits;
        }
        for (int d = 1; d < p.group / 8; d *= 2) {
            const uint32_t other = __shfl_xor(most, d);
            most = most > other ? most : other;
        }
        if ((threadIdx.x & 15) % (p.group / 8) == 0) {
            const int to = (threadIdx.x & 15) / (p.group / 8) * 16 + (threadIdx.x >> 4);
            const bool bad = most >= 0x7f800000u;
            const float scale = bad ? __uint_as_float(0x7fc00000u) : most < 0x0d800000u ? 0.f : bf16_up(bf16_bits(__uint_as_float(most) * (1.0f / 7.0f)));
            scales[to] = scale;
            factors[to] = scale > 0.f && !bad ? 1.0f / scale : 0.f;
        }
    }
    __syncthreads();
    lay_out4(p.packed + at * p.record, tile, block, threadIdx.x, p.m, p.n, p.group,
             [&](int r, int e) {
                 const float f = factors[(e % kBlock4) / p.group * 16 + (r & 15)];
                 const float x = f == 0.f ? 0.f : __builtin_rintf(load_elem<TYPE>(p.source, r * p.stride + e) * f);
                 return static_cast<int>(x < -8.f ? -8.f : x > 7.f ? 7.f : x);
             },
             [&](int r, int g) { return bf16_bits(scales[g * p.group % kBlock4 / p.group * 16 + (r & 15)]); });
}

// The weights' values.
static __global__ __launch_bounds__(256) void unpack4_kernel(const Pack4Params p) {
    const long long at = p.first + blockIdx.x;
    const int tile = static_cast<int>(at / p.blocks), block = static_cast<int>(at - static_cast<long long>(tile) * p.blocks);
    const int lane = threadIdx.x >> 2, j = threadIdx.x & 3, row = tile * 16 + (lane & 15), e0 = block * kBlock4 + 32 * j + 8 * (lane >> 4);
    const uint8_t* record = p.packed + at * p.record;
    const uint32_t w = reinterpret_cast<const uint32_t*>(record)[threadIdx.x];
    const int per = kBlock4 / p.group, r = lane & 15;
    const float scale = bf16_up(reinterpret_cast<const uint16_t*>(record + 1024)[((r >> 2) * per + 32 * j / p.group) * 4 + (r & 3)]);
    if (row >= p.m) return;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (e0 + i < p.n)
            p.out[row * p.stride + e0 + i] = static_cast<float>(static_cast<int>(w >> (i & 1 ? 16 + 4 * (i >> 1) : 4 * (i >> 1)) & 15u) - 8) * scale;
}

// ---- X as operands ------------------------------------------------------------------------------------------

// 32-bit elements are two 16-bit floats, the others one.
template <int XT> constexpr int kTerms4 = XT == BIQ_F32 ? 2 : 1;
template <int XT> struct X4 { typedef typename Elem<XT>::T T; };
template <> struct X4<kInt8> { typedef int8_t T; };
template <> struct X4<kFp8> { typedef uint8_t T; };

// The largest of 16 lanes' numbers (not below 0), in all of them: over quads, halves, all.
__device__ __forceinline__ float over_16_lanes(float x) {
    auto with = [&](int y) { x = fmaxf(x, __int_as_float(y)); };
    with(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0xb1, 0xf, 0xf, true));         // quad_perm [1,0,3,2]
    with(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x4e, 0xf, 0xf, true));         // quad_perm [2,3,0,1]
    with(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x141, 0xf, 0xf, true));        // row_half_mirror
    with(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x140, 0xf, 0xf, true));        // row_mirror
    return x;
}

// 8 adjacent elements of an input vector from e on, as they are.  Those at its end come from the last 8 there are (n >= 8), further
// on than they should be by `late`: a branch with loads of their own would make all loads in flight be waited for.
template <int XT>
struct Raw8 {
    typedef typename X4<XT>::T T;
    typedef T Loose __attribute__((ext_vector_type(8), aligned(sizeof(T))));
    T __attribute__((ext_vector_type(8))) v;
    __device__ __forceinline__ void request(const T* row, int e, int n) { v = *reinterpret_cast<const Loose*>(row + (e < n - 8 ? e : n - 8)); }
    __device__ __forceinline__ void request_few(const T* row, int e, int n) {          // (n < 8)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = row[e + i < n ? e + i : n - 1];
    }
};
__device__ __forceinline__ int late8(int e, int n) { return n < 8 || e <= n - 8 ? 0 : e - (n - 8); }

// As terms (zeros behind the vector's end); returned is what a 1 stands for.  The 16 lanes of a block of 128 call this together:
// 32-bit and bf16 elements are scaled by a power of two, the block's largest magnitude to [2^14, 2^15).  Elements keep 22 bits (8 of bf16), and
// none below 2^-39 of the block's largest.  A third term would keep 32-bit elements whole for half as many products and operands again; two
// leave 1.2e-7 of the result (48 vectors of 16384), the rounding of an output in 32 bits and less than a product in 32 bits loses by its sums (2.1e-6).
template <int XT>
__device__ __forceinline__ float operand8(const Raw8<XT>& raw, int e, int n, f16x8 (&out)[kTerms4<XT>]) {
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (XT == kFp8) x[i] = __builtin_amdgcn_cvt_f32_fp8(raw.v[i], 0);
        else x[i] = static_cast<float>(raw.v[i]);
    }
    if (__any(e + 8 > n)) {
        const int late = late8(e, n);
#pragma unroll
        for (int d = 4; d > 0; d /= 2)
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = !(late & d) ? x[i] : i + d < 8 ? x[i + d] : 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = e + i < n ? x[i] : 0.f;
    }
    float unit = 1.f;
    if constexpr (XT == BIQ_F32 || XT == BIQ_BF16) {
        // (a NaN does not count here, and comes through the products)
        float most = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(x[i]));
        most = over_16_lanes(most);
        int b = static_cast<int>(__float_as_uint(most) >> 23);  // biased exponent
        b = most == 0.f ? 127 + 14 : b < 27 ? 27 : b;
        const float up = __uint_as_float(static_cast<uint32_t>(127 + 14 + 127 - b) << 23);
        unit = __uint_as_float(static_cast<uint32_t>(b - 14) << 23);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= up;
    }
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        const f16x2 hi = __builtin_convertvector((f32x2){x[i], x[i + 1]}, f16x2);
        out[0][i] = hi[0];
        out[0][i + 1] = hi[1];
        if constexpr (kTerms4<XT> == 2) {
            const f16x2 lo = __builtin_convertvector((f32x2){x[i] - static_cast<float>(hi[0]), x[i + 1] - static_cast<float>(hi[1])}, f16x2);
            out[1][i] = lo[0];
            out[1][i + 1] = lo[1];
        }
    }
    return unit;
}

// ---- the product --------------------------------------------------------------------------------------------

// Where the operands of X are: [block][span of 32][term][lane / 16][column] of 16 bytes, and what units they have: [block][scale]
// [column].  columns: how many there are of them.
struct Operands4 {
    const f16x8* x;
    const float* units;
    int columns;
};

// A lane's part of a record: 16 bytes of codes, and the scales of its 4 rows of products, G spans of 32 elements each.
template <int G>
struct Part4 {
    typedef uint32_t Scales __attribute__((ext_vector_type(8 / G)));
    u32x4 codes;
    Scales scales;
    __device__ __forceinline__ void request(const uint8_t* record, int lane) {
        codes = *reinterpret_cast<const u32x4*>(record + 16u * static_cast<uint32_t>(lane));
        typedef uint32_t Loose __attribute__((ext_vector_type(8 / G), aligned(8)));
        scales = *reinterpret_cast<const Loose*>(record + 1024 + 32u / G * static_cast<uint32_t>(lane >> 4));
    }
    // Of span j.
    __device__ __forceinline__ f32x4 of(int j) const {
        const uint32_t a = scales[j / G * 2], b = scales[j / G * 2 + 1];
        return (f32x4){bf16_up(a), __uint_as_float(a & 0xffff0000u), bf16_up(b), __uint_as_float(b & 0xffff0000u)};
    }
};

// Sums of a group are multiplied by the weights' scale, then by X's unit or scale: with scales up to 2^100 the first product stays in range (sums are
// at most 2^26), and the second is the result.  (X's first would leave 32 bits from 1e36 on, whatever the weights are.)
//
// A wave's share of a tile of 16 rows: blocks `from`, from + step, ..., of NC times 16 columns.  F spans of 32 share both scales, G the
// weights'.  AHEAD records are requested before the first of them is used.
template <int TERMS, int F, int G, int NC, int AHEAD>
__device__ __forceinline__ void tile4(const uint8_t* tile, int record, int blocks, int from, int step, const Operands4& x, int x_scales,
                                      f32x4 (&acc)[NC]) {
    constexpr int FLUSHES = 4 / F;
    const int lane = threadIdx.x & 63, grp = lane >> 4;
    int col[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) col[c] = (lane & 15) + 16 * c < x.columns ? (lane & 15) + 16 * c : x.columns - 1;
    const Masks4 masks;
    Part4<G> parts[AHEAD];
    auto request = [&](int i, int block) { parts[i].request(tile + static_cast<long long>(block < blocks ? block : blocks - 1) * record, lane); };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) request(i, from + i * step);
    for (int b0 = from; b0 < blocks; b0 += AHEAD * step) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int block = b0 + i * step;
            if (block < blocks) {
#pragma unroll
                for (int f = 0; f < FLUSHES; ++f) {
                    f32x4 part[NC];
#pragma unroll
                    for (int c = 0; c < NC; ++c) part[c] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int j = f * F; j < f * F + F; ++j) {
                        const f16x8 w = weights_f16(parts[i].codes[j], masks);
#pragma unroll
                        for (int t = 0; t < TERMS; ++t)
#pragma unroll
                            for (int c = 0; c < NC; ++c)
                                part[c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(w, x.x[(((block * 4 + j) * TERMS + t) * 4 + grp) * x.columns + col[c]], part[c], 0, 0, 0);
                    }
                    const f32x4 ws = parts[i].of(f * F);
#pragma unroll
                    for (int c = 0; c < NC; ++c) {
                        const float unit = x.units[(block * x_scales + f * x_scales / FLUSHES) * x.columns + col[c]];
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[c][e] = __builtin_fmaf(part[c][e] * ws[e], unit, acc[c][e]);
                    }
                }
            }
            request(i, block + AHEAD * step);
        }
    }
}

// X's operands from its elements, all threads of a workgroup; AHEAD units of 8 elements are requested together (a block has 16 units, so
// lanes that exchange magnitudes are all there).  between: called once, with the first units requested.
template <int XT, typename Between>
__device__ __forceinline__ void stage4(const Gemm4Params& p, int column0, int columns, int x_scales, f16x8* to, float* units, const Between& between) {
    constexpr int THREADS = 64 * kWaves4, AHEAD = XT == BIQ_F32 ? 4 : 8;
    typedef typename X4<XT>::T T;
    const int per = p.blocks * 16, total = per * columns, every = 16 / x_scales;
    for (int first = threadIdx.x; first < total; first += AHEAD * THREADS) {
        Raw8<XT> raw[AHEAD];
        float scale[AHEAD];
        auto place = [&](int a, int& column, int& unit) {
            const int at = first + a * THREADS < total ? first + a * THREADS : first;           // (again: all loads are requested)
            column = at / per;
            unit = at - column * per;
        };
        auto request = [&](bool few) {
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) {
                int c, u;
                place(a, c, u);
                const T* row = static_cast<const T*>(p.x) + (column0 + c) * p.x_stride;
                if (few) raw[a].request_few(row, u * 8, p.n);
                else raw[a].request(row, u * 8, p.n);
                if constexpr (XT == kInt8 || XT == kFp8) {
                    int g = p.x_group == 0 ? 0 : u * 8 / p.x_group;     // (behind the last element: one that there is)
                    g = g < p.x_groups ? g : p.x_groups - 1;
                    scale[a] = p.x_scales[static_cast<long long>(column0 + c) * p.x_groups + g];
                }
            }
        };
        if (p.n < 8) request(true);
        else request(false);
        if (first == static_cast<int>(threadIdx.x)) between();
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            if (first + a * THREADS >= total) break;
            int c, u;
            place(a, c, u);
            f16x8 out[kTerms4<XT>];
            float unit = operand8<XT>(raw[a], u * 8, p.n, out);
#pragma unroll
            for (int t = 0; t < kTerms4<XT>; ++t) to[(((u >> 2) * kTerms4<XT> + t) * 4 + (u & 3)) * columns + c] = out[t];
            if constexpr (XT == kInt8 || XT == kFp8) unit = scale[a];
            if ((u & 15) % every == 0) units[((u >> 4) * x_scales + (u & 15) / every) * columns + c] = unit;
        }
    }
}

template <int TYPE>
__device__ __forceinline__ void store_y4(const Gemm4Params& p, int column, int row, f32x4 x) {
    typedef typename Elem<TYPE>::T T;
    T* to = static_cast<T*>(p.y) + column * p.y_stride + row;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (row + e < p.m) to[e] = static_cast<T>(x[e]);
}
__device__ __forceinline__ void store_y4(const Gemm4Params& p, int column, int row, f32x4 x) {
    if (p.y_type == BIQ_F32) store_y4<BIQ_F32>(p, column, row, x);
    else if (p.y_type == BIQ_BF16) store_y4<BIQ_BF16>(p, column, row, x);
    else store_y4<BIQ_F16>(p, column, row, x);
}

// A few vectors: all of them as operands in LDS.  The WAVES waves of a workgroup take WAVES / splits tiles; waves of a tile
// share its blocks and are joined through LDS.  Splitting blocks over waves costs a round through LDS, and pays as long as the chip is not full
// of waves: there are twice as many splits until tiles x splits fill 2048 waves.
//
// The weights bound large products: 32000 x 4096 with groups of 64 (70 MB) and one vector of bfloat16 takes 16.7 us from the kernel's start to its end,
// 15.2 a call among others (whose starts and ends overlap: 4.6 TB/s); the workgroups' start (X is the operand that all of it waits for) is
// not covered by loads.  16384 x 4096 with five vectors of codes (35 MB) 11.4 us, 10.3 a call; 4096 x 4096 with one vector 6.5 us, 5.6 a call, X, weights
// and join one after the other.  One load a wave touches the lines of its first four records while X is converted: without, a call takes 15.7, 10.8 and
// 5.5 us.  AHEAD records of weights are in flight: with 8 the head's kernel takes 23 us, with 2 17.4, with the weights asked for before X becomes
// operands 19.7 (registers).
template <int XT, int F, int G>
__global__ __launch_bounds__(64 * kWaves4) void gemm4_few_kernel(const Gemm4Params p, int x_scales) {
    extern __shared__ float lds[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int column0 = blockIdx.y * 16, columns = p.batch - column0 < 16 ? p.batch - column0 : 16;
    f16x8* operands = reinterpret_cast<f16x8*>(lds);
    float* units = reinterpret_cast<float*>(operands + p.blocks * 16 * kTerms4<XT> * columns);
    const int per = kWaves4 / p.splits, split = wave % p.splits, tile = (p.first + blockIdx.x) * per + wave / p.splits;
    const uint8_t* weights = p.weights + static_cast<long long>(tile < p.tiles ? tile : p.tiles - 1) * p.blocks * p.record;
    int touched = 0;
    stage4<XT>(p, column0, columns, x_scales, operands, units, [&]() {
        const int block = split + (lane >> 4) * p.splits, at = (lane & 15) * 128;
        touched = *reinterpret_cast<const int*>(weights + (block < p.blocks ? block : p.blocks - 1) * static_cast<long long>(p.record) + (at < p.record ? at : 0));
    });
    __syncthreads();
    f32x4 acc[1] = {{0.f, 0.f, 0.f, 0.f}};
    if (tile < p.tiles)
        tile4<kTerms4<XT>, F, G, 1, 4>(weights, p.record, p.blocks, split, p.splits,
                                    {operands, units, columns}, x_scales, acc);
    asm volatile("" : : "v"(touched));
    if (p.splits > 1) {
        __syncthreads();                                        // (the operands are read)
        f32x4* sums = reinterpret_cast<f32x4*>(lds);
        sums[wave * 64 + lane] = acc[0];
        __syncthreads();
        if (split > 0) return;
        for (int s = 1; s < p.splits; ++s) acc[0] += sums[(wave + s) * 64 + lane];
    }
    if (tile < p.tiles && (lane & 15) < columns) store_y4(p, column0 + (lane & 15), tile * 16 + 4 * (lane >> 4), acc[0]);
}

// Many vectors (of 8 elements at least): a workgroup takes kRows4 rows, 32 a wave, up to 64 vectors and a share of the blocks.  X becomes operands
// on the way to LDS, two blocks at a time, while the two before are multiplied; the weights go from memory to registers two blocks ahead.  Operand
// (j, lane / 16) of a vector lies `u` = 4 j + lane / 16 places further on among its 16 vectors: neither the threads that write a vector's operands
// nor the lanes that read 16 vectors' meet on a bank.
//
// 256 rows share the conversion of X, and 32 rows a wave the reads of its operands: that costs as many instructions as unpacking the weights.  48
// vectors of 32 bits, 4096 x 16384 with groups of 32 (37 MB, 6.4 GFLOP counted once): 22.8 us and 4.6 for the join, 24.7 a call among others (the
// join's start lies within the products' end); 95 with the kernel of few vectors.  64 vectors are what registers hold of sums and operands (up to 229
// of a wave's 256); more of them read and unpack the weights again for each 64.  4096 x 4096 in bfloat16: 64 vectors 14.4 us, 128 17.0, 512 34 (503 TFLOP/s),
// 2048 109 (628); int8 codes 14.1, 16.6, 32, 98 (699); 32 bits 16.6, 20.1, 47, 163 (422).
// A SIMD's vector instructions (3300 a wave: unpacking, X's terms, both scales every 32 elements) and its products (6100 cycles a wave, two
// terms) add up; memory waits 30 % of the time.  Requests fenced against the compiler's order gave nothing and spilt registers at groups of 32.
constexpr int kRows4 = 32 * kWaves4;
// PER_BLOCK: X has one scale in a block of 128.
template <int XT, int F, int G, int NC, bool PER_BLOCK>
__global__ __launch_bounds__(64 * kWaves4, 2) void gemm4_many_kernel(const Gemm4Params p, int x_scales) {
    constexpr int TERMS = kTerms4<XT>, FLUSHES = 4 / F, COLS = 16 * NC, AHEAD = 2;
    constexpr int SIDE = 2 * 4 * TERMS * 4 * COLS;              // operands of two blocks
    constexpr bool SUMS = PER_BLOCK && !(TERMS == 2 && F == 1 && NC == 4);      // X's scale once a block (there: no registers for the block's sums)
    extern __shared__ float lds[];
    f16x8* operands = reinterpret_cast<f16x8*>(lds);            // [2][block][j][term][lane / 16][column]
    float* units = reinterpret_cast<float*>(operands + 2 * SIDE);       // [2][block][scale][column]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), grp = lane >> 4;
    // (workgroups that read the same of X are `splits` apart: mostly on one XCD)
    const int split = blockIdx.x % p.splits, tile = blockIdx.x / p.splits * 2 * kWaves4 + 2 * wave;
    const int column0 = blockIdx.y * p.columns, columns = p.batch - column0 < p.columns ? p.batch - column0 : p.columns;
    const int block0 = static_cast<int>(static_cast<long long>(p.blocks) * split / p.splits);
    const int block1 = static_cast<int>(static_cast<long long>(p.blocks) * (split + 1) / p.splits);

    // this thread's 8 elements of every 16th vector: unit u of the two blocks
    const int u = threadIdx.x & 31, own = threadIdx.x >> 5;
    typedef typename X4<XT>::T T;
    const T* rows[NC];
    const float* row_scales[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const long long column = column0 + (own + 16 * c < columns ? own + 16 * c : columns - 1);
        rows[c] = static_cast<const T*>(p.x) + column * p.x_stride;
        row_scales[c] = p.x_scales + column * p.x_groups;
    }
    Raw8<XT> raw[NC];
    float scale[NC];
    auto request_x = [&](int block) {
        const int e = block * kBlock4 + u * 8;
#pragma unroll
        for (int c = 0; c < NC; ++c) raw[c].request(rows[c], e, p.n);
        if constexpr (XT == kInt8 || XT == kFp8) {
            int g = p.x_group == 0 ? 0 : e / p.x_group;         // (behind the last element: one that there is)
            g = g < p.x_groups ? g : p.x_groups - 1;
#pragma unroll
            for (int c = 0; c < NC; ++c) scale[c] = row_scales[c][g];
        }
    };
    auto lay_down = [&](int side, int block) {
        f16x8* to = operands + side * SIDE;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            f16x8 out[TERMS];
            float unit = operand8<XT>(raw[c], block * kBlock4 + u * 8, p.n, out);
            const int place = 16 * c + ((own + u) & 15);
#pragma unroll
            for (int t = 0; t < TERMS; ++t) to[(((u >> 2) * TERMS + t) * 4 + (u & 3)) * COLS + place] = out[t];
            if constexpr (XT == kInt8 || XT == kFp8) unit = scale[c];
            const int every = 16 / x_scales;
            if ((u & 15) % every == 0) units[((side * 2 + (u >> 4)) * x_scales + (u & 15) / every) * COLS + 16 * c + own] = unit;
        }
    };

    const Masks4 masks;
    const uint8_t* weights[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) weights[r] = p.weights + static_cast<long long>(tile + r < p.tiles ? tile + r : p.tiles - 1) * p.blocks * p.record;
    Part4<G> parts[AHEAD][2];
    auto request_w = [&](int i, int block) {
#pragma unroll
        for (int r = 0; r < 2; ++r) parts[i][r].request(weights[r] + static_cast<long long>(block < block1 ? block : block1 - 1) * p.record, lane);
    };

    f32x4 acc[2][NC];
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int c = 0; c < NC; ++c) acc[r][c] = (f32x4){0.f, 0.f, 0.f, 0.f};
    request_x(block0);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) request_w(i, block0 + i);
    lay_down(0, block0);
    __syncthreads();
    for (int side = 0, pair = block0; pair < block1; pair += 2, side ^= 1) {
        request_x(pair + 2 < block1 ? pair + 2 : pair);         // (always: a branch would make the loads before it be waited for)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            if (pair + b >= block1) continue;
            const f16x8* from = operands + side * SIDE + b * (SIDE / 2);
            const float* unit = units + (side * 2 + b) * x_scales * COLS;
            f32x4 sum[2][NC], part[2][NC];                      // of the block, of the spans that share scales
            f16x8 w[2];
            // operand (j, term, column tile) of X and its two products
            read_ahead<4 * TERMS * NC, 2, false>([&](int i) {
                const int j = i / (TERMS * NC), t = i / NC % TERMS, c = i % NC;
                return from[((j * TERMS + t) * 4 + grp) * COLS + 16 * c + ((lane + 4 * j + grp) & 15)];
            }, [&](int i, f16x8 x) {
                const int j = i / (TERMS * NC), t = i / NC % TERMS, c = i % NC, f = j / F;
                const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
                if (t == 0 && c == 0) {
                    w[0] = weights_f16(parts[b][0].codes[j], masks);
                    w[1] = weights_f16(parts[b][1].codes[j], masks);
                }
#pragma unroll
                for (int r = 0; r < 2; ++r) part[r][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(w[r], x, t == 0 && j % F == 0 ? zero : part[r][c], 0, 0, 0);
                if (t < TERMS - 1 || j % F != F - 1 || c < NC - 1) return;
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const f32x4 ws = parts[b][r].of(f * F);
#pragma unroll
                    for (int k = 0; k < NC; ++k) {
                        if constexpr (SUMS) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) sum[r][k][e] = f == 0 ? part[r][k][e] * ws[e] : __builtin_fmaf(part[r][k][e], ws[e], sum[r][k][e]);
                        } else {
                            const float v = unit[f * x_scales / FLUSHES * COLS + 16 * k + (lane & 15)];
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[r][k][e] = __builtin_fmaf(part[r][k][e] * ws[e], v, acc[r][k][e]);
                        }
                    }
                }
            });
            if constexpr (SUMS) {
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    const float v = unit[16 * c + (lane & 15)];
#pragma unroll
                    for (int r = 0; r < 2; ++r)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[r][c][e] = __builtin_fmaf(sum[r][c][e], v, acc[r][c][e]);
                }
            }
            request_w(b, pair + b + AHEAD);
        }
        if (pair + 2 < block1) lay_down(side ^ 1, pair + 2);
        __syncthreads();
    }
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int column = (lane & 15) + 16 * c, row = (tile + r) * 16 + 4 * grp;
            if (column >= columns || row >= p.m) continue;
            if (p.splits == 1) {
                store_y4(p, column0 + column, row, acc[r][c]);
            } else {
                // (rows of partial sums are whole tiles)
                *reinterpret_cast<f32x4*>(p.part + (static_cast<long long>(split) * p.batch + column0 + column) * (16ll * p.tiles) + row) = acc[r][c];
            }
        }
}

// The sums of all shares of the blocks, in their order: a thread for 4 rows of a vector.
static __global__ __launch_bounds__(256) void gemm4_join_kernel(const Gemm4Params p) {
    const long long quads = 4ll * p.tiles, at = static_cast<long long>(p.first + blockIdx.x) * 256 + threadIdx.x;
    if (at >= quads * p.batch) return;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int s = 0; s < p.splits; ++s) sum += *reinterpret_cast<const f32x4*>(p.part + 4 * (s * quads * p.batch + at));
    const int column = static_cast<int>(at / quads), row = static_cast<int>(at - column * quads) * 4;
    if (row < p.m) store_y4(p, column, row, sum);
}

}  // namespace biq
