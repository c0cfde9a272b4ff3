// Shared device-side definitions of the operators around the multiply in a decoder step: element types, the paged 8-bit
// cache, rows that belong to sequences.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "biq.h"

namespace biq {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

constexpr int kCacheBlock = BIQ_CACHE_BLOCK;

template <int TYPE> struct Elem { typedef float T; };
template <> struct Elem<BIQ_BF16> { typedef __bf16 T; };
template <> struct Elem<BIQ_F16> { typedef _Float16 T; };

template <int TYPE>
__device__ __forceinline__ float load_elem(const void* base, long long i) {
    return static_cast<float>(static_cast<const typename Elem<TYPE>::T*>(base)[i]);
}
template <int TYPE>
__device__ __forceinline__ void store_elem(void* base, long long i, float x) {
    static_cast<typename Elem<TYPE>::T*>(base)[i] = static_cast<typename Elem<TYPE>::T>(x);
}

// 4 adjacent elements at a multiple of 4 bytes (wide accesses to memory need no more).
template <int TYPE>
__device__ __forceinline__ void store_elem4(void* base, long long i, f32x4 x) {
    typedef typename Elem<TYPE>::T V __attribute__((ext_vector_type(4)));
    typedef typename Elem<TYPE>::T Loose __attribute__((ext_vector_type(4), aligned(4)));
    *reinterpret_cast<Loose*>(static_cast<typename Elem<TYPE>::T*>(base) + i) = __builtin_convertvector(x, V);
}

// N adjacent elements as they are, at any address of an element (wide loads need no more).  They become floats once everything
// that a block or a unit starts with is requested: a conversion in a branch with its load waits for it.
template <int TYPE, int N>
struct Elems {
    typedef typename Elem<TYPE>::T T;
    typedef T V __attribute__((ext_vector_type(N)));
    V v;
    __device__ __forceinline__ void request(const T* from) {
        typedef T Loose __attribute__((ext_vector_type(N), aligned(sizeof(T))));
        v = *reinterpret_cast<const Loose*>(from);
    }
    __device__ __forceinline__ void get(float (&x)[N], bool used) const {
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = used ? static_cast<float>(v[e]) : 0.f;
    }
};

// biq_rows, with what the host has checked: quads = every 4th element lies at a multiple of 4 bytes.
struct Rows {
    void* data;
    long long row_stride, head_stride;
    int quads;
};

// biq_cache, with the sizes that follow from it.
struct Cache {
    uint8_t* store;
    const int* table;
    const int* lens;
    long long page_bytes;
    int num_pages, table_stride, heads, dim;
    int page_blocks;         // blocks per page, 1 .. 16
    uint32_t page_magic;     // floor(2^32 / page_blocks) + 1, its low 32 bits ..
    uint32_t page_ones;      // .. and all ones where there is a 33rd (page_blocks = 1)

    // b / page_blocks for b < 2^27: the product is off by less than 2^27 * 16 < 2^32
    __device__ __forceinline__ int page_index(int b) const {
        return static_cast<int>(__umulhi(static_cast<uint32_t>(b), page_magic) + (static_cast<uint32_t>(b) & page_ones));
    }
    __device__ __forceinline__ int length(int s) const {
        const long long most = static_cast<long long>(table_stride) * page_blocks * kCacheBlock;
        const int n = lens[s];
        return n < 0 ? 0 : n > most ? static_cast<int>(most) : n;
    }
    // Page number of block b of sequence s, -1 if it has none.
    __device__ __forceinline__ int page_number(int s, int b) const {
        const int i = page_index(b);
        const int n = table[static_cast<long long>(s) * table_stride + (i < table_stride ? i : 0)];
        return (i < table_stride && static_cast<uint32_t>(n) < static_cast<uint32_t>(num_pages)) ? n : -1;
    }
    // Block `sub` of a head among the page's blocks.
    __device__ __forceinline__ int block_in_page(int b, int head) const {
        return head * page_blocks + (b - page_index(b) * page_blocks);
    }
    __device__ __forceinline__ uint8_t* page(int number) const { return store + number * page_bytes; }
    __device__ __forceinline__ long long codes_bytes() const {
        return static_cast<long long>(heads) * page_blocks * kCacheBlock * dim;
    }
};

// Rows of a sequence that are served: row `first` + i, i < count, is token `token` + i (below 0: before the first token).
struct RowRange { int first, count, token; };

struct Ragged {
    const int* starts;
    int rows, max_rows;
    // The n rows of sequence s are its last n tokens, whether or not all of them are served.
    __device__ __forceinline__ RowRange range(int s, int len) const {
        if (!starts) return {s * max_rows, max_rows, len - max_rows};
        int a = starts[s], e = starts[s + 1];
        a = a < 0 ? 0 : a > rows ? rows : a;
        e = e < a ? a : e > rows ? rows : e;
        const int n = e - a, token = len - n;
        // (a first row more than max_rows before token 0: no served one is a token, and sums of these numbers keep to 32 bits)
        return {a, n > max_rows ? max_rows : n, token < -max_rows ? -max_rows : token};
    }
};

// Sequence that block j of a launch grid works on etc. is decided per kernel; this is the number of XCDs that consecutive
// workgroups are dealt to in turn.
constexpr int kXcds = 8;

// ---- codes ---------------------------------------------------------------------------------------------

// Code i (0 .. 3) of a dword as a float.
template <int FMT, int I>
__device__ __forceinline__ float code_value(uint32_t w) {
    if constexpr (FMT == BIQ_CACHE_INT8)
        return static_cast<float>(static_cast<int>(w << (24 - 8 * I)) >> 24);
    else
        return __builtin_amdgcn_cvt_f32_fp8(w, I);
}

// 8 codes as 8 16-bit floats (exact).
template <int FMT>
__device__ __forceinline__ f16x8 codes_f16(uint32_t a, uint32_t b) {
    union { f16x8 v; f16x2 p[4]; uint32_t w[4]; } r;
    if constexpr (FMT == BIQ_CACHE_INT8) {
        // 0x6400 + u is 1024 + u: of the code + 128 as an unsigned byte
        const uint32_t ua = a ^ 0x80808080u, ub = b ^ 0x80808080u;
        r.w[0] = __builtin_amdgcn_perm(0x64646464u, ua, 0x04010400u);
        r.w[1] = __builtin_amdgcn_perm(0x64646464u, ua, 0x04030402u);
        r.w[2] = __builtin_amdgcn_perm(0x64646464u, ub, 0x04010400u);
        r.w[3] = __builtin_amdgcn_perm(0x64646464u, ub, 0x04030402u);
#pragma unroll
        for (int i = 0; i < 4; ++i) r.p[i] -= (f16x2){1152.0f16, 1152.0f16};
    } else {
        r.p[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, false);
        r.p[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, true);
        r.p[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, false);
        r.p[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, true);
    }
    return r.v;
}

// Values with the scale divided out -> 4 codes in a dword, rounded to nearest, ties to even.  int8: |x| <= 127.5; fp8: <= 448.
template <int FMT>
__device__ __forceinline__ uint32_t encode4(float x0, float x1, float x2, float x3) {
    if constexpr (FMT == BIQ_CACHE_INT8) {
        auto one = [](float x) {
            x = __builtin_rintf(x);
            x = x > 127.0f ? 127.0f : x < -127.0f ? -127.0f : x;
            return static_cast<uint32_t>(static_cast<int>(x)) & 255u;
        };
        return one(x0) | one(x1) << 8 | one(x2) << 16 | one(x3) << 24;
    } else {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(x0, x1, 0, false);
        return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(x2, x3, w, true));
    }
}

// Sum / maximum over the lanes l, l ^ 16, l ^ 32, l ^ 48.
__device__ __forceinline__ float max_over_groups(float x) {
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float sum_over_groups(float x) {
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

// READS operands from LDS and the EACH products of every one of them: read(i) four ahead of use(i, operand).  (Left alone, the compiler
// reads each operand right before its products and waits for it.)  Either the scheduler is asked for this order, which leaves it
// free to place what else there is to do (two prompts with heads of 128: 806 us instead of 812), or, FENCED, the reads stand where they
// are meant to be and only other vector and scalar instructions pass: with heads above 128 the scheduler gives up its own order now and
// then (heads of 256 in bf16: 365 us instead of 288).
template <int READS, int EACH, bool FENCED, typename Read, typename Use>
__device__ __forceinline__ void read_ahead(const Read& read, const Use& use) {
    constexpr int kAhead = 4;
    if constexpr (FENCED) {
        constexpr int kVectorAndScalar = 0x6;
        f16x8 ring[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) ring[i] = read(i);
#pragma unroll
        for (int i = 0; i < READS; ++i) {
            use(i, ring[i % kAhead]);
            if (i + kAhead < READS) ring[i % kAhead] = read(i + kAhead);
            __builtin_amdgcn_sched_barrier(kVectorAndScalar);
        }
    } else {
        constexpr int kReads = 0x100, kProducts = 0x8;
#pragma unroll
        for (int i = 0; i < READS; ++i) use(i, read(i));
        __builtin_amdgcn_sched_group_barrier(kReads, kAhead, 0);
#pragma unroll
        for (int i = 0; i < READS - kAhead; ++i) {
            __builtin_amdgcn_sched_group_barrier(kProducts, EACH, 0);
            __builtin_amdgcn_sched_group_barrier(kReads, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(kProducts, kAhead * EACH, 0);
    }
}

}  // namespace biq
