// Root-mean-square norm with the residual's addition (biq_norm).
//
//   s = x + residual,  r = 1 / sqrt(mean(s^2) + eps),  y = (s r) w,  codes of t = s w per group, their scale times r
//
// A row stays in registers: it is read once, summed, and written.  THREADS threads hold K times 8 adjacent elements each, so the
// 32, 64 or 128 elements of a group of codes are those of 4, 8 or 16 neighbouring lanes.  Squares are added in 32 bits, and in 64 where the
// sum leaves the range in which 32 bits keep their precision.
//
// Memory bounds many rows: 8192 x 4096 in bfloat16 with the sum written (268 MB) takes 54 us, 5.0 TB/s.  Few rows are bound by the launch and
// by what one waits for in turn, the row, its sum, (with one scale for the whole row) its largest, then codes and stores: 1 x 4096 2.8 to 3.1 us, 80 x
// 5003 with codes of groups 5.8 us.
#pragma once

#include "biq_cache.h"

namespace biq {

struct NormParams {
    const void* x;
    const void* residual;    // or NULL
    void* sum;               // or NULL
    const float* weight;     // NULL: ones
    void* y;                 // or NULL
    uint8_t* codes;          // or NULL
    float* scales;
    long long x_stride, residual_stride, sum_stride, y_stride, code_stride;
    int y_type, rows, n, group, groups, format;
    float eps, weight_add;
    unsigned first;          // first workgroup of this launch
};

// 8 adjacent elements, or those of them that there are, at any address of an element.
template <typename T>
__device__ __forceinline__ void request8(T (&v)[8], const T* row, int e, int n) {
    typedef T Loose __attribute__((ext_vector_type(8), aligned(sizeof(T))));
    if (e + 8 <= n) {
        const Loose all = *reinterpret_cast<const Loose*>(row + e);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = all[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = row[e + i < n ? e + i : n - 1];
    }
}
template <typename T>
__device__ __forceinline__ void store8(T* row, int e, int n, const T (&v)[8]) {
    typedef T Loose __attribute__((ext_vector_type(8), aligned(sizeof(T))));
    if (e + 8 <= n) {
        Loose all;
#pragma unroll
        for (int i = 0; i < 8; ++i) all[i] = v[i];
        *reinterpret_cast<Loose*>(row + e) = all;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (e + i < n) row[e + i] = v[i];
    }
}
template <int TYPE>
__device__ __forceinline__ void store8_as(void* base, long long at, int e, int n, const float (&x)[8]) {
    typedef typename Elem<TYPE>::T T;
    T v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = static_cast<T>(x[i]);
    store8(static_cast<T*>(base) + at, e, n, v);
}
// (the type is the same for the whole call)
__device__ __forceinline__ void store8_type(int type, void* base, long long at, int e, int n, const float (&x)[8]) {
    if (type == BIQ_F32) store8_as<BIQ_F32>(base, at, e, n, x);
    else if (type == BIQ_BF16) store8_as<BIQ_BF16>(base, at, e, n, x);
    else store8_as<BIQ_F16>(base, at, e, n, x);
}

// Over the THREADS threads of a row; all of them get the result.
template <int THREADS, typename T, typename Join>
__device__ __forceinline__ T over_row(T x, T* lds, const Join& join) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) x = join(x, __shfl_xor(x, d));
    if constexpr (THREADS > 64) {
        __syncthreads();                                        // (what was exchanged before is read)
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
        __syncthreads();
        x = lds[0];
#pragma unroll
        for (int w = 1; w < THREADS / 64; ++w) x = join(x, lds[w]);
    }
    return x;
}
struct Add { template <typename T> __device__ __forceinline__ T operator()(T a, T b) const { return a + b; } };
struct Largest { __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return a > b ? a : b; } };

// 1 / sqrt(mean(s^2) + eps) as r up, up a power of two: without eps, rows of the least numbers there are have one beyond 32 bits.  (Infinite for zeros.)
struct Root { float r, up; };
__device__ __forceinline__ Root root64(double sum, int n, float eps) {
    const double root = 1.0 / sqrt(sum / n + static_cast<double>(eps));
    const float up = root > 0x1p120 ? 0x1p64f : 1.f;
    return {static_cast<float>(root / up), up};
}

// Codes of 8 values and their group's scale.  bits: the group's largest magnitude as an integer.
template <int FMT>
__device__ __forceinline__ void put_codes8(const NormParams& p, long long row, int e, const float (&t)[8], uint32_t bits, Root root) {
#pragma clang fp contract(off)
    const BlockScale b = block_scale<FMT>(bits, 0.f);
    const bool none = b.fresh == 0.f;                           // zeros, or a group that is NaN altogether
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = none ? 0.f : t[i] * b.fresh;
    const uint32_t lo = encode4<FMT>(v[0], v[1], v[2], v[3]), hi = encode4<FMT>(v[4], v[5], v[6], v[7]);
    uint8_t c[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        c[i] = static_cast<uint8_t>(lo >> (8 * i));
        c[4 + i] = static_cast<uint8_t>(hi >> (8 * i));
    }
    store8(p.codes + row * p.code_stride, e, p.n, c);
    // (0 for zeros, with any r that is a number)
    const float r = root.r == INFINITY ? 0x1.fffffep127f : root.r;
    if (p.group == 0 ? e == 0 : e % p.group == 0) p.scales[row * p.groups + (p.group == 0 ? 0 : e / p.group)] = b.scale * root.up * r;
}

// 1 / sqrt(sum / n + eps) where the sum of squares is a number that 32 bits hold with all their precision.
__device__ __forceinline__ float root_of(float sum, int n, float eps) { return 1.0f / sqrtf(sum / static_cast<float>(n) + eps); }
__device__ __forceinline__ bool sum_fits(float sum) { return sum >= 0x1p-90f && sum <= 0x1p120f; }

template <int TYPE, int THREADS, int K>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void norm_kernel(const NormParams p) {
#pragma clang fp contract(off)
    typedef typename Elem<TYPE>::T T;
    constexpr int ROWS = THREADS < 256 ? 256 / THREADS : 1;
    __shared__ double lds[16];
    const int me = threadIdx.x % THREADS;
    const long long row = static_cast<long long>(p.first + blockIdx.x) * ROWS + (ROWS > 1 ? threadIdx.x / THREADS : 0);
    if (row >= p.rows) return;                                  // (whole waves; a workgroup of one row has it)
    const T* x = static_cast<const T*>(p.x) + row * p.x_stride;
    const T* residual = static_cast<const T*>(p.residual) + row * p.residual_stride;
    T raw[K][8], more[K][8];
    float w[K][8], s[K][8];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int e = (k * THREADS + me) * 8;
        request8(raw[k], x, e < p.n ? e : p.n - 1, p.n);
        if (p.residual) request8(more[k], residual, e < p.n ? e : p.n - 1, p.n);
        if (p.weight) request8(w[k], p.weight, e < p.n ? e : p.n - 1, p.n);
    }
    float total = 0.f;
    uint32_t most[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int e = (k * THREADS + me) * 8;
        most[k] = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            s[k][i] = static_cast<float>(raw[k][i]);
            if (p.residual) s[k][i] += static_cast<float>(more[k][i]);
            w[k][i] = (p.weight ? w[k][i] : 1.f) + p.weight_add;
            if (e + i >= p.n) s[k][i] = w[k][i] = 0.f;
            total += s[k][i] * s[k][i];
            const uint32_t bits = __float_as_uint(s[k][i] * w[k][i]) & 0x7fffffffu;
            most[k] = most[k] > bits ? most[k] : bits;
        }
    }
    total = over_row<THREADS>(total, reinterpret_cast<float*>(lds), Add());
    Root root = {root_of(total, p.n, p.eps), 1.f};
    if (!sum_fits(total)) {                                     // squares that leave 32 bits: the same in 64
        double wide = 0.0;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) wide += static_cast<double>(s[k][i]) * s[k][i];
        wide = over_row<THREADS>(wide, lds, Add());
        root = root64(wide, p.n, p.eps);
    }
    if (p.sum) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int e = (k * THREADS + me) * 8;
            if (e < p.n) store8_as<TYPE>(p.sum, row * p.sum_stride, e, p.n, s[k]);
        }
    }
    if (p.y) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int e = (k * THREADS + me) * 8;
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = s[k][i] * root.up * root.r * w[k][i];
            if (e < p.n) store8_type(p.y_type, p.y, row * p.y_stride, e, p.n, y);
        }
    }
    if (!p.codes) return;
    uint32_t all = 0;
    if (p.group == 0) {
#pragma unroll
        for (int k = 0; k < K; ++k) all = all > most[k] ? all : most[k];
        all = over_row<THREADS>(all, reinterpret_cast<uint32_t*>(lds), Largest());
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int e = (k * THREADS + me) * 8;
        uint32_t bits = most[k];
        for (int d = 1; d < p.group / 8; d *= 2) {
            const uint32_t other = __shfl_xor(bits, d);
            bits = bits > other ? bits : other;
        }
        if (p.group == 0) bits = all;
        float t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = s[k][i] * w[k][i];
        if (e >= p.n) continue;
        if (p.format == BIQ_CACHE_INT8) put_codes8<BIQ_CACHE_INT8>(p, row, e, t, bits, root);
        else put_codes8<BIQ_CACHE_FP8>(p, row, e, t, bits, root);
    }
}

// Rows that registers do not hold are read twice: for the sum (and the largest magnitude), then to be written.
template <int TYPE>
__global__ __launch_bounds__(1024) void norm_long_kernel(const NormParams p) {
#pragma clang fp contract(off)
    typedef typename Elem<TYPE>::T T;
    __shared__ double lds[16];
    const long long row = p.first + blockIdx.x;
    const T* x = static_cast<const T*>(p.x) + row * p.x_stride;
    const T* residual = static_cast<const T*>(p.residual) + row * p.residual_stride;
    float s[8], w[8];
    auto read = [&](int e) {
        T raw[8], more[8];
        request8(raw, x, e, p.n);
        if (p.residual) request8(more, residual, e, p.n);
        if (p.weight) request8(w, p.weight, e, p.n);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            s[i] = static_cast<float>(raw[i]);
            if (p.residual) s[i] += static_cast<float>(more[i]);
            w[i] = (p.weight ? w[i] : 1.f) + p.weight_add;
            if (e + i >= p.n) s[i] = w[i] = 0.f;
        }
    };
    double total = 0.0;
    uint32_t all = 0;
    for (int e = threadIdx.x * 8; e < p.n; e += 8192) {
        read(e);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            total += static_cast<double>(s[i]) * s[i];
            const uint32_t bits = __float_as_uint(s[i] * w[i]) & 0x7fffffffu;
            all = all > bits ? all : bits;
        }
    }
    total = over_row<1024>(total, lds, Add());
    all = over_row<1024>(all, reinterpret_cast<uint32_t*>(lds), Largest());
    const Root root = root64(total, p.n, p.eps);
    // (all threads together, as groups are lanes' that exchange their largest)
    for (int e0 = 0; e0 < p.n; e0 += 8192) {
        const int e = e0 + threadIdx.x * 8;
        read(e < p.n ? e : p.n - 1);
        float y[8], t[8];
        uint32_t bits = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            y[i] = s[i] * root.up * root.r * w[i];
            t[i] = s[i] * w[i];
            const uint32_t b = __float_as_uint(t[i]) & 0x7fffffffu;
            bits = e < p.n && b > bits ? b : bits;
        }
        for (int d = 1; d < p.group / 8; d *= 2) {
            const uint32_t other = __shfl_xor(bits, d);
            bits = bits > other ? bits : other;
        }
        if (p.group == 0) bits = all;
        if (e >= p.n) continue;
        if (p.sum) store8_as<TYPE>(p.sum, row * p.sum_stride, e, p.n, s);
        if (p.y) store8_type(p.y_type, p.y, row * p.y_stride, e, p.n, y);
        if (!p.codes) continue;
        if (p.format == BIQ_CACHE_INT8) put_codes8<BIQ_CACHE_INT8>(p, row, e, t, bits, root);
        else put_codes8<BIQ_CACHE_FP8>(p, row, e, t, bits, root);
    }
}

}  // namespace biq
