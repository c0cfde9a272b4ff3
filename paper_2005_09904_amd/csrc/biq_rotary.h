// Rotary positions (biq_rotary).
#pragma once

#include "biq_cache.h"

namespace biq {

struct RotaryParams {
    Rows x, y;
    const int* positions;
    Rotation rotation;
    int rows, heads, dim, inverse, copy;    // copy: y is another tensor, what is not turned is copied
    unsigned first;                         // first workgroup of this launch (rotary_kernel)
};

// One thread per row, head and pair (or element that is not turned): any sizes, strides and alignment.
template <int TYPE>
__global__ __launch_bounds__(256) void rotary_kernel(const RotaryParams p) {
    const int half = p.rotation.rot / 2, items = half + (p.copy ? p.dim - p.rotation.rot : 0);
    const long long at = static_cast<long long>(p.first + blockIdx.x) * 256 + threadIdx.x;
    const int item = static_cast<int>(at % items);
    const long long rh = at / items;
    const int head = static_cast<int>(rh % p.heads);
    const long long row = rh / p.heads;
    if (row >= p.rows) return;
    const long long x0 = row * p.x.row_stride + head * p.x.head_stride, y0 = row * p.y.row_stride + head * p.y.head_stride;
    if (item >= half) {
        const int d = item + half;
        store_elem<TYPE>(p.y.data, y0 + d, load_elem<TYPE>(p.x.data, x0 + d));
        return;
    }
    const int pos = p.positions[row];
    const bool known = pos >= 0 && pos < p.rotation.positions;
    const f32x2 cs = *reinterpret_cast<const f32x2*>(p.rotation.angles + static_cast<long long>(known ? pos : 0) * p.rotation.rot + 2 * item);
    const float c = known ? cs[0] : __uint_as_float(0x7fc00000u), s = p.inverse ? -cs[1] : cs[1];
    const int da = p.rotation.interleaved ? 2 * item : item, db = p.rotation.interleaved ? da + 1 : item + half;
    const float a = load_elem<TYPE>(p.x.data, x0 + da), b = load_elem<TYPE>(p.x.data, x0 + db);
    store_elem<TYPE>(p.y.data, y0 + da, turned(a, b, c, s, false));
    store_elem<TYPE>(p.y.data, y0 + db, turned(b, a, c, s, true));
}

// Memory bounds it: 16 bytes a lane and access, and a row's angles are read once for kHeads heads.  V elements are one access;
// a thread has one access of pairs (interleaved), two that form pairs (halves), or one that is copied, of the heads first,
// first + groups, ..  For parts of a head that are multiples of V on 16-byte aligned rows.  16384 rows of 40 heads of 128 in
// bf16 (336 MB): 62 us, 5.4 TB/s (a thread per pair: 165).
constexpr int kRotaryHeads = 4;
template <int TYPE, bool INTERLEAVED>
__global__ __launch_bounds__(256) void rotary_wide_kernel(const RotaryParams p, uint32_t items, uint32_t groups, uint32_t threads) {
    constexpr int V = TYPE == BIQ_F32 ? 4 : 8, PAIRS = INTERLEAVED ? V / 2 : V;
    typedef typename Elem<TYPE>::T T;
    typedef T Vec __attribute__((ext_vector_type(V)));
    const uint32_t at = blockIdx.x * 256u + threadIdx.x;
    if (at >= threads) return;
    const uint32_t rg = at / items, item = at - rg * items, row = rg / groups, first = rg - row * groups;
    const uint32_t half = p.rotation.rot / 2, turning = INTERLEAVED ? 2 * half / V : half / V;
    const bool turn = item < turning;
    // elements of the access (and of its partner, half a part further)
    const uint32_t d = turn ? item * V : p.rotation.rot + (item - turning) * V;
    const T* x = static_cast<const T*>(p.x.data) + row * p.x.row_stride + d;
    T* y = static_cast<T*>(p.y.data) + row * p.y.row_stride + d;
    Vec a[kRotaryHeads], b[kRotaryHeads];
#pragma unroll
    for (int i = 0; i < kRotaryHeads; ++i) {
        const uint32_t h = first + i * groups;
        if (h >= static_cast<uint32_t>(p.heads)) continue;
        a[i] = *reinterpret_cast<const Vec*>(x + h * p.x.head_stride);
        if (!INTERLEAVED && turn) b[i] = *reinterpret_cast<const Vec*>(x + h * p.x.head_stride + half);
    }
    float c[PAIRS], s[PAIRS];
    if (turn) {
        const int pos = p.positions[row];
        const bool known = pos >= 0 && pos < p.rotation.positions;
        const f32x2* angles = reinterpret_cast<const f32x2*>(p.rotation.angles + static_cast<long long>(known ? pos : 0) * p.rotation.rot) + item * PAIRS;
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
            const f32x2 cs = angles[i];
            c[i] = known ? cs[0] : __uint_as_float(0x7fc00000u);
            s[i] = p.inverse ? -cs[1] : cs[1];
        }
    }
#pragma unroll
    for (int i = 0; i < kRotaryHeads; ++i) {
        const uint32_t h = first + i * groups;
        if (h >= static_cast<uint32_t>(p.heads)) continue;
        T* to = y + h * p.y.head_stride;
        Vec ra = a[i], rb;
        if (turn) {
#pragma unroll
            for (int j = 0; j < PAIRS; ++j) {
                if constexpr (INTERLEAVED) {
                    const float u = static_cast<float>(a[i][2 * j]), v = static_cast<float>(a[i][2 * j + 1]);
                    ra[2 * j] = static_cast<T>(turned(u, v, c[j], s[j], false));
                    ra[2 * j + 1] = static_cast<T>(turned(v, u, c[j], s[j], true));
                } else {
                    const float u = static_cast<float>(a[i][j]), v = static_cast<float>(b[i][j]);
                    ra[j] = static_cast<T>(turned(u, v, c[j], s[j], false));
                    rb[j] = static_cast<T>(turned(v, u, c[j], s[j], true));
                }
            }
            if constexpr (!INTERLEAVED) *reinterpret_cast<Vec*>(to + half) = rb;
        }
        *reinterpret_cast<Vec*>(to) = ra;
    }
}

}  // namespace biq
