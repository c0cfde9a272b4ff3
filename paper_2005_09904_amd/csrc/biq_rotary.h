// Rotary positions (biq_rotary).
#pragma once

#include "biq_cache.h"

namespace biq {

struct RotaryParams {
    Rows x, y;
    const int* positions;
    Rotation rotation;
    int rows, heads, dim, inverse, copy;    // copy: y is another tensor, what is not turned is copied
};

// One thread per row, head and pair (or element that is not turned).
template <int TYPE>
__global__ __launch_bounds__(256) void rotary_kernel(const RotaryParams p) {
    const int half = p.rotation.rot / 2, items = half + (p.copy ? p.dim - p.rotation.rot : 0);
    const long long at = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x;
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

}  // namespace biq
