// Rotary positions and their table; verification of drafted tokens.
#include "biq_serve_launch.h"

namespace biq {
namespace {

// The product is reduced to a part of a turn in 64 bits (2^-53 of the turns in all), then to 32 bits.
__global__ __launch_bounds__(256) void rotary_table_kernel(const double* turns, float* angles, int pairs, int first, int positions,
                                                           double amplitude, unsigned first_group) {
    const long long at = static_cast<long long>(first_group + blockIdx.x) * 256 + threadIdx.x;
    if (at >= static_cast<long long>(positions) * pairs) return;
    const long long row = at / pairs;
    double t = static_cast<double>(first + row) * turns[at - row * pairs];
    t -= rint(t);
    double s, c;
    sincospi(2.0 * t, &s, &c);
    angles[2 * at] = static_cast<float>(amplitude * c);
    angles[2 * at + 1] = static_cast<float>(amplitude * s);
}

template <int TYPE>
hipError_t rotary_t(RotaryParams p, hipStream_t s) {
    constexpr int V = TYPE == BIQ_F32 ? 4 : 8;
    const int rot = p.rotation.rot, part = p.rotation.interleaved ? rot : rot / 2, rest = p.dim - rot;
    auto wide = [](const Rows& r) {
        return (reinterpret_cast<uintptr_t>(r.data) & 15) == 0 && r.row_stride % V == 0 && r.head_stride % V == 0;
    };
    if (part % V == 0 && (!p.copy || rest % V == 0) && wide(p.x) && wide(p.y)) {
        // a thread per access and head while all of them are on the GPU at once, then one for kRotaryHeads heads
        const long long items = part / V + (p.copy ? rest / V : 0);
        const long long all = items * p.heads * p.rows;
        const int groups = all < 1024 * 256 ? p.heads : (p.heads + kRotaryHeads - 1) / kRotaryHeads;
        const long long threads = items * groups * p.rows;
        if (threads < 0x7fffff00) {
            const dim3 grid(static_cast<unsigned>((threads + 255) / 256));
            if (p.rotation.interleaved)
                hipLaunchKernelGGL((rotary_wide_kernel<TYPE, true>), grid, dim3(256), 0, s, p, static_cast<uint32_t>(items),
                                   static_cast<uint32_t>(groups), static_cast<uint32_t>(threads));
            else
                hipLaunchKernelGGL((rotary_wide_kernel<TYPE, false>), grid, dim3(256), 0, s, p, static_cast<uint32_t>(items),
                                   static_cast<uint32_t>(groups), static_cast<uint32_t>(threads));
            return hipGetLastError();
        }
    }
    const int items = rot / 2 + (p.copy ? rest : 0);
    const long long threads = static_cast<long long>(p.rows) * p.heads * items;
    return launch_parts((threads + 255) / 256, 256, [&](unsigned first, unsigned grid) {
        p.first = first;
        hipLaunchKernelGGL(rotary_kernel<TYPE>, dim3(grid), dim3(256), 0, s, p);
        return hipGetLastError();
    });
}

template <int TYPE>
hipError_t verify_t(VerifyParams p, hipStream_t s) {
    if (p.spans <= kVerifyOneSpans) {
        hipLaunchKernelGGL(verify_one_kernel<TYPE>, dim3(p.seqs), dim3(kVerifyThreads), 0, s, p);
        return hipGetLastError();
    }
    const hipError_t e = launch_parts(static_cast<long long>(p.seqs) * ((p.spans + 3) / 4), 256, [&](unsigned first, unsigned grid) {
        p.first = first;
        hipLaunchKernelGGL(verify_sums_kernel<TYPE>, dim3(grid), dim3(256), 0, s, p);
        return hipGetLastError();
    });
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(verify_draw_kernel<TYPE>, dim3(p.seqs), dim3(kVerifyThreads), 0, s, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(int type, const RotaryParams& p, hipStream_t s) {
    switch (type) {
        case BIQ_F32: return rotary_t<BIQ_F32>(p, s);
        case BIQ_BF16: return rotary_t<BIQ_BF16>(p, s);
        case BIQ_F16: return rotary_t<BIQ_F16>(p, s);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_rotary_table(const double* turns, float* angles, int pairs, int first, int positions, double amplitude,
                               hipStream_t s) {
    const long long threads = static_cast<long long>(positions) * pairs;
    return launch_parts((threads + 255) / 256, 256, [&](unsigned first_group, unsigned grid) {
        hipLaunchKernelGGL(rotary_table_kernel, dim3(grid), dim3(256), 0, s, turns, angles, pairs, first, positions, amplitude, first_group);
        return hipGetLastError();
    });
}

hipError_t launch_verify(int type, const VerifyParams& p, hipStream_t s) {
    switch (type) {
        case BIQ_F32: return verify_t<BIQ_F32>(p, s);
        case BIQ_BF16: return verify_t<BIQ_BF16>(p, s);
        case BIQ_F16: return verify_t<BIQ_F16>(p, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace biq
