// The cache's writer and reader, one instantiation per element type, code format and head size in steps of 64.
#include "biq_serve_launch.h"

namespace biq {
namespace {

// Workgroups of four waves, a wave per head, kind (keys, values) and block.
template <typename P, typename Launch>
hipError_t blocks_of(P& p, const Launch& launch) {
    return launch_parts(static_cast<long long>(p.seqs) * p.blocks * ((2 * p.cache.heads + 3) / 4), 256, [&](unsigned first, unsigned grid) {
        p.first = first;
        launch(grid);
        return hipGetLastError();
    });
}

template <int TYPE, int FMT>
hipError_t append_t(int chunks, AppendParams p, hipStream_t s) {
    return blocks_of(p, [&](unsigned grid) {
        switch (chunks) {
            case 1: hipLaunchKernelGGL((cache_append_kernel<TYPE, FMT, 1>), dim3(grid), dim3(256), 0, s, p); break;
            case 2: hipLaunchKernelGGL((cache_append_kernel<TYPE, FMT, 2>), dim3(grid), dim3(256), 0, s, p); break;
            case 3: hipLaunchKernelGGL((cache_append_kernel<TYPE, FMT, 3>), dim3(grid), dim3(256), 0, s, p); break;
            case 4: hipLaunchKernelGGL((cache_append_kernel<TYPE, FMT, 4>), dim3(grid), dim3(256), 0, s, p); break;
        }
    });
}

template <int TYPE, int FMT>
hipError_t read_t(int chunks, ReadParams p, hipStream_t s) {
    return blocks_of(p, [&](unsigned grid) {
        switch (chunks) {
            case 1: hipLaunchKernelGGL((cache_read_kernel<TYPE, FMT, 1>), dim3(grid), dim3(256), 0, s, p); break;
            case 2: hipLaunchKernelGGL((cache_read_kernel<TYPE, FMT, 2>), dim3(grid), dim3(256), 0, s, p); break;
            case 3: hipLaunchKernelGGL((cache_read_kernel<TYPE, FMT, 3>), dim3(grid), dim3(256), 0, s, p); break;
            case 4: hipLaunchKernelGGL((cache_read_kernel<TYPE, FMT, 4>), dim3(grid), dim3(256), 0, s, p); break;
        }
    });
}

}  // namespace

hipError_t launch_append(int type, int fmt, int chunks, const AppendParams& p, hipStream_t s) {
    const bool int8 = fmt == BIQ_CACHE_INT8;
    switch (type) {
        case BIQ_F32: return int8 ? append_t<BIQ_F32, BIQ_CACHE_INT8>(chunks, p, s) : append_t<BIQ_F32, BIQ_CACHE_FP8>(chunks, p, s);
        case BIQ_BF16: return int8 ? append_t<BIQ_BF16, BIQ_CACHE_INT8>(chunks, p, s) : append_t<BIQ_BF16, BIQ_CACHE_FP8>(chunks, p, s);
        case BIQ_F16: return int8 ? append_t<BIQ_F16, BIQ_CACHE_INT8>(chunks, p, s) : append_t<BIQ_F16, BIQ_CACHE_FP8>(chunks, p, s);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_read(int type, int fmt, int chunks, const ReadParams& p, hipStream_t s) {
    const bool int8 = fmt == BIQ_CACHE_INT8;
    switch (type) {
        case BIQ_F32: return int8 ? read_t<BIQ_F32, BIQ_CACHE_INT8>(chunks, p, s) : read_t<BIQ_F32, BIQ_CACHE_FP8>(chunks, p, s);
        case BIQ_BF16: return int8 ? read_t<BIQ_BF16, BIQ_CACHE_INT8>(chunks, p, s) : read_t<BIQ_BF16, BIQ_CACHE_FP8>(chunks, p, s);
        case BIQ_F16: return int8 ? read_t<BIQ_F16, BIQ_CACHE_INT8>(chunks, p, s) : read_t<BIQ_F16, BIQ_CACHE_FP8>(chunks, p, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace biq
