// The cache's writer and reader, one instantiation per element type, code format and head size in steps of 64.
#include "biq_serve_launch.h"

namespace biq {
namespace {

template <int TYPE, int FMT>
hipError_t append_t(int chunks, const AppendParams& p, dim3 grid, hipStream_t s) {
    switch (chunks) {
        case 1: hipLaunchKernelGGL((cache_append_kernel<TYPE, FMT, 1>), grid, dim3(256), 0, s, p); break;
        case 2: hipLaunchKernelGGL((cache_append_kernel<TYPE, FMT, 2>), grid, dim3(256), 0, s, p); break;
        case 3: hipLaunchKernelGGL((cache_append_kernel<TYPE, FMT, 3>), grid, dim3(256), 0, s, p); break;
        case 4: hipLaunchKernelGGL((cache_append_kernel<TYPE, FMT, 4>), grid, dim3(256), 0, s, p); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

template <int TYPE, int FMT>
hipError_t read_t(int chunks, const ReadParams& p, dim3 grid, hipStream_t s) {
    switch (chunks) {
        case 1: hipLaunchKernelGGL((cache_read_kernel<TYPE, FMT, 1>), grid, dim3(256), 0, s, p); break;
        case 2: hipLaunchKernelGGL((cache_read_kernel<TYPE, FMT, 2>), grid, dim3(256), 0, s, p); break;
        case 3: hipLaunchKernelGGL((cache_read_kernel<TYPE, FMT, 3>), grid, dim3(256), 0, s, p); break;
        case 4: hipLaunchKernelGGL((cache_read_kernel<TYPE, FMT, 4>), grid, dim3(256), 0, s, p); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

// Workgroups of four waves, a wave per head, kind (keys, values) and block.
template <typename P>
dim3 block_grid(const P& p) {
    return dim3(static_cast<unsigned>(p.seqs) * p.blocks * ((2 * p.cache.heads + 3) / 4));
}

}  // namespace

hipError_t launch_append(int type, int fmt, int chunks, const AppendParams& p, hipStream_t s) {
    const dim3 grid = block_grid(p);
    const bool int8 = fmt == BIQ_CACHE_INT8;
    switch (type) {
        case BIQ_F32: return int8 ? append_t<BIQ_F32, BIQ_CACHE_INT8>(chunks, p, grid, s) : append_t<BIQ_F32, BIQ_CACHE_FP8>(chunks, p, grid, s);
        case BIQ_BF16: return int8 ? append_t<BIQ_BF16, BIQ_CACHE_INT8>(chunks, p, grid, s) : append_t<BIQ_BF16, BIQ_CACHE_FP8>(chunks, p, grid, s);
        case BIQ_F16: return int8 ? append_t<BIQ_F16, BIQ_CACHE_INT8>(chunks, p, grid, s) : append_t<BIQ_F16, BIQ_CACHE_FP8>(chunks, p, grid, s);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_read(int type, int fmt, int chunks, const ReadParams& p, hipStream_t s) {
    const dim3 grid = block_grid(p);
    const bool int8 = fmt == BIQ_CACHE_INT8;
    switch (type) {
        case BIQ_F32: return int8 ? read_t<BIQ_F32, BIQ_CACHE_INT8>(chunks, p, grid, s) : read_t<BIQ_F32, BIQ_CACHE_FP8>(chunks, p, grid, s);
        case BIQ_BF16: return int8 ? read_t<BIQ_BF16, BIQ_CACHE_INT8>(chunks, p, grid, s) : read_t<BIQ_BF16, BIQ_CACHE_FP8>(chunks, p, grid, s);
        case BIQ_F16: return int8 ? read_t<BIQ_F16, BIQ_CACHE_INT8>(chunks, p, grid, s) : read_t<BIQ_F16, BIQ_CACHE_FP8>(chunks, p, grid, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace biq
