// Launches of the products with 4-bit weights.
#include "biq_launch.h"
#include "biq_step_launch.h"

namespace biq {
namespace {

template <typename Kernel>
hipError_t per_record(Kernel kernel, Pack4Params p, long long records, hipStream_t s) {
    return launch_parts(records, 256, [&](unsigned first, unsigned grid) {
        p.first = first;
        hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, s, p);
        return hipGetLastError();
    });
}

template <int XT, int F>
hipError_t few(int x_scales, int lds, const Gemm4Params& p, hipStream_t s) {
    static unsigned long long granted = 0;
    const auto kernel = gemm4_few_kernel<XT, F>;
    if (hipError_t e = grant_large_lds(reinterpret_cast<const void*>(kernel), granted, false); e != hipSuccess) return e;
    const int per = kWaves4 / p.splits;
    hipLaunchKernelGGL(kernel, dim3((p.tiles + per - 1) / per, (p.batch + 15) / 16), dim3(64 * kWaves4), lds, s, p, x_scales);
    return hipGetLastError();
}
template <int XT>
hipError_t few_x(int f, int x_scales, int lds, const Gemm4Params& p, hipStream_t s) {
    return f == 4 ? few<XT, 4>(x_scales, lds, p, s) : f == 2 ? few<XT, 2>(x_scales, lds, p, s) : few<XT, 1>(x_scales, lds, p, s);
}

template <int TERMS, int F, int NC>
hipError_t many(int x_scales, long long group_bytes, const Gemm4Params& p, hipStream_t s) {
    const int per = kWaves4 / p.splits;
    hipLaunchKernelGGL((gemm4_many_kernel<TERMS, F, NC>), dim3((p.tiles + per - 1) / per, (p.batch + p.columns - 1) / p.columns), dim3(64 * kWaves4), 0, s, p,
                       x_scales, group_bytes);
    return hipGetLastError();
}
template <int TERMS, int F>
hipError_t many_f(int x_scales, long long group_bytes, const Gemm4Params& p, hipStream_t s) {
    switch ((p.columns + 15) / 16) {
        case 1: return many<TERMS, F, 1>(x_scales, group_bytes, p, s);
        case 2: return many<TERMS, F, 2>(x_scales, group_bytes, p, s);
        case 3: return many<TERMS, F, 3>(x_scales, group_bytes, p, s);
        default: return many<TERMS, F, 4>(x_scales, group_bytes, p, s);
    }
}
template <int XT>
hipError_t many_x(int f, int x_scales, long long group_bytes, const Gemm4Params& p, hipStream_t s) {
    hipLaunchKernelGGL(gemm4_operands_kernel<XT>, dim3((p.blocks + 15) / 16, p.batch), dim3(256), 0, s, p, x_scales, group_bytes);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    constexpr int terms = kTerms4<XT>;
    return f == 4 ? many_f<terms, 4>(x_scales, group_bytes, p, s)
                  : f == 2 ? many_f<terms, 2>(x_scales, group_bytes, p, s) : many_f<terms, 1>(x_scales, group_bytes, p, s);
}

}  // namespace

hipError_t launch_pack4(const Pack4Params& p, long long records, hipStream_t s) { return per_record(pack4_kernel, p, records, s); }
hipError_t launch_unpack4(const Pack4Params& p, long long records, hipStream_t s) { return per_record(unpack4_kernel, p, records, s); }
hipError_t launch_quantize4(int type, const Pack4Params& p, long long records, hipStream_t s) {
    switch (type) {
        case BIQ_F32: return per_record(quantize4_kernel<BIQ_F32>, p, records, s);
        case BIQ_BF16: return per_record(quantize4_kernel<BIQ_BF16>, p, records, s);
        case BIQ_F16: return per_record(quantize4_kernel<BIQ_F16>, p, records, s);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_gemm4_few(int x_type, int f, int x_scales, int lds, const Gemm4Params& p, hipStream_t s) {
    switch (x_type) {
        case BIQ_F32: return few_x<BIQ_F32>(f, x_scales, lds, p, s);
        case BIQ_BF16: return few_x<BIQ_BF16>(f, x_scales, lds, p, s);
        case BIQ_F16: return few_x<BIQ_F16>(f, x_scales, lds, p, s);
        case kInt8: return few_x<kInt8>(f, x_scales, lds, p, s);
        case kFp8: return few_x<kFp8>(f, x_scales, lds, p, s);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_gemm4_many(int x_type, int f, int x_scales, long long group_bytes, const Gemm4Params& p, hipStream_t s) {
    switch (x_type) {
        case BIQ_F32: return many_x<BIQ_F32>(f, x_scales, group_bytes, p, s);
        case BIQ_BF16: return many_x<BIQ_BF16>(f, x_scales, group_bytes, p, s);
        case BIQ_F16: return many_x<BIQ_F16>(f, x_scales, group_bytes, p, s);
        case kInt8: return many_x<kInt8>(f, x_scales, group_bytes, p, s);
        case kFp8: return many_x<kFp8>(f, x_scales, group_bytes, p, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace biq
