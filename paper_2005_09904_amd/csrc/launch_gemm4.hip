// Launches of the products with 4-bit weights.
#include <type_traits>

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

template <int XT, int F, int NC, bool PER_BLOCK>
hipError_t many(int x_scales, Gemm4Params p, hipStream_t s) {
    static unsigned long long granted = 0;
    const auto kernel = gemm4_many_kernel<XT, F, NC, PER_BLOCK>;
    if (hipError_t e = grant_large_lds(reinterpret_cast<const void*>(kernel), granted, false); e != hipSuccess) return e;
    const int lds = 2 * (2 * 4 * kTerms4<XT> * 4 * 16 * NC * 16 + 2 * x_scales * 16 * NC * 4);
    const int row_groups = (p.tiles + 2 * kWaves4 - 1) / (2 * kWaves4);
    hipLaunchKernelGGL(kernel, dim3(row_groups * p.splits, (p.batch + p.columns - 1) / p.columns), dim3(64 * kWaves4), lds, s, p, x_scales);
    if (hipError_t e = hipGetLastError(); e != hipSuccess || p.splits == 1) return e;
    return launch_parts((4ll * p.tiles * p.batch + 255) / 256, 256, [&](unsigned first, unsigned grid) {
        p.first = first;
        hipLaunchKernelGGL(gemm4_join_kernel, dim3(grid), dim3(256), 0, s, p);
        return hipGetLastError();
    });
}
template <int XT, int F>
hipError_t many_f(int x_scales, const Gemm4Params& p, hipStream_t s) {
    auto columns = [&](auto per_block) {
        constexpr bool PER_BLOCK = decltype(per_block)::value;
        switch ((p.columns + 15) / 16) {
            case 1: return many<XT, F, 1, PER_BLOCK>(x_scales, p, s);
            case 2: return many<XT, F, 2, PER_BLOCK>(x_scales, p, s);
            case 3: return many<XT, F, 3, PER_BLOCK>(x_scales, p, s);
            default: return many<XT, F, 4, PER_BLOCK>(x_scales, p, s);
        }
    };
    if constexpr (F < 4 && (XT == kInt8 || XT == kFp8))
        if (x_scales > 1) return columns(std::false_type());
    return columns(std::true_type());
}
template <int XT>
hipError_t many_x(int f, int x_scales, const Gemm4Params& p, hipStream_t s) {
    return f == 4 ? many_f<XT, 4>(x_scales, p, s) : f == 2 ? many_f<XT, 2>(x_scales, p, s) : many_f<XT, 1>(x_scales, p, s);
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

hipError_t launch_gemm4_many(int x_type, int f, int x_scales, const Gemm4Params& p, hipStream_t s) {
    switch (x_type) {
        case BIQ_F32: return many_x<BIQ_F32>(f, x_scales, p, s);
        case BIQ_BF16: return many_x<BIQ_BF16>(f, x_scales, p, s);
        case BIQ_F16: return many_x<BIQ_F16>(f, x_scales, p, s);
        case kInt8: return many_x<kInt8>(f, x_scales, p, s);
        case kFp8: return many_x<kFp8>(f, x_scales, p, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace biq
