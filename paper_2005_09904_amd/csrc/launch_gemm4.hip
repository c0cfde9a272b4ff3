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

// launch(spans of 32 elements that share both scales, that share the weights'): the same but for codes with smaller groups than the weights'.
template <int N> using Spans = std::integral_constant<int, N>;
template <int XT, typename Launch>
hipError_t by_spans(int f, int g, const Launch& launch) {
    if (f == g) return g == 4 ? launch(Spans<4>(), Spans<4>()) : g == 2 ? launch(Spans<2>(), Spans<2>()) : launch(Spans<1>(), Spans<1>());
    if constexpr (XT == kInt8 || XT == kFp8) {
        if (f == 2) return launch(Spans<2>(), Spans<4>());
        return g == 4 ? launch(Spans<1>(), Spans<4>()) : launch(Spans<1>(), Spans<2>());
    }
    return hipErrorInvalidValue;
}

template <int XT>
hipError_t few(int f, int g, int x_scales, int lds, const Gemm4Params& p, hipStream_t s) {
    return by_spans<XT>(f, g, [&](auto spans, auto weights) {
        static unsigned long long granted = 0;
        const auto kernel = gemm4_few_kernel<XT, decltype(spans)::value, decltype(weights)::value>;
        if (hipError_t e = grant_large_lds(reinterpret_cast<const void*>(kernel), granted, false); e != hipSuccess) return e;
        const int per = kWaves4 / p.splits;
        hipLaunchKernelGGL(kernel, dim3((p.tiles + per - 1) / per, (p.batch + 15) / 16), dim3(64 * kWaves4), lds, s, p, x_scales);
        return hipGetLastError();
    });
}

template <int XT, int F, int G, int NC, bool PER_BLOCK>
hipError_t many(int x_scales, Gemm4Params p, hipStream_t s) {
    static unsigned long long granted = 0;
    const auto kernel = gemm4_many_kernel<XT, F, G, NC, PER_BLOCK>;
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
template <int XT, int F, int G>
hipError_t many_f(int x_scales, const Gemm4Params& p, hipStream_t s) {
    auto columns = [&](auto per_block) {
        constexpr bool PER_BLOCK = decltype(per_block)::value;
        switch ((p.columns + 15) / 16) {
            case 1: return many<XT, F, G, 1, PER_BLOCK>(x_scales, p, s);
            case 2: return many<XT, F, G, 2, PER_BLOCK>(x_scales, p, s);
            case 3: return many<XT, F, G, 3, PER_BLOCK>(x_scales, p, s);
            default: return many<XT, F, G, 4, PER_BLOCK>(x_scales, p, s);
        }
    };
    if constexpr (F < 4 && (XT == kInt8 || XT == kFp8))
        if (x_scales > 1) return columns(std::false_type());
    return columns(std::true_type());
}
template <int XT>
hipError_t many_x(int f, int g, int x_scales, const Gemm4Params& p, hipStream_t s) {
    return by_spans<XT>(f, g, [&](auto spans, auto weights) { return many_f<XT, decltype(spans)::value, decltype(weights)::value>(x_scales, p, s); });
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

hipError_t launch_gemm4_few(int x_type, int f, int g, int x_scales, int lds, const Gemm4Params& p, hipStream_t s) {
    switch (x_type) {
        case BIQ_F32: return few<BIQ_F32>(f, g, x_scales, lds, p, s);
        case BIQ_BF16: return few<BIQ_BF16>(f, g, x_scales, lds, p, s);
        case BIQ_F16: return few<BIQ_F16>(f, g, x_scales, lds, p, s);
        case kInt8: return few<kInt8>(f, g, x_scales, lds, p, s);
        case kFp8: return few<kFp8>(f, g, x_scales, lds, p, s);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_gemm4_many(int x_type, int f, int g, int x_scales, const Gemm4Params& p, hipStream_t s) {
    switch (x_type) {
        case BIQ_F32: return many_x<BIQ_F32>(f, g, x_scales, p, s);
        case BIQ_BF16: return many_x<BIQ_BF16>(f, g, x_scales, p, s);
        case BIQ_F16: return many_x<BIQ_F16>(f, g, x_scales, p, s);
        case kInt8: return many_x<kInt8>(f, g, x_scales, p, s);
        case kFp8: return many_x<kFp8>(f, g, x_scales, p, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace biq
