// Launches of the norm and logits kernels.
#include "biq_launch.h"
#include "biq_step_launch.h"

namespace biq {
namespace {

template <int TYPE, int THREADS, int K>
hipError_t norm_rows(NormParams p, hipStream_t s) {
    constexpr int ROWS = THREADS < 256 ? 256 / THREADS : 1, GROUP = THREADS < 256 ? 256 : THREADS;
    return launch_parts((static_cast<long long>(p.rows) + ROWS - 1) / ROWS, GROUP, [&](unsigned first, unsigned grid) {
        p.first = first;
        hipLaunchKernelGGL((norm_kernel<TYPE, THREADS, K>), dim3(grid), dim3(GROUP), 0, s, p);
        return hipGetLastError();
    });
}

template <int TYPE>
hipError_t norm_t(NormParams p, hipStream_t s) {
    if (p.n <= 512) return norm_rows<TYPE, 64, 1>(p, s);
    if (p.n <= 2048) return norm_rows<TYPE, 256, 1>(p, s);
    if (p.n <= 4096) return norm_rows<TYPE, 256, 2>(p, s);
    if (p.n <= 8192) return norm_rows<TYPE, 1024, 1>(p, s);
    if (p.n <= 16384) return norm_rows<TYPE, 1024, 2>(p, s);
    return launch_parts(p.rows, 1024, [&](unsigned first, unsigned grid) {
        p.first = first;
        hipLaunchKernelGGL(norm_long_kernel<TYPE>, dim3(grid), dim3(1024), 0, s, p);
        return hipGetLastError();
    });
}

template <int TYPE, int WHAT>
hipError_t logits_pass(LogitsParams p, hipStream_t s) {
    const int lds = 4 * kLogitsSpan * ((p.history || p.drafts ? 1 : 0) + (p.biases > 0 ? 1 : 0));
    return launch_parts(static_cast<long long>(p.seqs) * p.spans, 256, [&](unsigned first, unsigned grid) {
        p.first = first;
        hipLaunchKernelGGL((logits_kernel<TYPE, 256, kLogitsSpan / 2048, WHAT>), dim3(grid), dim3(256), lds, s, p);
        return hipGetLastError();
    });
}

template <int TYPE>
hipError_t logits_t(bool probabilities, const LogitsParams& p, hipStream_t s) {
    if (!probabilities) return logits_pass<TYPE, 0>(p, s);
    if (p.spans == 1) return logits_pass<TYPE, 3>(p, s);
    if (hipError_t e = logits_pass<TYPE, 1>(p, s); e != hipSuccess) return e;
    return logits_pass<TYPE, 2>(p, s);
}

}  // namespace

hipError_t launch_norm(int type, const NormParams& p, hipStream_t s) {
    switch (type) {
        case BIQ_F32: return norm_t<BIQ_F32>(p, s);
        case BIQ_BF16: return norm_t<BIQ_BF16>(p, s);
        case BIQ_F16: return norm_t<BIQ_F16>(p, s);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_logits(int type, bool probabilities, const LogitsParams& p, hipStream_t s) {
    switch (type) {
        case BIQ_F32: return logits_t<BIQ_F32>(probabilities, p, s);
        case BIQ_BF16: return logits_t<BIQ_BF16>(probabilities, p, s);
        case BIQ_F16: return logits_t<BIQ_F16>(probabilities, p, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace biq
