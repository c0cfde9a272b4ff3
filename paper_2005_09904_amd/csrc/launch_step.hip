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

template <int TYPE, int THREADS, int U, int WHAT>
hipError_t logits_pass(LogitsParams p, hipStream_t s) {
    const int lds = 16 * (THREADS / 64) + 4 * THREADS * U * 8 * ((p.history || p.drafts ? 1 : 0) + (p.biases > 0 ? 1 : 0));
    return launch_parts(static_cast<long long>(p.seqs) * p.spans, THREADS, [&](unsigned first, unsigned grid) {
        p.first = first;
        return launch_large_lds<logits_kernel<TYPE, THREADS, U, WHAT>, false>(p, static_cast<int>(grid), THREADS, lds, s);
    });
}

template <int TYPE>
hipError_t logits_t(bool probabilities, bool whole, LogitsParams p, hipStream_t s) {
    if (!probabilities) return logits_pass<TYPE, 256, kLogitsSpan / 2048, 0>(p, s);
    if (whole) {
        p.spans = 1;
        if (p.vocab <= 2048) return logits_pass<TYPE, 256, 1, 3>(p, s);
        if (p.vocab <= 8192) return logits_pass<TYPE, 1024, 1, 3>(p, s);
        if (p.vocab <= 16384) return logits_pass<TYPE, 1024, 2, 3>(p, s);
        return logits_pass<TYPE, 1024, 4, 3>(p, s);
    }
    if (hipError_t e = logits_pass<TYPE, 256, kLogitsSpan / 2048, 1>(p, s); e != hipSuccess) return e;
    return logits_pass<TYPE, 256, kLogitsSpan / 2048, 2>(p, s);
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

hipError_t launch_logits(int type, bool probabilities, bool whole, const LogitsParams& p, hipStream_t s) {
    switch (type) {
        case BIQ_F32: return logits_t<BIQ_F32>(probabilities, whole, p, s);
        case BIQ_BF16: return logits_t<BIQ_BF16>(probabilities, whole, p, s);
        case BIQ_F16: return logits_t<BIQ_F16>(probabilities, whole, p, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace biq
