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

// The fewest threads that hold a row in 8 or 16 elements each, and so the most rows on a CU: in bfloat16, 8192 rows of 512 take 9.7 us (with 256
// threads a row 16.8), of 2048 28.8 (two parts of 256 threads 39.0), of 4096 55 (1024 threads 77), of 8192 109 (two parts 174), of 16384 241.  One row
// takes the same within 0.3 us, but 3.2 instead of 4.4 at 8192.
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

// 8 tokens a thread in spans (spans of 4096 tokens took the same), and whole rows by as few threads as hold them.
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
