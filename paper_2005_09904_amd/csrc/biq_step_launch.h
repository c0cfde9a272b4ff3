// Internal interface between the checks of the operators at the end of a decoder step (step_api.hip) and the translation units
// that instantiate and launch their kernels.  Not part of the ABI.
#pragma once

#include "biq_gemm4.h"
#include "biq_logits.h"
#include "biq_norm.h"
#include "biq_serve_launch.h"

namespace biq {

hipError_t launch_norm(int type, const NormParams& p, hipStream_t s);

hipError_t launch_pack4(const Pack4Params& p, long long records, hipStream_t s);
hipError_t launch_quantize4(int type, const Pack4Params& p, long long records, hipStream_t s);
hipError_t launch_unpack4(const Pack4Params& p, long long records, hipStream_t s);
// (x_scales: scales of X in 128 elements; f: spans of 32 elements that share both scales, g: the weights')
hipError_t launch_gemm4_few(int x_type, int f, int g, int x_scales, int lds, const Gemm4Params& p, hipStream_t s);
hipError_t launch_gemm4_many(int x_type, int f, int g, int x_scales, const Gemm4Params& p, hipStream_t s);

// Tokens of a span of the vocabulary.
constexpr int kLogitsSpan = 2048;
// (whole: a workgroup for a row)
hipError_t launch_logits(int type, bool probabilities, bool whole, const LogitsParams& p, hipStream_t s);

}  // namespace biq
