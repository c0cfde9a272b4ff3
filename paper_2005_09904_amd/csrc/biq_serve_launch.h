// Internal interface between the checks of the decoder-step operators (serve_api.hip) and the translation units that
// instantiate and launch their kernels.  Not part of the ABI.
#pragma once

#include "biq_attention.h"
#include "biq_rotary.h"
#include "biq_verify.h"

namespace biq {

// A launch has fewer than 2^32 threads, so larger grids go in parts: launch(first workgroup, workgroups).  Parts are multiples of
// the XCDs, so that workgroups keep to theirs.
template <typename Launch>
hipError_t launch_parts(long long workgroups, int threads, const Launch& launch) {
    const long long most = 0xffffffffll / threads / kXcds * kXcds;
    for (long long first = 0; first < workgroups; first += most) {
        const long long part = workgroups - first < most ? workgroups - first : most;
        if (hipError_t e = launch(static_cast<unsigned>(first), static_cast<unsigned>(part)); e != hipSuccess) return e;
    }
    return hipSuccess;
}

// (tiles: the kernel for many rows; nt: tiles of 16 rows per wave; waves: per workgroup)
hipError_t launch_attend_f32(int fmt, bool tiles, int nt, int waves, const AttendParams& p, hipStream_t s);
hipError_t launch_attend_bf16(int fmt, bool tiles, int nt, int waves, const AttendParams& p, hipStream_t s);
hipError_t launch_attend_f16(int fmt, bool tiles, int nt, int waves, const AttendParams& p, hipStream_t s);

// `groups` workgroups with pieces of the shared tokens and of the sequences' own ones, and the results joined of `sets` partial ones.
hipError_t launch_attend_shared_f32(int fmt, bool tiles, int nt, long long groups, const AttendParams& p, hipStream_t s);
hipError_t launch_attend_shared_bf16(int fmt, bool tiles, int nt, long long groups, const AttendParams& p, hipStream_t s);
hipError_t launch_attend_shared_f16(int fmt, bool tiles, int nt, long long groups, const AttendParams& p, hipStream_t s);
hipError_t launch_shared_join_f32(int sets, AttendParams p, hipStream_t s);
hipError_t launch_shared_join_bf16(int sets, AttendParams p, hipStream_t s);
hipError_t launch_shared_join_f16(int sets, AttendParams p, hipStream_t s);

// (chunks: 64 elements of a head each)
hipError_t launch_append(int type, int fmt, int chunks, const AppendParams& p, hipStream_t s);
hipError_t launch_read(int type, int fmt, int chunks, const ReadParams& p, hipStream_t s);
hipError_t launch_rotary(int type, const RotaryParams& p, hipStream_t s);
hipError_t launch_rotary_table(const double* turns, float* angles, int pairs, int first, int positions, double amplitude,
                               hipStream_t s);
hipError_t launch_verify(int type, const VerifyParams& p, hipStream_t s);

}  // namespace biq
