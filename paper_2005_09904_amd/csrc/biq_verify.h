// Verification of drafted tokens (biq_verify_drafts).
//
// The drawn token needs the sum of a row's weights before it needs their order, so a row of probabilities is read once in
// parts for their sums, and the part where the goal lies once more.  Weights are integers (40 bits below the point), so that
// every order of additions gives the same sums and the same token.
#pragma once

#include "biq_serve.h"

namespace biq {

constexpr int kVerifyThreads = 1024;
constexpr int kVerifyPart = 4 * kVerifyThreads;      // tokens whose weights are summed into one number

struct VerifyParams {
    const void* p;
    const void* q;
    long long p_seq_stride, p_stride, q_seq_stride, q_stride;
    const int* draft_tokens;
    const int* draft_lens;
    const float* uniform;
    int* tokens;
    int* accepted;
    unsigned long long* sums;    // [seqs][parts]
    int seqs, drafts, vocab, parts;
    int p_quads, q_quads;
};

// floor(2^40 min(1, max(0, r))), 0 for NaN: 20 bits, then 20 more of what is left (both exact).
__device__ __forceinline__ unsigned long long weight40(float r) {
    r = r > 0.f ? r : 0.f;
    r = r < 1.f ? r : 1.f;
    const float a = r * 0x1p20f;
    const uint32_t hi = static_cast<uint32_t>(a);
    const uint32_t lo = static_cast<uint32_t>((a - static_cast<float>(hi)) * 0x1p20f);
    return (static_cast<unsigned long long>(hi) << 20) + lo;
}

// What a sequence's drafts come to.
struct Verdict { int accepted, token; bool all; };

// Lanes of one wave: draft i is lane i's.
template <int TYPE>
__device__ __forceinline__ Verdict judge(const VerifyParams& p, int seq, int lane) {
    int drafts = p.draft_lens ? p.draft_lens[seq] : p.drafts;
    drafts = drafts < 0 ? 0 : drafts > p.drafts ? p.drafts : drafts;
    bool ok = false;
    int token = -1;
    if (lane < drafts) {
        token = p.draft_tokens[static_cast<long long>(seq) * p.drafts + lane];
        if (token >= 0 && token < p.vocab) {
            const float pt = load_elem<TYPE>(p.p, seq * p.p_seq_stride + lane * p.p_stride + token);
            const float qt = p.q ? load_elem<TYPE>(p.q, seq * p.q_seq_stride + lane * p.q_stride + token) : 1.f;
            const float u = p.uniform[static_cast<long long>(seq) * (p.drafts + 1) + lane];
            ok = u * qt < pt;
        }
    }
    const unsigned long long refused = ~__ballot(ok);            // (lane `drafts` refuses)
    const int n = __ffsll(refused) - 1;
    Verdict v;
    v.accepted = n;
    v.all = n == drafts;
    v.token = __shfl(token, n < 63 ? n : 63);
    return v;
}

// The row that is drawn from.
struct Source {
    long long p_at, q_at;
    int gone;                // token that a certain draft takes away, -1: none
    bool minus;              // q is subtracted
};
__device__ __forceinline__ Source source_of(const VerifyParams& p, int seq, const Verdict& v) {
    Source s;
    s.p_at = seq * p.p_seq_stride + v.accepted * p.p_stride;
    s.q_at = seq * p.q_seq_stride + v.accepted * p.q_stride;
    s.minus = !v.all && p.q;
    s.gone = !v.all && !p.q ? v.token : -1;
    return s;
}

// Weights of the tokens t .. t + 3 (0 beyond the vocabulary).
template <int TYPE>
__device__ __forceinline__ void weights4(const VerifyParams& p, const Source& s, int t, unsigned long long (&w)[4]) {
    float r[4] = {0.f, 0.f, 0.f, 0.f};
    const bool inside = t + 4 <= p.vocab;
    if (inside && p.p_quads) {
        const f32x4 x = load_elem4<TYPE>(p.p, s.p_at + t);
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = x[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (t + i < p.vocab) r[i] = load_elem<TYPE>(p.p, s.p_at + t + i);
    }
    if (s.minus) {
        if (inside && p.q_quads) {
            const f32x4 x = load_elem4<TYPE>(p.q, s.q_at + t);
#pragma unroll
            for (int i = 0; i < 4; ++i) r[i] -= x[i];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (t + i < p.vocab) r[i] -= load_elem<TYPE>(p.q, s.q_at + t + i);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (t + i == s.gone) r[i] -= 1.f;
        w[i] = weight40(r[i]);
    }
}

__device__ __forceinline__ unsigned long long sum_over_wave(unsigned long long x) {
#pragma unroll
    for (int d = 32; d > 0; d /= 2) x += __shfl_xor(x, d);
    return x;
}

// Sum over the workgroup, in every thread.
__device__ __forceinline__ unsigned long long sum_over_group(unsigned long long x, unsigned long long* lds) {
    x = sum_over_wave(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    unsigned long long total = 0;
#pragma unroll
    for (int w = 0; w < kVerifyThreads / 64; ++w) total += lds[w];
    return total;
}

// Sum of one part's weights: workgroup (sequence, part).
template <int TYPE>
__global__ __launch_bounds__(kVerifyThreads) void verify_sums_kernel(const VerifyParams p) {
    __shared__ unsigned long long lds[kVerifyThreads / 64];
    const int seq = blockIdx.x / p.parts, part = blockIdx.x % p.parts;
    const Verdict v = judge<TYPE>(p, seq, threadIdx.x & 63);
    const Source s = source_of(p, seq, v);
    unsigned long long w[4];
    weights4<TYPE>(p, s, part * kVerifyPart + 4 * static_cast<int>(threadIdx.x), w);
    const unsigned long long total = sum_over_group(w[0] + w[1] + w[2] + w[3], lds);
    if (threadIdx.x == 0) p.sums[static_cast<long long>(seq) * p.parts + part] = total;
}

// The token: a workgroup per sequence.
template <int TYPE>
__global__ __launch_bounds__(kVerifyThreads) void verify_draw_kernel(const VerifyParams p) {
    __shared__ unsigned long long lds[kVerifyThreads / 64];
    __shared__ int found;
    const int seq = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Verdict v = judge<TYPE>(p, seq, lane);
    Source s = source_of(p, seq, v);
    const unsigned long long* sums = p.sums + static_cast<long long>(seq) * p.parts;
    unsigned long long total = 0;
    for (int i = 0; i < p.parts; ++i) total += sums[i];
    bool own = true;                                            // the parts' sums are those of s
    if (total == 0 && !v.all) {                                 // nothing left of p - q: p alone
        s.minus = false;
        s.gone = -1;
        own = false;
        unsigned long long mine = 0, w[4];
        for (int t = 4 * threadIdx.x; t < p.vocab; t += kVerifyPart) {
            weights4<TYPE>(p, s, t, w);
            mine += w[0] + w[1] + w[2] + w[3];
        }
        total = sum_over_group(mine, lds);
    }
    const float u = p.uniform[static_cast<long long>(seq) * (p.drafts + 1) + p.drafts];
    float scaled = u > 0.f ? u * 0x1p31f : 0.f;
    const unsigned long long u31 = scaled < 0x1p31f ? static_cast<unsigned long long>(scaled) : 0x7fffffffull;
    // floor(u31 total / 2^31), total < 2^63
    unsigned long long goal = u31 * (total >> 32) * 2 + (u31 * (total & 0xffffffffull) >> 31);
    if (threadIdx.x == 0) found = -1;
    __syncthreads();
    if (total > 0) {
        int part = 0;
        if (own)
            for (; part < p.parts - 1 && sums[part] <= goal; ++part) goal -= sums[part];
        for (; part < p.parts; ++part) {
            unsigned long long w[4];
            const int t = part * kVerifyPart + 4 * static_cast<int>(threadIdx.x);
            weights4<TYPE>(p, s, t, w);
            const unsigned long long mine = w[0] + w[1] + w[2] + w[3];
            unsigned long long upto = mine;                     // running sum over the wave
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const unsigned long long y = __shfl_up(upto, d);
                if (lane >= d) upto += y;
            }
            __syncthreads();
            if (lane == 63) lds[wave] = upto;
            __syncthreads();
            unsigned long long before = 0, all = 0;
#pragma unroll
            for (int i = 0; i < kVerifyThreads / 64; ++i) {
                if (i < wave) before += lds[i];
                all += lds[i];
            }
            if (all > goal) {
                unsigned long long run = before + upto - mine;
                if (run <= goal && run + mine > goal) {
                    int i = 0;
#pragma unroll
                    for (int e = 0; e < 3; ++e) {
                        run += w[e];
                        i += run <= goal;                       // (sums rise: the tokens before the first above the goal)
                    }
                    found = t + i;
                }
                break;
            }
            goal -= all;
        }
        __syncthreads();
    }
    if (wave == 0 && lane <= p.drafts) {
        const int token = lane < v.accepted ? p.draft_tokens[static_cast<long long>(seq) * p.drafts + lane]
                                            : lane == v.accepted ? found : -1;
        p.tokens[static_cast<long long>(seq) * (p.drafts + 1) + lane] = token;
        if (lane == 0) p.accepted[seq] = v.accepted;
    }
}

}  // namespace biq
