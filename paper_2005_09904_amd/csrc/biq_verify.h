// Verification of drafted tokens (biq_verify_drafts).
//
// The drawn token needs the sum of a row's weights before it needs their order, so a row of probabilities is read once, a
// wave per span of 1024 tokens, for the spans' sums, and the span where the goal lies once more.  Weights are integers (40 bits below the point), so that
// every order of additions gives the same sums and the same token.  64 rows of 120011 (two of them each, 61 MB): 12 us for the
// sums, 5.1 TB/s, and 6 for the tokens, whose loads depend on each other.
#pragma once

#include "biq_serve.h"

namespace biq {

constexpr int kVerifySpan = 1024;                    // tokens whose weights are summed into one number
constexpr int kVerifyThreads = 1024;                 // of the kernel that draws: 4 spans each, as 2^22 tokens have 4096

struct VerifyParams {
    const void* p;
    const void* q;
    long long p_seq_stride, p_stride, q_seq_stride, q_stride;
    const int* draft_tokens;
    const int* draft_lens;
    const float* uniform;
    int* tokens;
    int* accepted;
    unsigned long long* sums;    // [seqs][spans]
    int* verdicts;               // [seqs][4] accepted drafts, the refused one's token, whether none was refused
    int seqs, drafts, vocab, spans;
    unsigned first;              // first workgroup of this launch (verify_sums_kernel)
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
__device__ __forceinline__ Verdict examine(const VerifyParams& p, int seq, int lane) {
    typedef typename Elem<TYPE>::T T;
    // (tokens and random numbers of drafts that the sequence does not have are requested as well: none waits for its number of them)
    const int mine = lane < p.drafts ? lane : 0;
    int token = -1;
    float u = 0.f;
    if (p.drafts > 0) {
        token = p.draft_tokens[static_cast<long long>(seq) * p.drafts + mine];
        u = p.uniform[static_cast<long long>(seq) * (p.drafts + 1) + mine];
    }
    int drafts = p.draft_lens ? p.draft_lens[seq] : p.drafts;
    drafts = drafts < 0 ? 0 : drafts > p.drafts ? p.drafts : drafts;
    const bool known = lane < drafts && token >= 0 && token < p.vocab;
    bool ok = false;
    if (known) {
        Elems<TYPE, 1> pt, qt;
        float px[1], qx[1] = {1.f};
        pt.request(static_cast<const T*>(p.p) + seq * p.p_seq_stride + lane * p.p_stride + token);
        if (p.q) {
            qt.request(static_cast<const T*>(p.q) + seq * p.q_seq_stride + lane * p.q_stride + token);
            qt.get(qx, true);
        }
        pt.get(px, true);
        ok = (u < 0.f ? 0.f : u) * qx[0] < px[0];              // (NaN stays, and accepts nothing)
    }
    token = lane < drafts ? token : -1;
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

// N times 4 adjacent tokens of a row, t + 256 i .., requested together.  whole(i): all 4 of them are there, else they are requested
// one by one, the last one for those that are not.
template <int TYPE, int N>
struct RowTokens {
    Elems<TYPE, 4> p[N], q[N];
    template <typename Whole>
    __device__ __forceinline__ void request_row(Elems<TYPE, 4> (&to)[N], const void* base, long long at, int t, int vocab, const Whole& whole) {
        const auto* row = static_cast<const typename Elem<TYPE>::T*>(base) + at;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (whole(i)) {
                to[i].request(row + (t + 256 * i));
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) to[i].v[e] = row[t + 256 * i + e < vocab ? t + 256 * i + e : vocab - 1];
            }
        }
    }
    template <typename Whole>
    __device__ __forceinline__ void request(const VerifyParams& params, const Source& s, int t, const Whole& whole) {
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) q[i].v[e] = typename Elem<TYPE>::T(0.f);
        request_row(p, params.p, s.p_at, t, params.vocab, whole);
        if (s.minus) request_row(q, params.q, s.q_at, t, params.vocab, whole);
    }
    // Weights of the tokens t + 256 i ..  (0 beyond the vocabulary)
    __device__ __forceinline__ void weights(const Source& s, int vocab, int i, int t, unsigned long long (&w)[4]) const {
        float r[4], less[4];
        p[i].get(r, true);
        q[i].get(less, true);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            r[e] -= less[e];
            if (t + 256 * i + e == s.gone) r[e] -= 1.f;
            w[e] = t + 256 * i + e < vocab ? weight40(r[e]) : 0;
        }
    }
};

__device__ __forceinline__ unsigned long long sum_over_wave(unsigned long long x) {
#pragma unroll
    for (int d = 32; d > 0; d /= 2) x += __shfl_xor(x, d);
    return x;
}

__device__ __forceinline__ unsigned long long running_sum(unsigned long long x, int lane) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const unsigned long long y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    return x;
}

// Sums of spans of weights, one per wave (workgroups of 4).  Every wave examines the drafts itself: it needs to know the row.
template <int TYPE>
__device__ __forceinline__ unsigned long long span_sum(const VerifyParams& p, const Source& s, int span, int lane) {
    RowTokens<TYPE, kVerifySpan / 256> row;
    const int t0 = span * kVerifySpan, t = t0 + 4 * lane;
    row.request(p, s, t, [&](int i) { return t0 + 256 * i + 256 <= p.vocab; });
    unsigned long long total = 0, w[4];
#pragma unroll
    for (int i = 0; i < kVerifySpan / 256; ++i) {
        row.weights(s, p.vocab, i, t, w);
        total += (w[0] + w[1]) + (w[2] + w[3]);
    }
    return sum_over_wave(total);
}

template <int TYPE>
__global__ __launch_bounds__(256) void verify_sums_kernel(const VerifyParams p) {
    const int lane = threadIdx.x & 63, groups = (p.spans + 3) / 4;
    const int group = p.first + blockIdx.x, seq = group / groups, span = (group - seq * groups) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (span >= p.spans) return;
    const Verdict v = examine<TYPE>(p, seq, lane);
    const Source s = source_of(p, seq, v);
    if (span == 0 && lane == 0) {
        p.verdicts[4 * seq] = v.accepted;
        p.verdicts[4 * seq + 1] = v.token;
        p.verdicts[4 * seq + 2] = v.all;
    }
    const unsigned long long total = span_sum<TYPE>(p, s, span, lane);
    if (lane == 0) p.sums[static_cast<long long>(seq) * p.spans + span] = total;
}

// Running sum over the workgroup up to and with this thread's x; all: over everything.
__device__ __forceinline__ unsigned long long running_over_group(unsigned long long x, unsigned long long* lds, unsigned long long& all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const unsigned long long mine = running_sum(x, lane);
    __syncthreads();                                            // (the sums before are read)
    if (lane == 63) lds[wave] = mine;
    __syncthreads();
    unsigned long long before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < kVerifyThreads / 64; ++w) {
        if (w < wave) before += lds[w];
        all += lds[w];
    }
    return before + mine;
}

// The token: the workgroup of a sequence finds the span where the running sum of the spans' sums passes the goal, then the token
// in it.
template <int TYPE>
__device__ __forceinline__ void draw_token(const VerifyParams& p, int seq, const Verdict& v, Source s, const unsigned long long* sums) {
    __shared__ unsigned long long lds[kVerifyThreads / 64];
    __shared__ unsigned long long rest;                         // the goal less the sums before the span
    __shared__ int found;
    const int me = threadIdx.x;
    const int draft = me < v.accepted ? p.draft_tokens[static_cast<long long>(seq) * p.drafts + me] : -1;
    unsigned long long x[4], total;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = 4 * me + i < p.spans ? sums[4 * me + i] : 0;
    const float u = p.uniform[static_cast<long long>(seq) * (p.drafts + 1) + p.drafts];
    unsigned long long upto = running_over_group((x[0] + x[1]) + (x[2] + x[3]), lds, total);
    if (total == 0 && !v.all) {                                 // nothing left of p - q: p alone
        s.minus = false;
        s.gone = -1;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = 0;
            if (4 * me + i >= p.spans) continue;
            for (int t = 0; t < kVerifySpan; t += 4) {
                unsigned long long w[4];
                RowTokens<TYPE, 1> row;
                const int at = (4 * me + i) * kVerifySpan + t;
                row.request(p, s, at, [&](int) { return at + 4 <= p.vocab; });
                row.weights(s, p.vocab, 0, at, w);
                x[i] += (w[0] + w[1]) + (w[2] + w[3]);
            }
        }
        upto = running_over_group((x[0] + x[1]) + (x[2] + x[3]), lds, total);
    }
    const float scaled = u > 0.f ? u * 0x1p31f : 0.f;
    const unsigned long long u31 = scaled < 0x1p31f ? static_cast<unsigned long long>(scaled) : 0x7fffffffull;
    // floor(u31 total / 2^31), total < 2^63
    const unsigned long long goal = u31 * (total >> 32) * 2 + (u31 * (total & 0xffffffffull) >> 31);
    if (me == 0) found = -1;
    __syncthreads();
    unsigned long long run = upto - ((x[0] + x[1]) + (x[2] + x[3]));
    if (run <= goal && upto > goal) {                           // one thread, as the sums rise; none where all is 0
        int i = 0;
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (run + x[e] <= goal && i == e) {
                run += x[e];
                ++i;
            }
        found = 4 * me + i;
        rest = goal - run;
    }
    __syncthreads();
    const int span = found;
    if (span >= 0) {
        const unsigned long long left = rest;
        unsigned long long w[4] = {0, 0, 0, 0}, all;
        const int t = span * kVerifySpan + 4 * me;
        if (me < kVerifySpan / 4) {
            RowTokens<TYPE, 1> row;
            row.request(p, s, t, [&](int) { return t + 4 <= p.vocab; });
            row.weights(s, p.vocab, 0, t, w);
        }
        const unsigned long long mine = (w[0] + w[1]) + (w[2] + w[3]);
        unsigned long long at = running_over_group(mine, lds, all) - mine;
        if (at <= left && at + mine > left) {
            int i = 0;
#pragma unroll
            for (int e = 0; e < 3; ++e) {
                at += w[e];
                i += at <= left;                                // (sums rise: the tokens before the first above the goal)
            }
            found = t + i;
        }
        __syncthreads();
    }
    if (me <= p.drafts) {
        const int token = me == v.accepted ? found : draft;
        p.tokens[static_cast<long long>(seq) * (p.drafts + 1) + me] = token;
        if (me == 0) p.accepted[seq] = v.accepted;
    }
}

template <int TYPE>
__global__ __launch_bounds__(kVerifyThreads) void verify_draw_kernel(const VerifyParams p) {
    const int seq = blockIdx.x;
    const Verdict v = {p.verdicts[4 * seq], p.verdicts[4 * seq + 1], p.verdicts[4 * seq + 2] != 0};
    draw_token<TYPE>(p, seq, v, source_of(p, seq, v), p.sums + static_cast<long long>(seq) * p.spans);
}

// Both in one launch, for a span per wave at most: the spans' sums stay in LDS.  (One sequence, 5000 tokens: 6.8 us instead of 8.3;
// 16000: 7.5 and 8.8; 32000, two spans a wave: 10.6 and 9.0.)
constexpr int kVerifyOneSpans = kVerifyThreads / 64;
template <int TYPE>
__global__ __launch_bounds__(kVerifyThreads) void verify_one_kernel(const VerifyParams p) {
    __shared__ unsigned long long sums[kVerifyOneSpans];
    const int seq = blockIdx.x, lane = threadIdx.x & 63;
    const Verdict v = examine<TYPE>(p, seq, lane);
    const Source s = source_of(p, seq, v);
    const int span = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (span < p.spans) {
        const unsigned long long total = span_sum<TYPE>(p, s, span, lane);
        if (lane == 0) sums[span] = total;
    }
    __syncthreads();
    draw_token<TYPE>(p, seq, v, s, sums);
}

}  // namespace biq
