// Penalties, biases, temperature and masks on logits, and the softmax over the vocabulary (biq_logits).
//
// A workgroup takes a span of the vocabulary for all rows of a sequence.  What the sequence's tokens change in the span is counted
// in LDS first (integers, so that no order of additions matters), the drafts before a row are added row by row.  The softmax needs
// the whole row: a first launch leaves every span's largest logit and its sum of exponentials, the second computes the logits again and
// writes; nothing that is rounded is stored between them.
#pragma once

#include "biq_norm.h"

namespace biq {

struct LogitsParams {
    const void* x;
    void* out;
    long long x_seq_stride, x_stride, out_seq_stride, out_stride, mask_seq_stride, mask_stride;
    const int* history;      // [seqs][width] or NULL
    const int* lens;
    const int* prompt_lens;  // or NULL: 0
    const int* drafts;       // [seqs][rows - 1] or NULL
    const float* repetition; // [seqs] or NULL, as the others
    const float* presence;
    const float* frequency;
    const float* temperature;
    const int* bias_tokens;  // [seqs][biases]
    const float* bias_values;
    const uint32_t* mask;
    f32x2* stats;            // [seqs][rows][spans] largest logit, sum of exponentials (or the place of the largest as an integer)
    int out_type, seqs, rows, vocab, width, biases, spans;
    unsigned first;
};

constexpr uint32_t kInPrompt = 0x80000000u;          // beside the count of a token: it is among the prompt's

// The largest logit and its lowest place; a NaN is larger than all.
struct Best { float z; int at; };
__device__ __forceinline__ Best better(Best a, Best b) {
    if (a.z != a.z || b.z != b.z) return a.z != a.z ? a : b;
    return b.z > a.z || (b.z == a.z && b.at < a.at) ? b : a;
}
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.4426950408889634f); }

// Over a workgroup of THREADS; all threads get the result.
template <int THREADS>
__device__ __forceinline__ Best best_over_group(Best b, Best* lds) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) b = better(b, Best{__shfl_xor(b.z, d), __shfl_xor(b.at, d)});
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = b;
    __syncthreads();
    b = lds[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) b = better(b, lds[w]);
    return b;
}

// What happens to a sequence's logits, but for what LDS holds.
struct Penalties {
    float repetition, presence, frequency, heat;                // heat: 1 / temperature
    bool greedy;
};
__device__ __forceinline__ Penalties penalties_of(const LogitsParams& p, int seq) {
    Penalties k;
    k.repetition = p.repetition ? p.repetition[seq] : 1.f;
    k.presence = p.presence ? p.presence[seq] : 0.f;
    k.frequency = p.frequency ? p.frequency[seq] : 0.f;
    const float t = p.temperature ? p.temperature[seq] : 1.f;
    k.greedy = !(t > 0.f);
    k.heat = k.greedy ? 1.f : 1.f / t;
    return k;
}

// Counts and biases of a span of SPAN tokens in LDS.
template <int THREADS, int SPAN>
__device__ __forceinline__ void count_tokens(const LogitsParams& p, int seq, int t0, uint32_t* counts, float* biases) {
    for (int i = threadIdx.x; i < SPAN; i += THREADS) {
        if (counts) counts[i] = 0;
        if (biases) biases[i] = 0.f;
    }
    __syncthreads();
    if (p.history) {
        int len = p.lens[seq], prompt = p.prompt_lens ? p.prompt_lens[seq] : 0;
        len = len < 0 ? 0 : len > p.width ? p.width : len;
        const int* tokens = p.history + static_cast<long long>(seq) * p.width;
        for (int i = threadIdx.x; i < len; i += THREADS) {
            const uint32_t at = static_cast<uint32_t>(tokens[i]) - static_cast<uint32_t>(t0);
            if (at >= static_cast<uint32_t>(SPAN)) continue;
            if (i < prompt) atomicOr(counts + at, kInPrompt);
            else atomicAdd(counts + at, 1u);
        }
    }
    if (biases) {
        // a token's biases are added in the list's order by the thread of the first of them
        const int* tokens = p.bias_tokens + static_cast<long long>(seq) * p.biases;
        const float* values = p.bias_values + static_cast<long long>(seq) * p.biases;
        for (int i = threadIdx.x; i < p.biases; i += THREADS) {
            const int token = tokens[i];
            const uint32_t at = static_cast<uint32_t>(token) - static_cast<uint32_t>(t0);
            if (at >= static_cast<uint32_t>(SPAN)) continue;
            bool first = true;
            for (int j = 0; j < i; ++j) first = first && tokens[j] != token;
            if (!first) continue;
            float sum = 0.f;
            for (int j = i; j < p.biases; ++j)
                if (tokens[j] == token) sum += values[j];
            biases[at] = sum;
        }
    }
    __syncthreads();
}

// WHAT: 0 writes logits, 1 leaves the stats of spans, 2 writes probabilities by them, 3 writes probabilities of a row that is one span.
template <int TYPE, int THREADS, int U, int WHAT>
__global__ __launch_bounds__(THREADS) void logits_kernel(const LogitsParams p) {
#pragma clang fp contract(off)
    typedef typename Elem<TYPE>::T T;
    constexpr int SPAN = THREADS * U * 8;
    extern __shared__ float lds[];
    __shared__ Best exchange[THREADS / 64];
    __shared__ float sums[THREADS / 64];
    const long long group = p.first + blockIdx.x;
    const int seq = static_cast<int>(group / p.spans), span = static_cast<int>(group - static_cast<long long>(seq) * p.spans), t0 = span * SPAN;
    const bool counting = p.history || p.drafts;
    uint32_t* counts = counting ? reinterpret_cast<uint32_t*>(lds) : nullptr;
    float* biases = p.biases > 0 ? lds + (counting ? SPAN : 0) : nullptr;
    const Penalties k = penalties_of(p, seq);
    if (counting || biases) count_tokens<THREADS, SPAN>(p, seq, t0, counts, biases);

    for (int row = 0; row < p.rows; ++row) {
        if (row > 0 && p.drafts) {
            __syncthreads();                                    // (the row before is counted)
            const uint32_t at = static_cast<uint32_t>(p.drafts[static_cast<long long>(seq) * (p.rows - 1) + row - 1]) - static_cast<uint32_t>(t0);
            if (threadIdx.x == 0 && at < static_cast<uint32_t>(SPAN)) counts[at] += 1;
            __syncthreads();
        }
        const T* x = static_cast<const T*>(p.x) + seq * p.x_seq_stride + row * p.x_stride;
        const uint32_t* mask = p.mask ? p.mask + seq * p.mask_seq_stride + row * p.mask_stride : nullptr;
        T raw[U][8];
        uint32_t allowed[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int at = (u * THREADS + static_cast<int>(threadIdx.x)) * 8, e = t0 + at;
            request8(raw[u], x, e < p.vocab ? e : p.vocab - 1, p.vocab);
            allowed[u] = 0xffu;
            if (mask) allowed[u] = mask[(e < p.vocab ? e : p.vocab - 1) >> 5] >> (e & 31);
        }
        float z[U][8];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int at = (u * THREADS + static_cast<int>(threadIdx.x)) * 8, e = t0 + at;
#pragma unroll
            for (int i = 0; i < 8; ++i) z[u][i] = static_cast<float>(raw[u][i]);
            if (counting) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t c = counts[at + i];
                    if (c == 0) continue;
                    z[u][i] = z[u][i] > 0.f ? z[u][i] / k.repetition : z[u][i] * k.repetition;
                    const uint32_t said = c & ~kInPrompt;
                    if (said) z[u][i] = z[u][i] - static_cast<float>(said) * k.frequency - k.presence;
                }
            }
            if (biases) {
#pragma unroll
                for (int i = 0; i < 8; ++i) z[u][i] += biases[at + i];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                z[u][i] *= k.heat;
                if (!((allowed[u] >> i) & 1u) || e + i >= p.vocab) z[u][i] = -INFINITY;
            }
        }
        float shift = 0.f, by = 1.f;
        Best best = {-INFINITY, 0x7fffffff};
        const long long r = static_cast<long long>(seq) * p.rows + row;
        if constexpr (WHAT == 1 || WHAT == 3) {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < 8; ++i) best = better(best, Best{z[u][i], t0 + (u * THREADS + static_cast<int>(threadIdx.x)) * 8 + i});
            best = best_over_group<THREADS>(best, exchange);
            float sum = 0.f;
            if (!k.greedy) {
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum += z[u][i] == -INFINITY ? 0.f : exp_of(z[u][i] - best.z);
                sum = over_row<THREADS>(sum, sums, Add());
            }
            if (WHAT == 1 && threadIdx.x == 0) p.stats[r * p.spans + span] = (f32x2){best.z, k.greedy ? __int_as_float(best.at) : sum};
            shift = best.z;
            by = sum;
        }
        if constexpr (WHAT == 1) continue;
        if constexpr (WHAT == 2) {
            // (every thread for itself where there are few spans would read them all: lanes share them)
            const f32x2* stats = p.stats + r * p.spans;
            const int lane = threadIdx.x & 63;
            for (int i = lane; i < p.spans; i += 64) best = better(best, Best{stats[i][0], k.greedy ? __float_as_int(stats[i][1]) : 0});
#pragma unroll
            for (int d = 1; d < 64; d *= 2) best = better(best, Best{__shfl_xor(best.z, d), __shfl_xor(best.at, d)});
            float sum = 0.f;
            if (!k.greedy) {
                for (int i = lane; i < p.spans; i += 64) sum += stats[i][0] == -INFINITY ? 0.f : stats[i][1] * exp_of(stats[i][0] - best.z);
#pragma unroll
                for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
            }
            shift = best.z;
            by = sum;
        }
        const bool bad = shift != shift;
        const float each = by == 0.f ? 0.f : 1.f / by;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int e = t0 + (u * THREADS + static_cast<int>(threadIdx.x)) * 8;
            if constexpr (WHAT != 0) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (k.greedy) z[u][i] = bad ? shift : e + i == best.at && shift != -INFINITY ? 1.f : 0.f;
                    else z[u][i] = bad ? shift : z[u][i] == -INFINITY ? 0.f * each : exp_of(z[u][i] - shift) * each;
                }
            }
            if (e < p.vocab) store8_type(p.out_type, p.out, seq * p.out_seq_stride + row * p.out_stride, e, p.vocab, z[u]);
        }
    }
}

}  // namespace biq
