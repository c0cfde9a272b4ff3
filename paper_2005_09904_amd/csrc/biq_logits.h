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
    f32x2* stats;            // [seqs][rows][spans * waves] largest logit, sum of exponentials (or the place of the largest as an integer)
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
    k.greedy = !(t > 0x1p-100f);
    k.heat = k.greedy ? 1.f : 1.f / fminf(t, 0x1p100f);         // (finite, and not 0: infinities stay what they are)
    return k;
}

// Counts and biases of a span of SPAN tokens in LDS.
template <int THREADS, int SPAN>
__device__ __forceinline__ void count_tokens(const LogitsParams& p, int seq, int t0, uint32_t* counts, float* biases) {
    constexpr int AHEAD = 4;                                    // times 4 tokens that a thread requests together
    typedef int Loose4 __attribute__((ext_vector_type(4), aligned(4)));
    int len = p.history ? p.lens[seq] : 0, prompt = p.prompt_lens ? p.prompt_lens[seq] : 0;
    len = len < 0 ? 0 : len > p.width ? p.width : len;
    const int* tokens = p.history + static_cast<long long>(seq) * p.width;
    int held[AHEAD][4];
    auto request = [&](int first) {
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            const int i = first + (a * THREADS + static_cast<int>(threadIdx.x)) * 4;
            if (i + 4 <= len) {
                const Loose4 v = *reinterpret_cast<const Loose4*>(tokens + i);
#pragma unroll
                for (int e = 0; e < 4; ++e) held[a][e] = v[e];
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) held[a][e] = i + e < len ? tokens[i + e] : -1;
            }
        }
    };
    request(0);
    for (int i = threadIdx.x; i < SPAN / 4; i += THREADS) {
        if (counts) reinterpret_cast<u32x4*>(counts)[i] = (u32x4){0, 0, 0, 0};
        if (biases) reinterpret_cast<f32x4*>(biases)[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    __syncthreads();
    for (int first = 0; first < len; first += AHEAD * THREADS * 4) {
        if (first > 0) request(first);
#pragma unroll
        for (int a = 0; a < AHEAD; ++a)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t at = static_cast<uint32_t>(held[a][e]) - static_cast<uint32_t>(t0);
                if (at >= static_cast<uint32_t>(SPAN) || held[a][e] < 0) continue;
                if (first + (a * THREADS + static_cast<int>(threadIdx.x)) * 4 + e < prompt) atomicOr(counts + at, kInPrompt);
                else atomicAdd(counts + at, 1u);
            }
    }
    if (biases) {
        // a token's biases are added in the list's order by the thread of the first of them
        const int* listed = p.bias_tokens + static_cast<long long>(seq) * p.biases;
        const float* values = p.bias_values + static_cast<long long>(seq) * p.biases;
        for (int i = threadIdx.x; i < p.biases; i += THREADS) {
            const int token = listed[i];
            const uint32_t at = static_cast<uint32_t>(token) - static_cast<uint32_t>(t0);
            if (at >= static_cast<uint32_t>(SPAN)) continue;
            bool first = true;
            for (int j = 0; j < i; ++j) first = first && listed[j] != token;
            if (!first) continue;
            float sum = 0.f;
            for (int j = i; j < p.biases; ++j)
                if (listed[j] == token) sum += values[j];
            biases[at] = sum;
        }
    }
    __syncthreads();
}

__device__ __forceinline__ float largest_of_wave(float x) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) x = fmaxf(x, __shfl_xor(x, d));
    return x;
}
__device__ __forceinline__ float sum_of_wave(float x) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) x += __shfl_xor(x, d);
    return x;
}
__device__ __forceinline__ Best best_of_wave(Best b) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) b = better(b, Best{__shfl_xor(b.z, d), __shfl_xor(b.at, d)});
    return b;
}

// What a row comes to: probabilities are exp2((z - top) scale) each, or for greedy sequences 1 at place `at`.  Numbers
// that are no numbers come through `each`: a NaN among the exponentials is one in their sum.
struct RowSum {
    float top, each;
    int at;
};
// Of n pairs (largest logit, sum of exponentials or place), all threads of a wave for all of them.
template <typename Pairs>
__device__ __forceinline__ RowSum row_sum(const Pairs& pairs, int n, bool greedy, float scale) {
    const int lane = threadIdx.x & 63;
    RowSum r = {-INFINITY, 0.f, -1};
    if (greedy) {
        Best best = {-INFINITY, 0x7fffffff};
        for (int i = lane; i < n; i += 64) best = better(best, Best{pairs[i][0], __float_as_int(pairs[i][1])});
        best = best_of_wave(best);
        r.top = best.z;
        r.at = best.z == -INFINITY ? -1 : best.at;
        return r;
    }
    for (int i = lane; i < n; i += 64) r.top = fmaxf(r.top, pairs[i][0]);
    r.top = largest_of_wave(r.top);
    float sum = 0.f;
    for (int i = lane; i < n; i += 64) sum += pairs[i][0] == -INFINITY ? pairs[i][1] : pairs[i][1] * __builtin_amdgcn_exp2f((pairs[i][0] - r.top) * scale);
    sum = sum_of_wave(sum);
    r.each = sum == 0.f ? 0.f : 1.f / sum;
    return r;
}

// WHAT: 0 writes logits, 1 leaves a pair of every wave, 2 writes probabilities by these, 3 writes probabilities of rows that a workgroup
// has whole.  A thread has U times 8 adjacent tokens, and their counts and biases are read by no other: a draft is counted by the thread
// that has it.
template <int TYPE, int THREADS, int U, int WHAT>
__global__ __launch_bounds__(THREADS) void logits_kernel(const LogitsParams p) {
#pragma clang fp contract(off)
    typedef typename Elem<TYPE>::T T;
    constexpr int SPAN = THREADS * U * 8, WAVES = THREADS / 64;
    constexpr bool EARLY = U <= 2;                              // the next row is requested before this one is used (32 tokens: no registers left)
    extern __shared__ float lds[];                              // pairs [2][WAVES], then counts and biases
    f32x2* pairs = reinterpret_cast<f32x2*>(lds);
    float* space = lds + 4 * WAVES;
    const long long group = p.first + blockIdx.x;
    const int seq = static_cast<int>(group / p.spans), span = static_cast<int>(group - static_cast<long long>(seq) * p.spans), t0 = span * SPAN;
    int me = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(me >> 6);
    const bool counting = p.history || p.drafts;
    uint32_t* counts = counting ? reinterpret_cast<uint32_t*>(space) : nullptr;
    float* biases = p.biases > 0 ? space + (counting ? SPAN : 0) : nullptr;
    T raw[U][8];
    uint32_t allowed[U];
    auto request = [&](int row) {
        const T* x = static_cast<const T*>(p.x) + seq * p.x_seq_stride + row * p.x_stride;
        const uint32_t* mask = p.mask + seq * p.mask_seq_stride + row * p.mask_stride;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int e = t0 + (u * THREADS + me) * 8, there = e < p.vocab ? e : p.vocab - 1;
            request8(raw[u], x, there, p.vocab);
            allowed[u] = p.mask ? mask[there >> 5] : ~0u;
        }
    };
    request(0);
    const Penalties k = penalties_of(p, seq);
    if (counting || biases) count_tokens<THREADS, SPAN>(p, seq, t0, counts, biases);
    const float scale = k.heat * 1.4426950408889634f;

    for (int row = 0; row < p.rows; ++row) {
        // (the tokens' places are worked out anew for each row: kept over the loop, they take the registers that the logits need)
        if (!EARLY) asm volatile("" : "+v"(me));
        if (!EARLY && row > 0) request(row);
        if (row > 0 && p.drafts) {
            const uint32_t at = static_cast<uint32_t>(p.drafts[static_cast<long long>(seq) * (p.rows - 1) + row - 1]) - static_cast<uint32_t>(t0);
            if (at < static_cast<uint32_t>(SPAN) && static_cast<int>((at >> 3) % THREADS) == me) counts[at] += 1;
        }
        float z[U][8];
        uint32_t keep[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int e = t0 + (u * THREADS + me) * 8;
#pragma unroll
            for (int i = 0; i < 8; ++i) z[u][i] = static_cast<float>(raw[u][i]);
            keep[u] = allowed[u] >> (e & 31);
            if (e + 8 > p.vocab) keep[u] &= e < p.vocab ? (1u << (p.vocab - e)) - 1u : 0u;
        }
        if (EARLY && row + 1 < p.rows) request(row + 1);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int at = (u * THREADS + me) * 8;
            if (counting) {
                const u32x4 c0 = *reinterpret_cast<const u32x4*>(counts + at), c1 = *reinterpret_cast<const u32x4*>(counts + at + 4);
                const u32x4 any = c0 | c1;
                if ((any[0] | any[1]) | (any[2] | any[3])) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const uint32_t c = i < 4 ? c0[i & 3] : c1[i & 3], said = c & ~kInPrompt;
                        const float y = z[u][i] > 0.f ? z[u][i] / k.repetition : z[u][i] * k.repetition;
                        const float less = y - static_cast<float>(said) * k.frequency - k.presence;
                        z[u][i] = c == 0 ? z[u][i] : said ? less : y;
                    }
                }
            }
            if (biases) {
                const f32x4 b0 = *reinterpret_cast<const f32x4*>(biases + at), b1 = *reinterpret_cast<const f32x4*>(biases + at + 4);
#pragma unroll
                for (int i = 0; i < 8; ++i) z[u][i] += i < 4 ? b0[i & 3] : b1[i & 3];
            }
            if (WHAT == 0) {
#pragma unroll
                for (int i = 0; i < 8; ++i) z[u][i] *= k.heat;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (!((keep[u] >> i) & 1u)) z[u][i] = -INFINITY;
            if (!EARLY) __builtin_amdgcn_sched_barrier(0);      // (one part's counts and biases at a time)
        }
        const long long r = static_cast<long long>(seq) * p.rows + row;
        RowSum sum = {0.f, 0.f, -1};
        if constexpr (WHAT == 1 || WHAT == 3) {
            f32x2 mine;
            if (k.greedy) {
                Best best = {-INFINITY, U * 8};
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int i = 0; i < 8; ++i) best = better(best, Best{z[u][i], u * 8 + i});     // (this thread's places: constants)
                best.at = t0 + ((best.at >> 3) * THREADS + me) * 8 + (best.at & 7);
                best = best_of_wave(best);
                mine = (f32x2){best.z, __int_as_float(best.at)};
            } else {
                float top = -INFINITY, all = 0.f;
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int i = 0; i < 8; ++i) top = fmaxf(top, z[u][i]);
                top = largest_of_wave(top);
                // (all of them -infinity: each counts nothing, but for a NaN)
                const float from = top == -INFINITY ? 0.f : top;
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int i = 0; i < 8; ++i) all += __builtin_amdgcn_exp2f((z[u][i] - from) * scale);
                mine = (f32x2){top, sum_of_wave(all)};
            }
            if (WHAT == 1) {
                if ((me & 63) == 0) p.stats[(r * p.spans + span) * WAVES + wave] = mine;
                continue;
            }
            f32x2* mine_at = pairs + (row & 1) * WAVES;         // (the other ones may still be read)
            if ((me & 63) == 0) mine_at[wave] = mine;
            __syncthreads();
            sum = row_sum(mine_at, WAVES, k.greedy, scale);
        }
        if constexpr (WHAT == 2) sum = row_sum(p.stats + r * p.spans * WAVES, p.spans * WAVES, k.greedy, scale);
        const float from = sum.top == -INFINITY ? 0.f : sum.top;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int e = t0 + (u * THREADS + me) * 8;
            if constexpr (WHAT != 0) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (k.greedy) z[u][i] = sum.top != sum.top ? sum.top : sum.at - e == i ? 1.f : 0.f;
                    else z[u][i] = __builtin_amdgcn_exp2f((z[u][i] - from) * scale) * sum.each;
                }
            }
            if (e < p.vocab) store8_type(p.out_type, p.out, seq * p.out_seq_stride + row * p.out_stride, e, p.vocab, z[u]);
        }
    }
}

}  // namespace biq
