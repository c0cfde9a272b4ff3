// Penalties, biases, temperature and masks on logits, and the softmax over the vocabulary (biq_logits).
//
//   z = (x > 0 ? x / repetition : x repetition  if said or in the prompt)  - presence [said] - frequency times said + bias,  z / temperature,  -inf where masked
//   p = exp(z - max) / sum exp(z - max), or all of it to the first of the largest where the temperature is 0
//
// A workgroup takes a span of the vocabulary, or the whole of a smaller one, for all rows of a sequence.  What the sequence's tokens change in the
// span is counted in LDS first (integers, so that no order of additions matters), the drafts before a row are added row by row.  The softmax
// needs the whole row: of spans, a first launch leaves the largest logit and the sum of exponentials, the second computes the logits again
// and writes; nothing that is rounded is stored between them.
//
// Many rows are bound by instructions, then by what is written: 32 sequences of 5 rows of 120011, bfloat16 to float (118 MB), 26.9 us
// for the sums (1.4 TB/s read; half of a SIMD's time goes to vector instructions, 1160 a wave) and 31.9 for the probabilities (3.7 TB/s
// read and written).  A few rows are two launches of dependent loads (lengths, tokens, counts, logits): one of 32000 5.0 and 5.3 us.
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

// Entry i0 + lane of a sequence's list of biases.
struct Bias { int token; float value; };
__device__ __forceinline__ Bias bias_of(const LogitsParams& p, int seq, int i0) {
    const int i = i0 + static_cast<int>(threadIdx.x & 63);
    const long long at = static_cast<long long>(seq) * p.biases + (i < p.biases ? i : p.biases - 1);
    return {p.bias_tokens[at], p.bias_values[at]};
}

// Counts and biases of a span of SPAN tokens in LDS.
template <int THREADS, int SPAN>
__device__ __forceinline__ void count_tokens(const LogitsParams& p, int seq, int t0, uint32_t* counts, float* biases) {
    constexpr int AHEAD = 4;                                    // times 4 tokens that a thread requests together
    constexpr int WAVES = THREADS / 64;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Bias mine = {-1, 0.f};
    if (biases) mine = bias_of(p, seq, 0);
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
        // 64 of the list at a time, a lane each; the waves share those that lie in the span.  A token's biases are added in the list's order
        // where the first of them is met, which looks at the rest of the list.
        for (int i0 = 0; i0 < p.biases; i0 += 64) {
            if (i0 > 0) mine = bias_of(p, seq, i0);
            unsigned long long here = __ballot(i0 + lane < p.biases && mine.token >= t0 && mine.token < t0 + SPAN);
            for (int n = 0; here; ++n) {
                const int l = __ffsll(here) - 1, token = __builtin_amdgcn_readlane(mine.token, l);
                here &= here - 1;
                if (n % WAVES != wave) continue;
                bool first = true;
                float sum = 0.f;
                for (int j0 = 0; j0 < p.biases && first; j0 += 64) {
                    const Bias other = j0 == i0 ? mine : bias_of(p, seq, j0);
                    unsigned long long same = __ballot(j0 + lane < p.biases && other.token == token);
                    first = !same || j0 + __ffsll(same) - 1 >= i0 + l;
                    while (first && same) {
                        sum += __int_as_float(__builtin_amdgcn_readlane(__float_as_int(other.value), __ffsll(same) - 1));
                        same &= same - 1;
                    }
                }
                if (first && lane == 0) biases[token - t0] = sum;
            }
        }
    }
    __syncthreads();
}

// Over a wave: within rows of 16 lanes, then over the rows' ends.
template <int CONTROL, int ROWS, typename Join>
__device__ __forceinline__ float moved(float x, float none, const Join& join) {
    return join(x, __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(none), __float_as_int(x), CONTROL, ROWS, 0xf, false)));
}
template <typename Join>
__device__ __forceinline__ float over_wave(float x, float none, const Join& join) {
    x = moved<0x111, 0xf>(x, none, join);                       // row_shr:1, 2, 4, 8
    x = moved<0x112, 0xf>(x, none, join);
    x = moved<0x114, 0xf>(x, none, join);
    x = moved<0x118, 0xf>(x, none, join);
    x = moved<0x142, 0xa>(x, none, join);                       // row_bcast:15 to rows 1 and 3
    x = moved<0x143, 0xc>(x, none, join);                       // row_bcast:31 to rows 2 and 3
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}
// (lanes without another keep their own)
template <int CONTROL, int ROWS>
__device__ __forceinline__ int from_lane(int x) { return __builtin_amdgcn_update_dpp(x, x, CONTROL, ROWS, 0xf, false); }
template <typename T, typename Join>
__device__ __forceinline__ T best_of_wave(T x, const Join& join) {
    x = join(x, from_lane<0x111, 0xf>(x));
    x = join(x, from_lane<0x112, 0xf>(x));
    x = join(x, from_lane<0x114, 0xf>(x));
    x = join(x, from_lane<0x118, 0xf>(x));
    x = join(x, from_lane<0x142, 0xa>(x));
    x = join(x, from_lane<0x143, 0xc>(x));
    return __builtin_amdgcn_readlane(x, 63);
}
// A float's order as an integer's: of negative ones the lower bits are turned over.
__device__ __forceinline__ int ordered(float x) {
    const int i = __float_as_int(x);
    return i ^ ((i >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float largest_of_wave(float x) {
    const int i = best_of_wave(ordered(x), [](int a, int b) { return a > b ? a : b; });
    return __int_as_float(i ^ ((i >> 31) & 0x7fffffff));
}
__device__ __forceinline__ int lowest_of_wave(int x) { return best_of_wave(x, [](int a, int b) { return a < b ? a : b; }); }
__device__ __forceinline__ float sum_of_wave(float x) { return over_wave(x, 0.f, [](float a, float b) { return a + b; }); }
// What a row comes to: probabilities are 2^((z - top) heat) / sum each, or for greedy sequences 1 at place `at`.  A NaN among the
// exponentials is one in their sum, and so comes to all of them.
struct RowSum {
    float top, sum;
    int at;
};
// Logits of probabilities are held in units of 2^16, before the temperature's factor, so that what stays within 2^143 loses nothing: rows that are
// all of the type's lowest value are (times a repetition).  (Powers of two round nothing; what lies below 2^-133 is gone.)  heat: that
// factor, log2 e and the unit, at most 2^117.
constexpr float kLogitUnit = 0x1p16f;
__device__ __forceinline__ float exp_of(float z, float top, float heat) { return __builtin_amdgcn_exp2f((z - top) * heat); }
// Of all of a thread's, 2^(z heat - near), near = top heat rounded; returned is what makes 2^((z - top) heat) of them, so that what is lost goes with
// z - top and not with z (logits around 1000: 1.8e-5 of the row where the factor was part of z, 1e-7 so).  One instruction each, where
// near is small enough for its rounding to be a factor close to 1; the difference first where it is not.
template <int U>
__device__ __forceinline__ float exps_of(float (&z)[U][8], float top, float heat) {
    const float from = top == -INFINITY ? 0.f : top, near = from * heat;
    if (fabsf(near) < 0x1p20f) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) z[u][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[u][i], heat, -near));
        return __builtin_amdgcn_exp2f(-__builtin_fmaf(from, heat, -near));
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < 8; ++i) z[u][i] = exp_of(z[u][i], from, heat);
    return 1.f;
}
// Of n pairs (largest logit, and the sum of exponentials or its place), all threads of a wave for all of them; `mine` is pair `lane`.
__device__ __forceinline__ RowSum row_sum(f32x2 mine, const f32x2* pairs, int n, bool greedy, float heat) {
    const int lane = threadIdx.x & 63;
    RowSum r = {-INFINITY, 0.f, -1};
    if (greedy) {
        // (a NaN among the largest: one is the row's)
        bool bad = lane < n && mine[0] != mine[0];
        if (lane < n) r.top = mine[0];
        for (int i = lane + 64; i < n; i += 64) {
            bad |= pairs[i][0] != pairs[i][0];
            r.top = fmaxf(r.top, pairs[i][0]);
        }
        r.top = largest_of_wave(r.top);
        r.at = lane < n && mine[0] == r.top ? __float_as_int(mine[1]) : 0x7fffffff;
        for (int i = lane + 64; i < n; i += 64)
            if (pairs[i][0] == r.top && __float_as_int(pairs[i][1]) < r.at) r.at = __float_as_int(pairs[i][1]);
        r.at = r.top == -INFINITY ? -1 : lowest_of_wave(r.at);
        if (__any(bad)) r.top = __uint_as_float(0x7fc00000u);
        return r;
    }
    if (lane < n) r.top = mine[0];
    for (int i = lane + 64; i < n; i += 64) r.top = fmaxf(r.top, pairs[i][0]);
    r.top = largest_of_wave(r.top);
    auto part = [&](f32x2 x) { return x[0] == -INFINITY ? x[1] : x[1] * exp_of(x[0], r.top, heat); };
    if (lane < n) r.sum = part(mine);
    for (int i = lane + 64; i < n; i += 64) r.sum += part(pairs[i]);
    r.sum = sum_of_wave(r.sum);
    return r;
}

// WHAT: 0 writes logits, 1 leaves a pair of every span, 2 writes probabilities by these, 3 writes probabilities of rows that a workgroup
// has whole.  A thread has U times 8 adjacent tokens for all rows, and holds what is taken from their logits (looks it up
// in LDS for every row where there are 32).
template <int TYPE, int THREADS, int U, int WHAT>
__global__ __launch_bounds__(THREADS) void logits_kernel(const LogitsParams p) {
    typedef typename Elem<TYPE>::T T;
    constexpr int SPAN = THREADS * U * 8, WAVES = THREADS / 64;
    constexpr bool EARLY = U <= 2;                              // the next row is requested before this one is used (32 tokens: no registers left)
    extern __shared__ float lds[];                              // pairs [2][WAVES], then counts and biases
    f32x2* pairs = reinterpret_cast<f32x2*>(lds);
    float* space = lds + 4 * WAVES;
    const long long group = p.first + blockIdx.x;
    const int seq = static_cast<int>(group / p.spans), span = static_cast<int>(group - static_cast<long long>(seq) * p.spans), t0 = span * SPAN;
    int me = threadIdx.x;
    const int lane = me & 63, wave = __builtin_amdgcn_readfirstlane(me >> 6);
    const bool counting = p.history || p.drafts;
    uint32_t* counts = counting ? reinterpret_cast<uint32_t*>(space) : nullptr;
    float* biases = p.biases > 0 ? space + (counting ? SPAN : 0) : nullptr;
    T raw[U][8];
    uint32_t allowed[U];
    f32x2 pair = {0.f, 0.f};
    auto request = [&](int row) {
        if (WHAT == 2) pair = p.stats[(static_cast<long long>(seq) * p.rows + row) * p.spans + (lane < p.spans ? lane : 0)];
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
    const int* drafts = p.drafts + static_cast<long long>(seq) * (p.rows - 1);
    int draft = p.drafts && lane < p.rows - 1 ? drafts[lane] : -1;      // of the row after lane `lane` (of the 64 that it is among)
    if (counting || biases) count_tokens<THREADS, SPAN>(p, seq, t0, counts, biases);
    // Logits times the temperature's reciprocal, or for exponentials (but for greedy sequences) in their unit.  z becomes z by - less: by is that
    // factor, for a token said before with its repetition's, less its penalties without its biases.
    const float scale = WHAT == 0 || k.greedy ? k.heat : 1.f / kLogitUnit, heat = k.heat * (1.4426950408889634f * kLogitUnit);
    const float again = k.repetition * scale, inverse = 1.f / k.repetition * scale;
    auto less_of = [&](uint32_t c, float bias) {
        const uint32_t said = c & ~kInPrompt;
        return ((said ? __builtin_fmaf(static_cast<float>(said), k.frequency, k.presence) : 0.f) - bias) * scale;
    };
    float less[U][8];
    bool seen[U][8];
    auto look_up = [&](int u) {
        const int at = (u * THREADS + me) * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t c = counting ? counts[at + i] : 0;
            seen[u][i] = c != 0;
            less[u][i] = less_of(c, biases ? biases[at + i] : 0.f);
        }
    };
    if (EARLY) {
#pragma unroll
        for (int u = 0; u < U; ++u) look_up(u);
    }
    const bool some = counting || biases;

    for (int row = 0; row < p.rows; ++row) {
        // (the tokens' places are worked out anew for each row: kept over the loop, they take the registers that the logits need)
        if (!EARLY) asm volatile("" : "+v"(me));
        if (!EARLY && row > 0) request(row);
        if (row > 0 && p.drafts) {
            if (row > 1 && ((row - 1) & 63) == 0) draft = row - 1 + lane < p.rows - 1 ? drafts[row - 1 + lane] : -1;
            const uint32_t at = static_cast<uint32_t>(__builtin_amdgcn_readlane(draft, (row - 1) & 63)) - static_cast<uint32_t>(t0);
            const int mine = static_cast<int>((at >> 3) % THREADS);
            if (at < static_cast<uint32_t>(SPAN) && mine >> 6 == wave) {       // (this wave's: the counts are read by nobody else)
                if (mine == me) counts[at] += 1;
#pragma unroll
                for (int u = 0; u < (EARLY ? U : 0); ++u)
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (mine == me && static_cast<int>(at) == (u * THREADS + mine) * 8 + i) {
                            seen[u][i] = true;
                            less[u][i] = less_of(counts[at], biases ? biases[at] : 0.f);
                        }
            }
        }
        const f32x2 my_pair = pair;
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
            if (some) {
                if (!EARLY) look_up(u);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float by = z[u][i] > 0.f ? inverse : again;
                    z[u][i] = __builtin_fmaf(z[u][i], seen[u][i] ? by : scale, -less[u][i]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) z[u][i] *= scale;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t bit = static_cast<uint32_t>(static_cast<int>(keep[u] << (31 - i)) >> 31);         // all ones or none
                z[u][i] = __uint_as_float((__float_as_uint(z[u][i]) & bit) | (0xff800000u & ~bit));
            }
            if (!EARLY) __builtin_amdgcn_sched_barrier(0);
        }
        const long long r = static_cast<long long>(seq) * p.rows + row;
        RowSum sum = {0.f, 0.f, -1};
        float by = 0.f;                                         // makes probabilities of z's exponentials
        if constexpr (WHAT == 1 || WHAT == 3) {
            f32x2 mine;
            float top = -INFINITY, fix = 1.f;
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < 8; ++i) top = fmaxf(top, z[u][i]);
            top = largest_of_wave(top);
            if (k.greedy) {
                // the lowest place with the largest logit, among this thread's (constants) and the wave's
                int at = U * 8;
                bool bad = false;
#pragma unroll
                for (int u = U - 1; u >= 0; --u)
#pragma unroll
                    for (int i = 7; i >= 0; --i) {
                        at = z[u][i] == top ? u * 8 + i : at;
                        bad |= z[u][i] != z[u][i];
                    }
                at = at == U * 8 ? 0x7fffffff : t0 + ((at >> 3) * THREADS + me) * 8 + (at & 7);
                mine = (f32x2){__any(bad) ? __uint_as_float(0x7fc00000u) : top, __int_as_float(lowest_of_wave(at))};
            } else {
                float all = 0.f;
                fix = exps_of(z, top, heat);                    // (all -infinity: sum 0, but for a NaN)
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int i = 0; i < 8; ++i) all += z[u][i];
                mine = (f32x2){top, sum_of_wave(all) * fix};
            }
            f32x2* mine_at = pairs + (row & 1) * WAVES;         // (the other ones may still be read)
            if (lane == 0) mine_at[wave] = mine;
            __syncthreads();
            if (WHAT == 1 && wave > 0) continue;
            sum = row_sum(mine_at[lane < WAVES ? lane : 0], mine_at, WAVES, k.greedy, heat);
            if (WHAT == 1) {
                if (lane == 0) p.stats[r * p.spans + span] = (f32x2){sum.top, k.greedy ? __int_as_float(sum.at) : sum.sum};
                continue;
            }
            by = sum.sum == 0.f ? 0.f : fix * (mine[0] == -INFINITY ? 1.f : exp_of(mine[0], sum.top, heat)) / sum.sum;
        }
        if constexpr (WHAT == 2) {
            sum = row_sum(my_pair, p.stats + r * p.spans, p.spans, k.greedy, heat);
            const float fix = k.greedy ? 1.f : exps_of(z, sum.top, heat);
            by = sum.sum == 0.f ? 0.f : fix / sum.sum;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int e = t0 + (u * THREADS + me) * 8;
            if constexpr (WHAT != 0) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (k.greedy) z[u][i] = sum.top != sum.top ? sum.top : sum.at - e == i ? 1.f : 0.f;
                    else z[u][i] *= by;
                }
            }
            if (e < p.vocab) store8_type(p.out_type, p.out, seq * p.out_seq_stride + row * p.out_stride, e, p.vocab, z[u]);
        }
    }
}

}  // namespace biq
