// Attention over the paged 8-bit cache (biq_attention).
//
//   s_t = scale q.k_t,  m = max s_t,  l = sum exp(s_t - m),  o = (1/l) sum exp(s_t - m) v_t
//
// in one pass over the tokens with a running m, l and o.  A wave takes 64 tokens (4 blocks of 16) at a time and computes the
// transposed products, so that nothing crosses lanes between the two of them:
//   S^T = K Q^T   4 tiles of 16 tokens x 16 rows.  Row m of tile t is token 16 (m / 4) + 4 t + m % 4, so that the 16 sums of a
//                 lane (16 x 16 x 32 MFMA: lane l holds column l % 16, rows 4 (l / 16) ..) are the 16 tokens of block l / 16:
//                 one scale per lane for the keys, one for the values.
//   O^T = V^T P^T The lane's probabilities are the right operand as they lie (k index 8 (l / 16) + j of step h is token
//                 16 (l / 16) + 8 h + j), and the left operand wants the 16 tokens of block l / 16 at one element: 16 adjacent
//                 bytes of the cache's value layout.
// The order of the elements along k of Q K^T is free as well: a lane reads 16 adjacent bytes of a key.
#pragma once

#include "biq_serve.h"

namespace biq {

struct AttendParams {
    Cache cache;
    Ragged ragged;
    Rows q, out;
    float* lse;
    float* part;             // pieces of units, [slot][row of the tile][dim] sums, ..
    float* stats;            // .. and [slot][row of the tile][2] references and sums of weights
    int* owners;             // [unit][2] first and last share with steps of the unit
    int q_heads, group, causal, window;
    int seqs, row_tiles;     // row_tiles: the most that a sequence's rows make
    int shares;              // > 0: workgroups that share all steps equally; 0: a workgroup per unit
    unsigned first;          // first workgroup of this launch (0 where they share the steps)
    int negative;            // the scale is below 0: q is negated
    float scale;             // |scale| * log2(e)
};

// What a workgroup spends on a unit beside its steps (rows, first keys, joining its waves, results), in steps: 32 sequences of 410 ..
// 4096 tokens take 44.7, 41.7, 39.9, 40.8 us with 2, 5, 10, 14, five rows of 16 sequences 50.0, 50.0, 48.6, 47.7.
constexpr int kUnitCost = 10;

// A unit is a tile of rows of a sequence and head; its work is steps of 64 tokens, [base, base + 64 steps), the same for all
// units of a sequence (every token that one of its rows sees).
struct SeqWork {
    RowRange range;
    int len, base, steps;    // steps of a unit: one at least, as a row that sees nothing has a result too
    int tiles;               // units per head
    __device__ __forceinline__ int cost() const { return steps + kUnitCost; }
    __device__ __forceinline__ int total(int heads) const { return cost() * tiles * heads; }
};
template <int ROWS>
__device__ __forceinline__ SeqWork seq_work(const AttendParams& p, int seq) {
    SeqWork w;
    w.len = p.cache.length(seq);
    w.range = p.ragged.range(seq, w.len);
    int lo = p.window > 0 ? w.range.token - p.window + 1 : 0;
    lo = lo < 0 ? 0 : lo;
    w.base = lo & ~63;
    w.steps = (w.len - w.base + 63) >> 6;
    w.steps = w.steps < 1 ? 1 : w.steps;
    w.tiles = (w.range.count * p.group + ROWS - 1) / ROWS;
    return w;
}

// All units of a call in a row, sequence by sequence, in it heads slowest, each taking kUnitCost places and one for each of
// its steps.  Every workgroup has an equal share of the places, whatever the lengths are.  Every wave finds its place by
// itself: a lane per sequence, 64 at a time.
template <int ROWS>
struct Shares {
    const AttendParams& p;
    int lane, upto, total;   // upto: running sum over the first 64 sequences
    int count;               // shares: none without a place
    __device__ __forceinline__ Shares(const AttendParams& params, int l, bool used = true) : p(params), lane(l), upto(0), total(0), count(0) {
        if (!used) return;
        for (int s = 0; s < p.seqs; s += 64) {
            const int x = running(s);
            if (s == 0) upto = x;
            total += __builtin_amdgcn_readlane(x, 63);
        }
        count = p.shares < total ? p.shares : total;
    }
    __device__ __forceinline__ int running(int s0) const {
        const int s = s0 + lane;
        int x = s < p.seqs ? seq_work<ROWS>(p, s).total(p.cache.heads) : 0;
        // running sum: in rows of 16 lanes, then the rows' ends
        x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);      // row_shr:1, 2, 4, 8
        x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
        x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
        x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
        x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);     // row_bcast:15 to rows 1 and 3
        x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);     // row_bcast:31 to rows 2 and 3
        return x;
    }
    // First place of share w.
    __device__ __forceinline__ int begin(int w) const {
        return static_cast<int>(static_cast<unsigned long long>(static_cast<unsigned>(total)) * static_cast<unsigned>(w) / static_cast<unsigned>(count));
    }
    // Share that place x belongs to.
    __device__ __forceinline__ int owner(int x) const {
        return static_cast<int>((static_cast<unsigned long long>(x + 1) * static_cast<unsigned>(count) - 1) / static_cast<unsigned>(total));
    }
    // Sequence of place x (x < total), which becomes the place's number in the sequence.
    __device__ __forceinline__ int find(int& x) const {
        for (int s = 0;; s += 64) {
            const int sums = s == 0 ? upto : running(s);
            const unsigned long long above = __ballot(sums > x);
            if (above) {
                const int l = __ffsll(above) - 1;
                if (l > 0) x -= __builtin_amdgcn_readlane(sums, l - 1);
                return s + l;
            }
            x -= __builtin_amdgcn_readlane(sums, 63);
        }
    }
};

__device__ __forceinline__ float exp2_raw(float x) { return __builtin_amdgcn_exp2f(x); }

// log(2^ref total): the exponent of total is taken off first, as ref and log2(total) mostly cancel.
__device__ __forceinline__ float log_sum(float ref, float total) {
    if (total == 0.f) return -INFINITY;
    const float m = __builtin_amdgcn_frexp_mantf(total);
    return ((ref + static_cast<float>(__builtin_amdgcn_frexp_expf(total))) + __builtin_amdgcn_logf(m)) * 0.69314718055994531f;
}

constexpr float kNoRef = -3.402823466e38f;            // reference of a row that has seen nothing

// 2^x, x <= 0, in two factors.  A sum of weights is brought to a later reference by both, one after the other: references follow the
// values' scales, so that zeros or tiny values beside large ones make x less than -126, and a sum of weights of 2^100 and more.
struct Factor {
    float half;
    __device__ __forceinline__ explicit Factor(float x) : half(exp2_raw(0.5f * x)) {}
    __device__ __forceinline__ float of(float sum) const { return sum * half * half; }
    __device__ __forceinline__ float whole() const { return half * half; }
};

// The matrix cores multiply 16-bit floats: both code formats fit them exactly, and a 32-bit number is two of them to 22 bits
// once it is scaled into their range.  Terms of q: two for 32-bit elements, one otherwise (bf16 values have 8 bits).
template <int TYPE> struct RowTerms { static constexpr int value = TYPE == BIQ_F32 ? 2 : 1; };
// Terms of the weights: one (11 bits) where the output has 8 bits, two otherwise.  (Prompts of 4096 rows in bf16 are off by 1.67e-3 from
// 64 bits with one, 1.66e-3 with 32-bit weights: the output's own rounding.)
template <int TYPE> struct WeightTerms { static constexpr int value = TYPE == BIQ_BF16 ? 1 : 2; };

template <int TERMS>
__device__ __forceinline__ void f16_terms(const float (&x)[8], f16x8 (&out)[TERMS]) {
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
        const f16x2 hi = __builtin_convertvector((f32x2){x[j], x[j + 1]}, f16x2);
        out[0][j] = hi[0];
        out[0][j + 1] = hi[1];
        if constexpr (TERMS == 2) {
            const f16x2 lo = __builtin_convertvector((f32x2){x[j] - static_cast<float>(hi[0]), x[j + 1] - static_cast<float>(hi[1])}, f16x2);
            out[1][j] = lo[0];
            out[1][j + 1] = lo[1];
        }
    }
}

template <int TYPE>
__device__ __forceinline__ void store_row4(const Rows& out, long long at, f32x4 x) {
    if (out.quads) store_elem4<TYPE>(out.data, at, x);
    else
#pragma unroll
        for (int j = 0; j < 4; ++j) store_elem<TYPE>(out.data, at + j, x[j]);
}

// Row tiles, their place in the tensors and what they see.
struct RowPlace {
    long long row;           // -1: none
    int head, lo, hi;
};
__device__ __forceinline__ RowPlace row_place(const AttendParams& p, RowRange range, int len, int head, int rr, int rows_all) {
    RowPlace r;
    const int i = rr / p.group, pos = range.token + i;
    r.row = rr < rows_all ? range.first + i : -1;
    r.head = head * p.group + (rr - i * p.group);
    r.hi = p.causal ? pos : len - 1;
    r.lo = p.window > 0 ? pos - p.window + 1 : 0;
    return r;
}

// Elements of the row of a lane's column: part (c, h) holds elements 64 c + 16 (lane / 16) + 8 h ..  Lanes without a row and parts
// beyond the head request some of a row that there is (row `other`), and get zeros.  HALF: of the last 64 elements only the first 32
// are there, and part (CH - 1, 0) holds 8 (lane / 16) .. of these.
template <int TYPE, int CH, bool HALF>
struct RowElems {
    Elems<TYPE, 8> part[CH][2];
    __device__ __forceinline__ static int element(int c, int h, int grp) { return c * 64 + (HALF && c == CH - 1 ? grp * 8 : grp * 16 + h * 8); }
    __device__ __forceinline__ void request(const AttendParams& p, const RowPlace& r, int other, int dim, int grp) {
        const auto* row = static_cast<const typename Elem<TYPE>::T*>(p.q.data) + (r.row >= 0 ? r.row : other) * p.q.row_stride + r.head * p.q.head_stride;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (HALF && c == CH - 1 && h == 1) continue;
                const int d = element(c, h, grp);
                part[c][h].request(row + (d < dim ? d : 0));
            }
    }
    __device__ __forceinline__ void get(const RowPlace& r, int dim, int grp, float (&x)[CH][2][8]) const {
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (HALF && c == CH - 1 && h == 1) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[c][h][j] = 0.f;
                } else {
                    part[c][h].get(x[c][h], r.row >= 0 && element(c, h, grp) < dim);
                }
            }
    }
};

// The same as right operands.  Rows of 32-bit or bf16 elements are scaled by a power of two, their largest magnitude to
// [2^14, 2^15); returned is what undoes it.
template <int TYPE, int CH>
__device__ __forceinline__ float row_terms(bool negative, float (&x)[CH][2][8], f16x8 (&q)[CH][2][RowTerms<TYPE>::value]) {
    float up = 1.f, down = 1.f;
    if constexpr (TYPE != BIQ_F16) {
        float most = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf(x[c][h][j]));
        most = max_over_groups(most);
        int e = static_cast<int>(__float_as_uint(most) >> 23);          // biased exponent
        e = most == 0.f ? 127 + 14 : e < 27 ? 27 : e;
        up = __uint_as_float(static_cast<uint32_t>(127 + 14 + 127 - e) << 23);
        down = __uint_as_float(static_cast<uint32_t>(e - 14) << 23);
    }
    if (negative) up = -up;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int j = 0; j < 8; ++j) x[c][h][j] *= up;
            f16_terms<RowTerms<TYPE>::value>(x[c][h], q[c][h]);
        }
    return down;
}

// A lane's 16 scores of one row against the tokens first .. first + 15 of a block -> weights times the block's value scale v,
//     y = 2^(score kscale - ref) v,  sum += range.unit * sum of 2^(score kscale - ref),
// as PT 16-bit terms per 8 tokens.
//
// y has to stay in the range of 16-bit floats whatever v is, so ref follows the running maximum of score + log2 v (v taken as
// 2^-108 at least, the least that the cache's writer makes), kRefStart below it, and only where y would pass 2^kRefRoom: then
// `grown` is set (for the whole wave), and what was summed is to be multiplied by `keep`.  A y below 2^-25 is lost to the sum of the
// values, so n tokens behind a dominant one lose n 2^-(25 + kRefStart) of the weight at most: 2^-38 for outputs of 32 and 16 bits
// and 2^-31 for bf16 (130000 tokens: 5e-7 and 6e-5).  The nearer to the maximum the more often the reference moves: ragged
// prompts in 32 bits take 79 us instead of 76, two prompts in bf16 would take 821 instead of 790.
// With one term v is added to the exponent as its logarithm, and divided out of the sum once, as long as all scales of the wave's
// steps were between 2^-60 and 2^40 (range.narrow): then no y that counts in the sum is below 2^-126.
//
// A weight without its v is up to 2^(15.9 - log2 v), which over many tokens of tiny or no values leaves 32 bits' range: from the
// first block with v below 2^-60 on a wave keeps its sum in units of 2^32 (range.unit), which 2^31 weights of 2^124 fit in.
// (Values above 2^105 beside such blocks would fall out of the sum at its other end.)
struct ScaleRange {
    bool narrow = true;
    float unit = 1.f;
    // Before a step whose value scales are v (valid: tokens of the lane's block).  (With branches prompts in fp32 are 2 to 3 % slower.)
    template <int NT>
    __device__ __forceinline__ void see(float v, int valid, float (&sum)[NT]) {
        narrow &= !__any((valid > 0) & !((v >= 0x1p-60f) & (v <= 0x1p40f)));
        const float by = (unit == 1.f) & static_cast<bool>(__any((valid > 0) & (v < 0x1p-60f))) ? 0x1p-32f : 1.f;
        unit *= by;
#pragma unroll
        for (int n = 0; n < NT; ++n) sum[n] *= by;
    }
    // After the last step: reference of a sum in that unit (the sums of values are to be multiplied by it).
    __device__ __forceinline__ float reference(float ref) const { return unit == 1.f ? ref : ref + 32.f; }
};
struct Sight { int lo, hi, first, valid; };           // tokens seen: lo .. hi, and the block's first `valid`
template <int PT> constexpr float kRefStart = PT == 1 ? 6.f : 13.f;
template <int PT> constexpr float kRefRoom = PT == 1 ? 14.f : 15.9f;
template <int PT>
__device__ __forceinline__ void weigh(const f32x4 (&s)[4], float kscale, float v, bool whole, Sight see, const ScaleRange& range, float& ref, float& sum,
                                      bool& grown, float& keep, f16x8 (&out)[2][PT]) {
    float x[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) x[j] = s[j >> 2][j & 3];
    if (!whole) {                                     // (scaled first: a block that is hidden may have any scale)
        const int lo = see.lo - see.first, hi = see.hi - see.first < see.valid - 1 ? see.hi - see.first : see.valid - 1;
#pragma unroll
        for (int j = 0; j < 16; ++j) x[j] = j < lo || j > hi ? -INFINITY : x[j] * kscale;
        kscale = 1.f;
        v = lo > 15 || hi < 0 || hi < lo ? 1.f : v;
    }
    float top = x[0];
#pragma unroll
    for (int j = 1; j < 16; ++j) top = fmaxf(top, x[j]);
    const float lv = fmaxf(__builtin_amdgcn_logf(v), -108.f);
    top = __builtin_fmaf(top, kscale, lv);            // (kscale >= 0, or NaN)
    grown = __any(top > ref + kRefRoom<PT>);
    keep = 1.f;
    if (grown) {
        const float most = max_over_groups(top);
        const float next = most > ref + kRefRoom<PT> ? most - kRefStart<PT> : ref;       // (a row's bits do not depend on its neighbours)
        const Factor down(ref - next);
        sum = down.of(sum);
        keep = down.whole();
        ref = next;
    }
    float part = 0.f;
    if (PT == 1 && range.narrow) {
        const float c = lv - ref;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const f32x2 y = {exp2_raw(__builtin_fmaf(x[8 * h + j], kscale, c)), exp2_raw(__builtin_fmaf(x[8 * h + j + 1], kscale, c))};
                const f16x2 w = __builtin_convertvector(y, f16x2);
                out[h][0][j] = w[0];
                out[h][0][j + 1] = w[1];
                part += y[0] + y[1];
            }
        part *= exp2_raw(-lv);
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float e = exp2_raw(__builtin_fmaf(x[8 * h + j], kscale, -ref));
                part += e;
                y[j] = e * v;
            }
            f16_terms<PT>(y, out[h]);
        }
    }
    sum = __builtin_fmaf(part, range.unit, sum);
}

// Where a lane finds the codes of a step of 64 tokens (4 blocks): keys of block kblock, values and scales of block vblock.  The
// step is the same for all lanes, so pages are looked up with scalar loads: a vector load would wait its turn behind all
// codes that were requested before it.  Blocks without a page point to page 0, and have no valid tokens.
struct StepPlace {
    const uint8_t* keys;
    const uint8_t* values;
    const float* scales;     // of the keys; of the values: heads * page_blocks further
    int valid;               // tokens of vblock that the sequence has
    bool all;                // the sequence has all 64
};
__device__ __forceinline__ StepPlace step_place(const Cache& c, int dim, int seq, int head, int t0, int len, int kblock, int vblock) {
    typedef const __attribute__((address_space(4))) int* ScalarInts;
    const ScalarInts table = (ScalarInts)(c.table + static_cast<long long>(seq) * c.table_stride);
    const int block_bytes = kCacheBlock * dim, b0 = t0 >> 4;
    const long long codes = static_cast<long long>(c.heads) * c.page_blocks * block_bytes;
    auto lookup = [&](int i) {
        const int n = table[i < c.table_stride ? i : 0];
        return i < c.table_stride && static_cast<uint32_t>(n) < static_cast<uint32_t>(c.num_pages) ? n : -1;
    };
    StepPlace s;
    int left;
    if ((c.page_blocks & 3) == 0) {                             // one page
        const int i = c.page_index(b0), n = lookup(i);
        const int block = head * c.page_blocks + (b0 - i * c.page_blocks);
        const uint8_t* page = c.store + (n < 0 ? 0 : n) * c.page_bytes;
        const uint8_t* first = page + static_cast<long long>(block) * block_bytes;
        s.keys = first + static_cast<uint32_t>(kblock * block_bytes);
        s.values = first + codes + static_cast<uint32_t>(vblock * block_bytes);
        s.scales = reinterpret_cast<const float*>(page + 2 * codes + 4ll * block) + static_cast<uint32_t>(vblock);
        s.all = n >= 0 && len - t0 >= 64;
        left = n < 0 ? 0 : len - t0 - vblock * kCacheBlock;
    } else {
        long long code_at[4], scale_at[4];
        int end[4];
        s.all = len - t0 >= 64;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = c.page_index(b0 + j), n = lookup(i);
            const int block = head * c.page_blocks + (b0 + j - i * c.page_blocks);
            const long long page = (n < 0 ? 0 : n) * c.page_bytes;
            code_at[j] = page + static_cast<long long>(block) * block_bytes;
            scale_at[j] = page + 2 * codes + 4ll * block;
            end[j] = n < 0 ? 0 : len - (b0 + j) * kCacheBlock;
            s.all = s.all && n >= 0;
        }
        // (by value: a choice between elements of an array would put the array into memory)
        auto of = [](auto x0, auto x1, auto x2, auto x3, int block) {
            const auto a = block & 1 ? x1 : x0, b = block & 1 ? x3 : x2;
            return block & 2 ? b : a;
        };
        s.keys = c.store + of(code_at[0], code_at[1], code_at[2], code_at[3], kblock);
        s.values = c.store + codes + of(code_at[0], code_at[1], code_at[2], code_at[3], vblock);
        s.scales = reinterpret_cast<const float*>(c.store + of(scale_at[0], scale_at[1], scale_at[2], scale_at[3], vblock));
        left = of(end[0], end[1], end[2], end[3], vblock);
    }
    s.valid = left < 0 ? 0 : left > kCacheBlock ? kCacheBlock : left;
    return s;
}

// Codes of tokens that the sequence does not have may be anything: zeros.
__device__ __forceinline__ u32x4 first_codes(u32x4 w, int valid) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int left = valid - 4 * i;
        w[i] &= left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
    }
    return w;
}

// Few rows of a sequence and head (one token with its heads, drafted tokens).  The waves of a workgroup hold the same rows and take
// steps of 64 tokens in turn, straight from memory to registers: every code is used by one wave only.  Keys are requested a
// step ahead, values before the scores.  The waves' sums are joined through LDS.
//
// Memory bounds it where units are long: one token of 32 heads over 131071 tokens (269 MB, fp8, bf16) takes 50.4 us, 5.3 TB/s.
// Where a workgroup has several shorter units, what it does beside their steps shows (10 steps' worth each), and with 32-bit rows
// the instructions of a step (4 waves of a CU issue 5000 cycles each: 320 of 520 vector instructions turn codes into 16-bit
// floats): 32 sequences of 410 .. 4096 tokens (155 MB, int8, fp32) take 35 us, 4.4 TB/s, 5 rows of 16 sequences 40 us
// (42 where 16-bit rows were converted one load after the other).
// CH: 64 elements of a head each; FULL: the head has all of them; NT: tiles of 16 rows.
template <int TYPE, int FMT, int CH, bool FULL, int NT, int WAVES>
__global__ __launch_bounds__(64 * WAVES, CH * NT == 1 ? 3 : CH * NT == 2 ? 2 : 1) void attend_rows_kernel(const AttendParams p) {
    constexpr int QT = RowTerms<TYPE>::value, PT = WeightTerms<TYPE>::value;
    constexpr int ROWS = 16 * NT;
    extern __shared__ float lds[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int col = lane & 15, grp = lane >> 4;
    const int dim = FULL ? 64 * CH : p.cache.dim;
    const int kblock = col >> 2;                                // block of this lane's key rows, 0 .. 3

    // steps of this workgroup: a share of all, or all of one unit
    const Shares<ROWS> shares(p, lane, p.shares > 0);
    int from = 0, upto = 1;
    if (p.shares > 0) {
        if (static_cast<int>(blockIdx.x) >= shares.count) return;
        from = shares.begin(blockIdx.x);
        upto = shares.begin(blockIdx.x + 1);
    }
    for (bool again = false; from < upto;) {
    int seq, unit, step = 0, stop;                              // (unit of the sequence: head * tiles + tile)
    if (p.shares > 0) {
        stop = from;
        seq = __builtin_amdgcn_readfirstlane(shares.find(stop));
    } else {
        seq = static_cast<int>(p.first + blockIdx.x) / (p.cache.heads * p.row_tiles);
    }
    const SeqWork work = seq_work<ROWS>(p, seq);
    if (p.shares > 0) {
        unit = stop / work.cost();
        const int place = stop - unit * work.cost(), left = upto - from;
        step = place > kUnitCost ? place - kUnitCost : 0;
        stop = place + left < work.cost() ? place + left - kUnitCost : work.steps;
        from += left < work.cost() - place ? left : work.cost() - place;
        if (stop <= step) continue;                             // no step in this share
    } else {
        const int r = static_cast<int>(p.first + blockIdx.x) - seq * (p.cache.heads * p.row_tiles), t = r % p.row_tiles;
        if (t >= work.tiles) return;
        unit = r / p.row_tiles * work.tiles + t;
        stop = work.steps;
        from = upto;
    }
    const int head = unit / work.tiles, tile = unit - head * work.tiles;
    // a piece that ends before its unit does: the share's second slot if it begins it, else the first
    const int slot = stop - step == work.steps ? -1 : 2 * static_cast<int>(blockIdx.x) + (step == 0 ? 1 : 0);
    if (p.shares > 0 && step == 0 && threadIdx.x == 0) {
        const int id = (seq * p.cache.heads + head) * p.row_tiles + tile;
        p.owners[2 * id] = blockIdx.x;
        p.owners[2 * id + 1] = stop == work.steps ? blockIdx.x : shares.owner(from - 1 - stop + work.steps);
    }
    const RowRange range = work.range;
    const int len = work.len;
    const int rows_all = range.count * p.group, row0 = tile * ROWS;     // (token, head of the group), heads fastest
    const int pos0 = range.token;                               // (negative: before the first token)
    const int pos_first = pos0 + row0 / p.group;
    const int pos_last = pos0 + ((row0 + ROWS < rows_all ? row0 + ROWS : rows_all) - 1) / p.group;
    const int begin = work.base + step * 64, end = work.base + stop * 64;

    // the rows are requested first: they are needed first
    RowPlace place[NT];
    RowElems<TYPE, CH, false> elems[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        place[n] = row_place(p, range, len, head, row0 + n * 16 + col, rows_all);
        elems[n].request(p, place[n], range.first, dim, grp);
    }
    u32x4 kc[4][CH];                                            // token 4 t + col % 4 of that block
    float ks = 0.f, vs = 0.f;
    const uint8_t* vbase = p.cache.store;
    int valid = 0;
    bool all_valid = false;
    auto request_keys = [&](int t0) {
        const StepPlace at = step_place(p.cache, dim, seq, head, t0, len, kblock, grp);
        vbase = at.values;
        valid = at.valid;
        all_valid = at.all;
        // (scales of blocks that do not exist are not used, whatever they are)
        ks = at.scales[0];
        vs = at.scales[p.cache.heads * p.cache.page_blocks];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                int d = c * 64 + grp * 16;
                d = FULL || d < dim ? d : 0;                    // (against zeros of q)
                kc[t][c] = *reinterpret_cast<const u32x4*>(at.keys + (4 * t + (col & 3)) * dim + d);
            }
    };
    int t0 = begin + __builtin_amdgcn_readfirstlane(wave) * 64;
    if (t0 < end) request_keys(t0);

    f16x8 q[NT][CH][2][QT];
    float unit_of[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        float x[CH][2][8];
        elems[n].get(place[n], dim, grp, x);
        unit_of[n] = row_terms<TYPE, CH>(p.negative, x, q[n]) * p.scale;
    }

    // tokens that every row of the tile sees
    const int all_lo = p.window > 0 ? pos_last - p.window + 1 : 0;
    const int all_hi = p.causal ? pos_first : len - 1;
    f32x4 o[NT][CH * 4];
    float ref[NT], l[NT];
    ScaleRange scales;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        ref[n] = kNoRef;
        l[n] = 0.f;
#pragma unroll
        for (int t = 0; t < CH * 4; ++t) o[n][t] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    for (; t0 < end; t0 += 64 * WAVES) {
        u32x4 vc[CH * 4];
#pragma unroll
        for (int t = 0; t < CH * 4; ++t) {
            const int d = FULL || t * 16 < dim ? t * 16 + col : col;    // (beyond the head: sums that are not stored)
            vc[t] = *reinterpret_cast<const u32x4*>(vbase + d * kCacheBlock);
        }
        const float kscale = ks, vscale = vs;
        const int nvalid = valid;
        const bool step_valid = all_valid;
        __builtin_amdgcn_sched_barrier(0);                      // (the requests stay ahead of the products)
        scales.see(vscale, nvalid, l);
        f32x4 s[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int t = 0; t < 4; ++t) s[n][t] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                f16x8 k[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) k[t] = codes_f16<FMT>(kc[t][c][2 * h], kc[t][c][2 * h + 1]);
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < QT; ++e)
#pragma unroll
                        for (int t = 0; t < 4; ++t) s[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k[t], q[n][c][h][e], s[n][t], 0, 0, 0);
            }
        // (always, the last ones again: loads under a condition would all be waited for before the values' products)
        __builtin_amdgcn_sched_barrier(0);
        request_keys(t0 + 64 * WAVES < end ? t0 + 64 * WAVES : t0);
        __builtin_amdgcn_sched_barrier(0);

        const bool whole = step_valid && t0 + 63 <= all_hi && t0 >= all_lo;
        if (!whole) {
#pragma unroll
            for (int t = 0; t < CH * 4; ++t) vc[t] = first_codes(vc[t], nvalid);
        }
        f16x8 w[NT][2][PT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            bool grown;
            float keep;
            const Sight see = {place[n].lo, place[n].hi, t0 + grp * kCacheBlock, nvalid};
            weigh<PT>(s[n], kscale * unit_of[n], vscale, whole, see, scales, ref[n], l[n], grown, keep, w[n]);
            if (grown) {
#pragma unroll
                for (int t = 0; t < CH * 4; ++t) o[n][t] *= keep;
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int t = 0; t < CH * 4; ++t) {
                const f16x8 v = codes_f16<FMT>(vc[t][2 * h], vc[t][2 * h + 1]);
#pragma unroll
                for (int e = 0; e < PT; ++e)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
                        o[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, w[n][h][e], o[n][t], 0, 0, 0);
            }
    }

    // ---- the waves' sums, joined: every wave's go to LDS, then every thread adds 4 elements of a row ------------------
    // Sums (tile i of 16 elements, lane) lie at 16-byte place 64 i + 16 grp + (col + 4 i + grp) % 16: neither the lanes that
    // write a tile nor those that read a row meet on a bank.
    float* stats = lds;                                         // [wave][ROWS][2]
    f32x4* sums = reinterpret_cast<f32x4*>(lds + WAVES * ROWS * 2);     // [wave][NT][CH * 4][64]
    if (again) __syncthreads();                                 // (the unit before is read)
    again = true;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const float total = sum_over_groups(l[n]);
        if (grp == 0) *reinterpret_cast<f32x2*>(stats + (wave * ROWS + n * 16 + col) * 2) = (f32x2){scales.reference(ref[n]), total};
#pragma unroll
        for (int i = 0; i < CH * 4; ++i)
            sums[((wave * NT + n) * (CH * 4) + i) * 64 + grp * 16 + ((col + 4 * i + grp) & 15)] = o[n][i] * scales.unit;
    }
    __syncthreads();
    const int quads = dim / 4, rows_here = rows_all - row0 < ROWS ? rows_all - row0 : ROWS;
    for (int at = threadIdx.x; at < rows_here * quads; at += 64 * WAVES) {
        const int rr = at / quads, d = at - rr * quads;         // row of the tile, its elements 4 d ..
        f32x2 st[WAVES];
        float now = kNoRef, total = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            st[w] = *reinterpret_cast<const f32x2*>(stats + (w * ROWS + rr) * 2);
            now = fmaxf(now, st[w][0]);
        }
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const Factor f(st[w][0] - now);
            total += f.of(st[w][1]);
            acc += sums[((w * NT + rr / 16) * (CH * 4) + d / 4) * 64 + (d & 3) * 16 + ((rr + d) & 15)] * f.whole();
        }
        if (slot >= 0) {
            const long long to = static_cast<long long>(slot) * ROWS + rr;
            *reinterpret_cast<f32x4*>(p.part + to * dim + 4 * d) = acc;
            if (d == 0) *reinterpret_cast<f32x2*>(p.stats + to * 2) = (f32x2){now, total};
            continue;
        }
        const RowPlace r = row_place(p, range, len, head, row0 + rr, rows_all);
        store_row4<TYPE>(p.out, r.row * p.out.row_stride + r.head * p.out.head_stride + 4 * d, acc * (total == 0.f ? 0.f : 1.f / total));
        if (p.lse && d == 0) p.lse[r.row * p.q_heads + r.head] = log_sum(now, total);
    }
    }
}

// READS operands from LDS and the EACH products of every one of them: read(i) four ahead of use(i, operand).  (Left alone, the compiler
// reads each operand right before its products and waits for it.)  Either the scheduler is asked for this order, which leaves it
// free to place what else there is to do (two prompts with heads of 128: 806 us instead of 812), or, FENCED, the reads stand where they
// are meant to be and only other vector and scalar instructions pass: with heads above 128 the scheduler gives up its own order now and
// then (heads of 256 in bf16: 365 us instead of 288).
template <int READS, int EACH, bool FENCED, typename Read, typename Use>
__device__ __forceinline__ void read_ahead(const Read& read, const Use& use) {
    constexpr int kAhead = 4;
    if constexpr (FENCED) {
        constexpr int kVectorAndScalar = 0x6;
        f16x8 ring[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) ring[i] = read(i);
#pragma unroll
        for (int i = 0; i < READS; ++i) {
            use(i, ring[i % kAhead]);
            if (i + kAhead < READS) ring[i % kAhead] = read(i + kAhead);
            __builtin_amdgcn_sched_barrier(kVectorAndScalar);
        }
    } else {
        constexpr int kReads = 0x100, kProducts = 0x8;
#pragma unroll
        for (int i = 0; i < READS; ++i) use(i, read(i));
        __builtin_amdgcn_sched_group_barrier(kReads, kAhead, 0);
#pragma unroll
        for (int i = 0; i < READS - kAhead; ++i) {
            __builtin_amdgcn_sched_group_barrier(kProducts, EACH, 0);
            __builtin_amdgcn_sched_group_barrier(kReads, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(kProducts, kAhead * EACH, 0);
    }
}

// Many rows of a sequence and head (prompts).  The waves of a workgroup hold different rows, NT tiles of 16 each, and share the
// tokens: a stage of WAVES / 4 steps of 64 is requested a stage ahead, each code by one wave, and laid down in LDS as the 16-bit
// operands that all waves read, in the order of the lanes that read them (lane after lane: no bank is met twice).  Two
// buffers, one barrier a stage.
//
// What the SIMDs issue bounds it: matrix products (64 a step of a wave with two tiles of bf16 rows, 19 cycles each), exponentials (32, 27
// cycles) and other vector instructions (240, 3 cycles) measured apart add up to 2800 cycles, a step takes 2300.  Two prompts of
// 4096 rows over 8192 tokens, 32 heads of 128: 806 us, 1.02 PFLOP/s.  Tiles of 16 x 16 rather than 32 x 32 as their products
// are 20 % faster a flop here and their layout gives a lane one scale.
template <int TYPE, int FMT, int CH, bool FULL, bool HALF, int NT, int WAVES>
__global__ __launch_bounds__(64 * WAVES, CH <= 2 ? 2 : 1) void attend_tile_kernel(const AttendParams p) {
    constexpr int QT = RowTerms<TYPE>::value, PT = WeightTerms<TYPE>::value;
    constexpr int STEPS = WAVES / 4, ROWS = 16 * NT * WAVES;
    constexpr int SIDE = 8 * CH * 64;                           // places for a step's keys as operands; as many for its values
    constexpr int KEYS = 2 * CH - HALF, VALUES = 4 * CH - 2 * HALF;      // operands of 32 elements; of 16
    extern __shared__ float lds[];
    f16x8* buffers = reinterpret_cast<f16x8*>(lds);             // [2][STEPS][keys [4][CH][2], values [CH * 4][2]][64]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, grp = lane >> 4;
    const int dim = FULL ? 64 * CH : p.cache.dim;
    // Later rows see more tokens and come first.  Where the sequences and heads can be dealt to the XCDs evenly, each keeps to
    // its own, whose tokens then stay in its L2.
    const int pairs = p.seqs * p.cache.heads, group = p.first + blockIdx.x;
    int pair, tile;
    if (pairs % kXcds == 0) {
        const int at = group / kXcds;
        pair = at / p.row_tiles * kXcds + group % kXcds;
        tile = p.row_tiles - 1 - at % p.row_tiles;
    } else {
        pair = group % pairs;
        tile = p.row_tiles - 1 - group / pairs;
    }
    const int seq = pair / p.cache.heads, head = pair - seq * p.cache.heads;
    const int len = p.cache.length(seq);
    const RowRange range = p.ragged.range(seq, len);
    const int rows_all = range.count * p.group, row0 = tile * ROWS;
    if (row0 >= rows_all) return;
    const int pos0 = range.token;
    const int last_row = (row0 + ROWS < rows_all ? row0 + ROWS : rows_all) - 1;
    int begin = p.window > 0 ? pos0 + row0 / p.group - p.window + 1 : 0;
    begin = begin < 0 ? 0 : begin & ~63;
    const int end = p.causal ? pos0 + last_row / p.group + 1 : len;

    // this wave's rows
    RowPlace place[NT];
    RowElems<TYPE, CH, HALF> elems[NT];
    f16x8 q[NT][CH][2][QT];
    float unit_of[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        place[n] = row_place(p, range, len, head, row0 + (wave * NT + n) * 16 + col, rows_all);
        elems[n].request(p, place[n], range.first, dim, grp);
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        float x[CH][2][8];
        elems[n].get(place[n], dim, grp, x);
        unit_of[n] = row_terms<TYPE, CH>(p.negative, x, q[n]) * p.scale;
    }
    // what all and what some of them see
    const int wave_row = row0 + wave * NT * 16;
    const int wave_last = wave_row + NT * 16 < rows_all ? wave_row + NT * 16 - 1 : rows_all - 1;
    const int pos_first = pos0 + wave_row / p.group, pos_last = pos0 + wave_last / p.group;
    const int all_lo = p.window > 0 ? pos_last - p.window + 1 : 0, all_hi = p.causal ? pos_first : len - 1;
    const int any_lo = p.window > 0 ? pos_first - p.window + 1 : 0, any_hi = wave_row < rows_all ? p.causal ? pos_last : len - 1 : -1;

    // this wave's part of a stage: of step wave / 4 the key rows of tile wave % 4 and the values of CH tiles of 16 elements
    const int my_step = wave >> 2, my_part = wave & 3;
    u32x4 kc[CH], vc[CH];
    float ks[STEPS], vs[STEPS];
    int valid[STEPS];
    bool all_valid[STEPS];
    auto request = [&](int t0) {
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const StepPlace at = step_place(p.cache, dim, seq, head, t0 + 64 * i, len, col >> 2, grp);
            valid[i] = at.valid;
            all_valid[i] = at.all;
            ks[i] = at.scales[0];
            vs[i] = at.scales[p.cache.heads * p.cache.page_blocks];
            if (i != my_step) continue;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int kd = c * 64 + grp * 16, vd = (my_part * CH + c) * 16;
                const uint8_t* key = at.keys + (4 * my_part + (col & 3)) * dim;
                if constexpr (HALF) {
                    if (c == CH - 1) {
                        const int hd = c * 64 + grp * 8;
                        const u32x2 eight = *reinterpret_cast<const u32x2*>(key + (hd < dim ? hd : 0));
                        kc[c] = (u32x4){eight[0], eight[1], 0u, 0u};
                    } else {
                        kc[c] = *reinterpret_cast<const u32x4*>(key + kd);
                    }
                } else {
                    kc[c] = *reinterpret_cast<const u32x4*>(key + (FULL || kd < dim ? kd : 0));
                }
                vc[c] = *reinterpret_cast<const u32x4*>(at.values + ((FULL || vd < dim ? vd : 0) + col) * kCacheBlock);
            }
        }
    };
    auto lay_down = [&](f16x8* to) {
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
            if (i == my_step && !all_valid[i]) {
#pragma unroll
                for (int c = 0; c < CH; ++c) vc[c] = first_codes(vc[c], valid[i]);
            }
        to += my_step * 2 * SIDE;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (!HALF || c < CH - 1 || h == 0) to[((my_part * CH + c) * 2 + h) * 64 + lane] = codes_f16<FMT>(kc[c][2 * h], kc[c][2 * h + 1]);
                if (HALF && my_part * CH + c >= VALUES) continue;
                to[SIDE + ((my_part * CH + c) * 2 + h) * 64 + lane] = codes_f16<FMT>(vc[c][2 * h], vc[c][2 * h + 1]);
            }
    };

    f32x4 o[NT][VALUES];
    float ref[NT], l[NT];
    ScaleRange scales;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        ref[n] = kNoRef;
        l[n] = 0.f;
#pragma unroll
        for (int t = 0; t < VALUES; ++t) o[n][t] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    auto see_scales = [&]() {
#pragma unroll
        for (int i = 0; i < STEPS; ++i) scales.see(vs[i], valid[i], l);
    };
    if (begin < end) {
        request(begin);
        lay_down(buffers);
        __syncthreads();
        see_scales();
    }
    int parity = 0;
    for (int stage = begin; stage < end; stage += 64 * STEPS) {
        float kscale[STEPS], vscale[STEPS];
        int nvalid[STEPS];
        bool step_valid[STEPS];
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            kscale[i] = ks[i];
            vscale[i] = vs[i];
            nvalid[i] = valid[i];
            step_valid[i] = all_valid[i];
        }
        request(stage + 64 * STEPS < end ? stage + 64 * STEPS : stage);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const int t0 = stage + 64 * i;
            const f16x8* from = buffers + (parity * STEPS + i) * 2 * SIDE;
            if (t0 >= end || t0 > any_hi || t0 + 63 < any_lo) continue;
            f32x4 s[NT][4];
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int n = 0; n < NT; ++n) s[n][t] = (f32x4){0.f, 0.f, 0.f, 0.f};
            read_ahead<4 * KEYS, QT * NT, (CH > 2)>([&](int r) { return from[(r / KEYS * 2 * CH + r % KEYS) * 64 + lane]; }, [&](int r, f16x8 k) {
                const int t = r / KEYS, c = r % KEYS / 2, h = r % KEYS % 2;
#pragma unroll
                for (int e = 0; e < QT; ++e)
#pragma unroll
                    for (int n = 0; n < NT; ++n) s[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, q[n][c][h][e], s[n][t], 0, 0, 0);
            });
            __builtin_amdgcn_sched_barrier(0);
            const bool whole = step_valid[i] && t0 + 63 <= all_hi && t0 >= all_lo;
            f16x8 w[NT][2][PT];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                bool grown;
                float keep;
                const Sight see = {place[n].lo, place[n].hi, t0 + grp * kCacheBlock, nvalid[i]};
                weigh<PT>(s[n], kscale[i] * unit_of[n], vscale[i], whole, see, scales, ref[n], l[n], grown, keep, w[n]);
                if (grown) {
#pragma unroll
                    for (int t = 0; t < VALUES; ++t) o[n][t] *= keep;
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            read_ahead<2 * VALUES, PT * NT, (CH > 2)>([&](int r) { return from[SIDE + r * 64 + lane]; }, [&](int r, f16x8 v) {
                const int t = r / 2, h = r % 2;
#pragma unroll
                for (int e = 0; e < PT; ++e)
#pragma unroll
                    for (int n = 0; n < NT; ++n) o[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, w[n][h][e], o[n][t], 0, 0, 0);
            });
        }
        __builtin_amdgcn_sched_barrier(0);
        parity ^= 1;
        lay_down(buffers + parity * STEPS * 2 * SIDE);
        __syncthreads();
        see_scales();
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const float total = sum_over_groups(l[n]);
        if (place[n].row < 0) continue;
        const float inv = total == 0.f ? 0.f : 1.f / total;
        const long long to = place[n].row * p.out.row_stride + place[n].head * p.out.head_stride + grp * 4;
#pragma unroll
        for (int i = 0; i < VALUES; ++i)
            if (FULL || i * 16 < dim) store_row4<TYPE>(p.out, to + i * 16, o[n][i] * scales.unit * inv);
        if (p.lse && grp == 0) p.lse[place[n].row * p.q_heads + place[n].head] = log_sum(scales.reference(ref[n]), total);
    }
}

// Units whose steps went to several workgroups, joined: a workgroup per row of a unit.  LANES lanes hold 4 elements each of one
// piece, so 256 / LANES pieces are read at once.  Latency bounds it: 4.3 us for 32 rows of 33 pieces, 5 for 1024 rows of 1 to 5.
template <int TYPE, int ROWS, int LANES>
__global__ __launch_bounds__(256) void attend_join_kernel(const AttendParams p, int tile_rows) {
    constexpr int GROUPS = 256 / LANES;
    __shared__ f32x4 sums[256];
    const int unit = blockIdx.x / tile_rows, rr = blockIdx.x - unit * tile_rows;
    const int tile = unit % p.row_tiles, head = unit / p.row_tiles % p.cache.heads, seq = unit / p.row_tiles / p.cache.heads;
    const SeqWork work = seq_work<ROWS>(p, seq);
    const int rows_all = work.range.count * p.group;
    if (tile * ROWS + rr >= rows_all) return;
    // pieces: the second slot of share w0, then the first ones of w0 + 1 .. w1
    const int w0 = p.owners[2 * unit], n = p.owners[2 * unit + 1] - w0 + 1;
    if (n == 1) return;                                         // in one piece: the output is there
    auto at = [&](int k) { return static_cast<long long>(k == 0 ? 2 * w0 + 1 : 2 * (w0 + k)) * ROWS + rr; };
    const f32x2* stats = reinterpret_cast<const f32x2*>(p.stats);
    const int lane = threadIdx.x & 63, dim = p.cache.dim;
    float ref = kNoRef;
    for (int k = lane; k < n; k += 64) ref = fmaxf(ref, stats[at(k)][0]);
#pragma unroll
    for (int d = 32; d > 0; d /= 2) ref = fmaxf(ref, __shfl_xor(ref, d));
    float total = 0.f;
    for (int k = lane; k < n; k += 64) total += Factor(stats[at(k)][0] - ref).of(stats[at(k)][1]);
#pragma unroll
    for (int d = 32; d > 0; d /= 2) total += __shfl_xor(total, d);
    const int g = threadIdx.x / LANES, d = threadIdx.x % LANES * 4;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    if (d < dim)
#pragma unroll 4
        for (int k = g; k < n; k += GROUPS) acc += *reinterpret_cast<const f32x4*>(p.part + at(k) * dim + d) * exp2_raw(stats[at(k)][0] - ref);
    sums[threadIdx.x] = acc;
    __syncthreads();
    if (g != 0 || d >= dim) return;
#pragma unroll
    for (int k = 1; k < GROUPS; ++k) acc += sums[k * LANES + threadIdx.x];
    const RowPlace place = row_place(p, work.range, work.len, head, tile * ROWS + rr, rows_all);
    store_row4<TYPE>(p.out, place.row * p.out.row_stride + place.head * p.out.head_stride + d, acc * (total == 0.f ? 0.f : 1.f / total));
    if (p.lse && threadIdx.x == 0) p.lse[place.row * p.q_heads + place.head] = log_sum(ref, total);
}

}  // namespace biq
