// C ABI of the operators at the end of a decoder step (include/biq.h): the norm, products with 4-bit weights, logits.  Argument
// checks, choice of the mapping, launches.
#include <math.h>

#include "biq_step_launch.h"

namespace biq {
namespace {

constexpr long long kMaxInt = 0x7fffffff;
constexpr long long kMaxStride = 1ll << 40;
constexpr int kMaxRow = 1 << 24;                     // elements of a row
// Up to 16 vectors are `few` if their operands take this much of LDS at most, so that two workgroups share a CU; more of them, and those
// of larger operands, are `many`.  32000 x 4096, bfloat16: 8 vectors (64 KB) 19.4 us and 16.7 + 4.7 for the join, in a launch of its
// own, 10 vectors 26.8 and 16.5 + 4.7; 4096 x 4096: 8.4 and 6.7 + 3.0, 9.8 and 6.6 + 2.2; 16384 x 2048, 16 vectors (64 KB): 11.0 and 8.2 + 3.7;
// 4096 x 16384, 3 vectors (96 KB): 16.8 and 13.0 + 3.9.
constexpr int kLdsFew4 = 80 * 1024;

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
bool type_ok(int type) { return type == BIQ_F32 || type == BIQ_BF16 || type == BIQ_F16; }
size_t type_bytes(int type) { return type == BIQ_F32 ? 4 : 2; }
bool group_ok(int group) { return group == 32 || group == 64 || group == 128; }
int groups_of(int n, int group) { return group == 0 ? 1 : (n + group - 1) / group; }
biq_status status(hipError_t e) { return e == hipSuccess ? BIQ_OK : BIQ_EHIP; }

// Rows that are read: any stride that is not below 0.  Rows that are written do not overlap.
bool read_ok(long long stride) { return stride >= 0 && stride <= kMaxStride; }
bool write_ok(long long stride, long long rows, int n) { return read_ok(stride) && (rows == 1 || stride >= n); }

// The rows (i, j), i < few, j < many, of n elements at i a + j b: no two of them share an element.  Of sequences' rows one stride spans the others'
// as a rule; else every difference of i is looked at with the two nearest ones of j.
bool rows_apart(long long few, long long a, long long many, long long b, int n) {
    typedef __int128 Wide;
    if (few > many) return rows_apart(many, b, few, a, n);
    if (few == 1) return many == 1 || b >= n;
    if (a < n || b < n) return false;
    if (a >= static_cast<Wide>(many - 1) * b + n || b >= static_cast<Wide>(few - 1) * a + n) return true;
    for (long long i = 1; i < few; ++i)
        for (Wide j = static_cast<Wide>(i) * a / b, last = j + 1; j <= last && j < many; ++j) {
            const Wide gap = static_cast<Wide>(i) * a - j * b;
            if (gap < n && gap > -n) return false;
        }
    return true;
}

// ---- products with 4-bit weights: how a call is mapped -------------------------------------------------------

struct Gemm4Plan {
    bool many;
    int x_scales, f, g, splits, columns, lds;
    size_t workspace;
};

int record_bytes(int group) { return 1024 + 32 * (kBlock4 / group); }

bool shape4_ok(int m, int n, int group) { return m >= 1 && n >= 1 && group_ok(group); }

biq_status gemm4_check(const biq_gemm4_args* a) {
    if (!a || !shape4_ok(a->m, a->n, a->group) || a->batch < 1 || !type_ok(a->y_type)) return BIQ_EINVAL;
    if (!type_ok(a->x_type) && a->x_type != BIQ_X_INT8 && a->x_type != BIQ_X_FP8) return BIQ_EINVAL;
    if (!type_ok(a->x_type) && a->x_group != 0 && !group_ok(a->x_group)) return BIQ_EINVAL;
    if (a->n > kMaxRow || a->m > (1 << 28) || a->batch > 65535) return BIQ_EUNSUPPORTED;
    return BIQ_OK;
}

Gemm4Plan gemm4_plan(const biq_gemm4_args& a) {
    Gemm4Plan pl{};
    const bool codes = !type_ok(a.x_type);
    const int blocks = (a.n + kBlock4 - 1) / kBlock4, tiles = (a.m + 15) / 16, terms = a.x_type == BIQ_F32 ? 2 : 1;
    pl.x_scales = codes && a.x_group != 0 ? kBlock4 / a.x_group : 1;
    const int spans = codes && a.x_group != 0 && a.x_group < a.group ? a.x_group : a.group;
    pl.f = spans / 32;
    pl.g = a.group / 32;
    const long long column = static_cast<long long>(blocks) * (256 * terms + 4 * pl.x_scales);      // bytes of a vector as operands
    pl.columns = a.batch < 16 ? a.batch : 16;
    pl.many = a.n >= 8 && (a.batch > 16 || column * pl.columns > kLdsFew4);
    pl.splits = 1;
    if (!pl.many) {
        while (pl.splits < kWaves4 && static_cast<long long>(tiles) * pl.splits < 256 * kWaves4) pl.splits *= 2;
        const long long lds = column * pl.columns, join = pl.splits > 1 ? kWaves4 * 64 * 16 : 0;
        pl.lds = static_cast<int>(lds > join ? lds : join);
        return pl;
    }
    const int groups = (a.batch + 63) / 64;
    pl.columns = (a.batch + groups - 1) / groups;
    // a workgroup for every CU, four blocks each at least (fewer do not pay for the join: 2 to 5 us in a launch of its own)
    const long long units = static_cast<long long>((a.m + kRows4 - 1) / kRows4) * groups;
    long long splits = units >= 256 ? 1 : 256 / units;
    splits = splits > (blocks + 3) / 4 ? (blocks + 3) / 4 : splits;
    pl.splits = static_cast<int>(splits);
    pl.workspace = splits == 1 ? 0 : static_cast<size_t>(splits) * a.batch * tiles * 64;
    return pl;
}

// Whether workgroups hold whole rows (1024 threads with up to 32 tokens each, whose counts and biases take 4 bytes of LDS each) in one launch,
// or spans in two.  Up to 16384 tokens a workgroup is quicker: one row of 8000 6.6 us instead of 9.6, of 16000 9.2 and 10.0 with
// the second launch's own time not counted.  Beyond, one row of 32000 takes 13.1 us and 10.4, so that it is left to spans until the
// sequences fill half of the CUs (256 of them: 22.7 and 36.6; 64 with four rows each 44.8 and 27).  A workgroup's rows follow one another: 5 rows
// of 8000 take 15.0 us instead of 18.4, of 2000 11.0 instead of 18.5, but 5 of 12000 20.6 and 18.5, of 16000 21.9 and 18.5 (64 rows: 215 and 153).
// Callers hold no workspace for these, so they stay.
bool logits_whole(int vocab, bool biases, int seqs) { return vocab <= 16384 || (vocab <= 32768 && !biases && seqs >= 128); }

}  // namespace
}  // namespace biq

using namespace biq;

extern "C" {

biq_status biq_norm(const biq_norm_args* a, void* stream) {
    if (!a || !a->x || !type_ok(a->type) || a->rows < 1 || a->n < 1 || (!a->y && !a->codes) || (a->sum && !a->residual)) return BIQ_EINVAL;
    if ((a->y && !type_ok(a->y_type)) || !(a->eps >= 0.f) || !isfinite(a->eps) || !isfinite(a->weight_add)) return BIQ_EINVAL;
    if (a->codes && (!a->scales || (a->group != 0 && !group_ok(a->group)) || (a->format != BIQ_CACHE_INT8 && a->format != BIQ_CACHE_FP8))) return BIQ_EINVAL;
    const size_t size = type_bytes(a->type);
    if (!aligned(a->x, size) || !aligned(a->residual, size) || !aligned(a->sum, size) || !aligned(a->weight, 4) || !aligned(a->scales, 4) ||
        (a->y && !aligned(a->y, type_bytes(a->y_type))))
        return BIQ_EINVAL;
    if (!read_ok(a->x_stride) || (a->residual && !read_ok(a->residual_stride)) || (a->sum && !write_ok(a->sum_stride, a->rows, a->n)) ||
        (a->y && !write_ok(a->y_stride, a->rows, a->n)) || (a->codes && !write_ok(a->code_stride, a->rows, a->n)))
        return BIQ_EINVAL;
    // a row is read before it is written, which only the same place of the same row may rely on
    if (a->sum == a->x && a->sum_stride != a->x_stride) return BIQ_EINVAL;
    if (a->sum && a->sum == a->residual && a->sum_stride != a->residual_stride) return BIQ_EINVAL;
    if (a->y == a->x && (a->y_type != a->type || a->y_stride != a->x_stride)) return BIQ_EINVAL;
    if (a->y && a->y == a->residual && (a->y_type != a->type || a->y_stride != a->residual_stride)) return BIQ_EINVAL;
    if (a->y && a->y == a->sum) return BIQ_EINVAL;
    if (a->n > kMaxRow) return BIQ_EUNSUPPORTED;
    NormParams p{};
    p.x = a->x;
    p.residual = a->residual;
    p.sum = a->sum;
    p.weight = a->weight;
    p.y = a->y;
    p.codes = static_cast<uint8_t*>(a->codes);
    p.scales = a->scales;
    p.x_stride = a->x_stride;
    p.residual_stride = a->residual_stride;
    p.sum_stride = a->sum_stride;
    p.y_stride = a->y_stride;
    p.code_stride = a->code_stride;
    p.y_type = a->y_type;
    p.rows = a->rows;
    p.n = a->n;
    p.group = a->codes ? a->group : 0;
    p.groups = groups_of(a->n, p.group);
    p.format = a->format;
    p.eps = a->eps;
    p.weight_add = a->weight_add;
    return status(launch_norm(a->type, p, static_cast<hipStream_t>(stream)));
}

size_t biq_packed4_bytes(int m, int n, int group) {
    if (!shape4_ok(m, n, group) || n > kMaxRow || m > (1 << 28)) return 0;
    return static_cast<size_t>((m + 15) / 16) * ((n + kBlock4 - 1) / kBlock4) * record_bytes(group);
}

static biq_status pack4(const int8_t* codes, const float* scales, const void* w, long long stride, int type, uint8_t* packed, float* out, int m, int n,
                        int group, void* stream) {
    if (!packed || !aligned(packed, 16) || !shape4_ok(m, n, group)) return BIQ_EINVAL;
    if (n > kMaxRow || m > (1 << 28)) return BIQ_EUNSUPPORTED;
    Pack4Params p{};
    p.codes = codes;
    p.source = w;
    p.scales = scales;
    p.packed = packed;
    p.out = out;
    p.stride = stride;
    p.m = m;
    p.n = n;
    p.group = group;
    p.groups = groups_of(n, group);
    p.blocks = (n + kBlock4 - 1) / kBlock4;
    p.record = record_bytes(group);
    const long long records = static_cast<long long>((m + 15) / 16) * p.blocks;
    if (records > 0xffffffffll) return BIQ_EUNSUPPORTED;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    return status(out ? launch_unpack4(p, records, s) : w ? launch_quantize4(type, p, records, s) : launch_pack4(p, records, s));
}

biq_status biq_pack4(const int8_t* codes, const float* scales, uint8_t* packed, int m, int n, int group, void* stream) {
    if (!codes || !scales || !aligned(scales, 4)) return BIQ_EINVAL;
    return pack4(codes, scales, nullptr, 0, 0, packed, nullptr, m, n, group, stream);
}

biq_status biq_quantize4(const void* W, int64_t stride, int type, uint8_t* packed, int m, int n, int group, void* stream) {
    if (!W || !type_ok(type) || !aligned(W, type_bytes(type)) || !read_ok(stride)) return BIQ_EINVAL;
    return pack4(nullptr, nullptr, W, stride, type, packed, nullptr, m, n, group, stream);
}

biq_status biq_unpack4(const uint8_t* packed, float* W, int64_t stride, int m, int n, int group, void* stream) {
    if (!W || !aligned(W, 4) || !write_ok(stride, m, n)) return BIQ_EINVAL;
    return pack4(nullptr, nullptr, nullptr, stride, 0, const_cast<uint8_t*>(packed), W, m, n, group, stream);
}

size_t biq_gemm4_workspace_bytes(const biq_gemm4_args* a) { return gemm4_check(a) == BIQ_OK ? gemm4_plan(*a).workspace : 0; }

biq_status biq_gemm4(const biq_gemm4_args* a, void* workspace, size_t workspace_bytes, void* stream) {
    if (biq_status s = gemm4_check(a); s != BIQ_OK) return s;
    const bool codes = !type_ok(a->x_type);
    if (!a->weights || !a->x || !a->y || !aligned(a->weights, 16) || !aligned(a->y, type_bytes(a->y_type))) return BIQ_EINVAL;
    if (codes ? !a->x_scales || !aligned(a->x_scales, 4) : !aligned(a->x, type_bytes(a->x_type))) return BIQ_EINVAL;
    if (!read_ok(a->x_stride) || !write_ok(a->y_stride, a->batch, a->m)) return BIQ_EINVAL;
    const Gemm4Plan pl = gemm4_plan(*a);
    if (pl.workspace > workspace_bytes) return BIQ_EWORKSPACE;
    if (pl.workspace && (!workspace || !aligned(workspace, 16))) return BIQ_EINVAL;
    Gemm4Params p{};
    p.weights = a->weights;
    p.x = a->x;
    p.x_scales = a->x_scales;
    p.y = a->y;
    p.part = static_cast<float*>(workspace);
    p.x_stride = a->x_stride;
    p.y_stride = a->y_stride;
    p.m = a->m;
    p.n = a->n;
    p.batch = a->batch;
    p.blocks = (a->n + kBlock4 - 1) / kBlock4;
    p.tiles = (a->m + 15) / 16;
    p.record = record_bytes(a->group);
    p.x_group = codes ? a->x_group : 0;
    p.x_groups = groups_of(a->n, p.x_group);
    p.y_type = a->y_type;
    p.splits = pl.splits;
    p.columns = pl.columns;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    return status(pl.many ? launch_gemm4_many(a->x_type, pl.f, pl.g, pl.x_scales, p, s)
                          : launch_gemm4_few(a->x_type, pl.f, pl.g, pl.x_scales, pl.lds, p, s));
}

size_t biq_logits_workspace_bytes(int seqs, int rows, int vocab) {
    if (seqs < 1 || rows < 1 || vocab < 1 || vocab > (1 << 22) || static_cast<long long>(seqs) * rows > kMaxInt) return 0;
    const size_t spans = (vocab + kLogitsSpan - 1) / kLogitsSpan;
    return logits_whole(vocab, true, seqs) ? 0 : static_cast<size_t>(seqs) * rows * spans * 8;
}

biq_status biq_logits(const biq_logits_args* a, void* workspace, size_t workspace_bytes, void* stream) {
    if (!a || !a->x || !a->out || !type_ok(a->type) || !type_ok(a->out_type) || a->seqs < 1 || a->rows < 1 || a->vocab < 1) return BIQ_EINVAL;
    if (!aligned(a->x, type_bytes(a->type)) || !aligned(a->out, type_bytes(a->out_type))) return BIQ_EINVAL;
    for (const void* q : {static_cast<const void*>(a->history), static_cast<const void*>(a->lens), static_cast<const void*>(a->prompt_lens),
                          static_cast<const void*>(a->drafts), static_cast<const void*>(a->repetition), static_cast<const void*>(a->presence),
                          static_cast<const void*>(a->frequency), static_cast<const void*>(a->temperature), static_cast<const void*>(a->bias_tokens),
                          static_cast<const void*>(a->bias_values), static_cast<const void*>(a->mask)})
        if (!aligned(q, 4)) return BIQ_EINVAL;
    if (a->history ? !a->lens || a->width < 1 : a->lens || a->prompt_lens) return BIQ_EINVAL;
    if (a->biases < 0 || (a->biases > 0 && (!a->bias_tokens || !a->bias_values))) return BIQ_EINVAL;
    for (long long stride : {a->x_seq_stride, a->x_stride, a->mask_seq_stride, a->mask_stride})
        if (!read_ok(stride)) return BIQ_EINVAL;
    if (!write_ok(a->out_stride, a->rows, a->vocab) || !write_ok(a->out_seq_stride, a->seqs, a->vocab)) return BIQ_EINVAL;
    if (a->x == a->out && (a->type != a->out_type || a->x_seq_stride != a->out_seq_stride || a->x_stride != a->out_stride)) return BIQ_EINVAL;
    if (a->vocab > (1 << 22) || a->biases > 4096 || static_cast<long long>(a->seqs) * a->rows > kMaxInt) return BIQ_EUNSUPPORTED;
    // (a workgroup steps over a history by up to 2^14 tokens, in 32 bits)
    if (a->history && a->width > kMaxInt - (1 << 16)) return BIQ_EUNSUPPORTED;
    if (!rows_apart(a->seqs, a->out_seq_stride, a->rows, a->out_stride, a->vocab)) return BIQ_EINVAL;
    const bool whole = logits_whole(a->vocab, a->biases > 0, a->seqs);
    const size_t need = a->probabilities ? biq_logits_workspace_bytes(a->seqs, a->rows, a->vocab) : 0;
    if (need > workspace_bytes) return BIQ_EWORKSPACE;
    if (need && (!workspace || !aligned(workspace, 16))) return BIQ_EINVAL;
    LogitsParams p{};
    p.x = a->x;
    p.out = a->out;
    p.x_seq_stride = a->x_seq_stride;
    p.x_stride = a->x_stride;
    p.out_seq_stride = a->out_seq_stride;
    p.out_stride = a->out_stride;
    p.mask_seq_stride = a->mask_seq_stride;
    p.mask_stride = a->mask_stride;
    p.history = a->history;
    p.lens = a->lens;
    p.prompt_lens = a->prompt_lens;
    p.drafts = a->rows > 1 ? a->drafts : nullptr;
    p.repetition = a->repetition;
    p.presence = a->presence;
    p.frequency = a->frequency;
    p.temperature = a->temperature;
    p.bias_tokens = a->bias_tokens;
    p.bias_values = a->bias_values;
    p.mask = a->mask;
    p.stats = static_cast<f32x2*>(workspace);
    p.out_type = a->out_type;
    p.seqs = a->seqs;
    p.rows = a->rows;
    p.vocab = a->vocab;
    p.width = a->width;
    p.biases = a->biases;
    p.spans = (a->vocab + kLogitsSpan - 1) / kLogitsSpan;
    if (static_cast<long long>(p.seqs) * p.spans > 0xffffffffll) return BIQ_EUNSUPPORTED;
    return status(launch_logits(a->type, a->probabilities != 0, whole, p, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
