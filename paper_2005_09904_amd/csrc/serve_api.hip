// C ABI of the operators around the multiply in a decoder step (include/biq.h): argument checks, choice of the mapping,
// launches.
#include <math.h>

#include "biq_serve_launch.h"

namespace biq {
namespace {

constexpr int kCus = 256;
constexpr long long kMaxInt = 0x7fffffff;

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
bool type_ok(int type) { return type == BIQ_F32 || type == BIQ_BF16 || type == BIQ_F16; }
size_t type_bytes(int type) { return type == BIQ_F32 ? 4 : 2; }

biq_status status(hipError_t e) { return e == hipSuccess ? BIQ_OK : BIQ_EHIP; }

// No stride below 0, and none whose product with a row or head number leaves 64 bits.
bool rows_ok(const biq_rows& r, int type) {
    const long long most = 1ll << 31;
    return r.data && aligned(r.data, type_bytes(type)) && r.row_stride >= 0 && r.head_stride >= 0 && r.row_stride <= most &&
           r.head_stride <= most;
}
Rows rows_of(const biq_rows& r, int type) {
    Rows out{r.data, r.row_stride, r.head_stride, 0};
    const int most = static_cast<int>(4 / type_bytes(type));    // elements in 4 bytes
    out.quads = aligned(r.data, 4) && r.row_stride % most == 0 && r.head_stride % most == 0;
    return out;
}

biq_status cache_check(const biq_cache& c) {
    if (!c.store || !c.table || !c.lens || !aligned(c.store, 16) || !aligned(c.table, 4) || !aligned(c.lens, 4)) return BIQ_EINVAL;
    if (c.num_pages < 1 || c.page_tokens < 1 || c.table_stride < 1 || c.seqs < 1 || c.heads < 1 || c.head_dim < 1) return BIQ_EINVAL;
    if (c.format != BIQ_CACHE_INT8 && c.format != BIQ_CACHE_FP8) return BIQ_EINVAL;
    if (c.page_tokens % kCacheBlock || c.page_tokens > 256 || c.head_dim % 16 || c.head_dim > 256) return BIQ_EUNSUPPORTED;
    if (c.heads > 65536 || static_cast<long long>(c.table_stride) * c.page_tokens > kMaxInt - 4096) return BIQ_EUNSUPPORTED;
    return BIQ_OK;
}
Cache cache_of(const biq_cache& c) {
    Cache d{};
    d.store = static_cast<uint8_t*>(c.store);
    d.table = c.table;
    d.lens = c.lens;
    d.page_bytes = static_cast<long long>(biq_cache_page_bytes(c.page_tokens, c.heads, c.head_dim));
    d.num_pages = c.num_pages;
    d.table_stride = c.table_stride;
    d.heads = c.heads;
    d.dim = c.head_dim;
    d.page_blocks = c.page_tokens / kCacheBlock;
    d.page_magic = static_cast<uint32_t>((1ull << 32) / d.page_blocks + 1);
    d.page_ones = d.page_blocks == 1 ? ~0u : 0u;
    return d;
}

bool ragged_ok(const biq_ragged& r, int seqs) {
    if (r.rows < 1 || r.max_rows < 1 || r.max_rows > r.rows || !aligned(r.starts, 4)) return false;
    return r.starts || static_cast<long long>(seqs) * r.max_rows == r.rows;
}

// Token numbers, counted from the first row (which may lie before token 0), stay within 32 bits.
bool tokens_fit(const biq_ragged& r, const biq_cache& c) {
    return static_cast<long long>(r.max_rows) + static_cast<long long>(c.table_stride) * c.page_tokens <= kMaxInt - 4096;
}

bool rotation_ok(const biq_rotation& r, int head_dim) {
    return aligned(r.angles, 8) && r.positions >= 1 && r.rot >= 2 && r.rot % 2 == 0 && r.rot <= head_dim;
}

// Most blocks of 16 that n adjacent tokens touch.
int blocks_touched(int n) { return (n - 1 + kCacheBlock - 1) / kCacheBlock + 1; }

int chunks_of(int head_dim) { return (head_dim + 63) / 64; }

// ---- attention: how a call is mapped ----------------------------------------------------------------------

struct AttendPlan {
    bool tiles;              // the kernel for many rows
    int nt, waves;           // tiles of 16 rows per wave, waves per workgroup
    long long row_tiles;
    int shares;              // workgroups that share all steps; 0: a workgroup per unit
    size_t workspace;
};

biq_status attend_check(const biq_attention_args* a) {
    if (!a) return BIQ_EINVAL;
    if (biq_status s = cache_check(a->cache); s != BIQ_OK) return s;
    if (!type_ok(a->type) || a->q_heads < 1 || a->max_len < 0 || a->window < 0 || !ragged_ok(a->ragged, a->cache.seqs)) return BIQ_EINVAL;
    if (a->q_heads % a->cache.heads) return BIQ_EINVAL;
    if (!tokens_fit(a->ragged, a->cache)) return BIQ_EUNSUPPORTED;
    if (a->q_heads > 65536 || static_cast<long long>(a->ragged.rows) * a->q_heads > kMaxInt) return BIQ_EUNSUPPORTED;
    return BIQ_OK;
}

AttendPlan attend_plan(const biq_attention_args& a) {
    AttendPlan pl{};
    const biq_cache& c = a.cache;
    const long long rows = static_cast<long long>(a.ragged.max_rows) * (a.q_heads / c.heads);      // of a sequence and head
    const long long room = static_cast<long long>(c.table_stride) * c.page_tokens;
    long long span = a.max_len > 0 ? a.max_len : room;
    if (a.window > 0 && static_cast<long long>(a.window) + a.ragged.max_rows + 64 < span) span = static_cast<long long>(a.window) + a.ragged.max_rows + 64;
    const long long steps = (span + 63) / 64, pairs = static_cast<long long>(c.seqs) * c.heads;

    // Few rows or many: by the time of a step of 64 tokens (bf16, us; heads of 64, 128, 192, 256).  For few rows the CUs share the
    // steps of all units: kRows each.  For many a workgroup walks through its steps alone: kAlone each, kShared where two of
    // them are on a CU (one for heads above 128).  Measured for 8 heads of 4, 1 .. 16 sequences of 4 .. 512 rows over 1024 and
    // 8192 tokens: 64 rows of 16 sequences and 8192 tokens 90 us by rows, 217 by tiles, 512 rows 660 and 318.  Other types change
    // both times alike: over these sizes in bf16, fp32 and fp16 the choice takes 1.00 to 1.02 of the better one's time on average for each
    // head size, at most 1.05 for heads of 64 and 128, 1.18 for 192 (256 rows of 16 sequences) and 1.45 for 256 (one sequence, tiles for half
    // of the CUs).
    static const double kRows[4] = {0.46, 0.64, 0.95, 1.19}, kAlone[4] = {1.25, 1.64, 2.0, 2.27}, kShared[4] = {1.7, 2.4, 2.0, 2.27};
    const int ch = chunks_of(c.head_dim) - 1;
    const int few = rows <= 16 || ch > 1 ? 16 : 32, many = ch <= 1 ? 128 : 64;
    const long long tiles = pairs * ((rows + many - 1) / many), slots = ch <= 1 ? 2 * kCus : kCus;
    const double by_rows = static_cast<double>(pairs * ((rows + few - 1) / few)) / kCus * kRows[ch];
    const double by_tiles = tiles <= kCus ? kAlone[ch] : kShared[ch] * static_cast<double>((tiles + slots - 1) / slots);
    if (rows > 16 && by_tiles < by_rows) {
        pl.tiles = true;
        // Eight waves a workgroup spread the tokens' conversion over twice the rows, but are fewer workgroups: where these still
        // fill the GPU four times (two prompts of 4096 rows: 806 us instead of 848; six ragged ones of up to 1500: 93 instead of 79).
        const long long wide = pairs * ((rows + 255) / 256);
        pl.waves = ch <= 1 && wide >= 4 * kCus ? 8 : 4;
        pl.nt = ch <= 1 ? 2 : 1;
        pl.row_tiles = (rows + 16 * pl.nt * pl.waves - 1) / (16 * pl.nt * pl.waves);
        return pl;
    }
    pl.nt = few / 16;
    pl.waves = 4;
    const int tile = few;
    pl.row_tiles = (rows + tile - 1) / tile;
    const long long units = pairs * pl.row_tiles;
    // Lengths are not known here, so a unit per workgroup is only taken where a unit is short: up to 8 steps (77 tokens, 8 units: 6.6 us
    // instead of 10.2: the join is a launch of its own), or 32 where there is a unit for every CU.  Beyond, one workgroup per
    // CU shares the steps (32 sequences of 410 .. 4096 tokens, 8 heads: 40 us instead of 46).
    // Two per CU are slower (41.6) as there are more pieces.
    if (steps > (units >= kCus ? 32 : 8) && units < 16 * kCus && units * (room / 64 + 1 + kUnitCost) < kMaxInt) {
        pl.shares = units * steps < kCus ? static_cast<int>(units * steps) : kCus;
        pl.workspace = static_cast<size_t>(pl.shares) * 2 * tile * (c.head_dim + 2) * 4 + static_cast<size_t>(units) * 8;
    }
    return pl;
}

}  // namespace
}  // namespace biq

using namespace biq;

extern "C" {

size_t biq_cache_page_bytes(int page_tokens, int heads, int head_dim) {
    if (page_tokens < 1 || heads < 1 || head_dim < 1 || page_tokens % kCacheBlock || page_tokens > 256 || head_dim % 16 ||
        head_dim > 256 || heads > 65536)
        return 0;
    const size_t bytes = 2ull * page_tokens * heads * head_dim + 8ull * heads * (page_tokens / kCacheBlock);
    return (bytes + 127) / 128 * 128;
}

biq_status biq_rotary_frequencies(double* turns, int rot, double base, int scaling, double factor, int trained, double slow,
                                  double fast) {
    if (!turns || rot < 2 || rot % 2 || !(base > 1.0) || !isfinite(base)) return BIQ_EINVAL;
    if (scaling < BIQ_ROTARY_PLAIN || scaling > BIQ_ROTARY_BY_PARTS) return BIQ_EINVAL;
    if (scaling != BIQ_ROTARY_PLAIN && (!(factor >= 1.0) || !isfinite(factor))) return BIQ_EINVAL;
    if (scaling == BIQ_ROTARY_BASE && rot < 4) return BIQ_EINVAL;
    if (scaling == BIQ_ROTARY_BY_PARTS && (trained < 1 || !(slow < fast) || !isfinite(slow) || !isfinite(fast))) return BIQ_EINVAL;
    const double two_pi = 6.283185307179586476925286766559;
    if (scaling == BIQ_ROTARY_BASE) base *= pow(factor, static_cast<double>(rot) / (rot - 2));
    for (int i = 0; i < rot / 2; ++i) {
        double f = pow(base, -2.0 * i / rot) / two_pi;
        if (scaling == BIQ_ROTARY_LINEAR) f /= factor;
        if (scaling == BIQ_ROTARY_BY_PARTS) {
            double keep = (f * trained - slow) / (fast - slow);     // 0: stretched, 1: as it is
            keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
            f = f / factor * (1.0 - keep) + f * keep;
        }
        turns[i] = f;
    }
    return BIQ_OK;
}

biq_status biq_rotary_table(const double* turns, float* angles, int rot, int first, int positions, double amplitude,
                            void* stream) {
    if (!turns || !angles || !aligned(turns, 8) || !aligned(angles, 4) || rot < 2 || rot % 2 || first < 0 || positions < 1 ||
        !isfinite(amplitude))
        return BIQ_EINVAL;
    if (static_cast<long long>(positions) * (rot / 2) > 255 * kMaxInt || static_cast<long long>(first) + positions > kMaxInt) return BIQ_EUNSUPPORTED;
    return status(launch_rotary_table(turns, angles, rot / 2, first, positions, amplitude, static_cast<hipStream_t>(stream)));
}

biq_status biq_rotary(const biq_rotary_args* a, void* stream) {
    if (!a || !type_ok(a->type) || a->rows < 1 || a->heads < 1 || a->head_dim < 1 || !a->positions || !aligned(a->positions, 4)) return BIQ_EINVAL;
    if (!a->rotation.angles || !rotation_ok(a->rotation, a->head_dim) || !rows_ok(a->x, a->type) || !rows_ok(a->y, a->type)) return BIQ_EINVAL;
    const bool in_place = a->x.data == a->y.data;
    if (in_place && (a->x.row_stride != a->y.row_stride || a->x.head_stride != a->y.head_stride)) return BIQ_EINVAL;
    if (static_cast<long long>(a->heads) * a->head_dim > kMaxInt ||
        static_cast<long long>(a->rows) * a->heads > 255 * kMaxInt / a->head_dim)
        return BIQ_EUNSUPPORTED;
    RotaryParams p{};
    p.x = rows_of(a->x, a->type);
    p.y = rows_of(a->y, a->type);
    p.positions = a->positions;
    p.rotation = {a->rotation.angles, a->rotation.positions, a->rotation.rot, a->rotation.interleaved != 0};
    p.rows = a->rows;
    p.heads = a->heads;
    p.dim = a->head_dim;
    p.inverse = a->inverse != 0;
    p.copy = !in_place;
    return status(launch_rotary(a->type, p, static_cast<hipStream_t>(stream)));
}

biq_status biq_cache_append(const biq_cache_append_args* a, void* stream) {
    if (!a) return BIQ_EINVAL;
    if (biq_status s = cache_check(a->cache); s != BIQ_OK) return s;
    if (!type_ok(a->type) || !rows_ok(a->k, a->type) || !rows_ok(a->v, a->type) || !ragged_ok(a->ragged, a->cache.seqs)) return BIQ_EINVAL;
    if (a->rotation.angles && !rotation_ok(a->rotation, a->cache.head_dim)) return BIQ_EINVAL;
    AppendParams p{};
    p.cache = cache_of(a->cache);
    p.ragged = {a->ragged.starts, a->ragged.rows, a->ragged.max_rows};
    p.k = rows_of(a->k, a->type);
    p.v = rows_of(a->v, a->type);
    if (a->rotation.angles) p.rotation = {a->rotation.angles, a->rotation.positions, a->rotation.rot, a->rotation.interleaved != 0};
    p.seqs = a->cache.seqs;
    p.blocks = blocks_touched(a->ragged.max_rows);
    if (!tokens_fit(a->ragged, a->cache) || static_cast<long long>(p.seqs) * p.blocks > kMaxInt / (2 * a->cache.heads)) return BIQ_EUNSUPPORTED;
    return status(launch_append(a->type, a->cache.format, chunks_of(a->cache.head_dim), p, static_cast<hipStream_t>(stream)));
}

biq_status biq_cache_read(const biq_cache_read_args* a, void* stream) {
    if (!a) return BIQ_EINVAL;
    if (biq_status s = cache_check(a->cache); s != BIQ_OK) return s;
    if (!type_ok(a->type) || !rows_ok(a->k, a->type) || !rows_ok(a->v, a->type) || !ragged_ok(a->ragged, a->cache.seqs)) return BIQ_EINVAL;
    ReadParams p{};
    p.cache = cache_of(a->cache);
    p.ragged = {a->ragged.starts, a->ragged.rows, a->ragged.max_rows};
    p.k = rows_of(a->k, a->type);
    p.v = rows_of(a->v, a->type);
    p.seqs = a->cache.seqs;
    p.blocks = blocks_touched(a->ragged.max_rows);
    if (!tokens_fit(a->ragged, a->cache) || static_cast<long long>(p.seqs) * p.blocks > kMaxInt / (2 * a->cache.heads)) return BIQ_EUNSUPPORTED;
    return status(launch_read(a->type, a->cache.format, chunks_of(a->cache.head_dim), p, static_cast<hipStream_t>(stream)));
}

size_t biq_attention_workspace_bytes(const biq_attention_args* a) {
    return attend_check(a) == BIQ_OK ? attend_plan(*a).workspace : 0;
}

biq_status biq_attention(const biq_attention_args* a, void* workspace, size_t workspace_bytes, void* stream) {
    if (biq_status s = attend_check(a); s != BIQ_OK) return s;
    if (!rows_ok(a->q, a->type) || !rows_ok(a->out, a->type) || !aligned(a->lse, 4)) return BIQ_EINVAL;
    const AttendPlan pl = attend_plan(*a);
    if (pl.workspace > workspace_bytes) return BIQ_EWORKSPACE;
    if (pl.workspace && (!workspace || !aligned(workspace, 16))) return BIQ_EINVAL;
    AttendParams p{};
    p.cache = cache_of(a->cache);
    p.ragged = {a->ragged.starts, a->ragged.rows, a->ragged.max_rows};
    p.q = rows_of(a->q, a->type);
    p.out = rows_of(a->out, a->type);
    p.lse = a->lse;
    p.q_heads = a->q_heads;
    p.group = a->q_heads / a->cache.heads;
    p.causal = a->causal != 0;
    // (a window that no token is outside of is none)
    p.window = a->window < static_cast<long long>(a->cache.table_stride) * a->cache.page_tokens ? a->window : 0;
    p.seqs = a->cache.seqs;
    p.shares = pl.shares;
    p.negative = a->scale < 0.f;
    p.scale = fabsf(a->scale) * 1.4426950408889634f;
    p.part = static_cast<float*>(workspace);
    p.stats = p.part + static_cast<size_t>(pl.shares) * 2 * 16 * pl.nt * a->cache.head_dim;
    p.owners = reinterpret_cast<int*>(p.stats + static_cast<size_t>(pl.shares) * 2 * 16 * pl.nt * 2);
    if (static_cast<long long>(a->cache.seqs) * a->cache.heads * pl.row_tiles > kMaxInt) return BIQ_EUNSUPPORTED;
    p.row_tiles = static_cast<int>(pl.row_tiles);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    switch (a->type) {
        case BIQ_F32: return status(launch_attend_f32(a->cache.format, pl.tiles, pl.nt, pl.waves, p, s));
        case BIQ_BF16: return status(launch_attend_bf16(a->cache.format, pl.tiles, pl.nt, pl.waves, p, s));
        default: return status(launch_attend_f16(a->cache.format, pl.tiles, pl.nt, pl.waves, p, s));
    }
}

size_t biq_verify_workspace_bytes(int seqs, int vocab) {
    if (seqs < 1 || vocab < 1 || vocab > (1 << 22)) return 0;
    return static_cast<size_t>(seqs) * (static_cast<size_t>((vocab + kVerifySpan - 1) / kVerifySpan) * 8 + 16);
}

biq_status biq_verify_drafts(const biq_verify_args* a, void* workspace, size_t workspace_bytes, void* stream) {
    if (!a || !type_ok(a->type) || !a->p || !a->uniform || !a->tokens || !a->accepted || a->seqs < 1 || a->drafts < 0 || a->vocab < 1)
        return BIQ_EINVAL;
    if (a->drafts > 0 && !a->draft_tokens) return BIQ_EINVAL;
    const size_t size = type_bytes(a->type);
    if (!aligned(a->p, size) || !aligned(a->q, size) || !aligned(a->draft_tokens, 4) || !aligned(a->draft_lens, 4) ||
        !aligned(a->uniform, 4) || !aligned(a->tokens, 4) || !aligned(a->accepted, 4))
        return BIQ_EINVAL;
    const long long most = 1ll << 40;
    for (long long stride : {a->p_seq_stride, a->p_stride, a->q_seq_stride, a->q_stride})
        if (stride < 0 || stride > most) return BIQ_EINVAL;
    if (a->drafts > 63 || a->vocab > (1 << 22) || a->seqs > (1 << 20)) return BIQ_EUNSUPPORTED;
    const size_t need = biq_verify_workspace_bytes(a->seqs, a->vocab);
    if (need > workspace_bytes) return BIQ_EWORKSPACE;
    if (need && (!workspace || !aligned(workspace, 16))) return BIQ_EINVAL;
    VerifyParams p{};
    p.p = a->p;
    p.q = a->drafts > 0 ? a->q : nullptr;
    p.p_seq_stride = a->p_seq_stride;
    p.p_stride = a->p_stride;
    p.q_seq_stride = a->q_seq_stride;
    p.q_stride = a->q_stride;
    p.draft_tokens = a->draft_tokens;
    p.draft_lens = a->draft_lens;
    p.uniform = a->uniform;
    p.tokens = a->tokens;
    p.accepted = a->accepted;
    p.sums = static_cast<unsigned long long*>(workspace);
    p.seqs = a->seqs;
    p.drafts = a->drafts;
    p.vocab = a->vocab;
    p.spans = (a->vocab + kVerifySpan - 1) / kVerifySpan;
    p.verdicts = reinterpret_cast<int*>(p.sums + static_cast<size_t>(a->seqs) * p.spans);
    return status(launch_verify(a->type, p, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
