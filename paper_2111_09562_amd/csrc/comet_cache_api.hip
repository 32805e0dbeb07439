// Host side of the compressed key/value cache: argument checks, launch geometry and the entry points of include/comet.h.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "comet_cache.h"

using namespace comet;

namespace {

#define HIP_TRY(expr)                                                   \
    do {                                                                \
        hipError_t e_ = (expr);                                         \
        if (e_ != hipSuccess) return hip_fail(e_, #expr);               \
    } while (0)

constexpr uint32_t kMaxHeads = 4096, kMaxQueryHeads = 16384, kMaxSeqs = 1u << 22, kMaxRopeDim = 4096;
constexpr uint64_t kMaxRows = 0x7fffffffull, kMaxGroups = 0xffffffull;        // workgroups of 256: fewer than 2^32 threads

bool valid_shape(comet_cache_shape s) {
    return s.n_pages && s.n_pages <= 0x7fffffffu && s.page_tokens && s.page_tokens % kBlk == 0u && s.page_tokens <= (1u << 20) && s.n_slots &&
           s.n_slots <= 0x7fffffffu && s.heads && s.heads <= kMaxHeads && s.dim && s.dim % 32u == 0u && s.dim <= kCacheMaxDim;
}
// Blocks of all pages and heads; false beyond 2^40 (or of the open blocks), far behind any memory.
bool count_blocks(comet_cache_shape s, uint64_t *n) {
    const uint64_t a = (uint64_t)s.n_pages * s.heads;                           // < 2^43
    if (a > (1ull << 40) || (uint64_t)s.n_slots * s.heads > (1ull << 40)) return false;
    *n = a * (s.page_tokens / kBlk);                                            // < 2^55
    return *n <= (1ull << 40);
}
inline uint64_t pad256(uint64_t v) { return (v + 255ull) / 256ull * 256ull; }

bool cache_args(const void *dev, comet_cache_shape s, CacheArgs *c) {
    uint64_t n;
    if (!dev || (uintptr_t)dev % 16u || !valid_shape(s) || !count_blocks(s, &n)) return false;
    uint8_t *p = const_cast<uint8_t *>(static_cast<const uint8_t *>(dev));
    c->blocks = p;
    c->scales = reinterpret_cast<float *>(p + n * 64u * s.dim);
    c->ring = p + n * 64u * s.dim + pad256(n * 8u);
    c->n_pages = s.n_pages; c->per = s.page_tokens / kBlk; c->n_slots = s.n_slots; c->heads = s.heads; c->dim = s.dim;
    return true;
}
bool batch_args(const comet_cache_batch *b, uint32_t n_tokens, int32_t *status, BatchArgs *a) {
    if (!b || b->n_seqs > kMaxSeqs || n_tokens > kMaxRows || (uint64_t)n_tokens / kBlk + 2ull * b->n_seqs > kMaxGroups) return false;
    if (n_tokens && (!b->n_seqs || !b->table_width || !b->dev_starts || !b->dev_lens || !b->dev_table)) return false;
    for (const void *p : {(const void *)b->dev_starts, (const void *)b->dev_lens, (const void *)b->dev_table, (const void *)b->dev_slots, (const void *)status})
        if ((uintptr_t)p % 4u) return false;
    a->starts = b->dev_starts; a->lens = b->dev_lens; a->table = b->dev_table; a->slots = b->dev_slots;
    a->width = b->table_width; a->n_seqs = b->n_seqs; a->n_tokens = n_tokens; a->status = status;
    return true;
}
inline uint32_t elem_size(int dtype) { return dtype == COMET_F32 ? 4u : 2u; }
bool rows_args(comet_rows r, int dtype, Rows *to) {
    if (!r.dev || (uintptr_t)r.dev % elem_size(dtype)) return false;
    to->p = static_cast<uint8_t *>(r.dev); to->token = r.token_stride; to->head = r.head_stride;
    return true;
}
// Rows that are written: no two of them may overlap.  So the rows of a token lie between those of two tokens, or the rows of a head between
// those of two heads.
bool out_args(comet_rows r, int dtype, uint32_t tokens, uint32_t heads, uint32_t dim, Rows *to) {
    const auto size = [](int64_t stride) { return stride < 0 ? 0 - (unsigned __int128)(__int128)stride : (unsigned __int128)stride; };
    const unsigned __int128 token = tokens < 2u ? 0 : size(r.token_stride), head = heads < 2u ? 0 : size(r.head_stride);
    const bool tokens_apart = tokens < 2u || token >= head * (heads - 1u) + dim, heads_apart = heads < 2u || head >= token * (tokens - 1u) + dim;
    return rows_args(r, dtype, to) && (tokens < 2u || token >= dim) && (heads < 2u || head >= dim) && (tokens_apart || heads_apart);
}
// Whether no row of one tensor meets one of another of the same tokens, in bytes.  Told by their ranges, else row by row, for which the
// token strides must be the same: rows of two heads then meet if some whole number of token strides lies near their distance.
// A step over all pairs of heads is one over the distances if the head strides are the same, too.
struct Span {
    __int128 token, head, low, high;                       // high: behind the last byte
    uint32_t heads;
    Span(const Rows &r, uint32_t tokens, uint32_t heads_, uint32_t dim, uint32_t size) : heads(heads_) {
        token = tokens < 2u ? 0 : (__int128)r.token * size;
        head = heads < 2u ? 0 : (__int128)r.head * size;
        const __int128 t = token * ((__int128)tokens - 1), h = head * ((__int128)heads - 1), at = (__int128)(uintptr_t)r.p;
        low = at + (t < 0 ? t : 0) + (h < 0 ? h : 0);
        high = at + (t > 0 ? t : 0) + (h > 0 ? h : 0) + (__int128)dim * size;
    }
};
bool rows_apart(const Rows &x, uint32_t x_heads, const Rows &y, uint32_t y_heads, uint32_t tokens, uint32_t dim, int dtype) {
    const uint32_t size = elem_size(dtype);
    const Span a(x, tokens, x_heads, dim, size), b(y, tokens, y_heads, dim, size);
    if (a.high <= b.low || b.high <= a.low) return true;
    if (a.token != b.token) return false;
    const __int128 length = (__int128)dim * size, base = (__int128)(uintptr_t)y.p - (__int128)(uintptr_t)x.p, step = a.token < 0 ? -a.token : a.token;
    const auto meet = [&](__int128 distance) {             // |distance - m step| < length for some |m| < tokens
        if (distance < 0) distance = -distance;
        if (!step) return distance < length;
        __int128 m = distance / step;
        if (m > (__int128)tokens - 1) m = (__int128)tokens - 1;
        return distance - m * step < length || (m + 1 < (__int128)tokens && (m + 1) * step - distance < length);
    };
    if (a.head == b.head || x_heads < 2u || y_heads < 2u) {
        const __int128 head = x_heads < 2u ? b.head : a.head;
        for (int64_t d = -(int64_t)(x_heads - 1u); d <= (int64_t)(y_heads - 1u); ++d)
            if (meet(base + d * head)) return false;
        return true;
    }
    if ((uint64_t)x_heads * y_heads > (1u << 20)) return false;
    for (uint32_t g = 0; g < y_heads; ++g)
        for (uint32_t h = 0; h < x_heads; ++h)
            if (meet(base + g * b.head - h * a.head)) return false;
    return true;
}
// A result and what it is computed from, which may be the same tensor.
bool same_or_apart(const Rows &x, const Rows &y, uint32_t heads, uint32_t tokens, uint32_t dim, int dtype) {
    return x.p == y.p ? x.token == y.token && x.head == y.head : rows_apart(x, heads, y, heads, tokens, dim, dtype);
}
bool rows_aligned(const Rows &r, int dtype) {                                   // every row begins at a multiple of 16 bytes
    const int64_t v = 16 / elem_size(dtype);
    return (uintptr_t)r.p % 16u == 0u && r.token % v == 0 && r.head % v == 0;
}
bool rope_args(const comet_rope_plan *p, uint32_t dim, const int32_t *positions, RopeArgs *r) {
    *r = RopeArgs{};
    if (!p) return true;
    if (!p->dev_steps || (uintptr_t)p->dev_steps % 8u || p->rot < 2u || p->rot % 2u || p->rot > dim || p->layout > COMET_ROPE_PAIRS ||
        !std::isfinite(p->amp) || (uintptr_t)positions % 4u) return false;
    r->steps = p->dev_steps; r->positions = positions; r->rot = p->rot; r->interleaved = p->layout == COMET_ROPE_PAIRS; r->amp = p->amp;
    return true;
}
inline uint32_t block_units(const BatchArgs &b) { return b.n_tokens / kBlk + 2u * b.n_seqs; }      // (first_unit)

template <typename T, int V>
void launch_rope(const RopeArgs &r, const Rows &x, const Rows &y, uint32_t n_tokens, uint32_t heads, uint32_t dim, bool in_place, uint32_t sign, hipStream_t st) {
    RopeGrid g;
    g.rot_chunks = r.rot / (2u * V);
    g.chunks = g.rot_chunks + (in_place ? 0u : (dim - r.rot) / V);
    // up to eight heads share a chunk's sines, while that leaves a thousand workgroups
    const uint64_t threads = (uint64_t)n_tokens * heads * g.chunks;
    uint64_t per = threads / (1024u * kRopeBlock);
    per = per < 1u ? 1u : (per > 8u ? 8u : per);
    g.groups = (uint32_t)((heads + per - 1u) / per);
    g.per_token = g.groups * g.chunks;
    g.tokens_wg = g.per_token <= (uint32_t)kRopeBlock ? kRopeBlock / g.per_token : 0u;
    uint32_t wg = g.tokens_wg ? (n_tokens - 1u) / g.tokens_wg + 1u : n_tokens;
    if (wg > kMaxGroups) wg = kMaxGroups;
    k_rope<T, V><<<wg, kRopeBlock, 0, st>>>(r, g, x, y, n_tokens, heads, dim, sign);
}

// Workgroups an attention call is cut into, about.  Few rows: 768 are resident at once for heads of 128; more than that even out sequences of
// different lengths (64 x 400 .. 16384 tokens, 8 heads: 119 us with 768, 113 with 1280, 116 with 1536), as long as a tile is not cut that has no more than
// 2048 / dim blocks, 128 KB of keys and values (one that has more falls into equal pieces, of 64 KB at least): beneath that, writing and joining the results costs
// more (64 x 300 .. 4000 tokens, 2 heads of 256: 33 us, with half of that 39; 128 x 500 .. 3000 tokens, 4 heads of 64: 29 and 33).  Short
// sequences gain nothing (48 x 8 .. 4096 tokens, 12 heads of 64: 26 us with either).  Where there are few tiles, two long sequences say (120000 tokens, 8
// heads), 512 pieces take 97 us, 768 take 103; one short sequence is cut down to four blocks, so that its latency is shared.
// Many rows: as many as are resident, one or two per compute unit.  Beyond that what they leave for the join costs more than shorter pieces save
// (prompts of 500 to 2000 tokens, 8 heads: 107 us with 512, 106 with 256, 185 with 768).
constexpr uint32_t kAttendPieces = 1280, kAttendPiecesLong = 512, kAttendTilePieces = 256;
struct AttendPlan {
    uint32_t pieces, grid, slots, tiles, tile_shift, min_blocks;
    bool few, wide, two;                                 // k_attend_few; k_attend_tile; that with two tiles of 32 rows per wavefront
    uint64_t off_s, off_dir, bytes;
};
bool plan_attend(comet_cache_shape s, uint32_t n_seqs, uint32_t n_tokens, uint32_t q_heads, AttendPlan *p) {
    if (!valid_shape(s) || !q_heads || q_heads > kMaxQueryHeads || q_heads % s.heads || n_seqs > kMaxSeqs) return false;
    const uint64_t rows = (uint64_t)n_tokens * (q_heads / s.heads);
    if (rows > kMaxRows) return false;
    p->wide = rows > 64ull * n_seqs;
    // Tiles of 256 rows for heads of up to 64, of 128 for those beyond 128 (what fits the registers); between, 256 rows once prompts are long:
    // 8 x 4 heads of 128, prompts of 500 to 2000 tokens 126 us (128 rows: 106), 4096 tokens behind 28672 2.14 ms (2.32).
    p->two = s.dim <= 64u || (s.dim <= 128u && n_tokens / 4096u >= n_seqs);
    p->few = rows <= 16ull * n_seqs;
    p->tile_shift = p->few ? 4u : !p->wide ? 5u : p->two ? 8u : 7u;
    p->tiles = (uint32_t)(rows >> p->tile_shift) + n_seqs;
    const bool lone = (uint64_t)p->tiles * s.heads < 128u;
    const uint32_t pieces = !p->wide ? (lone ? kAttendPiecesLong : kAttendPieces)
                                     : kAttendTilePieces * (tile_pairs((int)s.dim / 32, p->two ? 2 : 1) ? 2u : 1u);
    p->pieces = (pieces + s.heads - 1u) / s.heads;
    p->min_blocks = p->wide ? 16u : lone ? 4u : 2048u / s.dim;
    // A tile's pieces are counted as if it saw all of its sequence: of tiles of a causal prompt up to half have nothing to do.  Tiles that are cut
    // have more than total / pieces blocks, so there are at most `pieces` of them (twice that), each with one piece more than its share.
    const uint64_t most = (p->wide ? 2u : 1u) * (uint64_t)p->pieces, grid = (most + p->tiles) * s.heads, n = (uint64_t)(2u * most) * s.heads, per = 1ull << p->tile_shift;
    if (grid > kMaxGroups) return false;
    p->grid = (uint32_t)grid;
    p->slots = (uint32_t)(2u * most);
    p->off_s = n * per * s.dim * 4u;
    p->off_dir = p->off_s + n * per * 3u * 4u;
    p->bytes = p->off_dir + 8ull * (p->tiles + 1ull);
    return true;
}

template <int NC>
void launch_attend(const AttendArgs &a, const AttendPlan &p, uint32_t wg, hipStream_t st) {
    if constexpr (NC <= 4)
        if (p.wide && p.two) {
            k_attend_tile<NC, 2><<<wg, kAttendBlock, 0, st>>>(a);
            return;
        }
    if constexpr (NC > 2)
        if (p.wide) {
            k_attend_tile<NC, 1><<<wg, kAttendBlock, 0, st>>>(a);
            return;
        }
    if (p.few && a.bf16) k_attend_few<NC, false><<<wg, kAttendBlock, 0, st>>>(a);
    else if (p.few) k_attend_few<NC, true><<<wg, kAttendBlock, 0, st>>>(a);
    else if (a.bf16) k_attend<NC, false><<<wg, kAttendBlock, 0, st>>>(a);
    else k_attend<NC, true><<<wg, kAttendBlock, 0, st>>>(a);
}

}  // namespace

extern "C" {

int comet_rope_steps(const comet_rope_cfg *cfg, uint64_t *host_steps, float *amp) {
    if (!cfg || !host_steps || !amp) return COMET_ERR_INVALID;
    const comet_rope_cfg c = *cfg;
    if (c.rot < 2u || c.rot % 2u || c.rot > kMaxRopeDim || c.scaling > COMET_ROPE_PARTS || !std::isfinite(c.base) || !(c.base > 1.0) ||
        !std::isfinite(c.factor) || !(c.factor >= 1.0)) return COMET_ERR_INVALID;
    if (c.scaling == COMET_ROPE_PARTS && (!std::isfinite(c.original_len) || !(c.original_len > 0.0) || !std::isfinite(c.beta_fast) ||
        !(c.beta_slow >= 0.0) || !(c.beta_fast > c.beta_slow))) return COMET_ERR_INVALID;
    const long double two_pi = 6.283185307179586476925286766559005768L;
    long double base = c.base;
    const long double factor = c.factor;
    if (c.scaling == COMET_ROPE_BASE) base *= c.rot > 2u ? powl(factor, (long double)c.rot / (c.rot - 2u)) : factor;
    for (uint32_t i = 0; i < c.rot / 2u; ++i) {
        long double f = powl(base, -2.0L * i / c.rot);
        if (c.scaling == COMET_ROPE_LINEAR) f /= factor;
        if (c.scaling == COMET_ROPE_PARTS) {
            const long double turns = c.original_len * f / two_pi;
            long double keep = (turns - c.beta_slow) / ((long double)c.beta_fast - c.beta_slow);
            keep = keep < 0.0L ? 0.0L : (keep > 1.0L ? 1.0L : keep);
            f *= keep + (1.0L - keep) / factor;
        }
        host_steps[i] = (uint64_t)roundl(f / two_pi * 0x1p64L);                  // f <= 1 radian: less than a sixth of a turn
    }
    *amp = c.scaling == COMET_ROPE_PARTS ? (float)(0.1 * std::log(c.factor) + 1.0) : 1.0f;
    return COMET_OK;
}

int comet_rope(const comet_rope_plan *plan, comet_rows x, comet_rows y, uint32_t n_tokens, uint32_t heads, uint32_t dim, int dtype,
               const int32_t *dev_positions, int backward, void *stream) {
    RopeArgs r;
    Rows rx, ry;
    if (!plan || dtype < COMET_F32 || dtype > COMET_BF16 || !heads || heads > kMaxQueryHeads || dim > kMaxRopeDim || n_tokens > kMaxRows ||
        !rope_args(plan, dim, dev_positions, &r)) return COMET_ERR_INVALID;
    if (!n_tokens) return COMET_OK;
    if (!rows_args(x, dtype, &rx) || !out_args(y, dtype, n_tokens, heads, dim, &ry)) return COMET_ERR_INVALID;
    const bool in_place = x.dev == y.dev;
    if (!same_or_apart(rx, ry, heads, n_tokens, dim, dtype)) return COMET_ERR_INVALID;
    const uint32_t v = 16u / elem_size(dtype);
    const bool vec = r.rot % (2u * v) == 0u && (dim - r.rot) % v == 0u && rows_aligned(rx, dtype) && rows_aligned(ry, dtype);
    const uint32_t sign = backward ? 0x80000000u : 0u;
    hipStream_t st = (hipStream_t)stream;
    if (dtype == COMET_F32) {
        if (vec) launch_rope<float, 4>(r, rx, ry, n_tokens, heads, dim, in_place, sign, st);
        else launch_rope<float, 1>(r, rx, ry, n_tokens, heads, dim, in_place, sign, st);
    } else if (dtype == COMET_F16) {
        if (vec) launch_rope<_Float16, 8>(r, rx, ry, n_tokens, heads, dim, in_place, sign, st);
        else launch_rope<_Float16, 1>(r, rx, ry, n_tokens, heads, dim, in_place, sign, st);
    } else {
        if (vec) launch_rope<__bf16, 8>(r, rx, ry, n_tokens, heads, dim, in_place, sign, st);
        else launch_rope<__bf16, 1>(r, rx, ry, n_tokens, heads, dim, in_place, sign, st);
    }
    HIP_TRY(hipGetLastError());
    return COMET_OK;
}

uint64_t comet_cache_bytes(comet_cache_shape s) {
    uint64_t n;
    if (!valid_shape(s) || !count_blocks(s, &n)) return 0;
    return n * 64u * s.dim + pad256(n * 8u) + (uint64_t)s.n_slots * s.heads * 2u * ring_half_bytes(s.dim);
}

int comet_cache_append(void *dev_cache, comet_cache_shape shape, const comet_cache_batch *batch, uint32_t n_tokens, comet_rows k, comet_rows v,
                       comet_rows q, comet_rows q_out, uint32_t q_heads, int dtype, const comet_rope_plan *plan,
                       const int32_t *dev_positions, void *stream, int32_t *dev_status) {
    AppendArgs a{};
    if ((dtype != COMET_F16 && dtype != COMET_BF16) || q_heads > kMaxQueryHeads || !cache_args(dev_cache, shape, &a.c) ||
        !batch_args(batch, n_tokens, dev_status, &a.b) || !rope_args(plan, shape.dim, dev_positions, &a.rope)) return COMET_ERR_INVALID;
    if (!n_tokens) return COMET_OK;
    if (!rows_args(k, dtype, &a.k) || !rows_args(v, dtype, &a.v)) return COMET_ERR_INVALID;
    a.vec = rows_aligned(a.k, dtype) && rows_aligned(a.v, dtype) && a.rope.rot % 16u == 0u;
    a.q_heads = q_heads;
    uint32_t q_wg = 0;
    if (q_heads) {
        if (!rows_args(q, dtype, &a.q) || !out_args(q_out, dtype, n_tokens, q_heads, shape.dim, &a.q_out)) return COMET_ERR_INVALID;
        if (!same_or_apart(a.q, a.q_out, q_heads, n_tokens, shape.dim, dtype) || !rows_apart(a.k, shape.heads, a.q_out, q_heads, n_tokens, shape.dim, dtype) ||
            !rows_apart(a.v, shape.heads, a.q_out, q_heads, n_tokens, shape.dim, dtype)) return COMET_ERR_INVALID;
        a.vec = a.vec && rows_aligned(a.q, dtype) && rows_aligned(a.q_out, dtype);
        a.q_heads_wg = 8u;
        q_wg = (q_heads + a.q_heads_wg - 1u) / a.q_heads_wg;
    }
    const dim3 grid(block_units(a.b), shape.heads + q_wg);
    hipStream_t st = (hipStream_t)stream;
    if (dtype == COMET_F16) k_cache_append<_Float16><<<grid, kCacheBlock, cache_lds(shape.dim), st>>>(a);
    else k_cache_append<__bf16><<<grid, kCacheBlock, cache_lds(shape.dim), st>>>(a);
    HIP_TRY(hipGetLastError());
    return COMET_OK;
}

int comet_cache_fetch(const void *dev_cache, comet_cache_shape shape, const comet_cache_batch *batch, uint32_t n_tokens, comet_rows k, comet_rows v,
                      int dtype, void *stream, int32_t *dev_status) {
    FetchArgs a{};
    if ((dtype != COMET_F16 && dtype != COMET_BF16) || !cache_args(dev_cache, shape, &a.c) || !batch_args(batch, n_tokens, dev_status, &a.b))
        return COMET_ERR_INVALID;
    if (!n_tokens) return COMET_OK;
    if (!out_args(k, dtype, n_tokens, shape.heads, shape.dim, &a.k) || !out_args(v, dtype, n_tokens, shape.heads, shape.dim, &a.v) ||
        !rows_apart(a.k, shape.heads, a.v, shape.heads, n_tokens, shape.dim, dtype)) return COMET_ERR_INVALID;
    a.vec = rows_aligned(a.k, dtype) && rows_aligned(a.v, dtype);
    const dim3 grid(block_units(a.b), shape.heads);
    hipStream_t st = (hipStream_t)stream;
    if (dtype == COMET_F16) k_cache_fetch<_Float16><<<grid, kCacheBlock, cache_lds(shape.dim), st>>>(a);
    else k_cache_fetch<__bf16><<<grid, kCacheBlock, cache_lds(shape.dim), st>>>(a);
    HIP_TRY(hipGetLastError());
    return COMET_OK;
}

uint64_t comet_cache_attend_work(comet_cache_shape shape, uint32_t n_seqs, uint32_t n_tokens, uint32_t q_heads) {
    AttendPlan p;
    return plan_attend(shape, n_seqs, n_tokens, q_heads, &p) ? p.bytes : 0;
}

int comet_cache_attend(const void *dev_cache, comet_cache_shape shape, const comet_cache_batch *batch, uint32_t n_tokens, comet_rows q, uint32_t q_heads,
                       int dtype, float scale, int causal, comet_rows out, float *dev_lse, void *dev_work, uint64_t work_bytes,
                       void *stream, int32_t *dev_status) {
    AttendArgs a{};
    AttendPlan p;
    if ((dtype != COMET_F16 && dtype != COMET_BF16) || !cache_args(dev_cache, shape, &a.c) || !batch_args(batch, n_tokens, dev_status, &a.b) ||
        !std::isfinite(scale * 1.4426950408889634f) || scale < 0.0f || (uintptr_t)dev_lse % 4u || !plan_attend(shape, batch->n_seqs, n_tokens, q_heads, &p))
        return COMET_ERR_INVALID;
    if (!n_tokens) return COMET_OK;
    if (!rows_args(q, dtype, &a.q) || !out_args(out, dtype, n_tokens, q_heads, shape.dim, &a.out) ||
        !rows_apart(a.q, q_heads, a.out, q_heads, n_tokens, shape.dim, dtype) || !dev_work || (uintptr_t)dev_work % 16u) return COMET_ERR_INVALID;
    if (work_bytes < p.bytes) return COMET_ERR_NOMEM;
    a.lse = dev_lse; a.q_heads = q_heads; a.group = q_heads / shape.heads;
    a.bf16 = dtype == COMET_BF16; a.causal = causal != 0; a.wide = p.wide; a.vec = rows_aligned(a.q, dtype) && rows_aligned(a.out, dtype);
    a.pieces = p.pieces; a.slots = p.slots; a.min_blocks = p.min_blocks; a.tile_shift = p.tile_shift; a.tile_rows = 1u << p.tile_shift;
    a.scale = scale * 1.4426950408889634f;
    uint8_t *w = static_cast<uint8_t *>(dev_work);
    a.part_o = reinterpret_cast<float *>(w);
    a.part_s = reinterpret_cast<float *>(w + p.off_s);
    a.directory = reinterpret_cast<int32_t *>(w + p.off_dir);
    hipStream_t st = (hipStream_t)stream;
    const uint32_t wg = p.grid;
    switch (shape.dim / 32u) {
        case 1: launch_attend<1>(a, p, wg, st); break;
        case 2: launch_attend<2>(a, p, wg, st); break;
        case 3: launch_attend<3>(a, p, wg, st); break;
        case 4: launch_attend<4>(a, p, wg, st); break;
        case 5: launch_attend<5>(a, p, wg, st); break;
        case 6: launch_attend<6>(a, p, wg, st); break;
        case 7: launch_attend<7>(a, p, wg, st); break;
        default: launch_attend<8>(a, p, wg, st); break;
    }
    HIP_TRY(hipGetLastError());
    // the rows of a tile side by side while there are few tiles (4096 workgroups: with 8192 the starts of those without work cost 1 to 3 us, with
    // 1024 the rows that follow one another up to 9)
    const uint32_t groups = p.tiles * shape.heads, most = p.wide ? 8u : a.tile_rows;
    uint32_t side = (p.wide ? 2048u : 4096u) / groups;
    side = side < 1u ? 1u : (side > most ? most : side);
    if (p.wide) k_attend_join_tile<<<dim3(groups, side), kAttendBlock, 0, st>>>(a);
    else k_attend_join<<<dim3(groups, side), kAttendBlock, 0, st>>>(a);
    HIP_TRY(hipGetLastError());
    return COMET_OK;
}

}  // extern "C"
