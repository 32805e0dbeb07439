// Attention of the batch's queries over the compressed cache.
//
// One pass over the keys with a reference m near the running maximum and the sum l of every row.  With q the row, K and V the whole
// numbers of a block and a, b its scales:  x = (q . K) a c,  p = exp2(x - r + log2 b + lift),  O += p V,  l += exp2(x - m),
// o = O exp2(r - m - lift) / l.  r is a second reference, near the largest x + log2 b: p, which the matrix instruction takes in float16, is
// then at most 2^15 whatever the scales of the blocks are, and weights down to 2^-21 of the largest keep all bits float16 has, down to 2^-32 some
// (a hundred thousand tokens of next to no weight still count).  m and r move only once something exceeds them by 2^8: O
// is hardly ever rescaled.  The whole numbers are exact in float16.  Two roundings are below 32 bits:
//   p, to float16: at most 2^-11 of each weight.  bf16 results are rounded to 2^-8 themselves.  For float16 results the calls of up to 64 rows multiply
//     what the rounding leaves, too; prompts (k_attend_tile) do not, where it would make three products of two: 2048 tokens behind 30720, 16 heads of
//     256 on one, come out with 1.4 times the error of a sum in 32 bits rounded once (2.9e-4 of the result's size, 2.1e-4).
//   the query in bf16, to float16 times a power of two of its row: at most 2^-39 of the row's largest value, and nothing for values down to 2^-31 of
//     that.  A query in float16 goes in as it is.
#pragma once
#include "comet_cache.h"
#include "comet_scan.h"

namespace comet {

namespace {

constexpr float kNegInf = -__builtin_inff();
constexpr float kLift = 7.0f, kSlack = 8.0f;      // log2: weights are at most 2^(kLift + kSlack) on their way into float16

// A sequence as the batch has it: tiles of a.tile_rows rows (none if its numbers make no sense, which is reported) and blocks.
struct SeqWork {
    Seq s;
    uint32_t tiles, blocks;
    __device__ void read(const AttendArgs &a, uint32_t seq) {
        const int32_t s0 = a.b.starts[seq], s1 = a.b.starts[seq + 1], len = a.b.lens[seq];
        const bool sane = s0 >= 0 && s1 >= s0 && s1 <= (int32_t)a.b.n_tokens && len >= 0 && len <= kMaxLen;
        if (!sane && a.b.status) *a.b.status = COMET_ERR_FORMAT;
        s.start = s0;
        s.n = sane ? s1 - s0 : 0;
        s.len = len;
        tiles = (uint32_t)(((uint64_t)(uint32_t)s.n * a.group + a.tile_rows - 1u) >> a.tile_shift);
        blocks = sane ? ((uint32_t)len + 31u) / 32u : 0u;
    }
    __device__ void none() { s.start = s.n = s.len = 0; tiles = blocks = 0u; }
};

__device__ inline uint32_t lane_value(uint32_t v, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, lane); }
// Sum over the wavefront, the same in every lane.
__device__ inline float wave_total(float v) {
    const auto add = [](float x, int32_t y) { return x + __int_as_float(y); };
    v = add(v, dpp0<0x111, 0xf, true>(__float_as_int(v)));
    v = add(v, dpp0<0x112, 0xf, true>(__float_as_int(v)));
    v = add(v, dpp0<0x114, 0xf, true>(__float_as_int(v)));
    v = add(v, dpp0<0x118, 0xf, true>(__float_as_int(v)));
    v = add(v, dpp0<0x142, 0xa, false>(__float_as_int(v)));
    v = add(v, dpp0<0x143, 0xc, false>(__float_as_int(v)));
    return __uint_as_float(lane_value(__float_as_uint(v), kWave - 1));
}

constexpr uint32_t kSorted = 32;                   // sequences that are put in order

struct Piece {
    uint32_t seq, tile, part;
    uint32_t per;                         // blocks of a part
    uint32_t slot;                        // among the pieces of tiles that are cut: where its results go
    Seq s;
};
// Cuts the blocks of all tiles into pieces of the same length, so that sequences of very different lengths keep all compute units
// busy, and finds the piece `number`.  Everything comes from the lengths on the device: the host does not know
// them, and a captured call goes by what they are when it is replayed.  By the whole workgroup, a sequence per thread (a second
// read for those beyond 256); ends the same way for all threads.
__device__ inline bool find_piece(const AttendArgs &a, uint32_t number, Piece *p) {
    __shared__ float s_sum[kAttendBlock / kWave];
    __shared__ uint32_t s_scan[kAttendBlock / kWave][2], s_found[7];
    __shared__ uint32_t s_order[kSorted][6];
    const uint32_t tid = threadIdx.x, wave = tid / kWave;
    float total = 0.0f;                       // blocks of all tiles; the same sum in the same order in every workgroup
    SeqWork w;
    w.none();
    for (uint32_t b = tid; b < a.b.n_seqs; b += kAttendBlock) {
        SeqWork x;
        x.read(a, b);
        float v = (float)x.blocks;
        if (a.causal && a.wide) {                              // on the average a tile sees as much as its sequence's middle one
            const float half = (float)x.s.n * (1.0f / 64.0f);
            v = fmaxf(v - half, v * 0.5f);                     // (never less than half: the grid counts on it)
        }
        total += v * (float)x.tiles;
        if (b == tid) w = x;
    }
    total = wave_total(total);
    if (lane_id() == 0) s_sum[wave] = total;
    if (tid == 0u) s_found[0] = 0xffffffffu;
    __syncthreads();
    total = (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]);
    // an eighth more than the average (a tile that is just longer than that is not worth a second piece), which also keeps what float32
    // rounds from making more pieces than the grid has
    const float most = __builtin_ceilf(total * 1.125f / (float)a.pieces);
    uint32_t per = most < 2147483000.0f ? (uint32_t)most : 2147483000u;
    if (per < a.min_blocks) per = a.min_blocks;
    // A few prompts: the longest sequences first, so that no long tile begins when the others are done.
    uint32_t whose = tid;
    const bool sorted = a.wide && a.b.n_seqs > 1u && a.b.n_seqs <= kSorted;
    if (sorted) {
        if (wave == 0u) {
            uint32_t rank = 0;
            for (uint32_t k = 0; k < a.b.n_seqs; ++k) {
                const uint32_t other = lane_value(w.blocks, (int)k);
                rank += other > w.blocks || (other == w.blocks && k < tid);
            }
            if (tid < a.b.n_seqs) {
                uint32_t *o = s_order[rank];
                o[0] = tid; o[1] = w.tiles; o[2] = w.blocks; o[3] = (uint32_t)w.s.start; o[4] = (uint32_t)w.s.n; o[5] = (uint32_t)w.s.len;
            }
        }
        __syncthreads();
        if (tid < a.b.n_seqs) {
            const uint32_t *o = s_order[tid];
            whose = o[0]; w.tiles = o[1]; w.blocks = o[2]; w.s.start = (int32_t)o[3]; w.s.n = (int32_t)o[4]; w.s.len = (int32_t)o[5];
        }
    }
    uint32_t base = 0, cut_base = 0;
    for (uint32_t b0 = 0; b0 < a.b.n_seqs && base <= number; b0 += kAttendBlock) {
        const uint32_t b = b0 + tid;
        if (b0) {
            w.none();
            if (b < a.b.n_seqs) w.read(a, b);
        }
        const uint32_t parts = w.blocks > per ? (w.blocks + per - 1u) / per : 1u, count = w.tiles * parts;
        const uint32_t cut = parts > 1u ? count : 0u;
        const uint32_t incl = (uint32_t)run_scan<2>((int32_t)count, 0u, 64u), cut_incl = (uint32_t)run_scan<2>((int32_t)cut, 0u, 64u);
        if (lane_id() == kWave - 1) {
            s_scan[wave][0] = incl;
            s_scan[wave][1] = cut_incl;
        }
        __syncthreads();
        uint32_t before = base + incl - count, cut_before = cut_base + cut_incl - cut;
#pragma unroll
        for (uint32_t k = 0; k < kAttendBlock / kWave; ++k) {
            if (k < wave) {
                before += s_scan[k][0];
                cut_before += s_scan[k][1];
            }
            base += s_scan[k][0];
            cut_base += s_scan[k][1];
        }
        if (number - before < count) {
            const uint32_t local = number - before, tile = local / parts;
            if (tile < w.tiles) {                              // (not so only where the batch's numbers make no sense)
                s_found[0] = sorted ? whose : b;
                s_found[1] = a.causal ? w.tiles - 1u - tile : tile;    // a causal prompt's last tiles see most: they begin first
                s_found[2] = local - tile * parts;
                s_found[3] = (uint32_t)w.s.start;
                s_found[4] = (uint32_t)w.s.n;
                s_found[5] = (uint32_t)w.s.len;
                s_found[6] = cut_before + local;
            }
        }
        __syncthreads();
    }
    p->seq = (uint32_t)__builtin_amdgcn_readfirstlane((int)s_found[0]);
    p->tile = (uint32_t)__builtin_amdgcn_readfirstlane((int)s_found[1]);
    p->part = (uint32_t)__builtin_amdgcn_readfirstlane((int)s_found[2]);
    p->per = (uint32_t)__builtin_amdgcn_readfirstlane((int)per);
    p->slot = (uint32_t)__builtin_amdgcn_readfirstlane((int)s_found[6]);
    p->s.start = __builtin_amdgcn_readfirstlane((int)s_found[3]);
    p->s.n = __builtin_amdgcn_readfirstlane((int)s_found[4]);
    p->s.len = __builtin_amdgcn_readfirstlane((int)s_found[5]);
    return p->seq != 0xffffffffu;             // (a sequence whose numbers make no sense has no tiles)
}

// The last sequence whose units (first_unit) begin at or before `unit`, and which of its tiles that is, by all lanes of a wavefront: 64 candidates a
// turn, once 64 are left everything about them at once.  false: none of its tiles.  Starts that do not grow give some sequence, never one out of range.
__device__ inline bool find_tile(const AttendArgs &a, uint32_t unit, SeqWork *w, uint32_t *tile) {
    uint32_t lo = 0, len = a.b.n_seqs;
    while (len > 64u) {
        const uint32_t stride = (len + 63u) / 64u, off = (uint32_t)lane_id() * stride;
        const bool le = off < len && first_unit(a.b.starts, lo + off, a.group, a.tile_shift, 1u) <= unit;
        const uint32_t n = (uint32_t)__popcll(wave_ballot(le)), k = n > 0u ? n - 1u : 0u;
        lo += k * stride;
        len = len - k * stride < stride ? len - k * stride : stride;
    }
    const uint32_t mine = (uint32_t)lane_id() < len ? lo + (uint32_t)lane_id() : lo;
    SeqWork own;
    own.read(a, mine);
    const uint32_t first = first_unit(a.b.starts, mine, a.group, a.tile_shift, 1u);
    const uint32_t n = (uint32_t)__popcll(wave_ballot((uint32_t)lane_id() < len && first <= unit));
    const int k = (int)(n > 0u ? n - 1u : 0u);
    w->tiles = lane_value(own.tiles, k);
    w->blocks = lane_value(own.blocks, k);
    w->s.start = (int32_t)lane_value((uint32_t)own.s.start, k);
    w->s.n = (int32_t)lane_value((uint32_t)own.s.n, k);
    w->s.len = (int32_t)lane_value((uint32_t)own.s.len, k);
    const uint32_t f = lane_value(first, k);
    *tile = unit - f;
    return unit >= f && *tile < w->tiles;
}

// Eight whole numbers of 8 bits as float16: a byte u = v + 128 behind the byte 0x64 is the float16 number 1024 + u.
__device__ inline half8 whole8(uint32_t lo, uint32_t hi) {
    lo ^= 0x80808080u;
    hi ^= 0x80808080u;
    const uint32_t m = 0x64646464u;
    const half2v off = {(_Float16)1152.0f, (_Float16)1152.0f};
    const half2v a = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(m, lo, 0x04010400u)) - off;
    const half2v b = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(m, lo, 0x04030402u)) - off;
    const half2v c = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(m, hi, 0x04010400u)) - off;
    const half2v d = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(m, hi, 0x04030402u)) - off;
    return half8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Largest value and sum over the lanes of a row: l and l ^ 32, for tiles of 16 rows those that differ by a multiple of 16.
template <int ROWS>
__device__ inline float row_max(float v) {
    if constexpr (ROWS == 16) {
        const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
    }
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
template <int ROWS>
__device__ inline float row_sum(float v) {
    if constexpr (ROWS == 16) {
        const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}
__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ inline float log2_fast(float x) { return __builtin_amdgcn_logf(x); }

// Tiles of 32 or of 16 rows.  Which of a block's tokens lane l's score t is of, and where its values of the head are (ROWS registers of
// 32 * 32 or 16 * 16 results): as the matrix instruction leaves them.
template <int ROWS> constexpr int kScores = ROWS / 2;                    // scores of a lane per block
template <int ROWS> __device__ inline uint32_t token_of(int t) {
    if (ROWS == 32) return 8u * (t / 4) + 4u * ((uint32_t)lane_id() >> 5) + t % 4;
    return 16u * (t / 4) + 4u * ((uint32_t)lane_id() >> 4) + t % 4;
}

// What rounding a weight to float16 leaves, in float16 once more.
__device__ inline _Float16 rest_of(float w, _Float16 p) { return (_Float16)(w - (float)p); }

// A row's numbers, in the lanes l with l % ROWS its number in the tile.
template <int NO, typename ACC, int ROWS>
struct RowState {
    static constexpr int N = kScores<ROWS>;
    ACC o[NO];
    float m, r, l;              // l: of the lane's own tokens until the end
    __device__ void clear() {
#pragma unroll
        for (int c = 0; c < NO; ++c) o[c] = ACC{};
        m = r = kNegInf;
        l = 0.0f;
    }
    // top: the largest x of the row's new tokens, tope: of x + log2 b
    __device__ void follow(float top, float tope) {
        if (wave_ballot(top > m + kSlack || tope > r + kSlack || (m == kNegInf && top > kNegInf))) {
            const float m2 = fmaxf(m, top), r2 = fmaxf(r, tope);
            const float alpha = exp2_fast(r - (r2 == kNegInf ? 0.0f : r2));
            l *= exp2_fast(m - (m2 == kNegInf ? 0.0f : m2));
#pragma unroll
            for (int c = 0; c < NO; ++c) o[c] *= alpha;
            m = m2;
            r = r2;
        }
    }
    // The weights of a block that the whole tile sees, from its raw products; kc = a c, lb = log2 b.
    template <typename S>
    __device__ void weights(const S &s, float kc, float lb, half8 *p, half8 *rest = nullptr) {
        // where b is so small that p is 0 anyway, only l counts
        const float c1 = fmaxf(lb - r + kLift, -60.0f - m);
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int t = 0; t < N; ++t) {
            const float w = exp2_fast(__builtin_fmaf(s[t], kc, c1));
            sum[t % 4] += w;
            p[t / 8][t % 8] = (_Float16)w;
            if (rest) rest[t / 8][t % 8] = rest_of(w, (_Float16)w);
        }
        l = __builtin_fmaf((sum[0] + sum[1]) + (sum[2] + sum[3]), exp2_fast(-c1 - m), l);
    }
    // The same for a block of which rows see parts: x = -Inf elsewhere.  A poisoned block's lb is NaN, and so are the weights seen.
    __device__ void weights_some(const float *x, float lb, half8 *p, half8 *rest = nullptr) {
        const float ms = m == kNegInf ? 0.0f : m, c1 = lb - (r == kNegInf ? 0.0f : r) + kLift;
        float sum = 0.0f;
#pragma unroll
        for (int t = 0; t < N; ++t) {
            const float w = exp2_fast(x[t] + c1);
            sum += exp2_fast(x[t] - ms);
            p[t / 8][t % 8] = (_Float16)w;
            if (rest) rest[t / 8][t % 8] = rest_of(w, (_Float16)w);
        }
        l += sum;
        if (lb != lb) {
#pragma unroll
            for (int t = 0; t < N; ++t)
                if (x[t] == kNegInf) {
                    p[t / 8][t % 8] = (_Float16)0.0f;
                    if (rest) rest[t / 8][t % 8] = (_Float16)0.0f;
                }
        }
    }
    // ... and for tokens each with a scale of its own: lv = log2 b, 0 where x = -Inf.
    __device__ void weights_each(const float *x, const float *lv, half8 *p, half8 *rest = nullptr) {
        const float ms = m == kNegInf ? 0.0f : m, rs = r == kNegInf ? 0.0f : r;
#pragma unroll
        for (int t = 0; t < N; ++t) {
            const float w = exp2_fast(x[t] + (lv[t] - rs + kLift));
            l += exp2_fast(x[t] - ms);
            p[t / 8][t % 8] = (_Float16)w;
            if (rest) rest[t / 8][t % 8] = rest_of(w, (_Float16)w);
        }
    }
};

// What a row is: the query, where its values are and go, how many tokens it sees.
struct RowPlace {
    bool real;
    uint32_t qh;
    int64_t token;
    int32_t limit;
};
__device__ inline RowPlace row_place(const AttendArgs &a, const Seq &s, uint32_t head, uint32_t row) {
    RowPlace p;
    const uint32_t rows = (uint32_t)s.n * a.group;
    p.real = row < rows;
    const uint32_t query = p.real ? row / a.group : (uint32_t)s.n - 1u;
    p.qh = head * a.group + (p.real ? row - query * a.group : 0u);
    p.token = (int64_t)s.start + query;
    p.limit = a.causal ? s.len - s.n + (int32_t)query + 1 : s.len;
    return p;
}
// tokens seen by the first and by the last of the rows row0 .. row0 + count - 1 (those that there are)
__device__ inline void row_limits(const AttendArgs &a, const Seq &s, uint32_t row0, uint32_t count, int32_t *least, int32_t *most) {
    const uint32_t rows = (uint32_t)s.n * a.group, last = row0 + count - 1u < rows ? row0 + count - 1u : rows - 1u;
    *least = a.causal ? s.len - s.n + (int32_t)((row0 < rows ? row0 : rows - 1u) / a.group) + 1 : s.len;
    *most = a.causal ? s.len - s.n + (int32_t)(last / a.group) + 1 : s.len;
}

// The row's query as the right operand: float16 times a power of two, which is returned.  Requested first, so that other loads can follow
// before it is waited for.
template <int NW>
struct QueryRaw { uint32_t w[NW]; };             // pairs of 16-bit values, in the order of the operand
// COUNT values from every 32nd of the head on, `at` of them behind it.
template <int NC, int COUNT>
__device__ inline void request_query(const AttendArgs &a, const RowPlace &p, uint32_t at, QueryRaw<NC * COUNT / 2> *raw) {
    const uint16_t *src = reinterpret_cast<const uint16_t *>(a.q.p) + p.token * a.q.token + (int64_t)p.qh * a.q.head + at;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        if (a.vec) {
#pragma unroll
            for (int k = 0; k < COUNT / 8; ++k) {
                const u32x4 x = *reinterpret_cast<const u32x4 *>(src + c * 32 + 8 * k);
#pragma unroll
                for (int i = 0; i < 4; ++i) raw->w[c * COUNT / 2 + 4 * k + i] = x[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < COUNT / 2; ++i) raw->w[c * COUNT / 2 + i] = src[c * 32 + 2 * i] | (uint32_t)src[c * 32 + 2 * i + 1] << 16;
        }
    }
}
template <int ROWS, int NW>
__device__ inline float convert_query(const AttendArgs &a, const QueryRaw<NW> &raw, half8 *q) {
    if (!a.bf16) {
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            const half2v two = __builtin_bit_cast(half2v, raw.w[i]);
            q[i / 4][2 * (i % 4)] = two[0];
            q[i / 4][2 * (i % 4) + 1] = two[1];
        }
        return 1.0f;
    }
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < NW; ++i)
        top = fmaxf(top, fmaxf(fabsf(__uint_as_float(raw.w[i] << 16)), fabsf(__uint_as_float(raw.w[i] & 0xffff0000u))));
    top = row_max<ROWS>(top);
    uint32_t e = __float_as_uint(top) >> 23;
    e = e < 15u ? 15u : e;
    const float scale = __uint_as_float((e - 14u) << 23);              // 2^(exponent - 14): the largest comes to lie in [2^14, 2^15)
    const float inv = __uint_as_float((268u - e) << 23);               // 1 / scale (Inf in a row leaves Inf or NaN in it either way)
#pragma unroll
    for (int i = 0; i < NW; ++i) {
        q[i / 4][2 * (i % 4)] = (_Float16)(__uint_as_float(raw.w[i] << 16) * inv);
        q[i / 4][2 * (i % 4) + 1] = (_Float16)(__uint_as_float(raw.w[i] & 0xffff0000u) * inv);
    }
    return scale;
}

// Where a block lies and its scales: looked up by the lanes of a wavefront, one block each.  request() waits for the pages alone, so that what
// lies at the index can be loaded beside the scales, which finish() waits for.
struct Lookup {
    int64_t index;              // or -1: no such page
    float ks, lb;               // scale of the keys, log2 of the values'
    __device__ void request(const AttendArgs &a, uint32_t seq, uint32_t head, uint32_t j, uint32_t end) {
        const uint32_t col = j / a.c.per;
        const bool asked = j < end, listed = asked && col < a.b.width;
        const int32_t page = a.b.table[listed ? (uint64_t)seq * a.b.width + col : 0u];
        const bool there = listed && page >= 0 && (uint32_t)page < a.c.n_pages;
        index = there ? ((int64_t)page * a.c.heads + head) * a.c.per + (j - col * a.c.per) : -1;
        if (asked && !there && a.b.status) *a.b.status = COMET_ERR_FORMAT;
        const float *s = a.c.scales + (there ? 2 * index : 0);
        ks = s[0];
        lb = s[1];
    }
    // Where there is no page the scales read are another block's, of which anything can be left, Inf among it: the block is not seen, and an
    // ordinary scale keeps what is computed for it 0.
    __device__ void finish() {
        ks = index < 0 ? 0.0f : ks;
        lb = index < 0 ? 0.0f : log2_fast(lb);
    }
    __device__ void get(const AttendArgs &a, uint32_t seq, uint32_t head, uint32_t j, uint32_t end) {
        request(a, seq, head, j, end);
        finish();
    }
    __device__ int64_t index_of(uint32_t i) const {
        const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(uint64_t)index, (int)i);
        const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)((uint64_t)index >> 32), (int)i);
        return (int64_t)((uint64_t)hi << 32 | lo);
    }
    __device__ static float of(float v, uint32_t i) { return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), (int)i)); }
};

// x of a block's tokens from its raw products: visible are those before `limit`.
template <int ROWS, typename S>
__device__ inline void some_of_block(const S &s, float kc, float lb, uint32_t j, int32_t limit, float *x, float *top, float *tope) {
    const int32_t left = limit - (int32_t)(j * 32u) - (int32_t)token_of<ROWS>(0);
    float best = kNegInf;
#pragma unroll
    for (int t = 0; t < kScores<ROWS>; ++t) {
        const float v = s[t] * kc;
        x[t] = (ROWS == 32 ? 8 : 16) * (t / 4) + t % 4 < left ? v : kNegInf;
        best = fmaxf(best, x[t]);
    }
    *top = row_max<ROWS>(best);
    *tope = *top + lb;                        // (NaN for a poisoned block: no reference follows it)
}
// x and lv (weights_each) of the open block's tokens, with their own scales; `held` of its tokens are there.
template <int ROWS, typename S>
__device__ inline void each_of_open(const S &s, float qc, const float *ke, uint32_t held, uint32_t j, int32_t limit, float *x, float *lv, float *top, float *tope) {
    float best = kNegInf, bests = kNegInf;
#pragma unroll
    for (int t = 0; t < kScores<ROWS>; ++t) {
        const uint32_t tok = token_of<ROWS>(t);
        const bool see = tok < held && (int32_t)(j * 32u + tok) < limit;
        const float kt = ke[tok], vt = ke[32u + tok];
        x[t] = see ? s[t] * (kt * qc) : kNegInf;
        lv[t] = !see ? 0.0f : vt == vt ? (float)((int)(__float_as_uint(vt) >> 23) - 127) : vt;      // a power of two
        best = fmaxf(best, x[t]);
        bests = fmaxf(bests, x[t] + lv[t]);
    }
    *top = row_max<ROWS>(best);
    *tope = row_max<ROWS>(bests);
}
// The open block's values as an operand: places nobody has written yet may hold anything.
__device__ inline half8 open_values(const uint8_t *at, uint32_t u, uint32_t held) {
    const uint32_t h = (uint32_t)lane_id() >> 5;
    half8 v = *reinterpret_cast<const half8 *>(at);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (16u * u + 8u * (i / 4) + 4u * h + i % 4 >= held) v[i] = (_Float16)0.0f;
    return v;
}
__device__ inline float log_sum(float m, float l) {                     // natural logarithm of l 2^m
    return l > 0.0f ? (m + __log2f(l)) * 0.6931471805599453f : (l == l ? kNegInf : l);
}
__device__ inline f32x16 mfma(half8 a, half8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ inline f32x4 mfma(half8 a, half8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ inline void store_out(const AttendArgs &a, const RowPlace &p, uint32_t d, f32x4 v) {
    uint16_t *dst = reinterpret_cast<uint16_t *>(a.out.p) + p.token * a.out.token + (int64_t)p.qh * a.out.head + d;
    uint16_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = a.bf16 ? __builtin_bit_cast(uint16_t, (__bf16)v[i]) : __builtin_bit_cast(uint16_t, (_Float16)v[i]);
    if (a.vec) {
        *reinterpret_cast<uint2 *>(dst) = uint2{w[0] | (uint32_t)w[1] << 16, w[2] | (uint32_t)w[3] << 16};
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) dst[i] = w[i];
    }
}
// Parts of a tile that have something to do.
__device__ inline uint32_t parts_of(uint32_t seen, uint32_t per) { return seen > per ? (seen + per - 1u) / per : 1u; }

}  // namespace

}  // namespace comet
