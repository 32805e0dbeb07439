// Attention of the batch's queries over the compressed cache.
//
// One pass over the keys with a reference m near the running maximum and the sum l of every row.  With q the row, K and V the whole
// numbers of a block and a, b its scales:  x = (q . K) a c,  p = exp2(x - r + log2 b + lift),  O += p V,  l += exp2(x - m),
// o = O exp2(r - m - lift) / l.  r is a second reference, near the largest x + log2 b: p, which the matrix instruction takes in float16, is
// then at most 2^15 whatever the scales of the blocks are, and weights down to 2^-21 of the largest keep all bits float16 has, down to 2^-32 some
// (a hundred thousand tokens of next to no weight still count).  m and r move only once something exceeds them by 2^8: O
// is hardly ever rescaled.  The whole numbers are exact in float16, so the only rounding below 32 bits is that of p, at most
// 2^-11 of each weight.  The query goes in as float16 times a power of two of its row, which is exact for both 16-bit types but for
// values below 2^-38 of the row's largest.
#include "comet_cache.h"

namespace comet {

namespace {

constexpr float kNegInf = -__builtin_inff();
constexpr float kLift = 7.0f, kSlack = 8.0f;      // log2: weights are at most 2^(kLift + kSlack) on their way into float16

// Tiles of a.tile_rows rows and blocks of a sequence.
__device__ inline uint32_t tiles_of(const AttendArgs &a, uint32_t seq) {
    const int32_t s0 = a.b.starts[seq], s1 = a.b.starts[seq + 1];
    if (s0 < 0 || s1 <= s0 || s1 > (int32_t)a.b.n_tokens || a.b.lens[seq] < 0 || a.b.lens[seq] > kMaxLen) return 0u;
    return (uint32_t)(((uint64_t)(uint32_t)(s1 - s0) * a.group + a.tile_rows - 1u) >> a.tile_shift);
}
__device__ inline uint32_t blocks_of(const AttendArgs &a, uint32_t seq) { return (uint32_t)((a.b.lens[seq] + 31ll) / 32); }

struct Piece {
    uint32_t seq, tile, part;
    uint32_t per;                         // blocks of a part
    uint32_t number;                      // among all pieces of a head
};
// Cuts the blocks of all tiles into pieces of the same length, so that sequences of very different lengths keep all compute units
// busy, and finds the piece `number`.  Everything comes from the lengths on the device: the host does not know
// them, and a captured call goes by what they are when it is replayed.  All lanes of a wavefront.
__device__ inline bool find_piece(const AttendArgs &a, uint32_t number, Piece *p) {
    uint64_t total = 0;
    for (uint32_t b0 = 0; b0 < a.b.n_seqs; b0 += kWave) {
        const uint32_t b = b0 + (uint32_t)lane_id();
        uint64_t v = 0;
        if (b < a.b.n_seqs) {
            v = blocks_of(a, b);
            const uint64_t tiles = tiles_of(a, b);
            if (a.causal && a.wide && tiles) {                 // on the average a tile sees as much as its sequence's middle one
                const uint64_t half = (uint64_t)(uint32_t)(a.b.starts[b + 1] - a.b.starts[b]) / 64u;
                v = v > 2u * half ? v - half : (v + 1u) / 2u;  // (never less than half: a.slots counts on it)
            }
            v *= tiles;
        }
        total += wave_sum<uint64_t>(v);
    }
    uint64_t per64 = (total + a.pieces - 1u) / a.pieces;
    if (per64 < a.min_blocks) per64 = a.min_blocks;
    const uint32_t per = per64 > 0x7fffffffull ? 0x7fffffffu : (uint32_t)per64;
    uint32_t base = 0;
    for (uint32_t b0 = 0; b0 < a.b.n_seqs; b0 += kWave) {
        const uint32_t b = b0 + (uint32_t)lane_id();
        uint32_t tiles = 0, parts = 0;
        if (b < a.b.n_seqs) {
            tiles = tiles_of(a, b);
            parts = (blocks_of(a, b) + per - 1u) / per;
            if (parts < 1u) parts = 1u;
        }
        const uint32_t incl = wave_incl_scan<uint32_t>(tiles * parts);
        const uint64_t here = wave_ballot(base + incl > number);
        if (here) {
            const int l = __ffsll((unsigned long long)here) - 1;
            const uint32_t t = (uint32_t)__shfl((int)tiles, l, kWave), k = (uint32_t)__shfl((int)parts, l, kWave);
            const uint32_t local = number - (base + (uint32_t)__shfl((int)incl, l, kWave) - t * k);
            p->seq = (uint32_t)__builtin_amdgcn_readfirstlane((int)(b0 + (uint32_t)l));
            p->tile = (uint32_t)__builtin_amdgcn_readfirstlane((int)(local / k));
            p->part = (uint32_t)__builtin_amdgcn_readfirstlane((int)(local % k));
            p->per = per;
            p->number = number;
            return p->tile < t;                  // (not so only where the batch's numbers make no sense)
        }
        base += (uint32_t)__shfl((int)incl, kWave - 1, kWave);
    }
    return false;
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

// The other half of the wavefront's value for the same row.
__device__ inline float other_half(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(lane_id() < 32 ? r[1] : r[0]);
}
__device__ inline float other_half_max(float v) { return fmaxf(v, other_half(v)); }
__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ inline float log2_fast(float x) { return __builtin_amdgcn_logf(x); }

// A row's numbers: lane l has those of row l & 31, the accumulated values 32c + 8 * (i / 4) + 4 * (l >> 5) + i % 4 of it.
template <int NC>
struct RowState {
    f32x16 o[NC];
    float m, r, l;              // l: of the lane's own tokens until the end
    __device__ void clear() {
#pragma unroll
        for (int c = 0; c < NC; ++c) o[c] = f32x16{};
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
            for (int c = 0; c < NC; ++c) o[c] *= alpha;
            m = m2;
            r = r2;
        }
    }
    // The weights of a block that the whole tile sees, from its raw products; kc = a c, lb = log2 b.
    __device__ void weights(const f32x16 &s, float kc, float lb, half8 *p) {
        // where b is so small that p is 0 anyway, only l counts
        const float c1 = fmaxf(lb - r + kLift, -60.0f - m);
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int t = 0; t < 16; ++t) {
            const float w = exp2_fast(__builtin_fmaf(s[t], kc, c1));
            sum[t % 4] += w;
            p[t / 8][t % 8] = (_Float16)w;
        }
        l = __builtin_fmaf((sum[0] + sum[1]) + (sum[2] + sum[3]), exp2_fast(-c1 - m), l);
    }
    // The same for tokens each with a scale of its own and for rows that do not see all of them: x = -Inf and lv = 0 there.
    __device__ void weights_each(const float *x, const float *lv, half8 *p) {
        const float ms = m == kNegInf ? 0.0f : m, rs = r == kNegInf ? 0.0f : r;
#pragma unroll
        for (int t = 0; t < 16; ++t) {
            l += exp2_fast(x[t] - ms);
            p[t / 8][t % 8] = (_Float16)exp2_fast(x[t] + (lv[t] - rs + kLift));
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

// The row's query as the right operand: float16 times a power of two, which is returned.
template <int NC>
__device__ inline float load_query(const AttendArgs &a, const RowPlace &p, half8 *q) {
    const uint32_t h = (uint32_t)lane_id() >> 5;
    const uint16_t *src = reinterpret_cast<const uint16_t *>(a.q.p) + p.token * a.q.token + (int64_t)p.qh * a.q.head;
    uint32_t raw[NC][8];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const uint16_t *at = src + c * 32 + h * 16;
        if (a.vec) {
            const u32x4 x = *reinterpret_cast<const u32x4 *>(at), y = *reinterpret_cast<const u32x4 *>(at + 8);
#pragma unroll
            for (int i = 0; i < 4; ++i) { raw[c][i] = x[i]; raw[c][4 + i] = y[i]; }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) raw[c][i] = at[2 * i] | (uint32_t)at[2 * i + 1] << 16;
        }
    }
    if (!a.bf16) {
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const half2v two = __builtin_bit_cast(half2v, raw[c][i]);
                q[2 * c + i / 4][2 * (i % 4)] = two[0];
                q[2 * c + i / 4][2 * (i % 4) + 1] = two[1];
            }
        return 1.0f;
    }
    float top = 0.0f;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            top = fmaxf(top, fmaxf(fabsf(__uint_as_float(raw[c][i] << 16)), fabsf(__uint_as_float(raw[c][i] & 0xffff0000u))));
    top = other_half_max(top);
    uint32_t e = __float_as_uint(top) >> 23;
    e = e < 15u ? 15u : e;
    const float scale = __uint_as_float((e - 14u) << 23);              // 2^(exponent - 14): the largest comes to lie in [2^14, 2^15)
    const float inv = 1.0f / scale;                                    // exact (Inf in a row leaves Inf or NaN in it either way)
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            q[2 * c + i / 4][2 * (i % 4)] = (_Float16)(__uint_as_float(raw[c][i] << 16) * inv);
            q[2 * c + i / 4][2 * (i % 4) + 1] = (_Float16)(__uint_as_float(raw[c][i] & 0xffff0000u) * inv);
        }
    return scale;
}

// Where a block lies and its scales: looked up by the lanes of a wavefront, one block each.
struct Lookup {
    int64_t index;              // or -1: no such page
    float ks, lb;               // scale of the keys, log2 of the values'
    __device__ void get(const AttendArgs &a, uint32_t seq, uint32_t head, uint32_t j, uint32_t end) {
        index = -1;
        ks = lb = 0.0f;
        if (j < end) {
            const uint32_t col = j / a.c.per;
            const int32_t page = col < a.b.width ? a.b.table[(uint64_t)seq * a.b.width + col] : -1;
            if (page >= 0 && (uint32_t)page < a.c.n_pages) {
                index = ((int64_t)page * a.c.heads + head) * a.c.per + (j - col * a.c.per);
                ks = a.c.scales[2 * index];
                lb = log2_fast(a.c.scales[2 * index + 1]);
            } else if (a.b.status) {
                *a.b.status = COMET_ERR_FORMAT;
            }
        }
    }
    __device__ int64_t index_of(uint32_t i) const {
        const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(uint64_t)index, (int)i);
        const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)((uint64_t)index >> 32), (int)i);
        return (int64_t)((uint64_t)hi << 32 | lo);
    }
    __device__ static float of(float v, uint32_t i) { return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), (int)i)); }
};

// x and lv (weights_each) of a block's tokens from its raw products: visible are those before `limit`, if the block is there.
__device__ inline void each_of_block(const f32x16 &s, float kc, float lb, uint32_t j, int32_t limit, bool there, float *x, float *lv, float *top, float *tope) {
    const uint32_t h = (uint32_t)lane_id() >> 5;
    float best = kNegInf;
#pragma unroll
    for (int t = 0; t < 16; ++t) {
        const bool see = there && (int32_t)(j * 32u + 8u * (t / 4) + 4u * h + t % 4) < limit;
        x[t] = see ? s[t] * kc : kNegInf;
        lv[t] = see ? lb : 0.0f;
        best = fmaxf(best, x[t]);
    }
    *top = other_half_max(best);
    *tope = *top + lb;                        // (NaN for a poisoned block: no reference follows it)
}
// ... of the open block's, with the tokens' own scales; `held` of its tokens are there.
__device__ inline void each_of_open(const f32x16 &s, float qc, const float *ke, uint32_t held, uint32_t j, int32_t limit, float *x, float *lv, float *top, float *tope) {
    const uint32_t h = (uint32_t)lane_id() >> 5;
    float best = kNegInf, bests = kNegInf;
#pragma unroll
    for (int t = 0; t < 16; ++t) {
        const uint32_t tok = 8u * (t / 4) + 4u * h + t % 4;
        const bool see = tok < held && (int32_t)(j * 32u + tok) < limit;
        const float kt = ke[tok], vt = ke[32u + tok];
        x[t] = see ? s[t] * (kt * qc) : kNegInf;
        lv[t] = !see ? 0.0f : vt == vt ? (float)((int)(__float_as_uint(vt) >> 23) - 127) : vt;      // a power of two
        best = fmaxf(best, x[t]);
        bests = fmaxf(bests, x[t] + lv[t]);
    }
    *top = other_half_max(best);
    *tope = other_half_max(bests);
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

// Few rows: a wavefront holds 32 rows (queries of one key/value head, its group's heads side by side) and goes through every fourth
// block of its workgroup's piece straight from memory into the operands of the matrix instruction, with no LDS and no barrier
// in the loop.  Bound by HBM as long as rows are few.  grid: heads * a.slots workgroups of kAttendBlock threads, the heads of a piece side by side
template <int NC>
__global__ __launch_bounds__(kAttendBlock, NC <= 4 ? 2 : 1) void k_attend(AttendArgs a) {
    constexpr uint32_t dim = 32u * NC;
    __shared__ float s_stat[4][3][32];
    __shared__ __align__(16) float s_tile[4][1024];
    const uint32_t lane = (uint32_t)lane_id(), wave = threadIdx.x / kWave, n = lane & 31u, h = lane >> 5;
    const uint32_t number = blockIdx.x / a.c.heads, head = blockIdx.x - number * a.c.heads;
    Piece p;
    if (!find_piece(a, number, &p)) return;
    Seq s;
    if (!read_sequence(a.b, p.seq, &s)) return;
    const RowPlace place = row_place(a, s, head, p.tile * 32u + n);
    int32_t least, most;
    row_limits(a, s, p.tile * 32u, 32u, &least, &most);
    const uint32_t seen = most > 0 ? ((uint32_t)most + 31u) / 32u : 0u, parts = parts_of(seen, p.per);
    if (p.part >= parts) return;
    const uint32_t j0 = p.part * p.per, j1 = seen - j0 < p.per ? seen : j0 + p.per;
    const uint32_t whole = (uint32_t)s.len / 32u;                                             // complete blocks

    half8 q[2 * NC];
    const float qc = load_query<NC>(a, place, q) * a.scale;
    RowState<NC> row;
    row.clear();

    // the wavefront's blocks: j0 + wave, j0 + wave + 4, ...; where they lie is looked up for 64 of them at a time
    uint32_t j = j0 + wave;
    const uint32_t end = j1 < whole ? j1 : whole;
    u32x4 kr[NC], vr[NC];
    while (j < end) {
        Lookup look;
        look.get(a, p.seq, head, j + 4u * lane, end);
        const uint32_t left = (end - j + 3u) / 4u, count = left < 64u ? left : 64u;
        const auto load = [&](u32x4 *to, int64_t at, uint32_t which) {
            const uint8_t *from = a.c.blocks + (uint64_t)(at < 0 ? 0 : at) * (64u * dim) + which * (32u * dim) + n * 32u + h * 16u;
#pragma unroll
            for (int c = 0; c < NC; ++c) to[c] = *reinterpret_cast<const u32x4 *>(from + c * 1024);
        };
        int64_t at = look.index_of(0);
        load(kr, at, 0u);
        load(vr, at, 1u);
        for (uint32_t i = 0; i < count; ++i, j += 4u) {
            const int64_t next = i + 1u < count ? look.index_of(i + 1u) : -1;
            f32x16 acc = {};
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                acc = mfma(whole8(kr[c][0], kr[c][1]), q[2 * c], acc);
                acc = mfma(whole8(kr[c][2], kr[c][3]), q[2 * c + 1], acc);
            }
            if (next >= 0) load(kr, next, 0u);
            const float kc = Lookup::of(look.ks, i) * qc, lb = Lookup::of(look.lb, i);
            half8 pw[2];
            // (one place that moves the references, and x once more behind it: two such places cost a hundred registers)
            const bool all = at >= 0 && (int32_t)(j * 32u + 32u) <= least && lb == lb;
            float top, tope;
            if (all) {
                float best = acc[0];
#pragma unroll
                for (int t = 1; t < 16; ++t) best = fmaxf(best, acc[t]);
                top = other_half_max(best) * kc;
                tope = top + lb;
            } else {
                float x[16], lv[16];
                each_of_block(acc, kc, lb, j, place.limit, at >= 0, x, lv, &top, &tope);
            }
            row.follow(top, tope);
            if (all) {
                row.weights(acc, kc, lb, pw);
            } else {
                float x[16], lv[16];
                each_of_block(acc, kc, lb, j, place.limit, at >= 0, x, lv, &top, &tope);
                row.weights_each(x, lv, pw);
            }
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                row.o[c] = mfma(whole8(vr[c][0], vr[c][1]), pw[0], row.o[c]);
                row.o[c] = mfma(whole8(vr[c][2], vr[c][3]), pw[1], row.o[c]);
            }
            if (next >= 0) load(vr, next, 1u);
            at = next;
        }
    }

    // the open block, in 16 bits, with a scale for every token
    if (j == whole && j < j1) {
        uint32_t slot;
        if (read_slot(a.b, a.c, p.seq, &slot)) {
            const uint8_t *half = ring_half(a.c, slot, head, j);
            const uint32_t held = (uint32_t)s.len % 32u;
            f32x16 acc = {};
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    acc = mfma(*reinterpret_cast<const half8 *>(half + 2048u * c + 64u * n + 32u * h + 16u * u), q[2 * c + u], acc);
            float x[16], lv[16], top, tope;
            each_of_open(acc, qc, reinterpret_cast<const float *>(half + 128ull * dim), held, j, place.limit, x, lv, &top, &tope);
            row.follow(top, tope);
            half8 pw[2];
            row.weights_each(x, lv, pw);
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    row.o[c] = mfma(open_values(half + 64u * dim + 2048u * c + 64u * n + 32u * h + 16u * u, u, held), pw[u], row.o[c]);
        }
    }

    // The four wavefronts' results in one, in their order.
    row.l += other_half(row.l);
    if (h == 0u) { s_stat[wave][0][n] = row.m; s_stat[wave][1][n] = row.l; s_stat[wave][2][n] = row.r; }
    __syncthreads();
    float mm = kNegInf, rr = kNegInf, ll = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) { mm = fmaxf(mm, s_stat[w][0][n]); rr = fmaxf(rr, s_stat[w][2][n]); }
    const float mms = mm == kNegInf ? 0.0f : mm, rrs = rr == kNegInf ? 0.0f : rr;
#pragma unroll
    for (int w = 0; w < 4; ++w) ll += s_stat[w][1][n] * exp2_fast(s_stat[w][0][n] - mms);
    const float mine = exp2_fast(row.r - rrs);
    const bool last = parts == 1u;
    const uint64_t slot_no = ((uint64_t)p.number * a.c.heads + head) * 32u;
    if (wave == 0u && h == 0u) {
        if (last) {
            if (place.real && a.lse) a.lse[place.token * a.q_heads + place.qh] = log_sum(mms, ll);
        } else {
            float *st = a.part_s + 3u * (slot_no + n);
            st[0] = mm; st[1] = ll; st[2] = rr;
        }
        if (p.part == 0u && head == 0u && n == 0u) {
            int32_t *dir = a.directory + 2u * (first_unit(a.b.starts, p.seq, a.group, a.tile_shift, 1u) + p.tile);
            dir[0] = (int32_t)p.number;
            dir[1] = (int32_t)parts;
        }
    }
    // o of a row without tokens is 0
    const float fin = last ? (ll == 0.0f ? 0.0f : exp2_fast(rrs - mms - kLift) / ll) : 1.0f;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        if (c) __syncthreads();
#pragma unroll
        for (int t = 0; t < 4; ++t)
            *reinterpret_cast<f32x4 *>(&s_tile[wave][256 * t + 4 * lane]) =
                f32x4{row.o[c][4 * t] * mine, row.o[c][4 * t + 1] * mine, row.o[c][4 * t + 2] * mine, row.o[c][4 * t + 3] * mine};
        __syncthreads();
        // wavefront w takes registers 4w .. 4w + 3 of every lane: values 8w + 4h + i of the tile's 32
        f32x4 sum = *reinterpret_cast<const f32x4 *>(&s_tile[0][256 * wave + 4 * lane]);
#pragma unroll
        for (int w = 1; w < 4; ++w) sum += *reinterpret_cast<const f32x4 *>(&s_tile[w][256 * wave + 4 * lane]);
        sum *= fin;
        const uint32_t d = 32u * c + 8u * wave + 4u * h;
        if (place.real && last) store_out(a, place, d, sum);
        else if (place.real) *reinterpret_cast<f32x4 *>(a.part_o + (slot_no + n) * dim + d) = sum;
    }
}

// Many rows: the four wavefronts of a workgroup hold 32 * RT rows each and go through the same blocks together.  Every block is converted to
// float16 once per workgroup, in LDS, in the order of the operands (lane l's 16 bytes at 16 l: no bank conflicts).  Bound by the
// matrix instructions and by the vector instructions of the weights, about as many cycles of each for heads of 128.
// So with two tiles of rows per wavefront (A, B) the products of one are issued between the weights of the other:
//   A's weights of block j with  O_B += V(j-1) p_B  and  s_B = K(j) q_B;   B's weights with  O_A += V(j) p_A  and  s_A = K(j+1) q_A.
// The operands stay in registers for both tiles, which halves what is read from LDS.
template <int NC, int RT>
__global__ __launch_bounds__(kAttendBlock, 1) void k_attend_tile(AttendArgs a) {
    constexpr uint32_t dim = 32u * NC, rows_wave = 32u * RT, rows_wg = 4u * rows_wave;
    __shared__ __align__(16) uint8_t s_kv[2][128u * dim];             // a block: [keys, values][c][u][lane][16 bytes]
    const uint32_t lane = (uint32_t)lane_id(), wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave)), n = lane & 31u, h = lane >> 5;
    const uint32_t number = blockIdx.x / a.c.heads, head = blockIdx.x - number * a.c.heads;
    Piece p;
    if (!find_piece(a, number, &p)) return;
    Seq s;
    if (!read_sequence(a.b, p.seq, &s)) return;
    int32_t least, most;
    row_limits(a, s, p.tile * rows_wg, rows_wg, &least, &most);
    const uint32_t seen = most > 0 ? ((uint32_t)most + 31u) / 32u : 0u, parts = parts_of(seen, p.per);
    if (p.part >= parts) return;
    const uint32_t j0 = p.part * p.per, j1 = seen - j0 < p.per ? seen : j0 + p.per;
    const uint32_t whole = (uint32_t)s.len / 32u;
    const uint32_t row0 = p.tile * rows_wg + wave * rows_wave;
    RowPlace place[RT];
    half8 q[RT][2 * NC];
    float qc[RT];
    RowState<NC> row[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        place[rt] = row_place(a, s, head, row0 + 32u * rt + n);
        qc[rt] = load_query<NC>(a, place[rt], q[rt]) * a.scale;
        row[rt].clear();
    }

    // A wavefront converts the kilobytes wave, wave + 4, .. of a block's 2 NC.
    constexpr int kShare = (2 * NC + 3) / 4;
    const auto fetch = [&](u32x4 *to, int64_t at) {
        const uint8_t *from = a.c.blocks + (uint64_t)at * (64u * dim) + n * 32u + h * 16u;
#pragma unroll
        for (int i = 0; i < kShare; ++i)
            if (4 * i + 3 < 2 * NC || wave + 4u * i < 2u * NC) to[i] = *reinterpret_cast<const u32x4 *>(from + (wave + 4u * i) * 1024u);
    };
    const auto stage = [&](const u32x4 *from, uint32_t buf) {
#pragma unroll
        for (int i = 0; i < kShare; ++i)
            if (4 * i + 3 < 2 * NC || wave + 4u * i < 2u * NC) {
                uint8_t *to = &s_kv[buf][(wave + 4u * i) * 2048u + 16u * lane];
                *reinterpret_cast<half8 *>(to) = whole8(from[i][0], from[i][1]);
                *reinterpret_cast<half8 *>(to + 1024) = whole8(from[i][2], from[i][3]);
            }
    };
    const auto operands = [&](half8 *to, uint32_t buf, uint32_t which) {
#pragma unroll
        for (int c = 0; c < 2 * NC; ++c) to[c] = *reinterpret_cast<const half8 *>(&s_kv[buf][which * 64u * dim + 1024u * c + 16u * lane]);
    };
    const auto products = [&](const half8 *k, int rt) {
        f32x16 acc = {};
#pragma unroll
        for (int c = 0; c < 2 * NC; ++c) acc = mfma(k[c], q[rt][c], acc);
        return acc;
    };
    const auto accumulate = [&](const half8 *v, int rt, const half8 *pw) {
#pragma unroll
        for (int c = 0; c < NC; ++c) row[rt].o[c] = mfma(v[2 * c], pw[0], row[rt].o[c]);
#pragma unroll
        for (int c = 0; c < NC; ++c) row[rt].o[c] = mfma(v[2 * c + 1], pw[1], row[rt].o[c]);
    };
    const auto largest = [](const f32x16 &acc) {
        float best = acc[0];
#pragma unroll
        for (int t = 1; t < 16; ++t) best = fmaxf(best, acc[t]);
        return other_half_max(best);
    };

    // the blocks that every row sees whole, until one is missing or poisoned
    uint32_t j = j0;
    uint32_t fast = least > 0 ? (uint32_t)least / 32u : 0u;
    fast = fast < whole ? fast : whole;
    fast = fast < j1 ? fast : j1;
    while (j < fast) {
        Lookup look;
        look.get(a, p.seq, head, j + lane, fast);
        uint32_t count = fast - j < 64u ? fast - j : 64u;
        const uint64_t bad = wave_ballot(lane < count && (look.index < 0 || look.lb != look.lb));
        if (bad) {
            count = (uint32_t)__ffsll((unsigned long long)bad) - 1u;
            fast = j + count;
            if (!count) break;
        }
        u32x4 raw[kShare];
        fetch(raw, look.index_of(0));
        __syncthreads();                                               // (the batch before is done with the buffers)
        stage(raw, 0);
        fetch(raw, look.index_of(count > 1u ? 1u : 0u));
        __syncthreads();
        half8 kk[2 * NC], vv[2 * NC], pa[2] = {}, pb[2] = {};
        operands(kk, 0, 0);
        f32x16 sa = products(kk, 0), sb = {};
#pragma unroll
        for (int c = 0; c < 2 * NC; ++c) vv[c] = half8{};
        for (uint32_t i = 0; i < count; ++i) {
            const uint32_t buf = i & 1u;
            const float ks = Lookup::of(look.ks, i), lb = Lookup::of(look.lb, i);
            {
                const float kc = ks * qc[0], top = largest(sa) * kc;
                row[0].follow(top, top + lb);
                if constexpr (RT == 2) {
                    accumulate(vv, 1, pb);
                    sb = products(kk, 1);
                }
                row[0].weights(sa, kc, lb, pa);
            }
            operands(vv, buf, 1);
            stage(raw, buf ^ 1u);                                      // the block behind this one (the last is staged once more)
            fetch(raw, look.index_of(i + 2u < count ? i + 2u : count - 1u));
            __syncthreads();
            if constexpr (RT == 2) {
                const float kc = ks * qc[1], top = largest(sb) * kc;
                row[1].follow(top, top + lb);
                operands(kk, buf ^ 1u, 0);
                accumulate(vv, 0, pa);
                sa = products(kk, 0);
                row[1].weights(sb, kc, lb, pb);
            } else {
                operands(kk, buf ^ 1u, 0);
                accumulate(vv, 0, pa);
                sa = products(kk, 0);
            }
        }
        if constexpr (RT == 2) accumulate(vv, 1, pb);
        j += count;
    }

    // the others, one after another
    for (; j < j1; ++j) {
        int64_t at = -1;
        float ks = 0.0f, lb = 0.0f;
        const uint8_t *half = nullptr;
        uint32_t slot;
        if (j < whole) {
            Lookup look;
            look.get(a, p.seq, head, j, j + 1u);
            at = look.index; ks = look.ks; lb = look.lb;
            if (at < 0) continue;                                      // (the same for every lane of the workgroup)
        } else {
            if (!read_slot(a.b, a.c, p.seq, &slot)) break;
            half = ring_half(a.c, slot, head, j);
        }
        const uint32_t held = (uint32_t)s.len % 32u;
        __syncthreads();
        if (at >= 0) {
            u32x4 raw[kShare];
            fetch(raw, at);
            stage(raw, 0);
        } else {
            for (uint32_t i = wave; i < 2u * NC; i += 4u) {
                const uint8_t *from = half + 2048u * i + 64u * n + 32u * h;
                uint8_t *to = &s_kv[0][2048u * i + 16u * lane];
#pragma unroll
                for (uint32_t u = 0; u < 2u; ++u)
                    *reinterpret_cast<half8 *>(to + 1024u * u) = i < (uint32_t)NC ? *reinterpret_cast<const half8 *>(from + 16u * u) : open_values(from + 16u * u, u, held);
            }
        }
        __syncthreads();
        int32_t low, high;
        row_limits(a, s, row0, rows_wave, &low, &high);
        if ((int32_t)(j * 32u) >= high) continue;                      // nothing in it for this wavefront's rows
        half8 op[2 * NC];
        operands(op, 0, 0);
        half8 pw[RT][2];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const f32x16 acc = products(op, rt);
            float x[16], lv[16], top, tope;
            if (at >= 0) each_of_block(acc, ks * qc[rt], lb, j, place[rt].limit, true, x, lv, &top, &tope);
            else each_of_open(acc, qc[rt], reinterpret_cast<const float *>(half + 128ull * dim), held, j, place[rt].limit, x, lv, &top, &tope);
            row[rt].follow(top, tope);
            row[rt].weights_each(x, lv, pw[rt]);
        }
        operands(op, 0, 1);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) accumulate(op, rt, pw[rt]);
    }

    if (p.part == 0u && head == 0u && threadIdx.x == 0u) {
        int32_t *dir = a.directory + 2u * (first_unit(a.b.starts, p.seq, a.group, a.tile_shift, 1u) + p.tile);
        dir[0] = (int32_t)p.number;
        dir[1] = (int32_t)parts;
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        RowState<NC> &r = row[rt];
        const float l = r.l + other_half(r.l);
        const float ms = r.m == kNegInf ? 0.0f : r.m, rs = r.r == kNegInf ? 0.0f : r.r;
        if (parts == 1u) {
            const float fin = l == 0.0f ? 0.0f : exp2_fast(rs - ms - kLift) / l;
            if (place[rt].real) {
                if (a.lse && h == 0u) a.lse[place[rt].token * a.q_heads + place[rt].qh] = log_sum(ms, l);
#pragma unroll
                for (int c = 0; c < NC; ++c)
#pragma unroll
                    for (int t = 0; t < 4; ++t)
                        store_out(a, place[rt], 32u * c + 8u * t + 4u * h,
                                  f32x4{r.o[c][4 * t] * fin, r.o[c][4 * t + 1] * fin, r.o[c][4 * t + 2] * fin, r.o[c][4 * t + 3] * fin});
            }
        } else if (place[rt].real) {
            const uint64_t slot_no = ((uint64_t)p.number * a.c.heads + head) * rows_wg + wave * rows_wave + 32u * rt + n;
            if (h == 0u) {
                float *st = a.part_s + 3u * slot_no;
                st[0] = r.m; st[1] = l; st[2] = r.r;
            }
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int t = 0; t < 4; ++t)
                    *reinterpret_cast<f32x4 *>(a.part_o + slot_no * dim + 32u * c + 8u * t + 4u * h) =
                        f32x4{r.o[c][4 * t], r.o[c][4 * t + 1], r.o[c][4 * t + 2], r.o[c][4 * t + 3]};
        }
    }
}

// Joins the pieces of a row: a workgroup per row, its wavefronts (and the parts of one that a row does not fill) take the pieces in turn; their
// sums are added in a fixed order.  grid: (heads * tiles, rows at a time)
__global__ __launch_bounds__(kAttendBlock) void k_attend_join(AttendArgs a) {
    __shared__ __align__(16) float s_o[kAttendBlock][4];
    const uint32_t tid = threadIdx.x, lane = (uint32_t)lane_id(), dim = a.c.dim;
    const uint32_t unit = blockIdx.x / a.c.heads, head = blockIdx.x - unit * a.c.heads;
    const uint32_t seq = find_sequence(a.b.starts, a.b.n_seqs, unit, a.group, a.tile_shift, 1u);
    const uint32_t first = first_unit(a.b.starts, seq, a.group, a.tile_shift, 1u);
    const uint32_t tile = unit - first, tiles = tiles_of(a, seq);
    if (unit < first || tile >= tiles) return;
    const uint32_t number = (uint32_t)a.directory[2u * unit], parts = (uint32_t)a.directory[2u * unit + 1u];
    if (parts < 2u || number >= a.slots || parts > a.slots - number) return;   // (starts that make no sense leave entries unwritten)
    const uint32_t rows = (uint32_t)(a.b.starts[seq + 1] - a.b.starts[seq]) * a.group;
    const uint32_t quads = dim / 4u, lots = kAttendBlock / quads, lot = tid / quads, quad = tid - lot * quads;    // lots: pieces at a time
    for (uint32_t n = blockIdx.y; n < a.tile_rows && tile * a.tile_rows + n < rows; n += gridDim.y) {
        const uint32_t row = tile * a.tile_rows + n, query = row / a.group, qh = head * a.group + (row - query * a.group);
        const int64_t token = (int64_t)a.b.starts[seq] + query;
        const auto slot = [&](uint32_t k) { return ((uint64_t)(number + k) * a.c.heads + head) * a.tile_rows + n; };
        float m = kNegInf, r = kNegInf;
        for (uint32_t k = lane; k < parts; k += kWave) {                       // every wavefront for itself
            const float *st = a.part_s + 3u * slot(k);
            m = fmaxf(m, st[0]);
            r = fmaxf(r, st[2]);
        }
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) { m = fmaxf(m, __shfl_xor(m, o, kWave)); r = fmaxf(r, __shfl_xor(r, o, kWave)); }
        const float ms = m == kNegInf ? 0.0f : m, rs = r == kNegInf ? 0.0f : r;
        float l = 0.0f;
        for (uint32_t k = lane; k < parts; k += kWave) {
            const float *st = a.part_s + 3u * slot(k);
            l += st[1] * exp2_fast(st[0] - ms);
        }
        l = wave_sum<float>(l);
        f32x4 o = {};
        if (lot < lots)
            for (uint32_t k = lot; k < parts; k += lots)
                o += *reinterpret_cast<const f32x4 *>(a.part_o + slot(k) * dim + 4u * quad) * exp2_fast(a.part_s[3u * slot(k) + 2u] - rs);
        __syncthreads();
        *reinterpret_cast<f32x4 *>(s_o[tid]) = o;
        __syncthreads();
        if (tid < quads) {
            for (uint32_t k = 1; k < lots; ++k) o += *reinterpret_cast<const f32x4 *>(s_o[tid + k * quads]);
            const float fin = l == 0.0f ? 0.0f : exp2_fast(rs - ms - kLift) / l;
            if (tid == 0u && a.lse) a.lse[token * a.q_heads + qh] = log_sum(ms, l);
            RowPlace p;
            p.real = true; p.qh = qh; p.token = token; p.limit = 0;
            store_out(a, p, 4u * tid, o * fin);
        }
    }
}

template __global__ void k_attend<1>(AttendArgs);
template __global__ void k_attend<2>(AttendArgs);
template __global__ void k_attend<3>(AttendArgs);
template __global__ void k_attend<4>(AttendArgs);
template __global__ void k_attend<5>(AttendArgs);
template __global__ void k_attend<6>(AttendArgs);
template __global__ void k_attend<7>(AttendArgs);
template __global__ void k_attend<8>(AttendArgs);
template __global__ void k_attend_tile<1, 2>(AttendArgs);
template __global__ void k_attend_tile<2, 2>(AttendArgs);
template __global__ void k_attend_tile<3, 2>(AttendArgs);
template __global__ void k_attend_tile<4, 2>(AttendArgs);
template __global__ void k_attend_tile<5, 1>(AttendArgs);
template __global__ void k_attend_tile<6, 1>(AttendArgs);
template __global__ void k_attend_tile<7, 1>(AttendArgs);
template __global__ void k_attend_tile<8, 1>(AttendArgs);

}  // namespace comet
