// Attention of the batch's queries over the compressed cache.
//
// One pass over the keys with the running maximum m and sum l of every row.  With q the row, K and V the whole numbers of a
// block and a, b its scales:  x = (q . K) a c,  p = exp2(x - m),  l += p,  O += (p g) V,  g = exp2(m - r) b,  o = O exp2(r - m) / l.
// r is a second running reference: the largest x + log2 b so far.  p g, which the matrix instruction takes in float16, is
// lifted by 2^14 and so at most 2^15 whatever the scales of the blocks are, and weights down to 2^-28 of the largest keep all bits
// float16 has (a hundred thousand tokens of next to no weight still count).  The whole numbers are exact in float16, so the only
// rounding below 32 bits is that of p g, at most 2^-11 of each weight.  The query goes in as float16 times a power of two of its
// row, which is exact for both 16-bit types but for values below 2^-38 of the row's largest.
//
// A wavefront holds 32 rows (queries of one key/value head, its group's heads side by side) and goes through blocks of 32
// tokens straight from memory into the operands of the matrix instruction: no LDS and no barrier in the loop.
#include "comet_cache.h"

namespace comet {

namespace {

constexpr float kNegInf = -__builtin_inff();
constexpr float kLift = 14.0f;            // log2 of what the weights are multiplied with on their way into float16

// Tiles of 32 rows and blocks of a sequence.
__device__ inline uint32_t tiles_of(const AttendArgs &a, uint32_t seq) {
    const int32_t s0 = a.b.starts[seq], s1 = a.b.starts[seq + 1];
    if (s0 < 0 || s1 <= s0 || s1 > (int32_t)a.b.n_tokens || a.b.lens[seq] < 0 || a.b.lens[seq] > kMaxLen) return 0u;
    return (uint32_t)(((uint64_t)(uint32_t)(s1 - s0) * a.group + 31u) / 32u);
}
__device__ inline uint32_t blocks_of(const AttendArgs &a, uint32_t seq) { return (uint32_t)((a.b.lens[seq] + 31ll) / 32); }

struct Piece {
    uint32_t seq, tile, part, parts;      // `part` of `parts` of a tile's blocks
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
        if (b < a.b.n_seqs) v = (uint64_t)tiles_of(a, b) * blocks_of(a, b);
        total += wave_sum<uint64_t>(v);
    }
    uint64_t per64 = (total + a.pieces - 1u) / a.pieces;
    if (per64 < 8u) per64 = 8u;
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
            p->parts = (uint32_t)__builtin_amdgcn_readfirstlane((int)k);
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

__device__ inline float other_half_max(float v) { return fmaxf(v, __shfl_xor(v, 32, kWave)); }
__device__ inline float other_half_sum(float v) { return v + __shfl_xor(v, 32, kWave); }
__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

}  // namespace

// grid: heads * a.slots workgroups of kAttendBlock threads, the heads of a piece side by side
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
    const uint32_t rows = (uint32_t)s.n * a.group, row = p.tile * 32u + n;
    const bool real = row < rows;
    const uint32_t query = real ? row / a.group : (uint32_t)s.n - 1u, qh = head * a.group + (real ? row - query * a.group : 0u);
    const int64_t token = (int64_t)s.start + query;
    // tokens a row sees: all, or those up to its own place at the sequence's end (none if that lies in front of the beginning)
    const int32_t limit = a.causal ? s.len - s.n + (int32_t)query + 1 : s.len;
    const int32_t last_query = (int32_t)((p.tile * 32u + 31u < rows ? p.tile * 32u + 31u : rows - 1u) / a.group);
    const int32_t most = a.causal ? s.len - s.n + last_query + 1 : s.len;                        // the largest limit of the tile
    const int32_t least = a.causal ? s.len - s.n + (int32_t)(p.tile * 32u / a.group) + 1 : s.len;
    const uint32_t seen = most > 0 ? ((uint32_t)most + 31u) / 32u : 0u;
    const uint32_t j0 = p.part * p.per < seen ? p.part * p.per : seen, j1 = seen - j0 < p.per ? seen : j0 + p.per;
    const uint32_t whole = (uint32_t)s.len / 32u;                                             // complete blocks

    // the queries: float16 times a power of two
    half8 q[2 * NC];
    float q_scale = 1.0f;
    {
        const uint16_t *src = reinterpret_cast<const uint16_t *>(a.q.p) + token * a.q.token + (int64_t)qh * a.q.head;
        float top = 0.0f;
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
        if (a.bf16) {
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    top = fmaxf(top, fmaxf(fabsf(__uint_as_float(raw[c][i] << 16)), fabsf(__uint_as_float(raw[c][i] & 0xffff0000u))));
            top = other_half_max(top);
            uint32_t e = __float_as_uint(top) >> 23;
            e = e < 15u ? 15u : e;
            q_scale = __uint_as_float((e - 14u) << 23);                       // 2^(exponent - 14): the largest comes to lie in [2^14, 2^15)
            const float inv = 1.0f / q_scale;                                 // exact (Inf in a row leaves Inf or NaN in it either way)
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    q[2 * c + i / 4][2 * (i % 4)] = (_Float16)(__uint_as_float(raw[c][i] << 16) * inv);
                    q[2 * c + i / 4][2 * (i % 4) + 1] = (_Float16)(__uint_as_float(raw[c][i] & 0xffff0000u) * inv);
                }
        } else {
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const half2v two = __builtin_bit_cast(half2v, raw[c][i]);
                    q[2 * c + i / 4][2 * (i % 4)] = two[0];
                    q[2 * c + i / 4][2 * (i % 4) + 1] = two[1];
                }
        }
    }
    const float qc = q_scale * a.scale;

    f32x16 o[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) o[c] = f32x16{};
    float m = kNegInf, r = kNegInf, l = 0.0f;           // l: of the lane's own tokens until the end

    // One block: x and the whole (or 16-bit) values are given; masked: some row does not see all of it
    const auto softmax = [&](float *x, float top, float e, auto gain, half8 *pw) {
        // top: the lane's largest x, e: log2 of (a power of two of) the scale; gain(i): what token i's weight is multiplied with, on top of exp2(m + e - r)
        top = other_half_max(top);
        const float m2 = fmaxf(m, top), r2 = fmaxf(r, top + e);
        const float ms = m2 == kNegInf ? 0.0f : m2, rs = r2 == kNegInf ? 0.0f : r2;
        if (wave_ballot(m2 != m || r2 != r)) {
            l *= exp2_fast(m - ms);
            const float alpha = exp2_fast(r - rs);
#pragma unroll
            for (int c = 0; c < NC; ++c) o[c] *= alpha;
            m = m2;
            r = r2;
        }
        const float g = exp2_fast(ms + e - rs + kLift);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float w = exp2_fast(x[i] - ms);
            l += w;
            pw[i / 8][i % 8] = (_Float16)gain(i, w, g);
        }
    };

    // the wavefront's blocks: j0 + wave, j0 + wave + 4, ...; where they lie is looked up for 64 of them at a time
    uint32_t j = j0 + wave;
    const uint32_t end = j1 < whole ? j1 : whole;
    u32x4 kr[NC], vr[NC];
    while (j < end) {
        const uint32_t mine = j + 4u * lane;
        int64_t index = -1;
        float ks = 0.0f, vs = 0.0f;
        if (mine < end) {
            const uint32_t col = mine / a.c.per;
            const int32_t page = col < a.b.width ? a.b.table[(uint64_t)p.seq * a.b.width + col] : -1;
            if (page >= 0 && (uint32_t)page < a.c.n_pages) {
                index = ((int64_t)page * a.c.heads + head) * a.c.per + (mine - col * a.c.per);
                ks = a.c.scales[2 * index];
                vs = a.c.scales[2 * index + 1];
            } else if (a.b.status) {
                *a.b.status = COMET_ERR_FORMAT;
            }
        }
        const uint32_t left = (end - j + 3u) / 4u, count = left < 64u ? left : 64u;
        const auto place = [&](uint32_t i) -> int64_t {
            const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(uint64_t)index, (int)i);
            const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)((uint64_t)index >> 32), (int)i);
            return (int64_t)((uint64_t)hi << 32 | lo);
        };
        const auto load = [&](u32x4 *to, int64_t at, uint32_t which) {
            const uint8_t *from = a.c.blocks + (uint64_t)(at < 0 ? 0 : at) * (64u * dim) + which * (32u * dim) + n * 32u + h * 16u;
#pragma unroll
            for (int c = 0; c < NC; ++c) to[c] = *reinterpret_cast<const u32x4 *>(from + c * 1024);
        };
        int64_t at = place(0);
        load(kr, at, 0u);
        load(vr, at, 1u);
        for (uint32_t i = 0; i < count; ++i, j += 4u) {
            const int64_t next = i + 1u < count ? place(i + 1u) : -1;
            f32x16 acc = {};
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(whole8(kr[c][0], kr[c][1]), q[2 * c], acc, 0, 0, 0);
                acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(whole8(kr[c][2], kr[c][3]), q[2 * c + 1], acc, 0, 0, 0);
            }
            if (next >= 0) load(kr, next, 0u);
            const float bk = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(ks), (int)i));
            const float bv = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(vs), (int)i));
            // bv = 2^e * part, part in [1, 2)
            const float e = (float)((int)(__float_as_uint(bv) >> 23) - 127);
            const float part = __uint_as_float((__float_as_uint(bv) & 0x007fffffu) | 0x3f800000u);
            const float bad = bv != bv ? bv : 0.0f;                       // a poisoned block: NaN for every row that sees it
            float x[16], top = kNegInf;
            const float kc = bk * qc;
            half8 pw[2];
            if (at >= 0 && (int32_t)(j * 32u + 32u) <= least) {
#pragma unroll
                for (int t = 0; t < 16; ++t) { x[t] = acc[t] * kc; top = fmaxf(top, x[t]); }
                softmax(x, top, e, [&](int, float w, float g) { return __builtin_fmaf(w, g * part, bad); }, pw);
            } else {
#pragma unroll
                for (int t = 0; t < 16; ++t) {
                    const int32_t place_t = (int32_t)(j * 32u + 8u * (t / 4) + 4u * h + t % 4);
                    x[t] = at >= 0 && place_t < limit ? acc[t] * kc : kNegInf;
                    top = fmaxf(top, x[t]);
                }
                softmax(x, top, e, [&](int t, float w, float g) {
                    return x[t] == kNegInf ? 0.0f : __builtin_fmaf(w, g * part, bad); }, pw);
            }
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                o[c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(whole8(vr[c][0], vr[c][1]), pw[0], o[c], 0, 0, 0);
                o[c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(whole8(vr[c][2], vr[c][3]), pw[1], o[c], 0, 0, 0);
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
            const float *ke = reinterpret_cast<const float *>(half + 128ull * dim), *ve = ke + 32;
            const uint32_t held = (uint32_t)s.len % 32u;
            f32x16 acc = {};
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const half8 k = *reinterpret_cast<const half8 *>(half + 2048u * c + 64u * n + 32u * h + 16u * u);
                    acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(k, q[2 * c + u], acc, 0, 0, 0);
                }
            float x[16], w_e[16], bad[16], top = kNegInf, e = kNegInf;
#pragma unroll
            for (int t = 0; t < 16; ++t) {
                const uint32_t tok = 8u * (t / 4) + 4u * h + t % 4;
                const bool see = tok < held && (int32_t)(j * 32u + tok) < limit;
                const float kt = ke[tok], vt = ve[tok];
                x[t] = see ? acc[t] * (kt * qc) : kNegInf;
                top = fmaxf(top, x[t]);
                w_e[t] = see && vt == vt ? (float)((int)(__float_as_uint(vt) >> 23) - 127) : kNegInf;
                bad[t] = see && vt != vt ? vt : 0.0f;
                e = fmaxf(e, w_e[t]);
            }
            e = other_half_max(e);
            const float es = e == kNegInf ? 0.0f : e;
            half8 pw[2];
            softmax(x, top, es, [&](int t, float w, float g) {
                return x[t] == kNegInf ? 0.0f : __builtin_fmaf(w * g, exp2_fast(w_e[t] - es), bad[t]); }, pw);
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    half8 v = *reinterpret_cast<const half8 *>(half + 64u * dim + 2048u * c + 64u * n + 32u * h + 16u * u);
#pragma unroll
                    for (int i = 0; i < 8; ++i)                           // places nobody has written yet may hold anything
                        if (16u * u + 8u * (i / 4) + 4u * h + i % 4 >= held) v[i] = (_Float16)0.0f;
                    o[c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, pw[u], o[c], 0, 0, 0);
                }
        }
    }

    // The four wavefronts' results in one, in their order.
    l = other_half_sum(l);
    if (h == 0u) { s_stat[wave][0][n] = m; s_stat[wave][1][n] = l; s_stat[wave][2][n] = r; }
    __syncthreads();
    float mm = kNegInf, rr = kNegInf, ll = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) { mm = fmaxf(mm, s_stat[w][0][n]); rr = fmaxf(rr, s_stat[w][2][n]); }
    const float mms = mm == kNegInf ? 0.0f : mm, rrs = rr == kNegInf ? 0.0f : rr;
#pragma unroll
    for (int w = 0; w < 4; ++w) ll += s_stat[w][1][n] * exp2_fast(s_stat[w][0][n] - mms);
    const float mine = exp2_fast(r - rrs);
    const bool last = p.parts == 1u;
    const uint64_t slot_no = ((uint64_t)p.number * a.c.heads + head) * 32u;
    if (wave == 0u && h == 0u) {
        if (last) {
            if (real && a.lse) a.lse[token * a.q_heads + qh] = ll > 0.0f ? (mms + __log2f(ll)) * 0.6931471805599453f : (ll == ll ? kNegInf : ll);
        } else {
            float *st = a.part_s + 3u * (slot_no + n);
            st[0] = mm; st[1] = ll; st[2] = rr;
        }
        if (p.part == 0u && head == 0u && n == 0u) {
            int32_t *dir = a.directory + 2u * (first_unit(a.b.starts, p.seq, a.group, 1u) + p.tile);
            dir[0] = (int32_t)p.number;
            dir[1] = (int32_t)p.parts;
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
                f32x4{o[c][4 * t] * mine, o[c][4 * t + 1] * mine, o[c][4 * t + 2] * mine, o[c][4 * t + 3] * mine};
        __syncthreads();
        // wavefront w takes registers 4w .. 4w + 3 of every lane: values 8w + 4h + i of the tile's 32
        f32x4 sum = *reinterpret_cast<const f32x4 *>(&s_tile[0][256 * wave + 4 * lane]);
#pragma unroll
        for (int w = 1; w < 4; ++w) sum += *reinterpret_cast<const f32x4 *>(&s_tile[w][256 * wave + 4 * lane]);
        sum *= fin;
        const uint32_t d = 32u * c + 8u * wave + 4u * h;
        if (real && last) {
            uint16_t *dst = reinterpret_cast<uint16_t *>(a.out.p) + token * a.out.token + (int64_t)qh * a.out.head + d;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                dst[i] = a.bf16 ? __builtin_bit_cast(uint16_t, (__bf16)sum[i]) : __builtin_bit_cast(uint16_t, (_Float16)sum[i]);
        } else if (real) {
            *reinterpret_cast<f32x4 *>(a.part_o + (slot_no + n) * dim + d) = sum;
        }
    }
}

// Joins the pieces of a row: a wavefront per row.  grid: heads * tiles
__global__ __launch_bounds__(kAttendBlock) void k_attend_join(AttendArgs a) {
    const uint32_t unit = blockIdx.x / a.c.heads, head = blockIdx.x - unit * a.c.heads, dim = a.c.dim, lane = (uint32_t)lane_id(), wave = threadIdx.x / kWave;
    const uint32_t seq = find_sequence(a.b.starts, a.b.n_seqs, unit, a.group, 1u);
    const uint32_t first = first_unit(a.b.starts, seq, a.group, 1u);
    const uint32_t tile = unit - first, tiles = tiles_of(a, seq);
    if (unit < first || tile >= tiles) return;
    const uint32_t number = (uint32_t)a.directory[2u * unit], parts = (uint32_t)a.directory[2u * unit + 1u];
    if (parts < 2u || number >= a.slots || parts > a.slots - number) return;   // (starts that make no sense leave entries unwritten)
    const uint32_t rows = (uint32_t)(a.b.starts[seq + 1] - a.b.starts[seq]) * a.group;
    for (uint32_t n = wave; n < 32u && tile * 32u + n < rows; n += kAttendBlock / kWave) {
        const uint32_t row = tile * 32u + n, query = row / a.group, qh = head * a.group + (row - query * a.group);
        const int64_t token = (int64_t)a.b.starts[seq] + query;
        float m = kNegInf, r = kNegInf;
        for (uint32_t k = lane; k < parts; k += kWave) {
            const float *st = a.part_s + 3u * (((uint64_t)(number + k) * a.c.heads + head) * 32u + n);
            m = fmaxf(m, st[0]);
            r = fmaxf(r, st[2]);
        }
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) { m = fmaxf(m, __shfl_xor(m, o, kWave)); r = fmaxf(r, __shfl_xor(r, o, kWave)); }
        const float ms = m == kNegInf ? 0.0f : m, rs = r == kNegInf ? 0.0f : r;
        float l = 0.0f, o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (uint32_t k = 0; k < parts; ++k) {
            const uint64_t at = ((uint64_t)(number + k) * a.c.heads + head) * 32u + n;
            const float *st = a.part_s + 3u * at;
            l += st[1] * exp2_fast(st[0] - ms);
            const float f = exp2_fast(st[2] - rs);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (lane + 64u * i < dim) o[i] += a.part_o[at * dim + lane + 64u * i] * f;
        }
        const float fin = l == 0.0f ? 0.0f : exp2_fast(rs - ms - kLift) / l;
        if (lane == 0u && a.lse) a.lse[token * a.q_heads + qh] = l > 0.0f ? (ms + __log2f(l)) * 0.6931471805599453f : (l == l ? kNegInf : l);
        uint16_t *dst = reinterpret_cast<uint16_t *>(a.out.p) + token * a.out.token + (int64_t)qh * a.out.head;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (lane + 64u * i < dim)
                dst[lane + 64u * i] = a.bf16 ? __builtin_bit_cast(uint16_t, (__bf16)(o[i] * fin)) : __builtin_bit_cast(uint16_t, (_Float16)(o[i] * fin));
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

}  // namespace comet
