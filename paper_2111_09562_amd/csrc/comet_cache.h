// The compressed key/value cache: layout, arguments of its kernels, and the device code they share (the rotation by
// positions, the search for a sequence).
//
// A block is 32 tokens of one key/value head of one sequence.  Complete blocks lie in pages, 8 bits a value with a scale
// for the block's keys and one for its values; the block that is still open lies in 16 bits in a ring of two blocks per slot
// and head, so a block is compressed exactly once, from the same 16-bit values however its tokens arrived.
//
//   blocks  [page][head][block of the page][64 * dim bytes]   keys int8 [dim/32][32 tokens][32], values int8 [dim][32 places]
//   scales  [page][head][block of the page][2] float32        of the keys, of the values
//   ring    [slot][head][2][128 * dim + 256 bytes]            the same orders in float16, then 32 + 32 float32 scales of tokens
//
// The orders are those of the matrix instruction's operands.  v_mfma_f32_32x32x16_f16 with the keys on the left takes 8
// consecutive values of a token per lane (lane & 31 the token, lane >> 5 which 8 of 16) and leaves in lane l the scores of
// query l & 31 against the tokens 8 * (i / 4) + 4 * (l >> 5) + i % 4, i = 0 .. 15.  Those registers are the right operand
// of the product with the values as they are, if a lane of the left operand holds, for its row of the head, the values of the same tokens
// in the same sequence: place 16h + 8u + 4w + i of a row is token 16u + 8w + 4h + i.  So a wavefront
// loads both with whole contiguous kilobytes, and no score ever moves between lanes.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/comet.h"
#include "comet_dev.h"

namespace comet {

constexpr int kBlk = 32;                      // tokens of a block
constexpr uint32_t kCacheMaxDim = 256;
constexpr int32_t kMaxLen = 0x7fffff00;        // tokens of a sequence: places of whole blocks stay below 2^31
constexpr float kMinScale = 0x1p-100f;        // of a block, as for the error bounds of the codec: smaller values are 0

struct CacheArgs {
    uint8_t *blocks;
    float *scales;
    uint8_t *ring;
    uint32_t n_pages, per, n_slots, heads, dim;   // per: blocks of a page
};
struct BatchArgs {
    const int32_t *starts, *lens, *table, *slots;
    uint32_t width, n_seqs, n_tokens;
    int32_t *status;
};
struct Rows {                                 // [token][head][dim], strides in elements
    uint8_t *p;
    int64_t token, head;
};
struct RopeArgs {
    const uint64_t *steps;                    // turns per position, 0.64 fixed point; null: no rotation
    const int32_t *positions;                 // of every token; null: its index in its sequence
    uint32_t rot, interleaved;
    float amp;
};

__host__ __device__ inline uint64_t ring_half_bytes(uint32_t dim) { return 128ull * dim + 256ull; }

constexpr int kRopeBlock = 256;
// A thread turns a chunk of V pairs (or copies V values behind the rotated part) of one token in every `groups`-th head, so the
// sines of the chunk are computed once for several heads.
struct RopeGrid {
    uint32_t groups, rot_chunks, chunks, per_token;    // chunks: rot_chunks and those that are copied; per_token = groups * chunks
    uint32_t tokens_wg;                                // tokens of a workgroup, or 0: a token takes several turns of the workgroup
};
template <typename T, int V>
__global__ void k_rope(RopeArgs r, RopeGrid g, Rows x, Rows y, uint32_t n_tokens, uint32_t heads, uint32_t dim, uint32_t sign);

constexpr int kCacheBlock = 256;
struct AppendArgs {
    CacheArgs c;
    BatchArgs b;
    Rows k, v, q, q_out;
    RopeArgs rope;
    uint32_t q_heads, q_heads_wg;             // q_heads_wg heads of the queries per workgroup
    uint32_t vec;                             // every row may be read and written 16 bytes at a time
};
template <typename T>
__global__ void k_cache_append(AppendArgs a);
struct FetchArgs {
    CacheArgs c;
    BatchArgs b;
    Rows k, v;
    uint32_t vec;
};
template <typename T>
__global__ void k_cache_fetch(FetchArgs a);
__host__ __device__ inline uint32_t cache_lds(uint32_t dim) { return 2u * kBlk * (dim + 8u) * 2u; }

constexpr int kAttendBlock = 256;
struct AttendArgs {
    CacheArgs c;
    BatchArgs b;
    Rows q, out;
    float *lse;                               // [token][query head], or null
    uint32_t q_heads, group;                  // group: query heads of a key/value head
    uint32_t bf16, causal, vec, wide;         // wide: k_attend_tile
    uint32_t tile_rows, tile_shift;           // rows of a workgroup: 2^tile_shift
    uint32_t min_blocks;                      // of a piece
    uint32_t pieces;                          // pieces the work of a key/value head is cut into, about
    uint32_t slots;                           // pieces of tiles that are cut, per head, at most
    float scale;                              // of the scores, times log2(e)
    float *part_o;                            // [slot][head][tile_rows][dim]
    float *part_s;                            // [slot][head][tile_rows][3]: reference and sum of the weights, reference of the values
    int32_t *directory;                       // [tile][2]: first slot, number of pieces
};
template <int NC, bool EXACT>
__global__ void k_attend(AttendArgs a);
template <int NC, bool EXACT>
__global__ void k_attend_few(AttendArgs a);
// Where the registers are enough for two wavefronts per SIMD, those fill each other's gaps; a single one's instructions are interleaved by hand.
constexpr bool tile_pairs(int nc, int rt) { return nc * rt <= 4; }
template <int NC, int RT>
__global__ void k_attend_tile(AttendArgs a);
__global__ void k_attend_join(AttendArgs a);
__global__ void k_attend_join_tile(AttendArgs a);

// ---- types ------------------------------------------------------------------------------------------------------
using half8 = _Float16 __attribute__((ext_vector_type(8)));
using half4 = _Float16 __attribute__((ext_vector_type(4)));
using ushort2v = uint16_t __attribute__((ext_vector_type(2)));
using half2v = _Float16 __attribute__((ext_vector_type(2)));
using f32x16 = float __attribute__((ext_vector_type(16)));
using f32x4 = float __attribute__((ext_vector_type(4)));
using u32x4 = uint32_t __attribute__((ext_vector_type(4)));

template <typename T, int V> struct Vec { using type = T __attribute__((ext_vector_type(V))); };

template <typename T, int V>
__device__ inline void load_row(float *to, const T *from) {
    if constexpr (V == 1) {
        to[0] = (float)from[0];
    } else {
        const typename Vec<T, V>::type x = *reinterpret_cast<const typename Vec<T, V>::type *>(from);
#pragma unroll
        for (int i = 0; i < V; ++i) to[i] = (float)x[i];
    }
}
template <typename T, int V>
__device__ inline void store_row(T *to, const float *from) {
    if constexpr (V == 1) {
        to[0] = (T)from[0];
    } else {
        typename Vec<T, V>::type x;
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = (T)from[i];
        *reinterpret_cast<typename Vec<T, V>::type *>(to) = x;
    }
}

// ---- rotation ---------------------------------------------------------------------------------------------------
// Sine and cosine of u / 2^32 turns.  The position times the step, both whole numbers, is exact modulo a turn however
// far the position lies; an angle in 32 bits would be off by 0.03 radians at a position of a million.  What is left is at most an
// eighth of a turn, where the series up to x^9 and x^10 are off by less than 2^-28.
__device__ inline void turn_sincos(uint32_t u, float amp, float &s, float &c) {
    const uint32_t q = (u + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(u - (q << 30)) * 1.4629180792671596e-9f;       // 2 pi / 2^32
    const float z = x * x;
    float sp = __builtin_fmaf(z, 2.7557319e-6f, -1.9841270e-4f);
    sp = __builtin_fmaf(z, sp, 8.3333333e-3f);
    sp = __builtin_fmaf(z, sp, -1.6666667e-1f);
    sp = __builtin_fmaf(x * z, sp, x);
    float cp = __builtin_fmaf(z, -2.7557319e-7f, 2.4801587e-5f);
    cp = __builtin_fmaf(z, cp, -1.3888889e-3f);
    cp = __builtin_fmaf(z, cp, 4.1666667e-2f);
    cp = __builtin_fmaf(z, cp, -0.5f);
    cp = __builtin_fmaf(z, cp, 1.0f);
    const float a = (q & 1u) ? cp : sp, b = (q & 1u) ? sp : cp;
    s = (q & 2u) ? -a * amp : a * amp;
    c = ((q + 1u) & 2u) ? -b * amp : b * amp;
}
__device__ inline uint32_t turn(int32_t position, uint64_t step) { return (uint32_t)(((uint64_t)(int64_t)position * step) >> 32); }

// Where the V pairs of chunk `c` of a row begin, and how far their second halves are: (i, i + rot / 2), or side by side.
template <int V>
__device__ inline uint32_t chunk_at(const RopeArgs &r, uint32_t c) { return r.interleaved ? 2u * V * c : V * c; }

// sign: 0 forward, 0x80000000 backward (the sine changes its sign)
template <int V>
__device__ inline void chunk_angles(const RopeArgs &r, uint32_t c, int32_t position, uint32_t sign, float *sn, float *cs) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
        turn_sincos(turn(position, r.steps[c * V + i]), r.amp, sn[i], cs[i]);
        sn[i] = __uint_as_float(__float_as_uint(sn[i]) ^ sign);
    }
}
// Turns the chunk's pairs: a and b are the 2V values in the order of memory (V == 1 or even).
template <int V>
__device__ inline void chunk_turn(bool interleaved, float *a, float *b, const float *sn, const float *cs) {
    if (interleaved) {
        float x[2 * V];
#pragma unroll
        for (int i = 0; i < V; ++i) { x[i] = a[i]; x[V + i] = b[i]; }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float u = x[2 * i], w = x[2 * i + 1];
            x[2 * i] = __builtin_fmaf(u, cs[i], -(w * sn[i]));
            x[2 * i + 1] = __builtin_fmaf(u, sn[i], w * cs[i]);
        }
#pragma unroll
        for (int i = 0; i < V; ++i) { a[i] = x[i]; b[i] = x[V + i]; }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float u = a[i], w = b[i];
            a[i] = __builtin_fmaf(u, cs[i], -(w * sn[i]));
            b[i] = __builtin_fmaf(u, sn[i], w * cs[i]);
        }
    }
}
template <int V>
__device__ inline uint32_t chunk_second(const RopeArgs &r) { return r.interleaved ? (uint32_t)V : r.rot / 2u; }

// ---- sequences --------------------------------------------------------------------------------------------------
__device__ inline void raise(int32_t *status) {
    if (status && lane_id() == 0) *status = COMET_ERR_FORMAT;
}

// Sequence b's units of 2^shift of its tokens * mul are numbered from first_unit(b) on: at least as many numbers as it can need,
// whatever the lengths, and known without adding up those in front of it.  With `extra` = 2 there is room for the blocks of 32 that its
// tokens touch (shift 5, mul 1), with 1 for tiles that begin with the sequence.
__device__ inline uint32_t first_unit(const int32_t *starts, uint32_t b, uint32_t mul, uint32_t shift, uint32_t extra) {
    return (uint32_t)(((uint64_t)(uint32_t)starts[b] * mul) >> shift) + extra * b;
}
struct Seq {
    int32_t start, n, len;      // first token in the batch, new tokens, tokens held once they are in
};
// false: the batch's numbers for this sequence make no sense (reported) or it has no tokens in the batch
__device__ inline bool check_sequence(const BatchArgs &b, int32_t s0, int32_t s1, int32_t len, Seq *s) {
    if (s0 < 0 || s1 < s0 || s1 > (int32_t)b.n_tokens || len < 0 || len > kMaxLen) {
        raise(b.status);
        return false;
    }
    s->start = s0; s->n = s1 - s0; s->len = len;
    return s->n > 0;
}
__device__ inline bool check_slot(const BatchArgs &b, const CacheArgs &c, int32_t v) {
    if (v >= 0 && (uint32_t)v < c.n_slots) return true;
    raise(b.status);
    return false;
}
__device__ inline bool read_slot(const BatchArgs &b, const CacheArgs &c, uint32_t seq, uint32_t *slot) {
    const int32_t v = b.slots ? b.slots[seq] : (int32_t)seq;
    *slot = (uint32_t)v;
    return check_slot(b, c, v);
}
// The sequence whose blocks of new tokens `unit` is among (first_unit with shift 5, mul 1, extra 2), its numbers and its slot (unchecked), and
// which of its blocks that is.  Once 64 sequences are left everything about them is loaded at once: a step of up to 64 sequences
// waits for one load here instead of three.
struct Unit {
    uint32_t seq, block;
    int32_t slot;
    Seq s;
};
__device__ inline bool find_block(const BatchArgs &b, uint32_t unit, Unit *u) {
    uint32_t lo = 0, len = b.n_seqs;
    while (len > 64u) {
        const uint32_t stride = (len + 63u) / 64u, off = (uint32_t)lane_id() * stride;
        const bool le = off < len && first_unit(b.starts, lo + off, 1u, 5u, 2u) <= unit;
        const uint32_t n = (uint32_t)__popcll(wave_ballot(le)), k = n > 0u ? n - 1u : 0u;
        lo += k * stride;
        len = len - k * stride < stride ? len - k * stride : stride;
    }
    const uint32_t mine = (uint32_t)lane_id() < len ? lo + (uint32_t)lane_id() : lo;
    const int32_t s0 = b.starts[mine], s1 = b.starts[mine + 1u], held = b.lens[mine], slot = b.slots ? b.slots[mine] : (int32_t)mine;
    const uint32_t first = ((uint32_t)s0 >> 5) + 2u * mine;
    const uint32_t n = (uint32_t)__popcll(wave_ballot((uint32_t)lane_id() < len && first <= unit));
    const int k = (int)(n > 0u ? n - 1u : 0u);
    const auto of = [k](int32_t v) { return __builtin_amdgcn_readlane(v, k); };
    u->seq = lo + (uint32_t)k;
    u->slot = of(slot);
    const uint32_t f = (uint32_t)of((int32_t)first);
    if (!check_sequence(b, of(s0), of(s1), of(held), &u->s) || unit < f) return false;
    if (u->s.len < u->s.n) {
        raise(b.status);
        return false;
    }
    u->block = (uint32_t)(u->s.len - u->s.n) / kBlk + (unit - f);
    return u->block <= (uint32_t)(u->s.len - 1) / kBlk;
}
// Index of block j of a sequence's head among all blocks of the cache, or -1 (reported): behind the table's end or no page.
__device__ inline int64_t block_index(const BatchArgs &b, const CacheArgs &c, uint32_t seq, uint32_t head, uint32_t j) {
    const uint32_t col = j / c.per;
    const int32_t page = col < b.width ? b.table[(uint64_t)seq * b.width + col] : -1;
    if (page < 0 || (uint32_t)page >= c.n_pages) {
        raise(b.status);
        return -1;
    }
    return ((int64_t)page * c.heads + head) * c.per + (j - col * c.per);
}
__device__ inline uint8_t *ring_half(const CacheArgs &c, uint32_t slot, uint32_t head, uint32_t j) {
    return c.ring + (((uint64_t)slot * c.heads + head) * 2u + (j & 1u)) * ring_half_bytes(c.dim);
}
// token -> place in a row of the values
__device__ inline uint32_t place_of(uint32_t t) { return 16u * ((t >> 2) & 1u) + 8u * (t >> 4) + 4u * ((t >> 3) & 1u) + (t & 3u); }
__device__ inline uint32_t token_at(uint32_t p) { return 16u * ((p >> 3) & 1u) + 8u * ((p >> 2) & 1u) + 4u * (p >> 4) + (p & 3u); }

}  // namespace comet
