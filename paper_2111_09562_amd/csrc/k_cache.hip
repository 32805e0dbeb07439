// Keys and values into the compressed cache and out of it again.  Bound by HBM for prompts, by a chain of memory round trips for single tokens.
// 18792 tokens, 8 + 8 heads of 128, bf16: in 38 us (3.0 TB/s; 34 without the rotation), with 32 heads of queries 101 us (4.2 TB/s), out 20.5 us
// (5.6 TB/s; behind the append of the same tokens, whose writes are still on their way, 30).  64 single tokens: in 7.8 us, 12.7 if all of them complete a
// block, out 3.7.
#include <type_traits>

#include "comet_cache.h"

namespace comet {

namespace {

template <typename T> __device__ inline float widen(uint16_t raw);
template <> __device__ inline float widen<__bf16>(uint16_t raw) { return __uint_as_float((uint32_t)raw << 16); }
template <> __device__ inline float widen<_Float16>(uint16_t raw) { return (float)__builtin_bit_cast(_Float16, raw); }
template <typename T> __device__ inline uint16_t narrow(float v) { return __builtin_bit_cast(uint16_t, (T)v); }
template <typename T> constexpr uint32_t kInf16 = 0x7f80u;              // |bits| from here on: Inf and NaN
template <> constexpr uint32_t kInf16<_Float16> = 0x7c00u;

// The rows r0 .. of a block that are new and, with `old`, those the ring holds of it, in LDS: [32][dim + 8], the keys rotated and rounded to T.  The
// cache compresses the 16-bit keys that a model working in T would keep, so it does not matter in how many calls a
// block's tokens came.
template <typename T, int V>
__device__ void load_block(const AppendArgs &a, const Seq &s, uint32_t before, uint32_t head, uint32_t slot, uint32_t j, uint32_t r0, uint32_t r1, bool old,
                           uint16_t *kt, uint16_t *vt) {
    const uint32_t dim = a.c.dim, pitch = dim + 8u;
    const uint32_t rot = a.rope.steps ? a.rope.rot : 0u;
    const uint32_t rot_chunks = rot / (2u * V), chunks = rot_chunks + (dim - rot) / V;
    for (uint32_t i = threadIdx.x; i < (r1 - r0) * chunks; i += kCacheBlock) {
        const uint32_t row = r0 + i / chunks, c = i % chunks, t = j * kBlk + row;
        const int32_t token = s.start + (int32_t)(t - before);
        const T *p = reinterpret_cast<const T *>(a.k.p) + (int64_t)token * a.k.token + (int64_t)head * a.k.head;
        float x[V], y[V];
        if (c < rot_chunks) {
            float sn[V], cs[V];
            const uint32_t at = chunk_at<V>(a.rope, c), second = at + chunk_second<V>(a.rope);
            load_row<T, V>(x, p + at);
            load_row<T, V>(y, p + second);
            chunk_angles<V>(a.rope, c, a.rope.positions ? a.rope.positions[token] : (int32_t)t, 0u, sn, cs);
            chunk_turn<V>(a.rope.interleaved, x, y, sn, cs);
            store_row<T, V>(reinterpret_cast<T *>(kt + row * pitch + at), x);
            store_row<T, V>(reinterpret_cast<T *>(kt + row * pitch + second), y);
        } else {
            const uint32_t at = rot + (c - rot_chunks) * V;
            load_row<T, V>(x, p + at);
            store_row<T, V>(reinterpret_cast<T *>(kt + row * pitch + at), x);
        }
    }
    for (uint32_t i = threadIdx.x ^ 128u; i < (r1 - r0) * (dim / V); i += kCacheBlock) {      // (of few rows not by the wavefront that has the keys)
        const uint32_t row = r0 + i / (dim / V), d = i % (dim / V) * V, t = j * kBlk + row;
        const int32_t token = s.start + (int32_t)(t - before);
        float x[V];
        load_row<T, V>(x, reinterpret_cast<const T *>(a.v.p) + (int64_t)token * a.v.token + (int64_t)head * a.v.head + d);
        store_row<T, V>(reinterpret_cast<T *>(vt + row * pitch + d), x);
    }
    if (!old) return;
    const uint8_t *half = ring_half(a.c, slot, head, j);
    const uint16_t *kr = reinterpret_cast<const uint16_t *>(half), *vr = kr + 32u * dim;
    const float *e = reinterpret_cast<const float *>(half + 128ull * dim);
    // A round's loads, eight values of a key and four tokens of two values, wait for memory together (larger rounds cost a wavefront per SIMD:
    // when they were chosen, 64 tokens that all complete a block took 11.5 us, 10.9 with rounds twice that, 12.7 one load at a time; 18792 tokens 7 us more
    // with the large rounds).
    const uint32_t n_k = r0 * (dim / 8u), quad = token_at(4u * (threadIdx.x % 8u));           // (r0 <= 31 tokens of before)
    const f32x4 ve = *reinterpret_cast<const f32x4 *>(e + 32u + quad);
    for (uint32_t k0 = threadIdx.x, v0 = threadIdx.x; v0 < 8u * dim; k0 += kCacheBlock, v0 += 2u * kCacheBlock) {
        const bool there = k0 < n_k;
        const uint32_t row = there ? k0 / (dim / 8u) : 0u, d = there ? k0 % (dim / 8u) * 8u : 0u, v1 = v0 + kCacheBlock;
        const half8 k = *reinterpret_cast<const half8 *>(kr + (d / 32u * 32u + row) * 32u + d % 32u);
        const float ke = e[row];
        const half4 v[2] = {*reinterpret_cast<const half4 *>(vr + 4u * v0), *reinterpret_cast<const half4 *>(vr + 4u * (v1 < 8u * dim ? v1 : v0))};
        if (there) {
#pragma unroll
            for (uint32_t u = 0; u < 8u; ++u) kt[row * pitch + d + u] = narrow<T>((float)k[u] * ke);
        }
#pragma unroll
        for (uint32_t m = 0; m < 2u; ++m) {
            const uint32_t at = m ? v1 : v0;
            if (at < 8u * dim) {
#pragma unroll
                for (uint32_t u = 0; u < 4u; ++u)
                    if (quad + u < r0) vt[(quad + u) * pitch + at / 8u] = narrow<T>((float)v[m][u] * ve[u]);
            }
        }
    }
}

// Power of two by which a token's values are divided on their way into float16: the largest then lies in [2^14, 2^15), and float16 steps there end at
// 2^-24.  So a value is off by at most 2^-39 of the token's largest, and a bf16 value by nothing down to 2^-31 of that.  (A block's values in
// 8 bits do not notice: what was rounded here is 0 there.)
__device__ inline float token_scale(float amax) {
    uint32_t e = __float_as_uint(amax) >> 23;
    if (e < 15u) e = 15u;
    return __uint_as_float((e - 14u) << 23);
}

__device__ inline uint32_t larger16(uint32_t a, uint32_t b) { return a > b ? a : b; }

// A block's scale from the bits of its largest |value| a, and its values in whole numbers, rint(127 x / a) (ties to even).  With x = m 2^e, a = n 2^f a tie
// is 254 x / a = an odd number: x = a / 2 (63.5, whose even neighbour lies above), or n a multiple of 127.  Away from ties 127 x / a is at least 2^-19 of itself.
//   bf16 (n below 256: 127 and 254, powers of two times 127): inv is 127 / a rounded up, so x inv is above the quotient by less than 2^-22 of it,
//     exact at the ties of the second kind, and on the right side everywhere.
//   fp16 (seven other n up to 2047): inv + rest is 127 / a to 2^-46 of it, and x inv + x rest, rounded once, exact at a tie.  Two more instructions a
//     value (18792 tokens, 8 heads of 128, keys and values alone: bf16 40.3 us that way, 38.8 with one; fp16 40.3, with one 39.1).
// (A product with the rounded reciprocal of the rounded scale sends x = a / 2, which many blocks have, to 63 or 64 as those were rounded.)  Added to
// 1.5 * 2^23 a number of at most 127 is rounded to the nearest whole number, whose low byte is the result's.  A block with Inf or NaN has the scale NaN
// and zeros (0 times either is a NaN whose low byte is 0: a 16-bit NaN has none of its bits there).
template <typename T>
struct BlockScale {
    float scale, inv, rest;
    __device__ uint32_t bits(float x) const {
        constexpr float whole = 12582912.0f;
        if constexpr (std::is_same<T, __bf16>::value) return __float_as_uint(__builtin_fmaf(x, inv, whole));
        else return __float_as_uint(__builtin_fmaf(x, inv, x * rest) + whole);
    }
    __device__ uint32_t pack(float x0, float x1, float x2, float x3) const {
        const uint32_t lo = __builtin_amdgcn_perm(bits(x1), bits(x0), 0x0c0c0400u), hi = __builtin_amdgcn_perm(bits(x3), bits(x2), 0x04000c0cu);
        return lo | hi;
    }
};
template <typename T>
__device__ inline BlockScale<T> block_scale(uint32_t bits) {
    const float a = widen<T>((uint16_t)bits), q = a / 127.0f;
    const bool finite = bits < kInf16<T>, tiny = !(q > kMinScale);
    const float inv = 127.0f / a, left = __builtin_fmaf(-inv, a, 127.0f);
    const float up = __uint_as_float(__float_as_uint(inv) + (left > 0.0f ? 1u : 0u));
    BlockScale<T> s;
    s.scale = !finite ? __uint_as_float(0x7fc00000u) : tiny ? kMinScale : q;
    s.inv = !finite ? 0.0f : tiny ? 1.0f / kMinScale : std::is_same<T, __bf16>::value ? up : inv;
    s.rest = !finite || tiny ? 0.0f : left / a;
    return s;
}

// Larger of two pairs of 16-bit numbers, each for itself.
__device__ inline uint32_t larger16x2(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(ushort2v, a), __builtin_bit_cast(ushort2v, b)));
}

// A block all of whose tokens are new, from the tensors to the cache in registers.  A thread has 16 keys of one token (a chunk of eight pairs, or 16
// values that are not turned) and eight values of four tokens in a row, whose four bytes of a value lie side by side
// in the cache: a token's eight threads write 32 bytes each of up to 8 kilobytes, eight threads the 32 bytes of a value.
template <typename T>
__device__ void compress_block(const AppendArgs &a, const Seq &s, uint32_t before, uint32_t seq, uint32_t head, uint32_t j) {
    __shared__ uint32_t s_top[kCacheBlock / kWave];
    constexpr int kMost = kCacheMaxDim / 128;              // items of a thread, at most
    const uint32_t tid = threadIdx.x, dim = a.c.dim, per_row = dim / 16u;
    const uint32_t rot = a.rope.steps ? a.rope.rot : 0u, rot_chunks = rot / 16u;
    const int32_t token0 = s.start + (int32_t)(j * kBlk - before);
    typename Vec<T, 8>::type ka[kMost], kb[kMost], v[kMost / 2][4];
    uint32_t mk = 0, mv = 0;
    const auto top_of = [](const typename Vec<T, 8>::type &x, uint32_t m) {
        const u32x4 w = __builtin_bit_cast(u32x4, x);
#pragma unroll
        for (int i = 0; i < 4; ++i) m = larger16x2(m, w[i] & 0x7fff7fffu);
        return m;
    };
    const auto first_of = [&](uint32_t c) { return c < rot_chunks ? chunk_at<8>(a.rope, c) : rot + 16u * (c - rot_chunks); };
    const auto second_of = [&](uint32_t c) { return c < rot_chunks ? chunk_second<8>(a.rope) : 8u; };
    // The first item's steps and position are asked for before its rows: loads are waited for in their order, and the sines are computed
    // while the rows are on their way.
    const uint32_t row0 = tid / per_row, c0 = tid - row0 * per_row;
    const bool turns = row0 < (uint32_t)kBlk && c0 < rot_chunks;
    uint64_t step[8];
    int32_t position = (int32_t)(j * kBlk + row0);
    if (turns) {
        if (a.rope.positions) position = a.rope.positions[token0 + (int32_t)row0];
#pragma unroll
        for (int u = 0; u < 8; ++u) step[u] = a.rope.steps[c0 * 8u + u];
    }
#pragma unroll
    for (int n = 0; n < kMost; ++n) {
        const uint32_t i = tid + n * kCacheBlock, row = i / per_row, c = i - row * per_row;
        if (row < (uint32_t)kBlk) {
            const T *p = reinterpret_cast<const T *>(a.k.p) + (int64_t)(token0 + (int32_t)row) * a.k.token + (int64_t)head * a.k.head + first_of(c);
            ka[n] = *reinterpret_cast<const typename Vec<T, 8>::type *>(p);
            kb[n] = *reinterpret_cast<const typename Vec<T, 8>::type *>(p + second_of(c));
        }
    }
#pragma unroll
    for (int n = 0; n < kMost / 2; ++n) {
        const uint32_t i = tid + n * kCacheBlock, quad = i % 8u, d = 8u * (i / 8u);
        if (d < dim) {
            const T *p = reinterpret_cast<const T *>(a.v.p) + (int64_t)(token0 + 4 * (int32_t)quad) * a.v.token + (int64_t)head * a.v.head + d;
#pragma unroll
            for (int u = 0; u < 4; ++u) v[n][u] = *reinterpret_cast<const typename Vec<T, 8>::type *>(p + u * a.v.token);
        }
    }
    const int64_t index = block_index(a.b, a.c, seq, head, j);           // (asked for behind the rows, waited for with them)
    float sn[8], cs[8];
    if (turns) {
#pragma unroll
        for (int u = 0; u < 8; ++u) turn_sincos(turn(position, step[u]), a.rope.amp, sn[u], cs[u]);
    }
#pragma unroll
    for (int n = 0; n < kMost; ++n) {
        const uint32_t i = tid + n * kCacheBlock, row = i / per_row, c = i - row * per_row;
        if (row < (uint32_t)kBlk) {
            if (c < rot_chunks) {
                float x[8], y[8];
                if (n) chunk_angles<8>(a.rope, c, a.rope.positions ? a.rope.positions[token0 + (int32_t)row] : (int32_t)(j * kBlk + row), 0u, sn, cs);
#pragma unroll
                for (int u = 0; u < 8; ++u) { x[u] = (float)ka[n][u]; y[u] = (float)kb[n][u]; }
                chunk_turn<8>(a.rope.interleaved, x, y, sn, cs);
#pragma unroll
                for (int u = 0; u < 8; ++u) { ka[n][u] = (T)x[u]; kb[n][u] = (T)y[u]; }
            }
            mk = top_of(kb[n], top_of(ka[n], mk));
        }
    }
#pragma unroll
    for (int n = 0; n < kMost / 2; ++n)
        if (8u * ((tid + n * kCacheBlock) / 8u) < dim) {
#pragma unroll
            for (int u = 0; u < 4; ++u) mv = top_of(v[n][u], mv);
        }
    uint32_t both = larger16(mk & 0xffffu, mk >> 16) | larger16(mv & 0xffffu, mv >> 16) << 16;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) both = larger16x2(both, (uint32_t)__shfl_xor((int)both, o, kWave));
    if (lane_id() == 0) s_top[tid / kWave] = both;
    __syncthreads();
#pragma unroll
    for (uint32_t w = 0; w < kCacheBlock / kWave; ++w) both = larger16x2(both, s_top[w]);
    if (index < 0) return;
    const BlockScale<T> sk = block_scale<T>(both & 0xffffu), sv = block_scale<T>(both >> 16);
    uint8_t *to = a.c.blocks + (uint64_t)index * 64u * dim;
#pragma unroll
    for (int n = 0; n < kMost; ++n) {
        const uint32_t i = tid + n * kCacheBlock, row = i / per_row, c = i - row * per_row;
        if (row < (uint32_t)kBlk) {
            const uint32_t d = first_of(c), e = d + second_of(c);
            const auto quant = [&](const typename Vec<T, 8>::type &x) {
                return uint2{sk.pack((float)x[0], (float)x[1], (float)x[2], (float)x[3]), sk.pack((float)x[4], (float)x[5], (float)x[6], (float)x[7])};
            };
            *reinterpret_cast<uint2 *>(to + d / 32u * 1024u + row * 32u + d % 32u) = quant(ka[n]);
            *reinterpret_cast<uint2 *>(to + e / 32u * 1024u + row * 32u + e % 32u) = quant(kb[n]);
        }
    }
#pragma unroll
    for (int n = 0; n < kMost / 2; ++n) {
        const uint32_t i = tid + n * kCacheBlock, quad = i % 8u, d = 8u * (i / 8u);
        if (d < dim) {
            uint8_t *at = to + 32u * dim + 32u * d + place_of(4u * quad);
#pragma unroll
            for (int k = 0; k < 8; ++k)
                *reinterpret_cast<uint32_t *>(at + 32u * k) = sv.pack((float)v[n][0][k], (float)v[n][1][k], (float)v[n][2][k], (float)v[n][3][k]);
        }
    }
    if (tid < 2u) a.c.scales[2u * (uint64_t)index + tid] = tid ? sv.scale : sk.scale;
}

}  // namespace

// Wavefronts per SIMD: four are 128 registers.  Without a bound fp16 takes 132 (18792 tokens, keys and values alone, 43.4 us instead of 40.3); bf16 stays within them by
// itself, and single tokens lose 0.3 us of 12.8 with one.
template <typename T> constexpr int kAppendWaves = 1;
template <> constexpr int kAppendWaves<_Float16> = 4;
template <typename T>
__global__ __launch_bounds__(kCacheBlock, kAppendWaves<T>) void k_cache_append(AppendArgs a) {
    extern __shared__ __align__(16) uint16_t s_rows[];
    __shared__ uint32_t s_amax[2][kBlk];
    const uint32_t tid = threadIdx.x, unit = blockIdx.x, dim = a.c.dim, pitch = dim + 8u;
    Unit found;
    if (!find_block(a.b, unit, &found)) return;
    const uint32_t seq = found.seq, j = found.block;
    const Seq s = found.s;
    const uint32_t len = (uint32_t)s.len, before = len - (uint32_t)s.n, j0 = before / kBlk;

    if (blockIdx.y >= a.c.heads) {                         // queries: the block's new tokens, some heads
        const uint32_t h0 = (blockIdx.y - a.c.heads) * a.q_heads_wg;
        const uint32_t h1 = h0 + a.q_heads_wg < a.q_heads ? h0 + a.q_heads_wg : a.q_heads;
        const uint32_t t0 = j * kBlk > before ? j * kBlk : before, t1 = j * kBlk + kBlk < len ? j * kBlk + kBlk : len;
        const uint32_t rot = a.rope.steps ? a.rope.rot : 0u;
        const auto turn_all = [&](auto v) {
            constexpr int V = decltype(v)::value;
            const uint32_t rot_chunks = rot / (2u * V), chunks = rot_chunks + (dim - rot) / V, n = t1 - t0;
            // while there are few tokens the heads are dealt out too
            uint32_t groups = kCacheBlock / (n * chunks);
            if (groups > h1 - h0) groups = h1 - h0;
            if (groups < 1u) groups = 1u;
            for (uint32_t i = tid; i < n * chunks * groups; i += kCacheBlock) {
                const uint32_t row = i / (chunks * groups), rest = i - row * (chunks * groups), g = rest / chunks, c = rest - g * chunks;
                const int32_t token = s.start + (int32_t)(t0 + row - before);
                const T *p = reinterpret_cast<const T *>(a.q.p) + (int64_t)token * a.q.token;
                T *o = reinterpret_cast<T *>(a.q_out.p) + (int64_t)token * a.q_out.token;
                float sn[V], cs[V], x[V], y[V];
                if (c < rot_chunks) chunk_angles<V>(a.rope, c, a.rope.positions ? a.rope.positions[token] : (int32_t)(t0 + row), 0u, sn, cs);
                for (uint32_t h = h0 + g; h < h1; h += groups) {
                    const T *ph = p + (int64_t)h * a.q.head;
                    T *oh = o + (int64_t)h * a.q_out.head;
                    if (c < rot_chunks) {
                        const uint32_t at = chunk_at<V>(a.rope, c), second = at + chunk_second<V>(a.rope);
                        load_row<T, V>(x, ph + at);
                        load_row<T, V>(y, ph + second);
                        chunk_turn<V>(a.rope.interleaved, x, y, sn, cs);
                        store_row<T, V>(oh + at, x);
                        store_row<T, V>(oh + second, y);
                    } else {
                        const uint32_t at = rot + (c - rot_chunks) * V;
                        load_row<T, V>(x, ph + at);
                        store_row<T, V>(oh + at, x);
                    }
                }
            }
        };
        if (a.vec) turn_all(std::integral_constant<int, 8>{});
        else turn_all(std::integral_constant<int, 1>{});
        return;
    }

    const uint32_t head = blockIdx.y;
    if (!check_slot(a.b, a.c, found.slot)) return;
    const uint32_t slot = (uint32_t)found.slot, open = len / kBlk;
    if (a.vec && j * kBlk >= before && j + 1u < open) {     // all of it is new, and the ring does not hold it: no detour
        compress_block<T>(a, s, before, seq, head, j);
        return;
    }
    uint16_t *kt = s_rows, *vt = s_rows + kBlk * pitch;
    // The ring keeps the open block and the one before it, so the length may be set back to 32 tokens below the greatest it has been.  A half that holds the
    // beginning of block j0 is overwritten by a later block of the same parity: that one is left to the workgroup
    // of j0, which reads the half first.
    const bool leads = j == j0 && before % kBlk != 0u;
    const bool mine = leads || before % kBlk == 0u || ((j ^ j0) & 1u) != 0u;
    uint32_t again = 0u;                                   // block whose rows go into the ring behind those of j0, or 0
    if (leads && j + 1u < open) again = ((open ^ j0) & 1u) ? open - 1u : open;
    if (again * kBlk >= len) again = 0u;
    for (uint32_t turn_no = 0; turn_no < (again ? 2u : 1u); ++turn_no) {
        const uint32_t jj = turn_no ? again : j;
        if (turn_no) __syncthreads();
        const uint32_t r0 = jj * kBlk < before ? before - jj * kBlk : 0u;                                      // the block's new rows
        const uint32_t r1 = len - jj * kBlk < (uint32_t)kBlk ? len - jj * kBlk : (uint32_t)kBlk;
        const bool whole = !turn_no && j < open;           // complete: the rows the ring holds are needed, too
        const int64_t index = whole ? block_index(a.b, a.c, seq, head, j) : -1;          // (asked for with the rows)
        if (a.vec) load_block<T, 8>(a, s, before, head, slot, jj, r0, r1, whole, kt, vt);
        else load_block<T, 1>(a, s, before, head, slot, jj, r0, r1, whole, kt, vt);
        __syncthreads();
        const uint32_t mine_row = tid / 8u;
        if (mine_row < r1 && (whole || mine_row >= r0)) {  // largest |value| of every token, as bits: Inf and NaN are the largest
            const uint32_t part = tid % 8u;
            uint32_t mk = 0, mv = 0;
            for (uint32_t d = 2u * part; d < dim; d += 16u) {
                const uint32_t bk = *reinterpret_cast<const uint32_t *>(kt + mine_row * pitch + d), bv = *reinterpret_cast<const uint32_t *>(vt + mine_row * pitch + d);
                mk = larger16(mk, larger16(bk & 0x7fffu, bk >> 16 & 0x7fffu));
                mv = larger16(mv, larger16(bv & 0x7fffu, bv >> 16 & 0x7fffu));
            }
#pragma unroll
            for (int o = 1; o < 8; o <<= 1) {
                mk = larger16(mk, (uint32_t)__shfl_xor((int)mk, o, kWave));
                mv = larger16(mv, (uint32_t)__shfl_xor((int)mv, o, kWave));
            }
            if (part == 0u) { s_amax[0][mine_row] = mk; s_amax[1][mine_row] = mv; }
        }
        __syncthreads();
        if (whole) {                                       // compress
            if (index >= 0) {
                uint32_t m[2] = {0u, 0u};
#pragma unroll
                for (int kind = 0; kind < 2; ++kind) {
                    uint32_t v = s_amax[kind][lane_id() % kBlk];
#pragma unroll
                    for (int o = 1; o < kBlk; o <<= 1) {
                        const uint32_t w = __shfl_xor(v, o, kWave);
                        v = w > v ? w : v;
                    }
                    m[kind] = v;
                }
                const BlockScale<T> scale[2] = {block_scale<T>(m[0]), block_scale<T>(m[1])};
                uint8_t *to = a.c.blocks + (uint64_t)index * 64u * dim;
                for (uint32_t i = tid; i < 4u * dim; i += kCacheBlock) {       // 16 bytes each: keys, then values
                    uint32_t w[4];
                    float x[16];
                    if (i < 2u * dim) {
                        const uint32_t c = i / 64u, row = (i / 2u) % 32u, h = i % 2u;
                        load_row<T, 8>(x, reinterpret_cast<const T *>(kt + row * pitch + c * 32u + h * 16u));
                        load_row<T, 8>(x + 8, reinterpret_cast<const T *>(kt + row * pitch + c * 32u + h * 16u + 8u));
                    } else {
                        const uint32_t d = (i - 2u * dim) / 2u, h = i % 2u;
#pragma unroll
                        for (int u = 0; u < 16; ++u) x[u] = widen<T>(vt[token_at(16u * h + u) * pitch + d]);
                    }
                    const BlockScale<T> of = i < 2u * dim ? scale[0] : scale[1];
#pragma unroll
                    for (int u = 0; u < 4; ++u) w[u] = of.pack(x[4 * u], x[4 * u + 1], x[4 * u + 2], x[4 * u + 3]);
                    *reinterpret_cast<u32x4 *>(to + 16u * i) = u32x4{w[0], w[1], w[2], w[3]};
                }
                if (tid < 2u) a.c.scales[2u * (uint64_t)index + tid] = tid ? scale[1].scale : scale[0].scale;
            }
        }
        if (jj + 1u >= open && (turn_no || mine)) {        // the ring: the block's new tokens
            uint8_t *half = ring_half(a.c, slot, head, jj);
            _Float16 *kr = reinterpret_cast<_Float16 *>(half), *vr = kr + 32u * dim;
            float *e = reinterpret_cast<float *>(half + 128ull * dim);
            if (tid < 64u && tid % 32u >= r0 && tid % 32u < r1) {
                const uint32_t m = s_amax[tid / 32u][tid % 32u];
                e[tid] = m >= kInf16<T> ? __uint_as_float(0x7fc00000u) : token_scale(widen<T>((uint16_t)m));
            }
            for (uint32_t i = tid; i < (r1 - r0) * dim; i += kCacheBlock) {
                const uint32_t row = r0 + i / dim, d = i % dim;
                const uint32_t mk = s_amax[0][row], mv = s_amax[1][row];
                // a token with Inf or NaN is held as zeros and a scale of NaN
                kr[(d / 32u * 32u + row) * 32u + d % 32u] = mk >= kInf16<T> ? (_Float16)0.0f
                    : (_Float16)(widen<T>(kt[row * pitch + d]) / token_scale(widen<T>((uint16_t)mk)));
                vr[d * 32u + place_of(row)] = mv >= kInf16<T> ? (_Float16)0.0f
                    : (_Float16)(widen<T>(vt[row * pitch + d]) / token_scale(widen<T>((uint16_t)mv)));
            }
        }
    }
}

template <typename T>
__global__ __launch_bounds__(kCacheBlock) void k_cache_fetch(FetchArgs a) {
    extern __shared__ __align__(16) uint16_t s_rows[];
    const uint32_t tid = threadIdx.x, unit = blockIdx.x, head = blockIdx.y, dim = a.c.dim, pitch = dim + 8u;
    Unit found;
    if (!find_block(a.b, unit, &found)) return;
    const uint32_t seq = found.seq, j = found.block;
    const Seq s = found.s;
    const uint32_t len = (uint32_t)s.len, before = len - (uint32_t)s.n;
    uint16_t *kt = s_rows, *vt = s_rows + kBlk * pitch;
    if (j < len / kBlk) {
        const int64_t index = block_index(a.b, a.c, seq, head, j);
        if (index < 0) return;
        const uint8_t *from = a.c.blocks + (uint64_t)index * 64u * dim;
        const float ks = a.c.scales[2u * (uint64_t)index], vs = a.c.scales[2u * (uint64_t)index + 1u];
        if (a.vec) {                                       // in registers, as in compress_block
            const int32_t token0 = s.start + (int32_t)(j * kBlk) - (int32_t)before;
            const uint32_t r0 = j * kBlk < before ? before - j * kBlk : 0u, per_row = dim / 16u;
            for (uint32_t i = tid; i < 2u * dim; i += kCacheBlock) {
                const uint32_t row = i / per_row, c = i - row * per_row;
                if (row < r0) continue;
                const u32x4 w = *reinterpret_cast<const u32x4 *>(from + c / 2u * 1024u + row * 32u + c % 2u * 16u);
                T *to = reinterpret_cast<T *>(a.k.p) + (int64_t)(token0 + (int32_t)row) * a.k.token + (int64_t)head * a.k.head + 16u * c;
                float x[16];
#pragma unroll
                for (int u = 0; u < 16; ++u) x[u] = (float)(int8_t)(w[u / 4] >> (8 * (u % 4))) * ks;
                store_row<T, 8>(to, x);
                store_row<T, 8>(to + 8, x + 8);
            }
            for (uint32_t i = tid; i < dim; i += kCacheBlock) {
                const uint32_t quad = i % 8u, d = i / 8u * 8u;
                const uint8_t *at = from + 32u * dim + 32u * d + place_of(4u * quad);
                uint32_t w[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) w[k] = *reinterpret_cast<const uint32_t *>(at + 32u * k);
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const uint32_t row = 4u * quad + u;
                    if (row < r0) continue;
                    float x[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[k] = (float)(int8_t)(w[k] >> (8 * u)) * vs;
                    store_row<T, 8>(reinterpret_cast<T *>(a.v.p) + (int64_t)(token0 + (int32_t)row) * a.v.token + (int64_t)head * a.v.head + d, x);
                }
            }
            return;
        }
        for (uint32_t i = tid; i < 4u * dim; i += kCacheBlock) {
            const u32x4 w = *reinterpret_cast<const u32x4 *>(from + 16u * i);
            if (i < 2u * dim) {
                const uint32_t c = i / 64u, row = (i / 2u) % 32u, h = i % 2u;
#pragma unroll
                for (int u = 0; u < 16; ++u) kt[row * pitch + c * 32u + h * 16u + u] = narrow<T>((float)(int8_t)(w[u / 4] >> (8 * (u % 4))) * ks);
            } else {
                const uint32_t d = (i - 2u * dim) / 2u, h = i % 2u;
#pragma unroll
                for (int u = 0; u < 16; ++u) vt[token_at(16u * h + u) * pitch + d] = narrow<T>((float)(int8_t)(w[u / 4] >> (8 * (u % 4))) * vs);
            }
        }
    } else {
        if (!check_slot(a.b, a.c, found.slot)) return;
        const uint8_t *half = ring_half(a.c, (uint32_t)found.slot, head, j);
        const uint16_t *kr = reinterpret_cast<const uint16_t *>(half), *vr = kr + 32u * dim;
        const float *e = reinterpret_cast<const float *>(half + 128ull * dim);
        const uint32_t r0 = j * kBlk < before ? before - j * kBlk : 0u, r1 = len - j * kBlk;        // the rows asked for
        for (uint32_t i = tid; i < (r1 - r0) * (dim / 8u); i += kCacheBlock) {
            const uint32_t row = r0 + i / (dim / 8u), d = i % (dim / 8u) * 8u;
            const half8 k = *reinterpret_cast<const half8 *>(kr + (d / 32u * 32u + row) * 32u + d % 32u);
#pragma unroll
            for (uint32_t u = 0; u < 8u; ++u) {
                kt[row * pitch + d + u] = narrow<T>((float)k[u] * e[row]);
                vt[row * pitch + d + u] = narrow<T>(widen<_Float16>(vr[(d + u) * 32u + place_of(row)]) * e[32u + row]);
            }
        }
    }
    __syncthreads();
    const auto store_all = [&](auto v) {
        constexpr int V = decltype(v)::value;
        for (uint32_t i = tid; i < kBlk * (dim / V); i += kCacheBlock) {
            const uint32_t row = i / (dim / V), d = (i - row * (dim / V)) * V, t = j * kBlk + row;
            if (t < before || t >= len) continue;
            const int64_t token = s.start + (int64_t)(t - before);
            float x[V];
            load_row<T, V>(x, reinterpret_cast<const T *>(kt + row * pitch + d));
            store_row<T, V>(reinterpret_cast<T *>(a.k.p) + token * a.k.token + (int64_t)head * a.k.head + d, x);
            load_row<T, V>(x, reinterpret_cast<const T *>(vt + row * pitch + d));
            store_row<T, V>(reinterpret_cast<T *>(a.v.p) + token * a.v.token + (int64_t)head * a.v.head + d, x);
        }
    };
    if (a.vec) store_all(std::integral_constant<int, 8>{});
    else store_all(std::integral_constant<int, 1>{});
}

template __global__ void k_cache_append<_Float16>(AppendArgs);
template __global__ void k_cache_append<__bf16>(AppendArgs);
template __global__ void k_cache_fetch<_Float16>(FetchArgs);
template __global__ void k_cache_fetch<__bf16>(FetchArgs);

}  // namespace comet
