// Keys and values into the compressed cache and out of it again.  Bound by HBM for prompts, by latency for single tokens.
#include "comet_cache.h"

namespace comet {

namespace {

template <typename T> __device__ inline float widen(uint16_t raw);
template <> __device__ inline float widen<__bf16>(uint16_t raw) { return __uint_as_float((uint32_t)raw << 16); }
template <> __device__ inline float widen<_Float16>(uint16_t raw) { return (float)__builtin_bit_cast(_Float16, raw); }
template <typename T> __device__ inline uint16_t narrow(float v) { return __builtin_bit_cast(uint16_t, (T)v); }
template <typename T> constexpr uint32_t kInf16 = 0x7f80u;              // |bits| from here on: Inf and NaN
template <> constexpr uint32_t kInf16<_Float16> = 0x7c00u;

// The new rows of a block and those the ring holds of it, in LDS: [32][dim + 8], the keys rotated and rounded to T.  The
// cache compresses the 16-bit keys that a model working in T would keep, so it does not matter in how many calls a
// block's tokens came.
template <typename T, int V>
__device__ void load_block(const AppendArgs &a, const Seq &s, uint32_t before, uint32_t head, uint32_t slot, uint32_t j, uint16_t *kt, uint16_t *vt) {
    const uint32_t dim = a.c.dim, pitch = dim + 8u, len = (uint32_t)s.len;
    const uint32_t rot = a.rope.steps ? a.rope.rot : 0u;
    const uint32_t rot_chunks = rot / (2u * V), chunks = rot_chunks + (dim - rot) / V;
    for (uint32_t i = threadIdx.x; i < kBlk * chunks; i += kCacheBlock) {
        const uint32_t row = i / chunks, c = i - row * chunks, t = j * kBlk + row;
        if (t < before || t >= len) continue;
        const int32_t token = s.start + (int32_t)(t - before);
        const T *p = reinterpret_cast<const T *>(a.k.p) + (int64_t)token * a.k.token + (int64_t)head * a.k.head;
        float x[V], y[V];
        if (c < rot_chunks) {
            float sn[V], cs[V];
            chunk_angles<V>(a.rope, c, a.rope.positions ? a.rope.positions[token] : (int32_t)t, 0u, sn, cs);
            const uint32_t at = chunk_at<V>(a.rope, c), second = at + chunk_second<V>(a.rope);
            load_row<T, V>(x, p + at);
            load_row<T, V>(y, p + second);
            chunk_turn<V>(a.rope.interleaved, x, y, sn, cs);
            store_row<T, V>(reinterpret_cast<T *>(kt + row * pitch + at), x);
            store_row<T, V>(reinterpret_cast<T *>(kt + row * pitch + second), y);
        } else {
            const uint32_t at = rot + (c - rot_chunks) * V;
            load_row<T, V>(x, p + at);
            store_row<T, V>(reinterpret_cast<T *>(kt + row * pitch + at), x);
        }
    }
    for (uint32_t i = threadIdx.x; i < kBlk * (dim / V); i += kCacheBlock) {
        const uint32_t row = i / (dim / V), d = (i - row * (dim / V)) * V, t = j * kBlk + row;
        if (t >= before && t < len) {
            const int32_t token = s.start + (int32_t)(t - before);
            float x[V];
            load_row<T, V>(x, reinterpret_cast<const T *>(a.v.p) + (int64_t)token * a.v.token + (int64_t)head * a.v.head + d);
            store_row<T, V>(reinterpret_cast<T *>(vt + row * pitch + d), x);
        } else if (t < before) {
            const uint8_t *half = ring_half(a.c, slot, head, j);
            const uint16_t *kr = reinterpret_cast<const uint16_t *>(half), *vr = kr + 32u * dim;
            const float *e = reinterpret_cast<const float *>(half + 128ull * dim);
#pragma unroll
            for (int u = 0; u < V; ++u) {
                const uint32_t dd = d + u;
                kt[row * pitch + dd] = narrow<T>(widen<_Float16>(kr[(dd / 32u * 32u + row) * 32u + dd % 32u]) * e[row]);
                vt[row * pitch + dd] = narrow<T>(widen<_Float16>(vr[dd * 32u + place_of(row)]) * e[32u + row]);
            }
        } else {
#pragma unroll
            for (int u = 0; u < V; ++u) kt[row * pitch + d + u] = vt[row * pitch + d + u] = 0;
        }
    }
}

// Power of two by which a token's values are divided on their way into float16: the largest then lies in [2^14, 2^15),
// and only what is 2^-39 of it and less loses bits.
__device__ inline float token_scale(float amax) {
    uint32_t e = __float_as_uint(amax) >> 23;
    if (e < 15u) e = 15u;
    return __uint_as_float((e - 14u) << 23);
}

}  // namespace

template <typename T>
__global__ __launch_bounds__(kCacheBlock) void k_cache_append(AppendArgs a) {
    extern __shared__ __align__(16) uint16_t s_rows[];
    __shared__ uint32_t s_amax[2][kBlk];
    const uint32_t tid = threadIdx.x, unit = blockIdx.x, dim = a.c.dim, pitch = dim + 8u;
    const uint32_t seq = find_sequence(a.b.starts, a.b.n_seqs, unit, 1u, 5u, 2u);
    Seq s;
    if (!read_sequence(a.b, seq, &s)) return;
    const uint32_t first = first_unit(a.b.starts, seq, 1u, 5u, 2u);
    if (unit < first) return;
    if (s.len < s.n) {
        raise(a.b.status);
        return;
    }
    const uint32_t len = (uint32_t)s.len, before = len - (uint32_t)s.n, j0 = before / kBlk, j = j0 + (unit - first);
    if (j > (len - 1u) / kBlk) return;

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
    uint32_t slot;
    if (!read_slot(a.b, a.c, seq, &slot)) return;
    uint16_t *kt = s_rows, *vt = s_rows + kBlk * pitch;
    const uint32_t open = len / kBlk;
    // The ring keeps the open block and the one before it, so the length may be set back by up to a block.  A half that holds the
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
        if (a.vec) load_block<T, 8>(a, s, before, head, slot, jj, kt, vt);
        else load_block<T, 1>(a, s, before, head, slot, jj, kt, vt);
        __syncthreads();
        {                                                  // largest |value| of every token, as bits: Inf and NaN are the largest
            const uint32_t row = tid / 8u, part = tid % 8u, per = dim / 8u;
            uint32_t mk = 0, mv = 0;
            for (uint32_t d = part * per; d < (part + 1u) * per; ++d) {
                const uint32_t bk = kt[row * pitch + d] & 0x7fffu, bv = vt[row * pitch + d] & 0x7fffu;
                mk = bk > mk ? bk : mk;
                mv = bv > mv ? bv : mv;
            }
#pragma unroll
            for (int o = 1; o < 8; o <<= 1) {
                const uint32_t ok = __shfl_xor(mk, o, kWave), ov = __shfl_xor(mv, o, kWave);
                mk = ok > mk ? ok : mk;
                mv = ov > mv ? ov : mv;
            }
            if (part == 0u) { s_amax[0][row] = mk; s_amax[1][row] = mv; }
        }
        __syncthreads();
        if (!turn_no && j < open) {                        // complete: compress
            const int64_t index = block_index(a.b, a.c, seq, head, j);
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
                float scale[2], inv[2];
#pragma unroll
                for (int kind = 0; kind < 2; ++kind) {
                    const float q = widen<T>((uint16_t)m[kind]) / 127.0f;
                    scale[kind] = m[kind] >= kInf16<T> ? __uint_as_float(0x7fc00000u) : (q > kMinScale ? q : kMinScale);
                    inv[kind] = m[kind] >= kInf16<T> ? 0.0f : 1.0f / scale[kind];
                }
                const auto to8 = [](float x, float f) -> uint32_t {
                    const float y = __builtin_rintf(x * f);
                    return f == 0.0f ? 0u : (uint32_t)(int32_t)(y > 127.0f ? 127.0f : (y < -127.0f ? -127.0f : y)) & 0xffu;
                };
                uint8_t *to = a.c.blocks + (uint64_t)index * 64u * dim;
                for (uint32_t i = tid; i < 4u * dim; i += kCacheBlock) {       // 16 bytes each: keys, then values
                    uint32_t w[4] = {0u, 0u, 0u, 0u};
                    if (i < 2u * dim) {
                        const uint32_t c = i / 64u, row = (i / 2u) % 32u, h = i % 2u;
                        const uint16_t *p = kt + row * pitch + c * 32u + h * 16u;
#pragma unroll
                        for (int u = 0; u < 16; ++u) w[u / 4] |= to8(widen<T>(p[u]), inv[0]) << (8 * (u % 4));
                    } else {
                        const uint32_t d = (i - 2u * dim) / 2u, h = i % 2u;
#pragma unroll
                        for (int u = 0; u < 16; ++u) w[u / 4] |= to8(widen<T>(vt[token_at(16u * h + u) * pitch + d]), inv[1]) << (8 * (u % 4));
                    }
                    *reinterpret_cast<u32x4 *>(to + 16u * i) = u32x4{w[0], w[1], w[2], w[3]};
                }
                if (tid < 2u) a.c.scales[2u * (uint64_t)index + tid] = scale[tid];
            }
        }
        if (jj + 1u >= open && (turn_no || mine)) {        // the ring: the block's new tokens
            uint8_t *half = ring_half(a.c, slot, head, jj);
            _Float16 *kr = reinterpret_cast<_Float16 *>(half), *vr = kr + 32u * dim;
            float *e = reinterpret_cast<float *>(half + 128ull * dim);
            const uint32_t r0 = jj * kBlk < before ? before - jj * kBlk : 0u;
            const uint32_t r1 = len - jj * kBlk < (uint32_t)kBlk ? len - jj * kBlk : (uint32_t)kBlk;
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
    const uint32_t seq = find_sequence(a.b.starts, a.b.n_seqs, unit, 1u, 5u, 2u);
    Seq s;
    if (!read_sequence(a.b, seq, &s)) return;
    const uint32_t first = first_unit(a.b.starts, seq, 1u, 5u, 2u);
    if (unit < first) return;
    if (s.len < s.n) {
        raise(a.b.status);
        return;
    }
    const uint32_t len = (uint32_t)s.len, before = len - (uint32_t)s.n, j = before / kBlk + (unit - first);
    if (j > (len - 1u) / kBlk) return;
    uint16_t *kt = s_rows, *vt = s_rows + kBlk * pitch;
    if (j < len / kBlk) {
        const int64_t index = block_index(a.b, a.c, seq, head, j);
        if (index < 0) return;
        const uint8_t *from = a.c.blocks + (uint64_t)index * 64u * dim;
        const float ks = a.c.scales[2u * (uint64_t)index], vs = a.c.scales[2u * (uint64_t)index + 1u];
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
        uint32_t slot;
        if (!read_slot(a.b, a.c, seq, &slot)) return;
        const uint8_t *half = ring_half(a.c, slot, head, j);
        const uint16_t *kr = reinterpret_cast<const uint16_t *>(half), *vr = kr + 32u * dim;
        const float *e = reinterpret_cast<const float *>(half + 128ull * dim);
        for (uint32_t i = tid; i < kBlk * dim; i += kCacheBlock) {
            const uint32_t row = i / dim, d = i % dim;
            kt[row * pitch + d] = narrow<T>(widen<_Float16>(kr[(d / 32u * 32u + row) * 32u + d % 32u]) * e[row]);
            vt[row * pitch + d] = narrow<T>(widen<_Float16>(vr[d * 32u + place_of(row)]) * e[32u + row]);
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
