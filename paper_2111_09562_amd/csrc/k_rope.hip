// Rotary positions: every pair of a head's rotated part is turned by its position times the pair's step.  The gradient is the
// same rotation the other way, so the backward pass needs the positions and nothing of the forward pass.
// Bound by HBM: 16 bytes a lane and access, neighbouring lanes on neighbouring chunks of a head; a chunk's sines are computed once for up to eight
// heads.  16384 x 32 x 128 bf16: 56 us, 4.8 TB/s; 4099 x 20 x 96 fp32, 64 of them side by side: 12.2 us, 5.2 TB/s; 16 tokens: 3.5 us, a launch.
#include "comet_cache.h"

namespace comet {

template <typename T, int V>
__global__ __launch_bounds__(kRopeBlock) void k_rope(RopeArgs r, RopeGrid g, Rows x, Rows y, uint32_t n_tokens, uint32_t heads, uint32_t dim,
                                                     uint32_t sign) {
    const uint32_t tid = threadIdx.x;
    const uint32_t local = g.tokens_wg ? tid / g.per_token : 0u;
    const uint32_t tokens_wg = g.tokens_wg ? g.tokens_wg : 1u;
    if (local >= tokens_wg) return;
    for (uint64_t token = (uint64_t)blockIdx.x * tokens_wg + local; token < n_tokens; token += (uint64_t)gridDim.x * tokens_wg) {
        const int32_t position = r.positions ? r.positions[token] : (int32_t)token;
        const T *px = reinterpret_cast<const T *>(x.p) + (int64_t)token * x.token;
        T *py = reinterpret_cast<T *>(y.p) + (int64_t)token * y.token;
        for (uint32_t i = tid - local * g.per_token; i < g.per_token; i += g.tokens_wg ? g.per_token : (uint32_t)kRopeBlock) {
            const uint32_t group = i / g.chunks, c = i - group * g.chunks;
            if (c < g.rot_chunks) {
                float sn[V], cs[V];
                chunk_angles<V>(r, c, position, sign, sn, cs);
                const uint32_t at = chunk_at<V>(r, c), second = at + chunk_second<V>(r);
                for (uint32_t h = group; h < heads; h += g.groups) {
                    float a[V], b[V];
                    load_row<T, V>(a, px + h * x.head + at);
                    load_row<T, V>(b, px + h * x.head + second);
                    chunk_turn<V>(r.interleaved, a, b, sn, cs);
                    store_row<T, V>(py + h * y.head + at, a);
                    store_row<T, V>(py + h * y.head + second, b);
                }
            } else {
                const uint32_t at = r.rot + (c - g.rot_chunks) * V;
                for (uint32_t h = group; h < heads; h += g.groups) {
                    float a[V];
                    load_row<T, V>(a, px + h * x.head + at);
                    store_row<T, V>(py + h * y.head + at, a);
                }
            }
        }
    }
}

template __global__ void k_rope<float, 4>(RopeArgs, RopeGrid, Rows, Rows, uint32_t, uint32_t, uint32_t, uint32_t);
template __global__ void k_rope<float, 1>(RopeArgs, RopeGrid, Rows, Rows, uint32_t, uint32_t, uint32_t, uint32_t);
template __global__ void k_rope<_Float16, 8>(RopeArgs, RopeGrid, Rows, Rows, uint32_t, uint32_t, uint32_t, uint32_t);
template __global__ void k_rope<_Float16, 1>(RopeArgs, RopeGrid, Rows, Rows, uint32_t, uint32_t, uint32_t, uint32_t);
template __global__ void k_rope<__bf16, 8>(RopeArgs, RopeGrid, Rows, Rows, uint32_t, uint32_t, uint32_t, uint32_t);
template __global__ void k_rope<__bf16, 1>(RopeArgs, RopeGrid, Rows, Rows, uint32_t, uint32_t, uint32_t, uint32_t);

}  // namespace comet
