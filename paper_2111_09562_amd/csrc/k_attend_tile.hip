// Attention over the compressed cache: many rows (prompts).
#include "comet_attend.h"

namespace comet {

namespace {
// Puts the N matrix instructions of a stage between the vector instructions of its weights, some 80 of them, which must not move to
// the next stage (where alone they are needed).
template <int N, int PER>
__device__ inline void interleave(half8 *p, float &l) {
    asm volatile("" : "+v"(p[0]), "+v"(p[1]), "+v"(l));
#pragma unroll
    for (int i = 0; i < N; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);               // one matrix instruction
        __builtin_amdgcn_sched_group_barrier(0x402, PER, 0);             // vector instructions
    }
}
}  // namespace

// Many rows: the four wavefronts of a workgroup hold 32 * RT rows each and go through the same blocks together.  Every block is converted to
// float16 once per workgroup, in LDS, in the order of the operands (lane l's 16 bytes at 16 l: no bank conflicts).  Bound by the
// matrix instructions and by the vector instructions of the weights, about as many cycles of each for heads of 128.
// So with two tiles of rows per wavefront (A, B) the products of one are issued between the weights of the other:
//   A's weights of block j with  O_B += V(j-1) p_B  and  s_B = K(j) q_B;   B's weights with  O_A += V(j) p_A  and  s_A = K(j+1) q_A.
// The operands stay in registers for both tiles, which halves what is read from LDS.  One tile per wavefront (RT = 1): the next block's s beside the weights,
// then the values; the operands of the block after that are read meanwhile.
// 8 x 4 heads of 128, 4096 tokens behind 28672: RT = 2 2.12 ms (970 TFLOP/s; 797 when products and weights came one after another), RT = 1 2.32 ms; prompts of 582
// to 1966 tokens: RT = 1 103 us, with the join 106, RT = 2 126.  16 heads of 256 on one of keys, 2048 tokens behind 30720: 1.18 ms, 905 TFLOP/s (8192^3 products
// of the library: 1220 .. 1270).  Heads of 64, 4096 behind 28672: 710 TFLOP/s, the exponentials.
template <int NC, int RT>
__global__ __launch_bounds__(kAttendBlock, tile_pairs(NC, RT) ? 2 : 1) void k_attend_tile(AttendArgs a) {
    constexpr uint32_t dim = 32u * NC, rows_wave = 32u * RT, rows_wg = 4u * rows_wave;
    __shared__ __align__(16) uint8_t s_kv[2][2][64u * dim];           // [keys, values][block & 1][c][u][lane][16 bytes]
    const uint32_t lane = (uint32_t)lane_id(), wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave)), n = lane & 31u, h = lane >> 5;
    const uint32_t number = blockIdx.x / a.c.heads, head = blockIdx.x - number * a.c.heads;
    Piece p;
    if (!find_piece(a, number, &p)) return;
    const Seq s = p.s;
    int32_t least, most;
    row_limits(a, s, p.tile * rows_wg, rows_wg, &least, &most);
    const uint32_t seen = most > 0 ? ((uint32_t)most + 31u) / 32u : 0u, parts = parts_of(seen, p.per);
    if (p.part >= parts || (parts > 1u && p.slot >= a.slots)) return;     // (more slots than there are: numbers that make no sense)
    const uint32_t j0 = (uint32_t)((uint64_t)seen * p.part / parts), j1 = (uint32_t)((uint64_t)seen * (p.part + 1u) / parts);
    const uint32_t whole = (uint32_t)s.len / 32u;
    const uint32_t row0 = p.tile * rows_wg + wave * rows_wave;
    RowPlace place[RT];
    half8 q[RT][2 * NC];
    float qc[RT];
    QueryRaw<8 * NC> raw[RT];
    RowState<NC, f32x16, 32> row[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        place[rt] = row_place(a, s, head, row0 + 32u * rt + n);
        request_query<NC, 16>(a, place[rt], 16u * h, &raw[rt]);
        row[rt].clear();
    }

    // A wavefront converts the kilobytes wave, wave + 4, .. of a block's keys and as many of its values.
    constexpr int kShare = (NC + 3) / 4;
    const auto fetch = [&](u32x4 *to, int64_t at, uint32_t which) {
        const uint8_t *from = a.c.blocks + (uint64_t)at * (64u * dim) + which * 32u * dim + n * 32u + h * 16u;
#pragma unroll
        for (int i = 0; i < kShare; ++i)
            if (4 * i + 3 < NC || wave + 4u * i < (uint32_t)NC) to[i] = *reinterpret_cast<const u32x4 *>(from + (wave + 4u * i) * 1024u);
    };
    const auto stage = [&](const u32x4 *from, uint32_t which, uint32_t buf) {
#pragma unroll
        for (int i = 0; i < kShare; ++i)
            if (4 * i + 3 < NC || wave + 4u * i < (uint32_t)NC) {
                uint8_t *to = &s_kv[which][buf][(wave + 4u * i) * 2048u + 16u * lane];
                *reinterpret_cast<half8 *>(to) = whole8(from[i][0], from[i][1]);
                *reinterpret_cast<half8 *>(to + 1024) = whole8(from[i][2], from[i][3]);
            }
    };
    const auto operands = [&](half8 *to, uint32_t which, uint32_t buf) {
#pragma unroll
        for (int c = 0; c < 2 * NC; ++c) to[c] = *reinterpret_cast<const half8 *>(&s_kv[which][buf][1024u * c + 16u * lane]);
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
        return row_max<32>(best);
    };

    uint32_t j = j0;
    const uint32_t end = j1 < whole ? j1 : whole;                        // complete blocks of this piece
    uint32_t fast = least > 0 ? (uint32_t)least / 32u : 0u;             // ... that every row sees whole
    fast = fast < end ? fast : end;
    int32_t low, high;
    row_limits(a, s, row0, rows_wave, &low, &high);
    const bool opens = j1 > whole;                                        // the open block is the last of this piece
    uint32_t slot = 0;
    const bool has_slot = opens && read_slot(a.b, a.c, p.seq, &slot);
    const uint8_t *half = ring_half(a.c, slot, head, whole);
    Lookup look;
    look.get(a, p.seq, head, j + lane, end);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) qc[rt] = convert_query<32>(a, raw[rt], q[rt]) * a.scale;

    while (j < end) {
        const uint32_t count = end - j < 64u ? end - j : 64u;
        // In step i the keys of block i + 2 and the values of block i + 1 come into LDS, in the place of what was read before a barrier that every
        // wavefront has passed since: that of step i - 1, or, for what is read in front of step 0, the one behind that read.  Behind the last block it
        // is staged again, and not used.
        const auto at = [&](uint32_t i) {
            const int64_t index = look.index_of(i < count ? i : count - 1u);
            return index < 0 ? 0 : index;
        };
        u32x4 rk[kShare], rv[kShare];
        fetch(rk, at(0), 0);
        fetch(rv, at(0), 1);
        u32x4 rk1[kShare];
        fetch(rk1, at(1), 0);
        __syncthreads();                                               // (the batch before is done with the buffers)
        stage(rk, 0, 0);
        stage(rv, 1, 0);
        stage(rk1, 0, 1);
        fetch(rk, at(2), 0);
        fetch(rv, at(1), 1);
        __syncthreads();
        // Blocks that all rows see whole, until one is missing or poisoned.
        uint32_t n_fast = fast > j ? (fast - j < count ? fast - j : count) : 0u;
        const uint64_t bad = wave_ballot(lane < n_fast && (look.index < 0 || look.lb != look.lb));
        if (bad) n_fast = (uint32_t)__ffsll((unsigned long long)bad) - 1u;
        uint32_t i = 0;
        if (n_fast) {
            half8 kk[2 * NC], vv[2 * NC], pa[2] = {}, pb[2] = {};
            operands(kk, 0, 0);
            f32x16 sa = products(kk, 0), sb = {};
            __syncthreads();                                           // (step 0 puts the keys of block 2 where these were)
            if constexpr (RT == 1) operands(kk, 0, 1);
#pragma unroll
            for (int c = 0; c < 2 * NC; ++c) vv[c] = half8{};
            for (; i < n_fast; ++i) {
                const uint32_t buf = i & 1u;
                if constexpr (!tile_pairs(NC, RT)) {                           // the queries in accumulation registers, which only matrix instructions read
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                        for (int c = 0; c < 2 * NC; ++c) asm volatile("" : "+a"(q[rt][c]));
                }
                const float ks = Lookup::of(look.ks, i), lb = Lookup::of(look.lb, i);
                const auto next = [&] {
                    stage(rk, 0, buf);
                    stage(rv, 1, buf ^ 1u);
                    fetch(rk, at(i + 3u), 0);
                    fetch(rv, at(i + 2u), 1);
                };
                const float kc = ks * qc[0], top = largest(sa) * kc;
                row[0].follow(top, top + lb);
                if constexpr (RT == 2) {
                    accumulate(vv, 1, pb);
                    sb = products(kk, 1);
                    row[0].weights(sa, kc, lb, pa);
                    if constexpr (!tile_pairs(NC, RT)) interleave<4 * NC, 20 / NC>(pa, row[0].l);
                    operands(vv, 1, buf);
                    operands(kk, 0, buf ^ 1u);
                    next();
                    const float kd = ks * qc[1], top1 = largest(sb) * kd;
                    row[1].follow(top1, top1 + lb);
                    accumulate(vv, 0, pa);
                    sa = products(kk, 0);
                    row[1].weights(sb, kd, lb, pb);
                    if constexpr (!tile_pairs(NC, RT)) interleave<4 * NC, 20 / NC>(pb, row[1].l);
                } else {
                    operands(vv, 1, buf);
                    sb = products(kk, 0);
                    row[0].weights(sa, kc, lb, pa);
                    if constexpr (!tile_pairs(NC, RT)) interleave<2 * NC, 32 / NC>(pa, row[0].l);
                    next();
                    __syncthreads();
                    operands(kk, 0, buf);                                  // of block i + 2, while the values are multiplied
                    accumulate(vv, 0, pa);
                    sa = sb;
                }
                if constexpr (RT == 2) __syncthreads();
            }
            if constexpr (RT == 2) accumulate(vv, 1, pb);
        }
        // The others one after another: blocks of which rows see parts, missing and poisoned ones.  Here the keys of block i + 2 take the
        // place of those of block i, which are read in this step, so they are staged behind the barrier.
        for (; i < count; ++i) {
            const uint32_t buf = i & 1u, jj = j + i;
            if (look.index_of(i) >= 0 && (int32_t)(jj * 32u) < high) {                  // (else nothing in it for this wavefront's rows)
                const float ks = Lookup::of(look.ks, i), lb = Lookup::of(look.lb, i);
                half8 op[2 * NC], pw[RT][2];
                operands(op, 0, buf);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    const f32x16 acc = products(op, rt);
                    float x[16], top, tope;
                    some_of_block<32>(acc, ks * qc[rt], lb, jj, place[rt].limit, x, &top, &tope);
                    row[rt].follow(top, tope);
                    row[rt].weights_some(x, lb, pw[rt]);
                }
                operands(op, 1, buf);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) accumulate(op, rt, pw[rt]);
            }
            stage(rv, 1, buf ^ 1u);
            __syncthreads();
            stage(rk, 0, buf);
            fetch(rk, at(i + 3u), 0);
            fetch(rv, at(i + 2u), 1);
        }
        j += count;
        if (j < end) look.get(a, p.seq, head, j + lane, end);
    }

    // the open block, in 16 bits
    if (has_slot) {
        const uint32_t held = (uint32_t)s.len % 32u;
        __syncthreads();
        for (uint32_t i = wave; i < 2u * NC; i += 4u) {
            const uint8_t *from = half + 2048u * i + 64u * n + 32u * h;
            uint8_t *to = &s_kv[i < (uint32_t)NC ? 0 : 1][0][2048u * (i < (uint32_t)NC ? i : i - NC) + 16u * lane];
#pragma unroll
            for (uint32_t u = 0; u < 2u; ++u)
                *reinterpret_cast<half8 *>(to + 1024u * u) = i < (uint32_t)NC ? *reinterpret_cast<const half8 *>(from + 16u * u) : open_values(from + 16u * u, u, held);
        }
        __syncthreads();
        if ((int32_t)(whole * 32u) < high) {
            half8 op[2 * NC], pw[RT][2];
            operands(op, 0, 0);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const f32x16 acc = products(op, rt);
                float x[16], lv[16], top, tope;
                each_of_open<32>(acc, qc[rt], reinterpret_cast<const float *>(half + 128ull * dim), held, whole, place[rt].limit, x, lv, &top, &tope);
                row[rt].follow(top, tope);
                row[rt].weights_each(x, lv, pw[rt]);
            }
            operands(op, 1, 0);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) accumulate(op, rt, pw[rt]);
        }
    }

    if (p.part == 0u && head == 0u && threadIdx.x == 0u) {
        int32_t *dir = a.directory + 2u * (first_unit(a.b.starts, p.seq, a.group, a.tile_shift, 1u) + p.tile);
        dir[0] = (int32_t)p.slot;
        dir[1] = (int32_t)parts;
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const auto &r = row[rt];
        const float l = row_sum<32>(r.l);
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
            const uint64_t slot_no = ((uint64_t)p.slot * a.c.heads + head) * rows_wg + wave * rows_wave + 32u * rt + n;
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

template __global__ void k_attend_tile<1, 2>(AttendArgs);
template __global__ void k_attend_tile<2, 2>(AttendArgs);
template __global__ void k_attend_tile<3, 1>(AttendArgs);
template __global__ void k_attend_tile<3, 2>(AttendArgs);
template __global__ void k_attend_tile<4, 1>(AttendArgs);
template __global__ void k_attend_tile<4, 2>(AttendArgs);
template __global__ void k_attend_tile<5, 1>(AttendArgs);
template __global__ void k_attend_tile<6, 1>(AttendArgs);
template __global__ void k_attend_tile<7, 1>(AttendArgs);
template __global__ void k_attend_tile<8, 1>(AttendArgs);

}  // namespace comet
