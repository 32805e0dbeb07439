// Attention over the compressed cache: few rows, and what joins the pieces of a row.
#include "comet_attend.h"

namespace comet {

// Few rows: a wavefront holds 32 rows (queries of one key/value head, its group's heads side by side) and goes through every fourth
// block of its workgroup's piece straight from memory into the operands of the matrix instruction, with no LDS and no barrier
// in the loop.  Bound by HBM and the conversion to float16 together (64 sequences of 400 to 16384 tokens, 8 heads of 128, 32 rows each: 118 us,
// 4.5 TB/s).
// EXACT: what rounding the weights to float16 leaves is multiplied as well, for results in float16, as in k_attend_few (with the join,
// the same sequences 161 us, 156 without; 48 sequences of up to 4096 tokens, 12 heads of 64, 20 rows each 39 us and 37).
// grid: heads * pieces workgroups of kAttendBlock threads, the heads of a piece side by side
template <int NC, bool EXACT>
__global__ __launch_bounds__(kAttendBlock, NC <= 4 ? 2 : 1) void k_attend(AttendArgs a) {
    constexpr uint32_t dim = 32u * NC;
    __shared__ float s_stat[4][3][32];
    __shared__ __align__(16) float s_tile[4][1024];
    const uint32_t lane = (uint32_t)lane_id(), wave = threadIdx.x / kWave, n = lane & 31u, h = lane >> 5;
    const uint32_t number = blockIdx.x / a.c.heads, head = blockIdx.x - number * a.c.heads;
    Piece p;
    if (!find_piece(a, number, &p)) return;
    const Seq s = p.s;
    const RowPlace place = row_place(a, s, head, p.tile * 32u + n);
    int32_t least, most;
    row_limits(a, s, p.tile * 32u, 32u, &least, &most);
    const uint32_t seen = most > 0 ? ((uint32_t)most + 31u) / 32u : 0u, parts = parts_of(seen, p.per);
    if (p.part >= parts || (parts > 1u && p.slot >= a.slots)) return;     // (more slots than there are: numbers that make no sense)
    const uint32_t j0 = (uint32_t)((uint64_t)seen * p.part / parts), j1 = (uint32_t)((uint64_t)seen * (p.part + 1u) / parts);
    const uint32_t whole = (uint32_t)s.len / 32u;                                             // complete blocks

    QueryRaw<8 * NC> raw;
    request_query<NC, 16>(a, place, 16u * h, &raw);
    RowState<NC, f32x16, 32> row;
    row.clear();

    // the wavefront's blocks: j0 + wave, j0 + wave + 4, ...; where they lie is looked up for 64 of them at a time
    uint32_t j = j0 + wave;
    const uint32_t end = j1 < whole ? j1 : whole;
    u32x4 kr[NC], vr[NC];
    const auto load = [&](u32x4 *to, int64_t at, uint32_t which) {
        const uint8_t *from = a.c.blocks + (uint64_t)(at < 0 ? 0 : at) * (64u * dim) + which * (32u * dim) + n * 32u + h * 16u;
#pragma unroll
        for (int c = 0; c < NC; ++c) to[c] = *reinterpret_cast<const u32x4 *>(from + c * 1024);
    };
    Lookup look;
    look.request(a, p.seq, head, j + 4u * lane, end);
    int64_t at = look.index_of(0);
    if (j < end) {
        load(kr, at, 0u);
        load(vr, at, 1u);
    }
    half8 q[2 * NC];
    const float qc = convert_query<32>(a, raw, q) * a.scale;
    look.finish();
    while (j < end) {
        const uint32_t left = (end - j + 3u) / 4u, count = left < 64u ? left : 64u;
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
            half8 pw[2], rest[2] = {};
            // (one place that moves the references, and x once more behind it: two such places cost a hundred registers)
            const bool all = at >= 0 && (int32_t)(j * 32u + 32u) <= least && lb == lb;
            const int32_t limit = at >= 0 ? place.limit : 0;
            float top, tope;
            if (all) {
                float best = acc[0];
#pragma unroll
                for (int t = 1; t < 16; ++t) best = fmaxf(best, acc[t]);
                top = row_max<32>(best) * kc;
                tope = top + lb;
            } else {
                float x[16];
                some_of_block<32>(acc, kc, lb, j, limit, x, &top, &tope);
            }
            row.follow(top, tope);
            if (all) {
                row.weights(acc, kc, lb, pw, EXACT ? rest : nullptr);
            } else {
                float x[16];
                some_of_block<32>(acc, kc, lb, j, limit, x, &top, &tope);
                row.weights_some(x, lb, pw, EXACT ? rest : nullptr);
            }
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const half8 v0 = whole8(vr[c][0], vr[c][1]), v1 = whole8(vr[c][2], vr[c][3]);
                row.o[c] = mfma(v0, pw[0], row.o[c]);
                row.o[c] = mfma(v1, pw[1], row.o[c]);
                if constexpr (EXACT) {
                    row.o[c] = mfma(v0, rest[0], row.o[c]);
                    row.o[c] = mfma(v1, rest[1], row.o[c]);
                }
            }
            if (next >= 0) load(vr, next, 1u);
            at = next;
        }
        if (j < end) {
            look.get(a, p.seq, head, j + 4u * lane, end);
            at = look.index_of(0);
            load(kr, at, 0u);
            load(vr, at, 1u);
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
            each_of_open<32>(acc, qc, reinterpret_cast<const float *>(half + 128ull * dim), held, j, place.limit, x, lv, &top, &tope);
            row.follow(top, tope);
            half8 pw[2], rest[2];
            row.weights_each(x, lv, pw, EXACT ? rest : nullptr);
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const half8 v = open_values(half + 64u * dim + 2048u * c + 64u * n + 32u * h + 16u * u, u, held);
                    row.o[c] = mfma(v, pw[u], row.o[c]);
                    if constexpr (EXACT) row.o[c] = mfma(v, rest[u], row.o[c]);
                }
        }
    }

    // The four wavefronts' results in one, in their order.
    row.l = row_sum<32>(row.l);
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
    const uint64_t slot_no = ((uint64_t)p.slot * a.c.heads + head) * 32u;
    if (wave == 0u && h == 0u) {
        if (last) {
            if (place.real && a.lse) a.lse[place.token * a.q_heads + place.qh] = log_sum(mms, ll);
        } else {
            float *st = a.part_s + 3u * (slot_no + n);
            st[0] = mm; st[1] = ll; st[2] = rr;
        }
        if (p.part == 0u && head == 0u && n == 0u) {
            int32_t *dir = a.directory + 2u * (first_unit(a.b.starts, p.seq, a.group, a.tile_shift, 1u) + p.tile);
            dir[0] = (int32_t)p.slot;
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

// Fewer still: the same with tiles of 16 rows, half the registers and so twice the wavefronts and loads in flight.  Bound by HBM: the same sequences,
// 4 rows each, 106 us (5.0 TB/s), two of 120000 tokens 91 us (5.4 TB/s; a large copy reaches 5.1); one of 701 tokens 7.5 us, a chain of memory round trips.
// EXACT: what rounding the weights to float16 leaves is multiplied as well, for results in float16 (whose own rounding is no larger: together 1.45 times
// the error of one; the second product hides behind the loads).
template <int NC, bool EXACT>
__global__ __launch_bounds__(kAttendBlock, NC <= 3 ? 4 : NC <= 5 ? 3 : 2) void k_attend_few(AttendArgs a) {
    constexpr uint32_t dim = 32u * NC;
    __shared__ float s_stat[4][3][16];
    __shared__ __align__(16) float s_tile[4][1024];
    const uint32_t lane = (uint32_t)lane_id(), wave = threadIdx.x / kWave, n = lane & 15u, g = lane >> 4;
    const uint32_t number = blockIdx.x / a.c.heads, head = blockIdx.x - number * a.c.heads;
    Piece p;
    if (!find_piece(a, number, &p)) return;
    const Seq s = p.s;
    const RowPlace place = row_place(a, s, head, p.tile * 16u + n);
    int32_t least, most;
    row_limits(a, s, p.tile * 16u, 16u, &least, &most);
    const uint32_t seen = most > 0 ? ((uint32_t)most + 31u) / 32u : 0u, parts = parts_of(seen, p.per);
    if (p.part >= parts || (parts > 1u && p.slot >= a.slots)) return;     // (more slots than there are: numbers that make no sense)
    const uint32_t j0 = (uint32_t)((uint64_t)seen * p.part / parts), j1 = (uint32_t)((uint64_t)seen * (p.part + 1u) / parts);
    const uint32_t whole = (uint32_t)s.len / 32u;                                             // complete blocks

    // of 32 values of the head a lane's operands have the eight from `chunk` on
    const uint32_t chunk = 16u * (g & 1u) + 8u * (g >> 1);
    QueryRaw<4 * NC> raw;
    request_query<NC, 8>(a, place, chunk, &raw);
    RowState<2 * NC, f32x4, 16> row;
    row.clear();

    // the wavefront's blocks: j0 + wave, j0 + wave + 4, ...; where they lie is looked up for 64 of them at a time
    uint32_t j = j0 + wave;
    const uint32_t end = j1 < whole ? j1 : whole;
    u32x4 kr[NC], vr[NC];
    const auto load = [&](u32x4 *to, int64_t at, uint32_t which) {
        const uint8_t *from = a.c.blocks + (uint64_t)(at < 0 ? 0 : at) * (64u * dim) + which * (32u * dim) + n * 32u + (g >> 1) * 512u + (g & 1u) * 16u;
#pragma unroll
        for (int c = 0; c < NC; ++c) to[c] = *reinterpret_cast<const u32x4 *>(from + c * 1024);
    };
    Lookup look;
    look.request(a, p.seq, head, j + 4u * lane, end);
    int64_t at = look.index_of(0);
    if (j < end) {
        load(kr, at, 0u);
        load(vr, at, 1u);
    }
    half8 q[NC];
    const float qc = convert_query<16>(a, raw, q) * a.scale;
    look.finish();
    while (j < end) {
        const uint32_t left = (end - j + 3u) / 4u, count = left < 64u ? left : 64u;
        for (uint32_t i = 0; i < count; ++i, j += 4u) {
            const int64_t next = i + 1u < count ? look.index_of(i + 1u) : -1;
            // Lane l has loaded 16 values of one token (l & 15, 16 more in the upper half of the wavefront), the instruction wants eight of the token
            // l & 15 of either half: one exchange between the halves per two registers.
            f32x4 acc[2] = {};
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const auto x = __builtin_amdgcn_permlane32_swap(kr[c][0], kr[c][2], false, false), y = __builtin_amdgcn_permlane32_swap(kr[c][1], kr[c][3], false, false);
                acc[0] = mfma(whole8(x[0], y[0]), q[c], acc[0]);
                acc[1] = mfma(whole8(x[1], y[1]), q[c], acc[1]);
            }
            const float sc[8] = {acc[0][0], acc[0][1], acc[0][2], acc[0][3], acc[1][0], acc[1][1], acc[1][2], acc[1][3]};
            if (next >= 0) load(kr, next, 0u);
            const float kc = Lookup::of(look.ks, i) * qc, lb = Lookup::of(look.lb, i);
            half8 pw[1], rest[1] = {};
            // (one place that moves the references, and x once more behind it: two such places cost a hundred registers)
            const bool all = at >= 0 && (int32_t)(j * 32u + 32u) <= least && lb == lb;
            const int32_t limit = at >= 0 ? place.limit : 0;
            float top, tope;
            if (all) {
                float best = sc[0];
#pragma unroll
                for (int t = 1; t < 8; ++t) best = fmaxf(best, sc[t]);
                top = row_max<16>(best) * kc;
                tope = top + lb;
            } else {
                float x[8];
                some_of_block<16>(sc, kc, lb, j, limit, x, &top, &tope);
            }
            row.follow(top, tope);
            if (all) {
                row.weights(sc, kc, lb, pw, EXACT ? rest : nullptr);
            } else {
                float x[8];
                some_of_block<16>(sc, kc, lb, j, limit, x, &top, &tope);
                row.weights_some(x, lb, pw, EXACT ? rest : nullptr);
            }
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const auto x = __builtin_amdgcn_permlane32_swap(vr[c][0], vr[c][1], false, false), y = __builtin_amdgcn_permlane32_swap(vr[c][2], vr[c][3], false, false);
                const half8 v0 = whole8(x[0], y[0]), v1 = whole8(x[1], y[1]);
                row.o[2 * c] = mfma(v0, pw[0], row.o[2 * c]);
                row.o[2 * c + 1] = mfma(v1, pw[0], row.o[2 * c + 1]);
                if constexpr (EXACT) {
                    row.o[2 * c] = mfma(v0, rest[0], row.o[2 * c]);
                    row.o[2 * c + 1] = mfma(v1, rest[0], row.o[2 * c + 1]);
                }
            }
            if (next >= 0) load(vr, next, 1u);
            at = next;
        }
        if (j < end) {
            look.get(a, p.seq, head, j + 4u * lane, end);
            at = look.index_of(0);
            load(kr, at, 0u);
            load(vr, at, 1u);
        }
    }

    // the open block, in 16 bits, with a scale for every token
    if (j == whole && j < j1) {
        uint32_t slot;
        if (read_slot(a.b, a.c, p.seq, &slot)) {
            const uint8_t *half = ring_half(a.c, slot, head, j);
            const uint32_t held = (uint32_t)s.len % 32u;
            f32x4 acc[2] = {};
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (uint32_t t = 0; t < 2u; ++t)
                    acc[t] = mfma(*reinterpret_cast<const half8 *>(half + 2048u * c + 64u * (16u * t + n) + 2u * chunk), q[c], acc[t]);
            const float sc[8] = {acc[0][0], acc[0][1], acc[0][2], acc[0][3], acc[1][0], acc[1][1], acc[1][2], acc[1][3]};
            float x[8], lv[8], top, tope;
            each_of_open<16>(sc, qc, reinterpret_cast<const float *>(half + 128ull * dim), held, j, place.limit, x, lv, &top, &tope);
            row.follow(top, tope);
            half8 pw[1], rest[1];
            row.weights_each(x, lv, pw, EXACT ? rest : nullptr);
#pragma unroll
            for (int c = 0; c < 2 * NC; ++c) {
                const uint8_t *from = half + 64u * dim + 64u * (16u * c + n) + 32u * (g & 1u) + 8u * (g >> 1);
                half8 v;
#pragma unroll
                for (uint32_t u = 0; u < 2u; ++u) {
                    const half4 part = *reinterpret_cast<const half4 *>(from + 16u * u);
#pragma unroll
                    for (int i = 0; i < 4; ++i)                             // places nobody has written yet may hold anything
                        v[4 * u + i] = 16u * u + 4u * g + i < held ? part[i] : (_Float16)0.0f;
                }
                row.o[c] = mfma(v, pw[0], row.o[c]);
                if constexpr (EXACT) row.o[c] = mfma(v, rest[0], row.o[c]);
            }
        }
    }

    // The four wavefronts' results in one, in their order.
    row.l = row_sum<16>(row.l);
    if (g == 0u) { s_stat[wave][0][n] = row.m; s_stat[wave][1][n] = row.l; s_stat[wave][2][n] = row.r; }
    __syncthreads();
    float mm = kNegInf, rr = kNegInf, ll = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) { mm = fmaxf(mm, s_stat[w][0][n]); rr = fmaxf(rr, s_stat[w][2][n]); }
    const float mms = mm == kNegInf ? 0.0f : mm, rrs = rr == kNegInf ? 0.0f : rr;
#pragma unroll
    for (int w = 0; w < 4; ++w) ll += s_stat[w][1][n] * exp2_fast(s_stat[w][0][n] - mms);
    const float mine = exp2_fast(row.r - rrs);
    const bool last = parts == 1u;
    const uint64_t slot_no = ((uint64_t)p.slot * a.c.heads + head) * 16u;
    if (wave == 0u && g == 0u) {
        if (last) {
            if (place.real && a.lse) a.lse[place.token * a.q_heads + place.qh] = log_sum(mms, ll);
        } else {
            float *st = a.part_s + 3u * (slot_no + n);
            st[0] = mm; st[1] = ll; st[2] = rr;
        }
        if (p.part == 0u && head == 0u && n == 0u) {
            int32_t *dir = a.directory + 2u * (first_unit(a.b.starts, p.seq, a.group, a.tile_shift, 1u) + p.tile);
            dir[0] = (int32_t)p.slot;
            dir[1] = (int32_t)parts;
        }
    }
    // o of a row without tokens is 0
    const float fin = last ? (ll == 0.0f ? 0.0f : exp2_fast(rrs - mms - kLift) / ll) : 1.0f;
#pragma unroll
    for (int c = 0; c < 2 * NC; c += 4) {                                   // 64 values of the head at a time, 16 of them per wavefront
        if (c) __syncthreads();
#pragma unroll
        for (int t = 0; t < 4; ++t)
            if (c + t < 2 * NC) *reinterpret_cast<f32x4 *>(&s_tile[wave][256 * t + 4 * lane]) = row.o[c + t] * mine;
        __syncthreads();
        if (c + (int)wave < 2 * NC) {
            f32x4 sum = *reinterpret_cast<const f32x4 *>(&s_tile[0][256 * wave + 4 * lane]);
#pragma unroll
            for (int w = 1; w < 4; ++w) sum += *reinterpret_cast<const f32x4 *>(&s_tile[w][256 * wave + 4 * lane]);
            sum *= fin;
            const uint32_t d = 16u * (c + wave) + 4u * g;
            if (place.real && last) store_out(a, place, d, sum);
            else if (place.real) *reinterpret_cast<f32x4 *>(a.part_o + (slot_no + n) * dim + d) = sum;
        }
    }
}

// Joins the pieces of a row: a workgroup per row, its wavefronts (and the parts of one that a row does not fill) take the pieces in turn; their
// sums are added in a fixed order.  3.7 us for one sequence, 5.7 for 64, 32 if those have 32 rows each.  grid: (heads * tiles, rows at a time)
__global__ __launch_bounds__(kAttendBlock) void k_attend_join(AttendArgs a) {
    __shared__ __align__(16) float s_o[kAttendBlock][4];
    const uint32_t tid = threadIdx.x, lane = (uint32_t)lane_id(), dim = a.c.dim;
    const uint32_t unit = blockIdx.x / a.c.heads, head = blockIdx.x - unit * a.c.heads;
    // (units that no tile has are unwritten: whatever they hold, what follows finds out)
    const uint32_t slot0 = (uint32_t)a.directory[2u * unit], parts = (uint32_t)a.directory[2u * unit + 1u];
    SeqWork w;
    uint32_t tile;
    const bool there = find_tile(a, unit, &w, &tile);                     // (both asked for at once)
    if (parts < 2u || slot0 >= a.slots || parts > a.slots - slot0 || !there) return;
    const uint32_t rows = (uint32_t)w.s.n * a.group;
    const uint32_t quads = dim / 4u, lots = kAttendBlock / quads, lot = tid / quads, quad = tid - lot * quads;    // lots: pieces at a time
    for (uint32_t n = blockIdx.y; n < a.tile_rows && tile * a.tile_rows + n < rows; n += gridDim.y) {
        const uint32_t row = tile * a.tile_rows + n, query = row / a.group, qh = head * a.group + (row - query * a.group);
        const int64_t token = (int64_t)w.s.start + query;
        const auto slot = [&](uint32_t k) { return ((uint64_t)(slot0 + k) * a.c.heads + head) * a.tile_rows + n; };
        // the first pieces' sums and values are asked for together
        float m1 = kNegInf, l1 = 0.0f, r1 = kNegInf, first_r = kNegInf;
        f32x4 o = {};
        if (lane < parts) {                                                // every wavefront for itself
            const float *st = a.part_s + 3u * slot(lane);
            m1 = st[0]; l1 = st[1]; r1 = st[2];
        }
        if (lot < lots && lot < parts) {
            o = *reinterpret_cast<const f32x4 *>(a.part_o + slot(lot) * dim + 4u * quad);
            first_r = a.part_s[3u * slot(lot) + 2u];
        }
        float m = m1, r = r1;
        for (uint32_t k = lane + kWave; k < parts; k += kWave) {
            const float *st = a.part_s + 3u * slot(k);
            m = fmaxf(m, st[0]);
            r = fmaxf(r, st[2]);
        }
#pragma unroll
        for (int o2 = 1; o2 < kWave; o2 <<= 1) { m = fmaxf(m, __shfl_xor(m, o2, kWave)); r = fmaxf(r, __shfl_xor(r, o2, kWave)); }
        const float ms = m == kNegInf ? 0.0f : m, rs = r == kNegInf ? 0.0f : r;
        float l = l1 * exp2_fast(m1 - ms);
        for (uint32_t k = lane + kWave; k < parts; k += kWave) {
            const float *st = a.part_s + 3u * slot(k);
            l += st[1] * exp2_fast(st[0] - ms);
        }
        l = wave_sum<float>(l);
        o *= exp2_fast(first_r - rs);
        if (lot < lots)
            for (uint32_t k = lot + lots; k < parts; k += lots)
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

// ... of the tiles of k_attend_tile, many rows of few pieces: a wavefront per row.
__global__ __launch_bounds__(kAttendBlock) void k_attend_join_tile(AttendArgs a) {
    const uint32_t lane = (uint32_t)lane_id(), dim = a.c.dim;
    const uint32_t unit = blockIdx.x / a.c.heads, head = blockIdx.x - unit * a.c.heads;
    // (units that no tile has are unwritten: whatever they hold, what follows finds out)
    const uint32_t slot0 = (uint32_t)a.directory[2u * unit], parts = (uint32_t)a.directory[2u * unit + 1u];
    SeqWork w;
    uint32_t tile;
    const bool there = find_tile(a, unit, &w, &tile);
    if (parts < 2u || slot0 >= a.slots || parts > a.slots - slot0 || !there) return;
    const uint32_t rows = (uint32_t)w.s.n * a.group;
    for (uint32_t n = blockIdx.y * 4u + threadIdx.x / kWave; n < a.tile_rows && tile * a.tile_rows + n < rows; n += 4u * gridDim.y) {
        const uint32_t row = tile * a.tile_rows + n, query = row / a.group, qh = head * a.group + (row - query * a.group);
        const auto slot = [&](uint32_t k) { return ((uint64_t)(slot0 + k) * a.c.heads + head) * a.tile_rows + n; };
        float m = kNegInf, r = kNegInf, l = 0.0f;
        f32x4 o = {};
        for (uint32_t k = 0; k < parts; ++k) {
            const float *st = a.part_s + 3u * slot(k);
            const float m1 = st[0], l1 = st[1], r1 = st[2];
            f32x4 v = {};
            if (4u * lane < dim) v = *reinterpret_cast<const f32x4 *>(a.part_o + slot(k) * dim + 4u * lane);
            const float m2 = fmaxf(m, m1), r2 = fmaxf(r, r1), ms = m2 == kNegInf ? 0.0f : m2, rs = r2 == kNegInf ? 0.0f : r2;
            l = l * exp2_fast(m - ms) + l1 * exp2_fast(m1 - ms);
            o = o * exp2_fast(r - rs) + v * exp2_fast(r1 - rs);
            m = m2;
            r = r2;
        }
        const float ms = m == kNegInf ? 0.0f : m, rs = r == kNegInf ? 0.0f : r;
        const float fin = l == 0.0f ? 0.0f : exp2_fast(rs - ms - kLift) / l;
        RowPlace p;
        p.real = true; p.qh = qh; p.token = (int64_t)w.s.start + query; p.limit = 0;
        if (lane == 0u && a.lse) a.lse[p.token * a.q_heads + qh] = log_sum(ms, l);
        if (4u * lane < dim) store_out(a, p, 4u * lane, o * fin);
    }
}

template __global__ void k_attend<1, false>(AttendArgs);
template __global__ void k_attend<1, true>(AttendArgs);
template __global__ void k_attend<2, false>(AttendArgs);
template __global__ void k_attend<2, true>(AttendArgs);
template __global__ void k_attend<3, false>(AttendArgs);
template __global__ void k_attend<3, true>(AttendArgs);
template __global__ void k_attend<4, false>(AttendArgs);
template __global__ void k_attend<4, true>(AttendArgs);
template __global__ void k_attend<5, false>(AttendArgs);
template __global__ void k_attend<5, true>(AttendArgs);
template __global__ void k_attend<6, false>(AttendArgs);
template __global__ void k_attend<6, true>(AttendArgs);
template __global__ void k_attend<7, false>(AttendArgs);
template __global__ void k_attend<7, true>(AttendArgs);
template __global__ void k_attend<8, false>(AttendArgs);
template __global__ void k_attend<8, true>(AttendArgs);
template __global__ void k_attend_few<1, false>(AttendArgs);
template __global__ void k_attend_few<1, true>(AttendArgs);
template __global__ void k_attend_few<2, false>(AttendArgs);
template __global__ void k_attend_few<2, true>(AttendArgs);
template __global__ void k_attend_few<3, false>(AttendArgs);
template __global__ void k_attend_few<3, true>(AttendArgs);
template __global__ void k_attend_few<4, false>(AttendArgs);
template __global__ void k_attend_few<4, true>(AttendArgs);
template __global__ void k_attend_few<5, false>(AttendArgs);
template __global__ void k_attend_few<5, true>(AttendArgs);
template __global__ void k_attend_few<6, false>(AttendArgs);
template __global__ void k_attend_few<6, true>(AttendArgs);
template __global__ void k_attend_few<7, false>(AttendArgs);
template __global__ void k_attend_few<7, true>(AttendArgs);
template __global__ void k_attend_few<8, false>(AttendArgs);
template __global__ void k_attend_few<8, true>(AttendArgs);

}  // namespace comet
