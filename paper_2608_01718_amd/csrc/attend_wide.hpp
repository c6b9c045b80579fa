// attend_wide.hpp -- the attention kernel for more than 32 rows of a (sequence, kv head): several new tokens, or many
// query heads on a kv head.
//
// The mathematics and the division of the work are those of attend.hpp.  With many rows the matrix cores and the softmax
// bound the time, not memory, and each tile is used by all of a workgroup's waves: it goes through registers into LDS
// (as bfloat16 whatever the cache's type), in the order of memory, which is that of the operands; each wave reads every
// operand once for its R row tiles.  Row tiles are dealt out to the waves in turn, so that a group that is not full leaves
// every SIMD about as much to do.  Four waves and two workgroups on a compute unit where the registers allow it (up to 128
// columns), so that one is at the matrix cores while the other is at the softmax; eight waves of one row tile each for
// wider heads.  (Tried without gain: eight waves of two row tiles, with 256 rows a group; the upper four waves half a step
// behind; two tiles on their way instead of one; three workgroups; row groups of about the same number of rows, which left every
// time as it was.)
//
// 21 new tokens of 32 sequences of 512 to 4096, 32 query heads on 4, d = 128: 55 us, and 10 for the join of 30 MB of parts; the
// matrix cores are busy for 17 % of it, the vector unit 23 %; 27 us are start, parts and join whatever the length.  151 new
// tokens of 4 sequences of 5000 to 20,000, 16 heads on 2, d = 256: 160 to 188 us by card, 0.52 to 0.61 PFLOP/s beside which the
// weights' second term is half as much again.  There LDS is the busiest unit: the eight waves read each operand for one row tile each,
// 256 KB a tile of tokens, 61 bytes a clock of 128, beside 36 % of the matrix cores.
#pragma once

#include "attend.hpp"

namespace lacache {

template <int DP, int CT, int WAVES, int R, bool F32>
struct Wide {
    static constexpr int KC = DP / 32, NJ = DP / 16;
    static constexpr bool BYTES = CT != kKvBf16;
    static constexpr int NT = F32 ? 3 : 1, NP = F32 ? 3 : 2;      // terms of a query element and of a weight (attend.hpp)
    static constexpr int ROWS = 16 * R * WAVES;                   // of a row group
    static constexpr int BYTES_TILE = 32 * DP * (BYTES ? 1 : 2);
    static constexpr int LOADS = 2 * BYTES_TILE / 1024;           // 16-byte loads a lane of keys and values, all waves
    static constexpr int PER_WAVE = (LOADS + WAVES - 1) / WAVES;
    // waves on a SIMD: two where the registers of the sums and queries leave room
    static constexpr int OCC = R * DP * (F32 ? 2 : 1) <= 256 ? 2 : 1;
};

template <int DP, int CT, int WAVES, int R, bool F32>
__global__ __launch_bounds__(64 * WAVES, (Wide<DP, CT, WAVES, R, F32>::OCC)) void k_attend_wide(AttendArgs a,
                                                                                              AttendPlan p) {
    using W = Wide<DP, CT, WAVES, R, F32>;
    using A = Attend<DP, CT, R, F32>;
    __shared__ u32x4 keys[2][2 * W::KC * 64], vals[2][W::NJ * 64];  // operands of 1 KB each
    __shared__ f32x4 scales[2][16];  // 32 of the keys, 32 of the values
    __shared__ int odd_of[WAVES];    // whether a wave has taken out something that is no number
    const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 15, u = lane >> 4;
    // Workgroups go to the eight XCDs in turn; each XCD takes an eighth of the work in one piece, so that the row groups of
    // a (sequence, kv head) share its L2.
    const int eighth = (p.workers + 7) >> 3, worker = (blockIdx.x & 7) * eighth + (blockIdx.x >> 3);
    if (worker >= p.workers) return;

    // (two tiles or more: a part of 128 rows is four times the bytes of a tile to write, and again to read in the join; one
    // sequence of 4096 tokens, 16 new ones 40 us, 50 with one)
    AttendRange range = attend_range<WAVES>(a, p, worker, 1, 2);
    if (range.at >= range.end) {
        if (tid == 0) p.split[worker].n_rows = 0;
        return;
    }
    AttendSplit split{};
    const float scale2 = scale_of(a);
    const int tile_shift = a.pool.page_shift - 5;
    AttendSpan s = attend_span(a, p, range.b);

    while (true) {
        // the segment that begins at item range.at
        const int rel = range.at - range.before;
        const int unit = (int)((uint32_t)rel / (uint32_t)s.chunks), c0 = rel - unit * s.chunks;
        const int h = (int)((uint32_t)unit / (uint32_t)s.groups), rg = unit - h * s.groups;
        const int left = range.end - range.at, c1 = s.chunks - c0 <= left ? s.chunks : c0 + left;
        range.at += c1 - c0;
        const bool starts = c0 == 0, ends = c1 == s.chunks;
        const int tile0 = c0 << p.chunk_shift, tile1 = ends ? s.tiles : c1 << p.chunk_shift;
        const int r0 = rg << p.group_shift, n_rows = s.rows - r0 < W::ROWS ? s.rows - r0 : W::ROWS;
        // positions that one of the rows, that every row sees
        const int64_t p0 = s.pos0() + token_of(p, r0), p1 = s.pos0() + token_of(p, r0 + n_rows - 1);
        const int q0 = p0 < 0 ? -1 : (int)p0, q1 = p1 < 0 ? -1 : (int)p1;
        const int seen0 = a.window > 0 && q0 - a.window + 1 > 0 ? q0 - a.window + 1 : 0;
        const int all0 = a.window > 0 && q1 - a.window + 1 > 0 ? q1 - a.window + 1 : 0;
        const int seen1 = q1 < s.cap - 1 ? q1 : s.cap - 1, all1 = q0 < seen1 ? q0 : seen1;
        const int tiles_here = (n_rows + 15) >> 4, active = tiles_here > wid ? (tiles_here - wid + WAVES - 1) / WAVES : 0;

        A w;
        w.clear();
        w.load_q(a, p, s, h, r0 + 16 * wid, 16 * WAVES, lane);

        // The segment's tiles in turn, from the first whose number is a multiple of a full range's length on, and then those
        // before it: row groups of one (sequence, kv head), whose ranges begin anywhere, read the same tiles at about the
        // same time.
        const int64_t per = (int64_t)range.per << p.chunk_shift;
        const int count = tile1 - tile0, off = (int)(tile0 % per);
        const int from = off != 0 && per - off < count ? (int)(per - off) : 0;
        int t0 = 0, page = -1;
        uint64_t todo = 0;
        auto tile_at = [&](int i) {  // the segment's i-th tile in that order
            i += from;
            return s.first + tile0 + (i < count ? i : i - count);
        };
        auto load_pages = [&]() {  // 64 tiles from t0 on, a lane each: which of them are there and seen
            const int t = t0 + lane, mine = tile_at(t);
            page = -1;
            if (t < count && 32 * mine <= seen1 && 32 * mine + 31 >= seen0)
                page = (a.seqs.pages + (int64_t)range.b * a.seqs.max_pages)[mine >> tile_shift];
            todo = __ballot(page >= 0 && page < a.pool.n_pages);
        };
        load_pages();
        // Begins to load the next tile, the waves a part each; its number, or -1 (then nothing is read).
        auto fetch = [&](u32x4 (&stage)[W::PER_WAVE], float& scale) {
            while (!todo && t0 + 64 < count) {
                t0 += 64;
                load_pages();
            }
            const int there = todo ? 1 : 0, k = there ? __ffsll((unsigned long long)todo) - 1 : 0;
            todo &= todo - 1;
            const int index = tile_at(t0 + k);
            const int64_t pg = there ? __builtin_amdgcn_readlane(page, k) : 0;
            const int64_t place = ((pg * a.pool.heads + h) << tile_shift) + (index & ((1 << tile_shift) - 1));
#pragma unroll
            for (int i = 0; i < W::PER_WAVE; ++i) {
                const int at = wid * W::PER_WAVE + i;  // which KB of the tile's keys and values
                const bool values = at >= W::LOADS / 2;
                const auto r = tile_rsrc((values ? a.pool.v : a.pool.k) + place * W::BYTES_TILE,
                                         at < W::LOADS ? there * W::BYTES_TILE : 0);
                stage[i] = tile_load<false>(r, 0, (at - (values ? W::LOADS / 2 : 0)) * 1024 + lane * 16);
            }
            if constexpr (W::BYTES) {
                const int size = wid == 0 ? there * 128 : 0, at = (lane & 31) * 4;
                const auto rk = tile_rsrc(a.pool.k_scale + place * 32, size), rv = tile_rsrc(a.pool.v_scale + place * 32, size);
                const uint32_t ks = __builtin_amdgcn_raw_buffer_load_b32(rk, at, 0, 0),
                               vs = __builtin_amdgcn_raw_buffer_load_b32(rv, at, 0, 0);
                scale = __uint_as_float(lane < 32 ? ks : vs);
            }
            return there ? index : -1;
        };
        uint32_t odd = 0;
        // The loaded tile into buffer b; values that no row sees as zeros, and those that are no numbers taken out of tiles
        // that rows see different parts of.
        auto put_tile = [&](const u32x4 (&stage)[W::PER_WAVE], float scale, int b, int index) {
            const bool edge = 32 * index < seen0 || 32 * index + 31 > seen1;
            const bool takes = A::mixed(index, seen0, seen1, all0, all1);
            auto shown = [&](int t) { return 32 * index + t >= seen0 && 32 * index + t <= seen1; };
#pragma unroll
            for (int i = 0; i < W::PER_WAVE; ++i) {
                const int at = wid * W::PER_WAVE + i;
                if (at >= W::LOADS) continue;
                const bool values = at >= W::LOADS / 2;
                u32x4 x = stage[i];
                if (edge && values) {
#pragma unroll
                    for (int d = 0; d < 4; ++d) {
                        uint32_t keep = 0;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            // dword d: in 8 bits tokens 16 (d % 2) + 4 u + e, in bfloat16 16 (d / 2) + 4 u + 2 (d % 2) + e / 2
                            const int t = W::BYTES ? 16 * (d & 1) + 4 * u + e : 16 * (d >> 1) + 4 * u + 2 * (d & 1) + (e >> 1);
                            keep |= shown(t) ? 0xFFu << (8 * e) : 0u;
                        }
                        x[d] &= keep;
                    }
                }
                if (takes && values) {
#pragma unroll
                    for (int d = 0; d < 4; ++d) {
                        const uint32_t none = A::no_codes(x[d]);
                        x[d] = A::without(x[d], none);
                        odd |= none;
                    }
                }
                u32x4* to = values ? &vals[b][0] : &keys[b][0];
                const int kb = values ? at - W::LOADS / 2 : at;
                if constexpr (!W::BYTES) {
                    to[kb * 64 + lane] = x;
                } else {
                    to[2 * kb * 64 + lane] = widen8<CT>(x[0], x[1]);
                    to[(2 * kb + 1) * 64 + lane] = widen8<CT>(x[2], x[3]);
                }
            }
            if constexpr (W::BYTES)
                if (wid == 0) {
                    float f = lane >= 32 && edge && !shown(lane & 31) ? 0.0f : scale;
                    if (takes && lane >= 32 && A::no_scale(f)) {
                        f = 0.0f;
                        odd = 1;
                    }
                    ((float*)scales[b])[lane] = f;
                }
        };
        // All tiles, for a wave with RA row tiles.
        auto run = [&](auto count) {
            constexpr int RA = decltype(count)::value;
            u32x4 stage[W::PER_WAVE];  // the next tile, on its way
            float stage_scale = 0.0f;
            int now = fetch(stage, stage_scale), buf = 0;
            if (now < 0) return;
            put_tile(stage, stage_scale, 0, now);
            int next = fetch(stage, stage_scale);
            lds_barrier();
            while (true) {
                if constexpr (RA > 0) {
                    f32x4 sc[R][2];
                    u32x4 weights[R][W::NP];
                    w.template scores_lds<RA>(&keys[buf][lane], scales[buf], u, sc, scale2);
                    if (32 * now < all0 || 32 * now + 31 > all1) w.template hide_scores<RA>(now, sc, lane);
                    w.template weigh<RA>(sc, scale2);
                    w.template round_lds<RA>(sc, scales[buf] + 8, u, weights);
                    w.template gather_lds<RA>(&vals[buf][lane], weights);
                }
                if (next < 0) break;
                buf ^= 1;
                put_tile(stage, stage_scale, buf, next);
                now = next;
                next = fetch(stage, stage_scale);
                lds_barrier();
            }
        };
        if (R == 2 && active == 2) run(std::integral_constant<int, R>{});
        else if (active >= 1) run(std::integral_constant<int, 1>{});
        else run(std::integral_constant<int, 0>{});
        if (seen0 < all0 || seen1 > all1) {  // (the same for all waves)
            const int any = __any(odd != 0);
            if (lane == 0) odd_of[wid] = any;
            lds_barrier();
            int some = 0;
#pragma unroll
            for (int t = 0; t < WAVES; ++t) some |= odd_of[t];
            if (__builtin_amdgcn_readfirstlane(some))
                w.spoil(a, a.seqs.pages + (int64_t)range.b * a.seqs.max_pages, h, s.first, tile0, tile1, 1, seen0, seen1, all0, all1,
                        lane);
        }
        w.reduce();

        const bool whole = starts && ends;
        const int64_t slot = part_of(p, worker, !ends);
        if (ends && !starts) {
            const int first = (int)((uint32_t)(range.before + unit * s.chunks) / (uint32_t)range.per);
            split = AttendSplit{s.row0, h * a.group, r0, n_rows, first, worker - first + 1, {}};
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int row = 16 * (r * WAVES + wid) + n;
            if (row >= n_rows) continue;
            if (!whole) {
                float* po = p.part_o + (slot + row) * DP;
#pragma unroll
                for (int j = 0; j < W::NJ; ++j) *(f32x4*)(po + 16 * j + 4 * u) = w.o[r][j];
                if (u == 0) p.part_ml[slot + row] = make_float2(w.m[r], w.l[r]);
            } else {
                const int i = token_of(p, r0 + row), head = h * a.group + (r0 + row - i * a.group);
                const int64_t at = ((int64_t)s.row0 + i) * a.q_heads + head;
                const float f = w.l[r] == 0.0f ? 0.0f : 1.0f / w.l[r];
#pragma unroll
                for (int j = 0; j < W::NJ; ++j)
                    if (16 * j + 4 * u < a.pool.d) store4<F32>(a, at * a.pool.d + 16 * j + 4 * u, w.o[r][j] * f);
                if (u == 0 && a.lse) a.lse[at] = lse_of(w.m[r], w.l[r]);
            }
        }
        if (range.at >= range.end) break;
        if (range.at - range.before >= s.items(a)) {  // past this sequence, and those without rows
            range.before += s.items(a);
            do s = attend_span(a, p, ++range.b);
            while (s.n == 0);
        }
        lds_barrier();  // the buffers have been read
    }
    if (tid == 0) p.split[worker] = split;
}

template <int DP>
hipError_t launch_attend(const AttendArgs& a, const AttendPlan& p, hipStream_t s) {
    const dim3 grid((unsigned)(p.group_shift < 6 ? p.workers : (p.workers + 7) & ~7)), block(p.waves * 64);
    auto go = [&](auto ct) {
        constexpr int CT = decltype(ct)::value;
        if (a.dtype == 0) {
            if (p.join_here) k_attend<DP, CT, 1, true, true><<<grid, block, 0, s>>>(a, p);
            else if (p.group_shift == 4) k_attend<DP, CT, 1, true, false><<<grid, block, 0, s>>>(a, p);
            else if constexpr (DP <= 192) k_attend_wide<DP, CT, 4, 1, true><<<grid, block, 0, s>>>(a, p);
            return;
        }
        switch (p.group_shift) {
            case 4:
                if (p.join_here) k_attend<DP, CT, 1, false, true><<<grid, block, 0, s>>>(a, p);
                else k_attend<DP, CT, 1, false, false><<<grid, block, 0, s>>>(a, p);
                break;
            case 5:
                if constexpr (DP <= 128) k_attend<DP, CT, 2, false, false><<<grid, block, 0, s>>>(a, p);
                break;
            case 6:
                if constexpr (DP <= 192) k_attend_wide<DP, CT, 4, 1, false><<<grid, block, 0, s>>>(a, p);
                break;
            case 7:
                if constexpr (DP <= 128) k_attend_wide<DP, CT, 4, 2, false><<<grid, block, 0, s>>>(a, p);
                else k_attend_wide<DP, CT, 8, 1, false><<<grid, block, 0, s>>>(a, p);
                break;
        }
    };
    if (a.pool.type == kKvBf16) go(std::integral_constant<int, kKvBf16>{});
    else if (a.pool.type == kKvFp8) go(std::integral_constant<int, kKvFp8>{});
    else go(std::integral_constant<int, kKvInt8>{});
    return hipGetLastError();
}

// Workgroups of the wide kernels on a compute unit.
constexpr int wide_occupancy(int dp, int waves, int R, bool f32) { return (R * dp * (f32 ? 2 : 1) <= 256 ? 2 : 1) * 4 / waves; }

extern template hipError_t launch_attend<64>(const AttendArgs&, const AttendPlan&, hipStream_t);
extern template hipError_t launch_attend<96>(const AttendArgs&, const AttendPlan&, hipStream_t);
extern template hipError_t launch_attend<128>(const AttendArgs&, const AttendPlan&, hipStream_t);
extern template hipError_t launch_attend<192>(const AttendArgs&, const AttendPlan&, hipStream_t);
extern template hipError_t launch_attend<256>(const AttendArgs&, const AttendPlan&, hipStream_t);

}  // namespace lacache
