// attend_blocks.hpp -- attention of each row over the pages of its own list (instantiated per head width in k_attend_*.hip).
//
// The mathematics is that of attend.hpp, with its tiles: 32 tokens from memory to the matrix cores without LDS.  Every
// (row, kv head) has a list of its own, so that only its query heads share a tile: up to sixteen rows of an instruction.
// Lists have the same room, known to the host: each is cut into `splits` equal ranges of tiles, a workgroup of four waves
// each, and the workgroup that ends last joins their parts.
//
// Memory bounds it where there are many lists (64 rows of up to 48 pages of 64 tokens, 4 heads, fp8: 132 MB in 26 us, 5.0 TB/s;
// 64 rows of 64 pages, 8 heads, bfloat16: 160 us, 6.7 TB/s), else the chain of list, table, tile and join (one row 9 us).
#pragma once

#include "attend.hpp"

namespace lacache {

template <int DP, int CT, bool F32>
__global__ __launch_bounds__(256, (Attend<DP, CT, 1, F32>::OCC)) void k_attend_blocks(BlocksArgs x) {
    using A = Attend<DP, CT, 1, F32>;
    __shared__ float2 sml[4][16];
    __shared__ float so[4][16][A::CB + 4];
    __shared__ int last;
    const AttendArgs& a = x.a;
    const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row_tiles = (a.group + 15) >> 4, tile_shift = a.pool.page_shift - 5;
    const int unit = (int)(blockIdx.x / (unsigned)x.splits), split = (int)(blockIdx.x - (unsigned)unit * x.splits);
    const int list = unit / row_tiles, g0 = (unit - list * row_tiles) * 16;
    const int row = list / a.pool.heads, h = list - row * a.pool.heads;
    const int32_t* blocks = x.blocks + (int64_t)list * x.n_blocks;
    const int64_t tiles = (int64_t)x.n_blocks << tile_shift;
    const int64_t end64 = (int64_t)(split + 1) * x.per;
    const int end = (int)(end64 < tiles ? end64 : tiles);
    // the wave's tiles t0, t0 + 4, ... of the list, a lane each: the first lanes' pages are on their way while the sequence is looked for
    int t0 = split * x.per + wid;
    auto listed = [&]() {
        const int t = t0 + lane * 4;
        return t < end ? blocks[t >> tile_shift] : -1;
    };
    int block = listed();
    const int b = sequence_of(a.seqs, row, lane);
    if (b < 0) return;
    const KvSpan span = span_of(a.seqs, b);
    const int64_t pos64 = span.pos0 + (row - span.row0);
    const int pos = pos64 < 0 ? -1 : (int)pos64, n_rows = a.group - g0 < 16 ? a.group - g0 : 16;
    const int32_t* pages = a.seqs.pages + (int64_t)b * a.seqs.max_pages;
    A w;
    typename A::Tile tile;
    w.clear();
    int page = -1, index = 0, there = 0;
    uint64_t todo = 0;
    auto load_pages = [&]() {
        page = -1;
        if (block >= 0 && block < a.seqs.max_pages && (int64_t)block << a.pool.page_shift <= pos64) {
            index = (block << tile_shift) + ((t0 + lane * 4) & ((1 << tile_shift) - 1));
            if (32 * index <= pos) page = pages[block];
        }
    };
    auto look = [&]() { todo = __ballot(page >= 0 && page < a.pool.n_pages); };
    auto next = [&]() {
        while (!todo && t0 + 256 < end) {
            t0 += 256;
            block = listed();
            load_pages();
            look();
        }
        there = todo ? 1 : 0;
        const int k = there ? __ffsll((unsigned long long)todo) - 1 : 0;
        todo &= todo - 1;
        tile.index = __builtin_amdgcn_readlane(index, k);
        const int64_t pg = there ? __builtin_amdgcn_readlane(page, k) : 0;
        return ((pg * a.pool.heads + h) << tile_shift) + (tile.index & ((1 << tile_shift) - 1));
    };
    load_pages();
    AttendPlan p{};  // (a row's query heads are rows of their own)
    p.group_magic = x.magic, p.group_bits = x.bits, p.group_shift = 4;
    AttendSpan s{};
    s.row0 = row, s.n = 1, s.len = pos + 1, s.rows = a.group;
    w.load_q(a, p, s, h, g0, 16, lane);  // while the page numbers are on their way
    const float scale2 = scale_of(a);
    __builtin_amdgcn_sched_barrier(0);
    look();
    {
        const int64_t place = next();
        A::load_k(tile, a, place, there, lane);
        A::load_v(tile, a, place, there, lane);
    }
    __builtin_amdgcn_sched_barrier(0);
    while (there) {
        f32x4 sc[1][2];
        w.scores(tile, sc, scale2);
        const int now = tile.index;
        const int64_t place = next();
        A::load_k(tile, a, place, there, lane);
        if (32 * now + 31 > pos) w.hide(tile, now, sc, 0, pos, lane);
        w.weigh(sc, scale2);
        w.gather(tile, sc);
        A::load_v(tile, a, place, there, lane);
    }
    w.reduce();

    const int n = lane & 15, u = lane >> 4;
    const int64_t part = ((int64_t)unit * x.splits + split) << 4;
    auto finish = [&](int r, int col, f32x4 o, float m, float l) {
        const int64_t at = (int64_t)row * a.q_heads + h * a.group + g0 + r;
        if (col < a.pool.d) store4<F32>(a, at * a.pool.d + col, o * (l == 0.0f ? 0.0f : 1.0f / l));
        if (col == 0 && a.lse) a.lse[at] = lse_of(m, l);
    };
    p.part_o = x.part_o, p.part_ml = x.part_ml;
    if (u == 0) sml[wid][n] = make_float2(w.m[0], w.l[0]);
#pragma unroll
    for (int c0 = 0; c0 < DP; c0 += A::CB) {
        if (c0 > 0) lds_barrier();
        if (n < n_rows) {
#pragma unroll
            for (int j = 0; j < A::CB / 16; ++j) *(f32x4*)&so[wid][n][16 * j + 4 * u] = w.o[0][c0 / 16 + j];
        }
        lds_barrier();
        for (int e = tid; e < n_rows * (A::CB / 4); e += 256) {
            const int col = e % (A::CB / 4) * 4, r = e / (A::CB / 4);
            float2 ml[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) ml[t] = sml[t][r];
            const float M = fmaxf(fmaxf(ml[0].x, ml[1].x), fmaxf(ml[2].x, ml[3].x));
            const float base = M == -__builtin_inff() ? 0.0f : M;
            float L = 0.0f;
            f32x4 o{0, 0, 0, 0};
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const float f = __builtin_amdgcn_exp2f(ml[t].x - base);
                L += ml[t].y * f;
                o += *(const f32x4*)&so[t][r][col] * f;
            }
            if (x.splits == 1) {
                finish(r, c0 + col, o, M, L);
            } else {
                store_part<DP>(p, part, r, c0 + col, o);
                if (c0 + col == 0) store_part_ml(p, part, r, M, L);
            }
        }
    }
    if (x.splits == 1) return;

    last_workgroup_wait();
    __syncthreads();
    if (tid == 0) {
        last = __hip_atomic_fetch_add(x.done + unit, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)x.splits - 1;
        if (last) __hip_atomic_store(x.done + unit, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!last) return;
    // DP / 4 lanes a row; the lane groups that are left over share a row's parts
    constexpr int LANES = DP / 4, GROUPS = 256 / LANES;
    static_assert(sizeof(so) >= 256 * 24, "the join's scratch");
    f32x4* scratch = (f32x4*)&so[0][0][0];
    float2* ml_of = (float2*)(scratch + 256);
    int of_row = 1;
    while (2 * of_row * n_rows <= GROUPS) of_row *= 2;
    const int g = tid / LANES, col = tid % LANES * 4, sub = g % of_row, rows = GROUPS / of_row;
    auto load8 = [](const void* from) {
        const uint64_t v = __hip_atomic_load((const uint64_t*)from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
    };
    for (int r0 = 0; r0 < n_rows; r0 += rows) {
        const int r = r0 + g / of_row;
        const bool live = g < rows * of_row && r < n_rows;
        Joined j;
        if (live)
            for (int k0 = sub; k0 < x.splits; k0 += 4 * of_row) {
                float2 ml[4], lo[4], hi[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int k = k0 + i * of_row < x.splits ? k0 + i * of_row : x.splits - 1;
                    const int64_t at = (((int64_t)unit * x.splits + k) << 4) + r;
                    ml[i] = load8(x.part_ml + at);
                    lo[i] = load8(x.part_o + at * DP + col);
                    hi[i] = load8(x.part_o + at * DP + col + 2);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (k0 + i * of_row < x.splits) j.add(ml[i].x, ml[i].y, f32x4{lo[i].x, lo[i].y, hi[i].x, hi[i].y});
            }
        if (of_row > 1) {
            ml_of[tid] = make_float2(j.m, j.l);
            scratch[tid] = j.o;
            __syncthreads();
            if (sub == 0 && live)
                for (int k = 1; k < of_row; ++k) j.add(ml_of[tid + k * LANES].x, ml_of[tid + k * LANES].y, scratch[tid + k * LANES]);
            __syncthreads();
        }
        if (live && sub == 0) finish(r, col, j.o, j.m, j.l);
    }
}

template <int DP>
hipError_t launch_blocks(const BlocksArgs& x, int64_t units, hipStream_t s) {
    const dim3 grid((unsigned)(units * x.splits)), block(256);
    auto go = [&](auto ct) {
        constexpr int CT = decltype(ct)::value;
        if (x.a.dtype == 0) k_attend_blocks<DP, CT, true><<<grid, block, 0, s>>>(x);
        else k_attend_blocks<DP, CT, false><<<grid, block, 0, s>>>(x);
    };
    if (x.a.pool.type == kKvBf16) go(std::integral_constant<int, kKvBf16>{});
    else if (x.a.pool.type == kKvFp8) go(std::integral_constant<int, kKvFp8>{});
    else go(std::integral_constant<int, kKvInt8>{});
    return hipGetLastError();
}

extern template hipError_t launch_blocks<64>(const BlocksArgs&, int64_t, hipStream_t);
extern template hipError_t launch_blocks<96>(const BlocksArgs&, int64_t, hipStream_t);
extern template hipError_t launch_blocks<128>(const BlocksArgs&, int64_t, hipStream_t);
extern template hipError_t launch_blocks<192>(const BlocksArgs&, int64_t, hipStream_t);
extern template hipError_t launch_blocks<256>(const BlocksArgs&, int64_t, hipStream_t);

}  // namespace lacache
