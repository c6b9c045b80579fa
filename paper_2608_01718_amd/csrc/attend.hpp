// attend.hpp -- the attention kernel over the paged cache (instantiated per head width in k_attend_*.hip).
//
//   o = sum_j w_j v_j,  w = softmax(scale q . k_j)
//
// A pass over the keys and values with the running maximum and sum of the softmax, per 32-token tile and 16 R rows:
//   S^T = K Q^T    (16 tokens x 16 rows an instruction; the keys are the A operand as they lie in memory)
//   P = exp2(S - m), the sums and the weights in the registers that S^T left
//   O^T += V^T P^T (the values are the A operand as they lie in memory, P the B operand as it lies in registers)
// so keys and values go from memory to the matrix cores without LDS, and no weight changes lanes.  The rows of a
// (sequence, kv head) are its new tokens times the query heads that share the kv head.
//
// The work is the linear space (sequence, kv head, row group, tile), cut into equal ranges, one a workgroup, from the
// lengths on the device: ragged batches and single long contexts alike fill the chip.  A row group whose tiles lie in
// more than one range is joined by k_attend_join from the partial sums that the ranges leave in the workspace.
#pragma once

#include "kv.hpp"
#include "launch.hpp"

namespace lacache {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

// Workgroups on a compute unit, by the registers of a lane: the sums, the queries, a tile's keys and values, the scores
// and weights, and what goes around them.  (A wave of four has a SIMD's 512 registers to itself.)
constexpr int attend_occupancy(int dp, bool bytes, int R, bool f32) {
    const int terms = f32 ? 3 : 1;
    const int regs = R * dp / 4 + R * dp / 8 * terms + (bytes ? dp / 4 : dp / 2) + 12 * R + 4 * R * (f32 ? 3 : 2) + 4 * R +
                     8 * (terms - 1) + 56;
    return regs <= 170 ? 3 : regs <= 256 ? 2 : 1;
}

// What a launch works with besides the arguments: the shape of a row group, the grid, the workspace.
struct AttendPlan {
    int row_waves;   // the row group's rows are split over this many waves (1, 2 or 4), its tiles over the others
    int group_rows;  // rows of a row group: 16 R row_waves
    int workgroups;
    int64_t* base;   // [n_seq + 1] first item of each sequence; then the range of a workgroup
    float* part_o;   // [2 workgroups][group_rows][dp] partial sums of values
    float2* part_ml; // [2 workgroups][group_rows] their maxima and sums of weights
};

// What the work of a sequence is: its rows and their groups, its tiles.
struct AttendSpan {
    KvSpan span;
    int rows, groups;    // new tokens x group; row groups
    int first, tiles;    // the first tile that any row sees, the number of tiles
    int cap;             // positions that exist
};
__device__ inline AttendSpan attend_span(const AttendArgs& a, const AttendPlan& p, int b) {
    AttendSpan r;
    r.span = span_of(a.seqs, b);
    r.rows = r.span.n * a.group;
    r.groups = (r.rows + p.group_rows - 1) / p.group_rows;
    const int64_t held = (int64_t)a.seqs.max_pages << a.pool.page_shift;
    int64_t len = r.span.pos0 + r.span.n;
    len = len < 0 ? 0 : len > held ? held : len;
    int64_t lo = a.window > 0 ? r.span.pos0 - a.window + 1 : 0;
    lo = lo < 0 ? 0 : lo;
    r.cap = (int)len;
    r.first = (int)(lo >> 5);
    r.tiles = (int)((len + 31) >> 5) - r.first;
    if (r.tiles < 1) r.tiles = 1;  // rows that see nothing are written too
    return r;
}
__device__ inline int64_t attend_items(const AttendArgs& a, const AttendSpan& s) {
    return (int64_t)s.groups * a.pool.heads * s.tiles;
}

__device__ inline int64_t shfl_up64(int64_t x, int by) {
    const int lo = __shfl_up((int)x, by, kWave), hi = __shfl_up((int)(x >> 32), by, kWave);
    return (int64_t)hi << 32 | (uint32_t)lo;
}
__device__ inline int64_t shfl64(int64_t x, int from) {
    const int lo = __shfl((int)x, from, kWave), hi = __shfl((int)(x >> 32), from, kWave);
    return (int64_t)hi << 32 | (uint32_t)lo;
}
__device__ inline int64_t uniform64(int64_t x) {
    const int lo = __builtin_amdgcn_readfirstlane((int)x), hi = __builtin_amdgcn_readfirstlane((int)(x >> 32));
    return (int64_t)hi << 32 | (uint32_t)lo;
}

// four 8-bit codes as bfloat16 pairs
template <int CT>
__device__ __forceinline__ void widen4(uint32_t w, uint32_t& a, uint32_t& b) {
    if constexpr (CT == kKvFp8) {
        a = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.0f, false));
        b = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.0f, true));
    } else {  // integers up to 127 are exact in bfloat16: the high halves of their floats
        const float x0 = (float)(int8_t)w, x1 = (float)(int8_t)(w >> 8), x2 = (float)(int8_t)(w >> 16),
                    x3 = (float)(int8_t)(w >> 24);
        a = __builtin_amdgcn_perm(__float_as_uint(x1), __float_as_uint(x0), 0x07060302u);
        b = __builtin_amdgcn_perm(__float_as_uint(x3), __float_as_uint(x2), 0x07060302u);
    }
}
template <int CT>
__device__ __forceinline__ u32x4 widen8(uint32_t lo, uint32_t hi) {
    u32x4 r;
    uint32_t a, b;
    widen4<CT>(lo, a, b);
    r[0] = a, r[1] = b;
    widen4<CT>(hi, a, b);
    r[2] = a, r[3] = b;
    return r;
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    return (uint32_t)f32_to_bf16(a) | (uint32_t)f32_to_bf16(b) << 16;
}

template <int DP, int CT, int R, bool F32>
struct Attend {
    static constexpr int KC = DP / 32, NJ = DP / 16;       // column blocks of keys, of values
    static constexpr bool BYTES = CT != kKvBf16;
    static constexpr int NL = BYTES ? KC : 2 * KC;         // 16-byte loads a lane of a tile's keys (and of its values)
    // bfloat16 terms of a query element and of a weight: float32 rows need the 24 bits of three; with bfloat16 rows one
    // term of 8 bits would leave weights that are as far off as the result's own rounding, two are 2^8 times nearer
    static constexpr int NT = F32 ? 3 : 1, NP = F32 ? 3 : 2;
    static constexpr int OCC = attend_occupancy(DP, BYTES, R, F32);
    static constexpr int CB = DP <= 128 ? DP : DP / 2;     // columns joined at a time
    static constexpr int ESZ = F32 ? 4 : 2;

    u32x4 q[R][KC][NT];
    f32x4 o[R][NJ];
    float m[R], l[R];
    int hi[R], lo[R];  // the positions that the lane's row sees
    u32x4 kf[NL], vf[NL];
    f32x4 ks[2], vs[2];

    // 16 bytes of a row as KC operands: the three terms of a float32 sum back to it exactly, a bfloat16 is its own
    __device__ __forceinline__ void load_q(const AttendArgs& a, const AttendSpan& s, int h, int row0, int lane) {
        const int n = lane & 15, u = lane >> 4;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            int row = row0 + 16 * r + n;
            row = row < s.rows ? row : s.rows - 1;
            const int i = row / a.group, head = h * a.group + (row - i * a.group);
            const int64_t pos = s.span.pos0 + i;
            hi[r] = pos < 0 ? -1 : (int)pos;
            lo[r] = a.window > 0 && hi[r] - a.window + 1 > 0 ? hi[r] - a.window + 1 : 0;
            const char* src = a.q + ((s.span.row0 + i) * a.q_row + (int64_t)head * a.pool.d) * ESZ;
            const bool wide = ((uintptr_t)src & 15) == 0;
#pragma unroll
            for (int c = 0; c < KC; ++c) {
                const int col = 32 * c + 8 * u;
                u32x4 t[NT] = {};
                if (col < a.pool.d) {
                    if constexpr (F32) {
                        float x[8];
                        load8f(src, 0, a.pool.d, col, x);
#pragma unroll
                        for (int e = 0; e < 4; ++e) split2<NT>(x[2 * e], x[2 * e + 1], t, e);
                    } else if (wide) {
                        t[0] = *(const u32x4*)(src + col * 2);
                    } else {
                        const uint16_t* x = (const uint16_t*)src + col;
#pragma unroll
                        for (int e = 0; e < 4; ++e) t[0][e] = (uint32_t)x[2 * e] | (uint32_t)x[2 * e + 1] << 16;
                    }
                }
#pragma unroll
                for (int k = 0; k < NT; ++k) q[r][c][k] = t[k];
            }
        }
    }
    // two floats as pairs of bfloat16 terms
    template <int N>
    static __device__ __forceinline__ void split2(float x, float y, u32x4 (&t)[N], int e) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const uint32_t w = pack_bf16(x, y);
            t[k][e] = w;
            x -= __uint_as_float(w << 16);
            y -= __uint_as_float(w & 0xFFFF0000u);
        }
    }

    __device__ __forceinline__ void load_k(const char* p, const float* sc, int lane) {
#pragma unroll
        for (int i = 0; i < NL; ++i) kf[i] = ((const u32x4*)p)[i * 64 + lane];
        if constexpr (BYTES) {
            ks[0] = *(const f32x4*)(sc + 4 * (lane >> 4));
            ks[1] = *(const f32x4*)(sc + 16 + 4 * (lane >> 4));
        }
    }
    __device__ __forceinline__ void load_v(const char* p, const float* sc, int lane) {
#pragma unroll
        for (int i = 0; i < NL; ++i) vf[i] = ((const u32x4*)p)[i * 64 + lane];
        if constexpr (BYTES) {
            vs[0] = *(const f32x4*)(sc + 4 * (lane >> 4));
            vs[1] = *(const f32x4*)(sc + 16 + 4 * (lane >> 4));
        }
    }

    __device__ __forceinline__ u32x4 k_operand(int b, int c) const {
        if constexpr (!BYTES) return kf[2 * c + b];
        else return widen8<CT>(kf[c][2 * b], kf[c][2 * b + 1]);
    }
    __device__ __forceinline__ u32x4 v_operand(int j) const {
        if constexpr (!BYTES) return vf[j];
        else return widen8<CT>(vf[j >> 1][2 * (j & 1)], vf[j >> 1][2 * (j & 1) + 1]);
    }

    // scores of the tile in kf, in units of log2 e
    __device__ __forceinline__ void scores(f32x4 (&s)[R][2], float scale2) {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int b = 0; b < 2; ++b) s[r][b] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int c = 0; c < KC; ++c)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const u32x4 k = k_operand(b, c);
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int t = NT - 1; t >= 0; --t) s[r][b] = mfma16x16x32(k, q[r][c][t], s[r][b]);
            }
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float f = BYTES ? ks[b][i] * scale2 : scale2;
#pragma unroll
                for (int r = 0; r < R; ++r) s[r][b][i] *= f;
            }
    }

    // Hides the positions that a row does not see, and the values of those that no row of the wave sees (first .. last
    // are seen by one): what lies there may be anything.
    __device__ __forceinline__ void hide(f32x4 (&s)[R][2], int tile, int first, int last, int lane) {
        const int t0 = 32 * tile + 4 * (lane >> 4);
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            uint32_t keep[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int j = t0 + 16 * b + i;
#pragma unroll
                for (int r = 0; r < R; ++r)
                    s[r][b][i] = j >= lo[r] && j <= hi[r] ? s[r][b][i] : -__builtin_inff();
                keep[i] = j >= first && j <= last ? 0xFFFFFFFFu : 0u;
                if constexpr (BYTES) vs[b][i] = keep[i] ? vs[b][i] : 0.0f;
            }
            if constexpr (BYTES) {
                const uint32_t w = (keep[0] & 0xFFu) | (keep[1] & 0xFF00u) | (keep[2] & 0xFF0000u) | (keep[3] & 0xFF000000u);
#pragma unroll
                for (int i = 0; i < NL; ++i) {
                    vf[i][b] &= w;
                    vf[i][2 + b] &= w;
                }
            } else {
                const uint32_t w0 = (keep[0] & 0xFFFFu) | (keep[1] & 0xFFFF0000u),
                               w1 = (keep[2] & 0xFFFFu) | (keep[3] & 0xFFFF0000u);
#pragma unroll
                for (int i = 0; i < NL; ++i) {
                    vf[i][2 * b] &= w0;
                    vf[i][2 * b + 1] &= w1;
                }
            }
        }
    }

    // Weights of the tile (s becomes P), the running maximum and sum.  The sum stays a lane's own until the end.
    __device__ __forceinline__ void weigh(f32x4 (&s)[R][2]) {
        auto max2 = [](float x, float y) { return fmaxf(x, y); };
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float x = m[r];
#pragma unroll
            for (int i = 0; i < 4; ++i) x = fmaxf(fmaxf(x, s[r][0][i]), s[r][1][i]);
            x = xor_combine<16>(xor_combine<32>(x, max2), max2);
            if (__any(x > m[r])) {
                const float f = x > m[r] ? __builtin_amdgcn_exp2f(m[r] - x) : 1.0f;  // 0 where m was -infinity
                l[r] *= f;
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[r][j][i] *= f;
                m[r] = x;
            }
            const float base = m[r] == -__builtin_inff() ? 0.0f : m[r];
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[r][b][i] = __builtin_amdgcn_exp2f(s[r][b][i] - base);
                    l[r] += s[r][b][i];
                }
        }
    }

    // O^T += V^T P^T with the tile in vf
    __device__ __forceinline__ void gather(f32x4 (&s)[R][2]) {
        u32x4 p[R][NP];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float x = s[r][e >> 1][2 * (e & 1)], y = s[r][e >> 1][2 * (e & 1) + 1];
                if constexpr (BYTES) {
                    x *= vs[e >> 1][2 * (e & 1)];
                    y *= vs[e >> 1][2 * (e & 1) + 1];
                }
                split2<NP>(x, y, p[r], e);
            }
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            const u32x4 v = v_operand(j);
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int t = NP - 1; t >= 0; --t) o[r][j] = mfma16x16x32(v, p[r][t], o[r][j]);
        }
    }
};

// Four columns of a row of the result.
template <bool F32>
__device__ __forceinline__ void store4(const AttendArgs& a, int64_t row, int head, int col, f32x4 x) {
    const int64_t at = (row * a.q_heads + head) * a.pool.d + col;
    if (F32) {
        float* p = (float*)a.out + at;
        if (((uintptr_t)p & 15) == 0) *(f32x4*)p = x;
        else p[0] = x[0], p[1] = x[1], p[2] = x[2], p[3] = x[3];
    } else {
        uint16_t* p = (uint16_t*)a.out + at;
        if (((uintptr_t)p & 7) == 0) *(uint2*)p = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
        else p[0] = f32_to_bf16(x[0]), p[1] = f32_to_bf16(x[1]), p[2] = f32_to_bf16(x[2]), p[3] = f32_to_bf16(x[3]);
    }
}

__device__ __forceinline__ float lse_of(float m, float l) {
    return l == 0.0f ? -__builtin_inff() : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

template <int DP, int CT, int R, bool F32>
__global__ __launch_bounds__(256, (Attend<DP, CT, R, F32>::OCC)) void k_attend(AttendArgs a, AttendPlan p) {
    using A = Attend<DP, CT, R, F32>;
    __shared__ float sm[4][16 * R], sl[4][16 * R];
    __shared__ float so[4][16][A::CB + 4];
    const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tile_waves = 4 / p.row_waves, row_part = wid % p.row_waves, tile_part = wid / p.row_waves;

    // the range of this workgroup, and the sequence in which it begins
    const int n_seq = a.seqs.n_seq;
    int64_t total = 0;
    for (int b0 = 0; b0 < n_seq; b0 += 64) {
        const int b = b0 + lane;
        int64_t x = b < n_seq ? attend_items(a, attend_span(a, p, b)) : 0;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int64_t y = shfl_up64(x, o);
            if (lane >= o) x += y;
        }
        if (blockIdx.x == 0 && wid == 0 && b < n_seq) p.base[b + 1] = total + x;
        total += shfl64(x, 63);
    }
    total = uniform64(total);
    int64_t per = (total + p.workgroups - 1) / p.workgroups;
    per = (per + tile_waves - 1) / tile_waves * tile_waves;
    if (blockIdx.x == 0 && tid == 0) {
        p.base[0] = 0;
        p.base[n_seq + 1] = per;
    }
    int64_t at = (int64_t)blockIdx.x * per;
    const int64_t end = at + per < total ? at + per : total;
    if (at >= end) return;
    int b = 0;
    int64_t before = 0;  // items before sequence b
    for (int b0 = 0; b0 < n_seq; b0 += 64) {
        const int bb = b0 + lane;
        int64_t x = bb < n_seq ? attend_items(a, attend_span(a, p, bb)) : 0;
        const int64_t own = x;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int64_t y = shfl_up64(x, o);
            if (lane >= o) x += y;
        }
        const uint64_t past = __ballot(before + x > at);
        if (past) {
            const int i = __ffsll((unsigned long long)past) - 1;
            b = b0 + i;
            before = uniform64(before + shfl64(x - own, i));
            break;
        }
        before = uniform64(before + shfl64(x, 63));
    }
    b = __builtin_amdgcn_readfirstlane(b);

    A w;
    const float scale2 = a.scale * kLog2e;
    const int tile_shift = a.pool.page_shift - 5;
    while (at < end) {
        const AttendSpan s = attend_span(a, p, b);
        const int64_t items = attend_items(a, s);
        if (at - before >= items) {  // past this sequence (or it has no rows)
            before += items;
            ++b;
            continue;
        }
        const int unit = (int)((at - before) / s.tiles);                  // kv head and row group
        const int tile0 = (int)((at - before) - (int64_t)unit * s.tiles);
        const int h = unit / s.groups, rg = unit - h * s.groups;
        const int64_t left = end - at;
        const int tile1 = s.tiles - tile0 <= left ? s.tiles : tile0 + (int)left;
        const bool whole = tile0 == 0 && tile1 == s.tiles;

        const int row0 = rg * p.group_rows + row_part * 16 * R;  // the wave's rows
#pragma unroll
        for (int r = 0; r < R; ++r) {
            w.m[r] = -__builtin_inff();
            w.l[r] = 0.0f;
#pragma unroll
            for (int j = 0; j < A::NJ; ++j) w.o[r][j] = f32x4{0, 0, 0, 0};
        }
        if (row0 < s.rows) {
            w.load_q(a, s, h, row0, lane);
            // positions: seen by one of the wave's rows (first .. last), by all of them (first_all .. last_all)
            const int row1 = row0 + 16 * R - 1 < s.rows ? row0 + 16 * R - 1 : s.rows - 1;
            const int64_t p0 = s.span.pos0 + row0 / a.group, p1 = s.span.pos0 + row1 / a.group;
            const int last_all = p0 < 0 ? -1 : (int)p0;
            int last = p1 < 0 ? -1 : (int)p1;
            const int first = a.window > 0 && last_all - a.window + 1 > 0 ? last_all - a.window + 1 : 0;
            const int first_all = a.window > 0 && last - a.window + 1 > 0 ? last - a.window + 1 : 0;
            last = last < s.cap - 1 ? last : s.cap - 1;
            const int32_t* pages = a.seqs.pages + (int64_t)b * a.seqs.max_pages;

            for (int t0 = tile0 + tile_part; t0 < tile1; t0 += 64 * tile_waves) {
                // the next 64 tiles of the wave, a lane each: which are there and seen
                const int mine = s.first + t0 + lane * tile_waves;
                int page = -1;
                if (t0 + lane * tile_waves < tile1 && 32 * mine <= last && 32 * mine + 31 >= first)
                    page = pages[mine >> tile_shift];
                uint64_t todo = __ballot(page >= 0 && page < a.pool.n_pages);
                if (!todo) continue;
                auto place = [&](int i, int& tile) {
                    tile = s.first + t0 + i * tile_waves;
                    const int64_t pg = __builtin_amdgcn_readlane(page, i);
                    return ((pg * a.pool.heads + h) << tile_shift) + (tile & ((1 << tile_shift) - 1));
                };
                constexpr int TB = 32 * DP * (A::BYTES ? 1 : 2);  // bytes of a tile
                int i = __ffsll((unsigned long long)todo) - 1, tile;
                int64_t pl = place(i, tile);
                w.load_k(a.pool.k + pl * TB, a.pool.k_scale + pl * 32, lane);
                w.load_v(a.pool.v + pl * TB, a.pool.v_scale + pl * 32, lane);
                todo &= todo - 1;
                auto step = [&](auto more) {
                    f32x4 sc[R][2];
                    w.scores(sc, scale2);
                    int next = 0;
                    if constexpr (decltype(more)::value) {
                        i = __ffsll((unsigned long long)todo) - 1;
                        todo &= todo - 1;
                        pl = place(i, next);
                        w.load_k(a.pool.k + pl * TB, a.pool.k_scale + pl * 32, lane);
                    }
                    if (32 * tile < first_all || 32 * tile + 31 > last_all || 32 * tile + 31 > last)
                        w.hide(sc, tile, first, last, lane);
                    w.weigh(sc);
                    w.gather(sc);
                    if constexpr (decltype(more)::value) {
                        w.load_v(a.pool.v + pl * TB, a.pool.v_scale + pl * 32, lane);
                        tile = next;
                    }
                };
                while (todo) step(std::true_type{});
                step(std::false_type{});
            }
        }

        // the waves' results, joined where several waves had tiles of the same rows
        auto add2 = [](float x, float y) { return x + y; };
#pragma unroll
        for (int r = 0; r < R; ++r) w.l[r] = xor_combine<16>(xor_combine<32>(w.l[r], add2), add2);
        const int64_t slot = 2 * (int64_t)blockIdx.x + (tile1 < s.tiles ? 1 : 0);
        float* part_o = p.part_o + slot * p.group_rows * DP;
        float2* part_ml = p.part_ml + slot * p.group_rows;
        const int64_t out0 = s.span.row0;
        // one row's maximum and sum
        auto put_ml = [&](int in_group, float m, float l) {
            const int row = rg * p.group_rows + in_group;
            if (row >= s.rows) return;
            if (!whole) part_ml[in_group] = make_float2(m, l);
            else if (a.lse) {
                const int i = row / a.group;
                a.lse[(out0 + i) * a.q_heads + h * a.group + (row - i * a.group)] = lse_of(m, l);
            }
        };
        auto put_o = [&](int in_group, int col, f32x4 x, float l) {
            const int row = rg * p.group_rows + in_group;
            if (row >= s.rows) return;
            if (!whole) {
                *(f32x4*)(part_o + (int64_t)in_group * DP + col) = x;
            } else if (col < a.pool.d) {
                const float f = l == 0.0f ? 0.0f : 1.0f / l;
                const int i = row / a.group;
                store4<F32>(a, out0 + i, h * a.group + (row - i * a.group), col, x * f);
            }
        };
        const int n = lane & 15, g = lane >> 4;
        if (tile_waves == 1) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int in_group = row_part * 16 * R + 16 * r + n;
                if (g == 0) put_ml(in_group, w.m[r], w.l[r]);
#pragma unroll
                for (int j = 0; j < A::NJ; ++j) put_o(in_group, 16 * j + 4 * g, w.o[r][j], w.l[r]);
            }
        } else {
            if (g == 0) {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    sm[wid][16 * r + n] = w.m[r];
                    sl[wid][16 * r + n] = w.l[r];
                }
            }
            lds_barrier();
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float M = -__builtin_inff(), L = 0.0f;
                for (int t = 0; t < tile_waves; ++t) M = fmaxf(M, sm[t * p.row_waves + row_part][16 * r + n]);
                const float base = M == -__builtin_inff() ? 0.0f : M;
                for (int t = 0; t < tile_waves; ++t)
                    L += sl[t * p.row_waves + row_part][16 * r + n] *
                         __builtin_amdgcn_exp2f(sm[t * p.row_waves + row_part][16 * r + n] - base);
                const float f = __builtin_amdgcn_exp2f(w.m[r] - base);
                w.m[r] = M;
                w.l[r] = L;
#pragma unroll
                for (int j = 0; j < A::NJ; ++j) w.o[r][j] *= f;
                if (tile_part == 0 && g == 0) put_ml(row_part * 16 * R + 16 * r + n, M, L);
            }
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int c0 = 0; c0 < DP; c0 += A::CB) {
                    lds_barrier();  // what was read of so (and of sm and sl) has been read
                    if (r == 0 && c0 == 0 && tile_part == 0 && g == 0) {
                        // every row's sum, for the threads that divide by it
#pragma unroll
                        for (int rr = 0; rr < R; ++rr) sl[row_part][16 * rr + n] = w.l[rr];
                    }
#pragma unroll
                    for (int j = c0 / 16; j < (c0 + A::CB) / 16; ++j) *(f32x4*)&so[wid][n][16 * j - c0 + 4 * g] = w.o[r][j];
                    lds_barrier();
                    for (int e = tid; e < p.row_waves * 16 * (A::CB / 4); e += 256) {
                        const int col = e % (A::CB / 4) * 4, row = e / (A::CB / 4) % 16, part = e / (A::CB / 4) / 16;
                        f32x4 x = *(const f32x4*)&so[part][row][col];
                        for (int t = 1; t < tile_waves; ++t) x += *(const f32x4*)&so[t * p.row_waves + part][row][col];
                        put_o(part * 16 * R + 16 * r + row, c0 + col, x, sl[part][16 * r + row]);
                    }
                }
            lds_barrier();
        }
        at += tile1 - tile0;
    }
}

template <int DP>
hipError_t launch_attend(const AttendArgs& a, const AttendPlan& p, int R, hipStream_t s) {
    const dim3 grid((unsigned)p.workgroups), block(256);
    auto go = [&](auto ct) {
        constexpr int CT = decltype(ct)::value;
        if (a.dtype == 0) k_attend<DP, CT, 1, true><<<grid, block, 0, s>>>(a, p);
        else if (R == 1) k_attend<DP, CT, 1, false><<<grid, block, 0, s>>>(a, p);
        if constexpr (DP <= 192)
            if (R == 2 && a.dtype != 0) k_attend<DP, CT, 2, false><<<grid, block, 0, s>>>(a, p);
        if constexpr (DP <= 96)
            if (R == 4 && a.dtype != 0) k_attend<DP, CT, 4, false><<<grid, block, 0, s>>>(a, p);
    };
    if (a.pool.type == kKvBf16) go(std::integral_constant<int, kKvBf16>{});
    else if (a.pool.type == kKvFp8) go(std::integral_constant<int, kKvFp8>{});
    else go(std::integral_constant<int, kKvInt8>{});
    return hipGetLastError();
}

extern template hipError_t launch_attend<64>(const AttendArgs&, const AttendPlan&, int, hipStream_t);
extern template hipError_t launch_attend<96>(const AttendArgs&, const AttendPlan&, int, hipStream_t);
extern template hipError_t launch_attend<128>(const AttendArgs&, const AttendPlan&, int, hipStream_t);
extern template hipError_t launch_attend<192>(const AttendArgs&, const AttendPlan&, int, hipStream_t);
extern template hipError_t launch_attend<256>(const AttendArgs&, const AttendPlan&, int, hipStream_t);

}  // namespace lacache
