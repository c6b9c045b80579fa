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
// more than one range is joined from the partial sums that the ranges leave in the workspace: by the launch that follows
// (k_attend.hip), or, where there is little to do, by whichever of its workgroups ends last.
//
// Few rows: bound by reading keys and values (four query heads on a kv head: 4 operations a byte).  One token, 32 query heads
// on 8, d = 128: 131,071 positions in bfloat16 80 us (6.7 TB/s; a large read 6.8), 64 sequences of 256 to 16,384 in fp8 96 us
// (5.6 TB/s); 256 sequences of 512 to 2048, 16 heads of 64 columns 188 us (6.2 TB/s); 777 positions 13 us: launch, lengths, pages,
// tiles and the join one after another.  Joins 4 to 6 us more.
#pragma once

#include "kv.hpp"
#include "launch.hpp"

namespace lacache {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

// A running maximum is raised only when a score passes it by more than this (in units of log2 e): weights then reach
// 2^8 times the largest, which costs sums in float32 nothing, and the sums are rarely scaled.
constexpr float kSlack = 8.0f;

// Workgroups on a compute unit, by the registers of a lane: the sums, the queries, a tile's keys and values, the scores
// and weights, and what goes around them.  (A wave of four has a SIMD's 512 registers to itself.)
constexpr int attend_occupancy(int dp, bool bytes, int R, bool f32) {
    const int terms = f32 ? 3 : 1;
    const int regs = R * dp / 4 + R * dp / 8 * terms + (bytes ? dp / 4 + 16 : dp / 2) + 12 * R + 4 * R * (f32 ? 3 : 2) + 4 * R +
                     8 * (terms - 1) + 56;
    return regs <= 136 ? 4 : regs <= 170 ? 3 : regs <= 256 ? 2 : 1;
}

// What an attention launch is: all of it; the part over the prefixes that groups of sequences share, whose "sequences" are
// the groups; the part over each sequence's own tokens.  The launch behind the two parts puts them together.
enum AttendMode { kWhole = 0, kPrefix = 1, kOwn = 2 };

// The sums of a part for every (row, query head): where they lie, as the number of workers that have parts of its row group
// (0: all of it is in o and ml), the first of them, and the row's place in the group.
struct AttendSums {
    float* o;    // [rows q_heads][dp] sums of values
    float2* ml;  // [rows q_heads] their maxima and sums of weights
    int2* at;    // [rows q_heads] workers; first worker + 2^16 place
};

// The shared prefixes of a call, as k_attend_share has laid them out.
struct AttendShare {
    int n_groups;
    int4* span;        // [n_groups] first row, rows, shared tokens (whole pages), the sequence whose page table is read
    int32_t* first;    // [n_groups] the first tile that any row sees
    int32_t* held;     // [n_seq] tokens that a sequence shares (0: it is in no group)
    int32_t* row_pos;  // [rows] positions of rows (-1 before the first)
    int32_t* row_held; // [rows] whether a row's sequence shares tokens; -1: it is in no sequence
    int32_t* deal;     // of a launch of both parts the workgroups that see to the prefixes
    AttendSums sums[2];  // kPrefix, kOwn
};

// What a launch works with besides the arguments: the shape of a row group, its workers, the workspace.
struct AttendPlan {
    int group_shift;   // rows of a row group, as a shift
    int workers, waves;  // workgroups of the launch, and the waves of each
    int chunk_shift;   // the work is dealt out in chunks of this many tiles (a shift), so that counts fit in 32 bits
    int extra;         // chunks that a row group counts for besides its tiles' (kOwn)
    uint32_t group_magic, group_bits;  // row / group = row * magic >> bits
    int join_here;     // parts are joined by the workgroup that ends last; otherwise by the launch that follows
    uint32_t* done;    // [kMaxWorkers] parts that are there of the row group that begins with a worker; 0 between launches
    struct AttendSplit* split;  // [workers]: the row group whose last part a worker had
    float* part_o;     // [2 workers][group rows][dp] partial sums of values
    float2* part_ml;   // [2 workers][group rows] their maxima and sums of weights
};

// That of a part's launch.
struct AttendPartPlan : AttendPlan {
    AttendShare share;
};
template <int MODE>
using PlanOf = std::conditional_t<MODE == kWhole, AttendPlan, AttendPartPlan>;

constexpr int kMaxWorkers = 4096;

// A row group that several workers have parts of, the last of them the one whose entry in AttendPlan::split this is.
struct alignas(16) AttendSplit {
    int seq_row0, head0;   // the sequence's first row, the first query head
    int row, n_rows;       // rows row .. row + n_rows - 1 of the sequence's (0: there is no such row group)
    int worker0, parts;    // the first of its workers, their number
    int unused[2];
};

// What the work of a sequence is: its rows and their groups, its tiles.
struct AttendSpan {
    int row0, n, len;    // first row, new tokens, tokens with them
    int rows, groups;    // new tokens x group; row groups
    int first, tiles;    // the first tile that any row sees, the number of tiles
    int cap;             // positions that exist
    int chunks, stride;  // the tiles in chunks; the items of a row group: these, and what it counts for besides
    int table;           // the sequence whose page table holds them
    int held;            // positions that another launch sees to
    __device__ int64_t pos0() const { return (int64_t)len - n; }  // of the first row
    __device__ int items(const AttendArgs& a) const { return groups * a.pool.heads * stride; }
};
template <int MODE = kWhole>
__device__ inline AttendSpan attend_span(const AttendArgs& a, const PlanOf<MODE>& p, int b) {
    AttendSpan r;
    if constexpr (MODE == kPrefix) {
        const int4 g = p.share.span[b];
        r.row0 = g.x, r.n = g.y, r.len = r.cap = g.z, r.table = g.w;
        r.first = p.share.first[b];
        r.held = 0;
    } else {
        const KvSpan s = span_of(a.seqs, b);
        r.row0 = (int)s.row0, r.n = s.n;
        r.len = (int)(s.pos0 + s.n);
        const int64_t held = (int64_t)a.seqs.max_pages << a.pool.page_shift;
        r.cap = r.len < 0 ? 0 : r.len > held ? (int)held : r.len;
        const int64_t lo = a.window > 0 ? r.pos0() - a.window + 1 : 0;
        r.first = lo < 0 ? 0 : (int)(lo >> 5);
        r.table = b;
        r.held = 0;
        if constexpr (MODE == kOwn) r.held = p.share.held[b];
        if (MODE == kOwn && r.first < r.held >> 5) r.first = r.held >> 5;  // (whole pages)
    }
    r.rows = r.n * a.group;
    r.groups = (int)(((int64_t)r.rows + (1 << p.group_shift) - 1) >> p.group_shift);
    r.tiles = (int)(((int64_t)r.cap + 31) >> 5) - r.first;
    if (r.tiles < 1) r.tiles = 1;  // rows that see nothing are written too
    r.chunks = (r.tiles + (1 << p.chunk_shift) - 1) >> p.chunk_shift;
    r.stride = r.chunks + (MODE == kOwn ? p.extra : 0);
    return r;
}
__device__ __forceinline__ int token_of(const AttendPlan& p, int row) {
    return (int)(((uint64_t)(uint32_t)row * p.group_magic) >> p.group_bits);
}

// The positions of the first and the last of rows r0 .. r0 + n - 1 of a sequence, of those of the least and the greatest one where
// rows of several sequences are together (all lanes of the wave take part); -1 for those before the first position.
struct AttendEnds {
    int least, most;
};
template <int MODE>
__device__ __forceinline__ AttendEnds ends_of(const PlanOf<MODE>& p, const AttendSpan& s, int r0, int n, int lane) {
    const int i0 = token_of(p, r0), i1 = token_of(p, r0 + n - 1);
    if constexpr (MODE == kPrefix) {
        int least = INT32_MAX, most = -1;
        for (int i = i0 + lane; i <= i1; i += 64) {
            const int pos = p.share.row_pos[s.row0 + i];
            least = pos < 0 ? least : min(least, pos);  // (rows that see nothing: nothing_seen)
            most = max(most, pos);
        }
        least = wave_reduce(least, [](int x, int y) { return min(x, y); });
        most = wave_reduce(most, [](int x, int y) { return max(x, y); });
        return {__builtin_amdgcn_readfirstlane(most < 0 ? -1 : least), __builtin_amdgcn_readfirstlane(most)};
    } else {
        const int64_t p0 = s.pos0() + i0, p1 = s.pos0() + i1;
        return {p0 < 0 ? -1 : (int)p0, p1 < 0 ? -1 : (int)p1};
    }
}

// Sum over this lane and the lanes below it.
__device__ __forceinline__ int wave_scan(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);  // row_shr:1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);  // the last lane of rows 0 and 2 to rows 1 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);  // lane 31 to the upper half
    return x;
}

// The range of items of a worker: the sequence in which it begins, the items before that sequence, the range, and
// the items of a full range (a multiple of `grain`, and `least` or more).  All threads take part, a thread a sequence.
struct AttendRange {
    int b, before, at, end, per;
};
template <int WAVES, int MODE = kWhole>
__device__ __forceinline__ AttendRange attend_range(const AttendArgs& a, const PlanOf<MODE>& p, int worker, int grain, int least) {
    constexpr int THREADS = 64 * WAVES;
    __shared__ int total_of[WAVES], found[2], longest_of[WAVES];
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
    int n_seq = a.seqs.n_seq;
    if constexpr (MODE == kPrefix) n_seq = p.share.n_groups;
    int own = 0, sum = 0, all = 0, b = tid, longest = 1;
    // items up to sequence b within a round of THREADS (sum), and of the round (returned)
    auto scan = [&]() {
        int chunks = 0;
        own = 0;
        if (b < n_seq) {
            const AttendSpan s = attend_span<MODE>(a, p, b);
            own = s.items(a);
            chunks = own > 0 ? s.chunks : 0;
        }
        sum = wave_scan(own);
        const int length = __any(chunks > 2) ? 4 : __any(chunks == 2) ? 2 : 1;  // of a row group, up to 4
        __syncthreads();
        if (lane == 63) total_of[wid] = sum, longest_of[wid] = length;
        __syncthreads();
        int round = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const int t = total_of[w];
            sum += w < wid ? t : 0;
            round += t;
            longest = max(longest, longest_of[w]);
        }
        return round;
    };
    for (; b - tid < n_seq; b += THREADS) all += scan();
    all = __builtin_amdgcn_readfirstlane(all);
    AttendRange r;
    r.per = (int)(((uint32_t)all + (uint32_t)p.workers - 1) / (uint32_t)p.workers);
    // (no multiple of more than a row group has: a workgroup would get several of them)
    longest = __builtin_amdgcn_readfirstlane(longest);
    grain = grain < longest ? grain : longest;
    r.per = r.per < least ? least : r.per;
    r.per = (r.per + grain - 1) & ~(grain - 1);
    const int64_t at = (int64_t)worker * r.per;
    r.at = at < all ? (int)at : all;
    r.end = at + r.per < all ? (int)(at + r.per) : all;
    // the thread whose sequence holds item `at` finds it
    int before = 0;
    for (b = tid; b - tid < n_seq; b += THREADS) {
        const int round = n_seq > THREADS ? scan() : all;
        if (r.at >= before + sum - own && r.at < before + sum) {
            found[0] = b;
            found[1] = before + sum - own;
        }
        before += round;
    }
    __syncthreads();
    r.b = __builtin_amdgcn_readfirstlane(found[0]);
    r.before = __builtin_amdgcn_readfirstlane(found[1]);
    return r;
}

// Moves on to the next chunk of a worker's range: past sequences that are through and those without rows, and past the items
// behind a row group's chunks.  Whether there is one.
template <int MODE>
__device__ __forceinline__ bool attend_next(const AttendArgs& a, const PlanOf<MODE>& p, AttendRange& r, AttendSpan& s) {
    while (r.at < r.end) {
        const int items = s.items(a);
        if (r.at - r.before >= items) {
            r.before += items;
            do s = attend_span<MODE>(a, p, ++r.b);
            while (s.n == 0);
        }
        if (MODE != kOwn) return true;
        const int rel = r.at - r.before, c0 = rel - (int)((uint32_t)rel / (uint32_t)s.stride) * s.stride;
        if (c0 < s.chunks) return true;
        r.at += s.stride - c0;
    }
    return false;
}

// 16 bytes a lane from a tile whose bytes past `size` (0: there is no tile) are not read and come as zeros.  With few rows
// keys and values are read once (ONCE): non-temporal loads are 12 % faster (131,071 tokens 89 us, 102 without; 256 sequences of 512 to
// 2048 tokens, 16 heads of 64 columns 191 us, 214).
__device__ __forceinline__ __amdgpu_buffer_rsrc_t tile_rsrc(const void* p, int size) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, size, 0x00020000);
}
// (The constant part of an offset fits in the instruction up to 4095 bytes; whole 4 KB go into a scalar register.)
template <bool ONCE = true>
__device__ __forceinline__ u32x4 tile_load(__amdgpu_buffer_rsrc_t r, int at, int lane_offset) {
    return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, lane_offset + (at & 4095), at & ~4095, ONCE ? 2 : 0));
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

// The scale of the scores in units of log2 e, always above 0 (its sign and its being 0 are in the queries: load_q).
__device__ __forceinline__ float scale_of(const AttendArgs& a) {
    return a.scale == 0.0f ? 1.0f : fabsf(a.scale) * kLog2e;
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
    static constexpr int BYTES_TILE = 32 * DP * (BYTES ? 1 : 2);

    u32x4 q[R][KC][NT];
    f32x4 o[R][NJ];
    float m[R], l[R];
    int hi[R], lo[R];  // the positions that the lane's row sees
    struct Tile {
        u32x4 k[NL], v[NL];
        f32x4 ks[2], vs[2];
        int index;
    };

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            m[r] = -__builtin_inff();
            l[r] = 0.0f;
#pragma unroll
            for (int j = 0; j < NJ; ++j) o[r][j] = f32x4{0, 0, 0, 0};
        }
    }
    // Rows of no position among others' (kPrefix): what they summed up is left out, so that the others' tiles need not be hidden
    // from them.
    __device__ __forceinline__ void nothing_seen() {
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (hi[r] < 0) {
                m[r] = -__builtin_inff();
                l[r] = 0.0f;
#pragma unroll
                for (int j = 0; j < NJ; ++j) o[r][j] = f32x4{0, 0, 0, 0};
            }
    }
    // every lane's sum over the tokens of the four lane groups
    __device__ __forceinline__ void reduce() {
        auto add2 = [](float x, float y) { return x + y; };
#pragma unroll
        for (int r = 0; r < R; ++r) l[r] = xor_combine<16>(xor_combine<32>(l[r], add2), add2);
    }

    // 16 bytes of a row as KC operands: the three terms of a float32 sum back to it exactly, a bfloat16 is its own
    // Row tile r is rows row0 + step r .. + 15 of the sequence's (its last row in the place of those that it has not).
    template <int MODE = kWhole>
    __device__ __forceinline__ void load_q(const AttendArgs& a, const PlanOf<MODE>& p, const AttendSpan& s, int h, int row0,
                                           int step, int lane) {
        const int u = lane >> 4;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            int row = row0 + step * r + (lane & 15);
            row = row < s.rows ? row : s.rows - 1;
            const int i = token_of(p, row), head = h * a.group + (row - i * a.group);
            int64_t pos;
            if constexpr (MODE == kPrefix) pos = p.share.row_pos[s.row0 + i];
            else pos = s.pos0() + i;
            hi[r] = pos < 0 ? -1 : (int)pos;
            lo[r] = a.window > 0 && hi[r] - a.window + 1 > 0 ? hi[r] - a.window + 1 : 0;
            if (MODE == kOwn) lo[r] = lo[r] > s.held ? lo[r] : s.held;
            const char* src = a.q + (((int64_t)s.row0 + i) * a.q_row + (int64_t)head * a.pool.d) * ESZ;
#pragma unroll
            for (int c = 0; c < KC; ++c) {
                const int col = 32 * c + 8 * u;
                const bool in = col < a.pool.d;  // d is a multiple of 8
                const char* at = src + (in ? col : 0) * ESZ;
                u32x4 t[NT] = {};
                if constexpr (F32) {
                    const f32x4 x = *(const f32x4_any*)at, y = *(const f32x4_any*)(at + 16);
                    split2<NT>(x[0], x[1], t, 0);
                    split2<NT>(x[2], x[3], t, 1);
                    split2<NT>(y[0], y[1], t, 2);
                    split2<NT>(y[2], y[3], t, 3);
                } else {
                    t[0] = *(const u32x4_any*)at;
                }
#pragma unroll
                for (int k = 0; k < NT; ++k)
#pragma unroll
                    for (int e = 0; e < 4; ++e)  // a negative scale's sign, and a scale of 0, go into the queries
                        q[r][c][k][e] = in && a.scale != 0.0f ? t[k][e] ^ (a.scale < 0.0f ? 0x80008000u : 0u) : 0u;
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

    static __device__ __forceinline__ void load_k(Tile& t, const AttendArgs& a, int64_t place, int there, int lane) {
        const auto r = tile_rsrc(a.pool.k + place * BYTES_TILE, there * BYTES_TILE);
#pragma unroll
        for (int i = 0; i < NL; ++i) t.k[i] = tile_load(r, i * 1024, lane * 16);
        if constexpr (BYTES) {
            const auto rs = tile_rsrc(a.pool.k_scale + place * 32, there * 128);
#pragma unroll
            for (int b = 0; b < 2; ++b) t.ks[b] = __builtin_bit_cast(f32x4, tile_load(rs, 64 * b, (lane >> 4) * 16));
        }
    }
    static __device__ __forceinline__ void load_v(Tile& t, const AttendArgs& a, int64_t place, int there, int lane) {
        const auto r = tile_rsrc(a.pool.v + place * BYTES_TILE, there * BYTES_TILE);
#pragma unroll
        for (int i = 0; i < NL; ++i) t.v[i] = tile_load(r, i * 1024, lane * 16);
        if constexpr (BYTES) {
            const auto rs = tile_rsrc(a.pool.v_scale + place * 32, there * 128);
#pragma unroll
            for (int b = 0; b < 2; ++b) t.vs[b] = __builtin_bit_cast(f32x4, tile_load(rs, 64 * b, (lane >> 4) * 16));
        }
    }

    static __device__ __forceinline__ u32x4 k_operand(const Tile& t, int b, int c) {
        if constexpr (!BYTES) return t.k[2 * c + b];
        else return widen8<CT>(t.k[c][2 * b], t.k[c][2 * b + 1]);
    }
    static __device__ __forceinline__ u32x4 v_operand(const Tile& t, int j) {
        if constexpr (!BYTES) return t.v[j];
        else return widen8<CT>(t.v[j >> 1][2 * (j & 1)], t.v[j >> 1][2 * (j & 1) + 1]);
    }

    // scores of a tile: with 8-bit keys in units of log2 e, with bfloat16 ones before their scaling
    __device__ __forceinline__ void scores(const Tile& t_, f32x4 (&s)[R][2], float scale2) {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int b = 0; b < 2; ++b) s[r][b] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int c = 0; c < KC; ++c)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const u32x4 k = k_operand(t_, b, c);
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int t = NT - 1; t >= 0; --t) s[r][b] = mfma16x16x32(k, q[r][c][t], s[r][b]);
            }
        if constexpr (BYTES) {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const f32x4 f = t_.ks[b] * scale2;
#pragma unroll
                for (int r = 0; r < R; ++r) s[r][b] *= f;
            }
        }
    }

    // Hides the positions that a row does not see, and the values of those that no row of the wave sees (first .. last
    // are seen by one): what lies there may be anything.
    __device__ __forceinline__ void hide(Tile& t, int index, f32x4 (&s)[R][2], int first, int last, int lane) {
        const int t0 = 32 * index + 4 * (lane >> 4);
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
                if constexpr (BYTES) t.vs[b][i] = keep[i] ? t.vs[b][i] : 0.0f;
            }
            if constexpr (BYTES) {
                const uint32_t w = (keep[0] & 0xFFu) | (keep[1] & 0xFF00u) | (keep[2] & 0xFF0000u) | (keep[3] & 0xFF000000u);
#pragma unroll
                for (int i = 0; i < NL; ++i) {
                    t.v[i][b] &= w;
                    t.v[i][2 + b] &= w;
                }
            } else {
                const uint32_t w0 = (keep[0] & 0xFFFFu) | (keep[1] & 0xFFFF0000u),
                               w1 = (keep[2] & 0xFFFFu) | (keep[3] & 0xFFFF0000u);
#pragma unroll
                for (int i = 0; i < NL; ++i) {
                    t.v[i][2 * b] &= w0;
                    t.v[i][2 * b + 1] &= w1;
                }
            }
        }
    }

    // Weights of the tile (s becomes P), the running maximum and sum.  The sum stays a lane's own until the end.  Scores
    // are in units of log2 e times 1 / scale2 (8-bit keys: scaled already).
    template <int RA = R>
    __device__ __forceinline__ void weigh(f32x4 (&s)[R][2], float scale2) {
        auto max2 = [](float x, float y) { return fmaxf(x, y); };
        const float c = BYTES ? 1.0f : scale2;
        float x[RA];
        bool raise = false;
#pragma unroll
        for (int r = 0; r < RA; ++r) {
            float y = fmaxf(s[r][0][0], s[r][1][0]);
#pragma unroll
            for (int i = 1; i < 4; ++i) y = fmaxf(fmaxf(y, s[r][0][i]), s[r][1][i]);
            x[r] = c * xor_combine<16>(xor_combine<32>(y, max2), max2);
            raise |= x[r] > m[r] + kSlack;  // (from -infinity too)
        }
        if (__any(raise)) {
#pragma unroll
            for (int r = 0; r < RA; ++r) {
                const float to = fmaxf(x[r], m[r]);
                const float f = to > m[r] ? __builtin_amdgcn_exp2f(m[r] - to) : 1.0f;  // 0 where m was -infinity
                l[r] *= f;
#pragma unroll
                for (int j = 0; j < NJ; ++j) o[r][j] *= f;
                m[r] = to;
            }
        }
#pragma unroll
        for (int r = 0; r < RA; ++r) {
            const float base = m[r] == -__builtin_inff() ? 0.0f : m[r];
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[r][b][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r][b][i], c, -base));
                    l[r] += s[r][b][i];
                }
        }
    }

    // Values that are no numbers.  0 times an infinity or a NaN is NaN, so in a tile that some rows see more of than others
    // they must not meet the weight 0 of a row that does not see their token.  They are taken out of such tiles (hide,
    // put_tile in attend_wide.hpp), and if there were any, the rows that see them are made NaN when the segment is through,
    // by another look at its tiles and a product (is no number) times (is seen).
    //
    // The top bits of a dword's elements that are no numbers: of two bfloat16, of the cache's type (no integer is none);
    // without: the dword without them.
    static __device__ __forceinline__ uint32_t no_numbers(uint32_t w) {
        return ((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u;
    }
    static __device__ __forceinline__ uint32_t no_codes(uint32_t w) {
        if constexpr (CT == kKvInt8) return 0;
        return CT == kKvFp8 ? ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u : no_numbers(w);
    }
    static __device__ __forceinline__ uint32_t without(uint32_t w, uint32_t n) {
        return w & ~(n | (n - (n >> (CT == kKvFp8 ? 7 : 15))));
    }
    static __device__ __forceinline__ bool no_scale(float x) { return (__float_as_uint(x) & 0x7F800000u) == 0x7F800000u; }
    // Whether rows see more of a tile than others: seen0 .. seen1 are seen by one of them, all0 .. all1 by every one.
    static __device__ __forceinline__ bool mixed(int index, int seen0, int seen1, int all0, int all1) {
        return (seen0 < all0 && 32 * index < all0) || (seen1 > all1 && 32 * index + 31 > all1);
    }
    // Takes them out of a tile; whether there were any.
    static __device__ __forceinline__ uint32_t take_out(Tile& t) {
        uint32_t some = 0;
#pragma unroll
        for (int i = 0; i < NL; ++i)
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                const uint32_t n = no_codes(t.v[i][d]);
                t.v[i][d] = without(t.v[i][d], n);
                some |= n;
            }
        if constexpr (BYTES) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    some |= no_scale(t.vs[b][i]);
                    t.vs[b][i] = no_scale(t.vs[b][i]) ? 0.0f : t.vs[b][i];
                }
        }
        return some;
    }
    // The mixed tiles t0, t0 + step, ... < t1 of a segment: rows that see what is no number become NaN in its column.
    __device__ __forceinline__ void spoil(const AttendArgs& a, const int32_t* pages, int h, int first, int t0, int t1, int step,
                                          int seen0, int seen1, int all0, int all1, int lane) {
        const int shift = a.pool.page_shift - 5;
#pragma unroll 1
        for (int t = t0; t < t1; t += step) {
            const int index = first + t;
            if (32 * index > seen1 || 32 * index + 31 < seen0 || !mixed(index, seen0, seen1, all0, all1)) continue;
            const int64_t page = __builtin_amdgcn_readfirstlane(pages[index >> shift]);
            if (page < 0 || page >= a.pool.n_pages) continue;
            const int64_t place = ((page * a.pool.heads + h) << shift) + (index & ((1 << shift) - 1));
            const auto values = tile_rsrc(a.pool.v + place * BYTES_TILE, BYTES_TILE);
            u32x4 seen[R], odd{};
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int j = 32 * index + 16 * (e >> 2) + 4 * (lane >> 4) + (e & 3);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const uint32_t one = j >= lo[r] && j <= hi[r] ? 0x3F80u << (16 * (e & 1)) : 0u;
                    seen[r][e >> 1] = e & 1 ? seen[r][e >> 1] | one : one;
                }
                if constexpr (BYTES)
                    odd[e >> 1] |= no_scale(a.pool.v_scale[place * 32 + (j & 31)]) ? 0x4000u << (16 * (e & 1)) : 0u;
            }
            // (a few loads at a time, for the registers)
            constexpr int G = BYTES ? 2 : 8, EACH = BYTES ? 2 : 1;
#pragma unroll
            for (int i0 = 0; i0 < NL; i0 += G) {
                Tile x;
#pragma unroll
                for (int i = i0; i < i0 + G && i < NL; ++i) x.v[i] = tile_load(values, i * 1024, lane * 16);
#pragma unroll
                for (int j = EACH * i0; j < EACH * (i0 + G) && j < NJ; ++j) {
                    const u32x4 v = v_operand(x, j);
                    u32x4 none;  // twos (0x4000), from the value or from the token's scale
#pragma unroll
                    for (int d = 0; d < 4; ++d) none[d] = no_numbers(v[d]) >> 1 | odd[d];
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        const f32x4 hit = mfma16x16x32(none, seen[r], f32x4{0, 0, 0, 0});
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[r][j][i] = hit[i] > 0.0f ? __builtin_nanf("") : o[r][j][i];
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }

    // f(i, operand i) for COUNT operands in LDS, `at` this lane's 16 bytes of the first: G are read while the last G are
    // worked with, and no more (the compiler would read them all, and keep sums in scratch memory for it).
    template <int COUNT, class F>
    static __device__ __forceinline__ void each_operand(const u32x4* at, F f) {
        constexpr int G = COUNT % 4 == 0 ? 4 : 3;
        static_assert(COUNT % G == 0, "whole groups");
        u32x4 x[2][G];
#pragma unroll
        for (int g = 0; g < G; ++g) x[0][g] = at[g * 64];
#pragma unroll
        for (int i = 0; i < COUNT; i += G) {
            if (i + G < COUNT) {
#pragma unroll
                for (int g = 0; g < G; ++g) x[(i / G + 1) & 1][g] = at[(i + G + g) * 64];
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int g = 0; g < G; ++g) f(i + g, x[(i / G) & 1][g]);
        }
    }
    // scores, hide and gather for the first RA row tiles with a tile of operands in LDS (attend_wide.hpp): `k` and `v` this
    // lane's 16 bytes of the first, `ks` and `vs` the scales of the tile's 32 tokens.
    template <int RA>
    __device__ __forceinline__ void scores_lds(const u32x4* k, const f32x4* ks, int u, f32x4 (&s)[R][2], float scale2) {
#pragma unroll
        for (int r = 0; r < RA; ++r)
#pragma unroll
            for (int b = 0; b < 2; ++b) s[r][b] = f32x4{0, 0, 0, 0};
        each_operand<2 * KC>(k, [&](int i, u32x4 x) {
            const int c = i / 2, b = i % 2;
#pragma unroll
            for (int r = 0; r < RA; ++r)
#pragma unroll
                for (int t = NT - 1; t >= 0; --t) s[r][b] = mfma16x16x32(x, q[r][c][t], s[r][b]);
        });
        if constexpr (BYTES) {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const f32x4 f = ks[4 * b + u] * scale2;
#pragma unroll
                for (int r = 0; r < RA; ++r) s[r][b] *= f;
            }
        }
    }
    template <int RA>
    __device__ __forceinline__ void hide_scores(int index, f32x4 (&s)[R][2], int lane) {
        const int t0 = 32 * index + 4 * (lane >> 4);
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int j = t0 + 16 * b + i;
#pragma unroll
                for (int r = 0; r < RA; ++r)
                    s[r][b][i] = j >= lo[r] && j <= hi[r] ? s[r][b][i] : -__builtin_inff();
            }
    }
    template <int RA>
    __device__ __forceinline__ void round_lds(const f32x4 (&s)[R][2], const f32x4* vs, int u, u32x4 (&p)[R][NP]) {
#pragma unroll
        for (int r = 0; r < RA; ++r)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                f32x4 x = s[r][b];
                if constexpr (BYTES) x *= vs[4 * b + u];
                split2<NP>(x[0], x[1], p[r], 2 * b);
                split2<NP>(x[2], x[3], p[r], 2 * b + 1);
            }
    }
    template <int RA>
    __device__ __forceinline__ void gather_lds(const u32x4* v, const u32x4 (&p)[R][NP]) {
        each_operand<NJ>(v, [&](int j, u32x4 x) {
#pragma unroll
            for (int t = NP - 1; t >= 0; --t)
#pragma unroll
                for (int r = 0; r < RA; ++r) o[r][j] = mfma16x16x32(x, p[r][t], o[r][j]);
        });
    }

    // O^T += V^T P^T
    __device__ __forceinline__ void gather(const Tile& t_, f32x4 (&s)[R][2]) {
        u32x4 p[R][NP];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float x = s[r][e >> 1][2 * (e & 1)], y = s[r][e >> 1][2 * (e & 1) + 1];
                if constexpr (BYTES) {
                    x *= t_.vs[e >> 1][2 * (e & 1)];
                    y *= t_.vs[e >> 1][2 * (e & 1) + 1];
                }
                split2<NP>(x, y, p[r], e);
            }
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            const u32x4 v = v_operand(t_, j);
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int t = NP - 1; t >= 0; --t) o[r][j] = mfma16x16x32(v, p[r][t], o[r][j]);
        }
    }
};

// Four columns of the result, from element `at` on.
template <bool F32>
__device__ __forceinline__ void store4(const AttendArgs& a, int64_t at, f32x4 x) {
    if (F32) *(f32x4_any*)((float*)a.out + at) = x;
    else *(u32x2_any*)((uint16_t*)a.out + at) = u32x2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
}

__device__ __forceinline__ float lse_of(float m, float l) {
    return l == 0.0f ? -__builtin_inff() : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// Where a worker's part lies: its second slot if the row group goes on after it.
__device__ __forceinline__ int64_t part_of(const AttendPlan& p, int worker, bool goes_on) {
    return (2 * (int64_t)worker + (goes_on ? 1 : 0)) << p.group_shift;
}

struct Joined {
    float m = -__builtin_inff(), l = 0.0f;
    f32x4 o{0, 0, 0, 0};
    __device__ __forceinline__ void add(float m2, float l2, f32x4 o2) {
        if (m2 == -__builtin_inff() && l2 == 0.0f) return;  // nothing was seen (scores that are all NaN raise no maximum)
        const float M = fmaxf(m, m2);
        const float f = __builtin_amdgcn_exp2f(m - M), g = __builtin_amdgcn_exp2f(m2 - M);
        l = l * f + l2 * g;
        o = o * f + o2 * g;
        m = M;
    }
};

// Four columns of element `at` of a part's sums, and where they lie.
template <int MODE>
__device__ __forceinline__ void store_sums(const PlanOf<MODE>& p, int64_t at, int dp, int col, f32x4 o, float m, float l) {
    const AttendSums& x = p.share.sums[MODE - kPrefix];
    *(f32x4*)(x.o + at * dp + col) = o;
    if (col == 0) x.ml[at] = make_float2(m, l);
}
template <int MODE>
__device__ __forceinline__ void store_place(const PlanOf<MODE>& p, int64_t at, int parts, int worker0, int place) {
    p.share.sums[MODE - kPrefix].at[at] = make_int2(parts, worker0 | place << 16);
}

__device__ __forceinline__ void store_joined(const AttendArgs& a, const AttendPlan& p, const AttendSplit& s, int row,
                                             int col, const Joined& x) {
    const int r = s.row + row, i = token_of(p, r);
    const int64_t at = ((int64_t)s.seq_row0 + i) * a.q_heads + s.head0 + (r - i * a.group);
    const f32x4 o = x.o * (x.l == 0.0f ? 0.0f : 1.0f / x.l);
    if (col < a.pool.d) {
        if (a.dtype == 0) store4<true>(a, at * a.pool.d + col, o);
        else store4<false>(a, at * a.pool.d + col, o);
    }
    if (col == 0 && a.lse) a.lse[at] = lse_of(x.m, x.l);
}

// Joins the parts of a row group: of_row groups (a power of two) of dp / 4 lanes on a row, four parts loaded together.  The
// workgroup takes rows first, first + 1, ... as many as it has lane groups for, and again from `step` times as many on.
// load(part's first row + row, column, ml, o) loads four columns.  scratch: THREADS f32x4 and float2 of LDS.
template <int THREADS, class Load>
__device__ __forceinline__ void join_rows(const AttendArgs& a, const AttendPlan& p, const AttendSplit& s, int dp, int of_row, int tid,
                                          int first, int step, f32x4* scratch, Load load) {
    const int lanes = dp / 4, groups = THREADS / lanes;
    const int rows = groups / of_row, g = tid / lanes, col = tid % lanes * 4, sub = g % of_row;
    float2* ml_of = (float2*)(scratch + THREADS);
    for (int row0 = first * rows; row0 < s.n_rows; row0 += step * rows) {
        const int row = row0 + g / of_row;
        const bool live = g < rows * of_row && row < s.n_rows;
        Joined x;
        if (live)
            for (int k0 = sub; k0 < s.parts; k0 += 4 * of_row) {
                float2 ml[4];
                f32x4 o[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int k = k0 + u * of_row < s.parts ? k0 + u * of_row : s.parts - 1;
                    load(part_of(p, s.worker0 + k, k < s.parts - 1) + row, col, ml[u], o[u]);
                }
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (k0 + u * of_row < s.parts) x.add(ml[u].x, ml[u].y, o[u]);
            }
        if (of_row > 1) {
            ml_of[tid] = make_float2(x.m, x.l);
            scratch[tid] = x.o;
            __syncthreads();
            if (sub == 0 && live)
                for (int k = 1; k < of_row; ++k)
                    x.add(ml_of[tid + k * lanes].x, ml_of[tid + k * lanes].y, scratch[tid + k * lanes]);
            __syncthreads();
        }
        if (live && sub == 0) store_joined(a, p, s, row, col, x);
    }
}

// ---------------------------------------------------------------------------
// The join within the launch, for small calls (AttendPlan::join_here).  Parts are written and read with device-wide (sc1)
// accesses alone, so the hand-over of last_workgroup_wait holds for them: every workgroup of a row group waits for its
// stores, counts itself, and the one that counts last reads all parts and leaves the counter at 0.  Nobody waits for
// another.
// ---------------------------------------------------------------------------
constexpr int kDeviceWide = 16;  // the sc1 bit of a buffer access

template <int DP>
__device__ __forceinline__ void store_part(const AttendPlan& p, int64_t part, int row, int col, f32x4 x) {
    const auto r = __builtin_amdgcn_make_buffer_rsrc(p.part_o + part * DP, 0, DP * 4 << p.group_shift, 0x00020000);
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, x), r, (row * DP + col) * 4, 0, kDeviceWide);
}
__device__ __forceinline__ void store_part_ml(const AttendPlan& p, int64_t part, int row, float m, float l) {
    const auto r = __builtin_amdgcn_make_buffer_rsrc(p.part_ml + part, 0, 8 << p.group_shift, 0x00020000);
    __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(m), __float_as_uint(l)}, r, row * 8, 0, kDeviceWide);
}

// After a workgroup's part of a row group has been stored: counts it, and joins the parts if it is the last.  scratch:
// THREADS f32x4 and float2 of LDS that nothing else uses meanwhile.
template <int THREADS, int DP>
__device__ __forceinline__ void join_parts(const AttendArgs& a, const AttendPlan& p, const AttendSplit& s,
                                           f32x4* scratch) {
    __shared__ int last;
    const int tid = fresh_lane() + (__builtin_amdgcn_readfirstlane(threadIdx.x >> 6) << 6);  // (nothing kept from before)
    last_workgroup_wait();
    __syncthreads();
    if (tid == 0) {
        uint32_t* done = p.done + s.worker0;
        last = __hip_atomic_fetch_add(done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)s.parts - 1;
        if (last) __hip_atomic_store(done, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!last) return;
    // (all rows at once where they are few; a choice by the parts too costs more than it gains here)
    int of_row = 1;
    while (2 * of_row * s.n_rows <= THREADS / (DP / 4)) of_row *= 2;
    join_rows<THREADS>(a, p, s, DP, of_row, tid, 0, 1, scratch, [&](int64_t at, int col, float2& ml, f32x4& o) {
        auto load8 = [](const void* from) {
            const uint64_t w = __hip_atomic_load((const uint64_t*)from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            return make_float2(__uint_as_float((uint32_t)w), __uint_as_float((uint32_t)(w >> 32)));
        };
        ml = load8(p.part_ml + at);
        const float2 x = load8(p.part_o + at * DP + col), y = load8(p.part_o + at * DP + col + 2);
        o = f32x4{x.x, x.y, y.x, y.y};
    });
}

// A worker of four waves.  HERE: parts are joined within the launch.
template <int DP, int CT, int R, bool F32, bool HERE, int MODE>
__device__ __forceinline__ void attend_narrow(const AttendArgs& a, const PlanOf<MODE>& p, const int worker) {
    using A = Attend<DP, CT, R, F32>;
    constexpr int GR = 16 * R;  // rows of a row group
    __shared__ float2 sml[4][GR];
    __shared__ float so[4][16][A::CB + 4];
    const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid >> 6);

    AttendRange range = attend_range<4, MODE>(a, p, worker, 4 >> (p.chunk_shift < 2 ? p.chunk_shift : 2), 1);
    if (range.at >= range.end) {
        if (MODE == kWhole && !HERE && tid == 0) p.split[worker].n_rows = 0;
        return;
    }
    AttendSplit split{};
    const float scale2 = scale_of(a);
    const int tile_shift = a.pool.page_shift - 5;

    // A segment: tiles tile0 .. tile1 - 1 of one row group
    struct Segment {
        int h, rg, tile0, tile1, row0, rows, n_rows;  // n_rows: rows in the group
        int first, table, item0, items;               // the row group's first item, its items
        bool starts, ends;                            // whether it holds the first and the last tile
        int seen0, seen1, all0, all1;                 // positions that one of the rows, that every row sees
    };
    A w;
    typename A::Tile tile;
    int there = 0;
    Segment g;
    int page = -1, t0 = 0;
    uint64_t todo = 0;
    AttendSpan s = attend_span<MODE>(a, p, range.b);

    // the wave's tiles t0, t0 + 4, ... of the segment, a lane each: which of them are there and seen
    auto load_pages = [&]() {
        const int t = t0 + lane * 4, mine = g.first + t;
        page = -1;
        if (t < g.tile1 && 32 * mine <= g.seen1 && 32 * mine + 31 >= g.seen0)
            page = (a.seqs.pages + (int64_t)g.table * a.seqs.max_pages)[mine >> tile_shift];
    };
    auto look = [&]() { todo = __ballot(page >= 0 && page < a.pool.n_pages); };
    // the wave's next tile, if there is one
    auto next = [&]() {
        while (!todo && t0 + 256 < g.tile1) {
            t0 += 256;
            load_pages();
            look();
        }
        there = todo ? 1 : 0;
        const int k = there ? __ffsll((unsigned long long)todo) - 1 : 0;
        todo &= todo - 1;
        tile.index = g.first + t0 + k * 4;
        const int64_t pg = there ? __builtin_amdgcn_readlane(page, k) : 0;
        return ((pg * a.pool.heads + g.h) << tile_shift) + (tile.index & ((1 << tile_shift) - 1));
    };
    // the segment that begins at item `at`, its queries and its first tiles
    auto open = [&]() {
        const int rel = range.at - range.before;
        const int unit = (int)((uint32_t)rel / (uint32_t)s.stride), c0 = rel - unit * s.stride;
        g.h = (int)((uint32_t)unit / (uint32_t)s.groups);
        g.rg = unit - g.h * s.groups;
        const int left = range.end - range.at, c1 = s.chunks - c0 <= left ? s.chunks : c0 + left;
        range.at += c1 - c0;
        g.item0 = range.before + unit * s.stride;
        g.items = s.chunks;
        g.starts = c0 == 0;
        g.ends = c1 == s.chunks;
        g.tile0 = c0 << p.chunk_shift;
        g.tile1 = g.ends ? s.tiles : c1 << p.chunk_shift;
        const int r0 = g.rg << p.group_shift;
        g.row0 = s.row0, g.rows = s.rows, g.first = s.first, g.table = s.table;
        g.n_rows = s.rows - r0 < GR ? s.rows - r0 : GR;
        const AttendEnds ends = ends_of<MODE>(p, s, r0, g.n_rows, lane);
        const int q0 = ends.least, q1 = ends.most;
        g.seen0 = a.window > 0 && q0 - a.window + 1 > 0 ? q0 - a.window + 1 : 0;
        g.all0 = a.window > 0 && q1 - a.window + 1 > 0 ? q1 - a.window + 1 : 0;
        if (MODE == kOwn) g.seen0 = max(g.seen0, s.held), g.all0 = max(g.all0, s.held);
        g.seen1 = q1 < s.cap - 1 ? q1 : s.cap - 1;
        g.all1 = q0 < g.seen1 ? q0 : g.seen1;
        t0 = g.tile0 + wid;
        load_pages();
        w.template load_q<MODE>(a, p, s, g.h, r0, 16, lane);  // while the page numbers are on their way
        __builtin_amdgcn_sched_barrier(0);
        look();
        const int64_t pl = next();
        A::load_k(tile, a, pl, there, lane);
        A::load_v(tile, a, pl, there, lane);
        __builtin_amdgcn_sched_barrier(0);
    };
    if (MODE == kOwn && !attend_next<MODE>(a, p, range, s)) {
        return;
    }
    open();
    bool more = true;
    while (more) {
        w.clear();
        int odd = 0;  // whether something that is no number was taken out
        while (there) {
            f32x4 sc[R][2];
            w.scores(tile, sc, scale2);
            const int index = tile.index;
            if (A::mixed(index, g.seen0, g.seen1, g.all0, g.all1)) {
                const uint32_t some = A::take_out(tile);
                odd = __any(some != 0) ? 1 : odd;
            }
            const int64_t pl = next();  // its keys are loaded under this tile's weights, its values under its scores
            A::load_k(tile, a, pl, there, lane);
            if (32 * index < g.all0 || 32 * index + 31 > g.all1) w.hide(tile, index, sc, g.seen0, g.seen1, lane);
            w.weigh(sc, scale2);
            w.gather(tile, sc);
            A::load_v(tile, a, pl, there, lane);
        }

        if (odd)
            w.spoil(a, a.seqs.pages + (int64_t)g.table * a.seqs.max_pages, g.h, g.first, g.tile0 + wid, g.tile1, 4, g.seen0, g.seen1,
                    g.all0, g.all1, lane);
        // The next segment's loads are on their way while this one's results are joined and stored.
        const Segment old = g;
        if (MODE == kPrefix) w.nothing_seen();
        w.reduce();
        more = attend_next<MODE>(a, p, range, s);
        if (more) open();
        const bool whole = old.starts && old.ends;
        const int64_t part = part_of(p, worker, !old.ends);
        AttendSplit u0{};
        if (!whole) {
            const int first = (int)((uint32_t)old.item0 / (uint32_t)range.per);
            const int end = (int)((uint32_t)(old.item0 + old.items - 1) / (uint32_t)range.per);
            u0 = AttendSplit{old.row0, old.h * a.group, old.rg * GR, old.n_rows, first, end - first + 1, {}};
            if (old.ends) split = u0;
        }
        if constexpr (MODE != kWhole) {
            if (old.ends && tid < old.n_rows) {
                const int r = old.rg * GR + tid, i = token_of(p, r);
                store_place<MODE>(p, ((int64_t)old.row0 + i) * a.q_heads + old.h * a.group + (r - i * a.group), whole ? 0 : u0.parts,
                                  u0.worker0, tid);
            }
        }
        // four columns of a row of the group; its maximum and sum with the first of them
        auto put = [&](int row, int col, f32x4 x, float m, float l) {
            if (!whole) {
                if constexpr (HERE) {
                    store_part<DP>(p, part, row, col, x);
                    if (col == 0) store_part_ml(p, part, row, m, l);
                } else {
                    *(f32x4*)(p.part_o + (part + row) * DP + col) = x;
                    if (col == 0) p.part_ml[part + row] = make_float2(m, l);
                }
                return;
            }
            const int r = old.rg * GR + row, i = token_of(p, r), head = old.h * a.group + (r - i * a.group);
            const int64_t at = ((int64_t)old.row0 + i) * a.q_heads + head;
            if constexpr (MODE != kWhole) {
                store_sums<MODE>(p, at, DP, col, x, m, l);
                return;
            }
            if (col < a.pool.d) store4<F32>(a, at * a.pool.d + col, x * (l == 0.0f ? 0.0f : 1.0f / l));
            if (col == 0 && a.lse) a.lse[at] = lse_of(m, l);
        };
        const int n = lane & 15, u = lane >> 4;
        lds_barrier();  // the last segment's have been read
        if (u == 0) {
#pragma unroll
            for (int r = 0; r < R; ++r) sml[wid][16 * r + n] = make_float2(w.m[r], w.l[r]);
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c0 = 0; c0 < DP; c0 += A::CB) {
                if (r + c0 > 0) lds_barrier();
                if (16 * r + n < old.n_rows) {
#pragma unroll
                    for (int j = 0; j < A::CB / 16; ++j) *(f32x4*)&so[wid][n][16 * j + 4 * u] = w.o[r][c0 / 16 + j];
                }
                lds_barrier();
                const int rows = old.n_rows - 16 * r < 16 ? old.n_rows - 16 * r : 16;
                for (int e = tid; e < rows * (A::CB / 4); e += 256) {
                    const int col = e % (A::CB / 4) * 4, row = e / (A::CB / 4);
                    float2 ml[4];
#pragma unroll
                    for (int t = 0; t < 4; ++t) ml[t] = sml[t][16 * r + row];
                    const float M = fmaxf(fmaxf(ml[0].x, ml[1].x), fmaxf(ml[2].x, ml[3].x));
                    const float base = M == -__builtin_inff() ? 0.0f : M;
                    float L = 0.0f;
                    f32x4 x{0, 0, 0, 0};
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        const float f = __builtin_amdgcn_exp2f(ml[t].x - base);
                        L += ml[t].y * f;
                        x += *(const f32x4*)&so[t][row][col] * f;
                    }
                    put(16 * r + row, c0 + col, x, M, L);
                }
            }
        if constexpr (HERE) {
            static_assert(sizeof(so) >= 256 * 24, "the join's scratch");
            if (!whole) join_parts<256, DP>(a, p, u0, (f32x4*)&so[0][0][0]);
        }
    }
    if (MODE == kWhole && !HERE && tid == 0) p.split[worker] = split;
}

template <int DP, int CT, int R, bool F32, bool HERE, int MODE = kWhole>
__global__ __launch_bounds__(256, (Attend<DP, CT, R, F32>::OCC)) void k_attend(AttendArgs a, PlanOf<MODE> p) {
    attend_narrow<DP, CT, R, F32, HERE, MODE>(a, p, blockIdx.x);
}

}  // namespace lacache
