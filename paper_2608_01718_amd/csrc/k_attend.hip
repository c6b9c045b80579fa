// k_attend.hip -- attention over the paged cache: the launches' shape, and the join of row groups that several
// workgroups had tiles of.
#include "attend_wide.hpp"

namespace lacache {

constexpr int kJoinThreads = 256;
constexpr int64_t kMostItems = INT32_MAX / 2;  // chunks of tiles of all row groups

// Many row groups, of few parts each: a thread four columns of a row, part after part (four loaded together).
__global__ __launch_bounds__(256) void k_attend_join(AttendArgs a, AttendPlan p) {
    const AttendSplit s = p.split[blockIdx.x];
    const int dp = a.pool.dp, lanes = dp / 4, rows = 256 / lanes;
    const int col = threadIdx.x % lanes * 4, row_in = threadIdx.x / lanes;
    const int parts = s.parts;
    if (row_in >= rows) return;
    for (int row = blockIdx.y * rows + row_in; row < s.n_rows; row += gridDim.y * rows) {
        Joined x;
        for (int k0 = 0; k0 < parts; k0 += 4) {
            float2 ml[4];
            f32x4 o[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int64_t at = part_of(p, s.worker0 + (k0 + u < parts ? k0 + u : parts - 1), k0 + u < parts - 1) + row;
                ml[u] = p.part_ml[at];
                o[u] = *(const f32x4*)(p.part_o + at * dp + col);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (k0 + u < parts) x.add(ml[u].x, ml[u].y, o[u]);
        }
        store_joined(a, p, s, row, col, x);
    }
}

// Few row groups, often of many parts each: the workgroups (x, .) join those that ended with one of `of` workers, each a
// share of the rows.  The j-th of these workers is number (x + j) mod gridDim.x of the j-th gridDim.x of all, so that
// neighbours among the workers, and those in regular steps, go to different workgroups.
__global__ __launch_bounds__(kJoinThreads) void k_attend_join_few(AttendArgs a, AttendPlan p, int of) {
    __shared__ f32x4 scratch[kJoinThreads * 3 / 2];
    auto worker = [&](int j) { return j * (int)gridDim.x + (int)((blockIdx.x + j) % gridDim.x); };
    const int mine = worker(threadIdx.x & 63);
    uint64_t todo = __ballot((int)(threadIdx.x & 63) < of && mine < p.workers && p.split[mine].n_rows > 0);
    for (; todo; todo &= todo - 1) {
        const AttendSplit s = p.split[worker(__ffsll((unsigned long long)todo) - 1)];
        const int groups = kJoinThreads / (a.pool.dp / 4);
        int of_row = 1;
        while (2 * of_row <= groups && (8 * of_row <= s.parts || (4 * of_row <= s.parts && 2 * of_row * s.n_rows <= groups)))
            of_row *= 2;
        join_rows<kJoinThreads>(a, p, s, a.pool.dp, of_row, threadIdx.x, blockIdx.y, gridDim.y, scratch,
                                [&](int64_t at, int col, float2& ml, f32x4& o) {
                                    ml = p.part_ml[at];
                                    o = *(const f32x4*)(p.part_o + at * a.pool.dp + col);
                                });
    }
}

namespace {

// The rows of a row group (as a shift) and the waves of a workgroup, by the most rows of a (sequence, kv head).
struct Shape {
    int group_shift, waves, occupancy;
};
Shape shape_of(const KvPool& pool, bool f32, int64_t rows) {
    const bool bytes = pool.type != kKvBf16;
    if (rows <= 16 || (f32 && pool.dp > 192)) return {4, 4, attend_occupancy(pool.dp, bytes, 1, f32)};
    if (f32) return {6, 4, wide_occupancy(pool.dp, 4, 1, true)};
    if (rows <= 32 && pool.dp <= 128) return {5, 4, attend_occupancy(pool.dp, bytes, 2, false)};
    if (rows <= 64 && pool.dp <= 192) return {6, 4, wide_occupancy(pool.dp, 4, 1, false)};
    if (pool.dp > 128) return {7, 8, wide_occupancy(pool.dp, 8, 1, false)};
    return {7, 4, wide_occupancy(pool.dp, 4, 2, false)};
}

// The plan of a launch whose workspace begins at `space`, and the bytes it takes.
AttendPlan plan_of(const KvPool& pool, bool f32, int max_new, int group, int num_cu, char* space, int64_t* bytes, int occupancy = 0) {
    AttendPlan p{};
    // (the rows of a (sequence, kv head), if no bound is known: plenty)
    const Shape sh = shape_of(pool, f32, (int64_t)(max_new > 0 ? max_new : 64) * group);
    p.group_shift = sh.group_shift;
    p.waves = sh.waves;
    p.workers = num_cu * (occupancy ? occupancy : sh.occupancy);
    p.workers = p.workers < kMaxWorkers ? p.workers : kMaxWorkers;
    // (the counters first: at the same place in every launch)
    const int64_t done = 4 * kMaxWorkers, split = (int64_t)sizeof(AttendSplit) * p.workers;
    const int64_t slots = (2 * (int64_t)p.workers) << p.group_shift;
    p.done = (uint32_t*)space;
    p.split = (AttendSplit*)(space + done);
    p.part_ml = (float2*)(space + done + split);
    p.part_o = (float*)(space + done + split + 8 * slots);
    *bytes = done + split + 8 * slots + 4 * slots * pool.dp;
    return p;
}

// More than the row groups of all (sequence, kv head) together.  Sequences without rows have none.
int64_t row_groups(const KvPool& pool, int64_t rows, int n_seq, int group, int group_shift) {
    return (((rows * group) >> group_shift) + (n_seq < rows ? n_seq : rows)) * pool.heads;
}

}  // namespace

bool attend_fits(const KvPool& pool, int dtype, int64_t rows, int n_seq, int group, int max_new) {
    const Shape sh = shape_of(pool, dtype == 0, (int64_t)(max_new > 0 ? max_new : 64) * group);
    return row_groups(pool, rows, n_seq, group, sh.group_shift) <= kMostItems;
}

int64_t attend_workspace(const KvPool& pool, int dtype, int q_heads, int max_new, int num_cu) {
    int64_t bytes;
    plan_of(pool, dtype == 0, max_new, q_heads / pool.heads, num_cu, nullptr, &bytes);
    return bytes;
}

namespace {

// What a mode's launch works with besides its plan.  n_seq: what the mode counts as sequences; max_new: a bound (kPrefix: an
// average) on the rows of each.
template <int MODE>
void prepare(const AttendArgs& a, AttendPlan& p, int n_seq, int64_t max_new) {
    // row / group for rows below 2^31: magic = ceil(2^(31 + bits) / group), bits = ceil(log2 group)
    int bits = 0;
    while ((1 << bits) < a.group) ++bits;
    p.group_bits = 31 + bits;
    p.group_magic = (uint32_t)((((uint64_t)1 << p.group_bits) + a.group - 1) / a.group);
    // the chunks of all row groups are counted in 32 bits (a chunk holds a whole sequence at the latest: attend_fits)
    const int64_t tiles = ((int64_t)a.seqs.max_pages << (a.pool.page_shift - 5)) + 1;
    const int64_t units = row_groups(a.pool, a.seqs.rows, n_seq, a.group, p.group_shift);
    while (units * (((tiles - 1) >> p.chunk_shift) + 1) > kMostItems && p.chunk_shift < 30) ++p.chunk_shift;
    // Behind a shared prefix many sequences have a few tiles of their own, and beginning and ending a row group takes as long
    // as some tiles: it counts for as many more, so that workgroups get as much to do (64 sequences with 16 to 2048 tokens of
    // their own, 8 heads: 47 us by tiles alone, 30, 27, 28 and 32 with 4, 8, 12 and 20 more).
    constexpr int kExtra = 8;
    if (MODE == kOwn && units * (tiles + kExtra) <= kMostItems) p.extra = kExtra;
    // Small calls join their parts in the launch: where each wave has a tile at most, by what the page tables (or the
    // window) can hold, and a row group has few parts.  One launch less is 2 us on the host and 1 us on the GPU (one sequence of
    // 777 tokens, 8 heads 11.5 us, 13.7 in two); with more parts to join, or parts of many rows, the launch is faster (131,071
    // tokens 88 us, 93 joined in the launch; 64 sequences in fp8 99, 103; 151 new tokens 174, 208; 7 heads on one of 33,000
    // tokens, 260 parts 19, 53; of 1000 tokens 13.4, 10.5).
    const int64_t seen = a.window > 0 && a.window / 32 + 2 + max_new / 32 < tiles && max_new > 0
                             ? a.window / 32 + 2 + max_new / 32 : tiles;
    p.join_here = MODE == kWhole && p.group_shift == 4 && seen <= 64 && units * seen <= 4 * (int64_t)p.workers;
}

// The join of a whole attention's parts.
hipError_t launch_join(const AttendArgs& a, const AttendPlan& p, int n_seq, int64_t max_new, hipStream_t s) {
    // rows of a row group, row groups
    int64_t rows = (max_new <= 0 ? 64 : max_new < a.seqs.rows ? max_new : a.seqs.rows) * a.group;
    const int64_t live = n_seq < a.seqs.rows ? n_seq : a.seqs.rows;
    const int64_t groups_most = live * a.pool.heads * (((rows - 1) >> p.group_shift) + 1);
    rows = rows < (1 << p.group_shift) ? rows : 1 << p.group_shift;
    const int64_t lane_groups = kJoinThreads / (a.pool.dp / 4);
    if (groups_most >= 64) {
        k_attend_join<<<dim3((unsigned)p.workers, (unsigned)((rows + lane_groups - 1) / lane_groups)), dim3(kJoinThreads),
                              0, s>>>(a, p);
    } else {
        // About one row group that was split for each workgroup in x, and one pass over its rows, but no more than 2048
        // workgroups: of a launch of 16,384 that find nothing most of the time is theirs (4 sequences of 1024 tokens, 16 new
        // ones, 4 kv heads: 24 us for the whole call, 189 with a workgroup of 512 threads for each worker and 4 rows).  With
        // more row groups that end anywhere, workgroups would get several of them in turn (32 sequences of 512 to 4096
        // tokens, 21 new ones: 75 us this way, 65 with a launch for all workers).
        int of = 1;
        while (of < 16 && 2 * of * groups_most <= p.workers) of *= 2;
        const int64_t x = (p.workers + of - 1) / of, parts = p.workers / groups_most + 1;
        int64_t at_once = lane_groups;
        for (int64_t of_row = 1; at_once > 1 && 8 * of_row <= parts; of_row *= 2) at_once /= 2;
        int64_t y = (rows + at_once - 1) / at_once;
        y = y < 2048 / x ? y : 2048 / x;
        k_attend_join_few<<<dim3((unsigned)x, (unsigned)(y > 1 ? y : 1)), dim3(kJoinThreads), 0, s>>>(a, p, of);
    }
    return hipGetLastError();
}

// The launches of one mode.
template <int MODE>
hipError_t launch_mode(const AttendArgs& a, PlanOf<MODE> p, int n_seq, int64_t max_new, hipStream_t s) {
    prepare<MODE>(a, p, n_seq, max_new);
    const hipError_t e = a.pool.dp == 64    ? launch_attend<64, MODE>(a, p, s)
                         : a.pool.dp == 96  ? launch_attend<96, MODE>(a, p, s)
                         : a.pool.dp == 128 ? launch_attend<128, MODE>(a, p, s)
                         : a.pool.dp == 192 ? launch_attend<192, MODE>(a, p, s)
                                            : launch_attend<256, MODE>(a, p, s);
    return e != hipSuccess || p.join_here || MODE != kWhole ? e : launch_join(a, p, n_seq, max_new, s);
}

}  // namespace

hipError_t launch_kv_attend(const AttendArgs& a, int max_new, void* workspace, int num_cu, hipStream_t s) {
    if (a.seqs.rows <= 0 || a.seqs.n_seq <= 0) return hipSuccess;
    int64_t bytes;
    return launch_mode<kWhole>(a, plan_of(a.pool, a.dtype == 0, max_new, a.group, num_cu, (char*)workspace, &bytes), a.seqs.n_seq,
                               max_new, s);
}

// ---------------------------------------------------------------------------
// Groups of sequences that share a prefix.  The prefix of a group is attended to once, by all of the group's rows together: a
// tile is read for up to 128 of them instead of for one sequence's.  The prefixes and the sequences' own tokens (one launch or two)
// leave their rows' sums in the workspace, and k_attend_together puts them together.  (One token of 64 sequences that share 8192
// and have 16 to 2048 of their own, 32 query heads on 8, d = 128: 45 us, of which 36 both parts; 256 by every sequence's table.)
// ---------------------------------------------------------------------------

// How the workgroups of a launch of both parts are shared out.
struct AttendDeal {
    int workers;                       // 0: there is no such launch
    int prefix_shift, own_shift, extra;  // rows of a row group, what one counts for besides its tiles
    float weight;                      // a tile of the prefixes takes as long as so many of the sequences' own
};

// Half of them, or by the tiles of both, where that is much better: fewer workgroups begin row groups in more turns, more
// leave more parts to join.  A multiple of eight (XCDs).  Tiles are counted roughly: the results are right with any number.
// (64 sequences, 32 query heads on 8, d = 128: 65,536 shared tokens and 16 to 64 of their own 140 us, 174 by halves; 1024 and 1024
// to 8192 198, 226; 4096 and 16 to 64 33, by tiles 40.)
__device__ int deal_out(const AttendDeal& d, float prefix, float own, int lane) {
    auto time = [&](int n) {  // of the longer of both, in tiles of the sequences' own
        const int others = d.workers - n;
        return others < 8 ? __builtin_inff() : fmaxf(d.weight * ceilf(prefix / (float)n), ceilf(own / (float)others));
    };
    const int half = d.workers / 2 & ~7, step = ((d.workers + 63) / 64 + 7) & ~7;
    const float halves = time(half), mine = time(step * (lane + 1));
    const float least = wave_reduce(mine, [](float s, float t) { return fminf(s, t); });
    const int best = step * __ffsll((unsigned long long)__ballot(mine == least));
    return least < 0.75f * halves && least < halves - 24.0f ? best : half;
}

// What both parts need: workgroup b < n_seq the positions of sequence b's rows and what it shares, the others a group each, and
// one more deals out the workgroups of a launch of both.
// (64 sequences 4 us: lookups one after another.)
__global__ __launch_bounds__(64) void k_attend_share(AttendArgs a, AttendShare x, const int32_t* group, const int32_t* len,
                                                     AttendDeal d) {
    const int lane = threadIdx.x, n_seq = a.seqs.n_seq;
    const int64_t known = (int64_t)a.seqs.max_pages << a.pool.page_shift;
    // sequences and tokens of group g (one sequence shares nothing)
    auto group_of = [&](int g, int& from, int& to) {
        from = group[g], to = group[g + 1];
        from = from < 0 ? 0 : from > n_seq ? n_seq : from;
        to = to < from ? from : to > n_seq ? n_seq : to;
        const int64_t n = len[g] < 0 ? 0 : len[g] < known ? len[g] : known;
        return to - from > 1 ? (int)(n >> a.pool.page_shift << a.pool.page_shift) : 0;
    };
    if ((int)blockIdx.x < n_seq) {
        const int b = blockIdx.x;
        const int g = last_up_to(group, x.n_groups, b, lane);
        int from = 0, to = 0;
        const int held = g >= 0 ? group_of(g, from, to) : 0;
        const int mine = b >= from && b < to ? held : 0;
        if (lane == 0) x.held[b] = mine;
        const KvSpan s = span_of(a.seqs, b);
        for (int i = lane; i < s.n; i += 64) {
            x.row_pos[s.row0 + i] = s.pos0 + i < 0 ? -1 : (int)(s.pos0 + i);
            x.row_held[s.row0 + i] = mine > 0;
        }
        // rows of no sequence
        if (b == 0)
            for (int64_t i = lane; i < s.row0; i += 64) x.row_held[i] = -1;
        if (b == n_seq - 1)
            for (int64_t i = s.row0 + s.n + lane; i < a.seqs.rows; i += 64) x.row_held[i] = -1;
        return;
    }
    if ((int)blockIdx.x == n_seq + x.n_groups) {
        // (all lengths are looked at one after another: a few thousand; with a window nearly all work is in a few tiles a row)
        float prefix = 0.0f, own = 0.0f;
        if (a.window == 0 && n_seq + x.n_groups <= 8192) {
            for (int b = lane; b < n_seq; b += 64) {
                const KvSpan s = span_of(a.seqs, b);
                const int64_t end = s.pos0 + s.n, tiles = end < 0 ? 0 : (end < known ? end : known) >> 5;
                own += (float)(((int64_t)s.n * a.group + (1 << d.own_shift) - 1) >> d.own_shift) * (float)(tiles + d.extra);
            }
            for (int g = lane; g < x.n_groups; g += 64) {
                int from, to;
                const int held = group_of(g, from, to) >> 5;
                if (held == 0) continue;
                const KvSpan s = span_of(a.seqs, to - 1);
                const int64_t n = s.row0 + s.n - span_of(a.seqs, from).row0, rows = n < 0 ? 0 : n * a.group;
                const int64_t live = to - from < n ? to - from : n, of_own = rows >> d.own_shift;
                prefix += (float)((rows + (1 << d.prefix_shift) - 1) >> d.prefix_shift) * (float)held;
                own -= (float)(live > of_own ? live : of_own) * (float)held;
            }
        }
        auto add = [](float s, float t) { return s + t; };
        prefix = wave_reduce(prefix, add) * (float)a.pool.heads;
        own = fmaxf(wave_reduce(own, add), 0.0f) * (float)a.pool.heads;
        const int n = deal_out(d, prefix, own, lane);
        if (lane == 0) *x.deal = n;
        return;
    }
    const int g = blockIdx.x - n_seq;
    // The prefix is read through the page table of the longest of the sequences that have rows: all that any row sees of it is
    // there, whatever the tables of idle slots, and of shorter sequences behind their own tokens, hold.
    int from, to, least = INT32_MAX, longest = 0, table = INT32_MAX;
    const int held = group_of(g, from, to);
    for (int b = from + lane; b < to; b += 64) {
        const KvSpan s = span_of(a.seqs, b);
        const int64_t end = s.pos0 + s.n, first = s.pos0 < 0 ? 0 : s.pos0;
        if (s.n <= 0 || end <= 0) continue;
        least = first < least ? (int)first : least;
        if (end > longest) longest = (int)end, table = b;
    }
    auto min2 = [](int p, int q) { return p < q ? p : q; };
    least = wave_reduce(least, min2);
    const int most = wave_reduce(longest, [](int p, int q) { return p > q ? p : q; });
    table = wave_reduce(longest == most ? table : INT32_MAX, min2);
    if (lane == 0) {
        const int64_t row0 = from < n_seq ? span_of(a.seqs, from).row0 : 0;
        const int64_t end = to > from ? span_of(a.seqs, to - 1).row0 + span_of(a.seqs, to - 1).n : row0;
        x.span[g] = make_int4((int)row0, held > 0 && end > row0 ? (int)(end - row0) : 0, held, table < to ? table : from);
        const int64_t lo = a.window > 0 && least < INT32_MAX ? (int64_t)least - a.window + 1 : 0;
        x.first[g] = lo > 0 ? (int)(lo >> 5) : 0;
    }
}

// Puts the two parts of every (row, query head) together: dp / 4 lanes on four columns each, of_row lane groups (a power of two)
// one after another on the parts that workers have of it.  Reading the parts bounds it (64 rows of 32 heads, 17 MB of parts 8 us;
// 945 rows of 12 heads, three groups 7 us).
template <bool F32>
__global__ __launch_bounds__(256) void k_attend_together(AttendArgs a, AttendPartPlan prefix, AttendPartPlan own, int of_row) {
    __shared__ f32x4 sums[256];
    __shared__ float2 ml_of[256];
    const int dp = a.pool.dp, lanes = dp / 4, rows = 256 / lanes / of_row, g = threadIdx.x / lanes, sub = g % of_row;
    const int col = threadIdx.x % lanes * 4;
    const AttendShare& x = own.share;
    const int64_t all = a.seqs.rows * a.q_heads;
    for (int64_t at0 = (int64_t)blockIdx.x * rows; at0 < all; at0 += (int64_t)gridDim.x * rows) {
        const int64_t at = at0 + g / of_row;
        const int held = g < rows * of_row && at < all ? x.row_held[at / a.q_heads] : -1;
        Joined j;
        if (held >= 0) {
            const int2 of_own = x.sums[kOwn - kPrefix].at[at], of_prefix = held ? x.sums[0].at[at] : make_int2(0, 0);
            const int n_own = of_own.x ? of_own.x : 1, n = n_own + (!held ? 0 : of_prefix.x ? of_prefix.x : 1);
            for (int k0 = sub; k0 < n; k0 += 4 * of_row) {
                float2 ml[4];
                f32x4 o[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int k = k0 + i * of_row < n ? k0 + i * of_row : n - 1;
                    const bool mine = k < n_own;
                    const AttendPartPlan& p = mine ? own : prefix;
                    const AttendSums& whole = x.sums[mine ? kOwn - kPrefix : 0];
                    const int2 w = mine ? of_own : of_prefix;
                    const int part = mine ? k : k - n_own;
                    const int64_t slot = part_of(p, (w.y & 0xFFFF) + part, part < w.x - 1) + (w.y >> 16);
                    ml[i] = w.x ? p.part_ml[slot] : whole.ml[at];
                    o[i] = *(const f32x4*)(w.x ? p.part_o + slot * dp + col : whole.o + at * dp + col);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (k0 + i * of_row < n) j.add(ml[i].x, ml[i].y, o[i]);
            }
        }
        if (of_row > 1) {
            __syncthreads();
            sums[threadIdx.x] = j.o;
            ml_of[threadIdx.x] = make_float2(j.m, j.l);
            __syncthreads();
        }
        if (held < 0 || sub > 0) continue;
        for (int k = 1; k < of_row; ++k)
            j.add(ml_of[threadIdx.x + k * lanes].x, ml_of[threadIdx.x + k * lanes].y, sums[threadIdx.x + k * lanes]);
        if (col < a.pool.d) store4<F32>(a, at * a.pool.d + col, j.o * (j.l == 0.0f ? 0.0f : 1.0f / j.l));
        if (col == 0 && a.lse) a.lse[at] = lse_of(j.m, j.l);
    }
}

namespace {

int prefix_rows(int64_t rows, int n_groups) {  // of a group, on average
    const int64_t each = n_groups > 0 ? (rows + n_groups - 1) / n_groups : 1;
    return each < 1 ? 1 : (int)each;
}

// Whether both parts are in one launch: few rows of own tokens, or many of both, with room for two workgroups on a compute
// unit.  (16 sequences, 32 query heads on 8, d = 128, 8192 shared tokens and 16 to 2048 of their own: 32 us, 42 in two launches;
// 1024 and 16 to 512: 20, 28; 16 new tokens, 2048 and 60 to 512: 42, 61.)
bool both_at_once(const KvPool& pool, bool f32, const AttendPlan& prefix, const AttendPlan& own) {
    if (pool.dp > 128 || prefix.workers < 16) return false;
    if (own.group_shift >= 6) return prefix.group_shift == (f32 ? 6 : 7);
    return own.group_shift == 4 && attend_occupancy(pool.dp, pool.type != kKvBf16, prefix.group_shift == 5 ? 2 : 1, f32) >= 2;
}

// The plans of both parts, and what lies behind their memory.
int64_t shared_plan(const KvPool& pool, bool f32, int64_t rows, int n_seq, int n_groups, int q_heads, int max_new, int num_cu,
                    char* space, AttendPartPlan* prefix, AttendPartPlan* own, bool* both) {
    const int group = q_heads / pool.heads;
    int64_t at, bytes;
    auto take = [&](int64_t n) {
        at = (at + 15) & ~int64_t(15);
        char* p = space + at;
        at += n;
        return p;
    };
    auto plans = [&](int occupancy) {
        (AttendPlan&)*prefix = plan_of(pool, f32, prefix_rows(rows, n_groups), group, num_cu, space, &at, occupancy);
        (AttendPlan&)*own = plan_of(pool, f32, max_new, group, num_cu, take(0), &bytes, occupancy);
        at += bytes;
    };
    plans(0);
    *both = n_groups > 0 && both_at_once(pool, f32, *prefix, *own);
    if (*both) {
        plans(2);  // (as many workgroups as the launch has, for either)
        prefix->workers = own->workers &= ~7;
    }
    AttendShare x{};
    x.n_groups = n_groups;
    x.span = (int4*)take(16 * (int64_t)n_groups);
    x.first = (int32_t*)take(4 * (int64_t)n_groups);
    x.held = (int32_t*)take(4 * (int64_t)n_seq);
    x.row_pos = (int32_t*)take(4 * rows);
    x.row_held = (int32_t*)take(4 * rows);
    x.deal = (int32_t*)take(4);
    for (AttendSums& y : x.sums) {
        y.ml = (float2*)take(8 * rows * q_heads);
        y.at = (int2*)take(8 * rows * q_heads);
        y.o = (float*)take(4 * rows * q_heads * pool.dp);
    }
    prefix->share = own->share = x;
    return at;
}

}  // namespace

bool attend_shared_fits(const KvPool& pool, int dtype, int64_t rows, int n_groups, int group) {
    const Shape sh = shape_of(pool, dtype == 0, (int64_t)prefix_rows(rows, n_groups) * group);
    return row_groups(pool, rows, n_groups, group, sh.group_shift) <= kMostItems;
}

int64_t attend_shared_workspace(const KvPool& pool, int dtype, int64_t rows, int n_seq, int n_groups, int q_heads, int max_new,
                                int num_cu) {
    AttendPartPlan p, o;
    bool both;
    return shared_plan(pool, dtype == 0, rows, n_seq, n_groups, q_heads, max_new, num_cu, nullptr, &p, &o, &both);
}

hipError_t launch_kv_attend_shared(const AttendArgs& a, const int32_t* group, const int32_t* len, int n_groups, int max_new,
                                   void* workspace, int num_cu, hipStream_t s) {
    if (a.seqs.rows <= 0 || a.seqs.n_seq <= 0) return hipSuccess;
    AttendPartPlan prefix, own;
    bool both;
    shared_plan(a.pool, a.dtype == 0, a.seqs.rows, a.seqs.n_seq, n_groups, a.q_heads, max_new, num_cu, (char*)workspace, &prefix, &own,
                &both);
    const int each = prefix_rows(a.seqs.rows, n_groups);
    AttendDeal deal{};
    if (both) {
        prepare<kPrefix>(a, prefix, n_groups, each);
        prepare<kOwn>(a, own, a.seqs.n_seq, max_new);
        // (64 sequences, 8 heads, bfloat16: a tile for 128 rows 1.7 us, one for up to 16 about 0.6)
        const float weight = prefix.group_shift < 6 || prefix.group_shift == own.group_shift ? 1.0f
                             : own.group_shift == 6                                          ? 1.5f
                             : prefix.group_shift == 6 && a.dtype != 0                       ? 2.0f : 3.0f;
        deal = AttendDeal{own.workers, prefix.group_shift, own.group_shift, own.extra, weight};
    }
    k_attend_share<<<dim3((unsigned)(a.seqs.n_seq + n_groups + both)), dim3(64), 0, s>>>(a, prefix.share, group, len, deal);
    hipError_t e = hipGetLastError();
    if (both) {
        if (e == hipSuccess)
            e = a.pool.dp == 64   ? launch_attend_both<64>(a, prefix, own, s)
                : a.pool.dp == 96 ? launch_attend_both<96>(a, prefix, own, s)
                                  : launch_attend_both<128>(a, prefix, own, s);
    } else {
        if (e == hipSuccess && n_groups > 0) e = launch_mode<kPrefix>(a, prefix, n_groups, each, s);
        if (e == hipSuccess) e = launch_mode<kOwn>(a, own, a.seqs.n_seq, max_new, s);
    }
    if (e != hipSuccess) return e;
    // the parts of a row, about: its row group's share of the workers over the prefixes, and a few of its own; four to a lane group
    const int64_t groups_of = n_groups > 0 ? (((int64_t)each * a.group >> prefix.group_shift) + 1) * n_groups * a.pool.heads : 1;
    const int64_t parts = (n_groups > 0 ? prefix.workers / (both ? 2 : 1) / groups_of : 0) + 2;
    int of_row = 1;
    while (4 * of_row < parts && 2 * of_row <= 256 / (a.pool.dp / 4)) of_row *= 2;
    const int rows = 256 / (a.pool.dp / 4) / of_row;
    const dim3 grid((unsigned)grid_blocks((a.seqs.rows * a.q_heads + rows - 1) / rows));
    if (a.dtype == 0) k_attend_together<true><<<grid, dim3(256), 0, s>>>(a, prefix, own, of_row);
    else k_attend_together<false><<<grid, dim3(256), 0, s>>>(a, prefix, own, of_row);
    return hipGetLastError();
}

}  // namespace lacache
