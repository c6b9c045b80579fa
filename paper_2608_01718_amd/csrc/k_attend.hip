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
AttendPlan plan_of(const KvPool& pool, bool f32, int max_new, int group, int num_cu, char* space, int64_t* bytes) {
    AttendPlan p{};
    // (the rows of a (sequence, kv head), if no bound is known: plenty)
    const Shape sh = shape_of(pool, f32, (int64_t)(max_new > 0 ? max_new : 64) * group);
    p.group_shift = sh.group_shift;
    p.waves = sh.waves;
    p.workers = num_cu * sh.occupancy;
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

hipError_t launch_kv_attend(const AttendArgs& a, int max_new, void* workspace, int num_cu, hipStream_t s) {
    if (a.seqs.rows <= 0 || a.seqs.n_seq <= 0) return hipSuccess;
    int64_t bytes;
    AttendPlan p = plan_of(a.pool, a.dtype == 0, max_new, a.group, num_cu, (char*)workspace, &bytes);
    // row / group for rows below 2^31: magic = ceil(2^(31 + bits) / group), bits = ceil(log2 group)
    int bits = 0;
    while ((1 << bits) < a.group) ++bits;
    p.group_bits = 31 + bits;
    p.group_magic = (uint32_t)((((uint64_t)1 << p.group_bits) + a.group - 1) / a.group);
    // the chunks of all row groups are counted in 32 bits (a chunk holds a whole sequence at the latest: attend_fits)
    const int64_t tiles = ((int64_t)a.seqs.max_pages << (a.pool.page_shift - 5)) + 1;
    const int64_t units = row_groups(a.pool, a.seqs.rows, a.seqs.n_seq, a.group, p.group_shift);
    while (units * (((tiles - 1) >> p.chunk_shift) + 1) > kMostItems && p.chunk_shift < 30) ++p.chunk_shift;
    // Small calls join their parts in the launch: where each wave has a tile at most, by what the page tables (or the
    // window) can hold, and a row group has few parts.  One launch less is 2 us on the host and 1 us on the GPU (one sequence of
    // 777 tokens, 8 heads 11.5 us, 13.7 in two); with more parts to join, or parts of many rows, the launch is faster (131,071
    // tokens 88 us, 93 joined in the launch; 64 sequences in fp8 99, 103; 151 new tokens 174, 208; 7 heads on one of 33,000
    // tokens, 260 parts 19, 53; of 1000 tokens 13.4, 10.5).
    const int64_t seen = a.window > 0 && a.window / 32 + 2 + (int64_t)max_new / 32 < tiles && max_new > 0
                             ? a.window / 32 + 2 + max_new / 32 : tiles;
    p.join_here = p.group_shift == 4 && seen <= 64 && units * seen <= 4 * (int64_t)p.workers;
    const hipError_t e = a.pool.dp == 64    ? launch_attend<64>(a, p, s)
                         : a.pool.dp == 96  ? launch_attend<96>(a, p, s)
                         : a.pool.dp == 128 ? launch_attend<128>(a, p, s)
                         : a.pool.dp == 192 ? launch_attend<192>(a, p, s)
                                            : launch_attend<256>(a, p, s);
    if (e != hipSuccess || p.join_here) return e;
    // rows of a row group, row groups
    int64_t rows = (max_new <= 0 ? 64 : max_new < a.seqs.rows ? max_new : a.seqs.rows) * a.group;
    const int64_t live = a.seqs.n_seq < a.seqs.rows ? a.seqs.n_seq : a.seqs.rows;
    const int64_t groups_most = live * a.pool.heads * (((rows - 1) >> p.group_shift) + 1);
    rows = rows < (1 << p.group_shift) ? rows : 1 << p.group_shift;
    const int64_t lane_groups = kJoinThreads / (a.pool.dp / 4);
    if (groups_most >= 64) {
        k_attend_join<<<dim3((unsigned)p.workers, (unsigned)((rows + lane_groups - 1) / lane_groups)), dim3(kJoinThreads), 0,
                        s>>>(a, p);
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

}  // namespace lacache
