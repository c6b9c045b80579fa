// k_attend_blocks.hip -- attention over lists of pages: the launch's shape.
#include "attend_blocks.hpp"

namespace lacache {

namespace {

// Splits of a list: enough workgroups for every compute unit, of eight tiles or more (two a wave).  (Lists of 64 pages of 64
// tokens, 8 heads: one row 8.9 us, 11.2 with four tiles or more; four rows 14.1, 16.2 with twice the workgroups; 64 rows of up
// to 48 pages, 4 heads, fp8: 26, 29.)
int splits_of(const KvPool& pool, int64_t units, int n_blocks, int num_cu) {
    const int64_t tiles = (int64_t)n_blocks << (pool.page_shift - 5), most = (tiles + 7) / 8;
    int64_t want = units > 0 ? (int64_t)num_cu / units : 1;
    want = want < 1 ? 1 : want < most ? want : most;
    const int64_t per = (tiles + want - 1) / want;
    return (int)((tiles + per - 1) / per);
}
int64_t units_of(const KvPool& pool, int64_t rows, int group) { return rows * pool.heads * ((group + 15) / 16); }

}  // namespace

int64_t blocks_workspace(const KvPool& pool, int64_t rows, int group, int n_blocks, int num_cu) {
    const int64_t units = units_of(pool, rows, group), splits = splits_of(pool, units, n_blocks, num_cu);
    // (with counters for as many units as are ever split, at the place of attention's)
    return splits == 1 ? 0 : 4 * kMaxWorkers + units * splits * 16 * (8 + 4 * (int64_t)pool.dp);
}

hipError_t launch_attend_blocks(BlocksArgs x, void* workspace, int num_cu, hipStream_t s) {
    const KvPool& pool = x.a.pool;
    const int64_t units = units_of(pool, x.a.seqs.rows, x.a.group), tiles = (int64_t)x.n_blocks << (pool.page_shift - 5);
    x.splits = splits_of(pool, units, x.n_blocks, num_cu);
    x.per = (int)((tiles + x.splits - 1) / x.splits);
    int bits = 0;  // (token_of in attend.hpp: row / group)
    while ((1 << bits) < x.a.group) ++bits;
    x.bits = 31 + bits;
    x.magic = (uint32_t)((((uint64_t)1 << x.bits) + x.a.group - 1) / x.a.group);
    x.done = (uint32_t*)workspace;
    x.part_ml = (float2*)((char*)workspace + 4 * kMaxWorkers);
    x.part_o = (float*)((char*)workspace + 4 * kMaxWorkers + 8 * 16 * units * x.splits);
    return pool.dp == 64    ? launch_blocks<64>(x, units, s)
           : pool.dp == 96  ? launch_blocks<96>(x, units, s)
           : pool.dp == 128 ? launch_blocks<128>(x, units, s)
           : pool.dp == 192 ? launch_blocks<192>(x, units, s)
                            : launch_blocks<256>(x, units, s);
}

}  // namespace lacache
