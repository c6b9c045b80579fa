// k_attend.hip -- attention over the paged cache: the launches' shape, and the join of row groups that several
// workgroups had tiles of.
#include "attend_wide.hpp"

namespace lacache {

// The row groups that several workers had parts of: a workgroup a row of the group that ended with worker blockIdx.x,
// a thread four columns of every (4 THREADS / dp)-th part, four of them loaded together.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void k_attend_join(AttendArgs a, AttendPlan p) {
    __shared__ float2 sml[THREADS];
    __shared__ f32x4 so[THREADS];
    const AttendSplit s = p.split[blockIdx.x];
    const int tid = threadIdx.x, dp = a.pool.dp, lanes = dp / 4, groups = THREADS / lanes;
    const int col = tid % lanes * 4, part = tid / lanes;
    const int parts = (int)blockIdx.x - s.worker0 + 1;
    for (int row = blockIdx.y; row < s.n_rows; row += gridDim.y) {
        float m = -__builtin_inff(), l = 0.0f;
        f32x4 o{0, 0, 0, 0};
        if (part < groups)
            for (int k0 = part; k0 < parts; k0 += 4 * groups) {
                float2 ml[4];
                f32x4 x[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    // a worker's part of a row group that goes on after it lies in its second slot
                    const int k = k0 + u * groups < parts ? k0 + u * groups : parts - 1;
                    const int64_t at = (((2 * (int64_t)(s.worker0 + k)) + (k < parts - 1 ? 1 : 0)) << p.group_shift) + row;
                    ml[u] = p.part_ml[at];
                    x[u] = *(const f32x4*)(p.part_o + at * dp + col);
                }
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    if (k0 + u * groups >= parts || ml[u].x == -__builtin_inff()) continue;
                    const float M = fmaxf(m, ml[u].x);
                    const float f = __builtin_amdgcn_exp2f(m - M), g = __builtin_amdgcn_exp2f(ml[u].x - M);
                    l = l * f + ml[u].y * g;
                    o = o * f + x[u] * g;
                    m = M;
                }
            }
        __syncthreads();
        sml[tid] = make_float2(m, l);
        so[tid] = o;
        __syncthreads();
        const int live = groups < parts ? groups : parts;
        if (part == 0) {
            float M = -__builtin_inff();
            for (int k = 0; k < live; ++k) M = fmaxf(M, sml[k * lanes + tid].x);
            const float base = M == -__builtin_inff() ? 0.0f : M;
            float L = 0.0f;
            f32x4 O{0, 0, 0, 0};
            for (int k = 0; k < live; ++k) {
                const float f = __builtin_amdgcn_exp2f(sml[k * lanes + tid].x - base);
                L += sml[k * lanes + tid].y * f;
                O += so[k * lanes + tid] * f;
            }
            const int r = s.row + row, i = token_of(p, r);
            const int64_t at = ((int64_t)s.seq_row0 + i) * a.q_heads + s.head0 + (r - i * a.group);
            O *= L == 0.0f ? 0.0f : 1.0f / L;
            if (col < a.pool.d) {
                if (a.dtype == 0) store4<true>(a, at * a.pool.d + col, O);
                else store4<false>(a, at * a.pool.d + col, O);
            }
            if (tid == 0 && a.lse) a.lse[at] = lse_of(M, L);
        }
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
    if (rows <= 128) return {7, 4, wide_occupancy(pool.dp, 4, 2, false)};
    return {8, 8, wide_occupancy(pool.dp, 8, 2, false)};
}

// The plan of a launch whose workspace begins at `space`, and the bytes it takes.
AttendPlan plan_of(const KvPool& pool, bool f32, int n_seq, int max_new, int group, int num_cu, char* space,
                   int64_t* bytes) {
    AttendPlan p{};
    // (the rows of a (sequence, kv head), if no bound is known: plenty)
    const Shape sh = shape_of(pool, f32, (int64_t)(max_new > 0 ? max_new : 64) * group);
    p.group_shift = sh.group_shift;
    p.waves = sh.waves;
    p.workers = num_cu * sh.occupancy;
    const int64_t split = (int64_t)sizeof(AttendSplit) * p.workers, slots = (2 * (int64_t)p.workers) << p.group_shift;
    p.split = (AttendSplit*)space;
    p.part_ml = (float2*)(space + split);
    p.part_o = (float*)(space + split + 8 * slots);
    *bytes = split + 8 * slots + 4 * slots * pool.dp;
    return p;
}

}  // namespace

int64_t attend_workspace(const KvPool& pool, int dtype, int n_seq, int q_heads, int max_new, int num_cu) {
    int64_t bytes;
    plan_of(pool, dtype == 0, n_seq, max_new, q_heads / pool.heads, num_cu, nullptr, &bytes);
    return bytes;
}

hipError_t launch_kv_attend(const AttendArgs& a, int max_new, void* workspace, int num_cu, hipStream_t s) {
    if (a.seqs.rows <= 0 || a.seqs.n_seq <= 0) return hipSuccess;
    int64_t bytes;
    AttendPlan p = plan_of(a.pool, a.dtype == 0, a.seqs.n_seq, max_new, a.group, num_cu, (char*)workspace, &bytes);
    // row / group for rows below 2^31: magic = ceil(2^(31 + bits) / group), bits = ceil(log2 group)
    int bits = 0;
    while ((1 << bits) < a.group) ++bits;
    p.group_bits = 31 + bits;
    p.group_magic = (uint32_t)((((uint64_t)1 << p.group_bits) + a.group - 1) / a.group);
    // the chunks of all row groups are counted in 32 bits
    const int64_t tiles = ((int64_t)a.seqs.max_pages << (a.pool.page_shift - 5)) + 1;
    const int64_t groups = ((a.seqs.rows * a.group) >> p.group_shift) + a.seqs.n_seq;
    while (groups * a.pool.heads * (((tiles - 1) >> p.chunk_shift) + 1) > INT32_MAX / 2 && p.chunk_shift < 30)
        ++p.chunk_shift;
    const hipError_t e = a.pool.dp == 64    ? launch_attend<64>(a, p, s)
                         : a.pool.dp == 96  ? launch_attend<96>(a, p, s)
                         : a.pool.dp == 128 ? launch_attend<128>(a, p, s)
                         : a.pool.dp == 192 ? launch_attend<192>(a, p, s)
                                            : launch_attend<256>(a, p, s);
    if (e != hipSuccess) return e;
    const unsigned rows = 1u << p.group_shift;
    int64_t most = max_new > 0 && (int64_t)max_new * a.group < rows ? (int64_t)max_new * a.group : rows;
    most = most < 32 ? most : 32;
    if (a.seqs.n_seq * (int64_t)a.pool.heads < 64) k_attend_join<512><<<dim3((unsigned)p.workers, (unsigned)most), dim3(512), 0, s>>>(a, p);
    else k_attend_join<256><<<dim3((unsigned)p.workers, (unsigned)most), dim3(256), 0, s>>>(a, p);
    return hipGetLastError();
}

}  // namespace lacache
