// k_attend.hip -- attention over the paged cache: the launches' shape, and the join of row groups that several
// workgroups had tiles of.
#include "attend.hpp"

namespace lacache {

// A workgroup per row (of a sequence and kv head): a thread four columns of every 1024 / dp-th part.
__global__ __launch_bounds__(256) void k_attend_join(AttendArgs a, AttendPlan p) {
    __shared__ float sm[256], sl[256];
    __shared__ f32x4 so[256];
    const int tid = threadIdx.x, b = blockIdx.x, h = blockIdx.y;
    const int64_t per = p.base[a.seqs.n_seq + 1];
    const AttendSpan s = attend_span(a, p, b);
    const int dp = a.pool.dp, lanes = dp / 4, groups = 256 / lanes;
    const int col = tid % lanes * 4, part0 = tid / lanes;
    for (int row = blockIdx.z; row < s.rows; row += gridDim.z) {
        const int rg = row / p.group_rows, in_group = row - rg * p.group_rows;
        const int64_t lo = p.base[b] + (int64_t)(h * s.groups + rg) * s.tiles, hi = lo + s.tiles;
        const int64_t w0 = lo / per, w1 = (hi - 1) / per;
        if (w0 == w1) continue;
        // a workgroup's part of a row group that goes on after it lies in its second slot
        auto slot = [&](int64_t w) { return 2 * w + (w < w1 ? 1 : 0); };
        float m = -__builtin_inff(), l = 0.0f;
        f32x4 o{0, 0, 0, 0};
        if (part0 < groups)
            for (int64_t w = w0 + part0; w <= w1; w += groups) {
                const int64_t at = slot(w) * p.group_rows + in_group;
                const float2 ml = p.part_ml[at];
                const f32x4 x = *(const f32x4*)(p.part_o + at * dp + col);
                const float M = fmaxf(m, ml.x);
                if (M == -__builtin_inff()) continue;
                const float f = __builtin_amdgcn_exp2f(m - M), g = __builtin_amdgcn_exp2f(ml.x - M);
                l = l * f + ml.y * g;
                o = o * f + x * g;
                m = M;
            }
        __syncthreads();
        sm[tid] = m;
        sl[tid] = l;
        so[tid] = o;
        __syncthreads();
        if (part0 == 0) {
            float M = -__builtin_inff();
            for (int k = 0; k < groups; ++k) M = fmaxf(M, sm[k * lanes + tid]);
            const float base = M == -__builtin_inff() ? 0.0f : M;
            float L = 0.0f;
            f32x4 O{0, 0, 0, 0};
            for (int k = 0; k < groups; ++k) {
                const float f = __builtin_amdgcn_exp2f(sm[k * lanes + tid] - base);
                L += sl[k * lanes + tid] * f;
                O += so[k * lanes + tid] * f;
            }
            const int i = row / a.group, head = h * a.group + (row - i * a.group);
            O *= L == 0.0f ? 0.0f : 1.0f / L;
            if (col < a.pool.d) {
                if (a.dtype == 0) store4<true>(a, s.span.row0 + i, head, col, O);
                else store4<false>(a, s.span.row0 + i, head, col, O);
            }
            if (tid == 0 && a.lse) a.lse[(s.span.row0 + i) * a.q_heads + head] = lse_of(M, L);
        }
    }
}

namespace {

// Row tiles of 16 a wave and waves that share a row group's rows, by the most rows of a (sequence, kv head).
struct Shape {
    int R, row_waves;
};
Shape shape_of(int dp, bool f32, int64_t rows) {
    const int most = f32 ? 1 : dp <= 96 ? 4 : dp <= 192 ? 2 : 1;
    int R = 1, waves = 1;
    while (R < most && 16 * R < rows) R *= 2;
    while (waves < 4 && 16 * R * waves < rows) waves *= 2;
    return {R, waves};
}

int64_t round16(int64_t x) { return (x + 15) & ~int64_t(15); }

// The plan of a launch whose workspace begins at `space`, and the bytes it takes.
AttendPlan plan_of(const KvPool& pool, bool f32, int n_seq, int64_t rows, int num_cu, char* space, int64_t* bytes) {
    const Shape sh = shape_of(pool.dp, f32, rows);
    AttendPlan p{};
    p.row_waves = sh.row_waves;
    p.group_rows = 16 * sh.R * sh.row_waves;
    p.workgroups = num_cu * attend_occupancy(pool.dp, pool.type != kKvBf16, sh.R, f32);
    const int64_t base = round16(8 * ((int64_t)n_seq + 2)), slots = 2 * (int64_t)p.workgroups * p.group_rows;
    p.base = (int64_t*)space;
    p.part_ml = (float2*)(space + base);
    p.part_o = (float*)(space + base + 8 * slots);
    *bytes = base + 8 * slots + 4 * slots * pool.dp;
    return p;
}

}  // namespace

// The rows of a (sequence, kv head) if no bound is known: plenty.
static int64_t most_rows(int max_new, int group) { return (int64_t)(max_new > 0 ? max_new : 64) * group; }

int64_t attend_workspace(const KvPool& pool, int dtype, int n_seq, int q_heads, int max_new, int num_cu) {
    int64_t bytes;
    plan_of(pool, dtype == 0, n_seq, most_rows(max_new, q_heads / pool.heads), num_cu, nullptr, &bytes);
    return bytes;
}

hipError_t launch_kv_attend(const AttendArgs& a, int max_new, void* workspace, int num_cu, hipStream_t s) {
    if (a.seqs.rows <= 0 || a.seqs.n_seq <= 0) return hipSuccess;
    const bool f32 = a.dtype == 0;
    const int64_t rows = most_rows(max_new, a.group);
    int64_t bytes;
    const AttendPlan p = plan_of(a.pool, f32, a.seqs.n_seq, rows, num_cu, (char*)workspace, &bytes);
    const int R = shape_of(a.pool.dp, f32, rows).R;
    const hipError_t e = a.pool.dp == 64    ? launch_attend<64>(a, p, R, s)
                         : a.pool.dp == 96  ? launch_attend<96>(a, p, R, s)
                         : a.pool.dp == 128 ? launch_attend<128>(a, p, R, s)
                         : a.pool.dp == 192 ? launch_attend<192>(a, p, R, s)
                                            : launch_attend<256>(a, p, R, s);
    if (e != hipSuccess) return e;
    const int64_t join_rows = rows < a.seqs.rows * a.group ? rows : a.seqs.rows * a.group;
    k_attend_join<<<dim3((unsigned)a.seqs.n_seq, (unsigned)a.pool.heads, (unsigned)(join_rows < 1024 ? join_rows : 1024)),
                    dim3(256), 0, s>>>(a, p);
    return hipGetLastError();
}

}  // namespace lacache
