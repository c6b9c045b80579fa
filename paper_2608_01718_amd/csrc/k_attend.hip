// k_attend.hip -- attention of the newest tokens of every sequence over its cached keys and values.
#include "kv.hpp"
#include "launch.hpp"

namespace lacache {

// A workgroup per (row, query head).  Each wave takes every fourth block of 64 positions: a lane a position for the
// scores, a lane a column for the sum of values, with a running maximum and sum; the four waves' results are joined.
__global__ __launch_bounds__(256) void k_attend(AttendArgs a) {
    __shared__ float sq[256], so[4][256], sm[4], sl[4];
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
    const KvPool& p = a.pool;
    const bool bytes = p.type != kKvBf16;
    const int b = blockIdx.x, h = blockIdx.y, hk = h / a.group;
    const KvSpan span = span_of(a.seqs, b);
    for (int i = blockIdx.z; i < span.n; i += gridDim.z) {
        const int64_t row = span.row0 + i, pos = span.pos0 + i;
        __syncthreads();
        if (tid < p.d) {
            const int64_t o = row * a.q_row + (int64_t)h * p.d + tid;
            sq[tid] = a.dtype == 0 ? ((const float*)a.q)[o] : bf16_to_f32(((const uint16_t*)a.q)[o]);
        }
        __syncthreads();
        const int64_t first = a.window > 0 && pos - a.window + 1 > 0 ? pos - a.window + 1 : 0;
        float m = -__builtin_inff(), l = 0.0f, acc[4] = {};
        for (int64_t j0 = (first & ~int64_t(63)) + 64 * wid; j0 <= pos; j0 += 256) {
            const int64_t j = j0 + lane;
            const int64_t page = j >= first && j <= pos ? page_of(p, a.seqs, b, j) : -1;
            const int at = (int)(j & ((1 << p.page_shift) - 1));
            float s = -__builtin_inff(), vs = 1.0f;
            int64_t base = 0;
            if (page >= 0) {
                base = tile_base(p, page, hk, at);
                float dot = 0.0f;
                for (int c = 0; c < p.d; ++c) dot += sq[c] * kv_value(p.k, base + k_place(at & 31, c, bytes), p.type);
                if (bytes) {
                    dot *= p.k_scale[scale_at(p, page, hk, at)];
                    vs = p.v_scale[scale_at(p, page, hk, at)];
                }
                s = dot * a.scale;
            }
            const float M = fmaxf(m, wave_reduce(s, [](float u, float v) { return fmaxf(u, v); }));
            const uint64_t live = __ballot(page >= 0);
            if (M == -__builtin_inff()) continue;
            const float keep = m == -__builtin_inff() ? 0.0f : __expf(m - M);
            const float w = page >= 0 ? __expf(s - M) : 0.0f;
            l = l * keep + wave_sum_f32(w);
            m = M;
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] *= keep;
            for (int t = 0; t < 64; ++t) {
                if (!(live >> t & 1)) continue;
                const float wt = __shfl(w * vs, t, kWave);
                const int64_t bt = __shfl(base, t, kWave);
                const int place = (int)((j0 + t) & 31);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (lane + 64 * e < p.d)
                        acc[e] += wt * kv_value(p.v, bt + v_place(place, lane + 64 * e, bytes), p.type);
            }
        }
        if (lane == 0) {
            sm[wid] = m;
            sl[wid] = l;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) so[wid][lane + 64 * e] = acc[e];
        __syncthreads();
        float M = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3])), L = 0.0f, o = 0.0f;
        for (int w = 0; w < 4; ++w)
            if (sm[w] != -__builtin_inff()) {
                const float f = __expf(sm[w] - M);
                L += sl[w] * f;
                o += so[w][tid] * f;
            }
        if (tid < p.d) {
            const int64_t at = (row * a.q_heads + h) * p.d + tid;
            o = L > 0.0f ? o / L : 0.0f;
            if (a.dtype == 0) ((float*)a.out)[at] = o;
            else ((uint16_t*)a.out)[at] = f32_to_bf16(o);
        }
        if (tid == 0 && a.lse) a.lse[row * a.q_heads + h] = L > 0.0f ? M + __logf(L) : -__builtin_inff();
    }
}

int64_t attend_workspace(const KvPool&, int, int, int, int, int) { return 0; }

hipError_t launch_kv_attend(const AttendArgs& a, int max_new, void*, int, hipStream_t s) {
    if (a.seqs.rows <= 0 || a.seqs.n_seq <= 0) return hipSuccess;
    const int64_t most = max_new > 0 && max_new < a.seqs.rows ? max_new : a.seqs.rows;
    k_attend<<<dim3((unsigned)a.seqs.n_seq, (unsigned)a.q_heads, (unsigned)(most > 1024 ? 1024 : most)), dim3(256), 0,
               s>>>(a);
    return hipGetLastError();
}

}  // namespace lacache
