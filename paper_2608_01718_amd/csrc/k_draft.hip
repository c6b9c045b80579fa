// k_draft.hip -- sampled verification of drafted tokens (lacache_verify).
//
//   p = softmax(l / T), q = softmax(l' / T);  draft j is taken while u_j q(x_j) < p(x_j);  behind the n that were taken the
//   next token is the first v with r(0) + .. + r(v) > u sum r, r = max(0, p - q) of row n (p itself behind the last draft)
//
// How many drafts are taken and which token comes next are whole numbers, so both are what 64 bits give:
//   1. k_draft_stats reads all rows once: a workgroup takes a chunk of a row into registers and writes its maximum and its
//      sum of exponentials in float32.  This is the launch that the memory bounds.
//   2. k_draft_sums takes the drafts.  With numerators in 64 bits the relative error of p and q is that of the sums alone
//      (kSumError), so a comparison that is closer than that is done again with sums in 64 bits; about one in 50,000 is.
//      Then it adds up row n of both models in 64 bits.
//   3. k_draft_pick adds up r by chunks, and the last workgroup of a sequence finds the chunk and in it the token.
#include "common.hpp"
#include "draft.hpp"
#include "launch.hpp"

namespace lacache {

namespace {

constexpr int kThreads = 256;
constexpr int kPositions = 64;  // looked at together

// Relative error of a chunked float32 sum S = sum 2^t, t = (x - m) c <= 0.  An exponent's three roundings (c, the
// difference, the product) move 2^t by 3 |t| 2^-24 ln 2, the exponential is within 2^-22, adding up 32 of a thread in
// pairs and 256 threads in a tree are 13 roundings.  The mean of |t| under the weights is below log2 V + 2 (their entropy
// and the maximum's share), 33 for 2^31 logits: 33 * 1.24e-7 + 2.4e-7 + 13 * 6e-8 = 5.1e-6 for S, twice that for S_p / S_q.
constexpr double kSumError = 0x1p-16;

// 2^t for t <= 0: 2^n e^(f ln 2), |f| <= 1/2, by the exponential's series up to the 11th power (the 12th: 0.3466^12 / 12! =
// 6e-15).  Below 2^-1074 it is 0.
__device__ __forceinline__ double exp2_64(double t) {
    t = fmax(t, -1100.0);
    const double n = __builtin_rint(t), f = (t - n) * 0.693147180559945309417;
    double y = 1.0 / 39916800.0;
    y = __builtin_fma(y, f, 1.0 / 3628800.0);
    y = __builtin_fma(y, f, 1.0 / 362880.0);
    y = __builtin_fma(y, f, 1.0 / 40320.0);
    y = __builtin_fma(y, f, 1.0 / 5040.0);
    y = __builtin_fma(y, f, 1.0 / 720.0);
    y = __builtin_fma(y, f, 1.0 / 120.0);
    y = __builtin_fma(y, f, 1.0 / 24.0);
    y = __builtin_fma(y, f, 1.0 / 6.0);
    y = __builtin_fma(y, f, 0.5);
    y = __builtin_fma(y, f, 1.0);
    y = __builtin_fma(y, f, 1.0);
    return __builtin_ldexp(y, (int)n);
}
constexpr double kLog2e64 = 1.44269504088896340736;

// A sequence's temperature: log2 e / T, and whether it is greedy (T not in 2^-60 .. 2^60).
struct Heat {
    double c;
    bool greedy;
};
__device__ __forceinline__ Heat heat_of(const DraftArgs& a, int b) {
    const double t = a.temperature ? (double)a.temperature[b] : 1.0;
    const bool greedy = !(t >= 0x1p-60 && t <= 0x1p60);
    return {greedy ? kLog2e64 : kLog2e64 / t, greedy};
}
__device__ __forceinline__ int drafts_of(const DraftArgs& a, int b) {
    const int n = a.n_draft ? a.n_draft[b] : a.k;
    return n < 0 ? 0 : n > a.k ? a.k : n;
}

// Logits v .. v + 7 of a row (rows begin at any element), -infinity from V on.
__device__ __forceinline__ void logits8(const char* row, int dtype, int V, int64_t v, float (&x)[8]) {
    typedef u32x4 any2 __attribute__((aligned(2)));
    typedef f32x4 any4 __attribute__((aligned(4)));
    if (v + 8 <= V) {
        if (dtype == 0) {
            const f32x4 p = __builtin_nontemporal_load((const any4*)(row + v * 4)),
                        q = __builtin_nontemporal_load((const any4*)(row + v * 4 + 16));
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = p[e], x[4 + e] = q[e];
        } else {
            const u32x4 w = __builtin_nontemporal_load((const any2*)(row + v * 2));
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[2 * e] = __uint_as_float(w[e] << 16);
                x[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
            }
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            x[e] = v + e >= V     ? -__builtin_inff()
                   : dtype == 0 ? ((const float*)row)[v + e]
                                : bf16_to_f32(((const uint16_t*)row)[v + e]);
    }
}
__device__ __forceinline__ float logit(const char* row, int dtype, int64_t v) {
    return dtype == 0 ? ((const float*)row)[v] : bf16_to_f32(((const uint16_t*)row)[v]);
}
__device__ __forceinline__ const char* row_of(const DraftArgs& a, int b, int j, bool draft) {
    const int64_t at = draft ? b * a.d_seq + j * a.d_row : b * a.t_seq + j * a.t_row;
    return (draft ? a.draft_logits : a.logits) + at * (a.dtype == 0 ? 4 : 2);
}
// Where the statistics of a row lie: the target's k + 1 rows of a sequence, then the draft model's k.
__device__ __forceinline__ int64_t stat_row(const DraftArgs& a, int b, int j, bool draft) {
    return (int64_t)b * (2 * a.k + 1) + (draft ? a.k + 1 + j : j);
}

template <class T, class Op>
__device__ __forceinline__ T all_threads(T x, T (&lds)[kThreads / 64], Op op) {
    x = wave_reduce(x, op);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    x = lds[0];
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) x = op(x, lds[w]);
    return x;
}

// Maximum and sum of a row from its chunks, sixteen lanes a row (all of them get both).  A sum that is not finite, or no
// sum at all, is that of a row without probabilities; 0 stands for it.
struct Stat {
    float m;
    double s;
};
__device__ __forceinline__ Stat join_chunks(const DraftArgs& a, int64_t row, double c) {
    const float2* part = a.stats + row * a.chunks;
    float m = -__builtin_inff();
    for (int i = threadIdx.x & 15; i < a.chunks; i += 16) m = fmaxf(m, part[i].x);
    auto max2 = [](float x, float y) { return fmaxf(x, y); };
    m = xor_combine<1>(xor_combine<2>(xor_combine<4>(xor_combine<8>(m, max2), max2), max2), max2);
    double s = 0.0;
    const bool fine = m < __builtin_inff() && m > -__builtin_inff();
    for (int i = threadIdx.x & 15; i < a.chunks; i += 16) {
        const float2 x = part[i];
        s += x.y * (fine && x.x > -__builtin_inff() ? exp2_64(((double)x.x - m) * c) : 1.0);
    }
    auto add2 = [](double x, double y) { return x + y; };
    s = xor_combine<1>(xor_combine<2>(xor_combine<4>(xor_combine<8>(s, add2), add2), add2), add2);
    return {m, fine && s > 0.0 && s < __builtin_inf() ? s : 0.0};
}

}  // namespace

// A workgroup a chunk of NV x 2048 logits of a row.
template <int NV>
__global__ __launch_bounds__(kThreads) void k_draft_stats(DraftArgs a) {
    __shared__ float lds[kThreads / 64], lds2[kThreads / 64];
    const int tid = threadIdx.x;
    const int64_t rows = (int64_t)a.B * (2 * a.k + 1);
    for (int64_t item = blockIdx.x; item < rows * a.chunks; item += gridDim.x) {
        const int64_t row = item / a.chunks;
        const int chunk = (int)(item - row * a.chunks);
        const int b = (int)(row / (2 * a.k + 1)), i = (int)(row - (int64_t)b * (2 * a.k + 1));
        const bool draft = i > a.k;
        const int j = draft ? i - a.k - 1 : i, n = drafts_of(a, b);
        const Heat heat = heat_of(a, b);
        if (tid == 0 && chunk == 0 && i == 0) a.done[b] = 0;
        if (draft ? (j >= n || heat.greedy) : j > n) continue;
        const char* at = row_of(a, b, j, draft);
        const int64_t v0 = (int64_t)chunk * (NV * 8 * kThreads);
        float x[NV][8];
#pragma unroll
        for (int u = 0; u < NV; ++u) {
            const int64_t v = v0 + (u * kThreads + tid) * 8;
            if (v < a.V) {
                logits8(at, a.dtype, a.V, v, x[u]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[u][e] = -__builtin_inff();
            }
        }
        float m = -__builtin_inff();
        float nan = 0.0f;  // (the maximum leaves NaN out)
#pragma unroll
        for (int u = 0; u < NV; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                m = fmaxf(m, x[u][e]);
                nan = x[u][e] == x[u][e] ? nan : x[u][e];
            }
        m = all_threads(m, lds, [](float p, float q) { return fmaxf(p, q); });
        const float base = m > -__builtin_inff() ? m : 0.0f, c = (float)heat.c;
        float s = 0.0f;
#pragma unroll
        for (int u = 0; u < NV; ++u) {
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = __builtin_amdgcn_exp2f((x[u][e] - base) * c);
            s += ((y[0] + y[1]) + (y[2] + y[3])) + ((y[4] + y[5]) + (y[6] + y[7]));
        }
        s = all_threads(s + nan, lds2, [](float p, float q) { return p + q; });
        if (tid == 0) a.stats[row * a.chunks + chunk] = make_float2(m, s);
    }
}

namespace {

// The sum of a whole row in 64 bits, by all threads.
__device__ double row_sum(const DraftArgs& a, const char* row, float m, double c, double (&lds)[kThreads / 64]) {
    double s = 0.0;
    for (int64_t v = threadIdx.x * 8; v < a.V; v += kThreads * 8) {
        float x[8];
        logits8(row, a.dtype, a.V, v, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) s += exp2_64(((double)x[e] - m) * c);
    }
    return all_threads(s, lds, [](double p, double q) { return p + q; });
}

}  // namespace

// Workgroup b wides + w: how many drafts of sequence b are taken (every workgroup of b finds out, the first writes it down), and the
// w-th chunks of row n of both models in 64 bits.
__global__ __launch_bounds__(kThreads) void k_draft_sums(DraftArgs a) {
    __shared__ float max_of[2][kPositions];
    __shared__ double sum_of[2][kPositions], lds[kThreads / 64];
    __shared__ uint64_t flags[2];  // the positions that are not taken, and those that are too close
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
    const int b = blockIdx.x / a.wides, w = blockIdx.x % a.wides, n = drafts_of(a, b);
    const Heat heat = heat_of(a, b);
    int taken = n;
    for (int j0 = 0; j0 < n; j0 += kPositions) {
        const int here = n - j0 < kPositions ? n - j0 : kPositions;
        __syncthreads();
        for (int i = tid >> 4; i < 2 * here; i += kThreads / 16) {
            const bool draft = i >= here;
            const int j = draft ? i - here : i;
            Stat s{0.0f, 0.0};
            if (!(draft && heat.greedy)) s = join_chunks(a, stat_row(a, b, j0 + j, draft), heat.c);
            if ((tid & 15) == 0) max_of[draft][j] = s.m, sum_of[draft][j] = s.s;
        }
        __syncthreads();
        double pn = 0.0, qn = 0.0;  // numerators of p and q
        float u = 0.0f;
        if (wid == 0) {
            bool no = false, close = false;
            if (lane < here) {
                const int j = j0 + lane, t = a.tokens[(int64_t)b * a.k + j];
                u = a.u_accept[(int64_t)b * a.k + j];
                const bool there = t >= 0 && t < a.V;
                const double sp = sum_of[0][lane], sq = sum_of[1][lane];
                float p = 0.0f, q = 0.0f;
                if (there && sp > 0.0) {
                    const float x = logit(row_of(a, b, j, false), a.dtype, t);
                    pn = heat.greedy ? (x == max_of[0][lane] ? 1.0 : 0.0) : exp2_64(((double)x - max_of[0][lane]) * heat.c);
                    p = (float)(heat.greedy ? pn : pn / sp);
                }
                if (heat.greedy) {
                    q = 1.0f;
                    no = pn == 0.0;
                } else if (sp > 0.0 && sq > 0.0) {
                    if (there) {
                        const float x = logit(row_of(a, b, j, true), a.dtype, t);
                        qn = exp2_64(((double)x - max_of[1][lane]) * heat.c);
                        q = (float)(qn / sq);
                    }
                    const double l = u * (qn / sq), r = pn / sp;
                    no = !(l < r);
                    close = fabs(l - r) <= kSumError * r && r > 0.0;
                } else {
                    no = true;
                }
                if (w == 0) {
                    a.p_target[(int64_t)b * a.k + j] = p;
                    a.p_draft[(int64_t)b * a.k + j] = q;
                }
            }
            const uint64_t n0 = __ballot(no), n1 = __ballot(close);
            if (lane == 0) flags[0] = n0, flags[1] = n1;
        }
        __syncthreads();
        if (taken == n) {
            uint64_t no = flags[0], close = flags[1];
            while (no | close) {
                const int at = __ffsll((unsigned long long)(no | close)) - 1;
                if (close >> at & 1) {
                    const double sp = row_sum(a, row_of(a, b, j0 + at, false), max_of[0][at], heat.c, lds);
                    const double sq = row_sum(a, row_of(a, b, j0 + at, true), max_of[1][at], heat.c, lds);
                    __syncthreads();
                    if (tid == at) flags[0] = u * (qn / sq) < pn / sp;  // (the lane that has this position's numerators)
                    __syncthreads();
                    if (flags[0]) {
                        no &= ~(1ull << at);
                        close &= ~(1ull << at);
                        continue;
                    }
                }
                taken = j0 + at;
                break;
            }
        }
        if (taken < n && w != 0) break;
    }
    if (w == 0) {
        for (int j = n + tid; j < a.k; j += kThreads) a.p_target[(int64_t)b * a.k + j] = a.p_draft[(int64_t)b * a.k + j] = 0.0f;
    }
    // row `taken` of both
    const Stat t = join_chunks(a, stat_row(a, b, taken, false), heat.c);
    Stat d{0.0f, 0.0};
    if (taken < n && !heat.greedy) d = join_chunks(a, stat_row(a, b, taken, true), heat.c);
    if (w == 0 && tid == 0) {
        a.accept_len[b] = taken;
        a.rows[b] = DraftRow{taken, t.s > 0.0 ? 1 : 0, d.s > 0.0 ? 1 : 0, t.m, d.m};
    }
    if (heat.greedy) return;
    double sp = 0.0, sq = 0.0;
    const int64_t end = (int64_t)(w + 1) * a.wide < a.V ? (int64_t)(w + 1) * a.wide : a.V;
    const char *rt = row_of(a, b, taken, false), *rd = d.s > 0.0 ? row_of(a, b, taken, true) : nullptr;
    for (int64_t v = (int64_t)w * a.wide + tid * 8; v < end; v += kThreads * 8) {
        float x[8], y[8];
        logits8(rt, a.dtype, a.V, v, x);
        if (rd) logits8(rd, a.dtype, a.V, v, y);
#pragma unroll
        for (int e = 0; e < 8; ++e) sp += exp2_64(((double)x[e] - t.m) * heat.c);
        if (rd) {
#pragma unroll
            for (int e = 0; e < 8; ++e) sq += exp2_64(((double)y[e] - d.m) * heat.c);
        }
    }
    auto add2 = [](double p, double q) { return p + q; };
    sp = all_threads(sp, lds, add2);
    sq = all_threads(sq, lds, add2);
    if (tid == 0) a.sums[(int64_t)b * a.wides + w] = make_double2(sp, sq);
}

namespace {

// r of eight logits
struct Rest {
    const char *rt, *rd;  // rd null: nothing is taken off
    double mt, md, ft, fd, c;
    __device__ __forceinline__ void at(const DraftArgs& a, int64_t v, double (&r)[8]) const {
        float x[8];
        logits8(rt, a.dtype, a.V, v, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = exp2_64(((double)x[e] - mt) * c) * ft;
        if (rd) {
            logits8(rd, a.dtype, a.V, v, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) r[e] = fmax(0.0, r[e] - exp2_64(((double)x[e] - md) * c) * fd);
        }
    }
};

__device__ __forceinline__ double scan_wave(double x, int lane) {
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        const double y = __shfl_up(x, o, 64);
        if (lane >= o) x += y;
    }
    return x;
}

}  // namespace

// Workgroup b wides + w: the sum of r over the w-th chunk; the last workgroup of b finds the token.
__global__ __launch_bounds__(kThreads) void k_draft_pick(DraftArgs a) {
    __shared__ double lds[kThreads / 64], before[kThreads / 64 + 1];
    __shared__ int found, last;
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
    const int b = blockIdx.x / a.wides, w = blockIdx.x % a.wides;
    const Heat heat = heat_of(a, b);
    const DraftRow row = a.rows[b];
    if (!row.has_p) {
        if (w == 0 && tid == 0) a.next_token[b] = -1;
        return;
    }
    auto add2 = [](double p, double q) { return p + q; };
    const char* rt = row_of(a, b, row.n, false);
    const int64_t begin = (int64_t)w * a.wide, end = begin + a.wide < a.V ? begin + a.wide : a.V;
    // the parts of a sum over all chunks: device-wide, since workgroups of one launch write and read them
    auto put = [&](double x) {
        __hip_atomic_store((uint64_t*)(a.rest + (int64_t)b * a.wides + w), (uint64_t)__double_as_longlong(x), __ATOMIC_RELAXED,
                           __HIP_MEMORY_SCOPE_AGENT);
    };
    auto get = [&](int i) {
        return __longlong_as_double((long long)__hip_atomic_load((const uint64_t*)(a.rest + (int64_t)b * a.wides + i),
                                                                 __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
    };
    auto is_last = [&]() {
        last_workgroup_wait();
        __syncthreads();
        if (tid == 0)
            last = __hip_atomic_fetch_add(a.done + b, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)a.wides - 1;
        __syncthreads();
        return last;
    };
    if (heat.greedy) {  // the first of the largest
        int first = INT32_MAX;
        for (int64_t v = begin + tid * 8; v < end; v += kThreads * 8) {
            float x[8];
            logits8(rt, a.dtype, a.V, v, x);
#pragma unroll
            for (int e = 7; e >= 0; --e) first = x[e] == row.mt && v + e < first ? (int)(v + e) : first;
        }
        auto min2 = [](double p, double q) { return fmin(p, q); };
        const double f = all_threads((double)first, lds, min2);
        if (tid == 0) put(f);
        if (!is_last()) return;
        double x = INT32_MAX;
        for (int i = tid; i < a.wides; i += kThreads) x = fmin(x, get(i));
        x = all_threads(x, lds, min2);
        if (tid == 0) a.next_token[b] = (int)x;
        return;
    }
    double sp = 0.0, sq = 0.0;
    for (int i = tid; i < a.wides; i += kThreads) {
        const double2 s = a.sums[(int64_t)b * a.wides + i];
        sp += s.x, sq += s.y;
    }
    sp = all_threads(sp, lds, add2);
    sq = all_threads(sq, lds, add2);
    Rest rest{rt, row.has_q ? row_of(a, b, row.n, true) : nullptr, row.mt, row.md, 1.0 / sp, row.has_q ? 1.0 / sq : 0.0, heat.c};
    double s = 0.0;
    for (int64_t v = begin + tid * 8; v < end; v += kThreads * 8) {
        double r[8];
        rest.at(a, v, r);
#pragma unroll
        for (int e = 0; e < 8; ++e) s += r[e];
    }
    s = all_threads(s, lds, add2);
    if (tid == 0) put(s);
    if (!is_last()) return;

    double all = 0.0;
    for (int i = tid; i < a.wides; i += kThreads) all += get(i);
    all = all_threads(all, lds, add2);
    const bool none = rest.rd && !(all > 0x1p-30);  // p and q are the same: the token is drawn from p
    if (none) rest.rd = nullptr;
    auto part = [&](int i) { return none ? a.sums[(int64_t)b * a.wides + i].x * rest.ft : get(i); };
    // Finds the first of `count` ordered parts that takes the running sum past `goal` (the last one above 0 if none does): a
    // thread `each` of them, from tid * each on.  What lies before it is taken off goal.
    auto find = [&](auto part_at, int64_t count, int64_t each, double& goal, bool whole) -> int64_t {
        double own = 0.0;
        for (int64_t i = tid * each; i < (tid + 1) * each && i < count; ++i) own += part_at(i);
        double upto = scan_wave(own, lane);
        __syncthreads();
        if (lane == 63) lds[wid] = upto;
        if (tid == 0) found = -1;
        __syncthreads();
        double lead = 0.0, total = 0.0;
        for (int i = 0; i < kThreads / 64; ++i) {
            lead += i < wid ? lds[i] : 0.0;
            total += lds[i];
        }
        upto += lead;
        const double target = whole ? goal * total : goal;  // (a share of the sum, or a sum)
        const uint64_t past = __ballot(upto > target && own > 0.0), some = __ballot(own > 0.0);
        __shared__ int wave_past[kThreads / 64], wave_some[kThreads / 64];
        __syncthreads();
        if (lane == 0) {
            wave_past[wid] = past ? wid * 64 + __ffsll((unsigned long long)past) - 1 : -1;
            wave_some[wid] = some ? wid * 64 + 63 - __clzll((long long)some) : -1;
        }
        __syncthreads();
        int who = -1;
        for (int i = kThreads / 64 - 1; i >= 0; --i) who = wave_past[i] >= 0 ? wave_past[i] : who;
        const bool passes = who >= 0;
        if (!passes)
            for (int i = 0; i < kThreads / 64; ++i) who = wave_some[i] >= 0 ? wave_some[i] : who;
        if (tid == who) {
            double sum = upto - own;
            int64_t at = -1;
            for (int64_t i = tid * each; i < (tid + 1) * each && i < count; ++i) {
                const double x = part_at(i);
                if (x > 0.0) {
                    at = i;
                    before[0] = sum;
                    if (passes && sum + x > target) break;
                }
                sum += x;
            }
            found = (int)at;
            before[1] = target;
        }
        __syncthreads();
        goal = before[1] - before[0];
        return found;
    };
    double goal = a.u_next[b];
    const int64_t chunk = find(part, a.wides, (a.wides + kThreads - 1) / kThreads, goal, true);
    if (chunk < 0) {  // (a sum that is NaN)
        if (tid == 0) a.next_token[b] = -1;
        return;
    }
    const int64_t v0 = chunk * a.wide, count = a.V - v0 < a.wide ? a.V - v0 : a.wide;
    auto one = [&](int64_t eight) {
        double r[8], x = 0.0;
        rest.at(a, v0 + eight * 8, r);
#pragma unroll
        for (int e = 0; e < 8; ++e) x += r[e];
        return x;
    };
    const int64_t eights = (count + 7) / 8;
    const int64_t eight = find(one, eights, (eights + kThreads - 1) / kThreads, goal, false);
    if (tid == 0) {
        int64_t token = -1;
        if (eight >= 0) {
            double r[8], sum = 0.0;
            rest.at(a, v0 + eight * 8, r);
            bool past = false;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (!past && r[e] > 0.0) {
                    token = v0 + eight * 8 + e;
                    past = sum + r[e] > goal;
                }
                sum += r[e];
            }
        }
        a.next_token[b] = (int)token;
    }
}

namespace {

constexpr int64_t kSmall = 2048, kLarge = 8192;  // logits of a chunk of k_draft_stats

int64_t chunk_of(int V, int64_t rows) { return rows * ((V + kLarge - 1) / kLarge) >= 1024 ? kLarge : kSmall; }

void shape(DraftArgs& a, char* space, int64_t* bytes) {
    const int64_t rows = (int64_t)a.B * (2 * a.k + 1), chunk = chunk_of(a.V, rows);
    a.chunks = (int)((a.V + chunk - 1) / chunk);
    // about a thousand workgroups for the rows that 64 bits are needed for
    const int64_t least = (a.V + kSmall - 1) / kSmall, want = a.B < 1024 ? (1023 + a.B) / a.B : 1, wides = want < least ? want : least;
    a.wide = ((a.V + wides - 1) / wides + kSmall - 1) / kSmall * kSmall;
    a.wides = (int)((a.V + a.wide - 1) / a.wide);
    int64_t at = 0;
    auto take = [&](int64_t n) {
        char* p = space + at;
        at += (n + 15) & ~int64_t(15);
        return p;
    };
    a.sums = (double2*)take(16 * (int64_t)a.B * a.wides);
    a.rest = (double*)take(8 * (int64_t)a.B * a.wides);
    a.stats = (float2*)take(8 * rows * a.chunks);
    a.rows = (DraftRow*)take((int64_t)sizeof(DraftRow) * a.B);
    a.done = (uint32_t*)take(4 * (int64_t)a.B);
    *bytes = at;
}

}  // namespace

int64_t draft_workspace(int V, int B, int k) {
    DraftArgs a{};
    a.V = V, a.B = B, a.k = k;
    int64_t bytes = 0;
    if (B > 0) shape(a, nullptr, &bytes);
    return bytes;
}

hipError_t launch_verify_drafts(DraftArgs a, void* workspace, hipStream_t s) {
    int64_t bytes;
    shape(a, (char*)workspace, &bytes);
    const int64_t rows = (int64_t)a.B * (2 * a.k + 1);
    const dim3 grid((unsigned)grid_blocks(rows * a.chunks)), block(kThreads);
    if (chunk_of(a.V, rows) == kLarge) k_draft_stats<4><<<grid, block, 0, s>>>(a);
    else k_draft_stats<1><<<grid, block, 0, s>>>(a);
    k_draft_sums<<<dim3((unsigned)(a.wides * a.B)), block, 0, s>>>(a);
    k_draft_pick<<<dim3((unsigned)(a.wides * a.B)), block, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace lacache
