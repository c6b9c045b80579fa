// k_draft.hip -- sampled verification of drafted tokens (lacache_verify).
//
//   p = softmax(l / T), q = softmax(l' / T);  draft j is taken while u_j q(x_j) < p(x_j);  behind the n that were taken the
//   next token is the first v with r(0) + .. + r(v) > u sum r, r = max(0, p - q) of row n (p itself behind the last draft)
//
// How many drafts are taken and which token comes next are whole numbers, so both are what 64 bits give:
//   1. k_draft_stats reads all rows once: a wave takes a chunk of a row into registers and writes its maximum and its sum of
//      exponentials in float32.  This is the launch that the memory bounds.
//   2. k_draft_accept takes the drafts.  With numerators in 64 bits the relative error of p and q is that of the sums alone
//      (kSumError), so a comparison that is closer than that is done again with sums in 64 bits; few are.
//   3. k_draft_sums adds up row n of both models in 64 bits, a wave a piece, k_draft_rest r.  Exponentials bound them.
//   4. k_draft_pick finds a sequence's piece and in it the token.
// Where there are few pieces launches are most of the time: then every workgroup of k_draft_sums finds out by itself how many
// drafts are taken, and the last workgroup of a sequence in k_draft_rest finds the token (TOGETHER; a sequence with
// four drafts of 32,000 tokens 21 us, 31 in five launches).
#include "common.hpp"
#include "draft.hpp"
#include "launch.hpp"

namespace lacache {

namespace {

constexpr int kThreads = 256;
constexpr int kAccept = 512;    // threads of k_draft_accept
constexpr int kPositions = 64;  // looked at together

// Relative error of a chunked float32 sum S = sum 2^t, t = (x - m) c <= 0, of 2^log2_v logits.  Four roundings of an exponent (log2
// e, c, the difference, the product) move 2^t by 4 |t| 2^-24 ln 2, whether it is taken in one step or in several; the mean of |t|
// under the weights is below log2 V + 2 (their entropy and the maximum's share).  The exponentials (one, and up to five as the
// maximum rises and lanes are joined) are within 2^-22 each.  A lane adds a chunk of four steps up in 3 + 4 x 4 roundings, four
// more as the maximum rises, and a wave in 6.  (8.6e-6 for the longest rows, 6.3e-6 for 128,256 logits.)
constexpr double sum_error(double log2_v) {
    return (log2_v + 2) * 4 * 0x1p-24 * 0.6931472 + 6 * 0x1p-22 + (3 + 4 * 4 + 4 + 6) * 0x1p-24;
}
constexpr double kSumError = 0x1p-15;
static_assert(2 * sum_error(31) < kSumError, "S_p / S_q of rows of any length");

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

// 2^t for t <= 0 where many are needed: 2^f, |f| <= 1/2, by the polynomial of degree 9 that is exact at the zeros of the
// Chebyshev polynomial of degree 10 (2e-14 of 2^f), times 2^n; adding 1.5 2^52 leaves n in the low bits.  Below 2^-1074 it is 0.
// (Where little is left of p - q both have nearly the same t, and so the same error: running sums of r are 2e-8 of it off where its
// sum is 2^-32, 1e-8 with 64-bit exponentials; 7e-14 and 6e-15 where it is 4e-4.)
// (Both models' rows of 64 sequences, 16.4M logits: k_draft_sums 17 us, 27 with the series above.)
__device__ __forceinline__ double exp2_many(double t) {
    t = fmax(t, -1100.0);
    const double z = t + 0x1.8p52, f = t - (z - 0x1.8p52);
    double y = 1.0205905413765595e-07;
    y = __builtin_fma(y, f, 1.325964524488711e-06);
    y = __builtin_fma(y, f, 1.5252672924850737e-05);
    y = __builtin_fma(y, f, 0.0001540343375125101);
    y = __builtin_fma(y, f, 0.0013333558200794592);
    y = __builtin_fma(y, f, 0.009618129193934313);
    y = __builtin_fma(y, f, 0.05550410866465167);
    y = __builtin_fma(y, f, 0.2402265069564034);
    y = __builtin_fma(y, f, 0.6931471805599462);
    y = __builtin_fma(y, f, 1.0000000000000135);
    return __builtin_ldexp(y, (int)(uint32_t)__double_as_longlong(z));
}

// A sequence's temperature: log2 e / T, and whether it is greedy (T not in 2^-60 .. 2^60).
struct Heat {
    double c;
    bool greedy;
};
__device__ __forceinline__ bool is_greedy(float t) { return !(t >= 0x1p-60f && t <= 0x1p60f); }
__device__ __forceinline__ Heat heat_of(const DraftArgs& a, int b) {
    const float t = a.temperature ? a.temperature[b] : 1.0f;
    const bool greedy = is_greedy(t);
    return {greedy ? kLog2e64 : kLog2e64 / (double)t, greedy};
}
__device__ __forceinline__ int drafts_of(const DraftArgs& a, int b) {
    const int n = a.n_draft ? a.n_draft[b] : a.k;
    return n < 0 ? 0 : n > a.k ? a.k : n;
}

// Eight logits of a row (which begins at any element) as they lie in memory.  ONCE: they are not read again.
template <bool F32>
struct Raw8 {
    u32x4 w[F32 ? 2 : 1];
    template <bool ONCE>
    __device__ __forceinline__ void load(const char* row, int64_t v) {
        typedef u32x4 any __attribute__((aligned(2)));
        const any* p = (const any*)(row + v * (F32 ? 4 : 2));
        w[0] = ONCE ? __builtin_nontemporal_load(p) : *p;
        if constexpr (F32) w[1] = ONCE ? __builtin_nontemporal_load(p + 1) : p[1];
    }
    __device__ __forceinline__ void unpack(float (&x)[8]) const {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (F32) {
                x[e] = __uint_as_float(w[0][e]), x[4 + e] = __uint_as_float(w[1][e]);
            } else {
                x[2 * e] = __uint_as_float(w[0][e] << 16);
                x[2 * e + 1] = __uint_as_float(w[0][e] & 0xFFFF0000u);
            }
        }
    }
};
// NV times eight logits, from v on and `step` apart, -infinity from V on.  inside: all of the wave's are there, and their loads
// are issued together.
template <bool F32, int NV, bool ONCE>
__device__ __forceinline__ void logits8(const char* row, int V, int64_t v, int64_t step, bool inside, float (&x)[NV][8]) {
    Raw8<F32> raw[NV];
    if (inside) {
#pragma unroll
        for (int i = 0; i < NV; ++i) raw[i].template load<ONCE>(row, v + i * step);
#pragma unroll
        for (int i = 0; i < NV; ++i) raw[i].unpack(x[i]);
        return;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int64_t at = v + i * step;
        if (at + 8 <= V) {
            raw[i].template load<ONCE>(row, at);
            raw[i].unpack(x[i]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                x[i][e] = at + e >= V ? -__builtin_inff()
                          : F32       ? ((const float*)row)[at + e]
                                      : bf16_to_f32(((const uint16_t*)row)[at + e]);
        }
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

template <int THREADS, class T, class Op>
__device__ __forceinline__ T all_threads(T x, T (&lds)[THREADS / 64], Op op) {
    x = wave_reduce(x, op);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    x = lds[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) x = op(x, lds[w]);
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
    auto max2 = [](float x, float y) { return fmaxf(x, y); };
    auto add2 = [](double x, double y) { return x + y; };
    // (four at a time on their way, kept for the sum where that is all)
    float2 x[4];
    auto load = [&](int i0) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int i = i0 + 16 * k + (threadIdx.x & 15);
            x[k] = i < a.chunks ? part[i] : make_float2(-__builtin_inff(), 0.0f);
        }
    };
    float m = -__builtin_inff();
    for (int i0 = 0; i0 < a.chunks; i0 += 64) {
        load(i0);
#pragma unroll
        for (int k = 0; k < 4; ++k) m = fmaxf(m, x[k].x);
    }
    m = xor_combine<1>(xor_combine<2>(xor_combine<4>(xor_combine<8>(m, max2), max2), max2), max2);
    double s = 0.0;
    const bool fine = m < __builtin_inff() && m > -__builtin_inff();
    for (int i0 = 0; i0 < a.chunks; i0 += 64) {
        if (a.chunks > 64) load(i0);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            s += x[k].y * (fine && x[k].x > -__builtin_inff() ? exp2_64(((double)x[k].x - m) * c) : 1.0);
    }
    s = xor_combine<1>(xor_combine<2>(xor_combine<4>(xor_combine<8>(s, add2), add2), add2), add2);
    return {m, fine && s > 0.0 && s < __builtin_inf() ? s : 0.0};
}

}  // namespace

// A wave a chunk of a row: STEPS times NV x 512 logits, the next of them on their way while one is worked with.  The vector
// unit is busy for most of the time of the launch (32 logits a lane: 32 exponentials at a quarter of its rate), so what a wave
// works out for itself is spread over 8192 logits where there are many.  (64 sequences of up to 20 drafts of 128,256 in bfloat16,
// 552 MB: 84 us, 6.6 TB/s; 98 with 2048 logits a wave.)
template <int NV, int STEPS, bool F32>
__global__ __launch_bounds__(kThreads) void k_draft_stats(DraftArgs a) {
    constexpr int64_t kStep = NV * 512, kChunk = kStep * STEPS;
    const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t each = 2 * (uint32_t)a.k + 1;
    const int64_t items = (int64_t)a.B * each * a.chunks;
    for (int64_t item = (int64_t)blockIdx.x * (kThreads / 64) + wid; item < items; item += (int64_t)gridDim.x * (kThreads / 64)) {
        int64_t row;
        int chunk, b, i;
        if (items <= UINT32_MAX) {  // (divisions in 32 bits where that is enough)
            const uint32_t r = (uint32_t)item / (uint32_t)a.chunks;
            chunk = (int)((uint32_t)item - r * (uint32_t)a.chunks);
            b = (int)(r / each), i = (int)(r - (uint32_t)b * each), row = r;
        } else {
            row = item / a.chunks;
            chunk = (int)(item - row * a.chunks);
            b = (int)(row / each), i = (int)(row - (int64_t)b * each);
        }
        const bool draft = i > a.k;
        const int j = draft ? i - a.k - 1 : i, n = drafts_of(a, b);
        const float t = a.temperature ? a.temperature[b] : 1.0f;
        const bool greedy = is_greedy(t);
        if (chunk == 0 && i == 0 && lane == 0) a.done[b] = 0;
        if (draft ? (j >= n || greedy) : j > n) continue;
        const float c = greedy ? (float)kLog2e64 : (float)kLog2e64 / t;
        const char* at = row_of(a, b, j, draft);
        const int64_t v0 = (int64_t)chunk * kChunk;
        float m = -__builtin_inff(), s = 0.0f;
        auto add = [&](const float (&x)[NV][8]) {
            float top = m;
#pragma unroll
            for (int u = 0; u < NV; ++u)
#pragma unroll
                for (int e = 0; e < 8; ++e) top = fmaxf(top, x[u][e]);  // (leaves NaN out: the sum has it)
            const float base = top > -__builtin_inff() ? top : 0.0f;
            if constexpr (STEPS > 1) s *= __builtin_amdgcn_exp2f((m - base) * c);
            m = top;
#pragma unroll
            for (int u = 0; u < NV; ++u) {
                float y[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = __builtin_amdgcn_exp2f((x[u][e] - base) * c);
                s += ((y[0] + y[1]) + (y[2] + y[3])) + ((y[4] + y[5]) + (y[6] + y[7]));
            }
        };
        if (STEPS > 1 && v0 + kChunk <= a.V) {
            Raw8<F32> raw[2][NV];
            auto fetch = [&](int step, Raw8<F32> (&to)[NV]) {
#pragma unroll
                for (int u = 0; u < NV; ++u) to[u].template load<true>(at, v0 + step * kStep + u * 512 + lane * 8);
            };
            fetch(0, raw[0]);
#pragma unroll
            for (int step = 0; step < STEPS; ++step) {
                if (step + 1 < STEPS) fetch(step + 1, raw[(step + 1) & 1]);
                __builtin_amdgcn_sched_barrier(0);
                float x[NV][8];
#pragma unroll
                for (int u = 0; u < NV; ++u) raw[step & 1][u].unpack(x[u]);
                add(x);
            }
        } else {
            for (int64_t v = v0; v < v0 + kChunk && v < a.V; v += kStep) {
                float x[NV][8];
                logits8<F32, NV, true>(at, a.V, v + lane * 8, 512, v + kStep <= a.V, x);
                add(x);
            }
        }
        const float M = wave_reduce(m, [](float p, float q) { return fmaxf(p, q); });
        s *= __builtin_amdgcn_exp2f(M > -__builtin_inff() ? (m - M) * c : 0.0f);
        s = wave_sum_f32(s);
        if (lane == 0) a.stats[row * a.chunks + chunk] = make_float2(M, s);
    }
}

namespace {

// The sum of a whole row in 64 bits, by all threads.
template <bool F32, int THREADS>
__device__ double row_sum(const DraftArgs& a, const char* row, float m, double c, double (&lds)[THREADS / 64]) {
    double s = 0.0;
    for (int64_t v = threadIdx.x * 8; v < a.V; v += THREADS * 8) {
        float x[1][8];
        logits8<F32, 1, false>(row, a.V, v, 0, false, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) s += exp2_64(((double)x[0][e] - m) * c);
    }
    return all_threads<THREADS>(s, lds, [](double p, double q) { return p + q; });
}

// How many drafts of sequence b are taken, by a workgroup; writes: whether it writes the results down.
template <bool F32, int THREADS>
__device__ __forceinline__ DraftRow accept(const DraftArgs& a, int b, const Heat& heat, bool writes) {
    __shared__ float max_of[2][kPositions + 1];
    __shared__ double sum_of[2][kPositions + 1], lds[THREADS / 64];
    __shared__ uint64_t flags[2];  // the positions that are not taken, and those that are too close
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6, n = drafts_of(a, b);
    int taken = n;
    DraftRow row{};
    // positions j0 .. j0 + here - 1, and row n too with the last of them
    for (int j0 = 0; j0 <= n; j0 += kPositions) {
        const int here = n - j0 < kPositions ? n - j0 : kPositions, rows = n - j0 < kPositions ? here + 1 : here;
        // the drafts' own logits are on their way while the rows' sums are put together
        const int j = j0 + lane;
        int t = -1;
        float u = 0.0f, xp = 0.0f, xq = 0.0f;
        if (wid == 0 && lane < here) {
            t = a.tokens[(int64_t)b * a.k + j];
            u = a.u_accept[(int64_t)b * a.k + j];
            if (t >= 0 && t < a.V) {
                xp = logit(row_of(a, b, j, false), a.dtype, t);
                if (!heat.greedy) xq = logit(row_of(a, b, j, true), a.dtype, t);
            }
        }
        __syncthreads();
        for (int i = tid >> 4; i < rows + here; i += THREADS / 16) {
            const bool draft = i >= rows;
            const int at = draft ? i - rows : i;
            Stat s{0.0f, 0.0};
            if (!(draft && heat.greedy)) s = join_chunks(a, stat_row(a, b, j0 + at, draft), heat.c);
            if ((tid & 15) == 0) max_of[draft][at] = s.m, sum_of[draft][at] = s.s;
        }
        __syncthreads();
        double pn = 0.0, qn = 0.0;  // numerators of p and q
        if (wid == 0) {
            bool no = false, close = false;
            if (lane < here) {
                const bool there = t >= 0 && t < a.V;
                const double sp = sum_of[0][lane], sq = sum_of[1][lane];
                float p = 0.0f, q = 0.0f;
                if (there && sp > 0.0) {
                    pn = heat.greedy ? (xp == max_of[0][lane] ? 1.0 : 0.0) : exp2_64(((double)xp - max_of[0][lane]) * heat.c);
                    p = (float)(heat.greedy ? pn : pn / sp);
                }
                if (heat.greedy) {
                    q = 1.0f;
                    no = pn == 0.0;
                } else if (sp > 0.0 && sq > 0.0) {
                    if (there) {
                        qn = exp2_64(((double)xq - max_of[1][lane]) * heat.c);
                        q = (float)(qn / sq);
                    }
                    const double l = u * (qn / sq), r = pn / sp;
                    no = !(l < r);
                    close = fabs(l - r) <= kSumError * r && r > 0.0;
                } else {
                    no = true;
                }
                if (writes) {
                    a.p_target[(int64_t)b * a.k + j] = p;
                    a.p_draft[(int64_t)b * a.k + j] = q;
                }
            }
            const uint64_t n0 = __ballot(no), n1 = __ballot(close);
            if (lane == 0) flags[0] = n0, flags[1] = n1;
        }
        __syncthreads();
        const bool open = taken == n;
        if (open) {
            uint64_t no = flags[0], close = flags[1];
            while (no | close) {
                const int at = __ffsll((unsigned long long)(no | close)) - 1;
                if (close >> at & 1) {
                    const double sp = row_sum<F32, THREADS>(a, row_of(a, b, j0 + at, false), max_of[0][at], heat.c, lds);
                    const double sq = row_sum<F32, THREADS>(a, row_of(a, b, j0 + at, true), max_of[1][at], heat.c, lds);
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
            if (taken - j0 < rows) {
                const int at = taken - j0;
                const bool has_q = taken < n && !heat.greedy && sum_of[1][at] > 0.0;
                row = DraftRow{taken, sum_of[0][at] > 0.0 ? 1 : 0, has_q ? 1 : 0, max_of[0][at], has_q ? max_of[1][at] : 0.0f};
            }
        }
    }
    if (writes) {
        for (int j = n + tid; j < a.k; j += THREADS) a.p_target[(int64_t)b * a.k + j] = a.p_draft[(int64_t)b * a.k + j] = 0.0f;
        if (tid == 0) {
            a.accept_len[b] = taken;
            a.rows[b] = row;
        }
    }
    return row;
}

struct Add64 {
    __device__ double operator()(double p, double q) const { return p + q; }
};

}  // namespace

// Workgroup b: how many drafts of sequence b are taken.  (Sums of chunks, probabilities, decisions, one after another: 7 us for
// 64 sequences of 20 drafts.)
template <bool F32>
__global__ __launch_bounds__(kAccept) void k_draft_accept(DraftArgs a) {
    accept<F32, kAccept>(a, blockIdx.x, heat_of(a, blockIdx.x), true);
}

namespace {

// The wave's piece: NV times 512 logits of row n of a sequence's.
struct Piece {
    int b, w;
    bool live;
};
__device__ __forceinline__ Piece piece_of(const DraftArgs& a) {
    const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int groups = (a.pieces + kThreads / 64 - 1) / (kThreads / 64), b = (int)(blockIdx.x / (unsigned)groups);
    const int w = (int)(blockIdx.x - (unsigned)b * groups) * (kThreads / 64) + wid;
    return {b, w, w < a.pieces};
}

}  // namespace

// The sums over a piece of row n of both models in 64 bits.  The vector unit's 64-bit operations bound it, about 15 a logit (64
// sequences, two rows of 128,256: 17 us).
template <int NV, bool F32, bool TOGETHER>
__global__ __launch_bounds__(kThreads) void k_draft_sums(DraftArgs a) {
    const int lane = threadIdx.x & 63;
    const Piece p = piece_of(a);
    const Heat heat = heat_of(a, p.b);
    DraftRow row;
    if constexpr (TOGETHER) row = accept<F32, kThreads>(a, p.b, heat, p.w < kThreads / 64);
    if (!p.live) return;
    if constexpr (!TOGETHER) row = a.rows[p.b];
    if (heat.greedy || !row.has_p) return;
    const int64_t v0 = (int64_t)p.w * (NV * 512);
    const bool inside = v0 + NV * 512 <= a.V;
    float x[NV][8], y[NV][8];
    logits8<F32, NV, false>(row_of(a, p.b, row.n, false), a.V, v0 + lane * 8, 512, inside, x);
    if (row.has_q) logits8<F32, NV, false>(row_of(a, p.b, row.n, true), a.V, v0 + lane * 8, 512, inside, y);
    double sp = 0.0, sq = 0.0;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) sp += exp2_many(((double)x[i][e] - row.mt) * heat.c);
    if (row.has_q) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) sq += exp2_many(((double)y[i][e] - row.md) * heat.c);
    }
    sp = wave_reduce(sp, Add64{});
    sq = wave_reduce(sq, Add64{});
    if (lane == 0) a.sums[(int64_t)p.b * a.pieces + p.w] = make_double2(sp, sq);
}

namespace {

// The sums of a sequence's pieces, by all lanes of a wave: their reciprocals.
struct Scales {
    double p, q;
};
__device__ __forceinline__ Scales scales_of(const DraftArgs& a, int b, bool has_q, int lane) {
    double sp = 0.0, sq = 0.0;
    for (int i = lane; i < a.pieces; i += 64) {
        const double2 s = a.sums[(int64_t)b * a.pieces + i];
        sp += s.x, sq += s.y;
    }
    sp = wave_reduce(sp, Add64{});
    sq = wave_reduce(sq, Add64{});
    return {1.0 / sp, has_q ? 1.0 / sq : 0.0};
}
// r of a token.  Pieces with a sum above 0 are searched for a token with r above 0: it has to come out the same in every kernel,
// so which product is rounded is written down (a compiler may join either to the difference).
__device__ __forceinline__ double rest_of(float x, float y, const DraftRow& row, const Scales& f, double c, bool with_q) {
    const double p = exp2_many(((double)x - row.mt) * c);
    if (!with_q) return p * f.p;
    return fmax(0.0, __builtin_fma(p, f.p, -(exp2_many(((double)y - row.md) * c) * f.q)));
}

}  // namespace

namespace {

// The token of sequence b, by a workgroup.  WIDE: r's sums were written in this launch, and are read device-wide.
template <int NV, bool F32, bool WIDE>
__device__ __forceinline__ void pick(const DraftArgs& a, int b, const Heat& heat, const DraftRow& row, const Scales& f) {
    __shared__ double lds[kThreads / 64], lead[2];
    __shared__ int found[kThreads / 64][2], chosen;
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
    auto rest = [&](int i) {
        const double* at = a.rest + (int64_t)b * a.pieces + i;
        if (!WIDE) return *at;
        return __longlong_as_double((long long)__hip_atomic_load((const uint64_t*)at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
    };
    const double2* sums = a.sums + (int64_t)b * a.pieces;
    if (heat.greedy) {
        double least = INT32_MAX;
        for (int i = tid; i < a.pieces; i += kThreads) least = fmin(least, rest(i));
        least = all_threads<kThreads>(least, lds, [](double p, double q) { return fmin(p, q); });
        if (tid == 0) a.next_token[b] = (int)least;
        return;
    }
    // Finds the thread whose share `own` (in the order of threads) takes the running sum past `goal` (the last one with a
    // share if none does), or past goal times all of it: who it is, the sum before it, the goal (in lead[1]).
    auto find = [&](double own, double goal, bool whole, double& before, double& total) {
        double upto = own;
#pragma unroll
        for (int o = 1; o < 64; o *= 2) {
            const double y = __shfl_up(upto, o, 64);
            if (lane >= o) upto += y;
        }
        __syncthreads();
        if (lane == 63) lds[wid] = upto;
        __syncthreads();
        double ahead = 0.0;
        total = 0.0;
#pragma unroll
        for (int i = 0; i < kThreads / 64; ++i) {
            ahead += i < wid ? lds[i] : 0.0;
            total += lds[i];
        }
        upto += ahead;
        if (whole) goal *= total;
        const uint64_t past = __ballot(upto > goal && own > 0.0), some = __ballot(own > 0.0);
        if (lane == 0) {
            found[wid][0] = past ? wid * 64 + __ffsll((unsigned long long)past) - 1 : -1;
            found[wid][1] = some ? wid * 64 + 63 - __clzll((long long)some) : -1;
        }
        __syncthreads();
        int who = -1;
#pragma unroll
        for (int i = kThreads / 64 - 1; i >= 0; --i) who = found[i][0] >= 0 ? found[i][0] : who;
        if (who < 0) {
#pragma unroll
            for (int i = 0; i < kThreads / 64; ++i) who = found[i][1] >= 0 ? found[i][1] : who;
            goal = __builtin_inf();  // (its last one)
        }
        before = upto - own;
        if (tid == who) lead[1] = goal;
        return who;
    };
    const int each = (a.pieces + kThreads - 1) / kThreads, first = tid * each;
    const int end = first + each < a.pieces ? first + each : a.pieces;
    double all = 0.0;
    for (int i = first; i < end; ++i) all += rest(i);
    bool with_q = row.has_q;
    double before, total;
    int who = find(all, (double)a.u_next[b], true, before, total);
    if (with_q && !(total > 0x1p-30)) {  // p and q are the same: the token is drawn from p
        with_q = false;
        all = 0.0;
        for (int i = first; i < end; ++i) all += sums[i].x;
        __syncthreads();
        who = find(all, (double)a.u_next[b], true, before, total);
    }
    const bool shares = row.has_q && !with_q;  // sums are S_p's, not r's: weights are numerators
    const Scales scales = shares ? Scales{1.0, 0.0} : f;
    if (who < 0) {
        if (tid == 0) a.next_token[b] = -1;
        return;
    }
    if (tid == who) {  // the piece among its own, of which one has a sum above 0
        int piece = first;
        for (int i = first; i < end; ++i) {
            const double p = shares ? sums[i].x : rest(i);
            if (p > 0.0) {
                piece = i;
                lead[0] = before;
                if (before + p > lead[1]) break;
            }
            before += p;
        }
        chosen = piece;
        lead[1] -= lead[0];
    }
    __syncthreads();
    const double goal = lead[1];
    const int64_t v0 = (int64_t)chosen * (NV * 512), v = v0 + tid * 8;
    const bool mine = tid < NV * 64;
    float x[1][8], y[1][8];
    double r[8], own = 0.0;
    if (mine) {
        logits8<F32, 1, false>(row_of(a, b, row.n, false), a.V, v, 0, false, x);
        if (with_q) logits8<F32, 1, false>(row_of(a, b, row.n, true), a.V, v, 0, false, y);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            r[e] = rest_of(x[0][e], y[0][e], row, scales, heat.c, with_q);
            own += r[e];
        }
    }
    who = find(own, goal, false, before, total);
    if (tid == who) {
        int64_t token = -1;
        bool past = false;
        const double to = lead[1];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (!past && r[e] > 0.0) {
                token = v + e;
                past = before + r[e] > to;
            }
            before += r[e];
        }
        a.next_token[b] = (int)token;
    }
    if (who < 0 && tid == 0) a.next_token[b] = -1;
}

}  // namespace

// The sum of r over a piece; of a greedy sequence the first of the largest in it.  Bound as k_draft_sums is (18 us).
template <int NV, bool F32, bool TOGETHER>
__global__ __launch_bounds__(kThreads) void k_draft_rest(DraftArgs a) {
    const int lane = threadIdx.x & 63;
    const Piece p = piece_of(a);
    const Heat heat = heat_of(a, p.b);
    const DraftRow row = a.rows[p.b];
    if (!row.has_p) {
        if (TOGETHER && p.w == 0 && lane == 0) a.next_token[p.b] = -1;
        return;
    }
    Scales f{};
    if (p.live) {
        const int64_t v0 = (int64_t)p.w * (NV * 512);
        const bool inside = v0 + NV * 512 <= a.V;
        float x[NV][8], y[NV][8];
        logits8<F32, NV, false>(row_of(a, p.b, row.n, false), a.V, v0 + lane * 8, 512, inside, x);
        if (row.has_q) logits8<F32, NV, false>(row_of(a, p.b, row.n, true), a.V, v0 + lane * 8, 512, inside, y);
        double s;
        if (heat.greedy) {
            s = INT32_MAX;
#pragma unroll
            for (int i = NV - 1; i >= 0; --i)
#pragma unroll
                for (int e = 7; e >= 0; --e) s = x[i][e] == row.mt ? (double)(v0 + i * 512 + lane * 8 + e) : s;
            s = wave_reduce(s, [](double p, double q) { return fmin(p, q); });
        } else {
            f = scales_of(a, p.b, row.has_q, lane);
            s = 0.0;
            if (row.has_q) {
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int e = 0; e < 8; ++e) s += rest_of(x[i][e], y[i][e], row, f, heat.c, true);
            } else {
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int e = 0; e < 8; ++e) s += rest_of(x[i][e], 0.0f, row, f, heat.c, false);
            }
            s = wave_reduce(s, Add64{});
        }
        double* to = a.rest + (int64_t)p.b * a.pieces + p.w;
        if (lane == 0) {
            if (TOGETHER)
                __hip_atomic_store((uint64_t*)to, (uint64_t)__double_as_longlong(s), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            else *to = s;
        }
    }
    if constexpr (TOGETHER) {
        if (!p.live && !heat.greedy) f = scales_of(a, p.b, row.has_q, lane);
        __shared__ int last;
        last_workgroup_wait();
        __syncthreads();
        if (threadIdx.x == 0)
            last = __hip_atomic_fetch_add(a.done + p.b, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ==
                   (uint32_t)((a.pieces + kThreads / 64 - 1) / (kThreads / 64)) - 1;
        __syncthreads();
        if (last) pick<NV, F32, true>(a, p.b, heat, row, f);
    }
}

// Workgroup b: the token of sequence b (7 us, a chain of one wave's sums and one piece's logits).
template <int NV, bool F32>
__global__ __launch_bounds__(kThreads) void k_draft_pick(DraftArgs a) {
    const int b = blockIdx.x;
    const DraftRow row = a.rows[b];
    if (!row.has_p) {
        if (threadIdx.x == 0) a.next_token[b] = -1;
        return;
    }
    const Heat heat = heat_of(a, b);
    Scales f{};
    if (!heat.greedy) f = scales_of(a, b, row.has_q, threadIdx.x & 63);
    pick<NV, F32, false>(a, b, heat, row, f);
}

namespace {

// Logits of a chunk of k_draft_stats: the longest that leave eight waves on each SIMD, or two.
int chunk_of(int V, int64_t rows) {
    return rows * ((V + INT64_C(8191)) / 8192) >= 8192 ? 8192 : rows * ((V + INT64_C(2047)) / 2048) >= 2048 ? 2048 : 512;
}
// Logits of a piece of the row behind the drafts.
int piece_of(int V, int64_t B) { return B * ((V + INT64_C(8191)) / 8192) >= 1024 ? 1024 : 512; }

void shape(DraftArgs& a, char* space, int64_t* bytes) {
    const int64_t rows = (int64_t)a.B * (2 * a.k + 1);
    const int chunk = chunk_of(a.V, rows), piece = piece_of(a.V, a.B);
    a.chunks = (int)(((int64_t)a.V + chunk - 1) / chunk);
    a.pieces = (int)(((int64_t)a.V + piece - 1) / piece);
    int64_t at = 0;
    auto take = [&](int64_t n) {
        char* p = space + at;
        at += (n + 15) & ~int64_t(15);
        return p;
    };
    a.sums = (double2*)take(16 * (int64_t)a.B * a.pieces);
    a.rest = (double*)take(8 * (int64_t)a.B * a.pieces);
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
    const dim3 grid((unsigned)grid_blocks((rows * a.chunks + 3) / 4)), block(kThreads), pieces((unsigned)((int64_t)((a.pieces + 3) / 4) * a.B));
    auto go = [&](auto f32) {
        constexpr bool F32 = decltype(f32)::value;
        const int chunk = chunk_of(a.V, rows);
        if (chunk == 8192) k_draft_stats<4, 4, F32><<<grid, block, 0, s>>>(a);
        else if (chunk == 2048) k_draft_stats<4, 1, F32><<<grid, block, 0, s>>>(a);
        else k_draft_stats<1, 1, F32><<<grid, block, 0, s>>>(a);
        if (piece_of(a.V, a.B) == 1024) {
            k_draft_accept<F32><<<dim3((unsigned)a.B), dim3(kAccept), 0, s>>>(a);
            k_draft_sums<2, F32, false><<<pieces, block, 0, s>>>(a);
            k_draft_rest<2, F32, false><<<pieces, block, 0, s>>>(a);
            k_draft_pick<2, F32><<<dim3((unsigned)a.B), block, 0, s>>>(a);
        } else if ((int64_t)pieces.x > 1024) {
            k_draft_accept<F32><<<dim3((unsigned)a.B), dim3(kAccept), 0, s>>>(a);
            k_draft_sums<1, F32, false><<<pieces, block, 0, s>>>(a);
            k_draft_rest<1, F32, false><<<pieces, block, 0, s>>>(a);
            k_draft_pick<1, F32><<<dim3((unsigned)a.B), block, 0, s>>>(a);
        } else {
            k_draft_sums<1, F32, true><<<pieces, block, 0, s>>>(a);
            k_draft_rest<1, F32, true><<<pieces, block, 0, s>>>(a);
        }
    };
    if (a.dtype == 0) go(std::true_type{});
    else go(std::false_type{});
    return hipGetLastError();
}

}  // namespace lacache
