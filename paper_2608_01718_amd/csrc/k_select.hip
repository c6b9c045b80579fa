// k_select.hip -- the pages that a row's attention is likely to need: bounds of each page's keys, scores of all pages from
// them, and the best of a row's pages.
//
// A page's keys lie between lo and hi, column by column, so no score q . k of a page exceeds q+ . hi + q- . lo (q+ and q- the
// positive and the negative columns of q).  Bounds and queries are held in 8 bits, so that a score is a matrix product of
// whole numbers, the same in any order, times two scales.
#include "attend.hpp"
#include "launch.hpp"

namespace lacache {

namespace {

// The values of eight codes.
__device__ __forceinline__ void codes8(uint32_t lo, uint32_t hi, int type, float (&x)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int byte = (int)((e < 4 ? lo : hi) >> (8 * (e & 3)));
        x[e] = type == kKvInt8 ? (float)(int8_t)byte : __builtin_amdgcn_cvt_f32_fp8(byte & 0xFF, 0);
    }
}

}  // namespace

// Bounds of the pages that the newest tokens lie in: a workgroup a (sequence, page, head), a wave 32 columns at a time, a lane
// eight columns of every 16th token.  Products of codes and scales and the quotients are in 64 bits, where they are exact; the
// sixteen lanes of eight columns take a quotient each.  T: what holds a key's value exactly.  The chain of positions, table, tokens
// and quotients bounds it (64 sequences' one token, 8 heads of 128 columns, pages of 64 in bfloat16: 6 us; 8 prompts of 1024 to
// 2048 tokens in fp8, products in 64 bits: 10 us).
template <int CT, class T>
__global__ __launch_bounds__(256) void k_kv_bound(KvPool pool, KvBounds bounds, KvSeqs seqs, int per) {
    __shared__ T top_of[4];
    __shared__ int odd_of[4];
    constexpr bool BYTES = CT != kKvBf16;
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6, r = lane & 15, u = lane >> 4;
    const int h = blockIdx.y, page = 1 << pool.page_shift, blocks = pool.dp / 32;
    auto max2 = [](T p, T q) { return p > q ? p : q; };
    auto largest = [](T p, T q) {
        if constexpr (BYTES) return __builtin_fmax(p, q);
        else return __builtin_fmaxf(p, q);
    };
    auto least = [](T p, T q) {
        if constexpr (BYTES) return __builtin_fmin(p, q);
        else return __builtin_fminf(p, q);
    };
    for (int64_t unit = blockIdx.x; unit < (int64_t)seqs.n_seq * per; unit += gridDim.x) {
        const int b = (int)(unit / per);
        const KvSpan s = span_of(seqs, b);
        const int64_t len = s.pos0 + s.n, from = s.pos0 < 0 ? 0 : s.pos0;
        if (s.n == 0 || len <= 0) continue;
        const int64_t last = (len - 1) >> pool.page_shift;
        for (int64_t j = (from >> pool.page_shift) + (unit - (int64_t)b * per); j <= last; j += per) {
            const int64_t pg = page_of(pool, seqs, b, j << pool.page_shift);
            if (pg < 0) continue;
            const int held = len - (j << pool.page_shift) < page ? (int)(len - (j << pool.page_shift)) : page;  // its tokens
            T hi[2][8], lo[2][8];  // of column blocks wid and wid + 4
            T top = 0;
            uint32_t odd = 0;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int x = wid + 4 * i;
#pragma unroll
                for (int e = 0; e < 8; ++e) hi[i][e] = -__builtin_inf(), lo[i][e] = __builtin_inf();
                if (x >= blocks || 32 * x + 8 * u >= pool.d) continue;
                for (int t0 = 0; t0 < held; t0 += 64) {  // (two tiles' loads together)
                    u32x4 w[4];
                    float scale[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int t = t0 + 16 * k + r;
                        const bool in = t < held;
                        const int64_t tile = tile_base(pool, pg, h, in ? t0 + 16 * k : 0);
                        if constexpr (BYTES) {
                            const u32x2 p = *(const u32x2*)(pool.k + tile + ((x * 4 + u) * 16 + r) * 16 + (in ? 8 * (k & 1) : 0));
                            w[k] = u32x4{p[0], p[1], 0, 0};
                            scale[k] = pool.k_scale[scale_at(pool, pg, h, in ? t : 0)];
                        } else {
                            w[k] = *(const u32x4*)(pool.k + (tile + (((x * 2 + (in ? k & 1 : 0)) * 4 + u) * 16 + r) * 8) * 2);
                        }
                    }
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        if (t0 + 16 * k + r >= held) continue;
                        T y[8];
                        if constexpr (BYTES) {
                            float v[8];
                            codes8(w[k][0], w[k][1], CT, v);
#pragma unroll
                            for (int e = 0; e < 8; ++e) y[e] = (T)v[e] * (T)scale[k];
                            odd |= (__float_as_uint(scale[k]) & 0x7F800000u) == 0x7F800000u;
                            if constexpr (CT == kKvFp8)
                                odd |= (((w[k][0] & 0x7F7F7F7Fu) + 0x01010101u) | ((w[k][1] & 0x7F7F7F7Fu) + 0x01010101u)) & 0x80808080u;
                        } else {
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                y[2 * e] = __uint_as_float(w[k][e] << 16);
                                y[2 * e + 1] = __uint_as_float(w[k][e] & 0xFFFF0000u);
                                odd |= ((w[k][e] & 0x7F807F80u) + 0x00800080u) & 0x80008000u;
                            }
                        }
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            hi[i][e] = largest(hi[i][e], y[e]);
                            lo[i][e] = least(lo[i][e], y[e]);
                        }
                    }
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {  // the sixteen lanes of a column
                    hi[i][e] = xor_combine<1>(xor_combine<2>(xor_combine<4>(xor_combine<8>(hi[i][e], largest), largest), largest), largest);
                    lo[i][e] = xor_combine<1>(xor_combine<2>(xor_combine<4>(xor_combine<8>(lo[i][e], least), least), least), least);
                    top = max2(top, max2(hi[i][e], -lo[i][e]));
                }
            }
            top = wave_reduce(top, max2);
            const int some_odd = __any(odd != 0) ? 1 : 0;
            __syncthreads();
            if (lane == 0) top_of[wid] = top, odd_of[wid] = some_odd;
            __syncthreads();
            top = max2(max2(top_of[0], top_of[1]), max2(top_of[2], top_of[3]));
            const bool none = (odd_of[0] | odd_of[1] | odd_of[2] | odd_of[3]) != 0;
            const int64_t at = pg * pool.heads + h;
            const bool some = !none && top >= (T)kKvTiny;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int x = wid + 4 * i;
                if (x >= blocks) continue;
                // lane r: column r % 8 of the largest (r < 8) or the least
                T mine = hi[i][0];
#pragma unroll
                for (int e = 0; e < 8; ++e) mine = (r & 7) != e ? mine : r < 8 ? hi[i][e] : lo[i][e];
                int code = 0;
                if (some && 32 * x + 8 * u < pool.d) {
                    const double q = (double)mine * 127.0 / (double)top;
                    code = (int)(r < 8 ? ceil(q) : floor(q));
                }
                ((char*)bounds.code)[at * 2 * pool.dp + (r < 8 ? 0 : pool.dp) + 32 * x + 8 * u + (r & 7)] = (char)code;
            }
            if (tid == 0) bounds.scale[at] = none ? __builtin_nanf("") : some ? (float)((double)top / 127.0) : 0.0f;
        }
    }
}

// The bounds of given pages as the values that they stand for (3 us, a launch).
__global__ __launch_bounds__(256) void k_kv_bounds_read(KvPool pool, KvBounds bounds, const int32_t* pages, int64_t n, float* hi,
                                                        float* lo) {
    const int64_t all = n * pool.heads * (pool.d / 8);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int64_t at = i / (pool.d / 8), p = at / pool.heads;
        const int c = (int)(i - at * (pool.d / 8)) * 8;
        const int64_t pg = pages[p];
        float x[8] = {}, y[8] = {};
        if (pg >= 0 && pg < pool.n_pages) {
            const int64_t from = pg * pool.heads + (at - p * pool.heads);
            const float f = bounds.scale[from];
            const u32x2 a = *(const u32x2*)(bounds.code + from * 2 * pool.dp + c),
                        b = *(const u32x2*)(bounds.code + from * 2 * pool.dp + pool.dp + c);
            codes8(a[0], a[1], kKvInt8, x);
            codes8(b[0], b[1], kKvInt8, y);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] *= f, y[e] *= f;
        }
        if (hi) store_row8<true>((char*)(hi + at * pool.d), c, x);
        if (lo) store_row8<true>((char*)(lo + at * pool.d), c, y);
    }
}

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float max_nan(float a, float b) { return a != a ? a : b != b ? b : fmaxf(a, b); }

}  // namespace

namespace {

constexpr uint32_t kAlways = 0xFFFFFFFFu;  // the key of a page that is taken before others

// A page's key, in the order of scores: 0: there is no such page.
struct Keys {
    int count, first;   // pages of the row, those that are always taken
    int64_t last;       // always taken from here on
    __device__ __forceinline__ uint32_t operator()(int i, float x) const {
        if (i >= count || x == -__builtin_inff()) return 0;
        if (i < first || i >= last) return kAlways;
        return x != x ? kAlways - 1 : order_f32(x);
    }
};
// Those of the row of position p.
__device__ __forceinline__ Keys keys_of(const SelectArgs& a, int64_t p) {
    const int64_t most = p < 0 ? 0 : (p >> a.pool.page_shift) + 1;
    return {(int)(most < a.seqs.max_pages ? most : a.seqs.max_pages), a.first, most - a.last};
}

}  // namespace

// Scores of pages: a workgroup 64 pages at a time of a (sequence, head), each gridDim.z-th of them, and the queries of up to
// sixteen columns (tokens times query heads, `fold` of them a token: a power of two, the last query head in the place of those
// that there are not).
//   dot^T = bounds (16 pages x 2 D) . signs (2 D x 16 columns), signs = (q+, q-) in 8 bits
// KS: steps of 64 of the 2 D.  (Tried without gain: all pages of a row in one workgroup, which picks the best too: 26 us for
// 64 sequences of 256 to 32,768 tokens, 20 in two launches; each 64 pages more take 1.6 us of waiting one after another.)  One
// token over 2048 pages, 8 heads, d = 128: 5 us, latency; 64 sequences of 65,535 tokens 31 us, 4.4 TB/s of bounds.
template <int KS, bool F32>
__global__ __launch_bounds__(256) void k_kv_score(SelectArgs a) {
    __shared__ __attribute__((aligned(16))) uint32_t signs[KS * 64 * 4];
    __shared__ float unit_of[16];
    const KvPool& pool = a.pool;
    const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, u = lane >> 4;
    const int h = blockIdx.y, b = blockIdx.x / a.slots, dp = 32 * KS;
    const int32_t* pages = a.seqs.pages + (int64_t)b * a.seqs.max_pages;
    // the first page numbers are on their way while the rest is looked at
    const int j_first = 64 * (int)blockIdx.z + 16 * wid + n;
    const int page_first = pages[j_first < a.seqs.max_pages ? j_first : 0];
    const KvSpan s = span_of(a.seqs, b);
    const int64_t len = s.pos0 + s.n;
    const int64_t known = (int64_t)a.seqs.max_pages << pool.page_shift, cap = len < 0 ? 0 : len < known ? len : known;
    const int blocks = (int)((cap + (1 << pool.page_shift) - 1) >> pool.page_shift), tokens = 16 / a.fold;
    if ((int64_t)blockIdx.z * 64 >= blocks) return;
    struct Codes {
        u32x4 k[KS];
        float scale;
        int there;
    };
    auto page_of_tile = [&](int z) {
        const int j = 64 * z + 16 * wid + n;
        return j < blocks ? pages[j] : -1;
    };
    // (a page that is not there: another's bounds, which are not looked at)
    auto fetch = [&](Codes& c, int pg) {
        c.there = pg >= 0 && pg < pool.n_pages;
        if (pool.n_pages == 0) return;
        const int64_t at = (int64_t)(c.there ? pg : 0) * pool.heads + h;
#pragma unroll
        for (int t = 0; t < KS; ++t) c.k[t] = *(const u32x4*)(a.bounds.code + at * 2 * dp + 64 * t + 16 * u);
        c.scale = a.bounds.scale[at];
    };
    const int z0 = blockIdx.z, step = gridDim.z;
    Codes two[2];
    fetch(two[0], j_first < blocks ? page_first : -1);
    bool fresh = true;  // two[0] is of tile z0
    for (int j0 = (blockIdx.x - b * a.slots) * tokens; j0 < s.n; j0 += a.slots * tokens) {
        for (int pass = 0; pass * 16 < a.group; ++pass) {
            __syncthreads();
            // the queries in 8 bits, sixteen threads a column
            {
                const int col = tid >> 4, i = tid & 15;
                const int j = j0 + col / a.fold, g = pass * 16 + col % a.fold;
                const int64_t row = s.row0 + (j < s.n ? j : s.n - 1);
                const int head = h * a.group + (g < a.group ? g : a.group - 1);
                const char* from = a.q + (row * a.q_row + (int64_t)head * pool.d) * (F32 ? 4 : 2);
                float x[(KS + 3) / 4][8], top = 0.0f;
                int odd = 0;
#pragma unroll
                for (int k = 0; k < (KS + 3) / 4; ++k) {
                    const int c = 8 * (i + 16 * k);
                    if (c < pool.d) {
                        load_row8<F32>(from, c, x[k]);
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            top = fmaxf(top, fabsf(x[k][e]));
                            odd |= !(fabsf(x[k][e]) < __builtin_inff());
                        }
                    }
                }
                auto max2 = [](float p, float q) { return fmaxf(p, q); };
                auto or2 = [](int p, int q) { return p | q; };
                top = xor_combine<1>(xor_combine<2>(xor_combine<4>(xor_combine<8>(top, max2), max2), max2), max2);
                odd = xor_combine<1>(xor_combine<2>(xor_combine<4>(xor_combine<8>(odd, or2), or2), or2), or2);
                const float unit = odd ? __builtin_nanf("") : top * (1.0f / 127.0f);
#pragma unroll
                for (int k = 0; k < (KS + 3) / 4; ++k) {
                    const int c = 8 * (i + 16 * k);
                    if (c >= dp) continue;
                    uint32_t w[2][2] = {};
                    if (c < pool.d && unit > 0.0f) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const int v = (int)fminf(fmaxf(rintf(x[k][e] / unit), -127.0f), 127.0f);
                            w[0][e >> 2] |= ((uint32_t)(v > 0 ? v : 0) & 0xFFu) << (8 * (e & 3));
                            w[1][e >> 2] |= ((uint32_t)(v < 0 ? v : 0) & 0xFFu) << (8 * (e & 3));
                        }
                    }
#pragma unroll
                    for (int part = 0; part < 2; ++part) {
                        const int at = part * dp + c;
                        uint32_t* to = signs + ((at >> 6) * 64 + ((at >> 4) & 3) * 16 + col) * 4 + ((at >> 3) & 1) * 2;
                        to[0] = w[part][0];
                        to[1] = w[part][1];
                    }
                }
                if (i == 0) unit_of[col] = unit;
            }
            __syncthreads();
            const float unit = unit_of[n];
            const int token = j0 + n / a.fold;
            auto over = [](float p, float q) { return max_nan(p, q); };
            if (!fresh) fetch(two[0], page_of_tile(z0));
            fresh = false;
            int page_next = page_of_tile(z0 + step);
            auto tile = [&](int z, const Codes& now, Codes& next) {
                fetch(next, page_next);  // on its way under this tile's scores
                page_next = page_of_tile(z + 2 * step);
                __builtin_amdgcn_sched_barrier(0);
                i32x4 dot{0, 0, 0, 0};
#pragma unroll
                for (int t = 0; t < KS; ++t)
                    dot = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, now.k[t]),
                                                                *(const i32x4*)&signs[(t * 64 + lane) * 4], dot, 0, 0, 0);
                f32x4 x;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float f = __shfl(now.scale, 4 * u + i, 64);
                    const int is = __shfl(now.there, 4 * u + i, 64);
                    x[i] = is ? ((float)dot[i] * f) * unit : -__builtin_inff();
                    if (is && x[i] < -0x1.fffffep127f) x[i] = -0x1.fffffep127f;  // -infinity is a page that is not there
                    // over the query heads of a token
                    if (a.fold > 1) x[i] = xor_combine<1>(x[i], over);
                    if (a.fold > 2) x[i] = xor_combine<2>(x[i], over);
                    if (a.fold > 4) x[i] = xor_combine<4>(x[i], over);
                    if (a.fold > 8) x[i] = xor_combine<8>(x[i], over);
                }
                const int at = 64 * z + 16 * wid + 4 * u;
                if (n % a.fold == 0 && token < s.n && at < blocks) {
                    f32x4* to = (f32x4*)(a.scores + ((s.row0 + token) * pool.heads + h) * a.stride + at);
                    if (pass > 0) {
                        const f32x4 y = *to;
#pragma unroll
                        for (int i = 0; i < 4; ++i) x[i] = max_nan(y[i], x[i]);
                    }
                    *to = x;
                }
            };
            for (int z = z0; 64 * z < blocks; z += 2 * step) {
                tile(z, two[0], two[1]);
                if (64 * (z + step) >= blocks) break;
                tile(z + step, two[1], two[0]);
            }
        }
    }
}

namespace {

// Sum over the threads before this one, and over all.
__device__ __forceinline__ int scan_threads(int x, int (&lds)[4], int& all) {
    const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6, sum = wave_scan(x);
    __syncthreads();
    if (lane == 63) lds[wid] = sum;
    __syncthreads();
    int before = sum - x;
    all = 0;
    for (int w = 0; w < 4; ++w) {
        before += w < wid ? lds[w] : 0;
        all += lds[w];
    }
    return before;
}

constexpr int kClose = 32;  // keys of the same leading bytes that are ranked one against another

}  // namespace

// The best pages of a (row, head), a workgroup each, a thread a range of pages (of up to 16 it keeps the keys in registers,
// HELD).  The last page that is taken, in the order of (key, page), is found by bytes of (key - least key) from the top down,
// counted in a histogram each, until no more than kClose keys share them: these are ranked one against another.  Then the pages
// that come before it are written in their order.  (Keys of one row lie close together: counted from their least one the first
// byte spreads them.)  Barriers bound it, four or more a byte: 8 us for the best 64 of 2048 pages.
template <bool HELD>
__global__ __launch_bounds__(256) void k_kv_pick(SelectArgs a) {
    __shared__ uint32_t close_key[kClose], range[2][4];
    __shared__ int bins[256], lds[4], close_at[kClose], chosen[4], ends[2];
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
    for (int64_t unit = blockIdx.x; unit < a.seqs.rows * a.pool.heads; unit += gridDim.x) {
        const int64_t row = unit / a.pool.heads;
        const int h = (int)(unit - row * a.pool.heads);
        const int b = sequence_of(a.seqs, row, lane);
        if (b < 0) continue;
        __syncthreads();
        int32_t* out = a.blocks + ((row * a.pool.heads) + h) * a.n_blocks;
        const KvSpan s = span_of(a.seqs, b);
        const int64_t p = s.pos0 + (row - s.row0);
        const Keys make = keys_of(a, p);
        const int count = make.count;
        const float* scores = a.scores + (row * a.pool.heads + h) * a.stride;
        // (a row of scores ends in whole 64: fours can be loaded that begin in it)
        const int each = (count + 1023) / 1024 * 4, i0 = tid * each, i1 = i0 + each < count ? i0 + each : count;
        uint32_t held[HELD ? 16 : 1];
        if constexpr (HELD) {
            f32x4 x[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const bool in = 4 * k < each && i0 + 4 * k < count;  // (a table of no pages has no scores)
                x[k] = in ? *(const f32x4*)(scores + i0 + 4 * k) : f32x4{};
            }
#pragma unroll
            for (int k = 0; k < 16; ++k) held[k] = k < each ? make(i0 + k, x[k >> 2][k & 3]) : 0u;
        }
        // f(page, key) of the thread's pages that are there, in order
        auto own_pages = [&](auto f) {
            if constexpr (HELD) {
#pragma unroll
                for (int k = 0; k < 16; ++k)
                    if (held[k] != 0) f(i0 + k, held[k]);
            } else {
                for (int i = i0; i < i1; ++i) {
                    const uint32_t x = make(i, scores[i]);
                    if (x != 0) f(i, x);
                }
            }
        };
        // the keys' range, how many there are, and how many are taken in any case
        uint32_t least = kAlways, top = 0;
        int sure = 0, real = 0;
        own_pages([&](int, uint32_t x) {
            const bool is = x != kAlways;
            sure += !is;
            real += is;
            least = is && x < least ? x : least;
            top = is && x > top ? x : top;
        });
        least = wave_reduce(least, [](uint32_t p, uint32_t q) { return p < q ? p : q; });
        top = wave_reduce(top, [](uint32_t p, uint32_t q) { return p > q ? p : q; });
        sure = wave_reduce(sure, [](int p, int q) { return p + q; });
        real = wave_reduce(real, [](int p, int q) { return p + q; });
        if (lane == 0) range[0][wid] = least, range[1][wid] = top, lds[wid] = sure, chosen[wid] = real;
        if (tid == 0) ends[0] = 0;
        bins[tid] = 0;
        __syncthreads();
        least = min(min(range[0][0], range[0][1]), min(range[0][2], range[0][3]));
        top = max(max(range[1][0], range[1][1]), max(range[1][2], range[1][3]));
        sure = lds[0] + lds[1] + lds[2] + lds[3];
        real = chosen[0] + chosen[1] + chosen[2] + chosen[3];
        int need = a.n_blocks - sure;  // of the others
        uint32_t limit = 0;            // the last one's key
        int last = INT32_MAX;          // and its page
        if (real > need && need == 0) {
            limit = kAlways - 1, last = -1;
        } else if (real > need) {
            uint32_t from = least, left = top - least;  // keys from .. from + left hold it
            auto within = [&](uint32_t x) { return x != kAlways && x >= from && x - from <= left; };
            int close = real;
            while (close > kClose && left != 0) {
                const int bits = 32 - __builtin_clz(left), shift = bits > 8 ? bits - 8 : 0;
                own_pages([&](int, uint32_t x) {
                    if (within(x)) atomicAdd(&bins[(x - from) >> shift], 1);
                });
                __syncthreads();
                int all;
                const int own = bins[255 - tid], above = scan_threads(own, lds, all);  // from the top bin down
                bins[255 - tid] = 0;
                if (above < need && above + own >= need) chosen[0] = 255 - tid, chosen[1] = above, chosen[2] = own;
                __syncthreads();
                from += (uint32_t)chosen[0] << shift;
                left = shift ? (1u << shift) - 1 : 0;
                need -= chosen[1];
                close = chosen[2];
            }
            if (close <= kClose) {
                own_pages([&](int i, uint32_t x) {
                    if (within(x)) {
                        const int to = atomicAdd(&ends[0], 1);
                        close_key[to] = x;
                        close_at[to] = i;
                    }
                });
                __syncthreads();
                if (tid < close) {
                    const uint32_t x = close_key[tid];
                    const int i = close_at[tid];
                    int rank = 0;
                    for (int k = 0; k < close; ++k) rank += close_key[k] > x || (close_key[k] == x && close_at[k] < i);
                    if (rank == need - 1) range[0][0] = x, ends[1] = i;
                }
                __syncthreads();
                limit = range[0][0];
                last = ends[1];
            } else {  // more that are equal: the need-th of them
                int equal = 0, all;
                own_pages([&](int, uint32_t x) { equal += x == from; });
                int rank = scan_threads(equal, lds, all);
                if (rank < need && rank + equal >= need)
                    own_pages([&](int i, uint32_t x) {
                        if (x == from && ++rank == need) ends[1] = i;
                    });
                __syncthreads();
                limit = from;
                last = ends[1];
            }
        }
        auto taken = [&](int i, uint32_t x) { return x > limit || (x == limit && i <= last); };
        int mine = 0, all;
        own_pages([&](int i, uint32_t x) { mine += taken(i, x); });
        int to = scan_threads(mine, lds, all);
        own_pages([&](int i, uint32_t x) {
            if (taken(i, x)) out[to++] = i;
        });
        for (int i = all + tid; i < a.n_blocks; i += 256) out[i] = -1;
    }
}

hipError_t launch_kv_bound(const KvPool& pool, const KvBounds& bounds, const KvSeqs& seqs, int max_new, hipStream_t s) {
    // pages that a sequence's newest tokens lie in
    const int64_t new_most = max_new > 0 && max_new < seqs.rows ? max_new : max_new > 0 ? seqs.rows : seqs.rows < 1024 ? seqs.rows : 1024;
    const int64_t per = (new_most + (1 << pool.page_shift) - 2) / (1 << pool.page_shift) + 1;
    const dim3 grid((unsigned)grid_blocks(per * seqs.n_seq < kMaxGridBlocks / 16 ? per * seqs.n_seq : kMaxGridBlocks / 16), (unsigned)pool.heads);
    if (pool.type == kKvBf16) k_kv_bound<kKvBf16, float><<<grid, dim3(256), 0, s>>>(pool, bounds, seqs, (int)per);
    else if (pool.type == kKvFp8) k_kv_bound<kKvFp8, double><<<grid, dim3(256), 0, s>>>(pool, bounds, seqs, (int)per);
    else k_kv_bound<kKvInt8, double><<<grid, dim3(256), 0, s>>>(pool, bounds, seqs, (int)per);
    return hipGetLastError();
}

hipError_t launch_kv_bounds_read(const KvPool& pool, const KvBounds& bounds, const int32_t* pages, int64_t n, float* hi,
                                 float* lo, hipStream_t s) {
    const int64_t all = n * pool.heads * (pool.d / 8);
    k_kv_bounds_read<<<dim3((unsigned)grid_blocks((all + 255) / 256)), dim3(256), 0, s>>>(pool, bounds, pages, n, hi, lo);
    return hipGetLastError();
}

int64_t select_stride(int max_pages) { return ((int64_t)max_pages + 63) & ~int64_t(63); }

hipError_t launch_kv_select(SelectArgs a, int max_new, hipStream_t s) {
    a.stride = select_stride(a.seqs.max_pages);
    a.fold = 1;
    while (a.fold < a.group && a.fold < 16) a.fold *= 2;
    const int tokens = 16 / a.fold;
    const int64_t new_most = max_new > 0 && max_new < a.seqs.rows ? max_new : max_new > 0 ? a.seqs.rows : a.seqs.rows < 16 ? a.seqs.rows : 16;
    a.slots = (int)((new_most + tokens - 1) / tokens);
    while (a.slots > 1 && (int64_t)a.slots * a.seqs.n_seq > (1 << 20)) a.slots = (a.slots + 1) / 2;
    const int64_t tiles = (a.seqs.max_pages + 63) / 64, units = a.slots * (int64_t)a.seqs.n_seq * a.pool.heads;
    // as many workgroups as are at work at once, of 64 pages or more
    const int64_t most = units < 2048 ? 2048 / units : 1;
    const dim3 grid((unsigned)(a.slots * (int64_t)a.seqs.n_seq), (unsigned)a.pool.heads, (unsigned)(tiles < most ? tiles : most));
    auto go = [&](auto ks) {
        constexpr int KS = decltype(ks)::value;
        if (a.dtype == 0) k_kv_score<KS, true><<<grid, dim3(256), 0, s>>>(a);
        else k_kv_score<KS, false><<<grid, dim3(256), 0, s>>>(a);
    };
    if (tiles > 0) {
        if (a.pool.dp == 64) go(std::integral_constant<int, 2>{});
        else if (a.pool.dp == 96) go(std::integral_constant<int, 3>{});
        else if (a.pool.dp == 128) go(std::integral_constant<int, 4>{});
        else if (a.pool.dp == 192) go(std::integral_constant<int, 6>{});
        else go(std::integral_constant<int, 8>{});
    }
    const dim3 lists((unsigned)grid_blocks(a.seqs.rows * a.pool.heads));
    if (a.seqs.max_pages <= 4096) k_kv_pick<true><<<lists, dim3(256), 0, s>>>(a);
    else k_kv_pick<false><<<lists, dim3(256), 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace lacache
