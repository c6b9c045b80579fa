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

// f(x[8]) for eight columns of a token's keys: lane's 16 bytes are one token's in bfloat16, tokens r and 16 + r's in 8 bits.
__device__ __forceinline__ void codes8(uint32_t lo, uint32_t hi, int type, float (&x)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int byte = (int)((e < 4 ? lo : hi) >> (8 * (e & 3)));
        x[e] = type == kKvInt8 ? (float)(int8_t)byte : __builtin_amdgcn_cvt_f32_fp8(byte & 0xFF, 0);
    }
}

}  // namespace

// Bounds of the pages that the newest tokens lie in: a workgroup a (sequence, page, head), a wave 32 columns at a time.  A lane
// has eight columns of every 16th token; products of codes and scales and the quotients are in 64 bits, where they are exact.
// T: what holds a key's value exactly.
template <int CT, class T>
__global__ __launch_bounds__(256) void k_kv_bound(KvPool pool, KvBounds bounds, KvSeqs seqs, int per) {
    __shared__ T top_of[4];
    __shared__ int odd_of[4];
    constexpr bool BYTES = CT != kKvBf16;
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6, r = lane & 15, u = lane >> 4;
    const int h = blockIdx.y, page = 1 << pool.page_shift, blocks = pool.dp / 32;
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
            int odd = 0;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int x = wid + 4 * i;
#pragma unroll
                for (int e = 0; e < 8; ++e) hi[i][e] = -__builtin_inf(), lo[i][e] = __builtin_inf();
                if (x >= blocks || 32 * x + 8 * u >= pool.d) continue;
                for (int t0 = 0; t0 < held; t0 += 32) {
                    const int64_t tile = tile_base(pool, pg, h, t0);
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int t = t0 + 16 * k + r;
                        if (t >= held) continue;
                        float v[8];
                        T y[8];
                        if constexpr (BYTES) {
                            const u32x2 w = *(const u32x2*)(pool.k + tile + ((x * 4 + u) * 16 + r) * 16 + 8 * k);
                            const T scale = pool.k_scale[scale_at(pool, pg, h, t)];
                            codes8(w[0], w[1], CT, v);
#pragma unroll
                            for (int e = 0; e < 8; ++e) y[e] = (T)v[e] * scale;
                        } else {
                            const u32x4 w = *(const u32x4*)(pool.k + (tile + (((x * 2 + k) * 4 + u) * 16 + r) * 8) * 2);
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                y[2 * e] = __uint_as_float(w[e] << 16);
                                y[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
                            }
                        }
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            odd |= !(y[e] < (T)__builtin_inf() && y[e] > -(T)__builtin_inf());
                            hi[i][e] = y[e] > hi[i][e] ? y[e] : hi[i][e];
                            lo[i][e] = y[e] < lo[i][e] ? y[e] : lo[i][e];
                        }
                    }
                }
                auto max2 = [](T p, T q) { return p > q ? p : q; };
                auto min2 = [](T p, T q) { return p < q ? p : q; };
#pragma unroll
                for (int e = 0; e < 8; ++e) {  // the sixteen lanes of a column
                    hi[i][e] = xor_combine<1>(xor_combine<2>(xor_combine<4>(xor_combine<8>(hi[i][e], max2), max2), max2), max2);
                    lo[i][e] = xor_combine<1>(xor_combine<2>(xor_combine<4>(xor_combine<8>(lo[i][e], min2), min2), min2), min2);
                    top = max2(top, max2(hi[i][e], -lo[i][e]));
                }
            }
            auto max2 = [](T p, T q) { return p > q ? p : q; };
            top = wave_reduce(top, max2);
            odd = __any(odd) ? 1 : 0;
            __syncthreads();
            if (lane == 0) top_of[wid] = top, odd_of[wid] = odd;
            __syncthreads();
            top = max2(max2(top_of[0], top_of[1]), max2(top_of[2], top_of[3]));
            odd = odd_of[0] | odd_of[1] | odd_of[2] | odd_of[3];
            const int64_t at = pg * pool.heads + h;
            const bool some = !odd && top >= (T)kKvTiny;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int x = wid + 4 * i;
                if (x >= blocks || r != 0) continue;
                uint32_t c[2][2] = {};
                if (some && 32 * x + 8 * u < pool.d) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int p = (int)ceil((double)hi[i][e] * 127.0 / (double)top),
                                  q = (int)floor((double)lo[i][e] * 127.0 / (double)top);
                        c[0][e >> 2] |= ((uint32_t)p & 0xFFu) << (8 * (e & 3));
                        c[1][e >> 2] |= ((uint32_t)q & 0xFFu) << (8 * (e & 3));
                    }
                }
                char* to = (char*)bounds.code + at * 2 * pool.dp + 32 * x + 8 * u;
                *(u32x2*)to = u32x2{c[0][0], c[0][1]};
                *(u32x2*)(to + pool.dp) = u32x2{c[1][0], c[1][1]};
            }
            if (tid == 0) bounds.scale[at] = odd ? __builtin_nanf("") : some ? (float)((double)top / 127.0) : 0.0f;
        }
    }
}

// The bounds of given pages as the values that they stand for.
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

// Scores of pages: a workgroup 64 pages of a (sequence, head) and the queries of up to sixteen columns (tokens times query
// heads, `fold` of them a token: a power of two, the last query head in the place of those that there are not).
//   dot^T = bounds (16 pages x 2 D) . signs (2 D x 16 columns), signs = (q+, q-) in 8 bits
// KS: steps of 64 of the 2 D.
template <int KS, bool F32>
__global__ __launch_bounds__(256) void k_kv_score(SelectArgs a) {
    __shared__ __attribute__((aligned(16))) uint32_t signs[KS * 64 * 4];
    __shared__ float unit_of[16];
    const KvPool& pool = a.pool;
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6, n = lane & 15, u = lane >> 4;
    const int h = blockIdx.y, b = blockIdx.x / a.slots, dp = 32 * KS;
    const KvSpan s = span_of(a.seqs, b);
    const int64_t len = s.pos0 + s.n;
    if (s.n == 0 || len <= 0) return;
    const int64_t known = (int64_t)a.seqs.max_pages << pool.page_shift, cap = len < known ? len : known;
    const int blocks = (int)((cap + (1 << pool.page_shift) - 1) >> pool.page_shift), tokens = 16 / a.fold;
    if ((int64_t)blockIdx.z * 64 >= blocks) return;
    for (int j0 = (blockIdx.x - b * a.slots) * tokens; j0 < s.n; j0 += a.slots * tokens) {
        f32x4 best{};  // of this wave's pages, a lane four of column n
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
            // this wave's sixteen pages
            const int j = blockIdx.z * 64 + 16 * wid + n;
            int64_t pg = -1;
            if (j < blocks) {
                pg = (a.seqs.pages + (int64_t)b * a.seqs.max_pages)[j];
                if (pg >= pool.n_pages) pg = -1;
            }
            const int64_t at = (pg < 0 ? 0 : pg) * pool.heads + h;
            const int size = pg < 0 ? 0 : 2 * dp;
            i32x4 dot{0, 0, 0, 0};
            u32x4 k[KS];
#pragma unroll
            for (int t = 0; t < KS; ++t) k[t] = size ? *(const u32x4*)(a.bounds.code + at * 2 * dp + 64 * t + 16 * u) : u32x4{};
            const float scale = size ? a.bounds.scale[at] : 0.0f;
#pragma unroll
            for (int t = 0; t < KS; ++t)
                dot = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, k[t]),
                                                            *(const i32x4*)&signs[(t * 64 + lane) * 4], dot, 0, 0, 0);
            const float unit = unit_of[n];
            f32x4 x;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float f = __shfl(scale, 4 * u + i, 64);
                const int there = __shfl(size, 4 * u + i, 64);
                x[i] = there ? ((float)dot[i] * f) * unit : -__builtin_inff();
                if (there && x[i] < -0x1.fffffep127f) x[i] = -0x1.fffffep127f;  // -infinity is a page that is not there
            }
            // over the query heads of a token
            auto over = [](float p, float q) { return max_nan(p, q); };
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (a.fold > 1) x[i] = xor_combine<1>(x[i], over);
                if (a.fold > 2) x[i] = xor_combine<2>(x[i], over);
                if (a.fold > 4) x[i] = xor_combine<4>(x[i], over);
                if (a.fold > 8) x[i] = xor_combine<8>(x[i], over);
                best[i] = pass ? max_nan(best[i], x[i]) : x[i];
            }
        }
        const int token = j0 + n / a.fold, first = blockIdx.z * 64 + 16 * wid + 4 * u;
        if (n % a.fold == 0 && token < s.n && first < blocks)
            *(f32x4*)(a.scores + ((s.row0 + token) * pool.heads + h) * a.stride + first) = best;
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

constexpr int kHeld = 8192;  // keys that are kept in LDS

}  // namespace

// The best pages of a (row, head), a workgroup each: the key of the n-th best by its bytes from the top down, counted in a
// histogram each, then the pages above it and the first ones equal to it in their order.
__global__ __launch_bounds__(256) void k_kv_pick(SelectArgs a) {
    __shared__ uint32_t keys[kHeld];
    __shared__ int bins[256], lds[4], chosen[2];
    const int tid = threadIdx.x, lane = tid & 63;
    for (int64_t unit = blockIdx.x; unit < a.seqs.rows * a.pool.heads; unit += gridDim.x) {
        const int64_t row = unit / a.pool.heads;
        const int h = (int)(unit - row * a.pool.heads);
        const int b = sequence_of(a.seqs, row, lane);
        if (b < 0) continue;
        __syncthreads();
        int32_t* out = a.blocks + ((row * a.pool.heads) + h) * a.n_blocks;
        const KvSpan s = span_of(a.seqs, b);
        const int64_t p = s.pos0 + (row - s.row0);
        int64_t most = p < 0 ? 0 : (p >> a.pool.page_shift) + 1;
        const int64_t newest = most;
        most = most < a.seqs.max_pages ? most : a.seqs.max_pages;
        const int count = (int)most;
        const float* scores = a.scores + (row * a.pool.heads + h) * a.stride;
        auto make = [&](int i) -> uint32_t {
            const float x = scores[i];
            if (x == -__builtin_inff()) return 0;
            if (i < a.first || i >= newest - a.last) return 0xFFFFFFFFu;
            return x != x ? 0xFFFFFFFEu : order_f32(x);
        };
        const bool held = count <= kHeld;
        if (held) {
            for (int i = tid; i < count; i += 256) keys[i] = make(i);
            __syncthreads();
        }
        auto key = [&](int i) { return held ? keys[i] : make(i); };
        // the threshold: `need` of those equal to it are taken
        uint32_t limit = 0, known = 0;
        int need = a.n_blocks;
        bool everything = count <= a.n_blocks;
        if (!everything) {
            for (int shift = 24; shift >= 0; shift -= 8) {
                __syncthreads();
                bins[tid] = 0;
                __syncthreads();
                for (int i = tid; i < count; i += 256) {
                    const uint32_t x = key(i);
                    if ((x & known) == limit) atomicAdd(&bins[(x >> shift) & 255], 1);
                }
                __syncthreads();
                // threads from the top bin down
                int all;
                const int own = bins[255 - tid], above = scan_threads(own, lds, all);
                if (above < need && above + own >= need) chosen[0] = 255 - tid, chosen[1] = above;
                __syncthreads();
                limit |= (uint32_t)chosen[0] << shift;
                known |= 255u << shift;
                need -= chosen[1];
            }
            everything = limit == 0;  // there are no more pages than that
        }
        // in order: a thread a range of pages
        const int each = (count + 255) / 256, i0 = tid * each, i1 = i0 + each < count ? i0 + each : count;
        int equal = 0, sure = 0, all;
        for (int i = i0; i < i1; ++i) {
            const uint32_t x = key(i);
            equal += !everything && x == limit;
            sure += everything ? x != 0 : x > limit;
        }
        int rank = scan_threads(equal, lds, all);
        const int left = need - rank < 0 ? 0 : need - rank, mine = equal < left ? equal : left;
        int to = scan_threads(sure + mine, lds, all);
        for (int i = i0; i < i1; ++i) {
            const uint32_t x = key(i);
            const bool take = everything ? x != 0 : x > limit || (x == limit && rank < need);
            rank += !everything && x == limit;
            if (take) out[to++] = i;
        }
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
    const int64_t tiles = (a.seqs.max_pages + 63) / 64;
    while (a.slots > 1 && (int64_t)a.slots * a.seqs.n_seq > (1 << 20)) a.slots = (a.slots + 1) / 2;
    const dim3 grid((unsigned)(a.slots * (int64_t)a.seqs.n_seq), (unsigned)a.pool.heads, (unsigned)tiles);
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
    k_kv_pick<<<dim3((unsigned)grid_blocks(a.seqs.rows * a.pool.heads)), dim3(256), 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace lacache
