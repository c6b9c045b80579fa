// k_kv_store.hip -- writing new tokens into the pages of the key-value cache, and reading them back.
//
// A token's keys of one head (turned by its position, if a table is given) or values are rounded once: to bfloat16, or
// to 8-bit codes x * (top / m) with the scale m / top, m the largest magnitude of the d columns.
//
// Both are bound by memory: a tile of 32 tokens of one head passes through LDS, where its elements change from rows to
// the tile's order, so that rows and tiles are read and written 16 bytes a lane.  A tile of which only some tokens are
// concerned is written piece by piece, and read without LDS if they are few.  8 prompts of 1024 to 2048 tokens, 32 query and 8 kv
// heads of 128 bfloat16 columns into int8: 67 us to write (4.0 TB/s with the queries), 19 to read back (4.2 TB/s of codes and
// results); one token of 64 sequences 6.6 and 3.6 us, the launch.
#include "kv.hpp"
#include "launch.hpp"

namespace lacache {

namespace {

// The tiles that new tokens of a sequence lie in: the first, how many.
struct TileSpan {
    KvSpan span;
    int64_t first;
    int count;
};
__device__ inline TileSpan tiles_of(const KvSeqs& s, int b) {
    TileSpan t;
    t.span = span_of(s, b);
    const int64_t lo = t.span.pos0 < 0 ? 0 : t.span.pos0, hi = t.span.pos0 + t.span.n;  // positions lo .. hi - 1
    t.first = lo >> 5;
    t.count = hi > lo ? (int)(((hi - 1) >> 5) - t.first) + 1 : 0;
    return t;
}

// A tile's keys and then its values in LDS: pieces of 16 bytes in the tile's order with one to spare after every 16 (keys) and 64
// (values), so that a row's lanes, whose elements lie whole kilobytes apart in the tile, go to different banks.  (For reading: 19 us
// with it and the keys eight columns at a time, 26 without.  The write gains nothing.)
inline constexpr int lds_pieces(int dp, int csz) { return 32 * dp * csz / 16 * 17 / 16; }
template <bool KEYS>
__device__ __forceinline__ int lds_piece(int i) {
    return i + (i >> (KEYS ? 4 : 6));
}
// Where an element lies: its place in the tile, in bytes, with the spare pieces before it.
template <bool KEYS, bool BYTES>
__device__ __forceinline__ int lds_at(int t, int c) {
    const int at = (KEYS ? k_place(t, c, BYTES) : v_place(t, c, BYTES)) * (BYTES ? 1 : 2);
    return at + ((at >> (KEYS ? 8 : 10)) << 4);
}

// A power of two of lanes that holds a head's columns by eights.
constexpr int row_lanes(int dp) { return dp <= 64 ? 8 : dp <= 128 ? 16 : 32; }

// Eight columns from c on of a row of keys, turned.
template <bool F32>
__device__ __forceinline__ void load_turned(const char* row, int c, const RopeArgs& rope, const float2* cs,
                                            float (&x)[8]) {
    load_row8<F32>(row, c, x);
    const int half = rope.rot / 2;
    if (!rope.table || c >= rope.rot) return;
    if (rope.pairs && c + 8 <= rope.rot) {
#pragma unroll
        for (int e = 0; e < 8; e += 2) turn(x[e], x[e + 1], cs[(c + e) / 2].x, cs[(c + e) / 2].y);
    } else if (!rope.pairs && (c + 8 <= half || (c >= half && c + 8 <= rope.rot))) {
        float other[8];
        const bool first = c < half;
        load_row8<F32>(row, first ? c + half : c - half, other);
        const float2* w = cs + (first ? c : c - half);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float a = first ? x[e] : other[e], b = first ? other[e] : x[e];
            turn(a, b, w[e].x, w[e].y);
            x[e] = first ? a : b;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int col = c + e;
            if (col >= rope.rot) break;
            const bool first = rope.pairs ? !(col & 1) : col < half;
            const int i = rope.pairs ? col >> 1 : first ? col : col - half;
            const float o = load_row1<F32>(row, rope.pairs ? col ^ 1 : first ? col + half : col - half);
            float a = first ? x[e] : o, b = first ? o : x[e];
            turn(a, b, cs[i].x, cs[i].y);
            x[e] = first ? a : b;
        }
    }
}

}  // namespace

// Workgroup x = parts b + part takes tile y (and every gridDim.y-th) of sequence b: the keys and values of head `part`,
// or, from part `heads` on, a share of the queries of 32 rows.
template <bool F32, int CT>
__global__ __launch_bounds__(256) void k_kv_append(AppendArgs a, int parts, int turn_how) {
    constexpr bool BYTES = CT != kKvBf16;
    constexpr int CSZ = BYTES ? 1 : 2, ESZ = F32 ? 4 : 2;
    __shared__ u32x4 tile[2][32 * 256 * CSZ / 16];  // keys, values, in the tile's order
    const KvPool& p = a.pool;
    const int tid = threadIdx.x, b = blockIdx.x / parts, part = blockIdx.x - b * parts;
    const TileSpan t = tiles_of(a.seqs, b);

    if (part >= p.heads) {  // queries
        const int shares = parts - p.heads, share = part - p.heads;
        const int items = turn_items(p.d, a.rope.rot, turn_how), of_row = a.q_heads * items;
        for (int r0 = 32 * blockIdx.y; r0 < t.span.n; r0 += 32 * gridDim.y) {
            const int rows = t.span.n - r0 < 32 ? t.span.n - r0 : 32;
            for (int e = share * 256 + tid; e < rows * of_row; e += shares * 256) {
                const int r = (int)((uint32_t)e / (uint32_t)of_row), in_row = e - r * of_row;
                const int h = (int)((uint32_t)in_row / (uint32_t)items), i = in_row - h * items;
                const int64_t row = t.span.row0 + r0 + r;
                const char* x = a.q + (row * a.q_row + (int64_t)h * p.d) * ESZ;
                char* y = a.q_out + (row * a.q_heads + h) * p.d * ESZ;
                const float2* cs = table_row(a.rope, t.span.pos0 + r0 + r);
                if (turn_how == kTurnHalves) turn_item<F32, kTurnHalves>(x, y, p.d, a.rope, cs, i, 1.0f);
                else if (turn_how == kTurnPairs) turn_item<F32, kTurnPairs>(x, y, p.d, a.rope, cs, i, 1.0f);
                else turn_item<F32, kTurnOne>(x, y, p.d, a.rope, cs, i, 1.0f);
            }
        }
        return;
    }

    const int h = part, lanes = row_lanes(p.dp), at_once = 256 / lanes;
    const int c = tid % lanes * 8, row_in = tid / lanes;
    for (int k = blockIdx.y; k < t.count; k += gridDim.y) {
        const int64_t pos = 32 * (t.first + k);  // of the tile's first token
        const int64_t page = page_of(p, a.seqs, b, pos);
        if (page < 0) continue;
        // its tokens u0 .. u1 - 1 are new
        const int64_t i0 = pos - t.span.pos0;  // row of the first token; may be negative
        const int u0 = i0 < 0 ? (int)-i0 : 0, u1 = t.span.n - i0 < 32 ? (int)(t.span.n - i0) : 32, nu = u1 - u0;
        const int at = (int)(pos & ((1 << p.page_shift) - 1));
        __syncthreads();  // the last tile has been written
        // rows of keys and then of values, a group of lanes each
        for (int e = row_in; e < 2 * nu; e += at_once) {
            const bool keys = e < nu;
            const int u = u0 + (keys ? e : e - nu);
            const int64_t row = t.span.row0 + i0 + u;
            const char* src = keys ? a.k + (row * a.k_row + (int64_t)h * p.d) * ESZ
                                   : a.v + (row * a.v_row + (int64_t)h * p.d) * ESZ;
            float x[8] = {};
            if (c < p.d) {
                if (keys) load_turned<F32>(src, c, a.rope, a.rope.table ? table_row(a.rope, pos + u) : nullptr, x);
                else load_row8<F32>(src, c, x);
            }
            if constexpr (BYTES) {
                // the largest magnitude by its bits, so that a NaN is above everything: a head that holds one, or an infinity,
                // has no codes, and a scale that says so
                uint32_t m_bits = 0;
#pragma unroll
                for (int q = 0; q < 8; ++q) m_bits = max(m_bits, __float_as_uint(x[q]) & 0x7FFFFFFFu);
                for (int o = lanes / 2; o >= 1; o >>= 1) m_bits = max(m_bits, (uint32_t)__shfl_xor((int)m_bits, o, kWave));
                const float m = __uint_as_float(m_bits);
                const bool none = m_bits >= 0x7F800000u, some = m >= kKvTiny && !none;
                const float top = CT == kKvFp8 ? 448.0f : 127.0f, inv = some ? top / m : 0.0f;
                if (c == 0)
                    (keys ? p.k_scale : p.v_scale)[scale_at(p, page, h, at + u)] =
                        none ? __builtin_nanf("") : some ? m / top : 0.0f;
                uint8_t code[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const float y = none ? 0.0f : fminf(fmaxf(x[q] * inv, -top), top);
                    code[q] = CT == kKvInt8 ? (uint8_t)(int8_t)(int)rintf(y)
                                            : (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(y, y, 0, false);
                }
                if (c < p.dp) {
                    if (keys) {
                        u32x2 w;
                        __builtin_memcpy(&w, code, 8);
                        *(u32x2*)((char*)tile[0] + k_place(u, c, true)) = w;
                    } else {
#pragma unroll
                        for (int q = 0; q < 8; ++q) ((uint8_t*)tile[1])[v_place(u, c + q, true)] = code[q];
                    }
                }
            } else if (c < p.dp) {
                u32x4 w;
#pragma unroll
                for (int q = 0; q < 4; ++q) w[q] = pack_bf16(x[2 * q], x[2 * q + 1]);
                if (keys) {
                    *(u32x4*)((char*)tile[0] + 2 * k_place(u, c, false)) = w;
                } else {
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        ((uint16_t*)tile[1])[v_place(u, c + q, false)] = (uint16_t)(w[q >> 1] >> (16 * (q & 1)));
                }
            }
        }
        __syncthreads();
        const int64_t base = tile_base(p, page, h, at) * CSZ;
        const int pieces = 32 * p.dp * CSZ / 16;  // of 16 bytes
        for (int e = tid; e < 2 * pieces; e += 256) {
            const bool keys = e < pieces;
            const int i = keys ? e : e - pieces;
            const u32x4 w = tile[keys ? 0 : 1][i];
            char* dst = (keys ? p.k : p.v) + base + (int64_t)i * 16;
            if (nu == 32) {
                *(u32x4*)dst = w;
                continue;
            }
            auto is_new = [&](int u) { return u >= u0 && u < u1; };
            // the tokens of the piece's 16 bytes (k_place, v_place)
            if (keys) {
                if constexpr (BYTES) {  // [b][e]
#pragma unroll
                    for (int s = 0; s < 2; ++s)
                        if (is_new(16 * s + (i & 15))) *(u32x2*)(dst + 8 * s) = u32x2{w[2 * s], w[2 * s + 1]};
                } else if (is_new((i & 15) + 16 * ((i >> 6) & 1))) {
                    *(u32x4*)dst = w;
                }
            } else {
                const int g = (i >> 4) & 3;
#pragma unroll
                for (int q = 0; q < 16 / CSZ; ++q) {  // bfloat16 [s][i], 8 bits [y][s][i]
                    if (!is_new(16 * ((q >> 2) & 1) + 4 * g + (q & 3))) continue;
                    if constexpr (BYTES) ((uint8_t*)dst)[q] = (uint8_t)(w[q >> 2] >> (8 * (q & 3)));
                    else ((uint16_t*)dst)[q] = (uint16_t)(w[q >> 1] >> (16 * (q & 1)));
                }
            }
        }
    }
}

// Workgroup x = heads b + h takes tile y (and every gridDim.y-th) of sequence b.
template <bool F32, int CT>
__global__ __launch_bounds__(256) void k_kv_read(KvPool p, KvSeqs s, char* k_out, char* v_out) {
    constexpr bool BYTES = CT != kKvBf16;
    constexpr int CSZ = BYTES ? 1 : 2, ESZ = F32 ? 4 : 2;
    extern __shared__ u32x4 tile[];
    char *keys_lds = (char*)tile, *vals_lds = (char*)(tile + lds_pieces(p.dp, CSZ));
    const int tid = threadIdx.x, b = blockIdx.x / p.heads, h = blockIdx.x - b * p.heads;
    const TileSpan t = tiles_of(s, b);
    const int lanes = row_lanes(p.dp), at_once = 256 / lanes, c = tid % lanes * 8, row_in = tid / lanes;
    // rows of positions that do not exist
    const int before = t.span.pos0 < 0 ? (t.span.pos0 + t.span.n < 0 ? t.span.n : (int)-t.span.pos0) : 0;
    for (int r = blockIdx.y * at_once + row_in; r < before; r += gridDim.y * at_once) {
        const float zero[8] = {};
        const int64_t o = ((t.span.row0 + r) * p.heads + h) * p.d * ESZ;
        if (c < p.d && k_out) store_row8<F32>(k_out + o, c, zero);
        if (c < p.d && v_out) store_row8<F32>(v_out + o, c, zero);
    }
    for (int k = blockIdx.y; k < t.count; k += gridDim.y) {
        const int64_t pos = 32 * (t.first + k);
        const int64_t page = page_of(p, s, b, pos);
        const int64_t i0 = pos - t.span.pos0;
        const int u0 = i0 < 0 ? (int)-i0 : 0, u1 = t.span.n - i0 < 32 ? (int)(t.span.n - i0) : 32, nu = u1 - u0;
        const int at = (int)(pos & ((1 << p.page_shift) - 1));
        const int64_t base = page < 0 ? 0 : tile_base(p, page, h, at) * CSZ;
        const bool shared = nu > 4 && page >= 0;  // (uniform)
        if (shared) {
            const int pieces = 32 * p.dp * CSZ / 16;
            __syncthreads();
            for (int e = tid; e < 2 * pieces; e += 256) {
                const bool keys = e < pieces;
                const int i = keys ? e : e - pieces;
                u32x4* to = keys ? (u32x4*)keys_lds + lds_piece<true>(i) : (u32x4*)vals_lds + lds_piece<false>(i);
                *to = *(const u32x4*)((keys ? p.k : p.v) + base + (int64_t)i * 16);
            }
            __syncthreads();
        }
        for (int e = row_in; e < 2 * nu; e += at_once) {
            const bool keys = e < nu;
            char* out = keys ? k_out : v_out;
            if (!out || c >= p.d) continue;
            const int u = u0 + (keys ? e : e - nu);
            float x[8] = {};
            if (page >= 0) {
                const float sc = BYTES ? (keys ? p.k_scale : p.v_scale)[scale_at(p, page, h, at + u)] : 1.0f;
                const char* src = (keys ? p.k : p.v) + base;
                if (keys) {  // eight columns lie together
                    const char* at = shared ? keys_lds + lds_at<true, BYTES>(u, c) : src + k_place(u, c, BYTES) * CSZ;
                    if constexpr (BYTES) {
                        const u32x2 w = *(const u32x2*)at;
#pragma unroll
                        for (int q = 0; q < 8; ++q) {
                            const uint8_t code = (uint8_t)(w[q >> 2] >> (8 * (q & 3)));
                            x[q] = kv_value((const char*)&code, 0, CT);
                        }
                    } else {
                        load_row8<false>(at, 0, x);
                    }
                } else {
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        x[q] = shared ? kv_value(vals_lds + lds_at<false, BYTES>(u, c + q), 0, CT)
                                      : kv_value(src, v_place(u, c + q, BYTES), CT);
                }
                if constexpr (BYTES) {
#pragma unroll
                    for (int q = 0; q < 8; ++q) x[q] *= sc;
                }
            }
            store_row8<F32>(out + ((t.span.row0 + i0 + u) * p.heads + h) * p.d * ESZ, c, x);
        }
    }
}

namespace {

// Workgroups in a row for the tiles of a sequence; they step on from there.  At most a quarter more than the average
// sequence has: with one for every tile that the longest could have, most of a launch would be workgroups that find nothing
// to do (8 prompts of 1024 to 2048 tokens, rows of 13,000: 85 us of which half).
unsigned tile_steps(const KvSeqs& s, int max_new) {
    const int64_t most = max_new > 0 && max_new < s.rows ? max_new : s.rows;
    int64_t usual = s.rows / s.n_seq;
    usual += usual / 4 + (usual > 1 ? 1 : 0);
    usual = usual < most ? usual : most;
    const int64_t tiles = usual <= 1 ? 1 : (usual + 31) / 32 + 1;
    return (unsigned)(tiles > 4096 ? 4096 : tiles);
}

// LDS of a workgroup that reads: a tile of keys and one of values.
unsigned tile_bytes(const KvPool& p) { return 2 * 16 * (unsigned)lds_pieces(p.dp, p.type == kKvBf16 ? 2 : 1); }

template <class F>
void by_types(int dtype, int type, F f) {
    auto pick = [&](auto f32) {
        if (type == kKvBf16) f(f32, std::integral_constant<int, kKvBf16>{});
        else if (type == kKvFp8) f(f32, std::integral_constant<int, kKvFp8>{});
        else f(f32, std::integral_constant<int, kKvInt8>{});
    };
    if (dtype == 0) pick(std::true_type{});
    else pick(std::false_type{});
}

}  // namespace

hipError_t launch_kv_append(const AppendArgs& a, int max_new, hipStream_t s) {
    if (a.seqs.rows <= 0 || a.seqs.n_seq <= 0) return hipSuccess;
    const unsigned steps = tile_steps(a.seqs, max_new);
    const int how = a.q ? turn_by(a.pool.d, a.rope) : 0;
    // workgroups that share the queries of 32 rows: two items a thread, if the rows are so many
    const int64_t items = a.q ? (int64_t)(steps == 1 ? 1 : 32) * a.q_heads * turn_items(a.pool.d, a.rope.rot, how) : 0;
    int64_t shares = (items + 511) / 512;
    shares = shares > 64 ? 64 : shares;
    const int parts = a.pool.heads + (int)shares;
    if ((int64_t)a.seqs.n_seq * parts > INT32_MAX) return hipErrorInvalidValue;
    by_types(a.dtype, a.pool.type, [&](auto f32, auto ct) {
        k_kv_append<decltype(f32)::value, decltype(ct)::value>
            <<<dim3((unsigned)(a.seqs.n_seq * parts), steps), dim3(256), 0, s>>>(a, parts, how);
    });
    return hipGetLastError();
}

hipError_t launch_kv_read(const KvPool& pool, const KvSeqs& seqs, void* k_out, void* v_out, int dtype, int max_new,
                          hipStream_t s) {
    if (seqs.rows <= 0 || seqs.n_seq <= 0) return hipSuccess;
    if ((int64_t)seqs.n_seq * pool.heads > INT32_MAX) return hipErrorInvalidValue;
    by_types(dtype, pool.type, [&](auto f32, auto ct) {
        k_kv_read<decltype(f32)::value, decltype(ct)::value>
            <<<dim3((unsigned)(seqs.n_seq * pool.heads), tile_steps(seqs, max_new)), dim3(256), tile_bytes(pool), s>>>(
                pool, seqs, (char*)k_out, (char*)v_out);
    });
    return hipGetLastError();
}

}  // namespace lacache
