// kv.hpp -- the paged key-value cache of the decode operators: its description, layout and launchers.
#pragma once

#include "common.hpp"

namespace lacache {

enum KvType { kKvBf16 = 1, kKvFp8 = 2, kKvInt8 = 3 };

// A pool as the kernels see it (lacache_kv with its padded columns and its page size as a shift).
struct KvPool {
    char *k, *v;
    float *k_scale, *v_scale;
    int64_t n_pages;
    int page_shift, heads, d, dp, type;
};

// The sequences of a call (lacache_seqs) and its row count.
struct KvSeqs {
    const int32_t *start, *lens, *pages;
    int n_seq, max_pages;
    int64_t rows;
};

struct RopeArgs {
    const float* table;  // null: nothing turns
    int64_t n_pos;
    int rot;
    int pairs;  // LACACHE_ROPE_PAIRS
};

// Columns of a padded head.
inline int kv_padded(int d) { return d <= 64 ? 64 : d <= 96 ? 96 : d <= 128 ? 128 : d <= 192 ? 192 : 256; }

// ---------------------------------------------------------------------------
// A tile is 32 tokens x dp columns, its elements in the order of the matrix operands of k_attend.hip.  Keys: the A
// operand of S^T = K Q^T, 16 tokens x 32 columns a 16x16x32 instruction, lane 16 u + r holding columns 8 u .. 8 u + 7 of
// token r.  Values: the A operand of O^T = V^T P^T, 16 columns x 32 tokens, lane 16 g + m holding column m of tokens
// {4 g .. 4 g + 3} and {16 + 4 g ..}: those whose weights the same lane group holds after S^T, so that no weight changes
// lanes between the two products.  16 bytes a lane are one operand in bfloat16 and two in 8 bits (the tile's two token
// blocks of keys, two column blocks of values).
// ---------------------------------------------------------------------------
__host__ __device__ inline int k_place(int t, int c, bool bytes) {
    const int x = c >> 5, u = (c >> 3) & 3, e = c & 7, b = t >> 4, r = t & 15;
    return bytes ? (((x * 4 + u) * 16 + r) * 2 + b) * 8 + e : (((x * 2 + b) * 4 + u) * 16 + r) * 8 + e;
}
__host__ __device__ inline int v_place(int t, int c, bool bytes) {
    const int x = c >> 5, y = (c >> 4) & 1, m = c & 15, s = t >> 4, g = (t >> 2) & 3, i = t & 3;
    return bytes ? ((((x * 4 + g) * 16 + m) * 2 + y) * 2 + s) * 4 + i : ((((x * 2 + y) * 4 + g) * 16 + m) * 2 + s) * 4 + i;
}

// First element of the tile that holds place `at` of a page, for one head.
__device__ inline int64_t tile_base(const KvPool& p, int64_t page, int head, int at) {
    return (((page * p.heads + head) << (p.page_shift - 5)) + (at >> 5)) * (32 * p.dp);
}
__device__ inline int64_t scale_at(const KvPool& p, int64_t page, int head, int at) {
    return ((page * p.heads + head) << p.page_shift) + at;
}

// The page of position pos (>= 0) of sequence b; -1 if there is none.
__device__ inline int64_t page_of(const KvPool& p, const KvSeqs& s, int b, int64_t pos) {
    const int64_t i = pos >> p.page_shift;
    if (i >= s.max_pages) return -1;
    const int64_t page = s.pages[(int64_t)b * s.max_pages + i];
    return page >= 0 && page < p.n_pages ? page : -1;
}

// The newest tokens of sequence b: first row, number of rows, position of the first row.
struct KvSpan {
    int64_t row0;
    int n;
    int64_t pos0;
};
__device__ inline KvSpan span_of(const KvSeqs& s, int b) {
    int64_t a = s.start[b], e = s.start[b + 1];
    a = a < 0 ? 0 : a > s.rows ? s.rows : a;
    e = e < a ? a : e > s.rows ? s.rows : e;
    return {a, (int)(e - a), (int64_t)s.lens[b] - (e - a)};
}

__device__ inline float kv_value(const char* pool, int64_t i, int type) {
    if (type == kKvBf16) return bf16_to_f32(((const uint16_t*)pool)[i]);
    if (type == kKvInt8) return (float)((const int8_t*)pool)[i];
    return __builtin_amdgcn_cvt_f32_fp8((int)((const uint8_t*)pool)[i], 0);
}

// 16 bytes at any element boundary (gfx950 takes vector accesses of any alignment)
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef f32x4 f32x4_any __attribute__((aligned(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));

__device__ inline uint16_t f32_to_bf16(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    bf16x2 w;  // (converted as a pair: one instruction)
    w[0] = (__bf16)a;
    w[1] = (__bf16)b;
    return __builtin_bit_cast(uint32_t, w);
}

// The magnitude below which a head is stored as zeros (its reciprocal, times the largest code, would overflow).
constexpr float kKvTiny = 0x1p-100f;

// a c - b s and b c + a s, every product and sum rounded (no fused multiply-add: the codes of the 8-bit types are then
// those of the formula in float32, whatever computes it).
__device__ inline void turn(float& a, float& b, float c, float s) {
#pragma clang fp contract(off)
    const float x = a * c, y = b * s, z = b * c, w = a * s;
    a = x - y;
    b = z + w;
}

// Eight elements of activations, at any element boundary.
template <bool F32>
__device__ __forceinline__ void load_row8(const char* row, int c, float (&x)[8]) {
    if constexpr (F32) {
        const f32x4 a = *(const f32x4_any*)(row + c * 4), b = *(const f32x4_any*)(row + c * 4 + 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = a[e], x[4 + e] = b[e];
    } else {
        const u32x4 w = *(const u32x4_any*)(row + c * 2);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[2 * e] = __uint_as_float(w[e] << 16);
            x[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
        }
    }
}
template <bool F32>
__device__ __forceinline__ void store_row8(char* row, int c, const float (&x)[8]) {
    if constexpr (F32) {
        *(f32x4_any*)(row + c * 4) = f32x4{x[0], x[1], x[2], x[3]};
        *(f32x4_any*)(row + c * 4 + 16) = f32x4{x[4], x[5], x[6], x[7]};
    } else {
        u32x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = pack_bf16(x[2 * e], x[2 * e + 1]);
        *(u32x4_any*)(row + c * 2) = w;
    }
}
template <bool F32>
__device__ __forceinline__ float load_row1(const char* row, int c) {
    return F32 ? ((const float*)row)[c] : bf16_to_f32(((const uint16_t*)row)[c]);
}
template <bool F32>
__device__ __forceinline__ void store_row1(char* row, int c, float x) {
    if constexpr (F32) ((float*)row)[c] = x;
    else ((uint16_t*)row)[c] = f32_to_bf16(x);
}

// How a row of a head is turned, in items that no other item's columns overlap (the result may be written over the input):
// eight columns each with their cosines and sines (pairs of neighbours), sixteen (two times eight, half a head apart), or
// a pair at a time where the columns are not whole eights.
enum TurnBy { kTurnOne = 0, kTurnPairs = 1, kTurnHalves = 2 };
inline TurnBy turn_by(int d, const RopeArgs& r) {
    return d % 8 != 0 ? kTurnOne : r.pairs ? (r.rot % 8 == 0 ? kTurnPairs : kTurnOne) : r.rot % 16 == 0 ? kTurnHalves : kTurnOne;
}
__host__ __device__ inline int turn_items(int d, int rot, int by) {
    return by == kTurnPairs ? d / 8 : by == kTurnHalves ? d / 8 - rot / 16 : d - rot / 2;
}
// Item i of a head: from x to y, cs the table's row of its position, sign -1 for the transposed rotation.
template <bool F32, int BY>
__device__ __forceinline__ void turn_item(const char* x, char* y, int d, const RopeArgs& rope, const float2* cs, int i,
                                          float sign) {
    const int half = rope.rot / 2;
    float a[8], b[8];
    if constexpr (BY == kTurnOne) {
        if (i >= half) {
            store_row1<F32>(y, i + half, load_row1<F32>(x, i + half));
            return;
        }
        const int ca = rope.pairs ? 2 * i : i, cb = rope.pairs ? 2 * i + 1 : i + half;
        float u = load_row1<F32>(x, ca), v = load_row1<F32>(x, cb);
        turn(u, v, cs[i].x, sign * cs[i].y);
        store_row1<F32>(y, ca, u);
        store_row1<F32>(y, cb, v);
    } else if constexpr (BY == kTurnPairs) {
        load_row8<F32>(x, 8 * i, a);
        if (8 * i < rope.rot) {
            const f32x4 p = *(const f32x4_any*)&cs[4 * i], q = *(const f32x4_any*)&cs[4 * i + 2];
            turn(a[0], a[1], p[0], sign * p[1]);
            turn(a[2], a[3], p[2], sign * p[3]);
            turn(a[4], a[5], q[0], sign * q[1]);
            turn(a[6], a[7], q[2], sign * q[3]);
        }
        store_row8<F32>(y, 8 * i, a);
    } else {
        const bool turns = 16 * i < rope.rot;
        const int c = turns ? 8 * i : 8 * i + half;  // behind the turned columns: one eight an item
        load_row8<F32>(x, c, a);
        if (turns) {
            load_row8<F32>(x, c + half, b);
            f32x4 p[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e] = *(const f32x4_any*)&cs[c + 2 * e];
#pragma unroll
            for (int e = 0; e < 8; ++e) turn(a[e], b[e], p[e / 2][2 * (e & 1)], sign * p[e / 2][2 * (e & 1) + 1]);
            store_row8<F32>(y, c + half, b);
        }
        store_row8<F32>(y, c, a);
    }
}
__device__ inline const float2* table_row(const RopeArgs& rope, int64_t pos) {
    pos = pos < 0 ? 0 : pos >= rope.n_pos ? rope.n_pos - 1 : pos;
    return (const float2*)rope.table + pos * (rope.rot / 2);
}

hipError_t launch_rope_table(float* table, int64_t first, int64_t n, int rot, double base, double factor,
                             double original, double low, double high, double magnitude, hipStream_t s);
hipError_t launch_rope(const void* x, void* y, int dtype, int64_t rows, int H, int d, int64_t x_row, int64_t x_head,
                       int64_t y_row, int64_t y_head, const int32_t* pos, const RopeArgs& rope, bool backward,
                       hipStream_t s);
struct AppendArgs {
    KvPool pool;
    KvSeqs seqs;
    RopeArgs rope;
    const char *k, *v, *q;
    char* q_out;
    int dtype, q_heads;
    int64_t k_row, v_row, q_row;
};
hipError_t launch_kv_append(const AppendArgs& a, int max_new, hipStream_t s);
hipError_t launch_kv_read(const KvPool& pool, const KvSeqs& seqs, void* k_out, void* v_out, int dtype, int max_new,
                          hipStream_t s);
struct AttendArgs {
    KvPool pool;
    KvSeqs seqs;
    const char* q;
    char* out;
    float* lse;
    int dtype, q_heads, group, window;
    int64_t q_row;
    float scale;
};
// Whether the row groups of a call can be counted in 32 bits.
bool attend_fits(const KvPool& pool, int dtype, int64_t rows, int n_seq, int group, int max_new);
int64_t attend_workspace(const KvPool& pool, int dtype, int q_heads, int max_new, int num_cu);
hipError_t launch_kv_attend(const AttendArgs& a, int max_new, void* workspace, int num_cu, hipStream_t s);

}  // namespace lacache
