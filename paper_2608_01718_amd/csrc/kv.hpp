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

// Largest code of the 8-bit types, and the magnitude below which a head is stored as zeros (its reciprocal, times the
// largest code, would overflow).
__device__ inline float kv_top(int type) { return type == kKvFp8 ? 448.0f : 127.0f; }
constexpr float kKvTiny = 0x1p-100f;

// a c - b s and b c + a s, every product and sum rounded (no fused multiply-add: the codes of the 8-bit types are then
// those of the formula in float32, whatever computes it).
__device__ inline void turn(float& a, float& b, float c, float s) {
#pragma clang fp contract(off)
    const float x = a * c, y = b * s, z = b * c, w = a * s;
    a = x - y;
    b = z + w;
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
int64_t attend_workspace(const KvPool& pool, int dtype, int n_seq, int q_heads, int max_new, int num_cu);
hipError_t launch_kv_attend(const AttendArgs& a, int max_new, void* workspace, int num_cu, hipStream_t s);

}  // namespace lacache
