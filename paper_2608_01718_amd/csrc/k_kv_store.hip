// k_kv_store.hip -- writing new tokens into the pages of the key-value cache, and reading them back.
//
// A token's keys of one head (turned by its position, if a table is given) or values are rounded once: to bfloat16, or
// to 8-bit codes x * (top / m) with the scale m / top, m the largest magnitude of the d columns.
#include "kv.hpp"
#include "launch.hpp"

namespace lacache {

namespace {

// columns lane, lane + 64, ... of one head's row, turned
__device__ inline void load_row(const char* src, int dtype, int d, int lane, const RopeArgs& rope, int64_t pos,
                                float x[4]) {
    auto get = [&](int c) { return dtype == 0 ? ((const float*)src)[c] : bf16_to_f32(((const uint16_t*)src)[c]); };
    const int half = rope.rot / 2;
    const int64_t p = pos < 0 ? 0 : pos >= rope.n_pos ? rope.n_pos - 1 : pos;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int c = lane + 64 * e;
        x[e] = c < d ? get(c) : 0.0f;
        if (rope.table && c < rope.rot) {
            const int i = rope.pairs ? c >> 1 : c < half ? c : c - half;
            const bool first = rope.pairs ? !(c & 1) : c < half;
            const float2 cs = ((const float2*)rope.table)[p * half + i];
            float a = x[e], b = get(rope.pairs ? c ^ 1 : first ? c + half : c - half);
            if (!first) {
                const float t = a;
                a = b;
                b = t;
            }
            turn(a, b, cs.x, cs.y);
            x[e] = first ? a : b;
        }
    }
}

}  // namespace

// A wave per (token, head): the query heads, the key heads, the value heads.  blockIdx.y steps through the new tokens
// of sequence blockIdx.x.
__global__ __launch_bounds__(256) void k_kv_append(AppendArgs a) {
    const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
    const KvPool& p = a.pool;
    const bool bytes = p.type != kKvBf16;
    const size_t esz = a.dtype == 0 ? 4 : 2;
    const KvSpan span = span_of(a.seqs, blockIdx.x);
    const int Hq = a.q ? a.q_heads : 0;
    for (int i = blockIdx.y; i < span.n; i += gridDim.y) {
        const int64_t row = span.row0 + i, pos = span.pos0 + i;
        const int64_t page = pos < 0 ? -1 : page_of(p, a.seqs, blockIdx.x, pos);
        const int at = (int)(pos & ((1 << p.page_shift) - 1));
        for (int h = wid; h < Hq + 2 * p.heads; h += 4) {
            float x[4];
            if (h < Hq) {
                load_row(a.q + (row * a.q_row + (int64_t)h * p.d) * esz, a.dtype, p.d, lane, a.rope, pos, x);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int64_t o = (row * a.q_heads + h) * p.d + lane + 64 * e;
                    if (lane + 64 * e >= p.d) continue;
                    if (a.dtype == 0) ((float*)a.q_out)[o] = x[e];
                    else ((uint16_t*)a.q_out)[o] = f32_to_bf16(x[e]);
                }
                continue;
            }
            if (page < 0) continue;
            const bool keys = h < Hq + p.heads;
            const int hk = h - Hq - (keys ? 0 : p.heads);
            RopeArgs rope = a.rope;
            if (!keys) rope.table = nullptr;
            load_row((keys ? a.k + row * a.k_row * esz : a.v + row * a.v_row * esz) + (int64_t)hk * p.d * esz, a.dtype,
                     p.d, lane, rope, pos, x);
            float m = fmaxf(fmaxf(fabsf(x[0]), fabsf(x[1])), fmaxf(fabsf(x[2]), fabsf(x[3])));
            m = wave_reduce(m, [](float u, float v) { return fmaxf(u, v); });
            const bool some = m >= kKvTiny;
            const float top = kv_top(p.type), inv = some ? top / m : 0.0f;
            char* pool = (keys ? p.k : p.v);
            const int64_t base = tile_base(p, page, hk, at);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int c = lane + 64 * e;
                if (c >= p.dp) continue;
                const int64_t o = base + (keys ? k_place(at & 31, c, bytes) : v_place(at & 31, c, bytes));
                const float y = fminf(fmaxf(x[e] * inv, -top), top);
                if (!bytes) ((uint16_t*)pool)[o] = f32_to_bf16(x[e]);
                else if (p.type == kKvInt8) ((int8_t*)pool)[o] = (int8_t)(int)rintf(y);
                else ((uint8_t*)pool)[o] = (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(y, y, 0, false);
            }
            if (bytes && lane == 0)
                (keys ? p.k_scale : p.v_scale)[scale_at(p, page, hk, at)] = some ? m / top : 0.0f;
        }
    }
}

// A wave per (token, head) of keys and of values.
__global__ __launch_bounds__(256) void k_kv_read(KvPool p, KvSeqs s, void* k_out, void* v_out, int dtype) {
    const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
    const bool bytes = p.type != kKvBf16;
    const KvSpan span = span_of(s, blockIdx.x);
    for (int i = blockIdx.y; i < span.n; i += gridDim.y) {
        const int64_t row = span.row0 + i, pos = span.pos0 + i;
        const int64_t page = pos < 0 ? -1 : page_of(p, s, blockIdx.x, pos);
        const int at = (int)(pos & ((1 << p.page_shift) - 1));
        for (int h = wid; h < 2 * p.heads; h += 4) {
            const bool keys = h < p.heads;
            const int hk = keys ? h : h - p.heads;
            void* out = keys ? k_out : v_out;
            if (!out) continue;
            const int64_t base = page < 0 ? 0 : tile_base(p, page, hk, at);
            const float sc = bytes && page >= 0 ? (keys ? p.k_scale : p.v_scale)[scale_at(p, page, hk, at)] : 1.0f;
            for (int c = lane; c < p.d; c += 64) {
                float x = 0.0f;
                if (page >= 0)
                    x = kv_value(keys ? p.k : p.v, base + (keys ? k_place(at & 31, c, bytes) : v_place(at & 31, c, bytes)),
                                 p.type) * sc;
                const int64_t o = (row * p.heads + hk) * p.d + c;
                if (dtype == 0) ((float*)out)[o] = x;
                else ((uint16_t*)out)[o] = f32_to_bf16(x);
            }
        }
    }
}

static dim3 token_grid(const KvSeqs& s, int max_new) {
    int64_t most = max_new > 0 && max_new < s.rows ? max_new : s.rows;
    return dim3((unsigned)s.n_seq, (unsigned)(most > 1024 ? 1024 : most));
}

hipError_t launch_kv_append(const AppendArgs& a, int max_new, hipStream_t s) {
    if (a.seqs.rows <= 0 || a.seqs.n_seq <= 0) return hipSuccess;
    k_kv_append<<<token_grid(a.seqs, max_new), dim3(256), 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_kv_read(const KvPool& pool, const KvSeqs& seqs, void* k_out, void* v_out, int dtype, int max_new,
                          hipStream_t s) {
    if (seqs.rows <= 0 || seqs.n_seq <= 0) return hipSuccess;
    k_kv_read<<<token_grid(seqs, max_new), dim3(256), 0, s>>>(pool, seqs, k_out, v_out, dtype);
    return hipGetLastError();
}

}  // namespace lacache
