// decode.cpp -- the C ABI (include/lacache.h) of the decode operators: argument checks and launches.
#include "../../include/lacache.h"

#include <hip/hip_runtime.h>

#include <atomic>
#include <cmath>

#include "kv.hpp"

using namespace lacache;

namespace {

bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

bool is_dtype(lacache_dtype t) { return t == LACACHE_F32 || t == LACACHE_BF16; }

// `data`: the pools' memory is looked at too.
bool to_pool(const lacache_kv* kv, bool data, KvPool* p) {
    if (!kv || kv->n_pages < 0 || kv->n_pages > INT32_MAX || kv->heads < 1 || kv->heads > 65535 || kv->d < 8 ||
        kv->d > 256 || kv->d % 8 != 0 || kv->type < LACACHE_KV_BF16 || kv->type > LACACHE_KV_INT8)
        return false;
    const int shift = kv->page == 32 ? 5 : kv->page == 64 ? 6 : kv->page == 128 ? 7 : kv->page == 256 ? 8 : 0;
    if (!shift) return false;
    const bool bytes = kv->type != LACACHE_KV_BF16;
    if (data && kv->n_pages > 0 &&
        (!kv->k || !kv->v || !aligned(kv->k, 16) || !aligned(kv->v, 16) ||
         (bytes && (!kv->k_scale || !kv->v_scale || !aligned(kv->k_scale, 16) || !aligned(kv->v_scale, 16)))))
        return false;
    *p = {(char*)kv->k, (char*)kv->v, kv->k_scale, kv->v_scale, kv->n_pages, shift, kv->heads, kv->d,
          kv_padded(kv->d), (int)kv->type};
    return true;
}

bool to_seqs(const lacache_seqs* s, int64_t rows, KvSeqs* out) {
    if (!s || rows < 0 || rows > INT32_MAX || s->n_seq < 0 || s->max_pages < 0) return false;
    if (s->n_seq > 0 && rows > 0 && (!s->start || !s->lens || (s->max_pages > 0 && !s->pages))) return false;
    *out = {s->start, s->lens, s->pages, s->n_seq, s->max_pages, rows};
    return true;
}

bool to_rope(const lacache_rotary* r, int d, RopeArgs* out) {
    *out = {};
    if (!r) return true;
    if (!r->table || r->n_pos < 1 || r->rot < 2 || r->rot > d || r->rot % 2 != 0 || !aligned(r->table, 8) ||
        (r->style != LACACHE_ROPE_HALF && r->style != LACACHE_ROPE_PAIRS))
        return false;
    *out = {r->table, r->n_pos, r->rot, r->style == LACACHE_ROPE_PAIRS};
    return true;
}

// Compute units of the current device; 0 on a HIP error.  (Asked once for each of the first 64 devices.)
int compute_units() {
    static std::atomic<int> known[64];
    int dev = 0, n = 0;
    if (hipGetDevice(&dev) == hipSuccess) {
        if (dev < 64 && (n = known[dev].load(std::memory_order_relaxed))) return n;
        if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess) {
            if (dev < 64) known[dev].store(n, std::memory_order_relaxed);
            return n;
        }
    }
    (void)hipGetLastError();
    return 0;
}

}  // namespace

extern "C" {

int lacache_rope_table(float* table, int64_t first, int64_t n, int32_t rot, double base, double factor, double original,
                       double low, double high, double magnitude, void* stream) {
    if (first < 0 || n < 0 || n > INT32_MAX || first > INT32_MAX || rot < 2 || rot > 256 || rot % 2 != 0 ||
        !(base > 1.0) || !std::isfinite(base) || !(factor >= 1.0) || !std::isfinite(factor) || !(original >= 0.0) ||
        !std::isfinite(original) || !(low >= 0.0) || !(high > low) || !std::isfinite(high) || !std::isfinite(magnitude))
        return LACACHE_EINVAL;
    if (n == 0) return LACACHE_OK;
    if (!table || !aligned(table, 8)) return LACACHE_EINVAL;
    return launch_rope_table(table, first, n, rot, base, factor, original, low, high, magnitude,
                             (hipStream_t)stream) == hipSuccess ? LACACHE_OK : LACACHE_EHIP;
}

int lacache_rope(const void* x, void* y, lacache_dtype dtype, int64_t rows, int32_t H, int32_t d, int64_t x_row,
                 int64_t x_head, int64_t y_row, int64_t y_head, const int32_t* pos, const lacache_rotary* rope,
                 int32_t backward, void* stream) {
    RopeArgs r;
    if (!is_dtype(dtype) || rows < 0 || rows > INT32_MAX || H < 1 || H > 65535 || d < 1 || d > 4096 || x_row < 0 ||
        x_head < 0 || y_row < 0 || y_head < 0 || !rope || !to_rope(rope, d, &r))
        return LACACHE_EINVAL;
    if (rows == 0) return LACACHE_OK;
    const uintptr_t esz = dtype == LACACHE_F32 ? 4 : 2;
    if (!x || !y || !pos || !aligned(x, esz) || !aligned(y, esz)) return LACACHE_EINVAL;
    // rows and heads of the result that share elements; a result over its input in another order
    if ((rows > 1 && (y_row < d || (x == y && x_row != y_row))) || (H > 1 && (y_head < d || (x == y && x_head != y_head))))
        return LACACHE_EINVAL;
    return launch_rope(x, y, (int)dtype, rows, H, d, x_row, x_head, y_row, y_head, pos, r, backward != 0,
                       (hipStream_t)stream) == hipSuccess ? LACACHE_OK : LACACHE_EHIP;
}

int lacache_kv_append(const lacache_kv* kv, const lacache_seqs* seqs, const void* k, const void* v, lacache_dtype dtype,
                      int64_t rows, int64_t k_row, int64_t v_row, const void* q, void* q_out, int32_t q_heads,
                      int64_t q_row, const lacache_rotary* rope, int32_t max_new, void* stream) {
    AppendArgs a{};
    if (!to_pool(kv, true, &a.pool) || !to_seqs(seqs, rows, &a.seqs) || !is_dtype(dtype) || k_row < 0 || v_row < 0 ||
        q_row < 0 || max_new < 0 || !to_rope(rope, kv->d, &a.rope))
        return LACACHE_EINVAL;
    const bool with_q = q || q_out;
    if (with_q && (q_heads < 1 || q_heads > 65535 || !rope)) return LACACHE_EINVAL;
    if (rows == 0 || seqs->n_seq == 0) return LACACHE_OK;
    const uintptr_t esz = dtype == LACACHE_F32 ? 4 : 2;
    if (!k || !v || !aligned(k, esz) || !aligned(v, esz) || (with_q && (!q || !q_out || !aligned(q, esz) || !aligned(q_out, esz))))
        return LACACHE_EINVAL;
    a.k = (const char*)k, a.v = (const char*)v, a.q = (const char*)q, a.q_out = (char*)q_out;
    a.dtype = (int)dtype, a.q_heads = with_q ? q_heads : 0;
    a.k_row = k_row, a.v_row = v_row, a.q_row = q_row;
    return launch_kv_append(a, max_new, (hipStream_t)stream) == hipSuccess ? LACACHE_OK : LACACHE_EHIP;
}

int lacache_kv_read(const lacache_kv* kv, const lacache_seqs* seqs, void* k_out, void* v_out, lacache_dtype dtype,
                    int64_t rows, int32_t max_new, void* stream) {
    KvPool p;
    KvSeqs s;
    if (!to_pool(kv, true, &p) || !to_seqs(seqs, rows, &s) || !is_dtype(dtype) || max_new < 0) return LACACHE_EINVAL;
    const uintptr_t esz = dtype == LACACHE_F32 ? 4 : 2;
    if (!aligned(k_out, esz) || !aligned(v_out, esz)) return LACACHE_EINVAL;
    if (rows == 0 || seqs->n_seq == 0 || (!k_out && !v_out)) return LACACHE_OK;
    return launch_kv_read(p, s, k_out, v_out, (int)dtype, max_new, (hipStream_t)stream) == hipSuccess ? LACACHE_OK
                                                                                                      : LACACHE_EHIP;
}

int64_t lacache_kv_attend_workspace(const lacache_kv* kv, lacache_dtype dtype, int32_t n_seq, int32_t q_heads,
                                    int32_t max_new) {
    KvPool p;
    if (!to_pool(kv, false, &p) || !is_dtype(dtype) || n_seq < 0 || q_heads < 1 || q_heads > 65535 ||
        q_heads % kv->heads != 0 || max_new < 0)
        return LACACHE_EINVAL;
    const int cu = compute_units();
    return cu ? attend_workspace(p, (int)dtype, q_heads, max_new, cu) : LACACHE_EHIP;
}

int lacache_kv_attend(const lacache_kv* kv, const lacache_seqs* seqs, const void* q, lacache_dtype dtype, int64_t rows,
                      int32_t q_heads, int64_t q_row, int32_t max_new, float scale, int32_t window, void* out,
                      float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
    AttendArgs a{};
    if (!to_pool(kv, true, &a.pool) || !to_seqs(seqs, rows, &a.seqs) || !is_dtype(dtype) || q_heads < 1 ||
        q_heads > 65535 || q_heads % kv->heads != 0 || q_row < 0 || max_new < 0 || !std::isfinite(scale) ||
        rows * (q_heads / kv->heads) > INT32_MAX || window < 0 || workspace_bytes < 0 ||
        !attend_fits(a.pool, (int)dtype, rows, seqs->n_seq, q_heads / kv->heads, max_new))
        return LACACHE_EINVAL;
    if (rows == 0 || seqs->n_seq == 0) return LACACHE_OK;
    const uintptr_t esz = dtype == LACACHE_F32 ? 4 : 2;
    if (!q || !out || !aligned(q, esz) || !aligned(out, esz) || !aligned(lse, 4)) return LACACHE_EINVAL;
    const int cu = compute_units();
    if (!cu) return LACACHE_EHIP;
    const int64_t need = attend_workspace(a.pool, (int)dtype, q_heads, max_new, cu);
    if (workspace_bytes < need || (need > 0 && (!workspace || !aligned(workspace, 16)))) return LACACHE_EINVAL;
    a.q = (const char*)q, a.out = (char*)out, a.lse = lse;
    a.dtype = (int)dtype, a.q_heads = q_heads, a.group = q_heads / kv->heads, a.window = window;
    a.q_row = q_row, a.scale = scale;
    return launch_kv_attend(a, max_new, workspace, cu, (hipStream_t)stream) == hipSuccess ? LACACHE_OK : LACACHE_EHIP;
}

}  // extern "C"
