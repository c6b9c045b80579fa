// decode.cpp -- the C ABI (include/lacache.h) of the decode operators: argument checks and launches.
#include "../../include/lacache.h"

#include <hip/hip_runtime.h>

#include <atomic>
#include <cmath>

#include "draft.hpp"
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

constexpr int kMostChosen = 1 << 20;  // sequences, pages of a table and of a list where pages are chosen

bool to_bounds(const lacache_bounds* b, KvBounds* out) {
    if (!b || !b->code || !b->scale || !aligned(b->code, 16) || !aligned(b->scale, 4)) return false;
    *out = {b->code, b->scale};
    return true;
}

// Bytes of the scores of all pages; LACACHE_EINVAL where they do not fit in 64 bits.
int64_t select_space(const KvPool& p, int64_t rows, int max_pages) {
    const int64_t lists = rows * p.heads, each = 4 * select_stride(max_pages);
    return each == 0 || lists <= INT64_MAX / each ? lists * each : LACACHE_EINVAL;
}

// Strides that keep n of them (0 or more) far from the ends of 64 bits.
bool fits_far(int64_t stride, int64_t n) { return n < 2 || stride < (INT64_C(1) << 58) / n; }

// Whether bytes lo .. hi - 1 meet one of the rows (n elements of esz bytes each, `rows` of them `row` elements apart in each of
// `seqs` sequences, `seq` elements apart).  Where they lie between the first row's begin and the last one's end, sequence
// after sequence: they may lie between rows.
bool rows_meet(const void* base, int64_t esz, int64_t n, int64_t seq, int64_t seqs, int64_t row, int64_t rows, int64_t lo, int64_t hi) {
    if (lo >= hi || seqs < 1 || rows < 1) return false;
    lo -= (int64_t)base, hi -= (int64_t)base, n *= esz, seq *= seqs > 1 ? esz : 0, row *= rows > 1 ? esz : 0;
    if (hi <= 0 || lo >= (seqs - 1) * seq + (rows - 1) * row + n) return false;
    for (int64_t b = 0; b < seqs; ++b) {
        const int64_t from = lo - b * seq - n, to = hi - b * seq;  // a row that begins between these
        const int64_t j = from < 0 ? 0 : row > 0 ? from / row + 1 : rows;
        if (j < rows && j * row < to) return true;
    }
    return false;
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

int64_t lacache_kv_attend_shared_workspace(const lacache_kv* kv, lacache_dtype dtype, int64_t rows, int32_t n_seq,
                                           int32_t n_groups, int32_t q_heads, int32_t max_new) {
    KvPool p;
    if (!to_pool(kv, false, &p) || !is_dtype(dtype) || rows < 0 || rows > INT32_MAX || n_seq < 0 || n_seq > kMostChosen ||
        n_groups < 0 || n_groups > kMostChosen || q_heads < 1 || q_heads > 65535 || q_heads % kv->heads != 0 || max_new < 0)
        return LACACHE_EINVAL;
    const int cu = compute_units();
    return cu ? attend_shared_workspace(p, (int)dtype, rows, n_seq, n_groups, q_heads, max_new, cu) : LACACHE_EHIP;
}

int lacache_kv_attend_shared(const lacache_kv* kv, const lacache_seqs* seqs, const lacache_prefixes* prefixes,
                             const void* q, lacache_dtype dtype, int64_t rows, int32_t q_heads, int64_t q_row,
                             int32_t max_new, float scale, int32_t window, void* out, float* lse, void* workspace,
                             int64_t workspace_bytes, void* stream) {
    AttendArgs a{};
    if (!to_pool(kv, true, &a.pool) || !to_seqs(seqs, rows, &a.seqs) || !is_dtype(dtype) || q_heads < 1 ||
        q_heads > 65535 || q_heads % kv->heads != 0 || q_row < 0 || max_new < 0 || !std::isfinite(scale) ||
        rows * (q_heads / kv->heads) > INT32_MAX || window < 0 || workspace_bytes < 0 || !prefixes || prefixes->n_groups < 0 ||
        prefixes->n_groups > kMostChosen || a.seqs.n_seq > kMostChosen ||
        (prefixes->n_groups > 0 && (!prefixes->group || !prefixes->len || !aligned(prefixes->group, 4) || !aligned(prefixes->len, 4))) ||
        !attend_fits(a.pool, (int)dtype, rows, seqs->n_seq, q_heads / kv->heads, max_new) ||
        !attend_shared_fits(a.pool, (int)dtype, rows, prefixes->n_groups, q_heads / kv->heads))
        return LACACHE_EINVAL;
    if (rows == 0 || seqs->n_seq == 0) return LACACHE_OK;
    const uintptr_t esz = dtype == LACACHE_F32 ? 4 : 2;
    if (!q || !out || !aligned(q, esz) || !aligned(out, esz) || !aligned(lse, 4)) return LACACHE_EINVAL;
    const int cu = compute_units();
    if (!cu) return LACACHE_EHIP;
    const int64_t need = attend_shared_workspace(a.pool, (int)dtype, rows, seqs->n_seq, prefixes->n_groups, q_heads, max_new, cu);
    if (workspace_bytes < need || (need > 0 && (!workspace || !aligned(workspace, 16)))) return LACACHE_EINVAL;
    a.q = (const char*)q, a.out = (char*)out, a.lse = lse;
    a.dtype = (int)dtype, a.q_heads = q_heads, a.group = q_heads / kv->heads, a.window = window;
    a.q_row = q_row, a.scale = scale;
    return launch_kv_attend_shared(a, prefixes->group, prefixes->len, prefixes->n_groups, max_new, workspace, cu,
                                   (hipStream_t)stream) == hipSuccess ? LACACHE_OK : LACACHE_EHIP;
}

int lacache_kv_bound(const lacache_kv* kv, const lacache_bounds* bounds, const lacache_seqs* seqs, int64_t rows,
                     int32_t max_new, void* stream) {
    KvPool p;
    KvSeqs s;
    KvBounds b;
    if (!to_pool(kv, true, &p) || !to_seqs(seqs, rows, &s) || s.n_seq > kMostChosen || s.max_pages > kMostChosen || max_new < 0)
        return LACACHE_EINVAL;
    if (rows == 0 || s.n_seq == 0 || p.n_pages == 0) return LACACHE_OK;
    if (!to_bounds(bounds, &b)) return LACACHE_EINVAL;
    return launch_kv_bound(p, b, s, max_new, (hipStream_t)stream) == hipSuccess ? LACACHE_OK : LACACHE_EHIP;
}

int lacache_kv_bounds_read(const lacache_kv* kv, const lacache_bounds* bounds, const int32_t* pages, int64_t n,
                           float* most, float* least, void* stream) {
    KvPool p;
    KvBounds b;
    if (!to_pool(kv, false, &p) || n < 0 || n > INT32_MAX || !aligned(pages, 4) || !aligned(most, 4) || !aligned(least, 4))
        return LACACHE_EINVAL;
    if (n == 0 || (!most && !least)) return LACACHE_OK;
    if (!pages || (p.n_pages > 0 && !to_bounds(bounds, &b))) return LACACHE_EINVAL;
    return launch_kv_bounds_read(p, b, pages, n, most, least, (hipStream_t)stream) == hipSuccess ? LACACHE_OK : LACACHE_EHIP;
}

int64_t lacache_kv_select_workspace(const lacache_kv* kv, int64_t rows, int32_t max_pages) {
    KvPool p;
    if (!to_pool(kv, false, &p) || rows < 0 || rows > INT32_MAX || max_pages < 0 || max_pages > kMostChosen)
        return LACACHE_EINVAL;
    return select_space(p, rows, max_pages);
}

int lacache_kv_select(const lacache_kv* kv, const lacache_bounds* bounds, const lacache_seqs* seqs, const void* q,
                      lacache_dtype dtype, int64_t rows, int32_t q_heads, int64_t q_row, int32_t n_blocks, int32_t first,
                      int32_t last, int32_t max_new, int32_t* blocks, void* workspace, int64_t workspace_bytes,
                      void* stream) {
    SelectArgs a{};
    if (!to_pool(kv, false, &a.pool) || !to_seqs(seqs, rows, &a.seqs) || !is_dtype(dtype) || q_heads < 1 ||
        q_heads > 65535 || q_heads % kv->heads != 0 || q_row < 0 || max_new < 0 || a.seqs.n_seq > kMostChosen ||
        a.seqs.max_pages > kMostChosen || n_blocks < 1 || n_blocks > kMostChosen || first < 0 || last < 0 ||
        (int64_t)first + last > n_blocks || workspace_bytes < 0)
        return LACACHE_EINVAL;
    if (rows == 0 || a.seqs.n_seq == 0) return LACACHE_OK;
    const int64_t need = select_space(a.pool, rows, a.seqs.max_pages);
    if (need < 0 || !q || !blocks || !aligned(q, dtype == LACACHE_F32 ? 4 : 2) || !aligned(blocks, 4) || workspace_bytes < need ||
        (need > 0 && (!workspace || !aligned(workspace, 16))) || (a.pool.n_pages > 0 && !to_bounds(bounds, &a.bounds)))
        return LACACHE_EINVAL;
    a.q = (const char*)q, a.dtype = (int)dtype, a.group = q_heads / kv->heads, a.q_row = q_row;
    a.n_blocks = n_blocks, a.first = first, a.last = last, a.blocks = blocks, a.scores = (float*)workspace;
    return launch_kv_select(a, max_new, (hipStream_t)stream) == hipSuccess ? LACACHE_OK : LACACHE_EHIP;
}

int64_t lacache_kv_attend_blocks_workspace(const lacache_kv* kv, int64_t rows, int32_t q_heads, int32_t n_blocks) {
    KvPool p;
    if (!to_pool(kv, false, &p) || rows < 0 || rows > INT32_MAX || q_heads < 1 || q_heads > 65535 ||
        q_heads % kv->heads != 0 || n_blocks < 1 || n_blocks > kMostChosen)
        return LACACHE_EINVAL;
    const int cu = compute_units();
    return cu ? blocks_workspace(p, rows, q_heads / kv->heads, n_blocks, cu) : LACACHE_EHIP;
}

int lacache_kv_attend_blocks(const lacache_kv* kv, const lacache_seqs* seqs, const void* q, lacache_dtype dtype,
                             int64_t rows, int32_t q_heads, int64_t q_row, const int32_t* blocks, int32_t n_blocks,
                             float scale, void* out, float* lse, void* workspace, int64_t workspace_bytes,
                             void* stream) {
    BlocksArgs x{};
    AttendArgs& a = x.a;
    if (!to_pool(kv, true, &a.pool) || !to_seqs(seqs, rows, &a.seqs) || !is_dtype(dtype) || q_heads < 1 ||
        q_heads > 65535 || q_heads % kv->heads != 0 || q_row < 0 || !std::isfinite(scale) || a.seqs.n_seq > kMostChosen ||
        a.seqs.max_pages > kMostChosen || n_blocks < 1 || n_blocks > kMostChosen || workspace_bytes < 0)
        return LACACHE_EINVAL;
    a.group = q_heads / kv->heads;
    if (rows * kv->heads * ((a.group + 15) / 16) >= 1 << 24) return LACACHE_EINVAL;
    if (rows == 0 || a.seqs.n_seq == 0) return LACACHE_OK;
    const uintptr_t esz = dtype == LACACHE_F32 ? 4 : 2;
    if (!q || !out || !blocks || !aligned(q, esz) || !aligned(out, esz) || !aligned(lse, 4) || !aligned(blocks, 4))
        return LACACHE_EINVAL;
    const int cu = compute_units();
    if (!cu) return LACACHE_EHIP;
    const int64_t need = blocks_workspace(a.pool, rows, a.group, n_blocks, cu);
    if (workspace_bytes < need || (need > 0 && (!workspace || !aligned(workspace, 16)))) return LACACHE_EINVAL;
    a.q = (const char*)q, a.out = (char*)out, a.lse = lse;
    a.dtype = (int)dtype, a.q_heads = q_heads, a.window = 0, a.q_row = q_row, a.scale = scale;
    x.blocks = blocks, x.n_blocks = n_blocks;
    return launch_attend_blocks(x, workspace, cu, (hipStream_t)stream) == hipSuccess ? LACACHE_OK : LACACHE_EHIP;
}

int64_t lacache_verify_workspace(int32_t V, int32_t B, int32_t k) {
    return V < 1 || B < 0 || B > 65535 || k < 0 || k > 4096 ? LACACHE_EINVAL : draft_workspace(V, B, k);
}

int lacache_verify(const void* logits, const void* draft_logits, lacache_dtype dtype, int32_t V, int64_t t_seq,
                   int64_t t_row, int64_t d_seq, int64_t d_row, const int32_t* draft_tokens, const float* u_accept,
                   const float* u_next, const float* temperature, const int32_t* n_draft, int32_t B, int32_t k,
                   int32_t* accept_len, int32_t* next_token, float* p_target, float* p_draft, void* workspace,
                   int64_t workspace_bytes, void* stream) {
    if (!is_dtype(dtype) || V < 1 || B < 0 || B > 65535 || k < 0 || k > 4096 || t_seq < 0 || t_row < 0 || d_seq < 0 ||
        d_row < 0 || workspace_bytes < 0 || (int64_t)B * (V / 2048 + 1) >= 1 << 24)
        return LACACHE_EINVAL;
    if (B == 0) return LACACHE_OK;
    const uintptr_t esz = dtype == LACACHE_F32 ? 4 : 2;
    if (!logits || !u_next || !accept_len || !next_token || !workspace || !aligned(logits, esz) || !aligned(u_next, 4) ||
        !aligned(accept_len, 4) || !aligned(next_token, 4) || !aligned(temperature, 4) || !aligned(n_draft, 4) ||
        !aligned(workspace, 16) || workspace_bytes < draft_workspace(V, B, k))
        return LACACHE_EINVAL;
    if (k > 0 && (!draft_logits || !draft_tokens || !u_accept || !p_target || !p_draft || !aligned(draft_logits, esz) ||
                  !aligned(draft_tokens, 4) || !aligned(u_accept, 4) || !aligned(p_target, 4) || !aligned(p_draft, 4)))
        return LACACHE_EINVAL;
    if (!fits_far(t_seq, B) || !fits_far(d_seq, B) || !fits_far(t_row, k + 1) || !fits_far(d_row, k)) return LACACHE_EINVAL;
    // (workgroups write a sequence's results while others still read what they are found from)
    const struct {
        const void* at;
        int64_t n;
    } used[] = {{workspace, draft_workspace(V, B, k)}, {accept_len, 4 * (int64_t)B}, {next_token, 4 * (int64_t)B},
                {p_target, 4 * (int64_t)B * k}, {p_draft, 4 * (int64_t)B * k},  // written
                {draft_tokens, 4 * (int64_t)B * k}, {u_accept, 4 * (int64_t)B * k}, {u_next, 4 * (int64_t)B},
                {temperature, 4 * (int64_t)B}, {n_draft, 4 * (int64_t)B}};
    for (int i = 0; i < 5; ++i) {
        const int64_t x = (int64_t)used[i].at;
        for (int j = i + 1; j < 10; ++j) {
            const int64_t y = (int64_t)used[j].at;
            if (y && x < y + used[j].n && y < x + used[i].n) return LACACHE_EINVAL;
        }
        if (rows_meet(logits, (int64_t)esz, V, t_seq, B, t_row, k + 1, x, x + used[i].n) ||
            rows_meet(draft_logits, (int64_t)esz, V, d_seq, B, d_row, k, x, x + used[i].n))
            return LACACHE_EINVAL;
    }
    DraftArgs a{};
    a.logits = (const char*)logits, a.draft_logits = (const char*)draft_logits;
    a.dtype = (int)dtype, a.V = V, a.B = B, a.k = k;
    a.t_seq = t_seq, a.t_row = t_row, a.d_seq = d_seq, a.d_row = d_row;
    a.tokens = draft_tokens, a.n_draft = n_draft, a.u_accept = u_accept, a.u_next = u_next, a.temperature = temperature;
    a.accept_len = accept_len, a.next_token = next_token, a.p_target = p_target, a.p_draft = p_draft;
    return launch_verify_drafts(a, workspace, (hipStream_t)stream) == hipSuccess ? LACACHE_OK : LACACHE_EHIP;
}

}  // extern "C"
