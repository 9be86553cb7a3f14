// The C ABI of the operators on a paged cache: argument validation and dispatch.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <initializer_list>

#include "../../include/flashd.h"
#include "flashd_common.h"
#include "flashd_kernels.h"
#include "flashd_paged.h"

namespace {

using flashd::AppendArgs;
using flashd::EvictArgs;
using flashd::Paged;
using flashd::ScoreArgs;
using flashd::TreeArgs;
using flashd::VerifyArgs;

static_assert(FLASHD_CACHE_MAX_SEQS == flashd::kCacheMaxSeqs, "the header states the kernels' limit");

int esize(int dtype) { return dtype == FLASHD_F32 ? 4 : dtype == FLASHD_CACHE_FP8 ? 1 : 2; }

bool overlap(const void* a, int64_t abytes, const void* b, int64_t bbytes) {
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return abytes > 0 && bbytes > 0 && x < y + (uintptr_t)bbytes && y < x + (uintptr_t)abytes;
}

// A run of memory that a call reads or writes; none where `at` is NULL
struct Span {
    const void* at;
    int64_t bytes;
};
bool overlaps_any(Span out, std::initializer_list<Span> others) {
    for (const Span& x : others)
        if (x.at != nullptr && out.at != nullptr && overlap(out.at, out.bytes, x.at, x.bytes)) return true;
    return false;
}

// The struct as the kernels take it, for one layer (layer >= 0) or all of them (-1).
int take_cache(const flashd_cache* c, int layer, const int* q_start, int T, Paged& p) {
    if (!c || !c->k || !c->v || !c->table || !c->lens) return FLASHD_E_NULL;
    if (c->B < 1 || c->B > FLASHD_CACHE_MAX_SEQS || c->P < 1 || c->P > 1000000000 || c->layers < 1 ||
        c->layers > 65535 || c->Hkv < 1 || c->Hkv > 65535 || c->max_pages < 1)
        return FLASHD_E_SHAPE;
    if (c->dtype < FLASHD_F32 || c->dtype > FLASHD_CACHE_FP8) return FLASHD_E_DTYPE;
    if (c->d != 64 && c->d != 128) return FLASHD_E_HEADDIM;
    int log2 = 4;
    while (log2 < 8 && (1 << log2) < c->page) ++log2;
    if ((1 << log2) != c->page) return FLASHD_E_CACHE;
    if ((int64_t)c->max_pages * c->page > 1000000000 || (int64_t)c->B * c->max_pages > 0x7fffffff) return FLASHD_E_SHAPE;
    if (layer >= c->layers || layer < -1) return FLASHD_E_CACHE;
    // pages and layers lie apart: the layers of a page next to each other, or the pages of a layer
    const int64_t most = 1000000000000, one = (int64_t)c->Hkv * c->page * c->d;
    const int64_t ps = c->page_stride, ls = c->layers > 1 ? c->layer_stride : 0;
    if (ps < one || ps > most || ls < 0 || ls > most) return FLASHD_E_CACHE;
    if ((long double)ps * c->P + (long double)ls * c->layers > 1.0e12L) return FLASHD_E_SHAPE;
    if (c->layers > 1 && ls < (c->P - 1) * ps + one && (ls < one || ps < (c->layers - 1) * ls + one))
        return FLASHD_E_CACHE;
    const int esz = esize(c->dtype);
    if ((((uintptr_t)c->k | (uintptr_t)c->v) & 15u) != 0 || ((ps * esz) & 15) != 0 || ((ls * esz) & 15) != 0 ||
        (((uintptr_t)c->table | (uintptr_t)c->lens | (uintptr_t)q_start) & 3u) != 0)
        return FLASHD_E_ALIGN;
    const int64_t at = layer > 0 ? layer * ls * esz : 0;
    p.k = static_cast<char*>(c->k) + at;
    p.v = static_cast<char*>(c->v) + at;
    p.table = c->table;
    p.lens = c->lens;
    p.q_start = q_start;
    p.page_bytes = ps * esz;
    p.layer_bytes = ls * esz;
    p.head_bytes = (int64_t)c->page * c->d * esz;
    p.layers = c->layers;
    p.P = c->P;
    p.page_log2 = log2;
    p.max_pages = c->max_pages;
    p.B = c->B;
    p.Hkv = c->Hkv;
    p.d = c->d;
    p.esz = esz;
    p.T = T;
    p.kscale = c->kscale;
    p.vscale = c->vscale;
    return FLASHD_OK;
}

// The packed tensors' part: T rows of Hq heads, and their storage type against the cache's.
int take_rows(const flashd_cache* c, int T, int Hq, int dtype) {
    if (T < 0 || T > 10000000 || Hq < 1 || Hq > 65535 || (int64_t)T * Hq > 0x7fffffff) return FLASHD_E_SHAPE;
    if (dtype != FLASHD_F32 && dtype != FLASHD_F16 && dtype != FLASHD_BF16) return FLASHD_E_DTYPE;
    if (Hq % c->Hkv != 0) return FLASHD_E_GQA;
    if (c->dtype == FLASHD_CACHE_FP8 ? dtype == FLASHD_F32 : dtype != c->dtype) return FLASHD_E_VARIANT;
    return FLASHD_OK;
}

// Rows of `heads` heads, `stride` elements apart
int take_stride(long long stride, int T, int heads, int d, int dtype) {
    if (stride < (long long)heads * d || stride > 1000000000000 || (long double)stride * T > 1.0e12L) return FLASHD_E_SHAPE;
    return ((stride * esize(dtype)) & 15) != 0 ? FLASHD_E_ALIGN : FLASHD_OK;
}

int64_t extent(long long stride, int T, int heads, int d, int dtype) {
    return T < 1 ? 0 : ((int64_t)(T - 1) * stride + (int64_t)heads * d) * esize(dtype);
}

// bytes from the first element of a pool to behind its last
int64_t pool_extent(const Paged& p) {
    return (int64_t)(p.P - 1) * p.page_bytes + (int64_t)(p.layers - 1) * p.layer_bytes + (int64_t)p.Hkv * p.head_bytes;
}

int64_t layer_extent(const Paged& p) { return pool_extent(p) - (p.layers - 1) * p.layer_bytes; }

Span table_of(const Paged& p) { return {p.table, (int64_t)p.B * p.max_pages * 4}; }
Span lens_of(const Paged& p) { return {p.lens, (int64_t)p.B * 4}; }
Span starts_of(const Paged& p) { return {p.q_start, (int64_t)(p.B + 1) * 4}; }

// Whether rows of abytes at a share memory with rows of bbytes at b, both `stride` bytes apart, T of each
bool rows_overlap(const void* a, int64_t abytes, const void* b, int64_t bbytes, int64_t stride, int T) {
    if (!overlap(a, (T - 1) * stride + abytes, b, (T - 1) * stride + bbytes)) return false;
    const int64_t off = (int64_t)((uintptr_t)b - (uintptr_t)a) % stride, at = off < 0 ? off + stride : off;
    return T == 1 || at < abytes || at + bbytes > stride;
}

// Whether a page of K shares memory with one of V: page (l', p') of V lies off + (l' - l) layer_bytes + (p' - p) page_bytes behind page
// (l, p) of K.  Where one stride is a multiple of the other, as a rule, all of them lie at one remainder of the smaller one, which may
// settle it.  Else the difference with fewer values is gone through, and the other's nearest to the middle looked at (0.7 us with 80 layers).
bool kv_overlap(const Paged& p) {
    if (!overlap(p.k, pool_extent(p), p.v, pool_extent(p))) return false;
    const int64_t one = p.Hkv * p.head_bytes, off = (int64_t)((uintptr_t)p.v - (uintptr_t)p.k);
    const int64_t small = p.layers > 1 && p.layer_bytes < p.page_bytes ? p.layer_bytes : p.page_bytes;
    if (p.layers == 1 || (p.layer_bytes + p.page_bytes) % small == 0) {
        const int64_t at = (off % small + small) % small;
        if (at >= one && at <= small - one) return false;
    }
    const bool by_layer = p.layers <= p.P;
    const int64_t outer = by_layer ? p.layer_bytes : p.page_bytes, inner = by_layer ? p.page_bytes : p.layer_bytes;
    const int64_t most = (by_layer ? p.layers : p.P) - 1, last = (by_layer ? p.P : p.layers) - 1;
    for (int64_t d = -most; d <= most; ++d) {
        const int64_t rest = off + d * outer;
        if (rest - last * inner >= one || rest + last * inner <= -one) continue;
        const int64_t near = last == 0 ? 0 : -rest / inner;
        for (int64_t e = near - 1; e <= near + 1; ++e) {
            if (e < -last || e > last) continue;
            const int64_t gap = rest + e * inner;
            if (gap < one && gap > -one) return true;
        }
    }
    return false;
}

// Scores [(layers)][B][Hkv][stride]: a row has room for every key of a sequence.
int take_scores(const flashd_cache* c, long long stride) {
    const long long most = 1000000000000;
    return stride < (long long)c->max_pages * c->page || stride > most || (long double)stride * c->B * c->Hkv > 1.0e12L ? FLASHD_E_SHAPE
                                                                                                                     : FLASHD_OK;
}
// bytes from the first score of a layer to behind the last
int64_t score_extent(const flashd_cache* c, long long stride) {
    return (((int64_t)c->B * c->Hkv - 1) * stride + (int64_t)c->max_pages * c->page) * 4;
}

// Where the caller has brought no workspace: the stream's.
int stream_workspace(void* stream, size_t need, void** workspace) {
    if (*workspace != nullptr) return FLASHD_OK;
    // A graph would keep the stream's buffer, which other graphs and calls use as well.
    hipStreamCaptureStatus capturing = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(static_cast<hipStream_t>(stream), &capturing) != hipSuccess) (void)hipGetLastError();
    if (capturing != hipStreamCaptureStatusNone) return FLASHD_E_WORKSPACE;
    return flashd::api_cached_workspace(stream, (need + 255) & ~(size_t)255, workspace);
}

int done(hipError_t e) { return e == hipSuccess ? FLASHD_OK : FLASHD_E_HIP; }

int attn_fwd_tree(const flashd_cache* c, int layer, const void* q, long long q_stride, void* o, long long o_stride, int T, int max_q,
                  int Hq, const int* q_start, const unsigned long long* tree, int tree_words, float scale, int dtype, float* lse,
                  void* stream, void* workspace, size_t workspace_bytes) {
    Paged p;
    if (!q || !o || !q_start) return FLASHD_E_NULL;
    if (layer < 0) return FLASHD_E_CACHE;
    int rc = take_cache(c, layer, q_start, T, p);
    if (rc == FLASHD_OK) rc = take_rows(c, T, Hq, dtype);
    if (rc != FLASHD_OK) return rc;
    if (max_q < 1 || (tree && (tree_words < 1 || tree_words > 1000000))) return FLASHD_E_SHAPE;
    rc = take_stride(q_stride, T, Hq, c->d, dtype);
    if (rc == FLASHD_OK) rc = take_stride(o_stride, T, Hq, c->d, dtype);
    if (rc != FLASHD_OK) return rc;
    if ((((uintptr_t)q | (uintptr_t)o | (uintptr_t)workspace) & 15u) != 0 || ((uintptr_t)tree & 7u) != 0 || ((uintptr_t)lse & 3u) != 0)
        return FLASHD_E_ALIGN;
    const size_t need = flashd::attn_tree_workspace(Hq, c->Hkv, max_q, c->d, dtype);
    const Span out{o, extent(o_stride, T, Hq, c->d, dtype)}, in{q, extent(q_stride, T, Hq, c->d, dtype)}, kp{p.k, layer_extent(p)},
        vp{p.v, layer_extent(p)}, table = table_of(p), lens = lens_of(p), starts = starts_of(p), bits{tree, (int64_t)T * tree_words * 8},
        sums{lse, (int64_t)T * Hq * 4};
    if (overlaps_any(out, {in, kp, vp, table, lens, starts, bits, sums}) || overlaps_any(sums, {in, kp, vp, table, lens, starts, bits}))
        return FLASHD_E_OVERLAP;
    if (workspace != nullptr && workspace_bytes < need) return FLASHD_E_WORKSPACE;
    if (overlaps_any({workspace, (int64_t)need}, {out, in, kp, vp, table, lens, starts, bits, sums})) return FLASHD_E_OVERLAP;
    rc = flashd::api_check_arch();
    if (rc != FLASHD_OK || T == 0) return rc;
    rc = stream_workspace(stream, need, &workspace);
    if (rc != FLASHD_OK) return rc;
    TreeArgs a;
    a.q = q;
    a.o = o;
    a.tree = reinterpret_cast<const uint32_t*>(tree);
    a.q_stride = q_stride;
    a.o_stride = o_stride;
    a.words = tree != nullptr ? 2 * tree_words : 0;
    a.Hq = Hq;
    a.max_q = max_q;
    a.dtype = dtype;
    a.fp8 = c->dtype == FLASHD_CACHE_FP8;
    a.scale = scale;
    a.ws = static_cast<float*>(workspace);
    a.lse = lse;
    return done(flashd::launch_attn_tree(p, a, static_cast<hipStream_t>(stream)));
}

}  // namespace

extern "C" {

int flashd_cache_fork(const flashd_cache* c, int* refs, const int* parent, int B_out, int* table_out,
                      int* lens_out, void* stream) {
    Paged p;
    if (!refs || !parent || !table_out || !lens_out) return FLASHD_E_NULL;
    int rc = take_cache(c, -1, nullptr, 0, p);
    if (rc != FLASHD_OK) return rc;
    if (B_out < 1 || B_out > FLASHD_CACHE_MAX_SEQS || (int64_t)B_out * c->max_pages > 0x7fffffff) return FLASHD_E_SHAPE;
    if (((uintptr_t)refs | (uintptr_t)parent | (uintptr_t)table_out | (uintptr_t)lens_out) & 3u) return FLASHD_E_ALIGN;
    const Span r{refs, (int64_t)c->P * 4}, out{table_out, (int64_t)B_out * c->max_pages * 4}, lens{lens_out, (int64_t)B_out * 4};
    const Span from{parent, (int64_t)B_out * 4}, old = table_of(p), old_lens = lens_of(p);
    if (overlaps_any(r, {out, lens, from, old, old_lens}) || overlaps_any(out, {lens, from, old, old_lens}) ||
        overlaps_any(lens, {from, old, old_lens}))
        return FLASHD_E_OVERLAP;
    rc = flashd::api_check_arch();
    if (rc != FLASHD_OK) return rc;
    return done(flashd::launch_cache_fork(p, refs, parent, B_out, table_out, lens_out, static_cast<hipStream_t>(stream)));
}

int flashd_cache_reserve(const flashd_cache* c, int* refs, const int* q_start, int* report, void* stream) {
    Paged p;
    if (!refs || !q_start || !report) return FLASHD_E_NULL;
    int rc = take_cache(c, -1, q_start, 0x7fffffff, p);
    if (rc != FLASHD_OK) return rc;
    if (((uintptr_t)refs | (uintptr_t)report) & 3u) return FLASHD_E_ALIGN;
    const Span r{refs, (int64_t)c->P * 4}, rep{report, (int64_t)(c->B + 1) * 4}, table = table_of(p), lens = lens_of(p), starts = starts_of(p);
    if (overlaps_any(rep, {r, table, lens, starts}) || overlaps_any(r, {table, lens, starts}) || overlaps_any(table, {lens, starts}))
        return FLASHD_E_OVERLAP;
    for (const void* pool : {p.k, p.v})
        if (overlaps_any({pool, pool_extent(p)}, {r, rep, table, lens, starts})) return FLASHD_E_OVERLAP;
    if (kv_overlap(p)) return FLASHD_E_OVERLAP;
    rc = flashd::api_check_arch();
    if (rc != FLASHD_OK) return rc;
    return done(flashd::launch_cache_reserve(p, refs, report, static_cast<hipStream_t>(stream)));
}

int flashd_cache_append(const flashd_cache* c, int layer, const void* q, long long q_stride, const void* k,
                        long long k_stride, const void* v, long long v_stride, void* q_out,
                        long long q_out_stride, int T, int Hq, const int* q_start, const int* positions,
                        const float* inv_freq, int rot, int interleaved, const void* q_weight,
                        const void* k_weight, float eps, int dtype, void* stream) {
    Paged p;
    if (!q || !k || !v || !q_out || !q_start || (rot > 0 && !inv_freq)) return FLASHD_E_NULL;
    if (layer < 0) return FLASHD_E_CACHE;
    int rc = take_cache(c, layer, q_start, T, p);
    if (rc == FLASHD_OK) rc = take_rows(c, T, Hq, dtype);
    if (rc != FLASHD_OK) return rc;
    if (rot < 0 || rot > c->d || rot % 16 != 0) return FLASHD_E_SHAPE;
    const long long strides[4] = {q_stride, k_stride, v_stride, q_out_stride};
    for (int i = 0; i < 4; ++i) {
        rc = take_stride(strides[i], T, i == 0 || i == 3 ? Hq : c->Hkv, c->d, dtype);
        if (rc != FLASHD_OK) return rc;
    }
    if ((((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)q_out | (uintptr_t)q_weight | (uintptr_t)k_weight) & 15u) != 0 ||
        (((uintptr_t)positions | (uintptr_t)inv_freq) & 3u) != 0)
        return FLASHD_E_ALIGN;
    const int64_t nq = extent(q_stride, T, Hq, c->d, dtype), nk = extent(k_stride, T, c->Hkv, c->d, dtype),
                  nv = extent(v_stride, T, c->Hkv, c->d, dtype), no = extent(q_out_stride, T, Hq, c->d, dtype);
    // Tokens of k and v may lie between those of q (one projection's output), so q_out in place of q
    // may share their range, but not their elements; other outputs may not.
    const bool in_place = q_out == q && q_out_stride == q_stride;
    if (in_place && T > 0) {
        const int es = esize(dtype);
        const int64_t qb = (int64_t)Hq * c->d * es, kb = (int64_t)c->Hkv * c->d * es;
        // (tokens of another stride than q's: not between them)
        if (k_stride == q_stride ? rows_overlap(q, qb, k, kb, q_stride * es, T) : overlap(q, nq, k, nk)) return FLASHD_E_OVERLAP;
        if (v_stride == q_stride ? rows_overlap(q, qb, v, kb, q_stride * es, T) : overlap(q, nq, v, nv)) return FLASHD_E_OVERLAP;
    }
    if (!in_place && (overlap(q_out, no, q, nq) || overlap(q_out, no, k, nk) || overlap(q_out, no, v, nv))) return FLASHD_E_OVERLAP;
    const int64_t weights = (int64_t)c->d * esize(dtype);
    const Span table = table_of(p), lens = lens_of(p), starts = starts_of(p), at{positions, (int64_t)T * 4}, inv{inv_freq, (int64_t)rot * 2},
               qw{q_weight, weights}, kw{k_weight, weights};
    if (overlaps_any({q_out, no}, {table, lens, starts, at, inv, qw, kw})) return FLASHD_E_OVERLAP;
    for (const void* pool : {p.k, p.v})
        if (overlaps_any({pool, layer_extent(p)}, {{q, nq}, {k, nk}, {v, nv}, {q_out, no}, table, lens, starts, at, inv, qw, kw}))
            return FLASHD_E_OVERLAP;
    if (kv_overlap(p)) return FLASHD_E_OVERLAP;
    rc = flashd::api_check_arch();
    if (rc != FLASHD_OK || T == 0) return rc;
    AppendArgs a;
    a.q = q; a.k = k; a.v = v; a.q_out = q_out;
    a.positions = positions;
    a.inv_freq = inv_freq;
    a.q_weight = q_weight; a.k_weight = k_weight;
    a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride; a.qo_stride = q_out_stride;
    a.Hq = Hq;
    a.rot = rot;
    a.interleaved = interleaved != 0;
    a.dtype = dtype;
    a.fp8 = c->dtype == FLASHD_CACHE_FP8;
    a.eps = eps;
    return done(flashd::launch_cache_append(p, a, static_cast<hipStream_t>(stream)));
}

size_t flashd_tree_workspace_bytes(int Hq, int Hkv, int max_q, int d, int dtype) {
    if (Hq < 1 || Hkv < 1 || Hq > 65535 || Hkv > 65535 || Hq % Hkv != 0 || max_q < 1 || (d != 64 && d != 128) ||
        dtype < FLASHD_F32 || dtype > FLASHD_BF16)
        return 0;
    return flashd::attn_tree_workspace(Hq, Hkv, max_q, d, dtype);
}

int flashd_attn_fwd_tree(const flashd_cache* c, int layer, const void* q, long long q_stride, void* o,
                         long long o_stride, int T, int max_q, int Hq, const int* q_start,
                         const unsigned long long* tree, int tree_words, float scale, int dtype,
                         void* stream, void* workspace, size_t workspace_bytes) {
    return attn_fwd_tree(c, layer, q, q_stride, o, o_stride, T, max_q, Hq, q_start, tree, tree_words, scale, dtype, nullptr, stream,
                         workspace, workspace_bytes);
}

int flashd_attn_fwd_tree_lse(const flashd_cache* c, int layer, const void* q, long long q_stride, void* o,
                             long long o_stride, int T, int max_q, int Hq, const int* q_start,
                             const unsigned long long* tree, int tree_words, float scale, int dtype, float* lse,
                             void* stream, void* workspace, size_t workspace_bytes) {
    if (!lse) return FLASHD_E_NULL;
    return attn_fwd_tree(c, layer, q, q_stride, o, o_stride, T, max_q, Hq, q_start, tree, tree_words, scale, dtype, lse, stream,
                         workspace, workspace_bytes);
}

int flashd_cache_commit(const flashd_cache* c, const int* q_start, const int* keep, int max_keep,
                        const int* n_keep, int* lens_out, void* stream) {
    Paged p;
    if (!q_start || !lens_out) return FLASHD_E_NULL;
    int rc = take_cache(c, -1, q_start, 0x7fffffff, p);
    if (rc != FLASHD_OK) return rc;
    if (keep != nullptr ? max_keep < 1 || (int64_t)max_keep * c->B > 0x7fffffff : max_keep != 0) return FLASHD_E_SHAPE;
    if (((uintptr_t)keep | (uintptr_t)n_keep | (uintptr_t)lens_out) & 3u) return FLASHD_E_ALIGN;
    const Span out{lens_out, (int64_t)c->B * 4}, table = table_of(p), lens = lens_of(p), starts = starts_of(p),
        list{keep, (int64_t)c->B * max_keep * 4}, counts{n_keep, (int64_t)c->B * 4};
    if (overlaps_any(out, {table, lens, starts, list, counts})) return FLASHD_E_OVERLAP;
    for (const void* pool : {p.k, p.v})
        if (overlaps_any({pool, pool_extent(p)}, {out, table, lens, starts, list, counts})) return FLASHD_E_OVERLAP;
    if (kv_overlap(p)) return FLASHD_E_OVERLAP;
    rc = flashd::api_check_arch();
    if (rc != FLASHD_OK) return rc;
    return done(flashd::launch_cache_commit(p, keep, max_keep, n_keep, lens_out, static_cast<hipStream_t>(stream)));
}

int flashd_cache_score(const flashd_cache* c, int layer, const void* q, long long q_stride, int T, int Hq, const int* q_start,
                       const unsigned long long* tree, int tree_words, const float* lse, const float* row_weight, float scale,
                       int dtype, float* score, long long score_stride, float decay, void* stream) {
    Paged p;
    if (!q || !q_start || !lse || !score) return FLASHD_E_NULL;
    if (layer < 0) return FLASHD_E_CACHE;
    int rc = take_cache(c, layer, q_start, T, p);
    if (rc == FLASHD_OK) rc = take_rows(c, T, Hq, dtype);
    if (rc != FLASHD_OK) return rc;
    if (tree && (tree_words < 1 || tree_words > 1000000)) return FLASHD_E_SHAPE;
    rc = take_stride(q_stride, T, Hq, c->d, dtype);
    if (rc == FLASHD_OK) rc = take_scores(c, score_stride);
    if (rc != FLASHD_OK) return rc;
    if (((uintptr_t)q & 15u) != 0 || ((uintptr_t)tree & 7u) != 0 ||
        (((uintptr_t)lse | (uintptr_t)row_weight | (uintptr_t)score) & 3u) != 0)
        return FLASHD_E_ALIGN;
    const Span out{score, score_extent(c, score_stride)};
    if (overlaps_any(out, {{q, extent(q_stride, T, Hq, c->d, dtype)}, {p.k, layer_extent(p)}, table_of(p), lens_of(p), starts_of(p),
                           {tree, (int64_t)T * tree_words * 8}, {lse, (int64_t)T * Hq * 4}, {row_weight, (int64_t)T * 4}}))
        return FLASHD_E_OVERLAP;
    rc = flashd::api_check_arch();
    if (rc != FLASHD_OK || T == 0) return rc;
    ScoreArgs a;
    a.q = q;
    a.tree = reinterpret_cast<const uint32_t*>(tree);
    a.lse = lse;
    a.weight = row_weight;
    a.score = score;
    a.q_stride = q_stride;
    a.score_stride = score_stride;
    a.words = tree != nullptr ? 2 * tree_words : 0;
    a.Hq = Hq;
    a.dtype = dtype;
    a.fp8 = c->dtype == FLASHD_CACHE_FP8;
    a.scale = scale;
    a.decay = decay;
    return done(flashd::launch_cache_score(p, a, static_cast<hipStream_t>(stream)));
}

size_t flashd_evict_workspace_bytes(const flashd_cache* c, int budget) {
    Paged p;
    if (take_cache(c, -1, nullptr, 0, p) != FLASHD_OK || (int64_t)c->B * c->Hkv > flashd::kEvictMostUnits || budget < 0) return 0;
    return flashd::evict_workspace(p, budget);
}

int flashd_cache_evict(const flashd_cache* c, const int* refs, float* score, long long score_stride, long long score_layer_stride,
                       int budget, const int* budgets, int first, int recent, int* lens_out, void* stream, void* workspace,
                       size_t workspace_bytes) {
    Paged p;
    if (!refs || !score || !lens_out) return FLASHD_E_NULL;
    int rc = take_cache(c, -1, nullptr, 0, p);
    if (rc == FLASHD_OK) rc = take_scores(c, score_stride);
    if (rc != FLASHD_OK) return rc;
    if (budget < 0 || first < 0 || recent < 0 || (int64_t)c->B * c->Hkv > flashd::kEvictMostUnits) return FLASHD_E_SHAPE;
    const int64_t of_layer = (int64_t)c->B * c->Hkv * score_stride, layer = c->layers > 1 ? score_layer_stride : 0;
    if (c->layers > 1 && (layer < of_layer || layer > 1000000000000 || (long double)layer * c->layers > 1.0e12L)) return FLASHD_E_SHAPE;
    if ((((uintptr_t)refs | (uintptr_t)score | (uintptr_t)budgets | (uintptr_t)lens_out) & 3u) != 0 || ((uintptr_t)workspace & 15u) != 0)
        return FLASHD_E_ALIGN;
    const size_t need = flashd::evict_workspace(p, budget);
    if (workspace != nullptr && workspace_bytes < need) return FLASHD_E_WORKSPACE;
    const Span out{lens_out, (int64_t)c->B * 4}, scores{score, (c->layers - 1) * layer * 4 + score_extent(c, score_stride)}, ws{workspace, (int64_t)need},
        table = table_of(p), lens = lens_of(p), counts{refs, (int64_t)c->P * 4}, most{budgets, (int64_t)c->B * 4};
    if (overlaps_any(out, {scores, ws, table, lens, counts, most}) || overlaps_any(scores, {ws, table, lens, counts, most}) ||
        overlaps_any(ws, {table, lens, counts, most}))
        return FLASHD_E_OVERLAP;
    for (const void* pool : {p.k, p.v})
        if (overlaps_any({pool, pool_extent(p)}, {out, scores, ws, table, lens, counts, most})) return FLASHD_E_OVERLAP;
    if (kv_overlap(p)) return FLASHD_E_OVERLAP;
    rc = flashd::api_check_arch();
    if (rc == FLASHD_OK) rc = stream_workspace(stream, need, &workspace);
    if (rc != FLASHD_OK) return rc;
    EvictArgs a;
    a.refs = refs;
    a.budgets = budgets;
    a.score = score;
    a.score_stride = score_stride;
    a.score_layer_stride = layer;
    a.budget = budget;
    a.first = first;
    a.recent = recent;
    a.lens_out = lens_out;
    return done(flashd::launch_cache_evict(p, a, workspace, static_cast<hipStream_t>(stream)));
}

size_t flashd_verify_workspace_bytes(int T, int V) {
    if (T < 0 || T > 10000000 || V < 1 || V > FLASHD_VERIFY_MAX_V) return 0;
    return flashd::verify_workspace(T, V);
}

int flashd_draft_verify(const void* logits, long long logits_stride, const void* draft, long long draft_stride,
                        const int* tokens, const int* parent, const float* uniform, const float* temperature,
                        const int* q_start, int B, int T, int V, int dtype, int draft_dtype, int max_keep, int* keep,
                        int* n_keep, int* next, void* stream, void* workspace, size_t workspace_bytes) {
    if (!logits || !tokens || !uniform || !q_start || !keep || !n_keep || !next) return FLASHD_E_NULL;
    if (B < 1 || B > FLASHD_CACHE_MAX_SEQS || T < 0 || T > 10000000 || V < 1 || V > FLASHD_VERIFY_MAX_V || max_keep < 1 ||
        (int64_t)max_keep * B > 0x7fffffff)
        return FLASHD_E_SHAPE;
    if (dtype < FLASHD_F32 || dtype > FLASHD_BF16 || (draft && (draft_dtype < FLASHD_F32 || draft_dtype > FLASHD_BF16)))
        return FLASHD_E_DTYPE;
    const long long most = 1000000000000;
    if (logits_stride < V || logits_stride > most || (long double)logits_stride * T > 1.0e12L) return FLASHD_E_SHAPE;
    if (draft && (draft_stride < V || draft_stride > most || (long double)draft_stride * T > 1.0e12L)) return FLASHD_E_SHAPE;
    const int esz = esize(dtype), dsz = draft ? esize(draft_dtype) : 4;
    if ((uintptr_t)logits % esz != 0 || (uintptr_t)draft % dsz != 0 || ((uintptr_t)workspace & 15u) != 0 ||
        (((uintptr_t)tokens | (uintptr_t)parent | (uintptr_t)uniform | (uintptr_t)temperature | (uintptr_t)q_start | (uintptr_t)keep |
          (uintptr_t)n_keep | (uintptr_t)next) & 3u) != 0)
        return FLASHD_E_ALIGN;
    const size_t need = flashd::verify_workspace(T, V);
    if (workspace != nullptr && workspace_bytes < need) return FLASHD_E_WORKSPACE;
    const Span rows{logits, extent(logits_stride, T, 1, V, dtype)}, drafts{draft, draft ? extent(draft_stride, T, 1, V, draft_dtype) : 0},
        ids{tokens, (int64_t)T * 4}, from{parent, (int64_t)T * 4}, u{uniform, (int64_t)T * 4}, heat{temperature, (int64_t)B * 4},
        starts{q_start, (int64_t)(B + 1) * 4}, kept{keep, (int64_t)B * max_keep * 4}, counts{n_keep, (int64_t)B * 4}, then{next, (int64_t)B * 4};
    if (overlaps_any(kept, {rows, drafts, ids, from, u, heat, starts, counts, then}) ||
        overlaps_any(counts, {rows, drafts, ids, from, u, heat, starts, then}) || overlaps_any(then, {rows, drafts, ids, from, u, heat, starts}) ||
        overlaps_any({workspace, (int64_t)need}, {rows, drafts, ids, from, u, heat, starts, kept, counts, then}))
        return FLASHD_E_OVERLAP;
    int rc = flashd::api_check_arch();
    if (rc != FLASHD_OK) return rc;
    if (T > 0) rc = stream_workspace(stream, need, &workspace);
    if (rc != FLASHD_OK) return rc;
    VerifyArgs a;
    a.logits = logits;
    a.draft = draft;
    a.tokens = tokens;
    a.parent = parent;
    a.uniform = uniform;
    a.temperature = temperature;
    a.q_start = q_start;
    a.keep = keep;
    a.n_keep = n_keep;
    a.next = next;
    a.logits_stride = logits_stride;
    a.draft_stride = draft ? draft_stride : 0;
    a.B = B;
    a.T = T;
    a.V = V;
    a.dtype = dtype;
    a.draft_dtype = draft ? draft_dtype : FLASHD_F32;
    a.max_keep = max_keep;
    return done(flashd::launch_verify(a, workspace, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
