// C-ABI entry points of the paged cache: argument validation and dispatch.
// Every check runs before the first enqueue; on error nothing is launched and
// the outputs are untouched.
#include <math.h>

#include "../../include/mot.h"
#include "api_common.h"
#include "cache_internal.h"

using namespace mot;

namespace {

mot_status check_cache(const mot_cache_shapes* c) {
    if (!c) return fail(MOT_ERR_NULL_ARG, "cache is NULL");
    if (c->L < 1 || c->L > MOT_MAX_LAYERS)
        return fail(MOT_ERR_BAD_SHAPE, "L=%d must be in [1, %d]", c->L, MOT_MAX_LAYERS);
    if (c->n_pages < 1 || c->n_pages > 1 << 30)
        return fail(MOT_ERR_BAD_SHAPE, "n_pages=%d must be in [1, 2^30]", c->n_pages);
    if (c->B < 0 || c->B > 65535 || c->max_pages < 1)
        return fail(MOT_ERR_BAD_SHAPE, "B=%d max_pages=%d: need B in [0, 65535] and max_pages >= 1", c->B, c->max_pages);
    if (c->H_kv < 1 || c->D < 1 || (int64_t)c->H_kv * c->D > 65536)
        return fail(MOT_ERR_BAD_SHAPE, "H_kv=%d D=%d must be >= 1 and rows at most 65536 wide", c->H_kv, c->D);
    if (c->dtype != MOT_F32 && c->dtype != MOT_BF16)
        return fail(MOT_ERR_BAD_SHAPE, "dtype=%d is not MOT_F32 or MOT_BF16", c->dtype);
    if (c->page_layout != MOT_LAYOUT_BTHD && c->page_layout != MOT_LAYOUT_BHTD)
        return fail(MOT_ERR_BAD_SHAPE, "page_layout must be MOT_LAYOUT_BTHD or MOT_LAYOUT_BHTD");
    if (c->page_size < 1) return fail(MOT_ERR_BAD_SHAPE, "page_size=%d must be >= 1", c->page_size);
    if (c->page_size < 16 || c->page_size > 1024 || (c->page_size & (c->page_size - 1)))
        return fail(MOT_ERR_UNSUPPORTED, "page_size=%d: need a power of two from 16 to 1024", c->page_size);
    if ((int64_t)c->max_pages * c->page_size > 1 << 30 || (int64_t)c->B * c->max_pages > 1 << 30)
        return fail(MOT_ERR_BAD_SHAPE, "max_pages=%d: at most 2^30 positions per row and 2^30 entries", c->max_pages);
    if (c->D % 16 || c->D > 256)
        return fail(MOT_ERR_UNSUPPORTED, "D=%d: need a multiple of 16 up to 256", c->D);
    return MOT_OK;
}

size_t elem(const mot_cache_shapes* c) { return c->dtype == MOT_BF16 ? 2 : 4; }

// Bytes of a layer's pool of keys or values (a page is under 2 GiB: at most
// 1024 x 65536 x 4 bytes = 256 MiB)
size_t pool_bytes(const mot_cache_shapes* c) {
    return (size_t)c->n_pages * c->page_size * c->H_kv * c->D * elem(c);
}

PageTable page_table(const mot_cache_shapes* c) {
    PageTable t = {};
    t.B = c->B; t.max_pages = c->max_pages; t.n_pages = c->n_pages;
    t.page_shift = __builtin_ctz((unsigned)c->page_size);
    t.H_kv = c->H_kv; t.D = c->D;
    t.page_elems = (int64_t)c->page_size * c->H_kv * c->D;
    const bool heads_first = c->page_layout == MOT_LAYOUT_BHTD;
    t.ts = heads_first ? c->D : c->H_kv * c->D;
    t.hs = heads_first ? c->page_size * c->D : c->D;
    return t;
}

mot_status check_rows(const mot_cache_shapes* c, int n_new, int max_new, bool packed) {
    if (n_new < 0 || max_new < 0) return fail(MOT_ERR_BAD_SHAPE, "n_new=%d max_new=%d must be >= 0", n_new, max_new);
    if (n_new > 4 * kMostWorkgroups) return fail(MOT_ERR_BAD_SHAPE, "n_new=%d exceeds 2^26 - 32 tokens", n_new);
    if (max_new > n_new) return fail(MOT_ERR_BAD_SHAPE, "max_new=%d above n_new=%d", max_new, n_new);
    if (!packed && (int64_t)c->B * max_new != n_new)
        return fail(MOT_ERR_BAD_SHAPE, "n_new=%d is not B * max_new = %d * %d (no new_start)", n_new, c->B, max_new);
    return MOT_OK;
}

// Row tensor of `heads` heads: its strides are usable and its extent in bytes.
mot_status check_strides(const char* name, const mot_strides& s, const mot_cache_shapes* c, int n_new, int max_new,
                         int heads, int layers, bool packed, size_t* bytes) {
    const int64_t v[4] = {s.layer, s.batch, s.token, s.head}, m = c->dtype == MOT_BF16 ? 8 : 4;
    // an axis of one entry may have any stride
    const int64_t n[4] = {layers, packed ? 1 : c->B, packed ? n_new : max_new, heads};
    int64_t at = c->D;   // of the last element, and one
    double far = c->D;
    for (int i = 0; i < 4; ++i) {
        if (n[i] <= 1) continue;
        if (v[i] < 0 || v[i] > (int64_t)1 << 40) return fail(MOT_ERR_BAD_SHAPE, "a stride of %s is negative or above 2^40", name);
        if (v[i] % m) return fail(MOT_ERR_MISALIGNED, "a stride of %s is not a multiple of 16 bytes", name);
        far += (double)(n[i] - 1) * v[i];
        at += (n[i] - 1) * v[i];
    }
    if (far > 1e18) return fail(MOT_ERR_BAD_SHAPE, "%s spans more than the address space", name);
    *bytes = (size_t)at * elem(c);
    return MOT_OK;
}

// No two rows of an output share an element: from the smallest stride up, each
// passes over all that the smaller ones reach.
mot_status check_output(const char* name, const mot_strides& s, const mot_cache_shapes* c, int n_new, int max_new,
                        int heads, int layers, bool packed) {
    struct Axis {
        int64_t n, stride;
    } ax[4] = {{heads, s.head}, {packed ? n_new : max_new, s.token}, {packed ? 1 : c->B, s.batch}, {layers, s.layer}};
    int64_t reach = c->D;
    for (int done = 0; done < 4; ++done) {
        int best = -1;
        for (int i = 0; i < 4; ++i)
            if (ax[i].n > 1 && (best < 0 || ax[i].stride < ax[best].stride)) best = i;
        if (best < 0) break;
        if (ax[best].stride < reach) return fail(MOT_ERR_BAD_SHAPE, "rows of %s share elements", name);
        reach += (ax[best].n - 1) * ax[best].stride;
        ax[best].n = 1;
    }
    return MOT_OK;
}

RowStrides strides(const mot_strides& s) { return {s.layer, s.batch, s.token, s.head}; }

struct Extent {
    const char* name;
    const void* p;
    size_t bytes;
};
// `out` lies apart from every one of `others` (NULL entries hold nothing).
mot_status apart(const Extent& out, const Extent* others, int n) {
    for (int i = 0; i < n; ++i)
        if (others[i].p && out.p && overlaps(out.p, out.bytes, others[i].p, others[i].bytes))
            return fail(MOT_ERR_BAD_SHAPE, "%s overlaps %s", out.name, others[i].name);
    return MOT_OK;
}

// scale * log2(e)
float scale_log2(const mot_cache_shapes* c, const mot_attend_shapes* s) {
    return (float)((s->scale > 0.f ? (double)s->scale : 1.0 / sqrt((double)c->D)) * 1.4426950408889634);
}

mot_status check_attend(const mot_cache_shapes* c, const mot_attend_shapes* s, bool packed) {
    mot_status st = check_cache(c);
    if (st != MOT_OK) return st;
    if (!s) return fail(MOT_ERR_NULL_ARG, "shapes is NULL");
    if (c->L != 1) return fail(MOT_ERR_BAD_SHAPE, "L=%d: attention reads one layer's pools", c->L);
    st = check_rows(c, s->n_new, s->max_new, packed);
    if (st != MOT_OK) return st;
    if (s->H_q < 1 || s->H_q % c->H_kv || (int64_t)s->H_q * c->D > 1 << 20)
        return fail(MOT_ERR_BAD_SHAPE, "H_q=%d: need a positive multiple of H_kv=%d, rows up to 2^20 wide", s->H_q, c->H_kv);
    if ((int64_t)s->max_new * s->H_q > 1 << 30)
        return fail(MOT_ERR_BAD_SHAPE, "max_new=%d: more than 2^30 query rows of a sequence", s->max_new);
    if (s->window < 0 || s->max_kv < 0)
        return fail(MOT_ERR_BAD_SHAPE, "window=%d max_kv=%d must be >= 0", s->window, s->max_kv);
    // 0 * infinity would make rows of zeros NaN
    if (!(s->scale >= 0.f) || isinf(scale_log2(c, s)))
        return fail(MOT_ERR_BAD_SHAPE, "scale must be positive (0: 1 / sqrt(D)), scale * log2(e) a finite float");
    if (c->D != 64 && c->D != 128)
        return fail(MOT_ERR_UNSUPPORTED, "D=%d: paged attention supports head dims 64 and 128", c->D);
    return MOT_OK;
}

AttendProblem attend_problem(const mot_cache_shapes* c, const mot_attend_shapes* s) {
    AttendProblem p = {};
    p.c = page_table(c);
    p.c.n_new = s->n_new;
    p.c.max_new = s->max_new;
    p.H_q = s->H_q;
    const int most = c->max_pages * c->page_size;
    // A window of every position there can be is none.  Shorter ones are under 2^30, and new tokens
    // lie at -2^26 or later, so u - window fits in 32 bits.
    p.window = s->window < most ? s->window : 0;
    p.max_kv = s->max_kv > 0 && s->max_kv < most ? s->max_kv : most;
    p.scale_log2 = scale_log2(c, s);
    p.qs = strides(s->q);
    p.os = strides(s->o);
    return p;
}

mot_status launched(hipError_t e) {
    return e == hipSuccess ? MOT_OK : fail(MOT_ERR_HIP, "kernel launch: %s", hipGetErrorString(e));
}

}  // namespace

extern "C" {

size_t mot_attend_workspace_bytes(const mot_cache_shapes* c, const mot_attend_shapes* s) {
    clear_error();
    // packed or not, the same cuts: sizes that either form admits are taken
    if (check_attend(c, s, true) != MOT_OK) return SIZE_MAX;
    if (c->B == 0 || s->n_new == 0 || s->max_new == 0) return 0;
    AttendProblem p = attend_problem(c, s);
    return attend_plan(p, c->dtype == MOT_BF16);
}

mot_status mot_paged_attention(const void* q, const void* k_pages, const void* v_pages, const int32_t* table,
                               const int32_t* kv_len, const int32_t* new_start, void* o, const mot_cache_shapes* c,
                               const mot_attend_shapes* s, hipStream_t stream) {
    clear_error();
    const bool packed = new_start != nullptr;
    mot_status st = check_attend(c, s, packed);
    if (st != MOT_OK) return st;
    if (c->B == 0 || s->n_new == 0 || s->max_new == 0) return MOT_OK;
    if (!q || !k_pages || !v_pages || !table || !kv_len || !o)
        return fail(MOT_ERR_NULL_ARG, "q, the pools, the table, kv_len and o are required");
    for (const void* x : {q, k_pages, v_pages, (const void*)o})
        if (!aligned16(x)) return fail(MOT_ERR_MISALIGNED, "device pointer %p is not 16-byte aligned", x);
    for (const int32_t* x : {table, kv_len, new_start})
        if (!aligned4(x)) return fail(MOT_ERR_MISALIGNED, "device pointer %p is not 4-byte aligned", (const void*)x);
    size_t qb, ob;
    if ((st = check_strides("q", s->q, c, s->n_new, s->max_new, s->H_q, 1, packed, &qb)) != MOT_OK) return st;
    if ((st = check_strides("o", s->o, c, s->n_new, s->max_new, s->H_q, 1, packed, &ob)) != MOT_OK) return st;
    if ((st = check_output("o", s->o, c, s->n_new, s->max_new, s->H_q, 1, packed)) != MOT_OK) return st;
    const Extent in[] = {{"q", q, qb}, {"k_pages", k_pages, pool_bytes(c)}, {"v_pages", v_pages, pool_bytes(c)},
                         {"the table", table, (size_t)c->B * c->max_pages * 4}, {"kv_len", kv_len, (size_t)c->B * 4},
                         {"new_start", new_start, ((size_t)c->B + 1) * 4}, {"o", o, ob}};
    if ((st = apart(in[6], in, 6)) != MOT_OK) return st;
    AttendProblem p = attend_problem(c, s);
    p.q = q; p.k = k_pages; p.v = v_pages; p.o = o;
    p.c.table = table; p.c.kv_len = kv_len; p.c.start = new_start;
    const size_t need = attend_plan(p, c->dtype == MOT_BF16);
    if (need && s->workspace && s->workspace_bytes >= need) {
        if (!aligned16(s->workspace))
            return fail(MOT_ERR_MISALIGNED, "workspace %p is not 16-byte aligned", s->workspace);
        if ((st = apart({"workspace", s->workspace, need}, in, 7)) != MOT_OK) return st;
        p.part = reinterpret_cast<float*>(s->workspace);
    }
    if (!attend_fits(p, c->dtype == MOT_BF16))
        return fail(MOT_ERR_UNSUPPORTED, "more tiles of query rows than a launch holds (2^24 - 8 workgroups)");
    return launched(launch_paged_attention(p, c->dtype == MOT_BF16, stream));
}

mot_status mot_cache_append(const void* q, const void* k, const void* v, void* q_out, void* k_pages, void* v_pages,
                            const int32_t* table, const int32_t* kv_len, const int32_t* new_start,
                            const mot_rope* rope, const mot_cache_shapes* c, const mot_append_shapes* s,
                            hipStream_t stream) {
    clear_error();
    mot_status st = check_cache(c);
    if (st != MOT_OK) return st;
    if (!s) return fail(MOT_ERR_NULL_ARG, "shapes is NULL");
    const bool packed = new_start != nullptr;
    if ((st = check_rows(c, s->n_new, s->max_new, packed)) != MOT_OK) return st;
    const mot_rope none = {nullptr, nullptr, nullptr, nullptr};
    const mot_rope& r = rope ? *rope : none;
    const int rot = s->rotary_dim ? s->rotary_dim : c->D;
    if (rot < 0 || rot > c->D || rot % 16)
        return fail(MOT_ERR_BAD_SHAPE, "rotary_dim=%d: need a multiple of 16 up to D=%d", rot, c->D);
    if (s->interleaved != 0 && s->interleaved != 1) return fail(MOT_ERR_BAD_SHAPE, "interleaved=%d is not 0 or 1", s->interleaved);
    if (!(s->eps >= 0.f) || isinf(s->eps)) return fail(MOT_ERR_BAD_SHAPE, "eps must be >= 0 and finite");
    if ((q || q_out) && (s->H_q < 1 || (int64_t)s->H_q * c->D > 1 << 20))
        return fail(MOT_ERR_BAD_SHAPE, "H_q=%d must be >= 1, rows up to 2^20 wide", s->H_q);
    if (c->B == 0 || s->n_new == 0 || s->max_new == 0) return MOT_OK;
    if (!q != !q_out || !k != !v || (!q && !k))
        return fail(MOT_ERR_NULL_ARG, "q with q_out, k with v, and one pair at least");
    if (!kv_len || !table || (k && (!k_pages || !v_pages)))
        return fail(MOT_ERR_NULL_ARG, "the table, kv_len and, with k and v, the pools are required");
    for (const void* x : {q, k, v, (const void*)q_out, k ? (const void*)k_pages : nullptr, k ? (const void*)v_pages : nullptr,
                          r.q_gain, r.k_gain})
        if (!aligned16(x)) return fail(MOT_ERR_MISALIGNED, "device pointer %p is not 16-byte aligned", x);
    for (const void* x : {(const void*)table, (const void*)kv_len, (const void*)new_start, (const void*)r.inv_freq,
                          (const void*)r.positions})
        if (!aligned4(x)) return fail(MOT_ERR_MISALIGNED, "device pointer %p is not 4-byte aligned", x);
    size_t qb = 0, qob = 0, kb = 0, vb = 0;
    if (q && ((st = check_strides("q", s->q, c, s->n_new, s->max_new, s->H_q, c->L, packed, &qb)) != MOT_OK ||
              (st = check_strides("q_out", s->q_out, c, s->n_new, s->max_new, s->H_q, c->L, packed, &qob)) != MOT_OK ||
              (st = check_output("q_out", s->q_out, c, s->n_new, s->max_new, s->H_q, c->L, packed)) != MOT_OK))
        return st;
    if (k && ((st = check_strides("k", s->k, c, s->n_new, s->max_new, c->H_kv, c->L, packed, &kb)) != MOT_OK ||
              (st = check_strides("v", s->v, c, s->n_new, s->max_new, c->H_kv, c->L, packed, &vb)) != MOT_OK))
        return st;
    const bool same = q && q == q_out;
    if (same) {
        const mot_strides &a = s->q, &b = s->q_out;
        if ((c->L > 1 && a.layer != b.layer) || (!packed && c->B > 1 && a.batch != b.batch) ||
            ((packed ? s->n_new : s->max_new) > 1 && a.token != b.token) || (s->H_q > 1 && a.head != b.head))
            return fail(MOT_ERR_BAD_SHAPE, "q_out is q with other strides");
    }
    const size_t pb = k ? pool_bytes(c) * c->L : 0, gb = (size_t)c->L * c->D * elem(c);
    const Extent in[] = {{"k", k, kb}, {"v", v, vb}, {"q", q, qb}, {"the table", table, (size_t)c->B * c->max_pages * 4},
                         {"kv_len", kv_len, (size_t)c->B * 4}, {"new_start", new_start, ((size_t)c->B + 1) * 4},
                         {"q_gain", r.q_gain, gb}, {"k_gain", r.k_gain, gb}, {"inv_freq", r.inv_freq, (size_t)rot * 2},
                         {"positions", r.positions, (size_t)s->n_new * 4}};
    if (k) {
        const Extent kp = {"k_pages", k_pages, pb}, vp = {"v_pages", v_pages, pb};
        if ((st = apart(kp, in, 10)) != MOT_OK || (st = apart(vp, in, 10)) != MOT_OK || (st = apart(kp, &vp, 1)) != MOT_OK)
            return st;
    }
    if (q) {
        // in place, q may lie between k and v in one tensor; its rows are its own
        const Extent out = {"q_out", q_out, qob}, pools[] = {{"k_pages", k ? k_pages : nullptr, pb}, {"v_pages", k ? v_pages : nullptr, pb}};
        if ((st = apart(out, pools, 2)) != MOT_OK || (st = apart(out, in + 3, 7)) != MOT_OK) return st;
        if (!same && (st = apart(out, in, 3)) != MOT_OK) return st;
    }
    AppendProblem p = {};
    p.c = page_table(c);
    p.c.table = table; p.c.kv_len = kv_len; p.c.start = new_start;
    p.c.n_new = s->n_new; p.c.max_new = s->max_new;
    p.q = q; p.k = k; p.v = v; p.q_out = q_out; p.k_pages = k_pages; p.v_pages = v_pages;
    p.q_gain = r.q_gain; p.k_gain = r.k_gain; p.inv_freq = r.inv_freq; p.positions = r.positions;
    p.L = c->L; p.H_q = s->H_q; p.rot = rot; p.interleaved = s->interleaved; p.eps = s->eps;
    p.qs = strides(s->q); p.qos = strides(s->q_out); p.ks = strides(s->k); p.vs = strides(s->v);
    return launched(launch_cache_append(p, c->dtype == MOT_BF16, stream));
}

size_t mot_cache_workspace_bytes(const mot_cache_shapes* c, int32_t n_rows) {
    clear_error();
    if (check_cache(c) != MOT_OK) return SIZE_MAX;
    if (n_rows < 0 || n_rows > 4096) {
        fail(MOT_ERR_BAD_SHAPE, "n_rows=%d must be in [0, 4096]", n_rows);
        return SIZE_MAX;
    }
    return pages_workspace_bytes(c->n_pages, n_rows, n_rows ? n_rows : c->B, c->max_pages);
}

}  // extern "C"

namespace {

// Checks and launch that reordering and compaction share.
mot_status pages_call(void* k_pages, void* v_pages, const int32_t* table, const int32_t* source, const int32_t* keep,
                      const int32_t* want, int32_t* new_table, int32_t* count, const mot_cache_shapes* c, int32_t n_rows,
                      bool reorder, void* ws, size_t ws_bytes, hipStream_t stream) {
    if (!k_pages || !v_pages || !new_table || !count || (!table && c->B) || (reorder && (!source || !keep || !want)))
        return fail(MOT_ERR_NULL_ARG, "a required argument is NULL");
    const size_t need = pages_workspace_bytes(c->n_pages, reorder ? n_rows : 0, reorder ? n_rows : c->B, c->max_pages);
    if (need && !ws) return fail(MOT_ERR_NULL_ARG, "a workspace of %zu bytes is required", need);
    if (ws_bytes < need) return fail(MOT_ERR_WORKSPACE_TOO_SMALL, "workspace of %zu bytes, need %zu", ws_bytes, need);
    for (const void* x : {(const void*)k_pages, (const void*)v_pages, need ? (const void*)ws : nullptr})
        if (!aligned16(x)) return fail(MOT_ERR_MISALIGNED, "device pointer %p is not 16-byte aligned", x);
    for (const int32_t* x : {table, source, keep, want, (const int32_t*)new_table, (const int32_t*)count})
        if (!aligned4(x)) return fail(MOT_ERR_MISALIGNED, "device pointer %p is not 4-byte aligned", (const void*)x);
    const size_t rows = reorder ? n_rows : c->B, pb = pool_bytes(c) * c->L;
    const Extent all[] = {{"k_pages", k_pages, pb}, {"v_pages", v_pages, pb}, {"new_table", new_table, rows * c->max_pages * 4},
                          {"the count", count, 4}, {"workspace", ws, need},
                          {"the table", c->B ? table : nullptr, (size_t)c->B * c->max_pages * 4},
                          {"source", source, rows * 4}, {"keep", keep, rows * 4}, {"want", want, rows * 4}};
    for (int i = 0; i < 5; ++i) {   // what is written lies apart from everything after it
        const mot_status st = apart(all[i], all + i + 1, 8 - i);
        if (st != MOT_OK) return st;
    }
    PagesProblem p = {};
    p.c = page_table(c);
    p.c.table = table;
    p.k_pages = k_pages; p.v_pages = v_pages;
    p.source = source; p.keep = keep; p.want = want; p.new_table = new_table; p.count = count;
    p.L = c->L; p.n_rows = reorder ? n_rows : 0; p.elem_bytes = (int32_t)elem(c);
    p.heads_first = c->page_layout == MOT_LAYOUT_BHTD;
    p.ws = ws;
    return launched(reorder ? launch_cache_reorder(p, stream) : launch_cache_compact(p, stream));
}

}  // namespace

extern "C" {

mot_status mot_cache_reorder(void* k_pages, void* v_pages, const int32_t* table, const int32_t* source,
                             const int32_t* keep, const int32_t* want, int32_t* new_table, int32_t* missing,
                             const mot_cache_shapes* c, int32_t n_rows, void* workspace, size_t workspace_bytes,
                             hipStream_t stream) {
    clear_error();
    const mot_status st = check_cache(c);
    if (st != MOT_OK) return st;
    if (n_rows < 0 || n_rows > 4096) return fail(MOT_ERR_BAD_SHAPE, "n_rows=%d must be in [0, 4096]", n_rows);
    if ((int64_t)n_rows * c->max_pages > 1 << 30) return fail(MOT_ERR_BAD_SHAPE, "a new table of more than 2^30 entries");
    if (n_rows == 0) return MOT_OK;
    return pages_call(k_pages, v_pages, table, source, keep, want, new_table, missing, c, n_rows, true, workspace,
                      workspace_bytes, stream);
}

mot_status mot_cache_compact(void* k_pages, void* v_pages, const int32_t* table, int32_t* new_table, int32_t* used,
                             const mot_cache_shapes* c, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    clear_error();
    const mot_status st = check_cache(c);
    if (st != MOT_OK) return st;
    if (c->B == 0) return MOT_OK;
    return pages_call(k_pages, v_pages, table, nullptr, nullptr, nullptr, new_table, used, c, 0, false, workspace,
                      workspace_bytes, stream);
}

}  // extern "C"
