// Host entry points of the paged 8-bit cache and of rotary positions (include/occam_cache.h):
// argument validation, views and launches.  Validation runs before any HIP call, so an
// invalid call enqueues nothing.
#include <math.h>
#include <string.h>

#include "cache_internal.hpp"

using namespace occam;

namespace {

constexpr size_t kAlign = 256;
size_t align_up(size_t x) { return (x + kAlign - 1) & ~(kAlign - 1); }
bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
bool given(const void* p, size_t a) { return p && aligned(p, a); }
occam_status hip_ok(hipError_t e) { return e == hipSuccess ? OCCAM_OK : OCCAM_ERR_HIP; }

// `arrays`: whether the call touches the device arrays (the size queries do not).
occam_status pages_from(const occam_pages* p, bool arrays, PageView* out) {
    if (!p) return OCCAM_ERR_INVALID_ARG;
    if (p->num_pages < 1 || p->num_pages > (1 << 24) || p->num_seqs < 1 ||
        p->num_seqs > OCCAM_MAX_SLOTS || p->max_pages < 1)
        return OCCAM_ERR_INVALID_ARG;
    int shift = 0;
    for (int s = 4; s <= 8; ++s)
        if (p->page_tokens == 1 << s) shift = s;
    if (!shift) return OCCAM_ERR_INVALID_ARG;
    // Token positions are 32-bit, with room to round them up to pages and tiles.
    if (((long long)p->max_pages << shift) > (1LL << 31) - 4096) return OCCAM_ERR_UNSUPPORTED;
    if (arrays && (!given(p->table, 4) || !given(p->length, 4) || !given(p->refs, 4) ||
                   !given(p->taken, 4) || !given(p->status, 4)))
        return OCCAM_ERR_INVALID_ARG;
    *out = PageView{p->num_pages, shift, p->num_seqs, p->max_pages, p->table, p->length, p->refs,
                    p->taken, p->status};
    return OCCAM_OK;
}

occam_status shape_from(const PageView& p, int Hkv, int d, CacheView* out) {
    if (Hkv < 1 || d < 8 || d > 256 || d % 8) return OCCAM_ERR_INVALID_ARG;
    // (page, head) blocks of keys and values are numbered in 32 bits.
    if ((long long)p.num_pages * Hkv >= (1LL << 30)) return OCCAM_ERR_UNSUPPORTED;
    memset(out, 0, sizeof *out);
    out->Hkv = Hkv;
    out->d = d;
    out->dp = d <= 64 ? 64 : d <= 128 ? 128 : 256;
    out->block = (unsigned)out->dp << p.shift;
    return OCCAM_OK;
}

occam_status cache_from(const PageView& p, const occam_cache* c, CacheView* out) {
    if (!c) return OCCAM_ERR_INVALID_ARG;
    occam_status st = shape_from(p, c->num_kv_heads, c->head_dim, out);
    if (st != OCCAM_OK) return st;
    if (!given(c->k, 16) || !given(c->v, 16) || !given(c->k_scale, 4) || !given(c->v_scale, 4))
        return OCCAM_ERR_INVALID_ARG;
    out->k = c->k; out->v = c->v; out->ks = c->k_scale; out->vs = c->v_scale;
    return OCCAM_OK;
}

occam_status batch_from(const PageView& p, const occam_batch* b, BatchView* out) {
    if (!b || b->n < 1 || b->n > OCCAM_MAX_BATCH) return OCCAM_ERR_INVALID_ARG;
    if (b->row_offsets ? b->max_rows < 1 : b->rows < 1) return OCCAM_ERR_INVALID_ARG;
    if ((b->seq && !aligned(b->seq, 4)) || (b->row_offsets && !aligned(b->row_offsets, 4)))
        return OCCAM_ERR_INVALID_ARG;
    if (!b->seq && b->n > p.num_seqs) return OCCAM_ERR_INVALID_ARG;
    const long long most = b->row_offsets ? b->max_rows : b->rows;
    if (most * b->n >= (1LL << 31)) return OCCAM_ERR_UNSUPPORTED;
    *out = BatchView{b->n, b->rows, (int)most, b->seq, b->row_offsets};
    return OCCAM_OK;
}

occam_status check_plan(const PageView& p, int n, const void* plan, size_t bytes) {
    if (n < 1 || n > OCCAM_MAX_BATCH) return OCCAM_ERR_INVALID_ARG;
    if (bytes < plan_ints(n, p.max_pages, p.num_pages) * 4) return OCCAM_ERR_WORKSPACE;
    return given(plan, 4) ? OCCAM_OK : OCCAM_ERR_INVALID_ARG;
}

// A tensor of rows [.][Hkv][d]: 16-byte aligned, rows a multiple of 16 bytes apart.
bool rows_ok(const void* x, long long stride, const CacheView& c, int dtype) {
    const int per = dtype == OCCAM_F32 ? 4 : 8;
    return aligned(x, 16) && stride >= (long long)c.Hkv * c.d && stride % per == 0;
}

// Whether rows of `wa` and `wb` bytes, the first at a and b, `sa` and `sb` bytes apart, overlap.
// Rows as far apart as each other may interleave (slices of one projection); of rows otherwise
// apart those whose ranges meet count as overlapping.
bool rows_meet(uintptr_t a, long long sa, long long wa, uintptr_t b, long long sb, long long wb, int rows) {
    if (b < a) return rows_meet(b, sb, wb, a, sa, wa, rows);
    const long long gap = (long long)(b - a);
    if (rows < 1 || gap >= (rows - 1) * sa + wa) return false;
    if (rows == 1 || sa != sb) return true;
    const long long in = gap % sa;
    return in < wa || in + wb > sa;
}

struct AttendPlan {
    AttendArgs a;
    size_t off_l, off_cuts, total;
};

occam_status attend_plan(const PageView& p, const CacheView& c, const BatchView& b,
                         const occam_attention* at, AttendPlan* out) {
    if (!at || at->num_heads < 1 || at->num_heads % c.Hkv || at->max_tokens < 0 ||
        (at->causal != 0 && at->causal != 1) || !(at->softmax_scale >= 0.f) ||
        isinf(at->softmax_scale))
        return OCCAM_ERR_INVALID_ARG;
    memset(out, 0, sizeof *out);
    AttendArgs& a = out->a;
    a.pg = p; a.c = c; a.b = b;
    a.H = at->num_heads;
    a.g = a.H / c.Hkv;
    a.causal = at->causal;
    const float scale = at->softmax_scale > 0.f ? at->softmax_scale : 1.0f / sqrtf((float)c.d);
    a.scale2 = scale * kLog2e;
    if (isinf(a.scale2)) return OCCAM_ERR_INVALID_ARG;
    const long long cap = (long long)p.max_pages << p.shift;
    const long long most = at->max_tokens && at->max_tokens < cap ? at->max_tokens : cap;
    // (row, head) pairs are numbered in 32 bits, and so are row blocks.
    if ((long long)b.n * b.max_rows * a.H >= (1LL << 31) || c.Hkv > 65535) return OCCAM_ERR_UNSUPPORTED;
    // Units of at least 64 keys of all row blocks (of at least 16 rows), at the longest.
    if ((double)b.n * ((double)b.max_rows * a.g / 16 + 1) * ((double)cap / 64 + 1) >= 2147483648.0)
        return OCCAM_ERR_UNSUPPORTED;
    const AttendShape& x = a.shape = attend_shape(c, b, a.H, most);
    if (x.cuts > 65535) return OCCAM_ERR_UNSUPPORTED;      // a launch's grid.y
    // A launch has fewer than 2^32 threads: of the many-row form, two for every row of its blocks.
    if (!x.few && (double)b.n * x.blocks * x.ranges * c.Hkv * (2 * x.block_rows) >= 4294967296.0)
        return OCCAM_ERR_UNSUPPORTED;
    if (x.slots > 0) {
        const size_t rows = (size_t)c.Hkv * x.slots * x.block_rows;
        out->off_l = align_up(rows * c.dp * sizeof(float));
        out->off_cuts = align_up(out->off_l + rows * sizeof(float));
        out->total = align_up(out->off_cuts + (size_t)x.cuts * sizeof(int4));
    }
    if (x.ordered) out->total = align_up(x.ordered * sizeof(AttendBlock));     // (then nothing is cut)
    if (out->total < kAlign) out->total = kAlign;
    return OCCAM_OK;
}

// The largest power of two up to `most` that divides x.
int pow2_in(long long x, int most) {
    const long long low = x & -x;
    return low && low < most ? (int)low : most;
}

}  // namespace

extern "C" {

occam_status occam_rotary_init(occam_rotary* rotary, int32_t head_dim, int32_t pairs, int32_t axes,
                               int32_t layout, const double* inv_freq, const uint8_t* axis) {
    if (!rotary || !inv_freq || head_dim < 2 || head_dim > 256 || head_dim % 2 || pairs < 1 ||
        pairs > head_dim / 2 || axes < 1 || axes > 4 ||
        (layout != OCCAM_PAIRS_HALVES && layout != OCCAM_PAIRS_ADJACENT))
        return OCCAM_ERR_INVALID_ARG;
    for (int p = 0; p < pairs; ++p)
        if (!isfinite(inv_freq[p]) || (axis && axis[p] >= axes)) return OCCAM_ERR_INVALID_ARG;
    memset(rotary, 0, sizeof *rotary);
    rotary->head_dim = head_dim;
    rotary->pairs = pairs;
    rotary->axes = axes;
    rotary->layout = layout;
    for (int p = 0; p < pairs; ++p) {
        // Turns per position, whole turns dropped: positions are whole numbers.
        const long double turns = (long double)inv_freq[p] / 6.283185307179586476925286766559005768L;
        const long double f = turns - floorl(turns);                  // [0, 1]
        const long double u = f * 18446744073709551616.0L;            // 2^64
        rotary->turn[p] = u >= 18446744073709551615.5L ? 0 : (uint64_t)(u + 0.5L);
        rotary->axis[p] = axis ? axis[p] : 0;
    }
    return OCCAM_OK;
}

occam_status occam_rotate(const occam_rotary* rotary, int32_t rows, const int32_t* positions,
                          int32_t inverse, int32_t dtype, int32_t n, const occam_heads* tensors,
                          hipStream_t stream) {
    if (!rotary || rows < 0 || !given(positions, 4) || (dtype != OCCAM_F32 && dtype != OCCAM_BF16) ||
        n < 1 || n > OCCAM_MAX_ROW_TENSORS || !tensors)
        return OCCAM_ERR_INVALID_ARG;
    const occam_rotary& r = *rotary;
    if (r.head_dim < 2 || r.head_dim > 256 || r.head_dim % 2 || r.pairs < 1 ||
        r.pairs > r.head_dim / 2 || r.axes < 1 || r.axes > 4 ||
        (r.layout != OCCAM_PAIRS_HALVES && r.layout != OCCAM_PAIRS_ADJACENT))
        return OCCAM_ERR_INVALID_ARG;
    for (int p = 0; p < r.pairs; ++p)
        if (r.axis[p] >= r.axes) return OCCAM_ERR_INVALID_ARG;
    RotArgs a;
    const long long e = dtype == OCCAM_F32 ? 4 : 2;
    int vec = dtype == OCCAM_F32 ? 4 : 8;
    vec = pow2_in(r.head_dim, vec);
    vec = pow2_in(r.layout == OCCAM_PAIRS_HALVES ? r.pairs : 2 * r.pairs, vec);
    long long heads = 0;
    for (int i = 0; i < n; ++i) {
        const occam_heads& t = tensors[i];
        const long long row = (long long)t.heads * r.head_dim;
        if (!given(t.src, (size_t)e) || !given(t.dst, (size_t)e) || t.heads < 1 ||
            t.src_row_stride < row || t.dst_row_stride < row ||
            (t.src == t.dst && t.src_row_stride != t.dst_row_stride))
            return OCCAM_ERR_INVALID_ARG;
        const uintptr_t s0 = reinterpret_cast<uintptr_t>(t.src), d0 = reinterpret_cast<uintptr_t>(t.dst);
        const long long ss = t.src_row_stride * e, ds = t.dst_row_stride * e;
        if (s0 != d0 && rows_meet(s0, ss, row * e, d0, ds, row * e, rows)) return OCCAM_ERR_INVALID_ARG;
        // Nor does anything that one tensor writes lie in another one's rows.
        for (int j = 0; j < i; ++j) {
            const RotTensor& o = a.t[j];
            const uintptr_t os = reinterpret_cast<uintptr_t>(o.src), od = reinterpret_cast<uintptr_t>(o.dst);
            const long long ow = (long long)o.heads * r.head_dim * e;
            if (rows_meet(d0, ds, row * e, od, o.dst_stride, ow, rows) ||
                (os != od && rows_meet(d0, ds, row * e, os, o.src_stride, ow, rows)) ||
                (s0 != d0 && rows_meet(s0, ss, row * e, od, o.dst_stride, ow, rows)))
                return OCCAM_ERR_INVALID_ARG;
        }
        heads += t.heads;
        vec = pow2_in((long long)(s0 / e) | (long long)(d0 / e), vec);
        vec = pow2_in(t.src_row_stride | t.dst_row_stride, vec);
        a.t[i] = RotTensor{static_cast<const char*>(t.src), static_cast<char*>(t.dst), t.heads,
                           (int)(heads - t.heads), t.src_row_stride * e, t.dst_row_stride * e};
    }
    // A launch has fewer than 2^32 threads: 256 for every 2048 (row, pair) angles.
    if (heads > 4096 || rows / (2048 / r.pairs) >= (1 << 24) - 1) return OCCAM_ERR_UNSUPPORTED;
    if (rows == 0) return OCCAM_OK;
    a.n = n;
    a.heads = (int)heads;
    a.rows = rows;
    a.d = r.head_dim;
    a.pairs = r.pairs;
    a.axes = r.axes;
    a.inverse = inverse != 0;
    a.adjacent = r.layout == OCCAM_PAIRS_ADJACENT;
    a.pos = positions;
    memcpy(a.turn, r.turn, sizeof a.turn);
    memcpy(a.axis, r.axis, sizeof a.axis);
    return hip_ok(launch_rotate(a, dtype == OCCAM_F32, vec, stream));
}

size_t occam_pages_plan_size(const occam_pages* pages, int32_t n) {
    PageView p;
    if (pages_from(pages, false, &p) != OCCAM_OK || n < 1 || n > OCCAM_MAX_BATCH) return 0;
    return plan_ints(n, p.max_pages, p.num_pages) * 4;
}

size_t occam_cache_storage_size(const occam_pages* pages, int32_t num_kv_heads, int32_t head_dim) {
    PageView p;
    CacheView c;
    if (pages_from(pages, false, &p) != OCCAM_OK ||
        shape_from(p, num_kv_heads, head_dim, &c) != OCCAM_OK)
        return 0;
    return (size_t)p.num_pages * c.Hkv * c.block;
}

occam_status occam_pages_reset(const occam_pages* pages, hipStream_t stream) {
    PageView p;
    occam_status st = pages_from(pages, true, &p);
    if (st != OCCAM_OK) return st;
    return hip_ok(launch_pages_reset(p, stream));
}

occam_status occam_pages_reserve(const occam_pages* pages, const occam_batch* batch, void* plan,
                                 size_t plan_bytes, hipStream_t stream) {
    PageView p;
    BatchView b;
    occam_status st;
    if ((st = pages_from(pages, true, &p)) != OCCAM_OK || (st = batch_from(p, batch, &b)) != OCCAM_OK ||
        (st = check_plan(p, b.n, plan, plan_bytes)) != OCCAM_OK)
        return st;
    return hip_ok(launch_pages_reserve(p, b, static_cast<int*>(plan), stream));
}

occam_status occam_pages_fork(const occam_pages* pages, int32_t n, const int32_t* src,
                              const int32_t* dst, void* plan, size_t plan_bytes, hipStream_t stream) {
    PageView p;
    occam_status st;
    if ((st = pages_from(pages, true, &p)) != OCCAM_OK ||
        (st = check_plan(p, n, plan, plan_bytes)) != OCCAM_OK)
        return st;
    if (!given(src, 4) || !given(dst, 4)) return OCCAM_ERR_INVALID_ARG;
    return hip_ok(launch_pages_fork(p, n, src, dst, static_cast<int*>(plan), stream));
}

occam_status occam_pages_free(const occam_pages* pages, int32_t n, const int32_t* seq,
                              hipStream_t stream) {
    PageView p;
    occam_status st = pages_from(pages, true, &p);
    if (st != OCCAM_OK) return st;
    if (n < 1 || n > OCCAM_MAX_BATCH || !given(seq, 4)) return OCCAM_ERR_INVALID_ARG;
    return hip_ok(launch_pages_free(p, n, seq, stream));
}

occam_status occam_pages_keep(const occam_pages* pages, int32_t n, const int32_t* seq,
                              const int32_t* span_start, const int32_t* span_len,
                              const int32_t* kept_idx, const int32_t* kept_offsets, void* plan,
                              size_t plan_bytes, hipStream_t stream) {
    PageView p;
    occam_status st;
    if ((st = pages_from(pages, true, &p)) != OCCAM_OK ||
        (st = check_plan(p, n, plan, plan_bytes)) != OCCAM_OK)
        return st;
    if (!given(seq, 4) || !given(span_start, 4) || !given(span_len, 4) || !given(kept_idx, 4) ||
        !given(kept_offsets, 4))
        return OCCAM_ERR_INVALID_ARG;
    return hip_ok(launch_pages_keep(p, n, seq, span_start, span_len, kept_idx, kept_offsets,
                                    static_cast<int*>(plan), stream));
}

occam_status occam_cache_append(const occam_pages* pages, const occam_cache* cache,
                                const occam_batch* batch, const void* plan, size_t plan_bytes,
                                int32_t dtype, const void* k, int64_t k_row_stride, const void* v,
                                int64_t v_row_stride, hipStream_t stream) {
    PageView p;
    CacheView c;
    BatchView b;
    occam_status st;
    if ((st = pages_from(pages, true, &p)) != OCCAM_OK || (st = cache_from(p, cache, &c)) != OCCAM_OK ||
        (st = batch_from(p, batch, &b)) != OCCAM_OK ||
        (st = check_plan(p, b.n, plan, plan_bytes)) != OCCAM_OK)
        return st;
    if ((dtype != OCCAM_F32 && dtype != OCCAM_BF16) || !k || !v ||
        !rows_ok(k, k_row_stride, c, dtype) || !rows_ok(v, v_row_stride, c, dtype))
        return OCCAM_ERR_INVALID_ARG;
    return hip_ok(launch_cache_append(p, c, b, static_cast<const int*>(plan), dtype == OCCAM_F32, k,
                                      k_row_stride, v, v_row_stride, stream));
}

occam_status occam_cache_read(const occam_pages* pages, const occam_cache* cache,
                              const occam_batch* batch, const int32_t* start, int32_t dtype, void* k,
                              int64_t k_row_stride, void* v, int64_t v_row_stride,
                              hipStream_t stream) {
    PageView p;
    CacheView c;
    BatchView b;
    occam_status st;
    if ((st = pages_from(pages, true, &p)) != OCCAM_OK || (st = cache_from(p, cache, &c)) != OCCAM_OK ||
        (st = batch_from(p, batch, &b)) != OCCAM_OK)
        return st;
    if ((dtype != OCCAM_F32 && dtype != OCCAM_BF16) || (!k && !v) || (start && !aligned(start, 4)) ||
        (k && !rows_ok(k, k_row_stride, c, dtype)) || (v && !rows_ok(v, v_row_stride, c, dtype)))
        return OCCAM_ERR_INVALID_ARG;
    // A thread per group of four tokens, head and eight elements, numbered in 32 bits.
    if (((long long)b.max_rows / 4 + 2) * c.Hkv * (c.d / 8) >= (1LL << 31)) return OCCAM_ERR_UNSUPPORTED;
    return hip_ok(launch_cache_read(p, c, b, start, dtype == OCCAM_F32, k, k_row_stride, v,
                                    v_row_stride, stream));
}

occam_status occam_cache_move(const occam_pages* pages, const occam_cache* cache, int32_t n,
                              const void* plan, size_t plan_bytes, const int32_t* kept_idx,
                              const int32_t* kept_offsets, hipStream_t stream) {
    PageView p;
    CacheView c;
    occam_status st;
    if ((st = pages_from(pages, true, &p)) != OCCAM_OK || (st = cache_from(p, cache, &c)) != OCCAM_OK ||
        (st = check_plan(p, n, plan, plan_bytes)) != OCCAM_OK)
        return st;
    if (!given(kept_idx, 4) || !given(kept_offsets, 4)) return OCCAM_ERR_INVALID_ARG;
    // (Where the lists begin stands in the plan's records.)
    return hip_ok(launch_cache_move(p, c, n, static_cast<const int*>(plan), kept_idx, stream));
}

size_t occam_cache_workspace_size(const occam_pages* pages, const occam_cache* cache,
                                  const occam_batch* batch, const occam_attention* attention) {
    PageView p;
    CacheView c;
    BatchView b;
    AttendPlan ap;
    if (!cache || pages_from(pages, false, &p) != OCCAM_OK ||
        shape_from(p, cache->num_kv_heads, cache->head_dim, &c) != OCCAM_OK ||
        batch_from(p, batch, &b) != OCCAM_OK || attend_plan(p, c, b, attention, &ap) != OCCAM_OK)
        return 0;
    return ap.total;
}

occam_status occam_cache_attend(const occam_pages* pages, const occam_cache* cache,
                                const occam_batch* batch, const occam_attention* attention,
                                const void* q, int64_t q_row_stride, void* out,
                                int64_t out_row_stride, float* row_lse, void* workspace,
                                size_t ws_bytes, hipStream_t stream) {
    PageView p;
    CacheView c;
    BatchView b;
    AttendPlan ap;
    occam_status st;
    if ((st = pages_from(pages, true, &p)) != OCCAM_OK || (st = cache_from(p, cache, &c)) != OCCAM_OK ||
        (st = batch_from(p, batch, &b)) != OCCAM_OK ||
        (st = attend_plan(p, c, b, attention, &ap)) != OCCAM_OK)
        return st;
    const long long row = (long long)ap.a.H * c.d;
    if (!given(q, 16) || !given(out, 16) || q_row_stride < row || out_row_stride < row ||
        q_row_stride % 8 || out_row_stride % 8 || (row_lse && !aligned(row_lse, 4)))
        return OCCAM_ERR_INVALID_ARG;
    if (ws_bytes < ap.total) return OCCAM_ERR_WORKSPACE;
    // In place would not do: a row's queries are read by several workgroups.  (How many rows
    // there are is known here without row_offsets only.)
    if (!given(workspace, kAlign) || q == out ||
        (!b.off && rows_meet(reinterpret_cast<uintptr_t>(q), q_row_stride * 2, row * 2,
                             reinterpret_cast<uintptr_t>(out), out_row_stride * 2, row * 2, b.n * b.rows)))
        return OCCAM_ERR_INVALID_ARG;
    AttendArgs& a = ap.a;
    a.q = static_cast<const unsigned short*>(q);
    a.out = static_cast<unsigned short*>(out);
    a.q_stride = q_row_stride;
    a.out_stride = out_row_stride;
    a.lse = row_lse;
    a.part_o = static_cast<float*>(workspace);
    a.part_l = reinterpret_cast<float*>(static_cast<char*>(workspace) + ap.off_l);
    a.cuts = reinterpret_cast<int4*>(static_cast<char*>(workspace) + ap.off_cuts);
    a.order = a.shape.ordered ? static_cast<AttendBlock*>(workspace) : nullptr;
    return hip_ok(launch_cache_attend(a, stream));
}

}  // extern "C"
