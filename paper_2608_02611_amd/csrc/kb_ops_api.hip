// kb_ops_api.hip -- host side of the reference operators (include/kb.h):
// argument checks, then the launchers.
#include <hip/hip_runtime.h>

#include <cmath>

#include "kb_error.hpp"
#include "kb_internal.hpp"
#include "kb_ops.hpp"

namespace kb {
namespace {

bool float_dtype(int dt) { return dt == DT_F32 || dt == DT_F16 || dt == DT_BF16; }
int element_bytes(int dt) { return dt == DT_F32 ? 4 : 2; }

bool is_empty(const kb_tensor& t) {
    for (int i = 0; i < t.ndim; ++i)
        if (t.shape[i] == 0) return true;
    return false;
}

// A view of ndim dimensions of a float dtype, its last dimension contiguous,
// every offset below 2^62 elements.  An output's elements must be distinct:
// with its dimensions in order of their strides, each stride is at least the
// extent of the dimensions below it.
int check_view(const char* call, const char* name, const kb_tensor* t, int ndim, bool output) {
    if (t == nullptr) return fail(KB_ERR_INVALID_ARG, "%s: null %s", call, name);
    if (!float_dtype(t->dtype)) return fail(KB_ERR_DTYPE, "%s: %s has dtype %d", call, name, t->dtype);
    if (t->ndim != ndim) return fail(KB_ERR_INVALID_ARG, "%s: %s has %d dimensions, not %d", call, name, t->ndim, ndim);
    for (int i = 0; i < ndim; ++i)
        if (t->shape[i] < 0 || t->shape[i] > INT32_MAX)
            return fail(KB_ERR_INVALID_ARG, "%s: dimension %d of %s is %lld", call, i, name, (long long)t->shape[i]);
    if (is_empty(*t)) return KB_OK;
    if (t->data == nullptr) return fail(KB_ERR_INVALID_ARG, "%s: null data of %s", call, name);
    if ((uintptr_t)t->data % element_bytes(t->dtype))
        return fail(KB_ERR_ALIGNMENT, "%s: %s is not aligned to its element", call, name);
    if (t->shape[ndim - 1] > 1 && t->strides[ndim - 1] != 1)
        return fail(KB_ERR_INVALID_ARG, "%s: the last dimension of %s is not contiguous", call, name);
    for (int i = 0; i < ndim; ++i)
        if (t->shape[i] > 1 && (t->strides[i] < 0 || t->strides[i] > ((int64_t)1 << 60) / t->shape[i]))
            return fail(KB_ERR_INVALID_ARG, "%s: stride %d of %s is %lld", call, i, name, (long long)t->strides[i]);
    if (!output) return KB_OK;
    int order[KB_MAX_DIMS], n = 0;
    for (int i = 0; i < ndim; ++i) {
        if (t->shape[i] <= 1) continue;
        int at = n++;
        for (; at > 0 && t->strides[order[at - 1]] > t->strides[i]; --at) order[at] = order[at - 1];
        order[at] = i;
    }
    int64_t extent = 1;  // elements from the first to the last of the dimensions so far
    for (int k = 0; k < n; ++k) {
        const int i = order[k];
        if (t->strides[i] < extent)
            return fail(KB_ERR_INVALID_ARG, "%s: elements of %s share memory (stride %lld)", call, name,
                        (long long)t->strides[i]);
        extent += t->strides[i] * (t->shape[i] - 1);
    }
    return KB_OK;
}

int check_shape(const char* call, const char* name, const kb_tensor& t, const char* like, const kb_tensor& ref) {
    if (t.dtype != ref.dtype)
        return fail(KB_ERR_DTYPE, "%s: %s has dtype %d, %s has %d", call, name, t.dtype, like, ref.dtype);
    for (int i = 0; i < ref.ndim; ++i)
        if (t.shape[i] != ref.shape[i])
            return fail(KB_ERR_INVALID_ARG, "%s: dimension %d of %s is %lld, of %s %lld", call, i, name,
                        (long long)t.shape[i], like, (long long)ref.shape[i]);
    return KB_OK;
}

// A weight-like vector [cols]: of x's dtype or F32, and of the others'.
int check_vector(const char* call, const char* name, const kb_tensor* t, const kb_tensor& x, int* wdtype, bool output) {
    if (t == nullptr) return KB_OK;
    if (const int rc = check_view(call, name, t, 1, output)) return rc;
    if (t->shape[0] != x.shape[1])
        return fail(KB_ERR_INVALID_ARG, "%s: %s has %lld elements, not %lld", call, name, (long long)t->shape[0],
                    (long long)x.shape[1]);
    if (t->dtype != x.dtype && t->dtype != DT_F32)
        return fail(KB_ERR_DTYPE, "%s: %s has dtype %d, neither x's nor F32", call, name, t->dtype);
    if (*wdtype >= 0 && *wdtype != t->dtype)
        return fail(KB_ERR_DTYPE, "%s: %s has dtype %d, another vector %d", call, name, t->dtype, *wdtype);
    *wdtype = t->dtype;
    return KB_OK;
}

// [first, last] bytes of a view that is not empty.
void byte_range(const kb_tensor& t, uintptr_t* first, uintptr_t* last) {
    int64_t extent = 1;
    for (int i = 0; i < t.ndim; ++i)
        if (t.shape[i] > 1) extent += t.strides[i] * (t.shape[i] - 1);
    *first = (uintptr_t)t.data;
    *last = *first + (uintptr_t)extent * element_bytes(t.dtype) - 1;
}

// Whether two views can share memory: overlapping ranges, unless both walk the
// memory with strides that keep them apart (the q, k and v columns of one
// projection, its sequences any distance apart).
bool may_overlap(const kb_tensor& a, const kb_tensor& b) {
    if (is_empty(a) || is_empty(b)) return false;
    uintptr_t a0, a1, b0, b1;
    byte_range(a, &a0, &a1);
    byte_range(b, &b0, &b1);
    if (a1 < b0 || b1 < a0) return false;
    if (a.ndim != b.ndim || a.dtype != b.dtype) return true;
    int64_t off = (int64_t)((a0 < b0 ? b0 - a0 : a0 - b0));
    if (off % element_bytes(a.dtype)) return true;
    off /= element_bytes(a.dtype);
    const kb_tensor& lo = a0 < b0 ? a : b;
    const kb_tensor& hi = a0 < b0 ? b : a;
    // The strides of both from the largest down.  Where the dimensions below a
    // stride s stay within one period of s in both views, elements that coincide do
    // so at the same place of a period: s and what is larger (multiples of s, or
    // dealt with before) fall away, and the offset is taken modulo s.
    int64_t pending[2 * KB_MAX_DIMS];  // larger strides that did not fall away
    int n_pending = 0;
    for (int64_t bound = INT64_MAX;;) {
        // the largest stride below bound among the dimensions with more than one element
        int64_t s = -1;
        for (int i = 0; i < a.ndim; ++i) {
            if (lo.shape[i] > 1 && lo.strides[i] < bound && lo.strides[i] > s) s = lo.strides[i];
            if (hi.shape[i] > 1 && hi.strides[i] < bound && hi.strides[i] > s) s = hi.strides[i];
        }
        if (s <= 0) return true;
        int64_t ext_lo = 1, ext_hi = 1;  // of the dimensions with smaller strides
        for (int i = 0; i < a.ndim; ++i) {
            if (lo.shape[i] > 1 && lo.strides[i] < s) ext_lo += lo.strides[i] * (lo.shape[i] - 1);
            if (hi.shape[i] > 1 && hi.strides[i] < s) ext_hi += hi.strides[i] * (hi.shape[i] - 1);
        }
        const int64_t at = off % s;
        bool within = ext_lo <= s && at + ext_hi <= s;
        for (int k = 0; k < n_pending; ++k) within = within && pending[k] % s == 0;
        if (within) {
            if (at >= ext_lo) return false;
            off = at;
            n_pending = 0;
        } else {
            pending[n_pending++] = s;
        }
        bound = s;
    }
}

struct Named {
    const char* name;
    const kb_tensor* t;
};

// Every output apart from the inputs and from the other outputs.
int check_apart(const char* call, const Named* outs, int n_outs, const Named* ins, int n_ins) {
    for (int o = 0; o < n_outs; ++o) {
        if (outs[o].t == nullptr) continue;
        for (int k = 0; k < o + n_ins; ++k) {
            const Named& other = k < o ? outs[k] : ins[k - o];
            if (other.t != nullptr && may_overlap(*outs[o].t, *other.t))
                return fail(KB_ERR_INVALID_ARG, "%s: %s overlaps %s", call, outs[o].name, other.name);
        }
    }
    return KB_OK;
}

// A dense array of 4-byte elements as a view, for check_apart.
kb_tensor word_array(const void* p, int64_t n) {
    kb_tensor t{};
    t.data = p;
    t.dtype = DT_F32;
    t.ndim = 1;
    t.shape[0] = p ? n : 0;
    t.strides[0] = 1;
    return t;
}

int check_workspace(const char* call, const void* ws, size_t bytes, size_t need) {
    if (need == 0) return KB_OK;
    if (ws == nullptr || bytes < need)
        return fail(KB_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", call, ws ? bytes : (size_t)0, need);
    if ((uintptr_t)ws & 15u) return fail(KB_ERR_ALIGNMENT, "%s: workspace not 16-byte aligned", call);
    return KB_OK;
}

RowView row_view(const kb_tensor* t) {
    return t ? RowView{t->data, t->shape[0] > 1 ? t->strides[0] : 0} : RowView{nullptr, 0};
}

const void* data_of(const kb_tensor* t) { return t ? t->data : nullptr; }

int check_rows(const char* call, const kb_tensor& x) {
    if (x.shape[1] == 0 && x.shape[0] > 0) return fail(KB_ERR_INVALID_ARG, "%s: rows of no element", call);
    return KB_OK;
}

HeadView head_view(const kb_tensor* t) { return HeadView{t->data, t->strides[0], t->strides[1], t->strides[2]}; }

// Rows that can be read in aligned 16-byte chunks, kAttnReach of them within 2^31
// bytes.
bool whole_rows(const kb_tensor& t) {
    const int64_t n = 16 / element_bytes(t.dtype);
    if (((uintptr_t)t.data & 15u) || t.shape[3] % n) return false;
    for (int i = 0; i < 3; ++i)
        if (t.shape[i] > 1 && t.strides[i] % n) return false;
    return t.shape[2] <= 1 || t.strides[2] < ((int64_t)1 << 31) / kAttnReach / element_bytes(t.dtype);
}

constexpr int64_t kMaxLen = (int64_t)1 << 30;

// Sizes of an attention call; false if q and k do not fit together.
bool attn_sizes(const kb_tensor& q, const kb_tensor& k, AttnParams* p) {
    if (q.ndim != 4 || k.ndim != 4 || !float_dtype(q.dtype) || k.dtype != q.dtype) return false;
    for (int i = 0; i < 4; ++i)
        if (q.shape[i] < 0 || k.shape[i] < 0 || q.shape[i] > kMaxLen || k.shape[i] > kMaxLen) return false;
    if (k.shape[0] != q.shape[0] || k.shape[3] != q.shape[3] || q.shape[3] < 1 || q.shape[3] > KB_ATTN_MAX_DIM) return false;
    // key heads divide the query heads (none of either is an empty call)
    if (k.shape[1] == 0 ? q.shape[1] != 0 : q.shape[1] % k.shape[1] != 0) return false;
    // work-groups and rows are numbered with 31 bits at most
    const int64_t heads = q.shape[1] > k.shape[1] ? q.shape[1] : k.shape[1];
    const int64_t len = q.shape[2] > k.shape[2] ? q.shape[2] : k.shape[2];
    if (q.shape[0] * heads > kMaxLen || (len > 0 && q.shape[0] * heads > ((int64_t)1 << 36) / len)) return false;
    p->batch = (int)q.shape[0];
    p->heads = (int)q.shape[1];
    p->kv_heads = (int)k.shape[1];
    p->group = k.shape[1] ? (int)(q.shape[1] / k.shape[1]) : 0;
    p->len_q = (int)q.shape[2];
    p->len_k = (int)k.shape[2];
    p->dim = (int)q.shape[3];
    p->f32 = q.dtype == DT_F32;
    // a launch has fewer than 2^32 threads: 2^24 work-groups of 256
    const int64_t most = ((int64_t)1 << 24) - 1;
    const int64_t norm_blocks = q.shape[0] * k.shape[1] * ((k.shape[2] + kNormBlock - 1) / kNormBlock);
    return row_blocks(*p) <= most && key_blocks(*p) <= most && norm_blocks <= most;
}

// Sequences of different lengths take the more parts.
size_t forward_bytes(AttnParams p) {
    static const int32_t len = 0;
    p.k_lens = &len;
    return (size_t)forward_floats(p, forward_parts(p)) * sizeof(float);
}
// A causal mask takes the more parts.
size_t backward_bytes(AttnParams p) {
    p.causal = 1;
    return (size_t)(backward_layout(p).total + 3) / 4 * 16;
}

// q, k, v and what hangs on their sizes; fills p.
int check_attn(const char* call, const kb_tensor* q, const kb_tensor* k, const kb_tensor* v, const kb_attn_opts* opts,
               AttnParams* p) {
    int rc;
    if ((rc = check_view(call, "q", q, 4, false)) || (rc = check_view(call, "k", k, 4, false)) ||
        (rc = check_view(call, "v", v, 4, false)))
        return rc;
    if (k->dtype != q->dtype) return fail(KB_ERR_DTYPE, "%s: k has dtype %d, q has %d", call, k->dtype, q->dtype);
    if (q->shape[3] < 1 || q->shape[3] > KB_ATTN_MAX_DIM)
        return fail(KB_ERR_INVALID_ARG, "%s: head dimension %lld not in [1, %d]", call, (long long)q->shape[3],
                    KB_ATTN_MAX_DIM);
    if (!attn_sizes(*q, *k, p))
        return fail(KB_ERR_INVALID_ARG, "%s: q and k do not fit together, or are too large", call);
    if ((rc = check_shape(call, "v", *v, "k", *k))) return rc;
    if (opts == nullptr) return fail(KB_ERR_INVALID_ARG, "%s: null opts", call);
    if (!std::isfinite(opts->scale) || !(opts->scale > 0.f))
        return fail(KB_ERR_INVALID_ARG, "%s: scale not finite and > 0", call);
    if (opts->flags & ~(uint32_t)KB_ATTN_CAUSAL)
        return fail(KB_ERR_INVALID_ARG, "%s: unknown flags 0x%x", call, opts->flags);
    if (((uintptr_t)opts->q_lens | (uintptr_t)opts->k_lens) & 3u)
        return fail(KB_ERR_ALIGNMENT, "%s: q_lens or k_lens not aligned to its element", call);
    p->q = head_view(q);
    p->k = head_view(k);
    p->v = head_view(v);
    p->scale = opts->scale;
    p->causal = (opts->flags & KB_ATTN_CAUSAL) != 0;
    p->q_lens = opts->q_lens;
    p->k_lens = opts->k_lens;
    return KB_OK;
}

int check_lse(const char* call, const float* lse, const kb_tensor& q) {
    if (lse == nullptr && q.shape[0] * q.shape[1] * q.shape[2] > 0)
        return fail(KB_ERR_INVALID_ARG, "%s: null lse", call);
    if ((uintptr_t)lse & 3u) return fail(KB_ERR_ALIGNMENT, "%s: lse not aligned to its element", call);
    return KB_OK;
}

}  // namespace
}  // namespace kb

using namespace kb;

extern "C" {

int kb_norm_forward(const kb_tensor* x, const kb_tensor* w, const kb_tensor* b, float eps, const kb_tensor* y,
                    float* mean, float* rstd, hipStream_t stream) {
    clear_error();
    static const char* call = "kb_norm_forward";
    int rc, wdtype = -1;
    if ((rc = check_view(call, "x", x, 2, false)) || (rc = check_rows(call, *x)) ||
        (rc = check_view(call, "y", y, 2, true)) || (rc = check_shape(call, "y", *y, "x", *x)) ||
        (rc = check_vector(call, "w", w, *x, &wdtype, false)) || (rc = check_vector(call, "b", b, *x, &wdtype, false)))
        return rc;
    if (!std::isfinite(eps) || eps < 0.f) return fail(KB_ERR_INVALID_ARG, "%s: eps not finite and >= 0", call);
    if (((uintptr_t)mean | (uintptr_t)rstd) & 3u)
        return fail(KB_ERR_ALIGNMENT, "%s: mean or rstd not aligned to its element", call);
    if (is_empty(*x)) return KB_OK;
    const bool in_place = y->data == x->data && (x->shape[0] == 1 || y->strides[0] == x->strides[0]);
    const kb_tensor tm = word_array(mean, x->shape[0]), tr = word_array(rstd, x->shape[0]);
    const Named outs[] = {{"y", y}, {"mean", &tm}, {"rstd", &tr}};
    const Named ins[] = {{"w", w}, {"b", b}, {"x", x}};
    if ((rc = check_apart(call, outs, 1, ins, in_place ? 2 : 3)) || (rc = check_apart(call, outs, 3, ins, 2)) ||
        (rc = check_apart(call, outs + 1, 2, ins, 3)))
        return rc;
    const NormForwardParams p{row_view(x), row_view(y), data_of(w), data_of(b), mean, rstd, x->shape[0],
                              (int)x->shape[1], eps};
    const hipError_t e = launch_norm_forward(x->dtype, wdtype < 0 ? x->dtype : wdtype, p, stream);
    return e == hipSuccess ? KB_OK : fail_hip(e, "kb_norm_forward: launch");
}

size_t kb_norm_backward_workspace_bytes(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 0 || rows > INT32_MAX || cols > INT32_MAX) return 0;
    return norm_part_bytes(rows, cols);
}

int kb_norm_backward(const kb_tensor* dy, const kb_tensor* x, const kb_tensor* w, const float* mean, const float* rstd,
                     const kb_tensor* dx, const kb_tensor* dw, const kb_tensor* db, void* workspace,
                     size_t workspace_bytes, hipStream_t stream) {
    clear_error();
    static const char* call = "kb_norm_backward";
    int rc, wdtype = -1;
    if ((rc = check_view(call, "dy", dy, 2, false)) || (rc = check_view(call, "x", x, 2, false)) ||
        (rc = check_rows(call, *x)) || (rc = check_shape(call, "dy", *dy, "x", *x)) ||
        (dx && ((rc = check_view(call, "dx", dx, 2, true)) || (rc = check_shape(call, "dx", *dx, "x", *x)))) ||
        (rc = check_vector(call, "w", w, *x, &wdtype, false)) || (rc = check_vector(call, "dw", dw, *x, &wdtype, true)) ||
        (rc = check_vector(call, "db", db, *x, &wdtype, true)))
        return rc;
    if (!is_empty(*x) && (mean == nullptr || rstd == nullptr))
        return fail(KB_ERR_INVALID_ARG, "%s: null mean or rstd", call);
    if (((uintptr_t)mean | (uintptr_t)rstd) & 3u)
        return fail(KB_ERR_ALIGNMENT, "%s: mean or rstd not aligned to its element", call);
    const size_t need = dw || db ? norm_part_bytes(x->shape[0], x->shape[1]) : 0;
    if ((rc = check_workspace(call, workspace, workspace_bytes, need))) return rc;
    const kb_tensor tm = word_array(mean, x->shape[0]), tr = word_array(rstd, x->shape[0]);
    const kb_tensor tw = word_array(need ? workspace : nullptr, (int64_t)(need / sizeof(float)));
    const Named outs[] = {{"dx", dx}, {"dw", dw}, {"db", db}, {"the workspace", &tw}};
    const Named ins[] = {{"dy", dy}, {"x", x}, {"w", w}, {"mean", &tm}, {"rstd", &tr}};
    if ((rc = check_apart(call, outs, 4, ins, 5))) return rc;
    if (x->shape[1] == 0 || (x->shape[0] == 0 && !dw && !db)) return KB_OK;
    const NormBackwardParams p{row_view(dy), row_view(x), row_view(dx), data_of(w), mean, rstd, (void*)data_of(dw),
                               (void*)data_of(db), (float*)workspace, x->shape[0], (int)x->shape[1]};
    const hipError_t e = launch_norm_backward(x->dtype, wdtype < 0 ? x->dtype : wdtype, p, stream);
    return e == hipSuccess ? KB_OK : fail_hip(e, "kb_norm_backward: launch");
}

size_t kb_attn_forward_workspace_bytes(const kb_tensor* q, const kb_tensor* k) {
    AttnParams p{};
    if (q == nullptr || k == nullptr || !attn_sizes(*q, *k, &p)) return 0;
    return forward_bytes(p);
}

int kb_attn_forward(const kb_tensor* q, const kb_tensor* k, const kb_tensor* v, const kb_attn_opts* opts,
                    const kb_tensor* o, float* lse, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    clear_error();
    static const char* call = "kb_attn_forward";
    AttnParams p{};
    int rc;
    if ((rc = check_attn(call, q, k, v, opts, &p)) || (rc = check_view(call, "o", o, 4, true)) ||
        (rc = check_shape(call, "o", *o, "q", *q)) || (rc = check_lse(call, lse, *q)))
        return rc;
    p.parts = forward_parts(p);
    const size_t need = forward_bytes(p);
    if ((rc = check_workspace(call, workspace, workspace_bytes, need))) return rc;
    const kb_tensor tl = word_array(lse, q->shape[0] * q->shape[1] * q->shape[2]);
    const kb_tensor tw = word_array(need ? workspace : nullptr, (int64_t)(need / sizeof(float)));
    const kb_tensor ql = word_array(p.q_lens, p.batch), kl = word_array(p.k_lens, p.batch);
    const Named outs[] = {{"o", o}, {"lse", &tl}, {"the workspace", &tw}};
    const Named ins[] = {{"q", q}, {"k", k}, {"v", v}, {"q_lens", &ql}, {"k_lens", &kl}};
    if ((rc = check_apart(call, outs, 3, ins, 5))) return rc;
    if (is_empty(*q)) return KB_OK;
    p.o = head_view(o);
    p.whole = whole_rows(*q) && whole_rows(*k) && whole_rows(*v);
    p.lse = lse;
    p.ws = (float*)workspace;
    const hipError_t e = launch_attn_forward(q->dtype, p, stream);
    return e == hipSuccess ? KB_OK : fail_hip(e, "kb_attn_forward: launch");
}

size_t kb_attn_backward_workspace_bytes(const kb_tensor* q, const kb_tensor* k) {
    AttnParams p{};
    if (q == nullptr || k == nullptr || !attn_sizes(*q, *k, &p)) return 0;
    return backward_bytes(p);
}

int kb_attn_backward(const kb_tensor* dout, const kb_tensor* q, const kb_tensor* k, const kb_tensor* v,
                     const kb_tensor* o, const float* lse, const kb_attn_opts* opts, const kb_tensor* dq,
                     const kb_tensor* dk, const kb_tensor* dv, void* workspace, size_t workspace_bytes,
                     hipStream_t stream) {
    clear_error();
    static const char* call = "kb_attn_backward";
    AttnParams p{};
    int rc;
    if ((rc = check_attn(call, q, k, v, opts, &p)) || (rc = check_view(call, "dout", dout, 4, false)) ||
        (rc = check_shape(call, "dout", *dout, "q", *q)) || (rc = check_view(call, "o", o, 4, false)) ||
        (rc = check_shape(call, "o", *o, "q", *q)) || (rc = check_lse(call, lse, *q)) ||
        (rc = check_view(call, "dq", dq, 4, true)) || (rc = check_shape(call, "dq", *dq, "q", *q)) ||
        (rc = check_view(call, "dk", dk, 4, true)) || (rc = check_shape(call, "dk", *dk, "k", *k)) ||
        (rc = check_view(call, "dv", dv, 4, true)) || (rc = check_shape(call, "dv", *dv, "k", *k)))
        return rc;
    p.parts = row_parts(p);
    p.key_parts = key_parts(p);
    const size_t need = backward_bytes(p);
    if ((rc = check_workspace(call, workspace, workspace_bytes, need))) return rc;
    const kb_tensor tl = word_array(lse, q->shape[0] * q->shape[1] * q->shape[2]);
    const kb_tensor tw = word_array(need ? workspace : nullptr, (int64_t)(need / sizeof(float)));
    const kb_tensor ql = word_array(p.q_lens, p.batch), kl = word_array(p.k_lens, p.batch);
    const Named outs[] = {{"dq", dq}, {"dk", dk}, {"dv", dv}, {"the workspace", &tw}};
    const Named ins[] = {{"dout", dout}, {"q", q}, {"k", k}, {"v", v}, {"o", o}, {"lse", &tl}, {"q_lens", &ql}, {"k_lens", &kl}};
    if ((rc = check_apart(call, outs, 4, ins, 8))) return rc;
    if (row_blocks(p) == 0 && key_blocks(p) == 0) return KB_OK;  // (keys that no query head reads have gradients, of 0)
    p.dout = head_view(dout);
    p.whole = whole_rows(*q) && whole_rows(*k) && whole_rows(*v) && whole_rows(*dout) && whole_rows(*o);
    p.o = head_view(o);
    p.dq = head_view(dq);
    p.dk = head_view(dk);
    p.dv = head_view(dv);
    p.lse = (float*)lse;
    p.ws = (float*)workspace;
    const hipError_t e = launch_attn_backward(q->dtype, p, stream);
    return e == hipSuccess ? KB_OK : fail_hip(e, "kb_attn_backward: launch");
}

}  // extern "C"
