// The binding's work on the calls of the attention layers; included by host.cpp, whose helpers it uses.

int int_of(int64_t v) {
    require(v >= 0 && v <= INT32_MAX, "sizes below 2^31");
    return (int)v;
}
// An int32 array of this shape, dense; null for None.
int32_t *numbers(Arg a, std::initializer_list<int64_t> size, const char *text) {
    const Array t(a);
    require(t.type() == at::kInt && t.shaped(size) && t.is_contiguous(), text);
    return static_cast<int32_t *>(t.data_ptr());
}
int32_t *numbers_or_none(Arg a, std::initializer_list<int64_t> size, const char *text) {
    return a.o == Py_None ? nullptr : numbers(a, size, text);
}
// Every tensor of a call lies on the current device, whose stream the work goes to.
void on_device(std::initializer_list<Arg> all) {
    int64_t device = -1;
    for (const Arg &a : all) {
        if (a.o == Py_None || !a.plain()) continue;
        const at::Tensor &t = THPVariable_Unpack(a.o);
        require(t.is_cuda() && (device < 0 || t.get_device() == device), "tensors on one GPU");
        device = t.get_device();
    }
    if (device >= 0) require(device == c10::hip::getCurrentHIPStream().device_index(), "tensors on the current GPU");
}

// The cache, of one layer ([pages, heads, ...]) or, where `layers` allows, of several ([layers, pages, heads, ...]).
stree_kv make_kv(Arg k_cache, Arg v_cache, Arg table, bool layers) {
    const Array k(k_cache), v(v_cache), t(table);
    const int64_t n = k.dim(), l = n - 4;
    if (n != 4 && !(layers && n == 5)) raise(PyExc_ValueError, layers ? "k_cache [layers, pages, heads, page, headdim]" : "k_cache [pages, heads, page, headdim]");
    stree_kv c = {};
    c.nlayers = l ? int_of(k.size(0)) : 1, c.npages = int_of(k.size(l)), c.nheads_kv = int_of(k.size(l + 1));
    c.page = int_of(k.size(l + 2)), c.headdim = int_of(k.size(l + 3));
    require(l ? v.shaped({c.nlayers, c.npages, c.nheads_kv, c.headdim, c.page}) : v.shaped({c.npages, c.nheads_kv, c.headdim, c.page}),
            "v_cache has k_cache's shape with its last two dimensions exchanged");
    require(v.same_type(k) && k.is_contiguous() && v.is_contiguous(), "caches of one dtype, dense");
    dimensions(t, 2);
    c.max_pages = int_of(t.size(1));
    c.io_dtype = type_code(k);
    c.k = k.data_ptr(), c.v = v.data_ptr();
    c.table = numbers(table, {t.size(0), t.size(1)}, "table int32 [B, max_pages], dense");
    return c;
}
const int32_t *make_parent(Arg parent, int64_t B, int64_t N) {
    return numbers_or_none(parent, {B, N}, "parent int32 [B,N], dense, or None for a chain");
}
// Element stride between the tokens of [B,N,heads,headdim] rows.  0 means dense to the library, so rows that lie on one another
// (an expanded tensor) are refused; of a single row the stride means nothing.
int64_t rows_stride(const Array &t, int64_t B, int64_t N) {
    const int64_t s = token_stride(t, N);
    if (B * N <= 1) return 0;
    require(s >= t.size(2) * t.size(3), "rows apart from one another");
    return s;
}
float number_of(PyObject *o) {
    const double v = PyFloat_AsDouble(o);
    if (PyErr_Occurred()) throw Raised{};
    return (float)v;
}

PyObject *rope(const Args &a) {
    enum { parent, lengths, q, k, v, k_cache, v_cache, table, turns, q_norm, k_norm, eps, interleaved, rope_scale, out, status };
    const Array tq(a[q]), tk(a[k]), tv(a[v]);
    dimensions(tq, 4);
    const int64_t B = tq.size(0), N = tq.size(1), H = tq.size(2), P = tq.size(3);
    const stree_kv kv = make_kv(a[k_cache], a[v_cache], a[table], false);
    require(kv.headdim == P && kv.io_dtype == rows_code(a[q]), "q and the cache agree in headdim and dtype");
    require(tk.shaped({B, N, kv.nheads_kv, P}) && tv.shaped({B, N, kv.nheads_kv, P}) && tk.same_type(tq) && tv.same_type(tq), "k and v [B,N,heads of the cache,P]");
    require(Array(a[table]).size(0) == B, "a row of the table per sequence");
    stree_attn d = {};
    d.batch = int_of(B), d.nnodes = int_of(N), d.nheads = int_of(H);
    d.flags = truth(a[interleaved]) ? STREE_ROPE_INTERLEAVED : 0;
    d.eps = number_of(a[eps]), d.rope_scale = number_of(a[rope_scale]);
    const double *angles = nullptr;
    if (a[turns] != Py_None) {
        const Array t(a[turns]);
        require(t.dim() == 1 && t.type() == at::kDouble && t.is_contiguous() && 2 * t.size(0) <= P, "turns f64 [rotary_dim/2], dense");
        d.rotary_dim = (int)(2 * t.size(0));
        angles = static_cast<const double *>(t.data_ptr());
    }
    for (const Arg &w : {a[q_norm], a[k_norm]})
        if (w.o != Py_None) require(Array(w).shaped({P}) && Array(w).same_type(tq) && Array(w).is_contiguous(), "norm weights [P] in q's dtype");
    d.q_stride_n = rows_stride(tq, B, N), d.k_stride_n = rows_stride(tk, B, N), d.v_stride_n = rows_stride(tv, B, N);
    const int32_t *p0 = make_parent(a[parent], B, N), *p1 = numbers(a[lengths], {B}, "lengths int32 [B]");
    int32_t *p2 = numbers_or_none(a[status], {B}, "status int32 [B]");
    Result o;
    sized(o, a[out], a[q], {B, N, H, P}, a[q]);
    require(o.t().shaped({B, N, H, P}) && o.t().same_type(tq) && o.t().is_contiguous(), "out [B,N,H,P], dense");
    on_device({a[parent], a[lengths], a[q], a[k], a[v], a[k_cache], a[v_cache], a[table], a[turns], a[q_norm], a[k_norm], a[out], a[status]});
    const void *p3 = pointer(a[q]), *p4 = pointer(a[k]), *p5 = pointer(a[v]), *p6 = pointer(a[q_norm]), *p7 = pointer(a[k_norm]);
    void *p8 = o.ptr(), *st = stream();
    run("stree_tree_rope", [&] { return g_entry.tree_rope(&d, &kv, p0, p1, p3, p4, p5, p6, p7, angles, p8, p2, st); });
    return o.release();
}

PyObject *attn(const Args &a) {
    enum { parent, lengths, q, k_cache, v_cache, table, scale, out, status, workspace, plain };
    const Array tq(a[q]);
    dimensions(tq, 4);
    const int64_t B = tq.size(0), N = tq.size(1), H = tq.size(2), P = tq.size(3);
    const stree_kv kv = make_kv(a[k_cache], a[v_cache], a[table], false);
    require(kv.headdim == P && kv.io_dtype == rows_code(a[q]), "q and the cache agree in headdim and dtype");
    require(Array(a[table]).size(0) == B, "a row of the table per sequence");
    stree_attn d = {};
    d.batch = int_of(B), d.nnodes = int_of(N), d.nheads = int_of(H), d.flags = truth(a[plain]) ? STREE_ATTN_PLAIN : 0;
    if (a[scale] != Py_None) {
        d.softmax_scale = number_of(a[scale]);
        require(d.softmax_scale != 0.f, "a scale other than 0");
    }
    d.q_stride_n = rows_stride(tq, B, N);
    const int32_t *p0 = make_parent(a[parent], B, N), *p1 = numbers(a[lengths], {B}, "lengths int32 [B]");
    int32_t *p2 = numbers_or_none(a[status], {B}, "status int32 [B]");
    Result o;
    sized(o, a[out], a[q], {B, N, H, P}, a[q]);
    require(o.t().shaped({B, N, H, P}) && o.t().same_type(tq) && o.t().is_contiguous(), "out [B,N,H,P], dense");
    on_device({a[parent], a[lengths], a[q], a[k_cache], a[v_cache], a[table], a[out], a[status], a[workspace]});
    // scratch: the caller's, or torch's for this call (its memory goes back to the stream's pool when the call returns)
    size_t bytes = g_entry.attn_workspace_bytes(&d, &kv);
    if (bytes == (size_t)-1) bytes = 0;              // (the call says what is wrong)
    at::Tensor scratch;
    void *p3 = nullptr;
    if (a[workspace] != Py_None) {
        const Array w(a[workspace]);
        require(w.is_contiguous(), "a dense workspace");
        p3 = w.data_ptr();
        bytes = (size_t)(w.numel() * w.element_size());
    } else if (bytes) {
        scratch = at::empty({(int64_t)bytes}, THPVariable_Unpack(a[q].o).options().dtype(at::kByte).requires_grad(false));
        p3 = scratch.data_ptr();
    }
    const void *p4 = pointer(a[q]);
    void *p5 = o.ptr(), *st = stream();
    run("stree_tree_attn", [&] { return g_entry.tree_attn(&d, &kv, p0, p1, p4, p5, p2, p3, bytes, st); });
    return o.release();
}

PyObject *attn_workspace(const Args &a) {
    enum { q, k_cache, v_cache, table };
    const Array tq(a[q]);
    dimensions(tq, 4);
    const stree_kv kv = make_kv(a[k_cache], a[v_cache], a[table], false);
    stree_attn d = {};
    d.batch = int_of(tq.size(0)), d.nnodes = int_of(tq.size(1)), d.nheads = int_of(tq.size(2));
    const size_t bytes = g_entry.attn_workspace_bytes(&d, &kv);
    if (bytes == (size_t)-1) raise(PyExc_ValueError, "sizes outside the envelope");
    return PyLong_FromSize_t(bytes);
}

PyObject *commit_rows(const Args &a) {
    enum { parent, accepted, lengths, k_cache, v_cache, table, lengths_out, status, nnodes };
    const stree_kv kv = make_kv(a[k_cache], a[v_cache], a[table], true);
    const int64_t B = Array(a[table]).size(0);
    int64_t N;
    if (a[parent] == Py_None) {
        N = integer(a[nnodes]);                      // (a chain's length stands nowhere else)
    } else {
        const Array tp(a[parent]);
        dimensions(tp, 2);
        N = tp.size(1);
    }
    stree_attn d = {};
    d.batch = int_of(B), d.nnodes = int_of(N), d.nheads = kv.nheads_kv;
    const int32_t *p0 = make_parent(a[parent], B, N), *p1 = numbers(a[accepted], {B}, "accepted int32 [B]");
    const int32_t *p2 = numbers(a[lengths], {B}, "lengths int32 [B]");
    int32_t *p3 = numbers_or_none(a[status], {B}, "status int32 [B]");
    if (a[lengths_out] != Py_None) numbers(a[lengths_out], {B}, "lengths_out int32 [B]");
    on_device({a[parent], a[accepted], a[lengths], a[k_cache], a[v_cache], a[table], a[lengths_out], a[status]});
    Result o;
    like(o, a[lengths_out], a[lengths]);
    const auto p4 = (int32_t *)o.ptr();
    void *st = stream();
    run("stree_commit_kv", [&] { return g_entry.commit_kv(&d, &kv, p0, p1, p2, p4, p3, st); });
    return o.release();
}

stree_pool make_pool(Arg held, int64_t batch, Arg refs, Arg free, Arg nfree, int npages) {
    stree_pool p = {};
    p.held = numbers(held, {batch}, "held int32 [B]");
    p.refs = numbers(refs, {npages}, "refs int32 [pages]"), p.free = numbers(free, {npages}, "free int32 [pages]");
    p.nfree = numbers(nfree, {1}, "nfree int32 [1]");
    return p;
}

PyObject *resize(const Args &a) {
    enum { tokens, held, table, refs, free, nfree, page, status };
    const Array t(a[table]), r(a[refs]);
    dimensions(t, 2);
    dimensions(r, 1);
    const int64_t B = t.size(0);
    stree_kv kv = {};
    kv.nlayers = kv.nheads_kv = kv.headdim = 1;      // (no rows are moved)
    const int64_t size = integer(a[page]);
    kv.npages = int_of(r.size(0)), kv.max_pages = int_of(t.size(1)), kv.page = int_of(size);
    kv.table = numbers(a[table], {B, t.size(1)}, "table int32 [B, max_pages], dense");
    const stree_pool p = make_pool(a[held], B, a[refs], a[free], a[nfree], kv.npages);
    const int32_t *p0 = numbers(a[tokens], {B}, "tokens int32 [B]");
    int32_t *p1 = numbers_or_none(a[status], {B}, "status int32 [B]");
    on_device({a[tokens], a[held], a[table], a[refs], a[free], a[nfree], a[status]});
    void *st = stream();
    run("stree_resize_kv", [&] { return g_entry.resize_kv(&kv, &p, (int)B, p0, p1, st); });
    Py_INCREF(a[held].o);
    return a[held].o;
}

PyObject *fork_rows(const Args &a) {
    enum { src, dst, lengths, held, table, refs, free, nfree, k_cache, v_cache, status };
    const stree_kv kv = make_kv(a[k_cache], a[v_cache], a[table], true);
    const int64_t B = Array(a[table]).size(0);
    const Array s(a[src]);
    dimensions(s, 1);
    const int64_t F = s.size(0);
    const stree_pool p = make_pool(a[held], B, a[refs], a[free], a[nfree], kv.npages);
    const int32_t *p0 = numbers(a[src], {F}, "src int32 [forks]"), *p1 = numbers(a[dst], {F}, "dst int32 [forks]");
    int32_t *p2 = numbers(a[lengths], {B}, "lengths int32 [B]");
    if (a[status] != Py_None) numbers(a[status], {F}, "status int32 [forks]");
    on_device({a[src], a[dst], a[lengths], a[held], a[table], a[refs], a[free], a[nfree], a[k_cache], a[v_cache], a[status]});
    Result o;
    like(o, a[status], a[src]);
    const auto p3 = (int32_t *)o.ptr();
    void *st = stream();
    run("stree_fork_kv", [&] { return g_entry.fork_kv(&kv, &p, (int)B, int_of(F), p0, p1, p2, p3, st); });
    return o.release();
}

// entry points and how many arguments each takes
#define STREE_KV_METHODS(METHOD)                                                                                     \
    METHOD("tree_rope", rope, 16), METHOD("tree_attn", attn, 11), METHOD("attn_workspace", attn_workspace, 4),       \
        METHOD("commit_kv", commit_rows, 9), METHOD("resize_kv", resize, 8), METHOD("fork_kv", fork_rows, 11)
