// Python module _marshal: the checks and the argument passing of the attention operators' binding.
//
// Calls of these operators take 4 us on the GPU at the least and up to fifteen tensors each; read through Python attributes and
// ctypes their arguments cost 5 to 7 us of the host's time, here below one (the launch itself is 3.5).  Nothing is computed
// and nothing kept: every function checks types, shapes, strides and devices, allocates outputs that were not
// given, passes addresses and the current stream to the C entry of the same name, and counts the caller's outputs as
// changed in place.  The documented functions
// are those of binding.py, which also turns the status into an error.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "lory.h"

namespace {

struct Raised {};   // a Python error is set

[[noreturn]] void raise(PyObject *type, const char *format, ...)
{
    va_list args;
    va_start(args, format);
    PyErr_FormatV(type, format, args);
    va_end(args);
    throw Raised();
}

struct Call {
    PyObject *const *args;
    int device = -1;                   // of the first tensor
    const char *elsewhere = nullptr;   // an argument that is on no GPU, or on another one
    at::ScalarType type = at::kFloat;  // of the heads
    int written[9], outputs = 0;       // arguments that the call writes into

    const at::Tensor &tensor(int i, const char *name)
    {
        if (!THPVariable_Check(args[i])) raise(PyExc_TypeError, "%s must be a tensor", name);
        return THPVariable_Unpack(args[i]);
    }
    bool none(int i) const { return args[i] == Py_None; }
    void on_gpu(const at::Tensor &t, const char *name)
    {
        if (device < 0 && t.is_cuda()) device = t.get_device();
        if (!elsewhere && (!t.is_cuda() || t.get_device() != device)) elsewhere = name;
    }
    // The current stream.  What is on a wrong device is reported here, last: no address has been used until then.
    void *stream()
    {
        if (elsewhere) raise(PyExc_ValueError, "%s must live on the GPU, with all other tensors", elsewhere);
        const c10::hip::HIPStream s = c10::hip::getCurrentHIPStream();
        if (s.device_index() != device) raise(PyExc_ValueError, "the tensors must live on the current GPU");
        return (void *)s.stream();
    }
    // The caller's tensors at these places are outputs (None: a new one).
    void writes(std::initializer_list<int> at)
    {
        for (const int i : at)
            if (!none(i)) written[outputs++] = i;
    }
    // Status of the C entry.  Outputs have changed by now: autograd is to know if a graph had kept one of them.
    int done(int status)
    {
        for (int i = 0; status == LORY_OK && i < outputs; ++i) {
            const at::Tensor &t = THPVariable_Unpack(args[written[i]]);
            if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
        }
        return status;
    }
    void of_type(const at::Tensor &t, at::ScalarType want, const char *name)
    {
        if (t.scalar_type() != want) raise(PyExc_TypeError, "%s must be %s", name, c10::toString(want));
    }

    // dtype code of the tensor that the others are held against
    int dtype(const at::Tensor &t, const char *name)
    {
        type = t.scalar_type();
        if (type == at::kFloat) return LORY_F32;
        if (type == at::kBFloat16) return LORY_BF16;
        raise(PyExc_TypeError, "unsupported dtype %s of %s", c10::toString(type), name);
    }

    // [n, heads, dim] as it lies; only the last index has to be contiguous
    lory_heads heads(const at::Tensor &t, int64_t n, int64_t heads, int64_t dim, const char *name)
    {
        of_type(t, type, name);
        if (t.dim() != 3 || t.size(0) != n || t.size(1) != heads || t.size(2) != dim)
            raise(PyExc_ValueError, "%s must be [%lld, %lld, %lld]", name, (long long)n, (long long)heads, (long long)dim);
        if (dim > 1 && t.stride(2) != 1) raise(PyExc_ValueError, "the last dimension of %s must be contiguous", name);
        on_gpu(t, name);
        return {t.data_ptr(), t.stride(0), t.stride(1)};
    }
    void *array(const at::Tensor &t, at::ScalarType want, int64_t n, const char *name)
    {
        if (t.scalar_type() != want || t.dim() != 1 || t.size(0) != n)
            raise(PyExc_ValueError, "%s must be %s [%lld]", name, c10::toString(want), (long long)n);
        return contiguous(t, name);
    }
    void *contiguous(const at::Tensor &t, const char *name)
    {
        if (!t.is_contiguous()) raise(PyExc_ValueError, "%s must be contiguous", name);
        on_gpu(t, name);
        return t.data_ptr();
    }
    template <typename E> E *array(int i, at::ScalarType want, int64_t n, const char *name)
    {
        return (E *)array(tensor(i, name), want, n, name);
    }
    int32_t *ints(int i, int64_t n, const char *name) { return array<int32_t>(i, at::kInt, n, name); }
    int size32(int64_t n, const char *name)
    {
        if (n > INT32_MAX) raise(PyExc_ValueError, "%s is too large", name);
        return (int)n;
    }
    int32_t *table(int i, int64_t rows, int &width, int64_t &row, const char *name = "table")
    {
        const at::Tensor &t = tensor(i, name);
        if (t.scalar_type() != at::kInt || t.dim() != 2 || t.size(0) != rows || (t.size(1) > 1 && t.stride(1) != 1))
            raise(PyExc_ValueError, "%s must be int32 [%lld, width] with contiguous rows", name, (long long)rows);
        on_gpu(t, name);
        width = size32(t.size(1), name);
        row = rows > 1 ? t.stride(0) : width;
        return (int32_t *)t.data_ptr();
    }
    void *cache(int i, int64_t heads, int64_t dim, int &pages, int &page, const char *name)
    {
        const at::Tensor &t = tensor(i, name);
        of_type(t, type, name);
        const bool first = pages < 0;
        if (t.dim() != 4 || t.size(1) != heads || t.size(3) != dim || (!first && (t.size(0) != pages || t.size(2) != page)))
            raise(PyExc_ValueError, "k_cache and v_cache must be [pages, %lld, page, %lld]", (long long)heads, (long long)dim);
        pages = size32(t.size(0), name);
        page = size32(t.size(2), name);
        return contiguous(t, name);
    }
    // the output that was given, or a new one of the input's shape
    at::Tensor output(int i, const at::Tensor &like, const char *name)
    {
        return none(i) ? at::empty(like.sizes(), like.options()) : tensor(i, name);
    }
    void *workspace(int i, size_t &bytes)
    {
        if (none(i)) return nullptr;
        const at::Tensor &t = tensor(i, "workspace");
        bytes = t.numel() * t.element_size();
        return contiguous(t, "workspace");
    }
};

double number(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Raised();
    return v;
}

int whole(PyObject *o, const char *name)
{
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised();
    if (v < INT32_MIN || v > INT32_MAX) raise(PyExc_ValueError, "%s is too large", name);
    return (int)v;
}

// What the three rope calls share: q, k at 0 and 1; pos, freq, wq, wk, eps, interleaved from `at` on.
struct Rope {
    lory_rope_shape shape;
    lory_heads q, k;
    const int32_t *pos;
    const double *freq;
    const void *wq = nullptr, *wk = nullptr;
    int64_t n, Hq, Hkv, D;

    Rope(Call &c, int at)
    {
        const at::Tensor &tq = c.tensor(0, "q"), &tk = c.tensor(1, "k");
        const int dtype = c.dtype(tq, "q");
        if (tq.dim() != 3 || tk.dim() != 3) raise(PyExc_ValueError, "q and k must be [tokens, heads, head_dim]");
        n = tq.size(0);
        Hq = tq.size(1);
        Hkv = tk.size(1);
        D = tq.size(2);
        q = c.heads(tq, n, Hq, D, "q");
        k = c.heads(tk, n, Hkv, D, "k");
        pos = c.ints(at, n, "pos");
        const at::Tensor &tf = c.tensor(at + 1, "freq");
        const int64_t pairs = tf.dim() == 1 ? tf.size(0) : -1;
        freq = (const double *)c.array(tf, at::kDouble, pairs, "freq");
        for (int i = 0; i < 2; ++i) {
            if (c.none(at + 2 + i)) continue;
            const char *name = i ? "wk" : "wq";
            const at::Tensor &w = c.tensor(at + 2 + i, name);
            c.of_type(w, c.type, name);
            (i ? wk : wq) = c.array(w, c.type, D, name);
        }
        const int inter = PyObject_IsTrue(c.args[at + 5]);
        if (inter < 0) throw Raised();
        shape = {c.size32(n, "q"), c.size32(Hq, "q"), c.size32(Hkv, "k"), c.size32(D, "q"), c.size32(2 * pairs, "freq"), inter,
                 dtype, (float)number(c.args[at + 4])};
    }
};

PyObject *result(int status, std::initializer_list<at::Tensor> out)
{
    PyObject *t = PyTuple_New(1 + out.size());
    if (!t) throw Raised();
    PyTuple_SET_ITEM(t, 0, PyLong_FromLong(status));
    int i = 1;
    for (const at::Tensor &x : out) {
        PyObject *o;
        if (x.defined()) {
            o = THPVariable_Wrap(x);
            if (!o) {
                Py_DECREF(t);
                throw Raised();
            }
        } else {
            Py_INCREF(Py_None);
            o = Py_None;
        }
        PyTuple_SET_ITEM(t, i++, o);
    }
    return t;
}

typedef PyObject *(*Body)(Call &c);

// Runs a call; no C++ exception leaves it.
template <Body body, int N> PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != N) return PyErr_Format(PyExc_TypeError, "%d arguments expected", N);
    try {
        Call c = {args};
        return body(c);
    } catch (const Raised &) {
        return nullptr;
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
        return nullptr;
    }
}

// q, k, pos, freq, wq, wk, eps, interleaved, q_out, k_out
PyObject *qk_rope(Call &c)
{
    const Rope r(c, 2);
    const at::Tensor tq = c.output(8, c.tensor(0, "q"), "q_out"), tk = c.output(9, c.tensor(1, "k"), "k_out");
    const lory_heads q = c.heads(tq, r.n, r.Hq, r.D, "q_out"), k = c.heads(tk, r.n, r.Hkv, r.D, "k_out");
    void *stream = c.stream();
    c.writes({8, 9});
    return result(c.done(lory_qk_rope(&r.shape, &r.q, &r.k, r.pos, r.freq, r.wq, r.wk, &q, &k, stream)), {tq, tk});
}

// q, k, pos, freq, wq, wk, eps, interleaved, v, k_cache, v_cache, slots, q_out
PyObject *qk_rope_cache(Call &c)
{
    const Rope r(c, 2);
    const lory_heads v = c.heads(c.tensor(8, "v"), r.n, r.Hkv, r.D, "v");
    int pages = -1, page = -1;
    void *kc = c.cache(9, r.Hkv, r.D, pages, page, "k_cache"), *vc = c.cache(10, r.Hkv, r.D, pages, page, "v_cache");
    const int64_t *slots = c.array<int64_t>(11, at::kLong, r.n, "slots");
    const at::Tensor tq = c.output(12, c.tensor(0, "q"), "q_out");
    const lory_heads q = c.heads(tq, r.n, r.Hq, r.D, "q_out");
    void *stream = c.stream();
    c.writes({9, 10, 12});
    return result(c.done(lory_qk_rope_cache(&r.shape, &r.q, &r.k, &v, r.pos, r.freq, r.wq, r.wk, &q, kc, vc, pages, page, slots,
                                            stream)), {tq});
}

// q, k, pos, freq, wq, wk, eps, interleaved, dq_out, dk_out, dq, dk, dwq, dwk, workspace
PyObject *qk_rope_bwd(Call &c)
{
    const Rope r(c, 2);
    const at::Tensor &q = c.tensor(0, "q"), &k = c.tensor(1, "k");
    const lory_heads dyq = c.heads(c.tensor(8, "dq_out"), r.n, r.Hq, r.D, "dq_out"),
                     dyk = c.heads(c.tensor(9, "dk_out"), r.n, r.Hkv, r.D, "dk_out");
    const at::Tensor tq = c.output(10, q, "dq"), tk = c.output(11, k, "dk");
    const lory_heads dq = c.heads(tq, r.n, r.Hq, r.D, "dq"), dk = c.heads(tk, r.n, r.Hkv, r.D, "dk");
    at::Tensor dw[2], own;
    float *pw[2] = {nullptr, nullptr};
    void *ws = nullptr;
    size_t bytes = 0;
    if (r.wq || r.wk) {
        for (int i = 0; i < 2; ++i) {
            const char *name = i ? "dwk" : "dwq";
            dw[i] = c.none(12 + i) ? at::empty({r.D}, q.options().dtype(at::kFloat)) : c.tensor(12 + i, name);
            pw[i] = (float *)c.array(dw[i], at::kFloat, r.D, name);
        }
        ws = c.workspace(14, bytes);
        if (c.none(14) && lory_qk_rope_workspace_bytes(&r.shape, &bytes) == LORY_OK && bytes > 0) {
            own = at::empty({(int64_t)bytes}, q.options().dtype(at::kByte));
            ws = own.data_ptr();
        }
    } else if (!c.none(12) || !c.none(13)) {
        raise(PyExc_ValueError, "dwq and dwk need wq and wk");
    }
    void *stream = c.stream();
    c.writes({10, 11, 12, 13});
    return result(c.done(lory_qk_rope_bwd(&r.shape, &r.q, &r.k, &dyq, &dyk, r.pos, r.freq, r.wq, r.wk, &dq, &dk, pw[0], pw[1], ws,
                                          bytes, stream)), {tq, tk, dw[0], dw[1]});
}

// lens, add, table, free, count, page, lens_new, cu, positions, slots, count_new, status
PyObject *kv_plan(Call &c)
{
    const at::Tensor &lens = c.tensor(0, "lens"), &free = c.tensor(3, "free"), &positions = c.tensor(8, "positions");
    const int64_t B = lens.dim() == 1 ? lens.size(0) : -1, F = free.dim() == 1 ? free.size(0) : -1,
                  room = positions.dim() == 1 ? positions.size(0) : -1;
    lory_plan_shape s = {c.size32(B, "lens"), 0, whole(c.args[5], "page"), c.size32(F, "free"), c.size32(room, "positions"), 0};
    int32_t *p[11] = {c.ints(0, B, "lens"), c.ints(1, B, "add"), c.table(2, B, s.width, s.table_row), c.ints(3, F, "free"),
                      c.ints(4, 1, "count"), c.ints(6, B, "lens_new"), c.ints(7, B + 1, "cu"), c.ints(8, room, "positions"),
                      nullptr, c.ints(10, 1, "count_new"), c.ints(11, 1, "status")};
    int64_t *slots = c.array<int64_t>(9, at::kLong, room, "slots");
    void *stream = c.stream();
    c.writes({2, 3, 6, 7, 8, 9, 10, 11});
    return PyLong_FromLong(c.done(lory_kv_plan(&s, p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], slots, p[9], p[10], stream)));
}

// What the two attention calls share: q, k_cache, v_cache, table, lens at 0 to 4.
struct Paged {
    lory_paged_shape s = {};
    lory_heads q;
    const void *k, *v;
    const int32_t *table, *lens;
    int64_t B, Hq, D;

    Paged(Call &c, PyObject *scale)
    {
        const at::Tensor &tq = c.tensor(0, "q");
        s.dtype = c.dtype(tq, "q");
        if (tq.dim() != 3) raise(PyExc_ValueError, "q must be [rows, heads, head_dim]");
        B = tq.size(0), Hq = tq.size(1), D = tq.size(2);
        q = c.heads(tq, B, Hq, D, "q");
        const at::Tensor &kc = c.tensor(1, "k_cache");
        const int64_t Hkv = kc.dim() == 4 ? kc.size(1) : -1;
        s.pages = s.page = -1;
        k = c.cache(1, Hkv, D, s.pages, s.page, "k_cache"), v = c.cache(2, Hkv, D, s.pages, s.page, "v_cache");
        table = c.table(3, B, s.width, s.table_row), lens = c.ints(4, B, "lens");
        s.rows = c.size32(B, "q");
        s.q_heads = c.size32(Hq, "q");
        s.kv_heads = c.size32(Hkv, "k_cache");
        s.head_dim = c.size32(D, "q");
        s.scale = scale == Py_None ? (float)(1.0 / std::sqrt((double)(D > 0 ? D : 1))) : (float)number(scale);
    }
    float *lse(Call &c, int i) const
    {
        if (c.none(i)) return nullptr;
        const at::Tensor &t = c.tensor(i, "lse");
        if (t.scalar_type() != at::kFloat || t.dim() != 2 || t.size(0) != B || t.size(1) != Hq)
            raise(PyExc_ValueError, "lse must be fp32 [%lld, %lld]", (long long)B, (long long)Hq);
        return (float *)c.contiguous(t, "lse");
    }
};

// The workspace that was given at i, or a new one of the size that `size` reports.
template <typename Size> void *workspace_or_new(Call &c, int i, size_t &bytes, at::Tensor &own, const at::Tensor &like, const Size &size)
{
    void *ws = c.workspace(i, bytes);
    if (c.none(i) && size(&bytes) == LORY_OK && bytes > 0) {
        own = at::empty({(int64_t)bytes}, like.options().dtype(at::kByte));
        ws = own.data_ptr();
    }
    return ws;
}

// q, k_cache, v_cache, table, lens, scale, out, lse, workspace
PyObject *paged_attn(Call &c)
{
    const Paged p(c, c.args[5]);
    const at::Tensor &tq = c.tensor(0, "q");
    const at::Tensor to = c.output(6, tq, "out");
    const lory_heads out = c.heads(to, p.B, p.Hq, p.D, "out");
    float *lse = p.lse(c, 7);
    size_t bytes = 0;
    at::Tensor own;
    void *ws = workspace_or_new(c, 8, bytes, own, tq, [&](size_t *n) { return lory_paged_attn_workspace_bytes(&p.s, n); });
    void *stream = c.stream();
    c.writes({6, 7});
    return result(c.done(lory_paged_attn(&p.s, &p.q, p.k, p.v, p.table, p.lens, &out, lse, ws, bytes, stream)), {to});
}

// q, k_cache, v_cache, table, lens, shared, scale, out, lse, workspace
PyObject *prefix_attn(Call &c)
{
    const Paged p(c, c.args[6]);
    const at::Tensor &tq = c.tensor(0, "q"), &ts = c.tensor(5, "shared");
    const int64_t G = ts.dim() == 1 ? ts.size(0) : -1;
    const int32_t *shared = c.ints(5, G, "shared");
    const int groups = c.size32(G, "shared");
    if (groups > 0 ? p.B % groups != 0 || p.B == 0 : p.B != 0)
        raise(PyExc_ValueError, "shared must have a value for every group of neighbouring rows: %lld rows, %d groups", (long long)p.B, groups);
    const at::Tensor to = c.output(7, tq, "out");
    const lory_heads out = c.heads(to, p.B, p.Hq, p.D, "out");
    float *lse = p.lse(c, 8);
    size_t bytes = 0;
    at::Tensor own;
    void *ws = workspace_or_new(c, 9, bytes, own, tq, [&](size_t *n) { return lory_prefix_attn_workspace_bytes(&p.s, groups, n); });
    void *stream = c.stream();
    c.writes({7, 8});
    return result(c.done(lory_prefix_attn(&p.s, groups, &p.q, p.k, p.v, p.table, p.lens, shared, &out, lse, ws, bytes, stream)), {to});
}

// logits, score, k, score_out, token, parent, workspace
PyObject *beam_select(Call &c)
{
    const at::Tensor &x = c.tensor(0, "logits"), &score = c.tensor(1, "score");
    lory_beam_shape s = {};
    s.dtype = c.dtype(x, "logits");
    if (score.scalar_type() != at::kFloat || score.dim() != 2) raise(PyExc_ValueError, "score must be fp32 [requests, beams]");
    const int64_t R = score.size(0), K = score.size(1);
    const float *sc = (const float *)c.contiguous(score, "score");
    if (x.dim() != 2 || x.size(0) != R * K || (x.size(1) > 1 && x.stride(1) != 1))
        raise(PyExc_ValueError, "logits must be [%lld, vocab] with contiguous rows", (long long)(R * K));
    c.on_gpu(x, "logits");
    s.requests = c.size32(R, "score");
    s.beams = c.size32(K, "score");
    s.vocab = c.size32(x.size(1), "logits");
    s.k = whole(c.args[2], "k");
    s.row = R * K > 1 ? x.stride(0) : s.vocab;
    at::Tensor out[3];
    void *p[3];
    const char *const names[3] = {"score_out", "token", "parent"};
    for (int i = 0; i < 3; ++i) {
        const at::ScalarType type = i ? at::kInt : at::kFloat;
        out[i] = c.none(3 + i) ? at::empty({R, s.k > 0 ? s.k : 0}, score.options().dtype(type)) : c.tensor(3 + i, names[i]);
        if (out[i].scalar_type() != type || out[i].dim() != 2 || out[i].size(0) != R || out[i].size(1) != s.k)
            if (s.k > 0) raise(PyExc_ValueError, "%s must be %s [%lld, %d]", names[i], c10::toString(type), (long long)R, s.k);
        p[i] = c.contiguous(out[i], names[i]);
    }
    size_t bytes = 0;
    at::Tensor own;
    void *ws = workspace_or_new(c, 6, bytes, own, x, [&](size_t *n) { return lory_beam_select_workspace_bytes(&s, n); });
    void *stream = c.stream();
    c.writes({3, 4, 5});
    return result(c.done(lory_beam_select(&s, x.data_ptr(), sc, (float *)p[0], (int32_t *)p[1], (int32_t *)p[2], ws, bytes, stream)),
                  {out[0], out[1], out[2]});
}

// lens, src, table, free, count, page, pages, lens_new, table_new, count_new, copies, status, workspace
PyObject *kv_fork(Call &c)
{
    const at::Tensor &lens = c.tensor(0, "lens"), &src = c.tensor(1, "src"), &free = c.tensor(3, "free"), &copies = c.tensor(10, "copies");
    const int64_t old = lens.dim() == 1 ? lens.size(0) : -1, N = src.dim() == 1 ? src.size(0) : -1, F = free.dim() == 1 ? free.size(0) : -1;
    lory_fork_shape s = {c.size32(old, "lens"), c.size32(N, "src"), 0, whole(c.args[5], "page"), whole(c.args[6], "pages"),
                         c.size32(F, "free"), 0, 0};
    int32_t *p[9] = {c.ints(0, old, "lens"), c.ints(1, N, "src"), c.table(2, old, s.width, s.table_row), c.ints(3, F, "free"),
                     c.ints(4, 1, "count"), c.ints(7, N, "lens_new"), nullptr, c.ints(9, 1, "count_new"), c.ints(11, 1, "status")};
    int width = 0;
    p[6] = c.table(8, N, width, s.new_row, "table_new");
    if (width != s.width) raise(PyExc_ValueError, "table_new must have the width of table, %d", s.width);
    if (copies.scalar_type() != at::kInt || copies.dim() != 2 || copies.size(0) != 3 || copies.size(1) != N)
        raise(PyExc_ValueError, "copies must be int32 [3, %lld]", (long long)N);
    int32_t *pc = (int32_t *)c.contiguous(copies, "copies");
    size_t bytes = 0;
    at::Tensor own;
    void *ws = workspace_or_new(c, 12, bytes, own, lens, [&](size_t *n) { return lory_kv_fork_workspace_bytes(&s, n); });
    void *stream = c.stream();
    c.writes({3, 7, 8, 9, 10, 11});
    return PyLong_FromLong(c.done(lory_kv_fork(&s, p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], pc, p[8], ws, bytes, stream)));
}

// k_cache, v_cache, copies
PyObject *kv_copy(Call &c)
{
    const at::Tensor &k = c.tensor(0, "k_cache"), &v = c.tensor(1, "v_cache"), &copies = c.tensor(2, "copies");
    lory_copy_shape s = {};
    s.dtype = c.dtype(k, "k_cache");
    c.of_type(v, c.type, "v_cache");
    const int64_t d = k.dim();
    if ((d != 4 && d != 5) || v.sizes() != k.sizes())
        raise(PyExc_ValueError, "k_cache and v_cache must be [pages, heads, page, head_dim], or [layers, ...] of that");
    void *pk = c.contiguous(k, "k_cache"), *pv = c.contiguous(v, "v_cache");
    if (copies.scalar_type() != at::kInt || copies.dim() != 2 || copies.size(0) != 3) raise(PyExc_ValueError, "copies must be int32 [3, n]");
    const int32_t *pc = (const int32_t *)c.contiguous(copies, "copies");
    s.n = c.size32(copies.size(1), "copies");
    s.layers = d == 5 ? c.size32(k.size(0), "k_cache") : 1;
    s.pages = c.size32(k.size(d - 4), "k_cache");
    s.kv_heads = c.size32(k.size(d - 3), "k_cache");
    s.page = c.size32(k.size(d - 2), "k_cache");
    s.head_dim = c.size32(k.size(d - 1), "k_cache");
    void *stream = c.stream();
    c.writes({0, 1});
    return PyLong_FromLong(c.done(lory_kv_copy(&s, pk, pv, pc, stream)));
}

PyMethodDef methods[] = {
    {"qk_rope", (PyCFunction)(void (*)(void))entry<qk_rope, 10>, METH_FASTCALL, nullptr},
    {"qk_rope_cache", (PyCFunction)(void (*)(void))entry<qk_rope_cache, 13>, METH_FASTCALL, nullptr},
    {"qk_rope_bwd", (PyCFunction)(void (*)(void))entry<qk_rope_bwd, 15>, METH_FASTCALL, nullptr},
    {"kv_plan", (PyCFunction)(void (*)(void))entry<kv_plan, 12>, METH_FASTCALL, nullptr},
    {"paged_attn", (PyCFunction)(void (*)(void))entry<paged_attn, 9>, METH_FASTCALL, nullptr},
    {"prefix_attn", (PyCFunction)(void (*)(void))entry<prefix_attn, 10>, METH_FASTCALL, nullptr},
    {"beam_select", (PyCFunction)(void (*)(void))entry<beam_select, 7>, METH_FASTCALL, nullptr},
    {"kv_fork", (PyCFunction)(void (*)(void))entry<kv_fork, 13>, METH_FASTCALL, nullptr},
    {"kv_copy", (PyCFunction)(void (*)(void))entry<kv_copy, 3>, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "Argument passing of the attention operators.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
