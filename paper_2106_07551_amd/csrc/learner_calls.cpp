// The learner operators' calls from Python: the checks, allocations and descriptions
// of the binding's functions in one native call.  Small calls are bound by the host: a
// policy loss of 192 rows took 14.7 us through ctypes, of which the launch is 3.
//
// Every function takes device tensors as the binding's function of that name, and
// the raw stream last.  It returns None, having launched nothing, for arguments that it does
// not take (other types or layouts, what the library refuses, memory that cannot be
// had): the binding's own checks then name the error.  A launch that failed is raised: an
// earlier one of the call may have run, over an input that is an output too.
#include <Python.h>

#include <ATen/ATen.h>
#include <dlfcn.h>
#include <torch/csrc/autograd/python_variable.h>

#include "malib.h"

namespace {

decltype(&malib_linear) p_linear;
decltype(&malib_linear_backward) p_linear_backward;
decltype(&malib_linear_work) p_linear_work;
decltype(&malib_policy_loss) p_policy_loss;
decltype(&malib_distill_loss) p_distill_loss;
decltype(&malib_loss_work) p_loss_work;

// An argument that these functions do not take.
struct Other {};

// A Python error that is set.
struct Raised {};

void need(bool ok)
{
    if (!ok)
        throw Other();
}

// An optional tensor argument on the device.
class Arg {
  public:
    explicit Arg(PyObject* o) : obj_(o)
    {
        if (o == Py_None)
            return;
        need(THPVariable_Check(o));
        t_ = &THPVariable_Unpack(o);
        need(t_->is_cuda() && t_->layout() == at::kStrided);
    }
    explicit operator bool() const { return t_ != nullptr; }
    const at::Tensor& operator*() const { return *t_; }
    const at::Tensor* operator->() const { return t_; }
    void* ptr() const { return t_ ? t_->data_ptr() : nullptr; }
    PyObject* object() const { return obj_; }

  private:
    PyObject* obj_;
    const at::Tensor* t_ = nullptr;
};

// An output: the caller's tensor or a new one.
struct Out {
    explicit Out(const Arg& a) : given(a) {}
    void make(at::IntArrayRef shape, at::ScalarType type, const at::Tensor& like)
    {
        fresh = at::empty(shape, like.options().dtype(type));
    }
    const at::Tensor& tensor() const { return given ? *given : fresh; }
    // a new reference
    PyObject* object() const
    {
        if (!given)
            return fresh.defined() ? THPVariable_Wrap(fresh) : Py_NewRef(Py_None);
        return Py_NewRef(given.object());
    }
    void* ptr() const
    {
        return given ? given.ptr() : fresh.defined() ? fresh.data_ptr() : nullptr;
    }
    Arg given;
    at::Tensor fresh;
};

int type_code(const at::Tensor& t)
{
    need(t.scalar_type() == at::kFloat || t.scalar_type() == at::kBFloat16);
    return t.scalar_type() == at::kBFloat16 ? MALIB_DT_BF16 : MALIB_DT_F32;
}

int64_t integer(PyObject* o)
{
    const int64_t v = PyLong_AsLongLong(o);
    need(!(v == -1 && PyErr_Occurred()));
    return v;
}

float real(PyObject* o)
{
    const double v = PyFloat_AsDouble(o);
    need(!(v == -1.0 && PyErr_Occurred()));
    return (float)v;
}

bool truth(PyObject* o)
{
    const int v = PyObject_IsTrue(o);
    need(v >= 0);
    return v != 0;
}

// [rows][cols], or [groups][rows][cols] where `grouped`, with contiguous rows
malib_mat matrix(const at::Tensor& t, at::ScalarType type, bool grouped, int64_t groups,
                 int64_t rows, int64_t cols)
{
    const auto size = t.sizes();
    need(t.scalar_type() == type && (int)size.size() == 2 + grouped);
    need(size[grouped] == rows && size[1 + grouped] == cols && (!grouped || size[0] == groups));
    const auto stride = t.strides();
    need(stride[1 + grouped] == 1 || cols <= 1);
    const int64_t row = rows > 1 ? stride[grouped] : cols;
    return {t.data_ptr(), row, grouped ? (groups > 1 ? stride[0] : rows * row) : 0};
}

void buffer(const Arg& a, at::ScalarType type, int64_t numel)
{
    if (a)
        need(a->scalar_type() == type && a->numel() == numel && a->is_contiguous());
}

// Row stride of [n][a] with contiguous rows
int64_t row_stride(const at::Tensor& t, int64_t n, int64_t a)
{
    need(t.dim() == 2 && t.size(0) == n && t.size(1) == a && (t.stride(1) == 1 || a <= 1));
    return n > 1 ? t.stride(0) : a;
}

// A call's workspace: the caller's, or a new one.
struct Work {
    Work(const Arg& given, int64_t bytes, const at::Tensor& like)
    {
        if (given) {
            need(given->is_contiguous() && (int64_t)given->nbytes() >= bytes);
            ptr = given.ptr();
            size = (int64_t)given->nbytes();
        } else if (bytes > 0) {
            own = at::empty({bytes}, like.options().dtype(at::kByte));
            ptr = own.data_ptr();
            size = bytes;
        }
    }
    at::Tensor own;
    void* ptr = nullptr;
    int64_t size = 0;
};

// fn() where Other and errors of torch become None
template <typename F>
PyObject* guarded(Py_ssize_t n, Py_ssize_t want, F fn)
{
    if (n != want || !p_linear) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments, or no library loaded");
        return nullptr;
    }
    try {
        return fn();
    } catch (const Raised&) {
        return nullptr;
    } catch (...) {   // (nothing may pass the C entry)
        PyErr_Clear();
    }
    return Py_NewRef(Py_None);
}

// The error of a status as the binding raises it
[[noreturn]] void raise_status(malib_status s)
{
    PyObject* m = PyImport_ImportModule("paper_2106_07551_amd.binding");
    PyObject* r = m ? PyObject_CallMethod(m, "_check", "i", (int)s) : nullptr;
    Py_XDECREF(m);
    if (r) {
        Py_DECREF(r);
        PyErr_Format(PyExc_RuntimeError, "malib status %d", (int)s);
    }
    throw Raised();
}

// The library's call without the interpreter's lock.  `result`, made before it (behind it
// nothing may become None), is returned.
template <typename F>
PyObject* call(PyObject* result, F fn)
{
    need(result != nullptr);
    malib_status s;
    Py_BEGIN_ALLOW_THREADS
    s = fn();
    Py_END_ALLOW_THREADS
    if (s == MALIB_OK)
        return result;
    Py_DECREF(result);
    need(s != MALIB_E_INVAL && s != MALIB_E_UNSUPPORTED);   // checks, before the first launch
    raise_status(s);
}

// load(path of the library)
PyObject* load(PyObject*, PyObject* path)
{
    const char* p = PyUnicode_AsUTF8(path);
    if (!p)
        return nullptr;
    void* h = dlopen(p, RTLD_NOW | RTLD_LOCAL);
    if (h) {
        p_linear_backward = (decltype(p_linear_backward))dlsym(h, "malib_linear_backward");
        p_linear_work = (decltype(p_linear_work))dlsym(h, "malib_linear_work");
        p_policy_loss = (decltype(p_policy_loss))dlsym(h, "malib_policy_loss");
        p_distill_loss = (decltype(p_distill_loss))dlsym(h, "malib_distill_loss");
        p_loss_work = (decltype(p_loss_work))dlsym(h, "malib_loss_work");
        p_linear = (decltype(p_linear))dlsym(h, "malib_linear");
    }
    if (!h || !p_linear || !p_linear_backward || !p_linear_work || !p_policy_loss ||
        !p_distill_loss || !p_loss_work) {
        p_linear = nullptr;
        return PyErr_Format(PyExc_ImportError, "%s: not the library these calls need", p);
    }
    Py_RETURN_NONE;
}

struct Layer {
    malib_linear_desc d;
    bool grouped;
    at::ScalarType type;
};

// The layer that x (or dy) and w belong to
Layer layer(const at::Tensor& x, const at::Tensor& w, int64_t act)
{
    Layer l{};
    const auto ws = w.sizes();
    need((ws.size() == 2 || ws.size() == 3) && x.dim() == (int64_t)ws.size());
    need(act >= MALIB_ACT_NONE && act <= MALIB_ACT_SILU);
    l.grouped = ws.size() == 3;
    l.type = x.scalar_type();
    l.d.dtype = type_code(x);
    l.d.act = (int32_t)act;
    l.d.groups = l.grouped ? ws[0] : 1;
    l.d.rows = x.size(-2);
    l.d.out = ws[l.grouped];
    l.d.in = ws[1 + l.grouped];
    return l;
}

malib_mat matrix(const at::Tensor& t, const Layer& l, int64_t rows, int64_t cols)
{
    return matrix(t, l.type, l.grouped, l.d.groups, rows, cols);
}

void make(Out& o, const Layer& l, int64_t rows, int64_t cols, const at::Tensor& like)
{
    if (l.grouped)
        o.make({l.d.groups, rows, cols}, l.type, like);
    else
        o.make({rows, cols}, l.type, like);
}

int64_t layer_work(const Layer& l, int backward)
{
    int64_t bytes = 0;
    need(p_linear_work(&l.d, backward, &bytes) == MALIB_OK);
    return bytes;
}

// linear(x, w, bias, act, residual, pre, out, work, stream) -> out
PyObject* linear(PyObject*, PyObject* const* v, Py_ssize_t n)
{
    return guarded(n, 9, [&]() -> PyObject* {
        const Arg x(v[0]), w(v[1]), bias(v[2]), residual(v[4]), pre(v[5]), given(v[6]), ws(v[7]);
        void* stream = (void*)integer(v[8]);
        need(x && w);
        const Layer l = layer(*x, *w, integer(v[3]));
        const malib_linear_desc& d = l.d;
        const malib_mat mx = matrix(*x, l, d.rows, d.in), mw = matrix(*w, l, d.out, d.in);
        malib_mat mr{}, mp{};
        if (residual)
            mr = matrix(*residual, l, d.rows, d.out);
        if (pre)
            mp = matrix(*pre, l, d.rows, d.out);
        buffer(bias, at::kFloat, d.out * d.groups);
        Out out(given);
        if (!given)
            make(out, l, d.rows, d.out, *x);
        const malib_mat my = matrix(out.tensor(), l, d.rows, d.out);
        const Work work(ws, layer_work(l, 0), *x);
        return call(out.object(), [&] {
            return p_linear(&d, &mx, &mw, (const float*)bias.ptr(), residual ? &mr : nullptr,
                            pre ? &mp : nullptr, &my, work.ptr, work.size, stream);
        });
    });
}

// linear_backward(dy, x, w, act, pre, want, dx, dw, dbias, work, stream)
//   -> (dx, dw, dbias)
PyObject* linear_backward(PyObject*, PyObject* const* v, Py_ssize_t n)
{
    return guarded(n, 11, [&]() -> PyObject* {
        const Arg dy(v[0]), x(v[1]), w(v[2]), pre(v[4]), ws(v[9]);
        void* stream = (void*)integer(v[10]);
        need(dy && x && w && PyTuple_Check(v[5]) && PyTuple_GET_SIZE(v[5]) == 3);
        const Layer l = layer(*dy, *w, integer(v[3]));
        const malib_linear_desc& d = l.d;
        const bool act = d.act != MALIB_ACT_NONE;
        need(!act || pre);
        const malib_mat mdy = matrix(*dy, l, d.rows, d.out), mx = matrix(*x, l, d.rows, d.in),
                        mw = matrix(*w, l, d.out, d.in);
        malib_mat mp{}, mdx{}, mdw{};
        if (act)
            mp = matrix(*pre, l, d.rows, d.out);
        bool want[3];
        for (int i = 0; i < 3; ++i)
            want[i] = truth(PyTuple_GET_ITEM(v[5], i));
        Out dx{Arg(want[0] ? v[6] : Py_None)}, dw{Arg(want[1] ? v[7] : Py_None)},
            db{Arg(want[2] ? v[8] : Py_None)};
        if (want[0]) {
            if (!dx.given)
                make(dx, l, d.rows, d.in, *dy);
            mdx = matrix(dx.tensor(), l, d.rows, d.in);
        }
        if (want[1]) {
            if (!dw.given)
                make(dw, l, d.out, d.in, *dy);
            mdw = matrix(dw.tensor(), l, d.out, d.in);
        }
        if (want[2]) {
            buffer(db.given, at::kFloat, d.out * d.groups);
            if (!db.given && l.grouped)
                db.make({d.groups, d.out}, at::kFloat, *dy);
            else if (!db.given)
                db.make({d.out}, at::kFloat, *dy);
        }
        const Work work(ws, layer_work(l, 1), *dy);
        PyObject* result = Py_BuildValue("(NNN)", dx.object(), dw.object(), db.object());
        return call(result, [&] {
            return p_linear_backward(&d, &mdy, &mx, &mw, act ? &mp : nullptr,
                                     want[0] ? &mdx : nullptr, want[1] ? &mdw : nullptr,
                                     (float*)db.ptr(), work.ptr, work.size, stream);
        });
    });
}

// What both losses take of logits, mask and weight
struct Rows {
    int64_t n, a, logits, mask = 0;
    int dtype;

    Rows(const Arg& x, const Arg& m, const Arg& weight)
    {
        need((bool)x && x->dim() == 2 && x->size(1) >= 1);
        n = x->size(0);
        a = x->size(1);
        dtype = type_code(*x);
        logits = row_stride(*x, n, a);
        if (m) {
            need(m->scalar_type() == at::kBool || m->scalar_type() == at::kByte);
            mask = row_stride(*m, n, a);
        }
        buffer(weight, at::kFloat, n);
    }
    int64_t work() const
    {
        int64_t bytes = 0;
        need(p_loss_work(dtype, n, a, &bytes) == MALIB_OK);
        return bytes;
    }
    // of the gradient, made unless given
    int64_t gradient(Out& o, const at::Tensor& x) const
    {
        if (!o.given) {
            o.make({n, a}, x.scalar_type(), x);
            return a;
        }
        need(o.given->scalar_type() == x.scalar_type());
        return row_stride(*o.given, n, a);
    }
};

// policy_loss(logits, actions, old_logp, advantage, clip_low, clip_high, kl_coef,
//   entropy_coef, ref_logp, ref_logits, mask, weight, grad, total, stats, dlogits, work,
//   stream) -> (total, stats, dlogits)
PyObject* policy_loss(PyObject*, PyObject* const* v, Py_ssize_t n_args)
{
    return guarded(n_args, 18, [&]() -> PyObject* {
        const Arg x(v[0]), actions(v[1]), old_logp(v[2]), advantage(v[3]), ref_logp(v[8]),
            ref(v[9]), mask(v[10]), weight(v[11]), ws(v[16]);
        void* stream = (void*)integer(v[17]);
        const Rows r(x, mask, weight);
        need(actions && old_logp && advantage);
        malib_policy_loss_desc d{};
        d.dtype = r.dtype;
        d.rows = r.n;
        d.n_actions = r.a;
        d.logits_stride = r.logits;
        d.mask_stride = r.mask;
        const auto at = actions->scalar_type();
        d.action_bytes = at == at::kByte ? 1 : at == at::kInt ? 4 : at == at::kLong ? 8 : 0;
        need(d.action_bytes != 0);
        buffer(actions, at, r.n);
        buffer(old_logp, at::kFloat, r.n);
        buffer(advantage, at::kFloat, r.n);
        buffer(ref_logp, at::kFloat, r.n);
        if (ref) {
            need(ref->scalar_type() == x->scalar_type());
            d.ref_stride = row_stride(*ref, r.n, r.a);
        }
        d.clip_low = real(v[4]);
        d.clip_high = real(v[5]);
        d.kl_coef = real(v[6]);
        d.entropy_coef = real(v[7]);
        const bool grad = truth(v[12]);
        Out total{Arg(v[13])}, stats{Arg(v[14])}, dx{Arg(grad ? v[15] : Py_None)};
        buffer(total.given, at::kFloat, 1);
        buffer(stats.given, at::kFloat, 4 * r.n);
        if (!total.given)
            total.make({1}, at::kFloat, *x);
        if (!stats.given)
            stats.make({4, r.n}, at::kFloat, *x);
        if (grad)
            d.dlogits_stride = r.gradient(dx, *x);
        const Work work(ws, r.work(), *x);
        PyObject* result = Py_BuildValue("(NNN)", total.object(), stats.object(), dx.object());
        return call(result, [&] {
            return p_policy_loss(&d, x.ptr(), actions.ptr(), (const float*)old_logp.ptr(),
                                 (const float*)advantage.ptr(), (const float*)ref_logp.ptr(),
                                 ref.ptr(), (const uint8_t*)mask.ptr(),
                                 (const float*)weight.ptr(), (float*)total.ptr(),
                                 (float*)stats.ptr(), dx.ptr(), work.ptr, work.size, stream);
        });
    });
}

// distill_loss(logits, teacher_idx, teacher_logits, temperature, mask, weight, grad, total,
//   loss, dlogits, work, stream) -> (total, loss, dlogits)
PyObject* distill_loss(PyObject*, PyObject* const* v, Py_ssize_t n_args)
{
    return guarded(n_args, 12, [&]() -> PyObject* {
        const Arg x(v[0]), idx(v[1]), val(v[2]), mask(v[4]), weight(v[5]), ws(v[10]);
        void* stream = (void*)integer(v[11]);
        const Rows r(x, mask, weight);
        need((bool)idx && (bool)val && idx->dim() == 2 && idx->size(1) <= 256);
        malib_distill_desc d{};
        d.dtype = r.dtype;
        d.top = (int32_t)idx->size(1);
        d.rows = r.n;
        d.n_actions = r.a;
        d.logits_stride = r.logits;
        d.mask_stride = r.mask;
        d.temperature = real(v[3]);
        buffer(idx, at::kInt, r.n * d.top);
        buffer(val, at::kFloat, r.n * d.top);
        const bool grad = truth(v[6]);
        Out total{Arg(v[7])}, loss{Arg(v[8])}, dx{Arg(grad ? v[9] : Py_None)};
        buffer(total.given, at::kFloat, 1);
        buffer(loss.given, at::kFloat, r.n);
        if (!total.given)
            total.make({1}, at::kFloat, *x);
        if (!loss.given)
            loss.make({r.n}, at::kFloat, *x);
        if (grad)
            d.dlogits_stride = r.gradient(dx, *x);
        const Work work(ws, r.work(), *x);
        PyObject* result = Py_BuildValue("(NNN)", total.object(), loss.object(), dx.object());
        return call(result, [&] {
            return p_distill_loss(&d, x.ptr(), (const int32_t*)idx.ptr(),
                                  (const float*)val.ptr(), (const uint8_t*)mask.ptr(),
                                  (const float*)weight.ptr(), (float*)total.ptr(),
                                  (float*)loss.ptr(), dx.ptr(), work.ptr, work.size, stream);
        });
    });
}

PyMethodDef methods[] = {
    {"load", load, METH_O, nullptr},
    {"linear", (PyCFunction)(void (*)())linear, METH_FASTCALL, nullptr},
    {"linear_backward", (PyCFunction)(void (*)())linear_backward, METH_FASTCALL, nullptr},
    {"policy_loss", (PyCFunction)(void (*)())policy_loss, METH_FASTCALL, nullptr},
    {"distill_loss", (PyCFunction)(void (*)())distill_loss, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_learner_calls", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__learner_calls() { return PyModule_Create(&module); }
