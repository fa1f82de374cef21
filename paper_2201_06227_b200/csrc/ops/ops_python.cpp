// The operators' calls from Python: checks of the tensors, allocation of the results, and the argument structs of
// include/egeria_ops.h.  A call costs about as much here as its kernel's launch; done in Python the same
// checks cost several times that, which is what a small layer's call would then take.
//
// The functions take the address of the library's entry point and its handle as numbers (paper_2201_06227_b200/ops.py has them)
// and return the results, or the library's status as a number if that is not EGERIA_OK.
#include <ATen/ops/empty.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../../include/egeria_ops.h"

namespace {

using at::Tensor;

struct Matrix {
    void *p = nullptr;
    int64_t ld = 0;
};

int type_of(at::ScalarType t) {
    return t == at::kFloat ? EGERIA_F32 : t == at::kBFloat16 ? EGERIA_BF16 : t == at::kHalf ? EGERIA_F16 : -1;
}

[[noreturn]] void refuse(const std::string &what) {
    TORCH_CHECK_VALUE(false, what);
    std::abort();  // (not reached: the check throws)
}

// Passes on the error that Python has set.
[[noreturn]] void pass_on() {
    python_error e;
    e.persist();
    throw e;
}

// (no string streams: the process may hold a C++ runtime of another compiler, whose locales they would meet)
std::string describe(const Tensor &t) {
    std::string s = std::string(at::toString(t.scalar_type())) + " [";
    for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
    return s + "] on " + (t.is_cuda() ? "cuda:" + std::to_string(t.get_device()) : std::string("the host"));
}

const Tensor &tensor(PyObject *o, const char *name) {
    if (!THPVariable_Check(o)) refuse(std::string(name) + ": expected a tensor");
    return THPVariable_Unpack(o);
}

// A matrix whose rows are consecutive.
Matrix matrix(const Tensor &t, const char *name, int device, at::ScalarType type, int64_t rows, int64_t cols) {
    if (t.scalar_type() != type || !t.is_cuda() || t.get_device() != device || t.dim() != 2 || t.size(0) != rows || t.size(1) != cols) {
        refuse(std::string(name) + ": expected " + at::toString(type) + " [" + std::to_string(rows) + ", " + std::to_string(cols) + "] on cuda:" +
               std::to_string(device) + ", got " + describe(t));
    }
    if (cols > 1 && t.stride(1) != 1) refuse(std::string(name) + ": the values of a row have to be consecutive");
    if (rows > 1 && t.stride(0) < cols) refuse(std::string(name) + ": rows overlap");
    return Matrix{t.data_ptr(), rows > 1 ? t.stride(0) : cols};
}
Matrix matrix(PyObject *o, const char *name, int device, at::ScalarType type, int64_t rows, int64_t cols) {
    return o == Py_None ? Matrix{} : matrix(tensor(o, name), name, device, type, rows, cols);
}
void *vector(PyObject *o, const char *name, int device, at::ScalarType type, int64_t n) {
    if (o == Py_None) return nullptr;
    const Tensor &t = tensor(o, name);
    if (t.scalar_type() != type || !t.is_cuda() || t.get_device() != device || t.numel() != n || !t.is_contiguous()) {
        refuse(std::string(name) + ": expected " + std::to_string(n) + " consecutive " + at::toString(type) + " on cuda:" + std::to_string(device) +
               ", got " + describe(t));
    }
    return t.data_ptr();
}

Tensor make(const Tensor &like, at::IntArrayRef sizes) { return at::empty(sizes, like.options()); }

struct Call {   // the first arguments of every function: entry point, handle, device, stream
    void *fn, *handle, *stream;
    int device;
    PyObject *const *rest;
    Call(PyObject *const *args, Py_ssize_t n, Py_ssize_t expected) : rest(args + 4) {
        if (n != expected) refuse("wrong number of arguments");
        fn = PyLong_AsVoidPtr(args[0]);
        handle = PyLong_AsVoidPtr(args[1]);
        device = (int)PyLong_AsLong(args[2]);
        stream = PyLong_AsVoidPtr(args[3]);
        if (PyErr_Occurred()) pass_on();
    }
    int64_t whole(int i) const {
        const int64_t v = PyLong_AsLongLong(rest[i]);
        if (v == -1 && PyErr_Occurred()) pass_on();
        return v;
    }
    double real(int i) const {
        const double v = PyFloat_AsDouble(rest[i]);
        if (v == -1.0 && PyErr_Occurred()) pass_on();
        return v;
    }
    bool flag(int i) const { return PyObject_IsTrue(rest[i]) == 1; }
    bool given(int i) const { return rest[i] != Py_None; }
};

PyObject *wrap(const Tensor &t) {
    if (!t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(t);
}

// An argument that autograd follows, of those (tensors or None, as has been checked) at the given places.
const Tensor *followed(const Call &c, std::initializer_list<int> places) {
    if (at::GradMode::is_enabled())
        for (int i : places)
            if (c.given(i) && THPVariable_Unpack(c.rest[i]).requires_grad()) return &THPVariable_Unpack(c.rest[i]);
    return nullptr;
}
// A result of a forward call.  The calls keep no history for autograd, whose user would find a gradient left out in silence:
// where it follows an argument, going back through the result is an error that names the call which has the gradients.
PyObject *wrap(const Tensor &t, const Tensor *argument, const char *backward) {
    if (!argument || !t.defined()) return wrap(t);
    const auto fn = std::make_shared<torch::autograd::DelayedError>(
        std::string("the library's calls keep no history: the gradients are the results of ") + backward + " (torch.no_grad() where none is wanted)", 2);
    return wrap((*fn)({*argument, t})[1]);
}

// x, w, bias, act, residual, save_z, out -> y or (y, z)
PyObject *linear_forward(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const Call c(args, n, 4 + 7);
    const Tensor &x = tensor(c.rest[0], "x"), &w = tensor(c.rest[1], "w");
    if (x.dim() != 2 || w.dim() != 2) refuse("x and w are matrices");
    const at::ScalarType t = x.scalar_type();
    egeria_linear_forward_args a{};
    a.type = type_of(t);
    a.act = (int32_t)c.whole(3);
    a.rows = x.size(0), a.inp = x.size(1), a.out = w.size(0);
    const Matrix mx = matrix(x, "x", c.device, t, a.rows, a.inp), mw = matrix(w, "w", c.device, t, a.out, a.inp);
    const Matrix mr = matrix(c.rest[4], "residual", c.device, t, a.rows, a.out);
    a.x = mx.p, a.ldx = mx.ld, a.w = mw.p, a.ldw = mw.ld, a.residual = mr.p, a.ldr = mr.ld;
    a.bias = vector(c.rest[2], "bias", c.device, t, a.out);
    const Tensor y = c.given(6) ? tensor(c.rest[6], "out") : make(x, {a.rows, a.out});
    const Tensor z = c.flag(5) ? make(x, {a.rows, a.out}) : Tensor();
    const Matrix my = matrix(y, "out", c.device, t, a.rows, a.out);
    a.y = my.p, a.ldy = my.ld;
    if (z.defined()) a.z = z.data_ptr(), a.ldz = a.out;
    const egeria_status s = reinterpret_cast<decltype(&egeria_linear_forward)>(c.fn)(static_cast<egeria_ops *>(c.handle), c.stream, &a);
    if (s != EGERIA_OK) return PyLong_FromLong(s);
    if (c.given(6) && !y.is_inference()) y.unsafeGetTensorImpl()->bump_version();   // written in place
    const char *const back = "egeria_linear_backward";
    const Tensor *const from = followed(c, {0, 1, 2, 4});
    if (!z.defined()) return wrap(y, from, back);
    return Py_BuildValue("(NN)", wrap(y, from, back), wrap(z, from, back));
    END_HANDLE_TH_ERRORS
}

// dy, x, w, z, act, z_in, act_in, need_dx, need_dw, need_db -> (dx, dw, db)
PyObject *linear_backward(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const Call c(args, n, 4 + 10);
    const Tensor &dy = tensor(c.rest[0], "dy");
    const bool need_dx = c.flag(7), need_dw = c.flag(8), need_db = c.flag(9);
    if (dy.dim() != 2 || (need_dx && !c.given(2)) || (need_dw && !c.given(1)) || (!c.given(1) && !c.given(2)))
        refuse("dy is a matrix; dx needs w, dw needs x, and one of the two has to be there");
    const Tensor &inner = tensor(c.rest[c.given(1) ? 1 : 2], "x or w");
    if (inner.dim() != 2) refuse("x and w are matrices");
    const at::ScalarType t = dy.scalar_type();
    egeria_linear_backward_args a{};
    a.type = type_of(t);
    a.act = (int32_t)c.whole(4), a.act_in = (int32_t)c.whole(6);
    a.rows = dy.size(0), a.inp = inner.size(1), a.out = dy.size(1);
    const Matrix mdy = matrix(dy, "dy", c.device, t, a.rows, a.out), mx = matrix(c.rest[1], "x", c.device, t, a.rows, a.inp);
    const Matrix mw = matrix(c.rest[2], "w", c.device, t, a.out, a.inp), mz = matrix(c.rest[3], "z", c.device, t, a.rows, a.out);
    const Matrix mzi = matrix(c.rest[5], "z_in", c.device, t, a.rows, a.inp);
    a.dy = mdy.p, a.lddy = mdy.ld, a.x = mx.p, a.ldx = mx.ld, a.w = mw.p, a.ldw = mw.ld;
    a.z = mz.p, a.ldz = mz.ld, a.z_in = mzi.p, a.ldz_in = mzi.ld;
    const Tensor dx = need_dx ? make(dy, {a.rows, a.inp}) : Tensor(), dw = need_dw ? make(dy, {a.out, a.inp}) : Tensor();
    const Tensor db = need_db ? make(dy, {a.out}) : Tensor();
    if (need_dx) a.dx = dx.data_ptr(), a.lddx = a.inp;
    if (need_dw) a.dw = dw.data_ptr(), a.lddw = a.inp;
    if (need_db) a.db = db.data_ptr();
    const egeria_status s = reinterpret_cast<decltype(&egeria_linear_backward)>(c.fn)(static_cast<egeria_ops *>(c.handle), c.stream, &a);
    if (s != EGERIA_OK) return PyLong_FromLong(s);
    return Py_BuildValue("(NNN)", wrap(dx), wrap(dw), wrap(db));
    END_HANDLE_TH_ERRORS
}

// x, w_gate, w_up, w_down, b_gate, b_up, b_down, act, residual, save, out -> y or (y, g, u)
PyObject *gated_forward(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const Call c(args, n, 4 + 11);
    const Tensor &x = tensor(c.rest[0], "x"), &wg = tensor(c.rest[1], "w_gate"), &wu = tensor(c.rest[2], "w_up"), &wd = tensor(c.rest[3], "w_down");
    if (x.dim() != 2 || wg.dim() != 2 || wd.dim() != 2) refuse("x, w_gate, w_up and w_down are matrices");
    const at::ScalarType t = x.scalar_type();
    egeria_gated_forward_args a{};
    a.type = type_of(t);
    a.act = (int32_t)c.whole(7);
    a.rows = x.size(0), a.inp = x.size(1), a.hidden = wg.size(0), a.out = wd.size(0);
    const Matrix mx = matrix(x, "x", c.device, t, a.rows, a.inp), mg = matrix(wg, "w_gate", c.device, t, a.hidden, a.inp);
    const Matrix mu = matrix(wu, "w_up", c.device, t, a.hidden, a.inp), md = matrix(wd, "w_down", c.device, t, a.out, a.hidden);
    const Matrix mr = matrix(c.rest[8], "residual", c.device, t, a.rows, a.out);
    a.x = mx.p, a.ldx = mx.ld, a.w_gate = mg.p, a.ldw_gate = mg.ld, a.w_up = mu.p, a.ldw_up = mu.ld, a.w_down = md.p, a.ldw_down = md.ld;
    a.residual = mr.p, a.ldr = mr.ld;
    a.b_gate = vector(c.rest[4], "b_gate", c.device, t, a.hidden);
    a.b_up = vector(c.rest[5], "b_up", c.device, t, a.hidden);
    a.b_down = vector(c.rest[6], "b_down", c.device, t, a.out);
    const Tensor y = c.given(10) ? tensor(c.rest[10], "out") : make(x, {a.rows, a.out});
    const bool save = c.flag(9);
    const Tensor g = save ? make(x, {a.rows, a.hidden}) : Tensor(), u = save ? make(x, {a.rows, a.hidden}) : Tensor();
    const Matrix my = matrix(y, "out", c.device, t, a.rows, a.out);
    a.y = my.p, a.ldy = my.ld;
    if (save) a.g = g.data_ptr(), a.u = u.data_ptr(), a.ldg = a.ldu = a.hidden;
    const egeria_status s = reinterpret_cast<decltype(&egeria_gated_forward)>(c.fn)(static_cast<egeria_ops *>(c.handle), c.stream, &a);
    if (s != EGERIA_OK) return PyLong_FromLong(s);
    if (c.given(10) && !y.is_inference()) y.unsafeGetTensorImpl()->bump_version();   // written in place
    const char *const back = "egeria_gated_backward";
    const Tensor *const from = followed(c, {0, 1, 2, 3, 4, 5, 6, 8});
    if (!save) return wrap(y, from, back);
    return Py_BuildValue("(NNN)", wrap(y, from, back), wrap(g, from, back), wrap(u, from, back));
    END_HANDLE_TH_ERRORS
}

// dy, x, w_gate, w_up, w_down, g, u, act, need_dx, need_dw, need_db -> (dx, dw_gate, dw_up, dw_down, db_gate, db_up, db_down)
PyObject *gated_backward(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const Call c(args, n, 4 + 11);
    const Tensor &dy = tensor(c.rest[0], "dy"), &wd = tensor(c.rest[4], "w_down"), &g = tensor(c.rest[5], "g"), &u = tensor(c.rest[6], "u");
    const bool need_dx = c.flag(8), need_dw = c.flag(9), need_db = c.flag(10);
    if (dy.dim() != 2 || wd.dim() != 2 || (need_dx && (!c.given(2) || !c.given(3))) || (need_dw && !c.given(1)))
        refuse("dy and w_down are matrices; dx needs w_gate and w_up, the weights' gradients need x");
    const at::ScalarType t = dy.scalar_type();
    egeria_gated_backward_args a{};
    a.type = type_of(t);
    a.act = (int32_t)c.whole(7);
    a.rows = dy.size(0), a.out = dy.size(1), a.hidden = wd.size(1), a.inp = 1;
    for (int i = 1; i < 3; ++i)
        if (c.given(i)) {
            const Tensor &inner = tensor(c.rest[i], i == 1 ? "x" : "w_gate");
            if (inner.dim() != 2) refuse("x and the weights are matrices");
            a.inp = inner.size(1);
            break;
        }
    const Matrix mdy = matrix(dy, "dy", c.device, t, a.rows, a.out), mx = matrix(c.rest[1], "x", c.device, t, a.rows, a.inp);
    const Matrix mg = matrix(c.rest[2], "w_gate", c.device, t, a.hidden, a.inp), mu = matrix(c.rest[3], "w_up", c.device, t, a.hidden, a.inp);
    const Matrix md = matrix(wd, "w_down", c.device, t, a.out, a.hidden);
    const Matrix ga = matrix(g, "g", c.device, t, a.rows, a.hidden), ua = matrix(u, "u", c.device, t, a.rows, a.hidden);
    a.dy = mdy.p, a.lddy = mdy.ld, a.x = mx.p, a.ldx = mx.ld, a.w_gate = mg.p, a.ldw_gate = mg.ld, a.w_up = mu.p, a.ldw_up = mu.ld;
    a.w_down = md.p, a.ldw_down = md.ld, a.g = ga.p, a.ldg = ga.ld, a.u = ua.p, a.ldu = ua.ld;
    const Tensor dx = need_dx ? make(dy, {a.rows, a.inp}) : Tensor();
    // (one tensor for the two projections: a model that keeps them side by side has its gradient whole)
    Tensor dw, dw_gate, dw_up, dw_down, db, db_gate, db_up, db_down;
    if (need_dw) {
        dw = make(dy, {2 * a.hidden, a.inp});
        dw_gate = dw.narrow(0, 0, a.hidden), dw_up = dw.narrow(0, a.hidden, a.hidden);
        dw_down = make(dy, {a.out, a.hidden});
        a.dw_gate = dw_gate.data_ptr(), a.dw_up = dw_up.data_ptr(), a.dw_down = dw_down.data_ptr();
        a.lddw_gate = a.lddw_up = a.inp, a.lddw_down = a.hidden;
    }
    if (need_db) {
        db = make(dy, {2 * a.hidden});
        db_gate = db.narrow(0, 0, a.hidden), db_up = db.narrow(0, a.hidden, a.hidden);
        db_down = make(dy, {a.out});
        a.db_gate = db_gate.data_ptr(), a.db_up = db_up.data_ptr(), a.db_down = db_down.data_ptr();
    }
    if (need_dx) a.dx = dx.data_ptr(), a.lddx = a.inp;
    const egeria_status s = reinterpret_cast<decltype(&egeria_gated_backward)>(c.fn)(static_cast<egeria_ops *>(c.handle), c.stream, &a);
    if (s != EGERIA_OK) return PyLong_FromLong(s);
    return Py_BuildValue("(NNNNNNN)", wrap(dx), wrap(dw_gate), wrap(dw_up), wrap(dw_down), wrap(db_gate), wrap(db_up), wrap(db_down));
    END_HANDLE_TH_ERRORS
}

// The gate, the weights and the biases (five places of `c` from `first` on), which share a type.
template <typename Args>
at::ScalarType norm_vectors(const Call &c, int first, at::ScalarType type, Args &a) {
    static const char *const names[5] = {"gate", "w_post", "b_post", "w_pre", "b_pre"};
    at::ScalarType t = type;
    for (int i = 0; i < 5; ++i)
        if (c.given(first + i)) {
            t = tensor(c.rest[first + i], names[i]).scalar_type();
            break;
        }
    a.param_type = type_of(t);
    const int64_t groups = a.gate_rows > 0 ? (a.rows + a.gate_rows - 1) / a.gate_rows : 1;
    const void *p[5];
    for (int i = 0; i < 5; ++i) p[i] = vector(c.rest[first + i], names[i], c.device, t, (i ? 1 : groups) * a.cols);
    a.gate = p[0], a.w_post = p[1], a.b_post = p[2], a.w_pre = p[3], a.b_pre = p[4];
    return t;
}

// x, f, gate, w_post, b_post, w_pre, b_pre, gate_rows, kind, post, pre, alpha, eps -> (y, h, stats)
PyObject *norm_forward(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const Call c(args, n, 4 + 13);
    const Tensor &x = tensor(c.rest[0], "x"), &f = tensor(c.rest[1], "f");
    if (x.dim() != 2) refuse("x is a matrix");
    const at::ScalarType t = x.scalar_type();
    egeria_norm_forward_args a{};
    a.type = type_of(t);
    a.rows = x.size(0), a.cols = x.size(1), a.gate_rows = c.whole(7);
    a.kind = (int32_t)c.whole(8), a.post = c.flag(9), a.pre = c.flag(10);
    a.alpha = (float)c.real(11), a.eps = (float)c.real(12);
    norm_vectors(c, 2, t, a);
    const Matrix mx = matrix(x, "x", c.device, t, a.rows, a.cols), mf = matrix(f, "f", c.device, t, a.rows, a.cols);
    a.x = mx.p, a.ldx = mx.ld, a.f = mf.p, a.ldf = mf.ld;
    const Tensor y = make(x, {a.rows, a.cols}), h = a.pre ? make(x, {a.rows, a.cols}) : Tensor();
    const Tensor stats = at::empty({a.rows, 4}, x.options().dtype(at::kFloat));
    a.y = y.data_ptr(), a.ldy = a.ldh = a.cols;
    if (a.pre) a.h = h.data_ptr();
    a.stats = static_cast<float *>(stats.data_ptr());
    const egeria_status s = reinterpret_cast<decltype(&egeria_norm_forward)>(c.fn)(static_cast<egeria_ops *>(c.handle), c.stream, &a);
    if (s != EGERIA_OK) return PyLong_FromLong(s);
    const char *const back = "egeria_norm_backward";
    const Tensor *const from = followed(c, {0, 1, 2, 3, 4, 5, 6});
    return Py_BuildValue("(NNN)", wrap(y, from, back), wrap(h, from, back), wrap(stats, from, back));
    END_HANDLE_TH_ERRORS
}

// dy, dh, y, f, stats, gate, w_post, b_post, w_pre, b_pre, gate_rows, kind, post, pre, alpha, need_params
// -> (dx, df, dgate, dw_post, db_post, dw_pre, db_pre)
PyObject *norm_backward(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const Call c(args, n, 4 + 16);
    const Tensor &dy = tensor(c.rest[0], "dy");
    if (dy.dim() != 2) refuse("dy is a matrix");
    const at::ScalarType t = dy.scalar_type();
    egeria_norm_backward_args a{};
    a.type = type_of(t);
    a.rows = dy.size(0), a.cols = dy.size(1), a.gate_rows = c.whole(10);
    a.kind = (int32_t)c.whole(11), a.post = c.flag(12), a.pre = c.flag(13);
    a.alpha = (float)c.real(14);
    norm_vectors(c, 5, t, a);
    const Matrix mdy = matrix(dy, "dy", c.device, t, a.rows, a.cols), mdh = matrix(c.rest[1], "dh", c.device, t, a.rows, a.cols);
    const Matrix my = matrix(c.rest[2], "y", c.device, t, a.rows, a.cols), mf = matrix(c.rest[3], "f", c.device, t, a.rows, a.cols);
    a.dy = mdy.p, a.lddy = mdy.ld, a.dh = mdh.p, a.lddh = mdh.ld, a.y = my.p, a.ldy = my.ld, a.f = mf.p, a.ldf = mf.ld;
    a.stats = static_cast<const float *>(vector(c.rest[4], "stats", c.device, at::kFloat, 4 * a.rows));
    const Tensor dx = make(dy, {a.rows, a.cols}), df = make(dy, {a.rows, a.cols});
    a.dx = dx.data_ptr(), a.df = df.data_ptr(), a.lddx = a.lddf = a.cols;
    Tensor sums[5];
    const bool there[5] = {true, a.post != 0, a.post != 0, a.pre != 0, a.pre != 0}, need = c.flag(15);
    void **const to[5] = {&a.dgate, &a.dw_post, &a.db_post, &a.dw_pre, &a.db_pre};
    for (int i = 0; i < 5; ++i)
        if (need && there[i] && c.given(5 + i)) {
            const Tensor &p = tensor(c.rest[5 + i], "parameter");
            sums[i] = make(p, p.sizes());
            *to[i] = sums[i].data_ptr();
        }
    const egeria_status s = reinterpret_cast<decltype(&egeria_norm_backward)>(c.fn)(static_cast<egeria_ops *>(c.handle), c.stream, &a);
    if (s != EGERIA_OK) return PyLong_FromLong(s);
    return Py_BuildValue("(NNNNNNN)", wrap(dx), wrap(df), wrap(sums[0]), wrap(sums[1]), wrap(sums[2]), wrap(sums[3]), wrap(sums[4]));
    END_HANDLE_TH_ERRORS
}

// lr, beta1, beta2, eps, grad_scale, frozen, last module -> status
PyObject *adamw_step(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const Call c(args, n, 4 + 7);
    const void *scale = vector(c.rest[4], "grad_scale", c.device, at::kFloat, 1);
    const void *frozen = nullptr;
    if (c.given(5)) {
        const Tensor &f = tensor(c.rest[5], "frozen");
        frozen = vector(c.rest[5], "frozen", c.device, at::kByte, f.numel());
        if (f.numel() <= c.whole(6)) refuse("frozen: one entry per module is required");
    }
    const egeria_status s = reinterpret_cast<decltype(&egeria_adamw_step)>(c.fn)(
        static_cast<egeria_adamw *>(c.handle), c.stream, c.real(0), c.real(1), c.real(2), c.real(3), static_cast<const float *>(scale),
        static_cast<const uint8_t *>(frozen));
    return PyLong_FromLong(s);
    END_HANDLE_TH_ERRORS
}

// lr, beta, nesterov, eps, grad_scale, frozen, last module -> status
PyObject *muon_step(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const Call c(args, n, 4 + 7);
    const void *scale = vector(c.rest[4], "grad_scale", c.device, at::kFloat, 1);
    const void *frozen = nullptr;
    if (c.given(5)) {
        const Tensor &f = tensor(c.rest[5], "frozen");
        frozen = vector(c.rest[5], "frozen", c.device, at::kByte, f.numel());
        if (f.numel() <= c.whole(6)) refuse("frozen: one entry per module is required");
    }
    const egeria_status s = reinterpret_cast<decltype(&egeria_muon_step)>(c.fn)(static_cast<egeria_muon *>(c.handle), c.stream, c.real(0), c.real(1),
                                                                                c.flag(2), c.real(3), static_cast<const float *>(scale),
                                                                                static_cast<const uint8_t *>(frozen));
    return PyLong_FromLong(s);
    END_HANDLE_TH_ERRORS
}

template <typename F>
PyCFunction fast(F f) {
    return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f));
}
PyMethodDef methods[] = {
    {"linear_forward", fast(linear_forward), METH_FASTCALL, nullptr},   {"linear_backward", fast(linear_backward), METH_FASTCALL, nullptr},
    {"norm_forward", fast(norm_forward), METH_FASTCALL, nullptr},       {"norm_backward", fast(norm_backward), METH_FASTCALL, nullptr},
    {"gated_forward", fast(gated_forward), METH_FASTCALL, nullptr},     {"gated_backward", fast(gated_backward), METH_FASTCALL, nullptr},
    {"adamw_step", fast(adamw_step), METH_FASTCALL, nullptr},           {"muon_step", fast(muon_step), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ops_python", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__ops_python(void) { return PyModule_Create(&module); }
