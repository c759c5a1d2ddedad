// Extension module `_llm`: the functions of abs_llm.h on PyTorch tensors, called by llm.py with every argument by position.
//
// A call on a few tokens is bound by the host: through ctypes a policy loss of 7 x 8192 took 21.7 us a call, of which the
// library's own function was 6.7 us and the rest the interpreter's (arguments checked, outputs made, addresses converted);
// compiled, 9.2 us (preference of one pair 22.5 -> 12.2, residual forward of 5 x 1024 11.7 -> 4.2).  Arguments are checked,
// outputs and workspace come from PyTorch's allocator on the current stream, the library's function is called without the
// interpreter's lock, and nothing synchronises.  What is refused raises TypeError / ValueError, a status of the library
// binding.AbsError; no C++ exception leaves a function.

#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <optional>
#include <string>
#include <utility>

#include "abs_llm.h"

namespace {

using at::Tensor;
using c10::ScalarType;

PyObject *g_error = nullptr, *g_no_memory = nullptr;       // binding.AbsError, torch.OutOfMemoryError

struct Refused {
    PyObject* type;                  // null: the interpreter's error is set already
    std::string text;
};
[[noreturn]] void type_error(std::string s) { throw Refused{PyExc_TypeError, std::move(s)}; }
[[noreturn]] void value_error(std::string s) { throw Refused{PyExc_ValueError, std::move(s)}; }

std::string shape_of(c10::IntArrayRef s) {
    std::string o = "(";
    for (size_t i = 0; i < s.size(); ++i) o += (i ? ", " : "") + std::to_string(s[i]);
    return o + ")";
}
const char* name_of(ScalarType t) { return t == at::kFloat ? "float32" : t == at::kBFloat16 ? "bfloat16" : t == at::kInt ? "int32" : c10::toString(t); }

// A strided CUDA tensor of that type on device `index` (any device if < 0); null if the object is none.
const Tensor* tensor_of(PyObject* o) {
    if (!THPVariable_Check(o)) return nullptr;
    const Tensor& t = THPVariable_Unpack(o);
    return t.is_cuda() && t.layout() == at::kStrided && !t.is_neg() ? &t : nullptr;
}
const Tensor& typed(PyObject* o, const char* name, ScalarType dtype, int index) {
    const Tensor* t = tensor_of(o);
    if (!t || t->scalar_type() != dtype || t->get_device() != index)
        type_error(std::string(name) + " must be a torch." + name_of(dtype) + " tensor on cuda:" + std::to_string(index));
    return *t;
}

struct Matrix {
    void* p = nullptr;
    uint64_t ld = 0;
};
// A [rows, cols] matrix: rows contiguous, at any distance that keeps them apart.
Matrix matrix(const Tensor& t, const char* name, int64_t rows, int64_t cols, bool written) {
    if (t.dim() != 2 || t.size(0) != rows || t.size(1) != cols)
        value_error(std::string(name) + " has shape " + shape_of(t.sizes()) + ", " + shape_of({rows, cols}) + " is wanted");
    Matrix m;
    m.ld = (uint64_t)cols;
    if (!t.is_contiguous()) {
        const int64_t down = t.stride(0), along = t.stride(1);
        if ((along != 1 && cols > 1) || (down < cols && rows > 1))
            value_error(std::string(name) + ": rows must be contiguous and must not overlap");
        if (down > cols) m.ld = (uint64_t)down;
    }
    m.p = written ? t.mutable_data_ptr() : const_cast<void*>(t.const_data_ptr());
    return m;
}
void* vector(PyObject* o, const char* name, int64_t n, ScalarType dtype, int index, bool written = false) {
    const Tensor& t = typed(o, name, dtype, index);
    if (t.dim() != 1 || t.size(0) != n || !t.is_contiguous())
        value_error(std::string(name) + " must be contiguous with " + std::to_string(n) + " elements");
    return written ? t.mutable_data_ptr() : const_cast<void*>(t.const_data_ptr());
}

// The matrix that the others have to agree with.
struct Like {
    const Tensor* t;
    ScalarType dtype;
    uint32_t code;
    int64_t rows, cols;
    int index;
    Matrix m;
};
uint32_t code_of(ScalarType t, const char* name) {
    if (t == at::kFloat) return ABS_F32;
    if (t == at::kBFloat16) return ABS_BF16;
    type_error(std::string(name) + " has dtype " + c10::toString(t) + ", float32 or bfloat16 is wanted");
}
Like first(PyObject* o, const char* name) {
    const Tensor* t = tensor_of(o);
    if (!t || t->dim() != 2) type_error(std::string(name) + " must be a CUDA tensor of two dimensions");
    Like l{t, t->scalar_type(), code_of(t->scalar_type(), name), t->size(0), t->size(1), (int)t->get_device(), {}};
    l.m = matrix(*t, name, l.rows, l.cols, false);
    return l;
}
Matrix same(PyObject* o, const char* name, const Like& l) { return matrix(typed(o, name, l.dtype, l.index), name, l.rows, l.cols, false); }

Tensor made(c10::IntArrayRef shape, ScalarType dtype, int index) {
    return at::detail::empty_cuda(shape, dtype, c10::Device(c10::kCUDA, (c10::DeviceIndex)index), std::nullopt);
}
// An output: the given one, or a new one of that shape and type.
struct Out {
    Tensor t;
    Matrix m;
};
Out out(PyObject* o, const char* name, const Like& l) {
    if (o == Py_None) {
        Out r{made({l.rows, l.cols}, l.dtype, l.index), {}};
        r.m = {r.t.mutable_data_ptr(), (uint64_t)l.cols};
        return r;
    }
    const Tensor& t = typed(o, name, l.dtype, l.index);
    return {t, matrix(t, name, l.rows, l.cols, true)};
}
// A sum over the rows: the given vector, or a new one (zero where something is added to it).
struct Column {
    Tensor t;
    float* p = nullptr;
};
Column column(PyObject* o, const char* name, const Like& l, bool accumulate) {
    Column c;
    if (o == Py_None) {
        c.t = made({l.cols}, at::kFloat, l.index);
        if (accumulate) c.t.zero_();
        c.p = c.t.mutable_data_ptr<float>();
    } else {
        c.p = (float*)vector(o, name, l.cols, at::kFloat, l.index, true);
        c.t = THPVariable_Unpack(o);
    }
    return c;
}

// Element i of a vector as a tensor without dimensions that shares its memory.
Tensor element(const Tensor& t, int64_t i) {
    Tensor v = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(t.storage()), t.key_set(), t.dtype());
    v.unsafeGetTensorImpl()->set_sizes_and_strides(c10::IntArrayRef(), c10::IntArrayRef(), t.storage_offset() + i);
    return v;
}

float number(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Refused{nullptr, {}};
    return (float)v;
}
bool truth(PyObject* o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Refused{nullptr, {}};
    return v != 0;
}

// fn(stream) with device `index` current, on its current stream.
template <typename F>
void launch(int index, F fn) {
    int rc;
    {
        PyThreadState* lock = PyEval_SaveThread();
        try {
            c10::cuda::CUDAGuard guard((c10::DeviceIndex)index);
            rc = fn((void*)c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)index).stream());
        } catch (...) {
            PyEval_RestoreThread(lock);
            throw;
        }
        PyEval_RestoreThread(lock);
    }
    if (rc == ABS_OK) return;
    PyObject* what = Py_BuildValue("is", rc, abs_last_error(nullptr));
    if (what) PyErr_SetObject(g_error ? g_error : PyExc_RuntimeError, what);
    Py_XDECREF(what);
    throw Refused{nullptr, {}};
}

// Given outputs (None: not given) that have been written: autograd notices when it has saved one of them.
template <typename... O>
void written(O... objects) {
    auto bump = [](PyObject* o) {
        if (o != Py_None && !THPVariable_Unpack(o).is_inference()) THPVariable_Unpack(o).unsafeGetTensorImpl()->bump_version();
    };
    (bump(objects), ...);
}

// A tuple of what is given: tensors, None for one that is not defined.
template <typename... T>
PyObject* tuple(T&&... tensors) {
    PyObject* t = PyTuple_New(sizeof...(T));
    if (!t) return nullptr;
    Py_ssize_t i = 0;
    bool ok = true;
    auto put = [&](Tensor&& x) {
        PyObject* o = x.defined() ? THPVariable_Wrap(std::move(x)) : Py_NewRef(Py_None);
        if (!o) ok = false;
        PyTuple_SET_ITEM(t, i++, o);
    };
    (put(std::forward<T>(tensors)), ...);
    if (!ok) Py_CLEAR(t);
    return t;
}

Out gradient(PyObject* o, bool wanted, const Like& l) {
    if (wanted) return out(o, "dlogits", l);
    if (o != Py_None) value_error("dlogits is given but need_grad is False");
    return {};
}

// logits, labels, logp_old, advantage, weight, logp_ref, clip_low, clip_high, kl_coef, dlogits, need_grad
PyObject* policy_loss(PyObject* const* a) {
    const Like l = first(a[0], "logits");
    const int64_t T = l.rows;
    const auto* y = (const int32_t*)vector(a[1], "labels", T, at::kInt, l.index);
    auto of = [&](int i, const char* name) { return a[i] == Py_None && i == 5 ? nullptr : (const float*)vector(a[i], name, T, at::kFloat, l.index); };
    const float *old = of(2, "logp_old"), *adv = of(3, "advantage"), *w = of(4, "weight"), *ref = of(5, "logp_ref");
    const float lo = number(a[6]), hi = number(a[7]), kl = number(a[8]);
    Out d = gradient(a[9], truth(a[10]), l);
    Tensor logp = made({T}, at::kFloat, l.index), stats = made({3}, at::kFloat, l.index);
    static const size_t n = abs_policy_loss_workspace();
    const Tensor ws = made({(int64_t)n}, at::kByte, l.index);
    float *stats_p = stats.mutable_data_ptr<float>(), *logp_p = logp.mutable_data_ptr<float>();
    void* ws_p = ws.mutable_data_ptr();
    launch(l.index, [&](void* s) {
        return abs_policy_loss(l.m.p, l.code, T, l.cols, l.m.ld, y, old, ref, adv, w, lo, hi, kl, stats_p, logp_p, d.m.p, d.m.ld, ws_p, n, s);
    });
    written(a[9]);
    return tuple(element(stats, 0), element(stats, 1), element(stats, 2), std::move(logp), std::move(d.t));
}

// logits, labels, offsets, logp_ref, beta, smoothing, scale, dlogits, need_grad
PyObject* preference_loss(PyObject* const* a) {
    const Like l = first(a[0], "logits");
    const auto* y = (const int32_t*)vector(a[1], "labels", l.rows, at::kInt, l.index);
    const Tensor* offsets = tensor_of(a[2]);
    if (!offsets || offsets->dim() != 1 || offsets->size(0) % 2 != 1) value_error("offsets must have 2 pairs + 1 elements on the logits' device");
    const int64_t pairs = offsets->size(0) / 2;
    const auto* off = (const int32_t*)vector(a[2], "offsets", 2 * pairs + 1, at::kInt, l.index);
    const auto* ref = (const float*)vector(a[3], "logp_ref", 2 * pairs, at::kFloat, l.index);
    const float beta = number(a[4]), smoothing = number(a[5]);
    const float scale = a[6] != Py_None ? number(a[6]) : pairs ? (float)(1.0 / (double)pairs) : 0.f;
    Out d = gradient(a[7], truth(a[8]), l);
    Tensor loss = made({}, at::kFloat, l.index), each = made({pairs}, at::kFloat, l.index), seq = made({2 * pairs}, at::kFloat, l.index);
    const size_t n = abs_preference_loss_workspace(l.rows);
    const Tensor ws = made({(int64_t)n}, at::kByte, l.index);
    float *loss_p = loss.mutable_data_ptr<float>(), *each_p = each.mutable_data_ptr<float>(), *seq_p = seq.mutable_data_ptr<float>();
    void* ws_p = ws.mutable_data_ptr();
    launch(l.index, [&](void* s) {
        return abs_preference_loss(l.m.p, l.code, l.rows, l.cols, l.m.ld, y, off, pairs, ref, beta, smoothing, scale, loss_p, each_p, seq_p, d.m.p, d.m.ld, ws_p,
                                   n, s);
    });
    written(a[7]);
    return tuple(std::move(loss), std::move(each), std::move(seq), std::move(d.t));
}

struct Gate {
    uint32_t kind = ABS_GATE_NONE;
    Matrix m;
};
Gate gate_of(PyObject* o, const Like& l) {
    Gate g;
    if (o == Py_None) return g;
    const Tensor* t = tensor_of(o);
    if (t && t->dim() == 1) {
        g.kind = ABS_GATE_CHANNEL;
        g.m = {vector(o, "gate", l.cols, at::kFloat, l.index), 0};
    } else {
        g.kind = ABS_GATE_ELEMENT;
        g.m = same(o, "gate", l);
    }
    return g;
}

// x, h, w_pre, w_post, gate, scale, eps, y, n
PyObject* residual_norm(PyObject* const* a) {
    const Like l = first(a[0], "x");
    const Matrix h = same(a[1], "h", l);
    const auto* pre = (const float*)vector(a[2], "w_pre", l.cols, at::kFloat, l.index);
    const auto* post = a[3] == Py_None ? nullptr : (const float*)vector(a[3], "w_post", l.cols, at::kFloat, l.index);
    const Gate g = gate_of(a[4], l);
    const float scale = number(a[5]), eps = number(a[6]);
    Out y = out(a[7], "y", l), n = out(a[8], "n", l);
    launch(l.index, [&](void* s) {
        return abs_residual_norm(l.m.p, l.m.ld, h.p, h.ld, g.m.p, g.m.ld, g.kind, post, pre, scale, eps, l.code, l.rows, l.cols, y.m.p, y.m.ld, n.m.p, n.m.ld, s);
    });
    written(a[7], a[8]);
    return tuple(std::move(y.t), std::move(n.t));
}

// dn, dy, y, h, w_pre, w_post, gate, scale, eps, dx, dh, dgate, dw_pre, dw_post, accumulate
PyObject* residual_norm_backward(PyObject* const* a) {
    const Like l = first(a[2], "y");
    const Matrix dn = same(a[0], "dn", l), h = same(a[3], "h", l);
    const Matrix dy = a[1] == Py_None ? Matrix{} : same(a[1], "dy", l);
    const auto* pre = (const float*)vector(a[4], "w_pre", l.cols, at::kFloat, l.index);
    const auto* post = a[5] == Py_None ? nullptr : (const float*)vector(a[5], "w_post", l.cols, at::kFloat, l.index);
    const Gate g = gate_of(a[6], l);
    const float scale = number(a[7]), eps = number(a[8]);
    const bool accumulate = truth(a[14]);
    if (!post && a[13] != Py_None) value_error("dw_post without w_post");
    if (g.kind == ABS_GATE_NONE && a[11] != Py_None) value_error("dgate without a gate");
    c10::cuda::CUDAGuard guard((c10::DeviceIndex)l.index);           // new sums are cleared on the stream of that device
    Out dx = out(a[9], "dx", l), dh = out(a[10], "dh", l), dg;
    Column dpre = column(a[12], "dw_pre", l, accumulate), dpost;
    if (post) dpost = column(a[13], "dw_post", l, accumulate);
    if (g.kind == ABS_GATE_CHANNEL) {
        Column c = column(a[11], "dgate", l, accumulate);
        dg = {std::move(c.t), {c.p, 0}};
    } else if (g.kind == ABS_GATE_ELEMENT) dg = out(a[11], "dgate", l);
    const size_t n = abs_residual_norm_workspace(l.rows, l.cols);
    const Tensor ws = made({(int64_t)n}, at::kByte, l.index);
    void* ws_p = ws.mutable_data_ptr();
    launch(l.index, [&](void* s) {
        return abs_residual_norm_backward(dn.p, dn.ld, dy.p, dy.ld, l.m.p, l.m.ld, h.p, h.ld, g.m.p, g.m.ld, g.kind, post, pre, scale, eps, l.code, l.rows, l.cols,
                                          dx.m.p, dx.m.ld, dh.m.p, dh.m.ld, dg.m.p, dg.m.ld, dpre.p, dpost.p, accumulate, ws_p, n, s);
    });
    written(a[9], a[10], a[11], a[12], a[13]);
    return tuple(std::move(dx.t), std::move(dh.t), std::move(dg.t), std::move(dpre.t), std::move(dpost.t));
}

// x
PyObject* ckpt8_quantize(PyObject* const* a) {
    const Like l = first(a[0], "x");
    const int64_t W = (l.cols + 31) / 32 * 32;
    Tensor q = made({l.rows, W}, at::kChar, l.index), e = made({l.rows, W / 32}, at::kByte, l.index);
    auto* q_p = (int8_t*)q.mutable_data_ptr();
    auto* e_p = (uint8_t*)e.mutable_data_ptr();
    launch(l.index, [&](void* s) { return abs_ckpt8_quantize(l.m.p, l.m.ld, l.code, l.rows, l.cols, q_p, e_p, s); });
    return tuple(std::move(q), std::move(e));
}

struct Packed {
    const int8_t* q;
    const uint8_t* e;
    int64_t rows, width;
    int index;
};
Packed packed(PyObject* oq, PyObject* oe, PyObject* owidth) {
    const int64_t width = PyLong_AsLongLong(owidth);
    if (width == -1 && PyErr_Occurred()) throw Refused{nullptr, {}};
    const Tensor *q = tensor_of(oq), *e = tensor_of(oe);
    if (!q || !e || q->scalar_type() != at::kChar || e->scalar_type() != at::kByte || q->get_device() != e->get_device())
        type_error("a Ckpt8 holds an int8 and a uint8 tensor on one CUDA device");
    if (width < 0 || q->dim() != 2 || e->dim() != 2 || q->size(1) % 32 || q->size(1) < width || q->size(1) - width > 31 || e->size(0) != q->size(0) ||
        e->size(1) != q->size(1) / 32 || !q->is_contiguous() || !e->is_contiguous())
        value_error("a Ckpt8 holds q [tokens, width rounded up to 32] and e [tokens, same / 32], contiguous");
    return {(const int8_t*)q->const_data_ptr(), (const uint8_t*)e->const_data_ptr(), q->size(0), width, (int)q->get_device()};
}

// q, e, width, bfloat16 (else float32), out
PyObject* ckpt8_dequantize(PyObject* const* a) {
    const Packed c = packed(a[0], a[1], a[2]);
    const bool half = truth(a[3]);
    const Like l{nullptr, half ? at::kBFloat16 : at::kFloat, half ? ABS_BF16 : ABS_F32, c.rows, c.width, c.index, {}};
    Out x = out(a[4], "out", l);
    launch(l.index, [&](void* s) { return abs_ckpt8_dequantize(c.q, c.e, c.rows, c.width, x.m.p, x.m.ld, l.code, s); });
    written(a[4]);
    return THPVariable_Wrap(std::move(x.t));
}

// q, e, width, dy, out, accumulate
PyObject* ckpt8_wgrad(PyObject* const* a) {
    const Packed c = packed(a[0], a[1], a[2]);
    const Tensor* t = tensor_of(a[3]);
    if (!t || t->dim() != 2) type_error("dy must be a CUDA tensor of two dimensions");
    const int64_t N = t->size(1);
    const Matrix dy = matrix(typed(a[3], "dy", at::kBFloat16, c.index), "dy", c.rows, N, false);
    const bool accumulate = truth(a[5]);
    if (accumulate && a[4] == Py_None) value_error("accumulate needs an out to add to");
    const Like l{nullptr, at::kFloat, ABS_F32, c.width, N, c.index, {}};
    Out dw = out(a[4], "out", l);
    Tensor ws;
    const size_t n = abs_ckpt8_wgrad_workspace(c.rows, c.width, N, dy.p, dy.ld);
    if (n) ws = made({(int64_t)n}, at::kByte, c.index);
    void* ws_p = n ? ws.mutable_data_ptr() : nullptr;
    launch(c.index, [&](void* s) {
        return abs_ckpt8_wgrad(c.q, c.e, dy.p, dy.ld, c.rows, c.width, N, (float*)dw.m.p, dw.m.ld, accumulate, ws_p, n, s);
    });
    written(a[4]);
    return THPVariable_Wrap(std::move(dw.t));
}

// A tensor of other sizes and type on the device of `l`.
Like sized(const Like& l, ScalarType dtype, int64_t rows, int64_t cols) { return {nullptr, dtype, dtype == at::kFloat ? ABS_F32 : ABS_BF16, rows, cols, l.index, {}}; }
Matrix given(PyObject* o, const char* name, const Like& l) { return o == Py_None ? Matrix{} : same(o, name, l); }
const float* maybe_vector(PyObject* o, const char* name, int64_t n, int index) {
    return o == Py_None ? nullptr : (const float*)vector(o, name, n, at::kFloat, index);
}
int64_t whole(PyObject* o) {
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Refused{nullptr, {}};
    return v;
}
Like bf16_first(PyObject* o, const char* name) {
    const Like l = first(o, name);
    if (l.dtype != at::kBFloat16) type_error(std::string(name) + " must be bfloat16");
    return l;
}
// Workspace of n bytes; the tensor keeps it while the call is enqueued.
struct Workspace {
    Tensor t;
    void* p = nullptr;
    size_t n;
    Workspace(size_t bytes, int index) : n(bytes) {
        if (!n) return;
        t = made({(int64_t)n}, at::kByte, index);
        p = t.mutable_data_ptr();
    }
};

// ids, table, scale, bfloat16 (else float32), y
PyObject* embed(PyObject* const* a) {
    const Like table = first(a[1], "table");
    if (table.dtype != at::kFloat) type_error("table must be float32");
    const Tensor* t = tensor_of(a[0]);
    if (!t || t->dim() != 1) type_error("ids must be a CUDA tensor of one dimension");
    const int64_t T = t->size(0);
    const auto* ids = (const int32_t*)vector(a[0], "ids", T, at::kInt, table.index);
    const float scale = number(a[2]);
    const Like l = sized(table, truth(a[3]) ? at::kBFloat16 : at::kFloat, T, table.cols);
    Out y = out(a[4], "y", l);
    launch(l.index, [&](void* s) { return abs_embed(ids, T, (const float*)table.m.p, table.m.ld, table.rows, table.cols, scale, l.code, y.m.p, y.m.ld, s); });
    written(a[4]);
    return THPVariable_Wrap(std::move(y.t));
}

// dy, ids, vocab, scale, out, accumulate
PyObject* embed_backward(PyObject* const* a) {
    const Like l = first(a[0], "dy");
    const auto* ids = (const int32_t*)vector(a[1], "ids", l.rows, at::kInt, l.index);
    const int64_t V = whole(a[2]);
    if (V < 1) value_error("vocab must be at least 1");
    const float scale = number(a[3]);
    const bool accumulate = truth(a[5]);
    if (accumulate && a[4] == Py_None) value_error("accumulate needs an out to add to");
    Out d = out(a[4], "out", sized(l, at::kFloat, V, l.cols));
    const Workspace ws(abs_embed_backward_workspace(l.rows, V, l.cols), l.index);
    launch(l.index, [&](void* s) { return abs_embed_backward(l.m.p, l.m.ld, l.code, ids, l.rows, V, l.cols, scale, (float*)d.m.p, d.m.ld, accumulate, ws.p, ws.n, s); });
    written(a[4]);
    return THPVariable_Wrap(std::move(d.t));
}

// x, w, b, eps, n
PyObject* layer_norm(PyObject* const* a) {
    const Like l = first(a[0], "x");
    const auto* w = (const float*)vector(a[1], "w", l.cols, at::kFloat, l.index);
    const float* b = maybe_vector(a[2], "b", l.cols, l.index);
    const float eps = number(a[3]);
    Out n = out(a[4], "n", l);
    launch(l.index, [&](void* s) { return abs_layer_norm(l.m.p, l.m.ld, w, b, eps, l.code, l.rows, l.cols, n.m.p, n.m.ld, s); });
    written(a[4]);
    return THPVariable_Wrap(std::move(n.t));
}

// dn, x, w, dskip, bias, eps, dx, dw, db, accumulate
PyObject* layer_norm_backward(PyObject* const* a) {
    const Like l = first(a[1], "x");
    const Matrix dn = same(a[0], "dn", l), skip = given(a[3], "dskip", l);
    const auto* w = (const float*)vector(a[2], "w", l.cols, at::kFloat, l.index);
    const bool bias = truth(a[4]), accumulate = truth(a[9]);
    const float eps = number(a[5]);
    if (!bias && a[8] != Py_None) value_error("db is given but bias is False");
    c10::cuda::CUDAGuard guard((c10::DeviceIndex)l.index);           // new sums are cleared on the stream of that device
    Out dx = out(a[6], "dx", l);
    Column dw = column(a[7], "dw", l, accumulate), db;
    if (bias) db = column(a[8], "db", l, accumulate);
    const Workspace ws(abs_layer_norm_workspace(l.rows, l.cols), l.index);
    launch(l.index, [&](void* s) {
        return abs_layer_norm_backward(dn.p, dn.ld, l.m.p, l.m.ld, skip.p, skip.ld, w, eps, l.code, l.rows, l.cols, dx.m.p, dx.m.ld, dw.p, db.p, accumulate, ws.p, ws.n, s);
    });
    written(a[6], a[7], a[8]);
    return tuple(std::move(dx.t), std::move(dw.t), std::move(db.t));
}

// x, w, b, act, residual, keep, bfloat16 (else float32), y, z
PyObject* linear(PyObject* const* a) {
    const Like x = bf16_first(a[0], "x"), w = bf16_first(a[1], "w");
    if (w.index != x.index || w.rows != x.cols) value_error("w must have as many rows as x has columns, on its device");
    const Like l = sized(x, truth(a[6]) ? at::kBFloat16 : at::kFloat, x.rows, w.cols), lz = sized(x, at::kBFloat16, x.rows, w.cols);
    const float* b = maybe_vector(a[2], "b", w.cols, x.index);
    const uint32_t act = (uint32_t)whole(a[3]);
    const Matrix res = given(a[4], "residual", l);
    const bool keep = truth(a[5]);
    if (!keep && a[8] != Py_None) value_error("z is given but keep is False");
    Out y = out(a[7], "y", l), z;
    if (keep) z = out(a[8], "z", lz);
    const Workspace ws(abs_linear_workspace(x.rows, x.cols, w.cols, x.m.p, x.m.ld, w.m.p, w.m.ld), x.index);
    launch(x.index, [&](void* s) {
        return abs_linear(x.m.p, x.m.ld, w.m.p, w.m.ld, b, act, res.p, res.ld, l.code, x.rows, x.cols, w.cols, y.m.p, y.m.ld, z.m.p, z.m.ld, ws.p, ws.n, s);
    });
    written(a[7], a[8]);
    return tuple(std::move(y.t), std::move(z.t));
}

// dy, w, act, z, residual, bfloat16 (else float32), dx
PyObject* linear_dgrad(PyObject* const* a) {
    const Like dy = bf16_first(a[0], "dy"), w = bf16_first(a[1], "w");
    if (w.index != dy.index || w.cols != dy.cols) value_error("w must have as many columns as dy, on its device");
    const Like l = sized(dy, truth(a[5]) ? at::kBFloat16 : at::kFloat, dy.rows, w.rows), lz = sized(dy, at::kBFloat16, dy.rows, w.rows);
    const uint32_t act = (uint32_t)whole(a[2]);
    const Matrix z = given(a[3], "z", lz), res = given(a[4], "residual", l);
    if ((act != ABS_ACT_NONE) != (a[3] != Py_None)) value_error("z must be given exactly with an activation");
    Out dx = out(a[6], "dx", l);
    const Workspace ws(abs_linear_dgrad_workspace(dy.rows, w.rows, dy.cols, dy.m.p, dy.m.ld, w.m.p, w.m.ld), dy.index);
    launch(dy.index, [&](void* s) {
        return abs_linear_dgrad(dy.m.p, dy.m.ld, w.m.p, w.m.ld, act, z.p, z.ld, res.p, res.ld, l.code, dy.rows, w.rows, dy.cols, dx.m.p, dx.m.ld, ws.p, ws.n, s);
    });
    written(a[6]);
    return THPVariable_Wrap(std::move(dx.t));
}

// x, dy, bias, dw, db, accumulate
PyObject* linear_wgrad(PyObject* const* a) {
    const Like x = bf16_first(a[0], "x"), dy = bf16_first(a[1], "dy");
    if (dy.index != x.index || dy.rows != x.rows) value_error("dy must have as many rows as x, on its device");
    const bool bias = truth(a[2]), accumulate = truth(a[5]);
    if (!bias && a[4] != Py_None) value_error("db is given but bias is False");
    if (accumulate && (a[3] == Py_None || (bias && a[4] == Py_None))) value_error("accumulate needs sums to add to");
    Out dw = out(a[3], "dw", sized(x, at::kFloat, x.cols, dy.cols));
    Column db;
    if (bias) db = column(a[4], "db", dy, false);
    const Workspace ws(abs_linear_wgrad_workspace(x.rows, x.cols, dy.cols, x.m.p, x.m.ld, dy.m.p, dy.m.ld), x.index);
    launch(x.index, [&](void* s) {
        return abs_linear_wgrad(x.m.p, x.m.ld, dy.m.p, dy.m.ld, x.rows, x.cols, dy.cols, (float*)dw.m.p, dw.m.ld, db.p, accumulate, ws.p, ws.n, s);
    });
    written(a[3], a[4]);
    return tuple(std::move(dw.t), std::move(db.t));
}

// dy, z, act, dz
PyObject* activation_backward(PyObject* const* a) {
    const Like dy = first(a[0], "dy"), l = sized(dy, at::kBFloat16, dy.rows, dy.cols);
    const Matrix z = same(a[1], "z", l);
    const uint32_t act = (uint32_t)whole(a[2]);
    Out dz = out(a[3], "dz", l);
    launch(l.index, [&](void* s) { return abs_activation_backward(dy.m.p, dy.m.ld, dy.code, z.p, z.ld, act, l.rows, l.cols, dz.m.p, dz.m.ld, s); });
    written(a[3]);
    return THPVariable_Wrap(std::move(dz.t));
}

// Sequences of a packed matrix: offsets (None: one sequence) and how many there are.
struct Sequences {
    const int32_t* offsets = nullptr;
    int64_t n = 1;
};
Sequences sequences(PyObject* o, int index) {
    if (o == Py_None) return {};
    const Tensor* t = tensor_of(o);
    if (!t || t->dim() != 1 || t->size(0) < 1) value_error("offsets must have sequences + 1 elements on the device of x");
    return {(const int32_t*)vector(o, "offsets", t->size(0), at::kInt, index), t->size(0) - 1};
}
// [sequences, width] fp32, packed.
float* state(PyObject* o, const char* name, int64_t n, int64_t width, int index, bool is_out) {
    const Tensor& t = typed(o, name, at::kFloat, index);
    if (t.dim() != 2 || t.size(0) != n || t.size(1) != width || !t.is_contiguous())
        value_error(std::string(name) + " must be contiguous of shape " + shape_of({n, width}));
    return is_out ? t.mutable_data_ptr<float>() : const_cast<float*>(t.const_data_ptr<float>());
}
Out state_out(PyObject* o, const char* name, int64_t n, int64_t width, int index) {
    Out r;
    if (o == Py_None) {
        r.t = made({n, width}, at::kFloat, index);
        r.m.p = r.t.mutable_data_ptr();
    } else {
        r.m.p = state(o, name, n, width, index, true);
        r.t = THPVariable_Unpack(o);
    }
    return r;
}

// x, g, offsets, h0, kind, y, last
PyObject* recurrence(PyObject* const* a) {
    const Like l = first(a[0], "x");
    const Matrix g = same(a[1], "g", l);
    const Sequences q = sequences(a[2], l.index);
    const float* h0 = a[3] == Py_None ? nullptr : state(a[3], "h0", q.n, l.cols, l.index, false);
    const uint32_t kind = (uint32_t)whole(a[4]);
    Out y = out(a[5], "y", l), last = state_out(a[6], "last", q.n, l.cols, l.index);
    const Workspace ws(abs_recurrence_workspace(l.rows, l.cols), l.index);
    launch(l.index, [&](void* s) {
        return abs_recurrence(l.m.p, l.m.ld, g.p, g.ld, q.offsets, q.n, h0, kind, l.code, l.rows, l.cols, y.m.p, y.m.ld, (float*)last.m.p, ws.p, ws.n, s);
    });
    written(a[5], a[6]);
    return tuple(std::move(y.t), std::move(last.t));
}

// dy, x, g, y, offsets, h0, dlast, kind, dx, dg, dh0
PyObject* recurrence_backward(PyObject* const* a) {
    const Like l = first(a[1], "x");
    const Matrix dy = same(a[0], "dy", l), g = same(a[2], "g", l), y = same(a[3], "y", l);
    const Sequences q = sequences(a[4], l.index);
    const float* h0 = a[5] == Py_None ? nullptr : state(a[5], "h0", q.n, l.cols, l.index, false);
    const float* dlast = a[6] == Py_None ? nullptr : state(a[6], "dlast", q.n, l.cols, l.index, false);
    const uint32_t kind = (uint32_t)whole(a[7]);
    Out dx = out(a[8], "dx", l), dg = out(a[9], "dg", l), dh0;
    if (h0 || a[10] != Py_None) dh0 = state_out(a[10], "dh0", q.n, l.cols, l.index);
    const Workspace ws(abs_recurrence_workspace(l.rows, l.cols), l.index);
    launch(l.index, [&](void* s) {
        return abs_recurrence_backward(dy.p, dy.ld, l.m.p, l.m.ld, g.p, g.ld, y.p, y.ld, q.offsets, q.n, h0, dlast, kind, l.code, l.rows, l.cols, dx.m.p, dx.m.ld, dg.m.p, dg.m.ld,
                                       (float*)dh0.m.p, ws.p, ws.n, s);
    });
    written(a[8], a[9], a[10]);
    return tuple(std::move(dx.t), std::move(dg.t), std::move(dh0.t));
}

// x, g, h, kind, y, out
PyObject* recurrence_step(PyObject* const* a) {
    const Like l = first(a[0], "x");
    const Matrix g = same(a[1], "g", l);
    const float* h = state(a[2], "h", l.rows, l.cols, l.index, false);
    const uint32_t kind = (uint32_t)whole(a[3]);
    Out y = out(a[4], "y", l), o = state_out(a[5], "out", l.rows, l.cols, l.index);
    launch(l.index, [&](void* s) { return abs_recurrence_step(l.m.p, l.m.ld, g.p, g.ld, h, kind, l.code, l.rows, l.cols, y.m.p, y.m.ld, (float*)o.m.p, s); });
    written(a[4], a[5]);
    return tuple(std::move(y.t), std::move(o.t));
}

template <PyObject* (*fn)(PyObject* const*), int kArgs>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != kArgs) {
        PyErr_Format(PyExc_TypeError, "%d arguments are wanted, %zd are given", kArgs, n);
        return nullptr;
    }
    try {
        return fn(args);
    } catch (const Refused& r) {
        if (r.type) PyErr_SetString(r.type, r.text.c_str());
    } catch (const c10::OutOfMemoryError& e) {
        PyErr_SetString(g_no_memory ? g_no_memory : PyExc_MemoryError, e.what_without_backtrace());
    } catch (const c10::Error& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
    } catch (const std::exception& e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
    }
    return nullptr;
}
template <PyObject* (*fn)(PyObject* const*), int kArgs>
constexpr PyMethodDef method(const char* name) {
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<fn, kArgs>)), METH_FASTCALL, nullptr};
}

PyObject* set_errors(PyObject*, PyObject* args) {
    PyObject *status, *no_memory;
    if (!PyArg_ParseTuple(args, "OO", &status, &no_memory)) return nullptr;
    Py_XSETREF(g_error, Py_NewRef(status));
    Py_XSETREF(g_no_memory, Py_NewRef(no_memory));
    Py_RETURN_NONE;
}

PyMethodDef kMethods[] = {
    method<policy_loss, 11>("policy_loss"),
    method<preference_loss, 9>("preference_loss"),
    method<residual_norm, 9>("residual_norm"),
    method<residual_norm_backward, 15>("residual_norm_backward"),
    method<ckpt8_quantize, 1>("ckpt8_quantize"),
    method<ckpt8_dequantize, 5>("ckpt8_dequantize"),
    method<ckpt8_wgrad, 6>("ckpt8_wgrad"),
    method<embed, 5>("embed"),
    method<embed_backward, 6>("embed_backward"),
    method<layer_norm, 5>("layer_norm"),
    method<layer_norm_backward, 10>("layer_norm_backward"),
    method<linear, 9>("linear"),
    method<linear_dgrad, 7>("linear_dgrad"),
    method<linear_wgrad, 6>("linear_wgrad"),
    method<activation_backward, 4>("activation_backward"),
    method<recurrence, 7>("recurrence"),
    method<recurrence_backward, 11>("recurrence_backward"),
    method<recurrence_step, 6>("recurrence_step"),
    {"set_errors", set_errors, METH_VARARGS, "The exceptions of a status, called with (status, text), and of an allocation that failed."},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_llm", "Functions of llm.py; see there.", -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__llm() { return PyModule_Create(&kModule); }
