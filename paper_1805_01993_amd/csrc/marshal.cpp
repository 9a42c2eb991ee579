// Native argument marshalling for binding.py (the module _marshal): checks the tensors of a call, takes their addresses and
// torch's current stream, and calls the C entry point.  A small pass is bound by what the host does between two launches: a
// one-launch call took 4.8 us through ctypes and tensor attributes read from Python, 1.5 of them before the library was
// entered.  Only the ordinary case is taken: plain torch tensors that fit, and no mode that wants to see what is asked of
// tensors (torch.overrides.TorchFunctionMode).  Everything else is answered with
// None, and binding.py goes its own way, which accepts what it accepted and raises what it raised.
#include <Python.h>

#include <cstddef>
#include <cstdint>
#include <initializer_list>
#include <utility>

#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

namespace {

constexpr int kMaxTensors = 3, kMaxCalls = 16, kBuffers = 5;
using Call2 = int (*)(const void *, void *, void *, void *);
using Call3 = int (*)(const void *, void *, void *, void *, void *);
using NodeCall2 = int (*)(const void *, int, void *, void *, void *);
using NodeCall3 = int (*)(const void *, int, void *, void *, void *, void *);

// The entry points, as calls() has named them once: address, whether a node number comes first, the buffers.
struct Entry {
    uintptr_t fn = 0;
    bool node = false;
    int tensors = 0;
    int buffer[kMaxTensors] = {};
};
Entry table[kMaxCalls];
int entries = 0;

// The calls of one bound plan.
struct Marshal {
    PyObject_HEAD
    vectorcallfunc vectorcall;
    const void *plan;
    PyObject *fail;                   // fail(status, call) raises
    int64_t elem_bytes;
    int64_t numel[kBuffers];          // elements of V, Vbar, X, D, Phi
};

// marshal(call, [node,] tensor, ...) -> 0, or None: not an ordinary call.  Raises what fail() makes of another status.
PyObject *marshal_call(PyObject *self, PyObject *const *args, size_t nargsf, PyObject *kwnames)
{
    const Marshal *m = reinterpret_cast<const Marshal *>(self);
    const Py_ssize_t n = PyVectorcall_NARGS(nargsf);
    if (kwnames || n < 1 || at::impl::torch_function_mode_enabled()) Py_RETURN_NONE;
    const long id = PyLong_AsLong(args[0]);
    if (id < 0 || id >= entries) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    const Entry &e = table[id];
    const Py_ssize_t first = e.node ? 2 : 1;
    if (n != first + e.tensors) Py_RETURN_NONE;
    int node = 0;
    if (e.node) {
        if (!PyLong_CheckExact(args[1])) Py_RETURN_NONE;
        const long v = PyLong_AsLong(args[1]);
        if (v < -1 || v > INT32_MAX || (v == -1 && PyErr_Occurred())) {       // no long either: -1 and an exception
            PyErr_Clear();
            Py_RETURN_NONE;
        }
        node = (int)v;
    }
    void *ptr[kMaxTensors];
    void *stream;
    try {
        for (int i = 0; i < e.tensors; i++) {
            PyObject *o = args[first + i];
            if (!THPVariable_CheckExact(o)) Py_RETURN_NONE;
            const at::Tensor &t = THPVariable_Unpack(o);
            if (t.numel() != m->numel[e.buffer[i]] || !t.is_cuda() || !t.is_contiguous() || (int64_t)t.element_size() != m->elem_bytes)
                Py_RETURN_NONE;
            ptr[i] = t.data_ptr();
        }
        stream = c10::hip::getCurrentHIPStream().stream();
    } catch (...) {
        Py_RETURN_NONE;
    }
    int status;
    Py_BEGIN_ALLOW_THREADS
    const void *plan = m->plan;
    if (e.node)
        status = e.tensors == 2 ? reinterpret_cast<NodeCall2>(e.fn)(plan, node, ptr[0], ptr[1], stream)
                                : reinterpret_cast<NodeCall3>(e.fn)(plan, node, ptr[0], ptr[1], ptr[2], stream);
    else
        status = e.tensors == 2 ? reinterpret_cast<Call2>(e.fn)(plan, ptr[0], ptr[1], stream)
                                : reinterpret_cast<Call3>(e.fn)(plan, ptr[0], ptr[1], ptr[2], stream);
    Py_END_ALLOW_THREADS
    if (status != 0) return PyObject_CallFunction(m->fail, "il", status, id);
    return PyLong_FromLong(0);
}

// Marshal(plan, fail, elem_bytes, elements of V, Vbar, X, D, Phi)
PyObject *marshal_new(PyTypeObject *type, PyObject *args, PyObject *)
{
    unsigned long long plan;
    long long elem_bytes, numel[kBuffers];
    PyObject *fail;
    if (!PyArg_ParseTuple(args, "KOLLLLLL", &plan, &fail, &elem_bytes, &numel[0], &numel[1], &numel[2], &numel[3], &numel[4]))
        return nullptr;
    PyObject *self = type->tp_alloc(type, 0);
    if (!self) return nullptr;
    Marshal *m = reinterpret_cast<Marshal *>(self);
    m->vectorcall = marshal_call;
    m->plan = reinterpret_cast<const void *>((uintptr_t)plan);
    m->fail = Py_NewRef(fail);
    m->elem_bytes = elem_bytes;
    for (int i = 0; i < kBuffers; i++) m->numel[i] = numel[i];
    return self;
}

// calls([(function address, takes a node, (buffer, ...)), ...]): once, when the library is loaded
PyObject *set_calls(PyObject *, PyObject *calls)
{
    if (!PyList_Check(calls) || PyList_GET_SIZE(calls) > kMaxCalls) {
        PyErr_SetString(PyExc_ValueError, "a list of calls");
        return nullptr;
    }
    Entry read[kMaxCalls];
    for (Py_ssize_t i = 0; i < PyList_GET_SIZE(calls); i++) {
        unsigned long long fn;
        int node;
        PyObject *buffers;
        if (!PyArg_ParseTuple(PyList_GET_ITEM(calls, i), "KpO!", &fn, &node, &PyTuple_Type, &buffers)) return nullptr;
        Entry &e = read[i];
        e.fn = (uintptr_t)fn;
        e.node = node != 0;
        e.tensors = (int)PyTuple_GET_SIZE(buffers);
        for (int t = 0; t < e.tensors && t < kMaxTensors; t++) {
            const long b = PyLong_AsLong(PyTuple_GET_ITEM(buffers, t));
            if (b < 0 || b >= kBuffers) e.tensors = -1;
            else e.buffer[t] = (int)b;
        }
        if (PyErr_Occurred()) return nullptr;
        if (e.tensors < 2 || e.tensors > kMaxTensors) {
            PyErr_SetString(PyExc_ValueError, "two or three buffers of five");
            return nullptr;
        }
    }
    entries = (int)PyList_GET_SIZE(calls);
    for (int i = 0; i < entries; i++) table[i] = read[i];
    Py_RETURN_NONE;
}

void marshal_dealloc(PyObject *self)
{
    Py_XDECREF(reinterpret_cast<Marshal *>(self)->fail);
    Py_TYPE(self)->tp_free(self);
}

// The calls of one bound block (ccdc_block), in the same manner: what binding.py's Block would hand over, or None.  A call of
// ccdc_join_forward on eight rows took 10.7 us through Python, 6 of them the kernel.
enum BlockCall { kFfnForward, kFfnBackward, kJoinForward, kJoinBackward, kDropout, kQuantise, kPackedProduct, kTop, kDistill, kBlockCalls };

struct BlockMarshal {
    PyObject_HEAD
    vectorcallfunc vectorcall;
    const void *block;
    PyObject *fail;                   // fail(status, call) raises
    at::ScalarType type;
    int64_t width, hidden, tokens, files, saved_bytes;
    uintptr_t fn[kBlockCalls];
};

// The arguments of one call, read one after the other; `ok` is lost with the first that is not an ordinary one.
struct Reader {
    const BlockMarshal &m;
    bool ok = true;

    const at::Tensor *tensor(PyObject *o, bool typed = true)
    {
        if (!ok || !THPVariable_CheckExact(o)) return fail();
        const at::Tensor &t = THPVariable_Unpack(o);
        if (!t.is_cuda() || (typed && t.scalar_type() != m.type)) return fail();
        return &t;
    }
    const at::Tensor *fail()
    {
        ok = false;
        return nullptr;
    }
    // A matrix [rows][columns] with contiguous columns (rows -1: any, then they are its own); None: null, where that may be.
    void *matrix(PyObject *o, int64_t *rows, int64_t columns, int64_t *ld, bool none = false)
    {
        *ld = 0;
        if (none && o == Py_None) return nullptr;
        const at::Tensor *t = tensor(o);
        if (!t || t->dim() != 2 || t->size(1) != columns) return (void *)fail();
        if (*rows < 0) *rows = t->size(0);
        if (t->size(0) != *rows || (columns > 1 && t->stride(1) != 1) || (*rows > 1 && t->stride(0) < columns)) return (void *)fail();
        *ld = *rows > 1 || t->stride(0) > columns ? t->stride(0) : columns;
        return t->data_ptr();
    }
    void *parameter(PyObject *o, int64_t rows, int64_t columns, bool none = false)      // rows 0: a vector
    {
        if (none && o == Py_None) return nullptr;
        const at::Tensor *t = tensor(o);
        if (!t || !t->is_contiguous() || t->dim() != (rows ? 2 : 1) || t->size(-1) != columns || (rows && t->size(0) != rows))
            return (void *)fail();
        return t->data_ptr();
    }
    // Gradients by file, a file's part contiguous, no file's on another's; all that are given with one stride (0 in *ld: none yet, which
    // no stride is).
    void *gradient(PyObject *o, int64_t rows, int64_t columns, int64_t *ld)
    {
        if (o == Py_None) return nullptr;
        const at::Tensor *t = tensor(o);
        const int last = rows ? 2 : 1;
        if (!t || t->dim() != last + 1 || t->size(0) != m.files || t->size(last) != columns || (rows && t->size(1) != rows)) return (void *)fail();
        if ((columns > 1 && t->stride(last) != 1) || (rows > 1 && t->stride(1) != columns)) return (void *)fail();
        if (m.files > 1) {
            if (t->stride(0) < (rows ? rows : 1) * columns || (*ld && *ld != t->stride(0))) return (void *)fail();
            *ld = t->stride(0);
        }
        return t->data_ptr();
    }
    void *saved(PyObject *o, bool none)
    {
        if (none && o == Py_None) return nullptr;
        const at::Tensor *t = tensor(o, false);
        if (!t || !t->is_contiguous() || t->numel() * (int64_t)t->element_size() < m.saved_bytes) return (void *)fail();
        return t->data_ptr();
    }
    void *gate(PyObject *o, int64_t *ld)
    {
        *ld = 0;
        if (o == Py_None) return nullptr;
        const at::Tensor *t = tensor(o);
        if (!t) return nullptr;
        if (t->dim() == 1) return parameter(o, 0, m.width);
        int64_t files = m.files;
        return matrix(o, &files, m.width, ld);
    }
    // For the calls that learn from a teacher.  A tensor of this type on the current device, contiguous, of these sizes (columns 0: a
    // vector); None: null, where that may be.
    void *plain(PyObject *o, at::ScalarType type, int64_t rows, int64_t columns, bool none = false)
    {
        if (none && o == Py_None) return nullptr;
        const at::Tensor *t = tensor(o, false);
        if (!t || t->scalar_type() != type || !here(*t) || !t->is_contiguous() || t->dim() != (columns ? 2 : 1) || t->size(0) != rows ||
            (columns && t->size(1) != columns))
            return (void *)fail();
        return t->data_ptr();
    }
    // A matrix in 8 bits and its scales (rows, wide -1: any, then they are its own).
    void *eight(PyObject *o, PyObject *scales, int64_t *rows, int64_t *wide, void **scale)
    {
        const at::Tensor *t = tensor(o, false);
        if (!t || (t->scalar_type() != at::kFloat8_e4m3fn && t->scalar_type() != at::kByte) || t->dim() != 2) return (void *)fail();
        if (*rows < 0) *rows = t->size(0);
        if (*wide < 0) *wide = t->size(1);
        if (*wide <= 0 || *wide % 128 != 0) return (void *)fail();
        void *at = plain(o, t->scalar_type(), *rows, *wide);
        *scale = plain(scales, at::kByte, *rows, (*wide / 128 + 3) / 4 * 4);
        return at;
    }
    // A matrix of the block's elements, on the current device.
    void *logits(PyObject *o, int64_t *rows, int64_t *columns, int64_t *ld, bool none = false)
    {
        if (none && o == Py_None) return nullptr;
        const at::Tensor *t = tensor(o);
        if (!t || t->dim() != 2 || !here(*t)) return (void *)fail();
        if (*columns < 0) *columns = t->size(1);
        return matrix(o, rows, *columns, ld);
    }
    bool here(const at::Tensor &t) { return t.get_device() == c10::hip::current_device(); }
    double real(PyObject *o)
    {
        if (!PyFloat_CheckExact(o)) ok = false;
        return ok ? PyFloat_AS_DOUBLE(o) : 0.0;
    }
    int64_t listed(PyObject *o)               // columns of a list
    {
        const at::Tensor *t = tensor(o, false);
        if (!t || t->dim() != 2 || t->size(1) < 1) fail();
        return ok ? t->size(1) : 0;
    }
    unsigned long long number(PyObject *o)
    {
        if (!ok || !PyLong_CheckExact(o)) {
            ok = false;
            return 0;
        }
        const unsigned long long v = PyLong_AsUnsignedLongLong(o);
        if (PyErr_Occurred()) {
            PyErr_Clear();
            ok = false;
        }
        return v;
    }
    // The row stride that all matrices of more than one row have.
    int64_t common(int64_t rows, std::initializer_list<std::pair<void *, int64_t>> all)
    {
        int64_t ld = 0;
        for (const auto &one : all)
            if (one.first && rows > 1) {
                if (ld && ld != one.second) ok = false;
                ld = one.second;
            }
        return ld ? ld : m.width;
    }
};

using p = void *;
using FfnForward = int (*)(const void *, int64_t, p, int64_t, p, p, p, int64_t, p, uint64_t, p);
using FfnBackward = int (*)(const void *, p, int64_t, p, p, p, p, int64_t, p, int64_t, p, int64_t, p, int64_t, p);
using JoinForward = int (*)(const void *, int64_t, p, p, p, p, int64_t, p, p, p, int64_t, uint64_t, p);
using JoinBackward = int (*)(const void *, p, p, p, p, p, p, int64_t, p, p, p, int64_t, p, p, p, int64_t, uint64_t, p);
using Quantise = int (*)(const void *, int64_t, int64_t, p, int64_t, p, p, p);
using PackedProduct = int (*)(const void *, int64_t, int64_t, int64_t, p, p, p, p, p, int64_t, p);
using Top = int (*)(const void *, int64_t, int64_t, p, int64_t, int, double, p, p, p, p);
using Distill = int (*)(const void *, int64_t, int64_t, p, int64_t, int, p, p, p, double, p, double, p, p, int64_t, p);
using DropoutCall = int (*)(const void *, int64_t, int64_t, double, uint32_t, uint64_t, p, int64_t, p, int64_t, p, int64_t, p);

// block(call, argument, ...) in the order of binding.py's methods
PyObject *block_call(PyObject *self, PyObject *const *args, size_t nargsf, PyObject *kwnames)
{
    const BlockMarshal &m = *reinterpret_cast<const BlockMarshal *>(self);
    static constexpr Py_ssize_t count[kBlockCalls] = {6, 8, 8, 13, 6, 3, 5, 5, 9};
    const Py_ssize_t n = PyVectorcall_NARGS(nargsf);
    if (kwnames || n < 1 || at::impl::torch_function_mode_enabled()) Py_RETURN_NONE;
    const long id = PyLong_AsLong(args[0]);
    if (id < 0 || id >= kBlockCalls || n != 1 + count[id]) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    PyObject *const *a = args + 1;
    const int64_t d = m.width, F = m.hidden;
    Reader r{m};
    int status = 0;
    try {
        void *stream = c10::hip::getCurrentHIPStream().stream();
        int64_t rows = id == kFfnBackward || id == kJoinBackward ? m.tokens : -1, l[6];
        switch (id) {
        case kFfnForward: {
            p x = r.matrix(a[0], &rows, d, &l[0]), in = r.parameter(a[1], 2 * F, d), out = r.parameter(a[2], d, F);
            p y = r.matrix(a[3], &rows, d, &l[1]), saved = r.saved(a[4], true);
            const uint64_t seed = r.number(a[5]);
            if (!r.ok) Py_RETURN_NONE;
            Py_BEGIN_ALLOW_THREADS
            status = reinterpret_cast<FfnForward>(m.fn[id])(m.block, rows, x, l[0], in, out, y, l[1], saved, seed, stream);
            Py_END_ALLOW_THREADS
            break;
        }
        case kFfnBackward: {
            int64_t ld_in = 0, ld_out = 0;
            p x = r.matrix(a[0], &rows, d, &l[0]), in = r.parameter(a[1], 2 * F, d), out = r.parameter(a[2], d, F), saved = r.saved(a[3], false);
            p dy = r.matrix(a[4], &rows, d, &l[1]), dx = r.matrix(a[5], &rows, d, &l[2], true);
            p din = r.gradient(a[6], 2 * F, d, &ld_in), dout = r.gradient(a[7], d, F, &ld_out);
            if (!r.ok) Py_RETURN_NONE;
            Py_BEGIN_ALLOW_THREADS
            status = reinterpret_cast<FfnBackward>(m.fn[id])(m.block, x, l[0], in, out, saved, dy, l[1], dx, l[2], din, ld_in, dout, ld_out, stream);
            Py_END_ALLOW_THREADS
            break;
        }
        case kJoinForward: {
            int64_t lg;
            p x = r.matrix(a[0], &rows, d, &l[0]), f = r.matrix(a[1], &rows, d, &l[1], true), y = r.matrix(a[2], &rows, d, &l[2], true);
            p out = r.matrix(a[3], &rows, d, &l[3], true), post = r.parameter(a[4], 0, d, true), gate = r.gate(a[5], &lg);
            p pre = r.parameter(a[6], 0, d, true);
            const uint64_t seed = r.number(a[7]);
            const int64_t ld = r.common(rows, {{x, l[0]}, {f, l[1]}, {y, l[2]}, {out, l[3]}});
            if (!r.ok) Py_RETURN_NONE;
            Py_BEGIN_ALLOW_THREADS
            status = reinterpret_cast<JoinForward>(m.fn[id])(m.block, rows, x, f, post, gate, lg, pre, y, out, ld, seed, stream);
            Py_END_ALLOW_THREADS
            break;
        }
        case kJoinBackward: {
            int64_t lg, ld_file = 0;
            p t[6];
            for (int i = 0; i < 6; i++) t[i] = r.matrix(a[i], &rows, d, &l[i], true);
            p post = r.parameter(a[6], 0, d, true), gate = r.gate(a[7], &lg), pre = r.parameter(a[8], 0, d, true);
            p dpost = r.gradient(a[9], 0, d, &ld_file), dgate = r.gradient(a[10], 0, d, &ld_file), dpre = r.gradient(a[11], 0, d, &ld_file);
            const uint64_t seed = r.number(a[12]);
            const int64_t ld = r.common(rows, {{t[0], l[0]}, {t[1], l[1]}, {t[2], l[2]}, {t[3], l[3]}, {t[4], l[4]}, {t[5], l[5]}});
            if (!r.ok) Py_RETURN_NONE;
            Py_BEGIN_ALLOW_THREADS
            status = reinterpret_cast<JoinBackward>(m.fn[id])(m.block, t[0], t[1], t[2], t[3], post, gate, lg, pre, t[4], t[5], ld, dpost,
                                                              dgate, dpre, ld_file, seed, stream);
            Py_END_ALLOW_THREADS
            break;
        }
        case kQuantise: {
            int64_t columns = -1;
            p x = r.logits(a[0], &rows, &columns, &l[0]);
            if (!r.ok || columns < 1) Py_RETURN_NONE;
            int64_t wide = (columns + 127) / 128 * 128;
            p scale, q = r.eight(a[1], a[2], &rows, &wide, &scale);
            if (!r.ok) Py_RETURN_NONE;
            Py_BEGIN_ALLOW_THREADS
            status = reinterpret_cast<Quantise>(m.fn[id])(m.block, rows, columns, x, l[0], q, scale, stream);
            Py_END_ALLOW_THREADS
            break;
        }
        case kPackedProduct: {
            int64_t wide = -1, outputs = -1;
            p x_scale, w_scale, x = r.eight(a[0], a[1], &rows, &wide, &x_scale), w = r.eight(a[2], a[3], &outputs, &wide, &w_scale);
            p y = r.ok ? r.logits(a[4], &rows, &outputs, &l[0]) : nullptr;
            if (!r.ok) Py_RETURN_NONE;
            Py_BEGIN_ALLOW_THREADS
            status = reinterpret_cast<PackedProduct>(m.fn[id])(m.block, rows, outputs, wide, x, x_scale, w, w_scale, y, l[0], stream);
            Py_END_ALLOW_THREADS
            break;
        }
        case kTop: {
            int64_t columns = -1;
            p z = r.logits(a[0], &rows, &columns, &l[0]);
            const int64_t k = r.listed(a[1]);
            p index = r.plain(a[1], at::kInt, rows, k), value = r.plain(a[2], at::kFloat, rows, k), rest = r.plain(a[3], at::kFloat, rows, 0, true);
            const double temperature = r.real(a[4]);
            if (!r.ok || k > INT32_MAX) Py_RETURN_NONE;
            Py_BEGIN_ALLOW_THREADS
            status = reinterpret_cast<Top>(m.fn[id])(m.block, rows, columns, z, l[0], (int)k, temperature, index, value, rest, stream);
            Py_END_ALLOW_THREADS
            break;
        }
        case kDistill: {
            int64_t columns = -1;
            p z = r.logits(a[0], &rows, &columns, &l[0]);
            const int64_t k = r.listed(a[1]);
            p index = r.plain(a[1], at::kInt, rows, k), value = r.plain(a[2], at::kFloat, rows, k), loss = r.plain(a[3], at::kFloat, rows, 0, true);
            p dz = r.ok ? r.logits(a[4], &rows, &columns, &l[1], true) : nullptr, rest = r.plain(a[5], at::kFloat, rows, 0, true);
            const double temperature = r.real(a[6]);
            p weight = r.plain(a[7], at::kFloat, rows, 0, true);
            const double scale = r.real(a[8]);
            if (!r.ok || k > INT32_MAX) Py_RETURN_NONE;
            if (dz == nullptr) l[1] = 0;
            Py_BEGIN_ALLOW_THREADS
            status = reinterpret_cast<Distill>(m.fn[id])(m.block, rows, columns, z, l[0], (int)k, index, value, rest, temperature, weight, scale,
                                                         loss, dz, l[1], stream);
            Py_END_ALLOW_THREADS
            break;
        }
        default: {
            const at::Tensor *t = r.tensor(a[0]);
            if (!t || t->dim() != 2 || !PyFloat_CheckExact(a[2])) Py_RETURN_NONE;
            const int64_t columns = t->size(1);
            p x = r.matrix(a[0], &rows, columns, &l[0]), y = r.matrix(a[1], &rows, columns, &l[1]);
            const unsigned long long site = r.number(a[3]), seed = r.number(a[4]);
            p residual = r.matrix(a[5], &rows, columns, &l[2], true);
            if (!r.ok || site > UINT32_MAX) Py_RETURN_NONE;
            const double prob = PyFloat_AS_DOUBLE(a[2]);
            Py_BEGIN_ALLOW_THREADS
            status = reinterpret_cast<DropoutCall>(m.fn[id])(m.block, rows, columns, prob, (uint32_t)site, seed, x, l[0], residual, l[2], y, l[1], stream);
            Py_END_ALLOW_THREADS
        }
        }
    } catch (...) {
        Py_RETURN_NONE;
    }
    if (status != 0) return PyObject_CallFunction(m.fail, "il", status, id);
    return PyLong_FromLong(0);
}

// Block(block, fail, bytes of an element or 3 for binary16, width, hidden, tokens, files, saved bytes, address, ...)
PyObject *block_new(PyTypeObject *type, PyObject *args, PyObject *)
{
    unsigned long long block, fn[kBlockCalls];
    long long format, width, hidden, tokens, files, saved;
    PyObject *fail;
    if (!PyArg_ParseTuple(args, "KOLLLLLLKKKKKKKKK", &block, &fail, &format, &width, &hidden, &tokens, &files, &saved, &fn[0], &fn[1], &fn[2],
                          &fn[3], &fn[4], &fn[5], &fn[6], &fn[7], &fn[8]))
        return nullptr;
    PyObject *self = type->tp_alloc(type, 0);
    if (!self) return nullptr;
    BlockMarshal *m = reinterpret_cast<BlockMarshal *>(self);
    m->vectorcall = block_call;
    m->block = reinterpret_cast<const void *>((uintptr_t)block);
    m->fail = Py_NewRef(fail);
    m->type = format == 4 ? at::kFloat : format == 3 ? at::kHalf : at::kBFloat16;
    m->width = width, m->hidden = hidden, m->tokens = tokens, m->files = files, m->saved_bytes = saved;
    for (int i = 0; i < kBlockCalls; i++) m->fn[i] = (uintptr_t)fn[i];
    return self;
}

void block_dealloc(PyObject *self)
{
    Py_XDECREF(reinterpret_cast<BlockMarshal *>(self)->fail);
    Py_TYPE(self)->tp_free(self);
}

PyTypeObject marshal_type = {PyVarObject_HEAD_INIT(nullptr, 0)};
PyTypeObject block_type = {PyVarObject_HEAD_INIT(nullptr, 0)};
PyMethodDef functions[] = {{"calls", set_calls, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, functions, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void)
{
    marshal_type.tp_name = "_marshal.Marshal";
    marshal_type.tp_basicsize = sizeof(Marshal);
    marshal_type.tp_flags = Py_TPFLAGS_DEFAULT | Py_TPFLAGS_HAVE_VECTORCALL;
    marshal_type.tp_vectorcall_offset = offsetof(Marshal, vectorcall);
    marshal_type.tp_call = PyVectorcall_Call;
    marshal_type.tp_new = marshal_new;
    marshal_type.tp_dealloc = marshal_dealloc;
    block_type.tp_name = "_marshal.Block";
    block_type.tp_basicsize = sizeof(BlockMarshal);
    block_type.tp_flags = Py_TPFLAGS_DEFAULT | Py_TPFLAGS_HAVE_VECTORCALL;
    block_type.tp_vectorcall_offset = offsetof(BlockMarshal, vectorcall);
    block_type.tp_call = PyVectorcall_Call;
    block_type.tp_new = block_new;
    block_type.tp_dealloc = block_dealloc;
    if (PyType_Ready(&marshal_type) < 0 || PyType_Ready(&block_type) < 0) return nullptr;
    PyObject *m = PyModule_Create(&module);
    if (!m) return nullptr;
    for (auto [name, type] : {std::make_pair("Marshal", &marshal_type), std::make_pair("Block", &block_type)}) {
        Py_INCREF(type);
        if (PyModule_AddObject(m, name, reinterpret_cast<PyObject *>(type)) < 0) {
            Py_DECREF(type);
            Py_DECREF(m);
            return nullptr;
        }
    }
    return m;
}
