// Operator calls from Python without an interpreter in between: reads the tensors, the shape and the record,
// lays out the plan, allocates the output and the split-K workspace where the caller gave none, and launches.
//
// A small kernel runs for 4 to 6 us.  Marshalled in Python (a plan for the workspace size, eleven ctypes
// arguments, the stream lookup, a second plan inside the entry point) its call took 10 to 12 us of host time, so
// a program's small calls ran at the interpreter's pace; from here a call takes about 3 us, most of it the
// runtime's launch.
//
// The functions mirror the wrappers of api.py, which pass their arguments on and raise TTError for a status.
#include <Python.h>

#include <ATen/ops/empty.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "tt_internal.h"

using namespace tt;

namespace {

// What the binding hands over once: its structure types, and functions for what is rare enough for Python.
PyObject *conv_shape_type, *gemm_shape_type, *schedule_type;
PyObject *refuse_struct;  // (object, expected type): raises what ctypes raises for such an argument
PyObject *empty_tensor;   // (x, sizes): an output of x's type and place

// A reference that ends with the scope.
class Owned {
public:
    explicit Owned(PyObject *o) : o_(o)
    {
        if (!o) throw python_error();
    }
    ~Owned() { Py_DECREF(o_); }
    Owned(const Owned &) = delete;
    Owned &operator=(const Owned &) = delete;
    PyObject *get() const { return o_; }

private:
    PyObject *o_;
};

// The contents of a ctypes structure of one type (or a type derived from it): a buffer of the right size alone could be a
// structure of another layout.
template <class T> T struct_of(PyObject *obj, PyObject *type)
{
    TORCH_CHECK(type, "_ttcall is used through the binding");
    int ok = (PyObject *)Py_TYPE(obj) == type;
    if (!ok) ok = PyObject_IsInstance(obj, type);
    if (ok < 0) throw python_error();
    if (!ok) {
        Owned unreachable(PyObject_CallFunctionObjArgs(refuse_struct, obj, type, nullptr));
        TORCH_CHECK_TYPE(false, "wrong type");
    }
    Py_buffer view;
    if (PyObject_GetBuffer(obj, &view, PyBUF_SIMPLE) != 0) throw python_error();
    const bool whole = (size_t)view.len >= sizeof(T);
    T out{};
    if (whole) out = *static_cast<const T *>(view.buf);
    PyBuffer_Release(&view);
    TORCH_CHECK_TYPE(whole, "structure without its contents");
    return out;
}

// Address of an argument: null for None, and for anything but a plain tensor what its own data_ptr() says.
void *address_of(PyObject *o)
{
    if (o == Py_None) return nullptr;
    if (THPVariable_CheckExact(o)) return THPVariable_Unpack(o).data_ptr();
    Owned at(PyObject_CallMethod(o, "data_ptr", nullptr));
    if (at.get() == Py_None) return nullptr;
    void *const p = PyLong_AsVoidPtr(at.get());
    if (!p && PyErr_Occurred()) throw python_error();
    return p;
}

int64_t integer_from(PyObject *o, const char *method)
{
    Owned v(PyObject_CallMethod(o, method, nullptr));
    const long long n = PyLong_AsLongLong(v.get());
    if (n == -1 && PyErr_Occurred()) throw python_error();
    return n;
}
size_t bytes_of(PyObject *o)
{
    if (THPVariable_CheckExact(o)) return THPVariable_Unpack(o).nbytes();
    return (size_t)(integer_from(o, "numel") * integer_from(o, "element_size"));
}

// The output of a call: the caller's, or a new one of x's type and place, which becomes a Python object behind the launch.
class Output {
public:
    Output(PyObject *given, PyObject *x, at::IntArrayRef sizes)
    {
        if (given != Py_None) {
            object_ = Py_NewRef(given);
        } else if (THPVariable_CheckExact(x)) {
            made_ = at::empty(sizes, THPVariable_Unpack(x).options());
        } else {
            Owned tuple(PyTuple_New((Py_ssize_t)sizes.size()));
            for (size_t i = 0; i < sizes.size(); ++i) PyTuple_SET_ITEM(tuple.get(), i, PyLong_FromLongLong(sizes[i]));
            object_ = PyObject_CallFunctionObjArgs(empty_tensor, x, tuple.get(), nullptr);
            if (!object_) throw python_error();
        }
    }
    ~Output() { Py_XDECREF(object_); }
    Output(const Output &) = delete;
    Output &operator=(const Output &) = delete;
    void *address() const { return object_ ? address_of(object_) : made_.data_ptr(); }
    PyObject *result() { return object_ ? Py_NewRef(object_) : THPVariable_Wrap(std::move(made_)); }

private:
    PyObject *object_ = nullptr;
    at::Tensor made_;
};

int class_of(PyObject *o)
{
    const long cls = PyLong_AsLong(o);
    if (cls == -1 && PyErr_Occurred()) throw python_error();
    return (int)cls;
}

int64_t out_extent(int64_t in, int64_t pad, int64_t filter, int64_t stride)
{
    const int64_t n = in + 2 * pad - filter;
    if (stride == 0) {
        PyErr_SetString(PyExc_ZeroDivisionError, "integer division or modulo by zero");
        throw python_error();
    }
    return n / stride - (n % stride != 0 && (n < 0) != (stride < 0)) + 1; // rounded down
}

void *current_stream() { return c10::hip::getCurrentHIPStream().stream(); }

// Plan, workspace, launch.  Returns the output, or the status as a Python integer.
PyObject *call(int cls, const void *shape, PyObject *sched, OpPointers p, PyObject *ws, Output &out)
{
    int rc = TT_OK;
    at::Tensor own_ws;
    PreparedOp op;
    {
        tt_schedule rec;
        if (sched != Py_None) rec = struct_of<tt_schedule>(sched, schedule_type);
        if (ws != Py_None) {
            p.ws = address_of(ws);
            p.ws_bytes = bytes_of(ws);
        }
        p.out = out.address();
        rc = check_op_pointers(cls, p);
        if (rc == TT_OK) rc = prepare_op(sched != Py_None ? &rec : nullptr, cls, shape, &op);
        if (rc == TT_OK && ws == Py_None && op.plan.workspace_bytes > 0) {
            own_ws = at::empty({op.plan.workspace_bytes}, at::TensorOptions().dtype(at::kByte).device(at::kCUDA));
            p.ws = own_ws.data_ptr();
            p.ws_bytes = (size_t)op.plan.workspace_bytes;
        }
    }
    if (rc == TT_OK) {
        void *const stream = current_stream();
        Py_BEGIN_ALLOW_THREADS rc = launch_op(op, &p, 1, stream); // (a full queue makes a launch wait)
        Py_END_ALLOW_THREADS
    }
    return rc == TT_OK ? out.result() : PyLong_FromLong(rc);
}

// conv2d(x, w, bias, residual, shape, cls, sched, ws, y)
PyObject *py_conv2d(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    TORCH_CHECK_TYPE(n == 9, "conv2d takes nine arguments");
    const tt_conv_shape s = struct_of<tt_conv_shape>(a[4], conv_shape_type);
    const int cls = class_of(a[5]);
    const int64_t ho = out_extent(s.h, s.pad_h, s.r, s.stride_h), wo = out_extent(s.w, s.pad_w, s.s, s.stride_w);
    Output out(a[8], a[0], {s.n, s.k, ho, wo});
    if (!is_conv_class(cls)) return PyLong_FromLong(TT_ERR_BAD_ARG);
    return call(cls, &s, a[6], {address_of(a[0]), address_of(a[1]), address_of(a[2]), address_of(a[3]), nullptr, nullptr, 0}, a[7], out);
    END_HANDLE_TH_ERRORS
}

// dense(x, w, bias, shape, cls, sched, ws, y)
PyObject *py_dense(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    TORCH_CHECK_TYPE(n == 8, "dense takes eight arguments");
    const tt_gemm_shape s = struct_of<tt_gemm_shape>(a[3], gemm_shape_type);
    const int cls = class_of(a[4]);
    Output out(a[7], a[0], {s.m, s.n});
    if (!is_dense_class(cls)) return PyLong_FromLong(TT_ERR_BAD_ARG);
    return call(cls, &s, a[5], {address_of(a[0]), address_of(a[1]), address_of(a[2]), nullptr, nullptr, nullptr, 0}, a[6], out);
    END_HANDLE_TH_ERRORS
}

// matmul(a, b, shape, sched, ws, c)
PyObject *py_matmul(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    TORCH_CHECK_TYPE(n == 6, "matmul takes six arguments");
    const tt_gemm_shape s = struct_of<tt_gemm_shape>(a[2], gemm_shape_type);
    Output out(a[5], a[0], {s.batch, s.m, s.n});
    return call(TT_BATCH_MATMUL, &s, a[3], {address_of(a[0]), address_of(a[1]), nullptr, nullptr, nullptr, nullptr, 0}, a[4], out);
    END_HANDLE_TH_ERRORS
}

// dwconv(x, w, bias, shape, sched, y)
PyObject *py_dwconv(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    TORCH_CHECK_TYPE(n == 6, "dwconv takes six arguments");
    const tt_conv_shape s = struct_of<tt_conv_shape>(a[3], conv_shape_type);
    const int64_t ho = out_extent(s.h, s.pad_h, s.r, s.stride_h), wo = out_extent(s.w, s.pad_w, s.s, s.stride_w);
    Output out(a[5], a[0], {s.n, s.c, ho, wo});
    return call(TT_DWCONV_BIAS_RELU6, &s, a[4], {address_of(a[0]), address_of(a[1]), address_of(a[2]), nullptr, nullptr, nullptr, 0}, Py_None, out);
    END_HANDLE_TH_ERRORS
}

// ---- matrices held in 8 bits, group norm ----------------------------------------------------------------
// Unlike the records' operators these know the type and size of every argument, so a tensor is taken only if it is of that
// type, as large as the shape says, dense, and on the current device, whatever its class.  (What is no tensor is the caller's own
// memory.)

PyObject *quant_shape_type, *fp8_shape_type, *norm_shape_type;

class Checked {
public:
    void *address(PyObject *o, at::ScalarType type, int64_t numel)
    {
        if (!is_tensor(o)) return address_of(o);
        const at::Tensor &t = THPVariable_Unpack(o);
        good_ = good_ && t.scalar_type() == type && t.numel() == numel && t.is_contiguous() && on_device(t);
        void *const p = good_ ? address_of(o) : nullptr;
        good_ = p != nullptr; // (a tensor without memory is not an argument left out)
        return p;
    }
    // A workspace is memory of any type; `bytes`: how many there are.
    void *workspace(PyObject *o, size_t *bytes)
    {
        *bytes = o == Py_None ? 0 : bytes_of(o);
        if (!is_tensor(o)) return address_of(o);
        const at::Tensor &t = THPVariable_Unpack(o);
        good_ = good_ && t.is_contiguous() && on_device(t);
        return good_ ? address_of(o) : nullptr;
    }
    bool good() const { return good_; }

private:
    // (a call that asks Python about an argument's class is left to those that are neither)
    static bool is_tensor(PyObject *o) { return THPVariable_CheckExact(o) || (o != Py_None && THPVariable_Check(o)); }
    static bool on_device(const at::Tensor &t) { return t.is_cuda() && t.device().index() == c10::hip::current_device(); }
    bool good_ = true;
};

at::ScalarType type_of(int32_t dtype) { return dtype == TT_F32 ? at::kFloat : at::kBFloat16; }
int64_t blocks_of(int64_t n) { return (n + TT_FP8_BLOCK - 1) / TT_FP8_BLOCK; }

// A new tensor on the current device, or the caller's.
PyObject *output_object(PyObject *given, at::IntArrayRef sizes, at::ScalarType type)
{
    if (given != Py_None) return Py_NewRef(given);
    return THPVariable_Wrap(at::empty(sizes, at::TensorOptions().dtype(type).device(at::kCUDA, c10::hip::current_device())));
}
class Workspace {
public:
    Workspace(Checked &check, PyObject *given, int64_t needed)
    {
        at_ = check.workspace(given, &bytes_);
        if (given != Py_None || needed == 0 || !check.good()) return;
        own_ = at::empty({needed}, at::TensorOptions().dtype(at::kByte).device(at::kCUDA, c10::hip::current_device()));
        at_ = own_.data_ptr(), bytes_ = (size_t)needed;
    }
    void *at_;
    size_t bytes_;

private:
    at::Tensor own_;
};
template <class F> int launched(const Checked &check, F &&launch)
{
    if (!check.good()) return TT_ERR_BAD_ARG;
    int rc;
    Py_BEGIN_ALLOW_THREADS rc = launch();
    Py_END_ALLOW_THREADS
    return rc;
}

// quantize_fp8(x, shape, q, scale)
PyObject *py_quantize_fp8(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    TORCH_CHECK_TYPE(n == 4, "quantize_fp8 takes four arguments");
    const tt_quant_shape s = struct_of<tt_quant_shape>(a[1], quant_shape_type);
    if (const int rc = check_quant_shape(s); rc != TT_OK) return PyLong_FromLong(rc);
    Checked check;
    const int64_t kb = blocks_of(s.cols), rb = (s.rows + s.block_rows - 1) / s.block_rows;
    const void *const x = check.address(a[0], type_of(s.dtype), (int64_t)s.batch * s.rows * s.cols);
    if (!check.good()) return PyLong_FromLong(TT_ERR_BAD_ARG);
    Owned q(output_object(a[2], {s.batch, s.rows, kb * TT_FP8_BLOCK}, at::kFloat8_e4m3fn));
    Owned scale(output_object(a[3], {s.batch, kb, rb}, at::kFloat));
    void *const qp = check.address(q.get(), at::kFloat8_e4m3fn, (int64_t)s.batch * s.rows * kb * TT_FP8_BLOCK);
    void *const sp = check.address(scale.get(), at::kFloat, s.batch * kb * rb);
    void *const stream = current_stream();
    const int rc = launched(check, [&] { return tt_quantize_fp8(x, qp, static_cast<float *>(sp), &s, stream); });
    return rc == TT_OK ? PyTuple_Pack(2, q.get(), scale.get()) : PyLong_FromLong(rc);
    END_HANDLE_TH_ERRORS
}

// cls < 0: tt_batch_matmul_fp8
PyObject *product_fp8(PyObject *ap, PyObject *as, PyObject *bp, PyObject *bs, PyObject *bias, PyObject *shape, int cls, PyObject *ws, PyObject *out)
{
    const tt_fp8_shape s = struct_of<tt_fp8_shape>(shape, fp8_shape_type);
    tt_fp8_launch l;
    if (cls >= 0 && (!is_dense_class(cls) || s.batch != 1)) return PyLong_FromLong(TT_ERR_BAD_ARG);
    if (const int rc = tt_fp8_plan(&s, &l); rc != TT_OK) return PyLong_FromLong(rc);
    Checked check;
    const int64_t kb = blocks_of(s.k);
    const void *const a = check.address(ap, at::kFloat8_e4m3fn, (int64_t)s.batch * s.m * kb * TT_FP8_BLOCK);
    const void *const b = check.address(bp, at::kFloat8_e4m3fn, (int64_t)s.batch * s.n * kb * TT_FP8_BLOCK);
    const auto *const a_scale = static_cast<const float *>(check.address(as, at::kFloat, s.batch * kb * s.m));
    const auto *const b_scale = static_cast<const float *>(check.address(bs, at::kFloat, s.batch * kb * ((s.n + s.b_rows - 1) / s.b_rows)));
    const void *const bi = check.address(bias, type_of(s.dtype), s.n);
    if (!check.good()) return PyLong_FromLong(TT_ERR_BAD_ARG);
    const int64_t sizes[3] = {s.batch, s.m, s.n};
    Owned y(output_object(out, at::IntArrayRef(sizes + (cls >= 0), cls >= 0 ? 2 : 3), type_of(s.dtype)));
    void *const c = check.address(y.get(), type_of(s.dtype), (int64_t)s.batch * s.m * s.n);
    const Workspace w(check, ws, l.workspace_bytes);
    void *const stream = current_stream();
    const int rc = launched(check, [&] {
        return cls >= 0 ? tt_dense_fp8(a, a_scale, b, b_scale, bi, c, &s, cls, w.at_, w.bytes_, stream)
                        : tt_batch_matmul_fp8(a, a_scale, b, b_scale, c, &s, w.at_, w.bytes_, stream);
    });
    return rc == TT_OK ? Py_NewRef(y.get()) : PyLong_FromLong(rc);
}
// dense_fp8(x, x_scale, w, w_scale, bias, shape, cls, ws, y)
PyObject *py_dense_fp8(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    TORCH_CHECK_TYPE(n == 9, "dense_fp8 takes nine arguments");
    const int cls = class_of(a[6]);
    return product_fp8(a[0], a[1], a[2], a[3], a[4], a[5], cls < 0 ? TT_NUM_CLASSES : cls, a[7], a[8]);
    END_HANDLE_TH_ERRORS
}
// matmul_fp8(a, a_scale, b, b_scale, shape, ws, c)
PyObject *py_matmul_fp8(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    TORCH_CHECK_TYPE(n == 7, "matmul_fp8 takes seven arguments");
    return product_fp8(a[0], a[1], a[2], a[3], Py_None, a[4], -1, a[5], a[6]);
    END_HANDLE_TH_ERRORS
}

// `scale` null: tt_group_norm_act
PyObject *group_norm(PyObject *x, PyObject *gamma, PyObject *beta, PyObject *shape, PyObject *act_of, PyObject *eps_of, PyObject *ws, PyObject *out, PyObject *scale)
{
    const tt_norm_shape s = struct_of<tt_norm_shape>(shape, norm_shape_type);
    const int act = class_of(act_of);
    const double eps = PyFloat_AsDouble(eps_of);
    if (eps == -1.0 && PyErr_Occurred()) throw python_error();
    tt_norm_launch l;
    if (const int rc = tt_norm_plan(&s, scale != nullptr, &l); rc != TT_OK) return PyLong_FromLong(rc);
    Checked check;
    const int64_t rows = (int64_t)s.n * s.h * s.w, kb = blocks_of(s.c);
    const at::ScalarType type = type_of(s.dtype);
    const void *const xp = check.address(x, type, rows * s.c);
    const void *const gp = check.address(gamma, type, s.c), *const bp = check.address(beta, type, s.c);
    if (!check.good()) return PyLong_FromLong(TT_ERR_BAD_ARG);
    const Workspace w(check, ws, l.workspace_bytes);
    void *const stream = current_stream();
    if (!scale) {
        Owned y(output_object(out, {s.n, s.h, s.w, s.c}, type));
        void *const yp = check.address(y.get(), type, rows * s.c);
        const int rc = launched(check, [&] { return tt_group_norm_act(xp, gp, bp, yp, &s, act, (float)eps, w.at_, w.bytes_, stream); });
        return rc == TT_OK ? Py_NewRef(y.get()) : PyLong_FromLong(rc);
    }
    Owned q(output_object(out, {rows, kb * TT_FP8_BLOCK}, at::kFloat8_e4m3fn)), sc(output_object(scale, {kb, rows}, at::kFloat));
    void *const qp = check.address(q.get(), at::kFloat8_e4m3fn, rows * kb * TT_FP8_BLOCK);
    auto *const sp = static_cast<float *>(check.address(sc.get(), at::kFloat, kb * rows));
    const int rc = launched(check, [&] { return tt_group_norm_act_fp8(xp, gp, bp, qp, sp, &s, act, (float)eps, w.at_, w.bytes_, stream); });
    return rc == TT_OK ? PyTuple_Pack(2, q.get(), sc.get()) : PyLong_FromLong(rc);
}
// group_norm(x, gamma, beta, shape, act, eps, ws, y)
PyObject *py_group_norm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    TORCH_CHECK_TYPE(n == 8, "group_norm takes eight arguments");
    return group_norm(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], nullptr);
    END_HANDLE_TH_ERRORS
}
// group_norm_fp8(x, gamma, beta, shape, act, eps, ws, q, scale)
PyObject *py_group_norm_fp8(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    TORCH_CHECK_TYPE(n == 9, "group_norm_fp8 takes nine arguments");
    return group_norm(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8]);
    END_HANDLE_TH_ERRORS
}

// bind(conv shape type, gemm shape type, schedule type, refuse_struct, empty_tensor, quant shape type, fp8 shape type, norm shape
// type): once, by the binding
PyObject *py_bind(PyObject *, PyObject *args)
{
    PyObject *o[8];
    if (!PyArg_ParseTuple(args, "OOOOOOOO", &o[0], &o[1], &o[2], &o[3], &o[4], &o[5], &o[6], &o[7])) return nullptr;
    PyObject **const slots[8] = {&conv_shape_type, &gemm_shape_type, &schedule_type, &refuse_struct, &empty_tensor,
                                 &quant_shape_type, &fp8_shape_type, &norm_shape_type};
    for (int i = 0; i < 8; ++i) {
        PyObject *const before = *slots[i];
        *slots[i] = Py_NewRef(o[i]);
        Py_XDECREF(before);
    }
    Py_RETURN_NONE;
}

// The handle of the current stream of the current device.
PyObject *py_stream(PyObject *, PyObject *)
{
    HANDLE_TH_ERRORS
    return PyLong_FromVoidPtr(current_stream());
    END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"bind", py_bind, METH_VARARGS, nullptr},
    {"conv2d", (PyCFunction)(void (*)())py_conv2d, METH_FASTCALL, nullptr},
    {"dense", (PyCFunction)(void (*)())py_dense, METH_FASTCALL, nullptr},
    {"matmul", (PyCFunction)(void (*)())py_matmul, METH_FASTCALL, nullptr},
    {"dwconv", (PyCFunction)(void (*)())py_dwconv, METH_FASTCALL, nullptr},
    {"quantize_fp8", (PyCFunction)(void (*)())py_quantize_fp8, METH_FASTCALL, nullptr},
    {"dense_fp8", (PyCFunction)(void (*)())py_dense_fp8, METH_FASTCALL, nullptr},
    {"matmul_fp8", (PyCFunction)(void (*)())py_matmul_fp8, METH_FASTCALL, nullptr},
    {"group_norm", (PyCFunction)(void (*)())py_group_norm, METH_FASTCALL, nullptr},
    {"group_norm_fp8", (PyCFunction)(void (*)())py_group_norm_fp8, METH_FASTCALL, nullptr},
    {"stream", py_stream, METH_NOARGS, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ttcall", "Operator calls of libtt.", -1, methods, nullptr, nullptr, nullptr, nullptr};

} // namespace

extern "C" __attribute__((visibility("default"))) PyObject *PyInit__ttcall(void) { return PyModule_Create(&module); }
