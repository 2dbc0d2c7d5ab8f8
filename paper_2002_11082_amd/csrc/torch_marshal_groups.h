// The calls of ogq_groups.h on tensors, for torch_marshal.cpp (which holds the helpers used here): checks, allocation of what the caller left
// out, the call.  Part of that file: included once, inside its namespace.

// What bind_groups() was given.
struct BoundGroups {
    decltype(&ogq_group_codes_bytes) codes_bytes = nullptr;
    decltype(&ogq_group_exponents_count) exponents_count = nullptr;
    decltype(&ogq_group_quantize) quantize = nullptr;
    decltype(&ogq_group_dequantize) dequantize = nullptr;
    decltype(&ogq_activation_forward) forward = nullptr;
    decltype(&ogq_activation_backward) backward = nullptr;
    decltype(&ogq_weight_gradient_workspace) gradient_workspace = nullptr;
    decltype(&ogq_weight_gradient) gradient = nullptr;
    decltype(&ogq_group_matvec_workspace) matvec_workspace = nullptr;
    decltype(&ogq_group_matvec) matvec = nullptr;
    PyObject* check = nullptr;       // callable: raises OgqError for a status other than 0
    PyTypeObject* params = nullptr;  // the class of the caller's parameters
} bound_groups;

void check_groups(int status)
{
    if (status == OGQ_OK) return;
    PyObject* r = PyObject_CallFunction(bound_groups.check, "i", status);
    Py_XDECREF(r);
    if (r) PyErr_SetString(PyExc_RuntimeError, "a status other than 0 was not turned into an error");
    throw PythonError{};
}

template <class F>
PyObject* guarded_groups(F f)
{
    return guarded([&]() -> PyObject* {
        require(bound_groups.check != nullptr, "bind_groups() comes first");
        return f();
    });
}

[[noreturn]] void refuse_tensor(const char* what, const char* wanted)
{
    PyErr_Format(PyExc_ValueError, "%s: expected %s", what, wanted);
    throw PythonError{};
}

int dtype_code(at::ScalarType t) { return t == at::kFloat ? OGQ_FP32 : t == at::kBFloat16 ? OGQ_BF16 : t == at::kHalf ? OGQ_FP16 : -1; }

// A tensor of values: two dimensions on a GPU, consecutive values in a row.
struct Matrix {
    at::Tensor t;
    size_t rows = 0, cols = 0, stride = 0;
    uint32_t dtype = 0;
    Matrix() = default;
    Matrix(const at::Tensor& of, const char* what) : t(of)
    {
        const int code = dtype_code(of.scalar_type());
        if (!of.is_cuda() || of.dim() != 2 || code < 0 || (of.size(1) > 1 && of.stride(1) != 1))
            refuse_tensor(what, "a CUDA tensor of two dimensions in float32, bfloat16 or float16, with consecutive values in a row");
        dtype = static_cast<uint32_t>(code);
        rows = static_cast<size_t>(of.size(0)), cols = static_cast<size_t>(of.size(1));
        stride = rows > 1 ? static_cast<size_t>(of.stride(0)) : cols;
    }
    // As an input of the same shape, type and device.
    void like(const Matrix& other, const char* what) const
    {
        if (rows != other.rows || cols != other.cols || dtype != other.dtype || t.device() != other.t.device())
            refuse_tensor(what, "the shape, type and device of the first tensor");
    }
    const void* in() const { return t.const_data_ptr(); }
    void* out() const { return t.data_ptr(); }
};

// The caller's output, which has to fit, or a new one.
Matrix result(PyObject* given, size_t rows, size_t cols, at::ScalarType dtype, const at::Tensor& like, const char* what)
{
    if (given == Py_None)
        return Matrix(at::empty({static_cast<int64_t>(rows), static_cast<int64_t>(cols)}, at::TensorOptions().dtype(dtype).device(like.device())), what);
    Matrix m(tensor(given, what), what);
    if (m.rows != rows || m.cols != cols || m.t.scalar_type() != dtype || m.t.device() != like.device())
        refuse_tensor(what, "the result's shape, type and device");
    return m;
}

// Codes and exponents of a tensor [rows, cols].
struct Held {
    at::Tensor codes, exponents;
    size_t rows = 0;
    Held() = default;
    Held(PyObject* c, PyObject* e, size_t cols, const ogq_group_params_t& p, const char* what)
        : codes(tensor(c, what)), exponents(tensor(e, what))
    {
        rows = codes.dim() == 2 ? static_cast<size_t>(codes.size(0)) : 0;
        fits(cols, p, what);
    }
    // For results: the caller's, or new ones.
    Held(PyObject* c, PyObject* e, size_t n, size_t cols, const ogq_group_params_t& p, const at::Tensor& like, const char* what) : rows(n)
    {
        const auto made = [&](size_t width) {
            return at::empty({static_cast<int64_t>(n), static_cast<int64_t>(width)}, at::TensorOptions().dtype(at::kByte).device(like.device()));
        };
        codes = c == Py_None ? made(bound_groups.codes_bytes(1, cols, &p)) : tensor(c, what);
        exponents = e == Py_None ? made(bound_groups.exponents_count(1, cols, &p)) : tensor(e, what);
        fits(cols, p, what);
        on(like.device(), what);
    }
    void fits(size_t cols, const ogq_group_params_t& p, const char* what) const
    {
        const auto is = [&](const at::Tensor& t, size_t width) {
            return t.is_cuda() && t.scalar_type() == at::kByte && t.dim() == 2 && t.is_contiguous() && static_cast<size_t>(t.size(0)) == rows &&
                   static_cast<size_t>(t.size(1)) == width;
        };
        if (!is(codes, bound_groups.codes_bytes(1, cols, &p)) || !is(exponents, bound_groups.exponents_count(1, cols, &p)) ||
            codes.device() != exponents.device())
            refuse_tensor(what, "contiguous CUDA tensors of uint8, codes and exponents of as many rows and columns");
    }
    void on(const at::Device& device, const char* what) const
    {
        if (codes.device() != device) refuse_tensor(what, "tensors on one device");
    }
    const uint8_t* exponents_in() const { return static_cast<const uint8_t*>(exponents.const_data_ptr()); }
    uint8_t* exponents_out() const { return static_cast<uint8_t*>(exponents.data_ptr()); }
};

ogq_group_params_t group_params_of(PyObject* o)
{
    if (!PyObject_TypeCheck(o, bound_groups.params)) {
        PyErr_Format(PyExc_TypeError, "params: expected GroupParams, got %s", Py_TYPE(o)->tp_name);
        throw PythonError{};
    }
    Py_buffer view;
    if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) throw PythonError{};
    ogq_group_params_t p;
    const bool fits = view.len == static_cast<Py_ssize_t>(sizeof p);
    if (fits) std::memcpy(&p, view.buf, sizeof p);
    PyBuffer_Release(&view);
    require(fits, "params: not an ogq GroupParams structure");
    // sizes are asked for before the library checks the parameters
    if (bound_groups.codes_bytes(1, 1, &p) == 0)
        check_groups(p.group_size != 32 && p.group_size != 64 && p.group_size != 128 ? OGQ_ERR_GROUP_SIZE : OGQ_ERR_GROUP_BITS);
    return p;
}

// A whole number of at most `most`.
size_t number_of(PyObject* o, const char* what, size_t most)
{
    PyObject* n = PyNumber_Index(o);
    if (!n) throw PythonError{};
    const size_t v = PyLong_AsSize_t(n);
    Py_DECREF(n);
    if (v == static_cast<size_t>(-1) && PyErr_Occurred()) throw PythonError{};
    if (v > most) refuse_tensor(what, "a smaller number");
    return v;
}

constexpr size_t kMostColumns = static_cast<size_t>(1) << 31;  // (the library's own limit is below)

at::Tensor workspace_of(PyObject* given, size_t bytes, const at::Tensor& like)
{
    if (given == Py_None) {
        if (bytes == 0) return at::Tensor();
        return at::empty({static_cast<int64_t>(bytes)}, at::TensorOptions().dtype(at::kByte).device(like.device()));
    }
    const at::Tensor& t = tensor(given, "workspace");
    if (!t.is_cuda() || !t.is_contiguous() || t.device() != like.device()) refuse_tensor("workspace", "a contiguous CUDA tensor on the device");
    return t;
}

template <class F>
void call_library(const at::Tensor& on, F f)
{
    const c10::OptionalDeviceGuard guard(on.device());
    void* stream = stream_of(on);
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = f(stream);
    Py_END_ALLOW_THREADS
    check_groups(status);
}

// A tensor of the caller has been written: autograd, which may have kept it for a backward pass, is told so.
void written(PyObject* given, const at::Tensor& t)
{
    if (given != Py_None && !t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

PyObject* pack(std::initializer_list<at::Tensor> tensors)
{
    PyObject* all = PyTuple_New(static_cast<Py_ssize_t>(tensors.size()));
    if (!all) throw PythonError{};
    Py_ssize_t i = 0;
    for (const at::Tensor& t : tensors) PyTuple_SET_ITEM(all, i++, THPVariable_Wrap(t));
    return all;
}

// group_quantize(x, params, codes or None, exponents or None) -> (codes, exponents)
PyObject* group_quantize(PyObject*, PyObject* const* args, Py_ssize_t nargs)
{
    if (!argument_count(nargs, 4)) return nullptr;
    return guarded_groups([&]() -> PyObject* {
        const Matrix x(tensor(args[0], "x"), "x");
        const ogq_group_params_t p = group_params_of(args[1]);
        const Held to(args[2], args[3], x.rows, x.cols, p, x.t, "codes / exponents");
        const void* from = x.in();
        void* codes = to.codes.data_ptr();
        uint8_t* exponents = to.exponents_out();
        call_library(x.t, [&](void* st) { return bound_groups.quantize(from, x.stride, x.rows, x.cols, x.dtype, &p, codes, exponents, st); });
        written(args[2], to.codes), written(args[3], to.exponents);
        return pack({to.codes, to.exponents});
    });
}

// group_dequantize(codes, exponents, cols, params, dtype, out or None) -> out
PyObject* group_dequantize(PyObject*, PyObject* const* args, Py_ssize_t nargs)
{
    if (!argument_count(nargs, 6)) return nullptr;
    return guarded_groups([&]() -> PyObject* {
        const size_t cols = number_of(args[2], "cols", kMostColumns);
        const ogq_group_params_t p = group_params_of(args[3]);
        const Held x(args[0], args[1], cols, p, "codes / exponents");
        if (!THPDtype_Check(args[4]) || dtype_code(reinterpret_cast<THPDtype*>(args[4])->scalar_type) < 0)
            refuse_tensor("dtype", "torch.float32, torch.bfloat16 or torch.float16");
        const Matrix out = result(args[5], x.rows, cols, reinterpret_cast<THPDtype*>(args[4])->scalar_type, x.codes, "out");
        const void* codes = x.codes.const_data_ptr();
        void* to = out.out();
        call_library(out.t, [&](void* st) { return bound_groups.dequantize(codes, x.exponents_in(), x.rows, cols, &p, to, out.stride, out.dtype, st); });
        written(args[5], out.t);
        return THPVariable_Wrap(out.t);
    });
}

// activation_forward(x, activation, params, up or None, y or None, codes or None, exponents or None, up_codes or None, up_exponents or None)
//   -> (y, codes, exponents[, up_codes, up_exponents])
PyObject* activation_forward(PyObject*, PyObject* const* args, Py_ssize_t nargs)
{
    if (!argument_count(nargs, 9)) return nullptr;
    return guarded_groups([&]() -> PyObject* {
        const Matrix x(tensor(args[0], "x"), "x");
        const uint32_t act = static_cast<uint32_t>(number_of(args[1], "activation", 1000));
        const ogq_group_params_t p = group_params_of(args[2]);
        const bool gated = args[3] != Py_None;
        require(gated || (args[7] == Py_None && args[8] == Py_None), "up_codes / up_exponents: there is no up");
        Matrix up;
        if (gated) {
            up = Matrix(tensor(args[3], "up"), "up");
            up.like(x, "up");
        }
        const Matrix y = result(args[4], x.rows, x.cols, x.t.scalar_type(), x.t, "y");
        const Held to(args[5], args[6], x.rows, x.cols, p, x.t, "codes / exponents");
        Held up_to;
        if (gated) up_to = Held(args[7], args[8], x.rows, x.cols, p, x.t, "up_codes / up_exponents");
        const void *from = x.in(), *up_from = gated ? up.in() : nullptr;
        void *out = y.out(), *codes = to.codes.data_ptr(), *up_codes = gated ? up_to.codes.data_ptr() : nullptr;
        uint8_t *exponents = to.exponents_out(), *up_exponents = gated ? up_to.exponents_out() : nullptr;
        if (x.t.numel() != 0)  // (tensors without values have no addresses)
            call_library(x.t, [&](void* st) {
                return bound_groups.forward(from, x.stride, up_from, up.stride, x.rows, x.cols, x.dtype, act, &p, out, y.stride, codes, exponents, up_codes,
                                            up_exponents, st);
            });
        written(args[4], y.t), written(args[5], to.codes), written(args[6], to.exponents);
        if (gated) written(args[7], up_to.codes), written(args[8], up_to.exponents);
        return gated ? pack({y.t, to.codes, to.exponents, up_to.codes, up_to.exponents}) : pack({y.t, to.codes, to.exponents});
    });
}

// activation_backward(dy, activation, codes, exponents, params, up_codes or None, up_exponents or None, dx or None, dup or None)
//   -> dx, or (dx, dup)
PyObject* activation_backward(PyObject*, PyObject* const* args, Py_ssize_t nargs)
{
    if (!argument_count(nargs, 9)) return nullptr;
    return guarded_groups([&]() -> PyObject* {
        const Matrix dy(tensor(args[0], "dy"), "dy");
        const uint32_t act = static_cast<uint32_t>(number_of(args[1], "activation", 1000));
        const ogq_group_params_t p = group_params_of(args[4]);
        const Held x(args[2], args[3], dy.cols, p, "codes / exponents");
        require(x.rows == dy.rows, "codes / exponents: not as many rows as dy");
        x.on(dy.t.device(), "codes / exponents");
        require((args[5] == Py_None) == (args[6] == Py_None), "up_codes and up_exponents come together");
        const bool gated = args[5] != Py_None;
        require(gated || args[8] == Py_None, "dup: there are no up_codes");
        Held up;
        if (gated) {
            up = Held(args[5], args[6], dy.cols, p, "up_codes / up_exponents");
            require(up.rows == dy.rows, "up_codes / up_exponents: not as many rows as dy");
            up.on(dy.t.device(), "up_codes / up_exponents");
        }
        const Matrix dx = result(args[7], dy.rows, dy.cols, dy.t.scalar_type(), dy.t, "dx");
        Matrix dup;
        if (gated) dup = result(args[8], dy.rows, dy.cols, dy.t.scalar_type(), dy.t, "dup");
        const void *from = dy.in(), *codes = x.codes.const_data_ptr(), *up_codes = gated ? up.codes.const_data_ptr() : nullptr;
        const uint8_t* up_exponents = gated ? up.exponents_in() : nullptr;
        void *out = dx.out(), *up_out = gated ? dup.out() : nullptr;
        if (dy.t.numel() != 0)
            call_library(dy.t, [&](void* st) {
                return bound_groups.backward(from, dy.stride, codes, x.exponents_in(), up_codes, up_exponents, dy.rows, dy.cols, dy.dtype, act, &p, out,
                                             dx.stride, up_out, dup.stride, st);
            });
        written(args[7], dx.t);
        if (gated) written(args[8], dup.t);
        return gated ? pack({dx.t, dup.t}) : THPVariable_Wrap(dx.t);
    });
}

// weight_gradient(dy, codes, exponents, cols, params, dw or None, accumulate, workspace or None) -> dw
PyObject* weight_gradient(PyObject*, PyObject* const* args, Py_ssize_t nargs)
{
    if (!argument_count(nargs, 8)) return nullptr;
    return guarded_groups([&]() -> PyObject* {
        const Matrix dy(tensor(args[0], "dy"), "dy");
        const size_t cols = number_of(args[3], "cols", kMostColumns);
        const ogq_group_params_t p = group_params_of(args[4]);
        const Held x(args[1], args[2], cols, p, "codes / exponents");
        require(x.rows == dy.rows, "codes / exponents: not as many rows as dy");
        x.on(dy.t.device(), "codes / exponents");
        const int accumulate = PyObject_IsTrue(args[6]);
        if (accumulate < 0) throw PythonError{};
        require(!accumulate || args[5] != Py_None, "accumulate: there is no dw to add to");
        const Matrix dw = result(args[5], dy.cols, cols, at::kFloat, dy.t, "dw");
        const at::Tensor space = workspace_of(args[7], bound_groups.gradient_workspace(dy.rows, dy.cols, cols, dy.dtype, &p), dy.t);
        const void *from = dy.in(), *codes = x.codes.const_data_ptr();
        float* out = static_cast<float*>(dw.out());
        void* workspace = space.defined() ? space.data_ptr() : nullptr;
        const size_t bytes = space.defined() ? space.nbytes() : 0;
        call_library(dy.t, [&](void* st) {
            return bound_groups.gradient(from, dy.stride, dy.dtype, codes, x.exponents_in(), dy.rows, dy.cols, cols, &p, accumulate, out, dw.stride,
                                         workspace, bytes, st);
        });
        written(args[5], dw.t);
        return THPVariable_Wrap(dw.t);
    });
}

// group_matvec(codes, exponents, cols, params, x, y or None, workspace or None) -> y
PyObject* group_matvec(PyObject*, PyObject* const* args, Py_ssize_t nargs)
{
    if (!argument_count(nargs, 7)) return nullptr;
    return guarded_groups([&]() -> PyObject* {
        const size_t cols = number_of(args[2], "cols", kMostColumns);
        const ogq_group_params_t p = group_params_of(args[3]);
        const Held w(args[0], args[1], cols, p, "codes / exponents");
        const Matrix x(tensor(args[4], "x"), "x");
        require(x.cols == cols, "x: not as many columns as the weights");
        w.on(x.t.device(), "x");
        const Matrix y = result(args[5], x.rows, w.rows, x.t.scalar_type(), x.t, "y");
        const at::Tensor space = workspace_of(args[6], bound_groups.matvec_workspace(x.rows, w.rows, cols, x.dtype, &p), x.t);
        const void *from = x.in(), *codes = w.codes.const_data_ptr();
        void* out = y.out();
        void* workspace = space.defined() ? space.data_ptr() : nullptr;
        const size_t bytes = space.defined() ? space.nbytes() : 0;
        call_library(x.t, [&](void* st) {
            return bound_groups.matvec(codes, w.exponents_in(), w.rows, cols, &p, from, x.stride, x.rows, x.dtype, out, y.stride, workspace, bytes, st);
        });
        written(args[5], y.t);
        return THPVariable_Wrap(y.t);
    });
}

// bind_groups(addresses of the ten functions in the order of BoundGroups, check, GroupParams)
PyObject* bind_groups(PyObject*, PyObject* const* args, Py_ssize_t nargs)
{
    if (!argument_count(nargs, 12)) return nullptr;
    if (!PyType_Check(args[11])) {
        PyErr_SetString(PyExc_TypeError, "GroupParams: expected a class");
        return nullptr;
    }
    void* address[10];
    for (int i = 0; i < 10; ++i) {
        address[i] = PyLong_AsVoidPtr(args[i]);
        if (!address[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "address 0");
            return nullptr;
        }
    }
    BoundGroups& b = bound_groups;
    b.codes_bytes = reinterpret_cast<decltype(b.codes_bytes)>(address[0]);
    b.exponents_count = reinterpret_cast<decltype(b.exponents_count)>(address[1]);
    b.quantize = reinterpret_cast<decltype(b.quantize)>(address[2]);
    b.dequantize = reinterpret_cast<decltype(b.dequantize)>(address[3]);
    b.forward = reinterpret_cast<decltype(b.forward)>(address[4]);
    b.backward = reinterpret_cast<decltype(b.backward)>(address[5]);
    b.gradient_workspace = reinterpret_cast<decltype(b.gradient_workspace)>(address[6]);
    b.gradient = reinterpret_cast<decltype(b.gradient)>(address[7]);
    b.matvec_workspace = reinterpret_cast<decltype(b.matvec_workspace)>(address[8]);
    b.matvec = reinterpret_cast<decltype(b.matvec)>(address[9]);
    Py_INCREF(args[10]);
    Py_INCREF(args[11]);
    Py_XDECREF(b.check);
    Py_XDECREF(reinterpret_cast<PyObject*>(b.params));
    b.check = args[10];
    b.params = reinterpret_cast<PyTypeObject*>(args[11]);
    Py_RETURN_NONE;
}
