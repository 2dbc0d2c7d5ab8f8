// The calls of ogq_layers.h on tensors, for torch_marshal.cpp: checks, allocation of what the caller left out, the call.  Part of that file, behind
// torch_marshal_groups.h, whose helpers it uses: included once, inside its namespace.

// What bind_layers() was given.
struct BoundLayers {
    decltype(&ogq_layer_norm_forward) norm_forward = nullptr;
    decltype(&ogq_layer_norm_backward_workspace) norm_workspace = nullptr;
    decltype(&ogq_layer_norm_backward) norm_backward = nullptr;
    decltype(&ogq_linear_workspace) linear_workspace = nullptr;
    decltype(&ogq_linear) linear = nullptr;
    decltype(&ogq_linear_backward_workspace) linear_backward_workspace = nullptr;
    decltype(&ogq_linear_backward) linear_backward = nullptr;
    decltype(&ogq_embedding_forward) embedding_forward = nullptr;
    decltype(&ogq_embedding_gradient_workspace) embedding_workspace = nullptr;
    decltype(&ogq_embedding_gradient) embedding_gradient = nullptr;
    decltype(&ogq_distill_workspace) distill_workspace = nullptr;
    decltype(&ogq_distill_loss) distill_loss = nullptr;
    decltype(&ogq_distill_gradient) distill_gradient = nullptr;
    PyObject* check = nullptr;  // callable: raises OgqError for a status other than 0
} bound_layers;

void check_layers(int status)
{
    if (status == OGQ_OK) return;
    PyObject* r = PyObject_CallFunction(bound_layers.check, "i", status);
    Py_XDECREF(r);
    if (r) PyErr_SetString(PyExc_RuntimeError, "a status other than 0 was not turned into an error");
    throw PythonError{};
}

template <class F>
PyObject* guarded_layers(F f)
{
    return guarded([&]() -> PyObject* {
        require(bound_layers.check != nullptr, "bind_layers() comes first");
        return f();
    });
}

template <class F>
void call_layers(const at::Tensor& on, F f)
{
    const c10::OptionalDeviceGuard guard(on.device());
    void* stream = stream_of(on);
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = f(stream);
    Py_END_ALLOW_THREADS
    check_layers(status);
}

// A contiguous vector of fp32 on the device, or none.
struct Vector {
    at::Tensor t;
    Vector() = default;
    Vector(PyObject* given, size_t n, const at::Tensor& like, const char* what)
    {
        if (given == Py_None) return;
        t = tensor(given, what);
        if (!t.is_cuda() || t.scalar_type() != at::kFloat || t.dim() != 1 || !t.is_contiguous() || static_cast<size_t>(t.numel()) != n || t.device() != like.device())
            refuse_tensor(what, "a contiguous CUDA vector of float32, of the right length, on the device");
    }
    const float* in() const { return t.defined() ? static_cast<const float*>(t.const_data_ptr()) : nullptr; }
    float* out() const { return t.defined() ? static_cast<float*>(t.data_ptr()) : nullptr; }
};

at::Tensor made_vector(size_t n, const at::Tensor& like)
{
    return at::empty({static_cast<int64_t>(n)}, at::TensorOptions().dtype(at::kFloat).device(like.device()));
}

// The caller's vector, which has to fit, or a new one.
Vector vector_result(PyObject* given, size_t n, const at::Tensor& like, const char* what)
{
    Vector v(given, n, like, what);
    if (!v.t.defined()) v.t = made_vector(n, like);
    return v;
}

float float_of(PyObject* o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw PythonError{};
    return static_cast<float>(v);
}

uint32_t activation_of(PyObject* o) { return o == Py_None ? OGQ_IDENTITY : static_cast<uint32_t>(number_of(o, "activation", 1000)); }

// int32 or int64, contiguous, of `dims` dimensions, on a GPU.
uint32_t integer_of(const at::Tensor& t, int64_t dims, const char* what)
{
    const bool narrow = t.scalar_type() == at::kInt, wide = t.scalar_type() == at::kLong;
    if (!t.is_cuda() || !(narrow || wide) || t.dim() != dims || !t.is_contiguous()) refuse_tensor(what, "a contiguous CUDA tensor of int32 or int64 with as many dimensions as it should have");
    return narrow ? OGQ_INT32 : OGQ_INT64;
}

// layer_norm_forward(x, weight or None, bias or None, eps, y or None, mean or None, rstd or None) -> (y, mean, rstd)
PyObject* layer_norm_forward(PyObject*, PyObject* const* args, Py_ssize_t nargs)
{
    if (!argument_count(nargs, 7)) return nullptr;
    return guarded_layers([&]() -> PyObject* {
        const Matrix x(tensor(args[0], "x"), "x");
        const Vector weight(args[1], x.cols, x.t, "weight"), bias(args[2], x.cols, x.t, "bias");
        const float eps = float_of(args[3]);
        const Matrix y = result(args[4], x.rows, x.cols, x.t.scalar_type(), x.t, "y");
        const Vector mean = vector_result(args[5], x.rows, x.t, "mean"), rstd = vector_result(args[6], x.rows, x.t, "rstd");
        const void* from = x.in();
        void* to = y.out();
        float *to_mean = mean.out(), *to_rstd = rstd.out();
        call_layers(x.t, [&](void* st) {
            return bound_layers.norm_forward(from, x.stride, x.rows, x.cols, x.dtype, weight.in(), bias.in(), eps, to, y.stride, to_mean, to_rstd, st);
        });
        written(args[4], y.t), written(args[5], mean.t), written(args[6], rstd.t);
        return pack({y.t, mean.t, rstd.t});
    });
}

// layer_norm_backward(dy, x, mean, rstd, weight or None, dx or None, dweight or None, dbias or None, accumulate, workspace or None) -> dx, or (dx, dweight, dbias) where there is a weight
PyObject* layer_norm_backward(PyObject*, PyObject* const* args, Py_ssize_t nargs)
{
    if (!argument_count(nargs, 10)) return nullptr;
    return guarded_layers([&]() -> PyObject* {
        const Matrix dy(tensor(args[0], "dy"), "dy"), x(tensor(args[1], "x"), "x");
        x.like(dy, "x");
        require(args[2] != Py_None && args[3] != Py_None, "mean and rstd are those of the forward pass");
        const Vector mean(args[2], dy.rows, dy.t, "mean"), rstd(args[3], dy.rows, dy.t, "rstd"), weight(args[4], dy.cols, dy.t, "weight");
        const int accumulate = PyObject_IsTrue(args[8]);
        if (accumulate < 0) throw PythonError{};
        const bool sums = args[4] != Py_None;
        require(sums || (args[6] == Py_None && args[7] == Py_None && !accumulate), "dweight / dbias: there is no weight");
        require(!accumulate || (args[6] != Py_None && args[7] != Py_None), "accumulate: there are no dweight and dbias to add to");
        const Matrix dx = result(args[5], dy.rows, dy.cols, dy.t.scalar_type(), dy.t, "dx");
        Vector dweight, dbias;
        if (sums) dweight = vector_result(args[6], dy.cols, dy.t, "dweight"), dbias = vector_result(args[7], dy.cols, dy.t, "dbias");
        const at::Tensor space = workspace_of(args[9], sums ? bound_layers.norm_workspace(dy.rows, dy.cols, dy.dtype) : 0, dy.t);
        void* workspace = space.defined() ? space.data_ptr() : nullptr;
        const size_t bytes = space.defined() ? space.nbytes() : 0;
        const void *from = dy.in(), *from_x = x.in();
        void* to = dx.out();
        float *to_weight = dweight.out(), *to_bias = dbias.out();
        call_layers(dy.t, [&](void* st) {
            return bound_layers.norm_backward(from, dy.stride, from_x, x.stride, dy.rows, dy.cols, dy.dtype, weight.in(), mean.in(), rstd.in(), to, dx.stride, to_weight, to_bias,
                                              accumulate, workspace, bytes, st);
        });
        written(args[5], dx.t);
        if (!sums) return THPVariable_Wrap(dx.t);
        written(args[6], dweight.t), written(args[7], dbias.t);
        return pack({dx.t, dweight.t, dbias.t});
    });
}

// linear(x, weight, bias or None, activation or None, residual or None, transposed, keep, y or None, before or None, workspace or None) -> y, or (y, before)
PyObject* linear(PyObject*, PyObject* const* args, Py_ssize_t nargs)
{
    if (!argument_count(nargs, 10)) return nullptr;
    return guarded_layers([&]() -> PyObject* {
        const Matrix x(tensor(args[0], "x"), "x"), w(tensor(args[1], "weight"), "weight");
        const int transposed = PyObject_IsTrue(args[5]), keep = PyObject_IsTrue(args[6]);
        if (transposed < 0 || keep < 0) throw PythonError{};
        const size_t outs = transposed ? w.cols : w.rows;
        if ((transposed ? w.rows : w.cols) != x.cols || w.dtype != x.dtype || w.t.device() != x.t.device())
            refuse_tensor("weight", "a tensor of x's type and device, [outs, cols], or [cols, outs] where transposed");
        const Vector bias(args[2], outs, x.t, "bias");
        const uint32_t act = activation_of(args[3]);
        const Matrix y = result(args[7], x.rows, outs, x.t.scalar_type(), x.t, "y");
        Matrix residual, before;
        if (args[4] != Py_None) {
            residual = Matrix(tensor(args[4], "residual"), "residual");
            residual.like(y, "residual");
        }
        const bool kept = keep || args[8] != Py_None;
        if (kept) before = result(args[8], x.rows, outs, x.t.scalar_type(), x.t, "before");
        const at::Tensor space = workspace_of(args[9], bound_layers.linear_workspace(x.rows, outs, x.cols, x.dtype, transposed), x.t);
        void* workspace = space.defined() ? space.data_ptr() : nullptr;
        const size_t bytes = space.defined() ? space.nbytes() : 0;
        const void *from = x.in(), *weight = w.in(), *add = residual.t.defined() ? residual.in() : nullptr;
        void *to = y.out(), *to_before = kept ? before.out() : nullptr;
        if (y.t.numel() != 0)  // (tensors without values have no addresses)
            call_layers(x.t, [&](void* st) {
                return bound_layers.linear(from, x.stride, weight, w.stride, transposed, x.rows, outs, x.cols, x.dtype, bias.in(), act, add, residual.stride, to, y.stride, to_before,
                                           before.stride, workspace, bytes, st);
            });
        written(args[7], y.t);
        if (!kept) return THPVariable_Wrap(y.t);
        written(args[8], before.t);
        return pack({y.t, before.t});
    });
}

// linear_backward(dy, activation or None, before or None, dz or None, dbias or None, accumulate, workspace or None) -> (dz, dbias)
PyObject* linear_backward(PyObject*, PyObject* const* args, Py_ssize_t nargs)
{
    if (!argument_count(nargs, 7)) return nullptr;
    return guarded_layers([&]() -> PyObject* {
        const Matrix dy(tensor(args[0], "dy"), "dy");
        const uint32_t act = activation_of(args[1]);
        const bool identity = act == OGQ_IDENTITY;
        require(identity == (args[2] == Py_None), "before: what went into the activation, where there is one");
        require(!identity || args[3] == Py_None, "dz: dy itself where there is no activation");
        const int accumulate = PyObject_IsTrue(args[5]);
        if (accumulate < 0) throw PythonError{};
        require(!accumulate || args[4] != Py_None, "accumulate: there is no dbias to add to");
        Matrix before, dz;
        if (!identity) {
            before = Matrix(tensor(args[2], "before"), "before");
            before.like(dy, "before");
            dz = result(args[3], dy.rows, dy.cols, dy.t.scalar_type(), dy.t, "dz");
        }
        const Vector dbias = vector_result(args[4], dy.cols, dy.t, "dbias");
        const at::Tensor space = workspace_of(args[6], bound_layers.linear_backward_workspace(dy.rows, dy.cols, dy.dtype), dy.t);
        void* workspace = space.defined() ? space.data_ptr() : nullptr;
        const size_t bytes = space.defined() ? space.nbytes() : 0;
        const void *from = dy.in(), *from_before = identity ? nullptr : before.in();
        void* to = identity ? nullptr : dz.out();
        float* to_bias = dbias.out();
        call_layers(dy.t, [&](void* st) {
            return bound_layers.linear_backward(from, dy.stride, dy.rows, dy.cols, dy.dtype, act, from_before, before.stride, to, dz.stride, to_bias, accumulate, workspace, bytes, st);
        });
        if (!identity) written(args[3], dz.t);
        written(args[4], dbias.t);
        return pack({identity ? dy.t : dz.t, dbias.t});
    });
}

// embedding_forward(tokens, table, scale, y or None) -> y
PyObject* embedding_forward(PyObject*, PyObject* const* args, Py_ssize_t nargs)
{
    if (!argument_count(nargs, 4)) return nullptr;
    return guarded_layers([&]() -> PyObject* {
        const at::Tensor& tokens = tensor(args[0], "tokens");
        const uint32_t integer = integer_of(tokens, 1, "tokens");
        const Matrix table(tensor(args[1], "table"), "table");
        require(tokens.device() == table.t.device(), "tokens: not on the table's device");
        const float scale = float_of(args[2]);
        const size_t number = static_cast<size_t>(tokens.numel());
        const Matrix y = result(args[3], number, table.cols, table.t.scalar_type(), table.t, "y");
        const void *from = tokens.const_data_ptr(), *rows = table.in();
        void* to = y.out();
        call_layers(table.t, [&](void* st) {
            return bound_layers.embedding_forward(from, integer, number, rows, table.stride, table.rows, table.cols, table.dtype, scale, to, y.stride, st);
        });
        written(args[3], y.t);
        return THPVariable_Wrap(y.t);
    });
}

// embedding_gradient(tokens, dy, vocab, scale, dtable or None, accumulate, workspace or None) -> dtable
PyObject* embedding_gradient(PyObject*, PyObject* const* args, Py_ssize_t nargs)
{
    if (!argument_count(nargs, 7)) return nullptr;
    return guarded_layers([&]() -> PyObject* {
        const at::Tensor& tokens = tensor(args[0], "tokens");
        const uint32_t integer = integer_of(tokens, 1, "tokens");
        const Matrix dy(tensor(args[1], "dy"), "dy");
        require(tokens.device() == dy.t.device(), "tokens: not on dy's device");
        require(static_cast<size_t>(tokens.numel()) == dy.rows, "tokens: not as many as dy has rows");
        const size_t vocab = number_of(args[2], "vocab", kMostColumns);
        const float scale = float_of(args[3]);
        const int accumulate = PyObject_IsTrue(args[5]);
        if (accumulate < 0) throw PythonError{};
        require(!accumulate || args[4] != Py_None, "accumulate: there is no dtable to add to");
        const Matrix dtable = result(args[4], vocab, dy.cols, at::kFloat, dy.t, "dtable");
        const at::Tensor space = workspace_of(args[6], bound_layers.embedding_workspace(dy.rows, vocab, dy.cols), dy.t);
        void* workspace = space.defined() ? space.data_ptr() : nullptr;
        const size_t bytes = space.defined() ? space.nbytes() : 0;
        const void *from = tokens.const_data_ptr(), *rows = dy.in();
        float* to = static_cast<float*>(dtable.out());
        call_layers(dy.t, [&](void* st) {
            return bound_layers.embedding_gradient(from, integer, dy.rows, rows, dy.stride, vocab, dy.cols, dy.dtype, scale, accumulate, to, dtable.stride, workspace, bytes, st);
        });
        written(args[4], dtable.t);
        return THPVariable_Wrap(dtable.t);
    });
}

// What both calls of a divergence take: logits, places, values, temperature, row_weight or None.
struct Divergence {
    Matrix logits;
    at::Tensor places, values;
    uint32_t integer;
    size_t top;
    float temperature;
    Vector row_weight;
    explicit Divergence(PyObject* const* args) : logits(tensor(args[0], "logits"), "logits"), places(tensor(args[1], "places")), values(tensor(args[2], "values"))
    {
        integer = integer_of(places, 2, "places");
        if (!values.is_cuda() || values.scalar_type() != at::kFloat || values.dim() != 2 || !values.is_contiguous()) refuse_tensor("values", "a contiguous CUDA tensor of float32 of two dimensions");
        require(static_cast<size_t>(places.size(0)) == logits.rows && places.sizes() == values.sizes(), "places / values: a row to each row of logits, as many of the one as of the other");
        require(places.device() == logits.t.device() && values.device() == logits.t.device(), "places / values: not on the logits' device");
        top = static_cast<size_t>(places.size(1));
        temperature = float_of(args[3]);
        row_weight = Vector(args[4], logits.rows, logits.t, "row_weight");
    }
    at::Tensor workspace(PyObject* given) const { return workspace_of(given, bound_layers.distill_workspace(logits.rows, logits.cols, logits.dtype, top), logits.t); }
    const float* values_in() const { return static_cast<const float*>(values.const_data_ptr()); }
};

// distill_loss(logits, places, values, temperature, row_weight or None, loss or None, workspace or None) -> loss
PyObject* distill_loss(PyObject*, PyObject* const* args, Py_ssize_t nargs)
{
    if (!argument_count(nargs, 7)) return nullptr;
    return guarded_layers([&]() -> PyObject* {
        const Divergence d(args);
        const Vector loss = vector_result(args[5], d.logits.rows, d.logits.t, "loss");
        const at::Tensor space = d.workspace(args[6]);
        void* workspace = space.defined() ? space.data_ptr() : nullptr;
        const size_t bytes = space.defined() ? space.nbytes() : 0;
        const void *from = d.logits.in(), *places = d.places.const_data_ptr();
        float* to = loss.out();
        call_layers(d.logits.t, [&](void* st) {
            return bound_layers.distill_loss(from, d.logits.stride, d.logits.rows, d.logits.cols, d.logits.dtype, places, d.integer, d.values_in(), d.top, d.temperature,
                                             d.row_weight.in(), to, workspace, bytes, st);
        });
        written(args[5], loss.t);
        return THPVariable_Wrap(loss.t);
    });
}

// distill_gradient(logits, places, values, temperature, row_weight or None, dlogits or None, loss or None, workspace or None) -> (loss, dlogits)
PyObject* distill_gradient(PyObject*, PyObject* const* args, Py_ssize_t nargs)
{
    if (!argument_count(nargs, 8)) return nullptr;
    return guarded_layers([&]() -> PyObject* {
        const Divergence d(args);
        const Matrix dlogits = result(args[5], d.logits.rows, d.logits.cols, d.logits.t.scalar_type(), d.logits.t, "dlogits");
        const Vector loss = vector_result(args[6], d.logits.rows, d.logits.t, "loss");
        const at::Tensor space = d.workspace(args[7]);
        void* workspace = space.defined() ? space.data_ptr() : nullptr;
        const size_t bytes = space.defined() ? space.nbytes() : 0;
        const void *from = d.logits.in(), *places = d.places.const_data_ptr();
        void* to = dlogits.out();
        float* to_loss = loss.out();
        call_layers(d.logits.t, [&](void* st) {
            return bound_layers.distill_gradient(from, d.logits.stride, d.logits.rows, d.logits.cols, d.logits.dtype, places, d.integer, d.values_in(), d.top, d.temperature,
                                                 d.row_weight.in(), to_loss, to, dlogits.stride, workspace, bytes, st);
        });
        written(args[5], dlogits.t), written(args[6], loss.t);
        return pack({loss.t, dlogits.t});
    });
}

// bind_layers(addresses of the thirteen functions in the order of BoundLayers, check)
PyObject* bind_layers(PyObject*, PyObject* const* args, Py_ssize_t nargs)
{
    if (!argument_count(nargs, 14)) return nullptr;
    void* address[13];
    for (int i = 0; i < 13; ++i) {
        address[i] = PyLong_AsVoidPtr(args[i]);
        if (!address[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "address 0");
            return nullptr;
        }
    }
    BoundLayers& b = bound_layers;
    b.norm_forward = reinterpret_cast<decltype(b.norm_forward)>(address[0]);
    b.norm_workspace = reinterpret_cast<decltype(b.norm_workspace)>(address[1]);
    b.norm_backward = reinterpret_cast<decltype(b.norm_backward)>(address[2]);
    b.linear_workspace = reinterpret_cast<decltype(b.linear_workspace)>(address[3]);
    b.linear = reinterpret_cast<decltype(b.linear)>(address[4]);
    b.linear_backward_workspace = reinterpret_cast<decltype(b.linear_backward_workspace)>(address[5]);
    b.linear_backward = reinterpret_cast<decltype(b.linear_backward)>(address[6]);
    b.embedding_forward = reinterpret_cast<decltype(b.embedding_forward)>(address[7]);
    b.embedding_workspace = reinterpret_cast<decltype(b.embedding_workspace)>(address[8]);
    b.embedding_gradient = reinterpret_cast<decltype(b.embedding_gradient)>(address[9]);
    b.distill_workspace = reinterpret_cast<decltype(b.distill_workspace)>(address[10]);
    b.distill_loss = reinterpret_cast<decltype(b.distill_loss)>(address[11]);
    b.distill_gradient = reinterpret_cast<decltype(b.distill_gradient)>(address[12]);
    Py_INCREF(args[13]);
    Py_XDECREF(b.check);
    b.check = args[13];
    Py_RETURN_NONE;
}
