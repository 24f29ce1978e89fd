// Argument marshalling of the block operators, for the Python binding: checks
// every tensor (type, dtype, shape, row layout, device), fills the call's
// argument struct, takes the workspace from torch's caching allocator on the
// call's stream, and makes the library call.  A wrong argument raises TypeError
// or ValueError naming it, before anything is enqueued; a status of the library
// is returned.  One C call, because from Python each check costs about 0.7 us
// per tensor, more than the smallest kernels run.
//
// The workspace goes back to the allocator as soon as the call is enqueued: the
// allocator hands a block of one stream only to later work of that stream.

#include "marshal_call.h"

#include "fsdp_block.h"

namespace {

// The gate's rows: a vector [hidden] or a matrix [rows, hidden].
const void* gate_of(const at::Tensor* t, const char* name, int64_t hidden, int64_t* rows) {
    if (!t) return nullptr;
    if (t->dim() < 1 || t->dim() > 2 || t->size(-1) != hidden)
        raise(PyExc_ValueError, "%s must have the shape (%lld,) or (rows, %lld)", name, (long long)hidden, (long long)hidden);
    if (!t->is_contiguous()) raise(PyExc_ValueError, "%s must be contiguous", name);
    *rows = t->dim() == 1 ? 1 : t->size(0);
    if (*rows == 0) raise(PyExc_ValueError, "%s has no rows", name);
    return t->data_ptr();
}

// The stream and the weights have the block's type or are fp32.
void block_types(fsdp_dtype stream, fsdp_dtype block, fsdp_dtype weight) {
    if (stream != block && stream != FSDP_DTYPE_F32)
        raise(PyExc_TypeError, "the residual stream must be of the block's dtype %s or f32", name_of(block));
    if (weight != block && weight != FSDP_DTYPE_F32)
        raise(PyExc_TypeError, "the weights must be of the block's dtype %s or f32", name_of(block));
}

// norm(x, branch, post_weight, gate, pre_weight, y, h, eps, residual_scale, branch_scale, stream)
PyObject* norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return entry(n, 11, [&]() -> fsdp_status {
        Call c;
        const auto *x = c.tensor(a[0], "x", true), *branch = c.tensor(a[1], "branch", false),
                   *post = c.tensor(a[2], "post_weight", false), *gate = c.tensor(a[3], "gate", false),
                   *pre = c.tensor(a[4], "pre_weight", false), *y = c.tensor(a[5], "y", false), *h = c.tensor(a[6], "h", false);
        two_dims(*x, "x");
        fsdp_norm_args k{};
        k.tokens = x->size(0);
        k.hidden = x->size(1);
        k.stream_dtype = c.dtype(*x, "x");
        k.block_dtype = branch ? c.dtype(*branch, "branch") : h ? c.dtype(*h, "h") : k.stream_dtype;
        k.weight_dtype = post ? c.dtype(*post, "post_weight") : pre ? c.dtype(*pre, "pre_weight") : k.block_dtype;
        if (pre) c.dtype(*pre, "pre_weight", k.weight_dtype);
        if (gate) c.dtype(*gate, "gate", k.block_dtype);
        if (y) c.dtype(*y, "y", k.stream_dtype);
        if (h) c.dtype(*h, "h", k.block_dtype);
        block_types(k.stream_dtype, k.block_dtype, k.weight_dtype);
        if (!y && !h) raise(PyExc_ValueError, "neither y nor h is wanted");
        if (h && !pre) raise(PyExc_ValueError, "h needs pre_weight");
        k.x = c.matrix(x, "x", k.tokens, k.hidden, &k.x_stride);
        k.branch = c.matrix(branch, "branch", k.tokens, k.hidden, &k.branch_stride);
        k.post_weight = c.vector(post, "post_weight", k.hidden);
        k.pre_weight = c.vector(pre, "pre_weight", k.hidden);
        k.gate = gate_of(gate, "gate", k.hidden, &k.gate_rows);
        k.y = c.matrix(y, "y", k.tokens, k.hidden, &k.y_stride);
        k.h = c.matrix(h, "h", k.tokens, k.hidden, &k.h_stride);
        k.eps = float(number(a[7], "eps"));
        k.residual_scale = float(number(a[8], "residual_scale"));
        k.branch_scale = float(number(a[9], "branch_scale"));
        const hipStream_t s = c.stream(a[10]);
        if (k.tokens == 0) return FSDP_OK;
        const c10::hip::HIPGuard guard(c10::DeviceIndex(c.device()));
        return fsdp_block_norm(&k, s);
    });
}

// norm_grad(y, dy, dh, branch, post_weight, gate, pre_weight, dx, dbranch, dpre_weight, dpost_weight, dgate, eps,
//           residual_scale, branch_scale, stream)
PyObject* norm_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return entry(n, 16, [&]() -> fsdp_status {
        Call c;
        const auto *y = c.tensor(a[0], "y", true), *dy = c.tensor(a[1], "dy", false), *dh = c.tensor(a[2], "dh", false),
                   *branch = c.tensor(a[3], "branch", false), *post = c.tensor(a[4], "post_weight", false),
                   *gate = c.tensor(a[5], "gate", false), *pre = c.tensor(a[6], "pre_weight", false),
                   *dx = c.tensor(a[7], "dx", false), *dbranch = c.tensor(a[8], "dbranch", false),
                   *dpre = c.tensor(a[9], "dpre_weight", false), *dpost = c.tensor(a[10], "dpost_weight", false),
                   *dgate = c.tensor(a[11], "dgate", false);
        two_dims(*y, "y");
        fsdp_norm_grad_args k{};
        k.tokens = y->size(0);
        k.hidden = y->size(1);
        k.stream_dtype = c.dtype(*y, "y");
        k.block_dtype = branch ? c.dtype(*branch, "branch") : dh ? c.dtype(*dh, "dh") : k.stream_dtype;
        k.weight_dtype = post ? c.dtype(*post, "post_weight") : pre ? c.dtype(*pre, "pre_weight") : k.block_dtype;
        if (dh) c.dtype(*dh, "dh", k.block_dtype);
        if (pre) c.dtype(*pre, "pre_weight", k.weight_dtype);
        if (gate) c.dtype(*gate, "gate", k.block_dtype);
        if (dy) c.dtype(*dy, "dy", k.stream_dtype);
        if (dx) c.dtype(*dx, "dx", k.stream_dtype);
        if (dbranch) c.dtype(*dbranch, "dbranch", k.block_dtype);
        if (dpre) c.dtype(*dpre, "dpre_weight", k.weight_dtype);
        if (dpost) c.dtype(*dpost, "dpost_weight", k.weight_dtype);
        if (dgate) c.dtype(*dgate, "dgate", k.block_dtype);
        block_types(k.stream_dtype, k.block_dtype, k.weight_dtype);
        if (!dh != !pre) raise(PyExc_ValueError, "dh and pre_weight go together");
        if (dbranch && !branch) raise(PyExc_ValueError, "dbranch needs a branch");
        if (dgate && (!gate || dgate->sizes() != gate->sizes()))
            raise(PyExc_ValueError, "dgate must have the gate's shape");
        k.y = c.matrix(y, "y", k.tokens, k.hidden, &k.y_stride);
        k.dy = c.matrix(dy, "dy", k.tokens, k.hidden, &k.dy_stride);
        k.dh = c.matrix(dh, "dh", k.tokens, k.hidden, &k.dh_stride);
        k.branch = c.matrix(branch, "branch", k.tokens, k.hidden, &k.branch_stride);
        k.post_weight = c.vector(post, "post_weight", k.hidden);
        k.pre_weight = c.vector(pre, "pre_weight", k.hidden);
        k.gate = gate_of(gate, "gate", k.hidden, &k.gate_rows);
        k.dx = c.matrix(dx, "dx", k.tokens, k.hidden, &k.dx_stride);
        k.dbranch = c.matrix(dbranch, "dbranch", k.tokens, k.hidden, &k.dbranch_stride);
        k.dpre_weight = c.vector(dpre, "dpre_weight", k.hidden);
        k.dpost_weight = c.vector(dpost, "dpost_weight", k.hidden);
        int64_t rows;
        k.dgate = const_cast<void*>(gate_of(dgate, "dgate", k.hidden, &rows));
        // Without tokens the matrices have no memory; the library takes a branch for given where its weights are.
        if (k.tokens == 0 && branch) k.branch = post ? k.post_weight : k.gate;
        k.eps = float(number(a[12], "eps"));
        k.residual_scale = float(number(a[13], "residual_scale"));
        k.branch_scale = float(number(a[14], "branch_scale"));
        const hipStream_t s = c.stream(a[15]);
        const c10::hip::HIPGuard guard(c10::DeviceIndex(c.device()));
        int64_t bytes = 0;
        const fsdp_status st = fsdp_block_norm_grad_workspace(&k, &bytes);
        if (st != FSDP_OK) return st;
        const Workspace w(bytes, s);
        return fsdp_block_norm_grad(&k, w.data(), w.bytes(), s);
    });
}

// linear(x, weight, out, bias, activation, times, residual, pre, stream)
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return entry(n, 9, [&]() -> fsdp_status {
        Call c;
        const auto *x = c.tensor(a[0], "x", true), *weight = c.tensor(a[1], "weight", true), *out = c.tensor(a[2], "out", true),
                   *bias = c.tensor(a[3], "bias", false), *times = c.tensor(a[5], "times", false),
                   *residual = c.tensor(a[6], "residual", false), *pre = c.tensor(a[7], "pre", false);
        two_dims(*x, "x");
        two_dims(*weight, "weight");
        fsdp_linear_args k{};
        k.m = x->size(0);
        k.n = weight->size(0);
        k.k = x->size(1);
        k.dtype = c.dtype(*x, "x");
        c.dtype(*weight, "weight", k.dtype);
        c.dtype(*out, "out", k.dtype);
        if (bias) c.dtype(*bias, "bias", k.dtype);
        if (times) c.dtype(*times, "times", k.dtype);
        if (residual) c.dtype(*residual, "residual", k.dtype);
        if (pre) c.dtype(*pre, "pre", k.dtype);
        k.activation = activation_of(a[4]);
        k.x = c.matrix(x, "x", k.m, k.k, &k.x_stride);
        k.weight = c.matrix(weight, "weight", k.n, k.k, &k.weight_stride);
        k.bias = c.vector(bias, "bias", k.n);
        k.times = c.matrix(times, "times", k.m, k.n, &k.times_stride);
        k.residual = c.matrix(residual, "residual", k.m, k.n, &k.residual_stride);
        k.pre = c.matrix(pre, "pre", k.m, k.n, &k.pre_stride);
        k.out = c.matrix(out, "out", k.m, k.n, &k.out_stride);
        const hipStream_t s = c.stream(a[8]);
        const c10::hip::HIPGuard guard(c10::DeviceIndex(c.device()));
        int64_t bytes = 0;
        const fsdp_status st = fsdp_block_linear_workspace(&k, &bytes);
        if (st != FSDP_OK) return st;
        const Workspace w(bytes, s);
        return fsdp_block_linear(&k, w.data(), w.bytes(), s);
    });
}

// linear_grad(dout, x, weight, activation, pre, times, dx, dweight, dbias, dtimes, stream)
PyObject* linear_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return entry(n, 11, [&]() -> fsdp_status {
        Call c;
        const auto *dout = c.tensor(a[0], "dout", true), *x = c.tensor(a[1], "x", true), *weight = c.tensor(a[2], "weight", true),
                   *pre = c.tensor(a[4], "pre", false), *times = c.tensor(a[5], "times", false),
                   *dx = c.tensor(a[6], "dx", false), *dweight = c.tensor(a[7], "dweight", false),
                   *dbias = c.tensor(a[8], "dbias", false), *dtimes = c.tensor(a[9], "dtimes", false);
        two_dims(*x, "x");
        two_dims(*weight, "weight");
        fsdp_linear_grad_args k{};
        k.m = x->size(0);
        k.n = weight->size(0);
        k.k = x->size(1);
        k.dtype = c.dtype(*x, "x");
        c.dtype(*dout, "dout", k.dtype);
        c.dtype(*weight, "weight", k.dtype);
        if (pre) c.dtype(*pre, "pre", k.dtype);
        if (times) c.dtype(*times, "times", k.dtype);
        if (dx) c.dtype(*dx, "dx", k.dtype);
        if (dweight) c.dtype(*dweight, "dweight", k.dtype);
        if (dbias) c.dtype(*dbias, "dbias", k.dtype);
        if (dtimes) c.dtype(*dtimes, "dtimes", k.dtype);
        if (dtimes && !times) raise(PyExc_ValueError, "dtimes needs times");
        k.activation = activation_of(a[3]);
        k.dout = c.matrix(dout, "dout", k.m, k.n, &k.dout_stride);
        k.x = c.matrix(x, "x", k.m, k.k, &k.x_stride);
        k.weight = c.matrix(weight, "weight", k.n, k.k, &k.weight_stride);
        k.pre = c.matrix(pre, "pre", k.m, k.n, &k.pre_stride);
        k.times = c.matrix(times, "times", k.m, k.n, &k.times_stride);
        k.dx = c.matrix(dx, "dx", k.m, k.k, &k.dx_stride);
        k.dweight = c.matrix(dweight, "dweight", k.n, k.k, &k.dweight_stride);
        k.dbias = c.vector(dbias, "dbias", k.n);
        k.dtimes = c.matrix(dtimes, "dtimes", k.m, k.n, &k.dtimes_stride);
        const hipStream_t s = c.stream(a[10]);
        const c10::hip::HIPGuard guard(c10::DeviceIndex(c.device()));
        int64_t bytes = 0;
        const fsdp_status st = fsdp_block_linear_grad_workspace(&k, &bytes);
        if (st != FSDP_OK) return st;
        const Workspace w(bytes, s);
        return fsdp_block_linear_grad(&k, w.data(), w.bytes(), s);
    });
}

// distill(backward, logits, teacher, ids, teacher_lse, dloss, loss, lse, dlogits, temperature, stream)
PyObject* distill(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return entry(n, 11, [&]() -> fsdp_status {
        Call c;
        const int backward = PyObject_IsTrue(a[0]);
        if (backward < 0) throw Raised();
        const auto *logits = c.tensor(a[1], "logits", true), *teacher = c.tensor(a[2], "teacher", true),
                   *ids = c.tensor(a[3], "ids", true), *teacher_lse = c.tensor(a[4], "teacher_lse", false),
                   *dloss = c.tensor(a[5], "dloss", false), *loss = c.tensor(a[6], "loss", false),
                   *lse = c.tensor(a[7], "lse", false), *dlogits = c.tensor(a[8], "dlogits", false);
        two_dims(*logits, "logits");
        two_dims(*teacher, "teacher");
        fsdp_distill_args k{};
        k.tokens = logits->size(0);
        k.vocab = logits->size(1);
        k.top = teacher->size(1);
        k.dtype = c.dtype(*logits, "logits");
        k.teacher_dtype = c.dtype(*teacher, "teacher");
        if (ids->scalar_type() != at::kInt && ids->scalar_type() != at::kLong)
            raise(PyExc_TypeError, "ids must be of dtype int32 or int64");
        k.ids_64 = ids->scalar_type() == at::kLong;
        if (teacher_lse) c.dtype(*teacher_lse, "teacher_lse", FSDP_DTYPE_F32);
        if (dloss) c.dtype(*dloss, "dloss", FSDP_DTYPE_F32);
        if (loss) c.dtype(*loss, "loss", FSDP_DTYPE_F32);
        if (lse) c.dtype(*lse, "lse", FSDP_DTYPE_F32);
        if (dlogits) c.dtype(*dlogits, "dlogits", k.dtype);
        if (!dlogits != !dloss) raise(PyExc_ValueError, "dloss and dlogits go together");
        int64_t stride;
        k.logits = c.matrix(logits, "logits", k.tokens, k.vocab, &k.logits_stride);
        k.dlogits = c.matrix(dlogits, "dlogits", k.tokens, k.vocab, &k.dlogits_stride);
        k.teacher = c.matrix(teacher, "teacher", k.tokens, k.top, &stride);
        if (stride != k.top) raise(PyExc_ValueError, "teacher must be contiguous");
        k.ids = c.matrix(ids, "ids", k.tokens, k.top, &stride);
        if (stride != k.top) raise(PyExc_ValueError, "ids must be contiguous");
        k.teacher_lse = static_cast<const float*>(c.vector(teacher_lse, "teacher_lse", k.tokens));
        k.dloss = static_cast<const float*>(c.vector(dloss, "dloss", k.tokens));
        k.loss = static_cast<float*>(c.vector(loss, "loss", k.tokens));
        k.lse = static_cast<float*>(c.vector(lse, "lse", k.tokens));
        k.temperature = float(number(a[9], "temperature"));
        const hipStream_t s = c.stream(a[10]);
        const c10::hip::HIPGuard guard(c10::DeviceIndex(c.device()));
        return backward ? fsdp_block_distill_grad(&k, s) : fsdp_block_distill(&k, s);
    });
}

// last_error() -> the detail of the last status
PyObject* last_error(PyObject*, PyObject*) { return PyUnicode_FromString(fsdp_block_last_error()); }

PyMethodDef methods[] = {{"norm", FSDP_FAST(norm), nullptr},
                         {"norm_grad", FSDP_FAST(norm_grad), nullptr},
                         {"linear", FSDP_FAST(linear), nullptr},
                         {"linear_grad", FSDP_FAST(linear_grad), nullptr},
                         {"distill", FSDP_FAST(distill), nullptr},
                         {"last_error", last_error, METH_NOARGS, nullptr},
                         {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_block_marshal", "Argument marshalling of the block operators.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__block_marshal(void) { return PyModule_Create(&module); }
