// Argument marshalling of the operators of fsdp_step.h, for the Python binding;
// as block_marshal.cpp.

#include "marshal_call.h"

#include "fsdp_step.h"

namespace {

// A matrix that may be kept in 8 bits: a tensor, or a pair (codes, scales).
struct Kept {
    const at::Tensor *values = nullptr, *scales = nullptr;
    explicit operator bool() const { return values; }
    bool saved() const { return scales; }
};

Kept kept(Call& c, PyObject* o, const char* name, bool needed) {
    Kept k;
    if (!PyTuple_Check(o)) {
        k.values = c.tensor(o, name, needed);
        return k;
    }
    if (PyTuple_GET_SIZE(o) != 2) raise(PyExc_TypeError, "%s must be a tensor or a Checkpoint (codes, scales)", name);
    k.values = c.tensor(PyTuple_GET_ITEM(o, 0), name, true);
    k.scales = c.tensor(PyTuple_GET_ITEM(o, 1), name, true);
    if (k.values->scalar_type() != at::kChar) raise(PyExc_TypeError, "%s: its codes must be of dtype int8", name);
    if (k.scales->scalar_type() != at::kByte) raise(PyExc_TypeError, "%s: its scales must be of dtype uint8", name);
    return k;
}

// The shape of a kept matrix is given; the types of one that is not in 8 bits too.
void* kept_matrix(Call& c, const Kept& k, const char* name, int64_t rows, int64_t cols, fsdp_dtype dtype, int64_t* stride, void** scales,
                  int64_t* scales_stride) {
    *scales = nullptr;
    *scales_stride = 0;
    if (k.values && !k.scales) c.dtype(*k.values, name, dtype);
    if (k.scales) {
        const int64_t groups = (cols + FSDP_STEP_GROUP - 1) / FSDP_STEP_GROUP;
        if (k.scales->dim() != 2 || k.scales->size(0) != rows || k.scales->size(1) != groups)
            raise(PyExc_ValueError, "%s: its scales must have the shape (%lld, %lld)", name, (long long)rows, (long long)groups);
        *scales = c.matrix(k.scales, name, rows, groups, scales_stride);
    }
    return c.matrix(k.values, name, rows, cols, stride);
}

// save(x, codes_and_scales, stream)
PyObject* save(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return entry(n, 3, [&]() -> fsdp_status {
        Call c;
        const auto* x = c.tensor(a[0], "x", true);
        const Kept s = kept(c, a[1], "checkpoint", true);
        if (!s.saved()) raise(PyExc_TypeError, "checkpoint must be a Checkpoint (codes, scales)");
        two_dims(*x, "x");
        fsdp_step_save_args k{};
        k.rows = x->size(0);
        k.cols = x->size(1);
        k.dtype = c.dtype(*x, "x");
        k.x = c.matrix(x, "x", k.rows, k.cols, &k.x_stride);
        k.codes = kept_matrix(c, s, "checkpoint", k.rows, k.cols, k.dtype, &k.codes_stride, &k.scales, &k.scales_stride);
        const hipStream_t stream = c.stream(a[2]);
        const c10::hip::HIPGuard guard(c10::DeviceIndex(c.device()));
        return fsdp_step_save(&k, stream);
    });
}

// restore(codes_and_scales, x, stream)
PyObject* restore(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return entry(n, 3, [&]() -> fsdp_status {
        Call c;
        const Kept s = kept(c, a[0], "checkpoint", true);
        if (!s.saved()) raise(PyExc_TypeError, "checkpoint must be a Checkpoint (codes, scales)");
        const auto* x = c.tensor(a[1], "out", true);
        two_dims(*x, "out");
        fsdp_step_restore_args k{};
        k.rows = x->size(0);
        k.cols = x->size(1);
        k.dtype = c.dtype(*x, "out");
        void* scales;
        k.codes = kept_matrix(c, s, "checkpoint", k.rows, k.cols, k.dtype, &k.codes_stride, &scales, &k.scales_stride);
        k.scales = scales;
        k.x = c.matrix(x, "out", k.rows, k.cols, &k.x_stride);
        const hipStream_t stream = c.stream(a[2]);
        const c10::hip::HIPGuard guard(c10::DeviceIndex(c.device()));
        return fsdp_step_restore(&k, stream);
    });
}

// gated(x, gate_weight, up_weight, out, activation, gate, up, stream)
PyObject* gated(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return entry(n, 8, [&]() -> fsdp_status {
        Call c;
        const auto *x = c.tensor(a[0], "x", true), *gw = c.tensor(a[1], "gate_weight", true), *uw = c.tensor(a[2], "up_weight", true),
                   *out = c.tensor(a[3], "out", true);
        const Kept gate = kept(c, a[5], "gate", false), up = kept(c, a[6], "up", false);
        two_dims(*x, "x");
        two_dims(*gw, "gate_weight");
        if (!gate != !up) raise(PyExc_ValueError, "gate and up go together");
        if (gate.saved() != up.saved()) raise(PyExc_TypeError, "gate and up must both be tensors or both Checkpoints");
        fsdp_step_gated_args k{};
        k.m = x->size(0);
        k.n = gw->size(0);
        k.k = x->size(1);
        k.dtype = c.dtype(*x, "x");
        c.dtype(*gw, "gate_weight", k.dtype);
        c.dtype(*uw, "up_weight", k.dtype);
        c.dtype(*out, "out", k.dtype);
        k.activation = activation_of(a[4]);
        k.x = c.matrix(x, "x", k.m, k.k, &k.x_stride);
        k.gate_weight = c.matrix(gw, "gate_weight", k.n, k.k, &k.gate_weight_stride);
        k.up_weight = c.matrix(uw, "up_weight", k.n, k.k, &k.up_weight_stride);
        k.gate = kept_matrix(c, gate, "gate", k.m, k.n, k.dtype, &k.gate_stride, &k.gate_scales, &k.gate_scales_stride);
        k.up = kept_matrix(c, up, "up", k.m, k.n, k.dtype, &k.up_stride, &k.up_scales, &k.up_scales_stride);
        k.out = c.matrix(out, "out", k.m, k.n, &k.out_stride);
        const hipStream_t s = c.stream(a[7]);
        const c10::hip::HIPGuard guard(c10::DeviceIndex(c.device()));
        int64_t bytes = 0;
        const fsdp_status st = fsdp_step_gated_workspace(&k, &bytes);
        if (st != FSDP_OK) return st;
        const Workspace w(bytes, s);
        return fsdp_step_gated(&k, w.data(), w.bytes(), s);
    });
}

// gated_grad(dout, x, gate_weight, up_weight, gate, up, activation, out, dx, dgate_weight, dup_weight, stream)
PyObject* gated_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return entry(n, 12, [&]() -> fsdp_status {
        Call c;
        const auto* dout = c.tensor(a[0], "dout", true);
        const Kept x = kept(c, a[1], "x", true);
        const auto *gw = c.tensor(a[2], "gate_weight", true), *uw = c.tensor(a[3], "up_weight", true);
        const Kept gate = kept(c, a[4], "gate", true), up = kept(c, a[5], "up", true);
        const auto *out = c.tensor(a[7], "out", false), *dx = c.tensor(a[8], "dx", false),
                   *dgw = c.tensor(a[9], "dgate_weight", false), *duw = c.tensor(a[10], "dup_weight", false);
        two_dims(*dout, "dout");
        two_dims(*x.values, "x");
        if (gate.saved() != up.saved()) raise(PyExc_TypeError, "gate and up must both be tensors or both Checkpoints");
        if (!dgw != !duw) raise(PyExc_ValueError, "dgate_weight and dup_weight go together");
        fsdp_step_gated_grad_args k{};
        k.m = dout->size(0);
        k.n = dout->size(1);
        k.k = x.values->size(1);
        k.dtype = c.dtype(*dout, "dout");
        c.dtype(*gw, "gate_weight", k.dtype);
        c.dtype(*uw, "up_weight", k.dtype);
        if (out) c.dtype(*out, "out", k.dtype);
        if (dx) c.dtype(*dx, "dx", k.dtype);
        if (dgw) c.dtype(*dgw, "dgate_weight", k.dtype);
        if (duw) c.dtype(*duw, "dup_weight", k.dtype);
        k.activation = activation_of(a[6]);
        void *xs, *gs, *us;
        k.dout = c.matrix(dout, "dout", k.m, k.n, &k.dout_stride);
        k.x = kept_matrix(c, x, "x", k.m, k.k, k.dtype, &k.x_stride, &xs, &k.x_scales_stride);
        k.gate_weight = c.matrix(gw, "gate_weight", k.n, k.k, &k.gate_weight_stride);
        k.up_weight = c.matrix(uw, "up_weight", k.n, k.k, &k.up_weight_stride);
        k.gate = kept_matrix(c, gate, "gate", k.m, k.n, k.dtype, &k.gate_stride, &gs, &k.gate_scales_stride);
        k.up = kept_matrix(c, up, "up", k.m, k.n, k.dtype, &k.up_stride, &us, &k.up_scales_stride);
        k.x_scales = xs;
        k.gate_scales = gs;
        k.up_scales = us;
        k.out = c.matrix(out, "out", k.m, k.n, &k.out_stride);
        k.dx = c.matrix(dx, "dx", k.m, k.k, &k.dx_stride);
        k.dgate_weight = c.matrix(dgw, "dgate_weight", k.n, k.k, &k.dgate_weight_stride);
        k.dup_weight = c.matrix(duw, "dup_weight", k.n, k.k, &k.dup_weight_stride);
        const hipStream_t s = c.stream(a[11]);
        const c10::hip::HIPGuard guard(c10::DeviceIndex(c.device()));
        int64_t bytes = 0;
        const fsdp_status st = fsdp_step_gated_grad_workspace(&k, &bytes);
        if (st != FSDP_OK) return st;
        const Workspace w(bytes, s);
        return fsdp_step_gated_grad(&k, w.data(), w.bytes(), s);
    });
}

// linear_grad(dout, x, weight, activation, pre, times, dx, dweight, dbias, dtimes, stream)
PyObject* linear_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return entry(n, 11, [&]() -> fsdp_status {
        Call c;
        const auto* dout = c.tensor(a[0], "dout", true);
        const Kept x = kept(c, a[1], "x", true);
        const auto* weight = c.tensor(a[2], "weight", true);
        const Kept pre = kept(c, a[4], "pre", false);
        const auto *times = c.tensor(a[5], "times", false), *dx = c.tensor(a[6], "dx", false),
                   *dweight = c.tensor(a[7], "dweight", false), *dbias = c.tensor(a[8], "dbias", false),
                   *dtimes = c.tensor(a[9], "dtimes", false);
        two_dims(*x.values, "x");
        two_dims(*weight, "weight");
        fsdp_step_linear_grad_args k{};
        k.m = x.values->size(0);
        k.n = weight->size(0);
        k.k = x.values->size(1);
        k.dtype = c.dtype(*weight, "weight");
        c.dtype(*dout, "dout", k.dtype);
        if (times) c.dtype(*times, "times", k.dtype);
        if (dx) c.dtype(*dx, "dx", k.dtype);
        if (dweight) c.dtype(*dweight, "dweight", k.dtype);
        if (dbias) c.dtype(*dbias, "dbias", k.dtype);
        if (dtimes) c.dtype(*dtimes, "dtimes", k.dtype);
        if (dtimes && !times) raise(PyExc_ValueError, "dtimes needs times");
        k.activation = activation_of(a[3]);
        void *xs, *ps;
        k.dout = c.matrix(dout, "dout", k.m, k.n, &k.dout_stride);
        k.x = kept_matrix(c, x, "x", k.m, k.k, k.dtype, &k.x_stride, &xs, &k.x_scales_stride);
        k.weight = c.matrix(weight, "weight", k.n, k.k, &k.weight_stride);
        k.pre = kept_matrix(c, pre, "pre", k.m, k.n, k.dtype, &k.pre_stride, &ps, &k.pre_scales_stride);
        k.x_scales = xs;
        k.pre_scales = ps;
        k.times = c.matrix(times, "times", k.m, k.n, &k.times_stride);
        k.dx = c.matrix(dx, "dx", k.m, k.k, &k.dx_stride);
        k.dweight = c.matrix(dweight, "dweight", k.n, k.k, &k.dweight_stride);
        k.dbias = c.vector(dbias, "dbias", k.n);
        k.dtimes = c.matrix(dtimes, "dtimes", k.m, k.n, &k.dtimes_stride);
        const hipStream_t s = c.stream(a[10]);
        const c10::hip::HIPGuard guard(c10::DeviceIndex(c.device()));
        int64_t bytes = 0;
        const fsdp_status st = fsdp_step_linear_grad_workspace(&k, &bytes);
        if (st != FSDP_OK) return st;
        const Workspace w(bytes, s);
        return fsdp_step_linear_grad(&k, w.data(), w.bytes(), s);
    });
}

// policy(backward, logits, actions, old_logp, advantages, ref_logp, dloss, loss, logp, lse, dlogits, clip_low, clip_high, kl_weight,
//        temperature, stream)
PyObject* policy(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return entry(n, 16, [&]() -> fsdp_status {
        Call c;
        const int backward = PyObject_IsTrue(a[0]);
        if (backward < 0) throw Raised();
        const auto *logits = c.tensor(a[1], "logits", true), *actions = c.tensor(a[2], "actions", true);
        static const char* const names[] = {"old_logp", "advantages", "ref_logp", "dloss", "loss", "logp", "lse"};
        const at::Tensor* v[7];
        for (int i = 0; i < 7; ++i) {
            v[i] = c.tensor(a[3 + i], names[i], i < 2);
            if (v[i]) c.dtype(*v[i], names[i], FSDP_DTYPE_F32);
        }
        const auto* dlogits = c.tensor(a[10], "dlogits", false);
        two_dims(*logits, "logits");
        fsdp_step_policy_args k{};
        k.tokens = logits->size(0);
        k.vocab = logits->size(1);
        k.dtype = c.dtype(*logits, "logits");
        if (actions->scalar_type() != at::kInt && actions->scalar_type() != at::kLong)
            raise(PyExc_TypeError, "actions must be of dtype int32 or int64");
        k.actions_64 = actions->scalar_type() == at::kLong;
        if (dlogits) c.dtype(*dlogits, "dlogits", k.dtype);
        if (!dlogits != !v[3]) raise(PyExc_ValueError, "dloss and dlogits go together");
        k.logits = c.matrix(logits, "logits", k.tokens, k.vocab, &k.logits_stride);
        k.dlogits = c.matrix(dlogits, "dlogits", k.tokens, k.vocab, &k.dlogits_stride);
        k.actions = c.vector(actions, "actions", k.tokens);
        float* p[7];
        for (int i = 0; i < 7; ++i) p[i] = static_cast<float*>(c.vector(v[i], names[i], k.tokens));
        k.old_logp = p[0];
        k.advantages = p[1];
        k.ref_logp = p[2];
        k.dloss = p[3];
        k.loss = p[4];
        k.logp = p[5];
        k.lse = p[6];
        k.clip_low = float(number(a[11], "clip_low"));
        k.clip_high = float(number(a[12], "clip_high"));
        k.kl_weight = float(number(a[13], "kl_weight"));
        k.temperature = float(number(a[14], "temperature"));
        const hipStream_t s = c.stream(a[15]);
        const c10::hip::HIPGuard guard(c10::DeviceIndex(c.device()));
        return backward ? fsdp_step_policy_grad(&k, s) : fsdp_step_policy(&k, s);
    });
}

// last_error() -> the detail of the last status
PyObject* last_error(PyObject*, PyObject*) { return PyUnicode_FromString(fsdp_block_last_error()); }

PyMethodDef methods[] = {{"save", FSDP_FAST(save), nullptr},
                         {"restore", FSDP_FAST(restore), nullptr},
                         {"gated", FSDP_FAST(gated), nullptr},
                         {"gated_grad", FSDP_FAST(gated_grad), nullptr},
                         {"linear_grad", FSDP_FAST(linear_grad), nullptr},
                         {"policy", FSDP_FAST(policy), nullptr},
                         {"last_error", last_error, METH_NOARGS, nullptr},
                         {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_step_marshal", "Argument marshalling of the step's operators.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__step_marshal(void) { return PyModule_Create(&module); }
