// The Python entry points' host path in native code: argument checks, output and workspace tensors, the call into
// libspecverify, the result object.  A verification of a small batch takes about as long on the GPU as its arguments
// took to marshal through ctypes (six checked tensors, five allocations, two structures), so a decoding loop over small
// batches was bound by the host: one sequence at V = 1000 took 36 us a call, of which the GPU was busy for 19.
//
// The module holds no state but the library's entry points, the result classes and interned names.  Workspaces are
// the caller's (a Workspace object of binding.py, grown by it).
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <dlfcn.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <optional>
#include <vector>

#include <torch/csrc/autograd/python_variable.h>

#include "specverify.h"

namespace {

struct Library {
    decltype(&spec_workspace_bytes) workspace_bytes;
    decltype(&spec_analysis_workspace_bytes) analysis_workspace_bytes;
    decltype(&spec_verify_specinfer) specinfer, traversal;
    decltype(&spec_verify_otlp) otlp;
    decltype(&spec_tree_analysis) analysis;
    decltype(&spec_tree_probs) probs;
    decltype(&spec_sample_bonus) bonus;
} lib;
PyObject *verify_outputs_class, *analysis_outputs_class;
PyObject *n_buf, *n_get, *n_stream;
PyObject *n_out[10];
const char *const OUT_NAMES[10] = {"accepted_node", "accept_len", "out_tokens", "bonus_token", "status",
                                   "residual",      "node_thr",   "node_w_in",  "node_features", "margin"};

const char *error_name(int rc)
{
    static const char *const names[] = {"SPEC_OK", "SPEC_ERR_NULL", "SPEC_ERR_SHAPE", "SPEC_ERR_DTYPE", "SPEC_ERR_PARAM",
                                        "SPEC_ERR_WORKSPACE", "SPEC_ERR_UNSUPPORTED", "SPEC_ERR_CUDA"};
    return rc <= 0 && rc > -8 ? names[-rc] : "unknown error";
}

// an error that has been set as a Python exception
struct Raised {};
// a reference of this module's own
struct Owned {
    PyObject *o;
    explicit Owned(PyObject *p) : o(p) {}
    ~Owned() { Py_XDECREF(o); }
    Owned(const Owned &) = delete;
};
template <typename... A> [[noreturn]] void raise(const char *fmt, A... a)
{
    PyErr_Format(PyExc_RuntimeError, fmt, a...);
    throw Raised{};
}
void check(int rc, const char *what) { if (rc) raise("%s failed: %s", what, error_name(rc)); }

// Calls f, which touches no Python object, with the interpreter's lock released: a launch may wait (a full queue, the first use of
// a kernel), and other threads run meanwhile, as with ctypes.
template <typename F> int unlocked(F f)
{
    struct Released {
        PyThreadState *state = PyEval_SaveThread();
        ~Released() { PyEval_RestoreThread(state); }
    } released;
    return f();
}

const at::Tensor &tensor(PyObject *o, const char *name)
{
    if (!THPVariable_Check(o)) { PyErr_Format(PyExc_TypeError, "%s must be a tensor", name); throw Raised{}; }
    return THPVariable_Unpack(o);
}
const at::Tensor &cuda_tensor(PyObject *o, const char *name)
{
    const at::Tensor &t = tensor(o, name);
    if (!t.is_cuda()) raise("%s must live on a CUDA device (there is no CPU path)", name);
    return t;
}
void *pointer_or_null(PyObject *o, const char *name) { return o == Py_None ? nullptr : tensor(o, name).data_ptr(); }
double number(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Raised{};
    return v;
}
long long integer(PyObject *o)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised{};
    return v;
}
int truncated(PyObject *o)        // int(x), as the callers write it
{
    if (PyLong_Check(o)) return (int)integer(o);
    PyObject *i = PyNumber_Long(o);
    if (!i) throw Raised{};
    const long long v = PyLong_AsLongLong(i);
    Py_DECREF(i);
    if (v == -1 && PyErr_Occurred()) throw Raised{};
    return (int)v;
}
void *stream_of(PyObject *o)
{
    if (o == Py_None) return c10::cuda::getCurrentCUDAStream().stream();
    PyObject *s = PyObject_GetAttr(o, n_stream);
    if (!s) throw Raised{};
    void *p = PyLong_AsVoidPtr(s);
    Py_DECREF(s);
    if (!p && PyErr_Occurred()) throw Raised{};
    return p;
}
at::Tensor empty(at::IntArrayRef sizes, at::ScalarType t, const at::Device &d)
{
    return at::Tensor(at::detail::empty_cuda(sizes, t, d, std::nullopt));
}

// the caller's Workspace: its buffer, grown by the object itself when too small (held until the call has been enqueued: another
// thread may grow the object meanwhile)
struct Scratch { void *ptr; int64_t bytes; at::Tensor buf; };
Scratch scratch_of(PyObject *workspace, int64_t bytes)
{
    for (int attempt = 0;; ++attempt) {
        PyObject *buf = PyObject_GetAttr(workspace, n_buf);
        if (!buf) throw Raised{};
        if (buf != Py_None) {
            const Owned held(buf);
            const at::Tensor t = tensor(buf, "buf");
            const int64_t have = t.numel();
            char *base = (char *)t.data_ptr();
            if (have >= bytes + 256) {
                const int64_t off = (256 - ((intptr_t)base & 255)) & 255;
                return {base + off, have - off, t};
            }
        } else {
            Py_DECREF(buf);
        }
        if (attempt) raise("the workspace did not grow");
        PyObject *n = PyLong_FromLongLong(bytes), *r = n ? PyObject_CallMethodOneArg(workspace, n_get, n) : nullptr;
        Py_XDECREF(n);
        if (!r) throw Raised{};
        Py_DECREF(r);
    }
}

void check_vector(const at::Tensor &t, const char *name, at::ScalarType dt, const char *type)
{
    if (t.scalar_type() != dt || !t.is_contiguous()) raise("%s must be a contiguous %s tensor", name, type);
}

// arguments 0 .. 9 of every call on a batch of trees: target, draft, parent, token, u_accept, u_bonus, temperature, top_k,
// top_p, temperature_per_seq
SpecIn spec_in(PyObject *const *a)
{
    const at::Tensor &zp = cuda_tensor(a[0], "target_logits"), &zq = cuda_tensor(a[1], "draft_logits");
    const at::Tensor &parent = cuda_tensor(a[2], "parent"), &token = cuda_tensor(a[3], "token");
    const at::Tensor &ua = cuda_tensor(a[4], "u_accept"), &ub = cuda_tensor(a[5], "u_bonus");
    const auto dt = zp.scalar_type();
    if ((dt != at::kFloat && dt != at::kBFloat16) || zq.scalar_type() != dt) raise("logits must both be float32 or both bfloat16");
    if (zp.dim() != 3 || zp.stride(2) != 1 || zq.dim() != 3 || zq.strides() != zp.strides())
        raise("logits must be [B,N,V] with a contiguous vocabulary axis and equal strides");
    const int64_t B = zp.size(0), N = zp.size(1), V = zp.size(2);
    check_vector(parent, "parent", at::kInt, "torch.int32");
    check_vector(token, "token", at::kInt, "torch.int32");
    check_vector(ua, "u_accept", at::kFloat, "torch.float32");
    check_vector(ub, "u_bonus", at::kFloat, "torch.float32");
    const auto is_bn = [&](const at::Tensor &t) { return t.dim() == 2 && t.size(0) == B && t.size(1) == N; };
    if (!is_bn(token) || !is_bn(ua) || !is_bn(ub)) raise("token, u_accept and u_bonus must be [B,N]");
    if (!(parent.dim() == 1 && parent.size(0) == N) && !is_bn(parent)) raise("parent must be [N] or [B,N]");
    SpecIn in = {};
    in.B = (int32_t)B; in.N = (int32_t)N; in.V = (int32_t)V;
    in.logits_dtype = dt == at::kFloat ? SPEC_F32 : SPEC_BF16;
    in.target_logits = zp.data_ptr(); in.draft_logits = zq.data_ptr();
    in.seq_stride = zp.stride(0); in.node_stride = zp.stride(1);
    in.parent = (const int32_t *)parent.data_ptr(); in.topo_seq_stride = parent.dim() == 1 ? 0 : N;
    in.token = (const int32_t *)token.data_ptr();
    in.temperature = (float)number(a[6]); in.top_k = truncated(a[7]); in.top_p = (float)number(a[8]);
    in.temperature_per_seq = (const float *)pointer_or_null(a[9], "temperature_per_seq");
    in.u_accept = (const float *)ua.data_ptr(); in.u_bonus = (const float *)ub.data_ptr();
    return in;
}

template <typename F> PyObject *guarded(F f)
{
    try {
        return f();
    } catch (const Raised &) {
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}
bool arity(Py_ssize_t n, Py_ssize_t want)
{
    if (n == want) return true;
    PyErr_Format(PyExc_TypeError, "%zd arguments expected, got %zd", want, n);
    return false;
}

// an object of one of the result classes from n tensors (undefined ones: None)
PyObject *result(PyObject *cls, const at::Tensor *t, int n)
{
    PyObject *args[10];
    int made = 0;
    for (; made < n; ++made) {
        args[made] = t[made].defined() ? THPVariable_Wrap(t[made]) : Py_NewRef(Py_None);
        if (!args[made]) break;
    }
    PyObject *r = made == n ? PyObject_Vectorcall(cls, args, n, nullptr) : nullptr;
    while (made > 0) Py_DECREF(args[--made]);
    if (!r) throw Raised{};
    return r;
}

// verify(code, <10 batch arguments>, outputs, workspace, stream, flags): code 0 SpecInfer, 1 Traversal, 2 + s the walk with
// OTLP solver s; flags: optional outputs to allocate, bit i for output 5 + i
PyObject *py_verify(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!arity(n, 15)) return nullptr;
    return guarded([&]() -> PyObject * {
        const int code = (int)integer(a[0]), flags = (int)integer(a[14]);
        const SpecIn in = spec_in(a + 1);
        int64_t bytes = 0;
        check(lib.workspace_bytes(&in, &bytes), "spec_workspace_bytes");
        const Scratch ws = scratch_of(a[12], bytes);
        PyObject *given = a[11];
        at::Tensor t[10];
        void *p[10] = {};
        if (given == Py_None) {
            const at::Device dev = THPVariable_Unpack(a[1]).device();
            const int64_t B = in.B, N = in.N;
            for (int i = 0; i < 5; ++i) t[i] = i == 2 ? empty({B, N}, at::kInt, dev) : empty({B}, at::kInt, dev);
            if (flags & 1) t[5] = empty({B, (int64_t)in.V}, at::kFloat, dev);
            if (flags & 2) t[6] = empty({B, N}, at::kFloat, dev);
            if (flags & 4) t[7] = empty({B, N}, at::kFloat, dev);
            if (flags & 8) t[8] = empty({B, N, 4}, at::kFloat, dev);
            if (flags & 16) t[9] = empty({B, N + 1}, at::kFloat, dev);
            for (int i = 0; i < 10; ++i) if (t[i].defined()) p[i] = t[i].data_ptr();
        } else {
            for (int i = 0; i < 10; ++i) {
                const Owned o(PyObject_GetAttr(given, n_out[i]));
                if (!o.o) throw Raised{};
                if (o.o == Py_None) continue;
                t[i] = tensor(o.o, OUT_NAMES[i]);          // (held until the call has been enqueued: the attribute may be computed)
                p[i] = t[i].data_ptr();
            }
        }
        const SpecOut out = {(int32_t *)p[0], (int32_t *)p[1], (int32_t *)p[2], (int32_t *)p[3], (int32_t *)p[4],
                             (float *)p[5], (float *)p[6], (float *)p[7], (float *)p[8], (float *)p[9]};
        void *st = stream_of(a[13]);
        const int rc = unlocked([&] {
            return code == 0   ? lib.specinfer(&in, &out, ws.ptr, ws.bytes, st)
                   : code == 1 ? lib.traversal(&in, &out, ws.ptr, ws.bytes, st)
                               : lib.otlp(&in, &out, code - 2, ws.ptr, ws.bytes, st);
        });
        check(rc, code == 0 ? "spec_verify_specinfer" : code == 1 ? "spec_verify_traversal" : "spec_verify_otlp");
        return given == Py_None ? result(verify_outputs_class, t, 10) : Py_NewRef(given);
    });
}

// tree_analysis(<10 batch arguments>, workspace, stream)
PyObject *py_analysis(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!arity(n, 12)) return nullptr;
    return guarded([&]() -> PyObject * {
        const SpecIn in = spec_in(a);
        const at::Device dev = THPVariable_Unpack(a[0]).device();
        const int64_t B = in.B, N = in.N;
        at::Tensor t[5] = {empty({B, N, 4}, at::kFloat, dev), empty({B, N, 3}, at::kFloat, dev), empty({5, B, N}, at::kFloat, dev),
                           empty({5, B, N}, at::kFloat, dev), empty({5, B}, at::kFloat, dev)};
        int64_t bytes = 0;
        check(lib.analysis_workspace_bytes(&in, &bytes), "spec_analysis_workspace_bytes");
        const Scratch ws = scratch_of(a[10], bytes);
        const SpecAnalysisOut out = {(float *)t[0].data_ptr(), (float *)t[1].data_ptr(), (float *)t[2].data_ptr(),
                                     (float *)t[3].data_ptr(), (float *)t[4].data_ptr()};
        void *st = stream_of(a[11]);
        check(unlocked([&] { return lib.analysis(&in, &out, ws.ptr, ws.bytes, st); }), "spec_tree_analysis");
        return result(analysis_outputs_class, t, 5);
    });
}

// tree_probs(logits, which, temperature, top_k, top_p, temperature_per_seq, want_probs, want_stats, workspace, stream)
PyObject *py_probs(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!arity(n, 10)) return nullptr;
    return guarded([&]() -> PyObject * {
        const at::Tensor &z = cuda_tensor(a[0], "logits");
        const auto dt = z.scalar_type();
        if (z.dim() != 3 || z.stride(2) != 1 || (dt != at::kFloat && dt != at::kBFloat16))
            raise("logits must be [B,N,V] float32 / bfloat16 with a contiguous vocabulary axis");
        const int64_t B = z.size(0), N = z.size(1), V = z.size(2);
        SpecIn in = {};
        in.B = (int32_t)B; in.N = (int32_t)N; in.V = (int32_t)V;
        in.logits_dtype = dt == at::kFloat ? SPEC_F32 : SPEC_BF16;
        in.target_logits = in.draft_logits = z.data_ptr();
        in.seq_stride = z.stride(0); in.node_stride = z.stride(1);
        in.temperature = (float)number(a[2]); in.top_k = truncated(a[3]); in.top_p = (float)number(a[4]);
        in.temperature_per_seq = (const float *)pointer_or_null(a[5], "temperature_per_seq");
        at::Tensor probs, stats;
        if (PyObject_IsTrue(a[6])) probs = empty({B, N, V}, at::kFloat, z.device());
        if (PyObject_IsTrue(a[7])) stats = empty({B, N, 6}, at::kFloat, z.device());
        int64_t bytes = 0;
        check(lib.workspace_bytes(&in, &bytes), "spec_workspace_bytes");
        const Scratch ws = scratch_of(a[8], bytes);        // holds the rows' records when truncating
        const int which = truncated(a[1]);
        float *pr = probs.defined() ? (float *)probs.data_ptr() : nullptr, *st = stats.defined() ? (float *)stats.data_ptr() : nullptr;
        void *stream = stream_of(a[9]);
        check(unlocked([&] { return lib.probs(&in, which, pr, st, ws.ptr, ws.bytes, stream); }), "spec_tree_probs");
        PyObject *p = probs.defined() ? THPVariable_Wrap(probs) : Py_NewRef(Py_None);
        PyObject *s = stats.defined() ? THPVariable_Wrap(stats) : Py_NewRef(Py_None);
        PyObject *r = p && s ? PyTuple_Pack(2, p, s) : nullptr;
        Py_XDECREF(p);
        Py_XDECREF(s);
        return r;
    });
}

// sample_bonus(weights, u, want_margin, stream)
PyObject *py_bonus(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!arity(n, 4)) return nullptr;
    return guarded([&]() -> PyObject * {
        const at::Tensor &w = cuda_tensor(a[0], "weights"), &u = cuda_tensor(a[1], "u");
        if (w.scalar_type() != at::kFloat || !w.is_contiguous() || w.dim() != 2) raise("weights must be a contiguous [R,V] float32 tensor");
        if (u.scalar_type() != at::kFloat || !u.is_contiguous() || u.numel() != w.size(0))
            raise("u must be a contiguous float32 tensor with one entry per row");
        const bool want = PyObject_IsTrue(a[2]);
        at::Tensor token = empty({w.size(0)}, at::kInt, w.device()), margin;
        if (want) margin = empty({w.size(0)}, at::kFloat, w.device());
        const float *wp = (const float *)w.data_ptr(), *up = (const float *)u.data_ptr();
        const int32_t R = (int32_t)w.size(0), V = (int32_t)w.size(1);
        int32_t *tp = (int32_t *)token.data_ptr();
        float *mp = want ? (float *)margin.data_ptr() : nullptr;
        void *st = stream_of(a[3]);
        check(unlocked([&] { return lib.bonus(wp, R, V, up, tp, mp, nullptr, 0, st); }), "spec_sample_bonus");
        PyObject *t = THPVariable_Wrap(token);
        if (!want || !t) return t;
        PyObject *m = THPVariable_Wrap(margin), *r = m ? PyTuple_Pack(2, t, m) : nullptr;
        Py_DECREF(t);
        Py_XDECREF(m);
        return r;
    });
}

// launch(code, SpecIn address, SpecOut address, workspace address, workspace bytes, stream): one of the two verifiers on
// structures that the caller has filled and keeps
PyObject *py_launch(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!arity(n, 6)) return nullptr;
    return guarded([&]() -> PyObject * {
        const auto at_ = [&](int i) { return (void *)(intptr_t)integer(a[i]); };
        const bool traversal = integer(a[0]) != 0;
        const SpecIn *in = (const SpecIn *)at_(1);
        const SpecOut *out = (const SpecOut *)at_(2);
        void *ws = at_(3), *st = stream_of(a[5]);
        const int64_t bytes = integer(a[4]);
        check(unlocked([&] { return (traversal ? lib.traversal : lib.specinfer)(in, out, ws, bytes, st); }),
              traversal ? "spec_verify_traversal" : "spec_verify_specinfer");
        Py_RETURN_NONE;
    });
}

// init(path of libspecverify.so, VerifyOutputs, AnalysisOutputs)
PyObject *py_init(PyObject *, PyObject *args)
{
    const char *path;
    PyObject *v, *an;
    if (!PyArg_ParseTuple(args, "sOO", &path, &v, &an)) return nullptr;
    void *h = dlopen(path, RTLD_NOW | RTLD_LOCAL);
    if (!h) return PyErr_Format(PyExc_RuntimeError, "%s", dlerror());
    bool ok = true;
    const auto find = [&](auto &f, const char *name) {
        f = reinterpret_cast<std::remove_reference_t<decltype(f)>>(dlsym(h, name));
        ok = ok && f;
    };
    find(lib.workspace_bytes, "spec_workspace_bytes");
    find(lib.analysis_workspace_bytes, "spec_analysis_workspace_bytes");
    find(lib.specinfer, "spec_verify_specinfer");
    find(lib.traversal, "spec_verify_traversal");
    find(lib.otlp, "spec_verify_otlp");
    find(lib.analysis, "spec_tree_analysis");
    find(lib.probs, "spec_tree_probs");
    find(lib.bonus, "spec_sample_bonus");
    if (!ok) return PyErr_Format(PyExc_RuntimeError, "%s lacks an entry point", path);
    verify_outputs_class = Py_NewRef(v);
    analysis_outputs_class = Py_NewRef(an);
    n_buf = PyUnicode_InternFromString("buf");
    n_get = PyUnicode_InternFromString("get");
    n_stream = PyUnicode_InternFromString("cuda_stream");
    for (int i = 0; i < 10; ++i) n_out[i] = PyUnicode_InternFromString(OUT_NAMES[i]);
    Py_RETURN_NONE;
}

// ---- the operators around a verification ---------------------------------------------------------------------------------------
struct StepLibrary {
    decltype(&spec_cache_slots) slots;
    decltype(&spec_norm_rope_cache) norm_rope;
    decltype(&spec_tree_attention_workspace_bytes) attention_bytes;
    decltype(&spec_tree_attention) attention;
    decltype(&spec_cache_commit) commit;
    decltype(&spec_verify_probs) probs;
} step_lib;
PyObject *slot_outputs_class, *attention_outputs_class, *commit_outputs_class, *chain_outputs_class;

// Where a call runs: the device of its tensors, made current for the call, and its stream.  A stream that the caller names may be another than the
// current one: outputs and scratch then come from that stream's memory, and the allocator is told of both streams, so that memory
// freed on one is not handed out again while the other still uses it.
class Place {
public:
    Place(const at::Tensor &first, PyObject *stream) : device_(first.device()), guard_(device_), named_(stream != Py_None)
    {
        stream_ = stream_of(stream);
        if (!named_) return;
        caller_ = c10::cuda::getCurrentCUDAStream(device_.index());
        switch_.emplace(c10::cuda::getStreamFromExternal((cudaStream_t)stream_, device_.index()));
    }
    const at::Device &device() const { return device_; }
    void *stream() const { return stream_; }
    // an input: on the same device, and in use by the call's stream
    void uses(const at::Tensor &t, const char *name) const
    {
        if (t.device() != device_) raise("%s must live on the device of the other tensors", name);
        if (named_ && t.numel()) t.record_stream(switch_->current_stream().unwrap());
    }
    at::Tensor fresh(at::IntArrayRef sizes, at::ScalarType t) const
    {
        at::Tensor r = empty(sizes, t, device_);
        if (named_ && r.numel()) r.record_stream(caller_->unwrap());
        return r;
    }

private:
    c10::Device device_;
    c10::cuda::CUDAGuard guard_;
    bool named_;
    void *stream_;
    std::optional<c10::cuda::CUDAStream> caller_;
    std::optional<c10::cuda::CUDAStreamGuard> switch_;
};

// Several int32 outputs out of one allocation (an output each costs the host about as much as the rest of a small call), on 16 bytes each.
class Pieces {
public:
    Pieces(const Place &place, std::initializer_list<int64_t> counts)
    {
        int64_t total = 0;
        for (const int64_t n : counts) total += up(n);
        base_ = place.fresh({total}, at::kInt);
    }
    at::Tensor take(at::IntArrayRef sizes)
    {
        auto piece = c10::make_intrusive<c10::TensorImpl>(c10::Storage(base_.storage()), base_.key_set(), base_.dtype());
        piece->set_storage_offset(at_);
        piece->set_sizes_contiguous(sizes);
        int64_t n = 1;
        for (const int64_t s : sizes) n *= s;
        at_ += up(n);
        return at::Tensor(std::move(piece));
    }

private:
    static int64_t up(int64_t n) { return (n + 3) / 4 * 4; }
    at::Tensor base_;
    int64_t at_ = 0;
};

void need(const void *f) { if (!f) raise("the library lacks an entry point"); }
const at::Tensor &ints(PyObject *o, const char *name, const Place &place, int64_t count = -1)
{
    const at::Tensor &t = cuda_tensor(o, name);
    check_vector(t, name, at::kInt, "torch.int32");
    if (count >= 0 && t.numel() != count) raise("%s must have %lld entries", name, (long long)count);
    place.uses(t, name);
    return t;
}
const at::Tensor &floats(PyObject *o, const char *name, const Place &place, int64_t count = -1)
{
    const at::Tensor &t = cuda_tensor(o, name);
    check_vector(t, name, at::kFloat, "torch.float32");
    if (count >= 0 && t.numel() != count) raise("%s must have %lld entries", name, (long long)count);
    place.uses(t, name);
    return t;
}
int32_t *int_ptr(const at::Tensor &t) { return (int32_t *)t.data_ptr(); }
int32_t small(int64_t v, const char *what)
{
    if (v > 0x7FFFFFFF || v < 0) raise("%s is out of range", what);
    return (int32_t)v;
}
bool truth(PyObject *o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Raised{};
    return v != 0;
}
int32_t whole(PyObject *o, const char *what)        // an int argument, whole or refused
{
    const long long v = integer(o);
    if (v > 0x7FFFFFFFll || v < -0x7FFFFFFFll - 1) raise("%s is out of range", what);
    return (int32_t)v;
}
// the parents of one tree for all, or of one per request: row length, and the stride between requests
int64_t tree_of(PyObject *o, const Place &place, int64_t B, int64_t *N, const int32_t **parent)
{
    const at::Tensor &t = ints(o, "parent", place);
    if (t.dim() == 2 ? t.size(0) != B : t.dim() != 1) raise("parent must be [N] or [B,N]");
    *N = t.size(-1);
    *parent = int_ptr(t);
    return t.dim() == 1 ? 0 : *N;
}
struct Table { int32_t *ptr; int64_t stride; int32_t width; };
Table table_of(PyObject *o, const Place &place, int64_t B)
{
    const at::Tensor &t = cuda_tensor(o, "block_table");
    if (t.scalar_type() != at::kInt || t.dim() != 2 || t.size(0) != B || (t.size(1) > 1 && t.stride(1) != 1))
        raise("block_table must be a [B,W] torch.int32 tensor with contiguous rows");
    place.uses(t, "block_table");
    const int64_t W = t.size(1);
    return {int_ptr(t), B > 1 ? t.stride(0) : (W > t.stride(0) ? W : t.stride(0)), small(W, "the table's width")};
}
int element_type(at::ScalarType t)
{
    return t == at::kFloat ? SPEC_F32 : t == at::kBFloat16 ? SPEC_BF16 : t == at::kHalf ? SPEC_F16 : -1;
}
void rows_of(const at::Tensor &t, const char *name, int dims, at::ScalarType type, const Place &place)
{
    if (t.dim() != dims || t.scalar_type() != type || (t.size(dims - 1) > 1 && t.stride(dims - 1) != 1))
        raise("%s must have %d dimensions, the last contiguous, and the type of the other tensors", name, dims);
    place.uses(t, name);
}
void no_gradient(const at::Tensor &t, const char *name)
{
    if (t.requires_grad() && c10::GradMode::is_enabled()) raise("%s requires a gradient: the call has no backward pass", name);
    if (t._fw_grad(0).defined()) raise("%s carries a tangent: the call has no forward-mode derivative", name);
}
// A tensor that the call has written: what autograd has kept of it for a backward pass is out of date.
void written(const at::Tensor &t)
{
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
// a tensor that the call writes: an expanded one has several threads at the same place
void apart(const at::Tensor &t, const char *name)
{
    for (int64_t i = 0; i < t.dim(); ++i)
        if (t.size(i) > 1 && t.stride(i) == 0) raise("the entries of %s share memory: it cannot be written", name);
}
// strides of all but the last dimension; of a dimension of one entry, which nothing steps along: 0
void strides_of(const at::Tensor &t, int64_t *to)
{
    for (int64_t i = 0; i + 1 < t.dim(); ++i) to[i] = t.size(i) > 1 ? t.stride(i) : 0;
}

// cache_slots(lengths, parent, block_table, owned, free_blocks, free_range, block_size, n_nodes, stream)
PyObject *py_slots(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!arity(n, 9)) return nullptr;
    return guarded([&]() -> PyObject * {
        need((void *)step_lib.slots);
        const at::Tensor &lengths = cuda_tensor(a[0], "lengths");
        const Place place(lengths, a[8]);
        const int64_t B = ints(a[0], "lengths", place).numel();
        int64_t N;
        SpecSlots s = {};
        s.topo_seq_stride = tree_of(a[1], place, B, &N, &s.parent);
        const Table table = table_of(a[2], place, B);
        const at::Tensor &ring = ints(a[4], "free_blocks", place);
        s.B = small(B, "B"); s.N = small(N, "N"); s.block_size = whole(a[6], "block_size"); s.table_width = table.width;
        s.lengths = int_ptr(lengths); s.block_table = table.ptr; s.table_stride = table.stride;
        s.n_nodes = a[7] == Py_None ? nullptr : int_ptr(ints(a[7], "n_nodes", place, B));
        s.owned = int_ptr(ints(a[3], "owned", place, B));
        s.free_blocks = int_ptr(ring); s.free_size = small(ring.numel(), "free_blocks");
        s.free_range = int_ptr(ints(a[5], "free_range", place, 2));
        Pieces made(place, {B * N, B * N, B, 2, B});
        const at::Tensor t[6] = {made.take({B, N}), made.take({B, N}), THPVariable_Unpack(a[2]), made.take({B}), made.take({2}), made.take({B})};
        s.slots = int_ptr(t[0]); s.positions = int_ptr(t[1]); s.owned_out = int_ptr(t[3]); s.free_range_out = int_ptr(t[4]);
        s.status = int_ptr(t[5]);
        check(unlocked([&] { return step_lib.slots(&s, place.stream()); }), "spec_cache_slots");
        written(t[2]);
        return result(slot_outputs_class, t, 6);
    });
}

// norm_rope_cache(q, k, v, inv_freq, positions, slots, k_cache, v_cache, q_weight, k_weight, eps, pairs, q_out, stream)
PyObject *py_norm_rope(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!arity(n, 14)) return nullptr;
    return guarded([&]() -> PyObject * {
        need((void *)step_lib.norm_rope);
        const at::Tensor &q = cuda_tensor(a[0], "q"), &k = cuda_tensor(a[1], "k"), &v = cuda_tensor(a[2], "v");
        const at::Tensor &kc = cuda_tensor(a[6], "k_cache"), &vc = cuda_tensor(a[7], "v_cache");
        const Place place(q, a[13]);
        const auto type = q.scalar_type();
        if (element_type(type) < 0) raise("q must be float32, bfloat16 or float16");
        rows_of(q, "q", 3, type, place);
        rows_of(k, "k", 3, type, place);
        rows_of(v, "v", 3, type, place);
        rows_of(kc, "k_cache", 4, type, place);
        rows_of(vc, "v_cache", 4, type, place);
        no_gradient(q, "q"); no_gradient(k, "k"); no_gradient(v, "v"); no_gradient(kc, "k_cache"); no_gradient(vc, "v_cache");
        apart(kc, "k_cache"); apart(vc, "v_cache");
        const int64_t T = q.size(0), D = q.size(2), Hkv = k.size(1);
        if (k.size(0) != T || k.size(2) != D || v.sizes() != k.sizes()) raise("q, k and v must be [T,Hq,D], [T,Hkv,D] and [T,Hkv,D]");
        if (kc.size(2) != Hkv || kc.size(3) != D || vc.sizes() != kc.sizes()) raise("the caches must be [num_blocks, block_size, Hkv, D]");
        SpecNormRope s = {};
        const void **weight[2] = {&s.q_weight, &s.k_weight};
        for (int i = 0; i < 2; ++i) {
            if (a[8 + i] == Py_None) continue;
            const at::Tensor &w = cuda_tensor(a[8 + i], i ? "k_weight" : "q_weight");
            if (w.scalar_type() != type || !w.is_contiguous() || w.numel() != D) raise("the weights must be contiguous [D] tensors of the type of q");
            no_gradient(w, i ? "k_weight" : "q_weight");
            place.uses(w, "weight");
            *weight[i] = w.data_ptr();
        }
        const at::Tensor &freq = floats(a[3], "inv_freq", place);
        no_gradient(freq, "inv_freq");
        s.positions = int_ptr(ints(a[4], "positions", place, T));
        s.slots = int_ptr(ints(a[5], "slots", place, T));
        s.T = small(T, "T"); s.Hq = small(q.size(1), "Hq"); s.Hkv = small(Hkv, "Hkv"); s.D = small(D, "D");
        s.rot = small(2 * freq.numel(), "inv_freq"); s.pairs = whole(a[11], "pairs"); s.dtype = element_type(type); s.eps = (float)number(a[10]);
        s.num_blocks = small(kc.size(0), "num_blocks"); s.block_size = small(kc.size(1), "block_size");
        at::Tensor out;
        if (a[12] == Py_None) {
            out = place.fresh(q.sizes(), type);
        } else {
            out = cuda_tensor(a[12], "q_out");
            rows_of(out, "q_out", 3, type, place);
            if (out.sizes() != q.sizes()) raise("q_out must have the shape of q");
            no_gradient(out, "q_out");
            apart(out, "q_out");
        }
        s.q = q.data_ptr(); s.k = k.data_ptr(); s.v = v.data_ptr(); s.inv_freq = (const float *)freq.data_ptr();
        s.q_out = out.data_ptr(); s.k_cache = kc.data_ptr(); s.v_cache = vc.data_ptr();
        strides_of(q, s.q_stride); strides_of(k, s.k_stride); strides_of(v, s.v_stride); strides_of(out, s.q_out_stride);
        strides_of(kc, s.k_cache_stride); strides_of(vc, s.v_cache_stride);
        if (T) check(unlocked([&] { return step_lib.norm_rope(&s, place.stream()); }), "spec_norm_rope_cache");
        written(kc); written(vc);
        if (a[12] != Py_None) written(out);
        return THPVariable_Wrap(out);
    });
}

// What the calls of attention have alike: q, k_cache, v_cache, block_table, lengths, parent, n_nodes (a[0] .. a[6]), scale, out, want_lse.  The
// tensors that are made or written: out, status, lse.
SpecAttention attention_of(PyObject *const *a, PyObject *scale, PyObject *out, PyObject *want_lse, const Place &place, at::Tensor (&t)[3])
{
    const at::Tensor &q = cuda_tensor(a[0], "q"), &kc = cuda_tensor(a[1], "k_cache"), &vc = cuda_tensor(a[2], "v_cache");
    const auto type = q.scalar_type();
    if (type != at::kBFloat16 && type != at::kHalf) raise("q must be bfloat16 or float16");
    rows_of(q, "q", 4, type, place);
    rows_of(kc, "k_cache", 4, type, place);
    rows_of(vc, "v_cache", 4, type, place);
    no_gradient(q, "q"); no_gradient(kc, "k_cache"); no_gradient(vc, "v_cache");
    const int64_t B = q.size(0), Hq = q.size(2), D = q.size(3);
    if (kc.size(3) != D || vc.sizes() != kc.sizes()) raise("the caches must be [num_blocks, block_size, Hkv, D]");
    SpecAttention s = {};
    int64_t N;
    s.topo_seq_stride = tree_of(a[5], place, B, &N, &s.parent);
    if (N != q.size(1)) raise("q must be [B,N,Hq,D] with the N of parent");
    const Table table = table_of(a[3], place, B);
    s.B = small(B, "B"); s.N = small(N, "N"); s.Hq = small(Hq, "Hq"); s.Hkv = small(kc.size(2), "Hkv"); s.D = small(D, "D");
    s.dtype = element_type(type);
    s.num_blocks = small(kc.size(0), "num_blocks"); s.block_size = small(kc.size(1), "block_size"); s.table_width = table.width;
    s.scale = scale == Py_None ? (float)(1.0 / std::sqrt((double)(D > 0 ? D : 1))) : (float)number(scale);
    s.block_table = table.ptr; s.table_stride = table.stride;
    s.lengths = int_ptr(ints(a[4], "lengths", place, B));
    s.n_nodes = a[6] == Py_None ? nullptr : int_ptr(ints(a[6], "n_nodes", place, B));
    if (out == Py_None) {
        t[0] = place.fresh(q.sizes(), type);
    } else {
        t[0] = cuda_tensor(out, "out");
        rows_of(t[0], "out", 4, type, place);
        if (t[0].sizes() != q.sizes()) raise("out must have the shape of q");
        no_gradient(t[0], "out");
        apart(t[0], "out");
    }
    t[1] = place.fresh({B}, at::kInt);
    if (truth(want_lse)) t[2] = place.fresh({B, N, Hq}, at::kFloat);
    s.q = q.data_ptr(); s.k_cache = kc.data_ptr(); s.v_cache = vc.data_ptr(); s.out = t[0].data_ptr(); s.status = int_ptr(t[1]);
    s.lse = t[2].defined() ? (float *)t[2].data_ptr() : nullptr;
    strides_of(q, s.q_stride); strides_of(kc, s.k_cache_stride); strides_of(vc, s.v_cache_stride); strides_of(t[0], s.out_stride);
    return s;
}

// tree_attention(q, k_cache, v_cache, block_table, lengths, parent, n_nodes, scale, window, sinks, out, want_lse, stream)
PyObject *py_attention(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!arity(n, 13)) return nullptr;
    return guarded([&]() -> PyObject * {
        need((void *)step_lib.attention);
        const Place place(cuda_tensor(a[0], "q"), a[12]);
        at::Tensor t[3];
        SpecAttention s = attention_of(a, a[7], a[10], a[11], place, t);
        s.window = whole(a[8], "window"); s.sinks = whole(a[9], "sinks");
        int64_t bytes = 0;
        check(step_lib.attention_bytes(&s, &bytes), "spec_tree_attention_workspace_bytes");
        // scratch of this call alone (the allocator's blocks lie on 512 bytes): calls on several streams, or captured into several
        // graphs, never share it
        const at::Tensor ws = empty({bytes}, at::kByte, place.device());
        check(unlocked([&] { return step_lib.attention(&s, ws.data_ptr(), bytes, place.stream()); }), "spec_tree_attention");
        if (a[10] != Py_None) written(t[0]);
        return result(attention_outputs_class, t, 3);
    });
}

// cache_commit(cache, accepted_node, parent, lengths, block_table, n_nodes, stream)
PyObject *py_commit(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!arity(n, 7)) return nullptr;
    return guarded([&]() -> PyObject * {
        need((void *)step_lib.commit);
        const at::Tensor &cache = cuda_tensor(a[0], "cache");
        const Place place(cache, a[6]);
        place.uses(cache, "cache");
        no_gradient(cache, "cache");
        apart(cache, "cache");
        if (cache.dim() < 4) raise("cache must be [caches, num_blocks, block_size, ...]");
        int64_t row = 1;
        for (int64_t i = cache.dim() - 1; i >= 3; --i) {
            if (cache.size(i) > 1 && cache.stride(i) != row) raise("the entries of a slot of cache must be contiguous");
            row *= cache.size(i);
        }
        const at::Tensor &lengths = cuda_tensor(a[3], "lengths");
        const int64_t B = ints(a[3], "lengths", place).numel(), esz = cache.element_size();
        SpecCommit s = {};
        int64_t N;
        s.topo_seq_stride = tree_of(a[2], place, B, &N, &s.parent);
        const Table table = table_of(a[4], place, B);
        s.B = small(B, "B"); s.N = small(N, "N"); s.caches = small(cache.size(0), "caches");
        s.num_blocks = small(cache.size(1), "num_blocks"); s.block_size = small(cache.size(2), "block_size"); s.table_width = table.width;
        s.cache = cache.data_ptr(); s.row_bytes = row * esz;
        for (int i = 0; i < 3; ++i) s.stride[i] = cache.size(i) > 1 ? cache.stride(i) * esz : 0;
        s.block_table = table.ptr; s.table_stride = table.stride;
        s.lengths = int_ptr(lengths); s.accepted_node = int_ptr(ints(a[1], "accepted_node", place, B));
        s.n_nodes = a[5] == Py_None ? nullptr : int_ptr(ints(a[5], "n_nodes", place, B));
        Pieces made(place, {B, B});
        const at::Tensor t[2] = {made.take({B}), made.take({B})};
        s.lengths_out = int_ptr(t[0]); s.status = int_ptr(t[1]);
        check(unlocked([&] { return step_lib.commit(&s, place.stream()); }), "spec_cache_commit");
        written(cache);
        return result(commit_outputs_class, t, 2);
    });
}

// verify_probs(target_probs, draft_probs, token, cu_drafts, u_accept, u_bonus, max_drafts, stream)
PyObject *py_chains(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!arity(n, 8)) return nullptr;
    return guarded([&]() -> PyObject * {
        need((void *)step_lib.probs);
        const at::Tensor &p = cuda_tensor(a[0], "target_probs");
        const Place place(p, a[7]);
        const auto type = p.scalar_type();
        if (type != at::kFloat && type != at::kBFloat16) raise("target_probs must be float32 or bfloat16");
        rows_of(p, "target_probs", 2, type, place);
        const at::Tensor &token = ints(a[2], "token", place), &cu = ints(a[3], "cu_drafts", place);
        const int64_t T = token.numel(), B = cu.numel() - 1, V = p.size(1);
        if (p.size(0) != T + B) raise("target_probs must have a row per draft and one more per request");
        SpecChains s = {};
        s.target_stride = p.size(0) > 1 ? p.stride(0) : V;
        s.draft_stride = V;
        if (a[1] != Py_None) {
            const at::Tensor &q = cuda_tensor(a[1], "draft_probs");
            rows_of(q, "draft_probs", 2, type, place);
            if (q.size(0) != T || q.size(1) != V) raise("draft_probs must have a row of target_probs' length per draft");
            s.draft_probs = q.data_ptr();
            if (T > 1) s.draft_stride = q.stride(0);
        }
        s.B = small(B, "B"); s.V = small(V, "V"); s.max_drafts = whole(a[6], "max_drafts"); s.dtype = element_type(type); s.n_drafts = T;
        s.target_probs = p.data_ptr();
        s.token = int_ptr(token); s.cu_drafts = int_ptr(cu);
        s.u_accept = (const float *)floats(a[4], "u_accept", place, T).data_ptr();
        s.u_bonus = (const float *)floats(a[5], "u_bonus", place, T + B).data_ptr();
        const int64_t out = (int64_t)(s.max_drafts < 0 ? 0 : s.max_drafts) + 1;
        Pieces made(place, {B, B * out, B, B});
        const at::Tensor t[4] = {made.take({B}), made.take({B, out}), made.take({B}), made.take({B})};
        s.accept_len = int_ptr(t[0]); s.out_tokens = int_ptr(t[1]); s.bonus_token = int_ptr(t[2]); s.status = int_ptr(t[3]);
        check(unlocked([&] { return step_lib.probs(&s, place.stream()); }), "spec_verify_probs");
        return result(chain_outputs_class, t, 4);
    });
}

// init_step(path of libspecverify.so, SlotOutputs, AttentionOutputs, CommitOutputs, ChainOutputs): the entry points above
PyObject *py_init_step(PyObject *, PyObject *args)
{
    const char *path;
    PyObject *c[4];
    if (!PyArg_ParseTuple(args, "sOOOO", &path, &c[0], &c[1], &c[2], &c[3])) return nullptr;
    void *h = dlopen(path, RTLD_NOW | RTLD_LOCAL);
    if (!h) return PyErr_Format(PyExc_RuntimeError, "%s", dlerror());
    const auto find = [&](auto &f, const char *name) { f = reinterpret_cast<std::remove_reference_t<decltype(f)>>(dlsym(h, name)); };
    find(step_lib.slots, "spec_cache_slots");
    find(step_lib.norm_rope, "spec_norm_rope_cache");
    find(step_lib.attention_bytes, "spec_tree_attention_workspace_bytes");
    find(step_lib.attention, "spec_tree_attention");
    find(step_lib.commit, "spec_cache_commit");
    find(step_lib.probs, "spec_verify_probs");
    slot_outputs_class = Py_NewRef(c[0]);
    attention_outputs_class = Py_NewRef(c[1]);
    commit_outputs_class = Py_NewRef(c[2]);
    chain_outputs_class = Py_NewRef(c[3]);
    Py_RETURN_NONE;
}

// ---- shared prefixes, bounded caches, and what a service answers with ----------------------------------------------------------------------------
struct ServeLibrary {
    decltype(&spec_prefix_attention_workspace_bytes) prefix_bytes;
    decltype(&spec_prefix_attention) prefix;
    decltype(&spec_token_logprobs) logprobs;
    decltype(&spec_cache_weights_workspace_bytes) weights_bytes;
    decltype(&spec_cache_weights) weights;
    decltype(&spec_cache_evict_workspace_bytes) evict_bytes;
    decltype(&spec_cache_evict) evict;
} serve_lib;
PyObject *logprob_outputs_class, *evict_outputs_class;

// logprobs(logits, tokens, accepted_node, parent, temperature, top, stream): rows as they are where parent is None
PyObject *py_logprobs(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!arity(n, 7)) return nullptr;
    return guarded([&]() -> PyObject * {
        need((void *)serve_lib.logprobs);
        const at::Tensor &z = cuda_tensor(a[0], "logits");
        const Place place(z, a[6]);
        const auto type = z.scalar_type();
        if (element_type(type) < 0) raise("logits must be float32, bfloat16 or float16");
        const bool path = a[3] != Py_None;
        if (z.dim() != 2 && z.dim() != 3) raise("logits must be [R,V] or [B,N,V]");
        if (path && z.dim() != 3) raise("logits must be [B,N,V]");
        rows_of(z, "logits", (int)z.dim(), type, place);
        no_gradient(z, "logits");
        const int64_t B = z.size(0), N = z.dim() == 3 ? z.size(1) : 1, V = z.size(-1);
        const at::Tensor &token = ints(a[1], "tokens", place);
        SpecLogprobs s = {};
        std::vector<int64_t> rows(z.sizes().begin(), z.sizes().end() - 1), given = rows, best = rows;
        const int64_t lead = (int64_t)rows.size();
        if (token.dim() < lead || token.dim() > lead + 1 || !std::equal(rows.begin(), rows.end(), token.sizes().begin()))
            raise("tokens must have an entry, or a list of entries, per row of logits");
        if (path && token.dim() != 2) raise("tokens must be [B,N]");
        const int64_t K = token.dim() == lead ? 1 : token.size(lead);
        if (token.dim() > lead) given.push_back(K);
        s.B = small(B, "B"); s.N = small(N, "N"); s.V = small(V, "V"); s.K = small(K, "K"); s.top = whole(a[5], "top");
        s.dtype = element_type(type);
        s.logits = z.data_ptr();
        s.seq_stride = B > 1 ? z.stride(0) : 0;
        s.node_stride = N > 1 ? z.stride(1) : 0;
        s.token = int_ptr(token);
        s.temperature = (float)number(a[4]);
        if (path) {
            int64_t nodes;
            s.topo_seq_stride = tree_of(a[3], place, B, &nodes, &s.parent);
            if (nodes != N) raise("logits must be [B,N,V] with the N of parent");
            s.accepted_node = int_ptr(ints(a[2], "accepted_node", place, B));
        }
        best.push_back(std::clamp(s.top, 0, SPEC_MAX_TOP));        // (more is refused below)
        at::Tensor t[5];
        t[0] = place.fresh(given, at::kFloat);
        t[1] = place.fresh(rows, at::kFloat);
        if (s.top > 0) { t[2] = place.fresh(best, at::kInt); t[3] = place.fresh(best, at::kFloat); }
        t[4] = place.fresh(rows, at::kInt);
        s.logprob = (float *)t[0].data_ptr(); s.entropy = (float *)t[1].data_ptr(); s.status = int_ptr(t[4]);
        if (s.top > 0) { s.top_tokens = int_ptr(t[2]); s.top_logprobs = (float *)t[3].data_ptr(); }
        if (B * N) check(unlocked([&] { return serve_lib.logprobs(&s, place.stream()); }), "spec_token_logprobs");
        return result(logprob_outputs_class, t, 5);
    });
}

// a stack of caches [caches, num_blocks, block_size, ...] that the call writes: bytes of a row
int64_t stack_of(const at::Tensor &cache, const Place &place, int64_t (&stride)[3])
{
    place.uses(cache, "cache");
    no_gradient(cache, "cache");
    apart(cache, "cache");
    if (cache.dim() < 4) raise("cache must be [caches, num_blocks, block_size, ...]");
    int64_t row = 1;
    for (int64_t i = cache.dim() - 1; i >= 3; --i) {
        if (cache.size(i) > 1 && cache.stride(i) != row) raise("the entries of a slot of cache must be contiguous");
        row *= cache.size(i);
    }
    const int64_t esz = cache.element_size();
    for (int i = 0; i < 3; ++i) stride[i] = cache.size(i) > 1 ? cache.stride(i) * esz : 0;
    return row * esz;
}
// weights of entries, [num_blocks, block_size]
float *entry_weights(PyObject *o, const Place &place, int64_t blocks, int64_t block)
{
    const at::Tensor &t = cuda_tensor(o, "weights");
    check_vector(t, "weights", at::kFloat, "torch.float32");
    if (t.dim() != 2 || t.size(0) != blocks || t.size(1) != block) raise("weights must be [num_blocks, block_size]");
    no_gradient(t, "weights");
    place.uses(t, "weights");
    return (float *)t.data_ptr();
}

// cache_weights(weights, q, k_cache, lse, block_table, lengths, parent, n_nodes, scale, protected, fresh, stream)
PyObject *py_weights(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!arity(n, 12)) return nullptr;
    return guarded([&]() -> PyObject * {
        need((void *)serve_lib.weights);
        const at::Tensor &q = cuda_tensor(a[1], "q"), &kc = cuda_tensor(a[2], "k_cache");
        const Place place(q, a[11]);
        const auto type = q.scalar_type();
        if (type != at::kBFloat16 && type != at::kHalf) raise("q must be bfloat16 or float16");
        rows_of(q, "q", 4, type, place);
        rows_of(kc, "k_cache", 4, type, place);
        no_gradient(q, "q"); no_gradient(kc, "k_cache");
        const int64_t B = q.size(0), Hq = q.size(2), D = q.size(3);
        if (kc.size(3) != D) raise("the cache must be [num_blocks, block_size, Hkv, D]");
        SpecWeights s = {};
        int64_t N;
        s.topo_seq_stride = tree_of(a[6], place, B, &N, &s.parent);
        if (N != q.size(1)) raise("q must be [B,N,Hq,D] with the N of parent");
        const Table table = table_of(a[4], place, B);
        s.B = small(B, "B"); s.N = small(N, "N"); s.Hq = small(Hq, "Hq"); s.Hkv = small(kc.size(2), "Hkv"); s.D = small(D, "D");
        s.dtype = element_type(type);
        s.num_blocks = small(kc.size(0), "num_blocks"); s.block_size = small(kc.size(1), "block_size"); s.table_width = table.width;
        s.scale = a[8] == Py_None ? (float)(1.0 / std::sqrt((double)(D > 0 ? D : 1))) : (float)number(a[8]);
        s.fresh = truth(a[10]);
        s.block_table = table.ptr; s.table_stride = table.stride;
        s.lengths = int_ptr(ints(a[5], "lengths", place, B));
        s.n_nodes = a[7] == Py_None ? nullptr : int_ptr(ints(a[7], "n_nodes", place, B));
        s.protected_len = a[9] == Py_None ? nullptr : int_ptr(ints(a[9], "protected", place, B));
        const at::Tensor &lse = floats(a[3], "lse", place, B * N * Hq);
        no_gradient(lse, "lse");
        s.lse = (const float *)lse.data_ptr();
        s.weights = entry_weights(a[0], place, kc.size(0), kc.size(1));
        s.q = q.data_ptr(); s.k_cache = kc.data_ptr();
        strides_of(q, s.q_stride); strides_of(kc, s.k_cache_stride);
        const at::Tensor status = place.fresh({B}, at::kInt);
        s.status = int_ptr(status);
        int64_t bytes = 0;
        check(serve_lib.weights_bytes(&s, &bytes), "spec_cache_weights_workspace_bytes");
        const at::Tensor ws = empty({bytes}, at::kByte, place.device());         // (of this call alone)
        check(unlocked([&] { return serve_lib.weights(&s, ws.data_ptr(), bytes, place.stream()); }), "spec_cache_weights");
        written(THPVariable_Unpack(a[0]));
        return THPVariable_Wrap(status);
    });
}

// cache_evict(cache, weights, lengths, block_table, owned, free_blocks, free_range, budget, recent, protected, stream)
PyObject *py_evict(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!arity(n, 11)) return nullptr;
    return guarded([&]() -> PyObject * {
        need((void *)serve_lib.evict);
        const at::Tensor &cache = cuda_tensor(a[0], "cache");
        const Place place(cache, a[10]);
        SpecEvict s = {};
        s.row_bytes = stack_of(cache, place, s.stride);
        s.caches = small(cache.size(0), "caches"); s.num_blocks = small(cache.size(1), "num_blocks"); s.block_size = small(cache.size(2), "block_size");
        s.weights = entry_weights(a[1], place, cache.size(1), cache.size(2));
        const at::Tensor &lengths = cuda_tensor(a[2], "lengths");
        const int64_t B = ints(a[2], "lengths", place).numel();
        const Table table = table_of(a[3], place, B);
        const at::Tensor &ring = ints(a[5], "free_blocks", place);
        apart(ring, "free_blocks");
        s.B = small(B, "B"); s.budget = whole(a[7], "budget"); s.recent = whole(a[8], "recent");
        s.table_width = table.width; s.block_table = table.ptr; s.table_stride = table.stride;
        s.cache = cache.data_ptr();
        s.lengths = int_ptr(lengths); s.owned = int_ptr(ints(a[4], "owned", place, B));
        s.protected_len = a[9] == Py_None ? nullptr : int_ptr(ints(a[9], "protected", place, B));
        s.free_blocks = int_ptr(ring); s.free_size = small(ring.numel(), "free_blocks");
        s.free_range = int_ptr(ints(a[6], "free_range", place, 2));
        Pieces made(place, {B, B, 2, B});
        const at::Tensor t[4] = {made.take({B}), made.take({B}), made.take({2}), made.take({B})};
        s.lengths_out = int_ptr(t[0]); s.owned_out = int_ptr(t[1]); s.free_range_out = int_ptr(t[2]); s.status = int_ptr(t[3]);
        int64_t bytes = 0;
        check(serve_lib.evict_bytes(&s, &bytes), "spec_cache_evict_workspace_bytes");
        const at::Tensor ws = empty({bytes}, at::kByte, place.device());         // (of this call alone)
        check(unlocked([&] { return serve_lib.evict(&s, ws.data_ptr(), bytes, place.stream()); }), "spec_cache_evict");
        written(cache); written(THPVariable_Unpack(a[1])); written(ring);
        return result(evict_outputs_class, t, 4);
    });
}

// prefix_attention(q, k_cache, v_cache, block_table, lengths, parent, n_nodes, plan, scale, out, want_lse, stream); plan: a tuple of group, members,
// first, place, blocks and table
PyObject *py_prefix(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!arity(n, 12)) return nullptr;
    return guarded([&]() -> PyObject * {
        need((void *)serve_lib.prefix);
        const Place place(cuda_tensor(a[0], "q"), a[11]);
        if (!PyTuple_Check(a[7]) || PyTuple_GET_SIZE(a[7]) != 6) raise("plan must be a PrefixPlan");
        PyObject *part[6];
        for (int i = 0; i < 6; ++i) part[i] = PyTuple_GET_ITEM(a[7], i);
        at::Tensor t[3];
        SpecPrefixAttention s = {};
        s.attention = attention_of(a, a[8], a[9], a[10], place, t);
        const int64_t B = s.attention.B;
        s.group = int_ptr(ints(part[0], "plan.group", place, B));
        const at::Tensor &members = ints(part[1], "plan.members", place), &blocks = ints(part[4], "plan.blocks", place);
        const int64_t groups = blocks.numel();
        s.members = int_ptr(members);
        s.first = int_ptr(ints(part[2], "plan.first", place, groups + 1));
        s.place = int_ptr(ints(part[3], "plan.place", place, B));
        s.shared_blocks = int_ptr(blocks);
        const at::Tensor &table = cuda_tensor(part[5], "plan.table");
        if (table.scalar_type() != at::kInt || table.dim() != 2 || table.size(0) != groups || (table.size(1) > 1 && table.stride(1) != 1))
            raise("plan.table must be a [groups,W] torch.int32 tensor with contiguous rows");
        place.uses(table, "plan.table");
        s.prefix_table = int_ptr(table);
        s.n_groups = small(groups, "groups"); s.n_members = small(members.numel(), "members"); s.prefix_width = small(table.size(1), "the plan's width");
        s.prefix_stride = groups > 1 ? table.stride(0) : std::max<int64_t>(table.size(1), 1);
        int64_t bytes = 0;
        check(serve_lib.prefix_bytes(&s, &bytes), "spec_prefix_attention_workspace_bytes");
        const at::Tensor ws = empty({bytes}, at::kByte, place.device());         // (of this call alone)
        check(unlocked([&] { return serve_lib.prefix(&s, ws.data_ptr(), bytes, place.stream()); }), "spec_prefix_attention");
        if (a[9] != Py_None) written(t[0]);
        return result(attention_outputs_class, t, 3);
    });
}

// init_serve(path of libspecverify.so, LogprobOutputs, EvictOutputs): the entry points above
PyObject *py_init_serve(PyObject *, PyObject *args)
{
    const char *path;
    PyObject *c[2];
    if (!PyArg_ParseTuple(args, "sOO", &path, &c[0], &c[1])) return nullptr;
    void *h = dlopen(path, RTLD_NOW | RTLD_LOCAL);
    if (!h) return PyErr_Format(PyExc_RuntimeError, "%s", dlerror());
    const auto find = [&](auto &f, const char *name) { f = reinterpret_cast<std::remove_reference_t<decltype(f)>>(dlsym(h, name)); };
    find(serve_lib.prefix_bytes, "spec_prefix_attention_workspace_bytes");
    find(serve_lib.prefix, "spec_prefix_attention");
    find(serve_lib.logprobs, "spec_token_logprobs");
    find(serve_lib.weights_bytes, "spec_cache_weights_workspace_bytes");
    find(serve_lib.weights, "spec_cache_weights");
    find(serve_lib.evict_bytes, "spec_cache_evict_workspace_bytes");
    find(serve_lib.evict, "spec_cache_evict");
    logprob_outputs_class = Py_NewRef(c[0]);
    evict_outputs_class = Py_NewRef(c[1]);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"init", py_init, METH_VARARGS, nullptr},
    {"verify", (PyCFunction)(void *)py_verify, METH_FASTCALL, nullptr},
    {"tree_analysis", (PyCFunction)(void *)py_analysis, METH_FASTCALL, nullptr},
    {"tree_probs", (PyCFunction)(void *)py_probs, METH_FASTCALL, nullptr},
    {"sample_bonus", (PyCFunction)(void *)py_bonus, METH_FASTCALL, nullptr},
    {"launch", (PyCFunction)(void *)py_launch, METH_FASTCALL, nullptr},
    {"init_step", py_init_step, METH_VARARGS, nullptr},
    {"cache_slots", (PyCFunction)(void *)py_slots, METH_FASTCALL, nullptr},
    {"norm_rope_cache", (PyCFunction)(void *)py_norm_rope, METH_FASTCALL, nullptr},
    {"tree_attention", (PyCFunction)(void *)py_attention, METH_FASTCALL, nullptr},
    {"cache_commit", (PyCFunction)(void *)py_commit, METH_FASTCALL, nullptr},
    {"verify_probs", (PyCFunction)(void *)py_chains, METH_FASTCALL, nullptr},
    {"init_serve", py_init_serve, METH_VARARGS, nullptr},
    {"logprobs", (PyCFunction)(void *)py_logprobs, METH_FASTCALL, nullptr},
    {"prefix_attention", (PyCFunction)(void *)py_prefix, METH_FASTCALL, nullptr},
    {"cache_weights", (PyCFunction)(void *)py_weights, METH_FASTCALL, nullptr},
    {"cache_evict", (PyCFunction)(void *)py_evict, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_torch_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__torch_calls(void) { return PyModule_Create(&module_def); }
