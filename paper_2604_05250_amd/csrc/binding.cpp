// Native argument marshalling of the Python binding: torch tensors in, one C-ABI call (include/dd.h), torch tensors out.
//
// No step of the computation is here.  Per call: shapes, types and placement are checked, missing outputs are
// allocated, the scratch tensor of (device, stream) is looked up and the library is called on torch's current stream.
// It is native because the small calls of a cycle are shorter than their marshalling was: through ctypes a drafter call cost
// the host 13.7 us, an unmasking step 14.5 us (attribute reads on eight tensors, three allocations through Python, twenty
// converted arguments), for 9-12 us of GPU work; here 6.1 and 7.7 us, most of it the launches.  A whole cycle on one sequence
// of 512 positions (18 calls), host bound before, went from 268 to 211 us.
//
// Every function takes positional arguments only (the Python wrappers own names and defaults), absent tensors as None,
// absent dtype tags as None, and raises what the wrappers' documentation says: ValueError for a bad shape or placement,
// TypeError for a bad element type, the registered error class for a status of the library, torch's own classes for what
// torch throws (torch.OutOfMemoryError when an output or the scratch memory cannot be allocated).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/hip/EmptyTensor.h>
#include <ATen/record_function.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/hip/HIPGraphsC10Utils.h>
#include <c10/hip/HIPGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <map>
#include <mutex>
#include <utility>

#include "../../include/dd.h"

namespace {

struct Raised {};                                            // a Python exception is set

[[noreturn]] void value_error(const char *what, const char *msg)
{
    PyErr_Format(PyExc_ValueError, "%s%s%s", what, *what ? ": " : "", msg);
    throw Raised{};
}

const at::Tensor *opt_tensor(PyObject *o, const char *what)
{
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s: a tensor is required", what);
        throw Raised{};
    }
    return &THPVariable_Unpack(o);
}
const at::Tensor &tensor(PyObject *o, const char *what)
{
    const at::Tensor *t = opt_tensor(o, what);
    if (t == nullptr) {
        PyErr_Format(PyExc_TypeError, "%s: a tensor is required", what);
        throw Raised{};
    }
    return *t;
}
// int(o), and the value as a C int (its low bits, as through ctypes)
int integer(PyObject *o)
{
    PyObject *n = PyNumber_Long(o);
    if (n == nullptr) throw Raised{};
    const unsigned long v = PyLong_AsUnsignedLongMask(n);
    Py_DECREF(n);
    return (int)(unsigned)v;
}
// float(o)
double real(PyObject *o)
{
    PyObject *n = PyNumber_Float(o);
    if (n == nullptr) throw Raised{};
    const double v = PyFloat_AS_DOUBLE(n);
    Py_DECREF(n);
    return v;
}
// an integer as it stands: a float is refused, with the error ctypes has for it
PyObject *exact_integer(PyObject *o, const char *what)
{
    PyObject *n = PyNumber_Index(o);
    if (n != nullptr) return n;
    PyErr_Clear();
    PyObject *ctypes = PyImport_ImportModule("ctypes"), *cls = ctypes ? PyObject_GetAttrString(ctypes, "ArgumentError") : nullptr;
    if (cls != nullptr) PyErr_Format(cls, "%s: an integer is required, not %s", what, Py_TYPE(o)->tp_name);
    Py_XDECREF(cls);
    Py_XDECREF(ctypes);
    throw Raised{};
}

// device pointer of a tensor in GPU memory (nullptr for an absent one)
void *dev(const at::Tensor *t, const char *what)
{
    if (t == nullptr) return nullptr;
    if (!t->is_cuda()) value_error(what, "must live in GPU memory");
    if (!t->is_contiguous()) value_error(what, "must be contiguous");
    return t->data_ptr();
}
void *dev(const at::Tensor &t, const char *what) { return dev(&t, what); }

int dtype_tag(const at::Tensor &t, const char *what)
{
    switch (t.scalar_type()) {
    case at::kFloat: return DD_F32;
    case at::kBFloat16: case at::kShort: case at::kUInt16: return DD_BF16;
    case at::kByte: case at::kFloat8_e4m3fn: return DD_FP8_E4M3;
    default:
        PyErr_Format(PyExc_TypeError, "%s: unsupported tensor dtype %s", what, c10::toString(t.scalar_type()));
        throw Raised{};
    }
}
int tag_or(PyObject *given, const at::Tensor &t, const char *what)
{
    if (given == Py_None) return dtype_tag(t, what);
    PyObject *n = exact_integer(given, "dtype tag");
    const unsigned long v = PyLong_AsUnsignedLongMask(n);
    Py_DECREF(n);
    return (int)(unsigned)v;                                  // (the library refuses what is no tag)
}
// B and G of a verification or unmasking call, whose logits have P rows
std::pair<int64_t, int64_t> batch_and_rows(PyObject *pb, PyObject *pg, int64_t P, const char *rows_msg)
{
    long long v[2];
    PyObject *const o[2] = {pb, pg};
    bool fits = true;
    for (int i = 0; i < 2; ++i) {
        PyObject *n = exact_integer(o[i], i == 0 ? "B" : "G");
        int over = 0;
        v[i] = PyLong_AsLongLongAndOverflow(n, &over);
        Py_DECREF(n);
        fits = fits && over == 0;
    }
    if (!fits || (__int128)v[0] * v[1] != P) value_error("", rows_msg);
    return {v[0], v[1]};
}
void one_byte(const at::Tensor &t, const char *what, const char *msg)
{
    if (t.element_size() != 1) {
        PyErr_Format(PyExc_TypeError, "%s: %s", what, msg);
        throw Raised{};
    }
}
// Shapes say how many elements the library reads and writes, dtype tags how large they are: a tensor that holds fewer bytes
// than that never gets to a launch.
int64_t tag_bytes(int tag) { return tag == DD_F32 ? 4 : tag == DD_BF16 ? 2 : tag == DD_FP8_E4M3 ? 1 : 0; }
// A tensor of floating-point numbers has to be of the tag's kind (fp16 has bf16's width, e5m2 has e4m3's); integers are taken as the bits.
void elements_of(const at::Tensor *t, int tag, const char *what)
{
    if (t == nullptr || tag_bytes(tag) == 0) return;         // (no tag: the library refuses it)
    const at::ScalarType kind = tag == DD_F32 ? at::kFloat : tag == DD_BF16 ? at::kBFloat16 : at::kFloat8_e4m3fn;
    if ((int64_t)t->element_size() != tag_bytes(tag))
        PyErr_Format(PyExc_TypeError, "%s: elements of %lld bytes expected, has %s", what, (long long)tag_bytes(tag), c10::toString(t->scalar_type()));
    else if (t->scalar_type() != kind && !at::isIntegralType(t->scalar_type(), true))
        PyErr_Format(PyExc_TypeError, "%s: %s expected, has %s", what, c10::toString(kind), c10::toString(t->scalar_type()));
    else
        return;
    throw Raised{};
}
void room_for(const at::Tensor *t, int64_t elements, int64_t bytes_each, const char *what)
{
    if (t == nullptr || (__int128)t->numel() * t->element_size() >= (__int128)elements * bytes_each) return;
    PyErr_Format(PyExc_ValueError, "%s: too small for %lld elements of %lld bytes", what, (long long)elements, (long long)bytes_each);
    throw Raised{};
}
int64_t out_bytes(int v_tag) { return v_tag == DD_F32 ? 4 : 2; }
// per-head scales
void scales_of(const at::Tensor *t, int64_t heads, const char *what)
{
    if (t == nullptr) return;
    if (t->scalar_type() != at::kFloat) {
        PyErr_Format(PyExc_TypeError, "%s: float32 expected, has %s", what, c10::toString(t->scalar_type()));
        throw Raised{};
    }
    room_for(t, heads, 4, what);
}
bool has_shape(const at::Tensor &t, std::initializer_list<int64_t> s) { return t.sizes() == at::IntArrayRef(s.begin(), s.size()); }

// a per-position vector: n elements of the given type
void check_vec(const at::Tensor *t, int64_t n, at::ScalarType type, const char *what)
{
    if (t == nullptr || (t->scalar_type() == type && t->numel() == n)) return;
    PyErr_Format(PyExc_ValueError, "%s: must have %lld elements of %s, has %lld of %s", what, (long long)n, c10::toString(type),
                 (long long)t->numel(), c10::toString(t->scalar_type()));
    throw Raised{};
}

PyObject *error_class = nullptr;                             // DDError(status, where)
void check(int rc, const char *where)
{
    if (rc == 0) return;
    PyObject *e = error_class ? PyObject_CallFunction(error_class, "is", rc, where) : nullptr;
    if (e != nullptr) {
        PyErr_SetObject(error_class, e);
        Py_DECREF(e);
    } else if (!PyErr_Occurred()) {
        PyErr_Format(PyExc_RuntimeError, "%s: status %d", where, rc);
    }
    throw Raised{};
}

hipStream_t current_stream() { return c10::hip::getCurrentHIPStream().stream(); }

// ---- scratch memory: one tensor per (device, stream) - calls on one stream run in order and may share it, calls on
// different streams may overlap and must not - or the one a fixed_workspace() block of this thread has set.  Guarded by the interpreter
// lock; never destroyed (the runtime may be gone by then).
// A call that uses it can be several launches, of which the later ones read what the first one left there, and it is made without the
// interpreter lock.  So that no other thread's launches on the stream come in between, each scratch tensor has a lock of its own, held
// from a call's first launch to its last, and taken only without the interpreter lock.
struct Scratch {
    struct Held { at::Tensor memory; std::mutex launches; };
    std::map<std::pair<int, hipStream_t>, Held> by_stream;
    std::mutex fixed_launches, static_launches;              // of calls in fixed workspaces, and of those that use the library's own array
};
Scratch &scratch()
{
    static Scratch *s = new Scratch;
    return *s;
}
// What a thread has set, and the most that its calls have asked for: its own, so that one that captures a graph neither lends its
// scratch tensor to the calls of others nor takes their needs for its own.  (A pointer, as nothing may be freed when a thread ends late.)
thread_local at::Tensor *fixed = nullptr;
thread_local size_t peak = 0;
struct Workspace { at::Tensor memory; std::mutex *launches = nullptr; };
// (`or_less`: the library itself says whether a fixed workspace of fewer bytes serves the call)
Workspace workspace(size_t nbytes, const at::Device &device, hipStream_t stream, bool or_less)
{
    if (nbytes == 0) return {};
    if (nbytes > peak) peak = nbytes;
    if (fixed != nullptr) {
        if (((size_t)fixed->numel() < nbytes && !or_less) || fixed->device() != device) {
            PyErr_Format(PyExc_RuntimeError, "the fixed workspace holds %lld bytes on %s; this call needs %zu on %s",
                         (long long)fixed->numel(), fixed->device().str().c_str(), nbytes, device.str().c_str());
            throw Raised{};
        }
        return {*fixed, &scratch().fixed_launches};
    }
    if (c10::hip::currentStreamCaptureStatusMayInitCtx() != c10::hip::CaptureStatus::None) {
        // memory allocated under capture would come from that graph's private pool and a cached tensor of it
        // could be handed to a later, unrelated call: the scratch memory of captured calls is allocated beforehand
        PyErr_SetString(PyExc_RuntimeError,
                        "a call that needs scratch memory is being captured without a fixed workspace: "
                        "capture through paper_2604_05250_amd.step.capture_step, or inside fixed_workspace()");
        throw Raised{};
    }
    Scratch::Held &h = scratch().by_stream[{device.index(), stream}];
    if (!h.memory.defined() || (size_t)h.memory.numel() < nbytes)
        h.memory = at::empty({(int64_t)(nbytes > (1u << 20) ? nbytes : (1u << 20))}, at::TensorOptions().dtype(at::kByte).device(device));
    return {h.memory, &h.launches};
}

template <typename F> int unlocked(F &&f, std::mutex *launches = nullptr)      // the library call itself runs without the interpreter lock
{
    int rc;
    Py_BEGIN_ALLOW_THREADS
    if (launches != nullptr) {
        const std::lock_guard<std::mutex> whole(*launches);
        rc = f();
    } else {
        rc = f();
    }
    Py_END_ALLOW_THREADS
    return rc;
}
struct Call {                                                // one library call: stream, scratch
    hipStream_t stream;
    Workspace ws;
    Call(size_t need, const at::Tensor &on, bool or_less = false) : stream(current_stream()), ws(workspace(need, on.device(), stream, or_less)) {}
    void *ptr() const { return ws.memory.defined() ? ws.memory.data_ptr() : nullptr; }
    size_t bytes() const { return ws.memory.defined() ? (size_t)ws.memory.numel() : 0; }
    template <typename F> int run(F &&f) const { return unlocked(f, ws.launches); }
};

// An output.  The allocator is asked directly, past the dispatcher (a cycle of ten calls in fp32 51.1 -> 47.5 us on the host's side, 59.5 -> 56.1
// where it is slower), unless something may be listening there: a dispatch mode, tracer or transform (each adds keys to this thread's
// set), a profiler or another observer of calls, or the fill of uninitialised memory in deterministic mode.  Device, stream, capture pool
// and inference mode are the same either way.
at::Tensor empty_like_type(at::IntArrayRef shape, at::ScalarType type, const at::Tensor &on)
{
    const bool heard = !(c10::impl::tls_local_dispatch_key_set().included_ - c10::default_included_set).empty() || at::hasCallbacks() ||
                       at::globalContext().deterministicAlgorithms();
    if (heard) return at::empty(shape, at::TensorOptions().dtype(type).device(on.device()));
    return at::detail::empty_cuda(shape, type, on.device(), std::nullopt);
}

void want(Py_ssize_t got, Py_ssize_t n)
{
    if (got == n) return;
    PyErr_Format(PyExc_TypeError, "%zd arguments expected, %zd given", n, got);
    throw Raised{};
}

// (Q, K, V, O, q_scale, k_scale, qk_dtype, v_dtype) -> O
PyObject *bidir(PyObject *const *a, Py_ssize_t n)
{
    want(n, 8);
    const at::Tensor &Q = tensor(a[0], "Q"), &K = tensor(a[1], "K"), &V = tensor(a[2], "V");
    const at::Tensor *O = opt_tensor(a[3], "O"), *qs = opt_tensor(a[4], "q_scale"), *ks = opt_tensor(a[5], "k_scale");
    if (Q.dim() != 4 || K.dim() != 4) value_error("", "Q, K, V must have four dimensions");
    const int64_t B = Q.size(0), H = Q.size(1), N = Q.size(2), d = Q.size(3), Hkv = K.size(1);
    if (!has_shape(K, {B, Hkv, N, d}) || !has_shape(V, {B, Hkv, N, d})) value_error("", "K/V shape must be [B,Hkv,N,d] matching Q");
    const int qk = tag_or(a[6], Q, "Q"), vd = tag_or(a[7], V, "V");
    elements_of(&Q, qk, "Q"); elements_of(&K, qk, "K"); elements_of(&V, vd, "V");
    room_for(O, B * H * N * d, out_bytes(vd), "O");
    scales_of(qs, B * H, "q_scale"); scales_of(ks, B * Hkv, "k_scale");
    void *const q = dev(Q, "Q"), *const k = dev(K, "K"), *const v = dev(V, "V");
    const at::Tensor out = O ? *O : empty_like_type({B, H, N, d}, V.scalar_type(), V);
    void *const o = dev(out, "O");
    const float *q_s = (const float *)dev(qs, "q_scale"), *k_s = (const float *)dev(ks, "k_scale");
    const Call c(dd_bidir_attention_workspace_bytes(B, H, Hkv, N, d, (dd_dtype)qk, (dd_dtype)vd), Q);
    check(c.run([&] { return dd_bidir_attention(q, k, v, o, B, H, Hkv, N, d, (dd_dtype)qk, (dd_dtype)vd, q_s, k_s, c.ptr(),
                                                   c.bytes(), c.stream); }), "dd_bidir_attention");
    return THPVariable_Wrap(out);
}

enum { kCached = 0, kRefresh = 1, kWindow = 2, kBatched = 3 };
// (kind, Qblk, Kc, Vc, block_start | block_starts, win_start, win_len, O, Kblk, Vblk, q_scale, k_scale, qk_dtype, v_dtype) -> O
PyObject *block(PyObject *const *a, Py_ssize_t n)
{
    want(n, 14);
    const int kind = integer(a[0]);
    const at::Tensor &Q = tensor(a[1], "Qblk"), &Kc = tensor(a[2], "Kc"), &Vc = tensor(a[3], "Vc");
    const at::Tensor *O = opt_tensor(a[7], "O"), *Kb = opt_tensor(a[8], "Kblk"), *Vb = opt_tensor(a[9], "Vblk");
    const at::Tensor *qs = opt_tensor(a[10], "q_scale"), *ks = opt_tensor(a[11], "k_scale");
    if (Q.dim() != 4 || Kc.dim() != 4) value_error("", "Qblk, Kc, Vc must have four dimensions");
    const int64_t B = Q.size(0), H = Q.size(1), bl = Q.size(2), d = Q.size(3), Hkv = Kc.size(1), N = Kc.size(2);
    if (!has_shape(Kc, {B, Hkv, N, d}) || !has_shape(Vc, {B, Hkv, N, d})) value_error("", "Kc/Vc shape must be [B,Hkv,N,d]");
    if (kind == kBatched && (!Kb || !Vb)) value_error("", "Kblk and Vblk are required");
    if (Kb && !(has_shape(*Kb, {B, Hkv, bl, d}) && Vb && has_shape(*Vb, {B, Hkv, bl, d}))) value_error("", "Kblk/Vblk shape must be [B,Hkv,block_len,d]");
    const int qk = tag_or(a[12], Q, "Qblk"), vd = tag_or(a[13], Vc, "Vc");
    elements_of(&Q, qk, "Qblk"); elements_of(&Kc, qk, "Kc"); elements_of(&Vc, vd, "Vc");
    elements_of(Kb, qk, "Kblk"); elements_of(Vb, vd, "Vblk");
    room_for(O, B * H * bl * d, out_bytes(vd), "O");
    scales_of(qs, B * H, "q_scale"); scales_of(ks, B * Hkv, "k_scale");
    const at::Tensor *starts = nullptr;
    int bs = 0, ws0 = 0, wsn = 0;
    if (kind == kBatched) {
        starts = &tensor(a[4], "block_starts");
        if (starts->scalar_type() != at::kInt || starts->numel() != B) value_error("", "block_starts must be int32 with B entries");
    } else {
        bs = integer(a[4]);
    }
    if (kind == kWindow) {
        ws0 = integer(a[5]);
        wsn = integer(a[6]);
    }
    void *const q = dev(Q, "Qblk"), *const k = dev(Kc, "Kc"), *const v = dev(Vc, "Vc"), *const kb = dev(Kb, "Kblk"), *const vb = dev(Vb, "Vblk");
    const at::Tensor out = O ? *O : empty_like_type({B, H, bl, d}, Vc.scalar_type(), Vc);
    void *const o = dev(out, "O");
    const float *q_s = (const float *)dev(qs, "q_scale"), *k_s = (const float *)dev(ks, "k_scale");
    const int32_t *st = (const int32_t *)dev(starts, "block_starts");
    const dd_dtype tq = (dd_dtype)qk, tv = (dd_dtype)vd;
    const Call c(kind == kWindow ? dd_block_attention_window_workspace_bytes(bl, wsn, B, H, Hkv, N, d, tq, tv)
                                 : dd_block_attention_cached_workspace_bytes(bl, B, H, Hkv, N, d, tq, tv), Q);
    switch (kind) {
    case kCached:
        check(c.run([&] { return dd_block_attention_cached(q, k, v, o, bs, bl, kb, vb, B, H, Hkv, N, d, tq, tv, q_s, k_s, c.ptr(),
                                                              c.bytes(), c.stream); }), "dd_block_attention_cached");
        break;
    case kRefresh:
        check(c.run([&] { return dd_block_attention_refresh(q, k, v, o, bs, bl, kb, vb, B, H, Hkv, N, d, tq, tv, q_s, k_s, c.ptr(),
                                                               c.bytes(), c.stream); }), "dd_block_attention_refresh");
        break;
    case kWindow:
        check(c.run([&] { return dd_block_attention_window(q, k, v, o, bs, bl, ws0, wsn, kb, vb, B, H, Hkv, N, d, tq, tv, q_s, k_s,
                                                              c.ptr(), c.bytes(), c.stream); }), "dd_block_attention_window");
        break;
    default:
        check(c.run([&] { return dd_block_attention_batched(q, k, v, o, st, bl, kb, vb, B, H, Hkv, N, d, tq, tv, q_s, k_s, c.ptr(),
                                                               c.bytes(), c.stream); }), "dd_block_attention_batched");
    }
    return THPVariable_Wrap(out);
}

// (Q, K, V, q_scale, k_scale, v_scale, O) -> O
PyObject *bidir_fp8v(PyObject *const *a, Py_ssize_t n)
{
    want(n, 7);
    const at::Tensor &Q = tensor(a[0], "Q"), &K = tensor(a[1], "K"), &V = tensor(a[2], "V");
    const at::Tensor *qs = opt_tensor(a[3], "q_scale"), *ks = opt_tensor(a[4], "k_scale"), *vs = opt_tensor(a[5], "v_scale");
    const at::Tensor *O = opt_tensor(a[6], "O");
    if (Q.dim() != 4 || K.dim() != 4) value_error("", "Q, K, V must have four dimensions");
    const int64_t B = Q.size(0), H = Q.size(1), N = Q.size(2), d = Q.size(3), Hkv = K.size(1);
    if (!has_shape(K, {B, Hkv, N, d}) || !has_shape(V, {B, Hkv, N, d})) value_error("", "K/V shape must be [B,Hkv,N,d] matching Q");
    const char *msg = "one byte per element (e4m3 codes) expected";
    one_byte(Q, "Q", msg); one_byte(K, "K", msg); one_byte(V, "V", msg);
    room_for(O, B * H * N * d, 2, "O");
    scales_of(qs, B * H, "q_scale"); scales_of(ks, B * Hkv, "k_scale"); scales_of(vs, B * Hkv, "v_scale");
    void *const q = dev(Q, "Q"), *const k = dev(K, "K"), *const v = dev(V, "V");
    const at::Tensor out = O ? *O : empty_like_type({B, H, N, d}, at::kShort, V);
    void *const o = dev(out, "O");
    const float *q_s = (const float *)dev(qs, "q_scale"), *k_s = (const float *)dev(ks, "k_scale"), *v_s = (const float *)dev(vs, "v_scale");
    const hipStream_t stream = current_stream();
    check(unlocked([&] { return dd_bidir_attention_fp8v(q, k, v, o, B, H, Hkv, N, d, q_s, k_s, v_s, stream); }), "dd_bidir_attention_fp8v");
    return THPVariable_Wrap(out);
}

// (Q, Qs, K, Ks, V, Vs, O) -> O
PyObject *bidir_mx(PyObject *const *a, Py_ssize_t n)
{
    want(n, 7);
    const at::Tensor &Q = tensor(a[0], "Q"), &Qs = tensor(a[1], "Qs"), &K = tensor(a[2], "K"), &Ks = tensor(a[3], "Ks");
    const at::Tensor &V = tensor(a[4], "V"), &Vs = tensor(a[5], "Vs");
    const at::Tensor *O = opt_tensor(a[6], "O");
    if (Q.dim() != 4 || K.dim() != 4) value_error("", "Q, K, V must have four dimensions");
    const int64_t B = Q.size(0), H = Q.size(1), N = Q.size(2), d = Q.size(3), Hkv = K.size(1);
    if (!has_shape(K, {B, Hkv, N, d}) || !has_shape(V, {B, Hkv, N, d / 2})) value_error("", "K must be [B,Hkv,N,d] and V [B,Hkv,N,d/2] matching Q");
    if (!has_shape(Qs, {B, H, N, d / 32}) || !has_shape(Ks, {B, Hkv, N, d / 32}) || !has_shape(Vs, {B, Hkv, N, d / 32}))
        value_error("", "scales must be [..., d/32] matching their tensors");
    const char *msg = "one byte per entry expected";
    one_byte(Q, "Q", msg); one_byte(K, "K", msg); one_byte(V, "V", msg);
    one_byte(Qs, "Qs", msg); one_byte(Ks, "Ks", msg); one_byte(Vs, "Vs", msg);
    room_for(O, B * H * N * d, 2, "O");
    void *const q = dev(Q, "Q"), *const q_s = dev(Qs, "Qs"), *const k = dev(K, "K"), *const k_s = dev(Ks, "Ks"), *const v = dev(V, "V"), *const v_s = dev(Vs, "Vs");
    const at::Tensor out = O ? *O : empty_like_type({B, H, N, d}, at::kShort, V);
    void *const o = dev(out, "O");
    const hipStream_t stream = current_stream();
    check(unlocked([&] { return dd_bidir_attention_mx(q, q_s, k, k_s, v, v_s, o, B, H, Hkv, N, d, stream); }), "dd_bidir_attention_mx");
    return THPVariable_Wrap(out);
}

// (Qblk, Kc, Vc, block_start, q_scale, k_scale, v_scale, O, Kblk, Vblk) -> O
PyObject *block_fp8v(PyObject *const *a, Py_ssize_t n)
{
    want(n, 10);
    const at::Tensor &Q = tensor(a[0], "Qblk"), &Kc = tensor(a[1], "Kc"), &Vc = tensor(a[2], "Vc");
    const int bs = integer(a[3]);
    const at::Tensor *qs = opt_tensor(a[4], "q_scale"), *ks = opt_tensor(a[5], "k_scale"), *vs = opt_tensor(a[6], "v_scale");
    const at::Tensor *O = opt_tensor(a[7], "O"), *Kb = opt_tensor(a[8], "Kblk"), *Vb = opt_tensor(a[9], "Vblk");
    if (Q.dim() != 4 || Kc.dim() != 4) value_error("", "Qblk, Kc, Vc must have four dimensions");
    const int64_t B = Q.size(0), H = Q.size(1), bl = Q.size(2), d = Q.size(3), Hkv = Kc.size(1), N = Kc.size(2);
    if (!has_shape(Kc, {B, Hkv, N, d}) || !has_shape(Vc, {B, Hkv, N, d})) value_error("", "Kc/Vc shape must be [B,Hkv,N,d]");
    if (Kb && !(has_shape(*Kb, {B, Hkv, bl, d}) && Vb && has_shape(*Vb, {B, Hkv, bl, d}))) value_error("", "Kblk/Vblk shape must be [B,Hkv,block_len,d]");
    const char *msg = "one byte per element (e4m3 codes) expected";
    one_byte(Q, "Qblk", msg); one_byte(Kc, "Kc", msg); one_byte(Vc, "Vc", msg);
    if (Kb) { one_byte(*Kb, "Kblk", msg); one_byte(*Vb, "Vblk", msg); }
    room_for(O, B * H * bl * d, 2, "O");
    scales_of(qs, B * H, "q_scale"); scales_of(ks, B * Hkv, "k_scale"); scales_of(vs, B * Hkv, "v_scale");
    void *const q = dev(Q, "Qblk"), *const k = dev(Kc, "Kc"), *const v = dev(Vc, "Vc"), *const kb = dev(Kb, "Kblk"), *const vb = dev(Vb, "Vblk");
    const at::Tensor out = O ? *O : empty_like_type({B, H, bl, d}, at::kShort, Vc);
    void *const o = dev(out, "O");
    const float *q_s = (const float *)dev(qs, "q_scale"), *k_s = (const float *)dev(ks, "k_scale"), *v_s = (const float *)dev(vs, "v_scale");
    const Call c(dd_block_attention_cached_fp8v_workspace_bytes(bl, B, H, Hkv, N, d), Q);
    check(c.run([&] { return dd_block_attention_cached_fp8v(q, k, v, o, bs, bl, kb, vb, B, H, Hkv, N, d, q_s, k_s, v_s, c.ptr(), c.bytes(),
                                                               c.stream); }), "dd_block_attention_cached_fp8v");
    return THPVariable_Wrap(out);
}

// (Kc, Vc, Krows, Vrows, positions, qk_dtype, v_dtype) -> None
PyObject *cache_insert(PyObject *const *a, Py_ssize_t n)
{
    want(n, 7);
    const at::Tensor &Kc = tensor(a[0], "Kc"), &Vc = tensor(a[1], "Vc"), &Kr = tensor(a[2], "Krows"), &Vr = tensor(a[3], "Vrows");
    const at::Tensor &pos = tensor(a[4], "positions");
    if (Kc.dim() != 4 || Kr.dim() != 4) value_error("", "Kc, Vc, Krows, Vrows must have four dimensions");
    const int64_t B = Kc.size(0), Hkv = Kc.size(1), N = Kc.size(2), d = Kc.size(3), rows = Kr.size(2);
    if (!has_shape(Vc, {B, Hkv, N, d}) || !has_shape(Kr, {B, Hkv, rows, d}) || !has_shape(Vr, {B, Hkv, rows, d}))
        value_error("", "shapes must be Kc,Vc [B,Hkv,N,d] and Krows,Vrows [B,Hkv,n,d]");
    if (pos.scalar_type() != at::kInt || pos.numel() != B * rows) value_error("", "positions must be int32 with B*n entries");
    const int qk = tag_or(a[5], Kc, "Kc"), vd = tag_or(a[6], Vc, "Vc");
    elements_of(&Kc, qk, "Kc"); elements_of(&Kr, qk, "Krows"); elements_of(&Vc, vd, "Vc"); elements_of(&Vr, vd, "Vrows");
    void *const k = dev(Kc, "Kc"), *const v = dev(Vc, "Vc"), *const kr = dev(Kr, "Krows"), *const vr = dev(Vr, "Vrows"), *const p = dev(pos, "positions");
    const hipStream_t stream = current_stream();
    check(unlocked([&] { return dd_cache_insert_rows(k, v, kr, vr, (const int32_t *)p, rows, B, Hkv, N, d, (dd_dtype)qk, (dd_dtype)vd, stream); }),
          "dd_cache_insert_rows");
    Py_RETURN_NONE;
}

PyObject *triple(const at::Tensor &x, const at::Tensor &y, const at::Tensor &z)
{
    PyObject *t = PyTuple_New(3);
    if (t == nullptr) throw Raised{};
    PyTuple_SET_ITEM(t, 0, THPVariable_Wrap(x));
    PyTuple_SET_ITEM(t, 1, THPVariable_Wrap(y));
    PyTuple_SET_ITEM(t, 2, THPVariable_Wrap(z));
    return t;
}

// (static, logits_d, logits_v, mask, mode, threshold, seed, B, G, out_mask, out_tokens, out_scores, logit_dtype) -> the three outputs
PyObject *verify_remask(PyObject *const *a, Py_ssize_t n)
{
    want(n, 13);
    const bool fixed_scratch = integer(a[0]) != 0;
    const at::Tensor *D = opt_tensor(a[1], "logits_d");
    const at::Tensor &L = tensor(a[2], "logits_v");
    const at::Tensor *mask = opt_tensor(a[3], "mask"), *om = opt_tensor(a[9], "out_mask"), *ot = opt_tensor(a[10], "out_tokens"), *os = opt_tensor(a[11], "out_scores");
    const int mode = integer(a[4]);
    const float threshold = (float)real(a[5]);
    PyObject *seed_int = PyNumber_Long(a[6]);
    if (seed_int == nullptr) throw Raised{};
    const uint64_t seed = PyLong_AsUnsignedLongLongMask(seed_int);
    Py_DECREF(seed_int);
    if (PyErr_Occurred()) throw Raised{};
    if (L.dim() != 2) value_error("", "logits_v must have two dimensions");
    const int64_t P = L.size(0), V = L.size(1);
    const std::pair<int64_t, int64_t> bg = batch_and_rows(a[7], a[8], P, "logits_v must have B*G rows");
    const int64_t B = bg.first, G = bg.second;
    if (D && !has_shape(*D, {P, V})) value_error("", "logits_d shape must match logits_v");
    const dd_dtype dt = (dd_dtype)tag_or(a[12], L, "logits_v");
    elements_of(&L, dt, "logits_v");
    if (mode == DD_KL_THRESH || mode == DD_KL_PROB || mode == DD_KL_TOPK) elements_of(D, dt, "logits_d");   // (the other rules do not read them)
    check_vec(mask, P, at::kByte, "mask");
    check_vec(om, P, at::kByte, "out_mask");
    check_vec(ot, P, at::kInt, "out_tokens");
    check_vec(os, P, at::kFloat, "out_scores");
    void *const ld = dev(D, "logits_d"), *const lv = dev(L, "logits_v"), *const mk = dev(mask, "mask");
    // (with the static scratch an absent output stays absent: the library says what it makes of that)
    auto output = [&](const at::Tensor *given, at::ScalarType type) { return given ? *given : fixed_scratch ? at::Tensor() : empty_like_type({P}, type, L); };
    const at::Tensor rm = output(om, at::kByte), rt = output(ot, at::kInt), rs = output(os, at::kFloat);
    uint8_t *const pm = (uint8_t *)dev(rm.defined() ? &rm : nullptr, "out_mask");
    int32_t *const pt = (int32_t *)dev(rt.defined() ? &rt : nullptr, "out_tokens");
    float *const ps = (float *)dev(rs.defined() ? &rs : nullptr, "out_scores");
    if (fixed_scratch) {
        const hipStream_t stream = current_stream();
        check(unlocked([&] { return dd_verify_remask_static(ld, lv, (const uint8_t *)mk, (dd_mode)mode, threshold, seed, pm, pt, ps, B, G, V, dt, stream); },
                       &scratch().static_launches), "dd_verify_remask_static");
    } else {
        const Call c(dd_verify_remask_workspace_bytes(B, G, V, dt), L, true);
        check(c.run([&] { return dd_verify_remask(ld, lv, (const uint8_t *)mk, (dd_mode)mode, threshold, seed, pm, pt, ps, B, G, V, dt, c.ptr(),
                                                     c.bytes(), c.stream); }), "dd_verify_remask");
    }
    return triple(rm, rt, rs);
}

// (logits_d, mask, mode, threshold, B, G, x_tokens, out_mask, out_tokens, out_conf, logit_dtype) -> the three outputs
PyObject *unmask(PyObject *const *a, Py_ssize_t n)
{
    want(n, 11);
    const at::Tensor &L = tensor(a[0], "logits_d");
    const at::Tensor *mask = opt_tensor(a[1], "mask"), *x = opt_tensor(a[6], "x_tokens");
    const at::Tensor *om = opt_tensor(a[7], "out_mask"), *ot = opt_tensor(a[8], "out_tokens"), *oc = opt_tensor(a[9], "out_conf");
    const int mode = integer(a[2]);
    const float threshold = (float)real(a[3]);
    if (L.dim() != 2) value_error("", "logits_d must have two dimensions");
    const int64_t P = L.size(0), V = L.size(1);
    const std::pair<int64_t, int64_t> bg = batch_and_rows(a[4], a[5], P, "logits_d must have B*G rows");
    const int64_t B = bg.first, G = bg.second;
    const dd_dtype dt = (dd_dtype)tag_or(a[10], L, "logits_d");
    elements_of(&L, dt, "logits_d");
    check_vec(mask, P, at::kByte, "mask");
    check_vec(x, P, at::kInt, "x_tokens");
    check_vec(om, P, at::kByte, "out_mask");
    check_vec(ot, P, at::kInt, "out_tokens");
    check_vec(oc, P, at::kFloat, "out_conf");
    void *const ld = dev(L, "logits_d"), *const mk = dev(mask, "mask");
    int32_t *const px = (int32_t *)dev(x, "x_tokens");
    const at::Tensor rm = om ? *om : empty_like_type({P}, at::kByte, L);
    const at::Tensor rt = ot ? *ot : empty_like_type({P}, at::kInt, L);
    const at::Tensor rc = oc ? *oc : empty_like_type({P}, at::kFloat, L);
    uint8_t *const pm = (uint8_t *)dev(rm, "out_mask");
    int32_t *const pt = (int32_t *)dev(rt, "out_tokens");
    float *const pc = (float *)dev(rc, "out_conf");
    const Call c(dd_unmask_workspace_bytes(B, G, V, dt), L, true);
    check(c.run([&] { return dd_unmask(ld, (const uint8_t *)mk, (dd_unmask_mode)mode, threshold, px, pm, pt, pc, B, G, V, dt, c.ptr(), c.bytes(),
                                          c.stream); }), "dd_unmask");
    return triple(rm, rt, rc);
}

// (logits_d, logits_v, drafter, logit_dtype) -> (kl, conf_v, tok_v, conf_d | None, tok_d | None)
PyObject *verify_scores(PyObject *const *a, Py_ssize_t n)
{
    want(n, 4);
    const at::Tensor &D = tensor(a[0], "logits_d"), &L = tensor(a[1], "logits_v");
    const int drafter = PyObject_IsTrue(a[2]);
    if (drafter < 0) throw Raised{};
    if (L.dim() != 2) value_error("", "logits_v must have two dimensions");
    const int64_t P = L.size(0), V = L.size(1);
    if (!has_shape(D, {P, V})) value_error("", "logits_d and logits_v must have the same shape");
    const bool given = a[3] != Py_None;
    const dd_dtype dt = (dd_dtype)tag_or(a[3], L, "logits_v");
    if (!given && dtype_tag(D, "logits_d") != dt) value_error("", "logits_d and logits_v must have the same dtype");
    elements_of(&L, dt, "logits_v"); elements_of(&D, dt, "logits_d");
    void *const ld = dev(D, "logits_d"), *const lv = dev(L, "logits_v");
    const at::Tensor kl = empty_like_type({P}, at::kFloat, L), cv = empty_like_type({P}, at::kFloat, L), tv = empty_like_type({P}, at::kInt, L);
    const at::Tensor cd = drafter ? empty_like_type({P}, at::kFloat, L) : at::Tensor(), td = drafter ? empty_like_type({P}, at::kInt, L) : at::Tensor();
    const Call c(dd_verify_scores_workspace_bytes(P, V, dt), L, true);
    float *const pk = (float *)kl.data_ptr(), *const pcv = (float *)cv.data_ptr(), *const pcd = drafter ? (float *)cd.data_ptr() : nullptr;
    int32_t *const ptv = (int32_t *)tv.data_ptr(), *const ptd = drafter ? (int32_t *)td.data_ptr() : nullptr;
    check(c.run([&] { return dd_verify_scores(ld, lv, pk, pcv, ptv, pcd, ptd, P, V, dt, c.ptr(), c.bytes(), c.stream); }), "dd_verify_scores");
    PyObject *t = PyTuple_New(5);
    if (t == nullptr) throw Raised{};
    PyTuple_SET_ITEM(t, 0, THPVariable_Wrap(kl));
    PyTuple_SET_ITEM(t, 1, THPVariable_Wrap(cv));
    PyTuple_SET_ITEM(t, 2, THPVariable_Wrap(tv));
    if (drafter) {
        PyTuple_SET_ITEM(t, 3, THPVariable_Wrap(cd));
        PyTuple_SET_ITEM(t, 4, THPVariable_Wrap(td));
    } else {
        Py_INCREF(Py_None); PyTuple_SET_ITEM(t, 3, Py_None);
        Py_INCREF(Py_None); PyTuple_SET_ITEM(t, 4, Py_None);
    }
    return t;
}

// ---- rows before attention and the paged cache.  These calls run on the current stream of the device that their tensors are on,
// which need not be the current one; all of them have to be there.
struct OneDevice {
    const at::Tensor &on;
    explicit OneDevice(const at::Tensor &t) : on(t) {}
    void *operator()(const at::Tensor *t, const char *what, bool dense = true) const
    {
        if (t == nullptr) return nullptr;
        if (!t->is_cuda()) value_error(what, "must live in GPU memory");
        if (t->device() != on.device()) value_error(what, "must be on the device of the other tensors");
        if (dense && !t->is_contiguous()) value_error(what, "must be contiguous");
        return t->data_ptr();
    }
    void *operator()(const at::Tensor &t, const char *what, bool dense = true) const { return (*this)(&t, what, dense); }
};
// rows [B, heads, n, d] by strides: the last dimension dense
void rows_of(const at::Tensor &t, const char *what)
{
    if (t.size(3) > 1 && t.stride(3) != 1) value_error(what, "the last dimension must be contiguous");
}
void ints_of(const at::Tensor *t, int64_t n, const char *what)
{
    if (t == nullptr || (t->scalar_type() == at::kInt && t->numel() == n)) return;
    PyErr_Format(PyExc_ValueError, "%s: must be int32 with %lld entries", what, (long long)n);
    throw Raised{};
}
void weight_of(const at::Tensor *t, int tag, int64_t d, const char *what)
{
    if (t == nullptr) return;
    elements_of(t, tag, what);
    if (t->numel() == d) return;
    PyErr_Format(PyExc_ValueError, "%s: must have %lld elements", what, (long long)d);
    throw Raised{};
}
int rotated_dims(const at::Tensor *inv_freq, int64_t d)
{
    if (inv_freq == nullptr) return 0;
    if (inv_freq->scalar_type() != at::kFloat) {
        PyErr_Format(PyExc_TypeError, "inv_freq: float32 expected, has %s", c10::toString(inv_freq->scalar_type()));
        throw Raised{};
    }
    if (2 * inv_freq->numel() > d) value_error("inv_freq", "has more than d/2 entries");
    return (int)(2 * inv_freq->numel());
}
int truth(PyObject *o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Raised{};
    return v;
}
// sizes as the library takes them
void fits_int(std::initializer_list<int64_t> v)
{
    for (const int64_t x : v)
        if (x > 0x7fffffff) value_error("", "a size is out of range");
}

// (Q, K, q_weight, k_weight, eps, inv_freq, positions, interleaved, Qo, Ko, dtype) -> (Qo, Ko | None)
PyObject *qk_norm_rope(PyObject *const *a, Py_ssize_t n)
{
    want(n, 11);
    const at::Tensor &Q = tensor(a[0], "Q");
    const at::Tensor *K = opt_tensor(a[1], "K"), *qw = opt_tensor(a[2], "q_weight"), *kw = opt_tensor(a[3], "k_weight");
    const float eps = (float)real(a[4]);
    const at::Tensor *freq = opt_tensor(a[5], "inv_freq"), *pos = opt_tensor(a[6], "positions"), *Qo = opt_tensor(a[8], "Qo"), *Ko = opt_tensor(a[9], "Ko");
    const int interleaved = truth(a[7]);
    if (Q.dim() != 4 || (K && K->dim() != 4)) value_error("", "Q, K must have four dimensions");
    const int64_t B = Q.size(0), H = Q.size(1), rows = Q.size(2), d = Q.size(3), Hkv = K ? K->size(1) : 0;
    if (K && !has_shape(*K, {B, Hkv, rows, d})) value_error("", "K shape must be [B,Hkv,n,d] matching Q");
    if (!K && (Ko || kw)) value_error("", "Ko and k_weight go with K");
    fits_int({B, H, Hkv, rows, d});
    const int tag = tag_or(a[10], Q, "Q");
    elements_of(&Q, tag, "Q"); elements_of(K, tag, "K"); elements_of(Qo, tag, "Qo"); elements_of(Ko, tag, "Ko");
    weight_of(qw, tag, d, "q_weight"); weight_of(kw, tag, d, "k_weight");
    const int rot = rotated_dims(freq, d);
    ints_of(pos, B * rows, "positions");
    room_for(Qo, B * H * rows * d, tag_bytes(tag), "Qo"); room_for(Ko, B * Hkv * rows * d, tag_bytes(tag), "Ko");
    rows_of(Q, "Q");
    if (K) rows_of(*K, "K");
    const OneDevice dev(Q);
    void *const q = dev(Q, "Q", false), *const k = dev(K, "K", false), *const w = dev(qw, "q_weight"), *const v = dev(kw, "k_weight");
    void *const f = dev(freq, "inv_freq"), *const p = dev(pos, "positions");
    const c10::hip::HIPGuard guard(Q.device().index());
    const at::Tensor qo = Qo ? *Qo : empty_like_type({B, H, rows, d}, Q.scalar_type(), Q);
    const at::Tensor ko = Ko ? *Ko : K ? empty_like_type({B, Hkv, rows, d}, K->scalar_type(), Q) : at::Tensor();
    void *const x = dev(qo, "Qo"), *const y = dev(ko.defined() ? &ko : nullptr, "Ko");
    const hipStream_t stream = current_stream();
    const int64_t ks[3] = {K ? K->stride(0) : 0, K ? K->stride(1) : 0, K ? K->stride(2) : 0};
    check(unlocked([&] { return dd_qk_norm_rope(q, Q.stride(0), Q.stride(1), Q.stride(2), k, ks[0], ks[1], ks[2], w, v, eps, (const float *)f, rot,
                                                interleaved, (const int32_t *)p, x, y, B, H, Hkv, rows, d, (dd_dtype)tag, stream); }),
          "dd_qk_norm_rope");
    PyObject *t = PyTuple_New(2);
    if (t == nullptr) throw Raised{};
    PyTuple_SET_ITEM(t, 0, THPVariable_Wrap(qo));
    if (ko.defined()) {
        PyTuple_SET_ITEM(t, 1, THPVariable_Wrap(ko));
    } else {
        Py_INCREF(Py_None); PyTuple_SET_ITEM(t, 1, Py_None);
    }
    return t;
}

struct Pages { int64_t num, Hkv, size, d, B, max; int tag; };
Pages pages_of(const at::Tensor &Kc, const at::Tensor &Vc, const at::Tensor &table, const at::Tensor *ks, const at::Tensor *vs, PyObject *tag)
{
    if (Kc.dim() != 4) value_error("", "Kc, Vc must have four dimensions");
    Pages p{Kc.size(0), Kc.size(1), Kc.size(2), Kc.size(3), 0, 0, 0};
    if (!has_shape(Vc, {p.num, p.Hkv, p.d, p.size})) value_error("", "shapes must be Kc [pages,Hkv,page_size,d] and Vc [pages,Hkv,d,page_size]");
    if (table.dim() != 2 || table.scalar_type() != at::kInt) value_error("", "block_table must be int32 with two dimensions");
    p.B = table.size(0);
    p.max = table.size(1);
    fits_int({p.num, p.Hkv, p.size, p.d, p.B, p.max});
    p.tag = tag_or(tag, Kc, "Kc");
    elements_of(&Kc, p.tag, "Kc"); elements_of(&Vc, p.tag, "Vc");
    scales_of(ks, p.num * p.Hkv, "k_scale"); scales_of(vs, p.num * p.Hkv, "v_scale");
    return p;
}

// (Kc, Vc, K, V, block_table, starts, kv_lens, n_rows, k_scale, v_scale, k_weight, eps, inv_freq, interleaved, row_dtype, cache_dtype) -> None
PyObject *paged_append(PyObject *const *a, Py_ssize_t n)
{
    want(n, 16);
    const at::Tensor &Kc = tensor(a[0], "Kc"), &Vc = tensor(a[1], "Vc"), &K = tensor(a[2], "K"), &V = tensor(a[3], "V"), &table = tensor(a[4], "block_table");
    const at::Tensor &starts = tensor(a[5], "starts");
    const at::Tensor *lens = opt_tensor(a[6], "kv_lens"), *count = opt_tensor(a[7], "n_rows"), *ks = opt_tensor(a[8], "k_scale"), *vs = opt_tensor(a[9], "v_scale");
    const at::Tensor *kw = opt_tensor(a[10], "k_weight"), *freq = opt_tensor(a[12], "inv_freq");
    const float eps = (float)real(a[11]);
    const int interleaved = truth(a[13]);
    const Pages p = pages_of(Kc, Vc, table, ks, vs, a[15]);
    if (K.dim() != 4 || !has_shape(K, {p.B, p.Hkv, K.size(2), p.d}) || V.sizes() != K.sizes()) value_error("", "K and V shapes must be [B,Hkv,n,d] matching the cache");
    const int64_t rows = K.size(2);
    fits_int({rows});
    const int tag = tag_or(a[14], K, "K");
    elements_of(&K, tag, "K"); elements_of(&V, tag, "V");
    weight_of(kw, tag, p.d, "k_weight");
    const int rot = rotated_dims(freq, p.d);
    ints_of(&starts, p.B, "starts"); ints_of(lens, p.B, "kv_lens"); ints_of(count, p.B, "n_rows");
    rows_of(K, "K"); rows_of(V, "V");
    const OneDevice dev(Kc);
    void *const kc = dev(Kc, "Kc"), *const vc = dev(Vc, "Vc"), *const k = dev(K, "K", false), *const v = dev(V, "V", false), *const t = dev(table, "block_table");
    void *const st = dev(starts, "starts"), *const ln = dev(lens, "kv_lens"), *const ct = dev(count, "n_rows"), *const sk = dev(ks, "k_scale"), *const sv = dev(vs, "v_scale");
    void *const w = dev(kw, "k_weight"), *const f = dev(freq, "inv_freq");
    const c10::hip::HIPGuard guard(Kc.device().index());
    const hipStream_t stream = current_stream();
    check(unlocked([&] { return dd_paged_cache_append(kc, vc, (float *)sk, (float *)sv, k, K.stride(0), K.stride(1), K.stride(2), v, V.stride(0), V.stride(1),
                                                      V.stride(2), (const int32_t *)t, (const int32_t *)st, (const int32_t *)ln, (const int32_t *)ct, w, eps,
                                                      (const float *)f, rot, interleaved, rows, p.B, p.Hkv, p.d, p.num, p.size, p.max, (dd_dtype)tag,
                                                      (dd_dtype)p.tag, stream); }), "dd_paged_cache_append");
    Py_RETURN_NONE;
}

// (Q, Kc, Vc, block_table, kv_lens, k_scale, v_scale, O, cache_dtype) -> O
PyObject *paged_attention(PyObject *const *a, Py_ssize_t n)
{
    want(n, 9);
    const at::Tensor &Q = tensor(a[0], "Q"), &Kc = tensor(a[1], "Kc"), &Vc = tensor(a[2], "Vc"), &table = tensor(a[3], "block_table"), &lens = tensor(a[4], "kv_lens");
    const at::Tensor *ks = opt_tensor(a[5], "k_scale"), *vs = opt_tensor(a[6], "v_scale"), *O = opt_tensor(a[7], "O");
    const Pages p = pages_of(Kc, Vc, table, ks, vs, a[8]);
    if (Q.dim() != 4 || Q.size(0) != p.B || Q.size(3) != p.d) value_error("", "Q shape must be [B,H,n,d] matching the cache and block_table");
    const int64_t H = Q.size(1), rows = Q.size(2);
    fits_int({H, rows});
    elements_of(&Q, DD_BF16, "Q"); elements_of(O, DD_BF16, "O");
    ints_of(&lens, p.B, "kv_lens");
    room_for(O, p.B * H * rows * p.d, 2, "O");
    const OneDevice dev(Q);
    void *const q = dev(Q, "Q"), *const kc = dev(Kc, "Kc"), *const vc = dev(Vc, "Vc"), *const t = dev(table, "block_table"), *const ln = dev(lens, "kv_lens");
    void *const sk = dev(ks, "k_scale"), *const sv = dev(vs, "v_scale");
    const c10::hip::HIPGuard guard(Q.device().index());
    const at::Tensor out = O ? *O : empty_like_type({p.B, H, rows, p.d}, Q.scalar_type(), Q);
    void *const o = dev(out, "O");
    const Call c(dd_paged_attention_workspace_bytes(rows, p.B, H, p.Hkv, p.d, p.size, p.max, (dd_dtype)p.tag), Q);
    check(c.run([&] { return dd_paged_attention(q, kc, vc, (const float *)sk, (const float *)sv, (const int32_t *)t, (const int32_t *)ln, o, rows, p.B, H, p.Hkv,
                                                   p.d, p.num, p.size, p.max, (dd_dtype)p.tag, c.ptr(), c.bytes(), c.stream); }), "dd_paged_attention");
    return THPVariable_Wrap(out);
}

// (Q, Kc, Vc, prefix_table, prefix_lens, group_starts, block_table, kv_lens, k_scale, v_scale, O, cache_dtype) -> O
PyObject *paged_attention_shared(PyObject *const *a, Py_ssize_t n)
{
    want(n, 12);
    const at::Tensor &Q = tensor(a[0], "Q"), &Kc = tensor(a[1], "Kc"), &Vc = tensor(a[2], "Vc"), &prefix = tensor(a[3], "prefix_table");
    const at::Tensor &plens = tensor(a[4], "prefix_lens"), &starts = tensor(a[5], "group_starts"), &table = tensor(a[6], "block_table"), &lens = tensor(a[7], "kv_lens");
    const at::Tensor *ks = opt_tensor(a[8], "k_scale"), *vs = opt_tensor(a[9], "v_scale"), *O = opt_tensor(a[10], "O");
    const Pages p = pages_of(Kc, Vc, table, ks, vs, a[11]);
    if (prefix.dim() != 2 || prefix.scalar_type() != at::kInt) value_error("", "prefix_table must be int32 with two dimensions");
    const int64_t G = prefix.size(0), most = prefix.size(1);
    if (Q.dim() != 4 || Q.size(0) != p.B || Q.size(3) != p.d) value_error("", "Q shape must be [B,H,n,d] matching the cache and block_table");
    const int64_t H = Q.size(1), rows = Q.size(2);
    fits_int({H, rows, G, most});
    elements_of(&Q, DD_BF16, "Q"); elements_of(O, DD_BF16, "O");
    ints_of(&lens, p.B, "kv_lens"); ints_of(&plens, G, "prefix_lens"); ints_of(&starts, G + 1, "group_starts");
    room_for(O, p.B * H * rows * p.d, 2, "O");
    const OneDevice dev(Q);
    void *const q = dev(Q, "Q"), *const kc = dev(Kc, "Kc"), *const vc = dev(Vc, "Vc"), *const pt = dev(prefix, "prefix_table"), *const pl = dev(plens, "prefix_lens");
    void *const gs = dev(starts, "group_starts"), *const t = dev(table, "block_table"), *const ln = dev(lens, "kv_lens");
    void *const sk = dev(ks, "k_scale"), *const sv = dev(vs, "v_scale");
    const c10::hip::HIPGuard guard(Q.device().index());
    const at::Tensor out = O ? *O : empty_like_type({p.B, H, rows, p.d}, Q.scalar_type(), Q);
    void *const o = dev(out, "O");
    const Call c(dd_paged_attention_shared_workspace_bytes(rows, p.B, H, p.Hkv, p.d, p.size, G, most, p.max, (dd_dtype)p.tag), Q);
    check(c.run([&] { return dd_paged_attention_shared(q, kc, vc, (const float *)sk, (const float *)sv, (const int32_t *)pt, (const int32_t *)pl, (const int32_t *)gs,
                                                          (const int32_t *)t, (const int32_t *)ln, o, rows, p.B, H, p.Hkv, p.d, p.num, p.size, G, most, p.max,
                                                          (dd_dtype)p.tag, c.ptr(), c.bytes(), c.stream); }), "dd_paged_attention_shared");
    return THPVariable_Wrap(out);
}

// (block_table, free_pages, num_free, lens, new_lens, page_size, n, out_lens, positions, slots) -> (out_lens, positions | None, slots | None)
PyObject *paged_resize(PyObject *const *a, Py_ssize_t n)
{
    want(n, 10);
    const at::Tensor &table = tensor(a[0], "block_table"), &stack = tensor(a[1], "free_pages"), &count = tensor(a[2], "num_free");
    const at::Tensor &lens = tensor(a[3], "lens"), &new_lens = tensor(a[4], "new_lens");
    const at::Tensor *ol = opt_tensor(a[7], "out_lens"), *op = opt_tensor(a[8], "positions"), *os = opt_tensor(a[9], "slots");
    int64_t sizes[2];
    for (int i = 0; i < 2; ++i) {
        PyObject *v = exact_integer(a[5 + i], i == 0 ? "page_size" : "n");
        int over = 0;
        sizes[i] = PyLong_AsLongLongAndOverflow(v, &over);
        Py_DECREF(v);
        if (over != 0 || sizes[i] < 0) value_error(i == 0 ? "page_size" : "n", "is out of range");
    }
    const int64_t page = sizes[0], rows = sizes[1];
    if (table.dim() != 2 || table.scalar_type() != at::kInt) value_error("", "block_table must be int32 with two dimensions");
    const int64_t B = table.size(0), most = table.size(1), pages = stack.numel();
    fits_int({B, most, pages, page, rows});
    ints_of(&stack, pages, "free_pages"); ints_of(&count, 1, "num_free"); ints_of(&lens, B, "lens"); ints_of(&new_lens, B, "new_lens");
    ints_of(ol, B, "out_lens"); ints_of(op, B * rows, "positions"); ints_of(os, B * rows, "slots");
    const OneDevice dev(table);
    void *const t = dev(table, "block_table"), *const st = dev(stack, "free_pages"), *const nf = dev(count, "num_free"), *const ln = dev(lens, "lens");
    void *const nl = dev(new_lens, "new_lens");
    const c10::hip::HIPGuard guard(table.device().index());
    const at::Tensor rl = ol ? *ol : empty_like_type({B}, at::kInt, table);
    const at::Tensor rp = op ? *op : rows > 0 ? empty_like_type({B, rows}, at::kInt, table) : at::Tensor();
    const at::Tensor rs = os ? *os : rows > 0 ? empty_like_type({B, rows}, at::kInt, table) : at::Tensor();
    void *const wl = dev(rl, "out_lens"), *const wp = dev(rp.defined() ? &rp : nullptr, "positions"), *const wsl = dev(rs.defined() ? &rs : nullptr, "slots");
    const Call c(dd_paged_resize_workspace_bytes(rows, B, page, most), table);
    check(c.run([&] { return dd_paged_resize((int32_t *)t, (int32_t *)st, (int32_t *)nf, (const int32_t *)ln, (const int32_t *)nl, (int32_t *)wl, (int32_t *)wp,
                                             (int32_t *)wsl, rows, B, pages, page, most, c.ptr(), c.bytes(), c.stream); }), "dd_paged_resize");
    PyObject *out = PyTuple_New(3);
    if (out == nullptr) throw Raised{};
    PyTuple_SET_ITEM(out, 0, THPVariable_Wrap(rl));
    int i = 1;
    for (const at::Tensor *r : {&rp, &rs}) {
        if (r->defined()) {
            PyTuple_SET_ITEM(out, i++, THPVariable_Wrap(*r));
        } else {
            Py_INCREF(Py_None); PyTuple_SET_ITEM(out, i++, Py_None);
        }
    }
    return out;
}

// (logits_v, logits_d, tokens, uniforms, temperature, n_draft, out_tokens, out_accepted, out_chances, logit_dtype) -> the three outputs
PyObject *verify_draft(PyObject *const *a, Py_ssize_t n)
{
    want(n, 10);
    const at::Tensor &L = tensor(a[0], "logits_v"), &x = tensor(a[2], "tokens"), &u = tensor(a[3], "uniforms");
    const at::Tensor *D = opt_tensor(a[1], "logits_d"), *t = opt_tensor(a[4], "temperature"), *count = opt_tensor(a[5], "n_draft");
    const at::Tensor *ot = opt_tensor(a[6], "out_tokens"), *oa = opt_tensor(a[7], "out_accepted"), *oc = opt_tensor(a[8], "out_chances");
    if (L.dim() != 3 || x.dim() != 2) value_error("", "logits_v must have three dimensions, tokens two");
    const int64_t B = x.size(0), drafts = x.size(1), rows = L.size(1), V = L.size(2);
    fits_int({B, drafts, rows, V});
    if (L.size(0) != B || (rows != drafts && rows != drafts + 1)) value_error("", "logits_v shape must be [B,n,V] or, with a row behind the last draft, [B,n+1,V]");
    if (D && !has_shape(*D, {B, drafts, V})) value_error("", "logits_d shape must be [B,n,V]");
    const int bonus = rows == drafts + 1;
    const dd_dtype dt = (dd_dtype)tag_or(a[9], L, "logits_v");
    elements_of(&L, dt, "logits_v"); elements_of(D, dt, "logits_d");
    check_vec(&x, B * drafts, at::kInt, "tokens");
    check_vec(&u, B * (drafts + 1), at::kFloat, "uniforms");
    check_vec(t, B, at::kFloat, "temperature");
    check_vec(count, B, at::kInt, "n_draft");
    check_vec(ot, B * (drafts + 1), at::kInt, "out_tokens");
    check_vec(oa, B, at::kInt, "out_accepted");
    check_vec(oc, B * drafts, at::kFloat, "out_chances");
    const OneDevice dev(L);
    void *const lv = dev(L, "logits_v"), *const ld = dev(D, "logits_d"), *const px = dev(x, "tokens"), *const pu = dev(u, "uniforms");
    void *const pt = dev(t, "temperature"), *const pn = dev(count, "n_draft");
    const c10::hip::HIPGuard guard(L.device().index());
    const at::Tensor rt = ot ? *ot : empty_like_type({B, drafts + 1}, at::kInt, L);
    const at::Tensor ra = oa ? *oa : empty_like_type({B}, at::kInt, L);
    const at::Tensor rc = oc ? *oc : empty_like_type({B, drafts}, at::kFloat, L);
    void *const wt = dev(rt, "out_tokens"), *const wa = dev(ra, "out_accepted"), *const wc = dev(rc, "out_chances");
    const Call c(dd_verify_draft_workspace_bytes(B, drafts, bonus, V, D != nullptr, dt), L);
    check(c.run([&] { return dd_verify_draft(lv, ld, (const int32_t *)px, (const int32_t *)pn, (const float *)pu, (const float *)pt, (int32_t *)wt, (int32_t *)wa,
                                             (float *)wc, B, drafts, bonus, V, dt, c.ptr(), c.bytes(), c.stream); }), "dd_verify_draft");
    return triple(rt, ra, rc);
}

// (DDError) -> None
PyObject *set_error_class(PyObject *const *a, Py_ssize_t n)
{
    want(n, 1);
    Py_INCREF(a[0]);
    Py_XDECREF(error_class);
    error_class = a[0];
    Py_RETURN_NONE;
}
// (tensor | None) -> the one set before, or None
PyObject *set_fixed_workspace(PyObject *const *a, Py_ssize_t n)
{
    want(n, 1);
    const at::Tensor *t = opt_tensor(a[0], "workspace");
    if (t) dev(t, "workspace");
    const at::Tensor prev = fixed != nullptr ? *fixed : at::Tensor();
    delete fixed;
    fixed = t ? new at::Tensor(*t) : nullptr;
    if (!prev.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(prev);
}
PyObject *reset_workspace_peak(PyObject *const *, Py_ssize_t n)
{
    want(n, 0);
    peak = 0;
    Py_RETURN_NONE;
}
PyObject *workspace_peak(PyObject *const *, Py_ssize_t n)
{
    want(n, 0);
    return PyLong_FromSize_t(peak);
}

template <PyObject *(*F)(PyObject *const *, Py_ssize_t)>
PyObject *entry(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    try {
        return F(a, n);
    } catch (const Raised &) {
        return nullptr;
    } catch (...) {                                          // as torch itself raises it: torch.OutOfMemoryError for an allocation
        torch::translate_exception_to_python(std::current_exception());
        return nullptr;
    }
}
#define DD_METHOD(name) {#name, (PyCFunction)(void (*)(void))entry<name>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {DD_METHOD(bidir), DD_METHOD(block), DD_METHOD(bidir_fp8v), DD_METHOD(bidir_mx), DD_METHOD(block_fp8v),
                         DD_METHOD(cache_insert), DD_METHOD(verify_remask), DD_METHOD(unmask), DD_METHOD(verify_scores),
                         DD_METHOD(qk_norm_rope), DD_METHOD(paged_append), DD_METHOD(paged_attention), DD_METHOD(verify_draft),
                         DD_METHOD(paged_attention_shared), DD_METHOD(paged_resize),
                         DD_METHOD(set_error_class), DD_METHOD(set_fixed_workspace), DD_METHOD(reset_workspace_peak),
                         DD_METHOD(workspace_peak), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", "argument marshalling of paper_2604_05250_amd", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
