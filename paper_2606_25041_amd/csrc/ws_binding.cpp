// CPython marshalling of the package's entry points: torch tensors to the C
// ABI's pointers and strides, outputs and workspaces from torch's allocator,
// the current stream.  Host time bounds the smallest calls (a committed unit:
// 3 us of kernel behind 10 us of ctypes marshalling), so the common case runs
// here: device tensors, (host, device) pairs of int32 arrays.  Anything else
// (another type, a wrong shape or dtype) returns None before anything is
// enqueued, and the Python code, which states the checks and
// raises their errors, takes the call.  Python objects are read first; the
// allocations and the C ABI call (validation, planning, launches, which block
// on a full hardware queue) run without the GIL, as through ctypes.
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include <ATen/ops/empty.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>

#include <algorithm>
#include <cmath>

#include "../../include/ws_attn.h"

namespace {

// C ABI functions, by address (the package loads the library and hands its
// addresses over, so both speak to the same one)
struct Abi {
    decltype(&ws_kv_append) kv_append;
    decltype(&ws_kv_append_varlen) kv_append_varlen;
    decltype(&ws_block_causal_attn_fwd) fwd;
    decltype(&ws_block_causal_attn_fwd_text) fwd_text;
    decltype(&ws_block_causal_attn_fwd_varlen) fwd_varlen;
    decltype(&ws_block_causal_attn_fwd_noalloc) fwd_noalloc;
    decltype(&ws_block_causal_prefill) prefill;
    decltype(&ws_block_causal_prefill_text) prefill_text;
    decltype(&ws_block_causal_prefill_bwd) bwd;
    decltype(&ws_workspace_bytes) workspace_bytes;
    decltype(&ws_step_workspace_bytes_varlen) workspace_bytes_varlen;
} abi;

struct WindowAbi {
    decltype(&ws_block_causal_attn_fwd_window) fwd;
    decltype(&ws_step_workspace_bytes_window) step_bytes;
    decltype(&ws_block_causal_prefill_window) prefill;
    decltype(&ws_block_causal_prefill_window_bwd) bwd;
    decltype(&ws_prefill_window_bwd_workspace_bytes) bwd_bytes;
} wabi;

struct Cache4Abi {
    decltype(&ws_kv_append_4bit) append;
    decltype(&ws_kv_read_4bit) read;
    decltype(&ws_block_causal_attn_fwd_4bit) fwd;
    decltype(&ws_step_workspace_bytes_4bit) step_bytes;
} abi4;

PyObject *cache_class;    // PagedCache
PyObject *cache4_class;   // PagedCache4

bool take_addresses(void **to, size_t count, PyObject *const *args, Py_ssize_t n) {
    if (n != (Py_ssize_t)count) {
        PyErr_SetString(PyExc_TypeError, "one address per ABI function");
        return false;
    }
    for (Py_ssize_t i = 0; i < n; ++i) {
        void *p = PyLong_AsVoidPtr(args[i]);
        if (PyErr_Occurred()) return false;
        to[i] = p;
    }
    return true;
}

PyObject *bind_window(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (!take_addresses((void **)&wabi, sizeof wabi / sizeof(void *), args, n)) return nullptr;
    Py_RETURN_NONE;
}

PyObject *bind_cache4(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n < 1 || !take_addresses((void **)&abi4, sizeof abi4 / sizeof(void *), args + 1, n - 1)) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "the cache class first");
        return nullptr;
    }
    Py_INCREF(args[0]);
    Py_XSETREF(cache4_class, args[0]);
    Py_RETURN_NONE;
}

PyObject *bind(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 1 + (Py_ssize_t)(sizeof(Abi) / sizeof(void *))) {
        PyErr_SetString(PyExc_TypeError, "the cache class and one address per ABI function");
        return nullptr;
    }
    for (Py_ssize_t i = 1; i < n; ++i) {
        void *p = PyLong_AsVoidPtr(args[i]);
        if (PyErr_Occurred()) return nullptr;
        ((void **)&abi)[i - 1] = p;
    }
    Py_INCREF(args[0]);
    Py_XSETREF(cache_class, args[0]);
    Py_RETURN_NONE;
}

// A plain torch.Tensor (no subclass: those may hold no memory), else nullptr
const at::Tensor *tensor(PyObject *o) {
    if ((PyObject *)Py_TYPE(o) != THPVariableClass) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    return t.defined() && t.layout() == at::kStrided && t.has_storage() ? &t : nullptr;
}

// Whether a tensor is on the current device, whose stream the library launches
// on.  The device is asked for once a call, by its first device tensor (where
// there is none the question is an error).
thread_local c10::DeviceIndex device_now = -1;
void new_call() { device_now = -1; }
bool here(const at::Tensor &t) {
    if (!t.is_cuda()) return false;
    if (device_now < 0) device_now = c10::hip::current_device();
    return t.device().index() == device_now;
}

bool shaped(const at::Tensor &t, std::initializer_list<int64_t> shape) { return t.sizes() == at::IntArrayRef(shape); }

// descriptor of a [B][L][H][d] tensor of the current device with a contiguous last dim
bool token_tensor(const at::Tensor *t, std::initializer_list<int64_t> shape, ws_tensor4 &d) {
    if (!t || !here(*t) || !shaped(*t, shape) || t->stride(3) != 1) return false;
    const auto dt = t->scalar_type();
    if (dt != at::kBFloat16 && dt != at::kFloat) return false;
    d = ws_tensor4{t->data_ptr(), dt == at::kBFloat16 ? WS_DTYPE_BF16 : WS_DTYPE_F32, t->stride(0), t->stride(1),
                   t->stride(2)};
    return true;
}

struct Ints {
    const int32_t *host = nullptr, *dev = nullptr;
};

// a (host, device) pair of contiguous int32 arrays of the given shape (packed:
// of any shape of that many elements); None gives null pointers (so an empty
// array, whose pointers are null too, is declined)
bool int_pair(PyObject *o, std::initializer_list<int64_t> shape, bool packed, Ints &x) {
    if (o == Py_None) return true;
    if (!PyTuple_CheckExact(o) || PyTuple_GET_SIZE(o) != 2) return false;
    const at::Tensor *t[2] = {tensor(PyTuple_GET_ITEM(o, 0)), tensor(PyTuple_GET_ITEM(o, 1))};
    int64_t numel = 1;
    for (int64_t n : shape) numel *= n;
    if (numel == 0) return false;
    for (const at::Tensor *p : t) {
        if (!p || p->scalar_type() != at::kInt) return false;
        if (!p->is_contiguous() || (packed ? p->numel() != numel : !shaped(*p, shape))) return false;
    }
    if (!t[0]->is_cpu() || !here(*t[1])) return false;
    x.host = (const int32_t *)t[0]->data_ptr();
    x.dev = (const int32_t *)t[1]->data_ptr();
    return true;
}

// Runs its scope without the GIL.
struct NoGil {
    PyThreadState *state = PyEval_SaveThread();
    ~NoGil() { PyEval_RestoreThread(state); }
};

PyObject *names[7];   // attribute names of PagedCache, in the order below
PyObject *pool_name;  // PagedCache4: "pool" in place of the first two

// a contiguous tensor of the current device (of elements of `size` bytes; 0: any)
bool packed(const at::Tensor *t, int64_t size) {
    return t && here(*t) && t->is_contiguous() && (!size || (int64_t)t->element_size() == size);
}
// both copies of a page table of at least `batch` rows
bool table(const at::Tensor *h, const at::Tensor *d, int64_t batch) {
    return h && d && h->dim() == 2 && h->size(0) >= batch && d->sizes() == h->sizes() && h->scalar_type() == at::kInt &&
           d->scalar_type() == at::kInt && h->is_contiguous() && d->is_contiguous() && h->is_cpu() && here(*d);
}

// The paged cache's descriptor, with its table checked for `batch` rows.  The
// cache's tensors are held: without the GIL another thread may replace them.
struct Paged : ws_paged_kv {
    at::Tensor hold[4];
};
bool paged(PyObject *cache, int64_t batch, Paged &d) {
    // (another class may have a descriptor of its own: desc())
    if ((PyObject *)Py_TYPE(cache) != cache_class) return false;
    PyObject *v[7] = {};
    bool ok = true;
    for (int i = 0; i < 7 && ok; ++i) ok = (v[i] = PyObject_GetAttr(cache, names[i])) != nullptr;
    if (!ok) PyErr_Clear();
    const at::Tensor *k = nullptr, *vp = nullptr, *th = nullptr, *td = nullptr;
    if (ok) {
        k = tensor(v[0]);
        vp = tensor(v[1]);
        th = tensor(v[2]);
        td = tensor(v[3]);
        ok = packed(k, 2) && packed(vp, 2) && table(th, td, batch) && PyLong_CheckExact(v[4]) && PyLong_CheckExact(v[5]) &&
             PyLong_CheckExact(v[6]);
    }
    if (ok) {
        static_cast<ws_paged_kv &>(d) = ws_paged_kv{k->data_ptr(), vp->data_ptr(), (const int32_t *)td->data_ptr(), (const int32_t *)th->data_ptr(),
                        (int32_t)PyLong_AsLong(v[4]), WS_PAGE_SIZE, (int32_t)th->size(1), (int32_t)PyLong_AsLong(v[5]),
                        (int32_t)PyLong_AsLong(v[6])};
        d.hold[0] = *k, d.hold[1] = *vp, d.hold[2] = *th, d.hold[3] = *td;
    }
    for (PyObject *o : v) Py_XDECREF(o);
    return ok;
}

// The same of a PagedCache4
struct Paged4 : ws_paged_kv4 {
    at::Tensor hold[3];
};
bool paged4(PyObject *cache, int64_t batch, Paged4 &d) {
    if ((PyObject *)Py_TYPE(cache) != cache4_class) return false;
    PyObject *v[6] = {};
    bool ok = true;
    for (int i = 0; i < 6 && ok; ++i) ok = (v[i] = PyObject_GetAttr(cache, i ? names[i + 1] : pool_name)) != nullptr;
    if (!ok) PyErr_Clear();
    if (ok) {
        const at::Tensor *p = tensor(v[0]), *th = tensor(v[1]), *td = tensor(v[2]);
        ok = packed(p, 1) && table(th, td, batch) && PyLong_CheckExact(v[3]) && PyLong_CheckExact(v[4]) &&
             PyLong_CheckExact(v[5]);
        if (ok) {
            static_cast<ws_paged_kv4 &>(d) =
                ws_paged_kv4{p->data_ptr(), (const int32_t *)td->data_ptr(), (const int32_t *)th->data_ptr(),
                             (int32_t)PyLong_AsLong(v[3]), WS_PAGE_SIZE, (int32_t)th->size(1),
                             (int32_t)PyLong_AsLong(v[4]), (int32_t)PyLong_AsLong(v[5])};
            d.hold[0] = *p, d.hold[1] = *th, d.hold[2] = *td;
        }
    }
    for (PyObject *o : v) Py_XDECREF(o);
    return ok;
}

void *stream() { return (void *)c10::hip::getCurrentHIPStream().stream(); }

// scale: None (1 / sqrt(d)) or a float
bool scale_of(PyObject *o, int64_t d, float &s) {
    if (o == Py_None) {
        s = (float)(1.0 / std::sqrt((double)d));
        return true;
    }
    if (!PyFloat_CheckExact(o)) return false;
    s = (float)PyFloat_AS_DOUBLE(o);
    return true;
}

// The caller's output of the given shape, or, for None, undefined
bool given(PyObject *o, std::initializer_list<int64_t> shape, at::Tensor &t) {
    if (o == Py_None) return true;
    const at::Tensor *p = tensor(o);
    if (!p || !here(*p) || !shaped(*p, shape)) return false;
    t = *p;
    return true;
}

bool packed_f32(const at::Tensor &t) { return t.scalar_type() == at::kFloat && t.is_contiguous(); }

// A new output of the given shape where the caller gave none
void allocate(at::Tensor &t, std::initializer_list<int64_t> shape, at::ScalarType type, const at::Tensor &like) {
    if (!t.defined()) t = at::empty(at::IntArrayRef(shape), like.options().dtype(type));
}

bool flag(PyObject *o, bool &b) {
    if (o != Py_True && o != Py_False) return false;
    b = o == Py_True;
    return true;
}

// window and sinks, checked by the Python code (ints in [0, 2^31)); without them
// window is -1
struct Window {
    int32_t window = -1, sinks = 0;
};
bool window_of(PyObject *w, PyObject *s, Window &x) {
    if (!PyLong_CheckExact(w) || !PyLong_CheckExact(s)) return false;
    x.window = (int32_t)PyLong_AsLong(w);
    x.sinks = (int32_t)PyLong_AsLong(s);
    return true;
}

at::ScalarType dtype_of(PyObject *o) {
    return THPDtype_Check(o) ? ((THPDtype *)o)->scalar_type : at::kDouble;
}

// (status, tensors...), None for an undefined one
PyObject *result(int rc, std::initializer_list<at::Tensor> out) {
    THPObjectPtr r(PyTuple_New(1 + (Py_ssize_t)out.size()));
    if (!r) return nullptr;
    PyObject *s = PyLong_FromLong(rc);
    if (!s) return nullptr;
    PyTuple_SET_ITEM(r.get(), 0, s);
    Py_ssize_t i = 1;
    for (const at::Tensor &t : out) {
        PyObject *o = t.defined() ? THPVariable_Wrap(t) : (Py_INCREF(Py_None), Py_None);
        if (!o) return nullptr;
        PyTuple_SET_ITEM(r.get(), i++, o);
    }
    return r.release();
}

// append(cache, lens, k_new, v_new, new_lens) -> status, or None
PyObject *append(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    new_call();
    if (n != 5) Py_RETURN_NONE;
    const at::Tensor *k = tensor(a[2]);
    if (!k || k->dim() != 4) Py_RETURN_NONE;
    const int64_t B = k->size(0), L = k->size(1);
    Paged kv{};
    ws_tensor4 kd, vd;
    Ints lens, nl;
    if (!paged(a[0], B, kv) || !token_tensor(k, {B, L, kv.num_kv_heads, kv.head_dim}, kd) ||
        !token_tensor(tensor(a[3]), {B, L, kv.num_kv_heads, kv.head_dim}, vd) || a[1] == Py_None ||
        !int_pair(a[1], {B}, false, lens) || !int_pair(a[4], {B}, true, nl))
        Py_RETURN_NONE;
    int rc;
    {
        NoGil free;
        rc = nl.host ? abi.kv_append_varlen(&kv, B, lens.host, lens.dev, nl.host, nl.dev, L, kd, vd, stream())
                     : abi.kv_append(&kv, B, lens.host, lens.dev, L, kd, vd, stream());
    }
    return PyLong_FromLong(rc);
    END_HANDLE_TH_ERRORS
}

// append4(cache, lens, k_new, v_new, new_lens) -> status, or None
PyObject *append4(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    new_call();
    if (n != 5) Py_RETURN_NONE;
    const at::Tensor *k = tensor(a[2]);
    if (!k || k->dim() != 4) Py_RETURN_NONE;
    const int64_t B = k->size(0), L = k->size(1);
    Paged4 kv{};
    ws_tensor4 kd, vd;
    Ints lens, nl;
    if (!paged4(a[0], B, kv) || !token_tensor(k, {B, L, kv.num_kv_heads, kv.head_dim}, kd) ||
        !token_tensor(tensor(a[3]), {B, L, kv.num_kv_heads, kv.head_dim}, vd) || a[1] == Py_None ||
        !int_pair(a[1], {B}, false, lens) || !int_pair(a[4], {B}, true, nl))
        Py_RETURN_NONE;
    int rc;
    {
        NoGil free;
        rc = abi4.append(&kv, B, lens.host, lens.dev, nl.host, nl.dev, L, kd, vd, stream());
    }
    return PyLong_FromLong(rc);
    END_HANDLE_TH_ERRORS
}

// read4(cache, starts, length, k, v) -> (status, k, v), or None
PyObject *read4(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    new_call();
    if (n != 5 || !PyTuple_CheckExact(a[1]) || PyTuple_GET_SIZE(a[1]) != 2 || !PyLong_CheckExact(a[2])) Py_RETURN_NONE;
    const at::Tensor *h = tensor(PyTuple_GET_ITEM(a[1], 0));
    if (!h || h->dim() != 1) Py_RETURN_NONE;
    int over = 0;
    const int64_t B = h->size(0), L = PyLong_AsLongAndOverflow(a[2], &over);
    Paged4 kv{};
    ws_tensor4 kd, vd;
    Ints starts;
    if (over || L < 0 || L > INT32_MAX || !paged4(a[0], B, kv) || !int_pair(a[1], {B}, false, starts)) Py_RETURN_NONE;
    const int64_t H = kv.num_kv_heads, D = kv.head_dim;
    at::Tensor k, v;
    if (!given(a[3], {B, L, H, D}, k) || (k.defined() && !token_tensor(&k, {B, L, H, D}, kd)) ||
        !given(a[4], {B, L, H, D}, v) || (v.defined() && !token_tensor(&v, {B, L, H, D}, vd)))
        Py_RETURN_NONE;
    int rc;
    {
        NoGil free;
        allocate(k, {B, L, H, D}, at::kBFloat16, kv.hold[0]);
        allocate(v, {B, L, H, D}, at::kBFloat16, kv.hold[0]);
        token_tensor(&k, {B, L, H, D}, kd);
        token_tensor(&v, {B, L, H, D}, vd);
        rc = abi4.read(&kv, B, starts.host, starts.dev, L, kd, vd, stream());
    }
    return result(rc, {k, v});
    END_HANDLE_TH_ERRORS
}

// step(q, k_new, v_new, cache, lens, scale, fuse_append, out, out_dtype,
//      want_lse, lse, workspace, text_starts, new_lens, noalloc)
//   -> (status, out, lse), or None
// (step_window: and window, sinks; step4: a PagedCache4)
PyObject *step_of(PyObject *const *a, const Window &win, bool four = false) {
    new_call();
    const at::Tensor *q = tensor(a[0]);
    if (!q || q->dim() != 4) Py_RETURN_NONE;
    const int64_t B = q->size(0), L = q->size(1), H = q->size(2), D = q->size(3);
    if (B == 0 || L == 0) Py_RETURN_NONE;
    Paged kv{};
    Paged4 kv4{};
    ws_tensor4 qd, kd, vd, od;
    Ints lens, text, nl;
    bool fuse, want_lse, noalloc;
    float scale;
    if (!flag(a[6], fuse) || !flag(a[9], want_lse) || !flag(a[14], noalloc) ||
        !(four ? paged4(a[3], B, kv4) : paged(a[3], B, kv)))
        Py_RETURN_NONE;
    const int64_t hkv = four ? kv4.num_kv_heads : kv.num_kv_heads;
    if ((four ? kv4.head_dim : kv.head_dim) != D ||
        !token_tensor(q, {B, L, H, D}, qd) || !token_tensor(tensor(a[1]), {B, L, hkv, D}, kd) ||
        !token_tensor(tensor(a[2]), {B, L, hkv, D}, vd) || a[4] == Py_None ||
        !int_pair(a[4], {B}, false, lens) || !scale_of(a[5], D, scale) || !int_pair(a[12], {B}, true, text) ||
        !int_pair(a[13], {B}, true, nl))
        Py_RETURN_NONE;
    const at::ScalarType type = a[7] == Py_None ? dtype_of(a[8]) : at::kBFloat16;
    if (type != at::kBFloat16 && type != at::kFloat) Py_RETURN_NONE;
    const at::Tensor *wsp = a[11] == Py_None ? nullptr : tensor(a[11]);
    if (a[11] != Py_None && !packed(wsp, 0)) Py_RETURN_NONE;
    at::Tensor out, lse, own;
    const bool with_lse = want_lse || a[10] != Py_None;
    if (!given(a[7], {B, L, H, D}, out) || (out.defined() && !token_tensor(&out, {B, L, H, D}, od)) ||
        !given(a[10], {B, H, L}, lse) || (lse.defined() && !packed_f32(lse)))
        Py_RETURN_NONE;
    const int flags = fuse ? WS_FUSE_APPEND : 0;
    int rc;
    {
        NoGil free;
        allocate(out, {B, L, H, D}, type, *q);
        token_tensor(&out, {B, L, H, D}, od);
        if (with_lse) allocate(lse, {B, H, L}, at::kFloat, *q);
        float *lp = lse.defined() ? (float *)lse.data_ptr() : nullptr;
        void *wp = nullptr;
        size_t wn = 0;
        if (wsp) {
            wp = wsp->data_ptr();
            wn = wsp->numel();
        } else if (!noalloc) {
            int32_t most = 0;
            for (int64_t b = 0; b < B; ++b) most = std::max(most, lens.host[b]);
            wn = four ? abi4.step_bytes(B, H, hkv, L, lens.host, nl.host)
               : win.window >= 0 ? wabi.step_bytes(B, H, hkv, L, lens.host, nl.host, win.sinks, win.window)
               : nl.host ? abi.workspace_bytes_varlen(B, H, hkv, L, lens.host, nl.host)
                         : abi.workspace_bytes(WS_OP_STEP, B, H, hkv, L, (int32_t)std::min<int64_t>(most + L, INT32_MAX));
            if (wn) {
                own = at::empty({(int64_t)wn}, q->options().dtype(at::kByte));
                wp = own.data_ptr();
            }
        }
        if (four)
            rc = abi4.fwd(qd, kd, vd, &kv4, lens.host, lens.dev, nl.host, nl.dev, text.host, text.dev, B, L, H, scale, flags,
                          od, lp, wp, wn, stream());
        else if (win.window >= 0)
            rc = wabi.fwd(qd, kd, vd, &kv, lens.host, lens.dev, nl.host, nl.dev, text.host, text.dev, B, L, H, win.sinks,
                          win.window, scale, flags, od, lp, wp, wn, stream());
        else if (noalloc)
            rc = abi.fwd_noalloc(qd, kd, vd, &kv, lens.host, lens.dev, B, L, H, scale, flags, od, lp, stream());
        else if (nl.host)
            rc = abi.fwd_varlen(qd, kd, vd, &kv, lens.host, lens.dev, nl.host, nl.dev, text.host, text.dev, B, L, H, scale,
                                flags, od, lp, wp, wn, stream());
        else if (text.host)
            rc = abi.fwd_text(qd, kd, vd, &kv, lens.host, lens.dev, text.host, text.dev, B, L, H, scale, flags, od, lp, wp,
                              wn, stream());
        else
            rc = abi.fwd(qd, kd, vd, &kv, lens.host, lens.dev, B, L, H, scale, flags, od, lp, wp, wn, stream());
    }
    return result(rc, {out, lse});
}

PyObject *step(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 15) Py_RETURN_NONE;
    return step_of(a, Window{});
    END_HANDLE_TH_ERRORS
}

PyObject *step_window(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Window win;
    if (n != 17 || !window_of(a[15], a[16], win)) Py_RETURN_NONE;
    return step_of(a, win);
    END_HANDLE_TH_ERRORS
}

PyObject *step4(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 15) Py_RETURN_NONE;
    return step_of(a, Window{}, true);
    END_HANDLE_TH_ERRORS
}

// prefill(q, k, v, offsets, scale, cache, num_kv_heads, out, out_dtype,
//         want_lse, lse, text_starts) -> (status, out, lse), or None
// (prefill_window: and window, sinks)
PyObject *prefill_of(PyObject *const *a, const Window &win) {
    new_call();
    const at::Tensor *q = tensor(a[0]);
    if (!q || q->dim() != 4) Py_RETURN_NONE;
    const int64_t B = q->size(0), L = q->size(1), H = q->size(2), D = q->size(3);
    const bool contiguous = a[1] != Py_None;
    if (contiguous != (a[2] != Py_None)) Py_RETURN_NONE;
    Paged kv{};
    ws_tensor4 qd, kd{nullptr, WS_DTYPE_BF16, 0, 0, 0}, vd = kd, od;
    Ints off, text;
    bool want_lse;
    float scale;
    int64_t hkv = 0;
    if (!flag(a[9], want_lse) || !token_tensor(q, {B, L, H, D}, qd) || !scale_of(a[4], D, scale)) Py_RETURN_NONE;
    if (contiguous) {
        const at::Tensor *k = tensor(a[1]);
        if (!k || k->dim() != 4) Py_RETURN_NONE;
        hkv = k->size(2);
        if (!token_tensor(k, {B, L, hkv, D}, kd) || !token_tensor(tensor(a[2]), {B, L, hkv, D}, vd)) Py_RETURN_NONE;
    }
    if (a[5] != Py_None) {
        if (!paged(a[5], contiguous ? 0 : B, kv)) Py_RETURN_NONE;
    } else if (!contiguous) {
        Py_RETURN_NONE;
    }
    if (!contiguous) {
        hkv = kv.num_kv_heads;
        if (a[6] != Py_None) {
            if (!PyLong_CheckExact(a[6])) Py_RETURN_NONE;
            hkv = PyLong_AsLong(a[6]);
        }
    }
    if (!PyTuple_CheckExact(a[3]) || PyTuple_GET_SIZE(a[3]) != 2) Py_RETURN_NONE;
    const at::Tensor *oh = tensor(PyTuple_GET_ITEM(a[3], 0));
    if (!oh || oh->dim() != 2) Py_RETURN_NONE;
    const int64_t nb = oh->size(1) - 1;
    if (nb < 0 || !int_pair(a[3], {B, nb + 1}, false, off) || !int_pair(a[11], {B, nb}, true, text)) Py_RETURN_NONE;
    const at::ScalarType type = a[7] == Py_None ? dtype_of(a[8]) : at::kBFloat16;
    if (type != at::kBFloat16 && type != at::kFloat) Py_RETURN_NONE;
    at::Tensor out, lse;
    const bool with_lse = want_lse || a[10] != Py_None;
    if (!given(a[7], {B, L, H, D}, out) || (out.defined() && !token_tensor(&out, {B, L, H, D}, od)) ||
        !given(a[10], {B, H, L}, lse) || (lse.defined() && !packed_f32(lse)))
        Py_RETURN_NONE;
    const ws_paged_kv *kvp = a[5] != Py_None ? &kv : nullptr;
    int rc;
    {
        NoGil free;
        allocate(out, {B, L, H, D}, type, *q);
        token_tensor(&out, {B, L, H, D}, od);
        if (with_lse) allocate(lse, {B, H, L}, at::kFloat, *q);
        float *lp = lse.defined() ? (float *)lse.data_ptr() : nullptr;
        rc = win.window >= 0 ? wabi.prefill(qd, kd, vd, kvp, off.host, off.dev, text.host, text.dev, B, L, nb, H, hkv, D,
                                            win.sinks, win.window, scale, od, lp, stream())
           : text.host ? abi.prefill_text(qd, kd, vd, kvp, off.host, off.dev, text.host, text.dev, B, L, nb, H, hkv, D, scale,
                                          od, lp, stream())
                       : abi.prefill(qd, kd, vd, kvp, off.host, off.dev, B, L, nb, H, hkv, D, scale, od, lp, stream());
    }
    return result(rc, {out, lse});
}

PyObject *prefill(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 12) Py_RETURN_NONE;
    return prefill_of(a, Window{});
    END_HANDLE_TH_ERRORS
}

PyObject *prefill_window(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Window win;
    if (n != 14 || !window_of(a[12], a[13], win)) Py_RETURN_NONE;
    return prefill_of(a, win);
    END_HANDLE_TH_ERRORS
}

// prefill_bwd(q, k, v, o, dout, lse, offsets, scale, text_starts, dq, dk, dv,
//             workspace) -> (status, dq, dk, dv), or None
// (prefill_window_bwd: and window, sinks, grad_dtype)
PyObject *prefill_bwd_of(PyObject *const *a, const Window &win, at::ScalarType grads) {
    new_call();
    const at::Tensor *q = tensor(a[0]), *k = tensor(a[1]), *lse = tensor(a[5]);
    if (!q || q->dim() != 4 || !k || k->dim() != 4 || !lse) Py_RETURN_NONE;
    const int64_t B = q->size(0), L = q->size(1), H = q->size(2), D = q->size(3), hkv = k->size(2);
    if (B == 0 || L == 0) Py_RETURN_NONE;
    ws_tensor4 qd, kd, vd, od, dd, dqd, dkd, dvd;
    Ints off, text;
    float scale;
    if (!token_tensor(q, {B, L, H, D}, qd) || !token_tensor(k, {B, L, hkv, D}, kd) ||
        !token_tensor(tensor(a[2]), {B, L, hkv, D}, vd) || !token_tensor(tensor(a[3]), {B, L, H, D}, od) ||
        !token_tensor(tensor(a[4]), {B, L, H, D}, dd) || !here(*lse) || !shaped(*lse, {B, H, L}) || !packed_f32(*lse) ||
        !scale_of(a[7], D, scale) || !PyTuple_CheckExact(a[6]) || PyTuple_GET_SIZE(a[6]) != 2)
        Py_RETURN_NONE;
    const at::Tensor *oh = tensor(PyTuple_GET_ITEM(a[6], 0));
    if (!oh || oh->dim() != 2) Py_RETURN_NONE;
    const int64_t nb = oh->size(1) - 1;
    if (nb < 0 || !int_pair(a[6], {B, nb + 1}, false, off) || !int_pair(a[8], {B, nb}, true, text)) Py_RETURN_NONE;
    const at::Tensor *wsp = a[12] == Py_None ? nullptr : tensor(a[12]);
    if (a[12] != Py_None && !packed(wsp, 0)) Py_RETURN_NONE;
    at::Tensor dq, dk, dv, own;
    if (!given(a[9], {B, L, H, D}, dq) || (dq.defined() && !token_tensor(&dq, {B, L, H, D}, dqd)) ||
        !given(a[10], {B, L, hkv, D}, dk) || (dk.defined() && !token_tensor(&dk, {B, L, hkv, D}, dkd)) ||
        !given(a[11], {B, L, hkv, D}, dv) || (dv.defined() && !token_tensor(&dv, {B, L, hkv, D}, dvd)))
        Py_RETURN_NONE;
    int rc = -1;
    {
        NoGil free;
        const size_t need = wsp ? 0
                          : win.window >= 0 ? wabi.bwd_bytes(B, H, hkv, L, win.sinks, win.window)
                                            : abi.workspace_bytes(WS_OP_PREFILL_BWD, B, H, hkv, L, L);
        if (wsp || need) {
            allocate(dq, {B, L, H, D}, grads, *q);
            allocate(dk, {B, L, hkv, D}, grads, *q);
            allocate(dv, {B, L, hkv, D}, grads, *q);
            token_tensor(&dq, {B, L, H, D}, dqd);
            token_tensor(&dk, {B, L, hkv, D}, dkd);
            token_tensor(&dv, {B, L, hkv, D}, dvd);
            if (!wsp) {
                own = at::empty({(int64_t)need}, q->options().dtype(at::kByte));
                wsp = &own;
            }
            const float *lp = (const float *)lse->data_ptr();
            if (win.window >= 0)
                rc = wabi.bwd(qd, kd, vd, od, dd, lp, off.host, off.dev, text.host, text.dev, B, L, nb, H, hkv, D, win.sinks,
                              win.window, scale, dqd, dkd, dvd, wsp->data_ptr(), wsp->numel(), stream());
            else
                rc = abi.bwd(qd, kd, vd, od, dd, lp, off.host, off.dev, text.host, text.dev, B, L, nb, H, hkv, D, scale, dqd, dkd,
                             dvd, wsp->data_ptr(), wsp->numel(), stream());
        }
    }
    if (rc < 0) Py_RETURN_NONE;   // (the Python code names the mistake)
    return result(rc, {dq, dk, dv});
}

PyObject *prefill_bwd(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 13) Py_RETURN_NONE;
    return prefill_bwd_of(a, Window{}, at::kFloat);
    END_HANDLE_TH_ERRORS
}

PyObject *prefill_window_bwd(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Window win;
    if (n != 16 || !window_of(a[13], a[14], win)) Py_RETURN_NONE;
    return prefill_bwd_of(a, win, dtype_of(a[15]));
    END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"bind", (PyCFunction)(void (*)())bind, METH_FASTCALL, "the cache class, then the C ABI's addresses in Abi's order"},
    {"bind_window", (PyCFunction)(void (*)())bind_window, METH_FASTCALL, "the windowed ABI's addresses in WindowAbi's order"},
    {"bind_cache4", (PyCFunction)(void (*)())bind_cache4, METH_FASTCALL, "PagedCache4, then the 4-bit ABI's addresses"},
    {"append4", (PyCFunction)(void (*)())append4, METH_FASTCALL, nullptr},
    {"read4", (PyCFunction)(void (*)())read4, METH_FASTCALL, nullptr},
    {"step4", (PyCFunction)(void (*)())step4, METH_FASTCALL, nullptr},
    {"step_window", (PyCFunction)(void (*)())step_window, METH_FASTCALL, nullptr},
    {"prefill_window", (PyCFunction)(void (*)())prefill_window, METH_FASTCALL, nullptr},
    {"prefill_window_bwd", (PyCFunction)(void (*)())prefill_window_bwd, METH_FASTCALL, nullptr},
    {"append", (PyCFunction)(void (*)())append, METH_FASTCALL, nullptr},
    {"step", (PyCFunction)(void (*)())step, METH_FASTCALL, nullptr},
    {"prefill", (PyCFunction)(void (*)())prefill, METH_FASTCALL, nullptr},
    {"prefill_bwd", (PyCFunction)(void (*)())prefill_bwd, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_wsbinding", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__wsbinding() {
    const char *n[7] = {"k_pool", "v_pool", "page_table_host", "page_table", "num_pages", "num_kv_heads", "head_dim"};
    for (int i = 0; i < 7; ++i)
        if (!(names[i] = PyUnicode_InternFromString(n[i]))) return nullptr;
    if (!(pool_name = PyUnicode_InternFromString("pool"))) return nullptr;
    return PyModule_Create(&module);
}
