// Python calls of the paged functions without ctypes: checks of tensors, outputs and scratch from torch's allocator, the
// current stream, one call into libsubgen.so (whose addresses bind() takes). A call through ctypes costs 11 us on the
// host, more than the small kernels themselves; this one about half. Everything public is in binding.py.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>
#include <utility>
#include <stdexcept>
#include <string>

#include "../../include/subgen.h"

namespace {

decltype(&subgen_qk_norm_rope) f_qk;
decltype(&subgen_paged_append) f_append;
decltype(&subgen_paged_attend) f_attend;
decltype(&subgen_paged_workspace_bytes) f_bytes;
decltype(&subgen_paged4_append) f_append4;
decltype(&subgen_paged4_load) f_load4;
decltype(&subgen_paged4_attend) f_attend4;
decltype(&subgen_paged4_workspace_bytes) f_bytes4;
decltype(&subgen_page_step) f_step;
decltype(&subgen_last_error) f_error;
PyObject* g_error;                                    // SubgenError

struct Refused : std::runtime_error { using std::runtime_error::runtime_error; };      // -> ValueError
struct Failed : std::runtime_error { using std::runtime_error::runtime_error; };       // -> SubgenError

[[noreturn]] void refuse(const std::string& what) { throw Refused(what); }
void check(int rc) {
    if (rc < 0) throw Failed("subgen error " + std::to_string(rc) + ": " + f_error());
}

const at::Tensor* tensor(PyObject* o, const char* name) {             // NULL for None
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) refuse(std::string(name) + " must be a tensor");
    return &THPVariable_Unpack(o);
}
std::string said(const at::Tensor& x) {
    std::string s = "(";
    for (int64_t k : x.sizes()) s += std::to_string(k) + ",";
    return "(got " + std::string(at::toString(x.scalar_type())) + " " + s + ") on " + x.device().str() + ")";
}
struct Like {                                         // what every tensor of a call has in common
    at::ScalarType type;
    int device;
};
Like like(const at::Tensor& x, const char* name) {
    if (!x.is_cuda()) refuse(std::string(name) + " must be a CUDA tensor: this library has no CPU path");
    if (x.scalar_type() != at::kFloat && x.scalar_type() != at::kBFloat16) refuse("dtype must be torch.float32 or torch.bfloat16");
    if (x.dim() != 3) refuse(std::string(name) + " must have the axes tokens, heads, d " + said(x));
    return Like{x.scalar_type(), (int)x.get_device()};
}
subgen_heads rows(const at::Tensor& x, const char* name, const Like& w, int64_t n, int64_t heads, int64_t d) {
    if (x.scalar_type() != w.type || !x.is_cuda() || x.get_device() != w.device || x.dim() != 3 || x.size(0) != n || x.size(1) != heads ||
        x.size(2) != d || x.stride(2) != 1)
        refuse(std::string(name) + " must be a " + at::toString(w.type) + " tensor of shape (" + std::to_string(n) + "," + std::to_string(heads) + "," +
               std::to_string(d) + ") on cuda:" + std::to_string(w.device) + " with unit stride along the last axis " + said(x));
    if (n > INT_MAX || heads > INT_MAX) refuse(std::string(name) + ": too many rows");
    return subgen_heads{x.data_ptr(), x.stride(0), x.stride(1)};
}
const void* whole(PyObject* o, const char* name, at::ScalarType type, int device, int64_t n) {
    const at::Tensor* x = tensor(o, name);
    if (!x) return nullptr;
    if (x->scalar_type() != type || !x->is_cuda() || x->get_device() != device || x->dim() != 1 || x->size(0) != n || !x->is_contiguous())
        refuse(std::string(name) + " must be a contiguous " + at::toString(type) + " tensor of shape (" + std::to_string(n) + ",) on cuda:" +
               std::to_string(device) + " " + said(*x));
    return x->data_ptr();
}
// The output that was given, or a new one; `o` becomes a new reference to it.
subgen_heads output(PyObject*& o, const char* name, const at::Tensor& from, const Like& w, int64_t n, int64_t heads, int64_t d) {
    if (const at::Tensor* x = tensor(o, name)) {
        const subgen_heads h = rows(*x, name, w, n, heads, d);
        Py_INCREF(o);
        return h;
    }
    at::Tensor y = at::empty({n, heads, d}, from.options());
    const subgen_heads h{y.data_ptr(), heads * d, d};
    o = THPVariable_Wrap(std::move(y));
    if (!o) throw std::bad_alloc();
    return h;
}
// A tensor of its own in a part of another's memory, from byte `at` on: several outputs of one allocation, each of which (with the
// checks and bookkeeping that torch's dispatcher does for a view) would cost a microsecond on the host.
at::Tensor part_of(const at::Tensor& all, at::ScalarType type, at::IntArrayRef sizes, int64_t at) {
    const c10::Storage storage = all.storage();
    at::Tensor x = at::detail::make_tensor<c10::TensorImpl>(c10::TensorImpl::VIEW, c10::Storage(storage), all.key_set(), c10::scalarTypeToTypeMeta(type));
    x.unsafeGetTensorImpl()->set_storage_offset(at / (int64_t)c10::elementSize(type));
    x.unsafeGetTensorImpl()->set_sizes_contiguous(sizes);
    return x;
}
PyObject* wrapped(at::Tensor x) {
    PyObject* o = THPVariable_Wrap(std::move(x));
    if (!o) throw std::bad_alloc();
    return o;
}
int dtype_of(const Like& w) { return w.type == at::kFloat ? SUBGEN_DTYPE_FP32 : SUBGEN_DTYPE_BF16; }
int integer(PyObject* o) {
    const long x = PyLong_AsLong(o);
    if (x == -1 && PyErr_Occurred()) { PyErr_Clear(); refuse("a whole number is wanted"); }
    if (x < INT_MIN || x > INT_MAX) refuse("a whole number below 2^31 is wanted");
    return (int)x;
}
float real(PyObject* o) {
    const double x = PyFloat_AsDouble(o);
    if (x == -1.0 && PyErr_Occurred()) { PyErr_Clear(); refuse("a number is wanted"); }
    return (float)x;
}
bool truth(PyObject* o, const char* name) {
    const int x = PyObject_IsTrue(o);
    if (x < 0) { PyErr_Clear(); refuse(std::string(name) + " has no truth value"); }
    return x != 0;
}
// rope: None or (words, rotary_dim, interleaved, d, device)
subgen_rope rope_of(PyObject* o, int64_t d, int device) {
    if (o == Py_None) return subgen_rope{nullptr, 0, 0};
    if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 5) refuse("rope must be a Rope");
    if (integer(PyTuple_GET_ITEM(o, 3)) != d || integer(PyTuple_GET_ITEM(o, 4)) != device)
        refuse("rope was made for d = " + std::to_string(integer(PyTuple_GET_ITEM(o, 3))) + " on device " + std::to_string(integer(PyTuple_GET_ITEM(o, 4))));
    return subgen_rope{(const uint64_t*)PyLong_AsVoidPtr(PyTuple_GET_ITEM(o, 0)), integer(PyTuple_GET_ITEM(o, 1)), integer(PyTuple_GET_ITEM(o, 2))};
}

// New references that a call holds until it has gone well.
struct Held {
    PyObject* o;
    bool mine = false;
    explicit Held(PyObject* x) : o(x) {}
    ~Held() { if (mine) Py_XDECREF(o); }
    PyObject* release() {
        if (!mine) Py_INCREF(o);
        mine = false;
        return o;
    }
};

template <typename F>
PyObject* guarded(F f) {
    if (!f_qk) { PyErr_SetString(PyExc_RuntimeError, "the library is not loaded"); return nullptr; }
    try {
        return f();
    } catch (const Refused& e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const Failed& e) {
        PyErr_SetString(g_error, e.what());
    } catch (...) {                                   // torch's own: out of memory and the like
        if (!PyErr_Occurred()) torch::translate_exception_to_python(std::current_exception());
    }
    return nullptr;
}

bool count(Py_ssize_t got, Py_ssize_t want) {
    if (got == want) return true;
    PyErr_Format(PyExc_TypeError, "%zd arguments are wanted, %zd were given", want, got);
    return false;
}

// (q, k, positions, rope, wq, wk, eps, q_out, k_out) -> (q_out, k_out)
PyObject* qk_norm_rope(PyObject*, PyObject* const* a, Py_ssize_t got) {
    if (!count(got, 9)) return nullptr;
    return guarded([&]() -> PyObject* {
        const at::Tensor *q = tensor(a[0], "q"), *k = tensor(a[1], "k");
        const at::Tensor* x = q ? q : k;
        if (!x) refuse("q and k must not both be None");
        const Like w = like(*x, q ? "q" : "k");
        const int64_t n = x->size(0), d = x->size(2);
        const c10::cuda::CUDAGuard on((c10::DeviceIndex)w.device);
        subgen_qk_args p{};
        Held qo(q ? a[7] : Py_None), ko(k ? a[8] : Py_None);
        p.H = p.Hkv = 1;
        if (q) {
            p.H = (int)q->size(1);
            p.q = rows(*q, "q", w, n, p.H, d);
            p.q_out = output(qo.o, "q_out", *q, w, n, p.H, d);
            qo.mine = true;
        }
        if (k) {
            if (k->dim() != 3) refuse("k must have the axes tokens, heads, d " + said(*k));
            p.Hkv = (int)k->size(1);
            p.k = rows(*k, "k", w, n, p.Hkv, d);
            p.k_out = output(ko.o, "k_out", *k, w, n, p.Hkv, d);
            ko.mine = true;
        }
        p.positions = (const int*)whole(a[2], "positions", at::kInt, w.device, n);
        p.rope = rope_of(a[3], d, w.device);
        p.wq = whole(a[4], "wq", w.type, w.device, d);
        p.wk = whole(a[5], "wk", w.type, w.device, d);
        p.n = (int)n; p.d = (int)d; p.dtype = dtype_of(w); p.eps = real(a[6]);
        check(f_qk(&p, c10::cuda::getCurrentCUDAStream(w.device).stream()));
        PyObject* both = PyTuple_New(2);
        if (!both) throw std::bad_alloc();
        PyTuple_SET_ITEM(both, 0, qo.release());
        PyTuple_SET_ITEM(both, 1, ko.release());
        return both;
    });
}

const subgen_pages* cache_at(PyObject* o) { return (const subgen_pages*)PyLong_AsVoidPtr(o); }
const subgen_batch* batch_at(PyObject* o) { return (const subgen_batch*)PyLong_AsVoidPtr(o); }

const subgen_pages4* cache4_at(PyObject* o) { return (const subgen_pages4*)PyLong_AsVoidPtr(o); }

// call(args) appends; `w`: type and device of the tensors
template <typename F>
PyObject* append_with(PyObject* const* a, const Like& w, int Hkv, int64_t d, F call) {
    const at::Tensor *k = tensor(a[3], "k"), *v = tensor(a[4], "v"), *q = tensor(a[9], "q");
    if (!k || !v || k->dim() != 3) refuse("k and v must have the axes tokens, heads, d");
    const int64_t n = k->size(0);
    const c10::cuda::CUDAGuard on((c10::DeviceIndex)w.device);
    subgen_qk_args p{};
    p.k = rows(*k, "k", w, n, Hkv, d);
    p.v = rows(*v, "v", w, n, Hkv, d);
    Held qo(q ? a[11] : Py_None);
    p.H = 1;
    if (q) {
        if (q->dim() != 3) refuse("q must have the axes tokens, heads, d " + said(*q));
        p.H = (int)q->size(1);
        p.q = rows(*q, "q", w, n, p.H, d);
        p.fresh = qo.o == Py_None;
        p.q_out = output(qo.o, "q_out", *q, w, n, p.H, d);
        qo.mine = true;
    }
    p.positions = (const int*)whole(a[5], "positions", at::kInt, w.device, n);
    p.rope = rope_of(a[6], d, w.device);
    p.wk = whole(a[7], "wk", w.type, w.device, d);
    p.wq = whole(a[10], "wq", w.type, w.device, d);
    p.n = (int)n; p.eps = real(a[8]); p.dtype = dtype_of(w);
    check(call(&p, c10::cuda::getCurrentCUDAStream(w.device).stream()));
    return qo.release();
}

// call(args) attends; bytes(n, H): of the workspace
template <typename B, typename F>
PyObject* attend_with(PyObject* const* a, const at::Tensor& q, const Like& w, int64_t d, B bytes, F call) {
    const int64_t n = q.size(0), H = q.size(1);
    const c10::cuda::CUDAGuard on((c10::DeviceIndex)w.device);
    subgen_attend_args p{};
    p.q = rows(q, "q", w, n, H, d);
    Held out(a[6]);
    p.fresh = out.o == Py_None;
    p.out = output(out.o, "out", q, w, n, H, d);
    out.mine = true;
    p.workspace_bytes = bytes((int)n, (int)H);
    if (!p.workspace_bytes) throw Failed(f_error());
    const at::Tensor space = at::empty({(int64_t)p.workspace_bytes}, q.options().dtype(at::kByte));   // torch aligns to 512 bytes
    p.workspace = space.data_ptr();
    p.n = (int)n; p.H = (int)H; p.scale = real(a[4]); p.causal = truth(a[5], "causal");
    check(call(&p, c10::cuda::getCurrentCUDAStream(w.device).stream()));
    return out.release();
}

// (cache, device, batch, k, v, positions, rope, wk, eps, q, wq, q_out) -> q_out or None; cache, batch: addresses of descriptors
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t got) {
    if (!count(got, 12)) return nullptr;
    return guarded([&]() -> PyObject* {
        const subgen_pages* c = cache_at(a[0]);
        const Like w{c->dtype == SUBGEN_DTYPE_FP32 ? at::kFloat : at::kBFloat16, integer(a[1])};
        return append_with(a, w, c->Hkv, c->d, [&](const subgen_qk_args* p, void* st) { return f_append(c, batch_at(a[2]), p, st); });
    });
}

// the same for a cache in 4 bits
PyObject* append4(PyObject*, PyObject* const* a, Py_ssize_t got) {
    if (!count(got, 12)) return nullptr;
    return guarded([&]() -> PyObject* {
        const subgen_pages4* c = cache4_at(a[0]);
        const at::Tensor* k = tensor(a[3], "k");
        if (!k) refuse("k and v must have the axes tokens, heads, d");
        const Like w{like(*k, "k").type, integer(a[1])};
        return append_with(a, w, c->Hkv, c->d, [&](const subgen_qk_args* p, void* st) { return f_append4(c, batch_at(a[2]), p, st); });
    });
}

// (cache, device, batch, q, scale, causal, out) -> out
PyObject* attend(PyObject*, PyObject* const* a, Py_ssize_t got) {
    if (!count(got, 7)) return nullptr;
    return guarded([&]() -> PyObject* {
        const subgen_pages* c = cache_at(a[0]);
        const subgen_batch* b = batch_at(a[2]);
        const Like w{c->dtype == SUBGEN_DTYPE_FP32 ? at::kFloat : at::kBFloat16, integer(a[1])};
        const at::Tensor* q = tensor(a[3], "q");
        if (!q || q->dim() != 3) refuse("q must have the axes tokens, heads, d");
        return attend_with(a, *q, w, c->d, [&](int n, int H) { return f_bytes(c, b, n, H); },
                           [&](const subgen_attend_args* p, void* st) { return f_attend(c, b, p, st); });
    });
}

// the same for a cache in 4 bits
PyObject* attend4(PyObject*, PyObject* const* a, Py_ssize_t got) {
    if (!count(got, 7)) return nullptr;
    return guarded([&]() -> PyObject* {
        const subgen_pages4* c = cache4_at(a[0]);
        const subgen_batch* b = batch_at(a[2]);
        const at::Tensor* q = tensor(a[3], "q");
        if (!q) refuse("q must have the axes tokens, heads, d");
        const Like w{like(*q, "q").type, integer(a[1])};
        return attend_with(a, *q, w, c->d, [&](int n, int H) { return f_bytes4(c, b, n, H); },
                           [&](const subgen_attend_args* p, void* st) { return f_attend4(c, b, p, dtype_of(w), st); });
    });
}

// (cache, device, slots, dtype code, K or None, V or None) -> (K, V)
PyObject* load4(PyObject*, PyObject* const* a, Py_ssize_t got) {
    if (!count(got, 6)) return nullptr;
    return guarded([&]() -> PyObject* {
        const subgen_pages4* c = cache4_at(a[0]);
        const Like w{integer(a[3]) == SUBGEN_DTYPE_FP32 ? at::kFloat : at::kBFloat16, integer(a[1])};
        const at::Tensor* slots = tensor(a[2], "slots");
        if (!slots || slots->dim() != 1) refuse("slots must be a tensor of one axis");
        const int64_t n = slots->size(0);
        if (n > INT_MAX) refuse("slots: too many rows");
        const c10::cuda::CUDAGuard on((c10::DeviceIndex)w.device);
        const void* at_slots = whole(a[2], "slots", at::kLong, w.device, n);
        const bool new_k = a[4] == Py_None, new_v = a[5] == Py_None;
        const int64_t bytes = n * c->Hkv * c->d * (int64_t)c10::elementSize(w.type);        // (a multiple of 64)
        at::Tensor both_new;
        if (new_k || new_v) both_new = at::empty({bytes * (new_k + new_v)}, slots->options().dtype(at::kByte));
        auto out = [&](PyObject* o, const char* name, int64_t at) {
            Held h(o);
            if (o == Py_None) h.o = wrapped(part_of(both_new, w.type, {n, c->Hkv, c->d}, at));
            else Py_INCREF(o);
            h.mine = true;
            const subgen_heads lies = rows(*tensor(h.o, name), name, w, n, c->Hkv, c->d);           // before the release: it may refuse
            return std::make_pair(lies, h.release());
        };
        const auto [hk, ko] = out(a[4], "K", 0);
        Held k(ko);
        k.mine = true;
        const auto [hv, vo] = out(a[5], "V", new_k ? bytes : 0);
        Held v(vo);
        v.mine = true;
        check(f_load4(c, (const int64_t*)at_slots, (int)n, &hk, &hv, dtype_of(w), c10::cuda::getCurrentCUDAStream(w.device).stream()));
        PyObject* both = PyTuple_New(2);
        if (!both) throw std::bad_alloc();
        PyTuple_SET_ITEM(both, 0, k.release());
        PyTuple_SET_ITEM(both, 1, v.release());
        return both;
    });
}

// (lengths, table, free, free_count, added, page, n, ended, first, lengths_out, free_count_out, cu_q, slots, positions, status,
// sources) -> (cu_q, lengths_out, free_count_out, slots, positions); outputs among these that are None are made
PyObject* page_step(PyObject*, PyObject* const* a, Py_ssize_t got) {
    if (!count(got, 16)) return nullptr;
    return guarded([&]() -> PyObject* {
        const at::Tensor *lengths = tensor(a[0], "lengths"), *table = tensor(a[1], "table"), *free = tensor(a[2], "free");
        if (!lengths || !table || !free || lengths->dim() != 1 || table->dim() != 2 || free->dim() != 1) refuse("lengths, table and free must be tensors of one, two and one axes");
        if (!lengths->is_cuda()) refuse("lengths must be a CUDA tensor: this library has no CPU path");
        const int dev = (int)lengths->get_device();
        const int64_t B = lengths->size(0), n = integer(a[6]);
        const c10::cuda::CUDAGuard on((c10::DeviceIndex)dev);
        if (table->scalar_type() != at::kInt || !table->is_cuda() || table->get_device() != dev || table->size(0) != B || !table->is_contiguous() || table->size(1) > INT_MAX)
            refuse("table must be a contiguous Int tensor with " + std::to_string(B) + " rows on cuda:" + std::to_string(dev) + " " + said(*table));
        if (B > INT_MAX || free->size(0) > INT_MAX || n < 0) refuse("lengths, free and n must be in range");
        subgen_page_step_args p{};
        p.B = (int)B; p.n = (int)n; p.page = integer(a[5]); p.pages = (int)free->size(0); p.table_stride = (int)table->size(1);
        p.lengths = (const int*)whole(a[0], "lengths", at::kInt, dev, B);
        p.table = (int*)table->data_ptr();
        p.free_pages = (int*)whole(a[2], "free", at::kInt, dev, p.pages);
        p.free_count = (const int*)whole(a[3], "free_count", at::kInt, dev, 1);
        p.added = (const int*)whole(a[4], "added", at::kInt, dev, B);
        p.ended = (const int*)whole(a[7], "ended", at::kInt, dev, B);
        p.first = (const int*)whole(a[8], "first", at::kInt, dev, B);
        p.status = (int*)whole(a[14], "status", at::kInt, dev, 1);
        p.sources = (int*)whole(a[15], "sources", at::kInt, dev, n);
        PyObject* five = PyTuple_New(5);
        if (!five) throw std::bad_alloc();
        Held held(five);
        held.mine = true;
        at::Tensor all;                               // slots first: 8-byte aligned
        int64_t at_byte = 0;
        auto out = [&](int i, PyObject* o, const char* name, at::ScalarType type, int64_t count) {
            if (o == Py_None) {
                if (!all.defined()) all = at::empty({8 * n + 4 * (n + 2 * B + 2)}, lengths->options().dtype(at::kByte));
                o = wrapped(part_of(all, type, {count}, at_byte));
                at_byte += count * (int64_t)c10::elementSize(type);
            } else {
                Py_INCREF(o);
            }
            PyTuple_SET_ITEM(five, i, o);
            return const_cast<void*>(whole(o, name, type, dev, count));
        };
        p.slots = (int64_t*)out(3, a[12], "slots", at::kLong, n);
        p.cu_q = (int*)out(0, a[11], "cu_q", at::kInt, B + 1);
        p.lengths_out = (int*)out(1, a[9], "lengths_out", at::kInt, B);
        p.free_count_out = (int*)out(2, a[10], "free_count_out", at::kInt, 1);
        p.positions = (int*)out(4, a[13], "positions", at::kInt, n);
        check(f_step(&p, c10::cuda::getCurrentCUDAStream(dev).stream()));
        return held.release();
    });
}

// (SubgenError, addresses of subgen_qk_norm_rope, _paged_append, _paged_attend, _paged_workspace_bytes, the same three of paged4 and
// _paged4_load behind the first, _page_step, _last_error)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t got) {
    if (!count(got, 11)) return nullptr;
    void* p[10];
    for (int i = 0; i < 10; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i + 1]);
        if (!p[i]) { if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "a null address"); return nullptr; }
    }
    Py_INCREF(a[0]);
    Py_XSETREF(g_error, a[0]);
    f_qk = (decltype(f_qk))p[0]; f_append = (decltype(f_append))p[1]; f_attend = (decltype(f_attend))p[2];
    f_bytes = (decltype(f_bytes))p[3];
    f_append4 = (decltype(f_append4))p[4]; f_load4 = (decltype(f_load4))p[5]; f_attend4 = (decltype(f_attend4))p[6];
    f_bytes4 = (decltype(f_bytes4))p[7]; f_step = (decltype(f_step))p[8]; f_error = (decltype(f_error))p[9];
    Py_RETURN_NONE;
}

#define ENTRY(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(bind), ENTRY(qk_norm_rope), ENTRY(append), ENTRY(attend),
                         ENTRY(append4), ENTRY(load4), ENTRY(attend4), ENTRY(page_step), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() {
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_for", SUBGEN_BUILT_FOR)) Py_CLEAR(m);      // "built for <torch, python>", see build.py
    return m;
}
