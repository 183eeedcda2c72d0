// Python calls of the entry points without ctypes: torch tensors, numbers and ctypes structures in, the C ABI called, its
// status out.  A decode round makes dozens of calls of up to 20 arguments, and the commit takes the caches of every layer: the
// three attribute lookups per tensor from Python took 22 us for 96 caches, more than the kernels of the call.
//
// Every wrapper follows from the entry point's own signature (one template).  A pointer is a device pointer: it takes a contiguous
// tensor on the GPU or None, and nothing else, so that host memory never reaches a kernel as one.  The exceptions have types of
// their own: the descriptors (ctypes structures), host out-parameters (ENTRY_HOST names their position) and the stream (always the
// last argument, a raw handle).  An array of pointers takes a sequence of tensors, the projection jobs a sequence of sequences; size_t
// takes an integer or a tensor (its bytes); the rest are numbers.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <c10/core/impl/VirtualGuardImpl.h>
#include <cstdint>
#include <exception>
#include <tuple>
#include <utility>
#include <vector>
#include "dream.h"

namespace {

struct Failed {};     // a Python exception has been set

void *device_pointer(PyObject *o)
{
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda()) {
        PyErr_SetString(PyExc_ValueError, "device tensor expected");
        throw Failed();
    }
    if (!t.is_contiguous()) {
        PyErr_SetString(PyExc_ValueError, "contiguous tensor expected");
        throw Failed();
    }
    return t.data_ptr();
}

// One argument of type T, alive as long as the call.
template <class T>
struct Arg {
    static_assert(std::is_integral_v<T>, "numbers");
    T value;
    explicit Arg(PyObject *o)
    {
        if (std::is_same_v<T, size_t> && THPVariable_Check(o)) {
            value = (T)THPVariable_Unpack(o).nbytes();
            return;
        }
        const unsigned long long v = PyLong_AsUnsignedLongLongMask(o);
        if (PyErr_Occurred())
            throw Failed();
        value = (T)v;
    }
};
template <>
struct Arg<float> {
    float value;
    explicit Arg(PyObject *o) : value((float)PyFloat_AsDouble(o))
    {
        if (PyErr_Occurred())
            throw Failed();
    }
};
template <class T>
struct Arg<T *> {
    T *value = nullptr;
    explicit Arg(PyObject *o)
    {
        if (o == Py_None)
            return;
        if (!THPVariable_Check(o)) {
            PyErr_Format(PyExc_TypeError, "device tensor or None expected, not %.100s", Py_TYPE(o)->tp_name);
            throw Failed();
        }
        value = static_cast<T *>(device_pointer(o));
    }
};

// Host memory of exactly one T, through the buffer interface (ctypes structures and numbers are writable buffers).
template <class T>
struct HostObject {
    T *value = nullptr;
    Py_buffer view = {};
    explicit HostObject(PyObject *o, bool nullable)
    {
        if (nullable && o == Py_None)
            return;
        if (PyObject_GetBuffer(o, &view, PyBUF_WRITABLE))
            throw Failed();
        if (view.len != (Py_ssize_t)sizeof(T)) {
            PyBuffer_Release(&view);
            PyErr_Format(PyExc_TypeError, "an object of %d bytes is expected", (int)sizeof(T));
            throw Failed();
        }
        value = static_cast<T *>(view.buf);
    }
    ~HostObject()
    {
        if (view.obj)
            PyBuffer_Release(&view);
    }
    HostObject(const HostObject &) = delete;
};
template <>
struct Arg<const dream_attn_desc *> : HostObject<dream_attn_desc> {
    explicit Arg(PyObject *o) : HostObject(o, false) {}
};
template <>
struct Arg<const dream_page_desc *> : HostObject<dream_page_desc> {
    explicit Arg(PyObject *o) : HostObject(o, false) {}
};
struct HostInt : HostObject<int32_t> {
    explicit HostInt(PyObject *o) : HostObject(o, true) {}
};
struct Stream {
    void *value;
    explicit Stream(PyObject *o) : value(PyLong_AsVoidPtr(o))
    {
        if (PyErr_Occurred())
            throw Failed();
    }
};

template <>
struct Arg<void *const *> {
    std::vector<void *> pointers;
    void *const *value;
    explicit Arg(PyObject *o)
    {
        PyObject *seq = PySequence_Fast(o, "a sequence of tensors is expected");
        if (!seq)
            throw Failed();
        try {
            const Py_ssize_t n = PySequence_Fast_GET_SIZE(seq);
            pointers.reserve(n);
            for (Py_ssize_t i = 0; i < n; i++) {
                PyObject *t = PySequence_Fast_GET_ITEM(seq, i);
                if (!THPVariable_Check(t)) {
                    PyErr_SetString(PyExc_TypeError, "a sequence of tensors is expected");
                    throw Failed();
                }
                pointers.push_back(device_pointer(t));
            }
        } catch (...) {
            Py_DECREF(seq);
            throw;
        }
        Py_DECREF(seq);
        value = pointers.data();
    }
};

// A sequence of jobs, each a sequence of as many fields as the job has.
inline int32_t number(PyObject *o) { return Arg<int32_t>(o).value; }
inline void *pointer(PyObject *o) { return Arg<void *>(o).value; }
inline int32_t *pointer32(PyObject *o) { return static_cast<int32_t *>(pointer(o)); }
struct ProjFields {     // (x, w, n_heads, row_base, row_index, out)
    static constexpr const char *what = "a job is (x, w, n_heads, row_base, row_index, out)";
    static constexpr Py_ssize_t n = 6;
    static dream_proj_job job(PyObject *const *f) { return {pointer(f[0]), pointer(f[1]), number(f[2]), pointer32(f[3]), pointer32(f[4]), pointer(f[5])}; }
};
struct RotaryFields {
    static constexpr const char *what = "a job is (x, n_heads, row_base, row_index, out)";
    static constexpr Py_ssize_t n = 5;
    static dream_rotary_job job(PyObject *const *f) { return {pointer(f[0]), number(f[1]), pointer32(f[2]), pointer32(f[3]), pointer(f[4])}; }
};
template <class Job, class Fields>
struct Jobs {
    std::vector<Job> jobs;
    const Job *value;
    explicit Jobs(PyObject *o)
    {
        PyObject *seq = PySequence_Fast(o, "a sequence of jobs is expected");
        if (!seq)
            throw Failed();
        try {
            const Py_ssize_t n = PySequence_Fast_GET_SIZE(seq);
            for (Py_ssize_t i = 0; i < n; i++) {
                // (a tuple of its own: converting a field may run Python code, which must not take the others away)
                struct Owned {
                    PyObject *o;
                    ~Owned() { Py_XDECREF(o); }
                } job = {PySequence_Tuple(PySequence_Fast_GET_ITEM(seq, i))};
                if (!job.o)
                    throw Failed();
                if (PyTuple_GET_SIZE(job.o) != Fields::n) {
                    PyErr_SetString(PyExc_ValueError, Fields::what);
                    throw Failed();
                }
                PyObject *fields[Fields::n];
                for (Py_ssize_t k = 0; k < Fields::n; k++)
                    fields[k] = PyTuple_GET_ITEM(job.o, k);
                jobs.push_back(Fields::job(fields));
            }
        } catch (...) {
            Py_DECREF(seq);
            throw;
        }
        Py_DECREF(seq);
        value = jobs.data();
    }
};
template <>
struct Arg<const dream_proj_job *> : Jobs<dream_proj_job, ProjFields> {
    using Jobs::Jobs;
};
template <>
struct Arg<const dream_rotary_job *> : Jobs<dream_rotary_job, RotaryFields> {
    using Jobs::Jobs;
};

struct WithoutGil {
    PyThreadState *state = PyEval_SaveThread();
    ~WithoutGil() { PyEval_RestoreThread(state); }
};

// What the rotary, 4-bit, window and paged calls want of their tensors, checked before the call: the type, at least so many values, and the current device (the one the call is made on).  A
// None is the library's to accept or refuse, and so are sizes that are not positive.
thread_local c10::DeviceIndex current_device = -1;      // of this call; -1: not asked for yet (Sizes)
void want(PyObject *o, const char *name, __int128 values, at::ScalarType type, at::ScalarType also)
{
    if (!THPVariable_Check(o))
        return;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda())
        return;     // (refused where it is converted)
    if (t.scalar_type() != type && t.scalar_type() != also) {
        PyErr_Format(PyExc_ValueError, "%s: %s expected, not %s", name, c10::toString(type), c10::toString(t.scalar_type()));
        throw Failed();
    }
    if ((__int128)t.numel() < values) {
        PyErr_Format(PyExc_ValueError, "%s: %lld values expected, not %lld", name, (long long)values, (long long)t.numel());
        throw Failed();
    }
    if (current_device < 0)
        current_device = c10::impl::VirtualGuardImpl(c10::DeviceType::CUDA).getDevice().index();
    if (t.device().index() != current_device) {
        PyErr_Format(PyExc_ValueError, "%s: is not on the current device", name);
        throw Failed();
    }
}
void want(PyObject *o, const char *name, __int128 values, at::ScalarType type) { want(o, name, values, type, type); }
void want_all(PyObject *seq, const char *name, __int128 values, at::ScalarType type)
{
    if (!PyTuple_Check(seq))
        return;     // (the binding hands over tuples)
    for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(seq); i++)
        want(PyTuple_GET_ITEM(seq, i), name, values, type);
}

using Args = PyObject *const *;
struct Unchecked {
    static void check(Args) {}
};
struct Sizes {
    dream_attn_desc d = {};
    at::ScalarType type;
    __int128 b, hq, hkv, dim, row, cache;      // row: of a cache, in values
    explicit Sizes(PyObject *o)
    {
        const Arg<const dream_attn_desc *> desc(o);
        d = *desc.value;
        current_device = -1;
        type = d.dtype == DREAM_F32 ? at::kFloat : at::kBFloat16;
        b = d.batch; hq = d.n_q_heads; hkv = d.n_kv_heads; dim = d.head_dim;
        row = b * hkv * d.s_max;
        cache = row * dim;
    }
};
struct RotaryCheck {
    static void check(Args a)
    {
        const Sizes s(a[0]);
        const __int128 rows = s.b * number(a[3]), dim = s.dim;
        want(a[4], "pos", rows, at::kInt);
        want(a[5], "pos_base", s.b, at::kInt);
        want(a[6], "parent", rows, at::kInt);
        want(a[7], "inv_freq", number(a[8]) / 2, at::kFloat);
        if (!PyTuple_Check(a[1]))
            return;
        for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(a[1]); i++) {
            PyObject *j = PyTuple_GET_ITEM(a[1], i);
            if (!PyTuple_Check(j) || PyTuple_GET_SIZE(j) != RotaryFields::n)
                continue;
            const __int128 heads = number(PyTuple_GET_ITEM(j, 1));
            want(PyTuple_GET_ITEM(j, 0), "x", rows * heads * dim, s.type);
            want(PyTuple_GET_ITEM(j, 2), "row_base", s.b, at::kInt);
            want(PyTuple_GET_ITEM(j, 3), "row_index", rows, at::kInt);
            want(PyTuple_GET_ITEM(j, 4), "out", (PyTuple_GET_ITEM(j, 2) == Py_None ? rows : s.b * s.d.s_max) * heads * dim, s.type);
        }
    }
};
struct AppendCheck {
    static void check(Args a)
    {
        const Sizes s(a[0]);
        const __int128 rows = s.b * number(a[3]);
        for (int i : {1, 2})
            want(a[i], "rows", rows * s.hkv * s.dim, s.type);
        want(a[4], "row_base", s.b, at::kInt);
        want(a[5], "row_index", rows, at::kInt);
        for (int i : {6, 8}) {
            want(a[i], "codes", s.cache / 2, at::kByte);
            want(a[i + 1], "scales", s.cache / DREAM_MX_GROUP, at::kByte);
        }
    }
};
struct ReadCheck {
    static void check(Args a)
    {
        const Sizes s(a[0]);
        want_all(a[1], "codes", s.cache / 2, at::kByte);
        want_all(a[2], "scales", s.cache / DREAM_MX_GROUP, at::kByte);
        want(a[4], "row_base", s.b, at::kInt);
        want(a[6], "out", s.b * s.hkv * s.dim * number(a[5]) * number(a[3]), s.type);
    }
};
struct CommitCheck {
    static void check(Args a)
    {
        const Sizes s(a[0]);
        want_all(a[1], "codes", s.cache / 2, at::kByte);
        want_all(a[2], "scales", s.cache / DREAM_MX_GROUP, at::kByte);
        want(a[4], "prefix_len", s.b, at::kInt);
        want(a[6], "accept_path", s.b * number(a[7]), at::kInt);
        want(a[8], "accept_len", s.b, at::kInt);
        want(a[9], "prefix_len_out", s.b, at::kInt);
    }
};
// MX: positions behind the caches are two further on
template <bool MX>
struct WindowCheck {
    static void check(Args a)
    {
        const Sizes s(a[0]);
        Args r = a + (MX ? 6 : 4);      // prefix_len, n_tree, parent, tree_mask, window, n_sink, max_kv_len, out, lse, workspace
        const __int128 t = number(r[1]), rows = s.b * t;
        want(a[1], "q", rows * s.hq * s.dim, s.type);
        if (MX) {
            for (int i : {2, 4}) {
                want(a[i], "codes", s.cache / 2, at::kByte);
                want(a[i + 1], "scales", s.cache / DREAM_MX_GROUP, at::kByte);
            }
        } else {
            want(a[2], "k_cache", s.cache, s.type);
            want(a[3], "v_cache", s.cache, s.type);
        }
        want(r[0], "prefix_len", s.b, at::kInt);
        want(r[2], "parent", rows, at::kInt);
        want(r[3], "tree_mask", rows * ((t + 63) / 64), at::kLong, at::kUInt64);
        want(r[7], "out", rows * s.hq * s.dim, s.type);
        want(r[8], "lse", rows * s.hq, at::kFloat);
        if (THPVariable_Check(r[9]))
            want(r[9], "workspace", 0, THPVariable_Unpack(r[9]).scalar_type());
    }
};

// Caches held in pages
struct PagedSizes : Sizes {
    dream_page_desc p = {};
    __int128 table, pool;
    explicit PagedSizes(Args a) : Sizes(a[0])
    {
        const Arg<const dream_page_desc *> pages(a[1]);
        p = *pages.value;
        table = b * p.max_pages;
        pool = (__int128)p.n_pages * hkv * p.page_size * dim;
    }
};
struct PagedAppendCheck {
    static void check(Args a)
    {
        const PagedSizes s(a);
        const __int128 rows = s.b * number(a[6]);
        want(a[2], "page_table", s.table, at::kInt);
        want(a[3], "q", rows * s.hq * s.dim, s.type);
        want(a[4], "k", rows * s.hkv * s.dim, s.type);
        want(a[5], "v", rows * s.hkv * s.dim, s.type);
        want(a[7], "row_base", s.b, at::kInt);
        want(a[8], "row_index", rows, at::kInt);
        want(a[9], "n_live", s.b, at::kInt);
        want(a[10], "pos", rows, at::kInt);
        want(a[11], "pos_base", s.b, at::kInt);
        want(a[12], "parent", rows, at::kInt);
        want(a[13], "inv_freq", number(a[14]) / 2, at::kFloat);
        want(a[17], "q_out", rows * s.hq * s.dim, s.type);
        want(a[18], "k_pages", s.pool, s.type);
        want(a[19], "v_pages", s.pool, s.type);
    }
};
struct PagedCommitCheck {
    static void check(Args a)
    {
        const PagedSizes s(a);
        want(a[2], "page_table", s.table, at::kInt);
        want_all(a[3], "pools", s.pool, s.type);
        want(a[5], "prefix_len", s.b, at::kInt);
        want(a[7], "accept_path", s.b * number(a[8]), at::kInt);
        want(a[9], "accept_len", s.b, at::kInt);
        want(a[10], "prefix_len_out", s.b, at::kInt);
    }
};
// SPARSE: over selected pages
template <bool SPARSE>
struct PagedAttnCheck {
    static void check(Args a)
    {
        const PagedSizes s(a);
        Args r = a + (SPARSE ? 7 : 6), e = a + (SPARSE ? 13 : 15);      // prefix_len, n_tree, parent, tree_mask; out, lse, workspace
        const __int128 t = number(r[1]), rows = s.b * t, words = (t + 63) / 64;
        want(a[2], "q", rows * s.hq * s.dim, s.type);
        want(a[3], "k_pages", s.pool, s.type);
        want(a[4], "v_pages", s.pool, s.type);
        want(a[5], "page_table", s.table, at::kInt);
        if (SPARSE) {
            want(a[6], "page_nodes", s.table * s.hkv * words, at::kLong, at::kUInt64);
        } else {
            const __int128 groups = number(a[10]);
            want(a[11], "group_start", groups + 1, at::kInt);
            want(a[12], "shared_len", groups, at::kInt);
        }
        want(r[0], "prefix_len", s.b, at::kInt);
        want(r[2], "parent", rows, at::kInt);
        want(r[3], "tree_mask", rows * words, at::kLong, at::kUInt64);
        want(e[0], "out", rows * s.hq * s.dim, s.type);
        want(e[1], "lse", rows * s.hq, at::kFloat);
        if (THPVariable_Check(e[2]))
            want(e[2], "workspace", 0, THPVariable_Unpack(e[2]).scalar_type());
    }
};
struct PageBoundsCheck {
    static void check(Args a)
    {
        const PagedSizes s(a);
        want(a[2], "page_table", s.table, at::kInt);
        want(a[3], "k_pages", s.pool, s.type);
        want(a[4], "from_len", s.b, at::kInt);
        want(a[5], "to_len", s.b, at::kInt);
        want(a[7], "bounds", (__int128)s.p.n_pages * s.hkv * 2 * s.dim, s.type);
    }
};
struct PageSelectCheck {
    static void check(Args a)
    {
        const PagedSizes s(a);
        const __int128 t = number(a[6]);
        want(a[2], "page_table", s.table, at::kInt);
        want(a[3], "q", s.b * t * s.hq * s.dim, s.type);
        want(a[4], "bounds", (__int128)s.p.n_pages * s.hkv * 2 * s.dim, s.type);
        want(a[5], "prefix_len", s.b, at::kInt);
        want(a[11], "page_nodes", s.table * s.hkv * ((t + 63) / 64), at::kLong, at::kUInt64);
        if (THPVariable_Check(a[12]))
            want(a[12], "workspace", 0, THPVariable_Unpack(a[12]).scalar_type());
    }
};

// HOST: position of the host out-parameter, or -1
template <auto F, int HOST, class Check = Unchecked>
struct Entry;
template <class... A, int (*F)(A...), int HOST, class Check>
struct Entry<F, HOST, Check> {
    template <class T, int I>
    using ArgAt = std::conditional_t<I == (int)sizeof...(A) - 1, Stream, std::conditional_t<I == HOST, HostInt, Arg<T>>>;
    template <size_t... I>
    static int run(PyObject *const *args, std::index_sequence<I...>)
    {
        const std::tuple<ArgAt<A, I>...> a(args[I]...);     // (converted in place: some are neither copied nor moved)
        const WithoutGil unlocked;
        return F(std::get<I>(a).value...);
    }
    static PyObject *call(PyObject *, PyObject *const *args, Py_ssize_t n)
    {
        if (n != (Py_ssize_t)sizeof...(A))
            return PyErr_Format(PyExc_TypeError, "%d arguments expected, got %d", (int)sizeof...(A), (int)n);
        try {
            Check::check(args);
            return PyLong_FromLong(run(args, std::index_sequence_for<A...>{}));
        } catch (const Failed &) {
        } catch (...) {     // torch's own errors (a sparse tensor has no bytes) and the allocator's: nothing may leave a C function
            torch::translate_exception_to_python(std::current_exception());
        }
        return nullptr;
    }
};

#define ENTRY_HOST(name, host) {#name, (PyCFunction)(void (*)(void))&Entry<&name, host>::call, METH_FASTCALL, nullptr}
#define ENTRY(name) ENTRY_HOST(name, -1)
#define ENTRY_CHECKED(name, ...) {#name, (PyCFunction)(void (*)(void))&Entry<&name, -1, __VA_ARGS__>::call, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    ENTRY(dream_tree_verify_attn), ENTRY(dream_draft_xattn), ENTRY_HOST(dream_visual_compress, 14), ENTRY(dream_accept_path), ENTRY(dream_accept_path_static),
    ENTRY(dream_kv_commit), ENTRY(dream_project_rows), ENTRY(dream_project_rows_multi), ENTRY(dream_spec_accept), ENTRY(dream_attention_entropy),
    ENTRY(dream_tree_expand_level), ENTRY_HOST(dream_tree_finalize, 9), ENTRY_CHECKED(dream_rotary_rows, RotaryCheck),
    ENTRY_CHECKED(dream_mx_append, AppendCheck), ENTRY_CHECKED(dream_mx_read, ReadCheck), ENTRY_CHECKED(dream_mx_commit, CommitCheck),
    ENTRY_CHECKED(dream_window_verify_attn, WindowCheck<false>), ENTRY_CHECKED(dream_mx_verify_attn, WindowCheck<true>),
    ENTRY_CHECKED(dream_paged_append, PagedAppendCheck), ENTRY_CHECKED(dream_paged_commit, PagedCommitCheck), ENTRY_CHECKED(dream_paged_verify_attn, PagedAttnCheck<false>),
    ENTRY_CHECKED(dream_page_bounds, PageBoundsCheck), ENTRY_CHECKED(dream_page_select, PageSelectCheck), ENTRY_CHECKED(dream_sparse_verify_attn, PagedAttnCheck<true>), {nullptr, nullptr, 0, nullptr}};
#undef ENTRY
#undef ENTRY_HOST
#undef ENTRY_CHECKED
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__call(void) { return PyModule_Create(&module); }
