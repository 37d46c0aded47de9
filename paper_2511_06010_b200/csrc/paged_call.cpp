// Argument marshalling of the paged store's calls as a CPython module: checks the tensors, fills the C
// structs and calls the entry points of libmoska (their addresses are given by bind()).  The same in
// Python costs 10 us a call, more than the kernels of a decode step over few requests take (2.6 us for
// 64 new tokens); here it is one.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>

#include <memory>
#include <string>

#include "moska.h"

namespace {

using Append = int (*)(const uint16_t*, int64_t, const uint16_t*, int64_t, const uint16_t*, int64_t, const int32_t*,
                       const float*, int32_t, int32_t, int32_t, const int32_t*, int32_t, uint16_t*, const moska_paged_kv*,
                       const moska_shape*, moska_stream);
using Gather = int (*)(const int32_t*, int32_t, uint16_t*, uint16_t*, const moska_paged_kv*, const moska_shape*, moska_stream);
using Attend = int (*)(const uint16_t*, const moska_paged_kv*, uint16_t*, float*, float, const moska_shape*, void*, size_t,
                       moska_stream);
using Commit = int (*)(const int32_t*, int32_t, const int32_t*, const int32_t*, int32_t, int32_t*, const moska_paged_kv*,
                       const moska_shape*, moska_stream);
using TreeAttend = int (*)(const uint16_t*, const moska_paged_kv*, const int32_t*, const int32_t*, int32_t, uint16_t*, float*,
                           float, const moska_shape*, void*, size_t, moska_stream);
using Verify = int (*)(const void*, int64_t, const void*, int64_t, int32_t, int32_t, const int32_t*, const int32_t*,
                       const float*, const float*, const int32_t*, int32_t, int32_t, int32_t, int32_t*, int32_t*, int32_t*,
                       moska_stream);
Append g_append = nullptr;
Gather g_gather = nullptr;
Attend g_attend = nullptr;
Commit g_commit = nullptr;
TreeAttend g_tree_attend = nullptr;
Verify g_verify = nullptr;
PyObject* g_error = nullptr;  // MoskaError(status, where)

struct Failed {};  // a Python exception is set

[[noreturn]] void refuse(const std::string& text)
{
    PyErr_SetString(PyExc_ValueError, text.c_str());
    throw Failed{};
}

std::string text(at::IntArrayRef shape)
{
    std::string s = "(";
    for (size_t i = 0; i < shape.size(); ++i) s += (i > 0 ? ", " : "") + std::to_string(shape[i]);
    return s + ")";
}

std::string describe(const at::Tensor& t)
{
    return std::string("got ") + c10::toString(t.scalar_type()) + " " + text(t.sizes()) + " on " + t.device().str() +
           (t.is_contiguous() ? "" : ", not contiguous");
}

const at::Tensor& tensor(PyObject* o, const char* name)
{
    if (!THPVariable_Check(o)) refuse(std::string(name) + ": expected a tensor");
    return THPVariable_Unpack(o);
}

void* dense(const at::Tensor& t, const char* name, at::ScalarType type, at::IntArrayRef shape, c10::Device device)
{
    if (t.scalar_type() != type || t.sizes() != shape || t.device() != device || !t.is_contiguous())
        refuse(std::string(name) + ": expected a contiguous " + c10::toString(type) + " " + text(shape) + " on " + device.str() +
               ", " + describe(t));
    return t.data_ptr();
}

// [n][heads][D] rows whose heads are dense; rows may lie apart
uint16_t* rows(const at::Tensor& t, const char* name, at::IntArrayRef shape, c10::Device device, int64_t* stride)
{
    if (t.scalar_type() != at::kBFloat16 || t.sizes() != shape || t.device() != device)
        refuse(std::string(name) + ": expected BFloat16 " + text(shape) + " on " + device.str() + ", " + describe(t));
    if (shape[0] > 0 && (t.stride(2) != 1 || (shape[1] > 1 && t.stride(1) != shape[2])))
        refuse(std::string(name) + ": the heads of a row must be dense");
    *stride = shape[0] > 1 ? t.stride(0) : shape[1] * shape[2];
    return static_cast<uint16_t*>(t.data_ptr());
}

long whole(PyObject* o)
{
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) throw Failed{};
    return v;
}

// What a PagedKvStore keeps of its pools.
struct Store {
    moska_paged_kv kv;  // format, page_size, n_pages and the pools
    int32_t Hkv, D;
    c10::Device device;
    at::Tensor k, v;    // the pools (4 bits: no v)
};

Store* store_of(PyObject* o)
{
    auto* s = static_cast<Store*>(PyCapsule_GetPointer(o, "moska.store"));
    if (s == nullptr) throw Failed{};
    return s;
}

moska_paged_kv seen_through(const Store& s, PyObject* table_o, PyObject* len_o)
{
    const at::Tensor& table = tensor(table_o, "page_table");
    if (table.dim() != 2) refuse("page_table: expected [requests][pages], " + describe(table));
    moska_paged_kv kv = s.kv;
    kv.page_table = static_cast<const int32_t*>(dense(table, "page_table", at::kInt, table.sizes(), s.device));
    kv.kv_len = static_cast<const int32_t*>(dense(tensor(len_o, "kv_len"), "kv_len", at::kInt, {table.size(0)}, s.device));
    if (table.size(0) > INT32_MAX || table.size(1) > INT32_MAX) refuse("page_table: too large");
    kv.max_pages = static_cast<int32_t>(table.size(1));
    return kv;
}

moska_shape shape_of(int64_t B, int64_t Hq, int64_t Hkv, int64_t D, long q_len)
{
    if (B > INT32_MAX || Hq > INT32_MAX) refuse("too many rows or heads");
    return moska_shape{(int32_t)B, (int32_t)Hq, (int32_t)Hkv, (int32_t)D, 1, 128, 1, 1, 1, 0, (int32_t)q_len};
}

const int32_t* first_rows(PyObject* o, int64_t n_requests, int64_t n_rows, long q_len, c10::Device device)
{
    if (o != Py_None)
        return static_cast<const int32_t*>(dense(tensor(o, "row_start"), "row_start", at::kInt, {n_requests + 1}, device));
    if (n_rows != n_requests * q_len)
        refuse(std::to_string(n_rows) + " rows for " + std::to_string(n_requests) + " requests of " + std::to_string(q_len) +
               " each: give row_start");
    return nullptr;
}

// A Python stream address, or the device's current stream; the device and the stream are current while this
// lives.  What a call allocates then comes from the memory of the stream that writes it: a block of another
// stream's may still be in use there.  On a stream other than the one that the caller is on, the allocator
// is told who uses what: reads() for what the kernels touch, returns() for results, which the caller's
// stream goes on with.  Without that a tensor dropped early would be handed out again too soon.
struct OnDevice {
    c10::cuda::OptionalCUDAGuard guard;
    c10::cuda::OptionalCUDAStreamGuard stream_guard;
    moska_stream stream = nullptr;
    c10::optional<c10::cuda::CUDAStream> here, callers;  // set if they differ
    OnDevice(c10::Device device, PyObject* stream_o)
    {
        if (!device.is_cuda()) refuse("the tensors are not on a GPU");
        guard.set_device(device);
        const c10::cuda::CUDAStream current = c10::cuda::getCurrentCUDAStream(device.index());
        stream = current.stream();
        if (stream_o == Py_None) return;
        stream = PyLong_AsVoidPtr(stream_o);
        if (stream == nullptr && PyErr_Occurred()) throw Failed{};
        // (torch knows the legacy default stream as 0 alone)
        const auto known = stream == cudaStreamLegacy ? nullptr : static_cast<cudaStream_t>(stream);
        if (known == current.stream()) return;
        here = c10::cuda::getStreamFromExternal(known, device.index());
        callers = current;
        stream_guard.reset_stream(*here);
    }
    void reads(const at::Tensor& t) const
    {
        if (here && t.defined()) c10::cuda::CUDACachingAllocator::recordStream(t.storage().data_ptr(), *here);
    }
    void reads(PyObject* o) const
    {
        if (here && THPVariable_Check(o)) reads(THPVariable_Unpack(o));
    }
    void returns(const at::Tensor& t) const
    {
        reads(t);
        if (here && t.defined()) c10::cuda::CUDACachingAllocator::recordStream(t.storage().data_ptr(), *callers);
    }
};

void check(int status, const char* where)
{
    if (status == MOSKA_OK) return;
    PyObject* e = PyObject_CallFunction(g_error, "is", status, where);
    if (e != nullptr) {
        PyErr_SetObject(g_error, e);
        Py_DECREF(e);
    }
    throw Failed{};
}

// Runs `body`; C++ exceptions become Python's.
template <class Body>
PyObject* guarded(Py_ssize_t given, Py_ssize_t wanted, Body body)
{
    try {
        if (given != wanted) refuse("wrong number of arguments");
        return body();
    } catch (const Failed&) {
    } catch (...) {  // torch's own, out of memory among them
        torch::translate_exception_to_python(std::current_exception());
    }
    return nullptr;
}

PyObject* none()
{
    Py_INCREF(Py_None);
    return Py_None;
}

// bind(append, gather, paged_attn, commit, tree_attn, verify, MoskaError): addresses of the entry points
PyObject* py_bind(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded(n, 7, [&] {
        g_append = reinterpret_cast<Append>(PyLong_AsVoidPtr(a[0]));
        g_gather = reinterpret_cast<Gather>(PyLong_AsVoidPtr(a[1]));
        g_attend = reinterpret_cast<Attend>(PyLong_AsVoidPtr(a[2]));
        g_commit = reinterpret_cast<Commit>(PyLong_AsVoidPtr(a[3]));
        g_tree_attend = reinterpret_cast<TreeAttend>(PyLong_AsVoidPtr(a[4]));
        g_verify = reinterpret_cast<Verify>(PyLong_AsVoidPtr(a[5]));
        if (PyErr_Occurred()) throw Failed{};
        Py_INCREF(a[6]);
        Py_XDECREF(g_error);
        g_error = a[6];
        return none();
    });
}

// store(format, page_size, n_pages, Hkv, D, k_pages, v_pages or None): a handle; the pools are checked here
PyObject* py_store(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded(n, 7, [&] {
        const long format = whole(a[0]), page_size = whole(a[1]), n_pages = whole(a[2]), Hkv = whole(a[3]), D = whole(a[4]);
        if (n_pages > INT32_MAX || Hkv > INT32_MAX) refuse("too many pages or heads");
        const at::Tensor& k = tensor(a[5], "k_pages");
        auto s = std::make_unique<Store>(Store{{}, (int32_t)Hkv, (int32_t)D, k.device(), k, {}});
        s->kv.format = (int32_t)format;
        s->kv.page_size = (int32_t)page_size;
        s->kv.n_pages = (int32_t)n_pages;
        if (format == MOSKA_KV_FP4) {
            s->kv.k_pages = dense(k, "pages4", at::kByte, {n_pages, Hkv, page_size / 16, 18 * D}, s->device);
        } else {
            s->kv.k_pages = dense(k, "k_pages", at::kBFloat16, {n_pages, page_size, Hkv, D}, s->device);
            s->v = tensor(a[6], "v_pages");
            s->kv.v_pages = dense(s->v, "v_pages", at::kBFloat16, {n_pages, page_size, Hkv, D}, s->device);
        }
        PyObject* o = PyCapsule_New(s.get(), "moska.store", [](PyObject* c) {
            delete static_cast<Store*>(PyCapsule_GetPointer(c, "moska.store"));
        });
        if (o == nullptr) throw Failed{};
        s.release();
        return o;
    });
}

// view(store, page_table, kv_len) -> the eight fields of moska_paged_kv
PyObject* py_view(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded(n, 3, [&] {
        const moska_paged_kv kv = seen_through(*store_of(a[0]), a[1], a[2]);
        PyObject* o = Py_BuildValue("(iiiiKKKK)", kv.format, kv.page_size, kv.n_pages, kv.max_pages,
                                    (unsigned long long)(uintptr_t)kv.k_pages, (unsigned long long)(uintptr_t)kv.v_pages,
                                    (unsigned long long)(uintptr_t)kv.page_table, (unsigned long long)(uintptr_t)kv.kv_len);
        if (o == nullptr) throw Failed{};
        return o;
    });
}

// append(store, q, k, v, page_table, kv_len, positions, cos_sin, row_start, interleaved, q_out, q_len, stream)
PyObject* py_append(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    return guarded(n_args, 13, [&] {
        const Store& s = *store_of(a[0]);
        const moska_paged_kv kv = seen_through(s, a[4], a[5]);
        const at::Tensor &k = tensor(a[2], "k"), &v = tensor(a[3], "v");
        if (k.dim() != 3) refuse("k: expected [rows][heads][D], " + describe(k));
        const int64_t n = k.size(0), n_requests = tensor(a[4], "page_table").size(0);
        long q_len = whole(a[11]);
        const int32_t* first = first_rows(a[8], n_requests, n, q_len, s.device);
        if (first != nullptr) q_len = 1;
        int64_t qs = 0, ks = 0, vs = 0, Hq = s.Hkv;
        uint16_t* kp = rows(k, "k", {n, s.Hkv, s.D}, s.device, &ks);
        uint16_t* vp = rows(v, "v", {n, s.Hkv, s.D}, s.device, &vs);
        uint16_t *qp = nullptr, *to = nullptr;
        at::Tensor q_out;
        if (a[1] != Py_None) {
            const at::Tensor& q = tensor(a[1], "q");
            if (q.dim() != 3) refuse("q: expected [rows][heads][D], " + describe(q));
            Hq = q.size(1);
            const int64_t shape[3] = {n, Hq, s.D};
            qp = rows(q, "q", shape, s.device, &qs);
            if (a[10] != Py_None) {
                q_out = tensor(a[10], "q_out");
                to = static_cast<uint16_t*>(dense(q_out, "q_out", at::kBFloat16, shape, s.device));
            }
        } else if (a[10] != Py_None) {
            refuse("q_out without q");
        }
        int64_t n_positions = 0, rot_dim = 0;
        const int32_t* at_position = nullptr;
        const float* table = nullptr;
        if (a[7] != Py_None) {
            const at::Tensor& cs = tensor(a[7], "cos_sin");
            if (a[6] == Py_None || cs.dim() != 2) refuse("cos_sin is [positions][rot_dim] and comes with positions");
            n_positions = cs.size(0);
            rot_dim = cs.size(1);
            if (n_positions > INT32_MAX || rot_dim > INT32_MAX) refuse("cos_sin: too large");
            table = static_cast<const float*>(dense(cs, "cos_sin", at::kFloat, cs.sizes(), s.device));
            at_position = static_cast<const int32_t*>(dense(tensor(a[6], "positions"), "positions", at::kInt, {n}, s.device));
        }
        const int turned = PyObject_IsTrue(a[9]);
        if (turned < 0) throw Failed{};
        const auto result = [&] { return at::empty({n, Hq, s.D}, at::TensorOptions().dtype(at::kBFloat16).device(s.device)); };
        if (n > 0) {
            const moska_shape shape = shape_of(n, Hq, s.Hkv, s.D, q_len);
            const OnDevice on(s.device, a[12]);
            if (qp != nullptr && !q_out.defined()) {
                q_out = result();
                to = static_cast<uint16_t*>(q_out.data_ptr());
            }
            check(g_append(qp, qs, kp, ks, vp, vs, at_position, table, (int32_t)n_positions, (int32_t)rot_dim, turned, first,
                           (int32_t)n_requests, to, &kv, &shape, on.stream),
                  "moska_kv_append_paged");
            for (int i : {1, 2, 3, 4, 5, 8}) on.reads(a[i]);
            if (table != nullptr) {
                on.reads(a[6]);
                on.reads(a[7]);
            }
            on.reads(s.k);
            on.reads(s.v);
            on.returns(q_out);
        } else if (a[1] != Py_None && !q_out.defined()) {
            q_out = result();
        }
        return q_out.defined() ? THPVariable_Wrap(q_out) : none();
    });
}

// gather(store, page_table, kv_len, n_rows, row_start, q_len, k_out, v_out, stream)
PyObject* py_gather(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    return guarded(n_args, 9, [&] {
        const Store& s = *store_of(a[0]);
        const moska_paged_kv kv = seen_through(s, a[1], a[2]);
        const int64_t n = whole(a[3]), n_requests = tensor(a[1], "page_table").size(0);
        long q_len = whole(a[5]);
        if (n < 0) refuse("n_rows is negative");
        const int32_t* first = first_rows(a[4], n_requests, n, q_len, s.device);
        if (first != nullptr) q_len = 1;
        const int64_t shape[3] = {n, s.Hkv, s.D};
        const auto options = at::TensorOptions().dtype(at::kBFloat16).device(s.device);
        at::Tensor out[2];
        uint16_t* to[2] = {nullptr, nullptr};
        constexpr const char* names[2] = {"k_out", "v_out"};
        for (int i = 0; i < 2; ++i) {
            if (a[6 + i] == Py_None) continue;
            out[i] = tensor(a[6 + i], names[i]);
            to[i] = static_cast<uint16_t*>(dense(out[i], names[i], at::kBFloat16, shape, s.device));
        }
        const auto allocate = [&] {
            for (int i = 0; i < 2; ++i) {
                if (out[i].defined()) continue;
                out[i] = at::empty(shape, options);
                to[i] = static_cast<uint16_t*>(out[i].data_ptr());
            }
        };
        if (n > 0) {
            const moska_shape c_shape = shape_of(n, s.Hkv, s.Hkv, s.D, q_len);
            const OnDevice on(s.device, a[8]);
            allocate();
            check(g_gather(first, (int32_t)n_requests, to[0], to[1], &kv, &c_shape, on.stream), "moska_kv_gather_paged");
            for (int i : {1, 2, 4}) on.reads(a[i]);
            on.reads(s.k);
            on.reads(s.v);
            for (const at::Tensor& t : out) on.returns(t);
        } else {
            allocate();
        }
        PyObject* pair = PyTuple_New(2);
        if (pair == nullptr) throw Failed{};
        PyTuple_SET_ITEM(pair, 0, THPVariable_Wrap(out[0]));
        PyTuple_SET_ITEM(pair, 1, THPVariable_Wrap(out[1]));
        return pair;
    });
}

// attend(store, q, page_table, kv_len, out, lse, scale, q_len, n_unique_splits, ws, stream)
PyObject* py_attend(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    return guarded(n_args, 11, [&] {
        const Store& s = *store_of(a[0]);
        const moska_paged_kv kv = seen_through(s, a[2], a[3]);
        const at::Tensor &q = tensor(a[1], "q"), &out = tensor(a[4], "out"), &lse = tensor(a[5], "lse"), &ws = tensor(a[9], "ws");
        if (out.dim() != 3 || out.size(2) != s.D) refuse("out: expected [rows][heads][D], " + describe(out));
        const int64_t B = out.size(0), Hq = out.size(1), n_requests = tensor(a[2], "page_table").size(0);
        const long q_len = whole(a[7]);
        auto* qp = static_cast<uint16_t*>(dense(q, "q", at::kBFloat16, out.sizes(), s.device));
        auto* op = static_cast<uint16_t*>(dense(out, "out", at::kBFloat16, out.sizes(), s.device));
        auto* lp = static_cast<float*>(dense(lse, "lse", at::kFloat, {B, Hq}, s.device));
        void* wp = dense(ws, "ws", at::kByte, ws.sizes(), s.device);
        if (n_requests * (q_len > 1 ? q_len : 1) != B)
            refuse(std::to_string(n_requests) + " page-table rows for " + std::to_string(B) + " batch rows, " +
                   std::to_string(q_len) + " a request");
        if (B > 0) {
            moska_shape shape = shape_of(B, Hq, s.Hkv, s.D, q_len);
            shape.n_unique_splits = (int32_t)whole(a[8]);
            const double scale = PyFloat_AsDouble(a[6]);
            if (PyErr_Occurred()) throw Failed{};
            const OnDevice on(s.device, a[10]);
            check(g_attend(qp, &kv, op, lp, (float)scale, &shape, wp, (size_t)ws.numel(), on.stream), "moska_paged_attn");
            for (int i : {1, 2, 3, 9}) on.reads(a[i]);
            on.reads(s.k);
            on.reads(s.v);
            on.returns(out);
            on.returns(lse);
        }
        return none();
    });
}

// int32 [n], or nothing
const int32_t* whole_numbers(PyObject* o, const char* name, int64_t n, c10::Device device)
{
    return o == Py_None ? nullptr : static_cast<const int32_t*>(dense(tensor(o, name), name, at::kInt, {n}, device));
}

// the largest tree of a call whose requests have it (without row_start) or at most it
long most_nodes(PyObject* o)
{
    const long n = whole(o);
    if (n < 1 || n > MOSKA_TREE_MAX_NODES)
        refuse("max_nodes = " + std::to_string(n) + ", 1.." + std::to_string(MOSKA_TREE_MAX_NODES) + " are possible");
    return n;
}

// tree_attend(store, q, page_table, kv_len, parents, row_start, out, lse, scale, max_nodes, n_unique_splits, ws, stream)
PyObject* py_tree_attend(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    return guarded(n_args, 13, [&] {
        const Store& s = *store_of(a[0]);
        const moska_paged_kv kv = seen_through(s, a[2], a[3]);
        const at::Tensor &q = tensor(a[1], "q"), &out = tensor(a[6], "out"), &lse = tensor(a[7], "lse"), &ws = tensor(a[11], "ws");
        if (out.dim() != 3 || out.size(2) != s.D) refuse("out: expected [rows][heads][D], " + describe(out));
        const int64_t B = out.size(0), Hq = out.size(1), n_requests = tensor(a[2], "page_table").size(0);
        const long nodes = most_nodes(a[9]);
        auto* qp = static_cast<uint16_t*>(dense(q, "q", at::kBFloat16, out.sizes(), s.device));
        auto* op = static_cast<uint16_t*>(dense(out, "out", at::kBFloat16, out.sizes(), s.device));
        auto* lp = static_cast<float*>(dense(lse, "lse", at::kFloat, {B, Hq}, s.device));
        void* wp = dense(ws, "ws", at::kByte, ws.sizes(), s.device);
        const int32_t* parents = whole_numbers(a[4], "parents", B, s.device);
        const int32_t* first = first_rows(a[5], n_requests, B, nodes, s.device);
        if (B > 0) {
            moska_shape shape = shape_of(B, Hq, s.Hkv, s.D, nodes);
            shape.n_unique_splits = (int32_t)whole(a[10]);
            const double scale = PyFloat_AsDouble(a[8]);
            if (PyErr_Occurred()) throw Failed{};
            const OnDevice on(s.device, a[12]);
            check(g_tree_attend(qp, &kv, parents, first, (int32_t)n_requests, op, lp, (float)scale, &shape, wp,
                                (size_t)ws.numel(), on.stream),
                  "moska_tree_attn");
            for (int i : {1, 2, 3, 4, 5, 11}) on.reads(a[i]);
            on.reads(s.k);
            on.reads(s.v);
            on.returns(out);
            on.returns(lse);
        }
        return none();
    });
}

// commit(store, page_table, kv_len, path, n_path, row_start, max_nodes, kv_len_out, stream) -> kv_len_out
PyObject* py_commit(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    return guarded(n_args, 9, [&] {
        const Store& s = *store_of(a[0]);
        const moska_paged_kv kv = seen_through(s, a[1], a[2]);
        const int64_t n = tensor(a[1], "page_table").size(0);
        const long nodes = most_nodes(a[6]);
        const at::Tensor& path = tensor(a[3], "path");
        if (path.dim() != 2 || path.size(1) < 1 || path.size(1) > INT32_MAX) refuse("path: expected [requests][nodes], " + describe(path));
        auto* pp = static_cast<const int32_t*>(dense(path, "path", at::kInt, {n, path.size(1)}, s.device));
        auto* np = static_cast<const int32_t*>(dense(tensor(a[4], "n_path"), "n_path", at::kInt, {n}, s.device));
        const int32_t* first = whole_numbers(a[5], "row_start", n + 1, s.device);
        at::Tensor to;
        int32_t* tp = nullptr;
        if (a[7] != Py_None) {
            to = tensor(a[7], "kv_len_out");
            tp = static_cast<int32_t*>(dense(to, "kv_len_out", at::kInt, {n}, s.device));
        }
        if (n * nodes > INT32_MAX) refuse("too many nodes");
        const auto result = [&] { return at::empty({n}, at::TensorOptions().dtype(at::kInt).device(s.device)); };
        if (n > 0) {
            // (with row_start the rows themselves are not at hand)
            const moska_shape shape = shape_of(first == nullptr ? n * nodes : INT32_MAX, s.Hkv, s.Hkv, s.D, nodes);
            const OnDevice on(s.device, a[8]);
            if (tp == nullptr) {
                to = result();
                tp = static_cast<int32_t*>(to.data_ptr());
            }
            check(g_commit(pp, (int32_t)path.size(1), np, first, (int32_t)n, tp, &kv, &shape, on.stream), "moska_kv_commit_paged");
            for (int i : {1, 2, 3, 4, 5}) on.reads(a[i]);
            on.reads(s.k);
            on.reads(s.v);
            on.returns(to);
        } else if (tp == nullptr) {
            to = result();
        }
        return THPVariable_Wrap(to);
    });
}

// [rows][V] probabilities whose rows may lie apart
const void* probabilities(const at::Tensor& t, const char* name, at::ScalarType type, int64_t B, int64_t V, c10::Device device,
                          int64_t* stride)
{
    if (t.dim() != 2 || t.scalar_type() != type || t.size(0) != B || t.size(1) != V || t.device() != device)
        refuse(std::string(name) + ": expected " + c10::toString(type) + " (" + std::to_string(B) + ", " + std::to_string(V) + ") on " +
               device.str() + ", " + describe(t));
    if (V > 1 && t.stride(1) != 1) refuse(std::string(name) + ": the entries of a row must be neighbours");
    if (B > 1 && t.stride(0) < V) refuse(std::string(name) + ": rows must not overlap");
    *stride = B > 1 ? t.stride(0) : V;
    return t.data_ptr();
}

// verify(target_probs, draft_probs, tokens, parents, u_accept, u_next, row_start, max_nodes, path, n_path, next_token, stream)
// -> (path, n_path, next_token)
PyObject* py_verify(PyObject*, PyObject* const* a, Py_ssize_t n_args)
{
    return guarded(n_args, 12, [&] {
        const at::Tensor &target = tensor(a[0], "target_probs"), &u_next = tensor(a[5], "u_next");
        const c10::Device device = target.device();
        const at::ScalarType type = target.scalar_type();
        if (target.dim() != 2 || target.size(1) < 1 || (type != at::kFloat && type != at::kBFloat16))
            refuse("target_probs: expected Float or BFloat16 [rows][vocabulary], " + describe(target));
        if (u_next.dim() != 1) refuse("u_next: expected [requests], " + describe(u_next));
        const int64_t B = target.size(0), V = target.size(1), n = u_next.size(0);
        if (B > INT32_MAX || V > INT32_MAX || n > INT32_MAX) refuse("too many rows or requests, or too large a vocabulary");
        const long nodes = most_nodes(a[7]);
        int64_t t_stride = V, d_stride = V;
        const void* tp = probabilities(target, "target_probs", type, B, V, device, &t_stride);
        const void* dp = a[1] == Py_None ? nullptr
                                         : probabilities(tensor(a[1], "draft_probs"), "draft_probs", type, B, V, device, &d_stride);
        auto* tokens = static_cast<const int32_t*>(dense(tensor(a[2], "tokens"), "tokens", at::kInt, {B}, device));
        auto* parents = static_cast<const int32_t*>(dense(tensor(a[3], "parents"), "parents", at::kInt, {B}, device));
        auto* u = static_cast<const float*>(dense(tensor(a[4], "u_accept"), "u_accept", at::kFloat, {B}, device));
        auto* un = static_cast<const float*>(dense(u_next, "u_next", at::kFloat, {n}, device));
        const int32_t* first = first_rows(a[6], n, B, nodes, device);
        at::Tensor out[3];
        constexpr const char* names[3] = {"path", "n_path", "next_token"};
        const int64_t path_shape[2] = {n, nodes};
        const auto shape = [&](int i) { return i == 0 ? at::IntArrayRef(path_shape, 2) : at::IntArrayRef(path_shape, 1); };
        for (int i = 0; i < 3; ++i) {
            if (a[8 + i] == Py_None) continue;
            out[i] = tensor(a[8 + i], names[i]);
            dense(out[i], names[i], at::kInt, shape(i), device);
        }
        const auto allocate = [&] {
            for (int i = 0; i < 3; ++i)
                if (!out[i].defined()) out[i] = at::empty(shape(i), at::TensorOptions().dtype(at::kInt).device(device));
        };
        if (n > 0) {
            const OnDevice on(device, a[11]);
            allocate();
            check(g_verify(tp, t_stride, dp, d_stride, type == at::kFloat ? MOSKA_PROB_F32 : MOSKA_PROB_BF16, (int32_t)V, tokens,
                           parents, u, un, first, (int32_t)n, (int32_t)nodes, (int32_t)B, static_cast<int32_t*>(out[0].data_ptr()),
                           static_cast<int32_t*>(out[1].data_ptr()), static_cast<int32_t*>(out[2].data_ptr()), on.stream),
                  "moska_verify_tree");
            for (int i = 0; i < 7; ++i) on.reads(a[i]);
            for (const at::Tensor& t : out) on.returns(t);
        } else {
            allocate();
        }
        PyObject* three = PyTuple_New(3);
        if (three == nullptr) throw Failed{};
        for (int i = 0; i < 3; ++i) PyTuple_SET_ITEM(three, i, THPVariable_Wrap(out[i]));
        return three;
    });
}

#define METHOD(name, fn) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(fn)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD("bind", py_bind),     METHOD("store", py_store),   METHOD("view", py_view),
                         METHOD("append", py_append), METHOD("gather", py_gather), METHOD("attend", py_attend),
                         METHOD("commit", py_commit), METHOD("tree_attend", py_tree_attend), METHOD("verify", py_verify),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_paged_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__paged_call()
{
    PyObject* m = PyModule_Create(&module_def);
    if (m != nullptr && PyModule_AddStringConstant(m, "built_for", BUILT_FOR) < 0) Py_CLEAR(m);
    return m;
}
