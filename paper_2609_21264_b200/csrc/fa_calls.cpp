// The Python calls on drafted tokens: what binding.py's functions of the same names check, allocate and hand to the C entries of
// include/fa.h.  A call is made once per layer or step and its kernels take 2 to 15 us; checks and outputs in Python took 4 to 9 us of
// host time beside the launches' 3.5 each (tree_layout 11.0 us), here a fraction of one (tree_layout 5.4 us,
// forward_paged_tree 7.9, with what giving the interpreter's lock back costs, 0.1).
//
// Every function returns its results, or the entry's status code as an int where that is not FA_OK, and raises ValueError for arguments
// that no entry should see.  The C entries are bound by address: the library is the one that binding.py has loaded.  What can wait for the
// device, a launch into a full queue or memory that the allocator has to get, runs without the interpreter's lock.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

#include "../../include/fa.h"

namespace {

decltype(&fa_device) p_device = nullptr;
decltype(&fa_tree_layout) p_layout = nullptr;
decltype(&fa_append_paged_at) p_append = nullptr;
decltype(&fa_forward_paged_tree) p_tree = nullptr;
decltype(&fa_compact_paged) p_compact = nullptr;
decltype(&fa_copy_pages) p_copy = nullptr;

// An argument that is not to be had; the Python error has been set.
struct Refused {};

[[noreturn]] void refuse(const char* why) {
    PyErr_SetString(PyExc_ValueError, why);
    throw Refused{};
}

// Reads the arguments of a call one after the other.
struct Args {
    PyObject* const* a;
    Py_ssize_t n, at = 0;
    PyObject* next() {
        if (at >= n) refuse("too few arguments");
        return a[at++];
    }
    void* address() {
        PyObject* o = next();
        if (o == Py_None) return nullptr;
        void* p = PyLong_AsVoidPtr(o);
        if (!p && PyErr_Occurred()) throw Refused{};
        return p;
    }
    // whether the next argument is another one than None
    bool given() const { return at < n && a[at] != Py_None; }
    int64_t number() {
        const long long x = PyLong_AsLongLong(next());
        if (x == -1 && PyErr_Occurred()) throw Refused{};
        return x;
    }
    int integer(const char* what) {
        const int64_t x = number();
        if (x < INT32_MIN || x > INT32_MAX) refuse(what);
        return static_cast<int>(x);
    }
    double real() {
        const double x = PyFloat_AsDouble(next());
        if (x == -1.0 && PyErr_Occurred()) throw Refused{};
        return x;
    }
    bool truth() {
        const int x = PyObject_IsTrue(next());
        if (x < 0) throw Refused{};
        return x != 0;
    }
    // nullptr for None
    const at::Tensor* maybe() {
        PyObject* o = next();
        if (o == Py_None) return nullptr;
        if (!THPVariable_Check(o)) {
            PyErr_SetString(PyExc_TypeError, "a tensor is expected");
            throw Refused{};
        }
        return &THPVariable_Unpack(o);
    }
    const at::Tensor& tensor() {
        const at::Tensor* t = maybe();
        if (!t) refuse("a tensor is missing");
        return *t;
    }
};

int32_t* ints(const at::Tensor* t) { return t ? static_cast<int32_t*>(t->data_ptr()) : nullptr; }

bool on(const at::Tensor& t, int device) { return t.is_cuda() && t.get_device() == device; }

// A contiguous int32 vector of n numbers on the device.
bool vector_ok(const at::Tensor& t, int64_t n, int device) {
    return t.scalar_type() == at::kInt && t.dim() == 1 && t.size(0) == n && on(t, device) && t.is_contiguous();
}

const int32_t* offsets(const at::Tensor* cu, int64_t B, int device) {
    if (!cu) return nullptr;
    if (!vector_ok(*cu, B + 1, device)) refuse("cu_seqlens must be a contiguous int32 tensor of B + 1 offsets on the cache's device");
    return ints(cu);
}

// The largest number of drafts of a sequence.
int most_tokens(int given, bool ragged, int64_t total, int64_t B) {
    if (given > 0) return given;
    if (ragged || given < 0) refuse("max_tokens is needed with cu_seqlens");
    const int64_t n = total / (B > 0 ? B : 1);
    return n < 1 ? 1 : n > INT32_MAX ? INT32_MAX : static_cast<int>(n);
}

void check_mask(const at::Tensor& m, int64_t total, int64_t words, int device) {
    if (m.scalar_type() != at::kInt || m.dim() != 2 || !on(m, device) || m.size(0) != total || m.size(1) < words ||
        (m.size(1) > 1 && m.stride(1) != 1) || (total > 1 && m.stride(0) < words))
        refuse("mask must be int32 of shape [tokens, ceil(max_tokens / 32) or more] on the same device, its rows contiguous and apart");
}

// The fa_paged_seqs of a call, as binding._seqs makes it.
fa_paged_seqs sequences(fa_handle* h, const at::Tensor& table, const at::Tensor& lens, int device) {
    if (table.scalar_type() != at::kInt || table.dim() != 2 || !on(table, device)) refuse("block_table must be a 2-D int32 tensor on the cache's device");
    const int64_t B = table.size(0), pages = table.size(1);
    if ((pages > 1 && table.stride(1) != 1) || (B > 1 && table.stride(0) < pages)) refuse("the rows of block_table must be contiguous and lie apart");
    if (!vector_ok(lens, B, device)) refuse("seq_lens must be a contiguous int32 tensor of one length per row of block_table");
    if (B > INT32_MAX || pages > INT32_MAX) refuse("block_table is too large");
    if (p_device(h) != device) refuse("the handle belongs to another device than the cache");
    fa_paged_seqs s{};
    s.struct_size = sizeof s;
    s.B = static_cast<int32_t>(B);
    s.block_table = ints(&table);
    s.table_stride = B > 1 ? table.stride(0) : pages;
    s.seq_lens = ints(&lens);
    s.max_pages = static_cast<int32_t>(pages);
    return s;
}

// Tokens, heads and (token, head) strides of a [tokens, heads, d] bf16 tensor, as binding._rows finds them.
struct Rows { int64_t n, heads, strides[2]; };
Rows rows(const at::Tensor& t, int64_t d, int device, const char* why) {
    if (t.scalar_type() != at::kBFloat16 || t.dim() != 3 || !on(t, device) || t.size(2) != d || t.stride(2) != 1) refuse(why);
    Rows r{t.size(0), t.size(1), {t.stride(0), t.stride(1)}};
    if (r.n > INT32_MAX || r.heads > INT32_MAX) refuse(why);
    // (the stride of a dimension of one row is whatever the view left; the library wants it to be valid)
    auto valid = [&](int64_t s) { const int64_t up = (s + 7) / 8 * 8; return up > d ? up : d; };
    if (r.n <= 1) r.strides[0] = valid(r.strides[0]);
    if (r.heads == 1) r.strides[1] = valid(r.strides[1]);
    return r;
}

// f() with the interpreter's lock given back meanwhile: it touches no Python object.
template <typename F>
auto unlocked(F&& f) {
    struct Lock {
        PyThreadState* state = PyEval_SaveThread();
        ~Lock() { PyEval_RestoreThread(state); }
    } lock;
    return f();
}

at::Tensor fresh(at::IntArrayRef sizes, const at::TensorOptions& options) {
    return unlocked([&] { return at::empty(sizes, options); });
}

void* stream_of(int device) { return c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(device)).stream(); }

PyObject* status(fa_status s) { return PyLong_FromLong(s); }

// Two tensors, or one and None, as a tuple.
PyObject* both(at::Tensor a, at::Tensor b) {
    PyObject *x = THPVariable_Wrap(std::move(a)), *y = b.defined() ? THPVariable_Wrap(std::move(b)) : Py_NewRef(Py_None);
    PyObject* t = x && y ? PyTuple_Pack(2, x, y) : nullptr;
    Py_XDECREF(x);
    Py_XDECREF(y);
    return t;
}

PyObject* bind(Args& a) {
    p_device = reinterpret_cast<decltype(p_device)>(a.address());
    p_layout = reinterpret_cast<decltype(p_layout)>(a.address());
    p_append = reinterpret_cast<decltype(p_append)>(a.address());
    p_tree = reinterpret_cast<decltype(p_tree)>(a.address());
    p_compact = reinterpret_cast<decltype(p_compact)>(a.address());
    p_copy = reinterpret_cast<decltype(p_copy)>(a.address());
    Py_RETURN_NONE;
}

// (handle, parents, seq_lens, cu_seqlens, max_tokens, mask, positions) -> (mask, positions)
PyObject* tree_layout(Args& a) {
    auto* h = static_cast<fa_handle*>(a.address());
    const at::Tensor &parents = a.tensor(), &lens = a.tensor();
    const at::Tensor* cu = a.maybe();
    const int given = a.integer("max_tokens is out of range");
    const at::Tensor *mask_in = a.maybe(), *pos_in = a.maybe();
    if (parents.scalar_type() != at::kInt || !parents.is_cuda() || parents.dim() != 1 || !parents.is_contiguous())
        refuse("parents must be a contiguous 1-D int32 CUDA tensor");
    const int device = parents.get_device();
    if (lens.dim() != 1 || !vector_ok(lens, lens.size(0), device)) refuse("seq_lens must be a contiguous 1-D int32 tensor on parents' device");
    if (p_device(h) != device) refuse("the handle belongs to another device than the tensors");
    const int64_t total = parents.size(0), B = lens.size(0);
    if (total > INT32_MAX || B > INT32_MAX) refuse("too many tokens");
    const int32_t* cu_ptr = offsets(cu, B, device);
    const int most = most_tokens(given, cu != nullptr, total, B);
    const int64_t words = (static_cast<int64_t>(most) + 31) / 32;
    if (mask_in) check_mask(*mask_in, total, words, device);
    if (pos_in && !vector_ok(*pos_in, total, device)) refuse("positions must be a contiguous int32 tensor of one number per token");
    at::Tensor mask = mask_in ? *mask_in : fresh({total, words}, parents.options()), pos = pos_in ? *pos_in : fresh({total}, parents.options());
    const fa_status s = unlocked([&] {
        return p_layout(h, ints(&parents), cu_ptr, static_cast<int>(total), static_cast<int>(B), ints(&lens), most,
                        reinterpret_cast<uint32_t*>(mask.data_ptr()), total > 1 ? mask.stride(0) : words, ints(&pos), stream_of(device));
    });
    return s == FA_OK ? both(std::move(mask), std::move(pos)) : status(s);
}

// (handle, cache address, device, Hkv, dqk, dv, k, v, block_table, seq_lens, cu_seqlens, q, q_out, rope address, rope device, axes that the
// rope asks for, address of its axis numbers, positions) -> q_out or None
PyObject* append_at(Args& a) {
    auto* h = static_cast<fa_handle*>(a.address());
    auto* cache = static_cast<const fa_paged_cache*>(a.address());
    const int device = a.integer("device");
    const int64_t Hkv = a.number(), dqk = a.number(), dv = a.number();
    const at::Tensor &k = a.tensor(), &v = a.tensor(), &table = a.tensor(), &lens = a.tensor();
    const at::Tensor *cu = a.maybe(), *q = a.maybe(), *q_out = a.maybe();
    auto* rope = static_cast<const fa_rope*>(a.address());
    const int rope_device = a.integer("device"), rope_axes = a.integer("axes");
    auto* axis_of_pair = static_cast<const uint8_t*>(a.address());
    const at::Tensor& pos = a.tensor();
    const fa_paged_seqs seqs = sequences(h, table, lens, device);
    const Rows kr = rows(k, dqk, device, "k must be a 3-D bf16 tensor of the cache's head size on its device, contiguous along a head");
    const Rows vr = rows(v, dv, device, "v must be a 3-D bf16 tensor of the cache's head size on its device, contiguous along a head");
    if (vr.n != kr.n || kr.heads != Hkv || vr.heads != kr.heads) refuse("k and v must have the same tokens and the cache's heads");
    const int32_t* cu_ptr = offsets(cu, seqs.B, device);
    if (rope_device != device) refuse("the rotation table must be on the cache's device");
    if (pos.scalar_type() != at::kInt || !on(pos, device) || pos.dim() < 1 || pos.dim() > 2 || pos.size(pos.dim() - 1) != kr.n ||
        (kr.n > 1 && pos.stride(pos.dim() - 1) != 1))
        refuse("positions must be int32 of shape [T] or [axes, T] on the cache's device, contiguous along the tokens");
    const int64_t axes = pos.dim() == 1 ? 1 : pos.size(0);
    if (axes < rope_axes || axes < 1 || axes > FA_MAX_AXES) refuse("positions must have the axes that turn the pairs, 4 at most");
    Rows qr{0, 0, {0, 0}}, or_{0, 0, {0, 0}};
    at::Tensor out;
    if (q) {
        const char* why = "q must be a 3-D bf16 tensor of the cache's head size on its device, contiguous along a head";
        qr = rows(*q, dqk, device, why);
        if (qr.n != kr.n) refuse("q must have the tokens of k");
        out = q_out ? *q_out : fresh({qr.n, qr.heads, dqk}, q->options());
        or_ = rows(out, dqk, device, "q_out must be a 3-D bf16 tensor like q");
        if (or_.n != qr.n || or_.heads != qr.heads) refuse("q_out must have q's shape");
    } else if (q_out) {
        refuse("q_out without q");
    }
    fa_positions p{};
    p.struct_size = sizeof p;
    p.axes = static_cast<int32_t>(axes);
    p.pos = ints(&pos);
    p.stride = axes > 1 ? pos.stride(0) : kr.n;
    p.axis_of_pair = axis_of_pair;
    const fa_status s = unlocked([&] {
        return p_append(h, cache, &seqs, cu_ptr, static_cast<int>(kr.n), k.data_ptr(), v.data_ptr(), q ? q->data_ptr() : nullptr,
                        q ? out.data_ptr() : nullptr, static_cast<int>(qr.heads), kr.strides, vr.strides, qr.strides, or_.strides, rope, &p,
                        stream_of(device));
    });
    if (s != FA_OK) return status(s);
    return q ? THPVariable_Wrap(std::move(out)) : Py_NewRef(Py_None);
}

// (handle, cache address, device, dqk, dv, q, block_table, seq_lens, mask, cu_seqlens, max_tokens, scale, out, want_lse) -> (out, lse)
PyObject* paged_tree(Args& a) {
    auto* h = static_cast<fa_handle*>(a.address());
    auto* cache = static_cast<const fa_paged_cache*>(a.address());
    const int device = a.integer("device");
    const int64_t dqk = a.number(), dv = a.number();
    const at::Tensor &q = a.tensor(), &table = a.tensor(), &lens = a.tensor();
    const at::Tensor *mask = a.maybe(), *cu = a.maybe();
    const int given = a.integer("max_tokens is out of range");
    const double scale = a.real();
    const at::Tensor* out_in = a.maybe();
    const bool want_lse = a.truth();
    const fa_paged_seqs seqs = sequences(h, table, lens, device);
    const Rows qr = rows(q, dqk, device, "q must be a 3-D bf16 tensor of the cache's head size on its device, contiguous along a head");
    if (qr.n && (seqs.B == 0 || (!cu && qr.n % seqs.B))) refuse("q must hold the same number of tokens for every sequence, or cu_seqlens say how many");
    const int32_t* cu_ptr = offsets(cu, seqs.B, device);
    fa_tree tree{};
    tree.struct_size = sizeof tree;
    tree.max_tokens = most_tokens(given, cu != nullptr, qr.n, seqs.B);
    tree.cu_seqlens = cu_ptr;
    const int64_t words = (static_cast<int64_t>(tree.max_tokens) + 31) / 32;
    if (mask) {
        check_mask(*mask, qr.n, words, device);
        tree.mask = reinterpret_cast<const uint32_t*>(mask->data_ptr());
        tree.mask_stride = qr.n > 1 ? mask->stride(0) : words;
    }
    at::Tensor out = out_in ? *out_in : fresh({qr.n, qr.heads, dv}, q.options());
    const Rows or_ = rows(out, dv, device, "out must be a bf16 tensor of shape [tokens, heads, dv] on the cache's device, contiguous along a head");
    if (or_.n != qr.n || or_.heads != qr.heads) refuse("out must have shape [tokens, heads, dv]");
    at::Tensor lse;
    if (want_lse) lse = fresh({qr.heads, qr.n}, q.options().dtype(at::kFloat));
    const fa_status s = unlocked([&] {
        return p_tree(h, cache, &seqs, &tree, static_cast<int>(qr.n), q.data_ptr(), out.data_ptr(), want_lse ? static_cast<float*>(lse.data_ptr()) : nullptr,
                      static_cast<int>(qr.heads), static_cast<float>(scale), qr.strides, or_.strides, stream_of(device));
    });
    return s == FA_OK ? both(std::move(out), std::move(lse)) : status(s);
}

// (handle, address of the caches, their number, device, block_table, seq_lens, keep, keep_counts, cu_seqlens, total or None, new_lens) -> new_lens
PyObject* compact(Args& a) {
    auto* h = static_cast<fa_handle*>(a.address());
    auto* caches = static_cast<const fa_paged_cache*>(a.address());
    const int count = a.integer("caches"), device = a.integer("device");
    const at::Tensor &table = a.tensor(), &lens = a.tensor(), &keep = a.tensor(), &kept = a.tensor();
    const at::Tensor* cu = a.maybe();
    const bool has_total = a.given();
    const int total = has_total ? a.integer("total is out of range") : (a.next(), 0);
    const at::Tensor* new_in = a.maybe();
    if (!cu && !has_total && table.dim() > 0 && table.size(0) > 0) refuse("total, the number of drafts of all sequences, is needed without cu_seqlens");
    const fa_paged_seqs seqs = sequences(h, table, lens, device);
    if (keep.scalar_type() != at::kInt || keep.dim() != 2 || !on(keep, device) || keep.size(0) != seqs.B || keep.size(1) < 1 || keep.size(1) > INT32_MAX ||
        (keep.size(1) > 1 && keep.stride(1) != 1) || (seqs.B > 1 && keep.stride(0) < keep.size(1)))
        refuse("keep must be int32 of shape [B, most] on the cache's device, its rows contiguous and apart");
    if (!vector_ok(kept, seqs.B, device)) refuse("keep_counts must be a contiguous int32 tensor of B numbers");
    if (new_in && (!vector_ok(*new_in, seqs.B, device) || (seqs.B && new_in->data_ptr() == lens.data_ptr())))
        refuse("new_lens must be a contiguous int32 tensor of B numbers, another one than seq_lens");
    const int32_t* cu_ptr = offsets(cu, seqs.B, device);
    at::Tensor out = new_in ? *new_in : fresh({seqs.B}, lens.options());
    const fa_status s = unlocked([&] {
        return p_compact(h, caches, count, &seqs, cu_ptr, cu ? INT32_MAX : total, ints(&keep), seqs.B > 1 ? keep.stride(0) : keep.size(1), ints(&kept),
                         static_cast<int>(keep.size(1)), ints(&out), stream_of(device));
    });
    return s == FA_OK ? THPVariable_Wrap(std::move(out)) : status(s);
}

// (handle, address of the caches, their number, device, src, dst, slots) -> None
PyObject* copy_pages(Args& a) {
    auto* h = static_cast<fa_handle*>(a.address());
    auto* caches = static_cast<const fa_paged_cache*>(a.address());
    const int count = a.integer("caches"), device = a.integer("device");
    const at::Tensor &src = a.tensor(), &dst = a.tensor();
    const at::Tensor* slots = a.maybe();
    const int64_t n = src.dim() == 1 ? src.size(0) : -1;
    if (n < 0 || n > INT32_MAX || !vector_ok(src, n, device) || !vector_ok(dst, n, device) || (slots && !vector_ok(*slots, n, device)))
        refuse("src, dst and slots must be contiguous 1-D int32 tensors of one length on the caches' device");
    if (p_device(h) != device) refuse("the handle belongs to another device than the caches");
    const fa_status s = unlocked([&] { return p_copy(h, caches, count, ints(&src), ints(&dst), ints(slots), static_cast<int>(n), stream_of(device)); });
    return s == FA_OK ? Py_NewRef(Py_None) : status(s);
}

template <PyObject* (*kCall)(Args&)>
PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    try {
        Args a{args, n};
        return kCall(a);
    } catch (const Refused&) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&call<bind>)), METH_FASTCALL, nullptr},
    {"tree_layout", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&call<tree_layout>)), METH_FASTCALL, nullptr},
    {"append_at", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&call<append_at>)), METH_FASTCALL, nullptr},
    {"paged_tree", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&call<paged_tree>)), METH_FASTCALL, nullptr},
    {"compact", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&call<compact>)), METH_FASTCALL, nullptr},
    {"copy_pages", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&call<copy_pages>)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fa_calls", "Checks, outputs and launches of the calls on drafted tokens.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fa_calls() { return PyModule_Create(&module); }
