// Python entry points of the paged-cache calls: they check tensors, fill the C structures of bd.h and call the library.
// A decode step makes these calls once per layer with a dozen tensors each, and reading that many tensors' fields from
// Python takes longer than the kernels run; here a call costs the host about as much as its launches.
// Nothing is kept between calls.  Errors of the library go through the Python function given to set_check.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <stdexcept>
#include <string>

#include "../../include/bd.h"

namespace {

PyObject *g_check = nullptr;

struct Raised {};                                                  // a Python error is already set

[[noreturn]] void refuse(const std::string &text) { throw std::invalid_argument(text); }

const at::Tensor &tensor(PyObject *o, const char *what) {
    if (!THPVariable_Check(o)) refuse(std::string(what) + " must be a tensor");
    return THPVariable_Unpack(o);
}
void here(const at::Tensor &t, const char *what) {
    if (!t.is_cuda() || t.get_device() != c10::cuda::current_device()) refuse(std::string(what) + " must be on the current CUDA device");
}
bool dtype_of(at::ScalarType s, bd_dtype *dt) {
    if (s == at::kFloat) *dt = BD_F32;
    else if (s == at::kBFloat16) *dt = BD_BF16;
    else if (s == at::kHalf) *dt = BD_F16;
    else return false;
    return true;
}
at::ScalarType scalar_of(bd_dtype dt) { return dt == BD_F32 ? at::kFloat : dt == BD_BF16 ? at::kBFloat16 : at::kHalf; }
int64_t integer(PyObject *o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised();
    return v;
}
double real(PyObject *o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Raised();
    return v;
}
// The call's stream: the current one, or the one given, which then also is the stream of what the call allocates.
struct StreamScope {
    c10::cuda::OptionalCUDAStreamGuard guard;
    void *raw;
    explicit StreamScope(PyObject *o) {
        if (o != Py_None) {
            PyObject *v = PyObject_GetAttrString(o, "cuda_stream");
            if (!v) throw Raised();
            raw = PyLong_AsVoidPtr(v);
            Py_DECREF(v);
            if (PyErr_Occurred()) throw Raised();
            const auto current = c10::cuda::getCurrentCUDAStream();
            if (raw != current.stream()) guard.reset_stream(c10::cuda::getStreamFromExternal((cudaStream_t)raw, current.device_index()));
        } else {
            raw = c10::cuda::getCurrentCUDAStream().stream();
        }
    }
};
void check(bd_status s) {
    if (s == BD_OK) return;
    PyObject *r = PyObject_CallFunction(g_check, "i", (int)s);
    if (r) {
        Py_DECREF(r);
        PyErr_SetString(PyExc_RuntimeError, "the library returned an error");
    }
    throw Raised();
}
// A descriptor as Python keeps it, with the device its buffers are on.
template <typename T>
struct Held {
    T s;
    int64_t device;
};
template <typename T>
PyObject *hold(const T &s) {
    const Held<T> h{s, (int64_t)c10::cuda::current_device()};
    return PyBytes_FromStringAndSize((const char *)&h, sizeof h);
}
template <typename T>
const T &structure(PyObject *o) {
    if (!PyBytes_Check(o) || PyBytes_GET_SIZE(o) != (Py_ssize_t)sizeof(Held<T>)) refuse("not a descriptor of this module");
    const Held<T> &h = *(const Held<T> *)PyBytes_AS_STRING(o);
    if (h.device != c10::cuda::current_device()) refuse("cache and batch must be on the current CUDA device");
    return h.s;
}
void need(Py_ssize_t got, Py_ssize_t want) {
    if (got != want) refuse("wrong number of arguments");
}

// [rows, heads, head_dim] with a contiguous last axis; strides of axes of one element mean nothing
struct Rows {
    void *p;
    int64_t ld, hs;
};
Rows rows3(const at::Tensor &x, const char *what, int64_t heads, int64_t d, at::ScalarType dt) {
    if (x.dim() != 3 || x.size(1) != heads || x.size(2) != d || x.scalar_type() != dt || (x.stride(2) != 1 && x.numel()))
        refuse(std::string(what) + " must be [rows, " + std::to_string(heads) + ", " + std::to_string(d) + "] of " + c10::toString(dt) +
               " with a contiguous last axis");
    here(x, what);
    Rows r{x.data_ptr(), x.stride(0), heads > 1 ? x.stride(1) : d};
    if (x.size(0) <= 1) r.ld = heads * d;
    return r;
}

PyObject *cache(PyObject *const *a, Py_ssize_t n) {
    need(n, 3);
    const at::Tensor &pool = tensor(a[0], "pool"), &tail = tensor(a[1], "tail");
    bd_paged_cache c{};
    c.page_tokens = integer(a[2]);
    if (tail.dim() != 4 || !dtype_of(tail.scalar_type(), &c.dtype) || tail.size(2) != 64 || !tail.is_contiguous())
        refuse("tail must be contiguous [slots, kv_heads, 64, head_dim] of fp32/bf16/fp16");
    c.slots = tail.size(0); c.kv_heads = tail.size(1); c.head_dim = tail.size(3);
    if (pool.scalar_type() != at::kByte || pool.dim() != 4 || pool.size(1) != c.kv_heads || c.page_tokens <= 0 || c.page_tokens % 32 ||
        pool.size(2) != c.page_tokens / 32 || pool.size(3) != 35 * c.head_dim || !pool.is_contiguous())
        refuse("pool must be contiguous uint8 [pages, kv_heads, page_tokens / 32, 35 * head_dim]");
    here(pool, "pool");
    here(tail, "tail");
    c.pages = pool.size(0); c.pool = pool.data_ptr(); c.tail = tail.data_ptr();
    return hold(c);
}

PyObject *batch(PyObject *const *a, Py_ssize_t n) {
    need(n, 6);
    const at::Tensor &table = tensor(a[0], "page_table"), &slots = tensor(a[1], "slots"), &kv = tensor(a[2], "kv_len"), &start = tensor(a[3], "q_start");
    for (const at::Tensor *x : {&table, &slots, &kv, &start}) {
        if (x->scalar_type() != at::kInt || x->dim() == 0 || (x->stride(-1) != 1 && x->size(-1) > 1)) refuse("the batch's index tensors must be int32 with a contiguous last axis");
        here(*x, "the batch");
    }
    const int64_t m = kv.size(0);
    if (table.dim() != 2 || table.size(0) != m || slots.dim() != 1 || slots.size(0) != m || kv.dim() != 1 || start.dim() != 1 || start.size(0) != m + 1)
        refuse("page_table [n, width], slots [n], kv_len [n], q_start [n + 1]");
    if (m > 1 && table.stride(0) < table.size(1)) refuse("the page table's rows overlap");
    bd_paged_batch b{};
    b.page_table = (const int32_t *)table.data_ptr(); b.slot = (const int32_t *)slots.data_ptr();
    b.kv_len = (const int32_t *)kv.data_ptr(); b.q_start = (const int32_t *)start.data_ptr();
    b.ld_table = m > 1 ? table.stride(0) : table.size(1);
    b.n = m; b.max_q = integer(a[4]); b.max_kv = a[5] == Py_None ? -1 : integer(a[5]);
    b.rows = table.size(1);                                       // the table's width until a call's rows are known
    return hold(b);
}
// The descriptor of one call: bounds completed from the call's rows and the cache's pages.
bd_paged_batch batch_for(const bd_paged_batch &b0, const bd_paged_cache &c, int64_t rows) {
    bd_paged_batch b = b0;
    const int64_t held = b0.rows * c.page_tokens;
    if (b.max_kv > held) refuse("max_kv exceeds what the page table can hold");
    if (b.max_kv < 0) b.max_kv = held;
    b.rows = rows;
    b.max_q = std::min(b.max_q, rows);
    return b;
}

PyObject *append(PyObject *const *a, Py_ssize_t n) {
    need(n, 5);
    const bd_paged_cache &c = structure<bd_paged_cache>(a[0]);
    const at::Tensor &k = tensor(a[2], "keys"), &v = tensor(a[3], "values");
    const Rows rk = rows3(k, "keys", c.kv_heads, c.head_dim, scalar_of(c.dtype)), rv = rows3(v, "values", c.kv_heads, c.head_dim, scalar_of(c.dtype));
    if (k.size(0) != v.size(0)) refuse("keys and values must have the same number of rows");
    if (k.size(0)) {
        const bd_paged_batch b = batch_for(structure<bd_paged_batch>(a[1]), c, k.size(0));
        check(bd_paged_append(&c, &b, rk.p, rv.p, rk.ld, rk.hs, rv.ld, rv.hs, StreamScope(a[4]).raw));
    }
    Py_RETURN_NONE;
}

PyObject *read(PyObject *const *a, Py_ssize_t n) {
    need(n, 6);
    const bd_paged_cache &c = structure<bd_paged_cache>(a[0]);
    const at::ScalarType dt = scalar_of(c.dtype);
    const StreamScope stream(a[5]);
    at::Tensor out[2];
    for (int i = 0; i < 2; i++) {
        if (a[3 + i] != Py_None) { out[i] = tensor(a[3 + i], "out"); continue; }
        if (a[2] == Py_None) refuse("give the number of rows or both buffers");
        out[i] = at::empty({integer(a[2]), c.kv_heads, c.head_dim}, at::TensorOptions().dtype(dt).device(at::kCUDA, c10::cuda::current_device()));
    }
    const Rows rk = rows3(out[0], "out_k", c.kv_heads, c.head_dim, dt), rv = rows3(out[1], "out_v", c.kv_heads, c.head_dim, dt);
    if (out[0].size(0) != out[1].size(0)) refuse("the buffers must have the same number of rows");
    if (out[0].size(0)) {
        const bd_paged_batch b = batch_for(structure<bd_paged_batch>(a[1]), c, out[0].size(0));
        check(bd_paged_read(&c, &b, rk.p, rv.p, rk.ld, rk.hs, rv.ld, rv.hs, stream.raw));
    }
    PyObject *x = THPVariable_Wrap(out[0]), *y = THPVariable_Wrap(out[1]);
    PyObject *r = x && y ? PyTuple_Pack(2, x, y) : nullptr;
    Py_XDECREF(x);
    Py_XDECREF(y);
    return r;
}

PyObject *workspace_size(PyObject *const *a, Py_ssize_t n) {
    need(n, 4);
    const bd_paged_cache &c = structure<bd_paged_cache>(a[0]);
    const bd_paged_batch b = batch_for(structure<bd_paged_batch>(a[1]), c, integer(a[2]));
    size_t bytes = 0;
    check(bd_paged_attention_workspace_size(&c, &b, integer(a[3]), &bytes));
    return PyLong_FromSize_t(bytes);
}

PyObject *attention(PyObject *const *a, Py_ssize_t n) {
    need(n, 11);
    const bd_paged_cache &c = structure<bd_paged_cache>(a[0]);
    const at::Tensor &q = tensor(a[2], "q");
    if (q.dim() != 3) refuse("q must be [rows, q_heads, head_dim]");
    const int64_t rows = q.size(0), heads = q.size(1), d = c.head_dim;
    if (heads <= 0 || heads % c.kv_heads) refuse("the number of query heads must be a multiple of the number of KV heads");
    const Rows rq = rows3(q, "q", heads, d, scalar_of(c.dtype));
    const StreamScope stream(a[10]);
    at::Tensor out;
    if (a[6] != Py_None) {
        out = tensor(a[6], "out");
    } else {
        at::ScalarType dt = q.scalar_type();
        if (a[7] != Py_None) {
            if (!THPDtype_Check(a[7])) refuse("dtype must be a torch.dtype");
            dt = ((THPDtype *)a[7])->scalar_type;
        }
        out = at::empty({rows, heads, d}, q.options().dtype(dt));
    }
    bd_dtype odt;
    if (out.dim() != 3 || out.size(0) != rows || !dtype_of(out.scalar_type(), &odt)) refuse("out must have the rows of q");
    const Rows ro = rows3(out, "out", heads, d, out.scalar_type());
    float *lse = nullptr;
    if (a[8] != Py_None) {
        const at::Tensor &l = tensor(a[8], "lse");
        if (l.dim() != 2 || l.size(0) != rows || l.size(1) != heads || l.scalar_type() != at::kFloat || !l.is_contiguous()) refuse("lse must be contiguous fp32 [rows, q_heads]");
        here(l, "lse");
        lse = l.data_ptr<float>();
    }
    if (rows) {
        const bd_paged_batch b = batch_for(structure<bd_paged_batch>(a[1]), c, rows);
        at::Tensor ws;
        if (a[9] != Py_None) {
            ws = tensor(a[9], "workspace");
            here(ws, "workspace");
            if (!ws.is_contiguous()) refuse("workspace must be contiguous");
        } else {
            size_t bytes = 0;
            check(bd_paged_attention_workspace_size(&c, &b, heads, &bytes));
            if (bytes) ws = at::empty({(int64_t)bytes}, q.options().dtype(at::kByte));
        }
        const float scale = a[3] == Py_None ? 1.0f / std::sqrt((float)d) : (float)real(a[3]);
        check(bd_paged_attention(&c, &b, rq.p, heads, rq.ld, rq.hs, scale, (float)real(a[4]), integer(a[5]), ro.p, odt, ro.ld, ro.hs, lse,
                                 ws.defined() ? ws.data_ptr() : nullptr, ws.defined() ? (size_t)ws.nbytes() : 0, stream.raw));
    }
    return THPVariable_Wrap(out);
}

PyObject *rope(PyObject *const *a, Py_ssize_t n) {
    need(n, 11);
    const at::Tensor &q = tensor(a[0], "q");
    bd_dtype dt;
    if (q.dim() != 3 || !dtype_of(q.scalar_type(), &dt)) refuse("q must be [rows, heads, head_dim] of fp32/bf16/fp16");
    const int64_t rows = q.size(0), d = q.size(2);
    const at::Tensor &pos = tensor(a[2], "positions"), &table = tensor(a[3], "cos_sin");
    if (pos.scalar_type() != at::kInt || pos.dim() != 1 || pos.size(0) != rows || (rows > 1 && pos.stride(0) != 1)) refuse("positions must be int32 [rows]");
    if (table.scalar_type() != at::kFloat || table.dim() != 2 || !table.is_contiguous()) refuse("cos_sin must be contiguous fp32 [positions, rot]");
    here(pos, "positions");
    here(table, "cos_sin");
    const int il = PyObject_IsTrue(a[7]);
    if (il < 0) throw Raised();
    const StreamScope stream(a[10]);
    at::Tensor out[2];
    bd_rope_operand op[2] = {};
    for (int i = 0; i < 2; i++) {
        const char *what = i ? "k" : "q";
        if (a[i] == Py_None) continue;
        const at::Tensor &x = tensor(a[i], what);
        out[i] = a[8 + i] == Py_None ? at::empty(x.sizes(), x.options()) : tensor(a[8 + i], what);
        if (x.dim() != 3 || x.size(0) != rows || out[i].sizes() != x.sizes()) refuse("q, k and their outputs must have the same rows, an output its input's shape");
        const Rows rx = rows3(x, what, x.size(1), d, q.scalar_type()), ry = rows3(out[i], "output", x.size(1), d, q.scalar_type());
        const void *w = nullptr;
        if (a[4 + i] != Py_None) {
            const at::Tensor &t = tensor(a[4 + i], "weight");
            if (t.dim() != 1 || t.size(0) != d || t.scalar_type() != q.scalar_type() || !t.is_contiguous()) refuse("a weight must be contiguous [head_dim] of the rows' type");
            here(t, "weight");
            w = t.data_ptr();
        }
        op[i] = bd_rope_operand{rx.p, ry.p, w, x.size(1), rx.ld, rx.hs, ry.ld, ry.hs};
    }
    if (rows)
        check(bd_qk_norm_rope(&op[0], &op[1], dt, rows, d, pos.data_ptr<int32_t>(), table.data_ptr<float>(), table.size(0), table.size(1), il, (float)real(a[6]),
                              stream.raw));
    PyObject *x = THPVariable_Wrap(out[0]), *y = out[1].defined() ? THPVariable_Wrap(out[1]) : Py_NewRef(Py_None);
    PyObject *r = x && y ? PyTuple_Pack(2, x, y) : nullptr;
    Py_XDECREF(x);
    Py_XDECREF(y);
    return r;
}

PyObject *set_check(PyObject *const *a, Py_ssize_t n) {
    need(n, 1);
    Py_INCREF(a[0]);
    Py_XSETREF(g_check, a[0]);
    Py_RETURN_NONE;
}

// No C++ exception leaves an entry point.
template <PyObject *(*F)(PyObject *const *, Py_ssize_t)>
PyObject *entry(PyObject *, PyObject *const *a, Py_ssize_t n) {
    try {
        return F(a, n);
    } catch (const Raised &) {
    } catch (const std::invalid_argument &e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const c10::OutOfMemoryError &e) {
        PyErr_SetString(PyExc_MemoryError, e.what_without_backtrace());
    } catch (const c10::Error &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}
#define BD_ENTRY(f) {#f, (PyCFunction)(void (*)(void)) & entry<f>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {BD_ENTRY(cache), BD_ENTRY(batch), BD_ENTRY(append), BD_ENTRY(read), BD_ENTRY(workspace_size), BD_ENTRY(attention), BD_ENTRY(rope),
                         BD_ENTRY(set_check), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_paged", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__paged() { return PyModule_Create(&module); }
