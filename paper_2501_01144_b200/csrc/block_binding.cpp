// Python entry points of the mixture-of-experts and norm calls: they check tensors, fill the C structures of bd.h and call the library.
#include "binding_common.h"

namespace {

// A matrix [rows, cols] with a contiguous last axis; the stride of an axis of one element means nothing.
struct Matrix {
    void *p;
    int64_t ld;
};
Matrix matrix(const at::Tensor &x, const char *what, int64_t rows, int64_t cols, at::ScalarType dt) {
    if (x.dim() != 2 || x.size(0) != rows || x.size(1) != cols || x.scalar_type() != dt || (x.stride(1) != 1 && cols > 1 && rows > 0))
        refuse(std::string(what) + " must be [" + std::to_string(rows) + ", " + std::to_string(cols) + "] of " + c10::toString(dt) + " with a contiguous last axis");
    here(x, what);
    return Matrix{x.data_ptr(), rows > 1 ? x.stride(0) : cols};
}
const at::Tensor &whole(PyObject *o, const char *what, at::ScalarType dt, at::IntArrayRef shape) {
    const at::Tensor &x = tensor(o, what);
    if (x.scalar_type() != dt || x.sizes() != shape || !x.is_contiguous()) {
        std::string s;
        for (int64_t n : shape) s += (s.empty() ? "" : ", ") + std::to_string(n);
        refuse(std::string(what) + " must be contiguous " + c10::toString(dt) + " [" + s + "]");
    }
    here(x, what);
    return x;
}
at::TensorOptions on_device(at::ScalarType dt) { return at::TensorOptions().dtype(dt).device(at::kCUDA, c10::cuda::current_device()); }
bool truth(PyObject *o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Raised();
    return v != 0;
}

// A tensor on a part of another one's storage, `at` bytes in (as a view would be, without the dispatcher's share of its cost).
at::Tensor part(const at::Tensor &whole, int64_t at, at::ScalarType dt, at::IntArrayRef shape) {
    auto impl = c10::make_intrusive<c10::TensorImpl>(c10::Storage(whole.storage()), whole.key_set(), c10::scalarTypeToTypeMeta(dt));
    impl->set_storage_offset(at / (int64_t)c10::elementSize(dt));
    impl->set_sizes_contiguous(shape);
    return at::Tensor(std::move(impl));
}
int64_t padded(int64_t bytes) { return (bytes + 255) / 256 * 256; }

bd_expert_plan plan_of(const at::Tensor &count, const at::Tensor &start, const at::Tensor &place, const at::Tensor &scratch) {
    bd_expert_plan p{};
    p.count = count.data_ptr<int32_t>(); p.start = start.data_ptr<int32_t>(); p.place = place.data_ptr<int32_t>();
    p.scratch = scratch.numel() ? scratch.data_ptr() : nullptr;
    p.tokens = place.size(0); p.top_k = place.size(1); p.experts = count.size(0);
    return p;
}
struct PlanTensors {
    at::Tensor count, start, place, scratch;
};
// The tensors of a new plan, and `more` bytes in front of them, in one allocation.
PlanTensors new_plan(int64_t tokens, int64_t top_k, int64_t experts, int64_t more, at::Tensor *all) {
    size_t bytes = 0;
    check(bd_expert_plan_scratch(tokens, experts, &bytes));
    const int64_t index = padded(more), scratch = index + padded(4 * (2 * experts + 1 + tokens * top_k));
    *all = at::empty({scratch + (int64_t)bytes}, on_device(at::kByte));
    return {part(*all, index, at::kInt, {experts}), part(*all, index + 4 * experts, at::kInt, {experts + 1}), part(*all, index + 4 * (2 * experts + 1), at::kInt, {tokens, top_k}),
            part(*all, scratch, at::kByte, {(int64_t)bytes})};
}
PlanTensors given_plan(PyObject *o, int64_t tokens, int64_t top_k, int64_t experts) {
    if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 4) refuse("plan must be an ExpertPlan");
    size_t bytes = 0;
    check(bd_expert_plan_scratch(tokens, experts, &bytes));
    PlanTensors t;
    t.count = whole(PyTuple_GET_ITEM(o, 0), "the plan's count", at::kInt, {experts});
    t.start = whole(PyTuple_GET_ITEM(o, 1), "the plan's start", at::kInt, {experts + 1});
    t.place = whole(PyTuple_GET_ITEM(o, 2), "the plan's place", at::kInt, {tokens, top_k});
    t.scratch = whole(PyTuple_GET_ITEM(o, 3), "the plan's scratch", at::kByte, {(int64_t)bytes});
    return t;
}
PyObject *tuple_of(std::initializer_list<at::Tensor> tensors) {
    PyObject *r = PyTuple_New((Py_ssize_t)tensors.size());
    if (!r) throw Raised();
    Py_ssize_t i = 0;
    for (const at::Tensor &t : tensors) {
        PyObject *x = t.defined() ? THPVariable_Wrap(t) : Py_NewRef(Py_None);
        if (!x) {
            Py_DECREF(r);
            throw Raised();
        }
        PyTuple_SET_ITEM(r, i++, x);
    }
    return r;
}

// logits, top_k, sigmoid, bias, groups, top_groups, group_top, renormalise, scale, valid, out ids, out weights, plan tensors or None, wants a plan, stream
PyObject *route(PyObject *const *a, Py_ssize_t n) {
    need(n, 15);
    const at::Tensor &x = tensor(a[0], "logits");
    bd_dtype dt;
    if (x.dim() != 2 || !dtype_of(x.scalar_type(), &dt)) refuse("logits must be [tokens, experts] of fp32/bf16/fp16");
    const int64_t tokens = x.size(0), experts = x.size(1), k = integer(a[1]);
    if (experts < 1 || k < 1 || k > experts) refuse("top_k must lie between 1 and the number of experts");
    const Matrix m = matrix(x, "logits", tokens, experts, x.scalar_type());
    bd_route_rule r{};
    r.score = truth(a[2]) ? BD_SCORE_SIGMOID : BD_SCORE_SOFTMAX;
    r.experts = experts; r.top_k = k; r.groups = integer(a[4]); r.top_groups = integer(a[5]);
    r.group_top = (int)integer(a[6]); r.renormalise = truth(a[7]); r.scale = (float)real(a[8]);
    const float *bias = a[3] == Py_None ? nullptr : whole(a[3], "bias", at::kFloat, {experts}).data_ptr<float>();
    const int32_t *valid = nullptr;
    if (a[9] != Py_None) {
        const at::Tensor &v = tensor(a[9], "valid");
        if (v.scalar_type() != at::kInt || v.numel() != 1) refuse("valid must be one int32");
        here(v, "valid");
        valid = v.data_ptr<int32_t>();
    }
    const StreamScope stream(a[14]);
    const bool wants = truth(a[13]), fresh = wants && a[12] == Py_None;
    const int64_t ids_bytes = a[10] == Py_None ? padded(4 * tokens * k) : 0, w_bytes = a[11] == Py_None ? padded(4 * tokens * k) : 0;
    PlanTensors t;
    at::Tensor all;
    if (fresh) t = new_plan(tokens, k, experts, ids_bytes + w_bytes, &all);
    else if (ids_bytes + w_bytes || tokens == 0) all = at::empty({ids_bytes + w_bytes}, on_device(at::kByte));
    if (wants && !fresh) t = given_plan(a[12], tokens, k, experts);
    const at::Tensor ids = a[10] == Py_None ? part(all, 0, at::kInt, {tokens, k}) : whole(a[10], "ids", at::kInt, {tokens, k});
    const at::Tensor w = a[11] == Py_None ? part(all, ids_bytes, at::kFloat, {tokens, k}) : whole(a[11], "weights", at::kFloat, {tokens, k});
    bd_expert_plan p{};
    if (wants) p = plan_of(t.count, t.start, t.place, t.scratch);
    check(bd_route(m.p, dt, tokens, m.ld, bias, &r, valid, ids.data_ptr<int32_t>(), w.data_ptr<float>(), wants ? &p : nullptr, stream.raw));
    return tuple_of({ids, w, t.count, t.start, t.place, t.scratch});
}

// ids, experts, plan tensors or None, stream
PyObject *plan(PyObject *const *a, Py_ssize_t n) {
    need(n, 4);
    const at::Tensor &ids = tensor(a[0], "ids");
    const int64_t experts = integer(a[1]);
    if (ids.dim() != 2 || ids.scalar_type() != at::kInt || !ids.is_contiguous() || ids.size(1) < 1 || experts < 1) refuse("ids must be contiguous int32 [tokens, top_k]");
    here(ids, "ids");
    const int64_t tokens = ids.size(0), k = ids.size(1);
    const StreamScope stream(a[3]);
    PlanTensors t;
    if (a[2] == Py_None) {
        at::Tensor all;
        t = new_plan(tokens, k, experts, 0, &all);
    } else {
        t = given_plan(a[2], tokens, k, experts);
    }
    const bd_expert_plan p = plan_of(t.count, t.start, t.place, t.scratch);
    check(bd_make_expert_plan(ids.data_ptr<int32_t>(), &p, stream.raw));
    return tuple_of({t.count, t.start, t.place, t.scratch});
}

// codes, ids, scales, rows, K -> descriptor of a stack of operands
PyObject *experts(PyObject *const *a, Py_ssize_t n) {
    need(n, 5);
    bd_experts w{};
    w.rows = integer(a[3]); w.K = integer(a[4]);
    size_t bytes[3];
    check(bd_qtensor_sizes(w.rows, w.K, &bytes[0], &bytes[1], &bytes[2]));
    const at::Tensor &c = tensor(a[0], "codes");
    if (c.dim() != 2 || c.size(0) < 1) refuse("codes must be uint8 [experts, bytes of an operand]");
    w.experts = c.size(0);
    w.codes = whole(a[0], "codes", at::kByte, {w.experts, (int64_t)bytes[0]}).data_ptr();
    w.ids = whole(a[1], "ids", at::kByte, {w.experts, (int64_t)bytes[1]}).data_ptr();
    w.scales = whole(a[2], "scales", at::kByte, {w.experts, (int64_t)bytes[2]}).data_ptr();
    return hold(w);
}

const bd_experts &weights_of(PyObject *o) { return structure<bd_experts>(o, "the experts' weights"); }
bd_dtype output_type(PyObject *o, at::ScalarType *s) {
    if (!THPDtype_Check(o)) refuse("dtype must be a torch.dtype");
    bd_dtype dt;
    *s = ((THPDtype *)o)->scalar_type;
    if (!dtype_of(*s, &dt) || dt == BD_F16) refuse("output dtype must be float32 or bfloat16");
    return dt;
}
// tokens, top_k, up, down, dtype
PyObject *mlp_workspace_size(PyObject *const *a, Py_ssize_t n) {
    need(n, 5);
    at::ScalarType s;
    size_t bytes = 0;
    output_type(a[4], &s);                                         // (either type: room for the fp32 parts of all columns at once)
    check(bd_expert_mlp_workspace_size(integer(a[0]), integer(a[1]), &weights_of(a[2]), &weights_of(a[3]), BD_F32, &bytes));
    return PyLong_FromSize_t(bytes);
}

// x, count, start, place, weights, up, down, gelu, out, dtype, inner, workspace, stream
PyObject *mlp(PyObject *const *a, Py_ssize_t n) {
    need(n, 13);
    const bd_experts &up = weights_of(a[5]), &down = weights_of(a[6]);
    const at::Tensor &x = tensor(a[0], "x"), &place = tensor(a[3], "the plan's place");
    bd_dtype xdt;
    if (x.dim() != 2 || !dtype_of(x.scalar_type(), &xdt)) refuse("x must be [tokens, K] of fp32/bf16/fp16");
    const int64_t tokens = x.size(0);
    const Matrix mx = matrix(x, "x", tokens, up.K, x.scalar_type());
    if (place.dim() != 2 || place.size(0) != tokens) refuse("the plan must be one for the rows of x");
    const int64_t k = place.size(1);
    bd_expert_plan p{};
    p.count = whole(a[1], "the plan's count", at::kInt, {up.experts}).data_ptr<int32_t>();
    p.start = whole(a[2], "the plan's start", at::kInt, {up.experts + 1}).data_ptr<int32_t>();
    p.place = whole(a[3], "the plan's place", at::kInt, {tokens, k}).data_ptr<int32_t>();
    p.tokens = tokens; p.top_k = k; p.experts = up.experts;
    const float *w = whole(a[4], "weights", at::kFloat, {tokens, k}).data_ptr<float>();
    const bool gelu = truth(a[7]);
    const StreamScope stream(a[12]);
    at::ScalarType s;
    bd_dtype ydt = output_type(a[9], &s);
    at::Tensor out;
    if (a[8] != Py_None) {
        out = tensor(a[8], "out");
        if (!dtype_of(out.scalar_type(), &ydt) || ydt == BD_F16) refuse("output dtype must be float32 or bfloat16");
    } else {
        out = at::empty({tokens, down.rows}, on_device(s));
    }
    const Matrix my = matrix(out, "out", tokens, down.rows, out.scalar_type());
    float *inner = a[10] == Py_None ? nullptr : whole(a[10], "inner", at::kFloat, {tokens, k, down.K}).data_ptr<float>();
    if (tokens) {
        at::Tensor ws;
        if (a[11] != Py_None) {
            ws = tensor(a[11], "workspace");
            here(ws, "workspace");
            if (!ws.is_contiguous()) refuse("workspace must be contiguous");
        } else {
            size_t bytes = 0;
            check(bd_expert_mlp_workspace_size(tokens, k, &up, &down, BD_F32, &bytes));   // (room for the parts of all columns at once)
            ws = at::empty({(int64_t)bytes}, on_device(at::kByte));
        }
        check(bd_expert_mlp(mx.p, xdt, tokens, mx.ld, &p, w, &up, &down, gelu ? BD_ACT_GELU : BD_ACT_SILU, my.p, ydt, my.ld, inner, ws.data_ptr(), (size_t)ws.nbytes(),
                            stream.raw));
    }
    return THPVariable_Wrap(out);
}

// y, weight, residual, bias, post_weight, post_bias, gate, scale, layer, eps, offset, want_h, out_h, out_n, (codes, ids, scales) or True (new ones) or None, stream
PyObject *norm(PyObject *const *a, Py_ssize_t n) {
    need(n, 16);
    const at::Tensor &y = tensor(a[0], "y");
    bd_dtype dt;
    if (y.dim() != 2 || !dtype_of(y.scalar_type(), &dt)) refuse("y must be [rows, dim] of fp32/bf16/fp16");
    const at::ScalarType st = y.scalar_type();
    const int64_t rows = y.size(0), dim = y.size(1);
    bd_norm k{};
    auto rows_of = [&](const at::Tensor &x, const char *what, int64_t *ld) {
        const Matrix m = matrix(x, what, rows, dim, st);
        *ld = m.ld;
        return m.p;
    };
    auto vector = [&](PyObject *o, const char *what) -> const void * { return o == Py_None ? nullptr : whole(o, what, st, {dim}).data_ptr(); };
    k.y = rows_of(y, "y", &k.ldy);
    k.weight = vector(a[1], "weight"); k.bias = vector(a[3], "bias"); k.post_weight = vector(a[4], "post_weight"); k.post_bias = vector(a[5], "post_bias");
    if (a[2] != Py_None) k.residual = rows_of(tensor(a[2], "residual"), "residual", &k.ld_residual);
    if (a[6] != Py_None) {
        const at::Tensor &g = tensor(a[6], "gate");
        if (g.dim() != 2 || g.scalar_type() != st || (g.size(0) != rows && g.size(0) != 1) || (g.size(1) != dim && g.size(1) != 1) || (g.size(1) > 1 && g.stride(1) != 1))
            refuse("gate must be [rows or 1, dim or 1] of the rows' type with a contiguous last axis");
        here(g, "gate");
        k.gate = g.data_ptr();
        k.gate_row = g.size(0) == 1 ? 0 : g.stride(0);
        k.gate_col = g.size(1) == 1 ? 0 : 1;
    }
    k.scale = (float)real(a[7]); k.layer = truth(a[8]); k.eps = (float)real(a[9]); k.weight_offset = (float)real(a[10]);
    const StreamScope stream(a[15]);
    at::Tensor h, out;
    if (truth(a[11])) {
        h = a[12] == Py_None ? at::empty({rows, dim}, on_device(st)) : tensor(a[12], "out_h");
        k.h = rows_of(h, "out_h", &k.ldh);
    }
    bd_qtensor q{};
    at::Tensor operand[3];
    if (a[14] != Py_None) {
        size_t bytes[3] = {0, 0, 0};
        check(bd_qtensor_sizes(rows, dim, &bytes[0], &bytes[1], &bytes[2]));
        if (a[14] == Py_True) {
            int64_t at[3], total = 0;
            for (int i = 0; i < 3; i++) {
                at[i] = total;
                total += padded((int64_t)bytes[i]);
            }
            const at::Tensor all = at::empty({total}, on_device(at::kByte));
            for (int i = 0; i < 3; i++) operand[i] = part(all, at[i], at::kByte, {(int64_t)bytes[i]});
        } else {
            if (!PyTuple_Check(a[14]) || PyTuple_GET_SIZE(a[14]) != 3) refuse("out_n must be a QTensor");
            for (int i = 0; i < 3; i++) operand[i] = whole(PyTuple_GET_ITEM(a[14], i), "a buffer of out_n", at::kByte, {(int64_t)bytes[i]});
        }
        void **slot[3] = {&q.codes, &q.ids, &q.scales};
        for (int i = 0; i < 3; i++) *slot[i] = operand[i].data_ptr();
        q.rows = rows; q.K = dim;
        k.q = &q;
    } else if (k.weight) {
        out = a[13] == Py_None ? at::empty({rows, dim}, on_device(st)) : tensor(a[13], "out_n");
        k.n = rows_of(out, "out_n", &k.ldn);
    }
    if (rows) check(bd_residual_norm(&k, dt, rows, dim, stream.raw));
    return tuple_of({h, out, operand[0], operand[1], operand[2]});
}

// codes, ids, scales, rows, K, stream -> fp32 [rows, K]; None where the operand's buffers are not exactly its own on the current device
PyObject *dequantize(PyObject *const *a, Py_ssize_t n) {
    need(n, 6);
    bd_qtensor q{};
    q.rows = integer(a[3]); q.K = integer(a[4]);
    size_t bytes[3];
    check(bd_qtensor_sizes(q.rows, q.K, &bytes[0], &bytes[1], &bytes[2]));
    void **slot[3] = {&q.codes, &q.ids, &q.scales};
    for (int i = 0; i < 3; i++) {
        if (!THPVariable_Check(a[i])) Py_RETURN_NONE;
        const at::Tensor &x = THPVariable_Unpack(a[i]);
        if (x.scalar_type() != at::kByte || x.numel() != (int64_t)bytes[i] || !x.is_contiguous() || !x.is_cuda() || x.get_device() != c10::cuda::current_device()) Py_RETURN_NONE;
        *slot[i] = x.data_ptr();
    }
    const StreamScope stream(a[5]);
    const at::Tensor out = at::empty({q.rows, q.K}, on_device(at::kFloat));
    check(bd_dequantize(&q, out.data_ptr<float>(), q.K, stream.raw));
    return THPVariable_Wrap(out);
}

PyMethodDef methods[] = {BD_ENTRY(route), BD_ENTRY(plan), BD_ENTRY(experts), BD_ENTRY(mlp_workspace_size), BD_ENTRY(mlp), BD_ENTRY(norm), BD_ENTRY(dequantize), BD_ENTRY(set_check),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_block", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__block() { return PyModule_Create(&module); }
