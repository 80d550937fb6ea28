// The host side of the calls that stand in every layer of a step: argument structs of include/dlm.h filled from torch tensors.
//
// A call of dlm_paged_append looks at twelve tensors (type, device, shape, strides, pointer).  Read from Python that is 0.6 us a tensor and
// 18 us a call, four times the kernel of a decoding step; here the whole call is 1 us beside the launch.  Only marshalling: every function takes the
// raw stream and its arguments by position (binding.py has the names), refuses tensors that do not fit with ValueError,
// and returns the library's code.
#define PY_SSIZE_T_CLEAN
#include <torch/csrc/autograd/python_variable.h>

#include "dlm.h"

namespace {

struct Refused {};      // a Python error is set

[[noreturn]] void refuse(const char* name, const char* what) {
    PyErr_Format(PyExc_ValueError, "%s: %s", name, what);
    throw Refused();
}

// The arguments of one call; the first tensor decides the device.
struct Args {
    PyObject* const* v;
    int device = -1;

    // NULL for None
    const at::Tensor* tensor(int i, const char* name, at::ScalarType type, int dim) {
        if (v[i] == Py_None) return nullptr;
        if (!THPVariable_Check(v[i])) refuse(name, "a tensor expected");
        const at::Tensor& t = THPVariable_Unpack(v[i]);
        if (!t.is_cuda()) refuse(name, "must live on the GPU (no CPU path exists)");
        if (device < 0) device = t.get_device();
        if (t.get_device() != device) refuse(name, "must live on the GPU of the other tensors");
        if (t.scalar_type() != type) refuse(name, (std::string("dtype ") + c10::toString(t.scalar_type()) + ", expected " + c10::toString(type)).c_str());
        if (t.dim() != dim) refuse(name, (std::to_string(t.dim()) + " axes, expected " + std::to_string(dim)).c_str());
        if (dim && t.size(-1) > 1 && t.stride(-1) != 1) refuse(name, "innermost axis must be contiguous");
        return &t;
    }
    const at::Tensor& needed(int i, const char* name, at::ScalarType type, int dim) {
        const at::Tensor* t = tensor(i, name, type, dim);
        if (!t) refuse(name, "is needed");
        return *t;
    }
    // pointer of a contiguous tensor of these sizes (-1: any)
    template <typename T>
    T* flat(int i, const char* name, at::ScalarType type, std::initializer_list<int64_t> sizes) {
        const at::Tensor* t = tensor(i, name, type, (int)sizes.size());
        if (!t) return nullptr;
        fits(*t, name, sizes);
        if (!t->is_contiguous()) refuse(name, "must be contiguous");
        return (T*)t->data_ptr();
    }
    void fits(const at::Tensor& t, const char* name, std::initializer_list<int64_t> sizes) {
        int d = 0;
        for (int64_t s : sizes) {
            if (s >= 0 && t.size(d) != s) refuse(name, ("size " + std::to_string(t.size(d)) + " of axis " + std::to_string(d) + ", expected " + std::to_string(s)).c_str());
            ++d;
        }
    }
    // heads [T, H, d] of bf16 into a pointer and its strides
    template <typename P>
    void heads(int i, const char* name, int64_t T, int64_t H, int64_t d, P& ptr, int64_t& st, int64_t& sh) {
        const at::Tensor* t = tensor(i, name, at::kBFloat16, 3);
        if (!t) return;
        fits(*t, name, {T, H, d});
        ptr = t->data_ptr();
        st = t->stride(0);
        sh = t->stride(1);
    }
    double number(int i) {
        const double x = PyFloat_AsDouble(v[i]);
        if (x == -1.0 && PyErr_Occurred()) throw Refused();
        return x;
    }
    int32_t whole(int i) {
        const long long x = PyLong_AsLongLong(v[i]);
        if (x == -1 && PyErr_Occurred()) throw Refused();
        if (x != (int32_t)x) refuse("argument", "does not fit 32 bits");
        return (int32_t)x;
    }
    void* stream() {
        void* s = PyLong_AsVoidPtr(v[0]);
        if (!s && PyErr_Occurred()) throw Refused();
        return s;
    }
    void workspace(int i, void*& ptr, size_t& bytes) {
        if (v[i] == Py_None) return;
        if (!THPVariable_Check(v[i])) refuse("workspace", "a tensor expected");
        const at::Tensor& t = THPVariable_Unpack(v[i]);
        if (!t.is_cuda() || t.get_device() != device) refuse("workspace", "must live on the GPU of the other tensors");
        if (!t.is_contiguous()) refuse("workspace", "must be contiguous");
        ptr = t.data_ptr();
        bytes = t.nbytes();
    }
};

int32_t size32(int64_t v, const char* name) {
    if (v != (int32_t)v) refuse(name, "sizes must fit 32 bits");
    return (int32_t)v;
}

// T, Hq, Hkv, d of queries at `i` and keys at `j`, either of which may be None
template <typename S>
void head_sizes(Args& a, int i, const char* q_name, int j, const char* k_name, S& s) {
    const at::Tensor *q = a.tensor(i, q_name, at::kBFloat16, 3), *k = a.tensor(j, k_name, at::kBFloat16, 3);
    if (!q && !k) refuse(q_name, "queries or keys are needed");
    const at::Tensor& t = q ? *q : *k;
    s.T = size32(t.size(0), q_name);
    s.Hq = q ? size32(q->size(1), q_name) : 0;
    s.Hkv = k ? size32(k->size(1), k_name) : 0;
    s.d = size32(t.size(2), q_name);
}
void together(Args& a, int i, int j, const char* name) {
    if ((a.v[i] == Py_None) != (a.v[j] == Py_None)) refuse(name, "goes with its input");
}

// q_weight, k_weight, eps, rope, positions, rope_style from argument `i` on
void head_map(Args& a, int i, int64_t T, int64_t d, dlm_head_map& m) {
    m.q_weight = a.flat<void>(i, "q_weight", at::kBFloat16, {d});
    m.k_weight = a.flat<void>(i + 1, "k_weight", at::kBFloat16, {d});
    m.eps = (float)a.number(i + 2);
    if (const at::Tensor* r = a.tensor(i + 3, "rope", at::kFloat, 2)) {
        m.rope = a.flat<float>(i + 3, "rope", at::kFloat, {-1, -1});
        m.rope_len = size32(r->size(0), "rope");
        m.rot_dim = size32(r->size(1), "rope");
        if (a.v[i + 4] == Py_None) refuse("rope", "a rotation needs positions");
    }
    m.positions = a.flat<int32_t>(i + 4, "positions", at::kInt, {T});
    m.rope_style = a.whole(i + 5);
}

// caches at `i` and `i + 1`, scales at `s` and `s + 1`
void paged_kv(Args& a, int i, int s, int64_t heads, int64_t d, dlm_paged_kv& c) {
    if (!THPVariable_Check(a.v[i])) refuse("cache_k", "a tensor expected");
    const bool e4m3 = THPVariable_Unpack(a.v[i]).scalar_type() == at::kFloat8_e4m3fn;
    const auto type = e4m3 ? at::kFloat8_e4m3fn : at::kBFloat16;
    const at::Tensor &k = a.needed(i, "cache_k", type, 4), &v = a.needed(i + 1, "cache_v", type, 4);
    a.fits(k, "cache_k", {-1, heads, -1, d});
    if (k.sizes() != v.sizes() || k.strides() != v.strides()) refuse("cache_v", "must have cache_k's shape and strides");
    c.k = k.data_ptr();
    c.v = v.data_ptr();
    c.n_pages = size32(k.size(0), "cache_k");
    c.page_size = size32(k.size(2), "cache_k");
    c.stride_page = k.stride(0);
    c.stride_h = k.stride(1);
    c.stride_t = k.stride(2);
    c.type = e4m3 ? DLM_KV_E4M3 : DLM_KV_BF16;
    c.k_scale = a.flat<float>(s, "k_scale", at::kFloat, {heads < 0 ? k.size(1) : heads});
    c.v_scale = a.flat<float>(s + 1, "v_scale", at::kFloat, {heads < 0 ? k.size(1) : heads});
}

// (stream, q, k, q_out, k_out, q_weight, k_weight, eps, rope, positions, rope_style)
int qk_norm_rope(Args& a) {
    dlm_qk_args s = {};
    s.struct_size = sizeof s;
    head_sizes(a, 1, "q", 2, "k", s);
    together(a, 1, 3, "q_out");
    together(a, 2, 4, "k_out");
    a.heads(1, "q", s.T, s.Hq, s.d, s.q, s.q_stride_t, s.q_stride_h);
    a.heads(2, "k", s.T, s.Hkv, s.d, s.k, s.k_stride_t, s.k_stride_h);
    a.heads(3, "q_out", s.T, s.Hq, s.d, s.q_out, s.qo_stride_t, s.qo_stride_h);
    a.heads(4, "k_out", s.T, s.Hkv, s.d, s.k_out, s.ko_stride_t, s.ko_stride_h);
    head_map(a, 5, s.T, s.d, s.map);
    return dlm_qk_norm_rope(&s, a.stream());
}

// (stream, d_q_out, d_k_out, d_q, d_k, q, k, d_q_weight, d_k_weight, q_weight, k_weight, eps, rope, positions, rope_style, workspace)
int qk_norm_rope_bwd(Args& a) {
    dlm_qk_bwd_args s = {};
    s.struct_size = sizeof s;
    head_sizes(a, 1, "d_q_out", 2, "d_k_out", s);
    together(a, 1, 3, "d_q");
    together(a, 2, 4, "d_k");
    a.heads(1, "d_q_out", s.T, s.Hq, s.d, s.d_q_out, s.dqo_stride_t, s.dqo_stride_h);
    a.heads(2, "d_k_out", s.T, s.Hkv, s.d, s.d_k_out, s.dko_stride_t, s.dko_stride_h);
    a.heads(3, "d_q", s.T, s.Hq, s.d, s.d_q, s.dq_stride_t, s.dq_stride_h);
    a.heads(4, "d_k", s.T, s.Hkv, s.d, s.d_k, s.dk_stride_t, s.dk_stride_h);
    a.heads(5, "q", s.T, s.Hq, s.d, s.q, s.q_stride_t, s.q_stride_h);
    a.heads(6, "k", s.T, s.Hkv, s.d, s.k, s.k_stride_t, s.k_stride_h);
    s.d_q_weight = a.flat<float>(7, "d_q_weight", at::kFloat, {s.d});
    s.d_k_weight = a.flat<float>(8, "d_k_weight", at::kFloat, {s.d});
    head_map(a, 9, s.T, s.d, s.map);
    a.workspace(15, s.workspace, s.workspace_bytes);
    return dlm_qk_norm_rope_bwd(&s, a.stream());
}

// (T, Hq, Hkv, d)
size_t qk_norm_rope_bwd_workspace(Args& a) {
    dlm_qk_bwd_args s = {};
    s.struct_size = sizeof s;
    s.T = a.whole(0);
    s.Hq = a.whole(1);
    s.Hkv = a.whole(2);
    s.d = a.whole(3);
    return dlm_qk_norm_rope_bwd_workspace_bytes(&s);
}

// (stream, k, v, cache_k, cache_v, slots, q, q_out, k_scale, v_scale, q_weight, k_weight, eps, rope, positions, rope_style)
int paged_append(Args& a) {
    dlm_append_args s = {};
    s.struct_size = sizeof s;
    a.needed(1, "k", at::kBFloat16, 3);
    a.needed(2, "v", at::kBFloat16, 3);
    head_sizes(a, 6, "q", 1, "k", s);
    together(a, 6, 7, "q_out");
    a.heads(6, "q", s.T, s.Hq, s.d, s.q, s.q_stride_t, s.q_stride_h);
    a.heads(1, "k", s.T, s.Hkv, s.d, s.k, s.k_stride_t, s.k_stride_h);
    a.heads(2, "v", s.T, s.Hkv, s.d, s.v, s.v_stride_t, s.v_stride_h);
    a.heads(7, "q_out", s.T, s.Hq, s.d, s.q_out, s.qo_stride_t, s.qo_stride_h);
    a.needed(5, "slots", at::kInt, 1);
    s.slots = a.flat<int32_t>(5, "slots", at::kInt, {s.T});
    paged_kv(a, 3, 8, s.Hkv, s.d, s.cache);
    head_map(a, 10, s.T, s.d, s.map);
    return dlm_paged_append(&s, a.stream());
}

// (stream, q, out, cache_k, cache_v, block_table, kv_len, max_kv_len, q_len, mask_mode, block_size, scale, lse, k_scale, v_scale, workspace)
void paged_attn_args(Args& a, dlm_paged_attn_args& s) {
    s.struct_size = sizeof s;
    const at::Tensor &q = a.needed(1, "q", at::kBFloat16, 4), &out = a.needed(2, "out", at::kBFloat16, 4);
    if (out.sizes() != q.sizes()) refuse("out", "must have q's shape");
    s.B = size32(q.size(0), "q");
    s.Lq = size32(q.size(1), "q");
    s.Hq = size32(q.size(2), "q");
    s.d = size32(q.size(3), "q");
    s.q = q.data_ptr();
    s.q_stride_b = q.stride(0);
    s.q_stride_t = q.stride(1);
    s.q_stride_h = q.stride(2);
    s.out = out.data_ptr();
    s.o_stride_b = out.stride(0);
    s.o_stride_t = out.stride(1);
    s.o_stride_h = out.stride(2);
    paged_kv(a, 3, 13, -1, s.d, s.cache);
    s.Hkv = size32(THPVariable_Unpack(a.v[3]).size(1), "cache_k");
    const at::Tensor& table = a.needed(5, "block_table", at::kInt, 2);
    a.fits(table, "block_table", {s.B, -1});
    s.block_table = (const int32_t*)table.data_ptr();
    s.table_stride = s.B > 1 ? table.stride(0) : table.size(1);
    a.needed(6, "kv_len", at::kInt, 1);
    s.kv_len = a.flat<int32_t>(6, "kv_len", at::kInt, {s.B});
    const int64_t holds = std::min<int64_t>(table.size(1) * s.cache.page_size, 1 << 30);       // tokens of a row of the table
    s.max_kv_len = a.v[7] == Py_None ? (int32_t)holds : a.whole(7);
    if (s.max_kv_len > holds) refuse("max_kv_len", ("exceeds the " + std::to_string(holds) + " tokens of a row of block_table").c_str());
    s.q_len = a.flat<int32_t>(8, "q_len", at::kInt, {s.B});
    s.mask_mode = a.whole(9);
    s.block_size = a.whole(10);
    s.scale = (float)a.number(11);
    s.lse = a.flat<float>(12, "lse", at::kFloat, {s.B, s.Hq, s.Lq});
    a.workspace(15, s.workspace, s.workspace_bytes);
}
int paged_attn(Args& a) {
    dlm_paged_attn_args s = {};
    paged_attn_args(a, s);
    return dlm_paged_attn(&s, a.stream());
}
size_t paged_attn_workspace(Args& a) {
    dlm_paged_attn_args s = {};
    paged_attn_args(a, s);
    return dlm_paged_attn_workspace_bytes(&s);
}

template <auto F, int N>
PyObject* entry(PyObject*, PyObject* const* v, Py_ssize_t n) {
    if (n != N) return PyErr_Format(PyExc_TypeError, "%d arguments expected", N);
    try {
        Args a{v};
        return PyLong_FromLongLong((long long)F(a));
    } catch (const Refused&) {
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

PyMethodDef methods[] = {
    {"qk_norm_rope", (PyCFunction)(void*)entry<qk_norm_rope, 11>, METH_FASTCALL, nullptr},
    {"qk_norm_rope_bwd", (PyCFunction)(void*)entry<qk_norm_rope_bwd, 16>, METH_FASTCALL, nullptr},
    {"qk_norm_rope_bwd_workspace", (PyCFunction)(void*)entry<qk_norm_rope_bwd_workspace, 4>, METH_FASTCALL, nullptr},
    {"paged_append", (PyCFunction)(void*)entry<paged_append, 16>, METH_FASTCALL, nullptr},
    {"paged_attn", (PyCFunction)(void*)entry<paged_attn, 16>, METH_FASTCALL, nullptr},
    {"paged_attn_workspace", (PyCFunction)(void*)entry<paged_attn_workspace, 16>, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&module); }
