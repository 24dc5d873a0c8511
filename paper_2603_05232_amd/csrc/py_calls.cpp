// The calls of a model's forward pass (quantisation, sparse GEMMs, the 4-bit expert layer) as CPython functions: argument reading, output
// allocation and the C call without going through ctypes and torch's Python layer.  Layers of few tokens are bound by the time
// between launches, most of which was spent there (quantisation + GEMM of 16 x 512 x 512: see binding.py).
//
// Each function does plain calls only: exact torch.Tensor arguments on the GPU, exact ints, no active function or dispatch
// mode, and arguments that the C entry point accepts.  For anything else it returns None and the caller's general path does the
// call over, which is where arguments are refused and errors raised: the C entry points check their arguments before they launch
// anything.  A launch that failed is no argument to refuse: SS_ERR_HIP raises here, since a second attempt would launch
// again and find the runtime's error cleared.
//
// The module is not linked against libslidesparse.so: the binding hands it the addresses of the library that it has loaded by path.
// By name, the loader would give a second copy of the package in the process the first copy's library.
#include <Python.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <limits.h>
#include <string.h>
#include "slidesparse.h"

namespace {

struct Library {
    decltype(&::slide_lifted_ld) lifted_ld;
    decltype(&::act_lift_quant) lift_quant;
    decltype(&::slide_sparse_gemm_ws) sparse_gemm;
    decltype(&::slide_sparse_gemm_fused_ws) sparse_gemm_fused;
} lib;                                                // zeros until bind()
PyObject* error_type = nullptr;                       // SlideSparseError(status, where)

// the interpreter lock is given up while memory is allocated and kernels are launched (either may wait for the GPU)
struct Unlocked {
    PyThreadState* state = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(state); }
};

bool plain(PyObject* o)
{
    if (!THPVariable_CheckExact(o)) return false;
    constexpr c10::DispatchKeySet wrapped({c10::DispatchKey::Python, c10::DispatchKey::PythonTLSSnapshot, c10::DispatchKey::FuncTorchBatched,
                                           c10::DispatchKey::FuncTorchGradWrapper, c10::DispatchKey::Functionalize, c10::DispatchKey::Sparse,
                                           c10::DispatchKey::SparseCsr});
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.defined() && t.has_storage() && !t.key_set().has_any(wrapped);
}
bool plain_or_none(PyObject* o) { return o == Py_None || plain(o); }
void* address(PyObject* o) { return o == Py_None ? nullptr : THPVariable_Unpack(o).data_ptr(); }

bool integer(PyObject* o, int64_t lo, int64_t hi, int64_t& v)
{
    if (!PyLong_CheckExact(o)) return false;
    int over = 0;
    const long long x = PyLong_AsLongLongAndOverflow(o, &over);
    if (over || x < lo || x > hi) return false;
    v = x;
    return true;
}

struct Type { ss_dtype code; at::ScalarType storage; bool scaled; };
bool operand_type(PyObject* o, Type& t)
{
    if (!PyUnicode_CheckExact(o)) return false;
    if (PyUnicode_CompareWithASCIIString(o, "i8") == 0) t = {SS_I8, at::kChar, true};
    else if (PyUnicode_CompareWithASCIIString(o, "fp8") == 0) t = {SS_FP8_E4M3, at::kByte, true};
    else if (PyUnicode_CompareWithASCIIString(o, "bf16") == 0) t = {SS_BF16, at::kBFloat16, false};
    else if (PyUnicode_CompareWithASCIIString(o, "fp16") == 0) t = {SS_FP16, at::kHalf, false};
    else return false;
    return true;
}

bool modes_active() { return c10::impl::TorchDispatchModeTLS::any_modes_set() || at::impl::torch_function_mode_enabled(); }
void* current_stream() { return c10::hip::getCurrentHIPStream().stream(); }

// what a function returns for a status other than SS_OK
PyObject* refused(ss_status st, const char* where)
{
    if (st != SS_ERR_HIP) Py_RETURN_NONE;
    if (PyObject* e = PyObject_CallFunction(error_type, "is", (int)st, where)) {
        PyErr_SetObject(error_type, e);
        Py_DECREF(e);
    }
    return nullptr;
}

// act_lift_quant(X, N, dtype, out, s_x)
PyObject* py_act_lift_quant(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    int64_t N;
    Type t;
    if (!lib.lift_quant || n != 5 || !plain(a[0]) || !integer(a[1], INT_MIN, INT_MAX, N) || !operand_type(a[2], t) || !plain_or_none(a[3]) || !plain_or_none(a[4]) || modes_active()) Py_RETURN_NONE;
    const at::Tensor& X = THPVariable_Unpack(a[0]);
    if (!X.is_cuda() || X.dim() != 2 || X.stride(1) != 1 || (X.scalar_type() != at::kFloat && X.scalar_type() != at::kBFloat16)) Py_RETURN_NONE;
    const int64_t M = X.size(0), K = X.size(1), width = lib.lifted_ld(K, (int)N, t.code);
    if (width < 0) Py_RETURN_NONE;
    at::Tensor out, s_x;
    void *out_ptr = address(a[3]), *s_x_ptr = address(a[4]);
    ss_status st;
    {
        Unlocked u;
        if (a[3] == Py_None) { out = at::empty({M, width}, X.options().dtype(t.storage)); out_ptr = out.data_ptr(); }
        if (a[4] == Py_None && t.scaled) { s_x = at::empty({M}, X.options().dtype(at::kFloat)); s_x_ptr = s_x.data_ptr(); }
        st = lib.lift_quant(X.data_ptr(), X.scalar_type() == at::kFloat ? SS_IN_F32 : SS_IN_BF16, M, K, M > 1 ? X.stride(0) : K, (int)N, t.code, out_ptr,
                            static_cast<float*>(s_x_ptr), current_stream());
    }
    if (st != SS_OK) return refused(st, "act_lift_quant");
    PyObject* po = out.defined() ? THPVariable_Wrap(std::move(out)) : Py_NewRef(a[3]);
    PyObject* ps = s_x.defined() ? THPVariable_Wrap(std::move(s_x)) : Py_NewRef(a[4]);
    PyObject* r = po && ps ? PyTuple_Pack(2, po, ps) : nullptr;
    Py_XDECREF(po);
    Py_XDECREF(ps);
    return r;
    END_HANDLE_TH_ERRORS
}

// The operands common to both GEMMs: a = X, s_x, w_vals, w_meta, s_w; `out` and `workspace` may be None
struct Out { at::Tensor made; void* ptr; int64_t ld; };
bool gemm_operands(PyObject* const* a, PyObject* out, PyObject* workspace)
{
    return plain(a[0]) && plain_or_none(a[1]) && plain_or_none(a[2]) && plain_or_none(a[3]) && plain_or_none(a[4]) && plain_or_none(out) &&
           (out == Py_None || THPVariable_Unpack(out).dim() == 2) && plain_or_none(workspace) && !modes_active();
}
Out output(PyObject* out, const at::Tensor& X, int64_t M, int64_t O)
{
    if (out != Py_None) return {at::Tensor(), THPVariable_Unpack(out).data_ptr(), THPVariable_Unpack(out).stride(0)};
    Out r{at::empty({M, O}, X.options().dtype(at::kBFloat16)), nullptr, 0};
    r.ptr = r.made.data_ptr();
    r.ld = r.made.stride(0);
    return r;
}
PyObject* result(Out& r, PyObject* out) { return r.made.defined() ? THPVariable_Wrap(std::move(r.made)) : Py_NewRef(out); }

// slide_sparse_gemm(X_lifted, s_x, w_vals, w_meta, s_w, O, dtype, out, workspace)
PyObject* py_slide_sparse_gemm(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    int64_t O;
    Type t;
    if (!lib.sparse_gemm || n != 9 || !gemm_operands(a, a[7], a[8]) || !integer(a[5], 0, INT64_MAX, O) || !operand_type(a[6], t)) Py_RETURN_NONE;
    const at::Tensor& X = THPVariable_Unpack(a[0]);
    if (!X.is_cuda() || X.dim() != 2 || !X.is_contiguous()) Py_RETURN_NONE;
    void* const ws = address(a[8]);
    const size_t ws_bytes = a[8] == Py_None ? 0 : THPVariable_Unpack(a[8]).nbytes();
    const void *s_x = address(a[1]), *wv = address(a[2]), *wm = address(a[3]), *s_w = address(a[4]);
    Out y;
    ss_status st;
    {
        Unlocked u;
        y = output(a[7], X, X.size(0), O);
        st = lib.sparse_gemm(X.data_ptr(), static_cast<const float*>(s_x), wv, wm, static_cast<const float*>(s_w), X.size(0), O, X.size(1), t.code, y.ptr, y.ld, ws, ws_bytes,
                                  current_stream());
    }
    if (st != SS_OK) return refused(st, a[8] == Py_None ? "slide_sparse_gemm" : "slide_sparse_gemm_ws");
    return result(y, a[7]);
    END_HANDLE_TH_ERRORS
}

// slide_sparse_gemm_fused(Xq, s_x, w_vals, w_meta, s_w, O, K, N, dtype, out, workspace)
PyObject* py_slide_sparse_gemm_fused(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    int64_t O, K, N;
    Type t;
    if (!lib.sparse_gemm_fused || n != 11 || !gemm_operands(a, a[9], a[10]) || !integer(a[5], 0, INT64_MAX, O) || !integer(a[6], 0, INT64_MAX, K) || !integer(a[7], INT_MIN, INT_MAX, N) ||
        !operand_type(a[8], t))
        Py_RETURN_NONE;
    const at::Tensor& X = THPVariable_Unpack(a[0]);
    if (!X.is_cuda() || X.dim() != 2 || X.stride(1) != 1 || X.size(1) < K) Py_RETURN_NONE;
    const int64_t M = X.size(0);
    void* const ws = address(a[10]);
    const size_t ws_bytes = a[10] == Py_None ? 0 : (size_t)THPVariable_Unpack(a[10]).numel();
    const void *s_x = address(a[1]), *wv = address(a[2]), *wm = address(a[3]), *s_w = address(a[4]);
    Out y;
    ss_status st;
    {
        Unlocked u;
        y = output(a[9], X, M, O);
        st = lib.sparse_gemm_fused(X.data_ptr(), static_cast<const float*>(s_x), wv, wm, static_cast<const float*>(s_w), M, O, K, M > 1 ? X.stride(0) : X.size(1), (int)N,
                                        t.code, y.ptr, y.ld, ws, ws_bytes, current_stream());
    }
    if (st != SS_OK) return refused(st, a[10] == Py_None ? "slide_sparse_gemm_fused" : "slide_sparse_gemm_fused_ws");
    return result(y, a[9]);
    END_HANDLE_TH_ERRORS
}

// ---- microscaled 4-bit operands and layers of experts ----
struct Mx4 {
    decltype(&::mx4_row_bytes) row_bytes;
    decltype(&::mx4_quant) quant;
    decltype(&::mx4_dequant) dequant;
    decltype(&::mx4_packed_sizes) packed_sizes;
    decltype(&::mx4_gemm) gemm;
    decltype(&::mx4_grouped_gemm) grouped_gemm;
    decltype(&::expert_route_workspace_bytes) route_workspace;
    decltype(&::expert_route) route;
    decltype(&::expert_combine) combine;
} mx4;                                                // zeros until bind_mx4()

bool float_or_bf16(const at::Tensor& t) { return t.scalar_type() == at::kFloat || t.scalar_type() == at::kBFloat16; }
ss_act_dtype in_code(const at::Tensor& t) { return t.scalar_type() == at::kFloat ? SS_IN_F32 : SS_IN_BF16; }
// on the GPU of the operator's first tensor: kernels read and write through every address that they are given
bool beside(const at::Tensor& t, const at::Tensor& first) { return first.is_cuda() && t.device() == first.device(); }
// a matrix whose rows are dense, and the elements between its rows
bool matrix(const at::Tensor& t, const at::Tensor& first) { return beside(t, first) && t.dim() == 2 && (t.size(1) < 2 || t.stride(1) == 1); }
int64_t row_stride(const at::Tensor& t) { return t.size(0) > 1 ? t.stride(0) : t.size(1); }
bool dense(const at::Tensor& t, at::ScalarType type, const at::Tensor& first) { return beside(t, first) && t.scalar_type() == type && t.is_contiguous(); }
bool workspace(PyObject* o, const at::Tensor& first) { return o == Py_None || (beside(THPVariable_Unpack(o), first) && THPVariable_Unpack(o).is_contiguous()); }
// codes[R, 128 U] and scales[U, R, 8] of rows of K values
bool code_rows(const at::Tensor& codes, const at::Tensor& scales, int64_t K, const at::Tensor& first)
{
    const int64_t width = mx4.row_bytes(K);
    return width > 0 && dense(codes, at::kByte, first) && dense(scales, at::kByte, first) && codes.dim() == 2 && scales.dim() == 3 && codes.size(1) == width &&
           scales.size(0) == width / 128 && scales.size(1) == codes.size(0) && scales.size(2) == 8;
}
PyObject* wrap(at::Tensor& made, PyObject* given) { return made.defined() ? THPVariable_Wrap(std::move(made)) : Py_NewRef(given); }

// A tensor on elements `at` and following of `all`, of a type as wide as its own.  Several results share one allocation, which is 0.9 us on the host; this is 0.3.
at::Tensor part(const at::Tensor& all, int64_t at, c10::IntArrayRef sizes, at::ScalarType type)
{
    at::Tensor v = at::detail::make_tensor<at::TensorImpl>(at::Storage(all.storage()), all.key_set(), c10::scalarTypeToTypeMeta(type));
    v.unsafeGetTensorImpl()->set_storage_offset(at);
    v.unsafeGetTensorImpl()->set_sizes_contiguous(sizes);
    return v;
}

// mx4_quant(X, rows, codes, scales)
PyObject* py_mx4_quant(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (!mx4.quant || n != 4 || !plain(a[0]) || !plain_or_none(a[1]) || !plain_or_none(a[2]) || !plain_or_none(a[3]) || modes_active()) Py_RETURN_NONE;
    const at::Tensor& X = THPVariable_Unpack(a[0]);
    if (!matrix(X, X) || !float_or_bf16(X)) Py_RETURN_NONE;
    const int64_t M = X.size(0), K = X.size(1), width = mx4.row_bytes(K);
    if (width < 0 || (a[1] != Py_None && (THPVariable_Unpack(a[1]).dim() != 1 || !dense(THPVariable_Unpack(a[1]), at::kInt, X)))) Py_RETURN_NONE;
    const int64_t R = a[1] == Py_None ? M : THPVariable_Unpack(a[1]).size(0);
    at::Tensor codes, scales;
    ss_status st;
    {
        Unlocked u;
        const auto bytes = X.options().dtype(at::kByte);
        if (a[2] == Py_None && a[3] == Py_None) {
            const at::Tensor both = at::empty({R * (width + width / 16)}, bytes);
            codes = part(both, 0, {R, width}, at::kByte);
            scales = part(both, R * width, {width / 128, R, 8}, at::kByte);
        } else if (a[2] == Py_None) codes = at::empty({R, width}, bytes);
        else if (a[3] == Py_None) scales = at::empty({width / 128, R, 8}, bytes);
        const at::Tensor &c = codes.defined() ? codes : THPVariable_Unpack(a[2]), &s = scales.defined() ? scales : THPVariable_Unpack(a[3]);
        st = code_rows(c, s, K, X) && c.size(0) == R
                 ? mx4.quant(X.data_ptr(), in_code(X), M, K, row_stride(X), static_cast<const int32_t*>(address(a[1])), R, c.data_ptr(), s.data_ptr(), current_stream())
                 : SS_ERR_SHAPE;
    }
    if (st != SS_OK) return refused(st, "mx4_quant");
    PyObject *pc = wrap(codes, a[2]), *ps = wrap(scales, a[3]);
    PyObject* r = pc && ps ? PyTuple_Pack(2, pc, ps) : nullptr;
    Py_XDECREF(pc);
    Py_XDECREF(ps);
    return r;
    END_HANDLE_TH_ERRORS
}

// mx4_dequant(codes, scales, K, fp32 or bf16 as ss_act_dtype, out)
PyObject* py_mx4_dequant(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    int64_t K, type;
    if (!mx4.dequant || n != 5 || !plain(a[0]) || !plain(a[1]) || !integer(a[2], 1, INT64_MAX, K) || !integer(a[3], 0, 1, type) || !plain_or_none(a[4]) || modes_active()) Py_RETURN_NONE;
    const at::Tensor &codes = THPVariable_Unpack(a[0]), &scales = THPVariable_Unpack(a[1]);
    if (!code_rows(codes, scales, K, codes)) Py_RETURN_NONE;
    at::Tensor made;
    ss_status st;
    {
        Unlocked u;
        if (a[4] == Py_None) made = at::empty({codes.size(0), K}, codes.options().dtype(type == SS_IN_F32 ? at::kFloat : at::kBFloat16));
        const at::Tensor& y = made.defined() ? made : THPVariable_Unpack(a[4]);
        st = matrix(y, codes) && float_or_bf16(y) && y.size(0) == codes.size(0) && y.size(1) == K
                 ? mx4.dequant(codes.data_ptr(), scales.data_ptr(), codes.size(0), K, in_code(y), y.data_ptr(), row_stride(y), current_stream())
                 : SS_ERR_SHAPE;
    }
    if (st != SS_OK) return refused(st, "mx4_dequant");
    return wrap(made, a[4]);
    END_HANDLE_TH_ERRORS
}

// mx4_product(offsets or None, codes, scales, w_vals, w_meta, O, K, gated, out, workspace)
PyObject* py_mx4_product(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    int64_t O, K;
    if (!mx4.gemm || n != 10 || !plain_or_none(a[0]) || !plain(a[1]) || !plain(a[2]) || !plain(a[3]) || !plain(a[4]) || !integer(a[5], 0, INT_MAX, O) || !integer(a[6], 1, INT64_MAX, K) ||
        !PyBool_Check(a[7]) || !plain_or_none(a[8]) || !plain_or_none(a[9]) || modes_active())
        Py_RETURN_NONE;
    const bool grouped = a[0] != Py_None;
    const int gated = a[7] == Py_True;
    const at::Tensor &codes = THPVariable_Unpack(a[1]), &scales = THPVariable_Unpack(a[2]), &wv = THPVariable_Unpack(a[3]), &wm = THPVariable_Unpack(a[4]);
    if (!code_rows(codes, scales, K, codes) || (grouped && (THPVariable_Unpack(a[0]).dim() != 1 || !dense(THPVariable_Unpack(a[0]), at::kInt, codes))) || !workspace(a[9], codes)) Py_RETURN_NONE;
    const int64_t R = codes.size(0), E = grouped ? THPVariable_Unpack(a[0]).size(0) - 1 : 1;
    size_t vb, mb;
    if (mx4.packed_sizes(E, O, K, gated, &vb, &mb) != SS_OK || !dense(wv, at::kByte, codes) || !dense(wm, at::kByte, codes) || (size_t)wv.numel() != vb || (size_t)wm.numel() != mb) Py_RETURN_NONE;
    void* const ws = address(a[9]);
    const size_t ws_bytes = a[9] == Py_None ? 0 : THPVariable_Unpack(a[9]).nbytes();
    at::Tensor made;
    ss_status st;
    {
        Unlocked u;
        if (a[8] == Py_None) made = at::empty({R, O}, codes.options().dtype(at::kBFloat16));
        const at::Tensor& y = made.defined() ? made : THPVariable_Unpack(a[8]);
        if (!matrix(y, codes) || y.scalar_type() != at::kBFloat16 || y.size(0) != R || y.size(1) != O) st = SS_ERR_SHAPE;
        else if (grouped)
            st = mx4.grouped_gemm(codes.data_ptr(), scales.data_ptr(), static_cast<const int32_t*>(address(a[0])), wv.data_ptr(), wm.data_ptr(), R, E, O, K, gated, y.data_ptr(),
                                  row_stride(y), ws, ws_bytes, current_stream());
        else st = mx4.gemm(codes.data_ptr(), scales.data_ptr(), wv.data_ptr(), wm.data_ptr(), R, O, K, gated, y.data_ptr(), row_stride(y), ws, ws_bytes, current_stream());
    }
    if (st != SS_OK) return refused(st, grouped ? "mx4_grouped_gemm" : "mx4_gemm");
    return wrap(made, a[8]);
    END_HANDLE_TH_ERRORS
}

// expert_route(logits, k, renormalise, workspace)
PyObject* py_expert_route(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    int64_t k;
    if (!mx4.route || n != 4 || !plain(a[0]) || !integer(a[1], 1, 64, k) || !PyBool_Check(a[2]) || !plain_or_none(a[3]) || modes_active()) Py_RETURN_NONE;
    const at::Tensor& x = THPVariable_Unpack(a[0]);
    if (!matrix(x, x) || !float_or_bf16(x) || k > x.size(1) || !workspace(a[3], x)) Py_RETURN_NONE;
    const int64_t M = x.size(0), E = x.size(1);
    at::Tensor ids, weights, slots, rows, offsets, scratch;
    ss_status st;
    {
        Unlocked u;
        // one allocation for all five, each from a 16-byte line on
        const int64_t n = (M * k + 3) & ~(int64_t)3;
        const at::Tensor all = at::empty({4 * n + E + 1}, x.options().dtype(at::kInt));
        ids = part(all, 0, {M, k}, at::kInt);
        slots = part(all, n, {M, k}, at::kInt);
        rows = part(all, 2 * n, {M * k}, at::kInt);
        weights = part(all, 3 * n, {M, k}, at::kFloat);
        offsets = part(all, 4 * n, {E + 1}, at::kInt);
        void* ws = address(a[3]);
        size_t ws_bytes = a[3] == Py_None ? 0 : THPVariable_Unpack(a[3]).nbytes();
        if (a[3] == Py_None && (ws_bytes = mx4.route_workspace(M, E, k)) > 0) { scratch = at::empty({(int64_t)ws_bytes}, x.options().dtype(at::kByte)); ws = scratch.data_ptr(); }
        st = mx4.route(x.data_ptr(), in_code(x), M, E, row_stride(x), (int)k, a[2] == Py_True, static_cast<int32_t*>(ids.data_ptr()), static_cast<float*>(weights.data_ptr()),
                       static_cast<int32_t*>(slots.data_ptr()), static_cast<int32_t*>(rows.data_ptr()), static_cast<int32_t*>(offsets.data_ptr()), ws, ws_bytes, current_stream());
    }
    if (st != SS_OK) return refused(st, "expert_route");
    PyObject* r = PyTuple_New(5);
    at::Tensor* const all[5] = {&ids, &weights, &slots, &rows, &offsets};
    for (int i = 0; r && i < 5; ++i) {
        PyObject* const o = THPVariable_Wrap(std::move(*all[i]));
        if (o) PyTuple_SET_ITEM(r, i, o);
        else Py_CLEAR(r);
    }
    return r;
    END_HANDLE_TH_ERRORS
}

// expert_combine(Y, slots, weights, base, out)
PyObject* py_expert_combine(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (!mx4.combine || n != 5 || !plain(a[0]) || !plain(a[1]) || !plain(a[2]) || !plain_or_none(a[3]) || !plain_or_none(a[4]) || modes_active()) Py_RETURN_NONE;
    const at::Tensor &Y = THPVariable_Unpack(a[0]), &slots = THPVariable_Unpack(a[1]), &weights = THPVariable_Unpack(a[2]);
    if (!matrix(Y, Y) || Y.scalar_type() != at::kBFloat16 || slots.dim() != 2 || !dense(slots, at::kInt, Y) || !dense(weights, at::kFloat, Y) || weights.sizes() != slots.sizes()) Py_RETURN_NONE;
    const int64_t M = slots.size(0), k = slots.size(1), O = Y.size(1);
    if (k > INT_MAX) Py_RETURN_NONE;
    auto fits = [&](const at::Tensor& t) { return matrix(t, Y) && t.scalar_type() == at::kBFloat16 && t.size(0) == M && t.size(1) == O; };
    if (a[3] != Py_None && !fits(THPVariable_Unpack(a[3]))) Py_RETURN_NONE;
    at::Tensor made;
    ss_status st;
    {
        Unlocked u;
        if (a[4] == Py_None) made = at::empty({M, O}, Y.options());
        const at::Tensor& y = made.defined() ? made : THPVariable_Unpack(a[4]);
        st = fits(y) ? mx4.combine(Y.data_ptr(), Y.size(0), O, row_stride(Y), static_cast<const int32_t*>(slots.data_ptr()), static_cast<const float*>(weights.data_ptr()), M, (int)k, address(a[3]),
                                   a[3] == Py_None ? 0 : row_stride(THPVariable_Unpack(a[3])), y.data_ptr(), row_stride(y), current_stream())
                     : SS_ERR_SHAPE;
    }
    if (st != SS_OK) return refused(st, "expert_combine");
    return wrap(made, a[4]);
    END_HANDLE_TH_ERRORS
}

// bind_mx4(the addresses of Mx4's functions in their order), behind bind()
PyObject* py_bind_mx4(PyObject*, PyObject* args)
{
    unsigned long long f[9];
    if (!PyArg_ParseTuple(args, "KKKKKKKKK", &f[0], &f[1], &f[2], &f[3], &f[4], &f[5], &f[6], &f[7], &f[8])) return nullptr;
    mx4 = {reinterpret_cast<decltype(mx4.row_bytes)>(f[0]), reinterpret_cast<decltype(mx4.quant)>(f[1]), reinterpret_cast<decltype(mx4.dequant)>(f[2]),
           reinterpret_cast<decltype(mx4.packed_sizes)>(f[3]), reinterpret_cast<decltype(mx4.gemm)>(f[4]), reinterpret_cast<decltype(mx4.grouped_gemm)>(f[5]),
           reinterpret_cast<decltype(mx4.route_workspace)>(f[6]), reinterpret_cast<decltype(mx4.route)>(f[7]), reinterpret_cast<decltype(mx4.combine)>(f[8])};
    Py_RETURN_NONE;
}

// bind(SlideSparseError, slide_lifted_ld, act_lift_quant, slide_sparse_gemm_ws, slide_sparse_gemm_fused_ws), the last four as
// addresses; library() tells these
PyObject* py_bind(PyObject*, PyObject* args)
{
    PyObject* error;
    unsigned long long f[4];
    if (!PyArg_ParseTuple(args, "OKKKK", &error, &f[0], &f[1], &f[2], &f[3])) return nullptr;
    lib = {reinterpret_cast<decltype(lib.lifted_ld)>(f[0]), reinterpret_cast<decltype(lib.lift_quant)>(f[1]), reinterpret_cast<decltype(lib.sparse_gemm)>(f[2]),
           reinterpret_cast<decltype(lib.sparse_gemm_fused)>(f[3])};
    Py_INCREF(error);
    Py_XDECREF(error_type);
    error_type = error;
    Py_RETURN_NONE;
}
PyObject* py_library(PyObject*, PyObject*)
{
    return Py_BuildValue("KKKK", reinterpret_cast<unsigned long long>(lib.lifted_ld), reinterpret_cast<unsigned long long>(lib.lift_quant),
                         reinterpret_cast<unsigned long long>(lib.sparse_gemm), reinterpret_cast<unsigned long long>(lib.sparse_gemm_fused));
}

#define SS_PY(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(f)), METH_FASTCALL
PyMethodDef methods[] = {{"act_lift_quant", SS_PY(py_act_lift_quant), nullptr},
                         {"slide_sparse_gemm", SS_PY(py_slide_sparse_gemm), nullptr},
                         {"slide_sparse_gemm_fused", SS_PY(py_slide_sparse_gemm_fused), nullptr},
                         {"mx4_quant", SS_PY(py_mx4_quant), nullptr},
                         {"mx4_dequant", SS_PY(py_mx4_dequant), nullptr},
                         {"mx4_product", SS_PY(py_mx4_product), nullptr},
                         {"expert_route", SS_PY(py_expert_route), nullptr},
                         {"expert_combine", SS_PY(py_expert_combine), nullptr},
                         {"bind_mx4", py_bind_mx4, METH_VARARGS, nullptr},
                         {"bind", py_bind, METH_VARARGS, nullptr},
                         {"library", py_library, METH_NOARGS, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls(void)
{
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "torch_version", SS_TORCH_VERSION) < 0) Py_CLEAR(m);      // torch's C++ interface is another one in each version
    return m;
}
