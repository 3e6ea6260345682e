// Native marshalling of the Python binding's calls: tensors in, the C entry point called with their addresses, sizes and the
// current stream.  A call stands in front of kernels of a few microseconds; marshalled in Python through ctypes it cost about
// 6 us of host time, more than the kernel of a decode step takes.
//
// Every function takes plain strided CUDA tensors in the shapes that the entry point wants, outputs included, and returns the
// entry point's status.  Anything else - a subclass, a wrapper of a transform, a missing output, a wrong type or shape -
// returns None and nothing has happened: the binding's Python code then does the call or raises.
#include <Python.h>

#include <string.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include "mx4.h"

namespace {

struct Calls {  // the C entry points, by the addresses that the binding passes in
    decltype(&mx_quantize) quantize;
    decltype(&mx_quantize_mbs) quantize_mbs;
    decltype(&mx_quantize_mbs_pair) quantize_mbs_pair;
    decltype(&mx_quantize_mbs_dynamic) quantize_mbs_dynamic;
    decltype(&mx_quantize_elem) quantize_elem;
    decltype(&mx_dequantize) dequantize;
    decltype(&mx_gemm) gemm;
    decltype(&mx_gemm_mbs) gemm_mbs;
    decltype(&mx_gemm_mbs_grouped) gemm_mbs_grouped;
    decltype(&mx_gemm_mbs_quantize_a) gemm_mbs_quantize_a;
    decltype(&mx_gemm_mbs_elem) gemm_mbs_elem;
    decltype(&mx_gemm_mbs_elem_grouped) gemm_mbs_elem_grouped;
    decltype(&mx_kv_plan) kv_plan;
    decltype(&mx_qk_norm_rope) qk_norm_rope;
    decltype(&mx_kv_write) kv_write;
    decltype(&mx_qk_norm_rope_kv_write) qk_norm_rope_kv_write;
    decltype(&mx_kv_read) kv_read;
    decltype(&mx_attention_kv) attention_kv;
    decltype(&mx_attention_kv_workspace) attention_kv_workspace;
} calls;

struct Declined {};  // the arguments are not what is served here

void need(bool ok) {
    if (!ok) throw Declined();
}

// (the types of the arguments have been looked at: `served`)
const at::Tensor& tensor(PyObject* o) {
    const at::Tensor& t = THPVariable_Unpack(o);
    using K = c10::DispatchKey;
    need(t.defined() && t.is_cuda() && t.layout() == c10::kStrided && t.has_storage() && !t.unsafeGetTensorImpl()->is_python_dispatch() &&
         !t.key_set().has_any(c10::DispatchKeySet({K::Python, K::FuncTorchBatched, K::FuncTorchGradWrapper, K::Functionalize, K::BatchedNestedTensor})));
    return t;
}

template <typename T = uint8_t>
T* address(const at::Tensor& t) {
    return static_cast<T*>(t.data_ptr());
}
// the address of an optional operand array (its shape is not looked at)
const uint8_t* optional(PyObject* o) { return o == Py_None ? nullptr : address(tensor(o)); }

struct Rows {  // a bf16 matrix
    const void* data;
    int64_t rows, K, ld;
};
Rows bf16_rows(PyObject* o) {
    const at::Tensor& t = tensor(o);
    need(t.scalar_type() == at::kBFloat16 && t.dim() == 2);
    const int64_t rows = t.size(0), K = t.size(1), ld = t.stride(0);
    need(t.stride(1) == 1 || K <= 1);
    return {address<const void>(t), rows, K, rows > 1 ? ld : std::max(ld, K)};
}

const at::Tensor& matrix(PyObject* o) {
    const at::Tensor& t = tensor(o);
    need(t.dim() == 2);
    return t;
}
uint8_t* bytes(PyObject* o, int64_t rows, int64_t cols) {  // an output array of codes, scales or words
    const at::Tensor& t = matrix(o);
    need(t.scalar_type() == at::kByte && t.size(0) == rows && t.size(1) == cols && t.is_contiguous());
    return address(t);
}

mx_dtype_t out_type(PyObject* o) {
    if (PyUnicode_CheckExact(o)) {
        if (PyUnicode_CompareWithASCIIString(o, "bf16") == 0) return MX_OUT_BF16;
        need(PyUnicode_CompareWithASCIIString(o, "f32") == 0 || PyUnicode_CompareWithASCIIString(o, "fp32") == 0);
        return MX_OUT_F32;
    }
    const at::ScalarType s = reinterpret_cast<THPDtype*>(o)->scalar_type;
    need(s == at::kFloat || s == at::kBFloat16);
    return s == at::kFloat ? MX_OUT_F32 : MX_OUT_BF16;
}
struct Out {  // an output matrix
    mx_dtype_t type;
    void* data;
    int64_t ld;
};
Out out_matrix(PyObject* type, PyObject* o, int64_t rows, int64_t cols) {
    const mx_dtype_t code = out_type(type);
    const at::Tensor& t = matrix(o);
    need(t.scalar_type() == (code == MX_OUT_F32 ? at::kFloat : at::kBFloat16) && t.size(0) == rows && t.size(1) == cols);
    need(t.stride(1) == 1 || cols <= 1);
    return {code, address<void>(t), rows > 1 ? t.stride(0) : std::max(t.stride(0), cols)};
}

int64_t integer(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        throw Declined();
    }
    return v;
}
template <int N>
int name_of(PyObject* o, const char* const (&names)[N]) {
    for (int i = 0; i < N; ++i)
        if (PyUnicode_CompareWithASCIIString(o, names[i]) == 0) return i;
    throw Declined();
}
mx_rule_t rule(PyObject* o) {
    static const char* const kNames[] = {"ocp", "floor", "oas"};  // MX_RULE_OCP, MX_RULE_FLOOR, MX_RULE_OAS
    return (mx_rule_t)name_of(o, kNames);
}
mx_elem_t elem(PyObject* o) {
    static const char* const kNames[] = {"e2m1", "e4m3", "e5m2", "e2m3", "e3m2"};
    return (mx_elem_t)name_of(o, kNames);
}
int64_t code_bytes(mx_elem_t e, int64_t K) { return e == MX_ELEM_E2M3 || e == MX_ELEM_E3M2 ? K * 3 / 4 : K; }
bool flag(PyObject* o) { return o == Py_True; }

void* stream() { return c10::hip::getCurrentHIPStream().stream(); }

// Whether the arguments have the types that are served: t = tensor, o = tensor or None, s = text, d = text or torch dtype, i = int,
// b = bool, f = float.  Looked at before anything that throws: an exception costs 2 us, a third of the call that the binding's Python code then makes.
bool served(PyObject* const* a, Py_ssize_t n, const char* kinds) {
    for (Py_ssize_t i = 0; i < n; ++i) {
        bool ok = false;
        switch (kinds[i]) {
            case 'o': ok = a[i] == Py_None || THPVariable_CheckExact(a[i]); break;
            case 't': ok = THPVariable_CheckExact(a[i]); break;
            case 's': ok = PyUnicode_CheckExact(a[i]); break;
            case 'd': ok = PyUnicode_CheckExact(a[i]) || THPDtype_Check(a[i]); break;
            case 'i': ok = PyLong_CheckExact(a[i]); break;
            case 'b': ok = PyBool_Check(a[i]); break;
            case 'f': ok = PyFloat_CheckExact(a[i]); break;
        }
        if (!ok) return false;
    }
    return true;
}

// Runs a call's marshalling; the entry point itself runs without the interpreter's lock, as it did through ctypes.
template <typename F>
PyObject* run(PyObject* const* a, Py_ssize_t n, const char* kinds, F&& marshal) {
    if (n == (Py_ssize_t)strlen(kinds) && served(a, n, kinds) && !at::impl::torch_function_mode_enabled()) {
        try {
            auto call = marshal();
            // (noexcept: an exception out of the C entry point would leave here without the lock)
            const int status = [&]() noexcept {
                int st;
                Py_BEGIN_ALLOW_THREADS
                st = call();
                Py_END_ALLOW_THREADS
                return st;
            }();
            return PyLong_FromLong(status);
        } catch (...) {  // declined, or a tensor that has no address: nothing has been called
        }
    }
    Py_RETURN_NONE;
}

#define MX_CALL(name) PyObject* name(PyObject*, PyObject* const* a, Py_ssize_t n)

MX_CALL(quantize) {  // x, rule, codes, scales
    return run(a, n, "tstt", [&] {
        const Rows x = bf16_rows(a[0]);
        const mx_rule_t r = rule(a[1]);
        uint8_t *c = bytes(a[2], x.rows, x.K / 2), *s = bytes(a[3], x.rows, x.K / 32);
        void* st = stream();
        return [=] { return calls.quantize(x.data, x.rows, x.K, x.ld, r, c, s, st); };
    });
}
MX_CALL(quantize_mbs) {  // x, rule, codes, scales, mbs
    return run(a, n, "tsttt", [&] {
        const Rows x = bf16_rows(a[0]);
        const mx_rule_t r = rule(a[1]);
        uint8_t *c = bytes(a[2], x.rows, x.K / 2), *s = bytes(a[3], x.rows, x.K / 32), *m = bytes(a[4], x.rows, (x.K + 127) / 128);
        void* st = stream();
        return [=] { return calls.quantize_mbs(x.data, x.rows, x.K, x.ld, r, c, s, m, st); };
    });
}
MX_CALL(quantize_mbs_pair) {  // x0, x1, rule, codes0, scales0, mbs0, codes1, scales1, mbs1
    return run(a, n, "ttstttttt", [&] {
        const Rows x = bf16_rows(a[0]), y = bf16_rows(a[1]);
        need(x.K == y.K);
        const mx_rule_t r = rule(a[2]);
        uint8_t *c0 = bytes(a[3], x.rows, x.K / 2), *s0 = bytes(a[4], x.rows, x.K / 32), *m0 = bytes(a[5], x.rows, (x.K + 127) / 128);
        uint8_t *c1 = bytes(a[6], y.rows, y.K / 2), *s1 = bytes(a[7], y.rows, y.K / 32), *m1 = bytes(a[8], y.rows, (y.K + 127) / 128);
        void* st = stream();
        return [=] { return calls.quantize_mbs_pair(x.data, x.rows, x.ld, c0, s0, m0, y.data, y.rows, y.ld, c1, s1, m1, x.K, r, st); };
    });
}
MX_CALL(quantize_mbs_dynamic) {  // x, rule, first, count, stride, codes, scales, mbs
    return run(a, n, "tsiiittt", [&] {
        const Rows x = bf16_rows(a[0]);
        const mx_rule_t r = rule(a[1]);
        const int64_t first = integer(a[2]), count = integer(a[3]), stride = integer(a[4]);
        need(first == (int32_t)first && count == (int32_t)count && stride == (int32_t)stride);
        uint8_t *c = bytes(a[5], x.rows, x.K / 2), *s = bytes(a[6], x.rows, x.K / 32), *m = bytes(a[7], x.rows, (x.K + 127) / 128);
        void* st = stream();
        return [=] { return calls.quantize_mbs_dynamic(x.data, x.rows, x.K, x.ld, r, (int32_t)first, (int32_t)count, (int32_t)stride, c, s, m, st); };
    });
}
MX_CALL(quantize_elem) {  // x, elem, rule, use_mbs, codes, scales, mbs (looked at with use_mbs only)
    return run(a, n, "tssbtto", [&] {
        const Rows x = bf16_rows(a[0]);
        const mx_elem_t e = elem(a[1]);
        const mx_rule_t r = rule(a[2]);
        const bool words = flag(a[3]);
        uint8_t *c = bytes(a[4], x.rows, code_bytes(e, x.K)), *s = bytes(a[5], x.rows, x.K / 32), *m = words ? bytes(a[6], x.rows, (x.K + 127) / 128) : nullptr;
        void* st = stream();
        return [=] { return calls.quantize_elem(e, x.data, x.rows, x.K, x.ld, r, words, c, s, m, st); };
    });
}
MX_CALL(dequantize) {  // codes, scales, mbs, type, out
    return run(a, n, "toodt", [&] {
        const at::Tensor& c = matrix(a[0]);
        const int64_t rows = c.size(0), K = c.size(1) * 2;
        const uint8_t *s = optional(a[1]), *m = optional(a[2]), *cp = address(c);
        const Out o = out_matrix(a[3], a[4], rows, K);
        void* st = stream();
        return [=] { return calls.dequantize(cp, s, m, rows, K, o.type, o.data, o.ld, st); };
    });
}

struct Operands {  // MXFP4 operands of a GEMM
    const uint8_t *ac, *as, *am, *bc, *bs, *bm;
    int64_t M, N, K;  // (N: the rows of B)
};
Operands operands(PyObject* ac, PyObject* as, PyObject* am, PyObject* bc, PyObject* bs, PyObject* bm) {
    const at::Tensor &x = matrix(ac), &w = matrix(bc);
    need(x.size(1) == w.size(1));
    return {address(x), optional(as), optional(am), address(w), optional(bs), optional(bm), x.size(0), w.size(0), x.size(1) * 2};
}
MX_CALL(gemm) {  // a_codes, a_scales, b_codes, b_scales, type, out
    return run(a, n, "totodt", [&] {
        const Operands p = operands(a[0], a[1], Py_None, a[2], a[3], Py_None);
        const Out o = out_matrix(a[4], a[5], p.M, p.N);
        void* st = stream();
        return [=] { return calls.gemm(p.ac, p.as, p.bc, p.bs, p.M, p.N, p.K, o.type, o.data, o.ld, st); };
    });
}
MX_CALL(gemm_mbs) {  // a_codes, a_scales, a_mbs, b_codes, b_scales, b_mbs, type, out
    return run(a, n, "tootoodt", [&] {
        const Operands p = operands(a[0], a[1], a[2], a[3], a[4], a[5]);
        const Out o = out_matrix(a[6], a[7], p.M, p.N);
        void* st = stream();
        return [=] { return calls.gemm_mbs(p.ac, p.as, p.am, p.bc, p.bs, p.bm, p.M, p.N, p.K, o.type, o.data, o.ld, st); };
    });
}
struct Groups {
    const int64_t* offsets;
    int32_t count;
};
Groups groups(PyObject* offsets, PyObject* N, int64_t b_rows) {
    const at::Tensor& t = tensor(offsets);
    need(t.scalar_type() == at::kLong && t.is_contiguous());
    const int64_t count = t.numel() - 1;
    int64_t rows;
    need(count == (int32_t)count && !__builtin_mul_overflow(count, integer(N), &rows) && rows == b_rows);
    return {address<const int64_t>(t), (int32_t)count};
}
MX_CALL(gemm_mbs_grouped) {  // a_codes, a_scales, a_mbs, b_codes, b_scales, b_mbs, row_offsets, N, type, out
    return run(a, n, "tootootidt", [&] {
        const Operands p = operands(a[0], a[1], a[2], a[3], a[4], a[5]);
        const Groups g = groups(a[6], a[7], p.N);
        const int64_t N = integer(a[7]);
        const Out o = out_matrix(a[8], a[9], p.M, N);
        void* st = stream();
        return [=] { return calls.gemm_mbs_grouped(p.ac, p.as, p.am, p.bc, p.bs, p.bm, g.count, g.offsets, p.M, N, p.K, o.type, o.data, o.ld, st); };
    });
}
MX_CALL(gemm_mbs_quantize_a) {  // a, rule, a_use_mbs, b_codes, b_scales, b_mbs, type, out
    return run(a, n, "tsbtoodt", [&] {
        const Rows x = bf16_rows(a[0]);
        const mx_rule_t r = rule(a[1]);
        const bool words = flag(a[2]);
        const at::Tensor& w = matrix(a[3]);
        need(w.size(1) * 2 == x.K);
        const uint8_t *bc = address(w), *bs = optional(a[4]), *bm = optional(a[5]);
        const int64_t N = w.size(0);
        const Out o = out_matrix(a[6], a[7], x.rows, N);
        void* st = stream();
        return [=] { return calls.gemm_mbs_quantize_a(x.data, x.ld, r, words, bc, bs, bm, x.rows, N, x.K, o.type, o.data, o.ld, st); };
    });
}
struct ElemOperands {
    mx_elem_t ae, be;
    Operands p;
};
ElemOperands elem_operands(PyObject* const* a) {  // a_elem, a_codes, a_scales, a_mbs, b_elem, b_codes, b_scales, b_mbs
    ElemOperands q;
    q.ae = elem(a[0]);
    q.be = elem(a[4]);
    const at::Tensor &x = matrix(a[1]), &xs = matrix(a[2]), &w = matrix(a[5]), &ws = matrix(a[6]);
    const int64_t K = xs.size(1) * 32;
    need(ws.size(1) * 32 == K && x.size(1) == code_bytes(q.ae, K) && w.size(1) == code_bytes(q.be, K));
    q.p = {address(x), address(xs), optional(a[3]), address(w), address(ws), optional(a[7]), x.size(0), w.size(0), K};
    return q;
}
MX_CALL(gemm_mbs_elem) {  // a_elem .. b_mbs, type, out
    return run(a, n, "sttosttodt", [&] {
        const ElemOperands q = elem_operands(a);
        const Out o = out_matrix(a[8], a[9], q.p.M, q.p.N);
        void* st = stream();
        return [=] {
            const Operands& p = q.p;
            return calls.gemm_mbs_elem(q.ae, p.ac, p.as, p.am, q.be, p.bc, p.bs, p.bm, p.M, p.N, p.K, o.type, o.data, o.ld, st);
        };
    });
}
MX_CALL(gemm_mbs_elem_grouped) {  // a_elem .. b_mbs, row_offsets, N, type, out
    return run(a, n, "sttosttotidt", [&] {
        const ElemOperands q = elem_operands(a);
        const Groups g = groups(a[8], a[9], q.p.N);
        const int64_t N = integer(a[9]);
        const Out o = out_matrix(a[10], a[11], q.p.M, N);
        void* st = stream();
        return [=] {
            const Operands& p = q.p;
            return calls.gemm_mbs_elem_grouped(q.ae, p.ac, p.as, p.am, q.be, p.bc, p.bs, p.bm, g.count, g.offsets, p.M, N, p.K, o.type, o.data, o.ld, st);
        };
    });
}

// ---- the paged cache: every tensor is on the current device, or the call is declined ----
struct Here {
    c10::hip::HIPStream on = c10::hip::getCurrentHIPStream();
    void* stream() const { return on.stream(); }
    const at::Tensor& any(PyObject* o, at::ScalarType type) const {
        const at::Tensor& t = tensor(o);
        need(t.scalar_type() == type && t.device().index() == on.device_index());
        return t;
    }
    template <typename T>
    T* flat(PyObject* o, at::ScalarType type, at::IntArrayRef shape) const {
        const at::Tensor& t = any(o, type);
        need(t.sizes() == shape && t.is_contiguous());
        return address<T>(t);
    }
    template <typename T>
    T* flat_or_null(PyObject* o, at::ScalarType type, at::IntArrayRef shape) const {
        return o == Py_None ? nullptr : flat<T>(o, type, shape);
    }
    struct Heads {  // [T, heads, D], a token's heads next to each other
        void* data;
        int64_t T, H, D, ld;
    };
    Heads heads(PyObject* o, at::ScalarType type = at::kBFloat16) const {
        const at::Tensor& t = any(o, type);
        need(t.dim() == 3);
        const Heads h = {address<void>(t), t.size(0), t.size(1), t.size(2), t.stride(0)};
        if (h.T && h.H) need((t.stride(2) == 1 || h.D <= 1) && (t.stride(1) == h.D || h.H <= 1));
        return {h.data, h.T, h.H, h.D, h.T > 1 ? h.ld : std::max(h.ld, h.H * h.D)};
    }
    Heads heads(PyObject* o, at::ScalarType type, int64_t T, int64_t H, int64_t D) const {
        const Heads h = heads(o, type);
        need(h.T == T && h.H == H && h.D == D);
        return h;
    }
    struct Cache {
        uint8_t *kc, *ks, *km, *vc, *vs, *vm;
        int64_t pages, heads, page, D;
    };
    Cache cache(PyObject* const* a) const {  // k codes, scales, mbs, v codes, scales, mbs
        const at::Tensor& k = any(a[0], at::kByte);
        need(k.dim() == 5);
        const int64_t P = k.size(0), H = k.size(1), B = k.size(2), page = k.size(3), D = 32 * B;
        Cache c = {};
        c.kc = flat<uint8_t>(a[0], at::kByte, {P, H, B, page, 16});
        c.ks = flat<uint8_t>(a[1], at::kByte, {P, H, B, page});
        c.km = flat_or_null<uint8_t>(a[2], at::kByte, {P, H, (D + 127) / 128, page});
        c.vc = flat<uint8_t>(a[3], at::kByte, {P, H, page / 4, D / 8, 4, 4});
        c.vs = flat<uint8_t>(a[4], at::kByte, {P, H, B, page});
        c.vm = flat_or_null<uint8_t>(a[5], at::kByte, {P, H, (D + 127) / 128, page});
        need((a[2] == Py_None) == (a[5] == Py_None));
        c.pages = P; c.heads = H; c.page = page; c.D = D;
        return c;
    }
    struct Turn {
        Heads q, k;
        const int32_t* positions;
        const float* table;
        const void *qw, *kw;
        int64_t rows, R;
    };
    Turn turn(PyObject* q, PyObject* k, PyObject* positions, PyObject* table, PyObject* qw, PyObject* kw) const {
        Turn t = {heads(q), heads(k), nullptr, nullptr, nullptr, nullptr, 0, 0};
        need(t.k.T == t.q.T && t.k.D == t.q.D);
        if (table != Py_None) {
            const at::Tensor& x = any(table, at::kFloat);
            need(x.dim() == 2 && x.is_contiguous() && positions != Py_None);
            t.table = address<const float>(x);
            t.rows = x.size(0);
            t.R = x.size(1);
            t.positions = flat<const int32_t>(positions, at::kInt, {t.q.T});
        }
        t.qw = flat_or_null<const void>(qw, at::kBFloat16, {t.q.D});
        t.kw = flat_or_null<const void>(kw, at::kBFloat16, {t.q.D});
        return t;
    }
};
mx_rope_t style(PyObject* o) {
    static const char* const kNames[] = {"half", "pairs"};  // MX_ROPE_HALF, MX_ROPE_PAIRS
    return (mx_rope_t)name_of(o, kNames);
}

MX_CALL(kv_plan) {  // ctx_lens, new_lens, page, block_table, free_pages, free_start, tokens, row_offsets, kv_lens, slots, positions, free_next
    return run(a, n, "ttitttittttt", [&] {
        const Here at_;
        const at::Tensor &ctx = at_.any(a[0], at::kInt), &table = at_.any(a[3], at::kInt), &free = at_.any(a[4], at::kInt);
        need(ctx.dim() == 1 && table.dim() == 2 && free.dim() == 1);
        const int64_t S = ctx.size(0), width = table.size(1), count = free.size(0), page = integer(a[2]), T = integer(a[6]);
        need(T >= 0);
        const int32_t *c = at_.flat<int32_t>(a[0], at::kInt, {S}), *nw = at_.flat<int32_t>(a[1], at::kInt, {S}), *f = at_.flat<int32_t>(a[4], at::kInt, {count}),
                      *fs = at_.flat<int32_t>(a[5], at::kInt, {1});
        int32_t *b = at_.flat<int32_t>(a[3], at::kInt, {S, width}), *lens = at_.flat<int32_t>(a[8], at::kInt, {S}), *pos = at_.flat<int32_t>(a[10], at::kInt, {T}),
                *next = at_.flat<int32_t>(a[11], at::kInt, {1});
        int64_t *off = at_.flat<int64_t>(a[7], at::kLong, {S + 1}), *slots = at_.flat<int64_t>(a[9], at::kLong, {T});
        void* st = at_.stream();
        return [=] { return calls.kv_plan(c, nw, S, page, b, width, f, count, fs, T, off, lens, slots, pos, next, st); };
    });
}
MX_CALL(qk_norm_rope) {  // q, k, positions, cos_sin, q_weight, k_weight, eps, style, q_out, k_out
    return run(a, n, "ttoooofstt", [&] {
        const Here at_;
        const Here::Turn t = at_.turn(a[0], a[1], a[2], a[3], a[4], a[5]);
        const double eps = PyFloat_AS_DOUBLE(a[6]);
        const mx_rope_t how = style(a[7]);
        const Here::Heads qo = at_.heads(a[8], at::kBFloat16, t.q.T, t.q.H, t.q.D), ko = at_.heads(a[9], at::kBFloat16, t.k.T, t.k.H, t.k.D);
        void* st = at_.stream();
        return [=] {
            return calls.qk_norm_rope(t.q.data, t.q.ld, t.k.data, t.k.ld, t.positions, t.table, t.rows, t.qw, t.kw, eps, how, t.q.T, t.q.H, t.k.H, t.q.D, t.R,
                                      qo.data, qo.ld, ko.data, ko.ld, st);
        };
    });
}
MX_CALL(kv_write) {  // k, v, slots, the cache's six, rule
    return run(a, n, "tttttottos", [&] {
        const Here at_;
        const Here::Cache c = at_.cache(a + 3);
        const Here::Heads k = at_.heads(a[0]);
        need(k.H == c.heads && k.D == c.D);
        const Here::Heads v = at_.heads(a[1], at::kBFloat16, k.T, k.H, k.D);
        const int64_t* slots = at_.flat<int64_t>(a[2], at::kLong, {k.T});
        const mx_rule_t r = rule(a[9]);
        void* st = at_.stream();
        return [=] { return calls.kv_write(k.data, k.ld, v.data, v.ld, slots, r, c.kc, c.ks, c.km, c.vc, c.vs, c.vm, c.pages, c.page, k.T, c.heads, c.D, st); };
    });
}
MX_CALL(qk_norm_rope_kv_write) {  // q, k, v, positions, slots, cos_sin, the cache's six, q_weight, k_weight, eps, style, rule, q_out
    return run(a, n, "tttotottottooofsst", [&] {
        const Here at_;
        const Here::Cache c = at_.cache(a + 6);
        const Here::Turn t = at_.turn(a[0], a[1], a[3], a[5], a[12], a[13]);
        need(t.k.H == c.heads && t.k.D == c.D);
        const Here::Heads v = at_.heads(a[2], at::kBFloat16, t.k.T, t.k.H, t.k.D);
        const int64_t* slots = at_.flat<int64_t>(a[4], at::kLong, {t.k.T});
        const double eps = PyFloat_AS_DOUBLE(a[14]);
        const mx_rope_t how = style(a[15]);
        const mx_rule_t r = rule(a[16]);
        const Here::Heads qo = at_.heads(a[17], at::kBFloat16, t.q.T, t.q.H, t.q.D);
        void* st = at_.stream();
        return [=] {
            return calls.qk_norm_rope_kv_write(t.q.data, t.q.ld, t.k.data, t.k.ld, v.data, v.ld, t.positions, t.table, t.rows, t.qw, t.kw, eps, how, slots, r, c.kc, c.ks,
                                               c.km, c.vc, c.vs, c.vm, c.pages, c.page, t.q.T, t.q.H, t.k.H, t.q.D, t.R, qo.data, qo.ld, st);
        };
    });
}
MX_CALL(kv_read) {  // slots, the cache's six, type, k_out, v_out
    return run(a, n, "tttottodtt", [&] {
        const Here at_;
        const Here::Cache c = at_.cache(a + 1);
        const mx_dtype_t type = out_type(a[7]);
        const at::Tensor& s = at_.any(a[0], at::kLong);
        need(s.dim() == 1);
        const int64_t T = s.size(0);
        const int64_t* slots = at_.flat<int64_t>(a[0], at::kLong, {T});
        const at::ScalarType as = type == MX_OUT_F32 ? at::kFloat : at::kBFloat16;
        const Here::Heads k = at_.heads(a[8], as, T, c.heads, c.D), v = at_.heads(a[9], as, T, c.heads, c.D);
        void* st = at_.stream();
        return [=] { return calls.kv_read(slots, c.kc, c.ks, c.km, c.vc, c.vs, c.vm, c.pages, c.page, T, c.heads, c.D, type, k.data, k.ld, v.data, v.ld, st); };
    });
}
MX_CALL(attention_kv) {  // q, row_offsets, kv_lens, block_table, the cache's six, scale, causal, window, out, lse, workspace
    return run(a, n, "ttttttottofbitoo", [&] {
        const Here at_;
        const Here::Cache c = at_.cache(a + 4);
        const Here::Heads q = at_.heads(a[0]);
        need(q.D == c.D && c.heads && q.H % c.heads == 0);
        const at::Tensor &l = at_.any(a[2], at::kInt), &b = at_.any(a[3], at::kInt);
        need(l.dim() == 1 && b.dim() == 2);
        const int64_t S = l.size(0), width = b.size(1), window = integer(a[12]);
        const int32_t *lens = at_.flat<int32_t>(a[2], at::kInt, {S}), *table = at_.flat<int32_t>(a[3], at::kInt, {S, width});
        const int64_t* off = at_.flat<int64_t>(a[1], at::kLong, {S + 1});
        const float scale = (float)PyFloat_AS_DOUBLE(a[10]);
        const int causal = flag(a[11]);
        const Here::Heads o = at_.heads(a[13], at::kBFloat16, q.T, q.H, q.D);
        float* lse = at_.flat_or_null<float>(a[14], at::kFloat, {q.T, q.H});
        // (without a workspace of the caller's one from the allocator, which gives it to later work on this stream only)
        at::Tensor own;
        if (a[15] == Py_None) {
            const int64_t size = calls.attention_kv_workspace(S, q.T, q.H, c.heads, c.D);
            need(size >= 0);
            own = at::empty({size}, l.options().dtype(at::kByte));
        } else {
            own = at_.any(a[15], at::kByte);
            need(own.dim() == 1 && own.is_contiguous());
        }
        // (here, where an exception declines: under a dispatch mode of the caller's the allocator may give a tensor without an address)
        void* work = own.data_ptr();
        void* st = at_.stream();
        return [=] {
            return calls.attention_kv(q.data, q.ld, off, lens, table, width, c.kc, c.ks, c.km, c.vc, c.vs, c.vm, c.pages, c.page, S, q.T, q.H, c.heads, c.D, scale, causal,
                                      window, o.data, o.ld, lse, work, own.numel(), st);
        };
    });
}

// entry points' addresses, in the order of `Calls`
PyObject* use(PyObject*, PyObject* const* a, Py_ssize_t n) {
    constexpr Py_ssize_t kCount = sizeof(Calls) / sizeof(void*);
    if (n != kCount) {
        PyErr_SetString(PyExc_TypeError, "the address of every entry point is wanted");
        return nullptr;
    }
    void* found[kCount];
    for (Py_ssize_t i = 0; i < kCount; ++i) {
        found[i] = PyLong_AsVoidPtr(a[i]);
        if (!found[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null entry point");
            return nullptr;
        }
    }
    memcpy(&calls, found, sizeof calls);
    Py_RETURN_NONE;
}

// what this module was compiled against: the binding compares it before any other call (torch's objects are read through inline
// headers, at the offsets of that torch)
PyObject* built_for(PyObject*, PyObject* const*, Py_ssize_t) { return PyUnicode_FromString(MX_BUILT_FOR); }

#define MX_METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {MX_METHOD(built_for), MX_METHOD(use), MX_METHOD(quantize), MX_METHOD(quantize_mbs), MX_METHOD(quantize_mbs_pair), MX_METHOD(quantize_mbs_dynamic),
                         MX_METHOD(quantize_elem), MX_METHOD(dequantize), MX_METHOD(gemm), MX_METHOD(gemm_mbs), MX_METHOD(gemm_mbs_grouped),
                         MX_METHOD(gemm_mbs_quantize_a), MX_METHOD(gemm_mbs_elem), MX_METHOD(gemm_mbs_elem_grouped), MX_METHOD(kv_plan), MX_METHOD(qk_norm_rope), MX_METHOD(kv_write),
                         MX_METHOD(qk_norm_rope_kv_write), MX_METHOD(kv_read), MX_METHOD(attention_kv), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
