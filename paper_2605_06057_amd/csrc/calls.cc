// The Python side of the calls in 8 and 4 bits, of the experts' and of those that move tokens: the arguments of a call checked and handed to the C entry point.  With ctypes that takes
// 2 to 3 us of a call (five to seven tensors, each asked for type, shape, layout and device), as long as the launch; here it is 0.3.  What a small
// batch waits for is the host: a training step's five calls on 16 tokens took 31 us.
//
// Every function returns the call's status as a number (binding.py raises the error), and raises AssertionError for a tensor that the call cannot take.
#include <c10/hip/HIPGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>
#include <stdexcept>

#include "../../include/lcma.h"

namespace {

struct Refused : std::runtime_error {
    using std::runtime_error::runtime_error;
};
[[noreturn]] void refuse(const char *name, const char *why) { throw Refused(std::string(name) + ": expected " + why); }

const at::Tensor &tensor(PyObject *o, const char *name) {
    if (!THPVariable_Check(o)) refuse(name, "a tensor");
    return THPVariable_Unpack(o);
}
long long number(PyObject *o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw std::exception();
    return v;
}
lcma_dtype storage(const at::Tensor &t, const char *name) {
    switch (t.scalar_type()) {
    case at::kFloat: return LCMA_F32;
    case at::kBFloat16: return LCMA_BF16;
    case at::kHalf: return LCMA_F16;
    default: refuse(name, "float32, bfloat16 or float16");
    }
}
int gpu_of(const at::Tensor &t, const char *name) {
    if (!t.is_cuda()) refuse(name, "a tensor on the GPU");
    return t.get_device();
}
// Contiguous, of that type and shape, on that GPU.
void *whole(const at::Tensor &t, const char *name, at::ScalarType type, c10::IntArrayRef shape, int gpu) {
    if (t.scalar_type() != type) refuse(name, type == at::kChar ? "int8" : type == at::kInt ? "int32" : "float32");
    if (t.sizes() != shape) refuse(name, "another shape");
    if (!t.is_contiguous()) refuse(name, "a contiguous tensor");
    if (!t.is_cuda() || t.get_device() != gpu) refuse(name, "a tensor on the same GPU");
    return t.data_ptr();
}
void *whole(PyObject *o, const char *name, at::ScalarType type, c10::IntArrayRef shape, int gpu) { return whole(tensor(o, name), name, type, shape, gpu); }
// A matrix whose rows are contiguous; its leading dimension (of a single row, whose stride says nothing: the row).
struct Rows {
    char *at;
    int64_t ld;
};
Rows rows(const at::Tensor &t, const char *name, int64_t n, int64_t cols, int gpu, at::ScalarType type) {
    if (t.dim() != 2 || t.size(0) != n || t.size(1) != cols) refuse(name, "another shape");
    if (t.scalar_type() != type) refuse(name, "the other rows' type");
    if (cols > 1 && t.stride(1) != 1) refuse(name, "neighbouring elements in a row");
    if (!t.is_cuda() || t.get_device() != gpu) refuse(name, "a tensor on the same GPU");
    return {(char *)t.data_ptr(), n <= 1 ? cols : t.stride(0)};
}
Rows rows(PyObject *o, const char *name, int64_t n, int64_t cols, int gpu, at::ScalarType type) { return rows(tensor(o, name), name, n, cols, gpu, type); }
// Contiguous, of `type` and that shape, on that GPU: of a type that another operand has.
void *same(const at::Tensor &t, const char *name, at::ScalarType type, c10::IntArrayRef shape, int gpu) {
    if (t.scalar_type() != type) refuse(name, "the other operands' type");
    if (t.sizes() != shape) refuse(name, "another shape");
    if (!t.is_contiguous()) refuse(name, "a contiguous tensor");
    if (!t.is_cuda() || t.get_device() != gpu) refuse(name, "a tensor on the same GPU");
    return t.data_ptr();
}
// Weights in 4 bits as the library lays them out: bytes for every expert.
void *prepared(PyObject *o, int64_t experts, int64_t bytes, int gpu) {
    const at::Tensor &t = tensor(o, "Wp");
    if (t.scalar_type() != at::kByte) refuse("Wp", "uint8");
    if (bytes < 0) refuse("Wp", "sizes and a group (32, 64 or 128) that 4-bit weights have");
    if (experts < 0 ? t.sizes() != c10::IntArrayRef{bytes} : t.sizes() != c10::IntArrayRef{experts, bytes}) refuse("Wp", "another shape");
    if (!t.is_contiguous()) refuse("Wp", "a contiguous tensor");
    if (!t.is_cuda() || t.get_device() != gpu) refuse("Wp", "a tensor on the same GPU");
    return t.data_ptr();
}
void *stream_of(int gpu) { return (void *)c10::hip::getCurrentHIPStream((c10::DeviceIndex)gpu).stream(); }
// (a number that the C entry points refuse in place of one that an int does not hold)
int as_int(int64_t v) { return v > INT32_MAX ? INT32_MAX : (int)v; }
const at::Tensor &matrix(PyObject *o, const char *name) {
    const at::Tensor &t = tensor(o, name);
    if (t.dim() != 2) refuse(name, "two dimensions");
    return t;
}

template <int N, class F> PyObject *call(PyObject *const *, Py_ssize_t n, F &&f) {
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "expected %d arguments, got %zd", N, n);
        return nullptr;
    }
    try {
        return PyLong_FromLong(f());
    } catch (const Refused &e) {
        PyErr_SetString(PyExc_AssertionError, e.what());
    } catch (const std::exception &e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
    }
    return nullptr;
}

PyObject *i8_quantize(PyObject *, PyObject *const *a, Py_ssize_t n) { // X, Q, S, gated
    return call<4>(a, n, [&] {
        const at::Tensor &x = matrix(a[0], "X");
        const int gated = PyObject_IsTrue(a[3]);
        if (gated < 0) throw std::exception();
        const int64_t r = x.size(0), width = x.size(1), K = gated ? width / 2 : width;
        if (gated && width % 2) refuse("X", "rows x 2 K");
        const int gpu = gpu_of(x, "X");
        const Rows in = rows(x, "X", r, width, gpu, x.scalar_type());
        void *q = whole(a[1], "Q", at::kChar, {r, lcma_i8_code_pitch(K)}, gpu), *s = whole(a[2], "S", at::kFloat, {r}, gpu);
        return lcma_i8_quantize(r, K, in.at, in.ld, storage(x, "X"), gated, q, (float *)s, stream_of(gpu));
    });
}
PyObject *i8_quantize_dispatch(PyObject *, PyObject *const *a, Py_ssize_t n) { // X, position, Q, S
    return call<4>(a, n, [&] {
        const at::Tensor &x = matrix(a[0], "X"), &position = matrix(a[1], "position");
        const int64_t tokens = x.size(0), K = x.size(1), top = position.size(1);
        const int gpu = gpu_of(x, "X");
        const Rows in = rows(x, "X", tokens, K, gpu, x.scalar_type());
        void *to = whole(position, "position", at::kInt, {tokens, top}, gpu);
        void *q = whole(a[2], "Q", at::kChar, {tokens * top, lcma_i8_code_pitch(K)}, gpu), *s = whole(a[3], "S", at::kFloat, {tokens * top}, gpu);
        return lcma_i8_quantize_dispatch(tokens, K, in.at, in.ld, storage(x, "X"), as_int(top), (const int32_t *)to, q, (float *)s, stream_of(gpu));
    });
}
PyObject *i8_gemm_nt(PyObject *, PyObject *const *a, Py_ssize_t n) { // Aq, Sa, Wq, Sw, C, K, bias
    return call<7>(a, n, [&] {
        const at::Tensor &c = matrix(a[4], "C");
        const int64_t M = c.size(0), N = c.size(1), K = number(a[5]), pitch = lcma_i8_code_pitch(K);
        const int gpu = gpu_of(c, "C");
        const void *aq = whole(a[0], "Aq", at::kChar, {M, pitch}, gpu), *sa = whole(a[1], "Sa", at::kFloat, {M}, gpu);
        const void *wq = whole(a[2], "Wq", at::kChar, {N, pitch}, gpu), *sw = whole(a[3], "Sw", at::kFloat, {N}, gpu);
        const void *bias = a[6] == Py_None ? nullptr : whole(a[6], "bias", at::kFloat, {N}, gpu);
        const Rows out = rows(c, "C", M, N, gpu, c.scalar_type());
        return lcma_i8_gemm_nt(M, N, K, aq, (const float *)sa, wq, (const float *)sw, (const float *)bias, out.at, out.ld, storage(c, "C"), stream_of(gpu));
    });
}
PyObject *i8_gemm_experts(PyObject *, PyObject *const *a, Py_ssize_t n) { // Aq, Sa, offsets, Wq, Sw, C, K, bias
    return call<8>(a, n, [&] {
        const at::Tensor &c = matrix(a[5], "C"), &w = tensor(a[3], "Wq");
        const int64_t r = c.size(0), N = c.size(1), E = w.dim() ? w.size(0) : 0, K = number(a[6]), pitch = lcma_i8_code_pitch(K);
        const int gpu = gpu_of(c, "C");
        const void *aq = whole(a[0], "Aq", at::kChar, {r, pitch}, gpu), *sa = whole(a[1], "Sa", at::kFloat, {r}, gpu);
        const void *offsets = whole(a[2], "offsets", at::kInt, {E + 1}, gpu);
        const void *wq = whole(w, "Wq", at::kChar, {E, N, pitch}, gpu), *sw = whole(a[4], "Sw", at::kFloat, {E, N}, gpu);
        const void *bias = a[7] == Py_None ? nullptr : whole(a[7], "bias", at::kFloat, {E, N}, gpu);
        const Rows out = rows(c, "C", r, N, gpu, c.scalar_type());
        return lcma_i8_gemm_experts(r, N, K, as_int(E), (const int32_t *)offsets, aq, (const float *)sa, wq, (const float *)sw, (const float *)bias, out.at, out.ld,
                                    storage(c, "C"), stream_of(gpu));
    });
}
PyObject *tokens_sort(PyObject *, PyObject *const *a, Py_ssize_t n) { // ids, experts, order, position, offsets, workspace
    return call<6>(a, n, [&] {
        const at::Tensor &ids = matrix(a[0], "ids");
        const int64_t tokens = ids.size(0), top = ids.size(1), E = number(a[1]);
        if (E < 1 || E > INT32_MAX) refuse("experts", "at least one");
        const int gpu = gpu_of(ids, "ids");
        const void *in = whole(ids, "ids", at::kInt, {tokens, top}, gpu);
        void *order = whole(a[2], "order", at::kInt, {tokens * top}, gpu), *position = whole(a[3], "position", at::kInt, {tokens, top}, gpu);
        void *offsets = whole(a[4], "offsets", at::kInt, {E + 1}, gpu), *space = nullptr;
        int64_t size = 0;
        if (a[5] != Py_None) {
            const at::Tensor &w = tensor(a[5], "workspace");
            if (!w.is_contiguous() || !w.is_cuda() || w.get_device() != gpu) refuse("workspace", "a contiguous tensor on the same GPU");
            space = w.data_ptr();
            size = (int64_t)w.nbytes();
        }
        return lcma_tokens_sort(tokens, as_int(top), (int)E, (const int32_t *)in, (int32_t *)order, (int32_t *)position, (int32_t *)offsets, space, size, stream_of(gpu));
    });
}
PyObject *tokens_dispatch(PyObject *, PyObject *const *a, Py_ssize_t n) { // X, position, Y
    return call<3>(a, n, [&] {
        const at::Tensor &x = matrix(a[0], "X"), &position = matrix(a[1], "position");
        const int64_t tokens = x.size(0), H = x.size(1), top = position.size(1);
        const int gpu = gpu_of(x, "X");
        const Rows in = rows(x, "X", tokens, H, gpu, x.scalar_type()), out = rows(a[2], "Y", tokens * top, H, gpu, x.scalar_type());
        const void *to = whole(position, "position", at::kInt, {tokens, top}, gpu);
        return lcma_tokens_dispatch(tokens, as_int(top), H, in.at, in.ld, storage(x, "X"), (const int32_t *)to, out.at, out.ld, stream_of(gpu));
    });
}
PyObject *tokens_combine(PyObject *, PyObject *const *a, Py_ssize_t n) { // Y, position, weights, X
    return call<4>(a, n, [&] {
        const at::Tensor &y = matrix(a[0], "Y"), &position = matrix(a[1], "position");
        const int64_t tokens = position.size(0), top = position.size(1), H = y.size(1);
        const int gpu = gpu_of(y, "Y");
        const Rows in = rows(y, "Y", tokens * top, H, gpu, y.scalar_type()), out = rows(a[3], "X", tokens, H, gpu, y.scalar_type());
        const void *to = whole(position, "position", at::kInt, {tokens, top}, gpu);
        const void *w = a[2] == Py_None ? nullptr : whole(a[2], "weights", at::kFloat, {tokens, top}, gpu);
        return lcma_tokens_combine(tokens, as_int(top), H, in.at, in.ld, storage(y, "Y"), (const int32_t *)to, (const float *)w, out.at, out.ld, stream_of(gpu));
    });
}
PyObject *tokens_combine_grad(PyObject *, PyObject *const *a, Py_ssize_t n) { // dX, Y, position, weights, dY, dweights
    return call<6>(a, n, [&] {
        const at::Tensor &y = matrix(a[1], "Y"), &position = matrix(a[2], "position");
        const int64_t tokens = position.size(0), top = position.size(1), H = y.size(1);
        const int gpu = gpu_of(y, "Y");
        const at::ScalarType type = y.scalar_type();
        const Rows dx = rows(a[0], "dX", tokens, H, gpu, type), in = rows(y, "Y", tokens * top, H, gpu, type), dy = rows(a[4], "dY", tokens * top, H, gpu, type);
        const void *to = whole(position, "position", at::kInt, {tokens, top}, gpu), *w = whole(a[3], "weights", at::kFloat, {tokens, top}, gpu);
        void *dw = whole(a[5], "dweights", at::kFloat, {tokens, top}, gpu);
        return lcma_tokens_combine_grad(tokens, as_int(top), H, dx.at, dx.ld, in.at, in.ld, storage(y, "Y"), (const int32_t *)to, (const float *)w, dy.at, dy.ld, (float *)dw,
                                        stream_of(gpu));
    });
}

// (the calls below launch on their tensors' GPU, whichever is the current one)
using On = c10::hip::HIPGuard;

PyObject *gemm_experts(PyObject *, PyObject *const *a, Py_ssize_t n) { // A, offsets, W, C, b_nk
    return call<5>(a, n, [&] {
        const at::Tensor &x = matrix(a[0], "A"), &w = tensor(a[2], "W"), &c = matrix(a[3], "C");
        const int nk = PyObject_IsTrue(a[4]);
        if (nk < 0) throw std::exception();
        if (w.dim() != 3) refuse("W", "three dimensions");
        const int64_t r = x.size(0), K = x.size(1), N = c.size(1), E = w.size(0);
        const int gpu = gpu_of(x, "A");
        const On on((c10::DeviceIndex)gpu);
        const at::ScalarType type = x.scalar_type();
        const Rows in = rows(x, "A", r, K, gpu, type), out = rows(c, "C", r, N, gpu, type);
        const void *offsets = whole(a[1], "offsets", at::kInt, {E + 1}, gpu);
        const void *b = nk ? same(w, "W", type, {E, N, K}, gpu) : same(w, "W", type, {E, K, N}, gpu);
        return lcma_gemm_experts(nk ? 2 : 0, r, N, K, as_int(E), (const int32_t *)offsets, in.at, in.ld, b, out.at, out.ld, storage(x, "A"), stream_of(gpu));
    });
}
PyObject *gemm_experts_grad(PyObject *, PyObject *const *a, Py_ssize_t n) { // dC, A, offsets, dW
    return call<4>(a, n, [&] {
        const at::Tensor &dc = matrix(a[0], "dC"), &x = matrix(a[1], "A"), &dw = tensor(a[3], "dW");
        if (dw.dim() != 3) refuse("dW", "three dimensions");
        const int64_t r = x.size(0), N = dc.size(1), K = x.size(1), E = dw.size(0);
        const int gpu = gpu_of(x, "A");
        const On on((c10::DeviceIndex)gpu);
        const at::ScalarType type = x.scalar_type();
        const Rows in = rows(x, "A", r, K, gpu, type), grad = rows(dc, "dC", r, N, gpu, type);
        const void *offsets = whole(a[2], "offsets", at::kInt, {E + 1}, gpu);
        void *out = same(dw, "dW", type, {E, N, K}, gpu);
        return lcma_gemm_experts_grad(r, N, K, as_int(E), (const int32_t *)offsets, grad.at, grad.ld, in.at, in.ld, out, storage(x, "A"), stream_of(gpu));
    });
}
PyObject *gated_silu(PyObject *, PyObject *const *a, Py_ssize_t n) { // X, Y
    return call<2>(a, n, [&] {
        const at::Tensor &x = matrix(a[0], "X");
        const int64_t r = x.size(0), F = x.size(1) / 2;
        if (x.size(1) % 2) refuse("X", "rows x 2 F");
        const int gpu = gpu_of(x, "X");
        const On on((c10::DeviceIndex)gpu);
        const Rows in = rows(x, "X", r, 2 * F, gpu, x.scalar_type()), out = rows(a[1], "Y", r, F, gpu, x.scalar_type());
        return lcma_gated_silu(r, F, in.at, in.ld, out.at, out.ld, storage(x, "X"), stream_of(gpu));
    });
}
PyObject *gated_silu_grad(PyObject *, PyObject *const *a, Py_ssize_t n) { // dY, X, dX
    return call<3>(a, n, [&] {
        const at::Tensor &x = matrix(a[1], "X");
        const int64_t r = x.size(0), F = x.size(1) / 2;
        if (x.size(1) % 2) refuse("X", "rows x 2 F");
        const int gpu = gpu_of(x, "X");
        const On on((c10::DeviceIndex)gpu);
        const at::ScalarType type = x.scalar_type();
        const Rows dy = rows(a[0], "dY", r, F, gpu, type), in = rows(x, "X", r, 2 * F, gpu, type), out = rows(a[2], "dX", r, 2 * F, gpu, type);
        return lcma_gated_silu_grad(r, F, dy.at, dy.ld, in.at, in.ld, out.at, out.ld, storage(x, "X"), stream_of(gpu));
    });
}
int group_of(PyObject *o) { return as_int(std::max(number(o), -1LL)); }
PyObject *i4_quantize(PyObject *, PyObject *const *a, Py_ssize_t n) { // W, group, Wp
    return call<3>(a, n, [&] {
        const at::Tensor &w = tensor(a[0], "W");
        const int64_t d = w.dim();
        if (d != 2 && d != 3) refuse("W", "two or three dimensions");
        const int64_t E = d == 3 ? w.size(0) : 1, N = w.size(d - 2), K = w.size(d - 1), ld = N <= 1 && E <= 1 ? K : N <= 1 ? w.stride(0) : w.stride(d - 2);
        const int group = group_of(a[1]), gpu = gpu_of(w, "W");
        const On on((c10::DeviceIndex)gpu);
        if (K > 1 && w.stride(d - 1) != 1) refuse("W", "neighbouring elements in a row");
        if (d == 3 && E > 1 && N > 0 && w.stride(0) != N * ld) refuse("W", "experts one behind the other");
        void *q = prepared(a[2], d == 3 ? E : -1, lcma_i4_prepared_bytes(N, K, group), gpu);
        if (E == 0) return LCMA_OK;
        return lcma_i4_quantize(as_int(E), N, K, group, w.data_ptr(), ld, storage(w, "W"), q, stream_of(gpu));
    });
}
PyObject *i4_prepare(PyObject *, PyObject *const *a, Py_ssize_t n) { // codes, scales, group, Wp
    return call<4>(a, n, [&] {
        const at::Tensor &c = tensor(a[0], "codes"), &s = tensor(a[1], "scales");
        const int64_t d = c.dim();
        if (d != 2 && d != 3) refuse("codes", "two or three dimensions");
        const int64_t E = d == 3 ? c.size(0) : 1, N = c.size(d - 2), K = c.size(d - 1);
        const int group = group_of(a[2]), gpu = gpu_of(c, "codes");
        const On on((c10::DeviceIndex)gpu);
        void *q = prepared(a[3], d == 3 ? E : -1, lcma_i4_prepared_bytes(N, K, group), gpu);
        const int64_t G = (K + group - 1) / group;
        const void *codes = whole(c, "codes", at::kChar, c.sizes(), gpu);
        const void *scales = d == 3 ? whole(s, "scales", at::kFloat, {E, N, G}, gpu) : whole(s, "scales", at::kFloat, {N, G}, gpu);
        if (E == 0) return LCMA_OK;
        return lcma_i4_prepare(as_int(E), N, K, group, (const int8_t *)codes, (const float *)scales, q, stream_of(gpu));
    });
}
PyObject *i4_gemm_nt(PyObject *, PyObject *const *a, Py_ssize_t n) { // X, Wp, C, group, bias
    return call<5>(a, n, [&] {
        const at::Tensor &x = matrix(a[0], "X"), &c = matrix(a[2], "C");
        const int64_t M = x.size(0), K = x.size(1), N = c.size(1);
        const int group = group_of(a[3]), gpu = gpu_of(x, "X");
        const On on((c10::DeviceIndex)gpu);
        const Rows in = rows(x, "X", M, K, gpu, x.scalar_type()), out = rows(c, "C", M, N, gpu, x.scalar_type());
        const void *w = prepared(a[1], -1, lcma_i4_prepared_bytes(N, K, group), gpu), *bias = a[4] == Py_None ? nullptr : whole(a[4], "bias", at::kFloat, {N}, gpu);
        return lcma_i4_gemm_nt(M, N, K, group, in.at, in.ld, w, (const float *)bias, out.at, out.ld, storage(x, "X"), stream_of(gpu));
    });
}
PyObject *i4_gemm_experts(PyObject *, PyObject *const *a, Py_ssize_t n) { // X, offsets, Wp, C, group, bias
    return call<6>(a, n, [&] {
        const at::Tensor &x = matrix(a[0], "X"), &offsets = tensor(a[1], "offsets"), &c = matrix(a[3], "C");
        if (offsets.dim() != 1 || offsets.size(0) < 2) refuse("offsets", "experts + 1 row numbers");
        const int64_t r = x.size(0), K = x.size(1), N = c.size(1), E = offsets.size(0) - 1;
        const int group = group_of(a[4]), gpu = gpu_of(x, "X");
        const On on((c10::DeviceIndex)gpu);
        const Rows in = rows(x, "X", r, K, gpu, x.scalar_type()), out = rows(c, "C", r, N, gpu, x.scalar_type());
        const void *from = whole(offsets, "offsets", at::kInt, {E + 1}, gpu), *w = prepared(a[2], E, lcma_i4_prepared_bytes(N, K, group), gpu);
        const void *bias = a[5] == Py_None ? nullptr : whole(a[5], "bias", at::kFloat, {E, N}, gpu);
        return lcma_i4_gemm_experts(r, N, K, group, as_int(E), (const int32_t *)from, in.at, in.ld, w, (const float *)bias, out.at, out.ld, storage(x, "X"), stream_of(gpu));
    });
}

#define LCMA_CALL(NAME) {#NAME, (PyCFunction)(void *)NAME, METH_FASTCALL, nullptr}
PyMethodDef g_calls[] = {LCMA_CALL(i8_quantize), LCMA_CALL(i8_quantize_dispatch), LCMA_CALL(i8_gemm_nt), LCMA_CALL(i8_gemm_experts), LCMA_CALL(tokens_sort),
                         LCMA_CALL(tokens_dispatch), LCMA_CALL(tokens_combine), LCMA_CALL(tokens_combine_grad),
                         LCMA_CALL(gemm_experts), LCMA_CALL(gemm_experts_grad), LCMA_CALL(gated_silu), LCMA_CALL(gated_silu_grad), LCMA_CALL(i4_quantize),
                         LCMA_CALL(i4_prepare), LCMA_CALL(i4_gemm_nt), LCMA_CALL(i4_gemm_experts), {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, g_calls, nullptr, nullptr, nullptr, nullptr};

} // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&g_module); }
