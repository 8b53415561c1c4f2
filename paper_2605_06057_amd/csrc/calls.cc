// The Python side of the 8-bit-integer calls and of those that move tokens: the arguments of a call checked and handed to the C entry point.  With ctypes that takes
// 2 to 3 us of a call (five to seven tensors, each asked for type, shape, layout and device), as long as the launch; here it is 0.3.  What a small
// batch waits for is the host: a training step's five calls on 16 tokens took 31 us.
//
// Every function returns the call's status as a number (binding.py raises the error), and raises AssertionError for a tensor that the call cannot take.
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

#define LCMA_CALL(NAME) {#NAME, (PyCFunction)(void *)NAME, METH_FASTCALL, nullptr}
PyMethodDef g_calls[] = {LCMA_CALL(i8_quantize), LCMA_CALL(i8_quantize_dispatch), LCMA_CALL(i8_gemm_nt), LCMA_CALL(i8_gemm_experts), LCMA_CALL(tokens_sort),
                         LCMA_CALL(tokens_dispatch), LCMA_CALL(tokens_combine), LCMA_CALL(tokens_combine_grad), {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, g_calls, nullptr, nullptr, nullptr, nullptr};

} // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&g_module); }
