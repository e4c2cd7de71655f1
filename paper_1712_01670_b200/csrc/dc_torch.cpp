// Torch tensors to the entry points of libdeepcache that take a caller's own maps (dc_layer_norm and on): the module _tensors, which
// binding.py wraps.  These calls are short - a few microseconds on the GPU - and the same marshalling in Python and ctypes took longer than
// that (a normalisation into 8 bits and the product behind it, 196 x 384 x 1536: 15.3 us a pass, 6.1 so; gradients of 196 x 1024: 15.7
// and 9.2).  Argument marshalling only: addresses, pitches, types, the device and its current stream.  As in ctypes, the GIL is not held during the call itself.
#include <Python.h>

#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "deepcache.h"

namespace {

struct Refused { PyObject* type; std::string what; };

const at::Tensor* tensor(PyObject* o, const char* what, bool optional = false)
{
    if (o == Py_None && optional) return nullptr;
    if (!THPVariable_Check(o)) throw Refused{PyExc_TypeError, std::string(what) + ": a tensor is needed"};
    return &THPVariable_Unpack(o);
}

struct Rows { void* at = nullptr; size_t pitch = 0; int64_t rows = 0, channels = 0; int dtype = -1; };

// A map whose rows lie a constant stride apart.
Rows rows_of(const at::Tensor& t, const char* what, bool int8 = false)
{
    const auto type = t.scalar_type();
    Rows r;
    if (int8 ? type != at::kChar : type != at::kFloat && type != at::kBFloat16)
        throw Refused{PyExc_TypeError, std::string(what) + ": unsupported type " + c10::toString(type)};
    r.dtype = type == at::kBFloat16 ? DC_BF16 : DC_FP32;
    const int64_t size = (int64_t)t.element_size(), dims = t.dim();
    if (dims < 1) throw Refused{PyExc_ValueError, std::string(what) + ": no rows"};
    const auto n = t.sizes(), s = t.strides();
    r.channels = n[dims - 1];
    if (r.channels > 1 && s[dims - 1] != 1) throw Refused{PyExc_ValueError, std::string(what) + ": a row's elements have to lie side by side"};
    int64_t pitch = -1;
    r.rows = 1;
    for (int64_t d = dims - 2; d >= 0; --d) {
        if (n[d] == 0) { r.rows = 0; break; }
        if (n[d] == 1) continue;
        if (pitch < 0) pitch = s[d];
        else if (s[d] != pitch * r.rows) throw Refused{PyExc_ValueError, std::string(what) + ": rows do not lie a constant stride apart"};
        r.rows *= n[d];
    }
    r.at = t.data_ptr();
    // a single row's pitch is whatever the row needs (8-bit rows: a multiple of 16)
    r.pitch = pitch >= 0 && r.rows > 1 ? (size_t)(pitch * size) : int8 ? (size_t)((r.channels + 15) / 16 * 16) : (size_t)(r.channels * size);
    return r;
}

float* vector_of(const at::Tensor* t, int64_t n, const char* what, bool optional = true)
{
    if (!t) {
        if (!optional) throw Refused{PyExc_ValueError, std::string(what) + " is needed"};
        return nullptr;
    }
    if (t->scalar_type() != at::kFloat || t->numel() != n || !t->is_contiguous())
        throw Refused{PyExc_ValueError, std::string(what) + ": a contiguous float32 vector of " + std::to_string(n) + " values is needed"};
    return (float*)t->data_ptr();
}

void same(const Rows& a, const Rows& b, const char* what, bool type = true)
{
    if (a.rows != b.rows || a.channels != b.channels)
        throw Refused{PyExc_ValueError, std::string(what) + ": " + std::to_string(b.rows) + " rows of " + std::to_string(b.channels) + " where " + std::to_string(a.rows) + " of " +
                                           std::to_string(a.channels) + " are needed"};
    if (type && a.dtype != b.dtype) throw Refused{PyExc_TypeError, std::string(what) + " is of another type"};
}

// The device that all tensors are on, made the current one, and the stream: the caller's, or torch's current one there.
struct Place {
    c10::cuda::OptionalCUDAGuard guard;
    void* stream;
    Place(const char* where, std::initializer_list<const at::Tensor*> all, PyObject* given)
    {
        int device = -2;
        for (const at::Tensor* t : all) {
            if (!t) continue;
            const int d = t->is_cuda() ? (int)t->get_device() : -1;
            if (device == -2) device = d;
            if (d < 0 || d != device) throw Refused{PyExc_ValueError, std::string(where) + ": all tensors have to be on one CUDA device"};
        }
        guard.set_index(device);
        if (given == Py_None) stream = (void*)c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
        else {
            stream = PyLong_AsVoidPtr(given);
            if (PyErr_Occurred()) throw Refused{nullptr, ""};
        }
    }
};

double number(PyObject* o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Refused{nullptr, ""};
    return v;
}
int truth(PyObject* o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Refused{nullptr, ""};
    return v;
}
// The GIL is not held during the library's call: a launch waits where the stream's queue is full, and what the stream waits for may be another
// Python thread.  Everything that may run Python comes before it.  (0.1 us a call: 196 x 1024 gradients 9.2 us a pass, 8.9 with the GIL held.)
struct WithoutGil {
    PyThreadState* const state = PyEval_SaveThread();
    ~WithoutGil() { PyEval_RestoreThread(state); }
};
int32_t channels_of(const Rows& r) { return r.channels > INT32_MAX ? INT32_MAX : (int32_t)r.channels; }

int layer_norm(PyObject* const* o)       // x, gamma, beta, y, mean, rstd, eps, stream
{
    const at::Tensor *x = tensor(o[0], "x"), *gamma = tensor(o[1], "gamma", true), *beta = tensor(o[2], "beta", true), *y = tensor(o[3], "y"), *mean = tensor(o[4], "mean", true),
                     *rstd = tensor(o[5], "rstd", true);
    const Rows xr = rows_of(*x, "x"), yr = rows_of(*y, "y");
    same(xr, yr, "y");
    const float *g = vector_of(gamma, xr.channels, "gamma"), *b = vector_of(beta, xr.channels, "beta");
    float *m = vector_of(mean, xr.rows, "mean"), *r = vector_of(rstd, xr.rows, "rstd");
    const double eps = number(o[6]);
    const Place p("dc_layer_norm", {x, y, gamma, beta, mean, rstd}, o[7]);
    const WithoutGil call;
    return dc_layer_norm(xr.at, xr.pitch, g, b, xr.rows, channels_of(xr), eps, xr.dtype, yr.at, yr.pitch, m, r, p.stream);
}

int layer_norm_backward(PyObject* const* o)      // dy, x, gamma, mean, rstd, dx, dgamma, dbeta, workspace, stream
{
    const at::Tensor *dy = tensor(o[0], "dy"), *x = tensor(o[1], "x"), *gamma = tensor(o[2], "gamma", true), *mean = tensor(o[3], "mean", true), *rstd = tensor(o[4], "rstd", true),
                     *dx = tensor(o[5], "dx", true), *dgamma = tensor(o[6], "dgamma", true), *dbeta = tensor(o[7], "dbeta", true), *work = tensor(o[8], "workspace", true);
    const Rows xr = rows_of(*x, "x"), dr = rows_of(*dy, "dy");
    same(xr, dr, "dy");
    Rows ox;
    if (dx) { ox = rows_of(*dx, "dx"); same(xr, ox, "dx"); }
    if (work && !work->is_contiguous()) throw Refused{PyExc_ValueError, "workspace: has to be contiguous"};
    const float *g = vector_of(gamma, xr.channels, "gamma"), *m = vector_of(mean, xr.rows, "mean", false), *r = vector_of(rstd, xr.rows, "rstd", false);
    float *dg = vector_of(dgamma, xr.channels, "dgamma"), *db = vector_of(dbeta, xr.channels, "dbeta");
    const Place p("dc_layer_norm_backward", {x, dy, gamma, mean, rstd, dx, dgamma, dbeta, work}, o[9]);
    const WithoutGil call;
    return dc_layer_norm_backward(dr.at, dr.pitch, xr.at, xr.pitch, g, m, r, xr.rows, channels_of(xr), xr.dtype, ox.at, ox.pitch, dg, db, work ? work->data_ptr() : nullptr,
                                  work ? work->nbytes() : 0, p.stream);
}

int quantize_rows(PyObject* const* o)    // x, q, scale, stream
{
    const at::Tensor *x = tensor(o[0], "x"), *q = tensor(o[1], "q"), *scale = tensor(o[2], "scale");
    const Rows xr = rows_of(*x, "x"), qr = rows_of(*q, "q", true);
    same(xr, qr, "q", false);
    float* s = vector_of(scale, xr.rows, "scale");
    const Place p("dc_quantize_rows", {x, q, scale}, o[3]);
    const WithoutGil call;
    return dc_quantize_rows(xr.at, xr.pitch, xr.rows, channels_of(xr), xr.dtype, (int8_t*)qr.at, qr.pitch, s, p.stream);
}

int layer_norm_quantize(PyObject* const* o)      // x, gamma, beta, q, scale, y, eps, stream
{
    const at::Tensor *x = tensor(o[0], "x"), *gamma = tensor(o[1], "gamma", true), *beta = tensor(o[2], "beta", true), *q = tensor(o[3], "q"), *scale = tensor(o[4], "scale"),
                     *y = tensor(o[5], "y", true);
    const Rows xr = rows_of(*x, "x"), qr = rows_of(*q, "q", true);
    same(xr, qr, "q", false);
    Rows yr;
    if (y) { yr = rows_of(*y, "y"); same(xr, yr, "y"); }
    const float *g = vector_of(gamma, xr.channels, "gamma"), *b = vector_of(beta, xr.channels, "beta");
    float* s = vector_of(scale, xr.rows, "scale");
    const double eps = number(o[6]);
    const Place p("dc_layer_norm_quantize", {x, q, scale, gamma, beta, y}, o[7]);
    const WithoutGil call;
    return dc_layer_norm_quantize(xr.at, xr.pitch, g, b, xr.rows, channels_of(xr), eps, xr.dtype, yr.at, yr.pitch, (int8_t*)qr.at, qr.pitch, s, p.stream);
}

void fit(const Rows& a, const Rows& b, const Rows& out)
{
    if (a.channels != b.channels || out.rows != a.rows || out.channels != b.rows)
        throw Refused{PyExc_ValueError, std::to_string(a.rows) + " x " + std::to_string(a.channels) + ", " + std::to_string(b.rows) + " x " + std::to_string(b.channels) + " and " +
                                           std::to_string(out.rows) + " x " + std::to_string(out.channels) + " do not fit together"};
    if (b.rows > INT32_MAX) throw Refused{PyExc_ValueError, "too many rows of weights"};
}

int matmul_quantized(PyObject* const* o)         // a, a_scale, b, b_scale, bias, out, relu, stream
{
    const at::Tensor *a = tensor(o[0], "a"), *as = tensor(o[1], "a_scale", true), *b = tensor(o[2], "b"), *bs = tensor(o[3], "b_scale", true), *bias = tensor(o[4], "bias", true),
                     *out = tensor(o[5], "out");
    const Rows ar = rows_of(*a, "a", true), br = rows_of(*b, "b", true), r = rows_of(*out, "out");
    fit(ar, br, r);
    const float *sa = vector_of(as, ar.rows, "a_scale", false), *sb = vector_of(bs, br.rows, "b_scale", false), *c = vector_of(bias, br.rows, "bias");
    const int relu = truth(o[6]);
    const Place p("dc_matmul_quantized", {a, b, as, bs, bias, out}, o[7]);
    const WithoutGil call;
    return dc_matmul_quantized((const int8_t*)ar.at, ar.pitch, sa, (const int8_t*)br.at, br.pitch, sb, c, ar.rows, (int32_t)br.rows, channels_of(ar), relu, r.dtype, r.at, r.pitch,
                               p.stream);
}

int linear_quantized(PyObject* const* o)         // x, w, w_scale, bias, out, relu, workspace, stream
{
    const at::Tensor *x = tensor(o[0], "x"), *w = tensor(o[1], "w"), *ws = tensor(o[2], "w_scale", true), *bias = tensor(o[3], "bias", true), *out = tensor(o[4], "out"),
                     *work = tensor(o[6], "workspace", true);
    const Rows xr = rows_of(*x, "x"), wr = rows_of(*w, "w", true), r = rows_of(*out, "out");
    fit(xr, wr, r);
    if (xr.dtype != r.dtype) throw Refused{PyExc_TypeError, "x and out differ in type"};
    if (work && !work->is_contiguous()) throw Refused{PyExc_ValueError, "workspace: has to be contiguous"};
    const float *sw = vector_of(ws, wr.rows, "w_scale", false), *c = vector_of(bias, wr.rows, "bias");
    const int relu = truth(o[5]);
    const Place p("dc_linear_quantized", {x, w, ws, bias, out, work}, o[7]);
    const WithoutGil call;
    return dc_linear_quantized(xr.at, xr.pitch, (const int8_t*)wr.at, wr.pitch, sw, c, xr.rows, (int32_t)wr.rows, channels_of(xr), relu, xr.dtype, r.at, r.pitch,
                               work ? work->data_ptr() : nullptr, work ? work->nbytes() : 0, p.stream);
}

// ---- group normalisation, 8-bit floating point ----
// [maps, ..., channels]: the first dimension counts images, the last one channels.
int64_t maps_of(const at::Tensor& t, const char* what)
{
    if (t.dim() < 2) throw Refused{PyExc_ValueError, std::string(what) + ": [maps, ..., channels] is needed"};
    return t.size(0);
}
int64_t pixels_of(const at::Tensor& t)
{
    int64_t n = 1;
    for (int64_t d = 1; d < t.dim() - 1; ++d) n *= t.size(d);
    return n;
}
int32_t count(PyObject* o, const char* what)
{
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) throw Refused{nullptr, ""};
    if (v < INT32_MIN || v > INT32_MAX) throw Refused{PyExc_ValueError, std::string(what) + " is out of range"};
    return (int32_t)v;
}
int64_t ceil_of(int64_t a, int64_t b) { return (a + b - 1) / b; }
// Rows of e4m3.
Rows bytes_of(const at::Tensor& t, const char* what)
{
    if (t.scalar_type() != at::kFloat8_e4m3fn && t.scalar_type() != at::kByte)
        throw Refused{PyExc_TypeError, std::string(what) + ": unsupported type " + c10::toString(t.scalar_type()) + " (float8_e4m3fn, or uint8 that holds its bits)"};
    if (t.dim() != 2) throw Refused{PyExc_ValueError, std::string(what) + ": two dimensions are needed"};
    Rows r;
    r.rows = t.size(0); r.channels = t.size(1); r.at = t.data_ptr();
    if (r.channels > 1 && t.stride(1) != 1) throw Refused{PyExc_ValueError, std::string(what) + ": a row's elements have to lie side by side"};
    r.pitch = r.rows > 1 ? (size_t)t.stride(0) : (size_t)((r.channels + 15) / 16 * 16);
    return r;
}
float* table_of(const at::Tensor* t, int64_t rows, int64_t columns, const char* what)
{
    if (!t) return nullptr;
    if (t->scalar_type() != at::kFloat || t->dim() != 2 || t->size(0) != rows || t->size(1) != columns || !t->is_contiguous())
        throw Refused{PyExc_ValueError, std::string(what) + ": a contiguous float32 tensor [" + std::to_string(rows) + ", " + std::to_string(columns) + "] is needed"};
    return (float*)t->data_ptr();
}
// Scales of b: for 128 of its rows, or for each.  (The same for a single row.)
int32_t block_rows_of(const at::Tensor* t, int64_t rows, int64_t blocks, const char* what, float** at)
{
    if (!t) throw Refused{PyExc_ValueError, std::string(what) + " is needed"};
    const bool each = t->dim() == 2 && t->size(0) == rows && rows != ceil_of(rows, 128);
    *at = table_of(t, each ? rows : ceil_of(rows, 128), blocks, what);
    return each ? 1 : 128;
}
void whole(const at::Tensor* work)
{
    if (work && !work->is_contiguous()) throw Refused{PyExc_ValueError, "workspace: has to be contiguous"};
}

int group_norm(PyObject* const* o)       // x, groups, gamma, beta, y, mean, rstd, activation, eps, workspace, stream
{
    const at::Tensor *x = tensor(o[0], "x"), *gamma = tensor(o[2], "gamma", true), *beta = tensor(o[3], "beta", true), *y = tensor(o[4], "y"), *mean = tensor(o[5], "mean", true),
                     *rstd = tensor(o[6], "rstd", true), *work = tensor(o[9], "workspace", true);
    const int32_t groups = count(o[1], "groups"), activation = count(o[7], "activation");
    const Rows xr = rows_of(*x, "x"), yr = rows_of(*y, "y");
    same(xr, yr, "y");
    const int64_t maps = maps_of(*x, "x"), pixels = pixels_of(*x);
    const float *g = vector_of(gamma, xr.channels, "gamma"), *b = vector_of(beta, xr.channels, "beta");
    float *m = vector_of(mean, maps * groups, "mean"), *r = vector_of(rstd, maps * groups, "rstd");
    whole(work);
    const double eps = number(o[8]);
    const Place p("dc_group_norm", {x, y, gamma, beta, mean, rstd, work}, o[10]);
    const WithoutGil call;
    return dc_group_norm(xr.at, xr.pitch, g, b, maps, pixels, channels_of(xr), groups, eps, activation, xr.dtype, yr.at, yr.pitch, m, r, work ? work->data_ptr() : nullptr,
                         work ? work->nbytes() : 0, p.stream);
}

int group_norm_backward(PyObject* const* o)      // dy, x, groups, gamma, beta, mean, rstd, dx, dgamma, dbeta, activation, workspace, stream
{
    const at::Tensor *dy = tensor(o[0], "dy"), *x = tensor(o[1], "x"), *gamma = tensor(o[3], "gamma", true), *beta = tensor(o[4], "beta", true), *mean = tensor(o[5], "mean", true),
                     *rstd = tensor(o[6], "rstd", true), *dx = tensor(o[7], "dx", true), *dgamma = tensor(o[8], "dgamma", true), *dbeta = tensor(o[9], "dbeta", true),
                     *work = tensor(o[11], "workspace", true);
    const int32_t groups = count(o[2], "groups"), activation = count(o[10], "activation");
    const Rows xr = rows_of(*x, "x"), dr = rows_of(*dy, "dy");
    same(xr, dr, "dy");
    Rows ox;
    if (dx) { ox = rows_of(*dx, "dx"); same(xr, ox, "dx"); }
    const int64_t maps = maps_of(*x, "x"), pixels = pixels_of(*x);
    const float *g = vector_of(gamma, xr.channels, "gamma"), *b = vector_of(beta, xr.channels, "beta"), *m = vector_of(mean, maps * groups, "mean", false),
                *r = vector_of(rstd, maps * groups, "rstd", false);
    float *dg = vector_of(dgamma, xr.channels, "dgamma"), *db = vector_of(dbeta, xr.channels, "dbeta");
    whole(work);
    const Place p("dc_group_norm_backward", {x, dy, gamma, beta, mean, rstd, dx, dgamma, dbeta, work}, o[12]);
    const WithoutGil call;
    return dc_group_norm_backward(dr.at, dr.pitch, xr.at, xr.pitch, g, b, m, r, maps, pixels, channels_of(xr), groups, activation, xr.dtype, ox.at, ox.pitch, dg, db,
                                  work ? work->data_ptr() : nullptr, work ? work->nbytes() : 0, p.stream);
}

int quantize_blocks(PyObject* const* o)  // x, q, scale, q_t, scale_t, block_rows, stream
{
    const at::Tensor *x = tensor(o[0], "x"), *q = tensor(o[1], "q", true), *scale = tensor(o[2], "scale", true), *qt = tensor(o[3], "q_t", true), *scale_t = tensor(o[4], "scale_t", true);
    const int32_t block = count(o[5], "block_rows");
    const Rows xr = rows_of(*x, "x");
    const int64_t by = block == 128 ? 128 : 1;
    Rows qr, tr;
    if (q) { qr = bytes_of(*q, "q"); same(xr, qr, "q", false); }
    if (qt) {
        tr = bytes_of(*qt, "q_t");
        if (tr.rows != xr.channels || tr.channels != xr.rows)
            throw Refused{PyExc_ValueError, "q_t: [" + std::to_string(xr.channels) + ", " + std::to_string(xr.rows) + "] is needed"};
    }
    float *s = table_of(scale, ceil_of(xr.rows, by), ceil_of(xr.channels, 128), "scale"), *st = table_of(scale_t, ceil_of(xr.channels, by), ceil_of(xr.rows, 128), "scale_t");
    const Place p("dc_quantize_blocks", {x, q, scale, qt, scale_t}, o[6]);
    const WithoutGil call;
    return dc_quantize_blocks(xr.at, xr.pitch, xr.rows, channels_of(xr), xr.dtype, block, (uint8_t*)qr.at, qr.pitch, s, (uint8_t*)tr.at, tr.pitch, st, p.stream);
}

int matmul_blocks(PyObject* const* o)    // a, a_scale, b, b_scale, bias, out, relu, stream
{
    const at::Tensor *a = tensor(o[0], "a"), *as = tensor(o[1], "a_scale"), *b = tensor(o[2], "b"), *bs = tensor(o[3], "b_scale"), *bias = tensor(o[4], "bias", true), *out = tensor(o[5], "out");
    const Rows ar = bytes_of(*a, "a"), br = bytes_of(*b, "b"), r = rows_of(*out, "out");
    fit(ar, br, r);
    const int64_t blocks = ceil_of(ar.channels, 128);
    float* sb;
    const float *sa = table_of(as, ar.rows, blocks, "a_scale"), *c = vector_of(bias, br.rows, "bias");
    const int32_t by = block_rows_of(bs, br.rows, blocks, "b_scale", &sb);
    const int relu = truth(o[6]);
    const Place p("dc_matmul_blocks", {a, b, as, bs, bias, out}, o[7]);
    const WithoutGil call;
    return dc_matmul_blocks((const uint8_t*)ar.at, ar.pitch, sa, (const uint8_t*)br.at, br.pitch, sb, by, c, ar.rows, (int32_t)br.rows, channels_of(ar), relu, r.dtype, r.at, r.pitch, p.stream);
}

int linear_blocks(PyObject* const* o)    // x, w, w_scale, bias, out, relu, workspace, stream
{
    const at::Tensor *x = tensor(o[0], "x"), *w = tensor(o[1], "w"), *ws = tensor(o[2], "w_scale"), *bias = tensor(o[3], "bias", true), *out = tensor(o[4], "out"),
                     *work = tensor(o[6], "workspace", true);
    const Rows xr = rows_of(*x, "x"), wr = bytes_of(*w, "w"), r = rows_of(*out, "out");
    fit(xr, wr, r);
    if (xr.dtype != r.dtype) throw Refused{PyExc_TypeError, "x and out differ in type"};
    whole(work);
    float* sw;
    const int32_t by = block_rows_of(ws, wr.rows, ceil_of(wr.channels, 128), "w_scale", &sw);
    const float* c = vector_of(bias, wr.rows, "bias");
    const int relu = truth(o[5]);
    const Place p("dc_linear_blocks", {x, w, ws, bias, out, work}, o[7]);
    const WithoutGil call;
    return dc_linear_blocks(xr.at, xr.pitch, (const uint8_t*)wr.at, wr.pitch, sw, by, c, xr.rows, (int32_t)wr.rows, channels_of(xr), relu, xr.dtype, r.at, r.pitch,
                            work ? work->data_ptr() : nullptr, work ? work->nbytes() : 0, p.stream);
}

// Every function returns the call's status; nothing is thrown into Python.
template <int (*CALL)(PyObject* const*), int N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (n != N) { PyErr_Format(PyExc_TypeError, "%d arguments are needed, not %zd", N, n); return nullptr; }
    try {
        return PyLong_FromLong(CALL(args));
    } catch (const Refused& r) {
        if (r.type) PyErr_SetString(r.type, r.what.c_str());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown error");
    }
    return nullptr;
}

#define DC_ENTRY(name, n) {#name, (PyCFunction)(void (*)(void))entry<name, n>, METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {DC_ENTRY(layer_norm, 8), DC_ENTRY(layer_norm_backward, 10), DC_ENTRY(quantize_rows, 4), DC_ENTRY(layer_norm_quantize, 8),
                          DC_ENTRY(matmul_quantized, 8), DC_ENTRY(linear_quantized, 8),
                          DC_ENTRY(group_norm, 11), DC_ENTRY(group_norm_backward, 13), DC_ENTRY(quantize_blocks, 7), DC_ENTRY(matmul_blocks, 8), DC_ENTRY(linear_blocks, 8), {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_tensors", "Torch tensors to libdeepcache's entry points on maps of the caller's own.  " DC_BUILT_FOR, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors(void) { return PyModule_Create(&kModule); }
