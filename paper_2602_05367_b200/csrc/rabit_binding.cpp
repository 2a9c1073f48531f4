// The Python side of the hot calls, in native code: argument checks, output allocation, the current stream and the call
// into the C ABI, without the interpreter's and ctypes' cost per call.  At batch 1 a layer lasts two to seven
// microseconds on the device; the same steps in Python took 10.6 us per rabit_linear call (torch.empty 2.5,
// torch.cuda.current_stream 2.3, the ctypes call 3.3 of which the launch is most, the rest attribute look-ups), so an
// eager decoder was bound by its host.
//
// The module calls the library through addresses handed to init(), so that it serves whichever build of librabit.so the
// package has loaded.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/Functions.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include <cstdint>
#include <vector>

#include "../../include/rabit.h"

namespace {

typedef int (*LinearFn)(const void*, const void*, void*, int, void*);
typedef int (*GroupFn)(const void* const*, const void* const*, void* const*, int, int, void*);
typedef int (*GroupHostFn)(const void* const*, const void* const*, void* const*, int, int, void*, size_t, void*);
typedef int (*AdaptedFn)(const void*, const rabit_adapters*, const void*, const int*, void*, float*, int, void*);
typedef int (*GroupAdaptedFn)(const void* const*, const rabit_adapters* const*, const void* const*, const int*, void* const*, float* const*, int, int, void*);
typedef int (*FactorFn)(const rabit_adapters*, const void*, const float*, const void*, const float*, const int*, float*, float*, int, int, void*);
typedef int (*ClipFn)(const void*, float, float*, void*);
typedef int (*DimFn)(const void*);
typedef const char* (*ErrorFn)();

LinearFn p_linear = nullptr;
GroupFn p_group = nullptr;
GroupHostFn p_group_host = nullptr;
AdaptedFn p_adapted = nullptr;
GroupAdaptedFn p_group_adapted = nullptr;
FactorFn p_factor = nullptr;
ClipFn p_clip = nullptr;
DimFn p_M = nullptr, p_N = nullptr;
ErrorFn p_error = nullptr;
PyObject* g_error_type = nullptr;      // RabitError
// Names of the attributes that hold addresses for this module, one for each class, so that no object is taken for one of another class:
PyObject* g_layer_name = nullptr;      // "_layer_addr": the descriptor's address on a RabitLayer, None once freed
PyObject* g_addr_name = nullptr;       // "_addr": that of its rabit_adapters on a RabitAdapters
PyObject* g_gradients_name = nullptr;  // "_gradients_addr": the descriptor's on a RabitGradients, None once freed

PyObject* g_buf_name = nullptr;        // "dev_buf": the device memory of a RabitGradients
PyObject* g_device_name = nullptr;     // "_device": the index of the device that a RabitAdapters or RabitGradients lives on

constexpr Py_ssize_t kInline = 16;     // layers of a group whose pointers need no allocation

PyObject* raise_code(int code, const char* msg) {
    PyObject* args = Py_BuildValue("(is)", code, msg);
    if (args) {
        PyErr_SetObject(g_error_type, args);          // the type is called with (code, message)
        Py_DECREF(args);
    }
    return nullptr;
}

// the address under `name`, which objects of the class `what` have; nullptr with an exception set if it has none
void* address_of(PyObject* o, PyObject* name, const char* what) {
    PyObject* a = PyObject_GetAttr(o, name);
    if (!a) {
        if (PyErr_ExceptionMatches(PyExc_AttributeError)) PyErr_Format(PyExc_TypeError, "a %s is needed, not a %s", what, Py_TYPE(o)->tp_name);
        return nullptr;
    }
    void* p = nullptr;
    if (a == Py_None) raise_code(RABIT_INVALID_ARG, "already freed");
    else p = PyLong_AsVoidPtr(a);
    Py_DECREF(a);
    return p;
}
void* layer_handle(PyObject* o) { return address_of(o, g_layer_name, "RabitLayer"); }
const rabit_adapters* adapters_of(PyObject* o) { return (const rabit_adapters*)address_of(o, g_addr_name, "RabitAdapters"); }

// stream argument: an integer, or None for torch's current stream on that device
bool stream_of(PyObject* arg, c10::DeviceIndex device, void** out) {
    if (arg == Py_None) {
        *out = (void*)c10::cuda::getCurrentCUDAStream(device).stream();
        return true;
    }
    *out = PyLong_AsVoidPtr(arg);
    return !(*out == nullptr && PyErr_Occurred());
}

c10::cuda::CUDAStream torch_stream(void* stream, c10::DeviceIndex device) {
    if (stream == (void*)cudaStreamLegacy) stream = nullptr;                    // (another name of the default stream, which is no address)
    return c10::cuda::getStreamFromExternal((cudaStream_t)stream, device);
}

// Memory that a call on `stream` makes comes from the allocator's pool of that stream: a block of another stream's pool may still be in use by work that is
// pending there.  What the caller gets is recorded for torch's current stream as well, on which it is likely to be used.
at::Tensor empty_on(at::IntArrayRef sizes, at::ScalarType type, c10::DeviceIndex device, void* stream, bool returned) {
    const at::TensorOptions options = at::TensorOptions().dtype(type).device(at::kCUDA, device);
    const c10::cuda::CUDAStream current = c10::cuda::getCurrentCUDAStream(device);
    if (stream == (void*)current.stream()) return at::empty(sizes, options);
    c10::cuda::CUDAStreamGuard guard(torch_stream(stream, device));
    at::Tensor t = at::empty(sizes, options);
    if (returned) t.record_stream(current.unwrap());
    return t;
}

inline bool is_cuda_half(PyObject* o) {
    if (!THPVariable_Check(o)) return false;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.scalar_type() == at::kHalf && t.is_cuda() && t.is_contiguous();
}

// linear(layer, x, y | None, stream | None) -> y
PyObject* linear(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (nargs != 4) return PyErr_Format(PyExc_TypeError, "linear takes 4 arguments");
    HANDLE_TH_ERRORS
    if (!is_cuda_half(args[1])) return PyErr_Format(PyExc_ValueError, "x must be a contiguous CUDA float16 tensor");
    const void* h = layer_handle(args[0]);
    if (!h) return nullptr;
    const at::Tensor& x = THPVariable_Unpack(args[1]);
    const int64_t M = p_M(h), N = p_N(h);
    const bool flat = x.dim() != 2;
    const int64_t batch = flat ? 1 : x.size(0), cols = flat ? x.numel() : x.size(1);
    if (cols != N) return PyErr_Format(PyExc_ValueError, "x has %lld columns, layer expects %lld", (long long)cols, (long long)N);
    at::Tensor made;
    void *yp, *stream;
    if (!stream_of(args[3], x.device().index(), &stream)) return nullptr;
    if (args[2] == Py_None) {
        made = empty_on({batch, M}, at::kHalf, x.device().index(), stream, true);
        yp = made.data_ptr();
    } else {
        if (!is_cuda_half(args[2]) || THPVariable_Unpack(args[2]).numel() != batch * M)
            return PyErr_Format(PyExc_ValueError, "y must be a contiguous CUDA float16 tensor of batch*M elements");
        yp = THPVariable_Unpack(args[2]).data_ptr();
    }
    const void* xp = x.data_ptr();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = p_linear(h, xp, yp, (int)batch, stream);
    Py_END_ALLOW_THREADS
    if (rc != 0) return raise_code(rc, p_error());
    if (args[2] == Py_None) return THPVariable_Wrap(flat ? made.view({-1}) : made);
    if (flat) return THPVariable_Wrap(THPVariable_Unpack(args[2]).view({-1}));
    Py_INCREF(args[2]);
    return args[2];
    END_HANDLE_TH_ERRORS
}

// linear_group(layers, xs, ys, stream | None) -> ys
PyObject* linear_group(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (nargs != 4) return PyErr_Format(PyExc_TypeError, "linear_group takes 4 arguments");
    HANDLE_TH_ERRORS
    THPObjectPtr ls(PySequence_Fast(args[0], "layers must be a sequence")), xs(PySequence_Fast(args[1], "xs must be a sequence")),
        ys(PySequence_Fast(args[2], "ys must be a sequence"));
    if (!ls || !xs || !ys) return nullptr;
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(ls.get());
    if (n < 1 || PySequence_Fast_GET_SIZE(xs.get()) != n || PySequence_Fast_GET_SIZE(ys.get()) != n)
        return PyErr_Format(PyExc_ValueError, "layers, xs and ys must have the same, non-zero length");
    void* inl[3 * kInline];
    std::vector<void*> more;
    void** hp = inl;
    if (n > kInline) {
        more.resize(3 * (size_t)n);
        hp = more.data();
    }
    void **xp = hp + n, **yp = hp + 2 * n;
    int64_t batch = 0;
    c10::DeviceIndex device = 0;
    for (Py_ssize_t l = 0; l < n; ++l) {
        PyObject *xo = PySequence_Fast_GET_ITEM(xs.get(), l), *yo = PySequence_Fast_GET_ITEM(ys.get(), l);
        hp[l] = layer_handle(PySequence_Fast_GET_ITEM(ls.get(), l));
        if (!hp[l]) return nullptr;
        if (l == 0 && THPVariable_Check(xo)) {
            const at::Tensor& x0 = THPVariable_Unpack(xo);
            batch = x0.dim() == 1 ? 1 : x0.dim() > 0 ? x0.size(0) : 0;
            device = x0.device().index();
        }
        if (!is_cuda_half(xo) || THPVariable_Unpack(xo).numel() != batch * p_N(hp[l]))
            return PyErr_Format(PyExc_ValueError, "every x must be a contiguous CUDA float16 tensor of batch*N elements");
        if (!is_cuda_half(yo) || THPVariable_Unpack(yo).numel() != batch * p_M(hp[l]))
            return PyErr_Format(PyExc_ValueError, "every y must be a contiguous CUDA float16 tensor of batch*M elements");
        xp[l] = THPVariable_Unpack(xo).data_ptr();
        yp[l] = THPVariable_Unpack(yo).data_ptr();
    }
    void* stream;
    if (!stream_of(args[3], device, &stream)) return nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = p_group(hp, xp, yp, (int)n, (int)batch, stream);
    Py_END_ALLOW_THREADS
    if (rc != 0) return raise_code(rc, p_error());
    Py_INCREF(args[2]);
    return args[2];
    END_HANDLE_TH_ERRORS
}

// the device of a RabitAdapters or RabitGradients; -1 with an exception set if it has none
long device_of(PyObject* o) {
    THPObjectPtr d(PyObject_GetAttr(o, g_device_name));
    return d ? PyLong_AsLong(d.get()) : -1;
}
const rabit_adapters* adapters_on(PyObject* o, c10::DeviceIndex device) {
    const rabit_adapters* A = adapters_of(o);
    if (!A) return nullptr;
    const long d = device_of(o);
    if (d == -1 && PyErr_Occurred()) return nullptr;
    if (d == device) return A;
    PyErr_Format(PyExc_ValueError, "the adapters live on device %ld, the activations on device %d", d, (int)device);
    return nullptr;
}

// What the rows' adapters and low-rank products need: ids [batch] int32 and u [batch][rank] fp32 on the activations' device.
inline bool is_cuda(PyObject* o, at::ScalarType type, int64_t n, c10::DeviceIndex device) {
    if (!THPVariable_Check(o)) return false;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.scalar_type() == type && t.is_cuda() && t.is_contiguous() && t.numel() == n && t.device().index() == device;
}

// linear_adapted(layer, adapters, x, ids, y | None, u | None, stream | None) -> y
PyObject* linear_adapted(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (nargs != 7) return PyErr_Format(PyExc_TypeError, "linear_adapted takes 7 arguments");
    HANDLE_TH_ERRORS
    if (!is_cuda_half(args[2])) return PyErr_Format(PyExc_ValueError, "x must be a contiguous CUDA float16 tensor");
    const void* h = layer_handle(args[0]);
    if (!h) return nullptr;
    const at::Tensor& x = THPVariable_Unpack(args[2]);
    const rabit_adapters* A = adapters_on(args[1], x.device().index());
    if (!A) return nullptr;
    const int64_t M = p_M(h), N = p_N(h);
    const bool flat = x.dim() != 2;
    const int64_t batch = flat ? 1 : x.size(0), cols = flat ? x.numel() : x.size(1);
    const c10::DeviceIndex device = x.device().index();
    if (cols != N) return PyErr_Format(PyExc_ValueError, "x has %lld columns, layer expects %lld", (long long)cols, (long long)N);
    if (!is_cuda(args[3], at::kInt, batch, device)) return PyErr_Format(PyExc_ValueError, "ids must be a contiguous CUDA int32 tensor of batch elements on the device of x");
    at::Tensor made, made_u;
    void *yp, *stream;
    if (!stream_of(args[6], device, &stream)) return nullptr;
    if (args[4] == Py_None) {
        made = empty_on({batch, M}, at::kHalf, device, stream, true);
        yp = made.data_ptr();
    } else {
        if (!is_cuda(args[4], at::kHalf, batch * M, device)) return PyErr_Format(PyExc_ValueError, "y must be a contiguous CUDA float16 tensor of batch*M elements on the device of x");
        yp = THPVariable_Unpack(args[4]).data_ptr();
    }
    float* up;
    if (args[5] == Py_None) {
        made_u = empty_on({batch, A->rank}, at::kFloat, device, stream, false);
        up = made_u.data_ptr<float>();
    } else {
        if (!is_cuda(args[5], at::kFloat, batch * A->rank, device)) return PyErr_Format(PyExc_ValueError, "u must be a contiguous CUDA float32 tensor of batch*rank elements on the device of x");
        up = THPVariable_Unpack(args[5]).data_ptr<float>();
    }
    const void* xp = x.data_ptr();
    const int* ip = THPVariable_Unpack(args[3]).data_ptr<int>();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = batch > INT32_MAX ? RABIT_INVALID_ARG : p_adapted(h, A, xp, ip, yp, up, (int)batch, stream);
    Py_END_ALLOW_THREADS
    if (rc != 0) return raise_code(rc, batch > INT32_MAX ? "batch too large" : p_error());
    if (args[4] == Py_None) return THPVariable_Wrap(flat ? made.view({-1}) : made);
    if (flat) return THPVariable_Wrap(THPVariable_Unpack(args[4]).view({-1}));
    Py_INCREF(args[4]);
    return args[4];
    END_HANDLE_TH_ERRORS
}

// linear_group_adapted(layers, adapters (None: that layer has none), xs, ids, ys, us | None (an entry may be None), stream | None) -> ys
PyObject* linear_group_adapted(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (nargs != 7) return PyErr_Format(PyExc_TypeError, "linear_group_adapted takes 7 arguments");
    HANDLE_TH_ERRORS
    THPObjectPtr ls(PySequence_Fast(args[0], "layers must be a sequence")), as(PySequence_Fast(args[1], "adapters must be a sequence")),
        xs(PySequence_Fast(args[2], "xs must be a sequence")), ys(PySequence_Fast(args[4], "ys must be a sequence"));
    if (!ls || !as || !xs || !ys) return nullptr;
    THPObjectPtr us(args[5] == Py_None ? nullptr : PySequence_Fast(args[5], "us must be a sequence or None"));
    if (!us && args[5] != Py_None) return nullptr;
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(ls.get());
    if (n < 1 || PySequence_Fast_GET_SIZE(as.get()) != n || PySequence_Fast_GET_SIZE(xs.get()) != n || PySequence_Fast_GET_SIZE(ys.get()) != n || (us && PySequence_Fast_GET_SIZE(us.get()) != n))
        return PyErr_Format(PyExc_ValueError, "layers, adapters, xs, ys and us must have the same, non-zero length");
    void* inl[5 * kInline];
    std::vector<void*> more;
    std::vector<at::Tensor> made;
    void** hp = inl;
    if (n > kInline) {
        more.resize(5 * (size_t)n);
        hp = more.data();
    }
    void **xp = hp + n, **yp = hp + 2 * n, **ap = hp + 3 * n, **up = hp + 4 * n;
    int64_t batch = 0;
    c10::DeviceIndex device = 0;
    void* stream = nullptr;
    for (Py_ssize_t l = 0; l < n; ++l) {
        PyObject *xo = PySequence_Fast_GET_ITEM(xs.get(), l), *yo = PySequence_Fast_GET_ITEM(ys.get(), l), *ao = PySequence_Fast_GET_ITEM(as.get(), l);
        PyObject* uo = us ? PySequence_Fast_GET_ITEM(us.get(), l) : Py_None;
        hp[l] = layer_handle(PySequence_Fast_GET_ITEM(ls.get(), l));
        if (!hp[l]) return nullptr;
        ap[l] = up[l] = nullptr;
        if (l == 0) {
            if (!THPVariable_Check(xo) || !THPVariable_Unpack(xo).is_cuda()) return PyErr_Format(PyExc_ValueError, "every x must be a contiguous CUDA float16 tensor of batch*N elements");
            const at::Tensor& x0 = THPVariable_Unpack(xo);
            batch = x0.dim() == 1 ? 1 : x0.dim() > 0 ? x0.size(0) : 0;
            device = x0.device().index();
            if (!stream_of(args[6], device, &stream)) return nullptr;
        }
        if (ao != Py_None && !(ap[l] = (void*)adapters_on(ao, device))) return nullptr;
        if (!is_cuda(xo, at::kHalf, batch * p_N(hp[l]), device)) return PyErr_Format(PyExc_ValueError, "every x must be a contiguous CUDA float16 tensor of batch*N elements, all on one device");
        if (!is_cuda(yo, at::kHalf, batch * p_M(hp[l]), device)) return PyErr_Format(PyExc_ValueError, "every y must be a contiguous CUDA float16 tensor of batch*M elements, all on one device");
        xp[l] = THPVariable_Unpack(xo).data_ptr();
        yp[l] = THPVariable_Unpack(yo).data_ptr();
        if (!ap[l]) continue;
        const int64_t rank = ((const rabit_adapters*)ap[l])->rank;
        if (uo == Py_None) {
            made.push_back(empty_on({batch, rank}, at::kFloat, device, stream, false));
            up[l] = made.back().data_ptr();
        } else {
            if (!is_cuda(uo, at::kFloat, batch * rank, device)) return PyErr_Format(PyExc_ValueError, "every u must be a contiguous CUDA float32 tensor of batch*rank elements, all on one device");
            up[l] = THPVariable_Unpack(uo).data_ptr();
        }
    }
    if (!is_cuda(args[3], at::kInt, batch, device)) return PyErr_Format(PyExc_ValueError, "ids must be a contiguous CUDA int32 tensor of batch elements on the device of the xs");
    const int* ip = THPVariable_Unpack(args[3]).data_ptr<int>();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = batch > INT32_MAX ? RABIT_INVALID_ARG : p_group_adapted(hp, (const rabit_adapters* const*)ap, xp, ip, yp, (float* const*)up, (int)n, (int)batch, stream);
    Py_END_ALLOW_THREADS
    if (rc != 0) return raise_code(rc, batch > INT32_MAX ? "batch too large" : p_error());
    Py_INCREF(args[4]);
    return args[4];
    END_HANDLE_TH_ERRORS
}

// adapter_gradients(adapters, x, u, dy, p, ids, da | None, db | None, accumulate, stream | None) -> (da, db)
PyObject* adapter_gradients(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (nargs != 10) return PyErr_Format(PyExc_TypeError, "adapter_gradients takes 10 arguments");
    HANDLE_TH_ERRORS
    const rabit_adapters* A = adapters_of(args[0]);
    if (!A) return nullptr;
    const long d = device_of(args[0]);
    if (d == -1 && PyErr_Occurred()) return nullptr;
    const c10::DeviceIndex device = (c10::DeviceIndex)d;
    const int64_t batch = THPVariable_Check(args[5]) ? THPVariable_Unpack(args[5]).numel() : 0;
    struct { int at; const char* name; at::ScalarType type; int64_t n; } want[] = {
        {5, "ids", at::kInt, batch}, {1, "x", at::kHalf, batch * A->n_in}, {2, "u", at::kFloat, batch * A->rank}, {3, "dy", at::kHalf, batch * A->n_out}, {4, "p", at::kFloat, batch * A->rank},
        {6, "da", at::kFloat, (int64_t)A->count * A->rank * A->n_in}, {7, "db", at::kFloat, (int64_t)A->count * A->rank * A->n_out}};
    for (const auto& w : want)
        if (!(w.at >= 6 && args[w.at] == Py_None) && !is_cuda(args[w.at], w.type, w.n, device))
            return PyErr_Format(PyExc_ValueError, "%s must be a contiguous CUDA %s tensor of %lld elements on the adapters' device", w.name, w.type == at::kHalf ? "float16" : w.type == at::kInt ? "int32" : "float32", (long long)w.n);
    const int accumulate = PyObject_IsTrue(args[8]);
    if (accumulate < 0) return nullptr;
    if (accumulate && (args[6] == Py_None || args[7] == Py_None)) return PyErr_Format(PyExc_ValueError, "accumulate needs da and db");
    void* stream;
    if (!stream_of(args[9], device, &stream)) return nullptr;
    if (batch > INT32_MAX) return raise_code(RABIT_INVALID_ARG, "batch too large");
    c10::cuda::CUDAGuard guard(device);
    THPObjectPtr made[2];
    float* out[2];
    for (int i = 0; i < 2; ++i) {
        if (args[6 + i] == Py_None) made[i] = THPVariable_Wrap(empty_on({A->count, A->rank, i == 0 ? A->n_in : A->n_out}, at::kFloat, device, stream, true));
        else made[i] = Py_NewRef(args[6 + i]);
        out[i] = THPVariable_Unpack(made[i].get()).data_ptr<float>();
    }
    auto ptr = [&](int i) { return THPVariable_Unpack(args[i]).data_ptr(); };
    const void *x = ptr(1), *dy = ptr(3);
    const float *u = (const float*)ptr(2), *p = (const float*)ptr(4);
    const int* ids = (const int*)ptr(5);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = p_factor(A, x, u, dy, p, ids, out[0], out[1], (int)batch, accumulate, stream);
    Py_END_ALLOW_THREADS
    if (rc != 0) return raise_code(rc, p_error());
    return PyTuple_Pack(2, made[0].get(), made[1].get());
    END_HANDLE_TH_ERRORS
}

// clip(gradients, max_norm, norm | None, stream | None) -> norm
PyObject* clip(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (nargs != 4) return PyErr_Format(PyExc_TypeError, "clip takes 4 arguments");
    HANDLE_TH_ERRORS
    const void* h = address_of(args[0], g_gradients_name, "RabitGradients");
    if (!h) return nullptr;
    const long d = device_of(args[0]);
    if (d == -1 && PyErr_Occurred()) return nullptr;
    const c10::DeviceIndex device = (c10::DeviceIndex)d;
    const double max_norm = PyFloat_AsDouble(args[1]);
    if (max_norm == -1.0 && PyErr_Occurred()) return nullptr;
    if (args[2] != Py_None && !is_cuda(args[2], at::kFloat, 1, device)) return PyErr_Format(PyExc_ValueError, "norm must be a CUDA float32 tensor of one element on the gradients' device");
    void* stream;
    if (!stream_of(args[3], device, &stream)) return nullptr;
    c10::cuda::CUDAGuard guard(device);
    THPObjectPtr norm(args[2] == Py_None ? THPVariable_Wrap(empty_on({1}, at::kFloat, device, stream, true)) : Py_NewRef(args[2]));
    float* out = THPVariable_Unpack(norm.get()).data_ptr<float>();
    // the table and the partial sums belong to the RabitGradients, which may be freed before the stream has come this far
    THPObjectPtr buf(PyObject_GetAttr(args[0], g_buf_name));
    if (!buf) return nullptr;
    if (THPVariable_Check(buf.get()))                     // (past the dispatcher, which takes a microsecond)
        c10::cuda::CUDACachingAllocator::recordStream(THPVariable_Unpack(buf.get()).storage().data_ptr(), torch_stream(stream, device));
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = p_clip(h, (float)max_norm, out, stream);
    Py_END_ALLOW_THREADS
    if (rc != 0) return raise_code(rc, p_error());
    return norm.release();
    END_HANDLE_TH_ERRORS
}

// group_host((layers*, xs*, ys*, n, batch, stage*, stage bytes, device), stream | None): a call whose arrays were laid out before
PyObject* group_host(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (nargs != 2 || !PyTuple_Check(args[0]) || PyTuple_GET_SIZE(args[0]) != 8) return PyErr_Format(PyExc_TypeError, "group_host takes a prepared tuple and a stream");
    HANDLE_TH_ERRORS
    void* v[8];
    for (int i = 0; i < 8; ++i) v[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(args[0], i));
    if (PyErr_Occurred()) return nullptr;
    void* stream;
    if (!stream_of(args[1], (c10::DeviceIndex)(intptr_t)v[7], &stream)) return nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = p_group_host((const void* const*)v[0], (const void* const*)v[1], (void* const*)v[2], (int)(intptr_t)v[3], (int)(intptr_t)v[4], v[5],
                      (size_t)v[6], stream);
    Py_END_ALLOW_THREADS
    if (rc != 0) return raise_code(rc, p_error());
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

// current_stream(device index) -> the handle of torch's current stream
PyObject* current_stream(PyObject*, PyObject* arg) {
    HANDLE_TH_ERRORS
    const long d = PyLong_AsLong(arg);
    if (d == -1 && PyErr_Occurred()) return nullptr;
    return PyLong_FromVoidPtr((void*)c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)d).stream());
    END_HANDLE_TH_ERRORS
}

// empty(bytes, device index, stream) -> uint8 tensor for a call on that stream
PyObject* empty_bytes(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (nargs != 3) return PyErr_Format(PyExc_TypeError, "empty takes 3 arguments");
    HANDLE_TH_ERRORS
    const long long n = PyLong_AsLongLong(args[0]);
    const long device = PyLong_AsLong(args[1]);
    void* stream;
    if (PyErr_Occurred() || !stream_of(args[2], (c10::DeviceIndex)device, &stream)) return nullptr;
    return THPVariable_Wrap(empty_on({(int64_t)n}, at::kByte, (c10::DeviceIndex)device, stream, true));
    END_HANDLE_TH_ERRORS
}

// init(error type, address of rabit_linear, _linear_group, _linear_group_host, _layer_M, _layer_N, _last_error, _linear_adapted, _linear_group_adapted,
// _adapter_gradients, _clip_gradients)
PyObject* init(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (nargs != 11) return PyErr_Format(PyExc_TypeError, "init takes 11 arguments");
    void* v[10];
    for (int i = 0; i < 10; ++i) v[i] = PyLong_AsVoidPtr(args[1 + i]);
    if (PyErr_Occurred()) return nullptr;
    p_linear = (LinearFn)v[0];
    p_group = (GroupFn)v[1];
    p_group_host = (GroupHostFn)v[2];
    p_M = (DimFn)v[3];
    p_N = (DimFn)v[4];
    p_error = (ErrorFn)v[5];
    p_adapted = (AdaptedFn)v[6];
    p_group_adapted = (GroupAdaptedFn)v[7];
    p_factor = (FactorFn)v[8];
    p_clip = (ClipFn)v[9];
    Py_XSETREF(g_error_type, Py_NewRef(args[0]));
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"init", (PyCFunction)(void (*)(void))init, METH_FASTCALL, nullptr},
    {"linear", (PyCFunction)(void (*)(void))linear, METH_FASTCALL, nullptr},
    {"linear_group", (PyCFunction)(void (*)(void))linear_group, METH_FASTCALL, nullptr},
    {"linear_adapted", (PyCFunction)(void (*)(void))linear_adapted, METH_FASTCALL, nullptr},
    {"linear_group_adapted", (PyCFunction)(void (*)(void))linear_group_adapted, METH_FASTCALL, nullptr},
    {"adapter_gradients", (PyCFunction)(void (*)(void))adapter_gradients, METH_FASTCALL, nullptr},
    {"clip", (PyCFunction)(void (*)(void))clip, METH_FASTCALL, nullptr},
    {"group_host", (PyCFunction)(void (*)(void))group_host, METH_FASTCALL, nullptr},
    {"empty", (PyCFunction)(void (*)(void))empty_bytes, METH_FASTCALL, nullptr},
    {"current_stream", current_stream, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_rabit_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__rabit_binding(void) {
    g_layer_name = PyUnicode_InternFromString("_layer_addr");
    g_addr_name = PyUnicode_InternFromString("_addr");
    g_gradients_name = PyUnicode_InternFromString("_gradients_addr");
    g_device_name = PyUnicode_InternFromString("_device");
    g_buf_name = PyUnicode_InternFromString("dev_buf");
    return g_layer_name && g_addr_name && g_gradients_name && g_device_name && g_buf_name ? PyModule_Create(&module) : nullptr;
}
