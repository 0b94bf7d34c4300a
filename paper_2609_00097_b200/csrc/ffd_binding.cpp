// Argument checks and calls of the byte cache's and the shared prefix's entry points for ffd.py.
//
// The C functions see addresses only.  What they cannot check is checked here, on torch tensors: dtype, shape, contiguity, one
// device for all.  In Python these checks took 10 us a call, several times what a serving step's kernel takes.
//
// Every function takes the C function's address, the Config, the tensors and numbers in the order of ffd.py's function of that name,
// the workspace and the stream (None: the device's current one), and returns the ffd_status.  A tensor that does not fit raises
// ValueError before anything is called.  The call runs with the workspace's device current and without the interpreter's lock.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <string>

#include "../../include/ffd.h"

namespace {

struct Bad {};   // a Python exception is set

std::string shape_text(c10::IntArrayRef shape) {
    std::string s = "[";
    for (size_t i = 0; i < shape.size(); ++i) s += (i ? ", " : "") + std::to_string(shape[i]);
    return s + "]";
}

[[noreturn]] void refuse(const char* name, const std::string& want, const at::Tensor* got) {
    std::string text = std::string(name) + ": " + want + " is needed";
    if (got)
        text += std::string(", got ") + c10::toString(got->scalar_type()) + " " + shape_text(got->sizes()) + " with strides " +
                shape_text(got->strides()) + " on " + got->device().str();
    PyErr_SetString(PyExc_ValueError, text.c_str());
    throw Bad{};
}

const at::Tensor& tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) refuse(name, "a tensor", nullptr);
    return THPVariable_Unpack(o);
}

// The fields of a Config in the order of ffd_config's; made when the module is
const char* const kFieldNames[] = {"num_q_heads", "num_kv_heads", "head_dim", "block_tokens", "quant_bits", "n_sink_blocks",
                                   "n_local_blocks", "sm_scale", "out_dtype"};
constexpr int kFields = sizeof kFieldNames / sizeof kFieldNames[0], kScaleField = 7;
PyObject* field_names[kFields];

// A call's own copy of the Config's fields, read from the Python object while this call holds the interpreter's lock: the object
// may be a copy, come out of a pickle, or be changed by another thread once the lock is given up.  (An address of a structure,
// which says nothing of that structure's life, is not accepted; reading nine attributes takes no longer than asking for it did.)
ffd_config config_of(PyObject* o) {
    int32_t x[kFields] = {};
    float scale = 0.f;
    for (int i = 0; i < kFields; ++i) {
        PyObject* const value = PyObject_GetAttr(o, field_names[i]);
        if (!value) throw Bad{};
        bool good;
        if (i == kScaleField) {
            scale = (float)PyFloat_AsDouble(value);
            good = !PyErr_Occurred();
        } else {
            const long long n = PyLong_AsLongLong(value);
            x[i] = (int32_t)n;
            good = !PyErr_Occurred() && x[i] == n;
        }
        Py_DECREF(value);
        if (!good) {
            PyErr_Clear();
            PyErr_Format(PyExc_ValueError, "cfg.%s: %s is needed", kFieldNames[i], i == kScaleField ? "a number" : "an integer of 32 bits");
            throw Bad{};
        }
    }
    return ffd_config{x[0], x[1], x[2], x[3], x[4], x[5], x[6], scale, x[8]};
}

// One call: its configuration and the device that all its tensors have to be on, the workspace's
struct Call {
    const ffd_config own;
    const ffd_config* const cfg = &own;
    int64_t heads_q, heads_kv, block, dim;
    c10::Device device;
    const at::Tensor& workspace;
    PyObject* stream;

    Call(const Call&) = delete;
    Call(PyObject* config, PyObject* ws, PyObject* s)
        : own(config_of(config)), device(c10::kCPU), workspace(tensor(ws, "workspace")), stream(s) {
        heads_q = cfg->num_q_heads;
        heads_kv = cfg->num_kv_heads;
        block = cfg->block_tokens;
        dim = cfg->head_dim;
        device = workspace.device();
        if (!workspace.is_contiguous()) refuse("workspace", "a contiguous tensor", &workspace);
    }

    void* address(const at::Tensor& t, const char* name, c10::ScalarType type, std::initializer_list<int64_t> shape) const {
        if (t.scalar_type() != type || t.sizes() != c10::IntArrayRef(shape) || !t.is_contiguous() || t.device() != device)
            refuse(name, std::string("a contiguous ") + c10::toString(type) + " tensor " + shape_text(shape) + " on " + device.str(), &t);
        return t.data_ptr();
    }
    void* address(PyObject* o, const char* name, c10::ScalarType type, std::initializer_list<int64_t> shape) const {
        return address(tensor(o, name), name, type, shape);
    }
    // an index array of `count` elements in any shape; None where that is allowed
    const int32_t* index(PyObject* o, const char* name, int64_t count, bool optional = false) const {
        if (optional && o == Py_None) return nullptr;
        const at::Tensor& t = tensor(o, name);
        if (t.scalar_type() != c10::kInt || t.numel() != count || !t.is_contiguous() || t.device() != device)
            refuse(name, "a contiguous Int tensor of " + std::to_string(count) + " elements on " + device.str(), &t);
        return static_cast<const int32_t*>(t.data_ptr());
    }

    template <typename F>
    PyObject* run(F&& call) const {
        if (!device.is_cuda()) refuse("workspace", "a CUDA tensor", &workspace);
        const c10::cuda::CUDAGuard guard(device);
        void* s = nullptr;
        if (stream == Py_None) {
            s = c10::cuda::getCurrentCUDAStream(device.index()).stream();
        } else {
            PyObject* handle = PyObject_GetAttrString(stream, "cuda_stream");
            if (!handle) throw Bad{};
            s = PyLong_AsVoidPtr(handle);
            Py_DECREF(handle);
            if (PyErr_Occurred()) throw Bad{};
        }
        void* ws = workspace.data_ptr();
        const size_t bytes = workspace.nbytes();
        ffd_status status;
        {
            PyThreadState* const saved = PyEval_SaveThread();
            status = call(ws, bytes, s);
            PyEval_RestoreThread(saved);
        }
        return PyLong_FromLong(status);
    }
};

int32_t number(PyObject* o) {
    const long long x = PyLong_AsLongLong(o);
    if (PyErr_Occurred()) throw Bad{};
    if (x != (int32_t)x) {
        PyErr_SetString(PyExc_ValueError, "a number is beyond 32 bits");
        throw Bad{};
    }
    return (int32_t)x;
}

struct ByteCache {
    int32_t format, pages;
    void *k, *v;
    float *k_scale, *v_scale;

    ByteCache(const Call& c, PyObject* const* a) {   // k_byte, v_byte, k_scale, v_scale
        const at::Tensor& kt = tensor(a[0], "k_byte");
        const c10::ScalarType type = kt.scalar_type();
        if ((type != c10::kChar && type != c10::kFloat8_e4m3fn) || kt.dim() != 4) refuse("k_byte", "a pool of int8 or float8_e4m3fn pages", &kt);
        format = type == c10::kChar ? FFD_BYTE_INT8 : FFD_BYTE_E4M3;
        const int64_t n = kt.size(0);
        pages = (int32_t)n;
        if (pages != n) refuse("k_byte", "a pool of fewer pages", &kt);
        k = c.address(kt, "k_byte", type, {n, c.heads_kv, c.block, c.dim});
        v = c.address(a[1], "v_byte", type, {n, c.heads_kv, c.block, c.dim});
        k_scale = static_cast<float*>(c.address(a[2], "k_scale", c10::kFloat, {n, c.heads_kv, c.block}));
        v_scale = static_cast<float*>(c.address(a[3], "v_scale", c10::kFloat, {n, c.heads_kv, c.block}));
    }
};

struct HalfCache {
    int32_t pages;
    void *k, *v;

    HalfCache(const Call& c, PyObject* const* a) {   // k_cache, v_cache
        const at::Tensor& kt = tensor(a[0], "k_cache");
        const int64_t n = kt.dim() ? kt.size(0) : 0;
        pages = (int32_t)n;
        if (pages != n) refuse("k_cache", "a pool of fewer pages", &kt);
        k = c.address(kt, "k_cache", c10::kBFloat16, {n, c.heads_kv, c.block, c.dim});
        v = c.address(a[1], "v_cache", c10::kBFloat16, {n, c.heads_kv, c.block, c.dim});
    }
};

struct Results {
    int32_t batch;
    void *q, *out;
    float* lse;

    Results(const Call& c, PyObject* qo, PyObject* oo, PyObject* lo) {
        const at::Tensor& qt = tensor(qo, "q");
        const int64_t n = qt.dim() ? qt.size(0) : 0;
        batch = (int32_t)n;
        if (batch != n) refuse("q", "a smaller batch", &qt);
        q = c.address(qt, "q", c10::kBFloat16, {n, c.heads_q, c.dim});
        out = c.address(oo, "out", c.cfg->out_dtype == 0 ? c10::kBFloat16 : c10::kFloat, {n, c.heads_q, c.dim});
        lse = lo == Py_None ? nullptr : static_cast<float*>(c.address(lo, "lse", c10::kFloat, {n, c.heads_q}));
    }
};

template <typename F>
F* function(PyObject* address) {
    return reinterpret_cast<F*>(PyLong_AsVoidPtr(address));
}

// Runs `body` for a call of exactly `want` arguments.  Nothing that is thrown leaves it.
template <typename Body>
PyObject* guarded(const char* name, Py_ssize_t got, Py_ssize_t want, Body&& body) {
    if (got != want) {
        PyErr_Format(PyExc_TypeError, "%s: %zd arguments are needed, got %zd", name, want, got);
        return nullptr;
    }
    try {
        return body();
    } catch (const Bad&) {
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

// k_new, v_new, byte cache (4), block_table, seq_lens, max_blocks, row_start, first_token, workspace, stream
PyObject* write_kv_byte(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded("write_kv_byte", n, 15, [&] {
        const Call c(a[1], a[13], a[14]);
        const at::Tensor &k = tensor(a[2], "k_new"), &lens = tensor(a[9], "seq_lens");
        const int64_t rows = k.dim() ? k.size(0) : 0, stride = rows > 1 ? k.stride(0) : c.heads_kv * c.dim;
        for (int i = 0; i < 2; ++i) {
            const char* name = i ? "v_new" : "k_new";
            const at::Tensor& t = tensor(a[2 + i], name);
            if (t.scalar_type() != c10::kBFloat16 || t.sizes() != c10::IntArrayRef({rows, c.heads_kv, c.dim}) || t.device() != c.device ||
                (c.dim > 1 && t.stride(2) != 1) || (c.heads_kv > 1 && t.stride(1) != c.dim) || (rows > 1 && t.stride(0) != stride))
                refuse(name, "a BFloat16 tensor " + shape_text({rows, c.heads_kv, c.dim}) + " on " + c.device.str() +
                                 ", contiguous but for the stride " + std::to_string(stride) + " of its rows,", &t);
        }
        const ByteCache cache(c, a + 4);
        const int32_t batch = (int32_t)lens.numel(), blocks = number(a[10]);
        const int64_t entries = (int64_t)batch * blocks;
        const int32_t *table = c.index(a[8], "block_table", entries, true), *seq = c.index(a[9], "seq_lens", batch);
        const int32_t *start = c.index(a[11], "row_start", batch, true), *first = c.index(a[12], "first_token", batch, true);
        const void *kp = k.data_ptr(), *vp = tensor(a[3], "v_new").data_ptr();
        if (rows != (int32_t)rows) refuse("k_new", "a tensor of fewer rows", &k);
        auto* f = function<decltype(ffd_write_kv_byte)>(a[0]);
        return c.run([&](void* ws, size_t bytes, void* s) {
            if (rows == 0 && start && first) return FFD_OK;   // no sequence has a new token: nothing to launch
            return f(c.cfg, cache.format, kp, vp, stride, (int32_t)rows, start, cache.k, cache.v, cache.k_scale, cache.v_scale, table,
                     first, seq, batch, blocks, cache.pages, ws, bytes, s);
        });
    });
}

// byte cache (4), block_table, seq_lens, k_cache, v_cache, max_blocks, cache_table, first_token, workspace, stream
PyObject* read_kv_byte(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded("read_kv_byte", n, 15, [&] {
        const Call c(a[1], a[13], a[14]);
        const ByteCache cache(c, a + 2);
        const HalfCache half(c, a + 8);
        const int32_t batch = (int32_t)tensor(a[7], "seq_lens").numel(), blocks = number(a[10]);
        const int64_t entries = (int64_t)batch * blocks;
        const int32_t *table = c.index(a[6], "block_table", entries, true), *seq = c.index(a[7], "seq_lens", batch);
        const int32_t *to = c.index(a[11], "cache_table", entries, true), *first = c.index(a[12], "first_token", batch, true);
        auto* f = function<decltype(ffd_read_kv_byte)>(a[0]);
        return c.run([&](void* ws, size_t bytes, void* s) {
            return f(c.cfg, cache.format, cache.k, cache.v, cache.k_scale, cache.v_scale, table, first, seq, batch, blocks,
                     cache.pages, half.k, half.v, to, half.pages, ws, bytes, s);
        });
    });
}

// q, byte cache (4), block_table, seq_lens, out, max_blocks, lse, workspace, stream
PyObject* decode_byte(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded("decode_byte", n, 14, [&] {
        const Call c(a[1], a[12], a[13]);
        const Results r(c, a[2], a[9], a[11]);
        const ByteCache cache(c, a + 3);
        const int32_t blocks = number(a[10]);
        const int32_t *table = c.index(a[7], "block_table", (int64_t)r.batch * blocks, true), *seq = c.index(a[8], "seq_lens", r.batch);
        auto* f = function<decltype(ffd_decode_byte)>(a[0]);
        return c.run([&](void* ws, size_t bytes, void* s) {
            return f(c.cfg, cache.format, r.q, cache.k, cache.v, cache.k_scale, cache.v_scale, table, seq, r.batch, blocks,
                     cache.pages, r.out, r.lse, ws, bytes, s);
        });
    });
}

// q, k_cache, v_cache, prefix_table, prefix_len, block_table, seq_lens, out, max_prefix_blocks, max_blocks, lse, workspace, stream
PyObject* decode_prefix(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded("decode_prefix", n, 15, [&] {
        const Call c(a[1], a[13], a[14]);
        const Results r(c, a[2], a[9], a[12]);
        const HalfCache half(c, a + 3);
        const int32_t prefix_blocks = number(a[10]), blocks = number(a[11]);
        const int32_t *pre = c.index(a[5], "prefix_table", prefix_blocks), *len = c.index(a[6], "prefix_len", 1);
        const int32_t *table = c.index(a[7], "block_table", (int64_t)r.batch * blocks, true), *seq = c.index(a[8], "seq_lens", r.batch);
        auto* f = function<decltype(ffd_decode_prefix)>(a[0]);
        return c.run([&](void* ws, size_t bytes, void* s) {
            return f(c.cfg, r.q, half.k, half.v, pre, len, prefix_blocks, table, seq, r.batch, blocks, half.pages, r.out, r.lse, ws,
                     bytes, s);
        });
    });
}

// q, k_cache, v_cache, prefix_table, prefix_len, byte cache (4), block_table, seq_lens, out, max_prefix_blocks, max_blocks, lse,
// workspace, stream
PyObject* decode_prefix_byte(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded("decode_prefix_byte", n, 19, [&] {
        const Call c(a[1], a[17], a[18]);
        const Results r(c, a[2], a[13], a[16]);
        const HalfCache half(c, a + 3);
        const int32_t prefix_blocks = number(a[14]), blocks = number(a[15]);
        const int32_t *pre = c.index(a[5], "prefix_table", prefix_blocks), *len = c.index(a[6], "prefix_len", 1);
        const ByteCache cache(c, a + 7);
        const int32_t *table = c.index(a[11], "block_table", (int64_t)r.batch * blocks, true), *seq = c.index(a[12], "seq_lens", r.batch);
        auto* f = function<decltype(ffd_decode_prefix_byte)>(a[0]);
        return c.run([&](void* ws, size_t bytes, void* s) {
            return f(c.cfg, cache.format, r.q, half.k, half.v, pre, len, prefix_blocks, half.pages, cache.k, cache.v, cache.k_scale,
                     cache.v_scale, table, seq, r.batch, blocks, cache.pages, r.out, r.lse, ws, bytes, s);
        });
    });
}

#define FFD_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FFD_METHOD(write_kv_byte), FFD_METHOD(read_kv_byte), FFD_METHOD(decode_byte), FFD_METHOD(decode_prefix),
                         FFD_METHOD(decode_prefix_byte), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ffd_binding", "Checks and calls for ffd.py", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__ffd_binding() {
    for (int i = 0; i < kFields; ++i)
        if (!(field_names[i] = PyUnicode_InternFromString(kFieldNames[i]))) return nullptr;
    return PyModule_Create(&module);
}
