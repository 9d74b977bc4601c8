// Python module _ps_tensor_args: takes the torch tensors of ps_build_slots, ps_rope_append and ps_paged_attn apart,
// checks them and calls the library.
//
// The calls are made for every layer of every step and a small one takes 3 us on the device.  Asking 8 to 12 tensors
// for type, device, shape, strides and address took 5 to 8 us in Python; here it takes less than the launch.
//
// The functions take positional arguments only (binding.py has the signatures) and return (status, text) like the
// binding's other calls.  bind() is given the library's entry points, so that the module uses whichever build of the
// library the binding has loaded.
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <optional>
#include <sstream>
#include <string>
#include <type_traits>

#include "ps_kvswap.h"

namespace {

using at::ScalarType;

decltype(&ps_build_slots) g_build_slots = nullptr;
decltype(&ps_rope_append) g_rope_append = nullptr;
decltype(&ps_paged_attn) g_paged_attn = nullptr;
decltype(&ps_paged_attn_workspace) g_workspace = nullptr;

PyObject* answer(int32_t rc, const std::string& text) { return Py_BuildValue("(is)", (int)rc, text.c_str()); }

// What is wrong with an argument; becomes PS_ERR_INVALID with the text.
struct BadArg {
    std::string text;
};

std::string describe(const at::Tensor& t) {
    std::ostringstream s;
    s << "got " << t.scalar_type() << " " << t.sizes() << " strides " << t.strides() << " on " << t.device();
    return s.str();
}

const at::Tensor* tensor(const char* name, PyObject* o) {   // null for None
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) throw BadArg{std::string(name) + ": need a tensor"};
    return &THPVariable_Unpack(o);
}
const at::Tensor& must(const char* name, PyObject* o) {
    const at::Tensor* t = tensor(name, o);
    if (!t) throw BadArg{std::string(name) + ": need a tensor, got None"};
    return *t;
}

int32_t int_arg(const char* name, PyObject* o) {
    const Py_ssize_t v = PyIndex_Check(o) ? PyNumber_AsSsize_t(o, nullptr) : PY_SSIZE_T_MIN;   // clipped, not wrapped
    if (PyErr_Occurred()) PyErr_Clear();
    if (v < INT32_MIN || v > INT32_MAX) throw BadArg{std::string(name) + ": need an integer of 32 bits"};
    return (int32_t)v;
}
int32_t int_size(const char* name, int64_t v) {
    if (v > INT32_MAX) throw BadArg{std::string(name) + ": more than 2^31 - 1"};
    return (int32_t)v;
}

// Address of a contiguous tensor of dtype with at least `least` elements; null for None.
template <typename T>
T* vec(const char* name, PyObject* o, ScalarType dtype, int64_t least, const at::Device& dev) {
    const at::Tensor* t = tensor(name, o);
    if (!t) return nullptr;
    if (t->scalar_type() != dtype || t->device() != dev || t->numel() < least || !t->is_contiguous()) {
        std::ostringstream s;
        s << name << ": need a contiguous " << dtype << " tensor of at least " << least << " elements on " << dev << ", " << describe(*t);
        throw BadArg{s.str()};
    }
    return (T*)const_cast<void*>(std::is_const_v<T> ? t->const_data_ptr() : t->mutable_data_ptr());
}

// Stride of the outermost dimension of a tensor of this shape that is dense below it.
int64_t outer_stride(const char* name, const at::Tensor& t, at::IntArrayRef shape, ScalarType dtype, const at::Device& dev) {
    bool ok = t.scalar_type() == dtype && t.device() == dev && t.sizes() == shape;
    int64_t dense = 1;
    if (ok)
        for (size_t d = shape.size() - 1; d > 0; --d) {
            ok = ok && (shape[d] < 2 || t.stride(d) == dense);
            dense *= shape[d];
        }
    if (!ok) {
        std::ostringstream s;
        s << name << ": need " << dtype << " " << shape << " on " << dev << ", dense but for the first dimension, " << describe(t);
        throw BadArg{s.str()};
    }
    return shape[0] > 1 ? t.stride(0) : dense;
}

int32_t dtype_code(const at::Tensor& t) {
    if (t.scalar_type() == ScalarType::BFloat16) return PS_DTYPE_BF16;
    if (t.scalar_type() == ScalarType::Half) return PS_DTYPE_FP16;
    throw BadArg{"need bfloat16 or float16 tensors, " + describe(t)};
}

const at::Tensor& on_device(const char* what, const at::Tensor& t, int64_t dims) {
    if (!t.is_cuda() || t.dim() != dims) throw BadArg{std::string(what) + " on a device, " + describe(t)};
    return t;
}

template <typename Fn, typename Args>
PyObject* enqueue(Fn fn, const Args& args, const at::Device& dev) {
    char text[256];
    text[0] = 0;
    int32_t rc;
    {
        std::optional<c10::cuda::CUDAGuard> guard;
        if (c10::cuda::current_device() != dev.index()) guard.emplace(dev);
        cudaStream_t stream = c10::cuda::getCurrentCUDAStream(dev.index()).stream();
        // a launch waits when the device's queue is full, and what empties it may need the interpreter
        Py_BEGIN_ALLOW_THREADS
        rc = fn(&args, stream, text, sizeof text);
        Py_END_ALLOW_THREADS
    }
    return answer(rc, text);
}

template <typename Body>
PyObject* call(const char* name, Py_ssize_t n, Py_ssize_t want, Body body) {
    HANDLE_TH_ERRORS
    if (n != want || !g_build_slots) {
        PyErr_SetString(PyExc_TypeError, "_ps_tensor_args: wrong number of arguments, or bind() was not called");
        return nullptr;
    }
    try {
        return body();
    } catch (const BadArg& e) {
        return answer(PS_ERR_INVALID, std::string(name) + ": " + e.text);
    }
    END_HANDLE_TH_ERRORS
}

// ctx_lens, new_lens, block_tables, slots, positions, token_start, ctx_lens_out, block_size, num_gpu_blocks, free_ids,
// free_count, free_count_out, status_word
PyObject* py_build_slots(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call("ps_build_slots", n, 13, [&]() {
        const at::Tensor& slots = must("slots", a[3]);
        if (!slots.is_cuda()) throw BadArg{"slots: need a tensor on a device, " + describe(slots)};
        const at::Device dev = slots.device();
        const at::Tensor& tables = on_device("block_tables: need [batch][stride]", must("block_tables", a[2]), 2);
        ps_slots_args p{};
        p.batch = int_size("ctx_lens", must("ctx_lens", a[0]).numel());
        p.table_stride = int_size("block_tables", tables.size(1));
        p.max_tokens = int_size("slots", slots.numel());
        p.block_size = int_arg("block_size", a[7]);
        p.num_gpu_blocks = int_arg("num_gpu_blocks", a[8]);
        const ScalarType i32 = ScalarType::Int;
        must("new_lens", a[1]);
        must("token_start", a[5]);
        must("ctx_lens_out", a[6]);
        p.ctx_lens = vec<const int32_t>("ctx_lens", a[0], i32, p.batch, dev);
        p.new_lens = vec<const int32_t>("new_lens", a[1], i32, p.batch, dev);
        p.block_tables = vec<int32_t>("block_tables", a[2], i32, (int64_t)p.batch * p.table_stride, dev);
        p.slots = vec<int64_t>("slots", a[3], ScalarType::Long, 0, dev);
        p.positions = vec<int32_t>("positions", a[4], i32, p.max_tokens, dev);
        p.token_start = vec<int32_t>("token_start", a[5], i32, (int64_t)p.batch + 1, dev);
        p.ctx_lens_out = vec<int32_t>("ctx_lens_out", a[6], i32, p.batch, dev);
        p.free_ids = vec<int32_t>("free_ids", a[9], i32, p.num_gpu_blocks, dev);
        p.free_count = vec<const int32_t>("free_count", a[10], i32, 1, dev);
        p.free_count_out = vec<int32_t>("free_count_out", a[11], i32, 1, dev);
        p.status_word = vec<int32_t>("status_word", a[12], i32, 1, dev);
        return enqueue(g_build_slots, p, dev);
    });
}

// q, k, q_out, k_out, positions, inv_freq, v, kpool, vpool, slots, freq_axis, neighbours, inverse, status_word
PyObject* py_rope_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call("ps_rope_append", n, 14, [&]() {
        const at::Tensor *q = tensor("q", a[0]), *k = tensor("k", a[1]);
        if (!q && !k) throw BadArg{"need q or k"};
        const at::Tensor& ref = on_device("need q or k [tokens][heads][dim]", q ? *q : *k, 3);
        const at::Device dev = ref.device();
        const ScalarType dt = ref.scalar_type();
        const int64_t T = ref.size(0), D = ref.size(2);
        ps_rope_args p{};
        p.dtype = dtype_code(ref);
        p.tokens = int_size("tokens", T);
        p.head_dim = int_size("dim", D);
        p.slots = vec<const int64_t>("slots", a[9], ScalarType::Long, T, dev);
        p.status_word = vec<int32_t>("status_word", a[13], ScalarType::Int, 1, dev);
        auto rows = [&](const char* name, const at::Tensor& t, int64_t heads, bool out) {
            const int64_t s = outer_stride(name, t, {T, heads, D}, dt, dev);
            if (out && s < heads * D) throw BadArg{std::string(name) + ": rows overlap"};
            return s;
        };
        if (q) {
            const at::Tensor& q_out = must("q_out", a[2]);
            p.num_q_heads = int_size("heads", q->size(1));
            p.q_stride = rows("q", *q, q->size(1), false);
            p.q_out_stride = rows("q_out", q_out, q->size(1), true);
            p.q = q->const_data_ptr();
            p.q_out = q_out.mutable_data_ptr();
        }
        const at::Tensor *k_out = tensor("k_out", a[3]), *kpool = tensor("kpool", a[7]), *vpool = tensor("vpool", a[8]);
        if (!k && (k_out || kpool)) throw BadArg{"k_out and pools need k"};
        if (k) {
            const int64_t heads = k->dim() == 3 ? k->size(1) : 0;
            p.num_kv_heads = int_size("heads", heads);
            p.k_stride = rows("k", *k, heads, false);
            p.k = k->const_data_ptr();
            if (k_out) {
                p.k_out_stride = rows("k_out", *k_out, heads, true);
                p.k_out = k_out->mutable_data_ptr();
            }
            if (kpool || vpool) {
                const at::Tensor* v = tensor("v", a[6]);
                if (!kpool || !vpool || !v || a[9] == Py_None || kpool->dim() != 4)
                    throw BadArg{"an append needs k, v, slots and two pools [blocks][block_size][heads][dim]"};
                const int64_t shape[4] = {kpool->size(0), kpool->size(1), heads, D};
                p.num_gpu_blocks = int_size("blocks", shape[0]);
                p.block_size = int_size("block_size", shape[1]);
                p.k_block_stride = outer_stride("kpool", *kpool, shape, dt, dev);
                p.v_block_stride = outer_stride("vpool", *vpool, shape, dt, dev);
                p.v_stride = rows("v", *v, heads, false);
                p.v = v->const_data_ptr();
                p.kpool = kpool->mutable_data_ptr();
                p.vpool = vpool->mutable_data_ptr();
            }
        }
        const at::Tensor* inv = tensor("inv_freq", a[5]);
        if (inv && inv->numel() > 0) {
            const int64_t half = inv->numel();
            if (half > 256) throw BadArg{"inv_freq: at most 256 frequencies"};
            p.rot_dim = (int32_t)(2 * half);
            p.inv_freq = vec<const float>("inv_freq", a[5], ScalarType::Float, half, dev);
            const at::Tensor& pos = must("positions", a[4]);
            const int64_t dims = pos.dim();
            if (pos.scalar_type() != ScalarType::Int || pos.device() != dev || dims < 1 || dims > 2 || pos.size(dims - 1) != T ||
                (T > 1 && pos.stride(dims - 1) != 1))
                throw BadArg{"positions: need int32 [tokens] or [axes][tokens] on the tensors' device, " + describe(pos)};
            p.positions = (const int32_t*)pos.const_data_ptr();
            p.num_axes = dims == 1 ? 1 : int_size("axes", pos.size(0));
            p.axis_stride = p.num_axes > 1 ? pos.stride(0) : 0;
            if (a[10] != Py_None) {
                PyObject* list = PySequence_Fast(a[10], "");
                bool ok = list && PySequence_Fast_GET_SIZE(list) == half;
                for (int64_t i = 0; ok && i < half; ++i) {
                    PyObject* v = PySequence_Fast_GET_ITEM(list, i);
                    const Py_ssize_t axis = PyIndex_Check(v) ? PyNumber_AsSsize_t(v, nullptr) : -1;
                    ok = axis >= 0 && axis < 256;
                    p.freq_axis[i] = (uint8_t)axis;
                }
                Py_XDECREF(list);
                PyErr_Clear();
                if (!ok) throw BadArg{"freq_axis: need one axis, 0 or more, for every frequency"};
            }
        }
        const int neighbours = PyObject_IsTrue(a[11]), inverse = PyObject_IsTrue(a[12]);
        if (neighbours < 0 || inverse < 0) {
            PyErr_Clear();
            throw BadArg{"neighbours and inverse: need truth values"};
        }
        p.flags = (neighbours ? PS_ROPE_NEIGHBOURS : 0) | (inverse ? PS_ROPE_INVERSE : 0);
        return enqueue(g_rope_append, p, dev);
    });
}

// kpool, vpool, q, out, block_tables, ctx_lens, lse, window, scale, status_word, workspace
PyObject* py_paged_attn(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call("ps_paged_attn", n, 11, [&]() {
        const at::Tensor& q = on_device("q: need [batch][heads][dim]", must("q", a[2]), 3);
        const at::Tensor& kpool = on_device("kpool: need [blocks][block_size][heads][dim]", must("kpool", a[0]), 4);
        const at::Tensor& vpool = must("vpool", a[1]);
        const at::Tensor& out = must("out", a[3]);
        const at::Tensor& tables = on_device("block_tables: need [batch][stride]", must("block_tables", a[4]), 2);
        must("ctx_lens", a[5]);
        const at::Device dev = q.device();
        const ScalarType dt = q.scalar_type();
        ps_paged_attn_args p{};
        p.dtype = dtype_code(q);
        p.batch = int_size("batch", q.size(0));
        p.num_q_heads = int_size("heads", q.size(1));
        p.head_dim = int_size("dim", q.size(2));
        p.num_gpu_blocks = int_size("blocks", kpool.size(0));
        p.block_size = int_size("block_size", kpool.size(1));
        p.num_kv_heads = int_size("heads", kpool.size(2));
        p.table_stride = int_size("block_tables", tables.size(1));
        const int64_t shape[4] = {kpool.size(0), kpool.size(1), kpool.size(2), q.size(2)};
        p.k_block_stride = outer_stride("kpool", kpool, shape, dt, dev);
        p.v_block_stride = outer_stride("vpool", vpool, shape, dt, dev);
        p.q_stride = outer_stride("q", q, q.sizes(), dt, dev);
        p.out_stride = outer_stride("out", out, q.sizes(), dt, dev);
        p.kpool = kpool.const_data_ptr();
        p.vpool = vpool.const_data_ptr();
        p.q = q.const_data_ptr();
        p.out = out.mutable_data_ptr();
        p.lse = vec<float>("lse", a[6], ScalarType::Float, (int64_t)p.batch * p.num_q_heads, dev);
        p.block_tables = vec<const int32_t>("block_tables", a[4], ScalarType::Int, (int64_t)p.batch * p.table_stride, dev);
        p.ctx_lens = vec<const int32_t>("ctx_lens", a[5], ScalarType::Int, p.batch, dev);
        p.window = int_arg("window", a[7]);
        if (a[8] != Py_None) {
            const double s = PyFloat_AsDouble(a[8]);
            if (PyErr_Occurred() || (float)s == 0.f) {
                PyErr_Clear();
                throw BadArg{"scale: need a factor that is not 0"};
            }
            p.scale = (float)s;
        }
        p.status_word = vec<int32_t>("status_word", a[9], ScalarType::Int, 1, dev);
        at::Tensor scratch;   // kept until the launches are enqueued; then the allocator's order on the stream protects it
        if (a[10] == Py_None) {
            int64_t need = 0;
            {
                std::optional<c10::cuda::CUDAGuard> guard;
                if (c10::cuda::current_device() != dev.index()) guard.emplace(dev);
                const int32_t rc = g_workspace(p.num_kv_heads, p.num_q_heads, p.head_dim, &need);
                if (rc == PS_ERR_CUDA) return answer(rc, "ps_paged_attn: device");
            }
            if (need > 0) {   // else the shape is refused below
                scratch = at::empty({need}, at::TensorOptions().dtype(at::kByte).device(dev));
                p.workspace = scratch.mutable_data_ptr();
                p.workspace_bytes = need;
            }
        } else {
            p.workspace = vec<void>("workspace", a[10], ScalarType::Byte, 0, dev);
            p.workspace_bytes = THPVariable_Unpack(a[10]).numel();
        }
        return enqueue(g_paged_attn, p, dev);
    });
}

PyObject* py_bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    void* p[4];
    for (int i = 0; i < 4; ++i) {
        p[i] = n == 4 ? PyLong_AsVoidPtr(a[i]) : nullptr;
        if (!p[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "bind: need four addresses");
            return nullptr;
        }
    }
    g_build_slots = (decltype(g_build_slots))p[0];
    g_rope_append = (decltype(g_rope_append))p[1];
    g_paged_attn = (decltype(g_paged_attn))p[2];
    g_workspace = (decltype(g_workspace))p[3];
    Py_RETURN_NONE;
}

#define PS_FAST(f) (PyCFunction)(void (*)(void))f, METH_FASTCALL
PyMethodDef methods[] = {{"bind", PS_FAST(py_bind), nullptr},
                         {"build_slots", PS_FAST(py_build_slots), nullptr},
                         {"rope_append", PS_FAST(py_rope_append), nullptr},
                         {"paged_attn", PS_FAST(py_paged_attn), nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ps_tensor_args", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__ps_tensor_args() { return PyModule_Create(&module); }
