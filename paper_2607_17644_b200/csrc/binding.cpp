// Python's way into the rotary, cache and decode entry points of include/laga.h.
//
// A decode step makes a handful of these calls for 2 to 15 us of device work each, so what a call costs on the host is what a
// service that does not capture its steps pays.  Checks, allocations and the call are compiled here.  Measured per call, calls in a row, a
// B200's host, against ctypes with the same checks and allocations from Python: rotation 10.6 -> 5.0 us, latent norm 19.3 -> 9.1, its
// backward 23.2 -> 10.8, into the cache 12 -> 4.6, plan 16.2 -> 7.4, one token's attention 20.9 -> 12 (its three kernels then take 14.5).
// The kernels' library is not linked: `bind` takes the addresses of its functions from the one that the package has loaded (the
// ordinary or the checked build).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <cstring>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/zeros.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/laga.h"

namespace {

using at::Tensor;
using c10::ScalarType;

struct Library {
    decltype(&laga_rope) rope;
    decltype(&laga_latent_norm_rope) latent_norm_rope;
    decltype(&laga_latent_norm_rope_backward_workspace_bytes) backward_workspace_bytes;
    decltype(&laga_latent_norm_rope_backward) latent_norm_rope_backward;
    decltype(&laga_cache_plan) cache_plan;
    decltype(&laga_paged_decode_workspace_bytes) decode_workspace_bytes;
    decltype(&laga_paged_decode) paged_decode;
} library;
PyObject* fail = nullptr;                                     // fail(code, where) raises the package's error

// ---- arguments ---------------------------------------------------------------------------------------
const Tensor& tensor(PyObject* o, const char* name) {
    TORCH_CHECK_TYPE(THPVariable_Check(o), name, ": expected a tensor, got ", Py_TYPE(o)->tp_name);
    return THPVariable_Unpack(o);
}
Tensor maybe(PyObject* o, const char* name) { return o == Py_None ? Tensor() : tensor(o, name); }
void* data(const Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
template <class T>
T* data(const Tensor& t) { return static_cast<T*>(data(t)); }
double number(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw python_error();
    return v;
}
int integer(PyObject* o) {
    int overflow = 0;
    const long v = PyLong_AsLongAndOverflow(o, &overflow);
    if (v == -1 && PyErr_Occurred()) throw python_error();
    TORCH_CHECK_VALUE(overflow == 0 && v >= INT_MIN && v <= INT_MAX, "integer out of range");
    return static_cast<int>(v);
}
int size32(int64_t v, const char* name) {
    TORCH_CHECK_VALUE(v <= INT_MAX, name, ": size ", v, " does not fit 32 bits");
    return static_cast<int>(v);
}
bool truth(PyObject* o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw python_error();
    return v != 0;
}
void expect(const Tensor& t, ScalarType dtype, at::IntArrayRef shape, const char* name) {
    TORCH_CHECK_VALUE(t.is_cuda() && t.scalar_type() == dtype && t.is_contiguous() && t.sizes() == shape, name, ": expected contiguous CUDA ",
                      dtype, " tensor of shape ", shape, ", got ", t.scalar_type(), " ", t.sizes(), " strides ", t.strides(), " on ", t.device());
}
// A tensor whose rows (first axis) are dense and may be any pitch apart: the pitch in elements.
int64_t rows(const Tensor& t, int64_t dims, const char* name) {
    bool ok = t.is_cuda() && t.scalar_type() == ScalarType::BFloat16 && t.dim() == dims;
    int64_t dense = 1;
    for (int64_t i = dims - 1; ok && i >= 1; --i) {
        ok = t.stride(i) == dense || t.size(i) == 1;
        dense *= t.size(i);
    }
    const int64_t pitch = ok && t.size(0) > 1 ? t.stride(0) : dense;
    TORCH_CHECK_VALUE(ok && pitch >= dense, name, ": expected a ", dims, "-d CUDA BFloat16 tensor with dense rows, got ", t.scalar_type(), " ",
                      t.sizes(), " strides ", t.strides(), " on ", t.device());
    return pitch;
}
c10::Device one_device(std::initializer_list<const Tensor*> tensors) {
    const Tensor* first = nullptr;
    for (const Tensor* t : tensors) {
        if (!t->defined()) continue;
        if (first == nullptr) first = t;
        TORCH_CHECK_VALUE(t->device() == first->device(), "tensors of one call are on different devices: ", first->device(), " and ", t->device());
    }
    return first->device();
}

struct Plan {
    Tensor freqs;
    float mscale;
    int interleaved;
    int d_rot;
    Plan(PyObject* o, const Tensor& positions, int64_t M) {
        TORCH_CHECK_TYPE(PyTuple_Check(o) && PyTuple_GET_SIZE(o) == 3, "rope: expected a RopePlan, got ", Py_TYPE(o)->tp_name);
        freqs = tensor(PyTuple_GET_ITEM(o, 0), "freqs");
        mscale = static_cast<float>(number(PyTuple_GET_ITEM(o, 1)));
        interleaved = truth(PyTuple_GET_ITEM(o, 2)) ? LAGA_ROPE_INTERLEAVED : LAGA_ROPE_HALF;
        expect(freqs, ScalarType::Double, {freqs.numel()}, "freqs");
        expect(positions, ScalarType::Int, {M}, "positions");
        d_rot = 2 * size32(freqs.numel(), "freqs");
    }
    void is_as_wide_as(int64_t channels) const {
        TORCH_CHECK_VALUE(d_rot == channels, "the plan rotates ", d_rot, " channels, the tensor has ", channels);
    }
};

// ---- results -----------------------------------------------------------------------------------------
Tensor fresh(const Tensor& like, at::IntArrayRef shape, ScalarType dtype) { return at::empty(shape, like.options().dtype(dtype)); }
// Elements offset .. offset + n of `whole`: a tensor on the same storage, made directly (of six results, six allocations or six
// dispatched views would cost more than the call itself).
Tensor part(const Tensor& whole, int64_t offset, int64_t n) {
    auto impl = c10::make_intrusive<c10::TensorImpl>(c10::Storage(whole.storage()), whole.key_set(), whole.dtype());
    impl->set_storage_offset(offset);
    impl->set_sizes_contiguous({n});
    return Tensor(std::move(impl));
}
// 1024-byte aligned (the allocator aligns to 512 at least)
Tensor workspace_of(const Tensor& like, size_t bytes) {
    const int64_t n = static_cast<int64_t>(bytes);
    Tensor t = fresh(like, {n}, ScalarType::Byte);
    const auto at = [](const Tensor& x) { return reinterpret_cast<uintptr_t>(x.data_ptr()) & 1023u; };
    if (at(t) == 0) return t;
    t = fresh(like, {n + 1024}, ScalarType::Byte);
    const int64_t skip = (1024 - at(t)) & 1023;
    return t.narrow(0, skip, n);
}
PyObject* wrap(const Tensor& t) {
    if (!t.defined()) Py_RETURN_NONE;
    PyObject* o = THPVariable_Wrap(t);
    if (o == nullptr) throw python_error();
    return o;
}
template <class... Ts>
PyObject* wrap_all(const Ts&... ts) {
    PyObject* out = PyTuple_New(sizeof...(ts));
    if (out == nullptr) throw python_error();
    Py_ssize_t i = 0;
    (PyTuple_SET_ITEM(out, i++, wrap(ts)), ...);
    return out;
}
void raise_for(int code, const char* where) {
    if (code == LAGA_OK) return;
    PyObject* r = PyObject_CallFunction(fail, "is", code, where);
    Py_XDECREF(r);
    throw python_error();
}
// The call itself: on the tensors' device and its current stream, other Python threads running meanwhile.
struct Unlocked {
    PyThreadState* state = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(state); }
};
template <class Call>
void enqueue(c10::Device device, const char* where, Call call) {
    int code;
    {
        c10::cuda::CUDAGuard guard(device);
        void* stream = c10::cuda::getCurrentCUDAStream(device.index()).stream();
        Unlocked others_run;
        code = call(stream);
    }
    raise_for(code, where);
}
void arguments(Py_ssize_t given, Py_ssize_t wanted) { TORCH_CHECK_TYPE(given == wanted, "expected ", wanted, " arguments, got ", given); }

// ---- entry points ------------------------------------------------------------------------------------
// rope(x, positions, plan, rot_begin | None, inverse, y | None) -> y
PyObject* py_rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    arguments(n, 6);
    const Tensor& x = tensor(a[0], "x");
    const Tensor& positions = tensor(a[1], "positions");
    const int64_t x_pitch = rows(x, 3, "x"), M = x.size(0), h = x.size(1), d = x.size(2);
    const Plan plan(a[2], positions, M);
    Tensor y = maybe(a[5], "y");
    int64_t y_pitch = h * d;
    if (y.defined()) {
        y_pitch = rows(y, 3, "y");
        TORCH_CHECK_VALUE(y.sizes() == x.sizes(), "y: expected shape ", x.sizes(), ", got ", y.sizes());
    }
    const c10::Device device = one_device({&x, &positions, &plan.freqs, &y});
    if (!y.defined()) y = fresh(x, x.sizes(), ScalarType::BFloat16);
    const int begin = a[3] == Py_None ? size32(d, "x") - plan.d_rot : integer(a[3]);
    const bool inverse = truth(a[4]);
    if (M > 0)
        enqueue(device, "laga_rope", [&](void* stream) {
            return library.rope(data(x), x_pitch, data<int>(positions), data<double>(plan.freqs), size32(M, "x"), size32(h, "x"), size32(d, "x"), begin,
                                plan.d_rot, plan.interleaved, plan.mscale, inverse, data(y), y_pitch, stream);
        });
    return wrap(y);
    END_HANDLE_TH_ERRORS
}

// latent_norm_rope(kv_a, gamma, beta | None, positions, plan, eps, dense, latent | None, k_pe | None, cache | None, slots | None)
// -> (latent, k_pe, mean, rstd) if dense, else None
PyObject* py_latent_norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    arguments(n, 11);
    const Tensor& kv_a = tensor(a[0], "kv_a");
    const Tensor& gamma = tensor(a[1], "gamma");
    const Tensor beta = maybe(a[2], "beta"), cache = maybe(a[9], "cache"), slots = maybe(a[10], "slots");
    const Tensor& positions = tensor(a[3], "positions");
    const int64_t pitch = rows(kv_a, 2, "kv_a"), M = kv_a.size(0), D = gamma.numel(), R = kv_a.size(1) - D;
    const Plan plan(a[4], positions, M);
    const float eps = static_cast<float>(number(a[5]));
    const bool dense = truth(a[6]);
    plan.is_as_wide_as(R);
    expect(gamma, ScalarType::BFloat16, {D}, "gamma");
    if (beta.defined()) expect(beta, ScalarType::BFloat16, {D}, "beta");
    TORCH_CHECK_VALUE(cache.defined() == slots.defined(), "cache and slots go together");
    TORCH_CHECK_VALUE(dense || cache.defined(), "cache: expected a tensor");
    int64_t n_slots = 0;
    if (cache.defined()) {
        TORCH_CHECK_VALUE(cache.is_cuda() && cache.scalar_type() == ScalarType::BFloat16 && cache.is_contiguous() && cache.dim() >= 2 &&
                              cache.size(-1) == D + R,
                          "cache: expected contiguous CUDA BFloat16 [..., ", D + R, "], got ", cache.scalar_type(), " ", cache.sizes(), " on ",
                          cache.device());
        expect(slots, ScalarType::Int, {M}, "slots");
        n_slots = cache.numel() / (D + R);
    }
    Tensor latent = maybe(a[7], "latent"), k_pe = maybe(a[8], "k_pe"), mean, rstd;
    if (latent.defined()) expect(latent, ScalarType::BFloat16, {M, D}, "latent");
    if (k_pe.defined()) expect(k_pe, ScalarType::BFloat16, {M, R}, "k_pe");
    const c10::Device device = one_device({&kv_a, &gamma, &beta, &positions, &plan.freqs, &latent, &k_pe, &cache, &slots});
    if (dense) {
        if (!latent.defined()) latent = fresh(kv_a, {M, D}, ScalarType::BFloat16);
        if (!k_pe.defined()) k_pe = fresh(kv_a, {M, R}, ScalarType::BFloat16);
        const Tensor statistics = fresh(kv_a, {2 * M}, ScalarType::Float);
        mean = part(statistics, 0, M);
        rstd = part(statistics, M, M);
    }
    if (M > 0)
        enqueue(device, "laga_latent_norm_rope", [&](void* stream) {
            return library.latent_norm_rope(data(kv_a), pitch, data(gamma), data(beta), eps, data<int>(positions), data<double>(plan.freqs),
                                            size32(M, "kv_a"), size32(D, "gamma"), size32(R, "kv_a"), plan.interleaved, plan.mscale, data(latent),
                                            data(k_pe), data<float>(mean), data<float>(rstd), data(cache), data<int>(slots),
                                            size32(n_slots, "cache"), stream);
        });
    if (!dense) Py_RETURN_NONE;
    return wrap_all(latent, k_pe, mean, rstd);
    END_HANDLE_TH_ERRORS
}

// latent_norm_rope_backward(dlatent, dk_pe, kv_a, gamma, mean, rstd, positions, plan, with_beta, dkv_a | None, workspace | None)
// -> (dkv_a, dgamma, dbeta | None)
PyObject* py_latent_norm_rope_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    arguments(n, 11);
    const Tensor &dlatent = tensor(a[0], "dlatent"), &dk_pe = tensor(a[1], "dk_pe"), &kv_a = tensor(a[2], "kv_a"), &gamma = tensor(a[3], "gamma"),
                 &mean = tensor(a[4], "mean"), &rstd = tensor(a[5], "rstd"), &positions = tensor(a[6], "positions");
    TORCH_CHECK_VALUE(dlatent.dim() == 2 && dk_pe.dim() == 2, "dlatent and dk_pe: expected 2-d tensors, got ", dlatent.sizes(), " and ", dk_pe.sizes());
    const int64_t M = dlatent.size(0), D = dlatent.size(1), R = dk_pe.size(1);
    expect(dlatent, ScalarType::BFloat16, {M, D}, "dlatent");
    expect(dk_pe, ScalarType::BFloat16, {M, R}, "dk_pe");
    const int64_t pitch = rows(kv_a, 2, "kv_a");
    TORCH_CHECK_VALUE(kv_a.size(0) == M && kv_a.size(1) == D + R, "kv_a: expected shape [", M, ", ", D + R, "], got ", kv_a.sizes());
    expect(gamma, ScalarType::BFloat16, {D}, "gamma");
    expect(mean, ScalarType::Float, {M}, "mean");
    expect(rstd, ScalarType::Float, {M}, "rstd");
    const Plan plan(a[7], positions, M);
    plan.is_as_wide_as(R);
    const bool with_beta = truth(a[8]);
    Tensor dkv_a = maybe(a[9], "dkv_a"), workspace = maybe(a[10], "workspace"), dgamma, dbeta;
    if (dkv_a.defined()) expect(dkv_a, ScalarType::BFloat16, {M, D + R}, "dkv_a");
    TORCH_CHECK_VALUE(!workspace.defined() || workspace.is_contiguous(), "workspace: expected a contiguous tensor");
    const c10::Device device = one_device({&dlatent, &dk_pe, &kv_a, &gamma, &mean, &rstd, &positions, &plan.freqs, &dkv_a, &workspace});
    if (!dkv_a.defined()) dkv_a = fresh(dlatent, {M, D + R}, ScalarType::BFloat16);
    if (M == 0) {
        const auto options = mean.options();
        return wrap_all(dkv_a, at::zeros({D}, options), with_beta ? at::zeros({D}, options) : Tensor());
    }
    const int m = size32(M, "dlatent"), d = size32(D, "dlatent");
    if (!workspace.defined()) workspace = fresh(mean, {static_cast<int64_t>(library.backward_workspace_bytes(m, d)) / 4}, ScalarType::Float);
    dgamma = fresh(mean, {D}, ScalarType::Float);
    if (with_beta) dbeta = fresh(mean, {D}, ScalarType::Float);
    enqueue(device, "laga_latent_norm_rope_backward", [&](void* stream) {
        return library.latent_norm_rope_backward(data(dlatent), data(dk_pe), data(kv_a), pitch, data(gamma), data<float>(mean), data<float>(rstd),
                                                 data<int>(positions), data<double>(plan.freqs), m, d, size32(R, "dk_pe"), plan.interleaved,
                                                 plan.mscale, data(dkv_a), data<float>(dgamma), data<float>(dbeta), data(workspace),
                                                 workspace.nbytes(), stream);
    });
    return wrap_all(dkv_a, dgamma, dbeta);
    END_HANDLE_TH_ERRORS
}

// cache_plan(seq_lens, new_lens, block_table, free_pages, n_free, page_size, max_tokens, out | None) -> the six tensors (or out)
PyObject* py_cache_plan(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    arguments(n, 8);
    const Tensor &seq_lens = tensor(a[0], "seq_lens"), &new_lens = tensor(a[1], "new_lens"), &table = tensor(a[2], "block_table"),
                 &free_pages = tensor(a[3], "free_pages"), &n_free = tensor(a[4], "n_free");
    TORCH_CHECK_VALUE(table.dim() == 2, "block_table: expected [n, columns], got ", table.sizes());
    const int64_t requests = table.size(0), columns = table.size(1);
    expect(seq_lens, ScalarType::Int, {requests}, "seq_lens");
    expect(new_lens, ScalarType::Int, {requests}, "new_lens");
    expect(table, ScalarType::Int, {requests, columns}, "block_table");
    expect(free_pages, ScalarType::Int, {free_pages.numel()}, "free_pages");
    expect(n_free, ScalarType::Int, {1}, "n_free");
    const int page_size = integer(a[5]), max_tokens = integer(a[6]);
    if (max_tokens < 1) raise_for(LAGA_ERR_INVALID_ARG, "laga_cache_plan");
    const int64_t sizes[6] = {max_tokens, max_tokens, requests + 1, requests, 1, 1};
    static const char* const names[6] = {"slots", "positions", "cu_new_lens", "seq_lens (out)", "n_free (out)", "status"};
    Tensor out[6];
    if (a[7] != Py_None) {
        TORCH_CHECK_TYPE(PyTuple_Check(a[7]) && PyTuple_GET_SIZE(a[7]) == 6, "out: expected a CachePlan, got ", Py_TYPE(a[7])->tp_name);
        for (int i = 0; i < 6; ++i) {
            out[i] = tensor(PyTuple_GET_ITEM(a[7], i), names[i]);
            expect(out[i], ScalarType::Int, {sizes[i]}, names[i]);
        }
    }
    const c10::Device device = one_device({&seq_lens, &new_lens, &table, &free_pages, &n_free, &out[0], &out[1], &out[2], &out[3], &out[4], &out[5]});
    if (a[7] == Py_None) {
        const Tensor whole = fresh(seq_lens, {2ll * max_tokens + 2 * requests + 3}, ScalarType::Int);
        int64_t offset = 0;
        for (int i = 0; i < 6; offset += sizes[i++]) out[i] = part(whole, offset, sizes[i]);
    }
    if (requests == 0) {                                     // a step of nothing: the entry point takes at least one request
        if (page_size < 16 || page_size > 1024 || (page_size & (page_size - 1)) != 0) raise_for(LAGA_ERR_INVALID_ARG, "laga_cache_plan");
        out[0].fill_(-1);
        for (int i : {1, 2, 5}) out[i].zero_();
        out[4].copy_(n_free);
    } else enqueue(device, "laga_cache_plan", [&](void* stream) {
        return library.cache_plan(data<int>(seq_lens), data<int>(new_lens), size32(requests, "block_table"), page_size, data<int>(table),
                                  size32(columns, "block_table"), data<int>(free_pages), size32(free_pages.numel(), "free_pages"),
                                  data<int>(n_free), max_tokens, data<int>(out[0]), data<int>(out[1]), data<int>(out[2]), data<int>(out[3]),
                                  data<int>(out[4]), data(out[5]), stream);
    });
    if (a[7] != Py_None) return Py_NewRef(a[7]);
    return wrap_all(out[0], out[1], out[2], out[3], out[4], out[5]);
    END_HANDLE_TH_ERRORS
}

// paged_decode(q, w_kv_b, cache, block_table, seq_lens, softmax_scale | None, out | None, lse | None, workspace | None)
// -> (out, lse | None, workspace)
PyObject* py_paged_decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    arguments(n, 9);
    const Tensor &q = tensor(a[0], "q"), &w = tensor(a[1], "w_kv_b"), &cache = tensor(a[2], "cache"), &table = tensor(a[3], "block_table"),
                 &seq_lens = tensor(a[4], "seq_lens");
    TORCH_CHECK_VALUE(q.dim() == 3 && w.dim() == 2 && cache.dim() == 3 && table.dim() == 2, "paged_decode: expected q [B, h, d], w_kv_b [d_c, n], ",
                      "cache [pages, page_size, row] and block_table [B, columns], got ", q.sizes(), ", ", w.sizes(), ", ", cache.sizes(), ", ",
                      table.sizes());
    const int64_t B = q.size(0), h = q.size(1), d_qk = q.size(2), d_c = w.size(0), d_rope = cache.size(2) - d_c, d_nope = d_qk - d_rope,
                  d_v = h > 0 ? w.size(1) / h - d_nope : 0;
    TORCH_CHECK_VALUE(h > 0, "q: no heads");
    expect(q, ScalarType::BFloat16, {B, h, d_qk}, "q");
    expect(cache, ScalarType::BFloat16, cache.sizes(), "cache");
    expect(w, ScalarType::BFloat16, {d_c, h * (d_nope + d_v)}, "w_kv_b");
    expect(table, ScalarType::Int, {B, table.size(1)}, "block_table");
    expect(seq_lens, ScalarType::Int, {B}, "seq_lens");
    Tensor out = maybe(a[6], "out"), lse = maybe(a[7], "lse"), workspace = maybe(a[8], "workspace");
    const double scale = a[5] == Py_None ? std::pow(static_cast<double>(d_qk), -0.5) : number(a[5]);
    if (out.defined()) expect(out, ScalarType::BFloat16, {B, h, d_v}, "out");
    if (lse.defined()) expect(lse, ScalarType::Float, {B, h}, "lse");
    TORCH_CHECK_VALUE(!workspace.defined() || workspace.is_contiguous(), "workspace: expected a contiguous tensor");
    const c10::Device device = one_device({&q, &w, &cache, &table, &seq_lens, &out, &lse, &workspace});
    const int b = size32(B, "q"), heads = size32(h, "q"), dims[4] = {size32(d_c, "w_kv_b"), size32(d_nope, "q"), size32(d_rope, "cache"), size32(d_v, "w_kv_b")};
    const size_t need = library.decode_workspace_bytes(b > 0 ? b : 1, heads, dims[0], dims[1], dims[2], dims[3]);
    if (need == 0) raise_for(LAGA_ERR_UNSUPPORTED, "laga_paged_decode_workspace_bytes");
    if (B == 0) {                                            // nothing to do: a status word that says so
        if (!out.defined()) out = fresh(q, {0, h, d_v}, ScalarType::BFloat16);
        if (workspace.defined()) workspace.flatten().narrow(0, 0, std::min<int64_t>(workspace.numel(), 4)).zero_();
        else workspace = at::zeros({1024}, q.options().dtype(ScalarType::Byte));
        return wrap_all(out, lse, workspace);
    }
    if (!workspace.defined()) workspace = workspace_of(q, need);
    if (!out.defined()) out = fresh(q, {B, h, d_v}, ScalarType::BFloat16);
    enqueue(device, "laga_paged_decode", [&](void* stream) {
        return library.paged_decode(data(q), data(w), data(cache), size32(cache.size(0), "cache"), size32(cache.size(1), "cache"), data<int>(table),
                                    size32(table.size(1), "block_table"), data<int>(seq_lens), b, heads, dims[0], dims[1], dims[2], dims[3],
                                    static_cast<float>(scale), data(out), data<float>(lse), data(workspace), workspace.nbytes(), 0, stream);
    });
    return wrap_all(out, lse, workspace);
    END_HANDLE_TH_ERRORS
}

// bind(fail, address, ...): the addresses in the order of `Library`
PyObject* py_bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    constexpr Py_ssize_t kEntries = sizeof(Library) / sizeof(void*);
    arguments(n, 1 + kEntries);
    void* address[kEntries];
    for (Py_ssize_t i = 0; i < kEntries; ++i) {
        address[i] = PyLong_AsVoidPtr(a[1 + i]);
        if (address[i] == nullptr && PyErr_Occurred()) throw python_error();
        TORCH_CHECK_VALUE(address[i] != nullptr, "bind: no address");
    }
    static_assert(sizeof(library) == sizeof(address), "one address per entry point");
    memcpy(&library, address, sizeof(library));
    Py_XSETREF(fail, Py_NewRef(a[0]));
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

template <PyObject* (*f)(PyObject*, PyObject* const*, Py_ssize_t)>
PyMethodDef method(const char* name) {
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr};
}
PyMethodDef methods[] = {method<py_bind>("bind"),
                         method<py_rope>("rope"),
                         method<py_latent_norm_rope>("latent_norm_rope"),
                         method<py_latent_norm_rope_backward>("latent_norm_rope_backward"),
                         method<py_cache_plan>("cache_plan"),
                         method<py_paged_decode>("paged_decode"),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
