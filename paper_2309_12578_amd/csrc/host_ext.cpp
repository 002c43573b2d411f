// Native call path of the Python front end (module _spion_host): argument checks, output and workspace
// allocation from torch's caching allocator, and the autograd node, around the entry points of libspion.
// A forward + backward of a small problem is bound by the host: through ctypes and a Python autograd
// function it took 147 us of host time for 20 us of kernels.
//
// Plain CPython calling convention (METH_FASTCALL) and direct allocation: no dispatcher, no argument
// parsing by format strings.
#include <Python.h>

#include <cmath>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/autocast_mode.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPCachingAllocator.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/function.h>
#include <torch/csrc/autograd/functions/utils.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/autograd/saved_variable.h>
#include <torch/csrc/autograd/variable.h>
#include <torch/csrc/jit/frontend/tracer.h>

#include "spion_host.h"

namespace {

PyObject* g_error_class = nullptr;   // SpionError

// Sets SpionError(code, what); always returns nullptr.
PyObject* spion_error(int code, const char* what) {
    PyObject* e = g_error_class ? PyObject_CallFunction(g_error_class, "is", code, what) : nullptr;
    if (e) {
        PyErr_SetObject(g_error_class, e);
        Py_DECREF(e);
    } else if (!PyErr_Occurred()) {
        PyErr_Format(PyExc_RuntimeError, "%s: %s (%d)", what, spion_strerror(code), code);
    }
    return nullptr;
}

struct SpionFailure {   // thrown with the Python error to set
    int code;
    const char* what;
};

struct BadValue {   // thrown for a ValueError
    const char* msg;
};
[[noreturn]] void bad_value(const char* msg) { throw BadValue{msg}; }

void* device_ptr(const at::Tensor& t) {
    if (!t.is_cuda() || !t.is_contiguous()) bad_value("libspion needs contiguous device tensors");
    return t.data_ptr();
}

const at::Tensor& tensor_arg(PyObject* o) {
    if (!THPVariable_Check(o)) bad_value("libspion needs contiguous device tensors");
    return THPVariable_Unpack(o);
}
at::Tensor optional_arg(PyObject* o) { return o == Py_None ? at::Tensor() : tensor_arg(o); }

int int_arg(PyObject* o) {
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) throw python_error();
    return (int)v;
}
double double_arg(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw python_error();
    return v;
}

bool truth_arg(PyObject* o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw python_error();
    return v == 1;
}

void* current_stream() { return c10::hip::getCurrentHIPStream().stream(); }

at::Tensor new_like(const at::Tensor& t) {
    return at::Tensor(at::detail::empty_cuda(t.sizes(), t.scalar_type(), t.device(), std::nullopt));
}
at::Tensor new_bytes(size_t n, const at::Tensor& like) {
    return at::Tensor(at::detail::empty_cuda({(int64_t)(n < 256 ? 256 : n)}, at::kByte, like.device(), std::nullopt));
}

// One pattern index and the parameters of a call.
struct Index {
    at::Tensor row_ptr, col_idx, col_ptr, row_idx, bsr_pos;
    int nnzb = 0, block = 0;
    float scale = 0.f;
    unsigned flags = 0;
};

spion_attn_params params_of(const at::Tensor& q, const Index& ix) {
    if (q.dim() != 4) bad_value("expected tensors of shape [B, H, L, d]");
    spion_attn_params p;
    p.B = (int32_t)q.size(0);
    p.H = (int32_t)q.size(1);
    p.L = (int32_t)q.size(2);
    p.d = (int32_t)q.size(3);
    p.block = ix.block;
    if (q.scalar_type() == at::kFloat) p.dtype = SPION_F32;
    else if (q.scalar_type() == at::kBFloat16) p.dtype = SPION_BF16;
    else bad_value("unsupported dtype");
    p.scale = ix.scale;
    p.flags = ix.flags;
    return p;
}

// The kernels take every size from Q: a smaller tensor beside it would be read or written past its end.  A larger one,
// a buffer kept for several shapes, has its first elements used.
void room_for(const at::Tensor& q, const at::Tensor& t) {
    if (t.numel() < q.numel() || t.scalar_type() != q.scalar_type())
        bad_value("Q's companions must have its dtype and at least as many elements");
}
void room_for_rows(const at::Tensor& q, const at::Tensor& lse) {
    if (lse.numel() * q.size(3) < q.numel() || lse.scalar_type() != at::kFloat)
        bad_value("LSE must be fp32 with at least B * H * L elements");
}

// For the pieces of long rows (spion_attn_fwd_room), of this call alone: back to the allocator, in the order of the stream,
// when the call returns.
struct Room {
    c10::DataPtr memory;
    size_t bytes;
    void* ptr = nullptr;
    Room(const spion_attn_params& p, int nnzb) : bytes(spion_attn_fwd_room_bytes(&p, nnzb)) {
        if (bytes == 0) return;
        memory = c10::hip::HIPCachingAllocator::get()->allocate(bytes);
        ptr = memory.get();
    }
};

void forward(const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, const Index& ix, at::Tensor& o, at::Tensor& lse) {
    device_ptr(q);
    const spion_attn_params p = params_of(q, ix);
    room_for(q, k);
    room_for(q, v);
    if (!o.defined()) o = new_like(q);
    else room_for(q, o);
    if (!lse.defined())
        lse = at::Tensor(at::detail::empty_cuda({q.size(0), q.size(1), q.size(2)}, at::kFloat, q.device(), std::nullopt));
    else room_for_rows(q, lse);
    const Room room(p, ix.nnzb);
    const int rc = spion_attn_fwd_room(device_ptr(q), device_ptr(k), device_ptr(v), device_ptr(o), (float*)device_ptr(lse),
                                       (const int32_t*)device_ptr(ix.row_ptr), (const int32_t*)device_ptr(ix.col_idx),
                                       ix.nnzb, &p, room.ptr, room.bytes, current_stream());
    if (rc != SPION_OK) throw SpionFailure{rc, "spion_attn_fwd"};
}

void backward(const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, const at::Tensor& o, const at::Tensor& grad,
              const at::Tensor& lse, const Index& ix, at::Tensor& dq, at::Tensor& dk, at::Tensor& dv, at::Tensor& ws) {
    device_ptr(q);
    const spion_attn_params p = params_of(q, ix);
    for (const at::Tensor* t : {&k, &v, &o, &grad}) room_for(q, *t);
    room_for_rows(q, lse);
    for (at::Tensor* t : {&dq, &dk, &dv}) {
        if (!t->defined()) *t = new_like(q);
        else room_for(q, *t);
    }
    if (!ws.defined()) {
        const size_t n = spion_attn_workspace_bytes(&p, ix.nnzb, 1);
        if (n == (size_t)-1) throw SpionFailure{SPION_ERR_SHAPE, "spion_attn_workspace_bytes"};
        ws = new_bytes(n, q);
    }
    const int rc = spion_attn_bwd(device_ptr(q), device_ptr(k), device_ptr(v), device_ptr(o), device_ptr(grad),
                                  (const float*)device_ptr(lse), device_ptr(dq), device_ptr(dk), device_ptr(dv),
                                  (const int32_t*)device_ptr(ix.row_ptr), (const int32_t*)device_ptr(ix.col_idx),
                                  (const int32_t*)device_ptr(ix.col_ptr), (const int32_t*)device_ptr(ix.row_idx),
                                  (const int32_t*)device_ptr(ix.bsr_pos), ix.nnzb, &p, device_ptr(ws),
                                  (size_t)ws.nbytes(), current_stream());
    if (rc != SPION_OK) throw SpionFailure{rc, "spion_attn_bwd"};
}

template <class F>
PyObject* torch_guarded(F&& f) {
    HANDLE_TH_ERRORS
    return f();
    END_HANDLE_TH_ERRORS
}
// Runs f with C++ failures turned into Python errors.
template <class F>
PyObject* guarded(F&& f) {
    try {
        return torch_guarded(f);
    } catch (const SpionFailure& e) {
        return spion_error(e.code, e.what);
    } catch (const BadValue& e) {
        PyErr_SetString(PyExc_ValueError, e.msg);
        return nullptr;
    }
}

bool arg_count(Py_ssize_t got, Py_ssize_t want, const char* name) {
    if (got == want) return true;
    PyErr_Format(PyExc_TypeError, "%s takes %zd arguments, got %zd", name, want, got);
    return false;
}

PyObject* wrap(const at::Tensor& t) { return THPVariable_Wrap(t); }

// attn_fwd(Q, K, V, row_ptr, col_idx, nnzb, block, scale, flags, O | None, LSE | None) -> (O, LSE)
PyObject* py_attn_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arg_count(n, 11, "attn_fwd")) return nullptr;
    return guarded([&]() -> PyObject* {
        Index ix;
        ix.row_ptr = tensor_arg(a[3]);
        ix.col_idx = tensor_arg(a[4]);
        ix.nnzb = int_arg(a[5]);
        ix.block = int_arg(a[6]);
        ix.scale = (float)double_arg(a[7]);
        ix.flags = (unsigned)int_arg(a[8]);
        at::Tensor o = optional_arg(a[9]), lse = optional_arg(a[10]);
        forward(tensor_arg(a[0]), tensor_arg(a[1]), tensor_arg(a[2]), ix, o, lse);
        PyObject* r = PyTuple_New(2);
        if (!r) return nullptr;
        PyTuple_SET_ITEM(r, 0, wrap(o));
        PyTuple_SET_ITEM(r, 1, wrap(lse));
        return r;
    });
}

// attn_bwd(Q, K, V, O, dO, LSE, row_ptr, col_idx, col_ptr, row_idx, bsr_pos, nnzb, block, scale, flags,
//          dQ | None, dK | None, dV | None, workspace | None) -> (dQ, dK, dV)
PyObject* py_attn_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arg_count(n, 19, "attn_bwd")) return nullptr;
    return guarded([&]() -> PyObject* {
        Index ix;
        ix.row_ptr = tensor_arg(a[6]);
        ix.col_idx = tensor_arg(a[7]);
        ix.col_ptr = tensor_arg(a[8]);
        ix.row_idx = tensor_arg(a[9]);
        ix.bsr_pos = tensor_arg(a[10]);
        ix.nnzb = int_arg(a[11]);
        ix.block = int_arg(a[12]);
        ix.scale = (float)double_arg(a[13]);
        ix.flags = (unsigned)int_arg(a[14]);
        at::Tensor dq = optional_arg(a[15]), dk = optional_arg(a[16]), dv = optional_arg(a[17]), ws = optional_arg(a[18]);
        backward(tensor_arg(a[0]), tensor_arg(a[1]), tensor_arg(a[2]), tensor_arg(a[3]), tensor_arg(a[4]),
                 tensor_arg(a[5]), ix, dq, dk, dv, ws);
        PyObject* r = PyTuple_New(3);
        if (!r) return nullptr;
        PyTuple_SET_ITEM(r, 0, wrap(dq));
        PyTuple_SET_ITEM(r, 1, wrap(dk));
        PyTuple_SET_ITEM(r, 2, wrap(dv));
        return r;
    });
}

// The gradient of sparse_attention.  Saves what the backward entry point takes; one pass computes all three.
struct SparseAttentionBackward : public torch::autograd::Node {
    torch::autograd::SavedVariable q, k, v, o, lse;
    Index ix;

    std::string name() const override { return "SparseAttentionBackward"; }

    void release_variables() override {
        for (torch::autograd::SavedVariable* s : {&q, &k, &v, &o, &lse}) s->reset_data();
    }

    torch::autograd::variable_list apply(torch::autograd::variable_list&& grads) override {
        torch::autograd::variable_list out(3);
        const at::Tensor& g = grads[0];
        if (!g.defined()) return out;
        at::NoGradGuard no_grad;   // the gradients are not differentiated again
        at::Tensor ws;
        try {
            backward(q.unpack(), k.unpack(), v.unpack(), o.unpack(shared_from_this()), g.contiguous(), lse.unpack(), ix,
                     out[0], out[1], out[2], ws);
        } catch (const SpionFailure& e) {
            PyGILState_STATE gil = PyGILState_Ensure();
            spion_error(e.code, e.what);
            python_error err;
            err.persist();
            PyGILState_Release(gil);
            throw err;
        } catch (const BadValue& e) {
            TORCH_CHECK_VALUE(false, e.msg);
        }
        return out;
    }
};

// sparse_attention(Q, K, V, row_ptr, col_idx, col_ptr, row_idx, bsr_pos, nnzb, block, scale, flags) -> O, or None under
// torch.jit.trace: what is allocated and launched here is not seen by the tracer, which would record O as a constant.
PyObject* py_sparse_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arg_count(n, 12, "sparse_attention")) return nullptr;
    return guarded([&]() -> PyObject* {
        if (torch::jit::tracer::isTracing()) Py_RETURN_NONE;
        const at::Tensor &q = tensor_arg(a[0]), &k = tensor_arg(a[1]), &v = tensor_arg(a[2]);
        Index ix;
        ix.row_ptr = tensor_arg(a[3]);
        ix.col_idx = tensor_arg(a[4]);
        ix.nnzb = int_arg(a[8]);
        ix.block = int_arg(a[9]);
        ix.scale = (float)double_arg(a[10]);
        ix.flags = (unsigned)int_arg(a[11]);
        for (const at::Tensor* t : {&q, &k, &v})
            if (t->_fw_grad(0).defined()) {
                PyErr_SetString(PyExc_NotImplementedError, "sparse_attention has no forward-mode derivative");
                return nullptr;
            }
        const bool grad = torch::autograd::compute_requires_grad(q, k, v);
        at::Tensor o, lse, qc, kc, vc;
        {
            at::NoGradGuard no_grad;
            qc = q.contiguous();
            kc = k.contiguous();
            vc = v.contiguous();
            forward(qc, kc, vc, ix, o, lse);
        }
        if (grad) {
            ix.col_ptr = tensor_arg(a[5]);
            ix.row_idx = tensor_arg(a[6]);
            ix.bsr_pos = tensor_arg(a[7]);
            auto node = std::shared_ptr<SparseAttentionBackward>(new SparseAttentionBackward(), torch::autograd::deleteNode);
            node->set_next_edges(torch::autograd::collect_next_edges(q, k, v));
            node->q = torch::autograd::SavedVariable(qc, false);
            node->k = torch::autograd::SavedVariable(kc, false);
            node->v = torch::autograd::SavedVariable(vc, false);
            node->lse = torch::autograd::SavedVariable(lse, false);
            node->ix = std::move(ix);
            torch::autograd::set_history(o, node);
            node->o = torch::autograd::SavedVariable(o, true);
        }
        return wrap(o);
    });
}

// Whether torch is only computing: nobody traces, transforms, casts or watches its operators.
bool nothing_between() {
    using c10::DispatchKey;
    if (c10::impl::TorchDispatchModeTLS::any_modes_set() || at::impl::torch_function_mode_enabled()) return false;
    for (DispatchKey k : {DispatchKey::FuncTorchDynamicLayerFrontMode, DispatchKey::Functionalize, DispatchKey::Tracer})
        if (c10::impl::tls_is_dispatch_key_included(k)) return false;
    return !at::autocast::is_autocast_enabled(at::kCUDA);
}
// A plain strided tensor on the current device (whose stream the library is given): no subclass, no wrapper of a
// transform, no view whose values are not those in memory, no tangent.
bool plain(const at::Tensor& t) {
    using c10::DispatchKey;
    for (DispatchKey k : {DispatchKey::Python, DispatchKey::Functionalize, DispatchKey::FuncTorchBatched, DispatchKey::Batched,
                          DispatchKey::FuncTorchGradWrapper, DispatchKey::Negative, DispatchKey::ZeroTensor})
        if (t.key_set().has(k)) return false;
    return t.is_cuda() && t.get_device() == c10::hip::current_device() && t.layout() == at::kStrided && !t._fw_grad(0).defined();
}
bool plain(PyObject* o) { return THPVariable_CheckExact(o) && plain(THPVariable_Unpack(o)); }

// Whether a backward pass may compute in kernels of the library: it is not differentiated itself, backward (grad mode)
// or forward (a tangent on the incoming gradient), nor batched over incoming gradients, nor watched.
bool kernels_may_differentiate(const at::Tensor& grad) {
    return !at::GradMode::is_enabled() && nothing_between() && plain(grad);
}

// The gradient of Y = X W^T + b.  The weight's comes from spion_weight_grad where only numbers are wanted, else, as
// the others, from torch operators.
struct ProjectionBackward : public torch::autograd::Node {
    torch::autograd::SavedVariable x, w;
    bool has_bias = false;

    std::string name() const override { return "ProjectionBackward"; }

    void release_variables() override {
        x.reset_data();
        w.reset_data();
    }

    torch::autograd::variable_list apply(torch::autograd::variable_list&& grads) override {
        torch::autograd::variable_list out(has_bias ? 3 : 2);
        if (!grads[0].defined()) return out;
        const at::Tensor X = x.unpack(), W = w.unpack();
        const int64_t N = W.size(0), M = W.size(1);
        const at::Tensor g = grads[0].reshape({-1, N}), x2 = X.reshape({-1, M});
        if (task_should_compute_output(0)) out[0] = at::mm(g, W).view(X.sizes());
        if (task_should_compute_output(1)) {
            const bool kernel = kernels_may_differentiate(grads[0]) && plain(X);
            out[1] = kernel ? weight_grad(g.contiguous(), x2.contiguous()) : at::mm(g.t(), x2);
        }
        if (has_bias && task_should_compute_output(2)) out[2] = g.sum(0);
        return out;
    }

    static at::Tensor weight_grad(const at::Tensor& g, const at::Tensor& x) {
        const int rows = (int)x.size(0), N = (int)g.size(1), M = (int)x.size(1);
        at::Tensor dw(at::detail::empty_cuda({N, M}, x.scalar_type(), x.device(), std::nullopt));
        const at::Tensor ws = new_bytes(spion_weight_grad_workspace_bytes(rows, N, M), x);
        const int rc = spion_weight_grad(g.data_ptr(), x.data_ptr(), dw.data_ptr(), rows, N, M, ws.data_ptr(),
                                         (size_t)ws.nbytes(), current_stream());
        if (rc == SPION_ERR_PARAM) return at::mm(g.t(), x);   // an operand that is not aligned to 16 bytes
        TORCH_CHECK(rc == SPION_OK, "spion_weight_grad: ", spion_strerror(rc));
        return dw;
    }
};

void heads(bool split, const at::Tensor& merged, const at::Tensor* t, int n) {   // see spion_heads
    void* ptr[3];
    for (int i = 0; i < n; ++i) ptr[i] = t[i].data_ptr();
    const int rc = spion_heads(split, merged.data_ptr(), ptr, (int)t[0].size(0), (int)t[0].size(2), (int)t[0].size(1), n,
                               t[0].scalar_type() == at::kFloat ? SPION_F32 : SPION_BF16, current_stream());
    if (rc != SPION_OK) throw SpionFailure{rc, "spion_heads"};
}

at::Tensor new_heads(const at::Tensor& like, int64_t B, int64_t H, int64_t L) {
    return at::Tensor(at::detail::empty_cuda({B, H, L, 64}, like.scalar_type(), like.device(), std::nullopt));
}

// The kernels read and write the heads where the projections have them (spion_heads_attn_*); for other types and block
// sizes a head split and a head merge go around them.  8 x 2048 tokens, 4 heads, block 32: the sub-layer's step moves
// 26 us of copies less.
bool heads_in_place(const at::Tensor& qkv, const Index& ix) {
    return qkv.scalar_type() == at::kBFloat16 && (ix.block == 32 || ix.block == 64);
}
spion_attn_params heads_params(const at::Tensor& qkv, int64_t H, const Index& ix) {
    spion_attn_params p;
    p.B = (int32_t)qkv.size(0);
    p.H = (int32_t)H;
    p.L = (int32_t)qkv.size(1);
    p.d = 64;
    p.block = ix.block;
    p.dtype = SPION_BF16;
    p.scale = ix.scale;
    p.flags = ix.flags;
    return p;
}

// The gradient of heads_attention.
struct HeadsAttentionBackward : public torch::autograd::Node {
    torch::autograd::SavedVariable q, k, v, o, lse;   // in place: q = qkv, o = the node's output, no k and v
    Index ix;
    int64_t H = 0;
    bool in_place = false;

    std::string name() const override { return "HeadsAttentionBackward"; }

    void release_variables() override {
        for (torch::autograd::SavedVariable* s : {&q, &k, &v, &o, &lse}) s->reset_data();
    }

    torch::autograd::variable_list apply(torch::autograd::variable_list&& grads) override {
        torch::autograd::variable_list out(1);
        if (!grads[0].defined()) return out;
        at::NoGradGuard no_grad;   // the gradients are not differentiated again
        at::Tensor g = grads[0].contiguous(), d[3], ws;
        if ((uintptr_t)g.data_ptr() % 16 != 0) g = g.clone();
        const at::Tensor Q = q.unpack(), O = in_place ? o.unpack(shared_from_this()) : o.unpack();
        const int64_t B = Q.size(0), L = Q.size(in_place ? 1 : 2);
        try {
            if (in_place) {
                const spion_attn_params p = heads_params(Q, H, ix);
                const at::Tensor stat = lse.unpack();
                // what saved-tensor hooks hand back is looked at as the node's own tensors were
                if (Q.dim() != 3 || Q.size(2) != 3 * H * 64 || Q.scalar_type() != at::kBFloat16 || 3 * O.numel() != Q.numel() ||
                    O.scalar_type() != at::kBFloat16 || 3 * g.numel() != Q.numel() || g.scalar_type() != at::kBFloat16 ||
                    stat.numel() != B * H * L || stat.scalar_type() != at::kFloat)
                    bad_value("heads_attention: a saved tensor is not the one that was saved");
                const size_t n = spion_attn_workspace_bytes(&p, ix.nnzb, 1);
                if (n == (size_t)-1) throw SpionFailure{SPION_ERR_SHAPE, "spion_attn_workspace_bytes"};
                ws = new_bytes(n, Q);
                out[0] = new_like(Q);
                const int rc = spion_heads_attn_bwd(
                    device_ptr(Q), device_ptr(O), device_ptr(g), (const float*)device_ptr(stat), device_ptr(out[0]),
                    (const int32_t*)device_ptr(ix.row_ptr), (const int32_t*)device_ptr(ix.col_idx),
                    (const int32_t*)device_ptr(ix.col_ptr), (const int32_t*)device_ptr(ix.row_idx), ix.nnzb, &p,
                    device_ptr(ws), (size_t)ws.nbytes(), current_stream());
                if (rc != SPION_OK) throw SpionFailure{rc, "spion_heads_attn_bwd"};
                return out;
            }
            const at::Tensor dO = new_heads(Q, B, H, L);
            heads(true, g, &dO, 1);
            backward(Q, k.unpack(), v.unpack(), O, dO, lse.unpack(), ix, d[0], d[1], d[2], ws);
            out[0] = at::Tensor(at::detail::empty_cuda({B, L, 3 * H * 64}, Q.scalar_type(), Q.device(), std::nullopt));
            heads(false, out[0], d, 3);
        } catch (const SpionFailure& e) {
            PyGILState_STATE gil = PyGILState_Ensure();
            spion_error(e.code, e.what);
            python_error err;
            err.persist();
            PyGILState_Release(gil);
            throw err;
        } catch (const BadValue& e) {
            TORCH_CHECK_VALUE(false, e.msg);
        }
        return out;
    }
};

// heads_attention(qkv [B, L, 3 H 64], H, row_ptr, col_idx, col_ptr, row_idx, bsr_pos, nnzb, block, flags, apart = False)
// -> [B, L, H 64]: every head's attention as one node; None where the steps are to be taken one by one (see projection).
// apart: the node saves copies, so that the caller may let qkv and the result be changed in place before the backward pass.
PyObject* py_heads_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 11 && !arg_count(n, 10, "heads_attention")) return nullptr;
    return guarded([&]() -> PyObject* {
        if (!nothing_between() || !plain(a[0])) Py_RETURN_NONE;
        const at::Tensor& qkv = THPVariable_Unpack(a[0]);
        const int64_t H = int_arg(a[1]);
        const bool f32 = qkv.scalar_type() == at::kFloat;
        if ((!f32 && qkv.scalar_type() != at::kBFloat16) || qkv.dim() != 3 || !qkv.is_contiguous() || H <= 0 ||
            qkv.size(2) != 3 * H * 64 || qkv.size(1) % 4 != 0 || qkv.numel() == 0 ||
            qkv.numel() / (f32 ? 4 : 8) >= 0x7fffffffll || (uintptr_t)qkv.data_ptr() % 16 != 0)
            Py_RETURN_NONE;
        const int64_t B = qkv.size(0), L = qkv.size(1);
        Index ix;
        ix.row_ptr = tensor_arg(a[2]);
        ix.col_idx = tensor_arg(a[3]);
        ix.nnzb = int_arg(a[7]);
        ix.block = int_arg(a[8]);
        ix.flags = (unsigned)int_arg(a[9]);
        const bool grad = torch::autograd::compute_requires_grad(qkv);
        const bool in_place = heads_in_place(qkv, ix) && !(grad && n == 11 && a[10] == Py_True);
        at::Tensor t[3], o, lse, s;
        if (in_place) {
            const spion_attn_params p = heads_params(qkv, H, ix);
            s = at::Tensor(at::detail::empty_cuda({B, L, H * 64}, qkv.scalar_type(), qkv.device(), std::nullopt));
            lse = at::Tensor(at::detail::empty_cuda({B, H, L}, at::kFloat, qkv.device(), std::nullopt));
            const Room room(p, ix.nnzb);
            const int rc = spion_heads_attn_fwd(device_ptr(qkv), device_ptr(s), (float*)device_ptr(lse),
                                                (const int32_t*)device_ptr(ix.row_ptr), (const int32_t*)device_ptr(ix.col_idx),
                                                ix.nnzb, &p, room.ptr, room.bytes, current_stream());
            if (rc != SPION_OK) throw SpionFailure{rc, "spion_heads_attn_fwd"};
        } else {
            at::NoGradGuard no_grad;
            for (at::Tensor& x : t) x = new_heads(qkv, B, H, L);
            heads(true, qkv, t, 3);
            forward(t[0], t[1], t[2], ix, o, lse);
            s = at::Tensor(at::detail::empty_cuda({B, L, H * 64}, qkv.scalar_type(), qkv.device(), std::nullopt));
            heads(false, s, &o, 1);
        }
        if (grad) {
            ix.col_ptr = tensor_arg(a[4]);
            ix.row_idx = tensor_arg(a[5]);
            ix.bsr_pos = tensor_arg(a[6]);
            auto node = std::shared_ptr<HeadsAttentionBackward>(new HeadsAttentionBackward(), torch::autograd::deleteNode);
            node->set_next_edges(torch::autograd::collect_next_edges(qkv));
            node->H = H;
            node->in_place = in_place;
            node->lse = torch::autograd::SavedVariable(lse, false);
            node->ix = std::move(ix);
            torch::autograd::set_history(s, node);
            if (in_place) {
                node->q = torch::autograd::SavedVariable(qkv, false);
                node->o = torch::autograd::SavedVariable(s, true);
            } else {
                node->q = torch::autograd::SavedVariable(t[0], false);
                node->k = torch::autograd::SavedVariable(t[1], false);
                node->v = torch::autograd::SavedVariable(t[2], false);
                node->o = torch::autograd::SavedVariable(o, false);
            }
        }
        return wrap(s);
    });
}

// A norm's node, which can take the gradient of a residual from its input as its second (see residual).
struct TakesResidual : public torch::autograd::Node {};

// The gradient of layer_norm, all three in one pass over X and dY; torch's operator where more than numbers is wanted.  A
// second incoming gradient is that of a residual from X (see residual), whose sum with dX the same pass writes.
struct NormBackward : public TakesResidual {
    torch::autograd::SavedVariable x, w, b, mean, rstd;

    std::string name() const override { return "NormBackward"; }

    void release_variables() override {
        for (torch::autograd::SavedVariable* s : {&x, &w, &b, &mean, &rstd}) s->reset_data();
    }

    torch::autograd::variable_list apply(torch::autograd::variable_list&& grads) override {
        torch::autograd::variable_list out(3);
        const at::Tensor dr = grads.size() > 1 ? grads[1] : at::Tensor();
        if (!grads[0].defined()) {
            out[0] = dr;
            return out;
        }
        const at::Tensor X = x.unpack(), W = w.unpack(), m = mean.unpack(), r = rstd.unpack();
        const int64_t D = W.size(0);
        const at::Tensor g = grads[0].contiguous();
        if (!kernels_may_differentiate(grads[0]) || !plain(X) || !plain(W) || (uintptr_t)g.data_ptr() % 16 != 0) {
            std::vector<int64_t> stat(X.sizes().begin(), X.sizes().end());
            stat.back() = 1;
            std::tie(out[0], out[1], out[2]) = at::native_layer_norm_backward(
                g, X, {D}, m.view(stat), r.view(stat), W, b.unpack(),
                {task_should_compute_output(0), task_should_compute_output(1), task_should_compute_output(2)});
            if (dr.defined() && out[0].defined()) out[0] = out[0] + dr;   // X's gradient may not be asked for
            return out;
        }
        const bool add = dr.defined() && plain(dr) && dr.scalar_type() == X.scalar_type() && dr.is_contiguous() &&
                         dr.sizes() == X.sizes() && (uintptr_t)dr.data_ptr() % 16 == 0;
        const int rows = (int)(X.numel() / D);
        for (at::Tensor* t : {&out[0], &out[1], &out[2]}) *t = new_like(t == &out[0] ? X : W);
        const at::Tensor ws = new_bytes(spion_layer_norm_workspace_bytes(rows, (int)D), X);
        const int rc = spion_layer_norm_grad(g.data_ptr(), add ? dr.data_ptr() : nullptr, X.data_ptr(), W.data_ptr(), m.data_ptr<float>(), r.data_ptr<float>(),
                                             out[0].data_ptr(), out[1].data_ptr(), out[2].data_ptr(), rows, (int)D,
                                             X.scalar_type() == at::kFloat ? SPION_F32 : SPION_BF16, ws.data_ptr(),
                                             (size_t)ws.nbytes(), current_stream());
        TORCH_CHECK(rc == SPION_OK, "spion_layer_norm_grad: ", spion_strerror(rc));
        if (dr.defined() && !add) out[0] = out[0] + dr;
        for (int i = 0; i < 3; ++i)
            if (!task_should_compute_output(i)) out[i].reset();
        return out;
    }
};

// layer_norm(X, w, b, eps) -> Y over the last dimension, or None where torch's operator is to be called (see projection).
PyObject* py_layer_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arg_count(n, 4, "layer_norm")) return nullptr;
    return guarded([&]() -> PyObject* {
        if (!nothing_between() || !plain(a[0]) || !plain(a[1]) || !plain(a[2])) Py_RETURN_NONE;
        const at::Tensor &x = THPVariable_Unpack(a[0]), &w = THPVariable_Unpack(a[1]), &b = THPVariable_Unpack(a[2]);
        const auto type = x.scalar_type();
        if ((type != at::kFloat && type != at::kBFloat16) || w.scalar_type() != type || b.scalar_type() != type ||
            x.device() != w.device() || x.device() != b.device() || w.dim() != 1 || x.dim() < 2 || x.numel() == 0)
            Py_RETURN_NONE;
        const int64_t D = w.size(0);
        if (b.dim() != 1 || b.size(0) != D || x.size(-1) != D || D % 64 != 0 || D > 2048 || x.numel() / D > 0x40000000 ||
            !x.is_contiguous() || !w.is_contiguous() || !b.is_contiguous() ||
            ((uintptr_t)x.data_ptr() | (uintptr_t)w.data_ptr() | (uintptr_t)b.data_ptr()) % 16 != 0)
            Py_RETURN_NONE;
        const int64_t rows = x.numel() / D;
        at::Tensor y = new_like(x), mean(at::detail::empty_cuda({rows}, at::kFloat, x.device(), std::nullopt)),
                   rstd(at::detail::empty_cuda({rows}, at::kFloat, x.device(), std::nullopt));
        const int rc = spion_layer_norm(x.data_ptr(), w.data_ptr(), b.data_ptr(), y.data_ptr(), mean.data_ptr<float>(),
                                        rstd.data_ptr<float>(), (int)rows, (int)D, (float)double_arg(a[3]),
                                        type == at::kFloat ? SPION_F32 : SPION_BF16, current_stream());
        if (rc != SPION_OK) throw SpionFailure{rc, "spion_layer_norm"};
        if (torch::autograd::compute_requires_grad(x, w, b)) {
            auto node = std::shared_ptr<NormBackward>(new NormBackward(), torch::autograd::deleteNode);
            node->set_next_edges(torch::autograd::collect_next_edges(x, w, b));
            node->x = torch::autograd::SavedVariable(x, false);
            node->w = torch::autograd::SavedVariable(w, false);
            node->b = torch::autograd::SavedVariable(b, false);
            node->mean = torch::autograd::SavedVariable(mean, false);
            node->rstd = torch::autograd::SavedVariable(rstd, false);
            torch::autograd::set_history(y, node);
        }
        return wrap(y);
    });
}

// residual(X, Y) -> X for a residual around Y = layer_norm(X) or rms_norm(X): an alias whose gradient goes to Y's node, which adds it to
// its own, instead of an addition after it; X itself where Y did not come from that node alone.
PyObject* py_residual(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arg_count(n, 2, "residual")) return nullptr;
    return guarded([&]() -> PyObject* {
        auto as_it_is = [&]() {
            Py_INCREF(a[0]);
            return a[0];
        };
        if (!nothing_between() || !plain(a[0]) || !plain(a[1]) || !at::GradMode::is_enabled()) return as_it_is();
        const at::Tensor &x = THPVariable_Unpack(a[0]), &y = THPVariable_Unpack(a[1]);
        if (!x.requires_grad() || !y.grad_fn()) return as_it_is();
        const auto node = std::dynamic_pointer_cast<TakesResidual>(y.grad_fn());
        if (!node || node->num_inputs() != 1 || node->next_edge(0) != torch::autograd::impl::gradient_edge(x)) return as_it_is();
        at::Tensor r;
        {
            at::NoGradGuard no_grad;
            r = x.detach();
        }
        torch::autograd::set_history(r, node);
        return wrap(r);
    });
}

// x w^T + b, without gradients.  A view of the product (of matrices, which is nobody else's) becomes a tensor of its own: one made here may not be
// changed in place.
at::Tensor linear_of(const at::Tensor& x, const at::Tensor& w, const at::Tensor& b) {
    const at::Tensor y = at::linear(x, w, b.defined() ? std::optional<at::Tensor>(b) : std::nullopt);
    return y.is_view() ? at::_unsafe_view(y, y.sizes()) : y;
}

// projection(X, W, b | None) -> X W^T + b with the node above, or None where torch's own operator is to be called:
// nothing to differentiate, types or sizes the kernel does not take, or more than plain tensors in play.  Weights of
// more than 2^20 elements are torch's: with that many output tiles its product fills the machine.  Weight gradient,
// kernel / torch's product, us on the GPU: 1024 x 1024 at 4096, 8192, 16384 and 32768 tokens 32 / 29, 42 / 54, 67 / 103,
// 118 / 200; 1536 x 768 40 / 33, 61 / 61, 105 / 118, 193 / 200; 2304 x 768 67 / 35, 113 / 64, 206 / 127, 391 / 297.
// Up to 2048 tokens the product is the faster one on the GPU (1536 x 512 at 2048: 25 / 18; 256 x 256 at 256: 13 / 10), but
// the host takes longer to launch it and sets the pace there: forward and backward of the sub-layer with the product
// instead of the kernel for both weights took 300 us a call in place of 275.
PyObject* py_projection(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arg_count(n, 3, "projection")) return nullptr;
    return guarded([&]() -> PyObject* {
        if (!nothing_between() || !plain(a[0]) || !plain(a[1]) || (a[2] != Py_None && !plain(a[2]))) Py_RETURN_NONE;
        const at::Tensor &x = THPVariable_Unpack(a[0]), &w = THPVariable_Unpack(a[1]), b = optional_arg(a[2]);
        if (x.scalar_type() != at::kBFloat16 || w.scalar_type() != at::kBFloat16 || x.device() != w.device() ||
            x.dim() < 2 || w.dim() != 2 || !w.is_contiguous() || x.size(-1) != w.size(1) || x.numel() == 0 ||
            w.size(0) % 8 != 0 || w.size(1) % 8 != 0 || w.numel() == 0 || w.numel() > (1 << 20) ||
            x.numel() / x.size(-1) > 0x7fffffff - 4096)   // the kernel's row numbers run a little past the last
            Py_RETURN_NONE;
        if (!torch::autograd::compute_requires_grad(w)) Py_RETURN_NONE;
        at::Tensor y;
        {
            at::NoGradGuard no_grad;
            y = linear_of(x, w, b);
        }
        auto node = std::shared_ptr<ProjectionBackward>(new ProjectionBackward(), torch::autograd::deleteNode);
        node->has_bias = b.defined();
        node->set_next_edges(b.defined() ? torch::autograd::collect_next_edges(x, w, b) : torch::autograd::collect_next_edges(x, w));
        node->x = torch::autograd::SavedVariable(x, false);
        node->w = torch::autograd::SavedVariable(w, false);
        torch::autograd::set_history(y, node);
        return wrap(y);
    });
}

// ------------------------------------------------------------------------------------------------
// Attention with extras, the dense bias, dropout: nodes that save what their backward entry points take.
// ------------------------------------------------------------------------------------------------
[[noreturn]] void not_implemented(const char* what) {
    PyErr_SetString(PyExc_NotImplementedError, what);
    throw python_error();
}

// Whether a transform or a lazy view has made the tensor: its values are not those in memory.
bool transformed(const at::Tensor& t) {
    using c10::DispatchKey;
    for (DispatchKey k : {DispatchKey::Functionalize, DispatchKey::FuncTorchBatched, DispatchKey::Batched, DispatchKey::FuncTorchGradWrapper,
                          DispatchKey::Negative, DispatchKey::ZeroTensor})
        if (t.key_set().has(k)) return true;
    return false;
}
constexpr const char* kPlainTensors = "libspion's operators take plain tensors, none that a transform or a lazy view has made";
// A tensor that the kernels may read and an autograd node of this file may differentiate; `device`: the call's, once known.
void check_operand(const at::Tensor& t, const std::optional<at::Device>& device) {
    if (transformed(t)) not_implemented(kPlainTensors);
    if (t._fw_grad(0).defined()) not_implemented("libspion's operators have no forward-mode derivative");
    if (!t.is_cuda() || t.layout() != at::kStrided) bad_value("libspion needs device tensors");
    if (device && t.device() != *device) bad_value("the tensors of a call must be on one device");
}
void not_traced() {
    if (torch::jit::tracer::isTracing()) not_implemented("libspion's operators of this kind cannot be traced");
}
int dtype_code(const at::Tensor& t) {
    if (t.scalar_type() == at::kFloat) return SPION_F32;
    if (t.scalar_type() == at::kBFloat16) return SPION_BF16;
    bad_value("unsupported dtype");
}
// Contiguous, and aligned to the 16 bytes that the attention kernels load at once.
at::Tensor dense(const at::Tensor& t) {
    const at::Tensor c = t.contiguous();
    return (uintptr_t)c.data_ptr() % 16 == 0 ? c : c.clone();
}
int64_t long_arg(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw python_error();
    return v;
}
// {seed, offset} on the call's device
at::Tensor rng_arg(PyObject* o, const at::Device& device) {
    if (o == Py_None) bad_value("dropout needs rng, an int64 tensor {seed, offset}");
    const at::Tensor& t = tensor_arg(o);
    check_operand(t, device);
    if (t.scalar_type() != at::kLong || t.numel() != 2 || !t.is_contiguous()) bad_value("rng must be a contiguous int64 tensor {seed, offset}");
    return t;
}
unsigned stream_arg(PyObject* o) {
    const int64_t v = long_arg(o);
    if (v < 0 || v > 0xffffffffll) bad_value("stream must be a number of 32 bits");
    return (unsigned)v;
}
double dropout_arg(PyObject* o) {
    const double p = double_arg(o);
    if (!(p >= 0.0 && p < 1.0) || std::nearbyint(65536.0 * p) > 65535.0) bad_value("dropout must be a probability below 1 (steps of 2^-16)");
    return p;
}
at::Tensor new_longs(int64_t n, const at::Tensor& like) {
    return at::Tensor(at::detail::empty_cuda({n}, at::kLong, like.device(), std::nullopt));
}
// What a node of this kind does about exceptions, second derivatives and a gradient that is more or less than its numbers: one with a tangent or
// from a transform is refused, one that stands for its negative (autograd makes such from conjugates) is written out.
template <class F>
torch::autograd::variable_list differentiate(const char* twice, at::Tensor& grad, F&& f) {
    TORCH_CHECK_NOT_IMPLEMENTED(!at::GradMode::is_enabled(), twice);
    TORCH_CHECK_NOT_IMPLEMENTED(!grad._fw_grad(0).defined(), "libspion's operators have no forward-mode derivative, nor have their gradients");
    if (grad.is_neg()) grad = grad.resolve_neg();
    TORCH_CHECK_NOT_IMPLEMENTED(!transformed(grad), kPlainTensors);
    try {
        return f();
    } catch (const SpionFailure& e) {
        PyGILState_STATE gil = PyGILState_Ensure();
        spion_error(e.code, e.what);
        python_error err;
        err.persist();
        PyGILState_Release(gil);
        throw err;
    } catch (const BadValue& e) {
        TORCH_CHECK_VALUE(false, e.msg);
    }
}

// A bucket map as a backward pass keeps it: it must have been left as the forward pass read it.  By its version counter, without a saved variable, since a
// program keeps the map for good (no hook has anything to move away) and may have made it in inference mode, where nothing is counted.
struct BucketMap {
    at::Tensor map;
    int64_t version = 0;
    BucketMap() = default;
    explicit BucketMap(const at::Tensor& t) : map(t), version(t.defined() && !t.is_inference() ? t._version() : 0) {}
    const at::Tensor& unchanged() const {
        TORCH_CHECK(!map.defined() || map.is_inference() || map._version() == version,
                    "a bucket map needed for gradient computation has been modified by an inplace operation");
        return map;
    }
};

struct AttentionExtras {
    at::Tensor bucket_of, lengths;
    int n_buckets = 0;
    double dropout = 0.0;
    unsigned stream = 0;
    spion_attn_extras params(const at::Tensor& table) const {
        spion_attn_extras x = {};
        x.table = table.defined() ? table.data_ptr() : nullptr;
        x.bucket_of = table.defined() ? (const uint8_t*)bucket_of.data_ptr() : nullptr;
        x.lengths = lengths.defined() ? (const int32_t*)lengths.data_ptr() : nullptr;
        x.dropout = dropout;
        x.n_buckets = n_buckets;
        x.table_dtype = table.defined() ? dtype_code(table) : SPION_F32;
        x.stream = stream;
        return x;
    }
};

// Of a call; nothing where it needs none.
struct WithWorkspace {
    at::Tensor memory;
    void* ptr = nullptr;
    size_t bytes = 0;
    WithWorkspace(const spion_attn_params& p, const spion_attn_extras& x, const Index& ix, bool is_bwd, const at::Tensor& like) {
        const size_t n = spion_attn_with_workspace_bytes(&p, &x, ix.nnzb, is_bwd);
        if (n == 0 || n == (size_t)-1) return;   // what is unsupported the call itself tells
        memory = new_bytes(n, like);
        ptr = memory.data_ptr();
        bytes = n;
    }
};

// What the forward leaves for its backward besides O, in one tensor of bytes (each costs the host more than a microsecond): LSE, and where there are such,
// the generator's state and what rounding left of O.
struct WithState {
    size_t used = 0, rest = 0, bytes;   // where they are; 0: not there
    WithState(const spion_attn_params& p, bool draws, bool saved) {
        auto up = [](size_t n) { return (n + 255) / 256 * 256; };
        const size_t rows = (size_t)p.B * p.H * p.L;
        bytes = up(rows * 4);
        if (!saved) return;
        if (draws) {
            used = bytes;
            bytes += 256;
        }
        if (p.dtype == SPION_BF16) {
            rest = bytes;
            bytes += up(rows * 64 * 2);
        }
    }
    static void* at(const at::Tensor& state, size_t offset) { return offset ? static_cast<char*>(state.data_ptr()) + offset : nullptr; }
};
bool draws(const AttentionExtras& extras) { return std::nearbyint(65536.0 * extras.dropout) > 0.0; }

// The gradient of sparse_attention_with, and of heads_attention_with (q = qkv, no k and v).
struct AttentionWithBackward : public torch::autograd::Node {
    torch::autograd::SavedVariable q, k, v, o, state, table, lengths;
    Index ix;
    AttentionExtras extras;   // without the tensors
    BucketMap buckets;
    int64_t H = 0;   // of qkv's heads; 0: Q, K and V

    std::string name() const override { return "SparseAttentionWithBackward"; }

    void release_variables() override {
        for (torch::autograd::SavedVariable* s : {&q, &k, &v, &o, &state, &table, &lengths}) s->reset_data();
        buckets.map.reset();
    }

    torch::autograd::variable_list apply(torch::autograd::variable_list&& grads) override {
        const int inputs = H ? 1 : 3;
        torch::autograd::variable_list out(inputs + (extras.n_buckets ? 1 : 0));
        if (!grads[0].defined()) return out;
        return differentiate("sparse_attention cannot be differentiated twice", grads[0], [&] {
            const at::Tensor Q = q.unpack(), O = o.unpack(shared_from_this()), left = state.unpack(), T = table.unpack();
            const at::Tensor K = H ? Q : k.unpack(), V = H ? Q : v.unpack();
            AttentionExtras with = extras;
            with.lengths = lengths.unpack();
            with.bucket_of = buckets.unchanged();
            const at::Device device = grads[0].device();   // the call's: autograd hands on no gradient of another device or shape
            const c10::DeviceGuard guard(device);
            const at::Tensor g = dense(grads[0]);
            // What saved-tensor hooks hand back is looked at as the call's own tensors were: the kernels take sizes from Q and bare addresses of the rest.
            auto same = [](bool ok) {
                if (!ok) bad_value("sparse_attention: a saved tensor is not the one that was saved");
            };
            const at::Tensor& n = with.lengths;
            for (const at::Tensor* t : {&Q, &K, &V, &O, &left, &T, &n})
                same(!t->defined() || (t->device() == device && t->layout() == at::kStrided && t->is_contiguous() && !transformed(*t)));
            if (H) same(Q.dim() == 3 && Q.size(0) == g.size(0) && Q.size(1) == g.size(1) && Q.size(2) == 3 * g.size(2) && Q.scalar_type() == at::kBFloat16);
            else same(Q.sizes() == g.sizes() && K.sizes() == g.sizes() && V.sizes() == g.sizes());
            for (const at::Tensor* t : {&Q, &K, &V, &O}) same(t->scalar_type() == g.scalar_type());
            same(O.sizes() == g.sizes());
            const spion_attn_params p = H ? heads_params(Q, H, ix) : params_of(Q, ix);
            const WithState at(p, draws(extras), true);
            same(left.numel() == (int64_t)at.bytes && left.scalar_type() == at::kByte && (uintptr_t)left.data_ptr() % 16 == 0);
            same(!extras.n_buckets || (T.dim() == 2 && T.size(0) == extras.n_buckets && T.size(1) == p.H));
            same(!n.defined() || (n.numel() == p.B && n.scalar_type() == at::kInt));
            spion_attn_extras x = with.params(T);
            x.rng = (const int64_t*)WithState::at(left, at.used);
            x.o_rest = WithState::at(left, at.rest);
            const float* const stat = (const float*)device_ptr(left);
            const bool table_grad = extras.n_buckets && task_should_compute_output(inputs);
            for (int i = 0; i < inputs; ++i) out[i] = new_like(Q);
            if (table_grad) out[inputs] = new_like(T);
            void* const dtable = table_grad ? device_ptr(out[inputs]) : nullptr;
            const WithWorkspace ws(p, x, ix, true, Q);
            auto index = [](const at::Tensor& t) { return (const int32_t*)device_ptr(t); };
            if (H) {
                const int rc = spion_heads_attn_bwd_with(device_ptr(Q), device_ptr(O), device_ptr(g), stat, device_ptr(out[0]),
                                                         dtable, index(ix.row_ptr), index(ix.col_idx), index(ix.col_ptr), index(ix.row_idx), ix.nnzb,
                                                         &p, &x, ws.ptr, ws.bytes, current_stream());
                if (rc != SPION_OK) throw SpionFailure{rc, "spion_heads_attn_bwd_with"};
                return out;
            }
            const int rc = spion_attn_bwd_with(device_ptr(Q), device_ptr(K), device_ptr(V), device_ptr(O), device_ptr(g), stat,
                                               device_ptr(out[0]), device_ptr(out[1]), device_ptr(out[2]), dtable, index(ix.row_ptr), index(ix.col_idx),
                                               index(ix.col_ptr), index(ix.row_idx), index(ix.bsr_pos), ix.nnzb, &p, &x, ws.ptr, ws.bytes, current_stream());
            if (rc != SPION_OK) throw SpionFailure{rc, "spion_attn_bwd_with"};
            return out;
        });
    }
};

// The arguments table | None, bucket_of | None, lengths | None, dropout, rng | None, stream of a call on B sequences of L tokens.
struct ExtrasArgs {
    AttentionExtras extras;
    at::Tensor table, rng;   // rng: only where there is something to draw

    ExtrasArgs(PyObject* const* a, int64_t B, int64_t H, int64_t L, const at::Device& device) {
        table = optional_arg(a[0]);
        extras.lengths = optional_arg(a[2]);
        extras.dropout = dropout_arg(a[3]);
        extras.stream = stream_arg(a[5]);
        if (table.defined()) {
            check_operand(table, device);
            extras.bucket_of = tensor_arg(a[1]);
            check_operand(extras.bucket_of, device);
            dtype_code(table);
            if (table.dim() != 2 || table.size(1) != H) bad_value("the bias table must be [buckets, H]");
            if (table.size(0) < 1 || table.size(0) > 256) bad_value("the bias table must have 1 to 256 buckets");
            if (extras.bucket_of.scalar_type() != at::kByte || !extras.bucket_of.is_contiguous() || extras.bucket_of.numel() != 2 * L - 1)
                bad_value("the buckets must be a contiguous uint8 map of 2 L - 1 distances");
            extras.n_buckets = (int)table.size(0);
        }
        if (extras.lengths.defined()) {
            check_operand(extras.lengths, device);
            if (extras.lengths.scalar_type() != at::kInt || extras.lengths.numel() != B || !extras.lengths.is_contiguous())
                bad_value("lengths must be a contiguous int32 tensor [B]");
        }
        if (draws(extras)) rng = rng_arg(a[4], device);
    }
};

// The node of a call, but for q, k, v and o.
std::shared_ptr<AttentionWithBackward> with_node(AttentionExtras&& extras, Index&& ix, const at::Tensor& state, const at::Tensor& table) {
    auto node = std::shared_ptr<AttentionWithBackward>(new AttentionWithBackward(), torch::autograd::deleteNode);
    node->state = torch::autograd::SavedVariable(state, false);
    node->table = torch::autograd::SavedVariable(table, false);
    node->lengths = torch::autograd::SavedVariable(extras.lengths, false);
    node->buckets = BucketMap(extras.bucket_of);
    extras.lengths.reset();
    extras.bucket_of.reset();
    node->extras = std::move(extras);
    node->ix = std::move(ix);
    return node;
}

// What the kernels read of an index, one of whose directions is (ptr, idx), for sequences of L tokens: a pattern of another length would lead them past it.
void check_index(const at::Tensor& ptr, const at::Tensor& idx, const Index& ix, int64_t L, const at::Device& device) {
    check_operand(ptr, device);
    check_operand(idx, device);
    if (ix.block < 1 || L % ix.block != 0 || ptr.numel() != L / ix.block + 1 || ix.nnzb < 0 || idx.numel() < ix.nnzb || ptr.scalar_type() != at::kInt ||
        idx.scalar_type() != at::kInt || !ptr.is_contiguous() || !idx.is_contiguous())
        bad_value("the pattern is not one of sequences of this length, or its blocks are not counted");
}

// sparse_attention_with(Q, K, V, row_ptr, col_idx, col_ptr, row_idx, bsr_pos, nnzb, block, scale, table | None, bucket_of | None,
//                       lengths | None, dropout, rng | None, stream) -> O
PyObject* py_sparse_attention_with(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arg_count(n, 17, "sparse_attention_with")) return nullptr;
    return guarded([&]() -> PyObject* {
        not_traced();
        const at::Tensor &q = tensor_arg(a[0]), &k = tensor_arg(a[1]), &v = tensor_arg(a[2]);
        check_operand(q, std::nullopt);
        const at::Device device = q.device();
        check_operand(k, device);
        check_operand(v, device);
        if (q.dim() != 4 || k.sizes() != q.sizes() || v.sizes() != q.sizes() || k.scalar_type() != q.scalar_type() ||
            v.scalar_type() != q.scalar_type())
            bad_value("Q, K and V must have one shape [B, H, L, 64] and one dtype");
        Index ix;
        ix.row_ptr = tensor_arg(a[3]);
        ix.col_idx = tensor_arg(a[4]);
        ix.nnzb = int_arg(a[8]);
        ix.block = int_arg(a[9]);
        ix.scale = (float)double_arg(a[10]);
        check_index(ix.row_ptr, ix.col_idx, ix, q.size(2), device);
        ExtrasArgs with(a + 11, q.size(0), q.size(1), q.size(2), device);
        const at::Tensor& table = with.table;
        const c10::DeviceGuard guard(device);
        const bool grad = table.defined() ? torch::autograd::compute_requires_grad(q, k, v, table) : torch::autograd::compute_requires_grad(q, k, v);
        at::Tensor o, state, qc, kc, vc, tc;
        {
            at::NoGradGuard no_grad;
            qc = dense(q);
            kc = dense(k);
            vc = dense(v);
            if (table.defined()) tc = table.contiguous();
            const spion_attn_params p = params_of(qc, ix);
            o = new_like(qc);
            const WithState at(p, with.rng.defined(), grad);
            state = new_bytes(at.bytes, qc);
            spion_attn_extras x = with.extras.params(tc);
            if (with.rng.defined()) x.rng = (const int64_t*)with.rng.data_ptr();
            x.rng_used = (int64_t*)WithState::at(state, at.used);
            x.o_rest = WithState::at(state, at.rest);
            const WithWorkspace ws(p, x, ix, false, qc);
            const int rc = spion_attn_fwd_with(device_ptr(qc), device_ptr(kc), device_ptr(vc), device_ptr(o), (float*)device_ptr(state),
                                               (const int32_t*)device_ptr(ix.row_ptr), (const int32_t*)device_ptr(ix.col_idx), ix.nnzb, &p, &x,
                                               ws.ptr, ws.bytes, current_stream());
            if (rc != SPION_OK) throw SpionFailure{rc, "spion_attn_fwd_with"};
        }
        if (grad) {
            ix.col_ptr = tensor_arg(a[5]);
            ix.row_idx = tensor_arg(a[6]);
            ix.bsr_pos = tensor_arg(a[7]);
            check_operand(ix.bsr_pos, device);
            check_index(ix.col_ptr, ix.row_idx, ix, q.size(2), device);
            auto node = with_node(std::move(with.extras), std::move(ix), state, tc);
            node->set_next_edges(table.defined() ? torch::autograd::collect_next_edges(q, k, v, table) : torch::autograd::collect_next_edges(q, k, v));
            node->q = torch::autograd::SavedVariable(qc, false);
            node->k = torch::autograd::SavedVariable(kc, false);
            node->v = torch::autograd::SavedVariable(vc, false);
            torch::autograd::set_history(o, node);
            node->o = torch::autograd::SavedVariable(o, true);
        }
        return wrap(o);
    });
}

// heads_attention_with(qkv [B, L, 3 H 64], H, row_ptr, col_idx, col_ptr, row_idx, bsr_pos, nnzb, block, apart, table | None,
//                      bucket_of | None, lengths | None, dropout, rng | None, stream) -> [B, L, H 64]
// None where the steps are to be taken one by one (see heads_attention).
PyObject* py_heads_attention_with(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arg_count(n, 16, "heads_attention_with")) return nullptr;
    return guarded([&]() -> PyObject* {
        if (!nothing_between() || !plain(a[0]) || a[9] == Py_True) Py_RETURN_NONE;
        const at::Tensor& qkv = THPVariable_Unpack(a[0]);
        const int64_t H = int_arg(a[1]);
        Index ix;
        ix.nnzb = int_arg(a[7]);
        ix.block = int_arg(a[8]);
        if (!heads_in_place(qkv, ix) || qkv.dim() != 3 || !qkv.is_contiguous() || H <= 0 || qkv.size(2) != 3 * H * 64 || qkv.numel() == 0 ||
            (uintptr_t)qkv.data_ptr() % 16 != 0)
            Py_RETURN_NONE;
        const at::Device device = qkv.device();
        const int64_t B = qkv.size(0), L = qkv.size(1);
        ix.row_ptr = tensor_arg(a[2]);
        ix.col_idx = tensor_arg(a[3]);
        check_index(ix.row_ptr, ix.col_idx, ix, L, device);
        ExtrasArgs with(a + 10, B, H, L, device);
        const at::Tensor& table = with.table;
        const c10::DeviceGuard guard(device);
        const bool grad = table.defined() ? torch::autograd::compute_requires_grad(qkv, table) : torch::autograd::compute_requires_grad(qkv);
        at::Tensor tc, state;
        at::Tensor s(at::detail::empty_cuda({B, L, H * 64}, qkv.scalar_type(), device, std::nullopt));
        {
            at::NoGradGuard no_grad;
            if (table.defined()) tc = table.contiguous();
            const spion_attn_params p = heads_params(qkv, H, ix);
            const WithState at(p, with.rng.defined(), grad);
            state = new_bytes(at.bytes, qkv);
            spion_attn_extras x = with.extras.params(tc);
            if (with.rng.defined()) x.rng = (const int64_t*)with.rng.data_ptr();
            x.rng_used = (int64_t*)WithState::at(state, at.used);
            x.o_rest = WithState::at(state, at.rest);
            const WithWorkspace ws(p, x, ix, false, qkv);
            const int rc = spion_heads_attn_fwd_with(device_ptr(qkv), device_ptr(s), (float*)device_ptr(state), (const int32_t*)device_ptr(ix.row_ptr),
                                                     (const int32_t*)device_ptr(ix.col_idx), ix.nnzb, &p, &x, ws.ptr, ws.bytes,
                                                     current_stream());
            if (rc != SPION_OK) throw SpionFailure{rc, "spion_heads_attn_fwd_with"};
        }
        if (grad) {
            ix.col_ptr = tensor_arg(a[4]);
            ix.row_idx = tensor_arg(a[5]);
            ix.bsr_pos = tensor_arg(a[6]);
            check_index(ix.col_ptr, ix.row_idx, ix, L, device);
            auto node = with_node(std::move(with.extras), std::move(ix), state, tc);
            node->H = H;
            node->set_next_edges(table.defined() ? torch::autograd::collect_next_edges(qkv, table) : torch::autograd::collect_next_edges(qkv));
            node->q = torch::autograd::SavedVariable(qkv, false);
            torch::autograd::set_history(s, node);
            node->o = torch::autograd::SavedVariable(s, true);
        }
        return wrap(s);
    });
}

struct RelativeBiasBackward : public torch::autograd::Node {
    BucketMap buckets;   // kept after a pass: without saved tensors a second one needs no retain_graph
    at::ScalarType type = at::kFloat;
    int reach = 0, n_buckets = 0, H = 0, q_len = 0, k_len = 0, q_start = 0;

    std::string name() const override { return "RelativeBiasBackward"; }

    torch::autograd::variable_list apply(torch::autograd::variable_list&& grads) override {
        torch::autograd::variable_list out(1);
        if (!grads[0].defined()) return out;
        return differentiate("relative_bias cannot be differentiated twice", grads[0], [&] {
            const at::Tensor& bucket_of = buckets.unchanged();
            const c10::DeviceGuard guard(bucket_of.device());
            const at::Tensor g = grads[0].contiguous();
            if (g.scalar_type() != type || g.numel() != (int64_t)H * q_len * k_len) bad_value("relative_bias: a gradient of another shape");
            out[0] = at::Tensor(at::detail::empty_cuda({n_buckets, H}, type, g.device(), std::nullopt));
            const at::Tensor ws = new_bytes(spion_relative_bias_workspace_bytes(n_buckets, H, q_len, k_len), g);
            const int rc = spion_relative_bias_grad(device_ptr(g), (const uint8_t*)device_ptr(bucket_of), device_ptr(out[0]), reach, n_buckets, H, q_len,
                                                    k_len, q_start, dtype_code(g), device_ptr(ws), (size_t)ws.nbytes(), current_stream());
            if (rc != SPION_OK) throw SpionFailure{rc, "spion_relative_bias_grad"};
            return out;
        });
    }
};

// relative_bias(table, bucket_of, q_len, k_len, q_start) -> [H, q_len, k_len]
PyObject* py_relative_bias(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arg_count(n, 5, "relative_bias")) return nullptr;
    return guarded([&]() -> PyObject* {
        not_traced();
        const at::Tensor &table = tensor_arg(a[0]), &bucket_of = tensor_arg(a[1]);
        check_operand(table, std::nullopt);
        check_operand(bucket_of, table.device());
        const int64_t q_len = long_arg(a[2]), k_len = long_arg(a[3]), q_start = long_arg(a[4]);
        if (table.dim() != 2 || table.size(0) < 1 || table.size(0) > 256 || table.size(1) < 1) bad_value("the bias table must be [buckets, H], 1 to 256 buckets");
        if (bucket_of.scalar_type() != at::kByte || !bucket_of.is_contiguous() || bucket_of.numel() % 2 != 1)
            bad_value("the buckets must be a contiguous uint8 map of 2 L - 1 distances");
        const int64_t reach = (bucket_of.numel() + 1) / 2;
        if (q_len < 1 || k_len < 1 || q_start < 0 || q_len > reach || q_start > reach - q_len || k_len > reach)
            bad_value("the buckets do not reach over the positions asked for");
        const c10::DeviceGuard guard(table.device());
        const at::Tensor tc = table.contiguous();
        const int code = dtype_code(tc);
        at::Tensor bias(at::detail::empty_cuda({table.size(1), q_len, k_len}, tc.scalar_type(), tc.device(), std::nullopt));
        const int rc = spion_relative_bias(device_ptr(tc), (const uint8_t*)device_ptr(bucket_of), device_ptr(bias), (int)reach, (int)table.size(0),
                                           (int)table.size(1), (int)q_len, (int)k_len, (int)q_start, code, current_stream());
        if (rc != SPION_OK) throw SpionFailure{rc, "spion_relative_bias"};
        if (torch::autograd::compute_requires_grad(table)) {
            auto node = std::shared_ptr<RelativeBiasBackward>(new RelativeBiasBackward(), torch::autograd::deleteNode);
            node->set_next_edges(torch::autograd::collect_next_edges(table));
            node->buckets = BucketMap(bucket_of);
            node->type = tc.scalar_type();
            node->reach = (int)reach;
            node->n_buckets = (int)table.size(0);
            node->H = (int)table.size(1);
            node->q_len = (int)q_len;
            node->k_len = (int)k_len;
            node->q_start = (int)q_start;
            torch::autograd::set_history(bias, node);
        }
        return wrap(bias);
    });
}

void dropout_call(const at::Tensor& x, const at::Tensor& residual, const at::Tensor& y, double p, const at::Tensor& rng, const at::Tensor& used, unsigned stream) {
    if (x.numel() == 0) return;
    const int rc = spion_dropout_add(device_ptr(x), residual.defined() ? device_ptr(residual) : nullptr, device_ptr(y), x.numel(), dtype_code(x), p,
                                     (const int64_t*)device_ptr(rng), used.defined() ? (int64_t*)device_ptr(used) : nullptr, stream, current_stream());
    if (rc != SPION_OK) throw SpionFailure{rc, "spion_dropout_add"};
}

struct DropoutAddBackward : public torch::autograd::Node {
    torch::autograd::SavedVariable rng;
    double p = 0.0;
    unsigned stream = 0;
    bool has_residual = false;

    std::string name() const override { return "DropoutAddBackward"; }

    void release_variables() override { rng.reset_data(); }

    torch::autograd::variable_list apply(torch::autograd::variable_list&& grads) override {
        torch::autograd::variable_list out(has_residual ? 2 : 1);
        if (!grads[0].defined()) return out;
        return differentiate("dropout_add cannot be differentiated twice", grads[0], [&] {
            const c10::DeviceGuard guard(grads[0].device());
            if (has_residual && task_should_compute_output(1)) out[1] = grads[0];
            if (task_should_compute_output(0)) {
                const at::Tensor g = grads[0].contiguous(), used = rng.unpack();
                // looked at again: a saved-tensor hook may have handed back another one
                if (used.device() != g.device() || used.layout() != at::kStrided || used.scalar_type() != at::kLong || used.numel() != 2 || !used.is_contiguous() ||
                    transformed(used))
                    bad_value("dropout_add: a saved tensor is not the one that was saved");
                out[0] = new_like(g);
                dropout_call(g, at::Tensor(), out[0], p, used, at::Tensor(), stream);
            }
            return out;
        });
    }
};

// dropout_add(x, residual | None, p, rng, stream) -> residual + dropout(x)
PyObject* py_dropout_add(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arg_count(n, 5, "dropout_add")) return nullptr;
    return guarded([&]() -> PyObject* {
        not_traced();
        const at::Tensor& x = tensor_arg(a[0]);
        const at::Tensor residual = optional_arg(a[1]);
        check_operand(x, std::nullopt);
        dtype_code(x);
        if (residual.defined()) {
            check_operand(residual, x.device());
            if (residual.sizes() != x.sizes() || residual.scalar_type() != x.scalar_type()) bad_value("residual must have x's shape and dtype");
        }
        const double p = dropout_arg(a[2]);
        const at::Tensor rng = rng_arg(a[3], x.device());
        const unsigned stream = stream_arg(a[4]);
        const c10::DeviceGuard guard(x.device());
        const bool grad = residual.defined() ? torch::autograd::compute_requires_grad(x, residual) : torch::autograd::compute_requires_grad(x);
        at::Tensor y, used;
        {
            at::NoGradGuard no_grad;
            const at::Tensor xc = x.contiguous();
            y = new_like(xc);
            if (grad) used = new_longs(2, xc);
            dropout_call(xc, residual.defined() ? residual.contiguous() : at::Tensor(), y, p, rng, used, stream);
        }
        if (grad) {
            auto node = std::shared_ptr<DropoutAddBackward>(new DropoutAddBackward(), torch::autograd::deleteNode);
            node->set_next_edges(residual.defined() ? torch::autograd::collect_next_edges(x, residual) : torch::autograd::collect_next_edges(x));
            node->rng = torch::autograd::SavedVariable(used, false);
            node->p = p;
            node->stream = stream;
            node->has_residual = residual.defined();
            torch::autograd::set_history(y, node);
        }
        return wrap(y);
    });
}

// ------------------------------------------------------------------------------------------------
// Rotary positions, root-mean-square norm, rows in 8 bits.
// ------------------------------------------------------------------------------------------------
// A second gradient is looked at as the first (see differentiate).
void check_gradient(at::Tensor& grad) {
    if (!grad.defined()) return;
    TORCH_CHECK_NOT_IMPLEMENTED(!grad._fw_grad(0).defined(), "libspion's operators have no forward-mode derivative, nor have their gradients");
    if (grad.is_neg()) grad = grad.resolve_neg();
    TORCH_CHECK_NOT_IMPLEMENTED(!transformed(grad), kPlainTensors);
}
at::Tensor new_tensor(at::IntArrayRef sizes, at::ScalarType type, const at::Device& device) {
    return at::Tensor(at::detail::empty_cuda(sizes, type, device, std::nullopt));
}
// A saved tensor as the kernels may read it: where and what it was.
bool as_saved(const at::Tensor& t, const at::Device& device, at::ScalarType type) {
    return t.defined() && t.device() == device && t.layout() == at::kStrided && t.is_contiguous() && !transformed(t) && t.scalar_type() == type;
}
void saved(bool ok, const char* message) {
    if (!ok) bad_value(message);
}

struct RotaryArgs {
    at::Tensor turns, axis_of;
    int64_t axes = 0, rotated = 0;
    bool neighbours = false;
};

// Heads of x: [B, H, L, d], or [B, L, H d] with heads beside each other.
struct Heads {
    int64_t B, H, L, d, stride[3];   // strides of B, H, L
    Heads(const at::Tensor& x, int64_t d_) : d(d_) {
        const bool apart = x.dim() == 4;
        B = x.size(0);
        H = apart ? x.size(1) : x.size(2) / d;
        L = x.size(apart ? 2 : 1);
        stride[0] = x.stride(0);
        stride[1] = apart ? x.stride(1) : d;
        stride[2] = x.stride(apart ? 2 : 1);
    }
};

// y as x lies, if that is without gaps.
at::Tensor turn(const at::Tensor& x, const RotaryArgs& a, const at::Tensor& positions, bool back) {
    const at::Tensor y = x.is_non_overlapping_and_dense()
                             ? at::Tensor(at::detail::empty_strided_cuda(x.sizes(), x.strides(), x.scalar_type(), x.device()))
                             : new_like(x);
    if (x.numel() == 0) return y;
    const int64_t d = 2 * a.turns.size(0);
    const Heads from(x, d), to(y, d);
    spion_rotary_params p = {};
    p.B = (int32_t)from.B;
    p.H = (int32_t)from.H;
    p.L = (int32_t)from.L;
    p.d = (int32_t)d;
    p.rotated = (int32_t)a.rotated;
    p.axes = (int32_t)a.axes;
    p.dtype = dtype_code(x);
    p.position_bytes = positions.scalar_type() == at::kLong ? 8 : 4;
    for (int i = 0; i < 3; ++i) {
        p.x_stride[i] = from.stride[i];
        p.y_stride[i] = to.stride[i];
    }
    p.position_stride[0] = positions.stride(0);
    p.position_stride[1] = positions.dim() == 3 ? positions.stride(1) : 0;
    p.position_stride[2] = positions.stride(-1);
    p.flags = (a.neighbours ? SPION_ROTARY_NEIGHBOURS : 0u) | (back ? SPION_ROTARY_BACK : 0u);
    const int rc = spion_rotary(x.data_ptr(), y.data_ptr(), (const int64_t*)device_ptr(a.turns), (const uint8_t*)device_ptr(a.axis_of), positions.data_ptr(), &p,
                                current_stream());
    if (rc != SPION_OK) throw SpionFailure{rc, "spion_rotary"};
    return y;
}

struct RotaryBackward : public torch::autograd::Node {
    torch::autograd::SavedVariable positions;
    RotaryArgs args;
    BucketMap turns, axis_of;   // kept for good by the program, as a bucket map is
    std::vector<int64_t> position_sizes;
    at::ScalarType position_type = at::kLong;

    std::string name() const override { return "RotaryBackward"; }

    void release_variables() override { positions.reset_data(); }

    torch::autograd::variable_list apply(torch::autograd::variable_list&& grads) override {
        torch::autograd::variable_list out(1);
        if (!grads[0].defined()) return out;
        return differentiate("rotary cannot be differentiated twice", grads[0], [&] {
            const at::Device device = grads[0].device();
            const c10::DeviceGuard guard(device);
            const at::Tensor g = grads[0].stride(-1) == 1 ? grads[0] : grads[0].contiguous(), pos = positions.unpack();
            saved(pos.defined() && pos.device() == device && pos.layout() == at::kStrided && !transformed(pos) && pos.sizes() == at::IntArrayRef(position_sizes) &&
                      pos.scalar_type() == position_type, "rotary: a saved tensor is not the one that was saved");
            RotaryArgs a = args;
            a.turns = turns.unchanged();
            a.axis_of = axis_of.unchanged();
            out[0] = turn(g, a, pos, true);
            return out;
        });
    }
};

// rotary(x, turns, axis_of, positions, axes, rotated | None, neighbours) -> y
PyObject* py_rotary(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arg_count(n, 7, "rotary")) return nullptr;
    return guarded([&]() -> PyObject* {
        not_traced();
        const at::Tensor &x = tensor_arg(a[0]), &positions = tensor_arg(a[3]);
        check_operand(x, std::nullopt);
        const at::Device device = x.device();
        RotaryArgs args;
        args.turns = tensor_arg(a[1]);
        args.axis_of = tensor_arg(a[2]);
        args.axes = long_arg(a[4]);
        args.neighbours = truth_arg(a[6]);
        check_operand(positions, device);
        check_operand(args.turns, device);
        check_operand(args.axis_of, device);
        dtype_code(x);
        if (x.dim() != 4 && x.dim() != 3) bad_value("rotary takes tensors of shape [B, H, L, head_dim] or [B, L, H * head_dim]");
        if (args.turns.dim() != 1 || args.turns.size(0) < 1 || args.turns.scalar_type() != at::kLong || !args.turns.is_contiguous() ||
            args.axis_of.dim() != 1 || args.axis_of.size(0) != args.turns.size(0) || args.axis_of.scalar_type() != at::kByte || !args.axis_of.is_contiguous() ||
            (x.dim() == 4 ? x.size(3) != 2 * args.turns.size(0) : x.size(2) % (2 * args.turns.size(0)) != 0))
            bad_value("the axes are not those of heads of this dimension");
        const Heads heads(x, 2 * args.turns.size(0));
        args.rotated = a[5] == Py_None ? heads.H : long_arg(a[5]);
        if (args.rotated < 0 || args.rotated > heads.H) bad_value("heads must be a number of x's heads");
        if ((positions.scalar_type() != at::kLong && positions.scalar_type() != at::kInt) || positions.dim() < 2 || positions.dim() > 3 ||
            positions.size(0) != args.axes || positions.size(-1) != heads.L || (positions.dim() == 3 && positions.size(1) != heads.B))
            bad_value("positions must be int32 or int64 [axes, L] or [axes, B, L]");
        if (heads.B > 0x7fffffff || heads.H > 65535 || heads.L > 0x7fffffff) bad_value("rotary: too many heads or tokens");
        const c10::DeviceGuard guard(device);
        const bool grad = torch::autograd::compute_requires_grad(x);
        at::Tensor y;
        {
            at::NoGradGuard no_grad;
            y = turn(x.stride(-1) == 1 ? x : x.contiguous(), args, positions, false);
        }
        if (grad) {
            auto node = std::shared_ptr<RotaryBackward>(new RotaryBackward(), torch::autograd::deleteNode);
            node->set_next_edges(torch::autograd::collect_next_edges(x));
            node->positions = torch::autograd::SavedVariable(positions, false);
            node->position_sizes = positions.sizes().vec();
            node->position_type = positions.scalar_type();
            node->turns = BucketMap(args.turns);
            node->axis_of = BucketMap(args.axis_of);
            node->args = std::move(args);
            node->args.turns.reset();
            node->args.axis_of.reset();
            torch::autograd::set_history(y, node);
        }
        return wrap(y);
    });
}

// Codes and exponents of rows, as Packed8 has them.
struct Eight {
    at::Tensor codes, exponents;
    Eight() = default;
    // of rows like x's
    explicit Eight(const at::Tensor& x) {
        std::vector<int64_t> sizes = x.sizes().vec();
        sizes.back() = (sizes.back() + 63) / 64 * 64;
        codes = new_tensor(sizes, at::kChar, x.device());
        sizes.back() /= 64;
        exponents = new_tensor(sizes, at::kByte, x.device());
    }
    // those that a caller hands over, for x's rows
    Eight(const at::Tensor& c, const at::Tensor& e, at::IntArrayRef lead, int64_t D, const at::Device& device) : codes(c), exponents(e) {
        check_operand(codes, device);
        check_operand(exponents, device);
        std::vector<int64_t> sizes(lead.begin(), lead.end());
        sizes.push_back((D + 63) / 64 * 64);
        const bool fits = codes.sizes() == at::IntArrayRef(sizes) && codes.scalar_type() == at::kChar && codes.is_contiguous();
        sizes.back() /= 64;
        if (!fits || exponents.sizes() != at::IntArrayRef(sizes) || exponents.scalar_type() != at::kByte || !exponents.is_contiguous() ||
            (uintptr_t)codes.data_ptr() % 16 != 0)
            bad_value("codes must be contiguous int8 [..., P], exponents uint8 [..., P / 64], P the multiple of 64 from the rows' size on");
    }
    int8_t* c() const { return (int8_t*)codes.data_ptr(); }
    uint8_t* e() const { return (uint8_t*)exponents.data_ptr(); }
};

// Rows of a tensor [..., D].
int64_t rows_of(const at::Tensor& x) {
    if (x.dim() < 1 || x.size(-1) < 1) bad_value("expected rows of at least one element");
    return x.numel() / x.size(-1);
}

void pack(const at::Tensor& x, const Eight& to) {
    const int64_t rows = rows_of(x);
    if (rows == 0) return;
    const int rc = spion_pack_eight(device_ptr(x), to.c(), to.e(), rows, (int32_t)x.size(-1), dtype_code(x), current_stream());
    if (rc != SPION_OK) throw SpionFailure{rc, "spion_pack_eight"};
}

void check_width(int64_t D) {
    if (D > 1 << 20) bad_value("rows of more than 2^20 elements are not supported");
}

// pack8(x) -> (codes, exponents)
PyObject* py_pack8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arg_count(n, 1, "pack8")) return nullptr;
    return guarded([&]() -> PyObject* {
        not_traced();
        const at::Tensor& x = tensor_arg(a[0]);
        check_operand(x, std::nullopt);
        dtype_code(x);
        rows_of(x);
        check_width(x.size(-1));
        const c10::DeviceGuard guard(x.device());
        at::NoGradGuard no_grad;
        const Eight to(x);
        pack(x.contiguous(), to);
        PyObject* r = PyTuple_New(2);
        if (!r) return nullptr;
        PyTuple_SET_ITEM(r, 0, wrap(to.codes));
        PyTuple_SET_ITEM(r, 1, wrap(to.exponents));
        return r;
    });
}

// unpack8(codes, exponents, weight | None, D, dtype code) -> values
PyObject* py_unpack8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arg_count(n, 5, "unpack8")) return nullptr;
    return guarded([&]() -> PyObject* {
        not_traced();
        const at::Tensor& codes = tensor_arg(a[0]);
        check_operand(codes, std::nullopt);
        const at::Device device = codes.device();
        const int64_t D = long_arg(a[3]);
        if (D < 1 || codes.dim() < 1) bad_value("expected rows of at least one element");
        check_width(D);
        const Eight from(codes, tensor_arg(a[1]), codes.sizes().slice(0, codes.dim() - 1), D, device);
        at::Tensor weight = optional_arg(a[2]);
        if (weight.defined()) {
            check_operand(weight, device);
            dtype_code(weight);
            if (weight.dim() != 1 || weight.size(0) != D) bad_value("weight must be [size]");
        }
        const c10::DeviceGuard guard(device);
        at::NoGradGuard no_grad;
        if (weight.defined()) weight = weight.contiguous();
        std::vector<int64_t> sizes = codes.sizes().vec();
        sizes.back() = D;
        const int type = int_arg(a[4]);
        const at::Tensor y = new_tensor(sizes, type == SPION_F32 ? at::kFloat : at::kBFloat16, device);
        if (y.numel() > 0) {
            const int rc = spion_unpack_eight(from.c(), from.e(), weight.defined() ? device_ptr(weight) : nullptr, weight.defined() ? dtype_code(weight) : SPION_F32,
                                              device_ptr(y), rows_of(y), (int32_t)D, type, current_stream());
            if (rc != SPION_OK) throw SpionFailure{rc, "spion_unpack_eight"};
        }
        return wrap(y);
    });
}

// x, weight, residual | None of a norm; contiguous.
struct NormArgs {
    at::Tensor x, w, residual;
    int64_t rows, D;
    double eps;
    NormArgs(const at::Tensor& x_in, const at::Tensor& w_in, const at::Tensor& r_in, PyObject* e) {
        const at::Device device = x_in.device();
        check_operand(x_in, std::nullopt);
        check_operand(w_in, device);
        dtype_code(x_in);
        rows = rows_of(x_in);
        D = x_in.size(-1);
        if (D > 16384) bad_value("rows of more than 16384 elements are not supported");
        if (w_in.dim() != 1 || w_in.size(0) != D || w_in.scalar_type() != x_in.scalar_type()) bad_value("weight must be [D], of x's dtype");
        if (r_in.defined()) {
            check_operand(r_in, device);
            if (r_in.sizes() != x_in.sizes() || r_in.scalar_type() != x_in.scalar_type()) bad_value("residual must have x's shape and dtype");
        }
        eps = double_arg(e);
        if (!(eps >= 0.0) || std::isinf(eps)) bad_value("eps must be a number from 0 on");
        at::NoGradGuard no_grad;
        x = x_in.contiguous();
        w = w_in.contiguous();
        if (r_in.defined()) residual = r_in.contiguous();
    }
    void run(const at::Tensor& y, const at::Tensor& h, const at::Tensor& rstd, const Eight& eight, unsigned flags) const {
        if (rows == 0) return;
        auto ptr = [](const at::Tensor& t) { return t.defined() ? device_ptr(t) : nullptr; };
        const bool codes = eight.codes.defined();
        const int rc = spion_rms_norm(device_ptr(x), ptr(residual), device_ptr(w), ptr(y), ptr(h), (float*)ptr(rstd), codes ? eight.c() : nullptr,
                                      codes ? eight.e() : nullptr, rows, (int32_t)D, eps, dtype_code(x), flags, current_stream());
        if (rc != SPION_OK) throw SpionFailure{rc, "spion_rms_norm"};
    }
};

// The gradient of rms_norm: of x, weight and, if there was one, the residual, whose is x's.  The second incoming one is that of the stream h, or of a
// residual from x (see residual).
struct RmsNormBackward : public TakesResidual {
    torch::autograd::SavedVariable h, codes, exponents, w, rstd;   // h, which may be x, or codes and exponents
    std::vector<int64_t> sizes;
    bool has_residual = false, eight = false, h_is_output = false;
    at::ScalarType type = at::kFloat;

    std::string name() const override { return "RmsNormBackward"; }

    void release_variables() override {
        for (torch::autograd::SavedVariable* s : {&h, &codes, &exponents, &w, &rstd}) s->reset_data();
    }

    torch::autograd::variable_list apply(torch::autograd::variable_list&& grads) override {
        torch::autograd::variable_list out(has_residual ? 3 : 2);
        at::Tensor dh = grads.size() > 1 ? grads[1] : at::Tensor();
        auto give = [&](const at::Tensor& dx) {
            if (task_should_compute_output(0)) out[0] = dx;
            if (has_residual && task_should_compute_output(2)) out[2] = dx;
        };
        if (!grads[0].defined()) {
            give(dh);
            return out;
        }
        return differentiate("rms_norm cannot be differentiated twice", grads[0], [&] {
            check_gradient(dh);
            const char* const other = "rms_norm: a saved tensor is not the one that was saved";
            const at::Device device = grads[0].device();
            const c10::DeviceGuard guard(device);
            const at::Tensor g = grads[0].contiguous(), W = w.unpack(), rs = rstd.unpack();
            if (dh.defined()) dh = dh.contiguous();
            const int64_t D = sizes.back(), rows = rows_of(g);
            saved(as_saved(W, device, type) && W.dim() == 1 && W.size(0) == D && as_saved(rs, device, at::kFloat) && rs.numel() == rows, other);
            Eight from;
            at::Tensor H;
            if (eight) {
                from.codes = codes.unpack();
                from.exponents = exponents.unpack();
                const int64_t pitch = (D + 63) / 64 * 64;
                saved(as_saved(from.codes, device, at::kChar) && from.codes.numel() == rows * pitch && as_saved(from.exponents, device, at::kByte) &&
                          from.exponents.numel() == rows * (pitch / 64) && (uintptr_t)from.codes.data_ptr() % 8 == 0, other);
            } else {
                H = h_is_output ? h.unpack(shared_from_this()) : h.unpack();
                saved(as_saved(H, device, type) && H.numel() == g.numel(), other);
            }
            at::Tensor dx = new_like(g), dw;
            if (task_should_compute_output(1)) dw = rows == 0 ? at::zeros({D}, W.options()) : new_like(W);
            if (rows > 0) {
                at::Tensor ws;
                if (dw.defined()) ws = new_bytes(spion_rms_norm_workspace_bytes(rows, (int32_t)D), g);
                const int rc = spion_rms_norm_grad(device_ptr(g), dh.defined() ? device_ptr(dh) : nullptr, eight ? nullptr : device_ptr(H), eight ? from.c() : nullptr,
                                                   eight ? from.e() : nullptr, device_ptr(W), (const float*)device_ptr(rs), device_ptr(dx),
                                                   dw.defined() ? device_ptr(dw) : nullptr, rows, (int32_t)D, dtype_code(g), ws.defined() ? ws.data_ptr() : nullptr,
                                                   ws.defined() ? (size_t)ws.nbytes() : 0, current_stream());
                if (rc != SPION_OK) throw SpionFailure{rc, "spion_rms_norm_grad"};
            }
            give(dx);
            out[1] = dw;
            return out;
        });
    }
};

PyObject* optional(const at::Tensor& t) {
    if (t.defined()) return wrap(t);
    Py_RETURN_NONE;
}

// rms_norm(x, weight, residual | None, eps, checkpoint) -> (y, h | None, codes | None, exponents | None)
PyObject* py_rms_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arg_count(n, 5, "rms_norm")) return nullptr;
    return guarded([&]() -> PyObject* {
        not_traced();
        const at::Tensor &x = tensor_arg(a[0]), &w = tensor_arg(a[1]);
        const at::Tensor residual = optional_arg(a[2]);
        const NormArgs args(x, w, residual, a[3]);
        const bool checkpoint = truth_arg(a[4]);
        const c10::DeviceGuard guard(x.device());
        const bool grad = residual.defined() ? torch::autograd::compute_requires_grad(x, w, residual) : torch::autograd::compute_requires_grad(x, w);
        at::Tensor y = new_like(args.x), h, rstd;
        if (residual.defined()) h = new_like(args.x);
        if (grad) rstd = new_tensor({args.rows}, at::kFloat, x.device());
        const Eight eight = checkpoint ? Eight(args.x) : Eight();
        args.run(y, h, rstd, eight, 0);
        if (grad) {
            auto node = std::shared_ptr<RmsNormBackward>(new RmsNormBackward(), torch::autograd::deleteNode);
            node->set_next_edges(residual.defined() ? torch::autograd::collect_next_edges(x, w, residual) : torch::autograd::collect_next_edges(x, w));
            node->sizes = args.x.sizes().vec();
            node->type = args.x.scalar_type();
            node->has_residual = residual.defined();
            node->eight = checkpoint;
            node->w = torch::autograd::SavedVariable(args.w, false);
            node->rstd = torch::autograd::SavedVariable(rstd, false);
            torch::autograd::set_history(y, node);
            if (h.defined()) torch::autograd::set_history(h, node);
            if (checkpoint) {
                node->codes = torch::autograd::SavedVariable(eight.codes, false);
                node->exponents = torch::autograd::SavedVariable(eight.exponents, false);
            } else {
                node->h_is_output = h.defined();
                node->h = h.defined() ? torch::autograd::SavedVariable(h, true) : torch::autograd::SavedVariable(args.x, false);
            }
        }
        PyObject* r = PyTuple_New(4);
        if (!r) return nullptr;
        PyTuple_SET_ITEM(r, 0, wrap(y));
        PyTuple_SET_ITEM(r, 1, optional(h));
        PyTuple_SET_ITEM(r, 2, optional(eight.codes));
        PyTuple_SET_ITEM(r, 3, optional(eight.exponents));
        return r;
    });
}

// rms_norm8(x, weight, residual | None, eps) -> (codes, exponents, h | None)
PyObject* py_rms_norm8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arg_count(n, 4, "rms_norm8")) return nullptr;
    return guarded([&]() -> PyObject* {
        not_traced();
        const at::Tensor &x = tensor_arg(a[0]), &w = tensor_arg(a[1]);
        const at::Tensor residual = optional_arg(a[2]);
        if (residual.defined() ? torch::autograd::compute_requires_grad(x, w, residual) : torch::autograd::compute_requires_grad(x, w))
            bad_value("rms_norm8 has no gradient: call it under torch.no_grad()");
        const NormArgs args(x, w, residual, a[3]);
        const c10::DeviceGuard guard(x.device());
        at::Tensor h;
        if (residual.defined()) h = new_like(args.x);
        const Eight eight(args.x);
        args.run(at::Tensor(), h, at::Tensor(), eight, SPION_NORM_CODES_OF_Y);
        PyObject* r = PyTuple_New(3);
        if (!r) return nullptr;
        PyTuple_SET_ITEM(r, 0, wrap(eight.codes));
        PyTuple_SET_ITEM(r, 1, wrap(eight.exponents));
        PyTuple_SET_ITEM(r, 2, optional(h));
        return r;
    });
}

// The gradient of linear8: x's as a library product unless it is small, the weight's and the bias' from the codes.  x's is rounded to x's type, as autograd
// hands it on: in bf16 a norm in front of the projection has it with an error of up to 2^-8, and rounds its own gradient once more.
struct Linear8Backward : public torch::autograd::Node {
    torch::autograd::SavedVariable codes, exponents, column, w;   // column: the weight of the codes, if they have one
    std::vector<int64_t> sizes;   // of x
    bool has_bias = false, has_column = false;
    at::ScalarType type = at::kFloat;

    std::string name() const override { return "Linear8Backward"; }

    void release_variables() override {
        for (torch::autograd::SavedVariable* s : {&codes, &exponents, &column, &w}) s->reset_data();
    }

    torch::autograd::variable_list apply(torch::autograd::variable_list&& grads) override {
        torch::autograd::variable_list out(has_bias ? 3 : 2);
        if (!grads[0].defined()) return out;
        return differentiate("linear8 cannot be differentiated twice", grads[0], [&] {
            const char* const other = "linear8: a saved tensor is not the one that was saved";
            const at::Device device = grads[0].device();
            const c10::DeviceGuard guard(device);
            const c10::impl::ExcludeDispatchKeyGuard no_autocast(c10::autocast_dispatch_keyset);
            const int64_t M = sizes.back(), N = grads[0].size(-1);
            const at::Tensor g = grads[0].reshape({-1, N}).contiguous();
            const int64_t rows = g.size(0);
            const bool needs_w = task_should_compute_output(1), needs_b = has_bias && task_should_compute_output(2);
            if (task_should_compute_output(0)) {
                const at::Tensor W = w.unpack();
                saved(W.defined() && W.device() == device && W.dim() == 2 && W.size(0) == N && W.size(1) == M && W.scalar_type() == type, other);
                if (W.is_contiguous() && !transformed(W) && spion_input_grad_suits((int32_t)rows, (int32_t)N, (int32_t)M)) {
                    out[0] = new_tensor(sizes, type, device);
                    const int rc = spion_input_grad(device_ptr(g), device_ptr(W), device_ptr(out[0]), (int32_t)rows, (int32_t)N, (int32_t)M, dtype_code(g),
                                                    current_stream());
                    if (rc != SPION_OK) throw SpionFailure{rc, "spion_input_grad"};
                } else {
                    out[0] = at::mm(g, W).view(sizes);
                }
            }
            if (needs_w && rows > 0) {
                Eight from;
                from.codes = codes.unpack();
                from.exponents = exponents.unpack();
                const at::Tensor col = has_column ? column.unpack() : at::Tensor();
                const int64_t pitch = (M + 63) / 64 * 64;
                saved(as_saved(from.codes, device, at::kChar) && from.codes.numel() == rows * pitch && as_saved(from.exponents, device, at::kByte) &&
                          from.exponents.numel() == rows * (pitch / 64) && (uintptr_t)from.codes.data_ptr() % 16 == 0 &&
                          (!has_column || (as_saved(col, device, type) && col.numel() == M)), other);
                out[1] = new_tensor({N, M}, type, device);
                if (needs_b) out[2] = new_tensor({N}, type, device);
                const size_t bytes = spion_weight_grad_eight_workspace_bytes((int32_t)rows, (int32_t)N, (int32_t)M);
                if (bytes == (size_t)-1) throw SpionFailure{SPION_ERR_SHAPE, "spion_weight_grad_eight_workspace_bytes"};
                const at::Tensor ws = new_bytes(bytes, g);
                const int rc = spion_weight_grad_eight(device_ptr(g), from.c(), from.e(), has_column ? device_ptr(col) : nullptr, device_ptr(out[1]),
                                                       needs_b ? device_ptr(out[2]) : nullptr, (int32_t)rows, (int32_t)N, (int32_t)M, dtype_code(g), ws.data_ptr(),
                                                       (size_t)ws.nbytes(), current_stream());
                if (rc != SPION_OK) throw SpionFailure{rc, "spion_weight_grad_eight"};
            } else {
                if (needs_w) out[1] = at::zeros({N, M}, g.options());
                if (needs_b) out[2] = g.sum(0);
            }
            return out;
        });
    }
};

// linear8(x, weight, bias | None, codes | None, exponents | None, column weight | None) -> y
PyObject* py_linear8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arg_count(n, 6, "linear8")) return nullptr;
    return guarded([&]() -> PyObject* {
        not_traced();
        const at::Tensor &x = tensor_arg(a[0]), &w = tensor_arg(a[1]);
        const at::Tensor b = optional_arg(a[2]), c = optional_arg(a[3]);
        check_operand(x, std::nullopt);
        const at::Device device = x.device();
        check_operand(w, device);
        dtype_code(x);
        const int64_t rows = rows_of(x), M = x.size(-1);
        if (w.dim() != 2 || w.size(1) != M || w.size(0) < 1 || w.scalar_type() != x.scalar_type()) bad_value("weight must be [N, M] for x [..., M], of x's dtype");
        const int64_t N = w.size(0);
        if (b.defined()) {
            check_operand(b, device);
            if (b.dim() != 1 || b.size(0) != N || b.scalar_type() != x.scalar_type()) bad_value("bias must be [N], of x's dtype");
        }
        if (M > 1 << 20 || N > 1 << 20 || rows >= 0x7fffffff - 4096 || (rows > 0 && spion_weight_grad_eight_workspace_bytes((int32_t)rows, (int32_t)N, (int32_t)M) == (size_t)-1))
            bad_value("linear8: too many rows or too large a weight");
        const c10::DeviceGuard guard(device);
        Eight eight;
        at::Tensor column;
        if (c.defined()) {
            eight = Eight(c, tensor_arg(a[4]), x.sizes().slice(0, x.dim() - 1), M, device);
            column = optional_arg(a[5]);
            if (column.defined()) {
                check_operand(column, device);
                if (column.dim() != 1 || column.size(0) != M || column.scalar_type() != x.scalar_type()) bad_value("the checkpoint's weight must be [M], of x's dtype");
            }
        }
        const bool grad = b.defined() ? torch::autograd::compute_requires_grad(x, w, b) : torch::autograd::compute_requires_grad(x, w);
        const bool keeps = grad && w.requires_grad();
        at::Tensor y;
        {
            at::NoGradGuard no_grad;
            const c10::impl::ExcludeDispatchKeyGuard no_autocast(c10::autocast_dispatch_keyset);
            y = linear_of(x, w, b);
            if (keeps && !c.defined()) {
                const at::Tensor xc = x.contiguous();
                eight = Eight(xc);
                pack(xc, eight);
            }
            if (column.defined()) column = column.contiguous();
        }
        if (grad) {
            auto node = std::shared_ptr<Linear8Backward>(new Linear8Backward(), torch::autograd::deleteNode);
            node->set_next_edges(b.defined() ? torch::autograd::collect_next_edges(x, w, b) : torch::autograd::collect_next_edges(x, w));
            node->sizes = x.sizes().vec();
            node->type = x.scalar_type();
            node->has_bias = b.defined();
            node->w = torch::autograd::SavedVariable(w, false);
            if (keeps) {
                node->codes = torch::autograd::SavedVariable(eight.codes, false);
                node->exponents = torch::autograd::SavedVariable(eight.exponents, false);
                node->has_column = column.defined();
                if (column.defined()) node->column = torch::autograd::SavedVariable(column, false);
            }
            torch::autograd::set_history(y, node);
        }
        return wrap(y);
    });
}

// generate_pattern(A_s, L, block, filter, mode, value, flags, fl_out, row_ptr, col_idx, col_ptr, row_idx, bsr_pos,
//                  nnzb, pool_sum, workspace | None) -> nnzb, after the pattern is complete
PyObject* py_generate_pattern(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arg_count(n, 16, "generate_pattern")) return nullptr;
    return guarded([&]() -> PyObject* {
        const at::Tensor& A = tensor_arg(a[0]);
        device_ptr(A);
        spion_pattern_params p;
        p.L = int_arg(a[1]);
        p.block = int_arg(a[2]);
        p.filter = int_arg(a[3]);
        p.thresh_mode = int_arg(a[4]);
        p.thresh_value = double_arg(a[5]);
        p.flags = (uint32_t)int_arg(a[6]);
        p.reserved = 0;
        void* ptr[8];
        for (int i = 0; i < 8; ++i) ptr[i] = a[7 + i] == Py_None ? nullptr : device_ptr(tensor_arg(a[7 + i]));
        at::Tensor ws = optional_arg(a[15]);
        if (!ws.defined()) ws = new_bytes(spion_pattern_workspace_bytes(p.L, p.block), A);
        void *score = device_ptr(A), *work = device_ptr(ws), *stream = current_stream();
        const size_t work_bytes = (size_t)ws.nbytes();
        int32_t nnzb = -1;
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = spion_pattern_wait((const float*)score, &p, (uint8_t*)ptr[0], (int32_t*)ptr[1], (int32_t*)ptr[2],
                                (int32_t*)ptr[3], (int32_t*)ptr[4], (int32_t*)ptr[5], (int32_t*)ptr[6], (int64_t*)ptr[7],
                                work, work_bytes, stream, &nnzb);
        Py_END_ALLOW_THREADS
        if (rc != SPION_OK) throw SpionFailure{rc, "spion_pattern"};
        return PyLong_FromLong(nnzb);
    });
}

PyObject* py_set_error_class(PyObject*, PyObject* cls) {
    Py_INCREF(cls);
    Py_XSETREF(g_error_class, cls);
    Py_RETURN_NONE;
}

PyMethodDef kMethods[] = {
    {"attn_fwd", (PyCFunction)(void*)py_attn_fwd, METH_FASTCALL, nullptr},
    {"attn_bwd", (PyCFunction)(void*)py_attn_bwd, METH_FASTCALL, nullptr},
    {"sparse_attention", (PyCFunction)(void*)py_sparse_attention, METH_FASTCALL, nullptr},
    {"heads_attention_with", (PyCFunction)(void*)py_heads_attention_with, METH_FASTCALL, nullptr},
    {"heads_attention", (PyCFunction)(void*)py_heads_attention, METH_FASTCALL, nullptr},
    {"layer_norm", (PyCFunction)(void*)py_layer_norm, METH_FASTCALL, nullptr},
    {"residual", (PyCFunction)(void*)py_residual, METH_FASTCALL, nullptr},
    {"projection", (PyCFunction)(void*)py_projection, METH_FASTCALL, nullptr},
    {"sparse_attention_with", (PyCFunction)(void*)py_sparse_attention_with, METH_FASTCALL, nullptr},
    {"relative_bias", (PyCFunction)(void*)py_relative_bias, METH_FASTCALL, nullptr},
    {"dropout_add", (PyCFunction)(void*)py_dropout_add, METH_FASTCALL, nullptr},
    {"rotary", (PyCFunction)(void*)py_rotary, METH_FASTCALL, nullptr},
    {"pack8", (PyCFunction)(void*)py_pack8, METH_FASTCALL, nullptr},
    {"unpack8", (PyCFunction)(void*)py_unpack8, METH_FASTCALL, nullptr},
    {"rms_norm", (PyCFunction)(void*)py_rms_norm, METH_FASTCALL, nullptr},
    {"rms_norm8", (PyCFunction)(void*)py_rms_norm8, METH_FASTCALL, nullptr},
    {"linear8", (PyCFunction)(void*)py_linear8, METH_FASTCALL, nullptr},
    {"generate_pattern", (PyCFunction)(void*)py_generate_pattern, METH_FASTCALL, nullptr},
    {"set_error_class", py_set_error_class, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_spion_host", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__spion_host(void) { return PyModule_Create(&kModule); }
