// The Python binding's common calls, marshalled natively: tensors in, one C call of libtbik, the new output tensor out.
//
// A call on a few rows is over on the GPU before Python has issued it.  Host time of a call through ctypes -> here, its launches (2.2 us
// each) included: 1 x 4096 x 4096 in bf16, two launches, 9.95 -> 6.9 us, in 8 bits, one, 8.0 -> 4.0; RMSNorm of a row 5.3 -> 4.0, attention
// of two short sequences 10.2 -> 4.4; since output() puts tensors together itself, 0.4 less for each output (RMSNorm with the residual to 8
// bits, three of them, 5.8 -> 4.8).  What a function below returns:
//   the output tensor(s), or an int: the library's status where it is not TBIK_OK, or None: "not one of the common calls" --
// an argument of another type, a view it would refuse, a tensor subclass, anything odd.  The caller then takes the way
// through ctypes, which answers every call as it always did, its errors included.  Nothing is decided here and nothing is kept between calls
// but the entry points' addresses; scratch memory comes from the binding's own cache of workspaces, by device and stream.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <climits>
#include <cstdint>

#include <ATen/ATen.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPGraphsC10Utils.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include "tbik.h"

namespace {

enum Kind { GEMM, GEMM_F32, PARTIALS, PARTIALS_F32, SWIGLU, FP8, MX, MXFP4, RMSNORM, COMBINE, ROWS, ATTENTION,
            EPILOGUE, EPILOGUE_FP8, EPILOGUE_MX, EPILOGUE_COMBINE, NORM8, NORM8_MX, TAIL8, TAIL8_MX, SILU8, SILU8_MX,
            ROUTE, GROUPED, GROUPED_SWIGLU, GROUPED_PARTIALS, EXPERTS_SUM, W4, W4_PARTIALS, JOIN, KINDS };
struct Entry {
    int kind = -1;
    void *call = nullptr, *need = nullptr;      // the C entry point and its workspace query
    at::ScalarType dtype = at::kFloat;          // of its operands
};
constexpr int MAX_ENTRIES = 48;
Entry entries[MAX_ENTRIES];                     // written while the library is loaded, under the interpreter lock
PyObject *workspaces = nullptr;                 // the binding's dict: (device index, stream) -> uint8 tensor
PyObject *make_workspace = nullptr;             // the binding's function that fills it

// A plain strided GPU tensor: no subclass, no wrapper of a transform, real sizes and memory.
const at::Tensor *plain(PyObject *o, int dim) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    const auto *impl = t.unsafeGetTensorImpl();
    const auto keys = t.key_set();
    if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || !t.has_storage() || t.dim() != dim || impl->has_symbolic_sizes_strides() ||
        keys.has(c10::DispatchKey::Python) || keys.has(c10::DispatchKey::Functionalize) || keys.has(c10::DispatchKey::FuncTorchBatched) ||
        keys.has(c10::DispatchKey::FuncTorchGradWrapper) || keys.has(c10::DispatchKey::Conjugate) || keys.has(c10::DispatchKey::Negative))
        return nullptr;
    return &t;
}
const at::Tensor *matrix(PyObject *o, at::ScalarType dtype) {
    const at::Tensor *t = plain(o, 2);
    return t && t->scalar_type() == dtype && t->stride(1) == 1 && t->size(0) <= INT_MAX && t->size(1) <= INT_MAX ? t : nullptr;
}
bool integer(PyObject *o, int *v) {
    if (!PyLong_CheckExact(o)) return false;
    int overflow = 0;
    const long x = PyLong_AsLongAndOverflow(o, &overflow);
    if (overflow || x < INT_MIN || x > INT_MAX) return false;
    *v = (int)x;
    return true;
}
bool number(PyObject *o, float *v) {
    if (!PyFloat_CheckExact(o)) return false;
    *v = (float)PyFloat_AS_DOUBLE(o);
    return true;
}
int type_code(at::ScalarType t) { return t == at::kFloat ? TBIK_F32 : t == at::kBFloat16 ? TBIK_BF16 : t == at::kHalf ? TBIK_F16 : -1; }

// A new tensor on `like`'s device, undefined unless it is a real one (a dispatch mode may hand out something else).  Where only torch's default
// keys take part in a call it is put together here, from the allocator that torch's own come from: 0.27 us, through the dispatcher 0.70.
at::Tensor output(at::IntArrayRef sizes, const at::Tensor &like, at::ScalarType dtype) {
    const auto torchs = [&](at::IntArrayRef n, at::ScalarType type) { return at::empty(n, like.options().dtype(type).requires_grad(false)); };
    const auto real = [](const at::Tensor &t) { return t.is_cuda() && t.has_storage() && !t.key_set().has(c10::DispatchKey::Python); };
    static c10::Allocator *allocator = nullptr;               // the same for the life of the process; under the interpreter lock
    int64_t bytes = (int64_t)c10::elementSize(dtype);
    bool direct = (c10::impl::tls_local_dispatch_key_set().included_ - c10::default_included_set).empty() && like.device().index() == c10::hip::current_device();
    for (const int64_t n : sizes) direct = direct && !__builtin_mul_overflow(bytes, n, &bytes);
    if (direct && !allocator) {
        const at::Tensor t = torchs({1}, at::kByte);
        if (real(t)) allocator = t.storage().allocator();
    }
    if (!direct || !allocator) {
        at::Tensor t = torchs(sizes, dtype);
        return real(t) ? t : at::Tensor();
    }
    at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(
        c10::make_intrusive<c10::StorageImpl>(c10::StorageImpl::use_byte_size_t(), bytes, allocator->allocate((size_t)bytes), allocator, true),
        c10::DispatchKeySet(c10::DispatchKey::CUDA), c10::scalarTypeToTypeMeta(dtype));
    t.unsafeGetTensorImpl()->set_sizes_contiguous(sizes);
    return t;
}

// torch's current stream on the current device, as the binding passes it.
void *current_stream() { return (void *)c10::hip::getCurrentHIPStream(c10::hip::current_device()).stream(); }

// Holds its tensor: while the interpreter lock is released another thread may put a larger one into the dict, and the
// allocator would give this one's memory away before the call's kernels are queued.
struct Room {
    at::Tensor held;
    void *at = nullptr;
    size_t bytes = 0;
    void take(const at::Tensor &ws) {
        held = ws;
        at = held.data_ptr();
        bytes = (size_t)held.numel();
    }
};
// The workspace of `need` bytes for `like`'s device and this stream; false: an error is set.
bool room_for(size_t need, PyObject *like, const at::Tensor &t, void *stream, Room *room) {
    if (need == 0) return true;
    PyObject *key = Py_BuildValue("(iK)", (int)t.device().index(), (unsigned long long)(uintptr_t)stream);
    if (!key) return false;
    PyObject *w = PyDict_GetItemWithError(workspaces, key);       // borrowed
    Py_DECREF(key);
    if (!w && PyErr_Occurred()) return false;
    if (w && THPVariable_Check(w)) {
        const at::Tensor &ws = THPVariable_Unpack(w);
        if ((size_t)ws.numel() >= need) {
            room->take(ws);
            return true;
        }
    }
    PyObject *device = PyObject_GetAttrString(like, "device");
    if (!device) return false;
    PyObject *made = PyObject_CallFunction(make_workspace, "KO", (unsigned long long)need, device);
    Py_DECREF(device);
    if (!made) return false;
    room->take(THPVariable_Unpack(made));
    Py_DECREF(made);
    return true;
}

#define UNCOMMON Py_RETURN_NONE
PyObject *wrapped(at::Tensor t, int status) { return status == 0 ? THPVariable_Wrap(std::move(t)) : PyLong_FromLong(status); }
const Entry *entry_of(PyObject *o, int kind_from, int kind_to) {
    int i;
    if (!integer(o, &i) || i < 0 || i >= MAX_ENTRIES || entries[i].kind < kind_from || entries[i].kind > kind_to) return nullptr;
    return &entries[i];
}

// Entries are called through the types that tbik.h declares for them; those of one kind have one type.
#define SAME(a, b) static_assert(std::is_same<decltype(&a), decltype(&b)>::value, #a " and " #b)
SAME(tbik_gemm, tbik_gemm_f16);
SAME(tbik_gemm, tbik_gemm_swiglu);
SAME(tbik_gemm_shard_partials, tbik_gemm_shard_partials_f16);
SAME(tbik_gemm_shard_partials, tbik_gemm_shard_partials_f32);
SAME(tbik_gemm_mxfp8, tbik_gemm_mxfp6);
SAME(tbik_rmsnorm, tbik_rmsnorm_f16);
SAME(tbik_combine_residual_rmsnorm, tbik_combine_residual_rmsnorm_f16);
SAME(tbik_attention, tbik_attention_f16);
SAME(tbik_gemm_epilogue, tbik_gemm_fp8_epilogue);
SAME(tbik_gemm_16bit_workspace_bytes, tbik_gemm_f32_workspace_bytes);
SAME(tbik_gemm_16bit_workspace_bytes, tbik_gemm_swiglu_workspace_bytes);
SAME(tbik_gemm_16bit_workspace_bytes, tbik_gemm_fp8_workspace_bytes);
SAME(tbik_gemm_16bit_workspace_bytes, tbik_gemm_mxfp8_workspace_bytes);
SAME(tbik_gemm_16bit_workspace_bytes, tbik_gemm_mxfp6_workspace_bytes);
SAME(tbik_gemm_16bit_workspace_bytes, tbik_gemm_mxfp4_workspace_bytes);
SAME(tbik_gemm_16bit_workspace_bytes, tbik_attention_workspace_bytes);
#undef SAME
#define CALL(name) ((decltype(&name))e->call)
#define NEED(name) ((decltype(&name))e->need)
typedef void *P;
typedef int64_t L;

// product(entry, X, Xs, W, Ws, leaf, k_first, out dtype (None where the kind has one of its own), format or shards)
PyObject *product(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 9) UNCOMMON;
    const Entry *e = entry_of(a[0], GEMM, MXFP4);
    int leaf, k_first, extra;
    if (!e || !integer(a[5], &leaf) || !integer(a[6], &k_first) || !integer(a[8], &extra)) UNCOMMON;
    const int kind = e->kind;
    try {
        const at::Tensor *X = matrix(a[1], e->dtype), *W = matrix(a[3], e->dtype);
        if (!X || !W) UNCOMMON;
        const at::Tensor *Xs = nullptr, *Ws = nullptr;
        at::ScalarType out_type = at::kFloat;
        if (kind == GEMM || kind >= FP8) {                        // None there is for torch to answer: new_empty takes X's type
            if (!THPDtype_Check(a[7])) UNCOMMON;
            out_type = ((THPDtype *)a[7])->scalar_type;
        }
        if (type_code(out_type) < 0) UNCOMMON;
        const int M = (int)X->size(0);
        int K = (int)X->size(1), N;
        if (kind <= SWIGLU) {                                     // W [K, N]
            if (W->size(0) != K) UNCOMMON;
            N = (int)W->size(1);
            if (kind == SWIGLU) {
                if (N % 2) UNCOMMON;
                N /= 2;
            }
        } else {                                                  // W [N, bytes of K]
            if (W->size(1) != K) UNCOMMON;
            N = (int)W->size(0);
            if (kind != FP8) {
                Xs = matrix(a[2], at::kByte);
                Ws = matrix(a[4], at::kByte);
                if (!Xs || !Ws) UNCOMMON;
                if (kind == MXFP4) {
                    if (K > INT_MAX / 2) UNCOMMON;
                    K *= 2;
                } else if (extra >= 6) {                          // 6-bit elements: four in three bytes
                    if (K > INT_MAX / 4 || K % 3) UNCOMMON;
                    K = K / 3 * 4;
                }
                if (Xs->size(0) != M || Xs->size(1) != K / 32 || Ws->size(0) != N || Ws->size(1) != K / 32) UNCOMMON;
            }
        }
        const bool partials = kind == PARTIALS || kind == PARTIALS_F32;
        if (partials && extra < 1) UNCOMMON;
        at::Tensor Y = partials ? output({extra, M, N}, *X, at::kFloat)
                                : output({M, N}, *X, kind == SWIGLU ? e->dtype : kind == GEMM_F32 ? at::kFloat : out_type);
        if (!Y.defined()) UNCOMMON;
        void *stream = current_stream();
        Room ws;
        if (!room_for(e->need ? NEED(tbik_gemm_16bit_workspace_bytes)(M, N, K, leaf, k_first) : 0, a[1], *X, stream, &ws)) return nullptr;
        P x = X->data_ptr(), w = W->data_ptr(), y = Y.data_ptr(), xs = Xs ? Xs->data_ptr() : nullptr, wsc = Ws ? Ws->data_ptr() : nullptr;
        const L ldx = X->stride(0), ldw = W->stride(0), ldxs = Xs ? Xs->stride(0) : 0, ldws = Ws ? Ws->stride(0) : 0, ldy = partials ? 0 : Y.stride(0);
        const tbik_dtype yt = (tbik_dtype)type_code(Y.scalar_type());
        int st = 0;
        Py_BEGIN_ALLOW_THREADS
        switch (kind) {
            case GEMM:
            case SWIGLU: st = CALL(tbik_gemm)(x, ldx, w, ldw, y, ldy, yt, M, N, K, leaf, k_first, ws.at, ws.bytes, stream); break;
            case GEMM_F32: st = CALL(tbik_gemm_f32)(x, ldx, w, ldw, y, ldy, M, N, K, leaf, k_first, ws.at, ws.bytes, stream); break;
            case PARTIALS:
            case PARTIALS_F32: st = CALL(tbik_gemm_shard_partials)(x, ldx, w, ldw, (float *)y, M, N, K, leaf, k_first, extra, ws.at, ws.bytes, stream); break;
            case FP8: st = CALL(tbik_gemm_fp8)(x, ldx, w, ldw, y, ldy, yt, (tbik_dtype)extra, M, N, K, leaf, k_first, ws.at, ws.bytes, stream); break;
            case MX: st = CALL(tbik_gemm_mxfp8)(x, ldx, xs, ldxs, w, ldw, wsc, ldws, y, ldy, yt, (tbik_dtype)extra, M, N, K, leaf, k_first, ws.at, ws.bytes, stream); break;
            case MXFP4: st = CALL(tbik_gemm_mxfp4)(x, ldx, xs, ldxs, w, ldw, wsc, ldws, y, ldy, yt, M, N, K, leaf, k_first, ws.at, ws.bytes, stream); break;
        }
        Py_END_ALLOW_THREADS
        return wrapped(std::move(Y), st);
    } catch (const std::exception &) {
        if (PyErr_Occurred()) return nullptr;
        UNCOMMON;
    }
}

// A part of an epilogue: None, or a plain contiguous vector of n elements.  False: not a common one.
bool part(PyObject *o, int n, const at::Tensor **t) {
    *t = nullptr;
    if (o == Py_None) return true;
    *t = plain(o, 1);
    return *t && (*t)->size(0) == n && (n == 1 || (*t)->stride(0) == 1) && type_code((*t)->scalar_type()) >= 0;
}
bool elsewhere(const at::Tensor *t, const at::Tensor &like) { return t && t->device() != like.device(); }

// The parts of an epilogue (row_scale, col_scale, bias, activation, residual in a[0 .. 4]) of an output [M, N] like `like` of out_type.
bool epilogue_of(PyObject *const *a, int M, int N, const at::Tensor &like, at::ScalarType out_type, tbik_epilogue *e) {
    const at::Tensor *rs, *cs, *bias, *res = nullptr;
    int act;
    if (!part(a[0], M, &rs) || !part(a[1], N, &cs) || !part(a[2], N, &bias) || !integer(a[3], &act)) return false;
    if (a[4] != Py_None && !(res = matrix(a[4], out_type))) return false;
    if ((rs && rs->scalar_type() != at::kFloat) || (cs && cs->scalar_type() != at::kFloat) || (res && (res->size(0) != M || res->size(1) != N))) return false;
    if (like.device().index() != c10::hip::current_device() || elsewhere(rs, like) || elsewhere(cs, like) || elsewhere(bias, like) || elsewhere(res, like)) return false;
    *e = {rs ? (const float *)rs->data_ptr() : nullptr, cs ? (const float *)cs->data_ptr() : nullptr, bias ? bias->data_ptr() : nullptr,
          (tbik_dtype)(bias ? type_code(bias->scalar_type()) : 0), (tbik_activation)act, res ? res->data_ptr() : nullptr, res ? res->stride(0) : 0};
    return true;
}

// epilogue(entry, X, Xs, W, Ws, leaf, k_first, out dtype, format, row_scale, col_scale, bias, activation, residual); EPILOGUE_COMBINE: X the partial sums
PyObject *epilogue(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 14) UNCOMMON;
    const Entry *e = entry_of(a[0], EPILOGUE, EPILOGUE_COMBINE);
    int leaf, k_first, fmt;
    if (!e || !integer(a[5], &leaf) || !integer(a[6], &k_first) || !integer(a[8], &fmt) || !THPDtype_Check(a[7])) UNCOMMON;
    const int kind = e->kind;
    const at::ScalarType out_type = ((THPDtype *)a[7])->scalar_type;
    if (type_code(out_type) < 0) UNCOMMON;
    try {
        const at::Tensor *X = kind == EPILOGUE_COMBINE ? plain(a[1], 3) : matrix(a[1], e->dtype), *W = nullptr, *Xs = nullptr, *Ws = nullptr;
        if (!X) UNCOMMON;
        int M, N, K = 0;
        if (kind == EPILOGUE_COMBINE) {
            if (X->scalar_type() != at::kFloat || !X->is_contiguous() || X->size(0) > INT_MAX || X->size(1) > INT_MAX || X->size(2) > INT_MAX) UNCOMMON;
            M = (int)X->size(1);
            N = (int)X->size(2);
        } else {
            if (!(W = matrix(a[3], e->dtype))) UNCOMMON;
            M = (int)X->size(0);
            K = (int)X->size(1);
            N = (int)W->size(kind == EPILOGUE ? 1 : 0);
            if (W->size(kind == EPILOGUE ? 0 : 1) != K || elsewhere(W, *X)) UNCOMMON;
            if (kind == EPILOGUE_MX) {
                Xs = matrix(a[2], at::kByte);
                Ws = matrix(a[4], at::kByte);
                if (!Xs || !Ws || Xs->size(0) != M || Xs->size(1) != K / 32 || Ws->size(0) != N || Ws->size(1) != K / 32 || elsewhere(Xs, *X) || elsewhere(Ws, *X)) UNCOMMON;
            }
        }
        tbik_epilogue ends;
        if (!epilogue_of(a + 9, M, N, *X, out_type, &ends)) UNCOMMON;
        at::Tensor Y = output({M, N}, *X, out_type);
        if (!Y.defined()) UNCOMMON;
        void *stream = current_stream();
        Room ws;
        if (!room_for(e->need ? NEED(tbik_gemm_16bit_workspace_bytes)(M, N, K, leaf, k_first) : 0, a[1], *X, stream, &ws)) return nullptr;
        P x = X->data_ptr(), w = W ? W->data_ptr() : nullptr, y = Y.data_ptr(), xs = Xs ? Xs->data_ptr() : nullptr, wsc = Ws ? Ws->data_ptr() : nullptr;
        const L ldx = X->stride(0), ldw = W ? W->stride(0) : 0, ldxs = Xs ? Xs->stride(0) : 0, ldws = Ws ? Ws->stride(0) : 0, ldy = Y.stride(0);
        const int shards = kind == EPILOGUE_COMBINE ? (int)X->size(0) : 0;
        const tbik_dtype yt = (tbik_dtype)type_code(out_type), xt = (tbik_dtype)(kind == EPILOGUE ? type_code(e->dtype) : fmt);
        int st = 0;
        Py_BEGIN_ALLOW_THREADS
        if (kind == EPILOGUE_COMBINE) st = CALL(tbik_tree_combine_epilogue)((const float *)x, shards, &ends, y, ldy, yt, M, N, stream);
        else if (kind == EPILOGUE_MX) st = CALL(tbik_gemm_mxfp8_epilogue)(x, ldx, xs, ldxs, w, ldw, wsc, ldws, &ends, y, ldy, yt, xt, M, N, K, leaf, k_first, ws.at, ws.bytes, stream);
        else st = CALL(tbik_gemm_epilogue)(x, ldx, w, ldw, &ends, y, ldy, yt, xt, M, N, K, leaf, k_first, ws.at, ws.bytes, stream);
        Py_END_ALLOW_THREADS
        return wrapped(std::move(Y), st);
    } catch (const std::exception &) {
        if (PyErr_Occurred()) return nullptr;
        UNCOMMON;
    }
}

// A new reference to None or to the tensor, or nullptr with an error set.
PyObject *tensor_or_none(at::Tensor &t) {
    if (t.defined()) return THPVariable_Wrap(std::move(t));
    Py_RETURN_NONE;
}

// eight_bits(entry, x / partial sums / gate, residual or None / up, weight (None: the activation), eps, format)
//   -> (hidden or None, q, scale) of the norms, (q, scale) of the activation
PyObject *eight_bits(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 6) UNCOMMON;
    const Entry *e = entry_of(a[0], NORM8, SILU8_MX);
    float eps = 0.0f;
    int fmt;
    if (!e || !integer(a[5], &fmt)) UNCOMMON;
    const int kind = e->kind;
    const bool silu = kind == SILU8 || kind == SILU8_MX, tail = kind == TAIL8 || kind == TAIL8_MX, micro = kind == NORM8_MX || kind == TAIL8_MX || kind == SILU8_MX;
    if (!silu && !number(a[4], &eps)) UNCOMMON;
    try {
        const at::Tensor *x = plain(a[1], tail ? 3 : 2), *second = nullptr, *weight = nullptr;
        if (!x || x->size(-2) > INT_MAX || x->size(-1) > INT_MAX) UNCOMMON;
        const int M = (int)x->size(-2), H = (int)x->size(-1);
        if (H == 0) UNCOMMON;
        at::ScalarType dtype = x->scalar_type();
        if (tail) {
            if (dtype != at::kFloat || !x->is_contiguous() || x->size(0) > INT_MAX || a[2] == Py_None) UNCOMMON;
            second = plain(a[2], 2);
            if (!second) UNCOMMON;
            dtype = second->scalar_type();
        } else if (x->stride(1) != 1) UNCOMMON;
        if (dtype != at::kBFloat16 && dtype != at::kHalf) UNCOMMON;
        if (a[2] != Py_None && (!(second = matrix(a[2], dtype)) || second->size(0) != M || second->size(1) != H)) UNCOMMON;
        if (silu ? !second : !((weight = plain(a[3], 1)) && weight->size(0) == H && weight->scalar_type() == dtype && weight->is_contiguous())) UNCOMMON;
        if (x->device().index() != c10::hip::current_device() || elsewhere(second, *x) || elsewhere(weight, *x)) UNCOMMON;
        at::Tensor hidden, q = output({M, H}, *x, at::kByte), scale = micro ? output({M, H / 32}, *x, at::kByte) : output({M}, *x, at::kFloat);
        if (!q.defined() || !scale.defined()) UNCOMMON;
        if (!silu && second) {
            hidden = output({M, H}, *x, dtype);
            if (!hidden.defined()) UNCOMMON;
        }
        P px = x->data_ptr(), p2 = second ? second->data_ptr() : nullptr, pw = weight ? weight->data_ptr() : nullptr, ph = hidden.defined() ? hidden.data_ptr() : nullptr,
          pq = q.data_ptr(), ps = scale.data_ptr(), stream = current_stream();
        const L ldx = x->stride(-2), ld2 = second ? second->stride(0) : 0, ldq = q.stride(0), lds = micro ? scale.stride(0) : 0, ldh = hidden.defined() ? hidden.stride(0) : 0;
        const int shards = tail ? (int)x->size(0) : 0;
        const tbik_dtype t = (tbik_dtype)type_code(dtype), qt = (tbik_dtype)fmt;
        int st = 0;
        Py_BEGIN_ALLOW_THREADS
        switch (kind) {
            case NORM8: st = CALL(tbik_rmsnorm_fp8)(px, ldx, p2, ld2, pw, eps, ph, ldh, pq, ldq, (float *)ps, t, qt, M, H, stream); break;
            case NORM8_MX: st = CALL(tbik_rmsnorm_mxfp8)(px, ldx, p2, ld2, pw, eps, ph, ldh, pq, ldq, ps, lds, t, qt, M, H, stream); break;
            case TAIL8: st = CALL(tbik_combine_residual_rmsnorm_fp8)((const float *)px, shards, p2, ld2, pw, eps, ph, ldh, pq, ldq, (float *)ps, t, qt, M, H, stream); break;
            case TAIL8_MX: st = CALL(tbik_combine_residual_rmsnorm_mxfp8)((const float *)px, shards, p2, ld2, pw, eps, ph, ldh, pq, ldq, ps, lds, t, qt, M, H, stream); break;
            case SILU8: st = CALL(tbik_silu_mul_fp8)(px, ldx, p2, ld2, pq, ldq, (float *)ps, t, qt, M, H, stream); break;
            default: st = CALL(tbik_silu_mul_mxfp8)(px, ldx, p2, ld2, pq, ldq, ps, lds, t, qt, M, H, stream); break;
        }
        Py_END_ALLOW_THREADS
        if (st) return PyLong_FromLong(st);
        PyObject *o[3] = {silu ? nullptr : tensor_or_none(hidden), tensor_or_none(q), tensor_or_none(scale)};
        PyObject *all = !o[1] || !o[2] || (!silu && !o[0]) ? nullptr : silu ? PyTuple_Pack(2, o[1], o[2]) : PyTuple_Pack(3, o[0], o[1], o[2]);
        for (PyObject *i : o) Py_XDECREF(i);
        return all;
    } catch (const std::exception &) {
        if (PyErr_Occurred()) return nullptr;
        UNCOMMON;
    }
}

// rmsnorm(entry, x, weight, eps)
PyObject *rmsnorm(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 4) UNCOMMON;
    const Entry *e = entry_of(a[0], RMSNORM, RMSNORM);
    float eps;
    if (!e || !number(a[3], &eps)) UNCOMMON;
    try {
        const at::Tensor *x = matrix(a[1], e->dtype), *w = plain(a[2], 1);
        if (!x || !w || !x->is_contiguous() || !w->is_contiguous() || w->scalar_type() != e->dtype || w->numel() != x->size(1)) UNCOMMON;
        at::Tensor y = output({x->size(0), x->size(1)}, *x, e->dtype);
        if (!y.defined()) UNCOMMON;
        P px = x->data_ptr(), pw = w->data_ptr(), py = y.data_ptr(), stream = current_stream();
        const int M = (int)x->size(0), H = (int)x->size(1);
        int st;
        Py_BEGIN_ALLOW_THREADS
        st = CALL(tbik_rmsnorm)(px, pw, py, M, H, eps, stream);
        Py_END_ALLOW_THREADS
        return wrapped(std::move(y), st);
    } catch (const std::exception &) {
        if (PyErr_Occurred()) return nullptr;
        UNCOMMON;
    }
}

// combine(entry, partials, residual, weight, eps) -> (hidden, normed)
PyObject *combine(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 5) UNCOMMON;
    const Entry *e = entry_of(a[0], COMBINE, COMBINE);
    float eps;
    if (!e || !number(a[4], &eps)) UNCOMMON;
    try {
        const at::Tensor *p = plain(a[1], 3), *r = matrix(a[2], e->dtype), *w = plain(a[3], 1);
        if (!p || !r || !w || p->scalar_type() != at::kFloat || !p->is_contiguous() || !r->is_contiguous() || w->scalar_type() != e->dtype || !w->is_contiguous() ||
            p->size(0) > INT_MAX || r->size(0) != p->size(1) || r->size(1) != p->size(2) || w->size(0) != p->size(2))
            UNCOMMON;
        at::Tensor h = output({r->size(0), r->size(1)}, *r, e->dtype), y = output({r->size(0), r->size(1)}, *r, e->dtype);
        if (!h.defined() || !y.defined()) UNCOMMON;
        P pp = p->data_ptr(), pr = r->data_ptr(), pw = w->data_ptr(), ph = h.data_ptr(), py = y.data_ptr(), stream = current_stream();
        const int shards = (int)p->size(0), M = (int)r->size(0), H = (int)r->size(1);
        int st;
        Py_BEGIN_ALLOW_THREADS
        st = CALL(tbik_combine_residual_rmsnorm)((const float *)pp, shards, pr, pw, eps, ph, py, M, H, stream);
        Py_END_ALLOW_THREADS
        if (st) return PyLong_FromLong(st);
        PyObject *hidden = THPVariable_Wrap(std::move(h));
        if (!hidden) return nullptr;
        PyObject *normed = THPVariable_Wrap(std::move(y));
        if (!normed) {
            Py_DECREF(hidden);
            return nullptr;
        }
        PyObject *both = PyTuple_Pack(2, hidden, normed);
        Py_DECREF(hidden);
        Py_DECREF(normed);
        return both;
    } catch (const std::exception &) {
        if (PyErr_Occurred()) return nullptr;
        UNCOMMON;
    }
}

// row_reduce(entry, x, op)
PyObject *row_reduce(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 3) UNCOMMON;
    const Entry *e = entry_of(a[0], ROWS, ROWS);
    int op;
    if (!e || !integer(a[2], &op)) UNCOMMON;
    try {
        const at::Tensor *x = plain(a[1], 2);
        if (!x || !x->is_contiguous() || type_code(x->scalar_type()) < 0 || x->size(0) > INT_MAX) UNCOMMON;
        const int M = (int)x->size(0);
        const L V = x->size(1);
        at::Tensor y = op == TBIK_LOGSOFTMAX ? output({M, V}, *x, at::kFloat) : output({M}, *x, at::kFloat);
        if (!y.defined()) UNCOMMON;
        void *stream = current_stream();
        Room ws;
        // (the binding always passes a workspace here, of 256 bytes at least)
        const size_t need = NEED(tbik_row_reduce_workspace_bytes)(M, V, (tbik_rowop)op);
        if (!room_for(need ? need : 1, a[1], *x, stream, &ws)) return nullptr;
        P px = x->data_ptr(), py = y.data_ptr();
        const tbik_dtype t = (tbik_dtype)type_code(x->scalar_type());
        int st;
        Py_BEGIN_ALLOW_THREADS
        st = CALL(tbik_row_reduce)(px, t, py, (tbik_rowop)op, M, V, ws.at, ws.bytes, stream);
        Py_END_ALLOW_THREADS
        return wrapped(std::move(y), st);
    } catch (const std::exception &) {
        if (PyErr_Occurred()) return nullptr;
        UNCOMMON;
    }
}

// attention(entry, Q, K, V, cu_q, cu_k, max_seqlen_q, scale, causal, max_seqlen_k)
PyObject *attention(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 10) UNCOMMON;
    const Entry *e = entry_of(a[0], ATTENTION, ATTENTION);
    int max_q, max_k;
    float scale;
    if (!e || !integer(a[6], &max_q) || !number(a[7], &scale) || !PyBool_Check(a[8]) || !integer(a[9], &max_k)) UNCOMMON;
    try {
        const at::Tensor *t[3];
        for (int i = 0; i < 3; ++i) {
            t[i] = plain(a[1 + i], 3);
            if (!t[i] || t[i]->scalar_type() != e->dtype || t[i]->stride(2) != 1 || t[i]->stride(1) != t[i]->size(2) || t[i]->size(0) > INT_MAX || t[i]->size(1) > INT_MAX) UNCOMMON;
        }
        const at::Tensor &Q = *t[0], &K = *t[1], &V = *t[2];
        const at::Tensor *cq = plain(a[4], 1), *ck = plain(a[5], 1);
        if (!cq || !ck || cq->scalar_type() != at::kInt || ck->scalar_type() != at::kInt || !cq->is_contiguous() || !ck->is_contiguous() || cq->numel() < 1 ||
            cq->numel() != ck->numel() || cq->numel() > INT_MAX || K.size(0) != V.size(0) || K.size(1) != V.size(1) || K.size(2) != V.size(2) || K.size(2) != Q.size(2) ||
            Q.size(2) != 128)
            UNCOMMON;
        const int batch = (int)cq->numel() - 1, Tq = (int)Q.size(0), Tk = (int)K.size(0), Hq = (int)Q.size(1), Hkv = (int)K.size(1);
        at::Tensor O = output({Tq, Hq, 128}, Q, e->dtype);
        if (!O.defined()) UNCOMMON;
        void *stream = current_stream();
        Room ws;
        if (!room_for(NEED(tbik_attention_workspace_bytes)(batch, max_q, max_k < Tk ? max_k : Tk, Hq, Hkv), a[1], Q, stream, &ws)) return nullptr;
        P q = Q.data_ptr(), k = K.data_ptr(), v = V.data_ptr(), o = O.data_ptr(), pq = cq->data_ptr(), pk = ck->data_ptr();
        const L sq = Q.stride(0), sk = K.stride(0), sv = V.stride(0), so = O.stride(0);
        const int causal = a[8] == Py_True;
        int st;
        Py_BEGIN_ALLOW_THREADS
        st = CALL(tbik_attention)(
            q, k, v, o, (const int32_t *)pq, (const int32_t *)pk, batch, max_q, max_k, Tq, Tk, Hq, Hkv, 128, sq, sk, sv, so, scale, causal, ws.at, ws.bytes, stream);
        Py_END_ALLOW_THREADS
        return wrapped(std::move(O), st);
    } catch (const std::exception &) {
        if (PyErr_Occurred()) return nullptr;
        UNCOMMON;
    }
}

// ---- an MLP that is a mixture of experts, 4-bit weights, norms around a block ----
bool here(const at::Tensor &t) { return t.device().index() == c10::hip::current_device(); }
// A contiguous int32 vector or matrix.
const at::Tensor *indexes(PyObject *o, int dim) {
    const at::Tensor *t = plain(o, dim);
    return t && t->scalar_type() == at::kInt && t->is_contiguous() ? t : nullptr;
}
bool sixteen_bits(const at::Tensor &t) { return t.scalar_type() == at::kBFloat16 || t.scalar_type() == at::kHalf; }
tbik_dtype code_of(const at::Tensor &t) { return (tbik_dtype)type_code(t.scalar_type()); }
template <int N>
PyObject *tuple_of(at::Tensor (&t)[N], int status) {
    if (status) return PyLong_FromLong(status);
    PyObject *all = PyTuple_New(N);
    if (!all) return nullptr;
    for (int i = 0; i < N; ++i) {
        PyObject *o = t[i].defined() ? THPVariable_Wrap(std::move(t[i])) : Py_NewRef(Py_None);
        if (!o) {
            Py_DECREF(all);
            return nullptr;
        }
        PyTuple_SET_ITEM(all, i, o);
    }
    return all;
}

// route(entry, logits, k, renormalize) -> (experts, weights, offsets, rows, slots)
PyObject *route(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 4) UNCOMMON;
    const Entry *e = entry_of(a[0], ROUTE, ROUTE);
    int k;
    if (!e || !integer(a[2], &k) || !PyBool_Check(a[3])) UNCOMMON;
    try {
        const at::Tensor *l = plain(a[1], 2);
        if (!l || l->stride(1) != 1 || type_code(l->scalar_type()) < 0 || l->size(0) > (1 << 26) || l->size(1) > 512 || k < 1 || k > l->size(1) || l->size(0) * k > INT_MAX || !here(*l)) UNCOMMON;
        const int T = (int)l->size(0), E = (int)l->size(1);
        void *stream = current_stream();
        Room ws;
        const size_t need = NEED(tbik_route_topk_workspace_bytes)(T, E);
        if (need && c10::hip::currentStreamCaptureStatusMayInitCtx() != c10::hip::CaptureStatus::None) UNCOMMON;      // a workspace of the graph's own
        if (!room_for(need, a[1], *l, stream, &ws)) return nullptr;
        at::Tensor out[5] = {output({T, k}, *l, at::kInt), output({T, k}, *l, at::kFloat), output({E + 1}, *l, at::kInt), output({(L)T * k}, *l, at::kInt), output({T, k}, *l, at::kInt)};
        for (const at::Tensor &t : out)
            if (!t.defined()) UNCOMMON;
        P at[5], logits = l->data_ptr();
        for (int i = 0; i < 5; ++i) at[i] = out[i].data_ptr();
        const L ldl = l->stride(0);
        const tbik_dtype type = code_of(*l);
        const int renormalize = a[3] == Py_True;
        int st;
        Py_BEGIN_ALLOW_THREADS
        st = CALL(tbik_route_topk)(logits, ldl, type, T, E, k, renormalize, (int32_t *)at[0], (float *)at[1], (int32_t *)at[2], (int32_t *)at[3], (int32_t *)at[4], ws.at, ws.bytes, stream);
        Py_END_ALLOW_THREADS
        return tuple_of(out, st);
    } catch (const std::exception &) {
        if (PyErr_Occurred()) return nullptr;
        UNCOMMON;
    }
}

// grouped(entry, X, W, offsets, rows or None, leaf, k_first, out dtype or None, shards)
PyObject *grouped(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 9) UNCOMMON;
    const Entry *e = entry_of(a[0], GROUPED, GROUPED_PARTIALS);
    int leaf, k_first, shards;
    if (!e || !integer(a[5], &leaf) || !integer(a[6], &k_first) || !integer(a[8], &shards)) UNCOMMON;
    const int kind = e->kind;
    try {
        const at::Tensor *X = plain(a[1], 2), *W = plain(a[2], 3), *offsets = indexes(a[3], 1), *rows = nullptr;
        if (a[4] != Py_None && !(rows = indexes(a[4], 1))) UNCOMMON;
        if (!X || !W || !offsets || !sixteen_bits(*X) || W->scalar_type() != X->scalar_type() || X->stride(1) != 1 || W->stride(2) != 1 || X->size(0) > INT_MAX || X->size(1) > INT_MAX ||
            W->size(0) > 512 || W->size(1) != X->size(1) || W->size(2) > INT_MAX || offsets->size(0) != W->size(0) + 1 || (rows && rows->size(0) > INT_MAX) || !here(*X) || elsewhere(W, *X) ||
            elsewhere(offsets, *X) || elsewhere(rows, *X))
            UNCOMMON;
        at::ScalarType type = X->scalar_type();
        if (a[7] != Py_None) {
            if (!THPDtype_Check(a[7])) UNCOMMON;
            type = ((THPDtype *)a[7])->scalar_type;
            if (type_code(type) < 0) UNCOMMON;
        }
        const int tokens = (int)X->size(0), K = (int)X->size(1), groups = (int)W->size(0), N = (int)W->size(2), R = rows ? (int)rows->size(0) : tokens;
        if ((kind == GROUPED_SWIGLU && N % 2) || shards < 1) UNCOMMON;
        at::Tensor y = kind == GROUPED_PARTIALS ? output({shards, R, N}, *X, at::kFloat) : output({R, kind == GROUPED_SWIGLU ? N / 2 : N}, *X, type);
        if (!y.defined()) UNCOMMON;
        P px = X->data_ptr(), pw = W->data_ptr(), po = offsets->data_ptr(), pr = rows ? rows->data_ptr() : nullptr, py = y.data_ptr(), stream = current_stream();
        const L ldx = X->stride(0), ldw = W->stride(1), stride = W->stride(0), ldy = kind == GROUPED_PARTIALS ? 0 : y.stride(0);
        const tbik_dtype xt = code_of(*X), yt = code_of(y);
        int st;
        Py_BEGIN_ALLOW_THREADS
        if (kind == GROUPED)
            st = CALL(tbik_gemm_grouped)(px, ldx, tokens, (const int32_t *)pr, pw, ldw, stride, groups, (const int32_t *)po, py, ldy, yt, xt, R, N, K, leaf, k_first, stream);
        else if (kind == GROUPED_SWIGLU)
            st = CALL(tbik_gemm_grouped_swiglu)(px, ldx, tokens, (const int32_t *)pr, pw, ldw, stride, groups, (const int32_t *)po, py, ldy, xt, R, N / 2, K, leaf, k_first, stream);
        else
            st = CALL(tbik_gemm_grouped_shard_partials)(px, ldx, tokens, (const int32_t *)pr, pw, ldw, stride, groups, (const int32_t *)po, (float *)py, xt, R, N, K, leaf, k_first, shards, stream);
        Py_END_ALLOW_THREADS
        return wrapped(std::move(y), st);
    } catch (const std::exception &) {
        if (PyErr_Occurred()) return nullptr;
        UNCOMMON;
    }
}

// experts_sum(entry, Y, slots, weights, residual or None, out dtype or None)
PyObject *experts_sum(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 6) UNCOMMON;
    const Entry *e = entry_of(a[0], EXPERTS_SUM, EXPERTS_SUM);
    if (!e) UNCOMMON;
    try {
        const at::Tensor *y = plain(a[1], 3), *slots = indexes(a[2], 2), *w = plain(a[3], 2), *r = nullptr;
        const bool sums = y != nullptr;
        if (!sums) y = plain(a[1], 2);
        if (a[4] != Py_None && !(r = plain(a[4], 2))) UNCOMMON;
        if (!y || !slots || !w || type_code(y->scalar_type()) < 0 || (sums && y->scalar_type() != at::kFloat) || w->scalar_type() != at::kFloat || !w->is_contiguous() || w->sizes() != slots->sizes()) UNCOMMON;
        if (y->scalar_type() == at::kFloat ? !y->is_contiguous() : y->stride(1) != 1) UNCOMMON;
        at::ScalarType type = r ? r->scalar_type() : y->scalar_type();
        if (a[5] != Py_None) {
            if (!THPDtype_Check(a[5])) UNCOMMON;
            type = ((THPDtype *)a[5])->scalar_type;
        }
        const int d = sums ? 1 : 0;
        if (type_code(type) < 0 || y->size(0) > INT_MAX || y->size(d) > INT_MAX || y->size(d + 1) > INT_MAX || slots->size(0) > INT_MAX || slots->size(1) > INT_MAX || !here(*y) ||
            elsewhere(slots, *y) || elsewhere(w, *y) || elsewhere(r, *y))
            UNCOMMON;
        const int shards = sums ? (int)y->size(0) : 1, R = (int)y->size(d), H = (int)y->size(d + 1), T = (int)slots->size(0), k = (int)slots->size(1);
        if (r && (r->scalar_type() != type || r->size(0) != T || r->size(1) != H || r->stride(1) != 1)) UNCOMMON;
        at::Tensor out = output({T, H}, *y, type);
        if (!out.defined()) UNCOMMON;
        P py = y->data_ptr(), ps = slots->data_ptr(), pw = w->data_ptr(), pr = r ? r->data_ptr() : nullptr, po = out.data_ptr(), stream = current_stream();
        const L ldy = y->stride(d), ldr = r ? r->stride(0) : 0, ldo = out.stride(0);
        const tbik_dtype yt = code_of(*y), ot = code_of(out);
        int st;
        Py_BEGIN_ALLOW_THREADS
        st = CALL(tbik_combine_experts)(py, ldy, yt, shards, R, (const int32_t *)ps, (const float *)pw, pr, ldr, po, ldo, ot, T, H, k, stream);
        Py_END_ALLOW_THREADS
        return wrapped(std::move(out), st);
    } catch (const std::exception &) {
        if (PyErr_Occurred()) return nullptr;
        UNCOMMON;
    }
}

// w4(entry, X, Wq, scales, zeros or None, leaf, k_first, out dtype or None, shards)
PyObject *w4(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 9) UNCOMMON;
    const Entry *e = entry_of(a[0], W4, W4_PARTIALS);
    int leaf, k_first, shards;
    if (!e || !integer(a[5], &leaf) || !integer(a[6], &k_first) || !integer(a[8], &shards) || shards < 1) UNCOMMON;
    try {
        const at::Tensor *X = plain(a[1], 2), *W = matrix(a[2], at::kByte), *z = nullptr;
        if (!X || !W || !sixteen_bits(*X) || X->stride(1) != 1 || X->size(0) > INT_MAX || X->size(1) > INT_MAX) UNCOMMON;
        const at::Tensor *sc = matrix(a[3], X->scalar_type());
        if (!sc || (a[4] != Py_None && !(z = matrix(a[4], at::kByte)))) UNCOMMON;
        at::ScalarType type = X->scalar_type();
        if (a[7] != Py_None) {
            if (!THPDtype_Check(a[7])) UNCOMMON;
            type = ((THPDtype *)a[7])->scalar_type;
            if (type_code(type) < 0) UNCOMMON;
        }
        const int M = (int)X->size(0), K = (int)X->size(1), N = (int)W->size(0), groups = (int)sc->size(1);
        if (K % 2 || W->size(1) != K / 2 || sc->size(0) != N || groups < 1 || K % groups || (z && z->sizes() != sc->sizes()) || !here(*X) || elsewhere(W, *X) || elsewhere(sc, *X) || elsewhere(z, *X)) UNCOMMON;
        const bool partials = e->kind == W4_PARTIALS;
        void *stream = current_stream();
        Room ws;
        const size_t need = partials ? 0 : NEED(tbik_gemm_w4_workspace_bytes)(M, N, K, leaf, k_first);
        if (need && c10::hip::currentStreamCaptureStatusMayInitCtx() != c10::hip::CaptureStatus::None) UNCOMMON;      // a workspace of the graph's own
        if (!room_for(need, a[1], *X, stream, &ws)) return nullptr;
        at::Tensor y = partials ? output({shards, M, N}, *X, at::kFloat) : output({M, N}, *X, type);
        if (!y.defined()) UNCOMMON;
        P px = X->data_ptr(), pw = W->data_ptr(), ps = sc->data_ptr(), pz = z ? z->data_ptr() : nullptr, py = y.data_ptr();
        const L ldx = X->stride(0), ldw = W->stride(0), lds = sc->stride(0), ldz = z ? z->stride(0) : 0, ldy = partials ? 0 : y.stride(0);
        const tbik_dtype xt = code_of(*X), yt = code_of(y);
        int st;
        Py_BEGIN_ALLOW_THREADS
        if (partials) st = CALL(tbik_gemm_shard_partials_w4)(px, ldx, pw, ldw, ps, lds, pz, ldz, K / groups, (float *)py, xt, M, N, K, leaf, k_first, shards, stream);
        else st = CALL(tbik_gemm_w4)(px, ldx, pw, ldw, ps, lds, pz, ldz, K / groups, py, ldy, yt, xt, M, N, K, leaf, k_first, ws.at, ws.bytes, stream);
        Py_END_ALLOW_THREADS
        return wrapped(std::move(y), st);
    } catch (const std::exception &) {
        if (PyErr_Occurred()) return nullptr;
        UNCOMMON;
    }
}

// join(entry, y, residual, post_weight or None, next_weight or None, eps, residual_scale, gate or None) -> (hidden, normed or None)
PyObject *join(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 8) UNCOMMON;
    const Entry *e = entry_of(a[0], JOIN, JOIN);
    float eps, scale;
    if (!e || !number(a[5], &eps) || !number(a[6], &scale)) UNCOMMON;
    try {
        const at::Tensor *r = plain(a[2], 2);
        if (!r || !sixteen_bits(*r) || r->stride(1) != 1 || r->size(0) > INT_MAX || r->size(1) > INT_MAX) UNCOMMON;
        const at::ScalarType type = r->scalar_type();
        const int M = (int)r->size(0), H = (int)r->size(1);
        const at::Tensor *y = plain(a[1], 3), *w[2] = {nullptr, nullptr}, *gate = nullptr;
        const bool sums = y != nullptr;
        if (sums ? y->scalar_type() != at::kFloat || !y->is_contiguous() || y->size(0) > INT_MAX || y->size(1) != M || y->size(2) != H
                 : !(y = matrix(a[1], type)) || y->size(0) != M || y->size(1) != H)
            UNCOMMON;
        for (int i = 0; i < 2; ++i) {
            if (a[3 + i] == Py_None) continue;
            w[i] = plain(a[3 + i], 1);
            if (!w[i] || w[i]->scalar_type() != type || w[i]->size(0) != H || !w[i]->is_contiguous()) UNCOMMON;
        }
        L gate_row = 0;
        int gate_column = 0;
        if (a[7] != Py_None) {
            if ((gate = plain(a[7], 1))) {
                if (gate->size(0) != H) UNCOMMON;
            } else {
                gate = plain(a[7], 2);
                if (!gate || (gate->size(0) != 1 && gate->size(0) != M) || (gate->size(1) != 1 && gate->size(1) != H)) UNCOMMON;
                if (gate->size(0) == M && M > 1) gate_row = gate->stride(0);
            }
            const int last = (int)gate->dim() - 1;
            gate_column = gate->size(last) == H && H > 1;
            if (gate->scalar_type() != type || (gate_column && gate->stride(last) != 1)) UNCOMMON;
        }
        if (!here(*r) || elsewhere(y, *r) || elsewhere(w[0], *r) || elsewhere(w[1], *r) || elsewhere(gate, *r)) UNCOMMON;
        at::Tensor out[2] = {output({M, H}, *r, type), at::Tensor()};
        if (w[1]) out[1] = output({M, H}, *r, type);
        if (!out[0].defined() || (w[1] && !out[1].defined())) UNCOMMON;
        P py = y->data_ptr(), pr = r->data_ptr(), pw[2] = {w[0] ? w[0]->data_ptr() : nullptr, w[1] ? w[1]->data_ptr() : nullptr}, pg = gate ? gate->data_ptr() : nullptr,
          ph = out[0].data_ptr(), pn = w[1] ? out[1].data_ptr() : nullptr, stream = current_stream();
        const L ldy = sums ? 0 : y->stride(0), ldr = r->stride(0), ldh = out[0].stride(0);
        const int shards = sums ? (int)y->size(0) : 1;
        const tbik_dtype t = code_of(*r);
        int st;
        Py_BEGIN_ALLOW_THREADS
        st = CALL(tbik_rmsnorm_residual_rmsnorm)(sums ? nullptr : py, ldy, sums ? (const float *)py : nullptr, shards, pr, ldr, scale, pw[0], pg, gate_row, gate_column, pw[1], eps, ph, ldh, pn,
                                                 pn ? ldh : 0, t, M, H, stream);
        Py_END_ALLOW_THREADS
        return tuple_of(out, st);
    } catch (const std::exception &) {
        if (PyErr_Occurred()) return nullptr;
        UNCOMMON;
    }
}

// register(entry, kind, address, address of the workspace query or 0, operand dtype)
PyObject *register_entry(PyObject *, PyObject *args) {
    int i, kind;
    unsigned long long call, need;
    PyObject *dtype;
    if (!PyArg_ParseTuple(args, "iiKKO", &i, &kind, &call, &need, &dtype)) return nullptr;
    if (i < 0 || i >= MAX_ENTRIES || kind < 0 || kind >= KINDS || !call || !THPDtype_Check(dtype)) {
        PyErr_SetString(PyExc_ValueError, "entry");
        return nullptr;
    }
    entries[i].kind = kind;
    entries[i].call = (void *)(uintptr_t)call;
    entries[i].need = (void *)(uintptr_t)need;
    entries[i].dtype = ((THPDtype *)dtype)->scalar_type;
    Py_RETURN_NONE;
}

// use(dict of workspaces, function that makes one)
PyObject *use(PyObject *, PyObject *args) {
    PyObject *d, *f;
    if (!PyArg_ParseTuple(args, "O!O", &PyDict_Type, &d, &f)) return nullptr;
    Py_INCREF(d);
    Py_INCREF(f);
    Py_XDECREF(workspaces);
    Py_XDECREF(make_workspace);
    workspaces = d;
    make_workspace = f;
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"product", (PyCFunction)(void (*)(void))product, METH_FASTCALL, nullptr},
    {"rmsnorm", (PyCFunction)(void (*)(void))rmsnorm, METH_FASTCALL, nullptr},
    {"combine", (PyCFunction)(void (*)(void))combine, METH_FASTCALL, nullptr},
    {"row_reduce", (PyCFunction)(void (*)(void))row_reduce, METH_FASTCALL, nullptr},
    {"attention", (PyCFunction)(void (*)(void))attention, METH_FASTCALL, nullptr},
    {"epilogue", (PyCFunction)(void (*)(void))epilogue, METH_FASTCALL, nullptr},
    {"eight_bits", (PyCFunction)(void (*)(void))eight_bits, METH_FASTCALL, nullptr},
    {"route", (PyCFunction)(void (*)(void))route, METH_FASTCALL, nullptr},
    {"grouped", (PyCFunction)(void (*)(void))grouped, METH_FASTCALL, nullptr},
    {"experts_sum", (PyCFunction)(void (*)(void))experts_sum, METH_FASTCALL, nullptr},
    {"w4", (PyCFunction)(void (*)(void))w4, METH_FASTCALL, nullptr},
    {"join", (PyCFunction)(void (*)(void))join, METH_FASTCALL, nullptr},
    {"register", register_entry, METH_VARARGS, nullptr},
    {"use", use, METH_VARARGS, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
