// The operators' calls: a function's arguments, by position or by name, become the fields of the C ABI's structure.
//
// A buffer is a torch tensor, an object with data_ptr(), an address, or None where it is optional.  What a tensor says of
// itself is held against the call: it has to be on the current device and of the element type that the call names, its elements
// where the call takes them to be, and its storage, from its first element on, as long as the call's sizes and strides reach.
// Measured with the library's own checks and without the launch: a norm with eight buffers 0.46 us (0.42 without a look at types and
// strides), a lookup with three 0.33.
#include "nuna_py.h"

#include <c10/cuda/CUDAFunctions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstddef>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <exception>

#include "../nuna_spans.h"

namespace nuna_py {

namespace {

enum Kind { kBuffer, kSize, kLong, kInt, kFloat };
// What a buffer holds: bytes of any kind, elements of the dtype in an argument, ids of as many bytes as an argument says, or these.
enum Content { kBytes, kElements, kIds, kInt32, kFloat32 };
struct Field {
    const char* text;
    Kind kind;
    size_t at;                         // offset in the structure
    int span;                          // a buffer's place among spans_of()
    bool required;
    PyObject* name;
    Content content;
    size_t type_at, stride_at;         // offsets of the argument that says the type, and of the rows' stride (0: not rows)
};
constexpr int kMaxFields = 28;
// Behind an operator's own arguments.
PyObject* g_tail[3] = {};
const char* const kTail[3] = {"flags", "stream", "check"};

// A buffer's address, how many bytes it has from there on (all, if it does not say), and the tensor that it is, if its address is
// not null.  `device`: the current one, asked for with the first tensor (-1 before).
bool buffer_of(PyObject* x, void** at, size_t* bytes, const c10::TensorImpl** tensor, int* device, bool* elsewhere)
{
    *bytes = SIZE_MAX;
    if (x == Py_None) {
        *at = nullptr;
        return true;
    }
    if (!THPVariable_CheckExact(x)) return address_of(x, false, at);
    try {
        const at::Tensor& t = THPVariable_Unpack(x);
        *at = t.mutable_data_ptr();
        if (*at) {
            if (*device < 0 && t.is_cuda()) *device = c10::cuda::current_device();
            *elsewhere = *elsewhere || !t.is_cuda() || t.device().index() != *device;
        }
        const c10::TensorImpl* impl = t.unsafeGetTensorImpl();
        if (*at) *tensor = impl;
        const size_t all = impl->unsafe_storage().unsafeGetStorageImpl()->nbytes(), before = (size_t)impl->storage_offset() * impl->itemsize();
        *bytes = all > before ? all - before : 0;
        return true;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return false;
    }
}

// Unsigned integers are raw memory, of any type.
bool is_raw(c10::ScalarType is)
{
    using c10::ScalarType;
    return is == ScalarType::Byte || is == ScalarType::UInt16 || is == ScalarType::UInt32 || is == ScalarType::UInt64;
}

// Whether a tensor's elements are of the type that the call takes them for; `dtype`: that of the rows.  Types that the library does
// not take, alone or beside one another, are its own to refuse.
bool right_type(const c10::TensorImpl* t, const Field& f, const char* args, int dtype)
{
    using c10::ScalarType;
    const ScalarType is = c10::typeMetaToScalarType(t->dtype());
    ScalarType want = f.content == kInt32 ? ScalarType::Int : ScalarType::Float;
    int said = 0;
    if (f.type_at) memcpy(&said, args + f.type_at, sizeof said);
    if (f.content == kElements) {
        if (!nuna::is_dtype(said) || (said != dtype && said != NUNA_F32)) return true;
        want = said == NUNA_BF16 ? ScalarType::BFloat16 : said == NUNA_F16 ? ScalarType::Half : ScalarType::Float;
    } else if (f.content == kIds) {
        if (said != 4 && said != 8) return true;
        want = said == 4 ? ScalarType::Int : ScalarType::Long;
    }
    return is == want || is_raw(is);
}

// Whether a tensor's elements are where the call takes them to be: one after the other, or in rows of consecutive elements at equal
// distances, of which the call's distance is a multiple (one row, as the call's `bytes` tell, has none).  A tensor that is contiguous
// may stand for memory of any shape.
bool right_place(const c10::TensorImpl* t, const Field& f, const char* args, size_t hidden, size_t bytes)
{
    if (t->is_contiguous() || is_raw(c10::typeMetaToScalarType(t->dtype()))) return true;
    if (!f.stride_at) return false;
    size_t stride;
    memcpy(&stride, args + f.stride_at, sizeof stride);
    if (stride == 0) stride = hidden;
    const auto sizes = t->sizes(), strides = t->strides();
    int64_t d = (int64_t)sizes.size() - 1, next = 0;                 // next: the distance that the next outer dimension has to have
    if (hidden != 1) {
        if (sizes[d] > 1 && strides[d] != 1) return false;
        --d;
    }
    if (bytes <= hidden * t->itemsize()) return true;
    for (; d >= 0; --d) {
        if (sizes[d] == 1) continue;
        if (next ? strides[d] != next : (strides[d] <= 0 || stride % (size_t)strides[d] != 0)) return false;
        next = strides[d] * sizes[d];
    }
    return true;
}

bool put(PyObject* x, const Field& f, char* to)
{
    unsigned long long v;
    switch (f.kind) {
        case kFloat: {
            const double d = PyFloat_AsDouble(x);
            if (d == -1.0 && PyErr_Occurred()) return false;
            const float g = (float)d;
            memcpy(to, &g, sizeof g);
            return true;
        }
        case kSize: {
            if (!to_u64(x, &v)) return false;
            const size_t n = (size_t)v;
            memcpy(to, &n, sizeof n);
            return true;
        }
        case kLong: {
            if (!to_u64(x, &v)) return false;
            const long long n = (long long)v;
            memcpy(to, &n, sizeof n);
            return true;
        }
        default: {
            if (!to_u64(x, &v)) return false;
            const int n = (int)v;
            memcpy(to, &n, sizeof n);
            return true;
        }
    }
}

template <typename Args>
struct Op {
    const char* name;
    int (*call)(const Args*, unsigned, void*);
    size_t workspace_bytes;            // offset of the workspace's size, which its tensor tells; 0: none
    int workspace_span;
    size_t hidden_at, dtype_at;        // offsets of the rows' length and type; 0: none
    int n;
    Field field[kMaxFields];
};

template <typename Args>
PyObject* run(Op<Args>& op, Args a, PyObject* const* args, Py_ssize_t npos, PyObject* kwnames)
{
    PyObject* given[kMaxFields + 3] = {};
    const int total = op.n + 3;
    if (npos > total) return PyErr_Format(PyExc_TypeError, "%s() takes at most %d arguments (%zd given)", op.name, total, npos);
    for (Py_ssize_t i = 0; i < npos; ++i) given[i] = args[i];
    const auto name_of = [&](int i) { return i < op.n ? op.field[i].name : g_tail[i - op.n]; };
    int guess = (int)npos;                                           // names usually come in the arguments' own order
    for (Py_ssize_t k = 0, nkw = kwnames ? PyTuple_GET_SIZE(kwnames) : 0; k < nkw; ++k) {
        PyObject* key = PyTuple_GET_ITEM(kwnames, k);
        int at = total;
        for (int step = 0; step < total; ++step) {
            const int i = (guess + step) % total;
            if (key == name_of(i)) {
                at = i;
                break;
            }
        }
        if (at == total)
            for (at = 0; at < total && PyUnicode_Compare(key, name_of(at)) != 0;) ++at;
        if (at == total || given[at])
            return PyErr_Format(PyExc_TypeError, at == total ? "%s() got an unexpected keyword argument '%U'"
                                                             : "%s() got multiple values for argument '%U'", op.name, key);
        given[at] = args[npos + k];
        guess = at + 1;
    }
    size_t has[nuna::kMaxSpans];
    for (size_t& h : has) h = SIZE_MAX;
    struct Held {
        const c10::TensorImpl* tensor;
        const Field* field;
    } held[nuna::kMaxSpans];
    int tensors = 0;
    bool elsewhere = false, sized = false;
    int device = -1;
    char* base = reinterpret_cast<char*>(&a);
    for (int i = 0; i < op.n; ++i) {
        const Field& f = op.field[i];
        // a workspace's size is its tensor's where none is given, or None
        if (!given[i] || (given[i] == Py_None && op.workspace_bytes && f.at == op.workspace_bytes && f.kind == kSize)) {
            if (f.required) return PyErr_Format(PyExc_TypeError, "%s() missing required argument: '%s'", op.name, f.text);
            continue;
        }
        if (f.kind == kBuffer) {
            void* at = nullptr;
            const c10::TensorImpl* t = nullptr;
            if (!buffer_of(given[i], &at, &has[f.span], &t, &device, &elsewhere)) return nullptr;
            memcpy(base + f.at, &at, sizeof at);
            if (t && f.content != kBytes) held[tensors++] = {t, &f};
        } else {
            if (!put(given[i], f, base + f.at)) return nullptr;
            sized = sized || (op.workspace_bytes && f.at == op.workspace_bytes);
        }
    }
    if (op.workspace_bytes && !sized && has[op.workspace_span] != SIZE_MAX) memcpy(base + op.workspace_bytes, &has[op.workspace_span], sizeof(size_t));
    unsigned long long flags = 0;
    void* stream;
    if ((given[op.n] && !to_u64(given[op.n], &flags)) || !to_stream(given[op.n + 1] ? given[op.n + 1] : Py_None, &stream)) return nullptr;
    PyObject* check = given[op.n + 2] ? given[op.n + 2] : Py_True;
    const char *wrong = elsewhere ? "a tensor that is not on the current device" : nullptr, *which = "";
    const nuna::Spans s = nuna::spans_of(a);
    if (s.status == NUNA_OK)
        for (int i = 0; i < s.n && !wrong; ++i)
            if (s.v[i].at && s.v[i].bytes > has[i]) wrong = "a tensor shorter than the call's sizes";
    try {
        size_t hidden = 0;
        int dtype = 0;
        if (op.hidden_at) memcpy(&hidden, base + op.hidden_at, sizeof hidden);
        if (op.dtype_at) memcpy(&dtype, base + op.dtype_at, sizeof dtype);
        for (int i = 0; i < tensors && !wrong; ++i) {
            const Field& f = *held[i].field;
            if (!right_type(held[i].tensor, f, base, dtype)) wrong = " is a tensor of another type than the call says";
            else if (!right_place(held[i].tensor, f, base, hidden, s.v[f.span].bytes)) wrong = " is a tensor whose elements are not where the call takes them to be";
            which = f.text;
        }
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
    if (wrong) {
        char what[160];
        snprintf(what, sizeof what, "%s: %s%s", op.name, *wrong == ' ' ? which : "", wrong);
        return finish(NUNA_ERR_INVALID_ARG, what, check);
    }
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = op.call(&a, (unsigned)flags, stream);
    Py_END_ALLOW_THREADS
    return finish(st, op.name, check);
}

// Rows of elements, other elements and ids (`type`: the argument that says which), int32, binary32, bytes, values.
#define ROWS(T, f, span, required, type) {#f, kBuffer, offsetof(T, f), span, required, nullptr, kElements, offsetof(T, type), offsetof(T, f##_stride)}
#define ELEMS(T, f, span, required, type) {#f, kBuffer, offsetof(T, f), span, required, nullptr, kElements, offsetof(T, type), 0}
#define IDS(T, f, span, required) {#f, kBuffer, offsetof(T, f), span, required, nullptr, kIds, offsetof(T, id_bytes), 0}
#define I32(T, f, span, required) {#f, kBuffer, offsetof(T, f), span, required, nullptr, kInt32, 0, 0}
#define F32(T, f, span, required) {#f, kBuffer, offsetof(T, f), span, required, nullptr, kFloat32, 0, 0}
#define BYTES(T, f, span, required) {#f, kBuffer, offsetof(T, f), span, required, nullptr, kBytes, 0, 0}
#define VAL(T, f, kind, required) {#f, kind, offsetof(T, f), -1, required, nullptr, kBytes, 0, 0}

using LF = nuna_layernorm_t;
Op<LF> g_norm = {"nuna_layernorm_forward", nullptr, 0, -1, offsetof(LF, hidden), offsetof(LF, dtype), 17, {
    ROWS(LF, x, 0, true, dtype), ROWS(LF, y, 5, true, dtype), VAL(LF, rows, kSize, true), VAL(LF, hidden, kSize, true), ELEMS(LF, weight, 2, false, param_dtype),
    ELEMS(LF, bias, 3, false, param_dtype), ROWS(LF, residual, 1, false, dtype), ROWS(LF, summed, 4, false, dtype), F32(LF, mean, 6, false), F32(LF, rstd, 7, false),
    VAL(LF, eps, kFloat, false), VAL(LF, dtype, kInt, false), VAL(LF, param_dtype, kInt, false), VAL(LF, x_stride, kSize, false),
    VAL(LF, residual_stride, kSize, false), VAL(LF, summed_stride, kSize, false), VAL(LF, y_stride, kSize, false)}};

using LB = nuna_layernorm_grad_t;
Op<LB> g_norm_grad = {"nuna_layernorm_backward", nullptr, offsetof(LB, workspace_bytes), 9, offsetof(LB, hidden), offsetof(LB, dtype), 19, {
    ROWS(LB, dy, 0, true, dtype), ROWS(LB, x, 1, true, dtype), F32(LB, mean, 2, true), F32(LB, rstd, 3, true), ROWS(LB, dx, 6, true, dtype),
    VAL(LB, rows, kSize, true), VAL(LB, hidden, kSize, true), ELEMS(LB, weight, 4, false, param_dtype), ROWS(LB, dsummed, 5, false, dtype),
    ELEMS(LB, dweight, 7, false, param_dtype), ELEMS(LB, dbias, 8, false, param_dtype), BYTES(LB, workspace, 9, false), VAL(LB, dtype, kInt, false),
    VAL(LB, param_dtype, kInt, false), VAL(LB, dy_stride, kSize, false), VAL(LB, x_stride, kSize, false),
    VAL(LB, dsummed_stride, kSize, false), VAL(LB, dx_stride, kSize, false), VAL(LB, workspace_bytes, kSize, false)}};

using EF = nuna_embedding_t;
Op<EF> g_lookup = {"nuna_embedding_forward", nullptr, 0, -1, offsetof(EF, hidden), offsetof(EF, dtype), 12, {
    IDS(EF, ids, 0, true), ROWS(EF, table, 1, true, dtype), ROWS(EF, out, 2, true, dtype), VAL(EF, tokens, kSize, true), VAL(EF, hidden, kSize, true),
    VAL(EF, vocab_rows, kSize, true), VAL(EF, vocab_start, kLong, false), VAL(EF, scale, kFloat, false), VAL(EF, dtype, kInt, false),
    VAL(EF, id_bytes, kInt, false), VAL(EF, table_stride, kSize, false), VAL(EF, out_stride, kSize, false)}};

using EB = nuna_embedding_grad_t;
Op<EB> g_lookup_grad = {"nuna_embedding_backward", nullptr, offsetof(EB, workspace_bytes), 3, offsetof(EB, hidden), offsetof(EB, dtype), 15, {
    IDS(EB, ids, 0, true), ROWS(EB, dout, 1, true, dtype), ROWS(EB, dtable, 2, true, grad_dtype), VAL(EB, tokens, kSize, true), VAL(EB, hidden, kSize, true),
    VAL(EB, vocab_rows, kSize, true), BYTES(EB, workspace, 3, false), VAL(EB, vocab_start, kLong, false), VAL(EB, scale, kFloat, false),
    VAL(EB, dtype, kInt, false), VAL(EB, grad_dtype, kInt, false), VAL(EB, id_bytes, kInt, false), VAL(EB, dout_stride, kSize, false),
    VAL(EB, dtable_stride, kSize, false), VAL(EB, workspace_bytes, kSize, false)}};

using XS = nuna_expert_sort_t;
Op<XS> g_sort = {"nuna_expert_sort", nullptr, 0, -1, 0, 0, 11, {
    IDS(XS, experts, 0, true), I32(XS, row_of_pair, 1, true), I32(XS, pair_of_row, 2, true), I32(XS, offsets, 3, true),
    VAL(XS, tokens, kSize, true), VAL(XS, topk, kSize, true), VAL(XS, num_experts, kSize, true), I32(XS, counts, 4, false),
    VAL(XS, first_expert, kLong, false), VAL(XS, capacity, kSize, false), VAL(XS, id_bytes, kInt, false)}};

using XD = nuna_expert_dispatch_t;
Op<XD> g_dispatch = {"nuna_expert_dispatch", nullptr, 0, -1, offsetof(XD, hidden), offsetof(XD, dtype), 11, {
    ROWS(XD, x, 0, true, dtype), I32(XD, row_of_pair, 1, true), ROWS(XD, out, 3, true, dtype), VAL(XD, tokens, kSize, true), VAL(XD, topk, kSize, true),
    VAL(XD, rows, kSize, true), VAL(XD, hidden, kSize, true), I32(XD, pair_of_row, 2, false), VAL(XD, dtype, kInt, false),
    VAL(XD, x_stride, kSize, false), VAL(XD, out_stride, kSize, false)}};

using XC = nuna_expert_combine_t;
Op<XC> g_combine = {"nuna_expert_combine", nullptr, 0, -1, offsetof(XC, hidden), offsetof(XC, dtype), 11, {
    ROWS(XC, src, 0, true, dtype), I32(XC, row_of_pair, 1, true), ROWS(XC, y, 3, true, dtype), VAL(XC, tokens, kSize, true), VAL(XC, topk, kSize, true),
    VAL(XC, rows, kSize, true), VAL(XC, hidden, kSize, true), F32(XC, weights, 2, false), VAL(XC, dtype, kInt, false),
    VAL(XC, src_stride, kSize, false), VAL(XC, y_stride, kSize, false)}};

using XB = nuna_expert_combine_grad_t;
Op<XB> g_combine_grad = {"nuna_expert_combine_backward", nullptr, 0, -1, offsetof(XB, hidden), offsetof(XB, dtype), 15, {
    ROWS(XB, dy, 0, true, dtype), ROWS(XB, src, 1, true, dtype), F32(XB, weights, 2, true), I32(XB, row_of_pair, 3, true), ROWS(XB, dsrc, 5, true, dtype),
    F32(XB, dweights, 6, true), VAL(XB, tokens, kSize, true), VAL(XB, topk, kSize, true), VAL(XB, rows, kSize, true),
    VAL(XB, hidden, kSize, true), I32(XB, pair_of_row, 4, false), VAL(XB, dtype, kInt, false), VAL(XB, dy_stride, kSize, false),
    VAL(XB, src_stride, kSize, false), VAL(XB, dsrc_stride, kSize, false)}};

// The values of arguments that a call leaves out, where they are not zero.
LF defaults(const Op<LF>&) { LF a = {}; a.eps = 1e-5f; return a; }
EF defaults(const Op<EF>&) { EF a = {}; a.scale = 1.0f; a.id_bytes = 8; return a; }
EB defaults(const Op<EB>&) { EB a = {}; a.scale = 1.0f; a.id_bytes = 8; return a; }
XS defaults(const Op<XS>&) { XS a = {}; a.id_bytes = 8; return a; }
template <typename T> T defaults(const Op<T>&) { return T{}; }

template <auto* kOp>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t npos, PyObject* kwnames)
{
    return run(*kOp, defaults(*kOp), args, npos, kwnames);
}

// bind_operators(addresses of the eight entry points, in the order of _OPERATORS in binding.py)
PyObject* bind_operators(PyObject*, PyObject* fns)
{
    if (!PyTuple_Check(fns) || PyTuple_GET_SIZE(fns) != 8) {
        PyErr_SetString(PyExc_ValueError, "bind_operators: wrong number of entry points");
        return nullptr;
    }
    void* p[8];
    for (int i = 0; i < 8; ++i)
        if (!to_address(PyTuple_GET_ITEM(fns, i), &p[i])) return nullptr;
    g_norm.call = reinterpret_cast<decltype(g_norm.call)>(p[0]);
    g_norm_grad.call = reinterpret_cast<decltype(g_norm_grad.call)>(p[1]);
    g_lookup.call = reinterpret_cast<decltype(g_lookup.call)>(p[2]);
    g_lookup_grad.call = reinterpret_cast<decltype(g_lookup_grad.call)>(p[3]);
    g_sort.call = reinterpret_cast<decltype(g_sort.call)>(p[4]);
    g_dispatch.call = reinterpret_cast<decltype(g_dispatch.call)>(p[5]);
    g_combine.call = reinterpret_cast<decltype(g_combine.call)>(p[6]);
    g_combine_grad.call = reinterpret_cast<decltype(g_combine_grad.call)>(p[7]);
    Py_RETURN_NONE;
}

#define NUNA_KW(fn) (PyCFunction)(void (*)(void))(fn), METH_FASTCALL | METH_KEYWORDS
#define NUNA_TAIL ", flags=0, stream=None, check=True)\n--\n\n"

PyMethodDef g_methods[] = {
    {"nuna_layernorm_forward", NUNA_KW(entry<&g_norm>),
     "nuna_layernorm_forward(x, y, rows, hidden, weight=None, bias=None, residual=None, summed=None, mean=None, rstd=None, eps=1e-05, "
     "dtype=0, param_dtype=0, x_stride=0, residual_stride=0, summed_stride=0, y_stride=0" NUNA_TAIL},
    {"nuna_layernorm_backward", NUNA_KW(entry<&g_norm_grad>),
     "nuna_layernorm_backward(dy, x, mean, rstd, dx, rows, hidden, weight=None, dsummed=None, dweight=None, dbias=None, workspace=None, "
     "dtype=0, param_dtype=0, dy_stride=0, x_stride=0, dsummed_stride=0, dx_stride=0, workspace_bytes=None" NUNA_TAIL},
    {"nuna_embedding_forward", NUNA_KW(entry<&g_lookup>),
     "nuna_embedding_forward(ids, table, out, tokens, hidden, vocab_rows, vocab_start=0, scale=1.0, dtype=0, id_bytes=8, "
     "table_stride=0, out_stride=0" NUNA_TAIL},
    {"nuna_embedding_backward", NUNA_KW(entry<&g_lookup_grad>),
     "nuna_embedding_backward(ids, dout, dtable, tokens, hidden, vocab_rows, workspace=None, vocab_start=0, scale=1.0, dtype=0, "
     "grad_dtype=0, id_bytes=8, dout_stride=0, dtable_stride=0, workspace_bytes=None" NUNA_TAIL},
    {"nuna_expert_sort", NUNA_KW(entry<&g_sort>),
     "nuna_expert_sort(experts, row_of_pair, pair_of_row, offsets, tokens, topk, num_experts, counts=None, first_expert=0, capacity=0, "
     "id_bytes=8" NUNA_TAIL},
    {"nuna_expert_dispatch", NUNA_KW(entry<&g_dispatch>),
     "nuna_expert_dispatch(x, row_of_pair, out, tokens, topk, rows, hidden, pair_of_row=None, dtype=0, x_stride=0, out_stride=0" NUNA_TAIL},
    {"nuna_expert_combine", NUNA_KW(entry<&g_combine>),
     "nuna_expert_combine(src, row_of_pair, y, tokens, topk, rows, hidden, weights=None, dtype=0, src_stride=0, y_stride=0" NUNA_TAIL},
    {"nuna_expert_combine_backward", NUNA_KW(entry<&g_combine_grad>),
     "nuna_expert_combine_backward(dy, src, weights, row_of_pair, dsrc, dweights, tokens, topk, rows, hidden, pair_of_row=None, dtype=0, "
     "dy_stride=0, src_stride=0, dsrc_stride=0" NUNA_TAIL},
    {"bind_operators", (PyCFunction)bind_operators, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr}};

template <typename T>
bool intern(Op<T>& op)
{
    for (int i = 0; i < op.n; ++i)
        if (!(op.field[i].name = PyUnicode_InternFromString(op.field[i].text))) return false;
    return true;
}

}  // namespace

bool add_operators(PyObject* module)
{
    for (int i = 0; i < 3; ++i)
        if (!(g_tail[i] = PyUnicode_InternFromString(kTail[i]))) return false;
    return intern(g_norm) && intern(g_norm_grad) && intern(g_lookup) && intern(g_lookup_grad) && intern(g_sort) && intern(g_dispatch) &&
           intern(g_combine) && intern(g_combine_grad) && PyModule_AddFunctions(module, g_methods) == 0;
}

}  // namespace nuna_py
