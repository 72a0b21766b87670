// The calls of sequence.py for arguments that need no conversion, checked and marshalled in C++: a Python layer costs a
// single-token call more than its kernel.  Every function here takes all its arguments by position, returns None if anything
// about them is out of the ordinary (wrong types, shapes, devices, an error status), and leaves that case to the Python code,
// which decides and reports.  Nothing is computed here.
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>

#include "../../include/sysconv_sequence.h"

namespace {

using at::Tensor;

struct Unusual {};                                            // thrown and caught here only

void need(bool ok)
{
    if (!ok) throw Unusual();
}

Tensor tensor(PyObject *o)
{
    need(THPVariable_Check(o));
    return THPVariable_Unpack(o);
}
Tensor maybe(PyObject *o) { return o == Py_None ? Tensor() : tensor(o); }

struct Place {
    at::ScalarType kind;
    c10::DeviceIndex device;
    int type;
    at::IntArrayRef sizes;
};

Place place_of(const Tensor &x)
{
    need(x.is_cuda() && x.get_device() == c10::cuda::current_device() && x.layout() == at::kStrided);
    Place p{x.scalar_type(), static_cast<c10::DeviceIndex>(x.get_device()), 0, x.sizes()};
    if (p.kind == at::kFloat) p.type = SYSCONV_T_F32;
    else if (p.kind == at::kBFloat16) p.type = SYSCONV_T_BF16;
    else if (p.kind == at::kHalf) p.type = SYSCONV_T_F16;
    else throw Unusual();
    return p;
}

sysconv_tokens tokens(const Tensor &x, const Place &p)
{
    need(x.is_cuda() && x.get_device() == p.device && x.scalar_type() == p.kind && x.sizes() == p.sizes && x.stride(-1) == 1);
    const bool dense = x.dim() == 3;
    return {x.data_ptr(), dense ? x.stride(0) : 0, x.stride(dense ? 1 : 0)};
}
sysconv_tokens maybe_tokens(const Tensor &x, const Place &p) { return x.defined() ? tokens(x, p) : sysconv_tokens{nullptr, 0, 0}; }

void *param(const Tensor &x, at::IntArrayRef sizes, at::ScalarType kind, const Place &p)
{
    if (!x.defined()) return nullptr;
    need(x.is_cuda() && x.get_device() == p.device && x.scalar_type() == kind && x.sizes() == sizes && x.is_contiguous());
    return x.data_ptr();
}

Tensor like(const Tensor &x, at::IntArrayRef sizes) { return at::empty(sizes, x.options().memory_format(at::MemoryFormat::Contiguous)); }

sysconv_sequences sequences(const Tensor &x, const Tensor &offsets, long long longest)
{
    if (!offsets.defined()) {
        need(x.dim() == 3);
        return {x.size(0), x.size(1), 0, nullptr, 0};
    }
    need(x.dim() == 2 && offsets.dim() == 1 && offsets.size(0) >= 2 && offsets.is_cuda() && offsets.get_device() == x.get_device() &&
         offsets.is_contiguous());
    const bool wide = offsets.scalar_type() == at::kLong;
    need(wide || offsets.scalar_type() == at::kInt);
    const long long total = x.size(0);
    return {offsets.size(0) - 1, longest >= 0 && longest < total ? longest : total, total, offsets.data_ptr(), wide ? 1 : 0};
}

long long number(PyObject *o)
{
    if (o == Py_None) return -1;
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        throw Unusual();
    }
    return v;
}
bool truth(PyObject *o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) PyErr_Clear();
    need(v >= 0);
    return v != 0;
}
int activation(PyObject *o)
{
    if (o == Py_None) return SYSCONV_ACT_NONE;
    need(PyUnicode_Check(o));
    if (PyUnicode_CompareWithASCIIString(o, "silu") == 0) return SYSCONV_ACT_SILU;
    need(PyUnicode_CompareWithASCIIString(o, "none") == 0);
    return SYSCONV_ACT_NONE;
}

void *stream_of(const Place &p) { return c10::cuda::getCurrentCUDAStream(p.device).stream(); }
void *pointer(const Tensor &x) { return x.defined() ? x.data_ptr() : nullptr; }

PyObject *give(const Tensor &x)
{
    if (x.defined()) return THPVariable_Wrap(x);
    Py_RETURN_NONE;
}
PyObject *give_all(std::initializer_list<Tensor> all)
{
    PyObject *t = PyTuple_New(static_cast<Py_ssize_t>(all.size()));
    Py_ssize_t i = 0;
    for (const Tensor &x : all) PyTuple_SET_ITEM(t, i++, give(x));
    return t;
}

// Runs f(arguments); None for the unusual.  No C++ exception leaves.
template <typename F>
PyObject *guarded(Py_ssize_t have, Py_ssize_t want, F f)
{
    if (have != want) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    try {
        return f();
    } catch (const Unusual &) {
    } catch (const std::exception &e) {                       // an allocation that failed, say: reported by the Python path if it persists
    }
    Py_RETURN_NONE;
}

// ---- causal convolution ---------------------------------------------------------------------------------------------

struct Causal {
    Place p;
    long long d, k;
    const void *w, *b;
    int weight_type;
};
Causal causal(const Tensor &x, const Tensor &weight, const Tensor &bias)
{
    Causal c{place_of(x), 0, 0, nullptr, nullptr, 0};
    need(weight.dim() == 2 && x.dim() >= 2);
    c.d = x.size(-1);
    c.k = weight.size(1);
    const at::ScalarType kind = weight.scalar_type();
    need(kind == c.p.kind || kind == at::kFloat);
    c.weight_type = kind == at::kFloat ? SYSCONV_T_F32 : c.p.type;
    c.w = param(weight, {c.d, c.k}, kind, c.p);
    c.b = param(bias, {c.d}, kind, c.p);
    need(c.d > 0 && c.k > 0);
    return c;
}

// x, weight, bias, activation, state, offsets, return_state
PyObject *conv(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    return guarded(n, 7, [&]() -> PyObject * {
        const Tensor x = tensor(o[0]), weight = tensor(o[1]), bias = maybe(o[2]), state = maybe(o[4]), offsets = maybe(o[5]);
        const Causal c = causal(x, weight, bias);
        sysconv_causal_args a = {};
        a.seq = sequences(x, offsets, -1);
        need(a.seq.sequences > 0);
        a.channels = c.d;
        a.taps = c.k;
        a.type = c.p.type;
        a.weight_type = c.weight_type;
        a.activation = activation(o[3]);
        a.x = tokens(x, c.p);
        a.weight = c.w;
        a.bias = c.b;
        const std::array<int64_t, 3> st = {a.seq.sequences, c.k - 1, c.d};
        a.state = param(state, st, c.p.kind, c.p);
        const Tensor y = like(x, x.sizes()), final = truth(o[6]) ? like(x, st) : Tensor();
        a.y = tokens(y, c.p);
        a.final_state = pointer(final);
        need(sysconv1d_causal(&a, stream_of(c.p)) == SYSCONV_OK);
        return final.defined() ? give_all({y, final}) : give(y);
    });
}

// dy, x, weight, bias, activation, state, offsets, dfinal
PyObject *conv_backward(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    return guarded(n, 8, [&]() -> PyObject * {
        const Tensor dy = tensor(o[0]), x = tensor(o[1]), weight = tensor(o[2]), bias = maybe(o[3]), state = maybe(o[5]),
                     offsets = maybe(o[6]), dfinal = maybe(o[7]);
        const Causal c = causal(x, weight, bias);
        sysconv_causal_args a = {};
        a.seq = sequences(x, offsets, -1);
        need(a.seq.sequences > 0);
        a.channels = c.d;
        a.taps = c.k;
        a.type = c.p.type;
        a.weight_type = c.weight_type;
        a.activation = activation(o[4]);
        const std::array<int64_t, 3> st = {a.seq.sequences, c.k - 1, c.d};
        const Tensor dx = like(x, x.sizes()), dw = like(weight, weight.sizes()), db = bias.defined() ? like(bias, bias.sizes()) : Tensor(),
                     ds = state.defined() ? like(x, st) : Tensor();
        a.x = tokens(x, c.p);
        a.y = tokens(dy, c.p);
        a.dx = tokens(dx, c.p);
        a.weight = c.w;
        a.bias = c.b;
        a.state = param(state, st, c.p.kind, c.p);
        a.dfinal = param(dfinal, st, c.p.kind, c.p);
        a.dstate = pointer(ds);
        a.dweight = pointer(dw);
        a.dbias = pointer(db);
        a.workspace_bytes = sysconv1d_causal_backward_workspace_bytes(&a);
        need(a.workspace_bytes >= 0);
        const Tensor room = at::empty({a.workspace_bytes}, x.options().dtype(at::kByte));
        a.workspace = room.data_ptr();
        need(sysconv1d_causal_backward(&a, stream_of(c.p)) == SYSCONV_OK);
        return give_all({dx, dw, db, ds});
    });
}

const int *slots_of(const Tensor &slots, long long rows, const Place &p)
{
    return static_cast<const int *>(param(slots, {rows}, at::kInt, p));
}
// pointer and stride of a cache of states (a, b) per slot
std::pair<void *, long long> cache(const Tensor &s, long long a, long long b, at::ScalarType kind, const Place &p, bool slots, long long rows)
{
    need(s.is_cuda() && s.get_device() == p.device && s.scalar_type() == kind && s.dim() == 3 && s.size(1) == a && s.size(2) == b);
    need((b <= 1 || s.stride(2) == 1) && (a <= 1 || s.stride(1) == b) && (slots || s.size(0) >= rows));
    return {s.data_ptr(), s.stride(0)};
}

// x, state, weight, bias, activation, slots
PyObject *conv_step(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    return guarded(n, 6, [&]() -> PyObject * {
        const Tensor x = tensor(o[0]), state = tensor(o[1]), weight = tensor(o[2]), bias = maybe(o[3]), slots = maybe(o[5]);
        const Causal c = causal(x, weight, bias);
        need(x.dim() == 2 && x.size(0) > 0 && x.stride(1) == 1);
        sysconv_causal_step_args a = {};
        a.rows = x.size(0);
        a.slots = state.size(0);
        a.channels = c.d;
        a.taps = c.k;
        a.type = c.p.type;
        a.weight_type = c.weight_type;
        a.activation = activation(o[4]);
        const Tensor y = like(x, x.sizes());
        a.x = x.data_ptr();
        a.x_stride = x.stride(0);
        a.y = y.data_ptr();
        a.y_stride = c.d;
        std::tie(a.state, a.state_stride) = cache(state, c.k - 1, c.d, c.p.kind, c.p, slots.defined(), a.rows);
        a.weight = c.w;
        a.bias = c.b;
        a.slot_dev = slots_of(slots, a.rows, c.p);
        need(sysconv1d_causal_step(&a, stream_of(c.p)) == SYSCONV_OK);
        return give(y);
    });
}

// ---- state space scan -------------------------------------------------------------------------------------------------

// groups; B, C: (..., states) or (..., groups, states)
long long scan_groups(const Tensor &u, const Tensor &A, const Tensor &B, const Tensor &C)
{
    const int64_t lead = u.dim() - 1, d = u.size(-1);
    need(A.dim() == 2 && A.size(0) == d && B.sizes() == C.sizes() && (B.dim() == lead + 1 || B.dim() == lead + 2) &&
         B.size(-1) == A.size(1) && B.sizes().slice(0, lead) == u.sizes().slice(0, lead) && d > 0 && A.size(1) > 0);
    const int64_t g = B.dim() == lead + 1 ? 1 : B.size(lead);
    need(g > 0 && d % g == 0);
    return g;
}
sysconv_tokens bc_tokens(const Tensor &x, const Place &p, long long n, long long g, bool dense)
{
    need(x.is_cuda() && x.get_device() == p.device && x.scalar_type() == p.kind && x.stride(-1) == 1 && (g == 1 || x.stride(-2) == n));
    return {x.data_ptr(), dense ? x.stride(0) : 0, x.stride(dense ? 1 : 0)};
}

struct Scan {
    Tensor u, delta, A, B, C, D, z, bias;
    Place p;
    sysscan_args a = {};
};
// u, delta, A, B, C from o[0]; D, z, delta_bias, softplus, from o[at]; offsets, longest
void scan_common(Scan &s, PyObject *const *o, int at, PyObject *offsets, PyObject *longest)
{
    s.u = tensor(o[0]);
    s.delta = tensor(o[1]);
    s.A = tensor(o[2]);
    s.B = tensor(o[3]);
    s.C = tensor(o[4]);
    s.D = maybe(o[at]);
    s.z = maybe(o[at + 1]);
    s.bias = maybe(o[at + 2]);
    s.p = place_of(s.u);
    need(s.u.dim() >= 2);
    sysscan_args &a = s.a;
    a.seq = sequences(s.u, maybe(offsets), number(longest));
    need(a.seq.sequences > 0);
    a.channels = s.u.size(-1);
    a.groups = scan_groups(s.u, s.A, s.B, s.C);
    a.states = s.A.size(1);
    a.type = s.p.type;
    a.softplus = truth(o[at + 3]);
    const bool dense = s.u.dim() == 3;
    a.u = tokens(s.u, s.p);
    a.delta = tokens(s.delta, s.p);
    a.z = maybe_tokens(s.z, s.p);
    a.B = bc_tokens(s.B, s.p, a.states, a.groups, dense);
    a.C = bc_tokens(s.C, s.p, a.states, a.groups, dense);
    a.A = param(s.A, {a.channels, a.states}, at::kFloat, s.p);
    a.D = param(s.D, {a.channels}, at::kFloat, s.p);
    a.delta_bias = param(s.bias, {a.channels}, at::kFloat, s.p);
}

// u, delta, A, B, C, D, z, delta_bias, softplus, state, offsets, longest, return_state, save
PyObject *scan(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    return guarded(n, 14, [&]() -> PyObject * {
        Scan s;
        scan_common(s, o, 5, o[10], o[11]);
        sysscan_args &a = s.a;
        const std::array<int64_t, 3> st = {a.seq.sequences, a.channels, a.states};
        const Tensor state = maybe(o[9]);
        a.state = param(state, st, at::kFloat, s.p);
        const bool want = truth(o[12]), save = truth(o[13]);
        const Tensor y = like(s.u, s.u.sizes()), final = want ? like(s.A, st) : Tensor();
        a.y = tokens(y, s.p);
        a.final_state = pointer(final);
        Tensor saved, room;
        if (save) {
            saved = like(s.A, {sysscan_saved_blocks(&a), a.channels, a.states});
            a.saved = saved.data_ptr();
        }
        a.workspace_bytes = sysscan_workspace_bytes(&a);
        need(a.workspace_bytes >= 0);
        if (a.workspace_bytes > 0) {
            room = at::empty({a.workspace_bytes}, s.u.options().dtype(at::kByte));
            a.workspace = room.data_ptr();
        }
        need(sysscan(&a, stream_of(s.p)) == SYSCONV_OK);
        if (want && save) return give_all({y, final, saved});
        if (want) return give_all({y, final});
        return save ? give_all({y, saved}) : give(y);
    });
}

// u, delta, A, B, C, dy, saved, D, z, delta_bias, softplus, offsets, longest, dfinal, state_grad -> nine gradients
PyObject *scan_backward(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    return guarded(n, 15, [&]() -> PyObject * {
        Scan s;
        scan_common(s, o, 7, o[11], o[12]);
        sysscan_args &a = s.a;
        const std::array<int64_t, 3> st = {a.seq.sequences, a.channels, a.states};
        const Tensor dy = tensor(o[5]), saved = tensor(o[6]), dfinal = maybe(o[13]);
        a.saved = param(saved, {sysscan_saved_blocks(&a), a.channels, a.states}, at::kFloat, s.p);
        a.dfinal = param(dfinal, st, at::kFloat, s.p);
        const bool dense = s.u.dim() == 3;
        const Tensor du = like(s.u, s.u.sizes()), dd = like(s.u, s.u.sizes()), dz = s.z.defined() ? like(s.u, s.u.sizes()) : Tensor(),
                     dB = like(s.B, s.B.sizes()), dC = like(s.B, s.B.sizes()), dA = like(s.A, s.A.sizes()),
                     dD = s.D.defined() ? like(s.D, s.D.sizes()) : Tensor(), db = s.bias.defined() ? like(s.bias, s.bias.sizes()) : Tensor(),
                     ds = truth(o[14]) ? like(s.A, st) : Tensor();
        a.dy = tokens(dy, s.p);
        a.du = tokens(du, s.p);
        a.ddelta = tokens(dd, s.p);
        a.dz = maybe_tokens(dz, s.p);
        a.dB = bc_tokens(dB, s.p, a.states, a.groups, dense);
        a.dC = bc_tokens(dC, s.p, a.states, a.groups, dense);
        a.dA = dA.data_ptr();
        a.dD = pointer(dD);
        a.ddelta_bias = pointer(db);
        a.dstate = pointer(ds);
        a.workspace_bytes = sysscan_backward_workspace_bytes(&a);
        need(a.workspace_bytes >= 0);
        const Tensor room = at::empty({a.workspace_bytes}, s.u.options().dtype(at::kByte));
        a.workspace = room.data_ptr();
        need(sysscan_backward(&a, stream_of(s.p)) == SYSCONV_OK);
        return give_all({du, dd, dA, dB, dC, dD, dz, db, ds});
    });
}

// u, delta, A, B, C, state, D, z, delta_bias, softplus, slots
PyObject *scan_step(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    return guarded(n, 11, [&]() -> PyObject * {
        const Tensor u = tensor(o[0]), delta = tensor(o[1]), A = tensor(o[2]), B = tensor(o[3]), C = tensor(o[4]), state = tensor(o[5]),
                     D = maybe(o[6]), z = maybe(o[7]), bias = maybe(o[8]), slots = maybe(o[10]);
        const Place p = place_of(u);
        need(u.dim() == 2 && u.size(0) > 0);
        sysscan_step_args a = {};
        a.rows = u.size(0);
        a.slots = state.size(0);
        a.channels = u.size(1);
        a.groups = scan_groups(u, A, B, C);
        a.states = A.size(1);
        a.type = p.type;
        a.softplus = truth(o[9]);
        auto row = [&](const Tensor &x, const void *&at, long long &stride) {
            const sysconv_tokens t = maybe_tokens(x, p);
            at = t.ptr;
            stride = t.time_stride;
        };
        row(u, a.u, a.u_stride);
        row(delta, a.delta, a.delta_stride);
        row(z, a.z, a.z_stride);
        const sysconv_tokens tb = bc_tokens(B, p, a.states, a.groups, false), tc = bc_tokens(C, p, a.states, a.groups, false);
        a.B = tb.ptr;
        a.b_stride = tb.time_stride;
        a.C = tc.ptr;
        a.c_stride = tc.time_stride;
        a.A = param(A, {a.channels, a.states}, at::kFloat, p);
        a.D = param(D, {a.channels}, at::kFloat, p);
        a.delta_bias = param(bias, {a.channels}, at::kFloat, p);
        std::tie(a.state, a.state_stride) = cache(state, a.channels, a.states, at::kFloat, p, slots.defined(), a.rows);
        a.slot_dev = slots_of(slots, a.rows, p);
        const Tensor y = like(u, u.sizes());
        a.y = y.data_ptr();
        a.y_stride = a.channels;
        need(sysscan_step(&a, stream_of(p)) == SYSCONV_OK);
        return give(y);
    });
}

// ---- group norm -------------------------------------------------------------------------------------------------------

// x of three dimensions, groups, weight, bias, eps, activation, return_stats
PyObject *norm(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    return guarded(n, 7, [&]() -> PyObject * {
        const Tensor x = tensor(o[0]), weight = maybe(o[2]), bias = maybe(o[3]);
        const Place p = place_of(x);
        need(x.dim() == 3 && x.numel() > 0 && PyFloat_Check(o[4]));
        sysgroupnorm_args a = {};
        a.batch = x.size(0);
        a.space = x.size(1);
        a.channels = x.size(2);
        a.groups = number(o[1]);
        a.type = p.type;
        a.activation = activation(o[5]);
        a.eps = PyFloat_AS_DOUBLE(o[4]);
        need(a.groups > 0);
        a.weight = param(weight, {a.channels}, at::kFloat, p);
        a.bias = param(bias, {a.channels}, at::kFloat, p);
        a.x = tokens(x, p);
        const Tensor y = like(x, x.sizes());
        a.y = tokens(y, p);
        Tensor mean, rstd, room;
        const auto f32 = x.options().dtype(at::kFloat);
        if (truth(o[6])) {
            mean = at::empty({a.batch, a.groups}, f32);
            rstd = at::empty({a.batch, a.groups}, f32);
            a.mean = mean.data_ptr();
            a.rstd = rstd.data_ptr();
        }
        a.workspace_bytes = sysgroupnorm_workspace_bytes(&a);
        need(a.workspace_bytes >= 0);
        if (a.workspace_bytes > 0) {
            room = at::empty({a.workspace_bytes}, x.options().dtype(at::kByte));
            a.workspace = room.data_ptr();
        }
        need(sysgroupnorm(&a, stream_of(p)) == SYSCONV_OK);
        return mean.defined() ? give_all({y, mean, rstd}) : give(y);
    });
}

// dy, x of three dimensions, groups, mean, rstd, weight, bias, activation
PyObject *norm_backward(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    return guarded(n, 8, [&]() -> PyObject * {
        const Tensor dy = tensor(o[0]), x = tensor(o[1]), mean = tensor(o[3]), rstd = tensor(o[4]), weight = maybe(o[5]), bias = maybe(o[6]);
        const Place p = place_of(x);
        need(x.dim() == 3 && x.numel() > 0);
        sysgroupnorm_args a = {};
        a.batch = x.size(0);
        a.space = x.size(1);
        a.channels = x.size(2);
        a.groups = number(o[2]);
        need(a.groups > 0);
        a.type = p.type;
        a.activation = activation(o[7]);
        a.weight = param(weight, {a.channels}, at::kFloat, p);
        a.bias = param(bias, {a.channels}, at::kFloat, p);
        a.mean = param(mean, {a.batch, a.groups}, at::kFloat, p);
        a.rstd = param(rstd, {a.batch, a.groups}, at::kFloat, p);
        const Tensor dx = like(x, x.sizes()), dw = weight.defined() ? like(weight, weight.sizes()) : Tensor(),
                     db = bias.defined() ? like(bias, bias.sizes()) : Tensor();
        a.x = tokens(x, p);
        a.dy = tokens(dy, p);
        a.dx = tokens(dx, p);
        a.dweight = pointer(dw);
        a.dbias = pointer(db);
        a.workspace_bytes = sysgroupnorm_backward_workspace_bytes(&a);
        need(a.workspace_bytes >= 0);
        const Tensor room = at::empty({a.workspace_bytes}, x.options().dtype(at::kByte));
        a.workspace = room.data_ptr();
        need(sysgroupnorm_backward(&a, stream_of(p)) == SYSCONV_OK);
        return give_all({dx, dw, db});
    });
}

#define ENTRY(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(conv), ENTRY(conv_backward), ENTRY(conv_step), ENTRY(scan), ENTRY(scan_backward), ENTRY(scan_step),
                         ENTRY(norm), ENTRY(norm_backward), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_sequence", "Marshalling of the sequence operators' calls.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__sequence() { return PyModule_Create(&module); }
