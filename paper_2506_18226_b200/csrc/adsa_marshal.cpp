// The Python side of the calls that a decoder makes once per layer and step: reads torch tensors, checks them, calls the
// C functions (whose addresses bind() is given).  Argument marshalling only; done in C++ because the checks of a dozen
// tensors cost more in Python (3 to 6 us a call) than the kernels of a decode step take.
//
// Every function returns its tensors, or the negative adsa_status of the C call as an int; a tensor that is not what the
// call wants raises ValueError.
#include <Python.h>

#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/headeronly/version.h>

#include <initializer_list>
#include <string>

#include "../../include/adsa.h"

namespace {

decltype(&adsa_rope_axes) c_rope_axes;
decltype(&adsa_paged_append) c_paged_append;
decltype(&adsa_shared_prefix_workspace_bytes) c_workspace_bytes;
decltype(&adsa_shared_prefix_attn) c_shared_prefix_attn;
decltype(&adsa_norm_residual) c_norm_residual;
decltype(&adsa_prompt_workspace_bytes) c_prompt_workspace_bytes;
decltype(&adsa_packed_attn_status) c_packed_attn;
decltype(&adsa_chunk_attn) c_chunk_attn;
decltype(&adsa_sample) c_sample;

struct Raised {};                            // a Python exception is set

// (no streams here: a compiler that links its own C++ library into this module would mix two libraries' locales)
template <typename Sizes> std::string list_of(const Sizes &sizes)
{
    std::string s = "[";
    for (int64_t n : sizes) s += (s.size() > 1 ? ", " : "") + (n < 0 ? std::string("any") : std::to_string(n));
    return s + "]";
}

[[noreturn]] void refuse(const std::string &what)
{
    PyErr_SetString(PyExc_ValueError, what.c_str());
    throw Raised();
}

// None: undefined
const at::Tensor &tensor(PyObject *o, const char *call, const char *name)
{
    static const at::Tensor none;
    if (o == Py_None) return none;
    if (!THPVariable_Check(o)) refuse(std::string(call) + ": " + name + " must be a tensor");
    return THPVariable_Unpack(o);
}

// One call's checks: the device is the first tensor's.
struct Check {
    const char *call;
    int dev = -1;
    void device_of(const at::Tensor &t, const char *name)
    {
        if (!t.defined()) refuse(std::string(call) + ": " + name + " is missing");
        if (!t.is_cuda()) refuse(std::string(call) + ": " + name + " must be on a CUDA device");
        dev = t.get_device();
    }
    // shape: -1 for any size.  whole: dense throughout, else along the last dimension
    void wants(const at::Tensor &t, const char *name, at::ScalarType type, std::initializer_list<int64_t> shape, bool whole) const
    {
        bool ok = t.defined() && t.scalar_type() == type && t.dim() == (int64_t)shape.size();
        if (ok) {
            const int64_t *have = t.sizes().data();
            for (int64_t want : shape) {
                ok = ok && (want < 0 || want == *have);
                ++have;
            }
        }
        if (!ok) {
            refuse(std::string(call) + ": " + name + " must be " + c10::toString(type) + " " + list_of(shape) + ", got " +
                   (t.defined() ? std::string(c10::toString(t.scalar_type())) + " " + list_of(t.sizes()) : std::string("None")));
        }
        if (!(whole ? t.is_contiguous() : t.numel() == 0 || t.stride(-1) == 1))
            refuse(std::string(call) + ": " + name + " must be dense" + (whole ? "" : " along its last dimension"));
        if (!t.is_cuda() || t.get_device() != dev) refuse(std::string(call) + ": " + name + " must be on a CUDA device, the same for all tensors");
    }
    int code(const at::Tensor &t, const char *name, int64_t dims) const
    {
        if (t.dim() != dims || (t.scalar_type() != at::kBFloat16 && t.scalar_type() != at::kHalf))
            refuse(std::string(call) + ": " + name + " must be bfloat16 or float16 with " + std::to_string(dims) + " dimensions, got " +
                   c10::toString(t.scalar_type()) + " " + list_of(t.sizes()));
        return t.scalar_type() == at::kBFloat16 ? ADSA_BF16 : ADSA_F16;
    }
};

template <typename P> P *at_of(const at::Tensor &t) { return t.defined() ? static_cast<P *>(t.data_ptr()) : nullptr; }

adsa_stream_t stream_of(int dev) { return (adsa_stream_t)c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream(); }

// status, or `out` where the call went well
PyObject *answer(int rc, PyObject *out)
{
    if (rc == ADSA_OK) return out;
    Py_DECREF(out);
    return PyLong_FromLong(rc);
}
PyObject *wrap(const at::Tensor &t, PyObject *given)
{
    if (given != nullptr && given != Py_None) {
        Py_INCREF(given);
        return given;
    }
    if (!t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(t);
}

void need(Py_ssize_t n, Py_ssize_t want, const char *call)
{
    if (n != want) {
        PyErr_Format(PyExc_TypeError, "%s takes %zd arguments, got %zd", call, want, n);
        throw Raised();
    }
}
double number(PyObject *o)
{
    const double x = PyFloat_AsDouble(o);
    if (x == -1.0 && PyErr_Occurred()) throw Raised();
    return x;
}
const adsa_rotary *rotary(PyObject *o)
{
    if (o == Py_None) return nullptr;
    void *p = PyLong_AsVoidPtr(o);
    if (!p && PyErr_Occurred()) throw Raised();
    return static_cast<const adsa_rotary *>(p);
}

adsa_paged_kv pool_of(const Check &c, const at::Tensor &k, const at::Tensor &v, int code, at::ScalarType type, int64_t heads, int64_t head_dim)
{
    c.wants(k, "k_pool", type, {-1, heads, -1, -1}, true);
    c.wants(v, "v_pool", type, {k.size(0), k.size(1), k.size(2), k.size(3)}, true);
    for (int i = 0; i < 4; ++i)
        if (k.size(i) > 0x7fffffff) refuse(std::string(c.call) + ": the pools are too large");
    return {k.data_ptr(), v.data_ptr(), code, (int32_t)k.size(0), (int32_t)k.size(1), (int32_t)k.size(2), (int32_t)head_dim, (int32_t)k.size(3)};
}

// rotary address, x, pos, out
PyObject *rope_axes(PyObject *const *a, Py_ssize_t n)
{
    Check c{"rope_axes"};
    need(n, 4, c.call);
    const adsa_rotary *rot = rotary(a[0]);
    const at::Tensor &x = tensor(a[1], c.call, "x"), &pos = tensor(a[2], c.call, "pos");
    c.device_of(x, "x");
    const int code = c.code(x, "x", 3);
    const int64_t tokens = x.size(0), heads = x.size(1);
    c.wants(x, "x", x.scalar_type(), {-1, -1, rot->head_dim}, false);
    c.wants(pos, "pos", at::kInt, {tokens, rot->n_axes}, true);
    if (heads > 0x7fffffff) refuse("rope_axes: sizes out of range");
    at::Tensor out = tensor(a[3], c.call, "out");
    if (out.defined()) c.wants(out, "out", x.scalar_type(), {tokens, heads, rot->head_dim}, false);
    else out = at::empty(x.sizes(), x.options());
    const c10::cuda::CUDAGuard guard((c10::DeviceIndex)c.dev);
    const int rc = c_rope_axes(rot, code, x.data_ptr(), x.stride(0), x.stride(1), at_of<int32_t>(pos), tokens, (int)heads, out.data_ptr(), out.stride(0),
                               out.stride(1), stream_of(c.dev));
    return answer(rc, wrap(out, a[3]));
}

// k, v, k_pool, v_pool, page_table, n_rows, cu_tokens, rotary address, pos, q, q_out, status
PyObject *paged_append(PyObject *const *a, Py_ssize_t n)
{
    Check c{"paged_append"};
    need(n, 12, c.call);
    const at::Tensor &k = tensor(a[0], c.call, "k"), &v = tensor(a[1], c.call, "v"), &table = tensor(a[4], c.call, "page_table"),
                     &n_rows = tensor(a[5], c.call, "n_rows"), &cu = tensor(a[6], c.call, "cu_tokens"), &q = tensor(a[9], c.call, "q"),
                     &status = tensor(a[11], c.call, "status");
    const adsa_rotary *rot = rotary(a[7]);
    c.device_of(k, "k");
    const int code = c.code(k, "k", 3);
    const at::ScalarType type = k.scalar_type();
    const int64_t tokens = k.size(0), heads = k.size(1), d = k.size(2);
    c.wants(k, "k", type, {-1, -1, -1}, false);
    c.wants(v, "v", type, {tokens, heads, d}, false);
    const adsa_paged_kv kv = pool_of(c, tensor(a[2], c.call, "k_pool"), tensor(a[3], c.call, "v_pool"), code, type, heads, d);
    c.wants(table, "page_table", at::kInt, {-1, -1}, true);
    const int64_t batch = table.size(0);
    c.wants(n_rows, "n_rows", at::kInt, {batch}, true);
    if (cu.defined()) c.wants(cu, "cu_tokens", at::kInt, {batch + 1}, true);
    if (status.defined()) c.wants(status, "status", at::kInt, {1}, true);
    const at::Tensor none, &pos = rot ? tensor(a[8], c.call, "pos") : none;
    if (rot) {
        if (rot->head_dim != d) refuse("paged_append: the rotary is for another head dimension than k's");
        c.wants(pos, "pos", at::kInt, {tokens, rot->n_axes}, true);
    }
    at::Tensor q_out = tensor(a[10], c.call, "q_out");
    if (q_out.defined() && !q.defined()) refuse("paged_append: q_out needs q");
    int64_t q_heads = 0, qs[4] = {0, 0, 0, 0};
    if (q.defined()) {
        c.wants(q, "q", type, {tokens, -1, d}, false);
        q_heads = q.size(1);
        if (q_out.defined()) c.wants(q_out, "q_out", type, {tokens, q_heads, d}, false);
        else q_out = at::empty(q.sizes(), q.options());
        qs[0] = q.stride(0); qs[1] = q.stride(1); qs[2] = q_out.stride(0); qs[3] = q_out.stride(1);
    }
    if (batch > 0x7fffffff || table.size(1) > 0x7fffffff || q_heads > 0x7fffffff) refuse("paged_append: sizes out of range");
    const c10::cuda::CUDAGuard guard((c10::DeviceIndex)c.dev);
    const int rc = c_paged_append(&kv, at_of<int32_t>(table), (int)batch, (int)table.size(1), at_of<int32_t>(n_rows), at_of<int32_t>(cu), tokens,
                                  k.data_ptr(), k.stride(0), k.stride(1), v.data_ptr(), v.stride(0), v.stride(1), rot, at_of<int32_t>(pos), at_of<void>(q),
                                  (int)q_heads, qs[0], qs[1], at_of<void>(q_out), qs[2], qs[3], (uint32_t *)at_of<int32_t>(status), stream_of(c.dev));
    return answer(rc, wrap(q_out, q.defined() ? a[10] : nullptr));
}

// q, k_pool, v_pool, page_table, n_rows, prefix_table, prefix_rows, group_start, scale, out, out_f32, lse, workspace, status
PyObject *shared_prefix_attn(PyObject *const *a, Py_ssize_t n)
{
    Check c{"shared_prefix_attn"};
    need(n, 14, c.call);
    const at::Tensor &q = tensor(a[0], c.call, "q"), &table = tensor(a[3], c.call, "page_table"), &n_rows = tensor(a[4], c.call, "n_rows"),
                     &p_table = tensor(a[5], c.call, "prefix_table"), &p_rows = tensor(a[6], c.call, "prefix_rows"),
                     &start = tensor(a[7], c.call, "group_start"), &out_f32 = tensor(a[10], c.call, "out_f32"), &lse = tensor(a[11], c.call, "lse"),
                     &status = tensor(a[13], c.call, "status");
    c.device_of(q, "q");
    const int code = c.code(q, "q", 3);
    const at::ScalarType type = q.scalar_type();
    const int64_t batch = q.size(0), heads = q.size(1), d = q.size(2);
    c.wants(q, "q", type, {-1, -1, -1}, false);
    const adsa_paged_kv kv = pool_of(c, tensor(a[1], c.call, "k_pool"), tensor(a[2], c.call, "v_pool"), code, type, -1, d);
    c.wants(table, "page_table", at::kInt, {batch, -1}, true);
    c.wants(n_rows, "n_rows", at::kInt, {batch}, true);
    int64_t groups = 0, p_pages = 0;
    if (p_table.defined()) {
        c.wants(p_table, "prefix_table", at::kInt, {-1, -1}, true);
        groups = p_table.size(0);
        p_pages = p_table.size(1);
        c.wants(p_rows, "prefix_rows", at::kInt, {groups}, true);
        c.wants(start, "group_start", at::kInt, {groups + 1}, true);
    } else if (p_rows.defined() || start.defined()) {
        refuse("shared_prefix_attn: prefix_rows and group_start need prefix_table");
    }
    if (status.defined()) c.wants(status, "status", at::kInt, {1}, true);
    at::Tensor out = tensor(a[9], c.call, "out");
    if (out.defined()) c.wants(out, "out", type, {batch, heads, d}, true);
    if (out_f32.defined()) c.wants(out_f32, "out_f32", at::kFloat, {batch, heads, d}, true);
    if (lse.defined()) c.wants(lse, "lse", at::kFloat, {batch, heads}, true);
    if (batch > 0x7fffffff || heads > 0x7fffffff || table.size(1) > 0x7fffffff || groups > 0x7fffffff || p_pages > 0x7fffffff)
        refuse("shared_prefix_attn: sizes out of range");
    const float scale = (float)number(a[8]);
    const c10::cuda::CUDAGuard guard((c10::DeviceIndex)c.dev);
    if (!out.defined() && !out_f32.defined()) out = at::empty(q.sizes(), q.options());
    at::Tensor ws = tensor(a[12], c.call, "workspace");
    if (ws.defined()) {
        if (!ws.is_contiguous() || !ws.is_cuda() || ws.get_device() != c.dev) refuse("shared_prefix_attn: workspace must be dense, on the device of q");
    } else if (batch > 0) {
        size_t bytes = 0;
        const int rc = c_workspace_bytes((int)batch, (int)groups, (int)heads, kv.n_kv_heads, (int)d, &bytes);
        if (rc != ADSA_OK) return PyLong_FromLong(rc);
        ws = at::empty({(int64_t)bytes}, q.options().dtype(at::kByte));
    }
    const int rc = c_shared_prefix_attn(&kv, q.data_ptr(), q.stride(0), q.stride(1), (int)batch, (int)heads, at_of<int32_t>(table), (int)table.size(1),
                                        at_of<int32_t>(n_rows), at_of<int32_t>(p_table), (int)p_pages, at_of<int32_t>(p_rows), at_of<int32_t>(start),
                                        (int)groups, scale, at_of<void>(out), at_of<float>(out_f32), at_of<float>(lse), at_of<void>(ws),
                                        ws.defined() ? ws.nbytes() : 0, (uint32_t *)at_of<int32_t>(status), stream_of(c.dev));
    return answer(rc, out.defined() ? wrap(out, a[9]) : wrap(out_f32, a[10]));
}

// y, x, w_pre, w_post, gate, scale, eps, x_out, h
PyObject *norm_residual(PyObject *const *a, Py_ssize_t n)
{
    Check c{"norm_residual"};
    need(n, 9, c.call);
    const at::Tensor &y = tensor(a[0], c.call, "y"), &x = tensor(a[1], c.call, "x"), &w_pre = tensor(a[2], c.call, "w_pre"),
                     &w_post = tensor(a[3], c.call, "w_post"), &gate = tensor(a[4], c.call, "gate");
    c.device_of(y, "y");
    const int code = c.code(y, "y", 2);
    const at::ScalarType type = y.scalar_type();
    if (!x.defined()) refuse("norm_residual: x is missing");
    const at::ScalarType x_type = x.scalar_type() == at::kFloat ? at::kFloat : type;
    const int64_t rows = y.size(0), dim = y.size(1);
    c.wants(y, "y", type, {-1, -1}, true);
    c.wants(x, "x", x_type, {rows, dim}, true);
    if (w_post.defined()) c.wants(w_post, "w_post", type, {dim}, true);
    if (gate.defined()) c.wants(gate, "gate", type, {-1, dim}, true);
    at::Tensor x_out = tensor(a[7], c.call, "x_out"), h = tensor(a[8], c.call, "h");
    if (x_out.defined()) c.wants(x_out, "x_out", x_type, {rows, dim}, true);
    else x_out = at::empty(x.sizes(), x.options());
    if (w_pre.defined()) {
        c.wants(w_pre, "w_pre", type, {dim}, true);
        if (h.defined()) c.wants(h, "h", type, {rows, dim}, true);
        else h = at::empty(y.sizes(), y.options());
    } else if (h.defined()) {
        refuse("norm_residual: h needs w_pre");
    }
    if (dim > 0x7fffffff) refuse("norm_residual: sizes out of range");
    const float scale = (float)number(a[5]), eps = (float)number(a[6]);
    const c10::cuda::CUDAGuard guard((c10::DeviceIndex)c.dev);
    const int rc = c_norm_residual(code, x_type == at::kFloat ? ADSA_F32 : code, y.data_ptr(), x.data_ptr(), at_of<void>(w_post), at_of<void>(gate),
                                   gate.defined() ? gate.size(0) : 0, at_of<void>(w_pre), x_out.data_ptr(), at_of<void>(h), rows, (int)dim, scale, eps,
                                   stream_of(c.dev));
    PyObject *xo = wrap(x_out, a[7]), *ho = wrap(h, a[8]);
    PyObject *both = PyTuple_Pack(2, xo, ho);
    Py_DECREF(xo);
    Py_DECREF(ho);
    return answer(rc, both);
}

// whether two tensors (no negative strides) have bytes in common, by their first and last
bool touch(const at::Tensor &x, const at::Tensor &y)
{
    if (!x.defined() || !y.defined() || x.numel() == 0 || y.numel() == 0) return false;
    const auto end = [](const at::Tensor &t) {
        int64_t last = 0;
        for (int64_t i = 0; i < t.dim(); ++i) last += (t.size(i) - 1) * t.stride(i);
        return (uintptr_t)t.data_ptr() + (uintptr_t)(last + 1) * t.element_size();
    };
    return (uintptr_t)x.data_ptr() < end(y) && (uintptr_t)y.data_ptr() < end(x);
}

// outputs and workspace of the two calls with many query rows per sequence
struct RowsOut {
    at::Tensor out, ws;
    const at::Tensor &out_f32, &lse;
    int rc = ADSA_OK;
    // o: out, out_f32, lse, workspace
    RowsOut(const Check &c, const at::Tensor &q, const at::Tensor &k, const at::Tensor &v, PyObject *const *o, int64_t batch, int64_t kv_heads)
        : out(tensor(o[0], c.call, "out")), ws(tensor(o[3], c.call, "workspace")), out_f32(tensor(o[1], c.call, "out_f32")), lse(tensor(o[2], c.call, "lse"))
    {
        const int64_t tokens = q.size(0), heads = q.size(1), d = q.size(2);
        if (out.defined()) c.wants(out, "out", q.scalar_type(), {tokens, heads, d}, true);
        if (out_f32.defined()) c.wants(out_f32, "out_f32", at::kFloat, {tokens, heads, d}, true);
        if (lse.defined()) c.wants(lse, "lse", at::kFloat, {tokens, heads}, true);
        if (batch > 0x7fffffff || heads > 0x7fffffff || kv_heads > 0x7fffffff || d > 0x7fffffff) refuse(std::string(c.call) + ": sizes out of range");
        const at::Tensor *written[4] = {&out, &out_f32, &lse, &lse};    // (rows are read again after others are written)
        if (ws.defined()) {
            if (!ws.is_contiguous() || !ws.is_cuda() || ws.get_device() != c.dev) refuse(std::string(c.call) + ": workspace must be dense, on the device of q");
            written[3] = &ws;
        } else if (tokens > 0) {
            size_t bytes = 0;
            rc = c_prompt_workspace_bytes((int)batch, (int)heads, (int)kv_heads, (int)d, &bytes);
            if (rc == ADSA_OK) ws = at::empty({(int64_t)bytes}, q.options().dtype(at::kByte));
        }
        for (int i = 0; i < 4; ++i) {
            bool bad = touch(*written[i], q) || touch(*written[i], k) || touch(*written[i], v);
            for (int j = 0; j < i; ++j) bad = bad || (written[i] != written[j] && touch(*written[i], *written[j]));
            if (bad) refuse(std::string(c.call) + ": outputs and workspace must not overlap q, the cached rows or one another");
        }
        if (!out.defined() && !out_f32.defined()) out = at::empty(q.sizes(), q.options());
    }
    size_t ws_bytes() const { return ws.defined() ? ws.nbytes() : 0; }
    PyObject *result(int status, PyObject *const *o) const { return answer(status, out.defined() ? wrap(out, o[0]) : wrap(out_f32, o[1])); }
};

// q, k, v, cu_q, cu_k, causal, scale, out, out_f32, lse, workspace, status
PyObject *packed_attn(PyObject *const *a, Py_ssize_t n)
{
    Check c{"packed_attn"};
    need(n, 12, c.call);
    const at::Tensor &q = tensor(a[0], c.call, "q"), &k = tensor(a[1], c.call, "k"), &v = tensor(a[2], c.call, "v"), &cu_q = tensor(a[3], c.call, "cu_q"),
                     &status = tensor(a[11], c.call, "status");
    at::Tensor cu_k = tensor(a[4], c.call, "cu_k");
    c.device_of(q, "q");
    const int code = c.code(q, "q", 3);
    const at::ScalarType type = q.scalar_type();
    const int64_t d = q.size(2);
    c.wants(q, "q", type, {-1, -1, -1}, false);
    c.wants(k, "k", type, {-1, -1, d}, false);
    c.wants(v, "v", type, {k.size(0), k.size(1), d}, false);
    int64_t batch = 1;
    if (cu_q.defined()) {
        c.wants(cu_q, "cu_q", at::kInt, {-1}, true);
        batch = cu_q.size(0) - 1;
        if (batch < 1) refuse("packed_attn: cu_q must have two boundaries at least");
        if (!cu_k.defined()) cu_k = cu_q;
    }
    if (cu_k.defined()) {
        c.wants(cu_k, "cu_k", at::kInt, {cu_q.defined() ? batch + 1 : -1}, true);
        if (!cu_q.defined()) refuse("packed_attn: cu_k needs cu_q");
    }
    if (status.defined()) c.wants(status, "status", at::kInt, {1}, true);
    const int causal = PyObject_IsTrue(a[5]);
    if (causal < 0) throw Raised();
    const float scale = (float)number(a[6]);
    const c10::cuda::CUDAGuard guard((c10::DeviceIndex)c.dev);
    const RowsOut o(c, q, k, v, a + 7, batch, k.size(1));
    if (o.rc != ADSA_OK) return PyLong_FromLong(o.rc);
    const int rc = c_packed_attn(code, q.data_ptr(), q.stride(0), q.stride(1), k.data_ptr(), k.stride(0), k.stride(1), v.data_ptr(), v.stride(0),
                                 v.stride(1), at_of<int32_t>(cu_q), at_of<int32_t>(cu_k), (int)batch, q.size(0), k.size(0), (int)q.size(1),
                                 (int)k.size(1), (int)d, causal, scale, at_of<void>(o.out), at_of<float>(o.out_f32), at_of<float>(o.lse),
                                 at_of<void>(o.ws), o.ws_bytes(), (uint32_t *)at_of<int32_t>(status), stream_of(c.dev));
    return o.result(rc, a + 7);
}

// q, k_pool, v_pool, page_table, n_rows, cu_tokens, prefix_table, prefix_rows, group_start, scale, out, out_f32, lse, workspace, status
PyObject *chunk_attn(PyObject *const *a, Py_ssize_t n)
{
    Check c{"chunk_attn"};
    need(n, 15, c.call);
    const at::Tensor &q = tensor(a[0], c.call, "q"), &table = tensor(a[3], c.call, "page_table"), &n_rows = tensor(a[4], c.call, "n_rows"),
                     &cu = tensor(a[5], c.call, "cu_tokens"), &p_table = tensor(a[6], c.call, "prefix_table"),
                     &p_rows = tensor(a[7], c.call, "prefix_rows"), &start = tensor(a[8], c.call, "group_start"), &status = tensor(a[14], c.call, "status");
    c.device_of(q, "q");
    const int code = c.code(q, "q", 3);
    const at::ScalarType type = q.scalar_type();
    c.wants(q, "q", type, {-1, -1, -1}, false);
    const adsa_paged_kv kv = pool_of(c, tensor(a[1], c.call, "k_pool"), tensor(a[2], c.call, "v_pool"), code, type, -1, q.size(2));
    c.wants(table, "page_table", at::kInt, {-1, -1}, true);
    const int64_t batch = table.size(0);
    c.wants(n_rows, "n_rows", at::kInt, {batch}, true);
    if (cu.defined()) c.wants(cu, "cu_tokens", at::kInt, {batch + 1}, true);
    int64_t groups = 0, p_pages = 0;
    if (p_table.defined()) {
        c.wants(p_table, "prefix_table", at::kInt, {-1, -1}, true);
        groups = p_table.size(0);
        p_pages = p_table.size(1);
        c.wants(p_rows, "prefix_rows", at::kInt, {groups}, true);
        c.wants(start, "group_start", at::kInt, {groups + 1}, true);
    } else if (p_rows.defined() || start.defined()) {
        refuse("chunk_attn: prefix_rows and group_start need prefix_table");
    }
    if (status.defined()) c.wants(status, "status", at::kInt, {1}, true);
    if (table.size(1) > 0x7fffffff || groups > 0x7fffffff || p_pages > 0x7fffffff) refuse("chunk_attn: sizes out of range");
    const float scale = (float)number(a[9]);
    const c10::cuda::CUDAGuard guard((c10::DeviceIndex)c.dev);
    const RowsOut o(c, q, tensor(a[1], c.call, "k_pool"), tensor(a[2], c.call, "v_pool"), a + 10, batch, kv.n_kv_heads);
    if (o.rc != ADSA_OK) return PyLong_FromLong(o.rc);
    const int rc = c_chunk_attn(&kv, q.data_ptr(), q.stride(0), q.stride(1), at_of<int32_t>(cu), (int)batch, q.size(0), (int)q.size(1),
                                at_of<int32_t>(table), (int)table.size(1), at_of<int32_t>(n_rows), at_of<int32_t>(p_table), (int)p_pages,
                                at_of<int32_t>(p_rows), at_of<int32_t>(start), (int)groups, scale, at_of<void>(o.out), at_of<float>(o.out_f32),
                                at_of<float>(o.lse), at_of<void>(o.ws), o.ws_bytes(), (uint32_t *)at_of<int32_t>(status), stream_of(c.dev));
    return o.result(rc, a + 10);
}

// logits, uniforms, temperature, top_k, top_p, min_p, uncond, guidance, tokens, logprobs
PyObject *sample(PyObject *const *a, Py_ssize_t n)
{
    Check c{"sample"};
    need(n, 10, c.call);
    const at::Tensor &logits = tensor(a[0], c.call, "logits"), &uniforms = tensor(a[1], c.call, "uniforms"), &uncond = tensor(a[6], c.call, "uncond"),
                     &logprobs = tensor(a[9], c.call, "logprobs");
    c.device_of(logits, "logits");
    const at::ScalarType type = logits.scalar_type();
    const int code = type == at::kFloat && logits.dim() == 2 ? ADSA_F32 : c.code(logits, "logits", 2);
    c.wants(logits, "logits", type, {-1, -1}, false);
    const int64_t rows = logits.size(0), vocab = logits.size(1);
    c.wants(uniforms, "uniforms", at::kFloat, {rows}, true);
    if (uncond.defined()) c.wants(uncond, "uncond", type, {rows, vocab}, false);
    if (logprobs.defined()) c.wants(logprobs, "logprobs", at::kFloat, {rows}, true);
    at::Tensor tokens = tensor(a[8], c.call, "tokens");
    if (tokens.defined()) c.wants(tokens, "tokens", at::kInt, {rows}, true);
    adsa_sampling how = {1.f, 0, 1.f, 0.f, nullptr, nullptr, nullptr, nullptr, (float)number(a[7])};
    const auto setting = [&](PyObject *o, const char *name, float &all, const float *&each) {   // a number, or one per row
        if (!THPVariable_Check(o)) {
            all = (float)number(o);
            return;
        }
        const at::Tensor &t = THPVariable_Unpack(o);
        c.wants(t, name, at::kFloat, {rows}, true);
        each = at_of<float>(t);
    };
    setting(a[2], "temperature", how.temperature, how.temperatures);
    setting(a[4], "top_p", how.top_p, how.top_ps);
    setting(a[5], "min_p", how.min_p, how.min_ps);
    if (THPVariable_Check(a[3])) {
        const at::Tensor &t = THPVariable_Unpack(a[3]);
        c.wants(t, "top_k", at::kInt, {rows}, true);
        how.top_ks = at_of<int32_t>(t);
    } else {
        const long k = PyLong_AsLong(a[3]);
        if (k == -1 && PyErr_Occurred()) throw Raised();
        if (k > 0x7fffffff || k < -0x7fffffff) refuse("sample: top_k is out of range");
        how.top_k = (int32_t)k;
    }
    if (rows > 0x7fffffff || vocab > 0x7fffffff) refuse("sample: sizes out of range");
    bool over = touch(tokens, logprobs);
    for (const at::Tensor *x : std::initializer_list<const at::Tensor *>{&tokens, &logprobs}) {
        over = over || touch(*x, logits) || touch(*x, uncond) || touch(*x, uniforms);
        for (int i = 2; i < 6; ++i) over = over || (THPVariable_Check(a[i]) && touch(*x, THPVariable_Unpack(a[i])));
    }
    if (over) refuse("sample: tokens and logprobs must not overlap the inputs or one another");
    const c10::cuda::CUDAGuard guard((c10::DeviceIndex)c.dev);
    if (!tokens.defined()) tokens = at::empty({rows}, logits.options().dtype(at::kInt));
    const int rc = c_sample(&how, code, logits.data_ptr(), logits.stride(0), at_of<void>(uncond), uncond.defined() ? uncond.stride(0) : 0, (int)rows,
                            (int)vocab, at_of<float>(uniforms), at_of<int32_t>(tokens), at_of<float>(logprobs), stream_of(c.dev));
    return answer(rc, wrap(tokens, a[8]));
}

// the addresses of the C functions, in the order of the declarations above
PyObject *bind(PyObject *const *a, Py_ssize_t n)
{
    constexpr int kBound = 9;
    need(n, kBound, "bind");
    void *p[kBound];
    for (int i = 0; i < kBound; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (!p[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "bind: a function is missing");
            throw Raised();
        }
    }
    c_rope_axes = (decltype(c_rope_axes))p[0];
    c_paged_append = (decltype(c_paged_append))p[1];
    c_workspace_bytes = (decltype(c_workspace_bytes))p[2];
    c_shared_prefix_attn = (decltype(c_shared_prefix_attn))p[3];
    c_norm_residual = (decltype(c_norm_residual))p[4];
    c_prompt_workspace_bytes = (decltype(c_prompt_workspace_bytes))p[5];
    c_packed_attn = (decltype(c_packed_attn))p[6];
    c_chunk_attn = (decltype(c_chunk_attn))p[7];
    c_sample = (decltype(c_sample))p[8];
    Py_RETURN_NONE;
}

// nothing but a Python exception leaves a call
template <PyObject *(*F)(PyObject *const *, Py_ssize_t)>
PyObject *entry(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    try {
        return F(a, n);
    } catch (const Raised &) {
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown error");
    }
    return nullptr;
}

#define ADSA_ENTRY(name) {#name, (PyCFunction)(void *)entry<name>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ADSA_ENTRY(bind),          ADSA_ENTRY(rope_axes),     ADSA_ENTRY(paged_append),
                         ADSA_ENTRY(shared_prefix_attn), ADSA_ENTRY(norm_residual), ADSA_ENTRY(packed_attn),
                         ADSA_ENTRY(chunk_attn),    ADSA_ENTRY(sample),        {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "adsa_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// What this module was built against, for build.py to find in the file before anything of it is loaded
#define ADSA_TEXT_(x) #x
#define ADSA_TEXT(x) ADSA_TEXT_(x)
__attribute__((used)) const char built_against[] =
    "adsa_marshal built against torch " TORCH_VERSION ", Python " ADSA_TEXT(PY_MAJOR_VERSION) "." ADSA_TEXT(PY_MINOR_VERSION) ";";

PyMODINIT_FUNC PyInit_adsa_marshal() { return PyModule_Create(&module); }
