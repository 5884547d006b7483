// fast_cache.cpp -- native argument marshalling of the block cache's calls
// (cache.py), by the rules of fast.cpp: what it does not take, every error
// included, returns NotImplemented before any work, and the Python path runs.
#include "marshal.h"

namespace attn_py {
namespace {

using plan_t = int (*)(const attn_cache_plan_desc*);
using append_t = int (*)(const void*, const void*, const attn_cache*, const attn_cache_append_desc*);
using fwd_t = int (*)(const void*, void*, float*, const attn_cache*, const attn_cache_fwd_desc*, void*, int64_t);
using bytes_t = int64_t (*)(const attn_cache*, const attn_cache_fwd_desc*);
plan_t g_plan = nullptr;
append_t g_append = nullptr;
fwd_t g_fwd = nullptr;
bytes_t g_bytes = nullptr;

// A plain contiguous vector of `n` entries (any number where n < 0) on `dev`.
bool vector_of(PyObject* o, at::ScalarType type, const at::Device& dev, int64_t n, at::Tensor* t)
{
    return plain(o, t) && t->scalar_type() == type && t->device() == dev && t->dim() == 1 &&
           (n < 0 || t->size(0) == n) && t->is_contiguous() && t->numel() <= INT32_MAX;
}

bool table_of(PyObject* o, const at::Device* dev, int64_t batch, at::Tensor* t, int32_t* width, int64_t* stride)
{
    if (!plain(o, t) || t->scalar_type() != at::kInt || (dev && t->device() != *dev) || t->dim() != 2) return false;
    if (t->size(0) != batch || t->size(1) > INT32_MAX) return false;
    if (t->size(1) > 1 && t->stride(1) != 1) return false;
    if (batch > 1 && t->stride(0) < t->size(1)) return false;
    *width = (int32_t)t->size(1);
    *stride = batch > 1 ? t->stride(0) : t->size(1);
    return true;
}

bool dtype_of(const at::Tensor& t, int32_t* dtype)
{
    const auto s = t.scalar_type();
    *dtype = s == at::kBFloat16 ? ATTN_BF16 : ATTN_FP32;
    return s == at::kBFloat16 || s == at::kFloat;
}

// The pool of a KVCache (a tuple of four tensors).
bool pool_of(PyObject* o, at::Tensor t[4], attn_cache* c)
{
    if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 4) return false;
    for (int i = 0; i < 4; ++i)
        if (!plain(PyTuple_GET_ITEM(o, i), &t[i])) return false;
    const at::Tensor &k = t[0], &v = t[1];
    const auto type = k.scalar_type();
    if ((type != at::kFloat8_e4m3fn && type != at::kFloat8_e5m2) || k.dim() != 4) return false;
    const int64_t n = k.size(0), h = k.size(1), b = k.size(2), d = k.size(3);
    if (n > INT32_MAX || h > INT32_MAX || b > INT32_MAX || d > INT32_MAX) return false;
    if (v.scalar_type() != type || v.device() != k.device() || v.sizes() != at::IntArrayRef({n, h, d, b})) return false;
    for (int i = 0; i < 2; ++i)
        if (t[i].stride(3) != 1 || t[i].stride(2) != t[i].size(3) || broadcast(t[i])) return false;
    for (int i = 2; i < 4; ++i)
        if (t[i].scalar_type() != at::kFloat || t[i].device() != k.device() ||
            t[i].sizes() != at::IntArrayRef({n, h}) || (h > 1 && t[i].stride(1) != 1) || broadcast(t[i]))
            return false;
    c->struct_size = sizeof(*c);
    c->cache_dtype = type == at::kFloat8_e4m3fn ? ATTN_E4M3 : ATTN_E5M2;
    c->num_blocks = (int32_t)n;
    c->num_kv_heads = (int32_t)h;
    c->block_size = (int32_t)b;
    c->head_dim = (int32_t)d;
    c->k = k.data_ptr();
    c->v = v.data_ptr();
    c->k_scale = static_cast<float*>(t[2].data_ptr());
    c->v_scale = static_cast<float*>(t[3].data_ptr());
    if (n > 1) {
        c->stride_k_block = k.stride(0);
        c->stride_v_block = v.stride(0);
        c->stride_ks_block = t[2].stride(0);
        c->stride_vs_block = t[3].stride(0);
    }
    if (h > 1) {
        c->stride_k_head = k.stride(1);
        c->stride_v_head = v.stride(1);
    }
    return true;
}

void* stream_of(const at::Device& dev) { return c10::hip::getCurrentHIPStream(dev.index()).stream(); }

bool handled(int status) { return status == ATTN_OK || status == ATTN_ERR_LAUNCH; }

// A contiguous tensor of n entries in the storage of `base` (bytes), `at` bytes on.
at::Tensor part_of(const at::Tensor& base, int64_t at, int64_t n, const caffe2::TypeMeta& type)
{
    at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(base.storage()), base.key_set(), type);
    c10::TensorImpl* impl = t.unsafeGetTensorImpl();
    impl->set_storage_offset(at / (int64_t)type.itemsize());
    impl->set_sizes_contiguous({n});
    return t;
}

enum PlanArg { pCached, pNew, pTable, pFree, pNumFree, pBlock, pTotal, pArgs };

bool plan(PyObject* const* a, at::Tensor out[4], int* status)
{
    at::Tensor cached, fresh, table, free_blocks, num_free;
    attn_cache_plan_desc d = {};
    d.struct_size = sizeof(d);
    if (!plain(a[pCached], &cached) || cached.dim() != 1) return false;
    const at::Device dev = cached.device();
    const int64_t batch = cached.size(0);
    if (!vector_of(a[pCached], at::kInt, dev, -1, &cached) || !vector_of(a[pNew], at::kInt, dev, batch, &fresh) ||
        !table_of(a[pTable], &dev, batch, &table, &d.table_width, &d.stride_table) ||
        !vector_of(a[pFree], at::kInt, dev, -1, &free_blocks) || !vector_of(a[pNumFree], at::kInt, dev, 1, &num_free) ||
        !as_i32(a[pBlock], &d.block_size) || !as_int(a[pTotal], &d.total_new) || modes())
        return false;
    if (d.total_new < 0 || d.total_new > INT32_MAX) return false;
    const NoGil nogil;
    at::AutoDispatchBelowADInplaceOrView below;
    // one allocation for the four (each costs 0.8 us of 7.6 a call)
    const auto i32 = caffe2::TypeMeta::Make<int32_t>();
    const int64_t slots = 8 * d.total_new;
    const at::Tensor all = at::empty({slots + 4 * (2 * batch + 2)}, cached.options().dtype(at::kByte));
    out[0] = part_of(all, 0, d.total_new, caffe2::TypeMeta::Make<int64_t>());
    out[1] = part_of(all, slots, batch + 1, i32);
    out[2] = part_of(all, slots + 4 * (batch + 1), batch, i32);
    out[3] = part_of(all, slots + 4 * (2 * batch + 1), 1, i32);
    d.batch = (int32_t)batch;
    d.free_len = (int32_t)free_blocks.numel();
    d.cached_lens = cached.const_data_ptr<int32_t>();
    d.new_lens = fresh.const_data_ptr<int32_t>();
    d.block_tables = table.mutable_data_ptr<int32_t>();
    d.free_blocks = free_blocks.const_data_ptr<int32_t>();
    d.num_free = num_free.const_data_ptr<int32_t>();
    d.slots = out[0].mutable_data_ptr<int64_t>();
    d.cu_seqlens_q = out[1].mutable_data_ptr<int32_t>();
    d.seqlens_k = out[2].mutable_data_ptr<int32_t>();
    d.num_free_out = out[3].mutable_data_ptr<int32_t>();
    d.stream = stream_of(dev);
    const c10::DeviceGuard guard(dev);
    *status = g_plan(&d);
    return handled(*status);
}

enum AppendArg { aCache, aK, aV, aSlots, aArgs };

bool append(PyObject* const* a, int* status)
{
    at::Tensor pool[4], k, v, slots;
    attn_cache c = {};
    attn_cache_append_desc d = {};
    d.struct_size = sizeof(d);
    if (!pool_of(a[aCache], pool, &c) || !plain(a[aK], &k) || !plain(a[aV], &v) || modes()) return false;
    const at::Device dev = pool[0].device();
    if (!dtype_of(k, &d.dtype) || v.scalar_type() != k.scalar_type() || k.dim() != 3 || k.sizes() != v.sizes() ||
        k.size(1) != c.num_kv_heads || k.size(2) != c.head_dim)
        return false;
    for (const at::Tensor* t : {&k, &v})
        if (t->device() != dev || t->stride(2) != 1 || broadcast(*t)) return false;
    if (!vector_of(a[aSlots], at::kLong, dev, k.size(0), &slots)) return false;
    const bool many = k.size(0) > 1, heads = k.size(1) > 1;
    d.total_new = k.size(0);
    d.stride_k_h = heads ? k.stride(1) : 0;
    d.stride_v_h = heads ? v.stride(1) : 0;
    d.stride_k_s = many ? k.stride(0) : 0;
    d.stride_v_s = many ? v.stride(0) : 0;
    d.slots = slots.const_data_ptr<int64_t>();
    d.stream = stream_of(dev);
    const NoGil nogil;
    const c10::DeviceGuard guard(dev);
    *status = g_append(k.const_data_ptr(), v.const_data_ptr(), &c, &d);
    return handled(*status);
}

enum FwdArg {
    fQ, fCache, fTable, fLens, fCausal, fWindow, fSlopes, fSoftcap, fScale, fCuQ, fMaxQ, fMaxK, fOut, fLse,
    fReturnLse, fArgs
};

bool fwd(PyObject* const* a, at::Tensor* out, at::Tensor* lse, bool* with_lse, int* status)
{
    at::Tensor pool[4], q, table, lens, cu, slopes;
    attn_cache c = {};
    attn_cache_fwd_desc d = {};
    d.struct_size = sizeof(d);
    if (!plain(a[fQ], &q) || !pool_of(a[fCache], pool, &c) || modes()) return false;
    const at::Device dev = pool[0].device();
    const bool packed = a[fCuQ] != Py_None;
    const int64_t rank = packed ? 3 : 4;
    if (!dtype_of(q, &d.dtype) || q.dim() != rank || q.device() != dev || q.stride(rank - 1) != 1 || broadcast(q) ||
        q.size(rank - 1) != c.head_dim)
        return false;
    for (int64_t i = 0; i < rank; ++i)
        if (q.size(i) > INT32_MAX) return false;
    if (!vector_of(a[fLens], at::kInt, dev, -1, &lens)) return false;
    const int64_t batch = lens.size(0), hq = q.size(1);
    if (!table_of(a[fTable], &dev, batch, &table, &d.table_width, &d.stride_table)) return false;
    if (packed) {
        if (!vector_of(a[fCuQ], at::kInt, dev, batch + 1, &cu) || !as_i32(a[fMaxQ], &d.max_seqlen_q)) return false;
        d.cu_seqlens_q = cu.const_data_ptr<int32_t>();
        d.total_q = q.size(0);
    } else {
        if (q.size(0) != batch) return false;
        d.seqlen_q = (int32_t)q.size(2);
    }
    if (a[fMaxK] != Py_None) {
        if (!as_i32(a[fMaxK], &d.max_seqlen_k) || d.max_seqlen_k < 0) return false;
        if (d.max_seqlen_k == 0) d.max_seqlen_k = 1;
    }
    const int causal = PyObject_IsTrue(a[fCausal]), want_lse = PyObject_IsTrue(a[fReturnLse]);
    if (causal < 0 || want_lse < 0) {
        PyErr_Clear();
        return false;
    }
    d.window_left = d.window_right = -1;
    d.mask_kind = causal ? ATTN_MASK_CAUSAL : ATTN_MASK_NONE;
    if (a[fWindow] != Py_None) {
        d.mask_kind = ATTN_MASK_SLIDING_WINDOW;
        if (!PyTuple_CheckExact(a[fWindow]) || PyTuple_GET_SIZE(a[fWindow]) < 2 ||
            !as_i32(PyTuple_GET_ITEM(a[fWindow], 0), &d.window_left) ||
            !as_i32(PyTuple_GET_ITEM(a[fWindow], 1), &d.window_right))
            return false;
    }
    if (a[fScale] == Py_None)
        d.scale = (float)(1.0 / std::sqrt((double)c.head_dim));
    else if (!as_float(a[fScale], &d.scale))
        return false;
    if (!as_float(a[fSoftcap], &d.softcap)) return false;
    if (a[fSlopes] != Py_None) {
        if (!vector_of(a[fSlopes], at::kFloat, dev, hq, &slopes)) return false;
        d.alibi_slopes = slopes.const_data_ptr<float>();
    }
    if (a[fOut] != Py_None && (!plain(a[fOut], out) || out->scalar_type() != q.scalar_type() ||
                               out->sizes() != q.sizes() || out->device() != dev))
        return false;
    const at::DimVector shape = packed ? at::DimVector{hq, q.size(0)} : at::DimVector{q.size(0), hq, q.size(2)};
    if (a[fLse] != Py_None && (!plain(a[fLse], lse) || lse->scalar_type() != at::kFloat || !lse->is_contiguous() ||
                               lse->device() != dev || lse->sizes() != at::IntArrayRef(shape)))
        return false;
    *with_lse = want_lse;

    const NoGil nogil;
    at::AutoDispatchBelowADInplaceOrView below;
    if (!out->defined()) *out = at::empty_like(q);
    if (out->stride(rank - 1) != 1 || broadcast(*out)) return false;
    if (*with_lse && !lse->defined()) *lse = at::empty(shape, q.options().dtype(at::kFloat));
    auto strides = [&](const at::Tensor& t, int64_t* b, int64_t* h, int64_t* s) {
        const int64_t ss = packed ? 0 : 2;
        *b = !packed && t.size(0) > 1 ? t.stride(0) : 0;
        *h = t.size(1) > 1 ? t.stride(1) : 0;
        *s = t.size(ss) > 1 ? t.stride(ss) : 0;
    };
    strides(q, &d.stride_q_b, &d.stride_q_h, &d.stride_q_s);
    strides(*out, &d.stride_o_b, &d.stride_o_h, &d.stride_o_s);
    d.batch = (int32_t)batch;
    d.num_q_heads = (int32_t)hq;
    d.block_tables = table.const_data_ptr<int32_t>();
    d.seqlens_k = lens.const_data_ptr<int32_t>();
    d.stream = stream_of(dev);
    const int64_t bytes = g_bytes(&c, &d);
    if (bytes < 0) return false;
    at::Tensor ws;
    if (bytes > 0) {
        try {
            ws = at::empty({bytes}, q.options().dtype(at::kByte));
        } catch (const c10::OutOfMemoryError&) {  // computed without the split
        }
    }
    const c10::DeviceGuard guard(dev);
    *status = g_fwd(q.const_data_ptr(), out->mutable_data_ptr(),
                    lse->defined() ? lse->mutable_data_ptr<float>() : nullptr, &c, &d,
                    ws.defined() ? ws.mutable_data_ptr() : nullptr, ws.defined() ? bytes : 0);
    return handled(*status);
}

PyObject* wrong_count(const char* name, int want, Py_ssize_t got)
{
    PyErr_Format(PyExc_TypeError, "%s takes %d arguments, got %zd", name, want, got);
    return nullptr;
}

}  // namespace

PyObject* py_cache_plan(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != pArgs) return wrong_count("cache_plan", pArgs, n);
    try {
        at::Tensor out[4];
        int status = ATTN_OK;
        if (!g_plan || !plan(a, out, &status)) Py_RETURN_NOTIMPLEMENTED;
        if (status != ATTN_OK) return raise_status(status);
        PyObject* r = PyTuple_New(4);
        for (int i = 0; r && i < 4; ++i) {
            PyObject* t = THPVariable_Wrap(out[i]);
            if (!t) Py_CLEAR(r);
            else PyTuple_SET_ITEM(r, i, t);
        }
        return r;
    } catch (const std::exception&) {
        PyErr_Clear();
        Py_RETURN_NOTIMPLEMENTED;
    }
}

PyObject* py_cache_append(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != aArgs) return wrong_count("cache_append", aArgs, n);
    try {
        int status = ATTN_OK;
        if (!g_append || !append(a, &status)) Py_RETURN_NOTIMPLEMENTED;
        if (status != ATTN_OK) return raise_status(status);
        Py_RETURN_NONE;
    } catch (const std::exception&) {
        PyErr_Clear();
        Py_RETURN_NOTIMPLEMENTED;
    }
}

PyObject* py_cache_fwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != fArgs) return wrong_count("cache_fwd", fArgs, n);
    try {
        at::Tensor out, lse;
        bool with_lse = false;
        int status = ATTN_OK;
        if (!g_fwd || !fwd(a, &out, &lse, &with_lse, &status)) Py_RETURN_NOTIMPLEMENTED;
        if (status != ATTN_OK) return raise_status(status);
        return outputs(a[fOut], out, a[fLse], lse, with_lse);
    } catch (const std::exception&) {
        PyErr_Clear();
        Py_RETURN_NOTIMPLEMENTED;
    }
}

// bind_cache(addresses of attn_cache_plan, _append, _fwd and _workspace_bytes)
PyObject* py_bind_cache(PyObject*, PyObject* args)
{
    unsigned long long p, a, f, w;
    if (!PyArg_ParseTuple(args, "KKKK", &p, &a, &f, &w)) return nullptr;
    g_plan = reinterpret_cast<plan_t>((uintptr_t)p);
    g_append = reinterpret_cast<append_t>((uintptr_t)a);
    g_fwd = reinterpret_cast<fwd_t>((uintptr_t)f);
    g_bytes = reinterpret_cast<bytes_t>((uintptr_t)w);
    Py_RETURN_NONE;
}

}  // namespace attn_py
