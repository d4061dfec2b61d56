// Native half of the Python binding: the calls of a training loop, whose Python cost (checks, allocation of
// the outputs, marshalling of pointers) was a multiple of their time on the GPU for small batches.
//
// Every function here takes the arguments of the Python function of the same name, serves the plain case
// (exact torch tensors of the expected types, ordinary integers) and returns None for anything else, which the
// Python function then handles, or refuses, itself; so also where the library's own allocations find no memory.
// Errors of the C library become TaserError. The library's entry points come in as addresses (bind), so this file
// links against torch only.
//
// One mini-batch of 1800 roots with edge rows: 24.6 us a call when marshalled in Python, 11.5 us so, of which the
// two kernel launches take about 6; its kernels take 9.
#include <Python.h>

#include <cmath>

#include <ATen/ATen.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "taser.h"

namespace {

struct Api {
    decltype(&taser_sample_temporal) sample_temporal;
    decltype(&taser_sample_temporal_rows) sample_temporal_rows;
    decltype(&taser_gather_features) gather_features;
    decltype(&taser_candidate_encodings) candidate_encodings;
    decltype(&taser_select_weighted) select_weighted;
    decltype(&taser_cache_lookup) cache_lookup;
    decltype(&taser_selector_draw) selector_draw;
    decltype(&taser_selector_update) selector_update;
    decltype(&taser_selector_scores) selector_scores;
    decltype(&taser_cross_attention_bytes) cross_attention_bytes;
    decltype(&taser_cross_attention) cross_attention;
    decltype(&taser_cross_attention_grad) cross_attention_grad;
    decltype(&taser_relative_bias_bytes) relative_bias_bytes;
    decltype(&taser_relative_bias) relative_bias;
    decltype(&taser_relative_bias_grad) relative_bias_grad;
    decltype(&taser_policy_loss) policy_loss;
    decltype(&taser_last_error) last_error;
} api;
PyObject* error_class = nullptr;                                  // TaserError
PyObject *s_nbr, *s_eid, *s_ts, *s_count, *s_cuda_stream;         // interned names

struct Ref {   // an owned reference
    PyObject* p;
    explicit Ref(PyObject* o = nullptr) : p(o) {}
    ~Ref() { Py_XDECREF(p); }
    Ref(const Ref&) = delete;
    Ref& operator=(const Ref&) = delete;
    PyObject* release() { PyObject* o = p; p = nullptr; return o; }
};

// ---- arguments: false means "not the plain case" ------------------------------------
bool get_int(PyObject* o, int64_t low, int64_t high, int64_t* v) {
    if (!PyLong_CheckExact(o)) return false;
    int overflow = 0;
    *v = PyLong_AsLongLongAndOverflow(o, &overflow);
    return !overflow && *v >= low && *v <= high;
}
bool get_u64(PyObject* o, uint64_t* v) {   // modulo 2^64, as a C integer argument takes it
    if (!PyLong_CheckExact(o)) return false;
    *v = PyLong_AsUnsignedLongLongMask(o);
    return true;
}
bool get_handle(PyObject* o, void** p) {
    if (!PyLong_CheckExact(o)) return false;
    *p = PyLong_AsVoidPtr(o);
    return *p != nullptr;
}
const at::Tensor* plain(PyObject* o) { return THPVariable_CheckExact(o) ? &THPVariable_Unpack(o) : nullptr; }
const at::Tensor* device_array(PyObject* o, at::ScalarType type) {
    const at::Tensor* t = plain(o);
    return t && t->scalar_type() == type && t->is_cuda() && t->layout() == at::kStrided && t->is_contiguous() ? t : nullptr;
}
const at::Tensor* device_table(PyObject* o) {
    const at::Tensor* t = plain(o);
    return t && t->is_cuda() && t->layout() == at::kStrided && t->dim() == 2 && t->stride(1) == 1 ? t : nullptr;
}
bool get_stream(PyObject* o, void** stream) {
    if (o == Py_None) {
        *stream = c10::hip::getCurrentHIPStream().stream();
        return true;
    }
    Ref value(PyObject_GetAttr(o, s_cuda_stream));
    if (!value.p || !PyLong_CheckExact(value.p)) {
        PyErr_Clear();
        return false;
    }
    *stream = PyLong_AsVoidPtr(value.p);
    return true;
}

PyObject* not_plain() { Py_RETURN_NONE; }

PyObject* raise(int rc) {
    Ref e(PyObject_CallFunction(error_class, "is", rc, api.last_error()));
    if (e.p) PyErr_SetObject(error_class, e.p);
    return nullptr;
}

at::Tensor make(at::IntArrayRef size, at::ScalarType type, at::Device device) {
    return at::empty(size, at::TensorOptions().dtype(type).device(device));
}

bool put(PyObject* dict, PyObject* name, const at::Tensor& t) {
    Ref o(THPVariable_Wrap(t));
    return o.p && PyDict_SetItem(dict, name, o.p) == 0;
}

// ---- sample_temporal, sample_temporal_rows ---------------------------------------------
// (handle, roots, times, k, hops, policy, seed, m, edge_weight, stream[, table, row_elems])
PyObject* sample(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    if (n_args != 10 && n_args != 12) return not_plain();
    void *handle, *stream;
    int64_t k, hops, policy, m;
    uint64_t seed;
    const at::Tensor *roots = device_array(a[1], at::kInt), *times = device_array(a[2], at::kLong), *weight = nullptr, *table = nullptr;
    if (!get_handle(a[0], &handle) || !roots || !times || !get_int(a[3], 1, TASER_MAX_K, &k) || !get_int(a[4], 1, TASER_MAX_HOPS, &hops) ||
        !get_int(a[5], 0, 3, &policy) || !get_u64(a[6], &seed) || !get_int(a[7], INT32_MIN, INT32_MAX, &m))
        return not_plain();
    if (a[8] != Py_None && !(weight = device_array(a[8], at::kInt))) return not_plain();
    if (!get_stream(a[9], &stream)) return not_plain();
    const int64_t n = roots->numel();
    if (times->numel() != n) return not_plain();
    int64_t slots = n;
    for (int64_t h = 0; h < hops; ++h)
        if ((slots *= k) >= (int64_t)1 << 31) return not_plain();
    int64_t elems = 0, size = 0;
    if (n_args == 12) {
        if (!(table = device_table(a[10]))) return not_plain();
        size = table->element_size();
        elems = table->size(1);
        if (a[11] != Py_None && !get_int(a[11], 1, INT32_MAX, &elems)) return not_plain();
        if (elems * size > INT32_MAX) return not_plain();
    }
    taser_hop_out out[TASER_MAX_HOPS];
    void* rows_out[TASER_MAX_HOPS];
    Ref list(PyList_New(hops)), rows(table ? PyList_New(hops) : nullptr);
    if (!list.p || (table && !rows.p)) return nullptr;
    int64_t r = n;
    for (int64_t h = 0; h < hops; ++h) {
        const at::Device device = roots->device();
        const at::Tensor nbr = make({r, k}, at::kInt, device), eid = make({r, k}, at::kInt, device), ts = make({r, k}, at::kLong, device),
                         count = make({r}, at::kInt, device);
        out[h] = taser_hop_out{static_cast<int32_t*>(nbr.data_ptr()), static_cast<int32_t*>(eid.data_ptr()),
                               static_cast<int64_t*>(ts.data_ptr()), static_cast<int32_t*>(count.data_ptr())};
        PyObject* d = PyDict_New();
        if (!d) return nullptr;
        PyList_SET_ITEM(list.p, h, d);
        if (!put(d, s_nbr, nbr) || !put(d, s_eid, eid) || !put(d, s_ts, ts) || !put(d, s_count, count)) return nullptr;
        r *= k;
        if (table) {
            const at::Tensor t = make({r, elems}, table->scalar_type(), table->device());
            rows_out[h] = t.data_ptr();
            PyObject* o = THPVariable_Wrap(t);
            if (!o) return nullptr;
            PyList_SET_ITEM(rows.p, h, o);
        }
    }
    const int32_t* p_roots = static_cast<const int32_t*>(roots->data_ptr());
    const int64_t* p_times = static_cast<const int64_t*>(times->data_ptr());
    const uint32_t* p_weight = weight ? static_cast<const uint32_t*>(weight->data_ptr()) : nullptr;
    const void* p_table = table ? table->data_ptr() : nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    if (table)
        rc = api.sample_temporal_rows(static_cast<taser_tcsr*>(handle), p_roots, p_times, n, (int32_t)k, (int32_t)hops, (int32_t)policy, seed,
                                      (int32_t)m, p_weight, p_table, table->size(0), (int32_t)(elems * size), table->stride(0) * size, out,
                                      rows_out, stream);
    else
        rc = api.sample_temporal(static_cast<taser_tcsr*>(handle), p_roots, p_times, n, (int32_t)k, (int32_t)hops, (int32_t)policy, seed,
                                 (int32_t)m, p_weight, out, stream);
    Py_END_ALLOW_THREADS
    if (rc == TASER_E_OOM) return not_plain();
    if (rc != TASER_OK) return raise(rc);
    if (!table) return list.release();
    return PyTuple_Pack(2, list.p, rows.p);
    END_HANDLE_TH_ERRORS
}

// ---- gather_features(table, ids, out, row_elems, stream) --------------------------------
PyObject* gather(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    void* stream;
    const at::Tensor *table = n_args == 5 ? device_table(a[0]) : nullptr, *ids = table ? device_array(a[1], at::kInt) : nullptr;
    if (!ids) return not_plain();
    int64_t elems = table->size(1);
    const int64_t size = table->element_size(), n = ids->numel();
    if (a[3] != Py_None && !get_int(a[3], 1, INT32_MAX, &elems)) return not_plain();
    if (elems * size > INT32_MAX || !get_stream(a[4], &stream)) return not_plain();
    at::Tensor made;
    const at::Tensor* out = &made;
    if (a[2] == Py_None) made = make({n, elems}, table->scalar_type(), table->device());
    else if (!(out = device_array(a[2], table->scalar_type())) || out->numel() < n * elems) return not_plain();
    const void *p_table = table->data_ptr(), *p_ids = ids->data_ptr();
    void* p_out = out->data_ptr();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = api.gather_features(p_table, table->size(0), (int32_t)(elems * size), table->stride(0) * size, static_cast<const int32_t*>(p_ids), n,
                             p_out, stream);
    Py_END_ALLOW_THREADS
    if (rc != TASER_OK) return raise(rc);
    if (a[2] == Py_None) return THPVariable_Wrap(made);
    Py_INCREF(a[2]);
    return a[2];
    END_HANDLE_TH_ERRORS
}

// ---- candidate_encodings(nbr, count, want_identity, stream) -----------------------------
PyObject* encodings(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    void* stream;
    const at::Tensor *nbr = n_args == 4 ? device_array(a[0], at::kInt) : nullptr, *count = nbr ? device_array(a[1], at::kInt) : nullptr;
    if (!count || nbr->dim() != 2 || count->numel() != nbr->size(0) || !PyBool_Check(a[2]) || !get_stream(a[3], &stream)) return not_plain();
    const int64_t n = nbr->size(0), m = nbr->size(1);
    if (m < 1 || m > TASER_MAX_M) return not_plain();
    const at::Tensor freq = make({n, m}, at::kInt, nbr->device());
    at::Tensor identity;
    if (a[2] == Py_True) identity = make({n, m, m}, at::kByte, nbr->device());
    const void *p_nbr = nbr->data_ptr(), *p_count = count->data_ptr();
    void *p_freq = freq.data_ptr(), *p_identity = a[2] == Py_True ? identity.data_ptr() : nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = api.candidate_encodings(static_cast<const int32_t*>(p_nbr), static_cast<const int32_t*>(p_count), n, (int32_t)m,
                                 static_cast<int32_t*>(p_freq), static_cast<uint8_t*>(p_identity), stream);
    Py_END_ALLOW_THREADS
    if (rc != TASER_OK) return raise(rc);
    Ref f(THPVariable_Wrap(freq)), i(a[2] == Py_True ? THPVariable_Wrap(identity) : nullptr);
    if (!f.p || (a[2] == Py_True && !i.p)) return nullptr;
    return PyTuple_Pack(2, f.p, i.p ? i.p : Py_None);
    END_HANDLE_TH_ERRORS
}

// ---- select_weighted(weight, count, k, seed, hop, candidates, stream) --------------------
PyObject* select(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    void* stream;
    int64_t k, hop;
    uint64_t seed;
    const at::Tensor *weight = n_args == 7 ? device_array(a[0], at::kInt) : nullptr, *count = weight ? device_array(a[1], at::kInt) : nullptr;
    if (!count || weight->dim() != 2 || count->numel() != weight->size(0) || !get_int(a[2], 1, TASER_MAX_K, &k) || !get_u64(a[3], &seed) ||
        !get_int(a[4], 0, UINT32_MAX, &hop) || !get_stream(a[6], &stream))
        return not_plain();
    const int64_t n = weight->size(0), m = weight->size(1);
    if (m < 1 || m > TASER_MAX_M || n * (m > k ? m : k) >= (int64_t)1 << 31) return not_plain();
    taser_hop_out from = {}, to = {};
    const bool with = a[5] != Py_None;
    if (with) {
        if (!PyDict_CheckExact(a[5])) return not_plain();
        PyObject *o_nbr = PyDict_GetItem(a[5], s_nbr), *o_eid = PyDict_GetItem(a[5], s_eid), *o_ts = PyDict_GetItem(a[5], s_ts);
        if (!o_nbr || !o_eid || !o_ts) return not_plain();
        const at::Tensor *nbr = device_array(o_nbr, at::kInt), *eid = device_array(o_eid, at::kInt), *ts = device_array(o_ts, at::kLong);
        if (!nbr || !eid || !ts || nbr->numel() != n * m || eid->numel() != n * m || ts->numel() != n * m) return not_plain();
        from = taser_hop_out{static_cast<int32_t*>(nbr->data_ptr()), static_cast<int32_t*>(eid->data_ptr()),
                             static_cast<int64_t*>(ts->data_ptr()), nullptr};
    }
    const at::Device device = weight->device();
    const at::Tensor sel = make({n, k}, at::kInt, device), out_count = make({n}, at::kInt, device);
    Ref kept, o_sel(THPVariable_Wrap(sel)), o_count(THPVariable_Wrap(out_count));
    if (!o_sel.p || !o_count.p) return nullptr;
    if (with) {
        const at::Tensor nbr = make({n, k}, at::kInt, device), eid = make({n, k}, at::kInt, device), ts = make({n, k}, at::kLong, device);
        to = taser_hop_out{static_cast<int32_t*>(nbr.data_ptr()), static_cast<int32_t*>(eid.data_ptr()),
                           static_cast<int64_t*>(ts.data_ptr()), nullptr};
        kept.p = PyDict_New();
        if (!kept.p || !put(kept.p, s_nbr, nbr) || !put(kept.p, s_eid, eid) || !put(kept.p, s_ts, ts) ||
            PyDict_SetItem(kept.p, s_count, o_count.p) != 0)
            return nullptr;
    }
    const void *p_weight = weight->data_ptr(), *p_count = count->data_ptr();
    void *p_sel = sel.data_ptr(), *p_out_count = out_count.data_ptr();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = api.select_weighted(static_cast<const uint32_t*>(p_weight), static_cast<const int32_t*>(p_count), n, (int32_t)m, (int32_t)k, seed,
                             (uint32_t)hop, static_cast<int32_t*>(p_sel), static_cast<int32_t*>(p_out_count), with ? &from : nullptr,
                             with ? &to : nullptr, stream);
    Py_END_ALLOW_THREADS
    if (rc != TASER_OK) return raise(rc);
    return PyTuple_Pack(3, o_sel.p, o_count.p, kept.p ? kept.p : Py_None);
    END_HANDLE_TH_ERRORS
}

// ---- cache_lookup(handle, host_table, row_elems, ids, out, hit_miss, stream) --------------
PyObject* lookup(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    void *handle, *stream;
    int64_t elems;
    const at::Tensor *host = n_args == 7 ? plain(a[1]) : nullptr, *ids = host ? device_array(a[3], at::kInt) : nullptr, *hit_miss = nullptr;
    if (!ids || !get_handle(a[0], &handle) || !get_int(a[2], 1, INT32_MAX, &elems) || !get_stream(a[6], &stream)) return not_plain();
    if (a[5] != Py_None && !(hit_miss = device_array(a[5], at::kLong))) return not_plain();
    const int64_t n = ids->numel();
    at::Tensor made;
    const at::Tensor* out = &made;
    if (a[4] == Py_None) made = make({n, elems}, host->scalar_type(), ids->device());
    else if (!(out = device_array(a[4], host->scalar_type())) || out->numel() < n * elems) return not_plain();
    const void* p_ids = ids->data_ptr();
    void *p_out = out->data_ptr(), *p_hit_miss = hit_miss ? hit_miss->data_ptr() : nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = api.cache_lookup(static_cast<taser_cache*>(handle), static_cast<const int32_t*>(p_ids), n, p_out, static_cast<uint64_t*>(p_hit_miss),
                          stream);
    Py_END_ALLOW_THREADS
    if (rc == TASER_E_OOM) return not_plain();
    if (rc != TASER_OK) return raise(rc);
    if (a[4] == Py_None) return THPVariable_Wrap(made);
    Py_INCREF(a[4]);
    return a[4];
    END_HANDLE_TH_ERRORS
}

// ---- selector_draw(handle, b, seed, iteration, out, stream) --------------------------------
PyObject* draw(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    void *handle, *stream;
    int64_t b;
    uint64_t seed, iteration;
    if (n_args != 6 || !get_handle(a[0], &handle) || !get_int(a[1], 0, INT32_MAX, &b) || !get_u64(a[2], &seed) || !get_u64(a[3], &iteration) ||
        !get_stream(a[5], &stream))
        return not_plain();
    at::Tensor made;
    const at::Tensor* out = &made;
    if (a[4] == Py_None) made = make({b}, at::kInt, at::Device(at::kCUDA));
    else if (!(out = device_array(a[4], at::kInt)) || out->numel() < b) return not_plain();
    void* p_out = out->data_ptr();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = api.selector_draw(static_cast<taser_selector*>(handle), b, seed, iteration, static_cast<int32_t*>(p_out), stream);
    Py_END_ALLOW_THREADS
    if (rc != TASER_OK) return raise(rc);
    if (a[4] == Py_None) return THPVariable_Wrap(made);
    Py_INCREF(a[4]);
    return a[4];
    END_HANDLE_TH_ERRORS
}

// ---- selector_update(handle, batch, new_scores, stream) -> True -----------------------------
PyObject* update(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    void *handle, *stream;
    const at::Tensor *batch = n_args == 4 ? device_array(a[1], at::kInt) : nullptr, *scores = batch ? device_array(a[2], at::kInt) : nullptr;
    if (!scores || !get_handle(a[0], &handle) || batch->numel() != scores->numel() || !get_stream(a[3], &stream)) return not_plain();
    const void *p_batch = batch->data_ptr(), *p_scores = scores->data_ptr();
    const int64_t b = batch->numel();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = api.selector_update(static_cast<taser_selector*>(handle), static_cast<const int32_t*>(p_batch), static_cast<const uint32_t*>(p_scores),
                             b, stream);
    Py_END_ALLOW_THREADS
    if (rc != TASER_OK) return raise(rc);
    Py_RETURN_TRUE;
    END_HANDLE_TH_ERRORS
}

// ---- selector_scores(handle, n, stream) -> tensor (without the total) ------------------------
PyObject* scores(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    void *handle, *stream;
    int64_t n;
    if (n_args != 3 || !get_handle(a[0], &handle) || !get_int(a[1], 1, INT32_MAX, &n) || !get_stream(a[2], &stream)) return not_plain();
    const at::Tensor out = make({n}, at::kInt, at::Device(at::kCUDA));
    void* p_out = out.data_ptr();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = api.selector_scores(static_cast<taser_selector*>(handle), static_cast<uint32_t*>(p_out), nullptr, stream);
    Py_END_ALLOW_THREADS
    if (rc != TASER_OK) return raise(rc);
    return THPVariable_Wrap(out);
    END_HANDLE_TH_ERRORS
}

// ---- attention, the bias by distance, the policy loss ------------------------------------------
bool element_type(at::ScalarType t, int32_t* type) {
    *type = t == at::kFloat ? TASER_F32 : t == at::kHalf ? TASER_F16 : TASER_BF16;
    return t == at::kFloat || t == at::kHalf || t == at::kBFloat16;
}
// A device tensor of `dims` dimensions whose last one is adjacent in memory.
const at::Tensor* strided(PyObject* o, int64_t dims, at::ScalarType type) {
    const at::Tensor* t = plain(o);
    return t && t->scalar_type() == type && t->is_cuda() && t->layout() == at::kStrided && t->dim() == dims && (t->size(dims - 1) <= 1 || t->stride(dims - 1) == 1) ? t : nullptr;
}
bool get_float(PyObject* o, float* v) {
    if (!PyFloat_CheckExact(o)) return false;
    *v = (float)PyFloat_AS_DOUBLE(o);
    return true;
}
bool positions(const at::Tensor* t, int64_t batch, int64_t n, const int64_t** p, int64_t* stride) {
    if (!t || t->size(1) != n || (t->size(0) != 1 && t->size(0) != batch)) return false;
    *p = static_cast<const int64_t*>(t->data_ptr());
    *stride = t->size(0) > 1 ? t->stride(0) : 0;
    return true;
}

// (q, k, v, lengths, mask, bias, scale) -> the argument block
bool attention_block(PyObject* const* o, taser_attention* a, const at::Tensor** query) {
    const at::Tensor* q = plain(o[0]);
    *a = taser_attention{};
    if (!q || !element_type(q->scalar_type(), &a->type) || !(q = strided(o[0], 4, q->scalar_type()))) return false;
    const at::Tensor *k = strided(o[1], 4, q->scalar_type()), *v = k ? strided(o[2], 4, q->scalar_type()) : nullptr;
    if (!v || k->sizes() != v->sizes() || k->size(0) != q->size(0) || k->size(3) != q->size(3)) return false;
    if (q->size(2) > 65536 || k->size(2) > 65536 || q->size(3) < 1 || q->size(3) > TASER_MAX_HEAD_DIM) return false;
    a->batch = q->size(0);
    a->queries = q->size(1);
    a->heads = (int32_t)q->size(2);
    a->head_dim = (int32_t)q->size(3);
    a->keys = k->size(1);
    a->kv_heads = (int32_t)k->size(2);
    a->q = q->data_ptr();
    a->k = k->data_ptr();
    a->v = v->data_ptr();
    for (int i = 0; i < 3; ++i) {
        a->q_strides[i] = q->stride(i);
        a->k_strides[i] = k->stride(i);
        a->v_strides[i] = v->stride(i);
    }
    if (o[3] != Py_None) {
        const at::Tensor* t = device_array(o[3], at::kInt);
        if (!t || t->numel() != a->batch) return false;
        a->lengths = static_cast<const int32_t*>(t->data_ptr());
    }
    if (o[4] != Py_None) {
        const at::Tensor* t = strided(o[4], 2, at::kBool);
        if (!t || t->size(0) != a->batch || t->size(1) != a->keys) return false;
        a->mask = static_cast<const uint8_t*>(t->data_ptr());
        a->mask_stride = t->stride(0);
    }
    if (o[5] != Py_None) {
        if (!PyTuple_CheckExact(o[5]) || PyTuple_GET_SIZE(o[5]) != 4) return false;
        const at::Tensor *table = device_array(PyTuple_GET_ITEM(o[5], 0), q->scalar_type()), *bounds = device_array(PyTuple_GET_ITEM(o[5], 1), at::kLong);
        if (!table || !bounds || table->dim() != 2 || table->size(0) != a->heads || bounds->numel() != table->size(1) - 1 || table->size(1) > TASER_MAX_BUCKETS) return false;
        if (!positions(strided(PyTuple_GET_ITEM(o[5], 2), 2, at::kLong), a->batch, a->queries, &a->query_pos, &a->query_pos_stride) ||
            !positions(strided(PyTuple_GET_ITEM(o[5], 3), 2, at::kLong), a->batch, a->keys, &a->key_pos, &a->key_pos_stride))
            return false;
        a->buckets = (int32_t)table->size(1);
        a->bias_table = table->data_ptr();
        a->bounds = static_cast<const int64_t*>(bounds->data_ptr());
    }
    if (o[6] == Py_None) a->scale = (float)(1.0 / std::sqrt((double)a->head_dim));
    else if (!get_float(o[6], &a->scale)) return false;
    *query = q;
    return true;
}
at::Tensor scratch(uint64_t bytes, const at::Tensor& like) { return bytes ? make({(int64_t)bytes}, at::kByte, like.device()) : at::Tensor(); }

// (q, k, v, lengths, mask, bias, scale, want_stats), on torch's current stream
PyObject* attention(PyObject*, PyObject* const* o, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    taser_attention a;
    const at::Tensor* q;
    void* stream;
    uint64_t bytes = 0;
    if (n_args != 8 || !PyBool_Check(o[7]) || !attention_block(o, &a, &q) || !get_stream(Py_None, &stream)) return not_plain();
    if (const int rc = api.cross_attention_bytes(&a, &bytes, nullptr)) return raise(rc);
    const at::Tensor out = make(q->sizes(), q->scalar_type(), q->device()), work = scratch(bytes, *q);
    at::Tensor stats;
    if (o[7] == Py_True) stats = make({a.batch, a.queries, a.heads, TASER_ATTENTION_STATS(a.type, a.head_dim)}, at::kFloat, q->device());
    void *p_out = out.data_ptr(), *p_stats = stats.defined() ? stats.data_ptr() : nullptr, *p_work = bytes ? work.data_ptr() : nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = api.cross_attention(&a, p_out, static_cast<float*>(p_stats), p_work, bytes, stream);
    Py_END_ALLOW_THREADS
    if (rc != TASER_OK) return raise(rc);
    if (o[7] != Py_True) return THPVariable_Wrap(out);
    Ref x(THPVariable_Wrap(out)), y(THPVariable_Wrap(stats));
    return x.p && y.p ? PyTuple_Pack(2, x.p, y.p) : nullptr;
    END_HANDLE_TH_ERRORS
}

// (dout, q, k, v, out, stats, lengths, mask, bias, scale), on torch's current stream
PyObject* attention_grad(PyObject*, PyObject* const* o, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    taser_attention a;
    const at::Tensor* q;
    void* stream;
    uint64_t bytes = 0;
    if (n_args != 10) return not_plain();
    PyObject* const block[7] = {o[1], o[2], o[3], o[6], o[7], o[8], o[9]};
    if (!attention_block(block, &a, &q) || !get_stream(Py_None, &stream)) return not_plain();
    const at::Tensor *dout = device_array(o[0], q->scalar_type()), *out = device_array(o[4], q->scalar_type()), *stats = device_array(o[5], at::kFloat);
    if (!dout || !out || !stats || dout->sizes() != q->sizes() || out->sizes() != q->sizes() || stats->sizes() != at::IntArrayRef({a.batch, a.queries, a.heads, TASER_ATTENTION_STATS(a.type, a.head_dim)}))
        return not_plain();
    if (const int rc = api.cross_attention_bytes(&a, nullptr, &bytes)) return raise(rc);
    const at::IntArrayRef states = plain(o[2])->sizes();
    const at::Tensor dq = make(q->sizes(), q->scalar_type(), q->device()), dk = make(states, q->scalar_type(), q->device()), dv = make(states, q->scalar_type(), q->device()),
                     work = scratch(bytes, *q);
    at::Tensor dtable;
    if (a.bias_table) dtable = make({a.heads, a.buckets}, q->scalar_type(), q->device());
    const void *p_out = out->data_ptr(), *p_stats = stats->data_ptr(), *p_dout = dout->data_ptr();
    void *p_dq = dq.data_ptr(), *p_dk = dk.data_ptr(), *p_dv = dv.data_ptr(), *p_dtable = dtable.defined() ? dtable.data_ptr() : nullptr, *p_work = bytes ? work.data_ptr() : nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = api.cross_attention_grad(&a, p_out, static_cast<const float*>(p_stats), p_dout, p_dq, p_dk, p_dv, p_dtable, p_work, bytes, stream);
    Py_END_ALLOW_THREADS
    if (rc != TASER_OK) return raise(rc);
    Ref x(THPVariable_Wrap(dq)), y(THPVariable_Wrap(dk)), z(THPVariable_Wrap(dv)), t(dtable.defined() ? THPVariable_Wrap(dtable) : nullptr);
    if (!x.p || !y.p || !z.p || (dtable.defined() && !t.p)) return nullptr;
    return PyTuple_Pack(4, x.p, y.p, z.p, t.p ? t.p : Py_None);
    END_HANDLE_TH_ERRORS
}

// (bounds, query positions, key positions) of a bias over `batch` entries (-1: the larger of the positions')
bool distance_block(PyObject* const* o, int64_t batch, taser_distances* d) {
    const at::Tensor *bounds = device_array(o[0], at::kLong), *from = strided(o[1], 2, at::kLong), *to = strided(o[2], 2, at::kLong);
    if (!bounds || !from || !to || bounds->numel() >= TASER_MAX_BUCKETS) return false;
    d->batch = batch >= 0 ? batch : (from->size(0) > to->size(0) ? from->size(0) : to->size(0));
    d->queries = from->size(1);
    d->keys = to->size(1);
    d->buckets = (int32_t)bounds->numel() + 1;
    d->bounds = static_cast<const int64_t*>(bounds->data_ptr());
    return positions(from, d->batch, d->queries, &d->query_pos, &d->query_pos_stride) && positions(to, d->batch, d->keys, &d->key_pos, &d->key_pos_stride);
}

// (table, bounds, query positions, key positions), on torch's current stream
PyObject* bias(PyObject*, PyObject* const* o, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    taser_distances d = {};
    void* stream;
    const at::Tensor* table = n_args == 4 ? plain(o[0]) : nullptr;
    if (!table || !element_type(table->scalar_type(), &d.type) || !(table = device_array(o[0], table->scalar_type())) || table->dim() != 2 || table->size(0) > 65535 ||
        !distance_block(o + 1, -1, &d) || table->size(1) != d.buckets || !get_stream(Py_None, &stream))
        return not_plain();
    d.heads = (int32_t)table->size(0);
    const at::Tensor out = make({d.batch, d.heads, d.queries, d.keys}, table->scalar_type(), table->device());
    const void* p_table = table->data_ptr();
    void* p_out = out.data_ptr();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = api.relative_bias(&d, p_table, p_out, stream);
    Py_END_ALLOW_THREADS
    if (rc != TASER_OK) return raise(rc);
    return THPVariable_Wrap(out);
    END_HANDLE_TH_ERRORS
}

// (dbias, bounds, query positions, key positions), on torch's current stream
PyObject* bias_grad(PyObject*, PyObject* const* o, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    taser_distances d = {};
    void* stream;
    uint64_t bytes = 0;
    const at::Tensor* dbias = n_args == 4 ? plain(o[0]) : nullptr;
    if (!dbias || !element_type(dbias->scalar_type(), &d.type) || !(dbias = strided(o[0], 4, dbias->scalar_type())) || dbias->size(1) > 65535 ||
        !distance_block(o + 1, dbias->size(0), &d) || dbias->size(2) != d.queries || dbias->size(3) != d.keys || !get_stream(Py_None, &stream))
        return not_plain();
    d.heads = (int32_t)dbias->size(1);
    if (const int rc = api.relative_bias_bytes(&d, &bytes)) return raise(rc);
    const at::Tensor out = make({d.heads, d.buckets}, dbias->scalar_type(), dbias->device()), work = scratch(bytes, *dbias);
    const int64_t strides[3] = {dbias->stride(0), dbias->stride(1), dbias->stride(2)};
    const void* p_dbias = dbias->data_ptr();
    void *p_out = out.data_ptr(), *p_work = bytes ? work.data_ptr() : nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = api.relative_bias_grad(&d, p_dbias, strides, p_out, p_work, bytes, stream);
    Py_END_ALLOW_THREADS
    if (rc != TASER_OK) return raise(rc);
    return THPVariable_Wrap(out);
    END_HANDLE_TH_ERRORS
}

// (logits, actions, advantage, old_logp, ref_logp, count, weight, clip_low, clip_high, kl, want_grad, stream)
PyObject* policy(PyObject*, PyObject* const* o, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    taser_policy_batch p = {};
    void* stream;
    const at::Tensor* logits = n_args == 12 ? plain(o[0]) : nullptr;
    if (!logits || !element_type(logits->scalar_type(), &p.type) || !(logits = strided(o[0], 2, logits->scalar_type()))) return not_plain();
    const at::Tensor* actions = device_array(o[1], at::kInt);
    if (!actions || actions->dim() != 2 || actions->size(0) != logits->size(0) || actions->size(1) > TASER_MAX_PICKS) return not_plain();
    const float* given[4] = {};   // advantage, old_logp, ref_logp, weight
    PyObject* const of[4] = {o[2], o[3], o[4], o[6]};
    for (int i = 0; i < 4; ++i) {
        if (i && of[i] == Py_None) continue;
        const at::Tensor* t = device_array(of[i], at::kFloat);
        if (!t || t->sizes() != actions->sizes()) return not_plain();
        given[i] = static_cast<const float*>(t->data_ptr());
    }
    p.rows = logits->size(0);
    p.width = logits->size(1);
    p.logits_stride = p.rows > 1 ? logits->stride(0) : p.width;
    p.picks = (int32_t)actions->size(1);
    p.logits = logits->data_ptr();
    p.actions = static_cast<const int32_t*>(actions->data_ptr());
    p.advantage = given[0];
    p.old_logp = given[1];
    p.ref_logp = given[2];
    p.weight = given[3];
    if (o[5] != Py_None) {
        const at::Tensor* t = device_array(o[5], at::kInt);
        if (!t || t->numel() != p.rows) return not_plain();
        p.count = static_cast<const int32_t*>(t->data_ptr());
    }
    if (!get_float(o[7], &p.clip_low) || !get_float(o[8], &p.clip_high) || !get_float(o[9], &p.kl) || !PyBool_Check(o[10]) || !get_stream(o[11], &stream)) return not_plain();
    const at::Tensor loss = make(actions->sizes(), at::kFloat, logits->device()), logp = make(actions->sizes(), at::kFloat, logits->device());
    at::Tensor grad;
    if (o[10] == Py_True) grad = make({p.rows, p.width}, logits->scalar_type(), logits->device());
    void *p_loss = loss.data_ptr(), *p_logp = logp.data_ptr(), *p_grad = grad.defined() ? grad.data_ptr() : nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = api.policy_loss(&p, static_cast<float*>(p_loss), static_cast<float*>(p_logp), p_grad, stream);
    Py_END_ALLOW_THREADS
    if (rc != TASER_OK) return raise(rc);
    Ref x(THPVariable_Wrap(loss)), y(THPVariable_Wrap(logp)), z(grad.defined() ? THPVariable_Wrap(grad) : nullptr);
    if (!x.p || !y.p || (grad.defined() && !z.p)) return nullptr;
    return PyTuple_Pack(3, x.p, y.p, z.p ? z.p : Py_None);
    END_HANDLE_TH_ERRORS
}

// bind(TaserError, {entry point: address})
template <typename F> bool entry(PyObject* addresses, const char* name, F* to) {
    PyObject* o = PyDict_GetItemString(addresses, name);
    *to = o ? reinterpret_cast<F>(PyLong_AsVoidPtr(o)) : nullptr;
    if (*to) return true;
    if (!PyErr_Occurred()) PyErr_Format(PyExc_ValueError, "bind: no address for %s", name);
    return false;
}
PyObject* bind(PyObject*, PyObject* args) {
    PyObject *cls, *addresses;
    if (!PyArg_ParseTuple(args, "OO!", &cls, &PyDict_Type, &addresses)) return nullptr;
    Api to = {};
    if (!entry(addresses, "taser_sample_temporal", &to.sample_temporal) || !entry(addresses, "taser_sample_temporal_rows", &to.sample_temporal_rows) ||
        !entry(addresses, "taser_gather_features", &to.gather_features) || !entry(addresses, "taser_candidate_encodings", &to.candidate_encodings) ||
        !entry(addresses, "taser_select_weighted", &to.select_weighted) || !entry(addresses, "taser_cache_lookup", &to.cache_lookup) ||
        !entry(addresses, "taser_selector_draw", &to.selector_draw) || !entry(addresses, "taser_selector_update", &to.selector_update) ||
        !entry(addresses, "taser_selector_scores", &to.selector_scores) ||
        !entry(addresses, "taser_cross_attention_bytes", &to.cross_attention_bytes) || !entry(addresses, "taser_cross_attention", &to.cross_attention) ||
        !entry(addresses, "taser_cross_attention_grad", &to.cross_attention_grad) || !entry(addresses, "taser_relative_bias_bytes", &to.relative_bias_bytes) ||
        !entry(addresses, "taser_relative_bias", &to.relative_bias) || !entry(addresses, "taser_relative_bias_grad", &to.relative_bias_grad) ||
        !entry(addresses, "taser_policy_loss", &to.policy_loss) || !entry(addresses, "taser_last_error", &to.last_error))
        return nullptr;
    api = to;
    Py_INCREF(cls);
    Py_XSETREF(error_class, cls);
    Py_RETURN_NONE;
}

#define FAST(name, function) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(function)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"bind", bind, METH_VARARGS, nullptr}, FAST("sample", sample), FAST("gather", gather), FAST("encodings", encodings),
                         FAST("select", select), FAST("lookup", lookup), FAST("draw", draw), FAST("update", update), FAST("scores", scores),
                         FAST("attention", attention), FAST("attention_grad", attention_grad), FAST("bias", bias), FAST("bias_grad", bias_grad), FAST("policy", policy),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", "Native half of the Python binding, built for " TASER_BINDING_TAG ".", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() {
    s_nbr = PyUnicode_InternFromString("nbr");
    s_eid = PyUnicode_InternFromString("eid");
    s_ts = PyUnicode_InternFromString("ts");
    s_count = PyUnicode_InternFromString("count");
    s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    if (!s_nbr || !s_eid || !s_ts || !s_count || !s_cuda_stream) return nullptr;
    return PyModule_Create(&module);
}
