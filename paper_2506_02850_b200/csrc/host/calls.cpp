// Native half of binding.py: the entry points that a program calls once per video, per pruning layer or
// per cache, from Python arguments to the C ABI and back.
//
// What bounds a small call is host work: a ctypes call converts some twenty arguments, each output is
// a torch.empty from Python, each scalar output a fill kernel, and the workspace and the stream are looked
// up by name -- 35 to 50 us per call before and between the launches (a call's own launches take 2 to 3 us
// each).  Here a call costs a few microseconds: tensors are unpacked in place, outputs come straight from
// the caching allocator, and the library is called through its function pointer.
//
// The functions take positional arguments from the wrappers of the same name in binding.py, which hold the
// documented signatures, and return the result dict, or the library's status as an int if it is not zero.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/core/LegacyTypeDispatch.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <memory>
#include <vector>

#include "../../../include/metok.h"

namespace {

// ---- the library's entry points, set by bind() when binding.py loads a library -------------------
#define METOK_HOST_CALLS(X)                                                                              \
    X(metok_segment_events_workspace_bytes) X(metok_segment_events)                                      \
    X(metok_segment_score_events_workspace_bytes) X(metok_segment_score_events)                          \
    X(metok_compress_vision_bound) X(metok_compress_vision_workspace_bytes) X(metok_compress_vision)     \
    X(metok_prefill_prune_workspace_bytes) X(metok_prefill_prune)                                        \
    X(metok_retention_budgets) X(metok_prune_schedule_sizes) X(metok_prefill_prune_schedule_workspace_bytes)                        \
    X(metok_prefill_prune_schedule) X(metok_kv_compact_workspace_bytes) X(metok_kv_compact)               \
    X(metok_prefill_attention_workspace_bytes) X(metok_prefill_attention)                                \
    X(metok_paged_append) X(metok_paged_attention_workspace_bytes) X(metok_paged_attention)              \
    X(metok_paged_evict_workspace_bytes) X(metok_paged_evict) X(metok_rotate_heads)                      \
    X(metok_paged_append_q4) X(metok_paged_read_q4)                                                      \
    X(metok_paged_attention_q4_workspace_bytes) X(metok_paged_attention_q4)
struct Api {
#define X(name) decltype(&::name) name;
    METOK_HOST_CALLS(X)
#undef X
} api;

PyObject* bind(PyObject*, PyObject* table) {                  // {name: address}
#define X(name)                                                                                          \
    {                                                                                                    \
        PyObject* v = PyDict_GetItemString(table, #name);                                                \
        if (!v) return PyErr_Format(PyExc_KeyError, #name);                                              \
        api.name = reinterpret_cast<decltype(&::name)>(PyLong_AsVoidPtr(v));                             \
        if (PyErr_Occurred()) return nullptr;                                                            \
    }
    METOK_HOST_CALLS(X)
#undef X
    Py_RETURN_NONE;
}

// ---- small helpers ---------------------------------------------------------------------------------
struct Py {                                                   // owned reference
    PyObject* p;
    explicit Py(PyObject* o) : p(o) {}
    ~Py() { Py_XDECREF(p); }
    Py(const Py&) = delete;
    Py& operator=(const Py&) = delete;
};

// dict keys and argument names, interned once
#define METOK_HOST_NAMES(X)                                                                              \
    X(sims) X(boundaries) X(event_offsets) X(frame_event) X(_sims) X(_boundaries) X(_offsets)            \
    X(token_score) X(token_inv_norm) X(out_feats) X(out_src) X(out_event) X(out_members) X(assign)       \
    X(frame_score) X(event_score) X(event_is_key) X(n_out) X(status) X(scores) X(keep_idx) X(S_out)      \
    X(hidden_out) X(token_group) X(origin) X(n_vis) X(S) X(_inputs) X(keep_len) X(new_len) X(out) X(lse) \
    X(q) X(k) X(v) X(positions)
struct Names {
#define X(name) PyObject* name;
    METOK_HOST_NAMES(X)
#undef X
} names;

// Every failure sets a Python exception and throws this.
struct PyError {};
[[noreturn]] void fail(PyObject* type, const char* fmt, const char* what) {
    PyErr_Format(type, fmt, what);
    throw PyError();
}

const at::Tensor& tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) fail(PyExc_TypeError, "%s must be a tensor", name);
    return THPVariable_Unpack(o);
}
const at::Tensor& cuda_contig(PyObject* o, const char* name) {
    const at::Tensor& t = tensor(o, name);
    if (!t.is_cuda()) fail(PyExc_ValueError, "%s must be a CUDA tensor", name);
    if (!t.is_contiguous()) fail(PyExc_ValueError, "%s must be contiguous", name);
    return t;
}
const at::Tensor& of_dims(PyObject* o, const char* name, int dims) {
    const at::Tensor& t = cuda_contig(o, name);
    if (t.dim() != dims) fail(PyExc_ValueError, "%s has the wrong number of dimensions", name);
    return t;
}
int dtype_code(const at::Tensor& t) {
    if (t.scalar_type() == at::kFloat) return METOK_F32;
    if (t.scalar_type() == at::kBFloat16) return METOK_BF16;
    fail(PyExc_TypeError, "unsupported dtype %s", c10::toString(t.scalar_type()));
}
long integer(PyObject* o) {
    if (PyLong_Check(o)) {
        const long v = PyLong_AsLong(o);
        if (v == -1 && PyErr_Occurred()) throw PyError();
        return v;
    }
    Py i(PyNumber_Long(o));
    if (!i.p) throw PyError();
    const long v = PyLong_AsLong(i.p);
    if (v == -1 && PyErr_Occurred()) throw PyError();
    return v;
}
double number(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw PyError();
    return v;
}
struct Seq {                                                  // a sequence's items
    Py list;
    Py_ssize_t n;
    PyObject** items;
    explicit Seq(PyObject* o) : list(PySequence_Fast(o, "a sequence is wanted")), n(0), items(nullptr) {
        if (!list.p) throw PyError();
        n = PySequence_Fast_GET_SIZE(list.p);
        items = PySequence_Fast_ITEMS(list.p);
    }
};

at::Tensor empty(at::IntArrayRef shape, at::ScalarType dt, const at::Device& dev) {
    return at::Tensor(at::detail::empty_cuda(shape, dt, dev, std::nullopt));
}
at::Tensor empty_i32(int64_t n, const at::Device& dev) { return empty({n}, at::kInt, dev); }
at::Tensor empty_f32(int64_t n, const at::Device& dev) { return empty({n}, at::kFloat, dev); }

void put(PyObject* dict, PyObject* key, const at::Tensor& t) {
    Py v(THPVariable_Wrap(t));
    if (!v.p || PyDict_SetItem(dict, key, v.p) != 0) throw PyError();
}
void put_int(PyObject* dict, PyObject* key, long value) {
    Py v(PyLong_FromLong(value));
    if (!v.p || PyDict_SetItem(dict, key, v.p) != 0) throw PyError();
}
PyObject* item(PyObject* dict, PyObject* key) {
    PyObject* v = PyDict_GetItemWithError(dict, key);
    if (!v) {
        if (!PyErr_Occurred()) PyErr_SetObject(PyExc_KeyError, key);
        throw PyError();
    }
    return v;
}
const at::Tensor& get(PyObject* dict, PyObject* key) { return tensor(item(dict, key), "an output"); }

// The first n elements of the one-dimensional `whole` under `key`; an entry that `have` (the caller's
// dict, may be null) already holds is taken over.
void put_first(PyObject* dict, PyObject* key, PyObject* have, const at::Tensor& whole, int64_t n) {
    if (have) {
        PyObject* old = PyDict_GetItemWithError(have, key);
        if (old && THPVariable_Check(old)) {
            const at::Tensor& t = THPVariable_Unpack(old);
            if (t.dim() == 1 && t.numel() == n && t.data_ptr() == whole.data_ptr() && t.scalar_type() == whole.scalar_type()) {
                if (have != dict && PyDict_SetItem(dict, key, old) != 0) throw PyError();
                return;
            }
        }
        if (PyErr_Occurred()) throw PyError();
    }
    if (whole.numel() == n) {
        put(dict, key, whole);
        return;
    }
    at::AutoDispatchBelowADInplaceOrView guard;
    put(dict, key, whole.slice(0, 0, n));
}

// ---- workspaces ------------------------------------------------------------------------------------
// One buffer per device and stream: calls on one stream never overlap, calls on different streams may.
// Guarded by the interpreter lock.  A stream that outgrows its buffer gets a new one; at most kMaxWorkspaces
// are held, the one used longest ago goes first (the allocator keeps its memory from being reused before
// the stream's queued work is done).
struct Workspace {
    c10::DeviceIndex dev;
    cudaStream_t stream;
    at::Tensor buf, status;                                   // status: the first int32, the call's status word
    uint64_t used;
};
constexpr size_t kMaxWorkspaces = 256;                        // beyond the streams torch itself hands out per device
std::vector<Workspace>& workspaces() {
    static auto* v = new std::vector<Workspace>();            // never destroyed: tensors must not outlive the CUDA context's teardown
    return *v;
}
uint64_t ws_clock = 0;

Workspace workspace(size_t need, const at::Device& dev) {
    const auto stream = c10::cuda::getCurrentCUDAStream(dev.index());
    std::vector<Workspace>& all = workspaces();
    Workspace* w = nullptr;
    for (Workspace& x : all)
        if (x.stream == stream.stream() && x.dev == stream.device_index()) { w = &x; break; }
    if (!w) {
        if (all.size() >= kMaxWorkspaces) {
            size_t oldest = 0;
            for (size_t i = 1; i < all.size(); ++i)
                if (all[i].used < all[oldest].used) oldest = i;
            all.erase(all.begin() + oldest);
        }
        all.push_back({stream.device_index(), stream.stream(), at::Tensor(), at::Tensor(), 0});
        w = &all.back();
    }
    if (!w->buf.defined() || (size_t)w->buf.numel() < need) {
        const int64_t bytes = need > ((size_t)1 << 20) ? (int64_t)need : (int64_t)1 << 20;
        w->buf = empty({bytes}, at::kByte, dev);
        at::AutoDispatchBelowADInplaceOrView guard;
        w->status = w->buf.slice(0, 0, 4).view(at::kInt);
    }
    w->used = ++ws_clock;
    return *w;
}

void* current_stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

void want(Py_ssize_t n, Py_ssize_t expected) {
    if (n != expected) fail(PyExc_TypeError, "%s", "wrong number of arguments");
}

// ---- calls -----------------------------------------------------------------------------------------
PyObject* py_workspace(PyObject* const* a, Py_ssize_t n) {     // nbytes, any tensor's device given as a tensor or index
    want(n, 2);
    return THPVariable_Wrap(workspace((size_t)integer(a[0]), at::Device(at::kCUDA, (c10::DeviceIndex)integer(a[1]))).buf);
}

// The four arrays a segmentation writes: new, or those of an earlier result.
struct SegOut {
    at::Tensor sims, boundaries, offsets, frame_event;
};
SegOut seg_new(int64_t T, int64_t k, const at::Device& dev) {
    return {empty_f32(T > 1 ? T - 1 : 1, dev), empty_i32(k > 1 ? k - 1 : 1, dev), empty_i32(k > 0 ? k + 1 : 2, dev),
            empty_i32(T, dev)};
}
SegOut seg_from(PyObject* d) {
    return {get(d, names._sims), get(d, names._boundaries), get(d, names._offsets), get(d, names.frame_event)};
}
void seg_put(PyObject* dict, PyObject* have, const SegOut& o, int64_t T, int64_t k) {
    put_first(dict, names.sims, have, o.sims, T - 1);
    put_first(dict, names.boundaries, have, o.boundaries, k > 1 ? k - 1 : 0);
    put_first(dict, names.event_offsets, have, o.offsets, k + 1);
}

PyObject* segment_events(PyObject* const* a, Py_ssize_t n) {   // feats, k, sim_mode, out
    want(n, 4);
    const at::Tensor& feats = of_dims(a[0], "feats", 3);
    const int T = (int)feats.size(0), N = (int)feats.size(1), d = (int)feats.size(2);
    const int k = (int)integer(a[1]), sim = (int)integer(a[2]), dt = dtype_code(feats);
    PyObject* have = a[3] == Py_None ? nullptr : a[3];
    const SegOut o = have ? seg_from(have) : seg_new(T, k, feats.device());
    const Workspace ws = workspace(api.metok_segment_events_workspace_bytes(dt, T, N, d, sim), feats.device());
    const int st = api.metok_segment_events(feats.data_ptr(), dt, T, N, d, k, sim, (float*)o.sims.data_ptr(),
                                            (int32_t*)o.boundaries.data_ptr(), (int32_t*)o.offsets.data_ptr(),
                                            (int32_t*)o.frame_event.data_ptr(), ws.buf.data_ptr(), ws.buf.numel(),
                                            current_stream());
    if (st != METOK_OK) return PyLong_FromLong(st);
    Py res(PyDict_New());
    if (!res.p) throw PyError();
    seg_put(res.p, have, o, T, k);
    put(res.p, names.frame_event, o.frame_event);
    put(res.p, names._sims, o.sims);
    put(res.p, names._boundaries, o.boundaries);
    put(res.p, names._offsets, o.offsets);
    Py_INCREF(res.p);
    return res.p;
}

PyObject* segment_score_events(PyObject* const* a, Py_ssize_t n) {   // feats, k, text_emb, out
    want(n, 4);
    const at::Tensor& feats = of_dims(a[0], "feats", 3);
    const at::Tensor& text = cuda_contig(a[2], "text_emb");
    const int T = (int)feats.size(0), N = (int)feats.size(1), d = (int)feats.size(2);
    const int k = (int)integer(a[1]), dt = dtype_code(feats);
    const bool reuse = a[3] != Py_None;
    Py res(reuse ? a[3] : PyDict_New());
    if (!res.p) throw PyError();
    if (reuse) Py_INCREF(res.p);
    SegOut o;
    at::Tensor score, inv_norm;
    if (reuse) {
        o = seg_from(res.p);
        score = get(res.p, names.token_score);
        inv_norm = get(res.p, names.token_inv_norm);
    } else {
        o = seg_new(T, k, feats.device());
        score = empty_f32((int64_t)T * N, feats.device());
        inv_norm = empty_f32((int64_t)T * N, feats.device());
        put(res.p, names._sims, o.sims);
        put(res.p, names._boundaries, o.boundaries);
        put(res.p, names._offsets, o.offsets);
        put(res.p, names.frame_event, o.frame_event);
        put(res.p, names.token_score, score);
        put(res.p, names.token_inv_norm, inv_norm);
    }
    const Workspace ws = workspace(api.metok_segment_score_events_workspace_bytes(dt, T, N, d), feats.device());
    const int st = api.metok_segment_score_events(
        feats.data_ptr(), dt, T, N, d, k, text.data_ptr(), (float*)o.sims.data_ptr(), (int32_t*)o.boundaries.data_ptr(),
        (int32_t*)o.offsets.data_ptr(), (int32_t*)o.frame_event.data_ptr(), (float*)score.data_ptr(),
        (float*)inv_norm.data_ptr(), ws.buf.data_ptr(), ws.buf.numel(), current_stream());
    if (st != METOK_OK) return PyLong_FromLong(st);
    seg_put(res.p, reuse ? res.p : nullptr, o, T, k);
    Py_INCREF(res.p);
    return res.p;
}

// feats, event_offsets, text_emb, params, cap, out, scored, key_events, key_frames
PyObject* compress_vision(PyObject* const* a, Py_ssize_t n) {
    want(n, 9);
    const at::Tensor& feats = of_dims(a[0], "feats", 3);
    const at::Tensor& offsets = cuda_contig(a[1], "event_offsets");
    const at::Tensor& text = cuda_contig(a[2], "text_emb");
    const int T = (int)feats.size(0), N = (int)feats.size(1), d = (int)feats.size(2);
    const int k = (int)offsets.numel() - 1, dt = dtype_code(feats);
    const at::Device dev = feats.device();
    metok_vision_params p;
    {
        Py_buffer view;
        if (PyObject_GetBuffer(a[3], &view, PyBUF_SIMPLE) != 0) throw PyError();
        const bool fits = view.len == (Py_ssize_t)sizeof(p);
        if (fits) memcpy(&p, view.buf, sizeof(p));
        PyBuffer_Release(&view);
        if (!fits) fail(PyExc_TypeError, "%s must be a VisionParams", "p");
    }
    const bool reuse = a[5] != Py_None;
    int cap;
    if (reuse) {
        cap = (int)get(a[5], names.out_src).numel();
    } else if (a[4] == Py_None) {
        cap = api.metok_compress_vision_bound(T, N, k, &p);
        if (cap < 0) return PyLong_FromLong(cap);
    } else {
        cap = (int)integer(a[4]);
    }
    Py res(reuse ? a[5] : PyDict_New());
    if (!res.p) throw PyError();
    if (reuse) {
        Py_INCREF(res.p);
    } else {
        const int64_t tokens = (int64_t)T * N;
        put(res.p, names.out_feats, empty({cap, d}, feats.scalar_type(), dev));
        put(res.p, names.out_src, empty_i32(cap, dev));
        put(res.p, names.out_event, empty_i32(cap, dev));
        put(res.p, names.out_members, empty_i32(cap, dev));
        put(res.p, names.assign, empty_i32(tokens, dev));
        if (a[6] == Py_None) put(res.p, names.token_score, empty_f32(tokens, dev));
        put(res.p, names.frame_score, empty_f32(T, dev));
        put(res.p, names.event_score, empty_f32(k, dev));
        put(res.p, names.event_is_key, empty({k}, at::kByte, dev));
        put(res.p, names.n_out, empty_i32(1, dev));
    }
    if (a[6] != Py_None) {
        if (PyDict_SetItem(res.p, names.token_score, item(a[6], names.token_score)) != 0) throw PyError();
        p.token_inv_norm = (const float*)get(a[6], names.token_inv_norm).data_ptr();
    }
    if (a[7] != Py_None) {
        const at::Tensor& t = cuda_contig(a[7], "key_events");
        if (t.scalar_type() != at::kByte || t.numel() != k) fail(PyExc_ValueError, "%s must be uint8 [k]", "key_events");
        p.key_events_given = (const uint8_t*)t.data_ptr();
    }
    if (a[8] != Py_None) {
        const at::Tensor& t = cuda_contig(a[8], "key_frames");
        if (t.scalar_type() != at::kByte || t.numel() != T) fail(PyExc_ValueError, "%s must be uint8 [T]", "key_frames");
        p.key_frames_given = (const uint8_t*)t.data_ptr();
    }
    const Workspace ws = workspace(api.metok_compress_vision_workspace_bytes(dt, T, N, d, k, cap, &p), dev);
    auto ptr = [&](PyObject* key) { return get(res.p, key).data_ptr(); };
    const int st = api.metok_compress_vision(
        feats.data_ptr(), dt, T, N, d, (const int32_t*)offsets.data_ptr(), k, text.data_ptr(), &p, ptr(names.out_feats),
        (int32_t*)ptr(names.out_src), (int32_t*)ptr(names.out_event), (int32_t*)ptr(names.out_members),
        (int32_t*)ptr(names.assign), (float*)ptr(names.token_score), (float*)ptr(names.frame_score),
        (float*)ptr(names.event_score), (uint8_t*)ptr(names.event_is_key), (int32_t*)ptr(names.n_out), cap,
        ws.buf.data_ptr(), ws.buf.numel(), current_stream());
    if (st != METOK_OK) return PyLong_FromLong(st);
    put(res.p, names.status, ws.status);
    Py_INCREF(res.p);
    return res.p;
}

// q_text, k_all, hidden, vis_start, n_vis, token_group, group_budget, softmax_scale, out
PyObject* prefill_prune(PyObject* const* a, Py_ssize_t n) {
    want(n, 9);
    const at::Tensor& q = of_dims(a[0], "q_text", 3);
    const at::Tensor& kk = of_dims(a[1], "k_all", 3);
    const at::Tensor& group = cuda_contig(a[5], "token_group");
    const int Hq = (int)q.size(0), Lt = (int)q.size(1), dh = (int)q.size(2), Hkv = (int)kk.size(0), S = (int)kk.size(1);
    const int vis_start = (int)integer(a[3]), n_vis = (int)integer(a[4]), dt = dtype_code(q);
    const float scale = (float)number(a[7]);
    const at::Device dev = q.device();
    at::Tensor hidden;
    int D = 0;
    if (a[2] != Py_None) {
        hidden = cuda_contig(a[2], "hidden");
        D = (int)hidden.size(1);
    }
    int32_t few[METOK_MAX_GROUPS];
    std::vector<int32_t> many;
    int32_t* budgets = few;
    int G;
    {
        Seq b(a[6]);
        G = (int)b.n;
        if (G > METOK_MAX_GROUPS) { many.resize(G); budgets = many.data(); }
        for (int g = 0; g < G; ++g) budgets[g] = (int32_t)integer(b.items[g]);
    }
    const bool reuse = a[8] != Py_None;
    Py res(reuse ? a[8] : PyDict_New());
    if (!res.p) throw PyError();
    at::Tensor scores, keep, s_out, hidden_out;
    if (reuse) {
        Py_INCREF(res.p);
        scores = get(res.p, names.scores);
        keep = get(res.p, names.keep_idx);
        s_out = get(res.p, names.S_out);
        PyObject* h = item(res.p, names.hidden_out);
        if (h != Py_None) hidden_out = tensor(h, "hidden_out");
    } else {
        scores = empty_f32(n_vis, dev);
        keep = empty_i32(S, dev);
        s_out = empty_i32(1, dev);
        put(res.p, names.scores, scores);
        put(res.p, names.keep_idx, keep);
        put(res.p, names.S_out, s_out);
        if (hidden.defined()) {
            hidden_out = empty(hidden.sizes(), hidden.scalar_type(), hidden.device());
            put(res.p, names.hidden_out, hidden_out);
        } else if (PyDict_SetItem(res.p, names.hidden_out, Py_None) != 0) {
            throw PyError();
        }
    }
    const Workspace ws = workspace(api.metok_prefill_prune_workspace_bytes(dt, Hq, Hkv, Lt, S, dh, n_vis), dev);
    const int st = api.metok_prefill_prune(
        q.data_ptr(), kk.data_ptr(), hidden.defined() ? hidden.data_ptr() : nullptr, dt, Hq, Hkv, Lt, S, dh, D, vis_start,
        n_vis, (const int32_t*)group.data_ptr(), G, budgets, scale, (float*)scores.data_ptr(), (int32_t*)keep.data_ptr(),
        (int32_t*)s_out.data_ptr(), hidden_out.defined() ? hidden_out.data_ptr() : nullptr, ws.buf.data_ptr(),
        ws.buf.numel(), current_stream());
    if (st != METOK_OK) return PyLong_FromLong(st);
    put(res.p, names.status, ws.status);
    Py_INCREF(res.p);
    return res.p;
}

PyObject* retention_budgets(PyObject* const* a, Py_ssize_t n) {   // alpha, r, stage, N0
    want(n, 4);
    int32_t n0[2], b[2];
    Seq s(a[3]);
    if (s.n < 2) fail(PyExc_ValueError, "%s must hold two counts", "N0");
    n0[0] = (int32_t)integer(s.items[0]);
    n0[1] = (int32_t)integer(s.items[1]);
    const int st = api.metok_retention_budgets(number(a[0]), number(a[1]), (int)integer(a[2]), n0, b);
    return st == METOK_OK ? Py_BuildValue("[ii]", b[0], b[1]) : PyLong_FromLong(st);
}

// q_texts, k_alls, hiddens, vis_start, token_group, alpha, r, N0, softmax_scale, levels: the last argument is a
// writable buffer of one metok_prune_level per level, filled here (the caller keeps it for the K/V lists)
PyObject* prefill_prune_schedule(PyObject* const* a, Py_ssize_t n) {
    want(n, 10);
    Seq qs(a[0]), ks(a[1]);
    const int n_levels = (int)qs.n;
    std::unique_ptr<Seq> hs;
    if (a[2] != Py_None) hs = std::make_unique<Seq>(a[2]);
    if (n_levels < 1 || n_levels > 3) return PyLong_FromLong(METOK_ERR_INVALID_ARG);
    if (ks.n < n_levels || (hs && hs->n < n_levels)) fail(PyExc_ValueError, "%s: one per level is wanted", "k_alls / hiddens");
    const at::Tensor& group = cuda_contig(a[4], "token_group");
    const int n_vis = (int)group.numel(), vis_start = (int)integer(a[3]);
    const double alpha = number(a[5]), r = number(a[6]);
    int32_t n0[2], sizes[4];
    {
        Seq s(a[7]);
        if (s.n < 2) fail(PyExc_ValueError, "%s must hold two counts", "N0");
        n0[0] = (int32_t)integer(s.items[0]);
        n0[1] = (int32_t)integer(s.items[1]);
    }
    int st = api.metok_prune_schedule_sizes(n_levels, alpha, r, n0, sizes);
    if (st != METOK_OK) return PyLong_FromLong(st);
    const float scale = (float)number(a[8]);
    const at::Tensor& q0 = of_dims(qs.items[0], "q_text", 3);
    const at::Tensor& k0 = of_dims(ks.items[0], "k_all", 3);
    const int Hq = (int)q0.size(0), Lt = (int)q0.size(1), dh = (int)q0.size(2), Hkv = (int)k0.size(0), S = (int)k0.size(1);
    const int dt = dtype_code(q0);
    const int D = hs ? (int)of_dims(hs->items[0], "hidden", 2).size(1) : 0;
    const at::Device dev = group.device();
    Py_buffer view;
    if (PyObject_GetBuffer(a[9], &view, PyBUF_WRITABLE) != 0) throw PyError();
    struct Release { Py_buffer* v; ~Release() { PyBuffer_Release(v); } } release{&view};
    if (view.len < (Py_ssize_t)sizeof(metok_prune_level) * n_levels) fail(PyExc_ValueError, "%s is too small", "levels");
    metok_prune_level* lv = static_cast<metok_prune_level*>(view.buf);
    Py list(PyList_New(n_levels));
    if (!list.p) throw PyError();
    for (int s = 0; s < n_levels; ++s) {
        const at::Tensor& q = cuda_contig(qs.items[s], "q_text");
        const at::Tensor& kk = of_dims(ks.items[s], "k_all", 3);
        const int S_s = S - n_vis + sizes[s];
        if (kk.size(0) != Hkv || kk.size(1) != S_s || kk.size(2) != dh) {
            PyErr_Format(PyExc_ValueError, "level %d: k_all must be (%d, %d, %d), got (%d, %d, %d)", s + 1, Hkv, S_s, dh,
                         (int)kk.size(0), (int)kk.size(1), (int)kk.size(2));
            throw PyError();
        }
        PyObject* d = PyDict_New();
        if (!d) throw PyError();
        PyList_SET_ITEM(list.p, s, d);
        const int64_t nv = sizes[s] > 0 ? sizes[s] : 1;
        const at::Tensor scores = empty_f32(nv, dev), keep = empty_i32(S_s, dev), s_out = empty_i32(1, dev),
                         origin = empty_i32(nv, dev), grp = s == 0 ? group : empty_i32(nv, dev);
        put(d, names.scores, scores);
        put(d, names.keep_idx, keep);
        put(d, names.S_out, s_out);
        lv[s] = {q.data_ptr(), kk.data_ptr(), nullptr, nullptr, (float*)scores.data_ptr(), (int32_t*)keep.data_ptr(),
                 (int32_t*)s_out.data_ptr(), (int32_t*)grp.data_ptr(), (int32_t*)origin.data_ptr()};
        PyObject* hid = hs ? hs->items[s] : Py_None;
        if (hs) {
            const at::Tensor& h = cuda_contig(hid, "hidden");
            const at::Tensor ho = empty(h.sizes(), h.scalar_type(), h.device());
            put(d, names.hidden_out, ho);
            lv[s].hidden = h.data_ptr();
            lv[s].hidden_out = ho.data_ptr();
        } else if (PyDict_SetItem(d, names.hidden_out, Py_None) != 0) {
            throw PyError();
        }
        put(d, names.token_group, grp);
        put(d, names.origin, origin);
        put_int(d, names.n_vis, sizes[s]);
        put_int(d, names.S, S_s);
        Py inputs(PyTuple_Pack(3, qs.items[s], ks.items[s], hid));   // alive until the caller is done with the result
        if (!inputs.p || PyDict_SetItem(d, names._inputs, inputs.p) != 0) throw PyError();
    }
    const size_t need = api.metok_prefill_prune_schedule_workspace_bytes(n_levels, dt, Hq, Hkv, Lt, S, dh, n_vis, alpha, r, n0);
    if (need == 0) return PyLong_FromLong(METOK_ERR_INVALID_ARG);
    const Workspace ws = workspace(need, dev);
    const at::Tensor status = empty_i32(1, dev);
    st = api.metok_prefill_prune_schedule(lv, n_levels, dt, Hq, Hkv, Lt, S, dh, D, vis_start, n_vis, alpha, r, n0, scale,
                                          (int32_t*)status.data_ptr(), ws.buf.data_ptr(), ws.buf.numel(), current_stream());
    if (st != METOK_OK) return PyLong_FromLong(st);
    Py wrapped(THPVariable_Wrap(status));
    if (!wrapped.p) throw PyError();
    for (int s = 0; s < n_levels; ++s)
        if (PyDict_SetItem(PyList_GET_ITEM(list.p, s), names.status, wrapped.p) != 0) throw PyError();
    Py_INCREF(list.p);
    return list.p;
}

// k_layers, v_layers, S_cur, policy, vis_start, n_vis, l1, keep_ratio, scores, keep_idx, keep_len, new_len
PyObject* kv_compact(PyObject* const* a, Py_ssize_t n) {
    want(n, 12);
    Seq ks(a[0]), vs(a[1]);
    const int L = (int)ks.n;
    if (L < 1) fail(PyExc_ValueError, "%s is empty", "k_layers");
    if (vs.n != L) fail(PyExc_ValueError, "%s must hold one tensor per layer", "v_layers");
    std::vector<void*> kp(L), vp(L);
    for (int l = 0; l < L; ++l) {
        kp[l] = cuda_contig(ks.items[l], "k/v layer").data_ptr();
        vp[l] = cuda_contig(vs.items[l], "k/v layer").data_ptr();
    }
    const at::Tensor& k0 = of_dims(ks.items[0], "k/v layer", 3);
    const int Hkv = (int)k0.size(0), S_cap = (int)k0.size(1), dh = (int)k0.size(2), dt = dtype_code(k0);
    const at::Device dev = k0.device();
    const int S_cur = (int)integer(a[2]), policy = (int)integer(a[3]), vis_start = (int)integer(a[4]), n_vis = (int)integer(a[5]),
              l1 = (int)integer(a[6]);
    const double ratio = number(a[7]);
    at::Tensor scores, keep, len, new_len;
    int per_layer = 0;
    if (a[8] != Py_None) {
        scores = cuda_contig(a[8], "scores");
        per_layer = scores.dim() == 2;
    }
    if (a[9] == Py_None) {
        keep = empty({L, S_cur}, at::kInt, dev);
        len = empty_i32(L, dev);
    } else {
        keep = tensor(a[9], "keep_idx");
        len = tensor(a[10], "keep_len");
    }
    new_len = a[11] == Py_None ? empty_i32(L, dev) : tensor(a[11], "new_len");
    const Workspace ws = workspace(api.metok_kv_compact_workspace_bytes(dt, L, Hkv, S_cur, dh, policy, n_vis), dev);
    const int st = api.metok_kv_compact(kp.data(), vp.data(), dt, L, Hkv, S_cap, S_cur, dh, policy, l1, ratio, vis_start, n_vis,
                                        scores.defined() ? (const float*)scores.data_ptr() : nullptr, per_layer,
                                        (int32_t*)keep.data_ptr(), (int32_t*)len.data_ptr(), (int32_t*)new_len.data_ptr(),
                                        ws.buf.data_ptr(), ws.buf.numel(), current_stream());
    if (st != METOK_OK) return PyLong_FromLong(st);
    Py res(PyDict_New());
    if (!res.p) throw PyError();
    put(res.p, names.keep_idx, keep);
    put(res.p, names.keep_len, len);
    put(res.p, names.new_len, new_len);
    put(res.p, names.status, ws.status);
    Py_INCREF(res.p);
    return res.p;
}

// ---- the paged cache and the attention over it -------------------------------------------------------
// These calls run on the device of their tensors, whatever the current one is, on that device's current stream; all
// their tensors lie on it.  Their workspaces come from the caching allocator for the one call: no two calls share one,
// so that captured graphs may be replayed side by side.
const at::Tensor& on(PyObject* o, const char* name, const at::Device& dev) {
    const at::Tensor& t = tensor(o, name);
    if (t.device() != dev) fail(PyExc_ValueError, "%s is on another device than the call's first tensor", name);
    return t;
}
// A contiguous array of n elements (n < 0: any number) of the type, or an undefined tensor for None.
at::Tensor array(PyObject* o, const char* name, const at::Device& dev, at::ScalarType dt, int64_t n) {
    if (o == Py_None) return at::Tensor();
    const at::Tensor& t = on(o, name, dev);
    if (!t.is_contiguous()) fail(PyExc_ValueError, "%s must be contiguous", name);
    if (t.scalar_type() != dt) fail(PyExc_TypeError, dt == at::kInt ? "%s must be int32" : "%s must be float32", name);
    if (n >= 0 && t.numel() != n) fail(PyExc_ValueError, "%s has the wrong number of elements", name);
    return t;
}
template <typename T>
T* ptr_or_null(const at::Tensor& t) { return t.defined() ? static_cast<T*>(t.data_ptr()) : nullptr; }
// Rows [heads][rows][dh] whose elements are contiguous; other strides are free.
const at::Tensor& rows3(PyObject* o, const char* name, const at::Device& dev, at::ScalarType dt) {
    const at::Tensor& t = on(o, name, dev);
    if (t.dim() != 3) fail(PyExc_ValueError, "%s has the wrong number of dimensions", name);
    if (t.scalar_type() != dt) fail(PyExc_TypeError, "%s has another dtype than the call's first tensor", name);
    if (t.size(2) != 1 && t.stride(2) != 1) fail(PyExc_ValueError, "the elements of a row of %s must be contiguous", name);
    return t;
}
// A dimension's stride; one that is never stepped along counts as `dense` (torch leaves it arbitrary).
int64_t step(const at::Tensor& t, int dim, int64_t dense) { return t.size(dim) > 1 ? t.stride(dim) : dense; }

const at::Tensor& first_tensor(PyObject* o, const char* name) {
    const at::Tensor& t = tensor(o, name);
    if (!t.is_cuda()) fail(PyExc_ValueError, "%s must be a CUDA tensor", name);
    return t;
}
int size_of(const at::Tensor& t, int dim, const char* name) {
    if (t.size(dim) > 0x7FFFFFFF) fail(PyExc_ValueError, "%s is too large", name);
    return (int)t.size(dim);
}

// q, k, v, softmax_scale, seq_q, seq_k, prefix_len, causal, softcap, slopes, positions, with_lse, out
PyObject* prefill_attention(PyObject* const* a, Py_ssize_t n) {
    want(n, 13);
    const at::Tensor& q = first_tensor(a[0], "q");
    const at::Device dev = q.device();
    const c10::cuda::CUDAGuard guard(dev);
    const at::ScalarType dt = q.scalar_type();
    rows3(a[0], "q", dev, dt);
    const at::Tensor &k = rows3(a[1], "k", dev, dt), &v = rows3(a[2], "v", dev, dt);
    if (k.sizes() != v.sizes() || k.size(2) != q.size(2)) fail(PyExc_ValueError, "%s must be [Hkv, n_k, dh], q [Hq, n_q, dh]", "k, v");
    metok_attention_params p = {};
    p.Hq = size_of(q, 0, "q"); p.n_q = size_of(q, 1, "q"); p.dh = size_of(q, 2, "q");
    p.Hkv = size_of(k, 0, "k"); p.n_k = size_of(k, 1, "k");
    const at::Tensor seq_q = array(a[4], "seq_q", dev, at::kInt, -1), seq_k = array(a[5], "seq_k", dev, at::kInt, -1);
    if (seq_q.defined() != seq_k.defined()) fail(PyExc_ValueError, "%s: both or neither", "seq_q, seq_k");
    p.n_seq = 1;
    if (seq_q.defined()) {
        if (seq_q.numel() < 2 || seq_q.numel() != seq_k.numel()) fail(PyExc_ValueError, "%s must be int32 [documents + 1]", "seq_q, seq_k");
        if (seq_q.numel() > 0x7FFFFFFF) fail(PyExc_ValueError, "%s is too large", "seq_q");
        p.n_seq = (int)seq_q.numel() - 1;
    }
    const at::Tensor prefix = array(a[6], "prefix_len", dev, at::kInt, p.n_seq), slopes = array(a[9], "slopes", dev, at::kFloat, p.Hq),
                     pos = array(a[10], "positions", dev, at::kInt, p.n_k);
    const int causal = PyObject_IsTrue(a[7]), with_lse = PyObject_IsTrue(a[11]);
    if (causal < 0 || with_lse < 0) throw PyError();
    const at::Tensor out = a[12] == Py_None ? empty(q.sizes(), dt, dev) : rows3(a[12], "out", dev, dt);
    if (out.sizes() != q.sizes()) fail(PyExc_ValueError, "%s must have the shape of q", "out");
    at::Tensor lse;
    if (with_lse) lse = empty({p.Hq, p.n_q}, at::kFloat, dev);
    const at::Tensor status = empty_i32(1, dev);
    p.q = q.data_ptr(); p.k = k.data_ptr(); p.v = v.data_ptr(); p.out = out.data_ptr(); p.lse = ptr_or_null<float>(lse);
    p.q_head = step(q, 0, 0); p.q_row = step(q, 1, p.dh); p.k_head = step(k, 0, 0); p.k_row = step(k, 1, p.dh);
    p.v_head = step(v, 0, 0); p.v_row = step(v, 1, p.dh); p.out_head = step(out, 0, 0); p.out_row = step(out, 1, p.dh);
    p.seq_q = ptr_or_null<const int32_t>(seq_q); p.seq_k = ptr_or_null<const int32_t>(seq_k);
    p.prefix_len = ptr_or_null<const int32_t>(prefix); p.positions = ptr_or_null<const int32_t>(pos);
    p.slopes = ptr_or_null<const float>(slopes);
    p.softmax_scale = (float)number(a[3]); p.softcap = (float)number(a[8]); p.causal = causal;
    const int code = dtype_code(q);
    const size_t need = api.metok_prefill_attention_workspace_bytes(code, &p);
    at::Tensor ws;
    if (need > 0) ws = empty({(int64_t)need}, at::kByte, dev);
    const int st = api.metok_prefill_attention(code, &p, (int32_t*)status.data_ptr(), ptr_or_null<void>(ws), need, current_stream());
    if (st != METOK_OK) return PyLong_FromLong(st);
    Py res(PyDict_New());
    if (!res.p) throw PyError();
    put(res.p, names.out, out);
    if (with_lse) put(res.p, names.lse, lse);
    put(res.p, names.status, status);
    Py_INCREF(res.p);
    return res.p;
}

// The pools of one layer, the table and the lengths; `hold` keeps the last two.  q4: pools held in 4 bits.
metok_paged_cache paged_cache(const at::Tensor& k, PyObject* v_obj, PyObject* table_obj, PyObject* len_obj, at::Tensor* hold, bool q4 = false) {
    const at::Device dev = k.device();
    if (q4) {
        if (k.dim() != 4 || !k.is_contiguous() || k.size(3) % 9)
            fail(PyExc_ValueError, "%s must be a contiguous [n_pages, Hkv, page_size / 16, 9 * dh]", "a pool");
        if (k.scalar_type() != at::kByte) fail(PyExc_TypeError, "%s must be uint8", "a pool");
        if (k.size(2) > 0x7FFFFFF) fail(PyExc_ValueError, "%s is too large", "a pool");
    } else if (k.dim() != 4 || !k.is_contiguous()) {
        fail(PyExc_ValueError, "%s must be a contiguous [n_pages, Hkv, page_size, dh]", "a pool");
    }
    const at::Tensor& v = on(v_obj, "a pool", dev);
    if (v.sizes() != k.sizes() || !v.is_contiguous() || v.scalar_type() != k.scalar_type())
        fail(PyExc_ValueError, "%s must be contiguous, of one shape and type", "the pools");
    const at::Tensor& table = on(table_obj, "block_table", dev);
    if (table.dim() != 2) fail(PyExc_ValueError, "%s must be [n_seqs, max_pages]", "block_table");
    hold[0] = array(table_obj, "block_table", dev, at::kInt, -1);
    hold[1] = array(len_obj, "kv_len", dev, at::kInt, table.size(0));
    if (!hold[1].defined()) fail(PyExc_TypeError, "%s must be a tensor", "kv_len");
    return {k.data_ptr(), v.data_ptr(), (const int32_t*)hold[0].data_ptr(), (const int32_t*)hold[1].data_ptr(), size_of(k, 0, "a pool"),
            size_of(k, 1, "a pool"), size_of(k, 2, "a pool") * (q4 ? 16 : 1), size_of(k, 3, "a pool") / (q4 ? 9 : 1), size_of(table, 0, "block_table"),
            size_of(table, 1, "block_table")};
}

// k_new, v_new, k_pool, v_pool, block_table, kv_len, new_offsets, positions, pos_new, mass, mass_new, new_len
template <bool kQ4>
PyObject* paged_append(PyObject* const* a, Py_ssize_t n) {
    want(n, 12);
    const at::Tensor& kp = first_tensor(a[2], "k_pool");
    const at::Device dev = kp.device();
    const c10::cuda::CUDAGuard guard(dev);
    at::Tensor hold[2];
    const metok_paged_cache c = paged_cache(kp, a[3], a[4], a[5], hold, kQ4);
    const at::ScalarType dt = (kQ4 ? tensor(a[0], "k_new") : kp).scalar_type();
    const at::Tensor &kn = rows3(a[0], "k_new", dev, dt), &vn = rows3(a[1], "v_new", dev, dt);
    if (kn.sizes() != vn.sizes() || kn.size(0) != c.Hkv || kn.size(2) != c.dh) fail(PyExc_ValueError, "%s must be [Hkv, n_new, dh]", "k_new, v_new");
    const int n_new = size_of(kn, 1, "k_new");
    const int64_t S_cap = (int64_t)c.max_pages * c.page_size;
    const at::Tensor off = array(a[6], "new_offsets", dev, at::kInt, (int64_t)c.n_seqs + 1), pos = array(a[7], "positions", dev, at::kInt, c.n_seqs * S_cap),
                     pos_new = array(a[8], "pos_new", dev, at::kInt, n_new), mass = array(a[9], "mass", dev, at::kFloat, c.n_seqs * S_cap),
                     mass_new = array(a[10], "mass_new", dev, at::kFloat, n_new);
    at::Tensor new_len = array(a[11], "new_len", dev, at::kInt, c.n_seqs);
    if (!new_len.defined()) new_len = empty_i32(c.n_seqs, dev);
    const at::Tensor status = empty_i32(1, dev);
    const int st = (kQ4 ? api.metok_paged_append_q4 : api.metok_paged_append)(dtype_code(kn), &c, kn.data_ptr(), vn.data_ptr(), step(kn, 0, 0), step(kn, 1, c.dh), step(vn, 0, 0),
                                          step(vn, 1, c.dh), n_new, ptr_or_null<const int32_t>(off), ptr_or_null<int32_t>(pos),
                                          ptr_or_null<const int32_t>(pos_new), ptr_or_null<float>(mass), ptr_or_null<const float>(mass_new),
                                          (int32_t*)new_len.data_ptr(), (int32_t*)status.data_ptr(), current_stream());
    if (st != METOK_OK) return PyLong_FromLong(st);
    Py res(PyDict_New());
    if (!res.p) throw PyError();
    put(res.p, names.new_len, new_len);
    put(res.p, names.status, status);
    Py_INCREF(res.p);
    return res.p;
}

// q, k_pool, v_pool, block_table, kv_len, softmax_scale, softcap, slopes, positions, mass, with_lse, out
template <bool kQ4>
PyObject* paged_attention(PyObject* const* a, Py_ssize_t n) {
    want(n, 12);
    const at::Tensor& kp = first_tensor(a[1], "k_pool");
    const at::Device dev = kp.device();
    const c10::cuda::CUDAGuard guard(dev);
    at::Tensor hold[2];
    const metok_paged_cache c = paged_cache(kp, a[2], a[3], a[4], hold, kQ4);
    const at::Tensor& q = rows3(a[0], "q", dev, (kQ4 ? tensor(a[0], "q") : kp).scalar_type());
    if (q.size(0) != c.n_seqs || q.size(2) != c.dh) fail(PyExc_ValueError, "%s must be [n_seqs, Hq, dh]", "q");
    const int Hq = size_of(q, 1, "q"), dt = dtype_code(q);
    const int64_t S_cap = (int64_t)c.max_pages * c.page_size;
    const at::Tensor slopes = array(a[7], "slopes", dev, at::kFloat, Hq), pos = array(a[8], "positions", dev, at::kInt, c.n_seqs * S_cap),
                     mass = array(a[9], "mass", dev, at::kFloat, c.n_seqs * S_cap);
    const at::Tensor out = a[11] == Py_None ? empty(q.sizes(), q.scalar_type(), dev) : rows3(a[11], "out", dev, q.scalar_type());
    if (out.sizes() != q.sizes()) fail(PyExc_ValueError, "%s must have the shape of q", "out");
    const int with_lse = PyObject_IsTrue(a[10]);
    if (with_lse < 0) throw PyError();
    at::Tensor lse;
    if (with_lse) lse = empty({c.n_seqs, Hq}, at::kFloat, dev);
    const at::Tensor status = empty_i32(1, dev);
    const size_t need = (kQ4 ? api.metok_paged_attention_q4_workspace_bytes : api.metok_paged_attention_workspace_bytes)(dt, &c, Hq, mass.defined());
    const at::Tensor ws = empty({(int64_t)need}, at::kByte, dev);
    const int st = (kQ4 ? api.metok_paged_attention_q4 : api.metok_paged_attention)(
        dt, &c, q.data_ptr(), step(q, 0, 0), step(q, 1, c.dh), Hq, (float)number(a[5]), (float)number(a[6]), ptr_or_null<const float>(slopes),
        ptr_or_null<const int32_t>(pos), ptr_or_null<float>(mass), out.data_ptr(), step(out, 0, 0), step(out, 1, c.dh), ptr_or_null<float>(lse),
        (int32_t*)status.data_ptr(), ws.data_ptr(), need, current_stream());
    if (st != METOK_OK) return PyLong_FromLong(st);
    Py res(PyDict_New());
    if (!res.p) throw PyError();
    put(res.p, names.out, out);
    if (with_lse) put(res.p, names.lse, lse);
    put(res.p, names.status, status);
    Py_INCREF(res.p);
    return res.p;
}

// k_layers, v_layers, block_table, kv_len, mass, positions, budget, n_sink, n_recent, new_len
PyObject* paged_evict(PyObject* const* a, Py_ssize_t n) {
    want(n, 10);
    Seq ks(a[0]), vs(a[1]);
    if (ks.n < 1) fail(PyExc_ValueError, "%s is empty", "k_layers");
    if (vs.n != ks.n) fail(PyExc_ValueError, "%s must hold one pool per layer", "v_layers");
    const at::Tensor& k0 = first_tensor(ks.items[0], "a pool");
    const at::Device dev = k0.device();
    const c10::cuda::CUDAGuard guard(dev);
    at::Tensor hold[2];
    const bool q4 = k0.scalar_type() == at::kByte;
    const metok_paged_cache c = paged_cache(k0, vs.items[0], a[2], a[3], hold, q4);
    if (ks.n > 1024) return PyLong_FromLong(METOK_ERR_UNSUPPORTED);
    const int L = (int)ks.n;
    std::vector<void*> kp(L), vp(L);
    for (int l = 0; l < L; ++l) {
        const at::Tensor &k = on(ks.items[l], "a pool", dev), &v = on(vs.items[l], "a pool", dev);
        if (k.sizes() != k0.sizes() || v.sizes() != k0.sizes() || !k.is_contiguous() || !v.is_contiguous() || k.scalar_type() != k0.scalar_type() ||
            v.scalar_type() != k0.scalar_type())
            fail(PyExc_ValueError, "%s must be contiguous, of one shape and type", "the pools");
        kp[l] = k.data_ptr();
        vp[l] = v.data_ptr();
    }
    const int64_t S_cap = (int64_t)c.max_pages * c.page_size;
    const at::Tensor mass = array(a[4], "mass", dev, at::kFloat, L * c.n_seqs * S_cap), pos = array(a[5], "positions", dev, at::kInt, L * c.n_seqs * S_cap);
    const long budget = integer(a[6]), sink = integer(a[7]), recent = integer(a[8]);
    if (budget < 1 || budget > S_cap || sink < 0 || recent < 1) return PyLong_FromLong(METOK_ERR_INVALID_ARG);
    // (beyond the largest position nothing changes)
    const int n_sink = (int)(sink > (1 << 30) ? 1 << 30 : sink), n_recent = (int)(recent > (1 << 30) ? 1 << 30 : recent);
    at::Tensor new_len = array(a[9], "new_len", dev, at::kInt, c.n_seqs);
    if (!new_len.defined()) new_len = empty_i32(c.n_seqs, dev);
    const at::Tensor keep = empty({L, c.n_seqs, budget}, at::kInt, dev), status = empty_i32(1, dev);
    const size_t need = api.metok_paged_evict_workspace_bytes(&c, L, (int)budget);
    const at::Tensor ws = empty({(int64_t)need}, at::kByte, dev);
    const int st = api.metok_paged_evict(q4 ? METOK_Q4 : dtype_code(k0), &c, kp.data(), vp.data(), L, (int)budget, n_sink, n_recent, ptr_or_null<int32_t>(pos),
                                         ptr_or_null<float>(mass), (int32_t*)keep.data_ptr(), (int32_t*)new_len.data_ptr(),
                                         (int32_t*)status.data_ptr(), ws.data_ptr(), need, current_stream());
    if (st != METOK_OK) return PyLong_FromLong(st);
    Py res(PyDict_New());
    if (!res.p) throw PyError();
    put(res.p, names.keep_idx, keep);
    put(res.p, names.new_len, new_len);
    put(res.p, names.status, status);
    Py_INCREF(res.p);
    return res.p;
}

// k_pool, v_pool, block_table, kv_len, offsets, n_rows, first_row, positions, dtype, k_out, v_out
PyObject* paged_read_q4(PyObject* const* a, Py_ssize_t n) {
    want(n, 11);
    const at::Tensor& kp = first_tensor(a[0], "k_pool");
    const at::Device dev = kp.device();
    const c10::cuda::CUDAGuard guard(dev);
    at::Tensor hold[2];
    const metok_paged_cache c = paged_cache(kp, a[1], a[2], a[3], hold, true);
    const long rows = integer(a[5]);
    if (rows < 0 || rows > 0x7FFFFFFF) fail(PyExc_ValueError, "%s is out of range", "n_rows");
    const int64_t S_cap = (int64_t)c.max_pages * c.page_size;
    const at::Tensor off = array(a[4], "offsets", dev, at::kInt, (int64_t)c.n_seqs + 1), first = array(a[6], "first_row", dev, at::kInt, c.n_seqs),
                     pos = array(a[7], "positions", dev, at::kInt, c.n_seqs * S_cap);
    if (!off.defined()) fail(PyExc_TypeError, "%s must be a tensor", "offsets");
    const bool bf16 = PyObject_IsTrue(a[8]);           // the wrapper's answer
    const at::ScalarType dt = bf16 ? at::kBFloat16 : at::kFloat;
    const at::Tensor k = a[9] == Py_None ? empty({c.Hkv, rows, c.dh}, dt, dev) : rows3(a[9], "k_out", dev, dt),
                     v = a[10] == Py_None ? empty({c.Hkv, rows, c.dh}, dt, dev) : rows3(a[10], "v_out", dev, dt);
    if (k.sizes() != v.sizes() || k.size(0) != c.Hkv || k.size(1) != rows || k.size(2) != c.dh)
        fail(PyExc_ValueError, "%s must be [Hkv, n_rows, dh]", "k_out, v_out");
    at::Tensor pos_out;
    if (pos.defined()) pos_out = empty({rows}, at::kInt, dev);
    const at::Tensor status = empty_i32(1, dev);
    const int st = api.metok_paged_read_q4(bf16 ? METOK_BF16 : METOK_F32, &c, (const int32_t*)off.data_ptr(), ptr_or_null<const int32_t>(first), (int)rows,
                                           k.data_ptr(), v.data_ptr(), step(k, 0, 0), step(k, 1, c.dh), step(v, 0, 0), step(v, 1, c.dh),
                                           ptr_or_null<const int32_t>(pos), ptr_or_null<int32_t>(pos_out), (int32_t*)status.data_ptr(), current_stream());
    if (st != METOK_OK) return PyLong_FromLong(st);
    Py res(PyDict_New());
    if (!res.p) throw PyError();
    put(res.p, names.k, k);
    put(res.p, names.v, v);
    if (pos_out.defined()) put(res.p, names.positions, pos_out);
    put(res.p, names.status, status);
    Py_INCREF(res.p);
    return res.p;
}

// q, k, inv_freq, positions, pair_axis, interleaved, eps, q_weight, k_weight, q_out, k_out
PyObject* rotate_heads(PyObject* const* a, Py_ssize_t n) {
    want(n, 11);
    const at::Tensor& q = first_tensor(a[0], "q");
    const at::Device dev = q.device();
    const c10::cuda::CUDAGuard guard(dev);
    const at::ScalarType dt = q.scalar_type();
    const int code = dtype_code(q);
    rows3(a[0], "q", dev, dt);
    const bool with_k = a[1] != Py_None;
    at::Tensor k;
    if (with_k) {
        k = rows3(a[1], "k", dev, dt);
        if (k.size(1) != q.size(1) || k.size(2) != q.size(2)) fail(PyExc_ValueError, "%s must be [Hkv, n, dh], q [Hq, n, dh]", "k");
    }
    metok_rotate_params p = {};
    p.Hq = size_of(q, 0, "q"); p.n = size_of(q, 1, "q"); p.dh = size_of(q, 2, "q");
    p.Hkv = with_k ? size_of(k, 0, "k") : 0;
    if (with_k && p.Hkv < 1) fail(PyExc_ValueError, "%s has no heads", "k");
    const at::Tensor freq = array(a[2], "inv_freq", dev, at::kFloat, -1);
    if (freq.defined() && freq.numel() > 1 << 20) fail(PyExc_ValueError, "%s is too large", "inv_freq");
    p.rotary_dim = freq.defined() ? 2 * (int)freq.numel() : 0;
    p.inv_freq = ptr_or_null<const float>(freq);
    p.n_axes = 1;
    at::Tensor pos;
    if (a[3] != Py_None) {
        pos = array(a[3], "positions", dev, at::kInt, -1);
        if ((pos.dim() != 1 && pos.dim() != 2) || pos.size(-1) != p.n) fail(PyExc_ValueError, "%s must be [n] or [axes, n]", "positions");
        if (pos.dim() == 2) p.n_axes = size_of(pos, 0, "positions");
    }
    p.positions = ptr_or_null<const int32_t>(pos);
    int32_t axis[64];
    if (a[4] != Py_None) {
        Seq s(a[4]);
        if (s.n != p.rotary_dim / 2) fail(PyExc_ValueError, "%s must hold an axis for every pair", "pair_axis");
        if (s.n > 64) return PyLong_FromLong(METOK_ERR_INVALID_ARG);
        for (Py_ssize_t i = 0; i < s.n; ++i) {
            const long v = integer(s.items[i]);
            axis[i] = v < 0 || v > 127 ? -1 : (int32_t)v;
        }
        p.pair_axis = axis;
    }
    const int interleaved = PyObject_IsTrue(a[5]);
    if (interleaved < 0) throw PyError();
    p.interleaved = interleaved;
    p.norm = a[6] != Py_None;
    p.eps = p.norm ? (float)number(a[6]) : 0.f;
    const at::Tensor qw = array(a[7], "q_weight", dev, at::kFloat, p.dh), kw = array(a[8], "k_weight", dev, at::kFloat, p.dh);
    if (!p.norm && (qw.defined() || kw.defined())) fail(PyExc_ValueError, "%s: weights want eps", "q_weight, k_weight");
    p.q_weight = ptr_or_null<const float>(qw);
    p.k_weight = ptr_or_null<const float>(kw);
    const at::Tensor qo = a[9] == Py_None ? empty(q.sizes(), dt, dev) : rows3(a[9], "q_out", dev, dt);
    if (qo.sizes() != q.sizes()) fail(PyExc_ValueError, "%s must have the shape of q", "q_out");
    at::Tensor ko;
    if (with_k) {
        ko = a[10] == Py_None ? empty(k.sizes(), dt, dev) : rows3(a[10], "k_out", dev, dt);
        if (ko.sizes() != k.sizes()) fail(PyExc_ValueError, "%s must have the shape of k", "k_out");
        p.k = k.data_ptr(); p.k_out = ko.data_ptr();
        p.k_head = step(k, 0, 0); p.k_row = step(k, 1, 0); p.ko_head = step(ko, 0, 0); p.ko_row = step(ko, 1, 0);
    }
    p.q = q.data_ptr(); p.q_out = qo.data_ptr();
    p.q_head = step(q, 0, 0); p.q_row = step(q, 1, 0); p.qo_head = step(qo, 0, 0); p.qo_row = step(qo, 1, 0);
    const int st = api.metok_rotate_heads(code, &p, current_stream());
    if (st != METOK_OK) return PyLong_FromLong(st);
    Py res(PyDict_New());
    if (!res.p) throw PyError();
    put(res.p, names.q, qo);
    if (with_k) put(res.p, names.k, ko);
    Py_INCREF(res.p);
    return res.p;
}

// Runs a call and turns its failures into Python exceptions.
template <PyObject* (*F)(PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    try {
        return F(args, n);
    } catch (const PyError&) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

#define FAST(name, fn) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&guarded<fn>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    {"bind", bind, METH_O, nullptr},
    FAST("workspace", py_workspace),
    FAST("segment_events", segment_events),
    FAST("segment_score_events", segment_score_events),
    FAST("compress_vision", compress_vision),
    FAST("retention_budgets", retention_budgets),
    FAST("prefill_prune", prefill_prune),
    FAST("prefill_prune_schedule", prefill_prune_schedule),
    FAST("kv_compact", kv_compact),
    FAST("prefill_attention", prefill_attention),
    FAST("paged_append", paged_append<false>),
    FAST("paged_attention", paged_attention<false>),
    FAST("paged_evict", paged_evict),
    FAST("rotate_heads", rotate_heads),
    FAST("paged_append_q4", paged_append<true>),
    FAST("paged_read_q4", paged_read_q4),
    FAST("paged_attention_q4", paged_attention<true>),
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_metok_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__metok_calls(void) {
#define X(name)                                                  \
    names.name = PyUnicode_InternFromString(#name);              \
    if (!names.name) return nullptr;
    METOK_HOST_NAMES(X)
#undef X
    return PyModule_Create(&module);
}
