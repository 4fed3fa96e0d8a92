// Argument marshalling of the operators that need no context: torch tensors in, argument blocks of include/mtad.h out.  In C++ because a
// call of a few microseconds on the device is bound by its host side (checks, strides and pointers of a dozen tensors took 10 us in
// Python).  Functions return their outputs, or the library's negative status code; tensors of a wrong kind raise ValueError.
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <optional>
#include <string>

#include "mtad.h"

namespace {

using at::Tensor;

const Tensor& tensor(PyObject* o, const char* what) {
    TORCH_CHECK_VALUE(THPVariable_Check(o), what, ": a tensor is needed");
    return THPVariable_Unpack(o);
}
bool none(PyObject* o) { return o == Py_None; }
int64_t whole(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw python_error();
    return v;
}
int32_t small(PyObject* o) {                              // (what does not fit is out of every range there is)
    return (int32_t)std::clamp<int64_t>(whole(o), INT32_MIN, INT32_MAX);
}
float real(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw python_error();
    return (float)v;
}
int type_of(const Tensor& t) {
    switch (t.scalar_type()) {
        case at::kBFloat16: return MTAD_BF16;
        case at::kHalf: return MTAD_F16;
        case at::kFloat: return MTAD_F32;
        default: return -1;
    }
}

// (a dimension of one entry may have any stride)
int64_t step(const Tensor& t, int d) { return t.size(d) == 1 ? 0 : t.stride(d); }
bool alike(const Tensor& a, const Tensor& b) {
    if (a.sizes() != b.sizes() || a.scalar_type() != b.scalar_type() || a.device() != b.device()) return false;
    for (int d = 0; d < a.dim(); ++d)
        if (step(a, d) != step(b, d)) return false;
    return true;
}

// The device of a call, and its stream: what is allocated here belongs to the stream that uses it
struct On {
    c10::cuda::OptionalCUDAGuard device;
    std::optional<c10::cuda::CUDAStreamGuard> guard;
    void* stream;
    On(const Tensor& t, PyObject* handle) {
        TORCH_CHECK_VALUE(t.is_cuda(), "the operators run on CUDA tensors only");
        if (none(handle)) {
            device.set_index(t.get_device());
            stream = c10::cuda::getCurrentCUDAStream(t.get_device()).stream();
        } else {
            const cudaStream_t s = reinterpret_cast<cudaStream_t>(whole(handle));
            const auto st = s ? c10::cuda::getStreamFromExternal(s, t.get_device()) : c10::cuda::getDefaultCUDAStream(t.get_device());
            guard.emplace(st);
            stream = s;
        }
    }
};

// Pointer of an optional contiguous tensor of that type and shape
void* plain(PyObject* o, const char* what, at::ScalarType type, at::IntArrayRef shape, const Tensor& like) {
    if (none(o)) return nullptr;
    const Tensor& t = tensor(o, what);
    TORCH_CHECK_VALUE(t.scalar_type() == type && t.sizes() == shape && t.is_contiguous() && t.device() == like.device(), what, ": expected ",
                      c10::toString(type), " ", shape, ", contiguous, on ", like.device().str(), "; got ", c10::toString(t.scalar_type()), " ",
                      t.sizes(), " on ", t.device().str());
    return t.data_ptr();
}
template <typename P> P* as(void* p) { return static_cast<P*>(p); }

struct Pages {
    mtad_paged_kv kv;
    const Tensor& k;
    int64_t slots;                   // of a table row
    Pages(PyObject* k_, PyObject* v_, PyObject* table_, int64_t batch) : k(tensor(k_, "k_pages")) {
        const Tensor &v = tensor(v_, "v_pages"), &t = tensor(table_, "table");
        TORCH_CHECK_VALUE(k.dim() == 4 && alike(k, v), "k_pages and v_pages: [pages, kv heads, slots of a page, head_dim], alike in shape, strides, type and device");
        TORCH_CHECK_VALUE(t.dim() == 2 && t.scalar_type() == at::kInt && t.device() == k.device() && t.stride(1) == 1 && t.size(0) >= batch,
                          "table: int32 [sequences, pages] on the pages' device, a row for every sequence, a row contiguous");
        TORCH_CHECK_VALUE(t.size(0) <= 1 || t.stride(0) >= t.size(1), "table: rows lie apart, each of its own (of an expanded view: table.contiguous())");
        TORCH_CHECK_VALUE(k.stride(3) == 1 && (type_of(k) == MTAD_BF16 || type_of(k) == MTAD_F16), "pages hold rows of bf16 or fp16 that are contiguous");
        kv.k_pages = k.data_ptr();
        kv.v_pages = v.data_ptr();
        kv.table = static_cast<const int32_t*>(t.data_ptr());
        kv.page_stride = step(k, 0);
        kv.head_stride = step(k, 1);
        kv.slot_stride = k.size(2) == 1 ? k.size(3) : k.stride(2);
        kv.table_stride = t.size(0) <= 1 ? t.size(1) : t.stride(0);       // (of one row: whatever)
        kv.dtype = type_of(k);
        kv.n_pages = (int32_t)std::min<int64_t>(k.size(0), INT32_MAX);
        kv.page_size = (int32_t)std::min<int64_t>(k.size(2), INT32_MAX);
        kv.n_kv_heads = (int32_t)std::min<int64_t>(k.size(1), INT32_MAX);
        kv.head_dim = (int32_t)std::min<int64_t>(k.size(3), INT32_MAX);
        kv.max_pages = (int32_t)std::min<int64_t>(t.size(1), INT32_MAX);
        slots = t.size(1) * k.size(2);
    }
};

// [sequences, rows, heads, head_dim] with contiguous heads
void rows(const Tensor& t, const char* what, int64_t b, int64_t r, const Tensor& k) {
    TORCH_CHECK_VALUE(t.dim() == 4 && t.size(0) == b && t.size(1) == r && t.size(3) == k.size(3) && t.stride(3) == 1 && t.device() == k.device(), what,
                      ": [sequences, rows, heads, head_dim] with contiguous heads on the pages' device, got ", t.sizes());
}
// fp32 [sequences, kv heads, at least n slots]
void columns(const Tensor& t, const char* what, int64_t b, int64_t n, const Tensor& k) {
    TORCH_CHECK_VALUE(t.dim() == 3 && t.size(0) >= b && t.size(1) == k.size(1) && t.size(2) >= n && t.stride(2) == 1 && t.scalar_type() == at::kFloat &&
                          t.device() == k.device(), what, ": fp32 [sequences, kv heads, at least ", n, " slots] on the pages' device");
}

PyObject* status(int rc) { return PyLong_FromLong(rc); }

void count(Py_ssize_t got, Py_ssize_t want) { TORCH_CHECK_TYPE(got == want, "expected ", want, " arguments, got ", got); }

// (q, k, v, k_pages, v_pages, table, lens, n_rows, pos, rope_base, q_out, status, stream) -> q_out or None
PyObject* append(PyObject*, PyObject* const* x, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    count(n, 13);
    const Tensor &k = tensor(x[1], "k"), &v = tensor(x[2], "v");
    const int64_t b = k.dim() == 4 ? k.size(0) : 0, r = k.dim() == 4 ? k.size(1) : 0;
    const Pages p(x[3], x[4], x[5], b);
    rows(k, "k", b, r, p.k);
    TORCH_CHECK_VALUE(alike(k, v), "v: like k in shape, strides, type and device");
    TORCH_CHECK_VALUE(k.size(2) == p.k.size(1) && type_of(k) >= 0, "k: the pages' heads, bf16, fp16 or fp32");
    const On on(p.k, x[12]);
    mtad_paged_rows a{};
    Tensor out;
    if (!none(x[0])) {
        const Tensor& q = tensor(x[0], "q");
        rows(q, "q", b, r, p.k);
        TORCH_CHECK_VALUE(q.scalar_type() == k.scalar_type(), "q: k's type");
        out = none(x[10]) ? at::empty(q.sizes(), p.k.options()) : tensor(x[10], "q_out");
        rows(out, "q_out", b, r, p.k);
        TORCH_CHECK_VALUE(out.scalar_type() == p.k.scalar_type() && out.size(2) == q.size(2), "q_out: the pages' type, q's heads");
        a.q = q.data_ptr();
        a.q_out = out.data_ptr();
        a.q_stride_seq = step(q, 0); a.q_stride_row = step(q, 1); a.q_stride_head = step(q, 2);
        a.out_stride_seq = step(out, 0); a.out_stride_row = step(out, 1); a.out_stride_head = step(out, 2);
        a.n_q_heads = (int32_t)std::min<int64_t>(q.size(2), INT32_MAX);
    }
    a.lens = as<int32_t>(plain(x[6], "lens", at::kInt, {b}, p.k));
    a.n_rows = as<int32_t>(plain(x[7], "n_rows", at::kInt, {b}, p.k));
    a.pos = as<int32_t>(plain(x[8], "pos", at::kInt, {b}, p.k));
    a.status = as<uint32_t>(plain(x[11], "status", at::kInt, {b}, p.k));
    a.k = k.data_ptr();
    a.v = v.data_ptr();
    a.kv_stride_seq = step(k, 0); a.kv_stride_row = step(k, 1); a.kv_stride_head = step(k, 2);
    a.dtype = type_of(k);
    a.batch = (int32_t)std::min<int64_t>(b, INT32_MAX);
    a.rows = (int32_t)std::min<int64_t>(r, INT32_MAX);
    a.rope_base = real(x[9]);
    const int rc = mtad_paged_append(&p.kv, &a, on.stream);
    if (rc != MTAD_OK) return status(rc);
    if (!out.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(out);
    END_HANDLE_TH_ERRORS
}

// (q, k_pages, v_pages, table, lens, n_rows, window, sinks, scale, weights, out, lse, return_lse, max_len, status, stream) -> out or (out, lse)
PyObject* attention(PyObject*, PyObject* const* x, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    count(n, 16);
    const Tensor& q = tensor(x[0], "q");
    const int64_t b = q.dim() == 4 ? q.size(0) : 0, r = q.dim() == 4 ? q.size(1) : 0;
    const Pages p(x[1], x[2], x[3], b);
    rows(q, "q", b, r, p.k);
    TORCH_CHECK_VALUE(q.scalar_type() == p.k.scalar_type(), "q: the pages' type");
    const int64_t hq = q.size(2), most = none(x[13]) ? p.slots : std::min(whole(x[13]), p.slots);
    const On on(p.k, x[15]);
    Tensor out = none(x[10]) ? at::empty(q.sizes(), q.options()) : tensor(x[10], "out"), lse;
    rows(out, "out", b, r, p.k);
    TORCH_CHECK_VALUE(out.scalar_type() == q.scalar_type() && out.size(2) == hq && out.data_ptr() != q.data_ptr(), "out: like q, in memory of its own");
    mtad_paged_attn a{};
    const bool give = PyObject_IsTrue(x[12]);
    if (!none(x[11])) {
        lse = tensor(x[11], "lse");
        a.lse = as<float>(plain(x[11], "lse", at::kFloat, {b, r, hq}, p.k));
    } else if (give) {
        lse = at::empty({b, r, hq}, q.options().dtype(at::kFloat));
        a.lse = lse.data_ptr<float>();
    }
    if (!none(x[9])) {
        const Tensor& w = tensor(x[9], "weights");
        columns(w, "weights", b, most, p.k);
        a.weights = w.data_ptr<float>();
        a.weights_stride_seq = w.stride(0);
        a.weights_stride_head = w.stride(1);
    }
    a.lens = as<int32_t>(plain(x[4], "lens", at::kInt, {b}, p.k));
    a.n_rows = as<int32_t>(plain(x[5], "n_rows", at::kInt, {b}, p.k));
    a.status = as<uint32_t>(plain(x[14], "status", at::kInt, {b}, p.k));
    a.q = q.data_ptr();
    a.out = out.data_ptr();
    a.q_stride_seq = step(q, 0); a.q_stride_row = step(q, 1); a.q_stride_head = step(q, 2);
    a.out_stride_seq = step(out, 0); a.out_stride_row = step(out, 1); a.out_stride_head = step(out, 2);
    a.batch = (int32_t)std::min<int64_t>(b, INT32_MAX);
    a.rows = (int32_t)std::min<int64_t>(r, INT32_MAX);
    a.n_q_heads = (int32_t)std::min<int64_t>(hq, INT32_MAX);
    a.window = small(x[6]);
    a.sinks = small(x[7]);
    a.scale = real(x[8]);
    a.max_len = (int32_t)std::clamp<int64_t>(most, INT32_MIN, INT32_MAX);
    size_t need = 0;
    int rc = mtad_paged_attention_workspace(&p.kv, &a, &need);
    if (rc != MTAD_OK) return status(rc);
    Tensor scratch;
    if (need) scratch = at::empty({(int64_t)need}, q.options().dtype(at::kByte));
    rc = mtad_paged_attention(&p.kv, &a, need ? scratch.data_ptr() : nullptr, need, on.stream);
    if (rc != MTAD_OK) return status(rc);
    if (!give) return THPVariable_Wrap(out);
    PyObject* both = PyTuple_New(2);
    if (!both) throw python_error();
    PyTuple_SET_ITEM(both, 0, THPVariable_Wrap(out));
    PyTuple_SET_ITEM(both, 1, THPVariable_Wrap(lse));
    return both;
    END_HANDLE_TH_ERRORS
}

// (k_pages, v_pages, table, lens, scores, keep, first, recent, kept, new_lens, scores_out, max_len, status, stream) -> (kept, new_lens)
PyObject* evict(PyObject*, PyObject* const* x, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    count(n, 14);
    const Tensor &lens = tensor(x[3], "lens"), &scores = tensor(x[4], "scores");
    const int64_t b = lens.dim() == 1 ? lens.size(0) : 0;
    const Pages p(x[0], x[1], x[2], b);
    const int64_t most = std::min(p.slots, none(x[11]) ? (scores.dim() == 3 ? scores.size(2) : 0) : whole(x[11])), hkv = p.k.size(1);
    columns(scores, "scores", b, most, p.k);
    TORCH_CHECK_VALUE(scores.size(0) == b, "scores: as many sequences as lens");
    mtad_paged_eviction a{};
    a.keep = small(x[5]);
    a.first = small(x[6]);
    a.recent = small(x[7]);
    if (!none(x[10])) {
        const Tensor& o = tensor(x[10], "scores_out");
        columns(o, "scores_out", b, std::min<int64_t>(a.keep, most), p.k);
        TORCH_CHECK_VALUE(o.data_ptr() != scores.data_ptr() || (o.stride(0) == scores.stride(0) && o.stride(1) == scores.stride(1)),
                          "scores_out: scores itself, or memory of its own");
        a.scores_out = o.data_ptr<float>();
        a.out_stride_seq = o.stride(0);
        a.out_stride_head = o.stride(1);
    }
    const On on(p.k, x[13]);
    a.lens = as<int32_t>(plain(x[3], "lens", at::kInt, {b}, p.k));
    const int64_t wide = std::max(a.keep, 0);
    Tensor kept = none(x[8]) ? at::empty({b, hkv, wide}, lens.options()) : tensor(x[8], "kept");
    Tensor now = none(x[9]) ? at::empty({b}, lens.options()) : tensor(x[9], "new_lens");
    a.kept = none(x[8]) ? kept.data_ptr<int32_t>() : as<int32_t>(plain(x[8], "kept", at::kInt, {b, hkv, wide}, p.k));
    a.new_lens = none(x[9]) ? now.data_ptr<int32_t>() : as<int32_t>(plain(x[9], "new_lens", at::kInt, {b}, p.k));
    a.status = as<uint32_t>(plain(x[12], "status", at::kInt, {b}, p.k));
    a.scores = scores.data_ptr<float>();
    a.scores_stride_seq = scores.stride(0);
    a.scores_stride_head = scores.stride(1);
    a.batch = (int32_t)std::min<int64_t>(b, INT32_MAX);
    a.max_len = (int32_t)std::clamp<int64_t>(most, INT32_MIN, INT32_MAX);
    const int rc = mtad_paged_evict(&p.kv, &a, on.stream);
    if (rc != MTAD_OK) return status(rc);
    PyObject* both = PyTuple_New(2);
    if (!both) throw python_error();
    PyTuple_SET_ITEM(both, 0, THPVariable_Wrap(kept));
    PyTuple_SET_ITEM(both, 1, THPVariable_Wrap(now));
    return both;
    END_HANDLE_TH_ERRORS
}

// (logits, draft_tok, last_uniform, n_draft, temperature, stream, result, draft_logq, log_tau) or
// (.., result, draft_rows, accept_uniform, draft_temperature) -> status code
PyObject* accept(PyObject*, PyObject* const* x, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    TORCH_CHECK_TYPE(n == 9 || n == 10, "expected 9 or 10 arguments, got ", n);
    const Tensor& z = tensor(x[0], "logits");
    TORCH_CHECK_VALUE(z.dim() == 3 && z.stride(2) == 1 && type_of(z) >= 0, "logits: [sequences, drafted tokens + 1, vocab]");
    const int64_t b = z.size(0), g = z.size(1) - 1, v = z.size(2);
    const On on(z, x[5]);
    mtad_accept_rows a{};
    a.logits = z.data_ptr();
    a.logits_stride_seq = z.stride(0);
    a.logits_stride_row = z.stride(1);
    TORCH_CHECK_VALUE(g <= 0 || !none(x[1]), "draft_tok: the drafted tokens");
    if (g > 0) a.draft_tok = as<int32_t>(plain(x[1], "draft_tok", at::kInt, {b, g}, z));
    a.last_uniform = as<float>(plain(x[2], "last_uniform", at::kFloat, {b, v}, z));
    a.n_draft = as<int32_t>(plain(x[3], "n_draft", at::kInt, {b}, z));
    a.dtype = type_of(z);
    a.batch = (int32_t)std::min<int64_t>(b, INT32_MAX);
    a.gamma = (int32_t)std::min<int64_t>(g, INT32_MAX);
    a.vocab = (int32_t)std::min<int64_t>(v, INT32_MAX);
    a.temperature = real(x[4]);
    a.draft_temperature = 1.f;
    const mtad_result* out = reinterpret_cast<const mtad_result*>(whole(x[6]));
    if (n == 9) return status(mtad_accept_chain(&a, g > 0 ? as<float>(plain(x[7], "draft_logq", at::kFloat, {b, g}, z)) : nullptr, real(x[8]), out, on.stream));
    const Tensor& q = tensor(x[7], "draft_rows");
    TORCH_CHECK_VALUE(q.dim() == 3 && q.size(0) == b && q.size(1) == g && q.size(2) == v && q.stride(2) == 1 && q.scalar_type() == z.scalar_type() &&
                          q.device() == z.device(), "draft_rows: [sequences, drafted tokens, vocab], the logits' type");
    a.draft_stride_seq = q.stride(0);
    a.draft_stride_row = q.stride(1);
    a.draft_temperature = real(x[9]);
    return status(mtad_accept_chain_spd(&a, q.data_ptr(), as<float>(plain(x[8], "accept_uniform", at::kFloat, {b, g}, z)), out, on.stream));
    END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"append", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(append)), METH_FASTCALL, nullptr},
    {"attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(attention)), METH_FASTCALL, nullptr},
    {"evict", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(evict)), METH_FASTCALL, nullptr},
    {"accept", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(accept)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
// the torch that this was compiled for, "torch <version>;", as the build finds it in the file
__attribute__((used)) const char built_for[] = MTAD_TORCH;
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ops", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__ops(void) {
    PyObject* m = PyModule_Create(&module);
    const std::string name(built_for);
    if (m && PyModule_AddStringConstant(m, "torch_version", name.substr(6, name.size() - 7).c_str()) < 0) Py_CLEAR(m);
    return m;
}
