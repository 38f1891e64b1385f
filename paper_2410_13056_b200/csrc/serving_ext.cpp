// The serving calls on torch tensors.  They are made per layer and generated token, where marshalling in Python took
// longer than the kernels (append and read back of one token: 29 us against 7), so it is done here: checks of shapes and
// types, outputs and work spaces, the current stream.  Nothing is computed.
#include <ATen/ATen.h>
#include <c10/cuda/CUDAGraphsC10Utils.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/extension.h>

#include <cmath>
#include <optional>
#include <map>

#include "cmpq.h"

namespace py = pybind11;
using at::Tensor;
using OptTensor = std::optional<Tensor>;

namespace {

struct StatusError {
    int status;
    const char* where;
};

void check(cmpq_status s, const char* where) {
    if (s != CMPQ_OK) throw StatusError{(int)s, where};
}

[[noreturn]] void refuse(const std::string& what) { throw py::value_error(what); }

std::string shape_of(const Tensor& t) {
    std::string s = "[";
    for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
    return s + "]";
}

cmpq_dtype code(const Tensor& t) {
    if (t.scalar_type() == at::kHalf) return CMPQ_F16;
    if (t.scalar_type() == at::kBFloat16) return CMPQ_BF16;
    throw py::type_error(std::string("expected a float16 or bfloat16 tensor, got ") + c10::toString(t.scalar_type()));
}

void* stream_of(const Tensor& t) { return c10::cuda::getCurrentCUDAStream(t.get_device()).stream(); }

void on_gpu(const Tensor& t, const char* name, int64_t dims) {
    if (!t.is_cuda() || t.dim() != dims) refuse(std::string(name) + " needs to be a " + std::to_string(dims) + "-dimensional CUDA tensor, got shape " + shape_of(t));
}

// A kernel runs on one device and takes addresses as they are.
void beside(const Tensor& t, const Tensor& home, const char* name) {
    if (t.device() != home.device()) refuse(std::string(name) + " is on " + t.device().str() + ", the rest on " + home.device().str());
}
void beside(const OptTensor& t, const Tensor& home, const char* name) {
    if (t) beside(*t, home, name);
}

// Leading dimension of [n][width] or [n][heads][d] with contiguous rows.
int64_t rows(const Tensor& t, const char* name) {
    const bool three = t.dim() == 3;
    const int64_t n = t.size(0), width = three ? t.size(1) * t.size(2) : t.size(1);
    const bool ok = t.numel() == 0 || (three ? t.stride(2) == 1 && (t.size(1) == 1 || t.stride(1) == t.size(2)) : t.size(1) == 1 || t.stride(1) == 1);
    if (!ok) refuse(std::string(name) + " needs contiguous rows of " + std::to_string(width) + " elements");
    return n > 1 ? t.stride(0) : width;
}

bool capturing() { return c10::cuda::currentStreamCaptureStatusMayInitCtx() != c10::cuda::CaptureStatus::None; }

// Work spaces.  Eager calls of a device and stream share one buffer (they run one after the other), whatever layer or cache
// they are of.  A call that is being captured takes its own from the graph's memory, zeroed by a node of that graph, and
// leaves nothing behind: a graph never depends on another one, on eager calls, or on the stream that it is replayed on.
struct Spaces {
    int64_t zeroed;  // the first bytes, counters that start at 0
    std::map<std::pair<int, void*>, Tensor> held;

    Tensor get(const at::Device& device, void* stream, size_t bytes) {
        if (capturing()) return fresh(device, bytes);
        Tensor& t = held[{device.index(), stream}];
        if (!t.defined() || (size_t)t.numel() < bytes) t = fresh(device, bytes);
        return t;
    }
    Tensor fresh(const at::Device& device, size_t bytes) const {
        Tensor t = at::empty({(int64_t)bytes}, at::TensorOptions().dtype(at::kByte).device(device));
        if (zeroed) t.narrow(0, 0, zeroed).zero_();
        return t;
    }
    void drop(const at::Device& device) {
        for (auto i = held.begin(); i != held.end();) i = i->first.first == device.index() ? held.erase(i) : std::next(i);
    }
};
// Never destroyed: the allocator may be gone before static objects are.
Spaces& linear_spaces() {
    static Spaces* s = new Spaces{0, {}};
    return *s;
}
Spaces& attention_spaces() {
    static Spaces* s = new Spaces{CMPQ_ATTENTION_ZEROED, {}};
    return *s;
}
Spaces& gated_spaces() {
    static Spaces* s = new Spaces{0, {}};
    return *s;
}
Spaces& gated_states() {
    static Spaces* s = new Spaces{CMPQ_GATED_STATE_BYTES, {}};
    return *s;
}

// What the calls on this word have reported, once the current stream of its device has got there; it starts again from 0.
cmpq_status take_word(const Tensor& word) {
    const c10::cuda::CUDAGuard guard(word.device());
    const cmpq_status s = cmpq_check_cache(word.data_ptr<int32_t>(), stream_of(word));
    if (s != CMPQ_OK) word.zero_();
    return s;
}

cmpq_act act_of(const std::optional<std::string>& name) {
    static const char* const names[] = {"none", "relu", "silu", "gelu", "gelu_tanh"};  // in the order of cmpq_act
    if (!name) return CMPQ_ACT_NONE;
    for (int i = 0; i < 5; ++i)
        if (*name == names[i]) return (cmpq_act)i;
    refuse("activation needs to be none, relu, silu, gelu or gelu_tanh, got " + *name);
}

// Checks of what the calls of a layer take beside its weights, of which `home` is one.
struct Around {
    cmpq_dtype dt;
    int64_t n, ldr = 0;
    const void *norm = nullptr, *residual = nullptr;

    Around(const Tensor& x, int64_t d_in, int64_t d_out, const Tensor& home, const OptTensor& into, const OptTensor& res, const OptTensor& weight) {
        if (x.dim() != 2 || x.size(1) != d_in || !x.is_cuda()) refuse("x needs shape [n][" + std::to_string(d_in) + "] on the GPU, got " + shape_of(x));
        beside(x, home, "x"), beside(into, home, "out"), beside(res, home, "residual"), beside(weight, home, "norm");
        dt = code(x);
        n = x.size(0);
        for (const auto& [t, name] : {std::pair<const OptTensor&, const char*>(into, "out"), {res, "residual"}})
            if (t && (t->dim() != 2 || t->size(0) != n || t->size(1) != d_out || t->scalar_type() != x.scalar_type() || !t->is_cuda()))
                refuse(std::string(name) + " needs shape [n][" + std::to_string(d_out) + "] and x's dtype");
        if (res) residual = res->data_ptr(), ldr = rows(*res, "residual");
        if (weight) {
            if (weight->dim() != 1 || weight->size(0) != d_in || weight->scalar_type() != x.scalar_type() || !weight->is_contiguous())
                refuse("norm needs " + std::to_string(d_in) + " contiguous entries of x's dtype");
            norm = weight->data_ptr();
        }
    }
};

struct Linear {
    Tensor w, scale;
    OptTensor bias;
    Tensor nonfinite;
    int64_t d_in, d_out;

    Linear(const Tensor& w_codes, const Tensor& w_scale, const OptTensor& b) : w(w_codes), scale(w_scale) {
        on_gpu(w, "w_codes", 2);
        on_gpu(scale, "w_scale", 1);
        beside(scale, w, "w_scale"), beside(b, w, "bias");
        if (w.scalar_type() != at::kChar || scale.scalar_type() != at::kFloat) refuse("w_codes needs to be int8, w_scale float32");
        if (w.stride(1) != 1 || w.stride(0) % 16 || (uintptr_t)w.data_ptr() % 16) refuse("w_codes needs rows that start on multiples of 16 bytes");
        d_out = w.size(0), d_in = w.size(1);
        if (scale.size(0) != d_out || (b && (b->dim() != 1 || b->size(0) != d_out || !b->is_cuda()))) refuse("w_scale and bias need one entry per row of w_codes");
        scale = scale.contiguous();
        if (b) bias = b->contiguous(), (void)code(*bias);
        nonfinite = at::zeros({1}, at::TensorOptions().dtype(at::kInt).device(w.device()));
    }

    cmpq_weight_i8 weight() const {
        return {w.data_ptr<int8_t>(), d_out > 1 ? w.stride(0) : (d_in + 15) / 16 * 16, scale.data_ptr<float>(), bias ? bias->data_ptr() : nullptr};
    }

    void takes(const Tensor& x) const {
        if (bias && bias->scalar_type() != x.scalar_type()) throw py::type_error("bias and x need one dtype");
    }

    Tensor call(const Tensor& x, const OptTensor& into, const std::optional<std::string>& activation, const OptTensor& residual, const OptTensor& norm,
                double eps) {
        const Around a(x, d_in, d_out, w, into, residual, norm);
        takes(x);
        const cmpq_act act = act_of(activation);
        const c10::cuda::CUDAGuard guard(x.device());
        Tensor y = into ? *into : at::empty({a.n, d_out}, x.options());
        if (a.n == 0) return y;
        void* stream = stream_of(x);
        const Tensor ws = linear_spaces().get(x.device(), stream, cmpq_linear_i8_ws_bytes(a.n, d_in, d_out));
        const cmpq_weight_i8 weights = weight();
        check(cmpq_linear_i8_fused(x.data_ptr(), a.dt, a.n, d_in, rows(x, "x"), a.norm, (float)eps, &weights, d_out, act, a.residual, a.ldr, y.data_ptr(),
                                   rows(y, "out"), nonfinite.data_ptr<int32_t>(), ws.data_ptr(), ws.numel(), stream),
              "cmpq_linear_i8");
        return y;
    }

    void look() { check(take_word(nonfinite), "cmpq_linear_i8"); }
};

struct Gated {
    Linear gate, up, down;
    cmpq_act act;
    Tensor word;
    // States for captured calls of few tokens, one each, 0 from here on: a node that zeroed it would cost every replay 2 us.  They
    // live as long as the weights have to; calls beyond them take theirs from the graph, with such a node.  One more is for
    // calls of more tokens, which have a word and so leave their state alone.
    static constexpr int64_t kCaptured = 64;
    Tensor kept, untouched;
    int64_t taken = 0;

    Gated(const Linear& g, const Linear& u, const Linear& d, const std::optional<std::string>& activation) : gate(g), up(u), down(d), act(act_of(activation)) {
        beside(u.w, g.w, "up"), beside(d.w, g.w, "down");
        if (u.d_in != g.d_in || u.d_out != g.d_out || d.d_in != g.d_out)
            refuse("gate [" + std::to_string(g.d_out) + "][" + std::to_string(g.d_in) + "], up [" + std::to_string(u.d_out) + "][" + std::to_string(u.d_in) +
                   "] and down [" + std::to_string(d.d_out) + "][" + std::to_string(d.d_in) + "] do not fit together");
        word = at::zeros({1}, at::TensorOptions().dtype(at::kInt).device(g.w.device()));
        kept = at::zeros({kCaptured + 1, CMPQ_GATED_STATE_BYTES}, at::TensorOptions().dtype(at::kByte).device(g.w.device()));
        untouched = kept[kCaptured];
    }

    Tensor state(int64_t n, void* stream) {
        if (n > CMPQ_GATED_FEW_TOKENS) return untouched;
        return capturing() && taken < kCaptured ? kept[taken++] : gated_states().get(word.device(), stream, CMPQ_GATED_STATE_BYTES);
    }

    Tensor call(const Tensor& x, const OptTensor& into, const OptTensor& residual, const OptTensor& norm, double eps) {
        const Around a(x, gate.d_in, down.d_out, gate.w, into, residual, norm);
        gate.takes(x), up.takes(x), down.takes(x);
        const c10::cuda::CUDAGuard guard(x.device());
        Tensor y = into ? *into : at::empty({a.n, down.d_out}, x.options());
        if (a.n == 0) return y;
        void* stream = stream_of(x);
        const Tensor ws = gated_spaces().get(x.device(), stream, cmpq_gated_i8_ws_bytes(a.n, gate.d_in, gate.d_out, down.d_out));
        const Tensor st = state(a.n, stream);
        const cmpq_weight_i8 g = gate.weight(), u = up.weight(), d = down.weight();
        check(cmpq_gated_i8(x.data_ptr(), a.dt, a.n, gate.d_in, rows(x, "x"), a.norm, (float)eps, &g, &u, &d, gate.d_out, down.d_out, act, a.residual, a.ldr,
                            y.data_ptr(), rows(y, "out"), word.data_ptr<int32_t>(), st.data_ptr(), ws.data_ptr(), ws.numel(), stream),
              "cmpq_gated_i8");
        return y;
    }

    void look() {
        const cmpq_status s = take_word(word);
        if (s == CMPQ_ERR_INTERNAL) gated_states().drop(word.device()), kept.zero_();  // see Cache::look
        check(s, "cmpq_gated_i8");
    }
};

struct Cache {
    Tensor k_codes, k_scale, v_codes, v_scale, word;
    cmpq_cache c;

    Cache(const Tensor& kc, const Tensor& ks, const Tensor& vc, const Tensor& vs) : k_codes(kc), k_scale(ks), v_codes(vc), v_scale(vs) {
        for (const Tensor* t : {&kc, &vc}) {
            on_gpu(*t, "codes", 4);
            if (t->scalar_type() != at::kChar) refuse("codes need to be int8");
        }
        for (const Tensor* t : {&ks, &vs}) {
            on_gpu(*t, "scales", 2);
            if (t->scalar_type() != at::kFloat) refuse("scales need to be float32");
        }
        beside(ks, kc, "k_scale"), beside(vc, kc, "v_codes"), beside(vs, kc, "v_scale");
        if (kc.sizes() != vc.sizes() || ks.sizes() != kc.sizes().slice(0, 2) || vs.sizes() != ks.sizes())
            refuse("codes need shape [n_pages][n_kv][page_tokens][head_dim] and scales [n_pages][n_kv]");
        if (!kc.is_contiguous() || !vc.is_contiguous() || !ks.is_contiguous() || !vs.is_contiguous()) refuse("the cache's tensors need to be contiguous");
        c = {static_cast<int8_t*>(kc.data_ptr()), static_cast<float*>(ks.data_ptr()), static_cast<int8_t*>(vc.data_ptr()),
             static_cast<float*>(vs.data_ptr()),  kc.size(0),                         (int32_t)kc.size(1),
             (int32_t)kc.size(3),                 (int32_t)kc.size(2)};
        word = at::zeros({1}, at::TensorOptions().dtype(at::kInt).device(kc.device()));
    }

    cmpq_batch batch(const Tensor& off, const Tensor& lens, const Tensor& table, int64_t n_tok) const {
        on_gpu(off, "tok_off", 1);
        on_gpu(lens, "lens", 1);
        on_gpu(table, "table", 2);
        beside(off, k_codes, "tok_off"), beside(lens, k_codes, "lens"), beside(table, k_codes, "table");
        if (off.scalar_type() != at::kInt || lens.scalar_type() != at::kInt || table.scalar_type() != at::kInt) refuse("tok_off, lens and table need to be int32");
        const int64_t n = table.size(0);
        if (off.size(0) != n + 1 || lens.size(0) != n) refuse("tok_off needs n_seq + 1 entries and table n_seq rows, n_seq = " + std::to_string(lens.size(0)));
        if (!off.is_contiguous() || !lens.is_contiguous() || (table.size(1) > 1 && table.stride(1) != 1)) refuse("tok_off, lens and table need contiguous rows");
        return {off.data_ptr<int32_t>(), lens.data_ptr<int32_t>(), table.data_ptr<int32_t>(), n > 1 ? table.stride(0) : table.size(1), n, n_tok, table.size(1)};
    }

    void heads(const Tensor& t, const char* name, int64_t count) const {
        if (t.dim() != 3 || t.size(2) != c.head_dim || (count && t.size(1) != count) || !t.is_cuda())
            refuse(std::string(name) + " needs shape [n_tok][" + (count ? std::to_string(count) : std::string("heads")) + "][" + std::to_string(c.head_dim) +
                   "] on the GPU, got " + shape_of(t));
        beside(t, k_codes, name);
    }

    OptTensor append(const Tensor& k, const Tensor& v, const Tensor& off, const Tensor& lens, const Tensor& table, const OptTensor& q, const OptTensor& cos,
                     const OptTensor& sin, bool interleaved, const OptTensor& q_into) {
        heads(k, "k", c.n_kv_heads);
        heads(v, "v", c.n_kv_heads);
        const cmpq_dtype dt = code(k);
        if (v.scalar_type() != k.scalar_type() || v.size(0) != k.size(0)) refuse("k and v need one dtype and token count");
        if (cos.has_value() != sin.has_value()) refuse("cos and sin come together");
        if (cos && (cos->dim() != 2 || cos->sizes() != sin->sizes() || !cos->is_contiguous() || !sin->is_contiguous() || cos->scalar_type() != at::kFloat ||
                    sin->scalar_type() != at::kFloat || !cos->is_cuda() || !sin->is_cuda()))
            refuse("cos and sin need to be contiguous fp32 CUDA tensors of one shape");
        beside(cos, k_codes, "cos"), beside(sin, k_codes, "sin"), beside(q_into, k_codes, "q_out");
        if (q) heads(*q, "q", 0);
        const cmpq_batch b = batch(off, lens, table, k.size(0));
        const c10::cuda::CUDAGuard guard(k.device());
        OptTensor q_out;
        if (q) {
            if (q->scalar_type() != k.scalar_type() || q->size(0) != k.size(0)) refuse("q needs k's dtype and token count");
            if (q_into && (q_into->sizes() != q->sizes() || q_into->scalar_type() != q->scalar_type() || !q_into->is_cuda())) refuse("q_out needs q's shape and dtype");
            q_out = q_into ? *q_into : at::empty(q->sizes(), q->options());
        }
        check(cmpq_cache_append(&c, &b, k.data_ptr(), rows(k, "k"), v.data_ptr(), rows(v, "v"), dt, cos ? cos->data_ptr<float>() : nullptr,
                                sin ? sin->data_ptr<float>() : nullptr, cos ? cos->size(0) : 0, cos ? (int32_t)(2 * cos->size(1)) : 0, interleaved,
                                q ? q->data_ptr() : nullptr, q ? rows(*q, "q") : 0, q ? (int32_t)q->size(1) : 0, q ? q_out->data_ptr() : nullptr,
                                q ? rows(*q_out, "q_out") : 0, word.data_ptr<int32_t>(), stream_of(k)),
              "cmpq_cache_append");
        return q_out;
    }

    std::pair<Tensor, Tensor> read(const Tensor& off, const Tensor& lens, const Tensor& table, int64_t n_tok, bool bf16) {
        const cmpq_batch b = batch(off, lens, table, n_tok);
        const c10::cuda::CUDAGuard guard(k_codes.device());
        const auto options = k_codes.options().dtype(bf16 ? at::kBFloat16 : at::kHalf);
        Tensor k = at::empty({n_tok, c.n_kv_heads, c.head_dim}, options), v = at::empty({n_tok, c.n_kv_heads, c.head_dim}, options);
        check(cmpq_cache_read(&c, &b, bf16 ? CMPQ_BF16 : CMPQ_F16, k.data_ptr(), v.data_ptr(), (int64_t)c.n_kv_heads * c.head_dim, word.data_ptr<int32_t>(),
                              stream_of(k_codes)),
              "cmpq_cache_read");
        return {k, v};
    }

    std::pair<Tensor, OptTensor> attend(const Tensor& q, const Tensor& off, const Tensor& lens, const Tensor& table, int64_t max_new,
                                        std::optional<int64_t> max_len, std::optional<double> scale, bool causal, int64_t window, const OptTensor& into,
                                        bool want_lse, bool zero_behind) {
        heads(q, "q", 0);
        const cmpq_dtype dt = code(q);
        const int64_t n = q.size(0), h = q.size(1);
        if (h == 0 || h % c.n_kv_heads) refuse(std::to_string(h) + " query heads are no multiple of the cache's " + std::to_string(c.n_kv_heads) + " heads");
        if (into && (into->sizes() != q.sizes() || into->scalar_type() != q.scalar_type() || !into->is_cuda())) refuse("out needs q's shape and dtype");
        beside(into, k_codes, "out");
        const cmpq_batch b = batch(off, lens, table, n);
        const c10::cuda::CUDAGuard guard(q.device());
        const int64_t longest = max_len ? *max_len : table.size(1) * c.page_tokens;
        Tensor out = into ? *into : at::empty(q.sizes(), q.options());
        OptTensor lse;
        if (want_lse) lse = at::empty({n, h}, q.options().dtype(at::kFloat));
        void* stream = stream_of(q);
        const size_t bytes = cmpq_cache_attention_ws_bytes(b.n_seq, n, max_new, longest, (int32_t)h, c.n_kv_heads, c.head_dim);
        const Tensor ws = attention_spaces().get(q.device(), stream, bytes);
        check(cmpq_cache_attention(&c, &b, q.data_ptr(), rows(q, "q"), dt, (int32_t)h, max_new, longest,
                                   scale ? (float)*scale : 1.0f / std::sqrt((float)c.head_dim), causal | (zero_behind ? CMPQ_ZERO_BEHIND : 0), window, out.data_ptr(), rows(out, "out"),
                                   lse ? lse->data_ptr<float>() : nullptr, word.data_ptr<int32_t>(), ws.data_ptr(), ws.numel(), stream),
              "cmpq_cache_attention");
        return {out, lse};
    }

    void look() {
        const cmpq_status s = take_word(word);
        if (s == CMPQ_ERR_INTERNAL) attention_spaces().drop(word.device());  // a kernel gave up: its counters may not be 0
        check(s, "cmpq_check_cache");
    }
};

}  // namespace

PYBIND11_MODULE(_serving, m) {
    py::register_exception_translator([](std::exception_ptr p) {
        try {
            if (p) std::rethrow_exception(p);
        } catch (const StatusError& e) {
            py::object error = py::module_::import("paper_2410_13056_b200.binding").attr("CmpqError");
            PyErr_SetObject(error.ptr(), error(e.status, e.where).ptr());
        }
    });
    py::class_<Linear>(m, "Linear")
        .def(py::init<const Tensor&, const Tensor&, const OptTensor&>())
        .def("__call__", &Linear::call, py::arg("x"), py::arg("out") = py::none(), py::arg("activation") = py::none(), py::arg("residual") = py::none(),
             py::arg("norm") = py::none(), py::arg("eps") = 1e-6)
        .def("check", &Linear::look)
        .def_readonly("w_codes", &Linear::w)
        .def_readonly("w_scale", &Linear::scale)
        .def_readonly("bias", &Linear::bias)
        .def_readonly("nonfinite", &Linear::nonfinite)
        .def_readonly("d_in", &Linear::d_in)
        .def_readonly("d_out", &Linear::d_out);
    py::class_<Gated>(m, "Gated")
        .def(py::init<const Linear&, const Linear&, const Linear&, const std::optional<std::string>&>())
        .def("__call__", &Gated::call, py::arg("x"), py::arg("out") = py::none(), py::arg("residual") = py::none(), py::arg("norm") = py::none(),
             py::arg("eps") = 1e-6)
        .def("check", &Gated::look)
        .def_readonly("word", &Gated::word)
        .def_readonly("captured_states", &Gated::taken);
    py::class_<Cache>(m, "Cache")
        .def(py::init<const Tensor&, const Tensor&, const Tensor&, const Tensor&>())
        .def("append", &Cache::append, py::arg("k"), py::arg("v"), py::arg("tok_off"), py::arg("lens"), py::arg("table"), py::arg("q") = py::none(),
             py::arg("cos") = py::none(), py::arg("sin") = py::none(), py::arg("interleaved") = false, py::arg("q_out") = py::none())
        .def("read", &Cache::read)
        .def("attend", &Cache::attend, py::arg("q"), py::arg("tok_off"), py::arg("lens"), py::arg("table"), py::arg("max_new"), py::arg("max_len"), py::arg("scale"),
             py::arg("causal"), py::arg("window"), py::arg("out"), py::arg("want_lse"), py::arg("zero_behind") = false)
        .def("check", &Cache::look)
        .def_readonly("k_codes", &Cache::k_codes)
        .def_readonly("k_scale", &Cache::k_scale)
        .def_readonly("v_codes", &Cache::v_codes)
        .def_readonly("v_scale", &Cache::v_scale)
        .def_readonly("word", &Cache::word);
}
