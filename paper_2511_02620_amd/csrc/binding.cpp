// The Python side of the C ABI in native code: each function takes the tensors of one call, checks them, allocates the
// output tensors, and hands their device pointers and the current HIP stream to the entry point of the same name.
// No arithmetic of the method happens here.
//
// Why it is not Python: small batches spend their time here.  64 rows of 1024 fp32 logits (both scores, two poolings) took
// 55 us a pass with ctypes marshalling, all of it host work; the kernels need a third of that.
//
// Every function returns its outputs, or the difr_status as an int if the entry point refused the call, or None if an
// argument is not what it has to be: the Python caller then runs its own checks, which name the argument.
//
// The entry points are not linked: binding.py loads libdifr.so and passes their addresses to bind().
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include "../../include/difr.h"

namespace {

#define DIFR_ENTRIES(X)                                                                                                 \
    X(difr_gumbel_score)                                                                                                \
    X(difr_debug_gumbel_score_unfiltered)                                                                               \
    X(difr_ipt_score)                                                                                                   \
    X(difr_score_both)                                                                                                  \
    X(difr_score_both_peaked)                                                                                           \
    X(difr_score_both_admissible)                                                                                       \
    X(difr_ipt_score_filtered)                                                                                          \
    X(difr_gumbel_likelihood)                                                                                           \
    X(difr_score_both_filtered)                                                                                         \
    X(difr_admissible_count)                                                                                            \
    X(difr_split_workspace_bytes)                                                                                       \
    X(difr_score_split)                                                                                                 \
    X(difr_lmhead_workspace_bytes)                                                                                      \
    X(difr_lmhead_score)                                                                                                \
    X(difr_seq_reduce)                                                                                                  \
    X(difr_classify)                                                                                                    \
    X(difr_token_workspace_bytes)                                                                                       \
    X(difr_token_logprob)                                                                                               \
    X(difr_token_logprob_backward)                                                                                      \
    X(difr_policy_loss)                                                                                                 \
    X(difr_preference_loss)                                                                                             \
    X(difr_mx4_padded)                                                                                                  \
    X(difr_mx4_quantize)                                                                                                \
    X(difr_mx4_dequantize)                                                                                              \
    X(difr_mx4_product_workspace_bytes)                                                                                 \
    X(difr_mx4_product)                                                                                                 \
    X(difr_int4_padded)                                                                                                 \
    X(difr_int4_quantize)                                                                                               \
    X(difr_int4_dequantize)                                                                                             \
    X(difr_int4_product_workspace_bytes)                                                                                \
    X(difr_int4_product)                                                                                                \
    X(difr_draft_workspace_bytes)                                                                                       \
    X(difr_draft_verify)                                                                                                \
    X(difr_tree_verify)

struct Entries {
#define X(name) decltype(&::name) name = nullptr;
    DIFR_ENTRIES(X)
#undef X
} lib;

// dictionary keys, made once
#define DIFR_KEYS(X)                                                                                                    \
    X(margin) X(argmax) X(max_score) X(claimed_score) X(flags) X(logit_rank) X(dist) X(cdf_lo) X(cdf_hi) X(u)           \
    X(ipt_token) X(log_mass) X(count) X(log2_count) X(kept) X(pi) X(log_pi) X(tau) X(active) X(seq_mean) X(seq_max)     \
    X(seq_mismatch) X(seq_flag) X(cls) X(bits) X(logp) X(stats) X(entropy) X(loss) X(token_loss) X(kl) X(grad)           \
    X(grad_logp) X(pair_loss) X(seq_logp) X(codes) X(scales) X(zeros) X(accepted) X(tokens) X(nodes)
namespace key {
#define X(name) PyObject *name = nullptr;
DIFR_KEYS(X)
#undef X
}  // namespace key

// An argument that is not what the call needs: the caller gets None.
struct Refused {};

const at::Tensor &tensor(PyObject *o)
{
    if (!THPVariable_Check(o)) throw Refused();
    return THPVariable_Unpack(o);
}

// contiguous 1-D tensor of n elements (n < 0: any number) on `dev`
void *vec(PyObject *o, at::ScalarType type, int64_t n, const c10::Device &dev)
{
    const at::Tensor &t = tensor(o);
    if (t.scalar_type() != type || t.dim() != 1 || t.device() != dev || (n >= 0 && t.size(0) != n) || !t.is_contiguous()) throw Refused();
    return t.data_ptr();
}
void *vec_or_null(PyObject *o, at::ScalarType type, int64_t n, const c10::Device &dev)
{
    return o == Py_None ? nullptr : vec(o, type, n, dev);
}

double number(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw python_error();
    return v;
}
int64_t whole(PyObject *o)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw python_error();
    return v;
}
bool truth(PyObject *o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw python_error();
    return v != 0;
}

// The first eight arguments of every call on stored logits: logits, V, temperature, seeds, seq_ids, positions, claimed,
// temperatures.
struct Rows {
    difr_rows in;
    int64_t N;
    c10::Device dev;

    explicit Rows(PyObject *const *a) : dev(c10::kCUDA)
    {
        const at::Tensor &x = tensor(a[0]);
        if (!x.is_cuda() || x.dim() != 2 || (x.stride(1) != 1 && x.size(1) > 1)) throw Refused();
        if (x.scalar_type() == at::kBFloat16)
            in.dtype = DIFR_BF16;
        else if (x.scalar_type() == at::kFloat)
            in.dtype = DIFR_F32;
        else
            throw Refused();
        dev = x.device();
        N = x.size(0);
        in.logits = x.data_ptr();
        in.N = N;
        in.V = a[1] == Py_None ? x.size(1) : whole(a[1]);
        in.ld = N > 1 ? x.stride(0) : std::max(x.size(1), N ? x.stride(0) : (int64_t)0);
        in.temperature = (float)number(a[2]);
        const at::Tensor &s = tensor(a[3]);
        in.seeds = (const uint64_t *)vec(a[3], at::kLong, -1, dev);
        in.S = s.size(0);
        in.seq_ids = (const int32_t *)vec(a[4], at::kInt, N, dev);
        in.positions = (const uint32_t *)vec(a[5], at::kInt, N, dev);  // uint32 bit patterns held in int32
        in.claimed = (const int32_t *)vec_or_null(a[6], at::kInt, N, dev);
        in.temperatures = (const float *)vec_or_null(a[7], at::kFloat, N, dev);
    }
};
constexpr int kRowArgs = 8;

// One dictionary of output tensors, each in memory of its own, so that a caller may grow, save, keep or record any of them.  A call on
// few tokens has up to twelve: they come from torch's allocator without the way through its dispatcher (64 tokens, both scores and
// pooling, host time: 30 us by at::empty, 23 so; views of one allocation took 17, but one that was grown in place lay over the next).
struct Outputs {
    THPObjectPtr dict;
    c10::Device dev;
    const bool direct;  // nobody watches allocations, and nobody wants them filled
    explicit Outputs(c10::Device d)
        : dict(PyDict_New()), dev(d),
          direct(!c10::impl::TorchDispatchModeTLS::any_modes_set() && !at::globalContext().deterministicAlgorithms())
    {
        if (!dict) throw python_error();
    }
    at::Tensor make(at::ScalarType type, at::IntArrayRef shape)
    {
        if (!direct) return at::empty(shape, at::TensorOptions().dtype(type).device(dev));
        return at::Tensor(at::detail::empty_cuda(shape, type, dev, std::nullopt));
    }
    void *add(PyObject *name, at::ScalarType type, at::IntArrayRef shape)
    {
        at::Tensor t = make(type, shape);
        void *p = t.data_ptr();
        THPObjectPtr w(THPVariable_Wrap(std::move(t)));
        if (!w || PyDict_SetItem(dict, name, w) < 0) throw python_error();
        return p;
    }
    float *f32(PyObject *name, int64_t n) { return (float *)add(name, at::kFloat, {n}); }
    int32_t *i32(PyObject *name, int64_t n) { return (int32_t *)add(name, at::kInt, {n}); }
    uint8_t *u8(PyObject *name, int64_t n) { return (uint8_t *)add(name, at::kByte, {n}); }
};

void *stream_of(const c10::Device &dev) { return (void *)c10::hip::getCurrentHIPStream(dev.index()).stream(); }

// Calls the entry point on the device of its arguments, without the interpreter lock.
template <class F>
int enter(const c10::Device &dev, F &&f)
{
    const c10::DeviceGuard guard(dev);
    void *stream = stream_of(dev);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f(stream);
    Py_END_ALLOW_THREADS
    return rc;
}

PyObject *one(int rc, Outputs &a) { return rc ? PyLong_FromLong(rc) : a.dict.release(); }
PyObject *two(int rc, Outputs &a, Outputs &b) { return rc ? PyLong_FromLong(rc) : PyTuple_Pack(2, a.dict.get(), b.dict.get()); }
PyObject *three(int rc, Outputs &a, Outputs &b, Outputs &c)
{
    return rc ? PyLong_FromLong(rc) : PyTuple_Pack(3, a.dict.get(), b.dict.get(), c.dict.get());
}

// A small batch goes through difr_score_split, with a workspace from torch's allocator that belongs to the call's stream.
// Returns whether it did; the outputs are those of the call in `o`.
bool split(const Rows &r, const int32_t *claimed_ipt, const difr_scores &o, int *rc)
{
    const size_t need = lib.difr_split_workspace_bytes(r.in.N, r.in.V, r.in.dtype, o.count != nullptr);
    if (need == 0) return false;
    const at::Tensor ws = at::empty({(int64_t)need}, at::TensorOptions().dtype(at::kByte).device(r.dev));
    void *p = ws.data_ptr();
    *rc = enter(r.dev, [&](void *s) { return lib.difr_score_split(&r.in, claimed_ipt, &o, p, need, s); });
    return true;
}

// ---- one function per entry point; arguments beyond the row arguments in the comment ----

// claimed_gumbel side of a call that scores both estimators
struct GumbelSide {
    Outputs out;
    float *margin, *max_score, *claimed_score;
    int32_t *argmax, *rank = nullptr;
    uint8_t *flags;
    GumbelSide(c10::Device dev, int64_t N, bool want_rank) : out(dev)
    {
        margin = out.f32(key::margin, N);
        argmax = out.i32(key::argmax, N);
        max_score = out.f32(key::max_score, N);
        claimed_score = out.f32(key::claimed_score, N);
        flags = out.u8(key::flags, N);
        if (want_rank) rank = out.i32(key::logit_rank, N);
    }
};
struct IptSide {
    Outputs out;
    float *dist, *cdf_lo, *cdf_hi, *u, *log_mass = nullptr;
    int32_t *token = nullptr, *kept = nullptr;
    uint8_t *flags;
    IptSide(c10::Device dev, int64_t N, bool want_kept) : out(dev)
    {
        dist = out.f32(key::dist, N);
        cdf_lo = out.f32(key::cdf_lo, N);
        cdf_hi = out.f32(key::cdf_hi, N);
        u = out.f32(key::u, N);
        if (want_kept) kept = out.i32(key::kept, N);
        flags = out.u8(key::flags, N);
    }
};

difr_scores both_sides(const GumbelSide &g, const IptSide &i, double sigma, double eps)
{
    difr_scores sc = {};
    sc.margin = g.margin, sc.argmax = g.argmax, sc.max_score = g.max_score, sc.claimed_score = g.claimed_score;
    sc.flags_gumbel = g.flags, sc.rank_gumbel = g.rank;
    sc.dist = i.dist, sc.cdf_lo = i.cdf_lo, sc.cdf_hi = i.cdf_hi, sc.u = i.u, sc.ipt_token = i.token, sc.sigma = sigma, sc.eps = eps;
    sc.log_mass = i.log_mass, sc.flags_ipt = i.flags;
    return sc;
}

// rows, want_scores, unfiltered, want_rank
PyObject *gumbel_score(PyObject *const *a)
{
    Rows r(a);
    a += kRowArgs;
    Outputs o(r.dev);
    float *margin = o.f32(key::margin, r.N);
    int32_t *argmax = o.i32(key::argmax, r.N);
    uint8_t *flags = o.u8(key::flags, r.N);
    float *max_score = nullptr, *claimed_score = nullptr;
    if (truth(a[0])) {
        max_score = o.f32(key::max_score, r.N);
        claimed_score = o.f32(key::claimed_score, r.N);
    }
    const auto entry = truth(a[1]) ? lib.difr_debug_gumbel_score_unfiltered : lib.difr_gumbel_score;
    int32_t *rank = truth(a[2]) ? o.i32(key::logit_rank, r.N) : nullptr;
    int rc;
    difr_scores sc = {};
    sc.margin = margin, sc.argmax = argmax, sc.max_score = max_score, sc.claimed_score = claimed_score, sc.flags_gumbel = flags;
    sc.rank_gumbel = rank;
    if (entry == lib.difr_gumbel_score && split(r, nullptr, sc, &rc)) return one(rc, o);
    return one(enter(r.dev, [&](void *s) { return entry(&r.in, margin, argmax, max_score, claimed_score, flags, rank, s); }), o);
}

// rows, want_token, want_log_mass, sigma, eps, want_interval, want_rank
PyObject *ipt_score(PyObject *const *a)
{
    Rows r(a);
    a += kRowArgs;
    const double sigma = number(a[2]), eps = number(a[3]);
    Outputs o(r.dev);
    float *dist = o.f32(key::dist, r.N);
    uint8_t *flags = o.u8(key::flags, r.N);
    float *cdf_lo = nullptr, *cdf_hi = nullptr, *u = nullptr;
    if (truth(a[4])) {
        cdf_lo = o.f32(key::cdf_lo, r.N);
        cdf_hi = o.f32(key::cdf_hi, r.N);
        u = o.f32(key::u, r.N);
    }
    int32_t *token = truth(a[0]) ? o.i32(key::ipt_token, r.N) : nullptr;
    float *log_mass = truth(a[1]) ? o.f32(key::log_mass, r.N) : nullptr;
    int32_t *rank = truth(a[5]) ? o.i32(key::logit_rank, r.N) : nullptr;
    int rc;
    difr_scores sc = {};
    sc.dist = dist, sc.cdf_lo = cdf_lo, sc.cdf_hi = cdf_hi, sc.u = u, sc.ipt_token = token, sc.sigma = sigma, sc.eps = eps;
    sc.log_mass = log_mass, sc.flags_ipt = flags, sc.rank_ipt = rank;
    if (split(r, r.in.claimed, sc, &rc)) return one(rc, o);
    return one(enter(r.dev, [&](void *s) {
                   return lib.difr_ipt_score(&r.in, dist, cdf_lo, cdf_hi, u, token, sigma, eps, log_mass, flags, rank, s);
               }), o);
}

// Most peaked rows that are shared.  Shared rows regenerate the noise of all their vectors, the peaked kernel that of few, and is
// the faster one once the rows by themselves keep most of the chip busy.  Logits falling as -3 ln rank, T = 0.6, peaked kernel /
// shared rows, us: V = 151,936 256 rows 42.6 / 34.0, 384 rows 46.5 / 45.5, 512 rows 46.9 / 52.7, 740 rows 52 / 69; V = 100,000
// 256 rows 33.4 / 29.3, 384 rows 35.2 / 36.3; V = 65,000 256 rows 25.5 / 24.5, 310 rows 26.9 / 27.3.
constexpr int64_t kPeakedShared = 320;

// rows, claimed_ipt, peaked, want_rank, want_token, want_log_mass, sigma, eps
PyObject *score_both(PyObject *const *a)
{
    Rows r(a);
    a += kRowArgs;
    const int32_t *ci = (const int32_t *)vec_or_null(a[0], at::kInt, r.N, r.dev);
    const bool peaked = truth(a[1]);
    const auto entry = peaked ? lib.difr_score_both_peaked : lib.difr_score_both;
    const double sigma = number(a[5]), eps = number(a[6]);
    GumbelSide g(r.dev, r.N, truth(a[2]));
    IptSide i(r.dev, r.N, false);
    if (truth(a[3])) i.token = i.out.i32(key::ipt_token, r.N);
    if (truth(a[4])) i.log_mass = i.out.f32(key::log_mass, r.N);
    int rc;
    const bool whole = peaked && !g.rank && r.N > kPeakedShared;  // (with the rank the peaked call is the ordinary one)
    if (!whole && split(r, ci, both_sides(g, i, sigma, eps), &rc)) return two(rc, g.out, i.out);
    return two(enter(r.dev, [&](void *s) {
                   return entry(&r.in, ci, g.margin, g.argmax, g.max_score, g.claimed_score, g.flags, g.rank, i.dist, i.cdf_lo,
                                i.cdf_hi, i.u, i.token, sigma, eps, i.log_mass, i.flags, s);
               }), g.out, i.out);
}

// rows, claimed_ipt, delta
PyObject *score_both_admissible(PyObject *const *a)
{
    Rows r(a);
    a += kRowArgs;
    const int32_t *ci = (const int32_t *)vec_or_null(a[0], at::kInt, r.N, r.dev);
    const float delta = (float)number(a[1]);
    GumbelSide g(r.dev, r.N, false);
    IptSide i(r.dev, r.N, false);
    Outputs o(r.dev);
    int32_t *count = o.i32(key::count, r.N);
    float *log2_count = o.f32(key::log2_count, r.N);
    int rc;
    difr_scores sc = both_sides(g, i, 0.0, 0.0);
    sc.delta = delta, sc.count = count, sc.log2_count = log2_count;
    if (split(r, ci, sc, &rc)) return three(rc, g.out, i.out, o);
    return three(enter(r.dev, [&](void *s) {
                     return lib.difr_score_both_admissible(&r.in, ci, delta, g.margin, g.argmax, g.max_score, g.claimed_score,
                                                           g.flags, i.dist, i.cdf_lo, i.cdf_hi, i.u, i.flags, count, log2_count, s);
                 }), g.out, i.out, o);
}

// rows, max_score, delta, want_log2
PyObject *admissible_count(PyObject *const *a)
{
    Rows r(a);
    a += kRowArgs;
    const float *M = (const float *)vec_or_null(a[0], at::kFloat, r.N, r.dev);
    const float delta = (float)number(a[1]);
    Outputs o(r.dev);
    int32_t *count = o.i32(key::count, r.N);
    float *log2_count = truth(a[2]) ? o.f32(key::log2_count, r.N) : nullptr;
    return one(enter(r.dev, [&](void *s) { return lib.difr_admissible_count(&r.in, M, delta, count, log2_count, s); }), o);
}

// rows, top_k, top_p, want_token, want_log_mass, sigma, eps
PyObject *ipt_score_filtered(PyObject *const *a)
{
    Rows r(a);
    a += kRowArgs;
    const int32_t top_k = (int32_t)whole(a[0]);
    const float top_p = (float)number(a[1]);
    const double sigma = number(a[4]), eps = number(a[5]);
    IptSide i(r.dev, r.N, true);
    if (truth(a[2])) i.token = i.out.i32(key::ipt_token, r.N);
    if (truth(a[3])) i.log_mass = i.out.f32(key::log_mass, r.N);
    return one(enter(r.dev, [&](void *s) {
                   return lib.difr_ipt_score_filtered(&r.in, top_k, top_p, i.dist, i.cdf_lo, i.cdf_hi, i.u, i.token, sigma, eps,
                                                      i.log_mass, i.kept, i.flags, s);
               }), i.out);
}

// the likelihood side of the next two: z, top_k, top_p, s, sigma, want_active
struct Likelihood {
    difr_likelihood_params p;
    Outputs out;
    float *pi, *log_pi, *tau;
    int32_t *active = nullptr;
    uint8_t *flags;
    Likelihood(const Rows &r, PyObject *const *a) : out(r.dev)
    {
        p.z = (const float *)vec(a[0], at::kFloat, -1, r.dev);
        p.M = (int32_t)tensor(a[0]).size(0);
        p.top_k = (int32_t)whole(a[1]);
        p.top_p = (float)number(a[2]);
        const int64_t s = whole(a[3]);
        p.s = (int32_t)s;
        p.sigma = (float)number(a[4]);
        pi = out.f32(key::pi, r.N);
        log_pi = out.f32(key::log_pi, r.N);
        tau = out.f32(key::tau, r.N);
        flags = out.u8(key::flags, r.N);
        if (truth(a[5])) {
            void *q = out.add(key::active, at::kInt, {r.N, std::max(s, (int64_t)0)});
            if (s > 0) active = (int32_t *)q;
        }
    }
};

// rows, likelihood arguments
PyObject *gumbel_likelihood(PyObject *const *a)
{
    Rows r(a);
    Likelihood k(r, a + kRowArgs);
    return one(enter(r.dev, [&](void *s) { return lib.difr_gumbel_likelihood(&r.in, &k.p, k.pi, k.log_pi, k.tau, k.active, k.flags, s); }),
               k.out);
}

// rows, likelihood arguments, claimed_ipt, want_token, want_log_mass, sigma_ipt, eps
PyObject *score_both_filtered(PyObject *const *a)
{
    Rows r(a);
    Likelihood k(r, a + kRowArgs);
    a += kRowArgs + 6;
    const int32_t *ci = (const int32_t *)vec_or_null(a[0], at::kInt, r.N, r.dev);
    const double sigma = number(a[3]), eps = number(a[4]);
    IptSide i(r.dev, r.N, true);
    if (truth(a[1])) i.token = i.out.i32(key::ipt_token, r.N);
    if (truth(a[2])) i.log_mass = i.out.f32(key::log_mass, r.N);
    return two(enter(r.dev, [&](void *s) {
                   return lib.difr_score_both_filtered(&r.in, ci, &k.p, k.pi, k.log_pi, k.tau, k.active, k.flags, i.dist, i.cdf_lo,
                                                       i.cdf_hi, i.u, i.token, sigma, eps, i.log_mass, i.kept, i.flags, s);
               }), k.out, i.out);
}

// hidden, weight, temperature, seeds, seq_ids, positions, claimed_gumbel, claimed_ipt, temperatures, workspace,
// want_rank, want_log_mass, want_token, sigma, eps
PyObject *lmhead_score(PyObject *const *a)
{
    const at::Tensor &h = tensor(a[0]), &w = tensor(a[1]);
    for (const at::Tensor *t : {&h, &w})
        if (!t->is_cuda() || t->scalar_type() != at::kBFloat16 || t->dim() != 2 || (t->size(1) > 1 && t->stride(1) != 1)) throw Refused();
    const c10::Device dev = h.device();
    const int64_t N = h.size(0), d = h.size(1), V = w.size(0);
    if (w.size(1) != d || w.device() != dev) throw Refused();
    difr_lmhead in;
    in.hidden = h.data_ptr();
    in.weight = w.data_ptr();
    in.N = N;
    in.V = V;
    in.d = d;
    in.ldh = N > 1 ? h.stride(0) : d;
    in.ldw = V > 1 ? w.stride(0) : d;
    in.temperature = (float)number(a[2]);
    in.seeds = (const uint64_t *)vec(a[3], at::kLong, -1, dev);
    in.S = tensor(a[3]).size(0);
    in.seq_ids = (const int32_t *)vec(a[4], at::kInt, N, dev);
    in.positions = (const uint32_t *)vec(a[5], at::kInt, N, dev);
    in.claimed_gumbel = (const int32_t *)vec_or_null(a[6], at::kInt, N, dev);
    in.claimed_ipt = (const int32_t *)vec_or_null(a[7], at::kInt, N, dev);
    in.temperatures = (const float *)vec_or_null(a[8], at::kFloat, N, dev);
    const bool want_token = truth(a[12]);
    const double sigma = number(a[13]), eps = number(a[14]);
    at::Tensor ws;
    if (a[9] == Py_None) {
        const int64_t need = (int64_t)lib.difr_lmhead_workspace_bytes(N, V, d, want_token);
        ws = at::empty({std::max(need, (int64_t)8)}, at::TensorOptions().dtype(at::kByte).device(dev));
    } else {
        ws = tensor(a[9]);
        if (ws.device() != dev || ws.scalar_type() != at::kByte || !ws.is_contiguous()) throw Refused();
    }
    void *wsp = ws.data_ptr();
    const size_t wsn = (size_t)ws.numel();
    GumbelSide g(dev, N, truth(a[10]));
    IptSide i(dev, N, false);
    if (truth(a[11])) i.log_mass = i.out.f32(key::log_mass, N);
    if (want_token) i.token = i.out.i32(key::ipt_token, N);
    return two(enter(dev, [&](void *s) {
                   return lib.difr_lmhead_score(&in, g.margin, g.argmax, g.max_score, g.claimed_score, g.flags, g.rank, i.dist,
                                                i.cdf_lo, i.cdf_hi, i.u, i.token, sigma, eps, i.log_mass, i.flags, wsp, wsn, s);
               }), g.out, i.out);
}

// scores, row_flags, seq_offsets, threshold
PyObject *seq_reduce(PyObject *const *a)
{
    const at::Tensor &x = tensor(a[0]);
    if (!x.is_cuda()) throw Refused();
    const c10::Device dev = x.device();
    const float *scores = (const float *)vec(a[0], at::kFloat, -1, dev);
    const int64_t N = x.size(0);
    const uint8_t *flags = (const uint8_t *)vec_or_null(a[1], at::kByte, N, dev);
    const int64_t *off = (const int64_t *)vec(a[2], at::kLong, -1, dev);
    const int64_t S = tensor(a[2]).size(0) - 1;
    if (S < 0) throw Refused();
    const float threshold = (float)number(a[3]);
    Outputs o(dev);
    float *mean = o.f32(key::seq_mean, S), *mx = o.f32(key::seq_max, S);
    int32_t *mis = o.i32(key::seq_mismatch, S);
    uint8_t *fl = o.u8(key::seq_flag, S);
    return one(enter(dev, [&](void *s) { return lib.difr_seq_reduce(scores, flags, off, N, S, threshold, mean, mx, mis, fl, s); }), o);
}

// scores, ranks, tau, rank_cutoff, V, log2_admissible
PyObject *classify(PyObject *const *a)
{
    const at::Tensor &x = tensor(a[0]);
    if (!x.is_cuda()) throw Refused();
    const c10::Device dev = x.device();
    const float *scores = (const float *)vec(a[0], at::kFloat, -1, dev);
    const int64_t N = x.size(0);
    const int32_t *ranks = (const int32_t *)vec_or_null(a[1], at::kInt, N, dev);
    const float tau = (float)number(a[2]);
    const int64_t cutoff = whole(a[3]), V = whole(a[4]);
    const float *log2_adm = (const float *)vec_or_null(a[5], at::kFloat, N, dev);
    Outputs o(dev);
    uint8_t *cls = o.u8(key::cls, N);
    float *bits = o.f32(key::bits, N);
    return one(enter(dev, [&](void *s) { return lib.difr_classify(scores, ranks, N, tau, cutoff, V, log2_adm, cls, bits, s); }), o);
}

// ---- log-probabilities and losses ----

// The first five arguments of these calls: logits, V, temperature, tokens, temperatures.
struct TokenRows {
    difr_token_rows in;
    int64_t N;
    c10::Device dev;
    at::ScalarType type;

    explicit TokenRows(PyObject *const *a) : dev(c10::kCUDA)
    {
        const at::Tensor &x = tensor(a[0]);
        if (!x.is_cuda() || x.dim() != 2 || (x.stride(1) != 1 && x.size(1) > 1)) throw Refused();
        type = x.scalar_type();
        if (type != at::kBFloat16 && type != at::kFloat) throw Refused();
        in.dtype = type == at::kFloat ? DIFR_F32 : DIFR_BF16;
        dev = x.device();
        N = x.size(0);
        in.logits = x.data_ptr();
        in.N = N;
        in.V = a[1] == Py_None ? x.size(1) : whole(a[1]);
        if (in.V > x.size(1)) throw Refused();
        in.ld = N > 1 ? x.stride(0) : std::max(x.size(1), N ? x.stride(0) : (int64_t)0);
        in.temperature = (float)number(a[2]);
        in.tokens = (const int32_t *)vec(a[3], at::kInt, N, dev);
        in.temperatures = (const float *)vec_or_null(a[4], at::kFloat, N, dev);
    }
    size_t element() const { return in.dtype == DIFR_F32 ? 4 : 2; }
};
constexpr int kTokenRowArgs = 5;

// A tensor of the caller's has been written, if the call succeeded: its version goes up, as by torch's own operations in place, so that a
// graph that has saved it refuses to run backward.
void written(int rc, const at::Tensor &t)
{
    if (rc == 0 && t.defined() && !t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// Where a gradient [N, V] goes: a tensor of the caller's (the logits themselves, or one that does not overlap them), or a new one.
struct Grad {
    void *data = nullptr;
    int64_t ld = 0;
    at::Tensor t, theirs;
    Grad(const TokenRows &r, PyObject *out, Outputs &o)
    {
        if (out == Py_None) {
            t = o.make(r.type, {r.N, std::max(r.in.V, (int64_t)0)});
            data = t.data_ptr();
            ld = std::max(r.in.V, (int64_t)1);
            return;
        }
        theirs = t = tensor(out);
        if (t.device() != r.dev || t.scalar_type() != r.type || t.dim() != 2 || t.size(0) != r.N || t.size(1) != r.in.V ||
            (t.stride(1) != 1 && t.size(1) > 1))
            throw Refused();
        data = t.data_ptr();
        ld = r.N > 1 ? t.stride(0) : r.in.ld;  // (the pitch of a single row is never used)
        if (r.N > 1 && ld < r.in.V) throw Refused();
        const char *g = (const char *)data, *x = (const char *)r.in.logits;
        const size_t e = r.element();
        const size_t gn = r.N ? ((r.N - 1) * ld + r.in.V) * e : 0, xn = r.N ? ((r.N - 1) * r.in.ld + r.in.V) * e : 0;
        if (g < x + xn && x < g + gn && !(g == x && ld == r.in.ld)) throw Refused();
    }
    PyObject *wrap()
    {
        PyObject *w = THPVariable_Wrap(std::move(t));
        if (!w) throw python_error();
        return w;
    }
    void into(Outputs &o)
    {
        THPObjectPtr w(wrap());
        if (PyDict_SetItem(o.dict, key::grad, w) < 0) throw python_error();
    }
};

// The workspace of a call on token rows.
struct Scratch {
    at::Tensor t;
    void *data = nullptr;
    size_t bytes;
    Scratch(const TokenRows &r, Outputs &o) : bytes(lib.difr_token_workspace_bytes(r.in.N, r.in.V, r.in.dtype))
    {
        if (!bytes) return;
        t = o.make(at::kByte, {(int64_t)bytes});
        data = t.data_ptr();
    }
};

// token rows, want_entropy
PyObject *token_logprob(PyObject *const *a)
{
    TokenRows r(a);
    Outputs o(r.dev);
    float *logp = o.f32(key::logp, r.N);
    float *stats = (float *)o.add(key::stats, at::kFloat, {r.N, 2});
    float *entropy = truth(a[kTokenRowArgs]) ? o.f32(key::entropy, r.N) : nullptr;
    uint8_t *flags = o.u8(key::flags, r.N);
    const Scratch w(r, o);
    return one(enter(r.dev, [&](void *s) { return lib.difr_token_logprob(&r.in, logp, stats, entropy, flags, w.data, w.bytes, s); }), o);
}

// token rows, stats, grad_logp, entropy, grad_entropy, out
PyObject *token_logprob_backward(PyObject *const *a)
{
    TokenRows r(a);
    a += kTokenRowArgs;
    const at::Tensor &st = tensor(a[0]);
    if (st.device() != r.dev || st.scalar_type() != at::kFloat || st.dim() != 2 || st.size(0) != r.N || st.size(1) != 2 || !st.is_contiguous())
        throw Refused();
    const float *stats = (const float *)st.data_ptr(), *ga = (const float *)vec(a[1], at::kFloat, r.N, r.dev);
    const float *entropy = (const float *)vec_or_null(a[2], at::kFloat, r.N, r.dev);
    const float *ge = (const float *)vec_or_null(a[3], at::kFloat, r.N, r.dev);
    if (ge && !entropy) throw Refused();
    Outputs o(r.dev);
    Grad g(r, a[4], o);
    const int rc = enter(r.dev, [&](void *s) { return lib.difr_token_logprob_backward(&r.in, stats, entropy, ga, ge, g.data, g.ld, s); });
    written(rc, g.theirs);
    return rc ? PyLong_FromLong(rc) : g.wrap();
}

// token rows, advantages, weights, old_logp, ref_logp, clip_low, clip_high, kl_coef, entropy_coef, want_entropy, want_grad, out
PyObject *policy_loss(PyObject *const *a)
{
    TokenRows r(a);
    a += kTokenRowArgs;
    difr_policy p;
    p.advantages = (const float *)vec(a[0], at::kFloat, r.N, r.dev);
    p.weights = (const float *)vec_or_null(a[1], at::kFloat, r.N, r.dev);
    p.old_logp = (const float *)vec_or_null(a[2], at::kFloat, r.N, r.dev);
    p.ref_logp = (const float *)vec_or_null(a[3], at::kFloat, r.N, r.dev);
    p.clip_low = number(a[4]), p.clip_high = number(a[5]), p.kl_coef = number(a[6]), p.entropy_coef = number(a[7]);
    Outputs o(r.dev);
    float *loss = o.f32(key::loss, 1), *token_loss = o.f32(key::token_loss, r.N), *logp = o.f32(key::logp, r.N);
    float *entropy = truth(a[8]) ? o.f32(key::entropy, r.N) : nullptr;
    float *kl = p.ref_logp ? o.f32(key::kl, r.N) : nullptr;
    uint8_t *flags = o.u8(key::flags, r.N);
    void *grad = nullptr;
    int64_t ld = 0;
    at::Tensor theirs;
    if (truth(a[9])) {
        Grad g(r, a[10], o);
        grad = g.data, ld = g.ld, theirs = g.theirs;
        g.into(o);
    } else if (a[10] != Py_None) {
        throw Refused();
    }
    if (!r.N) grad = nullptr;
    const Scratch w(r, o);
    const int rc = enter(r.dev, [&](void *s) {
        return lib.difr_policy_loss(&r.in, &p, loss, token_loss, logp, entropy, kl, flags, grad, ld, w.data, w.bytes, s);
    });
    written(rc, theirs);
    return one(rc, o);
}

// token rows, seq_offsets, beta, mask, ref_seq_logp, pair_weights, label_smoothing, margin, average, want_grad, out
PyObject *preference_loss(PyObject *const *a)
{
    TokenRows r(a);
    a += kTokenRowArgs;
    difr_preference p;
    p.seq_offsets = (const int64_t *)vec(a[0], at::kLong, -1, r.dev);
    p.S = tensor(a[0]).size(0) - 1;
    if (p.S < 0 || p.S % 2) throw Refused();
    p.beta = number(a[1]);
    p.mask = (const uint8_t *)vec_or_null(a[2], at::kByte, r.N, r.dev);
    p.ref_seq_logp = (const float *)vec_or_null(a[3], at::kFloat, p.S, r.dev);
    p.pair_weights = (const float *)vec_or_null(a[4], at::kFloat, p.S / 2, r.dev);
    p.label_smoothing = number(a[5]), p.margin = number(a[6]), p.average = truth(a[7]);
    Outputs o(r.dev);
    float *loss = o.f32(key::loss, 1), *pair_loss = o.f32(key::pair_loss, p.S / 2), *seq_logp = o.f32(key::seq_logp, p.S);
    float *logp = o.f32(key::logp, r.N), *stats = nullptr, *grad_logp = nullptr;
    uint8_t *flags = o.u8(key::flags, r.N);
    void *grad = nullptr;
    int64_t ld = 0;
    at::Tensor theirs;
    if (truth(a[8])) {
        stats = (float *)o.add(key::stats, at::kFloat, {r.N, 2});
        grad_logp = o.f32(key::grad_logp, r.N);
        Grad g(r, a[9], o);
        grad = g.data, ld = g.ld, theirs = g.theirs;
        g.into(o);
    } else if (a[9] != Py_None) {
        throw Refused();
    }
    if (!r.N) grad = nullptr;
    const Scratch w(r, o);
    const int rc = enter(r.dev, [&](void *s) {
        return lib.difr_preference_loss(&r.in, &p, loss, pair_loss, seq_logp, logp, stats, grad_logp, flags, grad, ld, w.data,
                                        w.bytes, s);
    });
    written(rc, theirs);
    return one(rc, o);
}

// ---- 4-bit floating point ----

int32_t float_type(at::ScalarType t)
{
    if (t == at::kBFloat16) return DIFR_BF16;
    if (t == at::kFloat) return DIFR_F32;
    throw Refused();
}

// [rows, K / 2] codes and [rows, K / 32] scales
struct Coded {
    const uint8_t *codes, *scales;
    int64_t rows, K;
    c10::Device dev;
    Coded(PyObject *c, PyObject *s) : dev(c10::kCUDA)
    {
        const at::Tensor &x = tensor(c), &y = tensor(s);
        if (!x.is_cuda() || x.scalar_type() != at::kByte || x.dim() != 2 || !x.is_contiguous()) throw Refused();
        dev = x.device();
        rows = x.size(0), K = 2 * x.size(1);
        if (y.device() != dev || y.scalar_type() != at::kByte || y.dim() != 2 || !y.is_contiguous() || y.size(0) != rows || K % 128 ||
            y.size(1) != K / 32)
            throw Refused();
        codes = (const uint8_t *)x.data_ptr(), scales = (const uint8_t *)y.data_ptr();
    }
};

// x
PyObject *mx4_quantize(PyObject *const *a)
{
    const at::Tensor &x = tensor(a[0]);
    if (!x.is_cuda() || x.dim() != 2 || (x.stride(1) != 1 && x.size(1) > 1)) throw Refused();
    const int32_t dtype = float_type(x.scalar_type());
    const int64_t N = x.size(0), d = x.size(1), K = lib.difr_mx4_padded(d);
    const int64_t ld = N > 1 ? x.stride(0) : d;
    Outputs o(x.device());
    uint8_t *codes = (uint8_t *)o.add(key::codes, at::kByte, {N, K / 2}), *scales = (uint8_t *)o.add(key::scales, at::kByte, {N, K / 32});
    return one(enter(x.device(), [&](void *s) { return lib.difr_mx4_quantize(x.data_ptr(), dtype, N, d, ld, codes, scales, s); }), o);
}

PyObject *wrapped(int rc, at::Tensor &t)
{
    if (rc) return PyLong_FromLong(rc);
    PyObject *w = THPVariable_Wrap(std::move(t));
    if (!w) throw python_error();
    return w;
}

// codes, scales, columns, fp32
PyObject *mx4_dequantize(PyObject *const *a)
{
    const Coded c(a[0], a[1]);
    const int64_t d = whole(a[2]);
    if (d < 1 || lib.difr_mx4_padded(d) != c.K) throw Refused();
    const bool f32 = truth(a[3]);
    Outputs o(c.dev);
    at::Tensor t = o.make(f32 ? at::kFloat : at::kBFloat16, {c.rows, d});
    const int rc = enter(c.dev, [&](void *s) {
        return lib.difr_mx4_dequantize(c.codes, c.scales, c.rows, d, t.data_ptr(), f32 ? DIFR_F32 : DIFR_BF16, d, s);
    });
    return wrapped(rc, t);
}

// a_codes, a_scales, b_codes, b_scales, fp32, out
PyObject *mx4_product(PyObject *const *a)
{
    const Coded x(a[0], a[1]), y(a[2], a[3]);
    if (y.dev != x.dev || y.K != x.K || !x.K) throw Refused();
    bool f32 = truth(a[4]);
    Outputs o(x.dev);
    at::Tensor t;
    int64_t ld = y.rows;
    if (a[5] == Py_None) {
        t = o.make(f32 ? at::kFloat : at::kBFloat16, {x.rows, y.rows});
    } else {
        t = tensor(a[5]);
        if (t.device() != x.dev || t.scalar_type() != (f32 ? at::kFloat : at::kBFloat16) || t.dim() != 2 || t.size(0) != x.rows ||
            t.size(1) != y.rows || (t.stride(1) != 1 && y.rows > 1) || (x.rows > 1 && t.stride(0) < y.rows))
            throw Refused();
        if (x.rows > 1) ld = t.stride(0);
    }
    const size_t need = lib.difr_mx4_product_workspace_bytes(x.rows, y.rows, x.K);
    at::Tensor ws;
    if (need) ws = o.make(at::kByte, {(int64_t)need});
    void *wsp = need ? ws.data_ptr() : nullptr;
    const int rc = enter(x.dev, [&](void *s) {
        return lib.difr_mx4_product(x.codes, x.scales, x.rows, y.codes, y.scales, y.rows, x.K, t.data_ptr(), f32 ? DIFR_F32 : DIFR_BF16,
                                    ld, wsp, need, s);
    });
    if (a[5] != Py_None) written(rc, t);
    return wrapped(rc, t);
}

// ---- 4-bit integers ----

// [rows, K / 2] codes, [rows, K / group] scales, and zero points or None
struct Coded4 {
    const uint8_t *codes, *zeros = nullptr;
    const void *scales;
    int64_t rows, K, group;
    c10::Device dev;
    Coded4(PyObject *c, PyObject *s, PyObject *z) : dev(c10::kCUDA)
    {
        const at::Tensor &x = tensor(c), &y = tensor(s);
        if (!x.is_cuda() || x.scalar_type() != at::kByte || x.dim() != 2 || !x.is_contiguous()) throw Refused();
        dev = x.device();
        rows = x.size(0), K = 2 * x.size(1);
        if (y.device() != dev || y.scalar_type() != at::kBFloat16 || y.dim() != 2 || !y.is_contiguous() || y.size(0) != rows || !K ||
            K % 128 || !y.size(1) || K % y.size(1))
            throw Refused();
        group = K / y.size(1);
        if (group != 32 && group != 64 && group != 128) throw Refused();
        codes = (const uint8_t *)x.data_ptr(), scales = y.data_ptr();
        if (z == Py_None) return;
        const at::Tensor &t = tensor(z);
        if (t.device() != dev || t.scalar_type() != at::kByte || t.dim() != 2 || !t.is_contiguous() || t.size(0) != rows || t.size(1) != y.size(1))
            throw Refused();
        zeros = (const uint8_t *)t.data_ptr();
    }
};

// x, group, zero_points
PyObject *int4_quantize(PyObject *const *a)
{
    const at::Tensor &x = tensor(a[0]);
    if (!x.is_cuda() || x.dim() != 2 || (x.stride(1) != 1 && x.size(1) > 1)) throw Refused();
    const int32_t dtype = float_type(x.scalar_type());
    const int64_t N = x.size(0), d = x.size(1), K = lib.difr_int4_padded(d), group = whole(a[1]);
    if (group != 32 && group != 64 && group != 128) throw Refused();
    const int64_t ld = N > 1 ? x.stride(0) : d;
    Outputs o(x.device());
    uint8_t *codes = (uint8_t *)o.add(key::codes, at::kByte, {N, K / 2});
    void *scales = o.add(key::scales, at::kBFloat16, {N, K / group});
    uint8_t *zeros = truth(a[2]) ? (uint8_t *)o.add(key::zeros, at::kByte, {N, K / group}) : nullptr;
    return one(enter(x.device(), [&](void *s) { return lib.difr_int4_quantize(x.data_ptr(), dtype, N, d, ld, (int32_t)group, codes, scales, zeros, s); }), o);
}

// codes, scales, zeros, columns, fp32
PyObject *int4_dequantize(PyObject *const *a)
{
    const Coded4 c(a[0], a[1], a[2]);
    const int64_t d = whole(a[3]);
    if (d < 1 || lib.difr_int4_padded(d) != c.K) throw Refused();
    const bool f32 = truth(a[4]);
    Outputs o(c.dev);
    at::Tensor t = o.make(f32 ? at::kFloat : at::kBFloat16, {c.rows, d});
    const int rc = enter(c.dev, [&](void *s) {
        return lib.difr_int4_dequantize(c.codes, c.scales, c.zeros, c.rows, d, (int32_t)c.group, t.data_ptr(), f32 ? DIFR_F32 : DIFR_BF16, d, s);
    });
    return wrapped(rc, t);
}

// hidden, codes, scales, zeros, fp32, out
PyObject *int4_product(PyObject *const *a)
{
    const at::Tensor &h = tensor(a[0]);
    const Coded4 c(a[1], a[2], a[3]);
    if (h.device() != c.dev || h.dim() != 2 || (h.stride(1) != 1 && h.size(1) > 1)) throw Refused();
    const int32_t type = float_type(h.scalar_type());
    const int64_t N = h.size(0), d = h.size(1), ldh = N > 1 ? h.stride(0) : d;
    if (d < 1 || lib.difr_int4_padded(d) != c.K || ldh < d) throw Refused();
    const bool f32 = truth(a[4]);
    Outputs o(c.dev);
    at::Tensor t;
    int64_t ld = c.rows;
    if (a[5] == Py_None) {
        t = o.make(f32 ? at::kFloat : at::kBFloat16, {N, c.rows});
    } else {
        t = tensor(a[5]);
        if (t.device() != c.dev || t.scalar_type() != (f32 ? at::kFloat : at::kBFloat16) || t.dim() != 2 || t.size(0) != N || t.size(1) != c.rows ||
            (t.stride(1) != 1 && c.rows > 1) || (N > 1 && t.stride(0) < c.rows))
            throw Refused();
        if (N > 1) ld = t.stride(0);
    }
    const size_t need = lib.difr_int4_product_workspace_bytes(N, d, type, (int32_t)c.group);
    at::Tensor ws;
    if (need) ws = o.make(at::kByte, {(int64_t)need});
    void *wsp = need ? ws.data_ptr() : nullptr;
    const int rc = enter(c.dev, [&](void *s) {
        return lib.difr_int4_product(h.data_ptr(), type, N, d, ldh, c.codes, c.scales, c.zeros, c.rows, (int32_t)c.group, t.data_ptr(),
                                     f32 ? DIFR_F32 : DIFR_BF16, ld, wsp, need, s);
    });
    if (a[5] != Py_None) written(rc, t);
    return wrapped(rc, t);
}

// ---- drafted tokens ----

// The first six arguments of these calls: logits, V, temperature, tokens, offsets, temperatures.
struct Drafts {
    difr_drafts in;
    int64_t R;
    c10::Device dev;
    at::ScalarType type;
    explicit Drafts(PyObject *const *a) : dev(c10::kCUDA)
    {
        const at::Tensor &x = tensor(a[0]), &off = tensor(a[4]);
        if (!x.is_cuda() || x.dim() != 2 || (x.stride(1) != 1 && x.size(1) > 1)) throw Refused();
        type = x.scalar_type();
        in.dtype = float_type(type);
        dev = x.device();
        in.offsets = (const int64_t *)vec(a[4], at::kLong, -1, dev);
        in.B = off.size(0) - 1;
        in.tokens = (const int32_t *)vec(a[3], at::kInt, -1, dev);
        in.D = tensor(a[3]).size(0);
        R = x.size(0);
        if (in.B < 0 || R != in.D + in.B) throw Refused();
        in.logits = x.data_ptr();
        in.V = a[1] == Py_None ? x.size(1) : whole(a[1]);
        if (in.V > x.size(1)) throw Refused();
        in.ld = R > 1 ? x.stride(0) : std::max(x.size(1), R ? x.stride(0) : (int64_t)0);
        in.temperature = (float)number(a[2]);
        in.temperatures = (const float *)vec_or_null(a[5], at::kFloat, R, dev);
    }
};
constexpr int kDraftArgs = 6;

struct DraftScratch {
    at::Tensor t;
    void *data = nullptr;
    size_t bytes;
    DraftScratch(const Drafts &r, bool draft, Outputs &o) : bytes(lib.difr_draft_workspace_bytes(r.in.B, r.in.D, r.in.V, r.in.dtype, draft))
    {
        if (!bytes) return;
        t = o.make(at::kByte, {(int64_t)bytes});
        data = t.data_ptr();
    }
};

// drafts, accept_u, sample_u, draft, draft_temperature, draft_temperatures
PyObject *draft_verify(PyObject *const *a)
{
    const Drafts r(a);
    a += kDraftArgs;
    difr_draft_chain c;
    c.accept_u = (const float *)vec(a[0], at::kFloat, r.in.D, r.dev);
    c.sample_u = (const float *)vec(a[1], at::kFloat, r.in.B, r.dev);
    c.draft = nullptr, c.ld = r.in.V;
    if (a[2] != Py_None) {
        const at::Tensor &y = tensor(a[2]);
        if (y.device() != r.dev || y.scalar_type() != r.type || y.dim() != 2 || y.size(0) != r.in.D || y.size(1) < r.in.V ||
            (y.stride(1) != 1 && y.size(1) > 1))
            throw Refused();
        c.draft = r.in.D ? y.data_ptr() : nullptr;
        c.ld = r.in.D > 1 ? y.stride(0) : std::max(y.size(1), r.in.D ? y.stride(0) : (int64_t)0);
    }
    c.temperature = (float)number(a[3]);
    c.temperatures = (const float *)vec_or_null(a[4], at::kFloat, r.in.D, r.dev);
    Outputs o(r.dev);
    int32_t *accepted = o.i32(key::accepted, r.in.B), *tokens = o.i32(key::tokens, r.R);
    float *logp = o.f32(key::logp, r.R);
    uint8_t *flags = o.u8(key::flags, r.R);
    const DraftScratch w(r, c.draft != nullptr, o);
    return one(enter(r.dev, [&](void *s) { return lib.difr_draft_verify(&r.in, &c, accepted, tokens, logp, flags, w.data, w.bytes, s); }), o);
}

// drafts, parents, sample_u
PyObject *tree_verify(PyObject *const *a)
{
    const Drafts r(a);
    a += kDraftArgs;
    const int32_t *parents = (const int32_t *)vec_or_null(a[0], at::kInt, r.in.D, r.dev);
    const float *u = (const float *)vec(a[1], at::kFloat, r.R, r.dev);
    Outputs o(r.dev);
    int32_t *accepted = o.i32(key::accepted, r.in.B), *tokens = o.i32(key::tokens, r.R), *nodes = o.i32(key::nodes, r.R);
    float *logp = o.f32(key::logp, r.R);
    uint8_t *flags = o.u8(key::flags, r.R);
    const DraftScratch w(r, false, o);
    return one(enter(r.dev, [&](void *s) { return lib.difr_tree_verify(&r.in, parents, u, accepted, tokens, nodes, logp, flags, w.data, w.bytes, s); }), o);
}

// ---- module ----

template <PyObject *(*F)(PyObject *const *), int N>
PyObject *fast(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "expected %d arguments, got %zd", N, n);
        return nullptr;
    }
    try {
        return F(args);
    } catch (const Refused &) {
        Py_RETURN_NONE;
    }
    END_HANDLE_TH_ERRORS
}

// bind({entry point: address})
PyObject *bind(PyObject *, PyObject *addresses)
{
#define X(name)                                                                                                         \
    {                                                                                                                   \
        PyObject *o = PyDict_GetItemString(addresses, #name);                                                           \
        void *p = o ? PyLong_AsVoidPtr(o) : nullptr;                                                                    \
        if (!p) {                                                                                                       \
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_KeyError, #name);                                              \
            return nullptr;                                                                                             \
        }                                                                                                               \
        lib.name = reinterpret_cast<decltype(&::name)>(p);                                                              \
    }
    DIFR_ENTRIES(X)
#undef X
    Py_RETURN_NONE;
}

template <PyObject *(*F)(PyObject *const *), int N>
constexpr PyMethodDef method(const char *name)
{
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&fast<F, N>)), METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {
    {"bind", bind, METH_O, nullptr},
    method<gumbel_score, kRowArgs + 3>("gumbel_score"),
    method<ipt_score, kRowArgs + 6>("ipt_score"),
    method<score_both, kRowArgs + 7>("score_both"),
    method<score_both_admissible, kRowArgs + 2>("score_both_admissible"),
    method<admissible_count, kRowArgs + 3>("admissible_count"),
    method<ipt_score_filtered, kRowArgs + 6>("ipt_score_filtered"),
    method<gumbel_likelihood, kRowArgs + 6>("gumbel_likelihood"),
    method<score_both_filtered, kRowArgs + 11>("score_both_filtered"),
    method<lmhead_score, 15>("lmhead_score"),
    method<seq_reduce, 4>("seq_reduce"),
    method<classify, 6>("classify"),
    method<token_logprob, kTokenRowArgs + 1>("token_logprob"),
    method<token_logprob_backward, kTokenRowArgs + 5>("token_logprob_backward"),
    method<policy_loss, kTokenRowArgs + 11>("policy_loss"),
    method<preference_loss, kTokenRowArgs + 10>("preference_loss"),
    method<mx4_quantize, 1>("mx4_quantize"),
    method<mx4_dequantize, 4>("mx4_dequantize"),
    method<mx4_product, 6>("mx4_product"),
    method<int4_quantize, 3>("int4_quantize"),
    method<int4_dequantize, 5>("int4_dequantize"),
    method<int4_product, 6>("int4_product"),
    method<draft_verify, kDraftArgs + 5>("draft_verify"),
    method<tree_verify, kDraftArgs + 2>("tree_verify"),
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native()
{
#define X(name)                                          \
    key::name = PyUnicode_InternFromString(#name);       \
    if (!key::name) return nullptr;
    DIFR_KEYS(X)
#undef X
    return PyModule_Create(&module);
}
