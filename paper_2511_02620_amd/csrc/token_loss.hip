// Log-probabilities of logged tokens under stored logits, their gradient, and two losses on them: the clipped policy loss with a KL
// term and the preference loss over pairs of replies.  Formulas at the entry points in difr.h and in softmax_row.hpp.
#include <math.h>

#include <type_traits>

#include "difr_host.hpp"
#include "softmax_row.hpp"
#include "token_loss.hpp"

namespace difr {

constexpr double kLn2d = 0.69314718055994530942;

// An element at a uniform index of an array that the kernel does not write: a scalar load, which does not queue behind the row's.
template <class T>
__device__ __forceinline__ T uniform_load(const T *p, int64_t i)
{
    typedef const T __attribute__((address_space(4))) *constant;
    return ((constant)(uintptr_t)p)[i];
}

// A workgroup a row or a pair: grids of more threads than 32 bits count have a second dimension, and workgroups behind the last one.
constexpr int64_t kRowsAcross = (int64_t)1 << 21;
static dim3 row_grid(int64_t N)
{
    return dim3((unsigned)(N < kRowsAcross ? N : kRowsAcross), (unsigned)((N + kRowsAcross - 1) / kRowsAcross));
}
__device__ __forceinline__ int64_t row_of_workgroup() { return (int64_t)blockIdx.y * kRowsAcross + blockIdx.x; }

// Per-row scalars.
struct TokenRow {
    float T;
    ExponentScale c;
    int32_t t;
    bool temp_ok, token_ok;
};
__device__ __forceinline__ TokenRow load_token_row(const TokenRows &b, int64_t row)
{
    TokenRow r;
    r.T = b.temperatures ? uniform_load(b.temperatures, row) : b.temperature;
    r.temp_ok = r.T > 0.0f && r.T < __builtin_inff();
    r.t = uniform_load(b.tokens, row);
    r.token_ok = r.t >= 0 && (int64_t)r.t < b.V;
    r.c = b.temperatures ? exponent_scale(r.T) : b.scale;
    if (!r.temp_ok) r.c.hi = __builtin_nanf("");
    return r;
}

// A row's log-probability, entropy and flags from its sums.
struct RowResult {
    double logp, H;
    uint32_t flags;
};
__device__ __forceinline__ RowResult row_result(const TokenRow &r, const RowSums &s, float x_t)
{
    const double nan = __builtin_nan("");
    RowResult o;
    const bool ok = r.temp_ok && s.S > 0.0 && s.S < (double)__builtin_inff();
    o.flags = (ok ? 0u : kFlagNonfinite) | (r.token_ok ? 0u : kFlagInvalidClaim);
    o.logp = ok && r.token_ok ? row_log_prob(x_t, s.ref, s.S, (double)r.T) : nan;
    o.H = ok ? ln_of(s.S) - kLn2d * s.A / s.S : nan;
    return o;
}

// The row in vectors of 16 bytes from vector `first` on, U of a thread's in flight; f(values, index of the vector) is called by whole
// waves.  PAST: past the caches.
template <int DT, int THREADS, int U, bool PAST, class F>
__device__ __forceinline__ void stream_row(const typename Elem<DT>::type *row, int64_t first, int64_t V, F &&f)
{
    constexpr int E = Elem<DT>::kPerVec;
    const int tid = threadIdx.x;
    const int64_t nvec = V / E, total = (V + E - 1) / E;
    int64_t i = first;
    for (; i + (int64_t)U * THREADS <= nvec; i += (int64_t)U * THREADS) {
        u32x4 q[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const u32x4_any *p = reinterpret_cast<const u32x4_any *>(row + (i + u * THREADS + tid) * E);
            q[u] = PAST ? __builtin_nontemporal_load(p) : *p;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float x[E];
            unpack_vector<DT>(q[u], x);
            f(x, i + u * THREADS + tid);
        }
    }
    for (; i < total; i += THREADS) {
        float x[E];
        unpack_vector<DT>(row_vector<DT>(row, i + tid, V), x);
        f(x, i + tid);
    }
}

// A thread's first vector of a row with `lead` entries before it that are not its own.
template <int DT>
__device__ __forceinline__ void first_vector(u32x4 q, int lead, float x[Elem<DT>::kPerVec])
{
    unpack_vector<DT>(q, x);
#pragma unroll
    for (int j = 0; j < Elem<DT>::kPerVec - 1; ++j)
        if (threadIdx.x == 0 && j < lead) x[j] = kNoLogit;
}

// The row's sums, by all threads of the workgroup, for the first wave.
template <int DT, int THREADS, bool ENT>
__device__ __forceinline__ RowSums row_sums(const typename Elem<DT>::type *row, int64_t V, ExponentScale c, bool past, RowSums *lds)
{
    constexpr int E = Elem<DT>::kPerVec, W = THREADS / 64, U = 4;
    __shared__ float lds_first[W];
    const AlignedRow<DT> a = aligned_row<DT>(row, V);
    float x[E];
    first_vector<DT>(row_vector<DT>(a.x, threadIdx.x, a.V), a.lead, x);
    const float m = wave_top(vector_max<DT>(x));
    if ((threadIdx.x & 63) == 0) lds_first[threadIdx.x >> 6] = m;
    __syncthreads();
    float first = lds_first[0];
#pragma unroll
    for (int i = 1; i < W; ++i) first = fmaxf(first, lds_first[i]);
    SoftmaxSums<DT, ENT> s;
    s.begin(first, c);
    s.add(x);
    if (past)
        stream_row<DT, THREADS, U, true>(a.x, THREADS, a.V, [&](const float *v, int64_t) { s.add(v); });
    else
        stream_row<DT, THREADS, U, false>(a.x, THREADS, a.V, [&](const float *v, int64_t) { s.add(v); });
    return merge_sums<THREADS>(s, lds);
}

// Whether a row is read past the caches: all but the last 192 MB of the logits, which the 256 MB Infinity Cache may hold - they were
// written last, and a gradient that follows begins with them.  Forward pass, us, through the caches / past them: 8192 x 128,256 bf16 (2.1
// GB) 362 / 323, 2048 x 151,936 (622 MB) 119 / 102, 2048 x 50,257 (206 MB, read again and again) 35.6 / 44.7.
__device__ __forceinline__ bool read_past(const TokenRows &b, int64_t row)
{
    return (b.N - 1 - row) * b.ld * (b.dtype == 0 ? 2 : 4) > ((int64_t)192 << 20);
}

__device__ __forceinline__ void logprob_store(const LogProbOutputs &o, int64_t row, const TokenRow &r, const RowSums &s, float x_t)
{
    const RowResult q = row_result(r, s, x_t);
    o.logp[row] = (float)q.logp;
    if (o.stats) {
        o.stats[2 * row] = s.ref;
        o.stats[2 * row + 1] = (float)s.S;
    }
    if (o.entropy) o.entropy[row] = (float)q.H;
    o.flags[row] = (uint8_t)q.flags;
}
__device__ __forceinline__ void logprob_left_out(const LogProbOutputs &o, int64_t row)
{
    o.logp[row] = 0.0f;
    if (o.stats) o.stats[2 * row] = o.stats[2 * row + 1] = 0.0f;
    if (o.entropy) o.entropy[row] = 0.0f;
    o.flags[row] = 0;
}

template <int DT, int THREADS, bool ENT>
__global__ __launch_bounds__(THREADS) void token_logprob_kernel(TokenRows b, const uint8_t *mask, LogProbOutputs o)
{
    __shared__ RowSums lds[THREADS / 64];
    const int64_t row = row_of_workgroup();
    if (row >= b.N) return;
    typedef typename Elem<DT>::type elem;
    const elem *x = reinterpret_cast<const elem *>(b.logits) + row * b.ld;
    if (o.zero && threadIdx.x == 0) o.zero[row] = 0.0f;
    if (mask && mask[row] == 0) {
        if (threadIdx.x == 0) logprob_left_out(o, row);
        return;
    }
    const TokenRow r = load_token_row(b, row);
    const float x_t = r.token_ok ? Elem<DT>::to_float(x[r.t]) : 0.0f;
    const RowSums s = row_sums<DT, THREADS, ENT>(x, b.V, r.c, read_past(b, row), lds);
    if (threadIdx.x == 0) logprob_store(o, row, r, s, x_t);
}

// ---- few long rows: a row's sums by several workgroups ----

// A workgroup for every four rounds of a workgroup over the row, 64 to a row and 1024 in all at the most.  Two rounds and 2048, eight and
// 1024, eight and 512 are as fast where it counts.
constexpr int kPartRounds = 4, kMostParts = 64, kMostPartBlocks = 1024;
struct SplitRows {
    RowSums *sums;  // [N][parts]
    float *stats, *entropy, *grad_logp, *grad_entropy;  // [N][2], [N]: for the gradient of the policy loss
    int parts;
};

// One workgroup of `parts` to a row: the sums of its stretch, for a second kernel.  Rows that mask or weights leave out are not read.
template <int DT, bool ENT>
__global__ __launch_bounds__(kBlock) void row_part_kernel(TokenRows b, const uint8_t *mask, const float *weights, RowSums *sums, int parts)
{
    constexpr int E = Elem<DT>::kPerVec, U = 4;
    typedef typename Elem<DT>::type elem;
    __shared__ float lds_first[kWaves];
    __shared__ RowSums lds[kWaves];
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x / parts;
    const int part = blockIdx.x % parts;
    if ((mask && mask[row] == 0) || (weights && uniform_load(weights, row) == 0.0f)) return;
    const AlignedRow<DT> a = aligned_row<DT>(reinterpret_cast<const elem *>(b.logits) + row * b.ld, b.V);
    const int64_t nvec = a.V / E, begin = nvec * part / parts, end = nvec * (part + 1) / parts;
    const elem *x = a.x + begin * E;
    const int64_t len = part + 1 == parts ? a.V - begin * E : (end - begin) * E, total = (len + E - 1) / E;
    const int lead = part == 0 ? a.lead : 0;
    const ExponentScale c = load_token_row(b, row).c;
    SoftmaxSums<DT, ENT> s;
    for (int64_t i = 0; i < total; i += U * kBlock) {
        u32x4 q[U];
        if ((i + U * kBlock) * E <= len) {
#pragma unroll
            for (int u = 0; u < U; ++u) q[u] = *reinterpret_cast<const u32x4_any *>(x + (i + u * kBlock + tid) * E);
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) q[u] = row_vector<DT>(x, i + u * kBlock + tid, len);
        }
        float y[E];
        first_vector<DT>(q[0], i == 0 ? lead : 0, y);
        if (i == 0) {
            const float m = wave_top(vector_max<DT>(y));
            if ((tid & 63) == 0) lds_first[tid >> 6] = m;
            __syncthreads();
            s.begin(fmaxf(fmaxf(lds_first[0], lds_first[1]), fmaxf(lds_first[2], lds_first[3])), c);
        }
        s.add(y);
#pragma unroll
        for (int u = 1; u < U; ++u)
            if (i + u * kBlock < total) {
                unpack_vector<DT>(q[u], y);
                s.add(y);
            }
    }
    const RowSums r = merge_sums<kBlock>(s, lds);
    if (tid == 0) sums[blockIdx.x] = r;
}

// The sums of a row's parts (64 or fewer), for all lanes of a wave.
template <bool ENT>
__device__ __forceinline__ RowSums joined(const RowSums *sums, int parts, int64_t row, ExponentScale c)
{
    const int lane = threadIdx.x;
    return join_sums<64, ENT>(lane < parts ? sums[row * parts + lane] : RowSums{kNoLogit, 0.0, 0.0}, c);
}

template <int DT, bool ENT>
__global__ __launch_bounds__(64) void logprob_join_kernel(TokenRows b, const uint8_t *mask, LogProbOutputs o, const RowSums *sums, int parts)
{
    const int64_t row = blockIdx.x;
    const bool left_out = mask && mask[row] == 0;
    const TokenRow r = load_token_row(b, row);
    const float x_t = r.token_ok && !left_out ? Elem<DT>::to_float(reinterpret_cast<const typename Elem<DT>::type *>(b.logits)[row * b.ld + r.t]) : 0.0f;
    const RowSums s = joined<ENT>(sums, parts, row, r.c);
    if (threadIdx.x != 0) return;
    if (o.zero) o.zero[row] = 0.0f;
    if (left_out)
        logprob_left_out(o, row);
    else
        logprob_store(o, row, r, s, x_t);
}

// sum_n weight[n] value[n] by one workgroup, in 64 bits and a fixed order.  A weight of 0 leaves its value out.
struct WeightedSum {
    const float *value, *weight;  // weight null: `every`
    double every;
    int64_t n;
    float *out;
};
template <int THREADS>
__device__ __forceinline__ void weighted_sum(const WeightedSum &w)
{
    __shared__ double lds[THREADS / 64];
    double sum = 0.0;
    for (int64_t i = threadIdx.x; i < w.n; i += THREADS) {
        const double f = w.weight ? (double)w.weight[i] : w.every;
        if (f != 0.0) sum += f * (double)w.value[i];
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) sum += __shfl_xor(sum, off, 64);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        double s = lds[0];
        for (int i = 1; i < THREADS / 64; ++i) s += lds[i];
        *w.out = (float)s;
    }
}
constexpr int kSumThreads = 1024;
__global__ __launch_bounds__(kSumThreads) void weighted_sum_kernel(WeightedSum w) { weighted_sum<kSumThreads>(w); }

// The gradient of a row from its statistics: every workgroup has a stretch of 8 KB of it.  Bound by memory, and by how much of it is asked
// for at a time: two vectors of a thread and six waves to a SIMD, 12 MB over the device.  8192 x 128,256 bf16, forward and backward with
// the entropy / preference loss, us: 8 vectors in a loop 1178 / 1184; at once, eight waves: 4 vectors 1112 / 1122, 2 1073 / 1085,
// 1 1046 / 1024; 2 vectors and six waves 1018 / 1067, four 1057 / 1043; 1 vector and four 1320 / 1225 (2048 x 151,936, in the same order:
// 369 / 362, 329 / 329, 320 / 307, 356 / 311, 317 / 300, 343 / 308, 409 / 366).  The last rows come first, because the forward pass has
// left them in the Infinity Cache.
constexpr int kGradVectors = 2;  // of each thread

template <int DT, bool ENT>
__global__ __launch_bounds__(kBlock) __attribute__((amdgpu_waves_per_eu(6,6))) void token_grad_kernel(TokenRows b, const float *stats, const float *entropy, const float *grad_logp,
                                                            const float *grad_entropy, void *grad, int64_t ld_grad, WeightedSum sum)
{
    constexpr int E = Elem<DT>::kPerVec;
    typedef typename Elem<DT>::type elem;
    if (sum.out && blockIdx.x == 0 && blockIdx.y == 0) weighted_sum<kBlock>(sum);
    const int64_t row = b.N - 1 - blockIdx.y;
    const elem *x = reinterpret_cast<const elem *>(b.logits) + row * b.ld;
    elem *g = reinterpret_cast<elem *>(grad) + row * ld_grad;
    const int64_t first = (int64_t)blockIdx.x * (kBlock * kGradVectors), total = (b.V + E - 1) / E;
    const bool whole = (first + kBlock * kGradVectors) * E <= b.V;
    float a = uniform_load(grad_logp, row);
    const float h = ENT ? uniform_load(grad_entropy, row) : 0.0f;
    auto store = [&](int64_t i, u32x4 q) {
        if (whole)
            __builtin_nontemporal_store(q, reinterpret_cast<u32x4_any *>(g + i * E));
        else if (i < total)
            store_vector<DT>(g, i, b.V, q);
    };
    if (a == 0.0f && h == 0.0f) {
#pragma unroll
        for (int u = 0; u < kGradVectors; ++u) store(first + u * kBlock + threadIdx.x, u32x4{0u, 0u, 0u, 0u});
        return;
    }
    u32x4 q[kGradVectors];
#pragma unroll
    for (int u = 0; u < kGradVectors; ++u) {
        const int64_t i = first + u * kBlock + threadIdx.x;
        q[u] = whole ? *reinterpret_cast<const u32x4_any *>(x + i * E) : row_vector<DT>(x, i, b.V);
    }
    const TokenRow r = load_token_row(b, row);
    if (!r.token_ok && a != 0.0f) a = __builtin_nanf("");
    const float ref = uniform_load(stats, 2 * row), S = uniform_load(stats, 2 * row + 1), H = ENT ? uniform_load(entropy, row) : 0.0f;
    RowGrad k;
    k.set_stretch(ref, r.c, S, r.T, a, h, H);
    // the token's entry, where it is in this stretch (uniform)
    const bool here = r.token_ok && r.t >= first * E && r.t < (first + kBlock * kGradVectors) * E;
    float at_token = 0.0f;
    if (here) {
        const float x_t = Elem<DT>::to_float(x[r.t]);
        at_token = (float)token_entry((double)a, (double)h, (double)H, row_log_prob(x_t, ref, (double)S, (double)r.T), (double)r.T);
        __syncthreads();  // in place: every wave has read the token's logit before its place is written
    }
#pragma unroll
    for (int u = 0; u < kGradVectors; ++u) {
        const int64_t i = first + u * kBlock + threadIdx.x;
        float v[E];
        unpack_vector<DT>(q[u], v);
#pragma unroll
        for (int j = 0; j < E; ++j) v[j] = k.operator()<DT, ENT>(v[j]);
        if (here && i == r.t / E) {
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (r.t % E == j) v[j] = at_token;
        }
        store(i, pack_vector<DT>(v));
    }
}

// A row's part of the clipped policy loss, and what flows back into its log-probability and entropy (without the row's weight).
struct PolicyRow {
    double loss, kl, a;
    uint32_t flags;
};
__device__ __forceinline__ PolicyRow policy_row(const PolicyParams &p, int64_t row, double logp, double H)
{
    PolicyRow o;
    const double A = uniform_load(p.advantages, row);
    double ratio = p.old_logp ? exp_of(logp - (double)uniform_load(p.old_logp, row)) : (logp == logp ? 1.0 : logp);
    ratio = ratio > 1e300 ? 1e300 : ratio;  // a number, of which an advantage of 0 leaves nothing; any other makes it infinite in fp32
    const double lo = 1.0 - p.clip_low, hi = 1.0 + p.clip_high;
    const double inside = ratio < lo ? lo : (ratio > hi ? hi : ratio);
    const bool clipped = ratio * A > inside * A;
    o.flags = clipped ? kFlagClipped : 0u;
    o.loss = clipped ? -(inside * A) : -(ratio * A);
    o.a = clipped ? 0.0 : -(ratio * A);
    o.kl = 0.0;
    if (p.ref_logp) {
        const double d = (double)uniform_load(p.ref_logp, row) - logp, m = expm1_of(d);
        o.kl = exp_less_line(d);
        if (p.kl_coef != 0.0) {
            o.loss += p.kl_coef * o.kl;
            o.a -= p.kl_coef * m;
        }
    }
    if (p.entropy_coef != 0.0) o.loss -= p.entropy_coef * H;
    return o;
}

// What one wave makes of a row's sums: its outputs, and the coefficients of its gradient.
__device__ __forceinline__ PolicyRow policy_store(const PolicyParams &p, const PolicyOutputs &o, int64_t row, const RowResult &q)
{
    const PolicyRow l = policy_row(p, row, q.logp, q.H);
    o.row.logp[row] = (float)q.logp;
    o.token_loss[row] = (float)l.loss;
    if (o.row.entropy) o.row.entropy[row] = (float)q.H;
    if (o.kl) o.kl[row] = (float)l.kl;
    o.row.flags[row] = (uint8_t)(q.flags | l.flags);
    return l;
}
__device__ __forceinline__ RowGrad policy_finish(const PolicyParams &p, const PolicyOutputs &o, int64_t row, const TokenRow &r, const RowSums &s,
                                                 float x_t, double w)
{
    const RowResult q = row_result(r, s, x_t);
    const PolicyRow l = policy_store(p, o, row, q);
    RowGrad k;
    k.set(s.ref, r.c, s.S, (double)r.T, w * l.a, -p.entropy_coef * w, q.H, q.logp);
    return k;
}

__device__ __forceinline__ void policy_left_out(const PolicyOutputs &o, int64_t row)
{
    o.row.logp[row] = o.token_loss[row] = 0.0f;
    if (o.row.entropy) o.row.entropy[row] = 0.0f;
    if (o.kl) o.kl[row] = 0.0f;
    o.row.flags[row] = 0;
}

// The same for rows whose sums several workgroups have formed, with what token_grad_kernel needs.
template <int DT, bool ENT>
__global__ __launch_bounds__(64) void policy_join_kernel(TokenRows b, PolicyParams p, PolicyOutputs o, SplitRows ws)
{
    const int64_t row = blockIdx.x;
    const double w = p.weights ? (double)uniform_load(p.weights, row) : 1.0 / (double)b.N;
    const TokenRow r = load_token_row(b, row);
    const float x_t = r.token_ok && w != 0.0 ? Elem<DT>::to_float(reinterpret_cast<const typename Elem<DT>::type *>(b.logits)[row * b.ld + r.t]) : 0.0f;
    const RowSums s = joined<ENT>(ws.sums, ws.parts, row, r.c);
    if (threadIdx.x != 0) return;
    float a = 0.0f, h = 0.0f;
    if (w == 0.0) {
        policy_left_out(o, row);
    } else {
        const RowResult q = row_result(r, s, x_t);
        a = (float)(w * policy_store(p, o, row, q).a);
        h = (float)(-p.entropy_coef * w);
        ws.stats[2 * row] = s.ref;
        ws.stats[2 * row + 1] = (float)s.S;
        ws.entropy[row] = (float)q.H;
    }
    ws.grad_logp[row] = a;
    ws.grad_entropy[row] = h;
}

template <int DT, int THREADS>
__device__ __forceinline__ void zero_row(typename Elem<DT>::type *g, int64_t V)
{
    const int64_t total = (V + Elem<DT>::kPerVec - 1) / Elem<DT>::kPerVec;
    for (int64_t i = threadIdx.x; i < total; i += THREADS) store_vector<DT>(g, i, V, u32x4{0u, 0u, 0u, 0u});
}

// Loss and gradient of rows that fit a workgroup's registers: a row is read once and its gradient written once, which is all the memory
// traffic there has to be.  A thread holds R vectors of 16 bytes and one more of the row's ragged end; `full`, the number of vectors that
// every thread has, is R - 8 to R.  A compute unit's registers hold one row of 150,000 bf16 logits (512 threads of 256 registers: with
// 1024 of 128 each what is not the row does not fit), or a few shorter ones, so a workgroup keeps the memory busy by itself: as it
// forms the gradient of a row, vector by vector, the registers that come free take the next row.  LDS: what a longer row has beyond its
// registers, up to 17 rounds of vectors, is held in LDS, copied there by the memory system; a thread's vectors are its own there too.
// Stores go past the caches, loads do not: the gradient is not read soon, the logits may have been written just now (8192 x 151,936 bf16,
// us: stores through the caches 1105, past them 1045, loads too 1042; 256 rows that lie in the Infinity Cache 44, loads past it 50).
// AHEAD: a row that leaves LDS free, and has the compute unit to itself, has its first rounds copied there while the row before is still
// summed, when nothing else would ask for memory; half of the loads are out of the way then when the stores come.  us, before / with it:
// 8192 x 151,936 bf16 1059 / 1027 (a tenth of the tokens left out: 1049 / 985), x 128,256 875 / 813, x 100,000 727 / 629, 4096 x 65,536 fp32
// 427 / 390;  shorter rows, two to a compute unit, which cover each other's sums already: 8192 x 50,257 376 / 392, without it.
constexpr int kLdsRounds = 17, kAheadRounds = 19;
constexpr int wait_for(int left) { return (left & 15) | 0x0F70 | (left >> 4) << 14; }  // s_waitcnt, vector memory: until so many are left
template <int DT, int THREADS, int R, bool ENT, bool LDS>
__global__ __launch_bounds__(THREADS, R <= 8 ? 4 : R <= 16 ? 3 : 2) void policy_held_kernel(TokenRows b, PolicyParams p, PolicyOutputs o, int full,
                                                                                            int lds_rounds)
{
    constexpr int E = Elem<DT>::kPerVec, W = THREADS / 64, AHEAD = LDS || R < 24 || THREADS < 512 ? 0 : R - 8 < kAheadRounds ? R - 8 : kAheadRounds;
    __shared__ __attribute__((aligned(16))) uint8_t lds_row[LDS ? kLdsRounds * THREADS * 16 : AHEAD ? AHEAD * THREADS * 16 : 16];
    typedef typename Elem<DT>::type elem;
    __shared__ float lds_first[W];
    __shared__ RowSums lds[W];
    __shared__ RowGrad lds_grad;
    const int tid = threadIdx.x;
    const int64_t step = gridDim.x, V = b.V;
    const bool every = p.weights == nullptr;
    const double share = 1.0 / (double)b.N;
    const elem *const logits = reinterpret_cast<const elem *>(b.logits);
    elem *const grad = reinterpret_cast<elem *>(o.grad);

    u32x4 q[R], q_end;
    const int64_t end = (int64_t)(full + lds_rounds) * THREADS + tid;
    // a thread's vector in round r of them: a uniform address (kept from the compiler, which would carry 64-bit addresses for every
    // round in vector registers) and the same offset always
    const uint32_t off = (uint32_t)tid * 16u;
    auto round_of = [&](const elem *x, int r) {
        uint64_t a = (uint64_t)(uintptr_t)x + (uint64_t)(r * (THREADS * 16));
        asm("" : "+s"(a));
        return (__attribute__((address_space(1))) char *)a;
    };
    typedef __attribute__((address_space(1))) u32x4_any global_vector;
    auto load = [&](const elem *x, int r) { return *((const global_vector *)(round_of(x, r) + off)); };
    // rounds of a row from `first` on, into LDS
    const int wave_u = __builtin_amdgcn_readfirstlane(tid >> 6);
    auto copy_rounds = [&](const elem *x, int first, int rounds) {
        for (int l = 0; l < rounds; ++l) {
            const char *from = reinterpret_cast<const char *>(x) + (int64_t)(first + l) * (THREADS * 16);
            const uint32_t to = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)lds_row + (uint32_t)(l * THREADS * 16 + wave_u * 1024);
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
            asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %0" : : "s"(from), "v"(off), "s"(to) : "memory", "m0");
#pragma clang diagnostic pop
        }
    };
    auto lds_vector = [&](int l) { return *reinterpret_cast<const u32x4 *>(lds_row + (l * THREADS + tid) * 16); };
    // the next row that counts, from `row` on; those before it get their zeros
    auto next_live = [&](int64_t row, float &w) {
        while (row < b.N) {
            w = every ? 1.0f : uniform_load(p.weights, row);
            if (w != 0.0f) break;
            if (tid == 0) policy_left_out(o, row);
            zero_row<DT, THREADS>(grad + row * o.ld_grad, V);
            row += step;
        }
        return row;
    };
    float w;
    int64_t row = next_live(blockIdx.x, w);
    if (row < b.N) {
        const elem *x = logits + row * b.ld;
        if (LDS) copy_rounds(x, R, lds_rounds);
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (r < R - 8 || r < full) q[r] = load(x, r);
        q_end = row_vector_at<DT>(x, end, V);
    }
    while (row < b.N) {
        const TokenRow t = load_token_row(b, row);
        const elem x_t = logits[row * b.ld + (t.token_ok ? t.t : 0)];
        q_end = row_vector_end<DT>(q_end, end, V);
        // the reference, of the row's first and last entries
        {
            float y[E];
            unpack_vector<DT>(q_end, y);
            float m = vector_max<DT>(y);
            if (full > 0) {
                unpack_vector<DT>(q[0], y);
                m = fmaxf(m, vector_max<DT>(y));
            }
            m = wave_top(m);
            if ((tid & 63) == 0) lds_first[tid >> 6] = m;
        }
        __syncthreads();
        float first = lds_first[0];
#pragma unroll
        for (int i = 1; i < W; ++i) first = fmaxf(first, lds_first[i]);
        SoftmaxSums<DT, ENT> s;
        s.begin(first, t.c);
        if (LDS) {
            // (memory operations end in order: the copies are older than the loads and stores of the rounds that every row has)
            asm volatile("s_waitcnt vmcnt(%0)" : : "n"(R - 8) : "memory");
            for (int l = 0; l < lds_rounds; ++l) {
                float y[E];
                unpack_vector<DT>(lds_vector(l), y);
                s.add(y);
            }
        }
        auto add_rounds = [&](auto first, auto end) {
#pragma unroll
            for (int r = first; r < end; ++r)
                if (r < R - 8 || r < full) {
                    float y[E];
                    unpack_vector<DT>(q[r], y);
                    s.add(y);
                    __builtin_amdgcn_sched_barrier(0);
                }
        };
        float w_next = 0.0f;
        int64_t next = 0;
        add_rounds(std::integral_constant<int, 0>(), std::integral_constant<int, AHEAD>());
        if (AHEAD) {
            // every load of this row has ended before the next row's copies begin, so that no wait for a load is one for them
            __builtin_amdgcn_s_waitcnt(wait_for(0));
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (nor is a vector that they overwrite still on its way to its register)
            next = next_live(row + step, w_next);
            if (next < b.N) copy_rounds(logits + next * b.ld, 0, AHEAD);
        }
        add_rounds(std::integral_constant<int, AHEAD>(), std::integral_constant<int, R>());
        {
            float y[E];
            unpack_vector<DT>(q_end, y);
            s.add(y);
        }
        const RowSums sums = merge_sums<THREADS>(s, lds);
        if (AHEAD) {
            __builtin_amdgcn_s_waitcnt(wait_for(0));
            asm volatile("" ::: "memory");
        }
        if (tid == 0) lds_grad = policy_finish(p, o, row, t, sums, Elem<DT>::to_float(x_t), every ? share : (double)w);
        if (!AHEAD) next = next_live(row + step, w_next);
        __syncthreads();
        const RowGrad k = lds_grad;
        elem *const g = grad + row * o.ld_grad;
        const bool more = next < b.N;
        const elem *const xn = logits + (more ? next : row) * b.ld;  // (the last row is read again, and not used, rather than branched round)
        auto form = [&](u32x4 v) {
            float y[E];
            asm volatile("" : "+v"(v));  // unpacked anew: the compiler would keep the values from the first time, twice the registers
            unpack_vector<DT>(v, y);
#pragma unroll
            for (int j = 0; j < E; ++j) y[j] = k.operator()<DT, ENT>(y[j]);
            return pack_vector<DT>(y);
        };
        if (LDS) {
            for (int l = 0; l < lds_rounds; ++l)
                __builtin_nontemporal_store(form(lds_vector(l)), (global_vector *)(round_of(g, R + l) + off));
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // every vector has been read before its place is copied to
            copy_rounds(xn, R, lds_rounds);
        }
        {
            if (end * E < V) store_vector<DT>(g, end, V, form(q_end));
            if (more) q_end = row_vector_at<DT>(xn, end, V);
        }
        auto next_vector = [&](int r) { return r < AHEAD ? lds_vector(r) : load(xn, r); };
        auto form_rounds = [&](auto first, auto end) {
#pragma unroll
            for (int r = first; r < end; ++r)
                if (r < R - 8 || r < full) {
                    __builtin_nontemporal_store(form(q[r]), (global_vector *)(round_of(g, r) + off));
                    q[r] = next_vector(r);
                    __builtin_amdgcn_sched_barrier(0);
                }
        };
        form_rounds(std::integral_constant<int, 0>(), std::integral_constant<int, R>());
        // the token's own entry, by the thread that has written its vector (a wave's stores to one address keep their order)
        if (t.token_ok && (t.t / E) % THREADS == tid) store_element<DT>(g + t.t, (float)k.at_token);
        row = next;
        w = w_next;
    }
    if (LDS) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // no copy is on its way into LDS that the next workgroup has
}

// One workgroup a row, which it reads twice: the row's sums, then the gradient.  For rows that do not fit a compute unit, and for the
// loss alone.
template <int DT, int THREADS, bool ENT>
__global__ __launch_bounds__(THREADS) __attribute__((amdgpu_waves_per_eu(4, THREADS == 1024 ? 4 : 8))) void policy_kernel(TokenRows b, PolicyParams p, PolicyOutputs o)
{
    constexpr int E = Elem<DT>::kPerVec;
    __shared__ RowSums lds[THREADS / 64];
    __shared__ RowGrad lds_grad;
    const int64_t row = row_of_workgroup();
    if (row >= b.N) return;
    typedef typename Elem<DT>::type elem;
    const elem *x = reinterpret_cast<const elem *>(b.logits) + row * b.ld;
    elem *g = reinterpret_cast<elem *>(o.grad) + row * o.ld_grad;
    const double w = p.weights ? (double)uniform_load(p.weights, row) : 1.0 / (double)b.N;
    if (w == 0.0) {  // left out
        if (threadIdx.x == 0) policy_left_out(o, row);
        if (o.grad) zero_row<DT, THREADS>(g, b.V);
        return;
    }
    const TokenRow r = load_token_row(b, row);
    const float x_t = r.token_ok ? Elem<DT>::to_float(x[r.t]) : 0.0f;
    const RowSums s = row_sums<DT, THREADS, ENT>(x, b.V, r.c, !o.grad && read_past(b, row), lds);
    if (threadIdx.x == 0) lds_grad = policy_finish(p, o, row, r, s, x_t, w);
    if (!o.grad) return;
    __syncthreads();
    const RowGrad k = lds_grad;
    stream_row<DT, THREADS, 4, false>(x, 0, b.V, [&](const float *v, int64_t i) {
        float d[E];
#pragma unroll
        for (int j = 0; j < E; ++j) d[j] = k.operator()<DT, ENT>(v[j]);
        if (r.token_ok && i == r.t / E) {
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (r.t % E == j) d[j] = (float)k.at_token;
        }
        if (i * E < b.V) store_vector<DT>(g, i, b.V, pack_vector<DT>(d));
    });
}

// ---- pairs ----

// The pair of sequences 2 p (chosen) and 2 p + 1 (rejected): log-probabilities summed in 64 bits and a fixed order, the loss, and
// what flows back into each log-probability.
__global__ __launch_bounds__(kBlock) void pair_kernel(int64_t N, PreferenceParams p, PreferenceOutputs o)
{
    __shared__ double lds_sum[2][kWaves], lds_back[2];
    __shared__ int lds_count[2][kWaves];
    const int64_t pair = row_of_workgroup();
    if (pair >= p.S / 2) return;
    const int tid = threadIdx.x;
    int64_t lo[2], hi[2];
    for (int side = 0; side < 2; ++side) {
        lo[side] = max(p.seq_offsets[2 * pair + side], (int64_t)0);
        hi[side] = min(p.seq_offsets[2 * pair + side + 1], N);
        double sum = 0.0;
        int count = 0;
        for (int64_t n = lo[side] + tid; n < hi[side]; n += kBlock)
            if (!p.mask || p.mask[n]) {
                sum += (double)o.row.logp[n];
                ++count;
            }
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) {
            sum += __shfl_xor(sum, off, 64);
            count += __shfl_xor(count, off, 64);
        }
        if ((tid & 63) == 0) {
            lds_sum[side][tid >> 6] = sum;
            lds_count[side][tid >> 6] = count;
        }
    }
    __syncthreads();
    if (tid == 0) {
        double ratio[2], share[2];
        for (int side = 0; side < 2; ++side) {
            const double *l = lds_sum[side];
            const int *k = lds_count[side];
            const int count = k[0] + k[1] + k[2] + k[3];
            share[side] = p.average && count ? 1.0 / count : 1.0;
            const double total = ((l[0] + l[1]) + (l[2] + l[3])) * share[side];
            o.seq_logp[2 * pair + side] = (float)total;
            ratio[side] = total - (p.ref_seq_logp ? (double)p.ref_seq_logp[2 * pair + side] : 0.0);
        }
        const double h = p.beta * (ratio[0] - ratio[1]) - p.margin, eps = p.label_smoothing;
        const double soft = log1p(exp(-fabs(h)));  // -ln sigma(h) = soft + max(-h, 0)
        const double up = h >= 0.0 ? 1.0 / (1.0 + exp(-h)) : exp(h) / (1.0 + exp(h));
        const double down = h >= 0.0 ? exp(-h) / (1.0 + exp(-h)) : 1.0 / (1.0 + exp(h));
        // (a side of factor 0 is left out: it may be infinite, where a reply holds a token without probability)
        o.pair_loss[pair] = (float)((eps == 1.0 ? 0.0 : (1.0 - eps) * (soft + (h < 0.0 ? -h : 0.0))) + (eps == 0.0 ? 0.0 : eps * (soft + (h > 0.0 ? h : 0.0))));
        const double w = p.pair_weights ? (double)p.pair_weights[pair] : 2.0 / (double)p.S;
        const double back = w == 0.0 ? 0.0 : w * p.beta * (eps * up - (1.0 - eps) * down);
        lds_back[0] = back * share[0];
        lds_back[1] = -back * share[1];
    }
    if (!o.grad_logp) return;
    __syncthreads();
    for (int side = 0; side < 2; ++side) {
        const float back = (float)lds_back[side];
        for (int64_t n = lo[side] + tid; n < hi[side]; n += kBlock) o.grad_logp[n] = !p.mask || p.mask[n] ? back : 0.0f;
    }
}

// ---- launches ----

static int launched() { return hipGetLastError() == hipSuccess ? 0 : 1; }

// How many workgroups share a row.  One compute unit takes 10 us and more for the exponentials of a long row, two launches and a workspace
// cost 4 us of the host's time and 2 of the device's.  One workgroup a row / several, us a call (in a captured graph), log-probability
// with the entropy, policy loss with its gradient, bf16:  24 x 151,936 14.1 / 10.5 (13.7 / 8.3), 23.8 / 15.5 (23.2 / 12.4);  24 x 100,000
// 10.8 / 10.6 (10.6 / 8.0), 18.2 / 15.5 (17.9 / 12.1);  64 x 151,936 14.3 / 11.1 (13.7 / 9.7), 24.5 / 19.1 (23.4 / 18.1);  128 x 151,936
// 15.9 / 14.6, 28.0 / 28.0;  128 x 100,000 11.7 / 12.4, 20.2 / 22.7;  24 x 65,536 8.4 / 10.8 (8.1 / 6.8), 15.0 / 16.0 (14.5 / 10.7).
int token_parts(int64_t N, int64_t V, int dtype)
{
    if (N < 1 || N > 64 || V < 98304) return 1;
    const int64_t rounds = V / ((dtype == 0 ? 8 : 4) * kBlock);  // of a workgroup over a row
    int64_t parts = rounds / kPartRounds;
    if (parts > kMostParts) parts = kMostParts;
    return (int)(parts * N > kMostPartBlocks ? kMostPartBlocks / N : parts);
}

size_t token_workspace_bytes(int64_t N, int64_t V, int dtype)
{
    const int parts = token_parts(N, V, dtype);
    return parts < 2 ? 0 : (size_t)N * (parts * sizeof(RowSums) + 5 * sizeof(float));
}

static SplitRows split_rows(const TokenRows &b, void *workspace)
{
    SplitRows ws;
    ws.parts = token_parts(b.N, b.V, b.dtype);
    ws.sums = (RowSums *)workspace;
    ws.stats = (float *)(ws.sums + b.N * ws.parts);
    ws.entropy = ws.stats + 2 * b.N;
    ws.grad_logp = ws.entropy + b.N;
    ws.grad_entropy = ws.grad_logp + b.N;
    return ws;
}

template <int DT, bool ENT>
static void run_logprob(const TokenRows &b, const uint8_t *mask, const LogProbOutputs &o, const SplitRows &ws, hipStream_t stream)
{
    if (ws.parts > 1) {
        row_part_kernel<DT, ENT><<<dim3((unsigned)(b.N * ws.parts)), dim3(kBlock), 0, stream>>>(b, mask, nullptr, ws.sums, ws.parts);
        logprob_join_kernel<DT, ENT><<<dim3((unsigned)b.N), dim3(64), 0, stream>>>(b, mask, o, ws.sums, ws.parts);
    } else if (b.N <= 512 && b.V >= 32768) {
        // Long rows, two to a compute unit or fewer: all the threads that a workgroup can have for each.  256 / 1024 threads, us, bf16:
        // 256 x 151,936 24.8 / 16.8, 512 x 32,000 10.0 / 9.7, 512 x 16,384 6.2 / 7.2.
        token_logprob_kernel<DT, 1024, ENT><<<dim3((unsigned)b.N), dim3(1024), 0, stream>>>(b, mask, o);
    } else {
        token_logprob_kernel<DT, kBlock, ENT><<<row_grid(b.N), dim3(kBlock), 0, stream>>>(b, mask, o);
    }
}

int launch_token_logprob(const TokenRows &b, const uint8_t *mask, const LogProbOutputs &o, void *workspace, hipStream_t stream)
{
    const SplitRows ws = split_rows(b, workspace);
    if (b.dtype == 0)
        o.entropy ? run_logprob<0, true>(b, mask, o, ws, stream) : run_logprob<0, false>(b, mask, o, ws, stream);
    else
        o.entropy ? run_logprob<1, true>(b, mask, o, ws, stream) : run_logprob<1, false>(b, mask, o, ws, stream);
    return launched();
}

// `sum`: formed beside the gradient (out null: none)
static int run_backward(const TokenRows &b, const float *stats, const float *entropy, const float *grad_logp, const float *grad_entropy,
                        void *grad, int64_t ld_grad, WeightedSum sum, hipStream_t stream)
{
    const int64_t E = b.dtype == 0 ? 8 : 4, vectors = (b.V + E - 1) / E, per = kBlock * kGradVectors;
    constexpr int64_t kMostRows = 65535;  // of a launch: the grid's second dimension
    for (int64_t n = (b.N - 1) / kMostRows * kMostRows; n >= 0; n -= kMostRows) {
        TokenRows part = b;
        part.N = b.N - n < kMostRows ? b.N - n : kMostRows;
        part.logits = (const char *)b.logits + n * b.ld * (b.dtype == 0 ? 2 : 4);
        part.tokens = b.tokens + n;
        if (b.temperatures) part.temperatures = b.temperatures + n;
        void *g = (char *)grad + n * ld_grad * (b.dtype == 0 ? 2 : 4);
        const dim3 grid((unsigned)((vectors + per - 1) / per), (unsigned)part.N);
        const float *ent = entropy ? entropy + n : nullptr, *ge = grad_entropy ? grad_entropy + n : nullptr;
#define RUN(DT, ENT) token_grad_kernel<DT, ENT><<<grid, dim3(kBlock), 0, stream>>>(part, stats + 2 * n, ent, grad_logp + n, ge, g, ld_grad, sum)
        if (b.dtype == 0)
            ge ? RUN(0, true) : RUN(0, false);
        else
            ge ? RUN(1, true) : RUN(1, false);
#undef RUN
        sum.out = nullptr;
    }
    return launched();
}

int launch_token_logprob_backward(const TokenRows &b, const float *stats, const float *entropy, const float *grad_logp,
                                  const float *grad_entropy, void *grad, int64_t ld_grad, hipStream_t stream)
{
    return run_backward(b, stats, entropy, grad_logp, grad_entropy, grad, ld_grad, WeightedSum{nullptr, nullptr, 0.0, 0, nullptr}, stream);
}

template <int DT, bool ENT>
static void run_policy(const TokenRows &b, const PolicyParams &p, const PolicyOutputs &o, hipStream_t stream)
{
    constexpr int E = Elem<DT>::kPerVec;
    const int64_t vectors = b.V / E;
    // vectors that every thread has, for workgroups of so many threads; a row is held up to 38 of them, and 17 more in LDS
    const int64_t f256 = vectors / 256, f512 = vectors / 512;
    if (o.grad && f512 <= 38 + kLdsRounds) {
        const bool wide = f256 > 38 || (b.N <= 256 && f512 > 0);  // a row or fewer to a compute unit: more threads for it
        const int full = (int)(wide ? f512 : f256);
#define RUN(THREADS, R, LDS)                                                                                                     \
    {                                                                                                                            \
        const int64_t most = (int64_t)256 * ((R <= 8 ? 1024 : R <= 16 ? 768 : 512) / THREADS);                                   \
        policy_held_kernel<DT, THREADS, R, ENT, LDS><<<dim3((unsigned)(b.N < most ? b.N : most)), dim3(THREADS), 0, stream>>>(   \
            b, p, o, full < R ? full : R, full < R ? 0 : full - R);                                                              \
        return;                                                                                                                  \
    }
#define RUN_R(R)                                             \
    if (full <= R) {                                         \
        if (wide) RUN(512, R, false) else RUN(256, R, false) \
    }
        RUN_R(8) RUN_R(16) RUN_R(24) RUN_R(31) RUN_R(38)
        RUN(512, 38, true)
#undef RUN_R
#undef RUN
    }
    // With the gradient one workgroup to a compute unit, so that the rows stay in the Infinity Cache until they are read again.
    if (o.grad)
        policy_kernel<DT, 1024, ENT><<<row_grid(b.N), dim3(1024), 0, stream>>>(b, p, o);
    else
        policy_kernel<DT, kBlock, ENT><<<row_grid(b.N), dim3(kBlock), 0, stream>>>(b, p, o);
}

template <int DT, bool ENT>
static void run_policy_parts(const TokenRows &b, const PolicyParams &p, const PolicyOutputs &o, const SplitRows &ws, hipStream_t stream)
{
    row_part_kernel<DT, ENT><<<dim3((unsigned)(b.N * ws.parts)), dim3(kBlock), 0, stream>>>(b, nullptr, p.weights, ws.sums, ws.parts);
    policy_join_kernel<DT, ENT><<<dim3((unsigned)b.N), dim3(64), 0, stream>>>(b, p, o, ws);
}

int launch_policy_loss(const TokenRows &b, const PolicyParams &p, const PolicyOutputs &o, void *workspace, hipStream_t stream)
{
    const bool ent = o.row.entropy || p.entropy_coef != 0.0;
    if (token_parts(b.N, b.V, b.dtype) > 1) {
        const SplitRows ws = split_rows(b, workspace);
        if (b.dtype == 0)
            ent ? run_policy_parts<0, true>(b, p, o, ws, stream) : run_policy_parts<0, false>(b, p, o, ws, stream);
        else
            ent ? run_policy_parts<1, true>(b, p, o, ws, stream) : run_policy_parts<1, false>(b, p, o, ws, stream);
        if (o.grad)
            return run_backward(b, ws.stats, ws.entropy, ws.grad_logp, p.entropy_coef != 0.0 ? ws.grad_entropy : nullptr, o.grad, o.ld_grad,
                                WeightedSum{o.token_loss, p.weights, 1.0 / (double)b.N, b.N, o.loss}, stream);
    } else if (b.N > 0) {
        if (b.dtype == 0)
            ent ? run_policy<0, true>(b, p, o, stream) : run_policy<0, false>(b, p, o, stream);
        else
            ent ? run_policy<1, true>(b, p, o, stream) : run_policy<1, false>(b, p, o, stream);
    }
    weighted_sum_kernel<<<dim3(1), dim3(kSumThreads), 0, stream>>>(WeightedSum{o.token_loss, p.weights, b.N ? 1.0 / (double)b.N : 0.0, b.N, o.loss});
    return launched();
}

int launch_preference_loss(const TokenRows &b, const PreferenceParams &p, const PreferenceOutputs &o, void *workspace, hipStream_t stream)
{
    const int64_t pairs = p.S / 2;
    const bool back = o.grad && b.N > 0;
    LogProbOutputs row = o.row;
    row.zero = back ? o.grad_logp : nullptr;  // rows outside all sequences keep that
    if (b.N > 0 && launch_token_logprob(b, p.mask, row, workspace, stream)) return 1;
    if (pairs > 0) pair_kernel<<<row_grid(pairs), dim3(kBlock), 0, stream>>>(b.N, p, o);
    const WeightedSum sum{o.pair_loss, p.pair_weights, pairs ? 1.0 / (double)pairs : 0.0, pairs, o.loss};
    if (back) return run_backward(b, o.row.stats, nullptr, o.grad_logp, nullptr, o.grad, o.ld_grad, sum, stream);
    weighted_sum_kernel<<<dim3(1), dim3(kSumThreads), 0, stream>>>(sum);
    return launched();
}

}  // namespace difr
