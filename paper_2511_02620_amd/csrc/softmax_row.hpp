// Softmax statistics of one row of logits by one workgroup, and the gradient of a row, for the kernels of the log-probabilities and
// the losses (token_loss.hip).
//
//   t_j = (x_j - ref) C,  C = log2(e) / T;   e_j = 2^t_j;   S = sum e_j;   A = sum e_j t_j
//   ln p_j = ln 2 t_j - ln S;   H = -sum p_j ln p_j = ln S - ln 2 A / S
//
// The reference is the largest logit so far, of the workgroup's first entries to begin with, and of a wave's from there on: one scalar of a
// wave and one ballot for each vector instead of a running maximum per thread.  In the end it is the row's largest, whose term is 1
// exactly: S >= 1 and A <= 0, so no log-probability comes out above 0 and no entropy below, and where one token has nearly all of the
// probability, S - 1 is what the others have.  (A reference up to 60 orders below the largest needs hardly a new one, but puts the error of an
// exponent of that size on the largest term: of 256 rows with such a token 118 had a log-probability above 0.)  Rows in random order
// take no longer for it (8192 x 128,256 bf16 310 us either way), rows that rise along the vocabulary, with a new maximum in every vector, up
// to a tenth (4096 x 128,256 167 us / 153, the policy loss 402 / 404).
// C is held in two parts: one of 24 bits alone would move all exponents the same way.  The second is taken at a vector's largest logit, which
// leaves 2^-23 of a term's distance from that and costs two operations for a vector.  The 16 bytes of a vector are summed in fp32, what
// comes after that in 64 bits.  Error of the log-probabilities of 8192 x 128,256 bf16, T = 0.7, against 64 bits: 2.6e-8, as much as their rounding; with
// the one-part factor 2.2e-7, by torch in fp32 5.7e-8.
// t is formed as a difference first: a masked logit of -inf or of the type's lowest value has e = 0, and a row that holds nothing but
// the lowest value is uniform.
#pragma once

#include "difr_device.hpp"
#include "token_loss.hpp"

namespace difr {

// Entries of a vector that are not there, and t of entries without mass where e t is formed (0 times -inf is no number).
constexpr float kNoLogit = -__builtin_inff();
constexpr float kLeastExponent = -200.0f;

template <int DT>
__device__ __forceinline__ u32x4 no_logits()
{
    return DT == 0 ? u32x4{0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u} : u32x4{0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u};
}

// Vector `i` (E entries) of a row of V; past its end, no logits.  A row that ends within a vector gives its last E entries, one load as for
// any other vector, and `row_vector_end` makes the vector of them (entry by entry they would be E loads, some of them one after another:
// the policy loss of 8000 x 5003 bf16 takes 50 us, 55 with those).
template <int DT>
__device__ __forceinline__ u32x4 row_vector_at(const typename Elem<DT>::type *row, int64_t i, int64_t V)
{
    constexpr int E = Elem<DT>::kPerVec;
    const int64_t base = i * E;
    if (base >= V) return no_logits<DT>();
    if (V < E) return load_vector<DT>(row, base, V);
    return *reinterpret_cast<const u32x4_any *>(row + (base < V - E ? base : V - E));
}
template <int DT>
__device__ __forceinline__ u32x4 row_vector_end(u32x4 q, int64_t i, int64_t V)
{
    constexpr int E = Elem<DT>::kPerVec, kBytes = 16 / E;
    const int64_t over = i * E + E - V;  // entries behind the row's end
    if (V < E || over <= 0 || over >= E) return q;
    const uint32_t none = no_logits<DT>().x, words = (uint32_t)over * kBytes / 4, bytes = (uint32_t)over * kBytes % 4;
    uint32_t w[5] = {q.x, q.y, q.z, q.w, none};
    if (words & 1) w[0] = w[1], w[1] = w[2], w[2] = w[3], w[3] = none;
    if (words & 2) w[0] = w[2], w[1] = w[3], w[2] = w[3] = none;
    u32x4 r;
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = __builtin_amdgcn_alignbyte(w[j + 1], w[j], bytes);
    return r;
}
template <int DT>
__device__ __forceinline__ u32x4 row_vector(const typename Elem<DT>::type *row, int64_t i, int64_t V)
{
    return row_vector_end<DT>(row_vector_at<DT>(row, i, V), i, V);
}

// A row from the 16 bytes on that its first entry lies in: `lead` entries that are not its own, and 16-byte loads that do not straddle
// lines (read past the caches, those are fetched twice: log-probabilities of 8192 x 99,991 bf16 327 us by such loads, 257 by these, of 8192 x
// 50,257 159 and 127).  The 16 bytes hold an entry of the row, so they can be read.
template <int DT>
struct AlignedRow {
    const typename Elem<DT>::type *x;
    int64_t V;
    int lead;
};
template <int DT>
__device__ __forceinline__ AlignedRow<DT> aligned_row(const typename Elem<DT>::type *row, int64_t V)
{
    const int lead = (int)((uintptr_t)row % 16u / sizeof(typename Elem<DT>::type));
    return AlignedRow<DT>{row - lead, V + lead, lead};
}

template <int DT>
__device__ __forceinline__ float vector_max(const float x[Elem<DT>::kPerVec])
{
    float m = fmaxf(x[0], x[1]);
#pragma unroll
    for (int j = 2; j < Elem<DT>::kPerVec; ++j) m = fmaxf(m, x[j]);
    return m;
}

// Reductions over a wave in six steps between neighbouring lanes, rows of 16 and halves: 50 cycles, where as many exchanges through LDS
// take 300, which a row pays for its first maximum, its sums and each new maximum.
template <int CTRL>
__device__ __forceinline__ float lane_before(float v, float none)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(none), __float_as_int(v), CTRL, 0xF, 0xF, false));
}
template <int CTRL>
__device__ __forceinline__ double lane_before(double v)  // 0 where there is none
{
    const int lo = __builtin_amdgcn_update_dpp(0, __double2loint(v), CTRL, 0xF, 0xF, false);
    const int hi = __builtin_amdgcn_update_dpp(0, __double2hiint(v), CTRL, 0xF, 0xF, false);
    return __hiloint2double(hi, lo);
}
// the largest of the lanes' values, in all of them
__device__ __forceinline__ float wave_top(float v)
{
    v = fmaxf(v, lane_before<0x111>(v, v));  // one lane before, of the row of 16
    v = fmaxf(v, lane_before<0x112>(v, v));
    v = fmaxf(v, lane_before<0x114>(v, v));
    v = fmaxf(v, lane_before<0x118>(v, v));
    v = fmaxf(v, lane_before<0x142>(v, v));  // the last of the row before
    v = fmaxf(v, lane_before<0x143>(v, v));  // the last of the first half
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
// the lanes' sum, in the last of them
__device__ __forceinline__ double wave_total(double v)
{
    v += lane_before<0x111>(v);
    v += lane_before<0x112>(v);
    v += lane_before<0x114>(v);
    v += lane_before<0x118>(v);
    v += lane_before<0x142>(v);
    v += lane_before<0x143>(v);
    return v;
}

// One wave's share of a row's sums.
template <int DT, bool ENT>
struct SoftmaxSums {
    ExponentScale c;
    float ref, base;  // the reference, -inf as long as there is none; what is subtracted: the same, or 0
    double S, A;      // this lane's

    __device__ __forceinline__ void begin(float first, ExponentScale c_)
    {
        c = c_;
        S = A = 0.0;
        set(first);
    }
    __device__ __forceinline__ void set(float r)
    {
        ref = r;
        base = r == kNoLogit ? 0.0f : r;
    }
    __device__ __forceinline__ void add(const float x[Elem<DT>::kPerVec])
    {
        constexpr int E = Elem<DT>::kPerVec;
        const float m = vector_max<DT>(x);
        if (__builtin_amdgcn_ballot_w64(m > ref) != 0ull) raise(m);
        const float rest = (m - base) * c.lo;
        float e[E], t[E];
#pragma unroll
        for (int j = 0; j < E; ++j) {
            t[j] = __fmaf_rn(x[j] - base, c.hi, rest);
            e[j] = fast_exp2(t[j]);
            if (ENT) t[j] = fmaxf(t[j], kLeastExponent);
        }
        float s = (e[0] + e[1]) + (e[2] + e[3]);
        if constexpr (DT == 0) s += (e[4] + e[5]) + (e[6] + e[7]);
        S += (double)s;
        if constexpr (ENT) {
            float a = e[0] * t[0], o = e[1] * t[1];
#pragma unroll
            for (int j = 2; j < E; j += 2) {
                a = __fmaf_rn(e[j], t[j], a);
                o = __fmaf_rn(e[j + 1], t[j + 1], o);
            }
            a += o;
            A += (double)a;
        }
    }
    __device__ __forceinline__ void raise(float m)
    {
        asm volatile("" ::: "memory");  // keep this a real, rarely taken branch
        const float top = wave_top(m);
        const float low = ref - top;
        const float d = ref == kNoLogit ? 0.0f : fmaxf(__fmaf_rn(low, c.lo, low * c.hi), -1000.0f);
        const double f = (double)fast_exp2(d);
        if (ENT) A = f * (A + (double)d * S);
        S *= f;
        set(top);
    }
};

// What a row's statistics come to.
struct RowSums {
    float ref;    // -inf: a row without a finite logit
    double S, A;
};

// Sums that LANES neighbouring lanes hold, joined in a fixed order for all of them.
template <int LANES, bool ENT>
__device__ __forceinline__ RowSums join_sums(RowSums s, ExponentScale c)
{
    RowSums r = s;
#pragma unroll
    for (int off = LANES / 2; off >= 1; off >>= 1) r.ref = fmaxf(r.ref, __shfl_xor(r.ref, off, 64));
    if (__builtin_amdgcn_ballot_w64(s.ref != r.ref) != 0ull) {
        const double d = s.ref == kNoLogit ? 0.0 : fmax(((double)s.ref - (double)r.ref) * c.whole(), -1000.0);
        const double k = rint(d), f = ldexp((double)fast_exp2((float)(d - k)), (int)k);  // (sums without a reference are 0)
        r.A = f * (s.A + d * s.S);
        r.S = f * s.S;
    }
#pragma unroll
    for (int off = LANES / 2; off >= 1; off >>= 1) {
        r.S += __shfl_xor(r.S, off, 64);
        if (ENT) r.A += __shfl_xor(r.A, off, 64);
    }
    return r;
}

// The waves' sums, for the lanes of the first wave (the others get nothing of use).  lds: one for each wave.
template <int THREADS, int DT, bool ENT>
__device__ __forceinline__ RowSums merge_sums(const SoftmaxSums<DT, ENT> &w, RowSums *lds)
{
    constexpr int W = THREADS / 64;
    const double S = wave_total(w.S), A = ENT ? wave_total(w.A) : 0.0;
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 63) lds[wave] = RowSums{w.ref, S, A};
    __syncthreads();
    if (wave != 0) return RowSums{kNoLogit, 0.0, 0.0};
    return join_sums<W, ENT>(lds[threadIdx.x & (W - 1)], w.c);  // a lane for each wave's sums, and copies of them
}

// Functions of 64-bit arguments to 2e-7 of the value, ln near 1 and e^u - 1 near 0 too: the part that is a power of two is taken off in 64
// bits, the rest is small and goes through the fp32 function.  One wave evaluates them while the others wait; the 64-bit functions of
// the library take ten times as long.
__device__ __forceinline__ double ln_of(double S)
{
    const int k = S > 0.0 && S < (double)__builtin_inff() ? ilogb(S * 1.41421356) : 0;  // S 2^-k in [0.707, 1.414)
    const double m = ldexp(S, -k);
    const float f = (float)m;  // and what that leaves of m, at the slope 1 / m: near 1 it is the logarithm
    return (double)k * 0.69314718055994530942 + ((double)logf(f) + (m - (double)f) * (double)__builtin_amdgcn_rcpf(f));
}
// (without branches: e^u runs to infinity and to 0 by itself, and NaN stays what it is)
__device__ __forceinline__ double exp_of(double u)
{
    const double k = fmin(fmax(rint(u * 1.44269504088896340736), -3000.0), 3000.0);
    return ldexp((double)expf((float)(u - k * 0.69314718055994530942)), (int)k);
}
__device__ __forceinline__ double expm1_of(double u) { return fabs(u) < 0.35 ? (double)expm1f((float)u) : exp_of(u) - 1.0; }
// e^d - d - 1, by its series where the difference would cancel (the terms left out are below 1e-8 of the sum); it goes to infinity on both sides
__device__ __forceinline__ double exp_less_line(double d)
{
    if (fabs(d) >= 0.35) return exp_of(d) - (d > 1e300 ? 1e300 : d) - 1.0;
    return d * d * (0.5 + d * (1.0 / 6 + d * (1.0 / 24 + d * (1.0 / 120 + d * (1.0 / 720 + d * (1.0 / 5040 + d * (1.0 / 40320)))))));
}

// ln p of a logit
__device__ __forceinline__ double row_log_prob(float x, float ref, double S, double T) { return ((double)x - (double)ref) / T - ln_of(S); }

// g_t of the token, for upstream gradients a (of ln p_t) and b (of the entropy)
__device__ __forceinline__ double token_entry(double a, double b, double H, double logp, double T)
{
    return (-a * expm1_of(logp) - (b != 0.0 && logp > -700.0 ? b * exp_of(logp) * (logp + H) : 0.0)) / T;
}

// Upstream gradients a (of ln p_t) and b (of the entropy) to the gradient in the logits:
//   g_j = (1/T) [ a (1[j = t] - p_j) - b p_j (ln p_j + H) ] = e_j (k0 + k1 t_j)  for j != t
struct RowGrad {
    float base, k0, k1;
    ExponentScale c;
    double at_token;  // g_t
    __device__ __forceinline__ void set(float ref, ExponentScale c_, double S, double T, double a, double b, double H, double logp)
    {
        base = ref == kNoLogit ? 0.0f : ref;
        c = c_;
        const double z = 1.0 / (S * T);
        k0 = (float)(z * (-a - (b != 0.0 ? b * (H - ln_of(S)) : 0.0)));
        k1 = (float)(z * -b * 0.69314718055994530942);
        at_token = token_entry(a, b, H, logp, T);
    }
    // the same in fp32 and without the token's entry, for a stretch of a row (k0 and k1 to some 1e-7)
    __device__ __forceinline__ void set_stretch(float ref, ExponentScale c_, float S, float T, float a, float b, float H)
    {
        base = ref == kNoLogit ? 0.0f : ref;
        c = c_;
        const float z = 1.0f / S / T;
        k0 = z * (-a - (b != 0.0f ? b * (H - logf(S)) : 0.0f));
        k1 = z * -b * kLn2;
    }
    // (the factor's second part is less than a step of bf16 for any t that leaves an e)
    template <int DT, bool ENT>
    __device__ __forceinline__ float operator()(float x) const
    {
        const float d = x - base;
        const float t = DT == 0 ? d * c.hi : __fmaf_rn(d, c.lo, d * c.hi);
        const float e = fast_exp2(t);
        return ENT ? e * __fmaf_rn(fmaxf(t, kLeastExponent), k1, k0) : e * k0;
    }
};

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}

template <int DT>
__device__ __forceinline__ u32x4 pack_vector(const float g[Elem<DT>::kPerVec])
{
    if constexpr (DT == 0)
        return u32x4{pack_bf16(g[0], g[1]), pack_bf16(g[2], g[3]), pack_bf16(g[4], g[5]), pack_bf16(g[6], g[7])};
    else
        return u32x4{__float_as_uint(g[0]), __float_as_uint(g[1]), __float_as_uint(g[2]), __float_as_uint(g[3])};
}

template <int DT>
__device__ __forceinline__ void store_element(typename Elem<DT>::type *p, float v)
{
    if constexpr (DT == 0)
        *p = (uint16_t)pack_bf16(v, v);
    else
        *p = v;
}

// Vector `i` of a row of V: whole, or the entries that there are.
template <int DT>
__device__ __forceinline__ void store_vector(typename Elem<DT>::type *row, int64_t i, int64_t V, u32x4 q)
{
    constexpr int E = Elem<DT>::kPerVec;
    const int64_t base = i * E;
    if (base + E <= V) {
        *reinterpret_cast<u32x4_any *>(row + base) = q;
        return;
    }
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int j = 0; j < E; ++j)
        if (base + j < V) {
            if constexpr (DT == 0)
                row[base + j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
            else
                row[base + j] = __uint_as_float(w[j]);
        }
}

}  // namespace difr
