// Softmax statistics of one row of logits by one workgroup, and the gradient of a row, for the kernels of the log-probabilities and
// the losses (token_loss.hip).
//
//   t_j = (x_j - ref) c,  c = log2(e) / T;   e_j = 2^t_j;   S = sum e_j;   A = sum e_j t_j
//   ln p_j = ln 2 t_j - ln S;   H = -sum p_j ln p_j = ln S - ln 2 A / S
//
// The reference is a logit of the row and no exact maximum: the largest of the row's first entries, raised only where a later one
// exceeds it by 60 binary orders, which fp32 has room for.  So a wave keeps one scalar instead of a running maximum per thread, and
// the sums of the waves are on the same reference (which costs no rounding) unless one of them had to raise it.
// t is formed as a difference first: a masked logit of -inf or of the type's lowest value has e = 0, and a row that holds nothing but
// the lowest value is uniform.
#pragma once

#include "difr_device.hpp"

namespace difr {

// Entries of a vector that are not there, and t of entries without mass where e t is formed (0 times -inf is no number).
constexpr float kNoLogit = -__builtin_inff();
constexpr float kLeastExponent = -200.0f;
constexpr float kRaise = 60.0f;

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

// One wave's share of a row's sums.
template <int DT, bool ENT>
struct SoftmaxSums {
    float c;          // log2(e) / T
    float ref, base;  // the reference, -inf as long as there is none; what is subtracted: the same, or 0
    float most;       // logits beyond this raise the reference
    float S, A;       // this lane's

    __device__ __forceinline__ void begin(float first, float c_)
    {
        c = c_;
        S = A = 0.0f;
        set(first);
    }
    __device__ __forceinline__ void set(float r)
    {
        ref = r;
        base = r == kNoLogit ? 0.0f : r;
        most = r == kNoLogit ? r : r + kRaise / c;
    }
    __device__ __forceinline__ void add(const float x[Elem<DT>::kPerVec])
    {
        const float m = vector_max<DT>(x);
        if (__builtin_amdgcn_ballot_w64(m > most) != 0ull) raise(m);
#pragma unroll
        for (int j = 0; j < Elem<DT>::kPerVec; ++j) {
            const float t = (x[j] - base) * c;
            const float e = fast_exp2(t);
            S += e;
            if (ENT) A = __fmaf_rn(e, fmaxf(t, kLeastExponent), A);
        }
    }
    __device__ __forceinline__ void raise(float m)
    {
        asm volatile("" ::: "memory");  // keep this a real, rarely taken branch
        const float top = wave_max(m);
        const float d = ref == kNoLogit ? 0.0f : fmaxf((ref - top) * c, -1000.0f);
        const float f = fast_exp2(d);
        A = f * (A + d * S);
        S *= f;
        set(top);
    }
};

// What a row's statistics come to, in 64 bits.
struct RowSums {
    float ref;    // -inf: a row without a finite logit
    double S, A;
};

// Sums that LANES neighbouring lanes hold, joined in a fixed order for all of them.
template <int LANES, bool ENT>
__device__ __forceinline__ RowSums join_sums(RowSums s, float c)
{
    RowSums r = s;
#pragma unroll
    for (int off = LANES / 2; off >= 1; off >>= 1) r.ref = fmaxf(r.ref, __shfl_xor(r.ref, off, 64));
    if (__builtin_amdgcn_ballot_w64(s.ref != r.ref) != 0ull) {
        const double d = s.ref == kNoLogit ? 0.0 : fmax(((double)s.ref - (double)r.ref) * (double)c, -1000.0);
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

// The waves' sums, for the lanes of the first wave (the others get nothing of use).  lds: 3 floats for each wave.
template <int THREADS, int DT, bool ENT>
__device__ __forceinline__ RowSums merge_sums(const SoftmaxSums<DT, ENT> &w, float *lds)
{
    constexpr int W = THREADS / 64;
    const float S = wave_sum(w.S), A = ENT ? wave_sum(w.A) : 0.0f;
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) {
        lds[3 * wave] = w.ref;
        lds[3 * wave + 1] = S;
        lds[3 * wave + 2] = A;
    }
    __syncthreads();
    if (wave != 0) return RowSums{kNoLogit, 0.0, 0.0};
    const int i = threadIdx.x & (W - 1);  // a lane for each wave's sums, and copies of them
    return join_sums<W, ENT>(RowSums{lds[3 * i], lds[3 * i + 1], lds[3 * i + 2]}, w.c);
}

// Functions of 64-bit arguments to 1e-7 of the value (of 1, for the logarithm): the part that is a power of two is taken off in 64
// bits, the rest is small and goes through the fp32 function.  One wave evaluates them while the others wait; the 64-bit functions of
// the library take ten times as long.
__device__ __forceinline__ double ln_of(double S)
{
    const int k = S > 0.0 && S < (double)__builtin_inff() ? ilogb(S * 1.41421356) : 0;  // S 2^-k in [0.707, 1.414)
    return (double)k * 0.69314718055994530942 + (double)logf((float)ldexp(S, -k));
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
    float base, c, k0, k1;
    double at_token;  // g_t
    __device__ __forceinline__ void set(float ref, float c_, double S, double T, double a, double b, double H, double logp)
    {
        base = ref == kNoLogit ? 0.0f : ref;
        c = c_;
        const double z = 1.0 / (S * T);
        k0 = (float)(z * (-a - (b != 0.0 ? b * (H - ln_of(S)) : 0.0)));
        k1 = (float)(z * -b * 0.69314718055994530942);
        at_token = token_entry(a, b, H, logp, T);
    }
    // the same in fp32 and without the token's entry, for a stretch of a row (k0 and k1 to some 1e-7)
    __device__ __forceinline__ void set_stretch(float ref, float c_, float S, float T, float a, float b, float H)
    {
        base = ref == kNoLogit ? 0.0f : ref;
        c = c_;
        const float z = 1.0f / S / T;
        k0 = z * (-a - (b != 0.0f ? b * (H - logf(S)) : 0.0f));
        k1 = z * -b * kLn2;
    }
    template <bool ENT>
    __device__ __forceinline__ float operator()(float x) const
    {
        const float t = (x - base) * c;
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
