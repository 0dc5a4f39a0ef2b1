// Matrices in 4-bit integers, with a scale and a zero point for each group of 32, 64 or 128 elements of a row: quantisation and values
// (the product: int4_product.hip).  Format and formulas at the entry points in difr.h.
#include "difr_host.hpp"
#include "int4.hpp"
#include "softmax_row.hpp"

namespace difr {

// Eight elements of a row from k on, as fp32; zeros past the row's end.
template <int DT>
__device__ __forceinline__ void eight_elements(const typename Elem<DT>::type *p, int64_t k, int64_t d, float v[8])
{
    constexpr int E = Elem<DT>::kPerVec;
#pragma unroll
    for (int h = 0; h < 8; h += E) {
        if (k + h + E <= d) {
            unpack_vector<DT>(*reinterpret_cast<const u32x4_any *>(p + k + h), v + h);
        } else {
#pragma unroll
            for (int j = 0; j < E; ++j) v[h + j] = k + h + j < d ? Elem<DT>::to_float(p[k + h + j]) : 0.0f;
        }
    }
}

__device__ __forceinline__ uint16_t bf16_bits(float f)  // of a finite number that is not negative; ties to even
{
    const uint32_t u = __float_as_uint(f);
    return (uint16_t)((u + 0x7FFFu + (u >> 16 & 1u)) >> 16);
}

constexpr int kInt4Vectors = 2;  // of eight elements, of each thread

// A lane has eight elements of a row, GROUP / 8 lanes a group, whose extremes they exchange.  151,936 x 4096 bf16 400 to 455 us (1.56 GB at
// 3.4 to 3.9 TB/s).
template <int DT, int GROUP, bool ZEROS>
__global__ __launch_bounds__(kBlock) void int4_quantize_kernel(const typename Elem<DT>::type *x, int64_t N, int64_t d, int64_t ld,
                                                               uint8_t *codes, uint16_t *scales, uint8_t *zeros, uint32_t eights)
{
    const uint32_t first = blockIdx.x * (kBlock * kInt4Vectors) + threadIdx.x, total = (uint32_t)N * eights;
    float v[kInt4Vectors][8];
#pragma unroll
    for (int u = 0; u < kInt4Vectors; ++u) {
        const uint32_t i = first + u * kBlock, row = i < total ? i / eights : 0;
        eight_elements<DT>(x + row * ld, i < total ? (int64_t)(i - row * eights) * 8 : d, d, v[u]);
    }
#pragma unroll
    for (int u = 0; u < kInt4Vectors; ++u) {
        const uint32_t i = first + u * kBlock;
        float lo = 0.0f, hi = 0.0f;
        bool number = true;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            number &= fabsf(v[u][j]) < INFINITY;
            lo = fminf(lo, v[u][j]);
            hi = fmaxf(hi, v[u][j]);
        }
        hi = number ? hi : INFINITY;
        if (!ZEROS) hi = fmaxf(hi, -lo);
#pragma unroll
        for (int o = 1; o < GROUP / 8; o <<= 1) {
            hi = fmaxf(hi, __shfl_xor(hi, o));
            if (ZEROS) lo = fminf(lo, __shfl_xor(lo, o));
        }
        const float range = ZEROS ? hi - lo : hi;  // infinite where an element is no finite number
        const uint16_t bits = range < INFINITY ? bf16_bits(__fdiv_rn(range, ZEROS ? 15.0f : 7.0f)) : (uint16_t)0x7FC0u;
        const float s = __uint_as_float((uint32_t)bits << 16);
        const bool some = s > 0.0f;
        float z = 8.0f;
        if (ZEROS) z = some ? fminf(fmaxf(rintf(__fdiv_rn(-lo, s)), 0.0f), 15.0f) : 0.0f;
        // The quotient's whole number: by the inverse, which is off by less than 4e-6 (quotients are below 16), and by a division
        // where that lies as near to the middle of two (or is none: scales below the normal numbers)
        const float inverse = __fdiv_rn(1.0f, s);
        float n[8];
        bool sure = true;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float q = v[u][j] * inverse;
            n[j] = rintf(q);
            sure &= fabsf(q - n[j]) < 0.49999f;
        }
        if (!sure) {
#pragma unroll
            for (int j = 0; j < 8; ++j) n[j] = some ? rintf(__fdiv_rn(v[u][j], s)) : 0.0f;
        }
        uint32_t w = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) w |= (uint32_t)fminf(fmaxf(n[j] + z, 0.0f), 15.0f) << (4 * j);
        if (i < total) {
            reinterpret_cast<uint32_t *>(codes)[i] = w;
            if (i % (GROUP / 8) == 0) {
                scales[i / (GROUP / 8)] = bits;
                if (ZEROS) zeros[i / (GROUP / 8)] = (uint8_t)z;
            }
        }
    }
}

// One thread vectors of 16 bytes of the output, which go past the caches, a wave's without gaps between them: 151,936 x 4096 to fp32 515 us
// (5.4 TB/s); two vectors of a thread side by side, half lines of a wave's stores, 1201.
template <int DT>
__global__ __launch_bounds__(kBlock) void int4_dequantize_kernel(Int4Matrix m, int64_t d, typename Elem<DT>::type *x, int64_t ld, uint32_t per_row)
{
    constexpr int E = Elem<DT>::kPerVec;
    uint32_t w[kInt4Vectors];
    float s[kInt4Vectors], z[kInt4Vectors];
    int64_t row[kInt4Vectors], k[kInt4Vectors];
    const uint32_t total = (uint32_t)m.V * per_row;
#pragma unroll
    for (int u = 0; u < kInt4Vectors; ++u) {
        const uint32_t i = blockIdx.x * (kBlock * kInt4Vectors) + u * kBlock + threadIdx.x, r = i < total ? i / per_row : 0;
        row[u] = r;
        k[u] = i < total ? (int64_t)(i - r * per_row) * E : d;
        const int64_t at = k[u] < d ? k[u] : 0, g = row[u] * (m.K / m.group) + at / m.group;
        const uint8_t *const c = m.codes + row[u] * (m.K / 2) + at / 2;
        w[u] = DT == 0 ? *reinterpret_cast<const uint32_t *>(c) : (uint32_t) * reinterpret_cast<const uint16_t *>(c);
        s[u] = __uint_as_float((uint32_t)m.scales[g] << 16);
        z[u] = m.zeros ? (float)m.zeros[g] : 8.0f;
    }
#pragma unroll
    for (int u = 0; u < kInt4Vectors; ++u) {
        float v[E];
#pragma unroll
        for (int j = 0; j < E; ++j) v[j] = ((float)(w[u] >> (4 * j) & 15u) - z[u]) * s[u];
        if (k[u] + E <= d)
            __builtin_nontemporal_store(pack_vector<DT>(v), reinterpret_cast<u32x4_any *>(x + row[u] * ld + k[u]));
        else if (k[u] < d)
            store_vector<DT>(x + row[u] * ld, k[u] / E, d, pack_vector<DT>(v));
    }
}

static int launched() { return hipGetLastError() == hipSuccess ? 0 : 1; }

// Rows of a launch, of which the kernels count the eights in 32 bits.
static int64_t rows_at_once(int64_t eights) { return ((int64_t)1 << 30) / eights > 0 ? ((int64_t)1 << 30) / eights : 1; }

int launch_int4_quantize(const void *x, int dtype, int64_t N, int64_t d, int64_t ld, int group, uint8_t *codes, uint16_t *scales,
                         uint8_t *zeros, hipStream_t stream)
{
    const int64_t eights = (d + kInt4Slab - 1) / kInt4Slab * (kInt4Slab / 8), groups = eights * 8 / group, most = rows_at_once(eights), each = kBlock * kInt4Vectors;
    for (int64_t n = 0; n < N; n += most) {
        const int64_t rows = N - n < most ? N - n : most;
        const dim3 grid((unsigned)((rows * eights + each - 1) / each));
        uint8_t *c = codes + n * eights * 4, *z = zeros ? zeros + n * groups : nullptr;
        uint16_t *s = scales + n * groups;
#define RUN(DT, GROUP, ZEROS)                                                                                                              \
    int4_quantize_kernel<DT, GROUP, ZEROS><<<grid, dim3(kBlock), 0, stream>>>((const Elem<DT>::type *)x + n * ld, rows, d, ld, c, s, z, \
                                                                              (uint32_t)eights)
#define BY_GROUP(DT, ZEROS) group == 32 ? (void)(RUN(DT, 32, ZEROS)) : group == 64 ? (void)(RUN(DT, 64, ZEROS)) : (void)(RUN(DT, 128, ZEROS))
        if (dtype == 0) {
            if (zeros) BY_GROUP(0, true); else BY_GROUP(0, false);
        } else {
            if (zeros) BY_GROUP(1, true); else BY_GROUP(1, false);
        }
#undef BY_GROUP
#undef RUN
    }
    return launched();
}

int launch_int4_dequantize(const Int4Matrix &m, int64_t d, void *x, int dtype, int64_t ld, hipStream_t stream)
{
    const int64_t per_row = dtype == 0 ? (d + 7) / 8 : (d + 3) / 4, groups = m.K / m.group, most = rows_at_once(per_row), each = kBlock * kInt4Vectors;
    for (int64_t n = 0; n < m.V; n += most) {
        Int4Matrix part = m;
        part.V = m.V - n < most ? m.V - n : most;
        part.codes += n * (m.K / 2), part.scales += n * groups;
        if (m.zeros) part.zeros += n * groups;
        const dim3 grid((unsigned)((part.V * per_row + each - 1) / each));
        if (dtype == 0)
            int4_dequantize_kernel<0><<<grid, dim3(kBlock), 0, stream>>>(part, d, (uint16_t *)x + n * ld, ld, (uint32_t)per_row);
        else
            int4_dequantize_kernel<1><<<grid, dim3(kBlock), 0, stream>>>(part, d, (float *)x + n * ld, ld, (uint32_t)per_row);
    }
    return launched();
}

}  // namespace difr
