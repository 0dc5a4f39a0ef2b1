// Microscaled 4-bit floating point (E2M1 elements, one power-of-two scale for each 32 of a row): quantisation and values
// (the product: mx4_product.hip).
// Format and formulas at the entry points in difr.h.
#include "difr_host.hpp"
#include "softmax_row.hpp"
#include "token_loss.hpp"

namespace difr {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// A lane has eight elements of a row, four lanes a block of 32, whose largest magnitude they exchange; the conversion itself is the
// machine's (round to nearest, ties to even, saturating), two elements an instruction.  Bound by memory: 151,936 x 4096 bf16 258 us, 6.1
// TB/s (one element at a time by comparisons, a lane a block, 390 us).
constexpr int kQuantVectors = 2;  // of eight elements, of each thread

template <int DT>
__device__ __forceinline__ void load_eight(const typename Elem<DT>::type *p, int64_t k, int64_t d, u32x4 q[DT == 0 ? 1 : 2])
{
    constexpr int E = Elem<DT>::kPerVec;
#pragma unroll
    for (int h = 0; h < 8 / E; ++h) {
        const int64_t at = k + h * E;
        if (at + E <= d) {
            q[h] = *reinterpret_cast<const u32x4_any *>(p + at);
        } else {  // past the row's end: zeros
            uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (at + j < d) {
                    if constexpr (DT == 0)
                        w[j >> 1] |= (uint32_t)p[at + j] << (16 * (j & 1));
                    else
                        w[j] = __float_as_uint(p[at + j]);
                }
            q[h] = u32x4{w[0], w[1], w[2], w[3]};
        }
    }
}

template <int DT>
__global__ __launch_bounds__(kBlock) void mx4_quantize_kernel(const typename Elem<DT>::type *x, int64_t N, int64_t d, int64_t ld,
                                                              uint8_t *codes, uint8_t *scales, uint32_t eights)
{
    u32x4 q[kQuantVectors][DT == 0 ? 1 : 2];
    const uint32_t first = blockIdx.x * (kBlock * kQuantVectors) + threadIdx.x, total = (uint32_t)N * eights;
#pragma unroll
    for (int u = 0; u < kQuantVectors; ++u) {
        const uint32_t i = first + u * kBlock, row = i < total ? i / eights : 0;
        load_eight<DT>(x + row * ld, i < total ? (int64_t)(i - row * eights) * 8 : d, d, q[u]);
    }
#pragma unroll
    for (int u = 0; u < kQuantVectors; ++u) {
        const uint32_t i = first + u * kBlock;
        // the largest magnitude's bits: an infinity or a NaN is larger than any number
        uint32_t top = 0;
#pragma unroll
        for (int h = 0; h < (DT == 0 ? 1 : 2); ++h)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t w = q[u][h][j];
                if (DT == 0)
                    top = max(top, max(w & 0x7FFF0000u, w << 16 & 0x7FFF0000u));
                else
                    top = max(top, w & 0x7FFFFFFFu);
            }
        top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0xB1, 0xF, 0xF, false));  // lanes 1 0 3 2 of each four
        top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0x4E, 0xF, 0xF, false));  // lanes 2 3 0 1
        const bool number = top < 0x7F800000u;
        // floor(log2 amax) - 2 as a biased exponent: of a normal number its exponent field less 2
        const int field = (int)(top >> 23), e = field > 2 ? field - 2 : 0;
        uint32_t w = 0;
        // (the instruction takes the scale's exponent; 2^-127 is no normal fp32 number, so the smallest exponents are halved beforehand)
        if constexpr (DT == 0) {
            if (e > 0) {
                const float scale = __uint_as_float((uint32_t)e << 23);
                const uint32_t pair[4] = {q[u][0].x, q[u][0].y, q[u][0].z, q[u][0].w};
                w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, pair[0]), scale, 0);
                w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, pair[1]), scale, 1);
                w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, pair[2]), scale, 2);
                w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, pair[3]), scale, 3);
            }
        }
        if (DT != 0 || e == 0) {
            float v[8];
            if constexpr (DT == 0) {
                unpack_vector<0>(q[u][0], v);
            } else {
                unpack_vector<1>(q[u][0], v);
                unpack_vector<1>(q[u][1], v + 4);
            }
            const float up = __uint_as_float((uint32_t)(254 - e) << 23);  // 2^(127 - e), a normal number for every e there is (0 .. 252)
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v[0] * up, v[1] * up, 1.0f, 0);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2] * up, v[3] * up, 1.0f, 1);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4] * up, v[5] * up, 1.0f, 2);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6] * up, v[7] * up, 1.0f, 3);
        }
        if (i < total) {
            reinterpret_cast<uint32_t *>(codes)[i] = number ? w : 0u;
            if ((threadIdx.x & 3) == 0) scales[i >> 2] = number ? (uint8_t)e : 0xFFu;
        }
    }
}

// Two values of a byte of codes times 2^(e - 127).
template <int BYTE>
__device__ __forceinline__ void two_values(uint32_t w, float down, float v[2])
{
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const f32x2 p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, BYTE);
    v[0] = p[0] * down;
    v[1] = p[1] * down;
}

// One thread eight elements (a dword of codes).
template <int DT>
__global__ __launch_bounds__(kBlock) void mx4_dequantize_kernel(const uint8_t *codes, const uint8_t *scales, int64_t N, int64_t d,
                                                                int64_t blocks, typename Elem<DT>::type *x, int64_t ld)
{
    constexpr int E = Elem<DT>::kPerVec;
    const uint32_t per_row = (uint32_t)((d + 7) / 8), total = (uint32_t)N * per_row;
    uint32_t w[kQuantVectors], e[kQuantVectors];
    int64_t row[kQuantVectors], k[kQuantVectors];
#pragma unroll
    for (int u = 0; u < kQuantVectors; ++u) {
        const uint32_t i = blockIdx.x * (kBlock * kQuantVectors) + u * kBlock + threadIdx.x, r = i < total ? i / per_row : 0;
        row[u] = r;
        k[u] = i < total ? (int64_t)(i - r * per_row) * 8 : d;
        const int64_t at = k[u] < d ? k[u] : 0;
        w[u] = *reinterpret_cast<const uint32_t *>(codes + row[u] * blocks * 16 + at / 2);
        e[u] = scales[row[u] * blocks + at / 32];
    }
#pragma unroll
    for (int u = 0; u < kQuantVectors; ++u) {
        // 2^(e - 127): a normal number's exponent field, 2^-127 below, and a NaN for 255
        const float down = __uint_as_float(e[u] == 0xFFu ? 0x7FC00000u : e[u] == 0 ? 0x00400000u : e[u] << 23);
        float v[8];
        two_values<0>(w[u], down, v);
        two_values<1>(w[u], down, v + 2);
        two_values<2>(w[u], down, v + 4);
        two_values<3>(w[u], down, v + 6);
#pragma unroll
        for (int j = 0; j < 8; j += E) {
            const int64_t at = k[u] + j;
            if (at + E <= d)
                __builtin_nontemporal_store(pack_vector<DT>(v + j), reinterpret_cast<u32x4_any *>(x + row[u] * ld + at));
            else if (at < d)
                store_vector<DT>(x + row[u] * ld, at / E, d, pack_vector<DT>(v + j));
        }
    }
}

static int launched() { return hipGetLastError() == hipSuccess ? 0 : 1; }

// Rows of a launch, of which the kernels count the eights in 32 bits.
static int64_t rows_at_once(int64_t eights) { return ((int64_t)1 << 30) / eights > 0 ? ((int64_t)1 << 30) / eights : 1; }

int launch_mx4_quantize(const void *x, int dtype, int64_t N, int64_t d, int64_t ld, uint8_t *codes, uint8_t *scales, hipStream_t stream)
{
    const int64_t eights = (d + kMxSlab - 1) / kMxSlab * (kMxSlab / 8), each = kBlock * kQuantVectors, most = rows_at_once(eights);
    for (int64_t n = 0; n < N; n += most) {
        const int64_t rows = N - n < most ? N - n : most;
        const dim3 grid((unsigned)((rows * eights + each - 1) / each));
        uint8_t *c = codes + n * eights * 4, *s = scales + n * (eights / 4);
        if (dtype == 0)
            mx4_quantize_kernel<0><<<grid, dim3(kBlock), 0, stream>>>((const uint16_t *)x + n * ld, rows, d, ld, c, s, (uint32_t)eights);
        else
            mx4_quantize_kernel<1><<<grid, dim3(kBlock), 0, stream>>>((const float *)x + n * ld, rows, d, ld, c, s, (uint32_t)eights);
    }
    return launched();
}

int launch_mx4_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t N, int64_t d, void *x, int dtype, int64_t ld,
                          hipStream_t stream)
{
    const int64_t blocks = (d + kMxSlab - 1) / kMxSlab * (kMxSlab / kMxBlock), eights = (d + 7) / 8, each = kBlock * kQuantVectors;
    const int64_t most = rows_at_once(eights);
    for (int64_t n = 0; n < N; n += most) {
        const int64_t rows = N - n < most ? N - n : most;
        const dim3 grid((unsigned)((rows * eights + each - 1) / each));
        const uint8_t *c = codes + n * blocks * 16, *s = scales + n * blocks;
        if (dtype == 0)
            mx4_dequantize_kernel<0><<<grid, dim3(kBlock), 0, stream>>>(c, s, rows, d, blocks, (uint16_t *)x + n * ld, ld);
        else
            mx4_dequantize_kernel<1><<<grid, dim3(kBlock), 0, stream>>>(c, s, rows, d, blocks, (float *)x + n * ld, ld);
    }
    return launched();
}

}  // namespace difr
