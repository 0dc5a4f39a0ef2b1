// Microscaled 4-bit floating point (E2M1 elements, one power-of-two scale for each 32 of a row): quantisation and values
// (the product: mx4_product.hip).
// Format and formulas at the entry points in difr.h.
#include "difr_host.hpp"
#include "softmax_row.hpp"
#include "token_loss.hpp"

namespace difr {


// The code of x 2^-e: round to nearest, ties to even, everything from 5 on is 6.
__device__ __forceinline__ uint32_t e2m1_code(float v)
{
    const float m = fabsf(v);
    uint32_t c = (uint32_t)(m > 0.25f);
    c += (uint32_t)(m >= 0.75f);
    c += (uint32_t)(m > 1.25f);
    c += (uint32_t)(m >= 1.75f);
    c += (uint32_t)(m > 2.5f);
    c += (uint32_t)(m >= 3.5f);
    c += (uint32_t)(m > 5.0f);
    return c | (__float_as_uint(v) >> 31 << 3);
}

// One thread a block of 32 elements.
template <int DT>
__global__ __launch_bounds__(kBlock) void mx4_quantize_kernel(const typename Elem<DT>::type *x, int64_t N, int64_t d, int64_t ld,
                                                              uint8_t *codes, uint8_t *scales, int64_t blocks)
{
    constexpr int E = Elem<DT>::kPerVec;
    const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (i >= N * blocks) return;
    const int64_t row = i / blocks, k = (i - row * blocks) * kMxBlock;
    const typename Elem<DT>::type *p = x + row * ld;
    float v[kMxBlock];
#pragma unroll
    for (int j = 0; j < kMxBlock; j += E) {
        if (k + j + E <= d) {
            unpack_vector<DT>(*reinterpret_cast<const u32x4_any *>(p + k + j), v + j);
        } else {
#pragma unroll
            for (int q = 0; q < E; ++q) v[j + q] = k + j + q < d ? Elem<DT>::to_float(p[k + j + q]) : 0.0f;
        }
    }
    uint32_t top = 0;  // of the magnitudes' bits: an infinity or a NaN is the largest
#pragma unroll
    for (int j = 0; j < kMxBlock; ++j) top = max(top, __float_as_uint(v[j]) & 0x7FFFFFFFu);
    const bool number = top < 0x7F800000u;
    // floor(log2 amax) - 2, as a biased exponent: of a normal number its exponent field less 2
    const int field = (int)(top >> 23);
    const int e = field > 2 ? field - 2 : 0;
    const float up = __uint_as_float((uint32_t)(254 - e) << 23);  // 2^(127 - e), a normal number for every e there is (0 .. 252)
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < kMxBlock; ++j) {
        w[j >> 3] |= (number ? e2m1_code(v[j] * up) : 0u) << (4 * (j & 7));
    }
    *reinterpret_cast<u32x4 *>(codes + i * (kMxBlock / 2)) = u32x4{w[0], w[1], w[2], w[3]};
    scales[i] = number ? (uint8_t)e : 0xFFu;
}

__device__ __forceinline__ float e2m1_value(uint32_t c)
{
    const uint32_t m = c & 7u;
    const float v = m < 2 ? 0.5f * (float)m : __uint_as_float(((m >> 1) + 126u) << 23 | (m & 1u) << 22);
    return c & 8u ? -v : v;
}

// One thread eight elements (a dword of codes).
template <int DT>
__global__ __launch_bounds__(kBlock) void mx4_dequantize_kernel(const uint8_t *codes, const uint8_t *scales, int64_t N, int64_t d,
                                                                int64_t blocks, typename Elem<DT>::type *x, int64_t ld)
{
    constexpr int E = Elem<DT>::kPerVec;
    const int64_t per_row = (d + 7) / 8, i = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (i >= N * per_row) return;
    const int64_t row = i / per_row, k = (i - row * per_row) * 8;
    const uint32_t w = *reinterpret_cast<const uint32_t *>(codes + row * blocks * 16 + k / 2);
    const uint8_t e = scales[row * blocks + k / 32];
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = e == 0xFF ? __builtin_nanf("") : ldexpf(e2m1_value(w >> (4 * j) & 15u), (int)e - 127);
#pragma unroll
    for (int j = 0; j < 8; j += E) store_vector<DT>(x + row * ld, (k + j) / E, d, pack_vector<DT>(v + j));
}

static int launched() { return hipGetLastError() == hipSuccess ? 0 : 1; }

int launch_mx4_quantize(const void *x, int dtype, int64_t N, int64_t d, int64_t ld, uint8_t *codes, uint8_t *scales, hipStream_t stream)
{
    const int64_t blocks = (d + kMxSlab - 1) / kMxSlab * (kMxSlab / kMxBlock);
    const dim3 grid((unsigned)((N * blocks + kBlock - 1) / kBlock));
    if (dtype == 0)
        mx4_quantize_kernel<0><<<grid, dim3(kBlock), 0, stream>>>((const uint16_t *)x, N, d, ld, codes, scales, blocks);
    else
        mx4_quantize_kernel<1><<<grid, dim3(kBlock), 0, stream>>>((const float *)x, N, d, ld, codes, scales, blocks);
    return launched();
}

int launch_mx4_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t N, int64_t d, void *x, int dtype, int64_t ld,
                          hipStream_t stream)
{
    const int64_t blocks = (d + kMxSlab - 1) / kMxSlab * (kMxSlab / kMxBlock);
    const dim3 grid((unsigned)((N * ((d + 7) / 8) + kBlock - 1) / kBlock));
    if (dtype == 0)
        mx4_dequantize_kernel<0><<<grid, dim3(kBlock), 0, stream>>>(codes, scales, N, d, blocks, (uint16_t *)x, ld);
    else
        mx4_dequantize_kernel<1><<<grid, dim3(kBlock), 0, stream>>>(codes, scales, N, d, blocks, (float *)x, ld);
    return launched();
}

}  // namespace difr
