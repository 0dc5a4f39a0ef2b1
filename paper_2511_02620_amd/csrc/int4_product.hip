// out[n][v] = sum_k h[n][k] w[v][k] for a head w in 4-bit integers: few hidden states, of which one each is what a token takes.
#include "difr_host.hpp"
#include "int4.hpp"
#include "softmax_row.hpp"

namespace difr {

constexpr int kInt4Rows = 8;  // hidden states of a pass over the head

// A wave a row of the head, eight elements a lane at a time.
template <int HT, int DT>
__global__ __launch_bounds__(kBlock) void int4_product_kernel(const typename Elem<HT>::type *h, int64_t N, int64_t d, int64_t ldh, Int4Matrix m,
                                                              typename Elem<DT>::type *out, int64_t ld)
{
    const int lane = threadIdx.x & 63;
    const int64_t v = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6), n0 = (int64_t)blockIdx.y * kInt4Rows;
    if (v >= m.V) return;
    float acc[kInt4Rows] = {};
    for (int64_t k = lane * 8; k < m.K; k += 512) {
        const uint32_t w = *reinterpret_cast<const uint32_t *>(m.codes + v * (m.K / 2) + k / 2);
        const int64_t g = v * (m.K / m.group) + k / m.group;
        const float s = __uint_as_float((uint32_t)m.scales[g] << 16), z = m.zeros ? (float)m.zeros[g] : 8.0f;
#pragma unroll
        for (int i = 0; i < kInt4Rows; ++i) {
            if (n0 + i >= N) break;
            const typename Elem<HT>::type *row = h + (n0 + i) * ldh;
            float part = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (k + j < d) part = __builtin_fmaf((float)(w >> (4 * j) & 15u) - z, Elem<HT>::to_float(row[k + j]), part);
            acc[i] = __builtin_fmaf(s, part, acc[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < kInt4Rows; ++i) {
        const float sum = wave_sum(acc[i]);
        if (lane == 0 && n0 + i < N) store_element<DT>(out + (n0 + i) * ld + v, sum);
    }
}

int launch_int4_product(const void *h, int h_dtype, int64_t N, int64_t d, int64_t ldh, const Int4Matrix &m, void *out, int dtype, int64_t ld,
                        hipStream_t stream)
{
    const dim3 grid((unsigned)((m.V + kWaves - 1) / kWaves), (unsigned)((N + kInt4Rows - 1) / kInt4Rows));
#define RUN(HT, DT) \
    int4_product_kernel<HT, DT><<<grid, dim3(kBlock), 0, stream>>>((const Elem<HT>::type *)h, N, d, ldh, m, (Elem<DT>::type *)out, ld)
    if (h_dtype == 0) {
        if (dtype == 0) RUN(0, 0); else RUN(0, 1);
    } else {
        if (dtype == 0) RUN(1, 0); else RUN(1, 1);
    }
#undef RUN
    return hipGetLastError() == hipSuccess ? 0 : 1;
}

}  // namespace difr
