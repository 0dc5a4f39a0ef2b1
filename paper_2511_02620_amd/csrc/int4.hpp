// Launch functions of the matrices in 4-bit integers (int4.hip, int4_product.hip), shared with the C ABI layer.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace difr {

constexpr int kInt4Slab = 128;  // rows of codes are whole slabs

struct Int4Matrix {
    const uint8_t *codes;    // [V][K / 2]
    const uint16_t *scales;  // [V][K / group], bf16
    const uint8_t *zeros;    // [V][K / group], or null: 8 each
    int64_t V, K;
    int group;               // 32, 64 or 128
};

int launch_int4_quantize(const void *x, int dtype, int64_t N, int64_t d, int64_t ld, int group, uint8_t *codes, uint16_t *scales,
                         uint8_t *zeros, hipStream_t stream);
int launch_int4_dequantize(const Int4Matrix &m, int64_t d, void *x, int dtype, int64_t ld, hipStream_t stream);
int launch_int4_product(const void *h, int h_dtype, int64_t N, int64_t d, int64_t ldh, const Int4Matrix &m, void *out, int dtype, int64_t ld,
                        void *workspace, hipStream_t stream);
size_t int4_product_workspace_bytes(int64_t N, int64_t d, int dtype);

}  // namespace difr
