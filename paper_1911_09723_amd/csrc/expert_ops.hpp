// Internal interface between the C ABI (expert_api.cpp) and the kernels of
// 8-bit block products, routing and experts.  Arguments are validated by the
// caller.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstdint>

namespace spconv {

// Element types as they go through the C interface (spconv_dtype).
enum : int32_t { kF32 = 0, kF16 = 1, kBf16 = 2, kFp8 = 3 };

inline int32_t blocks_of(int64_t channels) { return static_cast<int32_t>((channels + 127) / 128); }

// x [rows][cols] (row stride ldx elements) to codes q [rows][128 kb] and scales:
// by row, scale [kb][rows]; for blocks of 128 rows, scale [ceil(rows / 128)][kb].
hipError_t launch_quantize_rows(const void *x, int32_t type, int64_t ldx, int32_t rows, int32_t cols, uint8_t *q,
                                float *scale, hipStream_t stream);
hipError_t launch_quantize_blocks(const void *x, int32_t type, int64_t ldx, int32_t rows, int32_t cols, uint8_t *q,
                                  float *scale, hipStream_t stream);

// y [n][cout] = clamp(x w^T + bias, lo, hi)
struct LinearArgs {
    const void *x;       // f32, f16 or bf16 rows (stride ldx elements), or codes [n][128 kb]
    int64_t ldx;
    const float *xs;     // scales of codes, [kb][n]
    const uint8_t *w;    // codes [cout][128 kb]
    const float *ws;     // [ceil(cout / 128)][kb]
    const float *bias;   // [cout] or null
    void *y;
    int32_t x_type, y_type;
    int32_t n, cin, cout, kb;
    float lo, hi;
};

// Whether rows that are not quantised yet are quantised inside the product's kernel.
bool linear_takes_rows(int32_t n, int32_t cin, int32_t cout);
hipError_t launch_linear_fp8(const LinearArgs &a, hipStream_t stream);

}  // namespace spconv
