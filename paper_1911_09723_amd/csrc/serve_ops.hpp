// Internal interface between the C ABI (serve_api.cpp) and the kernels around
// a served model's dense layers: norms, 4-bit block products and sampling.
// Arguments are validated by the caller.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstdint>

#include "expert_ops.hpp"

namespace spconv {

// y = h / sqrt(mean(h^2) + eps) * gain over rows, h = x (+ residual)
struct NormArgs {
    const void *x, *residual, *gain;  // residual, gain: or null
    void *total;                      // h in the residual's type, or null
    void *y;                          // or null
    uint8_t *q;                       // codes [rows][128 kb] with scales [kb][rows], or null
    float *scale;
    int64_t ldx, ldr, ldt, ldy;       // row strides in elements
    int32_t rows, cols, kb;
    float eps;
    bool y32;                         // y in f32, else in x's type
    // set by launch_norm: rows that can be read and written in pieces of 16 bytes, and how
    bool wide_x, wide_r, wide_g, wide_t, wide_y;
    bool stream;   // past the caches
    double share;  // 1 / cols
};
// type: of x; residual and gain are of that type or (residual32, gain32) in f32.
hipError_t launch_norm(NormArgs a, int32_t type, bool residual32, bool gain32, hipStream_t stream);

// Rows kept as 4-bit codes (spconv_dtype).
enum : int32_t { kMxfp4 = 4 };

// Lines of 256 channels, which are 128 bytes of 4-bit codes.
inline int32_t lines_of(int64_t channels) { return static_cast<int32_t>((channels + 255) / 256); }

// x [rows][cols] (row stride ldx elements) to codes [rows][128 lines] and scales [lines][rows][8].
hipError_t launch_quantize_mxfp4(const void *x, int32_t type, int64_t ldx, int32_t rows, int32_t cols, uint8_t *q,
                                 uint8_t *scale, hipStream_t stream);

// y [n][cout] = clamp(x w^T + bias, lo, hi)
struct Linear4Args {
    const void *x;        // f32, f16 or bf16 rows (stride ldx elements), or codes [n][128 lines]
    int64_t ldx;
    const uint8_t *xs;    // scales of codes, [lines][n][8]
    const uint8_t *w;     // codes [cout][128 lines]
    const uint8_t *ws;    // [lines][cout][8]
    const float *bias;    // [cout] or null
    void *y;
    int32_t x_type, y_type;
    int32_t n, cin, cout, lines;
    float lo, hi;
};
// Whether rows that are not quantised yet are quantised inside the product's kernel.
bool linear4_takes_rows(int32_t n, int32_t cin, int32_t cout);
hipError_t launch_linear_mxfp4(const Linear4Args &a, hipStream_t stream);

// Tokens [n] from logits [n][vocab] (row stride ld elements).
struct SampleArgs {
    const void *logits;
    int64_t ld;
    const float *u;  // [n]
    // by row, or null: then the values below hold for all
    const float *temperatures, *top_ps, *min_ps;
    const int32_t *top_ks;
    float temperature, top_p, min_p;
    int32_t top_k;
    int32_t *ids;
    int32_t n, vocab;
    void *workspace;
    int64_t words;  // set by launch_sample: 8-byte words of the workspace from row to row
};
constexpr int32_t kMostTokens = 1 << 20;
int64_t sample_workspace(int32_t n, int32_t vocab);
hipError_t launch_sample(const SampleArgs &a, int32_t type, hipStream_t stream);

}  // namespace spconv
