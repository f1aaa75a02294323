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
    float *partial;      // [splits][n][cout rounded up to 4] where workgroups share the input channels
    int32_t x_type, y_type;
    int32_t n, cin, cout, kb;
    float lo, hi;
};

// Whether rows that are not quantised yet are quantised inside the product's kernel.
bool linear_takes_rows(int32_t n, int32_t cin, int32_t cout);
// How many workgroups share the input channels of a tile; above 1 the call needs `partial`.
int32_t linear_splits(int32_t n, int32_t cin, int32_t cout);
hipError_t launch_linear_fp8(const LinearArgs &a, hipStream_t stream);

// Router: ids and weights [n][k] from logits [n][experts] (row stride ld elements).
struct RouteArgs {
    const void *logits;
    int64_t ld;
    const float *bias;  // [experts] or null
    int32_t *ids;
    float *weights;
    int32_t n, experts, k;
    int32_t groups, groups_kept, group_top;
    int32_t softmax, renorm;
    float factor;
    // set by launch_route: experts of a group and its inverse, lanes that look through one,
    // whether those hold its experts
    int32_t each;
    uint32_t each_inverse;
    int32_t group_lanes;
    bool whole_lanes;
};
constexpr int32_t kMostExperts = 1024;
constexpr int32_t kMostChoices = 64;
hipError_t launch_route(RouteArgs a, int32_t type, hipStream_t stream);

// The experts' networks over pairs (token, choice), pairs = n k.
struct ExpertArgs {
    const void *x;             // [n][hidden], row stride ldx elements
    int64_t ldx;
    const int32_t *ids;        // [n][k]
    const float *weights;      // [n][k]
    const uint8_t *w13, *w2;   // codes [experts][2][inner][128 hb], [experts][hidden][128 ib]
    const float *s13, *s2;     // scales [experts][2][ib][hb], [experts][hb][ib]
    void *y;                   // [n][hidden]
    int32_t type;              // of x and y
    int32_t n, k, pairs, experts, hidden, inner;
    int32_t hb, ib;            // blocks of 128 hidden and inner channels
    // workspace: the pairs sorted by expert (order[place] = token, place[pair], -1 where
    // the id is no expert, offsets[experts + 1] = each expert's first place), x's codes,
    // the inner rows' codes and the results by place; token by token only the inner rows,
    // in 32 bits by pair (h)
    int32_t *order, *place, *offsets;
    uint8_t *xq, *hq;
    float *xs, *hs, *h;
    void *z;    // f32, or f16 with scales zs [pairs][hb]
    float *zs;
    uint32_t k_inverse, ib_inverse;  // set by launch_experts: above 2^31 / k and 2^31 / ib by at most 1
};

// Whether a call runs token by token, each pair reading its expert's weights, instead of
// over tiles of the rows of one expert.
bool experts_by_token(int32_t n, int32_t k, int32_t experts, int32_t hidden, int32_t inner);
hipError_t launch_experts(ExpertArgs a, hipStream_t stream);

}  // namespace spconv
