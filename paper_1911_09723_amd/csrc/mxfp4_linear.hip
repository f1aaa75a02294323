// y = clamp(x W^T + b) for a weight and rows in 4 bits with a power of two for
// each 32 channels (mxfp4.hpp).
#include <algorithm>

#include "fp8_product.hpp"
#include "mxfp4.hpp"

namespace spconv {
namespace {

__device__ __forceinline__ void finish4(const Linear4Args &a, bool wide, int32_t row, int32_t ch, f4 v) {
    if (row >= a.n || ch >= a.cout)
        return;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        v[i] = clamp_to(v[i] + (a.bias && ch + i < a.cout ? a.bias[ch + i] : 0.0f), a.lo, a.hi);
    store4(a.y, a.y_type, static_cast<int64_t>(row) * a.cout + ch, v, a.cout - ch, wide);
}

// A lane's part of one line of a row: blocks 2 (lane / 16) and the next, whose
// powers are the lower bytes of `power`.
struct LinePart {
    u4 code[2];
    uint32_t power;
};

__device__ __forceinline__ LinePart line_part(const uint8_t *row, const uint8_t *scale, int32_t line, int lane) {
    const u4 *p = reinterpret_cast<const u4 *>(row + static_cast<int64_t>(line) * 128) + (lane >> 4) * 2;
    return {{p[0], p[1]}, *reinterpret_cast<const uint16_t *>(scale + (lane >> 4) * 2)};
}

// Few rows, no LDS but for the final sum: a workgroup has 16 channels and 16
// rows, its wavefronts share the lines.
__global__ void __launch_bounds__(1024) linear4_stream(Linear4Args a, int32_t ctiles, bool wide) {
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int waves = blockDim.x >> 6;
    const int32_t tt = static_cast<int32_t>(blockIdx.x) / ctiles, c0 = (static_cast<int32_t>(blockIdx.x) - tt * ctiles) * 16, t0 = tt * 16;
    const int32_t ch = min(c0 + (lane & 15), a.cout - 1), row = min(t0 + (lane & 15), a.n - 1);
    const int64_t pitch = static_cast<int64_t>(a.lines) * 128;
    f4 acc = {};
    for (int32_t b = wave; b < a.lines; b += waves) {
        const LinePart w = line_part(a.w + ch * pitch, a.ws + (static_cast<int64_t>(b) * a.cout + ch) * 8, b, lane);
        const LinePart x = line_part(static_cast<const uint8_t *>(a.x) + row * pitch,
                                     a.xs + (static_cast<int64_t>(b) * a.n + row) * 8, b, lane);
        acc = mfma4<0>(w.code[0], x.code[0], acc, w.power, x.power);
        acc = mfma4<1>(w.code[1], x.code[1], acc, w.power, x.power);
    }
    sum_waves<1>(&acc, reinterpret_cast<f4 *>(lds), waves, wave, lane, [&](int, f4 sum) {
        finish4(a, wide, t0 + (lane & 15), c0 + (lane >> 4) * 4, sum);
    });
}

}  // namespace

bool linear4_takes_rows(int32_t, int32_t, int32_t) { return false; }

int32_t linear4_splits(int32_t, int32_t, int32_t) { return 1; }

hipError_t launch_linear_mxfp4(const Linear4Args &a, hipStream_t stream) {
    const bool wide = a.cout % 4 == 0 && reinterpret_cast<uintptr_t>(a.y) % 16 == 0;
    const int waves = std::min(a.lines, 16);
    const int32_t ctiles = (a.cout + 15) / 16;
    linear4_stream<<<ctiles * ((a.n + 15) / 16), waves * 64, waves * 1024, stream>>>(a, ctiles, wide);
    return hipGetLastError();
}

}  // namespace spconv
