// Matrices to 8-bit floating point with a scale for each block (fp8.hpp).
//
// One pass over the data: a block stays in registers between the search for
// its largest magnitude and the conversion.  What bounds it is traffic (8192 x
// 4096 bf16, 101 MB: 23.8 us, 4.3 TB/s; a large copy 4.76), below some MB the
// launch (16 x 1280: 2.8 us).
#include <algorithm>

#include "expert_ops.hpp"
#include "fp8.hpp"

namespace spconv {
namespace {

template <typename T, int U>
__global__ void __launch_bounds__(256) quantize_rows(const T *x, int64_t ldx, int32_t rows, int32_t cols, uint8_t *q,
                                                     float *scale, int32_t kb, int32_t row_groups, bool wide) {
    const int32_t part = static_cast<int32_t>(blockIdx.x) / row_groups;
    quantize_group<T, U>(x, ldx, rows, cols, q, scale, kb, static_cast<int32_t>(blockIdx.x) - part * row_groups, part,
                         wide);
}

// Blocks of 128 x 128, one a workgroup: a thread holds 8 values of 8 rows.
template <typename T>
__global__ void __launch_bounds__(256) quantize_blocks(const T *x, int64_t ldx, int32_t rows, int32_t cols, uint8_t *q,
                                                       float *scale, int32_t kb, bool wide) {
    __shared__ uint32_t part[4];
    const int32_t rb = static_cast<int32_t>(blockIdx.x) / kb, b = static_cast<int32_t>(blockIdx.x) - rb * kb;
    const int l = threadIdx.x & 15, r0 = threadIdx.x >> 4;
    const int32_t c = b * kBlock + 8 * l;
    float v[8][8];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int32_t row = rb * kBlock + 16 * i + r0;
        load8_tail(x + row * ldx + c, row < rows ? cols - c : 0, wide, v[i]);
        m = max(m, most8(v[i]));
    }
#pragma unroll
    for (int s = 1; s < 64; s *= 2)
        m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), s)));
    if ((threadIdx.x & 63) == 0)
        part[threadIdx.x >> 6] = m;
    __syncthreads();
    const Scale s = scale_of(max(max(part[0], part[1]), max(part[2], part[3])));
    if (threadIdx.x == 0)
        scale[blockIdx.x] = s.scale;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int32_t row = rb * kBlock + 16 * i + r0;
        if (row < rows)
            *reinterpret_cast<u2 *>(q + (static_cast<int64_t>(row) * kb + b) * kBlock + 8 * l) =
                u2{codes4(v[i], s.inv), codes4(v[i] + 4, s.inv)};
    }
}

template <typename T>
bool aligned(const void *x, int64_t ldx) {
    return reinterpret_cast<uintptr_t>(x) % 16 == 0 && ldx * sizeof(T) % 16 == 0;
}

template <typename T>
hipError_t rows_of(const void *x, int64_t ldx, int32_t rows, int32_t cols, uint8_t *q, float *scale,
                   hipStream_t stream) {
    const int32_t kb = blocks_of(cols), groups = (rows + 15) / 16;
    const bool wide = aligned<T>(x, ldx);
    // four blocks a lane group once that still gives every compute unit several workgroups
    if (static_cast<int64_t>(groups) * kb >= 4096)
        quantize_rows<T, 4><<<groups * ((kb + 3) / 4), 256, 0, stream>>>(static_cast<const T *>(x), ldx, rows, cols, q,
                                                                        scale, kb, groups, wide);
    else
        quantize_rows<T, 1><<<groups * kb, 256, 0, stream>>>(static_cast<const T *>(x), ldx, rows, cols, q, scale, kb,
                                                             groups, wide);
    return hipGetLastError();
}

template <typename T>
hipError_t blocks(const void *x, int64_t ldx, int32_t rows, int32_t cols, uint8_t *q, float *scale,
                  hipStream_t stream) {
    const int32_t kb = blocks_of(cols);
    quantize_blocks<T><<<blocks_of(rows) * kb, 256, 0, stream>>>(static_cast<const T *>(x), ldx, rows, cols, q, scale,
                                                                 kb, aligned<T>(x, ldx));
    return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize_rows(const void *x, int32_t type, int64_t ldx, int32_t rows, int32_t cols, uint8_t *q,
                                float *scale, hipStream_t stream) {
    return type == kF32   ? rows_of<float>(x, ldx, rows, cols, q, scale, stream)
           : type == kF16 ? rows_of<_Float16>(x, ldx, rows, cols, q, scale, stream)
                          : rows_of<__bf16>(x, ldx, rows, cols, q, scale, stream);
}

hipError_t launch_quantize_blocks(const void *x, int32_t type, int64_t ldx, int32_t rows, int32_t cols, uint8_t *q,
                                  float *scale, hipStream_t stream) {
    return type == kF32   ? blocks<float>(x, ldx, rows, cols, q, scale, stream)
           : type == kF16 ? blocks<_Float16>(x, ldx, rows, cols, q, scale, stream)
                          : blocks<__bf16>(x, ldx, rows, cols, q, scale, stream);
}

}  // namespace spconv
