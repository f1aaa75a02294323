// Rows to 4-bit floating point with a power of two for each 32 channels (mxfp4.hpp).
#include "mxfp4.hpp"

namespace spconv {
namespace {

// A thread has 8 values, 4 neighbours a block, 32 a line; a workgroup covers 8
// rows, U lines of each, whose loads are under way together.  What bounds it is traffic (8192 x
// 4096 in bf16: 85 MB in 18.3 us, 4.6 TB/s), below some MB the launch (16 x 1280: 2.5 us).
template <typename T, int U, bool STREAM>
__global__ void __launch_bounds__(256) quantize4_rows(const T *x, int64_t ldx, int32_t rows, int32_t cols, uint8_t *q,
                                                      uint8_t *scale, int32_t lines, int32_t row_groups, bool wide) {
    const int32_t part = static_cast<int32_t>(blockIdx.x) / row_groups;
    const int32_t row = (static_cast<int32_t>(blockIdx.x) - part * row_groups) * 8 + (threadIdx.x >> 5);
    const int l = threadIdx.x & 31;
    if (row >= rows)
        return;
    const T *xr = x + row * ldx;
    const int32_t l0 = part * U;
    Eight<T> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int32_t c = (l0 + u) * kLine4 + 8 * l;
        v[u] = eight_tail<T, STREAM>(xr + c, cols - c, wide);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (l0 + u >= lines)
            break;
        uint32_t m = most_of(0, v[u]);
        if constexpr (sizeof(T) == 2)
            m = max(m & 0xffffu, m >> 16);
        m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 1)));
        m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 2)));
        const uint32_t power = power_of_most<T>(m);
        *reinterpret_cast<uint32_t *>(q + (static_cast<int64_t>(row) * lines + l0 + u) * 128 + 4 * l) = codes8(v[u], power);
        if ((l & 3) == 0)
            scale[(static_cast<int64_t>(l0 + u) * rows + row) * 8 + (l >> 2)] = static_cast<uint8_t>(power);
    }
}

template <typename T>
hipError_t rows_of(const void *x, int64_t ldx, int32_t rows, int32_t cols, uint8_t *q, uint8_t *scale,
                   hipStream_t stream) {
    const int32_t lines = lines_of(cols), groups = (rows + 7) / 8;
    const bool wide = reinterpret_cast<uintptr_t>(x) % 16 == 0 && ldx * sizeof(T) % 16 == 0;
    // Four lines a thread once that still gives every compute unit several workgroups; rows are
    // then read past the caches (8192 x 4096 in bf16 18.3 us, through them 22.4; 2048 x 4096 6.3 and 7.4;
    // not compared in f32, whose rows are twice the bytes).
    if (static_cast<int64_t>(groups) * lines >= 4096)
        quantize4_rows<T, 4, true><<<groups * ((lines + 3) / 4), 256, 0, stream>>>(static_cast<const T *>(x), ldx, rows, cols, q,
                                                                            scale, lines, groups, wide);
    else
        quantize4_rows<T, 1, false><<<groups * lines, 256, 0, stream>>>(static_cast<const T *>(x), ldx, rows, cols, q, scale,
                                                                 lines, groups, wide);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize_mxfp4(const void *x, int32_t type, int64_t ldx, int32_t rows, int32_t cols, uint8_t *q,
                                 uint8_t *scale, hipStream_t stream) {
    return type == kF32   ? rows_of<float>(x, ldx, rows, cols, q, scale, stream)
           : type == kF16 ? rows_of<_Float16>(x, ldx, rows, cols, q, scale, stream)
                          : rows_of<__bf16>(x, ldx, rows, cols, q, scale, stream);
}

}  // namespace spconv
