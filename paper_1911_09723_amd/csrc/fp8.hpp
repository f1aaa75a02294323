// Device helpers for matrices in 8-bit floating point (e4m3, the OCP form)
// with a 32-bit scale for each block of 128 input channels.
//
// Form.  A row of c channels is kept in whole blocks: 128 ceil(c / 128) bytes,
// zeros past c, so that every row starts on a 128-byte line and no kernel has
// a tail of channels in its products.  A block's scale is a / 448 with
// a = max(max |v|, 2^-100) over the block, a code is v * (448 / a) rounded to
// the nearest e4m3 value, ties to even; each of these steps is one correctly
// rounded 32-bit operation.  |v * (448 / a)| stays below 448 (1 + 2^-23), which
// rounds to 448, so the conversion needs no clamp.  The floor on a keeps both
// quotients finite and normal for blocks of zeros or of subnormal values.  An
// infinity or a NaN makes its block's scale infinite or NaN: every product
// with that block is NaN, and no other row's changes.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "expert_ops.hpp"

namespace spconv {

typedef float f2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef int i4 __attribute__((ext_vector_type(4)));
typedef int i8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));

constexpr int kBlock = 128;                          // channels of a scale
constexpr float kTop = 448.0f;                       // largest e4m3 value
constexpr uint32_t kTinyBits = (127u - 100u) << 23;  // 2^-100

// The element type of rows kept as codes.
struct Fp8 {
    uint8_t bits;
};

template <typename T>
__device__ __forceinline__ void load8(const T *p, float *v);

template <>
__device__ __forceinline__ void load8<float>(const float *p, float *v) {
    const f4 a = *reinterpret_cast<const f4 *>(p), b = *reinterpret_cast<const f4 *>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = a[i];
        v[i + 4] = b[i];
    }
}

template <>
__device__ __forceinline__ void load8<_Float16>(const _Float16 *p, float *v) {
    const h8 a = *reinterpret_cast<const h8 *>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        v[i] = static_cast<float>(a[i]);
}

template <>
__device__ __forceinline__ void load8<__bf16>(const __bf16 *p, float *v) {
    const u4 a = *reinterpret_cast<const u4 *>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(a[i] << 16);
        v[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
    }
}

// Eight values of a row from p, of which `left` exist (the others are zeros).
// `wide`: p is aligned for vector loads.
template <typename T>
__device__ __forceinline__ void load8_tail(const T *p, int left, bool wide, float *v) {
    if (wide && left >= 8) {
        load8(p, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        v[i] = i < left ? static_cast<float>(p[i]) : 0.0f;
}

// |v|'s bits: their order as whole numbers is that of the magnitudes, a NaN above all.
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

__device__ __forceinline__ uint32_t most8(const float *v) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        m = max(m, magnitude(v[i]));
    return m;
}

// Four codes; the conversion rounds to nearest even.
__device__ __forceinline__ uint32_t codes4(const float *v, float inv) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * inv, v[1] * inv, 0, false);
    return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(v[2] * inv, v[3] * inv, w, true));
}

struct Scale {
    float scale, inv;
};

__device__ __forceinline__ Scale scale_of(uint32_t most) {
    const float a = __uint_as_float(max(most, kTinyBits));
    return {a / kTop, kTop / a};
}

// Rows to codes: 16 lanes hold a block of 128 (8 values each), a workgroup covers
// blockDim / 16 rows, so that the scales of one channel block, which lie by row,
// leave it as neighbouring bytes.  Each lane group walks U blocks of its row at
// once to keep several loads in flight.  `group`: rows of this workgroup, in
// workgroups; `part`: its blocks, in U.
template <typename T, int U>
__device__ __forceinline__ void quantize_group(const T *x, int64_t ldx, int32_t rows, int32_t cols, uint8_t *q,
                                               float *scale, int32_t kb, int32_t group, int32_t part, bool wide) {
    const int32_t row = group * static_cast<int32_t>(blockDim.x >> 4) + (threadIdx.x >> 4);
    const int l = threadIdx.x & 15;
    if (row >= rows)
        return;
    const T *xr = x + row * ldx;
    const int32_t b0 = part * U;
    float v[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int32_t c = (b0 + u) * kBlock + 8 * l;
        load8_tail(xr + c, cols - c, wide, v[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (b0 + u >= kb)
            break;
        uint32_t m = most8(v[u]);
#pragma unroll
        for (int s = 1; s < 16; s *= 2)
            m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), s)));
        const Scale s = scale_of(m);
        const int64_t at = (static_cast<int64_t>(row) * kb + b0 + u) * kBlock + 8 * l;
        *reinterpret_cast<u2 *>(q + at) = u2{codes4(v[u], s.inv), codes4(v[u] + 4, s.inv)};
        if (l == 0)
            scale[static_cast<int64_t>(b0 + u) * rows + row] = s.scale;
    }
}

// Products.  p (16 x 16, f4 a lane) = A (16 rows x 128) B (16 columns x 128):
// lane l holds of each operand row l % 16, bytes 16 (l / 16) .. + 15 and 64
// further on (any places, the same for both), and of the result column (B)
// l % 16, rows (A) 4 (l / 16) .. + 3.
//
// Two forms.  The 8-bit instruction takes 128 channels at a time, but of each 8
// neighbouring channels it cuts every product off, toward zero, at 2^-13 of the
// power of two that the largest exponents of their codes make (codes below 2^-6
// count as 2^-6; measured), and only then adds in 32 bits: 8 channels' sum is up
// to 2^-10 of their largest product off.  Over 128 products of random codes the
// result is 4e-5 (rms, relative; measured) off, a 32-bit sum 1e-7.  Below the
// rounding of a 16-bit result (2e-4 and 1.7e-3 rms) that does not show, unless
// large products cancel each other; a 32-bit result, and one that is rounded to
// codes again, wants the second form: codes are also f16 values (2^-9 to 448),
// products of f16 values are exact in 32 bits, and the f16 instruction sums 32 of
// them with less error than 32 fused multiply-adds.  It has half the rate: with it
// 8192 x 4096 -> 4096 takes 207 us (results in 32 bits) in place of 125 (in 16),
// which is why 16-bit results over tiles take the first.
__device__ __forceinline__ f4 mfma128(i8 a, i8 b) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, f4{0, 0, 0, 0}, 0, 0, 0, 0, 0, 0);
}

struct Halves {
    h8 v[4];
};

__device__ __forceinline__ Halves halves(i8 code) {
    Halves r;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const h2 lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(code[2 * i + j], 1.0f, false);
            const h2 hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(code[2 * i + j], 1.0f, true);
            r.v[i][4 * j] = lo[0];
            r.v[i][4 * j + 1] = lo[1];
            r.v[i][4 * j + 2] = hi[0];
            r.v[i][4 * j + 3] = hi[1];
        }
    return r;
}

__device__ __forceinline__ f4 mfma128(const Halves &a, const Halves &b) {
    f4 p = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        p = __builtin_amdgcn_mfma_f32_16x16x32_f16(a.v[i], b.v[i], p, 0, 0, 0);
    return p;
}

// The form of a fragment of codes that mfma128 takes for exact products or for 8-bit ones.
template <bool EXACT>
__device__ __forceinline__ auto operand(i8 code) {
    if constexpr (EXACT)
        return halves(code);
    else
        return code;
}

__device__ __forceinline__ i8 join(u4 lo, u4 hi) {
    return i8{static_cast<int>(lo[0]), static_cast<int>(lo[1]), static_cast<int>(lo[2]), static_cast<int>(lo[3]),
              static_cast<int>(hi[0]), static_cast<int>(hi[1]), static_cast<int>(hi[2]), static_cast<int>(hi[3])};
}

// max(lo, min(v, hi)) that leaves a NaN as it is.
__device__ __forceinline__ float clamp_to(float v, float lo, float hi) {
    v = v < lo ? lo : v;
    return v > hi ? hi : v;
}

// Four values rounded once to f16 or bf16.
template <int TYPE>
__device__ __forceinline__ u2 rounded4(f4 v) {
    uint16_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        r[i] = TYPE == kF16 ? __builtin_bit_cast(uint16_t, static_cast<_Float16>(v[i]))
                            : __builtin_bit_cast(uint16_t, static_cast<__bf16>(v[i]));
    return u2{r[0] | static_cast<uint32_t>(r[1]) << 16, r[2] | static_cast<uint32_t>(r[3]) << 16};
}

// `left` (1 to 4) neighbouring values to y + at, rounded once to its type; `wide`:
// the four start on a multiple of their size.
__device__ __forceinline__ void store4(void *y, int32_t type, int64_t at, f4 v, int left, bool wide) {
    if (type == kF32) {
        float *p = static_cast<float *>(y) + at;
        if (wide && left >= 4) {
            *reinterpret_cast<f4 *>(p) = v;
            return;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < left)
                p[i] = v[i];
        return;
    }
    const u2 r = type == kF16 ? rounded4<kF16>(v) : rounded4<kBf16>(v);
    uint16_t *p = static_cast<uint16_t *>(y) + at;
    if (wide && left >= 4) {
        *reinterpret_cast<u2 *>(p) = r;
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < left)
            p[i] = static_cast<uint16_t>(r[i >> 1] >> (i & 1) * 16);
}

}  // namespace spconv
