// Device helpers for matrices in 4-bit floating point (e2m1, the OCP form) with
// a power of two for each block of 32 input channels.
//
// Form.  A code's magnitudes are 0, 0.5, 1, 1.5, 2, 3, 4 and 6.  A row of c
// channels is kept in whole lines of 256: 128 ceil(c / 256) bytes, two codes a
// byte (the lower channel in the lower half), zeros past c, so that every row
// starts on a 128-byte line.  A block's power 2^e is kept as the byte e + 127, by
// line and row: the 8 bytes of a row's line lie together, rows of one line side
// by side, so that a tile's scales of a line are one piece of memory.
//
// e is the least for which the block's largest magnitude a rounds to a code and
// not past 6: a / 2^e < 7.  (With e = floor(log2 a) - 2, which others take, values
// between 7 and 8 become 6.)  a's bits + 2^21 carry into the exponent from
// 1.75 2^k on, hence e + 127 = (bits + 2^21) / 2^23 - 2, at least 0.  v / 2^e is exact, so
// a code is v rounded once, to nearest, ties to even.  A block that holds an
// infinity or a NaN has byte 255, which is NaN, and codes 0: every product with
// it is NaN, and no other row's changes.
#pragma once

#include "fp8.hpp"
#include "serve_ops.hpp"

namespace spconv {

constexpr int kBlock4 = 32;   // channels of a scale
constexpr int kLine4 = 256;   // channels of 128 bytes

// The byte that a block whose largest magnitude has these bits keeps.
__device__ __forceinline__ uint32_t power_of(uint32_t most) {
    const uint32_t p = max((most + 0x200000u) >> 23, 2u) - 2u;
    return most >= 0x7f800000u ? 255u : p;
}

// Eight codes, the first in the lowest bits; the conversion divides by the power
// and rounds to nearest even.
__device__ __forceinline__ uint32_t codes8(const float *v, uint32_t power) {
    const float scale = __uint_as_float(power ? power << 23 : 1u << 22);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], scale, 3);
    return power == 255 ? 0 : w;
}

// The same of eight values as they lie in memory, f32, f16 or bf16.  Largest
// magnitudes of 16-bit values are found two at a time on their bits, and the
// conversion takes the pairs as they are.
template <typename T>
struct Eight {
    T v[8];
};

typedef uint16_t us2 __attribute__((ext_vector_type(2)));
typedef __bf16 bh2 __attribute__((ext_vector_type(2)));

// Eight neighbours from p, of which `left` exist; the others are zeros.  STREAM: past the caches.
template <typename T, bool STREAM = false>
__device__ __forceinline__ Eight<T> eight_tail(const T *p, int left, bool wide) {
    struct __attribute__((aligned(16))) Piece {
        T v[8];
    };
    Eight<T> r;
    if (STREAM && wide && left >= 8) {
        struct Pieces {
            u4 v[sizeof(T) / 2];
        } a;
#pragma unroll
        for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i)
            a.v[i] = __builtin_nontemporal_load(reinterpret_cast<const u4 *>(p) + i);
        return __builtin_bit_cast(Eight<T>, a);
    }
    if (wide && left >= 8) {
        const Piece a = *reinterpret_cast<const Piece *>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            r.v[i] = a.v[i];
        return r;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        r.v[i] = i < left ? p[i] : static_cast<T>(0.0f);
    return r;
}

// The largest magnitude's bits so far, in a form of T's own: starts at 0.
template <typename T>
__device__ __forceinline__ uint32_t most_of(uint32_t most, const Eight<T> &e) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            most = max(most, magnitude(e.v[i]));
    } else {
        const u4 pairs = __builtin_bit_cast(u4, e);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            most = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(us2, most),
                                                                          __builtin_bit_cast(us2, pairs[i] & 0x7fff7fffu)));
    }
    return most;
}

// That form as the byte that the block keeps.
template <typename T>
__device__ __forceinline__ uint32_t power_of_most(uint32_t most) {
    if constexpr (sizeof(T) == 4) {
        return power_of(most);
    } else {
        const uint16_t m = static_cast<uint16_t>(max(most & 0xffffu, most >> 16));
        return power_of(__float_as_uint(static_cast<float>(__builtin_bit_cast(T, m))));
    }
}

template <typename T>
__device__ __forceinline__ uint32_t codes8(const Eight<T> &e, uint32_t power) {
    if constexpr (sizeof(T) == 4) {
        return codes8(e.v, power);
    } else {
        const float scale = __uint_as_float(power ? power << 23 : 1u << 22);
        struct Pairs {
            uint32_t v[4];
        } pairs = __builtin_bit_cast(Pairs, e);
        uint32_t w = 0;
        if constexpr (__is_same(T, _Float16)) {
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, __builtin_bit_cast(h2, pairs.v[0]), scale, 0);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, __builtin_bit_cast(h2, pairs.v[1]), scale, 1);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, __builtin_bit_cast(h2, pairs.v[2]), scale, 2);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, __builtin_bit_cast(h2, pairs.v[3]), scale, 3);
        } else {
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bh2, pairs.v[0]), scale, 0);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bh2, pairs.v[1]), scale, 1);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bh2, pairs.v[2]), scale, 2);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bh2, pairs.v[3]), scale, 3);
        }
        return power == 255 ? 0 : w;
    }
}

// p (16 x 16, f4 a lane) = c + A (16 rows x 128) B (16 columns x 128), 4-bit codes
// with the scales of lane l in byte OP of sa and sb: lane l holds of each operand
// row l % 16 a block of 32 channels (any, the same for both), of the result column
// (B) l % 16, rows (A) 4 (l / 16) .. + 3.  Products and the sum of a block are
// exact; the scales are applied and the blocks and c added in 32 bits: 6e-8 of the
// terms' sum off (2e-7 where c is 1000 times as large; measured), as 32-bit additions are.
template <int OP>
__device__ __forceinline__ f4 mfma4(u4 a, u4 b, f4 c, uint32_t sa, uint32_t sb) {
    const i8 wide_a = {static_cast<int>(a[0]), static_cast<int>(a[1]), static_cast<int>(a[2]), static_cast<int>(a[3]), 0, 0, 0, 0};
    const i8 wide_b = {static_cast<int>(b[0]), static_cast<int>(b[1]), static_cast<int>(b[2]), static_cast<int>(b[3]), 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide_a, wide_b, c, 4, 4, OP, static_cast<int>(sa), OP,
                                                            static_cast<int>(sb));
}

}  // namespace spconv
