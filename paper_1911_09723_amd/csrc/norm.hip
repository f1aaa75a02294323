// Root-mean-square norm of rows, with the residual's addition in front and
// 8-bit codes behind it where asked:
//
//     h = x + r,  total = h rounded to r's type,  y = h * (1 / sqrt(sum h^2 / cols + eps)) * gain,
//
// in 32 bits but for what a row's threads found and the root, which are joined and taken in 64: a
// factor of all of a row is off by its rounding alone, and y by 4.3e-8 of it on average (5.5e-8
// with 32 bits there, 2048 columns; the time is the same.  With the products in 64 bits, or each
// with its rounding's error carried on, 3.6e-8, and 8192 x 4096 takes 28.0 to 32.6 and 30.3 us).  y
// is rounded once to its type, or quantised by blocks of 128 channels as quantize_fp8's rows are
// (fp8.hpp).  The norm is that of the 32-bit h, not of the rounded total: one rounding less
// between x and y.
//
// One pass: a row stays in registers between its sum of squares and its
// results, 8 neighbouring values a thread and piece, so that 16 lanes hold a
// block of 128.  What bounds it is traffic, below some MB the launch and one wait for
// the row's loads (1 x 1280: 2.9 us).
#include <type_traits>

#include "fp8.hpp"
#include "serve_ops.hpp"

namespace spconv {
namespace {

struct None {};

// A piece of 16 or 8 bytes, past the caches where `stream`: of a long call little is still there
// when the next one reads it, and it takes room from what is read.  bf16 with residual and codes,
// us, through the caches and past them: 8192 x 4096 52.2 and 46.3 (loads kept: 47.9), 2048 x 4096
// 16.6 and 14.4, 1024 x 4096 9.6 and 10.3.  The other types go by the same bytes of x; they were not
// compared.
template <typename V>
__device__ __forceinline__ void put(V *p, V v, bool stream) {
    if (stream)
        __builtin_nontemporal_store(v, p);
    else
        *p = v;
}

// `left` (any number) of 8 values to a row of T, rounded once.
template <typename T>
__device__ __forceinline__ void store8(T *p, int left, bool wide, bool stream, const float *v) {
    struct Eight {
        T v[8];
    } e;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        e.v[i] = static_cast<T>(v[i]);
    if (wide && left >= 8) {
        struct Pieces {
            u4 v[sizeof(T) / 2];
        };
        const Pieces pieces = __builtin_bit_cast(Pieces, e);
#pragma unroll
        for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i)
            put(reinterpret_cast<u4 *>(p) + i, pieces.v[i], stream);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < left)
            p[i] = e.v[i];
}

// Eight values, `left` of them there.
template <typename T>
__device__ __forceinline__ void read8(const T *p, int left, bool wide, bool stream, float *v) {
    if (stream && wide && left >= 8) {
        struct __attribute__((aligned(16))) Pieces {
            u4 v[sizeof(T) / 2];
        } pieces;
#pragma unroll
        for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i)
            pieces.v[i] = __builtin_nontemporal_load(reinterpret_cast<const u4 *>(p) + i);
        load8(reinterpret_cast<const T *>(&pieces), v);
        return;
    }
    load8_tail(p, left, wide, v);
}

// Eight values of h from column c on.
template <typename T, typename R>
__device__ __forceinline__ void load_sum(const NormArgs &a, int32_t row, int32_t c, float *h) {
    read8(static_cast<const T *>(a.x) + row * a.ldx + c, a.cols - c, a.wide_x, a.stream, h);
    if constexpr (!std::is_same_v<R, None>) {
        float r[8];
        read8(static_cast<const R *>(a.residual) + row * a.ldr + c, a.cols - c, a.wide_r, a.stream, r);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            h[i] += r[i];
    }
}

template <typename W>
__device__ __forceinline__ void load_gain(const NormArgs &a, int32_t c, float *g) {
    if (a.gain) {
        load8_tail(static_cast<const W *>(a.gain) + c, a.cols - c, a.wide_g, g);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        g[i] = 1.0f;
}

// What leaves for the eight values from column c on; every lane of a block's 16 comes here.
template <typename T, typename R>
__device__ __forceinline__ void finish8(const NormArgs &a, int32_t row, int32_t c, const float *h, const float *g,
                                        float inverse) {
    if constexpr (!std::is_same_v<R, None>)
        if (a.total)
            store8(static_cast<R *>(a.total) + row * a.ldt + c, a.cols - c, a.wide_t, a.stream, h);
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        v[i] = c + i < a.cols ? h[i] * inverse * g[i] : 0.0f;
    if (a.y) {
        if (a.y32)
            store8(static_cast<float *>(a.y) + row * a.ldy + c, a.cols - c, a.wide_y, a.stream, v);
        else
            store8(static_cast<T *>(a.y) + row * a.ldy + c, a.cols - c, a.wide_y, a.stream, v);
    }
    if (a.q) {
        uint32_t m = most8(v);
#pragma unroll
        for (int s = 1; s < 16; s *= 2)
            m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), s)));
        const int32_t b = c / kBlock;
        if (b >= a.kb)
            return;
        const Scale s = scale_of(m);
        put(reinterpret_cast<u2 *>(a.q + static_cast<int64_t>(row) * a.kb * kBlock + c),
            u2{codes4(v, s.inv), codes4(v + 4, s.inv)}, a.stream);
        if (c % kBlock == 0)
            a.scale[static_cast<int64_t>(b) * a.rows + row] = s.scale;
    }
}

// The sum over a row's THREADS threads, in a fixed order.
template <int THREADS>
__device__ __forceinline__ double row_sum(double v, double *part) {
#pragma unroll
    for (int s = 1; s < 64; s *= 2)
        v += __shfl_xor(v, s);
    if constexpr (THREADS > 64) {
        if ((threadIdx.x & 63) == 0)
            part[threadIdx.x >> 6] = v;
        __syncthreads();
        v = part[threadIdx.x & (THREADS / 64 - 1)];
#pragma unroll
        for (int s = 1; s < THREADS / 64; s *= 2)
            v += __shfl_xor(v, s);
    }
    return v;
}

__device__ __forceinline__ float add_squares(const float *h, float sum) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
        sum = fmaf(h[i], h[i], sum);
    return sum;
}

// 1 / sqrt(sum / cols + eps): the instruction's 2^-25 or so, and one step of Newton's.
__device__ __forceinline__ float inverse_of(const NormArgs &a, double sum) {
    const double mean = fma(sum, a.share, static_cast<double>(a.eps)), r = __builtin_amdgcn_rsq(mean);
    return static_cast<float>(mean > 0 && mean < INFINITY ? fma(0.5 * r, fma(-mean * r, r, 1.0), r) : r);
}

// THREADS a row, VECS pieces of 8 values each.
template <typename T, typename R, typename W, int THREADS, int VECS>
__global__ void __launch_bounds__(THREADS < 256 ? 256 : THREADS) norm_rows(NormArgs a) {
    __shared__ double part[16];
    const int32_t row = THREADS < 256 ? blockIdx.x * (256 / THREADS) + threadIdx.x / THREADS : blockIdx.x;
    if (row >= a.rows)  // whole wavefronts, of which each has its own row there
        return;
    const int32_t c0 = threadIdx.x % THREADS * 8;
    float h[VECS][8];
#pragma unroll
    for (int u = 0; u < VECS; ++u)
        load_sum<T, R>(a, row, c0 + u * THREADS * 8, h[u]);
    float sum = 0;
#pragma unroll
    for (int u = 0; u < VECS; ++u)
        sum = add_squares(h[u], sum);
    const float inverse = inverse_of(a, row_sum<THREADS>(sum, part));
#pragma unroll
    for (int u = 0; u < VECS; ++u) {
        float g[8];
        load_gain<W>(a, c0 + u * THREADS * 8, g);
        finish8<T, R>(a, row, c0 + u * THREADS * 8, h[u], g, inverse);
    }
}

// Rows that registers do not hold: read twice, past the caches both times where the call is long (512 x
// 40000 in bf16 41 us with residual, 4.0 TB/s by what has to move once; the first time through
// them was not compared).  A thread reads what it writes before it writes it, so total and y may lie
// where residual and x do.
template <typename T, typename R, typename W>
__global__ void __launch_bounds__(1024) norm_long(NormArgs a) {
    __shared__ double part[16];
    const int32_t row = blockIdx.x;
    float sum = 0;
    for (int32_t c = threadIdx.x * 8; c < a.cols; c += 8192) {
        float h[8];
        load_sum<T, R>(a, row, c, h);
        sum = add_squares(h, sum);
    }
    const float inverse = inverse_of(a, row_sum<1024>(sum, part));
    for (int32_t c0 = 0; c0 < a.cols; c0 += 8192) {  // whole wavefronts: blocks are found across lanes
        const int32_t c = c0 + threadIdx.x * 8;
        float h[8], g[8];
        load_sum<T, R>(a, row, c, h);
        load_gain<W>(a, c, g);
        finish8<T, R>(a, row, c, h, g, inverse);
    }
}

// Threads a row: as many as there are pieces where rows are few (16 x 4096: 4.0 us, half as many
// 4.8); else two pieces a thread, whose loads are under way together (bf16 with residual and codes:
// 8192 x 4096 46.3 us, 5.1 TB/s, one piece 48.9, four 53.5; 8192 x 2048 25.4 with one or two; 4096
// x 8192 45.8, one piece 49.8).
template <typename T, typename R, typename W>
hipError_t launch(const NormArgs &a, hipStream_t stream) {
    const int32_t pieces = (a.cols + 7) / 8;
    const bool few = a.rows < 512;
    if (pieces <= 64)
        norm_rows<T, R, W, 64, 1><<<(a.rows + 3) / 4, 256, 0, stream>>>(a);
    else if (pieces <= 128 && !few)
        norm_rows<T, R, W, 64, 2><<<(a.rows + 3) / 4, 256, 0, stream>>>(a);
    else if (pieces <= 256)
        norm_rows<T, R, W, 256, 1><<<a.rows, 256, 0, stream>>>(a);
    else if (pieces <= 512 && few)
        norm_rows<T, R, W, 512, 1><<<a.rows, 512, 0, stream>>>(a);
    else if (pieces <= 512)
        norm_rows<T, R, W, 256, 2><<<a.rows, 256, 0, stream>>>(a);
    else if (pieces <= 1024 && few)
        norm_rows<T, R, W, 1024, 1><<<a.rows, 1024, 0, stream>>>(a);
    else if (pieces <= 1024)
        norm_rows<T, R, W, 512, 2><<<a.rows, 512, 0, stream>>>(a);
    else if (pieces <= 2048)
        norm_rows<T, R, W, 1024, 2><<<a.rows, 1024, 0, stream>>>(a);
    else if (pieces <= 4096)
        norm_rows<T, R, W, 1024, 4><<<a.rows, 1024, 0, stream>>>(a);
    else
        norm_long<T, R, W><<<a.rows, 1024, 0, stream>>>(a);
    return hipGetLastError();
}

template <typename T, typename R>
hipError_t with_gain(const NormArgs &a, bool gain32, hipStream_t stream) {
    if constexpr (!std::is_same_v<T, float>)
        if (!gain32)
            return launch<T, R, T>(a, stream);
    return launch<T, R, float>(a, stream);
}

template <typename T>
hipError_t with_residual(const NormArgs &a, bool residual32, bool gain32, hipStream_t stream) {
    if (!a.residual)
        return with_gain<T, None>(a, gain32, stream);
    if constexpr (!std::is_same_v<T, float>)
        if (!residual32)
            return with_gain<T, T>(a, gain32, stream);
    return with_gain<T, float>(a, gain32, stream);
}

bool wide(const void *p, int64_t ld, int64_t size) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * size % 16 == 0;
}

}  // namespace

hipError_t launch_norm(NormArgs a, int32_t type, bool residual32, bool gain32, hipStream_t stream) {
    const int64_t size = type == kF32 ? 4 : 2, of_r = residual32 ? 4 : size;
    a.wide_x = wide(a.x, a.ldx, size);
    a.wide_r = wide(a.residual, a.ldr, of_r);
    a.wide_t = wide(a.total, a.ldt, of_r);
    a.wide_g = wide(a.gain, 0, 1);
    a.wide_y = wide(a.y, a.ldy, a.y32 ? 4 : size);
    a.share = 1.0 / a.cols;
    a.stream = static_cast<int64_t>(a.rows) * a.cols * size >= 16 << 20;
    return type == kF32   ? with_residual<float>(a, residual32, gain32, stream)
           : type == kF16 ? with_residual<_Float16>(a, residual32, gain32, stream)
                          : with_residual<__bf16>(a, residual32, gain32, stream);
}

}  // namespace spconv
