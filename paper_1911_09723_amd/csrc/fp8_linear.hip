// y = clamp(x W^T + b) for a weight in 8 bits with a scale for each 128 x 128
// block and rows with a scale for each 128 channels (fp8.hpp, fp8_product.hpp).
#include <algorithm>

#include "expert_ops.hpp"
#include "fp8_product.hpp"

namespace spconv {
namespace {

constexpr int kXcds = 8;

__device__ __forceinline__ f4 bias4(const float *bias, int32_t ch, int32_t cout) {
    f4 v{0, 0, 0, 0};
    if (bias)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            v[i] = ch + i < cout ? bias[ch + i] : 0.0f;
    return v;
}

__device__ __forceinline__ void finish(const LinearArgs &a, bool wide, int32_t row, int32_t ch, f4 v) {
    if (row >= a.n || ch >= a.cout)
        return;
    v += bias4(a.bias, ch, a.cout);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        v[i] = clamp_to(v[i], a.lo, a.hi);
    store4(a.y, a.y_type, static_cast<int64_t>(row) * a.cout + ch, v, a.cout - ch, wide);
}

// PARTS: groups of wavefronts that share the blocks of the input channels, each
// its own run of them in its own buffers; the first adds up the sums.  SPLIT:
// workgroups share them, too (gridDim.y), and linear_join adds up theirs.
template <class S, bool EXACT, int PARTS, bool SPLIT>
__global__ void __launch_bounds__(PARTS *S::kThreads) linear_tile(LinearArgs a, int32_t ctiles, int32_t ttiles, bool wide) {
    extern __shared__ __attribute__((aligned(1024))) unsigned char all_lds[];
    const int lane = threadIdx.x & 63, all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int part = PARTS > 1 ? all / S::kWaves : 0, wave = all - part * S::kWaves;
    unsigned char *lds = all_lds + part * S::kLds;
    // neighbouring tiles on one XCD, in groups of 8 row tiles: they share W and X in its L2
    const int32_t per = gridDim.x / kXcds, id = blockIdx.x % kXcds * per + blockIdx.x / kXcds;
    if (id >= ctiles * ttiles)
        return;
    const int32_t group = id / (8 * ctiles), high = min(8, ttiles - 8 * group), in = id - group * 8 * ctiles;
    const int32_t ct = in / high, tt = group * 8 + in - ct * high;
    const int32_t c0 = ct * S::BC, t0 = tt * S::BT;
    const uint32_t pitch = a.kb * kBlock;
    const int32_t run = SPLIT ? blockIdx.y * PARTS + part : part, runs = SPLIT ? gridDim.y * PARTS : PARTS;
    const int32_t loops = (a.kb + runs - 1) / runs, b0 = min(run * loops, a.kb - 1);
    const int32_t kb = min(max(a.kb - run * loops, 0), loops);
    TileSource<S> from;
    from.w = a.w + static_cast<int64_t>(c0) * pitch + b0 * kBlock;
    from.x = static_cast<const uint8_t *>(a.x) + static_cast<int64_t>(t0) * pitch + b0 * kBlock;
    from.w_bytes = min(S::BC, a.cout - c0) * pitch - b0 * kBlock;
    from.x_bytes = min(S::BT, a.n - t0) * pitch - b0 * kBlock;
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) {
        const int line = tile_line<S>(wave, lane, i);
        if (line < S::BC)
            from.at[i] = line < a.cout - c0 ? line * pitch + tile_byte(line, lane) : from.w_bytes;
        else
            from.at[i] = line - S::BC < a.n - t0 ? (line - S::BC) * pitch + tile_byte(line, lane) : from.x_bytes;
    }
    from.rows = a.n - t0;
    from.xs = a.xs + static_cast<int64_t>(b0) * a.n;
    from.xs_at = min(t0 + wave % (S::BT / 64) * 64 + lane, a.n - 1) * 4u;
    from.xs_step = a.n * 4u;
    from.xs_bytes = from.xs_step * (a.kb - b0);
    const int wc = channel_part<S>(wave);
    const int32_t cw = c0 + wc * S::NC * 16;
    const float *ws = a.ws + static_cast<int64_t>(min(cw, a.cout - 1) / kBlock) * a.kb + b0;
    f4 acc[S::NC][S::NT] = {};
    float total[S::NT] = {};
    tile_product<S, EXACT, false>(acc, total, from, ws, nullptr, kb, loops, lds, wave, lane);
    if constexpr (PARTS > 1) {
        constexpr int kPieces = S::NC * S::NT;
        static_assert(kPieces * S::kThreads * 16 <= S::kLds, "a part's sums fit where its operands were");
        auto at = [&](int p, int c, int t) {
            return reinterpret_cast<f4 *>(all_lds + p * S::kLds) + (wave * kPieces + c * S::NT + t) * 64 + lane;
        };
        if (part > 0)
#pragma unroll
            for (int c = 0; c < S::NC; ++c)
#pragma unroll
                for (int t = 0; t < S::NT; ++t)
                    *at(part, c, t) = acc[c][t];
        __syncthreads();
        if (part > 0)
            return;
#pragma unroll
        for (int p = 1; p < PARTS; ++p)
#pragma unroll
            for (int c = 0; c < S::NC; ++c)
#pragma unroll
                for (int t = 0; t < S::NT; ++t)
                    acc[c][t] += *at(p, c, t);
    }
    const int32_t ch = cw + (lane >> 4) * 4;
    if constexpr (SPLIT) {
        const int32_t pitch4 = (a.cout + 3) / 4 * 4;
        store_tile<S>(acc, a.partial + static_cast<int64_t>(blockIdx.y) * a.n * pitch4, kF32, t0, a.n - t0, ch, pitch4, true,
                      wave, lane, lds, [](f4 v, int, int) { return v; });
        return;
    }
    f4 bias[S::NC];
#pragma unroll
    for (int c = 0; c < S::NC; ++c)
        bias[c] = bias4(a.bias, ch + c * 16, a.cout);
    const bool clamp = a.lo > -INFINITY || a.hi < INFINITY;
    store_tile<S>(acc, a.y, a.y_type, t0, a.n - t0, ch, a.cout, wide, wave, lane, lds, [&](f4 v, int c, int) {
        v += bias[c];
        if (clamp)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                v[i] = clamp_to(v[i], a.lo, a.hi);
        return v;
    });
}

// The sum of `splits` workgroups' results, in their order; a thread has four channels.
__global__ void __launch_bounds__(256) linear_join(LinearArgs a, int32_t splits, bool wide) {
    const int32_t pieces = (a.cout + 3) / 4;
    const int64_t id = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int32_t row = static_cast<int32_t>(id / pieces), ch = static_cast<int32_t>(id - row * static_cast<int64_t>(pieces)) * 4;
    if (row >= a.n)
        return;
    const f4 *from = reinterpret_cast<const f4 *>(a.partial) + id;
    f4 sum = *from;
    for (int32_t s = 1; s < splits; ++s)
        sum += from[static_cast<int64_t>(s) * a.n * pieces];
    finish(a, wide, row, ch, sum);
}

// XT: Fp8 (codes) or the type of rows that are quantised here.
template <typename XT, int TT, int CT, int U>
__global__ void __launch_bounds__(1024) linear_stream(LinearArgs a, bool wide_x, bool wide) {
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int waves = blockDim.x >> 6;
    const int32_t c0 = blockIdx.x * 16 * CT, t0 = blockIdx.y * 16 * TT;
    const int64_t pitch = static_cast<int64_t>(a.kb) * kBlock;
    const uint8_t *w[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c)
        w[c] = a.w + min(c0 + c * 16 + (lane & 15), a.cout - 1) * pitch;
    const float *ws = a.ws + static_cast<int64_t>(c0 / kBlock) * a.kb;
    int32_t row[TT];
#pragma unroll
    for (int t = 0; t < TT; ++t)
        row[t] = min(t0 + t * 16 + (lane & 15), a.n - 1);
    f4 acc[CT * TT] = {};
    for (int32_t b0 = wave; b0 < a.kb; b0 += waves * U) {
        i8 wf[U][CT];
        RowPart xp[U][TT];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int32_t b = min(b0 + u * waves, a.kb - 1);
#pragma unroll
            for (int c = 0; c < CT; ++c)
                wf[u][c] = weight_part(w[c], b, lane);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int32_t b = min(b0 + u * waves, a.kb - 1);
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                if constexpr (sizeof(XT) == 1)
                    xp[u][t] = row_codes(static_cast<const uint8_t *>(a.x) + row[t] * pitch,
                                         a.xs + static_cast<int64_t>(b) * a.n + row[t], b, lane);
                else
                    xp[u][t] = row_quantized(static_cast<const XT *>(a.x) + row[t] * a.ldx, b, a.cin, wide_x, lane);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (b0 + u * waves >= a.kb)
                break;
            const float sw = ws[b0 + u * waves];
            Halves wh[CT];
#pragma unroll
            for (int c = 0; c < CT; ++c)
                wh[c] = halves(wf[u][c]);
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                const Halves xh = halves(xp[u][t].code);
                const float s = xp[u][t].scale * sw;
#pragma unroll
                for (int c = 0; c < CT; ++c) {
                    const f4 p = mfma128(wh[c], xh);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        acc[c * TT + t][i] = fmaf(s, p[i], acc[c * TT + t][i]);
                }
            }
        }
    }
    sum_waves<CT * TT>(acc, reinterpret_cast<f4 *>(lds), waves, wave, lane, [&](int i, f4 sum) {
        finish(a, wide, t0 + i % TT * 16 + (lane & 15), c0 + i / TT * 16 + (lane >> 4) * 4, sum);
    });
}

constexpr int32_t kStreamRows = 32;  // most rows that take the stream kernel
constexpr int kStreamWaves = 16;

size_t size_of(int32_t type) { return type == kF32 ? 4 : type == kFp8 ? 1 : 2; }

template <typename XT, int TT, int CT>
hipError_t stream_launch(const LinearArgs &a, bool wide_x, bool wide, hipStream_t stream) {
    const int waves = std::min(a.kb, kStreamWaves);
    const dim3 grid((a.cout + 16 * CT - 1) / (16 * CT), (a.n + 16 * TT - 1) / (16 * TT));
    const size_t lds = static_cast<size_t>(waves) * CT * TT * 1024;
    if (a.kb > waves)
        linear_stream<XT, TT, CT, 2><<<grid, waves * 64, lds, stream>>>(a, wide_x, wide);
    else
        linear_stream<XT, TT, CT, 1><<<grid, waves * 64, lds, stream>>>(a, wide_x, wide);
    return hipGetLastError();
}

template <class S, bool EXACT, int PARTS = 1, bool SPLIT = false>
hipError_t tile_launch(const LinearArgs &a, bool wide, hipStream_t stream, int32_t splits = 1) {
    const int64_t ct = (a.cout + S::BC - 1) / S::BC, tt = (a.n + S::BT - 1) / S::BT;
    static std::atomic<uint64_t> done{0};
    const hipError_t ready = allow_lds(linear_tile<S, EXACT, PARTS, SPLIT>, PARTS * S::kLds, done);
    if (ready != hipSuccess)
        return ready;
    const int64_t grid = (ct * tt + kXcds - 1) / kXcds * kXcds;
    linear_tile<S, EXACT, PARTS, SPLIT><<<dim3(static_cast<uint32_t>(grid), splits), PARTS * S::kThreads, PARTS * S::kLds, stream>>>(
        a, static_cast<int32_t>(ct), static_cast<int32_t>(tt), wide);
    return hipGetLastError();
}

}  // namespace

// The stream kernel quantises its rows itself, which saves a launch, but does so in every
// workgroup: a wavefront's blocks times a compute unit's workgroups are how often it waits for a
// conversion.  Measured (bf16, two launches in brackets): once, 1 x 1024 -> 1024 3.8 us (5.1); twice,
// 1 x 4096 -> 4096 8.9 (8.2), 1 x 1024 -> 8192 5.0 (5.7), 32 x 4096 -> 2048 9.7 (10.4), and the
// second launch costs the host 3.5; four times, 1 x 8192 -> 1024 13.3 (10.2), 32 x 1024 -> 8192 8.7
// (7.5), 24 x 4096 -> 4096 18.3 (10.8).
bool linear_takes_rows(int32_t n, int32_t cin, int32_t cout) {
    const int64_t groups = static_cast<int64_t>((cout + 15) / 16) * ((n + 15) / 16);
    return n <= kStreamRows && (blocks_of(cin) + kStreamWaves - 1) / kStreamWaves * ((groups + 255) / 256) <= 2;
}

namespace {
int64_t tiles_of(int32_t n, int32_t cout, int32_t channels, int32_t rows) {
    return static_cast<int64_t>((cout + channels - 1) / channels) * ((n + rows - 1) / rows);
}

// Whether codes take the stream kernel: few rows of a small weight, whose time is that of a few
// loads one after the other (16 x 2048 -> 4096: 4.5 us, the smallest tiles 5.9; 16 x 4096 -> 4096
// 7.0 and 8.2).  Every workgroup of it reads all rows, so that a larger weight is read faster by
// tiles: 16 x 5120 -> 5120 13.6 and 9.4, 1 x 8192 -> 8192 15.1 and 13.4; 24 x 2048 -> 4096 5.2 and
// 5.8, x 8192 7.6 and 5.9.  Results in 32 bits take exact products, half as fast in tiles and as fast
// here: 24 x 8192 -> 8192 20.7 and 25, but 32 x 2048 -> 32768 27.7 and 16.5.
bool streams(int32_t n, int32_t kb, int32_t cout, bool exact) {
    const int64_t weight = static_cast<int64_t>(kb) * kBlock * cout;
    return n <= kStreamRows && (weight < (n <= 16 ? 24 << 20 : 16 << 20) || (exact && cout <= 24576));
}
}  // namespace

// A compute unit takes in some 75 GB/s here, so a long axis of few tiles is shared by up to eight
// workgroups a tile, at the price of a second launch that adds up their sums: 128 x 8192 -> 1024
// 10.6 us, unshared 15.4; 32 x 16384 -> 512 9.8, over the stream kernel 24.6; 128 x 4096 -> 2048 9.7 and
// 9.4, 128 x 8192 -> 4096 (128 tiles) 14.7 and 16.4, the launch's 3.5 us on the host not counted.
int32_t linear_splits(int32_t n, int32_t cin, int32_t cout) {
    const int64_t tiles = tiles_of(n, cout, 64, 64);
    if (n <= 16 || blocks_of(cin) < 48 || tiles > 64)
        return 1;
    return static_cast<int32_t>(std::min<int64_t>(256 / tiles, 8));
}

// Which kernel.  Few rows of a small weight the stream kernel, with 32 channels a workgroup in
// place of 16 where every compute unit still has one (results in 32 bits, 32 x 8192 -> 8192: 22 us,
// with 16 channels 29; 16-bit ones of 32 x 8192 -> 4096 15.4, with 32 channels 19.6).  Then tiles, the
// largest that still give the card's 256 compute units work.  64 x 64, four blocks deep, where there are
// no more of those than compute units; from 8 blocks on two groups of wavefronts share them, since one
// wavefront a SIMD waits for itself at every step of a block (128 x 4096 -> 4096 9.8 us, one group
// 11.7; 128 x 512 -> 8192 4.6 and 4.2).  64 x 64, two on a compute unit, also where one tile has all rows and
// there are enough to level out (64 x 4096 -> 128256 121 us, 128 x 64 146; 16 x 2048 -> 32768
// 12.7 and 19.5; 64 x 4096 -> 20000, 313 tiles, 18.7 and 16.4).  256 x 256 from 112 on (2048 rows of
// 4096 -> 4096: 47.8 against 52.1; 1536: 39.4 against 39.0 with 96).  Between, while a compute unit has
// one: 128 x 64 with twice four wavefronts from 16 blocks on (300 rows of 4096 -> 4096: 12.9 us, with four
// 15.4; 192 of 8192 -> 8192 24.1 and 28.2), with eight below (1900 rows of 1024 -> 1000: 6.8, four 7.7),
// then 128 x 128 three deep (1024 rows of 4096 -> 4096: 23.4, 128 x 64 two deep 25.9); else 128 x 64
// two deep (1400 rows of 512 -> 4096: 8.5 against 10.9).  Results in 32 bits: 256 x 256 from 192 on (2048 rows,
// 128 tiles: 97 us against 69 in tiles of 128 x 128; 8192 rows, 512 tiles: 207 against 252).
hipError_t launch_linear_fp8(const LinearArgs &a, hipStream_t stream) {
    const bool wide_x = reinterpret_cast<uintptr_t>(a.x) % 16 == 0 && a.ldx * size_of(a.x_type) % 16 == 0;
    const bool wide = a.cout % 4 == 0 && reinterpret_cast<uintptr_t>(a.y) % 16 == 0;
    if (a.x_type != kFp8)
        return a.x_type == kF32   ? stream_launch<float, 1, 1>(a, wide_x, wide, stream)
               : a.x_type == kF16 ? stream_launch<_Float16, 1, 1>(a, wide_x, wide, stream)
                                  : stream_launch<__bf16, 1, 1>(a, wide_x, wide, stream);
    const bool exact = a.y_type == kF32;
    const int32_t splits = linear_splits(a.n, a.cin, a.cout);
    if (streams(a.n, a.kb, a.cout, exact) && splits == 1) {
        const bool pairs = a.n > 8 && a.cout >= 8192;
        if (a.n <= 16)
            return pairs ? stream_launch<Fp8, 1, 2>(a, wide_x, wide, stream) : stream_launch<Fp8, 1, 1>(a, wide_x, wide, stream);
        return pairs ? stream_launch<Fp8, 2, 2>(a, wide_x, wide, stream) : stream_launch<Fp8, 2, 1>(a, wide_x, wide, stream);
    }
    auto tiles = [&](int32_t channels, int32_t rows) { return tiles_of(a.n, a.cout, channels, rows); };
    if (splits > 1) {
        const hipError_t e = exact ? tile_launch<TileShape<64, 64, 1, 4, 4>, true, 2, true>(a, wide, stream, splits)
                                   : tile_launch<TileShape<64, 64, 1, 4, 4>, false, 2, true>(a, wide, stream, splits);
        if (e != hipSuccess)
            return e;
        const int64_t pieces = static_cast<int64_t>(a.n) * ((a.cout + 3) / 4);
        linear_join<<<static_cast<uint32_t>((pieces + 255) / 256), 256, 0, stream>>>(a, splits, wide);
        return hipGetLastError();
    }
    const int64_t small = tiles(64, 64);
    if (small <= 256 || (small > 384 && a.n <= 64))
        return a.kb < 8 || small > 256 ? exact ? tile_launch<TileShape<64, 64, 1, 4, 4>, true>(a, wide, stream)
                                : tile_launch<TileShape<64, 64, 1, 4, 4>, false>(a, wide, stream)
               : exact  ? tile_launch<TileShape<64, 64, 1, 4, 4>, true, 2>(a, wide, stream)
                        : tile_launch<TileShape<64, 64, 1, 4, 4>, false, 2>(a, wide, stream);
    if (tiles(256, 256) >= (exact ? 192 : 112))
        return exact ? tile_launch<TileShape<256, 256, 2, 4>, true>(a, wide, stream)
                     : tile_launch<TileShape<256, 256, 2, 4>, false>(a, wide, stream);
    if (tiles(128, 64) <= 256)
        return a.kb < 16 ? exact ? tile_launch<TileShape<128, 64, 2, 4, 4>, true>(a, wide, stream)
                                 : tile_launch<TileShape<128, 64, 2, 4, 4>, false>(a, wide, stream)
               : exact   ? tile_launch<TileShape<128, 64, 2, 2, 3>, true, 2>(a, wide, stream)
                         : tile_launch<TileShape<128, 64, 2, 2, 3>, false, 2>(a, wide, stream);
    if (tiles(128, 128) <= 256)
        return exact ? tile_launch<TileShape<128, 128, 2, 4, 3>, true>(a, wide, stream)
                     : tile_launch<TileShape<128, 128, 2, 4, 3>, false>(a, wide, stream);
    return exact ? tile_launch<TileShape<128, 128, 2, 2>, true>(a, wide, stream)
                 : tile_launch<TileShape<128, 64, 2, 2>, false>(a, wide, stream);
}

}  // namespace spconv
