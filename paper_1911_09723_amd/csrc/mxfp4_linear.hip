// y = clamp(x W^T + b) for a weight and rows in 4 bits with a power of two for
// each 32 channels (mxfp4.hpp).
#include <algorithm>

#include "mxfp4_product.hpp"

namespace spconv {
namespace {

constexpr int kXcds = 8;

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

// PARTS: groups of wavefronts that share the lines, each its own run of them in its
// own buffers; the first adds up the sums.
template <class S, int PARTS>
__global__ void __launch_bounds__(PARTS *S::kThreads) linear4_tile(Linear4Args a, int32_t ctiles, int32_t ttiles, bool wide) {
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
    const int32_t loops = (a.lines + PARTS - 1) / PARTS, b0 = min(part * loops, a.lines - 1);
    const int32_t lines = min(max(a.lines - part * loops, 0), loops);
    const TileSource4<S> from = tile_source<S>(a, c0, t0, b0, wave, lane);
    f4 acc[S::NC][S::NT] = {};
    tile_product4<S>(acc, from, lines, loops, lds, wave, lane);
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
    const int32_t ch = c0 + channel_part<S>(wave) * S::NC * 16 + (lane >> 4) * 4;
    f4 bias[S::NC];
#pragma unroll
    for (int c = 0; c < S::NC; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            bias[c][i] = a.bias && ch + c * 16 + i < a.cout ? a.bias[ch + c * 16 + i] : 0.0f;
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

// One line of n (at most 16) rows in f32, f16 or bf16, quantised by a wavefront into its own
// part of LDS: 32 lanes a row, 8 values each, pieces of 16 bytes at piece ^ turn(row), then
// the rows' powers.  Returns the part of row lane % 16.
constexpr int kOwnBytes = 16 * 128 + 16 * 8;

template <typename T>
__device__ __forceinline__ LinePart line_quantized(const T *x, int64_t ldx, int32_t n, int32_t line, int32_t cols, bool wide,
                                                   int lane, unsigned char *own) {
    const int l = lane & 31;
    const int32_t c = line * kLine4 + 8 * l;
    Eight<T> v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (2 * i >= n)
            break;
        const int32_t row = min(2 * i + (lane >> 5), n - 1);
        v[i] = eight_tail(x + row * ldx + c, cols - c, wide);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (2 * i >= n)
            break;
        const int row = 2 * i + (lane >> 5);
        uint32_t m = most_of(0, v[i]);
        if constexpr (sizeof(T) == 2)
            m = max(m & 0xffffu, m >> 16);
        m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 1)));
        m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 2)));
        const uint32_t power = power_of_most<T>(m);
        *reinterpret_cast<uint32_t *>(own + row * 128 + ((l >> 2) ^ turn(row)) * 16 + (l & 3) * 4) = codes8(v[i], power);
        if ((l & 3) == 0)
            own[2048 + row * 8 + (l >> 2)] = static_cast<unsigned char>(power);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const int row = min(lane & 15, static_cast<int>(n) - 1), at = row * 128 + ((lane >> 4) * 2 ^ turn(row)) * 16;
    LinePart r;
    r.code[0] = *reinterpret_cast<const u4 *>(own + at);
    r.code[1] = *reinterpret_cast<const u4 *>(own + (at ^ 16));
    r.power = *reinterpret_cast<const uint16_t *>(own + 2048 + row * 8 + (lane >> 4) * 2);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    return r;
}

// Up to 16 rows, LDS only for rows that are quantised here and for the final sum: a workgroup
// has 16 CT channels, its wavefronts share the lines, U of each under way at once.  XT: Fp8
// (codes) or the type of rows that are quantised here.
template <typename XT, int CT, int U>
__global__ void __launch_bounds__(1024) linear4_stream(Linear4Args a, bool wide_x, bool wide) {
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int waves = blockDim.x >> 6;
    const int32_t c0 = blockIdx.x * 16 * CT;
    const int64_t pitch = static_cast<int64_t>(a.lines) * 128;
    int32_t ch[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c)
        ch[c] = min(c0 + c * 16 + (lane & 15), a.cout - 1);
    const int32_t row = min(lane & 15, a.n - 1);
    f4 acc[CT] = {};
    for (int32_t b0 = wave; b0 < a.lines; b0 += waves * U) {
        LinePart w[U][CT], x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int32_t b = min(b0 + u * waves, a.lines - 1);
#pragma unroll
            for (int c = 0; c < CT; ++c)
                w[u][c] = line_part(a.w + ch[c] * pitch, a.ws + (static_cast<int64_t>(b) * a.cout + ch[c]) * 8, b, lane);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int32_t b = min(b0 + u * waves, a.lines - 1);
            if constexpr (sizeof(XT) == 1)
                x[u] = line_part(static_cast<const uint8_t *>(a.x) + row * pitch, a.xs + (static_cast<int64_t>(b) * a.n + row) * 8,
                                 b, lane);
            else
                x[u] = line_quantized(static_cast<const XT *>(a.x), a.ldx, a.n, b, a.cin, wide_x, lane, lds + wave * kOwnBytes);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (b0 + u * waves >= a.lines)
                break;
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                acc[c] = mfma4<0>(w[u][c].code[0], x[u].code[0], acc[c], w[u][c].power, x[u].power);
                acc[c] = mfma4<1>(w[u][c].code[1], x[u].code[1], acc[c], w[u][c].power, x[u].power);
            }
        }
    }
    if constexpr (sizeof(XT) > 1)
        __syncthreads();  // the sums lie where other wavefronts' rows were
    sum_waves<CT>(acc, reinterpret_cast<f4 *>(lds), waves, wave, lane, [&](int i, f4 sum) {
        finish4(a, wide, lane & 15, c0 + i * 16 + (lane >> 4) * 4, sum);
    });
}

// Channels of a workgroup that quantises its rows itself.
int32_t row_channels(int32_t cout) { return cout > 4096 ? 32 : 16; }

constexpr int32_t kStreamRows = 16;  // most rows that take the stream kernel
constexpr int kStreamWaves = 16;

template <typename XT, int CT>
hipError_t stream_launch(const Linear4Args &a, bool wide_x, bool wide, hipStream_t stream) {
    const int waves = std::min(a.lines, kStreamWaves);
    const int32_t grid = (a.cout + 16 * CT - 1) / (16 * CT);
    const size_t lds = static_cast<size_t>(waves) * std::max(CT * 1024, sizeof(XT) == 1 ? 0 : kOwnBytes);
    if (sizeof(XT) == 1 && a.lines > waves)
        linear4_stream<XT, CT, sizeof(XT) == 1 ? 2 : 1><<<grid, waves * 64, lds, stream>>>(a, wide_x, wide);
    else
        linear4_stream<XT, CT, 1><<<grid, waves * 64, lds, stream>>>(a, wide_x, wide);
    return hipGetLastError();
}

template <typename XT>
hipError_t rows_launch(const Linear4Args &a, bool wide_x, bool wide, hipStream_t stream) {
    return row_channels(a.cout) == 32 ? stream_launch<XT, 2>(a, wide_x, wide, stream) : stream_launch<XT, 1>(a, wide_x, wide, stream);
}

template <class S, int PARTS = 1>
hipError_t tile_launch(const Linear4Args &a, bool wide, hipStream_t stream) {
    const int64_t ct = (a.cout + S::BC - 1) / S::BC, tt = (a.n + S::BT - 1) / S::BT;
    static std::atomic<uint64_t> done{0};
    const hipError_t ready = allow_lds(linear4_tile<S, PARTS>, PARTS * S::kLds, done);
    if (ready != hipSuccess)
        return ready;
    const int64_t grid = (ct * tt + kXcds - 1) / kXcds * kXcds;
    linear4_tile<S, PARTS><<<static_cast<uint32_t>(grid), PARTS * S::kThreads, PARTS * S::kLds, stream>>>(
        a, static_cast<int32_t>(ct), static_cast<int32_t>(tt), wide);
    return hipGetLastError();
}

}  // namespace

namespace {
int64_t tiles_of(int32_t n, int32_t cout, int32_t channels, int32_t rows) {
    return static_cast<int64_t>((cout + channels - 1) / channels) * ((n + rows - 1) / rows);
}

// Whether the stream kernel's wavefronts, with so many channels a workgroup, fit the card's
// compute units at 16 each.
bool one_round(int32_t lines, int32_t cout, int32_t channels) {
    return static_cast<int64_t>((cout + channels - 1) / channels) * std::min(lines, kStreamWaves) <= 256 * kStreamWaves;
}
}  // namespace

// The stream kernel quantises its rows itself, in every workgroup again: in place of a launch,
// which costs the host 3.5 us, a pass over the rows' line for each line that a wavefront has.
// Measured (bf16, two launches in brackets): 1 x 1024 -> 1024 3.3 us (4.8), 1 x 4096 -> 4096 5.2
// (7.0), 1 x 8192 -> 8192 11.0 (13.0), 4 x 4096 -> 8192 7.8 (8.3), 8 x 4096 -> 4096 7.8 (7.4); beyond,
// 8 x 8192 -> 1024 10.5 (8.8), 16 x 4096 -> 4096 11.2 (7.6), and with more wavefronts than the
// card holds 1 x 4096 -> 14336 11.9 (10.1).  In f32, whose rows take twice the registers (63 of them are
// spilled above 4096 channels), on the device alone: 1 x 4096 -> 4096 5.9 (6.8), 8 x 4096 -> 4096 8.6 (7.3),
// 4 x 4096 -> 8192 11.3 (9.0), 1 x 8192 -> 8192 13.8 (11.4): less than the launch that is saved on the host,
// more than two launches in a graph.
bool linear4_takes_rows(int32_t n, int32_t cin, int32_t cout) {
    const int32_t lines = lines_of(cin);
    return static_cast<int64_t>(n) * ((lines + kStreamWaves - 1) / kStreamWaves) <= 8 &&
           one_round(lines, cout, row_channels(cout));
}

// Which kernel, for codes.  Up to 16 rows the stream kernel while the card holds all its
// wavefronts (1 x 4096 -> 4096 4.8 us, tiles 5.9; 16 x 8192 -> 4096 7.4 and 7.7; not 16 x 8192 ->
// 8192, 12.8 and 9.9).  Then tiles, the largest that still give the card's 256 compute units
// work: 32 channels x 64 rows, four lines deep, while there are no more of those than compute
// units (24 x 4096 -> 8192 6.3 us, 64 x 64 7.3), with two groups of wavefronts that share the lines
// where half of them stand idle or the axis is long (128 x 8192 -> 1024 8.8, one group 9.9; 100 x
// 16384 -> 4096 15.9 and 17.6).  64 x 32 for few rows of more channels (32 x 4096 -> 28672 15.4, 64
// x 64 16.2).  64 x 64 while one round of them covers the card (256 x 4096 -> 4096 8.4, 128 x 64
// 10.2), 128 x 64 (300 x 4096 -> 4096 9.5, with one group of wavefronts 10.1, 128 x 128 11.6), 128 x
// 128 three deep (1024 x 4096 -> 4096 14.6, 128 x 64 17.9, 256 x 128 18.6).  256 x 256 where there
// are 160 (3000 x 4096 -> 4096, 192 tiles, 36.7, 256 x 128 39.8; 2048 rows, 128 tiles, 32.9 and 24.0),
// 256 x 128 three deep between, and 128 x 128 two deep, two on a compute unit, for short axes, which
// are bound by their start and end (8192 x 512 -> 1024 9.3, 256 x 128 9.7).
hipError_t launch_linear_mxfp4(const Linear4Args &a, hipStream_t stream) {
    const bool wide_x = reinterpret_cast<uintptr_t>(a.x) % 16 == 0 && a.ldx * (a.x_type == kF32 ? 4 : 2) % 16 == 0;
    const bool wide = a.cout % 4 == 0 && reinterpret_cast<uintptr_t>(a.y) % 16 == 0;
    if (a.x_type != kMxfp4)
        return a.x_type == kF32   ? rows_launch<float>(a, wide_x, wide, stream)
               : a.x_type == kF16 ? rows_launch<_Float16>(a, wide_x, wide, stream)
                                  : rows_launch<__bf16>(a, wide_x, wide, stream);
    if (a.n <= kStreamRows && one_round(a.lines, a.cout, 16))
        return stream_launch<Fp8, 1>(a, wide_x, wide, stream);
    auto tiles = [&](int32_t channels, int32_t rows) { return tiles_of(a.n, a.cout, channels, rows); };
    const int64_t least = tiles(32, 64);
    if (least <= 256)
        return (a.lines >= 16 && least <= 128) || a.lines >= 64 ? tile_launch<TileShape4<32, 64, 1, 4, 4>, 2>(a, wide, stream)
                                                                : tile_launch<TileShape4<32, 64, 1, 4, 4>>(a, wide, stream);
    if (a.n <= 32)
        return tile_launch<TileShape4<64, 32, 2, 2, 4>>(a, wide, stream);
    if (tiles(64, 64) <= 256)
        return tile_launch<TileShape4<64, 64, 1, 4, 4>>(a, wide, stream);
    if (tiles(128, 64) <= 256 || a.n <= 64)
        return a.lines >= 16 && a.n > 64 ? tile_launch<TileShape4<128, 64, 2, 2, 3>, 2>(a, wide, stream)
                                         : tile_launch<TileShape4<128, 64, 2, 2, 3>>(a, wide, stream);
    if (tiles(128, 128) <= 256)
        return tile_launch<TileShape4<128, 128, 2, 4, 3>>(a, wide, stream);
    if (tiles(256, 256) >= 160)
        return tile_launch<TileShape4<256, 256, 2, 4>>(a, wide, stream);
    return a.lines >= 8 ? tile_launch<TileShape4<256, 128, 2, 4, 3>>(a, wide, stream)
                        : tile_launch<TileShape4<128, 128, 2, 2>>(a, wide, stream);
}

}  // namespace spconv
