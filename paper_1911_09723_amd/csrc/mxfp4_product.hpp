// The tile core of 4-bit rows and weights (mxfp4.hpp): channels r (rows of W) x
// rows t of X over lines b of 256 input channels,
//
//     acc[r][t] += sum over b of (W[r] . X[t] over line b),
//
// on the instruction that takes 128 channels with a power of two for each 32 and
// adds to the running sum itself.  W is its row operand: a lane holds one row of
// X and four neighbouring channels.
#pragma once

#include "fp8_product.hpp"
#include "mxfp4.hpp"

namespace spconv {

// BC channels x BT rows, WC x WT wavefronts, each NC x NT pieces of 16 x 16.
template <int BC_, int BT_, int WC_, int WT_, int STAGES_ = 2>
struct TileShape4 {
    static constexpr int BC = BC_, BT = BT_, WC = WC_, WT = WT_;
    static constexpr int kWaves = WC * WT, kThreads = 64 * kWaves;
    static constexpr int NC = BC / WC / 16, NT = BT / WT / 16;
    static constexpr int kLines = BC + BT;
    static constexpr int kLoads = kLines / 8 / kWaves;       // of lines: 8 an instruction
    static constexpr int kWeightLoads = BC / 8 / kWaves;     // the first of them: W's
    static constexpr int kScaleW = (BC * 8 + 1023) / 1024;   // instructions for W's scales of a line
    static constexpr int kScales = kScaleW + (BT * 8 + 1023) / 1024;
    static constexpr int kEach = kLoads + 1;                 // loads of a wavefront and line
    static constexpr int kProducts = 2 * NC * NT;            // of a wavefront and line
    static constexpr int kStages = STAGES_;
    static constexpr int kStage = kLines * 128 + kScales * 1024;
    static constexpr int kLds = kStages * kStage;
    static_assert(BC % (8 * kWaves) == 0 && BT % (8 * kWaves) == 0 && kScales <= kWaves && kProducts >= kEach,
                  "whole loads a wavefront");
};

// The byte of its line that this lane copies.  A line's 16-byte pieces are stored
// at piece ^ turn(line).  A wavefront reads LDS 16 lanes at a time, lanes 0 to 3
// and 12 to 15 of one quarter with 4 to 11 of the next, hence of lines 0 to 3 and
// 12 to 15 one piece and of lines 4 to 11 another, whose number differs in bit 1:
// with the three bits above line's lowest, rotated, for turn, those 16 lie in
// different 16-byte columns of LDS's 256 bytes (the bits as they are, which do for
// pieces that differ in bit 0: 44% of LDS's cycles were conflicts).
__device__ __forceinline__ int turn(int line) {
    const int k = line >> 1 & 7;
    return (k << 1 & 7) | k >> 2;
}
__device__ __forceinline__ int tile_byte4(int line, int lane) { return ((lane & 7) ^ turn(line)) * 16; }

// What a tile reads: W and X from their bases, this lane's offsets of its lines
// (line 0 of the channels), and the scales of its instruction, step bytes from
// line to line.  Bytes: what each base covers; past it reads are zeros, dword by
// dword: the last pair of rows may be half there.
template <class S>
struct TileSource4 {
    const uint8_t *w, *x, *s;
    uint32_t w_bytes, x_bytes, s_bytes, s_step;
    uint32_t at[S::kLoads], s_at;
    int32_t rows;  // how many of the tile's rows there are
};

// The tile at channel c0 and row t0, its lines from b0 on.
template <class S>
__device__ __forceinline__ TileSource4<S> tile_source(const Linear4Args &a, int32_t c0, int32_t t0, int32_t b0, int wave,
                                                      int lane) {
    const uint32_t pitch = a.lines * 128;
    TileSource4<S> from;
    from.w = a.w + static_cast<int64_t>(c0) * pitch + b0 * 128;
    from.x = static_cast<const uint8_t *>(a.x) + static_cast<int64_t>(t0) * pitch + b0 * 128;
    from.w_bytes = min(S::BC, a.cout - c0) * pitch - b0 * 128;
    from.x_bytes = min(S::BT, a.n - t0) * pitch - b0 * 128;
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) {
        const int line = tile_line<S>(wave, lane, i);
        if (line < S::BC)
            from.at[i] = line < a.cout - c0 ? line * pitch + tile_byte4(line, lane) : from.w_bytes;
        else
            from.at[i] = line - S::BC < a.n - t0 ? (line - S::BC) * pitch + tile_byte4(line, lane) : from.x_bytes;
    }
    // one instruction for 128 rows of scales; wavefronts past the last do one of them again
    const int part = wave % S::kScales;
    const bool of_w = part < S::kScaleW;
    const uint32_t all = of_w ? a.cout : a.n;
    from.s_step = all * 8;
    from.s = (of_w ? a.ws : a.xs) + static_cast<int64_t>(b0) * from.s_step;
    from.s_bytes = from.s_step * (a.lines - b0);
    from.s_at = ((of_w ? c0 + part * 128 : t0 + (part - S::kScaleW) * 128) + lane * 2) * 8u;
    from.rows = a.n - t0;
    return from;
}

// acc[c][t] += the products over `lines` lines; loops: that, or more where other
// wavefronts of the workgroup, which it meets line by line, have more.
template <class S>
__device__ __forceinline__ void tile_product4(f4 (&acc)[S::NC][S::NT], const TileSource4<S> &from, int32_t lines,
                                              int32_t loops, unsigned char *lds, int wave, int lane) {
#ifdef __HIP_DEVICE_COMPILE__  // the host's pass knows no buffer resources
    const int wc = channel_part<S>(wave), wt = row_part<S>(wave);
    auto load = [&](int i, int32_t b, unsigned char *buf) {
        if (i < S::kLoads) {
            const bool of_w = i < S::kWeightLoads;
            const uint32_t bytes = of_w ? from.w_bytes : from.x_bytes;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                make_rsrc(of_w ? from.w : from.x, b < lines ? bytes : 0),
                (__attribute__((address_space(3))) void *)(buf + (wave + i * S::kWaves) * 1024), 16, from.at[i], b * 128,
                0, 0);
        } else {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                make_rsrc(from.s, b < lines ? from.s_bytes : 0),
                (__attribute__((address_space(3))) void *)(buf + S::kLines * 128 + wave % S::kScales * 1024), 16,
                from.s_at + b * from.s_step, 0, 0, 0);
        }
    };
#pragma unroll
    for (int st = 0; st < S::kStages - 1; ++st)
#pragma unroll
        for (int i = 0; i < S::kEach; ++i)
            load(i, st, lds + st * S::kStage);
    int32_t at_stage = 0, to_stage = (S::kStages - 1) * S::kStage;
    auto next_stage = [](int32_t at) { return at == (S::kStages - 1) * S::kStage ? 0 : at + S::kStage; };
    if (wt * S::NT * 16 >= from.rows) {  // no rows of its own: only its share of the loads
        for (int32_t b = 0; b < loops; ++b) {
            wait_all<(S::kStages - 2) * S::kEach>();
#pragma unroll
            for (int i = 0; i < S::kEach; ++i)
                load(i, b + S::kStages - 1, lds + to_stage);
            to_stage = next_stage(to_stage);
        }
        __syncthreads();
        return;
    }
    // this lane's place in a piece of 16 lines: line lane % 16, 16-byte pieces 2 (lane / 16) and the next
    const int at = (lane & 15) * 128 + (((lane >> 4) * 2 ^ turn(lane & 15)) * 16);
    const int s_at = (lane & 15) * 8 + (lane >> 4) * 2;
    struct Piece {
        u4 code[2];
        uint32_t power;
    };
    auto fragment = [&](const unsigned char *lines_at, const unsigned char *scales_at, int piece) {
        const unsigned char *p = lines_at + piece * 16 * 128;
        return Piece{{*reinterpret_cast<const u4 *>(p + at), *reinterpret_cast<const u4 *>(p + (at ^ 16))},
                     *reinterpret_cast<const uint16_t *>(scales_at + piece * 16 * 8 + s_at)};
    };
    for (int32_t b = 0; b < loops; ++b) {
        wait_all<(S::kStages - 2) * S::kEach>();
        const unsigned char *buf = lds + at_stage;
        unsigned char *other = lds + to_stage;
        at_stage = next_stage(at_stage);
        to_stage = next_stage(to_stage);
        const unsigned char *wl = buf + wc * S::NC * 16 * 128, *xl = buf + (S::BC + wt * S::NT * 16) * 128;
        const unsigned char *wsl = buf + S::kLines * 128 + wc * S::NC * 16 * 8;
        const unsigned char *xsl = buf + S::kLines * 128 + S::kScaleW * 1024 + wt * S::NT * 16 * 8;
        Piece xf[S::NT];
        Piece wf = fragment(wl, wsl, 0);
#pragma unroll
        for (int t = 0; t < S::NT; ++t)
            xf[t] = fragment(xl, xsl, t);
        __builtin_amdgcn_sched_barrier(0);
        int id = 0, next = 0;
#pragma unroll
        for (int c = 0; c < S::NC; ++c) {
            const Piece w = wf;
            if (c + 1 < S::NC)
                wf = fragment(wl, wsl, c + 1);
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int t = 0; t < S::NT; ++t) {
                    acc[c][t] = half ? mfma4<1>(w.code[1], xf[t].code[1], acc[c][t], w.power, xf[t].power)
                                     : mfma4<0>(w.code[0], xf[t].code[0], acc[c][t], w.power, xf[t].power);
                    ++id;
                    if (next < S::kEach && id * S::kEach >= (next + 1) * S::kProducts * 3 / 4) {
                        __builtin_amdgcn_sched_barrier(0);
                        load(next++, b + S::kStages - 1, other);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
        }
#pragma unroll
        for (int i = 0; i < S::kEach; ++i)
            if (i >= next)
                load(i, b + S::kStages - 1, other);
    }
    __syncthreads();
#endif
}

}  // namespace spconv
