// The two product cores of 8-bit rows and weights (fp8.hpp): a tile of
// channels x rows staged through LDS, and a few rows against weights that are
// read once.  Both compute, for channels r (rows of W) and rows t of X,
//
//     sum over blocks b of  sx[b][t] * sw[r / 128][b] * (Wq[r] . Xq[t] over block b)
//
// One 8-bit matrix instruction spans exactly one block of 128 channels, so its result
// is a block's sum and is added to the 32-bit accumulator with one fused
// multiply-add by the block's scale (the exact form, fp8.hpp: four instructions
// of 32 channels).  W is the instruction's row operand: a
// lane then holds one row of X (one scale) and four neighbouring channels.
#pragma once

#include <atomic>

#include "fp8.hpp"

namespace spconv {

// Allows a kernel its LDS, once on each device (done: one bit for each).
template <typename F>
hipError_t allow_lds(F *kernel, int bytes, std::atomic<uint64_t> &done) {
    int device = 0;
    if (const hipError_t e = hipGetDevice(&device); e != hipSuccess)
        return e;
    const uint64_t bit = device < 64 ? uint64_t(1) << device : 0;
    if (done.load() & bit)
        return hipSuccess;
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == hipSuccess)
        done.fetch_or(bit);
    return e;
}

// ---------------------------------------------------------------------------
// Tile core.  BC channels x BT rows, WC x WT wavefronts, each NC x NT pieces of
// 16 x 16.  Per block of 128 channels, BC + BT lines of 128 bytes and BT scales
// go straight from global memory to LDS (16 bytes a lane, no registers between),
// STAGES - 1 blocks ahead of the products, into the buffer that the block before
// has left; a block begins with one barrier, after each wavefront has seen its
// own loads of that block arrive.
//
// A line's 16-byte pieces are stored in the order piece ^ (line / 2 % 8): 16
// lanes that read one piece of 16 neighbouring lines then touch each of LDS's
// 16-byte columns (256 bytes, two lines) once: no bank conflicts (counted).
// The permutation is done by the loads' global addresses, within a line, since
// their LDS places are fixed.
//
// Order of a block's instructions.  A load of 1 KiB to LDS takes about 17
// cycles of the compute unit's address path, and a wavefront that issues its
// loads in a row stands still for as long as all of them take (8 loads of 8
// wavefronts: 1080 cycles, a third of the block).  They are issued one after
// every second product instead, which also leaves them the rest of the block to
// arrive.  The multiply-adds of a piece follow one column of pieces later than
// its product, when the result is there.  The compiler would undo both (it
// gathers the loads and lets each multiply-add wait for its product), hence the
// scheduling barriers and the empty assembly that pins the sums.  8192 x 4096 ->
// 4096 over tiles of 256 x 256: 117 to 125 us (2.2 to 2.35 PFLOP/s; a large library
// product without block scales 94), in the compiler's order 143 to 167.  What bounds it
// are the products with their operands' reads from LDS (103 us alone; the matrix units
// work 44% of the time at 2.4 GHz), then the multiply-adds by the scales (10 us).
// ---------------------------------------------------------------------------
template <int BC_, int BT_, int WC_, int WT_, int STAGES_ = 2>
struct TileShape {
    static constexpr int BC = BC_, BT = BT_, WC = WC_, WT = WT_;
    static constexpr int kWaves = WC * WT, kThreads = 64 * kWaves;
    static constexpr int NC = BC / WC / 16, NT = BT / WT / 16;
    static constexpr int kLines = BC + BT;
    static constexpr int kLoads = kLines / 8 / kWaves;       // 8 lines an instruction
    static constexpr int kWeightLoads = BC / 8 / kWaves;     // the first of them: W's
    static constexpr int kStep = NC * NT >= 2 * kLoads ? 2 : 1;  // products from load to load
    static constexpr int kStages = STAGES_;
    static constexpr int kStage = kLines * kBlock + BT * 4;
    static constexpr int kLds = kStages * kStage;
    static_assert(BC % (8 * kWaves) == 0 && BT % (8 * kWaves) == 0 && BT % 64 == 0 && BT / 64 <= kWaves &&
                      NC * NT >= kLoads, "whole loads a wavefront");
};

using Rsrc = __amdgpu_buffer_rsrc_t;

__device__ __forceinline__ Rsrc make_rsrc(const void *p, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), static_cast<short>(0), static_cast<int>(bytes),
                                             0x00020000);
}

// The line (0 .. BC + BT - 1, W's first) and the byte in it that this lane
// copies with its i-th load.
template <class S>
__device__ __forceinline__ int tile_line(int wave, int lane, int i) {
    return (wave + i * S::kWaves) * 8 + (lane >> 3);
}
__device__ __forceinline__ int tile_byte(int line, int lane) { return ((lane & 7) ^ (line >> 1 & 7)) * 16; }

// What a tile reads: W and X from their bases, this lane's offsets of its lines
// (block 0); the rows' scales and this lane's offset there (wavefronts below
// BT / 64 only), step bytes from block to block.  Bytes: what each base covers;
// an offset of that size reads zeros.  rows: how many of the tile's rows there are.
template <class S>
struct TileSource {
    const uint8_t *w, *x;
    const float *xs;
    uint32_t w_bytes, x_bytes, xs_bytes, xs_step;
    uint32_t at[S::kLoads], xs_at;
    int32_t rows;
};

// A wavefront's channel and row pieces.  Wavefronts w and w + 4 share a SIMD:
// in this order a tile that is half empty leaves work on all four.
template <class S>
__device__ __forceinline__ int channel_part(int wave) { return wave % S::WC; }
template <class S>
__device__ __forceinline__ int row_part(int wave) { return wave / S::WC; }

// A scalar load: of an address that is the same in all lanes, of what no kernel
// in flight writes.
template <typename T>
__device__ __forceinline__ T uniform_load(const T *p) {
    return *reinterpret_cast<const __attribute__((address_space(4))) T *>(reinterpret_cast<uintptr_t>(p));
}

// Waits until all but the last N of this wavefront's loads have arrived and all
// its reads of LDS are done, then for the workgroup's other wavefronts.
template <int N>
__device__ __forceinline__ void wait_all() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// acc[c][t] += the products over kb blocks; ws0, ws1: the scales by block of
// the first and of the second half (HALVES) of the wavefront's channel pieces;
// total[t] += the scales' products without their signs, whose sum times 128 * 448^2 no result exceeds.
// loops: kb, or more where other wavefronts of the workgroup, which it meets
// block by block, have more blocks; those past kb are zeros.
template <class S, bool EXACT, bool HALVES>
__device__ __forceinline__ void tile_product(f4 (&acc)[S::NC][S::NT], float (&total)[S::NT],
                                             const TileSource<S> &from, const float *ws0, const float *ws1, int32_t kb,
                                             int32_t loops, unsigned char *lds, int wave, int lane) {
#ifdef __HIP_DEVICE_COMPILE__  // the host's pass knows no buffer resources
    const int wc = channel_part<S>(wave), wt = row_part<S>(wave);
    // Every wavefront issues the same number of loads a block, so that it can
    // count them: kLoads of lines, one of scales (the first BT / 64 wavefronts',
    // by the others again).  Past the last block they are out of their range and
    // read nothing.
    constexpr int kEach = S::kLoads + 1;
    auto load = [&](int i, int32_t b, unsigned char *buf) {
        if (i < S::kLoads) {
            const bool of_w = i < S::kWeightLoads;
            const uint32_t bytes = of_w ? from.w_bytes : from.x_bytes;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                make_rsrc(of_w ? from.w : from.x, b < kb ? bytes : 0),
                (__attribute__((address_space(3))) void *)(buf + (wave + i * S::kWaves) * 1024), 16, from.at[i],
                b * kBlock, 0, 0);
        } else {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                make_rsrc(from.xs, b < kb ? from.xs_bytes : 0),
                (__attribute__((address_space(3))) void *)(buf + S::kLines * kBlock + wave % (S::BT / 64) * 256), 4,
                from.xs_at, b * from.xs_step, 0, 0);
        }
    };
#pragma unroll
    for (int st = 0; st < S::kStages - 1; ++st)
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            load(i, st, lds + st * S::kStage);
    int32_t at_stage = 0, to_stage = (S::kStages - 1) * S::kStage;
    auto next_stage = [](int32_t at) { return at == (S::kStages - 1) * S::kStage ? 0 : at + S::kStage; };
    if (wt * S::NT * 16 >= from.rows) {  // no rows of its own: only its share of the loads
        for (int32_t b = 0; b < loops; ++b) {
            wait_all<(S::kStages - 2) * kEach>();
#pragma unroll
            for (int i = 0; i < kEach; ++i)
                load(i, b + S::kStages - 1, lds + to_stage);
            to_stage = next_stage(to_stage);
        }
        __syncthreads();
        return;
    }
    // this lane's place in a piece of 16 lines: line lane % 16, 16-byte piece lane / 16 (and 4 further)
    const int at = (lane & 15) * kBlock + (((lane >> 4) ^ ((lane & 15) >> 1)) * 16);
    auto fragment = [&](const unsigned char *p) {
        return join(*reinterpret_cast<const u4 *>(p + at), *reinterpret_cast<const u4 *>(p + (at ^ 64)));
    };
    const int32_t last = max(kb, 1) - 1;
    float sw0 = uniform_load(ws0), sw1 = HALVES ? uniform_load(ws1) : 0.0f;
    for (int32_t b = 0; b < loops; ++b) {
        wait_all<(S::kStages - 2) * kEach>();
        const unsigned char *buf = lds + at_stage;
        unsigned char *other = lds + to_stage;
        at_stage = next_stage(at_stage);
        to_stage = next_stage(to_stage);
        const unsigned char *wl = buf + wc * S::NC * 16 * kBlock;
        const unsigned char *xl = buf + (S::BC + wt * S::NT * 16) * kBlock;
        const float *sl = reinterpret_cast<const float *>(buf + S::kLines * kBlock) + wt * S::NT * 16 + (lane & 15);
        i8 code = fragment(wl);
        decltype(operand<EXACT>(i8{})) xf[S::NT];
        float s0[S::NT], s1[S::NT];
#pragma unroll
        for (int t = 0; t < S::NT; ++t)
            xf[t] = operand<EXACT>(fragment(xl + t * 16 * kBlock));
#pragma unroll
        for (int t = 0; t < S::NT; ++t)
            s0[t] = sl[t * 16];
        __builtin_amdgcn_sched_barrier(0);
        f4 p[2][S::NT];
        auto add = [&](int c, int t) {
            const float s = HALVES && c >= S::NC / 2 ? s1[t] : s0[t];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                acc[c][t][i] = fmaf(s, p[c & 1][t][i], acc[c][t][i]);
            asm volatile("" : "+v"(acc[c][t]));
        };
#pragma unroll
        for (int c = 0; c < S::NC; ++c) {
            const auto wf = operand<EXACT>(code);
            if (c + 1 < S::NC)
                code = fragment(wl + (c + 1) * 16 * kBlock);
#pragma unroll
            for (int t = 0; t < S::NT; ++t) {
                p[c & 1][t] = mfma128(wf, xf[t]);
                if (c == 0) {
                    s1[t] = HALVES ? s0[t] * sw1 : 0.0f;
                    s0[t] *= sw0;
                    total[t] += fabsf(s0[t]);
                }
                __builtin_amdgcn_sched_barrier(0);
                const int id = c * S::NT + t;
#pragma unroll
                for (int i = 0; i < kEach; ++i)
                    if (id == min(i * S::kStep + S::kStep - 1, S::NC * S::NT - 1))
                        load(i, b + S::kStages - 1, other);
                __builtin_amdgcn_sched_barrier(0);
                if (c > 0)
                    add(c - 1, t);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
#pragma unroll
        for (int t = 0; t < S::NT; ++t)
            add(S::NC - 1, t);
        // the next block's scales: asked for here, so that no later wait for operands in LDS is one for them
        sw0 = uniform_load(ws0 + min(b + 1, last));
        sw1 = HALVES ? uniform_load(ws1 + min(b + 1, last)) : 0.0f;
    }
    __syncthreads();
#endif
}

// A wavefront's results to rows of y: `row` is y's first row of the tile, `rows`
// how many it has, ch this lane's first channel of piece 0, `channels` y's row.
// `finish(v, c, t)` gives what is stored for piece (c, t).
template <class S, int TYPE, class F>
__device__ __forceinline__ void store_whole(const f4 (&acc)[S::NC][S::NT], void *y, int64_t row, int32_t rows, int32_t ch,
                                            int32_t channels, int wt, int lane, F finish) {
    constexpr int kSize = TYPE == kF32 ? 4 : 2;
#pragma unroll
    for (int t = 0; t < S::NT; ++t) {
        const int r = (wt * S::NT + t) * 16 + (lane & 15);
        if (r >= rows)
            continue;
        char *p = static_cast<char *>(y) + ((row + r) * channels + ch) * kSize;
#pragma unroll
        for (int c = 0; c < S::NC; ++c) {
            const f4 v = finish(acc[c][t], c, t);
            if constexpr (TYPE == kF32)
                *reinterpret_cast<f4 *>(p + c * 16 * kSize) = v;
            else
                *reinterpret_cast<u2 *>(p + c * 16 * kSize) = rounded4<TYPE>(v);
        }
    }
}

// The same for 16-bit results and rows of whole 16-byte pieces: through the
// wavefront's own part of LDS, from where each store writes whole 128-byte
// lines (straight from the registers it writes 32 bytes of each of 16 rows;
// 134 MB of results: 133 us against 111 us in all for 32768 x 1024 -> 2048 among
// other work; alone it takes 79, 13 of them for the stores).
// Piece p of row r lies at p ^ r % pieces: rows start on the same bank.
template <class S, int TYPE, class F>
__device__ __forceinline__ void store_lines(const f4 (&acc)[S::NC][S::NT], void *y, int64_t row, int32_t rows, int32_t ch,
                                            int32_t channels, int wave, int lane, unsigned char *lds, F finish) {
    constexpr int kRow = S::NC * 32, kPieces = kRow / 16;
    static_assert(S::kWaves * S::NT * 16 * kRow <= S::kLds, "the results fit where the operands were");
    const int wt = row_part<S>(wave);
    unsigned char *own = lds + wave * S::NT * 16 * kRow;
#pragma unroll
    for (int t = 0; t < S::NT; ++t)
#pragma unroll
        for (int c = 0; c < S::NC; ++c) {
            const int r = t * 16 + (lane & 15), piece = c * 2 + (lane >> 5);
            *reinterpret_cast<u2 *>(own + r * kRow + (piece ^ (r & (kPieces - 1))) * 16 + (lane >> 4 & 1) * 8) =
                rounded4<TYPE>(finish(acc[c][t], c, t));
        }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const int piece = lane % kPieces;
    uint16_t *to = static_cast<uint16_t *>(y) + row * channels + ch - (lane >> 4) * 4 + piece * 8;
#pragma unroll
    for (int i = 0; i < S::NT * 16 * kRow / 1024; ++i) {
        const int r = i * (64 / kPieces) + lane / kPieces;
        if (wt * S::NT * 16 + r < rows)
            *reinterpret_cast<u4 *>(to + static_cast<int64_t>(wt * S::NT * 16 + r) * channels) =
                *reinterpret_cast<const u4 *>(own + r * kRow + (piece ^ (r & (kPieces - 1))) * 16);
    }
}

// The same for any channels and alignment; `wide`: four neighbours may be stored at once.
template <class S, class F>
__device__ __forceinline__ void store_tile(const f4 (&acc)[S::NC][S::NT], void *y, int32_t type, int64_t row, int32_t rows,
                                           int32_t ch, int32_t channels, bool wide, int wave, int lane,
                                           unsigned char *lds, F finish) {
    const int wt = row_part<S>(wave);
    const bool whole = wide && ch - (lane >> 4) * 4 + S::NC * 16 <= channels;
    if (whole && channels % 8 == 0 && type != kF32) {
        if (type == kF16)
            store_lines<S, kF16>(acc, y, row, rows, ch, channels, wave, lane, lds, finish);
        else
            store_lines<S, kBf16>(acc, y, row, rows, ch, channels, wave, lane, lds, finish);
        return;
    }
    if (whole) {
        if (type == kF32)
            store_whole<S, kF32>(acc, y, row, rows, ch, channels, wt, lane, finish);
        else if (type == kF16)
            store_whole<S, kF16>(acc, y, row, rows, ch, channels, wt, lane, finish);
        else
            store_whole<S, kBf16>(acc, y, row, rows, ch, channels, wt, lane, finish);
        return;
    }
#pragma unroll
    for (int t = 0; t < S::NT; ++t) {
        const int r = (wt * S::NT + t) * 16 + (lane & 15);
#pragma unroll
        for (int c = 0; c < S::NC; ++c)
            if (r < rows && ch + c * 16 < channels)
                store4(y, type, (row + r) * channels + ch + c * 16, finish(acc[c][t], c, t), channels - ch - c * 16, wide);
    }
}

// ---------------------------------------------------------------------------
// Stream core: up to 16 TT rows against CT pieces of 16 channels, the blocks
// of the input channels dealt to the wavefronts of a workgroup in turn.
// Nothing is shared between wavefronts but the final sum, so operands go from
// global memory (rows: from L2) to registers in the instruction's layout.  What
// bounds it is a chain of a few loads and the bytes of weight and rows, so the
// products are the exact ones (1 x 1024 -> 1024: 3.1 us, 1 x 4096 -> 4096: 6.2 us,
// 2.7 TB/s).
// ---------------------------------------------------------------------------

// A lane's part (32 of 128 channels) of one row and block, and the block's scale.
struct RowPart {
    i8 code;
    float scale;
};

// Rows kept as codes.
__device__ __forceinline__ RowPart row_codes(const uint8_t *row, const float *scale, int32_t b, int lane) {
    const uint8_t *p = row + static_cast<int64_t>(b) * kBlock + (lane >> 4) * 16;
    return {join(*reinterpret_cast<const u4 *>(p), *reinterpret_cast<const u4 *>(p + 64)), *scale};
}

// Rows in f32, f16 or bf16, quantised here: the four lanes of a row hold the
// whole block between them.
template <typename T>
__device__ __forceinline__ RowPart row_quantized(const T *row, int32_t b, int32_t cols, bool wide, int lane) {
    const int32_t c = b * kBlock + (lane >> 4) * 16;
    float v[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int32_t at = c + (i >> 1) * 64 + (i & 1) * 8;
        load8_tail(row + at, cols - at, wide, v[i]);
    }
    uint32_t m = max(max(most8(v[0]), most8(v[1])), max(most8(v[2]), most8(v[3])));
    m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 16)));
    m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 32)));
    const Scale s = scale_of(m);
    i8 code;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        code[2 * i] = static_cast<int>(codes4(v[i], s.inv));
        code[2 * i + 1] = static_cast<int>(codes4(v[i] + 4, s.inv));
    }
    return {code, s.scale};
}

// A lane's part of one piece of 16 weight rows and block b; `row`: its row.
__device__ __forceinline__ i8 weight_part(const uint8_t *row, int32_t b, int lane) {
    const uint8_t *p = row + static_cast<int64_t>(b) * kBlock + (lane >> 4) * 16;
    return join(__builtin_nontemporal_load(reinterpret_cast<const u4 *>(p)),
                __builtin_nontemporal_load(reinterpret_cast<const u4 *>(p + 64)));
}

// Sum of every wavefront's accumulators, in the order of the wavefronts; the
// sum of piece i is returned to wavefront i % waves and visited with `then(i, sum)`.
// lds: waves * PIECES KiB.
template <int PIECES, class F>
__device__ __forceinline__ void sum_waves(const f4 *acc, f4 *lds, int waves, int wave, int lane, F then) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
        lds[(wave * PIECES + i) * 64 + lane] = acc[i];
    __syncthreads();
    for (int i = wave; i < PIECES; i += waves) {
        f4 sum = lds[i * 64 + lane];
        for (int w = 1; w < waves; ++w)
            sum += lds[(w * PIECES + i) * 64 + lane];
        then(i, sum);
    }
}

}  // namespace spconv
