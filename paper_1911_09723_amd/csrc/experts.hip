// The gated feed-forward networks of the experts that a router chose:
//
//   y[t] = sum_j weight[t][j] * W2_e q( silu(W1_e q(x_t)) * (W3_e q(x_t)) ),  e = ids[t][j]
//
// in 8 bits with block scales (fp8.hpp; q quantises by row).  A pair (token,
// choice) is one row of work.
#include <algorithm>

#include "expert_ops.hpp"
#include "fp8_product.hpp"

namespace spconv {
namespace {

constexpr int kXcds = 8;

// pair / k, for pairs below 2^25 and k up to 64.
__device__ __forceinline__ int32_t token_of(const ExpertArgs &a, int32_t pair) {
    return static_cast<int32_t>(static_cast<uint64_t>(pair) * a.k_inverse >> 31);
}

// block / ib, for the at most 384 blocks of a token's inner rows and those up to 32 past them.
__device__ __forceinline__ int32_t choice_of(const ExpertArgs &a, int32_t block) {
    return static_cast<int32_t>(static_cast<uint64_t>(block) * a.ib_inverse >> 31);
}

// Pairs (token, choice) sorted by expert: workgroup e finds the places of expert
// e's pairs.  It counts, over all pairs, those of lower experts (its first place)
// and its own, then hands out its places in the order of the pairs; no workgroup
// waits for another, and no place depends on timing.  A wavefront walks its
// share of the pairs 256 at a time, four neighbours a lane; the first kKept
// pieces stay in registers for the second walk.
__device__ __forceinline__ void sort_pairs(const ExpertArgs &a, int32_t e, bool wide) {
    __shared__ int32_t part[2][16];
    constexpr int kKept = 8;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int32_t pieces = (a.pairs + 255) / 256, per = (pieces + waves - 1) / waves;
    const int32_t first = min(wave * per, pieces), last = min(first + per, pieces);
    // four ids from pair 4 lane of a piece; past the end: none
    auto load = [&](int32_t piece) {
        const int32_t i = piece * 256 + lane * 4;
        if (wide && i + 4 <= a.pairs)
            return *reinterpret_cast<const i4 *>(a.ids + i);
        i4 v;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            v[j] = i + j < a.pairs ? a.ids[i + j] : -1;
        return v;
    };
    int32_t below = 0, own = 0;
    auto count = [&](i4 v) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            below += static_cast<uint32_t>(v[j]) < static_cast<uint32_t>(e);
            own += v[j] == e;
        }
    };
    i4 kept[kKept];
#pragma unroll
    for (int i = 0; i < kKept; ++i)
        kept[i] = first + i < last ? load(first + i) : i4{-1, -1, -1, -1};
#pragma unroll
    for (int i = 0; i < kKept; ++i)
        count(kept[i]);
#pragma unroll 4
    for (int32_t p = first + kKept; p < last; ++p)
        count(load(p));
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
        own += __shfl_xor(own, s);
        below += __shfl_xor(below, s);
    }
    if (lane == 0) {
        part[0][wave] = own;
        part[1][wave] = below;
    }
    __syncthreads();
    const int32_t owns = lane < waves ? part[0][lane] : 0;
    int32_t start = lane < waves ? part[1][lane] : 0, total = start + owns;
    start += lane < wave ? owns : 0;
#pragma unroll
    for (int s = 1; s < 16; s *= 2) {
        start += __shfl_xor(start, s);
        total += __shfl_xor(total, s);
    }
    int32_t at = __builtin_amdgcn_readfirstlane(start);
    if (threadIdx.x == 0) {
        a.offsets[e + 1] = total;
        if (e == 0)
            a.offsets[0] = 0;
    }
    auto give = [&](int32_t p, i4 v) {
        const int32_t i = p * 256 + lane * 4;
        int32_t before = at;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint64_t mine = __ballot(v[j] == e);
            before += __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(mine >> 32),
                                                __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(mine), 0));
            at += __popcll(mine);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (v[j] == e) {
                a.order[before] = token_of(a, i + j);
                a.place[i + j] = before++;
            } else if (e == 0 && i + j < a.pairs && static_cast<uint32_t>(v[j]) >= static_cast<uint32_t>(a.experts)) {
                a.place[i + j] = -1;
            }
        }
    };
#pragma unroll
    for (int i = 0; i < kKept; ++i)
        if (first + i < last)
            give(first + i, kept[i]);
    for (int32_t p = first + kKept; p < last; ++p)
        give(p, load(p));
}

// The sort and x's rows to codes, which do not need each other, in one launch:
// workgroups below a.experts sort.  4096 tokens of 2048 channels and 8 of 64
// experts: 13.4 us, of it the sort, a chain of two walks over 128 KB of ids; the
// rows alone would take 6.
template <typename T, int U>
__global__ void __launch_bounds__(1024) prepare_rows(ExpertArgs a, int32_t row_groups, bool wide_ids, bool wide) {
    if (static_cast<int32_t>(blockIdx.x) < a.experts) {
        sort_pairs(a, blockIdx.x, wide_ids);
        return;
    }
    const int32_t id = static_cast<int32_t>(blockIdx.x) - a.experts, part = id / row_groups;
    quantize_group<T, U>(static_cast<const T *>(a.x), a.ldx, a.n, a.hidden, a.xq, a.xs, a.hb, id - part * row_groups, part,
                         wide);
}

// g / (1 + exp(-g)) * u.  exp2 and the reciprocal are one last place off each;
// g log2(e) is taken to twice 32 bits so that the exponential stays there.
__device__ __forceinline__ float gated(float g, float u) {
    const float t = g * -1.44269504f, rest = fmaf(g, -1.44269504f, -t) + g * -1.92596299e-8f;
    const float e = __builtin_amdgcn_exp2f(t);
    const float exact = fabsf(t) < 128.0f ? fmaf(e, rest * 0.693147181f, e) : e;  // else 0 or infinite
    return g * __builtin_amdgcn_rcpf(1.0f + exact) * u;
}

// The power of two that v is 2^14 to 2^15 of, and its inverse (v at least 2^-112).
struct Power {
    float value, inverse;
};
__device__ __forceinline__ Power power_below(float v) {
    const uint32_t e = max(__float_as_uint(v) >> 23, 15u);
    return {__uint_as_float((e - 14) << 23), __uint_as_float((268 - e) << 23)};
}

// One tile of rows of one expert, places [row, row + rows).
struct RowTile {
    int32_t expert, row, rows;
};

// This workgroup's tile of all (tiles of `high` rows, `wide` column tiles each),
// in the order that gives each XCD one run of neighbouring tiles: tiles of one
// expert share its weights, and column tiles the rows, in an L2.  False past the
// last one.  Lanes take experts 64 at a time; what leaves is the same in all of
// them and is kept in scalar registers (readfirstlane, readlane), where the
// tile's buffer resources have to be: a resource that the compiler takes to
// differ between lanes costs a loop around every load.
__device__ __forceinline__ bool find_tile(const int32_t *offsets, int32_t experts, int32_t high, int32_t wide,
                                          int lane, RowTile *tile, int32_t *column) {
    auto tiles_of = [&](int32_t e) {
        return e < experts ? (offsets[e + 1] - offsets[e] + high - 1) / high : 0;
    };
    int32_t sum = 0;
    for (int32_t e0 = 0; e0 < experts; e0 += 64)
        sum += tiles_of(e0 + lane);
#pragma unroll
    for (int s = 1; s < 64; s *= 2)
        sum += __shfl_xor(sum, s);
    const int32_t total = __builtin_amdgcn_readfirstlane(sum) * wide;
    const int32_t per = (total + kXcds - 1) / kXcds;
    const int32_t in = blockIdx.x / kXcds, id = blockIdx.x % kXcds * per + in;
    if (in >= per || id >= total)
        return false;
    int32_t want = id / wide;
    *column = id - want * wide;
    for (int32_t e0 = 0; e0 < experts; e0 += 64) {
        const int32_t own = tiles_of(e0 + lane);
        int32_t upto = own;
#pragma unroll
        for (int s = 1; s < 64; s *= 2) {
            const int32_t o = __shfl_up(upto, s);
            upto += lane >= s ? o : 0;
        }
        const uint64_t past = __ballot(upto > want);
        if (past) {
            const int at = __ffsll(static_cast<unsigned long long>(past)) - 1;
            const int32_t before = __builtin_amdgcn_readlane(upto - own, at);
            tile->expert = e0 + at;
            tile->row = uniform_load(offsets + tile->expert) + (want - before) * high;
            tile->rows = min(high, uniform_load(offsets + tile->expert + 1) - tile->row);
            return true;
        }
        want -= __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

// First products over LDS tiles: 128 inner channels, gate and up, of a tile of
// rows, which are x's rows (codes) by token; the result leaves as codes.  A
// wavefront holds 64 gate and the same 64 up channels, so that the gate is
// applied in its registers; the block's largest magnitude is joined over the
// two wavefronts that share its rows.  32768 pairs of 64 experts, 2048 -> 2 x
// 1024: 326 us, 0.84 PFLOP/s.  Bound by issue: the conversions of codes and the
// gate take the vector units 48% of the time, the products, at half the 8-bit
// rate, the matrix units 34%; 634 MB read, 2.05 TB/s.  200 pairs of 32 experts,
// 1280 -> 2 x 960: 17 us, the weights at 4.6 TB/s.
template <class S>
__global__ void __launch_bounds__(S::kThreads) gated_tile(ExpertArgs a, int32_t columns) {
    static_assert(S::BC == 256 && S::WC == 2, "a wavefront holds half a block of gate and of up channels");
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    RowTile tile;
    int32_t fb;
    if (!find_tile(a.offsets, a.experts, S::BT, columns, lane, &tile, &fb))
        return;
    const uint32_t pitch = a.hb * kBlock;
    const float *ws = a.s13 + static_cast<int64_t>(tile.expert) * 2 * a.ib * a.hb + static_cast<int64_t>(fb) * a.hb;
    TileSource<S> from;
    from.w = a.w13 + static_cast<int64_t>(tile.expert) * 2 * a.inner * pitch;
    from.w_bytes = 2 * a.inner * pitch;
    from.x = a.xq;
    from.x_bytes = a.n * pitch;
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) {
        const int line = tile_line<S>(wave, lane, i);
        if (i < S::kWeightLoads) {  // lines of a wavefront: 64 gate, then 64 up channels
            const int32_t ch = fb * kBlock + line / 128 * 64 + line % 64;
            const uint32_t at = (ch + (line & 64 ? a.inner : 0)) * pitch + tile_byte(line, lane);
            from.at[i] = ch < a.inner ? at : from.w_bytes;
        } else {
            const int r = line - S::BC;
            const uint32_t at = a.order[tile.row + min(r, tile.rows - 1)] * pitch + tile_byte(line, lane);
            from.at[i] = r < tile.rows ? at : from.x_bytes;
        }
    }
    from.rows = tile.rows;
    from.xs = a.xs;
    from.xs_at = a.order[tile.row + min(wave % (S::BT / 64) * 64 + lane, tile.rows - 1)] * 4u;
    from.xs_step = a.n * 4u;
    from.xs_bytes = from.xs_step * a.hb;
    f4 acc[S::NC][S::NT] = {};
    float total[S::NT] = {};
    tile_product<S, true, true>(acc, total, from, ws, ws + static_cast<int64_t>(a.ib) * a.hb, a.hb, a.hb, lds, wave, lane);

    const int wc = channel_part<S>(wave), wt = row_part<S>(wave);
    float *most = reinterpret_cast<float *>(lds + S::BT * kBlock);  // [2][BT]
    constexpr int HC = S::NC / 2;
    const bool idle = wt * S::NT * 16 >= tile.rows;
    uint32_t m[S::NT];
    if (!idle) {
#pragma unroll
        for (int t = 0; t < S::NT; ++t) {
            m[t] = 0;
#pragma unroll
            for (int c = 0; c < HC; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float h = gated(acc[c][t][i], acc[c + HC][t][i]);  // channels past the last: 0
                    acc[c][t][i] = h;
                    m[t] = max(m[t], magnitude(h));
                }
            m[t] = max(m[t], static_cast<uint32_t>(__shfl_xor(static_cast<int>(m[t]), 16)));
            m[t] = max(m[t], static_cast<uint32_t>(__shfl_xor(static_cast<int>(m[t]), 32)));
            if (lane < 16)
                most[wc * S::BT + (wt * S::NT + t) * 16 + lane] = __uint_as_float(m[t]);
        }
    }
    __syncthreads();
    if (!idle) {
#pragma unroll
        for (int t = 0; t < S::NT; ++t) {
            const int r = (wt * S::NT + t) * 16 + (lane & 15);
            const Scale s = scale_of(max(m[t], __float_as_uint(most[(1 - wc) * S::BT + r])));
#pragma unroll
            for (int c = 0; c < HC; ++c) {
                const float v[4] = {acc[c][t][0], acc[c][t][1], acc[c][t][2], acc[c][t][3]};
                const int word = (wc * 16 + c * 4 + (lane >> 4)) ^ (r & 7) * 4;  // spread over LDS's banks
                reinterpret_cast<uint32_t *>(lds)[r * 32 + word] = codes4(v, s.inv);
            }
            if (wc == 0 && lane < 16 && r < tile.rows)
                a.hs[static_cast<int64_t>(fb) * a.pairs + tile.row + r] = s.scale;
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < S::BT * 8; i += S::kThreads) {
        const int r = i >> 3, piece = i & 7;
        if (r < tile.rows)
            *reinterpret_cast<u4 *>(a.hq + (static_cast<int64_t>(tile.row + r) * a.ib + fb) * kBlock + piece * 16) =
                *reinterpret_cast<const u4 *>(lds + r * kBlock + ((piece ^ (r & 7)) * 16));
    }
}

// Second products over LDS tiles: rows by place, results by place, in 32 bits
// or (HALF) in f16 with a scale for each 128 channels of a row.  The results are
// written once and read once by the weighted sum: at 4096 tokens of 8 experts
// and 2048 channels 537 MB in 32 bits, more than the products' operands.  An
// f16 value is 2^-11 off at most, an eighth of the rounding (2^-8) of a bf16
// result to come.  The scale is the power of two that brings the most that the row's and
// the weight's scales allow just below 2^15, so nothing overflows, and as the
// sum of random codes stays some 2^10 below that most, what is lost to f16's
// small numbers is 2^-30 of a usual value.  32768 pairs, 1024 -> 2048: 104 us, 1.32
// PFLOP/s, with 364 MB read and written (3.5 TB/s).
template <class S, bool EXACT, bool HALF>
__global__ void __launch_bounds__(S::kThreads) down_tile(ExpertArgs a, int32_t columns) {
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    RowTile tile;
    int32_t ct;
    if (!find_tile(a.offsets, a.experts, S::BT, columns, lane, &tile, &ct))
        return;
    const int32_t c0 = ct * S::BC;
    const uint32_t pitch = a.ib * kBlock;
    TileSource<S> from;
    from.w = a.w2 + (static_cast<int64_t>(tile.expert) * a.hidden + c0) * pitch;
    from.w_bytes = min(S::BC, a.hidden - c0) * pitch;
    from.x = a.hq + static_cast<int64_t>(tile.row) * pitch;
    from.x_bytes = tile.rows * pitch;
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) {
        const int line = tile_line<S>(wave, lane, i);
        if (i < S::kWeightLoads)
            from.at[i] = line < a.hidden - c0 ? line * pitch + tile_byte(line, lane) : from.w_bytes;
        else
            from.at[i] = line - S::BC < tile.rows ? (line - S::BC) * pitch + tile_byte(line, lane) : from.x_bytes;
    }
    from.rows = tile.rows;
    from.xs = a.hs + tile.row;
    from.xs_at = min(wave % (S::BT / 64) * 64 + lane, tile.rows - 1) * 4u;
    from.xs_step = a.pairs * 4u;
    from.xs_bytes = from.xs_step * (a.ib - 1) + tile.rows * 4u;
    const int wc = channel_part<S>(wave), wt = row_part<S>(wave);
    const int32_t cw = c0 + wc * S::NC * 16;
    const float *ws = a.s2 + (static_cast<int64_t>(tile.expert) * a.hb + min(cw, a.hidden - 1) / kBlock) * a.ib;
    f4 acc[S::NC][S::NT] = {};
    float total[S::NT] = {};
    tile_product<S, EXACT, false>(acc, total, from, ws, nullptr, a.ib, a.ib, lds, wave, lane);
    const int32_t ch = cw + (lane >> 4) * 4;
    float inverse[S::NT];
    if constexpr (HALF) {
        static_assert(S::NC * 16 == kBlock, "a wavefront's channels are one block");
#pragma unroll
        for (int t = 0; t < S::NT; ++t) {
            const int r = (wt * S::NT + t) * 16 + (lane & 15);
            const Power p = power_below(total[t] * (kTop * kTop * kBlock));
            inverse[t] = p.inverse;
            if (lane < 16 && r < tile.rows && cw < a.hidden)
                a.zs[static_cast<int64_t>(tile.row + r) * a.hb + cw / kBlock] = p.value;
        }
    }
    store_tile<S>(acc, a.z, HALF ? kF16 : kF32, tile.row, tile.rows, ch, a.hidden, a.hidden % 4 == 0, wave, lane, lds,
                  [&](f4 v, int, int t) { return HALF ? v * inverse[t] : v; });
}

// Single tokens.  What bounds them is the weights' bytes, and a compute unit takes
// in no more than its share of the card's rate (some 20 GB/s: what it can have
// outstanding, over the memory's latency), so the weights are spread evenly over
// all of them: workgroups of 8 channels.  (Workgroups of 128 channels, which
// could convert the inner rows to codes themselves, took 24 instead of 10 us for
// the first products of 6 x 4 MB.)  One row of x has no use for matrix
// instructions, and rows of W are read in whole lines: a lane takes 16 of 1024
// neighbouring channels, 8 lanes a block.  Sort and weighted sum fall away.
// One token, 6 experts of 2048 x 1024: 7.2 and 8.6 us for 25 and 13 MB.

// The sum of 16 products of codes.
__device__ __forceinline__ float dot16(const float *x, u4 w) {
    float even = 0.0f, odd = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w[i]), false);
        const f2 hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w[i]), true);
        even = fmaf(x[4 * i], lo[0], even);
        odd = fmaf(x[4 * i + 1], lo[1], odd);
        even = fmaf(x[4 * i + 2], hi[0], even);
        odd = fmaf(x[4 * i + 3], hi[1], odd);
    }
    return even + odd;
}

__device__ __forceinline__ void code_values(u4 c, float *v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(c[i]), false);
        const f2 hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(c[i]), true);
        v[4 * i] = lo[0];
        v[4 * i + 1] = lo[1];
        v[4 * i + 2] = hi[0];
        v[4 * i + 3] = hi[1];
    }
}

__device__ __forceinline__ float sum_lanes(float v) {
#pragma unroll
    for (int s = 1; s < 64; s *= 2)
        v += __shfl_xor(v, s);
    return v;
}

__device__ __forceinline__ u4 stream16(const uint8_t *p) { return __builtin_nontemporal_load(reinterpret_cast<const u4 *>(p)); }

constexpr int kTokenChannels = 2;  // gate and up channels of a wavefront

// First products of pair blockIdx.y; x is quantised here.
template <typename T>
__global__ void __launch_bounds__(256) gated_token(ExpertArgs a, bool wide) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t pair = blockIdx.y, c0 = (static_cast<int32_t>(blockIdx.x) * 4 + wave) * kTokenChannels;
    if (c0 >= a.inner)
        return;
    const int32_t pitch = a.hb * kBlock;
    const T *x = static_cast<const T *>(a.x) + token_of(a, pair) * a.ldx;
    constexpr int U = 2;
    float v[U][16];
    auto load_x = [&](int32_t k0) {
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int32_t k = k0 + j * 1024;
            load8_tail(x + k, k < pitch ? a.hidden - k : 0, wide, v[j]);
            load8_tail(x + k + 8, k < pitch ? a.hidden - k - 8 : 0, wide, v[j] + 8);
        }
    };
    load_x(lane * 16);  // asked for before the id, which the weights' addresses wait for
    const int32_t id = a.ids[pair];
    const bool some = id >= 0 && id < a.experts;  // else any expert's weights, and zeros
    const int64_t e = some ? id : 0;
    const uint8_t *row[2 * kTokenChannels];
#pragma unroll
    for (int i = 0; i < kTokenChannels; ++i) {
        row[i] = a.w13 + (e * 2 * a.inner + min(c0 + i, a.inner - 1)) * pitch;
        row[i + kTokenChannels] = row[i] + static_cast<int64_t>(a.inner) * pitch;
    }
    const float *sg = a.s13 + (e * 2 * a.ib + c0 / kBlock) * a.hb;
    const float *su = sg + static_cast<int64_t>(a.ib) * a.hb;
    float acc[2 * kTokenChannels] = {};
    for (int32_t k0 = lane * 16;;) {
        u4 w[U][2 * kTokenChannels];
        float g[U], u[U];
        // a lane past the last channel repeats the last block's, times 0
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int32_t k = min(k0 + j * 1024, pitch - 16);
#pragma unroll
            for (int i = 0; i < 2 * kTokenChannels; ++i)
                w[j][i] = stream16(row[i] + k);
            const bool there = k0 + j * 1024 < pitch;
            g[j] = there ? sg[k / kBlock] : 0.0f;
            u[j] = there ? su[k / kBlock] : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < U; ++j) {
            uint32_t m = max(most8(v[j]), most8(v[j] + 8));
#pragma unroll
            for (int s = 1; s < 8; s *= 2)
                m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), s)));
            const Scale s = scale_of(m);
            const u4 c = {codes4(v[j], s.inv), codes4(v[j] + 4, s.inv), codes4(v[j] + 8, s.inv), codes4(v[j] + 12, s.inv)};
            code_values(c, v[j]);
#pragma unroll
            for (int i = 0; i < kTokenChannels; ++i) {
                acc[i] = fmaf(dot16(v[j], w[j][i]), s.scale * g[j], acc[i]);
                acc[i + kTokenChannels] = fmaf(dot16(v[j], w[j][i + kTokenChannels]), s.scale * u[j], acc[i + kTokenChannels]);
            }
        }
        k0 += U * 1024;
        if (k0 - lane * 16 >= pitch)
            break;
        load_x(k0);
    }
#pragma unroll
    for (int i = 0; i < kTokenChannels; ++i) {
        const float h = gated(sum_lanes(acc[i]), sum_lanes(acc[i + kTokenChannels]));
        if (lane == 0 && c0 + i < a.inner)
            a.h[static_cast<int64_t>(pair) * a.inner + c0 + i] = some ? h : 0.0f;
    }
}

// Second products and weighted sum of token blockIdx.y, a channel a wavefront.
// The workgroup quantises the token's inner rows into LDS while the first
// weights are on their way.  lds: codes [k][128 ib], scales [k][ib].
__global__ void __launch_bounds__(512) down_token(ExpertArgs a) {
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t token = blockIdx.y, ch = min(static_cast<int32_t>(blockIdx.x) * 8 + wave, a.hidden - 1);
    const int32_t pitch = a.ib * kBlock;
    const int32_t *ids = a.ids + token * a.k;
    const float *weights = a.weights + token * a.k;
    float *scales = reinterpret_cast<float *>(lds + a.k * pitch);
    constexpr int U = 8;
    u4 w[U];
    float s[U];
    bool on[U];
    // items: choices, in each 1024 channels at a time, 16 a lane; those without a term (on) are
    // left out of the sum, not multiplied by 0: what they repeat may be NaN, and a weight of 0 has one
    struct Item {
        int32_t j, k0;
    };
    auto step = [&](Item &i) {
        i.k0 += 1024;
        if (i.k0 >= pitch)
            i = {i.j + 1, 0};
    };
    auto load = [&](Item i) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int32_t j = min(i.j, a.k - 1), k = i.k0 + lane * 16;
            const int32_t e = ids[j], at = min(k, pitch - 16);
            on[u] = i.j < a.k && k < pitch && e >= 0 && e < a.experts;
            const int64_t of = e >= 0 && e < a.experts ? e : 0;
            w[u] = stream16(a.w2 + (of * a.hidden + ch) * pitch + at);
            s[u] = on[u] ? a.s2[(of * a.hb + ch / kBlock) * a.ib + at / kBlock] * weights[j] : 0.0f;
            step(i);
        }
    };
    // inner rows to codes, 8 values a thread; the first are asked for before the ids, which
    // the weights' addresses wait for
    const int l = threadIdx.x & 15, groups = 512 / 16, blocks = a.k * a.ib;
    float v[8];
    auto load_h = [&](int32_t i) {
        const int32_t j = choice_of(a, i), c = (i - j * a.ib) * kBlock + 8 * l;
        load8_tail(a.h + (static_cast<int64_t>(token) * a.k + j) * a.inner + c, i < blocks ? a.inner - c : 0,
                   a.inner % 4 == 0, v);
    };
    load_h(threadIdx.x >> 4);
    Item item{0, 0};
    load(item);
    for (int32_t i = threadIdx.x >> 4; i < blocks; i += groups) {
        const int32_t j = choice_of(a, i), c = (i - j * a.ib) * kBlock + 8 * l;
        uint32_t m = most8(v);
#pragma unroll
        for (int d = 1; d < 16; d *= 2)
            m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), d)));
        const Scale q = scale_of(m);
        *reinterpret_cast<u2 *>(lds + j * pitch + c) = u2{codes4(v, q.inv), codes4(v + 4, q.inv)};
        if (l == 0)
            scales[i] = q.scale;
        load_h(i + groups);
    }
    __syncthreads();
    float acc = 0.0f;
    while (item.j < a.k) {
        if (item.j + item.k0 > 0)
            load(item);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int32_t j = min(item.j, a.k - 1), at = min(item.k0 + lane * 16, pitch - 16);
            step(item);
            float v[16];
            code_values(*reinterpret_cast<const u4 *>(lds + j * pitch + at), v);
            const float d = dot16(v, w[u]) * (scales[j * a.ib + at / kBlock] * s[u]);
            acc += on[u] ? d : 0.0f;
        }
    }
    acc = sum_lanes(acc);
    if (lane == 0 && static_cast<int32_t>(blockIdx.x) * 8 + wave < a.hidden)
        store4(a.y, a.type, static_cast<int64_t>(token) * a.hidden + ch, f4{acc, 0, 0, 0}, 1, false);
}

// y[t] = sum_j weights[t][j] * z[place of (t, j)], in 32 bits, in the order of
// j; a thread sums V neighbouring channels (V = 1: any number of channels).
// Bound by traffic (4096 tokens, 8 of them, 2048 channels: 29 us, 5.4 TB/s).
template <typename T, int V>
__global__ void __launch_bounds__(256) combine(ExpertArgs a, int32_t pieces, bool wide) {
    const int64_t id = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int32_t token = static_cast<int32_t>(id / pieces), ch = static_cast<int32_t>(id % pieces) * V;
    if (token >= a.n)
        return;
    float sum[V] = {};
    const int32_t *place = a.place + static_cast<int64_t>(token) * a.k;
    const float *weights = a.weights + static_cast<int64_t>(token) * a.k;
#pragma unroll 4
    for (int32_t j = 0; j < a.k; ++j) {
        const int64_t at = place[j];
        if (at < 0)
            continue;
        const T *z = reinterpret_cast<const T *>(a.z) + at * a.hidden + ch;
        float v[V];
        if constexpr (V == 8) {
            load8(z, v);
        } else if constexpr (V == 4) {
            struct alignas(4 * sizeof(T)) Four {
                T v[4];
            } f = *reinterpret_cast<const Four *>(z);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                v[i] = static_cast<float>(f.v[i]);
        } else {
            v[0] = static_cast<float>(z[0]);
        }
        float w = weights[j];
        if constexpr (sizeof(T) == 2)
            w *= a.zs[at * a.hb + ch / kBlock];
#pragma unroll
        for (int i = 0; i < V; ++i)
            sum[i] = fmaf(w, v[i], sum[i]);
    }
    const int64_t to = static_cast<int64_t>(token) * a.hidden + ch;
    if constexpr (V == 1) {
        store4(a.y, a.type, to, f4{sum[0], 0, 0, 0}, 1, false);
    } else {
#pragma unroll
        for (int i = 0; i < V; i += 4)
            store4(a.y, a.type, to + i, f4{sum[i], sum[i + 1], sum[i + 2], sum[i + 3]}, 4, wide);
    }
}

template <typename T, int V>
hipError_t combine_by(const ExpertArgs &a, bool wide, hipStream_t stream) {
    const int32_t pieces = a.hidden / V;
    const int64_t blocks = (static_cast<int64_t>(a.n) * pieces + 255) / 256;
    combine<T, V><<<static_cast<uint32_t>(blocks), 256, 0, stream>>>(a, pieces, wide);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_combine(const ExpertArgs &a, bool wide, hipStream_t stream) {
    return a.hidden % 8 == 0   ? combine_by<T, 8>(a, wide, stream)
           : a.hidden % 4 == 0 ? combine_by<T, 4>(a, wide, stream)
                               : combine_by<T, 1>(a, wide, stream);
}

// Most tiles of `high` rows that pairs of so many experts can make.
int64_t most_tiles(const ExpertArgs &a, int32_t high) {
    return std::min<int64_t>(a.pairs, a.pairs / high + std::min(a.experts, a.pairs));
}

uint32_t tile_grid(int64_t tiles, int64_t columns) {
    return static_cast<uint32_t>((tiles * columns + kXcds - 1) / kXcds * kXcds);
}

template <class S>
hipError_t gated_tiles(const ExpertArgs &a, hipStream_t stream) {
    static std::atomic<uint64_t> done{0};
    const hipError_t ready = allow_lds(gated_tile<S>, S::kLds, done);
    if (ready != hipSuccess)
        return ready;
    gated_tile<S><<<tile_grid(most_tiles(a, S::BT), a.ib), S::kThreads, S::kLds, stream>>>(a, a.ib);
    return hipGetLastError();
}

template <class S, bool EXACT, bool HALF>
hipError_t down_tiles(const ExpertArgs &a, hipStream_t stream) {
    static std::atomic<uint64_t> done{0};
    const hipError_t ready = allow_lds(down_tile<S, EXACT, HALF>, S::kLds, done);
    if (ready != hipSuccess)
        return ready;
    const int32_t columns = (a.hidden + S::BC - 1) / S::BC;
    down_tile<S, EXACT, HALF><<<tile_grid(most_tiles(a, S::BT), columns), S::kThreads, S::kLds, stream>>>(a, columns);
    return hipGetLastError();
}

// A tile's rows by the rows that an expert has on average, as long as compute units, which hold
// one tile of any size (LDS; so the smaller ones are three blocks deep), have one.  Measured
// (calls of 64 experts of 2048 x 1024 in bf16, by the first products' tiles): 512 rows each 477 us in
// tiles of 128, 516 in 256, 559 in 64; 150 rows 198, 262, 213; 100 rows 160, 198, 171; 50 rows 122, 169,
// 121; so the first products' are of 128 rows at most.  By tiles at most: 256 rows each, second
// products in 64 tiles of 256 rows 26.4 us, 96 of 128 rows 18.2, 160 of 64 14.2; 1024 rows each, 160 of 256
// 30.8, 288 of 128 36.2; 128 rows each, 128 tiles of 128 18.9, 192 of 64 14.6, but 256 of 128 10.1, 384
// of 64 13.2.
int32_t tile_rows(const ExpertArgs &a, int64_t columns, bool big) {
    const int64_t each = a.pairs / a.experts;
    if (big && each >= 192 && most_tiles(a, 256) * columns >= 144)
        return 256;
    return each >= 96 && most_tiles(a, 128) * columns >= 144 ? 128 : 64;
}

template <typename T>
hipError_t prepare(const ExpertArgs &a, hipStream_t stream) {
    const bool wide = reinterpret_cast<uintptr_t>(a.x) % 16 == 0 && a.ldx * static_cast<int64_t>(sizeof(T)) % 16 == 0;
    const bool wide_ids = reinterpret_cast<uintptr_t>(a.ids) % 16 == 0;
    const int32_t threads = a.pairs >= 4096 ? 1024 : 256;
    const int32_t groups = (a.n + threads / 16 - 1) / (threads / 16);
    if (static_cast<int64_t>(groups) * a.hb >= 1024)
        prepare_rows<T, 4><<<a.experts + groups * ((a.hb + 3) / 4), threads, 0, stream>>>(a, groups, wide_ids, wide);
    else
        prepare_rows<T, 1><<<a.experts + groups * a.hb, threads, 0, stream>>>(a, groups, wide_ids, wide);
    return hipGetLastError();
}

template <typename T>
hipError_t gated_tokens(const ExpertArgs &a, hipStream_t stream) {
    const bool wide = reinterpret_cast<uintptr_t>(a.x) % 16 == 0 && a.ldx * static_cast<int64_t>(sizeof(T)) % 16 == 0;
    const int32_t channels = 4 * kTokenChannels;
    gated_token<T><<<dim3((a.inner + channels - 1) / channels, a.pairs), 256, 0, stream>>>(a, wide);
    return hipGetLastError();
}

}  // namespace

// Token by token where pairs are of different experts mostly: one or two tokens, and a few more
// while the weights are small, so that two launches in place of four count.  Measured (bf16, over tiles in
// brackets): 2048 x 1024, 8 of 64 experts, 1 token 20.5 us (34.1), 2 29.9 (35.4), 4 51.3 (43.8);
// 1024 x 512, 4 of 128, 4 tokens 17.9 (21.1), 6 22.7 (22.2); 512 x 256, 8 of 64, 4 tokens 17.6 (19.1),
// 6 21.9 (19.1); 512 x 512, 1 of 32, 8 tokens 13.6 (17.6), 16 20.7 (17.5).
bool experts_by_token(int32_t n, int32_t k, int32_t experts, int32_t hidden, int32_t inner) {
    const int64_t pairs = static_cast<int64_t>(n) * k, weights = pairs * 3 * hidden * inner;
    if (pairs > experts || k * blocks_of(inner) > 384)  // inner rows in 50 KB of LDS
        return false;
    return n <= 2 ? pairs <= 64 : n <= 8 && pairs <= 32 && weights <= 32 << 20;
}

hipError_t launch_experts(ExpertArgs a, hipStream_t stream) {
    a.k_inverse = (uint32_t(1) << 31) / a.k + 1;
    a.ib_inverse = (uint32_t(1) << 31) / a.ib + 1;
    const bool wide = a.hidden % 4 == 0 && reinterpret_cast<uintptr_t>(a.y) % 16 == 0;
    hipError_t e;
    if (experts_by_token(a.n, a.k, a.experts, a.hidden, a.inner)) {
        e = a.type == kF32   ? gated_tokens<float>(a, stream)
            : a.type == kF16 ? gated_tokens<_Float16>(a, stream)
                             : gated_tokens<__bf16>(a, stream);
        if (e != hipSuccess)
            return e;
        const int32_t blocks = a.k * a.ib;
        down_token<<<dim3((a.hidden + 7) / 8, a.n), 512, blocks * (kBlock + 4), stream>>>(a);
        return hipGetLastError();
    }
    e = a.type == kF32 ? prepare<float>(a, stream) : a.type == kF16 ? prepare<_Float16>(a, stream) : prepare<__bf16>(a, stream);
    if (e != hipSuccess)
        return e;
    using Small = TileShape<256, 64, 2, 4, 3>;
    using Mid = TileShape<256, 128, 2, 4, 3>;
    using Big = TileShape<256, 256, 2, 4>;
    // The inner rows are rounded to codes again, which would turn the 8-bit instruction's error into
    // many times itself (4e-5 of well spread values into 1.2e-3, with loud channels into more than the
    // rounding of a bf16 result), so the first products are exact for every type.  The results' error
    // is their own: exact products for 32 bits only.
    const int32_t first = tile_rows(a, a.ib, false), second = tile_rows(a, (a.hidden + 255) / 256, true);
    e = first == 128 ? gated_tiles<Mid>(a, stream) : gated_tiles<Small>(a, stream);
    if (e != hipSuccess)
        return e;
    if (a.type == kF32)
        e = second == 256   ? down_tiles<Big, true, false>(a, stream)
            : second == 128 ? down_tiles<Mid, true, false>(a, stream)
                            : down_tiles<Small, true, false>(a, stream);
    else if (a.type == kF16)
        e = second == 256   ? down_tiles<Big, false, false>(a, stream)
            : second == 128 ? down_tiles<Mid, false, false>(a, stream)
                            : down_tiles<Small, false, false>(a, stream);
    else
        e = second == 256   ? down_tiles<Big, false, true>(a, stream)
            : second == 128 ? down_tiles<Mid, false, true>(a, stream)
                            : down_tiles<Small, false, true>(a, stream);
    if (e != hipSuccess)
        return e;
    return a.type == kBf16 ? launch_combine<_Float16>(a, wide, stream) : launch_combine<float>(a, wide, stream);
}

}  // namespace spconv
