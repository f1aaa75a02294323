// The next token of each row of logits, from a given random number.
//
// With l a row's logits (tokens of -infinity or NaN are off, +infinity counts as
// the largest finite number), m their maximum and t the temperature, a token
// weighs w = exp((l - m) / t).  Tokens are ordered by l, the largest first, equal
// ones by their index.  Kept are the first k of that order, of these the
// shortest start that reaches the share p of their weight, of these the ones
// with w >= min_p.  The token is the first, by index, at which the running sum of
// the kept weights exceeds u times their sum.
//
// The order is that of one whole number a token, its key: 32 bits of l, then 20 of
// the index from behind.  So every filter is a least key.  Weights are 64-bit
// exponentials, rounded to multiples of 2^-42 of the largest (of all, or of its
// chunk) before they are added: sums of up to 2^20 tokens stay below 2^62 and are
// exact in any order, which makes the atomics that collect some of them harmless,
// and next to a border the choice is the definition's but for those roundings
// (2e-11 of the largest weight's size over 2^17 tokens).  Nothing depends on the
// other rows of the call.
//
// The border of a filter lies in a bin of a histogram of the distance to m (in
// counts for k, in weights for p); the tokens of that bin are listed, sorted and
// added up.  A bin with more than the list holds goes digit by digit through the
// keys.
//
// Rows of up to 8192 tokens: one workgroup a row, which keeps it in LDS.  Longer
// rows are cut into chunks of 8192 neighbours, one a workgroup, so that a few rows
// fill the card; a launch ends where every chunk's part is needed:
//   A  each chunk's largest key, the largest of each 32 tokens (a segment), and,
//      where nothing is filtered, the sum of its weights;
//   B  where k or p has a border in a bin, or min_p alone is asked for: each chunk's sum (min_p) or
//      its part of the histogram;
//   C  each chunk adds up what is above the border's bin and lists what is in it;
//   D  the token, a workgroup a row: without a filter from the chunks' sums; of few kept tokens (k)
//      from the segments: the k-th largest of their keys bounds the k-th largest key from below, so
//      that only the segments above it are read again; else from the border in the list and the sums.
// Calls whose rows all need neither B nor C do without them.  Few kept tokens are D's although A is
// all that they wait for: in B, 64 x 131072 with parameters by row took 75 us in place of 57.
// k above 1024 together with p, and longer lists than 8192, go to one workgroup that
// walks over the whole row: a flat row of 131072 or a border among 2^20 tokens whose bin holds so many
// takes 0.9 and 4.2 ms with p = 0.9.
//
// What bounds it.  64 x 131072 in bf16 (16.8 MB, 3.3 us at a copy's rate), on the device alone: t = 0
// 8.6 us; no filter 21, of it 9 the exponentials (25 64-bit operations each); k = 50 18, of it 10
// the steps of D, one after the other, each some loads or a few LDS accesses and barriers long (1000
// to 2500 cycles; k = 500 31); p = 0.9 55: A 6.6, B 15 (exponentials and LDS atomics), C 13, D 20
// (the border in 1200 listed tokens 9, the token 5).  One row of 4000: 8.4 to 9.1, with p 13.3.
// Steps one after the other are why a workgroup has 512 threads and not 1024 (each thread's share
// of such a step is done by twice as many: k = 50 of 4000 took 14 us).  They wait for their own
// results, not for instructions: the same steps done again at once take nine tenths.
#include <algorithm>

#include "fp8.hpp"
#include "serve_ops.hpp"

namespace spconv {
namespace {

typedef unsigned long long Sum;

constexpr float kMostLogit = 3.402823466e38f;
constexpr int kIndexBits = 20;
constexpr int kBins = 2048;       // of a histogram
constexpr int kThreads = 512;     // of a workgroup but in A
constexpr int kWaves = kThreads / 64;
constexpr int kChunk = 8192;
constexpr int kSegments = 256;    // of a chunk: threads in A, 32 tokens each
constexpr int kFew = 1024;        // most tokens that a list in LDS holds
constexpr int kSorted = 128;      // most of them that are sorted at once
constexpr int kList = 8192;       // most tokens of a list in memory
constexpr float kLastBelow1 = 0x1.fffffep-1f;

// A logit as it counts: -infinity where its token is off, no -0.
__device__ __forceinline__ float counted(float l) { return l != l ? -INFINITY : fminf(l, kMostLogit) + 0.0f; }

__device__ __forceinline__ uint64_t key_of(float l, int32_t token) {
    const uint32_t b = __float_as_uint(l), order = b >> 31 ? ~b : b | 0x80000000u;
    return static_cast<uint64_t>(order) << kIndexBits | (kMostTokens - 1 - token);
}
__device__ __forceinline__ int32_t token_of(uint64_t key) {
    return kMostTokens - 1 - static_cast<int32_t>(key & (kMostTokens - 1));
}
__device__ __forceinline__ float logit_of(uint64_t key) {
    const uint32_t order = static_cast<uint32_t>(key >> kIndexBits);
    return __uint_as_float(order >> 31 ? order & 0x7fffffffu : ~order);
}

// Eight logits from p, of which `left` exist, as they count; any alignment.
template <typename T>
__device__ __forceinline__ void load_logits(const T *p, int left, float *v) {
    if (left >= 8) {
        struct __attribute__((packed, aligned(sizeof(T)))) Piece {
            T v[8];
        } e = *reinterpret_cast<const Piece *>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = counted(static_cast<float>(e.v[i]));
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        v[i] = i < left ? counted(static_cast<float>(p[i])) : -INFINITY;
}

enum Mode { kGreedy, kAll, kLeast, kFewKept, kShare, kCount, kDigits };

// Whether the first k of a row are listed in LDS.  Alone, 1000 take less as a histogram (on the device,
// one row of 131072 28 us and 83, 256 x 50001 67 and 90), 600 of one row as much (28), of many rows more
// (256 x 50001 67 and 38).  Together with a share, a list is what there is but for the walk over the
// whole row (64 x 131072 with p = 0.9: k = 1000 100 us, as a walk 314; k = 2000 330).
__host__ __device__ __forceinline__ bool few_kept(int32_t k, bool share) { return k <= (share ? kFew : 512); }

// A number that stays in scalar registers: else each use of it would be moved to vector registers.
__device__ __forceinline__ double scalar(double v) {
    asm("" : "+s"(v));
    return v;
}

// What a weight is computed with, at hand before the loops.
struct Numbers {
    double shift = scalar(42.0), least = scalar(-960.0), to_whole = scalar(0x1.8p52), to_units = scalar(0x1p52);
    double p9 = scalar(0x1.b638718fee5a8p-24), p8 = scalar(0x1.63d136366db24p-20), p7 = scalar(0x1.ffcb95269d85ap-17),
           p6 = scalar(0x1.4308ac85aa947p-13), p5 = scalar(0x1.5d87fe86f82cdp-10), p4 = scalar(0x1.3b2ab7181b755p-7),
           p3 = scalar(0x1.c6b08d7047e8bp-5), p2 = scalar(0x1.ebfbdff823cedp-3), p1 = scalar(0x1.62e42fefa39efp-1);
};

// A row's parameters, as they count.
struct Row {
    Numbers c;
    double scale;  // log2(e) / temperature
    double top_p, u;
    double min_p;  // times 2^42, as weights are
    int32_t top_k;
    Mode mode;
};

__device__ __forceinline__ Row row_of(const SampleArgs &a, int32_t row) {
    const float t = a.temperatures ? a.temperatures[row] : a.temperature;
    const float p = a.top_ps ? a.top_ps[row] : a.top_p, least = a.min_ps ? a.min_ps[row] : a.min_p;
    const float u = a.u[row];
    Row r;
    r.scale = 1.4426950408889634 / static_cast<double>(t);
    r.top_k = a.top_ks ? a.top_ks[row] : a.top_k;
    if (r.top_k <= 0 || r.top_k > a.vocab)
        r.top_k = a.vocab;
    r.top_p = p < 1 ? p : 1.0;  // a NaN is off, as 1 is
    r.min_p = least > 0 ? fminf(least, 1.0f) * 0x1p42 : 0.0;
    r.u = u > 0 ? fminf(u, kLastBelow1) : 0.0;
    const bool some = r.top_k < a.vocab, share = r.top_p < 1;
    r.mode = !(t > 0)            ? kGreedy
             : !some && !share   ? r.min_p > 0 ? kLeast : kAll
             : some && few_kept(r.top_k, share) ? kFewKept
             : !some             ? kShare
             : !share            ? kCount
                                 : kDigits;
    return r;
}

// A token's weight times 2^42: 2^z with z = (l - m) scale + 42, as 2^n times a polynomial in f = z -
// n, |f| <= 1/2: the one of degree 9 that agrees with 2^f at nine Chebyshev nodes, of which 0 is one,
// and at 0 in its slope, too; 3.7e-14 off, exact at 0, so that the largest weight is 2^42.  n is found
// by an addition whose sum's last place is one.  z is cut off at -960, which is far below what counts.
__device__ __forceinline__ double weight_of(float l, float most, const Row &r) {
    const double z = fmax(fma(static_cast<double>(l) - static_cast<double>(most), r.scale, r.c.shift), r.c.least);
    const double shifted = z + r.c.to_whole, f = z - (shifted - r.c.to_whole);
    double p = fma(r.c.p9, f, r.c.p8);
    p = fma(p, f, r.c.p7);
    p = fma(p, f, r.c.p6);
    p = fma(p, f, r.c.p5);
    p = fma(p, f, r.c.p4);
    p = fma(p, f, r.c.p3);
    p = fma(p, f, r.c.p2);
    p = fma(p, f, r.c.p1);
    p = fma(p, f, 1.0);
    const uint64_t bits = __builtin_bit_cast(uint64_t, p);
    const uint32_t n = static_cast<uint32_t>(__builtin_bit_cast(uint64_t, shifted));
    return __builtin_bit_cast(double, bits + (static_cast<uint64_t>(n) << 52));
}
// Such a weight as a whole number, rounded to nearest by the same kind of addition.
__device__ __forceinline__ Sum units(double w, const Row &r) {
    return __builtin_bit_cast(Sum, w + r.c.to_units) & ((Sum(1) << 52) - 1);
}
// Whether a 64-bit exponential of the token is above 0.
__device__ __forceinline__ bool weighs(float l, float most, const Row &r) {
    return (static_cast<double>(l) - static_cast<double>(most)) * r.scale > -1074.5;
}
// What a token that the keys keep adds to the last sum: its units, or for u = 0, which takes the
// first token however small, whether it weighs.
__device__ __forceinline__ Sum last_weight(float l, float most, const Row &r) {
    const double w = weight_of(l, most, r);
    return w < r.min_p ? 0 : r.u == 0 ? weighs(l, most, r) : units(w, r);
}

// Steps over the lanes of a wavefront by data-parallel moves, which take a fraction of a shuffle
// through LDS: CTRL 0x111, 0x112, 0x114, 0x118 shift rows of 16 lanes by 1, 2, 4, 8, 0x142 hands
// lane 15 of rows 0 and 2 on, 0x143 lane 31.  Lanes without a source get 0.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t moved(uint64_t v) {
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, ROWS, 0xf, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, static_cast<int>(v >> 32), CTRL, ROWS, 0xf, false);
    return static_cast<uint64_t>(hi) << 32 | lo;
}

__device__ __forceinline__ uint64_t from_lane(uint64_t v, int lane) {
    const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(v), lane);
    const uint32_t hi = __builtin_amdgcn_readlane(static_cast<int>(v >> 32), lane);
    return static_cast<uint64_t>(hi) << 32 | lo;
}

// The running sum over the lanes.
__device__ __forceinline__ Sum run_of(Sum v) {
    v += moved<0x111, 0xf>(v);
    v += moved<0x112, 0xf>(v);
    v += moved<0x114, 0xf>(v);
    v += moved<0x118, 0xf>(v);
    v += moved<0x142, 0xa>(v);
    v += moved<0x143, 0xc>(v);
    return v;
}

__device__ __forceinline__ uint64_t most_all(uint64_t v) {
    auto step = [&](uint64_t o) { v = o > v ? o : v; };
    step(moved<0x111, 0xf>(v));
    step(moved<0x112, 0xf>(v));
    step(moved<0x114, 0xf>(v));
    step(moved<0x118, 0xf>(v));
    step(moved<0x142, 0xa>(v));
    step(moved<0x143, 0xc>(v));
    return from_lane(v, 63);
}

// Of the wavefronts' parts of a workgroup the sum, and the sum of those before this one.
template <int WAVES>
__device__ __forceinline__ Sum sum_parts(const Sum *part, Sum &before) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Sum v = part[threadIdx.x & (WAVES - 1)];
    v += moved<0x111, 0xf>(v);
    v += moved<0x112, 0xf>(v);
    if (WAVES > 4)
        v += moved<0x114, 0xf>(v);
    before = wave ? from_lane(v, wave - 1) : 0;
    return from_lane(v, WAVES - 1);
}

// The largest over a workgroup; part: a place for each wavefront.
template <int WAVES>
__device__ __forceinline__ uint64_t most_block(uint64_t v, Sum *part) {
    v = most_all(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
        part[threadIdx.x >> 6] = v;
    __syncthreads();
    return most_all(part[threadIdx.x & (WAVES - 1)]);
}

// The sum over a workgroup, and the running sum up to and with each thread.
template <int WAVES>
__device__ __forceinline__ Sum sum_block(Sum v, Sum *part, Sum *run = nullptr) {
    const Sum up = run_of(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 63)
        part[threadIdx.x >> 6] = up;
    __syncthreads();
    Sum before;
    const Sum total = sum_parts<WAVES>(part, before);
    if (run)
        *run = before + up;
    return total;
}

// Where a call's workspace holds what of a row.
struct Space {
    uint64_t *best;      // [chunks] largest key, 0 without a token
    Sum *sums;           // [chunks]
    uint64_t *segments;  // [chunks][256] largest keys of 32 tokens
    Sum *bins;           // [kBins]
    uint64_t *list;      // [kList] keys
    uint32_t *count;     // tokens of the list
};

__host__ __device__ __forceinline__ int32_t chunks_of(int32_t vocab) { return (vocab + kChunk - 1) / kChunk; }
// Its words, and of those the first, which are all that rows without a histogram have.
__host__ __device__ __forceinline__ int64_t chunk_words(int32_t vocab) {
    return static_cast<int64_t>(chunks_of(vocab)) * (2 + kSegments);
}
__host__ __device__ __forceinline__ int64_t row_words(int32_t vocab) { return chunk_words(vocab) + kBins + kList + 1; }

__device__ __forceinline__ Space space_of(const SampleArgs &a, int32_t row) {
    uint64_t *p = static_cast<uint64_t *>(a.workspace) + row * a.words;
    const int32_t chunks = chunks_of(a.vocab);
    Space s;
    s.best = p;
    s.sums = reinterpret_cast<Sum *>(p + chunks);
    s.segments = p + 2 * chunks;
    s.bins = reinterpret_cast<Sum *>(p + chunk_words(a.vocab));
    s.list = p + chunk_words(a.vocab) + kBins;
    s.count = reinterpret_cast<uint32_t *>(s.list + kList);
    return s;
}

// The bin of a token's distance to the maximum, the nearest highest: 128 an octave, from 2^-8 to 2^8.
__device__ __forceinline__ int bin_of(float l, float most) {
    const uint32_t b = __float_as_uint(most - l) >> 16;
    constexpr uint32_t kFirst = (127 - 8) << 7;
    return kBins - 1 - static_cast<int>(b < kFirst ? 0 : min(b - kFirst + 1, static_cast<uint32_t>(kBins - 1)));
}

// The least distance, as bits, that lies behind a bin; none, infinity neither, behind the last or without one.
__device__ __forceinline__ uint32_t end_of(int bin) {
    constexpr uint32_t kFirst = (127 - 8) << 7;
    return bin == kBins - 1 ? kFirst << 16 : bin > 0 ? (kFirst + kBins - 1 - bin) << 16 : 0x7f800001u;
}

struct Found {
    int bin;  // -1: none
    Sum above, upto;  // of the bins above it, with it
    double target;
};

// LDS of all kernels but A: what finds borders, ...
struct Common {
    Sum part[kWaves];
    Found found;
    uint32_t count;
    struct {
        int32_t first;
        Sum before;
    } at;
};
struct OneRow : Common {
    Sum bins[kBins];
    uint64_t few[kFew];
    uint32_t rank[kFew];
};

// ... or a chunk with the chunks' sums.
struct Shared : Common {
    union {
        struct {
            Sum bins[kBins];
            uint64_t few[kFew];
            uint32_t rank[kFew];
        };
        struct {
            Sum sums[kMostTokens / kChunk];
            double mass[kMostTokens / kChunk], factor[kMostTokens / kChunk];
            __attribute__((aligned(16))) float held[kChunk];
        };
    };
};

// The first bin from above (and not empty) at which the running sum reaches a number, or passes it: k,
// or the share p of all bins where p < 1.
template <class S>
__device__ __forceinline__ Found find(S &sh, const Sum *bins, double k, double p, bool pass = false) {
    constexpr int kOwn = kBins / kThreads;
    if (threadIdx.x == 0)
        sh.found = {-1, 0, 0, 0};
    const int b0 = kBins - kOwn * (static_cast<int>(threadIdx.x) + 1);  // this thread's bins
    Sum own[kOwn], mine = 0, run;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
        own[j] = bins[b0 + j];
        mine += own[j];
    }
    const Sum total = sum_block<kWaves>(mine, sh.part, &run);
    const double least = p < 1 ? p * static_cast<double>(total) : k;
    auto reaches = [&](Sum v) { return pass ? static_cast<double>(v) > least : static_cast<double>(v) >= least; };
    Sum above = run - mine;
    if (mine && reaches(run) && !(above && reaches(above))) {
        for (int j = kOwn - 1; j >= 0; --j) {
            const Sum upto = above + own[j];
            if (own[j] && reaches(upto)) {
                sh.found = {b0 + j, above, upto, least};
                break;
            }
            above = upto;
        }
    }
    __syncthreads();
    const Found f = sh.found;
    __syncthreads();
    return f;
}

__device__ __forceinline__ void clear(Sum *bins, int count) {
    for (int b = threadIdx.x; b < count; b += blockDim.x)
        bins[b] = 0;
    __syncthreads();
}

// The largest key of a row from those of its chunks; 0 without a token.
__device__ __forceinline__ uint64_t best_of(const Space &s, int32_t chunks) {
    const int lane = threadIdx.x & 63;
    uint64_t best = 0;
    for (int c = lane; c < chunks; c += 64)
        best = s.best[c] > best ? s.best[c] : best;
    return most_all(best);
}

// The place in the list of the first of `count` entries of this lane; a wavefront asks as one.
__device__ __forceinline__ uint32_t place_in(uint32_t *total, uint32_t count) {
    const Sum run = run_of(count);
    uint32_t base = 0;
    if ((threadIdx.x & 63) == 63 && run)
        base = atomicAdd(total, static_cast<uint32_t>(run));
    return __builtin_amdgcn_readlane(static_cast<int>(base), 63) + static_cast<uint32_t>(run) - count;
}

// Puts the first m (at most kSorted) of sh.few, different where not 0, in order, the largest first:
// each counts the larger ones, blocks of 64 by wavefronts, which share the others.  (A network of
// exchanges, whose steps wait for each other, took 1.8 us for 64.)
template <class S>
__device__ __forceinline__ void sort_few(S &sh, int32_t m) {
    if (m < 2)
        return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t blocks = (m + 63) / 64, slices = kWaves / blocks, slice = wave / blocks, each = (m + slices - 1) / slices;
    const int32_t t = static_cast<int32_t>(threadIdx.x);
    if (t < m)
        sh.rank[t] = 0;
    __syncthreads();
    if (slice < slices) {
        const int32_t i = wave % blocks * 64 + lane, end = min(m, (slice + 1) * each);
        const uint64_t key = i < m ? sh.few[i] : 0;
        uint32_t larger = 0;
#pragma unroll 4
        for (int32_t j = slice * each; j < end; ++j)
            larger += sh.few[j] > key;
        if (i < m && larger)
            atomicAdd(&sh.rank[i], larger);
    }
    __syncthreads();
    const uint64_t key = t < m ? sh.few[t] : 0;
    const uint32_t rank = t < m ? sh.rank[t] : 0;
    __syncthreads();
    if (t < m)
        sh.few[rank] = key;
    __syncthreads();
}

// Of m values in sh.few (different where not 0) the first, from the largest on, at which the running
// weight(value) reaches `target`, or passes it; the least of them where a rounding leaves it short.
// More than can be sorted at once are narrowed down by their digits.  Uses sh.few and sh.bins up.
template <class S, class Weight>
__device__ __forceinline__ uint64_t border_of_few(S &sh, int32_t m, double target, bool pass, Weight weight) {
    constexpr int kOwn = kFew / kThreads;
    const int32_t t = static_cast<int32_t>(threadIdx.x);
    if (m > kSorted) {
        uint64_t own[kOwn], low = ~uint64_t(0), high = 0;
#pragma unroll
        for (int j = 0; j < kOwn; ++j) {
            own[j] = t + j * kThreads < m ? sh.few[t + j * kThreads] : 0;
            low = own[j] && own[j] < low ? own[j] : low;
            high = own[j] > high ? own[j] : high;
        }
        low = ~most_block<kWaves>(~low, sh.part);
        high = most_block<kWaves>(high, sh.part);
        int shift = low < high ? 64 - __builtin_clzll(low ^ high) : 0;
        while (m > kSorted && shift > 0) {
            const int width = min(shift, 11);
            const uint64_t prefix = shift < 64 ? high >> shift : 0;  // of all that are left
            shift -= width;
            if (t == 0)
                sh.count = 0;
            clear(sh.bins, kBins);
#pragma unroll
            for (int j = 0; j < kOwn; ++j)
                if (own[j])
                    if (const Sum w = weight(own[j]))
                        atomicAdd(&sh.bins[own[j] >> shift & ((1 << width) - 1)], w);
            __syncthreads();
            const Found f = find(sh, sh.bins, target, 1.0, pass);
            if (f.bin < 0)
                break;
            target -= static_cast<double>(f.above);
            high = (prefix << width | static_cast<uint64_t>(f.bin)) << shift;  // (its upper bits)
            uint32_t mine = 0;
#pragma unroll
            for (int j = 0; j < kOwn; ++j) {
                own[j] = own[j] && own[j] >> shift == high >> shift ? own[j] : 0;
                mine += own[j] != 0;
            }
            uint32_t at = place_in(&sh.count, mine);
#pragma unroll
            for (int j = 0; j < kOwn; ++j)
                if (own[j])
                    sh.few[at++] = own[j];
            __syncthreads();
            m = static_cast<int32_t>(sh.count);
            __syncthreads();
        }
        if (m > kSorted)
            return low;  // not reached by a rounding
    }
    sort_few(sh, m);
    const Sum own = t < m ? weight(sh.few[t]) : 0;
    Sum run;
    if (t == 0)
        sh.count = m - 1;
    sum_block<kWaves>(own, sh.part, &run);
    if (t < m && (pass ? static_cast<double>(run) > target : static_cast<double>(run) >= target))
        atomicMin(&sh.count, static_cast<uint32_t>(t));
    __syncthreads();
    const uint64_t least = sh.few[sh.count];
    __syncthreads();
    return least;
}

// The least key of those that a walk visits, digit by digit: with `each(f)` calling f(key, weight)
// for keys, the first, from the largest key on, at which the running weight reaches `target`;
// where it never does, the least key that has the prefix.  shift: bits below the ones that all
// keys have in common (prefix).
// enough: stops where so few weights (counts) are up to the end of a bin, at its least key.
template <class S, class Each>
__device__ __forceinline__ uint64_t least_key(S &sh, double target, uint64_t prefix, int shift, Sum enough, Each each) {
    Sum above = 0;
    while (shift > 0) {
        const int width = min(shift, 11), to = shift - width;
        clear(sh.bins, kBins);
        each([&](uint64_t key, Sum weight) {
            if (key >> shift == prefix)
                atomicAdd(&sh.bins[key >> to & ((1 << width) - 1)], weight);
        });
        __syncthreads();
        const Found f = find(sh, sh.bins, target, 1.0);
        if (f.bin < 0)
            break;  // all of these; behind the first digit by a rounding of `target` alone
        target -= static_cast<double>(f.above);
        prefix = prefix << width | static_cast<uint64_t>(f.bin);
        shift = to;
        if (enough && above + f.upto <= enough)
            break;
        above += f.above;
    }
    return prefix << shift;
}

// A filter's least key over all tokens of a row, of which `walk(f)` calls f(logit, token) for the
// ones that earlier filters kept: the first, from the largest on, at which the running weight(key)
// reaches k, or the share p of all where p < 1; 0 where all are kept.  `list(test)` appends the
// keys of those tokens that pass to sh.few, up to kFew, and counts all.
template <class S, class Walk, class List, class Weight>
__device__ __forceinline__ uint64_t border_of(S &sh, float most, double k, double p, Walk walk, List list, Weight weight) {
    if (threadIdx.x == 0)
        sh.count = 0;
    clear(sh.bins, kBins);
    walk([&](float v, int32_t i) {
        if (const Sum w = weight(key_of(v, i)))
            atomicAdd(&sh.bins[bin_of(v, most)], w);
    });
    __syncthreads();
    const Found f = find(sh, sh.bins, k, p);
    if (f.bin < 0)
        return 0;
    list([&](float v, int32_t i) { return bin_of(v, most) == f.bin; });
    __syncthreads();
    const int32_t m = static_cast<int32_t>(sh.count);
    const double target = f.target - static_cast<double>(f.above);
    if (m <= kFew)
        return border_of_few(sh, m, target, false, weight);
    uint64_t least = ~uint64_t(0);  // of the bin
    walk([&](float v, int32_t i) {
        const uint64_t key = key_of(v, i);
        least = bin_of(v, most) == f.bin && key < least ? key : least;
    });
    least = ~most_block<kWaves>(~least, sh.part);
    const uint64_t found = least_key(sh, target, 0, 32 + kIndexBits, 0, [&](auto g) {
        walk([&](float v, int32_t i) {
            if (bin_of(v, most) == f.bin)
                g(key_of(v, i), weight(key_of(v, i)));
        });
    });
    return found > least ? found : least;
}

// The token at which the running weight, from `before` on, exceeds `border`, of `count` neighbours
// from `first` on, of which token i adds kept(i); at the last one's end it does.  A thread adds up
// a run of them, an odd number (LDS is then read without conflicts), and one wavefront looks
// through the run that holds the border.
template <class S, class Kept>
__device__ __forceinline__ void pick(const SampleArgs &a, int32_t row, int32_t first, int32_t count, Sum before, double border,
                                     S &sh, Kept kept) {
    const int32_t each = ((count + kThreads - 1) / kThreads) | 1, i0 = static_cast<int32_t>(threadIdx.x) * each;
    const int32_t own = min(max(count - i0, 0), each);
    Sum mine = 0, run;
#pragma unroll 4
    for (int32_t j = 0; j < own; ++j)
        mine += kept(first + i0 + j);
    sum_block<kWaves>(mine, sh.part, &run);
    run += before;
    if (static_cast<double>(run) > border && !(static_cast<double>(run - mine) > border)) {
        sh.at.first = i0;
        sh.at.before = run - mine;
    }
    __syncthreads();
    if (threadIdx.x >= 64)
        return;
    Sum at = sh.at.before;
    for (int32_t j = sh.at.first; j < count; j += 64) {
        const int32_t i = j + static_cast<int32_t>(threadIdx.x);
        const Sum up = run_of(i < count ? kept(first + i) : 0) + at;
        const uint64_t past = __ballot(static_cast<double>(up) > border);
        if (past) {
            if (threadIdx.x == 0)
                a.ids[row] = first + j + __builtin_ctzll(past);
            return;
        }
        at = from_lane(up, 63);
    }
}

// The token from m keys in sh.few, among them the first k of the row: in their order, where each
// filter keeps a start of what the one before kept, then by index.
template <class S>
__device__ __forceinline__ void pick_few(const SampleArgs &a, int32_t row, const Row &r, int32_t m, float most, S &sh) {
    const int32_t t = static_cast<int32_t>(threadIdx.x);
    if (m <= kSorted) {
        sort_few(sh, m);
        const bool first = t < m && t < r.top_k;
        const uint64_t key = first ? sh.few[t] : 0;
        const float l = logit_of(key);
        const Sum weight = first ? units(weight_of(l, most, r), r) : 0, last = first ? last_weight(l, most, r) : 0;
        bool kept = last > 0;
        if (r.top_p < 1) {
            Sum run;
            const Sum share = sum_block<kWaves>(weight, sh.part, &run);
            kept = kept && (t == 0 || static_cast<double>(run - weight) < r.top_p * static_cast<double>(share));
        }
        const int32_t count = __syncthreads_count(kept);
        // by index: 20 bits of the index above 43 of the weight, the lowest index largest
        if (kept)
            sh.few[t] = (key & (kMostTokens - 1)) << 43 | last;
        __syncthreads();
        sort_few(sh, count);
        const uint64_t both = t < count ? sh.few[t] : 0;
        const Sum own = both & ((uint64_t(1) << 43) - 1);
        Sum upto;
        const double border = r.u * static_cast<double>(sum_block<kWaves>(own, sh.part, &upto));
        if (own && static_cast<double>(upto) > border && !(static_cast<double>(upto - own) > border))
            a.ids[row] = token_of(both >> 43);
        return;
    }
    constexpr int kOwn = kFew / kThreads;
    uint64_t key[kOwn], least = 0;
    auto put = [&](auto f) {
#pragma unroll
        for (int j = 0; j < kOwn; ++j)
            if (t + j * kThreads < m)
                sh.few[t + j * kThreads] = f(key[j]);
        __syncthreads();
    };
#pragma unroll
    for (int j = 0; j < kOwn; ++j)
        key[j] = t + j * kThreads < m ? sh.few[t + j * kThreads] : 0;
    auto weight = [&](uint64_t k) { return k >= least ? units(weight_of(logit_of(k), most, r), r) : 0; };
    if (m > r.top_k) {
        __syncthreads();
        least = border_of_few(sh, m, r.top_k, false, [&](uint64_t) { return Sum(1); });
    }
    if (r.top_p < 1) {
        Sum mine = 0;
#pragma unroll
        for (int j = 0; j < kOwn; ++j)
            mine += key[j] ? weight(key[j]) : 0;
        const Sum share = sum_block<kWaves>(mine, sh.part);
        put([&](uint64_t k) { return k; });
        const uint64_t border = border_of_few(sh, m, r.top_p * static_cast<double>(share), false, weight);
        least = border > least ? border : least;
    }
    Sum mine = 0;
    auto last = [&](uint64_t k) { return k && k >= least ? last_weight(logit_of(k), most, r) : 0; };
#pragma unroll
    for (int j = 0; j < kOwn; ++j)
        mine += last(key[j]);
    const double border = r.u * static_cast<double>(sum_block<kWaves>(mine, sh.part));
    put([&](uint64_t k) {
        const Sum w = last(k);
        return w ? (k & (kMostTokens - 1)) << 43 | w : 0;
    });
    const uint64_t both = border_of_few(sh, m, border, true, [&](uint64_t v) { return v & ((uint64_t(1) << 43) - 1); });
    if (t == 0)
        a.ids[row] = token_of(both >> 43);
}

// One row in one workgroup; held: LDS that takes the row, or null: then it is read anew for each
// step.
template <typename T, bool HELD, class S>
__device__ __forceinline__ void whole_row(const SampleArgs &a, int32_t row, const Row &r, S &sh, float *held) {
    const T *l = static_cast<const T *>(a.logits) + row * a.ld;
    const int32_t t = static_cast<int32_t>(threadIdx.x);
    float top = -INFINITY;  // of this thread's groups of eight neighbours
    int32_t token = 0;
#pragma unroll 4
    for (int32_t i = t * 8; i < a.vocab; i += kThreads * 8) {
        float v[8];
        load_logits(l + i, a.vocab - i, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            token = v[j] > top ? i + j : token;
            top = fmaxf(top, v[j]);
        }
        if (HELD) {
            *reinterpret_cast<f4 *>(held + i) = f4{v[0], v[1], v[2], v[3]};
            *reinterpret_cast<f4 *>(held + i + 4) = f4{v[4], v[5], v[6], v[7]};
        }
    }
    auto eight = [&](int32_t i, float *v) {
        if (HELD) {
            const f4 lo = *reinterpret_cast<const f4 *>(held + i), hi = *reinterpret_cast<const f4 *>(held + i + 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[j] = lo[j];
                v[j + 4] = hi[j];
            }
        } else {
            load_logits(l + i, a.vocab - i, v);
        }
    };
    auto walk = [&](auto f) {  // f(logit, token) for every token that is on
#pragma unroll 1
        for (int32_t i = t * 8; i < a.vocab; i += kThreads * 8) {
            float v[8];
            eight(i, v);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (v[j] > -INFINITY)
                    f(v[j], i + j);
        }
    };
    auto list = [&](auto test) {  // appends the keys of the tokens that are on and pass
#pragma unroll 1
        for (int32_t i0 = 0; i0 < a.vocab; i0 += kThreads * 8) {
            const int32_t i = i0 + t * 8;
            uint32_t hits = 0;
            float v[8];
            if (i < a.vocab) {
                eight(i, v);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    hits |= static_cast<uint32_t>(v[j] > -INFINITY && test(v[j], i + j)) << j;
            }
            if (__any(hits)) {
                uint32_t at = place_in(&sh.count, __popc(hits));
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (hits >> j & 1) {
                        if (at < kFew)
                            sh.few[at] = key_of(v[j], i + j);
                        ++at;
                    }
            }
        }
    };
    const uint64_t own = top > -INFINITY ? key_of(top, token) : 0, best = most_block<kWaves>(own, sh.part);
    if (best == 0 || r.mode == kGreedy) {
        if (t == 0)
            a.ids[row] = best == 0 ? -1 : token_of(best);
        return;
    }
    const float most = logit_of(best);
    if (HELD && r.mode == kFewKept) {
        // the k-th largest of the threads' largest keys bounds the k-th largest key from below;
        // where that lets too many through (or k is more than the threads), the tokens themselves do
#pragma unroll 1
        for (int all = r.top_k > kThreads / 2; all < 2; ++all) {
            if (t == 0)
                sh.count = 0;
            clear(sh.bins, kBins);
            if (all)
                walk([&](float v, int32_t) { atomicAdd(&sh.bins[bin_of(v, most)], Sum(1)); });
            else if (own)
                atomicAdd(&sh.bins[bin_of(top, most)], Sum(1));
            __syncthreads();
            const Found f = find(sh, sh.bins, r.top_k, 1.0);
            if (f.upto > kFew)
                break;
            list([&](float v, int32_t) { return bin_of(v, most) >= f.bin; });
            __syncthreads();
            const int32_t m = static_cast<int32_t>(sh.count);
            if (m <= kFew) {
                pick_few(a, row, r, m, most, sh);
                return;
            }
            __syncthreads();
        }
    }
    uint64_t least = 0;  // of the keys that are kept
#pragma unroll 1
    for (int filter = 0; filter < 2; ++filter) {
        const bool share = filter == 1;
        if (share ? r.top_p >= 1 : r.top_k >= a.vocab)
            continue;
        const uint64_t border = border_of(
            sh, most, r.top_k, share ? r.top_p : 1.0,
            [&](auto f) {
                walk([&](float v, int32_t i) {
                    if (key_of(v, i) >= least)
                        f(v, i);
                });
            },
            [&](auto test) { list([&](float v, int32_t i) { return key_of(v, i) >= least && test(v, i); }); },
            [&](uint64_t key) { return share ? units(weight_of(logit_of(key), most, r), r) : Sum(1); });
        least = border > least ? border : least;
    }
    auto kept = [&](float v, int32_t i) -> Sum {
        const Sum w = last_weight(v, most, r);
        return v > -INFINITY && key_of(v, i) >= least ? w : 0;
    };
    Sum sum = 0;
#pragma unroll 1
    for (int32_t i = t * 8; i < a.vocab; i += kThreads * 8) {
        float v[8];
        eight(i, v);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            sum += kept(v[j], i + j);
    }
    const double border = r.u * static_cast<double>(sum_block<kWaves>(sum, sh.part));
    pick(a, row, 0, a.vocab, 0, border, sh, [&](int32_t i) {
        return kept(HELD ? held[i] : counted(static_cast<float>(l[i])), i);
    });
}

// Rows that LDS holds.  What bounds it are the steps, one after the other: some microseconds a
// row, 512 rows at a time (62 KB of LDS and 79 registers: two workgroups a compute unit).
template <typename T>
__global__ void __launch_bounds__(kThreads) sample_short(SampleArgs a) {
    __shared__ OneRow sh;
    __shared__ __attribute__((aligned(16))) float held[kChunk];
    whole_row<T, true>(a, blockIdx.x, row_of(a, blockIdx.x), sh, held);
}

// A: a chunk a workgroup, thread t's segment: 8 tokens from 8 t, 2048 + 8 t, 4096 + 8 t and 6144 + 8 t on.
template <typename T>
__global__ void __launch_bounds__(kSegments) sample_chunks(SampleArgs a) {
    __shared__ Sum part[kSegments / 64];
    const int32_t row = blockIdx.y, chunk = blockIdx.x, chunks = gridDim.x;
    const T *l = static_cast<const T *>(a.logits) + row * a.ld;
    const Space s = space_of(a, row);
    float v[4][8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int32_t i = chunk * kChunk + j * 2048 + static_cast<int32_t>(threadIdx.x) * 8;
        load_logits(l + i, a.vocab - i, v[j]);
    }
    const Row r = row_of(a, row);
    if (r.mode == kShare || r.mode == kCount) {
        for (int b = chunk * kSegments + threadIdx.x; b < kBins; b += chunks * kSegments)
            s.bins[b] = 0;
        if (chunk == 0 && threadIdx.x == 0)
            *s.count = 0;
    }
    float top = -INFINITY;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            top = fmaxf(top, v[j][i]);
    int32_t token = 0;  // the first of that value
#pragma unroll
    for (int j = 3; j >= 0; --j)
#pragma unroll
        for (int i = 7; i >= 0; --i)
            token = v[j][i] == top ? j * 2048 + i : token;
    const uint64_t own = top > -INFINITY ? key_of(top, chunk * kChunk + static_cast<int32_t>(threadIdx.x) * 8 + token) : 0;
    s.segments[chunk * kSegments + threadIdx.x] = own;
    const uint64_t best = most_block<kSegments / 64>(own, part);
    if (threadIdx.x == 0)
        s.best[chunk] = best;
    if (r.mode != kAll)
        return;
    Sum sum = 0;
    if (best) {
        const float most = logit_of(best);
#pragma unroll 1
        for (int j = 0; j < 4; ++j) {  // moves, as registers take no index (A of 256 x 50001 23.5 us, reading again 25.6)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const Sum u = units(weight_of(v[0][e], most, r), r);
                sum += v[0][e] > -INFINITY ? u : 0;
                v[0][e] = v[1][e];
                v[1][e] = v[2][e];
                v[2][e] = v[3][e];
            }
        }
    }
    sum = sum_block<kSegments / 64>(sum, part);
    if (threadIdx.x == 0)
        s.sums[chunk] = sum;
}

// A chunk's logits, as they count: 8 neighbours of each piece of 4096.
constexpr int kPieces = kChunk / kThreads / 8;
template <typename T>
__device__ __forceinline__ void load_chunk(const SampleArgs &a, int32_t row, int32_t chunk, float (&v)[kPieces][8]) {
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
        const int32_t i = chunk * kChunk + (j * kThreads + static_cast<int32_t>(threadIdx.x)) * 8;
        load_logits(static_cast<const T *>(a.logits) + row * a.ld + i, a.vocab - i, v[j]);
    }
}

template <typename T>
__device__ __forceinline__ void hold(const SampleArgs &a, int32_t row, int32_t chunk, float *held) {
    float v[kPieces][8];
    load_chunk<T>(a, row, chunk, v);
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
        f4 *to = reinterpret_cast<f4 *>(held) + (j * kThreads + threadIdx.x) * 2;
        to[0] = f4{v[j][0], v[j][1], v[j][2], v[j][3]};
        to[1] = f4{v[j][4], v[j][5], v[j][6], v[j][7]};
    }
    __syncthreads();
}

// The first token of a row that kept(logit, token) keeps, for u = 0.
template <typename T, class Kept>
__device__ __forceinline__ void pick_first(const SampleArgs &a, int32_t row, int32_t chunks, Shared &sh, Kept kept) {
#pragma unroll 1
    for (int32_t c = 0; c < chunks; ++c) {
        hold<T>(a, row, c, sh.held);
        uint64_t first = 0;  // the smaller the token, the larger
#pragma unroll 1
        for (int32_t i = threadIdx.x; i < kChunk && !first; i += kThreads)
            first = kept(sh.held[i], c * kChunk + i) ? kMostTokens - (c * kChunk + i) : 0;
        first = most_block<kWaves>(first, sh.part);
        if (first) {
            if (threadIdx.x == 0)
                a.ids[row] = kMostTokens - static_cast<int32_t>(first);
            return;
        }
    }
}

// The token from the chunks' sums of kept weights, in units of the row's largest.
template <typename T, class Kept>
__device__ __forceinline__ void pick_by_sums(const SampleArgs &a, int32_t row, const Row &r, const Sum *sums, int32_t chunks,
                                             Shared &sh, Kept kept) {
    if (r.u == 0) {
        pick_first<T>(a, row, chunks, sh, kept);
        return;
    }
    Sum total = 0, before = 0;
    for (int c = 0; c < chunks; ++c)
        total += sums[c];
    const double border = r.u * static_cast<double>(total);
    int32_t chunk = 0;
    while (chunk < chunks - 1 && !(static_cast<double>(before + sums[chunk]) > border))
        before += sums[chunk++];
    hold<T>(a, row, chunk, sh.held);
    pick(a, row, chunk * kChunk, kChunk, before, border, sh, [&](int32_t i) { return kept(sh.held[i - chunk * kChunk], i); });
}

// Rows without a filter: chunks' sums are in units of their own largest weight.
template <typename T>
__device__ __forceinline__ void pick_all(const SampleArgs &a, int32_t row, const Row &r, const Space &s, int32_t chunks, float most,
                                         Shared &sh) {
    if (r.u == 0) {
        pick_first<T>(a, row, chunks, sh, [&](float v, int32_t) { return v > -INFINITY && weighs(v, most, r); });
        return;
    }
    double *mass = sh.mass, *factor = sh.factor;
    if (threadIdx.x < static_cast<unsigned>(chunks)) {
        const uint64_t best = s.best[threadIdx.x];
        const double f = best ? weight_of(logit_of(best), most, r) * 0x1p-42 : 0.0;
        factor[threadIdx.x] = f;
        mass[threadIdx.x] = best ? f * static_cast<double>(s.sums[threadIdx.x]) : 0.0;
    }
    __syncthreads();
    double total = 0, before = 0;
    int32_t chunk = 0, last = 0;
    for (int c = 0; c < chunks; ++c) {
        total += mass[c];
        last = mass[c] > 0 ? c : last;
    }
    const double border = r.u * total;
    while (chunk < last && !(before + mass[chunk] > border))
        before += mass[chunk++];
    // rounding may leave nothing above the border in the last chunk: then its last token
    const double own = static_cast<double>(s.sums[chunk]);
    const double rest = fmin((border - before) / factor[chunk], own * (1 - 0x1p-52));
    const float top = logit_of(s.best[chunk]);
    hold<T>(a, row, chunk, sh.held);
    pick(a, row, chunk * kChunk, kChunk, 0, rest, sh, [&](int32_t i) -> Sum {
        const float v = sh.held[i - chunk * kChunk];
        const Sum w = units(weight_of(v, top, r), r);
        return v > -INFINITY ? w : 0;
    });
}

// Up to 1024 tokens kept: the segments that can hold them, and their tokens.
template <typename T>
__device__ __forceinline__ void pick_segments(const SampleArgs &a, int32_t row, const Row &r, const Space &s, int32_t chunks, Shared &sh) {
    const int32_t segments = chunks * kSegments, t = static_cast<int32_t>(threadIdx.x);
    uint64_t head[8];  // of the first 4096 segments, asked for before the maximum is known
    auto eight = [&](int32_t g0, uint64_t (&k)[8]) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            k[j] = g0 + t + j * kThreads < segments ? s.segments[g0 + t + j * kThreads] : 0;
    };
    eight(0, head);
    auto eights = [&](auto f) {  // f(eight keys, the first one's segment) by all threads as often; kThreads from one to the next
        f(head, t);
#pragma unroll 1
        for (int32_t g0 = kThreads * 8; g0 < segments; g0 += kThreads * 8) {
            uint64_t k[8];
            eight(g0, k);
            f(k, g0 + t);
        }
    };
    auto keys = [&](auto f) {  // f(key) for every segment that has a token
        eights([&](const uint64_t (&k)[8], int32_t) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (k[j])
                    f(k[j]);
        });
    };
    const uint64_t best = best_of(s, chunks);
    if (best == 0) {
        if (t == 0)
            a.ids[row] = -1;
        return;
    }
    const float most = logit_of(best);
    clear(sh.bins, kBins);
    keys([&](uint64_t k) { atomicAdd(&sh.bins[bin_of(logit_of(k), most)], Sum(1)); });
    __syncthreads();
    const Found f = find(sh, sh.bins, r.top_k, 1.0);
    uint64_t least = 0;  // with fewer segments that have a token than k
    int bin = f.bin;
    if (f.bin >= 0 && f.upto > kFew) {  // more than 1024 up to the end of that bin
        bin = -1;
        least = least_key(sh, r.top_k, 0, 32 + kIndexBits, kFew, [&](auto g) {
            keys([&](uint64_t k) { g(k, Sum(1)); });
        });
    }
    // whether a token that is on, or a segment's largest, is above the bound: by its distance's bits, as bin_of
    uint32_t end = end_of(bin);
    auto in_bound = [&](uint64_t key, float l) {
        return __float_as_uint(most - l) < end && (least == 0 || key >= least);
    };
    uint32_t *ids = sh.rank;  // (until the list is sorted)
    if (threadIdx.x == 0)
        sh.count = 0;
    __syncthreads();
    eights([&](const uint64_t (&k)[8], int32_t g) {
        uint32_t hits = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            hits |= static_cast<uint32_t>(k[j] && in_bound(k[j], logit_of(k[j]))) << j;
        uint32_t at = place_in(&sh.count, __popc(hits));
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (hits >> j & 1)
                ids[at++] = g + j * kThreads;
    });
    __syncthreads();
    const int32_t few = static_cast<int32_t>(sh.count);
    // f(logits, first tokens) for four pieces of 8 of these segments at once, all threads as often: their
    // loads are under way together, and one place in the list is asked for (64 x 131072, k = 500: 27.1 us
    // with a place for each piece and for each of a thread's segments)
    auto walk = [&](auto f) {
#pragma unroll 1
        for (int32_t q = 0; q < few * 4; q += kThreads * 4) {
            float v[4][8];
            int32_t at[4];
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                const int32_t e = q + p * kThreads + static_cast<int32_t>(threadIdx.x);
                const int32_t g = e < few * 4 ? static_cast<int32_t>(ids[e >> 2]) : 0;
                at[p] = g / kSegments * kChunk + (e & 3) * 2048 + g % kSegments * 8;
                load_logits(static_cast<const T *>(a.logits) + row * a.ld + at[p], e < few * 4 ? a.vocab - at[p] : 0, v[p]);
            }
            f(v, at, few * 4 - q);
        }
    };
    auto every = [&](auto f) {
        walk([&](const float (&v)[4][8], const int32_t (&at)[4], int32_t) {
#pragma unroll
            for (int j = 0; j < 32; ++j)
                if (v[j / 8][j % 8] > -INFINITY)
                    f(v[j / 8][j % 8], at[j / 8] + j % 8);
        });
    };
    auto list = [&] {
        __syncthreads();
        if (threadIdx.x == 0)
            sh.count = 0;
        __syncthreads();
        walk([&](const float (&v)[4][8], const int32_t (&at)[4], int32_t left) {
            uint32_t hits = 0;
#pragma unroll
            for (int p = 0; p < 4; ++p)
                if (p * kThreads < left) {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        hits |= static_cast<uint32_t>(v[p][j] > -INFINITY && in_bound(key_of(v[p][j], at[p] + j), v[p][j])) << (p * 8 + j);
                }
            uint32_t to = place_in(&sh.count, __popc(hits));
#pragma unroll
            for (int p = 0; p < 4; ++p)
                if (p * kThreads < left) {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (hits >> (p * 8 + j) & 1) {
                            if (to < kFew)
                                sh.few[to] = key_of(v[p][j], at[p] + j);
                            ++to;
                        }
                }
        });
        __syncthreads();
    };
    list();
    if (sh.count > kFew) {  // of up to 32768 tokens: the same bound from them
        clear(sh.bins, kBins);
        every([&](float v, int32_t i) {
            if (key_of(v, i) >= least)
                atomicAdd(&sh.bins[bin_of(v, most)], Sum(1));
        });
        __syncthreads();
        const Found t = find(sh, sh.bins, r.top_k, 1.0);
        end = end_of(t.upto > kFew ? -1 : t.bin);
        if (t.upto > kFew) {
            least = least_key(sh, r.top_k, 0, 32 + kIndexBits, kFew, [&](auto g) {
                every([&](float v, int32_t i) { g(key_of(v, i), Sum(1)); });
            });
        }
        list();
    }
    pick_few(a, row, r, static_cast<int32_t>(sh.count), most, sh);
}

// B
template <typename T>
__global__ void __launch_bounds__(kThreads) sample_sums(SampleArgs a) {
    __shared__ Shared sh;
    const int32_t row = blockIdx.y, chunk = blockIdx.x, chunks = gridDim.x;
    const Row r = row_of(a, row);
    if (r.mode != kLeast && r.mode != kShare && r.mode != kCount)
        return;
    const Space s = space_of(a, row);
    const uint64_t best = best_of(s, chunks);
    if (best == 0)
        return;
    const float most = logit_of(best);
    float v[kPieces][8];
    load_chunk<T>(a, row, chunk, v);
    clear(sh.bins, kBins);
    Sum sum = 0;
#pragma unroll
    for (int j = 0; j < kPieces; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const double w = weight_of(v[j][e], most, r);
            const Sum u = r.mode == kCount ? Sum(1) : units(w, r);
            if (v[j][e] > -INFINITY && u) {
                if (r.mode != kLeast)
                    atomicAdd(&sh.bins[bin_of(v[j][e], most)], u);
                else if (w >= r.min_p)
                    sum += u;
            }
        }
    if (r.mode == kLeast) {
        sum = sum_block<kWaves>(sum, sh.part);
        if (threadIdx.x == 0)
            s.sums[chunk] = sum;
        return;
    }
    __syncthreads();
    for (int b = threadIdx.x; b < kBins; b += kThreads)
        if (const Sum w = sh.bins[b])
            atomicAdd(&s.bins[b], w);
}

// C
template <typename T>
__global__ void __launch_bounds__(kThreads) sample_lists(SampleArgs a) {
    __shared__ Shared sh;
    const int32_t row = blockIdx.y, chunk = blockIdx.x, chunks = gridDim.x;
    const Row r = row_of(a, row);
    if (r.mode != kShare && r.mode != kCount)
        return;
    const Space s = space_of(a, row);
    const uint64_t best = best_of(s, chunks);
    if (best == 0)
        return;
    const float most = logit_of(best);
    float v[kPieces][8];
    load_chunk<T>(a, row, chunk, v);
    const Found f = find(sh, s.bins, r.top_k, r.top_p);
    // of this thread's tokens those in the bin and above it: by their distance's bits, as bin_of
    const uint32_t end = end_of(f.bin), begin = f.bin < kBins - 1 ? end_of(f.bin + 1) : 0;
    uint32_t hits = 0, over = 0;
#pragma unroll
    for (int j = 0; j < kPieces; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t d = __float_as_uint(most - v[j][e]);
            const bool on = v[j][e] > -INFINITY;  // (two that are on may be infinitely far from each other)
            hits |= static_cast<uint32_t>(on && d < end) << (j * 8 + e);
            over |= static_cast<uint32_t>(on && d < begin) << (j * 8 + e);
        }
    hits ^= over;
    const Sum own = static_cast<Sum>(__popc(over)) << 32 | __popc(hits);
    Sum both;
    const Sum counts = sum_block<kWaves>(own, sh.part, &both);
    // the ones above it side by side, so that wavefronts are full of them (64 x 131072: p = 0.9 18.4
    // us before, k = 5000 16.8)
    int32_t to = static_cast<int32_t>((both - own) >> 32);
#pragma unroll
    for (int j = 0; j < kPieces; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (over >> (j * 8 + e) & 1)
                sh.held[to++] = v[j][e];
    __syncthreads();
    Sum sum = 0;
#pragma unroll 1
    for (int32_t i = threadIdx.x; i < static_cast<int32_t>(counts >> 32); i += kThreads) {
        const double w = weight_of(sh.held[i], most, r);
        sum += w >= r.min_p ? units(w, r) : 0;
    }
    sum = sum_block<kWaves>(sum, sh.part);
    if (threadIdx.x == 0)
        s.sums[chunk] = sum;
    const uint32_t mine = __popc(hits), run = static_cast<uint32_t>(both), all = static_cast<uint32_t>(counts);
    if (threadIdx.x == 0)
        sh.count = all ? atomicAdd(s.count, all) : 0;
    __syncthreads();
    uint32_t at = sh.count + run - mine;
    for (; hits; hits &= hits - 1) {  // few: read again, as registers take no index
        const int bit = __builtin_ctz(hits);
        const int32_t i = chunk * kChunk + (bit / 8 * kThreads + static_cast<int32_t>(threadIdx.x)) * 8 + bit % 8;
        if (at < kList)
            s.list[at] = key_of(counted(static_cast<float>(static_cast<const T *>(a.logits)[row * a.ld + i])), i);
        ++at;
    }
}

// D, a workgroup a row
template <typename T>
__global__ void __launch_bounds__(kThreads) sample_tokens(SampleArgs a) {
    __shared__ Shared sh;
    const int32_t row = blockIdx.x, chunks = chunks_of(a.vocab);
    const Row r = row_of(a, row);
    const Space s = space_of(a, row);
    if (r.mode == kFewKept) {
        pick_segments<T>(a, row, r, s, chunks, sh);
        return;
    }
    const uint64_t best = best_of(s, chunks);
    if (best == 0 || r.mode == kGreedy) {
        if (threadIdx.x == 0)
            a.ids[row] = best == 0 ? -1 : token_of(best);
        return;
    }
    if (r.mode == kAll) {
        pick_all<T>(a, row, r, s, chunks, logit_of(best), sh);
        return;
    }
    const uint32_t listed = r.mode == kShare || r.mode == kCount ? *s.count : 0;
    if (r.mode == kDigits || listed > kList) {
        whole_row<T, false>(a, row, r, sh, nullptr);
        return;
    }
    const float most = logit_of(best);
    uint64_t least = 0;
    auto kept = [&](float l, int32_t token) -> Sum {
        const Sum w = last_weight(l, most, r);
        return l > -INFINITY && key_of(l, token) >= least ? w : 0;
    };
    if (r.mode == kLeast) {
        pick_by_sums<T>(a, row, r, s.sums, chunks, sh, kept);
        return;
    }
    const Found f = find(sh, s.bins, r.top_k, r.top_p);
    const int32_t m = static_cast<int32_t>(listed);
    if (f.bin >= 0) {
        const double target = f.target - static_cast<double>(f.above);
        auto weight = [&](uint64_t key) { return r.mode == kCount ? Sum(1) : units(weight_of(logit_of(key), most, r), r); };
        if (m <= kFew) {
            for (int32_t e = threadIdx.x; e < m; e += kThreads)
                sh.few[e] = s.list[e];
            __syncthreads();
            least = border_of_few(sh, m, target, false, weight);
        } else {
            uint64_t low = ~uint64_t(0), high = 0;
            for (int32_t e = threadIdx.x; e < m; e += kThreads) {
                const uint64_t k = s.list[e];
                low = k < low ? k : low;
                high = k > high ? k : high;
            }
            low = ~most_block<kWaves>(~low, sh.part);
            high = most_block<kWaves>(high, sh.part);
            const int shift = 64 - __builtin_clzll(low ^ high);  // keys differ
            least = least_key(sh, target, high >> shift, shift, 0, [&](auto g) {
                for (int32_t e = threadIdx.x; e < m; e += kThreads)
                    g(s.list[e], weight(s.list[e]));
            });
            least = least > low ? least : low;
        }
    }
    Sum *sums = sh.sums;
    for (int32_t c = threadIdx.x; c < chunks; c += kThreads)
        sums[c] = s.sums[c];
    __syncthreads();
    for (int32_t e = threadIdx.x; e < m; e += kThreads) {
        const uint64_t k = s.list[e];
        const int32_t token = token_of(k);
        if (const Sum w = kept(logit_of(k), token))
            atomicAdd(&sums[token / kChunk], w);
    }
    __syncthreads();
    pick_by_sums<T>(a, row, r, sums, chunks, sh, kept);
}

// Most rows of a slice, which has the workspace for itself, one slice after the other: 0.7 to 3 GB of
// it, where a part for every row was 90 GB for 2^20 rows of 8193 tokens.  Calls without a histogram have
// smaller parts, hence slices of more rows.  Measured in bf16, all rows at once in brackets: 32768 x 8200
// with p = 0.9 2317 us (2370), t = 0 267 (271); 9000 x 32000 1142 (1126), 150 (162).  With 4096 rows a
// slice 6000 x 8200 with p = 0.9 took 438 (421).
constexpr int32_t kSlice = 8192;
constexpr int32_t kMostRows = 32768;  // a grid's second axis ends at 65535

template <typename T>
hipError_t launch(const SampleArgs &a, hipStream_t stream) {
    const int32_t chunks = chunks_of(a.vocab);
    if (chunks == 1) {
        sample_short<T><<<a.n, kThreads, 0, stream>>>(a);
        return hipGetLastError();
    }
    // rows that need no sums over all: a small k, t = 0, no filter
    const bool few = !a.top_ks && a.top_k > 0 && few_kept(a.top_k, !a.top_ps && a.top_p < 1);
    const bool greedy = !a.temperatures && !(a.temperature > 0);
    const bool all = !a.top_ks && (a.top_k == 0 || a.top_k >= a.vocab) && !a.top_ps && a.top_p >= 1 && !a.min_ps && !(a.min_p > 0);
    const bool some = a.top_ks || (a.top_k > 0 && a.top_k < a.vocab), share = a.top_ps || a.top_p < 1;
    const bool bins = !few && !greedy && (some || share);
    const int64_t space = std::min(a.n, kSlice) * row_words(a.vocab), words = bins ? row_words(a.vocab) : chunk_words(a.vocab);
    const int32_t slice = static_cast<int32_t>(std::min<int64_t>(space / words, kMostRows));
    for (int32_t row = 0; row < a.n; row += slice) {
        SampleArgs part = a;
        const int32_t rows = std::min(a.n - row, slice);
        part.logits = static_cast<const T *>(a.logits) + row * a.ld;
        part.u += row;
        part.ids += row;
        part.temperatures = a.temperatures ? a.temperatures + row : nullptr;
        part.top_ks = a.top_ks ? a.top_ks + row : nullptr;
        part.top_ps = a.top_ps ? a.top_ps + row : nullptr;
        part.min_ps = a.min_ps ? a.min_ps + row : nullptr;
        part.words = words;
        const dim3 grid(chunks, rows);
        sample_chunks<T><<<grid, kSegments, 0, stream>>>(part);
        if (!few && !greedy && !all) {
            sample_sums<T><<<grid, kThreads, 0, stream>>>(part);
            sample_lists<T><<<grid, kThreads, 0, stream>>>(part);
        }
        sample_tokens<T><<<rows, kThreads, 0, stream>>>(part);
    }
    return hipGetLastError();
}

}  // namespace

int64_t sample_workspace(int32_t n, int32_t vocab) {
    return chunks_of(vocab) == 1 ? 0 : std::min(n, kSlice) * row_words(vocab) * 8;
}

hipError_t launch_sample(const SampleArgs &a, int32_t type, hipStream_t stream) {
    return type == kF32   ? launch<float>(a, stream)
           : type == kF16 ? launch<_Float16>(a, stream)
                          : launch<__bf16>(a, stream);
}

}  // namespace spconv
