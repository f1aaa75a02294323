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
// The order is that of one whole number a token: 32 bits of l, then 20 of the
// index from behind.  So every filter is a least key, found digit by digit
// from histograms of the keys with the digits above in common: of counts for k,
// of weights for p.  Weights are whole multiples of 2^-42 there and in the final
// sums (2^20 tokens stay below 2^62): sums are exact in any order, which makes
// the atomics that collect them harmless, and next to a border the choice is the
// definition's but for the roundings of 2^-43 (2e-11 of the largest weight's size
// over 2^17 tokens).  Exponentials are 64-bit.
#include "fp8.hpp"
#include "serve_ops.hpp"

namespace spconv {
namespace {

typedef unsigned long long Sum;

constexpr float kMostLogit = 3.402823466e38f;
constexpr double kUnit = 4398046511104.0;  // 2^42
constexpr int kIndexBits = 20;
constexpr int kBins = 2048;
constexpr int kThreads = 1024;

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

// A row's parameters, as they count.
struct Row {
    double inverse;  // 1 / temperature
    double top_p, min_p, u;
    int32_t top_k;
    bool greedy;
};

__device__ __forceinline__ Row row_of(const SampleArgs &a, int32_t row) {
    const float t = a.temperatures ? a.temperatures[row] : a.temperature;
    const float p = a.top_ps ? a.top_ps[row] : a.top_p, least = a.min_ps ? a.min_ps[row] : a.min_p;
    const float u = a.u[row];
    Row r;
    r.greedy = !(t > 0);
    r.inverse = 1.0 / static_cast<double>(t);
    r.top_k = a.top_ks ? a.top_ks[row] : a.top_k;
    if (r.top_k <= 0 || r.top_k > a.vocab)
        r.top_k = a.vocab;
    r.top_p = p < 1 ? p : 1.0;  // a NaN is off, as 1 is
    r.min_p = least > 0 ? fminf(least, 1.0f) : 0.0;
    r.u = u > 0 ? fminf(u, 0x1.fffffep-1f) : 0.0;
    return r;
}

__device__ __forceinline__ double weight_of(float l, float most, double inverse) {
    return exp((static_cast<double>(l) - static_cast<double>(most)) * inverse);
}
__device__ __forceinline__ Sum units(double w) { return static_cast<Sum>(__double2ull_rn(w * kUnit)); }

template <typename V>
__device__ __forceinline__ V sum_all(V v) {
#pragma unroll
    for (int s = 1; s < 64; s *= 2)
        v += __shfl_xor(v, s);
    return v;
}

struct Found {
    int bin;
    Sum above, total;  // of the bins above the found one, of all
};

// The first bin from above at which the running sum reaches `least` (and is not empty).
__device__ __forceinline__ Found find(const Sum *bins, double least, Sum *part, Found *out) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int b0 = kBins - 2 - 2 * static_cast<int>(threadIdx.x);  // this thread's two bins, from above
    const Sum hi = bins[b0 + 1], lo = bins[b0];
    Sum run = hi + lo;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
        const Sum v = __shfl_up(run, s);
        run += lane >= s ? v : 0;
    }
    if (lane == 63)
        part[wave] = run;
    __syncthreads();
    Sum total = 0, before = 0;
    for (int w = 0; w < kThreads / 64; ++w) {
        before += w < wave ? part[w] : 0;
        total += part[w];
    }
    run += before;  // up to and with this thread's bins
    const Sum upto = run - lo, above = upto - hi;
    auto reaches = [&](Sum v) { return static_cast<double>(v) >= least; };
    if (hi && reaches(upto) && !(above && reaches(above)))
        *out = {b0 + 1, above, total};
    if (lo && reaches(run) && !(upto && reaches(upto)))
        *out = {b0, upto, total};
    __syncthreads();
    return *out;
}

// One workgroup a row, the row read anew for each step.
template <typename T>
__global__ void __launch_bounds__(kThreads) sample_row(SampleArgs a) {
    __shared__ Sum bins[kBins];
    __shared__ Sum part[kThreads / 64];
    __shared__ Found found;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int32_t row = blockIdx.x;
    const T *l = static_cast<const T *>(a.logits) + row * a.ld;
    const Row r = row_of(a, row);
    uint64_t best = 0;
    for (int32_t i = threadIdx.x; i < a.vocab; i += kThreads) {
        const float v = counted(static_cast<float>(l[i]));
        const uint64_t k = key_of(v, i);
        best = v > -INFINITY && k > best ? k : best;
    }
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
        const uint64_t k = __shfl_xor(best, s);
        best = k > best ? k : best;
    }
    if (lane == 0)
        part[wave] = best;
    __syncthreads();
    for (int w = 0; w < kThreads / 64; ++w)
        best = part[w] > best ? part[w] : best;
    if (best == 0 || r.greedy) {
        if (threadIdx.x == 0)
            a.ids[row] = best == 0 ? -1 : token_of(best);
        return;
    }
    const float most = logit_of(best);
    uint64_t least = 0;  // of the keys that are kept
    for (int filter = 0; filter < 2; ++filter) {
        const bool by_weight = filter == 1;
        if (by_weight ? r.top_p >= 1 : r.top_k >= a.vocab)
            continue;
        double target = r.top_k;
        uint64_t prefix = 0;
        int shift = 52;
        for (int digit = 0; digit < 5; ++digit) {
            const int width = digit < 2 ? 11 : digit == 2 ? 10 : 10;
            for (int b = threadIdx.x; b < kBins; b += kThreads)
                bins[b] = 0;
            __syncthreads();
            const int to = shift - width;
            for (int32_t i = threadIdx.x; i < a.vocab; i += kThreads) {
                const float v = counted(static_cast<float>(l[i]));
                const uint64_t k = key_of(v, i);
                if (v > -INFINITY && k >= least && k >> shift == prefix)
                    atomicAdd(&bins[k >> to & ((1 << width) - 1)],
                              by_weight ? units(weight_of(v, most, r.inverse)) : Sum(1));
            }
            __syncthreads();
            if (threadIdx.x == 0)
                found = {-1, 0, 0};
            __syncthreads();
            if (digit == 0 && by_weight) {  // the share is one of the whole sum
                Sum total = 0;
                for (int b = threadIdx.x; b < kBins; b += kThreads)
                    total += bins[b];
                total = sum_all(total);
                if (lane == 0)
                    part[wave] = total;
                __syncthreads();
                total = 0;
                for (int w = 0; w < kThreads / 64; ++w)
                    total += part[w];
                target = r.top_p * static_cast<double>(total);
                __syncthreads();
            }
            const Found f = find(bins, target, part, &found);
            if (f.bin < 0) {  // fewer tokens are on than k: all are kept
                prefix = 0;
                shift = 0;
                break;
            }
            target -= static_cast<double>(f.above);
            prefix = prefix << width | static_cast<uint64_t>(f.bin);
            shift = to;
            __syncthreads();
        }
        least = prefix > least ? prefix : least;
    }
    // sums of 8192 neighbouring tokens, then of each thread's eight in the one that holds the border
    constexpr int kSlab = 8 * kThreads;
    const bool zero = r.u == 0;  // the first kept token, however small
    auto kept = [&](int32_t i) -> Sum {
        if (i >= a.vocab)
            return 0;
        const float v = counted(static_cast<float>(l[i]));
        if (!(v > -INFINITY) || key_of(v, i) < least)
            return 0;
        const double w = weight_of(v, most, r.inverse);
        if (w < r.min_p)
            return 0;
        return zero ? w > 0 : units(w);
    };
    const int slabs = (a.vocab + kSlab - 1) / kSlab;
    for (int s = threadIdx.x; s < slabs; s += kThreads)
        bins[s] = 0;
    __syncthreads();
    auto eight = [&](int s) {
        Sum v = 0;
        for (int j = 0; j < 8; ++j)
            v += kept(s * kSlab + static_cast<int32_t>(threadIdx.x) * 8 + j);
        return v;
    };
    for (int s = 0; s < slabs; ++s) {
        const Sum v = sum_all(eight(s));
        if (lane == 0 && v)
            atomicAdd(&bins[s], v);
    }
    __syncthreads();
    Sum total = 0, before = 0;
    for (int s = 0; s < slabs; ++s)
        total += bins[s];
    const double border = r.u * static_cast<double>(total);
    int slab = 0;
    while (slab < slabs - 1 && !(static_cast<double>(before + bins[slab]) > border))
        before += bins[slab++];
    const Sum own = eight(slab);
    Sum run = own;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
        const Sum v = __shfl_up(run, s);
        run += lane >= s ? v : 0;
    }
    if (lane == 63)
        part[wave] = run;
    __syncthreads();
    for (int w = 0; w < wave; ++w)
        before += part[w];
    run += before;
    if (static_cast<double>(run) > border && !(static_cast<double>(run - own) > border)) {
        Sum at = run - own;
        int32_t token = slab * kSlab + static_cast<int32_t>(threadIdx.x) * 8;
        for (int j = 0; j < 7; ++j, ++token) {
            at += kept(token);
            if (static_cast<double>(at) > border)
                break;
        }
        a.ids[row] = token;
    }
}

}  // namespace

int64_t sample_workspace(int32_t, int32_t, int32_t) { return 0; }

hipError_t launch_sample(const SampleArgs &a, int32_t type, hipStream_t stream) {
    if (type == kF32)
        sample_row<float><<<a.n, kThreads, 0, stream>>>(a);
    else if (type == kF16)
        sample_row<_Float16><<<a.n, kThreads, 0, stream>>>(a);
    else
        sample_row<__bf16><<<a.n, kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace spconv
