// The experts of each token.
//
// Routing: s = softmax(l) or 1 / (1 + exp(-l)) over a token's logits, value =
// s + bias; experts in equal groups, a group's rank is the sum of its one or
// two largest values; the best k values of the best groups, ties to the lowest
// index, and the chosen s, divided by their sum where asked, times a factor.
// Scores and values are 64-bit: neither the rounding of exp nor the order of
// the softmax's sum then decides between two experts that are nearly tied, so
// that every program that follows the definition chooses the same ones.
#include <algorithm>

#include "expert_ops.hpp"
#include "fp8.hpp"

namespace spconv {
namespace {

// A 64-bit value as a whole number of the same order; 0 is below every value.
__device__ __forceinline__ uint64_t key_of(double v) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    return b >> 63 ? ~b : b | uint64_t(1) << 63;
}
__device__ __forceinline__ double value_of(uint64_t key) {
    return __builtin_bit_cast(double, key >> 63 ? key & ~(uint64_t(1) << 63) : ~key);
}

__device__ __forceinline__ uint32_t dpp_max(uint32_t v) {
#define SPCONV_STEP(ctrl, rows) \
    v = max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), ctrl, rows, 0xf, false)))
    SPCONV_STEP(0x111, 0xf);  // row_shr:1, 2, 4, 8
    SPCONV_STEP(0x112, 0xf);
    SPCONV_STEP(0x114, 0xf);
    SPCONV_STEP(0x118, 0xf);
    SPCONV_STEP(0x142, 0xa);  // row_bcast:15, 31
    SPCONV_STEP(0x143, 0xc);
#undef SPCONV_STEP
    return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(v), 63));
}

__device__ __forceinline__ double sum_lanes(double v, int lanes) {
    for (int s = 1; s < lanes; s *= 2)
        v += __shfl_xor(v, s);
    return v;
}

// 1 / v for v from 1 to infinity, to the last place or two.
__device__ __forceinline__ double inverse(double v) {
    double r = __builtin_amdgcn_rcp(v);
    r = fma(fma(-v, r, 1.0), r, r);
    return v < INFINITY ? fma(fma(-v, r, 1.0), r, r) : 0.0;
}

// A lane's keys in descending order; equal ones stay in the order of their
// experts, since only neighbours are exchanged.
template <int PER>
__device__ __forceinline__ void sort_keys(uint64_t (&key)[PER], int32_t (&id)[PER]) {
#pragma unroll
    for (int last = PER - 1; last > 0; --last)
#pragma unroll
        for (int i = 0; i < last; ++i) {
            const bool swap = key[i] < key[i + 1];
            const uint64_t k = swap ? key[i] : key[i + 1];
            const int32_t e = swap ? id[i] : id[i + 1];
            key[i] = swap ? key[i + 1] : key[i];
            id[i] = swap ? id[i + 1] : id[i];
            key[i + 1] = k;
            id[i + 1] = e;
        }
}

// A wavefront a token; a lane holds PER neighbouring experts, so that the
// lowest lane of a tie holds the lowest expert.  What bounds it is the count of
// instructions (16384 x 256 logits, 16.8 MB, 8 groups of 32, k = 8: 23 us
// against 3.7 for the bytes; 714 a wavefront, 19 us at the rate of issue): a
// 64-bit exponential for each logit, then for each choice a maximum over the
// lanes.  Each lane sorts its keys once, so that a choice looks at one key a
// lane, compares the upper 32 bits first, and only the winner's lane moves its
// next key up.
// lds: a wavefront's scores, and its keys where groups do not fall on whole lanes.
template <typename T, int PER>
__global__ void __launch_bounds__(256) route_kernel(RouteArgs a, bool wide) {
    extern __shared__ __attribute__((aligned(16))) uint64_t lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t token = blockIdx.x * 4 + wave;
    const int32_t e0 = lane * PER;
    if (token >= a.n)
        return;
    const T *l = static_cast<const T *>(a.logits) + token * a.ld + e0;
    float v[PER];
    if (wide && e0 + PER <= a.experts) {
        struct __attribute__((aligned(sizeof(T) * PER > 16 ? 16 : sizeof(T) * PER))) Piece {
            T v[PER];
        } p = *reinterpret_cast<const Piece *>(l);
#pragma unroll
        for (int i = 0; i < PER; ++i)
            v[i] = static_cast<float>(p.v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < PER; ++i)
            v[i] = e0 + i < a.experts ? static_cast<float>(l[i]) : -INFINITY;
    }
    double score[PER];
    if (a.softmax) {
        float most = -INFINITY;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            v[i] = fminf(v[i] != v[i] ? -INFINITY : v[i], 3.402823466e38f);
            most = fmaxf(most, v[i]);
        }
#pragma unroll
        for (int s = 1; s < 64; s *= 2)
            most = fmaxf(most, __shfl_xor(most, s));
        double sum = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            score[i] = v[i] > -INFINITY ? exp(static_cast<double>(v[i]) - static_cast<double>(most)) : 0.0;
            sum += score[i];
        }
        sum = sum_lanes(sum, 64);
#pragma unroll
        for (int i = 0; i < PER; ++i)
            score[i] = score[i] / sum;
    } else {
#pragma unroll
        for (int i = 0; i < PER; ++i)
            score[i] = inverse(1.0 + exp(-static_cast<double>(v[i])));
    }
    double *scores = reinterpret_cast<double *>(lds) + wave * PER * 64;
    uint64_t key[PER];
    int32_t id[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        scores[e0 + i] = score[i];
        const double bias = a.bias && e0 + i < a.experts ? static_cast<double>(a.bias[e0 + i]) : 0.0;
        // a value that is not a number (from the bias) counts as off, too
        const double value = score[i] + bias;
        key[i] = v[i] > -INFINITY && value > -INFINITY ? key_of(value) : 0;
        id[i] = e0 + i;
    }
    sort_keys(key, id);
    if (a.groups > 1) {
        // A group is looked through by `lanes` lanes.  Where its experts fill
        // whole lanes (whole_lanes), they are its own; else its keys come from LDS.
        const int lanes = a.group_lanes, g = lane / lanes, first = lane % lanes;
        uint64_t best = 0, next = 0;
        if (a.whole_lanes) {
            best = key[0];
            next = PER > 1 ? key[1 % PER] : 0;
        } else {
            uint64_t *mine = lds + (4 + wave) * PER * 64;
#pragma unroll
            for (int i = 0; i < PER; ++i)
                mine[id[i]] = key[i];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (g < a.groups)
                for (int i = first; i < a.each; i += lanes) {
                    const uint64_t k = mine[g * a.each + i];
                    next = max(next, min(best, k));
                    best = max(best, k);
                }
        }
        for (int s = 1; s < lanes; s *= 2) {
            const uint64_t b = __shfl_xor(best, s), m = __shfl_xor(next, s);
            next = max(max(next, m), min(best, b));
            best = max(best, b);
        }
        uint64_t rank = 0;
        if (best)
            rank = key_of(value_of(best) + (a.group_top > 1 && next ? value_of(next) : 0.0));
        int ahead = 0;  // groups that come before this lane's
        for (int o = 0; o < a.groups; ++o) {
            const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(rank), o * lanes);
            const uint32_t hi = __builtin_amdgcn_readlane(static_cast<int>(rank >> 32), o * lanes);
            const uint64_t r = static_cast<uint64_t>(hi) << 32 | lo;
            ahead += r > rank || (r == rank && o < g);
        }
        const bool stays = g < a.groups && ahead < a.groups_kept;
        if (a.whole_lanes) {
            key[0] = stays ? key[0] : 0;  // nothing below a lane's first key is looked at before it
        } else {
            const uint64_t kept = __ballot(stays && first == 0);
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const uint32_t of = static_cast<uint32_t>(id[i]) * a.each_inverse >> 20;
                key[i] = kept >> (of * lanes & 63) & 1 ? key[i] : 0;
            }
            sort_keys(key, id);
        }
    }
    int32_t chosen = -1;
    for (int j = 0; j < a.k; ++j) {
        const uint32_t mine = static_cast<uint32_t>(key[0] >> 32);
        const uint32_t hi = dpp_max(mine);
        if (hi == 0)  // no key of a value has an empty upper half
            break;
        uint64_t holders = __ballot(mine == hi);
        if (holders & (holders - 1)) {
            const uint32_t low = mine == hi ? static_cast<uint32_t>(key[0]) : 0;
            const uint32_t lo = dpp_max(low);
            holders = __ballot(mine == hi && low == lo);
        }
        const int winner = __ffsll(static_cast<unsigned long long>(holders)) - 1;
        const int32_t which = __builtin_amdgcn_readlane(id[0], winner);
        chosen = lane == j ? which : chosen;
        if (lane == winner) {
#pragma unroll
            for (int i = 0; i + 1 < PER; ++i) {
                key[i] = key[i + 1];
                id[i] = id[i + 1];
            }
            key[PER - 1] = 0;
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    double weight = lane < a.k && chosen >= 0 ? scores[chosen] : 0.0;
    if (a.renorm) {
        const double sum = sum_lanes(weight, a.k);
        weight = sum > 0 ? weight / sum : 0.0;
    }
    if (lane < a.k) {
        const int64_t to = static_cast<int64_t>(token) * a.k + lane;
        a.ids[to] = chosen;
        a.weights[to] = static_cast<float>(weight * static_cast<double>(a.factor));
    }
}

template <typename T, int PER>
hipError_t route_per(RouteArgs a, hipStream_t stream) {
    // groups of a power of two of whole lanes; else as many lanes as fit, a power of two
    const int32_t lanes = a.each / PER;
    a.whole_lanes = a.each % PER == 0 && (lanes & (lanes - 1)) == 0;
    a.group_lanes = a.whole_lanes ? lanes : 1;
    while (!a.whole_lanes && a.group_lanes * 2 * a.groups <= 64)
        a.group_lanes *= 2;
    const int64_t piece = static_cast<int64_t>(sizeof(T)) * PER;
    const bool wide = reinterpret_cast<uintptr_t>(a.logits) % std::min<int64_t>(piece, 16) == 0 &&
                      a.ld * static_cast<int64_t>(sizeof(T)) % std::min<int64_t>(piece, 16) == 0;
    const size_t lds = (a.groups > 1 && !a.whole_lanes ? 8 : 4) * PER * 64 * 8;
    route_kernel<T, PER><<<(a.n + 3) / 4, 256, lds, stream>>>(a, wide);
    return hipGetLastError();
}

template <typename T>
hipError_t route_of(const RouteArgs &a, hipStream_t stream) {
    return a.experts <= 64    ? route_per<T, 1>(a, stream)
           : a.experts <= 128 ? route_per<T, 2>(a, stream)
           : a.experts <= 256 ? route_per<T, 4>(a, stream)
           : a.experts <= 512 ? route_per<T, 8>(a, stream)
                              : route_per<T, 16>(a, stream);
}

}  // namespace

hipError_t launch_route(RouteArgs a, int32_t type, hipStream_t stream) {
    a.each = a.experts / a.groups;
    a.each_inverse = ((1u << 20) + a.each - 1) / a.each;  // e * this >> 20 = e / each below 1024
    return type == kF32 ? route_of<float>(a, stream)
           : type == kF16 ? route_of<_Float16>(a, stream)
                          : route_of<__bf16>(a, stream);
}

}  // namespace spconv
