// Checks of arguments that the files of the C ABI share.
#pragma once

#include <cstdint>
#include <limits>

#include "status.hpp"

namespace spconv {

inline bool is_float(int32_t type) { return type == SPCONV_F32 || type == SPCONV_F16 || type == SPCONV_BF16; }
inline int64_t size_of(int32_t type) { return type == SPCONV_F32 ? 4 : type == SPCONV_FP8 ? 1 : 2; }
inline bool aligned(const void *p, int64_t to) { return reinterpret_cast<uintptr_t>(p) % static_cast<uintptr_t>(to) == 0; }

struct Range {
    const void *p;
    int64_t bytes;
};

inline bool overlap(Range a, Range b) {
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.p), b0 = reinterpret_cast<uintptr_t>(b.p);
    return a.p && b.p && a.bytes > 0 && b.bytes > 0 && a0 < b0 + static_cast<uintptr_t>(b.bytes) &&
           b0 < a0 + static_cast<uintptr_t>(a.bytes);
}

// Whether an output overlaps an input or another output.
template <int OUT, int IN>
inline bool outputs_overlap(const Range (&out)[OUT], const Range (&in)[IN]) {
    for (int i = 0; i < OUT; ++i) {
        for (int j = 0; j < i; ++j)
            if (overlap(out[i], out[j]))
                return true;
        for (int j = 0; j < IN; ++j)
            if (overlap(out[i], in[j]))
                return true;
    }
    return false;
}

// Bytes that strided rows span; the caller keeps the product in range.
inline int64_t span(int64_t rows, int64_t cols, int64_t ld, int64_t size) { return rows ? ((rows - 1) * ld + cols) * size : 0; }
constexpr int64_t kMostStride = int64_t(1) << 34;

inline int64_t align16(int64_t v) { return (v + 15) / 16 * 16; }

inline void clamp_of(spconv_act act, float &lo, float &hi) {
    lo = act == SPCONV_ACT_NONE ? -std::numeric_limits<float>::infinity() : 0.0f;
    hi = act == SPCONV_ACT_RELU6 ? 6.0f : std::numeric_limits<float>::infinity();
}

inline spconv_status launched(hipError_t e) { return e == hipSuccess ? SPCONV_OK : spconv::set_hip_error("kernel launch", e); }

}  // namespace spconv
