// C ABI of the 8-bit products, the router and the experts (declared in
// include/spconv.h): argument checks, then asynchronous launches on the
// caller's stream.  Nothing is allocated and nothing synchronizes.
#include "spconv.h"

#include <hip/hip_runtime_api.h>

#include <limits>
#include <type_traits>

#include "expert_ops.hpp"
#include "status.hpp"

namespace {

using spconv::blocks_of;
using spconv::set_error;

constexpr int64_t kMostBlocks = int64_t(1) << 27;  // row blocks of a matrix: launches stay below 2^32 threads
constexpr int64_t kMostOutputs = int64_t(1) << 36;
constexpr int32_t kMostChannels = 1 << 22;          // a tile of 256 rows lies within 32-bit offsets
constexpr int64_t kMostExpertBlocks = int64_t(1) << 25;  // rows by token and by pair lie within 32-bit offsets

bool is_float(int32_t type) { return type == SPCONV_F32 || type == SPCONV_F16 || type == SPCONV_BF16; }
int64_t size_of(int32_t type) { return type == SPCONV_F32 ? 4 : type == SPCONV_FP8 ? 1 : 2; }
bool aligned(const void *p, int64_t to) { return reinterpret_cast<uintptr_t>(p) % static_cast<uintptr_t>(to) == 0; }

struct Range {
    const void *p;
    int64_t bytes;
};

bool overlap(Range a, Range b) {
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.p), b0 = reinterpret_cast<uintptr_t>(b.p);
    return a.p && b.p && a.bytes > 0 && b.bytes > 0 && a0 < b0 + static_cast<uintptr_t>(b.bytes) &&
           b0 < a0 + static_cast<uintptr_t>(a.bytes);
}

// Whether an output overlaps an input or another output.
template <int OUT, int IN>
bool outputs_overlap(const Range (&out)[OUT], const Range (&in)[IN]) {
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
int64_t span(int64_t rows, int64_t cols, int64_t ld, int64_t size) { return rows ? ((rows - 1) * ld + cols) * size : 0; }
constexpr int64_t kMostStride = int64_t(1) << 34;

int64_t code_bytes(int64_t rows, int64_t cols) { return rows * blocks_of(cols) * 128; }
int64_t align16(int64_t v) { return (v + 15) / 16 * 16; }

void clamp_of(spconv_act act, float &lo, float &hi) {
    lo = act == SPCONV_ACT_NONE ? -std::numeric_limits<float>::infinity() : 0.0f;
    hi = act == SPCONV_ACT_RELU6 ? 6.0f : std::numeric_limits<float>::infinity();
}

spconv_status launched(hipError_t e) { return e == hipSuccess ? SPCONV_OK : spconv::set_hip_error("kernel launch", e); }

// Sizes of a linear layer; SPCONV_OK also where there is nothing to do.
spconv_status check_linear(spconv_dtype x_dtype, int32_t n, int32_t cin, int32_t cout) {
    if (!is_float(x_dtype) && x_dtype != SPCONV_FP8)
        return set_error(SPCONV_E_ARG, "x_dtype must be SPCONV_F32, _F16, _BF16 or _FP8");
    if (n < 0 || cin < 0 || cout < 0)
        return set_error(SPCONV_E_ARG, "n, cin and cout must be >= 0");
    if (n == 0 || cout == 0)
        return SPCONV_OK;
    if (cin == 0)
        return set_error(SPCONV_E_SHAPE, "cin must be >= 1");
    if (cin > kMostChannels || cout > kMostChannels)
        return set_error(SPCONV_E_SHAPE, "cin and cout must be at most 2^22");
    if (static_cast<int64_t>(n) * blocks_of(cin) >= kMostBlocks)
        return set_error(SPCONV_E_SHAPE, "n * ceil(cin / 128) must be below 2^27");
    if (static_cast<int64_t>(n) * cout >= kMostOutputs)
        return set_error(SPCONV_E_SHAPE, "n * cout must be below 2^36");
    return SPCONV_OK;
}

// A call's workspace: rows that the product's kernel does not quantise itself, as codes and
// scales, then the sums of workgroups that share the input channels.
struct LinearSpace {
    int64_t rows, sums;
};
LinearSpace linear_workspace(spconv_dtype x_dtype, int32_t n, int32_t cin, int32_t cout) {
    if (n == 0 || cout == 0)
        return {0, 0};
    const bool as_is = x_dtype == SPCONV_FP8 || spconv::linear_takes_rows(n, cin, cout);
    const int64_t splits = spconv::linear_splits(n, cin, cout), cells = static_cast<int64_t>(n) * ((cout + 3) / 4 * 4);
    return {as_is ? 0 : code_bytes(n, cin) + align16(static_cast<int64_t>(n) * blocks_of(cin) * 4),
            splits > 1 ? splits * cells * 4 : 0};
}

constexpr int32_t kMostExpertChannels = 32768;

spconv_status check_experts(int32_t n, int32_t k, int32_t experts, int32_t hidden, int32_t inner) {
    if (n < 0 || k < 1)
        return set_error(SPCONV_E_ARG, "n must be >= 0 and k >= 1");
    if (experts < 1 || hidden < 1 || inner < 1)
        return set_error(SPCONV_E_SHAPE, "experts, hidden and inner must be >= 1");
    if (experts > spconv::kMostExperts || k > spconv::kMostChoices)
        return set_error(SPCONV_E_UNSUPPORTED, "at most 1024 experts and k = 64 are supported");
    if (hidden > kMostExpertChannels || inner > kMostExpertChannels)
        return set_error(SPCONV_E_UNSUPPORTED, "hidden and inner must be at most 32768");
    if (static_cast<int64_t>(n) * k * blocks_of(hidden > inner ? hidden : inner) >= kMostExpertBlocks)
        return set_error(SPCONV_E_SHAPE, "n * k * ceil(channels / 128) must be below 2^25");
    return SPCONV_OK;
}

// Lays the workspace of a call out from `base` (null: only counts) and returns its size.
int64_t experts_layout(spconv::ExpertArgs &a, uint8_t *base) {
    int64_t at = 0;
    auto take = [&](auto &p, int64_t bytes) {
        p = base ? reinterpret_cast<std::remove_reference_t<decltype(p)>>(base + at) : nullptr;
        at += (bytes + 255) / 256 * 256;  // codes on whole 128-byte lines: else a product reads two for one
    };
    const int64_t pairs = a.pairs;
    if (spconv::experts_by_token(a.n, a.k, a.experts, a.hidden, a.inner)) {
        take(a.h, pairs * a.inner * 4);
        return at;
    }
    take(a.order, pairs * 4);
    take(a.place, pairs * 4);
    take(a.offsets, (a.experts + 1) * int64_t(4));
    take(a.xq, code_bytes(a.n, a.hidden));
    take(a.xs, static_cast<int64_t>(a.n) * a.hb * 4);
    take(a.hq, code_bytes(pairs, a.inner));
    take(a.hs, pairs * a.ib * 4);
    take(a.z, pairs * a.hidden * 4);
    take(a.zs, pairs * a.hb * 4);
    return at;
}

spconv::ExpertArgs expert_sizes(int32_t n, int32_t k, int32_t experts, int32_t hidden, int32_t inner) {
    spconv::ExpertArgs a{};
    a.n = n;
    a.k = k;
    a.pairs = n * k;
    a.experts = experts;
    a.hidden = hidden;
    a.inner = inner;
    a.hb = blocks_of(hidden);
    a.ib = blocks_of(inner);
    return a;
}

}  // namespace

extern "C" {

spconv_status spconv_quantize_fp8(const void *x, spconv_dtype dtype, int64_t ldx, int32_t rows, int32_t cols,
                                  int32_t block_rows, void *q, float *scale, void *stream) {
    spconv::clear_error();
    if (!is_float(dtype))
        return set_error(SPCONV_E_ARG, "dtype must be SPCONV_F32, _F16 or _BF16");
    if (rows < 0 || cols < 0)
        return set_error(SPCONV_E_ARG, "rows and cols must be >= 0");
    if (block_rows != 1 && block_rows != 128)
        return set_error(SPCONV_E_UNSUPPORTED, "block_rows must be 1 or 128");
    if (rows == 0 || cols == 0)
        return SPCONV_OK;
    if (!x || !q || !scale)
        return set_error(SPCONV_E_ARG, "x, q or scale is NULL");
    if (ldx < cols)
        return set_error(SPCONV_E_ARG, "ldx must be at least cols");
    const int64_t kb = blocks_of(cols);
    if (cols > (1 << 30) || ldx > kMostStride || rows * kb >= kMostBlocks)
        return set_error(SPCONV_E_SHAPE, "rows * ceil(cols / 128) must be below 2^27, cols at most 2^30, ldx at most 2^34");
    if (!aligned(x, size_of(dtype)) || !aligned(scale, 4) || !aligned(q, 16))
        return set_error(SPCONV_E_ARG, "x and scale must be aligned to their element size, q to 16 bytes");
    const Range in[] = {{x, span(rows, cols, ldx, size_of(dtype))}};
    const Range out[] = {{q, code_bytes(rows, cols)}, {scale, (block_rows == 1 ? rows : blocks_of(rows)) * kb * 4}};
    if (outputs_overlap(out, in))
        return set_error(SPCONV_E_ARG, "x, q and scale must not overlap");
    const hipStream_t s = static_cast<hipStream_t>(stream);
    uint8_t *codes = static_cast<uint8_t *>(q);
    return launched(block_rows == 1 ? spconv::launch_quantize_rows(x, dtype, ldx, rows, cols, codes, scale, s)
                                    : spconv::launch_quantize_blocks(x, dtype, ldx, rows, cols, codes, scale, s));
}

spconv_status spconv_linear_fp8_workspace(spconv_dtype x_dtype, int32_t n, int32_t cin, int32_t cout, int64_t *bytes) {
    spconv::clear_error();
    if (!bytes)
        return set_error(SPCONV_E_ARG, "bytes is NULL");
    *bytes = 0;
    const spconv_status st = check_linear(x_dtype, n, cin, cout);
    if (st == SPCONV_OK) {
        const LinearSpace space = linear_workspace(x_dtype, n, cin, cout);
        *bytes = space.rows + space.sums;
    }
    return st;
}

spconv_status spconv_linear_fp8(const void *x, spconv_dtype x_dtype, int64_t ldx, const float *x_scale, const void *w,
                                const float *w_scale, const float *bias, spconv_act act, void *y, spconv_dtype y_dtype,
                                int32_t n, int32_t cin, int32_t cout, void *workspace, int64_t workspace_bytes,
                                void *stream) {
    spconv::clear_error();
    const spconv_status st = check_linear(x_dtype, n, cin, cout);
    if (st != SPCONV_OK)
        return st;
    if (!is_float(y_dtype))
        return set_error(SPCONV_E_ARG, "y_dtype must be SPCONV_F32, _F16 or _BF16");
    if (act < SPCONV_ACT_NONE || act > SPCONV_ACT_RELU6)
        return set_error(SPCONV_E_ARG, "act must be SPCONV_ACT_NONE, _RELU or _RELU6");
    if (n == 0 || cout == 0)
        return SPCONV_OK;
    if (!x || !w || !w_scale || !y)
        return set_error(SPCONV_E_ARG, "x, w, w_scale or y is NULL");
    const bool codes = x_dtype == SPCONV_FP8;
    if (codes != (x_scale != nullptr))
        return set_error(SPCONV_E_ARG, "x_scale belongs to SPCONV_FP8 rows, and to them only");
    if (!codes && ldx < cin)
        return set_error(SPCONV_E_ARG, "ldx must be at least cin");
    if (!codes && ldx > kMostStride)
        return set_error(SPCONV_E_SHAPE, "ldx must be at most 2^34");
    if (!aligned(x, codes ? 16 : size_of(x_dtype)) || !aligned(w, 16) || !aligned(y, size_of(y_dtype)) ||
        !aligned(x_scale, 4) || !aligned(w_scale, 4) || !aligned(bias, 4) || !aligned(workspace, 16))
        return set_error(SPCONV_E_ARG, "pointers must be aligned to their element size, codes and the workspace to 16 bytes");
    const LinearSpace space = linear_workspace(x_dtype, n, cin, cout);
    const int64_t kb = blocks_of(cin), need = space.rows + space.sums;
    if (need > 0 && (!workspace || workspace_bytes < need))
        return set_error(SPCONV_E_ARG, "the workspace is smaller than spconv_linear_fp8_workspace says");
    const Range in[] = {{x, codes ? code_bytes(n, cin) : span(n, cin, ldx, size_of(x_dtype))},
                        {x_scale, kb * n * 4},
                        {w, code_bytes(cout, cin)},
                        {w_scale, blocks_of(cout) * kb * 4},
                        {bias, static_cast<int64_t>(cout) * 4}};
    const Range out[] = {{y, static_cast<int64_t>(n) * cout * size_of(y_dtype)}, {workspace, need}};
    if (outputs_overlap(out, in))
        return set_error(SPCONV_E_ARG, "y and the workspace must not overlap each other or an input");
    const hipStream_t s = static_cast<hipStream_t>(stream);
    spconv::LinearArgs a{};
    a.x = x;
    a.ldx = ldx;
    a.xs = x_scale;
    a.w = static_cast<const uint8_t *>(w);
    a.ws = w_scale;
    a.bias = bias;
    a.y = y;
    a.x_type = x_dtype;
    a.y_type = y_dtype;
    a.n = n;
    a.cin = cin;
    a.cout = cout;
    a.kb = static_cast<int32_t>(kb);
    clamp_of(act, a.lo, a.hi);
    a.partial = reinterpret_cast<float *>(static_cast<uint8_t *>(workspace) + space.rows);
    if (space.rows > 0) {
        uint8_t *q = static_cast<uint8_t *>(workspace);
        float *scale = reinterpret_cast<float *>(q + code_bytes(n, cin));
        const hipError_t e = spconv::launch_quantize_rows(x, x_dtype, ldx, n, cin, q, scale, s);
        if (e != hipSuccess)
            return launched(e);
        a.x = q;
        a.xs = scale;
        a.x_type = spconv::kFp8;
    }
    return launched(spconv::launch_linear_fp8(a, s));
}

spconv_status spconv_route(const void *logits, spconv_dtype dtype, int64_t ld, const float *bias, spconv_score score,
                           int32_t n, int32_t experts, int32_t groups, int32_t groups_kept, int32_t group_top,
                           int32_t k, int32_t renorm, float factor, int32_t *ids, float *weights, void *stream) {
    spconv::clear_error();
    if (!is_float(dtype))
        return set_error(SPCONV_E_ARG, "dtype must be SPCONV_F32, _F16 or _BF16");
    if (score != SPCONV_SCORE_SOFTMAX && score != SPCONV_SCORE_SIGMOID)
        return set_error(SPCONV_E_ARG, "score must be SPCONV_SCORE_SOFTMAX or _SIGMOID");
    if (n < 0 || experts < 1 || k < 1)
        return set_error(SPCONV_E_ARG, "n must be >= 0, experts and k >= 1");
    if (groups < 1 || groups_kept < 1 || groups_kept > groups)
        return set_error(SPCONV_E_ARG, "groups must be >= 1 and groups_kept in [1, groups]");
    if (experts % groups != 0 || k > experts)
        return set_error(SPCONV_E_SHAPE, "experts must be a multiple of groups and k at most experts");
    if (experts > spconv::kMostExperts || groups > 64 || k > spconv::kMostChoices || group_top < 1 || group_top > 2)
        return set_error(SPCONV_E_UNSUPPORTED, "at most 1024 experts, 64 groups and k = 64, and group_top 1 or 2");
    if (n >= 1 << 25)
        return set_error(SPCONV_E_SHAPE, "n must be below 2^25");
    if (n == 0)
        return SPCONV_OK;
    if (!logits || !ids || !weights)
        return set_error(SPCONV_E_ARG, "logits, ids or weights is NULL");
    if (ld < experts)
        return set_error(SPCONV_E_ARG, "ld must be at least experts");
    if (ld > kMostStride)
        return set_error(SPCONV_E_SHAPE, "ld must be at most 2^34");
    if (!aligned(logits, size_of(dtype)) || !aligned(bias, 4) || !aligned(ids, 4) || !aligned(weights, 4))
        return set_error(SPCONV_E_ARG, "pointers must be aligned to their element size");
    const int64_t places = static_cast<int64_t>(n) * k * 4;
    const Range in[] = {{logits, span(n, experts, ld, size_of(dtype))}, {bias, experts * int64_t(4)}};
    const Range out[] = {{ids, places}, {weights, places}};
    if (outputs_overlap(out, in))
        return set_error(SPCONV_E_ARG, "ids and weights must not overlap each other or an input");
    spconv::RouteArgs a{};
    a.logits = logits;
    a.ld = ld;
    a.bias = bias;
    a.ids = ids;
    a.weights = weights;
    a.n = n;
    a.experts = experts;
    a.k = k;
    a.groups = groups;
    a.groups_kept = groups_kept;
    a.group_top = group_top;
    a.softmax = score == SPCONV_SCORE_SOFTMAX;
    a.renorm = renorm != 0;
    a.factor = factor;
    return launched(spconv::launch_route(a, dtype, static_cast<hipStream_t>(stream)));
}

spconv_status spconv_experts_fp8_workspace(int32_t n, int32_t k, int32_t experts, int32_t hidden, int32_t inner,
                                           int64_t *bytes) {
    spconv::clear_error();
    if (!bytes)
        return set_error(SPCONV_E_ARG, "bytes is NULL");
    *bytes = 0;
    const spconv_status st = check_experts(n, k, experts, hidden, inner);
    if (st != SPCONV_OK || n == 0)
        return st;
    spconv::ExpertArgs a = expert_sizes(n, k, experts, hidden, inner);
    *bytes = experts_layout(a, nullptr);
    return SPCONV_OK;
}

spconv_status spconv_experts_fp8(const void *x, spconv_dtype dtype, int64_t ldx, const int32_t *ids,
                                 const float *weights, const void *w13, const float *w13_scale, const void *w2,
                                 const float *w2_scale, void *y, int32_t n, int32_t k, int32_t experts, int32_t hidden,
                                 int32_t inner, void *workspace, int64_t workspace_bytes, void *stream) {
    spconv::clear_error();
    if (!is_float(dtype))
        return set_error(SPCONV_E_ARG, "dtype must be SPCONV_F32, _F16 or _BF16");
    const spconv_status st = check_experts(n, k, experts, hidden, inner);
    if (st != SPCONV_OK || n == 0)
        return st;
    if (!x || !ids || !weights || !w13 || !w13_scale || !w2 || !w2_scale || !y || !workspace)
        return set_error(SPCONV_E_ARG, "a pointer is NULL");
    if (ldx < hidden)
        return set_error(SPCONV_E_ARG, "ldx must be at least hidden");
    if (ldx > kMostStride)
        return set_error(SPCONV_E_SHAPE, "ldx must be at most 2^34");
    const int64_t size = size_of(dtype);
    if (!aligned(x, size) || !aligned(y, size) || !aligned(ids, 4) || !aligned(weights, 4) || !aligned(w13, 16) ||
        !aligned(w13_scale, 4) || !aligned(w2, 16) || !aligned(w2_scale, 4) || !aligned(workspace, 16))
        return set_error(SPCONV_E_ARG, "pointers must be aligned to their element size, codes and the workspace to 16 bytes");
    spconv::ExpertArgs a = expert_sizes(n, k, experts, hidden, inner);
    const int64_t need = experts_layout(a, static_cast<uint8_t *>(workspace));
    if (workspace_bytes < need)
        return set_error(SPCONV_E_ARG, "the workspace is smaller than spconv_experts_fp8_workspace says");
    const int64_t scales = static_cast<int64_t>(experts) * a.hb * a.ib * 4;
    const Range in[] = {{x, span(n, hidden, ldx, size)},
                        {ids, a.pairs * int64_t(4)},
                        {weights, a.pairs * int64_t(4)},
                        {w13, experts * 2 * code_bytes(inner, hidden)},
                        {w13_scale, 2 * scales},
                        {w2, experts * code_bytes(hidden, inner)},
                        {w2_scale, scales}};
    const Range out[] = {{y, static_cast<int64_t>(n) * hidden * size}, {workspace, need}};
    if (outputs_overlap(out, in))
        return set_error(SPCONV_E_ARG, "y and the workspace must not overlap each other or an input");
    a.x = x;
    a.ldx = ldx;
    a.type = dtype;
    a.ids = ids;
    a.weights = weights;
    a.w13 = static_cast<const uint8_t *>(w13);
    a.s13 = w13_scale;
    a.w2 = static_cast<const uint8_t *>(w2);
    a.s2 = w2_scale;
    a.y = y;
    return launched(spconv::launch_experts(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
