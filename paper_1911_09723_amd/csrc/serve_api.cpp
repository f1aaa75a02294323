// C ABI of norms, 4-bit block products and sampling (declared in
// include/spconv.h): argument checks, then asynchronous launches on the
// caller's stream.  Nothing is allocated and nothing synchronizes.
#include "spconv.h"

#include <hip/hip_runtime_api.h>

#include "checks.hpp"
#include "serve_ops.hpp"

namespace {

using spconv::align16;
using spconv::aligned;
using spconv::blocks_of;
using spconv::clamp_of;
using spconv::is_float;
using spconv::kMostStride;
using spconv::launched;
using spconv::lines_of;
using spconv::outputs_overlap;
using spconv::Range;
using spconv::set_error;
using spconv::size_of;
using spconv::span;

constexpr int64_t kMostBlocks = int64_t(1) << 27;  // row blocks of a matrix and
constexpr int32_t kMostRows = 1 << 25;             // its rows: launches stay below 2^32 threads
constexpr int64_t kMostLines = int64_t(1) << 28;   // lines of a weight: their scales lie within 32-bit offsets
constexpr int64_t kMostOutputs = int64_t(1) << 36;
constexpr int32_t kMostChannels = 1 << 22;         // a tile of 256 rows lies within 32-bit offsets

int64_t code_bytes(int64_t rows, int64_t cols) { return rows * lines_of(cols) * 128; }
int64_t scale_bytes(int64_t rows, int64_t cols) { return rows * lines_of(cols) * 8; }

// Whether an output that may lie where an input does lies so: same address, stride and element size.
bool in_place(const void *out, int64_t ldo, int64_t size, const void *in, int64_t ldi, int64_t in_size) {
    return out == in && ldo == ldi && size == in_size;
}

spconv_status check_linear(spconv_dtype x_dtype, int32_t n, int32_t cin, int32_t cout) {
    if (!is_float(x_dtype) && x_dtype != SPCONV_MXFP4)
        return set_error(SPCONV_E_ARG, "x_dtype must be SPCONV_F32, _F16, _BF16 or _MXFP4");
    if (n < 0 || cin < 0 || cout < 0)
        return set_error(SPCONV_E_ARG, "n, cin and cout must be >= 0");
    if (n == 0 || cout == 0)
        return SPCONV_OK;
    if (cin == 0)
        return set_error(SPCONV_E_SHAPE, "cin must be >= 1");
    if (cin > kMostChannels || cout > kMostChannels)
        return set_error(SPCONV_E_SHAPE, "cin and cout must be at most 2^22");
    if (n >= kMostRows || static_cast<int64_t>(n) * lines_of(cin) >= kMostBlocks)
        return set_error(SPCONV_E_SHAPE, "n must be below 2^25, n * ceil(cin / 256) below 2^27");
    if (static_cast<int64_t>(cout) * lines_of(cin) >= kMostLines)
        return set_error(SPCONV_E_SHAPE, "cout * ceil(cin / 256) must be below 2^28");
    if (static_cast<int64_t>(n) * cout >= kMostOutputs)
        return set_error(SPCONV_E_SHAPE, "n * cout must be below 2^36");
    return SPCONV_OK;
}

// A call's workspace: the codes and scales of rows that the product's kernel does not
// quantise itself.
int64_t linear_workspace(spconv_dtype x_dtype, int32_t n, int32_t cin, int32_t cout) {
    if (n == 0 || cout == 0 || x_dtype == SPCONV_MXFP4 || spconv::linear4_takes_rows(n, cin, cout))
        return 0;
    return code_bytes(n, cin) + align16(scale_bytes(n, cin));
}

spconv_status check_sample(spconv_dtype dtype, int32_t n, int32_t vocab) {
    if (!is_float(dtype))
        return set_error(SPCONV_E_ARG, "dtype must be SPCONV_F32, _F16 or _BF16");
    if (n < 0 || vocab < 1)
        return set_error(SPCONV_E_ARG, "n must be >= 0 and vocab >= 1");
    if (vocab > spconv::kMostTokens)
        return set_error(SPCONV_E_UNSUPPORTED, "at most 2^20 tokens are supported");
    if (n >= 1 << 20)
        return set_error(SPCONV_E_SHAPE, "n must be below 2^20");
    return SPCONV_OK;
}

}  // namespace

extern "C" {

spconv_status spconv_rms_norm(const void *x, spconv_dtype dtype, int64_t ldx, const void *residual,
                              spconv_dtype residual_dtype, int64_t ldr, void *total, int64_t ldt, const void *gain,
                              spconv_dtype gain_dtype, float eps, void *y, spconv_dtype y_dtype, int64_t ldy, void *q,
                              float *scale, int32_t rows, int32_t cols, void *stream) {
    spconv::clear_error();
    if (!is_float(dtype))
        return set_error(SPCONV_E_ARG, "dtype must be SPCONV_F32, _F16 or _BF16");
    auto other = [&](int32_t type) { return type != dtype && type != SPCONV_F32; };
    if ((residual && !is_float(residual_dtype)) || (gain && !is_float(gain_dtype)) || (y && !is_float(y_dtype)))
        return set_error(SPCONV_E_ARG, "residual_dtype, gain_dtype and y_dtype must be SPCONV_F32, _F16 or _BF16");
    if ((residual && other(residual_dtype)) || (gain && other(gain_dtype)) || (y && other(y_dtype)))
        return set_error(SPCONV_E_UNSUPPORTED, "residual_dtype, gain_dtype and y_dtype must be dtype or SPCONV_F32");
    if (rows < 0 || cols < 0)
        return set_error(SPCONV_E_ARG, "rows and cols must be >= 0");
    if (!(eps >= 0) || eps > std::numeric_limits<float>::max())
        return set_error(SPCONV_E_ARG, "eps must be finite and >= 0");
    if (rows == 0 || cols == 0)
        return SPCONV_OK;
    if (!x || (!y && !q) || !q != !scale)
        return set_error(SPCONV_E_ARG, "x is NULL, neither y nor q is asked for, or q comes without scale");
    if (total && !residual)
        return set_error(SPCONV_E_ARG, "total is the sum with a residual");
    if (ldx < cols || (residual && ldr < cols) || (total && ldt < cols) || (y && ldy < cols))
        return set_error(SPCONV_E_ARG, "row strides must be at least cols");
    if (cols > (1 << 30) || rows >= kMostRows || rows * static_cast<int64_t>(blocks_of(cols)) >= kMostBlocks || ldx > kMostStride ||
        (residual && ldr > kMostStride) || (total && ldt > kMostStride) || (y && ldy > kMostStride))
        return set_error(SPCONV_E_SHAPE, "rows must be below 2^25, rows * ceil(cols / 128) below 2^27, cols at most 2^30, strides at most 2^34");
    const int64_t size = size_of(dtype), size_r = size_of(residual_dtype), size_y = size_of(y_dtype);
    const int64_t size_g = size_of(gain_dtype);
    if (!aligned(x, size) || (residual && !aligned(residual, size_r)) || (total && !aligned(total, size_r)) ||
        (gain && !aligned(gain, size_g)) || (y && !aligned(y, size_y)) || !aligned(scale, 4) || !aligned(q, 16))
        return set_error(SPCONV_E_ARG, "pointers must be aligned to their element size, q to 16 bytes");
    // total and y may each lie exactly where x or residual does
    const bool t_at_r = total && in_place(total, ldt, size_r, residual, ldr, size_r);
    const bool t_at_x = total && in_place(total, ldt, size_r, x, ldx, size);
    const bool y_at_r = y && in_place(y, ldy, size_y, residual, ldr, size_r);
    const bool y_at_x = y && in_place(y, ldy, size_y, x, ldx, size);
    const Range of_x{x, span(rows, cols, ldx, size)}, of_r{residual, residual ? span(rows, cols, ldr, size_r) : 0};
    const Range of_g{gain, gain ? cols * size_g : 0};
    const Range of_t{total, total ? span(rows, cols, ldt, size_r) : 0}, of_y{y, y ? span(rows, cols, ldy, size_y) : 0};
    const Range codes[] = {{q, q ? int64_t(rows) * blocks_of(cols) * 128 : 0},
                           {scale, scale ? int64_t(rows) * blocks_of(cols) * 4 : 0}};
    const Range all[] = {of_x, of_r, of_g, of_t, of_y}, gains[] = {of_g}, ys[] = {of_y};
    const Range t_out[] = {of_t}, y_out[] = {of_y}, xs[] = {of_x}, rs[] = {of_r};
    if (outputs_overlap(codes, all) || outputs_overlap(t_out, gains) || outputs_overlap(y_out, gains) ||
        outputs_overlap(t_out, ys) || (!t_at_x && outputs_overlap(t_out, xs)) || (!t_at_r && outputs_overlap(t_out, rs)) ||
        (!y_at_x && outputs_overlap(y_out, xs)) || (!y_at_r && outputs_overlap(y_out, rs)))
        return set_error(SPCONV_E_ARG, "outputs must not overlap, but for total or y exactly in the place of x or residual");
    spconv::NormArgs a{};
    a.x = x;
    a.residual = residual;
    a.gain = gain;
    a.total = total;
    a.y = y;
    a.q = static_cast<uint8_t *>(q);
    a.scale = scale;
    a.ldx = ldx;
    a.ldr = ldr;
    a.ldt = ldt;
    a.ldy = ldy;
    a.rows = rows;
    a.cols = cols;
    a.kb = blocks_of(cols);
    a.eps = eps;
    a.y32 = y_dtype == SPCONV_F32;
    return launched(spconv::launch_norm(a, dtype, residual_dtype == SPCONV_F32, !gain || gain_dtype == SPCONV_F32,
                                        static_cast<hipStream_t>(stream)));
}

spconv_status spconv_quantize_mxfp4(const void *x, spconv_dtype dtype, int64_t ldx, int32_t rows, int32_t cols, void *q,
                                    void *scale, void *stream) {
    spconv::clear_error();
    if (!is_float(dtype))
        return set_error(SPCONV_E_ARG, "dtype must be SPCONV_F32, _F16 or _BF16");
    if (rows < 0 || cols < 0)
        return set_error(SPCONV_E_ARG, "rows and cols must be >= 0");
    if (rows == 0 || cols == 0)
        return SPCONV_OK;
    if (!x || !q || !scale)
        return set_error(SPCONV_E_ARG, "x, q or scale is NULL");
    if (ldx < cols)
        return set_error(SPCONV_E_ARG, "ldx must be at least cols");
    if (cols > (1 << 30) || ldx > kMostStride || rows >= kMostRows || rows * static_cast<int64_t>(lines_of(cols)) >= kMostLines)
        return set_error(SPCONV_E_SHAPE, "rows must be below 2^25, rows * ceil(cols / 256) below 2^28, cols at most 2^30, ldx at most 2^34");
    if (!aligned(x, size_of(dtype)) || !aligned(q, 16) || !aligned(scale, 16))
        return set_error(SPCONV_E_ARG, "x must be aligned to its element size, q and scale to 16 bytes");
    const Range in[] = {{x, span(rows, cols, ldx, size_of(dtype))}};
    const Range out[] = {{q, code_bytes(rows, cols)}, {scale, scale_bytes(rows, cols)}};
    if (outputs_overlap(out, in))
        return set_error(SPCONV_E_ARG, "x, q and scale must not overlap");
    return launched(spconv::launch_quantize_mxfp4(x, dtype, ldx, rows, cols, static_cast<uint8_t *>(q),
                                                  static_cast<uint8_t *>(scale), static_cast<hipStream_t>(stream)));
}

spconv_status spconv_linear_mxfp4_workspace(spconv_dtype x_dtype, int32_t n, int32_t cin, int32_t cout, int64_t *bytes) {
    spconv::clear_error();
    if (!bytes)
        return set_error(SPCONV_E_ARG, "bytes is NULL");
    *bytes = 0;
    const spconv_status st = check_linear(x_dtype, n, cin, cout);
    if (st == SPCONV_OK)
        *bytes = linear_workspace(x_dtype, n, cin, cout);
    return st;
}

spconv_status spconv_linear_mxfp4(const void *x, spconv_dtype x_dtype, int64_t ldx, const void *x_scale, const void *w,
                                  const void *w_scale, const float *bias, spconv_act act, void *y,
                                  spconv_dtype y_dtype, int32_t n, int32_t cin, int32_t cout, void *workspace,
                                  int64_t workspace_bytes, void *stream) {
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
    const bool codes = x_dtype == SPCONV_MXFP4;
    if (codes != (x_scale != nullptr))
        return set_error(SPCONV_E_ARG, "x_scale belongs to SPCONV_MXFP4 rows, and to them only");
    if (!codes && ldx < cin)
        return set_error(SPCONV_E_ARG, "ldx must be at least cin");
    if (!codes && ldx > kMostStride)
        return set_error(SPCONV_E_SHAPE, "ldx must be at most 2^34");
    if (!aligned(x, codes ? 16 : size_of(x_dtype)) || !aligned(w, 16) || !aligned(y, size_of(y_dtype)) ||
        !aligned(x_scale, 16) || !aligned(w_scale, 16) || !aligned(bias, 4) || !aligned(workspace, 16))
        return set_error(SPCONV_E_ARG, "pointers must be aligned to their element size, codes, scales and the workspace to 16 bytes");
    const int64_t need = linear_workspace(x_dtype, n, cin, cout);
    if (need > 0 && (!workspace || workspace_bytes < need))
        return set_error(SPCONV_E_ARG, "the workspace is smaller than spconv_linear_mxfp4_workspace says");
    const Range in[] = {{x, codes ? code_bytes(n, cin) : span(n, cin, ldx, size_of(x_dtype))},
                        {x_scale, scale_bytes(n, cin)},
                        {w, code_bytes(cout, cin)},
                        {w_scale, scale_bytes(cout, cin)},
                        {bias, static_cast<int64_t>(cout) * 4}};
    const Range out[] = {{y, static_cast<int64_t>(n) * cout * size_of(y_dtype)}, {workspace, need}};
    if (outputs_overlap(out, in))
        return set_error(SPCONV_E_ARG, "y and the workspace must not overlap each other or an input");
    const hipStream_t s = static_cast<hipStream_t>(stream);
    spconv::Linear4Args a{};
    a.x = x;
    a.ldx = ldx;
    a.xs = static_cast<const uint8_t *>(x_scale);
    a.w = static_cast<const uint8_t *>(w);
    a.ws = static_cast<const uint8_t *>(w_scale);
    a.bias = bias;
    a.y = y;
    a.x_type = x_dtype;
    a.y_type = y_dtype;
    a.n = n;
    a.cin = cin;
    a.cout = cout;
    a.lines = lines_of(cin);
    clamp_of(act, a.lo, a.hi);
    if (need > 0) {
        uint8_t *q = static_cast<uint8_t *>(workspace), *scale = q + code_bytes(n, cin);
        const hipError_t e = spconv::launch_quantize_mxfp4(x, x_dtype, ldx, n, cin, q, scale, s);
        if (e != hipSuccess)
            return launched(e);
        a.x = q;
        a.xs = scale;
        a.x_type = SPCONV_MXFP4;
    }
    return launched(spconv::launch_linear_mxfp4(a, s));
}

spconv_status spconv_sample_workspace(spconv_dtype dtype, int32_t n, int32_t vocab, int64_t *bytes) {
    spconv::clear_error();
    if (!bytes)
        return set_error(SPCONV_E_ARG, "bytes is NULL");
    *bytes = 0;
    const spconv_status st = check_sample(dtype, n, vocab);
    if (st == SPCONV_OK)
        *bytes = spconv::sample_workspace(n, vocab);
    return st;
}

spconv_status spconv_sample(const void *logits, spconv_dtype dtype, int64_t ld, const float *u, int32_t n, int32_t vocab,
                            const float *temperatures, const int32_t *top_ks, const float *top_ps, const float *min_ps,
                            float temperature, int32_t top_k, float top_p, float min_p, int32_t *ids, void *workspace,
                            int64_t workspace_bytes, void *stream) {
    spconv::clear_error();
    const spconv_status st = check_sample(dtype, n, vocab);
    if (st != SPCONV_OK)
        return st;
    if ((!temperatures && !(temperature >= 0)) || (!top_ks && top_k < 0) || (!top_ps && !(top_p >= 0 && top_p <= 1)) ||
        (!min_ps && !(min_p >= 0 && min_p <= 1)))
        return set_error(SPCONV_E_ARG, "temperature and top_k must be >= 0, top_p and min_p in [0, 1]");
    if (n == 0)
        return SPCONV_OK;
    if (!logits || !u || !ids)
        return set_error(SPCONV_E_ARG, "logits, u or ids is NULL");
    if (ld < vocab)
        return set_error(SPCONV_E_ARG, "ld must be at least vocab");
    if (ld > kMostStride)
        return set_error(SPCONV_E_SHAPE, "ld must be at most 2^34");
    if (!aligned(logits, size_of(dtype)) || !aligned(u, 4) || !aligned(temperatures, 4) || !aligned(top_ks, 4) ||
        !aligned(top_ps, 4) || !aligned(min_ps, 4) || !aligned(ids, 4) || !aligned(workspace, 16))
        return set_error(SPCONV_E_ARG, "pointers must be aligned to their element size, the workspace to 16 bytes");
    const int64_t need = spconv::sample_workspace(n, vocab), column = n * int64_t(4);
    if (need > 0 && (!workspace || workspace_bytes < need))
        return set_error(SPCONV_E_ARG, "the workspace is smaller than spconv_sample_workspace says");
    const Range in[] = {{logits, span(n, vocab, ld, size_of(dtype))}, {u, column}, {temperatures, column},
                        {top_ks, column}, {top_ps, column}, {min_ps, column}};
    const Range out[] = {{ids, column}, {workspace, need}};
    if (outputs_overlap(out, in))
        return set_error(SPCONV_E_ARG, "ids and the workspace must not overlap each other or an input");
    spconv::SampleArgs a{};
    a.logits = logits;
    a.ld = ld;
    a.u = u;
    a.temperatures = temperatures;
    a.top_ks = top_ks;
    a.top_ps = top_ps;
    a.min_ps = min_ps;
    a.temperature = temperature;
    a.top_k = top_k;
    a.top_p = top_p;
    a.min_p = min_p;
    a.ids = ids;
    a.n = n;
    a.vocab = vocab;
    a.workspace = workspace;
    return launched(spconv::launch_sample(a, dtype, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
