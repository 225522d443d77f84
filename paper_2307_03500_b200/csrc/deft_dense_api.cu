// C-ABI entry points of the dense row operators: argument checks and launches.
#include "deft_dense.cuh"
#include "deft_rows_args.h"

namespace deft {
namespace {

constexpr int64_t kMaxRows = 2147483647LL;

// The 16-byte granule that an address lies in.
const void* granule_of(const void* p) { return reinterpret_cast<const void*>(reinterpret_cast<uintptr_t>(p) & ~(uintptr_t)15); }

// The elements of a [batch, tokens, heads, dim] tensor in bytes: rows of contiguous columns, dimensions by falling stride.
struct Boxes {
    uintptr_t base;
    uint64_t row;
    int n;
    uint64_t count[3], stride[3];
};
Boxes boxes_of(const void* p, size_t elem, const int64_t* counts, const int64_t* strides, int64_t dim) {
    Boxes b{reinterpret_cast<uintptr_t>(p), (uint64_t)dim * elem, 0, {}, {}};
    for (int i = 0; i < 3; ++i) {
        if (counts[i] == 1) continue;
        int at = b.n++;
        for (; at > 0 && b.stride[at - 1] < (uint64_t)strides[i] * elem; --at) {
            b.stride[at] = b.stride[at - 1];
            b.count[at] = b.count[at - 1];
        }
        b.stride[at] = (uint64_t)strides[i] * elem;
        b.count[at] = (uint64_t)counts[i];
    }
    return b;
}
uint64_t reach(const Boxes& b, int from) {
    uint64_t r = b.row;
    for (int i = from; i < b.n; ++i) r += (b.count[i] - 1) * b.stride[i];
    return r;
}
// No two rows share a byte: every stride reaches over all that lies within it.  (Other layouts without shared bytes, rows
// interleaved at odd distances, are refused too.)
bool nested(const Boxes& b) {
    for (int i = 0; i < b.n; ++i)
        if (b.stride[i] < reach(b, i + 1)) return false;
    return true;
}
// Whether two nested tensors of one layout, `apart` bytes from one another, share a byte.
bool meet(const Boxes& b, int i, uint64_t apart) {
    if (i == b.n) return apart < b.row;
    const uint64_t steps = apart / b.stride[i], rest = apart % b.stride[i];
    if (steps < b.count[i] && meet(b, i + 1, rest)) return true;
    return steps + 1 < b.count[i] && meet(b, i + 1, b.stride[i] - rest);
}
bool same_layout(const Boxes& a, const Boxes& b) {
    for (int i = 0; i < a.n; ++i)
        if (a.stride[i] != b.stride[i] || a.count[i] != b.count[i]) return false;
    return a.row == b.row && a.n == b.n;
}

}  // namespace
}  // namespace deft

using namespace deft;

extern "C" {

deft_status deft_layer_norm(const void* x_d, int32_t x_type, int64_t ld_x, const void* add_d, int64_t ld_add, void* sum_d,
                            int64_t ld_sum, const void* gamma_d, const void* beta_d, int32_t w_type, void* y_d, int32_t y_type,
                            int64_t ld_y, int64_t rows, int64_t cols, double eps, float* mean_d, float* rstd_d, void* stream) {
    if (rows < 0 || cols < 1 || !type_ok(x_type) || !type_ok(y_type) || !type_ok(w_type) || !(eps >= 0.0) || !fits_f32(eps) ||
        (sum_d && !add_d) || !elem_aligned(gamma_d, type_bytes(w_type)) || !elem_aligned(beta_d, type_bytes(w_type)) ||
        !elem_aligned(mean_d, 4) || !elem_aligned(rstd_d, 4))
        return DEFT_ERR_INVALID_ARG;
    if (rows == 0) return DEFT_OK;
    if (rows > kMaxRows || cols > DEFT_NORM_MAX_COLS) return DEFT_ERR_TOO_LARGE;
    if (!matrix_ok(x_d, x_type, rows, cols, ld_x) || !matrix_ok(y_d, y_type, rows, cols, ld_y) ||
        (add_d && !matrix_ok(add_d, x_type, rows, cols, ld_add)) || (sum_d && !matrix_ok(sum_d, x_type, rows, cols, ld_sum)))
        return DEFT_ERR_INVALID_ARG;
    const Span x = span_of(x_d, x_type, cols, ld_x, rows), y = span_of(y_d, y_type, cols, ld_y, rows);
    if (!in_place_or_apart(y, x, x_type == y_type, rows)) return DEFT_ERR_INVALID_ARG;
    if (add_d && !in_place_or_apart(y, span_of(add_d, x_type, cols, ld_add, rows), x_type == y_type, rows)) return DEFT_ERR_INVALID_ARG;
    if (sum_d) {
        const Span s = span_of(sum_d, x_type, cols, ld_sum, rows);
        if (!in_place_or_apart(s, x, true, rows) || !in_place_or_apart(s, span_of(add_d, x_type, cols, ld_add, rows), true, rows) ||
            overlap(s, y, rows))
            return DEFT_ERR_INVALID_ARG;
    }
    LayerNormArgs a{};
    a.x = x_d;
    a.add = add_d;
    a.sum = sum_d;
    a.y = y_d;
    a.gamma = gamma_d;
    a.beta = beta_d;
    a.mean = mean_d;
    a.rstd = rstd_d;
    a.idle = granule_of(x_d);
    a.ld_x = ld_x;
    a.ld_add = ld_add;
    a.ld_sum = ld_sum;
    a.ld_y = ld_y;
    a.rows = rows;
    a.cols = (int32_t)cols;
    a.w_type = w_type;
    a.eps = (float)eps;
    return launch_layer_norm(a, x_type, y_type, static_cast<cudaStream_t>(stream));
}

size_t deft_layer_norm_workspace_bytes(int64_t rows, int64_t cols) {
    if (rows < 0 || rows > kMaxRows || cols < 1 || cols > DEFT_NORM_MAX_COLS) return 0;
    return layer_norm_grad_ws_bytes(rows, cols);
}

deft_status deft_layer_norm_grad(const void* grad_out_d, int32_t grad_out_type, int64_t ld_grad_out, const void* x_d,
                                 int32_t x_type, int64_t ld_x, const float* mean_d, const float* rstd_d, const void* gamma_d,
                                 int32_t w_type, const void* add_d, int64_t ld_add, void* grad_x_d, int64_t ld_grad_x,
                                 float* grad_gamma_d, float* grad_beta_d, int64_t rows, int64_t cols, int32_t accumulate,
                                 double scale, void* ws_d, size_t ws_bytes, void* stream) {
    const bool weights = grad_gamma_d || grad_beta_d;
    if (rows < 0 || cols < 1 || !type_ok(grad_out_type) || !type_ok(x_type) || !type_ok(w_type) || !fits_f32(scale) ||
        (rows > 0 && !weights && !grad_x_d) || !elem_aligned(gamma_d, type_bytes(w_type)) || !elem_aligned(grad_gamma_d, 4) ||
        !elem_aligned(grad_beta_d, 4) || !elem_aligned(mean_d, 4) || !elem_aligned(rstd_d, 4) || !elem_aligned(ws_d, 256) || (weights && !ws_d))
        return DEFT_ERR_INVALID_ARG;
    if (rows > kMaxRows || cols > DEFT_NORM_MAX_COLS) return DEFT_ERR_TOO_LARGE;
    if (rows > 0) {
        if (!matrix_ok(grad_out_d, grad_out_type, rows, cols, ld_grad_out) || !matrix_ok(x_d, x_type, rows, cols, ld_x) || !mean_d || !rstd_d ||
            (add_d && !matrix_ok(add_d, x_type, rows, cols, ld_add)) || (grad_x_d && !matrix_ok(grad_x_d, x_type, rows, cols, ld_grad_x)))
            return DEFT_ERR_INVALID_ARG;
        if (grad_x_d) {
            const Span g = span_of(grad_x_d, x_type, cols, ld_grad_x, rows);
            if (!in_place_or_apart(g, span_of(grad_out_d, grad_out_type, cols, ld_grad_out, rows), grad_out_type == x_type, rows) ||
                !in_place_or_apart(g, span_of(x_d, x_type, cols, ld_x, rows), true, rows) ||
                (add_d && !in_place_or_apart(g, span_of(add_d, x_type, cols, ld_add, rows), true, rows)))
                return DEFT_ERR_INVALID_ARG;
        }
    }
    if (weights && layer_norm_grad_ws_bytes(rows, cols) > ws_bytes) return DEFT_ERR_CAPACITY;
    if (rows == 0 && (accumulate || !weights)) return DEFT_OK;
    LayerNormGradArgs a{};
    a.dy = grad_out_d;
    a.x = x_d;
    a.add = grad_x_d ? add_d : nullptr;
    a.dx = grad_x_d;
    a.gamma = gamma_d;
    a.mean = mean_d;
    a.rstd = rstd_d;
    a.idle = granule_of(x_d);
    a.dgamma = grad_gamma_d;
    a.dbeta = grad_beta_d;
    a.ld_dy = ld_grad_out;
    a.ld_x = ld_x;
    a.ld_add = ld_add;
    a.ld_dx = ld_grad_x;
    a.rows = rows;
    a.cols = (int32_t)cols;
    a.w_type = w_type;
    a.accumulate = accumulate ? 1 : 0;
    a.scale = (float)scale;
    a.partial = static_cast<float*>(ws_d);
    return launch_layer_norm_grad(a, grad_out_type, x_type, static_cast<cudaStream_t>(stream));
}

deft_status deft_rotary(const void* x_d, const int64_t* x_strides_h, void* y_d, const int64_t* y_strides_h, int32_t type,
                        int64_t batch, int64_t tokens, int64_t heads, int64_t dim, const uint64_t* turns_d, int64_t rot,
                        int32_t interleaved, int32_t inverse, double gain, const void* pos_d, int32_t pos_bytes, void* stream) {
    if (batch < 0 || tokens < 0 || heads < 0 || dim < 1 || rot < 2 || (rot & 1) || rot > dim || !type_ok(type) || !fits_f32(gain) ||
        !x_strides_h || !y_strides_h || (pos_d && pos_bytes != 4 && pos_bytes != 8))
        return DEFT_ERR_INVALID_ARG;
    if (batch == 0 || tokens == 0 || heads == 0) return DEFT_OK;
    if (batch > kMaxRows || tokens > kMaxRows || batch * tokens > kMaxRows || heads > (1LL << 30) || dim > (1LL << 30) ||
        heads * dim > (1LL << 30) || rot > DEFT_ROTARY_MAX_ROT)
        return DEFT_ERR_TOO_LARGE;
    const size_t elem = type_bytes(type);
    if (!x_d || !y_d || !turns_d || !elem_aligned(x_d, elem) || !elem_aligned(y_d, elem) || !elem_aligned(turns_d, 8) ||
        (pos_d && !elem_aligned(pos_d, (size_t)pos_bytes)))
        return DEFT_ERR_INVALID_ARG;
    const int64_t counts[3] = {batch, tokens, heads};
    int64_t xs[3], ys[3];
    for (int i = 0; i < 3; ++i) {
        xs[i] = counts[i] == 1 ? 0 : x_strides_h[i];
        ys[i] = counts[i] == 1 ? 0 : y_strides_h[i];
        if (xs[i] < 0 || ys[i] < 0 || xs[i] > (1LL << 58) / counts[i] || ys[i] > (1LL << 58) / counts[i]) return DEFT_ERR_INVALID_ARG;   // offsets fit 64 bits
    }
    const Boxes x = boxes_of(x_d, elem, counts, xs, dim), y = boxes_of(y_d, elem, counts, ys, dim);
    if (!nested(y)) return DEFT_ERR_INVALID_ARG;
    // element for element the same place: every dimension's own stride, not the same list of them (a transposition)
    if (!(x.base == y.base && xs[0] == ys[0] && xs[1] == ys[1] && xs[2] == ys[2])) {
        const bool meeting = x.base < y.base ? y.base - x.base < reach(x, 0) : x.base - y.base < reach(y, 0);
        if (meeting && (!same_layout(x, y) || meet(x, 0, x.base < y.base ? y.base - x.base : x.base - y.base))) return DEFT_ERR_INVALID_ARG;
    }
    RotaryArgs a{};
    a.x = x_d;
    a.y = y_d;
    a.turns = turns_d;
    a.pos = pos_d;
    a.x_batch = xs[0];
    a.x_token = xs[1];
    a.x_head = xs[2];
    a.y_batch = ys[0];
    a.y_token = ys[1];
    a.y_head = ys[2];
    a.batch = batch;
    a.tokens = tokens;
    a.heads = (int32_t)heads;
    a.dim = (int32_t)dim;
    a.rot = (int32_t)rot;
    a.interleaved = interleaved ? 1 : 0;
    a.pos_bytes = pos_bytes;
    a.gain_cos = (float)gain;
    a.gain_sin = inverse ? -(float)gain : (float)gain;
    return launch_rotary(a, type, static_cast<cudaStream_t>(stream));
}

deft_status deft_distill(const void* logits_d, int32_t type, int64_t ld_logits, int64_t rows, int64_t vocab, const void* ids_d,
                         int32_t id_bytes, int64_t ld_ids, const void* teacher_d, int32_t teacher_type, int64_t ld_teacher,
                         int64_t top, const float* teacher_lse_d, double temperature, const float* weight_d, double scale,
                         float* loss_d, void* grad_d, int64_t ld_grad, void* stream) {
    if (rows < 0 || vocab < 1 || top < 1 || !type_ok(type) || !type_ok(teacher_type) || (id_bytes != 4 && id_bytes != 8) ||
        !(temperature >= 1e-6 && temperature <= 1e6) || !fits_f32(scale) || !fits_f32(scale * temperature) || (rows > 0 && !loss_d && !grad_d) ||
        !elem_aligned(teacher_lse_d, 4) || !elem_aligned(weight_d, 4) || !elem_aligned(loss_d, 4))
        return DEFT_ERR_INVALID_ARG;
    if (rows == 0) return DEFT_OK;
    if (rows >= (1LL << 28) || vocab > DEFT_DISTILL_MAX_VOCAB || top > DEFT_DISTILL_MAX_TOP) return DEFT_ERR_TOO_LARGE;
    if (!matrix_ok(logits_d, type, rows, vocab, ld_logits) || !matrix_ok(teacher_d, teacher_type, rows, top, ld_teacher) || !ids_d ||
        !elem_aligned(ids_d, (size_t)id_bytes) || ld_ids < top || ld_ids > (1LL << 60) / rows || (grad_d && !matrix_ok(grad_d, type, rows, vocab, ld_grad)))
        return DEFT_ERR_INVALID_ARG;
    if (grad_d && !in_place_or_apart(span_of(grad_d, type, vocab, ld_grad, rows), span_of(logits_d, type, vocab, ld_logits, rows), true, rows))
        return DEFT_ERR_INVALID_ARG;
    DistillArgs a{};
    a.logits = logits_d;
    a.ids = ids_d;
    a.teacher = teacher_d;
    a.grad = grad_d;
    a.teacher_lse = teacher_lse_d;
    a.weight = weight_d;
    a.loss = loss_d;
    a.ld = ld_logits;
    a.ld_ids = ld_ids;
    a.ld_teacher = ld_teacher;
    a.ld_grad = ld_grad;
    a.rows = rows;
    a.vocab = (int32_t)vocab;
    a.top = (int32_t)top;
    a.id_bytes = id_bytes;
    a.teacher_type = teacher_type;
    a.it_hi = (float)(1.0 / temperature);
    a.it_lo = (float)(1.0 / temperature - (double)a.it_hi);
    a.c1 = (float)(1.442695040888963407360 / temperature);
    const double by = (double)a.c1 * 0.693147180559945309417;
    a.by = (float)by;
    a.by_lo = (float)(by - (double)a.by);
    a.loss_factor = (float)(temperature * temperature);
    a.grad_factor = (float)(scale * temperature);
    return launch_distill(a, type, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
