// C-ABI entry points of the row operators: argument checks and launches.
#include "deft_rows.cuh"
#include "deft_rows_args.h"

namespace deft {
namespace {

constexpr int64_t kMaxTokens = 2147483647LL;   // token positions, rows and columns are 32-bit
constexpr int64_t kMaxWidth = (1LL << 30) - 1;   // of the gradient's matrices: a row's bytes are a 32-bit number

// Fills d from the dropout arguments; false if they are invalid.  p is rounded to a multiple of 2^-16 (at most
// 65535 / 65536); the gain is that of the rounded p, so that the expectation is kept exactly.
bool drop_args(double p, uint64_t seed, uint64_t offset, const uint64_t* offset_d, DropArgs* d, double* gain) {
    if (!(p >= 0.0 && p < 1.0) || !elem_aligned(offset_d, 8)) return false;
    uint32_t t = (uint32_t)std::floor(p * 65536.0 + 0.5);
    if (t > 65535u) t = 65535u;
    *gain = 65536.0 / (double)(65536u - t);
    philox_keys(seed, d->keys);
    d->offset = offset;
    d->offset_d = offset_d;
    d->threshold = t << 16;
    d->gain = (float)*gain;
    return true;
}

}  // namespace
}  // namespace deft

using namespace deft;

extern "C" {

deft_status deft_embed(const void* table_d, int32_t table_type, int64_t rows, int64_t width, int64_t ld_table,
                       const void* ids_d, int32_t id_bytes, int64_t n, double scale, const void* pos_d, int64_t pos_rows,
                       int64_t ld_pos, double p, uint64_t seed, uint64_t offset, const uint64_t* offset_d, void* out_d,
                       int32_t out_type, int64_t ld_out, void* stream) {
    if (n < 0 || rows < 1 || width < 1 || !type_ok(table_type) || !type_ok(out_type) || (id_bytes != 4 && id_bytes != 8) ||
        !fits_f32(scale))
        return DEFT_ERR_INVALID_ARG;
    EmbedArgs a{};
    double gain;
    if (!drop_args(p, seed, offset, offset_d, &a.drop, &gain)) return DEFT_ERR_INVALID_ARG;
    if (n == 0) return DEFT_OK;
    if (n > kMaxTokens || width > kMaxTokens || rows > kMaxTokens) return DEFT_ERR_TOO_LARGE;
    if (!matrix_ok(table_d, table_type, rows, width, ld_table) || !matrix_ok(out_d, out_type, n, width, ld_out) || !ids_d ||
        !elem_aligned(ids_d, (size_t)id_bytes))
        return DEFT_ERR_INVALID_ARG;
    if (pos_d && (pos_rows < 1 || !matrix_ok(pos_d, table_type, pos_rows, width, ld_pos))) return DEFT_ERR_INVALID_ARG;
    a.table = table_d;
    a.rows = rows;
    a.ld_table = ld_table;
    a.pos = pos_d;
    a.pos_rows = pos_d ? pos_rows : 1;
    a.ld_pos = ld_pos;
    a.ids = ids_d;
    a.out = out_d;
    a.ld_out = ld_out;
    a.n = n;
    a.width = width;
    a.scale = (float)scale;
    return launch_embed(a, table_type, out_type, id_bytes, static_cast<cudaStream_t>(stream));
}

size_t deft_embed_workspace_bytes(int64_t n, int64_t rows, int64_t width) {
    if (n < 0 || n > kMaxTokens || rows < 1 || rows > DEFT_EMBED_MAX_ROWS || width < 1 || width > kMaxWidth) return 0;
    return embed_grad_ws_bytes(n, rows, width);
}

deft_status deft_embed_grad(const void* grad_out_d, int32_t grad_out_type, int64_t ld_grad_out, const void* ids_d,
                            int32_t id_bytes, int64_t n, int64_t rows, int64_t width, int64_t skip_id, double scale, double p,
                            uint64_t seed, uint64_t offset, const uint64_t* offset_d, float* grad_d, int32_t accumulate,
                            void* ws_d, size_t ws_bytes, void* stream) {
    if (n < 0 || rows < 1 || width < 1 || !type_ok(grad_out_type) || (id_bytes != 4 && id_bytes != 8) || !grad_d ||
        !elem_aligned(grad_d, 4) || !ws_d || !elem_aligned(ws_d, 256))
        return DEFT_ERR_INVALID_ARG;
    EmbedGradArgs a{};
    double gain;
    if (!drop_args(p, seed, offset, offset_d, &a.drop, &gain) || !fits_f32(scale * gain)) return DEFT_ERR_INVALID_ARG;
    if (n > kMaxTokens || width > kMaxWidth || rows > DEFT_EMBED_MAX_ROWS || (n > 0 && ld_grad_out > kMaxWidth)) return DEFT_ERR_TOO_LARGE;
    if (n > 0 && (!matrix_ok(grad_out_d, grad_out_type, n, width, ld_grad_out) || !ids_d || !elem_aligned(ids_d, (size_t)id_bytes)))
        return DEFT_ERR_INVALID_ARG;
    if (embed_grad_ws_bytes(n, rows, width) > ws_bytes) return DEFT_ERR_CAPACITY;
    if (n == 0 && accumulate) return DEFT_OK;
    a.dy = grad_out_d;
    a.ld_dy = ld_grad_out;
    a.ids = ids_d;
    a.n = n;
    a.rows = rows;
    a.width = width;
    a.skip_id = skip_id;
    a.factor = (float)(scale * gain);
    a.grad = grad_d;
    a.accumulate = accumulate ? 1 : 0;
    a.ws = static_cast<char*>(ws_d);
    return launch_embed_grad(a, grad_out_type, id_bytes, static_cast<cudaStream_t>(stream));
}

deft_status deft_dropout(const void* x_d, int32_t x_type, int64_t ld_x, const void* add_d, int64_t ld_add, void* y_d,
                         int32_t y_type, int64_t ld_y, int64_t rows, int64_t cols, double p, uint64_t seed, uint64_t offset,
                         const uint64_t* offset_d, void* stream) {
    if (rows < 0 || cols < 0 || !type_ok(x_type) || !type_ok(y_type)) return DEFT_ERR_INVALID_ARG;
    DropoutArgs a{};
    double gain;
    if (!drop_args(p, seed, offset, offset_d, &a.drop, &gain)) return DEFT_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return DEFT_OK;
    if (rows > kMaxTokens || cols > kMaxTokens) return DEFT_ERR_TOO_LARGE;
    if (!matrix_ok(x_d, x_type, rows, cols, ld_x) || !matrix_ok(y_d, y_type, rows, cols, ld_y) ||
        (add_d && !matrix_ok(add_d, y_type, rows, cols, ld_add)))
        return DEFT_ERR_INVALID_ARG;
    const Span y = span_of(y_d, y_type, cols, ld_y, rows);
    if (!in_place_or_apart(y, span_of(x_d, x_type, cols, ld_x, rows), x_type == y_type, rows) ||
        (add_d && !in_place_or_apart(y, span_of(add_d, y_type, cols, ld_add, rows), true, rows)))
        return DEFT_ERR_INVALID_ARG;
    a.x = x_d;
    a.ld_x = ld_x;
    a.add = add_d;
    a.ld_add = ld_add;
    a.y = y_d;
    a.ld_y = ld_y;
    a.rows = rows;
    a.cols = cols;
    return launch_dropout(a, x_type, y_type, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
