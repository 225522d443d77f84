// The dense row operators (layer norm and its gradient, rotary positions, distillation loss): what their files share.
#pragma once
#include "deft_rows.cuh"

namespace deft {

// Shared memory that a CTA may ask for.  Every call that needs more than a kernel has by itself sets a kernel's limit to this,
// not to its own need: another host thread's call of the same kernel may lie between a call's setting and its launch.
constexpr size_t kMostSmem = 220 * 1024;

struct LayerNormArgs {
    const void *x, *add;                 // add: NULL, or of x's type
    void *sum, *y;                       // sum: NULL, or x + add in x's type
    const void *gamma, *beta;            // NULL: ones, zeros; of w_type
    float *mean, *rstd;                  // NULL, or [rows]
    const void* idle;                    // a 16-byte boundary that may be read: the granule in which x begins
    int64_t ld_x, ld_add, ld_sum, ld_y;
    int64_t rows;
    int32_t cols, w_type;
    float eps;
};
struct LayerNormGradArgs {
    const void *dy, *x, *add;            // add: NULL, or of x's type: added to dx
    void* dx;                            // NULL, or of x's type
    const void* gamma;                   // NULL: ones; of w_type
    const float *mean, *rstd;
    const void* idle;                    // as above
    float *dgamma, *dbeta;               // NULL, or [cols]
    int64_t ld_dy, ld_x, ld_add, ld_dx;
    int64_t rows;
    int32_t cols, w_type, accumulate;
    float scale;
    float* partial;                      // the workspace
};
struct RotaryArgs {
    const void* x;
    void* y;
    const uint64_t* turns;               // [rot / 2], in 2^-64 turns per position
    const void* pos;                     // NULL (a token's number in its sequence), or [batch * tokens]
    int64_t x_batch, x_token, x_head, y_batch, y_token, y_head;   // strides in elements
    int64_t batch, tokens;
    int32_t heads, dim, rot, interleaved, pos_bytes;
    float gain_cos, gain_sin;            // gain, and gain with the sign of the direction
};
struct DistillArgs {
    const void *logits, *ids, *teacher;
    void* grad;                          // NULL, or of the logits' type
    const float *teacher_lse, *weight;   // NULL: renormalised, ones
    float* loss;                         // NULL, or [rows]
    int64_t ld, ld_ids, ld_teacher, ld_grad;
    int64_t rows;
    int32_t vocab, top;
    int32_t id_bytes, teacher_type;
    float it_hi, it_lo;                  // 1 / T in two pieces
    float c1, by, by_lo;                 // log2(e) / T; that, as rounded, times ln 2 in two pieces
    float loss_factor, grad_factor;      // T^2, scale * T
};
size_t layer_norm_grad_ws_bytes(int64_t rows, int64_t cols);
deft_status launch_layer_norm(const LayerNormArgs& a, int x_type, int y_type, cudaStream_t stream);
deft_status launch_layer_norm_grad(const LayerNormGradArgs& a, int dy_type, int x_type, cudaStream_t stream);
deft_status launch_rotary(const RotaryArgs& a, int type, cudaStream_t stream);
deft_status launch_distill(const DistillArgs& a, int type, cudaStream_t stream);

}  // namespace deft
