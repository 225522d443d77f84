// Layer norm of the rows of a matrix.
//
// The mean is the first sum over the row's registers; the second pass over them sums d = v - mean and d^2, and the first of
// these takes out what the rounded mean was off by, so that rows far from zero lose nothing.  A team takes row after
// row with the next row's loads in flight.
#include "deft_norm_rows.cuh"

namespace deft {
namespace {

template <bool kAdd, typename TX, typename TY, bool kAligned, int kGroups>
__global__ void __launch_bounds__(kTeamMost) k_layer_norm(const __grid_constant__ LayerNormArgs a, const __grid_constant__ TeamShape shape) {
    extern __shared__ __align__(16) float params[];      // gamma, beta
    __shared__ float2 slots[2 * kTeamMostWarps];
    using Group = RowGroup<kAligned>;
    Team team(shape, slots);
    const int places = shape.places;
    const TX *x = static_cast<const TX*>(a.x), *add = static_cast<const TX*>(a.add);
    const uint32_t rows = (uint32_t)a.rows;
    Raw8<TX, Group::template align<TX>()> next[kGroups], next_add[kGroups];
    auto fetch = [&](uint32_t row) {
#pragma unroll
        for (int j = 0; j < kGroups; ++j) {
            const Group g(team.at + j * team.size, team.shift, a.cols);
            g.load(x + (int64_t)row * a.ld_x, next[j]);
            if (kAdd) g.load(add + (int64_t)row * a.ld_add, next_add[j]);
        }
    };
    if (team.row < rows) fetch(team.row);
    float* beta = params + places * kGroup;
    fill_places(params, a.gamma, a.w_type, a.cols, places, team.shift, 1.0f);
    fill_places(beta, a.beta, a.w_type, a.cols, places, team.shift, 0.0f);
    __syncthreads();
    const float cols = (float)a.cols;
    // all teams of a CTA take as many turns as its first one
    uint32_t turn_row = team.row - (uint32_t)team.team * (uint32_t)shape.step;
    for (uint32_t r = team.row; turn_row < rows; turn_row += team.stride, r += team.stride) {
        float v[kGroups][kGroup], sum = 0.0f;
#pragma unroll
        for (int j = 0; j < kGroups; ++j) {
            const Group g(team.at + j * team.size, team.shift, a.cols);
            next[j].unpack(v[j]);
            if (kAdd) next_add[j].add_to(v[j]);
            g.trim(v[j]);
#pragma unroll
            for (int k = 0; k < kGroup; ++k) sum += v[j][k];
        }
        const bool mine = r < rows;
        if (r + team.stride < rows) fetch(r + team.stride);
        const float mean = team.sum(sum, 0.0f).x / cols;
        float d1 = 0.0f, d2 = 0.0f;
#pragma unroll
        for (int j = 0; j < kGroups; ++j) {
            const Group g(team.at + j * team.size, team.shift, a.cols);
            if (kAdd && a.sum && mine) g.store(static_cast<TX*>(a.sum) + (int64_t)r * a.ld_sum, v[j]);
#pragma unroll
            for (int k = 0; k < kGroup; ++k) v[j][k] -= mean;
            g.trim(v[j]);
#pragma unroll
            for (int k = 0; k < kGroup; ++k) {
                d1 += v[j][k];
                d2 += v[j][k] * v[j][k];
            }
        }
        const float2 both = team.sum(d1, d2);
        if (!mine) continue;
        const float off = both.x / cols;
        float var = both.y / cols - off * off;
        var = var < 0.0f ? 0.0f : var;
        const float rstd = __frsqrt_rn(var + a.eps);
#pragma unroll
        for (int j = 0; j < kGroups; ++j) {
            const int place = team.at + j * team.size;
            if (place >= places) break;
            const Group g(place, team.shift, a.cols);
            float w[kGroup], b[kGroup];
            read_place(params, places, place, w);
            read_place(beta, places, place, b);
#pragma unroll
            for (int k = 0; k < kGroup; ++k) v[j][k] = (v[j][k] - off) * rstd * w[k] + b[k];
            g.store(static_cast<TY*>(a.y) + (int64_t)r * a.ld_y, v[j]);
        }
        if (team.at == 0) {
            if (a.mean) a.mean[r] = mean + off;
            if (a.rstd) a.rstd[r] = rstd;
        }
    }
}

}  // namespace

deft_status launch_layer_norm(const LayerNormArgs& a, int x_type, int y_type, cudaStream_t stream) {
    ShiftFinder m;
    m.add(a.x, a.ld_x, type_bytes(x_type));
    m.add(a.y, a.ld_y, type_bytes(y_type));
    m.add(a.add, a.ld_add, type_bytes(x_type));
    m.add(a.sum, a.ld_sum, type_bytes(x_type));
    const TeamShape s = team_shape(m, a.rows, a.cols, x_type == DEFT_F32 && a.cols <= kTeamMost * 16 - 8 ? 2 : 4, 4 * (int64_t)sm_count());
    const size_t smem = 2 * sizeof(float) * (size_t)(s.places * kGroup);
    return with_type(x_type, [&](auto x) {
        return with_type(y_type, [&](auto y) {
            return with_groups(s.aligned ? s.groups : 4, [&](auto g) -> deft_status {
                using TX = decltype(x);
                using TY = decltype(y);
                constexpr int kGroups = decltype(g)::value;
                auto run = [&](auto kernel) -> deft_status {
                    if (smem > 48 * 1024) DEFT_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
                    kernel<<<s.blocks, s.threads, smem, stream>>>(a, s);
                    DEFT_CUDA_TRY(cudaGetLastError());
                    return DEFT_OK;
                };
                if constexpr (kGroups == 4) {
                    if (!s.aligned) return a.add ? run(k_layer_norm<true, TX, TY, false, 4>) : run(k_layer_norm<false, TX, TY, false, 4>);
                }
                return a.add ? run(k_layer_norm<true, TX, TY, true, kGroups>) : run(k_layer_norm<false, TX, TY, true, kGroups>);
            });
        });
    });
}

}  // namespace deft
