// The gradient of layer norm.
//
// With h = (x - mean) rstd and d = dy gamma:  dx = rstd (d - mean(d) - h mean(d h)) + add, one pass over the row's registers,
// two sums.  The weight sums dy h and dy stay in registers over all rows of a thread's columns; they leave the CTA once as
// partial sums, and a second kernel adds those in a fixed order: the same bits on every call.
#include "deft_norm_rows.cuh"

namespace deft {
namespace {

constexpr int kPartials = 2 * 148;   // CTAs that leave partial sums at most; a constant: a call's bits do not depend on the device

template <bool kAdd, typename TD, typename TX, bool kAligned, int kGroups>
__global__ void __launch_bounds__(kTeamMost) k_layer_norm_grad(const __grid_constant__ LayerNormGradArgs a, const __grid_constant__ TeamShape shape) {
    extern __shared__ __align__(16) float params[];      // gamma; at the end the CTA's sums for gamma and beta
    __shared__ float2 slots[2 * kTeamMostWarps];
    using Group = RowGroup<kAligned>;
    Team team(shape, slots);
    const int places = shape.places;
    const TD* dy = static_cast<const TD*>(a.dy);
    const TX *x = static_cast<const TX*>(a.x), *add = static_cast<const TX*>(a.add);
    const uint32_t rows = (uint32_t)a.rows;
    Raw8<TX, Group::template align<TX>()> next_x[kGroups], next_add[kGroups];
    Raw8<TD, Group::template align<TD>()> next_dy[kGroups];
    float next_mean = 0.0f, next_rstd = 0.0f;
    auto fetch = [&](uint32_t row) {
        next_mean = a.mean[row];
        next_rstd = a.rstd[row];
#pragma unroll
        for (int j = 0; j < kGroups; ++j) {
            const Group g(team.at + j * team.size, team.shift, a.cols);
            g.load(x + (int64_t)row * a.ld_x, next_x[j]);
            g.load(dy + (int64_t)row * a.ld_dy, next_dy[j]);
            if (kAdd) g.load(add + (int64_t)row * a.ld_add, next_add[j]);
        }
    };
    if (team.row < rows) fetch(team.row);
    fill_places(params, a.gamma, a.w_type, a.cols, places, team.shift, 1.0f);
    __syncthreads();
    const float cols = (float)a.cols;
    float dg[kGroups][kGroup] = {}, db[kGroups][kGroup] = {};
    uint32_t turn_row = team.row - (uint32_t)team.team * (uint32_t)shape.step;
    for (uint32_t r = team.row; turn_row < rows; turn_row += team.stride, r += team.stride) {
        const float mean = next_mean, rstd = next_rstd;
        const bool mine = r < rows;
        float h[kGroups][kGroup], d[kGroups][kGroup], c1 = 0.0f, c2 = 0.0f;
        Raw8<TX, Group::template align<TX>()> more[kGroups];
#pragma unroll
        for (int j = 0; j < kGroups; ++j) {
            const int place = team.at + j * team.size;
            const Group g(place, team.shift, a.cols);
            float w[kGroup];
            read_place(params, places, place < places ? place : 0, w);
            next_x[j].unpack(h[j]);
            next_dy[j].unpack(d[j]);
            if (kAdd) more[j] = next_add[j];
#pragma unroll
            for (int k = 0; k < kGroup; ++k) h[j][k] = (h[j][k] - mean) * rstd;
            g.trim(h[j]);
            g.trim(d[j]);
            if (mine) {
#pragma unroll
                for (int k = 0; k < kGroup; ++k) {
                    db[j][k] += d[j][k];
                    dg[j][k] += d[j][k] * h[j][k];
                }
            }
#pragma unroll
            for (int k = 0; k < kGroup; ++k) {
                d[j][k] *= w[k];
                c1 += d[j][k];
                c2 += d[j][k] * h[j][k];
            }
        }
        if (r + team.stride < rows) fetch(r + team.stride);
        if (!a.dx) continue;
        float2 c = team.sum(c1, c2);
        if (!mine) continue;
        c.x /= cols;
        c.y /= cols;
#pragma unroll
        for (int j = 0; j < kGroups; ++j) {
            const Group g(team.at + j * team.size, team.shift, a.cols);
#pragma unroll
            for (int k = 0; k < kGroup; ++k) d[j][k] = rstd * (d[j][k] - c.x - h[j][k] * c.y);
            if (kAdd) more[j].add_to(d[j]);
            if (g.hi > g.lo) g.store(static_cast<TX*>(a.dx) + (int64_t)r * a.ld_dx, d[j]);
        }
    }
    if (!a.dgamma && !a.dbeta) return;
    // the teams' sums in order
    float* beta = params + places * kGroup;
    for (int t = 0; t < team.teams; ++t) {
        __syncthreads();
        if (t != team.team) continue;
#pragma unroll
        for (int j = 0; j < kGroups; ++j) {
            const int place = team.at + j * team.size;
            if (place >= places) break;
            if (t) {
                float was[kGroup];
                read_place(params, places, place, was);
#pragma unroll
                for (int k = 0; k < kGroup; ++k) dg[j][k] += was[k];
                read_place(beta, places, place, was);
#pragma unroll
                for (int k = 0; k < kGroup; ++k) db[j][k] += was[k];
            }
            write_place(params, places, place, dg[j]);
            write_place(beta, places, place, db[j]);
        }
    }
    __syncthreads();
    // in the order of the columns: CTAs of different shifts meet
    float* out = a.partial + (int64_t)blockIdx.x * 2 * a.cols;
    for (int c = threadIdx.x; c < a.cols; c += blockDim.x) {
        const int i = c + team.shift;
        out[c] = params[at_place(places, i >> 3, i & 7)];
        out[a.cols + c] = beta[at_place(places, i >> 3, i & 7)];
    }
}

// The CTAs' partial sums added up: a lane per column, eight warps that take every eighth CTA's.
constexpr int kJoinWarps = 8;
__global__ void __launch_bounds__(kJoinWarps * 32) k_layer_norm_join(const __grid_constant__ LayerNormGradArgs a, const int partials) {
    __shared__ float part[kJoinWarps][32];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t both = 2 * (int64_t)a.cols, at = (int64_t)blockIdx.x * 32 + lane;
    float sum = 0.0f;
    if (at < both) {
#pragma unroll 4
        for (int p = warp; p < partials; p += kJoinWarps) sum += a.partial[p * both + at];
    }
    part[warp][lane] = sum;
    __syncthreads();
    if (warp || at >= both) return;
    for (int w = 1; w < kJoinWarps; ++w) sum += part[w][lane];
    float* out = at < a.cols ? a.dgamma : a.dbeta;
    if (!out) return;
    out += at < a.cols ? at : at - a.cols;
    sum *= a.scale;
    *out = a.accumulate ? *out + sum : sum;
}

}  // namespace

size_t layer_norm_grad_ws_bytes(int64_t rows, int64_t cols) {
    // CTAs come in multiples of up to eight
    const int64_t partials = (rows + 7) / 8 * 8 < kPartials ? (rows ? (rows + 7) / 8 * 8 : 1) : kPartials;
    return (size_t)partials * 2 * sizeof(float) * (size_t)cols;
}

deft_status launch_layer_norm_grad(const LayerNormGradArgs& a, int dy_type, int x_type, cudaStream_t stream) {
    unsigned blocks = 0;
    if (a.rows) {
        ShiftFinder m;
        m.add(a.x, a.ld_x, type_bytes(x_type));
        m.add(a.dy, a.ld_dy, type_bytes(dy_type));
        m.add(a.add, a.ld_add, type_bytes(x_type));
        m.add(a.dx, a.ld_dx, type_bytes(x_type));
        const TeamShape s = team_shape(m, a.rows, a.cols, a.cols > kTeamMost * 16 - 8 ? 4 : 2, kPartials);
        blocks = s.blocks;
        const size_t smem = 2 * sizeof(float) * (size_t)(s.places * kGroup);
        const deft_status st = with_type(dy_type, [&](auto d) {
            return with_type(x_type, [&](auto x) {
                return with_groups(s.aligned ? s.groups : 4, [&](auto g) -> deft_status {
                    using TD = decltype(d);
                    using TX = decltype(x);
                    constexpr int kGroups = decltype(g)::value;
                    auto run = [&](auto kernel) -> deft_status {
                        if (smem > 48 * 1024) DEFT_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
                        kernel<<<s.blocks, s.threads, smem, stream>>>(a, s);
                        DEFT_CUDA_TRY(cudaGetLastError());
                        return DEFT_OK;
                    };
                    if constexpr (kGroups == 4) {
                        if (!s.aligned) return a.add ? run(k_layer_norm_grad<true, TD, TX, false, 4>) : run(k_layer_norm_grad<false, TD, TX, false, 4>);
                    }
                    return a.add ? run(k_layer_norm_grad<true, TD, TX, true, kGroups>) : run(k_layer_norm_grad<false, TD, TX, true, kGroups>);
                });
            });
        });
        if (st != DEFT_OK) return st;
    }
    if (!a.dgamma && !a.dbeta) return DEFT_OK;
    cudaLaunchAttribute follows{};
    follows.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    follows.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)((2 * (int64_t)a.cols + 31) / 32));
    cfg.blockDim = dim3(kJoinWarps * 32);
    cfg.stream = stream;
    cfg.attrs = &follows;
    cfg.numAttrs = a.rows ? 1 : 0;
    DEFT_CUDA_TRY(cudaLaunchKernelEx(&cfg, k_layer_norm_join, a, (int)blocks));
    return DEFT_OK;
}

}  // namespace deft
