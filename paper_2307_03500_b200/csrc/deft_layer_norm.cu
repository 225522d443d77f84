// Layer norm of the rows of a matrix.
//
// The mean is the first sum over the row's registers; the second pass over them sums d = v - mean and d^2, and the first of
// these takes out what the rounded mean was off by, so that rows far from zero lose nothing.
#include "deft_norm_rows.cuh"

namespace deft {
namespace {

template <bool kAdd, typename TX, typename TY, Feed kFeed, int kGroups, int kThreads>
__global__ void __launch_bounds__(kThreads, kGroups < 4 ? 4 : 1) k_layer_norm(const __grid_constant__ LayerNormArgs a, const __grid_constant__ TeamShape shape) {
    extern __shared__ __align__(16) char smem[];         // gamma, beta, the ring
    __shared__ float2 slots[2 * kTeamMostWarps];
    using Group = RowGroup<kFeed>;
    using Raw = Raw8<TX, Group::template align<TX>()>;
    constexpr int kRuns = kGroup * (int)sizeof(TX) / 16, kAll = kGroups * kRuns * (kAdd ? 2 : 1);
    Team team(shape, slots);
    const int places = shape.places;
    float *gamma = reinterpret_cast<float*>(smem), *beta = gamma + places * kGroup;
    Ring<kThreads, kAll> ring(smem + 2 * sizeof(float) * (size_t)(places * kGroup), shape.stages);
    const uint32_t rows = (uint32_t)a.rows;
    Group group[kGroups];
#pragma unroll
    for (int j = 0; j < kGroups; ++j) group[j].set(team.at + j * team.size, team.shift, a.cols);
    const int col = group[0].col;
    Walk<const TX> x(static_cast<const TX*>(a.x), a.ld_x, team.row, team.stride, col, team.size);
    Walk<const TX> add(static_cast<const TX*>(a.add), a.ld_add, team.row, team.stride, col, team.size);
    Walk<TX> sum_out(static_cast<TX*>(a.sum), a.ld_sum, team.row, team.stride, col, team.size);
    Walk<TY> y(static_cast<TY*>(a.y), a.ld_y, team.row, team.stride, col, team.size);
    uint32_t ahead = team.row;                           // the row that is copied next
    auto copy = [&](uint32_t stage) {
        if (ahead < rows) {
#pragma unroll
            for (int j = 0; j < kGroups; ++j) {
                group[j].copy(x.group(j), ring.target(stage, j * kRuns), ring.kRun);
                if (kAdd) group[j].copy(add.group(j), ring.target(stage, (kGroups + j) * kRuns), ring.kRun);
            }
        }
        ring.commit();
        ahead += team.stride;
        x.next();
        if (kAdd) add.next();
    };
    if constexpr (kFeed == Feed::kRing)
        for (uint32_t s = 0; s != ring.fill; s += kAll * ring.kRun) copy(s);
    fill_places(gamma, a.gamma, a.w_type, a.cols, places, team.shift, 1.0f);
    fill_places(beta, a.beta, a.w_type, a.cols, places, team.shift, 0.0f);
    __syncthreads();
    const float each = 1.0f / (float)a.cols;
    // all teams of a CTA take as many turns as its first one
    uint32_t turn_row = team.row - (uint32_t)team.team * (uint32_t)shape.step;
    for (uint32_t r = team.row; turn_row < rows; turn_row += team.stride, r += team.stride) {
        const bool mine = r < rows;
        if constexpr (kFeed == Feed::kRing) {
            copy(ring.fill);
            ring.wait();
        }
        Eight v[kGroups];
        uint64_t sum = 0;
#pragma unroll
        for (int j = 0; j < kGroups; ++j) {
            Raw raw, more;
            if constexpr (kFeed == Feed::kRing) {
                ring.read(j * kRuns, raw);
                if (kAdd) ring.read((kGroups + j) * kRuns, more);
            } else if (mine) {
                group[j].load(x.group(j), raw);
                if (kAdd) group[j].load(add.group(j), more);
            }
            v[j].from(raw);
            if (kAdd) {
                Eight m;
                m.from(more);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[j].p[i] = add2(v[j].p[i], m.p[i]);
            }
            if (!group[j].whole) v[j].trim(group[j].lo, group[j].hi);
            sum = add2(sum, v[j].sum());
            if (kAdd && a.sum && mine && group[j].any) group[j].store(sum_out.group(j), v[j]);
        }
        if constexpr (kFeed == Feed::kRing) ring.next();
        const float mean = team.sum(folded(sum), 0.0f).x * each;
        const uint64_t minus = both(-mean);
        uint64_t d1 = 0, d2 = 0;
#pragma unroll
        for (int j = 0; j < kGroups; ++j) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[j].p[i] = add2(v[j].p[i], minus);
            if (!group[j].whole) v[j].trim(group[j].lo, group[j].hi);
            d1 = add2(d1, v[j].sum());
#pragma unroll
            for (int i = 0; i < 4; ++i) d2 = fma2(v[j].p[i], v[j].p[i], d2);
        }
        const float2 sums = team.sum(folded(d1), folded(d2));
        const float off = sums.x * each;
        float var = sums.y * each - off * off;
        var = (var < 0.0f ? 0.0f : var) + a.eps;
        float rstd = rsqrtf(var);
        if (var > 1e-30f && var < 1e30f) rstd = __fmaf_rn(0.5f * rstd, __fmaf_rn(-var * rstd, rstd, 1.0f), rstd);    // (a step of Newton's)
        if (mine) {
            const uint64_t minus_off = both(-off), by = both(rstd);
#pragma unroll
            for (int j = 0; j < kGroups; ++j) {
                if (!group[j].any) continue;
                Eight w, b;
                read_place(gamma, places, team.at + j * team.size, w);
                read_place(beta, places, team.at + j * team.size, b);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[j].p[i] = fma2(mul2(add2(v[j].p[i], minus_off), by), w.p[i], b.p[i]);
                group[j].store(y.group(j), v[j]);
            }
            if (team.at == 0) {
                if (a.mean) a.mean[r] = mean + off;
                if (a.rstd) a.rstd[r] = rstd;
            }
        }
        y.next();
        if (kAdd) sum_out.next();
        if constexpr (kFeed != Feed::kRing) {
            x.next();
            if (kAdd) add.next();
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
    const TeamShape s = team_shape(m, a.rows, a.cols, kGroup * (int)type_bytes(x_type) * (a.add ? 2 : 1), 2, 4, 0);
    return with_type(x_type, [&](auto x) {
        return with_type(y_type, [&](auto y) {
            return with_groups(s.groups, [&](auto g) -> deft_status {
                using TX = decltype(x);
                using TY = decltype(y);
                constexpr int kGroups = decltype(g)::value;
                auto run = [&](auto kernel) -> deft_status {
                    if (s.smem > 40 * 1024) DEFT_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)s.smem));
                    kernel<<<s.blocks, s.threads, s.smem, stream>>>(a, s);
                    DEFT_CUDA_TRY(cudaGetLastError());
                    return DEFT_OK;
                };
                auto fed = [&](auto feed) {
                    constexpr Feed kFeed = decltype(feed)::value;
                    auto sized = [&](auto threads) {
                        constexpr int kThreads = decltype(threads)::value;
                        return a.add ? run(k_layer_norm<true, TX, TY, kFeed, kGroups, kThreads>) : run(k_layer_norm<false, TX, TY, kFeed, kGroups, kThreads>);
                    };
                    if constexpr (kGroups == 4) {
                        if (s.threads > kTeamThreads) return sized(AlignTag<kTeamMost>{});
                    }
                    return sized(AlignTag<kTeamThreads>{});
                };
                if constexpr (kGroups == 4) {
                    if (s.feed == Feed::kElements) return fed(FeedTag<Feed::kElements>{});
                    if (s.feed == Feed::kLoads) return fed(FeedTag<Feed::kLoads>{});
                }
                return fed(FeedTag<Feed::kRing>{});
            });
        });
    });
}

}  // namespace deft
