// Layer norm of the rows of a matrix.
//
// One pass over the row's registers sums v and v^2, joined by one reduction; the variance is their difference where the mean
// is no larger than the standard deviation.  Other rows (far from zero) take a second pass that sums d = v - mean and d^2, the
// first of which takes out what the rounded mean was off by, so that they lose nothing.
//
// Bound by memory: each matrix crosses once.  Measured (device time; floor: its bytes at the copy rate, 6561 GB/s):
//   16384 x 1024 bf16, branch and sum        24.9 us (5.39 TB/s; floor 20.5)      8192 x 4096 bf16, branch   50 us (floor 40.9)
//   16384 x  768 bf16                        12.5 us (floor 7.7)                  16384 x 1024 fp32          24.2 us (floor 20.5)
//   65536 x 1024 bf16, branch and sum          97 us (floor 81.9)                 4096 x 8192 bf16, branch   47 us (floor 40.9)
//   5003 x 1027 fp32 -> bf16                 11.7 us (floor 4.7; groups shifted with the row, CTAs of one shift, a few rows a team)
//   65536 x 1027 bf16                          71 us (floor 41)
//   64 x 1024                                 3.7 us (latency: parameters, one row, one reduction)
//   8192 x 4096 fp32, branch                  147 us (floor 82: parameters leave four CTAs an SM no room for a ring, so that rows come by loads)
//   4096 x 16384 bf16, branch                 107 us (floor 82)                   2048 x 16384 fp32, branch 135 us (floor 82: by loads)
//   16384 x 1024 bf16, branch, y one element off the others' place in a granule   82 us (floor 20.5: element by element)
// Four CTAs of 256 threads an SM (64 registers) hide one another's reductions; issue slots 54 %.  What keeps it from the copy
// rate is what a row waits for (the ring's reads, then the copies); the start and the end less so: 16384 rows, seven a team, take 1.22
// times their floor, 65536 rows 1.18.
#include "deft_norm_rows.cuh"

namespace deft {
namespace {

template <typename TX, typename TY> constexpr int kColsOf = sizeof(TX) == 4 || sizeof(TY) == 4 ? 4 : 8;

template <bool kAdd, typename TX, typename TY, Feed kFeed, int kGroups, int kThreads, bool kPlain>
__global__ void __launch_bounds__(kThreads, kThreads != kTeamThreads ? 1 : (kPlain && kGroups * kColsOf<TX, TY> == 16 ? 4 : 3)) k_layer_norm(const __grid_constant__ LayerNormArgs a, const __grid_constant__ TeamShape shape) {
    extern __shared__ __align__(16) char smem[];         // gamma, beta, the ring
    __shared__ float2 slots[2 * kTeamMostWarps];
    constexpr int kC = kColsOf<TX, TY>;
    using Group = RowGroup<kFeed, kC, kPlain>;
    using Raw = typename Group::template Raw<TX>;
    constexpr int kX = kC * (int)sizeof(TX), kAtAdd = kGroups * kX, kAll = kAtAdd * (kAdd ? 2 : 1);   // bytes of a thread in a stage
    Team team(shape, kC, slots);
    const int places = shape.places;
    float *gamma = reinterpret_cast<float*>(smem), *beta = gamma + places * kC;
    Ring<kThreads, kAll> ring(smem + 2 * sizeof(float) * (size_t)(places * kC), shape.stages);
    const uint32_t rows = (uint32_t)a.rows;
    Group group[kGroups];
#pragma unroll
    for (int j = 0; j < kGroups; ++j) group[j].set(team.at + j * team.size, team.shift, a.cols);
    const int col = team.at * kC - team.shift, across = team.size * kC;
    Walk<const TX> x(static_cast<const TX*>(a.x), a.ld_x, team.row, team.stride, col, across);
    Walk<const TX> add(static_cast<const TX*>(a.add), a.ld_add, team.row, team.stride, col, across);
    Walk<TX> sum_out(static_cast<TX*>(a.sum), a.ld_sum, team.row, team.stride, col, across);
    Walk<TY> y(static_cast<TY*>(a.y), a.ld_y, team.row, team.stride, col, across);
    uint32_t ahead = team.row;                           // the row that is copied next
    auto copy = [&](uint32_t stage) {
        if (ahead < rows) {
#pragma unroll
            for (int j = 0; j < kGroups; ++j) {
                group[j].copy(x.group(j), a.idle, ring.target(stage, j * kX, kX));
                if (kAdd) group[j].copy(add.group(j), a.idle, ring.target(stage, kAtAdd + j * kX, kX));
            }
        }
        ring.commit();
        ahead += team.stride;
        x.next();
        if (kAdd) add.next();
    };
    if constexpr (kFeed == Feed::kRing)
        for (uint32_t s = 0; s != ring.fill; s += ring.kStage) copy(s);
    fill_places<kC>(gamma, a.gamma, a.w_type, a.cols, places, team.shift, 1.0f);
    fill_places<kC>(beta, a.beta, a.w_type, a.cols, places, team.shift, 0.0f);
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
        Cols<kC> v[kGroups];
        uint64_t s1 = 0, s2 = 0;
#pragma unroll
        for (int j = 0; j < kGroups; ++j) {
            Raw raw, more;
            if constexpr (kFeed == Feed::kRing) {
                ring.read(j * kX, raw);
                if (kAdd) ring.read(kAtAdd + j * kX, more);
            } else if (mine) {
                group[j].load(x.group(j), raw);
                if (kAdd) group[j].load(add.group(j), more);
            }
            v[j].from(raw);
            if (kAdd) {
                Cols<kC> m;
                m.from(more);
#pragma unroll
                for (int i = 0; i < kC / 2; ++i) v[j].p[i] = add2(v[j].p[i], m.p[i]);
            }
            if (j == 0 || kFeed != Feed::kRing) group[j].clear(v[j]);      // (a thread's first group alone may begin before the row)
            if (kAdd && a.sum && mine && group[j].any) group[j].store(sum_out.group(j), v[j]);
#pragma unroll
            for (int i = 0; i < kC / 2; ++i) {
                s1 = add2(s1, v[j].p[i]);
                s2 = fma2(v[j].p[i], v[j].p[i], s2);
            }
        }
        if constexpr (kFeed == Feed::kRing) ring.next();
        float2 sums = team.sum(folded(s1), folded(s2));
        float mean = sums.x * each, var = __fmaf_rn(-mean, mean, sums.y * each);
        // A warp's teams go the same way, but only those that have to keep what the second pass gives: a row's bits depend on
        // neither its neighbours nor on what teams without a row find.
        const bool own = mine && !(mean * mean <= var);
        if (team.size < 32 ? __any_sync(0xffffffffu, own) : own) {
            const float first = own ? mean : 0.0f;
            const uint64_t minus = both(-first);         // (v - 0 is v)
            s1 = s2 = 0;
#pragma unroll
            for (int j = 0; j < kGroups; ++j) {
                Cols<kC> d;
#pragma unroll
                for (int i = 0; i < kC / 2; ++i) d.p[i] = add2(v[j].p[i], minus);
                if (!group[j].whole) d.trim(group[j].lo, group[j].hi);
                v[j] = d;
#pragma unroll
                for (int i = 0; i < kC / 2; ++i) {
                    s1 = add2(s1, d.p[i]);
                    s2 = fma2(d.p[i], d.p[i], s2);
                }
            }
            sums = team.sum(folded(s1), folded(s2));
            if (team.at == 0 && mine && a.mean) a.mean[r] = own ? first + sums.x * each : mean;
            if (own) {
                mean = sums.x * each;      // of what is in the registers now
                var = __fmaf_rn(-mean, mean, sums.y * each);
                if (var < 0.0f) var = 0.0f;
            }
        } else if (team.at == 0 && mine && a.mean) {
            a.mean[r] = mean;
        }
        var += a.eps;
        float rstd = rsqrtf(var);
        if (var > 1e-30f && var < 1e30f) rstd = __fmaf_rn(0.5f * rstd, __fmaf_rn(-var * rstd, rstd, 1.0f), rstd);    // (a step of Newton's)
        if (mine) {
            const uint64_t by = both(rstd), plus = both(-mean * rstd);
#pragma unroll
            for (int j = 0; j < kGroups; ++j) {
                Cols<kC> w, b;
                const int place = kPlain ? team.at + j * team.size : min(team.at + j * team.size, places - 1);
                read_place(gamma, places, place, w);
                read_place(beta, places, place, b);
#pragma unroll
                for (int i = 0; i < kC / 2; ++i) v[j].p[i] = fma2(fma2(v[j].p[i], by, plus), w.p[i], b.p[i]);
                if (group[j].any) group[j].store(y.group(j), v[j]);
            }
            if (team.at == 0 && a.rstd) a.rstd[r] = rstd;
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
    return with_type(x_type, [&](auto x) {
        return with_type(y_type, [&](auto y) {
            using TX = decltype(x);
            using TY = decltype(y);
            constexpr int kC = kColsOf<TX, TY>;
            Shifts m(kC);
            m.add(a.x, a.ld_x, sizeof(TX));
            m.add(a.y, a.ld_y, sizeof(TY));
            m.add(a.add, a.ld_add, sizeof(TX));
            m.add(a.sum, a.ld_sum, sizeof(TX));
            const TeamShape s = team_shape(m, a.rows, a.cols, (int)sizeof(TX) * (a.add ? 2 : 1), 2, 3, 4, 0, 0, true);
            return with_shape<kC, sizeof(TX) == 2>(s, [&](auto feed, auto groups, auto threads, auto plain) -> deft_status {
                constexpr Feed kFeed = decltype(feed)::value;
                constexpr int kGroups = decltype(groups)::value, kThreads = decltype(threads)::value;
                constexpr bool kPlain = decltype(plain)::value;
                auto kernel = k_layer_norm<false, TX, TY, kFeed, kGroups, kThreads, kPlain>;
                if constexpr (kGroups * kC != 24)        // (24 columns a thread: of one 16-bit matrix)
                    if (a.add) kernel = k_layer_norm<true, TX, TY, kFeed, kGroups, kThreads, kPlain>;
                if (s.smem > 40 * 1024) DEFT_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMostSmem));
                kernel<<<s.blocks, s.threads, s.smem, stream>>>(a, s);
                DEFT_CUDA_TRY(cudaGetLastError());
                return DEFT_OK;
            });
        });
    });
}

}  // namespace deft
