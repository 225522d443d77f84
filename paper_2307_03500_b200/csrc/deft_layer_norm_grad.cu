// The gradient of layer norm.
//
// With h = (x - mean) rstd and d = dy gamma:  dx = rstd (d - mean(d) - h mean(d h)) + add, one pass over the row's registers,
// two sums.  The weight sums dy h and dy stay in registers over all rows of a thread's columns; they leave the CTA once as
// partial sums, and a second kernel adds those in a fixed order: the same bits on every call.  The CTAs of a call of few rows (eight
// CTAs' teams with up to four rows each: 64 rows of 1024 columns, 32 of 1500) are a cluster instead and add up each other's
// sums where they lie (the second launch took a fifth of such a call's time).
//
// Bound by memory: grad_out, x and `add` in, grad_x out, 8 bytes a column for each CTA beside it.  Measured (device time, both
// launches; floor at the copy rate, 6561 GB/s):
//   131072 x 1024 bf16, weight sums added     130 us (6.19 TB/s; floor 122.9)
//   65536 x 1024 bf16, branch                 84.5 us (floor 81.9)                16384 x 1024 fp32, branch  47.4 us (floor 40.9)
//   16384 x 1024 bf16, branch                 28.4 us (floor 20.5: two CTAs an SM start, and 296 CTAs' sums are added up)
//   16384 x 1027 bf16, branch                 40.3 us (floor 20.5: 130 groups take 65 threads with two each, which are three warps, a third
//                                             of whose lanes have nothing; rows of one shift of eight a CTA; elements at the edges)
//   700 x 1500 fp32, branch                   11.2 us (floor 2.6; latency: parameters, four rows a CTA, 175 CTAs' partial sums, the second
//                                             launch, which begins when the first has ended)
//   131072 x 64 bf16                          17.1 us (floor 7.8: a row is a few lanes' work, its reductions and statistics stay)
//   4096 x 16384 bf16                         206 us (floor 61.4), with a branch 325 (81.9); 2048 x 16384 fp32, branch 284 (81.9)
//   16384 x 1024 bf16, branch, one matrix off the others' place in a granule   142 us (floor 20.5: element by element)
// Two CTAs an SM: the sums of sixteen columns in fp32 pairs, the row and its groups take 128 registers, so that bytes in flight
// have to come from the ring, not from warps.  The last two lines' instances have 32 columns a thread and 512 threads, for whose
// state 128 registers are too few (300 to 800 bytes spilled).
#include <cooperative_groups.h>

#include "deft_norm_rows.cuh"

namespace deft {
namespace {

constexpr int kJoinTurns = 4;        // rows a team takes at most, where the call is one cluster
constexpr int kPartials = 2 * 148;   // CTAs that leave partial sums at most; a constant: a call's bits do not depend on the device

template <typename TD, typename TX> constexpr int kColsOf = sizeof(TD) == 4 || sizeof(TX) == 4 ? 4 : 8;

// A column's sum to its place: scaled and rounded, and then (accumulate) added, not both in one operation: what is added is what would
// be written.
__device__ __forceinline__ void store_sum(const LayerNormGradArgs& a, float* out, float sum) {
    sum = __fmul_rn(sum, a.scale);
    *out = a.accumulate ? __fadd_rn(*out, sum) : sum;
}

template <bool kAdd, typename TD, typename TX, Feed kFeed, int kGroups, int kThreads, bool kPlain>
__global__ void __launch_bounds__(kThreads, kThreads == kTeamThreads ? 2 : 1) k_layer_norm_grad(const __grid_constant__ LayerNormGradArgs a, const __grid_constant__ TeamShape shape) {
    extern __shared__ __align__(16) char smem[];         // gamma and room for a second vector (at the end the CTA's sums), the ring
    __shared__ float2 slots[2 * kTeamMostWarps];
    constexpr int kC = kColsOf<TD, TX>;
    using Group = RowGroup<kFeed, kC, kPlain>;
    using RawX = typename Group::template Raw<TX>;
    using RawD = typename Group::template Raw<TD>;
    // bytes of a thread in a stage
    constexpr int kX = kC * (int)sizeof(TX), kD = kC * (int)sizeof(TD), kAtX = kGroups * kD, kAtAdd = kAtX + kGroups * kX, kAll = kAtAdd + (kAdd ? kGroups * kX : 0);
    Team team(shape, kC, slots);
    const int places = shape.places;
    float *params = reinterpret_cast<float*>(smem), *beta = params + places * kC;
    Ring<kThreads, kAll> ring(smem + 2 * sizeof(float) * (size_t)(places * kC), shape.stages);
    const uint32_t rows = (uint32_t)a.rows;
    Group group[kGroups];
#pragma unroll
    for (int j = 0; j < kGroups; ++j) group[j].set(team.at + j * team.size, team.shift, a.cols);
    const int col = team.at * kC - team.shift, across = team.size * kC;
    Walk<const TD> dy(static_cast<const TD*>(a.dy), a.ld_dy, team.row, team.stride, col, across);
    Walk<const TX> x(static_cast<const TX*>(a.x), a.ld_x, team.row, team.stride, col, across);
    Walk<const TX> add(static_cast<const TX*>(a.add), a.ld_add, team.row, team.stride, col, across);
    Walk<TX> dx(static_cast<TX*>(a.dx), a.ld_dx, team.row, team.stride, col, across);
    uint32_t ahead = team.row;
    auto copy = [&](uint32_t stage) {
        if (ahead < rows) {
#pragma unroll
            for (int j = 0; j < kGroups; ++j) {
                group[j].copy(dy.group(j), a.idle, ring.target(stage, j * kD, kD));
                group[j].copy(x.group(j), a.idle, ring.target(stage, kAtX + j * kX, kX));
                if (kAdd) group[j].copy(add.group(j), a.idle, ring.target(stage, kAtAdd + j * kX, kX));
            }
        }
        ring.commit();
        ahead += team.stride;
        dy.next();
        x.next();
        if (kAdd) add.next();
    };
    if constexpr (kFeed == Feed::kRing)
        for (uint32_t s = 0; s != ring.fill; s += ring.kStage) copy(s);
    float next_mean = 0.0f, next_rstd = 0.0f;
    if (team.row < rows) {
        next_mean = a.mean[team.row];
        next_rstd = a.rstd[team.row];
    }
    fill_places<kC>(params, a.gamma, a.w_type, a.cols, places, team.shift, 1.0f);
    __syncthreads();
    const float each = 1.0f / (float)a.cols;
    Cols<kC> dg[kGroups] = {}, db[kGroups] = {};
    uint32_t turn_row = team.row - (uint32_t)team.team * (uint32_t)shape.step;
    for (uint32_t r = team.row; turn_row < rows; turn_row += team.stride, r += team.stride) {
        const bool mine = r < rows;
        const uint64_t minus_mean = both(-next_mean), by = both(next_rstd);
        if (r + team.stride < rows) {
            next_mean = a.mean[r + team.stride];
            next_rstd = a.rstd[r + team.stride];
        }
        if constexpr (kFeed == Feed::kRing) {
            copy(ring.fill);
            ring.wait();
        }
        Cols<kC> h[kGroups], d[kGroups];
        uint64_t c1 = 0, c2 = 0;
#pragma unroll
        for (int j = 0; j < kGroups; ++j) {
            RawX raw_x;
            RawD raw_d;
            if constexpr (kFeed == Feed::kRing) {
                ring.read(j * kD, raw_d);
                ring.read(kAtX + j * kX, raw_x);
            } else if (mine) {
                group[j].load(dy.group(j), raw_d);
                group[j].load(x.group(j), raw_x);
            }
            d[j].from(raw_d);
            h[j].from(raw_x);
#pragma unroll
            for (int i = 0; i < kC / 2; ++i) h[j].p[i] = mul2(add2(h[j].p[i], minus_mean), by);
            // What lies behind the row's end has come as zeros, for which d's are enough; what lies before it, in a thread's first group alone,
            // may be no number and is cleared in both.
            if (j == 0 || kFeed != Feed::kRing) {
                group[j].clear(h[j]);
                group[j].clear(d[j]);
            }
            if (mine) {
#pragma unroll
                for (int i = 0; i < kC / 2; ++i) {
                    db[j].p[i] = add2(db[j].p[i], d[j].p[i]);
                    dg[j].p[i] = fma2(d[j].p[i], h[j].p[i], dg[j].p[i]);
                }
            }
            Cols<kC> w;
            read_place(params, places, kPlain ? team.at + j * team.size : min(team.at + j * team.size, places - 1), w);
#pragma unroll
            for (int i = 0; i < kC / 2; ++i) {
                d[j].p[i] = mul2(d[j].p[i], w.p[i]);
                c1 = add2(c1, d[j].p[i]);
                c2 = fma2(d[j].p[i], h[j].p[i], c2);
            }
        }
        if (a.dx) {
            const float2 c = team.sum(folded(c1), folded(c2));
            if (mine) {
                const uint64_t minus_c1 = both(-(c.x * each)), minus_c2 = both(-(c.y * each));
#pragma unroll
                for (int j = 0; j < kGroups; ++j) {
                    if (!group[j].any) continue;
#pragma unroll
                    for (int i = 0; i < kC / 2; ++i) d[j].p[i] = mul2(fma2(h[j].p[i], minus_c2, add2(d[j].p[i], minus_c1)), by);
                    if (kAdd) {
                        RawX raw;
                        Cols<kC> m;
                        if constexpr (kFeed == Feed::kRing) ring.read(kAtAdd + j * kX, raw);
                        else group[j].load(add.group(j), raw);
                        m.from(raw);
#pragma unroll
                        for (int i = 0; i < kC / 2; ++i) d[j].p[i] = add2(d[j].p[i], m.p[i]);
                    }
                    group[j].store(dx.group(j), d[j]);
                }
            }
        }
        dx.next();
        if constexpr (kFeed == Feed::kRing) {
            ring.next();
        } else {
            dy.next();
            x.next();
            if (kAdd) add.next();
        }
    }
    if (!a.dgamma && !a.dbeta) return;
    // a warp's teams, then the teams or warps in order
    int units = team.teams, unit = team.team;
    bool first = true;
    if (team.size < 32) {
        for (int o = team.size; o < 32; o *= 2)
#pragma unroll
            for (int j = 0; j < kGroups; ++j)
#pragma unroll
                for (int i = 0; i < kC / 2; ++i) {
                    dg[j].p[i] = add2(dg[j].p[i], __shfl_xor_sync(0xffffffffu, dg[j].p[i], o));
                    db[j].p[i] = add2(db[j].p[i], __shfl_xor_sync(0xffffffffu, db[j].p[i], o));
                }
        units = (int)blockDim.x >> 5;
        unit = (int)threadIdx.x >> 5;
        first = ((int)threadIdx.x & 31) < team.size;
    }
    for (int t = 0; t < units; ++t) {
        __syncthreads();
        if (t != unit || !first) continue;
#pragma unroll
        for (int j = 0; j < kGroups; ++j) {
            const int place = team.at + j * team.size;
            if (place >= places) break;
            if (t) {
                Cols<kC> was;
                read_place(params, places, place, was);
#pragma unroll
                for (int i = 0; i < kC / 2; ++i) dg[j].p[i] = add2(dg[j].p[i], was.p[i]);
                read_place(beta, places, place, was);
#pragma unroll
                for (int i = 0; i < kC / 2; ++i) db[j].p[i] = add2(db[j].p[i], was.p[i]);
            }
            write_place(params, places, place, dg[j]);
            write_place(beta, places, place, db[j]);
        }
    }
    __syncthreads();
    if (shape.joined) {
        namespace cg = cooperative_groups;
        cg::cluster_group cluster = cg::this_cluster();
        cluster.sync();
        const int ctas = (int)gridDim.x;
        for (int i = (int)(blockIdx.x * blockDim.x + threadIdx.x); i < 2 * a.cols; i += ctas * (int)blockDim.x) {
            const bool second = i >= a.cols;
            const int c = second ? i - a.cols : i;
            float sum = 0.0f;
            for (int b = 0; b < ctas; ++b) {
                const int shift = (shape.first + b % shape.step * shape.ld) & (kC - 1);
                sum += *(cluster.map_shared_rank(second ? beta : params, b) + at_place<kC>(places, c + shift));
            }
            float* out = second ? a.dbeta : a.dgamma;
            if (!out) continue;
            store_sum(a, out + c, sum);
        }
        cluster.sync();                    // nobody leaves while others read its sums
        return;
    }
    // in the order of the columns: CTAs of different shifts meet
    float* out = a.partial + (int64_t)blockIdx.x * 2 * a.cols;
    for (int c = threadIdx.x; c < a.cols; c += blockDim.x) {
        const int i = c + team.shift;
        out[c] = params[at_place<kC>(places, i)];
        out[a.cols + c] = beta[at_place<kC>(places, i)];
    }
}

// The CTAs' partial sums added up: a lane per column, warps that take every kJoinWarps-th CTA's, whose loads are all under way together
// (sixteen warps with eight loads at a time: 16384 x 1024 29.0 us for both launches).
constexpr int kJoinWarps = 32, kJoinLoads = (kPartials + kJoinWarps - 1) / kJoinWarps;
__global__ void __launch_bounds__(kJoinWarps * 32) k_layer_norm_join(const __grid_constant__ LayerNormGradArgs a, const int partials) {
    __shared__ float part[kJoinWarps][32];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t both = 2 * (int64_t)a.cols, at = (int64_t)blockIdx.x * 32 + lane;
    float sum = 0.0f;
    if (at < both) {
        float part_of[kJoinLoads];
#pragma unroll
        for (int i = 0; i < kJoinLoads; ++i) part_of[i] = warp + i * kJoinWarps < partials ? a.partial[(warp + i * kJoinWarps) * both + at] : 0.0f;
#pragma unroll
        for (int i = 0; i < kJoinLoads; ++i) sum += part_of[i];
    }
    part[warp][lane] = sum;
    __syncthreads();
    if (warp || at >= both) return;
#pragma unroll
    for (int w = 1; w < kJoinWarps; ++w) sum += part[w][lane];
    float* out = at < a.cols ? a.dgamma : a.dbeta;
    if (!out) return;
    out += at < a.cols ? at : at - a.cols;
    store_sum(a, out, sum);
}

}  // namespace

size_t layer_norm_grad_ws_bytes(int64_t rows, int64_t cols) {
    // CTAs come in multiples of up to eight
    const int64_t partials = (rows + 7) / 8 * 8 < kPartials ? (rows ? (rows + 7) / 8 * 8 : 1) : kPartials;
    return (size_t)partials * 2 * sizeof(float) * (size_t)cols;
}

deft_status launch_layer_norm_grad(const LayerNormGradArgs& a, int dy_type, int x_type, cudaStream_t stream) {
    unsigned blocks = 0;
    bool joined = false;
    if (a.rows) {
        const deft_status st = with_type(dy_type, [&](auto d) {
            return with_type(x_type, [&](auto x) {
                using TD = decltype(d);
                using TX = decltype(x);
                constexpr int kC = kColsOf<TD, TX>;
                Shifts m(kC);
                m.add(a.x, a.ld_x, sizeof(TX));
                m.add(a.dy, a.ld_dy, sizeof(TD));
                m.add(a.add, a.ld_add, sizeof(TX));
                m.add(a.dx, a.ld_dx, sizeof(TX));
                const TeamShape s = team_shape(m, a.rows, a.cols, (int)(sizeof(TD) + sizeof(TX) * (a.add ? 2 : 1)), 2, 2, 2, kPartials, a.dgamma || a.dbeta ? kJoinTurns : 0, false);
                blocks = s.blocks;
                return with_shape<kC, false>(s, [&](auto feed, auto groups, auto threads, auto plain) -> deft_status {
                    constexpr Feed kFeed = decltype(feed)::value;
                    constexpr int kGroups = decltype(groups)::value, kThreads = decltype(threads)::value;
                    constexpr bool kPlain = decltype(plain)::value;
                    // a ring of rows beyond 8192 columns: of three matrices it has room for a stage where x and `add` have 16 bits
                    constexpr bool kAddToo = kFeed != Feed::kRing || kGroups * kC != 32 || sizeof(TX) == 2;
                    auto kernel = k_layer_norm_grad<false, TD, TX, kFeed, kGroups, kThreads, kPlain>;
                    if constexpr (kAddToo)
                        if (a.add) kernel = k_layer_norm_grad<true, TD, TX, kFeed, kGroups, kThreads, kPlain>;
                    static_assert(kAddToo || kTeamMost * 32 * (sizeof(TD) + 2 * sizeof(TX)) + 2 * sizeof(float) * kTeamMost * 16 > kMostSmem, "no stage fits");
                    if (s.smem > 40 * 1024) DEFT_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMostSmem));
                    joined = s.joined;
                    if (joined) {
                        cudaLaunchAttribute cluster{};
                        cluster.id = cudaLaunchAttributeClusterDimension;
                        cluster.val.clusterDim.x = s.blocks;
                        cluster.val.clusterDim.y = cluster.val.clusterDim.z = 1;
                        cudaLaunchConfig_t cfg{};
                        cfg.gridDim = dim3(s.blocks);
                        cfg.blockDim = dim3((unsigned)s.threads);
                        cfg.dynamicSmemBytes = s.smem;
                        cfg.stream = stream;
                        cfg.attrs = &cluster;
                        cfg.numAttrs = 1;
                        DEFT_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, a, s));
                        return DEFT_OK;
                    }
                    kernel<<<s.blocks, s.threads, s.smem, stream>>>(a, s);
                    DEFT_CUDA_TRY(cudaGetLastError());
                    return DEFT_OK;
                });
            });
        });
        if (st != DEFT_OK) return st;
    }
    if (joined || (!a.dgamma && !a.dbeta)) return DEFT_OK;
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
