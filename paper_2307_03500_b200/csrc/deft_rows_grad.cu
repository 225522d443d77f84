// The embedding's gradient: the rows of the incoming gradient summed by token.
//
// 1. k_group_tokens puts the token positions in order of their table rows (positions of one row ascending) and
//    writes, per table row, where its positions start and how many there are.
// 2. k_rows_reduce adds up each row's tokens in fp32, in an order that does not depend on how the work was
//    scheduled.
#include "deft_rows.cuh"

namespace deft {
namespace {

// ---- 1. grouping ----
// Table row v belongs to CTA v % kOwners.  Every CTA reads all ids (they stay in L2) and keeps its own: no CTA
// needs anything from another, so there is no barrier over the grid and no pass over global counters.  Inside
// the CTA warp w takes the w-th contiguous part of the tokens, so "warp, then place in the warp's part" is the
// order of the positions; a table of counts per (warp, row) turns into places by a prefix over the warps and one
// over the rows.
constexpr int kOwners = 128;                 // CTAs (a power of two below the 148 SMs)
constexpr int kListCap = 128;                // own tokens a warp remembers; one that has more reads the ids again
constexpr size_t kGroupSmem = 220 * 1024;

struct GroupOut {
    uint2* sorted;      // [n] (table row, token position)
    uint2* row_tab;     // [rows] (first place in sorted, tokens)
    uint32_t* total;    // tokens in sorted: those whose id is a row of the table and not the one left out
    uint32_t* arrived;  // the second kernel's counters, cleared here
    size_t arrived_n;
};

inline size_t group_smem(int warps, int64_t per_cta) {
    return sizeof(uint32_t) * (size_t)(warps + 1) * (size_t)per_cta + sizeof(uint2) * (size_t)kListCap * (size_t)warps + 256 + sizeof(uint32_t) * 64;
}

template <typename Id>
__global__ void __launch_bounds__(1024) k_group_tokens(const Id* __restrict__ ids, uint32_t n, int64_t rows, int64_t skip_id,
                                                        int per_cta, const GroupOut out) {
    extern __shared__ __align__(16) unsigned char smem[];
    const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t me = blockIdx.x, lt = (1u << lane) - 1u;
    uint2* list = reinterpret_cast<uint2*>(smem) + warp * kListCap;
    uint32_t* cnt = reinterpret_cast<uint32_t*>(smem + sizeof(uint2) * kListCap * warps);   // [warps][per_cta]
    uint32_t* start = cnt + (size_t)warps * per_cta;                                        // [per_cta]
    uint32_t* red = start + per_cta;                                                        // [2][32]
    asm volatile("griddepcontrol.launch_dependents;");
    for (int i = threadIdx.x; i < warps * per_cta; i += blockDim.x) cnt[i] = 0u;
    for (size_t i = (size_t)me * blockDim.x + threadIdx.x; i < out.arrived_n; i += (size_t)kOwners * blockDim.x) out.arrived[i] = 0u;
    __syncthreads();
    uint32_t* mine = cnt + (size_t)warp * per_cta;
    const uint32_t part = (n + warps - 1) / warps;
    const uint32_t lo = min((uint32_t)warp * part, n), hi = min(lo + part, n);
    uint32_t below = 0, have = 0;   // valid tokens of lower CTAs (per lane); own tokens of this warp
    for (uint32_t p = lo; p < hi; p += 256) {
        Id v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t pos = p + j * 32 + lane;
            v[j] = pos < hi ? __ldg(ids + pos) : (Id)-1;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int64_t id = (int64_t)v[j];
            const bool ok = id >= 0 && id < rows && id != skip_id;
            const uint32_t owner = (uint32_t)id & (kOwners - 1);
            below += ok && owner < me;
            const bool own = ok && owner == me;
            const uint32_t mask = __ballot_sync(0xffffffffu, own);
            if (own) {
                const uint32_t r = (uint32_t)(id / kOwners), at = have + __popc(mask & lt);
                atomicAdd(mine + r, 1u);
                if (at < kListCap) list[at] = make_uint2(r, p + j * 32 + lane);
            }
            have += __popc(mask);
        }
    }
    below = __reduce_add_sync(0xffffffffu, below);
    if (lane == 0) red[warp] = below;
    __syncthreads();
    // counts -> places: over the warps for each row, then over the rows (a contiguous chunk per thread)
    const int chunk = (per_cta + (int)blockDim.x - 1) / (int)blockDim.x;
    const int r0 = min((int)threadIdx.x * chunk, per_cta), r1 = min(r0 + chunk, per_cta);
    uint32_t sum = 0;
    for (int r = r0; r < r1; ++r) {
        uint32_t run = 0;
        for (int w = 0; w < warps; ++w) {
            const uint32_t c = cnt[(size_t)w * per_cta + r];
            cnt[(size_t)w * per_cta + r] = run;
            run += c;
        }
        start[r] = run;
        sum += run;
    }
    uint32_t incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t x = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += x;
    }
    if (lane == 31) red[32 + warp] = incl;
    __syncthreads();
    uint32_t at = incl - sum;
    for (int w = 0; w < warps; ++w) {
        at += red[w];                            // the tokens of lower CTAs
        if (w < warp) at += red[32 + w];
    }
    for (int r = r0; r < r1; ++r) {
        const uint32_t c = start[r];
        start[r] = at;
        const int64_t row = (int64_t)r * kOwners + me;
        if (row < rows) out.row_tab[row] = make_uint2(at, c);
        at += c;
    }
    if (me == kOwners - 1 && threadIdx.x == blockDim.x - 1) *out.total = at;
    __syncthreads();
    // each warp puts its tokens in place, 32 at a time in order of position
    const bool again = have > kListCap;
    const uint32_t steps = again ? hi - lo : have;
    for (uint32_t i0 = 0; i0 < steps; i0 += 32) {
        const uint32_t i = i0 + lane;
        uint32_t r = 0xffffffffu, pos = 0;
        if (!again) {
            if (i < have) { r = list[i].x; pos = list[i].y; }
        } else if (i < steps) {
            pos = lo + i;
            const int64_t id = (int64_t)__ldg(ids + pos);
            if (id >= 0 && id < rows && id != skip_id && ((uint32_t)id & (kOwners - 1)) == me) r = (uint32_t)(id / kOwners);
        }
        const uint32_t same = __match_any_sync(0xffffffffu, r);
        if (r != 0xffffffffu) {
            const uint32_t place = start[r] + mine[r] + __popc(same & lt);
            out.sorted[place] = make_uint2(r * kOwners + me, pos);
        }
        __syncwarp();
        if (r != 0xffffffffu && (same & lt) == 0) mine[r] += __popc(same);
        __syncwarp();
    }
}

// ---- 2. the sums ----
// The grouped tokens are cut into units of kUnit consecutive ones, whatever rows they belong to: every unit is the
// same work, and all its loads are known from the start (a warp per row would wait for one token's load after the
// other, and a frequent token's row would keep one warp busy for the whole launch).  A warp takes one unit and 256
// columns, eight per lane.  Runs of one row that lie inside a unit are finished there.  A run that crosses units
// leaves a partial sum per unit; the warp that arrives last at the run's counter adds them in order (in two levels of
// kJoin when there are more), so the bits do not depend on the order of arrival.
constexpr int kReduceThreads = 256;
constexpr int kJoin = 32;        // units whose partial sums one warp adds up
constexpr int kDeep = 4;         // tokens whose loads a warp has in flight
constexpr int kZeroRows = 8;     // rows a warp clears if they have no tokens

struct ReduceArgs {
    const uint2* sorted;
    const uint2* row_tab;
    const uint32_t* total;
    float* partial;              // [2 * units][slices * 256]: a unit's first run (even) and last run (odd)
    uint32_t* arrived;           // [2][2 * units * slices]: units of a group, groups of a run
    int unit, units, slices;
};

__device__ __forceinline__ float4 load_cg(const float* p) { return __ldcg(reinterpret_cast<const float4*>(p)); }

// Adds one row's 8 columns to the gradient (or writes them).
template <int kGradAlign>
__device__ __forceinline__ void emit8(float* dst, int count, const float (&sum)[kGroup], const float (&old)[kGroup], float factor, bool accumulate) {
    float g[kGroup];
#pragma unroll
    for (int c = 0; c < kGroup; ++c) {
        g[c] = __fmul_rn(sum[c], factor);
        if (accumulate) g[c] = __fadd_rn(old[c], g[c]);
    }
    store8<float, kGradAlign>(dst, count, g);
}

template <typename T, int kAlign, int kGradAlign>
__global__ void __launch_bounds__(kReduceThreads) k_rows_reduce(const EmbedGradArgs a, const ReduceArgs r) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = threadIdx.x & 31;
    const int64_t task = (int64_t)blockIdx.x * (kReduceThreads / 32) + (threadIdx.x >> 5);
    const int64_t reduce_tasks = (int64_t)r.units * r.slices;
    if (task >= reduce_tasks) {
        // rows without tokens, where the gradient is written
        if (a.accumulate) return;
        const int64_t row0 = (task - reduce_tasks) * kZeroRows;
        const bool empty = lane < kZeroRows && row0 + lane < a.rows && r.row_tab[row0 + lane].y == 0;
        for (uint32_t m = __ballot_sync(0xffffffffu, empty); m; m &= m - 1) {
            float* dst = a.grad + (row0 + __ffs((int)m) - 1) * a.width;
            const float zero[kGroup] = {};
            for (int64_t col = lane * kGroup; col < a.width; col += 32 * kGroup)
                store8<float, kGradAlign>(dst + col, a.width - col < kGroup ? (int)(a.width - col) : kGroup, zero);
        }
        return;
    }
    const int unit_id = (int)(task / r.slices), slice = (int)(task - (int64_t)unit_id * r.slices);
    const uint32_t total = *r.total, first = (uint32_t)unit_id * (uint32_t)r.unit;
    if (first >= total) return;
    const int have = (int)min(total - first, (uint32_t)r.unit);
    const uint2 item = lane < have ? r.sorted[first + lane] : make_uint2(0xffffffffu, 0u);
    const uint32_t before = first > 0 ? r.sorted[first - 1].x : 0xffffffffu;
    const uint32_t after = first + have < total ? r.sorted[first + have].x : 0xffffffffu;
    const uint32_t next_row = __shfl_down_sync(0xffffffffu, item.x, 1);
    const uint32_t ends = __ballot_sync(0xffffffffu, lane < have && (lane == have - 1 || next_row != item.x));
    const bool open_front = before == __shfl_sync(0xffffffffu, item.x, 0);
    const bool open_back = after == __shfl_sync(0xffffffffu, item.x, have - 1);
    const int first_end = __ffs((int)ends) - 1;

    const uint32_t group = (uint32_t)slice * 32 + lane;
    const int64_t col = (int64_t)group * kGroup;
    const int count = col >= a.width ? 0 : (a.width - col < kGroup ? (int)(a.width - col) : kGroup);
    const uint64_t offset = drop_offset(a.drop);
    const T* dy = static_cast<const T*>(a.dy) + col;
    const size_t pitch = (size_t)r.slices * 256;
    float sum[kGroup] = {};
    for (int i0 = 0; i0 < have; i0 += kDeep) {
        float v[kDeep][kGroup], old[kDeep][kGroup];
#pragma unroll
        for (int k = 0; k < kDeep; ++k) {
            const int i = i0 + k;
            const uint32_t pos = __shfl_sync(0xffffffffu, item.y, i & 31), row = __shfl_sync(0xffffffffu, item.x, i & 31);
            if (i < have && count) {
                load8<T, kAlign>(dy + (int64_t)pos * a.ld_dy, count, v[k]);
                const bool closed = !(i == first_end && open_front) && !(i == have - 1 && open_back);
                if (a.accumulate && (ends >> i & 1u) && closed) load8<float, kGradAlign>(a.grad + (int64_t)row * a.width + col, count, old[k]);
            }
        }
#pragma unroll
        for (int k = 0; k < kDeep; ++k) {
            const int i = i0 + k;
            if (i >= have) break;
            const uint32_t pos = __shfl_sync(0xffffffffu, item.y, i), row = __shfl_sync(0xffffffffu, item.x, i);
            if (count) {
                if (a.drop.threshold) drop8<false>(v[k], a.drop, offset, pos, group);
#pragma unroll
                for (int c = 0; c < kGroup; ++c) sum[c] += v[k][c];
            }
            if (!(ends >> i & 1u)) continue;
            const bool front = i == first_end && open_front, back = i == have - 1 && open_back;
            float* dst = a.grad + (int64_t)row * a.width + col;
            if (!front && !back) {
                if (count) emit8<kGradAlign>(dst, count, sum, old[k], a.factor, a.accumulate);
            } else {
                // the run's units are s .. t; this unit's partial sum goes to its odd place where the run starts here
                const uint2 tab = r.row_tab[row];
                const int s = (int)(tab.x / (uint32_t)r.unit), t = (int)((tab.x + tab.y - 1) / (uint32_t)r.unit);
                auto place = [&](int u) { return (size_t)(2 * u + (u == s ? 1 : 0)); };
                float* mine = r.partial + place(unit_id) * pitch + col;
                *reinterpret_cast<float4*>(mine) = make_float4(sum[0], sum[1], sum[2], sum[3]);
                *reinterpret_cast<float4*>(mine + 4) = make_float4(sum[4], sum[5], sum[6], sum[7]);
                // true for the last of `expected` warps to arrive at a place
                auto last_at = [&](size_t at, int level, int expected) {
                    __threadfence();
                    __syncwarp();
                    uint32_t n = 0;
                    if (lane == 0) n = atomicAdd(r.arrived + ((size_t)level * 2 * r.units + at) * r.slices + slice, 1u);
                    n = __shfl_sync(0xffffffffu, n, 0);
                    __threadfence();
                    return n == (uint32_t)(expected - 1);
                };
                // the partial sums of the units u, u + step, ... below end, in order
                auto add_up = [&](int u, int step, int end) {
                    float total8[kGroup] = {};
#pragma unroll 4
                    for (; u < end; u = (u / step + 1) * step) {
                        const float* p = r.partial + place(u) * pitch + col;
                        const float4 x = load_cg(p), y = load_cg(p + 4);
                        total8[0] += x.x; total8[1] += x.y; total8[2] += x.z; total8[3] += x.w;
                        total8[4] += y.x; total8[5] += y.y; total8[6] += y.z; total8[7] += y.w;
                    }
#pragma unroll
                    for (int c = 0; c < kGroup; ++c) sum[c] = total8[c];
                };
                const int u0 = max(s, unit_id / kJoin * kJoin), u1 = min(t + 1, (unit_id / kJoin + 1) * kJoin);
                const int groups = t / kJoin - s / kJoin + 1;
                bool done = false;
                if (last_at(place(u0), 0, u1 - u0)) {
                    add_up(u0, 1, u1);
                    done = groups == 1;
                    if (!done) {
                        float* joined = r.partial + place(u0) * pitch + col;
                        *reinterpret_cast<float4*>(joined) = make_float4(sum[0], sum[1], sum[2], sum[3]);
                        *reinterpret_cast<float4*>(joined + 4) = make_float4(sum[4], sum[5], sum[6], sum[7]);
                        if (last_at(place(s), 1, groups)) {
                            add_up(s, kJoin, t + 1);
                            done = true;
                        }
                    }
                }
                if (done && count) {
                    float was[kGroup];
                    if (a.accumulate) load8<float, kGradAlign>(dst, count, was);
                    emit8<kGradAlign>(dst, count, sum, was, a.factor, a.accumulate);
                }
            }
#pragma unroll
            for (int c = 0; c < kGroup; ++c) sum[c] = 0.0f;
        }
    }
}

// Tokens per unit: 32 where there are enough for every SM's warps, fewer for small calls.
constexpr int64_t kMinTasks = 4096;
inline int unit_of(int64_t n, int64_t slices) {
    int unit = 32;
    while (unit > 4 && (n + unit - 1) / unit * slices < kMinTasks) unit >>= 1;
    return unit;
}
// Upper bound of units * slices over all calls of up to n tokens and up to `slices` slices (unit_of() gives fewer
// tokens more units): what the workspace is sized by, so that it serves smaller calls too.
inline size_t most_tasks(int64_t n, int64_t slices) {
    const int64_t few = (n + 3) / 4 * slices, many = (n + 31) / 32 * slices;
    const int64_t small = few < 2 * kMinTasks + slices ? few : 2 * kMinTasks + slices;
    return (size_t)(small > many ? small : many);
}

struct GradWs { size_t total, row_tab, sorted, arrived, arrived_n, partial, bytes; int unit, units, slices; };
inline GradWs grad_ws(int64_t n, int64_t rows, int64_t width) {
    GradWs w{};
    w.slices = (int)((width + 255) / 256);
    w.unit = unit_of(n, w.slices);
    w.units = (int)((n + w.unit - 1) / w.unit);
    w.arrived_n = 4 * (size_t)w.units * (size_t)w.slices;
    w.total = 0;
    w.row_tab = 256;
    w.sorted = w.row_tab + align_up(sizeof(uint2) * (size_t)rows, 256);
    w.arrived = w.sorted + align_up(sizeof(uint2) * (size_t)n, 256);
    w.partial = w.arrived + align_up(sizeof(uint32_t) * w.arrived_n, 256);
    const size_t most = most_tasks(n, w.slices);
    w.bytes = w.arrived + align_up(sizeof(uint32_t) * 4 * most, 256) + sizeof(float) * 2 * most * 256;
    return w;
}

}  // namespace

size_t embed_grad_ws_bytes(int64_t n, int64_t rows, int64_t width) { return grad_ws(n, rows, width).bytes; }

deft_status launch_embed_grad(const EmbedGradArgs& a, int dy_type, int id_bytes, cudaStream_t stream) {
    const int per_cta = (int)((a.rows + kOwners - 1) / kOwners);
    int warps = 32;
    while (warps > 1 && group_smem(warps, per_cta) > kGroupSmem) warps >>= 1;
    const size_t smem = group_smem(warps, per_cta);
    if (smem > kGroupSmem) return DEFT_ERR_TOO_LARGE;
    const GradWs w = grad_ws(a.n, a.rows, a.width);
    const int64_t tasks = (int64_t)w.units * w.slices + (a.accumulate ? 0 : (a.rows + kZeroRows - 1) / kZeroRows);
    const int64_t blocks = (tasks + kReduceThreads / 32 - 1) / (kReduceThreads / 32);
    if (blocks > 0x7fffffff) return DEFT_ERR_TOO_LARGE;
    GroupOut out{reinterpret_cast<uint2*>(a.ws + w.sorted), reinterpret_cast<uint2*>(a.ws + w.row_tab), reinterpret_cast<uint32_t*>(a.ws + w.total),
                 reinterpret_cast<uint32_t*>(a.ws + w.arrived), w.arrived_n};
    auto group = [&](auto id) -> deft_status {
        using Id = decltype(id);
        DEFT_CUDA_TRY(cudaFuncSetAttribute(k_group_tokens<Id>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kGroupSmem));
        k_group_tokens<Id><<<kOwners, warps * 32, smem, stream>>>(static_cast<const Id*>(a.ids), (uint32_t)a.n, a.rows, a.skip_id, per_cta, out);
        DEFT_CUDA_TRY(cudaGetLastError());
        return DEFT_OK;
    };
    const deft_status s = id_bytes == 8 ? group(int64_t{}) : group(int32_t{});
    if (s != DEFT_OK) return s;
    const ReduceArgs r{out.sorted, out.row_tab, out.total, reinterpret_cast<float*>(a.ws + w.partial), out.arrived, w.unit, w.units, w.slices};
    // The second kernel's CTAs take their places while the first still runs and wait there for its end.
    cudaLaunchAttribute early{};
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(kReduceThreads);
    cfg.stream = stream;
    cfg.attrs = &early;
    cfg.numAttrs = 1;
    auto reduce = [&](auto t, auto al, auto gal) -> deft_status {
        DEFT_CUDA_TRY(cudaLaunchKernelEx(&cfg, k_rows_reduce<decltype(t), decltype(al)::value, decltype(gal)::value>, a, r));
        return DEFT_OK;
    };
    const bool wide = row_align(a.grad, a.width, sizeof(float)) == 16;
    return with_type(dy_type, [&](auto t) {
        return with_align(row_align(a.dy, a.ld_dy, type_bytes(dy_type)), [&](auto al) -> deft_status {
            return wide ? reduce(t, al, AlignTag<16>{}) : reduce(t, al, AlignTag<0>{});
        });
    });
}

}  // namespace deft
