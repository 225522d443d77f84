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
// What bounds it: latency.  4.3 us for 700 tokens, 8.6 us for 16384 (one read of the ids, two prefixes, five barriers),
// 4.2 + 10.6 us for 131072 with the splitting pass before it (33.7 without).
// Table row v belongs to CTA v % kOwners.  Every CTA reads all ids (they stay in L2) and keeps its own: no CTA
// needs anything from another, so there is no barrier over the grid and no pass over global counters.  With many
// tokens that reading is most of the work (34 us for 131072), and k_split_tokens orders tiles of them by CTA first.
// Inside the CTA warp w takes the w-th contiguous part of the tokens, so "warp, then place in the warp's part" is the
// order of the positions; a table of counts per (warp, row) turns into places by a prefix over the warps and one
// over the rows.
constexpr int kOwners = 128;                 // CTAs (a power of two below the 148 SMs)
constexpr size_t kGroupSmem = 220 * 1024;
constexpr int kTokenTile = 1024;             // tokens per tile of the splitting pass
constexpr int64_t kSplitFrom = 16384;        // calls of more tokens split first (16384: 3.9 + 6.9 us against 9.2 without, 20000: 11.2 against 12.3, 131072: 14.8 against 33.7)
constexpr int kSplitPitch = kOwners + 2;     // a tile's first entry of every CTA, and their number
constexpr int kListMost = 1024;              // own tokens a warp remembers at most; one that has more reads the ids again

struct GroupOut {
    uint2* sorted;      // [n] (table row, token position)
    uint2* row_tab;     // [rows] (first place in sorted, tokens)
    uint32_t* total;    // tokens in sorted: those whose id is a row of the table and not the one left out
    uint32_t* arrived;  // the second kernel's counters, cleared here
    size_t arrived_n;
};

// Shared memory: [warps][list_cap] (row of the CTA, token) | [warps][per_cta] counts | [per_cta] first places | sums.
inline size_t group_smem(int warps, int64_t per_cta, int list_cap) {
    return sizeof(uint2) * (size_t)list_cap * (size_t)warps + sizeof(uint32_t) * ((size_t)(warps + 1) * (size_t)per_cta + 64);
}

// Puts a tile's tokens in order of their CTAs (tokens of one CTA in order of position) and writes where each CTA's begin.
template <typename Id>
__global__ void __launch_bounds__(256) k_split_tokens(const Id* __restrict__ ids, uint32_t n, uint32_t rows, uint32_t skip, uint2* entries, uint16_t* first) {
    constexpr int kWarps = 8, kEach = kTokenTile / 256;
    __shared__ uint32_t cnt[kWarps][kOwners + 1], start[kOwners + 1], sums[4];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t lt = (1u << lane) - 1u, t0 = blockIdx.x * (uint32_t)kTokenTile;
    for (int i = threadIdx.x; i < kWarps * (kOwners + 1); i += 256) (&cnt[0][0])[i] = 0u;
    uint32_t row[kEach], owner[kEach], rank[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const uint32_t pos = t0 + warp * (kTokenTile / kWarps) + j * 32 + lane;
        row[j] = pos < n ? row_of(__ldg(ids + pos), rows, skip) : kNoRow;
        owner[j] = row[j] == kNoRow ? kOwners : row[j] % kOwners;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const uint32_t same = __match_any_sync(0xffffffffu, owner[j]);
        rank[j] = cnt[warp][owner[j]] + __popc(same & lt);
        __syncwarp();
        if ((same & lt) == 0) cnt[warp][owner[j]] += __popc(same);
        __syncwarp();
    }
    __syncthreads();
    uint32_t total = 0, incl = 0;
    if (threadIdx.x < kOwners) {
        for (int w = 0; w < kWarps; ++w) {
            const uint32_t c = cnt[w][threadIdx.x];
            cnt[w][threadIdx.x] = total;
            total += c;
        }
        incl = total;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t x = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += x;
        }
        if (lane == 31) sums[warp] = incl;
    }
    __syncthreads();
    if (threadIdx.x < kOwners) {
        uint32_t at = incl - total;
        for (int w = 0; w < warp; ++w) at += sums[w];
        start[threadIdx.x] = at;
        first[(size_t)blockIdx.x * kSplitPitch + threadIdx.x] = (uint16_t)at;
        if (threadIdx.x == kOwners - 1) first[(size_t)blockIdx.x * kSplitPitch + kOwners] = (uint16_t)(at + total);
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kEach; ++j)
        if (row[j] != kNoRow)
            entries[t0 + start[owner[j]] + cnt[warp][owner[j]] + rank[j]] = make_uint2(row[j], t0 + warp * (kTokenTile / kWarps) + j * 32 + lane);
}

template <typename Id, bool kSplit>
__global__ void __launch_bounds__(1024) k_group_tokens(const Id* __restrict__ ids, uint32_t n, uint32_t rows, uint32_t skip,
                                                        const uint2* entries, const uint16_t* first, int per_cta, int list_cap,
                                                        const GroupOut out) {
    extern __shared__ __align__(16) unsigned char smem[];
    const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t me = blockIdx.x, lt = (1u << lane) - 1u;
    uint2* list = reinterpret_cast<uint2*>(smem) + warp * list_cap;
    uint32_t* cnt = reinterpret_cast<uint32_t*>(smem + sizeof(uint2) * list_cap * warps);   // [warps][per_cta]
    uint32_t* start = cnt + (size_t)warps * per_cta;                                        // [per_cta]
    uint32_t* red = start + per_cta;                                                        // [2][32]
    for (int i = threadIdx.x; i < warps * per_cta; i += blockDim.x) cnt[i] = 0u;
    for (size_t i = (size_t)me * blockDim.x + threadIdx.x; i < out.arrived_n; i += (size_t)kOwners * blockDim.x) out.arrived[i] = 0u;
    __syncthreads();
    if (kSplit) asm volatile("griddepcontrol.wait;" ::: "memory");
    uint32_t* mine = cnt + (size_t)warp * per_cta;
    // this warp's part: tokens, or whole tiles of them
    constexpr uint32_t kStep = kSplit ? kTokenTile : 1;
    const uint32_t steps_all = (n + kStep - 1) / kStep, part = (steps_all + warps - 1) / warps;
    const uint32_t lo = min((uint32_t)warp * part, steps_all), hi = min(lo + part, steps_all);
    uint32_t below = 0, have = 0;   // valid tokens of lower CTAs (per lane); own tokens of this warp
    auto keep = [&](uint32_t r, uint32_t pos, uint32_t at) {
        atomicAdd(mine + r, 1u);
        if (at < (uint32_t)list_cap) list[at] = make_uint2(r, pos);
    };
    if constexpr (kSplit) {
        constexpr int kAhead = 8;
        for (uint32_t t = lo; t < hi; t += kAhead) {
            uint32_t a[kAhead], c[kAhead];
            uint2 e[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                a[j] = c[j] = 0;
                if (t + j < hi) {
                    a[j] = first[(size_t)(t + j) * kSplitPitch + me];
                    c[j] = first[(size_t)(t + j) * kSplitPitch + me + 1] - a[j];
                }
            }
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
                if ((uint32_t)lane < c[j]) e[j] = entries[(size_t)(t + j) * kTokenTile + a[j] + lane];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                if (lane == 0) below += a[j];
                if ((uint32_t)lane < c[j]) keep(e[j].x / kOwners, e[j].y, have + lane);
                for (uint32_t i = 32 + lane; i < c[j]; i += 32) {
                    const uint2 x = entries[(size_t)(t + j) * kTokenTile + a[j] + i];
                    keep(x.x / kOwners, x.y, have + i);
                }
                have += c[j];
            }
        }
    } else {
        constexpr int kAhead = 16;
        for (uint32_t p = lo; p < hi; p += 32 * kAhead) {
            uint32_t row[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const uint32_t pos = p + j * 32 + lane;
                row[j] = pos < hi ? row_of(__ldg(ids + pos), rows, skip) : kNoRow;
            }
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const uint32_t owner = row[j] % kOwners;
                below += row[j] != kNoRow && owner < me;
                const bool own = row[j] != kNoRow && owner == me;
                const uint32_t mask = __ballot_sync(0xffffffffu, own);
                if (own) keep(row[j] / kOwners, p + j * 32 + lane, have + __popc(mask & lt));
                have += __popc(mask);
            }
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
        const uint32_t row = (uint32_t)r * kOwners + me;
        if (row < rows) out.row_tab[row] = make_uint2(at, c);
        at += c;
    }
    if (me == kOwners - 1 && threadIdx.x == blockDim.x - 1) *out.total = at;
    __syncthreads();
    // each warp puts its tokens in place, 32 at a time in order of position
    __syncwarp();
    auto place32 = [&](uint32_t r, uint32_t pos) {      // r = kNoRow: nothing in this lane
        const uint32_t same = __match_any_sync(0xffffffffu, r);
        if (r != kNoRow) out.sorted[start[r] + mine[r] + __popc(same & lt)] = make_uint2(r * kOwners + me, pos);
        __syncwarp();
        if (r != kNoRow && (same & lt) == 0) mine[r] += __popc(same);
        __syncwarp();
    };
    if (have <= (uint32_t)list_cap) {
        for (uint32_t i = 0; i < have; i += 32) {
            const bool some = i + lane < have;
            place32(some ? list[i + lane].x : kNoRow, some ? list[i + lane].y : 0u);
        }
    } else if constexpr (kSplit) {                      // more than the list holds: the entries once more
        for (uint32_t t = lo; t < hi; ++t) {
            const uint32_t a = first[(size_t)t * kSplitPitch + me], c = first[(size_t)t * kSplitPitch + me + 1] - a;
            for (uint32_t i = 0; i < c; i += 32) {
                uint2 e = make_uint2(kNoRow, 0u);
                if (i + lane < c) e = entries[(size_t)t * kTokenTile + a + i + lane];
                place32(e.x == kNoRow ? kNoRow : e.x / kOwners, e.y);
            }
        }
    } else {                                            // ... or the ids
        for (uint32_t p = lo; p < hi; p += 32) {
            const uint32_t row = p + lane < hi ? row_of(__ldg(ids + p + lane), rows, skip) : kNoRow;
            place32(row != kNoRow && row % kOwners == me ? row / kOwners : kNoRow, p + lane);
        }
    }
}

// ---- 2. the sums ----
// G[v] = factor * sum of the kept elements of v's tokens.  The grouped tokens are cut into units of consecutive ones,
// whatever rows they belong to: every unit is the same work, and all its loads are known from the start (a warp per row
// waits for one token's load after the other, and a frequent token's row keeps one warp busy for the whole launch:
// 4.9 ms instead of 0.12 at 131072 x 1024).  A warp takes one unit and 256 columns, eight per lane.  Its tokens' slices,
// and where the gradient is added the target rows', come through a ring of asynchronous copies in shared memory: the
// loads in flight do not cost registers (with them in registers the kernel spilled, or ran on half the warps: 0.15 to
// 0.33 ms).  Runs of one row that lie inside a unit are finished there.  A run that crosses units leaves a partial sum per
// unit; the warp that arrives last at the run's counter adds them in order (in two levels of kJoin when there are
// more), so the bits do not depend on the order of arrival.
//
// What bounds it, 131072 x 1024 bf16 added with dropout: 103 us for 464 MB, 0.70 of the measured copy rate; the
// schedulers issue in 68 % of the cycles (137 instructions per token and 256 columns, 34 of them the generator's
// products and exclusive ors); no single resource is full.  The whole call takes 116 us, 109 without
// dropout, 218 with fp32 input (floor 113).  Small calls are bound by latency: 9 us for 700 x 1500, of which a third is the joins.
constexpr int kReduceThreads = 128;
constexpr int kReduceBlocks = 8; // CTAs an SM holds (64 registers a thread; with 48 it spills)
constexpr int kJoin = 32;        // units whose partial sums one warp adds up
constexpr int kClearing = 2;     // clearing CTAs per SM beside many sums
constexpr int kRing = 6144;      // bytes of shared memory a warp's copies go to: 192 KB on an SM

struct ReduceArgs {
    const uint2* sorted;
    const uint2* row_tab;
    const uint32_t* total;
    float* partial;              // [2 * units][slices * 256]: a unit's first run (even) and last run (odd)
    uint32_t* arrived;           // [2][2 * units * slices]: units of a group, groups of a run
    int unit, units, slices;
    int clear_blocks;            // CTAs that clear rows (0 where the gradient is added)
};

// How a warp shares out the 256 columns of its slice.  kWide (rows of both matrices start on 16-byte boundaries): eight
// per lane side by side, and a lane copies and reads its own bytes only.  Else they are dealt out one by one (lane l has
// the columns 32 k + l), the warp copies the 16-byte granules that the slice lies in, and the lanes read at its offset.
// left: columns from the lane's first one (kWide) or the slice's first one (else) to the row's end, 256 at most.
template <bool kWide>
__device__ __forceinline__ int lane_first() { return kWide ? (int)(threadIdx.x & 31) * kGroup : 0; }

template <bool kWide>
__device__ __forceinline__ void store_slice(float* p, int left, const float (&v)[kGroup]) {
    if constexpr (kWide) {   // the width is a multiple of four
        if (left > 4 && (reinterpret_cast<uintptr_t>(p) & 31) == 0) {   // one store of whole sectors instead of two of half ones
            store32(p, v);
            return;
        }
        if (left > 0) reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
        if (left > 4) reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
        store_dealt<false>(p, left, v);
    }
}

__device__ __forceinline__ void copy16(void* to, const void* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kPending>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kPending) : "memory"); }

// Room for one slice of a row, and the copy into it and the reading of it.
template <typename T, bool kWide>
struct Slot {
    static constexpr int kBytes = 256 * (int)sizeof(T) + (kWide ? 0 : 16);
    static __device__ __forceinline__ void copy(char* slot, const T* p, int left) {
        const int lane = threadIdx.x & 31;
        if constexpr (kWide) {
            constexpr int per = 16 / (int)sizeof(T);
#pragma unroll
            for (int i = 0; i < kGroup / per; ++i)
                if (i * per < left) copy16(slot + (i * 32 + lane) * 16, p + i * per);   // (no bank twice in a quarter-warp)
        } else {
            const char* from = reinterpret_cast<const char*>(reinterpret_cast<uintptr_t>(p) & ~(uintptr_t)15);
            const int bytes = (int)(reinterpret_cast<const char*>(p) - from) + left * (int)sizeof(T);
#pragma unroll
            for (int i = 0; i < (kBytes + 511) / 512; ++i)
                if ((i * 32 + lane) * 16 < bytes) copy16(slot + (i * 32 + lane) * 16, from + (i * 32 + lane) * 16);
        }
    }
    static __device__ __forceinline__ void read(const char* slot, uint32_t at, int left, T (&v)[kGroup]) {   // at: the slice's address
        const int lane = threadIdx.x & 31;
        if constexpr (kWide) {
            Raw8<T, 16> raw;
#pragma unroll
            for (int i = 0; i < Raw8<T, 16>::kPieces; ++i) raw.piece[i] = *reinterpret_cast<const uint4*>(slot + (i * 32 + lane) * 16);
#pragma unroll
            for (int i = 0; i < kGroup; ++i) v[i] = reinterpret_cast<const T*>(raw.piece)[i];
        } else {
            const T* e = reinterpret_cast<const T*>(slot + (at & 15u)) + lane;
#pragma unroll
            for (int k = 0; k < kGroup; ++k) v[k] = k * 32 + lane < left ? e[k * 32] : from_f32<T>(0.0f);
        }
    }
};

// One row's columns: its tokens' sum times the factor, written or added to what was there.
template <bool kAdd, bool kWide>
__device__ __forceinline__ void emit(float* dst, int left, const float (&sum)[kGroup], const float (&was)[kGroup], float factor) {
    float g[kGroup];
#pragma unroll
    for (int c = 0; c < kGroup; ++c) {
        g[c] = __fmul_rn(sum[c], factor);
        if (kAdd) g[c] = __fadd_rn(was[c], g[c]);
    }
    store_slice<kWide>(dst, left, g);
}

// A run that crosses units leaves a partial sum in each: at the unit's odd place where the run starts in it, else at its
// even one.
__device__ __forceinline__ float4* partial_at(const ReduceArgs& r, int unit, bool starts, int slice) {
    return reinterpret_cast<float4*>(r.partial + (size_t)(2 * unit + (starts ? 1 : 0)) * (size_t)r.slices * 256 + (size_t)slice * 256 +
                                     (threadIdx.x & 31) * kGroup);
}
__device__ __forceinline__ void leave(float4* at, const float (&sum)[kGroup]) {
    at[0] = make_float4(sum[0], sum[1], sum[2], sum[3]);
    at[1] = make_float4(sum[4], sum[5], sum[6], sum[7]);
}

// The warp has left its unit's partial sum of a run: the last one to arrive adds them all up.
template <bool kAdd, bool kWide>
__device__ __forceinline__ void join(const EmbedGradArgs& a, const ReduceArgs& r, uint32_t row, int unit_id, int slice, int left) {
    const int lane = threadIdx.x & 31;
    const uint2 tab = r.row_tab[row];
    const int s = (int)(tab.x / (uint32_t)r.unit), t = (int)((tab.x + tab.y - 1) / (uint32_t)r.unit);   // the run's units
    float sum[kGroup];
    // true for the last of `expected` warps to arrive at a unit's place
    auto last_at = [&](int u, int level, int expected) {
        __threadfence();
        __syncwarp();
        uint32_t n = 0;
        if (lane == 0) n = atomicAdd(r.arrived + ((size_t)level * 2 * r.units + 2 * u + (u == s ? 1 : 0)) * r.slices + slice, 1u);
        if (__shfl_sync(0xffffffffu, n, 0) != (uint32_t)(expected - 1)) return false;
        __threadfence();
        return true;
    };
    // the partial sums of the units u, the next multiple of step, ... below end, in order
    auto add_up = [&](int u, int step, int end) {
        float4 lo = make_float4(0.0f, 0.0f, 0.0f, 0.0f), hi = lo;
#pragma unroll 4
        for (; u < end; u = (u / step + 1) * step) {
            const float4* at = partial_at(r, u, u == s, slice);
            const float4 x = __ldcg(at), y = __ldcg(at + 1);
            lo.x += x.x; lo.y += x.y; lo.z += x.z; lo.w += x.w;
            hi.x += y.x; hi.y += y.y; hi.z += y.z; hi.w += y.w;
        }
        sum[0] = lo.x; sum[1] = lo.y; sum[2] = lo.z; sum[3] = lo.w;
        sum[4] = hi.x; sum[5] = hi.y; sum[6] = hi.z; sum[7] = hi.w;
    };
    const int u0 = max(s, unit_id / kJoin * kJoin), u1 = min(t + 1, (unit_id / kJoin + 1) * kJoin);
    const int groups = t / kJoin - s / kJoin + 1;
    if (!last_at(u0, 0, u1 - u0)) return;
    add_up(u0, 1, u1);
    if (groups > 1) {
        leave(partial_at(r, u0, u0 == s, slice), sum);
        if (!last_at(s, 1, groups)) return;
        add_up(s, kJoin, t + 1);
    }
    float* dst = a.grad + (int64_t)row * a.width + (int64_t)slice * 256 + lane_first<kWide>();
    float was[kGroup];
    if (kAdd) {
#pragma unroll
        for (int c = 0; c < kGroup; ++c) {
            const int i = kWide ? c : c * 32 + lane;
            was[c] = i < left ? dst[i] : 0.0f;
        }
    }
    emit<kAdd, kWide>(dst, left, sum, was, a.factor);
}

// Rows without tokens, where the gradient is written.  A warp looks up as many rows as make 4 KB, clears those without
// tokens, and goes on: with kClearing CTAs on each SM that is some three quarters of the memory's rate, and the other
// CTAs' reads get through.  (Looking up 32 rows ahead clears faster and the call takes longer: 16384 x 1024 into
// 30522 rows 45 to 53 us, against 42.)
template <bool kWide>
__device__ __forceinline__ void clear_rows(const EmbedGradArgs& a, const ReduceArgs& r, int warp, int warps) {
    const int lane = threadIdx.x & 31, some = max(1, min(32, (int)(1024 / a.width)));
    for (int64_t row0 = (int64_t)warp * some; row0 < a.rows; row0 += (int64_t)warps * some) {
        const bool empty = lane < some && row0 + lane < a.rows && r.row_tab[row0 + lane].y == 0;
        for (uint32_t m = __ballot_sync(0xffffffffu, empty); m; m &= m - 1) {
            float* dst = a.grad + (row0 + __ffs((int)m) - 1) * a.width;
            if constexpr (kWide)
                for (int64_t col = lane * 4; col < a.width; col += 128) *reinterpret_cast<float4*>(dst + col) = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            else
                for (int64_t col = lane; col < a.width; col += 32) dst[col] = 0.0f;
        }
    }
}

template <bool kAdd, typename T, bool kWide>
__global__ void __launch_bounds__(kReduceThreads, kReduceBlocks) k_rows_reduce(const __grid_constant__ EmbedGradArgs a, const __grid_constant__ ReduceArgs r) {
    // a warp's ring of slots: a token's slice and, where the gradient is added, the row's own
    constexpr int kSlot = Slot<T, kWide>::kBytes + (kAdd ? Slot<float, kWide>::kBytes : 0);
    constexpr int kSlots = kRing / kSlot > 8 ? 8 : kRing / kSlot;
    static_assert(kSlots >= 2, "a slot in use and one on its way");
    __shared__ __align__(16) char ring_all[kReduceThreads / 32][kSlots * kSlot];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = threadIdx.x & 31;
    // the first CTAs clear, some on each SM: they write while the others wait for what they read
    if (!kAdd && (int)blockIdx.x < r.clear_blocks) {
        constexpr int kWarps = kReduceThreads / 32;
        clear_rows<kWide>(a, r, (int)blockIdx.x * kWarps + (int)(threadIdx.x >> 5), r.clear_blocks * kWarps);
        return;
    }
    const int64_t block = (int64_t)blockIdx.x - r.clear_blocks;
    const int64_t task = block * (kReduceThreads / 32) + (threadIdx.x >> 5);
    if (task >= (int64_t)r.units * r.slices) return;
    const int unit_id = (int)(task / r.slices), slice = (int)(task - (int64_t)unit_id * r.slices);
    const uint32_t total = *r.total, first = (uint32_t)unit_id * (uint32_t)r.unit;
    if (first >= total) return;
    const int have = (int)min(total - first, (uint32_t)r.unit);
    const uint2 item = lane < have ? r.sorted[first + lane] : make_uint2(kNoRow, 0u);
    const uint32_t before = first > 0 ? r.sorted[first - 1].x : kNoRow;
    const uint32_t after = first + have < total ? r.sorted[first + have].x : kNoRow;
    const uint32_t next_row = __shfl_down_sync(0xffffffffu, item.x, 1);
    // where runs end, and which of them lie inside the unit
    const uint32_t ends = __ballot_sync(0xffffffffu, lane < have && (lane == have - 1 || next_row != item.x));
    uint32_t closed = ends;
    const bool from_before = before == __shfl_sync(0xffffffffu, item.x, 0);
    if (from_before) closed &= closed - 1;
    if (after == __shfl_sync(0xffffffffu, item.x, have - 1)) closed &= ~(1u << (have - 1));

    const int64_t col = (int64_t)slice * 256 + lane_first<kWide>();
    const int left = (int)max(min(a.width - col, (int64_t)256), (int64_t)0);
    const uint64_t offset = drop_offset(a.drop);
    const T* dy = static_cast<const T*>(a.dy) + col;
    float* grad = a.grad + col;
    char* ring = ring_all[threadIdx.x >> 5];
    auto token = [&](int i) { return dy + (int64_t)__shfl_sync(0xffffffffu, item.y, i) * a.ld_dy; };
    auto target = [&](int i) { return grad + (int64_t)__shfl_sync(0xffffffffu, item.x, i) * a.width; };
    auto start = [&](int i, int slot) {      // everything token i needs, as one group of copies (an empty one behind the last)
        if (i < have) {
            Slot<T, kWide>::copy(ring + slot * kSlot, token(i), left);
            if (kAdd && (closed >> i & 1u)) Slot<float, kWide>::copy(ring + slot * kSlot + Slot<T, kWide>::kBytes, target(i), left);
        }
        copies_end();
    };
    for (int i = 0; i < kSlots; ++i) start(i, i);
    float sum[kGroup] = {};
    for (int i = 0, slot = 0; i < have; ++i, slot = slot + 1 < kSlots ? slot + 1 : 0) {
        copies_wait<kSlots - 1>();
        if (!kWide) __syncwarp();            // other lanes' copies are read
        T x[kGroup];
        const uint32_t pos = __shfl_sync(0xffffffffu, item.y, i);
        Slot<T, kWide>::read(ring + slot * kSlot, (uint32_t)reinterpret_cast<uintptr_t>(dy) + pos * (uint32_t)a.ld_dy * (uint32_t)sizeof(T), left, x);
        if (a.drop.threshold) {
            if constexpr (kWide) {
                const uint4 w = drop_words(a.drop, offset, pos, (uint32_t)slice * 32 + lane);
                const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    bool even, odd;
                    kept2(u[c], a.drop.threshold, even, odd);
                    if (even) sum[2 * c] = add_elem(sum[2 * c], x[2 * c]);
                    if (odd) sum[2 * c + 1] = add_elem(sum[2 * c + 1], x[2 * c + 1]);
                }
            } else {
                for_kept_dealt(a.drop, offset, pos, (uint32_t)slice, [&](int c, bool kept) { if (kept) sum[c] = add_elem(sum[c], x[c]); });
            }
        } else {
#pragma unroll
            for (int c = 0; c < kGroup; ++c) sum[c] = add_elem(sum[c], x[c]);
        }
        if (ends >> i & 1u) {
            if (closed >> i & 1u) {
                float* dst = target(i);
                float was[kGroup];
                if (kAdd) Slot<float, kWide>::read(ring + slot * kSlot + Slot<T, kWide>::kBytes, (uint32_t)reinterpret_cast<uintptr_t>(dst), left, was);
                emit<kAdd, kWide>(dst, left, sum, was, a.factor);
            } else {                         // goes on in the next unit (and starts here unless it is the first, too), or began before
                leave(partial_at(r, unit_id, i == have - 1 && !((ends & ((1u << i) - 1u)) == 0 && from_before), slice), sum);
            }
#pragma unroll
            for (int c = 0; c < kGroup; ++c) sum[c] = 0.0f;
        }
        if (!kWide) __syncwarp();            // the slot has been read by all
        start(i + kSlots, slot);
    }
    copies_wait<0>();
    // at most two runs cross the unit's ends: its first and its last (or one that is both)
    for (uint32_t open = ends & ~closed; open; open &= open - 1)
        join<kAdd, kWide>(a, r, __shfl_sync(0xffffffffu, item.x, __ffs((int)open) - 1), unit_id, slice, left);
}

// Tokens per unit: as few as make one round of warps (a second, broken one costs as much as the first: 16384 x 1024
// written in units of 16 took 14 us longer for the tenth of the CTAs that had to wait), but eight at least: the more
// units, the more partial sums are joined (700 x 1500: 17.2, 13.9, 11.4, 10.9 us with units of 1, 2, 4, 8), and 32 at
// most (a lane for each).  The numbers of SMs and CTAs are constants: a call's bits do not depend on the device.
constexpr int kLeastUnit = 8, kMostUnit = 32;
constexpr int64_t kRound = 148 * (kReduceBlocks - kClearing) * (kReduceThreads / 32);
inline int unit_of(int64_t n, int64_t slices) {
    const int64_t units = kRound / slices;      // of one round
    const int64_t unit = units > 0 ? (n + units - 1) / units : kMostUnit;
    return (int)(unit < kLeastUnit ? kLeastUnit : (unit > kMostUnit ? kMostUnit : unit));
}
// Upper bound of units * slices over all calls of up to n tokens and up to `slices` slices (fewer tokens can make more
// units): what the workspace is sized by, so that it serves smaller calls too.
inline size_t most_tasks(int64_t n, int64_t slices) {
    const int64_t few = (n + kLeastUnit - 1) / kLeastUnit * slices, many = (n + kMostUnit - 1) / kMostUnit * slices;
    const int64_t round = kRound + slices, small = few < round ? few : round;
    return (size_t)(small > many ? small : many);
}

struct GradWs { size_t total, row_tab, sorted, entries, first, arrived, arrived_n, partial, bytes; int unit, units, slices; };
inline GradWs grad_ws(int64_t n, int64_t rows, int64_t width) {
    GradWs w{};
    w.slices = (int)((width + 255) / 256);
    w.unit = unit_of(n, w.slices);
    w.units = (int)((n + w.unit - 1) / w.unit);
    w.arrived_n = 4 * (size_t)w.units * (size_t)w.slices;
    w.total = 0;
    w.row_tab = 256;
    w.sorted = w.row_tab + align_up(sizeof(uint2) * (size_t)rows, 256);
    w.entries = w.sorted + align_up(sizeof(uint2) * (size_t)n, 256);
    w.first = w.entries + (n > kSplitFrom ? align_up(sizeof(uint2) * (size_t)n, 256) : 0);
    w.arrived = w.first + (n > kSplitFrom ? align_up(sizeof(uint16_t) * kSplitPitch * (size_t)((n + kTokenTile - 1) / kTokenTile), 256) : 0);
    w.partial = w.arrived + align_up(sizeof(uint32_t) * w.arrived_n, 256);
    const size_t most = most_tasks(n, w.slices);
    w.bytes = w.arrived + align_up(sizeof(uint32_t) * 4 * most, 256) + sizeof(float) * 2 * most * 256;
    return w;
}

}  // namespace

size_t embed_grad_ws_bytes(int64_t n, int64_t rows, int64_t width) { return grad_ws(n, rows, width).bytes; }

deft_status launch_embed_grad(const EmbedGradArgs& a, int dy_type, int id_bytes, cudaStream_t stream) {
    const int per_cta = (int)((a.rows + kOwners - 1) / kOwners);
    int warps = 4;                                          // a warp has 512 tokens' ids in flight
    while (warps < 32 && (int64_t)warps * 512 < a.n) warps <<= 1;
    while (warps > 1 && group_smem(warps, per_cta, 128) > kGroupSmem) warps >>= 1;
    if (group_smem(warps, per_cta, 1) > kGroupSmem) return DEFT_ERR_TOO_LARGE;
    int list_cap = (int)((kGroupSmem - group_smem(warps, per_cta, 0)) / (sizeof(uint2) * (size_t)warps));
    const int part = (int)((a.n + warps - 1) / warps);      // more than a warp can have
    if (list_cap > kListMost) list_cap = kListMost;
    if (list_cap > part) list_cap = part > 1 ? part : 1;
    const size_t smem = group_smem(warps, per_cta, list_cap);
    // -1, and any other number that is no row, leaves nothing out
    const uint32_t skip = a.skip_id >= 0 && a.skip_id < a.rows ? (uint32_t)a.skip_id : kNoRow;
    const GradWs w = grad_ws(a.n, a.rows, a.width);
    constexpr int64_t kWarps = kReduceThreads / 32;
    // kClearing CTAs on each SM clear; where the sums take two of the places there, all others (one token into 100000 x 512:
    // 42 against 54 us, 700 x 1500 into 33278 rows 47 against 50; with half of the places taken it costs 2 us of 35)
    const int64_t sms = sm_count(), sum_blocks = ((int64_t)w.units * w.slices + kWarps - 1) / kWarps;
    const int64_t clearing = sum_blocks <= 2 * sms ? kReduceBlocks - 2 : kClearing;
    const int64_t needed = (a.rows + kWarps - 1) / kWarps;
    const int clear_blocks = a.accumulate ? 0 : (int)(needed < clearing * sms ? needed : clearing * sms);
    const int64_t blocks = sum_blocks + clear_blocks;
    if (blocks > 0x7fffffff) return DEFT_ERR_TOO_LARGE;
    GroupOut out{reinterpret_cast<uint2*>(a.ws + w.sorted), reinterpret_cast<uint2*>(a.ws + w.row_tab), reinterpret_cast<uint32_t*>(a.ws + w.total),
                 reinterpret_cast<uint32_t*>(a.ws + w.arrived), w.arrived_n};
    // A kernel that waits for the one before it: its launch is prepared while that one still runs.  None lets the next one
    // start before its own end: CTAs that start beside one that has most of the SM's shared memory run, and go on
    // running, with what little is left for the L1 (0.33 against 0.24 ms at 131072 x 1024).
    cudaLaunchAttribute follows{};
    follows.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    follows.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.stream = stream;
    cfg.attrs = &follows;
    auto group = [&](auto id) -> deft_status {
        using Id = decltype(id);
        const Id* ids = static_cast<const Id*>(a.ids);
        const bool split = a.n > kSplitFrom;
        uint2* entries = reinterpret_cast<uint2*>(a.ws + w.entries);
        uint16_t* first = reinterpret_cast<uint16_t*>(a.ws + w.first);
        if (split) {
            k_split_tokens<Id><<<(unsigned)((a.n + kTokenTile - 1) / kTokenTile), 256, 0, stream>>>(ids, (uint32_t)a.n, (uint32_t)a.rows, skip, entries, first);
            DEFT_CUDA_TRY(cudaGetLastError());
        }
        auto kernel = split ? k_group_tokens<Id, true> : k_group_tokens<Id, false>;
        if (smem > 48 * 1024) DEFT_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kGroupSmem));
        cfg.gridDim = dim3(kOwners);
        cfg.blockDim = dim3((unsigned)warps * 32);
        cfg.dynamicSmemBytes = smem;
        cfg.numAttrs = split ? 1 : 0;
        DEFT_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, ids, (uint32_t)a.n, (uint32_t)a.rows, skip, (const uint2*)entries, (const uint16_t*)first, per_cta, list_cap, out));
        return DEFT_OK;
    };
    const deft_status s = id_bytes == 8 ? group(int64_t{}) : group(int32_t{});
    if (s != DEFT_OK) return s;
    const ReduceArgs r{out.sorted, out.row_tab, out.total, reinterpret_cast<float*>(a.ws + w.partial), out.arrived, w.unit, w.units, w.slices, clear_blocks};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(kReduceThreads);
    cfg.dynamicSmemBytes = 0;
    cfg.numAttrs = 1;
    const bool wide = row_align(a.grad, a.width, sizeof(float)) == 16 && (a.n == 0 || row_align(a.dy, a.ld_dy, type_bytes(dy_type)) == 16);
    return with_type(dy_type, [&](auto t) -> deft_status {
        using T = decltype(t);
        auto run = [&](auto kernel) { return cudaLaunchKernelEx(&cfg, kernel, a, r); };
        if (wide) DEFT_CUDA_TRY(a.accumulate ? run(k_rows_reduce<true, T, true>) : run(k_rows_reduce<false, T, true>));
        else DEFT_CUDA_TRY(a.accumulate ? run(k_rows_reduce<true, T, false>) : run(k_rows_reduce<false, T, false>));
        return DEFT_OK;
    });
}

}  // namespace deft
