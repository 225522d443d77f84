// The embedding's gradient: the rows of the incoming gradient summed by token.
//
// 1. k_group_tokens puts the token positions in order of their table rows (positions of one row ascending) and
//    writes, per table row, where its positions start and how many there are.
// 2. k_rows_sum adds up each row's tokens in fp32, in that order: the result does not depend on how the work
//    was scheduled.
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
    for (int i = threadIdx.x; i < warps * per_cta; i += blockDim.x) cnt[i] = 0u;
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
// One warp per table row and 256 columns.
template <typename T, int kAlign>
__global__ void __launch_bounds__(256) k_rows_sum(const EmbedGradArgs a, const uint2* __restrict__ sorted, const uint2* __restrict__ row_tab, int slices) {
    const int lane = threadIdx.x & 31;
    const int64_t task = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int64_t row = task / slices;
    if (row >= a.rows) return;
    const uint32_t group = (uint32_t)(task - row * slices) * 32 + lane;
    const int64_t col = (int64_t)group * kGroup;
    const uint2 tab = row_tab[row];
    if (col >= a.width || (a.accumulate && tab.y == 0)) return;
    const int count = a.width - col < kGroup ? (int)(a.width - col) : kGroup;
    const uint64_t offset = drop_offset(a.drop);
    float sum[kGroup] = {};
    for (uint32_t i = 0; i < tab.y; ++i) {
        const uint32_t pos = sorted[tab.x + i].y;
        float v[kGroup];
        load8<T, kAlign>(static_cast<const T*>(a.dy) + (int64_t)pos * a.ld_dy + col, count, v);
        if (a.drop.threshold) drop8<false>(v, a.drop, offset, pos, group);
#pragma unroll
        for (int c = 0; c < kGroup; ++c) sum[c] += v[c];
    }
    float* dst = a.grad + row * a.width + col;
#pragma unroll
    for (int c = 0; c < kGroup; ++c)
        if (c < count) {
            const float g = tab.y ? __fmul_rn(sum[c], a.factor) : 0.0f;   // (+0 also where the factor is negative)
            dst[c] = a.accumulate ? __fadd_rn(dst[c], g) : g;
        }
}

struct GradWs { size_t total, row_tab, sorted, bytes; };
inline GradWs grad_ws(int64_t n, int64_t rows) {
    GradWs w{};
    w.total = 0;
    w.row_tab = 256;
    w.sorted = w.row_tab + align_up(sizeof(uint2) * (size_t)rows, 256);
    w.bytes = w.sorted + align_up(sizeof(uint2) * (size_t)n, 256);
    return w;
}

}  // namespace

size_t embed_grad_ws_bytes(int64_t n, int64_t rows, int64_t width) { return grad_ws(n, rows).bytes; }

deft_status launch_embed_grad(const EmbedGradArgs& a, int dy_type, int id_bytes, cudaStream_t stream) {
    const int per_cta = (int)((a.rows + kOwners - 1) / kOwners);
    int warps = 32;
    while (warps > 1 && group_smem(warps, per_cta) > kGroupSmem) warps >>= 1;
    const size_t smem = group_smem(warps, per_cta);
    if (smem > kGroupSmem) return DEFT_ERR_TOO_LARGE;
    const GradWs w = grad_ws(a.n, a.rows);
    GroupOut out{reinterpret_cast<uint2*>(a.ws + w.sorted), reinterpret_cast<uint2*>(a.ws + w.row_tab), reinterpret_cast<uint32_t*>(a.ws + w.total)};
    auto group = [&](auto id) -> deft_status {
        using Id = decltype(id);
        DEFT_CUDA_TRY(cudaFuncSetAttribute(k_group_tokens<Id>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kGroupSmem));
        k_group_tokens<Id><<<kOwners, warps * 32, smem, stream>>>(static_cast<const Id*>(a.ids), (uint32_t)a.n, a.rows, a.skip_id, per_cta, out);
        DEFT_CUDA_TRY(cudaGetLastError());
        return DEFT_OK;
    };
    const deft_status s = id_bytes == 8 ? group(int64_t{}) : group(int32_t{});
    if (s != DEFT_OK) return s;
    const int slices = (int)((a.width + 255) / 256);
    const int64_t blocks = (a.rows * slices + 7) / 8;
    if (blocks > 0x7fffffff) return DEFT_ERR_TOO_LARGE;
    return with_type(dy_type, [&](auto t) {
        return with_align(row_align(a.dy, a.ld_dy, type_bytes(dy_type)), [&](auto al) -> deft_status {
            k_rows_sum<decltype(t), decltype(al)::value><<<(unsigned)blocks, 256, 0, stream>>>(a, out.sorted, out.row_tab, slices);
            DEFT_CUDA_TRY(cudaGetLastError());
            return DEFT_OK;
        });
    });
}

}  // namespace deft
