// Rows in registers: how layer norm and its gradient split a matrix.
//
// A row belongs to a team of 4 to 512 threads; a thread has up to four of the row's groups of eight columns, every
// `size`-th one.  Groups start on 16-byte boundaries whatever the row's address is: with odd widths the groups of row r are
// shifted left by (first + r ld) mod 8 columns, which suits 16-bit and 32-bit matrices alike as long as they agree in
// `first` and `ld` modulo 8.  A CTA takes rows of one shift only (every step-th row), so that the shift is a
// constant of the CTA and a thread's columns stay the same from row to row.
#pragma once
#include "deft_dense.cuh"

namespace deft {

constexpr int kTeamThreads = 256;        // of a CTA; more where a row takes more
constexpr int kTeamMost = 512;
constexpr int kTeamMostWarps = kTeamMost / 32;

// The geometry of a call.
struct TeamShape {
    int size, groups, threads;           // threads of a team, groups of each, threads of a CTA
    int places;                          // groups of a row with its shift: what the parameters in shared memory are laid out by
    int step;                            // rows r, r + step, ... have the same shift
    int first, ld;                       // the shift of row r is (first + r ld) mod 8
    unsigned blocks;                     // a multiple of step
    bool aligned;                        // 16-byte pieces; else single elements
};

// The matrices of a call: whether one shift serves all of them.
struct ShiftFinder {
    int first = -1, ld = 0;
    bool any = false, ok = true, half = false;   // half: only 32-bit matrices so far (shifts count modulo 4)
    void add(const void* p, int64_t pitch, size_t elem) {
        if (!p) return;
        const int f = (int)(reinterpret_cast<uintptr_t>(p) / elem & 7), l = (int)(pitch & 7);
        const bool wide = elem == 4;
        if (!any) {
            first = f, ld = l, half = wide, any = true;
            return;
        }
        const int mask = wide || half ? 3 : 7;
        if (((f ^ first) & mask) || ((l ^ ld) & mask)) ok = false;
        if (half && !wide) first = f, ld = l, half = false;
    }
};

inline TeamShape team_shape(const ShiftFinder& m, int64_t rows, int cols, int most, int64_t most_blocks) {
    TeamShape s{};
    s.aligned = m.ok;
    const int count = m.half ? 3 : 7;    // shifts of 32-bit matrices alone count modulo 4
    s.first = m.ok ? m.first & count : 0;
    s.ld = m.ok ? m.ld & count : 0;
    s.step = s.ld == 0 ? 1 : (s.ld == 4 ? 2 : (s.ld & 1 ? 8 : 4));
    s.places = (cols + (s.step > 1 ? 7 : s.first) + kGroup - 1) / kGroup;
    if (s.places > kTeamMost * 4) {      // the longest rows leave no room for a shift
        s.aligned = false;
        s.first = s.ld = 0;
        s.step = 1;
        s.places = (cols + kGroup - 1) / kGroup;
    }
    s.size = 4;
    while (s.size < kTeamMost && s.size * most < s.places) s.size *= 2;
    // few rows: more threads for each, so that all SMs' schedulers have work
    while (s.size < kTeamThreads && s.size < s.places && rows * s.size * 2 <= 148 * 512) s.size *= 2;
    const int each = (s.places + s.size - 1) / s.size;
    s.groups = each <= 1 ? 1 : (each <= 2 ? 2 : 4);
    s.threads = s.size > kTeamThreads ? s.size : kTeamThreads;
    const int64_t teams = s.threads / s.size, needed = ((rows + s.step - 1) / s.step + teams - 1) / teams;   // CTAs for the rows of a shift
    const int64_t most_each = most_blocks / s.step;
    s.blocks = (unsigned)((needed < most_each ? needed : most_each) * s.step);
    return s;
}

// One of a thread's groups: its columns, and which of them are the row's.
template <bool kAligned>
struct RowGroup {
    int col, lo, hi;                     // first column (may lie before the row); the group's elements lo .. hi are the row's
    __device__ __forceinline__ RowGroup(int place, int shift, int cols) {
        col = place * kGroup - shift;
        lo = col < 0 ? -col : 0;
        hi = cols - col < kGroup ? cols - col : kGroup;
    }
    __device__ __forceinline__ bool whole() const { return lo == 0 && hi == kGroup; }
    __device__ __forceinline__ bool has(int k) const { return k >= lo && k < hi; }
    template <typename T> static __host__ __device__ constexpr int align() { return kAligned ? 16 : (int)sizeof(T); }
    // Plain loads: a row may be overwritten by its own threads later.
    template <typename T>
    __device__ __forceinline__ void load(const T* row, Raw8<T, align<T>()>& raw) const {
        using R = Raw8<T, align<T>()>;
        constexpr int per = kGroup / R::kPieces;
        const typename R::P* p = reinterpret_cast<const typename R::P*>(row + col);
        if (whole()) {
#pragma unroll
            for (int i = 0; i < R::kPieces; ++i) raw.piece[i] = p[i];
        } else {
#pragma unroll
            for (int i = 0; i < R::kPieces; ++i)
                if ((i + 1) * per > lo && i * per < hi) raw.piece[i] = p[i];
        }
    }
    // What is not the row's becomes zero.
    __device__ __forceinline__ void trim(float (&v)[kGroup]) const {
        if (whole()) return;
#pragma unroll
        for (int k = 0; k < kGroup; ++k) v[k] = has(k) ? v[k] : 0.0f;
    }
    template <typename T>
    __device__ __forceinline__ void store(T* row, const float (&v)[kGroup]) const {
        using R = Raw8<T, align<T>()>;
        constexpr int per = kGroup / R::kPieces;
        R raw;
#pragma unroll
        for (int k = 0; k < kGroup; ++k) reinterpret_cast<T*>(raw.piece)[k] = from_f32<T>(v[k]);
        typename R::P* p = reinterpret_cast<typename R::P*>(row + col);
        if (whole()) {
#pragma unroll
            for (int i = 0; i < R::kPieces; ++i) p[i] = raw.piece[i];
        } else {
#pragma unroll
            for (int k = 0; k < kGroup; ++k)
                if (has(k)) row[col + k] = reinterpret_cast<const T*>(raw.piece)[k];
        }
    }
};

// Parameters and sums of the places in shared memory: the first halves of all groups, then the second ones, so that
// consecutive threads' 16-byte accesses are consecutive.
__device__ __forceinline__ int at_place(int places, int place, int k) { return ((k >> 2) * places + place) * 4 + (k & 3); }
__device__ __forceinline__ void read_place(const float* s, int places, int place, float (&v)[kGroup]) {
    const float4 a = reinterpret_cast<const float4*>(s)[place], b = reinterpret_cast<const float4*>(s)[places + place];
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}
__device__ __forceinline__ void write_place(float* s, int places, int place, const float (&v)[kGroup]) {
    reinterpret_cast<float4*>(s)[place] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(s)[places + place] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ float param(const void* p, int type, int i) {
    return type == DEFT_F32 ? static_cast<const float*>(p)[i]
                            : (type == DEFT_BF16 ? to_f32(static_cast<const __nv_bfloat16*>(p)[i]) : to_f32(static_cast<const __half*>(p)[i]));
}
__device__ __forceinline__ void fill_places(float* s, const void* p, int type, int cols, int places, int shift, float otherwise) {
    for (int i = threadIdx.x; i < places * kGroup; i += blockDim.x) {
        const int c = i - shift;
        s[at_place(places, i >> 3, i & 7)] = p && c >= 0 && c < cols ? param(p, type, c) : otherwise;
    }
}

// The threads that share a row, the rows they take, and their sums.
struct Team {
    int size, at, team, teams, turn;     // threads; this one's number; the team's number in the CTA; teams of a CTA
    uint32_t row, stride;                // first row, distance to the next
    int shift;
    float2* slots;                       // [2][warps of the CTA]
    __device__ __forceinline__ Team(const TeamShape& s, float2* slots_) : size(s.size), turn(0), slots(slots_) {
        team = (int)threadIdx.x / size;
        at = (int)threadIdx.x - team * size;
        teams = (int)blockDim.x / size;
        const uint32_t step = (uint32_t)s.step, same = blockIdx.x / step, rest = blockIdx.x - same * step;
        row = (same * teams + team) * step + rest;
        stride = gridDim.x * teams;      // (CTAs of a shift) x teams x step
        shift = (int)((uint32_t)s.first + rest * (uint32_t)s.ld) & 7;
    }
    // The sums of a and b over the team.  All threads of a CTA call it equally often.
    __device__ __forceinline__ float2 sum(float a, float b) {
        const int in_warp = size < 32 ? size : 32;
        for (int o = in_warp >> 1; o; o >>= 1) {
            a += __shfl_xor_sync(0xffffffffu, a, o);
            b += __shfl_xor_sync(0xffffffffu, b, o);
        }
        if (size <= 32) return make_float2(a, b);
        // two sets of slots in turn: whoever writes a set again has passed the barrier that all pass after they have read it
        const int warps = size >> 5;
        float2* s = slots + turn * kTeamMostWarps + team * warps;
        turn ^= 1;
        if ((threadIdx.x & 31) == 0) s[at >> 5] = make_float2(a, b);
        asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(size) : "memory");
        a = b = 0.0f;
        for (int i = 0; i < warps; ++i) {
            a += s[i].x;
            b += s[i].y;
        }
        return make_float2(a, b);
    }
};

template <typename F>
deft_status with_groups(int groups, F&& f) {
    switch (groups) {
        case 1: return f(AlignTag<1>{});
        case 2: return f(AlignTag<2>{});
        default: return f(AlignTag<4>{});
    }
}

}  // namespace deft
