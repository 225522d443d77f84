// How layer norm and its gradient split a matrix, and how its rows reach them.
//
// A row belongs to a team of 4 to 512 threads; a thread has up to four of the row's groups of eight columns, every
// `size`-th one, in registers.  Groups come through a ring of asynchronous copies in shared memory, a few rows ahead of the one that
// is worked on, each thread its own (no barrier); loads into registers ahead of their use take the registers that the
// weight sums need, and give half of the bytes in flight.  Groups start on 16-byte boundaries whatever the row's address is: with odd widths the groups of row r are
// shifted left by (first + r ld) mod 8 columns, which suits 16-bit and 32-bit matrices alike as long as they agree in
// `first` and `ld` modulo 8.  A CTA takes rows of one shift only (every step-th row), so that the shift is a
// constant of the CTA and a thread's columns stay the same from row to row.
#pragma once
#include "deft_dense.cuh"
#include "deft_pairs.cuh"

namespace deft {

constexpr int kTeamThreads = 256;        // of a CTA; more where a row takes more
constexpr int kTeamMost = 512;
constexpr int kTeamMostWarps = kTeamMost / 32;
constexpr int kMostStages = 4;

// How a thread gets its groups: through the ring, by 16-byte loads (where the ring finds no room), or element by element (rows that
// no shift suits).
enum class Feed { kRing, kLoads, kElements };
template <Feed kFeed> struct FeedTag { static constexpr Feed value = kFeed; };

// The geometry of a call.
struct TeamShape {
    int size, groups, threads;           // threads of a team, groups of each, threads of a CTA
    int places;                          // groups of a row with its shift: what the parameters in shared memory are laid out by
    int step;                            // rows r, r + step, ... have the same shift
    int first, ld;                       // the shift of row r is (first + r ld) mod 8
    unsigned blocks;                     // a multiple of step
    Feed feed;
    int stages;                          // of the ring
    size_t smem;
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

// row_bytes: bytes of eight columns of all matrices that are read; params: fp32 vectors of the row's length in shared memory; per_sm:
// CTAs of kTeamThreads threads with up to two groups each that an SM holds; most_blocks: of the launch (0: as many as the device holds).
// Rows of up to 4096 columns have two groups a thread (their registers leave room for enough warps), longer ones four.
inline TeamShape team_shape(const ShiftFinder& m, int64_t rows, int cols, int row_bytes, int params, int per_sm, int64_t most_blocks) {
    TeamShape s{};
    bool shifted = m.ok;
    const int count = m.half ? 3 : 7;    // shifts of 32-bit matrices alone count modulo 4
    auto place = [&]() {
        s.first = shifted ? m.first & count : 0;
        s.ld = shifted ? m.ld & count : 0;
        s.step = s.ld == 0 ? 1 : (s.ld == 4 ? 2 : (s.ld & 1 ? 8 : 4));
        s.places = (cols + (s.step > 1 ? 7 : s.first) + kGroup - 1) / kGroup;
    };
    place();
    if (s.places > kTeamMost * 4) {      // the longest rows leave no room for a shift
        shifted = false;
        place();
    }
    const int most = s.places <= kTeamThreads * 2 ? 2 : 4;
    if (most == 4) per_sm = s.places <= kTeamThreads * 4 ? 2 : 1;
    s.size = 4;
    while (s.size < kTeamMost && s.size * most < s.places) s.size *= 2;
    // few rows: more threads for each, so that all SMs' schedulers have work
    while (s.size < kTeamThreads && s.size < s.places && rows * s.size * 2 <= 148 * 512) s.size *= 2;
    const int each = (s.places + s.size - 1) / s.size;
    s.groups = most == 4 ? 4 : (each <= 1 ? 1 : 2);
    s.threads = s.size > kTeamThreads ? s.size : kTeamThreads;
    if (most_blocks == 0) most_blocks = (int64_t)sm_count() * per_sm;
    const int64_t teams = s.threads / s.size, needed = ((rows + s.step - 1) / s.step + teams - 1) / teams;   // CTAs for the rows of a shift
    const int64_t most_each = most_blocks / s.step;
    s.blocks = (unsigned)((needed < most_each ? needed : most_each) * s.step);
    // the ring: as many stages as a CTA's share of an SM's shared memory has room for, and as a team has rows
    const size_t stage = (size_t)s.threads * s.groups * row_bytes;
    s.smem = (size_t)params * sizeof(float) * (size_t)(s.places * kGroup);
    const size_t share = (size_t)220 * 1024 / per_sm;
    const int64_t turns = (needed * s.step + s.blocks - 1) / s.blocks;
    s.stages = share > s.smem ? (int)((share - s.smem) / stage) : 0;
    if (s.stages > kMostStages) s.stages = kMostStages;
    if (s.stages > turns) s.stages = (int)turns;
    s.feed = !shifted ? Feed::kElements : (s.stages >= 1 ? Feed::kRing : Feed::kLoads);
    if (s.feed == Feed::kRing) s.smem += stage * s.stages;
    else s.groups = 4;
    return s;
}

// One of a thread's groups: which of its elements are the row's.  Made once, as a CTA's rows all lie alike.
template <Feed kFeed>
struct RowGroup {
    int col, lo, hi;                     // first column (may lie before the row); elements lo .. hi are the row's
    bool whole, any;
    __device__ __forceinline__ void set(int place, int shift, int cols) {
        col = place * kGroup - shift;
        lo = col < 0 ? -col : 0;
        hi = cols - col < kGroup ? cols - col : kGroup;
        any = hi > lo;
        whole = lo == 0 && hi == kGroup;
    }
    template <typename T> static __host__ __device__ constexpr int align() { return kFeed != Feed::kElements ? 16 : (int)sizeof(T); }
    // `row` points to the group's first column throughout.  16-byte pieces that hold an element of the row, to shared memory: the
    // first piece to `to`, a second one `apart` bytes further.
    template <typename T>
    __device__ __forceinline__ void copy(const T* row, uint32_t to, uint32_t apart) const {
        constexpr int pieces = kGroup * (int)sizeof(T) / 16, per = kGroup / pieces;
        const char* from = reinterpret_cast<const char*>(row);
#pragma unroll
        for (int i = 0; i < pieces; ++i)
            if (whole || ((i + 1) * per > lo && i * per < hi))
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + (uint32_t)i * apart), "l"(from + i * 16) : "memory");
    }
    // Plain loads: a row may be overwritten by its own threads later.
    template <typename T>
    __device__ __forceinline__ void load(const T* row, Raw8<T, align<T>()>& raw) const {
        using R = Raw8<T, align<T>()>;
        constexpr int per = kGroup / R::kPieces;
        const typename R::P* p = reinterpret_cast<const typename R::P*>(row);
#pragma unroll
        for (int i = 0; i < R::kPieces; ++i)
            if (whole || ((i + 1) * per > lo && i * per < hi)) raw.piece[i] = p[i];
    }
    template <typename T>
    __device__ __forceinline__ void store(T* row, const Eight& v) const {
        using R = Raw8<T, align<T>()>;
        R raw;
        v.to(raw);
        if (whole) {
            typename R::P* p = reinterpret_cast<typename R::P*>(row);
#pragma unroll
            for (int i = 0; i < R::kPieces; ++i) p[i] = raw.piece[i];
        } else {
#pragma unroll
            for (int k = 0; k < kGroup; ++k)
                if (k >= lo && k < hi) row[k] = reinterpret_cast<const T*>(raw.piece)[k];
        }
    }
};

// A matrix's rows as a thread meets them: the address of its first group in the row that comes next, and the distance to its
// next group.
template <typename T>
struct Walk {
    T* at;
    int64_t down;                        // elements to the next row of this team
    int across;
    __device__ __forceinline__ Walk(T* base, int64_t ld, uint32_t row, uint32_t stride, int col, int size)
        : at(base ? base + (int64_t)row * ld + col : nullptr), down((int64_t)stride * ld), across(size * kGroup) {}
    __device__ __forceinline__ T* group(int j) const { return at + j * across; }
    __device__ __forceinline__ void next() { at += down; }
};

// The ring of a CTA.  A stage holds, for each matrix, group and piece, a run of 16 bytes for every thread.
template <int kThreads, int kAll>
struct Ring {
    static constexpr uint32_t kRun = kThreads * 16u;
    const char* mine;                    // this thread's place in the first run of the first stage, and the same as a shared address
    uint32_t at;
    uint32_t now, fill, end;             // the row's stage, the one that is filled meanwhile, behind the last: offsets
    int ahead;                           // stages that may still be under way
    __device__ __forceinline__ Ring(const char* base, int stages)
        : mine(base + threadIdx.x * 16u), at((uint32_t)__cvta_generic_to_shared(base) + threadIdx.x * 16u), now(0), fill((uint32_t)(stages - 1) * kAll * kRun),
          end((uint32_t)stages * kAll * kRun), ahead(stages - 1) {}
    __device__ __forceinline__ uint32_t target(uint32_t stage, int run) const { return at + stage + (uint32_t)run * kRun; }
    template <typename T>
    __device__ __forceinline__ void read(int run, Raw8<T, 16>& raw) const {
#pragma unroll
        for (int i = 0; i < Raw8<T, 16>::kPieces; ++i) raw.piece[i] = *reinterpret_cast<const uint4*>(mine + now + (uint32_t)(run + i) * kRun);
    }
    static __device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
    // Waits for the row's stage.
    __device__ __forceinline__ void wait() const {
        if (ahead >= 3) asm volatile("cp.async.wait_group 3;" ::: "memory");
        else if (ahead == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
        else if (ahead == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
        else asm volatile("cp.async.wait_group 0;" ::: "memory");
    }
    __device__ __forceinline__ void next() {
        fill = now;
        now += kAll * kRun;
        if (now == end) now = 0;
    }
};

// Parameters and sums of the places in shared memory: the first halves of all groups, then the second ones, so that
// consecutive threads' 16-byte accesses are consecutive.
__device__ __forceinline__ int at_place(int places, int place, int k) { return ((k >> 2) * places + place) * 4 + (k & 3); }
__device__ __forceinline__ void read_place(const float* s, int places, int place, Eight& v) {
    const ulonglong2 a = reinterpret_cast<const ulonglong2*>(s)[place], b = reinterpret_cast<const ulonglong2*>(s)[places + place];
    v.p[0] = a.x, v.p[1] = a.y, v.p[2] = b.x, v.p[3] = b.y;
}
__device__ __forceinline__ void write_place(float* s, int places, int place, const Eight& v) {
    reinterpret_cast<ulonglong2*>(s)[place] = make_ulonglong2(v.p[0], v.p[1]);
    reinterpret_cast<ulonglong2*>(s)[places + place] = make_ulonglong2(v.p[2], v.p[3]);
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
        if (size < 32) {
            for (int o = size >> 1; o; o >>= 1) {
                a += __shfl_xor_sync(0xffffffffu, a, o);
                b += __shfl_xor_sync(0xffffffffu, b, o);
            }
            return make_float2(a, b);
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            a += __shfl_xor_sync(0xffffffffu, a, o);
            b += __shfl_xor_sync(0xffffffffu, b, o);
        }
        if (size == 32) return make_float2(a, b);
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
