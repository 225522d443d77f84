// How layer norm and its gradient split a matrix, and how its rows reach them.
//
// A row belongs to a team of 4 to 512 threads; a thread has some of the row's groups, every `size`-th one, in registers.  A group is
// what fills 16 bytes: eight columns of 16-bit matrices, four where one of the matrices is fp32 (two such pieces side by
// side for each thread would make every access touch each 32-byte sector twice: 16384 x 1024 fp32 36 us).  Groups come through a ring of asynchronous copies in shared memory, a few rows ahead of the one that
// is worked on, each thread its own (no barrier); loads into registers ahead of their use take the registers that the
// weight sums need, and give half of the bytes in flight.  Groups start on 16-byte boundaries whatever the row's address is: with odd widths the groups of row r are
// shifted left by (first + r ld) mod 8 columns, which suits 16-bit and 32-bit matrices alike as long as they agree in
// `first` and `ld` modulo 8.  A CTA takes rows of one shift only (every step-th row), so that the shift is a
// constant of the CTA and a thread's columns stay the same from row to row.
#pragma once
#include <type_traits>

#include "deft_dense.cuh"
#include "deft_pairs.cuh"

namespace deft {

constexpr int kTeamThreads = 256;        // of a CTA; more where a row takes more
constexpr int kTeamMost = 512;
constexpr int kTeamMostWarps = kTeamMost / 32;
constexpr int kMostStages = 4;

// How a thread gets its groups: through the ring; by 16-byte loads, where the parameters leave the ring no room for a stage beside as many
// CTAs as an SM holds (fp32 rows with a branch: of 4096 columns and some widths from 2500 on, and from 11800 on; gradients of the longest rows); or element by element (rows that
// no shift suits: matrices on different places of a granule).  The last two have one shape, that of the longest rows.
enum class Feed { kRing, kLoads, kElements };
template <Feed kFeed> struct FeedTag { static constexpr Feed value = kFeed; };

// The geometry of a call.
struct TeamShape {
    int size, groups, threads;           // threads of a team, groups of each, threads of a CTA
    int places;                          // groups of a row with its shift: what the parameters in shared memory are laid out by
    int step;                            // rows r, r + step, ... have the same shift
    int first, ld;                       // the shift of row r is (first + r ld) modulo the length of a group
    unsigned blocks;                     // a multiple of step
    Feed feed;
    int stages;                          // of the ring
    bool plain;                          // every group of every thread is the row's in full: no tests
    bool joined;                         // the CTAs are one cluster (and join their sums themselves)
    size_t smem;
};
constexpr int kMostJoined = 8;           // CTAs of a cluster

// The matrices of a call: how long a group is, and whether one shift serves all of them.
struct Shifts {
    int cols, first = -1, ld = 0;
    bool ok = true;
    explicit Shifts(int cols_) : cols(cols_) {}
    void add(const void* p, int64_t pitch, size_t elem) {
        if (!p) return;
        const int f = (int)(reinterpret_cast<uintptr_t>(p) / elem) & (cols - 1), l = (int)pitch & (cols - 1);
        if (first >= 0 && (f != first || l != ld)) ok = false;
        first = f;
        ld = l;
    }
};

// row_bytes: bytes of a column of all matrices that are read; params: fp32 vectors of the row's length in shared memory; per_sm:
// CTAs of kTeamThreads threads with up to sixteen columns each that an SM holds (per_sm_plain: without tests); most_blocks: of the launch (0: as many as the device holds).
// Rows of up to 8192 columns have sixteen columns a thread (their registers leave room for enough warps), longer ones 32; from 4096
// columns on a CTA has a row at a time and an SM one CTA, whose parameters and ring fill its shared memory.
// three: threads may have 24 columns of one 16-bit matrix, where that takes fewer of them for a row (768 columns: one warp, no lane idle; 17 -> 15 us at
// 16384 rows) and the ring still has two stages.
// join_turns: the call is one cluster of up to kMostJoined CTAs where a team then takes no more rows than that (0: never).
inline TeamShape team_shape(const Shifts& m, int64_t rows, int cols, int row_bytes, int params, int per_sm, int per_sm_plain, int64_t most_blocks, int join_turns, bool three) {
    TeamShape s{};
    bool shifted = m.ok;
    const int len = m.cols;
    auto place = [&]() {
        s.first = shifted ? m.first : 0;
        s.ld = shifted ? m.ld : 0;
        s.step = 1;
        while ((s.ld * s.step) & (len - 1)) s.step *= 2;
        s.places = (cols + (s.step > 1 ? len - 1 : s.first) + len - 1) / len;
    };
    place();
    if (s.places * len > kTeamMost * 32) {      // the longest rows leave no room for a shift
        shifted = false;
        place();
    }
    const bool large = s.places * len > kTeamThreads * 16;
    if (large) per_sm = 1;
    int most = (s.places * len > kTeamMost * 16 ? 32 : 16) / len;
    auto size_for = [&](int columns) {
        const int need = (s.places * len + columns - 1) / columns;
        int size = 4;
        while (size < 32 && size < need) size *= 2;
        return need > 32 ? (need + 31) / 32 * 32 : size;
    };
    s.size = large ? kTeamMost : size_for(16);
    const bool by_three = three && row_bytes <= 2 && s.size >= 64 && s.size <= 96 && size_for(24) < s.size && rows * size_for(24) * 2 > 148 * 512;
    if (by_three) {
        s.size = size_for(24);
        most = 24 / len;
    }
    // few rows: more threads for each, so that all SMs' schedulers have work
    while (!by_three && s.size * 2 <= kTeamThreads && s.size < s.places && rows * s.size * 2 <= 148 * 512) s.size *= 2;
    s.groups = large || by_three || s.size * (most / 2) < s.places ? most : most / 2;
    s.threads = s.size > kTeamThreads ? s.size : kTeamThreads / s.size * s.size;
    s.plain = shifted && s.first == 0 && s.ld == 0 && cols % len == 0 && s.places == s.size * s.groups && (s.groups * len == 16 || by_three);
    if (!large) per_sm = (s.plain && !by_three ? per_sm_plain : per_sm) * kTeamThreads / s.threads;
    if (most_blocks == 0) most_blocks = (int64_t)sm_count() * per_sm;
    const int64_t teams = s.threads / s.size, needed = ((rows + s.step - 1) / s.step + teams - 1) / teams;   // CTAs for the rows of a shift
    s.joined = needed * s.step <= (int64_t)kMostJoined * join_turns;
    if (s.joined) most_blocks = kMostJoined;
    const int64_t most_each = most_blocks / s.step, turns = (needed + most_each - 1) / most_each;
    s.blocks = (unsigned)((needed + turns - 1) / turns * s.step);      // (no more than take as many turns)
    // the ring: as many stages as a CTA's share of an SM's shared memory has room for, and as a team has rows
    const size_t stage = (size_t)(s.threads > kTeamThreads ? kTeamMost : kTeamThreads) * s.groups * len * row_bytes;
    s.smem = (size_t)params * sizeof(float) * (size_t)(s.places * len);
    const size_t share = kMostSmem / per_sm;
    s.stages = share > s.smem ? (int)((share - s.smem) / stage) : 0;
    if (s.stages > kMostStages) s.stages = kMostStages;
    if (s.stages > turns) s.stages = (int)turns;
    s.feed = !shifted ? Feed::kElements : (s.stages >= 1 ? Feed::kRing : Feed::kLoads);
    if (s.feed == Feed::kRing) s.smem += stage * s.stages;
    else s.groups = 32 / len;
    return s;
}

// One of a thread's groups: which of its elements are the row's.  Made once, as a CTA's rows all lie alike.
template <Feed kFeed, int kC, bool kPlain>
struct RowGroup {
    static constexpr bool kPieces = kFeed != Feed::kElements;
    int lo, hi;                          // elements lo .. hi are the row's
    struct Always { __device__ __forceinline__ constexpr operator bool() const { return true; } __device__ __forceinline__ void operator=(bool) {} };
    typename std::conditional<kPlain, Always, bool>::type whole, any;     // kPlain: all of every thread's groups are
    __device__ __forceinline__ void set(int place, int shift, int cols) {
        const int col = place * kC - shift;
        lo = col < 0 ? -col : 0;
        hi = cols - col < kC ? cols - col : kC;
        any = hi > lo;
        whole = lo == 0 && hi == kC;
    }
    template <typename T> using Raw = RawCols<T, kC, kPieces>;
    // `row` points to the group's first column throughout (which may lie before the row).  To shared memory: what lies behind the row's
    // end becomes zero there (`other`: for groups that have nothing; no byte is read there, but a copy's address lies on a 16-byte boundary
    // all the same).
    template <typename T>
    __device__ __forceinline__ void copy(const T* row, const void* other, uint32_t to) const {
        constexpr int kBytes = kC * (int)sizeof(T);
        const void* from = any ? static_cast<const void*>(row) : other;
        const int bytes = any ? hi * (int)sizeof(T) : 0;
        if constexpr (kPlain && kBytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(row) : "memory");
        else if constexpr (kPlain) asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(row) : "memory");
        else if constexpr (kBytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
        else asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
    }
    // Of a group that has come through the ring, elements before the row remain to be cleared (plain rows begin with a group).
    template <int kN>
    __device__ __forceinline__ void clear(Cols<kN>& v) const {
        if constexpr (kPlain) return;
        if constexpr (kFeed == Feed::kRing) {
            if (lo > 0) v.trim(lo, kC);
        } else {
            if (!whole) v.trim(lo, hi);
        }
    }
    // Plain loads: a row may be overwritten by its own threads later.
    template <typename T>
    __device__ __forceinline__ void load(const T* row, Raw<T>& raw) const {
        using R = Raw<T>;
#pragma unroll
        for (int i = 0; i < R::kPieces; ++i)
            if ((i + 1) * R::kPer > lo && i * R::kPer < hi) raw.piece[i] = reinterpret_cast<const typename R::P*>(row)[i];
    }
    template <typename T>
    __device__ __forceinline__ void store(T* row, const Cols<kC>& v) const {
        using R = Raw<T>;
        R raw;
        v.to(raw);
        if (whole) {
#pragma unroll
            for (int i = 0; i < R::kPieces; ++i) reinterpret_cast<typename R::P*>(row)[i] = raw.piece[i];
        } else {
#pragma unroll
            for (int k = 0; k < kC; ++k)
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
    __device__ __forceinline__ Walk(T* base, int64_t ld, uint32_t row, uint32_t stride, int col, int across_)
        : at(base ? base + (int64_t)row * ld + col : nullptr), down((int64_t)stride * ld), across(across_) {}
    __device__ __forceinline__ T* group(int j) const { return at + j * across; }
    __device__ __forceinline__ void next() { at += down; }
};

// The ring of a CTA.  A stage holds, for each matrix and group, a run of kC elements for every thread; kBytes: of a thread in a stage.
template <int kThreads, int kBytes>
struct Ring {
    static constexpr uint32_t kStage = kThreads * (uint32_t)kBytes;
    const char* base;
    uint32_t at;                         // the same as a shared address
    uint32_t now, fill, end;             // the row's stage, the one that is filled meanwhile, behind the last: offsets
    int ahead;                           // stages that may still be under way
    __device__ __forceinline__ Ring(const char* base_, int stages)
        : base(base_), at((uint32_t)__cvta_generic_to_shared(base_)), now(0), fill((uint32_t)(stages - 1) * kStage), end((uint32_t)stages * kStage), ahead(stages - 1) {}
    // Where a thread's group lies in a stage: `before` bytes a thread of runs before it, `bytes` of it.
    static __device__ __forceinline__ uint32_t offset(int before, int bytes) { return kThreads * (uint32_t)before + threadIdx.x * (uint32_t)bytes; }
    __device__ __forceinline__ uint32_t target(uint32_t stage, int before, int bytes) const { return at + stage + offset(before, bytes); }
    template <typename R>
    __device__ __forceinline__ void read(int before, R& raw) const { raw.piece[0] = *reinterpret_cast<const typename R::P*>(base + now + offset(before, (int)sizeof(typename R::P))); }
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
        now += kStage;
        if (now == end) now = 0;
    }
};

// Parameters and sums of the places in shared memory: the first four columns of all groups, then the next four, so that
// consecutive threads' 16-byte accesses are consecutive.
template <int kC>
__device__ __forceinline__ int at_place(int places, int i) { return kC == 4 ? i : (((i >> 2) & 1) * places + (i >> 3)) * 4 + (i & 3); }
template <int kC>
__device__ __forceinline__ void read_place(const float* s, int places, int place, Cols<kC>& v) {
#pragma unroll
    for (int i = 0; i < kC / 4; ++i) {
        const ulonglong2 a = reinterpret_cast<const ulonglong2*>(s)[i * places + place];
        v.p[2 * i] = a.x, v.p[2 * i + 1] = a.y;
    }
}
template <int kC>
__device__ __forceinline__ void write_place(float* s, int places, int place, const Cols<kC>& v) {
#pragma unroll
    for (int i = 0; i < kC / 4; ++i) reinterpret_cast<ulonglong2*>(s)[i * places + place] = make_ulonglong2(v.p[2 * i], v.p[2 * i + 1]);
}
// A vector (NULL: `otherwise` throughout) to its places.  The loads of eight turns are under way together: one after the other they
// took longer than a row (5003 x 1027 fp32 15 us).
template <int kC, typename T>
__device__ __forceinline__ void fill_places(float* s, const T* p, int cols, int places, int shift, float otherwise) {
    constexpr int kDeep = 8;
    const int all = places * kC, step = (int)blockDim.x;
    for (int i0 = threadIdx.x; i0 < all; i0 += kDeep * step) {
        T v[kDeep];
#pragma unroll
        for (int k = 0; k < kDeep; ++k) {
            const int c = i0 + k * step - shift;
            v[k] = from_f32<T>(otherwise);
            if (p && c >= 0 && c < cols) v[k] = p[c];
        }
#pragma unroll
        for (int k = 0; k < kDeep; ++k)
            if (i0 + k * step < all) s[at_place<kC>(places, i0 + k * step)] = to_f32(v[k]);
    }
}
template <int kC>
__device__ __forceinline__ void fill_places(float* s, const void* p, int type, int cols, int places, int shift, float otherwise) {
    if (type == DEFT_F32) fill_places<kC>(s, static_cast<const float*>(p), cols, places, shift, otherwise);
    else if (type == DEFT_BF16) fill_places<kC>(s, static_cast<const __nv_bfloat16*>(p), cols, places, shift, otherwise);
    else fill_places<kC>(s, static_cast<const __half*>(p), cols, places, shift, otherwise);
}

// The threads that share a row, the rows they take, and their sums.
struct Team {
    int size, at, team, teams, turn;     // threads; this one's number; the team's number in the CTA; teams of a CTA
    uint32_t row, stride;                // first row, distance to the next
    int shift;
    float2* slots;                       // [2][warps of the CTA]
    __device__ __forceinline__ Team(const TeamShape& s, int len, float2* slots_) : size(s.size), turn(0), slots(slots_) {
        team = (int)threadIdx.x / size;
        at = (int)threadIdx.x - team * size;
        teams = (int)blockDim.x / size;
        const uint32_t step = (uint32_t)s.step, same = blockIdx.x / step, rest = blockIdx.x - same * step;
        row = (same * teams + team) * step + rest;
        stride = gridDim.x * teams;      // (CTAs of a shift) x teams x step
        shift = (int)((uint32_t)s.first + rest * (uint32_t)s.ld) & (len - 1);
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
        // (numbers that the compiler knows: of CTAs with a number in a register an SM holds four)
        switch (team) {
            case 0: asm volatile("bar.sync 1, %0;" ::"r"(size) : "memory"); break;
            case 1: asm volatile("bar.sync 2, %0;" ::"r"(size) : "memory"); break;
            case 2: asm volatile("bar.sync 3, %0;" ::"r"(size) : "memory"); break;
            default: asm volatile("bar.sync 4, %0;" ::"r"(size) : "memory"); break;
        }
        a = b = 0.0f;
        for (int i = 0; i < warps; ++i) {
            a += s[i].x;
            b += s[i].y;
        }
        return make_float2(a, b);
    }
};

// Calls f with the feed, the number of groups of a thread, the threads of a CTA and `plain` as constants (a ring of short rows; its long
// ones; other feeds).  Without their tests 16384 x 1024 takes 3 per cent less, 8192 x 4096 7.
template <int kC, bool kThree, typename F>
deft_status with_shape(const TeamShape& s, F&& f) {
    using Ring = FeedTag<Feed::kRing>;
    using Small = AlignTag<kTeamThreads>;
    using Large = AlignTag<kTeamMost>;
    if (s.feed == Feed::kElements) return f(FeedTag<Feed::kElements>{}, AlignTag<32 / kC>{}, Large{}, AlignTag<0>{});
    if (s.feed == Feed::kLoads) return f(FeedTag<Feed::kLoads>{}, AlignTag<32 / kC>{}, Large{}, AlignTag<0>{});
    const bool large = s.threads > kTeamThreads;
    if constexpr (kThree) {
        if (s.groups * kC == 24) return s.plain ? f(Ring{}, AlignTag<24 / kC>{}, Small{}, AlignTag<1>{}) : f(Ring{}, AlignTag<24 / kC>{}, Small{}, AlignTag<0>{});
    }
    if (s.plain) return large ? f(Ring{}, AlignTag<16 / kC>{}, Large{}, AlignTag<1>{}) : f(Ring{}, AlignTag<16 / kC>{}, Small{}, AlignTag<1>{});
    if (large) return s.groups * kC == 32 ? f(Ring{}, AlignTag<32 / kC>{}, Large{}, AlignTag<0>{}) : f(Ring{}, AlignTag<16 / kC>{}, Large{}, AlignTag<0>{});
    if (s.groups * kC == 16) return f(Ring{}, AlignTag<16 / kC>{}, Small{}, AlignTag<0>{});
    return f(Ring{}, AlignTag<8 / kC>{}, Small{}, AlignTag<0>{});
}

}  // namespace deft
