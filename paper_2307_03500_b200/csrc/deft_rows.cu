// Embedding lookup and dropout: rows of a matrix taken in groups of eight columns.
//
// A thread keeps its columns and takes every `stride`-th row (up to four rows' loads in flight), so that consecutive
// threads read consecutive groups whatever the width, one division places it, and the parts of the generator's first
// two rounds that depend on the column or the offset alone are computed once.  Loads of several rows are in flight before
// the first is converted (converting each as it came made the kernel wait for every load: 0.44 instead of 0.17 ms).
//
// What bounds them: dropout of 65536 x 4096 bf16 the memory (174 us, 0.96 of the measured copy rate, in short runs; 187 us,
// 0.89, in long ones, where the clocks fall and the generator's integer work, half of the pipes' time, shows), of 16384 x 1024
// with a residual added 18.6 us (0.84), of 32768 x 1024 fp32 with one 68 us (0.92).  Lookup of 131072 x 1024 fp32 -> bf16
// with positions and dropout 104 us (0.55 of the copy rate over the bytes it cannot do without; 0.84 GB move between
// L2 and the SMs, because a table row is read again for each of its tokens): the wait for a table row behind its id,
// with two rows in flight per thread.  Calls of up to a few hundred thousand elements: the launch (3 to 4 us).  Rows that start on no 8-byte boundary are taken by warps in slices of
// 256 columns instead, dealt out one by one.
#include "deft_rows.cuh"

namespace deft {
namespace {

constexpr int kRowThreads = 256;
constexpr int kInFlight = 16;    // words a thread that takes several rows has in flight
constexpr int kMostDeep = 4;     // rows it has in flight, when a row's group is four words
constexpr int kMostEach = 16;    // rows it takes in all
constexpr int kRounds = 8;       // rounds of CTAs a launch has at least before threads take several rows ...
constexpr int kEmbedRounds = 3;  // ... fewer where a thread waits for an id before it can load a row
// CTAs an SM holds where threads take one row (32 registers) and where they take several (64).  Chosen on bf16 without
// positions or residual, which fits.  181 of the 324 instances spill: most with single elements (dropout with a residual up to
// 656 bytes stored and loaded), lookup of one row with positions (up to 408), fp32 dropout with a residual (304 with 16-byte
// alignment).  Other bounds for those have not been measured.
constexpr int kBlocksOne = 8;
constexpr int kBlocksDeep = 4;

// Rows in flight of a thread that loads `words` words of each; two where the rows are not 16-byte aligned (their pieces and
// tests take the registers that four would: dropout 32768 x 1020 bf16 39 against 50 us).
__host__ __device__ constexpr int deep_of(int words, int align) {
    const int fit = kInFlight / words < 2 || align != 16 ? 2 : kInFlight / words;
    return fit > kMostDeep ? kMostDeep : fit;
}

// How the matrix is split: `units` (groups of a row, or slices of it) times `stride` rows are taken at a time.
struct RowSplit {
    FastDiv units;
    uint32_t stride, rows;
    bool same_pos;       // all rows of a thread have the same position row
};

// What one thread (kAlign != 0) or warp (kAlign == 0) works on.
template <int kAlign>
struct Place {
    static constexpr int kSpan = kAlign ? kGroup : 256;
    uint32_t row, unit;
    int64_t col;      // first column of the group or slice
    __device__ __forceinline__ explicit Place(const RowSplit& s) {
        const uint32_t at = kAlign ? blockIdx.x * (uint32_t)kRowThreads + threadIdx.x
                                   : blockIdx.x * (uint32_t)(kRowThreads / 32) + (threadIdx.x >> 5);
        row = s.units.div(at);
        unit = at - row * s.units.d;
        col = (int64_t)unit * kSpan;
    }
};

// What an id outside the table is looked up in: a share of a row at most.
__device__ __align__(16) const char g_zeros[256 * sizeof(float)] = {};

// kAlign != 0: eight columns of this thread; else this lane's share of the slice.  kFull: the group (slice) has all its
// columns; left = columns from its first one to the row's end.
template <bool kFull, typename T, int kAlign>
__device__ __forceinline__ void fetch_share(const T* p, int left, Raw8<T, kAlign>& raw) {
    if constexpr (kAlign != 0) fetch8<kFull>(p, left, raw);
    else fetch_dealt<kFull>(p, left, raw);
}
template <bool kFull, typename T, int kAlign>
__device__ __forceinline__ void store_share(T* p, int left, const float (&v)[kGroup]) {
    if constexpr (kAlign != 0) store8<kFull, T, kAlign>(p, left, v);
    else store_dealt<kFull>(p, left, v);
}
template <int kAlign>
__device__ __forceinline__ void drop_share(float (&v)[kGroup], const DropArgs& d, uint64_t offset, uint32_t row, uint32_t unit) {
    if constexpr (kAlign != 0) drop8(v, d, offset, row, unit);
    else drop8_dealt(v, d, offset, row, unit);
}

// Whether threads whose group (slice) is whole run code of their own.  With 8-byte alignment nearly every row ends in a
// broken group, whose warp would run both: there all threads test their pieces (lookup 32768 x 1020 bf16 35 against 44 us).
template <int kAlign> __device__ constexpr bool full_apart() { return kAlign != 8; }

template <bool kFull, int kDeep, bool kPos, typename TW, typename TO, typename Id, int kAlign>
__device__ __forceinline__ void embed_rows(const EmbedArgs& a, const RowSplit& split, const FastDiv& pos_rows, const Place<kAlign>& at, int left) {
    const uint64_t offset = drop_offset(a.drop);
    const TW* table = static_cast<const TW*>(a.table) + at.col;
    const TW* pos = static_cast<const TW*>(a.pos) + at.col;
    TO* out = static_cast<TO*>(a.out) + at.col;
    const Id* ids = static_cast<const Id*>(a.ids);
    Raw8<TW, kAlign> q;
    if (kPos) fetch_share<kFull>(pos + (int64_t)(at.row - pos_rows.div(at.row) * pos_rows.d) * a.ld_pos, left, q);
    uint32_t next[kDeep];                // the table rows of the next turn's tokens
    auto look = [&](uint32_t t0) {
#pragma unroll
        for (int k = 0; k < kDeep; ++k) {
            const uint32_t t = t0 + k * split.stride;
            next[k] = t < split.rows ? row_of(__ldg(ids + t), (uint32_t)a.rows, kNoRow) : kNoRow;
        }
    };
    look(at.row);
    for (uint32_t t0 = at.row; t0 < split.rows; t0 += kDeep * split.stride) {
        Raw8<TW, kAlign> w[kDeep];
#pragma unroll
        for (int k = 0; k < kDeep; ++k)
            fetch_share<kFull>(next[k] != kNoRow ? table + next[k] * a.ld_table : reinterpret_cast<const TW*>(g_zeros), left, w[k]);
        if (kDeep > 1) look(t0 + kDeep * split.stride);
#pragma unroll
        for (int k = 0; k < kDeep; ++k) {
            const uint32_t t = t0 + k * split.stride;
            if (t >= split.rows) break;
            float v[kGroup];
            w[k].unpack(v);
            if (a.scale != 1.0f) {
#pragma unroll
                for (int i = 0; i < kGroup; ++i) v[i] = __fmul_rn(v[i], a.scale);
            }
            if (kPos) {
                if (!split.same_pos) fetch_share<kFull>(pos + (int64_t)(t - pos_rows.div(t) * pos_rows.d) * a.ld_pos, left, q);
                q.add_to(v);
            }
            if (a.drop.threshold) drop_share<kAlign>(v, a.drop, offset, t, at.unit);
            store_share<kFull, TO, kAlign>(out + (int64_t)t * a.ld_out, left, v);
        }
    }
}

template <int kDeep, bool kPos, typename TW, typename TO, typename Id, int kAlign>
__global__ void __launch_bounds__(kRowThreads, kDeep == 1 ? kBlocksOne : kBlocksDeep) k_embed(const __grid_constant__ EmbedArgs a, const RowSplit split, const FastDiv pos_rows) {
    const Place<kAlign> at(split);
    if (at.row >= split.stride) return;
    const int left = (int)min(a.width - at.col, (int64_t)at.kSpan);
    constexpr bool kApart = full_apart<kAlign>();
    if (kApart && left == at.kSpan) embed_rows<kApart, kDeep, kPos, TW, TO, Id, kAlign>(a, split, pos_rows, at, left);
    else embed_rows<false, kDeep, kPos, TW, TO, Id, kAlign>(a, split, pos_rows, at, left);
}

template <bool kFull, int kDeep, bool kAdd, typename TX, typename TY, int kAlign>
__device__ __forceinline__ void dropout_rows(const DropoutArgs& a, const RowSplit& split, const Place<kAlign>& at, int left) {
    const uint64_t offset = drop_offset(a.drop);
    const TX* x = static_cast<const TX*>(a.x) + at.col;
    const TY* add = static_cast<const TY*>(a.add) + at.col;
    TY* y = static_cast<TY*>(a.y) + at.col;
    for (uint32_t r0 = at.row; r0 < split.rows; r0 += kDeep * split.stride) {
        Raw8<TX, kAlign> w[kDeep];
        Raw8<TY, kAlign> q[kDeep];
#pragma unroll
        for (int k = 0; k < kDeep; ++k) {
            const uint32_t r = r0 + k * split.stride;
            if (r < split.rows) {
                fetch_share<kFull>(x + (int64_t)r * a.ld_x, left, w[k]);
                if (kAdd) fetch_share<kFull>(add + (int64_t)r * a.ld_add, left, q[k]);
            }
        }
#pragma unroll
        for (int k = 0; k < kDeep; ++k) {
            const uint32_t r = r0 + k * split.stride;
            if (r >= split.rows) break;
            float v[kGroup];
            w[k].unpack(v);
            if (a.drop.threshold) drop_share<kAlign>(v, a.drop, offset, r, at.unit);
            if (kAdd) q[k].add_to(v);
            store_share<kFull, TY, kAlign>(y + (int64_t)r * a.ld_y, left, v);
        }
    }
}

template <int kDeep, bool kAdd, typename TX, typename TY, int kAlign>
__global__ void __launch_bounds__(kRowThreads, kDeep == 1 ? kBlocksOne : kBlocksDeep) k_dropout(const __grid_constant__ DropoutArgs a, const RowSplit split) {
    const Place<kAlign> at(split);
    if (at.row >= split.stride) return;
    const int left = (int)min(a.cols - at.col, (int64_t)at.kSpan);
    constexpr bool kApart = full_apart<kAlign>();
    if (kApart && left == at.kSpan) dropout_rows<kApart, kDeep, kAdd, TX, TY, kAlign>(a, split, at, left);
    else dropout_rows<false, kDeep, kAdd, TX, TY, kAlign>(a, split, at, left);
}

// Threads take up to kMostEach rows each, as many as leave every SM several rounds of CTAs (the last round is rarely
// full).  pos_rows != 0: `stride` becomes a multiple of it where that is possible, so that a thread reads its position
// row once for all its tokens.
inline RowSplit row_split(int64_t rows, int64_t cols, int align, int rounds, int64_t pos_rows, unsigned* blocks) {
    const int64_t units = align ? (cols + kGroup - 1) / kGroup : (cols + 255) / 256;
    const int64_t per_block = align ? kRowThreads : kRowThreads / 32;
    int64_t each = rows * units / ((int64_t)sm_count() * kBlocksDeep * per_block * rounds);
    each = each < 1 ? 1 : (each > kMostEach ? kMostEach : each);
    int64_t stride = (rows + each - 1) / each;
    // a turn that goes past the last row counts up to eight strides further, in 32 bits: no rounding that would not fit
    // (without it the stride is a sixteenth of the rows wherever they are many)
    if (pos_rows && each > 1 && pos_rows < rows) {
        const int64_t rounded = (stride + pos_rows - 1) / pos_rows * pos_rows;
        if (rows + 8 * rounded <= 0xffffffffLL) stride = rounded;
    }
    const int64_t most = (0x7fffffff - 255) / units;   // places are 31-bit; a larger matrix takes more turns of the loop
    if (stride > most) stride = most;
    if (stride > rows) stride = rows;
    *blocks = (unsigned)((stride * units + per_block - 1) / per_block);
    return RowSplit{fast_div((uint32_t)units), (uint32_t)stride, (uint32_t)rows, pos_rows && (stride % pos_rows == 0 || stride == rows)};
}

}  // namespace

deft_status launch_embed(const EmbedArgs& a, int table_type, int out_type, int id_bytes, cudaStream_t stream) {
    int align = row_align(a.table, a.ld_table, type_bytes(table_type));
    const int ao = row_align(a.out, a.ld_out, type_bytes(out_type));
    if (ao < align) align = ao;
    if (a.pos) {
        const int ap = row_align(a.pos, a.ld_pos, type_bytes(table_type));
        if (ap < align) align = ap;
    }
    unsigned blocks;
    const RowSplit split = row_split(a.n, a.width, align, kEmbedRounds, a.pos ? a.pos_rows : 0, &blocks);
    // a token's number is below 2^31: more position rows than that are never wrapped around
    const FastDiv pos_rows = fast_div((uint32_t)(a.pos_rows < 0x7fffffff ? a.pos_rows : 0x7fffffff));
    return with_type(table_type, [&](auto w) {
        return with_type(out_type, [&](auto o) {
            return with_align(align, [&](auto al) -> deft_status {
                using TW = decltype(w);
                using TO = decltype(o);
                constexpr int kAlign = decltype(al)::value;
                auto run = [&](auto kernel) { kernel<<<blocks, kRowThreads, 0, stream>>>(a, split, pos_rows); };
                auto with_id = [&](auto id) {
                    using Id = decltype(id);
                    constexpr int kDeep = deep_of((int)sizeof(TW) * 2, kAlign);
                    if (split.stride == split.rows) a.pos ? run(k_embed<1, true, TW, TO, Id, kAlign>) : run(k_embed<1, false, TW, TO, Id, kAlign>);
                    else a.pos ? run(k_embed<kDeep, true, TW, TO, Id, kAlign>) : run(k_embed<kDeep, false, TW, TO, Id, kAlign>);
                };
                id_bytes == 8 ? with_id(int64_t{}) : with_id(int32_t{});
                DEFT_CUDA_TRY(cudaGetLastError());
                return DEFT_OK;
            });
        });
    });
}

deft_status launch_dropout(const DropoutArgs& a, int x_type, int y_type, cudaStream_t stream) {
    int align = row_align(a.x, a.ld_x, type_bytes(x_type));
    const int ay = row_align(a.y, a.ld_y, type_bytes(y_type));
    if (ay < align) align = ay;
    if (a.add) {
        const int aa = row_align(a.add, a.ld_add, type_bytes(y_type));
        if (aa < align) align = aa;
    }
    unsigned blocks;
    const RowSplit split = row_split(a.rows, a.cols, align, kRounds, 0, &blocks);
    return with_type(x_type, [&](auto x) {
        return with_type(y_type, [&](auto y) {
            return with_align(align, [&](auto al) -> deft_status {
                auto run = [&](auto kernel) { kernel<<<blocks, kRowThreads, 0, stream>>>(a, split); };
                using TX = decltype(x);
                using TY = decltype(y);
                constexpr int kAlign = decltype(al)::value;
                constexpr int kPlain = deep_of((int)sizeof(TX) * 2, kAlign), kBoth = deep_of((int)sizeof(TX) * 2 + (int)sizeof(TY) * 2, kAlign);
                if (split.stride == split.rows) a.add ? run(k_dropout<1, true, TX, TY, kAlign>) : run(k_dropout<1, false, TX, TY, kAlign>);
                else a.add ? run(k_dropout<kBoth, true, TX, TY, kAlign>) : run(k_dropout<kPlain, false, TX, TY, kAlign>);
                DEFT_CUDA_TRY(cudaGetLastError());
                return DEFT_OK;
            });
        });
    });
}

}  // namespace deft
