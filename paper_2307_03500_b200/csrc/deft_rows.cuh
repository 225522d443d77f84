// Shared device code of the row operators (embedding lookup, its gradient, dropout): element types,
// eight-column groups of a row, and the counter-based generator of the dropout mask.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "deft_common.cuh"

namespace deft {

constexpr int kGroup = 8;   // columns a thread takes at a time: one call of the generator gives eight 16-bit numbers

// What dropout needs to know.  threshold = t << 16, where an element is kept when its 16-bit number is at
// least t = round(65536 p); 0 means no dropout.  gain = 65536 / (65536 - t), rounded once to fp32.
struct DropArgs {
    uint32_t keys[20];          // the ten rounds' two key words
    uint64_t offset;
    const uint64_t* offset_d;   // added to offset when not NULL (device memory: a replayed graph draws new masks)
    uint32_t threshold;
    float gain;
};

// Philox4x32 with ten rounds (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3",
// SC 2011).  The rounds' keys come from the host, as operands from the constant bank: a round is two wide products and
// two three-way exclusive ors.
__device__ __forceinline__ uint4 philox10(uint4 c, const uint32_t (&keys)[20]) {
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)0xD2511F53u * c.x, b = (uint64_t)0xCD9E8D57u * c.z;
        c = make_uint4((uint32_t)(b >> 32) ^ c.y ^ keys[2 * r], (uint32_t)b, (uint32_t)(a >> 32) ^ c.w ^ keys[2 * r + 1], (uint32_t)a);
    }
    return c;
}
inline void philox_keys(uint64_t seed, uint32_t (&keys)[20]) {
    uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
    for (int r = 0; r < 10; ++r, k0 += 0x9E3779B9u, k1 += 0xBB67AE85u) {
        keys[2 * r] = k0;
        keys[2 * r + 1] = k1;
    }
}

__device__ __forceinline__ uint64_t drop_offset(const DropArgs& d) {
    return d.threshold && d.offset_d ? d.offset + *d.offset_d : d.offset;
}

// The random words of (row, columns 8 * group .. + 7).
__device__ __forceinline__ uint4 drop_words(const DropArgs& d, uint64_t offset, uint32_t row, uint32_t group) {
    return philox10(make_uint4(group, row, (uint32_t)offset, (uint32_t)(offset >> 32)), d.keys);
}

// Whether the even (low half) and the odd column (high half) of a word are kept: what lies below a half does not change
// how it compares with the threshold.
__device__ __forceinline__ void kept2(uint32_t word, uint32_t threshold, bool& even, bool& odd) {
    even = (word << 16) >= threshold;
    odd = word >= threshold;
}

// Applies a group's mask to v: kept elements are multiplied by the gain, dropped ones become +0 whatever they were.
__device__ __forceinline__ void drop8(float (&v)[kGroup], const DropArgs& d, uint64_t offset, uint32_t row, uint32_t group) {
    const uint4 w = drop_words(d, offset, row, group);
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        bool even, odd;
        kept2(u[i], d.threshold, even, odd);
        v[2 * i] = even ? __fmul_rn(v[2 * i], d.gain) : 0.0f;
        v[2 * i + 1] = odd ? __fmul_rn(v[2 * i + 1], d.gain) : 0.0f;
    }
}

// The same where a warp's 256 columns are dealt out one by one (lane l has the columns 32 k + l): every lane draws the
// eight bits of its own group and fetches those of its columns from the lanes that have them.
template <typename F>
__device__ __forceinline__ void for_kept_dealt(const DropArgs& d, uint64_t offset, uint32_t row, uint32_t slice, F&& f) {
    const int lane = threadIdx.x & 31;
    const uint4 w = drop_words(d, offset, row, slice * 32 + lane);
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        bool even, odd;
        kept2(u[i], d.threshold, even, odd);
        bits |= (even ? 1u << (2 * i) : 0u) | (odd ? 2u << (2 * i) : 0u);
    }
#pragma unroll
    for (int k = 0; k < kGroup; ++k) f(k, (__shfl_sync(0xffffffffu, bits, k * 4 + (lane >> 3)) >> (lane & 7) & 1u) != 0);
}
__device__ __forceinline__ void drop8_dealt(float (&v)[kGroup], const DropArgs& d, uint64_t offset, uint32_t row, uint32_t slice) {
    for_kept_dealt(d, offset, row, slice, [&](int k, bool kept) { v[k] = kept ? __fmul_rn(v[k], d.gain) : 0.0f; });
}

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }

// sum + x, x converted exactly: one instruction, without unpacking the 16-bit type first.
__device__ __forceinline__ float add_elem(float sum, float x) { return sum + x; }
__device__ __forceinline__ float add_elem(float sum, __nv_bfloat16 x) {
    asm("add.f32.bf16 %0, %1, %0;" : "+f"(sum) : "h"(__bfloat16_as_ushort(x)));
    return sum;
}
__device__ __forceinline__ float add_elem(float sum, __half x) {
    asm("add.f32.f16 %0, %1, %0;" : "+f"(sum) : "h"(__half_as_ushort(x)));
    return sum;
}

template <int kBytes> struct Piece;
template <> struct Piece<16> { using type = uint4; };
template <> struct Piece<8> { using type = uint2; };
template <> struct Piece<4> { using type = uint32_t; };
template <> struct Piece<2> { using type = uint16_t; };

// Eight elements as they lie in memory.  Loading and converting are apart so that a thread can have several groups'
// loads in flight before it waits for the first.
template <typename T, int kAlign>
struct Raw8 {
    static constexpr int kPiece = kAlign ? kAlign : (int)sizeof(T);
    using P = typename Piece<kPiece>::type;
    static constexpr int kPieces = kGroup * (int)sizeof(T) / kPiece;
    P piece[kPieces];
    __device__ __forceinline__ void unpack(float (&v)[kGroup]) const {
        const T* e = reinterpret_cast<const T*>(piece);
#pragma unroll
        for (int i = 0; i < kGroup; ++i) v[i] = to_f32(e[i]);
    }
    __device__ __forceinline__ void add_to(float (&v)[kGroup]) const {
        const T* e = reinterpret_cast<const T*>(piece);
#pragma unroll
        for (int i = 0; i < kGroup; ++i) v[i] = add_elem(v[i], e[i]);
    }
};

// A group of eight consecutive elements of which the first `left` (or more) belong to the row.  kAlign: 16 or 8 when
// every group of the matrix starts on such a boundary (base and row pitch are multiples of it).  A piece that starts
// inside the row is read whole (what lies behind the row's end in it is not used); pieces behind the end are not
// touched.  Plain loads: what is read may be what the same thread writes afterwards (dropout in place, rows added to).
// kFull: left is eight or more.
template <bool kFull, typename T, int kAlign>
__device__ __forceinline__ void fetch8(const T* p, int left, Raw8<T, kAlign>& raw) {
    using P = typename Raw8<T, kAlign>::P;
    constexpr int per = kAlign / (int)sizeof(T);
#pragma unroll
    for (int i = 0; i < Raw8<T, kAlign>::kPieces; ++i)
        if (kFull || i * per < left) raw.piece[i] = reinterpret_cast<const P*>(p)[i];
}

// Writes the first `left` of a group (or all eight): whole pieces, and the elements of one that the row's end crosses.
template <bool kFull, typename T, int kAlign>
__device__ __forceinline__ void store8(T* p, int left, const float (&v)[kGroup]) {
    using P = typename Piece<kAlign>::type;
    constexpr int per = kAlign / (int)sizeof(T), pieces = kGroup / per;
    P raw[pieces];
#pragma unroll
    for (int i = 0; i < kGroup; ++i) reinterpret_cast<T*>(raw)[i] = from_f32<T>(v[i]);
#pragma unroll
    for (int i = 0; i < pieces; ++i) {
        if (kFull || (i + 1) * per <= left) {
            reinterpret_cast<P*>(p)[i] = raw[i];
        } else {
#pragma unroll
            for (int j = 0; j < per; ++j)
                if (i * per + j < left) p[i * per + j] = reinterpret_cast<const T*>(raw)[i * per + j];
        }
    }
}

// Eight fp32 values to a 32-byte boundary.
__device__ __forceinline__ void store32(float* p, const float (&v)[kGroup]) {
    asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]),
                 "f"(v[5]), "f"(v[6]), "f"(v[7]) : "memory");
}

// A slice of 256 columns dealt out one by one: lane l has the columns 32 k + l, so that loads and stores of a matrix whose
// rows start on no vector boundary are whole sectors all the same (eight consecutive elements per lane would touch 32
// sectors with every load).  kFull: the slice has all 256; else the first `left`.
template <bool kFull, typename T>
__device__ __forceinline__ void fetch_dealt(const T* p, int left, Raw8<T, 0>& raw) {
    const int lane = threadIdx.x & 31;
    T* e = reinterpret_cast<T*>(raw.piece);
#pragma unroll
    for (int k = 0; k < kGroup; ++k) e[k] = kFull || k * 32 + lane < left ? p[k * 32 + lane] : from_f32<T>(0.0f);
}
template <bool kFull, typename T>
__device__ __forceinline__ void store_dealt(T* p, int left, const float (&v)[kGroup]) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int k = 0; k < kGroup; ++k)
        if (kFull || k * 32 + lane < left) p[k * 32 + lane] = from_f32<T>(v[k]);
}

// n / d for n < 2^31 by a product (d >= 1): m = ceil(2^p / d) with p = 31 + ceil(log2 d) is exact in that range.
struct FastDiv {
    uint32_t d, m, shift;
    __device__ __forceinline__ uint32_t div(uint32_t n) const { return d == 1 ? n : __umulhi(n, m) >> shift; }
};
inline FastDiv fast_div(uint32_t d) {
    uint32_t log = 0;
    while ((1ull << log) < d) ++log;
    const uint32_t p = 31 + log;
    return FastDiv{d, (uint32_t)(((1ull << p) + d - 1) / d), p - 32};
}

// An id as a row of the table, or kNoRow (no table has that many).
constexpr uint32_t kNoRow = 0xffffffffu;
__device__ __forceinline__ uint32_t row_of(int32_t id, uint32_t rows, uint32_t skip) {
    return (uint32_t)id < rows && (uint32_t)id != skip ? (uint32_t)id : kNoRow;
}
__device__ __forceinline__ uint32_t row_of(int64_t id, uint32_t rows, uint32_t skip) {
    return (uint64_t)id < rows && (uint32_t)id != skip ? (uint32_t)id : kNoRow;
}

// ---- launchers ----
struct EmbedArgs {
    const void* table;
    int64_t rows, ld_table;
    const void* pos;         // NULL, or [pos_rows, width]: row t % pos_rows is added to token t's row
    int64_t pos_rows, ld_pos;
    const void* ids;
    void* out;
    int64_t ld_out;
    int64_t n, width;
    float scale;
    DropArgs drop;
};
struct DropoutArgs {
    const void* x;
    const void* add;         // NULL, or added after dropout (the type of y)
    void* y;
    int64_t ld_x, ld_add, ld_y;
    int64_t rows, cols;
    DropArgs drop;
};
struct EmbedGradArgs {
    const void* dy;
    int64_t ld_dy;
    const void* ids;
    int64_t n, rows, width;
    int64_t skip_id;
    float factor;            // scale x the survivors' gain: applied once to a row's sum
    DropArgs drop;
    float* grad;
    int32_t accumulate;
    char* ws;
};
deft_status launch_embed(const EmbedArgs& a, int table_type, int out_type, int id_bytes, cudaStream_t stream);
deft_status launch_dropout(const DropoutArgs& a, int x_type, int y_type, cudaStream_t stream);
size_t embed_grad_ws_bytes(int64_t n, int64_t rows, int64_t width);
deft_status launch_embed_grad(const EmbedGradArgs& a, int dy_type, int id_bytes, cudaStream_t stream);

// Widest boundary every row of a matrix starts on: 16, 8 or 0 (single elements only).
inline int row_align(const void* p, int64_t ld, size_t elem) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(p) | (uintptr_t)((size_t)ld * elem);
    return (x & 15u) == 0 ? 16 : ((x & 7u) == 0 ? 8 : 0);
}
inline size_t type_bytes(int type) { return type == DEFT_F32 ? 4 : 2; }

// Calls f(T{}) with the element type behind a DEFT_* code.
template <typename F>
deft_status with_type(int type, F&& f) {
    switch (type) {
        case DEFT_F32: return f(float{});
        case DEFT_BF16: return f(__nv_bfloat16{});
        default: return f(__half{});
    }
}
template <int kAlign> struct AlignTag { static constexpr int value = kAlign; };
template <typename F>
deft_status with_align(int align, F&& f) {
    switch (align) {
        case 16: return f(AlignTag<16>{});
        case 8: return f(AlignTag<8>{});
        default: return f(AlignTag<0>{});
    }
}

}  // namespace deft
