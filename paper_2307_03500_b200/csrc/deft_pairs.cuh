// Two fp32 numbers in a register pair, which one instruction adds, multiplies or both (sm_100a).  Device code.
#pragma once
#include "deft_rows.cuh"

namespace deft {

// Two fp32 numbers side by side: one instruction for both.
__device__ __forceinline__ uint64_t pair(float a, float b) {
    uint64_t p;
    asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "f"(a), "f"(b));
    return p;
}
__device__ __forceinline__ float2 unpair(uint64_t p) {
    float2 v;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(v.x), "=f"(v.y) : "l"(p));
    return v;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint64_t both(float a) { return pair(a, a); }

// Sixteen bits each, in a word, and back (rounded to nearest).
template <typename T> __device__ __forceinline__ uint64_t widened(uint32_t w);
template <> __device__ __forceinline__ uint64_t widened<__nv_bfloat16>(uint32_t w) { return pair(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
template <> __device__ __forceinline__ uint64_t widened<__half>(uint32_t w) {
    const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&w));
    return pair(v.x, v.y);
}
template <typename T> __device__ __forceinline__ uint32_t narrowed(uint64_t p);
template <> __device__ __forceinline__ uint32_t narrowed<__nv_bfloat16>(uint64_t p) {
    const float2 v = unpair(p);
    const __nv_bfloat162 h = __floats2bfloat162_rn(v.x, v.y);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <> __device__ __forceinline__ uint32_t narrowed<__half>(uint64_t p) {
    const float2 v = unpair(p);
    const __half2 h = __floats2half2_rn(v.x, v.y);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// kC consecutive elements as they lie in memory: in one piece of up to 16 bytes (kWhole), or one by one.
template <typename T, int kC, bool kWhole>
struct RawCols {
    static constexpr int kPiece = kWhole ? kC * (int)sizeof(T) : (int)sizeof(T), kPieces = kC * (int)sizeof(T) / kPiece, kPer = kC / kPieces;
    using P = typename Piece<kPiece>::type;
    P piece[kPieces];
};
// kC numbers as pairs.
template <int kC>
struct Cols {
    static constexpr int kPairs = kC / 2;
    uint64_t p[kPairs];
    template <typename T, bool kWhole>
    __device__ __forceinline__ void from(const RawCols<T, kC, kWhole>& raw) {
        if constexpr (kWhole && sizeof(T) == 2) {
            const uint32_t* w = reinterpret_cast<const uint32_t*>(raw.piece);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) p[i] = widened<T>(w[i]);
        } else {
            const T* e = reinterpret_cast<const T*>(raw.piece);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) p[i] = pair(to_f32(e[2 * i]), to_f32(e[2 * i + 1]));
        }
    }
    template <typename T, bool kWhole>
    __device__ __forceinline__ void to(RawCols<T, kC, kWhole>& raw) const {
        if constexpr (kWhole && sizeof(T) == 2) {
            uint32_t* w = reinterpret_cast<uint32_t*>(raw.piece);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) w[i] = narrowed<T>(p[i]);
        } else {
            T* e = reinterpret_cast<T*>(raw.piece);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) {
                const float2 v = unpair(p[i]);
                e[2 * i] = from_f32<T>(v.x);
                e[2 * i + 1] = from_f32<T>(v.y);
            }
        }
    }
    // Elements outside lo .. hi become zero.
    __device__ __forceinline__ void trim(int lo, int hi) {
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
            const float2 v = unpair(p[i]);
            p[i] = pair(2 * i >= lo && 2 * i < hi ? v.x : 0.0f, 2 * i + 1 >= lo && 2 * i + 1 < hi ? v.y : 0.0f);
        }
    }
};
__device__ __forceinline__ float folded(uint64_t p) {
    const float2 v = unpair(p);
    return v.x + v.y;
}

}  // namespace deft
