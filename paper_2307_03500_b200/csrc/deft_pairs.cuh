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

// Eight numbers as four pairs.
struct Eight {
    uint64_t p[4];
    template <typename T, int kAlign>
    __device__ __forceinline__ void from(const Raw8<T, kAlign>& raw) {
        if constexpr (kAlign == 16 && sizeof(T) == 2) {
            p[0] = widened<T>(raw.piece[0].x), p[1] = widened<T>(raw.piece[0].y), p[2] = widened<T>(raw.piece[0].z), p[3] = widened<T>(raw.piece[0].w);
        } else if constexpr (kAlign == 16) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                p[2 * i] = pair(__uint_as_float(raw.piece[i].x), __uint_as_float(raw.piece[i].y));
                p[2 * i + 1] = pair(__uint_as_float(raw.piece[i].z), __uint_as_float(raw.piece[i].w));
            }
        } else {
            float v[kGroup];
            raw.unpack(v);
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = pair(v[2 * i], v[2 * i + 1]);
        }
    }
    template <typename T, int kAlign>
    __device__ __forceinline__ void to(Raw8<T, kAlign>& raw) const {
        if constexpr (kAlign == 16 && sizeof(T) == 2) {
            raw.piece[0] = make_uint4(narrowed<T>(p[0]), narrowed<T>(p[1]), narrowed<T>(p[2]), narrowed<T>(p[3]));
        } else if constexpr (kAlign == 16) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float2 u = unpair(p[2 * i]), v = unpair(p[2 * i + 1]);
                raw.piece[i] = make_uint4(__float_as_uint(u.x), __float_as_uint(u.y), __float_as_uint(v.x), __float_as_uint(v.y));
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 v = unpair(p[i]);
                reinterpret_cast<T*>(raw.piece)[2 * i] = from_f32<T>(v.x);
                reinterpret_cast<T*>(raw.piece)[2 * i + 1] = from_f32<T>(v.y);
            }
        }
    }
    // Elements outside lo .. hi become zero.
    __device__ __forceinline__ void trim(int lo, int hi) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 v = unpair(p[i]);
            p[i] = pair(2 * i >= lo && 2 * i < hi ? v.x : 0.0f, 2 * i + 1 >= lo && 2 * i + 1 < hi ? v.y : 0.0f);
        }
    }
    __device__ __forceinline__ uint64_t sum() const { return add2(add2(p[0], p[1]), add2(p[2], p[3])); }
};
__device__ __forceinline__ float folded(uint64_t p) {
    const float2 v = unpair(p);
    return v.x + v.y;
}

}  // namespace deft
