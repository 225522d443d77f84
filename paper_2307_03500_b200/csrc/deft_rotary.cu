// Rotary positions: pairs of a head's columns turned by an angle that grows with the token's position.
//
// A frequency is a number of turns per position in units of 2^-64, so that the product with a position, taken modulo
// 2^64, is the angle modulo a turn, exactly: far positions cost no accuracy.  A CTA takes a few tokens: their cosines and
// sines once into shared memory, then all heads with them.
//
// Bound by memory: a vector in, a vector out, nothing else (angles are formed, not read).  Measured (device time; floor at the copy rate,
// 6561 GB/s):
//   8 x 2048 tokens, 32 heads of 128, bf16, halves    43.5 us (6.17 TB/s; floor 40.9); neighbours 44.9
//   16 x 1024 tokens, 32 heads of 64, bf16            24.3 us (floor 20.5)
//   5003 tokens, 12 heads of 160, 40 turned, fp32     17.3 us (floor 11.7: borders at 160 bytes leave threads of a warp in two kinds of work)
//   48 tokens, 24 heads of 128                        2.4 us (latency: a table, a vector)
// Odd widths go element by element: 65 us for 8 x 2048 tokens, 32 heads of 66 with 50 turned, bf16 (floor 21).
#include "deft_dense.cuh"

namespace deft {
namespace {

constexpr int kRotThreads = 256;
constexpr int kRotSmem = 32 * 1024;
constexpr int kRotItems = 4;         // heads' vectors a thread takes, where there are tokens enough

// kVec elements of a row, in pieces of up to 16 bytes, or (kSingle) one by one.
template <typename T, int kVec, bool kSingle>
struct Vec {
    static constexpr int kBytes = kVec * (int)sizeof(T), kPiece = kSingle ? (int)sizeof(T) : (kBytes < 16 ? kBytes : 16), kPieces = kBytes / kPiece;
    using P = typename Piece<kPiece>::type;
    P piece[kPieces];
    __device__ __forceinline__ void load(const T* p) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) piece[i] = reinterpret_cast<const P*>(p)[i];
    }
    __device__ __forceinline__ void store(T* p) const {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) reinterpret_cast<P*>(p)[i] = piece[i];
    }
    __device__ __forceinline__ float get(int i) const { return to_f32(reinterpret_cast<const T*>(piece)[i]); }
    __device__ __forceinline__ void set(int i, float v) { reinterpret_cast<T*>(piece)[i] = from_f32<T>(v); }
};

// A thread keeps its columns and its token, whose cosines and sines stay in registers, and goes through the heads.
struct RotarySplit {
    FastDiv units, lanes;                // of a head: vectors of pairs, then vectors that are copied; heads taken side by side
    int turned;                          // units that are turned
    int tokens;                          // of a CTA
};

// The cosine and sine of a fraction of a turn (unsigned, 2^-64 turns): what is left after the nearest quarter turn is exact
// to 2^-28 turns in fp32.
__device__ __forceinline__ float2 cos_sin(uint64_t turns) {
    const uint32_t t = (uint32_t)(turns >> 32) + (uint32_t)((turns >> 31) & 1u);
    const uint32_t quarter = (t + 0x20000000u) >> 30;
    const int32_t rest = (int32_t)(t - (quarter << 30));             // in [-2^29, 2^29)
    float s, c;
    sincospif((float)rest * 4.656612873077392578125e-10f, &s, &c);   // 2^-31: half turns
    const bool swap = quarter & 1;
    const float cc = swap ? s : c, ss = swap ? c : s;
    return make_float2(quarter == 1 || quarter == 2 ? -cc : cc, quarter == 2 || quarter == 3 ? -ss : ss);
}

// kAll: no columns are copied.
template <typename T, int kVec, bool kPairs, bool kSingle, bool kAll>
__global__ void __launch_bounds__(kRotThreads) k_rotary(const __grid_constant__ RotaryArgs a, const RotarySplit split, const FastDiv tokens) {
    extern __shared__ float2 table[];    // [tokens of the CTA][rot / 2]
    const int half = a.rot >> 1;
    const uint32_t all = (uint32_t)(a.batch * a.tokens);
    const uint32_t first = blockIdx.x * (uint32_t)split.tokens;
    const int have = (int)min((uint32_t)split.tokens, all - first);
    for (int i = threadIdx.x; i < have * half; i += kRotThreads) {
        const int k = i / half, p = i - k * half;
        const uint32_t token = first + k;
        int64_t pos;
        if (!a.pos) pos = token - tokens.div(token) * tokens.d;
        else pos = a.pos_bytes == 8 ? static_cast<const int64_t*>(a.pos)[token] : static_cast<const int32_t*>(a.pos)[token];
        float2 cs = cos_sin((uint64_t)pos * a.turns[p]);
        table[i] = make_float2(cs.x * a.gain_cos, cs.y * a.gain_sin);
    }
    __syncthreads();
    const T* x = static_cast<const T*>(a.x);
    T* y = static_cast<T*>(a.y);
    using V = Vec<T, kVec, kSingle>;
    const uint32_t places = split.units.d * split.lanes.d * (uint32_t)have;
    for (uint32_t i = threadIdx.x; i < places; i += kRotThreads) {
        const uint32_t r = split.units.div(i), unit = i - r * split.units.d;
        const uint32_t k = split.lanes.div(r), head = r - k * split.lanes.d;
        const uint32_t token = first + k, b = tokens.div(token), t = token - b * tokens.d;
        const bool turned = kAll || (int)unit < split.turned;
        const int c = turned ? (int)unit * kVec : a.rot + ((int)unit - split.turned) * kVec;
        const T* from = x + (int64_t)b * a.x_batch + (int64_t)t * a.x_token + (int64_t)head * a.x_head + c;
        T* to = y + (int64_t)b * a.y_batch + (int64_t)t * a.y_token + (int64_t)head * a.y_head + c;
        const int64_t down_x = (int64_t)split.lanes.d * a.x_head, down_y = (int64_t)split.lanes.d * a.y_head;
        const bool odd = !kAll && kSingle && c + kVec > a.dim;                    // the last one of an odd head
        constexpr int kTurns = kPairs ? kVec / 2 : kVec;
        float2 w[kTurns];
        if (turned) {
#pragma unroll
            for (int e = 0; e < kTurns; ++e) w[e] = table[k * half + (kPairs ? c / 2 : c) + e];
        }
        for (int h = (int)head; h < a.heads; h += (int)split.lanes.d, from += down_x, to += down_y) {
            V u, v;
            if (odd) {
                to[0] = from[0];
                continue;
            }
            u.load(from);
            if (!kPairs && turned) v.load(from + half);
            if (turned) {
#pragma unroll
                for (int e = 0; e < kTurns; ++e) {
                    const float m = u.get(kPairs ? 2 * e : e), n = kPairs ? u.get(2 * e + 1) : v.get(e);
                    u.set(kPairs ? 2 * e : e, m * w[e].x - n * w[e].y);
                    (kPairs ? u : v).set(kPairs ? 2 * e + 1 : e, m * w[e].y + n * w[e].x);
                }
                if (!kPairs) v.store(to + half);
            }
            u.store(to);
        }
    }
}

// Elements a thread takes at a time: up to 16 bytes (two such pieces side by side would touch every sector twice), as every head's
// row and the borders in it are aligned (strides of dimensions of one element are 0).
inline int vec_of(const RotaryArgs& a, size_t elem) {
    const int64_t inner = (a.interleaved ? a.rot : a.rot / 2) | a.dim;
    const int64_t strides = a.x_head | a.x_token | a.x_batch | a.y_head | a.y_token | a.y_batch;
    const uint64_t bytes = (uint64_t)((inner | strides) * (int64_t)elem) | reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.y);
    for (int v = (int)(16 / elem); v > 1; v /= 2)
        if ((bytes & (v * elem - 1)) == 0) return v;
    return 1;
}

}  // namespace

deft_status launch_rotary(const RotaryArgs& a, int type, cudaStream_t stream) {
    const int vec = vec_of(a, type_bytes(type));
    const bool single = a.interleaved && vec == 1;       // a pair is two elements, however it is aligned
    const int step = single ? 2 : vec, half = a.rot / 2;
    RotarySplit s{};
    s.turned = (a.interleaved ? a.rot : half) / step;
    const int64_t units = s.turned + (a.x == a.y ? 0 : (a.dim - a.rot + step - 1) / step);
    const int64_t all = a.batch * a.tokens;
    const int64_t per_token = units * a.heads;
    int64_t tokens = (kRotItems * kRotThreads + per_token - 1) / per_token;
    const int64_t fit = kRotSmem / ((int64_t)half * (int64_t)sizeof(float2));
    if (tokens > fit) tokens = fit;
    if (tokens > all) tokens = all;
    while (tokens > 1 && (all + tokens - 1) / tokens < 2 * 148) tokens = (tokens + 1) / 2;
    int64_t lanes = kRotThreads / (units * tokens);
    if (lanes > a.heads) lanes = a.heads;
    if (lanes < 1) lanes = 1;
    s.tokens = (int)tokens;
    s.units = fast_div((uint32_t)units);
    s.lanes = fast_div((uint32_t)lanes);
    const unsigned blocks = (unsigned)((all + tokens - 1) / tokens);
    const size_t smem = (size_t)tokens * half * sizeof(float2);
    const FastDiv t = fast_div((uint32_t)a.tokens);
    return with_type(type, [&](auto e) -> deft_status {
        using T = decltype(e);
        auto run = [&](auto vecs, auto pairs, auto single) {
            constexpr int kVec = decltype(vecs)::value;
            constexpr bool kPairs = decltype(pairs)::value, kSingle = decltype(single)::value;
            auto kernel = units == s.turned ? k_rotary<T, kVec, kPairs, kSingle, true> : k_rotary<T, kVec, kPairs, kSingle, false>;
            kernel<<<blocks, kRotThreads, smem, stream>>>(a, s, t);
        };
        if (a.interleaved) {
            switch (vec) {
                case 8:
                    if constexpr (sizeof(T) == 2) run(AlignTag<8>{}, AlignTag<1>{}, AlignTag<0>{});
                    break;
                case 4: run(AlignTag<4>{}, AlignTag<1>{}, AlignTag<0>{}); break;
                case 2: run(AlignTag<2>{}, AlignTag<1>{}, AlignTag<0>{}); break;
                default: run(AlignTag<2>{}, AlignTag<1>{}, AlignTag<1>{}); break;
            }
        } else {
            switch (vec) {
                case 8:
                    if constexpr (sizeof(T) == 2) run(AlignTag<8>{}, AlignTag<0>{}, AlignTag<0>{});
                    break;
                case 4: run(AlignTag<4>{}, AlignTag<0>{}, AlignTag<0>{}); break;
                case 2: run(AlignTag<2>{}, AlignTag<0>{}, AlignTag<0>{}); break;
                default: run(AlignTag<1>{}, AlignTag<0>{}, AlignTag<1>{}); break;
            }
        }
        DEFT_CUDA_TRY(cudaGetLastError());
        return DEFT_OK;
    });
}

}  // namespace deft
