// Distillation from a teacher's top logits: per row T^2 KL(teacher || student) and its gradient.
//
// A row of logits is read once.  A cluster of 1 to 8 CTAs shares it: each copies a part of its 16-byte granules into
// shared memory.  The first warp, meanwhile, works out the teacher's probabilities and marks the entries' elements: what is
// left is the rest of the vocabulary, whose sum must not come from a difference.  All warps sum the powers of the rest,
// the CTAs exchange their sums, and the gradient is formed from shared memory and written.
#include <cooperative_groups.h>

#include "deft_dense.cuh"

namespace deft {
namespace {

constexpr int kMostCluster = 8;
constexpr int kMostThreads = 512;         // that work on the row
constexpr int kPartBytes = 51712;         // of a row, per CTA, where there are rows enough: four CTAs per SM

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
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
__device__ __forceinline__ uint64_t exp2_pair(uint64_t x) {
    const float2 v = unpair(x);
    return pair(exp2_fast(v.x), exp2_fast(v.y));
}

// The natural logarithm of a positive float to 2^-26 or so, whatever its size: the exponent's part in 64 bits.
__device__ __forceinline__ double log_of(float x) {
    if (!(x > 0.0f && x < INFINITY)) return (double)logf(x);
    int e = 0;
    if (x < 1.17549435e-38f) x *= 16777216.0f, e = -24;
    const int bits = __float_as_int(x) - 0x3f3504f3;          // of sqrt(1/2): the rest lies in [sqrt(1/2), sqrt(2))
    e += bits >> 23;
    return (double)e * 0.693147180559945309417 + (double)logf(__int_as_float((bits & 0x7fffff) + 0x3f3504f3));
}

// Powers of a part's logits: 2^(z c1 - from), or, where that could lose them, 2^((z - from) c1).
struct Reference {
    bool careful;
    float from;
    double exponent;                       // what the powers are relative to, in powers of two
};

// What the CTAs of a row tell each other: two sums, the exponents they are relative to, and
// sum over the part's entries of q (log q - z / T).
struct PartSums {
    double rest_at, entries_at, cross;
    float rest, entries;
};

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// Over groups of eight lanes.
template <typename F>
__device__ __forceinline__ F eight_sum(F v) {
#pragma unroll
    for (int o = 4; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ double eight_max(double v) {
#pragma unroll
    for (int o = 4; o; o >>= 1) v = fmax(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
__device__ __forceinline__ float warps_max(const float* slots, int warps) {
    const int lane = threadIdx.x & 31;
    return warp_max(lane < warps ? slots[lane] : -INFINITY);
}
__device__ __forceinline__ float warps_sum(const float* slots, int warps) {
    const int lane = threadIdx.x & 31;
    return warp_sum(lane < warps ? slots[lane] : 0.0f);
}

// Sixteen bytes of a row as pairs of fp32 numbers.
template <typename T> struct Granule;
template <>
struct Granule<float> {
    static constexpr int kPer = 4, kPairs = 2;
    uint4 raw;
    __device__ __forceinline__ uint64_t get(int i) const { return i ? pair(__uint_as_float(raw.z), __uint_as_float(raw.w)) : pair(__uint_as_float(raw.x), __uint_as_float(raw.y)); }
    __device__ __forceinline__ void set(int i, uint64_t p) {
        const float2 v = unpair(p);
        if (i) raw.z = __float_as_uint(v.x), raw.w = __float_as_uint(v.y);
        else raw.x = __float_as_uint(v.x), raw.y = __float_as_uint(v.y);
    }
};
template <>
struct Granule<__nv_bfloat16> {
    static constexpr int kPer = 8, kPairs = 4;
    uint4 raw;
    __device__ __forceinline__ uint32_t& word(int i) { return i == 0 ? raw.x : (i == 1 ? raw.y : (i == 2 ? raw.z : raw.w)); }
    __device__ __forceinline__ uint64_t get(int i) const {
        const uint32_t w = const_cast<Granule*>(this)->word(i);
        return pair(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    }
    __device__ __forceinline__ void set(int i, uint64_t p) {
        const float2 v = unpair(p);
        const __nv_bfloat162 h = __floats2bfloat162_rn(v.x, v.y);
        word(i) = *reinterpret_cast<const uint32_t*>(&h);
    }
};
template <>
struct Granule<__half> {
    static constexpr int kPer = 8, kPairs = 4;
    uint4 raw;
    __device__ __forceinline__ uint32_t& word(int i) { return i == 0 ? raw.x : (i == 1 ? raw.y : (i == 2 ? raw.z : raw.w)); }
    __device__ __forceinline__ uint64_t get(int i) const {
        const uint32_t w = const_cast<Granule*>(this)->word(i);
        const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&w));
        return pair(v.x, v.y);
    }
    __device__ __forceinline__ void set(int i, uint64_t p) {
        const float2 v = unpair(p);
        const __half2 h = __floats2half2_rn(v.x, v.y);
        word(i) = *reinterpret_cast<const uint32_t*>(&h);
    }
};

__device__ __forceinline__ float teacher_at(const DistillArgs& a, int64_t row, int j) {
    const int64_t at = row * a.ld_teacher + j;
    if (a.teacher_type == DEFT_F32) return static_cast<const float*>(a.teacher)[at];
    if (a.teacher_type == DEFT_BF16) return to_f32(static_cast<const __nv_bfloat16*>(a.teacher)[at]);
    return to_f32(static_cast<const __half*>(a.teacher)[at]);
}
__device__ __forceinline__ int id_at(const DistillArgs& a, int64_t row, int j) {
    const int64_t at = row * a.ld_ids + j;
    const int64_t id = a.id_bytes == 8 ? static_cast<const int64_t*>(a.ids)[at] : static_cast<const int32_t*>(a.ids)[at];
    return id >= 0 && id < a.vocab ? (int)id : -1;
}

// The teacher's entries of a row in shared memory, and a byte for each granule of the part: which of its elements are entries.
struct Entries {
    int* col;                              // column; -1: none; -2: another CTA's; -3 - column: not the first of its column
    float *value, *prob;                   // t, then the student's logit; q
    unsigned* marks;
    __device__ __forceinline__ Entries(char* at, int top) : col(reinterpret_cast<int*>(at)) {
        value = reinterpret_cast<float*>(col + top);
        prob = value + top;
        marks = reinterpret_cast<unsigned*>(prob + top);
    }
    __device__ __forceinline__ unsigned marked(int granule) const { return reinterpret_cast<const unsigned char*>(marks)[granule]; }
};
constexpr size_t kEntryBytes = 12;

// What stands for an element without a share.
template <typename T> __device__ __forceinline__ T lowest();
template <> __device__ __forceinline__ float lowest<float>() { return __int_as_float(0xff800000); }
template <> __device__ __forceinline__ __nv_bfloat16 lowest<__nv_bfloat16>() { return __ushort_as_bfloat16(0xff80); }
template <> __device__ __forceinline__ __half lowest<__half>() { return __ushort_as_half(0xfc00); }

// The largest element of a granule.
template <typename T>
__device__ __forceinline__ float most_of(const Granule<T>& g) {
    float most = -INFINITY;
#pragma unroll
    for (int p = 0; p < Granule<T>::kPairs; ++p) {
        const float2 v = unpair(g.get(p));
        most = fmaxf(most, fmaxf(v.x, v.y));
    }
    return most;
}
template <typename T, bool kCareful>
__device__ __forceinline__ uint64_t powers(uint64_t z, uint64_t c, uint64_t minus_from) {
    return exp2_pair(kCareful ? mul2(add2(z, minus_from), c) : fma2(z, c, minus_from));
}
// A granule of this thread without its entries.
template <typename T>
__device__ __forceinline__ Granule<T> rest_of(const Granule<T>* cells, int i, const Entries& entry) {
    Granule<T> g = cells[i];
    const unsigned marked = entry.marked(i);
    if (marked) {
#pragma unroll
        for (int e = 0; e < Granule<T>::kPer; ++e)
            if (marked >> e & 1u) reinterpret_cast<T*>(&g.raw)[e] = lowest<T>();
    }
    return g;
}
// The sum of the powers of this thread's granules.
template <typename T, bool kCareful>
__device__ __forceinline__ float sum_powers(const Granule<T>* cells, int n, int threads, const Entries& entry, const Reference& ref, float c1) {
    const uint64_t c = pair(c1, c1), from = pair(-ref.from, -ref.from);
    uint64_t s[2] = {0, 0};
    for (int i = threadIdx.x; i < n; i += threads) {
        const Granule<T> g = rest_of(cells, i, entry);
#pragma unroll
        for (int p = 0; p < Granule<T>::kPairs; ++p) s[p & 1] = add2(s[p & 1], powers<T, kCareful>(g.get(p), c, from));
    }
    const float2 v = unpair(add2(s[0], s[1]));
    return v.x + v.y;
}
// The gradient of this thread's granules, as if there were no entries among them.  kWhole: the gradient's granules lie like the logits'.
template <typename T, bool kCareful, bool kWhole>
__device__ __forceinline__ void write_grad(const Granule<T>* cells, int n, int threads, int base, int vocab, T* g, const Reference& ref, float c1, float k1) {
    constexpr int kPer = Granule<T>::kPer;
    const uint64_t c = pair(c1, c1), from = pair(-ref.from, -ref.from), k = pair(k1, k1);
    for (int i = threadIdx.x; i < n; i += threads) {
        const Granule<T> in = cells[i];
        Granule<T> o;
#pragma unroll
        for (int p = 0; p < Granule<T>::kPairs; ++p) o.set(p, mul2(powers<T, kCareful>(in.get(p), c, from), k));
        const int first = base + i * kPer;
        if (kWhole && first >= 0 && first + kPer <= vocab) {
            *reinterpret_cast<uint4*>(g + first) = o.raw;
        } else {
            for (int e = 0; e < kPer; ++e)
                if (first + e >= 0 && first + e < vocab) g[first + e] = reinterpret_cast<const T*>(&o.raw)[e];
        }
    }
}

// What the first warp works out for all: factors of the gradient, the exponent that the row's sum is relative to.
struct Factors {
    double all_at;
    float rest, top;
};

// The loss of a row and the factors of its gradient from the CTAs' sums.  One warp; a lane for each CTA, four times over.
__device__ __forceinline__ Factors factors_of(const DistillArgs& a, const PartSums& o, float rest_here, double here_at, double q_sum, float weight, int64_t row, bool write_loss) {
    const double none = -(double)INFINITY, rest_at = !(o.rest == 0.0f) ? o.rest_at : none, entries_at = !(o.entries == 0.0f) ? o.entries_at : none;
    const double rest_most = eight_max(rest_at), all_most = fmax(rest_most, eight_max(entries_at));
    const float total = eight_sum((rest_at == none ? 0.0f : o.rest * exp2_fast((float)(rest_at - all_most))) +
                                  (entries_at == none ? 0.0f : o.entries * exp2_fast((float)(entries_at - all_most))));
    const float all_rest = eight_sum(rest_at == none ? 0.0f : o.rest * exp2_fast((float)(rest_at - rest_most)));
    // the teacher's probability outside its entries; none where there is no other logit
    const float left = a.teacher_lse && !(all_rest == 0.0f) ? (float)fmax(0.0, 1.0 - q_sum) : 0.0f;
    const float mass = (float)(q_sum + (double)left);
    const float f = weight * a.grad_factor, top = mass / total * f;
    // (a part with nothing but -inf: the share is 0, and NaN where the whole row has no other)
    const float rest = rest_here == 0.0f ? 0.0f * top : (mass / total * exp2_fast((float)(here_at - all_most)) - left / all_rest * exp2_fast((float)(here_at - rest_most))) * f;
    if (write_loss) {
        const double cross = eight_sum(o.cross);
        if ((threadIdx.x & 31) == 0) {
            const double ln2 = 0.693147180559945309417, lse = all_most * ln2 + log_of(total);
            double loss = cross + q_sum * lse;
            if (left > 0.0f) loss += (double)left * (log_of(left) - log_of(all_rest) - rest_most * ln2 + lse);
            if (q_sum == 0.0 && left == 0.0f) loss = 0.0;
            a.loss[row] = (float)(loss * (double)weight * a.loss_factor);
        }
    }
    return Factors{all_most, rest, top};
}

// The last warp of a CTA works on the entries, the others on the part of the row.
template <typename T>
__global__ void __launch_bounds__(kMostThreads + 32, 1) k_distill(const __grid_constant__ DistillArgs a, const int granules_most, const int ctas) {
    constexpr int kPer = Granule<T>::kPer;
    extern __shared__ __align__(16) char smem[];
    T* part = reinterpret_cast<T*>(smem);                                        // this CTA's granules
    Granule<T>* cells = reinterpret_cast<Granule<T>*>(smem);
    const Entries entry(smem + (size_t)granules_most * 16, a.top);
    __shared__ float slots[2][kMostThreads / 32];
    __shared__ PartSums sums[kMostCluster];
    __shared__ Factors factors;
    __shared__ int twice;
    const int tid = threadIdx.x, threads = (int)blockDim.x - 32, warps = threads >> 5, warp = tid >> 5, lane = tid & 31;
    const bool for_entries = warp == warps;
    int rank = 0;
    if (ctas > 1) {
        asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
        asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");    // (waited for before others' shared memory is written)
    }
    const int64_t row = blockIdx.x / (unsigned)ctas;
    const T* z = static_cast<const T*>(a.logits) + row * a.ld;
    T* g = a.grad ? static_cast<T*>(a.grad) + row * a.ld_grad : nullptr;
    // the row's granules, the first of which may begin before it; this CTA's share and its columns
    const int shift = (int)(reinterpret_cast<uintptr_t>(z) & 15u) / (int)sizeof(T);
    const int granules = (a.vocab + shift + kPer - 1) / kPer;
    const int g0 = (int)((int64_t)granules * rank / ctas), g1 = (int)((int64_t)granules * (rank + 1) / ctas), n = g1 - g0;
    const int c0 = max(0, g0 * kPer - shift), c1 = min(a.vocab, g1 * kPer - shift);
    const int base = g0 * kPer - shift;                                          // column of part[0]

    const float weight = a.weight ? a.weight[row] : 1.0f;
    if (weight == 0.0f) {                  // nothing is read of a row that does not count (the same for the whole cluster)
        if (g) for (int c = c0 + tid; c < c1; c += blockDim.x) g[c] = from_f32<T>(0.0f);
        if (a.loss && rank == 0 && tid == 0) a.loss[row] = 0.0f;
        if (ctas > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        return;
    }
    double norm = 0.0, q_sum = 0.0, cross = 0.0;   // of the last warp: log q_j = t_j / T - norm; sums of q and, over the part's entries, q log q
    if (for_entries) {
        // (The loss is what is left of sums that nearly cancel: its terms are added in 64 bits.)
        int id[2] = {-1, -1};
        float t[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < 2; ++i)        // the first entries' loads are under way together
            if (lane + 32 * i < a.top) {
                id[i] = id_at(a, row, lane + 32 * i);
                t[i] = teacher_at(a, row, lane + 32 * i);
            }
        if (a.teacher_lse) norm = (double)a.teacher_lse[row];
        for (int i = lane; i < (n + 3) / 4; i += 32) entry.marks[i] = 0;
        if (lane == 0) twice = 0;
        float most = -INFINITY;
        auto keep = [&](int j, int col, float value) {
            entry.col[j] = col;
            entry.value[j] = value;
            if (col >= 0) most = fmaxf(most, value);
        };
        if (lane < a.top) keep(lane, id[0], t[0]);
        if (lane + 32 < a.top) keep(lane + 32, id[1], t[1]);
        for (int j = lane + 64; j < a.top; j += 32) keep(j, id_at(a, row, j), teacher_at(a, row, j));
        if (!a.teacher_lse) {
            most = warp_max(most);
            float sum = 0.0f;
            for (int j = lane; j < a.top; j += 32)
                if (entry.col[j] >= 0 && most != -INFINITY) sum += expf((float)(((double)entry.value[j] - (double)most) * a.inv_temp));
            norm = most == -INFINITY ? 0.0 : (double)most * a.inv_temp + log_of(warp_sum(sum));
        }
        __syncwarp();
        for (int j = lane; j < a.top; j += 32) {
            const int col = entry.col[j];
            const double log_q = (double)entry.value[j] * a.inv_temp - norm;
            const float q = col >= 0 ? expf((float)log_q) : 0.0f;
            entry.prob[j] = q;
            q_sum += (double)q;
            if (col < 0) continue;
            if (col < c0 || col >= c1) {
                entry.col[j] = -2;
                continue;
            }
            if (q != 0.0f) cross += (double)q * log_q;
            const int cell = (col - base) / kPer, bit = (cell & 3) * 8 + (col - base) % kPer;
            if (atomicOr(entry.marks + (cell >> 2), 1u << bit) >> bit & 1u) {
                entry.col[j] = -3 - col;
                twice = 1;
            }
        }
        q_sum = warp_sum(q_sum);
    } else {
        // every thread copies the granules that it works on
        const uint4* from = reinterpret_cast<const uint4*>(z - shift) + g0;
        for (int i = tid; i < n; i += threads)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(smem) + (uint32_t)i * 16u), "l"(from + i) : "memory");
        asm volatile("cp.async.wait_all;" ::: "memory");
        // what the first and last granule hold beside the row
        if (n > 0 && tid == 0)
            for (int c = base; c < 0; ++c) part[c - base] = lowest<T>();
        if (n > 0 && tid == (n - 1) % threads)
            for (int c = max(c1, base); c < base + n * kPer; ++c) part[c - base] = lowest<T>();
        // what the powers are relative to: the largest of a granule of every thread, which is seldom far from the largest of all
        const float most = warp_max(tid < n ? most_of<T>(cells[tid]) : -INFINITY);
        if (lane == 0) slots[0][warp] = most;
    }
    __syncthreads();
    Reference ref{false, 0.0f, 0.0};
    {
        const float most = warps_max(slots[0], warps);
        ref.from = most == -INFINITY ? 0.0f : most * a.c1;
        ref.exponent = (double)ref.from;
    }
    if (for_entries) {                     // the entries' logits
        float most = -INFINITY;
        for (int j = lane; j < a.top; j += 32) {
            const int col = entry.col[j];
            if (col == -1 || col == -2) continue;
            const float own = to_f32(part[(col < 0 ? -3 - col : col) - base]);
            entry.value[j] = own;
            if (entry.prob[j] != 0.0f) cross -= (double)entry.prob[j] * ((double)own * ((double)a.c1 * 0.693147180559945309417));
            if (col >= 0) most = fmaxf(most, own);
        }
        most = warp_max(most);
        const float near = most == -INFINITY ? 0.0f : most;
        float entries = 0.0f;
        for (int j = lane; j < a.top; j += 32)
            if (entry.col[j] >= 0) entries += exp2_fast((entry.value[j] - near) * a.c1);
        entries = warp_sum(entries);
        cross = warp_sum(cross);
        if (lane == 0) sums[rank] = PartSums{0.0, (double)near * (double)a.c1, cross, 0.0f, entries};
        __syncwarp();
    } else {
        const float rest = warp_sum(sum_powers<T, false>(cells, n, threads, entry, ref, a.c1));
        if (lane == 0) slots[1][warp] = rest;
    }
    __syncthreads();
    float rest = warps_sum(slots[1], warps);
    // the sample is too far off (or something is no number).  Powers and factors below 2^-126 are 0: within these bounds no
    // probability above 2^-96 is lost
    if (!(rest > 9.5367431640625e-07f && rest < 1073741824.0f)) {             // 2^-20, 2^30
        if (!for_entries) {
            float most = -INFINITY;
            for (int i = tid; i < n; i += threads) most = fmaxf(most, most_of<T>(rest_of(cells, i, entry)));
            most = warp_max(most);
            if (lane == 0) slots[0][warp] = most;
        }
        __syncthreads();
        const float most = warps_max(slots[0], warps);
        ref.careful = true;
        ref.from = most == -INFINITY ? 0.0f : most;
        ref.exponent = (double)ref.from * (double)a.c1;
        if (!for_entries) {
            rest = warp_sum(sum_powers<T, true>(cells, n, threads, entry, ref, a.c1));
            if (lane == 0) slots[1][warp] = rest;
        }
        __syncthreads();
        rest = warps_sum(slots[1], warps);
    }
    PartSums mine{};
    if (for_entries) {
        mine = sums[rank];
        mine.rest = rest;
        mine.rest_at = ref.exponent;
        __syncwarp();
    }
    if (ctas > 1) {
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");      // all CTAs run: their shared memory may be written
        if (for_entries) {
            if (lane < ctas) *cooperative_groups::this_cluster().map_shared_rank(&sums[rank], lane) = mine;
            asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        } else {
            asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
        }
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        if (for_entries) mine = sums[lane & 7];
    }
    if (for_entries) {
        if ((lane & 7) >= ctas) mine = PartSums{};
        const Factors k = factors_of(a, mine, rest, ref.exponent, q_sum, weight, row, a.loss && rank == 0);
        if (lane == 0) factors = k;
    }
    if (!g) return;
    __syncthreads();
    const Factors k = factors;
    if (!for_entries) {
        const bool whole = (reinterpret_cast<uintptr_t>(g) & 15u) == (reinterpret_cast<uintptr_t>(z) & 15u);
        if (ref.careful) write_grad<T, true, false>(cells, n, threads, base, a.vocab, g, ref, a.c1, k.rest);
        else if (whole) write_grad<T, false, true>(cells, n, threads, base, a.vocab, g, ref, a.c1, k.rest);
        else write_grad<T, false, false>(cells, n, threads, base, a.vocab, g, ref, a.c1, k.rest);
    }
    __syncthreads();
    // the entries' own elements: the probabilities of a column's entries added in their order
    for (int j = tid; j < a.top; j += blockDim.x) {
        const int c = entry.col[j];
        if (c < 0) continue;
        float q = entry.prob[j];
        if (twice) {
            q = 0.0f;
            for (int i = 0; i < a.top; ++i)
                if (entry.col[i] == c || entry.col[i] == -3 - c) q += entry.prob[i];
        }
        g[c] = from_f32<T>(exp2_fast((float)((double)entry.value[j] * (double)a.c1 - k.all_at)) * k.top - q * (weight * a.grad_factor));
    }
}

}  // namespace

deft_status launch_distill(const DistillArgs& a, int type, cudaStream_t stream) {
    const int64_t elem = (int64_t)type_bytes(type), bytes = a.vocab * elem + 16;
    int ctas = 1;
    while (ctas < kMostCluster && bytes / ctas > kPartBytes) ctas *= 2;
    while (ctas < kMostCluster && a.rows * ctas < 2 * 148 && bytes / ctas > 8 * 1024) ctas *= 2;
    const int64_t blocks = a.rows * ctas;
    if (blocks > 0x7fffffffLL) return DEFT_ERR_TOO_LARGE;
    const int granules = ((int)((bytes + 15) / 16 / ctas) + 2 + 3) & ~3;
    const size_t smem = (size_t)granules * 17 + (size_t)a.top * kEntryBytes;
    int threads = 32;
    while (threads < kMostThreads && granules > threads * 16) threads *= 2;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)ctas;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3((unsigned)threads + 32);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cfg.attrs = &attr;
    cfg.numAttrs = ctas > 1 ? 1 : 0;
    return with_type(type, [&](auto t) -> deft_status {
        using T = decltype(t);
        auto kernel = k_distill<T>;
        if (smem > 40 * 1024) DEFT_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
        DEFT_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, a, granules, ctas));
        return DEFT_OK;
    });
}

}  // namespace deft
