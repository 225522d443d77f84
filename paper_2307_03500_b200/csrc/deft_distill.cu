// Distillation from a teacher's top logits: per row T^2 KL(teacher || student) and its gradient.
//
// A row of logits is read once.  A cluster of 1 to 8 CTAs shares it: each copies a part of its 16-byte granules into
// shared memory, takes the teacher's entries out of that part (they are few; what is left is the rest of the vocabulary, whose
// sum must not come from a difference), sums the exponentials of the rest and of the entries apart, and the CTAs exchange
// these sums.  The gradient is then formed from shared memory and written; the entries' elements last.
#include <cooperative_groups.h>

#include "deft_dense.cuh"

namespace deft {
namespace {

namespace cg = cooperative_groups;

constexpr int kMostCluster = 8;
constexpr int kPartBytes = 52 * 1024;     // of a row, per CTA, where there are rows enough: four CTAs per SM

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// What the CTAs of a row tell each other.  The two sums have a reference of their own each: the rest may lie far below the
// entries, and its logarithm counts all the same.
struct PartSums {
    float rest_most, entry_most;           // the largest logits
    float rest, entries;                   // sums of 2^((z - most) c1)
    double cross;                          // sum over the part's entries of q (log q - z / T)
};
// What the logits of a sum are taken relative to: the largest, unless there is nothing but -inf.  (The difference is formed before
// it is scaled: a logit of the type's lowest value times c1 would be beyond it.)
__device__ __forceinline__ float reference(float most) { return most == -INFINITY ? 0.0f : most; }
__device__ __forceinline__ float power(float z, float from, float c1) { return exp2_fast((z - from) * c1); }

template <typename T> __device__ __forceinline__ T lowest();
template <> __device__ __forceinline__ float lowest<float>() { return __int_as_float(0xff800000); }
template <> __device__ __forceinline__ __nv_bfloat16 lowest<__nv_bfloat16>() { return __ushort_as_bfloat16(0xff80); }
template <> __device__ __forceinline__ __half lowest<__half>() { return __ushort_as_half(0xfc00); }

// Takes an element out of shared memory: -inf takes its place.  True for the one thread that found it there first (an element
// that was -inf has no share in any sum, whoever claims it).
__device__ __forceinline__ bool claim(float* p) { return atomicExch(reinterpret_cast<unsigned*>(p), 0xff800000u) != 0xff800000u; }
template <typename T>
__device__ __forceinline__ bool claim(T* p) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    unsigned* word = reinterpret_cast<unsigned*>(at & ~(uintptr_t)3);
    const int up = (at & 2) ? 16 : 0;
    const T low = lowest<T>();
    const unsigned mark = *reinterpret_cast<const unsigned short*>(&low);
    unsigned was = *reinterpret_cast<volatile unsigned*>(word);
    while (true) {
        if (((was >> up) & 0xffffu) == mark) return false;
        const unsigned seen = atomicCAS(word, was, (was & ~(0xffffu << up)) | (mark << up));
        if (seen == was) return true;
        was = seen;
    }
}

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
// Over the CTA; `slots` has 32 places and is free again after the next barrier.
__device__ __forceinline__ float cta_max(float v, float* slots) {
    v = warp_max(v);
    if ((threadIdx.x & 31) == 0) slots[threadIdx.x >> 5] = v;
    __syncthreads();
    const int warps = blockDim.x >> 5;
    return warp_max((int)(threadIdx.x & 31) < warps ? slots[threadIdx.x & 31] : -INFINITY);
}
__device__ __forceinline__ float cta_sum(float v, float* slots) {
    v = warp_sum(v);
    if ((threadIdx.x & 31) == 0) slots[threadIdx.x >> 5] = v;
    __syncthreads();
    const int warps = blockDim.x >> 5;
    return warp_sum((int)(threadIdx.x & 31) < warps ? slots[threadIdx.x & 31] : 0.0f);
}
__device__ __forceinline__ double cta_sum(double v, double* slots) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0) slots[threadIdx.x >> 5] = v;
    __syncthreads();
    const int warps = blockDim.x >> 5;
    v = (int)(threadIdx.x & 31) < warps ? slots[threadIdx.x & 31] : 0.0;
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

template <typename T>
struct Granule {
    static constexpr int kPer = 16 / (int)sizeof(T);
    uint4 raw;
    __device__ __forceinline__ float get(int i) const { return to_f32(reinterpret_cast<const T*>(&raw)[i]); }
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

template <typename T>
__global__ void __launch_bounds__(512) k_distill(const __grid_constant__ DistillArgs a, const int granules_most) {
    constexpr int kPer = Granule<T>::kPer;
    extern __shared__ __align__(16) char smem[];
    T* part = reinterpret_cast<T*>(smem);                                        // this CTA's granules
    int* col = reinterpret_cast<int*>(smem + (size_t)granules_most * 16);         // [top] an entry's column, or -1
    float* prob = reinterpret_cast<float*>(col + a.top);                          // [top] q
    float* own = prob + a.top;                                                    // [top] the logit, where this CTA has it and claimed it
    __shared__ float slots[3][32];
    __shared__ double dslots[2][32];
    __shared__ PartSums sums;
    __shared__ int twice;
    cg::cluster_group cluster = cg::this_cluster();
    const int ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank(), tid = threadIdx.x, threads = blockDim.x;
    const int64_t row = blockIdx.x / ctas;
    const T* z = static_cast<const T*>(a.logits) + row * a.ld;
    T* g = a.grad ? static_cast<T*>(a.grad) + row * a.ld_grad : nullptr;
    // the row's granules, the first of which may begin before it; this CTA's share and its columns
    const int shift = (int)(reinterpret_cast<uintptr_t>(z) & 15u) / (int)sizeof(T);
    const int granules = (a.vocab + shift + kPer - 1) / kPer;
    const int g0 = (int)((int64_t)granules * rank / ctas), g1 = (int)((int64_t)granules * (rank + 1) / ctas);
    const int c0 = max(0, g0 * kPer - shift), c1 = min(a.vocab, g1 * kPer - shift);
    const int base = g0 * kPer - shift;                                          // column of part[0]
    // where the gradient's 16-byte granules lie
    const int g_shift = g ? (int)(reinterpret_cast<uintptr_t>(g) & 15u) / (int)sizeof(T) : 0;

    const float weight = a.weight ? a.weight[row] : 1.0f;
    if (weight == 0.0f) {                  // nothing is read of a row that does not count (the same for the whole cluster)
        if (g) for (int c = c0 + tid; c < c1; c += threads) g[c] = from_f32<T>(0.0f);
        if (a.loss && rank == 0 && tid == 0) a.loss[row] = 0.0f;
        return;
    }
    const uint4* from = reinterpret_cast<const uint4*>(z - shift) + g0;
    for (int i = tid; i < g1 - g0; i += threads)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(smem) + (uint32_t)i * 16u), "l"(from + i) : "memory");
    asm volatile("cp.async.commit_group;" ::: "memory");

    // the teacher: log q_j = t_j / T - norm
    if (tid == 0) twice = 0;
    double norm;
    if (a.teacher_lse) {
        norm = (double)a.teacher_lse[row];
    } else {
        float most = -INFINITY;
        for (int j = tid; j < a.top; j += threads)
            if (id_at(a, row, j) >= 0) most = fmaxf(most, teacher_at(a, row, j));
        most = cta_max(most, slots[0]);
        float sum = 0.0f;
        for (int j = tid; j < a.top; j += threads)
            if (id_at(a, row, j) >= 0 && most != -INFINITY) sum += expf((float)(((double)teacher_at(a, row, j) - (double)most) * a.inv_temp));
        sum = cta_sum(sum, slots[1]);
        norm = most == -INFINITY ? 0.0 : (double)most * a.inv_temp + log((double)sum);
    }
    // in 64 bits: the loss is what is left of sums that nearly cancel
    double q_sum = 0.0;
    for (int j = tid; j < a.top; j += threads) {
        const int id = id_at(a, row, j);
        const float q = id >= 0 ? expf((float)((double)teacher_at(a, row, j) * a.inv_temp - norm)) : 0.0f;
        col[j] = id;
        prob[j] = q;
        q_sum += (double)q;
    }
    q_sum = cta_sum(q_sum, dslots[0]);

    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    // what the first and last granule hold beside the row
    if (tid < kPer) {
        if (base + tid < 0) part[tid] = lowest<T>();
        const int last = (g1 - g0 - 1) * kPer + tid;
        if (g1 > g0 && base + last >= a.vocab) part[last] = lowest<T>();
    }
    double cross = 0.0;
    for (int j = tid; j < a.top; j += threads) {
        const bool here = col[j] >= c0 && col[j] < c1;
        const float v = here ? to_f32(part[col[j] - base]) : 0.0f;
        own[j] = v;
        if (here && prob[j] != 0.0f)
            cross += (double)prob[j] * ((double)teacher_at(a, row, j) * a.inv_temp - norm - (double)v * ((double)a.c1 * 0.693147180559945309417));
    }
    __syncthreads();
    float entry_most = -INFINITY, rest_most = -INFINITY;
    for (int j = tid; j < a.top; j += threads) {
        const bool here = col[j] >= c0 && col[j] < c1;
        if (!here) {
            if (col[j] >= 0) col[j] = -2;              // another CTA's
        } else if (claim(part + (col[j] - base))) {
            entry_most = fmaxf(entry_most, own[j]);
        } else {
            if (own[j] != -INFINITY) twice = 1;
            col[j] = -3 - col[j];                      // not the first of its column, or an element without any share: below -2
        }
    }
    entry_most = cta_max(entry_most, slots[2]);
    const Granule<T>* cells = reinterpret_cast<const Granule<T>*>(part);
    for (int i = tid; i < g1 - g0; i += threads) {
        const Granule<T> c = cells[i];
#pragma unroll
        for (int e = 0; e < kPer; ++e) rest_most = fmaxf(rest_most, c.get(e));
    }
    rest_most = cta_max(rest_most, slots[1]);
    float from_rest = reference(rest_most), rest = 0.0f, entries = 0.0f;
    for (int i = tid; i < g1 - g0; i += threads) {
        const Granule<T> c = cells[i];
        float s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int e = 0; e < kPer; ++e) s[e & 1] += power(c.get(e), from_rest, a.c1);
        rest += s[0] + s[1];
    }
    float from_entry = reference(entry_most);
    for (int j = tid; j < a.top; j += threads)
        if (col[j] >= 0) entries += power(own[j], from_entry, a.c1);
    rest = cta_sum(rest, slots[0]);
    entries = cta_sum(entries, slots[2]);
    cross = cta_sum(cross, dslots[1]);
    if (ctas > 1) {
        if (tid == 0) sums = PartSums{rest_most, entry_most, rest, entries, cross};
        cluster.sync();
        rest_most = entry_most = -INFINITY;
        for (int c = 0; c < ctas; ++c) {
            const PartSums* o = cluster.map_shared_rank(&sums, c);
            rest_most = fmaxf(rest_most, o->rest_most);
            entry_most = fmaxf(entry_most, o->entry_most);
        }
        from_rest = reference(rest_most);
        from_entry = reference(entry_most);
        rest = entries = 0.0f;
        cross = 0.0;
        for (int c = 0; c < ctas; ++c) {               // (a part without any is 0, or NaN, whatever it is multiplied by)
            const PartSums* o = cluster.map_shared_rank(&sums, c);
            rest += o->rest_most == -INFINITY ? o->rest : o->rest * power(o->rest_most, from_rest, a.c1);
            entries += o->entry_most == -INFINITY ? o->entries : o->entries * power(o->entry_most, from_entry, a.c1);
            cross += o->cross;
        }
        cluster.sync();                    // nobody leaves while others read its sums
    }
    // total: the sum over the vocabulary relative to from_all
    const float from_all = rest_most == -INFINITY ? from_entry : (entry_most == -INFINITY ? from_rest : fmaxf(from_rest, from_entry));
    const float rest_up = power(from_rest, from_all, a.c1);
    const float total = (rest == 0.0f ? 0.0f : rest * rest_up) + (entries == 0.0f ? 0.0f : entries * power(from_entry, from_all, a.c1));
    // the teacher's probability outside its entries; none where there is no other logit
    const float left = a.teacher_lse && !(rest == 0.0f) ? (float)fmax(0.0, 1.0 - q_sum) : 0.0f;
    const float mass = (float)(q_sum + (double)left);
    if (a.loss && rank == 0 && tid == 0) {
        const double by = (double)a.c1 * 0.693147180559945309417, lse = (double)from_all * by + log((double)total);
        double loss = cross + q_sum * lse;
        if (left > 0.0f) loss += (double)left * (log((double)left) - log((double)rest) - (double)from_rest * by + lse);
        if (q_sum == 0.0 && left == 0.0f) loss = 0.0;
        a.loss[row] = (float)(loss * (double)weight * a.loss_factor);
    }
    if (!g) return;
    const float f = weight * a.grad_factor;
    const float k_top = mass / total * f;
    // (rest = 0: nothing but -inf, whose share is 0, and NaN where the entries have none either)
    const float k_rest = rest == 0.0f ? 0.0f * k_top : (mass * rest_up / total - left / rest) * f;
    if (g_shift == shift) {
        uint4* to = reinterpret_cast<uint4*>(g - shift) + g0;
        for (int i = tid; i < g1 - g0; i += threads) {
            const Granule<T> c = cells[i];
            Granule<T> o;
#pragma unroll
            for (int e = 0; e < kPer; ++e) reinterpret_cast<T*>(&o.raw)[e] = from_f32<T>(power(c.get(e), from_rest, a.c1) * k_rest);
            const int first = base + i * kPer;
            if (first >= 0 && first + kPer <= a.vocab) {
                to[i] = o.raw;
            } else {
#pragma unroll
                for (int e = 0; e < kPer; ++e)
                    if (first + e >= 0 && first + e < a.vocab) g[first + e] = reinterpret_cast<const T*>(&o.raw)[e];
            }
        }
    } else {
        for (int c = c0 + tid; c < c1; c += threads) g[c] = from_f32<T>(power(to_f32(part[c - base]), from_rest, a.c1) * k_rest);
    }
    __syncthreads();
    // the entries' own elements: the probabilities of a column's entries added in their order
    for (int j = tid; j < a.top; j += threads) {
        int c = col[j];
        float v = own[j], q = prob[j];
        if (c < -2) {                      // no share in the sums: an element that is -inf; its first entry writes it
            c = -3 - c;
            if (v > -INFINITY || v != v) continue;
            bool earlier = false;
            for (int i = 0; i < j; ++i) earlier |= col[i] == col[j];
            if (earlier) continue;
            for (int i = j + 1; i < a.top; ++i)
                if (col[i] == col[j]) q += prob[i];
        } else if (c < 0) {
            continue;
        } else if (twice) {
            q = 0.0f;
            for (int i = 0; i < a.top; ++i)
                if (col[i] == c || col[i] == -3 - c) q += prob[i];
        }
        g[c] = from_f32<T>(power(v, from_all, a.c1) * k_top - q * f);
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
    const int granules = (int)((bytes + 15) / 16 / ctas + 2);
    const size_t smem = (size_t)granules * 16 + (size_t)a.top * 12;
    int threads = 128;
    while (threads < 512 && granules > threads * 8) threads *= 2;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)ctas;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return with_type(type, [&](auto t) -> deft_status {
        using T = decltype(t);
        auto kernel = k_distill<T>;
        if (smem > 40 * 1024) DEFT_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
        DEFT_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, a, granules));
        return DEFT_OK;
    });
}

}  // namespace deft
