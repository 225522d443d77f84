// Distillation from a teacher's top logits: per row T^2 KL(teacher || student) and its gradient.
//
// A row of logits is read once.  A cluster of 1 to 8 CTAs shares it, each a part of its 16-byte granules in shared memory; a
// thread works on the granules that it has copied.  While the part is on its way the threads work out the
// teacher's probabilities, an entry each; then they take the entries' elements out of the part (-inf takes their place: what is
// left is the rest of the vocabulary, whose sum must not come from a difference).  Every warp sums the powers of its
// granules relative to a logit of its own, the last warp joins the sums, exchanges them with the other CTAs and has
// the gradient's factors, with which the gradient is formed from shared memory and written, the entries' elements last; meanwhile
// it works out the loss.
//
// Of the loss, what an entry adds is held in two fp32 pieces, what joins them in 64 bits: relative errors of 1e-7 to 6e-7 where the rest is
// a class (T up to 4; fp32 forms of the same terms have 2e-7 to 6e-4), 2e-8 to 6e-8 renormalised (a rounding to fp32 is up to 6e-8).
//
// Bytes: the logits once, the gradient once.  Operations: two powers an element with a gradient (one of the sum, one of the
// gradient: keeping the first would take the room of a second part), so 16 elements a cycle and SM of the special function unit, about
// 0.7 of the copy's time in 16 bits; the rest are conversions and fp32 pairs.  Measured (device time; floor at the copy rate, 6561 GB/s):
//   8192 x 50257 bf16, 64 entries, gradient           329 us (5.0 TB/s; floor 252)
//   2048 x 30522 bf16, a quarter masked               49.2 us (floor 33.4)
//   2048 x 50257 fp32                                 163 us (floor 126)
//   700 x 33278 fp32, loss alone                      33.4 us (2.8 TB/s; floor 14.2: a part is parked and read again, though nothing is
//                                                     written back, and 3.5 rounds of CTAs each copy, sum and join in turn)
//   65536 x 1000 bf16                                 192 us (floor 41: some 1600 instructions a row that do not depend on its width)
//   16384 x 4000 bf16                                 92 us (floor 40: likewise)
// Special function unit 56 %, issue slots 55 %, waits at the row's barriers: a CTA copies, sums and writes in turn, and the four
// of an SM overlap one another's phases.  What was tried against it and was slower: one CTA an SM with three parts in a ring and the powers
// kept (550 to 750 us), a share of the powers by a polynomial (339 to 416).  Larger and smaller parts gave nothing.
#include <cooperative_groups.h>

#include "deft_dense.cuh"
#include "deft_pairs.cuh"

namespace deft {
namespace {

constexpr int kMostCluster = 8;
constexpr int kEachThread = 128;          // elements a thread works on at most, where there are threads enough (64, 128, 256: 700 x 33278 fp32 34.4, 32.9, 35.9 us, 8192 x 50257 bf16 837, 331, 358)
constexpr int kMostThreads = 512;         // that work on the row
constexpr int kPartBytes = 52224;         // of a row, per CTA: four CTAs per SM

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint64_t exp2_pair(uint64_t x) {
    const float2 v = unpair(x);
    return pair(exp2_fast(v.x), exp2_fast(v.y));
}

// A sum of fp32 numbers and what its roundings have left out: the loss is what remains of terms that nearly cancel.
struct Exact {
    float hi, lo;
    __device__ __forceinline__ void add(float x) {
        const float s = __fadd_rn(hi, x), b = __fsub_rn(s, hi);
        lo += __fadd_rn(__fsub_rn(hi, __fsub_rn(s, b)), __fsub_rn(x, b));
        hi = s;
    }
    __device__ __forceinline__ void add(Exact x) {
        add(x.hi);
        lo += x.lo;
    }
    __device__ __forceinline__ void add_product(float a, float b) {
        const float p = __fmul_rn(a, b);
        add(p);
        lo += __fmaf_rn(a, b, -p);
    }
};
// d (hi + lo) - norm; an infinite d stays what it is (the lower piece may be 0).
__device__ __forceinline__ Exact log_prob(float d, float hi, float lo, Exact norm) {
    Exact y{-norm.hi, -norm.lo};
    if (!isfinite(d)) return Exact{d, 0.0f};
    y.add_product(d, hi);
    y.lo += d * lo;
    return y;
}
// e to the power of both pieces: a piece that the argument's rounding would lose is a relative error of the probability.
__device__ __forceinline__ float exp_of(Exact x) {
    const float y = expf(x.hi);
    return x.lo != 0.0f ? __fmaf_rn(y, x.lo, y) : y;
}
// (where it is infinite, what its roundings have left out is no number)
__device__ __forceinline__ double value_of(Exact x) { return isfinite(x.hi) ? (double)x.hi + (double)x.lo : (double)x.hi; }
__device__ __forceinline__ Exact log_of(Exact x) {
    const double y = log(value_of(x));
    const float hi = (float)y;
    return Exact{hi, isfinite(hi) ? (float)(y - (double)hi) : 0.0f};
}
__device__ __forceinline__ Exact shuffled(Exact x, int o) { return Exact{__shfl_xor_sync(0xffffffffu, x.hi, o), __shfl_xor_sync(0xffffffffu, x.lo, o)}; }

// 2^(d c1) for d <= 0 to a unit in the last place, the argument's rounding made good: a polynomial of degree six on [-1/2, 1/2], fitted for the least relative error (2e-9).
__device__ __forceinline__ float power_of(float d, float c1) {
    const float p = d * c1;
    if (!(p > -126.0f)) return p <= -126.0f ? 0.0f : p;      // (no number stays none)
    const float n = rintf(p), f = (p - n) + __fmaf_rn(d, c1, -p);
    float y = 1.534580214352e-4f;
    y = __fmaf_rn(y, f, 1.339993113957e-3f);
    y = __fmaf_rn(y, f, 9.618488993764e-3f);
    y = __fmaf_rn(y, f, 5.550328777213e-2f);
    y = __fmaf_rn(y, f, 0.240226468903f);
    y = __fmaf_rn(y, f, 0.693147205737f);
    y = __fmaf_rn(y, f, 1.0f);
    return __int_as_float(__float_as_int(y) + ((int)n << 23));
}

// What a warp has summed: of the rest and of the entries the powers; over the entries q (log q - (z - near) / T), and q.
struct Sums {
    float rest_near, rest, entries_near;
    Exact entries, cross, q;             // (an error of the entries' share is one of the loss, one of the rest's cancels where q0 is near p0)
};
// What the gradient needs of it, for a CTA.
struct Brief {
    float rest_near, rest, entries_near, entries, q;
};
// What the gradient of a row is formed with: an element's is K 2^((z - rest) c1), an entry's own A 2^((z - all) c1) - q f.
struct Factors {
    float all, rest, A, K;
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
template <int kLanes>
__device__ __forceinline__ double joined(double x) {
#pragma unroll
    for (int o = kLanes / 2; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
template <int kLanes>
__device__ __forceinline__ Exact joined(Exact x) {
#pragma unroll
    for (int o = kLanes / 2; o; o >>= 1) x.add(shuffled(x, o));
    return x;
}
// The sum of what the lanes hold (over groups of kLanes), relative to the largest logit among them, which `near` becomes (0: none).
template <int kLanes>
__device__ __forceinline__ float joined(float& near, float sum, float c1) {
    float most = sum == 0.0f ? -INFINITY : near;
#pragma unroll
    for (int o = kLanes / 2; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
    if (most == -INFINITY) most = 0.0f;
    sum = sum == 0.0f ? 0.0f : sum * exp2_fast((near - most) * c1);
#pragma unroll
    for (int o = kLanes / 2; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    near = most;
    return sum;
}
template <int kLanes>
__device__ __forceinline__ Brief joined(Brief s, float c1) {
    s.rest = joined<kLanes>(s.rest_near, s.rest, c1);
    s.entries = joined<kLanes>(s.entries_near, s.entries, c1);
#pragma unroll
    for (int o = kLanes / 2; o; o >>= 1) s.q += __shfl_xor_sync(0xffffffffu, s.q, o);
    return s;
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

// An entry as it lies in memory: nothing waits for its loads before it is looked at.
struct RawEntry {
    uint32_t id, id_high, t;
};
__device__ __forceinline__ RawEntry entry_at(const DistillArgs& a, int64_t row, int j) {
    RawEntry e{0, 0, 0};
    const int64_t at = row * a.ld_teacher + j, id = row * a.ld_ids + j;
    if (a.id_bytes == 8) {
        const uint2 both = static_cast<const uint2*>(a.ids)[id];
        e.id = both.x;
        e.id_high = both.y;
    } else {
        e.id = static_cast<const uint32_t*>(a.ids)[id];
    }
    if (a.teacher_type == DEFT_F32) e.t = static_cast<const uint32_t*>(a.teacher)[at];
    else e.t = static_cast<const uint16_t*>(a.teacher)[at];
    return e;
}
// The entry's column, or -1.
__device__ __forceinline__ int column_of(const DistillArgs& a, const RawEntry& e) { return e.id < (uint32_t)a.vocab && e.id_high == 0 ? (int)e.id : -1; }
__device__ __forceinline__ float value_of(const DistillArgs& a, uint32_t t) {
    if (a.teacher_type == DEFT_F32) return __uint_as_float(t);
    return a.teacher_type == DEFT_BF16 ? to_f32(__ushort_as_bfloat16((unsigned short)t)) : to_f32(__ushort_as_half((unsigned short)t));
}

// A row's entries in shared memory.
struct Entries {
    int* col;                              // column; -1: none; -2: another CTA's; -3 - column: not the first of its column
    float *log_q, *log_q_lo, *prob, *own;  // log q in two pieces; own: the student's logit
    __device__ __forceinline__ Entries(char* at, int top) : col(reinterpret_cast<int*>(at)) {
        log_q = reinterpret_cast<float*>(col + top);
        log_q_lo = log_q + top;
        prob = log_q_lo + top;
        own = prob + top;
    }
};
constexpr size_t kEntryBytes = 20;

// What stands for an element without a share.
template <typename T> __device__ __forceinline__ T lowest();
template <> __device__ __forceinline__ float lowest<float>() { return __int_as_float(0xff800000); }
template <> __device__ __forceinline__ __nv_bfloat16 lowest<__nv_bfloat16>() { return __ushort_as_bfloat16(0xff80); }
template <> __device__ __forceinline__ __half lowest<__half>() { return __ushort_as_half(0xfc00); }

// Takes an element out of a part and returns what was there: -inf for all but the first that asks.
__device__ __forceinline__ float take(float* p) { return __uint_as_float(atomicExch(reinterpret_cast<unsigned*>(p), 0xff800000u)); }
template <typename T>
__device__ __forceinline__ float take(T* p) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    unsigned* word = reinterpret_cast<unsigned*>(at & ~(uintptr_t)3);
    const int up = (at & 2) ? 16 : 0;
    const T low = lowest<T>();
    const unsigned mark = *reinterpret_cast<const unsigned short*>(&low);
    unsigned was = *reinterpret_cast<volatile unsigned*>(word);
    while (true) {
        const unsigned seen = atomicCAS(word, was, (was & ~(0xffffu << up)) | (mark << up));
        if (seen == was) break;
        was = seen;
    }
    const unsigned short old = (unsigned short)(was >> up);
    return to_f32(*reinterpret_cast<const T*>(&old));
}

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
// The sum of the powers of this thread's granules.
template <typename T, bool kCareful>
__device__ __forceinline__ float sum_powers(const Granule<T>* cells, int n, int threads, float from1, float c1) {
    const uint64_t c = pair(c1, c1), from = pair(-from1, -from1);
    uint64_t s[2] = {0, 0};
    for (int i = threadIdx.x; i < n; i += threads) {
        const Granule<T> g = cells[i];
#pragma unroll
        for (int p = 0; p < Granule<T>::kPairs; ++p) s[p & 1] = add2(s[p & 1], powers<T, kCareful>(g.get(p), c, from));
    }
    const float2 v = unpair(add2(s[0], s[1]));
    return v.x + v.y;
}
// The first elements of a granule (col: the first one's column) that are the row's.
template <typename T>
__device__ __forceinline__ void put_some(const Granule<T>& o, int col, int vocab, T* g) {
    for (int e = 0; e < Granule<T>::kPer; ++e)
        if (col + e >= 0 && col + e < vocab) g[col + e] = reinterpret_cast<const T*>(&o.raw)[e];
}
// The gradient of this thread's granules, the entries' elements zero.  whole: the granules of the gradient lie like the logits';
// inner: granules lo .. hi are the row's in full.
template <typename T, bool kCareful>
__device__ __forceinline__ void write_grad(const Granule<T>* cells, int n, int base, int lo, int hi, int threads, int vocab, T* g, float from1, float c1, float k1) {
    constexpr int kPer = Granule<T>::kPer;
    const uint64_t c = pair(c1, c1), from = pair(-from1, -from1), k = pair(k1, k1);
    for (int i = threadIdx.x; i < n; i += threads) {
        const Granule<T> in = cells[i];
        Granule<T> o;
#pragma unroll
        for (int p = 0; p < Granule<T>::kPairs; ++p) o.set(p, mul2(powers<T, kCareful>(in.get(p), c, from), k));
        if (i >= lo && i < hi) *reinterpret_cast<uint4*>(g + base + i * kPer) = o.raw;
        else put_some(o, base + i * kPer, vocab, g);
    }
}

// Barriers of a CTA: between the warps that work on the row and the last one, and among the former.  (An SM has barriers for as many
// CTAs only as their numbers allow: with three instead of five, small rows run 16 side by side, not ten.)
enum { kSummed = 1, kFactors, kRow };
template <int kId>
__device__ __forceinline__ void bar_sync(int threads) {
    __syncwarp();
    asm volatile("bar.sync %0, %1;" ::"n"(kId), "r"(threads) : "memory");
}
template <int kId>
__device__ __forceinline__ void bar_arrive(int threads) {
    __syncwarp();
    asm volatile("bar.arrive %0, %1;" ::"n"(kId), "r"(threads) : "memory");
}
template <int kMost>
__device__ __forceinline__ void bar_row(int threads) {
    if (kMost == 32) __syncwarp();
    else bar_sync<kRow>(threads);
}
__device__ __forceinline__ void cluster_arrive() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_arrive_release() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// How a call is split: CTAs of a cluster, granules of a part; threads that work on the row.
struct DistillShape {
    int ctas, granules, threads;
    size_t smem;
};

// kMost: threads that work on the row, at most; four CTAs of 256 fit an SM.
template <typename T, int kMost>
__global__ void __launch_bounds__(kMost + 32, kMost == 32 ? 16 : (kMost == 256 ? 4 : 1)) k_distill(const __grid_constant__ DistillArgs a, const __grid_constant__ DistillShape shape) {
    constexpr int kPer = Granule<T>::kPer;
    extern __shared__ __align__(16) char smem[];
    Granule<T>* const cells = reinterpret_cast<Granule<T>*>(smem);
    __shared__ Sums warp_sums[kMost / 32];
    __shared__ Brief briefs[kMostCluster];
    __shared__ Factors factors;
    __shared__ volatile int twice;         // the last row in which an entry found nothing in its place: another one's column, or -inf (several threads may say so)
    const int ctas = shape.ctas, threads = shape.threads, warps = threads >> 5, all_threads = threads + 32;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    int rank = 0;
    int64_t row = blockIdx.x;
    if (ctas > 1) {
        uint32_t cluster;
        asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
        asm volatile("mov.u32 %0, %%clusterid.x;" : "=r"(cluster));
        row = cluster;
        cluster_arrive();                  // (waited for before others' shared memory is written)
    }
    T* const g = a.grad ? static_cast<T*>(a.grad) + row * a.ld_grad : nullptr;
    const float weight = a.weight ? a.weight[row] : 1.0f;

    if (warp == warps) {                   // ---- the last warp ----
        if (weight == 0.0f) {
            if (a.loss && rank == 0 && lane == 0) a.loss[row] = 0.0f;
            if (ctas > 1) cluster_wait();
            return;
        }
        bar_sync<kSummed>(all_threads);
        const int entry_warps = min(warps, (a.top + 31) >> 5);
        // in short what the gradient waits for
        Sums* const others = reinterpret_cast<Sums*>(smem + (size_t)shape.granules * 16 + (size_t)a.top * kEntryBytes);   // [ctas][entry_warps], in the first CTA
        auto brief = [&](int w) { return Brief{warp_sums[w].rest_near, warp_sums[w].rest, warp_sums[w].entries_near, warp_sums[w].entries.hi, warp_sums[w].q.hi}; };
        Brief s{};
        if (warps > 8) {
            if (lane < warps) s = brief(lane);
            s = joined<32>(s, a.c1);
        } else if (warps > 1) {            // eight lanes, four times over
            if ((lane & 7) < warps) s = brief(lane & 7);
            s = joined<8>(s, a.c1);
        } else {
            s = brief(0);
        }
        if (ctas > 1) {
            cluster_wait();                // all CTAs run: their shared memory may be written
            if (lane < ctas) *cooperative_groups::this_cluster().map_shared_rank(&briefs[rank], lane) = s;
            if (a.loss && rank != 0 && lane < entry_warps) *cooperative_groups::this_cluster().map_shared_rank(others + rank * entry_warps + lane, 0) = warp_sums[lane];
            cluster_arrive_release();
            cluster_wait();
            s = Brief{};
            if ((lane & 7) < ctas) s = briefs[lane & 7];
            s = joined<8>(s, a.c1);
        }
        const float all = s.rest == 0.0f ? s.entries_near : (s.entries == 0.0f ? s.rest_near : fmaxf(s.rest_near, s.entries_near));
        if (g) {
            // (one of the two lies at `all`)
            const float step = power_of(fminf(s.rest_near, s.entries_near) - all, a.c1);
            const float rest = s.rest == 0.0f ? 0.0f : (s.rest_near == all ? s.rest : s.rest * step);
            const float entries = s.entries == 0.0f ? 0.0f : (s.entries_near == all ? s.entries : s.entries * step), total = rest + entries;
            // the teacher's probability outside its entries; none where there is no other logit
            const float left = a.teacher_lse && !(s.rest == 0.0f) ? fmaxf(0.0f, 1.0f - s.q) : 0.0f, f = weight * a.grad_factor;
            // p (q + left) - left p / p0 of the rest, p0 = rest / total: with the common left rest taken out, as 1 - left / p0 would lose what
            // lies between the two
            const float p = left * entries, d = __fmaf_rn(s.q, rest, -p) - __fmaf_rn(left, entries, -p);
            if (lane == 0) factors = Factors{all, s.rest_near, (s.q + left) / total * f, s.rest == 0.0f ? 0.0f : d / (total * s.rest) * f};
            bar_arrive<kFactors>(all_threads);
        }
        if (a.loss && rank == 0) {         // the loss, from all warps' sums: what remains of terms that nearly cancel, in 64 bits
            const double c1 = a.c1, by = (double)a.by + (double)a.by_lo;
            double cross = 0.0, q = 0.0, entries = 0.0;
            const int all_entry_warps = ctas * entry_warps;
            for (int i = lane; i < all_entry_warps; i += 32) {
                const Sums w = i < entry_warps ? warp_sums[i] : others[i];
                const double near = (double)w.entries_near - (double)s.entries_near, of_warp = value_of(w.q);
                cross += value_of(w.cross);
                if (near != 0.0) cross -= of_warp * (near * by);
                q += of_warp;
                if (w.entries.hi != 0.0f) entries += near != 0.0 ? value_of(w.entries) * exp2(near * c1) : value_of(w.entries);
            }
            if (all_entry_warps > 8) {
                cross = joined<32>(cross);
                q = joined<32>(q);
                entries = joined<32>(entries);
            } else if (all_entry_warps > 1) {
                cross = joined<8>(cross);
                q = joined<8>(q);
                entries = joined<8>(entries);
            }
            if (lane == 0) {
                // of the rest and of the entries one lies at `all`
                const double to_rest = (double)all - (double)s.rest_near, to_entries = (double)all - (double)s.entries_near;
                double total = 0.0;
                if (s.rest != 0.0f) total += to_rest != 0.0 ? s.rest * exp2(-to_rest * c1) : (double)s.rest;
                if (entries != 0.0) total += to_entries != 0.0 ? entries * exp2(-to_entries * c1) : entries;
                const double log_total = log(total), left = a.teacher_lse && !(s.rest == 0.0f) ? 1.0 - q : 0.0;
                double loss = cross;
                if (q != 0.0) loss += q * (to_entries * by + log_total);
                if (left > 0.0) loss += left * (log(left) - log((double)s.rest) + to_rest * by + log_total);
                a.loss[row] = (float)(loss * weight * a.loss_factor);
            }
        }
        return;
    }

    // this CTA's granules of the row, the first of which may begin before it
    const T* const z = static_cast<const T*>(a.logits) + row * a.ld;
    const int shift = (int)(reinterpret_cast<uintptr_t>(z) & 15u) / (int)sizeof(T);
    const int first = rank * shape.granules, base = first * kPer - shift;        // column of the first element
    const int n = max(0, min(shape.granules, (a.vocab + shift + kPer - 1) / kPer - first));
    const bool whole = ((reinterpret_cast<uintptr_t>(g) ^ reinterpret_cast<uintptr_t>(z)) & 15u) == 0;
    const int lo = whole ? (base < 0 ? 1 : 0) : n, hi = whole ? min(n, (a.vocab - base) / kPer) : n;   // granules written in one piece
    if (weight == 0.0f) {                  // nothing is read of a row that does not count
        Granule<T> zero;
        zero.raw = make_uint4(0, 0, 0, 0);
        if (g)
            for (int i = tid; i < n; i += threads) {
                if (i >= lo && i < hi) *reinterpret_cast<uint4*>(g + base + i * kPer) = zero.raw;
                else put_some(zero, base + i * kPer, a.vocab, g);
            }
        if (ctas > 1) cluster_wait();
        return;
    }
    // an entry for each thread: its load goes ahead of the copies
    const Entries entry(smem + (size_t)shape.granules * 16, a.top);
    const bool has_entries = warp * 32 < a.top;
    if (tid == 0) twice = -1;
    RawEntry raw{0, 0, 0};
    Exact norm{0.0f, 0.0f};
    if (tid < a.top) raw = entry_at(a, row, tid);
    if (has_entries && a.teacher_lse) norm.hi = a.teacher_lse[row];
    {
        const T* from = z + base + tid * kPer;
        uint32_t to = (uint32_t)__cvta_generic_to_shared(smem) + (uint32_t)tid * 16u;
        for (int i = tid; i < n; i += threads, from += threads * kPer, to += (uint32_t)threads * 16u)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    // the teacher, while the copies are under way: log q = (t - near) / T - norm
    Exact q_sum{};
    if (has_entries) {
        float near = 0.0f;
        if (!a.teacher_lse) {              // every warp goes through all entries
            float most = -INFINITY;
            for (int j = lane; j < a.top; j += 32) {
                const RawEntry e = entry_at(a, row, j);
                if (column_of(a, e) >= 0) most = fmaxf(most, value_of(a, e.t));
            }
            most = warp_max(most);
            if (most != -INFINITY) {
                near = most;
                Exact sum{0.0f, 0.0f};     // (what it is off by is an error of the loss)
                for (int j = lane; j < a.top; j += 32) {
                    const RawEntry e = entry_at(a, row, j);
                    const float d = value_of(a, e.t) - near;
                    if (column_of(a, e) >= 0) sum.add(exp_of(log_prob(d, a.it_hi, a.it_lo, Exact{0.0f, 0.0f})));
                }
                norm = log_of(joined<32>(sum));
            }
        }
        for (int j = tid; j < a.top; j += threads) {
            if (j >= threads) raw = entry_at(a, row, j);
            const int col = column_of(a, raw);
            const bool valid = col >= 0;
            const Exact log_q = log_prob(value_of(a, raw.t) - near, a.it_hi, a.it_lo, norm);
            const float q = valid ? exp_of(log_q) : 0.0f;
            const bool here = valid && col >= base && col < base + n * kPer;
            entry.col[j] = valid && !here ? -2 : col;
            entry.log_q[j] = log_q.hi;
            entry.log_q_lo[j] = log_q.lo;
            entry.prob[j] = q;
            if (here) q_sum.add(q);
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    T* const e = reinterpret_cast<T*>(smem) - base;
    // what the first and last granule hold beside the row, marked by whoever has copied them: behind the barrier an entry's element may
    // be taken out of the same word
    if (tid == 0)
        for (int c = base; c < 0; ++c) e[c] = lowest<T>();
    if (n > 0 && tid == ((n - 1) & (threads - 1)))     // (a power of two)
        for (int c = max(a.vocab, base); c < base + n * kPer; ++c) e[c] = lowest<T>();
    bar_row<kMost>(threads);
    Sums s{};
    if (has_entries) {
        for (int j = tid; j < a.top; j += threads) {
            const int col = entry.col[j];
            if (col < 0) continue;
            float own = take(e + col);
            if (own == -INFINITY) {        // another entry of this column was first, or the logit is -inf
                own = to_f32(z[col]);
                twice = (int)row;
            }
            entry.own[j] = own;
        }
    }
    bar_row<kMost>(threads);
    if (has_entries) {
        if (twice == (int)row) {           // of a column's entries the first one counts: who was first above is a matter of chance
            for (int j = tid; j < a.top; j += threads) {
                const int col = entry.col[j];
                bool earlier = false;
                for (int m = 0; m < j && col >= 0; ++m) {
                    const int other = *const_cast<volatile int*>(entry.col + m);      // (may have become -3 - column meanwhile)
                    earlier |= other == col || other == -3 - col;
                }
                if (earlier) *const_cast<volatile int*>(entry.col + j) = -3 - col;
            }
        }
        float most = -INFINITY;
        for (int j = tid; j < a.top; j += threads)
            if (entry.col[j] >= 0) most = fmaxf(most, entry.own[j]);
        most = warp_max(most);
        s.entries_near = most == -INFINITY ? 0.0f : most;
        for (int j = tid; j < a.top; j += threads) {
            const int col = entry.col[j];
            if (col == -1 || col == -2) continue;
            const float own = entry.own[j], q = entry.prob[j], d = own - s.entries_near;
            if (q != 0.0f) {
                Exact t{entry.log_q[j], entry.log_q_lo[j]};
                if (isfinite(d)) {
                    t.add_product(-d, a.by);
                    t.lo -= d * a.by_lo;
                    s.cross.add_product(q, t.hi);
                    s.cross.lo += q * t.lo;
                } else {
                    s.cross.add(-d);       // (an entry without any share: an infinite loss; no number stays none)
                }
            }
            if (col >= 0) s.entries.add(power_of(d, a.c1));
        }
    }
    // what the powers are relative to: the largest of a granule of every lane, which is seldom far from the largest of all
    float most = warp_max(tid < n ? most_of<T>(cells[tid]) : -INFINITY);
    bool careful = false;
    s.rest_near = most == -INFINITY ? 0.0f : most;
    float from = s.rest_near * a.c1;
    // (from is rounded: what the powers are relative to instead of near)
    float off = exp2_fast(__fmaf_rn(-s.rest_near, a.c1, from));
    float rest = warp_sum(sum_powers<T, false>(cells, n, threads, from, a.c1));
    // the sample is too far off (or something is no number).  Powers and factors below 2^-126 are 0: within these bounds
    // no probability above 2^-96 is lost
    if (!(rest > 9.5367431640625e-07f && rest < 1073741824.0f)) {                // 2^-20, 2^30
        most = -INFINITY;
        for (int c = tid; c < n; c += threads) most = fmaxf(most, most_of<T>(cells[c]));
        most = warp_max(most);
        careful = true;
        s.rest_near = from = most == -INFINITY ? 0.0f : most;
        off = 1.0f;
        rest = warp_sum(sum_powers<T, true>(cells, n, threads, from, a.c1));
    }
    s.rest = rest * off;
    if (has_entries) {
        if (a.top <= 8) {                  // (lanes without an entry have nothing to join)
            s.entries = joined<8>(s.entries);
            s.cross = joined<8>(s.cross);
            s.q = joined<8>(q_sum);
        } else {
            s.entries = joined<32>(s.entries);
            s.cross = joined<32>(s.cross);
            s.q = joined<32>(q_sum);
        }
    }
    if (lane == 0) warp_sums[warp] = s;
    bar_arrive<kSummed>(all_threads);
    if (ctas > 1) {
        cluster_wait();
        cluster_arrive();
    }
    if (g) {
        bar_sync<kFactors>(all_threads);
        const Factors f = factors;
        // (nothing but -inf: the share is 0, and NaN where the whole row has no other)
        const float k = rest == 0.0f ? 0.0f * f.A : f.K * exp2_fast((s.rest_near - f.rest) * a.c1) * off;
        if (careful) write_grad<T, true>(cells, n, base, lo, hi, threads, a.vocab, g, from, a.c1, k);
        else write_grad<T, false>(cells, n, base, lo, hi, threads, a.vocab, g, from, a.c1, k);
        bar_row<kMost>(threads);
        // the entries' own elements: the probabilities of a column's entries added in their order
        for (int j = tid; j < a.top; j += threads) {
            const int c = entry.col[j];
            if (c < 0) continue;
            float q = entry.prob[j];
            if (twice == (int)row) {
                q = 0.0f;
                for (int m = 0; m < a.top; ++m)
                    if (entry.col[m] == c || entry.col[m] == -3 - c) q += entry.prob[m];
            }
            g[c] = from_f32<T>(power_of(entry.own[j] - f.all, a.c1) * f.A - q * (weight * a.grad_factor));
        }
    }
    if (ctas > 1) cluster_wait();
}

}  // namespace

deft_status launch_distill(const DistillArgs& a, int type, cudaStream_t stream) {
    const int64_t elem = (int64_t)type_bytes(type), bytes = a.vocab * elem + 16;
    int64_t ctas = (bytes + kPartBytes - 1) / kPartBytes;
    while (ctas < kMostCluster && a.rows * ctas < 2 * 148 && bytes / ctas > 8 * 1024) ctas *= 2;      // few rows
    if (ctas > kMostCluster) ctas = kMostCluster;
    if (a.rows * ctas > 0x7fffffffLL) return DEFT_ERR_TOO_LARGE;
    DistillShape s{};
    s.ctas = (int)ctas;
    s.granules = (int)(((bytes + 15) / 16 + ctas - 1) / ctas);
    s.threads = 32;
    while (s.threads < kMostThreads && s.granules * (16 / elem) > s.threads * kEachThread) s.threads *= 2;
    const size_t entry_warps = (size_t)((a.top + 31) / 32 < s.threads / 32 ? (a.top + 31) / 32 : s.threads / 32);
    s.smem = (size_t)s.granules * 16 + (size_t)a.top * kEntryBytes + (s.ctas > 1 ? s.ctas * entry_warps * sizeof(Sums) : 0);
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)s.ctas;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(a.rows * ctas));
    cfg.blockDim = dim3((unsigned)s.threads + 32);
    cfg.dynamicSmemBytes = s.smem;
    cfg.stream = stream;
    cfg.attrs = &attr;
    cfg.numAttrs = s.ctas > 1 ? 1 : 0;
    return with_type(type, [&](auto t) -> deft_status {
        using T = decltype(t);
        auto kernel = s.threads > 256 ? k_distill<T, 512> : (s.threads > 32 ? k_distill<T, 256> : k_distill<T, 32>);
        if (s.smem > 40 * 1024) DEFT_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMostSmem));
        DEFT_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, a, s));
        return DEFT_OK;
    });
}

}  // namespace deft
