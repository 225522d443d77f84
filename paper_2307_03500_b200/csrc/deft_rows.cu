// Embedding lookup and dropout: rows of a matrix taken in groups of eight columns.
#include "deft_rows.cuh"

namespace deft {
namespace {

constexpr int kRowThreads = 256;

template <typename TW, typename TO, typename Id, int kAlign>
__global__ void __launch_bounds__(kRowThreads) k_embed(const EmbedArgs a, uint32_t groups, int64_t total) {
    const uint64_t offset = drop_offset(a.drop);
    for (int64_t g = (int64_t)blockIdx.x * kRowThreads + threadIdx.x; g < total; g += (int64_t)gridDim.x * kRowThreads) {
        const int64_t t = g / groups;
        const uint32_t group = (uint32_t)(g - t * groups);
        const int64_t col = (int64_t)group * kGroup;
        const int count = a.width - col < kGroup ? (int)(a.width - col) : kGroup;
        const int64_t id = (int64_t)static_cast<const Id*>(a.ids)[t];
        float v[kGroup] = {};
        if (id >= 0 && id < a.rows) load8<TW, kAlign>(static_cast<const TW*>(a.table) + id * a.ld_table + col, count, v);
#pragma unroll
        for (int i = 0; i < kGroup; ++i) v[i] = __fmul_rn(v[i], a.scale);
        if (a.pos) {
            float q[kGroup];
            load8<TW, kAlign>(static_cast<const TW*>(a.pos) + (t % a.pos_rows) * a.ld_pos + col, count, q);
#pragma unroll
            for (int i = 0; i < kGroup; ++i) v[i] = __fadd_rn(v[i], q[i]);
        }
        if (a.drop.threshold) drop8<true>(v, a.drop, offset, (uint32_t)t, group);
        store8<TO, kAlign>(static_cast<TO*>(a.out) + t * a.ld_out + col, count, v);
    }
}

template <typename TX, typename TY, int kAlign>
__global__ void __launch_bounds__(kRowThreads) k_dropout(const DropoutArgs a, uint32_t groups, int64_t total) {
    const uint64_t offset = drop_offset(a.drop);
    for (int64_t g = (int64_t)blockIdx.x * kRowThreads + threadIdx.x; g < total; g += (int64_t)gridDim.x * kRowThreads) {
        const int64_t r = g / groups;
        const uint32_t group = (uint32_t)(g - r * groups);
        const int64_t col = (int64_t)group * kGroup;
        const int count = a.cols - col < kGroup ? (int)(a.cols - col) : kGroup;
        float v[kGroup];
        load8<TX, kAlign>(static_cast<const TX*>(a.x) + r * a.ld_x + col, count, v);
        if (a.drop.threshold) drop8<true>(v, a.drop, offset, (uint32_t)r, group);
        if (a.add) {
            float q[kGroup];
            load8<TY, kAlign>(static_cast<const TY*>(a.add) + r * a.ld_add + col, count, q);
#pragma unroll
            for (int i = 0; i < kGroup; ++i) v[i] = __fadd_rn(v[i], q[i]);
        }
        store8<TY, kAlign>(static_cast<TY*>(a.y) + r * a.ld_y + col, count, v);
    }
}

inline unsigned grid_of(int64_t total) {
    const int64_t want = (total + kRowThreads - 1) / kRowThreads;
    return (unsigned)(want < 0x7fffffff ? want : 0x7fffffff);
}

}  // namespace

deft_status launch_embed(const EmbedArgs& a, int table_type, int out_type, int id_bytes, cudaStream_t stream) {
    const uint32_t groups = (uint32_t)((a.width + kGroup - 1) / kGroup);
    const int64_t total = a.n * groups;
    int align = row_align(a.table, a.ld_table, type_bytes(table_type));
    const int ao = row_align(a.out, a.ld_out, type_bytes(out_type));
    if (ao < align) align = ao;
    if (a.pos) {
        const int ap = row_align(a.pos, a.ld_pos, type_bytes(table_type));
        if (ap < align) align = ap;
    }
    return with_type(table_type, [&](auto w) {
        return with_type(out_type, [&](auto o) {
            return with_align(align, [&](auto al) -> deft_status {
                using TW = decltype(w);
                using TO = decltype(o);
                constexpr int kAlign = decltype(al)::value;
                if (id_bytes == 8) k_embed<TW, TO, int64_t, kAlign><<<grid_of(total), kRowThreads, 0, stream>>>(a, groups, total);
                else k_embed<TW, TO, int32_t, kAlign><<<grid_of(total), kRowThreads, 0, stream>>>(a, groups, total);
                DEFT_CUDA_TRY(cudaGetLastError());
                return DEFT_OK;
            });
        });
    });
}

deft_status launch_dropout(const DropoutArgs& a, int x_type, int y_type, cudaStream_t stream) {
    const uint32_t groups = (uint32_t)((a.cols + kGroup - 1) / kGroup);
    const int64_t total = a.rows * groups;
    int align = row_align(a.x, a.ld_x, type_bytes(x_type));
    const int ay = row_align(a.y, a.ld_y, type_bytes(y_type));
    if (ay < align) align = ay;
    if (a.add) {
        const int aa = row_align(a.add, a.ld_add, type_bytes(y_type));
        if (aa < align) align = aa;
    }
    return with_type(x_type, [&](auto x) {
        return with_type(y_type, [&](auto y) {
            return with_align(align, [&](auto al) -> deft_status {
                k_dropout<decltype(x), decltype(y), decltype(al)::value><<<grid_of(total), kRowThreads, 0, stream>>>(a, groups, total);
                DEFT_CUDA_TRY(cudaGetLastError());
                return DEFT_OK;
            });
        });
    });
}

}  // namespace deft
