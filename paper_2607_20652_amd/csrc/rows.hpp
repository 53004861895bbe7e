// Embedding and RMS norm: arguments of their launches, and rows in chunks.
#pragma once

#include "device_common.hpp"

namespace dpb {

struct NormArgs {
    const void *x, *residual, *weight;
    int64_t x_stride, residual_stride;   // bytes
    int64_t rows;
    int dim;
    float eps;
    void *out, *total;                   // contiguous
    float* rstd;
    int weight_bf16;
};
struct NormBwdArgs {
    const void *grad, *grad_total, *total, *weight;
    int64_t grad_stride, grad_total_stride, total_stride;   // bytes
    const float* rstd;
    int64_t rows;
    int dim;
    void *dx, *dweight;                  // either may be null
    float* part;
    int weight_bf16;
};
size_t norm_bwd_ws_bytes(int64_t rows, int dim);
hipError_t launch_rms_norm(const NormArgs& a, bool bf16, hipStream_t stream);
hipError_t launch_rms_norm_bwd(const NormBwdArgs& a, bool bf16, hipStream_t stream);

struct EmbedArgs {
    const void* table;                   // forward: [vocab, dim];  backward: grad_out [count, dim]
    int64_t stride;                      // bytes
    int64_t vocab, count;
    int dim;
    const void* tokens;
    int wide;                            // tokens are int64
    float scale;
    void* out;                           // contiguous
    char* ws;
};
size_t embed_bwd_ws_bytes(int64_t vocab, int dim, int64_t count);
hipError_t launch_embedding(const EmbedArgs& a, bool bf16, hipStream_t stream);
hipError_t launch_embedding_bwd(const EmbedArgs& a, bool bf16, hipStream_t stream);

// E consecutive elements of a row: 16 bytes, or one element where rows do not start on 16 bytes
// or end within them.
template <typename T, int E>
__device__ __forceinline__ void load_chunk(const void* row, int64_t e, float (&v)[E])
{
    if constexpr (E == 1) {
        v[0] = load_act<sizeof(T) == 2>(row, e);
    } else if constexpr (sizeof(T) == 2) {
        const u32x4 w = *(const u32x4*)((const char*)row + e * 2);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    } else {
        const f32x4 w = *(const f32x4*)((const char*)row + e * 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = w[i];
    }
}

template <typename T, int E>
__device__ __forceinline__ void store_chunk(void* row, int64_t e, const float (&v)[E])
{
    if constexpr (E == 1) {
        store_act<sizeof(T) == 2>(row, e, v[0]);
    } else if constexpr (sizeof(T) == 2) {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
        *(u32x4*)((char*)row + e * 2) = w;
    } else {
        *(f32x4*)((char*)row + e * 4) = (f32x4){v[0], v[1], v[2], v[3]};
    }
}

}  // namespace dpb
