// Softmax cross entropy over a vocabulary: arguments of its launches.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

namespace dpb {

struct LossArgs {
    const void *hidden, *weight;          // [rows, dim], [vocab, dim]
    int64_t hidden_stride, weight_stride; // bytes, multiples of 16
    const void* targets;                  // int32 or int64 [rows]
    int wide_targets;
    int64_t rows, vocab;
    int64_t dim;                          // rounded up to 16 bytes in the operands
    float scale;
    float *loss, *lse;                    // forward: written;  backward: lse read
    const float *grad_loss, *grad_lse;    // backward, either may be null
    void *grad_hidden, *grad_weight;      // contiguous [rows, out_dim], [vocab, out_dim]; either may be null
    int64_t out_dim;
    char* ws;
};

// Bytes of workspace, without that of laid out operands.
size_t loss_ws_bytes(int64_t rows, int64_t vocab, int64_t dim, bool bf16);
size_t loss_bwd_ws_bytes(int64_t rows, int64_t vocab, int64_t dim, bool bf16);
// Every launch of a call of these sizes is possible.
bool loss_launchable(int64_t rows, int64_t vocab, int64_t dim, bool backward);
hipError_t launch_loss(const LossArgs& a, bool bf16, hipStream_t stream);
hipError_t launch_loss_bwd(const LossArgs& a, bool bf16, hipStream_t stream);
// Rows of dim values as rows of `padded`, the rest zeros.
hipError_t launch_lay_out(const void* from, int64_t from_stride, int64_t rows, int64_t dim, int64_t padded, void* to, bool bf16,
                          hipStream_t stream);

}  // namespace dpb
