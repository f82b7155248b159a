// Host-side launch interface of the operators between the quantized linears (layer norm, dropout, attention).
#pragma once
#include <cuda_runtime.h>
#include <atomic>
#include <cstdint>
#include "../../include/ue5m3.h"

namespace ue5m3 {

// Raises a kernel's limit of dynamic shared memory once per device (the attribute lasts as long as the device's context, and
// asking for it again costs as much as half a launch).
template <typename Kernel>
inline cudaError_t allow_smem(Kernel* kernel, int bytes, std::atomic<int> (&granted)[64]) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64 && granted[dev].load(std::memory_order_relaxed) >= bytes) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess && dev >= 0 && dev < 64) granted[dev].store(bytes, std::memory_order_relaxed);
    return e;
}

// Failure-detection self-test: the bound of every device-side wait in SM clocks, with the copies switched off (0: a normal launch).
struct StallTest { long long wait_limit = 0; };

struct LayerNormArgs {
    const void* x; int64_t ldx;
    const void* weight; const void* bias;
    void* y; int64_t ldy;                 // backward: dx
    const void* dy; int64_t lddy;         // backward only
    float* mean; float* rstd;
    void* dweight; void* dbias;           // backward only
    float* partial;                       // backward only: [groups][2][cols]
    int64_t rows, cols;
    float eps;
};
// CTAs of the backward kernel = rows of column sums it leaves in the workspace
int layer_norm_backward_groups(int64_t rows);
cudaError_t launch_layer_norm(const LayerNormArgs& a, int dtype, int weight_dtype, int num_sms, cudaStream_t st, const StallTest& stall = {});
cudaError_t launch_layer_norm_backward(const LayerNormArgs& a, int dtype, int weight_dtype, cudaStream_t st, const StallTest& stall = {});

struct DropoutArgs {
    const void* x; const void* residual; void* y;
    int64_t ldx, ldr, ldy, rows, cols;
    uint32_t limit;                       // (t << 16) - 1: a draw in the upper 16 bits of a word keeps its element when above it
    int drop;                             // 0: t = 0, nothing is dropped and no bits are drawn
    float inv_keep;                       // 65536 / (65536 - t); 0 when t = 65536
    uint64_t seed;
};
cudaError_t launch_dropout_add(const DropoutArgs& a, int dtype, cudaStream_t st);

// returns a UE5M3_* status
int launch_attention(const ue5m3_attention_shape& s, const ue5m3_heads& q, const ue5m3_heads& k, const ue5m3_heads& v,
                     const ue5m3_heads& o, float* lse, float* workspace, int num_sms, cudaStream_t st, const StallTest& stall = {});
int attention_splits(const ue5m3_attention_shape& s);      // parts into which the keys are shared out (1: none)
int launch_attention_backward(const ue5m3_attention_shape& s, const ue5m3_heads& dout, const ue5m3_heads& q,
                              const ue5m3_heads& k, const ue5m3_heads& v, const ue5m3_heads& o, const float* lse,
                              const ue5m3_heads& dq, const ue5m3_heads& dk, const ue5m3_heads& dv, float* workspace,
                              cudaStream_t st, const StallTest& stall = {});
int attention_backward_splits(const ue5m3_attention_shape& s);        // the same for the queries' gradient
int read_and_clear_norm_status();                 // these three synchronise the device
int read_and_clear_attention_status();
int read_and_clear_attention_backward_status();

// Queries padded to whole tiles: rows of the backward pass's workspace.
inline int64_t attention_padded_q(int64_t q_len) { return (q_len + 127) / 128 * 128; }

}  // namespace ue5m3
