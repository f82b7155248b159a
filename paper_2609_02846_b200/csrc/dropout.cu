// Dropout added to a residual, with a mask that is drawn again wherever it is needed and never stored (sm_100a).
//
//   y_i = residual_i + [r_i >= t] x_i 65536 / (65536 - t),   r_i = 16 bits of Philox4x32-7(key = seed, counter = (i >> 3, 0, 1, 0))
//
// One call of the generator serves a group of eight consecutive elements: 16 bytes of BF16, 32 bytes of FP32.  A thread takes one
// group, its loads first; the generator's ~70 instructions hide behind the memory latency of the other warps.
// Bound by memory: 6 bytes per BF16 element with a residual, 4 without; without one the generator begins to show.  16384 x 4096 BF16
// with a residual: 57.5 us, 7.0 TB/s (two groups per thread 57.8, a persistent grid 66.8), calls from Python in a row 61.5; without
// 45.4 us, 5.9 TB/s (48.6, 56.2).
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cstdint>
#include "../../include/ue5m3.h"
#include "block_ops.h"
#include "common.cuh"

namespace ue5m3 {
namespace {

constexpr int kThreads = 256;

struct DropoutParams {
    DropoutArgs a;
    PhiloxKeys keys;
    int64_t groups;          // ceil(rows * cols / 8)
};

template <bool SMALL>
__device__ __forceinline__ void draw8(const PhiloxKeys& K, uint64_t group, uint32_t w[4]) {
    if (SMALL) philox4x32_c0<1>((uint32_t)group, K, w);
    else philox4x32((uint32_t)group, (uint32_t)(group >> 32), 1u, 0u, K, w);
}
// Element lane j of the group: kept when its half of the draw word, moved to the top of a 32-bit word, is above the limit.
__device__ __forceinline__ bool kept(const uint32_t w[4], int j, uint32_t limit) {
    const uint32_t v = w[j >> 1];
    return ((j & 1) ? v : (v << 16)) > limit;      // bits below the half only break the tie with the limit's low 16 ones: never
}

template <typename T> struct Group8;               // eight elements in memory
template <> struct Group8<__nv_bfloat16> {
    uint4 v;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void get(float f[8]) const { unpack_bf16x8(v, f); }
    static __device__ __forceinline__ void store(__nv_bfloat16* p, const float f[8]) {
        uint4 o;
        uint32_t* q = &o.x;
#pragma unroll
        for (int j = 0; j < 4; ++j) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(q[j]) : "f"(f[2 * j + 1]), "f"(f[2 * j]));
        *reinterpret_cast<uint4*>(p) = o;
    }
};
template <> struct Group8<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float* p) { a = reinterpret_cast<const float4*>(p)[0]; b = reinterpret_cast<const float4*>(p)[1]; }
    __device__ __forceinline__ void get(float f[8]) const {
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    }
    static __device__ __forceinline__ void store(float* p, const float f[8]) {
        reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
    }
};
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// LAYOUT 0: contiguous tensors, groups at 16-byte boundaries, the last one may be short.  1: rows of whole groups at 16-byte
// boundaries, any leading dimensions.  2: anything, element by element.
template <typename T, int LAYOUT, bool DROP, bool SMALL>
__global__ void __launch_bounds__(kThreads) dropout_add_kernel(const DropoutParams p) {
    const DropoutArgs& a = p.a;
    const T* x = static_cast<const T*>(a.x);
    const T* res = static_cast<const T*>(a.residual);
    T* y = static_cast<T*>(a.y);
    const int64_t g = (int64_t)blockIdx.x * kThreads + threadIdx.x, n = a.rows * a.cols;
    if (g >= p.groups) return;
    int64_t row = 0, col = g * 8;                      // where the group begins; LAYOUT 0: all one row
    if (LAYOUT != 0) {
        row = g * 8 / a.cols;
        col = g * 8 - row * a.cols;
    }
    if (LAYOUT == 2 || g * 8 + 8 > n) {
        uint32_t w[4] = {};
        if (DROP) draw8<SMALL>(p.keys, (uint64_t)g, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (g * 8 + j < n) {
                const float v = to_f32(x[row * a.ldx + col]);
                const float k = !DROP || kept(w, j, a.limit) ? v * a.inv_keep : 0.0f;
                put(y + row * a.ldy + col, res ? to_f32(res[row * a.ldr + col]) + k : k);
                ++col;
                if (LAYOUT != 0 && col == a.cols) { col = 0; ++row; }
            }
        }
        return;
    }
    Group8<T> vx, vr;
    vx.load(x + row * a.ldx + col);
    if (res) vr.load(res + row * a.ldr + col);
    uint32_t w[4] = {};
    if (DROP) draw8<SMALL>(p.keys, (uint64_t)g, w);
    float f[8], r[8];
    vx.get(f);
    if (res) vr.get(r);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float k = !DROP || kept(w, j, a.limit) ? f[j] * a.inv_keep : 0.0f;
        f[j] = res ? r[j] + k : k;
    }
    Group8<T>::store(y + row * a.ldy + col, f);
}

template <typename T, int LAYOUT>
cudaError_t run(const DropoutParams& p, cudaStream_t st) {
    const bool small = p.groups < ((int64_t)1 << 32);
    const unsigned grid = (unsigned)((p.groups + kThreads - 1) / kThreads);
    if (!p.a.drop) dropout_add_kernel<T, LAYOUT, false, true><<<grid, kThreads, 0, st>>>(p);
    else if (small) dropout_add_kernel<T, LAYOUT, true, true><<<grid, kThreads, 0, st>>>(p);
    else dropout_add_kernel<T, LAYOUT, true, false><<<grid, kThreads, 0, st>>>(p);
    return cudaGetLastError();
}

template <typename T>
cudaError_t run_of(const DropoutParams& p, cudaStream_t st) {
    const DropoutArgs& a = p.a;
    auto at16 = [](const void* q) { return (reinterpret_cast<uintptr_t>(q) & 15) == 0; };
    const int64_t sz = sizeof(T);
    const bool ptrs = at16(a.x) && at16(a.y) && at16(a.residual);
    const bool contiguous = a.rows == 1 || (a.ldx == a.cols && a.ldy == a.cols && (!a.residual || a.ldr == a.cols));
    if (ptrs && contiguous) return run<T, 0>(p, st);
    const bool lds = (a.ldx * sz) % 16 == 0 && (a.ldy * sz) % 16 == 0 && (!a.residual || (a.ldr * sz) % 16 == 0);
    if (ptrs && lds && a.cols % 8 == 0) return run<T, 1>(p, st);
    return run<T, 2>(p, st);
}

}  // namespace

cudaError_t launch_dropout_add(const DropoutArgs& a, int dtype, cudaStream_t st) {
    DropoutParams p{a, philox_round_keys(a.seed), (a.rows * a.cols + 7) / 8};
    return dtype == UE5M3_BF16 ? run_of<__nv_bfloat16>(p, st) : run_of<float>(p, st);
}

}  // namespace ue5m3
