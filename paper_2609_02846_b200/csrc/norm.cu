// Layer norm of the rows of a matrix, forward and backward, for sm_100a.
//
//   forward   mean = sum x / n, rstd = rsqrt(sum (x - mean)^2 / n + eps), y = (x - mean) rstd w + b
//   backward  xh = (x - mean) rstd, g = dy w:  dx = rstd (g - sum g / n - xh sum(g xh) / n),  dw = sum_r dy xh, db = sum_r dy
//
// Both are bound by memory (2 and 3 elements moved per element, 8 and 14 operations).  The kernels are persistent: a group of
// T threads owns a row at a time, every thread the same 16 columns of each of its rows, so the weights are read once per CTA
// into registers, the column sums of dw and db stay in registers until the CTA ends, and the row itself stays in registers
// between the reductions (the variance is that of the centred values: no cancellation for a large mean).  The next row's loads
// are issued before the current row's reductions, which keeps the memory system busy across the two barriers of a row.
// Column sums leave as one binary32 row per CTA and are added by a second small kernel in a fixed order: no atomics.
// Rows longer than 16 * 1024 columns take a kernel that re-reads the row instead.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cstdint>
#include "../../include/ue5m3.h"
#include "block_ops.h"
#include "common.cuh"

namespace ue5m3 {
namespace {

constexpr int kPerThread = 16;                       // columns a thread holds at most
constexpr int kMaxRowThreads = 1024;
constexpr int kBwdGroups = 148;                      // CTAs of the backward kernel: one per SM of a B200

// VEC consecutive elements of one row as they lie in memory.
template <typename T, int VEC> struct Raw;
template <> struct Raw<__nv_bfloat16, 8> { uint4 v; };
template <> struct Raw<float, 4> { uint4 v; };
template <> struct Raw<__nv_bfloat16, 1> { unsigned short v; };
template <> struct Raw<float, 1> { float v; };

__device__ __forceinline__ void load_raw(Raw<__nv_bfloat16, 8>& r, const __nv_bfloat16* p) { r.v = ldg_nc_v4(p); }
__device__ __forceinline__ void load_raw(Raw<float, 4>& r, const float* p) { r.v = ldg_nc_v4(p); }
__device__ __forceinline__ void load_raw(Raw<__nv_bfloat16, 1>& r, const __nv_bfloat16* p) { r.v = __ldg(reinterpret_cast<const unsigned short*>(p)); }
__device__ __forceinline__ void load_raw(Raw<float, 1>& r, const float* p) { r.v = __ldg(p); }

__device__ __forceinline__ void unpack(const Raw<__nv_bfloat16, 8>& r, float* f) { unpack_bf16x8(r.v, f); }
__device__ __forceinline__ void unpack(const Raw<float, 4>& r, float* f) {
    f[0] = __uint_as_float(r.v.x); f[1] = __uint_as_float(r.v.y); f[2] = __uint_as_float(r.v.z); f[3] = __uint_as_float(r.v.w);
}
__device__ __forceinline__ void unpack(const Raw<__nv_bfloat16, 1>& r, float* f) { f[0] = __uint_as_float((uint32_t)r.v << 16); }
__device__ __forceinline__ void unpack(const Raw<float, 1>& r, float* f) { f[0] = r.v; }

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <int VEC> __device__ __forceinline__ void store_vec(__nv_bfloat16* p, const float* f) {
    if constexpr (VEC == 8)
        *reinterpret_cast<uint4*>(p) = make_uint4(bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3]), bf16_pair(f[4], f[5]), bf16_pair(f[6], f[7]));
    else
        *p = __float2bfloat16_rn(f[0]);
}
template <int VEC> __device__ __forceinline__ void store_vec(float* p, const float* f) {
    if constexpr (VEC == 4) *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
    else *p = f[0];
}
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
// VEC parameters of type TW (read once per CTA: plain loads of the element type, 4 or 16 bytes wide where the compiler may)
template <int VEC, typename TW> __device__ __forceinline__ void load_params(const TW* p, float* f) {
#pragma unroll
    for (int j = 0; j < VEC; ++j) f[j] = to_f32(p[j]);
}

// Sums of N values over the T threads of a row group (T a multiple of 32), the same order every time.  `scratch` is this
// group's [2][32][N] floats; `turn` alternates between the two halves, so one barrier per sum is enough.
template <int N>
__device__ __forceinline__ void group_sum(float (&v)[N], float* scratch, int& turn, int threads, int barrier_id) {
#pragma unroll
    for (int o = 16; o; o >>= 1)
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], o);
    if (threads == 32) return;
    float* s = scratch + turn * 32 * N;
    turn ^= 1;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (lane == 0)
#pragma unroll
        for (int k = 0; k < N; ++k) s[warp * N + k] = v[k];
    asm volatile("bar.sync %0, %1;" ::"r"(barrier_id), "r"(threads) : "memory");
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = lane < (threads >> 5) ? s[lane * N + k] : 0.0f;
#pragma unroll
    for (int o = 16; o; o >>= 1)
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], o);
}

// ------------------------------------------------------------------------------------------------ forward
// blockDim = (T, R): R groups of T threads, a row each.  NV vectors of VEC columns per thread.  MAXT bounds the CTA: with up to
// 512 threads there are registers for the weights; the 1024-thread CTA of rows over 8192 columns reads them per row (from L1).
template <typename TX, typename TW, int VEC, int NV, int MAXT>
__global__ void __launch_bounds__(MAXT)
layer_norm_kernel(const LayerNormArgs a) {
    constexpr bool KEEP = MAXT <= 512;
    extern __shared__ float scratch_all[];
    float* scratch = scratch_all + threadIdx.y * 64;
    const int T = blockDim.x, bar_id = 1 + threadIdx.y;
    const int nvec = (int)(a.cols / VEC);
    const TX* x = static_cast<const TX*>(a.x);
    TX* y = static_cast<TX*>(a.y);
    auto params = [&](int vi, float* w, float* b) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) { w[j] = 1.0f; b[j] = 0.0f; }
        if (vi < nvec) {
            if (a.weight) load_params<VEC>(static_cast<const TW*>(a.weight) + (int64_t)vi * VEC, w);
            if (a.bias) load_params<VEC>(static_cast<const TW*>(a.bias) + (int64_t)vi * VEC, b);
        }
    };
    float w[KEEP ? NV : 1][VEC], b[KEEP ? NV : 1][VEC];
    if constexpr (KEEP)
#pragma unroll
        for (int k = 0; k < NV; ++k) params(threadIdx.x + k * T, w[k], b[k]);
    const float inv_n = 1.0f / (float)a.cols;
    const int64_t step = (int64_t)gridDim.x * blockDim.y;
    int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    Raw<TX, VEC> next[NV] = {};
    if (row < a.rows)
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (threadIdx.x + k * T < nvec) load_raw(next[k], x + row * a.ldx + (int64_t)(threadIdx.x + k * T) * VEC);
    int turn = 0;
    for (; row < a.rows; row += step) {
        float f[NV][VEC];
#pragma unroll
        for (int k = 0; k < NV; ++k) unpack(next[k], f[k]);
        if (row + step < a.rows)
#pragma unroll
            for (int k = 0; k < NV; ++k)
                if (threadIdx.x + k * T < nvec) load_raw(next[k], x + (row + step) * a.ldx + (int64_t)(threadIdx.x + k * T) * VEC);
        float s[1] = {0.0f};
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < VEC; ++j) s[0] += f[k][j];               // columns beyond the row hold zeros
        group_sum<1>(s, scratch, turn, T, bar_id);
        const float mean = s[0] * inv_n;
        float q[1] = {0.0f};
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (threadIdx.x + k * T < nvec)
#pragma unroll
                for (int j = 0; j < VEC; ++j) { f[k][j] -= mean; q[0] = fmaf(f[k][j], f[k][j], q[0]); }
        group_sum<1>(q, scratch, turn, T, bar_id);
        const float rstd = 1.0f / sqrtf(fmaf(q[0], inv_n, a.eps));
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (threadIdx.x + k * T < nvec) {
                constexpr int one = KEEP ? 1 : 0;
                if constexpr (!KEEP) params(threadIdx.x + k * T, w[0], b[0]);
                float o[VEC];
#pragma unroll
                for (int j = 0; j < VEC; ++j) o[j] = fmaf(f[k][j] * rstd, w[k * one][j], b[k * one][j]);
                store_vec<VEC>(y + row * a.ldy + (int64_t)(threadIdx.x + k * T) * VEC, o);
            }
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

// Rows of any length: the row is read three times (from L1/L2 after the first).
template <typename TX, typename TW>
__global__ void __launch_bounds__(kMaxRowThreads) layer_norm_long_kernel(const LayerNormArgs a) {
    __shared__ float scratch[64];
    const float inv_n = 1.0f / (float)a.cols;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const TX* x = static_cast<const TX*>(a.x) + row * a.ldx;
        TX* y = static_cast<TX*>(a.y) + row * a.ldy;
        float s[1] = {0.0f};
        for (int64_t c = threadIdx.x; c < a.cols; c += blockDim.x) s[0] += to_f32(x[c]);
        group_sum<1>(s, scratch, turn, blockDim.x, 1);
        const float mean = s[0] * inv_n;
        float q[1] = {0.0f};
        for (int64_t c = threadIdx.x; c < a.cols; c += blockDim.x) { const float d = to_f32(x[c]) - mean; q[0] = fmaf(d, d, q[0]); }
        group_sum<1>(q, scratch, turn, blockDim.x, 1);
        const float rstd = 1.0f / sqrtf(fmaf(q[0], inv_n, a.eps));
        for (int64_t c = threadIdx.x; c < a.cols; c += blockDim.x) {
            const float w = a.weight ? to_f32(static_cast<const TW*>(a.weight)[c]) : 1.0f;
            const float b = a.bias ? to_f32(static_cast<const TW*>(a.bias)[c]) : 0.0f;
            const float o = fmaf((to_f32(x[c]) - mean) * rstd, w, b);
            store_vec<1>(y + c, &o);
        }
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

// ------------------------------------------------------------------------------------------------ backward
template <typename TX, typename TW, int VEC, int NV>
__global__ void __launch_bounds__(512)
layer_norm_backward_kernel(const LayerNormArgs a) {
    extern __shared__ float smem[];                       // [R][128] reduction scratch, then [R][2][T * NV * VEC] column sums
    asm volatile("griddepcontrol.launch_dependents;");    // the adding kernel may take its place; it waits for this grid's end
    float* scratch = smem + threadIdx.y * 128;
    const int T = blockDim.x, R = blockDim.y, bar_id = 1 + threadIdx.y;
    const int nvec = (int)(a.cols / VEC);
    const TX* x = static_cast<const TX*>(a.x);
    const TX* dy = static_cast<const TX*>(a.dy);
    TX* dx = static_cast<TX*>(a.y);
    float w[NV][VEC], dw[NV][VEC], db[NV][VEC];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int vi = threadIdx.x + k * T;
#pragma unroll
        for (int j = 0; j < VEC; ++j) { w[k][j] = 1.0f; dw[k][j] = 0.0f; db[k][j] = 0.0f; }
        if (a.weight && vi < nvec) load_params<VEC>(static_cast<const TW*>(a.weight) + (int64_t)vi * VEC, w[k]);
    }
    const float inv_n = 1.0f / (float)a.cols;
    const int64_t step = (int64_t)gridDim.x * R;
    int64_t row = (int64_t)blockIdx.x * R + threadIdx.y;
    Raw<TX, VEC> nx[NV] = {}, ny[NV] = {};
    float next_mean = 0.0f, next_rstd = 0.0f;
    auto fetch = [&](int64_t r) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int vi = threadIdx.x + k * T;
            if (vi < nvec) {
                load_raw(nx[k], x + r * a.ldx + (int64_t)vi * VEC);
                load_raw(ny[k], dy + r * a.lddy + (int64_t)vi * VEC);
            }
        }
        next_mean = __ldg(a.mean + r);
        next_rstd = __ldg(a.rstd + r);
    };
    if (row < a.rows) fetch(row);
    int turn = 0;
    for (; row < a.rows; row += step) {
        float xh[NV][VEC], g[NV][VEC];
        const float mean = next_mean, rstd = next_rstd;
        float s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            unpack(nx[k], xh[k]);
            unpack(ny[k], g[k]);
            if (threadIdx.x + k * T < nvec)
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    xh[k][j] = (xh[k][j] - mean) * rstd;
                    dw[k][j] = fmaf(g[k][j], xh[k][j], dw[k][j]);
                    db[k][j] += g[k][j];
                    g[k][j] *= w[k][j];
                    s[0] += g[k][j];
                    s[1] = fmaf(g[k][j], xh[k][j], s[1]);
                }
        }
        if (row + step < a.rows) fetch(row + step);
        group_sum<2>(s, scratch, turn, T, bar_id);
        const float mg = s[0] * inv_n, mgx = s[1] * inv_n;
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (threadIdx.x + k * T < nvec) {
                float o[VEC];
#pragma unroll
                for (int j = 0; j < VEC; ++j) o[j] = rstd * (g[k][j] - mg - xh[k][j] * mgx);
                store_vec<VEC>(dx + row * a.ldy + (int64_t)(threadIdx.x + k * T) * VEC, o);
            }
    }
    if (!a.partial) return;
    // the R groups' column sums, added in order by the first group
    const int per_group = T * NV * VEC;
    float* sums = smem + R * 128;
    if (threadIdx.y > 0)
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                // [.. ][k][j][thread]: a warp's stores fall into 32 different banks
                sums[(threadIdx.y - 1) * 2 * per_group + (k * VEC + j) * T + threadIdx.x] = dw[k][j];
                sums[(threadIdx.y - 1) * 2 * per_group + per_group + (k * VEC + j) * T + threadIdx.x] = db[k][j];
            }
    __syncthreads();
    if (threadIdx.y > 0) return;
    float* out = a.partial + (int64_t)blockIdx.x * 2 * a.cols;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int vi = threadIdx.x + k * T;
        if (vi >= nvec) continue;
#pragma unroll
        for (int j = 0; j < VEC; ++j)
            for (int r = 0; r < R - 1; ++r) {
                dw[k][j] += sums[r * 2 * per_group + (k * VEC + j) * T + threadIdx.x];
                db[k][j] += sums[r * 2 * per_group + per_group + (k * VEC + j) * T + threadIdx.x];
            }
        if constexpr (VEC % 4 == 0) {
#pragma unroll
            for (int j = 0; j < VEC; j += 4) {
                *reinterpret_cast<float4*>(out + (int64_t)vi * VEC + j) = make_float4(dw[k][j], dw[k][j + 1], dw[k][j + 2], dw[k][j + 3]);
                *reinterpret_cast<float4*>(out + a.cols + (int64_t)vi * VEC + j) = make_float4(db[k][j], db[k][j + 1], db[k][j + 2], db[k][j + 3]);
            }
        } else {
            out[vi] = dw[k][0];
            out[a.cols + vi] = db[k][0];
        }
    }
}

// Rows of any length: column sums are kept in this CTA's row of the workspace.
template <typename TX, typename TW>
__global__ void __launch_bounds__(kMaxRowThreads) layer_norm_backward_long_kernel(const LayerNormArgs a) {
    __shared__ float scratch[128];
    asm volatile("griddepcontrol.launch_dependents;");
    const float inv_n = 1.0f / (float)a.cols;
    float* out = a.partial ? a.partial + (int64_t)blockIdx.x * 2 * a.cols : nullptr;
    if (out)
        for (int64_t c = threadIdx.x; c < a.cols; c += blockDim.x) { out[c] = 0.0f; out[a.cols + c] = 0.0f; }   // own columns only
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const TX* x = static_cast<const TX*>(a.x) + row * a.ldx;
        const TX* dy = static_cast<const TX*>(a.dy) + row * a.lddy;
        TX* dx = static_cast<TX*>(a.y) + row * a.ldy;
        const TW* wp = static_cast<const TW*>(a.weight);
        const float mean = a.mean[row], rstd = a.rstd[row];
        float s[2] = {0.0f, 0.0f};
        for (int64_t c = threadIdx.x; c < a.cols; c += blockDim.x) {
            const float xh = (to_f32(x[c]) - mean) * rstd, d = to_f32(dy[c]), g = d * (wp ? to_f32(wp[c]) : 1.0f);
            if (out) { out[c] = fmaf(d, xh, out[c]); out[a.cols + c] += d; }
            s[0] += g;
            s[1] = fmaf(g, xh, s[1]);
        }
        group_sum<2>(s, scratch, turn, blockDim.x, 1);
        const float mg = s[0] * inv_n, mgx = s[1] * inv_n;
        for (int64_t c = threadIdx.x; c < a.cols; c += blockDim.x) {
            const float xh = (to_f32(x[c]) - mean) * rstd, g = to_f32(dy[c]) * (wp ? to_f32(wp[c]) : 1.0f);
            const float o = rstd * (g - mg - xh * mgx);
            store_vec<1>(dx + c, &o);
        }
    }
}

// Adds the CTAs' column sums: 32 columns of dw (blockIdx.y = 0) or db (1) per CTA, rows of sums dealt to 16 warps.
template <typename TW>
__global__ void __launch_bounds__(512) layer_norm_columns_kernel(const float* partial, int groups, int64_t cols, TW* dw, TW* db) {
    __shared__ float part[16][33];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    TW* out = blockIdx.y ? db : dw;
    if (!out) return;
    const int64_t c = (int64_t)blockIdx.x * 32 + threadIdx.x;
    float s = 0.0f;
    if (c < cols) {
        const float* p = partial + blockIdx.y * cols + c;
#pragma unroll 4
        for (int g = threadIdx.y; g < groups; g += 16) s += p[(int64_t)g * 2 * cols];
    }
    part[threadIdx.y][threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.y == 0 && c < cols) {
#pragma unroll
        for (int g = 1; g < 16; ++g) s += part[g][threadIdx.x];
        store_vec<1>(out + c, &s);
    }
}

// ------------------------------------------------------------------------------------------------ host
inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

struct RowShape { int threads, groups; };
// Threads of a row group that hold `cols` columns at per_thread each, and how many groups make a CTA of about `cta` threads.
RowShape row_shape(int64_t cols, int per_thread, int cta) {
    const int t = (int)((cols + (int64_t)per_thread * 32 - 1) / ((int64_t)per_thread * 32)) * 32;
    int r = cta / t;
    r = r < 1 ? 1 : (r > 15 ? 15 : r);                   // named barriers 1..15
    return RowShape{t, r};
}

template <typename TX, typename TW, int VEC, int NV, int MAXT>
cudaError_t run_forward(const LayerNormArgs& a, int num_sms, cudaStream_t st) {
    const RowShape s = row_shape(a.cols, VEC * NV, 128);
    const size_t smem = (size_t)s.groups * 64 * sizeof(float);
    int per_sm = 0;
    cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, layer_norm_kernel<TX, TW, VEC, NV, MAXT>, s.threads * s.groups, smem);
    if (e != cudaSuccess) return e;
    const int64_t need = (a.rows + s.groups - 1) / s.groups, room = (int64_t)num_sms * (per_sm < 1 ? 1 : per_sm);
    layer_norm_kernel<TX, TW, VEC, NV, MAXT><<<(unsigned)(need < room ? need : room), dim3(s.threads, s.groups), smem, st>>>(a);
    return cudaGetLastError();
}

template <typename TX, typename TW>
cudaError_t forward_of(const LayerNormArgs& a, int num_sms, cudaStream_t st) {
    constexpr int V = 16 / sizeof(TX);
    if (a.cols > (int64_t)kPerThread * kMaxRowThreads) {
        layer_norm_long_kernel<TX, TW><<<(unsigned)(a.rows < 2 * num_sms ? a.rows : 2 * num_sms), kMaxRowThreads, 0, st>>>(a);
        return cudaGetLastError();
    }
    const bool vec = a.cols % V == 0 && (a.ldx * (int64_t)sizeof(TX)) % 16 == 0 && (a.ldy * (int64_t)sizeof(TX)) % 16 == 0 &&
                     aligned(a.x, 16) && aligned(a.y, 16);
    if (a.cols > kPerThread * 512)
        return vec ? run_forward<TX, TW, V, kPerThread / V, kMaxRowThreads>(a, num_sms, st) : run_forward<TX, TW, 1, kPerThread, kMaxRowThreads>(a, num_sms, st);
    if (vec) return run_forward<TX, TW, V, kPerThread / V, 512>(a, num_sms, st);
    return a.cols <= 4 * 256 ? run_forward<TX, TW, 1, 4, 256>(a, num_sms, st) : run_forward<TX, TW, 1, kPerThread, 512>(a, num_sms, st);
}

template <typename TW>
cudaError_t add_columns(const LayerNormArgs& a, int groups, cudaStream_t st) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)((a.cols + 31) / 32), a.dbias ? 2 : 1);
    cfg.blockDim = dim3(32, 16);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, layer_norm_columns_kernel<TW>, (const float*)a.partial, groups, a.cols, (TW*)a.dweight, (TW*)a.dbias);
}

template <typename TX, typename TW, int VEC, int NV>
cudaError_t run_backward(const LayerNormArgs& a, int num_sms, cudaStream_t st) {
    const RowShape s = row_shape(a.cols, VEC * NV, 512);
    const size_t smem = ((size_t)s.groups * 128 + (size_t)(s.groups - 1) * 2 * s.threads * NV * VEC) * sizeof(float);
    cudaError_t e = cudaFuncSetAttribute(layer_norm_backward_kernel<TX, TW, VEC, NV>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    const int64_t need = (a.rows + s.groups - 1) / s.groups;
    const int grid = (int)(need < kBwdGroups ? need : kBwdGroups);
    if (grid > 0) layer_norm_backward_kernel<TX, TW, VEC, NV><<<grid, dim3(s.threads, s.groups), smem, st>>>(a);
    e = cudaGetLastError();
    return e != cudaSuccess || !a.partial ? e : add_columns<TW>(a, grid, st);
}

template <typename TX, typename TW>
cudaError_t backward_of(const LayerNormArgs& a, int num_sms, cudaStream_t st) {
    constexpr int V = 16 / sizeof(TX);
    if (a.cols > (int64_t)kPerThread * 512) {
        const int grid = (int)(a.rows < kBwdGroups ? a.rows : kBwdGroups);
        if (grid > 0) layer_norm_backward_long_kernel<TX, TW><<<grid, kMaxRowThreads, 0, st>>>(a);
        const cudaError_t e = cudaGetLastError();
        return e != cudaSuccess || !a.partial ? e : add_columns<TW>(a, grid, st);
    }
    const bool vec = a.cols % V == 0 && (a.ldx * (int64_t)sizeof(TX)) % 16 == 0 && (a.ldy * (int64_t)sizeof(TX)) % 16 == 0 &&
                     (a.lddy * (int64_t)sizeof(TX)) % 16 == 0 && aligned(a.x, 16) && aligned(a.y, 16) && aligned(a.dy, 16);
    if (vec) return run_backward<TX, TW, V, kPerThread / V>(a, num_sms, st);
    return run_backward<TX, TW, 1, kPerThread>(a, num_sms, st);
}

}  // namespace

int layer_norm_backward_groups(int64_t rows) { return (int)(rows < kBwdGroups ? (rows < 1 ? 1 : rows) : kBwdGroups); }

cudaError_t launch_layer_norm(const LayerNormArgs& a, int dtype, int weight_dtype, int num_sms, cudaStream_t st) {
    if (dtype == UE5M3_BF16)
        return weight_dtype == UE5M3_BF16 ? forward_of<__nv_bfloat16, __nv_bfloat16>(a, num_sms, st) : forward_of<__nv_bfloat16, float>(a, num_sms, st);
    return weight_dtype == UE5M3_BF16 ? forward_of<float, __nv_bfloat16>(a, num_sms, st) : forward_of<float, float>(a, num_sms, st);
}
cudaError_t launch_layer_norm_backward(const LayerNormArgs& a, int dtype, int weight_dtype, int num_sms, cudaStream_t st) {
    if (dtype == UE5M3_BF16)
        return weight_dtype == UE5M3_BF16 ? backward_of<__nv_bfloat16, __nv_bfloat16>(a, num_sms, st) : backward_of<__nv_bfloat16, float>(a, num_sms, st);
    return weight_dtype == UE5M3_BF16 ? backward_of<float, __nv_bfloat16>(a, num_sms, st) : backward_of<float, float>(a, num_sms, st);
}

}  // namespace ue5m3
