// Rotary positions of queries and keys, alone or behind a norm of every head's row, with the backward pass, for sm_100a.
//
//   rotary     pair (a, b) of frequency f at position p: t = p f;  a' = A (a cos t - b sin t),  b' = A (a sin t + b cos t)
//   with norm  r = 1 / sqrt(mean x^2 + eps);  y = rotate(x r w)
//   backward   g' = rotate(dy) by -t;  g = g' w, xh = x r:  dx = r (g - xh mean(g xh)),  dw = sum over rows of g' xh
//
// All three are bound by memory: every element is read once (backward: x and dy) and written once.  Queries and keys of a token go in
// one launch and share its angles.  Angles are products in binary64, in turns, of which only the fraction goes on in binary32: p f in
// binary32 would be off by 2^-24 p f radians, 0.06 at a million positions.
//
// A warp takes a token.  G lanes hold a head's row, each VEC pairs of it (two vectors: the two halves of the pairs, or one piece of
// neighbouring pairs), 32 / G heads side by side, and the warp walks the heads with a lane's pairs, and so its angles and weights,
// staying the same.  The norm's sum over a row is log2(G) shuffles; nothing passes through shared memory.  Where there are few tokens the heads of
// one are shared out among warps.  VEC is 16 bytes where the pairs and the addresses allow it, else 8, 4 or 2.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <algorithm>
#include <cstdint>
#include "../../include/ue5m3.h"
#include "block_ops.h"
#include "common.cuh"

namespace ue5m3 {
namespace {

constexpr int kThreads = 128, kWarps = kThreads / 32;

struct Side {                                          // queries or keys
    const void* x; const void* dy; void* y;            // backward: y is dx
    int64_t xs[3], ds[3], ys[3];                       // batch, token, head
    const void* weight;
    int heads, groups;                                 // groups of 32 / G heads
};
struct RotaryParams {
    Side side[2];
    const double* frequencies;
    const void* positions;
    int64_t position_stride, first_position;
    int64_t items, tokens;                             // items: batch * tokens * parts
    int wide_positions, half_rotary, dim, lanes, parts;        // lanes: log2(G)
    int weight_f32;
    float amplitude, eps, inv_dim;
    float sign;                                        // -1: angles negated
    float* partial;                                    // backward: [CTAs][2][dim] sums for the weights' gradients
};

template <int BYTES> struct Raw;                       // a vector as it lies in memory
template <> struct Raw<16> { uint4 v; };
template <> struct Raw<8> { uint2 v; };
template <> struct Raw<4> { uint32_t v; };
template <> struct Raw<2> { unsigned short v; };
// (plain loads: the output may be the input, and a load through the read-only path promises that the kernel writes nothing there)
template <int BYTES> __device__ __forceinline__ Raw<BYTES> load_raw(const void* p) { return *reinterpret_cast<const Raw<BYTES>*>(p); }

template <int VEC> __device__ __forceinline__ void unpack(const Raw<VEC * 2>& r, float* f, __nv_bfloat16) {
    if constexpr (VEC == 1) f[0] = __uint_as_float((uint32_t)r.v << 16);
    else if constexpr (VEC == 2) unpack_bf16x2(r.v, f[0], f[1]);
    else if constexpr (VEC == 4) { unpack_bf16x2(r.v.x, f[0], f[1]); unpack_bf16x2(r.v.y, f[2], f[3]); }
    else unpack_bf16x8(r.v, f);
}
template <int VEC> __device__ __forceinline__ void unpack(const Raw<VEC * 4>& r, float* f, float) {
    if constexpr (VEC == 1) f[0] = __uint_as_float(r.v);
    else if constexpr (VEC == 2) { f[0] = __uint_as_float(r.v.x); f[1] = __uint_as_float(r.v.y); }
    else { f[0] = __uint_as_float(r.v.x); f[1] = __uint_as_float(r.v.y); f[2] = __uint_as_float(r.v.z); f[3] = __uint_as_float(r.v.w); }
}
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <int VEC> __device__ __forceinline__ void store_vec(__nv_bfloat16* p, const float* f) {
    if constexpr (VEC == 1) *p = __float2bfloat16_rn(f[0]);
    else if constexpr (VEC == 2) *reinterpret_cast<uint32_t*>(p) = bf16_pair(f[0], f[1]);
    else if constexpr (VEC == 4) *reinterpret_cast<uint2*>(p) = make_uint2(bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3]));
    else *reinterpret_cast<uint4*>(p) = make_uint4(bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3]), bf16_pair(f[4], f[5]), bf16_pair(f[6], f[7]));
}
template <int VEC> __device__ __forceinline__ void store_vec(float* p, const float* f) {
    if constexpr (VEC == 1) *p = f[0];
    else if constexpr (VEC == 2) *reinterpret_cast<float2*>(p) = make_float2(f[0], f[1]);
    else *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
}

// What a lane holds of a row: NU units of VEC pairs.  Unit u of a row: the pairs u VEC .. of the rotary part, behind them pieces of 2 VEC
// columns that are not turned.
template <int VEC, int NU, bool NEIGHBOURS> struct Lane {
    int at[NU][2];                                     // first column of the two vectors
    int turned[NU];                                    // pairs of the unit that are turned
    bool here[NU];                                     // the row has this unit
    bool some_still;                                   // some pair of this lane is not turned
    __device__ __forceinline__ void place(int first, int lanes, int half, int dim) {
        some_still = false;
#pragma unroll
        for (int k = 0; k < NU; ++k) {
            const int u = first + (k << lanes);
            here[k] = u * 2 * VEC < dim;
            const bool split = !NEIGHBOURS && u * VEC < half;
            at[k][0] = here[k] ? (split ? u * VEC : u * 2 * VEC) : 0;
            at[k][1] = here[k] ? (split ? half + u * VEC : u * 2 * VEC + VEC) : VEC;
            turned[k] = min(max(half - u * VEC, 0), VEC);
            some_still |= turned[k] < VEC;
        }
    }
};
// Columns x[0 .. 2 VEC) of a unit -> turned by (c, s); x[i], x[j] is pair k.
template <int VEC, bool NEIGHBOURS> __device__ __forceinline__ void turn(float* x, const float* c, const float* s, int turned, bool some_still) {
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
        const int i = NEIGHBOURS ? 2 * k : k, j = NEIGHBOURS ? 2 * k + 1 : VEC + k;
        const float a = x[i], b = x[j];
        const float u = a * c[k] - b * s[k], v = a * s[k] + b * c[k];
        // a pair that stays is kept as it is: a product with a sine of zero would carry an infinity over to its partner
        x[i] = !some_still || k < turned ? u : a;
        x[j] = !some_still || k < turned ? v : b;
    }
}
// Cosines and sines (times the amplitude) of a lane's pairs at a position.
template <int VEC, int NU> __device__ __forceinline__ void angles(const RotaryParams& p, double position, const int (&first)[NU], float* c, float* s) {
#pragma unroll
    for (int k = 0; k < NU; ++k)
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const int i = first[k] + j;
            const double f = __ldg(p.frequencies + min(i, p.half_rotary - 1));
            const double turns = i < p.half_rotary ? position * (f * 0.15915494309189533577) : 0.0;
            const float part = (float)(turns - rint(turns));           // -1/2 .. 1/2
            float sn, cs;
            sincospif(2.0f * part, &sn, &cs);
            c[k * VEC + j] = cs * p.amplitude;
            s[k * VEC + j] = sn * (p.amplitude * p.sign);
        }
}
__device__ __forceinline__ double position_of(const RotaryParams& p, int64_t b, int64_t t) {
    if (!p.positions) return (double)(p.first_position + t);
    const char* at = static_cast<const char*>(p.positions) + ((b * p.position_stride + t) << (p.wide_positions ? 3 : 2));
    return p.wide_positions ? (double)__ldg(reinterpret_cast<const long long*>(at)) : (double)__ldg(reinterpret_cast<const int*>(at));
}
__device__ const float g_ones[256] = {
#define ONES8 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f
#define ONES64 ONES8, ONES8, ONES8, ONES8, ONES8, ONES8, ONES8, ONES8
    ONES64, ONES64, ONES64, ONES64
#undef ONES64
#undef ONES8
};
// A lane's weights (1 without).
template <int VEC, int NU, bool NB> __device__ __forceinline__ void load_weights(const RotaryParams& p, const Side& s, const Lane<VEC, NU, NB>& l, float* w) {
    const void* weight = s.weight ? s.weight : g_ones;
    const bool f32 = p.weight_f32 || !s.weight;
#pragma unroll
    for (int k = 0; k < NU; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const int i = l.at[k][h] + j;
                w[(k * 2 + h) * VEC + j] = f32 ? static_cast<const float*>(weight)[i] : __bfloat162float(static_cast<const __nv_bfloat16*>(weight)[i]);
            }
}
__device__ __forceinline__ float row_sum(float v, int lanes) {
    for (int d = (1 << lanes) >> 1; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    return v;
}

template <typename T, int VEC, int NU> struct RowRaw { Raw<VEC * sizeof(T)> v[NU][2]; };
// Every address is one of the tensor's: what a lane does not have is read from the row's start, and what does not exist from another row.
template <typename T, int VEC, int NU, bool NB>
__device__ __forceinline__ void load_row(RowRaw<T, VEC, NU>& r, const T* row, const Lane<VEC, NU, NB>& l) {
#pragma unroll
    for (int k = 0; k < NU; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h) r.v[k][h] = load_raw<VEC * sizeof(T)>(row + l.at[k][h]);
}
template <typename T, int VEC, int NU> __device__ __forceinline__ void unpack_row(const RowRaw<T, VEC, NU>& r, float* x) {
#pragma unroll
    for (int k = 0; k < NU; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h) unpack<VEC>(r.v[k][h], x + (k * 2 + h) * VEC, T());
}
template <typename T, int VEC, int NU, bool NB>
__device__ __forceinline__ void store_row(T* row, const float* x, const Lane<VEC, NU, NB>& l, bool exists) {
#pragma unroll
    for (int k = 0; k < NU; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (exists && l.here[k]) store_vec<VEC>(row + l.at[k][h], x + (k * 2 + h) * VEC);
}

// One item of a warp: the head groups [g, g_end) of one token, queries before keys.
struct Item { int64_t b, t; int g, g_end; };
__device__ __forceinline__ Item item_of(const RotaryParams& p, int64_t index) {
    const int64_t token = p.parts == 1 ? index : index / p.parts;
    const int part = p.parts == 1 ? 0 : (int)(index - token * p.parts), groups = p.side[0].groups + p.side[1].groups;
    Item w;
    w.b = token / p.tokens;
    w.t = token - w.b * p.tokens;
    w.g = (int)((int64_t)groups * part / p.parts);
    w.g_end = (int)((int64_t)groups * (part + 1) / p.parts);
    return w;
}

template <typename T, int VEC, bool NEIGHBOURS, bool NORM>
__global__ void __launch_bounds__(kThreads) rotary_kernel(const __grid_constant__ RotaryParams p) {
    constexpr int NU = VEC >= 4 ? 1 : 4 / VEC, U = VEC >= 4 ? 4 : 2;       // rows in flight per lane
    const int lane = threadIdx.x & 31;
    const int64_t index = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
    if (index >= p.items) return;
    const Item item = item_of(p, index);
    Lane<VEC, NU, NEIGHBOURS> l;
    l.place(lane & ((1 << p.lanes) - 1), p.lanes, p.half_rotary, p.dim);
    const int slot = lane >> p.lanes, slots = 32 >> p.lanes;
    float c[NU * VEC], s[NU * VEC], w[NU * 2 * VEC];
    bool turned = false;
    for (int g = item.g; g < item.g_end;) {
        const int k_side = g >= p.side[0].groups;
        const Side& sd = p.side[k_side];
        const int skip = k_side ? p.side[0].groups : 0, end = k_side ? item.g_end : min(item.g_end, p.side[0].groups);
        const T* x = static_cast<const T*>(sd.x) + item.b * sd.xs[0] + item.t * sd.xs[1];
        T* y = static_cast<T*>(sd.y) + item.b * sd.ys[0] + item.t * sd.ys[1];
        bool weights = false;
        for (; g < end; g += U) {
            RowRaw<T, VEC, NU> raw[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int h = (g - skip + u) * slots + slot;
                load_row(raw[u], x + (g + u < end && h < sd.heads ? h : 0) * sd.xs[2], l);
            }
            if (!turned) {                                             // under the first loads
                int first[NU];
#pragma unroll
                for (int k = 0; k < NU; ++k) first[k] = ((lane & ((1 << p.lanes) - 1)) + (k << p.lanes)) * VEC;
                angles<VEC, NU>(p, position_of(p, item.b, item.t), first, c, s);
                turned = true;
            }
            if (NORM && !weights) {
                load_weights(p, sd, l, w);
                weights = true;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int h = (g - skip + u) * slots + slot;
                float f[NU * 2 * VEC];
                unpack_row<T, VEC, NU>(raw[u], f);
                if (NORM) {
                    float sum = 0.0f;
#pragma unroll
                    for (int k = 0; k < NU; ++k) {
                        float part = 0.0f;
#pragma unroll
                        for (int i = k * 2 * VEC; i < (k + 1) * 2 * VEC; ++i) part = fmaf(f[i], f[i], part);
                        sum += l.here[k] ? part : 0.0f;
                    }
                    const float r = rsqrtf(row_sum(sum, p.lanes) * p.inv_dim + p.eps);
#pragma unroll
                    for (int i = 0; i < NU * 2 * VEC; ++i) f[i] *= r * w[i];
                }
#pragma unroll
                for (int k = 0; k < NU; ++k) turn<VEC, NEIGHBOURS>(f + k * 2 * VEC, c + k * VEC, s + k * VEC, l.turned[k], l.some_still);
                store_row(y + h * sd.ys[2], f, l, g + u < end && h < sd.heads);
            }
        }
        g = end;
    }
}

// Persistent: a warp walks its tokens, the sums for the weights' gradients stay in its lanes, are added over the CTA at the end and leave as
// one binary32 row per CTA, which rotary_weights_kernel adds in a fixed order: no atomics.
template <typename T, int VEC, bool NEIGHBOURS>
__global__ void __launch_bounds__(kThreads) rotary_backward_kernel(const __grid_constant__ RotaryParams p) {
    constexpr int NU = VEC >= 4 ? 1 : 4 / VEC, N = NU * 2 * VEC, U = 2;
    __shared__ float sums[kWarps][2][256];
    if (p.partial) asm volatile("griddepcontrol.launch_dependents;");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Lane<VEC, NU, NEIGHBOURS> l;
    l.place(lane & ((1 << p.lanes) - 1), p.lanes, p.half_rotary, p.dim);
    int first[NU];
#pragma unroll
    for (int k = 0; k < NU; ++k) first[k] = ((lane & ((1 << p.lanes) - 1)) + (k << p.lanes)) * VEC;
    const int slot = lane >> p.lanes, slots = 32 >> p.lanes;
    float acc[2][N];
#pragma unroll
    for (int i = 0; i < N; ++i) acc[0][i] = acc[1][i] = 0.0f;
    for (int64_t index = (int64_t)blockIdx.x * kWarps + warp; index < p.items; index += (int64_t)gridDim.x * kWarps) {
        const Item item = item_of(p, index);
        float c[NU * VEC], s[NU * VEC];
        bool turned = false;
        int g = item.g;
#pragma unroll
        for (int k_side = 0; k_side < 2; ++k_side) {
            const Side& sd = p.side[k_side];
            const int skip = k_side ? p.side[0].groups : 0, end = k_side ? item.g_end : min(item.g_end, p.side[0].groups);
            if (g >= end) continue;
            const T* x = static_cast<const T*>(sd.x) + item.b * sd.xs[0] + item.t * sd.xs[1];
            const T* dy = static_cast<const T*>(sd.dy) + item.b * sd.ds[0] + item.t * sd.ds[1];
            T* dx = static_cast<T*>(sd.y) + item.b * sd.ys[0] + item.t * sd.ys[1];
            float w[N];
            bool weights = false;
            for (; g < end; g += U) {
                RowRaw<T, VEC, NU> rx[U], rd[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int h = (g - skip + u) * slots + slot;
                    const int row = g + u < end && h < sd.heads ? h : 0;
                    load_row(rx[u], x + row * sd.xs[2], l);
                    load_row(rd[u], dy + row * sd.ds[2], l);
                }
                if (!turned) {
                    angles<VEC, NU>(p, position_of(p, item.b, item.t), first, c, s);
                    turned = true;
                }
                if (!weights) {
                    load_weights(p, sd, l, w);
                    weights = true;
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int h = (g - skip + u) * slots + slot;
                    float f[N], d[N];
                    unpack_row<T, VEC, NU>(rx[u], f);
                    unpack_row<T, VEC, NU>(rd[u], d);
#pragma unroll
                    for (int k = 0; k < NU; ++k) turn<VEC, NEIGHBOURS>(d + k * 2 * VEC, c + k * VEC, s + k * VEC, l.turned[k], l.some_still);
                    float sum = 0.0f, along = 0.0f;
#pragma unroll
                    for (int k = 0; k < NU; ++k) {
                        float a = 0.0f, b = 0.0f;
#pragma unroll
                        for (int i = k * 2 * VEC; i < (k + 1) * 2 * VEC; ++i) {
                            a = fmaf(f[i], f[i], a);
                            b = fmaf(d[i] * w[i], f[i], b);
                        }
                        sum += l.here[k] ? a : 0.0f;
                        along += l.here[k] ? b : 0.0f;
                    }
                    for (int o = (1 << p.lanes) >> 1; o > 0; o >>= 1) {
                        sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
                        along += __shfl_xor_sync(0xFFFFFFFFu, along, o);
                    }
                    const float r = rsqrtf(sum * p.inv_dim + p.eps), m = along * r * p.inv_dim;
                    const bool exists = g + u < end && h < sd.heads;
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        const float xh = f[i] * r;
                        if (exists) acc[k_side][i] = fmaf(d[i], xh, acc[k_side][i]);
                        f[i] = r * fmaf(d[i], w[i], -xh * m);
                    }
                    store_row(dx + h * sd.ys[2], f, l, exists);
                }
            }
            g = end;
        }
    }
    if (!p.partial) return;
#pragma unroll
    for (int side = 0; side < 2; ++side)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float v = acc[side][i];
            for (int o = 1 << p.lanes; o < 32; o <<= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
            if (slot == 0 && l.here[i / (2 * VEC)]) sums[warp][side][l.at[i / (2 * VEC)][(i / VEC) & 1] + i % VEC] = v;
        }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * p.dim; i += kThreads) {
        const int side = i >= p.dim, col = i - side * p.dim;
        float v = 0.0f;
#pragma unroll
        for (int k = 0; k < kWarps; ++k) v += sums[k][side][col];
        p.partial[(int64_t)blockIdx.x * 2 * p.dim + i] = v;
    }
}

// Column sums of the CTAs' rows: 8 columns per CTA, 32 threads to a column.
__global__ void __launch_bounds__(256) rotary_weights_kernel(const float* partial, int rows, int dim, void* dq, void* dk, int weight_f32) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    __shared__ float sums[32][9];
    const int col = blockIdx.x * 8 + (threadIdx.x & 7), part = threadIdx.x >> 3;
    float v = 0.0f;
    if (col < 2 * dim) {
#pragma unroll 8
        for (int r = part; r < rows; r += 32) v += partial[(int64_t)r * 2 * dim + col];
    }
    sums[part][threadIdx.x & 7] = v;
    __syncthreads();
    if (threadIdx.x >= 8 || col >= 2 * dim) return;
    v = 0.0f;
#pragma unroll
    for (int k = 0; k < 32; ++k) v += sums[k][threadIdx.x];
    void* out = col < dim ? dq : dk;
    if (!out) return;
    const int c = col < dim ? col : col - dim;
    if (weight_f32) static_cast<float*>(out)[c] = v;
    else static_cast<__nv_bfloat16*>(out)[c] = __float2bfloat16_rn(v);
}

template <typename T, int VEC, bool NB>
cudaError_t run(const RotaryArgs& a, RotaryParams& p, cudaStream_t st) {
    constexpr int NU = VEC >= 4 ? 1 : 4 / VEC;
    const int units = (int)((a.s.head_dim + 2 * VEC - 1) / (2 * VEC));
    p.lanes = 0;
    while ((NU << p.lanes) < units) ++p.lanes;
    const int slots = 32 >> p.lanes;
    for (Side& s : p.side) s.groups = (s.heads + slots - 1) / slots;
    const int64_t rows = a.s.batch * a.s.tokens;
    const int groups = p.side[0].groups + p.side[1].groups;
    // Few tokens: the heads of one are shared out, so that about eight warps per SM have something to do.
    p.parts = (int)std::min<int64_t>(groups, std::max<int64_t>(1, 148 * 8 / rows));
    p.items = rows * p.parts;
    const int64_t ctas = (p.items + kWarps - 1) / kWarps;
    if (ctas > 0x7FFFFFFF) return cudaErrorInvalidConfiguration;
    if (a.op == RotaryArgs::kBackward) {
        const int grid = (int)std::min<int64_t>(ctas, rotary_backward_ctas());
        rotary_backward_kernel<T, VEC, NB><<<grid, kThreads, 0, st>>>(p);
        cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess || !p.partial) return e;
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3((unsigned)((2 * p.dim + 7) / 8));
        cfg.blockDim = dim3(256);
        cfg.stream = st;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        return cudaLaunchKernelEx(&cfg, rotary_weights_kernel, (const float*)p.partial, grid, p.dim, a.dweight[0], a.dweight[1], p.weight_f32);
    }
    if (a.op == RotaryArgs::kNorm) rotary_kernel<T, VEC, NB, true><<<(unsigned)ctas, kThreads, 0, st>>>(p);
    else rotary_kernel<T, VEC, NB, false><<<(unsigned)ctas, kThreads, 0, st>>>(p);
    return cudaGetLastError();
}
template <typename T, int VEC>
cudaError_t run(const RotaryArgs& a, RotaryParams& p, cudaStream_t st) {
    return a.s.interleaved ? run<T, VEC, true>(a, p, st) : run<T, VEC, false>(a, p, st);
}

}  // namespace

int rotary_backward_ctas() { return 148 * 4; }

cudaError_t launch_rotary(const RotaryArgs& a, cudaStream_t st) {
    const ue5m3_rotary_shape& s = a.s;
    const int64_t size = s.dtype == UE5M3_BF16 ? 2 : 4;
    RotaryParams p{};
    uint64_t bits = 0;                                     // of every address and stride, in elements
    for (int k = 0; k < 2; ++k) {
        const RotaryArgs::Tensors& t = a.side[k];
        Side& d = p.side[k];
        d.heads = (int)(k ? s.kv_heads : s.heads);
        if (d.heads == 0) {                                // no keys: addresses that nothing is read from
            d = p.side[0];
            d.heads = 0;
            d.weight = nullptr;
            continue;
        }
        auto take = [&](const ue5m3_heads& h, int64_t (&strides)[3]) {
            const int64_t all[3] = {s.batch > 1 ? h.batch_stride : 0, s.tokens > 1 ? h.token_stride : 0, d.heads > 1 ? h.head_stride : 0};
            bits |= reinterpret_cast<uintptr_t>(h.data) / (uint64_t)size;
            for (int i = 0; i < 3; ++i) { strides[i] = all[i]; bits |= (uint64_t)all[i]; }
            return h.data;
        };
        d.x = take(t.x, d.xs);
        d.y = take(t.y, d.ys);
        if (a.op == RotaryArgs::kBackward) d.dy = take(t.dy, d.ds);
        d.weight = a.weight[k];
    }
    p.frequencies = s.frequencies;
    p.positions = s.positions;
    p.position_stride = s.position_stride;
    p.first_position = s.first_position;
    p.tokens = s.tokens;
    p.wide_positions = s.position_bytes == 8;
    p.half_rotary = (int)(s.rotary_dim / 2);
    p.dim = (int)s.head_dim;
    p.weight_f32 = a.weight_dtype == UE5M3_F32;
    p.amplitude = s.amplitude;
    p.eps = a.eps;
    p.inv_dim = 1.0f / (float)s.head_dim;
    p.sign = a.inverse ? -1.0f : 1.0f;
    p.partial = a.partial;
    // The largest vector that the addresses allow and that no row's end, and of halves no pair's end, cuts.
    bits |= (uint64_t)s.head_dim / 2;
    if (!s.interleaved) bits |= (uint64_t)p.half_rotary;
    const int vec = (int)(bits & (0 - bits) & 7) ? (int)(bits & (0 - bits)) : 8;
    if (s.dtype == UE5M3_BF16) {
        if (vec >= 8) return run<__nv_bfloat16, 8>(a, p, st);
        if (vec == 4) return run<__nv_bfloat16, 4>(a, p, st);
        if (vec == 2) return run<__nv_bfloat16, 2>(a, p, st);
        return run<__nv_bfloat16, 1>(a, p, st);
    }
    if (vec >= 4) return run<float, 4>(a, p, st);
    if (vec == 2) return run<float, 2>(a, p, st);
    return run<float, 1>(a, p, st);
}

}  // namespace ue5m3
