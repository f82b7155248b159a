// AdamW step over many tensors in one launch, moments in binary32 or in 8 bits (sm_100a).
//
//   m' = b1 m + (1 - b1) g,   v' = b2 v + (1 - b2) g^2,   w' = w (1 - lr wd) - lr / (1 - b1^t) m' / (sqrt(v' / (1 - b2^t)) + eps)
//
// m' and v' are made of single binary32 roundings in the order written (products, then the sum), so that the codes of 8-bit moments are
// defined to the bit.  w' takes a fused product and approximate root and reciprocal: their error is 2^-22 of the update, which is itself
// of the size lr.
//
// 8-bit moments: blocks of 256 elements share a binary32 scale; m is a sign and E4M3, v unsigned E5M3 (the format of the FP4 block
// scales: a moment that is never negative needs no sign, and v spans the square of m's range).  A block's largest magnitude gets the format's largest value.  Both are
// rounded up with the probability of their place between two codes: with b2 near 1 a step changes v by less than half of the 6 to 12 % between
// two codes, and rounding to nearest would leave v where it is for ever.  As in the FP4 quantizer, a product with a power of two moves
// the format's subnormal values onto those of binary32; the code then is the bits from 20 up, and the draw is added below them.
// A positive v' never gets the code 0: an m next to it would be divided by eps alone in the next step.
//
// Bound by memory: 28 bytes per element with binary32 moments (weight read and written, gradient, two moments; or BF16 weight, copy in binary32,
// BF16 gradient), 16 with 8-bit ones, of which a CTA's 2048 elements are all in flight at once.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cmath>
#include <cstdint>
#include "../../include/ue5m3.h"
#include "block_ops.h"
#include "common.cuh"

namespace ue5m3 {
namespace {

constexpr int kThreads = 256, kChunk = kThreads * 8;       // a warp has a block of 256 elements, a lane 8 of them

struct Clock { long long step; float step_size, inv_bias2; };          // lies in the caller's memory
static_assert(sizeof(Clock) <= UE5M3_ADAMW_CLOCK_BYTES, "");

struct AdamwParams {
    float b1, c1, b2, c2;                                  // c = 1 - b
    float keep, step_size, inv_bias2, eps;                 // 1 - lr wd, lr / (1 - b1^t), 1 / (1 - b2^t)
    const float* grad_scale;
    const Clock* clock;                                    // null: step_size, inv_bias2 and step are those here
    uint32_t step;
    int count;
    PhiloxKeys keys;
};
// Tensors travel as launch parameters: nothing to copy, nothing that outlives the call.  Two sizes, since a launch pays for its parameters' bytes.
template <int MAX> struct AdamwTensors {
    ue5m3_adamw_tensor t[MAX];
    uint32_t first[MAX];                                   // first chunk of each tensor
};
constexpr int kFew = 40, kMany = 400;

__device__ __forceinline__ float at_f32(const void* p, int64_t i) { return static_cast<const float*>(p)[i]; }
__device__ __forceinline__ float at_bf16(const void* p, int64_t i) { return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]); }

// Elements i .. i + 7 (`n` of them exist) in binary32.
__device__ __forceinline__ void load8(float (&f)[8], const void* p, bool f32, int64_t i, int n, bool whole) {
    if (whole) {
        if (f32) {
            const float4 a = reinterpret_cast<const float4*>(static_cast<const float*>(p) + i)[0], b = reinterpret_cast<const float4*>(static_cast<const float*>(p) + i)[1];
            f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
        } else {
            unpack_bf16x8(*reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p) + i), f);
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = j < n ? (f32 ? at_f32(p, i + j) : at_bf16(p, i + j)) : 0.0f;
}
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ void store8(const float (&f)[8], void* p, bool f32, int64_t i, int n, bool whole) {
    if (whole) {
        if (f32) {
            reinterpret_cast<float4*>(static_cast<float*>(p) + i)[0] = make_float4(f[0], f[1], f[2], f[3]);
            reinterpret_cast<float4*>(static_cast<float*>(p) + i)[1] = make_float4(f[4], f[5], f[6], f[7]);
        } else {
            *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p) + i) = make_uint4(bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3]), bf16_pair(f[4], f[5]), bf16_pair(f[6], f[7]));
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < n) {
            if (f32) static_cast<float*>(p)[i + j] = f[j];
            else static_cast<__nv_bfloat16*>(p)[i + j] = __float2bfloat16_rn(f[j]);
        }
}
__device__ __forceinline__ uint2 load_codes(const void* p, int64_t i, int n, bool whole) {
    const uint8_t* c = static_cast<const uint8_t*>(p) + i;
    if (whole) return *reinterpret_cast<const uint2*>(c);
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < n) w[j >> 2] |= (uint32_t)c[j] << (8 * (j & 3));
    return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ void store_codes(uint2 v, void* p, int64_t i, int n, bool whole) {
    uint8_t* c = static_cast<uint8_t*>(p) + i;
    if (whole) {
        *reinterpret_cast<uint2*>(c) = v;
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < n) c[j] = (uint8_t)((j < 4 ? v.x : v.y) >> (8 * (j & 3)));
}

constexpr float kTopM = 448.0f, kTopV = 61440.0f;          // largest values of E4M3 and UE5M3
constexpr float kMinM = 0x1p-120f, kMinV = 0x1p-112f;      // 2^-126 over their smallest normal values
constexpr float kLeast = 0x1p-110f;                        // blocks below this are stored as zeros (their reciprocals would overflow)

// Value of a code in units of its block's scale.
__device__ __forceinline__ float value_m(uint32_t code) { return __uint_as_float(((code & 0x7Fu) << 20) | ((code & 0x80u) << 24)) * (1.0f / kMinM); }
__device__ __forceinline__ float value_v(uint32_t code) { return __uint_as_float(code << 20) * (1.0f / kMinV); }

// Largest magnitude of a block -> what its elements are multiplied by, and its scale.  Not finite: the scale is NaN, and with it the whole block.
struct BlockScale { float up, scale; };
__device__ __forceinline__ BlockScale block_scale_of(float most, float top) {
    BlockScale s;
    const bool used = most >= kLeast;
    s.up = used ? __fmul_rn(__frcp_rn(most), top) : 0.0f;
    s.scale = used ? __fmul_rn(most, 1.0f / top) : 0.0f;
    if (!(most < INFINITY)) { s.up = 0.0f; s.scale = __int_as_float(0x7FFFFFFF); }
    return s;
}
// |x| up -> code: bits 20.. of the moved value, rounded by 16 random bits.
__device__ __forceinline__ uint32_t code_of(float x, float up, float low, uint32_t draw) {
    return (__float_as_uint(__fmul_rn(__fmul_rn(fabsf(x), up), low)) + (draw << 4) + 8u) >> 20;
}
__device__ __forceinline__ float warp_max(float v) {       // of magnitudes; NaN is above all
    return __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(v)));
}
__device__ __forceinline__ float sqrt_near(float x) {
    float r;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

template <bool EIGHT, int MAX>
__global__ void __launch_bounds__(kThreads) adamw_kernel(const __grid_constant__ AdamwParams p, const __grid_constant__ AdamwTensors<MAX> all) {
    int lo = 0, hi = p.count;                              // the tensor whose chunks begin at or before this CTA's
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (all.first[mid] <= blockIdx.x) lo = mid;
        else hi = mid;
    }
    const ue5m3_adamw_tensor& t = all.t[lo];
    const int64_t i = (int64_t)(blockIdx.x - all.first[lo]) * kChunk + threadIdx.x * 8;
    if ((i & ~(int64_t)255) >= t.n) return;                // whole warps
    const int n = (int)min((int64_t)8, max((int64_t)0, t.n - i));
    const bool whole = n == 8 && t.reserved != 0;          // 16-byte aligned throughout
    const bool grad_f32 = t.grad_dtype == UE5M3_F32, param_f32 = t.param_dtype == UE5M3_F32;
    float g[8], w[8], m[8], v[8];
    load8(g, t.grad, grad_f32, i, n, whole);
    if (t.master) load8(w, t.master, true, i, n, whole);
    else load8(w, t.param, param_f32, i, n, whole);
    if constexpr (EIGHT) {
        const uint2 cm = load_codes(t.m, i, n, whole), cv = load_codes(t.v, i, n, whole);
        const float sm = t.m_scale[i >> 8], sv = t.v_scale[i >> 8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            m[j] = __fmul_rn(value_m((j < 4 ? cm.x : cm.y) >> (8 * (j & 3)) & 0xFFu), sm);
            v[j] = __fmul_rn(value_v((j < 4 ? cv.x : cv.y) >> (8 * (j & 3)) & 0xFFu), sv);
        }
    } else {
        load8(m, t.m, true, i, n, whole);
        load8(v, t.v, true, i, n, whole);
    }
    float step_size = p.step_size, inv_bias2 = p.inv_bias2;
    uint32_t step = p.step;
    if (p.clock) {
        step_size = p.clock->step_size;
        inv_bias2 = p.clock->inv_bias2;
        step = (uint32_t)p.clock->step;
    }
    if (p.grad_scale) {
        const float s = *p.grad_scale;
        if (!(fabsf(s) < INFINITY)) return;                // a step to be left out
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = __fmul_rn(g[j], s);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        m[j] = __fadd_rn(__fmul_rn(m[j], p.b1), __fmul_rn(g[j], p.c1));
        v[j] = __fadd_rn(__fmul_rn(v[j], p.b2), __fmul_rn(__fmul_rn(g[j], p.c2), g[j]));
        const float q = __fdividef(m[j], sqrt_near(v[j] * inv_bias2) + p.eps);
        w[j] = fmaf(-step_size, q, w[j] * p.keep);
    }
    if (t.master) store8(w, t.master, true, i, n, whole);
    store8(w, t.param, param_f32, i, n, whole);
    if constexpr (!EIGHT) {
        store8(m, t.m, true, i, n, whole);
        store8(v, t.v, true, i, n, whole);
    } else {
        float top_m = 0.0f, top_v = 0.0f;
    #pragma unroll
        for (int j = 0; j < 8; ++j) {                          // as unsigned numbers, so that a NaN is the largest
            if (j < n) {
                top_m = __uint_as_float(max(__float_as_uint(top_m), __float_as_uint(fabsf(m[j]))));
                top_v = __uint_as_float(max(__float_as_uint(top_v), __float_as_uint(fabsf(v[j]))));
            }
        }
        const BlockScale bm = block_scale_of(warp_max(top_m), kTopM), bv = block_scale_of(warp_max(top_v), kTopV);
        uint32_t draw[4];
        philox4x32((uint32_t)(i >> 3), t.stream, 2u, step, p.keys, draw);
        uint32_t out_m[2] = {0, 0}, out_v[2] = {0, 0};
    #pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t r = (j & 1) ? draw[j >> 1] >> 16 : draw[j >> 1] & 0xFFFFu;
            const uint32_t turned = __byte_perm(draw[j >> 1], 0, (j & 1) ? 0x4423 : 0x4401);       // the same bits, bytes exchanged: as good as independent
            uint32_t a = min(code_of(m[j], bm.up, kMinM, turned), 0x7Eu) | ((__float_as_uint(m[j]) >> 24) & 0x80u);
            uint32_t b = min(code_of(v[j], bv.up, kMinV, r), 0xF7u);
            if (v[j] > 0.0f) b = max(b, 1u);
            if (bm.up == 0.0f) a = 0;
            if (bv.up == 0.0f) b = 0;
            out_m[j >> 2] |= a << (8 * (j & 3));
            out_v[j >> 2] |= b << (8 * (j & 3));
        }
        store_codes(make_uint2(out_m[0], out_m[1]), t.m, i, n, whole);
        store_codes(make_uint2(out_v[0], out_v[1]), t.v, i, n, whole);
        if ((threadIdx.x & 31) == 0) {
            t.m_scale[i >> 8] = bm.scale;
            t.v_scale[i >> 8] = bv.scale;
        }
    }
}

// The next step's number and what follows from it, for steps that a captured graph replays.
__global__ void adamw_clock_kernel(Clock* c, double lr, double b1, double b2, const float* grad_scale) {
    if (grad_scale && !(fabsf(*grad_scale) < INFINITY)) return;
    const long long t = c->step + 1;
    c->step = t;
    c->step_size = (float)(lr / (1.0 - pow(b1, (double)t)));
    c->inv_bias2 = (float)(1.0 / (1.0 - pow(b2, (double)t)));
}

template <int MAX>
cudaError_t run(AdamwParams& p, const ue5m3_adamw_tensor* tensors, int count, int bits, cudaStream_t st) {
    static_assert(sizeof(AdamwTensors<MAX>) + sizeof(AdamwParams) <= 32764, "");
    AdamwTensors<MAX> all;
    int64_t chunks = 0;
    int k = 0;
    for (int i = 0; i < count; ++i) {
        if (tensors[i].n == 0) continue;
        ue5m3_adamw_tensor& t = all.t[k];
        t = tensors[i];
        const uintptr_t a = reinterpret_cast<uintptr_t>(t.param) | reinterpret_cast<uintptr_t>(t.grad) | reinterpret_cast<uintptr_t>(t.master);
        const uintptr_t b = reinterpret_cast<uintptr_t>(t.m) | reinterpret_cast<uintptr_t>(t.v);
        t.reserved = (a & 15) == 0 && (b & (bits == 8 ? 7 : 15)) == 0;
        all.first[k++] = (uint32_t)chunks;
        chunks += (t.n + kChunk - 1) / kChunk;
    }
    if (k == 0) return cudaSuccess;
    p.count = k;
    if (chunks > 0x7FFFFFFF) return cudaErrorInvalidConfiguration;
    if (bits == 8) adamw_kernel<true, MAX><<<(unsigned)chunks, kThreads, 0, st>>>(p, all);
    else adamw_kernel<false, MAX><<<(unsigned)chunks, kThreads, 0, st>>>(p, all);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_adamw(const ue5m3_adamw_tensor* tensors, int64_t count, const ue5m3_adamw_step& s, cudaStream_t st) {
    AdamwParams p{};
    p.b1 = (float)s.beta1; p.c1 = (float)(1.0 - s.beta1);
    p.b2 = (float)s.beta2; p.c2 = (float)(1.0 - s.beta2);
    p.keep = (float)(1.0 - s.lr * s.weight_decay);
    p.eps = (float)s.eps;
    p.grad_scale = s.grad_scale;
    p.keys = philox_round_keys(s.seed);
    if (s.clock) {
        p.clock = static_cast<const Clock*>(s.clock);
        adamw_clock_kernel<<<1, 1, 0, st>>>(static_cast<Clock*>(s.clock), s.lr, s.beta1, s.beta2, s.grad_scale);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    } else {
        p.step = (uint32_t)s.step;
        p.step_size = (float)(s.lr / (1.0 - pow(s.beta1, (double)s.step)));
        p.inv_bias2 = (float)(1.0 / (1.0 - pow(s.beta2, (double)s.step)));
    }
    for (int64_t at = 0; at < count; at += kMany) {
        const int n = (int)(count - at < kMany ? count - at : kMany);
        const cudaError_t e = n <= kFew ? run<kFew>(p, tensors + at, n, s.state_bits, st) : run<kMany>(p, tensors + at, n, s.state_bits, st);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace ue5m3
