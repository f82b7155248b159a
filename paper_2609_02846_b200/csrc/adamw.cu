// AdamW step over many tensors in one launch, moments in binary32 or in 8 bits (sm_100a).
//
//   m' = b1 m + (1 - b1) g,   v' = b2 v + (1 - b2) g^2,   w' = w (1 - lr wd) - lr / (1 - b1^t) m' / (sqrt(v' / (1 - b2^t)) + eps)
//
// m' and v' are made of single binary32 roundings in the order written (products, then the sum), so that the codes of 8-bit moments are
// defined to the bit.  w' takes a fused product and approximate root and reciprocal.  The update, itself of the size lr, is off by at most 2^-21 of it where
// v' / (1 - b2^t) is a normal number: bias correction and its product, each halved by the root, 2^-24 together, root 2^-23, sum 2^-24, reciprocal 2^-23, its
// product 2^-24, step size 2^-24 (a subnormal product adds its own rounding); the weight's factor and its product by 2^-24 each, and w' is rounded once more.
//
// 8-bit moments: blocks of 256 elements share a binary32 scale; m is a sign and E4M3, v unsigned E5M3 (the format of the FP4 block
// scales: a moment that is never negative needs no sign, and v spans the square of m's range).  A block's largest magnitude gets the format's largest value.  Both are
// rounded up with the probability of their place between two codes: with b2 near 1 a step changes v by less than half of the 6 to 12 % between
// two codes, and rounding to nearest would leave v where it is for ever.  As in the FP4 quantizer, a product with a power of two moves
// the format's subnormal values onto those of binary32; the code then is the bits from 20 up, and the draw is added below them.
// A positive v' never gets the code 0: an m next to it would be divided by eps alone in the next step.
//
// Bound by memory: 28 bytes per element with binary32 moments (weight read and written, gradient, two moments; or BF16 weight, copy in binary32,
// BF16 gradient): 176 M weights in 713 us, 6.9 TB/s.  16 bytes with 8-bit ones: 462 us, 6.1 TB/s (0.93 of the measured copy rate) at 75
// instructions per element, in 0.79 of the SMs' issue slots.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <cmath>
#include <cstdint>
#include "../../include/ue5m3.h"
#include "block_ops.h"
#include "common.cuh"

namespace ue5m3 {
namespace {

// A warp has a block of 256 elements, a lane 8 of them.  8-bit moments want as many warps as there are (64 registers, 32 warps per SM: us for 176 M weights
// with 16 CTAs of 64 threads 460, with 14 485, 12 514; 8 of 128 464, 4 of 256 566) and, in CTAs of their own chunks only, 495.
constexpr int kThreads = 64, kChunk = kThreads * 8, kRounds = 4;

struct Clock { long long step; float step_size, inv_bias2; };          // lies in the caller's memory
static_assert(sizeof(Clock) <= UE5M3_ADAMW_CLOCK_BYTES, "");

struct AdamwParams {
    float b1, c1, b2, c2;                                  // c = 1 - b
    float keep, step_size, inv_bias2, eps;                 // 1 - lr wd, lr / (1 - b1^t), 1 / (1 - b2^t)
    const float* grad_scale;
    const Clock* clock;                                    // null: step_size, inv_bias2 and step are those here
    uint32_t step;
    int count, rounds;                                     // tensors; chunks that a CTA takes
    PhiloxKeys keys;
};
// Tensors travel as launch parameters: nothing to copy, nothing that outlives the call.  Two sizes, since a launch pays for its parameters' bytes.
template <int MAX> struct AdamwTensors {
    ue5m3_adamw_tensor t[MAX];
    uint32_t first[MAX];                                   // first CTA of each tensor
};
constexpr int kFew = 40, kMany = 400;

__device__ __forceinline__ float at_f32(const void* p, int64_t i) { return static_cast<const float*>(p)[i]; }
__device__ __forceinline__ float at_bf16(const void* p, int64_t i) { return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]); }

// Elements i .. i + 7 (`n` of them exist, the others are zero) in binary32, one by one.
__device__ __forceinline__ void load8(float (&f)[8], const void* p, bool f32, int64_t i, int n) {
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
__device__ __forceinline__ uint2 load_codes(const void* p, int64_t i, int n) {
    const uint8_t* c = static_cast<const uint8_t*>(p) + i;
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

// Values of four codes in units of their block's scale.  E4M3 has a conversion; a UE5M3 code is the upper byte of a positive FP16, one bit
// down.
__device__ __forceinline__ void values_m(uint32_t codes, float* f) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t v;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(v) : "h"((unsigned short)(codes >> (16 * h))));
        const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&v));
        f[2 * h] = x.x;
        f[2 * h + 1] = x.y;
    }
}
__device__ __forceinline__ void values_v(uint32_t codes, float* f) {
    const uint32_t even = (codes & 0x00FF00FFu) << 7, odd = (codes >> 1) & 0x7F807F80u;
    const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&even)), y = __half22float2(*reinterpret_cast<const __half2*>(&odd));
    f[0] = x.x; f[1] = y.x; f[2] = x.y; f[3] = y.y;
}

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
// |x| up, moved to the bottom of the binary32 range and rounded by the low (HIGH: high) 16 bits of `draw`: bits 20.. are the code.
template <bool HIGH> __device__ __forceinline__ uint32_t rounded(float x, float up, float low, uint32_t draw) {
    return dp2a_lo_u32(draw, HIGH ? 0x1000u : 0x0010u, __float_as_uint(__fmul_rn(__fmul_rn(fabsf(x), up), low)) + 8u);
}
// The codes of two elements in the upper bytes of two words.  m and v share 16 bits of draws, the bytes exchanged for m: each is uniform, so each code is right on
// average; together they are not independent (a draw's high byte is the other one's low byte: a correlation of 512 / 65537 = 0.008), which nothing asks for.
__device__ __forceinline__ void encode_m(const float* x, float up, uint32_t draw, uint32_t* out) {
    const uint32_t most = (0x7Eu << 20) | 0xFFFFFu;
    const uint32_t turned = __byte_perm(draw, 0, 0x2301);          // v's bits with the bytes of each half exchanged
    out[0] = min(rounded<false>(x[0], up, kMinM, turned), most) << 4;
    out[1] = min(rounded<true>(x[1], up, kMinM, turned), most) << 4;
#pragma unroll
    for (int k = 0; k < 2; ++k) out[k] = (out[k] & 0x7FFFFFFFu) | (__float_as_uint(x[k]) & 0x80000000u);
}
__device__ __forceinline__ void encode_v(const float* x, float up, uint32_t draw, uint32_t* out) {
    const uint32_t most = (0xF7u << 20) | 0xFFFFFu;
    out[0] = min(rounded<false>(x[0], up, kMinV, draw), most);
    out[1] = min(rounded<true>(x[1], up, kMinV, draw), most);
#pragma unroll
    for (int k = 0; k < 2; ++k) out[k] = (x[k] > 0.0f ? max(out[k], 1u << 20) : out[k]) << 4;
}
__device__ __forceinline__ uint32_t upper_bytes(const uint32_t* w) {   // of four words
    return __byte_perm(__byte_perm(w[0], w[1], 0x0073), __byte_perm(w[2], w[3], 0x0073), 0x5410);
}
__device__ __forceinline__ float max_nan(float a, float b) {            // a NaN wins
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float warp_max(float v) {       // of magnitudes; NaN is above all
    return __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(v)));
}
// m / (sqrt(v) + eps).  FLUSH: v below 2^-126 counts as zero in the root, which beside an eps of kFlushEps or more is 2^-23 of the sum.  Else it counts as what
// it is (an eps of 0 is allowed, and then the root is all there is); the sum is 0 or a normal number, since an eps is.
constexpr float kFlushEps = 0x1p-40f;
template <bool FLUSH> __device__ __forceinline__ float quotient(float m, float v, float eps) {
    float root, inverse;
    if constexpr (FLUSH) asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(root) : "f"(v));
    else asm("sqrt.approx.f32 %0, %1;" : "=f"(root) : "f"(v));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inverse) : "f"(root + eps));
    return m * inverse;
}

// What a thread reads of eight elements, as it lies in memory.
template <bool EIGHT> struct Read {
    uint4 g[2], w[2];                                      // BF16: the first one
    uint4 m[EIGHT ? 1 : 2], v[EIGHT ? 1 : 2];              // 8 bits: two words
    float sm, sv;
    __device__ __forceinline__ void load(const ue5m3_adamw_tensor& t, int64_t i) {
        const bool grad_f32 = t.grad_dtype == UE5M3_F32, weight_f32 = t.master || t.param_dtype == UE5M3_F32;
        const uint4* pg = reinterpret_cast<const uint4*>(static_cast<const char*>(t.grad) + i * (grad_f32 ? 4 : 2));
        const uint4* pw = reinterpret_cast<const uint4*>((t.master ? reinterpret_cast<const char*>(t.master) : static_cast<const char*>(t.param)) + i * (weight_f32 ? 4 : 2));
        g[0] = pg[0];
        if (grad_f32) g[1] = pg[1];
        w[0] = pw[0];
        if (weight_f32) w[1] = pw[1];
        if constexpr (EIGHT) {
            const uint2 a = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(t.m) + i), b = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(t.v) + i);
            m[0].x = a.x; m[0].y = a.y;
            v[0].x = b.x; v[0].y = b.y;
            sm = t.m_scale[i >> 8];
            sv = t.v_scale[i >> 8];
        } else {
            m[0] = reinterpret_cast<const uint4*>(static_cast<const float*>(t.m) + i)[0];
            m[1] = reinterpret_cast<const uint4*>(static_cast<const float*>(t.m) + i)[1];
            v[0] = reinterpret_cast<const uint4*>(static_cast<const float*>(t.v) + i)[0];
            v[1] = reinterpret_cast<const uint4*>(static_cast<const float*>(t.v) + i)[1];
        }
    }
    static __device__ __forceinline__ void numbers(const uint4* x, bool f32, float (&f)[8]) {
        if (f32) {
            f[0] = __uint_as_float(x[0].x); f[1] = __uint_as_float(x[0].y); f[2] = __uint_as_float(x[0].z); f[3] = __uint_as_float(x[0].w);
            f[4] = __uint_as_float(x[1].x); f[5] = __uint_as_float(x[1].y); f[6] = __uint_as_float(x[1].z); f[7] = __uint_as_float(x[1].w);
        } else {
            unpack_bf16x8(x[0], f);
        }
    }
};

// A CTA takes `rounds` chunks in a row of one tensor (all / gridDim: the last CTA of a tensor fewer).  What the next chunk needs is loaded
// under this one's arithmetic.
template <bool EIGHT, int MAX>
__global__ void __launch_bounds__(kThreads, EIGHT ? 16 : 12) adamw_kernel(const __grid_constant__ AdamwParams p, const __grid_constant__ AdamwTensors<MAX> all) {
    int lo = 0, hi = p.count;                              // the tensor whose CTAs begin at or before this one
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (all.first[mid] <= blockIdx.x) lo = mid;
        else hi = mid;
    }
    const ue5m3_adamw_tensor& t = all.t[lo];
    int64_t i = (int64_t)(blockIdx.x - all.first[lo]) * p.rounds * kChunk + threadIdx.x * 8;
    const int64_t end = min(t.n, (int64_t)(blockIdx.x - all.first[lo] + 1) * p.rounds * kChunk);
    const bool grad_f32 = t.grad_dtype == UE5M3_F32, param_f32 = t.param_dtype == UE5M3_F32, aligned = t.reserved != 0;
    const bool weight_f32 = t.master || param_f32;
    Read<EIGHT> next;
    if (aligned && i + 8 <= end) next.load(t, i);
    float step_size = p.step_size, inv_bias2 = p.inv_bias2, grad_scale = 1.0f;
    uint32_t step = p.step;
    if (p.clock) {
        step_size = p.clock->step_size;
        inv_bias2 = p.clock->inv_bias2;
        step = (uint32_t)p.clock->step;
    }
    if (p.grad_scale) {
        grad_scale = *p.grad_scale;
        if (!(fabsf(grad_scale) < INFINITY)) return;       // a step to be left out
    }
#pragma unroll 1
    for (; (i & ~(int64_t)255) < end; i += kChunk) {       // whole warps: a block of 256 each
        const int n = (int)min((int64_t)8, max((int64_t)0, end - i));
        const bool whole = n == 8 && aligned;
        float g[8], w[8], m[8], v[8];
        if (whole) {
            Read<EIGHT>::numbers(next.g, grad_f32, g);
            Read<EIGHT>::numbers(next.w, weight_f32, w);
            if constexpr (EIGHT) {
                values_m(next.m[0].x, m); values_m(next.m[0].y, m + 4);
                values_v(next.v[0].x, v); values_v(next.v[0].y, v + 4);
#pragma unroll
                for (int j = 0; j < 8; ++j) { m[j] = __fmul_rn(m[j], next.sm); v[j] = __fmul_rn(v[j], next.sv); }
            } else {
                Read<EIGHT>::numbers(next.m, true, m);
                Read<EIGHT>::numbers(next.v, true, v);
            }
        } else {
            load8(g, t.grad, grad_f32, i, n);
            load8(w, t.master ? static_cast<const void*>(t.master) : t.param, weight_f32, i, n);
            if constexpr (EIGHT) {
                const uint2 cm = load_codes(t.m, i, n), cv = load_codes(t.v, i, n);
                const float sm = t.m_scale[i >> 8], sv = t.v_scale[i >> 8];
                values_m(cm.x, m); values_m(cm.y, m + 4);
                values_v(cv.x, v); values_v(cv.y, v + 4);
#pragma unroll
                for (int j = 0; j < 8; ++j) { m[j] = __fmul_rn(m[j], sm); v[j] = __fmul_rn(v[j], sv); }
            } else {
                load8(m, t.m, true, i, n);
                load8(v, t.v, true, i, n);
            }
        }
        if (aligned && i + kChunk + 8 <= end) next.load(t, i + kChunk);
        if (p.grad_scale) {
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] = __fmul_rn(g[j], grad_scale);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            m[j] = __fadd_rn(__fmul_rn(m[j], p.b1), __fmul_rn(g[j], p.c1));
            v[j] = __fadd_rn(__fmul_rn(v[j], p.b2), __fmul_rn(__fmul_rn(g[j], p.c2), g[j]));
        }
        // (8 bits have no issue slots to spare: 462 us with the flushing root, 467 with the other one; 32 bits are bound by memory, 716 with both)
        if (EIGHT && p.eps >= kFlushEps) {
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = fmaf(-step_size, quotient<true>(m[j], v[j] * inv_bias2, p.eps), w[j] * p.keep);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = fmaf(-step_size, quotient<false>(m[j], v[j] * inv_bias2, p.eps), w[j] * p.keep);
        }
        if (t.master) store8(w, t.master, true, i, n, whole);
        store8(w, t.param, param_f32, i, n, whole);
        if constexpr (!EIGHT) {
            store8(m, t.m, true, i, n, whole);
            store8(v, t.v, true, i, n, whole);
        } else {
            float top_m = 0.0f, top_v = 0.0f;              // (elements behind the end are zeros)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                top_m = max_nan(top_m, fabsf(m[j]));
                top_v = max_nan(top_v, v[j]);
            }
            const BlockScale bm = block_scale_of(warp_max(top_m), kTopM), bv = block_scale_of(warp_max(top_v), kTopV);
            uint32_t draw[4];
            philox4x32((uint32_t)(i >> 3), t.stream, 2u, step, p.keys, draw);
            uint32_t out_m[8], out_v[8];
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                encode_m(m + j, bm.up, draw[j >> 1], out_m + j);
                encode_v(v + j, bv.up, draw[j >> 1], out_v + j);
            }
            const uint32_t keep_m = bm.up == 0.0f ? 0u : 0xFFFFFFFFu, keep_v = bv.up == 0.0f ? 0u : 0xFFFFFFFFu;      // a block stored as zeros
            store_codes(make_uint2(upper_bytes(out_m) & keep_m, upper_bytes(out_m + 4) & keep_m), t.m, i, n, whole);
            store_codes(make_uint2(upper_bytes(out_v) & keep_v, upper_bytes(out_v + 4) & keep_v), t.v, i, n, whole);
            if ((threadIdx.x & 31) == 0) {
                t.m_scale[i >> 8] = bm.scale;
                t.v_scale[i >> 8] = bv.scale;
            }
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
    int64_t chunks = 0, ctas = 0;
    for (int i = 0; i < count; ++i) chunks += (tensors[i].n + kChunk - 1) / kChunk;
    // Several chunks in a row where that still leaves every SM twice the CTAs it holds: the next chunk is loaded under this one's arithmetic, which
    // moments of 8 bits have much of (32 bits: 713 us either way).
    p.rounds = bits == 8 && chunks >= 148 * 16 * 2 * kRounds ? kRounds : 1;
    int k = 0;
    for (int i = 0; i < count; ++i) {
        if (tensors[i].n == 0) continue;
        ue5m3_adamw_tensor& t = all.t[k];
        t = tensors[i];
        const uintptr_t a = reinterpret_cast<uintptr_t>(t.param) | reinterpret_cast<uintptr_t>(t.grad) | reinterpret_cast<uintptr_t>(t.master);
        const uintptr_t b = reinterpret_cast<uintptr_t>(t.m) | reinterpret_cast<uintptr_t>(t.v);
        t.reserved = (a & 15) == 0 && (b & (bits == 8 ? 7 : 15)) == 0;
        all.first[k++] = (uint32_t)ctas;
        ctas += (t.n + p.rounds * kChunk - 1) / (p.rounds * kChunk);
    }
    if (k == 0) return cudaSuccess;
    p.count = k;
    if (ctas > 0x7FFFFFFF) return cudaErrorInvalidConfiguration;
    if (bits == 8) adamw_kernel<true, MAX><<<(unsigned)ctas, kThreads, 0, st>>>(p, all);
    else adamw_kernel<false, MAX><<<(unsigned)ctas, kThreads, 0, st>>>(p, all);
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
