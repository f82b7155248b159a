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
// neighbouring pairs), 32 / G heads side by side (a group), and the warp walks its groups, a few at a time, with a lane's pairs, and so its
// angles and weights, staying the same.  VEC is 4 pairs where the addresses allow it and no pair's end cuts a vector, else 2 or 1 (8 pairs of BF16 in a lane
// were slower: half of the lanes' rows side by side, twice the registers).  The next rows are loaded under the arithmetic, the first ones under the angles.  A
// token's sines and cosines are computed once, by all lanes, and read from shared memory (each lane for itself: a third of all instructions).  The norm's sum over
// a row is log2(G) shuffles.  A ring of asynchronous copies in shared memory in place of registers was slower (47 us): the arithmetic's own
// latency is what counts, not the bytes in flight.  Where there are few tokens the heads of one are shared out among warps.
//
// GPU time, of which the floor at the measured copy rate: rotation of 4 x 4096 tokens, 32 + 8 heads of 128, BF16 54.8 us (0.93 of it); norm and rotation
// of 2 x 4096 30.5 (0.84); backward of 4 x 4096 97 (0.79), bound by the latency of a row's chain at 12 warps per SM.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <algorithm>
#include <cstdint>
#include "../../include/ue5m3.h"
#include "block_ops.h"
#include "common.cuh"
#include "tcgen05.cuh"

namespace ue5m3 {
namespace {

constexpr int kThreads = 128, kWarps = kThreads / 32;
// Groups that a warp works on at a time, and CTAs per SM (backward: of a persistent grid).  Rows side by side hide the latency of the norm's chain (sum,
// shuffles, root), more warps do too, and both want registers.  Norm and rotation of 2 x 4096 tokens, BF16, us: 4 groups in 5 CTAs 30.5; 2 in 4
// 36.1, 2 in 6 35.5, 4 in 4 33.1, 6 in 4 32.5 and, where registers spill, 4 in 6 64.7.  Backward of 4 x 4096, BF16: 4 in 3 96.0; 2 in 4 99.7, 1 in 5
// 122, 3 in 3 110, 4 in 2 106, 4 in 4 147 (spilled); 3 x 517 of 80 in binary32: 2 in 4 15.2, 4 in 3 18.4.
template <typename T, int VEC> constexpr bool kNarrow = sizeof(T) == 2 && VEC == 4;      // four pairs of BF16: the fewest registers
template <typename T, int VEC> constexpr int kBatch = kNarrow<T, VEC> ? 4 : 2;
template <typename T, int VEC> constexpr int kForwardCtas = kNarrow<T, VEC> ? 5 : 4;
template <typename T, int VEC> constexpr int kBackwardBatch = kNarrow<T, VEC> ? 4 : 2;
template <typename T, int VEC> constexpr int kBackwardCtas = kNarrow<T, VEC> ? 3 : 4;
constexpr int kMostBackwardCtas = 4;

struct Side {                                          // queries or keys
    const void* x; const void* dy; void* y;            // backward: y is dx
    int64_t xs[3], ds[3], ys[3];                       // batch, token, head
    const void* weight;                                // (without one: an address that can be read)
    int weighted;
    int heads, groups, batches;                        // groups of 32 / G heads, batches of a few groups
    int64_t group_stride, group_stride_up, group_stride_out;       // bytes from a group to the next in x, dy, y
};
struct RotaryParams {
    Side side[2];
    const double* frequencies;
    const void* positions;
    int64_t position_stride, first_position;
    int items, batch, tokens;                          // items: batch * tokens * parts
    int wide_positions, half_rotary, dim, lanes, parts;        // lanes: log2(G)
    int weight_f32;
    float amplitude, eps, inv_dim;
    float signed_amplitude;                            // of the sines: negative where the angles are negated
    int full;                                          // every pair is turned
    float* partial;                                    // backward: [CTAs][2][dim] sums for the weights' gradients
};

template <int BYTES> struct Raw;                       // a vector as it lies in memory
template <> struct Raw<16> { uint4 v; };
template <> struct Raw<8> { uint2 v; };
template <> struct Raw<4> { uint32_t v; };
template <> struct Raw<2> { unsigned short v; };
// Loads that stay where they are written (the output may be the input, so not by the read-only path).
template <int BYTES> __device__ __forceinline__ Raw<BYTES> load_raw(const void* p) {
    Raw<BYTES> r;
    if constexpr (BYTES == 16) asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.v.x), "=r"(r.v.y), "=r"(r.v.z), "=r"(r.v.w) : "l"(p));
    else if constexpr (BYTES == 8) asm volatile("ld.global.v2.u32 {%0, %1}, [%2];" : "=r"(r.v.x), "=r"(r.v.y) : "l"(p));
    else if constexpr (BYTES == 4) asm volatile("ld.global.u32 %0, [%1];" : "=r"(r.v) : "l"(p));
    else asm volatile("ld.global.u16 %0, [%1];" : "=h"(r.v) : "l"(p));
    return r;
}

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
// columns that are not turned (and whose "pairs" are the columns j and VEC + j, or neighbours, all the same).
template <int VEC, int NU, bool NEIGHBOURS> struct Lane {
    int at[NU][2];                                     // first column of the two vectors
    int first[NU];                                     // first pair
    bool here[NU];                                     // the row has this unit
    __device__ __forceinline__ void place(int lane, int lanes, int half, int dim) {
#pragma unroll
        for (int k = 0; k < NU; ++k) {
            const int u = (lane & ((1 << lanes) - 1)) + (k << lanes);
            here[k] = u * 2 * VEC < dim;
            const bool split = !NEIGHBOURS && u * VEC < half;
            at[k][0] = here[k] ? (split ? u * VEC : u * 2 * VEC) : 0;
            at[k][1] = here[k] ? (split ? half + u * VEC : u * 2 * VEC + VEC) : VEC;
            first[k] = here[k] ? u * VEC : 0;
        }
    }
    // column of member m (0: a, 1: b) of pair k
    __device__ __forceinline__ int column(int k, int m) const {
        const int u = k / VEC, j = k % VEC;
        if (NEIGHBOURS) return at[u][(2 * j + m) / VEC] + (2 * j + m) % VEC;
        return at[u][m] + j;
    }
};

// A row in a lane: P = NU VEC pairs (a, b), two neighbouring pairs' a in one packed value, their b in another: one instruction for both.
template <int P> struct Pairs { f32x2 a[P / 2], b[P / 2]; };
template <typename T, int VEC, int NU> struct RowRaw { Raw<VEC * sizeof(T)> v[NU][2]; };
// `row`: where the lane's first vector of the row lies.
template <typename T, int VEC, int NU, bool NB>
__device__ __forceinline__ void load_row(RowRaw<T, VEC, NU>& r, const char* row, const Lane<VEC, NU, NB>& l) {
#pragma unroll
    for (int k = 0; k < NU; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h) r.v[k][h] = load_raw<VEC * sizeof(T)>(row + (l.at[k][h] - l.at[0][0]) * (int)sizeof(T));
}
template <typename T, int VEC, int NU, bool NB> __device__ __forceinline__ void unpack_row(const RowRaw<T, VEC, NU>& r, Pairs<NU * VEC>& x) {
    float f[NU * VEC][2];
#pragma unroll
    for (int k = 0; k < NU; ++k) {
        float v[2 * VEC];
        unpack<VEC>(r.v[k][0], v, T());
        unpack<VEC>(r.v[k][1], v + VEC, T());
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            f[k * VEC + j][0] = NB ? v[2 * j] : v[j];
            f[k * VEC + j][1] = NB ? v[2 * j + 1] : v[VEC + j];
        }
    }
#pragma unroll
    for (int i = 0; i < NU * VEC / 2; ++i) {
        x.a[i] = f2_pack(f[2 * i][0], f[2 * i + 1][0]);
        x.b[i] = f2_pack(f[2 * i][1], f[2 * i + 1][1]);
    }
}
template <typename T, int VEC, int NU, bool NB>
__device__ __forceinline__ void store_row(char* row, const Pairs<NU * VEC>& y, const Lane<VEC, NU, NB>& l) {
    float f[NU * VEC][2];
#pragma unroll
    for (int i = 0; i < NU * VEC / 2; ++i) {
        f2_unpack(y.a[i], f[2 * i][0], f[2 * i + 1][0]);
        f2_unpack(y.b[i], f[2 * i][1], f[2 * i + 1][1]);
    }
#pragma unroll
    for (int k = 0; k < NU; ++k) {
        float v[2 * VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            v[NB ? 2 * j : j] = f[k * VEC + j][0];
            v[NB ? 2 * j + 1 : VEC + j] = f[k * VEC + j][1];
        }
        if (l.here[k]) {
            store_vec<VEC>(reinterpret_cast<T*>(row + (l.at[k][0] - l.at[0][0]) * (int)sizeof(T)), v);
            store_vec<VEC>(reinterpret_cast<T*>(row + (l.at[k][1] - l.at[0][0]) * (int)sizeof(T)), v + VEC);
        }
    }
}
// Pair k stays as it is: a product with a sine of zero would carry an infinity over to its partner, so what was turned is put back.
template <int VEC, int NU, bool NB>
__device__ __forceinline__ void keep_still(Pairs<NU * VEC>& y, const Pairs<NU * VEC>& x, const Lane<VEC, NU, NB>& l, int half) {
#pragma unroll
    for (int i = 0; i < NU * VEC / 2; ++i) {
        float ya[2], yb[2], xa[2], xb[2];
        f2_unpack(y.a[i], ya[0], ya[1]); f2_unpack(y.b[i], yb[0], yb[1]);
        f2_unpack(x.a[i], xa[0], xa[1]); f2_unpack(x.b[i], xb[0], xb[1]);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = 2 * i + h;
            const bool still = l.first[k / VEC] + k % VEC >= half;
            ya[h] = still ? xa[h] : ya[h];
            yb[h] = still ? xb[h] : yb[h];
        }
        y.a[i] = f2_pack(ya[0], ya[1]);
        y.b[i] = f2_pack(yb[0], yb[1]);
    }
}

__device__ __forceinline__ double position_of(const RotaryParams& p, int64_t b, int64_t t) {
    if (!p.positions) return (double)(p.first_position + t);
    const char* at = static_cast<const char*>(p.positions) + ((b * p.position_stride + t) << (p.wide_positions ? 3 : 2));
    return p.wide_positions ? (double)__ldg(reinterpret_cast<const long long*>(at)) : (double)__ldg(reinterpret_cast<const int*>(at));
}
// VEC floats of shared memory (aligned to them), by loads that stay where they are written: the backward pass has no registers to keep
// them in from row to row.
template <int VEC> __device__ __forceinline__ void read_floats(const float* p, float* f) {
    const uint32_t at = smem_u32(p);
    if constexpr (VEC >= 4) {
#pragma unroll
        for (int i = 0; i < VEC; i += 4)
            asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(f[i]), "=f"(f[i + 1]), "=f"(f[i + 2]), "=f"(f[i + 3]) : "r"(at + 4 * i) : "memory");
    } else if constexpr (VEC == 2) {
        asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(f[0]), "=f"(f[1]) : "r"(at) : "memory");
    } else {
        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(f[0]) : "r"(at) : "memory");
    }
}
// Cosines and sines (times the amplitude) of a token's pairs in the warp's table, every pair once (1 and 0 for those that stay): the lanes
// that hold a pair of different heads read it there.
struct Table { alignas(16) float c[128], s[128], minus_s[128]; };
__device__ __forceinline__ void fill_table(const RotaryParams& p, Table& t, double position, int lane) {
    for (int i = lane; i < p.dim / 2; i += 32) {
        float sn = 0.0f, cs = 1.0f;
        if (i < p.half_rotary) {
            const double turns = position * (__ldg(p.frequencies + i) * 0.15915494309189533577);
            sincospif(2.0f * (float)(turns - rint(turns)), &sn, &cs);
            cs *= p.amplitude;
            sn *= p.signed_amplitude;
        }
        t.c[i] = cs;
        t.s[i] = sn;
        t.minus_s[i] = -sn;
    }
}
template <int VEC, int NU, bool NB> __device__ __forceinline__ void read_table(const float* t, const Lane<VEC, NU, NB>& l, f32x2* out) {
    float v[NU * VEC];
#pragma unroll
    for (int k = 0; k < NU; ++k) read_floats<VEC>(t + l.first[k], v + k * VEC);
#pragma unroll
    for (int i = 0; i < NU * VEC / 2; ++i) out[i] = f2_pack(v[2 * i], v[2 * i + 1]);
}
// Both weights in binary32 (1 without) for the whole CTA.
struct Weights { alignas(16) float w[2][256]; };
__device__ __forceinline__ void load_weights(const RotaryParams& p, Weights& out) {
    for (int i = threadIdx.x; i < 2 * p.dim; i += kThreads) {
        const int side = i >= p.dim, c = i - side * p.dim;
        const bool some = p.side[side].weighted != 0;
        const int at = some ? c : 0;
        const float v = p.weight_f32 ? static_cast<const float*>(p.side[side].weight)[at] : __bfloat162float(static_cast<const __nv_bfloat16*>(p.side[side].weight)[at]);
        out.w[side][c] = some ? v : 1.0f;
    }
}
template <int VEC, int NU, bool NB> __device__ __forceinline__ void read_weights(const float* w, const Lane<VEC, NU, NB>& l, Pairs<NU * VEC>& out) {
    float f[NU * VEC][2];
#pragma unroll
    for (int k = 0; k < NU; ++k) {
        float v[2 * VEC];
        read_floats<VEC>(w + l.at[k][0], v);
        read_floats<VEC>(w + l.at[k][1], v + VEC);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            f[k * VEC + j][0] = NB ? v[2 * j] : v[j];
            f[k * VEC + j][1] = NB ? v[2 * j + 1] : v[VEC + j];
        }
    }
#pragma unroll
    for (int i = 0; i < NU * VEC / 2; ++i) {
        out.a[i] = f2_pack(f[2 * i][0], f[2 * i + 1][0]);
        out.b[i] = f2_pack(f[2 * i][1], f[2 * i + 1][1]);
    }
}
__device__ __forceinline__ f32x2 twice(float x) { return f2_pack(x, x); }
// sum over a lane's columns that exist of x y
template <int VEC, int NU, bool NB> __device__ __forceinline__ float dot(const Pairs<NU * VEC>& x, const Pairs<NU * VEC>& y, const Lane<VEC, NU, NB>& l) {
    float sum = 0.0f;
    if constexpr (NU == 1) {
        f32x2 v = f2_mul(x.a[0], y.a[0]);
#pragma unroll
        for (int i = 1; i < VEC / 2; ++i) v = f2_fma(x.a[i], y.a[i], v);
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) v = f2_fma(x.b[i], y.b[i], v);
        float lo, hi;
        f2_unpack(v, lo, hi);
        sum = l.here[0] ? lo + hi : 0.0f;
    } else {
#pragma unroll
        for (int i = 0; i < NU * VEC / 2; ++i) {
            float u[2], v[2];
            f2_unpack(f2_mul(x.a[i], y.a[i]), u[0], u[1]);
            f2_unpack(f2_mul(x.b[i], y.b[i]), v[0], v[1]);
#pragma unroll
            for (int h = 0; h < 2; ++h) sum += l.here[(2 * i + h) / VEC] ? u[h] + v[h] : 0.0f;
        }
    }
    return sum;
}
// Sums over the lanes of a row.
template <int N> __device__ __forceinline__ void row_sums(float (&v)[N], int lanes) {
    if (lanes == 3) {                                      // 16-bit rows of 66 to 128, 32-bit ones of 34 to 64: without the branches
#pragma unroll
        for (int d = 2; d >= 0; --d)
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], 1 << d);
        return;
    }
#pragma unroll
    for (int d = 4; d >= 0; --d)
        if (lanes > d) {
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], 1 << d);
        }
}


// A warp takes one item: the batches [first, last) of U groups of one token, queries before keys.  The next batch is loaded while one is
// worked on, the first one under the angles; U rows side by side hide the latency of the norm's chain (sum, shuffles, root).
template <typename T, int VEC, bool NEIGHBOURS, bool NORM>
__global__ void __launch_bounds__(kThreads, kForwardCtas<T, VEC>) rotary_kernel(const __grid_constant__ RotaryParams p) {
    constexpr int NU = VEC >= 4 ? 1 : 4 / VEC, P = NU * VEC, U = kBatch<T, VEC>;
    __shared__ Table tables[kWarps];
    __shared__ Weights weights;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int slot = lane >> p.lanes, slots = 32 >> p.lanes;
    const unsigned index = blockIdx.x * kWarps + warp;
    const bool any = index < (unsigned)p.items;
    Lane<VEC, NU, NEIGHBOURS> l;
    l.place(lane, p.lanes, p.half_rotary, p.dim);
    const int q_batches = p.side[0].batches;
    unsigned token = index;
    int i = 0, last = q_batches + p.side[1].batches;
    if (p.parts > 1) {
        token = index / (unsigned)p.parts;
        const int part = index - token * p.parts, all = last;
        i = all * part / p.parts;
        last = all * (part + 1) / p.parts;
    }
    const unsigned b = p.batch == 1 ? 0 : token / (unsigned)p.tokens, t = token - b * p.tokens;
    RowRaw<T, VEC, NU> raw[U];
    // of the batch that is loaded next, and of the one that is worked on: side, first head and where it lies (this lane's part of it)
    auto place_of = [&](int batch, const Side& sd, const void* base, const int64_t (&strides)[3]) {
        return static_cast<const char*>(base) + (b * strides[0] + t * strides[1] + (int64_t)(batch * U * slots + slot) * strides[2] + l.at[0][0]) * (int64_t)sizeof(T);
    };
    int ahead_side = i >= q_batches, ahead_head = (i - (ahead_side ? q_batches : 0)) * U * slots + slot;
    const char* ahead = any ? place_of(i - (ahead_side ? q_batches : 0), p.side[ahead_side], p.side[ahead_side].x, p.side[ahead_side].xs) : nullptr;
    auto load = [&]() {
        const Side& sd = p.side[ahead_side];
        const int64_t group = sd.group_stride;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (ahead_head < sd.heads) load_row(raw[u], ahead, l);
            ahead += group;
            ahead_head += slots;
        }
    };
    if (any) {
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = RowRaw<T, VEC, NU>{};
        load();
    }
    if (NORM) load_weights(p, weights);
    if (any) fill_table(p, tables[warp], position_of(p, b, t), lane);
    if (NORM) __syncthreads();
    else __syncwarp();
    if (!any) return;
    f32x2 ca[P / 2], cb[P / 2], sa[P / 2], sb[P / 2];
    int side_now = -1, head = 0;
    char* to = nullptr;
#pragma unroll 1
    for (; i < last; ++i) {
        const int side = i >= q_batches;
        if (side != side_now) {                            // a' = a ca - b sb, b' = b cb + a sa: the weights go into the angles
            side_now = side;
            const int first = i - (side ? q_batches : 0);
            head = first * U * slots + slot;
            to = const_cast<char*>(place_of(first, p.side[side], p.side[side].y, p.side[side].ys));
            read_table(tables[warp].c, l, ca);
            read_table(tables[warp].s, l, sa);
            read_table(tables[warp].minus_s, l, sb);
            Pairs<P> w;
            if (NORM) read_weights(weights.w[side], l, w);
#pragma unroll
            for (int k = 0; k < P / 2; ++k) {
                cb[k] = NORM ? f2_mul(ca[k], w.b[k]) : ca[k];
                sb[k] = NORM ? f2_mul(sb[k], w.b[k]) : sb[k];
                ca[k] = NORM ? f2_mul(ca[k], w.a[k]) : ca[k];
                sa[k] = NORM ? f2_mul(sa[k], w.a[k]) : sa[k];
            }
        }
        Pairs<P> f[U];
#pragma unroll
        for (int u = 0; u < U; ++u) unpack_row<T, VEC, NU, NEIGHBOURS>(raw[u], f[u]);
        if (i + 1 < last) {
            if (i + 1 == q_batches) {
                ahead_side = 1;
                ahead_head = slot;
                ahead = place_of(0, p.side[1], p.side[1].x, p.side[1].xs);
            }
            load();
        }
        if (NORM) {
            float sum[U];
#pragma unroll
            for (int u = 0; u < U; ++u) sum[u] = dot(f[u], f[u], l);
            row_sums(sum, p.lanes);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const f32x2 r = twice(rsqrtf(fmaf(sum[u], p.inv_dim, p.eps)));
#pragma unroll
                for (int k = 0; k < P / 2; ++k) { f[u].a[k] = f2_mul(f[u].a[k], r); f[u].b[k] = f2_mul(f[u].b[k], r); }
            }
        }
        const int heads = p.side[side].heads;
        const int64_t group = p.side[side].group_stride_out;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            Pairs<P> o;
#pragma unroll
            for (int k = 0; k < P / 2; ++k) {
                o.a[k] = f2_fma(f[u].b[k], sb[k], f2_mul(f[u].a[k], ca[k]));
                o.b[k] = f2_fma(f[u].a[k], sa[k], f2_mul(f[u].b[k], cb[k]));
            }
            if (!p.full) {
                if (NORM) {
#pragma unroll
                    for (int k = 0; k < P / 2; ++k) { f[u].a[k] = f2_mul(f[u].a[k], ca[k]); f[u].b[k] = f2_mul(f[u].b[k], cb[k]); }
                }
                keep_still(o, f[u], l, p.half_rotary);
            }
            if (head < heads) store_row<T, VEC, NU, NEIGHBOURS>(to, o, l);
            to += group;
            head += slots;
        }
    }
}

// Persistent: a warp walks its tokens, the next group is loaded while one is worked on, over the end of a token too.  The sums for the weights' gradients are
// kept by every lane for its columns (in shared memory between tokens, in registers within one), added over the CTA at the end and leave as one
// binary32 row per CTA, which rotary_weights_kernel adds in a fixed order: no atomics.
template <typename T, int VEC, bool NEIGHBOURS>
__global__ void __launch_bounds__(kThreads, kBackwardCtas<T, VEC>) rotary_backward_kernel(const __grid_constant__ RotaryParams p) {
    constexpr int NU = VEC >= 4 ? 1 : 4 / VEC, P = NU * VEC, U = kBackwardBatch<T, VEC>;
    __shared__ Table tables[kWarps];
    __shared__ Weights weights;
    __shared__ float sums[2][2 * P][kThreads];
    if (p.partial) asm volatile("griddepcontrol.launch_dependents;");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int slot = lane >> p.lanes, slots = 32 >> p.lanes;
    Lane<VEC, NU, NEIGHBOURS> l;
    l.place(lane, p.lanes, p.half_rotary, p.dim);
    const int q_batches = p.side[0].batches, batches = q_batches + p.side[1].batches;
    const unsigned step = gridDim.x * kWarps, items = p.items;
    struct Work { unsigned b, t; int i, last; };           // a token and its batches [i, last)
    auto work_of = [&](unsigned index) {
        Work w;
        unsigned token = index;
        w.i = 0;
        w.last = batches;
        if (p.parts > 1) {
            token = index / (unsigned)p.parts;
            const int part = index - token * p.parts;
            w.i = batches * part / p.parts;
            w.last = batches * (part + 1) / p.parts;
        }
        w.b = p.batch == 1 ? 0 : token / (unsigned)p.tokens;
        w.t = token - w.b * p.tokens;
        return w;
    };
    RowRaw<T, VEC, NU> rx[U], rd[U];
    // the batch that is loaded next: side, this lane's first head, where its x and dy lie (this lane's part of them)
    int ahead_side = 0, ahead_head = 0;
    const char *ahead_x = nullptr, *ahead_d = nullptr;
    auto place = [&](const Work& w, int i) {
        ahead_side = i >= q_batches;
        const Side& sd = p.side[ahead_side];
        ahead_head = (i - (ahead_side ? q_batches : 0)) * U * slots + slot;
        ahead_x = static_cast<const char*>(sd.x) + (w.b * sd.xs[0] + w.t * sd.xs[1] + ahead_head * sd.xs[2] + l.at[0][0]) * (int64_t)sizeof(T);
        ahead_d = static_cast<const char*>(sd.dy) + (w.b * sd.ds[0] + w.t * sd.ds[1] + ahead_head * sd.ds[2] + l.at[0][0]) * (int64_t)sizeof(T);
    };
    auto load = [&]() {
        const Side& sd = p.side[ahead_side];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (ahead_head < sd.heads) {
                load_row(rx[u], ahead_x, l);
                load_row(rd[u], ahead_d, l);
            } else {                                       // a head that does not exist: nothing is added up for it
                rx[u] = RowRaw<T, VEC, NU>{};
                rd[u] = RowRaw<T, VEC, NU>{};
            }
            ahead_head += slots;
            ahead_x += sd.group_stride;
            ahead_d += sd.group_stride_up;
        }
    };
    unsigned index = blockIdx.x * kWarps + warp;
    Work now{};
    if (index < items) {
        now = work_of(index);
        place(now, now.i);
        load();
    }
#pragma unroll
    for (int i = 0; i < 2 * P; ++i) sums[0][i][threadIdx.x] = sums[1][i][threadIdx.x] = 0.0f;
    load_weights(p, weights);
    __syncthreads();
#pragma unroll 1
    while (index < items) {
        index += step;
        Work next = now;
        if (index < items) next = work_of(index);
        __syncwarp();
        fill_table(p, tables[warp], position_of(p, now.b, now.t), lane);
        __syncwarp();
#pragma unroll 1
        for (int side = now.i >= q_batches; side < 2; ++side) {
            const Side& sd = p.side[side];
            const int skip = side ? q_batches : 0, end = side ? now.last : min(now.last, q_batches);
            int head = (now.i - skip) * U * slots + slot;
            char* to = static_cast<char*>(sd.y) + (now.b * sd.ys[0] + now.t * sd.ys[1] + head * sd.ys[2] + l.at[0][0]) * (int64_t)sizeof(T);
            Pairs<P> acc;
#pragma unroll
            for (int i = 0; i < P / 2; ++i) acc.a[i] = acc.b[i] = 0;
#pragma unroll 1
            for (; now.i < end; ++now.i) {
                Pairs<P> f[U], e[U];                       // x, and dy turned back
                {
                    Pairs<P> d[U];
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        unpack_row<T, VEC, NU, NEIGHBOURS>(rx[u], f[u]);
                        unpack_row<T, VEC, NU, NEIGHBOURS>(rd[u], d[u]);
                    }
                    if (now.i + 1 < now.last) {
                        if (now.i + 1 == q_batches) place(now, q_batches);
                        load();
                    } else if (index < items) {
                        place(next, next.i);
                        load();
                    }
                    f32x2 c[P / 2], sn[P / 2];             // (the sines are those of the negated angles)
                    read_table(tables[warp].c, l, c);
                    read_table(tables[warp].s, l, sn);
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int i = 0; i < P / 2; ++i) {
                            e[u].a[i] = f2_mul(d[u].a[i], c[i]);
                            e[u].b[i] = f2_fma(d[u].a[i], sn[i], f2_mul(d[u].b[i], c[i]));
                        }
                    read_table(tables[warp].minus_s, l, sn);
#pragma unroll
                    for (int u = 0; u < U; ++u) {
#pragma unroll
                        for (int i = 0; i < P / 2; ++i) e[u].a[i] = f2_fma(d[u].b[i], sn[i], e[u].a[i]);
                        if (!p.full) keep_still(e[u], d[u], l, p.half_rotary);
                    }
                }
                float sum[2 * U];
                {
                    Pairs<P> w;
                    read_weights(weights.w[side], l, w);
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        Pairs<P> g;
#pragma unroll
                        for (int i = 0; i < P / 2; ++i) { g.a[i] = f2_mul(e[u].a[i], w.a[i]); g.b[i] = f2_mul(e[u].b[i], w.b[i]); }
                        sum[2 * u] = dot(f[u], f[u], l);
                        sum[2 * u + 1] = dot(g, f[u], l);
                    }
                }
                row_sums(sum, p.lanes);
                Pairs<P> w;                                // (read again: no registers to keep them in meanwhile)
                read_weights(weights.w[side], l, w);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const bool exists = head < sd.heads;   // (else a row of zeros, whose root is 0 with an eps of 0)
                    const float r = exists ? rsqrtf(fmaf(sum[2 * u], p.inv_dim, p.eps)) : 0.0f;
                    const f32x2 r2 = twice(r), m2 = twice(-(sum[2 * u + 1] * r * p.inv_dim));
                    Pairs<P> d;
#pragma unroll
                    for (int i = 0; i < P / 2; ++i) {      // xh = x r, dx = r (g - xh m)
                        f[u].a[i] = f2_mul(f[u].a[i], r2);
                        f[u].b[i] = f2_mul(f[u].b[i], r2);
                        acc.a[i] = f2_fma(e[u].a[i], f[u].a[i], acc.a[i]);
                        acc.b[i] = f2_fma(e[u].b[i], f[u].b[i], acc.b[i]);
                        d.a[i] = f2_mul(f2_fma(e[u].a[i], w.a[i], f2_mul(f[u].a[i], m2)), r2);
                        d.b[i] = f2_mul(f2_fma(e[u].b[i], w.b[i], f2_mul(f[u].b[i], m2)), r2);
                    }
                    if (exists) store_row<T, VEC, NU, NEIGHBOURS>(to, d, l);
                    head += slots;
                    to += sd.group_stride_out;
                }
            }
#pragma unroll
            for (int i = 0; i < P / 2; ++i) {
                float v[4];
                f2_unpack(acc.a[i], v[0], v[1]);
                f2_unpack(acc.b[i], v[2], v[3]);
#pragma unroll
                for (int k = 0; k < 4; ++k) sums[side][4 * i + k][threadIdx.x] += v[k];
            }
        }
        now = next;
    }
    if (!p.partial) return;
    __syncthreads();
    // a column's sum: over the warps and the heads side by side in each, in order
    for (int i = threadIdx.x; i < 2 << p.lanes; i += kThreads) {
        const int side = i >> p.lanes, holder = i & ((1 << p.lanes) - 1);
        Lane<VEC, NU, NEIGHBOURS> of;
        of.place(holder, p.lanes, p.half_rotary, p.dim);
#pragma unroll
        for (int k = 0; k < P; ++k)
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                float v = 0.0f;
                for (int t = holder; t < kThreads; t += 1 << p.lanes) v += sums[side][4 * (k / 2) + 2 * m + (k & 1)][t];
                if (of.here[k / VEC]) p.partial[((int64_t)blockIdx.x * 2 + side) * p.dim + of.column(k, m)] = v;
            }
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
    const bool backward = a.op == RotaryArgs::kBackward;
    const int batch = backward ? kBackwardBatch<T, VEC> : kBatch<T, VEC>, resident = 148 * (backward ? kBackwardCtas<T, VEC> : kForwardCtas<T, VEC>);
    for (Side& s : p.side) {
        s.groups = (s.heads + slots - 1) / slots;
        s.batches = (s.groups + batch - 1) / batch;
        s.group_stride = slots * s.xs[2] * (int64_t)sizeof(T);
        s.group_stride_up = slots * s.ds[2] * (int64_t)sizeof(T);
        s.group_stride_out = slots * s.ys[2] * (int64_t)sizeof(T);
    }
    const int64_t rows = a.s.batch * a.s.tokens, warps = kWarps * resident;
    const int pieces = p.side[0].batches + p.side[1].batches;
    // The heads of a token are shared out where that makes the longest warp's work shorter: rounds of items times batches of an item, with
    // what every item costs besides (angles, addresses) taken as one batch.
    int64_t least = INT64_MAX;
    for (int n = 1; n <= pieces; n = n < 32 ? n + 1 : n < pieces && 2 * n > pieces ? pieces : 2 * n) {
        const int64_t cost = (rows * n + warps - 1) / warps * ((pieces + n - 1) / n + 1);
        if (cost < least) {
            least = cost;
            p.parts = n;
        }
    }
    p.items = (int)(rows * p.parts);
    const int64_t ctas = (p.items + kWarps - 1) / kWarps;
    const unsigned grid = (unsigned)(backward ? std::min<int64_t>(ctas, resident) : ctas);
    if (backward) {
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
        return cudaLaunchKernelEx(&cfg, rotary_weights_kernel, (const float*)p.partial, (int)grid, p.dim, a.dweight[0], a.dweight[1], p.weight_f32);
    }
    if (a.op == RotaryArgs::kNorm) rotary_kernel<T, VEC, NB, true><<<grid, kThreads, 0, st>>>(p);
    else rotary_kernel<T, VEC, NB, false><<<grid, kThreads, 0, st>>>(p);
    return cudaGetLastError();
}
template <typename T, int VEC>
cudaError_t run(const RotaryArgs& a, RotaryParams& p, cudaStream_t st) {
    return a.s.interleaved ? run<T, VEC, true>(a, p, st) : run<T, VEC, false>(a, p, st);
}

}  // namespace

int rotary_backward_ctas() { return 148 * kMostBackwardCtas; }

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
            continue;
        }
        auto take = [&](const ue5m3_heads& h, int64_t (&strides)[3]) {
            strides[0] = s.batch > 1 ? h.batch_stride : 0;
            strides[1] = s.tokens > 1 ? h.token_stride : 0;
            strides[2] = d.heads > 1 ? h.head_stride : 0;
            bits |= reinterpret_cast<uintptr_t>(h.data) / (uint64_t)size;
            for (int64_t x : strides) bits |= (uint64_t)x;
            return h.data;
        };
        d.x = take(t.x, d.xs);
        d.y = take(t.y, d.ys);
        if (a.op == RotaryArgs::kBackward) d.dy = take(t.dy, d.ds);
        d.weighted = a.weight[k] != nullptr;
        d.weight = d.weighted ? a.weight[k] : s.frequencies;
    }
    p.frequencies = s.frequencies;
    p.positions = s.positions;
    p.position_stride = s.position_stride;
    p.first_position = s.first_position;
    p.batch = (int)s.batch;
    p.tokens = (int)s.tokens;
    p.wide_positions = s.position_bytes == 8;
    p.half_rotary = (int)(s.rotary_dim / 2);
    p.dim = (int)s.head_dim;
    p.weight_f32 = a.weight_dtype == UE5M3_F32;
    p.amplitude = s.amplitude;
    p.eps = a.eps;
    p.inv_dim = 1.0f / (float)s.head_dim;
    p.signed_amplitude = a.inverse ? -s.amplitude : s.amplitude;
    p.full = s.rotary_dim == s.head_dim;
    p.partial = a.partial;
    // The largest vector that the addresses allow and that no row's end, and of halves no pair's end, cuts.
    bits |= (uint64_t)s.head_dim / 2;
    if (!s.interleaved) bits |= (uint64_t)p.half_rotary;
    const int vec = (int)(bits & (0 - bits) & 7) ? (int)(bits & (0 - bits)) : 8;
    if (s.dtype == UE5M3_BF16) {
        if (vec >= 4) return run<__nv_bfloat16, 4>(a, p, st);
        if (vec == 2) return run<__nv_bfloat16, 2>(a, p, st);
        return run<__nv_bfloat16, 1>(a, p, st);
    }
    if (vec >= 4) return run<float, 4>(a, p, st);
    if (vec == 2) return run<float, 2>(a, p, st);
    return run<float, 1>(a, p, st);
}

}  // namespace ue5m3
