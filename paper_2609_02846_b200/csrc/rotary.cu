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
// neighbouring pairs), 32 / G heads side by side (a group), and the warp walks the groups with a lane's pairs, and so its angles and weights,
// staying the same.  The norm's sum over a row is log2(G) shuffles.  Rows come through a ring of asynchronous copies in shared memory, a
// ring per warp, several groups ahead and on into the warp's next token; registers cannot hold enough of them: with four groups loaded
// into registers at a time norm and rotation of 2 x 4096 tokens took 43 us.  The copies are of 16 bytes wherever addresses allow it, whatever VEC is,
// which is 16 bytes where no pair's end cuts it, else 8, 4 or 2.  Where there are few tokens the groups of one are shared out among warps.
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
constexpr int kBatch = 2;                              // groups that a forward warp works on at a time

struct Side {                                          // queries or keys
    const void* x; const void* dy; void* y;            // backward: y is dx
    int64_t xs[3], ds[3], ys[3];                       // batch, token, head
    const void* weight;                                // (without one: an address that can be read)
    int weighted;
    int heads, groups, batches;                        // groups of 32 / G heads, batches of kBatch groups
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

// A row in a lane: P = NU VEC pairs (a, b), two neighbouring pairs' a in one packed value, their b in another.
template <int P> struct Pairs { f32x2 a[P / 2], b[P / 2]; };
template <typename T, int VEC, int NU> struct RowRaw { Raw<VEC * sizeof(T)> v[NU][2]; };
template <typename T, int VEC, int NU, bool NB>
__device__ __forceinline__ void load_row(RowRaw<T, VEC, NU>& r, const T* row, const Lane<VEC, NU, NB>& l) {
#pragma unroll
    for (int k = 0; k < NU; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h) r.v[k][h] = load_raw<VEC * sizeof(T)>(row + l.at[k][h]);
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
__device__ __forceinline__ void store_row(T* row, const Pairs<NU * VEC>& y, const Lane<VEC, NU, NB>& l) {
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
            store_vec<VEC>(row + l.at[k][0], v);
            store_vec<VEC>(row + l.at[k][1], v + VEC);
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
// VEC floats of shared memory (aligned to them).
template <int VEC> __device__ __forceinline__ void read_floats(const float* p, float* f) {
    if constexpr (VEC >= 4) {
#pragma unroll
        for (int i = 0; i < VEC; i += 4) {
            const float4 v = *reinterpret_cast<const float4*>(p + i);
            f[i] = v.x; f[i + 1] = v.y; f[i + 2] = v.z; f[i + 3] = v.w;
        }
    } else if constexpr (VEC == 2) {
        const float2 v = *reinterpret_cast<const float2*>(p);
        f[0] = v.x; f[1] = v.y;
    } else {
        f[0] = *p;
    }
}
// Cosines and sines (times the amplitude) of a token's pairs in the warp's table, every pair once (1 and 0 for those that stay): the lanes
// that hold a pair of different heads read it there.
struct Table { alignas(16) float c[128], s[128]; };
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
    }
}
template <int VEC, int NU, bool NB>
__device__ __forceinline__ void read_table(const Table& t, const Lane<VEC, NU, NB>& l, f32x2* c, f32x2* s) {
    float cs[NU * VEC], sn[NU * VEC];
#pragma unroll
    for (int k = 0; k < NU; ++k) {
        read_floats<VEC>(t.c + l.first[k], cs + k * VEC);
        read_floats<VEC>(t.s + l.first[k], sn + k * VEC);
    }
#pragma unroll
    for (int i = 0; i < NU * VEC / 2; ++i) {
        c[i] = f2_pack(cs[2 * i], cs[2 * i + 1]);
        s[i] = f2_pack(sn[2 * i], sn[2 * i + 1]);
    }
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
__device__ __forceinline__ f32x2 f2_minus(f32x2 x) {
    float a, b;
    f2_unpack(x, a, b);
    return f2_pack(-a, -b);
}
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
#pragma unroll
    for (int d = 4; d >= 0; --d)
        if (lanes > d) {
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], 1 << d);
        }
}

constexpr int kForwardCtas = 4, kBackwardCtas = 4;     // CTAs per SM (backward: of a persistent grid)

// A warp takes one item: the batches [first, last) of U groups of one token, queries before keys.  The next batch is loaded while one is
// worked on, the first one under the angles; U rows side by side hide the latency of the norm's chain (sum, shuffles, root).
template <typename T, int VEC, bool NEIGHBOURS, bool NORM>
__global__ void __launch_bounds__(kThreads, kForwardCtas) rotary_kernel(const __grid_constant__ RotaryParams p) {
    constexpr int NU = VEC >= 4 ? 1 : 4 / VEC, P = NU * VEC, U = kBatch;
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
    const T* from[2];
    T* to[2];
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        const Side& sd = p.side[side];
        from[side] = static_cast<const T*>(sd.x) + b * sd.xs[0] + t * sd.xs[1] + slot * sd.xs[2];
        to[side] = static_cast<T*>(sd.y) + b * sd.ys[0] + t * sd.ys[1] + slot * sd.ys[2];
    }
    RowRaw<T, VEC, NU> raw[U];
    auto load = [&](int batch) {
        const int side = batch >= q_batches, h0 = (batch - (side ? q_batches : 0)) * U * slots, heads = p.side[side].heads - slot;
        const int64_t stride = p.side[side].xs[2];
        const T* row = (side ? from[1] : from[0]) + h0 * stride;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (h0 + u * slots < heads) load_row(raw[u], row + u * slots * stride, l);
    };
    if (any) {
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = RowRaw<T, VEC, NU>{};
        load(i);
    }
    if (NORM) load_weights(p, weights);
    if (any) fill_table(p, tables[warp], position_of(p, b, t), lane);
    if (NORM) __syncthreads();
    else __syncwarp();
    if (!any) return;
    f32x2 ca[P / 2], cb[P / 2], sa[P / 2], sb[P / 2];
    int side_now = -1;
#pragma unroll 1
    for (; i < last; ++i) {
        const int side = i >= q_batches;
        if (side != side_now) {                            // a' = a ca - b sb, b' = b cb + a sa: the weights go into the angles
            side_now = side;
            read_table(tables[warp], l, ca, sa);
            Pairs<P> w;
            if (NORM) read_weights(weights.w[side], l, w);
#pragma unroll
            for (int k = 0; k < P / 2; ++k) {
                cb[k] = NORM ? f2_mul(ca[k], w.b[k]) : ca[k];
                sb[k] = f2_minus(NORM ? f2_mul(sa[k], w.b[k]) : sa[k]);
                ca[k] = NORM ? f2_mul(ca[k], w.a[k]) : ca[k];
                sa[k] = NORM ? f2_mul(sa[k], w.a[k]) : sa[k];
            }
        }
        Pairs<P> f[U];
#pragma unroll
        for (int u = 0; u < U; ++u) unpack_row<T, VEC, NU, NEIGHBOURS>(raw[u], f[u]);
        if (i + 1 < last) load(i + 1);
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
        const int h0 = (i - (side ? q_batches : 0)) * U * slots, heads = p.side[side].heads - slot;
        const int64_t stride = p.side[side].ys[2];
        T* row = (side ? to[1] : to[0]) + h0 * stride;
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
            if (h0 + u * slots < heads) store_row(row + u * slots * stride, o, l);
        }
    }
}

// Persistent: a warp walks its tokens, the next group is loaded while one is worked on, over the end of a token too.  The sums for the weights' gradients are
// kept by every lane for its columns (in shared memory between tokens, in registers within one), added over the CTA at the end and leave as one
// binary32 row per CTA, which rotary_weights_kernel adds in a fixed order: no atomics.
template <typename T, int VEC, bool NEIGHBOURS>
__global__ void __launch_bounds__(kThreads, kBackwardCtas) rotary_backward_kernel(const __grid_constant__ RotaryParams p) {
    constexpr int NU = VEC >= 4 ? 1 : 4 / VEC, P = NU * VEC;
    __shared__ Table tables[kWarps];
    __shared__ Weights weights;
    __shared__ float sums[2][2 * P][kThreads];
    if (p.partial) asm volatile("griddepcontrol.launch_dependents;");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int slot = lane >> p.lanes, slots = 32 >> p.lanes;
    Lane<VEC, NU, NEIGHBOURS> l;
    l.place(lane, p.lanes, p.half_rotary, p.dim);
    const int q_groups = p.side[0].groups, groups = q_groups + p.side[1].groups;
    const unsigned step = gridDim.x * kWarps, items = p.items;
    struct Work { unsigned b, t; int g, g_end; };
    auto work_of = [&](unsigned index) {
        Work w;
        unsigned token = index;
        w.g = 0;
        w.g_end = groups;
        if (p.parts > 1) {
            token = index / (unsigned)p.parts;
            const int part = index - token * p.parts;
            w.g = groups * part / p.parts;
            w.g_end = groups * (part + 1) / p.parts;
        }
        w.b = p.batch == 1 ? 0 : token / (unsigned)p.tokens;
        w.t = token - w.b * p.tokens;
        return w;
    };
    RowRaw<T, VEC, NU> rx{}, rd{};
    auto load = [&](const Work& w, int g) {                // group g of the token of w
        const int side = g >= q_groups, h = (g - (side ? q_groups : 0)) * slots + slot;
        const Side& sd = p.side[side];
        if (h < sd.heads) {
            load_row(rx, static_cast<const T*>(sd.x) + w.b * sd.xs[0] + w.t * sd.xs[1] + h * sd.xs[2], l);
            load_row(rd, static_cast<const T*>(sd.dy) + w.b * sd.ds[0] + w.t * sd.ds[1] + h * sd.ds[2], l);
        }
    };
    unsigned index = blockIdx.x * kWarps + warp;
    Work now{};
    if (index < items) {
        now = work_of(index);
        load(now, now.g);
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
        f32x2 c[P / 2], s[P / 2];
        read_table(tables[warp], l, c, s);
#pragma unroll 1
        for (int side = now.g >= q_groups; side < 2; ++side) {
            const Side& sd = p.side[side];
            const int skip = side ? q_groups : 0, end = side ? now.g_end : min(now.g_end, q_groups);
            T* to = static_cast<T*>(sd.y) + now.b * sd.ys[0] + now.t * sd.ys[1];
            Pairs<P> w, acc;
            read_weights(weights.w[side], l, w);
#pragma unroll
            for (int i = 0; i < P / 2; ++i) acc.a[i] = acc.b[i] = 0;
#pragma unroll 1
            for (; now.g < end; ++now.g) {
                Pairs<P> f, d, e;
                unpack_row<T, VEC, NU, NEIGHBOURS>(rx, f);
                unpack_row<T, VEC, NU, NEIGHBOURS>(rd, d);
                if (now.g + 1 < now.g_end) load(now, now.g + 1);
                else if (index < items) load(next, next.g);
                const int h = (now.g - skip) * slots + slot;
#pragma unroll
                for (int i = 0; i < P / 2; ++i) {          // (the sines are those of the negated angles)
                    e.a[i] = f2_fma(f2_minus(d.b[i]), s[i], f2_mul(d.a[i], c[i]));
                    e.b[i] = f2_fma(d.a[i], s[i], f2_mul(d.b[i], c[i]));
                }
                if (!p.full) keep_still(e, d, l, p.half_rotary);
#pragma unroll
                for (int i = 0; i < P / 2; ++i) { d.a[i] = f2_mul(e.a[i], w.a[i]); d.b[i] = f2_mul(e.b[i], w.b[i]); }
                float sum[2] = {dot(f, f, l), dot(d, f, l)};
                row_sums(sum, p.lanes);
                const float r = rsqrtf(fmaf(sum[0], p.inv_dim, p.eps));
                const f32x2 r2 = twice(r), m2 = twice(-(sum[1] * r * p.inv_dim));
                const bool exists = h < sd.heads;
#pragma unroll
                for (int i = 0; i < P / 2; ++i) {          // xh = x r, dx = r (g - xh m)
                    f.a[i] = f2_mul(f.a[i], r2);
                    f.b[i] = f2_mul(f.b[i], r2);
                    if (exists) {
                        acc.a[i] = f2_fma(e.a[i], f.a[i], acc.a[i]);
                        acc.b[i] = f2_fma(e.b[i], f.b[i], acc.b[i]);
                    }
                    d.a[i] = f2_mul(f2_fma(f.a[i], m2, d.a[i]), r2);
                    d.b[i] = f2_mul(f2_fma(f.b[i], m2, d.b[i]), r2);
                }
                if (exists) store_row(to + h * sd.ys[2], d, l);
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
    for (Side& s : p.side) {
        s.groups = (s.heads + slots - 1) / slots;
        s.batches = (s.groups + kBatch - 1) / kBatch;
    }
    const bool backward = a.op == RotaryArgs::kBackward;
    const int64_t rows = a.s.batch * a.s.tokens, warps = 148 * kWarps * (backward ? kBackwardCtas : kForwardCtas);
    const int pieces = backward ? p.side[0].groups + p.side[1].groups : p.side[0].batches + p.side[1].batches;
    // Few tokens: the heads of one are shared out, so that there is an item for every warp.
    p.parts = (int)std::min<int64_t>(pieces, (warps + rows - 1) / rows);
    p.items = (int)(rows * p.parts);
    const int64_t ctas = (p.items + kWarps - 1) / kWarps;
    const unsigned grid = (unsigned)(backward ? std::min<int64_t>(ctas, 148 * kBackwardCtas) : ctas);
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

int rotary_backward_ctas() { return 148 * kBackwardCtas; }

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
