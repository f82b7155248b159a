// Attention, backward, for sm_100a.  Nothing of the forward pass is kept but o and lse; with s = scale log2(e) q.k
//     P_ij = 2^(s_ij - lse2_i),  dP_ij = dout_i . v_j,  dS_ij = P_ij (dP_ij - D_i),  D_i = dout_i . o_i
//     dv_j = sum_i P_ij dout_i,  dk_j = scale sum_i dS_ij q_i,  dq_i = scale sum_j dS_ij k_j
//
// Three launches:
//   rows     -D_i and -log2(e) lse_i of every query (padded to whole tiles; -inf where a query sees nothing, so that P = 0)
//   keys     a CTA owns 128 keys of one key/value head and walks the queries that see them, through all query heads of the
//            group: S^T = K Q^T, dP^T = V dO^T, then dV += P^T dO and dK += dS^T Q
//   queries  a CTA owns 128 queries of one head and walks the keys they see: S = Q K^T, dP = dO V^T, dQ += dS K
// S and dP are computed in both (7 products instead of 5): in exchange every gradient is summed by one CTA in one fixed order
// in tensor memory; there is no atomic and nothing that changes from call to call (few queries for many keys share the keys out
// and add binary32 parts in order).  The three overlap: the keys kernel sets itself up under the rows kernel, the queries kernel fills
// the tail of the keys kernel.
//
// 2 x 4096 tokens, 32 / 8 heads of 128, causal: rows 25 us (5.4 TB/s), keys 403, queries 371 (ncu), together 757 to 780 us in short
// bursts: about 890 TFLOP/s of the 5 products that the gradients need, 1250 of the 7 that are computed, 0.76 of the measured burst rate
// of a BF16 product.  One call after the other, under the power cap, 878 to 888 us: 1090 TFLOP/s of the 7, 0.79 of the sustained
// rate.  A step of the keys kernel takes 2620 cycles (products 2048), of the queries kernel about 2200 (1536): what bounds both is the
// chain of a step, S - P - dP - dS - product, with two tiles in tensor memory to overlap it.
//
// P and dS are rounded to BF16 for the products that add them up, since the other operand (dO, Q, K) is BF16 and a product has one type:
// 2^-8 of each value at most, in binary32 before and after.  Against 64 bits the gradients are off by a relative 0.0024 of their norm (up
// to 0.0032 where a few pairs carry it), of which their own rounding makes 0.0017.
//
// P and dS never touch shared memory: the softmax warps read S and dP from tensor memory and write P and dS (BF16) over them,
// from where the tensor core takes them as the A operand.  Both kernels have the same roles:
//   warp 0      copies     warp 1   issues the MMAs     warp 2   tensor-memory allocation
//   warps 4-11  two groups of four; a thread owns one row of S (a key, or a query) and half of its 128 columns
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cstdint>
#include "../../include/ue5m3.h"
#include "attention.cuh"
#include "block_ops.h"
#include "common.cuh"

namespace ue5m3 {

__device__ int g_attention_backward_status = 0;

namespace {

constexpr int kThreads = 384;
constexpr int B128 = 128;

__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, long long limit) {
    return wait_inline(bar, parity, abort_flag, &g_attention_backward_status, limit);
}
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, long long limit) {
    return wait_warp(bar, parity, abort_flag, &g_attention_backward_status, limit);
}
__device__ __forceinline__ void drain_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, long long limit) {
    wait_inline(bar, parity, abort_flag, &g_attention_backward_status, limit, true);
}

// ------------------------------------------------------------------------------------------------ rows
struct RowParams {
    const __nv_bfloat16* o; const __nv_bfloat16* dout;
    int64_t o_stride[3], d_stride[3];               // batch, token, head
    const float* lse;
    float* lse2; float* delta;
    int q_len, q_pad, heads, dim;
    int64_t rows;                                   // batch * heads * q_pad
};
// Eight threads per query, 16 bytes of o and dout at a time.
__global__ void __launch_bounds__(256) attention_rows_kernel(const RowParams p) {
    asm volatile("griddepcontrol.launch_dependents;");          // the keys kernel sets itself up meanwhile
    const int64_t r = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 3;
    const int sub = threadIdx.x & 7;
    if (r >= p.rows) return;                        // whole groups of eight
    const int64_t bh = r / p.q_pad;
    const int i = (int)(r - bh * p.q_pad), b = (int)(bh / p.heads), h = (int)(bh - (int64_t)b * p.heads);
    float sum = 0.0f, lse2 = -INFINITY;
    bool seen = true;
    if (i < p.q_len) {
        const __nv_bfloat16* o = p.o + b * p.o_stride[0] + i * p.o_stride[1] + h * p.o_stride[2];
        const __nv_bfloat16* d = p.dout + b * p.d_stride[0] + i * p.d_stride[1] + h * p.d_stride[2];
        const float lse = p.lse[bh * p.q_len + i];
        uint4 u[2], w[2];                           // head dimension up to 128: all four loads at once
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int c = sub * 8 + k * 64;
            u[k] = c < p.dim ? ldg_nc_v4(o + c) : make_uint4(0, 0, 0, 0);
            w[k] = c < p.dim ? ldg_nc_v4(d + c) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            float x[8], y[8];
            unpack_bf16x8(u[k], x);
            unpack_bf16x8(w[k], y);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum = fmaf(x[j], y[j], sum);
        }
        if (lse != -INFINITY) lse2 = lse * -1.4426950408889634f;
        else seen = false;
    }
#pragma unroll
    for (int k = 4; k; k >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, k, 8);
    if (sub == 0) { p.lse2[r] = lse2; p.delta[r] = seen ? -sum : 0.0f; }       // a query that sees nothing: dout may hold anything
}

// ------------------------------------------------------------------------------------------------ shared pieces
template <int DP> struct Tiles {
    static constexpr int PANELS = DP / 64;
    static constexpr int TILE = 128 * DP * 2;
    static constexpr int PANEL = 128 * 128;
};
// tensor-memory columns: S, dP, then the accumulators
constexpr uint32_t COL_S = 0, COL_DP = 128, COL_ACC0 = 256, COL_ACC1 = 384;

// Writes a 128-row tile (this warp: 32 rows) of a binary32 accumulator times `f` as BF16 through shared memory.
template <int DP>
__device__ __forceinline__ void store_accumulator(uint32_t tm_lane, uint8_t* smem_gen, uint32_t smem, uint32_t tile_off, int q, int lane,
                                                  const CUtensorMap* map, float f, bool zero, int row0, int head, int b) {
#pragma unroll 1
    for (int c = 0; c < DP / 64; ++c) {
        const uint32_t off = tile_off + c * (128 * 128) + q * 4096;
        uint8_t* mine = smem_gen + off + lane * 128;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            uint32_t o[32];
            if (!zero) {
                tmem_ld32(tm_lane + c * 64 + half * 32, o);
                tmem_ld_wait();
            }
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                uint4 w = make_uint4(0, 0, 0, 0);
                if (!zero) {
                    w.x = pack_bf16x2(__uint_as_float(o[8 * v]) * f, __uint_as_float(o[8 * v + 1]) * f);
                    w.y = pack_bf16x2(__uint_as_float(o[8 * v + 2]) * f, __uint_as_float(o[8 * v + 3]) * f);
                    w.z = pack_bf16x2(__uint_as_float(o[8 * v + 4]) * f, __uint_as_float(o[8 * v + 5]) * f);
                    w.w = pack_bf16x2(__uint_as_float(o[8 * v + 6]) * f, __uint_as_float(o[8 * v + 7]) * f);
                }
                *reinterpret_cast<uint4*>(mine + (((half * 4 + v) ^ (lane & 7)) << 4)) = w;
            }
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) tma_store_4d(map, smem + off, c * 64, row0, head, b);
    }
    if (lane == 0) tma_store_wait_all();
}

// ------------------------------------------------------------------------------------------------ keys: dK and dV
template <int DP> struct KeySmem {
    using T = Tiles<DP>;
    static constexpr int STAGES = DP == 128 ? 2 : 4;
    static constexpr int RING = 2 * T::TILE;                          // K, V, then STAGES x (Q, dO)
    static constexpr int ROWS = RING + STAGES * 2 * T::TILE;          // STAGES x (128 lse2, 128 delta)
    static constexpr int BAR = ROWS + STAGES * 1024;
    static constexpr int SIZE = BAR + 256 + 1024;
};

// IDLE: queries that see no key may exist.  Looking for their tiles takes the issuing warp 1 to 2 % of the kernel's time (2501 tokens,
// window 511: 66.9 us against 65.8 of the whole backward pass), so calls without such queries do not.
// SINKS: key tile 0 holds keys that all queries see, many times the work of another tile, so its queries are shared out among the first
// `sink_parts` CTAs of a head, whose binary32 sums attention_sinks_kernel adds.
template <int DP, bool IDLE, bool SINKS>
__global__ void __launch_bounds__(kThreads, 1)
attention_keys_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_do,
                      const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                      const __grid_constant__ CUtensorMap map_dk, const __grid_constant__ CUtensorMap map_dv, const AttentionParams p,
                      const int kv_heads) {
    using T = Tiles<DP>;
    using M = KeySmem<DP>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* smem_gen = smem_raw + (smem - smem_u32(smem_raw));
    const uint32_t bars = smem + M::BAR;
    const uint32_t k_full = bars, v_full = bars + 8, s_full = bars + 16, dp_full = bars + 24, p_full = bars + 32, ds_full = bars + 40;
    const uint32_t acc_full = bars + 48, drain = bars + 56, p_half = bars + 64, q_full = bars + 72, q_empty = q_full + 8 * M::STAGES;
    const uint32_t d_full = q_empty + 8 * M::STAGES, d_empty = d_full + 8 * M::STAGES;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem_gen + M::BAR + 208);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem_gen + M::BAR + 212);

    // key tiles of one head side by side, those that most queries see (causal: the first) at the front
    const int bh_count = p.batch * kv_heads;
    const int bh = blockIdx.x % bh_count, turn = (int)(blockIdx.x / bh_count);
    const int j0 = SINKS ? max(turn - p.sink_parts + 1, 0) * B128 : turn * B128;
    const bool shared = SINKS && p.sink_parts > 1 && j0 == 0;         // this CTA has a part of tile 0
    const int b = bh / kv_heads, kvh = bh - b * kv_heads;
    const int keys = p.keys_of(b);
    const int j1 = min(j0 + B128, keys) - 1;                          // last key of the tile
    int lo = 0, hi = 0;                                               // query tiles
    if (j0 < keys) {
        const int a = p.query_lo(j0), z = SINKS ? max(p.query_hi_of<SINKS>(j0), p.query_hi(j1)) : p.query_hi(j1);
        if (z > a) { lo = a / B128; hi = (z + B128 - 1) / B128; }
    }
    if (shared) {
        const int first = lo, n = hi - lo;
        lo = first + (int)((int64_t)n * turn / p.sink_parts);
        hi = first + (int)((int64_t)n * (turn + 1) / p.sink_parts);
    }
    const int per_head = hi - lo, steps = per_head * p.group;

    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        *abort_flag = 0;
        const uint32_t ones[] = {k_full, v_full, s_full, dp_full, acc_full, drain};
        for (uint32_t x : ones) mbar_init(x, 1);
        mbar_init(p_half, 8);
        mbar_init(p_full, 8);
        mbar_init(ds_full, 8);
        for (int s = 0; s < M::STAGES; ++s) {
            mbar_init(q_full + 8 * s, 1); mbar_init(q_empty + 8 * s, 1);
            mbar_init(d_full + 8 * s, 1); mbar_init(d_empty + 8 * s, 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        prefetch_tmap(&map_q); prefetch_tmap(&map_do); prefetch_tmap(&map_k); prefetch_tmap(&map_v); prefetch_tmap(&map_dk); prefetch_tmap(&map_dv);
    }
    if (warp == 2) tmem_alloc1(smem_u32(tmem_slot), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    asm volatile("griddepcontrol.wait;" ::: "memory");           // the rows are there
    // The queries kernel needs nothing of this one and may fill its tail.  It does need the rows, and has no wait of its own in front of
    // them (that would be a wait for this grid's end): it starts once every CTA of this grid is past the line above, so once the rows grid
    // has ended and its writes have been performed at device scope, and reads them with loads of that scope.
    asm volatile("griddepcontrol.launch_dependents;");

    if (warp == 0) {
        // ------------------------------------------------------------------ copies
        if (lane == 0 && steps > 0 && !p.stall) {
            auto tile = [&](uint32_t dst, const CUtensorMap* m, uint32_t bar, int row, int head) {
#pragma unroll
                for (int c = 0; c < T::PANELS; ++c) tma_load_4d(dst + c * T::PANEL, m, bar, c * 64, row, head, b);
            };
            mbar_expect_tx(k_full, T::TILE);
            tile(smem, &map_k, k_full, j0, kvh);
            int it = 0;
            bool v_out = false;
            for (; it < steps; ++it) {
                const int s = it % M::STAGES, h = kvh * p.group + it / per_head, i0 = (lo + it % per_head) * B128;
                const uint32_t ph = (it / M::STAGES) & 1;
                const uint32_t st = smem + M::RING + s * 2 * T::TILE, rows = smem + M::ROWS + s * 1024;
                const int64_t row = ((int64_t)b * p.heads + h) * p.q_pad + i0;
                if (!wait(q_empty + 8 * s, ph ^ 1, abort_flag, p.wait_limit)) break;
                mbar_expect_tx(q_full + 8 * s, T::TILE + 1024);
                tile(st, &map_q, q_full + 8 * s, i0, h);
                bulk_load(rows, p.lse2 + row, 512, q_full + 8 * s);
                bulk_load(rows + 512, p.delta + row, 512, q_full + 8 * s);
                if (!v_out) {
                    mbar_expect_tx(v_full, T::TILE);
                    tile(smem + T::TILE, &map_v, v_full, j0, kvh);
                    v_out = true;
                }
                if (!wait(d_empty + 8 * s, ph ^ 1, abort_flag, p.wait_limit)) {
                    drain_wait(q_full + 8 * s, ph, abort_flag, p.wait_limit);
                    break;
                }
                mbar_expect_tx(d_full + 8 * s, T::TILE);
                tile(st + T::TILE, &map_do, d_full + 8 * s, i0, h);
            }
            drain_wait(k_full, 0, abort_flag, p.wait_limit);
            if (v_out) drain_wait(v_full, 0, abort_flag, p.wait_limit);
            for (int back = 0; back < M::STAGES && back < it; ++back) {
                const int j = it - 1 - back;
                drain_wait(q_full + 8 * (j % M::STAGES), (j / M::STAGES) & 1, abort_flag, p.wait_limit);
                drain_wait(d_full + 8 * (j % M::STAGES), (j / M::STAGES) & 1, abort_flag, p.wait_limit);
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer
        // S(0) dP(0) | dV(0) S(1) dK(0) dP(1) | dV(1) S(2) dK(1) dP(2) | ...   S is in order behind dV, which reads P out of its columns
        const bool elected = elect_one();
        const uint32_t tm = __shfl_sync(0xFFFFFFFFu, tmem, 0);
        const int n = uniform(steps), q_end = uniform(p.queries_end_of<SINKS>(keys)), i_first = uniform(lo) * B128, i_end = uniform(hi) * B128;
        bool ok = true;
        auto pass = [&](uint32_t bar, uint32_t parity) {   // the phase is complete, or `ok` is false in the whole warp
            if (!__all_sync(0xFFFFFFFFu, try_wait_cta(bar, parity))) ok = ok && __all_sync(0xFFFFFFFFu, wait(bar, parity, abort_flag, p.wait_limit));
            tc_fence_after();
        };
        // Q and dO of queries that see no key may hold anything (P and dS are zero there): they become zeros.  Rows behind q_len are.
        auto clean = [&](uint32_t tile, int i0) {
            if (!IDLE) return;
            if (i0 < p.first_query || (q_end < p.q_len && i0 + B128 > q_end)) keep_rows<DP>(smem_gen + M::RING + tile * T::TILE, p.first_query - i0, q_end - i0, lane);
        };
        int i0 = i_first;                                  // first query of the tile whose S was issued last
        const uint32_t k_low = desc_low_k(smem), v_low = desc_low_k(smem + T::TILE);
        const uint32_t q_k = desc_low_k(smem + M::RING), q_mn = desc_low_mn(smem + M::RING, T::PANEL);      // stage 0: Q, then dO
        constexpr uint32_t DO = T::TILE >> 4, STAGE = 2 * T::TILE >> 4;
        uint32_t s = 0, ph = 0;                            // ring stage of step it and its phase
        if (n > 0) {
            pass(k_full, 0);
            pass(q_full, 0);
            clean(0, i0);
            if (ok) issue_square<DP>(elected, tm + COL_S, k_low, q_k, s_full);
            pass(v_full, 0);
            pass(d_full, 0);
            clean(1, i0);
            if (ok) issue_square<DP>(elected, tm + COL_DP, v_low, q_k + DO, dp_full);
        }
        for (int it = 0; it < n && ok; ++it) {
            const uint32_t s1 = s + 1 == M::STAGES ? 0 : s + 1, ph1 = s + 1 == M::STAGES ? ph ^ 1 : ph;
            const bool more = it + 1 < n;
            pass(p_half, it & 1);                          // half of dV's product runs under the other half's exponentials
            if (!ok) break;
            issue_accumulate<DP, 0>(elected, tm + COL_ACC0, tm + COL_S, q_mn + s * STAGE + DO, it != 0);
            pass(p_full, it & 1);
            if (!ok) break;
            issue_accumulate<DP, 1>(elected, tm + COL_ACC0, tm + COL_S, q_mn + s * STAGE + DO, 1);
            issue_commit(elected, d_empty + 8 * s);
            if (more) {
                pass(q_full + 8 * s1, ph1);
                if (!ok) break;
                i0 = i0 + B128 == i_end ? i_first : i0 + B128;
                clean(2 * s1, i0);
                issue_square<DP>(elected, tm + COL_S, k_low, q_k + s1 * STAGE, s_full);
            }
            pass(ds_full, it & 1);
            if (!ok) break;
            issue_accumulate<DP>(elected, tm + COL_ACC1, tm + COL_DP, q_mn + s * STAGE, it != 0);
            issue_commit(elected, q_empty + 8 * s);
            if (more) {
                pass(d_full + 8 * s1, ph1);
                if (!ok) break;
                clean(2 * s1 + 1, i0);
                issue_square<DP>(elected, tm + COL_DP, v_low, q_k + s1 * STAGE + DO, dp_full);
            } else {
                issue_commit(elected, acc_full);
            }
            s = s1;
            ph = ph1;
        }
        if (elected) {
            umma1_commit(drain);
            drain_wait(drain, 0, abort_flag, p.wait_limit);
        }
        __syncwarp();
    } else if (warp >= 4) {
        // ------------------------------------------------------------------ P, dS and the outputs
        const int g = (warp - 4) >> 2, q = warp & 3;                  // column half, tensor-memory lane quarter
        const int key = j0 + q * 32 + lane;
        const uint32_t lane_base = tmem + ((uint32_t)(q * 32) << 16);
        const uint32_t ts = lane_base + COL_S + g * 64, td = lane_base + COL_DP + g * 64;
        const int q_lo = key < keys ? p.query_lo(key) : 0, q_hi = key < keys ? p.query_hi_of<SINKS>(key) : 0;
        // query tiles [plain_lo, plain_hi) see every key of this tile
        const int plain_lo = j0 + B128 <= keys ? (p.query_lo(j0 + B128 - 1) + B128 - 1) / B128 : hi;
        const int plain_hi = p.left >= 0 ? max(p.query_hi_of<SINKS>(SINKS && j0 == 0 ? min(p.sinks, B128 - 1) : j0), 0) / B128 : p.q_len / B128 + 1;
        const bool upper = p.left >= 0 || j0 + B128 > keys;
        // Some keys of the tile take no part (behind the sequence's end, in front of every window): what they hold may be NaN, and so then
        // is their dP.
        const bool idle_keys = j0 + B128 > keys || j0 < p.first_key;
        const f32x2 c2 = f2_pack(p.scale_log2, p.scale_log2);
        bool ok = true;
        for (int it = 0; it < steps; ++it) {
            const int qt = lo + it % per_head;
            const float* rows = reinterpret_cast<const float*>(smem_gen + M::ROWS + (it % M::STAGES) * 1024) + g * 64;
            const bool cut_lo = p.causal && qt < plain_lo, cut_hi = upper && (qt >= plain_hi || j0 + B128 > keys);
            const int base = qt * B128 + g * 64 - q_lo, width = q_hi - q_lo;
            if (!(ok = warp_wait(s_full, it & 1, abort_flag, p.wait_limit))) break;
            // this query tile's rows of lse2 and delta came with Q, whose barrier S waited for; seen by every thread
            if (!(ok = warp_wait(q_full + 8 * (it % M::STAGES), (it / M::STAGES) & 1, abort_flag, p.wait_limit))) break;
            tc_fence_after();
            uint32_t s[64];
            tmem_ld32(ts, s);
            tmem_ld32(ts + 32, s + 32);
            tmem_ld_wait();
            f32x2 pr[32];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
#pragma unroll
                for (int c = half * 32; c < half * 32 + 32; c += 4) {
                    const ulonglong2 e = *reinterpret_cast<const ulonglong2*>(rows + c);          // -lse2 of four queries
                    pr[c / 2] = ex2_pair(f2_fma(pair_of(s + c), c2, e.x));
                    pr[c / 2 + 1] = ex2_pair(f2_fma(pair_of(s + c + 2), c2, e.y));
                }
                if (cut_lo || cut_hi) hide_pairs<16>(pr + half * 16, -base - half * 32, width - base - half * 32, cut_lo, cut_hi);
                uint32_t pk[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) pk[i] = pack_pair(pr[half * 16 + i]);
                tmem_st16(ts + half * 16, pk);
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(half ? p_full : p_half);
            }
            if (!(ok = warp_wait(dp_full, it & 1, abort_flag, p.wait_limit))) break;
            tc_fence_after();
            uint32_t pk[32];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                uint32_t d[32];
                tmem_ld32(td + half * 32, d);
                tmem_ld_wait();
#pragma unroll
                for (int c = 0; c < 32; c += 4) {
                    const ulonglong2 e = *reinterpret_cast<const ulonglong2*>(rows + 128 + half * 32 + c);          // -delta
                    const f32x2 p0 = pr[half * 16 + c / 2], p1 = pr[half * 16 + c / 2 + 1];
                    pk[half * 16 + c / 2] = pack_pair(f2_mul(p0, f2_add(pair_of(d + c), e.x)));
                    pk[half * 16 + c / 2 + 1] = pack_pair(f2_mul(p1, f2_add(pair_of(d + c + 2), e.y)));
                }
            }
            if (idle_keys) {
#pragma unroll
                for (int i = 0; i < 32; ++i) pk[i] = q_lo < q_hi ? pk[i] : 0u;
            }
            tmem_st32(td, pk);
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(ds_full);
        }
        if (ok && steps > 0) {
            ok = warp_wait(acc_full, 0, abort_flag, p.wait_limit);
            tc_fence_after();
        }
        if (shared) {
            if (ok) {                                                 // the accumulators as they are, a thread its row
                float* dst = p.part_kv + ((((int64_t)turn * bh_count + bh) * 2 + g) * B128 + q * 32 + lane) * p.dim;
#pragma unroll 1
                for (int c = 0; c < DP; c += 32) {
                    uint32_t o[32];
#pragma unroll
                    for (int v = 0; v < 32; ++v) o[v] = 0u;
                    if (steps > 0) {
                        tmem_ld32(lane_base + (g == 0 ? COL_ACC0 : COL_ACC1) + c, o);
                        tmem_ld_wait();
                    }
#pragma unroll
                    for (int v = 0; v < 32; v += 4)
                        if (c + v < p.dim) *reinterpret_cast<uint4*>(dst + c + v) = make_uint4(o[v], o[v + 1], o[v + 2], o[v + 3]);
                }
            }
        } else
        // group 0 writes dV over V's tile, group 1 dK over K's: no MMA reads them any more (or they were never loaded)
        if (ok && j0 + q * 32 < p.k_len) {
            if (g == 0) store_accumulator<DP>(lane_base + COL_ACC0, smem_gen, smem, T::TILE, q, lane, &map_dv, 1.0f, steps == 0, j0 + q * 32, kvh, b);
            else store_accumulator<DP>(lane_base + COL_ACC1, smem_gen, smem, 0, q, lane, &map_dk, p.scale, steps == 0, j0 + q * 32, kvh, b);
        }
        tc_fence_before();
    }
    __syncthreads();
    if (warp == 2) { tc_fence_after(); tmem_dealloc1(tmem, 512); }
}

// ------------------------------------------------------------------------------------------------ queries: dQ
// Q and dO stay with the CTA as A operands, so they move into tensor memory at the start: S and dP then read only K and V from
// shared memory (with both operands there, a 128 x 128 product needs its whole bandwidth), and all of it is ring for K and V,
// whose copies take up to 1500 cycles.
template <int DP> struct QuerySmem {
    using T = Tiles<DP>;
    static constexpr int STAGES = DP == 128 ? 7 : 10;                 // ring: Q, dO, then K and V tiles
    static constexpr int BAR = STAGES * T::TILE;
    static constexpr int SIZE = BAR + 256 + 1024;
};
constexpr uint32_t COL_Q = 384, COL_DO = 448;                         // in place of the second accumulator

// PARTS: a CTA takes a share of the keys and leaves a binary32 sum for attention_sum_kernel.  SINKS: key tile 0 comes in front of
// the window's.
template <int DP, bool PARTS, bool SINKS>
__global__ void __launch_bounds__(kThreads, 1)
attention_queries_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_do,
                         const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                         const __grid_constant__ CUtensorMap map_dq, const AttentionParams p, const int q_tiles) {
    using T = Tiles<DP>;
    using M = QuerySmem<DP>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* smem_gen = smem_raw + (smem - smem_u32(smem_raw));
    const uint32_t bars = smem + M::BAR;
    const uint32_t qd_ready = bars, s_full = bars + 8, s_free = bars + 16, dp_full = bars + 24, ds_full = bars + 32, acc_full = bars + 40;
    const uint32_t drain = bars + 48, full = bars + 56, empty = full + 8 * M::STAGES;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem_gen + M::BAR + 240);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem_gen + M::BAR + 244);

    const int bh_count = p.batch * p.heads;
    const int part = PARTS ? (int)(blockIdx.x % p.parts) : 0, block = PARTS ? (int)(blockIdx.x / p.parts) : (int)blockIdx.x;
    const int bh = block % bh_count, i0 = (q_tiles - 1 - block / bh_count) * B128;
    const int b = bh / p.heads, h = bh - b * p.heads, kvh = h / p.group;
    const int keys = p.keys_of(b);
    const int i1 = min(i0 + B128, p.q_len) - 1;
    int lo = 0, hi = 0;                                               // key tiles
    {
        const int a = p.key_lo(i0), z = p.key_hi(i1, keys);
        if (z > a) { lo = a / B128; hi = (z + B128 - 1) / B128; }
        if (PARTS) {                                                  // this part's share of all key tiles
            const int n = (p.k_len + B128 - 1) / B128;
            lo = max(lo, (int)((int64_t)n * part / p.parts));
            hi = max(min(hi, (int)((int64_t)n * (part + 1) / p.parts)), lo);
        }
    }
    // SINKS: tile 0 comes first, for the sinks that lie in front of a row's window (and again where that begins in it)
    const int front = SINKS && part == 0 && p.key_hi(i1, keys) > 0 && p.key_lo(i1) > 0;
    const int steps = hi - lo + front;
    auto key_tile = [&](int it) { return SINKS ? (front && it == 0 ? 0 : lo + it - front) : lo + it; };

    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        *abort_flag = 0;
        const uint32_t ones[] = {s_full, dp_full, acc_full, drain}, eights[] = {qd_ready, s_free, ds_full};
        for (uint32_t x : ones) mbar_init(x, 1);
        for (uint32_t x : eights) mbar_init(x, 8);
        for (int s = 0; s < M::STAGES; ++s) { mbar_init(full + 8 * s, 1); mbar_init(empty + 8 * s, 1); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        prefetch_tmap(&map_q); prefetch_tmap(&map_do); prefetch_tmap(&map_k); prefetch_tmap(&map_v); prefetch_tmap(&map_dq);
    }
    if (PARTS) asm volatile("griddepcontrol.launch_dependents;");      // the adding kernel waits for this grid's end
    if (warp == 2) tmem_alloc1(smem_u32(tmem_slot), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;

    if (warp == 0) {
        // ------------------------------------------------------------------ copies
        if (lane == 0 && steps > 0 && !p.stall) {
            auto tile = [&](uint32_t dst, const CUtensorMap* m, uint32_t bar, int row, int head) {
#pragma unroll
                for (int c = 0; c < T::PANELS; ++c) tma_load_4d(dst + c * T::PANEL, m, bar, c * 64, row, head, b);
            };
            int it = 0;                                               // ring: Q, dO, K(0), V(0), K(1), V(1), ...
            for (; it < 2 * steps + 2; ++it) {
                const int s = it % M::STAGES;
                if (!wait(empty + 8 * s, ((it / M::STAGES) & 1) ^ 1, abort_flag, p.wait_limit)) break;
                mbar_expect_tx(full + 8 * s, T::TILE);
                if (it < 2) tile(smem + s * T::TILE, it ? &map_do : &map_q, full + 8 * s, i0, h);
                else tile(smem + s * T::TILE, (it & 1) ? &map_v : &map_k, full + 8 * s, key_tile((it >> 1) - 1) * B128, kvh);
            }
            for (int back = 0; back < M::STAGES && back < it; ++back) {
                const int j = it - 1 - back;
                drain_wait(full + 8 * (j % M::STAGES), (j / M::STAGES) & 1, abort_flag, p.wait_limit);
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer
        // S(0) dP(0) S(1) | dQ(0) dP(1) S(2) | dQ(1) dP(2) S(3) | ...   S is read into registers at once, so it runs a step ahead; dP is in
        // order behind the product that reads dS out of its columns
        const bool elected = elect_one();
        const uint32_t tm = __shfl_sync(0xFFFFFFFFu, tmem, 0);
        const int n = uniform(steps), n_keys = uniform(keys), first = uniform(lo), lead = SINKS ? uniform(front) : 0;
        bool ok = true;
        auto pass = [&](uint32_t bar, uint32_t parity) {   // the phase is complete, or `ok` is false in the whole warp
            if (!__all_sync(0xFFFFFFFFu, try_wait_cta(bar, parity))) ok = ok && __all_sync(0xFFFFFFFFu, wait(bar, parity, abort_flag, p.wait_limit));
            tc_fence_after();
        };
        const uint32_t r_k = desc_low_k(smem), r_mn = desc_low_mn(smem, T::PANEL);
        constexpr uint32_t TILE = T::TILE >> 4;
        uint32_t slot = 2, phase = 0;                      // of the next ring tile: K, V, K, V, ...
        auto next_tile = [&]() {
            const uint32_t s = slot;
            pass(full + 8 * s, phase);
            if (++slot == M::STAGES) { slot = 0; phase ^= 1; }
            return s;
        };
        auto clean_k = [&](int it, uint32_t s) {
            // keys behind the sequence's end and in front of every window may hold anything (dS is zero there): they become zeros
            const bool sinks = SINKS && lead && it == 0;
            const int at = (sinks ? 0 : first + it - lead) * B128, from = p.first_key - at, valid = n_keys - at;
            if ((p.k_lens && valid < B128) || from > 0) keep_rows<DP>(smem_gen + s * T::TILE, sinks ? 0 : from, sinks ? min(valid, p.sinks) : valid, lane);
        };
        uint32_t k0 = 0, k1 = 0, k2 = 0;                   // slots of K(it), K(it + 1), K(it + 2)
        auto issue_s = [&](int it) {
            const uint32_t s = next_tile();
            clean_k(it, s);
            if (it > 0) pass(s_free, (it - 1) & 1);        // the softmax warps have read S(it - 1)
            if (ok) issue_square_ts<DP>(elected, tm + COL_S, tm + COL_Q, r_k + s * TILE, s_full);
            return s;
        };
        auto issue_dp = [&]() {
            const uint32_t s = next_tile();
            if (ok) issue_square_ts<DP>(elected, tm + COL_DP, tm + COL_DO, r_k + s * TILE, dp_full);
            if (ok) issue_commit(elected, empty + 8 * s);
        };
        if (n > 0) {
            pass(qd_ready, 0);
            if (ok && elected) { mbar_arrive(empty); mbar_arrive(empty + 8); }
            __syncwarp();
            k0 = issue_s(0);
            issue_dp();
            if (n > 1 && ok) k1 = issue_s(1);
        }
        for (int it = 0; it < n && ok; ++it) {
            pass(ds_full, it & 1);
            if (!ok) break;
            issue_accumulate<DP>(elected, tm + COL_ACC0, tm + COL_DP, r_mn + k0 * TILE, it != 0);
            issue_commit(elected, empty + 8 * k0);
            if (it + 1 == n) issue_commit(elected, acc_full);
            else issue_dp();
            if (it + 2 < n && ok) k2 = issue_s(it + 2);
            k0 = k1;
            k1 = k2;
        }
        if (elected) {
            umma1_commit(drain);
            drain_wait(drain, 0, abort_flag, p.wait_limit);
        }
        __syncwarp();
    } else if (warp >= 4) {
        // ------------------------------------------------------------------ P, dS and the output
        const int g = (warp - 4) >> 2, q = warp & 3;
        const int row = i0 + q * 32 + lane;
        const uint32_t lane_base = tmem + ((uint32_t)(q * 32) << 16);
        const int k_lo = p.key_lo(row), k_hi = p.key_hi(row, keys), sinks_hi = SINKS ? p.sinks_hi(row, keys) : 0;
        const int plain_lo = p.left >= 0 ? (p.key_lo(i0 + B128 - 1) + B128 - 1) / B128 : 0;
        const int plain_hi = max(p.key_hi(i0, keys), 0) / B128;
        const bool idle_queries = i0 < p.first_query || i1 >= p.queries_end_of<SINKS>(keys);
        const int64_t at = ((int64_t)b * p.heads + h) * p.q_pad + row;
        const float nl = load_device(p.lse2 + at), nd = load_device(p.delta + at);         // visible: see launch_dependents in the keys kernel
        const f32x2 c2 = f2_pack(p.scale_log2, p.scale_log2), nl2 = f2_pack(nl, nl), nd2 = f2_pack(nd, nd);
        bool ok = true;
        if (steps > 0) {
            // group 0 moves Q into tensor memory, group 1 dO: a thread its own row, undoing the swizzle
            ok = warp_wait(full + 8 * g, 0, abort_flag, p.wait_limit);
            if (ok) {
#pragma unroll
                for (int c = 0; c < T::PANELS; ++c) {
                    const uint8_t* mine = smem_gen + g * T::TILE + c * T::PANEL + (q * 32 + lane) * 128;
                    uint32_t w[32];
#pragma unroll
                    for (int v = 0; v < 8; ++v) *reinterpret_cast<uint4*>(w + 4 * v) = *reinterpret_cast<const uint4*>(mine + ((v ^ (lane & 7)) << 4));
                    tmem_st32(lane_base + (g ? COL_DO : COL_Q) + c * 32, w);
                }
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(qd_ready);
            }
        }
        for (int it = 0; ok && it < steps; ++it) {
            const int kt = key_tile(it);
            const bool sinks = SINKS && front && it == 0, lower = !sinks && kt < plain_lo, upper = sinks || kt >= plain_hi;
            // columns from <= column < to are seen
            const int from = sinks ? 0 : k_lo - kt * B128 - g * 64, to = (sinks ? sinks_hi : k_hi - kt * B128) - g * 64;
            const uint32_t ts = lane_base + COL_S + g * 64, td = lane_base + COL_DP + g * 64;
            if (!(ok = warp_wait(s_full, it & 1, abort_flag, p.wait_limit))) break;
            tc_fence_after();
            uint32_t s[64];
            tmem_ld32(ts, s);
            tmem_ld32(ts + 32, s + 32);
            tmem_ld_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(s_free);
            f32x2 pr[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) pr[i] = ex2_pair(f2_fma(pair_of(s + 2 * i), c2, nl2));
            if (lower || upper) hide_pairs<32>(pr, from, to, lower, upper);
            // values, and dO of queries, that take no part may be NaN, and so then is dP
            const bool idle = (p.k_lens && (kt + 1) * B128 > keys) || kt * B128 < p.first_key || idle_queries;
            if (!(ok = warp_wait(dp_full, it & 1, abort_flag, p.wait_limit))) break;
            tc_fence_after();
            uint32_t pk[32];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                uint32_t d[32];
                tmem_ld32(td + half * 32, d);
                tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const f32x2 pp = pr[half * 16 + i];
                    f32x2 x = f2_mul(pp, f2_add(pair_of(d + 2 * i), nd2));
                    if (idle) x = where_p(pp, x);
                    pk[half * 16 + i] = pack_pair(x);
                }
            }
            tmem_st32(td, pk);
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(ds_full);
        }
        if (ok && steps > 0) {
            ok = warp_wait(acc_full, 0, abort_flag, p.wait_limit);
            tc_fence_after();
        }
        if (PARTS) {
            if (ok && g == 0) {
                float* dst = p.part_o + ((((int64_t)part * p.batch + b) * p.heads + h) * p.q_len + row) * p.dim;
#pragma unroll 1
                for (int c = 0; c < DP; c += 32) {
                    uint32_t o[32];
                    if (steps > 0) {
                        tmem_ld32(lane_base + COL_ACC0 + c, o);
                        tmem_ld_wait();
                    }
                    if (row < p.q_len)
#pragma unroll
                        for (int v = 0; v < 32; v += 4)
                            if (c + v < p.dim)
                                *reinterpret_cast<float4*>(dst + c + v) = steps == 0 ? make_float4(0.0f, 0.0f, 0.0f, 0.0f)
                                    : make_float4(__uint_as_float(o[v]), __uint_as_float(o[v + 1]), __uint_as_float(o[v + 2]), __uint_as_float(o[v + 3]));
                }
            }
        } else if (ok && g == 0 && i0 + q * 32 < p.q_len)
            store_accumulator<DP>(lane_base + COL_ACC0, smem_gen, smem, 0, q, lane, &map_dq, p.scale, steps == 0, i0 + q * 32, h, b);
        tc_fence_before();
    }
    __syncthreads();
    if (warp == 2) { tc_fence_after(); tmem_dealloc1(tmem, 512); }
    asm volatile("griddepcontrol.wait;" ::: "memory");           // this grid ends after the keys kernel: what follows is behind both
}

// dq of a query from its parts, added in order: four values per thread.
__global__ void __launch_bounds__(256) attention_sum_kernel(const AttentionParams p, __nv_bfloat16* dq, const int64_t batch_stride,
                                                            const int64_t token_stride, const int64_t head_stride) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int per_row = p.dim / 4;
    const int64_t rows = (int64_t)p.batch * p.heads * p.q_len, at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= rows * per_row) return;
    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int k = 0; k < p.parts; ++k) {
        const float4 v = reinterpret_cast<const float4*>(p.part_o)[k * rows * per_row + at];
        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
    const int64_t r = at / per_row, i = r % p.q_len, bh = r / p.q_len, b = bh / p.heads, h = bh - b * p.heads;
    *reinterpret_cast<uint2*>(dq + b * batch_stride + i * token_stride + h * head_stride + (at - r * per_row) * 4) =
        make_uint2(pack_bf16x2(s.x * p.scale, s.y * p.scale), pack_bf16x2(s.z * p.scale, s.w * p.scale));
}

// dk and dv of key tile 0 from the parts its queries were shared out into, added in order: four values per thread.
struct SinkOutputs { __nv_bfloat16* out[2]; int64_t stride[2][3]; };       // dv, dk: batch, token, head
__global__ void __launch_bounds__(256) attention_sinks_kernel(const AttentionParams p, const SinkOutputs o) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int per_row = p.dim / 4;
    const int64_t all = (int64_t)p.batch * p.kv_heads * 2 * B128 * per_row, at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= all) return;
    const int64_t row = at / per_row;
    const int c = (int)(at - row * per_row) * 4, key = (int)(row % B128), which = (int)(row / B128 % 2);
    if (key >= p.k_len) return;
    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int k = 0; k < p.sink_parts; ++k) {
        const float4 v = reinterpret_cast<const float4*>(p.part_kv)[k * all + at];
        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
    const float f = which ? p.scale : 1.0f;
    const int64_t bh = row / (2 * B128), b = bh / p.kv_heads, h = bh - b * p.kv_heads;
    *reinterpret_cast<uint2*>(o.out[which] + b * o.stride[which][0] + key * o.stride[which][1] + h * o.stride[which][2] + c) =
        make_uint2(pack_bf16x2(s.x * f, s.y * f), pack_bf16x2(s.z * f, s.w * f));
}

struct Maps { CUtensorMap q, dout, k, v, dq, dk, dv; };

// A launch that may begin before the one in front of it has ended (`early`): the kernel says itself what it waits for.
template <typename... Args>
int launch(void (*kernel)(Args...), int64_t grid, int threads, int smem, bool early, cudaStream_t st, Args... args) {
    if (grid > 0x7FFFFFFF) return UE5M3_ERR_UNSUPPORTED;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = early ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess ? UE5M3_OK : UE5M3_ERR_CUDA;
}

template <int DP, bool PARTS, bool SINKS>
int run_queries(const Maps& m, const AttentionParams& p, int64_t grid, int q_tiles, bool early, cudaStream_t st) {
    static std::atomic<int> granted[64];
    if (allow_smem(attention_queries_kernel<DP, PARTS, SINKS>, QuerySmem<DP>::SIZE, granted) != cudaSuccess) return UE5M3_ERR_CUDA;
    return launch(attention_queries_kernel<DP, PARTS, SINKS>, grid, kThreads, QuerySmem<DP>::SIZE, early, st, m.q, m.dout, m.k, m.v, m.dq, p, q_tiles);
}

template <int DP, bool IDLE, bool SINKS>
int run_keys(const Maps& m, const AttentionParams& p, int64_t grid, int kv_heads, bool early, cudaStream_t st) {
    static std::atomic<int> granted[64];
    if (allow_smem(attention_keys_kernel<DP, IDLE, SINKS>, KeySmem<DP>::SIZE, granted) != cudaSuccess) return UE5M3_ERR_CUDA;
    return launch(attention_keys_kernel<DP, IDLE, SINKS>, grid, kThreads, KeySmem<DP>::SIZE, early, st, m.q, m.dout, m.k, m.v, m.dk, m.dv, p, kv_heads);
}

template <int DP, bool SINKS>
int run(const ue5m3_attention_shape& s, const ue5m3_heads& dq, const ue5m3_heads& dk, const ue5m3_heads& dv, const Maps& m, const AttentionParams& p,
        cudaStream_t st) {
    const int64_t k_tiles = (s.k_len + 127) / 128, q_tiles = (s.q_len + 127) / 128;
    const int64_t ck = k_tiles > 0 ? (k_tiles + p.sink_parts - 1) * s.batch * s.kv_heads : 0, cq = q_tiles * s.batch * s.heads * p.parts;
    if (ck > 0) {
        // queries in front of every key, or with a window that begins behind the end of their sequence
        const bool idle = p.first_query > 0 || (!SINKS && p.left >= 0 && p.k_lens);
        const int r = idle ? run_keys<DP, true, SINKS>(m, p, ck, (int)s.kv_heads, cq > 0, st) : run_keys<DP, false, SINKS>(m, p, ck, (int)s.kv_heads, cq > 0, st);
        if (r != UE5M3_OK) return r;
    }
    if (cq == 0) return UE5M3_OK;
    const int r = p.parts == 1 ? run_queries<DP, false, SINKS>(m, p, cq, (int)q_tiles, ck > 0, st) : run_queries<DP, true, SINKS>(m, p, cq, (int)q_tiles, ck > 0, st);
    if (r != UE5M3_OK) return r;
    if (p.parts > 1) {
        const int64_t rows = s.batch * s.heads * s.q_len;
        const int e = launch(attention_sum_kernel, (rows * (s.head_dim / 4) + 255) / 256, 256, 0, true, st, p, static_cast<__nv_bfloat16*>(dq.data),
                             dq.batch_stride, dq.token_stride, dq.head_stride);
        if (e != UE5M3_OK) return e;
    }
    if (p.sink_parts == 1) return UE5M3_OK;
    const SinkOutputs o{{static_cast<__nv_bfloat16*>(dv.data), static_cast<__nv_bfloat16*>(dk.data)},
                        {{dv.batch_stride, dv.token_stride, dv.head_stride}, {dk.batch_stride, dk.token_stride, dk.head_stride}}};
    return launch(attention_sinks_kernel, (s.batch * s.kv_heads * 2 * B128 * (s.head_dim / 4) + 255) / 256, 256, 0, true, st, p, o);
}

}  // namespace

// As attention_splits, for the tiles of 128 queries of the queries kernel, but no part below 16 key tiles: this kernel runs into the
// tail of the keys kernel, so SMs are rarely idle for it.  Whole against shared out, us of the whole backward pass: one query on
// 8192 keys, 32 heads 147 / 89; 100 on 8192, 16 heads 129 / 82.  Smaller parts: 600 on 2000, 8 heads 32.4 / 36.0 (of 8 tiles), 1 on
// 512, 8 heads 13.1 / 18.0 and 1000 on 1000, 8 heads 20.6 / 28.0 (of 2).
int attention_backward_splits(const ue5m3_attention_shape& s) {
    const int64_t ctas = (s.q_len + 127) / 128 * s.batch * s.heads, tiles = (s.k_len + 127) / 128;
    if (ctas == 0 || ctas > 74) return 1;
    const int64_t fill = 148 / ctas, most = tiles / 16;
    const int64_t n = fill < most ? fill : most;
    return n < 1 ? 1 : (int)n;
}

// Parts into which the queries of key tile 0 are shared out: as many as leave none longer than another tile's window, or than half of what
// every SM has to do in all (these parts start first).
int attention_sink_parts(const ue5m3_attention_shape& s, int64_t sinks) {
    const AttentionParams p = attention_params(s, sinks);
    if (p.sinks == 0 || s.q_len == 0 || s.k_len == 0 || s.batch == 0) return 1;
    const int64_t q_tiles = (s.q_len + 127) / 128 - p.query_lo(0) / 128, k_tiles = (s.k_len + 127) / 128;
    const int64_t window = std::min<int64_t>(q_tiles, (p.left + 127) / 128 + 1);
    const int64_t most = std::max<int64_t>(window, k_tiles * s.batch * s.kv_heads * window / (2 * 148));
    return (int)std::max<int64_t>(1, (q_tiles + most - 1) / most);
}

int launch_attention_backward(const ue5m3_attention_shape& s, int64_t sinks, const ue5m3_heads& dout, const ue5m3_heads& q, const ue5m3_heads& k,
                              const ue5m3_heads& v, const ue5m3_heads& o, const float* lse, const ue5m3_heads& dq,
                              const ue5m3_heads& dk, const ue5m3_heads& dv, float* workspace, cudaStream_t st, const StallTest& stall) {
    if (s.batch == 0 || (s.q_len == 0 && s.k_len == 0)) return UE5M3_OK;
    Maps m;
    const int64_t B = s.batch, D = s.head_dim;
    if (s.q_len > 0 && (!make_heads_map(&m.q, q, B, s.q_len, s.heads, D, 128) || !make_heads_map(&m.dout, dout, B, s.q_len, s.heads, D, 128) ||
                        !make_heads_map(&m.dq, dq, B, s.q_len, s.heads, D, 32)))
        return UE5M3_ERR_CUDA;
    if (s.k_len > 0 && (!make_heads_map(&m.k, k, B, s.k_len, s.kv_heads, D, 128) || !make_heads_map(&m.v, v, B, s.k_len, s.kv_heads, D, 128) ||
                        !make_heads_map(&m.dk, dk, B, s.k_len, s.kv_heads, D, 32) || !make_heads_map(&m.dv, dv, B, s.k_len, s.kv_heads, D, 32)))
        return UE5M3_ERR_CUDA;
    if (s.q_len == 0) m.q = m.dout = m.k;                  // an empty side is never read
    if (s.k_len == 0) m.k = m.v = m.q;
    AttentionParams p = attention_params(s, sinks);
    if (stall.wait_limit > 0) { p.wait_limit = stall.wait_limit; p.stall = 1; }
    if (s.q_len > 0) {
        RowParams r{};
        r.o = static_cast<const __nv_bfloat16*>(o.data); r.dout = static_cast<const __nv_bfloat16*>(dout.data);
        r.o_stride[0] = o.batch_stride; r.o_stride[1] = o.token_stride; r.o_stride[2] = o.head_stride;
        r.d_stride[0] = dout.batch_stride; r.d_stride[1] = dout.token_stride; r.d_stride[2] = dout.head_stride;
        r.lse = lse;
        r.q_len = (int)s.q_len; r.q_pad = p.q_pad; r.heads = (int)s.heads; r.dim = (int)D;
        r.rows = B * s.heads * p.q_pad;
        r.lse2 = workspace; r.delta = workspace + r.rows;
        p.lse2 = r.lse2; p.delta = r.delta;
        p.parts = attention_backward_splits(s);
        p.part_o = workspace + 2 * r.rows;
        p.sink_parts = attention_sink_parts(s, sinks);
        p.part_kv = p.part_o + (p.parts > 1 ? p.parts * B * s.heads * s.q_len * D : 0);
        const int64_t grid = (r.rows * 8 + 255) / 256;
        if (grid > 0x7FFFFFFF) return UE5M3_ERR_UNSUPPORTED;
        attention_rows_kernel<<<(unsigned)grid, 256, 0, st>>>(r);
        if (cudaGetLastError() != cudaSuccess) return UE5M3_ERR_CUDA;
    }
    if (p.sinks > 0) return D <= 64 ? run<64, true>(s, dq, dk, dv, m, p, st) : run<128, true>(s, dq, dk, dv, m, p, st);
    return D <= 64 ? run<64, false>(s, dq, dk, dv, m, p, st) : run<128, false>(s, dq, dk, dv, m, p, st);
}

int read_and_clear_attention_backward_status() {
    if (cudaDeviceSynchronize() != cudaSuccess) return UE5M3_ERR_CUDA;
    int v = 0;
    if (cudaMemcpyFromSymbol(&v, g_attention_backward_status, sizeof(int)) != cudaSuccess) return UE5M3_ERR_CUDA;
    if (v != 0) {
        const int zero = 0;
        if (cudaMemcpyToSymbol(g_attention_backward_status, &zero, sizeof(int)) != cudaSuccess) return UE5M3_ERR_CUDA;
    }
    return v;
}

}  // namespace ue5m3
