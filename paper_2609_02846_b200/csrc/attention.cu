// Attention, forward, for sm_100a:  o_i = sum_j softmax_j(scale q_i . k_j) v_j over the keys query i sees.
//
// One pass over the keys per tile of queries, with a running maximum m and sum l of every row (binary32):
//     p_j = 2^(s_j - m) with s = scale log2(e) q.k;  l = l 2^(m_old - m) + sum p_j;  O = O 2^(m_old - m) + P V;  o = O / l
//
// A CTA owns two tiles of 128 queries of one head and walks the keys 128 at a time.  Both products run on the tensor core with
// accumulators in tensor memory: S = Q K^T from shared memory, O += P V with P (BF16) taken from tensor memory, where it
// overwrites S.  While one tile's softmax warps turn S into P, the tensor core works for the other tile.  Warp roles:
//   warp 0      tensor-memory allocation; copies: Q once, then K and V tiles through a ring
//   warp 1      issues the MMAs (the whole warp runs the loop, one elected lane issues)
//   warps 4-7 / 8-11   softmax of tile 0 / 1: thread = query row, so maxima and sums need no exchange between threads; a thread
//               holds a whole row of S (128 scores), so these warps take registers over from the first four
// The running maximum that scales O is raised only when a row's maximum grew by more than 2^8 (then O is rescaled in tensor
// memory by its softmax warps): p stays below 2^8, l and O in binary32 lose nothing, and o = O / l does not depend on m.
// P is rounded to BF16 because the tensor core takes both operands of a product in one type and V is BF16 (binary32 operands would run at
// half of the rate and take twice the room): 2^-8 of each p at most, while l adds the p as they were.  Against 64 bits o is off by a
// relative 0.0018 to 0.0022 of its norm, of which rounding o itself makes 0.0017.
// Tensor memory: S0, S1 (128 columns each), O0, O1 (head dimension columns each).
//
// Per pair of tiles (2 x 128 queries, 128 keys, dimension 128) the products take 2048 cycles, the exponentials 2048 on their own unit,
// and S with both operands in shared memory uses all of its bandwidth; a step takes 2775, because a tile's softmax (1700) and its
// products (1000) follow one another and two tiles in flight are all that tensor memory has room for.  2 x 4096 tokens, 32 / 8 heads
// of 128, causal: 232 us in short bursts, 1184 TFLOP/s (0.72 of the measured burst rate of a BF16 product); one call after the other,
// under the power cap, 272 to 276 us, 1010 TFLOP/s (0.73 of the sustained rate).
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <algorithm>
#include <cmath>
#include <cstdint>
#include "../../include/ue5m3.h"
#include "attention.cuh"
#include "block_ops.h"

namespace ue5m3 {

__device__ int g_attention_status = 0;

namespace {

constexpr int kThreads = 384;
constexpr int BQ = 128, BK = 128;
constexpr float kRaise = 8.0f;                            // log2 of the growth of a row's maximum that is tolerated

template <int DP> struct Tiles {                          // DP: head dimension padded to 64 or 128
    static constexpr int PANELS = DP / 64;
    static constexpr int TILE = 128 * DP * 2;             // bytes of a tile of 128 rows
    static constexpr int PANEL = 128 * 128;
    static constexpr int RING = DP == 128 ? 5 : 9;        // K and V tiles in the ring, odd
    static constexpr int PAIRS = (RING + 1) / 2;          // barriers: one for V of a key tile and K of the next together
    static constexpr int SMEM_BAR = (2 + RING) * TILE;
    static constexpr int SMEM = SMEM_BAR + 256 + 1024;    // + alignment slack
};

__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, long long limit) {
    return wait_inline(bar, parity, abort_flag, &g_attention_status, limit);
}
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, long long limit) {
    return wait_warp(bar, parity, abort_flag, &g_attention_status, limit);
}
__device__ __forceinline__ void drain_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, long long limit) {
    wait_inline(bar, parity, abort_flag, &g_attention_status, limit, true);
}

struct OutputParams { __nv_bfloat16* o; int64_t batch_stride, token_stride, head_stride; };

// One piece of work: two tiles of 128 queries of one head (PARTS: on a share of the keys).  PACK (few queries per head): a tile holds
// the queries of `pack` heads that share keys, row = head * q_len + query; h is the first of them in tile 0, tile 1 goes on behind.
struct Item {
    int b, h, h_end, kvh, part, q0, keys;                 // h_end: heads of the group of h end there (PACK)
    int lo[2], hi[2];                                     // key tiles of the two query tiles
    int first, last;                                      // ... and of both together
    __device__ __forceinline__ bool on(int t) const { return hi[t] > lo[t]; }
};
// Heads fastest (heads that share keys run side by side), long query tiles first.
template <bool PARTS, bool PACK>
__device__ __forceinline__ Item item_of(const AttentionParams& p, int index, int q_tiles) {
    Item w;
    w.part = PARTS ? index % p.parts : 0;
    const int heads = PACK ? p.kv_heads : p.heads, bh_count = p.batch * heads, block = PARTS ? index / p.parts : index;
    const int turn = block / bh_count, bh = block - turn * bh_count;
    w.b = bh / heads;
    w.h = bh - w.b * heads;
    w.h_end = 0;
    if (PACK) {
        w.kvh = w.h;
        w.h = w.kvh * p.group + turn * 2 * p.pack;
        w.h_end = (w.kvh + 1) * p.group;
        w.q0 = 0;
    } else {
        w.kvh = w.h / p.group;
        w.q0 = (q_tiles - 1 - turn) * 2 * BQ;
    }
    w.keys = p.keys_of(w.b);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int r0 = PACK ? 0 : w.q0 + t * BQ, r1 = min(r0 + BQ, p.q_len) - 1;
        const int a = p.key_lo(r0), z = (PACK ? w.h + t * p.pack < w.h_end : r0 < p.q_len) ? p.key_hi(r1, w.keys) : 0;
        w.lo[t] = a / BK;
        w.hi[t] = z > a ? (z + BK - 1) / BK : w.lo[t];
        if (PARTS) {                                      // this part's share of all key tiles
            const int n = (p.k_len + BK - 1) / BK;
            w.lo[t] = max(w.lo[t], (int)((int64_t)n * w.part / p.parts));
            w.hi[t] = max(min(w.hi[t], (int)((int64_t)n * (w.part + 1) / p.parts)), w.lo[t]);
        }
    }
    w.first = w.on(0) ? (w.on(1) ? min(w.lo[0], w.lo[1]) : w.lo[0]) : w.lo[1];
    w.last = w.on(0) ? (w.on(1) ? max(w.hi[0], w.hi[1]) : w.hi[0]) : (w.on(1) ? w.hi[1] : w.first);
    return w;
}

// Persistent: a CTA takes items in turn (forwards, then backwards, so that long and short ones even out) and every role walks them
// by itself: the next item's Q and keys are copied and its first S computed while the softmax warps still write this one's output.
// 233 us at 2 x 4096 tokens against 240 with a CTA per item.
// PARTS: binary32 results for attention_join_kernel.
template <int DP, bool PARTS, bool PACK>
__global__ void __launch_bounds__(kThreads, 1)
attention_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                 const __grid_constant__ CUtensorMap map_v, const AttentionParams p, const OutputParams out, const int q_tiles, const int items) {
    using T = Tiles<DP>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* smem_gen = smem_raw + (smem - smem_u32(smem_raw));
    const uint32_t ring = smem + 2 * T::TILE;
    const uint32_t bars = smem + T::SMEM_BAR;
    const uint32_t q_full = bars, kv_full = bars + 16, kv_empty = kv_full + 8 * T::PAIRS;
    const uint32_t s_full = bars + 96, p_full = bars + 112 /* two halves per tile */, o_full = bars + 144, q_empty = bars + 160, o_empty = bars + 176;
    const uint32_t drain = bars + 192;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem_gen + T::SMEM_BAR + 200);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem_gen + T::SMEM_BAR + 204);
    const int G = gridDim.x;
    auto item_at = [&](int turn) { return turn * G + ((turn & 1) ? G - 1 - (int)blockIdx.x : (int)blockIdx.x); };

    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        *abort_flag = 0;
        for (int t = 0; t < 2; ++t) {
            mbar_init(q_full + 8 * t, 1);
            mbar_init(s_full + 8 * t, 1);
            mbar_init(p_full + 16 * t, 4);
            mbar_init(p_full + 16 * t + 8, 4);
            mbar_init(o_full + 8 * t, 1);
            mbar_init(q_empty + 8 * t, 1);
            mbar_init(o_empty + 8 * t, 4);
        }
        for (int s = 0; s < T::PAIRS; ++s) {
            mbar_init(kv_full + 8 * s, 2);                // V's copies and K's
            mbar_init(kv_empty + 8 * s, 1);
        }
        mbar_init(drain, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        prefetch_tmap(&map_q); prefetch_tmap(&map_k); prefetch_tmap(&map_v);
    }
    if (PARTS) asm volatile("griddepcontrol.launch_dependents;");    // the joining kernel waits for this grid's end
    if (warp == 0) tmem_alloc1(smem_u32(tmem_slot), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;

    if (warp < 4) registers_few();
    if (warp == 0) {
        // ------------------------------------------------------------------ copies
        if (lane == 0) {
            // Pair i of an item: V of key tile first + i - 1 (none in the first) and K of key tile first + i (none in the last).  Pairs are
            // numbered through all items; pair n's tiles are number 2n - 1 and 2n of the ring, of which the one takes the place of pair
            // n - PAIRS's K, the other that of the next pair's V.
            auto emptied = [&](int pair) { return pair < 0 || wait(kv_empty + 8 * (pair % T::PAIRS), (pair / T::PAIRS) & 1, abort_flag, p.wait_limit); };
            int n = 0, q_uses[2] = {0, 0};
            bool go = !p.stall;
            for (int turn = 0, index; go && (index = item_at(turn)) < items; ++turn) {
                const Item w = item_of<PARTS, PACK>(p, index, q_tiles);
                const int pairs = w.last > w.first ? w.last - w.first + 1 : 0;
                auto load = [&](int tile_n, const CUtensorMap* m, uint32_t bar, int tile) {
                    mbar_expect_tx(bar, T::TILE);
#pragma unroll
                    for (int c = 0; c < T::PANELS; ++c)
                        tma_load_4d(ring + (tile_n % T::RING) * T::TILE + c * T::PANEL, m, bar, c * 64, tile * BK, w.kvh, w.b);
                };
#pragma unroll
                for (int t = 0; t < 2; ++t)
                    if (go && w.on(t)) {
                        go = wait(q_empty + 8 * t, (q_uses[t] & 1) ^ 1, abort_flag, p.wait_limit);
                        if (!go) break;
                        ++q_uses[t];
                        mbar_expect_tx(q_full + 8 * t, PACK ? p.pack * p.q_len * DP * 2 : T::TILE);
#pragma unroll
                        for (int c = 0; c < T::PANELS; ++c)
                            tma_load_4d(smem + t * T::TILE + c * T::PANEL, &map_q, q_full + 8 * t, c * 64, PACK ? 0 : w.q0 + t * BQ, PACK ? w.h + t * p.pack : w.h, w.b);
                    }
                for (int i = 0; go && i < pairs; ++i, ++n) {
                    const uint32_t bar = kv_full + 8 * (n % T::PAIRS);
                    if (!(go = emptied(n - T::PAIRS))) break;
                    if (i > 0) load(2 * n - 1, &map_v, bar, w.first + i - 1);
                    else mbar_arrive(bar);
                    go = emptied(n - T::PAIRS + 1);
                    if (go && i + 1 < pairs) load(2 * n, &map_k, bar, w.first + i);
                    else mbar_arrive(bar);
                }
            }
            // copies in flight land before the shared memory goes away, whatever the other roles did
#pragma unroll
            for (int t = 0; t < 2; ++t)
                if (q_uses[t] > 0) drain_wait(q_full + 8 * t, (q_uses[t] - 1) & 1, abort_flag, p.wait_limit);
            for (int back = 0; back < T::PAIRS && back < n; ++back) {
                const int j = n - 1 - back;
                drain_wait(kv_full + 8 * (j % T::PAIRS), (j / T::PAIRS) & 1, abort_flag, p.wait_limit);
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer
        // Per key tile j:  PV0 S0' | PV1 S1'  with S' = S of key tile j + 1.  The two query tiles stay half a period apart by this
        // order (an issuing warp per tile let their softmax phases fall together: 293 us against 260 at 2 x 4096 tokens).  What this
        // warp does between two products is idle time of the tensor core, so a pair of tiles has one barrier, waited for once and
        // released once, right behind the last product that reads it (260 us -> 240).
        const bool elected = elect_one();
        const uint32_t tm = __shfl_sync(0xFFFFFFFFu, tmem, 0);
        constexpr uint32_t id_s = umma_idesc(BK, false), id_o = umma_idesc(DP, true);
        bool ok = true;
        auto wait_all = [&](uint32_t bar, uint32_t parity) {
            if (!__all_sync(0xFFFFFFFFu, try_wait_cta(bar, parity))) ok = ok && __all_sync(0xFFFFFFFFu, wait(bar, parity, abort_flag, p.wait_limit));
            return ok;
        };
        uint32_t slot = 0, phase = 0, v_tile = T::RING - 1;          // of the next pair: barrier, and ring tile of its V
        auto next_pair = [&](const Item& w, int j) {       // waits for the pair with V of key tile j
            wait_all(kv_full + 8 * slot, phase);
            if (++slot == T::PAIRS) { slot = 0; phase ^= 1; }
            // values behind the sequence's end and in front of every window may hold anything: they become zeros
            const int from = p.first_key - j * BK, valid = w.keys - j * BK;
            if (j >= w.first && ((p.k_lens && valid < BK) || from > 0)) keep_rows<DP>(smem_gen + (2 + v_tile) * T::TILE, from, valid, lane);
            const uint32_t v = v_tile;
            v_tile = v + 2 >= T::RING ? v + 2 - T::RING : v + 2;
            return v;
        };
        auto k_tile = [&](uint32_t v) { return v + 1 == T::RING ? 0 : v + 1; };
        const uint64_t qd = umma_smem_desc(smem), kd0 = umma_smem_desc(ring), vd0 = umma_mn_desc(ring, T::PANEL);
        auto issue_s = [&](int t, uint32_t tile) {         // S_t = Q_t K^T
            if (elected) {
                const uint64_t kd = kd0 + tile * (T::TILE >> 4);
#pragma unroll
                for (int k = 0; k < DP / 16; ++k) {
                    const uint32_t off = (k / 4) * (T::PANEL >> 4) + (k % 4) * 2;
                    umma1_ss(tm + t * BK, qd + t * (T::TILE >> 4) + off, kd + off, id_s, k != 0);
                }
                umma1_commit(s_full + 8 * t);
            }
            __syncwarp();
        };
        uint32_t np[2] = {0, 0}, uses[2] = {0, 0};         // probability tiles consumed and items begun, per query tile
        auto issue_o = [&](int t, uint32_t tile, int half, bool begin, bool end) {     // O_t (+)= P_t V, 64 keys
            if (!wait_all(p_full + 16 * t + 8 * half, np[t] & 1)) return;
            tc_fence_after();
            if (elected) {
                const uint64_t vd = vd0 + tile * (T::TILE >> 4);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    umma1_ts(tm + 2 * BK + t * 128, tm + t * BK + half * 32 + k * 8, vd + (half * 4 + k) * (2048 >> 4), id_o, !begin || half != 0 || k != 0);
                if (end) umma1_commit(o_full + 8 * t);
            }
            __syncwarp();
        };
        uint32_t done = 0;                                 // barrier of the pair whose products are all issued
        auto release = [&]() {
            if (elected) umma1_commit(kv_empty + 8 * done);
            if (++done == T::PAIRS) done = 0;
        };
        for (int turn = 0, index; ok && (index = item_at(turn)) < items; ++turn) {
            const Item w = item_of<PARTS, PACK>(p, index, q_tiles);
            if (w.last <= w.first) continue;
            const uint32_t k0 = k_tile(next_pair(w, w.first - 1));
#pragma unroll
            for (int t = 0; t < 2; ++t)
                if (ok && w.on(t)) {
                    wait_all(q_full + 8 * t, uses[t] & 1);
                    ++uses[t];
                    if (ok && w.lo[t] == w.first) {
                        issue_s(t, k0);
                        if (w.hi[t] == w.first + 1 && elected) umma1_commit(q_empty + 8 * t);
                    }
                }
            release();
            for (int j = w.first; j < w.last && ok; ++j) {
                const uint32_t v = next_pair(w, j), k = k_tile(v);
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const bool here = j >= w.lo[t] && j < w.hi[t], more = j + 1 < w.hi[t] && j + 1 >= w.lo[t];
                    if (here && ok) {
                        const bool begin = j == w.lo[t];
                        // the item before has read its O_t out
                        if (begin && !wait_all(o_empty + 8 * t, uses[t] & 1)) break;
                        issue_o(t, v, 0, begin, false);
                        if (ok) issue_o(t, v, 1, false, !more);
                        ++np[t];
                    }
                    if (more && ok) {
                        issue_s(t, k);
                        if (j + 2 == w.hi[t] && elected) umma1_commit(q_empty + 8 * t);       // the last S of this tile: Q is free behind it
                    }
                }
                release();
            }
        }
        if (elected) {
            umma1_commit(drain);
            drain_wait(drain, 0, abort_flag, p.wait_limit);
        }
        __syncwarp();
    } else if (warp >= 4) {
        registers_many();
        // ------------------------------------------------------------------ softmax and output of one query tile
        const int t = (warp - 4) >> 2, q = warp & 3;       // tile, tensor-memory lane quarter
        const uint32_t lane_base = tmem + ((uint32_t)(q * 32) << 16);
        const uint32_t ts = lane_base + t * BK, to = lane_base + 2 * BK + t * 128;
        const f32x2 c2 = f2_pack(p.scale_log2, p.scale_log2);
        // this thread's row of the tile; PACK: head and query in it.  Rows that no copy fills hold anything and stay among themselves.
        const int r = q * 32 + lane, r_head = PACK ? r / p.q_len : 0, r_query = PACK ? r - r_head * p.q_len : r;
        uint32_t n = 0, uses = 0;                          // S tiles and items of this query tile so far
        bool ok = true;
        for (int turn = 0, index; ok && (index = item_at(turn)) < items; ++turn) {
        const Item w = item_of<PARTS, PACK>(p, index, q_tiles);
        const int r0 = PACK ? 0 : w.q0 + t * BQ, r_last = PACK ? p.q_len - 1 : r0 + BQ - 1;
        const int h = PACK ? w.h + t * p.pack + r_head : w.h, row = r0 + r_query;
        const bool exists = PACK ? r_head < p.pack && h < w.h_end : row < p.q_len;
        const int key_lo = p.key_lo(row), key_hi = p.key_hi(row, w.keys);
        const int n0 = t == 0 ? w.lo[0] : w.lo[1], n1 = t == 0 ? w.hi[0] : w.hi[1];
        // key tiles [plain_lo, plain_hi) are seen whole by every row of the tile
        const int plain_lo = p.left >= 0 ? (p.key_lo(r_last) + BK - 1) / BK : 0;
        const int plain_hi = max(p.key_hi(r0, w.keys), 0) / BK;
        float m = -INFINITY;
        f32x2 l2 = 0;
        // raises the running maximum to at least `top`: l and (after the first tile) O are scaled down.  S of the current tile was
        // issued after the previous P V, so O is at rest.
        auto raise = [&](float top, bool first_tile) {
            const float up = fmaxf(m, top);
            const float f = m == up ? 1.0f : ex2(m - up);              // m = -inf: l and O hold zeros
            m = up;
            l2 = f2_mul(l2, f2_pack(f, f));
            if (first_tile) return;
#pragma unroll 1
            for (int c = 0; c < DP; c += 32) {
                uint32_t o[32];
                tmem_ld32(to + c, o);
                tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                tmem_st32(to + c, o);
            }
        };
        auto publish = [&](int half, const uint32_t (&pk)[32]) {       // 64 probabilities per row, over S's first columns
            tmem_st32(ts + half * 32, pk);
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(p_full + 16 * t + 8 * half);
        };
        for (int j = n0; j < n1; ++j, ++n) {
            if (!(ok = warp_wait(s_full + 8 * t, n & 1, abort_flag, p.wait_limit))) break;
            tc_fence_after();
            uint32_t s[128];
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld32(ts + c * 32, s + c * 32);
            tmem_ld_wait();
            const bool masked = j < plain_lo || j >= plain_hi;
            const int from = key_lo - j * BK, to = key_hi - j * BK;    // columns of this tile that the row sees
            if (masked) hide_scores<128>(s, from, to, p.left >= 0);
            uint32_t pk[32];
            float base = m == -INFINITY ? 0.0f : m;
            // The first half's exponentials are taken against the maximum so far, while this tile's is being found: it raises the
            // running maximum (and makes them void) only in the first tiles of a row, as a rule.
            f32x2 sum = 0;
            exp_scores<32>(s, pk, sum, c2, f2_pack(-base, -base));
            float top[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                top[k] = __uint_as_float(s[k]);
#pragma unroll
                for (int c = k + 4; c + 4 < 128; c += 8) top[k] = max3(top[k], __uint_as_float(s[c]), __uint_as_float(s[c + 4]));
                top[k] = fmaxf(top[k], __uint_as_float(s[124 + k]));
            }
            float tile_top = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * p.scale_log2;
            if (PACK && !exists) tile_top = -INFINITY;
            if (__any_sync(0xFFFFFFFFu, tile_top > m + kRaise)) {
                raise(tile_top, j == n0);
                base = m == -INFINITY ? 0.0f : m;
                sum = 0;
                uint32_t again[64];                                    // S still stands in tensor memory
                tmem_ld32(ts, again);
                tmem_ld32(ts + 32, again + 32);
                tmem_ld_wait();
                if (masked) hide_scores<64>(again, from, to, p.left >= 0);
                exp_scores<32>(again, pk, sum, c2, f2_pack(-base, -base));
            }
            publish(0, pk);
            exp_scores<32>(s + 64, pk, sum, c2, f2_pack(-base, -base));
            publish(1, pk);
            l2 = f2_add(l2, sum);
        }
        if (!ok) break;
        float l;
        {
            float a, b2;
            f2_unpack(l2, a, b2);
            l = a + b2;
        }
        const int64_t lse_at = (((int64_t)w.part * p.batch + w.b) * p.heads + h) * p.q_len + row;
        const bool some = l > 0.0f || l != l;              // this query sees a key
        if (exists) (PARTS ? p.part_lse : p.lse)[lse_at] = some ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
        const bool any = n1 > n0;
        if (any) {
            ok = warp_wait(o_full + 8 * t, uses & 1, abort_flag, p.wait_limit);
            ++uses;
            tc_fence_after();
        }
        if (!ok) break;
        const float f = some ? 1.0f / l : 0.0f;
        __nv_bfloat16* dst = out.o + w.b * out.batch_stride + row * out.token_stride + h * out.head_stride;
#pragma unroll 1
        for (int c = 0; c < DP; c += 32) {
            uint32_t o[32];
            if (any) {
                tmem_ld32(to + c, o);
                tmem_ld_wait();
                if (c + 32 >= DP) {
                    // O has been read: the next item's first product may overwrite it
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(o_empty + 8 * t);
                }
            }
            if (!any || !some) {
#pragma unroll
                for (int v = 0; v < 32; ++v) o[v] = 0u;
            }
            if (exists && (!PARTS || any)) {                   // a part without keys: lse says so, o is not read
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    float x[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[k] = __uint_as_float(o[8 * v + k]) * f;
                    if (c + 8 * v < p.dim) {
                        if constexpr (PARTS) {
                            float4* to4 = reinterpret_cast<float4*>(p.part_o + lse_at * p.dim + c + 8 * v);
                            to4[0] = make_float4(x[0], x[1], x[2], x[3]);
                            to4[1] = make_float4(x[4], x[5], x[6], x[7]);
                        } else {
                            *reinterpret_cast<uint4*>(dst + c + 8 * v) =
                                make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
                        }
                    }
                }
            }
            __syncwarp();
        }
        }
        tc_fence_before();
    }
    __syncthreads();
    if (warp == 0) { tc_fence_after(); tmem_dealloc1(tmem, 512); }
}

// Joins the parts of a query:  lse = log sum exp lse_p,  o = sum exp(lse_p - lse) o_p, parts in order.  A warp per query.  A part
// that saw no key (lse = -inf) has written no o: what is loaded there, before lse is known, is not used.
__global__ void __launch_bounds__(256) attention_join_kernel(const AttentionParams p, __nv_bfloat16* o, const int64_t batch_stride,
                                                             const int64_t token_stride, const int64_t head_stride) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int64_t rows = (int64_t)p.batch * p.heads * p.q_len, r = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (r >= rows) return;
    const int lane = threadIdx.x & 31;
    auto lse_of = [&](int k) { return k < p.parts ? p.part_lse[k * rows + r] : -INFINITY; };
    const float mine = lse_of(lane);                       // a lane per part
    float top = mine;
    for (int k = lane + 32; k < p.parts; k += 32) top = fmaxf(top, lse_of(k));
    float4 v[4];
    auto load = [&](int k0) {                              // four at a time; they do not wait for lse
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (k0 + u < p.parts && lane * 4 < p.dim) v[u] = *reinterpret_cast<const float4*>(p.part_o + ((k0 + u) * rows + r) * p.dim + lane * 4);
    };
    load(0);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
    const float base = top == -INFINITY ? 0.0f : top;
    float sum = 0.0f, acc[4] = {0.0f, 0.0f, 0.0f, 0.0f}, weight = 0.0f;
    for (int k0 = 0; k0 < p.parts; k0 += 4) {
        if (k0 > 0) load(k0);
        if ((k0 & 31) == 0) {
            const float lse = k0 == 0 ? mine : lse_of(k0 + lane);
            weight = lse == -INFINITY ? -1.0f : exp2f((lse - base) * 1.4426950408889634f);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const float w = __shfl_sync(0xFFFFFFFFu, weight, (k0 + u) & 31);
            if (w == -1.0f) continue;                      // no keys, or no such part
            sum += w;
            acc[0] = fmaf(w, v[u].x, acc[0]); acc[1] = fmaf(w, v[u].y, acc[1]); acc[2] = fmaf(w, v[u].z, acc[2]); acc[3] = fmaf(w, v[u].w, acc[3]);
        }
    }
    const float f = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
    const int64_t i = r % p.q_len, bh = r / p.q_len, b = bh / p.heads, h = bh - b * p.heads;
    if (lane * 4 < p.dim) {
        uint2 w = make_uint2(0, 0);
        if (f != 0.0f) w = make_uint2(pack_bf16x2(acc[0] * f, acc[1] * f), pack_bf16x2(acc[2] * f, acc[3] * f));
        *reinterpret_cast<uint2*>(o + b * batch_stride + i * token_stride + h * head_stride + lane * 4) = w;
    }
    if (lane == 0) p.lse[r] = sum > 0.0f || sum != sum ? base + logf(sum) : -INFINITY;
}

// Heads of a group whose queries share a tile of 128 rows, evenly over the tiles they need; 0: a head's queries have their own tiles.
// Few queries leave most rows of a tile empty, and every head of a group walks the same keys: together they walk them once.  On their
// own / together, us, 32 heads on 8 key/value heads of 128: one query on 8192 keys 31.1 / 16.8; 16 sequences of that 338 / 89.6
// (6.0 TB/s, 0.91 of the measured copy rate); 4 x 8 on 4096 47.8 / 22.5; 1 on 300 9.3 / 9.0.  A group that needs more than one tile puts two
// of them into a CTA, one behind the other: that pays once the heads alone are more than the 148 SMs take at a time (8 x 100 on
// 2000 53.4 / 36.2, 8 x 100 on 128 12.5 / 9.9) and costs before (4 x 100 on 128 8.0 / 9.4, 61 on 61, 8 heads 5.9 / 7.5).
int packed_heads(const ue5m3_attention_shape& s) {
    const int64_t group = s.heads / s.kv_heads;
    if (group == 1 || s.q_len == 0 || s.q_len > BQ || (s.q_len * group > BQ && s.batch * s.heads <= 148)) return 0;
    const int64_t most = BQ / s.q_len, tiles = (group + most - 1) / most;
    return (int)((group + tiles - 1) / tiles);
}
// Pairs of query tiles.
int64_t query_pairs(const ue5m3_attention_shape& s) {
    const int64_t pack = packed_heads(s), group = s.heads / s.kv_heads;
    return pack ? s.batch * s.kv_heads * ((group + 2 * pack - 1) / (2 * pack)) : (s.q_len + 2 * BQ - 1) / (2 * BQ) * s.batch * s.heads;
}

template <int DP, bool PARTS, bool PACK>
int run(const ue5m3_attention_shape& s, const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const AttentionParams& p,
        const OutputParams& o, int num_sms, cudaStream_t st) {
    using T = Tiles<DP>;
    const int64_t q_tiles = (s.q_len + 2 * BQ - 1) / (2 * BQ), items = query_pairs(s) * p.parts;
    if (items > 0x7FFFFFFF - 2 * num_sms) return UE5M3_ERR_UNSUPPORTED;
    static std::atomic<int> granted[64];
    if (allow_smem(attention_kernel<DP, PARTS, PACK>, T::SMEM, granted) != cudaSuccess) return UE5M3_ERR_CUDA;
    attention_kernel<DP, PARTS, PACK><<<(unsigned)(items < num_sms ? items : num_sms), kThreads, T::SMEM, st>>>(q, k, v, p, o, (int)q_tiles, (int)items);
    return cudaGetLastError() == cudaSuccess ? UE5M3_OK : UE5M3_ERR_CUDA;
}
template <bool PARTS>
int run(const ue5m3_attention_shape& s, const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const AttentionParams& p,
        const OutputParams& o, int num_sms, cudaStream_t st) {
    if (p.pack) return s.head_dim <= 64 ? run<64, PARTS, true>(s, q, k, v, p, o, num_sms, st) : run<128, PARTS, true>(s, q, k, v, p, o, num_sms, st);
    return s.head_dim <= 64 ? run<64, PARTS, false>(s, q, k, v, p, o, num_sms, st) : run<128, PARTS, false>(s, q, k, v, p, o, num_sms, st);
}

}  // namespace

// Parts into which the key tiles are shared out when the query tiles alone leave at least half of the 148 SMs idle: as many as fill
// them, none below two key tiles, and no more than pay (a quarter of the time at least).  In units of a key tile's step (1.5 us) a call takes tiles / n, and sharing
// out costs 2 (the second kernel) and, per part, its binary32 results through memory twice at about 5 TB/s: rows * dim / 0.9e6.  Whole
// against shared out, us: one query on 8192 keys, 32 heads 88.9 / 29.6; 100 on 8192, 16 heads 91.0 / 25.3; 600 on 2000, 8 heads
// 33.4 / 22.4; and where it does not pay: 100 on 512, 32 heads 11.1 / 13.4; 8 x 64 on 1000, 32 / 8 heads 23.0 / 28.8.
int attention_splits(const ue5m3_attention_shape& s) {
    const int64_t ctas = query_pairs(s), tiles = (s.k_len + BK - 1) / BK;
    if (ctas == 0 || ctas > 74 || tiles < 4) return 1;
    const double part = (double)s.batch * s.heads * s.q_len * s.head_dim / 0.9e6;
    const int64_t fill = 148 / ctas, most = tiles / 2, pays = (int64_t)sqrt((double)tiles / part);
    const int64_t n = std::min(std::min(fill, most), pays);
    return n > 1 && (double)tiles / n + 2 + n * part < 0.75 * (double)tiles ? (int)n : 1;
}

int launch_attention(const ue5m3_attention_shape& s, const ue5m3_heads& q, const ue5m3_heads& k, const ue5m3_heads& v,
                     const ue5m3_heads& o, float* lse, float* workspace, int num_sms, cudaStream_t st, const StallTest& stall) {
    if (s.batch == 0 || s.q_len == 0) return UE5M3_OK;
    CUtensorMap mq, mk, mv;
    const int pack = packed_heads(s);
    if (!make_heads_map(&mq, q, s.batch, s.q_len, s.heads, s.head_dim, pack ? (uint32_t)s.q_len : BQ, pack ? pack : 1)) return UE5M3_ERR_CUDA;
    if (s.k_len == 0) mk = mv = mq;                        // no key tile is ever read
    else if (!make_heads_map(&mk, k, s.batch, s.k_len, s.kv_heads, s.head_dim, BK) || !make_heads_map(&mv, v, s.batch, s.k_len, s.kv_heads, s.head_dim, BK))
        return UE5M3_ERR_CUDA;
    AttentionParams p = attention_params(s);
    p.lse = lse;
    p.parts = attention_splits(s);
    p.pack = pack;
    if (stall.wait_limit > 0) { p.wait_limit = stall.wait_limit; p.stall = 1; }
    const OutputParams out{static_cast<__nv_bfloat16*>(o.data), o.batch_stride, o.token_stride, o.head_stride};
    if (p.parts == 1) return run<false>(s, mq, mk, mv, p, out, num_sms, st);
    const int64_t rows = s.batch * s.heads * s.q_len;
    p.part_o = workspace;
    p.part_lse = workspace + p.parts * rows * s.head_dim;
    const int r = run<true>(s, mq, mk, mv, p, out, num_sms, st);
    if (r != UE5M3_OK) return r;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)((rows + 7) / 8));
    cfg.blockDim = dim3(256);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, attention_join_kernel, p, static_cast<__nv_bfloat16*>(o.data), o.batch_stride, o.token_stride, o.head_stride) == cudaSuccess
               ? UE5M3_OK : UE5M3_ERR_CUDA;
}

int read_and_clear_attention_status() {
    if (cudaDeviceSynchronize() != cudaSuccess) return UE5M3_ERR_CUDA;
    int v = 0;
    if (cudaMemcpyFromSymbol(&v, g_attention_status, sizeof(int)) != cudaSuccess) return UE5M3_ERR_CUDA;
    if (v != 0) {
        const int zero = 0;
        if (cudaMemcpyToSymbol(g_attention_status, &zero, sizeof(int)) != cudaSuccess) return UE5M3_ERR_CUDA;
    }
    return v;
}

}  // namespace ue5m3
