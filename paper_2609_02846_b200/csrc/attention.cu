// Attention, forward, for sm_100a:  o_i = sum_j softmax_j(scale q_i . k_j) v_j over the keys query i sees.
//
// One pass over the keys per tile of queries, with a running maximum m and sum l of every row (binary32):
//     p_j = 2^(s_j - m) with s = scale log2(e) q.k;  l = l 2^(m_old - m) + sum p_j;  O = O 2^(m_old - m) + P V;  o = O / l
//
// A CTA owns two tiles of 128 queries of one head and walks the keys 128 at a time.  Both products run on the tensor core with
// accumulators in tensor memory: S = Q K^T from shared memory, O += P V with P (BF16) taken from tensor memory, where it
// overwrites S.  While one tile's softmax warps turn S into P, the tensor core works for the other tile.  Warp roles:
//   warp 0      copies: Q once, then K and V tiles through a ring
//   warp 1      issues the MMAs (the whole warp runs the loop, one elected lane issues)
//   warp 2      tensor-memory allocation
//   warps 4-7 / 8-11   softmax of tile 0 / 1: thread = query row, so maxima and sums need no exchange between threads
// The running maximum that scales O is raised only when a row's maximum grew by more than 2^8 (then O is rescaled in tensor
// memory by its softmax warps): p stays below 2^8, l and O in binary32 lose nothing, and o = O / l does not depend on m.
// Tensor memory: S0, S1 (128 columns each), O0, O1 (head dimension columns each).
#include <cuda.h>
#include <cuda_runtime.h>
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
    static constexpr int STAGES = DP == 128 ? 5 : 8;
    static constexpr int SMEM_BAR = 2 * TILE + STAGES * TILE;
    static constexpr int SMEM = SMEM_BAR + 256 + 1024;    // + alignment slack
};

__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, long long limit) {
    return mbar_wait_status(bar, parity, abort_flag, &g_attention_status, limit);
}

template <int DP>
__global__ void __launch_bounds__(kThreads, 1)
attention_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                 const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_o, const AttentionParams p,
                 const int q_tiles) {
    using T = Tiles<DP>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* smem_gen = smem_raw + (smem - smem_u32(smem_raw));
    const uint32_t ring = smem + 2 * T::TILE;
    const uint32_t bars = smem + T::SMEM_BAR;
    const uint32_t q_full = bars, kv_full = bars + 16, kv_empty = kv_full + 8 * T::STAGES;
    const uint32_t s_full = bars + 144, p_full = bars + 160, o_full = bars + 176, drain = bars + 192;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem_gen + T::SMEM_BAR + 200);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem_gen + T::SMEM_BAR + 204);

    // work of this CTA: heads fastest (heads that share keys run side by side), long query tiles first
    const int bh_count = p.batch * p.heads;
    const int bh = blockIdx.x % bh_count, qt = q_tiles - 1 - blockIdx.x / bh_count;
    const int b = bh / p.heads, h = bh - b * p.heads, kvh = h / p.group;
    const int q0 = qt * 2 * BQ;
    const int keys = p.keys_of(b);
    int lo[2], hi[2];                                     // key tiles of the two query tiles
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int r0 = q0 + t * BQ, r1 = min(r0 + BQ, p.q_len) - 1;
        const int a = p.key_lo(r0), z = r0 < p.q_len ? p.key_hi(r1, keys) : 0;
        lo[t] = a / BK;
        hi[t] = z > a ? (z + BK - 1) / BK : lo[t];
    }
    const bool on0 = hi[0] > lo[0], on1 = hi[1] > lo[1];
    const int first = on0 ? (on1 ? min(lo[0], lo[1]) : lo[0]) : lo[1];
    const int last = on0 ? (on1 ? max(hi[0], hi[1]) : hi[0]) : (on1 ? hi[1] : first);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        *abort_flag = 0;
        for (int t = 0; t < 2; ++t) {
            mbar_init(q_full + 8 * t, 1);
            mbar_init(s_full + 8 * t, 1);
            mbar_init(p_full + 8 * t, 4);
            mbar_init(o_full + 8 * t, 1);
        }
        for (int s = 0; s < T::STAGES; ++s) {
            mbar_init(kv_full + 8 * s, 1);
            mbar_init(kv_empty + 8 * s, 1);
        }
        mbar_init(drain, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        prefetch_tmap(&map_q); prefetch_tmap(&map_k); prefetch_tmap(&map_v); prefetch_tmap(&map_o);
    }
    if (warp == 2) tmem_alloc1(smem_u32(tmem_slot), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;

    if (warp == 0) {
        // ------------------------------------------------------------------ copies
        if (lane == 0) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
                if (hi[t] > lo[t]) {
                    mbar_expect_tx(q_full + 8 * t, T::TILE);
#pragma unroll
                    for (int c = 0; c < T::PANELS; ++c)
                        tma_load_4d(smem + t * T::TILE + c * T::PANEL, &map_q, q_full + 8 * t, c * 64, q0 + t * BQ, h, b);
                }
            uint32_t it = 0;                              // tile 2i = K, 2i + 1 = V of key tile first + i
            for (; it < 2u * (uint32_t)(last - first); ++it) {
                const uint32_t s = it % T::STAGES, ph = (it / T::STAGES) & 1;
                if (!wait(kv_empty + 8 * s, ph ^ 1, abort_flag, p.wait_limit)) break;
                mbar_expect_tx(kv_full + 8 * s, T::TILE);
                const CUtensorMap* m = (it & 1) ? &map_v : &map_k;
#pragma unroll
                for (int c = 0; c < T::PANELS; ++c)
                    tma_load_4d(ring + s * T::TILE + c * T::PANEL, m, kv_full + 8 * s, c * 64, (first + (int)(it >> 1)) * BK, kvh, b);
            }
            // copies in flight land before the shared memory goes away, whatever the other roles did
#pragma unroll
            for (int t = 0; t < 2; ++t)
                if (hi[t] > lo[t]) mbar_wait_drain(q_full + 8 * t, 0, &g_attention_status, p.wait_limit);
            for (uint32_t back = 0; back < T::STAGES && back < it; ++back) {
                const uint32_t j = it - 1 - back;
                mbar_wait_drain(kv_full + 8 * (j % T::STAGES), (j / T::STAGES) & 1, &g_attention_status, p.wait_limit);
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer
        const bool elected = elect_one();
        const uint32_t tm = __shfl_sync(0xFFFFFFFFu, tmem, 0);
        constexpr uint32_t id_s = umma_idesc(BK, false), id_o = umma_idesc(DP, true);
        bool ok = true;
        auto wait_all = [&](uint32_t bar, uint32_t parity) {
            ok = ok && __all_sync(0xFFFFFFFFu, wait(bar, parity, abort_flag, p.wait_limit));
            tc_fence_after();
            return ok;
        };
        auto stage_of = [&](int n) { return ring + (uint32_t)(n % T::STAGES) * T::TILE; };
        auto full = [&](int n) { return wait_all(kv_full + 8 * (n % T::STAGES), (n / T::STAGES) & 1); };
        auto issue_s = [&](int t, int n) {                 // S_t = Q_t K^T, K in ring tile n
            const uint64_t qd = umma_smem_desc(smem + t * T::TILE), kd = umma_smem_desc(stage_of(n));
            if (elected) {
#pragma unroll
                for (int k = 0; k < DP / 16; ++k) {
                    const uint32_t off = (k / 4) * (T::PANEL >> 4) + (k % 4) * 2;
                    umma1_ss(tm + t * BK, qd + off, kd + off, id_s, k != 0);
                }
                umma1_commit(s_full + 8 * t);
            }
            __syncwarp();
        };
        uint32_t np[2] = {0, 0};                           // probability tiles consumed per query tile
        if (on0) wait_all(q_full, 0);
        if (on1) wait_all(q_full + 8, 0);
        if (last > first && full(0)) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
                if (hi[t] > lo[t] && lo[t] == first) issue_s(t, 0);
            if (elected) umma1_commit(kv_empty);
            __syncwarp();
        }
        for (int j = first; j < last && ok; ++j) {
            const int nv = 2 * (j - first) + 1, nk = nv + 1;
            if (!full(nv)) break;
            const int valid = keys - j * BK;               // rows of this V tile that exist
            if (p.k_lens && valid < BK) {
                // values behind the sequence's end may hold anything (0 * NaN is NaN): they become zeros
                for (int i = valid * (DP / 8) + lane; i < BK * (DP / 8); i += 32) {
                    const int r = i / (DP / 8), c = i % (DP / 8);
                    *reinterpret_cast<uint4*>(smem_gen + (stage_of(nv) - smem) + (c / 8) * T::PANEL + r * 128 + (c % 8) * 16) = make_uint4(0, 0, 0, 0);
                }
                fence_proxy_async();
                __syncwarp();
            }
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const bool here = j >= lo[t] && j < hi[t], more = j + 1 < hi[t] && j + 1 >= lo[t];
                if (here) {
                    if (!wait_all(p_full + 8 * t, np[t] & 1)) break;
                    const uint64_t vd = umma_mn_desc(stage_of(nv), T::PANEL);
                    if (elected) {
#pragma unroll
                        for (int k = 0; k < BK / 16; ++k)
                            umma1_ts(tm + 2 * BK + t * 128, tm + t * BK + k * 8, vd + k * (2048 >> 4), id_o, (np[t] | k) != 0);
                        if (!more) umma1_commit(o_full + 8 * t);
                    }
                    __syncwarp();
                    ++np[t];
                }
                if (more) {
                    if (!full(nk)) break;
                    issue_s(t, nk);
                }
            }
            if (!ok) break;
            if (elected) {
                umma1_commit(kv_empty + 8 * (nv % T::STAGES));
                if (j + 1 < last) umma1_commit(kv_empty + 8 * (nk % T::STAGES));
            }
            __syncwarp();
        }
        if (elected) {
            umma1_commit(drain);
            mbar_wait_drain(drain, 0, &g_attention_status, p.wait_limit);
        }
        __syncwarp();
    } else if (warp >= 4) {
        // ------------------------------------------------------------------ softmax and output of one query tile
        const int t = (warp - 4) >> 2, q = warp & 3;       // tile, tensor-memory lane quarter
        const int r0 = q0 + t * BQ, row = r0 + q * 32 + lane;
        const uint32_t lane_base = tmem + ((uint32_t)(q * 32) << 16);
        const uint32_t ts = lane_base + t * BK, to = lane_base + 2 * BK + t * 128;
        const int key_lo = p.key_lo(row), key_hi = p.key_hi(row, keys);
        const int n0 = t == 0 ? lo[0] : lo[1], n1 = t == 0 ? hi[0] : hi[1];
        // key tiles [plain_lo, plain_hi) are seen whole by every row of the tile
        const int plain_lo = p.left >= 0 ? (p.key_lo(r0 + BQ - 1) + BK - 1) / BK : 0;
        const int plain_hi = max(p.key_hi(r0, keys), 0) / BK;
        float m = -INFINITY, l = 0.0f;
        bool ok = true;
        uint32_t n = 0;
        for (int j = n0; j < n1; ++j, ++n) {
            if (!(ok = wait(s_full + 8 * t, n & 1, abort_flag, p.wait_limit))) break;
            tc_fence_after();
            uint32_t s[128];
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld32(ts + c * 32, s + c * 32);
            tmem_ld_wait();
            if (j < plain_lo || j >= plain_hi) {
                const int base = j * BK - key_lo, width = key_hi - key_lo;
#pragma unroll
                for (int c = 0; c < 128; ++c)
                    if (!(base + c >= 0 && base + c < width)) s[c] = 0xFF800000u;
            }
            float top0 = __uint_as_float(s[0]), top1 = __uint_as_float(s[1]), top2 = __uint_as_float(s[2]), top3 = __uint_as_float(s[3]);
#pragma unroll
            for (int c = 4; c < 128; c += 4) {
                top0 = fmaxf(top0, __uint_as_float(s[c]));
                top1 = fmaxf(top1, __uint_as_float(s[c + 1]));
                top2 = fmaxf(top2, __uint_as_float(s[c + 2]));
                top3 = fmaxf(top3, __uint_as_float(s[c + 3]));
            }
            const float top = fmaxf(fmaxf(top0, top1), fmaxf(top2, top3)) * p.scale_log2;
            if (n == 0) m = top;
            else if (__any_sync(0xFFFFFFFFu, top > m + kRaise)) {
                // S of this tile was issued after the previous P V, so O is at rest
                const float up = fmaxf(m, top);
                const float f = m == up ? 1.0f : ex2(m - up);          // m = -inf: O holds zeros
                m = up;
                l *= f;
#pragma unroll 1
                for (int c = 0; c < DP; c += 32) {
                    uint32_t o[32];
                    tmem_ld32(to + c, o);
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                    tmem_st32(to + c, o);
                }
            }
            const float base = m == -INFINITY ? 0.0f : m;
            float sum0 = 0.0f, sum1 = 0.0f;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                uint32_t pk[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    const float e0 = ex2(fmaf(__uint_as_float(s[c * 64 + 2 * i]), p.scale_log2, -base));
                    const float e1 = ex2(fmaf(__uint_as_float(s[c * 64 + 2 * i + 1]), p.scale_log2, -base));
                    sum0 += e0;
                    sum1 += e1;
                    pk[i] = pack_bf16x2(e0, e1);
                }
                tmem_st32(ts + c * 32, pk);
            }
            l += sum0 + sum1;
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(p_full + 8 * t);
        }
        if (row < p.q_len) {
            const float v = l > 0.0f || l != l ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
            p.lse[((int64_t)b * p.heads + h) * p.q_len + row] = v;
        }
        const int box0 = r0 + q * 32;                      // this warp's 32 rows
        bool any = n1 > n0;
        if (any && ok) {
            ok = wait(o_full + 8 * t, 0, abort_flag, p.wait_limit);
            tc_fence_after();
        }
        if (ok && box0 < p.q_len) {
            // staged over this tile's Q (no MMA reads it any more, or it was never loaded)
            const float f = l > 0.0f || l != l ? 1.0f / l : 0.0f;
            const uint32_t stage = t * T::TILE + q * 4096;
#pragma unroll 1
            for (int c = 0; c < T::PANELS; ++c) {
                uint8_t* mine = smem_gen + stage + c * T::PANEL + lane * 128;
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    uint32_t o[32];
                    if (any) {
                        tmem_ld32(to + c * 64 + half * 32, o);
                        tmem_ld_wait();
                    }
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        uint4 w = make_uint4(0, 0, 0, 0);
                        if (any && f != 0.0f) {
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
                if (lane == 0) tma_store_4d(&map_o, smem + stage + c * T::PANEL, c * 64, box0, h, b);
            }
            if (lane == 0) tma_store_wait_all();
        }
        tc_fence_before();
    }
    __syncthreads();
    if (warp == 2) { tc_fence_after(); tmem_dealloc1(tmem, 512); }
}

template <int DP>
int run(const ue5m3_attention_shape& s, const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const CUtensorMap& o,
        const AttentionParams& p, cudaStream_t st) {
    using T = Tiles<DP>;
    const int64_t q_tiles = (s.q_len + 2 * BQ - 1) / (2 * BQ), ctas = q_tiles * s.batch * s.heads;
    if (ctas > 0x7FFFFFFF) return UE5M3_ERR_UNSUPPORTED;
    static std::atomic<int> granted[64];
    if (allow_smem(attention_kernel<DP>, T::SMEM, granted) != cudaSuccess) return UE5M3_ERR_CUDA;
    attention_kernel<DP><<<(unsigned)ctas, kThreads, T::SMEM, st>>>(q, k, v, o, p, (int)q_tiles);
    return cudaGetLastError() == cudaSuccess ? UE5M3_OK : UE5M3_ERR_CUDA;
}

}  // namespace

int launch_attention(const ue5m3_attention_shape& s, const ue5m3_heads& q, const ue5m3_heads& k, const ue5m3_heads& v,
                     const ue5m3_heads& o, float* lse, int num_sms, cudaStream_t st) {
    (void)num_sms;
    if (s.batch == 0 || s.q_len == 0) return UE5M3_OK;
    CUtensorMap mq, mk, mv, mo;
    if (!make_heads_map(&mq, q, s.batch, s.q_len, s.heads, s.head_dim, BQ) || !make_heads_map(&mo, o, s.batch, s.q_len, s.heads, s.head_dim, 32))
        return UE5M3_ERR_CUDA;
    if (s.k_len == 0) mk = mv = mq;                        // no key tile is ever read
    else if (!make_heads_map(&mk, k, s.batch, s.k_len, s.kv_heads, s.head_dim, BK) || !make_heads_map(&mv, v, s.batch, s.k_len, s.kv_heads, s.head_dim, BK))
        return UE5M3_ERR_CUDA;
    AttentionParams p = attention_params(s);
    p.lse = lse;
    return s.head_dim <= 64 ? run<64>(s, mq, mk, mv, mo, p, st) : run<128>(s, mq, mk, mv, mo, p, st);
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
