// What the attention kernels share: one-CTA tcgen05 wrappers, matrix descriptors, the mask and the tensor maps (sm_100a only).
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <algorithm>
#include <cstdint>
#include "../../include/ue5m3.h"
#include "block_ops.h"
#include "common.cuh"
#include "tcgen05.cuh"

namespace ue5m3 {

// ----------------------------------------------------------------------------- PTX wrappers (cta_group::1)
__device__ __forceinline__ void tmem_alloc1(uint32_t dst_smem, uint32_t ncols) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst_smem), "r"(ncols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_dealloc1(uint32_t taddr, uint32_t ncols) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols) : "memory");
}
__device__ __forceinline__ void umma1_ss(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void umma1_ts(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(tmem_d), "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
// Arrives on the barrier once every MMA issued so far by this thread has completed.
__device__ __forceinline__ void umma1_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2, int c3) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3) : "memory");
}
__device__ __forceinline__ void tma_store_4d(const CUtensorMap* map, uint32_t src, int c0, int c1, int c2, int c3) {
    asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.bulk_group [%0, {%2, %3, %4, %5}], [%1];"
                 ::"l"(map), "r"(src), "r"(c0), "r"(c1), "r"(c2), "r"(c3) : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
// 16 consecutive 32-bit columns of this thread's tensor-memory lane.
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t r[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
                   "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// Load at device scope: from where every SM sees the same value, not from this SM's first-level cache or the read-only path.
__device__ __forceinline__ float load_device(const float* p) {
    float r;
    asm volatile("ld.relaxed.gpu.global.f32 %0, [%1];" : "=f"(r) : "l"(p) : "memory");
    return r;
}

// Acquire at CTA scope: these kernels have no clusters, and the cluster-scope wait costs over a hundred cycles even when the phase
// is complete (the issuing warp passes six of them per pair of tiles).
__device__ __forceinline__ bool try_wait_cta(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "mbarrier.try_wait.parity.acquire.cta.shared::cta.b64 p, [%1], %2;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// Bounded waits as in tcgen05.cuh, but without calls: a kernel that moves registers between its warps (setmaxnreg) may make none.
// `drain`: for something this thread issued itself, whatever the other roles did (the abort flag is not looked at).
__device__ __forceinline__ bool wait_inline(uint32_t bar, uint32_t parity, volatile int* abort_flag, int* status_word, long long limit, bool drain = false) {
    if (try_wait_cta(bar, parity)) return true;
    const long long t0 = clock64();
#pragma unroll 1
    for (;;) {
#pragma unroll 1
        for (int i = 0; i < 64; ++i)
            if (try_wait_cta(bar, parity)) return true;
        if (!drain && *abort_flag) return false;
        if (clock64() - t0 > limit) {
            if (!drain) *abort_flag = 1;
            atomicExch(status_word, (int)UE5M3_ERR_TIMEOUT);
            return false;
        }
    }
}
// The same for a whole warp: complete for every lane, or given up by every lane.  A lane that gave up alone (the clock and the abort
// flag are read lane by lane) would leave the others in front of tensor-memory instructions and votes that want the whole warp.
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, volatile int* abort_flag, int* status_word, long long limit) {
    return __all_sync(0xFFFFFFFFu, wait_inline(bar, parity, abort_flag, status_word, limit));
}
// 384 threads are launched with 168 registers each (64,512 in all): the four warps that copy and issue give theirs up, the eight
// that do the arithmetic take them (128 x 88 + 256 x 208 = 64,512).
__device__ __forceinline__ void registers_few() { asm volatile("setmaxnreg.dec.sync.aligned.u32 88;"); }
__device__ __forceinline__ void registers_many() { asm volatile("setmaxnreg.inc.sync.aligned.u32 208;"); }

__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// Scores of pairs that do not exist become -inf: only columns from <= column < to stay (`from` is looked at where it can be above 0).
template <int N>
__device__ __forceinline__ void hide_scores(uint32_t* s, int from, int to, bool window) {
    if (window) {
#pragma unroll
        for (int c = 0; c < N; ++c) s[c] = c >= from && c < to ? s[c] : 0xFF800000u;
    } else {
#pragma unroll
        for (int c = 0; c < N; ++c) s[c] = c < to ? s[c] : 0xFF800000u;
    }
}
// The same by the bounds that cut some row's columns in this tile.  (With sinks 187 -> 183 us at 2 x 4096 tokens with a window of 1023; where there is no window
// in most calls the third branch costs more than it saves: 275 -> 292 without one.)
template <int N>
__device__ __forceinline__ void hide_scores_by(uint32_t* s, int from, int to, bool lower, bool upper) {
    if (lower && upper) {
#pragma unroll
        for (int c = 0; c < N; ++c) s[c] = c >= from && c < to ? s[c] : 0xFF800000u;
    } else if (upper) {
#pragma unroll
        for (int c = 0; c < N; ++c) s[c] = c < to ? s[c] : 0xFF800000u;
    } else if (lower) {
#pragma unroll
        for (int c = 0; c < N; ++c) s[c] = c >= from ? s[c] : 0xFF800000u;
    }
}
__device__ __forceinline__ f32x2 ex2_pair(f32x2 x) {
    float a, b;
    f2_unpack(x, a, b);
    return f2_pack(ex2(a), ex2(b));
}
__device__ __forceinline__ uint32_t pack_pair(f32x2 x) {
    float a, b;
    f2_unpack(x, a, b);
    return pack_bf16x2(a, b);
}
__device__ __forceinline__ f32x2 pair_of(const uint32_t* s) { return f2_pack(__uint_as_float(s[0]), __uint_as_float(s[1])); }

// 2^(s c - base) of 2 N scores: packed products, one exponential each.  Adds them to `sum` and packs them as BF16.
template <int N>
__device__ __forceinline__ void exp_scores(const uint32_t* s, uint32_t* packed, f32x2& sum, f32x2 c, f32x2 minus_base) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const f32x2 x = ex2_pair(f2_fma(pair_of(s + 2 * i), c, minus_base));
        sum = f2_add(sum, x);
        packed[i] = pack_pair(x);
    }
}
// Probabilities of pairs that do not exist become zero: only columns from <= column < to stay.  `lower`, `upper`: which of the two
// bounds the mask has at all.
template <int N>
__device__ __forceinline__ void hide_pairs(f32x2* p, int from, int to, bool lower, bool upper) {
    if (lower && upper) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float a, b;
            f2_unpack(p[i], a, b);
            p[i] = f2_pack(2 * i >= from && 2 * i < to ? a : 0.0f, 2 * i + 1 >= from && 2 * i + 1 < to ? b : 0.0f);
        }
    } else if (upper) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float a, b;
            f2_unpack(p[i], a, b);
            p[i] = f2_pack(2 * i < to ? a : 0.0f, 2 * i + 1 < to ? b : 0.0f);
        }
    } else if (lower) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float a, b;
            f2_unpack(p[i], a, b);
            p[i] = f2_pack(2 * i >= from ? a : 0.0f, 2 * i + 1 >= from ? b : 0.0f);
        }
    }
}
// x where p is not zero (0 * NaN would be NaN where a pair does not exist)
__device__ __forceinline__ f32x2 where_p(f32x2 p, f32x2 x) {
    float a, b, u, v;
    f2_unpack(p, a, b);
    f2_unpack(x, u, v);
    return f2_pack(a != 0.0f ? u : 0.0f, b != 0.0f ? v : 0.0f);
}

// ----------------------------------------------------------------------------- tiles in shared memory
// A tile is ROWS x (64 * panels) BF16 values in panels of 64 columns: a panel is ROWS rows of 128 bytes, 128-byte swizzle, as a
// tensor-map box of 64 x ROWS delivers it.  Read along the columns (contraction over the head dimension) it is a K-major
// operand; read along the rows (contraction over queries or keys) an MN-major one.
//
// K-major: umma_smem_desc (8-row groups 1024 bytes apart); 16 columns further = 32 bytes, next panel = ROWS * 128 bytes.
// MN-major: 64 consecutive columns per swizzle row; the next 64 (leading byte offset) are a panel further, the next 8 rows
// of the contraction (stride byte offset) 1024 bytes further; 16 rows further = 2048 bytes.
__device__ __forceinline__ uint64_t umma_mn_desc(uint32_t saddr, uint32_t panel_bytes) {
    uint64_t d = 0;
    d |= (uint64_t)((saddr & 0x3FFFFu) >> 4);
    d |= (uint64_t)(panel_bytes >> 4) << 16;
    d |= (uint64_t)(1024 >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}
// kind::f16 instruction descriptor: D = F32, A = B = BF16, M = 128, N given; b_mn: B is MN-major.
__host__ __device__ constexpr uint32_t umma_idesc(uint32_t n, bool b_mn) {
    return (1u << 4) | (1u << 7) | (1u << 10) | ((b_mn ? 1u : 0u) << 16) | ((n >> 3) << 17) | ((128u >> 4) << 24);
}

// Issue of a whole product by an elected lane of the converged issuing warp.  Addresses and descriptors must be warp-uniform to the
// compiler's eye, and so must the loops around: an operand that is not already in a uniform register is moved there before
// every MMA, which takes longer than the MMA (75 cycles against 64).  So kernels take their loop bounds through uniform().
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(0xFFFFFFFFu, x, 0); }
__device__ __forceinline__ uint64_t desc64(uint32_t high, uint32_t low) { return ((uint64_t)high << 32) | low; }
constexpr uint32_t kDescHighK = (1024u >> 4) | (1u << 14) | (2u << 29);            // upper words: stride 1024, version, 128-byte swizzle
__device__ __forceinline__ uint32_t desc_low_k(uint32_t saddr) { return ((saddr & 0x3FFFFu) >> 4) | (1u << 16); }
__device__ __forceinline__ uint32_t desc_low_mn(uint32_t saddr, uint32_t panel_bytes) { return ((saddr & 0x3FFFFu) >> 4) | ((panel_bytes >> 4) << 16); }
// D [128 x 128] = A B^T, both K-major tiles of 128 rows and DP columns.
template <int DP>
__device__ __forceinline__ void issue_square(bool elected, uint32_t d, uint32_t a_low, uint32_t b_low, uint32_t bar) {
    if (elected) {
#pragma unroll
        for (int k = 0; k < DP / 16; ++k) {
            const uint32_t off = (k / 4) * (128 * 128 >> 4) + (k % 4) * 2;
            umma1_ss(d, desc64(kDescHighK, a_low + off), desc64(kDescHighK, b_low + off), umma_idesc(128, false), k != 0);
        }
        umma1_commit(bar);
    }
    __syncwarp();
}
// The same with A in tensor memory (BF16 pairs, DP / 2 columns).
template <int DP>
__device__ __forceinline__ void issue_square_ts(bool elected, uint32_t d, uint32_t a, uint32_t b_low, uint32_t bar) {
    if (elected) {
#pragma unroll
        for (int k = 0; k < DP / 16; ++k)
            umma1_ts(d, a + k * 8, desc64(kDescHighK, b_low + (k / 4) * (128 * 128 >> 4) + (k % 4) * 2), umma_idesc(128, false), k != 0);
        umma1_commit(bar);
    }
    __syncwarp();
}
// D [128 x DP] += A B over 128 of the contraction: A (BF16) in tensor memory, 64 values each from columns a and a + 64, B an
// MN-major tile.  HALF 0 or 1: only the first or last 32 of each 64.
template <int DP, int HALF = -1>
__device__ __forceinline__ void issue_accumulate(bool elected, uint32_t d, uint32_t a, uint32_t b_low, uint32_t add) {
    if (elected) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (HALF < 0 || ((k >> 1) & 1) == HALF)
                umma1_ts(d, a + k * 8 + (k / 4) * 32, desc64(kDescHighK, b_low + k * (2048 >> 4)), umma_idesc(DP, true), k == 0 ? add : 1u);
    }
    __syncwarp();
}
__device__ __forceinline__ void issue_commit(bool elected, uint32_t bar) {
    if (elected) umma1_commit(bar);
    __syncwarp();
}

// Zeroes the rows of a tile (128 rows, DP columns, as the copies laid it out) that are not from <= row < to, by a whole warp, ahead of the
// products that read it: rows that take no part may hold anything, and a product with a zero on the other side would keep their NaN.
// One loop for both ends: with two the compiler gives up the issuing warp's uniform registers (forward 2 x 4096: 250 us against 230).
template <int DP>
__device__ __forceinline__ void keep_rows(uint8_t* tile, int from, int to, int lane) {
    for (int i = (from > 0 ? 0 : max(to, 0) * (DP / 8)) + lane; i < 128 * (DP / 8); i += 32) {
        const int r = i / (DP / 8), c = i % (DP / 8);
        if (r < from || r >= to) *reinterpret_cast<uint4*>(tile + (c / 8) * (128 * 128) + r * 128 + (c % 8) * 16) = make_uint4(0, 0, 0, 0);
    }
    fence_proxy_async();
    __syncwarp();
}

// ----------------------------------------------------------------------------- which pairs exist
struct AttentionParams {
    int q_len, k_len, heads, group;      // group = heads per key/value head
    int causal, left;                    // left < 0: all
    int batch;
    const int* k_lens;
    float scale, scale_log2;             // scale * log2(e)
    float* lse;                          // forward: [batch, heads, q_len]
    const float* lse2;                   // backward: -lse * log2(e) per query, padded to whole tiles (-inf: contributes nothing)
    const float* delta;                  // backward: -(dout . o) per query, padded
    int q_pad;
    int first_key;                       // keys in front of this one lie before every query's window
    int first_query;                     // queries in front of this one stand before every key (causal)
    int kv_heads, pack;                         // forward: heads that share a query tile (0: none do)
    int dim, parts;                      // head dimension; parts into which the key tiles of a query are shared out
    float* part_o; float* part_lse;      // parts > 1: o (backward: dq) [parts][batch][heads][q_len][dim]; forward: lse [..][q_len]
    long long wait_limit;
    int stall;                           // self-test: no copy is issued, so every wait for one runs out
    int sinks;                           // first keys that a window does not hide (0 without a window), at most one key tile
    int sink_parts;                      // backward: CTAs that share the queries of key tile 0 ...
    float* part_kv;                      // ... and then leave binary32 sums here: [sink_parts][batch][kv_heads][dv, dk][128][dim]

    __device__ __forceinline__ int keys_of(int b) const {
        if (!k_lens) return k_len;
        const int n = __ldg(k_lens + b);
        return n < 0 ? 0 : (n > k_len ? k_len : n);
    }
    // keys [lo, hi) that query i sees (empty when hi <= lo)
    __host__ __device__ __forceinline__ int key_lo(int i) const { return left >= 0 ? max(0, i + (k_len - q_len) - left) : 0; }
    __host__ __device__ __forceinline__ int key_hi(int i, int keys) const { return causal ? min(keys, i + (k_len - q_len) + 1) : keys; }
    // queries from this one on see no key: their windows begin behind the sequence's end
    __host__ __device__ __forceinline__ int queries_end(int keys) const { return left >= 0 ? min(q_len, keys - k_len + q_len + left) : q_len; }
    // queries [lo, hi) that see key j, given that j < keys
    __host__ __device__ __forceinline__ int query_lo(int j) const { return causal ? max(0, j - (k_len - q_len)) : 0; }
    __host__ __device__ __forceinline__ int query_hi(int j) const { return left >= 0 ? min(q_len, j - (k_len - q_len) + left + 1) : q_len; }
    // With sinks (SINKS): every query from query_lo on sees the first keys, and with them every query sees some key if there are any.
    template <bool SINKS> __host__ __device__ __forceinline__ int queries_end_of(int keys) const { return SINKS ? q_len : queries_end(keys); }
    template <bool SINKS> __host__ __device__ __forceinline__ int query_hi_of(int j) const { return SINKS && j < sinks ? q_len : query_hi(j); }
    // Where keys are walked, a query sees its window, and apart from that the keys from 0 up to here: sinks in front of the window.
    __host__ __device__ __forceinline__ int sinks_hi(int i, int keys) const { return min(min(sinks, key_lo(i)), key_hi(i, keys)); }
};

// ----------------------------------------------------------------------------- host side
// [batch, tokens, heads, dim] with element strides -> map (dim, tokens, heads, batch); box 64 x rows (x box_heads).  Dimensions of size 1 get
// a stride that is always valid.
inline bool make_heads_map(CUtensorMap* m, const ue5m3_heads& t, int64_t batch, int64_t tokens, int64_t heads, int64_t dim, uint32_t rows, uint32_t box_heads = 1) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[4] = {(cuuint64_t)dim, (cuuint64_t)tokens, (cuuint64_t)heads, (cuuint64_t)batch};
    const cuuint64_t any = (cuuint64_t)((dim + 7) / 8 * 8) * 2;
    cuuint64_t strides[3] = {tokens > 1 ? (cuuint64_t)t.token_stride * 2 : any, heads > 1 ? (cuuint64_t)t.head_stride * 2 : any,
                             batch > 1 ? (cuuint64_t)t.batch_stride * 2 : any};
    cuuint32_t box[4] = {64, rows, box_heads, 1};
    cuuint32_t estr[4] = {1, 1, 1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, t.data, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

inline AttentionParams attention_params(const ue5m3_attention_shape& s, int64_t sinks = 0) {
    AttentionParams p{};
    p.q_len = (int)s.q_len; p.k_len = (int)s.k_len; p.heads = (int)s.heads; p.group = (int)(s.heads / s.kv_heads);
    p.kv_heads = (int)s.kv_heads; p.causal = s.causal; p.batch = (int)s.batch; p.k_lens = s.k_lens;
    // no query stands behind the last key, so a window that reaches from there to the first one hides nothing; a shorter one keeps
    // every sum of positions below within 32 bits (lengths end at 2^30)
    p.left = s.window_left < s.k_len - 1 ? (int)s.window_left : -1;
    p.scale = s.scale;
    p.scale_log2 = s.scale * 1.4426950408889634f;
    p.q_pad = (int)attention_padded_q(s.q_len);
    p.wait_limit = WAIT_LIMIT_CYCLES;
    p.first_query = p.causal ? (int)std::max<int64_t>(0, s.q_len - s.k_len) : 0;
    p.first_key = p.left >= 0 ? (int)std::max<int64_t>(0, s.k_len - s.q_len - p.left) : 0;
    p.dim = (int)s.head_dim;
    p.parts = 1;
    p.sinks = p.left >= 0 ? (int)sinks : 0;
    p.sink_parts = 1;
    return p;
}

}  // namespace ue5m3
