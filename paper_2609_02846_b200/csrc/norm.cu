// Layer norm of the rows of a matrix, forward and backward, for sm_100a.
//
//   forward   mean = sum x / n, rstd = rsqrt(sum (x - mean)^2 / n + eps), y = (x - mean) rstd w + b
//   backward  xh = (x - mean) rstd, g = dy w:  dx = rstd (g - sum g / n - xh sum(g xh) / n),  dw = sum_r dy xh, db = sum_r dy
//
// Both are bound by memory (2 and 3 elements moved per element, 8 and 14 operations).  The kernels are persistent: a group of
// T threads owns a row at a time, every thread the same columns of each of its rows (aligned rows: 32 forward from 2048 columns on, else
// 16; others: 16, or 4 and 6 where that was faster, see there), so the weights are read once per CTA into registers, the column sums of dw and db stay in registers until the CTA ends, and the row itself stays in registers
// between the reductions (the variance is that of the centred values: no cancellation for a large mean).
// Rows that are 16-byte aligned come through a ring in shared memory, filled by bulk copies several rows ahead: about 100 KB are
// in flight per SM, which a prefetch in registers cannot hold.  Other rows are prefetched element by element, one row ahead.
// Column sums leave as one binary32 row per CTA and are added by a second small kernel in a fixed order: no atomics.
// Rows of more than 16384 columns (backward: 8192) take kernels that re-read the row instead.
// Times below are GPU time, calls back to back in a graph; calls from Python in a row take up to 8 % longer where the GPU is what
// takes the time (forward 8192 x 4096 26.6 us, backward 16384 x 4096 77.4) and the host's 14 to 21 us where it is not.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cstdint>
#include "../../include/ue5m3.h"
#include "block_ops.h"
#include "common.cuh"
#include "tcgen05.cuh"

namespace ue5m3 {

__device__ int g_norm_status = 0;

namespace {

constexpr int kPerThread = 16;                       // columns a thread holds at most
constexpr int kMaxRowThreads = 1024;
constexpr int64_t kRegisterCols = 16384;             // longest row the forward kernels hold in registers (backward: 8192)
constexpr int kBwdGroups = 148;                      // CTAs of the backward kernel: one per SM of a B200

// One element of a row as it lies in memory.
template <typename T> struct Raw;
template <> struct Raw<__nv_bfloat16> { unsigned short v; };
template <> struct Raw<float> { float v; };

// (plain loads: y may be x, and a load through the read-only path promises that the kernel writes nothing there)
__device__ __forceinline__ void load_raw(Raw<__nv_bfloat16>& r, const __nv_bfloat16* p) { r.v = *reinterpret_cast<const unsigned short*>(p); }
__device__ __forceinline__ void load_raw(Raw<float>& r, const float* p) { r.v = *p; }
__device__ __forceinline__ float unpack(const Raw<__nv_bfloat16>& r) { return __uint_as_float((uint32_t)r.v << 16); }
__device__ __forceinline__ float unpack(const Raw<float>& r) { return r.v; }

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ void store_one(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void store_one(float* p, float v) { *p = v; }
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
// VEC consecutive columns: one element, or 16 bytes
template <int VEC> __device__ __forceinline__ void load_vec(float* f, const __nv_bfloat16* p) {
    if constexpr (VEC == 8) unpack_bf16x8(*reinterpret_cast<const uint4*>(p), f);
    else f[0] = __bfloat162float(*p);
}
template <int VEC> __device__ __forceinline__ void load_vec(float* f, const float* p) {
    if constexpr (VEC == 4) {
        const float4 v = *reinterpret_cast<const float4*>(p);
        f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
    } else {
        f[0] = *p;
    }
}
template <int VEC> __device__ __forceinline__ void store_vec(__nv_bfloat16* p, const float* f) {
    if constexpr (VEC == 8)
        *reinterpret_cast<uint4*>(p) = make_uint4(bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3]), bf16_pair(f[4], f[5]), bf16_pair(f[6], f[7]));
    else *p = __float2bfloat16_rn(f[0]);
}
template <int VEC> __device__ __forceinline__ void store_vec(float* p, const float* f) {
    if constexpr (VEC == 4) *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
    else *p = f[0];
}
// VEC parameters of type TW (16-byte aligned for VEC > 1)
template <int VEC> __device__ __forceinline__ void load_params(const float* p, float* f) {
    if constexpr (VEC > 1) {
#pragma unroll
        for (int j = 0; j < VEC; j += 4) load_vec<4>(f + j, p + j);
    } else {
        f[0] = p[0];
    }
}
template <int VEC> __device__ __forceinline__ void load_params(const __nv_bfloat16* p, float* f) {
    if constexpr (VEC == 4) {
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        unpack_bf16x2(v.x, f[0], f[1]);
        unpack_bf16x2(v.y, f[2], f[3]);
    } else {
        load_vec<VEC>(f, p);
    }
}

// Sums of N values over the T threads of a row group (T a multiple of 32), the same order every time.  `scratch` is this
// group's [2][N][32] floats, zero to begin with; `turn` alternates between the two halves, so one barrier per sum is enough.
template <int N>
__device__ __forceinline__ void group_sum(float (&v)[N], float* scratch, int& turn, int threads, int barrier_id) {
#pragma unroll
    for (int o = 16; o; o >>= 1)
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], o);
    if (threads == 32) return;
    float* s = scratch + turn * 32 * N;
    turn ^= 1;
    if ((threadIdx.x & 31) == 0) {
#pragma unroll
        for (int k = 0; k < N; ++k) s[k * 32 + (threadIdx.x >> 5)] = v[k];
    }
    asm volatile("bar.sync %0, %1;" ::"r"(barrier_id), "r"(threads) : "memory");
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = 0.0f;
#pragma unroll 2
    for (int w = 0; w < threads >> 5; w += 4) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float4 p = *reinterpret_cast<const float4*>(s + k * 32 + w);
            v[k] += (p.x + p.y) + (p.z + p.w);
        }
    }
}
// Zeroes the CTA's scratch of `floats` values; the caller's __syncthreads follows.
__device__ __forceinline__ void zero_scratch(float* scratch, int floats) {
    for (int i = threadIdx.y * blockDim.x + threadIdx.x; i < floats; i += blockDim.x * blockDim.y) scratch[i] = 0.0f;
}

// ------------------------------------------------------------------------------------------------ rows through a ring
// A row group's ring of `slots` entries in shared memory: entry i % slots receives row `first + i * step` of one or two matrices.
// Thread 0 of the group issues the copies; an entry is refilled once the whole group has read it into registers (behind the
// barrier of the row's first sum).  Waits are bounded.  One that gives up sets the status word and the CTA's flag, and the threads, which
// still have to meet at the barriers, go through the rows that are left with what is there: no wait is tried a second time, nothing
// more is copied (an entry is refilled only by a thread that has seen its copy end), and the copies in flight are seen out.
struct RingHead {                                  // at the front of the CTA's dynamic shared memory
    int gave_up;
    int slots;
    long long limit;                               // of a wait, SM clocks
    int64_t step, rows;
};
constexpr int kRingHead = 32;
static_assert(sizeof(RingHead) == kRingHead, "RingHead");
extern __shared__ __align__(16) uint8_t ring_raw[];
constexpr int64_t kNoMore = (int64_t)1 << 61;      // the next row to be copied, where no more are (rows end at 2^60)
// A wait that did not end at once: true when it was given up.  Thread 0 then waits, bounded too, for its copies in flight (if there are):
// those of this row and of the slots - 1 that it takes after it.  A function of its own, with what it needs in shared memory: in line it
// cost the backward kernel 4 % (16384 x 4096 BF16 71.7 -> 74.8 us), and with more arguments 20 % by spilling (16384 x 1000 29.0 -> 34.7).
__device__ __noinline__ bool ring_wait_slow(uint32_t bars, int slot, uint32_t phase, int64_t row, bool in_flight) {
    RingHead* head = reinterpret_cast<RingHead*>(ring_raw);
    volatile int* gave_up = &head->gave_up;
    const long long limit = head->limit;
    if (!*gave_up && mbar_wait_slow(bars + 8u * (uint32_t)slot, phase, gave_up, &g_norm_status, limit)) return false;
    if (threadIdx.x == 0 && in_flight)
        for (int i = 0; i < head->slots && row < head->rows; ++i, row += head->step) {
            mbar_wait_drain(bars + 8u * (uint32_t)slot, phase, &g_norm_status, limit);
            if (++slot == head->slots) { slot = 0; phase ^= 1; }
        }
    return true;
}
__device__ __forceinline__ void init_ring_head(int slots, long long limit, int64_t step, int64_t rows) {
    if (threadIdx.x == 0 && threadIdx.y == 0) *reinterpret_cast<RingHead*>(ring_raw) = RingHead{0, slots, limit > 0 ? limit : WAIT_LIMIT_CYCLES, step, rows};
}
struct RowRing {
    uint32_t base, bars, entry_bytes;
    int slots;
    int slot = 0;                      // entry of the current row, and its phase
    uint32_t phase = 0;
    __device__ __forceinline__ uint32_t entry() const { return base + (uint32_t)slot * entry_bytes; }
    __device__ __forceinline__ uint32_t bar() const { return bars + 8u * (uint32_t)slot; }
    __device__ __forceinline__ void wait(int64_t row, int64_t& next) const {          // next: the thread's next row to be copied
        if (!mbar_try_wait(bar(), phase) && ring_wait_slow(bars, slot, phase, row, next < kNoMore)) next = kNoMore;
    }
    __device__ __forceinline__ void advance() {
        if (++slot == slots) { slot = 0; phase ^= 1; }
    }
};
// 16 bytes of a row (4 or 8 values) as pairs of binary32 values
__device__ __forceinline__ void lds_pairs(f32x2 (&f)[4], uint32_t addr, const __nv_bfloat16*) {
    uint32_t a, b, c, d;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(a), "=r"(b), "=r"(c), "=r"(d) : "r"(addr));
    f[0] = f2_from_bf16x2(a); f[1] = f2_from_bf16x2(b); f[2] = f2_from_bf16x2(c); f[3] = f2_from_bf16x2(d);
}
__device__ __forceinline__ void lds_pairs(f32x2 (&f)[2], uint32_t addr, const float*) {
    asm volatile("ld.shared.v2.u64 {%0, %1}, [%2];" : "=l"(f[0]), "=l"(f[1]) : "r"(addr));
}
__device__ __forceinline__ void stg_pairs(__nv_bfloat16* p, const f32x2 (&f)[4]) {
    uint32_t o[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float lo, hi;
        f2_unpack(f[j], lo, hi);
        o[j] = bf16_pair(lo, hi);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(o[0], o[1], o[2], o[3]);
}
__device__ __forceinline__ void stg_pairs(float* p, const f32x2 (&f)[2]) { *reinterpret_cast<ulonglong2*>(p) = make_ulonglong2(f[0], f[1]); }
__device__ __forceinline__ float f2_total(f32x2 v) {
    float lo, hi;
    f2_unpack(v, lo, hi);
    return lo + hi;
}

// ------------------------------------------------------------------------------------------------ forward
// blockDim = (T, R): R groups of T threads, a row each, NV 16-byte vectors per thread: 32 columns from 2048 columns on, 16 below.
// What a row costs besides its columns (two sums through shuffles and a barrier, ~150 instructions per warp) made 16 columns per
// thread issue-bound: 30.6 us at 8192 x 4096 BF16 against 24.4 us with 32 (24.4 to 27 by box; 5.5 TB/s, 0.84 of the measured copy; FP32 48.9 us, 0.84).  FULL: the columns fill the group's threads exactly, so
// nothing is conditional (a fifth of the instructions of a row go).
template <typename TX, typename TW, int NV, bool FULL>
__global__ void __launch_bounds__(512)
layer_norm_ring_kernel(const LayerNormArgs a, const int slots, const long long wait_limit) {
    constexpr int VEC = 16 / sizeof(TX), PAIRS = VEC / 2;
    uint8_t* ring_smem = ring_raw + kRingHead;
    const int T = blockDim.x, R = blockDim.y, bar_id = 1 + threadIdx.y;
    const uint32_t row_bytes = (uint32_t)a.cols * sizeof(TX), smem = smem_u32(ring_smem);
    // the head, [R][64] scratch, [R][slots] rows, [R][slots] barriers
    float* scratch = reinterpret_cast<float*>(ring_smem) + threadIdx.y * 64;
    RowRing ring{smem + R * 256 + threadIdx.y * slots * row_bytes, smem + R * 256 + R * slots * row_bytes + threadIdx.y * slots * 8, row_bytes, slots};
    const int nvec = (int)(a.cols / VEC);
    auto mine = [&](int k) { return FULL || threadIdx.x + k * T < nvec; };
    const int64_t step = (int64_t)gridDim.x * R, first = (int64_t)blockIdx.x * R + threadIdx.y;
    const TX* x = static_cast<const TX*>(a.x);
    const TX* src = x + first * a.ldx;                     // the next row to be copied
    int64_t next = wait_limit > 0 ? kNoMore : first;      // the self-test copies nothing
    auto fill = [&](uint32_t entry, uint32_t bar) {
        if (next < a.rows) {
            mbar_expect_tx(bar, row_bytes);
            bulk_load(entry, src, row_bytes, bar);
        }
        next += step;
        src += step * a.ldx;
    };
    if (threadIdx.x == 0) {
        for (int i = 0; i < slots; ++i) mbar_init(ring.bars + 8 * i, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_proxy_async();
        for (int i = 0; i < slots; ++i) fill(ring.base + i * row_bytes, ring.bars + 8 * i);
    }
    f32x2 w[NV][PAIRS], b[NV][PAIRS];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        float t[VEC], u[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) { t[j] = 1.0f; u[j] = 0.0f; }
        if (mine(k)) {
            if (a.weight) load_params<VEC>(static_cast<const TW*>(a.weight) + (int64_t)(threadIdx.x + k * T) * VEC, t);
            if (a.bias) load_params<VEC>(static_cast<const TW*>(a.bias) + (int64_t)(threadIdx.x + k * T) * VEC, u);
        }
#pragma unroll
        for (int j = 0; j < PAIRS; ++j) { w[k][j] = f2_pack(t[2 * j], t[2 * j + 1]); b[k][j] = f2_pack(u[2 * j], u[2 * j + 1]); }
    }
    zero_scratch(reinterpret_cast<float*>(ring_smem), R * 64);
    init_ring_head(slots, wait_limit, step, a.rows);
    __syncthreads();                                       // the barriers, the scratch and the head exist
    const float inv_n = 1.0f / (float)a.cols;
    int turn = 0;
    TX* dst = static_cast<TX*>(a.y) + first * a.ldy + threadIdx.x * VEC;
    for (int64_t row = first; row < a.rows; row += step, dst += step * a.ldy) {
        f32x2 f[NV][PAIRS], acc = 0;
        ring.wait(row, next);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if constexpr (!FULL) {
#pragma unroll
                for (int j = 0; j < PAIRS; ++j) f[k][j] = 0;
            }
            if (mine(k)) lds_pairs(f[k], ring.entry() + (threadIdx.x + k * T) * 16, x);
        }
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < PAIRS; ++j) acc = f2_add(acc, f[k][j]);   // columns beyond the row hold zeros
        float s[1] = {f2_total(acc)};
        group_sum<1>(s, scratch, turn, T, bar_id);
        __syncwarp();
        if (threadIdx.x == 0) fill(ring.entry(), ring.bar());
        ring.advance();
        const float mean = s[0] * inv_n;
        const f32x2 minus = f2_pack(-mean, -mean);
        acc = 0;
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (mine(k)) {
#pragma unroll
                for (int j = 0; j < PAIRS; ++j) { f[k][j] = f2_add(f[k][j], minus); acc = f2_fma(f[k][j], f[k][j], acc); }
            }
        s[0] = f2_total(acc);
        group_sum<1>(s, scratch, turn, T, bar_id);
        const float rstd = rsqrtf(fmaf(s[0], inv_n, a.eps));
        const f32x2 rr = f2_pack(rstd, rstd);
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (mine(k)) {
                f32x2 o[PAIRS];
#pragma unroll
                for (int j = 0; j < PAIRS; ++j) o[j] = f2_fma(f2_mul(f[k][j], rr), w[k][j], b[k][j]);
                stg_pairs(dst + (int64_t)k * T * VEC, o);
            }
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

// Rows without 16-byte alignment: NV single columns per thread, prefetched one row ahead; otherwise as above.  8000 x 1537 FP32 27.1 us
// (3.6 TB/s, 0.55 of the measured copy), 8192 x 1537 BF16 29.9 (1.7 TB/s): bound by the number of loads, one per element.
template <typename TX, typename TW, int NV, int MAXT>
__global__ void __launch_bounds__(MAXT)
layer_norm_kernel(const LayerNormArgs a) {
    constexpr bool KEEP = MAXT <= 512;
    extern __shared__ __align__(16) float scratch_all[];
    float* scratch = scratch_all + threadIdx.y * 64;
    zero_scratch(scratch_all, blockDim.y * 64);
    __syncthreads();
    const int T = blockDim.x, bar_id = 1 + threadIdx.y, n = (int)a.cols;
    const TX* x = static_cast<const TX*>(a.x);
    TX* y = static_cast<TX*>(a.y);
    auto weight = [&](int c) { return a.weight ? to_f32(static_cast<const TW*>(a.weight)[c]) : 1.0f; };
    auto bias = [&](int c) { return a.bias ? to_f32(static_cast<const TW*>(a.bias)[c]) : 0.0f; };
    float w[KEEP ? NV : 1], b[KEEP ? NV : 1];
    if constexpr (KEEP) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = threadIdx.x + k * T;
            w[k] = c < n ? weight(c) : 0.0f;
            b[k] = c < n ? bias(c) : 0.0f;
        }
    }
    const float inv_n = 1.0f / (float)a.cols;
    const int64_t step = (int64_t)gridDim.x * blockDim.y, first = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    Raw<TX> next[NV] = {};
    auto fetch = [&](int64_t r) {
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (threadIdx.x + k * T < n) load_raw(next[k], x + r * a.ldx + threadIdx.x + k * T);
    };
    if (first < a.rows) fetch(first);
    int turn = 0;
    for (int64_t row = first; row < a.rows; row += step) {
        float f[NV], s[1] = {0.0f};
#pragma unroll
        for (int k = 0; k < NV; ++k) { f[k] = unpack(next[k]); s[0] += f[k]; }      // columns beyond the row hold zeros
        if (row + step < a.rows) fetch(row + step);
        group_sum<1>(s, scratch, turn, T, bar_id);
        const float mean = s[0] * inv_n;
        s[0] = 0.0f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (threadIdx.x + k * T < n) { f[k] -= mean; s[0] = fmaf(f[k], f[k], s[0]); }
        group_sum<1>(s, scratch, turn, T, bar_id);
        const float rstd = rsqrtf(fmaf(s[0], inv_n, a.eps));
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = threadIdx.x + k * T;
            if (c < n) store_one(y + row * a.ldy + c, fmaf(f[k] * rstd, KEEP ? w[KEEP ? k : 0] : weight(c), KEEP ? b[KEEP ? k : 0] : bias(c)));
        }
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

// Rows of any length: the row is read three times (from L1/L2 after the first), VEC columns per access.
template <typename TX, typename TW, int VEC>
__global__ void __launch_bounds__(kMaxRowThreads) layer_norm_long_kernel(const LayerNormArgs a) {
    __shared__ __align__(16) float scratch[64];
    zero_scratch(scratch, 64);
    __syncthreads();
    const float inv_n = 1.0f / (float)a.cols;
    const int64_t stride = (int64_t)blockDim.x * VEC, c0 = (int64_t)threadIdx.x * VEC;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const TX* x = static_cast<const TX*>(a.x) + row * a.ldx;
        TX* y = static_cast<TX*>(a.y) + row * a.ldy;
        float s[1] = {0.0f};
#pragma unroll 2
        for (int64_t c = c0; c < a.cols; c += stride) {
            float f[VEC];
            load_vec<VEC>(f, x + c);
#pragma unroll
            for (int j = 0; j < VEC; ++j) s[0] += f[j];
        }
        group_sum<1>(s, scratch, turn, blockDim.x, 1);
        const float mean = s[0] * inv_n;
        s[0] = 0.0f;
#pragma unroll 2
        for (int64_t c = c0; c < a.cols; c += stride) {
            float f[VEC];
            load_vec<VEC>(f, x + c);
#pragma unroll
            for (int j = 0; j < VEC; ++j) s[0] = fmaf(f[j] - mean, f[j] - mean, s[0]);
        }
        group_sum<1>(s, scratch, turn, blockDim.x, 1);
        const float rstd = rsqrtf(fmaf(s[0], inv_n, a.eps));
        for (int64_t c = c0; c < a.cols; c += stride) {
            float f[VEC], w[VEC], b[VEC];
            load_vec<VEC>(f, x + c);
#pragma unroll
            for (int j = 0; j < VEC; ++j) { w[j] = 1.0f; b[j] = 0.0f; }
            if (a.weight) load_params<VEC>(static_cast<const TW*>(a.weight) + c, w);
            if (a.bias) load_params<VEC>(static_cast<const TW*>(a.bias) + c, b);
#pragma unroll
            for (int j = 0; j < VEC; ++j) f[j] = fmaf((f[j] - mean) * rstd, w[j], b[j]);
            store_vec<VEC>(y + c, f);
        }
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

// ------------------------------------------------------------------------------------------------ backward
// The R groups' column sums, added in order by the first group, to this CTA's row of the workspace.  `get(which, k, j)` is this
// thread's sum of column (thread + k T) VEC + j; `sums` has room for [R - 1][2][T * NV * VEC] values.
template <int VEC, int NV, typename Get>
__device__ __forceinline__ void leave_columns(const LayerNormArgs& a, float* sums, int nvec, Get get) {
    const int T = blockDim.x, R = blockDim.y, per_group = T * NV * VEC;
    __syncthreads();
    if (threadIdx.y > 0) {
        float* mine = sums + (threadIdx.y - 1) * 2 * per_group + threadIdx.x;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                // [.. ][k][j][thread]: a warp's stores fall into 32 different banks
                mine[(k * VEC + j) * T] = get(0, k, j);
                mine[per_group + (k * VEC + j) * T] = get(1, k, j);
            }
    }
    __syncthreads();
    if (threadIdx.y > 0) return;
    float* out = a.partial + (int64_t)blockIdx.x * 2 * a.cols;
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int vi = threadIdx.x + k * T;
            if (vi >= nvec) continue;
            float v[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                v[j] = get(which, k, j);
                for (int r = 0; r < R - 1; ++r) v[j] += sums[(r * 2 + which) * per_group + (k * VEC + j) * T + threadIdx.x];
            }
            float* p = out + which * a.cols + (int64_t)vi * VEC;
            if constexpr (VEC % 4 == 0) {
#pragma unroll
                for (int j = 0; j < VEC; j += 4) *reinterpret_cast<float4*>(p + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
            } else {
                *p = v[0];
            }
        }
}

// Rows of x and dy come through the ring (an entry holds both).  Dynamic shared memory: the head, [R][128] reduction scratch, [R][slots]
// barriers, [R][slots][2] rows; at the end the column sums over them.  16 columns per thread: weights, both column sums and both rows
// are 80 registers already.  16384 x 4096 BF16 with the adding kernel: 71.5 us, 5.6 TB/s (0.86 of the measured copy).
template <typename TX, typename TW, int NV, bool FULL>
__global__ void __launch_bounds__(512)
layer_norm_backward_ring_kernel(const LayerNormArgs a, const int slots, const long long wait_limit) {
    constexpr int VEC = 16 / sizeof(TX), PAIRS = VEC / 2;
    float* smem = reinterpret_cast<float*>(ring_raw + kRingHead);
    asm volatile("griddepcontrol.launch_dependents;");    // the adding kernel may take its place; it waits for this grid's end
    const int T = blockDim.x, R = blockDim.y, bar_id = 1 + threadIdx.y;
    float* scratch = smem + threadIdx.y * 128;
    const int nvec = (int)(a.cols / VEC);
    auto mine = [&](int k) { return FULL || threadIdx.x + k * T < nvec; };
    const uint32_t row_bytes = (uint32_t)a.cols * sizeof(TX), bars = smem_u32(smem + R * 128), rows0 = (bars + R * slots * 8 + 15u) & ~15u;
    RowRing ring{rows0 + threadIdx.y * slots * 2 * row_bytes, bars + threadIdx.y * slots * 8, 2 * row_bytes, slots};
    const int64_t step = (int64_t)gridDim.x * R, first = (int64_t)blockIdx.x * R + threadIdx.y;
    const TX* x = static_cast<const TX*>(a.x);
    const TX* src_x = x + first * a.ldx;                  // the next row to be copied
    const TX* src_dy = static_cast<const TX*>(a.dy) + first * a.lddy;
    int64_t next = wait_limit > 0 ? kNoMore : first;      // the self-test copies nothing
    auto fill = [&](uint32_t entry, uint32_t bar) {
        if (next < a.rows) {
            mbar_expect_tx(bar, 2 * row_bytes);
            bulk_load(entry, src_x, row_bytes, bar);
            bulk_load(entry + row_bytes, src_dy, row_bytes, bar);
        }
        next += step;
        src_x += step * a.ldx;
        src_dy += step * a.lddy;
    };
    if (threadIdx.x == 0) {
        for (int i = 0; i < slots; ++i) mbar_init(ring.bars + 8 * i, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_proxy_async();
        for (int i = 0; i < slots; ++i) fill(ring.base + i * 2 * row_bytes, ring.bars + 8 * i);
    }
    f32x2 w[NV][PAIRS], dw[NV][PAIRS], db[NV][PAIRS];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int vi = threadIdx.x + k * T;
        float t[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) t[j] = 1.0f;
        if (a.weight && mine(k)) load_params<VEC>(static_cast<const TW*>(a.weight) + (int64_t)vi * VEC, t);
#pragma unroll
        for (int j = 0; j < PAIRS; ++j) { w[k][j] = f2_pack(t[2 * j], t[2 * j + 1]); dw[k][j] = 0; db[k][j] = 0; }
    }
    zero_scratch(smem, R * 128);
    init_ring_head(slots, wait_limit, step, a.rows);
    __syncthreads();                                       // the barriers, the scratch and the head exist
    const float inv_n = 1.0f / (float)a.cols;
    float next_mean = 0.0f, next_rstd = 0.0f;
    if (first < a.rows) { next_mean = __ldg(a.mean + first); next_rstd = __ldg(a.rstd + first); }
    int turn = 0;
    TX* dst = static_cast<TX*>(a.y) + first * a.ldy + threadIdx.x * VEC;
    for (int64_t row = first; row < a.rows; row += step, dst += step * a.ldy) {
        const float mean = next_mean, rstd = next_rstd;
        if (row + step < a.rows) { next_mean = __ldg(a.mean + row + step); next_rstd = __ldg(a.rstd + row + step); }
        const f32x2 minus = f2_pack(-mean, -mean), rr = f2_pack(rstd, rstd);
        f32x2 xh[NV][PAIRS], g[NV][PAIRS], sg = 0, sgx = 0;
        ring.wait(row, next);
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (mine(k)) {
                lds_pairs(xh[k], ring.entry() + (threadIdx.x + k * T) * 16, x);
                lds_pairs(g[k], ring.entry() + row_bytes + (threadIdx.x + k * T) * 16, x);
#pragma unroll
                for (int j = 0; j < PAIRS; ++j) {
                    xh[k][j] = f2_mul(f2_add(xh[k][j], minus), rr);
                    dw[k][j] = f2_fma(g[k][j], xh[k][j], dw[k][j]);
                    db[k][j] = f2_add(db[k][j], g[k][j]);
                    g[k][j] = f2_mul(g[k][j], w[k][j]);
                    sg = f2_add(sg, g[k][j]);
                    sgx = f2_fma(g[k][j], xh[k][j], sgx);
                }
            }
        float s[2] = {f2_total(sg), f2_total(sgx)};
        group_sum<2>(s, scratch, turn, T, bar_id);
        __syncwarp();
        if (threadIdx.x == 0) fill(ring.entry(), ring.bar());
        ring.advance();
        // dx = g rstd - xh (mean(g xh) rstd) - mean(g) rstd
        const float mg = -s[0] * inv_n * rstd, mgx = -s[1] * inv_n * rstd;
        const f32x2 mg2 = f2_pack(mg, mg), mgx2 = f2_pack(mgx, mgx);
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (mine(k)) {
                f32x2 o[PAIRS];
#pragma unroll
                for (int j = 0; j < PAIRS; ++j) o[j] = f2_fma(g[k][j], rr, f2_fma(xh[k][j], mgx2, mg2));
                stg_pairs(dst + (int64_t)k * T * VEC, o);
            }
    }
    if (!a.partial) return;
    // every copy has been waited for: the rings' memory is free once all groups are here
    leave_columns<VEC, NV>(a, smem + R * 128, nvec, [&](int which, int k, int j) {
        float lo, hi;
        f2_unpack(which ? db[k][j / 2] : dw[k][j / 2], lo, hi);
        return (j & 1) ? hi : lo;
    });
}

// Rows without 16-byte alignment: single columns, prefetched one row ahead.  The fewer columns a thread has, the more loads of
// different rows are in flight and the shorter a row's chain, until a wide row's group leaves no second one beside it.  us at
// 4 columns per thread (768 threads) / 6 (768) / 16 (512):  FP32 1000 x 1537 11.3 / 11.6 / 16.6, 8000 x 1537 57.1 / 42.3 / 58.3; BF16
// 3000 x 1023 13.9 / 15.5 / -, 10000 x 333 15.0 / 15.5 / 25.0.  So 4 to 1024 columns, 6 as far as 768 threads reach, 16 beyond.
template <typename TX, typename TW, int NV, int MAXT>
__global__ void __launch_bounds__(MAXT)
layer_norm_backward_kernel(const LayerNormArgs a) {
    extern __shared__ __align__(16) float smem[];          // [R][128] reduction scratch, then the column sums
    asm volatile("griddepcontrol.launch_dependents;");
    const int T = blockDim.x, R = blockDim.y, bar_id = 1 + threadIdx.y, n = (int)a.cols;
    float* scratch = smem + threadIdx.y * 128;
    zero_scratch(smem, R * 128);
    __syncthreads();
    const TX* x = static_cast<const TX*>(a.x);
    const TX* dy = static_cast<const TX*>(a.dy);
    TX* dx = static_cast<TX*>(a.y);
    float w[NV], dw[NV], db[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int c = threadIdx.x + k * T;
        w[k] = a.weight && c < n ? to_f32(static_cast<const TW*>(a.weight)[c]) : 1.0f;
        dw[k] = db[k] = 0.0f;
    }
    const float inv_n = 1.0f / (float)a.cols;
    const int64_t step = (int64_t)gridDim.x * R, first = (int64_t)blockIdx.x * R + threadIdx.y;
    Raw<TX> nx[NV] = {}, ny[NV] = {};
    float next_mean = 0.0f, next_rstd = 0.0f;
    auto fetch = [&](int64_t r) {
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (threadIdx.x + k * T < n) {
                load_raw(nx[k], x + r * a.ldx + threadIdx.x + k * T);
                load_raw(ny[k], dy + r * a.lddy + threadIdx.x + k * T);
            }
        next_mean = __ldg(a.mean + r);
        next_rstd = __ldg(a.rstd + r);
    };
    if (first < a.rows) fetch(first);
    int turn = 0;
    for (int64_t row = first; row < a.rows; row += step) {
        float xh[NV], g[NV], s[2] = {0.0f, 0.0f};
        const float mean = next_mean, rstd = next_rstd;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            xh[k] = unpack(nx[k]);
            g[k] = unpack(ny[k]);
            if (threadIdx.x + k * T < n) {
                xh[k] = (xh[k] - mean) * rstd;
                dw[k] = fmaf(g[k], xh[k], dw[k]);
                db[k] += g[k];
                g[k] *= w[k];
                s[0] += g[k];
                s[1] = fmaf(g[k], xh[k], s[1]);
            }
        }
        if (row + step < a.rows) fetch(row + step);
        group_sum<2>(s, scratch, turn, T, bar_id);
        const float mg = s[0] * inv_n, mgx = s[1] * inv_n;
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (threadIdx.x + k * T < n) {
                store_one(dx + row * a.ldy + threadIdx.x + k * T, rstd * (g[k] - mg - xh[k] * mgx));
            }
    }
    if (a.partial) leave_columns<1, NV>(a, smem + R * 128, n, [&](int which, int k, int) { return which ? db[k] : dw[k]; });
}

// Rows of any length (over 8192 columns), one row per CTA at a time: x and dy are read twice, the second time from the caches.
// The column sums stay in shared memory up to 24576 columns, beyond that in this CTA's row of the workspace; a thread always
// has the same columns, so they need no order between threads.  VEC columns per access (1 where rows are not 16-byte aligned).
// 4096 x 16384 BF16: 191 us, 2.1 TB/s (0.32 of the measured copy): a row at a time per SM waits for its own loads.
template <typename TX, typename TW, int VEC>
__global__ void __launch_bounds__(kMaxRowThreads) layer_norm_backward_long_kernel(const LayerNormArgs a, const int sums_in_smem) {
    extern __shared__ __align__(16) float smem[];          // [128] reduction scratch, [2][cols] sums
    asm volatile("griddepcontrol.launch_dependents;");
    zero_scratch(smem, 128);
    const float inv_n = 1.0f / (float)a.cols;
    float* out = a.partial ? a.partial + (int64_t)blockIdx.x * 2 * a.cols : nullptr;
    const int64_t stride = (int64_t)blockDim.x * VEC, c0 = (int64_t)threadIdx.x * VEC;
    // where the sums of column c + j are: in shared memory a warp's threads side by side (no bank conflicts), else in order
    float* sums = sums_in_smem ? smem + 128 : out;
    const int64_t half = sums_in_smem ? (a.cols + stride - 1) / stride * stride : a.cols;
    auto at = [&](int64_t c, int j) { return sums_in_smem ? (c - c0) + j * (int64_t)blockDim.x + threadIdx.x : c + j; };
    if (sums)
        for (int64_t c = c0; c < a.cols; c += stride)
#pragma unroll
            for (int j = 0; j < VEC; ++j) sums[at(c, j)] = sums[half + at(c, j)] = 0.0f;
    __syncthreads();
    const TW* wp = static_cast<const TW*>(a.weight);
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const TX* x = static_cast<const TX*>(a.x) + row * a.ldx;
        const TX* dy = static_cast<const TX*>(a.dy) + row * a.lddy;
        TX* dx = static_cast<TX*>(a.y) + row * a.ldy;
        const float mean = a.mean[row], rstd = a.rstd[row];
        float s[2] = {0.0f, 0.0f};
#pragma unroll 2
        for (int64_t c = c0; c < a.cols; c += stride) {
            float xh[VEC], g[VEC], w[VEC];
            load_vec<VEC>(xh, x + c);
            load_vec<VEC>(g, dy + c);
            if (wp) load_params<VEC>(wp + c, w);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                xh[j] = (xh[j] - mean) * rstd;
                if (sums) {
                    sums[at(c, j)] = fmaf(g[j], xh[j], sums[at(c, j)]);
                    sums[half + at(c, j)] += g[j];
                }
                const float gw = wp ? g[j] * w[j] : g[j];
                s[0] += gw;
                s[1] = fmaf(gw, xh[j], s[1]);
            }
        }
        group_sum<2>(s, smem, turn, blockDim.x, 1);
        const float mg = s[0] * inv_n, mgx = s[1] * inv_n;
#pragma unroll 2
        for (int64_t c = c0; c < a.cols; c += stride) {
            float xh[VEC], g[VEC], w[VEC];
            load_vec<VEC>(xh, x + c);
            load_vec<VEC>(g, dy + c);
            if (wp) load_params<VEC>(wp + c, w);
#pragma unroll
            for (int j = 0; j < VEC; ++j) g[j] = rstd * ((wp ? g[j] * w[j] : g[j]) - mg - (xh[j] - mean) * rstd * mgx);
            store_vec<VEC>(dx + c, g);
        }
    }
    if (out && sums_in_smem)
        for (int64_t c = c0; c < a.cols; c += stride)
#pragma unroll
            for (int j = 0; j < VEC; ++j) { out[c + j] = sums[at(c, j)]; out[a.cols + c + j] = sums[half + at(c, j)]; }
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
        store_one(out + c, s);
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

// Ring entries per row group: as many as fit into about 100 KB with all groups of the CTA, 2 to 8.
int ring_slots(int groups, int64_t entry_bytes) {
    const int64_t fit = (100 * 1024) / (groups * entry_bytes);
    return (int)(fit < 2 ? 2 : (fit > 8 ? 8 : fit));
}
constexpr int kRingSmem = 200 * 1024;                    // dynamic shared memory asked for; the largest use is 2 x 64 KB + scratch

template <typename TX, typename TW, int PER, bool FULL>
cudaError_t run_forward_ring(const LayerNormArgs& a, long long wait_limit, int num_sms, cudaStream_t st) {
    constexpr int NV = PER * sizeof(TX) / 16;
    RowShape s = row_shape(a.cols, PER, 512);
    const int64_t spread = (a.rows + num_sms - 1) / num_sms;             // few rows: one group per SM rather than full CTAs
    if (s.groups > spread) s.groups = (int)spread;
    const int64_t row_bytes = a.cols * (int64_t)sizeof(TX);
    const int slots = ring_slots(s.groups, row_bytes);
    const size_t smem = (size_t)s.groups * (64 * sizeof(float) + slots * (row_bytes + 8)) + kRingHead;
    static std::atomic<int> granted[64];
    const cudaError_t e = allow_smem(layer_norm_ring_kernel<TX, TW, NV, FULL>, kRingSmem, granted);
    if (e != cudaSuccess) return e;
    const int64_t need = (a.rows + s.groups - 1) / s.groups;
    layer_norm_ring_kernel<TX, TW, NV, FULL><<<(unsigned)(need < num_sms ? need : num_sms), dim3(s.threads, s.groups), smem, st>>>(a, slots, wait_limit);
    return cudaGetLastError();
}

template <typename TX, typename TW, int NV, int MAXT>
cudaError_t run_forward(const LayerNormArgs& a, int num_sms, cudaStream_t st) {
    const RowShape s = row_shape(a.cols, NV, 128);
    const size_t smem = (size_t)s.groups * 64 * sizeof(float);
    // resident CTAs per SM of a CTA of so many warps: asked once (the library runs on one kind of device)
    static std::atomic<int> resident[kMaxRowThreads / 32 + 1];
    int per_sm = resident[s.threads * s.groups / 32].load(std::memory_order_relaxed);
    if (per_sm == 0) {
        const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, layer_norm_kernel<TX, TW, NV, MAXT>, s.threads * s.groups, smem);
        if (e != cudaSuccess) return e;
        resident[s.threads * s.groups / 32].store(per_sm, std::memory_order_relaxed);
    }
    const int64_t need = (a.rows + s.groups - 1) / s.groups, room = (int64_t)num_sms * (per_sm < 1 ? 1 : per_sm);
    layer_norm_kernel<TX, TW, NV, MAXT><<<(unsigned)(need < room ? need : room), dim3(s.threads, s.groups), smem, st>>>(a);
    return cudaGetLastError();
}

template <typename TX, typename TW>
cudaError_t forward_of(const LayerNormArgs& a, long long wait_limit, int num_sms, cudaStream_t st) {
    constexpr int V = 16 / sizeof(TX);
    const bool vec = a.cols % V == 0 && (a.ldx * (int64_t)sizeof(TX)) % 16 == 0 && (a.ldy * (int64_t)sizeof(TX)) % 16 == 0 &&
                     aligned(a.x, 16) && aligned(a.y, 16) && aligned(a.weight, 16) && aligned(a.bias, 16);
    if (a.cols > kRegisterCols) {
        const unsigned grid = (unsigned)(a.rows < 2 * num_sms ? a.rows : 2 * num_sms);
        if (vec) layer_norm_long_kernel<TX, TW, V><<<grid, kMaxRowThreads, 0, st>>>(a);
        else layer_norm_long_kernel<TX, TW, 1><<<grid, kMaxRowThreads, 0, st>>>(a);
        return cudaGetLastError();
    }
    if (vec && a.cols >= 2048) return a.cols % 1024 == 0 ? run_forward_ring<TX, TW, 32, true>(a, wait_limit, num_sms, st) : run_forward_ring<TX, TW, 32, false>(a, wait_limit, num_sms, st);
    if (vec) return a.cols % 512 == 0 ? run_forward_ring<TX, TW, 16, true>(a, wait_limit, num_sms, st) : run_forward_ring<TX, TW, 16, false>(a, wait_limit, num_sms, st);
    if (a.cols > kPerThread * 512) return run_forward<TX, TW, kPerThread, kMaxRowThreads>(a, num_sms, st);
    return a.cols <= 4 * 256 ? run_forward<TX, TW, 4, 256>(a, num_sms, st) : run_forward<TX, TW, kPerThread, 512>(a, num_sms, st);
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

template <typename TX, typename TW, bool RING, bool FULL, int PER, int CTA>
cudaError_t run_backward(const LayerNormArgs& a, long long wait_limit, cudaStream_t st) {
    RowShape s = row_shape(a.cols, PER, CTA);
    const int64_t spread = (a.rows + kBwdGroups - 1) / kBwdGroups;
    if (s.groups > spread) s.groups = spread < 1 ? 1 : (int)spread;
    const int64_t row_bytes = a.cols * (int64_t)sizeof(TX);
    const int slots = RING ? ring_slots(s.groups, 2 * row_bytes) : 0;
    const size_t ring = (size_t)s.groups * slots * (2 * row_bytes + 8) + 16;
    const size_t sums = (size_t)(s.groups - 1) * 2 * s.threads * PER * sizeof(float);
    const size_t smem = (RING ? kRingHead : 0) + (size_t)s.groups * 128 * sizeof(float) + (ring > sums ? ring : sums);
    const int64_t need = (a.rows + s.groups - 1) / s.groups;
    const int grid = (int)(need < kBwdGroups ? need : kBwdGroups);
    static std::atomic<int> granted[64];
    cudaError_t e = cudaSuccess;
    if constexpr (RING) {
        constexpr int NV = PER * sizeof(TX) / 16;
        e = allow_smem(layer_norm_backward_ring_kernel<TX, TW, NV, FULL>, kRingSmem, granted);
        if (e == cudaSuccess && grid > 0) layer_norm_backward_ring_kernel<TX, TW, NV, FULL><<<grid, dim3(s.threads, s.groups), smem, st>>>(a, slots, wait_limit);
    } else {
        e = allow_smem(layer_norm_backward_kernel<TX, TW, PER, CTA>, kRingSmem, granted);
        if (e == cudaSuccess && grid > 0) layer_norm_backward_kernel<TX, TW, PER, CTA><<<grid, dim3(s.threads, s.groups), smem, st>>>(a);
    }
    if (e == cudaSuccess) e = cudaGetLastError();
    return e != cudaSuccess || !a.partial ? e : add_columns<TW>(a, grid, st);
}

template <typename TX, typename TW>
cudaError_t backward_of(const LayerNormArgs& a, long long wait_limit, cudaStream_t st) {
    constexpr int V = 16 / sizeof(TX);
    const bool vec = a.cols % V == 0 && (a.ldx * (int64_t)sizeof(TX)) % 16 == 0 && (a.ldy * (int64_t)sizeof(TX)) % 16 == 0 &&
                     (a.lddy * (int64_t)sizeof(TX)) % 16 == 0 && aligned(a.x, 16) && aligned(a.y, 16) && aligned(a.dy, 16) && aligned(a.weight, 16);
    if (a.cols > (int64_t)kPerThread * 512) {
        const int grid = (int)(a.rows < kBwdGroups ? a.rows : kBwdGroups);
        const int in_smem = a.partial && a.cols <= 24576;
        const int64_t whole = vec ? (int64_t)kMaxRowThreads * V : kMaxRowThreads;          // columns of one trip of the CTA
        const size_t smem = 128 * sizeof(float) + (in_smem ? 2 * (size_t)((a.cols + whole - 1) / whole * whole) * sizeof(float) : 0);
        static std::atomic<int> granted[2][64];
        cudaError_t e = cudaSuccess;
        if (vec) {
            e = allow_smem(layer_norm_backward_long_kernel<TX, TW, V>, kRingSmem, granted[0]);
            if (e == cudaSuccess && grid > 0) layer_norm_backward_long_kernel<TX, TW, V><<<grid, kMaxRowThreads, smem, st>>>(a, in_smem);
        } else {
            e = allow_smem(layer_norm_backward_long_kernel<TX, TW, 1>, kRingSmem, granted[1]);
            if (e == cudaSuccess && grid > 0) layer_norm_backward_long_kernel<TX, TW, 1><<<grid, kMaxRowThreads, smem, st>>>(a, in_smem);
        }
        if (e == cudaSuccess) e = cudaGetLastError();
        return e != cudaSuccess || !a.partial ? e : add_columns<TW>(a, grid, st);
    }
    if (!vec && a.cols <= 1024) return run_backward<TX, TW, false, false, 4, 768>(a, wait_limit, st);
    if (!vec && a.cols <= 6 * 768) return run_backward<TX, TW, false, false, 6, 768>(a, wait_limit, st);
    if (!vec) return run_backward<TX, TW, false, false, kPerThread, 512>(a, wait_limit, st);
    return a.cols % (kPerThread * 32) == 0 ? run_backward<TX, TW, true, true, kPerThread, 512>(a, wait_limit, st) : run_backward<TX, TW, true, false, kPerThread, 512>(a, wait_limit, st);
}

}  // namespace

int layer_norm_backward_groups(int64_t rows) { return (int)(rows < kBwdGroups ? (rows < 1 ? 1 : rows) : kBwdGroups); }

cudaError_t launch_layer_norm(const LayerNormArgs& a, int dtype, int weight_dtype, int num_sms, cudaStream_t st, const StallTest& stall) {
    const long long limit = stall.wait_limit;
    if (dtype == UE5M3_BF16)
        return weight_dtype == UE5M3_BF16 ? forward_of<__nv_bfloat16, __nv_bfloat16>(a, limit, num_sms, st) : forward_of<__nv_bfloat16, float>(a, limit, num_sms, st);
    return weight_dtype == UE5M3_BF16 ? forward_of<float, __nv_bfloat16>(a, limit, num_sms, st) : forward_of<float, float>(a, limit, num_sms, st);
}
cudaError_t launch_layer_norm_backward(const LayerNormArgs& a, int dtype, int weight_dtype, cudaStream_t st, const StallTest& stall) {
    const long long limit = stall.wait_limit;
    if (dtype == UE5M3_BF16)
        return weight_dtype == UE5M3_BF16 ? backward_of<__nv_bfloat16, __nv_bfloat16>(a, limit, st) : backward_of<__nv_bfloat16, float>(a, limit, st);
    return weight_dtype == UE5M3_BF16 ? backward_of<float, __nv_bfloat16>(a, limit, st) : backward_of<float, float>(a, limit, st);
}

int read_and_clear_norm_status() {
    if (cudaDeviceSynchronize() != cudaSuccess) return UE5M3_ERR_CUDA;
    int v = 0;
    if (cudaMemcpyFromSymbol(&v, g_norm_status, sizeof(int)) != cudaSuccess) return UE5M3_ERR_CUDA;
    if (v != 0) {
        const int zero = 0;
        if (cudaMemcpyToSymbol(g_norm_status, &zero, sizeof(int)) != cudaSuccess) return UE5M3_ERR_CUDA;
    }
    return v;
}

}  // namespace ue5m3
