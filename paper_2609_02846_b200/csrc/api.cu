// C ABI of the UE5M3-FP4 library: argument checks on the host, then kernel launches.
#include <cuda_runtime.h>
#include <nvtx3/nvToolsExt.h>
#include <algorithm>
#include <cstdint>
#include <mutex>
#include "../../include/ue5m3.h"
#include "block_ops.h"
#include "launch.h"

namespace ue5m3 {

struct DeviceInfo { int ok; int sms; int major; };

static DeviceInfo device_info() {
    // one entry per device ordinal; filled once, on first use with that device current (concurrent first calls
    // are serialised by the once-flag; a failed query leaves ok = 0 for good)
    static DeviceInfo cache[64];
    static std::once_flag asked[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return DeviceInfo{0, 0, 0};
    std::call_once(asked[dev], [&]() {
        int sms = 0, major = 0;
        if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess &&
            cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) == cudaSuccess)
            cache[dev] = DeviceInfo{1, sms, major};
    });
    return cache[dev];
}

// One NVTX range per C-ABI call (visible in a timeline profiler; a no-op when no tool is attached).
struct ApiRange {
    explicit ApiRange(const char* name) { nvtxRangePushA(name); }
    ~ApiRange() { nvtxRangePop(); }
};

static inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace ue5m3

using namespace ue5m3;

extern "C" {

const char* ue5m3_status_string(int status) {
    switch (status) {
        case UE5M3_OK: return "UE5M3_OK";
        case UE5M3_ERR_INVALID_ARG: return "UE5M3_ERR_INVALID_ARG: null pointer, unknown enum value or non-positive size";
        case UE5M3_ERR_SHAPE: return "UE5M3_ERR_SHAPE: a dimension is not a multiple of what the call requires";
        case UE5M3_ERR_ALIGN: return "UE5M3_ERR_ALIGN: pointer or leading dimension not 16-byte aligned";
        case UE5M3_ERR_UNSUPPORTED: return "UE5M3_ERR_UNSUPPORTED: not implemented for these arguments or this device";
        case UE5M3_ERR_CUDA: return "UE5M3_ERR_CUDA: the CUDA runtime reported an error";
        case UE5M3_ERR_TIMEOUT: return "UE5M3_ERR_TIMEOUT: a device-side wait gave up";
        default: return "unknown UE5M3 status";
    }
}

size_t ue5m3_scales_bytes(int64_t rows, int64_t cols, int layout, int scale_layout) {
    if (rows <= 0 || cols <= 0 || (rows % 16) || (cols % 16)) return 0;
    if (layout == UE5M3_LAYOUT_2D) {
        if (scale_layout != UE5M3_SCALES_ROWMAJOR) return 0;
        return (size_t)(rows / 16) * (size_t)(cols / 16);
    }
    int64_t R, kb;
    if (layout == UE5M3_LAYOUT_1D_ROW) { R = rows; kb = cols / 16; }
    else if (layout == UE5M3_LAYOUT_1D_COL) { R = cols; kb = rows / 16; }
    else return 0;
    if (scale_layout == UE5M3_SCALES_ROWMAJOR) return (size_t)R * (size_t)kb;
    if (scale_layout == UE5M3_SCALES_TILED) return (size_t)((R + 127) / 128) * (size_t)((kb + 15) / 16) * 2048;
    return 0;
}

int ue5m3_sample_amax(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ld, float* amax_out, void* stream) {
    const ApiRange range_("ue5m3_sample_amax");
    if (!x || !amax_out || rows <= 0 || cols <= 0 || ld < cols) return UE5M3_ERR_INVALID_ARG;
    if (dtype != UE5M3_F32 && dtype != UE5M3_BF16) return UE5M3_ERR_INVALID_ARG;
    if (cols % 8) return UE5M3_ERR_SHAPE;
    const int64_t esz = dtype == UE5M3_F32 ? 4 : 2;
    if (!aligned16(x) || ((ld * esz) % 16) || (reinterpret_cast<uintptr_t>(amax_out) & 3u)) return UE5M3_ERR_ALIGN;
    const DeviceInfo di = device_info();
    if (!di.ok) return UE5M3_ERR_CUDA;
    if (di.major != 10) return UE5M3_ERR_UNSUPPORTED;
    return launch_amax(x, dtype, rows, cols, ld, amax_out, di.sms, (cudaStream_t)stream) == cudaSuccess ? UE5M3_OK
                                                                                                        : UE5M3_ERR_CUDA;
}

// Argument checks of ue5m3_quantize (layout without the block-size flag).
static int check_quantize_args(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ld, int layout, int block32,
                               int rounding, const float* amax_held, float target_T, const uint8_t* payload,
                               const uint8_t* scales, const uint8_t* payload_t, const uint8_t* scales_t,
                               const float* decode_out, const uint64_t* stats, int scale_layout) {
    if (!x || !amax_held || !payload || !scales || rows <= 0 || cols <= 0 || ld < cols) return UE5M3_ERR_INVALID_ARG;
    if (dtype != UE5M3_F32 && dtype != UE5M3_BF16) return UE5M3_ERR_INVALID_ARG;
    if (layout != UE5M3_LAYOUT_1D_ROW && layout != UE5M3_LAYOUT_1D_COL && layout != UE5M3_LAYOUT_2D) return UE5M3_ERR_INVALID_ARG;
    if (rounding != UE5M3_ROUND_RNE && rounding != UE5M3_ROUND_SR) return UE5M3_ERR_INVALID_ARG;
    if (scale_layout != UE5M3_SCALES_ROWMAJOR && scale_layout != UE5M3_SCALES_TILED) return UE5M3_ERR_INVALID_ARG;
    if (!(target_T > 0.0f) || target_T > 61440.0f || target_T != (float)(int)target_T) return UE5M3_ERR_INVALID_ARG;
    if ((payload_t == nullptr) != (scales_t == nullptr)) return UE5M3_ERR_INVALID_ARG;
    if (layout != UE5M3_LAYOUT_2D && payload_t) return UE5M3_ERR_INVALID_ARG;
    if (layout == UE5M3_LAYOUT_2D && scale_layout != UE5M3_SCALES_ROWMAJOR) return UE5M3_ERR_INVALID_ARG;
    if ((rows % 16) || (cols % 16)) return UE5M3_ERR_SHAPE;
    if (block32 && ((layout != UE5M3_LAYOUT_1D_COL && (cols % 32)) || (layout != UE5M3_LAYOUT_1D_ROW && (rows % 32)))) return UE5M3_ERR_SHAPE;
    const int64_t esz = dtype == UE5M3_F32 ? 4 : 2;
    if (!aligned16(x) || ((ld * esz) % 16) || !aligned16(payload) || !aligned16(scales)) return UE5M3_ERR_ALIGN;
    if (payload_t && (!aligned16(payload_t) || !aligned16(scales_t))) return UE5M3_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(amax_held) & 3u) || (reinterpret_cast<uintptr_t>(decode_out) & 3u) ||
        (reinterpret_cast<uintptr_t>(stats) & 7u))
        return UE5M3_ERR_ALIGN;
    if (rows * (cols / 16) >= ((int64_t)1 << 32) - 256) return UE5M3_ERR_UNSUPPORTED;   // 32-bit block index
    return UE5M3_OK;
}

int ue5m3_quantize(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ld, int layout, int rounding,
                   const float* amax_held, float target_T, uint64_t seed, uint8_t* payload, uint8_t* scales,
                   uint8_t* payload_t, uint8_t* scales_t, float* decode_out, uint64_t* stats, int scale_layout,
                   void* stream) {
    const ApiRange range_("ue5m3_quantize");
    const int block32 = (layout & UE5M3_BLOCK_32) ? 1 : 0;
    layout &= ~UE5M3_BLOCK_32;
    const int bad = check_quantize_args(x, dtype, rows, cols, ld, layout, block32, rounding, amax_held, target_T, payload, scales,
                                        payload_t, scales_t, decode_out, stats, scale_layout);
    if (bad != UE5M3_OK) return bad;
    const DeviceInfo di = device_info();
    if (!di.ok) return UE5M3_ERR_CUDA;
    if (di.major != 10) return UE5M3_ERR_UNSUPPORTED;
    QuantArgs a{x, rows, cols, ld, amax_held, target_T, seed, payload, scales, payload_t, scales_t, decode_out,
                reinterpret_cast<unsigned long long*>(stats)};
    a.block32 = block32;
    return launch_quantize(a, dtype, layout, rounding, scale_layout == UE5M3_SCALES_TILED, di.sms, (cudaStream_t)stream) == cudaSuccess
               ? UE5M3_OK
               : UE5M3_ERR_CUDA;
}

int ue5m3_quantize_current(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ld, int layout, int rounding,
                           float* amax_out, float target_T, uint64_t seed, uint8_t* payload, uint8_t* scales,
                           uint8_t* payload_t, uint8_t* scales_t, float* decode_out, uint64_t* stats, int scale_layout,
                           void* stream) {
    const ApiRange range_("ue5m3_quantize_current");
    // both calls' arguments are checked before anything is launched
    const int bad = check_quantize_args(x, dtype, rows, cols, ld, layout & ~UE5M3_BLOCK_32, (layout & UE5M3_BLOCK_32) ? 1 : 0,
                                        rounding, amax_out, target_T, payload, scales, payload_t, scales_t, decode_out, stats,
                                        scale_layout);
    if (bad != UE5M3_OK) return bad;
    const int rc = ue5m3_sample_amax(x, dtype, rows, cols, ld, amax_out, stream);
    if (rc != UE5M3_OK) return rc;
    return ue5m3_quantize(x, dtype, rows, cols, ld, layout, rounding, amax_out, target_T, seed, payload, scales, payload_t,
                          scales_t, decode_out, stats, scale_layout, stream);
}

int ue5m3_quantize_dual(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ld, int rounding,
                        const float* amax_held, float target_T_row, float target_T_col, uint64_t seed_row, uint64_t seed_col,
                        uint8_t* payload_row, uint8_t* scales_row, uint8_t* payload_col, uint8_t* scales_col,
                        float* decode_row, float* decode_col, uint64_t* stats_row, uint64_t* stats_col, int scale_layout,
                        void* stream) {
    const ApiRange range_("ue5m3_quantize_dual");
    if (!x || !amax_held || !payload_row || !scales_row || !payload_col || !scales_col || rows <= 0 || cols <= 0 || ld < cols)
        return UE5M3_ERR_INVALID_ARG;
    if (dtype != UE5M3_F32 && dtype != UE5M3_BF16) return UE5M3_ERR_INVALID_ARG;
    if (rounding != UE5M3_ROUND_RNE && rounding != UE5M3_ROUND_SR) return UE5M3_ERR_INVALID_ARG;
    if (scale_layout != UE5M3_SCALES_ROWMAJOR && scale_layout != UE5M3_SCALES_TILED) return UE5M3_ERR_INVALID_ARG;
    for (float T : {target_T_row, target_T_col})
        if (!(T > 0.0f) || T > 61440.0f || T != (float)(int)T) return UE5M3_ERR_INVALID_ARG;
    if ((stats_row == nullptr) != (stats_col == nullptr)) return UE5M3_ERR_INVALID_ARG;
    if ((rows % 16) || (cols % 16)) return UE5M3_ERR_SHAPE;
    const int64_t esz = dtype == UE5M3_F32 ? 4 : 2;
    if (!aligned16(x) || ((ld * esz) % 16) || !aligned16(payload_row) || !aligned16(scales_row) || !aligned16(payload_col) ||
        !aligned16(scales_col))
        return UE5M3_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(amax_held) & 3u) || (reinterpret_cast<uintptr_t>(decode_row) & 3u) ||
        (reinterpret_cast<uintptr_t>(decode_col) & 3u) || (reinterpret_cast<uintptr_t>(stats_row) & 7u) ||
        (reinterpret_cast<uintptr_t>(stats_col) & 7u))
        return UE5M3_ERR_ALIGN;
    if (rows * (cols / 16) >= ((int64_t)1 << 32) - 256) return UE5M3_ERR_UNSUPPORTED;
    const DeviceInfo di = device_info();
    if (!di.ok) return UE5M3_ERR_CUDA;
    if (di.major != 10) return UE5M3_ERR_UNSUPPORTED;
    QuantArgs a{x, rows, cols, ld, amax_held, target_T_col, seed_col, payload_col, scales_col, nullptr, nullptr, decode_col,
                reinterpret_cast<unsigned long long*>(stats_col),
                payload_row, scales_row, target_T_row, seed_row, decode_row, reinterpret_cast<unsigned long long*>(stats_row),
                0};
    return launch_quantize_dual(a, dtype, rounding, scale_layout == UE5M3_SCALES_TILED, (cudaStream_t)stream) == cudaSuccess
               ? UE5M3_OK
               : UE5M3_ERR_CUDA;
}

static int check_gemm_args(int op, int64_t Mo, int64_t No, int64_t Kc, const uint8_t* a_payload, const uint8_t* a_scales,
                           int a_scale_mode, const float* a_decode, const uint8_t* b_payload, const uint8_t* b_scales,
                           int b_scale_mode, const float* b_decode, void* out, int out_dtype, int64_t ldo, int64_t k_multiple) {
    if (op != UE5M3_FPROP && op != UE5M3_DGRAD && op != UE5M3_WGRAD) return UE5M3_ERR_INVALID_ARG;
    if (!a_payload || !a_scales || !a_decode || !b_payload || !b_scales || !b_decode || !out) return UE5M3_ERR_INVALID_ARG;
    if (Mo <= 0 || No <= 0 || Kc <= 0 || ldo < No) return UE5M3_ERR_INVALID_ARG;
    if (out_dtype != UE5M3_F32 && out_dtype != UE5M3_BF16) return UE5M3_ERR_INVALID_ARG;
    for (int m : {a_scale_mode, b_scale_mode})
        if (m != UE5M3_SCALE_1D && m != UE5M3_SCALE_1D_TILED && m != UE5M3_SCALE_2D) return UE5M3_ERR_INVALID_ARG;
    if ((Mo % 128) || (No % 128) || (Kc % k_multiple)) return UE5M3_ERR_SHAPE;
    const int64_t osz = out_dtype == UE5M3_F32 ? 4 : 2;
    if (!aligned16(a_payload) || !aligned16(b_payload) || !aligned16(a_scales) || !aligned16(b_scales) || !aligned16(out) ||
        ((ldo * osz) % 16))
        return UE5M3_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(a_decode) & 3u) || (reinterpret_cast<uintptr_t>(b_decode) & 3u)) return UE5M3_ERR_ALIGN;
    return UE5M3_OK;
}

int ue5m3_gemm(int op, int64_t Mo, int64_t No, int64_t Kc, const uint8_t* a_payload, const uint8_t* a_scales,
               int a_scale_mode, const float* a_decode, const uint8_t* b_payload, const uint8_t* b_scales,
               int b_scale_mode, const float* b_decode, void* out, int out_dtype, int64_t ldo, void* stream) {
    const ApiRange range_("ue5m3_gemm");
    const int bad = check_gemm_args(op, Mo, No, Kc, a_payload, a_scales, a_scale_mode, a_decode, b_payload, b_scales,
                                    b_scale_mode, b_decode, out, out_dtype, ldo, 128);
    if (bad != UE5M3_OK) return bad;
    const DeviceInfo di = device_info();
    if (!di.ok) return UE5M3_ERR_CUDA;
    if (di.major != 10) return UE5M3_ERR_UNSUPPORTED;
    GemmArgs g{Mo, No, Kc, a_payload, a_scales, a_scale_mode, a_decode, b_payload, b_scales, b_scale_mode, b_decode,
               out, out_dtype, ldo};
    if (!native_eligible(g)) return launch_gemm(g, nullptr, di.sms, (cudaStream_t)stream);
    // Three launches: the windows of the scale rows and the re-ordered scales, the native FP4 kernel (the tiles all of
    // whose scale rows have a UE4M3 window: normally all) and the FP16 kernel (the other tiles: normally none).
    int* ws = native_workspace(native_layout(g).bytes, (cudaStream_t)stream);
    if (!ws) return UE5M3_ERR_CUDA;
    int r = launch_scale_prepare(g, ws, di.sms, (cudaStream_t)stream);
    if (r != UE5M3_OK) return r;
    r = launch_gemm_native(g, ws, di.sms, (cudaStream_t)stream);
    if (r != UE5M3_OK) return r;
    return launch_gemm(g, ws, di.sms, (cudaStream_t)stream);
}

int ue5m3_gemm_static(int op, int64_t Mo, int64_t No, int64_t Kc, const uint8_t* a_payload, const uint8_t* a_scales,
                      int a_scale_mode, const float* a_decode, const uint8_t* b_payload, const uint8_t* b_scales,
                      int b_scale_mode, const float* b_decode, void* out, int out_dtype, int64_t ldo, void* stream) {
    const ApiRange range_("ue5m3_gemm_static");
    const int bad = check_gemm_args(op, Mo, No, Kc, a_payload, a_scales, a_scale_mode, a_decode, b_payload, b_scales,
                                    b_scale_mode, b_decode, out, out_dtype, ldo, 128);
    if (bad != UE5M3_OK) return bad;
    const DeviceInfo di = device_info();
    if (!di.ok) return UE5M3_ERR_CUDA;
    if (di.major != 10) return UE5M3_ERR_UNSUPPORTED;
    GemmArgs g{Mo, No, Kc, a_payload, a_scales, a_scale_mode, a_decode, b_payload, b_scales, b_scale_mode, b_decode,
               out, out_dtype, ldo};
    if (Kc % 256) return launch_gemm(g, nullptr, di.sms, (cudaStream_t)stream);      // the FP16 kernel alone: no workspace
    int* ws = static_workspace(native_layout(g).bytes);
    if (!ws) return UE5M3_ERR_UNSUPPORTED;            // larger operands than the file-scope array has room for
    int r = launch_scale_prepare(g, ws, di.sms, (cudaStream_t)stream);
    if (r != UE5M3_OK) return r;
    r = launch_gemm_native(g, ws, di.sms, (cudaStream_t)stream);
    if (r != UE5M3_OK) return r;
    return launch_gemm(g, ws, di.sms, (cudaStream_t)stream);
}

int ue5m3_gemm_fp16(int op, int64_t Mo, int64_t No, int64_t Kc, const uint8_t* a_payload, const uint8_t* a_scales,
                    int a_scale_mode, const float* a_decode, const uint8_t* b_payload, const uint8_t* b_scales,
                    int b_scale_mode, const float* b_decode, void* out, int out_dtype, int64_t ldo, void* stream) {
    const ApiRange range_("ue5m3_gemm_fp16");
    const int bad = check_gemm_args(op, Mo, No, Kc, a_payload, a_scales, a_scale_mode, a_decode, b_payload, b_scales,
                                    b_scale_mode, b_decode, out, out_dtype, ldo, 128);
    if (bad != UE5M3_OK) return bad;
    const DeviceInfo di = device_info();
    if (!di.ok) return UE5M3_ERR_CUDA;
    if (di.major != 10) return UE5M3_ERR_UNSUPPORTED;
    GemmArgs g{Mo, No, Kc, a_payload, a_scales, a_scale_mode, a_decode, b_payload, b_scales, b_scale_mode, b_decode,
               out, out_dtype, ldo};
    return launch_gemm(g, nullptr, di.sms, (cudaStream_t)stream);
}

size_t ue5m3_gemm_native_workspace_bytes(int64_t Mo, int64_t No, int64_t Kc, int a_scale_mode, int b_scale_mode) {
    if (Mo <= 0 || No <= 0 || Kc <= 0 || Kc % 256) return 0;
    GemmArgs g{};
    g.Mo = Mo; g.No = No; g.Kc = Kc; g.a_scale_mode = a_scale_mode; g.b_scale_mode = b_scale_mode;
    return native_layout(g).bytes;
}

int ue5m3_gemm_native(int op, int64_t Mo, int64_t No, int64_t Kc, const uint8_t* a_payload, const uint8_t* a_scales,
                      int a_scale_mode, const float* a_decode, const uint8_t* b_payload, const uint8_t* b_scales,
                      int b_scale_mode, const float* b_decode, void* out, int out_dtype, int64_t ldo, int32_t* workspace,
                      void* stream) {
    const ApiRange range_("ue5m3_gemm_native");
    const int bad = check_gemm_args(op, Mo, No, Kc, a_payload, a_scales, a_scale_mode, a_decode, b_payload, b_scales,
                                    b_scale_mode, b_decode, out, out_dtype, ldo, 256);
    if (bad != UE5M3_OK) return bad;
    if (!workspace) return UE5M3_ERR_INVALID_ARG;
    if (!aligned16(workspace)) return UE5M3_ERR_ALIGN;
    const DeviceInfo di = device_info();
    if (!di.ok) return UE5M3_ERR_CUDA;
    if (di.major != 10) return UE5M3_ERR_UNSUPPORTED;
    GemmArgs g{Mo, No, Kc, a_payload, a_scales, a_scale_mode, a_decode, b_payload, b_scales, b_scale_mode, b_decode,
               out, out_dtype, ldo};
    if (Kc % 256) return UE5M3_ERR_UNSUPPORTED;
    const int r = launch_scale_prepare(g, workspace, di.sms, (cudaStream_t)stream);
    if (r != UE5M3_OK) return r;
    return launch_gemm_native(g, workspace, di.sms, (cudaStream_t)stream);
}

int ue5m3_gemm_probe_matched(int op, int64_t Mo, int64_t No, int64_t Kc, const uint8_t* a_payload, const uint8_t* a_scales,
                             int a_scale_mode, const float* a_decode, const uint8_t* b_payload, const uint8_t* b_scales,
                             int b_scale_mode, const float* b_decode, int cross_rounding, int grid_denominator,
                             void* out, int out_dtype, int64_t ldo, void* stream) {
    const ApiRange range_("ue5m3_gemm_probe_matched");
    const int bad = check_gemm_args(op, Mo, No, Kc, a_payload, a_scales, a_scale_mode, a_decode, b_payload, b_scales,
                                    b_scale_mode, b_decode, out, out_dtype, ldo, 256);
    if (bad != UE5M3_OK) return bad;
    if (cross_rounding != 0 && cross_rounding != 1) return UE5M3_ERR_INVALID_ARG;
    if (grid_denominator < 0 || grid_denominator > 65536 || (grid_denominator & (grid_denominator - 1)))
        return UE5M3_ERR_INVALID_ARG;
    const DeviceInfo di = device_info();
    if (!di.ok) return UE5M3_ERR_CUDA;
    if (di.major != 10) return UE5M3_ERR_UNSUPPORTED;
    GemmArgs g{Mo, No, Kc, a_payload, a_scales, a_scale_mode, a_decode, b_payload, b_scales, b_scale_mode, b_decode,
               out, out_dtype, ldo};
    return launch_gemm_probe(g, cross_rounding, grid_denominator, di.sms, (cudaStream_t)stream);
}

int ue5m3_gemm_stall_selftest(int which, int64_t Mo, int64_t No, int64_t Kc, const uint8_t* a_payload, const uint8_t* a_scales,
                               int a_scale_mode, const float* a_decode, const uint8_t* b_payload, const uint8_t* b_scales,
                               int b_scale_mode, const float* b_decode, void* out, int out_dtype, int64_t ldo,
                               int64_t wait_limit_cycles, void* stream) {
    const ApiRange range_("ue5m3_gemm_stall_selftest");
    if (which != 0 && which != 1 && which != 2) return UE5M3_ERR_INVALID_ARG;
    if (wait_limit_cycles < 1000 || wait_limit_cycles > 4000000000LL) return UE5M3_ERR_INVALID_ARG;
    const int bad = check_gemm_args(UE5M3_FPROP, Mo, No, Kc, a_payload, a_scales, a_scale_mode, a_decode, b_payload, b_scales,
                                    b_scale_mode, b_decode, out, out_dtype, ldo, 256);
    if (bad != UE5M3_OK) return bad;
    const DeviceInfo di = device_info();
    if (!di.ok) return UE5M3_ERR_CUDA;
    if (di.major != 10) return UE5M3_ERR_UNSUPPORTED;
    GemmArgs g{Mo, No, Kc, a_payload, a_scales, a_scale_mode, a_decode, b_payload, b_scales, b_scale_mode, b_decode,
               out, out_dtype, ldo};
    g.wait_limit_cycles = wait_limit_cycles;
    g.stall_producer = 1;
    if (which == 2) {
        // the native kernel: its workspace is filled by the preparing kernel as in ue5m3_gemm (the operands must have windows)
        if (!native_eligible(g)) return UE5M3_ERR_UNSUPPORTED;
        int* ws = native_workspace(native_layout(g).bytes, (cudaStream_t)stream);
        if (!ws) return UE5M3_ERR_CUDA;
        const int r = launch_scale_prepare(g, ws, di.sms, (cudaStream_t)stream);
        if (r != UE5M3_OK) return r;
        return launch_gemm_native(g, ws, di.sms, (cudaStream_t)stream);
    }
    return which == 0 ? launch_gemm(g, nullptr, di.sms, (cudaStream_t)stream) : launch_gemm_probe(g, 0, 0, di.sms, (cudaStream_t)stream);
}

int ue5m3_unswizzle_scales(const uint8_t* in, uint8_t* out, int64_t R, int64_t kblocks, void* stream) {
    const ApiRange range_("ue5m3_unswizzle_scales");
    if (!in || !out || R <= 0 || kblocks <= 0) return UE5M3_ERR_INVALID_ARG;
    const DeviceInfo di = device_info();
    if (!di.ok) return UE5M3_ERR_CUDA;
    return launch_unswizzle(in, out, R, kblocks, (cudaStream_t)stream) == cudaSuccess ? UE5M3_OK : UE5M3_ERR_CUDA;
}

// ---------------------------------------------------------------------------------------------
// the operators between the linears
static inline bool known_dtype(int t) { return t == UE5M3_F32 || t == UE5M3_BF16; }
static inline bool aligned_to(const void* p, int dtype) { return (reinterpret_cast<uintptr_t>(p) & (dtype == UE5M3_F32 ? 3u : 1u)) == 0; }

static int device_ready(int& sms) {
    const DeviceInfo di = device_info();
    if (!di.ok) return UE5M3_ERR_CUDA;
    sms = di.sms;
    return di.major == 10 ? UE5M3_OK : UE5M3_ERR_UNSUPPORTED;
}

// Largest matrix these calls take: element offsets stay far inside 63 bits.
static inline bool too_large(int64_t rows, int64_t cols, int64_t ld) {
    const int64_t most = (int64_t)1 << 60;
    return cols > ((int64_t)1 << 31) - 8192 || (rows > 0 && ld > most / rows) || rows > most;
}

int ue5m3_layer_norm(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ldx, const void* weight, const void* bias,
                     int weight_dtype, float eps, void* y, int64_t ldy, float* mean, float* rstd, void* stream) {
    const ApiRange range_("ue5m3_layer_norm");
    if (rows < 0 || cols <= 0 || ldx < cols || ldy < cols || !known_dtype(dtype) || !known_dtype(weight_dtype)) return UE5M3_ERR_INVALID_ARG;
    if (!(eps >= 0.0f) || eps > 3.0e38f) return UE5M3_ERR_INVALID_ARG;
    if (rows > 0 && (!x || !y)) return UE5M3_ERR_INVALID_ARG;
    if (too_large(rows, cols, ldx) || too_large(rows, cols, ldy)) return UE5M3_ERR_UNSUPPORTED;
    if (!aligned_to(x, dtype) || !aligned_to(y, dtype) || !aligned_to(weight, weight_dtype) || !aligned_to(bias, weight_dtype) ||
        !aligned_to(mean, UE5M3_F32) || !aligned_to(rstd, UE5M3_F32))
        return UE5M3_ERR_ALIGN;
    int sms = 0;
    const int bad = device_ready(sms);
    if (bad != UE5M3_OK) return bad;
    if (rows == 0) return UE5M3_OK;
    LayerNormArgs a{};
    a.x = x; a.ldx = ldx; a.weight = weight; a.bias = bias; a.y = y; a.ldy = ldy; a.mean = mean; a.rstd = rstd;
    a.rows = rows; a.cols = cols; a.eps = eps;
    return launch_layer_norm(a, dtype, weight_dtype, sms, (cudaStream_t)stream) == cudaSuccess ? UE5M3_OK : UE5M3_ERR_CUDA;
}

size_t ue5m3_layer_norm_backward_workspace_bytes(int64_t rows, int64_t cols) {
    if (rows < 0 || cols <= 0 || too_large(rows, cols, cols)) return 0;
    return (size_t)layer_norm_backward_groups(rows) * 2 * (size_t)cols * sizeof(float);
}

int ue5m3_layer_norm_backward(const void* dy, int64_t lddy, const void* x, int dtype, int64_t rows, int64_t cols, int64_t ldx,
                              const void* weight, int weight_dtype, const float* mean, const float* rstd, void* dx, int64_t lddx,
                              void* dweight, void* dbias, void* workspace, void* stream) {
    const ApiRange range_("ue5m3_layer_norm_backward");
    if (rows < 0 || cols <= 0 || ldx < cols || lddy < cols || lddx < cols || !known_dtype(dtype) || !known_dtype(weight_dtype))
        return UE5M3_ERR_INVALID_ARG;
    if (rows > 0 && (!x || !dy || !dx || !mean || !rstd)) return UE5M3_ERR_INVALID_ARG;
    const bool sums = dweight || dbias;
    if (sums && !workspace) return UE5M3_ERR_INVALID_ARG;
    if (too_large(rows, cols, ldx) || too_large(rows, cols, lddy) || too_large(rows, cols, lddx)) return UE5M3_ERR_UNSUPPORTED;
    if (!aligned_to(x, dtype) || !aligned_to(dy, dtype) || !aligned_to(dx, dtype) || !aligned_to(weight, weight_dtype) ||
        !aligned_to(mean, UE5M3_F32) || !aligned_to(rstd, UE5M3_F32) || !aligned_to(dweight, weight_dtype) ||
        !aligned_to(dbias, weight_dtype) || !aligned16(workspace))
        return UE5M3_ERR_ALIGN;
    int sms = 0;
    const int bad = device_ready(sms);
    if (bad != UE5M3_OK) return bad;
    if (rows == 0 && !sums) return UE5M3_OK;
    LayerNormArgs a{};
    a.x = x; a.ldx = ldx; a.dy = dy; a.lddy = lddy; a.weight = weight; a.y = dx; a.ldy = lddx;
    a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd);
    a.dweight = dweight; a.dbias = dbias; a.partial = sums ? static_cast<float*>(workspace) : nullptr;
    a.rows = rows; a.cols = cols;
    return launch_layer_norm_backward(a, dtype, weight_dtype, (cudaStream_t)stream) == cudaSuccess ? UE5M3_OK : UE5M3_ERR_CUDA;
}

int ue5m3_dropout_add(const void* x, int64_t ldx, const void* residual, int64_t ldr, int dtype, int64_t rows, int64_t cols, float p,
                      uint64_t seed, void* y, int64_t ldy, void* stream) {
    const ApiRange range_("ue5m3_dropout_add");
    if (rows < 0 || cols < 0 || ldx < cols || ldy < cols || (residual && ldr < cols) || !known_dtype(dtype)) return UE5M3_ERR_INVALID_ARG;
    if (!(p >= 0.0f && p <= 1.0f)) return UE5M3_ERR_INVALID_ARG;
    const bool empty = rows == 0 || cols == 0;
    if (!empty && (!x || !y)) return UE5M3_ERR_INVALID_ARG;
    if (too_large(rows, cols, ldx) || too_large(rows, cols, ldy) || (residual && too_large(rows, cols, ldr))) return UE5M3_ERR_UNSUPPORTED;
    if (rows * cols > ((int64_t)1 << 40)) return UE5M3_ERR_UNSUPPORTED;      // blocks of 2048 elements are counted in 31 bits
    if (!aligned_to(x, dtype) || !aligned_to(residual, dtype) || !aligned_to(y, dtype)) return UE5M3_ERR_ALIGN;
    int sms = 0;
    const int bad = device_ready(sms);
    if (bad != UE5M3_OK) return bad;
    if (empty) return UE5M3_OK;
    const uint32_t t = (uint32_t)((double)p * 65536.0 + 0.5);
    DropoutArgs a{};
    a.x = x; a.residual = residual; a.y = y; a.ldx = ldx; a.ldr = ldr; a.ldy = ldy; a.rows = rows; a.cols = cols; a.seed = seed;
    a.drop = t != 0;
    a.limit = t ? (t << 16) - 1u : 0u;                     // t = 65536: no draw is above it
    a.inv_keep = t < 65536 ? (float)(65536.0 / (65536.0 - (double)t)) : 0.0f;
    return launch_dropout_add(a, dtype, (cudaStream_t)stream) == cudaSuccess ? UE5M3_OK : UE5M3_ERR_CUDA;
}

static int check_attention_shape(const ue5m3_attention_shape* s) {
    if (!s || s->batch < 0 || s->q_len < 0 || s->k_len < 0 || s->heads <= 0 || s->kv_heads <= 0 || s->head_dim <= 0) return UE5M3_ERR_INVALID_ARG;
    if (s->window_left < -1 || (s->causal != 0 && s->causal != 1) || !(s->scale > 0.0f) || s->scale > 3.0e38f) return UE5M3_ERR_INVALID_ARG;
    if (!known_dtype(s->dtype)) return UE5M3_ERR_INVALID_ARG;
    if ((s->head_dim % 8) || (s->heads % s->kv_heads)) return UE5M3_ERR_SHAPE;
    if (s->dtype != UE5M3_BF16 || s->head_dim > 128) return UE5M3_ERR_UNSUPPORTED;
    const int64_t most = (int64_t)1 << 30;
    if (s->q_len > most || s->k_len > most || s->batch > most || s->heads > most || s->batch * s->heads > most) return UE5M3_ERR_UNSUPPORTED;
    if (reinterpret_cast<uintptr_t>(s->k_lens) & 3u) return UE5M3_ERR_ALIGN;
    return UE5M3_OK;
}
// Where the elements of a tensor of an attention call lie, in units of eight elements (16 bytes): pointers, strides and the head
// dimension are whole numbers of them.  Dimensions of size 1 have no stride.
struct Extent { int64_t base, sizes[4], strides[4], last; };             // last: units from the first to the last
static Extent extent_of(const ue5m3_heads& t, int64_t batch, int64_t tokens, int64_t heads, int64_t dim) {
    Extent e{(int64_t)(reinterpret_cast<uintptr_t>(t.data) >> 4), {batch, tokens, heads, dim / 8},
             {t.batch_stride / 8, t.token_stride / 8, t.head_stride / 8, 1}, 0};
    for (int i = 0; i < 4; ++i) e.last += (e.sizes[i] - 1) * (e.sizes[i] > 1 ? e.strides[i] : 0);
    return e;
}
// Do two tensors have an element in common?  base_a - base_b + sum of strides * indices of a - those of b = 0 is solved stride by stride
// from the largest down: what the smaller ones reach leaves one or two values of each index where rows do not lie on one another, as in
// all views of a buffer.  Layouts that need more than a few thousand steps are taken as apart: this check finds mistakes, and the
// caller's promise covers the rest.
struct Term { int64_t stride, lo, hi; };
static bool meets(const Term* t, int n, int64_t r, int& budget) {
    if (n == 0) return r == 0;
    int64_t least = 0, most = 0;
    for (int i = 1; i < n; ++i) { least += t[i].lo * t[i].stride; most += t[i].hi * t[i].stride; }
    auto down = [](int64_t a, int64_t b) { return a >= 0 ? a / b : -((-a + b - 1) / b); };
    const int64_t from = std::max(t[0].lo, -down(r + most, t[0].stride)), to = std::min(t[0].hi, down(-r - least, t[0].stride));
    for (int64_t x = from; x <= to && budget-- > 0; ++x)
        if (meets(t + 1, n - 1, r + x * t[0].stride, budget)) return true;
    return false;
}
static bool overlap(const Extent& a, const Extent& b) {
    if (a.base > b.base + b.last || b.base > a.base + a.last) return false;
    Term t[8];
    int n = 0;
    auto add = [&](int64_t stride, int64_t lo, int64_t hi) {
        for (int i = 0; i < n; ++i)
            if (t[i].stride == stride) { t[i].lo += lo; t[i].hi += hi; return; }
        t[n++] = Term{stride, lo, hi};
    };
    for (int i = 0; i < 4; ++i) {
        if (a.sizes[i] > 1) add(a.strides[i], 0, a.sizes[i] - 1);
        if (b.sizes[i] > 1) add(b.strides[i], 1 - b.sizes[i], 0);
    }
    std::sort(t, t + n, [](const Term& x, const Term& y) { return x.stride > y.stride; });
    int budget = 4096;
    return meets(t, n, a.base - b.base, budget);
}
static bool same_layout(const Extent& a, const Extent& b) {               // of tensors of the same sizes
    for (int i = 0; i < 3; ++i)
        if (a.sizes[i] > 1 && a.strides[i] != b.strides[i]) return false;
    return a.base == b.base;
}

// One tensor [batch, tokens, heads, head_dim] of an attention call.
static int check_heads(const ue5m3_heads* t, int64_t batch, int64_t tokens, int64_t heads) {
    if (!t) return UE5M3_ERR_INVALID_ARG;
    if (batch == 0 || tokens == 0) return UE5M3_OK;
    if (!t->data) return UE5M3_ERR_INVALID_ARG;
    if (!aligned16(t->data)) return UE5M3_ERR_ALIGN;
    const int64_t sizes[3] = {batch, tokens, heads}, strides[3] = {t->batch_stride, t->token_stride, t->head_stride};
    for (int i = 0; i < 3; ++i) {
        if (sizes[i] <= 1) continue;
        if (strides[i] <= 0 || strides[i] % 8) return UE5M3_ERR_ALIGN;
        if (strides[i] >= ((int64_t)1 << 39)) return UE5M3_ERR_UNSUPPORTED;      // a tensor map's strides end at 2^40 bytes
        if (sizes[i] > ((int64_t)1 << 58) / strides[i]) return UE5M3_ERR_UNSUPPORTED;       // no such memory
    }
    return UE5M3_OK;
}

// Binary32 o and lse of every part.
size_t ue5m3_attention_workspace_bytes(const ue5m3_attention_shape* shape) {
    if (check_attention_shape(shape) != UE5M3_OK) return 0;
    const int parts = attention_splits(*shape);
    if (parts <= 1) return 0;
    return (size_t)parts * (size_t)shape->batch * (size_t)shape->heads * (size_t)shape->q_len * (size_t)(shape->head_dim + 4) * sizeof(float);
}

int ue5m3_attention(const ue5m3_attention_shape* shape, const ue5m3_heads* q, const ue5m3_heads* k, const ue5m3_heads* v,
                    const ue5m3_heads* o, float* lse, void* workspace, void* stream) {
    const ApiRange range_("ue5m3_attention");
    int bad = check_attention_shape(shape);
    if (bad != UE5M3_OK) return bad;
    const ue5m3_attention_shape& s = *shape;
    for (const ue5m3_heads* t : {q, o})
        if ((bad = check_heads(t, s.batch, s.q_len, s.heads)) != UE5M3_OK) return bad;
    for (const ue5m3_heads* t : {k, v})
        if ((bad = check_heads(t, s.batch, s.k_len, s.kv_heads)) != UE5M3_OK) return bad;
    if (!lse && s.batch * s.q_len > 0) return UE5M3_ERR_INVALID_ARG;
    if (!workspace && attention_splits(s) > 1) return UE5M3_ERR_INVALID_ARG;
    if (s.batch * s.q_len > 0) {
        const Extent eo = extent_of(*o, s.batch, s.q_len, s.heads, s.head_dim), eq = extent_of(*q, s.batch, s.q_len, s.heads, s.head_dim);
        // in place of q: a CTA that writes rows of o is the only one that reads these rows of q, and has read them
        if (!same_layout(eo, eq) && overlap(eo, eq)) return UE5M3_ERR_INVALID_ARG;
        if (s.k_len > 0)
            for (const ue5m3_heads* t : {k, v})
                if (overlap(eo, extent_of(*t, s.batch, s.k_len, s.kv_heads, s.head_dim))) return UE5M3_ERR_INVALID_ARG;
    }
    if (!aligned_to(lse, UE5M3_F32) || !aligned16(workspace)) return UE5M3_ERR_ALIGN;
    int sms = 0;
    if ((bad = device_ready(sms)) != UE5M3_OK) return bad;
    return launch_attention(s, *q, *k, *v, *o, lse, static_cast<float*>(workspace), sms, (cudaStream_t)stream);
}

size_t ue5m3_attention_backward_workspace_bytes(const ue5m3_attention_shape* shape) {
    if (check_attention_shape(shape) != UE5M3_OK) return 0;
    const int parts = attention_backward_splits(*shape);
    const size_t heads = (size_t)shape->batch * (size_t)shape->heads;
    // two numbers per query, padded to whole tiles; binary32 dq of every part
    return (heads * (size_t)attention_padded_q(shape->q_len) * 2 +
            (parts > 1 ? (size_t)parts * heads * (size_t)shape->q_len * (size_t)shape->head_dim : 0)) * sizeof(float);
}

int ue5m3_attention_backward(const ue5m3_attention_shape* shape, const ue5m3_heads* dout, const ue5m3_heads* q, const ue5m3_heads* k,
                             const ue5m3_heads* v, const ue5m3_heads* o, const float* lse, const ue5m3_heads* dq, const ue5m3_heads* dk,
                             const ue5m3_heads* dv, void* workspace, void* stream) {
    const ApiRange range_("ue5m3_attention_backward");
    int bad = check_attention_shape(shape);
    if (bad != UE5M3_OK) return bad;
    const ue5m3_attention_shape& s = *shape;
    for (const ue5m3_heads* t : {dout, q, o, dq})
        if ((bad = check_heads(t, s.batch, s.q_len, s.heads)) != UE5M3_OK) return bad;
    for (const ue5m3_heads* t : {k, v, dk, dv})
        if ((bad = check_heads(t, s.batch, s.k_len, s.kv_heads)) != UE5M3_OK) return bad;
    if ((!lse || !workspace) && s.batch * s.q_len > 0) return UE5M3_ERR_INVALID_ARG;
    {
        // dk and dv are written while dq still reads the inputs, and the other way round; o is read before either
        Extent e[7];                                          // dq, dk, dv, then what they may not meet
        int n = 0;
        bool is_output[7];
        auto take = [&](const ue5m3_heads* t, int64_t tokens, int64_t heads, bool output) {
            if (s.batch * tokens == 0) return;
            is_output[n] = output;
            e[n++] = extent_of(*t, s.batch, tokens, heads, s.head_dim);
        };
        take(dq, s.q_len, s.heads, true);
        for (const ue5m3_heads* t : {dk, dv}) take(t, s.k_len, s.kv_heads, true);
        for (const ue5m3_heads* t : {dout, q}) take(t, s.q_len, s.heads, false);
        for (const ue5m3_heads* t : {k, v}) take(t, s.k_len, s.kv_heads, false);
        for (int i = 0; i < n && is_output[i]; ++i)
            for (int j = i + 1; j < n; ++j)
                if (overlap(e[i], e[j])) return UE5M3_ERR_INVALID_ARG;
    }
    if (!aligned_to(lse, UE5M3_F32) || !aligned16(workspace)) return UE5M3_ERR_ALIGN;
    int sms = 0;
    if ((bad = device_ready(sms)) != UE5M3_OK) return bad;
    return launch_attention_backward(s, *dout, *q, *k, *v, *o, lse, *dq, *dk, *dv, static_cast<float*>(workspace), (cudaStream_t)stream);
}

// Self-test problems: 4500 rows of 64 columns in BF16, three to each of the 148 x 15 row groups; one sequence, heads of 64 that share one key/value head, 300 queries of two heads on 300 keys or one query of
// four on 4096 (one tile for all heads, keys shared out).  The tensors lie one behind the other in the caller's buffer.
int ue5m3_block_stall_selftest(int which, void* buffer, size_t bytes, int64_t wait_limit_cycles, void* stream) {
    const ApiRange range_("ue5m3_block_stall_selftest");
    if (which < 0 || which > 4 || !buffer || bytes < UE5M3_BLOCK_SELFTEST_BYTES) return UE5M3_ERR_INVALID_ARG;
    if (wait_limit_cycles < 1000 || wait_limit_cycles > 4000000000LL) return UE5M3_ERR_INVALID_ARG;
    if (!aligned16(buffer)) return UE5M3_ERR_ALIGN;
    int sms = 0;
    const int bad = device_ready(sms);
    if (bad != UE5M3_OK) return bad;
    const StallTest stall{wait_limit_cycles};
    char* at = static_cast<char*>(buffer);
    auto take = [&](size_t n) { char* p = at; at += (n + 255) / 256 * 256; return static_cast<void*>(p); };
    if (which >= 3) {
        const int64_t rows = 4500, cols = 64;
        const size_t matrix = (size_t)(rows * cols) * 2;
        LayerNormArgs a{};
        a.y = take(matrix);
        a.x = take(matrix);
        a.ldx = a.ldy = a.lddy = a.cols = cols;
        a.mean = static_cast<float*>(take(rows * sizeof(float)));
        a.rstd = static_cast<float*>(take(rows * sizeof(float)));
        a.rows = rows;
        if (which == 3) return launch_layer_norm(a, UE5M3_BF16, UE5M3_F32, sms, (cudaStream_t)stream, stall) == cudaSuccess ? UE5M3_OK : UE5M3_ERR_CUDA;
        a.dy = take(matrix);
        a.dweight = take(cols * sizeof(float));
        a.dbias = take(cols * sizeof(float));
        a.partial = static_cast<float*>(take(ue5m3_layer_norm_backward_workspace_bytes(rows, cols)));
        return launch_layer_norm_backward(a, UE5M3_BF16, UE5M3_F32, (cudaStream_t)stream, stall) == cudaSuccess ? UE5M3_OK : UE5M3_ERR_CUDA;
    }
    ue5m3_attention_shape s{};
    s.batch = s.kv_heads = 1;
    s.heads = which == 1 ? 4 : 2;
    s.q_len = which == 1 ? 1 : 300;
    s.k_len = which == 1 ? 4096 : 300;
    s.head_dim = 64;
    s.window_left = -1;
    s.scale = 0.125f;
    s.dtype = UE5M3_BF16;
    auto tensor = [&](int64_t tokens, int64_t heads) {
        return ue5m3_heads{take((size_t)(tokens * heads * s.head_dim) * 2), tokens * heads * s.head_dim, heads * s.head_dim, s.head_dim};
    };
    const ue5m3_heads o = tensor(s.q_len, s.heads), q = tensor(s.q_len, s.heads), k = tensor(s.k_len, 1), v = tensor(s.k_len, 1);
    float* lse = static_cast<float*>(take((size_t)(s.heads * s.q_len) * sizeof(float)));
    if (which < 2) {
        float* ws = static_cast<float*>(take(ue5m3_attention_workspace_bytes(&s)));
        return launch_attention(s, q, k, v, o, lse, ws, sms, (cudaStream_t)stream, stall);
    }
    const ue5m3_heads dout = tensor(s.q_len, s.heads), dq = tensor(s.q_len, s.heads), dk = tensor(s.k_len, 1), dv = tensor(s.k_len, 1);
    float* ws = static_cast<float*>(take(ue5m3_attention_backward_workspace_bytes(&s)));
    return launch_attention_backward(s, dout, q, k, v, o, lse, dq, dk, dv, ws, (cudaStream_t)stream, stall);
}

int ue5m3_last_device_status(void) {
    const int a = read_and_clear_device_status();
    const int b = read_and_clear_probe_status();
    const int c = read_and_clear_native_status();
    const int d = read_and_clear_attention_status();
    const int e = read_and_clear_attention_backward_status();
    const int f = read_and_clear_norm_status();
    for (int v : {a, b, c, d, e, f})
        if (v != UE5M3_OK) return v;
    return UE5M3_OK;
}

}  // extern "C"
