// The microscaled operators' C ABI (include/ssd_mx.h): validation and dispatch.
#include <cmath>

#include "../../include/ssd_mx.h"
#include "mx.h"
#include "ssd_internal.h"

#define SSD_API extern "C" __attribute__((visibility("default")))

static bool off16(const void* p) { return ((uintptr_t)p & 15) != 0; }

// rows and columns of a microscaled matrix
static int check_shape(const char* who, long long rows, long long cols) {
    if (rows < 1 || cols < 32 || cols % 32) return fail_without_ctx(SSD_EINVAL, "%s: %lld rows of %lld columns: at least one row, columns a multiple of 32", who, rows, cols);
    if (cols > SSD_MX_MAX_COLS || rows > SSD_MX_MAX_ROWS) return fail_without_ctx(SSD_ERANGE, "%s: %lld x %lld is beyond the supported size", who, rows, cols);
    return SSD_OK;
}
static int launched(const char* who) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SSD_OK : fail_without_ctx(SSD_EHIP, "%s: %s", who, hipGetErrorString(e));
}

SSD_API size_t ssd_mx_scale_bytes(int rows, int cols) {
    if (check_shape("ssd_mx_scale_bytes", rows, cols) != SSD_OK) return 0;
    return (size_t)mx_groups(cols) * mx_pad_rows(rows) * 4;
}

SSD_API int ssd_mx_quantize(const void* src, int dtype, int rows, int cols, int format, void* codes, void* scales, void* values, void* hip_stream) {
    const char* who = "ssd_mx_quantize";
    if (!src || !codes || !scales) return fail_without_ctx(SSD_EINVAL, "%s: null pointer", who);
    if (dtype != SSD_F32 && dtype != SSD_BF16) return fail_without_ctx(SSD_EINVAL, "%s: dtype must be SSD_F32 or SSD_BF16", who);
    if (format != SSD_MX_FP4 && format != SSD_MX_FP8) return fail_without_ctx(SSD_EINVAL, "%s: format must be SSD_MX_FP4 or SSD_MX_FP8", who);
    const int rc = check_shape(who, rows, cols);
    if (rc != SSD_OK) return rc;
    if (off16(src) || off16(codes) || off16(scales) || off16(values)) return fail_without_ctx(SSD_EINVAL, "%s: a pointer off a 16-byte boundary", who);
    mx_launch_quantize(src, dtype, rows, cols, format, codes, scales, values, (hipStream_t)hip_stream);
    return launched(who);
}

SSD_API int ssd_mx_norm(const float* h, const float* partials, int n_part, const float* gain, float eps, int rows, int cols, float* h_out,
                        void* codes, void* scales, void* hip_stream) {
    const char* who = "ssd_mx_norm";
    if (!h || !gain || !codes || !scales || (n_part > 0 && !partials)) return fail_without_ctx(SSD_EINVAL, "%s: null pointer", who);
    if (n_part < 0) return fail_without_ctx(SSD_EINVAL, "%s: n_part < 0", who);
    if (n_part > SSD_MAX_SPLIT) return fail_without_ctx(SSD_ERANGE, "%s: %d partial sums, at most %d", who, n_part, SSD_MAX_SPLIT);
    if (!(eps >= 0.f)) return fail_without_ctx(SSD_EINVAL, "%s: eps must not be negative", who);
    const int rc = check_shape(who, rows, cols);
    if (rc != SSD_OK) return rc;
    if (cols > 8192) return fail_without_ctx(SSD_ERANGE, "%s: %d columns, at most 8192", who, cols);
    if (off16(h) || off16(partials) || off16(gain) || off16(h_out) || off16(codes) || off16(scales)) return fail_without_ctx(SSD_EINVAL, "%s: a pointer off a 16-byte boundary", who);
    mx_launch_norm(h, partials, n_part, (size_t)rows * cols, gain, eps, rows, cols, h_out, codes, scales, (hipStream_t)hip_stream);
    return launched(who);
}

static int check_linear(const char* who, int M, int N, int K, int result) {
    if (result != SSD_MX_OUT_F32 && result != SSD_MX_OUT_BF16 && result != SSD_MX_OUT_SWIGLU) return fail_without_ctx(SSD_EINVAL, "%s: unknown result %d", who, result);
    int rc = check_shape(who, M, K);
    if (rc == SSD_OK) rc = check_shape(who, N, 32);
    if (rc != SSD_OK) return rc;
    if (result == SSD_MX_OUT_SWIGLU && N % 64) return fail_without_ctx(SSD_EINVAL, "%s: gate and up rows need N a multiple of 64, got %d", who, N);
    if ((long long)M * N > SSD_MX_MAX_OUT) return fail_without_ctx(SSD_ERANGE, "%s: %d x %d outputs are beyond the supported size", who, M, N);
    return SSD_OK;
}
// Slices with columns in them: fewer than mx_split asks for where the columns run out
static int slices_of(int N, int K, int result) { return mx_slices(K, mx_split(N, K, result == SSD_MX_OUT_SWIGLU)); }

SSD_API size_t ssd_mx_linear_workspace(int M, int N, int K, int result) {
    if (check_linear("ssd_mx_linear_workspace", M, N, K, result) != SSD_OK) return 0;
    const int s = slices_of(N, K, result);
    return s > 1 ? (size_t)s * M * N * 4 : 0;
}

SSD_API int ssd_mx_linear(const void* x_codes, const void* x_scales, int M, const void* w_codes, const void* w_scales, int N, int K, int result,
                          void* out, void* out_scales, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const char* who = "ssd_mx_linear";
    if (!x_codes || !x_scales || !w_codes || !w_scales || !out || (result == SSD_MX_OUT_SWIGLU && !out_scales)) return fail_without_ctx(SSD_EINVAL, "%s: null pointer", who);
    const int rc = check_linear(who, M, N, K, result);
    if (rc != SSD_OK) return rc;
    if (off16(x_codes) || off16(x_scales) || off16(w_codes) || off16(w_scales) || off16(out) || off16(out_scales) || off16(workspace))
        return fail_without_ctx(SSD_EINVAL, "%s: a pointer off a 16-byte boundary", who);
    const size_t need = ssd_mx_linear_workspace(M, N, K, result);
    if (need && (!workspace || workspace_bytes < need)) return fail_without_ctx(SSD_ENOMEM, "%s: %zu bytes of workspace, %zu needed", who, workspace ? workspace_bytes : 0, need);
    MxArgs a;
    a.x = (const uint8_t*)x_codes; a.w = (const uint8_t*)w_codes;
    a.xs = (const uint32_t*)x_scales; a.ws = (const uint32_t*)w_scales;
    a.M = M; a.N = N; a.K = K; a.split = slices_of(N, K, result); a.st = (hipStream_t)hip_stream;
    a.out_s = (uint32_t*)out_scales;
    a.part_stride = (size_t)M * N;
    const int all = mx_choose_all(M, N, K, a.split);
    if (all >= 0) {
        a.out = out;
        return (result == SSD_MX_OUT_F32 ? mx_gemm_all_f32(a, all) : mx_gemm_all_bf16(a, all)) ? launched(who) : fail_without_ctx(SSD_EHIP, "%s: no kernel could be set up", who);
    }
    a.out = a.split > 1 ? workspace : out;
    int parts = 1;
    if (!mx_launch_gemm(a, a.split > 1 ? SSD_MX_OUT_F32 : result, &parts)) return fail_without_ctx(SSD_EHIP, "%s: no kernel could be set up", who);
    if (a.split > 1) mx_launch_join((const float*)workspace, parts, a.part_stride, result, out, (size_t)M * N, a.st);
    return launched(who);
}
