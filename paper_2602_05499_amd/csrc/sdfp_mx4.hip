// Entry points of the MXFP4 operators (include/sdfp.h): argument checks and launches.
#include "sdfp_mx4.hip.h"
#include "sdfp.h"

using namespace sdfp;

static_assert(SD_F32 == MX4_X_F32 && SD_BF16 == MX4_X_BF16 && SD_MX4 == MX4_X_MX4, "type codes");

namespace {
bool row_type(int t) { return t == SD_F32 || t == SD_BF16; }
bool size_ok(int rows, int cols) { return rows >= 1 && cols >= 1 && cols <= INT32_MAX - MX4_COLS; }
// panels of a matrix, as the grid of a launch: SD_EINVAL past what a launch can hold
bool grid_ok(int rows, int cols) { return (int64_t)mx4_row_panels(rows) * mx4_col_panels(cols) <= INT32_MAX; }
bool rows_ok(const void* x, int type, int64_t ld, int cols) {
    return x && row_type(type) && ld >= cols && ((uintptr_t)x & (type == SD_F32 ? 3 : 1)) == 0;
}
int status(hipError_t e) { return e == hipSuccess ? SD_OK : SD_EHIP; }
}  // namespace

namespace sdfp {

template <int XT>
static void launch_rows(const Mx4Product& a, dim3 grid, hipStream_t s) {
    if constexpr (XT == MX4_X_MX4) {
        hipLaunchKernelGGL((k_mx4_rows<XT, 1>), grid, dim3(mx4_rows_waves(XT, 1) * 64), 0, s, a);
    } else {
    if (a.M == 1) hipLaunchKernelGGL((k_mx4_rows<XT, 1>), grid, dim3(mx4_rows_waves(XT, 1) * 64), 0, s, a);
    else if (a.M <= 4) hipLaunchKernelGGL((k_mx4_rows<XT, 4>), grid, dim3(mx4_rows_waves(XT, 4) * 64), 0, s, a);
    else hipLaunchKernelGGL((k_mx4_rows<XT, 16>), grid, dim3(mx4_rows_waves(XT, 16) * 64), 0, s, a);
    }
}

hipError_t mx4_product(const Mx4Product& a, hipStream_t stream) {
    const int64_t n = (int64_t)mx4_row_panels(a.N) * ((a.M + 15) / 16);
    if (n > INT32_MAX) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)n);
    if (a.x_type == MX4_X_F32) launch_rows<MX4_X_F32>(a, grid, stream);
    else if (a.x_type == MX4_X_BF16) launch_rows<MX4_X_BF16>(a, grid, stream);
    else launch_rows<MX4_X_MX4>(a, grid, stream);
    return hipGetLastError();
}

hipError_t mx4_quantize(const void* x, int x_type, int64_t ldx, int rows, int cols, void* q, hipStream_t stream) {
    const dim3 grid((unsigned)(mx4_row_panels(rows) * mx4_col_panels(cols)));
    if (x_type == MX4_X_F32) hipLaunchKernelGGL(k_mx4_quantize<MX4_X_F32>, grid, dim3(256), 0, stream, x, ldx, rows, cols, (char*)q);
    else hipLaunchKernelGGL(k_mx4_quantize<MX4_X_BF16>, grid, dim3(256), 0, stream, x, ldx, rows, cols, (char*)q);
    return hipGetLastError();
}

}  // namespace sdfp

extern "C" {

size_t sd_mx4_bytes(int32_t rows, int32_t cols) { return size_ok(rows, cols) ? mx4_bytes(rows, cols) : 0; }

int sd_mx4_quantize(const void* x, int dtype, int64_t ld, int32_t rows, int32_t cols, void* q, size_t q_bytes, void* hip_stream) {
    if (!size_ok(rows, cols) || !grid_ok(rows, cols) || !rows_ok(x, dtype, ld, cols) || !q || ((uintptr_t)q & 255)) return SD_EINVAL;
    if (q_bytes < mx4_bytes(rows, cols)) return SD_ENOMEM;
    return status(mx4_quantize(x, dtype, ld, rows, cols, q, (hipStream_t)hip_stream));
}

int sd_mx4_dequantize(const void* q, size_t q_bytes, int32_t rows, int32_t cols, void* x, int dtype, int64_t ld, void* hip_stream) {
    if (!size_ok(rows, cols) || !grid_ok(rows, cols) || !rows_ok(x, dtype, ld, cols) || !q || ((uintptr_t)q & 255)) return SD_EINVAL;
    if (q_bytes < mx4_bytes(rows, cols)) return SD_ENOMEM;
    const dim3 grid((unsigned)(mx4_row_panels(rows) * mx4_col_panels(cols)));
    hipStream_t s = (hipStream_t)hip_stream;
    if (dtype == SD_F32) hipLaunchKernelGGL(k_mx4_dequantize<MX4_X_F32>, grid, dim3(256), 0, s, (const char*)q, rows, cols, x, ld);
    else hipLaunchKernelGGL(k_mx4_dequantize<MX4_X_BF16>, grid, dim3(256), 0, s, (const char*)q, rows, cols, x, ld);
    return status(hipGetLastError());
}

int sd_mx4_matmul(const void* w, size_t w_bytes, int32_t N, int32_t K, const void* x, int x_dtype, int64_t ldx, int32_t M,
                  const float* gain, float eps, void* y, int y_dtype, int64_t ldy, void* hip_stream) {
    if (!size_ok(N, K) || M < 1 || !grid_ok(N, K) || !w || ((uintptr_t)w & 255) || !rows_ok(y, y_dtype, ldy, N)) return SD_EINVAL;
    if (x_dtype == SD_MX4 ? !x || ((uintptr_t)x & 255) || ldx < 0 || !grid_ok(M, K) : !rows_ok(x, x_dtype, ldx, K)) return SD_EINVAL;
    if (gain && (x_dtype != SD_F32 || ((uintptr_t)gain & 3) || !(eps >= 0.f))) return SD_EINVAL;
    if (w_bytes < mx4_bytes(N, K) || (x_dtype == SD_MX4 && (size_t)ldx < mx4_bytes(M, K))) return SD_ENOMEM;
    if ((int64_t)mx4_row_panels(N) * (((int64_t)M + 15) / 16) > INT32_MAX) return SD_EINVAL;
    const Mx4Product a{(const char*)w, x, gain, y, ldx, ldy, M, N, K, x_dtype, y_dtype, eps};
    return status(mx4_product(a, (hipStream_t)hip_stream));
}

}  // extern "C"
