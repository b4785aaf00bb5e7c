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

// One launch of the kernel for a few rows.  A workgroup takes a panel of 64 outputs; one 16-row tile of it where that makes
// too few workgroups (one row, 4096 outputs: 5.8 us against 6.9; 8192, 128 panels: equal; 11008: 9.3 against 8.0); two panels
// where there are plenty and a row's cutting into pieces weighs (float32, 9 rows, 32000 outputs: 21.0 us against 25.8; for
// one row two panels are slower, 16.4 against 15.3).
template <int XT, int MP>
static void launch_rows(const Mx4Product& a, hipStream_t s) {
    const unsigned my = (unsigned)((a.M + 15) / 16), n_pan = (unsigned)mx4_row_panels(a.N);
    const dim3 blk(MX4_WAVES * 64);
    if (n_pan * my < 128) {
        hipLaunchKernelGGL((k_mx4_rows<XT, MP, 1, 1>), dim3(n_pan * 4 * my), blk, 0, s, a);
        return;
    }
    if constexpr (XT == MX4_X_F32 && MP >= 8)
        if (n_pan * my >= 384) {
            hipLaunchKernelGGL((k_mx4_rows<XT, MP, 2, 4>), dim3((n_pan + 1) / 2 * my), blk, 0, s, a);
            return;
        }
    hipLaunchKernelGGL((k_mx4_rows<XT, MP, 1, 4>), dim3(n_pan * my), blk, 0, s, a);
}

hipError_t mx4_product(const Mx4Product& a, hipStream_t stream) {
    if ((int64_t)mx4_row_panels(a.N) * (((int64_t)a.M + 15) / 16) > INT32_MAX) return hipErrorInvalidConfiguration;
    if (a.x_type == MX4_X_F32) {
        if (a.M == 1) launch_rows<MX4_X_F32, 1>(a, stream);
        else if (a.M <= 5) launch_rows<MX4_X_F32, 5>(a, stream);
        else if (a.M <= 8) launch_rows<MX4_X_F32, 8>(a, stream);
        else launch_rows<MX4_X_F32, 16>(a, stream);
    } else if (a.x_type == MX4_X_BF16) {
        if (a.M == 1) launch_rows<MX4_X_BF16, 1>(a, stream);
        else if (a.M <= 4) launch_rows<MX4_X_BF16, 4>(a, stream);
        else if (a.M <= 8) launch_rows<MX4_X_BF16, 8>(a, stream);
        else launch_rows<MX4_X_BF16, 16>(a, stream);
    } else {
        launch_rows<MX4_X_MX4, 16>(a, stream);
    }
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
