// Microscaled 4-bit matrices (MXFP4): the panel format and the host-side launches that the context's draft head shares with
// the entry points of include/sdfp.h.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace sdfp {

// A panel: 64 rows x 128 columns in 4352 bytes -- per 16-row tile t one kilobyte of codes, then 256 bytes of scales.  Lane
// l = 16 b + r of a wave finds the 16 bytes of row r, block b (32 columns) of tile t at t * 1024 + l * 16, and the scales of
// its four tiles' blocks in the word at 4096 + l * 4: what the matrix cores take as an operand is one contiguous kilobyte.
constexpr int MX4_ROWS = 64, MX4_COLS = 128, MX4_BLOCK = 32;
constexpr int MX4_TILE_BYTES = 1024, MX4_CODE_BYTES = 4096, MX4_PANEL_BYTES = 4352;

inline int mx4_row_panels(int rows) { return (int)(((int64_t)rows + MX4_ROWS - 1) / MX4_ROWS); }
inline int mx4_col_panels(int cols) { return (int)(((int64_t)cols + MX4_COLS - 1) / MX4_COLS); }
inline size_t mx4_bytes(int rows, int cols) {
    return (size_t)mx4_row_panels(rows) * (size_t)mx4_col_panels(cols) * MX4_PANEL_BYTES;
}

enum { MX4_X_F32 = 0, MX4_X_BF16 = 1, MX4_X_MX4 = 2 };   // the codes of SD_F32, SD_BF16, SD_MX4

struct Mx4Product {        // y[M][N] = x[M][K] w[N][K]^T
    const char* w;         // panels of [N][K]
    const void* x;         // rows of float32 or bfloat16 (ldx elements apart), or panels of [M][K]
    const float* gain;     // float32 x: RMS-normalise the rows and multiply by gain first; or nullptr
    void* y;               // rows of float32 or bfloat16, ldy elements apart
    int64_t ldx, ldy;
    int M, N, K, x_type, y_type;
    float eps;
};
hipError_t mx4_product(const Mx4Product& a, hipStream_t stream);
hipError_t mx4_quantize(const void* x, int x_type, int64_t ldx, int rows, int cols, void* q, hipStream_t stream);

}  // namespace sdfp
