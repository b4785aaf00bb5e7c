// Entry points of the MXFP4 operators (include/sdfp.h): argument checks and launches.
#include "sdfp_mx4.hip.h"
#include "sdfp.h"

#include <atomic>

using namespace sdfp;

static_assert(SD_F32 == MX4_X_F32 && SD_BF16 == MX4_X_BF16 && SD_MX4 == MX4_X_MX4, "type codes");

namespace {
bool row_type(int t) { return t == SD_F32 || t == SD_BF16; }
bool size_ok(int rows, int cols) { return rows >= 1 && cols >= 1 && rows <= INT32_MAX - 1024 && cols <= INT32_MAX - 1024; }   // (sizes are rounded up in int)
// workgroups of a launch, which holds 2^32 - 1 threads; a matrix's panels by 256 threads each
bool launch_ok(int64_t groups, int threads) { return groups <= UINT32_MAX / threads; }
bool grid_ok(int rows, int cols) { return launch_ok((int64_t)mx4_row_panels(rows) * mx4_col_panels(cols), 256); }
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
template <int XT, int MP, bool ONCE>
static void launch_rows(const Mx4Product& a, hipStream_t s) {
    const unsigned my = (unsigned)((a.M + 15) / 16), n_pan = (unsigned)mx4_row_panels(a.N);
    const dim3 blk(MX4_WAVES * 64);
    if (n_pan * my < 128) {
        hipLaunchKernelGGL((k_mx4_rows<XT, MP, 1, 1, ONCE>), dim3(n_pan * 4 * my), blk, 0, s, a);
        return;
    }
    if constexpr (XT == MX4_X_F32 && MP >= 8)
        if (n_pan * my >= 384) {
            hipLaunchKernelGGL((k_mx4_rows<XT, MP, 2, 4, ONCE>), dim3((n_pan + 1) / 2 * my), blk, 0, s, a);
            return;
        }
    hipLaunchKernelGGL((k_mx4_rows<XT, MP, 1, 4, ONCE>), dim3(n_pan * my), blk, 0, s, a);
}

// A kernel's dynamic LDS limit, raised once per device.
static hipError_t raise_lds(const void* kernel, int bytes, std::atomic<uint64_t>& done) {
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    const uint64_t bit = dev >= 0 && dev < 64 ? (uint64_t)1 << dev : 0;
    if (done.load(std::memory_order_relaxed) & bit) return hipSuccess;
    if ((e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes)) == hipSuccess) done.fetch_or(bit);
    return e;
}
template <int XT, int CT, int WN, int WM, int KW>
static hipError_t launch_tiles(const Mx4Product& a, hipStream_t s) {
    typedef Mx4Tile<XT, CT, WN, WM, KW> S;
    static std::atomic<uint64_t> done{0};
    const hipError_t e = raise_lds(reinterpret_cast<const void*>(k_mx4_tiles<XT, CT, WN, WM, KW>), S::LDS, done);
    if (e != hipSuccess) return e;
    const int64_t n = (int64_t)((mx4_row_panels(a.N) + WN - 1) / WN) * ((a.M + S::TM - 1) / S::TM);
    hipLaunchKernelGGL((k_mx4_tiles<XT, CT, WN, WM, KW>), dim3((unsigned)((n + 7) / 8 * 8)), dim3(S::THREADS), S::LDS, s, a);
    return hipGetLastError();
}
template <int CT, int WN, int WM>
static hipError_t launch_tiles_mx4(const Mx4Product& a, hipStream_t s) {
    typedef Mx4TileX<CT, WN, WM> S;
    static std::atomic<uint64_t> done{0};
    const hipError_t e = raise_lds(reinterpret_cast<const void*>(k_mx4_tiles_mx4<CT, WN, WM>), S::LDS, done);
    if (e != hipSuccess) return e;
    const int64_t n = (int64_t)((mx4_row_panels(a.N) + WN - 1) / WN) * ((mx4_row_panels(a.M) + S::XP - 1) / S::XP);
    hipLaunchKernelGGL((k_mx4_tiles_mx4<CT, WN, WM>), dim3((unsigned)((n + 7) / 8 * 8)), dim3(64 * S::WAVES), S::LDS, s, a);
    return hipGetLastError();
}

// Which kernel: the one for a few rows while its workgroups' 16-row by 64-output pieces (each reads the codes and cuts the rows
// up anew) make two rounds of the 256 compute units, or four in float32, whose tiles have three times the work; a small tile whose
// waves split the reduction while those make one round, a middle one for the next, the large tile from there on.
// Microseconds, K 4096 (few rows / small / middle / large):
//   bfloat16  128 x 4096 14/16/28/44, 64 x 11008 18/16/28/44, 512 x 4096 32/32/29/44, 256 x 11008 46/43/29/44, 512 x 11008 83/82/56/45,
//             4096 x 14336 866/757/421/351 (1.37 PFLOP/s; the library's bfloat16 product of that size 396)
//   float32   128 x 4096 23/46/49/121, 512 x 4096 70/52/54/121, 256 x 11008 95/90/78/120, 2048 x 4096 249/181/162/134,
//             4096 x 14336 1786/1256/1111/935 (three products: 1.54 PFLOP/s)
//   MXFP4     128 x 4096 13/14/-/23, 64 x 11008 16/14/-/22, 256 x 11008 32/19/-/24, 2048 x 4096 66/28/-/27, 4096 x 14336 522/196/-/150 (3.2
//             PFLOP/s)
// K does not enter: over 14 sizes from 16 x 4096 to 4096 x 14336 the choice is within 7 % of the best at K 512, 4096 and 14336, but for
// float32 (K 512: 64 x 11008 12.7 against 10.7 by the middle tile, 512 x 4096 13.0 against 11.8; K 14336: 256 x 4096 118 against 108 by
// few rows, 512 x 4096 176 against 161 by the small tile, 1024 x 4096 307 against 286 by the middle one) and for 2048 x 4096 x 512 in
// MXFP4 (12.0 against 11.1 by the small tile).
hipError_t mx4_product(const Mx4Product& a, hipStream_t stream) {
    const int64_t n_pan = mx4_row_panels(a.N), pieces = n_pan * (((int64_t)a.M + 15) / 16);
    auto tiles = [&](int n, int m) { return (((int64_t)a.N + n - 1) / n) * (((int64_t)a.M + m - 1) / m); };
    if (a.x_type == MX4_X_F32) {
        if (a.M > 16 && pieces > 1024) {
            if (tiles(256, 32) <= 256) return launch_tiles<MX4_X_F32, 2, 4, 1, 2>(a, stream);
            if (tiles(256, 32) <= 512) return launch_tiles<MX4_X_F32, 2, 4, 1, 1>(a, stream);
            return launch_tiles<MX4_X_F32, 4, 8, 1, 1>(a, stream);
        }
        if (a.M == 1) launch_rows<MX4_X_F32, 1, true>(a, stream);
        else if (a.M <= 5) launch_rows<MX4_X_F32, 5, true>(a, stream);
        else if (a.M <= 8) launch_rows<MX4_X_F32, 8, true>(a, stream);
        else if (a.M <= 16) launch_rows<MX4_X_F32, 16, true>(a, stream);
        else launch_rows<MX4_X_F32, 16, false>(a, stream);
    } else if (a.x_type == MX4_X_BF16) {
        if (a.M > 16 && pieces > 512) {
            if (tiles(128, 32) <= 256) return launch_tiles<MX4_X_BF16, 2, 2, 1, 4>(a, stream);
            if (tiles(256, 64) <= 256) return launch_tiles<MX4_X_BF16, 4, 4, 1, 2>(a, stream);
            return launch_tiles<MX4_X_BF16, 4, 8, 1, 1>(a, stream);
        }
        if (a.M == 1) launch_rows<MX4_X_BF16, 1, true>(a, stream);
        else if (a.M <= 4) launch_rows<MX4_X_BF16, 4, true>(a, stream);
        else if (a.M <= 8) launch_rows<MX4_X_BF16, 8, true>(a, stream);
        else if (a.M <= 16) launch_rows<MX4_X_BF16, 16, true>(a, stream);
        else launch_rows<MX4_X_BF16, 16, false>(a, stream);
    } else {
        if (a.M > 16 && pieces > 512) {
            if (tiles(256, 128) < 256) return launch_tiles_mx4<4, 2, 1>(a, stream);
            return launch_tiles_mx4<8, 4, 1>(a, stream);
        }
        if (a.M <= 16) launch_rows<MX4_X_MX4, 16, true>(a, stream);
        else launch_rows<MX4_X_MX4, 16, false>(a, stream);
    }
    return hipGetLastError();
}

template <int XT>
static void launch_quantize(const void* x, int64_t ldx, int rows, int cols, void* q, hipStream_t s) {
    const dim3 grid((unsigned)(mx4_row_panels(rows) * mx4_col_panels(cols)));
    const bool once = (int64_t)rows * cols * (int64_t)sizeof(typename Mx4In<XT>::T) >= (int64_t)64 << 20;
    if (once) hipLaunchKernelGGL((k_mx4_quantize<XT, true>), grid, dim3(256), 0, s, x, ldx, rows, cols, (char*)q);
    else hipLaunchKernelGGL((k_mx4_quantize<XT, false>), grid, dim3(256), 0, s, x, ldx, rows, cols, (char*)q);
}
hipError_t mx4_quantize(const void* x, int x_type, int64_t ldx, int rows, int cols, void* q, hipStream_t stream) {
    if (x_type == MX4_X_F32) launch_quantize<MX4_X_F32>(x, ldx, rows, cols, q, stream);
    else launch_quantize<MX4_X_BF16>(x, ldx, rows, cols, q, stream);
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
    if (!size_ok(N, K) || !size_ok(M, K) || !grid_ok(N, K) || !w || ((uintptr_t)w & 255) || !rows_ok(y, y_dtype, ldy, N)) return SD_EINVAL;
    if (x_dtype == SD_MX4 ? !x || ((uintptr_t)x & 255) || ldx < 0 || !grid_ok(M, K) : !rows_ok(x, x_dtype, ldx, K)) return SD_EINVAL;
    if (gain && (x_dtype != SD_F32 || ((uintptr_t)gain & 3) || !(eps >= 0.f))) return SD_EINVAL;
    if (w_bytes < mx4_bytes(N, K) || (x_dtype == SD_MX4 && (size_t)ldx < mx4_bytes(M, K))) return SD_ENOMEM;
    if (!launch_ok(M <= 16 ? mx4_row_panels(N) : (((int64_t)N + 255) / 256) * (((int64_t)M + 63) / 64), 512)) return SD_EINVAL;
    const Mx4Product a{(const char*)w, x, gain, y, ldx, ldy, M, N, K, x_dtype, y_dtype, eps};
    return status(mx4_product(a, (hipStream_t)hip_stream));
}

}  // extern "C"
