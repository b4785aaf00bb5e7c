// MXFP4 kernels: quantisation to panels, reading back, and the product of rows with a matrix in panels.
#pragma once
#include "sdfp_common.hip.h"
#include "sdfp_mx4.h"

#include <type_traits>

namespace sdfp {

typedef u32x4 __attribute__((aligned(2))) u32x4_any;   // 16 bytes at any element's address
typedef u32x2 __attribute__((aligned(2))) u32x2_any;
typedef int i32x8 __attribute__((ext_vector_type(8)));

template <int XT> struct Mx4In;     // storage of unquantised rows; VE elements fill 16 bytes
template <> struct Mx4In<MX4_X_F32> {
    typedef float T;
    static constexpr int VE = 4;
    static __device__ __forceinline__ float val(float v) { return v; }
    static __device__ __forceinline__ void unpack(const u32x4& r, float (&v)[4]) {
        v[0] = __uint_as_float(r.x); v[1] = __uint_as_float(r.y); v[2] = __uint_as_float(r.z); v[3] = __uint_as_float(r.w);
    }
    static __device__ __forceinline__ u32x4 pack(const float (&v)[4]) {
        return u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    }
    static __device__ __forceinline__ float out(float v) { return v; }
};
template <> struct Mx4In<MX4_X_BF16> {
    typedef bf16_t T;
    static constexpr int VE = 8;
    static __device__ __forceinline__ float val(bf16_t v) { return bf16_to_f32(v); }
    static __device__ __forceinline__ void unpack(const u32x4& r, float (&v)[8]) { ST<bf16_t>::unpack(r, v); }
    static __device__ __forceinline__ u32x4 pack(const float (&v)[8]) {
        return u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
    }
    static __device__ __forceinline__ bf16_t out(float v) { return (bf16_t)pack_bf16(v, v); }
};

// VE elements of a row from column k on, zeros past its end; full: all of them exist.  ONCE: the caller reads them once and for
// all (the caches need not keep them)
template <int XT, bool ONCE = false>
__device__ __forceinline__ u32x4 mx4_load(const typename Mx4In<XT>::T* row, int64_t k, int cols, bool full) {
    const SDFP_GLOBAL u32x4_any* p = reinterpret_cast<const SDFP_GLOBAL u32x4_any*>(as_global(row + k));
    if (full) return ONCE ? __builtin_nontemporal_load(p) : *p;
    u32x4 r{0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < Mx4In<XT>::VE; ++i)
        if (k + i < cols) {
            if (XT == MX4_X_F32) r[i] = reinterpret_cast<const unsigned*>(row)[k + i];
            else r[i / 2] |= (unsigned)reinterpret_cast<const bf16_t*>(row)[k + i] << (16 * (i % 2));
        }
    return r;
}

// ---- quantisation.  A block of 32 columns shares the scale s = 2^(floor(log2 max|x|) - 2), at least 2^-126, so that the
// largest magnitude lands in [4, 8) of the grid {0, .5, 1, 1.5, 2, 3, 4, 6}; values are rounded to nearest, ties to the even
// code, and saturate at 6.  |x| / s is exact (a power of two; what underflows rounds to zero either way).  A block with an
// infinity or a NaN gets the scale 255, NaN throughout.  One workgroup per panel: a block is held by 32 / VE neighbouring
// lanes, which exchange the maximum of their bit patterns (as integers: NaN above infinity above all finite magnitudes); the
// panel is put together in LDS and leaves as 4352 contiguous bytes.  Bound by the read of the rows: 32000 x 4096 in bfloat16 55 us, 6.0
// TB/s.  ONCE: rows beyond what the caches hold pass them by (55 against 62 us there; 16 million values the other way round, 9.7
// against 9.2).
template <int XT, bool ONCE>
__global__ __launch_bounds__(256) void k_mx4_quantize(const void* __restrict__ x_, int64_t ld, int rows, int cols, char* __restrict__ q) {
    typedef typename Mx4In<XT>::T T;
    constexpr int VE = Mx4In<XT>::VE, PER_ROW = MX4_COLS / VE, PER_BLOCK = MX4_BLOCK / VE, RP = 256 / PER_ROW, NP = MX4_ROWS / RP;
    __shared__ __attribute__((aligned(16))) char sh[MX4_PANEL_BYTES];
    const int kps = (cols + MX4_COLS - 1) / MX4_COLS, kp = blockIdx.x % kps, tid = threadIdx.x, lc = tid % PER_ROW;
    const int64_t row0 = (int64_t)(blockIdx.x / kps) * MX4_ROWS;
    const int k = kp * MX4_COLS + lc * VE;
    const bool full = kp * (int64_t)MX4_COLS + MX4_COLS <= cols;
    const T* x = reinterpret_cast<const T*>(x_);
    u32x4 raw[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int64_t row = row0 + i * RP + tid / PER_ROW;
        raw[i] = row < rows ? mx4_load<XT, ONCE>(x + row * ld, k, cols, full) : u32x4{0u, 0u, 0u, 0u};
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int r = i * RP + tid / PER_ROW, t = r / 16, b = lc / PER_BLOCK;
        float v[VE];
        Mx4In<XT>::unpack(raw[i], v);
        unsigned amax = 0;
#pragma unroll
        for (int e = 0; e < VE; ++e) amax = max(amax, __float_as_uint(v[e]) & 0x7FFFFFFFu);
#pragma unroll
        for (int o = 1; o < PER_BLOCK; o <<= 1) amax = max(amax, (unsigned)__shfl_xor((int)amax, o));
        const int ex = (int)(amax >> 23);                        // biased exponent of the largest magnitude
        const int sc = ex == 255 ? 255 : max(ex - 2, 1);
        const float inv = ex == 255 ? 0.f : __uint_as_float((unsigned)(254 - sc) << 23);   // 1 / s
        unsigned w = 0;
#pragma unroll
        for (int e = 0; e < VE; e += 2) {
            const float a = ex == 255 ? 0.f : v[e] * inv, c = ex == 255 ? 0.f : v[e + 1] * inv;
            if (e == 0) w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, a, c, 1.0f, 0);
            if (e == 2) w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, a, c, 1.0f, 1);
            if (e == 4) w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, a, c, 1.0f, 2);
            if (e == 6) w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, a, c, 1.0f, 3);
        }
        char* code = sh + ((t * 4 + b) * 16 + r % 16) * 16 + (lc % PER_BLOCK) * (VE / 2);
        if (VE == 8) *reinterpret_cast<unsigned*>(code) = w;
        else *reinterpret_cast<unsigned short*>(code) = (unsigned short)w;
        if (lc % PER_BLOCK == 0) sh[MX4_CODE_BYTES + (b * 16 + r % 16) * 4 + t] = (char)sc;
    }
    __syncthreads();
    char* dst = q + (size_t)blockIdx.x * MX4_PANEL_BYTES;
    for (int o = tid * 16; o < MX4_PANEL_BYTES; o += 256 * 16)
        *reinterpret_cast<u32x4*>(dst + o) = *reinterpret_cast<const u32x4*>(sh + o);
}

// the scale 2^(e - 127) of a scale byte as a float32; 0 stands for 2^-127, 255 for NaN
__device__ __forceinline__ float mx4_scale(unsigned e) {
    return e == 255u ? __uint_as_float(0x7FC00000u) : e == 0u ? __uint_as_float(0x00400000u) : __uint_as_float(e << 23);
}

// ---- reading back: the values that panels stand for, as float32 or bfloat16 rows, written past the caches (50 against 63 us for
// 32000 x 4096 in bfloat16: 6.6 TB/s).  One workgroup per panel.
template <int XT>
__global__ __launch_bounds__(256) void k_mx4_dequantize(const char* __restrict__ q, int rows, int cols, void* __restrict__ x_, int64_t ld) {
    typedef typename Mx4In<XT>::T T;
    constexpr int VE = Mx4In<XT>::VE, PER_ROW = MX4_COLS / VE, PER_BLOCK = MX4_BLOCK / VE, RP = 256 / PER_ROW, NP = MX4_ROWS / RP;
    __shared__ __attribute__((aligned(16))) char sh[MX4_PANEL_BYTES];
    const int kps = (cols + MX4_COLS - 1) / MX4_COLS, kp = blockIdx.x % kps, tid = threadIdx.x, lc = tid % PER_ROW;
    const int64_t row0 = (int64_t)(blockIdx.x / kps) * MX4_ROWS;
    const int k = kp * MX4_COLS + lc * VE, b = lc / PER_BLOCK;
    const bool full = kp * (int64_t)MX4_COLS + MX4_COLS <= cols;
    const char* src = q + (size_t)blockIdx.x * MX4_PANEL_BYTES;
    for (int o = tid * 16; o < MX4_PANEL_BYTES; o += 256 * 16)
        *reinterpret_cast<u32x4*>(sh + o) = *reinterpret_cast<const u32x4*>(src + o);
    __syncthreads();
    T* x = reinterpret_cast<T*>(x_);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int r = i * RP + tid / PER_ROW, t = r / 16;
        const int64_t row = row0 + r;
        if (row >= rows) continue;
        const char* code = sh + ((t * 4 + b) * 16 + r % 16) * 16 + (lc % PER_BLOCK) * (VE / 2);
        const unsigned w = VE == 8 ? *reinterpret_cast<const unsigned*>(code) : *reinterpret_cast<const unsigned short*>(code);
        const float s = mx4_scale((unsigned char)sh[MX4_CODE_BYTES + (b * 16 + r % 16) * 4 + t]);
        float v[VE];
#pragma unroll
        for (int e = 0; e < VE; e += 2) {
            f32x2_t f = {0.f, 0.f};
            if (e == 0) f = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0);
            if (e == 2) f = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1);
            if (e == 4) f = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2);
            if (e == 6) f = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3);
            v[e] = f.x * s; v[e + 1] = f.y * s;
        }
        T* to = x + row * ld + k;
        if (full) {
            __builtin_nontemporal_store(Mx4In<XT>::pack(v), reinterpret_cast<u32x4_any*>(to));
        } else {
#pragma unroll
            for (int e = 0; e < VE; ++e)
                if (k + e < cols) to[e] = Mx4In<XT>::out(v[e]);
        }
    }
}

// Float32 values as three bfloat16 pieces by truncation, x = x0 + x1 + x2 exactly (8 bits of the significand each; what is
// below the smallest bfloat16 is lost): pk[p][i] holds piece p of values 2 i and 2 i + 1.  Truncation keeps the first piece of
// a large finite value finite; an infinity is its first piece alone, a NaN stays one.
template <int N>
__device__ __forceinline__ void trunc3(const float (&x)[N], unsigned (&pk)[3][N / 2]) {
    auto hi = [](float v) { return __uint_as_float(__float_as_uint(v) & 0xFFFF0000u); };
    auto pair = [](float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u); };   // upper halves
    bool odd = false;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        const float a = x[2 * i], b = x[2 * i + 1];
        const float ra = sub_rn(a, hi(a)), rb = sub_rn(b, hi(b));
        odd |= __builtin_isunordered(ra, rb);      // an infinity or a NaN left a NaN
        pk[0][i] = pair(a, b);
        pk[1][i] = pair(ra, rb);
        pk[2][i] = pair(sub_rn(ra, hi(ra)), sub_rn(rb, hi(rb)));
    }
    if (odd)
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const unsigned half = e % 2 ? 0xFFFF0000u : 0x0000FFFFu;
            if ((__float_as_uint(x[e]) & 0x7F800000u) != 0x7F800000u) continue;
            if (x[e] != x[e]) pk[0][e / 2] = (pk[0][e / 2] & ~half) | (0x7FC07FC0u & half);
            pk[1][e / 2] &= ~half; pk[2][e / 2] &= ~half;
        }
}

// 8 values of a block -- the codes of one word -- as a bfloat16 matrix-core operand, scale applied (exact)
__device__ __forceinline__ bf16x8 mx4_decode(unsigned w, float s) {
    const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1),
                   c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3);
    return bf16x8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}
__device__ __forceinline__ f32x4 mx4_mfma(const u32x4& a, int sa, const u32x4& b, int sb, const f32x4& c) {
    const i32x8 A = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0}, B = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(A, B, c, 4, 4, 0, sa, 0, sb);
}
// the high bit of every byte of s that is 255
__device__ __forceinline__ unsigned mx4_nan_bytes(unsigned s) { return ((s & 0x7F7F7F7Fu) + 0x01010101u) & s & 0x80808080u; }

// The same for bytes from 253 on, whose larger values pass float32.  Where float32 x has its three pieces in one sum, an infinity among
// w's values multiplies all three and makes NaN of the pieces that are zero; outputs whose row of w has such a byte (or a 255) are
// therefore added up again, one thread each.
__device__ __forceinline__ unsigned mx4_far_bytes(unsigned s) { return ((s & 0x7F7F7F7Fu) + 0x03030303u) & s & 0x80808080u; }
// Output (m, n): NaN with a block of NaN, y if w's values are all finite, else the sum of the terms that are not finite.  rs: the row's
// factor.
__device__ __forceinline__ float mx4_far_output(const Mx4Product& a, int64_t m, int64_t n, float rs, float y) {
    const int kps = (a.K + MX4_COLS - 1) / MX4_COLS, t = (int)(n % MX4_ROWS) / 16, r = (int)(n % 16);
    const char* w = a.w + (size_t)(n / MX4_ROWS) * kps * MX4_PANEL_BYTES;
    auto block = [&](int k) { return k % MX4_COLS / MX4_BLOCK * 16 + r; };
    auto scale = [&](int k) { return (int)(unsigned char)w[(size_t)(k / MX4_COLS) * MX4_PANEL_BYTES + MX4_CODE_BYTES + block(k) * 4 + t]; };
#pragma unroll 1
    for (int k = 0; k < a.K; k += MX4_BLOCK)
        if (scale(k) == 255) return __uint_as_float(0x7FC00000u);
    const float* x = (const float*)a.x + m * a.ldx;
    bool inf = false;
    float sum = 0.f;
#pragma unroll 1
    for (int k = 0; k < a.K; ++k) {
        const int e = scale(k);
        const int code = (unsigned char)w[(size_t)(k / MX4_COLS) * MX4_PANEL_BYTES + t * MX4_TILE_BYTES + block(k) * 16 + k % MX4_BLOCK / 2] >> (4 * (k % 2)) & 15;
        const bool far = (code & 7) >= (e == 254 ? 4 : e == 253 ? 6 : 8);          // 2 * 2^127, 4 * 2^126
        const float v = a.gain ? x[k] * a.gain[k] : x[k], c = far ? INFINITY : code & 7 ? 1.f : 0.f;
        if (far || !__builtin_isfinite(v)) sum += v * (code & 8 ? -c : c);
        inf |= far;
    }
    return inf ? sum * rs : y;
}

// A lane's word of scales in the last panel.  Blocks past column K hold zero codes, but any scale byte: theirs become 0, so that a 255
// there counts for nothing.
__device__ __forceinline__ unsigned mx4_last_scales(unsigned s, int lane, int kps, int K) {
    return (kps - 1) * MX4_COLS + lane / 16 * MX4_BLOCK < K ? s : 0u;
}

// four neighbouring outputs n .. n + 3 of row m (those that exist)
__device__ __forceinline__ void mx4_store(const Mx4Product& a, int64_t m, int64_t n, const float (&v)[4]) {
    const bool whole = n + 4 <= a.N;
    if (a.y_type == MX4_X_F32) {
        float* y = (float*)a.y + m * a.ldy + n;
        if (whole) *reinterpret_cast<u32x4_any*>(y) = Mx4In<MX4_X_F32>::pack(v);
        else for (int i = 0; n + i < a.N; ++i) y[i] = v[i];
    } else {
        bf16_t* y = (bf16_t*)a.y + m * a.ldy + n;
        if (whole) *reinterpret_cast<u32x2_any*>(y) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
        else for (int i = 0; n + i < a.N; ++i) y[i] = (bf16_t)pack_bf16(v[i], v[i]);
    }
}

// What a wave of the kernels for many rows has computed for 16 rows of x, m0 .. m0 + 15, and 64 outputs, n0 .. n0 + 63: lane 16 g + r
// holds in v[t] the outputs 16 t + 4 g .. of row r.  It goes through 4352 bytes of LDS of the wave's own, so that each store
// writes whole lines of 128 bytes (x in MXFP4, 4096 rows x 14336 x 4096, float32 result: 153 us, from the lanes as they are 158;
// past the caches 153).
constexpr int MX4_OUT_BYTES = 16 * 68 * 4;
__device__ __forceinline__ void mx4_store_tile(const Mx4Product& a, char* lds, int64_t m0, int64_t n0, const f32x4 (&v)[4]) {
    const int lane = threadIdx.x & 63;
    float* sh = reinterpret_cast<float*>(lds);
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int t = 0; t < 4; ++t) *reinterpret_cast<f32x4*>(sh + (lane & 15) * 68 + t * 16 + (lane >> 4) * 4) = v[t];
    __builtin_amdgcn_wave_barrier();
    if (a.y_type == MX4_X_F32) {
        const int64_t n = n0 + lane % 16 * 4;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = i * 4 + lane / 16;
            const u32x4 o = *reinterpret_cast<const u32x4*>(sh + r * 68 + lane % 16 * 4);
            float* y = (float*)a.y + (m0 + r) * a.ldy + n;
            if (m0 + r >= a.M || n >= a.N) continue;
            if (n + 4 > a.N)
                for (int e = 0; n + e < a.N; ++e) y[e] = __uint_as_float(o[e]);
            else *reinterpret_cast<u32x4_any*>(y) = o;
        }
    } else {
        const int64_t n = n0 + lane % 8 * 8;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = i * 8 + lane / 8;
            const f32x4 p = *reinterpret_cast<const f32x4*>(sh + r * 68 + lane % 8 * 8), q = *reinterpret_cast<const f32x4*>(sh + r * 68 + lane % 8 * 8 + 4);
            const u32x4 o{pack_bf16(p.x, p.y), pack_bf16(p.z, p.w), pack_bf16(q.x, q.y), pack_bf16(q.z, q.w)};
            bf16_t* y = (bf16_t*)a.y + (m0 + r) * a.ldy + n;
            if (m0 + r >= a.M || n >= a.N) continue;
            if (n + 8 > a.N)
                for (int e = 0; n + e < a.N; ++e) y[e] = (bf16_t)(o[e / 2] >> (16 * (e % 2)));
            else *reinterpret_cast<u32x4_any*>(y) = o;
        }
    }
}

// ---- product of a few rows: bound by the read of the panels (one row of a 32000 x 4096 head that lies in no cache 15.3 us, 4.6 TB/s
// with the launch's ends; 128256 x 4096 46.5 us, 6.0 TB/s; x in MXFP4 5 rows 43.3 us, 6.5 TB/s).  A workgroup computes NPAN panels of outputs, or TT of the four 16-row tiles of one,
// for 16 rows of x; its waves split the reduction dimension by panels and add their sums in wave order at the end.  The codes
// go from memory straight into the A operand (lane l: weight row l % 16, the block l / 16 of 32 columns; sub-step j multiplies
// the 8 values of word j), one panel ahead (x in MXFP4: two), x through a few kilobytes of LDS
// that belong to the wave into the B operand, in the same order of columns.  x in MXFP4 goes as it is into the scaled 4-bit
// instruction; float32 x is cut into three exact bfloat16 pieces, which take three of the operand's 16 columns for each row
// while rows are few (MP <= 5: one instruction where three would run, 17.7 -> 15.5 us) and three instructions otherwise.  MP:
// rows of x that are staged; lanes of the operand past them read values whose results are dropped.  ONCE: one pass over the codes,
// which then pass the caches by (codes not in any cache: 21.0 -> 19.3 us for 32000 x 5120).
constexpr bool mx4_rows_in_columns(int xt, int mp) { return xt == MX4_X_F32 && mp <= 5; }
constexpr int MX4_WAVES = 8;
template <int XT, int MP, int NPAN, int TT, bool ONCE>
__global__ __launch_bounds__(MX4_WAVES * 64) void k_mx4_rows(Mx4Product a) {
    constexpr int W = MX4_WAVES;
    constexpr bool COLS = mx4_rows_in_columns(XT, MP);
    constexpr int NPC = XT == MX4_X_F32 ? 3 : 1;                             // pieces of a value
    constexpr int NI = COLS ? 1 : NPC;                                       // instructions per sub-step and tile
    constexpr bool FAR = XT == MX4_X_F32 && !COLS;                           // s_bad_n: outputs to be added up again (else: NaN)
    // the staged panel of x, one piece after the other (or with the pieces as columns): 16 entries -- sub-step j, block b -- of
    // 16 bytes per column, a multiple of 16 bytes apart that is no power of two, so that the lanes of a row write to different
    // banks
    constexpr int COLUMNS = COLS ? 3 * MP : MP;
    constexpr int ENTRY = (COLUMNS % 2 ? COLUMNS : COLUMNS + 1) * 16;
    constexpr int STAGE = XT == MX4_X_MX4 ? 0 : 16 * ENTRY;                 // bytes, each wave's own
    constexpr int RED = W * TT * 64 * 16;
    __shared__ __attribute__((aligned(16))) char sh[W * STAGE > RED ? W * STAGE : RED];
    __shared__ float s_sq[W][16];
    __shared__ unsigned s_bad_n[NPAN * MX4_ROWS], s_bad_m[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c16 = lane & 15, g = lane >> 4;
    const int kps = (a.K + MX4_COLS - 1) / MX4_COLS, n_pan = (a.N + MX4_ROWS - 1) / MX4_ROWS;
    const int my = (a.M + 15) / 16, unit = blockIdx.x / my;
    const int panel0 = NPAN > 1 ? unit * NPAN : unit / (4 / TT), t0 = NPAN > 1 ? 0 : unit % (4 / TT) * TT;
    const int64_t m0 = (int64_t)(blockIdx.x % my) * 16;

    const char* wp[NPAN];                                                    // (panels past the end repeat the last one)
    f32x4 acc[NPAN][TT];
    unsigned bad[NPAN], bad_x = 0;
#pragma unroll
    for (int q = 0; q < NPAN; ++q) {
        wp[q] = a.w + (size_t)min(panel0 + q, n_pan - 1) * kps * MX4_PANEL_BYTES;
        bad[q] = 0;
#pragma unroll
        for (int t = 0; t < TT; ++t) acc[q][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    constexpr int VE = XT == MX4_X_F32 ? 4 : 8;
    constexpr int PER_ROW = MX4_COLS / VE;                                   // lanes per row of a staged panel
    constexpr int NL = XT == MX4_X_MX4 ? 1 : (MP * PER_ROW + 63) / 64;       // loads per lane
    float sq[NL];
#pragma unroll
    for (int i = 0; i < NL; ++i) sq[i] = 0.f;
    char* stage = sh + wave * STAGE;
    const float* gain = a.gain ? a.gain : (const float*)a.x;                 // (without a gain: loaded, not used)
    const int col = COLS ? min(c16, COLUMNS - 1) : c16 & (MP - 1);

    struct Load { u32x4 code[NPAN][TT]; unsigned scale[NPAN]; u32x4 x[NL]; u32x4 gain; };
    auto fetch = [&](int kp, Load& L, bool tail) {
#pragma unroll
        for (int q = 0; q < NPAN; ++q) {
            const char* p = wp[q] + (size_t)kp * MX4_PANEL_BYTES;
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                const SDFP_GLOBAL u32x4* c = reinterpret_cast<const SDFP_GLOBAL u32x4*>(as_global(p + (t0 + t) * MX4_TILE_BYTES + lane * 16));
                L.code[q][t] = ONCE ? __builtin_nontemporal_load(c) : *c;
            }
            L.scale[q] = *reinterpret_cast<const SDFP_GLOBAL unsigned*>(as_global(p + MX4_CODE_BYTES + lane * 4)) >> (8 * t0);
        }
        if constexpr (XT == MX4_X_MX4) {
            const char* xp = (const char*)a.x + ((size_t)(m0 / MX4_ROWS) * kps + kp) * MX4_PANEL_BYTES;
            const int t = (int)(m0 / 16) & 3;
            L.x[0] = *reinterpret_cast<const SDFP_GLOBAL u32x4*>(as_global(xp + t * MX4_TILE_BYTES + lane * 16));
            L.gain.x = *reinterpret_cast<const SDFP_GLOBAL unsigned*>(as_global(xp + MX4_CODE_BYTES + lane * 4)) >> (8 * t) & 255u;
        } else {
            typedef typename Mx4In<XT>::T T;
            const int k = kp * MX4_COLS + (lane % PER_ROW) * VE;
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                const int64_t row = min(m0 + min((i * 64 + lane) / PER_ROW, MP - 1), (int64_t)a.M - 1);
                L.x[i] = mx4_load<XT>((const T*)a.x + row * a.ldx, k, a.K, !tail);
            }
            if constexpr (XT == MX4_X_F32) L.gain = mx4_load<XT>(gain, k, a.K, !tail);
        }
    };
    auto multiply = [&](const Load& L) {
        if constexpr (XT == MX4_X_MX4) {
            bad_x |= L.gain.x == 255u;
#pragma unroll
            for (int q = 0; q < NPAN; ++q) {
                bad[q] |= mx4_nan_bytes(L.scale[q]);
#pragma unroll
                for (int t = 0; t < TT; ++t) acc[q][t] = mx4_mfma(L.code[q][t], (int)(L.scale[q] >> (8 * t)), L.x[0], (int)L.gain.x, acc[q][t]);
            }
        } else {
            bf16x8 xb[4][NI];
            auto at = [&](int i) { const int cc = (lane % PER_ROW) * VE; return stage + (cc % 32 / 8 * 4 + cc / 32) * ENTRY + (i * 64 + lane) / PER_ROW * 16; };
            auto staged = [&](int i) { return MP * PER_ROW % 64 == 0 || (i * 64 + lane) / PER_ROW < MP; };
            auto take = [&](int p) {
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int j = 0; j < 4; ++j) xb[j][p] = *reinterpret_cast<const bf16x8*>(stage + (j * 4 + g) * ENTRY + col * 16);
                __builtin_amdgcn_wave_barrier();
            };
            if constexpr (XT == MX4_X_F32) {
                unsigned pk[NL][3][2];
#pragma unroll
                for (int i = 0; i < NL; ++i) {
                    float v[4], gn[4];
                    Mx4In<XT>::unpack(L.x[i], v);
                    if (a.gain) {
                        Mx4In<XT>::unpack(L.gain, gn);
#pragma unroll
                        for (int e = 0; e < 4; ++e) { sq[i] = fmaf(v[e], v[e], sq[i]); v[e] *= gn[e]; }
                    }
                    trunc3(v, pk[i]);
                }
#pragma unroll
                for (int p = 0; p < 3; ++p) {
#pragma unroll
                    for (int i = 0; i < NL; ++i)
                        if (staged(i)) *reinterpret_cast<u32x2*>(at(i) + (COLS ? p * MP * 16 : 0) + lane % 2 * 8) = u32x2{pk[i][p][0], pk[i][p][1]};
                    if (!COLS) take(p);
                }
                if (COLS) take(0);
            } else {
#pragma unroll
                for (int i = 0; i < NL; ++i)
                    if (staged(i)) *reinterpret_cast<u32x4*>(at(i)) = L.x[i];
                take(0);
            }
#pragma unroll
            for (int q = 0; q < NPAN; ++q) {
                bad[q] |= FAR ? mx4_far_bytes(L.scale[q]) : mx4_nan_bytes(L.scale[q]);
#pragma unroll
                for (int t = 0; t < TT; ++t) {
                    const unsigned e = L.scale[q] >> (8 * t) & 255u;
                    const float s = __uint_as_float(e == 0u ? 0x00400000u : e << 23);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const bf16x8 wb = mx4_decode(L.code[q][t][j], s);
#pragma unroll
                        for (int p = 0; p < NI; ++p) acc[q][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb, xb[j][p], acc[q][t], 0, 0, 0);
                    }
                }
            }
        }
    };

    const int full = XT == MX4_X_MX4 ? kps : a.K / MX4_COLS;                 // panels without a ragged end
    // Every load inside the loops is unconditional (x in rows: past the end the last panel once more; x in MXFP4: the loop ends before
    // that): behind a load under a condition the compiler waits for everything in flight, the panel ahead included.
    Load nxt;
    if (wave < full) fetch(wave, nxt, false);
    for (int i = tid; i < NPAN * MX4_ROWS; i += W * 64) s_bad_n[i] = 0;
    if (tid < 16) s_bad_m[tid] = 0;
    if constexpr (XT == MX4_X_MX4) {
        // two panels ahead, each loaded into the registers that are done with (one row of 32000 x 4096 13.1 us, one panel ahead
        // 13.8; the other kinds' longer steps gain nothing from it: five float32 rows 19.8 against 17.6)
        Load aft;
        int kp = wave;
        if (kp + W < full) fetch(kp + W, aft, false);
        for (; kp + 3 * W < full; kp += 2 * W) {
            multiply(nxt);
            __builtin_amdgcn_sched_barrier(0);
            fetch(kp + 2 * W, nxt, false);
            multiply(aft);
            __builtin_amdgcn_sched_barrier(0);
            fetch(kp + 3 * W, aft, false);
        }
        auto finish = [&](int p, Load& L) {
            if (p >= full) return;
            if (p == full - 1) {
#pragma unroll
                for (int q = 0; q < NPAN; ++q) L.scale[q] = mx4_last_scales(L.scale[q], lane, kps, a.K);
                L.gain.x = mx4_last_scales(L.gain.x, lane, kps, a.K);
            }
            multiply(L);
        };
        finish(kp, nxt);
        if (kp + 2 * W < full) fetch(kp + 2 * W, nxt, false);
        finish(kp + W, aft);
        finish(kp + 2 * W, nxt);
    } else {
        for (int kp = wave; kp < full; kp += W) {
            const Load cur = nxt;
            fetch(min(kp + W, full - 1), nxt, false);
            multiply(cur);
        }
        if (full < kps && full % W == wave) {
            fetch(full, nxt, true);
#pragma unroll
            for (int q = 0; q < NPAN; ++q) nxt.scale[q] = mx4_last_scales(nxt.scale[q], lane, kps, a.K);
            multiply(nxt);
        }
    }

    // the waves' sums, in wave order (and the pieces' after one another), a panel at a time
    __syncthreads();
#pragma unroll
    for (int q = 0; q < NPAN; ++q)
        if (bad[q])
#pragma unroll
            for (int t = 0; t < TT; ++t)
                if (bad[q] >> (8 * t) & 128u) s_bad_n[q * MX4_ROWS + t * 16 + c16] = 1u;
    if (bad_x) s_bad_m[c16] = 1u;
    if constexpr (XT == MX4_X_F32)
        if (a.gain)
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                float v = sq[i];
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) v += __shfl_xor(v, o);
                const int m = (i * 64 + lane) / PER_ROW;
                if (lane % 32 == 0 && m < 16) s_sq[wave][m] = v;
            }
#pragma unroll
    for (int q = 0; q < NPAN; ++q) {
        if (q > 0) __syncthreads();
#pragma unroll
        for (int t = 0; t < TT; ++t) *reinterpret_cast<f32x4*>(sh + ((wave * TT + t) * 64 + lane) * 16) = acc[q][t];
        __syncthreads();
        const int64_t m = m0 + c16;
        const int nr = (tid >> 6) * 16 + g * 4;
        const int64_t n = (int64_t)(panel0 + q) * MX4_ROWS + t0 * 16 + nr;
        if (tid >= TT * 64 || c16 >= MP || m >= a.M || n >= a.N) continue;
        float v[4] = {0.f, 0.f, 0.f, 0.f}, first[4], rs = 1.f;
#pragma unroll
        for (int p = 0; p < (COLS ? 3 : 1); ++p) {
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const f32x4 o = *reinterpret_cast<const f32x4*>(sh + (w * TT * 64 + tid + p * MP) * 16);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] += o[i];
            }
            if (p == 0)
#pragma unroll
                for (int i = 0; i < 4; ++i) first[i] = v[i];
        }
        if (COLS)       // an infinity of w times a zero second or third piece is NaN: the first piece alone has IEEE's result
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = v[i] == v[i] ? v[i] : first[i];
        if constexpr (XT == MX4_X_F32)
            if (a.gain) {
                float ss = 0.f;
#pragma unroll
                for (int w = 0; w < W; ++w) ss += s_sq[w][c16];
                rs = rms_recip(ss, a.K, a.eps);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] *= rs;
            }
        if constexpr (FAR) {
            unsigned again = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) again |= n + i < a.N ? s_bad_n[q * MX4_ROWS + nr + i] << i : 0u;
            if (__builtin_expect(again != 0u, 0))
#pragma unroll 1
                for (; again; again &= again - 1) {
                    const int at = __builtin_ctz(again);
                    const float y = mx4_far_output(a, m, n + at, rs, at == 0 ? v[0] : at == 1 ? v[1] : at == 2 ? v[2] : v[3]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = i == at ? y : v[i];
                }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (s_bad_n[q * MX4_ROWS + nr + i] | s_bad_m[c16]) v[i] = __uint_as_float(0x7FC00000u);
        }
        mx4_store(a, m, n, v);
    }
}

// ---- product of many rows: bound by the matrix cores.  A workgroup of WN x WM x KW waves computes WN panels of 64 outputs for
// 16 CT WM rows of x, a wave one panel for 16 CT rows over every KW-th 128 columns (their sums are added at the end: with few
// tiles it takes several waves per SIMD to hide what a step waits for).  x goes through LDS (as bfloat16 pieces, two buffers, the
// columns of the next two steps on their way in registers), in operand order: the operand of 16 rows and sub-step j is a
// kilobyte of which lane l = 16 b + r reads its 16 bytes at l * 16, free of bank conflicts however the hardware groups the lanes.  A wave
// stages a quarter of each block (sub-step) at a time: lane 16 g + r brings columns 32 i + 8 g .. of row r.  The codes go straight into
// the wave's registers and are turned into bfloat16 operands there: 64 conversions for 64 CT matrix instructions per piece.
template <int XT, int CT, int WN, int WM, int KW>
struct Mx4Tile {
    static constexpr int THREADS = 64 * WN * WM * KW, TM = 16 * CT * WM, NPC = XT == MX4_X_F32 ? 3 : 1;
    static constexpr int PANEL = NPC * TM * 256, BUF = KW * PANEL; // bytes of x: 128 columns, a step
    static constexpr int RED = (KW - 1) * WN * WM * 64 * 16 * CT * 4;
    static constexpr int LDS = 2 * BUF > RED + WN * WM * MX4_OUT_BYTES ? 2 * BUF : RED + WN * WM * MX4_OUT_BYTES;
    static constexpr int WAVES = WN * WM * KW;
    static constexpr int PER_K = TM / 4 / WAVES, NCH = KW * PER_K; // 8-element pieces of x that a thread stages: of 128 columns, in all
    static constexpr int AHEAD = NPC == 3 ? 2 : 4;                 // units whose operands are read ahead
    static_assert(TM / 4 % WAVES == 0 && WAVES % 4 == 0, "a wave stages one block of the columns of some row tiles");
};
// Workgroup -> tile of n_n x n_m: workgroups run on XCD id % 8, each XCD takes a stretch of tiles of its own, and a stretch
// goes through the outputs for 8 row tiles at a time, row tiles fastest: its L2 sees the same codes and rows again soon.
__device__ __forceinline__ bool mx4_tile_of(int n_n, int n_m, int& n, int& m) {
    const int per = (n_n * n_m + 7) / 8, tile = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per || tile >= n_n * n_m) return false;
    const int group = tile / (8 * n_n), r = tile - group * 8 * n_n, in = min(8, n_m - group * 8);
    n = r / in; m = group * 8 + r % in;
    return true;
}
// which of a tile's 16 weight rows have a NaN block, by the high bits that mx4_nan_bytes found (bit t of every byte's lane)
__device__ __forceinline__ unsigned mx4_nan_rows(unsigned bad, int t) {
    const unsigned long long v = __ballot(bad >> (8 * t) & 128u);
    return (unsigned)(v | v >> 16 | v >> 32 | v >> 48) & 0xFFFFu;
}
template <int XT, int CT, int WN, int WM, int KW>
__global__ __launch_bounds__(64 * WN * WM * KW, 2) void k_mx4_tiles(Mx4Product a) {
    typedef Mx4Tile<XT, CT, WN, WM, KW> S;
    typedef typename Mx4In<XT>::T T;
    extern __shared__ __attribute__((aligned(16))) char sh[];
    __shared__ float s_sq[KW * 4][S::TM];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c16 = lane & 15, g = lane >> 4;
    const int wn = wave % WN, wm = wave / WN % WM, kg = wave / (WN * WM);
    const int kps = (a.K + MX4_COLS - 1) / MX4_COLS, steps = (kps + KW - 1) / KW, n_pan = (a.N + MX4_ROWS - 1) / MX4_ROWS;
    int tn, tm;
    if (!mx4_tile_of((n_pan + WN - 1) / WN, (a.M + S::TM - 1) / S::TM, tn, tm)) return;
    const int panel = tn * WN + wn;
    const int64_t m0 = (int64_t)tm * S::TM;
    const char* wp = a.w + (size_t)min(panel, n_pan - 1) * kps * MX4_PANEL_BYTES;
    constexpr int XV = XT == MX4_X_F32 ? 2 : 1;
    // what this wave stages: block wave % 4 of the columns, sub-step g, of row tiles wave / 4, + WAVES / 4 ..
    const int blk = wave % 4, tile0 = wave / 4;

    struct Load { u32x4 x[S::NCH][XV], gain[KW][XV], code[4]; unsigned scale; };   // what a step brings, on its way
    Load f0, f1;
    unsigned bad = 0;
    float sq[S::NCH];
    f32x4 acc[4][CT];
#pragma unroll
    for (int i = 0; i < S::NCH; ++i) sq[i] = 0.f;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int c = 0; c < CT; ++c) acc[t][c] = f32x4{0.f, 0.f, 0.f, 0.f};

    const T* xrow[S::PER_K];
#pragma unroll
    for (int i = 0; i < S::PER_K; ++i) xrow[i] = (const T*)a.x + min(m0 + (tile0 + i * (S::WAVES / 4)) * 16 + c16, (int64_t)a.M - 1) * a.ldx;
    const float* gain = a.gain ? a.gain : (const float*)a.x;       // (without a gain: loaded, not used)
    auto fetch_codes = [&](int st, Load& f) {
        const char* p = wp + (size_t)min(st * KW + kg, kps - 1) * MX4_PANEL_BYTES;
#pragma unroll
        for (int t = 0; t < 4; ++t) f.code[t] = *reinterpret_cast<const SDFP_GLOBAL u32x4*>(as_global(p + t * MX4_TILE_BYTES + lane * 16));
        f.scale = *reinterpret_cast<const SDFP_GLOBAL unsigned*>(as_global(p + MX4_CODE_BYTES + lane * 4));
    };
    auto fetch_x = [&](int st, Load& f, bool full) {
#pragma unroll
        for (int z = 0; z < KW; ++z) {
            const int64_t k = (int64_t)(st * KW + z) * MX4_COLS + blk * 32 + g * 8;
#pragma unroll
            for (int v = 0; v < XV; ++v) {
#pragma unroll
                for (int i = 0; i < S::PER_K; ++i) f.x[z * S::PER_K + i][v] = mx4_load<XT>(xrow[i], k + v * 4, a.K, full);
                if constexpr (XT == MX4_X_F32) f.gain[z][v] = mx4_load<XT>(gain, k + v * 4, a.K, full);
            }
        }
    };
    auto store_x = [&](const Load& f, char* buf, bool count) {   // count: their squares belong to the rows' sums
#pragma unroll
        for (int i = 0; i < S::NCH; ++i) {
            char* to = buf + i / S::PER_K * S::PANEL + ((tile0 + i % S::PER_K * (S::WAVES / 4)) * 4 + g) * 1024 + (blk * 16 + c16) * 16;
            if constexpr (XT == MX4_X_F32) {
                float v[8], gn[8];
                Mx4In<XT>::unpack(f.x[i][0], *reinterpret_cast<float(*)[4]>(v));
                Mx4In<XT>::unpack(f.x[i][1], *reinterpret_cast<float(*)[4]>(v + 4));
                if (a.gain) {
                    Mx4In<XT>::unpack(f.gain[i / S::PER_K][0], *reinterpret_cast<float(*)[4]>(gn));
                    Mx4In<XT>::unpack(f.gain[i / S::PER_K][1], *reinterpret_cast<float(*)[4]>(gn + 4));
                    float ss = sq[i];
#pragma unroll
                    for (int e = 0; e < 8; ++e) { ss = fmaf(v[e], v[e], ss); v[e] *= gn[e]; }
                    sq[i] = count ? ss : sq[i];
                }
                unsigned pk[3][4];
                trunc3(v, pk);
#pragma unroll
                for (int p = 0; p < 3; ++p) *reinterpret_cast<u32x4*>(to + p * S::TM * 256) = u32x4{pk[p][0], pk[p][1], pk[p][2], pk[p][3]};
            } else {
                *reinterpret_cast<u32x4*>(to) = f.x[i][0];
            }
        }
    };
    // decoded: called when the codes in f are not needed any more
    auto multiply = [&](const char* buf, Load& f, auto decoded) {
        buf += kg * S::PANEL + wm * CT * 4096 + lane * 16;
        bad |= XT == MX4_X_F32 ? mx4_far_bytes(f.scale) : mx4_nan_bytes(f.scale);
        float s[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const unsigned e = f.scale >> (8 * t) & 255u;
            s[t] = __uint_as_float(e == 0u ? 0x00400000u : e << 23);
        }
        // unit u: sub-step u / CT, row tile u % CT; its operands are read S::AHEAD units earlier, and while a sub-step's units
        // run the weights of the next are decoded, a few tiles per unit
        bf16x8 xb[S::AHEAD][S::NPC], wb[2][4];
        auto read = [&](int u) {
#pragma unroll
            for (int p = 0; p < S::NPC; ++p)
                xb[u % S::AHEAD][p] = *reinterpret_cast<const bf16x8*>(buf + p * S::TM * 256 + (u % CT * 4 + u / CT) * 1024);
        };
#pragma unroll
        for (int u = 0; u < S::AHEAD; ++u) read(u);
#pragma unroll
        for (int t = 0; t < 4; ++t) wb[0][t] = mx4_decode(f.code[t][0], s[t]);
#pragma unroll
        for (int u = 0; u < 4 * CT; ++u) {
            const int j = u / CT, c = u % CT;
#pragma unroll
            for (int p = 0; p < S::NPC; ++p)
#pragma unroll
                for (int t = 0; t < 4; ++t) acc[t][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb[j & 1][t], xb[u % S::AHEAD][p], acc[t][c], 0, 0, 0);
            if (u + S::AHEAD < 4 * CT) read(u + S::AHEAD);
            if (j < 3)
#pragma unroll
                for (int t = 4 * c / CT; t < 4 * (c + 1) / CT; ++t) wb[~j & 1][t] = mx4_decode(f.code[t][j + 1], s[t]);
            __builtin_amdgcn_sched_barrier(0);
            if (u == 3 * CT - 1) decoded();
        }
    };
    // Step st: x lies in LDS, the codes in f; next, on its way since the step before, goes to LDS.  What step st + 2 needs is loaded
    // into f as this step is done with its parts: loaded into other registers, it is copied at the loop's end, and a copy waits
    // for its load.  Every load and store of the loop is unconditional (past the end the last step once more): behind a load under
    // a condition the compiler waits for everything in flight.
    const int full = a.K / (MX4_COLS * KW);                        // steps without a ragged end
    auto step = [&](int st, Load& f, const Load& next) {
        const int then = min(st + 2, full - 1);
        fetch_x(then, f, true);
        multiply(sh + (st & 1) * S::BUF, f, [&] { fetch_codes(then, f); });
        store_x(next, sh + (~st & 1) * S::BUF, st + 1 < full);
        __syncthreads();
    };
    auto fetch = [&](int st, Load& f, bool full) { fetch_codes(st, f); fetch_x(st, f, full); };
    if (full > 0) {
        fetch(0, f0, true);
        fetch(min(1, full - 1), f1, true);
        store_x(f0, sh, true);
        __syncthreads();
        int st = 0;
        for (; st + 1 < full; st += 2) { step(st, f0, f1); step(st + 1, f1, f0); }
        if (st < full) step(st, f0, f1);
    }
    if (full < steps) {
        fetch(full, f0, false);
        store_x(f0, sh, true);
        __syncthreads();
        if (full * KW + kg == kps - 1) f0.scale = mx4_last_scales(f0.scale, lane, kps, a.K);
        if (full * KW + kg < kps) multiply(sh, f0, [] {});
        __syncthreads();
    }
    if constexpr (XT == MX4_X_F32)
        if (a.gain)
#pragma unroll
            for (int i = 0; i < S::NCH; ++i) {
                float v = sq[i];
                v += __shfl_xor(v, 16);
                v += __shfl_xor(v, 32);
                if (g == 0) s_sq[i / S::PER_K * 4 + blk][(tile0 + i % S::PER_K * (S::WAVES / 4)) * 16 + c16] = v;
            }
    __shared__ unsigned s_bad[KW > 1 ? S::THREADS : 1];
    if constexpr (KW > 1) {   // the other waves' sums of this tile, in their order
        f32x4* red = reinterpret_cast<f32x4*>(sh);
        if (kg > 0) {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int c = 0; c < CT; ++c) red[((wave - WN * WM) * 4 * CT + t * CT + c) * 64 + lane] = acc[t][c];
        }
        s_bad[tid] = bad;
        __syncthreads();
        if (kg > 0) return;
#pragma unroll
        for (int z = 1; z < KW; ++z) {
            bad |= s_bad[tid + z * WN * WM * 64];
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int c = 0; c < CT; ++c) {
                    const f32x4 o = red[((wave + (z - 1) * WN * WM) * 4 * CT + t * CT + c) * 64 + lane];
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[t][c][i] += o[i];
                }
        }
    } else if (XT == MX4_X_F32 && a.gain) {
        __syncthreads();
    }
    unsigned odd = 0;               // bit 4 t + i: that output of the lane is NaN, or (float32) to be added up again
#pragma unroll
    for (int t = 0; t < 4; ++t) odd |= (mx4_nan_rows(bad, t) >> (g * 4) & 15u) << (4 * t);
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        const int mr = (wm * CT + c) * 16;
        float rs = 1.f;
        if constexpr (XT == MX4_X_F32)
            if (a.gain) {
                float ss = 0.f;
#pragma unroll
                for (int z = 0; z < KW * 4; ++z) ss += s_sq[z][mr + c16];
                rs = rms_recip(ss, a.K, a.eps);
            }
        f32x4 v[4];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[t][i] = acc[t][c][i];
                if (XT == MX4_X_F32 && a.gain) v[t][i] *= rs;
                if (XT != MX4_X_F32 && odd >> (4 * t + i) & 1u) v[t][i] = __uint_as_float(0x7FC00000u);
            }
        if (XT == MX4_X_F32 && __builtin_expect(odd != 0u, 0))
#pragma unroll 1
            for (unsigned left = odd; left; left &= left - 1) {
                const int at = __builtin_ctz(left);
                const int64_t m = m0 + mr + c16, n = (int64_t)panel * MX4_ROWS + at / 4 * 16 + g * 4 + at % 4;
                if (m >= a.M || n >= a.N) continue;
                float y = 0.f;
#pragma unroll
                for (int k = 0; k < 16; ++k) y = k == at ? v[k / 4][k % 4] : y;
                y = mx4_far_output(a, m, n, rs, y);
#pragma unroll
                for (int k = 0; k < 16; ++k) v[k / 4][k % 4] = k == at ? y : v[k / 4][k % 4];
            }
        mx4_store_tile(a, sh + S::RED + wave * MX4_OUT_BYTES, m0 + mr, (int64_t)panel * MX4_ROWS, v);
    }
}

// Both sides in MXFP4: the codes are the operands of the scaled 4-bit instruction as they lie in memory.  A workgroup of WN x WM
// waves computes WN panels of w for CT WM / 4 of x, a wave one panel of w for CT 16-row tiles of x.  x, codes and scales, goes
// through LDS (two buffers), a wave's panel of w straight into its registers, everything two steps of 128 columns ahead: with w
// in LDS as well its bandwidth was the bound, and scales of x that every wave loads for itself wait for one another (1024 rows x
// 4096 x 14336: 44 us, those loads 50).  4096 rows x 14336 x 4096 at 3.2 PFLOP/s, 4096 x 4096 x 14336 at 4.3, of the 8.0 that these
// instructions reach without loads.  Of the former's 150 us 42 go with the write of 235 MB of float32 results, which a workgroup does
// at its end with nothing else in flight (workgroups started at different times: the same), and its 1792 tiles are three and a half
// rounds of the two workgroups that a compute unit holds.
template <int CT, int WN, int WM>
struct Mx4TileX {
    static constexpr int WAVES = WN * WM, XP = CT * WM / 4, BUF = XP * MX4_PANEL_BYTES;   // all tiles of x, then their scales
    static constexpr int LDS = 2 * BUF > WAVES * MX4_OUT_BYTES ? 2 * BUF : WAVES * MX4_OUT_BYTES;
    static constexpr int NT = XP * 4 / WAVES;                      // tiles of x that a wave fetches
    static constexpr int NS = XP * 64 / WAVES;                     // words of scales of x
    static_assert(XP * 4 % WAVES == 0 && 4 % NT == 0 && CT % 4 == 0 && 64 % NS == 0, "a wave fetches parts of one panel");
};
template <int CT, int WN, int WM>
__global__ __launch_bounds__(64 * WN * WM, 2) void k_mx4_tiles_mx4(Mx4Product a) {
    typedef Mx4TileX<CT, WN, WM> S;
    extern __shared__ __attribute__((aligned(16))) char sh[];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c16 = lane & 15, g = lane >> 4, wn = wave % WN, wm = wave / WN;
    const int kps = (a.K + MX4_COLS - 1) / MX4_COLS;
    const int n_pan = (a.N + MX4_ROWS - 1) / MX4_ROWS, m_pan = (a.M + MX4_ROWS - 1) / MX4_ROWS;
    int tn, tm;
    if (!mx4_tile_of((n_pan + WN - 1) / WN, (m_pan + S::XP - 1) / S::XP, tn, tm)) return;
    struct Load { u32x4 w[4], x[S::NT]; unsigned sw, sx; };
    auto x_panel = [&](int i) { return (const char*)a.x + (size_t)min(tm * S::XP + i, m_pan - 1) * kps * MX4_PANEL_BYTES; };
    const char* w_src = a.w + (size_t)min(tn * WN + wn, n_pan - 1) * kps * MX4_PANEL_BYTES;
    const char* x_src = x_panel(wave * S::NT / 4) + wave * S::NT % 4 * MX4_TILE_BYTES;   // the tiles of x this wave brings to LDS
    const int s_at = wave * S::NS + lane % S::NS;                                        // and the word of their scales
    const char* s_src = x_panel(s_at / 64) + MX4_CODE_BYTES + s_at % 64 * 4;
    Load f0, f1;
    unsigned bad = 0, bad_x[CT / 4];
    f32x4 acc[4][CT];
#pragma unroll
    for (int i = 0; i < CT / 4; ++i) bad_x[i] = 0;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int c = 0; c < CT; ++c) acc[t][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    // loads of a step (past the end: the last columns again, not used), each into the registers that the step two before has
    // done with: loaded into others, they are copied at the loop's end, and a copy waits for its load
    auto at = [&](int st) { return (size_t)min(st, kps - 1) * MX4_PANEL_BYTES; };
    auto fetch_x = [&](int st, Load& f) {
#pragma unroll
        for (int i = 0; i < S::NT; ++i) f.x[i] = *reinterpret_cast<const SDFP_GLOBAL u32x4*>(as_global(x_src + at(st) + i * MX4_TILE_BYTES + lane * 16));
        f.sx = *reinterpret_cast<const SDFP_GLOBAL unsigned*>(as_global(s_src + at(st)));
    };
    auto fetch_w = [&](int st, int t, Load& f) {
        f.w[t] = *reinterpret_cast<const SDFP_GLOBAL u32x4*>(as_global(w_src + at(st) + t * MX4_TILE_BYTES + lane * 16));
    };
    auto fetch_s = [&](int st, Load& f) {
        f.sw = *reinterpret_cast<const SDFP_GLOBAL unsigned*>(as_global(w_src + at(st) + MX4_CODE_BYTES + lane * 4));
    };
    auto store = [&](const Load& f, char* buf) {
#pragma unroll
        for (int i = 0; i < S::NT; ++i) *reinterpret_cast<u32x4*>(buf + (wave * S::NT + i) * MX4_TILE_BYTES + lane * 16) = f.x[i];
        *reinterpret_cast<unsigned*>(buf + S::XP * MX4_CODE_BYTES + s_at * 4) = f.sx;
    };
    // step st: the tiles of x lie in LDS, the rest in f; next's tiles go to LDS (more: there is a next step)
    auto step = [&](int st, Load& f, const Load& next, auto more) {
        const char* px = sh + (st & 1) * S::BUF + wm * CT * MX4_TILE_BYTES + lane * 16;
        const char* ps = sh + (st & 1) * S::BUF + S::XP * MX4_CODE_BYTES + wm * CT * 64 + lane * 4;
        unsigned sx[CT / 4];
        u32x4 x[CT];
#pragma unroll
        for (int i = 0; i < CT / 4; ++i) sx[i] = *reinterpret_cast<const unsigned*>(ps + i * 256);
#pragma unroll
        for (int c = 0; c < CT; ++c) x[c] = *reinterpret_cast<const u32x4*>(px + c * MX4_TILE_BYTES);
        if (more) fetch_x(st + 2, f);
        bad |= mx4_nan_bytes(f.sw);
#pragma unroll
        for (int i = 0; i < CT / 4; ++i) bad_x[i] |= mx4_nan_bytes(sx[i]);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
            for (int c = 0; c < CT; ++c) acc[t][c] = mx4_mfma(f.w[t], (int)(f.sw >> (8 * t)), x[c], (int)(sx[c / 4] >> (8 * (c % 4))), acc[t][c]);
            __builtin_amdgcn_sched_barrier(0);
            if (more) fetch_w(st + 2, t, f);
        }
        if (more) {
            fetch_s(st + 2, f);
            store(next, sh + (~st & 1) * S::BUF);
        }
        __syncthreads();
    };
    auto fetch = [&](int st, Load& f) {
        fetch_x(st, f);
#pragma unroll
        for (int t = 0; t < 4; ++t) fetch_w(st, t, f);
        fetch_s(st, f);
    };
    fetch(0, f0);
    fetch(1, f1);
    store(f0, sh);
    __syncthreads();
    const int last = kps - 1;
    int st = 0;
    for (; st + 1 < last; st += 2) { step(st, f0, f1, std::true_type()); step(st + 1, f1, f0, std::true_type()); }
    if (st < last) { step(st, f0, f1, std::true_type()); f0 = f1; }
    if (last * MX4_COLS + 3 * MX4_BLOCK >= a.K) {   // blocks past the matrix: the last step by itself (their test in the loop: 1024 x 4096 x 14336 46 -> 50 us)
        f0.sw = mx4_last_scales(f0.sw, lane, kps, a.K);
        unsigned* sx = reinterpret_cast<unsigned*>(sh + (last & 1) * S::BUF + S::XP * MX4_CODE_BYTES + s_at * 4);
        *sx = mx4_last_scales(*sx, s_at % 64, kps, a.K);
        __syncthreads();
    }
    step(last, f0, f0, std::false_type());
    unsigned nan[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) nan[t] = mx4_nan_rows(bad, t) >> (g * 4);
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        const unsigned nan_x = mx4_nan_rows(bad_x[c / 4], c % 4) >> c16 & 1u;
        f32x4 v[4];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[t][i] = nan_x | (nan[t] >> i & 1u) ? __uint_as_float(0x7FC00000u) : acc[t][c][i];
        mx4_store_tile(a, sh + wave * MX4_OUT_BYTES, (int64_t)tm * S::XP * MX4_ROWS + (wm * CT + c) * 16, (int64_t)(tn * WN + wn) * MX4_ROWS, v);
    }
}

}  // namespace sdfp
