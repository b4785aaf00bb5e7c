// Rules on logits: penalties for repeated tokens, a bias, bit masks of allowed tokens.
#pragma once
#include "sdfp_common.hip.h"

namespace sdfp {

// One logit under the rules.  n: occurrences of the token in its row's history.  Penalties in the order multiplicative,
// frequency, presence; then the bias; then the mask.  Every step is one float32 operation, rounded once.
struct RuleSet {
    float repetition, presence, frequency;   // 1, 0, 0: no penalty
    const float* bias;                       // [vocab] or nullptr
    const unsigned* allowed;                 // [n_masks][words]: bit j % 32 of word j / 32 allows token j; or nullptr
    int n_masks;
};
__device__ __forceinline__ float apply_penalties(float z, unsigned n, const RuleSet& r) {
    const float m = z > 0.f ? div_rn(z, r.repetition) : mul_rn(z, r.repetition);
    const float p = sub_rn(sub_rn(m, mul_rn(r.frequency, (float)n)), r.presence);
    return n ? p : z;
}
__host__ __device__ __forceinline__ bool has_penalties(float repetition, float presence, float frequency) {
    return !(repetition == 1.f && presence == 0.f && frequency == 0.f);
}

typedef u32x4 __attribute__((aligned(4))) u32x4_w;     // 16 bytes at any 4-byte address
typedef u32x2 __attribute__((aligned(2))) u32x2_h;
// four neighbouring logits of a row as float32; n_have: how many exist (at least 4: all)
template <typename T>
__device__ __forceinline__ f32x4 rules_load4(const T* p, int n_have) {
    f32x4 v{0.f, 0.f, 0.f, 0.f};
    if (n_have >= 4) {
        if constexpr (sizeof(T) == 4) {
            v = __builtin_bit_cast(f32x4, *reinterpret_cast<const SDFP_GLOBAL u32x4_w*>(as_global(p)));
        } else {
            const u32x2 r = *reinterpret_cast<const SDFP_GLOBAL u32x2_h*>(as_global(p));
            v = f32x4{__uint_as_float(r.x << 16), __uint_as_float(r.x & 0xFFFF0000u), __uint_as_float(r.y << 16), __uint_as_float(r.y & 0xFFFF0000u)};
        }
        return v;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < n_have) v[i] = sizeof(T) == 4 ? (float)reinterpret_cast<const float*>(p)[i] : bf16_to_f32(reinterpret_cast<const bf16_t*>(p)[i]);
    return v;
}
template <typename T>
__device__ __forceinline__ void rules_store4(T* p, const f32x4& v, int n_have) {
    if (n_have >= 4) {
        if constexpr (sizeof(T) == 4) *reinterpret_cast<SDFP_GLOBAL u32x4_w*>(as_global(p)) = __builtin_bit_cast(u32x4, v);
        else *reinterpret_cast<SDFP_GLOBAL u32x2_h*>(as_global(p)) = u32x2{pack_bf16(v.x, v.y), pack_bf16(v.z, v.w)};
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < n_have) {
            if constexpr (sizeof(T) == 4) p[i] = v[i];
            else p[i] = (T)pack_bf16(v[i], v[i]);
        }
}

// ---- rows of logits with a token history each.  A workgroup takes CH neighbouring entries of one row: it counts the history
// tokens that fall among them in LDS (integer adds: any order, same counts), then reads, changes and writes its entries.  No
// count ever leaves the workgroup, nothing is cleared beforehand, one launch.  The price is that every chunk of a row reads
// the row's history (from L2); longer chunks read it less often, shorter ones spread few rows over the chip.  Bound by the
// logits' read and write for many rows, by latency -- history, counts, entries one after the other -- for a few.
constexpr int RULES_THREADS = 256;
struct RulesRows {
    const void* z; void* out;
    int64_t ld, ld_out;
    int row0, vocab;              // the launch's first row
    RuleSet r;
    const int* tokens;            // [n_tokens], or nullptr: no penalties
    int64_t n_tokens;
    const int64_t *begin, *end;   // [rows]: the row's history is tokens[begin .. end)
    const int* mask_row;          // [rows] or nullptr: row i under mask i (mask 0 if there is one mask)
};
template <typename T, int THREADS, int NV>
__global__ __launch_bounds__(THREADS) void k_logits_rules(RulesRows a) {
    constexpr int CH = THREADS * 4 * NV;
    __shared__ __attribute__((aligned(16))) unsigned cnt[CH];
    const int tid = threadIdx.x, chunks = (a.vocab + CH - 1) / CH, in = blockIdx.x / chunks, row = a.row0 + in;
    const int lo = (blockIdx.x - in * chunks) * CH;
    const T* z = reinterpret_cast<const T*>(a.z) + (int64_t)row * a.ld + lo;
    const int have = a.vocab - lo;
    const unsigned* mask = nullptr;
    if (a.r.allowed) {
        const int mr = a.mask_row ? a.mask_row[row] : a.r.n_masks == 1 ? 0 : row;
        if (mr >= 0 && mr < a.r.n_masks) mask = a.r.allowed + (int64_t)mr * ((a.vocab + 31) / 32) + (lo >> 5);
    }
    // everything that the entries need is on its way while the history is counted
    f32x4 v[NV], bi[NV];
    unsigned w[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int j = (i * THREADS + tid) * 4;
        v[i] = rules_load4(z + j, have - j);
        if (a.r.bias) bi[i] = rules_load4(a.r.bias + lo + j, have - j);
        if (mask && j < have) w[i] = mask[j >> 5];
    }
    if (a.tokens) {
#pragma unroll
        for (int i = 0; i < NV; ++i) *reinterpret_cast<u32x4*>(cnt + (i * THREADS + tid) * 4) = u32x4{0u, 0u, 0u, 0u};
        const int64_t b = min(max(a.begin[row], (int64_t)0), a.n_tokens), e = min(a.end[row], a.n_tokens);
        __syncthreads();
        auto count = [&](int tok) {
            const unsigned at = (unsigned)tok - (unsigned)lo;
            if (at < (unsigned)CH && tok >= 0) atomicAdd(&cnt[at], 1u);
        };
        for (int64_t i = b + tid * 4; i < e; i += THREADS * 4) {
            if (i + 4 <= e) {
                const u32x4 t = *reinterpret_cast<const SDFP_GLOBAL u32x4_w*>(as_global(a.tokens + i));
                count((int)t.x); count((int)t.y); count((int)t.z); count((int)t.w);
            } else {
                for (int64_t k = i; k < e; ++k) count(a.tokens[k]);
            }
        }
        __syncthreads();
    }
    T* out = reinterpret_cast<T*>(a.out) + (int64_t)row * a.ld_out + lo;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int j = (i * THREADS + tid) * 4;
        if (j >= have) continue;
        f32x4 x = v[i];
        if (a.tokens) {
            const u32x4 n = *reinterpret_cast<const u32x4*>(cnt + j);
            if (n.x | n.y | n.z | n.w)       // few entries have a history: most waves go past the divisions
#pragma unroll
                for (int k = 0; k < 4; ++k) x[k] = apply_penalties(x[k], n[k], a.r);
        }
        if (a.r.bias)
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = add_rn(x[k], bi[i][k]);
        if (mask)
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = w[i] >> (j & 31) >> k & 1u ? x[k] : -INFINITY;
        rules_store4(out + j, x, have - j);
    }
}

}  // namespace sdfp
