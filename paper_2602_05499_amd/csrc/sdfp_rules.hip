// Entry point of the rules on rows of logits (include/sdfp.h): argument checks and the launch.
#include "sdfp_rules_args.h"
#include "sdfp.h"

using namespace sdfp;

namespace {

// Short chunks for few rows: 2048 entries of a 512-thread workgroup, one quad of them per thread (one row of 32000 3.3 us, 4096
// entries 4.0 to 6.0; five of 128256 4.6 against 5.2 to 6.8).  Once 4096-entry chunks of 256 threads still make four
// workgroups per compute unit, those: a row's history is read half as often (256 rows of 32003 in bfloat16 13.4 us against
// 16.7, 64 of 128256 13.8 against 16.4 -- 4.9 TB/s, a large copy 4.7).
// A launch holds 2^32 - 1 threads: beyond those (millions of rows) several follow each other.
template <typename T, int THREADS, int NV>
hipError_t launch_rows(RulesRows a, int rows, hipStream_t s) {
    constexpr int CH = THREADS * 4 * NV;
    const int chunks = (a.vocab + CH - 1) / CH, most = (int)(UINT32_MAX / THREADS) / chunks;
    for (int64_t r = 0; r < rows; r += most) {
        a.row0 = (int)r;
        const unsigned n = (unsigned)(rows - r < most ? rows - r : most) * (unsigned)chunks;
        hipLaunchKernelGGL((k_logits_rules<T, THREADS, NV>), dim3(n), dim3(THREADS), 0, s, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
template <typename T>
hipError_t launch(const RulesRows& a, int rows, hipStream_t s) {
    if ((int64_t)rows * ((a.vocab + 4095) / 4096) >= 1024) return launch_rows<T, 256, 4>(a, rows, s);
    return launch_rows<T, 512, 1>(a, rows, s);
}

}  // namespace

extern "C" int sd_logits_rules(const void* z, int dtype, int64_t ld, int32_t rows, int32_t vocab, const sd_rules* rules,
                               const int32_t* tokens, int64_t n_tokens, const int64_t* begin, const int64_t* end,
                               const int32_t* mask_row, void* out, int64_t ld_out, void* hip_stream) {
    if (!z || !out || !rules || rows < 1 || vocab < 1 || vocab > INT32_MAX - 8192 || ld < vocab || ld_out < vocab) return SD_EINVAL;
    if (dtype != SD_F32 && dtype != SD_BF16) return SD_EINVAL;
    const uintptr_t es = dtype == SD_F32 ? 4 : 2;
    if (((uintptr_t)z | (uintptr_t)out) & (es - 1)) return SD_EINVAL;
    if (!rules_ok(*rules)) return SD_EINVAL;
    if (z == out && ld != ld_out) return SD_EINVAL;     // in place: the same rows
    if (z != out && ld == ld_out) {                     // rows of out across rows of z
        const uintptr_t d = ((uintptr_t)z > (uintptr_t)out ? (uintptr_t)z - (uintptr_t)out : (uintptr_t)out - (uintptr_t)z) / es;
        const uint64_t n = d / (uint64_t)ld, q = d % (uint64_t)ld;
        if ((q < (uint64_t)vocab && n < (uint64_t)rows) || ((uint64_t)ld - q < (uint64_t)vocab && n + 1 < (uint64_t)rows)) return SD_EINVAL;
    }
    RulesRows a = {};
    a.z = z; a.out = out; a.ld = ld; a.ld_out = ld_out; a.vocab = vocab;
    a.r = rule_set(*rules);
    if (has_penalties(a.r.repetition, a.r.presence, a.r.frequency)) {
        if (n_tokens < 0 || (n_tokens > 0 && !tokens) || !begin || !end) return SD_EINVAL;
        if (((uintptr_t)tokens & 3) || (((uintptr_t)begin | (uintptr_t)end) & 7)) return SD_EINVAL;
        if (n_tokens > 0) { a.tokens = tokens; a.n_tokens = n_tokens; a.begin = begin; a.end = end; }
    }
    if (rules->allowed) {
        if ((uintptr_t)mask_row & 3) return SD_EINVAL;
        if (!mask_row && rules->n_masks != 1 && rules->n_masks != rows) return SD_EINVAL;
        a.mask_row = mask_row;
    }
    hipStream_t s = (hipStream_t)hip_stream;
    return (dtype == SD_F32 ? launch<float>(a, rows, s) : launch<bf16_t>(a, rows, s)) == hipSuccess ? SD_OK : SD_EHIP;
}
