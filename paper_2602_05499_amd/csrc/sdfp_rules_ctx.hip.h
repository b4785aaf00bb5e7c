// Rules on logits inside a decode context, and the greedy picks that come with them (part of the sdfp_api.hip unit).
#pragma once
#include "sdfp_rules.hip.h"
#include "sdfp_select.hip.h"

namespace sdfp {

// ---- the same rules inside a decode context (sd_set_rules).  The history is the prompt and the committed tokens, kept as a
// count per token; row i of a step has the i draft tokens in front of it on top.  A grammar is a table of states: state s
// masks with row s of `allowed`, token t leads to next[s][t].  A state of -1, or one whose mask allows nothing, masks nothing.
struct CtxRules {
    RuleSet r;
    const int* next;       // [n_masks][vocab] or nullptr: the state never changes
    unsigned* counts;      // [vocab], or nullptr: no rules (the rows are only searched for their maxima)
    int* state;            // the state in front of the pending step's first row
    const int* usable;     // [n_masks]: the mask allows a token
};
__device__ __forceinline__ int rules_step(const CtxRules& c, int s, int tok, int V) {
    if (s < 0 || !c.next) return s;
    if (tok < 0 || tok >= V) return -1;
    const int n = c.next[(int64_t)s * V + tok];
    return n >= 0 && n < c.r.n_masks ? n : -1;
}
// usable[m]: mask m allows some token of the vocabulary.  A workgroup per mask, up to RULES_MASK_GRID of them (a launch does not
// hold one for each of 2^24 masks).
constexpr int RULES_MASK_GRID = 65536;
__global__ __launch_bounds__(256) void k_rules_usable(const unsigned* __restrict__ allowed, int n_masks, int V, int* __restrict__ usable) {
    const int words = (V + 31) / 32;
    for (int64_t i = blockIdx.x; i < n_masks; i += gridDim.x) {
        const unsigned* m = allowed + i * words;
        unsigned any = 0;
        for (int w = threadIdx.x; w < words; w += 256) any |= w == words - 1 && V % 32 ? m[w] & ((1u << (V % 32)) - 1u) : m[w];
        const int r = __syncthreads_or(any != 0u);
        if (threadIdx.x == 0) usable[i] = r ? 1 : 0;
    }
}
// counts (cleared before) += the prompt and, unless the sequence is new, the committed tokens; the start state
__global__ __launch_bounds__(256) void k_rules_history(CtxRules c, int V, int start, const int* __restrict__ prompt, int n_prompt,
                                                       const int* __restrict__ out_tokens, const DevState* st) {
    const int n_out = out_tokens ? min(st->n_out, st->max_out) : 0;
    if (blockIdx.x == 0 && threadIdx.x == 0) *c.state = start;
    for (int i = blockIdx.x * 256 + threadIdx.x; i < n_prompt + n_out; i += gridDim.x * 256) {
        const int t = i < n_prompt ? prompt[i] : out_tokens[i - n_prompt];
        if (t >= 0 && t < V) atomicAdd(c.counts + t, 1u);
    }
}
// after a step's (or the prompt's) commit: its tokens join the history and move the state on
__global__ void k_rules_commit(CtxRules c, int V, const DevState* st) {
    if (threadIdx.x != 0 || blockIdx.x != 0) return;
    int s = *c.state;
    for (int i = 0; i <= st->n_acc; ++i) {
        const int t = i < st->n_acc ? st->d[i] : st->x;
        if (t >= 0 && t < V) c.counts[t] += 1u;
        s = rules_step(c, s, t, V);
    }
    *c.state = s;
}

// Entries of a chunk of k_rows_select: 1024, or as many thousands as keep all rows within SEL_CHUNKS chunks -- also those of a
// verify forward: every workgroup's arrival is an atomic on one word (five rows of 128256 in 630 workgroups 14.3 us, in
// 210 12.0).
__host__ __device__ constexpr int rules_chunk_len(int V, int rows) {
    return (int)(((int64_t)V * rows + SEL_CHUNKS * 1024 - 1) / (SEL_CHUNKS * 1024)) * 1024;
}
// Rows of a context's logits under its rules, in place, and (pick) their arg-maxes, lowest index first: what a greedy draft,
// verify or prompt needs in one launch.  Row r comes after r0 + r draft tokens.  Grid (chunks, rows); the last workgroup to
// arrive reduces the chunks' maxima, a wave per row.  A row without a number above -inf picks token 0.  Latency throughout:
// one row of 32000 6.6 us, five of them 8.6, one of 128256 7.7, five 12.0.
__global__ __launch_bounds__(RULES_THREADS) void k_rows_select(float* __restrict__ z, int V, int len, CtxRules c, int r0, int pick, SelBuf b,
                                                               DevState* st, int dst, int off) {
    __shared__ int s_state, s_extra[MAX_K];
    __shared__ unsigned long long s_best[RULES_THREADS / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, row = blockIdx.y, chunk = blockIdx.x, n_extra = min(r0 + row, MAX_K);
    float* zr = z + (int64_t)row * V;
    const bool ruled = c.counts != nullptr, counted = ruled && has_penalties(c.r.repetition, c.r.presence, c.r.frequency);
    f32x4 x, bi;
    u32x4 n;
    auto load = [&](int j) {   // (the counts' room is whole 256 bytes)
        x = rules_load4(zr + j, V - j);
        if (counted) n = *reinterpret_cast<const u32x4*>(c.counts + j);
        if (ruled && c.r.bias) bi = rules_load4(c.r.bias + j, V - j);
    };
    const int hi = min(V, (chunk + 1) * len);
    int j = chunk * len + tid * 4;
    if (j < hi) load(j);       // on its way while the state is found
    const unsigned* mask = nullptr;
    if (ruled) {
        if (tid < n_extra) s_extra[tid] = st->d[tid];
        if (tid == 0) {
            int s = -1;
            if (c.r.allowed) {
                s = *c.state;
                if (s >= c.r.n_masks) s = -1;
                for (int i = 0; i < n_extra; ++i) s = rules_step(c, s, st->d[i], V);
                if (s >= 0 && !c.usable[s]) s = -1;
            }
            s_state = s;
        }
        __syncthreads();
        if (s_state >= 0) mask = c.r.allowed + (int64_t)s_state * ((V + 31) / 32);
    }
    // the largest entry so far as (ordered bits, complement of the index): the maximum of these is the lowest index of the
    // largest value; NaN and -inf entries do not take part
    unsigned long long best = 0;
    while (j < hi) {
        if (ruled) {
            const unsigned w = mask ? mask[j >> 5] >> (j & 31) : ~0u;
            if (counted) {
                for (int i = 0; i < n_extra; ++i) {
                    const unsigned at = (unsigned)s_extra[i] - (unsigned)j;
#pragma unroll
                    for (int k = 0; k < 4; ++k) n[k] += at == (unsigned)k;
                }
                if (n.x | n.y | n.z | n.w)
#pragma unroll
                    for (int k = 0; k < 4; ++k) x[k] = apply_penalties(x[k], n[k], c.r);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (c.r.bias) x[k] = add_rn(x[k], bi[k]);
                if (!(w >> k & 1u)) x[k] = -INFINITY;
            }
            rules_store4(zr + j, x, V - j);
        }
        if (pick)
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (j + k < V && x[k] > -INFINITY) {
                    const unsigned u = __float_as_uint(x[k] + 0.f);                    // -0 counts as 0
                    const unsigned long long key = (unsigned long long)(u >> 31 ? ~u : u | 0x80000000u) << 32 | (unsigned)~(j + k);
                    best = key > best ? key : best;
                }
        j += RULES_THREADS * 4;
        if (j < hi) load(j);
    }
    if (!pick) return;
    auto wave_best = [&](unsigned long long v) -> unsigned long long {
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            const unsigned long long t = __shfl_xor(v, o);
            v = t > v ? t : v;
        }
        return v;
    };
    best = wave_best(best);
    if (lane == 0) s_best[wave] = best;
    __syncthreads();
    double* part = b.sum;   // [rows][SEL_CHUNKS], the keys' bits
    if (tid == 0) {
#pragma unroll
        for (int w = 1; w < RULES_THREADS / 64; ++w) best = s_best[w] > best ? s_best[w] : best;
        st_coh(part + row * SEL_CHUNKS + chunk, __longlong_as_double((long long)best));
    }
    if (!sel_last_arrival(b.counter, gridDim.x * gridDim.y)) return;
    for (int r = wave; r < (int)gridDim.y; r += RULES_THREADS / 64) {
        unsigned long long k = 0;
#pragma unroll
        for (int i = 0; i < SEL_CHUNKS / 64; ++i)
            if (i * 64 + lane < (int)gridDim.x) {
                const unsigned long long t = (unsigned long long)__double_as_longlong(ld_coh(part + r * SEL_CHUNKS + i * 64 + lane));
                k = t > k ? t : k;
            }
        k = wave_best(k);
        const int tok = k ? (int)~(unsigned)k : 0;
        if (lane == 0) {
            if (dst == ROWS_DRAFT) st->d[off + r] = tok;
            else st->amax[off + r] = tok;
        }
    }
}

}  // namespace sdfp
