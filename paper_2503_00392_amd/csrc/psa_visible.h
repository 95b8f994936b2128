// What the two attention kernels with a window share (psa_window.hip over the 16-bit cache, psa_packed.hip over the 4-bit
// one): which tokens a query sees, the weights of the value product in parts, and how the waves' and the splits' running
// sums come together.
#pragma once

#include "psa_attend.h"

namespace psa {

constexpr int kMaxSplits = 1024;      // splits of a request at most: their weights are an array in the merge's LDS
constexpr int kSplitStride = 132;     // floats of one split's result for one head: M, l, error bits (head 0), pad, acc[128]

// The query stands at position ctx - 1 and sees token t < ctx if t < sinks or t >= start = ctx - window.  The blocks that
// hold a visible token are 0 .. head-1 and tail .. N-1, and only these are ever looked at: a table entry or a page between
// them may hold anything.  They are counted through as 0 .. count-1.
struct Visible {
    int ctx, sinks, start, head, skip, count;
    __device__ __forceinline__ int block(int i) const { return i < head ? i : i + skip; }
    // (Without branches, and used in selections only: where lanes branched on it to overwrite an element of a vector, the
    // compiler lost the overwriting for the first element.)
    __device__ __forceinline__ bool sees(int t) const { return (t < ctx) & ((t < sinks) | (t >= start)); }
    __device__ __forceinline__ bool sees_all(int b) const {
        const int t = b * kPage;
        return t + kPage <= ctx && (t + kPage <= sinks || t >= start);
    }
};
__device__ __forceinline__ Visible make_visible(int ctx, int window, int num_sinks) {
    Visible v;
    v.ctx = ctx;
    v.sinks = min(num_sinks, ctx);
    v.start = max(0, ctx - window);
    const int N = (ctx + kPage - 1) / kPage;
    v.head = (v.sinks + kPage - 1) / kPage;
    const int tail = window > 0 ? max(v.head, v.start / kPage) : N;
    v.skip = tail - v.head;
    v.count = v.head + N - tail;
    return v;
}

// The weights of the value product, p in (0, 2^kSlack], are given to the matrix cores in 16-bit parts in neighbouring rows of one
// operand: upper and lower half in binary16 (22 bits of p), three parts in bfloat16 (all 24 bits: each is what truncation
// leaves of the rest).  Two bfloat16 parts leave an error of about 1e-6 of the output; three cost nothing where a head has four rows,
// and a second product of the same values where it has two (eight heads).
template <int G>
constexpr int kRowsPerHead = G == 8 ? 2 : 4;
template <int DT, int G>
constexpr int kProducts = (DT == 1 && G == 8) ? 2 : 1;

// The part of two weights that the lane's row gets in product `which`, packed.  What to take off is a mask per lane, so that
// nothing branches: bfloat16 parts are p, p less its upper 16 bits, and that less its own upper 16 bits, each cut to 16 bits
// (a row beyond the parts gets the last part again, and store_parts leaves it out).  Binary16 parts are p cut to 11
// bits, exactly, and the rest, rounded.
template <int DT, int G>
struct WeightParts {
    uint32_t m1, m2;
    __device__ __forceinline__ explicit WeightParts(int part) {
        if constexpr (DT == 0) {
            m1 = part == 0 ? 0xffffe000u : ~0u;
            m2 = part == 0 ? 0u : 0xffffe000u;
        } else if constexpr (G == 8) {
            m1 = part == 0 ? 0u : 0xffff0000u;
            m2 = part == 0 ? 0xffff0000u : 0u;
        } else {
            m1 = part == 0 ? 0u : 0xffff0000u;
            m2 = part < 2 ? 0u : 0xffff0000u;
        }
    }
    __device__ __forceinline__ static float masked(float x, uint32_t m) { return __uint_as_float(__float_as_uint(x) & m); }
    __device__ __forceinline__ float pick(float p, int which) const {
        if constexpr (DT == 0) {
            return masked(p, m1) - masked(p, m2);
        } else if constexpr (G == 8) {
            if (which == 0) return p - masked(p, m1);
            const float r = p - masked(p, 0xffff0000u);
            return masked(r - masked(r, 0xffff0000u), m2);
        } else {
            const float r = p - masked(p, m1);
            return r - masked(r, m2);
        }
    }
    __device__ __forceinline__ uint32_t operator()(float p0, float p1, int which) const {
        const float a = pick(p0, which), b = pick(p1, which);
        if constexpr (DT == 0) {
            const half2_t h = {(_Float16)a, (_Float16)b};
            return __builtin_bit_cast(uint32_t, h);
        } else {
            return upper_halves(a, b);
        }
    }
    __device__ __forceinline__ static uint32_t upper_halves(float a, float b) {
        return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
    }
};
// The lower (or upper) 16-bit halves of two words, packed.
template <bool UPPER>
__device__ __forceinline__ uint32_t pick_halves(uint32_t a, uint32_t b) {
    return __builtin_amdgcn_perm(b, a, UPPER ? 0x07060302u : 0x05040100u);
}

// The lane's sums, rows 4 rg .. 4 rg + 3 of channels 8 cl .. 8 cl + 7, to rows[head][channel]: the parts of a head are added.
template <int DT, int G>
__device__ __forceinline__ void store_parts(const f32x4_t (&acc)[8], float (*rows)[kHeadDim], int rg, int cl) {
    constexpr int kHeads = 4 / kRowsPerHead<G>;
#pragma unroll
    for (int k = 0; k < kHeads; ++k) {
        const int g = kHeads * rg + k;
        if (g < G) {
            f32x4_t *row = reinterpret_cast<f32x4_t *>(&rows[g][cl * 8]);
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                f32x4_t o;
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const f32x4_t &a = acc[4 * y + t];
                    if constexpr (G == 8) o[t] = a[2 * k] + a[2 * k + 1];
                    else if constexpr (DT == 0) o[t] = a[0] + a[1];
                    else o[t] = a[0] + (a[1] + a[2]);
                }
                row[y] = o;
            }
        }
    }
}

// Weights are taken against a reference that follows the running maximum of a head in leaps: a logit (log2 units) may exceed it
// by kSlack before it moves, so that most steps exchange nothing between the lanes and rescale nothing; a weight is 2^kSlack
// at most.  `limit` is ref + kSlack, -inf until the first logit above -inf (ref is 0 then).  All lanes of the wave
// together; bm is the maximum over the lane's own tokens.
constexpr float kSlack = 8.0f;
__device__ __forceinline__ void raise_reference(float bm, float &ref, float &limit, float &l, f32x4_t (&acc)[8], int rg) {
    bm = fmaxf(bm, __shfl_xor(bm, 16));
    bm = fmaxf(bm, __shfl_xor(bm, 32));
    const bool raise = bm > limit;
    const float alpha = raise ? (limit == -INFINITY ? 1.0f : exp2_fast(ref - bm)) : 1.0f;      // (nothing, or NaN, in the sums before)
    ref = raise ? bm : ref;
    limit = raise ? bm + kSlack : limit;
    l *= alpha;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        const float a = __shfl(alpha, 4 * rg + x);
#pragma unroll
        for (int t = 0; t < 8; ++t) acc[t][x] *= a;
    }
}

// 2^(m - M) for a running maximum m and the maximum M over several.  Where nothing has been seen (or nothing but NaN or
// -inf logits) m is -inf: the weight is 0, which keeps a NaN in the sums that it multiplies.
__device__ __forceinline__ float join_weight(float m, float M) { return m == -INFINITY ? 0.0f : exp2_fast(m - M); }

// One head's result from its joined numerator, denominator and maximum: 0 and -inf where no token was seen, NaN where a
// logit or a value was NaN.
__device__ __forceinline__ float joined_out(float n, float den) { return den == 0.0f ? 0.0f : n / den; }
__device__ __forceinline__ float joined_lse(float M, float den) { return den == 0.0f ? -INFINITY : (M + log2_fast(den)) * kLn2; }

// The four waves of a workgroup, joined through LDS: rows[wave][head][channel] and the waves' maxima and sums.  Either the
// request's results (one split) or the split's record.
template <int G>
struct WaveSums {
    float acc[4][G][kHeadDim];
    float m[4][G], l[4][G];
    int err[4];
};
template <int G>
__device__ __forceinline__ void join_waves(const WaveSums<G> &w, int tid, bool direct, float *out, float *lse, float *record) {
    if (!direct && tid == 0) record[2] = __int_as_float(w.err[0] | w.err[1] | w.err[2] | w.err[3]);
    for (int idx = tid; idx < G * kHeadDim; idx += 256) {
        const int g = idx / kHeadDim, ch = idx % kHeadDim;
        const float M = fmaxf(fmaxf(w.m[0][g], w.m[1][g]), fmaxf(w.m[2][g], w.m[3][g]));
        float den = 0.0f, num = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float f = join_weight(w.m[i][g], M);
            den += w.l[i][g] * f;
            num += w.acc[i][g][ch] * f;
        }
        if (direct) {
            out[g * kHeadDim + ch] = joined_out(num, den);
            if (lse && ch == 0) lse[g] = joined_lse(M, den);
        } else {
            float *r = record + g * kSplitStride;
            r[4 + ch] = num;
            if (ch == 0) { r[0] = M; r[1] = den; }
        }
    }
}

// The error word where no launch follows that could collect it: one workgroup looks at every length and every visible table
// entry of the call (`blocks` of a request at most) and stores the word, so that nobody has to clear it first.  It has
// read them before the others have read the pages, as long as there are few: beyond kCheckedEntries the word is cleared by
// a launch of its own, and whoever finds something sets it.
constexpr int kCheckedEntries = 8192;
__device__ __forceinline__ void check_tables(const KvView &kv, int window, int num_sinks, int blocks, int32_t *header, int *shared_err) {
    if (threadIdx.x == 0) *shared_err = 0;
    __syncthreads();
    int err = 0;
    const int total = kv.batch * max(blocks, 1);
#pragma unroll 8
    for (int x = threadIdx.x; x < total; x += 256) {
        const int r = x / max(blocks, 1), i = x % max(blocks, 1), ctx = ctx_clamped_quiet(kv, r);
        const Visible vis = make_visible(ctx, window, num_sinks);
        const int page = kv.block_table[(size_t)r * kv.max_blocks + (i < vis.count ? vis.block(i) : 0)];
        err |= (ctx != kv.ctx_lens[r] ? PSA_DEVERR_CTX_RANGE : 0) |
               (i < vis.count && (unsigned)page >= (unsigned)kv.num_pages ? PSA_DEVERR_PAGE_RANGE : 0);
    }
    if (err) atomicOr(shared_err, err);
    __syncthreads();
    if (threadIdx.x < 64) header[threadIdx.x] = threadIdx.x == 1 ? *shared_err : 0;
}

// How a call is cut: a request's visible blocks into nsplit splits at most, of `least` blocks at least.
struct SplitPlan {
    int window, num_sinks, nsplit, least, blocks;        // blocks: visible ones of a request at most
    bool checked;                                        // one split, and few enough table entries for check_tables
};
// Blocks of one split (but the last) of a request.
__device__ __forceinline__ int split_blocks(const SplitPlan &p, int count) { return max((count + p.nsplit - 1) / p.nsplit, p.least); }

// groups: workgroups that fill the GPU.
SplitPlan visible_plan(const psa_kv_desc *d, int window, int num_sinks, int groups, int least_blocks);
size_t visible_workspace_bytes(const psa_kv_desc *d, const SplitPlan &p);
hipError_t launch_clear(int32_t *header, hipStream_t st);
hipError_t launch_join(const KvView &kv, const SplitPlan &plan, const float *partial, float *out, float *lse, int32_t *header,
                       hipStream_t st);

}  // namespace psa
