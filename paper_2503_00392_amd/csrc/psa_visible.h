// What the two attention kernels with a window share (psa_window.hip over the 16-bit cache, psa_packed.hip over the 4-bit
// one): which tokens a query sees, the weights of the value product in parts, and how the work is cut and how
// running sums come together.
#pragma once

#include "psa_attend.h"

namespace psa {

constexpr int kSplitStride = 132;     // floats of one record for one head: M, l, error bits (head 0), pad, acc[128]

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

// The weights of the value product, p in [0, 2^kSlack], are given to the matrix cores in three bfloat16 parts (all 24 bits: each is
// what truncation leaves of the rest) in neighbouring rows of one operand.  bfloat16 whatever the cache's type, because a weight
// far below the reference counts as much as its value makes it: where a first token holds nearly everything and its value is near
// zero, the output is made of weights of 2^-20 and less, of which binary16 would lose the lower bits, and below 2^-25 all of them
// (65536 tokens 25.5 octaves below the first lost a quarter of the output).  Two bfloat16 parts leave an error of about 1e-6 of the output;
// three cost nothing where a head has four rows, and a second product of the same values where it has two (eight heads).
template <int G>
constexpr int kRowsPerHead = G == 8 ? 2 : 4;
template <int G>
constexpr int kProducts = G == 8 ? 2 : 1;

// The part of two weights that the lane's row gets in product `which`, packed.  What to take off is a mask per lane, so that
// nothing branches: the parts are p, p less its upper 16 bits, and that less its own upper 16 bits, each cut to 16 bits
// (a row beyond the parts gets the last part again, and store_parts leaves it out).
template <int G>
struct WeightParts {
    uint32_t m1, m2;
    __device__ __forceinline__ explicit WeightParts(int part) {
        m1 = part == 0 ? 0u : 0xffff0000u;
        if constexpr (G == 8) m2 = part == 0 ? 0xffff0000u : 0u;
        else m2 = part < 2 ? 0u : 0xffff0000u;
    }
    __device__ __forceinline__ static float masked(float x, uint32_t m) { return __uint_as_float(__float_as_uint(x) & m); }
    __device__ __forceinline__ float pick(float p, int which) const {
        if constexpr (G == 8) {
            if (which == 0) return p - masked(p, m1);
            const float r = p - masked(p, 0xffff0000u);
            return masked(r - masked(r, 0xffff0000u), m2);
        } else {
            const float r = p - masked(p, m1);
            return r - masked(r, m2);
        }
    }
    __device__ __forceinline__ uint32_t operator()(float p0, float p1, int which) const { return upper_halves(pick(p0, which), pick(p1, which)); }
    __device__ __forceinline__ static uint32_t upper_halves(float a, float b) {
        return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
    }
    // what its upper 16 bits leave of a number
    __device__ __forceinline__ static float rest(float x) { return x - masked(x, 0xffff0000u); }
};
// The lower (or upper) 16-bit halves of two words, packed.
template <bool UPPER>
__device__ __forceinline__ uint32_t pick_halves(uint32_t a, uint32_t b) {
    return __builtin_amdgcn_perm(b, a, UPPER ? 0x07060302u : 0x05040100u);
}

// The lane's sums, rows 4 rg .. 4 rg + 3 of channels 8 cl .. 8 cl + 7, to rows[head][channel]: the parts of a head are added.
template <int G>
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
// request's results (`whole`) or a record; a record's error bits in any case.
template <int G>
struct WaveSums {
    float acc[4][G][kHeadDim];
    float m[4][G], l[4][G];
    int err[4];
};
template <int G>
__device__ __forceinline__ void join_waves(const WaveSums<G> &w, int tid, bool whole, float *out, float *lse, float *record) {
    if (record && tid == 0) record[2] = __int_as_float(w.err[0] | w.err[1] | w.err[2] | w.err[3]);
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
        if (whole) {
            out[g * kHeadDim + ch] = joined_out(num, den);
            if (lse && ch == 0) lse[g] = joined_lse(M, den);
        } else {
            float *r = record + g * kSplitStride;
            r[4 + ch] = num;
            if (ch == 0) { r[0] = M; r[1] = den; }
        }
    }
}

__device__ __forceinline__ int clamp_ctx(const KvView &kv, int ctx) { return min(max(ctx, 0), kv.max_blocks * kPage); }

// The error word where no launch follows that could collect it: one workgroup looks at every length and every visible table
// entry of the call (`blocks` of a request at most) and stores the word, so that nobody has to clear it first.  The lengths of 256
// requests at a time go to LDS, then sixteen entries a thread are under way at once: about 0.75 ns an entry (3.9 when each
// entry waited for its request's length).  The others read the entry's page for every KV head, 0.36 ns over 4 bits, so
// for full requests this is hidden with four KV heads or more, and for kCheckedEntries in any case; else a launch of its own
// clears the word, and whoever finds something sets it.  A thread steps through all places that the table's width and the window
// allow, so requests far shorter than these wait for it: 256 of 64 tokens with windows of 4000 and 8 KV heads take 31 us over 16
// bits and 30 over 4 (in pieces, which need no such workgroup, 26 and 24); of 500 tokens 102 and 37 (110 and 43).
constexpr int kCheckedEntries = 4096;
__device__ __forceinline__ void check_tables(const KvView &kv, int window, int num_sinks, int blocks, int32_t *header) {
    __shared__ int lengths[256];
    const int tid = threadIdx.x, W = max(blocks, 1), step_r = 256 / W, step_i = 256 % W;
    int err = 0;
    for (int r0 = 0; r0 < kv.batch; r0 += 256) {
        const int here = min(256, kv.batch - r0);
        __syncthreads();
        if (tid < here) {
            const int given = kv.ctx_lens[r0 + tid], ctx = clamp_ctx(kv, given);
            if (ctx != given) err |= PSA_DEVERR_CTX_RANGE;
            lengths[tid] = ctx;
        }
        __syncthreads();
        int r = tid / W, i = tid % W;                    // entry i of request r0 + r
        while (r < here) {
            int page[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                const Visible vis = make_visible(lengths[min(r, here - 1)], window, num_sinks);
                const bool seen = r < here && i < vis.count;
                page[k] = seen ? kv.block_table[(size_t)(r0 + r) * kv.max_blocks + vis.block(i)] : 0;
                r += step_r;
                i += step_i;
                if (i >= W) { i -= W; ++r; }
            }
#pragma unroll
            for (int k = 0; k < 16; ++k)
                if ((unsigned)page[k] >= (unsigned)kv.num_pages) err |= PSA_DEVERR_PAGE_RANGE;
        }
    }
    __syncthreads();
    if (tid == 0) lengths[0] = 0;
    __syncthreads();
    if (err) atomicOr(&lengths[0], err);
    __syncthreads();
    if (tid < 64) header[tid] = tid == 1 ? lengths[0] : 0;
}

// How a call is cut.
//   direct   a workgroup for every (request, KV head), which writes the results: where none has more than kDirectBlocks to read
//            and there are direct_from of them, or, as the second launch costs 3 to 4 us, where they are fewer and have little to read.
//   planned  workgroups take pieces of requests: a piece is what the visible blocks of all requests come to, divided by the
//            workgroups that fill the GPU, and a request gets as many as it takes -- one long request among short ones is
//            shared by many (direct, it is one workgroup's: the host knows what the widths allow, not the lengths).  A
//            piece's result is a record, unless it is all of its request, and a second launch joins the records of a request.  Up to kFoundRequests requests every workgroup finds its piece from the lengths by
//            itself (less than a microsecond), and the first one leaves the requests' first records for the launch that joins; for
//            more requests a launch before lists the pieces.
// Few pieces, because what a workgroup does before its first block and after its last (dependent trips to memory, the
// exchange between its waves) costs 5 us and more: the same bytes in pieces of half the size and two rounds of
// workgroups took 18 % longer.  So a request keeps one piece (or two, ...) up to a quarter more than these hold.  (Trying six lengths
// and taking the one whose rounds would end first cost every workgroup 1.5 us and gained no more than that.)  One request of
// 64K tokens among 63 of 1000: 93 us over 16 bits, 40 over 4; with the same number of pieces for every request 772 and 192.
// Direct calls keep that price up to kDirectBlocks: one request of 5000 tokens among 31 of 100, 8 KV heads, 60 us over 16 bits and 31
// over 4 (in pieces 15 and 10), among 127 67 and 33 (27 and 19); they win where the lengths are alike or evenly spread: 64 requests
// of up to 4000 tokens 117 and 37.8 (129 and 38.5), 256 of 4000 663 and 196 (682 and 200).
struct VisiblePlan {
    int window, num_sinks;
    int blocks;                    // visible blocks of a request at most
    int groups, least;             // planned: workgroups for a KV head that fill the GPU; blocks of a piece at least
    bool direct, checked, listed;  // checked: direct, and few enough table entries for check_tables; listed: planned, with a list
};
VisiblePlan visible_plan(const psa_kv_desc *d, int window, int num_sinks, int groups, int least, int direct_from);
size_t visible_workspace_bytes(const psa_kv_desc *d, const VisiblePlan &p);

constexpr int kDirectBlocks = 320;
constexpr int kFoundRequests = 64, kListedRequests = 65536;      // (beyond: direct)
// The workspace: header (word 1: error bits, word 2: length of a piece, word 3: pieces in the list), the requests' first records,
// the list (request, first and last block, record or -1 where the piece is all of the request), the records.
struct VisibleWs {
    int32_t *header;
    uint32_t *first;               // [batch]
    int4 *list;                    // [groups + batch] if listed
    float *records;                // [groups + batch][num_kv_heads][G][kSplitStride]; listed: [2 groups]..., for requests in several pieces
};
VisibleWs visible_ws(const psa_kv_desc *d, const VisiblePlan &p, void *ws);
hipError_t launch_clear(int32_t *header, hipStream_t st);
hipError_t launch_list(const KvView &kv, const VisiblePlan &plan, const VisibleWs &ws, hipStream_t st);
hipError_t launch_join(const KvView &kv, const VisiblePlan &plan, const VisibleWs &ws, float *out, float *lse, hipStream_t st);

__device__ __forceinline__ int visible_count(const KvView &kv, const VisiblePlan &plan, int r) {
    return make_visible(ctx_clamped_quiet(kv, r), plan.window, plan.num_sinks).count;
}

// Pieces of a request of `count` visible blocks.
__device__ __forceinline__ uint32_t pieces_of(uint32_t count, uint32_t length) {
    const uint32_t over = length / 4;
    return count == 0 ? 0u : (count <= over ? 1u : (count - over + length - 1) / length);
}

struct Piece {
    int r, b0, b1;                 // r = batch: there is no such piece
    int length;                    // the request's, as given
    int record;                    // -1: none
    bool whole;                    // all of its request
};
// Length of a piece; the last one of a request is a quarter of a piece too short in the mean: that much is left for it.
__device__ __forceinline__ uint32_t piece_length(const KvView &kv, const VisiblePlan &plan, uint32_t total) {
    const uint32_t share = (uint32_t)max(plan.groups - kv.batch / 4, (plan.groups + 1) / 2);
    return max((total + share - 1) / share, (uint32_t)plan.least);
}
// Piece u; `leave`: this workgroup leaves the requests' first records and the length of a piece.
__device__ __forceinline__ Piece find_piece(const KvView &kv, const VisiblePlan &plan, uint32_t u, bool leave, const VisibleWs &ws) {
    if (plan.listed) {
        const int4 e = ws.list[u];
        if (u >= (uint32_t)ws.header[3]) return {kv.batch, 0, 0, 0, -1, false};
        return {e.x, e.y, e.z, kv.ctx_lens[e.x], e.w, e.w < 0};
    }
    const int lane = threadIdx.x & 63;                   // every wave by itself, a lane for each request
    const int given = lane < kv.batch ? kv.ctx_lens[lane] : 0;
    const uint32_t count = (uint32_t)make_visible(clamp_ctx(kv, given), plan.window, plan.num_sinks).count;
    const uint32_t length = piece_length(kv, plan, (uint32_t)__builtin_amdgcn_readlane((int)wave_prefix_sum(count), 63));
    const uint32_t n = pieces_of(count, length), first = wave_prefix_sum(n) - n;
    if (leave && lane < kv.batch) ws.first[lane] = first;
    if (leave) ws.header[lane] = lane == 2 ? (int32_t)length : 0;
    const unsigned long long hit = __ballot(u >= first && u < first + n);
    if (!hit) return {kv.batch, 0, 0, 0, -1, false};
    const int r = __builtin_ctzll(hit);
    const uint32_t at = u - (uint32_t)__builtin_amdgcn_readlane((int)first, r), all = (uint32_t)__builtin_amdgcn_readlane((int)count, r),
                   of = (uint32_t)__builtin_amdgcn_readlane((int)n, r), per = (all + of - 1) / of;
    return {r, (int)(at * per), (int)min(all, (at + 1) * per), __builtin_amdgcn_readlane(given, r), (int)u, of == 1};
}

}  // namespace psa
