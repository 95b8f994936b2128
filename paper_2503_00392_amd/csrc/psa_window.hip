// Decode attention over the paged 16-bit cache with a sliding window and a few first tokens that stay visible (sinks):
// softmax(q k / sqrt d) v over the tokens t < sinks and t >= ctx - window, with one pass over them, and the launch that
// joins the splits of a request (also those of the 4-bit cache).
#include "psa_fold.h"
#include "psa_host.h"
#include "psa_visible.h"

namespace psa {

// grid: one workgroup of four waves per split and (request, KV head), before them the one that checks the tables (if any).  A wave takes every fourth of the split's visible blocks and carries its own online softmax over them, as
// the dense control does (see there): logits with four 16x16x32 products, lane (kq, n) = (lane / 16, lane % 16) getting the
// logits of the head of row n for tokens kq, 4+kq, 8+kq, 12+kq; values with eight 16x16x16 products, the weights in parts in
// a head's rows.  Tokens of a block that the query does not see get the logit -inf and a zero value row (the page may hold NaN there).
template <int DT, int G>
__global__ __launch_bounds__(256, 3) void window_kernel(KvView kv, const uint8_t *__restrict__ q, SplitPlan plan,
                                                        float *__restrict__ partial, float *__restrict__ out,
                                                        float *__restrict__ lse, int32_t *header) {
    constexpr int kRows = kRowsPerHead<G>;
    __shared__ uint4 stage[4][16 * 17];                  // per wave: a key slice on its way into the operand's layout
    __shared__ __attribute__((aligned(16))) WaveSums<G> sums;
    const int tid = threadIdx.x, lane = tid & 63, rg = lane >> 4, cl = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);     // (so that what hangs on it is a scalar)
    int wg = blockIdx.x;
    if (plan.checked && wg-- == 0) {
        check_tables(kv, plan.window, plan.num_sinks, plan.blocks, header, &sums.err[0]);
        return;
    }
    const int s = wg / plan.nsplit, split = wg % plan.nsplit, r = s / kv.num_kv_heads, h = s % kv.num_kv_heads;
    if (plan.nsplit > 1 && wg == 0 && tid < 64) header[tid] = 0;      // the launch that joins the splits sets the error word
    const int raw_ctx = kv.ctx_lens[r], ctx = ctx_clamped_quiet(kv, r);
    int err = raw_ctx != ctx ? PSA_DEVERR_CTX_RANGE : 0;
    const Visible vis = make_visible(ctx, plan.window, plan.num_sinks);
    const int per = split_blocks(plan, vis.count), b0 = split * per, b1 = min(vis.count, b0 + per);
    if (split > 0 && b0 >= vis.count) return;            // (the first split has a result even of no blocks)

    const int hd = cl / kRows, part = cl % kRows;
    const WeightParts<DT, G> parts(part);
    uint4 qb[4];                                         // B operand of the logits: a head's rows all hold its query
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
        qb[kk] = make_uint4(0, 0, 0, 0);
        if (hd < G) qb[kk] = ld16(q + ((size_t)(r * kv.num_q_heads + h * G + hd) * kHeadDim + (4 * kk + rg) * 8) * 2);
    }
    float ref = 0.0f, limit = -INFINITY, l = 0.0f;       // head hd: see raise_reference; exp-sum of this row group
    f32x4_t acc[8];
#pragma unroll
    for (int t = 0; t < 8; ++t) acc[t] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};

    const int32_t *table = kv.block_table + (size_t)r * kv.max_blocks;
    int pages = 0;                                       // lane j: page of the wave's block j of 64
    auto slice_of = [&](int b, int i) __attribute__((always_inline)) {      // where block b, the wave's i-th, lies in the pools
        if ((i & 63) == 0) {
            const int page = table[vis.block(min(b + 4 * lane, b1 - 1))];
            pages = clamp_page_quiet(page, kv.num_pages);
            if (pages != page) err |= PSA_DEVERR_PAGE_RANGE;
        }
        return ((size_t)__builtin_amdgcn_readlane(pages, i & 63) * kv.num_kv_heads + h) * kSliceBytes;
    };
    Slice nk, nv;
    if (b0 + wave < b1) {
        const size_t off = slice_of(b0 + wave, 0);
        nk = load_slice(kv.k_pool + off, lane);
        nv = load_slice(kv.v_pool + off, lane);
    }
    for (int b = b0 + wave, i = 0; b < b1; b += 4, ++i) {
        const Slice kc = nk;
        Slice v = nv;
        if (b + 4 < b1) {                                // the next block is under way while this one is worked on
            const size_t off = slice_of(b + 4, i + 1);
            nk = load_slice(kv.k_pool + off, lane);
            nv = load_slice(kv.v_pool + off, lane);
        }
        const f32x4_t d = block_logits<DT>(kc.r, qb, stage[wave], lane, kPage);
        float sc[4] = {d[0], d[1], d[2], d[3]};
        const int lb = vis.block(b);
        if (!vis.sees_all(lb)) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool seen = vis.sees(lb * kPage + 4 * j + rg);
                sc[j] = seen ? sc[j] : -INFINITY;
                v.r[j] = seen ? v.r[j] : make_uint4(0, 0, 0, 0);
            }
        }
        const float bm = fmaxf(fmaxf(sc[0], sc[1]), fmaxf(sc[2], sc[3]));
        if (__ballot(bm > limit)) raise_reference(bm, ref, limit, l, acc, rg);
        float p[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) p[j] = exp2_fast(sc[j] - ref);
        l += (p[0] + p[1]) + (p[2] + p[3]);
        uint2 a[kProducts<DT, G>];
#pragma unroll
        for (int y = 0; y < kProducts<DT, G>; ++y) a[y] = make_uint2(parts(p[0], p[1], y), parts(p[2], p[3], y));
        static_for<8>([&](auto t) __attribute__((always_inline)) {
            constexpr int w = t / 2;
            constexpr bool odd = t & 1;
            const uint2 bv = make_uint2(pick_halves<odd>(pick_word(v.r[0], w), pick_word(v.r[1], w)),
                                        pick_halves<odd>(pick_word(v.r[2], w), pick_word(v.r[3], w)));
#pragma unroll
            for (int y = 0; y < kProducts<DT, G>; ++y) acc[t] = mfma_16x16x16<DT>(a[y], bv, acc[t]);
        });
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    store_parts<DT, G>(acc, sums.acc[wave], rg, cl);
    if (rg == 0 && hd < G && part == 0) { sums.m[wave][hd] = limit == -INFINITY ? -INFINITY : ref; sums.l[wave][hd] = l; }
    const bool bad_ctx = __ballot(err & PSA_DEVERR_CTX_RANGE) != 0ull, bad_page = __ballot(err & PSA_DEVERR_PAGE_RANGE) != 0ull;
    if (lane == 0) sums.err[wave] = (bad_ctx ? PSA_DEVERR_CTX_RANGE : 0) | (bad_page ? PSA_DEVERR_PAGE_RANGE : 0);
    if (plan.nsplit == 1 && !plan.checked && sums.err[wave] && lane == 0) set_error(header, sums.err[wave]);
    __syncthreads();
    const size_t row = (size_t)r * kv.num_q_heads + h * G;
    join_waves<G>(sums, tid, plan.nsplit == 1, out + row * kHeadDim, lse ? lse + row : nullptr,
                  partial + ((size_t)s * plan.nsplit + split) * G * kSplitStride);
}

// grid (S * G); 512 threads = 16 split lanes x 32 quarters of a row.  Split lane j takes splits j, j + 16, ... in ascending
// order, four rows under way -- the first four before the maximum over the splits is known, so that up to 64 splits cost one
// trip to memory and not two; the sixteen are added in a fixed order.
__global__ __launch_bounds__(512) void join_kernel(KvView kv, SplitPlan plan, const float *__restrict__ partial,
                                                   float *__restrict__ out, float *__restrict__ lse, int32_t *header) {
    __shared__ float red[8];
    __shared__ f32x4_t num_part[16][32];
    __shared__ float den_part[16];
    const int G = kv.num_q_heads / kv.num_kv_heads, s = blockIdx.x / G, g = blockIdx.x % G, r = s / kv.num_kv_heads;
    const int tid = threadIdx.x, quarter = tid & 31, sl = tid >> 5;
    const float *src = partial + ((size_t)s * plan.nsplit * G + g) * kSplitStride;
    const size_t stride = (size_t)G * kSplitStride;
    f32x4_t a[4];
    float m[4], l[4];
    auto load = [&](int i0) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float *row = src + (size_t)min(i0 + 16 * k, plan.nsplit - 1) * stride;
            a[k] = *reinterpret_cast<const f32x4_t *>(row + 4 + 4 * quarter);
            m[k] = row[0];
            l[k] = row[1];
        }
    };
    load(sl);                                            // (beyond the splits that have a result: not used)
    const float *mine = src + (size_t)min(tid, plan.nsplit - 1) * stride;
    float M = mine[0];
    int err = __float_as_int(mine[2]);
    const int count = make_visible(ctx_clamped_quiet(kv, r), plan.window, plan.num_sinks).count, per = split_blocks(plan, count);
    const int nsplit = max(1, (count + per - 1) / per);  // splits that have a result
    if (tid >= nsplit) {
        M = -INFINITY;
        err = 0;
    }
    for (int i = tid + 512; i < nsplit; i += 512) {
        M = fmaxf(M, src[i * stride]);
        err |= __float_as_int(src[i * stride + 2]);
    }
    if (g == 0 && err) set_error(header, err);
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) M = fmaxf(M, __shfl_xor(M, d));
    if ((tid & 63) == 0) red[tid >> 6] = M;
    __syncthreads();
    M = fmaxf(fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])), fmaxf(fmaxf(red[4], red[5]), fmaxf(red[6], red[7])));
    f32x4_t num = {0.0f, 0.0f, 0.0f, 0.0f};
    float den = 0.0f;
    for (int i0 = sl; i0 < nsplit; i0 += 64) {
        if (i0 != sl) load(i0);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (i0 + 16 * k < nsplit) {
                const float w = join_weight(m[k], M);
                num += a[k] * w;
                den = fmaf(l[k], w, den);
            }
        }
    }
    num_part[sl][quarter] = num;
    if (quarter == 0) den_part[sl] = den;
    __syncthreads();
    if (tid < kHeadDim) {
        float n[16], d[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            n[j] = reinterpret_cast<const float *>(num_part[j])[tid];
            d[j] = den_part[j];
        }
#pragma unroll
        for (int w = 8; w >= 1; w >>= 1) {
#pragma unroll
            for (int j = 0; j < w; ++j) {
                n[j] += n[j + w];
                d[j] += d[j + w];
            }
        }
        const size_t row = (size_t)s * G + g;            // = r * num_q_heads + h * G + g
        out[row * kHeadDim + tid] = joined_out(n[0], d[0]);
        if (lse && tid == 0) lse[row] = joined_lse(M, d[0]);
    }
}

__global__ void clear_error_word_kernel(int32_t *header) { header[threadIdx.x] = 0; }

// ---- host side ----------------------------------------------------------------------------------
SplitPlan visible_plan(const psa_kv_desc *d, int window, int num_sinks, int groups, int least_blocks) {
    const long long S = (long long)d->batch * d->num_kv_heads;
    // a window of w tokens lies in at most (w + 14) / 16 + 1 blocks
    const long long tail = window > 0 ? ((long long)window + 14) / kPage + 1 : 0, head = ((long long)num_sinks + kPage - 1) / kPage;
    const long long blocks = head + tail < d->max_blocks_per_seq ? head + tail : d->max_blocks_per_seq;
    const long long want = S > 0 ? (groups + S - 1) / S : 1, by_length = (blocks + least_blocks - 1) / least_blocks;
    SplitPlan p{window, num_sinks, 1, least_blocks, (int)blocks, false};
    p.nsplit = (int)(want < by_length ? want : by_length);
    if (p.nsplit > kMaxSplits) p.nsplit = kMaxSplits;
    if (p.nsplit < 1) p.nsplit = 1;
    p.checked = p.nsplit == 1 && d->batch * (blocks > 0 ? blocks : 1) <= kCheckedEntries;
    return p;
}

size_t visible_workspace_bytes(const psa_kv_desc *d, const SplitPlan &p) {
    return 256 + (p.nsplit > 1 ? (size_t)d->batch * d->num_q_heads * p.nsplit * kSplitStride * sizeof(float) : 0);
}

hipError_t launch_clear(int32_t *header, hipStream_t st) {
    clear_error_word_kernel<<<1, 64, 0, st>>>(header);
    return hipGetLastError();
}

hipError_t launch_join(const KvView &kv, const SplitPlan &plan, const float *partial, float *out, float *lse, int32_t *header,
                       hipStream_t st) {
    join_kernel<<<kv.batch * kv.num_q_heads, 512, 0, st>>>(kv, plan, partial, out, lse, header);
    return hipGetLastError();
}

constexpr int kWindowGroups = 512, kWindowLeastBlocks = 4;

size_t window_workspace_bytes(const psa_kv_desc *d, int window, int num_sinks) {
    return visible_workspace_bytes(d, visible_plan(d, window, num_sinks, kWindowGroups, kWindowLeastBlocks));
}

template <int DT, int G>
static hipError_t launch_window_t(const KvView &kv, const void *q, const SplitPlan &plan, float *out, float *lse, void *ws,
                                  hipStream_t st) {
    int32_t *header = reinterpret_cast<int32_t *>(ws);
    float *partial = reinterpret_cast<float *>(reinterpret_cast<uint8_t *>(ws) + 256);
    const unsigned grid = (unsigned)(kv.batch * kv.num_kv_heads * plan.nsplit + plan.checked);
    if (plan.nsplit == 1 && !plan.checked && launch_clear(header, st) != hipSuccess) return hipErrorLaunchFailure;
    window_kernel<DT, G><<<grid, 256, 0, st>>>(kv, (const uint8_t *)q, plan, partial, out, lse, header);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && plan.nsplit > 1) e = launch_join(kv, plan, partial, out, lse, header, st);
    return e;
}

hipError_t launch_window(const psa_kv_desc *d, const void *q, int window, int num_sinks, float *out, float *lse, void *ws,
                         hipStream_t st) {
    const KvView kv = make_view(d);
    if (kv.num_pages == 0) {
        DecodeArgs a{};
        a.out = out;
        a.lse_out = lse;
        return launch_no_pages(kv, a, reinterpret_cast<int32_t *>(ws), st);
    }
    const int G = d->num_q_heads / d->num_kv_heads;
    const SplitPlan plan = visible_plan(d, window, num_sinks, kWindowGroups, kWindowLeastBlocks);
#define PSA_CASE(DT, GG) \
    if (d->dtype == DT && G == GG) return launch_window_t<DT, GG>(kv, q, plan, out, lse, ws, st);
    PSA_CASE(0, 1) PSA_CASE(0, 2) PSA_CASE(0, 4) PSA_CASE(0, 8)
    PSA_CASE(1, 1) PSA_CASE(1, 2) PSA_CASE(1, 4) PSA_CASE(1, 8)
#undef PSA_CASE
    return hipErrorInvalidValue;
}

}  // namespace psa
