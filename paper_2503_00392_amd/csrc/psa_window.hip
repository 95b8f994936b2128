// Decode attention over the paged 16-bit cache with a sliding window and a few first tokens that stay visible (sinks):
// softmax(q k / sqrt d) v over the tokens t < sinks and t >= ctx - window, with one pass over them, and the launch that
// joins the splits of a request (also those of the 4-bit cache).
#include "psa_fold.h"
#include "psa_host.h"
#include "psa_visible.h"

namespace psa {

// grid: one workgroup of four waves per split and (request, KV head); with one split a first workgroup more, which writes
// the error word.  A wave takes every fourth of the split's visible blocks and carries its own online softmax over them, as
// the dense control does (see there): logits with four 16x16x32 products, lane (kq, n) = (lane / 16, lane % 16) getting the
// logits of the head of row n for tokens kq, 4+kq, 8+kq, 12+kq; values with eight 16x16x16 products, the weights in parts in
// a head's rows.  Tokens of a block that the query does not see get the logit -inf and a zero value row (the page may hold NaN there).
template <int DT, int G>
__global__ __launch_bounds__(256, 3) void window_kernel(KvView kv, const uint8_t *__restrict__ q, int window, int num_sinks,
                                                        int nsplit, float *__restrict__ partial, float *__restrict__ out,
                                                        float *__restrict__ lse, int32_t *header) {
    constexpr int kRows = kRowsPerHead<G>;
    __shared__ uint4 stage[4][16 * 17];                  // per wave: a key slice on its way into the operand's layout
    __shared__ __attribute__((aligned(16))) WaveSums<G> sums;
    const int tid = threadIdx.x, lane = tid & 63, rg = lane >> 4, cl = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);     // (so that what hangs on it is a scalar)
    int wg = blockIdx.x;
    if (nsplit == 1 && wg-- == 0) {
        check_tables(kv, window, num_sinks, header, &sums.err[0]);
        return;
    }
    const int s = wg / nsplit, split = wg % nsplit, r = s / kv.num_kv_heads, h = s % kv.num_kv_heads;
    if (nsplit > 1 && wg == 0 && tid < 64) header[tid] = 0;      // the launch that joins the splits sets the error word
    const int raw_ctx = kv.ctx_lens[r], ctx = ctx_clamped_quiet(kv, r);
    int err = raw_ctx != ctx ? PSA_DEVERR_CTX_RANGE : 0;
    const Visible vis = make_visible(ctx, window, num_sinks);
    const int per = (vis.count + nsplit - 1) / nsplit, b0 = split * per, b1 = min(vis.count, b0 + per);

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
    size_t off = 0;
    Slice k;
    if (b0 + wave < b1) {
        off = slice_of(b0 + wave, 0);
        k = load_slice(kv.k_pool + off, lane);
    }
    for (int b = b0 + wave, i = 0; b < b1; b += 4, ++i) {
        const Slice kc = k;
        Slice v = load_slice(kv.v_pool + off, lane);
        if (b + 4 < b1) {                                // (the next keys are under way while these are worked on)
            off = slice_of(b + 4, i + 1);
            k = load_slice(kv.k_pool + off, lane);
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
    __syncthreads();
    const size_t row = (size_t)r * kv.num_q_heads + h * G;
    join_waves<G>(sums, tid, nsplit == 1, out + row * kHeadDim, lse ? lse + row : nullptr,
                  partial + ((size_t)s * nsplit + split) * G * kSplitStride);
}

// grid (S * G); 512 threads = 4 split lanes x 128 channels.  Split lane j takes splits j, j + 4, ... in ascending order, four
// loads under way; the four are added in a fixed order.
__global__ __launch_bounds__(512) void join_kernel(const float *__restrict__ partial, int nsplit, int G, int num_kv_heads,
                                                   int num_q_heads, float *__restrict__ out, float *__restrict__ lse,
                                                   int32_t *header) {
    __shared__ float red[8];
    __shared__ float wgt[kMaxSplits];
    __shared__ float num_part[4][kHeadDim];
    __shared__ float den_part[4];
    const int s = blockIdx.x / G, g = blockIdx.x % G, tid = threadIdx.x, ch = tid & 127, sl = tid >> 7;
    const int r = s / num_kv_heads, h = s % num_kv_heads;
    const float *src = partial + ((size_t)s * nsplit * G + g) * kSplitStride;
    const size_t stride = (size_t)G * kSplitStride;
    float M = -INFINITY;
    int err = 0;
    for (int i = tid; i < nsplit; i += 512) {
        const float mi = src[i * stride];
        wgt[i] = mi;
        M = fmaxf(M, mi);
        if (g == 0) err |= __float_as_int(src[i * stride + 2]);
    }
    if (err) set_error(header, err);
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) M = fmaxf(M, __shfl_xor(M, d));
    if ((tid & 63) == 0) red[tid >> 6] = M;
    __syncthreads();
    M = fmaxf(fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])), fmaxf(fmaxf(red[4], red[5]), fmaxf(red[6], red[7])));
    for (int i = tid; i < nsplit; i += 512) wgt[i] = join_weight(wgt[i], M);
    __syncthreads();
    float num = 0.0f, den = 0.0f;
    for (int i0 = sl; i0 < nsplit; i0 += 16) {
        float a[4], l[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int i = min(i0 + 4 * k, nsplit - 1);
            a[k] = src[i * stride + 4 + ch];
            l[k] = src[i * stride + 1];
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (i0 + 4 * k < nsplit) {
                num = fmaf(a[k], wgt[i0 + 4 * k], num);
                den = fmaf(l[k], wgt[i0 + 4 * k], den);
            }
        }
    }
    num_part[sl][ch] = num;
    if (ch == 0) den_part[sl] = den;
    __syncthreads();
    if (tid < kHeadDim) {
        const float n = (num_part[0][tid] + num_part[1][tid]) + (num_part[2][tid] + num_part[3][tid]);
        const float d = (den_part[0] + den_part[1]) + (den_part[2] + den_part[3]);
        const size_t row = (size_t)r * num_q_heads + h * G + g;
        out[row * kHeadDim + tid] = joined_out(n, d);
        if (lse && tid == 0) lse[row] = joined_lse(M, d);
    }
}

// ---- host side ----------------------------------------------------------------------------------
SplitPlan visible_plan(const psa_kv_desc *d, int window, int num_sinks, int least_blocks) {
    const long long S = (long long)d->batch * d->num_kv_heads;
    // a window of w tokens lies in at most (w + 14) / 16 + 1 blocks
    const long long tail = window > 0 ? ((long long)window + 14) / kPage + 1 : 0, head = ((long long)num_sinks + kPage - 1) / kPage;
    SplitPlan p;
    p.blocks = (int)(head + tail < d->max_blocks_per_seq ? head + tail : d->max_blocks_per_seq);
    const long long want = S > 0 ? (2048 + S - 1) / S : 1, by_length = (p.blocks + least_blocks - 1) / least_blocks;
    p.nsplit = (int)(want < by_length ? want : by_length);
    if (p.nsplit > kMaxSplits) p.nsplit = kMaxSplits;
    if (p.nsplit < 1) p.nsplit = 1;
    return p;
}

size_t visible_workspace_bytes(const psa_kv_desc *d, const SplitPlan &p) {
    return 256 + (p.nsplit > 1 ? (size_t)d->batch * d->num_q_heads * p.nsplit * kSplitStride * sizeof(float) : 0);
}

hipError_t launch_join(const KvView &kv, int G, int nsplit, const float *partial, float *out, float *lse, int32_t *header,
                       hipStream_t st) {
    join_kernel<<<kv.batch * kv.num_q_heads, 512, 0, st>>>(partial, nsplit, G, kv.num_kv_heads, kv.num_q_heads, out, lse, header);
    return hipGetLastError();
}

constexpr int kWindowLeastBlocks = 8;

size_t window_workspace_bytes(const psa_kv_desc *d, int window, int num_sinks) {
    return visible_workspace_bytes(d, visible_plan(d, window, num_sinks, kWindowLeastBlocks));
}

template <int DT, int G>
static hipError_t launch_window_t(const KvView &kv, const void *q, int window, int num_sinks, int nsplit, float *out, float *lse,
                                  void *ws, hipStream_t st) {
    int32_t *header = reinterpret_cast<int32_t *>(ws);
    float *partial = reinterpret_cast<float *>(reinterpret_cast<uint8_t *>(ws) + 256);
    const unsigned grid = (unsigned)(kv.batch * kv.num_kv_heads * nsplit + (nsplit == 1));
    window_kernel<DT, G><<<grid, 256, 0, st>>>(kv, (const uint8_t *)q, window, num_sinks, nsplit, partial, out, lse, header);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && nsplit > 1) e = launch_join(kv, G, nsplit, partial, out, lse, header, st);
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
    const int G = d->num_q_heads / d->num_kv_heads, nsplit = visible_plan(d, window, num_sinks, kWindowLeastBlocks).nsplit;
#define PSA_CASE(DT, GG) \
    if (d->dtype == DT && G == GG) return launch_window_t<DT, GG>(kv, q, window, num_sinks, nsplit, out, lse, ws, st);
    PSA_CASE(0, 1) PSA_CASE(0, 2) PSA_CASE(0, 4) PSA_CASE(0, 8)
    PSA_CASE(1, 1) PSA_CASE(1, 2) PSA_CASE(1, 4) PSA_CASE(1, 8)
#undef PSA_CASE
    return hipErrorInvalidValue;
}

}  // namespace psa
