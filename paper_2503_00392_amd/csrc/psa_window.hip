// Decode attention over the paged 16-bit cache with a sliding window and a few first tokens that stay visible (sinks):
// softmax(q k / sqrt d) v over the tokens t < sinks and t >= ctx - window, with one pass over them; and what it shares with the
// 4-bit cache's attention: how a call is cut, the list of pieces, the launch that joins the pieces of a request.
#include "psa_fold.h"
#include "psa_host.h"
#include "psa_visible.h"

namespace psa {

// grid: one workgroup of four waves per piece (or request) and KV head, before them the one that checks the tables (if any).
// A wave takes every fourth visible block and carries its own online softmax over them: logits with four 16x16x32 products,
// lane (kq, n) = (lane / 16, lane % 16) getting the logits of the head of row n for tokens kq, 4+kq, 8+kq, 12+kq; values with eight
// 16x16x16 products, the weights in parts in a head's rows; values in binary16 are split into two bfloat16 parts, exactly, that share
// one 16x16x32 product with the weights twice.  Tokens of a block that the query does not see get the logit -inf and a
// zero value row (the page may hold NaN there).
// Bound by memory: 4 requests of 64K tokens, 8 KV heads, G = 4, bfloat16: 171 us a call = 6.3 TB/s; 64 ragged requests with a window of
// 4096 and 16 sinks, G = 8, binary16: 153 us = 6.6, vector ALUs 32 % busy (14 % with weights in binary16 parts, in the same time);
// 240 ragged ones with a window of 130, 4 KV heads: 17 us = 3.8, of which 5 are the way to the first block and from the last.  Keys and values are both loaded a block ahead: with the values loaded when their block's turn came
// the second took 178 us at the best number of workgroups.  Two workgroups on a CU are enough and more get in each
// other's way: 155 us with 512 of them, 184 to 188 with 1024 to 2048 (limited to two on a CU by LDS: 175 to 184).
template <int DT, int G>
__global__ __launch_bounds__(256, 3) void window_kernel(KvView kv, const uint8_t *__restrict__ q, VisiblePlan plan,
                                                        VisibleWs ws, float *__restrict__ out, float *__restrict__ lse) {
    constexpr int kRows = kRowsPerHead<G>;
    __shared__ uint4 stage[4][16 * 17];                  // per wave: a key slice on its way into the operand's layout
    __shared__ __attribute__((aligned(16))) WaveSums<G> sums;
    const int tid = threadIdx.x, lane = tid & 63, rg = lane >> 4, cl = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);     // (so that what hangs on it is a scalar)
    int wg = blockIdx.x;
    if (plan.checked && wg-- == 0) {
        check_tables(kv, plan.window, plan.num_sinks, plan.blocks, ws.header);
        return;
    }
    const int h = wg % kv.num_kv_heads, u = wg / kv.num_kv_heads;       // all of request u, or piece u
    Piece piece{u, 0, 0, 0, -1, true};
    if (plan.direct) {
        piece.length = kv.ctx_lens[u];
    } else {
        piece = find_piece(kv, plan, (uint32_t)u, wg == 0, ws);
        if (piece.r >= kv.batch) return;
    }
    const int r = piece.r, ctx = clamp_ctx(kv, piece.length);
    int err = ctx != piece.length ? PSA_DEVERR_CTX_RANGE : 0;
    const Visible vis = make_visible(ctx, plan.window, plan.num_sinks);
    const int b0 = piece.b0, b1 = plan.direct ? vis.count : piece.b1;

    const int hd = cl / kRows, part = cl % kRows;
    const WeightParts<G> parts(part);
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
        uint2 a[kProducts<G>];
#pragma unroll
        for (int y = 0; y < kProducts<G>; ++y) a[y] = make_uint2(parts(p[0], p[1], y), parts(p[2], p[3], y));
        static_for<8>([&](auto t) __attribute__((always_inline)) {
            constexpr int w = t / 2;
            constexpr bool odd = t & 1;
            if constexpr (DT == 1) {
                const uint2 bv = make_uint2(pick_halves<odd>(pick_word(v.r[0], w), pick_word(v.r[1], w)),
                                            pick_halves<odd>(pick_word(v.r[2], w), pick_word(v.r[3], w)));
#pragma unroll
                for (int y = 0; y < kProducts<G>; ++y) acc[t] = mfma_16x16x16<1>(a[y], bv, acc[t]);
            } else {                                     // the weights with the values' upper parts, and again with the rest
                float x[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = odd ? cvt_hi<0>(pick_word(v.r[j], w)) : cvt_lo<0>(pick_word(v.r[j], w));
                using W = WeightParts<G>;
                const uint4 bv = make_uint4(W::upper_halves(x[0], x[1]), W::upper_halves(x[2], x[3]),
                                            W::upper_halves(W::rest(x[0]), W::rest(x[1])), W::upper_halves(W::rest(x[2]), W::rest(x[3])));
#pragma unroll
                for (int y = 0; y < kProducts<G>; ++y) acc[t] = mfma_16x16x32<1>(make_uint4(a[y].x, a[y].y, a[y].x, a[y].y), bv, acc[t]);
            }
        });
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    store_parts<G>(acc, sums.acc[wave], rg, cl);
    if (rg == 0 && hd < G && part == 0) { sums.m[wave][hd] = limit == -INFINITY ? -INFINITY : ref; sums.l[wave][hd] = l; }
    const bool bad_ctx = __ballot(err & PSA_DEVERR_CTX_RANGE) != 0ull, bad_page = __ballot(err & PSA_DEVERR_PAGE_RANGE) != 0ull;
    if (lane == 0) sums.err[wave] = (bad_ctx ? PSA_DEVERR_CTX_RANGE : 0) | (bad_page ? PSA_DEVERR_PAGE_RANGE : 0);
    // (where the header was cleared by a launch before; otherwise the checking workgroup or the joining launch sets the word)
    if ((plan.listed || (plan.direct && !plan.checked)) && sums.err[wave] && lane == 0) set_error(ws.header, sums.err[wave]);
    __syncthreads();
    const size_t row = (size_t)r * kv.num_q_heads + h * G;
    join_waves<G>(sums, tid, piece.whole, out + row * kHeadDim, lse ? lse + row : nullptr,
                  piece.record < 0 ? nullptr : ws.records + ((size_t)piece.record * kv.num_kv_heads + h) * G * kSplitStride);
}

// grid (batch * num_q_heads); LANES record lanes x 32 quarters of a row.  Lane j takes the request's records j, j + LANES, ... in
// ascending order, four rows under way; the lanes are added in a fixed order.  A request in one piece has its results already.
template <int LANES>
__global__ __launch_bounds__(32 * LANES) void join_kernel(KvView kv, VisiblePlan plan, VisibleWs ws, float *__restrict__ out,
                                                   float *__restrict__ lse) {
    constexpr int kWaves = LANES / 2;
    __shared__ float red[kWaves];
    __shared__ f32x4_t num_part[LANES][32];
    __shared__ float den_part[LANES];
    const int G = kv.num_q_heads / kv.num_kv_heads, s = blockIdx.x / G, g = blockIdx.x % G, r = s / kv.num_kv_heads, h = s % kv.num_kv_heads;
    const int tid = threadIdx.x, quarter = tid & 31, sl = tid >> 5;
    const int ctx = ctx_clamped_quiet(kv, r), count = make_visible(ctx, plan.window, plan.num_sinks).count;
    const uint32_t first = ws.first[r], n = pieces_of((uint32_t)count, (uint32_t)ws.header[2]);
    const float *src = ws.records + (((size_t)first * kv.num_kv_heads + h) * G + g) * kSplitStride;
    const size_t stride = (size_t)kv.num_kv_heads * G * kSplitStride;
    f32x4_t a[4];
    float m[4], l[4];
    auto load = [&](uint32_t i0) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float *row = src + (size_t)min(i0 + LANES * k, n - 1) * stride;
            a[k] = *reinterpret_cast<const f32x4_t *>(row + 4 + 4 * quarter);
            m[k] = row[0];
            l[k] = row[1];
        }
    };
    if (n > 1) load(sl);
    float M = -INFINITY;
    int err = ctx != kv.ctx_lens[r] ? PSA_DEVERR_CTX_RANGE : 0;
    if (n == 1 && plan.listed) return;                   // (there is no record, and the word is set)
    for (uint32_t i = tid; i < n; i += 32 * LANES) {
        M = fmaxf(M, src[i * stride]);
        if (g == 0) err |= __float_as_int(src[i * stride + 2]);
    }
    if (err) set_error(ws.header, err);
    if (n == 1) return;
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) M = fmaxf(M, __shfl_xor(M, d));
    if ((tid & 63) == 0) red[tid >> 6] = M;
    __syncthreads();
    M = red[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) M = fmaxf(M, red[w]);
    f32x4_t num = {0.0f, 0.0f, 0.0f, 0.0f};
    float den = 0.0f;
    for (uint32_t i0 = sl; i0 < n; i0 += 4 * LANES) {
        if (i0 != sl) load(i0);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (i0 + LANES * k < n) {
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
        float nn[LANES], d[LANES];
#pragma unroll
        for (int j = 0; j < LANES; ++j) {
            nn[j] = reinterpret_cast<const float *>(num_part[j])[tid];
            d[j] = den_part[j];
        }
#pragma unroll
        for (int w = LANES / 2; w >= 1; w >>= 1) {
#pragma unroll
            for (int j = 0; j < w; ++j) {
                nn[j] += nn[j + w];
                d[j] += d[j + w];
            }
        }
        const size_t row = (size_t)s * G + g;            // = r * num_q_heads + h * G + g
        out[row * kHeadDim + tid] = joined_out(nn[0], d[0]);
        if (lse && tid == 0) lse[row] = joined_lse(M, d[0]);
    }
}

__global__ void clear_error_word_kernel(int32_t *header) { header[threadIdx.x] = 0; }

// The list of pieces of more than kFoundRequests requests, by one workgroup: the sum of the visible blocks, then, 1024 requests at a
// time, how many pieces come before each.
__global__ __launch_bounds__(1024) void list_kernel(KvView kv, VisiblePlan plan, VisibleWs ws) {
    __shared__ uint32_t part[2][16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    uint32_t sum = 0;
    for (int r = tid; r < kv.batch; r += 1024) sum += (uint32_t)visible_count(kv, plan, r);
    sum = wave_prefix_sum(sum);
    if (lane == 63) part[0][wave] = sum;
    __syncthreads();
    uint32_t total = 0, pieces = 0, records = 0;         // the latter two: before the requests at hand
    for (int w = 0; w < 16; ++w) total += part[0][w];
    const uint32_t length = piece_length(kv, plan, total);
    for (int r0 = 0; r0 < kv.batch; r0 += 1024) {
        const int r = r0 + tid;
        const uint32_t count = r < kv.batch ? (uint32_t)visible_count(kv, plan, r) : 0u;
        const uint32_t n = pieces_of(count, length), several = n > 1 ? n : 0u;
        const uint32_t upto = wave_prefix_sum(n), upto_several = wave_prefix_sum(several);
        __syncthreads();                                 // (what the step before left has been read)
        if (lane == 63) { part[0][wave] = upto; part[1][wave] = upto_several; }
        __syncthreads();
        uint32_t at = pieces + upto - n, record = records + upto_several - several;
        for (int w = 0; w < 16; ++w) {
            if (w < wave) { at += part[0][w]; record += part[1][w]; }
            pieces += part[0][w];
            records += part[1][w];
        }
        if (r < kv.batch) ws.first[r] = record;
        if (n) {
            const uint32_t per = (count + n - 1) / n;
            for (uint32_t i = 0; i < n; ++i)
                ws.list[at + i] = make_int4(r, (int)(i * per), (int)min(count, (i + 1) * per), n > 1 ? (int)(record + i) : -1);
        }
    }
    if (tid < 64) ws.header[tid] = tid == 2 ? (int32_t)length : (tid == 3 ? (int32_t)pieces : 0);
}

// ---- host side ----------------------------------------------------------------------------------
VisiblePlan visible_plan(const psa_kv_desc *d, int window, int num_sinks, int groups, int least, int direct_from) {
    const long long H = d->num_kv_heads, S = d->batch * H;
    // a window of w tokens lies in at most (w + 14) / 16 + 1 blocks
    const long long tail = window > 0 ? ((long long)window + 14) / kPage + 1 : 0, head = ((long long)num_sinks + kPage - 1) / kPage;
    const long long blocks = head + tail < d->max_blocks_per_seq ? head + tail : d->max_blocks_per_seq, all = d->batch * blocks;
    VisiblePlan p{window, num_sinks, (int)blocks, 1, least, false, false, false};
    p.direct = blocks <= least || blocks <= (S >= direct_from ? kDirectBlocks : S / 2) || all > INT32_MAX || d->batch > kListedRequests;
    p.checked = p.direct && (all <= kCheckedEntries || (H >= 4 && all <= INT32_MAX));
    if (!p.direct) {
        const long long most = (all + least - 1) / least, want = (groups + H - 1) / H;
        p.groups = (int)(want < most ? want : (most > 0 ? most : 1));
        p.listed = d->batch > kFoundRequests;
    }
    return p;
}

static size_t first_bytes(const psa_kv_desc *d) { return ((size_t)d->batch * 4 + 255) / 256 * 256; }
static size_t list_bytes(const psa_kv_desc *d, const VisiblePlan &p) {
    return p.listed ? ((size_t)(p.groups + d->batch) * sizeof(int4) + 255) / 256 * 256 : 0;
}

size_t visible_workspace_bytes(const psa_kv_desc *d, const VisiblePlan &p) {
    if (p.direct) return 256;
    // A request in n > 1 pieces of length L has more than 5/4 L blocks, and n < blocks / L + 1 < 9/5 blocks / L: listed, all those
    // together have fewer than twice as many records as there are groups.
    const size_t records = p.listed ? 2 * (size_t)p.groups : (size_t)d->batch + p.groups;
    return 256 + first_bytes(d) + list_bytes(d, p) + records * d->num_q_heads * kSplitStride * sizeof(float);
}

VisibleWs visible_ws(const psa_kv_desc *d, const VisiblePlan &p, void *ws) {
    uint8_t *base = static_cast<uint8_t *>(ws), *list = base + 256 + first_bytes(d);
    return {reinterpret_cast<int32_t *>(base), reinterpret_cast<uint32_t *>(base + 256), reinterpret_cast<int4 *>(list),
            reinterpret_cast<float *>(list + list_bytes(d, p))};
}

hipError_t launch_clear(int32_t *header, hipStream_t st) {
    clear_error_word_kernel<<<1, 64, 0, st>>>(header);
    return hipGetLastError();
}

hipError_t launch_list(const KvView &kv, const VisiblePlan &plan, const VisibleWs &ws, hipStream_t st) {
    list_kernel<<<1, 1024, 0, st>>>(kv, plan, ws);
    return hipGetLastError();
}

hipError_t launch_join(const KvView &kv, const VisiblePlan &plan, const VisibleWs &ws, float *out, float *lse, hipStream_t st) {
    // many requests have few pieces each: smaller workgroups, of which more are resident
    const int rows = kv.batch * kv.num_q_heads;
    if (rows >= 1024) join_kernel<4><<<rows, 128, 0, st>>>(kv, plan, ws, out, lse);
    else join_kernel<16><<<rows, 512, 0, st>>>(kv, plan, ws, out, lse);
    return hipGetLastError();
}

// 512 workgroups: see the kernel.  One launch up to 320 blocks (windows of 5K) from 256 (request, KV head) pairs on: ragged and equal
// batches of 32 to 128 requests and 8 KV heads with windows of 4000 tokens took 79 to 365 us that way, 90 to 381 in pieces; with
// windows of 8000 it is 122 against 113 and 168 against 189.  16 requests: of 1024 tokens 16.3 against 18.0, of 2048 29.4 against 28.0, of
// 4096 61 against 49; 8 requests: of 600 10.5 against 11.0, of 1024 15.0 against 13.0.
constexpr int kWindowGroups = 512, kWindowLeastBlocks = 4, kWindowDirectFrom = 256;
static VisiblePlan window_plan(const psa_kv_desc *d, int window, int num_sinks) {
    return visible_plan(d, window, num_sinks, kWindowGroups, kWindowLeastBlocks, kWindowDirectFrom);
}

size_t window_workspace_bytes(const psa_kv_desc *d, int window, int num_sinks) {
    return visible_workspace_bytes(d, window_plan(d, window, num_sinks));
}

template <int DT, int G>
static hipError_t launch_window_t(const KvView &kv, const void *q, const VisiblePlan &plan, const VisibleWs &ws, float *out, float *lse,
                                  hipStream_t st) {
    const unsigned grid = (unsigned)(kv.num_kv_heads * (plan.direct ? kv.batch : plan.groups + kv.batch) + plan.checked);
    if (plan.direct && !plan.checked && launch_clear(ws.header, st) != hipSuccess) return hipErrorLaunchFailure;
    if (plan.listed && launch_list(kv, plan, ws, st) != hipSuccess) return hipErrorLaunchFailure;
    window_kernel<DT, G><<<grid, 256, 0, st>>>(kv, (const uint8_t *)q, plan, ws, out, lse);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess && !plan.direct ? launch_join(kv, plan, ws, out, lse, st) : e;
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
    const VisiblePlan plan = window_plan(d, window, num_sinks);
    const VisibleWs vws = visible_ws(d, plan, ws);
#define PSA_CASE(DT, GG) \
    if (d->dtype == DT && G == GG) return launch_window_t<DT, GG>(kv, q, plan, vws, out, lse, st);
    PSA_CASE(0, 1) PSA_CASE(0, 2) PSA_CASE(0, 4) PSA_CASE(0, 8)
    PSA_CASE(1, 1) PSA_CASE(1, 2) PSA_CASE(1, 4) PSA_CASE(1, 8)
#undef PSA_CASE
    return hipErrorInvalidValue;
}

}  // namespace psa
